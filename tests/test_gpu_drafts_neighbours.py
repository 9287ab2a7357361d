"""Attention over the paged 16-bit cache (not in the paper): NaN and infinities in the queries that fill up an item's rows, of the next
sequence, of nobody or of another node, do not reach a row whose scores pass the maximum in use by far.  Oracle and bounds:
tests/test_gpu_drafts.py."""
import numpy as np
import pytest

from tests.test_gpu_drafts import starts_of
from tests.test_gpu_drafts_nan import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("first", ["low", "-inf"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,few,many", [(1, 2, 9), (2, 1, 8), (4, 2, 8), (1, 3, 30), (4, 3, 16), (1, 20, 64)])
def test_a_neighbours_query_does_not_reach_a_leading_score(G, few, many, D, first):
    """The first sequence has few nodes, so the rows of its items are filled up with the next one's, which hold NaN (or infinities); a key of its
    second and third tile leads all in front of it by 2^8 and more: sums taken so far must go, or they overflow."""
    starts = starts_of([few, many, few])

    def plant(q, pool, place):
        q[:] = 1.0
        q[starts[1]:starts[2]:2] = np.nan
        q[starts[1] + 1:starts[2]:2] = np.inf
        q[starts[3]:] = np.nan                                         # behind the last sequence, too
        pool[:, 0] = 0.0
        for b in (0, 2):
            for t in range(128):
                p, r = place(b, t)
                pool[p, 0, :, r] = -np.inf if first == "-inf" else -1.0
            for t, size in ((150, 4.0), (300, 8.0)):
                p, r = place(b, t)
                pool[p, 0, :, r] = size
    # scores -D, 0, 4 D and 8 D: leads of 256 and 512 at the least; fp32 holds them exactly, so the bounds stay
    lost = check((G * 2, 2, D, 64, [400, 20, 350], [few, many, few], 1), False, plant, scale=1.0)
    assert lost == many * G * 2


@pytest.mark.parametrize("G,n", [(1, 6), (2, 8), (4, 16), (1, 60)])
def test_a_nodes_query_does_not_reach_the_others_leading_scores(G, n):
    """The same within a tree: one head of one node is NaN."""
    def plant(q, pool, place):
        q[:] = 1.0
        q[n - 1, 0, 7] = np.nan
        pool[:, 0] = 0.0
        for t, size in ((150, 4.0), (300, 8.0)):
            p, r = place(0, t)
            pool[p, 0, :, r] = size
    assert check((G * 2, 2, 128, 64, [400], [n], 1), False, plant, scale=1.0) == 1
