"""Attention over the paged 16-bit cache (not in the paper) with NaN and infinities that somebody sees: they reach the rows that see them,
as in the definition, and no others, however the rows are laid out and the work is cut.  Oracle and bounds: tests/test_gpu_drafts.py."""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from paper_2412_00876_b200 import workloads as wl
from tests.test_gpu_drafts import DEV, HALF, bf, books, cache_rows, context, i32, random_tree, starts_of, up

pytestmark = pytest.mark.gpu
BAD = {"nan": np.nan, "inf": np.inf, "-inf": -np.inf}

# heads, K/V heads, dim, page, rows held, nodes, columns of the table beyond what is needed: up to 16, 32 and 64 rows an item, up to 128,
# and more; few short contexts are not cut, long ones go to many parts, a few sequences of middling length to two or three
SHAPES = {
    "16 rows, whole": (4, 2, 128, 64, [200, 0, 70], [1, 8, 3], 1), "16 rows, many parts": (8, 2, 64, 32, [3000, 900], [4, 2], 40),
    "32 rows, few parts": (8, 2, 128, 64, [500] * 30, [7] * 30, 40), "64 rows, whole": (4, 4, 64, 16, [300, 130], [60, 41], 1),
    "64 rows, many parts": (8, 1, 128, 128, [2500, 300], [8, 5], 40), "64 rows, few parts": (4, 4, 128, 64, [400] * 20, [40] * 20, 40),
    "128 rows, whole": (16, 2, 128, 64, [250, 40], [12, 16], 1), "128 rows, many parts": (16, 1, 64, 64, [3000], [7], 40),
    "128 rows, few parts": (8, 4, 128, 32, [600] * 20, [50] * 20, 60),
    "more rows, whole": (8, 2, 128, 64, [300, 20], [50, 70], 1), "more rows, many parts": (8, 1, 64, 64, [3000, 10], [33, 20], 40),
    "more rows, few parts": (8, 4, 128, 64, [500] * 10, [90] * 10, 60)}


def check(shape, masked, plant, touched=None, seed=0, scale=None):
    """plant(q, pool, place) puts values into the queries and the cache (of the sequences `touched`; None: of all): rows that are not finite
    in the oracle have to be NaN, all others within the bounds; other sequences have the bits that they have without those values.
    Returns the number of rows that are NaN."""
    H, Hk, D, page, held, nodes, cols = SHAPES[shape] if isinstance(shape, str) else shape
    dl, ctx = context(H, D, B=64)
    rng = np.random.default_rng(seed + H + D + sum(held) + sum(nodes))
    st, total, gap = starts_of(nodes), sum(nodes), 5
    pages, table = books(dl, rng, [h + n for h, n in zip(held, nodes)], held, page, cols=cols)
    pool, q = bf(rng, pages.n_pages, 2, Hk, page, D), bf(rng, total + gap, H, D)
    words, mask = -(-max(nodes) // 32), None
    if masked:
        mask, _ = od.tree_plan([random_tree(rng, n) for n in nodes], [0] * len(nodes), words)
    out, clean = (torch.full((total + gap, H, D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    scale = D ** -0.5 if scale is None else scale
    dev_mask = None if mask is None else i32(np.concatenate([mask.view(np.int32), np.full((gap, words), -1, np.int32)]))
    args = (i32(st), max(nodes), dev_mask, scale)
    if touched is not None:
        ctx.kv16_attn_tree(pages, up(pool), up(q), *args, clean)
    plant(q, pool, lambda b, t: (table[b, t // page], t % page))
    ctx.kv16_attn_tree(pages, up(pool), up(q), *args, out)
    assert ctx.device_status()[0] == 0
    got, lost = wl.from_torch(out).astype(np.float64), 0
    assert (got[total:] == 7).all()
    for b, (a, e) in enumerate(zip(st, st[1:])):
        if touched is not None and b not in touched:
            assert torch.equal(out[a:e], clean[a:e]) and bool(out[a:e].isfinite().all())
            continue
        k, v = cache_rows(pool, table, b, held[b] + nodes[b], page)
        m = None if mask is None else mask[a:e]
        with np.errstate(all="ignore"):
            ref = od.attention_tree(q[a:e], k, v, held[b], m, scale)
            size = od.attention_tree(q[a:e], k, np.abs(v), held[b], m, scale)
        there = np.isfinite(ref)
        assert (there.all(-1) | ~there.any(-1)).all()                  # (keys and queries take a row with them, whole)
        wrong = np.isnan(got[a:e]) == there
        assert not wrong.any(), f"sequence {b}: {wrong.sum()} of {wrong.size}, {(~there).sum()} should be NaN; {np.argwhere(wrong)[:4]}"
        bound = HALF * (size + np.abs(ref)) + (2.0 ** -12 + (held[b] + nodes[b]) * 2.0 ** -24) * size
        assert (np.abs(got[a:e] - ref) <= bound)[there].all(), f"sequence {b}"
        lost += int((~there.any(-1)).sum())
    ctx.close()
    return lost


@pytest.mark.parametrize("what", BAD)
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_key_that_rows_see(shape, masked, what):
    """One value of a key: in a row held, which a whole sequence sees, in its first, a middle or its last tile, and in a node's."""
    H, Hk, D, page, held, nodes, _ = SHAPES[shape]
    b = int(np.argmax(held))
    for t in (0, held[b] // 2, held[b] - 1, held[b] + nodes[b] // 2) if what == "nan" else (held[b] // 3, held[b]):
        def plant(q, pool, place):
            p, r = place(b, t)
            pool[p, 0, Hk - 1, r, 3] = BAD[what]
        lost = check(shape, masked, plant, [b], seed=t)
        assert lost if what == "nan" else True


@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_query(shape, masked):
    """NaN in one head of one node, and in all heads of another."""
    H, Hk, D, page, held, nodes, _ = SHAPES[shape]
    starts = starts_of(nodes)

    def plant(q, pool, place):
        q[starts[-1] - 1, 1, 5] = np.nan
        q[starts[1] // 2, :, 0] = np.nan
        q[starts[-1]:] = np.nan                                        # rows of no sequence
    assert check(shape, masked, plant, [0, len(nodes) - 1]) in (H, H + 1)
