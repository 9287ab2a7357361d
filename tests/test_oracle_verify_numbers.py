"""The oracle's verification (not in the paper) with random numbers outside [0, 1): each counts as the nearest number inside, NaN as 0."""
import numpy as np
import pytest

from oracle import drafts as od

LAST = 1 - 2.0 ** -24
OUTSIDE = [(-1.0, 0.0), (-np.inf, 0.0), (np.nan, 0.0), (-1e-30, 0.0), (1.0, LAST), (2.0, LAST), (np.inf, LAST)]


@pytest.mark.parametrize("u,inside", OUTSIDE)
@pytest.mark.parametrize("mode", ["sample", "replaced", "point"])
def test_numbers_outside_count_as_the_nearest_inside(mode, u, inside):
    rng = np.random.default_rng(3)
    for parent in ([-1, 0, 0, 0], [-1, 0, 1, 2], [-1, 0, 0, 1]):
        for tokens in ([0, 2, 2, 4], [0, 4, 2, 2], [0, 1, 1, 1]):
            p, q = (np.zeros((4, 5), np.float32) for _ in range(2))
            p[:, 2:], q[:] = rng.dirichlet(np.ones(3), 4), rng.dirichlet(np.ones(5), 4)
            for draft in (q, p):
                draft = None if mode == "point" else draft
                call = lambda x: od.verify(p, draft, np.array([0.5, x, x, x], np.float32), tokens, parent, mode)
                assert call(u) == call(inside)


@pytest.mark.parametrize("mode", ["sample", "replaced", "point"])
def test_a_token_without_probability_is_never_accepted(mode):
    p, q = np.array([[0.0, 1.0]] * 2, np.float32), np.array([[0.5, 0.5]] * 2, np.float32)
    for u in (-1.0, -np.inf, 0.0, np.nan):
        keep, token = od.verify(p, None if mode == "point" else q, np.array([0.5, u], np.float32), [0, 0], [-1, 0], mode)
        assert keep == [True, False] and token == 1


@pytest.mark.parametrize("mode", ["sample", "replaced"])
def test_a_draft_equal_to_the_target_is_always_accepted(mode):
    p = np.array([[0.25, 0.75]] * 2, np.float32)
    for u in (0.5, LAST, 1.0, 7.0, np.inf):
        assert od.verify(p, p, np.array([0.5, u], np.float32), [0, 0], [-1, 0], mode)[0] == [True, True]
