"""Verification of drafts (not in the paper) with random numbers outside [0, 1): decisions as the oracle's, and as those of the nearest
numbers inside, bit for bit.  No tolerance: whole numbers and truth values."""
import numpy as np
import pytest

from tests.test_gpu_drafts import check_verify, context, probabilities, random_tree, run_verify
from tests.test_oracle_verify_numbers import LAST, OUTSIDE

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("u,inside", OUTSIDE)
@pytest.mark.parametrize("mode", ["sample", "replaced", "point"])
def test_numbers_outside_count_as_the_nearest_inside(mode, u, inside):
    """Children's numbers outside, among them those of tokens without probability and of siblings of the same token."""
    _, ctx = context(2, 64)
    rng = np.random.default_rng(11)
    for V in (5, 40000):
        parents = [random_tree(rng, n) for n in (6, 1, 40)]
        total = sum(len(p) for p in parents)
        p, q = probabilities(rng, total, V), probabilities(rng, total, V)
        p[:, 0] = 0.0                                                  # a token that the target never gives
        tokens = rng.integers(0, 3, total)
        numbers = rng.random(total).astype(np.float32)
        out, hit = numbers.copy(), rng.random(total) < 0.6
        hit[[0, 6, 7]] = False                                         # (the roots' numbers draw the token: not here)
        out[hit] = u
        numbers[hit] = inside
        for draft in ([None] if mode == "point" else [q, p]):
            check_verify(ctx, p, draft, out, tokens, parents, mode)
            assert run_verify(ctx, p, draft, out, tokens, parents, mode) == run_verify(ctx, p, draft, numbers, tokens, parents, mode)
    assert ctx.device_status()[0] == 0
    ctx.close()


@pytest.mark.parametrize("mode", ["sample", "replaced", "point"])
def test_roots_numbers_outside(mode):
    """The root's number draws: below 0 and NaN the first token that is left, from 1 on the last."""
    _, ctx = context(2, 64)
    p = np.zeros((1, 9), np.float32)
    p[0, [2, 5, 7]] = 0.25, 0.5, 0.25
    for u, token in [(-1.0, 2), (np.nan, 2), (-np.inf, 2), (LAST, 7), (1.0, 7), (3.0, 7), (np.inf, 7)]:
        args = (p, None if mode == "point" else p, np.array([u], np.float32), np.array([0]), [[-1]], mode)
        assert run_verify(ctx, *args) == ([[True]], [1], [token])
        check_verify(ctx, *args)
    ctx.close()


@pytest.mark.parametrize("mode", ["sample", "replaced", "point"])
def test_a_token_without_probability_is_never_accepted(mode):
    _, ctx = context(2, 64)
    p, q = np.array([[0.0, 1.0]] * 2, np.float32), np.array([[0.5, 0.5]] * 2, np.float32)
    for u in (-1.0, -np.inf, 0.0, np.nan):
        got = run_verify(ctx, p, None if mode == "point" else q, np.array([0.5, u], np.float32), np.array([0, 0]), [[-1, 0]], mode)
        assert got == ([[True, False]], [1], [1])
    ctx.close()
