"""Attention over the paged 16-bit cache (not in the paper): a probability is rounded to bf16 once, also where the row's maximum is raised behind
it in the same tile of keys.

Every row's keys score 0 (32 keys and more), then z of up to 8 in log2 units, so that the maximum stays, then more than 8, so that it is
raised.  Only the second one has values.  Bound as in tests/test_gpu_drafts.py: one rounding of the probability, one of the output (2^-8
each), 2^-12 for scores and exponentials.  The queries are those for which rounding twice would come to nearly two half steps."""
import numpy as np
import pytest
import torch

from tests.test_gpu_drafts import DEV, HALF, books, context, i32, up
from paper_2412_00876_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).double().numpy()


def queries(rng, n, lead):
    """Two dims of n queries whose sum is about 5: scores z = sum / ln 2 and lead * z, bad ones when 2^z is rounded, then 2^z 2^(-lead z)."""
    q = bf16(np.stack([rng.uniform(4.8, 5.0, 400000), rng.uniform(0.0005, 0.06, 400000)], -1))
    z = q.sum(-1) / np.log(2)
    z, first = np.unique(np.where((z < 7.99) & (lead * z > 8.01), z, 7.5), return_index=True)
    q = q[first]
    twice = bf16(bf16(2.0 ** z) * 2.0 ** (-lead * z)) / 2.0 ** (z - lead * z) - 1
    worst = np.flatnonzero((np.abs(twice) > 1.6 * HALF) & (z != 7.5))
    assert len(worst) > 8
    return q[worst[np.arange(n) % len(worst)]]


@pytest.mark.parametrize("lead", [1.140625, 1.28125])
@pytest.mark.parametrize("second,third", [(5, 40), (40, 70), (33, 127), (70, 100)])
@pytest.mark.parametrize("D,n,masked", [(128, 128, True), (64, 100, True), (128, 300, True), (64, 260, False), (128, 60, True)])
def test_a_probability_is_rounded_once(D, n, masked, second, third, lead):
    dl, ctx = context(2, D, B=1)
    rng = np.random.default_rng(n + second)
    last = min(n, 128)                                                 # (the first tile of keys; later ones score 0)
    second, third = (min(t, last - 8 + i) for i, t in enumerate((second, third)))
    pages, table = books(dl, rng, [n], [0], 64)
    pool, q = np.zeros((pages.n_pages, 2, 2, 64, D), np.float32), np.zeros((n, 2, D), np.float32)
    q[:, :, :2] = queries(rng, 2 * n, lead).reshape(n, 2, 2)
    values = 1 + np.arange(D) % 128 / 128 * (128 // min(D, 128))
    for t, size in ((second, 1.0), (third, lead)):
        pool[table[0, t // 64], 0, :, t % 64, :2] = size
    pool[table[0, second // 64], 1, :, second % 64] = values
    words = -(-n // 32)
    out = torch.zeros(n, 2, D, dtype=torch.bfloat16, device=DEV)
    mask = torch.full((n, words), -1, dtype=torch.int32, device=DEV) if masked else None
    ctx.kv16_attn_tree(pages, up(pool), up(q), i32([0, n]), n, mask, 1.0, out)
    assert ctx.device_status()[0] == 0
    z = q.astype(np.float64).sum(-1)
    sees = np.full(n, n) if masked else np.arange(1, n + 1)
    e2, e3 = np.exp(z) * (sees > second)[:, None], np.exp(lead * z) * (sees > third)[:, None]
    zeros = (sees - (sees > second) - (sees > third))[:, None]
    ref = (e2 / (zeros + e2 + e3))[..., None] * values
    got = wl.from_torch(out).astype(np.float64)
    bound = (2 * HALF + 2.0 ** -12 + n * 2.0 ** -24) * ref
    assert (np.abs(got - ref) <= bound).all(), f"{(np.abs(got - ref) > bound).sum()} off, {(np.abs(got - ref) / np.maximum(ref, 1e-30)).max() / HALF} half steps"
    ctx.close()
