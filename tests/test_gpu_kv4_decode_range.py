"""Decode attention over the 4-bit cache where the weights p and the scales s of the values span many powers of two: rows
that nobody attends, scores that lead by far, groups of 64 dims of different size, parts that are kept and begun anew.

Bound.  With the values v = s code + z the kernel adds up  sum (p s) code  and  sum p z.  Written as factors of the exact sums:
  - p s is rounded to fp16 once, 2^-11 of itself; below 2^-14 (of what the kernel scales it to) 2^-25 absolute instead.  The
    scale puts the largest p s that a head and group of dims have met at 2^9 or above, so that n rows are off by
    n 2^-34 of the largest p s code together;
  - the matrix accumulators cut additions off, 64 of them before a sum is kept: 2^-17 of sum p (v - z);
  - a score is an fp32 sum of D products and a few more operations on terms that add up to A = sum |q| (|z| + 15 s) scale:
    (D + 16) 2^-23 A (cut off, too), and the exponential adds 2^-21.  A relative error of that size, `delta`, in every p
    changes an output by up to twice it, of sum p |v| + sum p (v - z);
  - the output is rounded to bf16, 2^-8 of itself.
All sums over p are divided by sum p; the token's own row takes part with its exact value."""
import numpy as np
import pytest
import torch

from oracle import paged_kv4 as pk
from paper_2412_00876_b200 import workloads as wl
from tests.test_gpu_serving_ops import DEV, EPS, bf, books, context, i32, lift, starts_of, up

pytestmark = pytest.mark.gpu


def reference(q, kt, vt, k, v, scale):
    """One head and sequence: the output over the rows' 4-bit values, and its bound."""
    kc, ks, kz = pk.quantise(k)
    kh, vh, vl = pk.values(kc, ks, kz), pk.held(v), lift(v)
    q, kt, vt = (np.asarray(t, np.float64) for t in (q, kt, vt))
    z = np.append(kh @ q, q @ kt) * scale
    p = np.exp(z - z.max())
    p /= p.sum()
    out = p[:-1] @ vh + p[-1] * vt
    most = np.repeat(np.abs(kz) + 15 * ks, 64, -1)
    A = max((most @ np.abs(q)).max(initial=0.0), np.abs(q) @ np.abs(kt)) * scale
    delta = (q.shape[-1] + 16) * 2.0 ** -23 * A + 2.0 ** -21
    lifted, size = p[:-1] @ vl, p[:-1] @ np.abs(vh) + p[-1] * np.abs(vt)
    rows = len(k) * 2.0 ** -34 * (p[:-1, None] * vl).max(0, initial=0.0)
    return out, EPS * np.abs(out) + (2.0 ** -11 + 2.0 ** -17) * lifted + 2 * delta * (lifted + size) + rows + 2.0 ** -120


def attend(H, D, Hk, page, lens, q, kt, vt, kv, scale):
    """The kernel's output, checked against `reference` for every sequence and head."""
    dl, ctx = context(H, D, B=len(lens))
    rng = np.random.default_rng(H + D)
    st = starts_of(lens)
    pg = books(dl, len(lens), sum(-(-n // page) for n in lens) + 1, max(-(-n // page) for n in lens) + 1, page, lens, rng)
    pool = ctx.kv4_pool(pg, Hk)
    d = up(kv)
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32(st))
    out = torch.zeros(len(lens), H, D, dtype=torch.bfloat16, device=DEV)
    ctx.kv4_attn_decode(pg, pool, up(q), up(kt), up(vt), None, scale, out)
    got = wl.from_torch(out)
    G = H // Hk
    for b in range(len(lens)):
        rows = kv[st[b]:st[b + 1]]
        for h in range(H):
            ref, bound = reference(q[b, h], kt[b, h // G], vt[b, h // G], rows[:, h // G], rows[:, Hk + h // G], scale)
            off = np.abs(got[b, h] - ref)
            assert np.all(off <= bound), f"sequence {b}, head {h}: worst {(off / bound).max()} of the bound, error {off.max()}"
    assert ctx.device_status()[0] == 0
    ctx.close()


def scores_in_dim_0(rng, B, H, Hk, D, total, spread=1.0):
    """q, k_t, v_t and K/V rows whose scores (scale 1) are k[0] plus a little of the others."""
    q, kt, vt = bf(rng, B, H, D, scale=0.1), bf(rng, B, Hk, D, scale=0.1), bf(rng, B, Hk, D)
    kv = bf(rng, total, 2 * Hk, D)
    kv[:, :Hk] *= 0.125
    q[:, :, 0] = 1.0
    kv[:, :Hk, 0] = wl.round_to_storage(rng.normal(0, spread, (total, Hk)).astype(np.float32), "bf16")
    return q, kt, vt, kv


FORMS = [(2, 2), (8, 2), (16, 1), (12, 1)]


@pytest.mark.parametrize("H,Hk", FORMS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("k", [12, 18, 20, 24, 30])
def test_a_large_row_that_nobody_attends_costs_the_others_nothing(H, Hk, D, k):
    """V rows 2^k times the others with scores 30 + k ln 2 below them: early, so that all later ones would be scaled by them, in
    one group of dims and in both, and late."""
    lens = [64, 64, 200, 333]
    rng = np.random.default_rng(100 * k + H)
    q, kt, vt, kv = scores_in_dim_0(rng, len(lens), H, Hk, D, sum(lens))
    st = starts_of(lens)
    for b, at, dims in ((0, 0, slice(0, D)), (1, 5, slice(0, 64)), (2, 150, slice(0, D)), (3, 0, slice(D - 64, D)), (3, 331, slice(0, D))):
        kv[st[b] + at, :Hk, 0] = wl.round_to_storage(np.float32([-30 - k * np.log(2)]), "bf16")[0]
        kv[st[b] + at, Hk:, dims] *= 2.0 ** k
    attend(H, D, Hk, 16, lens, q, kt, vt, kv, 1.0)


@pytest.mark.parametrize("H,Hk", FORMS)
@pytest.mark.parametrize("lead", [5.0, 17.0, 40.0])
@pytest.mark.parametrize("small", [0.0, 2.0 ** -20])
def test_a_leading_score_with_a_small_value_leaves_the_rest_its_bits(H, Hk, lead, small):
    """A row whose score stands `lead` (base e) above all others and whose value is zero, or small, as a sequence's first row
    often is: the output is what the others add up to."""
    D, lens = 128, [40, 200, 700, 700, 333]
    rng = np.random.default_rng(int(lead) + H)
    q, kt, vt, kv = scores_in_dim_0(rng, len(lens), H, Hk, D, sum(lens), 0.5)
    st = starts_of(lens)
    for b, at in ((0, 0), (1, 199), (2, 0), (3, 400), (4, 100), (4, 300)):
        kv[st[b] + at, :Hk, 0] = lead
        kv[st[b] + at, Hk:] *= small
    attend(H, D, Hk, 32, lens, q, kt, vt, kv, 1.0)


@pytest.mark.parametrize("H,Hk", FORMS)
def test_values_and_weights_of_many_sizes(H, Hk):
    """V rows of sizes 2^-20 .. 2^20 at random against scores that spread over e^+-20."""
    D, lens = 128, [77, 500, 1, 900]
    rng = np.random.default_rng(H)
    q, kt, vt, kv = scores_in_dim_0(rng, len(lens), H, Hk, D, sum(lens), 8.0)
    kv[:, Hk:] *= 2.0 ** rng.integers(-20, 21, (sum(lens), Hk, 1))
    attend(H, D, Hk, 64, lens, q, kt, vt, kv, 1.0)


@pytest.mark.parametrize("H,Hk", FORMS)
@pytest.mark.parametrize("sizes", [(40, -40), (-40, 40), (15, -15), (110, 110), (-100, -100), (100, -100), (0, -118)])
def test_the_two_groups_of_dims_may_be_of_different_size(H, Hk, sizes):
    D, lens = 128, [100, 257]
    rng = np.random.default_rng(1000 + H + sizes[0])
    q, kt, vt, kv = scores_in_dim_0(rng, len(lens), H, Hk, D, sum(lens), 2.0)
    for g in range(2):
        kv[:, Hk:, 64 * g:64 * g + 64] *= np.float32(2.0 ** sizes[g])
        vt[:, :, 64 * g:64 * g + 64] *= np.float32(2.0 ** sizes[g])
    attend(H, D, Hk, 16, lens, q, kt, vt, kv, 1.0)


@pytest.mark.parametrize("H,Hk", [(16, 16), (64, 16), (192, 16)])
@pytest.mark.parametrize("what", ["lead", "large"])
def test_sums_that_are_kept_and_begun_anew(H, Hk, what):
    """128 sequences that name the same pages, 4096 rows, so that a warp's sums are kept several times within a part: leading
    scores with values of zero, or large rows that nobody attends, at different places for each K/V head; sampled sequences."""
    D, page, n, B = 128, 128, 4096, 128
    dl, ctx = context(H, D, B=B)
    rng = np.random.default_rng(H)
    q, kt, vt, kv = scores_in_dim_0(rng, B, H, Hk, D, n, 0.5)
    for hk in range(Hk):
        at = hk * 273
        if what == "lead":
            kv[at, hk, 0], kv[at, Hk + hk] = 20.0, 0.0
        else:
            kv[at, hk, 0] = -40.0
            kv[at, Hk + hk] *= 2.0 ** 26
    pg = dl.Pages(B, n // page, n // page, page, DEV)
    pool = ctx.kv4_pool(pg, Hk)
    pg.table.copy_(torch.arange(n // page, dtype=torch.int32, device=DEV).repeat(B, 1))
    d = up(kv)
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32([0] + [n] * B))
    pg.cache_len.fill_(n)
    out = torch.zeros(B, H, D, dtype=torch.bfloat16, device=DEV)
    ctx.kv4_attn_decode(pg, pool, up(q), up(kt), up(vt), None, 1.0, out)
    got, G = wl.from_torch(out), H // Hk
    for b in (0, 31, 77, 127):
        for hk in range(Hk):
            h = hk * G + b % G
            ref, bound = reference(q[b, h], kt[b, hk], vt[b, hk], kv[:, hk], kv[:, Hk + hk], 1.0)
            off = np.abs(got[b, h] - ref)
            assert np.all(off <= bound), f"sequence {b}, head {h}: worst {(off / bound).max()} of the bound"
    assert ctx.device_status()[0] == 0
    ctx.close()
