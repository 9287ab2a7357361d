"""GPU parity of the serving extensions (not in the paper) against oracle/paged_kv4.py: attention over packed prompts with
grouped heads, the paged 4-bit cache (append, read, decode attention), page bookkeeping, and a run of them together.

Tolerances.  Books, page bytes and codes are compared exactly.  A value read back is one rounding to bf16 away from the
oracle's (2^-8 relative, plus the fp32 rounding of s * code + z).  Attention: every probability is rounded once (bf16 for
prompts, 2^-9 of itself on average and 2^-8 at most; fp16 for the 4-bit cache) before it multiplies a value, so an output
is off by at most 2^-8 * sum p |v| / sum p for that, plus its own rounding to bf16, 2^-8 of itself; scores carry fp32 sums
of D products (relative 2^-24 * D of sum |q k|, times ln 2^-1 through the exponential) and exponentials 2^-13 relative.
With |v| up to vmax this is bounded by  2^-8 * (vmean + |out|) * 1.1 + 1e-4 * vmax,  vmean = sum p |v| (taken from the
oracle); `close` checks that bound elementwise with vmean replaced by the oracle's attention over |v|.
The 4-bit kernel adds sum p s code and sum p z up apart, and rounds p s to fp16 (2^-11 relative at most) in the first sum
only: the error of one key is up to 2^-11 p s code = 2^-11 p (v - z), which can exceed 2^-11 p |v| since z < 0 < v - z
where v is near 0.  So its bound has a further term 2^-11 * sum p (v - z) / sum p, taken from the oracle (`lift`)."""
import numpy as np
import pytest
import torch

from oracle import paged_kv4 as pk
from paper_2412_00876_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)
EPS = 2.0 ** -8                               # half a bf16 step, relative


def bf(rng, *shape, scale=1.0):
    return wl.round_to_storage(rng.normal(0, scale, shape).astype(np.float32), "bf16")


def up(x):
    return wl.to_torch(x, "bf16", DEV)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def starts_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def context(H, D, B=8, **kw):
    from paper_2412_00876_b200 import binding as dl
    return dl, dl.Context(64, H, D, 64, torch.bfloat16, 0, max_batch=B, cap=64, **kw)


def lift(x):
    """v - z of rows held in 4 bits"""
    code, s, _ = pk.quantise(x)
    return pk.values(code, s, np.zeros_like(s))


def close(got, ref, ref_abs, what, ref_lift=0.0):
    got = np.asarray(got, np.float64)
    bound = EPS * 1.1 * (ref_abs + np.abs(ref)) + 2.0 ** -11 * ref_lift + 1e-4 * max(1.0, np.abs(ref_abs).max(initial=0.0))
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} values off, worst {np.abs(got - ref)[bad].max()} at {np.argwhere(bad)[:4]}"


# ---- packed prompts -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hk,D,lens", [
    (4, 4, 128, [1]), (4, 4, 64, [1, 2, 3]), (2, 2, 128, [15, 16, 17, 0, 33]), (8, 2, 128, [31, 32, 33, 1, 64]),
    (8, 1, 64, [127, 128, 129]), (16, 1, 128, [7, 8, 9, 150]), (6, 2, 128, [130, 5]), (5, 1, 64, [257, 0, 0, 3]),
    (2, 2, 128, [255, 256, 257, 300]), (7, 7, 64, [0, 97, 300]), (12, 1, 128, [65, 66, 400]), (4, 2, 64, [513, 140])])
def test_packed_prompts(H, Hk, D, lens):
    dl, ctx = context(H, D)
    rng = np.random.default_rng(H * 1000 + D + sum(lens))
    st, total = starts_of(lens), sum(lens)
    q, k, v = bf(rng, total, H, D), bf(rng, total, Hk, D), bf(rng, total, Hk, D)
    qkv = up(np.concatenate([q, k, v], 1))                        # one projection's output: strided rows
    out = torch.full((total, H, D), 7.0, dtype=torch.bfloat16, device=DEV)
    ctx.attn_prefill_packed(qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], i32(st), max(lens), D ** -0.5, out)
    ref = pk.attention_packed(q, k, v, st, D ** -0.5)
    close(wl.from_torch(out), ref, pk.attention_packed(q, k, np.abs(v), st, D ** -0.5), "packed prompts")
    assert ctx.device_status()[0] == 0
    # dense rows give the same bits, and so does a larger max_rows
    out2 = torch.zeros_like(out)
    ctx.attn_prefill_packed(up(q), up(k), up(v), i32(st), max(lens) + 400, D ** -0.5, out2)
    assert torch.equal(out, out2)
    ctx.close()


def test_packed_prompts_long_rows_sampled():
    """Thousands of keys: sampled rows against the oracle."""
    H, Hk, D, lens = 4, 2, 128, [2500, 1, 1111]
    dl, ctx = context(H, D)
    rng = np.random.default_rng(5)
    st, total = starts_of(lens), sum(lens)
    q, k, v = bf(rng, total, H, D, scale=2.0), bf(rng, total, Hk, D), bf(rng, total, Hk, D)
    out = torch.zeros((total, H, D), dtype=torch.bfloat16, device=DEV)
    ctx.attn_prefill_packed(up(q), up(k), up(v), i32(st), max(lens), D ** -0.5, out)
    got = wl.from_torch(out)
    for b, n in enumerate(lens):
        for i in sorted({0, n // 3, n - 1, max(0, n - 130)}):
            r = st[b] + i
            args = [np.asarray(t, np.float64) for t in (q[r], k[st[b] + i], v[st[b] + i], k[st[b]:r], v[st[b]:r])]
            ref = pk.attention_decode(*args, D ** -0.5)
            args[2], args[4] = np.abs(args[2]), np.abs(args[4])
            close(got[r], ref, pk.attention_decode(*args, D ** -0.5), f"row {i} of {n}")
    assert ctx.device_status()[0] == 0
    ctx.close()


def test_packed_rows_of_no_sequence_are_left_and_neighbours_do_not_leak():
    """NaN rows between and behind the sequences: nothing of them arrives, and their output rows stay as they were."""
    H, Hk, D, lens, gap = 4, 2, 128, [37, 130, 5], 9
    dl, ctx = context(H, D)
    rng = np.random.default_rng(6)
    st = starts_of(lens)
    total = int(st[-1]) + gap
    q, k, v = bf(rng, total, H, D), bf(rng, total, Hk, D), bf(rng, total, Hk, D)
    dq, dk, dv = up(q), up(k), up(v)
    for t in (dq, dk, dv):
        t[st[-1]:] = float("nan")
    out = torch.full((total, H, D), 3.0, dtype=torch.bfloat16, device=DEV)
    ctx.attn_prefill_packed(dq, dk, dv, i32(st), 130, D ** -0.5, out)
    n = int(st[-1])
    ref = pk.attention_packed(q[:n], k[:n], v[:n], st, D ** -0.5)
    close(wl.from_torch(out)[:n], ref, pk.attention_packed(q[:n], k[:n], np.abs(v[:n]), st, D ** -0.5), "packed")
    assert torch.all(out[n:] == 3.0)
    # a sequence of NaN leaves its neighbours clean
    dk[st[1]:st[2]] = float("nan")
    dv[st[1]:st[2]] = float("nan")
    out2 = torch.zeros_like(out)
    ctx.attn_prefill_packed(dq, dk, dv, i32(st), 130, D ** -0.5, out2)
    assert torch.equal(out2[:st[1]], out[:st[1]]) and torch.equal(out2[st[2]:n], out[st[2]:n])
    assert torch.isnan(out2[st[1]:st[2]]).all()
    assert ctx.device_status()[0] == 0
    ctx.close()


def test_packed_reports_bad_starts():
    H, D = 4, 64
    dl, ctx = context(H, D)
    x = torch.zeros(40, 3 * H, D, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(40, H, D, dtype=torch.bfloat16, device=DEV)
    for starts, rows, bad in (([0, 50], 40, 0), ([0, 10, 5], 40, 1), ([-3, 10], 40, 0), ([0, 10, 40], 20, 1)):
        ctx.attn_prefill_packed(x[:, :H], x[:, H:2 * H], x[:, 2 * H:], i32(starts), rows, 0.1, out)
        assert ctx.device_status() == (dl.DL_ERR_INVALID_ARG, bad), starts
    ctx.close()


# ---- 4-bit rows -----------------------------------------------------------------------------------------------------
def books(dl, B, n_pages, width, page, rows, rng):
    """Pages for `rows[b]` rows each, at random places."""
    pg = dl.Pages(B, n_pages, width, page, DEV)
    order, at = rng.permutation(n_pages), 0
    table = np.full((B, width), -1, np.int32)
    for b, n in enumerate(rows):
        c = -(-n // page)
        table[b, :c] = order[at:at + c]
        at += c
    pg.table.copy_(i32(table))
    pg.refs.copy_(i32(np.bincount(table[table >= 0], minlength=n_pages)))
    return pg


def read(ctx, pg, pool, Hk, D, first, lens):
    n = int(sum(lens))
    k, v = (torch.full((n, Hk, D), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.kv4_read(pg, pool, i32(first), i32(starts_of(lens)), k, v)
    return wl.from_torch(k), wl.from_torch(v)


def same_values(got, ref, what):
    """one rounding to bf16 of the oracle's value (and the fp32 rounding of s * code + z before it)"""
    ref = np.asarray(ref, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what
    assert np.all(np.isnan(ref) | (np.abs(got - ref) <= EPS * np.abs(ref) + 1e-6 * np.nanmax(np.abs(ref), initial=0.0))), what


@pytest.mark.parametrize("Hk,D,page,lens,keep,before", [
    (1, 64, 16, [1], None, 0), (1, 128, 16, [1, 0, 17], None, 3), (2, 128, 32, [40, 31, 33], 0.5, 15),
    (3, 64, 64, [100, 5], 0.3, 60), (8, 128, 128, [200, 130, 1], 0.7, 127), (5, 128, 16, [64, 64], 0.0, 16)])
def test_append_and_read(Hk, D, page, lens, keep, before):
    dl, ctx = context(Hk, D)
    rng = np.random.default_rng(D + page + sum(lens))
    st, total, B = starts_of(lens), sum(lens), len(lens)
    kv = bf(rng, total, 2 * Hk, D)
    kv[:, :, ::17] *= 8
    if total > 3:
        kv[0, 0, :64] = 1.5                                        # one value: s is 0
        kv[1, 0, :64] = np.arange(64) % 16                        # codes exact
        kv[2, 0, :64] = wl.round_to_storage(np.linspace(-1e-38, 1e-38, 64), "bf16")
    flags = (rng.random(total) < keep).astype(np.uint8) if keep is not None else np.ones(total, np.uint8)
    kept = [int(flags[a:e].sum()) for a, e in zip(st, st[1:])]
    rows = [before + n for n in kept]
    pg = books(dl, B, sum(-(-n // page) for n in rows) + 2, max(-(-n // page) for n in rows) + 1, page, rows, rng)
    pool = ctx.kv4_pool(pg, Hk)
    pool.fill_(0xA5)
    was = pool.clone()
    pg.cache_len.fill_(before)
    d = up(kv)
    kw = dict(keep=torch.from_numpy(flags).to(DEV)) if keep is not None else {}
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32(st), commit=False, **kw)
    assert pg.cache_len.tolist() == [before] * B
    once = pool.clone()
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32(st), **kw)
    assert torch.equal(pool, once) and pg.cache_len.tolist() == rows
    gk, gv = read(ctx, pg, pool, Hk, D, [before] * B, kept)
    ref = pk.held(kv[flags != 0])
    same_values(gk, ref[:, :Hk], "K")
    same_values(gv, ref[:, Hk:], "V")
    # pages nobody was given and rows below `before` keep their bytes
    unused = (pg.refs == 0).nonzero().flatten()
    assert torch.equal(pool[unused], was[unused])
    if before:
        a = pool.clone()
        pool.copy_(was)
        bk, bv = read(ctx, pg, pool, Hk, D, [0] * B, [before] * B)
        pool.copy_(a)
        ck, cv = read(ctx, pg, pool, Hk, D, [0] * B, [before] * B)
        assert np.array_equal(bk, ck, equal_nan=True) and np.array_equal(bv, cv, equal_nan=True)
    assert ctx.device_status()[0] == 0
    ctx.close()


@pytest.mark.parametrize("Hk,D", [(1, 64), (2, 64), (3, 128)])
def test_append_and_read_at_every_allowed_alignment(Hk, D):
    """Sources and outputs at multiples of 16 bytes that are not multiples of 32, and rows an odd number of 16 bytes apart:
    the same bits as at multiples of 32."""
    dl, ctx = context(Hk, D)
    rng = np.random.default_rng(Hk + D)
    lens, page = [37, 0, 1, 64], 32
    st, total, w = starts_of(lens), sum(lens), 2 * Hk * D
    kv = up(bf(rng, total, 2 * Hk, D))
    flags = torch.from_numpy((rng.random(total) < 0.7).astype(np.uint8)).to(DEV)
    kept = [int(flags[a:e].sum()) for a, e in zip(st, st[1:])]
    pg = books(dl, 4, 12, 3, page, lens, rng)
    seen = []
    for shift, gap in [(0, 0), (8, 0), (0, 8), (8, 8), (16, 24)]:
        rows = torch.zeros(shift + total * (w + gap), dtype=torch.bfloat16, device=DEV)[shift:].view(total, w + gap)[:, :w].view(total, 2 * Hk, D)
        rows.copy_(kv)
        pool = ctx.kv4_pool(pg, Hk)
        pg.cache_len.zero_()
        ctx.kv4_append(pg, pool, rows[:, :Hk], rows[:, Hk:], i32(st), keep=flags)
        got = [torch.full((shift + sum(kept) * Hk * D + 8,), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        k, v = (t[shift:shift + sum(kept) * Hk * D].view(sum(kept), Hk, D) for t in got)
        ctx.kv4_read(pg, pool, i32([0] * 4), i32(starts_of(kept)), k, v)
        assert all(bool((t[:shift] == 7).all()) and bool((t[-8:] == 7).all()) for t in got)
        seen.append((pool.clone(), k.clone(), v.clone()))
    ref = pk.held(kv.float().cpu().numpy()[flags.cpu().numpy() != 0])
    same_values(seen[0][1].float().cpu().numpy(), ref[:, :Hk], "K")
    same_values(seen[0][2].float().cpu().numpy(), ref[:, Hk:], "V")
    for other in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(seen[0], other))
    assert ctx.device_status()[0] == 0
    ctx.close()


def test_rows_with_nan_and_infinity_hold_nan_in_their_group_only():
    Hk, D = 1, 128
    dl, ctx = context(Hk, D)
    rng = np.random.default_rng(3)
    kv = bf(rng, 4, 2, D)
    kv[0, 0, 3], kv[1, 0, 100], kv[2, 1, 64] = np.nan, np.inf, -np.inf
    kv[3, 1, 0], kv[3, 1, 1] = wl.round_to_storage(np.float32([3e38, -3e38]), "bf16")
    pg = books(dl, 1, 1, 1, 16, [4], rng)
    pool = ctx.kv4_pool(pg, Hk)
    d = up(kv)
    ctx.kv4_append(pg, pool, d[:, :1], d[:, 1:], i32([0, 4]))
    gk, gv = read(ctx, pg, pool, Hk, D, [0], [4])
    ref = pk.held(kv)
    assert np.isnan(ref).sum() == 4 * 64
    same_values(gk, ref[:, :1], "K")
    same_values(gv, ref[:, 1:], "V")
    ctx.close()


def test_append_refuses_missing_pages_and_leaves_the_sequence():
    Hk, D, page = 2, 64, 16
    dl, ctx = context(Hk, D)
    rng = np.random.default_rng(4)
    lens = [20, 20, 20, 20]
    d = up(bf(rng, 80, 2 * Hk, D))
    pg = books(dl, 4, 8, 3, page, [20, 16, 20, 40], rng)
    pg.table[2, 1] = 1000                                          # no such page
    pg.cache_len.copy_(i32([0, 0, 0, 30]))                          # 30 + 20 rows do not fit 3 pages of 16
    pool = ctx.kv4_pool(pg, Hk)
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32(starts_of(lens)))
    assert pg.cache_len.tolist() == [20, 0, 0, 30]
    code, detail = ctx.device_status()
    assert code == dl.DL_ERR_CAPACITY and detail in (1, 2, 3)
    for b in (1, 2, 3):
        for p in pg.table[b].tolist():
            if 0 <= p < 8:
                assert int(pool[p].sum()) == 0
    # reading past the pages gives zeros and says so
    gk, _ = read(ctx, pg, pool, Hk, D, [0, 16, 16, 32], [1, 1, 1, 1])
    assert np.all(gk[1:3] == 0)
    assert ctx.device_status()[0] == dl.DL_ERR_INVALID_ARG
    ctx.close()


# ---- decode attention -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hk,D,page,lens", [
    (4, 4, 128, 16, [0]), (4, 4, 128, 16, [1, 15, 16, 17]), (8, 2, 128, 32, [31, 0, 33, 300]), (8, 1, 64, 64, [63, 64, 65, 1]),
    (5, 1, 128, 64, [700, 5, 0]), (16, 1, 128, 16, [100, 257]), (12, 1, 64, 128, [129, 400, 3]), (32, 8, 128, 64, [1000, 20]),
    (6, 2, 64, 16, [0, 0, 0, 37]), (14, 1, 128, 32, [511]), (3, 3, 64, 16, [5000])])
@pytest.mark.parametrize("spread", [1.0, 30.0])
def test_decode_attention(H, Hk, D, page, lens, spread):
    """Ragged lengths, grouped heads, pairs split over many warps (5000 rows) and many pairs; garbage past the lengths."""
    dl, ctx = context(H, D)
    rng = np.random.default_rng(H + D + page + len(lens))
    B, st, total = len(lens), starts_of(lens), sum(lens)
    kv = bf(rng, total, 2 * Hk, D)
    kv[:, Hk:] *= 2.0 ** rng.integers(-6, 7, (total, 1, 1))        # values of very different sizes from row to row
    q, kt, vt = bf(rng, B, H, D, scale=spread ** 0.5), bf(rng, B, Hk, D), bf(rng, B, Hk, D)
    rows = [n + 1 for n in lens]
    pg = books(dl, B, sum(-(-n // page) for n in rows) + 2, max(-(-n // page) for n in rows) + 2, page, rows, rng)
    pool = ctx.kv4_pool(pg, Hk)
    pool.fill_(0xFF)                                               # words that are NaN
    d = up(kv)
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32(st))
    out = torch.zeros(B, H, D, dtype=torch.bfloat16, device=DEV)
    keep = (np.arange(B) % 2 == 0).astype(np.uint8)
    before = pool.clone()
    ctx.kv4_attn_decode(pg, pool, up(q), up(kt), up(vt), torch.from_numpy(keep).to(DEV), D ** -0.5, out)
    got, h, lifted = wl.from_torch(out), pk.held(kv), lift(kv)
    for b in range(B):
        kr, vr, lr = h[st[b]:st[b + 1], :Hk], h[st[b]:st[b + 1], Hk:], lifted[st[b]:st[b + 1], Hk:]
        ref = pk.attention_decode(q[b], kt[b], vt[b], kr, vr, D ** -0.5)
        close(got[b], ref, pk.attention_decode(q[b], kt[b], np.abs(vt[b]), kr, np.abs(vr), D ** -0.5), f"sequence {b}",
              pk.attention_decode(q[b], kt[b], 0 * vt[b], kr, lr, D ** -0.5))
    assert pg.cache_len.tolist() == lens
    gk, gv = read(ctx, pg, pool, Hk, D, lens, [1] * B)
    for b in range(B):
        if keep[b]:
            same_values(gk[b], pk.held(kt[b]), "appended K")
            same_values(gv[b], pk.held(vt[b]), "appended V")
        else:
            assert np.isnan(gk[b]).all() and np.isnan(gv[b]).all()
    # the same call gives the same bits, and so does one without the append
    out2 = torch.zeros_like(out)
    ctx.kv4_attn_decode(pg, before, up(q), up(kt), up(vt), None, D ** -0.5, out2)
    assert torch.equal(out, out2)
    assert ctx.device_status()[0] == 0
    ctx.close()


@pytest.mark.parametrize("H,D,page,lens", [
    (1, 64, 16, [1]), (2, 64, 32, [31, 32, 33, 63]), (5, 128, 32, [300, 31, 33, 0, 1200]), (32, 128, 64, [90, 700]),
    (8, 64, 128, [2000, 5]), (1, 128, 16, [15, 17, 47, 48, 49])])
def test_decode_one_query_head_per_kv_head(H, D, page, lens):
    """The form whose lanes share a unit's keys out: at the edges of tiles and units, split and whole pairs."""
    test_decode_attention(H, H, D, page, lens, 1.0)
    test_decode_attention(H, H, D, page, lens, 30.0)


@pytest.mark.parametrize("H,Hk", [(2, 2), (4, 2), (12, 1)])
def test_decode_a_spoilt_row_or_page_stays_where_it_is(H, Hk):
    """A NaN in a group of V spoils that group's outputs alone, one in K its head's; rows of a page that is not there count
    nothing, in every form of the kernel."""
    D, page, n = 128, 16, 75
    dl, ctx = context(H, D)
    rng = np.random.default_rng(H)
    kv = np.stack([bf(rng, n, 2 * Hk, D)] * 4)
    kv[1, 37, Hk, 3] = np.nan                                      # V, head 0, group 0
    kv[2, 20, Hk, 127] = np.inf                                    # V, head 0, group 1
    kv[3, 9, 0, 64] = np.nan                                       # K, head 0
    q, kt, vt = (np.repeat(bf(rng, 1, h, D), 4, 0) for h in (H, Hk, Hk))
    pg = books(dl, 4, 24, 6, page, [n] * 4, rng)
    pool = ctx.kv4_pool(pg, Hk)
    d = up(kv.reshape(4 * n, 2 * Hk, D))
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32(starts_of([n] * 4)))
    out = torch.zeros(4, H, D, dtype=torch.bfloat16, device=DEV)
    ctx.kv4_attn_decode(pg, pool, up(q), up(kt), up(vt), None, 0.1, out)
    assert ctx.device_status()[0] == 0
    o, G = wl.from_torch(out), H // Hk
    bad = np.zeros(o.shape, bool)
    bad[1, :G, :64] = bad[2, :G, 64:] = bad[3, :G] = True
    assert np.array_equal(np.isnan(o), bad)
    h, lifted = pk.held(kv[0]), lift(kv[0])
    ref = pk.attention_decode(q[0], kt[0], vt[0], h[:, :Hk], h[:, Hk:], 0.1)
    ref_abs = pk.attention_decode(q[0], kt[0], np.abs(vt[0]), h[:, :Hk], np.abs(h[:, Hk:]), 0.1)
    ref_lift = pk.attention_decode(q[0], kt[0], 0 * vt[0], h[:, :Hk], lifted[:, Hk:], 0.1)
    for b in range(4):
        close(np.where(bad[b], ref, o[b]), ref, ref_abs, f"sequence {b}", ref_lift)
    hole = int(pg.table[0, 2])
    pg.table[0, 2] = 24                                            # no such page
    ctx.kv4_attn_decode(pg, pool, up(q), up(kt), up(vt), None, 0.1, out)
    left = np.concatenate([kv[0, :32], kv[0, 48:]])
    h, lifted = pk.held(left), lift(left)
    ref = pk.attention_decode(q[0], kt[0], vt[0], h[:, :Hk], h[:, Hk:], 0.1)
    close(wl.from_torch(out)[0], ref, pk.attention_decode(q[0], kt[0], np.abs(vt[0]), h[:, :Hk], np.abs(h[:, Hk:]), 0.1), "hole",
          pk.attention_decode(q[0], kt[0], 0 * vt[0], h[:, :Hk], lifted[:, Hk:], 0.1))
    assert ctx.device_status() == (dl.DL_ERR_INVALID_ARG, 0) and 0 <= hole < 24
    ctx.close()


@pytest.mark.parametrize("H,Hk", [(16, 16), (64, 16)])
def test_decode_sums_over_long_rows_keep_their_bits(H, Hk):
    """100k rows of 16 heads, so that a warp adds up about 900 rows, with even weights, so that the output is a small mean of
    large codes.  The output's rounding is at most 2^-8 of it.  The roundings of P s are independent: 2^-11 of
    sqrt(sum p^2) rms(v - z).  About 56 additions into an accumulator, each cut off at 2^-23 of a sum that grows evenly:
    28 * 2^-23, below 2^-18, of sum p (v - z)."""
    D, page, n, head = 128, 128, 100_000, 5
    dl, ctx = context(H, D)
    gen = torch.Generator(device=DEV).manual_seed(3)
    rows = lambda *s: torch.randn(*s, generator=gen, device=DEV).bfloat16()
    k, v, q, kt, vt = rows(n, Hk, D), rows(n, Hk, D), rows(1, H, D) * 0.25, rows(1, Hk, D), rows(1, Hk, D)
    pg = dl.Pages(1, 800, 800, page, DEV)
    ctx.pages_reserve(pg, i32([n]))
    pool = ctx.kv4_pool(pg, Hk)
    ctx.kv4_append(pg, pool, k, v, i32([0, n]))
    out = torch.zeros(1, H, D, dtype=torch.bfloat16, device=DEV)
    ctx.kv4_attn_decode(pg, pool, q, kt, vt, None, D ** -0.5, out)
    G = H // Hk
    mine = slice(head * G, head * G + G)
    kh, vh = wl.from_torch(k[:, head]), wl.from_torch(v[:, head])
    kt, vt, q = wl.from_torch(kt[0, head]), wl.from_torch(vt[0, head]), wl.from_torch(q[0, mine])
    z = np.concatenate([pk.held(kh) @ q.T, (q @ kt)[None]]) * D ** -0.5
    p = np.exp(z - z.max(0))
    p /= p.sum(0)
    ref, spread = p.T @ np.concatenate([pk.held(vh), vt[None]]), p[:-1].T @ lift(vh)
    rms = lambda x: np.sqrt((x ** 2).mean())
    bound = EPS * rms(ref) + (2.0 ** -11 * np.sqrt((p ** 2).sum(0).max()) + 2.0 ** -18) * rms(spread)
    assert rms(wl.from_torch(out[0, mine]) - ref) <= bound
    assert ctx.device_status()[0] == 0
    ctx.close()


@pytest.mark.parametrize("H,Hk", [(16, 16), (64, 16)])
def test_decode_sums_do_not_shrink_with_the_number_of_rows(H, Hk):
    """4M rows of 16 heads, 40 times the same pages, so that a warp adds up about 36k rows.  The bounds are those above: a
    sum that is cut off is kept and begun anew after 32 units, 64 additions, 32 * 2^-23 = 2^-18 in all.  (The roundings of P s
    repeat with the rows: p as of one time.)"""
    D, page, n, head, times = 128, 128, 782 * 128, 5, 40
    dl, ctx = context(H, D)
    gen = torch.Generator(device=DEV).manual_seed(4)
    rows = lambda *s: torch.randn(*s, generator=gen, device=DEV).bfloat16()
    k, v, q, kt, vt = rows(n, Hk, D), rows(n, Hk, D), rows(1, H, D) * 0.25, rows(1, Hk, D), rows(1, Hk, D)
    pg = dl.Pages(1, 782, 782 * times, page, DEV)
    ctx.pages_reserve(pg, i32([n]))
    pool = ctx.kv4_pool(pg, Hk)
    ctx.kv4_append(pg, pool, k, v, i32([0, n]))
    pg.table.copy_(pg.table[:, :782].repeat(1, times))
    pg.cache_len.fill_(n * times)
    out = torch.zeros(1, H, D, dtype=torch.bfloat16, device=DEV)
    ctx.kv4_attn_decode(pg, pool, q, kt, vt, None, D ** -0.5, out)
    G = H // Hk
    mine = slice(head * G, head * G + G)
    kh, vh = pk.held(wl.from_torch(k[:, head])), wl.from_torch(v[:, head])
    kt, vt, q = wl.from_torch(kt[0, head]), wl.from_torch(vt[0, head]), wl.from_torch(q[0, mine])
    z = np.concatenate([kh @ q.T, (q @ kt)[None]]) * D ** -0.5
    p = np.exp(z - z.max(0))
    p[:-1] *= times
    p /= p.sum(0)
    ref, spread = p.T @ np.concatenate([pk.held(vh), vt[None]]), p[:-1].T @ lift(vh)
    rms = lambda x: np.sqrt((x ** 2).mean())
    bound = EPS * rms(ref) + (2.0 ** -11 * np.sqrt((p ** 2).sum(0).max()) + 2.0 ** -18) * rms(spread)
    assert rms(wl.from_torch(out[0, mine]) - ref) <= bound
    assert ctx.device_status()[0] == 0
    ctx.close()


def test_decode_leaves_out_rows_without_pages_and_reports_full_caches():
    H, Hk, D, page = 4, 2, 128, 16
    dl, ctx = context(H, D)
    rng = np.random.default_rng(9)
    lens = [40, 32, 48]
    st = starts_of(lens)
    kv = bf(rng, 120, 2 * Hk, D)
    pg = books(dl, 3, 10, 3, page, lens, rng)
    pool = ctx.kv4_pool(pg, Hk)
    d = up(kv)
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32(st))
    assert ctx.device_status()[0] == 0
    q, kt, vt = bf(rng, 3, H, D), bf(rng, 3, Hk, D), bf(rng, 3, Hk, D)
    out = torch.zeros(3, H, D, dtype=torch.bfloat16, device=DEV)
    keep = torch.tensor([0, 1, 1], dtype=torch.uint8, device=DEV)      # 1: its third page is not reserved; 2: full
    was = pool.clone()
    ctx.kv4_attn_decode(pg, pool, up(q), up(kt), up(vt), keep, 0.1, out)
    assert torch.equal(pool, was)
    code, detail = ctx.device_status()
    assert code == dl.DL_ERR_CAPACITY and detail in (1, 2)
    pg.table[0, 1] = -1                                            # rows 16..31 of sequence 0 are nowhere
    ctx.kv4_attn_decode(pg, pool, up(q), up(kt), up(vt), None, 0.1, out)
    left = np.concatenate([kv[:16], kv[32:40]])
    h, lifted = pk.held(left), lift(left)
    ref = pk.attention_decode(q[0], kt[0], vt[0], h[:, :Hk], h[:, Hk:], 0.1)
    close(wl.from_torch(out)[0], ref, pk.attention_decode(q[0], kt[0], np.abs(vt[0]), h[:, :Hk], np.abs(h[:, Hk:]), 0.1), "hole",
          pk.attention_decode(q[0], kt[0], 0 * vt[0], h[:, :Hk], lifted[:, Hk:], 0.1))
    assert ctx.device_status() == (dl.DL_ERR_INVALID_ARG, 0)
    ctx.close()


# ---- pages ----------------------------------------------------------------------------------------------------------
def random_books(dl, rng, B, page, width, n_pages, L, extra=True):
    """Books and pools in a random state (some reserved pages, some sequences sharing full pages), here and in the oracle."""
    order, at = list(rng.permutation(n_pages)), 0
    pages, length = [], []
    for b in range(B):
        n = int(rng.integers(0, (width - 1) * page + 1))
        row = []
        if b and rng.random() < 0.4:                                # shares the full pages of an earlier sequence
            src = int(rng.integers(0, b))
            full = min(length[src], n) // page
            row = pages[src][:full]
        c = -(-n // page) + (1 if extra and rng.random() < 0.3 else 0)
        take = max(0, c - len(row))
        row = row + [int(p) for p in order[at:at + take]]
        at += take
        pages.append(row)
        length.append(n)
    assert at <= n_pages
    pools = [torch.from_numpy(rng.integers(0, 256, (n_pages, 48), dtype=np.uint8)).to(DEV) for _ in range(L)]
    o = pk.Books(n_pages, page, width, pages, length, list(range(n_pages)))
    pg = dl.Pages(B, n_pages, width, page, DEV)
    pg.table.copy_(i32(o.table()))
    pg.refs.copy_(i32(o.refs()))
    pg.cache_len.copy_(i32(length))
    return o, pg, pools


def agree(o, pg, pools, was):
    assert np.array_equal(pg.table.cpu().numpy(), o.table())
    assert pg.refs.tolist() == o.refs() and pg.cache_len.tolist() == o.length
    for p, w in zip(pools, was):
        assert torch.equal(p, w[torch.tensor(o.data, device=DEV)])


@pytest.mark.parametrize("B,page,width,n_pages,L", [(1, 16, 2, 4, 1), (5, 16, 6, 40, 2), (9, 64, 4, 60, 3), (40, 32, 9, 1500, 70),
                                                    (3, 128, 3, 12, 0)])
def test_pages_random_histories(B, page, width, n_pages, L):
    dl, ctx = context(4, 64, B=B)
    rng = np.random.default_rng(B * 7 + n_pages)
    for trial in range(6):
        o, pg, pools = random_books(dl, rng, B, page, width, n_pages, L)
        was = [p.clone() for p in pools]
        for step in range(5):
            kind = rng.integers(0, 4)
            if kind == 0:
                parent = rng.integers(-1, B, B)
                parent = np.where(rng.random(B) < 0.5, np.arange(B), parent)
                ok = o.fork(parent.tolist())
                ctx.pages_fork(pg, i32(parent), pools)
            elif kind == 1:
                need = rng.integers(-5, 2 * page, B)
                ok = o.reserve(need.tolist())
                ctx.pages_reserve(pg, i32(need))
            elif kind == 2:
                gone = rng.random(B) < 0.3
                o.release(gone)
                ctx.pages_free(pg, torch.tensor(gone, dtype=torch.uint8, device=DEV))
                ok = True
            else:
                live = torch.zeros(1, dtype=torch.int32, device=DEV)
                n = o.compact()
                ctx.pages_compact(pg, pools, live)
                assert live.item() == n
                ok = True
            agree(o, pg, pools, was)
            assert ctx.device_status()[0] == (0 if ok else dl.DL_ERR_CAPACITY)
    ctx.close()


def test_fork_refuses_a_parent_out_of_range_and_an_empty_pool():
    dl, ctx = context(4, 64)
    pg = dl.Pages(4, 5, 3, 16, DEV)
    pg.cache_len.copy_(i32([20, 7, 0, 0]))
    pg.table.copy_(i32([[4, 1, -1], [0, -1, -1], [-1, -1, -1], [-1, -1, -1]]))
    pg.refs.copy_(i32([1, 1, 0, 0, 1]))
    pool = torch.arange(5, dtype=torch.uint8, device=DEV).repeat_interleave(32).view(5, 32).contiguous()
    ctx.pages_fork(pg, i32([0, 9, 0, -7]), [pool])                 # 1 and 3 stay, 2 becomes 0
    assert ctx.device_status()[0] == dl.DL_ERR_INVALID_ARG
    assert pg.table.tolist() == [[4, 1, -1], [0, -1, -1], [4, 2, -1], [-1, -1, -1]]
    assert pg.refs.tolist() == [1, 1, 1, 0, 2] and pg.cache_len.tolist() == [20, 7, 20, 0]
    assert pool[2, 0].item() == 1
    book = pg.book.clone()
    pg.refs[3] = 1
    ctx.pages_fork(pg, i32([0, 1, 2, 1]), [pool])                  # no page left for 1's last rows
    assert ctx.device_status() == (dl.DL_ERR_CAPACITY, -1)
    pg.refs[3] = 0
    assert torch.equal(pg.book, book)
    ctx.close()


# ---- refusals, streams, graphs --------------------------------------------------------------------------------------
def test_refusals():
    from paper_2412_00876_b200 import binding as dl
    H, D, B = 8, 64, 2
    _, ctx = context(H, D, B=B)
    bf16 = dict(dtype=torch.bfloat16, device=DEV)
    pg = dl.Pages(B, 4, 2, 16, DEV)
    pool = ctx.kv4_pool(pg, 2)
    q, k, out = torch.zeros(B, H, D, **bf16), torch.zeros(B, 2, D, **bf16), torch.zeros(B, H, D, **bf16)
    st = i32([0, 1, 2])

    def refused(code, f, *a):
        with pytest.raises(dl.DlError) as e:
            f(*a)
        assert e.value.code == code

    with pytest.raises(ValueError):
        ctx.kv4_attn_decode(pg, pool[:3], q, k, k, None, 0.1, out)          # a pool of other books
    with pytest.raises(ValueError):
        ctx.kv4_attn_decode(pg, pool, q.float(), k, k, None, 0.1, out)
    with pytest.raises(ValueError):
        ctx.kv4_attn_decode(pg, pool, q, k, k, None, 0.1, out[:1])
    with pytest.raises(ValueError):
        ctx.attn_prefill_packed(q.transpose(1, 2).contiguous().transpose(1, 2), k, k, st, 2, 0.1, out)
    with pytest.raises(ValueError):
        ctx.kv4_append(pg, pool, k, k.view(B, 2, D)[:, :, ::2], st)
    with pytest.raises(ValueError):
        ctx.pages_fork(pg, i32([0]), [pool])
    with pytest.raises(ValueError):
        ctx.pages_reserve(pg, torch.zeros(B, dtype=torch.int64, device=DEV))
    refused(dl.DL_ERR_INVALID_ARG, ctx.kv4_attn_decode, pg, pool, q, k, k, None, 0.0, out)
    k3 = torch.zeros(B, 3, D, **bf16)
    refused(dl.DL_ERR_INVALID_ARG, ctx.kv4_attn_decode, pg, ctx.kv4_pool(pg, 3), q, k3, k3, None, 0.1, out)      # 8 heads, 3 of K/V
    refused(dl.DL_ERR_INVALID_ARG, ctx.attn_prefill_packed, q, k3, k3, st, 2, 0.1, out)
    odd = torch.zeros(B * (H + 4) * D + 4, **bf16)[4:].view(B, H + 4, D)                  # 8 bytes off
    refused(dl.DL_ERR_ALIGNMENT, ctx.attn_prefill_packed, odd[:, :H], k, k, st, 2, 0.1, out)
    big = dl.Pages(B + 1, 4, 2, 16, DEV)
    z = torch.zeros(B + 1, H, D, **bf16)
    refused(dl.DL_ERR_WORKSPACE, ctx.kv4_attn_decode, big, ctx.kv4_pool(big, 2), z, z[:, :2].contiguous(), z[:, :2].contiguous(), None, 0.1, z.clone())
    p9 = dl.Pages(B, 4, 2, 9, DEV)
    refused(dl.DL_ERR_UNSUPPORTED, ctx.pages_free, p9, torch.zeros(B, dtype=torch.uint8, device=DEV))
    refused(dl.DL_ERR_ALIGNMENT, ctx.pages_fork, pg, i32([0, 1]), [torch.zeros(4, 24, dtype=torch.uint8, device=DEV)])
    wide = dl.Context(64, 32, D, 64, torch.bfloat16, 0, max_batch=B, cap=64)
    z = torch.zeros(B, 32, D, **bf16)
    refused(dl.DL_ERR_UNSUPPORTED, wide.kv4_attn_decode, pg, wide.kv4_pool(pg, 1), z, z[:, :1].contiguous(), z[:, :1].contiguous(), None, 0.1, z.clone())
    f32 = dl.Context(64, H, D, 64, torch.float32, 0, max_batch=B, cap=64)
    z = torch.zeros(B, H, D, device=DEV)
    refused(dl.DL_ERR_UNSUPPORTED, f32.attn_prefill_packed, z, z, z, st, 2, 0.1, z.clone())
    refused(dl.DL_ERR_UNSUPPORTED, f32.kv4_append, pg, f32.kv4_pool(pg, H), z, z, st)
    # nothing to do is fine
    ctx.attn_prefill_packed(q[:0], k[:0], k[:0], i32([0, 0, 0]), 0, 0.1, out[:0])
    ctx.kv4_append(pg, pool, k[:0], k[:0], i32([0, 0, 0]))
    assert ctx.device_status()[0] == 0
    for c in (ctx, wide, f32):
        c.close()


def test_a_serving_run_together_also_captured():
    """Prompts are attended, their kept rows appended, a request forked into beams, decode steps taken with reserved pages
    and kept tokens, one beam freed, the pool compacted, and another step taken; the same run from a captured graph (all of
    the device work of the decode step) on a side stream gives the same bits."""
    H, Hk, D, page, B = 8, 2, 128, 16, 4
    dl, ctx = context(H, D, B=B)
    rng = np.random.default_rng(11)
    lens = [50, 0, 33, 0]
    st, total = starts_of(lens), sum(lens)
    q, k, v = bf(rng, total, H, D), bf(rng, total, Hk, D), bf(rng, total, Hk, D)
    flags = (rng.random(total) < 0.6).astype(np.uint8)
    pg = dl.Pages(B, 40, 8, page, DEV)
    pool = ctx.kv4_pool(pg, Hk)
    out = torch.zeros(total, H, D, dtype=torch.bfloat16, device=DEV)
    ctx.attn_prefill_packed(up(q), up(k), up(v), i32(st), 50, D ** -0.5, out)
    ctx.pages_reserve(pg, i32(lens))
    ctx.kv4_append(pg, pool, up(k), up(v), i32(st), torch.from_numpy(flags).to(DEV))
    close(wl.from_torch(out), pk.attention_packed(q, k, v, st, D ** -0.5),
          pk.attention_packed(q, k, np.abs(v), st, D ** -0.5), "prompts")
    ctx.pages_fork(pg, i32([0, 0, 2, 0]), [pool])
    kept = {b: flags[st[b]:st[b + 1]] != 0 for b in (0, 2)}
    rows = {b: [list(k[st[s]:st[s + 1]][kept[s]]), list(v[st[s]:st[s + 1]][kept[s]])] for b, s in ((0, 0), (1, 0), (2, 2), (3, 0))}
    one = torch.ones(B, dtype=torch.int32, device=DEV)
    cap = pg.max_pages * page

    def step(dq, dk, dv, keep, o):
        ctx.pages_reserve(pg, one)
        ctx.kv4_attn_decode(pg, pool, dq, dk, dv, keep, D ** -0.5, o)
        ctx.commit_len(keep, pg.cache_len, cap)

    bufs = [torch.zeros(B, h, D, dtype=torch.bfloat16, device=DEV) for h in (H, Hk, Hk, H)]
    keep_d = torch.zeros(B, dtype=torch.uint8, device=DEV)
    graph = None
    alive = [0, 1, 2, 3]
    for t in range(40):
        qt, kt, vt = bf(rng, B, H, D), bf(rng, B, Hk, D), bf(rng, B, Hk, D)
        keep = (rng.random(B) < 0.6).astype(np.uint8)
        for d, x in zip(bufs, (qt, kt, vt)):
            d.copy_(up(x))
        keep_d.copy_(torch.from_numpy(keep))
        if t < 20:
            step(*bufs[:3], keep_d, bufs[3])
        else:
            if graph is None:
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    step(*bufs[:3], keep_d, bufs[3])
            graph.replay()
        got = wl.from_torch(bufs[3])
        for b in alive:
            kr, vr = (np.array(x, np.float32).reshape(len(x), Hk, D) for x in rows[b])
            hk_, hv_ = pk.held(kr), pk.held(vr)
            ref = pk.attention_decode(qt[b], kt[b], vt[b], hk_, hv_, D ** -0.5)
            close(got[b], ref, pk.attention_decode(qt[b], kt[b], np.abs(vt[b]), hk_, np.abs(hv_), D ** -0.5), f"step {t}, sequence {b}",
                  pk.attention_decode(qt[b], kt[b], 0 * vt[b], hk_, lift(vr), D ** -0.5))
            if keep[b]:
                rows[b][0].append(kt[b])
                rows[b][1].append(vt[b])
        if t == 10:
            ctx.pages_free(pg, torch.tensor([1, 0, 0, 0], dtype=torch.uint8, device=DEV))
            live = torch.zeros(1, dtype=torch.int32, device=DEV)
            ctx.pages_compact(pg, [pool], live)
            assert live.item() == int((pg.refs > 0).sum()) and int(pg.table.max()) == live.item() - 1
            alive = [1, 2, 3]
    assert [pg.cache_len[b].item() for b in alive] == [len(rows[b][0]) for b in alive]
    assert ctx.device_status()[0] == 0
    ctx.close()


# ---- paths that ordinary inputs do not take -------------------------------------------------------------------------
@pytest.mark.parametrize("D,Hk", [(128, 2), (64, 1)])
@pytest.mark.parametrize("where", [10, 70, 130, 200, 300, 700])
@pytest.mark.parametrize("lead", [12.0, 60.0, 3000.0])
def test_packed_scores_that_pass_the_maximum_by_far(D, Hk, where, lead):
    """From key `where` on the scores stand `lead` (base e) above all earlier ones, then fall back: whatever an item's first
    tile took for its maximum is wrong by far in the first half, the second half or an edge tile of a later one."""
    H, lens = 2, [900]
    dl, ctx = context(H, D)
    rng = np.random.default_rng(where + D)
    q, k, v = bf(rng, 900, H, D, scale=0.1), bf(rng, 900, Hk, D, scale=0.1), bf(rng, 900, Hk, D)
    q[:, :, 0] = 1.0
    k[:, :, 0] = 0.0
    k[where:where + 90:9, :, 0] = wl.round_to_storage(np.float32([lead]), "bf16")[0]
    k[where + 45, :, 0] = wl.round_to_storage(np.float32([lead * 1.25]), "bf16")[0]
    out = torch.zeros((900, H, D), dtype=torch.bfloat16, device=DEV)
    ctx.attn_prefill_packed(up(q), up(k), up(v), i32(starts_of(lens)), 900, 1.0, out)
    rows = np.unique(np.concatenate([np.arange(max(0, where - 2), min(900, where + 60)), np.arange(0, 900, 61), [899]]))
    ref, ref_abs = np.zeros((len(rows), H, D)), np.zeros((len(rows), H, D))
    for n, r in enumerate(rows):
        args = [np.asarray(t, np.float64) for t in (q[r], k[r], v[r], k[:r], v[:r])]
        ref[n] = pk.attention_decode(*args, 1.0)
        args[2], args[4] = np.abs(args[2]), np.abs(args[4])
        ref_abs[n] = pk.attention_decode(*args, 1.0)
    close(wl.from_torch(out)[rows], ref, ref_abs, "leading scores")
    assert ctx.device_status()[0] == 0
    ctx.close()


@pytest.mark.parametrize("B,H,Hk,D,lo,hi", [(40, 16, 16, 64, 20, 30), (74, 8, 8, 128, 250, 300), (40, 32, 8, 64, 60, 70)])
def test_packed_batches_of_like_lengths(B, H, Hk, D, lo, hi):
    """Enough (sequence, head) columns of like lengths that CTAs take them one at a time; sampled sequences."""
    dl, ctx = context(H, D, B=B)
    rng = np.random.default_rng(B + D)
    lens = rng.integers(lo, hi + 1, B).tolist()
    st, total = starts_of(lens), sum(lens)
    q, k, v = bf(rng, total, H, D), bf(rng, total, Hk, D), bf(rng, total, Hk, D)
    out = torch.full((total, H, D), 9.0, dtype=torch.bfloat16, device=DEV)
    ctx.attn_prefill_packed(up(q), up(k), up(v), i32(st), max(lens), D ** -0.5, out)
    got = wl.from_torch(out)
    assert not np.any(got == 9.0)
    for b in sorted({0, 1, B // 2, B - 2, B - 1}):
        a, e = st[b], st[b + 1]
        for h in (0, H - 1):
            sl = lambda t, i: t[a:e, i:i + 1]
            args = sl(q, h), sl(k, h // (H // Hk)), sl(v, h // (H // Hk))
            ref = pk.attention_packed(*args, [0, e - a], D ** -0.5)
            close(got[a:e, h:h + 1], ref, pk.attention_packed(args[0], args[1], np.abs(args[2]), [0, e - a], D ** -0.5), f"sequence {b}, head {h}")
    assert ctx.device_status()[0] == 0
    ctx.close()


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GB: its last pages hold, read, attend, fork and compact as its first do."""
    H = Hk = 8
    D, page = 128, 128
    dl, ctx = context(H, D)
    rng = np.random.default_rng(21)
    page_bytes = Hk * page * 144
    n_pages = (1 << 32) // page_bytes + 600
    lens = [300, 260]
    pg = dl.Pages(2, n_pages, 4, page, DEV)
    pool = torch.empty(n_pages, page_bytes, dtype=torch.uint8, device=DEV)
    pg.table[0, :3] = i32([n_pages - 1, 5, n_pages - 400])
    pg.table[1, :3] = i32([n_pages - 7, n_pages - 2, 0])
    for p in pg.table[:, :3].flatten().tolist():
        pg.refs[p] = 1
    st = starts_of(lens)
    kv = bf(rng, sum(lens), 2 * Hk, D)
    d = up(kv)
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32(st))
    q, kt, vt = bf(rng, 2, H, D), bf(rng, 2, Hk, D), bf(rng, 2, Hk, D)
    h, lifted = pk.held(kv), lift(kv)

    def check():
        gk, gv = read(ctx, pg, pool, Hk, D, [0, 0], lens)
        same_values(gk, h[:, :Hk], "K")
        same_values(gv, h[:, Hk:], "V")
        out = torch.zeros(2, H, D, dtype=torch.bfloat16, device=DEV)
        ctx.kv4_attn_decode(pg, pool, up(q), up(kt), up(vt), None, D ** -0.5, out)
        for b in range(2):
            r = slice(st[b], st[b + 1])
            args = q[b], kt[b], vt[b], h[r, :Hk], h[r, Hk:]
            close(wl.from_torch(out)[b], pk.attention_decode(*args, D ** -0.5),
                  pk.attention_decode(q[b], kt[b], np.abs(vt[b]), h[r, :Hk], np.abs(h[r, Hk:]), D ** -0.5), f"sequence {b}",
                  pk.attention_decode(q[b], kt[b], 0 * vt[b], h[r, :Hk], lifted[r, Hk:], D ** -0.5))

    check()
    live = torch.zeros(1, dtype=torch.int32, device=DEV)
    ctx.pages_compact(pg, [pool], live)
    assert live.item() == 6 and int(pg.table.max()) == 5
    check()
    ctx.pages_fork(pg, i32([0, 0]), [pool])
    pg.cache_len.copy_(i32([300, 300]))
    gk, _ = read(ctx, pg, pool, Hk, D, [0, 0], [300, 300])
    same_values(gk[300:], h[:300, :Hk], "forked K")
    assert ctx.device_status()[0] == 0
    ctx.close()


def test_another_stream_and_graphs_that_share_a_context():
    """Calls given a stream run on it; two graphs captured with one context, replayed in turn, give what the calls give."""
    H, Hk, D, page = 8, 2, 64, 16
    dl, ctx = context(H, D)
    rng = np.random.default_rng(31)
    lens = [700, 90]
    st = starts_of(lens)
    kv = bf(rng, sum(lens), 2 * Hk, D)
    pg = books(dl, 2, 60, 45, page, lens, rng)
    pool = ctx.kv4_pool(pg, Hk)
    d, q, kt, vt = up(kv), up(bf(rng, 2, H, D)), up(bf(rng, 2, Hk, D)), up(bf(rng, 2, Hk, D))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.zeros(2, H, D, dtype=torch.bfloat16, device=DEV)
    ctx.kv4_append(pg, pool, d[:, :Hk], d[:, Hk:], i32(st), stream=s)
    ctx.kv4_attn_decode(pg, pool, q, kt, vt, None, 0.1, out, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    ref = out.clone()
    q2 = up(bf(rng, 2, H, D))
    out2 = torch.zeros_like(out)
    ctx.kv4_attn_decode(pg, pool, q2, kt, vt, None, 0.1, out2)
    ref2 = out2.clone()
    graphs = []
    for a, o in ((q, out), (q2, out2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            ctx.kv4_attn_decode(pg, pool, a, kt, vt, None, 0.1, o)
        graphs.append(g)
    for _ in range(3):
        out.zero_()
        out2.zero_()
        for g in graphs:
            g.replay()
        assert torch.equal(out, ref) and torch.equal(out2, ref2)
    assert ctx.device_status()[0] == 0
    ctx.close()


def test_clean_under_the_checked_build():
    """The library with -DDL_BOUNDS=1 compares every computed store with its buffer: none of these may lie outside."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    env = dict(os.environ, DL_SPARSE_CHECKED="1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", os.path.abspath(__file__), "-k",
                        "test_packed_prompts or test_append or test_decode or test_pages or together"],
                       capture_output=True, text=True, env=env, cwd=root, timeout=900)
    assert r.returncode == 0 and " passed" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
