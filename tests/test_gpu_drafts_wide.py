"""Appending rows of many heads to the paged 16-bit cache (not in the paper): values that are moved bit for bit, rotated ones within the
bound of tests/test_gpu_drafts.py."""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from paper_2412_00876_b200 import workloads as wl
from tests.test_gpu_drafts import DEV, HALF, bf, books, context, i32, starts_of, u8, up


def units_of(row, heads_units):
    """how the kernel takes index `row` apart: the product with 2^32 / units, rounded up"""
    inverse = ((1 << 32) + heads_units - 1) // heads_units
    return (row * inverse) >> 32


def test_rows_of_the_widest_call_are_told_apart():
    """Units of 32 bytes of up to four rows, at every border between rows, for all widths that a call may have."""
    for units in list(range(4, 4000)) + list(range(32768 - 3000, 32768)):
        for row in range(4):
            assert units_of(row * units, units) == row and units_of((row + 1) * units - 1, units) == row
        assert (4 * units - 1) * (units - 1) < 1 << 32                 # why: the inverse is too large by less than units / 2^32


@pytest.mark.gpu
@pytest.mark.parametrize("H,Hk,D,lens", [(96, 96, 128, [5, 0, 30]), (256, 256, 64, [1, 3]), (512, 64, 128, [700, 40]), (1000, 1000, 128, [3, 2])])
@pytest.mark.parametrize("masked", [False, True])
def test_append_of_many_heads(H, Hk, D, lens, masked):
    dl, ctx = context(H, D, B=4)
    rng = np.random.default_rng(H + D)
    st, total, page = starts_of(lens), sum(lens), 16
    held = [3] * len(lens)
    flags = (rng.random(total) < 0.6).astype(np.uint8) if masked else np.ones(total, np.uint8)
    kept = [int(flags[a:e].sum()) for a, e in zip(st, st[1:])]
    pages, table = books(dl, rng, [h + k for h, k in zip(held, kept)], held, page)
    rope = dl.Rope(D, device=DEV)
    x, pos = bf(rng, total, H + 2 * Hk, D), np.arange(total) * 7
    pool, qkv = ctx.kv16_pool(pages, Hk), up(x)
    q_out = torch.zeros(total, H, D, dtype=torch.bfloat16, device=DEV)
    ctx.kv16_append(pages, pool, qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], i32(st), i32(pos), rope, keep=u8(flags) if masked else None,
                    q_out=q_out, commit=True)
    assert ctx.device_status()[0] == 0 and pages.cache_len.tolist() == [h + k for h, k in zip(held, kept)]
    freqs = rope.freqs.cpu().numpy()
    want = od.turned(x[:, :H + Hk], pos, freqs, False)
    half = D // 2
    size = np.abs(x[:, :H + Hk].astype(np.float64))
    pair = size[..., :half] + size[..., half:]
    bound = HALF * np.abs(want) + 2.0 ** -21 * np.concatenate([pair, pair], -1)
    assert (np.abs(wl.from_torch(q_out) - want[:, :H]) <= bound[:, :H]).all()
    host = wl.from_torch(pool)
    for b, (a, e) in enumerate(zip(st, st[1:])):
        for t, r in enumerate(a + np.flatnonzero(flags[a:e]), held[b]):
            k, v = host[table[b, t // page], :, :, t % page]
            assert (np.abs(k - want[r, H:]) <= bound[r, H:]).all() and np.array_equal(v, x[r, H + Hk:])
    ctx.close()


@pytest.mark.gpu
def test_rows_wider_than_a_call_takes_are_refused():
    dl, ctx = context(2048, 128, B=1)
    pages = dl.Pages(1, 1, 1, 16, DEV)
    pool = ctx.kv16_pool(pages, 2048)
    x = torch.zeros(1, 2048, 128, dtype=torch.bfloat16, device=DEV)
    args = (i32([0, 1]), None, None)
    for call in (lambda: ctx.kv16_append(pages, pool, x, x, x, *args, q_out=x), lambda: ctx.kv16_append(pages, pool, None, x, x, *args),
                 lambda: ctx.kv16_append(None, None, x, x, None, None, None, None, q_out=x, k_out=x)):
        with pytest.raises(dl.DlError) as e:
            call()
        assert e.value.code == dl.DL_ERR_UNSUPPORTED
    ctx.kv16_append(None, None, None, x, None, None, None, None, k_out=x)                  # the rotation of k alone is half as wide
    assert ctx.device_status()[0] == 0
    ctx.close()


@pytest.mark.gpu
def test_append_of_the_widest_rows_several_a_block():
    """Nearly 2^19 values a row and enough rows that a block takes four of them: without rotation everything is moved bit for bit."""
    H, D, total, page = 1360, 128, 2400, 128
    dl, ctx = context(H, D, B=1)
    pages = dl.Pages(1, 20, 20, page, DEV)
    ctx.pages_reserve(pages, i32([total]))
    pool, x = ctx.kv16_pool(pages, H), torch.randn(total, 3 * H, D, dtype=torch.bfloat16, device=DEV)
    q_out, k_out = (torch.zeros(total, H, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.kv16_append(pages, pool, x[:, :H], x[:, H:2 * H], x[:, 2 * H:], i32([0, total]), None, None, q_out=q_out, k_out=k_out)
    assert ctx.device_status()[0] == 0 and torch.equal(q_out, x[:, :H]) and torch.equal(k_out, x[:, H:2 * H])
    rows = pool[pages.table[0, :-(-total // page)].long()].transpose(2, 3).transpose(1, 2).flatten(0, 1)[:total]
    assert torch.equal(rows[:, 0], x[:, H:2 * H]) and torch.equal(rows[:, 1], x[:, 2 * H:])
    ctx.close()
