"""GPU parity of the drafted-token calls (not in the paper) against oracle/drafts.py: append with the position rotation, tree
masks, attention of tree nodes over the paged 16-bit cache, verification, accepted rows, and a run of them together.

Tolerances.  Masks, positions, decisions, tokens, lengths and rows that are only moved are compared exactly.
Rotation: the angle's fraction of a half turn is rounded to fp32 (2^-25 at most, times pi: 2^-23.3), sine and cosine are good to
2 ulp (2^-23), the amplitude and each of two products and their sum round once (2^-24 each): a value x c - y s is off by
at most (2^-23.3 + 2^-23 + 3 * 2^-24) amplitude (|x| + |y|) < 2^-21 amplitude (|x| + |y|), and by its rounding to bf16, 2^-8 of
itself (half of torch.finfo(bfloat16).eps).
Attention: every probability is rounded to bf16 before it multiplies a value: at most 2^-8 * A, A = sum p |v| / sum p; the output's
own rounding 2^-8 |out|; fp32 scores are off by D 2^-24 sum |q k| scale (below 2^-13 here, sums of 128 terms of which few exceed
1) and exponentials by 2^-13, together 2^-12 A; fp32 sums over n keys by n 2^-24 A.  Joined parts round once more in fp32."""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from paper_2412_00876_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)
HALF = torch.finfo(torch.bfloat16).eps / 2


def bf(rng, *shape, scale=1.0):
    return wl.round_to_storage(rng.normal(0, scale, shape).astype(np.float32), "bf16")


def up(x):
    return wl.to_torch(x, "bf16", DEV)


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def u8(x):
    return torch.tensor(np.asarray(x), dtype=torch.uint8, device=DEV)


def starts_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def context(H, D, B=8, **kw):
    from paper_2412_00876_b200 import binding as dl
    return dl, dl.Context(64, H, D, 64, torch.bfloat16, 0, max_batch=B, cap=64, **kw)


def books(dl, rng, rows, held, page, spare=2, cols=1):
    """Books in which sequence b has the pages of rows[b] rows, at random places, and holds held[b] rows."""
    counts = [-(-n // page) for n in rows]
    n_pages, width = sum(counts) + spare, max(max(counts), 1) + cols
    pages = dl.Pages(len(rows), n_pages, width, page, DEV)
    order, table, at = rng.permutation(n_pages), np.full((len(rows), width), -1, np.int32), 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    pages.table.copy_(i32(table))
    pages.refs.copy_(i32(np.bincount(table[table >= 0], minlength=n_pages)))
    pages.cache_len.copy_(i32(held))
    return pages, table


def cache_rows(pool, table, b, n, page):
    """K and V [n][Hk][D] of sequence b's first n rows, float64 (NaN where there is no page)"""
    kv = np.full((2, n, pool.shape[2], pool.shape[4]), np.nan)
    for t in range(n):
        p = table[b, t // page] if t // page < table.shape[1] else -1
        if 0 <= p < pool.shape[0]:
            kv[:, t] = pool[p, :, :, t % page]
    return kv


def random_tree(rng, n, chain=False):
    return [-1] + [i - 1 if chain else int(rng.integers(max(0, i - 6), i)) for i in range(1, n)]


# ---- rotation and append --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hk,D,rot,inter,page,lens,far,amplitude", [
    (4, 4, 128, 128, False, 64, [5], 0, 1.0), (4, 2, 64, 64, True, 16, [1, 17, 0, 33], 1000, 1.0),
    (8, 1, 128, 64, False, 32, [3, 64, 65], 1000000, 1.25), (6, 3, 64, 32, False, 128, [130, 1], 2 ** 31 - 200, 1.0),
    (16, 2, 128, 16, True, 16, [15, 16, 31], 70000, 0.5), (5, 5, 64, 0, False, 32, [40, 2], 10, 1.0),
    (32, 8, 128, 96, True, 64, [200, 1, 300], 131072, 1.0), (40, 1, 128, 112, False, 16, [700] * 9, 5000, 1.0)])
@pytest.mark.parametrize("keep", ["none", "some"])
def test_append(H, Hk, D, rot, inter, page, lens, far, amplitude, keep):
    dl, ctx = context(H, D, B=16)
    rng = np.random.default_rng(H * 100 + D + rot + len(lens))
    st, total, gap = starts_of(lens), sum(lens), 3
    held = rng.integers(0, 40, len(lens))
    freqs = rng.random(rot // 2) * np.logspace(0, -5, max(rot // 2, 1))[:rot // 2]
    rope = dl.Rope(rot, interleaved=inter, freqs=freqs, amplitude=amplitude, device=DEV)
    x = bf(rng, total + gap, H + 2 * Hk, D)
    pos = np.concatenate([far + np.arange(n) for n in lens] + [np.arange(gap)]) - (50 if far < 1000 else 0)
    flags = rng.integers(0, 2, total + gap).astype(np.uint8) * 3 if keep == "some" else np.ones(total + gap, np.uint8)
    kept = [int((flags[a:e] != 0).sum()) for a, e in zip(st, st[1:])]
    pages, table = books(dl, rng, held + kept, held, page)
    pool = up(bf(rng, pages.n_pages, 2, Hk, page, D))
    before, qkv = pool.clone(), up(x)
    q_out = torch.full((total + gap, H, D), 7.0, dtype=torch.bfloat16, device=DEV)
    k_out = torch.full((total + gap, Hk + 1, D), 7.0, dtype=torch.bfloat16, device=DEV)         # strided rows
    ctx.kv16_append(pages, pool, qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], i32(st), i32(pos), rope,
                    keep=u8(flags) if keep == "some" else None, q_out=q_out, k_out=k_out[:, :Hk], commit=True)
    assert ctx.device_status()[0] == 0
    assert pages.cache_len.tolist() == [int(h) + k for h, k in zip(held, kept)]
    want = od.turned(x[:total, :H + Hk], pos[:total], freqs, inter, amplitude)
    size = np.abs(x[:total, :H + Hk].astype(np.float64))
    pair = od.turned(np.zeros_like(size), pos[:total], freqs, inter)           # |x| + |y| of every pair
    half = rot // 2
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if inter else (i, i + half)
        pair[..., a] = pair[..., b] = size[..., a] + size[..., b]
    bound = HALF * np.abs(want) + 2.0 ** -21 * amplitude * pair
    got = np.concatenate([wl.from_torch(q_out)[:total], wl.from_torch(k_out)[:total, :Hk]], 1)
    assert (np.abs(got - want) <= bound).all(), np.abs(got - want).max()
    assert np.array_equal(got[..., rot:], x[:total, :H + Hk, rot:])            # what does not turn is moved bit for bit
    assert (q_out[total:] == 7).all() and (k_out[total:] == 7).all() and (k_out[:, Hk:] == 7).all()
    # the cache: rotated keys as in k_out, values bit for bit, every other row as it was
    ref = before.clone()
    for b, (a, e) in enumerate(zip(st, st[1:])):
        t = int(held[b])
        for r in range(a, e):
            if flags[r]:
                ref[table[b, t // page], 0, :, t % page] = k_out[r, :Hk]
                ref[table[b, t // page], 1, :, t % page] = qkv[r, H + Hk:]
                t += 1
    assert torch.equal(ref, pool)
    # without commit lengths stay; in place and without a cache the same rows come out
    pages.cache_len.copy_(i32(held))
    pool.copy_(before)
    ctx.kv16_append(pages, pool, None, qkv[:, H:H + Hk], qkv[:, H + Hk:], i32(st), i32(pos), rope, keep=u8(flags), commit=False)
    assert torch.equal(ref, pool) and pages.cache_len.tolist() == list(held)
    alone = qkv.clone()
    ctx.kv16_append(None, None, alone[:, :H], alone[:, H:H + Hk], None, None, i32(pos), rope, q_out=alone[:, :H], k_out=alone[:, H:H + Hk])
    assert torch.equal(alone[:total, :H], q_out[:total]) and torch.equal(alone[:total, H:H + Hk], k_out[:total, :Hk])
    assert torch.equal(alone[:, H + Hk:], qkv[:, H + Hk:])
    ctx.close()


def test_append_of_long_masked_sequences():
    """Flags counted 16 at a time from any alignment, over sequences of thousands of rows."""
    dl, ctx = context(2, 64)
    rng = np.random.default_rng(3)
    lens, page = [5, 9001, 0, 4099], 128
    st, total = starts_of(lens), sum(lens)
    flags = (rng.random(total) < 0.3).astype(np.uint8) * 255
    kept = [int((flags[a:e] != 0).sum()) for a, e in zip(st, st[1:])]
    pages, table = books(dl, rng, kept, [0] * 4, page)
    pool, kv = ctx.kv16_pool(pages, 1), up(bf(rng, total, 2, 64))
    shifted = torch.zeros(total + 16, dtype=torch.uint8, device=DEV)
    for off in (0, 1, 7, 15):
        pages.cache_len.zero_()
        pool.zero_()
        shifted[off:off + total] = u8(flags)
        ctx.kv16_append(pages, pool, None, kv[:, :1], kv[:, 1:], i32(st), None, None, keep=shifted[off:off + total])
        for b, (a, e) in enumerate(zip(st, st[1:])):
            rows = kv[a:e][torch.from_numpy(flags[a:e] != 0).to(DEV)].cpu()
            got = cache_rows(wl.from_torch(pool), table, b, kept[b], page)
            assert np.array_equal(np.moveaxis(got, 0, 1)[:, :, 0], wl.from_torch(rows.to(DEV)).reshape(kept[b], 2, 64))
    ctx.close()


def test_append_leaves_a_sequence_that_lacks_pages():
    dl, ctx = context(4, 64)
    rng = np.random.default_rng(4)
    lens, held, page = [20, 5, 30], [3, 0, 2], 16
    st, total = starts_of(lens), sum(lens)
    for with_plan in (False, True):
        pages, table = books(dl, rng, [23, 5, 16], held, page)                # the last lacks its second page
        pool, x = ctx.kv16_pool(pages, 2), up(bf(rng, total, 8, 64))
        rope = dl.Rope(64, device=DEV)
        q_out = torch.zeros(total, 4, 64, dtype=torch.bfloat16, device=DEV)
        ctx.kv16_append(pages, pool, x[:, :4], x[:, 4:6], x[:, 6:], i32(st), i32(np.arange(total)), rope, q_out=q_out, commit=with_plan)
        assert ctx.device_status() == (dl.DL_ERR_CAPACITY, 2)
        assert pages.cache_len.tolist() == ([23, 5, 2] if with_plan else held)
        assert (pool[table[2, 0]] == 0).all() and (pool[table[1, 0], :, :, :5] != 0).any() and (q_out[-1] != 0).any()
    ctx.close()


# ---- trees ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("lens,words", [([1], 1), ([5, 0, 32, 31], 1), ([33, 64, 1], 2), ([700, 3], 22), ([2048], 64)])
def test_tree_plan(lens, words):
    dl, ctx = context(2, 64)
    rng = np.random.default_rng(sum(lens))
    parents = [random_tree(rng, n) if n else [] for n in lens]
    pos0 = rng.integers(0, 100000, len(lens))
    total = sum(lens)
    mask = torch.full((total + 2, words), 5, dtype=torch.int32, device=DEV)
    pos = torch.full((total + 2,), 5, dtype=torch.int32, device=DEV)
    parent = i32(np.concatenate([p for p in parents if p] + [[9, 9]]))
    ctx.tree_plan(parent, i32(starts_of(lens)), i32(pos0), mask, pos)
    m, p = od.tree_plan([q for q in parents if q], [f for f, n in zip(pos0, lens) if n], words)
    assert np.array_equal(mask[:total].cpu().numpy().view(np.uint32), m) and np.array_equal(pos[:total].cpu().numpy(), p)
    assert (mask[total:] == 5).all() and (pos[total:] == 5).all() and ctx.device_status()[0] == 0
    ctx.tree_plan(parent, i32(starts_of(lens)), None, mask)
    assert np.array_equal(mask[:total].cpu().numpy().view(np.uint32), m)
    ctx.close()


def test_tree_plan_reports_bad_parents_and_too_many_nodes():
    dl, ctx = context(2, 64)
    mask, pos = (torch.zeros(*s, dtype=torch.int32, device=DEV) for s in ((40, 1), (40,)))
    for parent, lens, bad, want in [([-1, 1, 0], [3], 0, [1, 2, 5]), ([-1, 0, -1, 7], [2, 2], 1, [1, 3, 1, 2]), ([-1, -2], [2], 0, [1, 2])]:
        n = len(parent)
        ctx.tree_plan(i32(parent), i32(starts_of(lens)), None, mask[:n], pos[:n])
        assert ctx.device_status() == (dl.DL_ERR_INVALID_ARG, bad) and mask[:n, 0].tolist() == want
    mask.fill_(9)
    ctx.tree_plan(i32([-1] + list(range(39))), i32([0, 40]), None, mask, pos)
    assert ctx.device_status() == (dl.DL_ERR_INVALID_ARG, 0)
    assert mask[31, 0] == -1 and (mask[32:] == 9).all()
    ctx.close()


# ---- attention ------------------------------------------------------------------------------------------------------
def check_attention(H, Hk, D, page, held, nodes, masked, seed=0, extra_rows=0, q_scale=1.0, pool_edit=None, table_edit=None, status=None):
    dl, ctx = context(H, D, B=64)
    rng = np.random.default_rng(seed + H + D + sum(held) + sum(nodes))
    st, total, gap = starts_of(nodes), sum(nodes), 2
    pages, table = books(dl, rng, [h + n for h, n in zip(held, nodes)], held, page)
    pool = bf(rng, pages.n_pages, 2, Hk, page, D)
    pool[:, 0, :, :, : D // 8] *= 2.0
    dev_pool = up(pool)
    # rows behind a sequence's last and pages of nobody hold NaN and infinities
    used = np.zeros(pool.shape[:1] + (page,), bool)
    for b, n in enumerate(h + n for h, n in zip(held, nodes)):
        for t in range(n):
            used[table[b, t // page], t % page] = True
    for p, r in np.argwhere(~used):
        dev_pool[p, 0, :, r] = float("nan")
        dev_pool[p, 1, :, r] = float("inf") if r % 2 else float("nan")
    if pool_edit is not None:
        pool_edit(pool, dev_pool, table)
    if table_edit is not None:
        table_edit(table)
        pages.table.copy_(i32(table))
    q = bf(rng, total + gap, H, D, scale=q_scale)
    words = -(-max(nodes) // 32)
    mask = None
    if masked == "tree":
        mask, _ = od.tree_plan([random_tree(rng, n) for n in nodes if n], [0] * len(nodes), words)
    elif masked == "random":
        mask = rng.integers(0, 2 ** 32, (total, words), dtype=np.uint64).astype(np.uint32)
        mask[rng.random(total) < 0.3] = 0                                     # rows that see none of the nodes
    wide = torch.zeros(total + gap, H + 1, D, dtype=torch.bfloat16, device=DEV)
    wide[:, :H] = up(q)                                                        # strided rows
    out = torch.full((total + gap, H, D), 7.0, dtype=torch.bfloat16, device=DEV)
    dev_mask = None
    if mask is not None:
        dev_mask = i32(np.concatenate([mask.view(np.int32), np.full((gap, words), -1, np.int32)]))
    scale = D ** -0.5
    ctx.kv16_attn_tree(pages, dev_pool, wide[:, :H], i32(st), max(nodes) + extra_rows, dev_mask, scale, out)
    code, detail = ctx.device_status()
    assert (code, detail) == status if status else code == 0, (code, detail)
    got = wl.from_torch(out).astype(np.float64)
    assert (got[total:] == 7).all()
    for b, (a, e) in enumerate(zip(st, st[1:])):
        k, v = cache_rows(pool, table, b, held[b] + nodes[b], page)
        m = None if mask is None else mask[a:e]
        ref = od.attention_tree(q[a:e], k, v, held[b], m, scale)
        size = od.attention_tree(q[a:e], k, np.abs(v), held[b], m, scale)
        bound = HALF * (size + np.abs(ref)) + (2.0 ** -12 + (held[b] + nodes[b]) * 2.0 ** -24) * size
        bad = ~(np.abs(got[a:e] - ref) <= bound)
        assert not bad.any(), f"sequence {b}: {bad.sum()} off, worst {np.abs(got[a:e] - ref)[bad].max()} at {np.argwhere(bad)[:4]}"
    out2 = torch.zeros_like(out)
    ctx.kv16_attn_tree(pages, dev_pool, up(q), i32(st), max(nodes) + extra_rows, dev_mask, scale, out2)
    assert torch.equal(out[:total], out2[:total])                              # dense rows, and the same bits again
    ctx.close()


@pytest.mark.parametrize("H,Hk,D,page,held,nodes", [
    (4, 4, 128, 64, [0], [1]), (4, 4, 64, 16, [0, 1, 15], [1, 1, 1]), (16, 4, 64, 16, [300, 77], [1, 8]),
    (8, 1, 128, 32, [127, 128, 129, 0], [5, 16, 1, 17]), (6, 2, 128, 128, [255, 256, 257], [3, 1, 43]),
    (7, 1, 64, 64, [500, 3], [18, 19]), (5, 5, 128, 16, [64, 63, 65, 1], [32, 33, 31, 64]), (32, 2, 128, 64, [700, 20], [9, 8]),
    (16, 1, 64, 32, [1000, 0, 50], [20, 0, 4]), (12, 1, 128, 16, [90, 300], [11, 30]), (2, 2, 64, 128, [10, 900], [130, 90]),
    (128, 1, 64, 16, [33], [2]), (4, 1, 128, 64, [2100, 40], [40, 64])])
@pytest.mark.parametrize("masked", ["tree", "random", "chain"])
def test_attention(H, Hk, D, page, held, nodes, masked):
    check_attention(H, Hk, D, page, held, nodes, None if masked == "chain" else masked, extra_rows=0 if masked != "chain" else 50)


@pytest.mark.parametrize("H,Hk,D,page,held,nodes", [
    (8, 2, 128, 64, [200], [300]), (4, 1, 64, 16, [0, 90], [257, 130]), (3, 1, 128, 32, [127], [140]), (2, 2, 128, 128, [0, 5], [400, 256])])
def test_attention_of_chunks(H, Hk, D, page, held, nodes):
    check_attention(H, Hk, D, page, held, nodes, None)


@pytest.mark.parametrize("B", [1, 3, 40])
def test_attention_of_many_and_few_sequences(B):
    rng = np.random.default_rng(B)
    held = [int(x) for x in rng.integers(0, 4000 // B, B)]
    check_attention(8, 2, 128, 32, held, [int(x) for x in rng.integers(0, 9, B - 1)] + [4], "tree")


def test_attention_with_leading_scores():
    """Large queries: a few keys take nearly all of the weight, in any tile."""
    check_attention(4, 2, 128, 64, [600, 130], [7, 40], "tree", q_scale=6.0)
    check_attention(4, 2, 64, 16, [900], [3], None, q_scale=30.0)


def test_attention_leaves_out_rows_without_pages():
    def edit(table):
        table[0, 1] = -1
        table[0, 4] = 10 ** 6
    check_attention(8, 2, 128, 64, [600, 130], [7, 3], "tree", table_edit=edit, status=(-1, 0))


def test_attention_reports_more_nodes_than_said():
    dl, ctx = context(4, 64)
    rng = np.random.default_rng(5)
    pages, table = books(dl, rng, [50, 50], [40, 40], 16)
    pool, q = up(bf(rng, pages.n_pages, 2, 2, 16, 64)), up(bf(rng, 14, 4, 64))
    full, cut = torch.zeros_like(q), torch.full_like(q, 7.0)
    ctx.kv16_attn_tree(pages, pool, q, i32([0, 10, 14]), 10, None, 0.1, full)
    assert ctx.device_status()[0] == 0
    ctx.kv16_attn_tree(pages, pool, q, i32([0, 10, 14]), 6, None, 0.1, cut)
    assert ctx.device_status() == (dl.DL_ERR_INVALID_ARG, 0)
    assert torch.equal(cut[:6], full[:6]) and (cut[6:10] == 7).all() and torch.equal(cut[10:], full[10:])
    ctx.close()


# ---- verification ---------------------------------------------------------------------------------------------------
def probabilities(rng, n, V, sharp=2.0):
    z = rng.normal(0, sharp, (n, V))
    p = np.exp(z - z.max(1, keepdims=True))
    return (p / p.sum(1, keepdims=True)).astype(np.float32)


def run_verify(ctx, target, draft, u, tokens, parents, mode, pad=0, dtype=torch.float32):
    lens = [len(p) for p in parents]
    st, total = starts_of(lens), sum(lens)
    V = target.shape[1]

    def dev(x, dt):
        wide = torch.full((total + pad, V + 3 * pad), 0.5, dtype=dt, device=DEV)
        wide[:total, :V] = torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(dt)
        return wide[:, :V]
    def more(x, dt):
        return torch.cat([torch.tensor(np.asarray(x), dtype=dt, device=DEV), torch.full((pad,), 3, dtype=dt, device=DEV)])
    keep = torch.full((total + pad,), 9, dtype=torch.uint8, device=DEV)
    count, nxt = (torch.full((len(lens),), 9, dtype=torch.int32, device=DEV) for _ in range(2))
    ctx.tree_verify(dev(target, dtype), None if draft is None else dev(draft, torch.float32), None if u is None else more(u, torch.float32),
                    more(tokens, torch.int32), more(np.concatenate([np.asarray(p, np.int64) for p in parents]), torch.int32), i32(st), mode,
                    keep, count, nxt)
    assert (keep[total:] == 9).all()
    return [keep[a:e].cpu().numpy().astype(bool).tolist() for a, e in zip(st, st[1:])], count.tolist(), nxt.tolist()


def check_verify(ctx, target, draft, u, tokens, parents, mode, **kw):
    got = run_verify(ctx, target, draft, u, tokens, parents, mode, **kw)
    at = 0
    for b, p in enumerate(parents):
        n = len(p)
        rows = slice(at, at + n)
        keep, nxt = od.verify(target[rows], None if draft is None else draft[rows], None if u is None else u[rows], tokens[rows], p, mode)
        assert got[0][b] == keep and got[1][b] == sum(keep) and got[2][b] == nxt, (mode, b, got[0][b], keep, got[2][b], nxt)
        at += n


@pytest.mark.parametrize("mode", ["greedy", "sample", "replaced", "point"])
@pytest.mark.parametrize("V,lens", [(1, [1, 2]), (7, [5, 0, 9]), (100, [64, 1, 3, 70]), (1000, [20]), (4097, [12, 8]), (32000, [9, 17]),
                                    (50257, [6]), (131072, [4])])
def test_verify(mode, V, lens):
    dl, ctx = context(2, 64)
    for seed in range(4 if V < 5000 else 1):
        rng = np.random.default_rng(V + len(mode) + 31 * seed)
        parents = [random_tree(rng, n, chain=seed == 2) if n else [] for n in lens]
        total = sum(lens)
        target = probabilities(rng, total, V)
        draft = None
        if mode in ("sample", "replaced"):
            draft = (0.5 * target + 0.5 * probabilities(rng, total, V)).astype(np.float32)
        # tokens the target likes, and now and then any; twice the same among some siblings
        tokens = np.array([int(rng.integers(0, V)) for _ in range(total)], np.int64)
        at = 0
        for p in parents:
            for i in range(1, len(p)):
                if rng.random() < 0.7:
                    tokens[at + i] = np.argsort(target[at + p[i]])[-1 - int(rng.integers(0, min(2, V)))]
            at += len(p)
        u = None if mode == "greedy" else rng.random(total).astype(np.float32)
        check_verify(ctx, target, draft, u, tokens, parents, mode, pad=seed)
        if mode == "greedy":
            t16 = torch.from_numpy(target).to(torch.bfloat16).float().numpy()              # many ties
            check_verify(ctx, t16, None, None, tokens, parents, mode, pad=seed, dtype=torch.bfloat16)
    assert ctx.device_status()[0] == 0
    ctx.close()


@pytest.mark.parametrize("mode", ["sample", "replaced", "point"])
def test_verify_numbers_at_the_borders(mode):
    """u of 0 and just below 1, probabilities of 0, of 1 and equal ones; rows of which nothing is left."""
    dl, ctx = context(2, 64)
    one = np.float32(1 - 2.0 ** -24)
    p = np.zeros((6, 9), np.float32)
    p[:, 3], p[1, 3], p[1, 8], p[4, 0] = 1.0, 0.5, 0.5, 0.25
    for u0 in (0.0, 0.5, one):
        for u1 in (0.0, 0.5, one):
            u = np.array([u0, u1, u1, u1, u1, u1], np.float32)
            for tokens in ([0, 3, 8, 3, 3, 3], [0, 8, 3, 3, 0, 3], [0, 0, 0, 3, 3, 3]):
                for parent in ([-1, 0, 1, 2, 3, 4], [-1, 0, 0, 0, 1, 4]):
                    for q in (p, np.full_like(p, 1 / 9), np.roll(p, 1, 1)):
                        check_verify(ctx, p, None if mode == "point" else q, u, np.array(tokens), [parent], mode)
    assert ctx.device_status()[0] == 0
    ctx.close()


def test_verify_reports_what_it_cannot_take():
    dl, ctx = context(2, 64)
    rng = np.random.default_rng(9)
    p, q = probabilities(rng, 4, 50), probabilities(rng, 4, 50)
    u = np.full(4, 0.5, np.float32)
    for parents, tokens in [([[-1, 0], [-1, 1]], [0, 1, 0, 1]), ([[-1, 0], [-1, 0]], [0, 1, 0, 50]), ([[-1, 0], [-1, -5]], [0, 1, 0, 0])]:
        got = run_verify(ctx, p, q, u, np.array(tokens), parents, "sample")
        assert ctx.device_status() == (dl.DL_ERR_INVALID_ARG, 1)
        want = od.verify(p[2:], q[2:], u[2:], [0, 0], [-1, -9], "sample")                  # as if the node were not there
        assert got[0][1] == want[0] and got[2][1] == want[1]
    for mode, row in (("point", np.zeros((2, 50), np.float32)), ("point", np.full((2, 50), np.nan, np.float32)),
                      ("sample", np.zeros((2, 50), np.float32))):
        got = run_verify(ctx, row, row if mode == "sample" else None, u[:2], np.array([0, 1]), [[-1, 0]], mode)
        assert ctx.device_status() == (dl.DL_ERR_INVALID_ARG, 0) and got == ([[True, False]], [1], [-1])
    # NaN and infinite entries: NaN never counts, and values are held to 1
    row = np.zeros((2, 50), np.float32)
    row[:, 7], row[:, 9], row[:, 11] = np.nan, np.inf, 0.5
    check_verify(ctx, row, None, u[:2], np.array([0, 7]), [[-1, 0]], "point")
    z = np.full((2, 50), -np.inf, np.float32)
    z[1, 4], z[1, 5] = np.nan, -1.0
    z[0, 10], z[0, 20], z[0, 3] = 0.0, -0.0, -1.0
    check_verify(ctx, z, None, None, np.array([0, 10]), [[-1, 0]], "greedy")
    check_verify(ctx, np.full((2, 50), np.nan, np.float32), None, None, np.array([0, 10]), [[-1, 0]], "greedy")
    ctx.close()


# ---- accepted rows --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("Hk,D,page,held,nodes,L,share", [
    (1, 64, 16, [0], [1], 1, 1.0), (4, 128, 64, [60, 0, 7], [8, 26, 0], 3, 0.3), (2, 64, 16, [5, 100], [64, 40], 70, 0.5),
    (3, 128, 32, [31, 32, 33, 1], [33, 70, 300, 2], 2, 0.4), (8, 128, 128, [1000], [700], 1, 0.7), (2, 64, 32, [9, 9], [20, 30], 2, 0.0)])
def test_commit(Hk, D, page, held, nodes, L, share):
    dl, ctx = context(2 * Hk, D)
    rng = np.random.default_rng(Hk + D + sum(nodes) + L)
    pages, table = books(dl, rng, [h + n for h, n in zip(held, nodes)], held, page)
    pools = [up(bf(rng, pages.n_pages, 2, Hk, page, D)) for _ in range(L)]
    before = [p.clone() for p in pools]
    st, total = starts_of(nodes), sum(nodes)
    keep = (rng.random(total + 3) < share).astype(np.uint8) * 2
    ctx.kv16_commit(pages, pools, i32(st), u8(keep))
    assert ctx.device_status()[0] == 0
    for b, (a, e) in enumerate(zip(st, st[1:])):
        rows = np.flatnonzero(keep[a:e])
        for r, i in enumerate(rows):
            s, d = held[b] + int(i), held[b] + r
            for x in before:
                x[table[b, d // page], :, :, d % page] = x[table[b, s // page], :, :, s % page].clone()
        assert int(pages.cache_len[b]) == held[b] + len(rows)
    assert all(torch.equal(x, y) for x, y in zip(before, pools))
    ctx.close()


def test_commit_leaves_a_sequence_that_lacks_pages():
    dl, ctx = context(4, 64)
    rng = np.random.default_rng(8)
    pages, table = books(dl, rng, [16, 40], [10, 10], 16)                      # the first has no page for rows 16..
    pool = up(bf(rng, pages.n_pages, 2, 2, 16, 64))
    before = pool.clone()
    keep = np.zeros(30, np.uint8)
    keep[[0, 2, 9, 15, 20]] = 1
    ctx.kv16_commit(pages, [pool], i32([0, 12, 30]), u8(keep))
    assert ctx.device_status() == (dl.DL_ERR_CAPACITY, 0) and pages.cache_len.tolist() == [10, 12]
    p = table[0, 0]
    assert torch.equal(pool[p], before[p]) and torch.equal(pool[table[1, 0], :, :, 10], before[table[1, 0], :, :, 13])
    ctx.kv16_commit(pages, [], i32([0, 12, 30]), u8(keep * 0))
    assert pages.cache_len.tolist() == [10, 12]
    ctx.close()


@pytest.mark.parametrize("H,Hk,D,page,B,held,n", [(32, 8, 128, 32, 24, 5000, 1), (16, 2, 64, 16, 16, 9000, 2), (8, 2, 128, 64, 6, 6000, 40)])
def test_attention_launched_behind_itself_without_a_gap(H, Hk, D, page, B, held, n):
    """Hundreds of launches in the queue, shares of many key tiles: the launches' borders overlap, loads arrive in any order."""
    dl, ctx = context(H, D, B=B)
    rng = np.random.default_rng(B)
    lens = [int(x) for x in rng.integers(held // 4, held, B)]
    pages, _ = books(dl, rng, [h + n for h in lens], lens, page)
    pool, q = (torch.randn(*s, device=DEV).to(torch.bfloat16) for s in ((pages.n_pages, 2, Hk, page, D), (B * n, H, D)))
    st = i32(np.arange(B + 1) * n)
    first, out = torch.zeros_like(q), torch.zeros_like(q)
    ctx.kv16_attn_tree(pages, pool, q, st, n, None, D ** -0.5, first)
    for _ in range(400):
        ctx.kv16_attn_tree(pages, pool, q, st, n, None, D ** -0.5, out)
    assert ctx.device_status()[0] == 0 and torch.equal(first, out) and bool(first.isfinite().all())
    ctx.close()
