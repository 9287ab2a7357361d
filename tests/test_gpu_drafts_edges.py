"""Drafted tokens over a paged 16-bit cache (not in the paper), beyond single calls: whole steps of a server, captured and replayed,
on other streams; random shapes; scores that pass the maximum in use by far, wherever they stand; pools beyond 4 GB; large
vocabularies and long trees; refusals of the interface.  Oracles and tolerances: tests/test_gpu_drafts.py."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import drafts as od
from tests import test_gpu_drafts as base
from tests.test_gpu_drafts import DEV, HALF, bf, books, cache_rows, context, i32, probabilities, random_tree, starts_of, u8, up
from paper_2412_00876_b200 import workloads as wl

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---- a server's steps -----------------------------------------------------------------------------------------------
class Server:
    """Two layers over one set of books; everything that a step needs lies in tensors that stay, so that it can be captured."""

    def __init__(self, seed, stream=None, B=5, H=8, Hk=2, D=128, page=16, V=300, nodes=9):
        self.dl, self.ctx = context(H, D, B=B)
        self.B, self.H, self.Hk, self.D, self.V, self.n = B, H, Hk, D, V, nodes
        self.pages = self.dl.Pages(B, 60, 20, page, DEV)
        self.pools = [self.ctx.kv16_pool(self.pages, Hk) for _ in range(2)]
        self.rope = self.dl.Rope(D // 2, scaling="parts", factor=4.0, orig_len=64, device=DEV)
        self.starts = i32(np.arange(B + 1) * nodes)
        total = B * nodes
        z = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt, device=DEV)
        self.need, self.pos0 = torch.full((B,), nodes, dtype=torch.int32, device=DEV), z(B)
        self.parent, self.tokens, self.pos, self.mask = z(total), z(total), z(total), z(total, 1)
        self.keep, self.count, self.next = z(total, dt=torch.uint8), z(B), z(B)
        self.qkv = z(2, total, H + 2 * Hk, D, dt=torch.bfloat16)
        self.q, self.out = z(2, total, H, D, dt=torch.bfloat16), z(2, total, H, D, dt=torch.bfloat16)
        self.target, self.draft, self.u = z(total, V, dt=torch.float32), z(total, V, dt=torch.float32), z(total, dt=torch.float32)
        self.rng, self.held = np.random.default_rng(seed), [0] * B

    def prompts(self, lens):
        ctx, st, total = self.ctx, starts_of(lens), sum(lens)
        x = bf(self.rng, 2, total, self.H + 2 * self.Hk, self.D)
        flags = (self.rng.random(total) < 0.6).astype(np.uint8)
        pos = np.concatenate([np.arange(n) for n in lens])
        ctx.pages_reserve(self.pages, i32(lens))
        for layer in range(2):
            d = up(x[layer])
            ctx.kv16_append(self.pages, self.pools[layer], None, d[:, self.H:self.H + self.Hk], d[:, self.H + self.Hk:], i32(st), i32(pos),
                            self.rope, keep=u8(flags), commit=layer == 1)
        self.pos0.copy_(i32(lens))
        self.held = [int(flags[a:e].sum()) for a, e in zip(st, st[1:])]
        assert self.pages.cache_len.tolist() == self.held and ctx.device_status()[0] == 0

    def new_inputs(self):
        """a step's inputs, into the tensors that stay"""
        rng, total = self.rng, self.B * self.n
        self.parents = [random_tree(rng, self.n) for _ in range(self.B)]
        self.parent.copy_(i32(np.concatenate(self.parents)))
        t = probabilities(rng, total, self.V)
        self.target.copy_(torch.from_numpy(t))
        self.draft.copy_(torch.from_numpy((0.6 * t + 0.4 * probabilities(rng, total, self.V)).astype(np.float32)))
        likely = np.argsort(t, 1)[:, ::-1]
        tok = [0 if i == 0 else int(likely[b * self.n + self.parents[b][i], int(rng.integers(0, 3))])
               for b in range(self.B) for i in range(self.n)]
        self.tokens.copy_(i32(tok))
        self.u.copy_(torch.from_numpy(rng.random(total).astype(np.float32)))
        self.qkv.copy_(up(bf(rng, 2, total, self.H + 2 * self.Hk, self.D)))

    def step(self, stream=None):
        ctx, H, Hk = self.ctx, self.H, self.Hk
        ctx.pages_reserve(self.pages, self.need, stream)
        ctx.tree_plan(self.parent, self.starts, self.pos0, self.mask, self.pos, stream)
        for layer in range(2):
            x = self.qkv[layer]
            ctx.kv16_append(self.pages, self.pools[layer], x[:, :H], x[:, H:H + Hk], x[:, H + Hk:], self.starts, self.pos, self.rope,
                            q_out=self.q[layer], commit=False, stream=stream)
            ctx.kv16_attn_tree(self.pages, self.pools[layer], self.q[layer], self.starts, self.n, self.mask, self.D ** -0.5, self.out[layer],
                               stream)
        ctx.tree_verify(self.target, self.draft, self.u, self.tokens, self.parent, self.starts, "sample", self.keep, self.count, self.next,
                        stream)
        ctx.kv16_commit(self.pages, self.pools, self.starts, self.keep, stream)

    def check(self, before):
        """a step's results against the oracle; before: both pools, the table and the lengths in front of it"""
        pools, held = before
        table = self.pages.table.cpu().numpy()
        kept = self.keep.cpu().numpy()
        for b in range(self.B):
            rows = slice(b * self.n, (b + 1) * self.n)
            mask, pos = od.tree_plan([self.parents[b]], [int(self.pos0[b])], 1)
            assert np.array_equal(self.mask[rows].cpu().numpy().view(np.uint32), mask) and np.array_equal(self.pos[rows].cpu().numpy(), pos)
            keep, nxt = od.verify(self.target[rows].cpu().numpy(), self.draft[rows].cpu().numpy(), self.u[rows].cpu().numpy(),
                                  self.tokens[rows].cpu().numpy(), self.parents[b], "sample")
            assert kept[rows].astype(bool).tolist() == keep and int(self.count[b]) == sum(keep) and int(self.next[b]) == nxt
            assert int(self.pages.cache_len[b]) == held[b] + sum(keep)
            for layer in range(2):
                # the cache in front of the step with the nodes' rows behind it, which the commit has moved since
                was = cache_rows(pools[layer], table, b, held[b], self.pages.page_rows)
                x = wl.from_torch(self.qkv[layer, rows])
                freqs, amplitude = self.rope.freqs.cpu().numpy(), self.rope.desc.amplitude
                turned = od.turned(x[:, :self.H + self.Hk], pos, freqs, False, amplitude)
                k = np.concatenate([was[0], turned[:, self.H:]])
                v = np.concatenate([was[1], x[:, self.H + self.Hk:]])
                q = wl.from_torch(self.q[layer, rows])
                assert np.abs(q - turned[:, :self.H]).max() <= 2.0 ** -7 * np.abs(turned).max()
                # (node keys of the oracle are not rounded: HALF of each |q k|, through the exponential, on top)
                k16 = np.concatenate([was[0], base.wl.round_to_storage(turned[:, self.H:].astype(np.float32), "bf16")])
                ref = od.attention_tree(q, k16, v, held[b], mask, self.D ** -0.5)
                size = od.attention_tree(q, k16, np.abs(v), held[b], mask, self.D ** -0.5)
                got = wl.from_torch(self.out[layer, rows]).astype(np.float64)
                # a node key may round the other way where the two rotations differ: one step of a value, 2^-7 |q| |k| of one dim
                slack = 2.0 ** -7 * np.abs(q).max() * np.abs(k).max() * self.D ** -0.5
                bound = HALF * (size + np.abs(ref)) + (2.0 ** -12 + k.shape[0] * 2.0 ** -24 + slack) * size
                assert (np.abs(got - ref) <= bound).all(), (b, layer, np.abs(got - ref).max())
                now = cache_rows(wl.from_torch(self.pools[layer]), table, b, held[b] + sum(keep), self.pages.page_rows)
                assert np.array_equal(now[:, :held[b]], was)
                assert np.array_equal(now[1, held[b]:], x[np.array(keep), self.H + self.Hk:])
                # within the rotation's bound (tests/test_gpu_drafts.py)
                want = turned[np.array(keep), self.H:]
                assert (np.abs(now[0, held[b]:] - want) <= HALF * np.abs(want) + 2.0 ** -20 * amplitude * np.abs(x).max()).all()
        self.held = [h + int(c) for h, c in zip(held, self.count.tolist())]

    def state(self):
        return [wl.from_torch(p) for p in self.pools], list(self.held)


def test_steps_together_with_forks():
    s = Server(11)
    s.prompts([40, 17, 1, 64, 33])
    for turn in range(3):
        s.new_inputs()
        before = s.state()
        s.step()
        assert s.ctx.device_status()[0] == 0
        s.check(before)
        s.pos0 += s.count
        parent = [[1, 1, 3, 3, 0], [0, 1, 2, 3, 4], [4, 4, 4, 0, 1]][turn]
        s.ctx.pages_fork(s.pages, i32(parent), s.pools)
        s.held = [s.held[p] for p in parent]
        s.pos0.copy_(s.pos0[i32(parent).long()])
        assert s.pages.cache_len.tolist() == s.held and s.ctx.device_status()[0] == 0
    s.ctx.pages_compact(s.pages, s.pools)
    s.new_inputs()
    before = s.state()
    s.step()
    s.check(before)
    s.ctx.close()


def test_steps_captured_and_replayed_give_the_same_bits():
    a, b = Server(12), Server(12)
    for s in (a, b):
        s.prompts([40, 17, 1, 64, 33])
    side = torch.cuda.Stream()
    a.new_inputs()
    b.new_inputs()
    warm = Server(13)                                             # (first calls set attributes: not while capturing)
    warm.prompts([3, 3, 3, 3, 3])
    warm.new_inputs()
    warm.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.step(torch.cuda.current_stream())
    for turn in range(3):
        if turn:
            a.new_inputs()
            b.new_inputs()
        torch.cuda.synchronize()
        a.step(side)
        side.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("mask", "pos", "q", "out", "keep", "count", "next"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (turn, name)
        assert torch.equal(a.pages.book, b.pages.book) and all(torch.equal(x, y) for x, y in zip(a.pools, b.pools))
        for s in (a, b):
            s.pos0 += s.count
            assert s.ctx.device_status()[0] == 0
    del graph
    for s in (a, b, warm):
        s.ctx.close()


# ---- attention: random shapes, leading scores, alignments, large pools ------------------------------------------------
@pytest.mark.parametrize("seed", range(24))
def test_attention_of_random_shapes(seed):
    rng = np.random.default_rng(1000 + seed)
    D, page = int(rng.choice([64, 128])), int(rng.choice([16, 32, 64, 128]))
    Hk = int(rng.choice([1, 2, 3]))
    G = int(rng.choice([1, 2, 3, 4, 5, 7, 8, 16]))
    top = int(rng.choice([1, 1, 4, 12, 40]))
    B = int(rng.integers(1, 7))
    nodes = [int(x) for x in rng.integers(0, top + 1, B)]
    nodes[int(rng.integers(0, B))] = top
    held = [int(x) for x in rng.integers(0, int(rng.choice([3, 130, 700])), B)]
    base.check_attention(G * Hk, Hk, D, page, held, nodes, [None, "tree", "random"][int(rng.integers(0, 3))], seed=seed)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 3), (2, 30), (4, 12), (4, 25), (8, 30)])
@pytest.mark.parametrize("where", [0, 127, 128, 300, 511, 777])
def test_scores_that_pass_the_maximum_by_far(D, G, n, where):
    """One row of the cache scores 2^5 .. 2^7 times log2 units above all in front of it, another one in the next tile again: what was
    summed up before must go, and nothing may overflow."""
    held = 800

    def edit(pool, dev_pool, table):
        for t, size in ((where, 3.0), (min(where + 128, held - 1), 8.0)):
            row = np.full(pool.shape[-1], size, np.float32)
            pool[table[0, t // 64], 0, :, t % 64] = row
            dev_pool[table[0, t // 64], 0, :, t % 64] = up(row)
    rng = np.random.default_rng(where + n)
    dl, ctx = context(G * 2, D, B=4)
    pages, table = books(dl, rng, [held + n, 40 + n], [held, 40], 64)
    pool = bf(rng, pages.n_pages, 2, 2, 64, D, scale=0.3)
    dev_pool = up(pool)
    edit(pool, dev_pool, table)
    q = np.abs(bf(rng, 2 * n, G * 2, D)) + np.float32(0.5)         # every query likes large positive keys
    q = base.wl.round_to_storage(q.astype(np.float32), "bf16")
    out = torch.zeros(2 * n, G * 2, D, dtype=torch.bfloat16, device=DEV)
    ctx.kv16_attn_tree(pages, dev_pool, up(q), i32([0, n, 2 * n]), n, None, 0.5, out)
    assert ctx.device_status()[0] == 0
    for b, h in ((0, held), (1, 40)):
        k, v = cache_rows(pool, table, b, h + n, 64)
        rows = slice(b * n, (b + 1) * n)
        ref = od.attention_tree(q[rows], k, v, h, None, 0.5)
        size = od.attention_tree(q[rows], k, np.abs(v), h, None, 0.5)
        got = wl.from_torch(out[rows]).astype(np.float64)
        # scores of up to 2^10 carry D 2^-24 of themselves in fp32, through the exponential (ln 2 is below 1)
        bound = HALF * (size + np.abs(ref)) + (2.0 ** -12 + D * 2.0 ** -14) * size
        assert (np.abs(got - ref) <= bound).all(), (b, np.abs(got - ref).max())
    ctx.close()


@pytest.mark.parametrize("n", [2, 20, 60])
def test_outputs_on_16_bytes_and_rows_of_minus_infinity(n):
    """out that begins on 16 but not on 32 bytes; keys whose scores are all -inf weigh nothing, wherever their tile stands."""
    dl, ctx = context(4, 128, B=4)
    rng = np.random.default_rng(n)
    held = 300
    pages, table = books(dl, rng, [held + n], [held], 32)
    pool = up(bf(rng, pages.n_pages, 2, 2, 32, 128))
    q = torch.ones(n, 4, 128, dtype=torch.bfloat16, device=DEV)
    flat = torch.zeros(n * 512 + 8, dtype=torch.bfloat16, device=DEV)
    plain = torch.zeros(n, 4, 128, dtype=torch.bfloat16, device=DEV)
    args = (pages, pool, q, i32([0, n]), n, None, 0.1)
    ctx.kv16_attn_tree(*args, plain)
    ctx.kv16_attn_tree(*args, flat[8:].view(n, 4, 128))
    assert torch.equal(flat[8:].view(n, 4, 128), plain) and (flat[:8] == 0).all()
    for first, last in ((0, 128), (128, 256), (5, 290)):
        bad, few = pool.clone(), pool.clone()
        t = np.arange(first, last)
        pg, row = torch.from_numpy(table[0, t // 32].astype(np.int64)).to(DEV), torch.from_numpy(t % 32).to(DEV)
        bad[pg, 0, :, row] = float("-inf")
        got = torch.zeros_like(plain)
        ctx.kv16_attn_tree(pages, bad, q, i32([0, n]), n, None, 0.1, got)
        k, v = cache_rows(wl.from_torch(few), table, 0, held + n, 32)
        k[first:last] = np.nan                                        # the oracle leaves such rows out
        ref = od.attention_tree(wl.from_torch(q), k, v, held, None, 0.1)
        size = od.attention_tree(wl.from_torch(q), k, np.abs(v), held, None, 0.1)
        assert (np.abs(wl.from_torch(got) - ref) <= HALF * (size + np.abs(ref)) + 2.0 ** -11 * size).all()
    ctx.close()


def test_pools_beyond_4_gb():
    """Pages at either end of a pool of more than 2^32 bytes: append, attention and accepted rows."""
    dl, ctx = context(8, 128, B=2)
    page, Hk, n_pages = 128, 4, 17000                                  # 4.46 GB
    pages = dl.Pages(2, n_pages, 4, page, DEV)
    table = np.array([[n_pages - 1, 3, n_pages - 2, -1], [1, n_pages // 2, n_pages - 3, -1]], np.int32)
    pages.table.copy_(i32(table))
    pages.cache_len.zero_()
    pool = torch.zeros(n_pages, 2, Hk, page, 128, dtype=torch.bfloat16, device=DEV)
    rng = np.random.default_rng(1)
    lens = [300, 280]
    x = up(bf(rng, sum(lens), 2 * Hk, 128))
    st = i32(starts_of(lens))
    ctx.kv16_append(pages, pool, None, x[:, :Hk], x[:, Hk:], st, None, None)
    q = up(bf(rng, 10, 8, 128))
    out, ref_out = torch.zeros_like(q), torch.zeros_like(q)
    pages.cache_len -= 5                                                # the last five rows are the nodes'
    ctx.kv16_attn_tree(pages, pool, q, i32([0, 5, 10]), 5, None, 0.1, out)
    small = dl.Pages(2, 6, 4, page, DEV)
    small.table.copy_(i32([[0, 1, 2, -1], [3, 4, 5, -1]]))
    small.cache_len.copy_(pages.cache_len)
    near = pool[torch.from_numpy(table[:, :3].reshape(-1).astype(np.int64)).to(DEV)].contiguous()
    ctx.kv16_attn_tree(small, near, q, i32([0, 5, 10]), 5, None, 0.1, ref_out)
    assert torch.equal(out, ref_out) and bool((out != 0).any())
    keep = u8([1, 0, 1, 0, 0, 0, 1, 1, 0, 1])
    ctx.kv16_commit(pages, [pool], i32([0, 5, 10]), keep)
    ctx.kv16_commit(small, [near], i32([0, 5, 10]), keep)
    assert torch.equal(pool[torch.from_numpy(table[:, :3].reshape(-1).astype(np.int64)).to(DEV)], near)
    assert pages.cache_len.tolist() == [297, 278] and ctx.device_status()[0] == 0
    ctx.close()


# ---- verification -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("mode", ["greedy", "sample", "replaced", "point"])
def test_verify_of_the_largest_vocabulary_and_of_long_trees(mode):
    dl, ctx = context(2, 64)
    rng = np.random.default_rng(5)
    for V, n, chain in ((262144, 3, False), (262143, 2, True), (40, 2048, True), (33, 700, False)):
        parents = [random_tree(rng, n, chain)]
        target = probabilities(rng, n, V, 1.0)
        draft = target if chain and V < 100 else probabilities(rng, n, V, 1.0)      # (a draft that is the target is accepted all along)
        tokens = rng.integers(0, V, n)
        if V < 100:
            tokens = np.array([0] + [int(np.argmax(target[parents[0][i]])) for i in range(1, n)])
        u = None if mode == "greedy" else rng.random(n).astype(np.float32)
        base.check_verify(ctx, target, draft if mode in ("sample", "replaced") else None, u, tokens, parents, mode)
    assert ctx.device_status()[0] == 0
    ctx.close()


def test_verify_of_many_sequences_at_once():
    """More clusters than the GPU holds at a time."""
    dl, ctx = context(2, 64)
    rng = np.random.default_rng(6)
    parents = [random_tree(rng, int(n)) for n in rng.integers(1, 5, 300)]
    total = sum(len(p) for p in parents)
    target = probabilities(rng, total, 97)
    draft = probabilities(rng, total, 97)
    base.check_verify(ctx, target, draft, rng.random(total).astype(np.float32), rng.integers(0, 97, total), parents, "sample")
    ctx.close()


# ---- refusals of the interface ------------------------------------------------------------------------------------------
def test_nodes_beyond_what_a_call_takes_are_never_kept():
    """2048 nodes of a sequence are verified; those behind are reported and count as rejected, whatever lay in the output."""
    dl, ctx = context(4, 64)
    n, vocab = 2060, 8
    target = torch.zeros(n + 6, vocab, device=DEV)
    target[:, 3] = 1
    parent = np.concatenate([np.arange(-1, n - 1), np.arange(-1, 5)])
    keep = torch.full((n + 6,), 7, dtype=torch.uint8, device=DEV)
    count, nxt = i32([0, 0]), i32([0, 0])
    ctx.tree_verify(target, None, None, i32(np.full(n + 6, 3)), i32(parent), i32([0, n, n + 6]), "greedy", keep, count, nxt)
    status = ctx.device_status()
    assert status[0] == dl.DL_ERR_INVALID_ARG and status[1] == 0
    assert keep.tolist() == [1] * 2048 + [0] * 12 + [1] * 6
    assert count.tolist() == [2048, 6] and nxt.tolist() == [3, 3]


def test_plans_of_long_chains():
    """2048 nodes in a row: every word of the mask, in front of the node and behind it."""
    dl, ctx = context(4, 64)
    n = 2048
    mask, pos = torch.full((n + 3, 64), -9, dtype=torch.int32, device=DEV), torch.full((n + 3,), -9, dtype=torch.int32, device=DEV)
    ctx.tree_plan(i32(np.concatenate([np.arange(-1, n - 1), [-1, 0, 0]])), i32([0, n, n + 3]), i32([5, 7]), mask, pos)
    want = np.zeros((n + 3, 64), np.uint64)
    for i in range(n):
        want[i, :i // 32] = 0xFFFFFFFF
        want[i, i // 32] = (1 << (i % 32 + 1)) - 1
    want[n:, 0] = [1, 3, 5]
    assert np.array_equal(mask.cpu().numpy().view(np.uint32), want.astype(np.uint32))
    assert pos.tolist() == list(range(5, 5 + n)) + [7, 8, 8] and ctx.device_status()[0] == 0


def test_no_pool_is_committed_twice():
    """The same rows would move up twice: the call is refused, and nothing has moved."""
    dl, ctx = context(4, 64)
    pages = dl.Pages(1, 4, 4, 16, DEV)
    pools = [ctx.kv16_pool(pages, 2) for _ in range(3)]
    ctx.pages_reserve(pages, i32([8]))
    for i, p in enumerate(pools):
        p.copy_(torch.arange(p.numel(), device=DEV).reshape(p.shape) % 97 + i)
    before = [p.clone() for p in pools]
    with pytest.raises(dl.DlError) as e:
        ctx.kv16_commit(pages, [pools[0], pools[1], pools[2], pools[0]], i32([0, 4]), u8(np.array([1, 0, 1, 1])))
    assert e.value.code == dl.DL_ERR_INVALID_ARG
    assert all(torch.equal(a, b) for a, b in zip(pools, before)) and pages.cache_len.tolist() == [0]


def test_refusals():
    import ctypes as C
    dl, ctx = context(8, 64, B=4)
    L, ok = dl.lib(), dl.DL_OK
    pages = dl.Pages(4, 8, 2, 16, DEV)
    pool = ctx.kv16_pool(pages, 2)
    x = torch.zeros(6, 12, 64, dtype=torch.bfloat16, device=DEV)
    st, pos, keep = i32([0, 1, 2, 4, 6]), i32(np.zeros(6)), u8(np.ones(6))
    rope = dl.Rope(64, device=DEV)
    p = lambda t: t.data_ptr()

    def append(**kw):
        a = dict(pages=pages.ref, kv=2, pool=p(pool), q=p(x), qs=768, k=p(x), v=p(x), ks=768, pos=p(pos), rope=rope.ref, starts=p(st),
                 keep=None, total=6, qo=p(x), qos=768, ko=None, kos=0)
        a.update(kw)
        return L.dl_kv16_append(ctx._h, a["pages"], a["kv"], a["pool"], a["q"], a["qs"], a["k"], a["v"], a["ks"], a["pos"], a["rope"],
                                a["starts"], a["keep"], a["total"], a["qo"], a["qos"], a["ko"], a["kos"], 0, None)

    def rope_of(**kw):
        return C.pointer(dl.RopeDesc(*[kw.get(n, getattr(rope.desc, n)) for n in ("rot_dim", "interleaved", "freqs", "amplitude")]))
    inv, mis, uns, wsp = dl.DL_ERR_INVALID_ARG, dl.DL_ERR_ALIGNMENT, dl.DL_ERR_UNSUPPORTED, dl.DL_ERR_WORKSPACE
    assert append(total=0) == ok
    for kw, want in [(dict(kv=3), inv), (dict(kv=0), inv), (dict(pool=None), inv), (dict(pages=None), inv), (dict(q=None), inv),
                     (dict(qo=None), inv), (dict(k=None), inv), (dict(v=None), inv), (dict(starts=None), inv), (dict(pos=None), inv),
                     (dict(total=-1), inv), (dict(qs=500), inv), (dict(ks=100), inv), (dict(ks=772), mis), (dict(k=p(x) + 8), mis),
                     (dict(pool=p(pool) + 8), mis), (dict(qos=520), inv), (dict(rope=rope_of(rot_dim=24)), uns),
                     (dict(rope=rope_of(rot_dim=80)), inv), (dict(rope=rope_of(freqs=None)), inv), (dict(qs=1 << 33, qos=1 << 33), uns)]:
        assert append(**kw) == want, kw
    out, mask = torch.zeros(6, 8, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(6, 1, dtype=torch.int32, device=DEV)

    def attend(**kw):
        a = dict(pages=pages.ref, kv=2, pool=p(pool), q=p(x), qs=768, starts=p(st), total=6, rows=2, mask=p(mask), words=1, scale=0.1, out=p(out))
        a.update(kw)
        return L.dl_kv16_attn_tree(ctx._h, a["pages"], a["kv"], a["pool"], a["q"], a["qs"], a["starts"], a["total"], a["rows"], a["mask"],
                                   a["words"], a["scale"], a["out"], None)
    assert attend(total=0) == ok and attend(rows=0) == ok
    for kw, want in [(dict(kv=5), inv), (dict(scale=0.0), inv), (dict(scale=float("nan")), inv), (dict(words=0), inv), (dict(q=None), inv),
                     (dict(out=None), inv), (dict(pool=None), inv), (dict(starts=None), inv), (dict(rows=-1), inv), (dict(total=-1), inv),
                     (dict(qs=100), inv), (dict(qs=770), mis), (dict(out=p(out) + 4), mis), (dict(pages=None), inv)]:
        assert attend(**kw) == want, kw
    bad = dl.Pages(4, 8, 2, 16, DEV)
    bad.desc.page_rows = 48
    assert attend(pages=bad.ref) == uns and append(pages=bad.ref) == uns
    bad.desc.page_rows, bad.desc.n_pages = 16, 1 << 26
    assert attend(pages=bad.ref) == uns
    many = dl.Pages(40, 8, 2, 16, DEV)
    assert attend(pages=many.ref) == wsp
    t, d, u, one = torch.zeros(6, 9, device=DEV), torch.zeros(6, 9, device=DEV), torch.zeros(6, device=DEV), i32(np.zeros(6))

    def verify(**kw):
        a = dict(t=p(t), dt=dl.DL_F32, ts=0, d=p(d), ds=0, u=p(u), tok=p(one), par=p(one), st=p(st), B=4, total=6, V=9, mode=1, keep=p(keep),
                 count=p(one), nxt=p(one))
        a.update(kw)
        return L.dl_tree_verify(ctx._h, a["t"], a["dt"], a["ts"], a["d"], a["ds"], a["u"], a["tok"], a["par"], a["st"], a["B"], a["total"], a["V"],
                                a["mode"], a["keep"], a["count"], a["nxt"], None)
    assert verify(B=0) == ok
    for kw, want in [(dict(t=None), inv), (dict(d=None), inv), (dict(u=None), inv), (dict(V=0), inv), (dict(V=1 << 19), uns), (dict(mode=4), inv),
                     (dict(mode=-1), inv), (dict(dt=dl.DL_BF16), uns), (dict(dt=7, mode=0), uns), (dict(ts=8), inv), (dict(ds=3), inv),
                     (dict(t=p(t) + 4), mis), (dict(keep=None), inv), (dict(total=-1), inv), (dict(count=None), inv)]:
        assert verify(**kw) == want, kw
    ptrs = (C.c_void_p * 1)(p(pool))

    def commit(**kw):
        a = dict(pages=pages.ref, kv=2, n=1, pools=ptrs, st=p(st), keep=p(keep), total=6)
        a.update(kw)
        return L.dl_kv16_commit(ctx._h, a["pages"], a["kv"], a["n"], a["pools"], a["st"], a["keep"], a["total"], None)
    assert commit(total=0) == ok
    for kw, want in [(dict(kv=3), inv), (dict(n=-1), inv), (dict(pools=None), inv), (dict(pools=(C.c_void_p * 1)(None)), inv),
                     (dict(pools=(C.c_void_p * 1)(p(pool) + 8)), mis), (dict(keep=None), inv), (dict(st=None), inv), (dict(total=-3), inv)]:
        assert commit(**kw) == want, kw
    plan = lambda words, par=p(one), out=p(mask): L.dl_tree_plan(ctx._h, par, p(st), None, 4, 6, words, out, None, None)
    assert plan(0) == uns and plan(65) == uns and plan(1, par=None) == inv and plan(1, out=None) == inv
    f32 = dl.Context(64, 8, 64, 64, torch.float32, 0, max_batch=4, cap=64)
    assert L.dl_kv16_attn_tree(f32._h, pages.ref, 2, p(pool), p(x), 768, p(st), 6, 2, None, 0, 0.1, p(out), None) == uns
    assert L.dl_kv16_append(f32._h, pages.ref, 2, p(pool), None, 0, p(x), p(x), 768, None, None, p(st), None, 6, None, 0, None, 0, 0, None) == uns
    torch.cuda.synchronize()
    assert ctx.device_status()[0] == 0
    f32.close()
    ctx.close()


def test_clean_under_the_checked_build():
    """Stores through computed indices are compared with their buffers first: nothing is recorded, the same results."""
    if os.environ.get("DL_SPARSE_CHECKED") == "1":
        pytest.skip("running under it")
    env = dict(os.environ, DL_SPARSE_CHECKED="1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "tests/test_gpu_drafts.py", "tests/test_gpu_drafts_edges.py", "-k",
                        "test_append or test_commit or test_tree or (test_attention and not gap) or steps or replayed"],
                       capture_output=True, text=True, env=env, cwd=ROOT, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
