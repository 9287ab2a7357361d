"""Pins of oracle/drafts.py, the host helper of rotary frequencies, and what the binding of the drafted-token calls refuses: no GPU."""
import math

import numpy as np
import pytest
import torch

from oracle import drafts as od
from paper_2412_00876_b200 import binding as dl


def test_a_turn_keeps_lengths_and_depends_on_distances_only():
    rng = np.random.default_rng(0)
    f = [1.0, 0.1, 0.01, 0.003]
    for inter in (False, True):
        x, y = rng.normal(size=(1, 1, 10)), rng.normal(size=(1, 1, 10))
        dots = []
        for p in (0, 5, 100000, 2 ** 31 - 8):
            a, b = od.turned(x, [p], f, inter), od.turned(y, [p + 7], f, inter)
            assert np.allclose(np.linalg.norm(a), np.linalg.norm(x), atol=1e-12)
            assert np.array_equal(a[..., 8:], x[..., 8:])
            dots.append(float((a * b).sum()))
        assert np.allclose(dots, dots[0], atol=1e-6)
    assert np.allclose(od.turned(x, [1], [math.pi / 2] + [0.0] * 3, True)[0, 0, :2], [-x[0, 0, 1], x[0, 0, 0]], atol=1e-12)
    assert np.allclose(od.turned(x, [1], [0.0] * 4, False, 2.0)[0, 0], np.concatenate([2 * x[0, 0, :8], x[0, 0, 8:]]))


def test_tree_plan_by_hand():
    mask, pos = od.tree_plan([[-1, 0, 0, 1, 3], [-1]], [10, 3], 1)
    assert mask[:, 0].tolist() == [0b1, 0b11, 0b101, 0b1011, 0b11011, 0b1]
    assert pos.tolist() == [10, 11, 11, 12, 13, 3]
    mask, _ = od.tree_plan([[-1] + list(range(39))], [0], 2)
    assert mask[39].tolist() == [0xFFFFFFFF, 0xFF]


def test_attention_rows_that_see_nothing_are_zero():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(2, 2, 8)), rng.normal(size=(2, 1, 8)), rng.normal(size=(2, 1, 8))
    out = od.attention_tree(q, k, v, 0, np.array([[0], [2]], np.uint32), 0.3)
    assert not out[0].any() and np.allclose(out[1], v[1])
    assert np.allclose(od.attention_tree(q, k, v, 0, None, 0.3)[0], v[0])


@pytest.mark.parametrize("mode", ["sample", "replaced", "point"])
def test_verified_tokens_are_distributed_as_the_targets(mode):
    """One node deep, two children: over many draws the first token behind the root has the target's distribution (the
    accepted child, or the token drawn).  5 tokens, 40k draws: a share is off by 0.0025 on average, 0.0125 is five of those."""
    rng = np.random.default_rng(7)
    p = np.array([0.4, 0.3, 0.15, 0.1, 0.05], np.float32)
    q = np.array([0.1, 0.5, 0.2, 0.1, 0.1], np.float32)
    hits, N = np.zeros(5), 40000
    for _ in range(N):
        if mode == "sample":
            kids = rng.choice(5, 2, replace=False, p=q.astype(np.float64) / q.astype(np.float64).sum())
        elif mode == "replaced":
            kids = rng.choice(5, 2, p=q.astype(np.float64) / q.astype(np.float64).sum())
        else:
            kids = [1, 4]
        u = rng.random(3).astype(np.float32)
        keep, nxt = od.verify([p, p, p], [q, q, q], u, [0, *kids], [-1, 0, 0], mode)
        hits[kids[0] if keep[1] else kids[1] if keep[2] else nxt] += 1
    assert np.abs(hits / N - p).max() < 0.0125


def test_verify_by_hand():
    p = np.array([[0.5, 0.5, 0.0], [0.0, 1.0, 0.0], [1.0, 0.0, 0.0]], np.float32)
    assert od.verify(p, None, [0, 0, 0], [0, 0, 1], [-1, 0, 1], "greedy") == ([True, True, True], 0)
    assert od.verify(p, None, [0, 0, 0], [0, 1, 1], [-1, 0, 1], "greedy") == ([True, False, False], 0)
    # chain of two: the first accepted whatever u is (p >= q), the second never (p = 0); then only token 1 is left
    keep, nxt = od.verify(p, p, [0.9, 0.99, 0.0], [0, 0, 2], [-1, 0, 1], "sample")
    assert (keep, nxt) == ([True, True, False], 1)
    # all of p goes to rejected children: what is left is nothing, and p itself is drawn from
    keep, nxt = od.verify(p[1:2], None, [0.3], [0], [-1], "point")
    assert (keep, nxt) == ([True], 1)
    assert od.verify(np.zeros((1, 4), np.float32), None, [0.3], [0], [-1], "point") == ([True], -1)


# ---- the host helper
@pytest.mark.parametrize("rot", [16, 64, 128])
@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("linear", 4.0), ("ntk", 8.0), ("parts", 16.0)])
def test_rope_freqs(rot, scaling, factor):
    got, amplitude = dl.rope_freqs(rot, 10000.0, scaling, factor, 2048)
    base = 10000.0 * (factor ** (rot / (rot - 2)) if scaling == "ntk" else 1.0)
    want = [base ** (-2 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        want = [f / factor for f in want]
    if scaling == "parts":
        part = [min(max((2048 * f / (2 * math.pi) - 1) / 31, 0), 1) for f in want]
        want = [f * (g + (1 - g) / factor) for f, g in zip(want, part)]
        assert part[0] == 1 and part[-1] == 0
    assert np.allclose(got.numpy(), want, rtol=1e-13)
    assert amplitude == (0.1 * math.log(factor) + 1 if scaling == "parts" else 1.0)


@pytest.mark.parametrize("bad", [dict(rot_dim=-2), dict(rot_dim=7), dict(base=1.0), dict(factor=0.5), dict(scaling="parts", orig_len=0),
                                 dict(base=float("nan"))])
def test_rope_freqs_refuses(bad):
    with pytest.raises((dl.DlError, RuntimeError)):
        dl.rope_freqs(**{"rot_dim": 16, "factor": 2.0, **bad})


# ---- refusals of the binding
class NoLibrary:
    """Stands in for the library: a call that gets this far was not refused."""

    def __getattr__(self, name):
        def call(*a):
            raise AssertionError(f"{name} was called")
        return call


@pytest.fixture
def ctx(monkeypatch):
    c = dl.Context.__new__(dl.Context)
    c._h, c.device, c.dtype, c.H, c.D = None, torch.device("cuda", 0), torch.bfloat16, 4, 64
    monkeypatch.setattr(dl, "lib", lambda: NoLibrary())
    monkeypatch.setattr(c, "_on", lambda stream: 0)
    return c


class Device:
    """what a device of the CPU's tensors is called: index -1"""
    index = -1


def rows(n, heads, D=64):
    return torch.zeros(n, heads, D, dtype=torch.bfloat16)


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


CALLS = {
    "append": lambda c, pg, rope: c.kv16_append(pg, torch.zeros(4, 2, 2, 16, 64, dtype=torch.bfloat16), rows(3, 4), rows(3, 2), rows(3, 2),
                                                ints(3), ints(3), rope, q_out=rows(3, 4)),
    "attend": lambda c, pg, rope: c.kv16_attn_tree(pg, torch.zeros(4, 2, 2, 16, 64, dtype=torch.bfloat16), rows(3, 4), ints(3), 2, None,
                                                   0.1, rows(3, 4)),
    "commit": lambda c, pg, rope: c.kv16_commit(pg, [torch.zeros(4, 2, 2, 16, 64, dtype=torch.bfloat16)], ints(3),
                                                torch.zeros(3, dtype=torch.uint8)),
}


@pytest.mark.parametrize("call", sorted(CALLS))
def test_books_on_another_device_are_refused(monkeypatch, ctx, call):
    monkeypatch.setattr(dl, "_arg", lambda t, dtype, shape, what, index: t.data_ptr())
    monkeypatch.setattr(dl, "_rows", lambda t, dtype, shape, what, index: (t.data_ptr(), 0))
    with pytest.raises(ValueError, match="books on cuda:0, got cpu"):
        CALLS[call](ctx, dl.Pages(2, 4, 2, 16, device="cpu"), None)


def test_frequencies_on_another_device_are_refused(monkeypatch, ctx):
    monkeypatch.setattr(dl, "_arg", lambda t, dtype, shape, what, index: t.data_ptr())
    monkeypatch.setattr(dl, "_rows", lambda t, dtype, shape, what, index: (t.data_ptr(), 0))
    monkeypatch.setattr(ctx, "_books", lambda pages: None)
    with pytest.raises(ValueError, match="frequencies on cuda:0, got cpu"):
        CALLS["append"](ctx, dl.Pages(2, 4, 2, 16, device="cpu"), dl.Rope(16, freqs=[1.0] * 8, device="cpu"))


@pytest.mark.parametrize("what,change", [
    ("k", dict(k=rows(3, 2).expand(3, 2, 64).float())), ("k", dict(k=rows(1, 2).expand(3, 2, 64))), ("row stride", dict(v=rows(6, 2)[::2])),
    ("q_out", dict(q_out=rows(4, 4))), ("pos", dict(pos=ints(2))), ("starts", dict(starts=ints(2))),
    ("keep", dict(keep=torch.ones(3))), ("pool", dict(pool=torch.zeros(4, 2, 2, 32, 64, dtype=torch.bfloat16))),
    ("go together", dict(v=None))])
def test_append_refuses(monkeypatch, ctx, what, change):
    ctx.device = Device
    args = dict(pages=dl.Pages(2, 4, 2, 16, device="cpu"), pool=torch.zeros(4, 2, 2, 16, 64, dtype=torch.bfloat16), q=rows(3, 4),
                k=rows(3, 2), v=rows(3, 2), starts=ints(3), pos=ints(3), rope=None, keep=torch.ones(3, dtype=torch.uint8), q_out=rows(3, 4))
    with pytest.raises(AssertionError, match="dl_kv16_append was called"):
        ctx.kv16_append(**args)
    with pytest.raises(ValueError, match=what):
        ctx.kv16_append(**{**args, **change})


@pytest.mark.parametrize("what,change", [
    ("target", dict(target=torch.zeros(3, 9, dtype=torch.float16))), ("target", dict(target=torch.zeros(2, 9))),
    ("overlap", dict(target=torch.zeros(1, 9).expand(3, 9))), ("overlap", dict(draft=torch.zeros(9, 3).t())),
    ("vocabulary", dict(draft=torch.zeros(3, 8))), ("u", dict(u=torch.zeros(2))), ("tokens", dict(tokens=torch.zeros(3))),
    ("parent", dict(parent=ints(4))), ("keep_out", dict(keep_out=ints(3))), ("next_out", dict(next_out=ints(3)))])
def test_verify_refuses(ctx, what, change):
    ctx.device = Device
    args = dict(target=torch.zeros(3, 9), draft=torch.zeros(3, 9), u=torch.zeros(3), tokens=ints(3), parent=ints(3), starts=ints(3),
                mode="sample", keep_out=torch.zeros(3, dtype=torch.uint8), count_out=ints(2), next_out=ints(2))
    with pytest.raises(AssertionError, match="dl_tree_verify was called"):
        ctx.tree_verify(**args)
    with pytest.raises(ValueError, match=what):
        ctx.tree_verify(**{**args, **change})
    with pytest.raises(ValueError, match="target"):
        ctx.tree_verify(**{**args, "target": torch.zeros(3, 9, dtype=torch.bfloat16)})     # 16 bits: greedy only


def test_attend_and_commit_refuse(ctx):
    ctx.device = Device
    pages, pool = dl.Pages(2, 4, 2, 16, device="cpu"), torch.zeros(4, 2, 2, 16, 64, dtype=torch.bfloat16)
    args = dict(pages=pages, pool=pool, q=rows(3, 4), starts=ints(3), max_rows=2, mask=ints(3, 1), scale=0.1, out=rows(3, 4))
    with pytest.raises(AssertionError, match="dl_kv16_attn_tree was called"):
        ctx.kv16_attn_tree(**args)
    for what, change in [("mask", dict(mask=ints(2, 1))), ("out", dict(out=rows(3, 2))), ("starts", dict(starts=ints(4))),
                         ("q", dict(q=rows(3, 2))), ("pool", dict(pool=pool[:3]))]:
        with pytest.raises(ValueError, match=what):
            ctx.kv16_attn_tree(**{**args, **change})
    keep = torch.zeros(3, dtype=torch.uint8)
    with pytest.raises(AssertionError, match="dl_kv16_commit was called"):
        ctx.kv16_commit(pages, [pool, pool], ints(3), keep)
    for pools in ([pool, pool[:3]], [pool.float()]):
        with pytest.raises(ValueError, match="pool"):
            ctx.kv16_commit(pages, pools, ints(3), keep)
