"""What the binding of the serving calls refuses before a kernel sees it (no GPU needed: tensors of the CPU stand in for
those of device -1)."""
import pytest
import torch

from paper_2412_00876_b200 import binding as dl


def rows(t, what="k"):
    return dl._rows(t, torch.bfloat16, tuple(t.shape), what, -1)


@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_rows_that_lie_over_one_another_are_refused(what):
    one = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match=what):
        rows(one.expand(1000, 2, 64), what)                       # one row of 256 bytes, not a thousand
    flat = torch.zeros(4096, dtype=torch.bfloat16)
    for step in (8, 64, 120):
        with pytest.raises(ValueError, match=what):
            rows(flat.as_strided((10, 2, 64), (step, 64, 1)), what)


def test_rows_that_do_not_are_taken_with_their_stride():
    flat = torch.zeros(8192, dtype=torch.bfloat16)
    for step in (128, 136, 400):
        assert rows(flat.as_strided((10, 2, 64), (step, 64, 1))) == (flat.data_ptr(), step)
    assert rows(flat.as_strided((1, 2, 64), (0, 64, 1))) == (flat.data_ptr(), 128)          # one row has no next
    assert rows(flat[:0].view(0, 2, 64))[1] in (0, 128)
    with pytest.raises(ValueError, match="dense heads"):
        rows(flat.as_strided((10, 2, 64), (256, 128, 1)))


class NoLibrary:
    """Stands in for the library: a call that gets this far was not refused."""

    def __getattr__(self, name):
        def call(*a):
            raise AssertionError(f"{name} was called")
        return call


@pytest.mark.parametrize("call", ["reserve", "free", "fork", "compact", "append", "read", "attend"])
def test_books_on_another_device_are_refused(monkeypatch, call):
    """The books' pointers go to the kernels: books of the CPU (or of another GPU) must not get there."""
    monkeypatch.setattr(dl, "lib", lambda: NoLibrary())
    monkeypatch.setattr(dl, "_arg", lambda t, dtype, shape, what, index: t.data_ptr())      # every other tensor is in order
    monkeypatch.setattr(dl, "_rows", lambda t, dtype, shape, what, index: (t.data_ptr(), 0))
    ctx = dl.Context.__new__(dl.Context)
    ctx._h, ctx.device, ctx.dtype, ctx.H, ctx.D = None, torch.device("cuda", 0), torch.bfloat16, 2, 64
    monkeypatch.setattr(ctx, "_on", lambda stream: 0)
    monkeypatch.setattr(ctx, "_pools", lambda pages, pools: (0, None, 0))
    pages, x = dl.Pages(2, 4, 2, 16, device="cpu"), torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    n = torch.zeros(3, dtype=torch.int32)
    calls = {"reserve": lambda: ctx.pages_reserve(pages, n), "free": lambda: ctx.pages_free(pages, n),
             "fork": lambda: ctx.pages_fork(pages, n, []), "compact": lambda: ctx.pages_compact(pages, []),
             "append": lambda: ctx.kv4_append(pages, x, x, x, n), "read": lambda: ctx.kv4_read(pages, x, n, n, x, x),
             "attend": lambda: ctx.kv4_attn_decode(pages, x, x, x, x, None, 1.0, x)}
    with pytest.raises(ValueError, match="books on cuda:0, got cpu"):
        calls[call]()
