"""Edges of the serving calls that ordinary batches do not reach."""
import numpy as np
import pytest
import torch

from oracle import paged_kv4 as pk
from paper_2412_00876_b200 import workloads as wl
from tests.test_gpu_serving_ops import DEV, bf, close, context, i32, up

pytestmark = pytest.mark.gpu


def test_compacting_the_pages_of_no_sequence_says_that_none_is_in_use():
    dl, ctx = context(4, 64)
    pg = dl.Pages(0, 6, 2, 16, DEV)
    live = torch.full((1,), 7, dtype=torch.int32, device=DEV)
    ctx.pages_compact(pg, [], live)
    assert live.item() == 0
    ctx.pages_compact(pg, [])
    assert ctx.device_status()[0] == 0
    ctx.close()


@pytest.mark.parametrize("n_pages", [12100, 12120, 12168, 12184, 12185, 12300])
def test_fork_with_books_of_about_48_kb(n_pages):
    """The shared memory of the bookkeeping on either side of what a kernel may have without asking for more."""
    dl, ctx = context(4, 64)
    pg = dl.Pages(8, n_pages, 4, 16, DEV)
    pg.table[0, :2] = i32([3, n_pages - 1])
    pg.refs[[3, n_pages - 1]] = 1
    pg.cache_len[0] = 20
    pool = torch.arange(n_pages, device=DEV).to(torch.int32).repeat_interleave(4).view(n_pages, 4).contiguous()
    ctx.pages_fork(pg, i32([0, 0, 2, 3, 4, 5, 6, 7]), [pool])
    assert pg.table[:2].tolist() == [[3, n_pages - 1, -1, -1], [3, 0, -1, -1]]
    assert pg.cache_len.tolist() == [20, 20] + [0] * 6 and pool[0].tolist() == [n_pages - 1] * 4
    assert ctx.device_status()[0] == 0
    ctx.close()


@pytest.mark.parametrize("B,n_pages,width", [(2048, 30000, 16), (300, 50000, 20), (300, 20000, 100), (2048, 9000, 4), (2048, 50000, 16)])
def test_books_that_shared_memory_does_not_hold(B, n_pages, width):
    """Fork, reserve, free and compact with counts, rows or both in global memory; and a fork that finds too few pages."""
    dl, ctx = context(4, 64, B=B)
    rng = np.random.default_rng(B)
    page = 16
    rows = rng.integers(0, (width - 1) * page, B)
    order, at, pages = rng.permutation(n_pages).tolist(), 0, []
    room = n_pages * 3 // 4
    for b in range(B):
        c = min(-(-int(rows[b]) // page), max(0, room - at))
        rows[b] = min(rows[b], c * page)
        pages.append(order[at:at + c])
        at += c
    o = pk.Books(n_pages, page, width, pages, rows.tolist(), list(range(n_pages)))
    pg = dl.Pages(B, n_pages, width, page, DEV)
    pg.table.copy_(i32(o.table()))
    pg.refs.copy_(i32(o.refs()))
    pg.cache_len.copy_(i32(o.length))
    pool = torch.arange(n_pages, device=DEV).to(torch.int32).repeat_interleave(4).view(n_pages, 4).contiguous()

    def agree():
        assert np.array_equal(pg.table.cpu().numpy(), o.table())
        assert pg.refs.tolist() == o.refs() and pg.cache_len.tolist() == o.length
        assert torch.equal(pool[:, 0].cpu(), torch.tensor(o.data, dtype=torch.int32))

    parent = np.where(rng.random(B) < 0.6, np.arange(B), rng.integers(-1, B, B))
    assert o.fork(parent.tolist())
    ctx.pages_fork(pg, i32(parent), [pool])
    agree()
    need = rng.integers(0, page, B)
    ok = o.reserve(need.tolist())
    ctx.pages_reserve(pg, i32(need))
    assert ctx.device_status()[0] == (0 if ok else dl.DL_ERR_CAPACITY)
    agree()
    # no free page is left: a fork that has to copy changes nothing
    free = (pg.refs == 0)
    was, bytes_was = pg.book.clone(), pool.clone()
    pg.refs[free] = 1
    full = pg.book.clone()
    src = int(np.argmax([n % page != 0 for n in o.length]))
    parent = np.where(np.arange(B) % 2 == 0, src, np.arange(B))
    ctx.pages_fork(pg, i32(parent), [pool])
    lost = sum(len(o.pages[b]) for b in range(0, B, 2))
    if ctx.device_status() == (dl.DL_ERR_CAPACITY, -1):
        assert torch.equal(pg.book, full) and torch.equal(pool, bytes_was)
        pg.book.copy_(was)
    else:
        assert lost > 0                                           # what the others gave back was enough
        pg.book.copy_(was)
        pool.copy_(bytes_was)
    gone = rng.random(B) < 0.5
    o.release(gone)
    ctx.pages_free(pg, torch.tensor(gone, dtype=torch.uint8, device=DEV))
    live = torch.zeros(1, dtype=torch.int32, device=DEV)
    n = o.compact()
    ctx.pages_compact(pg, [pool], live)
    assert live.item() == n
    assert np.array_equal(pg.table.cpu().numpy(), o.table()) and pg.refs.tolist() == o.refs()
    assert torch.equal(pool[:n, 0].cpu(), torch.tensor(o.data[:n], dtype=torch.int32))
    assert ctx.device_status()[0] == 0
    ctx.close()


FIRST_CALLS = """
import threading, torch
from paper_2412_00876_b200 import binding as dl

def one(H, Hk, D, B, ready, out, errors):
    try:
        torch.cuda.set_device(0)
        ctx = dl.Context(64, H, D, 64, torch.bfloat16, 0, max_batch=B, cap=64)
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            pg = dl.Pages(B, B, 1, 16)
            pool = ctx.kv4_pool(pg, Hk)
            q, k = torch.ones(B, H, D, device="cuda").bfloat16(), torch.ones(B, Hk, D, device="cuda").bfloat16()
            o = torch.zeros_like(q)
            s.synchronize()
            ready.wait()
            ctx.kv4_attn_decode(pg, pool, q, k, k, None, 0.1, o)
            s.synchronize()
        out.append(bool((o == 1).all()) and ctx.device_status()[0] == 0)
    except Exception as e:
        errors.append(repr(e))

for H, Hk, D in ((2, 2, 64), (2, 1, 64), (16, 1, 64), (2, 2, 128), (2, 1, 128), (16, 1, 128)):
    sizes = (1, 2000, 1, 2000, 300, 1, 2000, 600)
    ready, out, errors = threading.Barrier(len(sizes)), [], []
    threads = [threading.Thread(target=one, args=(H, Hk, D, B, ready, out, errors)) for B in sizes]
    for t in threads: t.start()
    for t in threads: t.join()
    assert not errors and out == [True] * len(sizes), (H, Hk, D, out, errors)
print("first calls agree")
"""


def test_first_calls_from_several_threads():
    """Batches of different sizes ask for different amounts of shared memory: the first calls of a form, from threads with a
    context and a stream each, must not leave a smaller limit behind one another's launches."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, cwd=root, timeout=300)
    assert r.returncode == 0 and "first calls agree" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]


@pytest.mark.parametrize("D,first", [(64, 128), (128, 128), (128, 300), (128, 40)])
def test_packed_rows_whose_first_keys_score_minus_infinity(D, first):
    """Keys of infinite size that score -inf for every query weigh nothing, however many come first; a row that sees no other
    is NaN."""
    H, Hk, n = 4, 2, 600
    dl, ctx = context(H, D)
    rng = np.random.default_rng(first)
    q, k, v = bf(rng, n, H, D), bf(rng, n, Hk, D), bf(rng, n, Hk, D)
    q[:, :, 0] = -1.0
    k[:first, :, 0] = np.inf
    out = torch.zeros((n, H, D), dtype=torch.bfloat16, device=DEV)
    ctx.attn_prefill_packed(up(q), up(k), up(v), i32([0, n]), n, D ** -0.5, out)
    got = wl.from_torch(out)
    assert np.isnan(got[:first]).all()
    args = q[first:], k[first:], v[first:], [0, n - first], D ** -0.5
    close(got[first:], pk.attention_packed(*args), pk.attention_packed(args[0], args[1], np.abs(args[2]), *args[3:]), "rows behind")
    assert ctx.device_status()[0] == 0
    ctx.close()
