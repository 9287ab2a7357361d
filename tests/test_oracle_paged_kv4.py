"""Pins of the serving oracle (oracle/paged_kv4.py) against what the definitions and the mathematics fix, and the refusals of
the serving entry points that need no GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_kv4 as pk


def row(values):
    """64 bf16 values that begin with `values`, the rest between their extremes"""
    x = np.full(64, np.float32(values[0]))
    x[:len(values)] = values
    return x[None]


def test_codes_of_whole_steps_are_exact():
    x = row(np.arange(16))
    code, s, z = pk.quantise(x)
    assert s[0, 0] == 1 and z[0, 0] == 0 and np.array_equal(code[0, :16], np.arange(16))
    assert np.array_equal(pk.held(x), x)
    # the same shifted and scaled by powers of two
    code, s, z = pk.quantise(x * 0.25 - 8)
    assert s[0, 0] == 0.25 and z[0, 0] == -8 and np.array_equal(code[0, :16], np.arange(16))


def test_ties_go_to_the_even_code_and_both_ends_are_reached():
    code, s, _ = pk.quantise(row([0, 15, 0.5, 1.5, 2.5, 14.5]))
    assert s[0, 0] == 1 and code[0, :6].tolist() == [0, 15, 0, 2, 2, 14]


def test_a_constant_group_has_no_scale_and_a_spoilt_one_is_nan():
    code, s, z = pk.quantise(row([1.5]))
    assert s[0, 0] == 0 and z[0, 0] == 1.5 and not code.any()
    for bad in (np.nan, np.inf, -np.inf):
        x = np.concatenate([row([bad, 1]), row([1, 2])], 1)
        v = pk.held(x)
        assert np.isnan(v[0, :64]).all() and np.isfinite(v[0, 64:]).all()
    big = np.float32(3e38)
    assert np.isnan(pk.held(row([-big, big]))).all()               # a range beyond float32


def test_error_is_at_most_half_a_step():
    rng = np.random.default_rng(0)
    x = pk.bf16((rng.normal(0, 1, (200, 128)) * 2.0 ** rng.integers(-8, 8, (200, 1))).astype(np.float32))
    code, s, _ = pk.quantise(x)
    step = np.repeat(s.astype(np.float64), 64, -1)
    # s is (max - min) / 15 rounded to bf16 (2^-8 relative at most): the largest value can lie 15 * 2^-8 steps past code 15
    assert np.all(np.abs(pk.held(x) - x) <= step * (0.5 + 15 * 2.0 ** -8))
    assert code.max() == 15 and code.min() == 0


def test_packed_attention_is_plain_causal_attention_of_each_sequence():
    rng = np.random.default_rng(1)
    q, k, v = rng.normal(size=(9, 4, 8)), rng.normal(size=(9, 2, 8)), rng.normal(size=(9, 2, 8))
    out = pk.attention_packed(q, k, v, [0, 4, 4, 7], 0.3)
    assert not out[7:].any()
    for a, e in ((0, 4), (4, 7)):
        assert np.allclose(out[a], np.repeat(v[a], 2, 0))            # the first row sees itself alone
        for h in range(4):
            z = q[a:e, h] @ k[a:e, h // 2].T * 0.3
            z[np.triu_indices(e - a, 1)] = -np.inf
            p = np.exp(z)
            assert np.allclose(out[a:e, h], (p / p.sum(1, keepdims=True)) @ v[a:e, h // 2])


def test_decode_attention_of_no_rows_is_the_tokens_own_value():
    rng = np.random.default_rng(2)
    q, kt, vt = rng.normal(size=(4, 8)), rng.normal(size=(2, 8)), rng.normal(size=(2, 8))
    none = np.zeros((0, 2, 8))
    assert np.allclose(pk.attention_decode(q, kt, vt, none, none, 0.5), np.repeat(vt, 2, 0))


def books(pages, length, n_pages=8, page_rows=16, width=4):
    return pk.Books(n_pages, page_rows, width, pages, length, list(range(n_pages)))


def test_reserve_gives_the_lowest_free_pages_or_nothing():
    b = books([[3], []], [16, 0])
    assert b.reserve([1, 20]) and b.pages == [[3, 0], [1, 2]]
    assert not b.reserve([64, 0]) and b.pages == [[3, 0], [1, 2]]    # five pages, four columns
    assert b.reserve([40, 40]) and b.pages == [[3, 0, 4, 5], [1, 2, 6]]
    b = books([[3], []], [16, 0], n_pages=6)
    assert not b.reserve([40, 40]) and b.free() == [0, 1, 2, 4, 5]   # three and three more pages, five are free


def test_fork_shares_full_pages_and_copies_partial_ones():
    b = books([[0, 1], [2]], [20, 5])
    assert b.fork([0, 0]) and b.pages == [[0, 1], [0, 2]] and b.length == [20, 20]
    assert b.data[2] == 1 and b.refs()[:3] == [2, 1, 1]             # page 2, given back by the call, holds the copy
    # nobody stays: the lowest child takes the partial page over
    b = books([[0, 1], [], []], [20, 0, 0])
    assert b.fork([-1, 0, 0]) and b.pages == [[], [0, 1], [0, 2]] and b.length == [0, 20, 20]
    b = books([[0], []], [5, 0], n_pages=1)
    assert not b.fork([0, 0]) and b.pages == [[0], []]


def test_compact_moves_the_highest_pages_down_in_order():
    b = books([[6, 2], [7]], [20, 3])
    assert b.compact() == 3
    assert b.pages == [[0, 2], [1]] and b.data[:3] == [6, 7, 2]


# ---- refusals without a GPU
def test_entry_points_refuse_a_missing_context():
    from paper_2412_00876_b200 import binding as dl
    lib, d = dl.lib(), dl.PagesDesc(1, 1, 1, 16, None, None, None)
    bad = dl.DL_ERR_INVALID_ARG
    assert lib.dl_attn_prefill_packed(None, None, None, None, 0, 0, None, 1, 1, 1, 1, 1.0, None, None) == bad
    assert lib.dl_pages_scratch_bytes(None, C.byref(d)) == bad
    assert lib.dl_pages_reserve(None, C.byref(d), None, None) == bad
    assert lib.dl_pages_free(None, C.byref(d), None, None) == bad
    assert lib.dl_pages_fork(None, C.byref(d), None, 0, None, 0, None, 0, None) == bad
    assert lib.dl_pages_compact(None, C.byref(d), 0, None, 0, None, None, 0, None) == bad
    assert lib.dl_kv4_page_bytes(None, 1, 16) == bad
    assert lib.dl_kv4_append(None, C.byref(d), 1, None, None, None, 0, None, None, 1, 1, None) == bad
    assert lib.dl_kv4_read(None, C.byref(d), 1, None, None, None, 1, None, None, None) == bad
    assert lib.dl_kv4_attn_decode(None, C.byref(d), 1, None, None, None, None, None, 1.0, None, None) == bad


def test_books_are_views_of_one_tensor_at_16_byte_steps():
    from paper_2412_00876_b200 import binding as dl
    for B, n, w in ((1, 1, 1), (3, 5, 7), (8, 33, 2)):
        pg = dl.Pages(B, n, w, 32, device="cpu")
        assert pg.table.shape == (B, w) and pg.refs.shape == (n,) and pg.cache_len.shape == (B,)
        assert bool((pg.table == -1).all()) and not pg.refs.any() and not pg.cache_len.any()
        assert all(t.data_ptr() % 16 == pg.book.data_ptr() % 16 for t in (pg.refs, pg.cache_len))
        pg.refs.fill_(1), pg.cache_len.fill_(2)
        assert bool((pg.table == -1).all()) and bool((pg.refs == 1).all())


@pytest.mark.parametrize("t,what", [
    (torch.zeros(4, dtype=torch.int64), "type"), (torch.zeros(5, dtype=torch.int32), "shape"),
    (torch.zeros(8, dtype=torch.int32)[::2], "strides"), (torch.zeros(4, dtype=torch.int32), "device")])
def test_tensors_of_another_kind_are_refused(t, what):
    from paper_2412_00876_b200 import binding as dl
    with pytest.raises(ValueError, match="starts"):
        dl._arg(t, torch.int32, (4,), "starts", 0)
