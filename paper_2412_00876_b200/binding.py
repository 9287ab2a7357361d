"""ctypes binding of libdl_sparse.so: same names as include/dl.h, argument marshalling only.

Tensors are torch CUDA tensors (device memory and streams are torch's); every step of the
path runs in the library's kernels.  There is no fallback: if the library has not been
built the import of this module's `lib()` raises.
"""
from __future__ import annotations

import array
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# DL_SPARSE_CHECKED=1 in the environment selects the checked twin (stores through computed indices are compared with
# their buffers first; see include/dl.h)
LIB_PATH = os.path.join(_HERE, "libdl_sparse_checked.so" if os.environ.get("DL_SPARSE_CHECKED") == "1"
                        else "libdl_sparse.so")

DL_F32, DL_BF16 = 0, 1
DL_OK = 0
DL_ERR_INVALID_ARG, DL_ERR_ALIGNMENT, DL_ERR_UNSUPPORTED, DL_ERR_WORKSPACE = -1, -2, -3, -4
DL_ERR_CUDA, DL_ERR_CAPACITY, DL_ERR_TIMEOUT, DL_WARN_NAN = -5, -6, -7, 1
DL_ERR_BOUNDS = -8
DL_OPT_PREDICTOR_IMPL, DL_OPT_PREFILL_ATTN_IMPL, DL_OPT_DECODE_CHUNK, DL_OPT_DECODE_IMPL = 1, 2, 3, 4
DL_OPT_COMPACT_IMPL = 5

EXPORTS = [
    "dl_create", "dl_destroy", "dl_workspace_bytes", "dl_set_workspace", "dl_set_option",
    "dl_device_status", "dl_status_str", "dl_last_cuda_error", "dl_predictor_scores",
    "dl_topk_from_scores", "dl_prefill_select", "dl_compact_kv", "dl_sparse_attn_prefill",
    "dl_sparse_attn_decode", "dl_decode_keep", "dl_commit_len", "dl_decode_step", "dl_decode_step_host",
    "dl_sparse_attn_decode_static", "dl_sparse_attn_decode_layers", "dl_decode_nocache_select",
    "dl_decode_steps_host", "dl_compact_kv_host", "dl_selftest_wait_timeout", "dl_compact_kv_layers",
    "dl_predictor2_scratch_bytes", "dl_predictor2_values", "dl_prefill_select2", "dl_decode_keep2",
    "dl_decode_step_stack", "dl_quantize_kv_fp8", "dl_sparse_attn_decode_fp8", "dl_build_is_checked",
    "dl_selftest_bounds", "dl_sparse_attn_decode_fp8_layers",
    "dl_attn_prefill_packed", "dl_pages_scratch_bytes", "dl_pages_reserve", "dl_pages_free", "dl_pages_fork",
    "dl_pages_compact", "dl_kv4_page_bytes", "dl_kv4_append", "dl_kv4_read", "dl_kv4_attn_decode",
    "dl_rope_freqs", "dl_tree_plan", "dl_kv16_page_bytes", "dl_kv16_append", "dl_kv16_attn_tree", "dl_tree_verify",
    "dl_kv16_commit",
]
ROPE_SCALING = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}                        # DL_ROPE_*
VERIFY_MODES = {"greedy": 0, "sample": 1, "replaced": 2, "point": 3}                # DL_VERIFY_*


class ModelDesc(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32),
                ("pred_hidden", C.c_int32), ("dtype", C.c_int32)]


class LinearDesc(C.Structure):
    _fields_ = [("w", C.c_void_p), ("b", C.c_void_p)]


class VitBlockDesc(C.Structure):
    _fields_ = [("ln1_g", C.c_void_p), ("ln1_b", C.c_void_p), ("qkv", LinearDesc), ("proj", LinearDesc),
                ("ln2_g", C.c_void_p), ("ln2_b", C.c_void_p), ("fc1", LinearDesc), ("fc2", LinearDesc)]


class LayerStackDesc(C.Structure):
    _fields_ = [("L", C.c_int32), ("l_dense", C.c_int32), ("k_caches", C.POINTER(C.c_void_p)),
                ("v_caches", C.POINTER(C.c_void_p)), ("cap_dense", C.c_int32), ("cap", C.c_int32),
                ("len_dense", C.c_void_p), ("cache_len", C.c_void_p)]


class Predictor2Desc(C.Structure):
    _fields_ = [("inp", LinearDesc), ("n_blocks", C.c_int32), ("blocks", C.POINTER(VitBlockDesc)),
                ("h1", LinearDesc), ("h2", LinearDesc), ("w3", C.c_void_p), ("b3", C.c_void_p)]


class PagesDesc(C.Structure):
    _fields_ = [("B", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("page_rows", C.c_int32),
                ("table", C.c_void_p), ("refs", C.c_void_p), ("len", C.c_void_p)]


class Pages:
    """The books of a paged cache (dl_pages in dl.h) as device tensors: `table` [B, max_pages] (-1 where there is no
    page), `refs` [n_pages], `cache_len` [B], all int32 views of one tensor, `book`."""

    def __init__(self, B: int, n_pages: int, max_pages: int, page_rows: int, device="cuda"):
        self.B, self.n_pages, self.max_pages, self.page_rows = B, n_pages, max_pages, page_rows
        up = lambda n: (n + 3) // 4 * 4                              # 16-byte steps
        a, b = up(B * max_pages), up(n_pages)
        self.book = torch.zeros(a + b + up(B), dtype=torch.int32, device=device)
        self.table = self.book[:B * max_pages].view(B, max_pages)
        self.table.fill_(-1)
        self.refs = self.book[a:a + n_pages]
        self.cache_len = self.book[a + b:a + b + B]
        self.desc = PagesDesc(B, n_pages, max_pages, page_rows, self.table.data_ptr(), self.refs.data_ptr(),
                              self.cache_len.data_ptr())
        self.ref = C.pointer(self.desc)
        self._scratch = None

    def scratch(self, ctx: "Context") -> torch.Tensor:
        """Scratch of dl_pages_fork and dl_pages_compact, allocated at the first use."""
        if self._scratch is None:
            n = lib().dl_pages_scratch_bytes(ctx._h, self.ref)
            if n < 0:
                raise DlError(int(n), "dl_pages_scratch_bytes")
            self._scratch = torch.empty(max(int(n), 256), dtype=torch.uint8, device=self.book.device)
        return self._scratch


class RopeDesc(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("freqs", C.c_void_p), ("amplitude", C.c_float)]


def rope_freqs(rot_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, orig_len: int = 4096):
    """dl_rope_freqs: turning of the pairs per position (a float64 tensor of the host) and what rotated values are multiplied by."""
    freqs = torch.zeros(max(rot_dim // 2, 1), dtype=torch.float64)
    amplitude = C.c_double()
    st = lib().dl_rope_freqs(rot_dim, float(base), ROPE_SCALING[scaling], float(factor), int(orig_len), freqs.data_ptr(),
                             C.byref(amplitude))
    if st != DL_OK:
        raise DlError(st, "dl_rope_freqs")
    return freqs[:rot_dim // 2], amplitude.value


class Rope:
    """Rotary positions (dl_rope in dl.h): the first rot_dim dims of a head in half or interleaved layout, with frequencies by
    dl_rope_freqs or given (`freqs`, radians per position, and `amplitude`)."""

    def __init__(self, rot_dim: int, base: float = 10000.0, interleaved: bool = False, scaling: str = "none",
                 factor: float = 1.0, orig_len: int = 4096, freqs=None, amplitude: float = 1.0, device="cuda"):
        if freqs is None:
            freqs, amplitude = rope_freqs(rot_dim, base, scaling, factor, orig_len)
        freqs = torch.as_tensor(freqs, dtype=torch.float64)
        if freqs.shape != (rot_dim // 2,):
            raise ValueError(f"freqs: want {rot_dim // 2} of them, got {tuple(freqs.shape)}")
        self.freqs = freqs.to(device).contiguous()
        self.desc = RopeDesc(rot_dim, 1 if interleaved else 0, self.freqs.data_ptr(), amplitude)
        self.ref = C.pointer(self.desc)


class PredictorDesc(C.Structure):
    _fields_ = [("w1", C.c_void_p), ("b1", C.c_void_p), ("w2", C.c_void_p), ("b2", C.c_float)]


class Predictor2:
    """Device tensors of a predictor in the paper's architecture and the descriptor that points at them.
    `params` is the dictionary layout of workloads.make_predictor_paper with torch CUDA tensors as values
    (matrices bf16, vectors float32); the tensors are kept alive here."""

    def __init__(self, params: dict):
        self.params = params
        lin = lambda w, b: LinearDesc(w.data_ptr(), b.data_ptr())
        blocks = params["blocks"]
        self._blocks = (VitBlockDesc * max(len(blocks), 1))()
        for i, k in enumerate(blocks):
            self._blocks[i] = VitBlockDesc(k["ln1_g"].data_ptr(), k["ln1_b"].data_ptr(), lin(k["w_qkv"], k["b_qkv"]),
                                           lin(k["w_o"], k["b_o"]), k["ln2_g"].data_ptr(), k["ln2_b"].data_ptr(),
                                           lin(k["w_fc1"], k["b_fc1"]), lin(k["w_fc2"], k["b_fc2"]))
        h = params["head"]
        self.desc = Predictor2Desc(lin(params["w_in"], params["b_in"]), len(blocks),
                                   C.cast(self._blocks, C.POINTER(VitBlockDesc)), lin(h["w1"], h["b1"]),
                                   lin(h["w2"], h["b2"]), h["w3"].data_ptr(), h["b3"].data_ptr())


_lib = None


def lib() -> C.CDLL:
    """Opens the CUDA library (once).  Raises if it is missing: build it with
    `python -m paper_2412_00876_b200.build`."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} not found: run `python -m paper_2412_00876_b200.build` "
                               "(there is no CPU or PyTorch fallback)")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
        P = C.POINTER(PredictorDesc)
        sig = {
            "dl_create": (i32, [C.POINTER(vp), i32, C.POINTER(ModelDesc)]),
            "dl_destroy": (i32, [vp]),
            "dl_workspace_bytes": (i64, [vp, i32, i32, i32]),
            "dl_set_workspace": (i32, [vp, vp, i64, i32, i32, i32, vp]),
            "dl_set_option": (i32, [vp, i32, i32]),
            "dl_device_status": (i32, [vp, vp, C.POINTER(i32), C.POINTER(i64)]),
            "dl_status_str": (C.c_char_p, [i32]),
            "dl_last_cuda_error": (C.c_char_p, [vp]),
            "dl_predictor_scores": (i32, [vp, P, vp, i32, vp, vp]),
            "dl_topk_from_scores": (i32, [vp, vp, vp, vp, i32, i32, vp, i32, vp, vp]),
            "dl_prefill_select": (i32, [vp, P, vp, vp, vp, i32, i32, vp, vp, i32, vp, vp]),
            "dl_compact_kv": (i32, [vp, vp, vp, vp, i32, vp, i32, i32, vp, vp, i32, vp, i32, vp]),
            "dl_compact_kv_host": (i32, [vp, vp, vp, vp, i32, vp, i32, i32, vp, vp, i32, vp, i32, vp]),
            "dl_compact_kv_layers": (i32, [vp, i32, C.POINTER(vp), C.POINTER(vp), vp, i32, vp, i32, i32, i32, vp, i32, vp]),
            "dl_sparse_attn_prefill": (i32, [vp, vp, vp, vp, vp, i32, i32, i32, f32, vp, vp]),
            "dl_sparse_attn_decode": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, vp, vp]),
            "dl_sparse_attn_decode_static": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, vp, vp]),
            "dl_sparse_attn_decode_layers": (i32, [vp, i32, vp, vp, vp, C.POINTER(vp), C.POINTER(vp), vp, vp, i32, i32,
                                                  f32, vp, vp]),
            "dl_decode_keep": (i32, [vp, P, vp, i32, f32, vp, vp, vp]),
            "dl_selftest_wait_timeout": (i32, [vp, i32, vp]),
            "dl_predictor2_scratch_bytes": (i64, [vp, i64]),
            "dl_predictor2_values": (i32, [vp, C.POINTER(Predictor2Desc), vp, vp, i32, i32, vp, i64, vp, vp, vp, vp]),
            "dl_prefill_select2": (i32, [vp, C.POINTER(Predictor2Desc), vp, vp, vp, i32, i32, vp, i64, vp, vp, vp, i32,
                                         vp, vp]),
            "dl_decode_keep2": (i32, [vp, C.POINTER(Predictor2Desc), vp, i32, vp, i64, vp, vp, vp]),
            "dl_decode_nocache_select": (i32, [vp, P, vp, vp, i32, i32, f32, vp, vp, vp]),
            "dl_commit_len": (i32, [vp, vp, i32, i32, vp, vp]),
            "dl_decode_step": (i32, [vp, P, vp, i32, f32, vp, vp, i32, vp, vp, vp, C.POINTER(vp),
                                     C.POINTER(vp), i32, vp, f32, vp, vp]),
            "dl_decode_step_stack": (i32, [vp, P, vp, i32, f32, vp, vp, C.POINTER(LayerStackDesc), vp, vp, vp, f32,
                                           vp, vp]),
            "dl_sparse_attn_decode_fp8_layers": (i32, [vp, i32, vp, vp, vp, C.POINTER(vp), C.POINTER(vp), vp, vp, vp, vp,
                                                       i32, i32, f32, vp, i32, vp]),
            "dl_build_is_checked": (i32, []),
            "dl_selftest_bounds": (i32, [vp, vp]),
            "dl_quantize_kv_fp8": (i32, [vp, vp, vp, vp, i32, i32, vp, vp]),
            "dl_sparse_attn_decode_fp8": (i32, [vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, vp, vp]),
            "dl_attn_prefill_packed": (i32, [vp, vp, vp, vp, i64, i64, vp, i32, i32, i32, i32, f32, vp, vp]),
            "dl_pages_scratch_bytes": (i64, [vp, C.POINTER(PagesDesc)]),
            "dl_pages_reserve": (i32, [vp, C.POINTER(PagesDesc), vp, vp]),
            "dl_pages_free": (i32, [vp, C.POINTER(PagesDesc), vp, vp]),
            "dl_pages_fork": (i32, [vp, C.POINTER(PagesDesc), vp, i32, vp, i64, vp, i64, vp]),
            "dl_pages_compact": (i32, [vp, C.POINTER(PagesDesc), i32, vp, i64, vp, vp, i64, vp]),
            "dl_kv4_page_bytes": (i64, [vp, i32, i32]),
            "dl_kv4_append": (i32, [vp, C.POINTER(PagesDesc), i32, vp, vp, vp, i64, vp, vp, i32, i32, vp]),
            "dl_kv4_read": (i32, [vp, C.POINTER(PagesDesc), i32, vp, vp, vp, i32, vp, vp, vp]),
            "dl_kv4_attn_decode": (i32, [vp, C.POINTER(PagesDesc), i32, vp, vp, vp, vp, vp, f32, vp, vp]),
            "dl_rope_freqs": (i32, [i32, C.c_double, i32, C.c_double, i32, vp, C.POINTER(C.c_double)]),
            "dl_tree_plan": (i32, [vp, vp, vp, vp, i32, i32, i32, vp, vp, vp]),
            "dl_kv16_page_bytes": (i64, [vp, i32, i32]),
            "dl_kv16_append": (i32, [vp, C.POINTER(PagesDesc), i32, vp, vp, i64, vp, vp, i64, vp, C.POINTER(RopeDesc), vp, vp,
                                     i32, vp, i64, vp, i64, i32, vp]),
            "dl_kv16_attn_tree": (i32, [vp, C.POINTER(PagesDesc), i32, vp, vp, i64, vp, i32, i32, vp, i32, f32, vp, vp]),
            "dl_tree_verify": (i32, [vp, vp, i32, i64, vp, i64, vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp]),
            "dl_kv16_commit": (i32, [vp, C.POINTER(PagesDesc), i32, i32, vp, vp, vp, i32, vp]),
            "dl_decode_step_host": (i32, [vp, P, vp, i32, f32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                          vp, vp, C.POINTER(vp), C.POINTER(vp), i32, vp, f32, vp]),
            "dl_decode_steps_host": (i32, [vp, P, i32, i32, f32, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                           C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), vp, vp, vp, vp, vp, vp, vp,
                                           C.POINTER(vp), C.POINTER(vp), i32, vp, f32, vp]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


class DlError(RuntimeError):
    def __init__(self, code: int, where: str, extra: str = ""):
        self.code = code
        msg = lib().dl_status_str(code).decode()
        super().__init__(f"{where}: {msg} ({code}){' - ' + extra if extra else ''}")


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        if not t.is_contiguous():
            raise ValueError("tensor must be contiguous")
        return t.data_ptr()
    return int(t)


# raw handle of a device's current stream; the public call builds a Stream object around it, a few microseconds a call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _refuse(t, dtype, shape, what, index):
    raise ValueError(f"{what}: want a contiguous {dtype} {tuple(shape)} on cuda:{index}, got {t.dtype} {tuple(t.shape)} "
                     f"with strides {t.stride()} on {t.device}")


def _arg(t, dtype, shape, what: str, index: int) -> int:
    """Pointer of a tensor that the kernels read or write by this type and shape."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        _refuse(t, dtype, shape, what, index)
    return t.data_ptr()


def _rows(t, dtype, shape, what: str, index: int):
    """Pointer and row stride (in elements) of packed rows [rows, heads, D] whose last two dimensions are dense."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        _refuse(t, dtype, shape, what, index)
    s0, s1, s2 = t.stride()
    if s2 == 1 and s1 == shape[2] and s0 >= shape[1] * s1 and shape[0] > 1:          # (what nearly every call passes)
        return t.data_ptr(), s0
    if shape[0] > 0 and (s2 != 1 or (s1 != shape[2] and shape[1] > 1)):
        raise ValueError(f"{what}: want rows with dense heads, got strides {t.stride()}")
    if shape[0] > 1 and s0 < shape[1] * shape[2]:                    # (0 would mean dense rows to the library)
        raise ValueError(f"{what}: rows must not overlap, got strides {t.stride()}")
    return t.data_ptr(), (s0 if shape[0] > 1 else shape[1] * shape[2])


def _stream(stream=None):
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


class Predictor:
    """Device copy of one predictor's weights (see dl_predictor in dl.h)."""

    def __init__(self, w1: torch.Tensor, b1: torch.Tensor, w2: torch.Tensor, b2: float):
        assert b1.dtype == torch.float32 and w2.dtype == torch.float32
        self.w1, self.b1, self.w2, self.b2 = w1.contiguous(), b1.contiguous(), w2.contiguous(), float(b2)
        self.desc = PredictorDesc(self.w1.data_ptr(), self.b1.data_ptr(), self.w2.data_ptr(), self.b2)


class Context:
    """Owns a dl_ctx and the torch tensor that serves as its workspace."""

    def __init__(self, hidden: int, n_heads: int, head_dim: int, pred_hidden: int, dtype: torch.dtype,
                 device: int = 0, max_batch: int = 1, max_rows: int = 0, cap: int = 64):
        self._h = C.c_void_p()
        self.dtype = dtype
        self.device = torch.device("cuda", device)
        self.H, self.D, self.hidden = n_heads, head_dim, hidden
        d = ModelDesc(hidden, n_heads, head_dim, pred_hidden, DL_F32 if dtype == torch.float32 else DL_BF16)
        st = lib().dl_create(C.byref(self._h), device, C.byref(d))
        if st != DL_OK:
            raise DlError(st, "dl_create")
        self._ws = None
        self.set_workspace(max_batch, max(max_rows, max_batch), cap)

    def close(self):
        if self._h:
            lib().dl_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int, where: str):
        if st != DL_OK:
            extra = lib().dl_last_cuda_error(self._h).decode() if st == DL_ERR_CUDA else ""
            raise DlError(st, where, extra)

    # ---- context calls
    def set_workspace(self, max_batch: int, max_rows: int, cap: int, stream=None):
        n = lib().dl_workspace_bytes(self._h, max_batch, max_rows, cap)
        if n < 0:
            raise DlError(int(n), "dl_workspace_bytes")
        self._ws = torch.empty(int(n) + 256, dtype=torch.uint8, device=self.device)
        base = (self._ws.data_ptr() + 255) // 256 * 256
        self._check(lib().dl_set_workspace(self._h, base, n, max_batch, max_rows, cap, _stream(stream)),
                    "dl_set_workspace")
        self.max_batch, self.max_rows, self.cap = max_batch, max_rows, cap

    def set_option(self, option: int, value: int):
        self._check(lib().dl_set_option(self._h, option, value), "dl_set_option")

    def device_status(self, stream=None):
        code, detail = C.c_int32(0), C.c_int64(0)
        self._check(lib().dl_device_status(self._h, _stream(stream), C.byref(code), C.byref(detail)),
                    "dl_device_status")
        return code.value, detail.value

    # ---- the path
    def predictor_scores(self, p: Predictor, x, score_out, stream=None):
        rows = x.numel() // self.hidden
        self._check(lib().dl_predictor_scores(self._h, C.byref(p.desc), _ptr(x), rows, _ptr(score_out),
                                              _stream(stream)), "dl_predictor_scores")

    def topk_from_scores(self, score, n_vis, k, kept_idx_out, keep_out, stream=None):
        B, n_max = score.shape
        k_max = 0 if kept_idx_out is None else kept_idx_out.shape[1]
        self._check(lib().dl_topk_from_scores(self._h, _ptr(score), _ptr(n_vis), _ptr(k), B, n_max,
                                              _ptr(kept_idx_out), k_max, _ptr(keep_out), _stream(stream)),
                    "dl_topk_from_scores")

    def prefill_select(self, p: Predictor, x_vis, n_vis, k, score_out, kept_idx_out, keep_out, stream=None):
        B, n_max = x_vis.shape[0], x_vis.shape[1]
        k_max = 0 if kept_idx_out is None else kept_idx_out.shape[1]
        self._check(lib().dl_prefill_select(self._h, C.byref(p.desc), _ptr(x_vis), _ptr(n_vis), _ptr(k), B,
                                            n_max, _ptr(score_out), _ptr(kept_idx_out), k_max, _ptr(keep_out),
                                            _stream(stream)), "dl_prefill_select")

    def compact_kv(self, k_src, v_src, keep, t_src, k_cache, v_cache, cache_len, commit=True, stream=None):
        B, T = k_src.shape[0], k_src.shape[1]
        cap = k_cache.shape[2]
        keep_cols = 0 if keep is None else keep.shape[1]
        self._check(lib().dl_compact_kv(self._h, _ptr(k_src), _ptr(v_src), _ptr(keep), keep_cols, _ptr(t_src), B, T,
                                        _ptr(k_cache), _ptr(v_cache), cap, _ptr(cache_len), int(bool(commit)),
                                        _stream(stream)), "dl_compact_kv")

    def compact_kv_layers(self, srcs, caches, keep, t_src, cache_len, commit=True, stream=None):
        """dl_compact_kv_layers: len(srcs) tensors (K, V, Q ... of any number of layers) under one decision."""
        n = len(srcs)
        B, T = srcs[0].shape[0], srcs[0].shape[1]
        cap = caches[0].shape[2]
        keep_cols = 0 if keep is None else keep.shape[1]
        sp, cp = self.pointer_array(srcs), self.pointer_array(caches)
        self._check(lib().dl_compact_kv_layers(self._h, n, sp, cp, _ptr(keep), keep_cols, _ptr(t_src), B, T, cap,
                                               _ptr(cache_len), int(bool(commit)), _stream(stream)),
                    "dl_compact_kv_layers")

    def compact_kv_host(self, k_src_host, v_src_host, keep, t_src, k_cache, v_cache, cache_len, commit=True,
                        stream=None):
        """dl_compact_kv with the source rows in pinned host tensors: the kernel fetches the kept rows itself."""
        B, T = k_src_host.shape[0], k_src_host.shape[1]
        cap = k_cache.shape[2]
        keep_cols = 0 if keep is None else keep.shape[1]
        self._check(lib().dl_compact_kv_host(self._h, _ptr(k_src_host), _ptr(v_src_host), _ptr(keep), keep_cols,
                                             _ptr(t_src), B, T, _ptr(k_cache), _ptr(v_cache), cap, _ptr(cache_len),
                                             int(bool(commit)), _stream(stream)), "dl_compact_kv_host")

    def sparse_attn_prefill(self, q, k_cache, v_cache, cache_len, n_max, scale, out, stream=None):
        B, cap = k_cache.shape[0], k_cache.shape[2]
        self._check(lib().dl_sparse_attn_prefill(self._h, _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(cache_len),
                                                 B, cap, n_max, float(scale), _ptr(out), _stream(stream)),
                    "dl_sparse_attn_prefill")

    def sparse_attn_decode(self, q_t, k_t, v_t, k_cache, v_cache, cache_len, keep, scale, out, stream=None):
        B, cap = k_cache.shape[0], k_cache.shape[2]
        self._check(lib().dl_sparse_attn_decode(self._h, _ptr(q_t), _ptr(k_t), _ptr(v_t), _ptr(k_cache),
                                                _ptr(v_cache), _ptr(cache_len), _ptr(keep), B, cap, float(scale),
                                                _ptr(out), _stream(stream)), "dl_sparse_attn_decode")

    def selftest_bounds(self, stream=None):
        """Checked build: one store a word past a buffer's end, which must be skipped and recorded."""
        return lib().dl_selftest_bounds(self._h, _stream(stream))

    def quantize_kv_fp8(self, src, cache_len, scale, dst, stream=None):
        """Extension (not in the paper): rows of a bf16 cache as E4M3 bytes under per-head scales."""
        B, cap = src.shape[0], src.shape[2]
        self._check(lib().dl_quantize_kv_fp8(self._h, _ptr(src), _ptr(cache_len), _ptr(scale), B, cap, _ptr(dst),
                                             _stream(stream)), "dl_quantize_kv_fp8")

    def sparse_attn_decode_fp8(self, q_t, k_t, v_t, k_cache, v_cache, k_scale, v_scale, cache_len, keep, scale, out,
                               stream=None):
        B, cap = k_cache.shape[0], k_cache.shape[2]
        self._check(lib().dl_sparse_attn_decode_fp8(self._h, _ptr(q_t), _ptr(k_t), _ptr(v_t), _ptr(k_cache),
                                                    _ptr(v_cache), _ptr(k_scale), _ptr(v_scale), _ptr(cache_len),
                                                    _ptr(keep), B, cap, float(scale), _ptr(out), _stream(stream)),
                    "dl_sparse_attn_decode_fp8")

    def sparse_attn_decode_fp8_layers(self, q_t, k_t, v_t, k_caches, v_caches, k_scales, v_scales, cache_len, keep,
                                      scale, out, commit=False, stream=None):
        """k_caches / v_caches: lists of the L layers' byte caches; k_scales / v_scales [L][H]."""
        L, B, cap = len(k_caches), k_caches[0].shape[0], k_caches[0].shape[2]
        kp, vp_ = self.pointer_array(k_caches), self.pointer_array(v_caches)
        self._check(lib().dl_sparse_attn_decode_fp8_layers(
            self._h, L, _ptr(q_t), _ptr(k_t), _ptr(v_t), kp, vp_, _ptr(k_scales), _ptr(v_scales), _ptr(cache_len),
            _ptr(keep), B, cap, float(scale), _ptr(out), int(bool(commit)), _stream(stream)),
            "dl_sparse_attn_decode_fp8_layers")

    def sparse_attn_decode_static(self, q_t, k_t, v_t, k_cache, v_cache, cache_len, keep, scale, out, stream=None):
        """dl_sparse_attn_decode for callers that may not allocate device memory: the kernel's scratch
        is the library's built-in array (see dl.h for its size limit and the sharing rules)."""
        B, cap = k_cache.shape[0], k_cache.shape[2]
        self._check(lib().dl_sparse_attn_decode_static(self._h, _ptr(q_t), _ptr(k_t), _ptr(v_t), _ptr(k_cache),
                                                       _ptr(v_cache), _ptr(cache_len), _ptr(keep), B, cap,
                                                       float(scale), _ptr(out), _stream(stream)),
                    "dl_sparse_attn_decode_static")

    def sparse_attn_decode_layers(self, q_t, k_t, v_t, k_ptrs, v_ptrs, L, cap, cache_len, keep, scale, out,
                                  stream=None):
        B = cache_len.shape[0]
        self._check(lib().dl_sparse_attn_decode_layers(self._h, L, _ptr(q_t), _ptr(k_t), _ptr(v_t), k_ptrs, v_ptrs,
                                                       _ptr(cache_len), _ptr(keep), B, cap, float(scale), _ptr(out),
                                                       _stream(stream)), "dl_sparse_attn_decode_layers")

    def decode_keep(self, p: Predictor | None, x_t, logit_inout, keep_out, threshold=0.0, stream=None):
        B = logit_inout.shape[0]
        pd = C.byref(p.desc) if p is not None else None
        self._check(lib().dl_decode_keep(self._h, pd, _ptr(x_t), B, float(threshold), _ptr(logit_inout),
                                         _ptr(keep_out), _stream(stream)), "dl_decode_keep")

    def decode_nocache_select(self, p: Predictor | None, x_gen, n_gen, logit_inout, keep_out, threshold=0.0,
                              stream=None):
        B, n_max = logit_inout.shape
        pd = C.byref(p.desc) if p is not None else None
        self._check(lib().dl_decode_nocache_select(self._h, pd, _ptr(x_gen), _ptr(n_gen), B, n_max, float(threshold),
                                                   _ptr(logit_inout), _ptr(keep_out), _stream(stream)),
                    "dl_decode_nocache_select")

    def commit_len(self, keep, cache_len, cap, stream=None):
        self._check(lib().dl_commit_len(self._h, _ptr(keep), keep.shape[0], cap, _ptr(cache_len),
                                        _stream(stream)), "dl_commit_len")

    # ---- the paper's own predictors
    def predictor2_scratch(self, rows: int) -> torch.Tensor:
        """Scratch tensor of the size dl_predictor2_values wants for `rows` rows."""
        n = lib().dl_predictor2_scratch_bytes(self._h, int(rows))
        if n < 0:
            raise DlError(int(n), "dl_predictor2_scratch_bytes")
        return torch.empty(max(int(n), 256), dtype=torch.uint8, device=self.device)

    def predictor2_values(self, p: "Predictor2", x, n_vis, scratch, d_out=None, score_out=None, keep_out=None, stream=None):
        B, n_max = x.shape[0], x.shape[1]
        self._check(lib().dl_predictor2_values(self._h, C.byref(p.desc), _ptr(x), _ptr(n_vis), B, n_max, _ptr(scratch),
                                               scratch.numel(), _ptr(d_out), _ptr(score_out), _ptr(keep_out),
                                               _stream(stream)), "dl_predictor2_values")

    def prefill_select2(self, p: "Predictor2", x_vis, n_vis, k, scratch, d_out, score_out, kept_idx_out, keep_out,
                        stream=None):
        B, n_max = x_vis.shape[0], x_vis.shape[1]
        self._check(lib().dl_prefill_select2(self._h, C.byref(p.desc), _ptr(x_vis), _ptr(n_vis), _ptr(k), B, n_max,
                                             _ptr(scratch), scratch.numel(), _ptr(d_out), _ptr(score_out),
                                             _ptr(kept_idx_out), kept_idx_out.shape[1], _ptr(keep_out), _stream(stream)),
                    "dl_prefill_select2")

    def decode_keep2(self, p: "Predictor2", x_t, scratch, d_out, keep_out, stream=None):
        self._check(lib().dl_decode_keep2(self._h, C.byref(p.desc), _ptr(x_t), x_t.shape[0], _ptr(scratch),
                                          scratch.numel(), _ptr(d_out), _ptr(keep_out), _stream(stream)),
                    "dl_decode_keep2")

    # ---- packed prompts, pages, the 4-bit cache (extensions, not in the paper)
    # These check type, shape and device of every tensor, and the books' device; without `stream` they use the current one
    # of the context's device.
    def _on(self, stream):
        return _raw_stream(self.device.index) if stream is None else stream.cuda_stream

    def _books(self, pages: Pages):
        """The books for the library, which follows their pointers on the context's device."""
        if pages.book.get_device() != self.device.index:
            raise ValueError(f"pages: want books on cuda:{self.device.index}, got {pages.book.device}")
        return pages.ref

    def attn_prefill_packed(self, q, k, v, starts, max_rows, scale, out, stream=None):
        """dl_attn_prefill_packed: q [total, n_heads, D], k / v [total, n_kv_heads, D] (parts of one projection's output
        will do: rows may be strided), starts int32 [B + 1], max_rows: length of the longest sequence."""
        total, n_kv, D, i = q.shape[0], k.shape[1], self.D, self.device.index
        qp, qs = _rows(q, self.dtype, (total, self.H, D), "q", i)
        kp, ks = _rows(k, self.dtype, (total, n_kv, D), "k", i)
        vp, vs = _rows(v, self.dtype, (total, n_kv, D), "v", i)
        if ks != vs:
            raise ValueError("k and v must have the same row stride")
        n = starts.shape[0]
        self._check(lib().dl_attn_prefill_packed(
            self._h, qp, kp, vp, qs, ks, _arg(starts, torch.int32, (n,), "starts", i), n - 1, n_kv, total, max_rows, scale,
            _arg(out, self.dtype, (total, self.H, D), "out", i), self._on(stream)), "dl_attn_prefill_packed")

    def pages_reserve(self, pages: Pages, need, stream=None):
        """dl_pages_reserve: need int32 [B]."""
        self._check(lib().dl_pages_reserve(
            self._h, self._books(pages), _arg(need, torch.int32, (pages.B,), "need", self.device.index), self._on(stream)),
            "dl_pages_reserve")

    def pages_free(self, pages: Pages, gone, stream=None):
        """dl_pages_free: gone uint8 [B]."""
        self._check(lib().dl_pages_free(
            self._h, self._books(pages), _arg(gone, torch.uint8, (pages.B,), "gone", self.device.index), self._on(stream)),
            "dl_pages_free")

    def _pools(self, pages: Pages, pools):
        """Count, array of pointers and bytes of a page of `pools`, tensors [n_pages, ...] that are alike."""
        if not pools:
            return 0, None, 0
        n_bytes, index = pools[0].nbytes, self.device.index
        for p in pools:
            if p.nbytes != n_bytes or not p.is_contiguous() or p.get_device() != index:
                raise ValueError(f"pools: want contiguous tensors of one size on cuda:{index}")
        if pools[0].shape[0] != pages.n_pages:
            raise ValueError(f"pools: want {pages.n_pages} pages, got {tuple(pools[0].shape)}")
        ptrs = array.array("Q", [p.data_ptr() for p in pools])
        return len(ptrs), ptrs, n_bytes // pages.n_pages

    def pages_fork(self, pages: Pages, parent, pools, stream=None):
        """dl_pages_fork: parent int32 [B]; pools: list of tensors [n_pages, ...], one per layer."""
        books = self._books(pages)
        n, ptrs, page_bytes = self._pools(pages, pools)
        scratch = pages.scratch(self)
        self._check(lib().dl_pages_fork(
            self._h, books, _arg(parent, torch.int32, (pages.B,), "parent", self.device.index), n,
            ptrs.buffer_info()[0] if n else None, page_bytes, scratch.data_ptr(), scratch.shape[0], self._on(stream)),
            "dl_pages_fork")

    def pages_compact(self, pages: Pages, pools, n_live=None, stream=None):
        """dl_pages_compact; n_live: int32 tensor [1] for the number of pages in use, or None."""
        books = self._books(pages)
        n, ptrs, page_bytes = self._pools(pages, pools)
        scratch = pages.scratch(self)
        live = None if n_live is None else _arg(n_live, torch.int32, (1,), "n_live", self.device.index)
        self._check(lib().dl_pages_compact(self._h, books, n, ptrs.buffer_info()[0] if n else None, page_bytes, live,
                                           scratch.data_ptr(), scratch.shape[0], self._on(stream)), "dl_pages_compact")

    def kv4_page_bytes(self, n_kv_heads: int, page_rows: int) -> int:
        n = lib().dl_kv4_page_bytes(self._h, n_kv_heads, page_rows)
        if n < 0:
            raise DlError(int(n), "dl_kv4_page_bytes")
        return int(n)

    def kv4_pool(self, pages: Pages, n_kv_heads: int) -> torch.Tensor:
        """A pool of 4-bit pages (uint8 [n_pages, page bytes]) for these books."""
        return torch.zeros(pages.n_pages, self.kv4_page_bytes(n_kv_heads, pages.page_rows), dtype=torch.uint8,
                           device=pages.book.device)

    def _pool(self, pages: Pages, pool, n_kv: int) -> int:
        return _arg(pool, torch.uint8, (pages.n_pages, n_kv * pages.page_rows * 9 * self.D // 8), "pool", self.device.index)

    def kv4_append(self, pages: Pages, pool, k, v, starts, keep=None, commit=True, stream=None):
        """dl_kv4_append: k, v [total, n_kv_heads, D] bf16 (rows may be strided), starts int32 [B + 1], keep uint8 [total]."""
        total, n_kv, i = k.shape[0], k.shape[1], self.device.index
        kp, ks = _rows(k, self.dtype, (total, n_kv, self.D), "k", i)
        vp, vs = _rows(v, self.dtype, (total, n_kv, self.D), "v", i)
        if ks != vs:
            raise ValueError("k and v must have the same row stride")
        self._check(lib().dl_kv4_append(
            self._h, self._books(pages), n_kv, self._pool(pages, pool, n_kv), kp, vp, ks,
            _arg(starts, torch.int32, (pages.B + 1,), "starts", i),
            None if keep is None else _arg(keep, torch.uint8, (total,), "keep", i), total, 1 if commit else 0,
            self._on(stream)), "dl_kv4_append")

    def kv4_read(self, pages: Pages, pool, row0, starts, k_out, v_out, stream=None):
        """dl_kv4_read: rows from row0[b] on of every sequence into k_out, v_out [total, n_kv_heads, D] bf16."""
        total, n_kv, i = k_out.shape[0], k_out.shape[1], self.device.index
        shape = (total, n_kv, self.D)
        self._check(lib().dl_kv4_read(
            self._h, self._books(pages), n_kv, self._pool(pages, pool, n_kv),
            _arg(row0, torch.int32, (pages.B,), "row0", i), _arg(starts, torch.int32, (pages.B + 1,), "starts", i), total,
            _arg(k_out, self.dtype, shape, "k_out", i), _arg(v_out, self.dtype, shape, "v_out", i), self._on(stream)),
            "dl_kv4_read")

    def kv4_attn_decode(self, pages: Pages, pool, q_t, k_t, v_t, keep, scale, out, stream=None):
        """dl_kv4_attn_decode: q_t, out [B, n_heads, D]; k_t, v_t [B, n_kv_heads, D]; keep uint8 [B] or None."""
        n_kv, B, i = k_t.shape[1], pages.B, self.device.index
        big, small = (B, self.H, self.D), (B, n_kv, self.D)
        self._check(lib().dl_kv4_attn_decode(
            self._h, self._books(pages), n_kv, self._pool(pages, pool, n_kv),
            _arg(q_t, self.dtype, big, "q_t", i), _arg(k_t, self.dtype, small, "k_t", i),
            _arg(v_t, self.dtype, small, "v_t", i),
            None if keep is None else _arg(keep, torch.uint8, (B,), "keep", i), scale,
            _arg(out, self.dtype, big, "out", i), self._on(stream)), "dl_kv4_attn_decode")

    # ---- drafted tokens over a paged 16-bit cache (extension, not in the paper)
    def kv16_page_bytes(self, n_kv_heads: int, page_rows: int) -> int:
        n = lib().dl_kv16_page_bytes(self._h, n_kv_heads, page_rows)
        if n < 0:
            raise DlError(int(n), "dl_kv16_page_bytes")
        return int(n)

    def kv16_pool(self, pages: Pages, n_kv_heads: int) -> torch.Tensor:
        """A pool of 16-bit pages (bf16 [n_pages, K and V, n_kv_heads, page_rows, D]) for these books."""
        self.kv16_page_bytes(n_kv_heads, pages.page_rows)
        return torch.zeros(pages.n_pages, 2, n_kv_heads, pages.page_rows, self.D, dtype=self.dtype, device=pages.book.device)

    def _pool16(self, pages: Pages, pool, n_kv: int) -> int:
        return _arg(pool, self.dtype, (pages.n_pages, 2, n_kv, pages.page_rows, self.D), "pool", self.device.index)

    def tree_plan(self, parent, starts, pos0, mask_out, pos_out=None, stream=None):
        """dl_tree_plan: parent int32 [total], starts int32 [B + 1], pos0 int32 [B] or None; mask_out int32 [total, words],
        pos_out int32 [total] or None."""
        i, total, B = self.device.index, parent.shape[0], starts.shape[0] - 1
        words = mask_out.shape[1]
        self._check(lib().dl_tree_plan(
            self._h, _arg(parent, torch.int32, (total,), "parent", i), _arg(starts, torch.int32, (B + 1,), "starts", i),
            None if pos0 is None else _arg(pos0, torch.int32, (B,), "pos0", i), B, total, words,
            _arg(mask_out, torch.int32, (total, words), "mask_out", i),
            None if pos_out is None else _arg(pos_out, torch.int32, (total,), "pos_out", i), self._on(stream)), "dl_tree_plan")

    def _rope(self, rope):
        """The rotation for the library, which follows the pointer of its frequencies on the context's device."""
        if rope is None:
            return None
        if rope.freqs.get_device() != self.device.index:
            raise ValueError(f"rope: want frequencies on cuda:{self.device.index}, got {rope.freqs.device}")
        return rope.ref

    def kv16_append(self, pages, pool, q, k, v, starts, pos, rope, keep=None, q_out=None, k_out=None, commit=True, stream=None):
        """dl_kv16_append: q [total, n_heads, D] with q_out (or both None), k, v [total, n_kv_heads, D], k_out like k or None, all
        bf16 (rows may be strided); pos int32 [total]; rope: a Rope or None; starts int32 [B + 1]; keep uint8 [total] or None.
        pages, pool and v None: the rotation alone."""
        total, n_kv, i = k.shape[0], k.shape[1], self.device.index
        big, small, none = (total, self.H, self.D), (total, n_kv, self.D), (None, 0)
        kp, ks = _rows(k, self.dtype, small, "k", i)
        vp, vs = _rows(v, self.dtype, small, "v", i) if v is not None else (None, ks)
        if ks != vs:
            raise ValueError("k and v must have the same row stride")
        qp, qs = _rows(q, self.dtype, big, "q", i) if q is not None else none
        qop, qos = _rows(q_out, self.dtype, big, "q_out", i) if q_out is not None else none
        kop, kos = _rows(k_out, self.dtype, small, "k_out", i) if k_out is not None else none
        if (pages is None) != (pool is None) or (pages is not None and v is None):
            raise ValueError("pages, pool and v go together")
        self._check(lib().dl_kv16_append(
            self._h, None if pages is None else self._books(pages), n_kv, None if pool is None else self._pool16(pages, pool, n_kv),
            qp, qs, kp, vp, ks, None if pos is None else _arg(pos, torch.int32, (total,), "pos", i), self._rope(rope),
            None if pages is None else _arg(starts, torch.int32, (pages.B + 1,), "starts", i),
            None if keep is None else _arg(keep, torch.uint8, (total,), "keep", i), total, qop, qos, kop, kos,
            1 if commit else 0, self._on(stream)), "dl_kv16_append")

    def kv16_attn_tree(self, pages: Pages, pool, q, starts, max_rows, mask, scale, out, stream=None):
        """dl_kv16_attn_tree: q [total, n_heads, D] (rows may be strided), starts int32 [B + 1], max_rows: most nodes of a
        sequence; mask int32 [total, words] or None (each node sees those in front of it and itself); out [total, n_heads, D]."""
        total, n_kv, i = q.shape[0], pool.shape[2], self.device.index
        qp, qs = _rows(q, self.dtype, (total, self.H, self.D), "q", i)
        words = 0 if mask is None else mask.shape[1]
        self._check(lib().dl_kv16_attn_tree(
            self._h, self._books(pages), n_kv, self._pool16(pages, pool, n_kv), qp, qs,
            _arg(starts, torch.int32, (pages.B + 1,), "starts", i), total, max_rows,
            None if mask is None else _arg(mask, torch.int32, (total, words), "mask", i), words, scale,
            _arg(out, self.dtype, (total, self.H, self.D), "out", i), self._on(stream)), "dl_kv16_attn_tree")

    def _dist(self, t, dtype, total, what):
        """Pointer and row stride of rows [total, vocab] whose entries lie side by side."""
        if t.dtype is not dtype or t.dim() != 2 or t.shape[0] != total or t.get_device() != self.device.index:
            raise ValueError(f"{what}: want {dtype} [{total}, vocab] on cuda:{self.device.index}, got {t.dtype} {tuple(t.shape)} "
                             f"on {t.device}")
        if total > 0 and (t.stride(1) != 1 or (total > 1 and t.stride(0) < t.shape[1])):
            raise ValueError(f"{what}: want dense rows that do not overlap, got strides {t.stride()}")
        return t.data_ptr(), (t.stride(0) if total > 1 else t.shape[1])

    def tree_verify(self, target, draft, u, tokens, parent, starts, mode, keep_out, count_out, next_out, stream=None):
        """dl_tree_verify: target [total, vocab] float32 (mode "greedy": or bf16), draft like it (modes "sample" and "replaced")
        or None, u float32 [total] (None for "greedy"), tokens and parent int32 [total], starts int32 [B + 1]; keep_out uint8
        [total], count_out and next_out int32 [B]."""
        i, total, B = self.device.index, tokens.shape[0], starts.shape[0] - 1
        code = VERIFY_MODES[mode]
        drafted = mode in ("sample", "replaced")
        dtype = torch.bfloat16 if mode == "greedy" and target.dtype is torch.bfloat16 else torch.float32
        tp, ts = self._dist(target, dtype, total, "target")
        vocab = target.shape[1]
        dp, ds = None, 0
        if drafted:
            dp, ds = self._dist(draft, torch.float32, total, "draft")
            if draft.shape[1] != vocab:
                raise ValueError(f"draft: want a vocabulary of {vocab}, got {draft.shape[1]}")
        self._check(lib().dl_tree_verify(
            self._h, tp, DL_BF16 if dtype is torch.bfloat16 else DL_F32, ts, dp, ds,
            None if mode == "greedy" else _arg(u, torch.float32, (total,), "u", i), _arg(tokens, torch.int32, (total,), "tokens", i),
            _arg(parent, torch.int32, (total,), "parent", i), _arg(starts, torch.int32, (B + 1,), "starts", i), B, total, vocab, code,
            _arg(keep_out, torch.uint8, (total,), "keep_out", i), _arg(count_out, torch.int32, (B,), "count_out", i),
            _arg(next_out, torch.int32, (B,), "next_out", i), self._on(stream)), "dl_tree_verify")

    def kv16_commit(self, pages: Pages, pools, starts, keep, stream=None):
        """dl_kv16_commit: pools: the list of all layers' pools; starts int32 [B + 1]; keep uint8 [total]."""
        i, total = self.device.index, keep.shape[0]
        books = self._books(pages)
        n_kv = pools[0].shape[2] if pools else 1
        ptrs = array.array("Q", [self._pool16(pages, p, n_kv) for p in pools])
        self._check(lib().dl_kv16_commit(
            self._h, books, n_kv, len(ptrs), ptrs.buffer_info()[0] if pools else None,
            _arg(starts, torch.int32, (pages.B + 1,), "starts", i), _arg(keep, torch.uint8, (total,), "keep", i), total,
            self._on(stream)), "dl_kv16_commit")

    def selftest_wait_timeout(self, polls: int = 64, stream=None):
        self._check(lib().dl_selftest_wait_timeout(self._h, int(polls), _stream(stream)), "dl_selftest_wait_timeout")

    @staticmethod
    def pointer_array(tensors):
        arr = (C.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
        return arr

    def decode_step(self, p: Predictor | None, x_t, logit_inout, keep_out, q_t, k_t, v_t, k_ptrs, v_ptrs, L,
                    cap, cache_len, scale, out, threshold=0.0, stream=None):
        B = logit_inout.shape[0]
        pd = C.byref(p.desc) if p is not None else None
        self._check(lib().dl_decode_step(self._h, pd, _ptr(x_t), B, float(threshold), _ptr(logit_inout),
                                         _ptr(keep_out), L, _ptr(q_t), _ptr(k_t), _ptr(v_t), k_ptrs, v_ptrs, cap,
                                         _ptr(cache_len), float(scale), _ptr(out), _stream(stream)),
                    "dl_decode_step")

    def decode_step_stack(self, p: Predictor | None, x_t, logit_inout, keep_out, k_caches, v_caches, l_dense,
                          cap_dense, cap, len_dense, cache_len, q_t, k_t, v_t, scale, out, threshold=0.0,
                          stream=None):
        """One decode step over a stack whose first l_dense layers keep every token (k_caches / v_caches: lists of
        the L layers' cache tensors)."""
        B, L = logit_inout.shape[0], len(k_caches)
        kp = (C.c_void_p * max(L, 1))(*[t.data_ptr() for t in k_caches])
        vp_ = (C.c_void_p * max(L, 1))(*[t.data_ptr() for t in v_caches])
        st = LayerStackDesc(L, l_dense, kp, vp_, cap_dense, cap, _ptr(len_dense), _ptr(cache_len))
        pd = C.byref(p.desc) if p is not None else None
        self._check(lib().dl_decode_step_stack(self._h, pd, _ptr(x_t), B, float(threshold), _ptr(logit_inout),
                                               _ptr(keep_out), C.byref(st), _ptr(q_t), _ptr(k_t), _ptr(v_t),
                                               float(scale), _ptr(out), _stream(stream)), "dl_decode_step_stack")

    def decode_steps_host(self, p: Predictor, x_hosts, q_hosts, k_hosts, v_hosts, out_hosts, keep_hosts, stage_x,
                          stage_q, stage_k, stage_v, stage_out, logit_dev, keep_dev, k_ptrs, v_ptrs, L, cap,
                          cache_len, scale, threshold=0.0, stream=None):
        """len(x_hosts) decode steps fed from (pinned) host tensors, copies pipelined against the compute;
        the staging tensors hold two sets each (leading dimension 2)."""
        n = len(x_hosts)
        B = logit_dev.shape[-1]
        arr = lambda ts: (C.c_void_p * n)(*[(t.data_ptr() if t is not None else None) for t in ts])
        keep_arr = arr(keep_hosts) if keep_hosts is not None else None
        self._check(lib().dl_decode_steps_host(
            self._h, C.byref(p.desc), n, B, float(threshold), L, arr(x_hosts), arr(q_hosts), arr(k_hosts),
            arr(v_hosts), arr(out_hosts), keep_arr, _ptr(stage_x), _ptr(stage_q), _ptr(stage_k), _ptr(stage_v),
            _ptr(stage_out), _ptr(logit_dev), _ptr(keep_dev), k_ptrs, v_ptrs, cap, _ptr(cache_len), float(scale),
            _stream(stream)), "dl_decode_steps_host")

    def decode_step_host(self, p: Predictor, x_host, q_host, k_host, v_host, out_host, keep_host, stage_x,
                         stage_q, stage_k, stage_v, stage_out, logit_dev, keep_dev, k_ptrs, v_ptrs, L, cap,
                         cache_len, scale, threshold=0.0, stream=None):
        B = logit_dev.shape[0]
        self._check(lib().dl_decode_step_host(
            self._h, C.byref(p.desc), _ptr(x_host), B, float(threshold), L, _ptr(q_host), _ptr(k_host),
            _ptr(v_host), _ptr(out_host), _ptr(keep_host), _ptr(stage_x), _ptr(stage_q), _ptr(stage_k),
            _ptr(stage_v), _ptr(stage_out), _ptr(logit_dev), _ptr(keep_dev), k_ptrs, v_ptrs, cap,
            _ptr(cache_len), float(scale), _stream(stream)), "dl_decode_step_host")
