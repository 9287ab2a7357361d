"""CPU oracle for the serving extensions (NOT in the paper): packed prompts with grouped heads, a cache in pages, rows held
in 4 bits.

Test infrastructure only: imported by tests/, never by the product.  Everything is written out from the definitions in
include/dl.h, in plain loops and fp64; where a definition names 32-bit steps (the codes of a 4-bit row) those are taken
in float32.
"""
from __future__ import annotations

import numpy as np

GROUP = 64
TINY = np.float32(2.0 ** -126)


def bf16(x) -> np.ndarray:
    """float32 values rounded to bf16 (nearest, ties to even); finite inputs."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)


def quantise(x):
    """Rows [..., D] of bf16 values -> codes [..., D] (0..15), s and z [..., D / 64] (float32, exact in bf16)."""
    x = np.asarray(x, dtype=np.float32)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    lo, hi = g.min(-1), g.max(-1)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        span = (hi - lo).astype(np.float32)
        odd = ~np.isfinite(g).all(-1) | ~np.isfinite(span)
        s = bf16(np.where(odd, np.float32(0), span) / np.float32(15))
        inv = np.where(s >= TINY, np.float32(1) / s, np.float32(0)).astype(np.float32)
        t = np.where(odd[..., None], np.float32(0), ((g - lo[..., None]).astype(np.float32) * inv[..., None]).astype(np.float32))
    code = np.where(s[..., None] >= TINY, np.clip(np.rint(t), 0, 15), 0).astype(np.uint8)
    z = np.where(odd, np.float32(np.nan), lo)
    return code.reshape(x.shape), np.where(odd, np.float32(0), s), z


def values(code, s, z) -> np.ndarray:
    """float64 values that codes stand for"""
    g = np.asarray(code, np.float64).reshape(*code.shape[:-1], code.shape[-1] // GROUP, GROUP)
    return (s.astype(np.float64)[..., None] * g + z.astype(np.float64)[..., None]).reshape(code.shape)


def held(x) -> np.ndarray:
    return values(*quantise(x))


def attention_packed(q, k, v, starts, scale) -> np.ndarray:
    """Causal attention of packed rows; q [T][H][D], k, v [T][Hkv][D]; rows of no sequence come back as zero."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    G = q.shape[1] // k.shape[1]
    out = np.zeros_like(q)
    for a, e in zip(starts, starts[1:]):
        for h in range(q.shape[1]):
            for i in range(a, e):
                z = (k[a:i + 1, h // G] @ q[i, h]) * scale
                p = np.exp(z - z.max())
                out[i, h] = (p / p.sum()) @ v[a:i + 1, h // G]
    return out


def attention_decode(q, k_t, v_t, k_rows, v_rows, scale) -> np.ndarray:
    """Eq. 6 for one sequence: q [H][D] attends k_rows, v_rows [n][Hkv][D] (values) and the token's own k_t, v_t [Hkv][D]."""
    q = np.asarray(q, np.float64)
    k = np.concatenate([np.asarray(k_rows, np.float64), np.asarray(k_t, np.float64)[None]])
    v = np.concatenate([np.asarray(v_rows, np.float64), np.asarray(v_t, np.float64)[None]])
    G = q.shape[0] // k.shape[1]
    out = np.empty_like(q)
    for h in range(q.shape[0]):
        z = (k[:, h // G] @ q[h]) * scale
        p = np.exp(z - z.max())
        out[h] = (p / p.sum()) @ v[:, h // G]
    return out


class Books:
    """Pages as plain lists: pages[b] the page numbers of sequence b, length[b] its rows; data[p] whatever page p holds."""

    def __init__(self, n_pages: int, page_rows: int, width: int, pages, length, data):
        self.n_pages, self.page_rows, self.width = n_pages, page_rows, width
        self.pages, self.length, self.data = [list(p) for p in pages], list(length), list(data)

    def refs(self):
        r = [0] * self.n_pages
        for row in self.pages:
            for p in row:
                r[p] += 1
        return r

    def free(self):
        return [p for p, r in enumerate(self.refs()) if r == 0]

    def table(self):
        return np.array([row + [-1] * (self.width - len(row)) for row in self.pages], np.int32).reshape(-1, self.width)

    def _need(self, rows: int) -> int:
        return -(-rows // self.page_rows)

    def reserve(self, need) -> bool:
        add = [max(0, self._need(n + max(0, m)) - len(row)) for n, m, row in zip(self.length, need, self.pages)]
        if any(self._need(n + max(0, m)) > self.width for n, m in zip(self.length, need)) or sum(add) > len(self.free()):
            return False
        free = self.free()
        for row, c in zip(self.pages, add):
            row += free[:c]
            free = free[c:]
        return True

    def release(self, gone):
        for b, g in enumerate(gone):
            if g:
                self.pages[b], self.length[b] = [], 0

    def fork(self, parent) -> bool:
        old, old_len, old_data = [list(p) for p in self.pages], list(self.length), list(self.data)
        copies = []
        for b, p in enumerate(parent):
            if p == b:
                continue
            self.pages[b] = old[p][:self._need(old_len[p])] if p >= 0 else []
            self.length[b] = old_len[p] if p >= 0 else 0
            holder = p if p >= 0 and parent[p] == p else min(c for c in range(len(parent)) if parent[c] == p)
            if p >= 0 and old_len[p] % self.page_rows and holder != b:
                copies.append(b)
        for b in copies:
            self.pages[b][-1] = None
        used = {p for row in self.pages for p in row if p is not None}
        free = [p for p in range(self.n_pages) if p not in used]
        if len(free) < len(copies):
            self.pages, self.length = old, old_len
            return False
        for b, d in zip(copies, free):
            src = old[parent[b]][self._need(old_len[parent[b]]) - 1]
            self.pages[b][-1] = d
            self.data[d] = old_data[src]
        return True

    def compact(self) -> int:
        refs = self.refs()
        live = sum(r > 0 for r in refs)
        movers = [p for p in range(live, self.n_pages) if refs[p] > 0]
        holes = [p for p in range(live) if refs[p] == 0]
        new = dict(zip(movers, holes))
        for s, d in new.items():
            self.data[d] = self.data[s]
        self.pages = [[new.get(p, p) for p in row] for row in self.pages]
        return live
