"""CPU oracle for drafted tokens over a paged 16-bit cache (NOT in the paper): rotary positions, tree masks, attention of tree
nodes, verification of drafts, accepted rows.

Test infrastructure only: imported by tests/, never by the product.  Everything is written out from the definitions in
include/dl.h, in plain loops and fp64; verification, which is defined bit for bit, in Python's floats (fp64) and whole numbers.
"""
from __future__ import annotations

import math

import numpy as np


def turned(x, pos, freqs, interleaved, amplitude=1.0) -> np.ndarray:
    """Rows x [n][heads][D], pair by pair turned by pos * freqs[i]: fp64."""
    y = np.array(x, np.float64)
    half = len(freqs)
    for i, f in enumerate(freqs):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        for r, p in enumerate(pos):
            # the angle within one turn, in whole arithmetic of longer floats
            t = math.fmod(float(np.fmod(np.longdouble(int(p)) * np.longdouble(float(f)), 2 * np.longdouble(np.pi))), 2 * math.pi)
            c, s = amplitude * math.cos(t), amplitude * math.sin(t)
            u, v = np.array(x[r, :, a], np.float64), np.array(x[r, :, b], np.float64)
            y[r, :, a], y[r, :, b] = u * c - v * s, v * c + u * s
    return y


def tree_plan(parents, pos0, words):
    """mask words (uint32 [total][words]) and positions of every sequence's nodes"""
    mask, pos = [], []
    for p, first in zip(parents, pos0):
        depth = []
        for i, up in enumerate(p):
            row = np.zeros(words, np.uint32)
            if up >= 0:
                row[:] = mask[len(mask) - (i - up)]
            row[i // 32] |= np.uint32(1 << (i % 32))
            mask.append(row)
            depth.append(0 if up < 0 else depth[up] + 1)
            pos.append(first + depth[-1])
    return np.array(mask, np.uint32).reshape(-1, words), np.array(pos, np.int64)


def visible(mask_row, j) -> bool:
    return bool((int(mask_row[j // 32]) >> (j % 32)) & 1)


def attention_tree(q, k, v, held, mask, scale) -> np.ndarray:
    """One sequence: q [n][H][D]; k, v [held + n][Hk][D] (rows that are NaN all over have no page and are left out);
    mask uint32 [n][words] or None."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    G, n = q.shape[1] // k.shape[1], q.shape[0]
    out = np.zeros_like(q)
    there = ~np.isnan(k).all((1, 2))
    for i in range(n):
        see = [t for t in range(held + n)
               if there[t] and (t < held or (t - held <= i if mask is None else visible(mask[i], t - held)))]
        if not see:
            continue
        for h in range(q.shape[1]):
            z = (k[see, h // G] @ q[i, h]) * scale
            p = np.exp(z - z.max())
            out[i, h] = (p / p.sum()) @ v[see, h // G]
    return out


UNIT = 2.0 ** 44


def held01(x: float) -> float:
    return (x if x < 1.0 else 1.0) if x > 0.0 else 0.0


def number(u, last: float = 1.0 - 2.0 ** -24) -> float:
    """a random number held to [0, last]; NaN counts as 0"""
    return min(max(float(u), 0.0), last) if float(u) == float(u) else 0.0


def first_largest(row) -> int:
    best, at = -math.inf, 0
    for v, x in enumerate(row):
        x = float(x)
        if x > best:
            best, at = x, v
    return at


def verify(target, draft, u, tokens, parent, mode):
    """One sequence's tree; rows of `target` and `draft` float32.  Returns (kept flags, token drawn)."""
    n = len(parent)
    keep = [False] * n
    if n == 0:
        return keep, -1
    keep[0] = True
    V = len(target[0])
    at, s, R, a, dead = 0, 0.0, 1.0, 1.0, set()

    def left(s_):
        p = np.asarray(target[at], np.float64)
        if mode == "point":
            p = p.copy()
            p[list(dead)] = 0.0
            r = p
        else:
            r = p - np.float64(s_) * np.asarray(draft[at], np.float64)
        r = np.where(r > 0, np.minimum(r, 1.0), 0.0)
        return [int(x) for x in np.trunc(r * UNIT)]

    best = first_largest(target[0]) if mode == "greedy" else None
    for i in range(1, n):
        if parent[i] != at or not 0 <= parent[i] < i or not 0 <= tokens[i] < V:
            continue
        c = int(tokens[i])
        if mode == "greedy":
            yes = c == best
        elif mode == "point":
            p = 0.0 if c in dead else float(target[at][c])
            yes = number(u[i]) * R < p
            if not yes:
                R -= p
                dead.add(c)
        else:
            p, q = float(target[at][c]), float(draft[at][c])
            yes = a > 0.0 and (number(u[i]) * q) * R < held01(p - s * q) * a
            if not yes and a > 0.0:
                s = s + R / a
                R = float(sum(left(s))) / UNIT
                if mode == "sample":
                    a -= q
        if yes:
            keep[i] = True
            at, s, R, a, dead = i, 0.0, 1.0, 1.0, set()
            if mode == "greedy":
                best = first_largest(target[at])
    if mode == "greedy":
        return keep, best
    w = left(s)
    if sum(w) == 0:
        w = [int(held01(float(x)) * UNIT) for x in target[at]]
    W = sum(w)
    if W == 0:
        return keep, -1
    k = int(number(u[0], 1.0 - 2.0 ** -31) * 2.0 ** 31)
    bound, run = (k * W) >> 31, 0
    for v, x in enumerate(w):
        run += x
        if run > bound:
            return keep, v
    raise AssertionError("unreachable: the bound lies below the sum")
