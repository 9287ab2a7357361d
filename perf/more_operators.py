"""Drafted tokens over a paged 16-bit K/V cache, as measured work: appending rows to the cache with the position rotation on
the way, attention for trees of drafted tokens (and for chunks of a prompt, and single tokens) over it, verification of
the drafts against the target's probabilities, and keeping the accepted rows.

`run` computes them in plain form (elementary torch operations) or, where `own` is true, with the calls a user makes of
this library.  Conventions of the plain form, which are the operators' definitions:

  rotation     the first `rot` dims of a head are rot / 2 pairs, (i, i + rot / 2) in half layout or (2 i, 2 i + 1) interleaved;
               pair i of a row at position p turns by p * f_i and is multiplied by `amplitude`;
               f_i = base^(-2 i / rot), or scaled for long contexts (`_frequencies`).
  pages        a pool is [n_pages][K, V][kv heads][page rows][dim] bf16; row t of sequence b is row t % page of its page
               table[b][t / page].  `len` rows are held; drafted rows lie behind them until they are accepted.
  trees        a sequence's new rows are its nodes; node 0 is the last token that is certain, parent[i] < i; a row sees all rows
               held and the nodes whose bits are set in its mask (a tree: itself and its ancestors).
  verification node by node in index order: a node whose parent is the node reached so far is tested, and becomes the node
               reached if it is accepted.  With p the target's distribution there, q the draft's, and at first s = 0, R = 1, a = 1:
                 accepted iff  a > 0  and  (u * q(token)) * R < r(token) * a,   r(v) = p(v) - s * q(v) held to 0..1,
                 else, if a > 0:  s += R / a,  R = sum of r under the new s,  a -= q(token) (unless drawn with replacement);
               tokens chosen without randomness:  accepted iff u * R < p(token), else R -= p(token), p(token) = 0;
               greedily: accepted iff the token is the target's first largest.
               At the end a token is drawn from what r is there by the root's number (from p if nothing is left of it).
               All in 64-bit floats, sums over r in units of 2^-44 cut off, so that they are whole numbers: the first v
               whose running sum exceeds (trunc(u * 2^31) * sum) >> 31.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
UNIT = 2.0 ** 44


# ---- cases ----------------------------------------------------------------------------------------------------------
def listed():
    return [
        # a batch of prompts behind the selection: 144 of 576 image tokens kept, at the positions they had, then the text
        dict(name="append_selected", op="append", seqs=32, lo=660, hi=704, heads=32, kv=32, dim=128, page=64, sizes=2,
             what="kept", masked=576, keep=0.25, before=0, rot=128, inter=False, scaling="none", factor=1.0, far=0),
        # chunks of long prompts: queries and keys rotated for the attention among them, rows appended; half of each head, scaled
        dict(name="append_long", op="append", seqs=6, lo=2900, hi=5000, heads=32, kv=8, dim=128, page=32, sizes=3, what="all",
             before=77, rot=64, inter=True, scaling="parts", factor=8.0, far=100000),
        # one or two users' trees early in a conversation: latency
        dict(name="attend_few", op="attend", seqs=2, lo=100, hi=400, n_lo=1, n_hi=8, heads=16, kv=4, dim=64, page=16, sizes=4,
             causal=False),
        # a serving batch half way through its 1024 generated tokens, every head its own, trees of up to 26 nodes
        dict(name="attend_serving", op="attend", seqs=32, lo=272, hi=1296, n_lo=20, n_hi=26, heads=32, kv=32, dim=128, page=64,
             sizes=5, causal=False),
        # few sequences over very long contexts, grouped heads, larger trees
        dict(name="attend_long", op="attend", seqs=4, lo=60000, hi=131072, n_lo=32, n_hi=48, heads=32, kv=4, dim=128, page=64,
             sizes=6, causal=False),
        # a decode step without drafts: one token each, contexts of all lengths
        dict(name="attend_single", op="attend", seqs=48, lo=500, hi=9000, n_lo=1, n_hi=1, heads=32, kv=8, dim=128, page=32,
             sizes=7, causal=True),
        # the next chunks of prompts whose first ones are in the cache
        dict(name="attend_chunk", op="attend", seqs=4, lo=3000, hi=8000, n_lo=900, n_hi=1100, heads=32, kv=8, dim=128, page=128,
             sizes=8, causal=True),
        # one user's chain of drafts: latency
        dict(name="verify_few", op="verify", seqs=1, n_lo=5, n_hi=5, vocab=32000, sizes=9, mode="sample", chain=True, bits=32),
        # trees of a serving batch, drawn from the draft's distribution
        dict(name="verify_serving", op="verify", seqs=48, n_lo=40, n_hi=64, vocab=32000, sizes=10, mode="sample", chain=False,
             bits=32),
        # the same at temperature 0, straight from the logits
        dict(name="verify_greedy", op="verify", seqs=48, n_lo=20, n_hi=26, vocab=32000, sizes=11, mode="greedy", chain=False,
             bits=16),
        # what a step does to the caches of a few layers: the trees' masks and positions, nodes appended, accepted rows kept
        dict(name="accept_serving", op="accept", seqs=32, lo=272, hi=900, n_lo=20, n_hi=26, heads=32, kv=8, dim=128, page=64,
             sizes=12, layers=4, rot=128, inter=False, scaling="linear", factor=4.0, far=2000),
        # the same for two users on a small model: latency
        dict(name="accept_few", op="accept", seqs=2, lo=100, hi=400, n_lo=3, n_hi=8, heads=16, kv=4, dim=64, page=16, sizes=13,
             layers=2, rot=64, inter=False, scaling="none", factor=1.0, far=0),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "verify", "verify", "accept"])
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 5, 8, 16, 32])
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 5, 6, 7, 8, 12, 16) if kv * g <= 40])
    case = dict(op=op, heads=heads, kv=kv, dim=dim, sizes=rng.randrange(1, 1 << 30), page=rng.choice([16, 32, 64, 128]))
    if op in ("append", "accept"):
        case.update(rot=rng.choice([r for r in (16, 32, 64, 96, 128) if r <= dim]), inter=rng.random() < 0.5,
                    scaling=rng.choice(["none", "linear", "ntk", "parts"]), far=rng.choice([0, 1000, 100000, 1000000]))
        case["factor"] = 1.0 if case["scaling"] == "none" else rng.choice([2.0, 4.0, 8.0, 32.0])
    if op == "append":
        what = rng.choice(["tree", "kept", "all"])
        hi = _log(rng, 2, 64) if what == "tree" else _log(rng, 2, 5000)
        most = 23000 * 48 * 128 // (hi * (heads + 2 * kv) * dim)
        case.update(what=what, seqs=max(1, min(_log(rng, 1, 48), most)), lo=max(1, int(hi * rng.random())), hi=hi,
                    before=rng.choice([0, rng.randrange(1, 200)]))
        if what == "kept":
            case.update(masked=int(hi * rng.random()), keep=rng.choice([0.0, 0.25, 0.5]))
    elif op == "attend":
        form = rng.choice(["single", "tree", "tree", "chunk"])
        n_hi = {"single": 1, "tree": _log(rng, 2, 90), "chunk": _log(rng, 64, 2000)}[form]
        hi = _log(rng, 2, 100000)
        rows = 400000 * 4 * 128 // (kv * dim)                                    # as much cache as the largest listed case
        flops = 3.4e11 // (4.0 * dim * heads * n_hi)                            # and as many products
        case.update(seqs=max(1, int(min(_log(rng, 1, 96), rows // (hi + n_hi), flops // (hi + n_hi)))), lo=int(hi * rng.random()),
                    hi=hi, n_lo=max(1, int(n_hi * rng.random())), n_hi=n_hi, causal=form != "tree")
        if hi + n_hi > min(rows, flops):
            case.update(hi=int(min(rows, flops)) // 2, lo=min(case["lo"], int(min(rows, flops)) // 2))
    elif op == "verify":
        vocab, n_hi = _log(rng, 300, 130000), _log(rng, 1, 64)
        mode = rng.choice(["sample", "sample", "replaced", "point", "greedy"])
        most = 48 * 60 * 32000 // (vocab * n_hi)
        case = dict(op=op, sizes=case["sizes"], vocab=vocab, n_hi=n_hi, n_lo=max(1, int(n_hi * rng.random())), mode=mode,
                    seqs=max(1, min(_log(rng, 1, 64), most)), chain=rng.random() < 0.3,
                    bits=rng.choice([16, 32]) if mode == "greedy" else 32)
    else:
        hi = _log(rng, 20, 1000)
        n_hi = _log(rng, 2, 40)
        case.update(kv=min(kv, 8), heads=heads if kv <= 8 else 8, seqs=rng.randrange(1, 40), hi=hi, lo=int(hi * rng.random()),
                    n_hi=n_hi, n_lo=max(1, int(n_hi * rng.random())), layers=rng.randrange(1, 5))
    return case


def _lens(case):
    """rows held by every sequence (or new rows, of an append)"""
    r = random.Random(case["sizes"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]


def _nodes(case):
    r = random.Random(case["sizes"] + 1)
    return [r.randint(case["n_lo"], case["n_hi"]) for _ in range(case["seqs"])]


def _parents(case, counts):
    """parents of every sequence's nodes: node i hangs on any earlier one (or on the one before it)"""
    r = random.Random(case["sizes"] + 2)
    return [[-1] + [i - 1 if case.get("chain") else r.randrange(i) for i in range(1, n)] for n in counts]


def _kept_counts(case):
    if case.get("what") != "kept":
        return _lens(case)
    return [round(min(n, case["masked"]) * case["keep"]) + max(0, n - case["masked"]) for n in _lens(case)]


def _accepted(case, counts):
    """a path from the root, of every sequence's tree: the nodes on it"""
    r = random.Random(case["sizes"] + 3)
    got = []
    for p in _parents(case, counts):
        path, at = [0], 0
        for i in range(1, len(p)):
            if p[i] == at and r.random() < 0.7:
                path.append(i)
                at = i
        got.append(path)
    return got


def work(case):
    op = case["op"]
    if op == "verify":
        # one row at least of every sequence's, of the target and where it takes part of the draft
        rows = 2 if case["mode"] in ("sample", "replaced") else 1
        return {"bytes": case["seqs"] * case["vocab"] * rows * case["bits"] // 8 + 12 * sum(_nodes(case)),
                "flops": 2 * case["seqs"] * case["vocab"]}
    D, H, Hk = case["dim"], case["heads"], case["kv"]
    if op == "append":
        q = 0 if case["what"] == "kept" else H * sum(_lens(case))
        k_too = Hk * sum(_lens(case)) if case["what"] == "all" else 0          # the rotated keys, packed
        rows = sum(_kept_counts(case))
        return {"bytes": 2 * D * (2 * q + k_too + 4 * Hk * rows) + 4 * sum(_lens(case)), "flops": 3 * case["rot"] * (q + Hk * rows)}
    n = _nodes(case)
    if op == "attend":
        held = _lens(case)
        rows = sum(held) + sum(n)
        seen = sum(a * b for a, b in zip(held, n))
        if case["causal"]:
            seen += sum(c * (c + 1) // 2 for c in n)
        else:
            seen += sum(_depth_sum(p) for p in _parents(case, n))
        return {"bytes": 2 * D * (2 * Hk * rows + 2 * H * sum(n)), "flops": 4 * D * H * seen}
    moved = sum(sum(i != r for r, i in enumerate(path)) for path in _accepted(case, n))
    return {"bytes": 2 * D * case["layers"] * (2 * H * sum(n) + 4 * Hk * (sum(n) + moved)) + 12 * sum(n), "flops": 3 * case["rot"] * (H + Hk) * sum(n)}


def _depth_sum(parent):
    d = []
    for p in parent:
        d.append(1 if p < 0 else d[p] + 1)
    return sum(d)


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + stream) % (1 << 62))
    return g


def _normal(shape, seed, stream, dtype=torch.bfloat16):
    return torch.randn(shape, generator=_gen(seed, stream), device=DEV, dtype=torch.float32).to(dtype)


def _starts(lens):
    c = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return torch.from_numpy(c).to(DEV), int(c[-1])


def _i32(v):
    return torch.from_numpy(np.ascontiguousarray(v, np.int32)).to(DEV)


def _mask_words(parents, words):
    """bit j of a row: node j is the row's own or an ancestor"""
    rows = []
    for p in parents:
        own_rows = np.zeros((len(p), words), np.uint32)
        for i, up in enumerate(p):
            if up >= 0:
                own_rows[i] = own_rows[up]
            own_rows[i, i // 32] |= np.uint32(1 << (i % 32))
        rows.append(own_rows)
    return np.concatenate(rows).view(np.int32)


def _frequencies(case):
    """turning of the pairs per position, in radians, and what the rotated values are multiplied by"""
    rot, base, factor = case["rot"], 10000.0, case["factor"]
    if case["scaling"] == "ntk" and rot > 2:
        base *= factor ** (rot / (rot - 2.0))
    f = base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    amplitude = 1.0
    if case["scaling"] == "linear":
        f = f / factor
    elif case["scaling"] == "parts":
        part = np.clip((4096 * f / (2 * math.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        f = f * (part + (1.0 - part) / factor)
        amplitude = 0.1 * math.log(factor) + 1.0
    return f, amplitude


def _rope(case):
    from paper_2412_00876_b200 import binding as dl
    return dl.Rope(case["rot"], base=10000.0, interleaved=case["inter"], scaling=case["scaling"], factor=case["factor"],
                   orig_len=4096, device=DEV)


def _context(case):
    from paper_2412_00876_b200 import binding as dl
    return dl.Context(64, case.get("heads", 1), case.get("dim", 64), 64, torch.bfloat16, 0, max_batch=case["seqs"], cap=64)


def _table(counts, width, n_pages, seed):
    order = np.random.RandomState(int(seed) % (1 << 31)).permutation(n_pages)
    t, at = np.full((len(counts), width), -1, np.int32), 0
    for b, c in enumerate(counts):
        t[b, :c] = order[at:at + c]
        at += c
    return t


def _pages(s, case, rows, held, seed):
    """the books of `rows` rows a sequence, of which `held` are there; returns the number of pages"""
    counts = [-(-n // case["page"]) for n in rows]
    n_pages, width = sum(counts) + 3, max(max(counts), 1) + 1
    table = _table(counts, width, n_pages, seed)
    if own:
        from paper_2412_00876_b200 import binding as dl
        s["pages"] = dl.Pages(case["seqs"], n_pages, width, case["page"], DEV)
        s["pages"].table.copy_(_i32(table))
        s["pages"].cache_len.copy_(held)
    s["table"], s["held"] = _i32(table), held
    return n_pages


def _tree_draft(case, seed):
    """target and draft probabilities (or logits) of every node, and tokens: each node's children drawn from its draft"""
    counts, V = _nodes(case), case["vocab"]
    parents = _parents(case, counts)
    starts = np.concatenate([[0], np.cumsum(counts)])
    total = int(starts[-1])
    z = 2.5 * _normal((total, V), seed, 1, torch.float32)
    zq = z + 0.7 * _normal((total, V), seed, 2, torch.float32)
    kids, rank = np.zeros(total, np.int64), np.zeros(total, np.int64)
    up = np.full(total, -1, np.int64)
    for b, p in enumerate(parents):
        for i in range(1, len(p)):
            up[starts[b] + i] = starts[b] + p[i]
            rank[starts[b] + i] = kids[starts[b] + p[i]]
            kids[starts[b] + p[i]] += 1
    noise = torch.rand((total, V), generator=_gen(seed, 3), device=DEV).clamp_(1e-9, 1 - 1e-7)
    best = (zq - torch.log(-torch.log(noise))).topk(max(1, min(V, int(kids.max()))), dim=1).indices
    del noise
    if case["mode"] == "greedy":
        best = zq.topk(max(1, min(V, int(kids.max()))), dim=1).indices            # the draft's likeliest tokens
    rank = np.minimum(rank, best.shape[1] - 1)
    tokens = best[torch.from_numpy(np.maximum(up, 0)).to(DEV), torch.from_numpy(rank).to(DEV)].int()
    x = {"parents": parents, "counts": counts, "tokens": tokens, "u": torch.rand(total, generator=_gen(seed, 4), device=DEV)}
    if case["mode"] == "greedy":
        x["target"], x["draft"] = (z.to(torch.bfloat16) if case["bits"] == 16 else z), None
        return x
    for name, v in (("target", z), ("draft", zq)):
        v -= v.amax(1, keepdim=True)
        v.exp_()
        v /= v.sum(1, keepdim=True)
        x[name] = v
    if case["mode"] == "point":
        x["draft"] = None
    return x


def _inputs(case, seed):
    """Tensors of one case, the same for the plain form, the library's calls and the 64-bit values."""
    op = case["op"]
    if op == "verify":
        return _tree_draft(case, seed)
    D, H, Hk = case["dim"], case["heads"], case["kv"]
    x = {}
    if op == "append":
        lens = x["lens"] = _lens(case)
        x["starts"], total = _starts(lens)
        x["qkv"] = _normal((total, H + 2 * Hk, D), seed, 1)                      # as one projection emits them
        first = np.random.RandomState(int(seed) % (1 << 31)).randint(0, case["far"] + 1, case["seqs"])
        if case["what"] == "tree":
            x["parents"] = _parents(case, lens)
            x["pos0"] = _i32(first)
        else:
            x["pos"] = _i32(np.concatenate([f + np.arange(n) for f, n in zip(first, lens)]))
        x["keep"], x["kept"] = None, _kept_counts(case)
        if case["what"] == "kept":
            keep, at = np.ones(total, np.uint8), 0
            r = np.random.RandomState((int(seed) + 1) % (1 << 31))
            for n, kept in zip(lens, x["kept"]):
                m = min(n, case["masked"])
                keep[at:at + m] = 0
                keep[at + r.permutation(m)[:kept - (n - m)]] = 1
                at += n
            x["keep"] = torch.from_numpy(keep).to(DEV)
        return x
    x["lens"], x["nodes"] = _lens(case), _nodes(case)
    x["starts"], total = _starts(x["nodes"])
    if op == "attend":
        x["q"] = _normal((total, H, D), seed, 1)
        x["parents"] = None if case["causal"] else _parents(case, x["nodes"])
        return x
    x["qkv"] = _normal((case["layers"], total, H + 2 * Hk, D), seed, 1)
    keep = np.zeros(total, np.uint8)
    at = 0
    for n, path in zip(x["nodes"], _accepted(case, x["nodes"])):
        keep[[at + i for i in path]] = 1
        at += n
    x["keep"] = torch.from_numpy(keep).to(DEV)
    x["parents"] = _parents(case, x["nodes"])
    x["pos0"] = _i32(np.random.RandomState(int(seed) % (1 << 31)).randint(0, case["far"] + 1, case["seqs"]))
    return x


def _depths(parent):
    d = []
    for p in parent:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _plan_buffers(s, counts):
    s["counts"], s["words"] = counts, -(-max(counts) // 32)
    s["parent"] = _i32(np.concatenate([np.array(p) for p in s["parents"]]))
    s["pos"] = torch.zeros(sum(counts), dtype=torch.int32, device=DEV)
    s["mask"] = torch.zeros(sum(counts), s["words"], dtype=torch.int32, device=DEV)


def prepare(case, seed):
    s = {"case": dict(case), **_inputs(case, seed)}
    op, B = case["op"], case["seqs"]
    if op == "verify":
        s["parent"] = _i32(np.concatenate([np.array(p) for p in s["parents"]]))
        s["starts"], total = _starts(s["counts"])
        if own:
            s["ctx"] = _context(case)
            s["keep"] = torch.zeros(total, dtype=torch.uint8, device=DEV)
            s["count"], s["next"] = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2))
        return s
    D, H, Hk, page = case["dim"], case["heads"], case["kv"], case["page"]
    if op == "append":
        s["before"] = torch.full((B,), case["before"], dtype=torch.int32, device=DEV)
        n_pages = _pages(s, case, [case["before"] + k for k in s["kept"]], s["before"], seed)
        total = sum(s["lens"])
        s["q"], s["k"], s["v"] = s["qkv"][:, :H], s["qkv"][:, H:H + Hk], s["qkv"][:, H + Hk:]
        if case["what"] == "tree":
            _plan_buffers(s, s["lens"])
        s["q_out"] = None if case["what"] == "kept" else torch.zeros(total, H, D, dtype=torch.bfloat16, device=DEV)
        s["k_out"] = torch.zeros(total, Hk, D, dtype=torch.bfloat16, device=DEV) if case["what"] == "all" else None
        s["pool"] = torch.zeros(n_pages, 2, Hk, page, D, dtype=torch.bfloat16, device=DEV)
    elif op == "attend":
        s["held_list"] = s["lens"]
        n_pages = _pages(s, case, [a + n for a, n in zip(s["lens"], s["nodes"])], _i32(s["lens"]), seed)
        s["pool"] = _normal((n_pages, 2, Hk, page, D), seed, 5)
        s["pool"][:, :, :, :, : D // 8] *= 2.0                                   # some channels stand out, as keys' do
        s["mask"] = None
        if s["parents"] is not None:
            s["mask"] = torch.from_numpy(_mask_words(s["parents"], -(-max(s["nodes"]) // 32))).to(DEV)
        s["out"] = torch.empty_like(s["q"])
        s["scale"] = D ** -0.5
    else:
        _plan_buffers(s, s["nodes"])
        n_pages = _pages(s, case, [a + n for a, n in zip(s["lens"], s["nodes"])], _i32(s["lens"]), seed)
        s["pool"] = _normal((case["layers"], n_pages, 2, Hk, page, D), seed, 5)
        s["q_out"] = torch.zeros(case["layers"], s["qkv"].shape[1], H, D, dtype=torch.bfloat16, device=DEV)
    if own:
        s["ctx"] = _context(case)
        if op != "attend":
            s["rope"] = _rope(case)
    elif op != "attend":
        f, s["amplitude"] = _frequencies(case)
        s["freqs"] = torch.from_numpy(f).to(DEV)
    return s


# ---- the library's calls --------------------------------------------------------------------------------------------
def _run_own(s):
    case, ctx, op = s["case"], s["ctx"], s["case"]["op"]
    if op == "verify":
        ctx.tree_verify(s["target"], s["draft"], s["u"], s["tokens"], s["parent"], s["starts"], case["mode"], s["keep"], s["count"],
                        s["next"])
        return {"keep": s["keep"], "count": s["count"], "next": s["next"]}
    pg = s["pages"]
    if op == "attend":
        ctx.kv16_attn_tree(pg, s["pool"], s["q"], s["starts"], max(s["nodes"]), s["mask"], s["scale"], s["out"])
        return s["out"]
    if op == "append":
        pg.cache_len.copy_(s["before"])                          # the same lengths in front of every pass
        got = {}
        if case["what"] == "tree":
            ctx.tree_plan(s["parent"], s["starts"], s["pos0"], s["mask"], s["pos"])
            got.update(mask=s["mask"], pos=s["pos"])
        ctx.kv16_append(pg, s["pool"], s["q"] if s["q_out"] is not None else None, s["k"], s["v"], s["starts"], s["pos"], s["rope"],
                        keep=s["keep"], q_out=s["q_out"], k_out=s["k_out"], commit=case["what"] != "tree")
        got.update(len=pg.cache_len, pool=s["pool"], **{n: s[n] for n in ("q_out", "k_out") if s[n] is not None})
        return got
    pg.cache_len.copy_(s["held"])
    H, Hk = case["heads"], case["kv"]
    ctx.tree_plan(s["parent"], s["starts"], s["pos0"], s["mask"], s["pos"])
    for layer in range(case["layers"]):
        x = s["qkv"][layer]
        ctx.kv16_append(pg, s["pool"][layer], x[:, :H], x[:, H:H + Hk], x[:, H + Hk:], s["starts"], s["pos"], s["rope"],
                        q_out=s["q_out"][layer], commit=False)
    ctx.kv16_commit(pg, list(s["pool"].unbind(0)), s["starts"], s["keep"])
    return {"mask": s["mask"], "pos": s["pos"], "q_out": s["q_out"], "pool": s["pool"], "len": pg.cache_len}


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _plain_turn(s, x, pos):
    """rows [n, heads, D] turned to their positions, in 32 bits; angles in 64"""
    rot, inter = s["case"]["rot"], s["case"]["inter"]
    angle = pos.double()[:, None] * s["freqs"][None]
    c, n = ((f(angle) * s["amplitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    x = x.float()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., : rot // 2], x[..., rot // 2:rot])
    ra, rb = a * c - b * n, b * c + a * n
    turned = torch.stack([ra, rb], -1).flatten(-2) if inter else torch.cat([ra, rb], -1)
    return torch.cat([turned, x[..., rot:]], -1).to(torch.bfloat16)


def _places(table, page, first, counts):
    """pool page and row in it of rows first[b], first[b] + 1, ... of every sequence, packed; counts on the host"""
    seq = torch.repeat_interleave(torch.arange(len(counts), device=DEV), torch.tensor(counts, device=DEV),
                                  output_size=sum(counts))
    start, _ = _starts(counts)
    at = torch.arange(sum(counts), device=DEV) - start.long()[seq] + first.long()[seq]
    return table[seq, at // page].long(), at % page


def _plain_plan(s):
    """masks and positions of the trees' nodes, one generation after the other"""
    parent, lens = s["parent"].long(), s["counts"]
    start = torch.repeat_interleave(s["starts"][:-1].long(), torch.tensor(lens, device=DEV), output_size=sum(lens))
    me = torch.arange(sum(lens), device=DEV)
    local = me - start
    bit = (torch.ones_like(local) << (local % 32)).int()
    mine = torch.where(torch.arange(s["words"], device=DEV)[None] == (local // 32)[:, None], bit[:, None], 0)
    s["mask"].copy_(mine)
    up = torch.where(parent >= 0, start + parent, -1)
    depth = torch.zeros_like(local)
    for _ in range(max(lens)):
        depth += up >= 0
        at = up.clamp(min=0)
        s["mask"] |= torch.where((up >= 0)[:, None], mine[at], 0)
        up = torch.where(up >= 0, torch.where(parent[at] >= 0, start[at] + parent[at], -1), -1)
    s["pos"].copy_(depth + torch.repeat_interleave(s["pos0"].long(), torch.tensor(lens, device=DEV), output_size=sum(lens)))


def _plain_append(s):
    case, got = s["case"], {}
    if case["what"] == "tree":
        _plain_plan(s)
        got.update(mask=s["mask"], pos=s["pos"])
    k, v, pos = s["k"], s["v"], s["pos"]
    if s["q_out"] is not None:
        s["q_out"].copy_(_plain_turn(s, s["q"], pos))
        got["q_out"] = s["q_out"]
    if s["keep"] is not None:
        rows = torch.argsort(s["keep"] == 0, stable=True)[:sum(s["kept"])]       # the kept rows, in order
        k, v, pos = k[rows], v[rows], pos[rows]
    k = _plain_turn(s, k, pos)
    if s["k_out"] is not None:
        s["k_out"].copy_(k)
        got["k_out"] = s["k_out"]
    page, row = _places(s["table"], case["page"], s["before"], s["kept"])
    s["pool"][page, 0, :, row] = k
    s["pool"][page, 1, :, row] = v
    kept = torch.tensor(s["kept"], dtype=torch.int32, device=DEV)
    return {"len": s["before"] + kept if case["what"] != "tree" else s["before"], "pool": s["pool"], **got}


def _rows_of(pool, table_row, n, page):
    """K and V [kv heads, n, D] of a sequence's first n rows"""
    got = pool[table_row[: -(-n // page)].long()]                                # [pages, 2, kv, page, D]
    kv = got.permute(1, 2, 0, 3, 4).reshape(2, got.shape[2], -1, got.shape[4])
    return kv[0, :, :n], kv[1, :, :n]


def _visible(mask, at, i, j, held, n):
    """what nodes i..j-1 of a tree of n see: rows held, then nodes"""
    node = torch.arange(n, device=DEV)
    if mask is None:
        own_part = node[None] <= torch.arange(i, j, device=DEV)[:, None]
    else:
        own_part = (mask[at + i:at + j][:, node // 32] >> (node % 32)) & 1 != 0
    return torch.cat([torch.ones(j - i, held, dtype=torch.bool, device=DEV), own_part], 1)


def _plain_attend(s):
    case = s["case"]
    D, H, Hk = case["dim"], case["heads"], case["kv"]
    G, at = H // Hk, 0
    for b, (held, n) in enumerate(zip(s["held_list"], s["nodes"])):
        k, v = _rows_of(s["pool"], s["table"][b], held + n, case["page"])
        k, v = k.float(), v.float()
        step = max(1, 100000000 // (H * (held + n)))
        for i in range(0, n, step):
            j = min(n, i + step)
            q = s["q"][at + i:at + j].float().view(j - i, Hk, G, D).permute(1, 2, 0, 3).reshape(Hk, G * (j - i), D)
            sc = (torch.matmul(q, k.transpose(1, 2)) * s["scale"]).view(Hk, G, j - i, held + n)
            sc = sc.masked_fill(~_visible(s["mask"], at, i, j, held, n), float("-inf"))
            p = torch.exp(sc - sc.amax(-1, keepdim=True))
            o = torch.matmul(p.view(Hk, G * (j - i), held + n), v).view(Hk, G, j - i, D) / p.sum(-1, keepdim=True)
            s["out"][at + i:at + j] = o.permute(2, 0, 1, 3).reshape(j - i, H, D).to(torch.bfloat16)
        at += n
    return s["out"]


def _held01(x):
    return torch.where(x > 0, x.clamp(max=1.0), torch.zeros_like(x))


def _plain_verify(s):
    case, B, V = s["case"], s["case"]["seqs"], s["case"]["vocab"]
    mode, counts = case["mode"], s["counts"]
    start = s["starts"][:-1].long()
    number = torch.tensor(counts, device=DEV)
    at = torch.zeros(B, dtype=torch.long, device=DEV)
    keep = torch.zeros(sum(counts), dtype=torch.uint8, device=DEV)
    keep[start] = 1
    count = torch.ones(B, dtype=torch.int32, device=DEV)
    every = torch.arange(V, device=DEV)

    def first_largest():
        z = s["target"][start + at].float()
        return torch.where(z == z.amax(1, keepdim=True), every[None], V).amin(1)

    def settle(acc, i):
        nonlocal at, count
        at = torch.where(acc, i, at)
        count = count + acc.int()
        keep.index_put_((torch.where(acc, start + i, start),), torch.ones((), dtype=torch.uint8, device=DEV))

    if mode == "greedy":
        for i in range(1, max(counts)):
            j = (start + i).clamp(max=len(keep) - 1)
            settle((number > i) & (s["parent"][j] == at) & (s["tokens"][j] == first_largest()), i)
        return {"keep": keep, "count": count, "next": first_largest().int()}
    S, R, A = (torch.full((B,), v, dtype=torch.float64, device=DEV) for v in (0.0, 1.0, 1.0))
    dead = torch.zeros(B, V, dtype=torch.bool, device=DEV)
    b = torch.arange(B, device=DEV)

    def left(S_):
        p = s["target"][start + at].double()
        if mode == "point":
            return _held01(p.masked_fill(dead, 0.0))
        return _held01(p - S_[:, None] * s["draft"][start + at].double())

    for i in range(1, max(counts)):
        j = (start + i).clamp(max=len(keep) - 1)
        tok = s["tokens"][j].long()
        here = (number > i) & (s["parent"][j] == at)
        p, u = s["target"][start + at, tok].double(), s["u"][j].double()
        if mode == "point":
            p = torch.where(dead[b, tok], 0.0, p)
            acc = here & (u * R < p)
            rej = here & ~acc
            R = torch.where(acc, 1.0, torch.where(rej, R - p, R))
            dead[b, tok] |= rej
            dead &= ~acc[:, None]
        else:
            q = s["draft"][start + at, tok].double()
            acc = here & (A > 0) & (u * q * R < _held01(p - S * q) * A)
            rej = here & ~acc & (A > 0)
            S2 = torch.where(rej, S + R / A, S)
            R2 = (left(S2) * UNIT).long().sum(1).double() / UNIT
            A2 = A if mode == "replaced" else A - q
            S, R, A = (torch.where(acc, one, torch.where(rej, new, old)) for one, new, old in ((0.0, S2, S), (1.0, R2, R), (1.0, A2, A)))
        settle(acc, i)
    w = (left(S) * UNIT).long()
    w = torch.where(w.sum(1, keepdim=True) > 0, w, (_held01(s["target"][start + at].double()) * UNIT).long())
    run_sum = w.cumsum(1)
    W = run_sum[:, -1]
    k = (s["u"][start].double() * 2.0 ** 31).long().clamp(0, 2 ** 31 - 1)
    T = k * (W >> 31) + ((k * (W & (2 ** 31 - 1))) >> 31)
    nxt = torch.where(W > 0, (run_sum <= T[:, None]).sum(1), -1)
    return {"keep": keep, "count": count, "next": nxt.int()}


def _plain_accept(s):
    case, H, Hk = s["case"], s["case"]["heads"], s["case"]["kv"]
    _plain_plan(s)
    page, row = _places(s["table"], case["page"], s["held"], s["nodes"])
    kept_lists = _accepted(case, s["nodes"])
    for layer in range(case["layers"]):
        x, pool = s["qkv"][layer], s["pool"][layer]
        s["q_out"][layer] = _plain_turn(s, x[:, :H], s["pos"])
        pool[page, 0, :, row] = _plain_turn(s, x[:, H:H + Hk], s["pos"])
        pool[page, 1, :, row] = x[:, H + Hk:]
    kept = [len(p) for p in kept_lists]
    rows = torch.argsort(s["keep"] == 0, stable=True)[:sum(kept)]
    to_page, to_row = _places(s["table"], case["page"], s["held"], kept)
    for layer in range(case["layers"]):
        pool = s["pool"][layer]
        pool.permute(0, 3, 1, 2, 4)[to_page, to_row] = pool.permute(0, 3, 1, 2, 4)[page[rows], row[rows]]
    return {"mask": s["mask"], "pos": s["pos"], "q_out": s["q_out"], "pool": s["pool"],
            "len": s["held"] + torch.tensor(kept, dtype=torch.int32, device=DEV)}


def run(s):
    if own:
        return _run_own(s)
    return {"append": _plain_append, "attend": _plain_attend, "verify": _plain_verify, "accept": _plain_accept}[s["case"]["op"]](s)


# ---- the same in 64 bits --------------------------------------------------------------------------------------------
def _exact_turn(case, x, pos):
    """[n, heads, D] as complex numbers times e^(i angle)"""
    f, amplitude = _frequencies(case)
    angle = np.asarray(pos, np.float64)[:, None] * f[None]
    e = torch.from_numpy(amplitude * np.exp(1j * angle)).to(DEV)[:, None]
    y, rot = x.double().clone(), case["rot"]
    i = torch.arange(rot // 2, device=DEV)
    re, im = (2 * i, 2 * i + 1) if case["inter"] else (i, i + rot // 2)
    z = torch.complex(y[..., re], y[..., im]) * e
    y[..., re], y[..., im] = z.real, z.imag
    return y


def _exact_append(case, seed):
    x, H, Hk, page = _inputs(case, seed), case["heads"], case["kv"], case["page"]
    if case["what"] == "tree":
        first = x["pos0"].cpu().numpy()
        pos = np.concatenate([f + np.array(_depths(p)) for f, p in zip(first, x["parents"])])
    else:
        pos = x["pos"].cpu().numpy()
    got = {"len": None, "mask": None, "pos": None}
    if case["what"] != "tree":
        del got["mask"], got["pos"]
    if case["what"] != "kept":
        got["q_out"] = _exact_turn(case, x["qkv"][:, :H], pos)
    keep = np.ones(len(pos), bool) if x["keep"] is None else x["keep"].cpu().numpy() != 0
    k = _exact_turn(case, x["qkv"][:, H:H + Hk], pos)
    if case["what"] == "all":
        got["k_out"] = k
    counts = [-(-(case["before"] + c) // page) for c in x["kept"]]
    table = _table(counts, max(max(counts), 1) + 1, sum(counts) + 3, seed)
    where = [(table[b, t // page], t % page) for b, c in enumerate(x["kept"]) for t in range(case["before"], case["before"] + c)]
    pool = torch.zeros(sum(counts) + 3, 2, Hk, page, case["dim"], dtype=torch.float64, device=DEV)
    if where:
        pg, row = (torch.tensor(np.array(v, np.int64), device=DEV) for v in zip(*where))
        src = torch.from_numpy(np.flatnonzero(keep)).to(DEV)
        pool[pg, 0, :, row] = k[src]
        pool[pg, 1, :, row] = x["qkv"][src][:, H + Hk:].double()
    got["pool"] = pool
    return got


def _exact_attend(case, seed):
    x, H, Hk, D, page = _inputs(case, seed), case["heads"], case["kv"], case["dim"], case["page"]
    rows = [a + n for a, n in zip(x["lens"], x["nodes"])]
    counts = [-(-n // page) for n in rows]
    table = torch.from_numpy(_table(counts, max(max(counts), 1) + 1, sum(counts) + 3, seed)).to(DEV).long()
    pool = _normal((sum(counts) + 3, 2, Hk, page, D), seed, 5)
    pool[:, :, :, :, : D // 8] *= 2.0
    out = torch.empty(x["q"].shape, dtype=torch.float64, device=DEV)
    at = 0
    for b, (held, n) in enumerate(zip(x["lens"], x["nodes"])):
        seen = torch.ones(n, held + n, dtype=torch.bool)
        if case["causal"]:
            seen = seen.tril(held)
        else:
            seen[:, held:] = False
            for i, up in enumerate(x["parents"][b]):
                if up >= 0:
                    seen[i, held:] = seen[up, held:]
                seen[i, held + i] = True
        seen = seen.to(DEV)
        for h in range(H):
            kv = pool[table[b, :counts[b]], :, h // (H // Hk)].double()             # [pages, 2, page, D]
            k, v = kv[:, 0].reshape(-1, D)[:held + n], kv[:, 1].reshape(-1, D)[:held + n]
            z = (x["q"][at:at + n, h].double() @ k.T) * D ** -0.5
            out[at:at + n, h] = torch.softmax(torch.where(seen, z, -torch.inf), 1) @ v
        at += n
    return out


def _exact_accept(case, seed):
    x, H, Hk, page = _inputs(case, seed), case["heads"], case["kv"], case["page"]
    rows = [a + n for a, n in zip(x["lens"], x["nodes"])]
    counts = [-(-n // page) for n in rows]
    table = _table(counts, max(max(counts), 1) + 1, sum(counts) + 3, seed)
    pool = _normal((case["layers"], sum(counts) + 3, 2, Hk, page, case["dim"]), seed, 5).double()
    pos = np.concatenate([f + np.array(_depths(p)) for f, p in zip(x["pos0"].cpu().numpy(), x["parents"])])
    paths = _accepted(case, x["nodes"])
    src, pg, row, at = [], [], [], 0
    for b, (held, n, path) in enumerate(zip(x["lens"], x["nodes"], paths)):
        order = path + list(range(len(path), n))                 # which node's row lies at each place in the end
        src += [at + i for i in order]
        pg += [table[b, t // page] for t in range(held, held + n)]
        row += [t % page for t in range(held, held + n)]
        at += n
    src, pg, row = (torch.tensor(np.array(v, np.int64), device=DEV) for v in (src, pg, row))
    q = []
    for layer in range(case["layers"]):
        y = x["qkv"][layer]
        q.append(_exact_turn(case, y[:, :H], pos))
        pool[layer, pg, 0, :, row] = _exact_turn(case, y[:, H:H + Hk], pos)[src]
        pool[layer, pg, 1, :, row] = y[src][:, H + Hk:].double()
    return {"mask": None, "pos": None, "q_out": torch.stack(q), "pool": pool, "len": None}


def exact(case, seed):
    op = case["op"]
    if op == "verify":
        return None                                       # decisions and tokens: whole numbers, which have to be equal
    return {"append": _exact_append, "attend": _exact_attend, "accept": _exact_accept}[op](case, seed)
