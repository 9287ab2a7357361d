"""The serving operators around a paged 4-bit K/V cache, as measured work: attention over packed prompts with grouped
heads, appending rows to a 4-bit paged cache (and reading them back), decode attention over such a cache, forking
sequences that share pages, and freeing and compacting pages.

`run` computes them in plain form (elementary torch operations in 32 bits) or, where `own` is true, with the calls a
user makes of this library.  Conventions of the plain form, which are the operators' definitions:

  4-bit rows   a row of D values is cut into groups of 64; per group  z = min,  s = bf16((max - min) / 15),
               code = nearest((x - z) * (1 / s)) clipped to 0..15, with every operation rounded to 32 bits;
               the value held is s * code + z.  A group whose s is zero holds z.
  pages        sequence b owns the pages table[b][0], table[b][1], ... of page_rows rows each; refs counts the table
               entries that name a page; a page nobody names is free, and free pages are handed out in index order.
"""
import random

import numpy as np
import torch

own = False

DEV = "cuda"
GROUP = 64


# ---- cases ----------------------------------------------------------------------------------------------------------
def listed():
    return [
        # a handful of short text prompts on a small model: latency
        dict(name="prompt_short", op="prompt", seqs=4, lo=1, hi=96, heads=16, kv=4, dim=64, sizes=1),
        # the dense layers in front of the token selection: 576 image and about 128 text tokens, every head its own
        dict(name="prompt_image_text", op="prompt", seqs=32, lo=624, hi=743, heads=32, kv=32, dim=128, sizes=2),
        # two long documents, grouped heads
        dict(name="prompt_long", op="prompt", seqs=2, lo=7001, hi=8192, heads=32, kv=8, dim=128, sizes=3),
        # a batch of prompts behind the selection: 144 of 576 image tokens kept, then the text
        dict(name="append_selected", op="append", seqs=32, lo=660, hi=704, heads=32, kv=32, dim=128, sizes=4, page=64,
             masked=576, keep=0.25, before=0),
        # every row of long prompts behind rows that are there already, grouped heads
        dict(name="append_long", op="append", seqs=6, lo=2900, hi=5000, heads=32, kv=8, dim=128, sizes=5, page=32,
             masked=0, keep=1.0, before=77),
        # one or two users early in a conversation: latency
        dict(name="attend_few", op="attend", seqs=2, lo=100, hi=400, heads=16, kv=4, dim=64, sizes=6, page=16),
        # a decode step of the serving batch, half way through its 1024 generated tokens
        dict(name="attend_serving", op="attend", seqs=32, lo=272, hi=1296, heads=32, kv=32, dim=128, sizes=7, page=64),
        # few sequences over very long contexts, grouped heads
        dict(name="attend_long", op="attend", seqs=4, lo=60000, hi=131072, heads=32, kv=4, dim=128, sizes=8, page=64),
        # one request's beams change places
        dict(name="fork_beams", op="fork", seqs=4, beams=4, lo=200, hi=900, heads=32, kv=8, dim=128, sizes=9, page=16,
             layers=2, spare=8),
        # the beams of a serving batch change places, all layers of a stack
        dict(name="fork_serving", op="fork", seqs=64, beams=4, lo=300, hi=1296, heads=32, kv=8, dim=128, sizes=10,
             page=64, layers=32, spare=80),
        # a few requests leave a small pool
        dict(name="compact_few", op="compact", seqs=8, lo=100, hi=700, heads=32, kv=8, dim=128, sizes=11, page=16,
             layers=2, gone=0.4),
        # a third of a serving batch leaves; the rest moves to the front of the pool
        dict(name="compact_serving", op="compact", seqs=64, lo=300, hi=1296, heads=32, kv=8, dim=128, sizes=12, page=64,
             layers=16, gone=0.35),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "append", "attend", "attend", "fork", "compact"])
    dim = rng.choice([64, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 5, 8, 16])
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 5, 6, 7, 8, 12, 16) if kv * g <= 40])
    case = dict(op=op, heads=heads, kv=kv, dim=dim, sizes=rng.randrange(1, 1 << 30))
    if op == "prompt":
        hi = _log(rng, 2, 8000)
        most = 1.1e12 / (2.0 * dim * heads * hi * hi)                  # no dearer than the largest listed case
        case.update(seqs=max(1, min(_log(rng, 1, 40), int(most), 60000 // hi)), lo=max(1, int(hi * rng.random())), hi=hi)
    elif op == "append":
        hi = _log(rng, 2, 5000)
        most = 23000 * 8 * 128 // (hi * kv * dim)
        masked = rng.choice([0, int(hi * rng.random())])
        case.update(seqs=max(1, min(_log(rng, 1, 48), most)), lo=max(1, int(hi * rng.random())), hi=hi,
                    page=rng.choice([16, 32, 64, 128]), masked=masked, keep=rng.choice([0.0, 0.25, 0.5]) if masked else 1.0,
                    before=rng.choice([0, rng.randrange(1, 200)]))
    elif op == "attend":
        hi = _log(rng, 2, 120000)
        most = 400000 * 4 * 128 // (hi * kv * dim)
        case.update(seqs=max(1, min(_log(rng, 1, 96), most)), lo=int(hi * rng.random()), hi=hi,
                    page=rng.choice([16, 32, 64, 128]))
        if kv * hi * dim > 400000 * 4 * 128:
            case.update(kv=4, heads=4 * rng.choice([1, 4, 8]), dim=128, lo=min(case["lo"], 100000), hi=min(hi, 100000))
    elif op == "fork":
        beams = rng.choice([2, 3, 4, 5])
        seqs = beams * rng.randrange(1, 13)
        case.update(beams=beams, seqs=seqs, hi=_log(rng, 20, 1300), page=rng.choice([16, 32, 64]), layers=_log(rng, 1, 16),
                    spare=seqs + rng.randrange(0, 20), kv=min(kv, 8), heads=heads if kv <= 8 else 8)
        case["lo"] = max(1, int(case["hi"] * rng.random()))
    else:
        case.update(seqs=rng.randrange(2, 60), hi=_log(rng, 20, 1300), page=rng.choice([16, 32, 64]),
                    layers=_log(rng, 1, 12), gone=0.1 + 0.7 * rng.random(), kv=min(kv, 8), heads=heads if kv <= 8 else 8)
        case["lo"] = max(1, int(case["hi"] * rng.random()))
    return case


def _lens(case):
    r = random.Random(case["sizes"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["seqs"])]


def _kept_counts(case):
    """Rows of each sequence that are appended: of the first `masked` rows the share `keep`, and all later ones."""
    return [round(min(n, case["masked"]) * case["keep"]) + max(0, n - case["masked"]) for n in _lens(case)]


def _page_bytes(case):
    return case["kv"] * case["page"] * 2 * (case["dim"] // 2 + 4 * (case["dim"] // GROUP))


def work(case):
    D, H, Hk, lens = case["dim"], case["heads"], case["kv"], _lens(case)
    if case["op"] == "prompt":
        total = sum(lens)
        return {"bytes": 2 * D * total * (2 * H + 2 * Hk), "flops": sum(2 * D * H * n * (n + 1) for n in lens)}
    row4 = 2 * (D // 2 + 4 * (D // GROUP))                               # K and V of a row and head in 4 bits
    if case["op"] == "append":
        rows = sum(_kept_counts(case))
        # the kept rows read, held in 4 bits, read back from there and written out as values
        return {"bytes": rows * Hk * (4 * D + row4 + row4 + 4 * D) + sum(min(n, case["masked"]) for n in lens),
                "flops": rows * Hk * 2 * D * 6}
    if case["op"] == "attend":
        rows = sum(lens)
        return {"bytes": rows * Hk * row4 + 2 * D * case["seqs"] * (2 * H + 2 * Hk), "flops": 4 * D * H * (rows + len(lens))}
    book = 4 * sum(-(-n // case["page"]) for n in lens)
    if case["op"] == "fork":
        moves = sum(_fork_plan(case)[1])
    else:
        moves = _compact_plan(case)[1]
    return {"bytes": 2 * moves * _page_bytes(case) * case["layers"] + 2 * book, "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _fork_plan(case):
    """parent of every sequence (within its group of beams), and whether it has to copy a partly filled page."""
    r = random.Random(case["sizes"] + 1)
    B, m, lens = case["seqs"], case["beams"], _lens(case)
    parent = [b // m * m + r.randrange(m) for b in range(B)]
    need = []
    for b, p in enumerate(parent):
        holder = p if parent[p] == p else min(c for c in range(B) if parent[c] == p)
        need.append(lens[p] % case["page"] != 0 and holder != b)
    return parent, need


def _compact_plan(case):
    """which sequences leave, and how many of the others' pages lie behind the last page that is still needed."""
    r = random.Random(case["sizes"] + 1)
    gone = [r.random() < case["gone"] for _ in range(case["seqs"])]
    counts = [-(-n // case["page"]) for n in _lens(case)]
    order = list(range(sum(counts)))
    random.Random(case["sizes"] + 2).shuffle(order)
    rows, at = [], 0
    for c in counts:
        rows.append(order[at:at + c])
        at += c
    live = [p for g, row in zip(gone, rows) if not g for p in row]
    return gone, sum(p >= len(live) for p in live), rows


def _gen(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + stream) % (1 << 62))
    return g


def _normal(shape, seed, stream):
    return torch.randn(shape, generator=_gen(seed, stream), device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _starts(lens):
    c = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return torch.from_numpy(c).to(DEV), int(c[-1])


def _context(case, **kw):
    from paper_2412_00876_b200 import binding as dl
    return dl.Context(64, case["heads"], case["dim"], 64, torch.bfloat16, 0, max_batch=case["seqs"], cap=64, **kw)


def _inputs(case, seed):
    """Tensors of one case, the same for the plain form, the library's calls and the 64-bit values."""
    D, H, Hk, lens = case["dim"], case["heads"], case["kv"], _lens(case)
    x = {"lens": lens}
    if case["op"] == "prompt":
        x["starts"], total = _starts(lens)
        # queries, keys and values as one projection emits them: a token's heads side by side
        x["qkv"] = _normal((total, H + 2 * Hk, D), seed, 1)
    elif case["op"] == "append":
        x["starts"], total = _starts(lens)
        x["kv"] = _normal((total, 2 * Hk, D), seed, 1)
        x["kv"][:, :, : D // 8] *= 3.0                                   # some channels stand out, as keys' do
        keep = np.ones(total, np.uint8)
        r = np.random.RandomState(int(seed) % (1 << 31))
        at = 0
        for n, kept in zip(lens, _kept_counts(case)):
            m = min(n, case["masked"])
            keep[at:at + m] = 0
            keep[at + r.permutation(m)[:kept - (n - m)]] = 1
            at += n
        x["keep"] = torch.from_numpy(keep).to(DEV) if case["masked"] else None
        x["kept"] = _kept_counts(case)
    elif case["op"] == "attend":
        x["starts"], total = _starts(lens)
        x["kv"] = _normal((total, 2 * Hk, D), seed, 1)
        x["kv"][:, :, : D // 8] *= 3.0
        B = case["seqs"]
        x["q"], x["k"], x["v"] = (_normal((B, h, D), seed, i + 2) for i, h in enumerate((H, Hk, Hk)))
    return x


def _table(case, counts, width, n_pages, seed):
    """pages of the sequences at random places of the pool."""
    order = np.random.RandomState(int(seed) % (1 << 31)).permutation(n_pages)
    t, at = np.full((len(counts), width), -1, np.int32), 0
    for b, c in enumerate(counts):
        t[b, :c] = order[at:at + c]
        at += c
    return t


def prepare(case, seed):
    s = {"case": dict(case), **_inputs(case, seed)}
    D, H, Hk, B, lens = case["dim"], case["heads"], case["kv"], case["seqs"], s["lens"]
    s["scale"] = D ** -0.5
    if case["op"] == "prompt":
        s["q"], s["k"], s["v"] = s["qkv"][:, :H], s["qkv"][:, H:H + Hk], s["qkv"][:, H + Hk:]
        s["out"] = torch.empty(s["q"].shape, dtype=torch.bfloat16, device=DEV)
        if own:
            s["ctx"] = _context(case)
        return s
    page = case["page"]
    if case["op"] in ("append", "attend"):
        rows = [case["before"] + k for k in s["kept"]] if case["op"] == "append" else [n + 1 for n in lens]
        counts = [-(-n // page) for n in rows]
        n_pages, width = sum(counts) + 3, max(max(counts), 1) + 1
        table = torch.from_numpy(_table(case, counts, width, n_pages, seed)).to(DEV)
        s["k_src"], s["v_src"] = s["kv"][:, :Hk], s["kv"][:, Hk:]
        before = torch.full((B,), case.get("before", 0), dtype=torch.int32, device=DEV)
        if case["op"] == "append":
            s["row0"] = before
            s["kept_starts"], n = _starts(s["kept"])
            s["k_out"], s["v_out"] = (torch.empty((n, Hk, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        if own:
            from paper_2412_00876_b200 import binding as dl
            s["ctx"] = _context(case)
            s["pages"] = dl.Pages(B, n_pages, width, page, DEV)
            s["pages"].table.copy_(table)
            s["pages"].cache_len.copy_(before)
            s["pool"] = s["ctx"].kv4_pool(s["pages"], Hk)
        else:
            s["table"] = table
            s["len"] = before.clone()
            shape = (n_pages, Hk, page)
            s["codes"] = [torch.zeros(*shape, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
            s["sz"] = [torch.zeros(*shape, 2, D // GROUP, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        if case["op"] == "attend":
            s["out"] = torch.empty((B, H, D), dtype=torch.bfloat16, device=DEV)
            if own:
                s["ctx"].kv4_append(s["pages"], s["pool"], s["k_src"], s["v_src"], s["starts"])
            else:
                _plain_append(s, None, lens)
            for key in ("kv", "k_src", "v_src"):
                del s[key]
        return s
    # pools of pages whose bytes are whatever they are: forking and compacting only move them
    counts = [-(-n // page) for n in lens]
    width = max(counts) + 1
    if case["op"] == "fork":
        parent, need = _fork_plan(case)
        m = case["beams"]
        shared = [min(lens[g * m:g * m + m]) // page // 2 for g in range(B // m)]     # full pages a group has in common
        own_counts = [c - shared[b // m] for b, c in enumerate(counts)]
        n_pages = sum(own_counts) + sum(shared) + case["spare"] + B
        order = np.random.RandomState(int(seed) % (1 << 31)).permutation(n_pages)
        table, at, common = np.full((B, width), -1, np.int32), 0, []
        for g, c in enumerate(shared):
            common.append(order[at:at + c])
            at += c
        for b, c in enumerate(own_counts):
            g = b // m
            table[b, :shared[g]] = common[g]
            table[b, shared[g]:shared[g] + c] = order[at:at + c]
            at += c
        s["parent"] = torch.tensor(parent, dtype=torch.int32, device=DEV)
        s["more"] = torch.ones(B, dtype=torch.int32, device=DEV)
    else:
        gone, s["moves"], rows = _compact_plan(case)
        n_pages = sum(counts)
        table = np.full((B, width), -1, np.int32)
        for b, row in enumerate(rows):
            table[b, :len(row)] = row
        s["gone"] = torch.tensor(gone, dtype=torch.uint8, device=DEV)
        s["live"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    refs = np.bincount(table[table >= 0].ravel(), minlength=n_pages).astype(np.int32)
    s["pool"] = torch.randint(0, 256, (case["layers"], n_pages, _page_bytes(case)), generator=_gen(seed, 9), device=DEV,
                              dtype=torch.uint8)
    table, refs, ln = (torch.from_numpy(np.asarray(v, np.int32)).to(DEV) for v in (table, refs, np.array(lens)))
    if own:
        from paper_2412_00876_b200 import binding as dl
        s["ctx"] = _context(case)
        s["pages"] = dl.Pages(B, n_pages, width, page, DEV)
        s["pages"].table.copy_(table)
        s["pages"].refs.copy_(refs)
        s["pages"].cache_len.copy_(ln)
        s["book"] = s["pages"].book.clone()
        s["pools"] = list(s["pool"].unbind(0))
    else:
        s["table"], s["refs"], s["len"] = table, refs, ln
    return s


# ---- the library's calls --------------------------------------------------------------------------------------------
def _run_own(s):
    op, ctx = s["case"]["op"], s["ctx"]
    if op == "prompt":
        ctx.attn_prefill_packed(s["q"], s["k"], s["v"], s["starts"], max(s["lens"]), s["scale"], s["out"])
        return s["out"]
    pg = s["pages"]
    if op == "append":
        pg.cache_len.copy_(s["row0"])
        ctx.kv4_append(pg, s["pool"], s["k_src"], s["v_src"], s["starts"], s["keep"])
        ctx.kv4_read(pg, s["pool"], s["row0"], s["kept_starts"], s["k_out"], s["v_out"])
        return {"len": pg.cache_len, "k": s["k_out"], "v": s["v_out"]}
    if op == "attend":
        ctx.kv4_attn_decode(pg, s["pool"], s["q"], s["k"], s["v"], None, s["scale"], s["out"])
        return s["out"]
    pg.book.copy_(s["book"])                                  # the same bookkeeping in front of every pass
    if op == "fork":
        ctx.pages_fork(pg, s["parent"], s["pools"])
        ctx.pages_reserve(pg, s["more"])
        return {"table": pg.table, "refs": pg.refs, "len": pg.cache_len, "pool": s["pool"]}
    ctx.pages_free(pg, s["gone"])
    ctx.pages_compact(pg, s["pools"], s["live"])
    return {"table": pg.table, "refs": pg.refs, "len": pg.cache_len, "live": s["live"], "pool": s["pool"]}


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _plain_prompt(s):
    D, H, Hk = s["case"]["dim"], s["case"]["heads"], s["case"]["kv"]
    G, at = H // Hk, 0
    for n in s["lens"]:
        q = s["q"][at:at + n].float().view(n, Hk, G, D).permute(1, 2, 0, 3)               # [Hk][G][n][D]
        k = s["k"][at:at + n].float().permute(1, 0, 2)
        v = s["v"][at:at + n].float().permute(1, 0, 2)
        for i in range(0, n, 1024):
            j = min(n, i + 1024)
            sc = torch.matmul(q[:, :, i:j].reshape(Hk, G * (j - i), D), k[:, :j].transpose(1, 2)) * s["scale"]
            sc = sc.view(Hk, G, j - i, j)
            later = torch.arange(j, device=DEV)[None, :] > torch.arange(i, j, device=DEV)[:, None]
            sc = sc.masked_fill(later, float("-inf"))
            p = torch.exp(sc - sc.amax(-1, keepdim=True))
            o = torch.matmul(p.view(Hk, G * (j - i), j), v[:, :j]).view(Hk, G, j - i, D) / p.sum(-1, keepdim=True)
            s["out"][at + i:at + j] = o.permute(2, 0, 1, 3).reshape(j - i, H, D).to(torch.bfloat16)
        at += n
    return s["out"]


def _plain_quantise(x):
    """rows [..., D] -> codes [..., D] (one a byte), scale and lowest value [..., 2, D / 64] bf16"""
    g = x.float().reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    z, top = g.amin(-1), g.amax(-1)
    sc = ((top - z) / torch.full_like(z, 15.0)).to(torch.bfloat16)
    w = sc.float()
    inv = torch.where(w > 0, torch.ones_like(w) / w, torch.zeros_like(w))
    code = torch.round((g - z[..., None]) * inv[..., None]).clamp(0, 15).to(torch.uint8)
    return code.view(x.shape), torch.stack([sc, z.to(torch.bfloat16)], -2)


def _plain_places(s, first, counts):
    """pool page and row in it of rows first[b], first[b] + 1, ... of every sequence, packed; counts on the host"""
    page = s["case"]["page"]
    seq = torch.repeat_interleave(torch.arange(len(counts), device=DEV), torch.tensor(counts, device=DEV),
                                  output_size=sum(counts))
    start, _ = _starts(counts)
    pos = torch.arange(sum(counts), device=DEV) - start.long()[seq] + first.long()[seq]
    return s["table"][seq, pos // page].long(), pos % page


def _plain_append(s, keep, kept):
    src = [s["k_src"], s["v_src"]]
    if keep is not None:
        rows = torch.argsort(keep == 0, stable=True)[:sum(kept)]                # the kept rows, in order
        src = [x[rows] for x in src]
    page, row = _plain_places(s, s["len"], kept)
    for x, codes, sz in zip(src, s["codes"], s["sz"]):
        c, m = _plain_quantise(x)
        codes[page, :, row] = c
        sz[page, :, row] = m
    s["len"] += torch.tensor(kept, dtype=torch.int32, device=DEV)


def _plain_read(s, first, counts):
    page, row = _plain_places(s, first, counts)
    got = []
    for codes, sz in zip(s["codes"], s["sz"]):
        c, m = codes[page, :, row].float(), sz[page, :, row].float()
        got.append((c.view(*c.shape[:-1], c.shape[-1] // GROUP, GROUP) * m[..., 0, :, None] + m[..., 1, :, None]).view(c.shape))
    return got


def _plain_attend(s):
    D, H, Hk = s["case"]["dim"], s["case"]["heads"], s["case"]["kv"]
    G = H // Hk
    for b, n in enumerate(s["lens"]):
        zero = torch.zeros(1, dtype=torch.int32, device=DEV)
        one = {"case": s["case"], "table": s["table"][b:b + 1], "codes": s["codes"], "sz": s["sz"]}
        k, v = _plain_read(one, zero, [n])
        k = torch.cat([k, s["k"][b:b + 1].float()]).permute(1, 2, 0)                 # [Hk][D][n + 1]
        v = torch.cat([v, s["v"][b:b + 1].float()]).permute(1, 0, 2)
        sc = torch.matmul(s["q"][b].float().view(Hk, G, D), k) * s["scale"]
        p = torch.exp(sc - sc.amax(-1, keepdim=True))
        s["out"][b] = (torch.matmul(p, v) / p.sum(-1, keepdim=True)).view(H, D).to(torch.bfloat16)
    return s["out"]


def _copy_pages(pool, src, dst):
    pool[:, dst] = pool[:, src]


def _plain_reserve(table, refs, ln, more, page):
    B, W = table.shape
    have = (table >= 0).sum(1)
    add = ((ln + more + page - 1) // page - have).clamp(min=0)
    first = torch.cumsum(add, 0) - add
    free = torch.argsort(refs != 0, stable=True)                               # free pages in index order, then the others
    col = torch.arange(W, device=DEV)[None]
    fresh = (col >= have[:, None]) & (col < (have + add)[:, None])
    place = (first[:, None] + col - have[:, None]).clamp(0, refs.numel() - 1)
    table = torch.where(fresh, free[place].int(), table)
    return table, refs.index_add(0, table.clamp(min=0).view(-1).long(), fresh.view(-1).int())


def _plain_fork(s):
    page, table, ln, par = s["case"]["page"], s["table"], s["len"], s["parent"].long()
    B, W = table.shape
    me, col = torch.arange(B, device=DEV), torch.arange(W, device=DEV)[None]
    stay = (par == me)[:, None]
    length = ln[par]
    used = (length + page - 1) // page
    new = torch.where(stay | (col < used[:, None]), table[par], -1)
    first = torch.where(par[None] == par[:, None], me[None], B).amin(1)         # lowest sequence with the same parent
    holder = torch.where(par[par] == par, par, first)
    need = (length % page != 0) & (holder != me)
    last = (need[:, None] & (col == used[:, None] - 1))
    refs = s["refs"].clone()
    refs.index_add_(0, table.clamp(min=0).view(-1).long(), -((table >= 0) & ~stay).view(-1).int())
    refs.index_add_(0, new.clamp(min=0).view(-1).long(), ((new >= 0) & ~stay & ~last).view(-1).int())
    free = torch.argsort(refs != 0, stable=True)
    mine = free[(torch.cumsum(need, 0) - 1).clamp(min=0)]
    src = torch.where(last, new, 0).amax(1).long()
    new = torch.where(last, mine[:, None].int(), new)
    refs.index_add_(0, mine, need.int())
    # sequences that copy nothing repeat the first copy
    at = torch.where(need, me, B).amin().clamp(max=B - 1)
    some = need.any()
    src = torch.where(need, src, torch.where(some, src[at], 0))
    dst = torch.where(need, mine, torch.where(some, mine[at], 0))
    for layer in range(s["pool"].shape[0]):
        _copy_pages(s["pool"][layer:layer + 1], src, dst)
    table, refs = _plain_reserve(new, refs, length, s["more"], page)
    return {"table": table, "refs": refs, "len": length, "pool": s["pool"]}


def _plain_compact(s):
    table, gone = s["table"], s["gone"].bool()
    N = s["refs"].numel()
    refs = s["refs"].index_add(0, table.clamp(min=0).view(-1).long(), -((table >= 0) & gone[:, None]).view(-1).int())
    table = torch.where(gone[:, None], -1, table)
    ln = torch.where(gone, 0, s["len"])
    live = (refs > 0).sum()
    idx = torch.arange(N, device=DEV)
    src = torch.argsort(~((refs > 0) & (idx >= live)), stable=True)[:s["moves"]]
    dst = torch.argsort(~((refs == 0) & (idx < live)), stable=True)[:s["moves"]]
    new = idx.index_copy(0, src, dst).int()
    table = torch.where(table >= 0, new[table.clamp(min=0).long()], -1)
    refs = refs.index_copy(0, dst, refs[src]).index_copy(0, src, torch.zeros_like(refs[src]))
    for layer in range(s["pool"].shape[0]):
        _copy_pages(s["pool"][layer:layer + 1], src, dst)
    return {"table": table, "refs": refs, "len": ln, "live": live.int().view(1), "pool": s["pool"]}


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    if op == "prompt":
        return _plain_prompt(s)
    if op == "append":
        s["len"].copy_(s["row0"])
        _plain_append(s, s["keep"], s["kept"])
        k, v = _plain_read(s, s["row0"], s["kept"])
        return {"len": s["len"], "k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}
    if op == "attend":
        return _plain_attend(s)
    return _plain_fork(s) if op == "fork" else _plain_compact(s)


# ---- the same in 64 bits --------------------------------------------------------------------------------------------
def _exact_held(x):
    """the values a row's 4-bit form stands for: the codes by the definition's 32-bit steps, the values in 64 bits"""
    x = x.float().cpu().numpy()
    g = x.reshape(x.size // GROUP, GROUP)
    lo, hi = g.min(1, keepdims=True), g.max(1, keepdims=True)
    step = ((hi - lo) / np.float32(15)).astype(np.float32)
    bits = step.view(np.uint32)
    step = ((bits + 0x7FFF + ((bits >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)        # to bf16, ties to even
    with np.errstate(divide="ignore"):
        inv = np.where(step > 0, np.float32(1) / step, np.float32(0)).astype(np.float32)
    code = np.clip(np.rint((g - lo) * inv), 0, 15)
    held = step.astype(np.float64) * code.astype(np.float64) + lo.astype(np.float64)
    return torch.from_numpy(held.reshape(x.shape)).to(DEV)


def _exact_rows(q, k, v, scale):
    """softmax(q k^T) v of one head: q [r][D] attends all of k, v [n][D], r of them at a time"""
    z = torch.einsum("rd,nd->rn", q, k) * scale
    return torch.einsum("rn,nd->rd", torch.softmax(z, 1), v)


def exact(case, seed):
    op, D, H, Hk = case["op"], case["dim"], case["heads"], case["kv"]
    if op in ("fork", "compact"):
        return None                                       # nothing is computed: pages and indices are moved
    x = _inputs(case, seed)
    scale, starts = D ** -0.5, x["starts"].tolist()
    if op == "prompt":
        out = torch.empty((starts[-1], H, D), dtype=torch.float64, device=DEV)
        for a, e in zip(starts, starts[1:]):
            for h in range(H):
                q, k, v = (x["qkv"][a:e, i].double() for i in (h, H + h // (H // Hk), H + Hk + h // (H // Hk)))
                for i in range(0, e - a, 2048):
                    j = min(e - a, i + 2048)
                    z = (q[i:j] @ k[:j].T) * scale
                    z = torch.where(torch.ones_like(z).tril(i) > 0, z, -torch.inf)
                    out[a + i:a + j, h] = torch.softmax(z, 1) @ v[:j]
        return out
    if op == "append":
        rows = x["kv"] if x["keep"] is None else x["kv"][x["keep"] != 0]
        held = _exact_held(rows)
        return {"len": None, "k": held[:, :Hk], "v": held[:, Hk:]}
    out = torch.empty((case["seqs"], H, D), dtype=torch.float64, device=DEV)
    for b, (a, e) in enumerate(zip(starts, starts[1:])):
        held = _exact_held(x["kv"][a:e])
        for h in range(H):
            m = h // (H // Hk)
            k = torch.cat([held[:, m], x["k"][b, m:m + 1].double()])
            v = torch.cat([held[:, Hk + m], x["v"][b, m:m + 1].double()])
            out[b, h] = _exact_rows(x["q"][b, h:h + 1].double(), k, v, scale)[0]
    return out
