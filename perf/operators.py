"""The paged-cache operators and the beam selection: cases, plain forms and the framework's calls.

A paged cache holds the keys and values of many sequences in pages of `page` slots:
kv_pages [layers][pages][2][kv heads][page][head dimension]; tables[sequence][i] names the page that holds the
sequence's slots [i*page, (i+1)*page), -1 behind its last page; refs[page] counts the sequences that hold a page.

  attend   a step's new keys and values are written behind each sequence's committed slots (append), then the rows of
           every sequence's draft tree (one row: plain decoding) attend to the committed slots and to their ancestors
  compact  the accepted path of every sequence becomes contiguous behind its committed slots, in all layers
  remap    sequences are reordered, forked, grown, cut or freed: whole pages are shared, a partly filled page that
           stays shared is copied, the lowest free pages are handed out
  beam     the best continuations of every group of beams over beams x vocabulary
"""
import math
import random

import numpy as np
import torch

own = False

# the head layouts of the repository's model shapes: query heads, key/value heads, head dimension
HEADS = {"8b": (32, 8, 128), "13b": (40, 40, 128), "mid": (8, 2, 128), "small": (8, 2, 64), "toy": (4, 4, 64),
         "tiny": (6, 2, 32)}


def listed():
    return [
        # one sequence, one token a step, 1024 committed slots: the latency of plain decoding
        {"name": "attend decode 1x1024", "kind": "attend", "heads": "8b", "dtype": "bf16", "batch": 1, "rows": 1,
         "ragged": False, "prefix": 1024, "page": 16, "append": True},
        # one sequence's tree of 80 tokens and its root over a long context
        {"name": "attend tree81 1x8192", "kind": "attend", "heads": "8b", "dtype": "bf16", "batch": 1, "rows": 81,
         "ragged": False, "prefix": 8192, "page": 64, "append": False},
        # a serving batch: 16 trees of up to 61 rows over contexts of 4096 to 8191 slots
        {"name": "attend tree61 16x8191", "kind": "attend", "heads": "8b", "dtype": "bf16", "batch": 16, "rows": 61,
         "ragged": True, "prefix": 8191, "page": 16, "append": True},
        # a serving batch of 64 sequences, one token each
        {"name": "attend decode 64x8000", "kind": "attend", "heads": "8b", "dtype": "bf16", "batch": 64, "rows": 1,
         "ragged": False, "prefix": 8000, "page": 32, "append": True},
        # head dimension 64, short odd contexts, trees of up to 25 rows
        {"name": "attend small 7x300", "kind": "attend", "heads": "small", "dtype": "bf16", "batch": 7, "rows": 25,
         "ragged": True, "prefix": 300, "page": 16, "append": True},
        # the check mode in 32 bits, pages of an odd size
        {"name": "attend check 3x517", "kind": "attend", "heads": "toy", "dtype": "fp32", "batch": 3, "rows": 15,
         "ragged": True, "prefix": 517, "page": 24, "append": False},
        # commit of one sequence's round in a two-layer model
        {"name": "compact 1x2", "kind": "compact", "heads": "small", "dtype": "bf16", "batch": 1, "layers": 2,
         "prefix": 300, "rows": 25, "page": 16},
        # commit of 16 sequences' rounds in a 32-layer model
        {"name": "compact 16x32", "kind": "compact", "heads": "8b", "dtype": "bf16", "batch": 16, "layers": 32,
         "prefix": 500, "rows": 61, "page": 16},
        # reordering of one group of 4 beams after a step
        {"name": "remap beams 4x700", "kind": "remap", "heads": "mid", "dtype": "bf16", "layers": 2, "before": 4,
         "after": 4, "prefix": 700, "page": 16, "room": 1},
        # reordering of 16 groups of 4 beams in a 32-layer model
        {"name": "remap beams 64x509", "kind": "remap", "heads": "8b", "dtype": "bf16", "layers": 32, "before": 64,
         "after": 64, "prefix": 509, "page": 64, "room": 1},
        # beam search of one sequence over a 32000-token vocabulary
        {"name": "beam 1x4x32000", "kind": "beam", "batch": 1, "beams": 4, "vocab": 32000, "dtype": "fp32"},
        # beam search of 32 sequences with 8 beams over a 128256-token vocabulary
        {"name": "beam 32x8x128256", "kind": "beam", "batch": 32, "beams": 8, "vocab": 128256, "dtype": "fp32"},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "compact", "remap", "beam"])
    if kind == "attend":
        heads = rng.choice(["8b", "8b", "13b", "mid", "small", "toy", "tiny"])
        dtype = "fp32" if heads in ("toy", "tiny") else "bf16"
        rows = rng.choice([1, _spread(rng, 1, 128)])
        hq, hkv, d = HEADS[heads]
        prefix = _spread(rng, 1, 12000 if dtype == "bf16" else 2000) - 1
        batch = _spread(rng, 1, 64)
        slots = prefix + rows + 64
        while batch > 1 and (batch * hq * rows * slots > 200_000_000 or batch * slots * hkv * d > 400_000_000):
            batch -= 1
        return {"kind": kind, "heads": heads, "dtype": dtype, "batch": batch, "rows": rows,
                "ragged": rng.random() < 0.5, "prefix": prefix,
                "page": rng.choice([16, 16, 32, 64, 128, 256]) if dtype == "bf16" else rng.choice([8, 16, 24, 64]),
                "append": rng.random() < 0.5}
    if kind == "compact":
        return {"kind": kind, "heads": rng.choice(["8b", "mid", "small", "tiny"]), "dtype": rng.choice(["bf16", "fp32"]),
                "batch": _spread(rng, 1, 16), "layers": _spread(rng, 1, 16), "prefix": _spread(rng, 1, 400),
                "rows": rng.randint(2, 128), "page": rng.choice([8, 16, 24, 64])}
    if kind == "remap":
        return {"kind": kind, "heads": rng.choice(["8b", "mid", "small", "tiny"]), "dtype": rng.choice(["bf16", "fp32"]),
                "layers": _spread(rng, 1, 8), "before": _spread(rng, 1, 64), "after": _spread(rng, 1, 64),
                "prefix": _spread(rng, 1, 500), "page": rng.choice([8, 16, 24, 64]), "room": rng.randint(0, 130)}
    return {"kind": kind, "batch": _spread(rng, 1, 32), "beams": rng.randint(1, 8), "vocab": _spread(rng, 100, 128256),
            "dtype": rng.choice(["fp32", "bf16"])}


# ------------------------------------------------------------------ sizes that a case fixes
def _lengths(case):
    """Committed slots of each sequence: spread over the upper half of [0, prefix], one of them at prefix."""
    b, p = case.get("before", case.get("batch")), case["prefix"]
    return [p - int((i * 0.6180339887) % 1.0 * (p // 2 + 1)) for i in range(b)]


def _tree_rows(case):
    """Rows of each sequence's tree: all alike, or spread over [1, rows]."""
    b, r = case["batch"], case["rows"]
    return [r - int((i * 0.7548776662) % 1.0 * r) if case["ragged"] else r for i in range(b)]


def _max_pages(case):
    more = case["room"] if case["kind"] == "remap" else case["rows"]
    return -(-(case["prefix"] + more) // case["page"]) + 1


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _tables(lengths, page, max_pages, n_pages, seed):
    """Pages of each sequence, from a pool whose free pages lie in no order."""
    order = np.random.RandomState(seed % (1 << 31)).permutation(n_pages)
    t = np.full((len(lengths), max_pages), -1, dtype=np.int32)
    at = 0
    for i, n in enumerate(lengths):
        k = -(-n // page)
        t[i, :k] = order[at:at + k]
        at += k
    return t


def _masks(batch, rows, seed):
    """Ancestor bits of random trees: row 0 is the root, a row's parent is an earlier row."""
    rs = np.random.RandomState(seed % (1 << 31))
    words = (rows + 63) // 64
    m = np.zeros((batch, rows, words), dtype=np.uint64)
    every = np.arange(batch)
    for r in range(rows):
        if r:
            parent = r - 1 - (rs.random_sample(batch) * min(r, 12)).astype(np.int64)
            m[:, r] = m[every, parent]
        m[:, r, r // 64] |= np.uint64(1) << np.uint64(r % 64)
    return m.view(np.int64)


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dev = "cuda"

    def cuda(a):
        return torch.from_numpy(np.ascontiguousarray(a)).to(dev)

    if case["kind"] == "beam":
        b, k, v, dt = case["batch"], case["beams"], case["vocab"], _dtype(case)
        # logits of a language model: wide, a few far above the rest; beams a few steps into the search
        x = torch.randn(b, k, v, device=dev, generator=gen) * 2.5
        scores = -torch.rand(b, k, device=dev, generator=gen) * 4 - 8
        finished = (torch.rand(b, k, device=dev, generator=gen) < 0.15).to(torch.int32)
        return {"case": case, "logits": x.to(dt), "scores": scores, "finished": finished, "eos": 2}

    hq, hkv, d = HEADS[case["heads"]]
    page, dt = case["page"], _dtype(case)
    mp = _max_pages(case)
    lengths = _lengths(case)
    random.Random(seed).shuffle(lengths)
    if case["kind"] == "attend":
        b, r = case["batch"], case["rows"]
        rows = _tree_rows(case)
        random.Random(seed + 1).shuffle(rows)
        held = [n + m for n, m in zip(lengths, rows)]
        n_pages = sum(-(-(n + r) // page) for n in lengths) + 7
        q = torch.randn(b, r, hq, d, device=dev, generator=gen).to(dt)
        new = torch.randn(2, b, r, hkv, d, device=dev, generator=gen).to(dt)
        return {"case": case, "pages": torch.randn(1, n_pages, 2, hkv, page, d, device=dev, dtype=dt, generator=gen),
                "tables": cuda(_tables(held, page, mp, n_pages, seed)), "q": q, "k": new[0], "v": new[1],
                "prefix": cuda(np.array(lengths, np.int32)), "rows": cuda(np.array(rows, np.int32)),
                "mask": cuda(_masks(b, r, seed)), "scale": 1.0 / math.sqrt(d), "out": torch.zeros_like(q)}
    if case["kind"] == "compact":
        b, r = case["batch"], case["rows"]
        held = [n + r for n in lengths]
        n_pages = sum(-(-n // page) for n in held) + 7
        rs = np.random.RandomState(seed % (1 << 31))
        path = np.zeros((b, 17), dtype=np.int32)
        acc = np.zeros(b, dtype=np.int32)
        for i in range(b):      # a path through a tree of r rows: root first, every node behind its parent
            a = int(rs.randint(0, min(8, r - 1) + 1))
            path[i, 1:a + 1] = np.sort(rs.permutation(np.arange(1, r))[:a])
            acc[i] = a
        pages = torch.randn(case["layers"], n_pages, 2, hkv, page, d, device=dev, dtype=dt, generator=gen)
        return {"case": case, "pages": pages, "tables": cuda(_tables(held, page, mp, n_pages, seed)),
                "prefix": cuda(np.array(lengths, np.int32)), "path": cuda(path), "accepted": cuda(acc)}
    # remap: groups of 4 sequences pick their parents inside their group, one sequence ends and one starts empty
    nb, na = case["before"], case["after"]
    rs = np.random.RandomState(seed % (1 << 31))
    parents = np.array([min(nb - 1, i // 4 * 4 + rs.randint(0, 4)) for i in range(na)], dtype=np.int32)
    if na > 4:
        parents[rs.randint(0, na)] = -1
    n_pages = sum(-(-n // page) for n in lengths) + na * (-(-case["room"] // page) + 2) + 7
    tables = _tables(lengths, page, mp, n_pages, seed)
    refs = np.zeros(n_pages, dtype=np.int32)
    refs[tables[tables >= 0]] = 1
    pages = torch.randn(case["layers"], n_pages, 2, hkv, page, d, device=dev, dtype=dt, generator=gen)
    return {"case": case, "pages": pages, "tables": cuda(tables), "len": cuda(np.array(lengths, np.int32)),
            "refs": cuda(refs), "parents": cuda(parents), "room": torch.full((na,), case["room"], dtype=torch.int32, device=dev)}


# ------------------------------------------------------------------ plain forms
def _append_plain(s):
    pages, page = s["pages"], s["case"]["page"]
    b, r = s["k"].shape[:2]
    at = torch.arange(r, device="cuda")
    slot = s["prefix"].long()[:, None] + at                                             # [b][r]
    live = at < s["rows"][:, None]
    p = s["tables"].long().gather(1, slot // page)
    # rows behind a sequence's last one write nothing: they go where the first row goes, with its values
    p, off = torch.where(live, p, p[:, :1]), torch.where(live, slot % page, slot[:, :1] % page)
    for which, new in ((0, s["k"]), (1, s["v"])):
        pages[0, p, which, :, off] = torch.where(live[..., None, None], new, new[:, :1])


def _attend_plain(s):
    b, r, hq, d = s["q"].shape
    pages, tables = s["pages"][0], s["tables"].long().clamp(min=0)
    hkv, page = pages.shape[2], pages.shape[3]
    g, slots = hq // hkv, tables.shape[1] * page
    if s["case"]["append"]:
        _append_plain(s)
    k, v = (pages[:, w][tables].permute(0, 2, 1, 3, 4).reshape(b, hkv, slots, d).float() for w in (0, 1))
    q = s["q"].view(b, r, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, r * g, d).float()
    at = torch.arange(slots, device="cuda") - s["prefix"][:, None]                      # [b][slots]: place in the tree
    j = at.clamp(0, r - 1)
    bits = s["mask"].gather(2, (j // 64)[:, None].expand(b, r, slots).long()) >> (j % 64)[:, None]
    seen = (at < 0)[:, None] | ((bits & 1).bool() & ((at >= 0) & (at < s["rows"][:, None]))[:, None])
    x = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(b, hkv, r, g, slots)
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_().view(b, hkv, r * g, slots)
    o = (x @ v / x.sum(-1, keepdim=True)).view(b, hkv, r, g, d).permute(0, 2, 1, 3, 4).reshape(b, r, hq, d)
    live = torch.arange(r, device="cuda") < s["rows"][:, None]
    s["out"].copy_(torch.where(live[..., None, None], o.to(s["out"].dtype), s["out"]))
    return {"out": s["out"], "pages": s["pages"]} if s["case"]["append"] else {"out": s["out"]}


def _compact_plain(s):
    pages, page, b = s["pages"], s["case"]["page"], s["prefix"].shape[0]
    k = torch.arange(s["path"].shape[1], device="cuda").expand(b, -1)
    moved = k <= s["accepted"][:, None]
    src = s["prefix"].long()[:, None] + torch.where(moved, s["path"].long(), 0)
    dst = s["prefix"].long()[:, None] + torch.where(moved, k, 0)          # (a row that stays: the root onto itself)
    t = s["tables"].long()
    rows = pages[:, t.gather(1, src // page), :, :, src % page]
    pages[:, t.gather(1, dst // page), :, :, dst % page] = rows
    return {"pages": pages, "len": s["prefix"] + s["accepted"] + 1}


def _remap_plain(s):
    pages, page, refs = s["pages"], s["case"]["page"], s["refs"]
    n_pages, na, mp = refs.shape[0], s["parents"].shape[0], s["tables"].shape[1]
    parent = s["parents"].long()
    has = parent >= 0
    kept = torch.where(has, s["len"][parent.clamp(min=0)], 0).long()
    old = torch.where(has[:, None], s["tables"][parent.clamp(min=0)], -1).long()          # [after][max pages]
    place = torch.arange(mp, device="cuda").expand(na, mp)
    needed = place < ((kept + s["room"] + page - 1) // page)[:, None]
    takes = needed & (old >= 0)
    writes = takes & (place >= (kept // page)[:, None])
    # references: the old sequences leave, the new ones come
    out = torch.cat([refs, refs.new_zeros(1)]).long()
    was = s["tables"].long()
    out.index_add_(0, torch.where(was >= 0, was, n_pages).view(-1), torch.full((was.numel(),), -1, device="cuda"))
    at = torch.where(takes, old, n_pages).view(-1)
    out.index_add_(0, at, torch.ones_like(at))
    # a page that will be written has one holder: of several, each but the last one in order takes a fresh page
    seq = torch.arange(na, device="cuda")[:, None].expand(na, mp)
    at_w = torch.where(writes, old, n_pages).view(-1)
    writers = torch.zeros_like(out).index_add_(0, at_w, torch.ones_like(at_w))
    last = torch.full_like(out, -1).scatter_reduce_(0, at_w, seq.reshape(-1), "amax")
    stays = writes & (out[old] == writers[old]) & (last[old] == seq)
    leaves = writes & ~stays
    fresh = leaves | (needed & (old < 0))
    out.index_add_(0, torch.where(leaves, old, n_pages).view(-1), torch.full((na * mp,), -1, device="cuda"))
    free = torch.sort((out[:n_pages] != 0).to(torch.int32), stable=True).indices          # free pages first, in order
    nth = (torch.cumsum(fresh.view(-1).long(), 0) - 1).clamp(min=0).view(na, mp)
    page_of = torch.where(fresh, free[nth.clamp(max=n_pages - 1)], torch.where(takes, old, -1))
    out[torch.where(fresh, page_of, n_pages).view(-1)] = 1
    # the partly filled page of a sequence that left it
    i = (kept // page).clamp(max=mp - 1)[:, None]
    copies = (leaves.gather(1, i) & (kept % page > 0)[:, None])[:, 0]
    # (a sequence that copies nothing writes a page back that no copy goes to)
    is_dst = torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda")
    is_dst[torch.where(copies, page_of.gather(1, i)[:, 0], n_pages)] = 1
    idle = is_dst[:n_pages].argmin()
    src = torch.where(copies, old.gather(1, i)[:, 0], idle)
    dst = torch.where(copies, page_of.gather(1, i)[:, 0], idle)
    part = (torch.arange(page, device="cuda") < (kept % page)[:, None])[None, :, None, None, :, None]
    pages[:, dst] = torch.where(part & copies[None, :, None, None, None, None], pages[:, src], pages[:, dst])
    return {"tables": page_of.to(torch.int32), "refs": out[:n_pages].to(torch.int32), "len": kept.to(torch.int32),
            "free": (out[:n_pages] == 0).sum(dtype=torch.int32).view(1), "pages": pages}


def _beam_plain(s):
    b, k, v = s["logits"].shape
    x = s["logits"].double()
    x = torch.where(torch.isfinite(x), x, -math.inf)
    top = x.amax(-1, keepdim=True)
    total = s["scores"].double()[..., None] + (x - (top + (x - top).exp().sum(-1, keepdim=True).log()))
    done = s["finished"].bool()[..., None]
    only = torch.where(torch.arange(v, device="cuda") == s["eos"], s["scores"].double()[..., None], -math.inf)
    total = torch.where(done, only, total).view(b, k * v)
    best, at = torch.sort(total, dim=-1, descending=True, stable=True)
    best, at = best[:, :k], at[:, :k]
    beam, token = at // v, at % v
    ends = torch.gather(s["finished"], 1, beam) | (token == s["eos"]).to(torch.int32)
    return {"tokens": token.to(torch.int32), "parents": (beam + torch.arange(b, device="cuda")[:, None] * k).to(torch.int32),
            "scores": best.float(), "finished": ends}


# ------------------------------------------------------------------ the framework's calls
def _own(s):
    import paper_2506_03566_b200 as lib
    kind = s["case"]["kind"]
    if kind == "attend":
        if s["case"]["append"]:
            lib.poss_pages_append(s["k"], s["v"], s["pages"], 0, s["tables"], s["prefix"], n_rows=s["rows"])
        out = lib.poss_paged_tree_attention(s["q"], s["pages"], 0, s["tables"], s["prefix"], s["mask"], s["scale"],
                                            n_rows=s["rows"], out=s["out"])
        return {"out": out, "pages": s["pages"]} if s["case"]["append"] else {"out": out}
    if kind == "compact":
        n = lib.poss_pages_compact(s["pages"], s["tables"], s["prefix"], s["path"], s["accepted"])
        return {"pages": s["pages"], "len": n}
    if kind == "remap":
        r = lib.poss_pages_remap(s["pages"], s["tables"], s["len"], s["refs"], s["parents"], s["room"])
        return {"tables": r["tables"], "refs": r["refs"], "len": r["seq_len"], "free": r["n_free"], "pages": s["pages"]}
    r = lib.poss_beam_select(s["logits"], s["scores"], finished=s["finished"], eos=s["eos"])
    return {"tokens": r["tokens"], "parents": r["parents"], "scores": r["scores"], "finished": r["finished"]}


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    return {"attend": _attend_plain, "compact": _compact_plain, "remap": _remap_plain, "beam": _beam_plain}[kind](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "beam":
        n = case["batch"] * case["beams"]
        # every logit read once; an exponential, a sum and a comparison each
        return {"bytes": n * case["vocab"] * size + n * 24, "flops": n * case["vocab"] * 4}
    hq, hkv, d = HEADS[case["heads"]]
    lengths = _lengths(case)
    if case["kind"] == "attend":
        rows = sorted(_tree_rows(case))
        slot = 2 * hkv * d * size
        n_rows, total = sum(rows), sum(lengths)
        # keys and values of the committed slots and of the trees once, queries and outputs once, new rows read and written
        bytes_ = (total + n_rows) * slot + 2 * n_rows * hq * d * size + (2 * n_rows * slot if case["append"] else 0)
        # (the rows of a sequence, on average: which sequence has which rows goes by the seed)
        pairs = total * n_rows / len(rows) + sum(m * (m + 1) / 2 for m in rows)
        return {"bytes": bytes_, "flops": 4 * pairs * hq * d}
    layer = 2 * hkv * d * size
    if case["kind"] == "compact":
        moved = case["batch"] * min(8, case["rows"] - 1) / 2
        return {"bytes": 2 * moved * case["layers"] * layer + case["batch"] * 80, "flops": 0}
    page, mp = case["page"], _max_pages(case)
    held = (sum(lengths) / page + case["before"]) * 4
    # a sequence in three leaves a partly filled page that it shares: half a page read and written in every layer
    copied = case["after"] / 3 * page / 2 * layer * case["layers"]
    return {"bytes": held + case["after"] * mp * 4 + 2 * copied, "flops": 0}


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "compact": _exact_compact, "remap": _exact_remap, "beam": _exact_beam}[case["kind"]](s)


def _exact_attend(s):
    b, r, hq, d = s["q"].shape
    pages = s["pages"][0]
    hkv, page = pages.shape[2], pages.shape[3]
    g = hq // hkv
    tables, prefix, rows = s["tables"].tolist(), s["prefix"].tolist(), s["rows"].tolist()
    mask = s["mask"].cpu().numpy().view(np.uint64)
    out = s["out"].double()
    for i in range(b):
        n, m = prefix[i], rows[i]
        held = tables[i][:-(-(n + m) // page)]
        kv = pages[held].transpose(0, 1).transpose(1, 2).reshape(2, hkv, len(held) * page, d)[:, :, :n + m].double()
        if s["case"]["append"]:
            kv[0, :, n:], kv[1, :, n:] = s["k"][i, :m].transpose(0, 1).double(), s["v"][i, :m].transpose(0, 1).double()
            for t in range(m):
                pages[held[(n + t) // page], 0, :, (n + t) % page] = s["k"][i, t]
                pages[held[(n + t) // page], 1, :, (n + t) % page] = s["v"][i, t]
        bits = [[bool(int(mask[i, x, y // 64]) >> (y % 64) & 1) for y in range(m)] for x in range(m)]
        hidden = torch.zeros(m, n + m, dtype=torch.bool, device="cuda")
        hidden[:, n:] = ~torch.tensor(bits, device="cuda").view(m, m)
        for h in range(hq):
            x = s["q"][i, :m, h].double() @ kv[0, h // g].T * s["scale"]
            p = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
            out[i, :m, h] = p @ kv[1, h // g]
    return {"out": out, "pages": s["pages"].double()} if s["case"]["append"] else {"out": out}


def _exact_compact(s):
    page = s["case"]["page"]
    tables, prefix = s["tables"].tolist(), s["prefix"].tolist()
    path, acc = s["path"].tolist(), s["accepted"].tolist()
    for i, (n, a) in enumerate(zip(prefix, acc)):
        for k in range(1, a + 1):
            src, dst = n + path[i][k], n + k
            s["pages"][:, tables[i][dst // page], :, :, dst % page] = s["pages"][:, tables[i][src // page], :, :, src % page]
    return {"pages": s["pages"].double(), "len": None}


def _exact_remap(s):
    page, pages = s["case"]["page"], s["pages"]
    tables, refs, lens = s["tables"].tolist(), s["refs"].tolist(), s["len"].tolist()
    parents, room = s["parents"].tolist(), s["room"].tolist()
    for t in tables:
        for p in t:
            if p >= 0:
                refs[p] -= 1
    new = []
    for p, n in zip(parents, room):
        need = -(-((lens[p] if p >= 0 else 0) + n) // page)
        new.append([x for x in (tables[p] if p >= 0 else []) if x >= 0][:need])
        for x in new[-1]:
            refs[x] += 1
    gone = []      # places that take a fresh page, in order of sequence and place
    for i, t in enumerate(new):
        kept = lens[parents[i]] if parents[i] >= 0 else 0
        for at in range(kept // page, -(-(kept + room[i]) // page)):
            if at < len(t) and refs[t[at]] > 1:
                refs[t[at]] -= 1
                gone.append((i, at, t[at], min(page, kept - at * page)))
            elif at >= len(t):
                gone.append((i, at, None, 0))
    free = [x for x, n in enumerate(refs) if n == 0]
    for (i, at, src, n), dst in zip(gone, free):
        if n > 0:
            pages[:, dst, :, :, :n] = pages[:, src, :, :, :n]
    return {"tables": None, "refs": None, "len": None, "free": None, "pages": pages.double()}


def _exact_beam(s):
    b, k, v = s["logits"].shape
    best = torch.full((b, k), -math.inf, dtype=torch.float64, device="cuda")
    fin = s["finished"].tolist()
    for i in range(b):
        every = []
        for j in range(k):
            x = s["logits"][i, j].double()
            sc = s["scores"][i, j].double()
            every.append(sc.view(1) if fin[i][j] else torch.topk(sc + torch.log_softmax(x, -1), min(k, v)).values)
        got = torch.sort(torch.cat(every), descending=True).values[:k]
        best[i, :got.numel()] = got
    return {"tokens": None, "parents": None, "scores": best, "finished": None}
