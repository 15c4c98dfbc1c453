"""Operators around long paged caches and their answers: cases, plain forms and the framework's calls.

A paged cache holds the keys and values of many sequences in pages of `page` slots:
kv_pages [layers][pages][2][kv heads][page][head dimension]; tables[sequence][i] names the page that holds the
sequence's slots [i*page, (i+1)*page), -1 behind its last page.  mass [layers][batch][kv heads][slots] holds the attention
weight that each slot has drawn so far.

  rotate  rotary positions on queries and keys: halves or neighbours of a head as pairs, a part of the head, frequencies
          scaled for long contexts; the rotated keys and the values go behind each sequence's slots in its pages (append),
          or the queries of a contiguous batch are rotated alone
  mass    tree attention over pages (one row: plain decoding) that also adds up each slot's attention weight
  evict   of every sequence's slots the first, the last and the most attended ones stay and move to the front, per layer and
          KV head
  score   log-probabilities of given tokens, the rows' entropies and their best alternatives, over the vocabulary
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
        # one sequence, one token a step, far into a long context: the latency of plain decoding
        {"name": "rotate decode 1", "kind": "rotate", "heads": "8b", "dtype": "bf16", "batch": 1, "rows": 1, "ragged": False,
         "part": 1, "pairs": "half", "scaled": True, "page": 16, "append": True},
        # a serving batch of 16 draft trees of up to 61 rows; neighbours as pairs, half of the head
        {"name": "rotate tree61 16", "kind": "rotate", "heads": "8b", "dtype": "bf16", "batch": 16, "rows": 61, "ragged": True,
         "part": 2, "pairs": "neighbours", "scaled": False, "page": 16, "append": True},
        # four prompts of 2048 tokens
        {"name": "rotate prompt 4x2048", "kind": "rotate", "heads": "8b", "dtype": "bf16", "batch": 4, "rows": 2048,
         "ragged": False, "part": 1, "pairs": "half", "scaled": True, "page": 64, "append": True},
        # the check mode in 32 bits, queries alone, a quarter of the head
        {"name": "rotate check 5x300", "kind": "rotate", "heads": "toy", "dtype": "fp32", "batch": 5, "rows": 300,
         "ragged": False, "part": 4, "pairs": "half", "scaled": True, "page": 24, "append": False},
        # one sequence, one token a step, 1024 slots: the latency of plain decoding
        {"name": "mass decode 1x1024", "kind": "mass", "heads": "8b", "dtype": "bf16", "batch": 1, "rows": 1,
         "ragged": False, "prefix": 1024, "page": 16, "weighted": False},
        # a serving batch of 64 sequences, one token each
        {"name": "mass decode 64x8000", "kind": "mass", "heads": "8b", "dtype": "bf16", "batch": 64, "rows": 1,
         "ragged": False, "prefix": 8000, "page": 32, "weighted": False},
        # a serving batch: 16 trees of up to 61 rows over 4096 to 8191 slots, every row with its draft probability
        {"name": "mass tree61 16x8191", "kind": "mass", "heads": "8b", "dtype": "bf16", "batch": 16, "rows": 61,
         "ragged": True, "prefix": 8191, "page": 16, "weighted": True},
        # three short sequences of a two-layer check model, pages of an odd size
        {"name": "evict check 3x700", "kind": "evict", "heads": "toy", "dtype": "fp32", "batch": 3, "layers": 2,
         "length": 700, "keep": 301, "page": 24},
        # four sequences of up to 8191 slots cut to 2048 in eight layers
        {"name": "evict 4x8191 to 2048", "kind": "evict", "heads": "8b", "dtype": "bf16", "batch": 4, "layers": 8,
         "length": 8191, "keep": 2048, "page": 64},
        # a draft tree of 60 tokens and its root: the target's log-probability of every drafted token in its parent's row
        {"name": "score tree61x32000", "kind": "score", "dtype": "bf16", "rows": 61, "vocab": 32000, "topk": 4, "tree": True,
         "temperature": 1.0},
        # one sampled token with its ten best alternatives
        {"name": "score 1x128256", "kind": "score", "dtype": "fp32", "rows": 1, "vocab": 128256, "topk": 10, "tree": False,
         "temperature": 0.7},
        # a prompt of 2048 tokens scored
        {"name": "score 2048x128256", "kind": "score", "dtype": "bf16", "rows": 2048, "vocab": 128256, "topk": 1,
         "tree": False, "temperature": 1.0},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "mass", "mass", "evict", "score"])
    if kind == "rotate":
        heads, dtype = rng.choice(list(HEADS)), rng.choice(["bf16", "bf16", "fp32"])
        hq, hkv, d = HEADS[heads]
        rows, batch = rng.choice([1, _spread(rng, 1, 2048)]), _spread(rng, 1, 64)
        while batch > 1 and batch * rows * (hq + 2 * hkv) * d * (2 if dtype == "bf16" else 4) > 90_000_000:
            batch -= 1
        while rows > 1 and rows * (hq + 2 * hkv) * d * (2 if dtype == "bf16" else 4) > 90_000_000:
            rows //= 2
        return {"kind": kind, "heads": heads, "dtype": dtype, "batch": batch, "rows": rows, "ragged": rng.random() < 0.5,
                "part": rng.choice([1, 1, 2, 4]), "pairs": rng.choice(["half", "neighbours"]), "scaled": rng.random() < 0.5,
                "page": rng.choice([16, 24, 32, 64, 128]), "append": rng.random() < 0.7}
    if kind == "mass":
        heads = rng.choice(["8b", "8b", "13b", "mid", "small", "toy", "tiny"])
        dtype = "fp32" if heads in ("toy", "tiny") else "bf16"
        rows = rng.choice([1, _spread(rng, 1, 128)])
        hq, hkv, d = HEADS[heads]
        prefix = _spread(rng, 1, 12000 if dtype == "bf16" else 2000) - 1
        batch = _spread(rng, 1, 64)
        slots = prefix + rows + 64
        while batch > 1 and (batch * hq * rows * slots > 150_000_000 or batch * slots * hkv * d > 400_000_000):
            batch -= 1
        return {"kind": kind, "heads": heads, "dtype": dtype, "batch": batch, "rows": rows, "ragged": rng.random() < 0.5,
                "prefix": prefix, "page": rng.choice([16, 16, 32, 64, 128, 256]) if dtype == "bf16" else rng.choice([8, 16, 24, 64]),
                "weighted": rng.random() < 0.5}
    if kind == "evict":
        heads, dtype = rng.choice(list(HEADS)), rng.choice(["bf16", "bf16", "fp32"])
        hq, hkv, d = HEADS[heads]
        length, layers, batch = _spread(rng, 20, 12000), _spread(rng, 1, 16), _spread(rng, 1, 16)
        while batch * layers > 1 and batch * layers * length * hkv * d > 120_000_000:
            batch, layers = max(1, batch - 1), max(1, layers - 1)
        return {"kind": kind, "heads": heads, "dtype": dtype, "batch": batch, "layers": layers, "length": length,
                "keep": max(12, int(length * rng.uniform(0.1, 0.95))), "page": rng.choice([8, 16, 24, 32, 64])}
    rows, vocab = rng.choice([_spread(rng, 1, 2048), rng.randint(1, 128)]), _spread(rng, 100, 128256)
    return {"kind": kind, "dtype": rng.choice(["fp32", "bf16"]) if rows * vocab < 120_000_000 else "bf16", "rows": rows,
            "vocab": vocab, "topk": rng.randint(0, 16), "tree": rng.random() < 0.5,
            "temperature": rng.choice([0.6, 1.0, 1.0, 1.5])}


# ------------------------------------------------------------------ sizes that a case fixes
FIRST, RECENT = 4, 8        # slots at both ends that an eviction keeps in any case


def _lengths(case):
    """Slots of each sequence: spread over the upper half of [0, prefix], one of them at prefix."""
    b, p = case["batch"], case.get("prefix", case.get("length"))
    return [p - int((i * 0.6180339887) % 1.0 * (p // 2 + 1)) for i in range(b)]


def _tree_rows(case):
    """Rows of each sequence's tree: all alike, or spread over [1, rows]."""
    b, r = case["batch"], case["rows"]
    return [r - int((i * 0.7548776662) % 1.0 * r) if case["ragged"] else r for i in range(b)]


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


def _parents(batch, rows, seed):
    """Random trees: row 0 is the root, a row's parent is an earlier row."""
    rs = np.random.RandomState(seed % (1 << 31))
    parents = np.full((batch, rows), -1, dtype=np.int64)
    for r in range(1, rows):
        parents[:, r] = r - 1 - (rs.random_sample(batch) * min(r, 12)).astype(np.int64)
    return parents


def _masks(parents):
    """Ancestor bits of the trees."""
    batch, rows = parents.shape
    m = np.zeros((batch, rows, (rows + 63) // 64), dtype=np.uint64)
    every = np.arange(batch)
    for r in range(rows):
        if r:
            m[:, r] = m[every, parents[:, r]]
        m[:, r, r // 64] |= np.uint64(1) << np.uint64(r % 64)
    return m.view(np.int64)


def _frequencies(case, d):
    """Radians per position of each pair; scaled: the slow ones divided by 8, the ones between blended, for contexts of 8 x 8192."""
    r = d // case["part"]
    f = [500000.0 ** (-2.0 * i / r) for i in range(r // 2)]
    if case["scaled"]:
        turns = [8192 * x / (2 * math.pi) for x in f]
        share = [min(1.0, max(0.0, (t - 1.0) / (4.0 - 1.0))) for t in turns]
        f = [x * s + x / 8 * (1 - s) for x, s in zip(f, share)]
    return f


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    dev = "cuda"

    def cuda(a):
        return torch.from_numpy(np.ascontiguousarray(a)).to(dev)

    def randn(*shape):
        return torch.randn(*shape, device=dev, generator=gen).to(dt)

    dt = _dtype(case)
    if case["kind"] == "score":
        rows, v = case["rows"], case["vocab"]
        # logits of a language model: wide, a few far above the rest; the tokens are likely ones
        x = torch.randn(rows, v, device=dev, generator=gen).mul_(2.5).to(dt)
        tokens = torch.multinomial(torch.rand(rows, min(v, 64), device=dev, generator=gen), 1, generator=gen)[:, 0]
        tokens = (tokens * 37 % v).to(torch.int32)
        rows_of = cuda(_parents(1, rows, seed)[0].astype(np.int32)) if case["tree"] else None
        return {"case": case, "logits": x, "tokens": tokens, "rows_of": rows_of}

    hq, hkv, d = HEADS[case["heads"]]
    page, b = case["page"], case["batch"]
    if case["kind"] == "rotate":
        r = case["rows"]
        rows = _tree_rows(case)
        random.Random(seed + 1).shuffle(rows)
        rs = np.random.RandomState(seed % (1 << 31))
        # what the caches hold is short (an eviction cut it), the positions are far on: a chain, or a tree's depths
        far = rs.randint(0, 200000, b)
        prefix = rs.permutation(np.arange(b) * 37 % 100).astype(np.int32)
        depth = np.tile(np.arange(r), (b, 1))
        if 1 < r <= 128:
            parents, depth = _parents(b, r, seed), np.zeros((b, r), np.int64)
            for i in range(1, r):
                depth[:, i] = depth[np.arange(b), parents[:, i]] + 1
        state = {"case": case, "q": randn(b, r, hq, d), "rows": cuda(np.array(rows, np.int32)), "out_q": torch.zeros(b, r, hq, d, dtype=dt, device=dev),
                 "at": cuda((far[:, None] + depth).astype(np.int32)), "freq": torch.tensor(_frequencies(case, d), dtype=torch.float64, device=dev),
                 "magnitude": 1.1 if case["scaled"] else 1.0}
        if case["append"]:
            held = [int(n) + m for n, m in zip(prefix, rows)]
            n_pages = sum(-(-(int(n) + r) // page) for n in prefix) + 3
            mp = max(-(-(int(n) + r) // page) for n in prefix)
            # (keys and values as they lie in a fused projection's output)
            kv = randn(b, r, 2 * hkv, d)
            state |= {"k": kv[:, :, :hkv], "v": kv[:, :, hkv:], "prefix": cuda(prefix), "pages": randn(1, n_pages, 2, hkv, page, d),
                      "tables": cuda(_tables(held, page, mp, n_pages, seed))}
        return state

    lengths = _lengths(case)
    random.Random(seed).shuffle(lengths)
    if case["kind"] == "mass":
        r = case["rows"]
        rows = _tree_rows(case)
        random.Random(seed + 1).shuffle(rows)
        held = [n + m for n, m in zip(lengths, rows)]
        n_pages = sum(-(-n // page) for n in held) + 7
        mp = -(-(case["prefix"] + r) // page) + 1
        weights = torch.rand(b, r, device=dev, generator=gen) if case["weighted"] else None
        # what a few steps have left
        mass = torch.rand(1, b, hkv, mp * page, device=dev, generator=gen) * (16.0 / (case["prefix"] + 1))
        return {"case": case, "pages": torch.randn(1, n_pages, 2, hkv, page, d, device=dev, dtype=dt, generator=gen),
                "tables": cuda(_tables(held, page, mp, n_pages, seed)), "q": randn(b, r, hq, d), "mass": mass,
                "prefix": cuda(np.array(lengths, np.int32)), "rows": cuda(np.array(rows, np.int32)), "weights": weights,
                "mask": cuda(_masks(_parents(b, r, seed))), "scale": 1.0 / math.sqrt(d), "out": torch.zeros(b, r, hq, d, dtype=dt, device=dev)}
    # evict: attention weight as it comes about, a few slots with much of it; the budgets of some sequences are wider
    layers = case["layers"]
    n_pages = sum(-(-n // page) for n in lengths) + 7
    mp = -(-case["length"] // page) + 1
    mass = torch.rand(layers, b, hkv, mp * page, device=dev, generator=gen).pow_(6) * 8
    keep = [case["keep"] if i % 5 < 4 else case["keep"] * 2 for i in range(b)]
    return {"case": case, "pages": torch.randn(layers, n_pages, 2, hkv, page, d, device=dev, dtype=dt, generator=gen),
            "tables": cuda(_tables(lengths, page, mp, n_pages, seed)), "len": cuda(np.array(lengths, np.int32)), "mass": mass,
            "keep": cuda(np.array(keep, np.int32)), "out_mass": torch.zeros_like(mass)}


# ------------------------------------------------------------------ plain forms
def _turn(x, at, freq, pairs, magnitude):
    """x [...][heads][d] in 32 bits turned by at [...] positions; the angles in 64."""
    half = freq.shape[0]
    a = at.double()[..., None] * freq
    c, s = (a.cos() * magnitude).float()[..., None, :], (a.sin() * magnitude).float()[..., None, :]
    x = x.float()
    if pairs == "half":
        u, v, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
        return torch.cat([u * c - v * s, v * c + u * s, rest], -1)
    u, v, rest = x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]
    return torch.cat([torch.stack([u * c - v * s, v * c + u * s], -1).flatten(-2), rest], -1)


def _rotate_plain(s):
    case, dt = s["case"], s["q"].dtype
    b, r = s["q"].shape[:2]
    at = torch.arange(r, device="cuda")
    if not case["append"]:
        s["out_q"].copy_(_turn(s["q"], s["at"], s["freq"], case["pairs"], s["magnitude"]))
        return {"q": s["out_q"]}
    live = at < s["rows"][:, None]
    q = _turn(s["q"], s["at"], s["freq"], case["pairs"], s["magnitude"]).to(dt)
    s["out_q"].copy_(torch.where(live[..., None, None], q, s["out_q"]))
    k = _turn(s["k"], s["at"], s["freq"], case["pairs"], s["magnitude"]).to(dt)
    pages, page = s["pages"], case["page"]
    slot = s["prefix"].long()[:, None] + at
    p = s["tables"].long().gather(1, slot // page)
    # rows behind a sequence's last one write nothing: they go where the first row goes, with its values
    p, off = torch.where(live, p, p[:, :1]), torch.where(live, slot % page, slot[:, :1] % page)
    for which, new in ((0, k), (1, s["v"])):
        pages[0, p, which, :, off] = torch.where(live[..., None, None], new, new[:, :1])
    return {"q": s["out_q"], "pages": pages}


def _mass_plain(s):
    b, r, hq, d = s["q"].shape
    pages, tables = s["pages"][0], s["tables"].long().clamp(min=0)
    hkv, page = pages.shape[2], pages.shape[3]
    g, slots = hq // hkv, tables.shape[1] * page
    k, v = (pages[:, w][tables].permute(0, 2, 1, 3, 4).reshape(b, hkv, slots, d).float() for w in (0, 1))
    q = s["q"].view(b, r, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, r * g, d).float()
    at = torch.arange(slots, device="cuda") - s["prefix"][:, None]                      # [b][slots]: place in the tree
    j = at.clamp(0, r - 1)
    live = torch.arange(r, device="cuda") < s["rows"][:, None]
    bits = s["mask"].gather(2, (j // 64)[:, None].expand(b, r, slots).long()) >> (j % 64)[:, None]
    seen = (at < 0)[:, None] | ((bits & 1).bool() & ((at >= 0) & (at < s["rows"][:, None]))[:, None])
    x = (q @ k.transpose(2, 3)).mul_(s["scale"]).view(b, hkv, r, g, slots)
    x.masked_fill_(~seen[:, None, :, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    x = x.div_(x.sum(-1, keepdim=True)).view(b, hkv, r * g, slots)
    o = (x @ v).view(b, hkv, r, g, d).permute(0, 2, 1, 3, 4).reshape(b, r, hq, d)
    s["out"].copy_(torch.where(live[..., None, None], o.to(s["out"].dtype), s["out"]))
    w = live.float() if s["weights"] is None else torch.where(live, s["weights"], 0.0)
    new = (x.view(b, hkv, r, g, slots).sum(3) * w[:, None, :, None]).sum(2)             # [b][hkv][slots]
    old = s["mass"][0]
    mine, tree = (at < 0)[:, None], ((at >= 0) & (at < s["rows"][:, None]))[:, None]
    old.copy_(torch.where(mine, old + new, torch.where(tree, new, old)))
    return {"out": s["out"], "mass": s["mass"]}


def _evict_plain(s):
    pages, page = s["pages"], s["case"]["page"]
    layers, b, hkv, slots = s["mass"].shape
    at = torch.arange(slots, device="cuda")
    n, keep = s["len"].long(), torch.minimum(s["keep"].long(), s["len"].long())
    held = at < n[:, None]                                                              # [b][slots]
    always = held & ((at < FIRST) | (at >= (n - RECENT)[:, None]) | (n <= keep)[:, None])
    x = torch.where(always[:, None], math.inf, torch.where(held[:, None], s["mass"], -math.inf))
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices                 # greatest first, ties by slot
    rank = torch.empty_like(order).scatter_(-1, order, at.expand_as(order).contiguous())
    stays = rank < keep[:, None, None]
    # kept slots first, in their order
    src = torch.sort((~stays).to(torch.int32), dim=-1, stable=True).indices             # [layers][b][hkv][slots]
    most = min(slots, s["case"]["keep"] * (2 if b > 4 else 1))                           # of no sequence more stay
    dst = at[:most].expand(layers, b, hkv, most)
    src = torch.where(dst < keep[:, None, None], src[..., :most], dst)
    moved = torch.where(dst < keep[:, None, None], s["mass"].gather(-1, src), s["out_mass"][..., :most])
    s["out_mass"][..., :most] = moved
    # places behind the kept ones write a slot that stays onto itself: the first
    src, dst = (torch.where(dst < keep[:, None, None], i, 0) for i in (src, dst))
    t = s["tables"].long().clamp(min=0)
    seq = torch.arange(b, device="cuda")[:, None, None]
    lay, head = torch.arange(layers, device="cuda")[:, None, None, None], torch.arange(hkv, device="cuda")[:, None]
    for w in (0, 1):
        new = pages[lay, t[seq, src // page], w, head, src % page]
        new = torch.where((dst == 0)[..., None], new[..., :1, :], new)
        pages[lay, t[seq, dst // page], w, head, dst % page] = new
    return {"pages": pages, "mass": s["out_mass"], "len": keep.to(torch.int32)}


def _score_plain(s):
    case, x = s["case"], s["logits"].float()
    rows, v = x.shape
    x = torch.where(x.abs() < math.inf, x, -math.inf) / case["temperature"]
    top = x.amax(-1, keepdim=True)
    z = x - top
    e = z.exp()
    total = e.sum(-1, keepdim=True, dtype=torch.float64)
    lse = total.log()
    entropy = lse[:, 0] - (e * torch.where(e > 0, z, 0.0)).sum(-1, dtype=torch.float64) / total[:, 0]
    of = torch.arange(rows, device="cuda") if s["rows_of"] is None else s["rows_of"].long()
    logp = z[of.clamp(min=0), s["tokens"].long()].double() - lse[of.clamp(min=0), 0]
    out = {"logp": torch.where(of >= 0, logp, 0.0).float(), "entropy": entropy.float()}
    if case["topk"]:
        # values in order, ties by token: both in one whole number
        bits = s["logits"].float().add(0.0).view(torch.int32).long()
        key = torch.where(bits >= 0, bits, -(bits & 0x7fffffff) - 1)
        best = torch.topk(key * (1 << 31) + (v - 1 - torch.arange(v, device="cuda")), case["topk"], dim=-1).values
        at = v - 1 - best % (1 << 31)
        out |= {"tokens": at.to(torch.int32), "best": (z.gather(-1, at).double() - lse).float()}
    return out


# ------------------------------------------------------------------ the framework's calls
def _own(s):
    import paper_2506_03566_b200 as lib
    case = s["case"]
    if case["kind"] == "rotate":
        how = {"interleaved": case["pairs"] == "neighbours", "magnitude": s["magnitude"]}
        if not case["append"]:
            return {"q": lib.poss_rotary(s["q"], s["at"], s["freq"], out=s["out_q"], **how)}
        q = lib.poss_pages_append_rotary(s["k"], s["v"], s["pages"], 0, s["tables"], s["prefix"], s["freq"], positions=s["at"], q=s["q"],
                                         out_q=s["out_q"], n_rows=s["rows"], **how)
        return {"q": q, "pages": s["pages"]}
    if case["kind"] == "mass":
        out = lib.poss_paged_tree_attention_mass(s["q"], s["pages"], s["mass"], 0, s["tables"], s["prefix"], s["mask"], s["scale"],
                                                 n_rows=s["rows"], row_weights=s["weights"], out=s["out"])
        return {"out": out, "mass": s["mass"]}
    if case["kind"] == "evict":
        n = lib.poss_pages_evict(s["pages"], s["mass"], s["tables"], s["len"], s["keep"], first=FIRST, recent=RECENT, out_mass=s["out_mass"])
        return {"pages": s["pages"], "mass": s["out_mass"], "len": n}
    r = lib.poss_token_logprobs(s["logits"], s["tokens"], token_rows=s["rows_of"], topk=case["topk"], temperature=case["temperature"])
    out = {"logp": r["logp"], "entropy": r["entropy"]}
    return out | {"tokens": r["top_tokens"], "best": r["top_logp"]} if case["topk"] else out


def run(state):
    if own:
        return _own(state)
    return {"rotate": _rotate_plain, "mass": _mass_plain, "evict": _evict_plain, "score": _score_plain}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "score":
        n = case["rows"] * case["vocab"]
        # every logit read once; an exponential, a sum, a product and a comparison each
        return {"bytes": n * size + case["rows"] * (12 + 8 * case["topk"]), "flops": 5 * n}
    hq, hkv, d = HEADS[case["heads"]]
    if case["kind"] == "rotate":
        n = sum(_tree_rows(case)) if case["append"] else case["batch"] * case["rows"]
        heads = hq + (2 * hkv if case["append"] else 0)
        turned = hq + (hkv if case["append"] else 0)
        return {"bytes": 2 * n * heads * d * size + 4 * n, "flops": 3 * n * turned * d // case["part"]}
    total = sum(_lengths(case))
    if case["kind"] == "mass":
        rows = _tree_rows(case)
        n_rows = sum(rows)
        # keys, values and queries once, outputs once, the slots' weights read and written
        bytes_ = (total + n_rows) * (2 * hkv * d * size + 8 * hkv) + 2 * n_rows * hq * d * size
        # (the rows of a sequence, on average: which sequence has which rows goes by the seed)
        pairs = total * n_rows / len(rows) + sum(m * (m + 1) / 2 for m in rows)
        return {"bytes": bytes_, "flops": 4 * pairs * hq * d}
    # every slot's weight once, every kept slot behind the first ones from its place to the new one
    kept = sum(min(n, case["keep"]) for n in _lengths(case))
    per = case["layers"] * hkv
    return {"bytes": per * (4 * total + 4 * kept + 4 * d * size * (kept - FIRST * case["batch"])), "flops": 0}


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "mass": _exact_mass, "evict": _exact_evict, "score": _exact_score}[case["kind"]](s)


def _exact_turned(x, at, freq, pairs, magnitude):
    """One row [heads][d] as complex numbers times e^(i at f)."""
    half = freq.shape[0]
    y = x.double().clone()
    u, v = (slice(0, half), slice(half, 2 * half)) if pairs == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = torch.complex(y[..., u], y[..., v]) * torch.polar(torch.full_like(freq, magnitude), at[..., None, None].double() * freq)
    y[..., u], y[..., v] = z.real, z.imag
    return y


def _exact_rotate(s):
    case = s["case"]
    how = (s["freq"], case["pairs"], s["magnitude"])
    out = s["out_q"].double()
    rows = s["rows"].tolist() if case["append"] else [case["rows"]] * case["batch"]
    pages = s["pages"].double() if case["append"] else None
    for i, m in enumerate(rows):
        out[i, :m] = _exact_turned(s["q"][i, :m], s["at"][i, :m], *how)
        if case["append"]:
            n, page = int(s["prefix"][i]), case["page"]
            slot = torch.arange(n, n + m, device="cuda")
            p = s["tables"][i].long()[slot // page]
            pages[0, p, 0, :, slot % page] = _exact_turned(s["k"][i, :m], s["at"][i, :m], *how)
            pages[0, p, 1, :, slot % page] = s["v"][i, :m].double()
    return {"q": out, "pages": pages} if case["append"] else {"q": out}


def _exact_mass(s):
    b, r, hq, d = s["q"].shape
    pages = s["pages"][0]
    hkv, page = pages.shape[2], pages.shape[3]
    g = hq // hkv
    tables, prefix, rows = s["tables"].tolist(), s["prefix"].tolist(), s["rows"].tolist()
    mask = s["mask"].cpu().numpy().view(np.uint64)
    out, mass = s["out"].double(), s["mass"].double()
    for i in range(b):
        n, m = prefix[i], rows[i]
        held = tables[i][:-(-(n + m) // page)]
        kv = pages[held].transpose(0, 1).transpose(1, 2).reshape(2, hkv, len(held) * page, d)[:, :, :n + m].double()
        bits = [[bool(int(mask[i, x, y // 64]) >> (y % 64) & 1) for y in range(m)] for x in range(m)]
        hidden = torch.zeros(m, n + m, dtype=torch.bool, device="cuda")
        hidden[:, n:] = ~torch.tensor(bits, device="cuda").view(m, m)
        w = torch.ones(m, dtype=torch.float64, device="cuda") if s["weights"] is None else s["weights"][i, :m].double()
        mass[0, i, :, n:n + m] = 0.0
        for h in range(hq):
            x = s["q"][i, :m, h].double() @ kv[0, h // g].T * s["scale"]
            p = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
            out[i, :m, h] = p @ kv[1, h // g]
            mass[0, i, h // g, :n + m] += w @ p
    return {"out": out, "mass": mass}


def _exact_evict(s):
    page, pages, mass = s["case"]["page"], s["pages"], s["out_mass"].double()
    layers, b, hkv, _ = s["mass"].shape
    if layers * b * hkv > 2000:
        return None
    every = s["mass"].cpu().numpy()
    for i in range(b):
        n, keep = int(s["len"][i]), int(s["keep"][i])
        t = s["tables"][i].long()
        for la in range(layers):
            for h in range(hkv):
                x = every[la, i, h, :n]
                kept = np.arange(n)
                if n > keep:
                    inner = np.arange(FIRST, n - RECENT)
                    best = inner[np.lexsort((inner, -x[inner].astype(np.float64)))][:keep - FIRST - RECENT]
                    kept = np.sort(np.concatenate([np.arange(FIRST), best, np.arange(n - RECENT, n)]))
                src = torch.from_numpy(kept).cuda()
                dst = torch.arange(len(kept), device="cuda")
                pages[la, t[dst // page], :, h, dst % page] = pages[la, t[src // page], :, h, src % page]
                mass[la, i, h, :len(kept)] = torch.from_numpy(x[kept].astype(np.float64)).cuda()
    return {"pages": pages.double(), "mass": mass, "len": None}


def _exact_score(s):
    case = s["case"]
    rows, k = case["rows"], case["topk"]
    of = list(range(rows)) if s["rows_of"] is None else s["rows_of"].tolist()
    tokens = s["tokens"].long()
    entropy = torch.zeros(rows, dtype=torch.float64, device="cuda")
    best = torch.zeros(rows, k, dtype=torch.float64, device="cuda")
    logp = torch.zeros(rows, dtype=torch.float64, device="cuda")
    at = torch.tensor(of, device="cuda")
    for r in range(rows):
        x = torch.log_softmax(s["logits"][r].double() / case["temperature"], -1)
        entropy[r] = -(x.exp() * x).sum()
        if k:
            best[r] = torch.topk(x, k).values
        logp += torch.where(at == r, x[tokens], 0.0)
    out = {"logp": logp, "entropy": entropy}
    return out | {"tokens": None, "best": best} if k else out
