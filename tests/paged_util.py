"""Plain 64-bit forms of the paged-cache calls, and case makers, for the tests.

Tolerance of the attention, per output element, derived from the arithmetic (worst cases, no statistics):
  * the output is rounded once: half a step of its type, eps/2 relative to the value;
  * bf16 on the tensor cores: every probability is rounded to bf16 before the second product, half a step (2^-8)
    relative: the output moves by at most 2^-8 x A, A = sum_s w_s |v_s| (the same attention over |V|);
  * a score is a sum of d fp32 products: off by at most (d + 8) x 2^-22 x scale x sum |q k| (2^-24 per addition, a factor
    four for products that the tensor cores align before they add), and a score error e changes every probability by a
    factor within exp(+-e), so the output by at most 2 e A (numerator and denominator);
  * 2^x to 2^-21 relative, sums over n keys in any order: n x 2^-24 relative, in numerator and denominator each.
"""
import math

import numpy as np
import torch


def tree_masks(rng, batch, rows):
    """Ancestor bits of random trees, int64 [batch][rows][words], and the same as bool [batch][rows][rows]."""
    anc = np.zeros((batch, rows, rows), dtype=bool)
    for b in range(batch):
        for r in range(rows):
            if r:
                anc[b, r] = anc[b, rng.integers(max(0, r - 6), r)]
            anc[b, r, r] = True
    return pack(anc), anc


def pack(anc):
    batch, rows, _ = anc.shape
    words = (rows + 63) // 64
    m = np.zeros((batch, rows, words), dtype=np.uint64)
    for j in range(rows):
        m[:, :, j // 64] |= anc[:, :, j].astype(np.uint64) << np.uint64(j % 64)
    return m.view(np.int64)


def make_tables(rng, lens, page, n_pages, max_pages):
    order = rng.permutation(n_pages)
    t = np.full((len(lens), max_pages), -1, dtype=np.int32)
    at = 0
    for i, n in enumerate(lens):
        k = -(-n // page)
        t[i, :k] = order[at:at + k]
        at += k
    assert at <= n_pages
    return t


def attention(q, pages, tables, prefix, n_rows, anc, scale):
    """64-bit tree attention over one layer's pages [n][2][heads][page][d] (all on the CPU); returns (out, tolerance
    without the roundings that depend on the kernel, A): three arrays [batch][rows][query heads][d].  Unseen slots are not
    touched.  Rows that see nothing are zeros; rows behind n_rows stay NaN in `out`."""
    batch, rows, hq, d = q.shape
    hkv, page = pages.shape[2], pages.shape[3]
    g = hq // hkv
    out = torch.full(q.shape, math.nan, dtype=torch.float64)
    tol = torch.zeros_like(out)
    big = torch.zeros_like(out)
    for b in range(batch):
        p, n = int(prefix[b]), int(n_rows[b])
        for r in range(n):
            slots = [s for s in range(p + n) if (s < p or anc[b][r][s - p])
                     and 0 <= tables[b][s // page] < pages.shape[0]]
            if not slots:
                out[b, r] = 0.0
                continue
            pg = torch.tensor([int(tables[b][s // page]) for s in slots])
            off = torch.tensor([s % page for s in slots])
            kv = pages[pg, :, :, off].double()                     # [slots][2][heads][d]
            for h in range(hq):
                k, v = kv[:, 0, h // g], kv[:, 1, h // g]
                x = (k @ q[b, r, h].double()) * scale
                w = torch.softmax(x, 0)
                e = (d + 8) * 2.0 ** -22 * abs(scale) * float((k.abs() @ q[b, r, h].double().abs()).max())
                a = w @ v.abs()
                out[b, r, h] = w @ v
                big[b, r, h] = a
                tol[b, r, h] = a * (2 * e + 2.0 ** -19 + 2 * len(slots) * 2.0 ** -24)
    return out, tol, big


def check_attention(got, want, tol, big, dtype, tensor_cores):
    live = ~torch.isnan(want)
    bound = tol + want.abs() * torch.finfo(dtype).eps / 2 + (big * 2.0 ** -8 if tensor_cores else 0.0) + 1e-30
    err = (got.double().cpu() - want).abs()
    assert torch.isfinite(got.float().cpu()[live]).all()
    worst = float((err[live] / bound[live]).max()) if live.any() else 0.0
    assert worst <= 1.0, worst
    return worst


def remap(tables, seq_len, refs, parents, room, page):
    """The definition, one new sequence after the other.  Returns (tables, refs, lengths, free, copies) or None and the
    number of missing pages; copies: (source, target, slots)."""
    max_pages = len(tables[0]) if len(tables) else 0
    refs = [int(x) for x in refs]
    for t in tables:
        for p in t:
            if p >= 0:
                refs[p] -= 1
    new, kept = [], []
    for i, p in enumerate(parents):
        n = int(seq_len[p]) if p >= 0 else 0
        need = -(-(n + int(room[i])) // page)
        row = [(int(tables[p][at]) if p >= 0 else -1) for at in range(need)]
        for x in row:
            if x >= 0:
                refs[x] += 1
        new.append(row)
        kept.append(n)
    gone = []
    for i, row in enumerate(new):
        for at, x in enumerate(row):
            if x < 0:
                gone.append((i, at, -1, 0))
            elif at >= kept[i] // page and refs[x] > 1:
                refs[x] -= 1
                gone.append((i, at, x, max(0, min(page, kept[i] - at * page))))
    free = [x for x, n in enumerate(refs) if n == 0]
    if len(free) < len(gone):
        return None, len(gone) - len(free)
    copies = []
    for (i, at, src, n), dst in zip(gone, free):
        new[i][at] = dst
        refs[dst] = 1
        if n > 0:
            copies.append((src, dst, n))
    out = np.full((len(parents), max_pages), -1, dtype=np.int32)
    for i, row in enumerate(new):
        out[i, :len(row)] = row
    return (out, np.array(refs, np.int32), np.array(kept, np.int32), sum(n == 0 for n in refs), copies), 0


def beam_select(logits, scores, finished, eos):
    """The definition in 64 bits: logits float64 [batch][beams][vocab]."""
    batch, k, v = logits.shape
    tok = np.full((batch, k), -1, np.int32)
    par = np.full((batch, k), -1, np.int32)
    sc = np.full((batch, k), -np.inf)
    fin = np.ones((batch, k), np.int32)
    for b in range(batch):
        cand = []
        for j in range(k):
            if not np.isfinite(scores[b, j]):
                continue
            if finished is not None and finished[b, j]:
                cand.append((float(scores[b, j]), j, eos))
                continue
            x = logits[b, j]
            on = np.isfinite(x)
            if not on.any():
                continue
            top = x[on].max()
            lse = top + math.log(math.fsum(np.exp(x[on] - top)))
            s = float(scores[b, j]) + (x - lse)
            order = np.lexsort((np.arange(v), -np.where(on, x, -np.inf)))[:k]
            cand += [(float(s[t]), j, int(t)) for t in order if on[t]]
        cand.sort(key=lambda c: (-c[0], c[1], c[2]))
        for r, (s, j, t) in enumerate(cand[:k]):
            tok[b, r], par[b, r], sc[b, r] = t, b * k + j, s
            fin[b, r] = int(bool(finished is not None and finished[b, j]) or t == eos)
    return tok, par, sc, fin
