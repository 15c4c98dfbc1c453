"""Plain 64-bit forms of the rotary, slot-weight, eviction and token-score calls, with their tolerances.

Rotary, per element u c - v s (times the magnitude g): the fraction of a turn is rounded to fp32 (half a step of a number up to 1/2:
2^-26 turns, 2^-23.3 radians), cosine and sine are within 2^-22 of their own, g's product and the two products and their difference
round by 2^-24 each: in all at most 2^-21 of g (|u| + |v|), and half a step of the result's type.

Slot weights, per term w p: a score is off by e as in tests/paged_util.py, which moves p by a factor within exp(+-2 e) (numerator and
denominator); scale times log2 e is rounded, 2^-24 of the exponent |scale s| and of the maximum's, together 2^-22 (|scale s| + 1); 2^x
2^-21 in numerator and denominator, the sum over n slots n 2^-24, the quotient and the weight 2^-22; the sum over R rows of G heads
R G 2^-24 of its terms, and what the slot held before one rounding, 2^-24.

Token scores: let B = sum p |x - max| / T.  Exponents are off by 2^-23 of themselves (the factor log2 e / T, a difference and a
product), which moves the sum by at most B 2^-22 of it, 2^x by 2^-21, and additions by (V / 256 + 64) 2^-24 (a thread adds every 256th
logit, or fewer; then a few dozen joins): r in all.  ln of the sum is off by r, a log-probability by r and half a step.  The entropy is
ln s - w / s with w the sum of p (x - max): off by r (1 + B) + 2^-22 B + r, and half a step.
"""
import math

import numpy as np
import torch

from tests import paged_util as pg


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def turn(x, positions, freq, interleaved, magnitude):
    """x [...][heads][d], positions [...], freq float64 [half], all on the CPU.  Returns (y, tolerance without the last rounding)."""
    half = len(freq)
    x = x.double()
    f = torch.as_tensor(freq, dtype=torch.float64)
    # whole turns are taken off in whole numbers as far as they go: the product of a position and a frequency in 80 bits
    a = torch.from_numpy(np.remainder(positions.numpy().astype(np.longdouble)[..., None] * f.numpy().astype(np.longdouble),
                                      2 * np.arccos(np.longdouble(-1))).astype(np.float64))[..., None, :]
    c, s = a.cos() * magnitude, a.sin() * magnitude
    y, tol = x.clone(), torch.zeros_like(x)
    u, v = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., v] * c + x[..., u] * s
    t = (x[..., u].abs() + x[..., v].abs()) * abs(magnitude) * 2.0 ** -21
    # a frequency in turns is rounded to 64 bits as well
    t = t + (x[..., u].abs() + x[..., v].abs()) * abs(magnitude) * (positions.double().abs()[..., None, None] * f.abs() * 2.0 ** -52)
    tol[..., u] = t
    tol[..., v] = t
    return y, tol


def check_close(got, want, tol, dtype):
    got = got.cpu()
    bound = tol + want.abs() * half_step(dtype) * (1 + 2.0 ** -20) + 1e-38
    same = torch.isnan(want) & torch.isnan(got.double())
    err = (got.double() - want).abs()
    bad = ~(err <= bound) & ~same
    assert not bad.any(), (int(bad.sum()), float((err / bound)[~same].max()))


def frequencies(rot_dim, theta, scaling=None, factor=1.0, low=1.0, high=4.0, original_len=0.0):
    if scaling == "base":
        theta = theta * factor ** (rot_dim / (rot_dim - 2))
    f = [theta ** (-2 * i / rot_dim) for i in range(rot_dim // 2)]
    if scaling == "linear":
        return [x / factor for x in f]
    if scaling == "bands":
        out = []
        for x in f:
            wave = 2 * math.pi / x
            if wave < original_len / high:
                out.append(x)
            elif wave > original_len / low:
                out.append(x / factor)
            else:
                s = (original_len / wave - low) / (high - low)
                out.append((1 - s) * x / factor + s * x)
        return out
    if scaling == "ramp":
        at = [rot_dim * math.log(original_len / (n * 2 * math.pi)) / (2 * math.log(theta)) for n in (high, low)]
        a, b = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot_dim - 1)
        b = b if b > a else a + 0.001
        ramp = [min(1.0, max(0.0, (i - a) / (b - a))) for i in range(rot_dim // 2)]
        return [x / factor * r + x * (1 - r) for x, r in zip(f, ramp)]
    return f


def slot_weights(q, pages, tables, prefix, n_rows, anc, scale, weights, mass):
    """The weights of one layer: mass float64 [batch][kv heads][slots] before the call.  Returns (mass after it, tolerance)."""
    batch, rows, hq, d = q.shape
    hkv, page = pages.shape[2], pages.shape[3]
    g = hq // hkv
    out, tol = mass.double().clone(), torch.zeros_like(mass, dtype=torch.float64)
    for b in range(batch):
        p, n = int(prefix[b]), int(n_rows[b])
        if n == 0:
            continue
        new, err = torch.zeros(hkv, p + n, dtype=torch.float64), torch.zeros(hkv, p + n, dtype=torch.float64)
        for r in range(n):
            slots = [s for s in range(p + n) if (s < p or anc[b][r][s - p]) and 0 <= tables[b][s // page] < pages.shape[0]]
            if not slots:
                continue
            at = torch.tensor(slots)
            pgs = torch.tensor([int(tables[b][s // page]) for s in slots])
            k = pages[pgs, 0, :, at % page].double()                # [slots][heads][d]
            w = 1.0 if weights is None else float(weights[b, r])
            for h in range(hq):
                x = (k[:, h // g] @ q[b, r, h].double()) * scale
                e = (d + 8) * 2.0 ** -22 * abs(scale) * float((k[:, h // g].abs() @ q[b, r, h].double().abs()).max())
                share = torch.softmax(x, 0) * w
                new[h // g, at] += share
                rel = 2 * e + 2.0 ** -22 * (x.abs() + x.abs().max() + 1) + 2.0 ** -20 + 2 * len(slots) * 2.0 ** -24 + 2.0 ** -22
                err[h // g, at] += share.abs() * (rel + n * g * 2.0 ** -24)
        out[b, :, :p] += new[:, :p]
        out[b, :, p:p + n] = new[:, p:]
        tol[b, :, :p + n] = err + out[b, :, :p + n].abs() * 2.0 ** -23
    return out, tol


def chosen(mass, n, keep, first, recent):
    """The slots of one (layer, sequence, head) that stay, in order."""
    if n <= keep:
        return np.arange(n)
    x = np.where(np.isnan(mass[:n]), -np.inf, mass[:n]).astype(np.float64)
    nan = np.isnan(mass[:n])
    inner = np.arange(first, n - recent)
    best = inner[np.lexsort((inner, nan[inner], -x[inner]))][:keep - first - recent]
    return np.sort(np.concatenate([np.arange(first), best, np.arange(n - recent, n)])).astype(np.int64)


def evict(pages, mass, out_mass, tables, lens, keep, first, recent):
    """pages [layers][pages][2][heads][page][d], mass [layers][batch][heads][slots] on the CPU, in place of copies.  Returns (pages,
    out_mass, lengths)."""
    page = pages.shape[4]
    new_pages, new_mass, new_len = pages.clone(), out_mass.clone(), []
    layers, batch, heads = mass.shape[:3]
    for b in range(batch):
        t = torch.as_tensor(np.asarray(tables[b]).astype(np.int64))
        new_len.append(min(int(lens[b]), int(keep[b])))
        for la in range(layers):
            for h in range(heads):
                src = torch.from_numpy(chosen(mass[la, b, h].numpy(), int(lens[b]), int(keep[b]), first, recent))
                dst = torch.arange(len(src))
                new_pages[la, t[dst // page], :, h, dst % page] = pages[la, t[src // page], :, h, src % page]
                new_mass[la, b, h, :len(src)] = mass[la, b, h, src]
    return new_pages, new_mass, np.array(new_len, np.int32)


def scores(logits, tokens, token_rows, topk, temperature):
    """float64 logits [rows][vocab] on the CPU.  Returns a dict of (value, tolerance) or whole numbers."""
    rows, v = logits.shape
    temperature = float(np.float32(temperature))                      # (the call takes it in 32 bits: 0.2 is 1.5e-8 of itself off)
    x = torch.where(logits.abs() < math.inf, logits, torch.tensor(-math.inf, dtype=torch.float64))
    lse, ent = torch.full((rows,), -math.inf, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    r, b = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    top = torch.full((rows, topk), -1, dtype=torch.int32)
    top_logp = torch.full((rows, topk), -math.inf, dtype=torch.float64)
    logp_of = torch.full((rows, v), -math.inf, dtype=torch.float64)
    for i in range(rows):
        on = torch.isfinite(x[i])
        if not on.any():
            continue
        m = x[i].max()
        z = (x[i][on] - m) / temperature
        s = torch.exp(z).sum()
        p = torch.exp(z) / s
        b[i] = float((p * z.abs())[p > 0].sum())
        r[i] = b[i] * 2.0 ** -22 + 2.0 ** -21 + (v / 256 + 64) * 2.0 ** -24
        lse[i] = m / temperature + torch.log(s)
        ent[i] = torch.log(s) - float((p * z)[p > 0].sum())
        logp_of[i, on] = z - torch.log(s)
        order = np.lexsort((np.arange(v), -np.where(on.numpy(), x[i].numpy(), -np.inf)))[:topk]
        order = [int(t) for t in order if on[t]]
        top[i, :len(order)] = torch.tensor(order, dtype=torch.int32)
        top_logp[i, :len(order)] = logp_of[i, order]
    n = 0 if tokens is None else len(tokens)
    logp, tol = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    for i in range(n):
        row, t = (i if token_rows is None else int(token_rows[i])), int(tokens[i])
        if row < 0 or t < 0:
            continue
        logp[i] = logp_of[row, t] if row < rows and t < v else -math.inf
        tol[i] = r[row] if row < rows else 0.0
    return {"logp": (logp, tol), "lse": (lse, r), "entropy": (ent, r * (2 + b) + 2.0 ** -22 * b), "top_tokens": top,
            "top_logp": (top_logp, r[:, None].expand(rows, topk))}


def check_scores(got, want):
    assert torch.equal(got["top_tokens"].cpu(), want["top_tokens"])
    for key in ("logp", "lse", "entropy", "top_logp"):
        y, tol = want[key]
        g = got[key].cpu()
        inf = torch.isinf(y.float())                              # (a log-sum may pass fp32's range)
        assert torch.equal(g[inf], y[inf].float()), key
        check_close(g[~inf], y[~inf], tol[~inf], torch.float32)
    assert (got["logp"] <= 0).all() and (got["top_logp"] <= 0).all() and (got["entropy"] >= 0).all()


make_tables, tree_masks = pg.make_tables, pg.tree_masks
