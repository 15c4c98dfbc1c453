"""GPU tests of the rotary, slot-weight and eviction calls against their plain 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from tests import long_util as lu
from tests import paged_util as pg
from tests.test_gpu_paged import BF, F32, Case, cu, i32, lib

pytestmark = pytest.mark.gpu

BITS = {BF: torch.int16, F32: torch.int32}


def bits(t):
    """The same memory as whole numbers (NaN equals itself)."""
    return t.contiguous().view(BITS[t.dtype])


def graph_of(f):
    """f captured once, after a call on the capture's stream."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        f()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f()
    return g


# ------------------------------------------------------------------ rotary
@pytest.mark.parametrize("dtype,batch,rows,heads,d,rot,interleaved", [
    (F32, 1, 1, 1, 4, 2, False), (F32, 2, 3, 3, 32, 32, False), (F32, 1, 7, 5, 64, 24, False), (F32, 3, 2, 2, 64, 6, True),
    (F32, 1, 2, 40, 128, 128, True), (F32, 1, 3, 2, 100, 100, False), (BF, 1, 1, 32, 128, 128, False), (BF, 2, 61, 8, 128, 64, True),
    (BF, 3, 5, 7, 64, 64, False), (BF, 1, 9, 3, 64, 20, False), (BF, 1, 9, 3, 64, 20, True), (BF, 2, 2, 1, 8, 8, False),
    (BF, 1, 4, 6, 96, 48, False), (BF, 1, 3, 2, 1024, 512, False), (BF, 1, 300, 2, 32, 16, False), (F32, 1, 1, 129, 128, 64, False),
])
def test_rotary_matches_the_plain_form(dtype, batch, rows, heads, d, rot, interleaved):
    gen = torch.Generator().manual_seed(d + rot)
    x = torch.randn(batch, rows, heads, d, generator=gen).to(dtype)
    at = torch.randint(0, 1 << 20, (batch, rows), generator=gen, dtype=torch.int32)
    at.view(-1)[0] = 0
    f = torch.tensor(lu.frequencies(rot, 10000.0), dtype=torch.float64)
    want, tol = lu.turn(x, at, f, interleaved, 1.25)
    got = lib().poss_rotary(x.cuda(), at.cuda(), f.cuda(), interleaved=interleaved, magnitude=1.25)
    lu.check_close(got, want, tol, dtype)
    assert torch.equal(bits(got.cpu()[..., rot:]), bits(x[..., rot:]))        # what does not turn stays as it is
    y = x.cuda()
    assert lib().poss_rotary(y, at.cuda(), f.cuda(), out=y, interleaved=interleaved, magnitude=1.25) is y
    assert torch.equal(bits(y), bits(got))                                    # in place the same bits


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_far_and_negative_positions(dtype, interleaved):
    at = torch.tensor([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1000003, 16777217, -131071]], dtype=torch.int32)
    x = torch.randn(1, 8, 2, 64, generator=torch.Generator().manual_seed(1)).to(dtype)
    f = torch.tensor([1.0, 6.28, 0.5, 3.0] + lu.frequencies(56, 1e6), dtype=torch.float64)
    want, tol = lu.turn(x, at, f, interleaved, 1.0)
    got = lib().poss_rotary(x.cuda(), at.cuda(), f.cuda(), interleaved=interleaved)
    lu.check_close(got, want, tol, dtype)
    back = lib().poss_rotary(got.float(), (-at).cuda(), f.cuda(), interleaved=interleaved)
    # turned back from what was rounded: both roundings and both angles' errors
    keep = [i for i in range(8) if int(at[0, i]) != -2 ** 31]
    err = (back.cpu().double() - x.double()).abs()[0, keep]
    assert float(err.max()) <= float(x.double().abs().max()) * (2 * lu.half_step(dtype) + 2.0 ** -18)


def test_rotary_of_strided_rows_special_values_and_streams():
    gen = torch.Generator().manual_seed(2)
    f = torch.tensor(lu.frequencies(64, 10000.0), dtype=torch.float64)
    whole = torch.randn(2, 5, 12, 64, generator=gen).to(BF)                  # a fused projection: 8 query heads, 2 of keys, 2 of values
    whole[0, 0, 0, 3] = math.nan
    whole[0, 1, 0, 3] = math.inf
    at = torch.arange(10, dtype=torch.int32).view(2, 5) * 999
    x = whole[:, :, :8]
    want, tol = lu.turn(x, at, f, False, 1.0)
    w = whole.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = lib().poss_rotary(w[:, :, :8], at.cuda(), f.cuda())
        lib().poss_rotary(w[:, :, 8:10], at.cuda(), f.cuda(), out=w[:, :, 8:10])
    s.synchronize()
    g = got.cpu()
    odd = torch.zeros_like(g, dtype=torch.bool)
    odd[0, :2, 0, 3] = odd[0, :2, 0, 35] = True
    assert not torch.isfinite(g[0, :2, 0, 3]).any() and torch.isfinite(g[~odd]).all()   # a pair's NaN or infinity stays in its pair
    lu.check_close(g[~odd], want[~odd], tol[~odd], BF)
    wk, tk = lu.turn(whole[:, :, 8:10], at, f, False, 1.0)
    lu.check_close(w[:, :, 8:10], wk, tk, BF)
    assert torch.equal(bits(w[:, :, 10:].cpu()), bits(whole[:, :, 10:])) and torch.equal(bits(w[:, :, :8].cpu()), bits(whole[:, :, :8]))
    out = torch.full((2, 5, 20, 64), 3.0, dtype=BF, device="cuda")           # a target whose rows lie apart
    lib().poss_rotary(w[:, :, :8], at.cuda(), f.cuda(), out=out[:, :, 4:12])
    assert torch.equal(bits(out[:, :, 4:12].cpu()), bits(g)) and (out[:, :, 12:] == 3).all() and (out[:, :, :4] == 3).all()
    empty = torch.zeros(0, 5, 8, 64, device="cuda")
    assert lib().poss_rotary(empty, torch.zeros(0, 5, dtype=torch.int32, device="cuda"), f.cuda()).shape == empty.shape


@pytest.mark.parametrize("dtype,hq,hkv,d,page,prefix,rows,n_rows,rot,interleaved,own_positions", [
    (F32, 4, 4, 64, 24, [0, 5, 131], 1, None, 64, False, False),
    (F32, 6, 2, 32, 8, [37, 0, 200], 14, [14, 1, 0], 6, False, True),
    (F32, 0, 3, 128, 1, [9, 40], 7, None, 128, True, False),
    (BF, 32, 8, 128, 16, [1023], 1, None, 128, False, True),
    (BF, 32, 8, 128, 64, [63, 100, 0], 61, [61, 0, 13], 64, True, True),
    (BF, 8, 2, 64, 16, [0, 300], 200, [200, 77], 20, False, False),
    (BF, 3, 1, 32, 1024, [1020], 40, None, 32, True, True),
])
def test_append_rotary_matches_the_plain_form(dtype, hq, hkv, d, page, prefix, rows, n_rows, rot, interleaved, own_positions):
    rng, gen = np.random.default_rng(3), torch.Generator().manual_seed(3)
    b = len(prefix)
    n_rows = n_rows or [rows] * b
    held = [p + n for p, n in zip(prefix, n_rows)]
    n_pages = sum(-(-n // page) for n in held) + 2
    tables = lu.make_tables(rng, held, page, n_pages, max(-(-(p + rows) // page) for p in prefix))
    qkv = torch.randn(b, rows, hq + 2 * hkv, d, generator=gen).to(dtype)
    pages = torch.randn(2, n_pages, 2, hkv, page, d, generator=gen).to(dtype)
    at = torch.randint(0, 1 << 20, (b, rows), generator=gen, dtype=torch.int32)
    f = torch.tensor(lu.frequencies(rot, 10000.0), dtype=torch.float64)
    used = at if own_positions else torch.tensor(prefix, dtype=torch.int32)[:, None] + torch.arange(rows, dtype=torch.int32)
    want, tol = lu.turn(qkv, used, f, interleaved, 0.9)
    g, gp, status = qkv.cuda(), pages.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    q, k, v = (g[:, :, :hq], g[:, :, hq:hq + hkv], g[:, :, hq + hkv:])
    args = (k, v, gp, 1, cu(tables), i32(prefix), f.cuda())
    kw = {"positions": at.cuda() if own_positions else None, "interleaved": interleaved, "magnitude": 0.9, "n_rows": i32(n_rows),
          "status": status}
    fill = torch.full((b, rows, hq, d), 7.5, dtype=dtype, device="cuda")
    out = lib().poss_pages_append_rotary(*args, q=q if hq else None, out_q=fill.clone() if hq else None, **kw)
    assert int(status) == 0
    expect, where = pages.clone(), torch.zeros(pages.shape, dtype=torch.bool)
    full, ftol = pages.double(), torch.zeros(pages.shape, dtype=torch.float64)
    for i in range(b):
        for r in range(n_rows[i]):
            s = prefix[i] + r
            p = int(tables[i][s // page])
            full[1, p, 0, :, s % page] = want[i, r, hq:hq + hkv]
            ftol[1, p, 0, :, s % page] = tol[i, r, hq:hq + hkv]
            where[1, p, 0, :, s % page] = True
            expect[1, p, 1, :, s % page] = qkv[i, r, hq + hkv:]
        if hq:
            m = n_rows[i]
            lu.check_close(out[i, :m], want[i, :m, :hq], tol[i, :m, :hq], dtype)
            assert torch.equal(out[i, m:], fill[i, m:])
    lu.check_close(gp.cpu()[where], full[where], ftol[where], dtype)
    assert torch.equal(bits(gp.cpu()[~where]), bits(expect[~where]))
    # queries in place, between the keys and values of the same projection: the same bits
    if hq:
        lib().poss_pages_append_rotary(*args, q=q, out_q=q, **kw)
        for i in range(b):
            assert torch.equal(bits(q[i, :n_rows[i]]), bits(out[i, :n_rows[i]]))
            assert torch.equal(bits(g[i, :, hq:].cpu()), bits(qkv[i, :, hq:]))


def test_append_rotary_bad_sequences_and_pages_and_replay():
    hq, hkv, d, page, rows = 4, 2, 64, 16, 3
    gen = torch.Generator().manual_seed(4)
    f = torch.tensor(lu.frequencies(64, 10000.0), dtype=torch.float64).cuda()
    q, k, v = (torch.randn(5, rows, h, d, generator=gen).to(BF).cuda() for h in (hq, hkv, hkv))
    pages = torch.zeros(1, 8, 2, hkv, page, d, dtype=BF, device="cuda")
    tables = i32([[0, 1], [2, -1], [3, 99], [4, 5], [6, 7]])
    prefix, n_rows = i32([-1, 15, 16, 30, 4]), i32([3, 3, 3, 3, 4])   # below 0, second page gone, none such, too long, too many rows
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 2.0)
    kw = {"q": q, "out_q": out, "n_rows": n_rows, "status": status}
    lib().poss_pages_append_rotary(k, v, pages, 0, tables, prefix, f, **kw)
    assert int(status) == 1
    assert (out[[0, 3, 4]] == 2).all()                                # sequences with lengths out of range have no rows
    assert (out[[1, 2]] != 2).any(-1).all()                           # a missing page keeps no query from turning
    live = pages.abs().sum((0, 2, 3, 5)).nonzero().tolist()
    assert live == [[2, 15]]                                          # the one row whose page is there
    # a captured call goes by the lengths of its replay
    tables.copy_(i32([[0, 1], [2, 3], [4, 5], [6, 7], [-1, -1]]))
    status.zero_()
    prefix.copy_(i32([0, 15, 16, 20, 0]))
    n_rows.copy_(i32([3, 3, 3, 3, 0]))
    g = graph_of(lambda: lib().poss_pages_append_rotary(k, v, pages, 0, tables, prefix, f, **kw))
    prefix.copy_(i32([7, 1, 29, 0, 0]))
    pages.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert int(status) == 0
    again = torch.zeros_like(pages)
    o2 = lib().poss_pages_append_rotary(k, v, again, 0, tables, prefix, f, q=q, n_rows=n_rows)
    assert torch.equal(again, pages) and torch.equal(o2[:4], out[:4])


# ------------------------------------------------------------------ slot weights
def mass_case(c, seed=0, weighted=True, layers=None):
    """Weights before the call, and the rows' own."""
    gen = torch.Generator().manual_seed(seed)
    hkv = c.pages.shape[3]
    slots = c.tables.shape[1] * c.page
    mass = torch.rand(c.pages.shape[0], c.b, hkv, slots, generator=gen) * 0.1
    w = torch.rand(c.b, c.rows, generator=gen) if weighted else None
    return mass, w


def run_mass(c, mass, weights, pages=None, out=None, n_rows=None, prefix=None, tables=None, q=None, **kw):
    c.gpu_status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = lib().poss_paged_tree_attention_mass(
        c.q.cuda() if q is None else q, c.pages.cuda() if pages is None else pages, mass, c.layer, cu(c.tables if tables is None else tables),
        i32(c.prefix if prefix is None else prefix), cu(c.mask), c.scale, n_rows=i32(c.n_rows if n_rows is None else n_rows),
        row_weights=None if weights is None else weights.cuda(), out=out, status=c.gpu_status, **kw)
    torch.cuda.synchronize()
    return r


def check_mass(c, got, mass, weights):
    want, tol = lu.slot_weights(c.q, c.pages[c.layer], c.tables, c.prefix, c.n_rows, c.anc, c.scale, weights, mass[c.layer])
    lu.check_close(got[c.layer], want, tol, F32)
    others = [i for i in range(mass.shape[0]) if i != c.layer]
    assert torch.equal(got[others].cpu(), mass[others])
    for b in range(c.b):                                              # what lies behind the rows, and sequences without rows
        end = c.prefix[b] + c.n_rows[b] if c.n_rows[b] else 0
        assert torch.equal(got[c.layer, b, :, end:].cpu(), mass[c.layer, b, :, end:])


SHAPES = [
    (F32, 4, 4, 64, 24, [0, 5, 131], 1, None),
    (F32, 6, 2, 32, 16, [37, 0, 200, 63], 14, [14, 1, 0, 9]),
    (F32, 8, 1, 128, 8, [300, 17], 61, [61, 33]),
    (F32, 4, 2, 64, 1, [9, 40], 7, None),
    (BF, 6, 2, 32, 16, [100, 3], 14, None),                           # bf16 off the tensor cores
    (BF, 8, 2, 64, 24, [100, 3], 25, [25, 2]),
    (BF, 32, 8, 128, 16, [0], 1, None),                               # one token that sees itself alone
    (BF, 32, 8, 128, 16, [127, 128, 126, 255, 63, 64], 1, None),      # around the key tiles
    (BF, 32, 8, 128, 16, [127, 1, 250], 3, [3, 2, 3]),
    (BF, 8, 2, 64, 32, [300, 0, 17, 129, 64, 5, 255], 25, [25, 1, 24, 0, 13, 25, 7]),
    (BF, 32, 8, 128, 64, [700, 31], 61, [61, 60]),
    (BF, 8, 1, 128, 128, [513], 16, None),
    (BF, 8, 1, 128, 256, [513, 1000], 17, [17, 16]),
    (BF, 4, 1, 64, 256, [257], 128, None),                            # 512 query rows, two mask words
    (BF, 5, 1, 128, 32, [70, 0], 128, [128, 77]),                     # five heads to a key head
    (BF, 6, 2, 64, 16, [400], 65, None),
    (BF, 40, 40, 128, 16, [200], 2, None),                            # multi-head
    (BF, 2, 1, 128, 16, [5000], 2, None),                             # a long context in many pages
    (BF, 130, 1, 64, 16, [90], 2, None),                              # more heads to a key head than a slot of rows
    (BF, 128, 1, 64, 64, [90, 300], 3, [3, 2]),
    (BF, 16, 1, 128, 16, [40, 700, 3], 1, None),
    (BF, 17, 1, 128, 16, [40, 700, 3], 1, [1, 1, 0]),
]


@pytest.mark.parametrize("dtype,hq,hkv,d,page,prefix,rows,n_rows", SHAPES)
def test_slot_weights_match_the_plain_form(dtype, hq, hkv, d, page, prefix, rows, n_rows):
    c = Case(21, dtype, hq, hkv, d, page, prefix, rows, n_rows, layers=2, layer=1)
    for weighted in (True, False):
        mass, w = mass_case(c, 1, weighted)
        got = mass.cuda()
        fill = torch.full((c.b, rows, hq, d), 7.5, dtype=dtype, device="cuda")
        out = run_mass(c, got, w, out=fill.clone())
        assert int(c.gpu_status) == 0
        check_mass(c, got, mass, w)
        assert torch.equal(bits(out), bits(c.run(out=fill.clone())))  # the attention is the attention
        again = mass.cuda()
        run_mass(c, again, w, out=fill.clone())
        assert torch.equal(bits(again), bits(got))                    # equal calls, equal bits


@pytest.mark.parametrize("dtype,hq,hkv,d,page", [(F32, 4, 2, 64, 24), (BF, 8, 2, 64, 16), (BF, 4, 1, 128, 16), (BF, 32, 2, 128, 64)])
@pytest.mark.parametrize("rows,prefix", [(1, [3, 125, 64]), (5, [3, 125, 0]), (61, [120, 64, 0]), (128, [1, 200, 63])])
def test_unseen_slots_draw_nothing_whatever_they_hold(dtype, hq, hkv, d, page, rows, prefix):
    """Infinities and NaN behind the last slot, in pages that nobody holds and in the keys and values of tree slots that most rows do not
    see; a missing page's slots draw nothing and give the rest its share."""
    n_rows = [rows, max(1, rows - 1), rows]
    anc = np.eye(rows, dtype=bool)
    anc[:, 0] = True                                                  # all rows see the root and themselves
    if rows > 4:
        anc[3] = False                                                # and one row of a committed context sees that alone
    c = Case(31, dtype, hq, hkv, d, page, prefix, rows, n_rows, anc=anc)
    c.tables[1, 1 if page < 100 else 0] = -1
    held = {int(p) for t in c.tables for p in t if p >= 0}
    for p in range(c.pages.shape[1]):
        if p not in held:
            c.pages[0, p] = math.nan
    for b in range(c.b):
        end = c.prefix[b] + c.n_rows[b]
        for s in range(end, -(-end // page) * page):
            if c.tables[b, s // page] >= 0:
                c.pages[0, int(c.tables[b, s // page]), :, :, s % page] = [math.nan, math.inf, -math.inf][s % 3]
    mass, w = mass_case(c, 2)
    got = mass.cuda()
    run_mass(c, got, w)
    assert int(c.gpu_status) == 1                                     # the missing page
    check_mass(c, got, mass, w)
    if rows > 4:
        # a tree slot that only its own row sees: NaN for that row's terms, the others' are as before
        s = c.prefix[0] + 4
        c.pages[0, int(c.tables[0, s // page]), 0, :, s % page, 1] = math.nan
        bad = mass.cuda()
        run_mass(c, bad, w)
        x, y = bad[0].cpu(), got[0].cpu()
        seen_by_4 = list(range(c.prefix[0])) + [c.prefix[0], s]
        rest = [i for i in range(c.prefix[0] + rows) if i not in seen_by_4]
        assert torch.isnan(x[0][:, [s]]).all() and torch.equal(x[0][:, rest], y[0][:, rest]) and torch.equal(x[1:], y[1:])


def test_slot_weights_extreme_scores_and_negative_scale():
    """Scores far apart (2^x under- and overflows unless the maximum is taken off), a negative scale, a row weight of 0, an infinite one."""
    for dtype, d, scale in [(F32, 64, 40.0), (BF, 64, 40.0), (BF, 128, 40.0), (BF, 64, -0.3), (F32, 32, -0.3), (BF, 64, 0.0)]:
        c = Case(41, dtype, 8, 2, d, 16, [200, 77], 9, [9, 4])
        c.scale = scale
        mass, w = mass_case(c, 3)
        w[0, 2] = 0.0
        got = mass.cuda()
        run_mass(c, got, w)
        check_mass(c, got, mass, w)
    w[0, 1] = math.inf
    got = mass.cuda()
    run_mass(c, got, w)
    assert torch.isinf(got[0, 0]).any() and torch.isfinite(got[0, 1]).all()


def test_slot_weights_replayed_on_other_lengths_two_streams_and_shared_scratch():
    c = Case(51, BF, 32, 8, 128, 16, [300, 40, 800], 7, [7, 2, 5])
    mass, w = mass_case(c, 4)
    q, pages, tables, mask, wg = c.q.cuda(), c.pages.cuda(), cu(c.tables), cu(c.mask), w.cuda()
    prefix, n_rows = i32([1, 1, 1]), i32([1, 1, 1])
    ws = torch.empty(lib().poss_paged_attention_mass_workspace_bytes(pages, 3, 7, 32, tables.shape[1]), dtype=torch.uint8, device="cuda")
    got, other = mass.cuda(), mass.cuda()

    def call(m):
        return lib().poss_paged_tree_attention_mass(q, pages, m, 0, tables, prefix, mask, c.scale, n_rows=n_rows, row_weights=wg,
                                                    workspace=ws)
    one, two = graph_of(lambda: call(got)), graph_of(lambda: call(other))
    prefix.copy_(i32(c.prefix))
    n_rows.copy_(i32(c.n_rows))
    got.copy_(mass)
    other.copy_(mass)
    ws.fill_(255)                                                     # scratch needs no initial value
    one.replay()
    two.replay()                                                      # in one stream both may use one scratch
    torch.cuda.synchronize()
    check_mass(c, got, mass, w)
    assert torch.equal(got, other)
    a, b = mass.cuda(), mass.cuda()                                   # two calls at once, scratch of their own
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for s, m in ((s1, a), (s2, b)):
        with torch.cuda.stream(s):
            lib().poss_paged_tree_attention_mass(q, pages, m, 0, tables, prefix, mask, c.scale, n_rows=n_rows, row_weights=wg)
    torch.cuda.synchronize()
    assert torch.equal(a, got) and torch.equal(b, got)


def test_slot_weights_of_bad_sequences():
    c = Case(61, BF, 8, 2, 64, 16, [100, 50, 20], 3)
    mass, w = mass_case(c, 5)
    got = mass.cuda()
    fill = torch.full((3, 3, 8, 64), 7.5, dtype=BF, device="cuda")
    out = run_mass(c, got, w, prefix=[-1, 50, 1 << 20], n_rows=[3, 4, 3], out=fill.clone())
    assert int(c.gpu_status) == 1 and torch.equal(out, fill) and torch.equal(got.cpu(), mass)
    run_mass(c, got, w, n_rows=[0, 0, 0])
    assert torch.equal(got.cpu(), mass)
    none = torch.zeros(1, 0, 2, 64, device="cuda")
    e = lib().poss_paged_tree_attention_mass(torch.zeros(0, 3, 8, 64, dtype=BF, device="cuda"), c.pages.cuda(), none, 0,
                                             torch.zeros(0, 4, dtype=torch.int32, device="cuda"), i32([]),
                                             torch.zeros(0, 3, 1, dtype=torch.int64, device="cuda"), 0.1)
    assert e.shape == (0, 3, 8, 64)


# ------------------------------------------------------------------ eviction
def evict_case(seed, dtype, layers, hkv, d, page, lens, kind):
    rng, gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    n_pages = sum(-(-n // page) for n in lens) + 3
    mp = max(-(-n // page) for n in lens) + 1
    tables = lu.make_tables(rng, lens, page, n_pages, mp)
    pages = torch.randn(layers, n_pages, 2, hkv, page, d, generator=gen).to(dtype)
    shape = (layers, len(lens), hkv, mp * page + 5)
    mass = torch.rand(shape, generator=gen)
    if kind == "ties":
        mass = (mass * 4).floor()
    elif kind == "equal":
        mass.fill_(0.25)
    elif kind == "odd":                                               # signed zeros, infinities, NaN, denormals, negative ones
        pick = torch.randint(0, 9, shape, generator=gen)
        for i, x in enumerate([0.0, -0.0, math.inf, -math.inf, math.nan, 1e-42, -1e-42, -3.0]):
            mass[pick == i] = x
    elif kind == "rising":
        mass = torch.arange(shape[-1], dtype=torch.float32).expand(shape).contiguous()
    elif kind == "falling":
        mass = -torch.arange(shape[-1], dtype=torch.float32).expand(shape).contiguous()
    elif kind == "close":                                             # they differ in the last bits alone
        mass = (torch.randint(0, 2000, shape, generator=gen, dtype=torch.int32) + 0x3f800000).view(torch.float32)
    return pages, mass, tables


@pytest.mark.parametrize("dtype,layers,hkv,d,page,lens,keep,first,recent", [
    (F32, 1, 1, 32, 1, [5], [2], 0, 0),
    (F32, 2, 4, 64, 24, [700, 10, 0, 301, 302], [301] * 5, 4, 8),
    (F32, 1, 3, 128, 1024, [1500], [700], 0, 64),
    (BF, 1, 2, 32, 16, [600, 513, 512, 511, 1], [300, 512, 511, 0, 0], 0, 0),
    (BF, 3, 2, 64, 8, [100, 99, 98], [12, 98, 97], 4, 8),
    (BF, 2, 8, 128, 16, [1025, 300], [128, 299], 1, 0),
    (BF, 1, 1, 128, 64, [9000], [4000], 4, 100),
    (BF, 1, 2, 64, 16, [40, 40], [40, 12], 12, 0),                    # the first ones are all that stays
    (BF, 1, 2, 64, 16, [40, 40], [39, 12], 0, 12),                    # the last ones are
])
@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd", "rising", "falling", "close"])
def test_eviction_matches_the_plain_form(dtype, layers, hkv, d, page, lens, keep, first, recent, kind):
    pages, mass, tables = evict_case(7, dtype, layers, hkv, d, page, lens, kind)
    if kind == "odd":
        pages.view(-1)[::7] = math.nan                                # moved like everything else
    start = torch.rand(mass.shape, generator=torch.Generator().manual_seed(1))
    for apart in (True, False):
        want_pages, want_mass, want_len = lu.evict(pages, mass, start if apart else mass, tables, lens, keep, first, recent)
        gp, gm = pages.cuda(), mass.cuda()
        to = start.cuda() if apart else None
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        n = lib().poss_pages_evict(gp, gm, cu(tables), i32(lens), i32(keep), first=first, recent=recent, out_mass=to, status=status)
        assert int(status) == 0 and n.cpu().tolist() == want_len.tolist()
        assert torch.equal(bits(gp.cpu()), bits(want_pages))          # every slot of the pool, those behind the kept ones too
        assert torch.equal(bits((to if apart else gm).cpu()), bits(want_mass))
        if apart:
            assert torch.equal(bits(gm.cpu()), bits(mass))


def test_eviction_of_bad_sequences_leaves_them_as_they_were():
    lens = [100, 100, 100, 100, 100, 100]
    pages, mass, tables = evict_case(8, BF, 2, 2, 64, 16, lens, "random")
    tables[3, 2] = -1                                                 # a page that it needs is gone
    tables[4, 6] = pages.shape[1] + 7
    lens[0], lens[1] = -1, tables.shape[1] * 16 + 1
    keep = [50, 50, 9, 50, 50, 50]                                    # 9: fewer than must stay
    gp, to, status = pages.cuda(), torch.full(mass.shape, 9.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    n = lib().poss_pages_evict(gp, mass.cuda(), cu(tables), i32(lens), i32(keep), first=4, recent=6, out_mass=to, status=status)
    assert int(status) == 1 and n.cpu().tolist() == lens[:5] + [50]
    ok = lu.evict(pages[:, :], mass[:, 5:], torch.full(mass[:, 5:].shape, 9.0), tables[5:], lens[5:], keep[5:], 4, 6)
    assert torch.equal(gp.cpu(), ok[0]) and torch.equal(to[:, 5:].cpu(), ok[1]) and (to[:, :5] == 9).all()


def test_eviction_replayed_and_with_shared_scratch():
    lens = [300, 200]
    pages, mass, tables = evict_case(9, BF, 2, 2, 64, 16, lens, "random")
    gp, gm, t = pages.cuda(), mass.cuda(), cu(tables)
    n0, keep = i32([20, 20]), i32([20, 20])
    ws = torch.empty(lib().poss_pages_evict_workspace_bytes(gp, 2, t.shape[1]), dtype=torch.uint8, device="cuda")
    out = torch.zeros(2, dtype=torch.int32, device="cuda")
    g = graph_of(lambda: lib().poss_pages_evict(gp, gm, t, n0, keep, first=1, recent=2, out_len=out, workspace=ws))
    assert torch.equal(gp.cpu(), pages)
    n0.copy_(i32(lens))
    keep.copy_(i32([100, 199]))
    ws.fill_(255)
    g.replay()
    torch.cuda.synchronize()
    want = lu.evict(pages, mass, mass, tables, lens, [100, 199], 1, 2)
    assert torch.equal(gp.cpu(), want[0]) and torch.equal(gm.cpu(), want[1]) and out.cpu().tolist() == [100, 199]


def test_commit_takes_the_weights_along():
    c = Case(71, F32, 4, 2, 32, 16, [100, 30, 7], 9)
    mass, _ = mass_case(c, 6)
    path = np.zeros((3, 17), np.int32)
    path[0, 1:4] = [2, 5, 8]
    path[1, 1:3] = [1, 2]
    path[2, 1:3] = [5, 3]                                             # out of order: nothing moves
    acc = [3, 2, 2]
    a, b, gm = c.pages.cuda(), c.pages.cuda(), mass.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    n1 = lib().poss_pages_compact(a, cu(c.tables), i32(c.prefix), cu(path), i32(acc))
    n2 = lib().poss_pages_compact(b, cu(c.tables), i32(c.prefix), cu(path), i32(acc), mass=gm, status=status)
    assert torch.equal(a, b) and torch.equal(n1, n2) and int(status) == 1
    want = mass.clone()
    for i in (0, 1):
        for k in range(1, acc[i] + 1):
            want[:, i, :, c.prefix[i] + k] = mass[:, i, :, c.prefix[i] + int(path[i, k])]
    assert torch.equal(gm.cpu(), want)


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,hq,hkv,d,page", [(F32, 4, 2, 64, 24), (BF, 8, 2, 128, 16)])
def test_rounds_of_a_cache_that_is_kept_short(dtype, hq, hkv, d, page):
    """Two sequences over two layers: a tree's rows are turned and written, attend, their weights add up; the accepted path is committed;
    what exceeds the budget goes; surplus pages go back.  Positions run on.  Every call is held to its plain form on the state that the
    calls before have left."""
    rng, gen = np.random.default_rng(5), torch.Generator().manual_seed(5)
    b, rows, layers, budget, first, recent = 2, 6, 2, 24, 2, 8
    f = lib().poss_rotary_frequencies(d // 2, 10000.0, "bands", factor=4.0, original_len=64.0)
    n_pages, mp = 24, -(-(budget + 3 * rows) // page) + 1
    pages = torch.zeros(layers, n_pages, 2, hkv, page, d, dtype=dtype, device="cuda")
    mass = torch.zeros(layers, b, hkv, mp * page, device="cuda")
    tables, refs = torch.full((b, mp), -1, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    lens, at = i32([0, 0]), [1000, 70000]                             # slots held; the next row's position
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    evicted = 0
    for step in range(14):
        t = lib().poss_pages_remap(pages, tables, lens, refs, room=i32([rows, rows]), status=status)
        tables, refs = t["tables"], t["refs"]
        assert int(t["n_free"]) >= 0
        prefix = lens.clone()
        mask, anc = lu.tree_masks(rng, b, rows)
        depth = anc.sum(-1) - 1
        pos = torch.tensor([[at[i] + int(depth[i, r]) for r in range(rows)] for i in range(b)], dtype=torch.int32)
        for layer in range(layers):
            qkv = torch.randn(b, rows, hq + 2 * hkv, d, generator=gen).to(dtype)
            g = qkv.cuda()
            q = lib().poss_pages_append_rotary(g[:, :, hq:hq + hkv], g[:, :, hq + hkv:], pages, layer, tables, prefix, f, positions=pos.cuda(),
                                               q=g[:, :, :hq], interleaved=True, status=status)
            want_q, tol_q = lu.turn(qkv[:, :, :hq], pos, f.cpu(), True, 1.0)
            lu.check_close(q, want_q, tol_q, dtype)
            before, w = mass.cpu(), torch.rand(b, rows, generator=gen)
            out = lib().poss_paged_tree_attention_mass(q, pages, mass, layer, tables, prefix, cu(mask), d ** -0.5, row_weights=w.cuda(),
                                                       status=status)
            p, n = prefix.cpu().tolist(), [rows] * b
            want, tol = lu.slot_weights(q.cpu(), pages[layer].cpu(), tables.cpu().numpy(), p, n, anc, d ** -0.5, w, before[layer])
            lu.check_close(mass[layer], want, tol, F32)
            pg.check_attention(out, *pg.attention(q.cpu(), pages[layer].cpu(), tables.cpu().numpy(), p, n, anc, d ** -0.5), dtype,
                               dtype == BF)
        path = np.zeros((b, 17), np.int32)
        acc = []
        for i in range(b):                                            # the longest path of the tree
            r = int(depth[i].argmax())
            nodes = [j for j in range(rows) if anc[i, r, j]]
            path[i, :len(nodes)] = nodes
            acc.append(len(nodes) - 1)
            at[i] += len(nodes)
        lens = lib().poss_pages_compact(pages, tables, prefix, cu(path), i32(acc), mass=mass, status=status)
        p0, m0, l0, tab = pages.cpu(), mass.cpu(), lens.cpu().tolist(), tables.cpu().numpy()
        lens = lib().poss_pages_evict(pages, mass, tables, lens, i32([budget, budget + 3]), first=first, recent=recent, status=status)
        want = lu.evict(p0, m0, m0, tab, l0, [budget, budget + 3], first, recent)
        assert torch.equal(pages.cpu(), want[0]) and torch.equal(mass.cpu(), want[1]) and lens.cpu().tolist() == want[2].tolist()
        evicted += sum(l0) - int(lens.sum())
    assert evicted > 10 and int(status) == 0


def test_offsets_beyond_32_bits():
    """A pool of 2^32 bytes a layer and more: pages at its far end are written, read and moved like near ones."""
    hq, hkv, d, page, layers = 2, 1, 128, 256, 2
    n_pages = 33200                                                   # 33200 x 2 x 256 x 128 x 2 bytes = 4.35 GB a layer
    pages = torch.empty(layers, n_pages, 2, hkv, page, d, dtype=BF, device="cuda")
    gen = torch.Generator().manual_seed(6)
    tables = np.array([[n_pages - 1, n_pages - 5, 3, n_pages - 2, n_pages - 9]], np.int32)
    near = torch.randn(1, 5, 2, hkv, page, d, generator=gen).to(BF)
    for i, p in enumerate(tables[0]):
        pages[1, int(p)] = near[0, i].cuda()
    small, t2 = near.cuda(), i32([[0, 1, 2, 3, 4]])
    kv = torch.randn(1, 3, 2, d, generator=gen).to(BF).cuda()
    f = lib().poss_rotary_frequencies(128, 10000.0)
    prefix, q = i32([1100]), torch.randn(1, 3, hq, d, generator=gen).to(BF).cuda()
    mask = cu(pg.pack(np.tril(np.ones((1, 3, 3), bool))))
    res = []
    for pool, layer, t in ((pages, 1, i32(tables)), (small, 0, t2)):
        nl = pool.shape[0]
        mass = torch.zeros(nl, 1, hkv, 5 * page, device="cuda")
        lib().poss_pages_append_rotary(kv[:, :, :1], kv[:, :, 1:], pool, layer, t, prefix, f)
        out = lib().poss_paged_tree_attention_mass(q, pool, mass, layer, t, prefix, mask, 0.1)
        if nl == 2:
            mass[0] = mass[1]
            lib().poss_pages_evict(pool, mass, t, i32([1103]), i32([200]), first=1, recent=1)
        else:
            lib().poss_pages_evict(pool, mass, t, i32([1103]), i32([200]), first=1, recent=1)
        res.append((out, mass[layer], pool[layer, t[0].long()]))
    for x, y in zip(*res):
        assert torch.equal(x, y)


def test_tensors_that_are_not_as_wanted_are_named():
    c = Case(81, BF, 8, 2, 64, 16, [40, 20], 3)
    q, pages, tables, mask = c.q.cuda(), c.pages.cuda(), cu(c.tables), cu(c.mask)
    prefix, mass = i32(c.prefix), torch.zeros(1, 2, 2, tables.shape[1] * 16, device="cuda")
    f = lib().poss_rotary_frequencies(64, 1e4)
    at = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    k = torch.zeros(2, 3, 2, 64, dtype=BF, device="cuda")
    p = lib()
    bad = [
        (lambda: p.poss_rotary(q.cpu(), at, f), "x"), (lambda: p.poss_rotary(q, at.long(), f), "positions"),
        (lambda: p.poss_rotary(q, at, f.float()), "freq"), (lambda: p.poss_rotary(q[0], at, f), "x"),
        (lambda: p.poss_rotary(q.half(), at, f), "x"), (lambda: p.poss_rotary(q, at, f, out=k), "out"),
        (lambda: p.poss_rotary(q.transpose(1, 2), at, f), "x|positions"),
        (lambda: p.poss_pages_append_rotary(k, k[:, :2], pages, 0, tables, prefix, f), "^v: "),
        (lambda: p.poss_pages_append_rotary(k, k, pages, 0, tables, prefix, f, out_q=q), "out_q"),
        (lambda: p.poss_pages_append_rotary(k, k, pages, 0, tables, prefix, f, q=q[:1]), "q"),
        (lambda: p.poss_paged_tree_attention_mass(q, pages, mass.double(), 0, tables, prefix, mask, 0.1), "mass"),
        (lambda: p.poss_paged_tree_attention_mass(q, pages, mass[:, :1], 0, tables, prefix, mask, 0.1), "mass"),
        (lambda: p.poss_paged_tree_attention_mass(q, pages, mass, 0, tables, prefix, mask, 0.1, row_weights=at.float()[:1]), "row_weights"),
        (lambda: p.poss_pages_evict(pages, mass, tables, prefix, prefix.long()), "keep"),
        (lambda: p.poss_pages_evict(pages, mass, tables, prefix, prefix, out_mass=mass[..., 1:]), "out_mass"),
        (lambda: p.poss_pages_compact(pages, tables, prefix, i32(np.zeros((2, 17))), prefix, mass=mass[0]), "mass"),
        (lambda: p.poss_token_logprobs(q), "logits"), (lambda: p.poss_token_logprobs(torch.zeros(3, 4, device="cuda").t()), "logits"),
        (lambda: p.poss_token_logprobs(torch.zeros(3, 4, device="cuda"), tokens=at[0].long()), "tokens"),
        (lambda: p.poss_token_logprobs(torch.zeros(3, 4, device="cuda"), topk=17), "topk"),
    ]
    for f_, name in bad:
        with pytest.raises(ValueError, match=name):
            f_()
    with pytest.raises(p.PossError):
        p.poss_paged_tree_attention_mass(q, pages, mass[..., :-1].contiguous(), 0, tables, prefix, mask, 0.1)
    with pytest.raises(p.PossError):
        p.poss_rotary(q, at, p.poss_rotary_frequencies(66, 1e4))
    with pytest.raises(p.PossError):
        p.poss_token_logprobs(torch.zeros(3, 4, device="cuda"), temperature=0.0)
    torch.cuda.synchronize()
