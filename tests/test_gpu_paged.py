"""GPU tests of the paged-cache and beam calls against their plain 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from tests import paged_util as pg

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def lib():
    import paper_2506_03566_b200 as p
    return p


def cu(a, dtype=None):
    t = torch.as_tensor(a)
    return (t if dtype is None else t.to(dtype)).cuda()


def i32(a):
    return torch.as_tensor(np.asarray(a, np.int32)).cuda()


def tensor_cores(dtype, d, page):
    return dtype == BF and d in (64, 128) and page in (16, 32, 64, 128, 256)


class Case:
    """A batch over one pool; everything also kept on the CPU for the plain form."""

    def __init__(self, seed, dtype, hq, hkv, d, page, prefix, rows, n_rows=None, layers=1, layer=0, anc=None, spare=3,
                 extra_places=1):
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.b, self.rows, self.page, self.d, self.dtype, self.layer = len(prefix), rows, page, d, dtype, layer
        self.prefix, self.n_rows = list(prefix), list(n_rows if n_rows is not None else [rows] * len(prefix))
        held = [p + n for p, n in zip(self.prefix, self.n_rows)]
        n_pages = sum(-(-n // page) for n in held) + spare
        mp = max(-(-(p + rows) // page) for p in self.prefix) + extra_places
        self.tables = pg.make_tables(rng, held, page, n_pages, mp)
        if anc is None:
            self.mask, self.anc = pg.tree_masks(rng, self.b, rows)
        else:
            self.anc = np.broadcast_to(np.asarray(anc, bool), (self.b, rows, rows)).copy()
            self.mask = pg.pack(self.anc)
        self.pages = torch.randn(layers, n_pages, 2, hkv, page, d, generator=gen).to(dtype)
        self.q = torch.randn(self.b, rows, hq, d, generator=gen).to(dtype)
        self.scale = 1.0 / math.sqrt(d)
        self.status = torch.zeros(1, dtype=torch.int32)

    def run(self, out=None, q=None, pages=None, prefix=None, n_rows=None, tables=None, **kw):
        self.gpu_status = self.status.cuda()
        r = lib().poss_paged_tree_attention(
            self.q.cuda() if q is None else q, self.pages.cuda() if pages is None else pages, self.layer,
            cu(self.tables if tables is None else tables), i32(self.prefix if prefix is None else prefix), cu(self.mask),
            self.scale, n_rows=i32(self.n_rows if n_rows is None else n_rows), out=out, status=self.gpu_status, **kw)
        torch.cuda.synchronize()
        return r

    def want(self, **kw):
        return pg.attention(self.q, self.pages[self.layer], self.tables, self.prefix, self.n_rows, self.anc, self.scale, **kw)

    def check(self, got, want=None):
        w, tol, big = self.want() if want is None else want
        return pg.check_attention(got, w, tol, big, self.dtype, tensor_cores(self.dtype, self.d, self.page))


@pytest.mark.parametrize("dtype,hq,hkv,d,page,prefix,rows,n_rows", [
    (F32, 4, 4, 64, 24, [0, 5, 131], 1, None),                    # single tokens, an odd page, an empty context
    (F32, 6, 2, 32, 16, [37, 0, 200, 63], 14, [14, 1, 0, 9]),
    (F32, 8, 1, 128, 8, [300, 17], 61, [61, 33]),
    (F32, 4, 2, 64, 1, [9, 40], 7, None),                         # one slot per page
    (F32, 3, 3, 128, 1024, [1500], 3, None),                      # the largest page
    (BF, 6, 2, 32, 16, [100, 3], 14, None),                       # bf16 off the tensor cores
    (BF, 8, 2, 64, 24, [100, 3], 25, [25, 2]),
    (BF, 32, 8, 128, 16, [0], 1, None),                           # one token that sees itself alone
    (BF, 32, 8, 128, 16, [127, 128, 126, 255], 1, None),          # around the 128-key tiles
    (BF, 32, 8, 128, 16, [127, 1, 250], 3, [3, 2, 3]),
    (BF, 8, 2, 64, 32, [300, 0, 17, 129, 64, 5, 255], 25, [25, 1, 24, 0, 13, 25, 7]),
    (BF, 32, 8, 128, 64, [700, 31], 61, [61, 60]),                # 244 query rows: two tiles of 128
    (BF, 8, 1, 128, 128, [513], 16, None),                        # 128 query rows exactly
    (BF, 8, 1, 128, 256, [513, 1000], 17, [17, 16]),              # just past one tile, pages of two key tiles
    (BF, 4, 1, 64, 256, [257], 128, None),                        # 512 query rows, two mask words
    (BF, 5, 1, 128, 32, [70, 0], 128, [128, 77]),                 # five heads to a key head
    (BF, 6, 2, 64, 16, [400], 65, None),
    (BF, 40, 40, 128, 16, [200], 61, None),                       # multi-head
    (BF, 2, 1, 128, 16, [5000], 2, None),                         # a long context in many pages
])
def test_attention_matches_the_plain_form(dtype, hq, hkv, d, page, prefix, rows, n_rows):
    c = Case(11, dtype, hq, hkv, d, page, prefix, rows, n_rows, layers=2, layer=1)
    fill = torch.full((c.b, rows, hq, d), 7.5, dtype=dtype, device="cuda")
    got = c.run(out=fill.clone())
    assert int(c.gpu_status) == 0
    c.check(got)
    for b in range(c.b):                                          # rows behind the last one are left as they were
        assert torch.equal(got[b, c.n_rows[b]:], fill[b, c.n_rows[b]:])
    assert torch.equal(c.run(out=fill.clone()), got)              # equal calls, equal bits


@pytest.mark.parametrize("dtype,d,page", [(F32, 64, 24), (BF, 64, 16), (BF, 128, 16)])
@pytest.mark.parametrize("rows,prefix", [(5, [3, 125]), (61, [120, 64]), (128, [1, 200])])
def test_what_is_not_seen_has_no_influence_whatever_it_holds(dtype, d, page, rows, prefix):
    """Infinities and NaN behind the last slot of a page, in pages that nobody holds and in tree slots that a row does not
    see; the rows that do see such a slot are the only ones that it reaches."""
    hq, hkv = 8, 2
    n_rows = [rows - 1, rows]
    # chains of three: rows 0..2 see only one another, and so on
    anc = np.zeros((rows, rows), bool)
    for r in range(rows):
        anc[r, r - r % 3:r + 1] = True
    c = Case(5, dtype, hq, hkv, d, page, prefix, rows, n_rows, anc=anc)
    clean = c.want()
    used = set()
    bad = [math.nan, math.inf, -math.inf]
    for b in range(c.b):
        total = c.prefix[b] + c.n_rows[b]
        for s in range(-(-total // page) * page):
            p = int(c.tables[b][s // page])
            used.add(p)
            if s >= total:
                c.pages[0, p, :, :, s % page] = bad[s % 3]
        # the slots of the second chain: keys and values
        for r in (3, 4):
            s = c.prefix[b] + r
            c.pages[0, int(c.tables[b][s // page]), 0, :, s % page, 1] = math.nan
            c.pages[0, int(c.tables[b][s // page]), 1, :, s % page, r] = bad[r % 3]
    for p in range(c.pages.shape[1]):
        if p not in used:
            c.pages[0, p] = math.nan
    got = c.run().cpu()
    want, tol, big = clean
    for b in range(c.b):
        for r in range(c.n_rows[b]):
            if 3 <= r < 6:
                assert not torch.isfinite(got[b, r].float()).all()
                want[b, r] = math.nan
    pg.check_attention(got, want, tol, big, dtype, tensor_cores(dtype, d, page))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,prefix", [(4, [40, 129]), (61, [100, 10])])
def test_infinite_values_reach_the_rows_that_see_them_and_their_columns_only(d, rows, prefix):
    """A value of +inf in a tree slot: the rows that see it get +inf in that column, everything else is as without it."""
    c = Case(6, BF, 8, 2, d, 16, prefix, rows)
    want, tol, big = c.want()
    for b in range(c.b):
        s = c.prefix[b] + 1
        c.pages[0, int(c.tables[b][s // 16]), 1, :, s % 16, 5] = math.inf
    got = c.run().cpu()
    for b in range(c.b):
        for r in range(rows):
            if c.anc[b][r][1]:
                assert (got[b, r, :, 5] == math.inf).all()
                want[b, r, :, 5] = math.nan
    pg.check_attention(got, want, tol, big, BF, True)


@pytest.mark.parametrize("dtype,d,page", [(F32, 64, 24), (BF, 64, 16), (BF, 128, 32)])
def test_rows_whose_mask_leaves_nothing_become_zeros(dtype, d, page):
    anc = np.eye(9, dtype=bool)
    anc[4] = False                                              # not even itself
    c = Case(7, dtype, 4, 2, d, page, [0, 0, 50], 9, [9, 5, 9], anc=anc)
    got = c.run(out=torch.full((3, 9, 4, d), 3.0, dtype=dtype, device="cuda"))
    assert (got[0, 4] == 0).all() and (got[1, 4] == 0).all() and (got[1, 5:] == 3).all()
    c.check(got)


@pytest.mark.parametrize("dtype,d,page", [(F32, 32, 7), (BF, 64, 16), (BF, 128, 64)])
def test_mask_bits_behind_the_last_row_are_not_followed(dtype, d, page):
    c = Case(8, dtype, 4, 4, d, page, [30, 140], 70, [40, 64])
    want = c.want()
    c.mask = np.full_like(c.mask, -1) & ~0                      # every bit set: rows see all rows that exist
    anc = np.ones((2, 70, 70), bool)
    c.anc = anc
    got = c.run()
    w, tol, big = c.want()
    c.check(got, (w, tol, big))
    assert not torch.equal(w.nan_to_num(), want[0].nan_to_num())


@pytest.mark.parametrize("dtype,d,page", [(F32, 64, 24), (BF, 64, 16), (BF, 128, 16), (BF, 128, 256)])
def test_missing_pages_count_as_unseen_and_are_reported(dtype, d, page):
    c = Case(9, dtype, 4, 2, d, page, [600, 90], 5)
    n = c.pages.shape[1]
    c.tables[0][1] = -1
    c.tables[1][0] = n                                          # the first page behind the pool
    got = c.run()
    assert int(c.gpu_status) == 1
    c.check(got)                                                # the plain form leaves those slots out
    c.tables[1][:] = 2 ** 31 - 1
    c.tables[0][:] = -5
    got = c.run()
    assert int(c.gpu_status) == 1 and (got == 0).all()


@pytest.mark.parametrize("dtype,d,page", [(F32, 64, 24), (BF, 128, 16)])
def test_lengths_out_of_range_leave_a_sequence_without_rows(dtype, d, page):
    c = Case(10, dtype, 4, 2, d, page, [100, 60, 33, 7, 1], 5)
    slots = c.tables.shape[1] * page
    out = torch.full((5, 5, 4, d), 2.0, dtype=dtype, device="cuda")
    got = c.run(out=out, prefix=[-1, 60, slots - 4, 7, 2 ** 31 - 1], n_rows=[5, 6, 5, -2, 5])
    assert int(c.gpu_status) == 1 and (got == 2).all()
    # the others are not touched by it
    got = c.run(out=out.clone(), prefix=[100, 60, -3, 7, 1], n_rows=[5, 5, 5, 5, 99])
    assert int(c.gpu_status) == 1 and (got[2] == 2).all() and (got[4] == 2).all()
    w, tol, big = c.want()
    w[2], w[4] = math.nan, math.nan
    c.check(got, (w, tol, big))


@pytest.mark.parametrize("dtype,d", [(F32, 64), (BF, 128)])
def test_queries_cut_out_of_a_fused_projection_and_a_negative_scale(dtype, d):
    c = Case(12, dtype, 4, 2, d, 16, [77, 200], 9)
    fused = torch.randn(2, 9, 8, d).to(dtype).cuda()
    fused[:, :, 2:6] = c.q.cuda()
    assert torch.equal(c.run(q=fused[:, :, 2:6]), c.run())
    c.scale = -0.2
    c.check(c.run())
    c.scale = 0.0                                               # every seen slot counts alike
    c.check(c.run())


def test_attention_argument_checks_of_the_binding():
    c = Case(13, BF, 4, 2, 64, 16, [20], 3)
    q, pages, tables = c.q.cuda(), c.pages.cuda(), cu(c.tables)
    f = lib().poss_paged_tree_attention
    p, m = i32(c.prefix), cu(c.mask)
    for args in ((q.float(), pages, 0, tables, p, m), (q, pages[:, :, :, :, ::2], 0, tables, p, m),
                 (q, pages, 0, tables.long(), p, m), (q, pages, 0, tables, p.cpu(), m), (q, pages, 0, tables, p, m[:, :2]),
                 (q.transpose(1, 2), pages, 0, tables, p, m), (q, pages[0], 0, tables, p, m)):
        with pytest.raises(ValueError):
            f(*args, 0.1)
    with pytest.raises(lib().PossError):
        f(q, pages, 1, tables, p, m, 0.1)
    with pytest.raises(lib().PossError):
        f(q, pages, 0, tables, p, m, 0.1, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert f(q[:0], pages, 0, tables[:0], p[:0], m[:0], 0.1).shape == (0, 3, 4, 64)


@pytest.mark.parametrize("dtype,d,page", [(F32, 64, 24), (BF, 64, 16), (BF, 128, 16)])
def test_captured_attention_replays_with_new_lengths_tables_and_contents(dtype, d, page):
    """Two graphs that share one scratch, replayed in turn, while eager calls run between them."""
    a = Case(14, dtype, 8, 2, d, page, [300, 20], 9, [9, 4], extra_places=40)
    c = Case(15, dtype, 8, 2, d, page, [40, 700], 9, [2, 9], extra_places=40)
    L = lib()
    sz = 0
    graphs = []
    for x in (a, c):
        x.t = {k: v for k, v in (("q", x.q.cuda()), ("pages", x.pages.cuda()), ("tables", cu(x.tables)),
                                 ("prefix", i32(x.prefix)), ("n", i32(x.n_rows)), ("mask", cu(x.mask)))}
        sz = max(sz, L.poss_paged_attention_workspace_bytes(x.t["pages"], 2, 9, 8, x.tables.shape[1]))
    ws = torch.empty(sz, dtype=torch.uint8, device="cuda")

    def call(x):
        return L.poss_paged_tree_attention(x.t["q"], x.t["pages"], 0, x.t["tables"], x.t["prefix"], x.t["mask"], x.scale,
                                           n_rows=x.t["n"], out=x.o, workspace=ws)

    for x in (a, c):
        x.o = torch.zeros_like(x.t["q"])
        call(x)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(x)
        graphs.append(g)
    for _ in range(3):
        for x, g in zip((a, c), graphs):
            x.o.zero_()
            g.replay()
            x.check(x.o)
    a.prefix, a.n_rows = [150, 0], [1, 9]                        # other lengths over the same pages
    a.t["prefix"].copy_(i32(a.prefix))
    a.t["n"].copy_(i32(a.n_rows))
    a.tables[1] = a.tables[0]
    a.t["tables"].copy_(cu(a.tables))
    a.o.zero_()
    graphs[0].replay()
    a.check(a.o)


@pytest.mark.parametrize("d", [64, 128])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_sound(d):
    """The value tiles of one launch are withheld: its bounded waits run out, the status word says so, nothing faults."""
    c = Case(18, BF, 8, 2, d, 16, [300, 5], 9)
    want = c.want()
    c.check(c.run(), want)
    assert lib().load_library().poss_debug_paged_lose_load(1) == 0
    c.run()
    assert int(c.gpu_status) == 6
    c.check(c.run(), want)
    assert int(c.gpu_status) == 0


def test_attention_on_another_stream():
    c = Case(16, BF, 8, 2, 128, 16, [300, 5], 9)
    want = c.want()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        outs = [c.run() for _ in range(4)]
    s.synchronize()
    for o in outs:
        c.check(o, want)


@pytest.mark.parametrize("dtype,page", [(BF, 64), (F32, 24)])
def test_attention_and_append_far_into_a_large_pool(dtype, page):
    """Elements past 2^32 of a pool of several gigabytes, in the last layer and the last pages."""
    hq, hkv, d, layers = 8, 8, 128, 3
    n_pages = (2 ** 31 + 2 ** 29) // (2 * hkv * page * d) if dtype == BF else (2 ** 30 + 2 ** 29) // (2 * hkv * page * d)
    pages = torch.empty(layers, n_pages, 2, hkv, page, d, dtype=dtype, device="cuda")
    assert pages.numel() > 2 ** 32
    c = Case(17, dtype, hq, hkv, d, page, [130, 40], 9)
    n = c.pages.shape[1]
    pages[2, n_pages - n:] = c.pages[0].cuda()
    tables = np.where(c.tables >= 0, c.tables + n_pages - n, -1).astype(np.int32)
    c.layer = 2
    got = c.run(pages=pages, tables=tables)
    assert int(c.gpu_status) == 0
    c.check(got, pg.attention(c.q, c.pages[0], c.tables, c.prefix, c.n_rows, c.anc, c.scale))
    k = torch.randn(2, 9, hkv, d).to(dtype).cuda()
    lib().poss_pages_append(k, -k, pages, 2, cu(tables), i32(c.prefix))
    for b in range(2):
        for r in range(9):
            s = c.prefix[b] + r
            assert torch.equal(pages[2, int(tables[b][s // page]), 0, :, s % page], k[b, r])
            assert torch.equal(pages[2, int(tables[b][s // page]), 1, :, s % page], -k[b, r])


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype,hkv,d,page,prefix,rows,n_rows", [
    (BF, 8, 128, 16, [0], 1, None), (BF, 8, 128, 16, [15, 16, 1000], 61, [61, 3, 0]), (F32, 2, 32, 24, [7, 100], 14, [1, 14]),
    (BF, 2, 32, 7, [3, 50], 33, None), (F32, 40, 128, 64, [130], 128, None), (BF, 1, 64, 256, [100, 0], 1500, [700, 1500]),
])
def test_append_writes_its_slots_and_nothing_else(dtype, hkv, d, page, prefix, rows, n_rows):
    c = Case(20, dtype, hkv, hkv, d, page, prefix, rows, n_rows, layers=2, layer=1,
             anc=np.eye(rows, dtype=bool) if rows > 128 else None)
    kv = torch.randn(c.b, rows, 2 * hkv + 3, d).to(dtype).cuda()
    k, v = kv[:, :, 1:1 + hkv], kv[:, :, 2 + hkv:2 + 2 * hkv]          # slices of a wider row
    pages = c.pages.cuda()
    want = c.pages.clone()
    kc, vc = k.cpu(), v.cpu()
    for b in range(c.b):
        for r in range(c.n_rows[b]):
            s = c.prefix[b] + r
            want[1, int(c.tables[b][s // page]), 0, :, s % page] = kc[b, r]
            want[1, int(c.tables[b][s // page]), 1, :, s % page] = vc[b, r]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib().poss_pages_append(k, v, pages, 1, cu(c.tables), i32(c.prefix), n_rows=i32(c.n_rows), status=status)
    assert torch.equal(pages.cpu(), want) and int(status) == 0


def test_append_leaves_out_missing_pages_and_bad_lengths():
    c = Case(21, BF, 2, 2, 64, 16, [10, 20, 5], 30)
    pages = c.pages.cuda()
    c.tables[0][1] = -1
    c.tables[1][2] = c.pages.shape[1]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    k = torch.ones(3, 30, 2, 64, dtype=BF, device="cuda")
    lib().poss_pages_append(k, k, pages, 0, cu(c.tables), i32([10, 20, c.tables.shape[1] * 16 - 29]), status=status)
    assert int(status) == 1
    want = c.pages.clone()
    for b in (0, 1):
        for r in range(30):
            s = c.prefix[b] + r
            p = int(c.tables[b][s // 16])
            if 0 <= p < want.shape[1]:
                want[0, p, :, :, s % 16] = 1
    assert torch.equal(pages.cpu(), want)


# ------------------------------------------------------------------ compact
@pytest.mark.parametrize("dtype,hkv,d,page,layers", [(BF, 8, 128, 16, 3), (F32, 2, 32, 24, 2), (BF, 2, 64, 1, 1),
                                                     (F32, 40, 128, 64, 1), (BF, 3, 32, 1024, 2)])
def test_compact_moves_the_accepted_paths(dtype, hkv, d, page, layers):
    rng = np.random.default_rng(30)
    prefix = [0, 15, 16, 130, 77]
    rows = 100
    c = Case(30, dtype, hkv, hkv, d, page, prefix, rows, layers=layers)
    path = rng.integers(-9, 999, (5, 17)).astype(np.int32)          # entries behind the path are not read
    acc = np.array([0, 16, 1, 6, 3], np.int32)
    for b, a in enumerate(acc):
        path[b, 1:a + 1] = np.sort(rng.permutation(np.arange(1, rows))[:a])
    path[3, 1:7] = [1, 2, 3, 4, 5, 6]                                # already in place
    path[4, 1:4] = [2, 3, 4]                                         # each target is the next step's source
    want = c.pages.clone()
    for b, a in enumerate(acc):
        for k in range(1, a + 1):
            s, t = prefix[b] + path[b, k], prefix[b] + k
            want[:, c.tables[b][t // page], :, :, t % page] = want[:, c.tables[b][s // page], :, :, s % page].clone()
    pages = c.pages.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    n = lib().poss_pages_compact(pages, cu(c.tables), i32(prefix), cu(path), cu(acc), status=status)
    assert torch.equal(pages.cpu(), want) and n.tolist() == [p + int(a) + 1 for p, a in zip(prefix, acc)]
    assert int(status) == 0


def test_compact_leaves_a_sequence_with_bad_arguments_alone():
    c = Case(31, BF, 2, 2, 64, 16, [20] * 9, 30, layers=2)
    mp = c.tables.shape[1]
    path = np.zeros((9, 17), np.int32)
    path[:, 1:4] = [3, 7, 9]
    acc = np.full(9, 3, np.int32)
    prefix = np.full(9, 20, np.int32)
    acc[0] = -1
    acc[1] = 17
    path[2, 1:4] = [3, 3, 9]
    path[3, 1:4] = [0, 3, 9]
    path[4, 1:4] = [3, 9, mp * 16 - 20]
    prefix[5] = -1
    c.tables[6][1] = -1
    c.tables[7][1] = c.pages.shape[1]
    want = c.pages.clone()
    for k, s in ((1, 3), (2, 7), (3, 9)):
        want[:, c.tables[8][(20 + k) // 16], :, :, (20 + k) % 16] = want[:, c.tables[8][(20 + s) // 16], :, :, (20 + s) % 16]
    pages = c.pages.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    n = lib().poss_pages_compact(pages, cu(c.tables), cu(prefix), cu(path), cu(acc), status=status)
    assert torch.equal(pages.cpu(), want) and int(status) == 1
    assert n.tolist() == [20, 20, 20, 20, 20, -1, 20, 20, 24]


def test_paged_compact_equals_the_contiguous_one():
    """poss_kv_compact on a contiguous cache and poss_pages_compact on pages with the same contents."""
    import poss_synth as ps
    L = lib()
    cfg = ps.CONFIGS["t_bf16"]
    cap = 128
    P = L.Poss(L.make_config(cfg, 64, cap), ps.make_weights(cfg, 1))
    kv = torch.randn_like(P.new_target_kv())                         # [layers][2][heads][slots][d]
    page = 16
    order = torch.randperm(cap // page)
    pages = torch.zeros(kv.shape[0], cap // page, 2, kv.shape[2], page, kv.shape[4], dtype=kv.dtype, device="cuda")
    for i, p in enumerate(order.tolist()):
        pages[:, p] = kv[:, :, :, i * page:(i + 1) * page]
    path = torch.zeros(17, dtype=torch.int32)
    path[1:5] = torch.tensor([2, 5, 6, 20])
    n = torch.tensor([4], dtype=torch.int32).cuda()
    P.poss_kv_compact(kv, 50, path.cuda(), n)
    L.poss_pages_compact(pages, order.to(torch.int32).view(1, -1).cuda(), i32([50]), path.view(1, 17).cuda(), n)
    for i, p in enumerate(order.tolist()):
        assert torch.equal(pages[:, p], kv[:, :, :, i * page:(i + 1) * page])


# ------------------------------------------------------------------ remap
def run_remap(pages, tables, lens, refs, parents, room, **kw):
    return lib().poss_pages_remap(pages, i32(tables), i32(lens), i32(refs), i32(parents) if parents is not None else None,
                                  i32(room) if room is not None else None, **kw)


def check_remap(pages, tables, lens, refs, parents, room):
    """One call against the definition; returns the new state (tables, refs, lengths, free) or None when it did not fit."""
    page = pages.shape[4]
    n1 = len(parents)
    want, missing = pg.remap(tables, lens, refs, parents, room, page)
    before = pages.cpu()
    out = {"tables": torch.full((n1, tables.shape[1]), 77, dtype=torch.int32, device="cuda"),
           "refs": torch.empty(len(refs), dtype=torch.int32, device="cuda"),
           "seq_len": torch.full((n1,), 77, dtype=torch.int32, device="cuda"),
           "n_free": torch.empty(1, dtype=torch.int32, device="cuda")}
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run_remap(pages, tables, lens, refs, parents, room, out=out, status=status)
    assert int(status) == 0
    if want is None:
        assert int(got["n_free"]) == -missing and got["refs"].tolist() == list(refs)
        assert (got["tables"] == 77).all() and (got["seq_len"] == 77).all() and torch.equal(pages.cpu(), before)
        return None
    t, r, n, free, copies = want
    assert np.array_equal(got["tables"].cpu().numpy(), t)
    assert np.array_equal(got["refs"].cpu().numpy(), r)
    assert np.array_equal(got["seq_len"].cpu().numpy(), n) and int(got["n_free"]) == free
    for src, dst, m in copies:
        before[:, dst, :, :, :m] = before[:, src, :, :, :m]
    assert torch.equal(pages.cpu(), before)
    return t, r, n, free


@pytest.mark.parametrize("dtype,hkv,d,page,layers,n,mp,n_pages", [
    (BF, 2, 64, 16, 2, 6, 12, 60), (F32, 1, 32, 5, 1, 33, 9, 300), (BF, 8, 128, 64, 3, 4, 4, 14), (BF, 1, 32, 1, 1, 5, 70, 200),
    (F32, 2, 32, 3, 1, 64, 40, 2500),
])
def test_remap_over_many_random_steps(dtype, hkv, d, page, layers, n, mp, n_pages):
    """Forks, reorderings, cuts, growth, sequences that end and start, pages pinned from outside, steps that do not fit."""
    rng = np.random.default_rng(40)
    pages = torch.randn(layers, n_pages, 2, hkv, page, d, device="cuda").to(dtype)
    refs = np.zeros(n_pages, np.int32)
    refs[3] = 2                                                      # held from outside
    tables, lens = np.full((n, mp), -1, np.int32), np.zeros(n, np.int32)
    fits = 0
    for step in range(25):
        n1 = n if step % 5 else int(rng.integers(1, n + 1))
        parents = rng.integers(-1, len(lens), n1)
        cut = np.maximum(0, lens - np.where(rng.random(len(lens)) < 0.3, rng.integers(0, 2 * page + 1, len(lens)), 0)).astype(np.int32)
        kept = np.where(parents >= 0, cut[np.maximum(parents, 0)], 0)
        room = np.minimum(rng.integers(0, 3 * page + 2, n1), mp * page - kept)
        if step == 4 and len(lens) > 1:                              # a page of the table pinned from outside as well
            held = tables[tables >= 0]
            if held.size:
                refs[held[-1]] += 1
        state = check_remap(pages, tables, cut, refs, parents.tolist(), room.tolist())
        if state is None:                                            # start over, the pinned pages stay
            for p in tables[tables >= 0]:
                refs[p] -= 1
            tables, lens = np.full((n1, mp), -1, np.int32), np.zeros(n1, np.int32)
            continue
        fits += 1
        tables, refs, lens, _ = state
        lens = (lens + np.array([int(rng.integers(0, x + 1)) for x in room])).astype(np.int32)
    assert fits > 10


def test_remap_frees_everything_and_takes_no_parents_or_room():
    pages = torch.randn(1, 20, 2, 2, 16, 64, device="cuda").to(BF)
    tables = np.array([[4, 5, -1], [6, -1, -1], [4, 9, -1]], np.int32)
    refs = np.zeros(20, np.int32)
    refs[[4, 5, 6, 9]] = [2, 1, 1, 1]
    lens = [20, 16, 30]
    r = run_remap(pages, tables, lens, refs, None, None)             # as they are: nothing moves
    assert r["tables"].tolist() == tables.tolist() and r["refs"].tolist() == refs.tolist() and int(r["n_free"]) == 16
    r = run_remap(pages, tables, lens, refs, [-1, -1, -1], None)
    assert (r["tables"] == -1).all() and (r["refs"] == 0).all() and int(r["n_free"]) == 20 and r["seq_len"].tolist() == [0] * 3
    r = run_remap(pages, tables, lens, refs, [], [])                 # no sequence at all
    assert (r["refs"] == 0).all() and int(r["n_free"]) == 20 and r["tables"].shape == (0, 3)
    r = run_remap(pages, np.zeros((0, 3), np.int32), [], np.zeros(20), [-1, -1], [17, 0])
    assert r["tables"].tolist() == [[0, 1, -1], [-1, -1, -1]] and int(r["n_free"]) == 18


def test_remap_treats_bad_arguments_as_empty_sequences_and_absent_entries():
    pages = torch.randn(1, 20, 2, 2, 16, 64, device="cuda").to(BF)
    tables = np.array([[4, 20, -1], [6, 2 ** 31 - 1, -1]], np.int32)
    refs = np.zeros(20, np.int32)
    refs[[4, 6]] = 1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = pages.clone()
    r = run_remap(pages, tables, [20, 49], refs, [0, 1, 2, 99, 0], [0, 0, 5, 5, -1], status=status)
    assert int(status) == 1
    # sequence 0: its second page was never there, a fresh one takes its place; 1 is too long; 2 and 3 have no such
    # parent; 4 has no such room
    assert r["tables"].tolist() == [[4, 0, -1]] + [[-1, -1, -1]] * 4 and r["seq_len"].tolist() == [20, 0, 0, 0, 0]
    want = np.zeros(20, np.int32)
    want[[0, 4]] = 1
    assert r["refs"].tolist() == want.tolist() and int(r["n_free"]) == 18 and torch.equal(pages, before)


def test_captured_remap_and_compact_replay():
    L = lib()
    pages = torch.randn(2, 30, 2, 2, 16, 64, device="cuda").to(BF)
    tables, lens = i32([[1, 2, -1, -1], [3, 4, -1, -1]]), i32([20, 25])
    refs = torch.zeros(30, dtype=torch.int32, device="cuda")
    refs[1:5] = 1
    parents, room = i32([1, 1]), i32([3, 3])
    path = torch.zeros(2, 17, dtype=torch.int32, device="cuda")
    path[:, 1] = 2
    acc = i32([1, 1])
    out = L.poss_pages_remap(pages, tables, lens, refs, parents, room)
    L.poss_pages_compact(pages, out["tables"], out["seq_len"], path, acc)
    torch.cuda.synchronize()
    start = torch.randn_like(pages)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r = L.poss_pages_remap(pages, tables, lens, refs, parents, room)
        n = L.poss_pages_compact(pages, r["tables"], r["seq_len"], path, acc)
    for par in ([1, 1], [0, 1], [1, 0], [0, 0]):
        pages.copy_(start)
        parents.copy_(i32(par))
        g.replay()
        torch.cuda.synchronize()
        want, _ = pg.remap(tables.cpu().numpy(), lens.tolist(), refs.tolist(), par, [3, 3], 16)
        w = start.cpu()
        for src, dst, m in want[4]:
            w[:, dst, :, :, :m] = w[:, src, :, :, :m]
        for b in range(2):
            s, t = int(want[2][b]) + 2, int(want[2][b]) + 1
            w[:, want[0][b][t // 16], :, :, t % 16] = w[:, want[0][b][s // 16], :, :, s % 16].clone()
        assert np.array_equal(r["tables"].cpu().numpy(), want[0]) and r["refs"].tolist() == want[1].tolist()
        assert n.tolist() == [int(x) + 2 for x in want[2]] and torch.equal(pages.cpu(), w)


# ------------------------------------------------------------------ beam selection
def check_beams(x, scores, finished=None, eos=-1):
    r = lib().poss_beam_select(x, cu(scores, F32), finished=None if finished is None else i32(finished), eos=eos)
    torch.cuda.synchronize()
    tok, par, sc, fin = pg.beam_select(x.double().cpu().numpy(), np.asarray(scores, np.float32), finished, eos)
    assert np.array_equal(r["tokens"].cpu().numpy(), tok)
    assert np.array_equal(r["parents"].cpu().numpy(), par)
    assert np.array_equal(r["finished"].cpu().numpy(), fin)
    got = r["scores"].double().cpu().numpy()
    on = np.isfinite(sc)
    assert np.array_equal(np.isneginf(got), ~on)
    # rounded once (2^-24 of the score); lse from fp32 exponentials and chunk sums: 2^-20 absolute
    assert (np.abs(got[on] - sc[on]) <= np.abs(sc[on]) * 2.0 ** -24 + 2.0 ** -20).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("batch,k,v", [(1, 1, 1), (2, 4, 3), (1, 4, 100), (3, 8, 777), (2, 16, 5000), (5, 3, 8192),
                                       (1, 7, 8193), (4, 4, 32003), (2, 9, 128256)])
def test_beam_selection_matches_the_definition(dtype, batch, k, v):
    torch.manual_seed(50)
    x = (torch.randn(batch, k, v, device="cuda") * 3).to(dtype)
    s = -np.random.default_rng(51).random((batch, k)).astype(np.float32) * 5
    check_beams(x, s)
    fin = (np.random.default_rng(52).random((batch, k)) < 0.3).astype(np.int32)
    check_beams(x, s, fin, eos=min(2, v - 1))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("v", [50, 8192, 20001])
def test_equal_logits_go_to_the_lower_beam_and_token(dtype, v):
    """Constant rows (every logit at the bound: the selection's slow rounds) and rows of few different values."""
    x = torch.zeros(2, 6, v, device="cuda", dtype=dtype)
    check_beams(x, np.zeros((2, 6), np.float32))
    torch.manual_seed(53)
    x = torch.randint(0, 3, (2, 6, v), device="cuda").to(dtype)
    check_beams(x, np.zeros((2, 6), np.float32))
    check_beams(x, np.full((2, 6), -1.5, np.float32), np.ones((2, 6), np.int32), eos=1)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_banned_tokens_dead_beams_and_too_few_continuations(dtype):
    torch.manual_seed(54)
    v, k = 30000, 12
    x = torch.randn(6, k, v, device="cuda").to(dtype)
    x[0, :, 5:] = -math.inf                                          # a handful of tokens allowed
    x[1, :, :29000] = math.nan
    x[2, ::2] = -math.inf                                            # every other beam banned outright
    x[3, :, 7] = math.inf                                            # not a number to compare with: banned too
    x[4, 0, :8192] = -math.inf
    x[4, 1, 1024:] = -math.inf
    x[5] = -math.inf
    x[5, 3, [9, 100, 29999]] = 1.0
    s = -torch.rand(6, k).numpy()
    s[2, 1] = math.nan
    s[2, 3] = -math.inf
    s[4, 2:] = -math.inf                                             # the first step of a search, nearly
    check_beams(x, s)
    fin = np.zeros((6, k), np.int32)
    fin[5, :2] = 1
    fin[2, 3] = 1                                                    # finished, but without a score: dead
    check_beams(x, s, fin, eos=0)


def test_sorted_and_steep_logits():
    v, k = 40000, 5
    up = torch.arange(v, device="cuda", dtype=F32) * 1e-3
    x = torch.stack([up, up.flip(0), torch.roll(up, 777), up * 100, -up * 100]).view(1, k, v).contiguous()
    check_beams(x, np.linspace(-3, 0, k).astype(np.float32).reshape(1, k))


def test_beam_selection_in_a_graph_with_a_shared_scratch_and_misaligned_rows():
    L = lib()
    torch.manual_seed(55)
    v, k = 10007, 4                                                  # odd: the rows start at every place of 16 bytes
    xs = [torch.randn(2, k, v, device="cuda") for _ in range(2)]
    s = torch.zeros(2, k, device="cuda")
    ws = torch.empty(L.poss_beam_select_workspace_bytes(2, k, v), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for x in xs:
        L.poss_beam_select(x, s, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(L.poss_beam_select(x, s, workspace=ws))
        graphs.append(g)
    for _ in range(2):
        for x, g, o in zip(xs, graphs, outs):
            x.normal_()
            g.replay()
            torch.cuda.synchronize()
            tok, par, sc, _ = pg.beam_select(x.double().cpu().numpy(), s.cpu().numpy(), None, -1)
            assert np.array_equal(o["tokens"].cpu().numpy(), tok) and np.array_equal(o["parents"].cpu().numpy(), par)


# ------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype,d,page", [(F32, 32, 5), (BF, 64, 16), (BF, 128, 16)])
def test_a_beam_search_over_shared_pages(dtype, d, page):
    """Steps of a beam search as a program runs them -- select, remap with the selected parents, append, attend, logits from
    the attention's output -- against the same search over caches that every beam holds for itself."""
    L = lib()
    torch.manual_seed(60)
    hq, hkv, k, v, steps, mp = 4, 2, 4, 300, 24, 8 if page > 5 else 14
    emb = torch.randn(v, (hq + 2 * hkv), d, device="cuda").to(dtype)
    head = torch.randn(hq * d, v, device="cuda")
    n_pages = 3 * k
    pages = torch.full((1, n_pages, 2, hkv, page, d), math.nan, device="cuda").to(dtype)
    state = {"tables": torch.full((k, mp), -1, dtype=torch.int32, device="cuda"),
             "refs": torch.zeros(n_pages, dtype=torch.int32, device="cuda"),
             "seq_len": torch.zeros(k, dtype=torch.int32, device="cuda")}
    if page == 5:
        n_pages = 10 * k
        pages = torch.full((1, n_pages, 2, hkv, page, d), math.nan, device="cuda").to(dtype)
        state["refs"] = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    one = torch.ones(k, dtype=torch.int32, device="cuda")
    mask = torch.ones(k, 1, 1, dtype=torch.int64, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tokens = torch.full((k,), 7, dtype=torch.int32, device="cuda")
    parents = torch.arange(k, dtype=torch.int32, device="cuda")
    scores = torch.tensor([[0.0] + [-math.inf] * (k - 1)], device="cuda")
    own = [[] for _ in range(k)]                                    # every beam's (key, value) rows
    for step in range(steps):
        r = L.poss_pages_remap(pages, state["tables"], state["seq_len"], state["refs"], parents, one, status=status)
        assert int(r["n_free"]) >= 0
        qkv = emb[tokens.long()].view(k, 1, hq + 2 * hkv, d)
        L.poss_pages_append(qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:], pages, 0, r["tables"], r["seq_len"], status=status)
        o = L.poss_paged_tree_attention(qkv[:, :, :hq], pages, 0, r["tables"], r["seq_len"], mask, 0.3, status=status)
        own = [own[p] + [qkv[i, 0, hq:].cpu()] for i, p in enumerate(parents.tolist())]
        for i in range(k):
            kv = torch.stack(own[i])
            flat = torch.stack([kv[:, :hkv], kv[:, hkv:]], 1).permute(1, 2, 0, 3)[None]   # one page holds it all
            want, tol, big = pg.attention(qkv[i:i + 1, :, :hq].cpu(), flat, [[0]], [step], [1], [[[True]]], 0.3)
            pg.check_attention(o[i:i + 1], want, tol, big, dtype, tensor_cores(dtype, d, page))
        x = (o.view(k, hq * d).float() @ head).view(1, k, v).contiguous()
        b = L.poss_beam_select(x, scores, eos=-1)
        tok, par, sc, _ = pg.beam_select(x.double().cpu().numpy(), scores.cpu().numpy(), None, -1)
        assert np.array_equal(b["tokens"].cpu().numpy(), tok) and np.array_equal(b["parents"].cpu().numpy(), par)
        tokens, parents, scores = b["tokens"].view(-1), b["parents"].view(-1), b["scores"]
        state = {"tables": r["tables"], "refs": r["refs"], "seq_len": r["seq_len"] + 1}
    assert int(status) == 0


def test_rounds_of_drafted_trees_over_pages():
    """Rounds of a batch -- room for the trees, append, attention, acceptance, compaction, surplus pages given back -- against
    contiguous caches and the contiguous calls (poss_tree_attention, poss_kv_compact)."""
    import poss_synth as ps
    L = lib()
    torch.manual_seed(61)
    rng = np.random.default_rng(61)
    cfg = ps.CONFIGS["t_bf16"].replace(n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=1024, vocab=64, ffn=64, n_target_layers=1)
    cap, rows, batch, page, mp = 320, 21, 3, 16, 20
    P = L.Poss(L.make_config(cfg, 64, cap), ps.make_weights(cfg, 1))
    flat = [torch.zeros_like(P.new_target_kv()) for _ in range(batch)]
    pages = torch.full((1, 45, 2, 2, page, 128), math.nan, device="cuda").to(BF)
    refs = torch.zeros(45, dtype=torch.int32, device="cuda")
    tables = torch.full((batch, mp), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
    room = torch.full((batch,), rows, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    scale = 1.0 / math.sqrt(128)
    for rnd in range(12):
        r = L.poss_pages_remap(pages, tables, lens, refs, None, room, status=status)
        assert int(r["n_free"]) >= 0
        tables, refs = r["tables"], r["refs"]
        qkv = torch.randn(batch, rows, 12, 128, device="cuda").to(BF)
        mask, anc = pg.tree_masks(rng, batch, rows)
        m = cu(mask)
        k, v = qkv[:, :, 8:10], qkv[:, :, 10:]
        L.poss_pages_append(k, v, pages, 0, tables, lens, status=status)
        o = L.poss_paged_tree_attention(qkv[:, :, :8], pages, 0, tables, lens, m, scale, status=status)
        path = np.zeros((batch, 17), np.int32)
        acc = rng.integers(0, 8, batch).astype(np.int32)
        for b in range(batch):
            n = int(lens[b])
            flat[b][0, 0, :, n:n + rows] = k[b].transpose(0, 1)
            flat[b][0, 1, :, n:n + rows] = v[b].transpose(0, 1)
            want = P.poss_tree_attention(qkv[b, :, :8].contiguous(), flat[b][0], n, m[b].contiguous(), scale)
            # both are within half a bf16 step of sums that differ by the rounding of the probabilities (2^-8 of the
            # sum of |w v|, itself below the largest |v| seen)
            top = float(v.abs().max()) if n == 0 else float(flat[b][0, 1, :, :n + rows].abs().max())
            assert ((o[b].float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 2.0 ** -8 * top).all()
            path[b, 1:acc[b] + 1] = np.sort(rng.permutation(np.arange(1, rows))[:acc[b]])
            P.poss_kv_compact(flat[b], n, cu(path[b]), i32([acc[b]]))
        lens = L.poss_pages_compact(pages, tables, lens, cu(path), cu(acc), status=status)
        r = L.poss_pages_remap(pages, tables, lens, refs, status=status)
        tables, refs = r["tables"], r["refs"]
        for b in range(batch):
            n = int(lens[b])
            assert int((tables[b] >= 0).sum()) == -(-n // page)
            for s in range(n):
                assert torch.equal(pages[0, int(tables[b][s // page]), :, :, s % page], flat[b][0, :, :, s])
    assert int(status) == 0 and int(refs.sum()) == sum(-(-int(n) // page) for n in lens.tolist())


# ------------------------------------------------------------------ what the cut of the work over the SMs can meet
@pytest.mark.parametrize("dtype,hq,hkv,d,page,prefix,rows,n_rows", [
    (BF, 3, 1, 128, 16, [3000, 0], 5, [5, 4]),                    # three heads to a key head, one item over many SMs
    (BF, 7, 1, 64, 64, [1500, 2], 40, [40, 11]),                  # seven: slots of 18 rows, three items
    (BF, 130, 1, 64, 16, [70], 2, None),                          # more heads to a key head than a slot has rows
    (BF, 128, 1, 128, 16, [333], 3, None),                        # a slot per row
    (BF, 4, 2, 64, 128, [190, 64, 63, 0], 70, [70, 1, 65, 70]),   # trees over page and tile ends
    (BF, 4, 2, 128, 256, [250, 511], 128, [128, 100]),
    (BF, 8, 2, 128, 16, [64 * i + j for i in range(8) for j in (-1 + (i == 0), 0, 1)], 2, None),   # all around the tiles
])
def test_attention_over_uneven_cuts(dtype, hq, hkv, d, page, prefix, rows, n_rows):
    c = Case(60, dtype, hq, hkv, d, page, prefix, rows, n_rows)
    got = c.run()
    assert int(c.gpu_status) == 0
    c.check(got)
    for _ in range(20):
        assert torch.equal(c.run()[:, :1], got[:, :1])


@pytest.mark.parametrize("d,batch,rows", [(64, 200, 3), (128, 33, 5), (64, 1024, 1)])
def test_attention_of_many_short_sequences(d, batch, rows):
    """More sequences than a warp has lanes, most with a tile or less, some without rows; a long one in their middle."""
    rng = np.random.default_rng(61)
    prefix = rng.integers(0, 70, batch).tolist()
    prefix[batch // 2] = 900
    n_rows = rng.integers(0, rows + 1, batch).tolist()
    n_rows[batch // 2] = rows
    c = Case(62, BF, 2, 1, d, 16, prefix, rows, n_rows)
    fill = torch.full((batch, rows, 2, d), -3.0, dtype=BF, device="cuda")
    got = c.run(out=fill.clone())
    assert int(c.gpu_status) == 0
    c.check(got)
    for b in range(batch):
        assert torch.equal(got[b, n_rows[b]:], fill[b, n_rows[b]:])


@pytest.mark.parametrize("d", [64, 128])
def test_a_batch_without_rows_or_slots_writes_nothing(d):
    c = Case(63, BF, 4, 2, d, 16, [30, 0, 7], 3, [0, 0, 0])
    fill = torch.full((3, 3, 4, d), 2.0, dtype=BF, device="cuda")
    assert torch.equal(c.run(out=fill.clone()), fill) and int(c.gpu_status) == 0


@pytest.mark.parametrize("dtype,d,page", [(F32, 64, 24), (BF, 64, 16), (BF, 128, 16)])
def test_two_attention_calls_at_once(dtype, d, page):
    """Two streams, each with scratch of its own, many calls in flight."""
    cases = [Case(64 + i, dtype, 8, 2, d, page, [700 - 300 * i, 33, 5], 9 + 20 * i) for i in range(2)]
    wants = [c.want() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    args = [(c.q.cuda(), c.pages.cuda(), 0, cu(c.tables), i32(c.prefix), cu(c.mask), c.scale) for c in cases]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(12):
        for s, a, o in zip(streams, args, outs):
            with torch.cuda.stream(s):
                o.append(lib().poss_paged_tree_attention(*a))
    torch.cuda.synchronize()
    for c, w, o in zip(cases, wants, outs):
        c.check(o[0], w)
        assert all(torch.equal(x, o[0]) for x in o)


def test_two_captured_graphs_share_scratch_in_turn():
    """Scratch needs no initial value: graphs that use the same, replayed one behind the other, leave each other alone."""
    cases = [Case(66 + i, BF, 8, 2, 128, 16, [900 - 500 * i, 64], 3 + 30 * i) for i in range(2)]
    L = lib()
    ws = torch.empty(max(L.poss_paged_attention_workspace_bytes(c.pages.cuda(), 2, c.rows, 8, c.tables.shape[1])
                         for c in cases), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for c in cases:
        a = (c.q.cuda(), c.pages.cuda(), 0, cu(c.tables), i32(c.prefix), cu(c.mask), c.scale)
        out = torch.empty(2, c.rows, 8, 128, dtype=BF, device="cuda")
        L.poss_paged_tree_attention(*a, out=out, workspace=ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            L.poss_paged_tree_attention(*a, out=out, workspace=ws)
        graphs.append((g, a))
        outs.append(out)
    wants = [c.want() for c in cases]
    for _ in range(3):
        for o in outs:
            o.fill_(9.0)
        ws.fill_(255)                                             # (NaN wherever it is read before it is written)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for c, o, w in zip(cases, outs, wants):
            c.check(o, w)


# ------------------------------------------------------------------ beams: the selection's rare paths, and in place
def test_beam_selection_with_more_entries_than_the_merge_ranks():
    """One part of the merge's lists holds nothing but poor heads, so the bound keeps out none of the others' entries."""
    torch.manual_seed(70)
    k, v = 16, 32 * 8192 - 7
    x = torch.randn(1, k, v, device="cuda")
    for chunk in (15, 31):
        x[:, :, chunk * 8192 - 8:(chunk + 1) * 8192 + 8] = -60.0
    check_beams(x, -np.random.default_rng(71).random((1, k)).astype(np.float32))
    x[0, 3] = 0.0                                                 # (and equal logits in one of the beams)
    check_beams(x, np.zeros((1, k), np.float32))


@pytest.mark.parametrize("k,v", [(4, 32003), (16, 9000), (1, 40000)])
def test_beam_selection_in_place(k, v):
    torch.manual_seed(72)
    L = lib()
    x = torch.randn(3, k, v, device="cuda")
    s = -torch.rand(3, k, device="cuda")
    f = (torch.rand(3, k, device="cuda") < 0.3).to(torch.int32)
    want = L.poss_beam_select(x, s, finished=f, eos=1)
    out = {"tokens": torch.empty_like(f), "parents": torch.empty_like(f), "scores": s, "finished": f}
    got = L.poss_beam_select(x, s, finished=f, eos=1, out=out)
    assert all(torch.equal(got[n], want[n]) for n in want) and got["scores"] is s
    with pytest.raises(L.PossError):
        L.poss_beam_select(x, s, out={**out, "tokens": out["parents"]})


def test_outputs_over_inputs_are_refused():
    L = lib()
    pages = torch.zeros(1, 4, 2, 2, 16, 64, dtype=BF, device="cuda")
    t, n = i32([[0, 1], [2, -1]]), i32([20, 3])
    path, acc = torch.zeros(2, L.POSS_MAX_DEPTH + 1, dtype=torch.int32, device="cuda"), i32([0, 0])
    with pytest.raises(L.PossError):
        L.poss_pages_compact(pages, t, n, path, acc, out_len=n)
    refs = i32([1, 1, 1, 0])
    out = {"tables": torch.empty_like(t), "refs": torch.empty_like(refs), "seq_len": n, "n_free": i32([0])}
    with pytest.raises(L.PossError):
        L.poss_pages_remap(pages, t, n, refs, out=out)
    q = torch.zeros(2, 1, 4, 64, dtype=BF, device="cuda")
    with pytest.raises(L.PossError):
        L.poss_paged_tree_attention(q, pages, 0, t, n, torch.ones(2, 1, 1, dtype=torch.int64, device="cuda"), 0.1, out=q)
    assert L.poss_pages_compact(pages, t, n, path, acc).tolist() == [21, 4]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("v", [255, 256, 257, 1000, 2047, 8192 + 3, 8192 + 700, 16384 + 2049])
def test_beam_selection_over_chunks_that_the_vocabulary_does_not_fill(dtype, v):
    torch.manual_seed(73)
    for k in (1, 5, 16):
        x = (torch.randn(2, k, v, device="cuda") * 2).to(dtype)
        x[0, 0, -1] = 30.0                                        # the row's last logit is the best
        x[1, :, 0] = 25.0
        check_beams(x, -np.random.default_rng(74).random((2, k)).astype(np.float32))


@pytest.mark.parametrize("n_pages", [12 * 1024, 12 * 1024 + 1, 20000])
def test_remap_of_a_pool_larger_than_shared_memory_counts(n_pages):
    """Either side of the pool size up to which the counts lie in shared memory; most pages pinned, so that the free ones lie far up."""
    rng = np.random.default_rng(75)
    n, mp, page = 40, 12, 4
    pages = torch.randn(1, n_pages, 2, 1, page, 32, device="cuda")
    refs = (rng.random(n_pages) < 0.98).astype(np.int32)
    refs[-50:] = 0
    tables, lens = np.full((n, mp), -1, np.int32), np.zeros(n, np.int32)
    fits = 0
    for step in range(8):
        parents = rng.integers(-1, n, n)
        kept = np.where(parents >= 0, lens[np.maximum(parents, 0)], 0)
        room = np.minimum(rng.integers(0, 2 * page + 2, n), mp * page - kept)
        state = check_remap(pages, tables, lens, refs, parents.tolist(), room.tolist())
        if state is None:
            for p in tables[tables >= 0]:
                refs[p] -= 1
            tables, lens = np.full((n, mp), -1, np.int32), np.zeros(n, np.int32)
            continue
        fits += 1
        tables, refs, lens, _ = state
        lens = (lens + room).astype(np.int32)
    assert fits > 3
