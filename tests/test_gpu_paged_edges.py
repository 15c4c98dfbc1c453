"""GPU tests of the paged-cache and beam calls at the edges of what they document: logits of any finite size, beams that are
alike, outputs of a call that did not fit, items of one key tile behind longer ones."""
import math

import numpy as np
import pytest
import torch

from tests import paged_util as pg
from tests.test_gpu_paged import BF, F32, Case, i32, lib

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ beams
def check_selection(x, scores, finished=None, eos=-1):
    """The definition in 64 bits.  A score is off by half a step of fp32 (2^-24 of it), by 2^-20 for the sum of exponentials (fp32
    terms and chunk sums), and by what 64 bits leave of maximum + log(sum) and of the logit minus it: two roundings, 2^-53 of the
    row's largest finite logit each, on either side."""
    s = np.asarray(scores, np.float32)
    out = {"tokens": torch.full(s.shape, 77, dtype=torch.int32, device="cuda"), "parents": torch.full(s.shape, 77, dtype=torch.int32, device="cuda"),
           "scores": torch.full(s.shape, 77.0, device="cuda"), "finished": torch.full(s.shape, 77, dtype=torch.int32, device="cuda")}
    r = lib().poss_beam_select(x, torch.as_tensor(s).cuda(), finished=None if finished is None else i32(finished), eos=eos, out=out)
    torch.cuda.synchronize()
    rows = x.double().cpu().numpy()
    tok, par, sc, fin = pg.beam_select(rows, s, finished, eos)
    assert np.array_equal(r["tokens"].cpu().numpy(), tok)
    assert np.array_equal(r["parents"].cpu().numpy(), par)
    assert np.array_equal(r["finished"].cpu().numpy(), fin)
    got = r["scores"].double().cpu().numpy()
    on = np.isfinite(sc)
    assert np.array_equal(np.isneginf(got), ~on)
    top = np.where(np.isfinite(rows), np.abs(rows), 0.0).max(-1).reshape(-1)[np.maximum(par, 0)]
    assert (np.abs(got[on] - sc[on]) <= np.abs(sc[on]) * 2.0 ** -24 + 2.0 ** -20 + top[on] * 2.0 ** -51).all()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("low", ["lowest", -1e30, -1e10, -3e9, -1e9, -1e4])
def test_finite_masks_of_any_size_leave_the_other_logits_alone(dtype, low):
    """Tokens masked with the type's lowest value, or another very negative number: whole chunks of 8192, a last chunk that the
    vocabulary does not fill, whole rows, and all but a few tokens."""
    low = torch.finfo(dtype).min if low == "lowest" else low
    torch.manual_seed(80)
    k, v = 4, 30000
    x = (torch.randn(7, k, v, device="cuda") * 2).to(dtype)
    x[0, :, 8192:] = low
    x[1, :, :29000] = low
    x[2] = low                                                  # a row of equal logits, however low
    x[3, 1:3] = low
    x[4, :, 3:] = low                                           # fewer tokens left than beams
    x[5, :, 8192:16384] = low
    x[5, :, 9000] = -math.inf
    x[6, :, 16384:] = low
    x[6, :, 16384:24576] = -math.inf
    x[6, :, 29999] = math.nan
    check_selection(x, -np.random.default_rng(81).random((7, k)).astype(np.float32))
    check_selection(x, np.zeros((7, k), np.float32), np.eye(7, k, dtype=np.int32), eos=3)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("high", [1e4, 1e9, 1e10, 1e30, 3e38])
def test_logits_of_any_finite_size(dtype, high):
    torch.manual_seed(82)
    k, v = 5, 20011
    x = (torch.randn(3, k, v, device="cuda") * 2).to(dtype)
    x[0, :, 100:117] = high
    x[1, 2] = high
    x[2] *= high / 16                                           # logits spread over the whole size, both signs
    check_selection(x, -np.random.default_rng(83).random((3, k)).astype(np.float32))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("k,v", [(4, 10007), (16, 8193), (7, 32003), (8, 50257), (3, 24578), (5, 32000)])
def test_beams_that_are_alike_tie_wherever_their_rows_start(dtype, k, v):
    """Equal logits and scores are equal continuations: the lower beam comes first.  Rows of these lengths start at every place of
    16 bytes."""
    torch.manual_seed(84)
    x = torch.randn(3, 1, v, device="cuda").to(dtype).expand(3, k, v).contiguous()
    check_selection(x, np.zeros((3, k), np.float32))
    check_selection(x, np.full((3, k), -2.3, np.float32))
    y = torch.randn(1, 1, v, device="cuda").to(dtype)
    x[2, 1::2] = y[0]                                             # two kinds in turn
    check_selection(x, np.full((3, k), 0.7, np.float32))


# ------------------------------------------------------------------ attention
@pytest.mark.parametrize("d,lens", [(128, (150, 20, 40)), (64, (150, 20, 40)), (128, (700, 3, 60, 1, 64))])
def test_items_of_one_tile_behind_longer_ones(d, lens):
    """Few rows, so the two slots of a CTA share them and take the key tiles in turn: over a short sequence the second slot has
    nothing to do and is at the next item at once, while the first still joins both slots' sums of the one before."""
    batch, rows = 600, 2
    prefix = [lens[i % len(lens)] - rows for i in range(batch)]
    c = Case(90, BF, 2, 1, d, 16, [max(0, p) for p in prefix], rows)
    got = c.run()
    assert int(c.gpu_status) == 0
    c.check(got)
    args = (c.q.cuda(), c.pages.cuda(), 0, torch.as_tensor(c.tables).cuda(), i32(c.prefix), torch.as_tensor(c.mask).cuda(), c.scale)
    outs = [lib().poss_paged_tree_attention(*args) for _ in range(100)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, got) for o in outs)


@pytest.mark.parametrize("d,hq,hkv,rows", [(128, 32, 8, 61), (64, 8, 8, 128), (128, 4, 1, 2)])
def test_a_wait_that_runs_out_with_many_items_in_a_cta(d, hq, hkv, rows):
    """The value tiles of one launch are withheld from CTAs that hold several items of few tiles, with rows for both slots or for
    one: every role comes to the end of its walk, the status word says so, and the next call is sound."""
    batch = 64 if rows > 2 else 600
    c = Case(91, BF, hq, hkv, d, 16, [100 - rows // 2] * batch, rows)
    first = c.run()
    assert int(c.gpu_status) == 0
    assert lib().load_library().poss_debug_paged_lose_load(1) == 0
    c.run()
    assert int(c.gpu_status) == 6
    assert torch.equal(c.run(), first) and int(c.gpu_status) == 0


def test_waits_that_run_out_at_once_in_many_launches():
    """Launches without their value tiles one behind the other, on two streams: each ends with its queries and tiles landed, and its
    TMEM given back, so that the launches behind it and beside it are sound."""
    cases = [Case(92 + i, BF, 8, 2, 128, 16, [300 - 200 * i, 40, 5], 9 + 50 * i) for i in range(2)]
    wants = [c.want() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    args = [(c.q.cuda(), c.pages.cuda(), 0, torch.as_tensor(c.tables).cuda(), i32(c.prefix), torch.as_tensor(c.mask).cuda(), c.scale)
            for c in cases]
    torch.cuda.synchronize()
    assert lib().load_library().poss_debug_paged_lose_load(2) == 0
    status = [[torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(3)] for _ in cases]
    torch.cuda.synchronize()
    outs = [[], []]
    for i in range(3):
        for s, a, o, st in zip(streams, args, outs, status):
            with torch.cuda.stream(s):
                o.append(lib().poss_paged_tree_attention(*a, status=st[i]))
    torch.cuda.synchronize()
    assert [[int(x) for x in st] for st in status] == [[6, 0, 0], [6, 0, 0]]
    for c, w, o in zip(cases, wants, outs):
        c.check(o[1], w)
        assert torch.equal(o[2], o[1])


# ------------------------------------------------------------------ remap
def test_a_remap_that_does_not_fit_returns_empty_tables_of_its_own():
    """Too few free pages, and no outputs given: the tables that the call made name no page, its lengths are zero, so that a step
    that runs before n_free has been read writes nothing and is reported."""
    L = lib()
    for n_pages in (4, 13000):                                    # counts in shared memory, and in scratch
        pages = torch.randn(1, n_pages, 2, 2, 16, 64, device="cuda").to(BF)
        tables, lens = i32([[0, 1, -1], [2, -1, -1]]), i32([20, 9])
        refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
        parents, room = i32([0, 0, 1]), i32([12, 12, 30])
        for filler in (1, 2):                                     # whatever torch's allocator hands out next held these
            junk = [torch.full((3, 3), filler, dtype=torch.int32, device="cuda"), torch.full((3,), 5, dtype=torch.int32, device="cuda")]
            del junk
            before = pages.clone()
            r = L.poss_pages_remap(pages, tables, lens, refs, parents, room)
            assert int(r["n_free"]) < 0 and torch.equal(r["refs"], refs) and torch.equal(pages, before)
            assert (r["tables"] == -1).all() and (r["seq_len"] == 0).all()
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            k = torch.ones(3, 1, 2, 64, dtype=BF, device="cuda")
            L.poss_pages_append(k, k, pages, 0, r["tables"], r["seq_len"], status=status)
            assert int(status) == 1 and torch.equal(pages, before)
        # the same in a graph, replayed when it fits and when it does not
        refs[-3:] = 0
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = L.poss_pages_remap(pages, tables, lens, refs, parents, room)
        for fits in (n_pages > 4, False, n_pages > 4):
            refs.fill_(1)
            if fits:
                refs[-3:] = 0
            g.replay()
            torch.cuda.synchronize()
            assert (int(r["n_free"]) >= 0) == fits
            assert r["seq_len"].tolist() == ([20, 20, 9] if fits else [0, 0, 0])
            assert fits or ((r["tables"] == -1).all() and torch.equal(r["refs"], refs))


@pytest.mark.parametrize("dtype,d,batch,scale", [(F32, 32, 295, 0.2), (F32, 32, 296, 0.2), (F32, 32, 297, 0.2), (F32, 128, 7, 0.1),
                                                 (BF, 64, 295, -0.2), (BF, 64, 297, -0.2), (BF, 64, 297, 0.2), (BF, 128, 3, 0.1)])
def test_attention_stays_inside_its_scratch(dtype, d, batch, scale):
    """Either side of the 592 blocks from which on the SIMT kernel leaves no parts; what lies behind the scratch is as it was."""
    c = Case(95, dtype, 2, 2, d, 16, [70] * (batch - 1) + [300], 2)
    c.scale = scale
    need = lib().poss_paged_attention_workspace_bytes(c.pages.cuda(), batch, 2, 2, c.tables.shape[1])
    buf = torch.full((need + 65536,), 0xA5, dtype=torch.uint8, device="cuda")
    got = c.run(workspace=buf[:need])
    assert int(c.gpu_status) == 0 and (buf[need:] == 0xA5).all()
    c.check(got) if scale > 0 else pg.check_attention(got, *c.want(), dtype, False)


@pytest.mark.parametrize("hq,hkv,d,page,prefix,rows,n_rows", [
    (32, 8, 128, 16, [1024], 1, None), (8, 2, 128, 64, [700, 31, 2000], 61, [61, 60, 7]), (8, 2, 64, 32, [300, 0, 17, 129], 25, [25, 1, 24, 13]),
    (4, 1, 64, 256, [257], 128, None), (4, 4, 128, 16, [5000, 63], 3, None), (128, 1, 128, 16, [333], 3, None),
])
def test_tensor_core_attention_keeps_sixteen_bits_of_a_probability(hq, hkv, d, page, prefix, rows, n_rows):
    """The bounds of the plain form without the 2^-8 that a probability in one bf16 would need: 2^-15 of A instead, the cut and the
    rounding of its two parts.  And the bound of the contiguous call: 2^-8 of the element, 2e-3 of the output's RMS."""
    c = Case(96, BF, hq, hkv, d, page, prefix, rows, n_rows)
    got = c.run(out=torch.zeros(c.b, rows, hq, d, dtype=BF, device="cuda"))
    want, tol, big = c.want()
    pg.check_attention(got, want, tol + big * 2.0 ** -15, big, BF, False)
    live = ~torch.isnan(want)
    err, w = (got.double().cpu() - want).abs()[live], want[live]
    assert (err <= 2.0 ** -8 * w.abs() + 2e-3 * w.pow(2).mean().sqrt()).all()


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("rows", [1, 9, 61])
def test_an_infinite_value_of_a_committed_slot_comes_out_as_infinity(d, page, rows):
    """Every row sees it: +inf or -inf in its column whatever the slot's score, the greatest one among them; all else as without it."""
    c = Case(97, BF, 8, 2, d, page, [200, 77], rows)
    want, tol, big = c.want()
    c.q[1] = 0.0                                                  # every slot's score is the row's greatest
    c.pages[0, int(c.tables[0][0]), 1, :, 3, 5] = math.inf
    c.pages[0, int(c.tables[1][0]), 1, :, 7, 9] = -math.inf
    got = c.run().cpu().float()
    assert (got[0, :, :, 5] == math.inf).all() and (got[1, :, :, 9] == -math.inf).all()
    keep = [i for i in range(d) if i != 5]
    pg.check_attention(got[:1, ..., keep], want[:1, ..., keep], tol[:1, ..., keep], big[:1, ..., keep], BF, True)
    assert torch.isfinite(got[1, ..., [i for i in range(d) if i != 9]]).all()


@pytest.mark.parametrize("dtype,d,page", [(BF, 128, 16), (BF, 64, 64), (F32, 64, 24)])
@pytest.mark.parametrize("size", [1e3, 1e6, 2.0 ** 28])
def test_scores_of_any_size_up_to_the_documented_one(dtype, d, page, size):
    """Queries and keys of one column each, so that scores are single products; the greatest one takes all where they lie apart."""
    c = Case(98, dtype, 4, 2, d, page, [150, 3], 9)
    c.q[..., 1:] = 0
    c.pages[:, :, 0, :, :, 1:] = 0
    c.scale = 0.25
    top = max(float(c.q.float().abs().max()) * float(c.pages[:, :, 0].float().abs().max()) * 0.25, 1.0)
    for x in (c.q, c.pages[:, :, 0]):
        x *= 2.0 ** math.floor(0.5 * math.log2(size / top))       # (exact)
    want, tol, big = c.want()
    # the plain bound holds a score error e in exp(e) ~ 1 + e; where e is not small the row's greatest score and the others lie a
    # whole score step apart or tie, and the output is within the sum of both weights' reach: 2 A
    tol = torch.minimum(tol, 2 * big)
    got = c.run()
    assert int(c.gpu_status) == 0
    pg.check_attention(got, want, tol, big, dtype, dtype == BF)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("v", [3, 100, 8192, 50257])
def test_no_continuation_scores_better_than_its_beam(dtype, v):
    """Log-probabilities are 0 at the most, also where one token has nearly all of the probability: the scores of a search never rise."""
    torch.manual_seed(85)
    for spread in (1.0, 30.0, 300.0):
        x = (torch.randn(16, 8, v, device="cuda") * spread).to(dtype)
        x[::2, ::2] += 1000.0
        s = -torch.rand(16, 8, device="cuda")
        r = lib().poss_beam_select(x, s)
        there = r["parents"] >= 0
        assert (r["scores"][there] <= s.view(-1)[r["parents"][there].long()]).all()
