"""GPU tests of the rare paths of the slot weights, the eviction and the token scores."""
import math

import numpy as np
import pytest
import torch

from tests import long_util as lu
from tests.test_gpu_long_context import bits, check_mass, evict_case, graph_of, mass_case, run_mass
from tests.test_gpu_paged import BF, F32, Case, cu, i32, lib
from tests.test_gpu_token_scores import check

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ slot weights
@pytest.mark.parametrize("hq,hkv,d,rows", [(4, 2, 64, 20), (32, 8, 128, 3)])
def test_many_sequences_most_of_them_without_rows(hq, hkv, d, rows):
    """More sequences than a warp has lanes, with gaps: where the cut of the work finds its places."""
    rng = np.random.default_rng(3)
    prefix = [int(x) for x in rng.integers(0, 200, 100)]
    n_rows = [int(x) if i % 3 == 0 else 0 for i, x in enumerate(rng.integers(1, rows + 1, 100))]
    n_rows[0:40] = [0] * 40
    c = Case(91, BF, hq, hkv, d, 16, prefix, rows, n_rows)
    mass, w = mass_case(c, 1)
    got = mass.cuda()
    out = torch.zeros(100, rows, hq, d, dtype=BF, device="cuda")
    run_mass(c, got, w, out=out)
    check_mass(c, got, mass, w)
    c.check(out)


@pytest.mark.parametrize("hq,hkv,d,page,prefix,rows", [
    (16, 2, 128, 128, [4000, 3900], 128),          # 1024 lines: four passes over a CTA's slots
    (24, 2, 64, 32, [2050], 40),                   # 480 lines, of twelve heads: a pass's last lines are no whole row
    (9, 1, 64, 16, [1000], 57),                    # 513: one line in the third pass
    (40, 8, 128, 64, [1500, 10], 6),               # 30 lines: the attention's own scores
    (33, 1, 128, 16, [900], 1),                    # 33: just too many for them
    (16, 1, 64, 16, [900, 2], 1), (17, 1, 64, 16, [900, 2], 1),   # the same bounds with half the elements
])
def test_passes_and_routes(hq, hkv, d, page, prefix, rows):
    c = Case(93, BF, hq, hkv, d, page, prefix, rows)
    mass, w = mass_case(c, 2)
    got, out = mass.cuda(), None
    out = run_mass(c, got, w)
    assert int(c.gpu_status) == 0
    check_mass(c, got, mass, w)
    assert torch.equal(bits(out), bits(c.run()))


def test_a_table_with_room_for_far_more_slots():
    """Scores of so many slots are not kept: the keys are read again, with the same weights."""
    c = Case(95, BF, 32, 8, 128, 256, [700], 1, extra_places=16400)
    assert c.tables.shape[1] * 256 > 2 ** 22
    mass = torch.zeros(1, 1, 8, c.tables.shape[1] * 256, device="cuda")
    small = torch.zeros(1, 1, 8, 1024, device="cuda")
    run_mass(c, mass, None)
    run_mass(c, small, None, tables=c.tables[:, :4].copy())
    want, tol = lu.slot_weights(c.q, c.pages[0], c.tables, c.prefix, c.n_rows, c.anc, c.scale, None, torch.zeros(1, 8, 1024))
    lu.check_close(mass[0, :, :, :1024], want, tol, F32)
    lu.check_close(small[0], want, tol, F32)
    assert not mass[0, 0, :, 701:].any()


@pytest.mark.parametrize("dtype,d", [(F32, 32), (F32, 128), (BF, 32)])
def test_a_table_with_room_for_far_more_slots_off_the_tensor_cores(dtype, d):
    c = Case(96, dtype, 32, 8, d, 1024, [50], 128, [90], extra_places=40)
    assert c.tables.shape[1] * 1024 * 32 * 128 * 4 > 2 ** 29
    mass, w = mass_case(c, 5)
    got = mass.cuda()
    run_mass(c, got, w)
    check_mass(c, got, mass, w)
    c.tables = c.tables[:, :2].copy()                                 # and one without: the attention's own scores
    mass = mass[..., :2048].contiguous()
    got = mass.cuda()
    run_mass(c, got, w)
    check_mass(c, got, mass, w)


def test_lost_loads_run_out_and_the_context_lives_on():
    c = Case(97, BF, 8, 2, 128, 16, [300, 5], 40)
    mass, w = mass_case(c, 4)
    want = mass.cuda()
    out = run_mass(c, want, w).clone()
    assert lib().load_library().poss_debug_paged_lose_load(2) == 0        # the attention's and the weights' launch
    run_mass(c, mass.cuda(), w)
    assert int(c.gpu_status) == 6
    got = mass.cuda()
    assert torch.equal(run_mass(c, got, w), out) and torch.equal(got, want)
    assert int(c.gpu_status) == 0


@pytest.mark.parametrize("heads,d", [((8, 2), 128), ((4, 4), 64)])
def test_a_lost_load_of_the_weights_alone_raises_the_status(heads, d):
    """The attention of the call goes on; the launch that forms weights from the keys waits for its queries in vain and says so."""
    c = Case(98, BF, *heads, d, 16, [700, 5], 40)
    mass, w = mass_case(c, 4)
    want = mass.cuda()
    out = run_mass(c, want, w).clone()
    assert int(c.gpu_status) == 0
    assert lib().load_library().poss_debug_paged_lose_load_after(1, 1) == 0
    got = run_mass(c, mass.cuda(), w)
    assert int(c.gpu_status) == 6 and torch.equal(bits(got), bits(out))
    again = mass.cuda()
    assert torch.equal(bits(run_mass(c, again, w)), bits(out)) and torch.equal(again, want) and int(c.gpu_status) == 0
    # both launches have been counted: one spared, one that lost its load
    assert lib().load_library().poss_debug_paged_lose_load_after(2, 0) == 0
    assert torch.equal(bits(run_mass(c, mass.cuda(), w)), bits(out)) and int(c.gpu_status) == 0


@pytest.mark.parametrize("hkv,d,page", [(2, 128, 16), (20, 64, 1)])
def test_commit_in_bf16_takes_the_weights_along(hkv, d, page):
    """Paths of every length up to the longest, across pages; more heads than a block has warps."""
    c = Case(99, BF, 2 * hkv, hkv, d, page, [15, 0, 100], 40)
    mass, _ = mass_case(c, 6)
    path, acc = np.zeros((3, 17), np.int32), [16, 1, 0]
    path[0, 1:17] = [1, 2, 4, 5, 7, 9, 12, 13, 17, 20, 22, 30, 31, 33, 38, 39]
    path[1, 1] = 39
    a, b, gm = c.pages.cuda(), c.pages.cuda(), mass.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    n1 = lib().poss_pages_compact(a, cu(c.tables), i32(c.prefix), cu(path), i32(acc))
    n2 = lib().poss_pages_compact(b, cu(c.tables), i32(c.prefix), cu(path), i32(acc), mass=gm, status=status)
    assert torch.equal(a, b) and n1.cpu().tolist() == n2.cpu().tolist() == [32, 2, 101] and int(status) == 0
    want = mass.clone()
    for i in range(3):
        for k in range(1, acc[i] + 1):
            want[:, i, :, c.prefix[i] + k] = mass[:, i, :, c.prefix[i] + int(path[i, k])]
    assert torch.equal(gm.cpu(), want)


# ------------------------------------------------------------------ eviction
@pytest.mark.parametrize("kind", ["ties", "equal", "random", "rising"])
def test_eviction_of_long_sequences(kind):
    """Several chunks of slots per block: equal weights that stay and go in different chunks, in place."""
    lens, keep = [20000, 8193, 8192, 16385], [12345, 8192, 1, 16000]
    pages, mass, tables = evict_case(17, BF, 1, 1, 32, 64, lens, kind)
    want = lu.evict(pages, mass, mass, tables, lens, keep, 1, 0)
    gp, gm = pages.cuda(), mass.cuda()
    n = lib().poss_pages_evict(gp, gm, cu(tables), i32(lens), i32(keep), first=1)
    assert torch.equal(gp.cpu(), want[0]) and torch.equal(gm.cpu(), want[1]) and n.cpu().tolist() == want[2].tolist()


def test_eviction_at_once_on_two_streams():
    lens, keep = [500, 300], [200, 100]
    pages, mass, tables = evict_case(19, F32, 2, 2, 32, 16, lens, "random")
    want = lu.evict(pages, mass, mass, tables, lens, keep, 2, 2)
    sets = [(pages.cuda(), mass.cuda()) for _ in range(2)]
    t, a, b = cu(tables), i32(lens), i32(keep)
    torch.cuda.synchronize()
    for gp, gm in sets:
        with torch.cuda.stream(torch.cuda.Stream()):
            lib().poss_pages_evict(gp, gm, t, a, b, first=2, recent=2)
    torch.cuda.synchronize()
    for gp, gm in sets:
        assert torch.equal(gp.cpu(), want[0]) and torch.equal(gm.cpu(), want[1])


@pytest.mark.parametrize("dtype,layers,hkv,d", [(BF, 2, 2, 64), (F32, 1, 3, 32)])
def test_eviction_of_forks_and_pinned_prefixes(dtype, layers, hkv, d):
    """With the holders of every page, a sequence that would write to a page of another holder keeps its slots, in every layer and head."""
    pages, _, tables = evict_case(23, dtype, layers, hkv, d, 16, [100, 60], "random")
    pages = torch.cat([pages, torch.zeros_like(pages[:, :4])], 1)             # (room for the forks' own pages)
    refs = np.zeros(pages.shape[1], np.int32)
    refs[tables[tables >= 0]] = 1
    gp, status = pages.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    forks = lib().poss_pages_remap(gp, cu(tables), i32([100, 60]), i32(refs), parents=i32([0, 0, 1]), room=i32([0, 0, 0]))
    t, held = forks["tables"], forks["refs"]
    tab, lens, start = t.cpu().numpy(), [100, 100, 60], gp.cpu()
    assert int(forks["n_free"]) >= 0 and (tab[0, :6] == tab[1, :6]).all() and tab[0, 6] != tab[1, 6]
    mass = torch.rand(layers, 3, hkv, tab.shape[1] * 16, generator=torch.Generator().manual_seed(2))
    gm = mass.cuda()

    def cut(keep, first, recent, want_len, refs=held, raised=0):
        status.zero_()
        to = torch.full_like(gm, 9.0)
        n = lib().poss_pages_evict(gp, gm, t, i32(lens), i32(keep), first=first, recent=recent, out_mass=to, status=status, refs=refs)
        assert n.cpu().tolist() == want_len and int(status) == raised
        ok = [i for i in range(3) if want_len[i] == min(lens[i], keep[i])]
        want = lu.evict(start, mass[:, ok], torch.full_like(mass[:, ok], 9.0), tab[ok], [lens[i] for i in ok], [keep[i] for i in ok], first, recent)
        assert torch.equal(bits(gp.cpu()), bits(want[0])) and torch.equal(to[:, ok].cpu(), want[1])
        assert all((to[:, i] == 9).all() for i in range(3) if i not in ok)
        gp.copy_(start)

    cut([40, 99, 30], 2, 4, [100, 100, 30], raised=1)                 # both siblings' shared pages stay as they were
    cut([98, 97, 60], 96, 1, [98, 97, 60])                            # what they share ends before the first place that changes
    cut([98, 97, 60], 95, 1, [100, 100, 60], raised=1)                # the place before lies in a shared page
    cut([95, 100, 60], 95, 0, [95, 100, 60])                          # none changes
    pinned = held.clone()
    pinned[int(tab[2, 1])] += 1                                       # slots 16 to 31 of the third
    cut([100, 100, 16], 4, 4, [100, 100, 16], refs=pinned)            # (its places end before them)
    cut([100, 100, 17], 4, 4, [100, 100, 60], refs=pinned, raised=1)
    cut([100, 100, 40], 32, 4, [100, 100, 40], refs=pinned)
    alone = lib().poss_pages_remap(gp, t, i32(lens), held, parents=i32([0, -1, 2]))
    assert torch.equal(alone["tables"][0], t[0]) and int(alone["refs"].max()) == 1
    t, tab, lens = alone["tables"], alone["tables"].cpu().numpy(), [100, 0, 60]
    cut([40, 5, 30], 2, 4, [40, 0, 30], refs=alone["refs"])           # the sibling has gone: the pages are its own
    # a captured call goes by the holders of its replay
    live, out = alone["refs"].clone(), torch.zeros(3, dtype=torch.int32, device="cuda")
    live[int(tab[0, 0])] = 2
    n0, keep = i32(lens), i32([40, 0, 30])
    g = graph_of(lambda: lib().poss_pages_evict(gp, gm, t, n0, keep, first=2, recent=4, out_mass=torch.empty_like(gm), out_len=out, refs=live))
    gp.copy_(start)
    g.replay()
    assert out.cpu().tolist() == [100, 0, 30]
    live[int(tab[0, 0])] = 1
    gp.copy_(start)
    g.replay()
    assert out.cpu().tolist() == [40, 0, 30]
    with pytest.raises(ValueError, match="refs"):
        lib().poss_pages_evict(gp, gm, t, n0, keep, refs=live[1:])


# ------------------------------------------------------------------ token scores
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,vocab", [(2, 40000), (600, 40000), (1, 128256)])
def test_lists_that_overflow(dtype, rows, vocab):
    """Logits that rise, that are equal, that begin low or banned by the thousand: more candidates than a list holds."""
    gen = torch.Generator().manual_seed(8)
    x = torch.empty(rows, vocab, dtype=dtype)
    base = torch.randn(vocab, generator=gen)
    kinds = [torch.arange(vocab) / 100.0, torch.full((vocab,), 2.0), torch.cat([torch.full((16384,), -math.inf), base[16384:]]),
             torch.cat([base[:9000] - 30.0, base[9000:] + 30.0]), torch.where(torch.rand(vocab, generator=gen) < 0.001, base, -math.inf)]
    for r in range(rows):
        x[r] = kinds[r % len(kinds)].to(dtype) if r < 10 else base.to(dtype)
    few = min(rows, 12)
    got = lib().poss_token_logprobs(x.cuda(), i32([vocab - 1] * rows), topk=16)
    want = lu.scores(x[:few].double(), [vocab - 1] * few, None, 16, 1.0)
    lu.check_scores({k: v[:few] for k, v in got.items()}, want)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_logits_far_apart_within_a_row(dtype):
    """One logit above all by hundreds, late in the row; steps between magnitudes that fp32 holds exactly and those it does not; NaN beside them."""
    x = torch.zeros(6, 30000)
    x[0, 29999] = 500.0
    x[1, :100] = 1e30
    x[2, 15000] = 1e30
    x[3] = torch.linspace(-2000, 2000, 30000)
    x[4, 20000:] = 3e5
    x[4, 5] = math.nan
    x[5, ::3] = 1e6
    x[5, 1::3] = -math.inf
    for t in (1.0, 0.2, 30.0):
        check(x.to(dtype), [29999, 0, 15000, 29998, 25000, 3], None, 3, t)
