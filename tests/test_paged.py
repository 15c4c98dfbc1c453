"""CPU checks of the paged-cache and beam calls: refusals on the host, the rule that finds a slot's page, and the plain
forms that the GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest
import torch

from tests import paged_util as pg

INVALID, SHAPE, CAPACITY, WORKSPACE = 1, 2, 3, 4
P = 1 << 20       # a non-NULL, aligned address: every call here is refused before a device is touched


@pytest.fixture(scope="module")
def lib():
    from paper_2506_03566_b200 import build as b
    b.build()
    from paper_2506_03566_b200.binding import load_library
    return load_library()


def pool(**kw):
    from paper_2506_03566_b200 import poss_page_pool
    v = dict(n_layers=2, n_pages=64, n_kv_heads=2, page_slots=16, head_dim=64, dtype=1)
    v.update(kw)
    return poss_page_pool(**v)


BAD_POOLS = [(dict(n_layers=0), INVALID), (dict(n_pages=0), INVALID), (dict(n_kv_heads=-1), INVALID),
             (dict(page_slots=0), INVALID), (dict(dtype=2), INVALID), (dict(head_dim=48), SHAPE),
             (dict(page_slots=1025), CAPACITY), (dict(n_pages=1 << 30), CAPACITY)]


def append(lib, p=None, layer=0, pages=P, tables=P, mp=8, batch=2, rows=3, k=P, v=P, ld=128, prefix=P):
    p = p if p is not None else pool()
    return lib.poss_pages_append(C.byref(p), layer, pages, tables, mp, batch, rows, k, v, ld, prefix, None, None, None)


def attend(lib, p=None, layer=0, pages=P, tables=P, mp=8, batch=2, rows=3, hq=4, q=P, ld=256, prefix=P, mask=P, scale=1.0,
           out=P, ws=P, ws_bytes=1 << 30):
    p = p if p is not None else pool()
    return lib.poss_paged_tree_attention(C.byref(p), layer, pages, tables, mp, batch, rows, hq, q, ld, prefix, None, mask,
                                         scale, out, ws, ws_bytes, None, None)


def compact(lib, p=None, pages=P, tables=P, mp=8, batch=2, prefix=P, path=P, acc=P, out=P):
    p = p if p is not None else pool()
    return lib.poss_pages_compact(C.byref(p), pages, tables, mp, batch, prefix, path, acc, out, None, None)


def remap(lib, p=None, pages=P, tables=P, out_tables=2 * P, mp=8, n0=2, n1=2, lens=P, refs=P, out_refs=2 * P, parents=P,
          out_len=P, free=P, ws=P, ws_bytes=1 << 30):
    p = p if p is not None else pool()
    return lib.poss_pages_remap(C.byref(p), pages, tables, out_tables, mp, n0, n1, lens, refs, out_refs, parents, None,
                                out_len, free, ws, ws_bytes, None, None)


def beam(lib, x=P, dtype=0, batch=2, beams=4, vocab=100, scores=P, fin=None, eos=2, tok=P, par=P, sc=P, of=P, ws=P,
         ws_bytes=1 << 30):
    return lib.poss_beam_select(x, dtype, batch, beams, vocab, scores, fin, eos, tok, par, sc, of, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", BAD_POOLS)
def test_bad_pools_are_refused_by_every_call(lib, kw, code):
    p = pool(**kw)
    assert append(lib, p) == code and attend(lib, p) == code and compact(lib, p) == code and remap(lib, p) == code
    assert lib.poss_paged_attention_workspace_bytes(C.byref(p), 1, 1, 2, 1) == 0
    assert lib.poss_pages_remap_workspace_bytes(C.byref(p), 1, 1, 1) == 0


def test_append_refusals(lib):
    for kw in (dict(pages=None), dict(tables=None), dict(k=None), dict(v=None), dict(prefix=None), dict(layer=2),
               dict(layer=-1), dict(mp=0), dict(batch=-1), dict(rows=-1), dict(ld=127), dict(ld=132), dict(k=P + 8),
               dict(v=P + 2), dict(pages=P + 4)):
        assert append(lib, **kw) == INVALID, kw
    assert append(lib, rows=65536) == CAPACITY and append(lib, batch=1025) == CAPACITY
    assert append(lib, mp=1 << 27) == CAPACITY
    assert append(lib, batch=0) == 0 and append(lib, rows=0) == 0


def test_attention_refusals(lib):
    nan, inf = float("nan"), float("inf")
    for kw in (dict(pages=None), dict(tables=None), dict(q=None), dict(prefix=None), dict(mask=None), dict(out=None),
               dict(layer=2), dict(mp=0), dict(batch=-1), dict(rows=-1), dict(hq=0), dict(ld=255), dict(ld=260),
               dict(scale=nan), dict(scale=inf), dict(q=P + 8), dict(out=P + 8), dict(pages=P + 8)):
        assert attend(lib, **kw) == INVALID, kw
    assert attend(lib, hq=5) == SHAPE
    assert attend(lib, rows=129) == CAPACITY and attend(lib, batch=1025) == CAPACITY
    need = lib.poss_paged_attention_workspace_bytes(C.byref(pool()), 2, 3, 4, 8)
    assert need > 0 and need % 256 == 0
    assert attend(lib, ws=None) == WORKSPACE and attend(lib, ws=P + 16) == WORKSPACE
    assert attend(lib, ws_bytes=need - 1) == WORKSPACE
    assert attend(lib, batch=0) == 0 and attend(lib, rows=0) == 0


@pytest.mark.parametrize("kw", [dict(), dict(dtype=0), dict(page_slots=24), dict(head_dim=128), dict(head_dim=32)])
def test_attention_scratch_made_for_the_largest_call_serves_the_smaller_ones(lib, kw):
    p = pool(**kw)
    size = lambda *a: lib.poss_paged_attention_workspace_bytes(C.byref(p), *a)
    for hq in (2, 8, 14):
        for mp in (1, 3, 64):
            last = 0
            for batch in (1, 2, 3, 7, 16, 64, 300):
                assert size(batch, 5, hq, mp) >= last
                last = size(batch, 5, hq, mp)
            last = 0
            for rows in range(1, 129):
                assert size(3, rows, hq, mp) >= last
                last = size(3, rows, hq, mp)
        assert size(3, 5, hq, 2) <= size(3, 5, hq, 9)
    assert size(1, 0, 2, 1) == 0 and size(1, 129, 2, 1) == 0 and size(0, 1, 2, 1) == 0 and size(1, 1, 3, 1) == 0


def test_compact_refusals(lib):
    for kw in (dict(pages=None), dict(tables=None), dict(prefix=None), dict(path=None), dict(acc=None), dict(out=None),
               dict(mp=0), dict(batch=-1), dict(pages=P + 8)):
        assert compact(lib, **kw) == INVALID, kw
    assert compact(lib, batch=1025) == CAPACITY and compact(lib, batch=0) == 0


def test_remap_refusals(lib):
    for kw in (dict(pages=None), dict(tables=None), dict(out_tables=None), dict(lens=None), dict(refs=None),
               dict(out_refs=None), dict(out_len=None), dict(free=None), dict(mp=0), dict(n0=-1), dict(n1=-1),
               dict(out_tables=P), dict(out_refs=P), dict(parents=None, n1=3), dict(pages=P + 8)):
        assert remap(lib, **kw) == INVALID, kw
    assert remap(lib, n0=1025) == CAPACITY and remap(lib, n1=1025) == CAPACITY
    need = lib.poss_pages_remap_workspace_bytes(C.byref(pool()), 2, 2, 8)
    assert need > 0 and need % 256 == 0
    assert remap(lib, ws_bytes=need - 1) == WORKSPACE and remap(lib, ws=P + 8) == WORKSPACE and remap(lib, ws=None) == WORKSPACE


def test_beam_refusals(lib):
    for kw in (dict(x=None), dict(scores=None), dict(tok=None), dict(par=None), dict(sc=None), dict(of=None), dict(dtype=3),
               dict(batch=-1), dict(beams=0), dict(vocab=0), dict(eos=100), dict(fin=P, eos=-1), dict(x=P + 4)):
        assert beam(lib, **kw) == INVALID, kw
    assert beam(lib, beams=17) == CAPACITY and beam(lib, batch=65535) == CAPACITY
    need = lib.poss_beam_select_workspace_bytes(2, 4, 100)
    assert need > 0 and beam(lib, ws_bytes=need - 1) == WORKSPACE and beam(lib, ws=P + 8) == WORKSPACE
    assert beam(lib, batch=0) == 0
    assert lib.poss_beam_select_workspace_bytes(1, 17, 5) == 0 and lib.poss_beam_select_workspace_bytes(0, 1, 5) == 0


def test_page_of_a_slot_never_leaves_the_table_or_the_pool(lib):
    table = (C.c_int32 * 5)(3, 9, -1, 10, 2147483647)
    page, off = C.c_int(), C.c_int()

    def at(slot, n_pages=10, slots=16):
        assert lib.poss_debug_page_of_slot(table, 5, slots, n_pages, slot, C.byref(page), C.byref(off)) == 0
        return page.value, off.value

    assert at(0) == (3, 0) and at(15) == (3, 15) and at(16) == (9, 0)
    assert at(33) == (-1, 1)                                   # a negative entry
    assert at(48) == (-1, 0) and at(48, n_pages=11) == (10, 0)  # the first page behind the pool
    assert at(64)[0] == -1 and at(80)[0] == -1 and at(1 << 40)[0] == -1 and at(-1)[0] == -1
    assert at(7, slots=3) == (-1, 1)
    assert lib.poss_debug_page_of_slot(None, 5, 16, 10, 0, C.byref(page), C.byref(off)) == INVALID
    assert lib.poss_debug_page_of_slot(table, 0, 16, 10, 0, C.byref(page), C.byref(off)) == INVALID


def test_plain_attention_agrees_with_a_dense_softmax():
    rng = np.random.default_rng(3)
    gen = torch.Generator().manual_seed(3)
    b, r, hq, hkv, d, page = 2, 5, 4, 2, 32, 3
    prefix, rows = [7, 0], [5, 3]
    tables = pg.make_tables(rng, [p + n for p, n in zip(prefix, rows)], page, 20, 9)
    _, anc = pg.tree_masks(rng, b, r)
    pages = torch.randn(20, 2, hkv, page, d, generator=gen)
    q = torch.randn(b, r, hq, d, generator=gen)
    out, tol, big = pg.attention(q, pages, tables, prefix, rows, anc, 0.3)
    for i in range(b):
        n = prefix[i] + rows[i]
        dense = torch.stack([pages[int(tables[i][s // page]), :, :, s % page] for s in range(n)]).double()
        for x in range(rows[i]):
            seen = torch.tensor([s < prefix[i] or bool(anc[i][x][s - prefix[i]]) for s in range(n)])
            for h in range(hq):
                s = (dense[:, 0, h // 2] @ q[i, x, h].double() * 0.3).masked_fill(~seen, -np.inf)
                assert torch.allclose(out[i, x, h], torch.softmax(s, 0) @ dense[:, 1, h // 2])
    assert torch.isnan(out[1, 3:]).all() and (tol >= 0).all() and (big + 1e-12 >= out.nan_to_num().abs()).all()


def test_plain_remap_keeps_its_own_promises():
    """Many random steps: counts equal the holders, written pages have one, kept slots are found again."""
    rng = np.random.default_rng(5)
    page, n_pages, mp, n = 4, 60, 12, 6
    refs = np.zeros(n_pages, np.int32)
    refs[7] = 1                                                 # pinned from outside
    tables = np.full((n, mp), -1, np.int32)
    lens = np.zeros(n, np.int32)
    content = {}
    names = [[] for _ in range(n)]
    step = 0
    for _ in range(200):
        parents = [int(rng.integers(-1, n)) for _ in range(n)]
        room = [int(rng.integers(0, 9)) for _ in range(n)]
        cut = np.array([int(rng.integers(max(0, x - 5), x + 1)) for x in lens], np.int32)
        got, missing = pg.remap(tables, cut, refs, parents, room, page)
        if got is None:
            assert missing > 0
            tables[:], lens[:], names = -1, 0, [[] for _ in range(n)]
            refs[:] = 0
            refs[7] = 1
            continue
        names = [names[p][:cut[p]] if p >= 0 else [] for p in parents]
        tables, refs, lens, free, copies = got
        for src, dst, m in copies:
            for s in range(m):
                content[dst, s] = content[src, s]
        held = np.bincount(tables[tables >= 0].ravel(), minlength=n_pages)
        held[7] += 1
        assert np.array_equal(held, refs) and free == int((refs == 0).sum())
        for i in range(n):
            for s, x in enumerate(names[i]):
                assert content[tables[i][s // page], s % page] == x
            more = int(rng.integers(0, room[i] + 1))
            for s in range(lens[i], lens[i] + more):
                assert refs[tables[i][s // page]] == 1
                content[tables[i][s // page], s % page] = step
                names[i].append(step)
                step += 1
            lens[i] += more


def test_the_binding_names_what_is_wrong(lib):
    """Refusals that need no device: what is no tensor, or none on the current device, and shapes that no call takes."""
    from paper_2506_03566_b200 import (poss_beam_select, poss_paged_attention_workspace_bytes, poss_paged_tree_attention,
                                       poss_pages_append, poss_pages_compact, poss_pages_remap)
    pages, ints = torch.zeros(1, 3, 2, 2, 16, 64), torch.zeros(2, 3, dtype=torch.int32)
    calls = (lambda x: poss_pages_append(x, x, x, 0, ints, ints[:, 0]),
             lambda x: poss_paged_tree_attention(x, x, 0, ints, ints[:, 0], ints, 1.0),
             lambda x: poss_pages_compact(x, ints, ints[:, 0], ints, ints[:, 0]),
             lambda x: poss_pages_remap(x, ints, ints[:, 0], ints[:, 0]))
    for f in calls:
        for x, word in ((pages, "current device"), (pages[0], "six dimensions"), (pages[..., ::2], "six dimensions"),
                        (pages[:, :, :1], "six dimensions"), (pages[:, :, :1].contiguous(), "kv heads"), (pages.half(), "bf16 or fp32"), ("pages", "got str"), (None, "got NoneType")):
            with pytest.raises(ValueError, match="kv_pages.*" + word):
                f(x)
    for x, word in ((torch.zeros(1, 2, 5), "current device"), (torch.zeros(2, 5), "vocab"), (torch.zeros(1, 2, 5).half(), "fp32 or bf16"),
                    (3, "got int"), (torch.zeros(1, 2, 5).to_sparse(), "dense")):
        with pytest.raises(ValueError, match="logits.*" + word):
            poss_beam_select(x, torch.zeros(1, 2))
    with pytest.raises(TypeError):
        poss_beam_select(torch.zeros(1, 2, 5))
    with pytest.raises(ValueError, match="kv_pages"):
        poss_paged_attention_workspace_bytes(pages.half(), 1, 1, 2, 1)


def test_outputs_that_overlap_inputs_are_refused(lib):
    """Everything else is in order: only the addresses meet.  (Distinct ones are used for all the others.)"""
    at = lambda i: P + (i << 24)
    for kw in (dict(out=at(1)), dict(out=at(1) + 4), dict(out=at(2) + 40), dict(out=at(3) - 4), dict(out=at(4))):
        args = dict(pages=at(0), prefix=at(1), path=at(2), acc=at(3), tables=at(4), out=at(5))
        assert compact(lib, **{**args, **kw}) == INVALID, kw
    outs, ins = ("out_tables", "out_refs", "out_len", "free"), ("tables", "refs", "lens", "parents")
    names = outs + ins
    args = dict(pages=at(0), ws=at(20), **{x: at(i + 1) for i, x in enumerate(names)})
    for o in outs:
        for x in names:
            if x != o:
                assert remap(lib, **{**args, o: args[x]}) == INVALID, (o, x)
    assert attend(lib, q=at(1), out=at(1), pages=at(0), ws=at(5), ld=512) == INVALID
    assert attend(lib, q=at(1), out=at(1) + 5 * 1024 + 496, pages=at(0), ws=at(5), ld=512) == INVALID      # the last row's end
    assert attend(lib, q=at(1), out=at(1) - 6 * 512 + 16, pages=at(0), ws=at(5), ld=512) == INVALID
    b = dict(x=at(0), scores=at(1), fin=at(2), tok=at(3), par=at(4), sc=at(5), of=at(6), ws=at(7))
    for kw in (dict(tok=at(1)), dict(par=at(2)), dict(sc=at(1) + 4), dict(sc=at(2)), dict(of=at(2) - 4), dict(of=at(1)),
               dict(par=at(3)), dict(of=at(5) + 28)):
        assert beam(lib, **{**b, **kw}) == INVALID, kw


def test_attention_refuses_more_units_than_it_can_count(lib):
    p = pool(n_pages=1 << 20, page_slots=128, head_dim=128)
    at = lambda i: P + (i << 24)
    args = dict(pages=at(0), tables=at(1), q=at(2), prefix=at(3), mask=at(4), out=at(40), ws=at(80), ws_bytes=1 << 40)
    # 1024 sequences x 2 heads x 1 item x 2^20 tiles of 64 slots = 2^31
    assert attend(lib, p, batch=1024, rows=3, hq=4, ld=512, mp=1 << 19, **args) == CAPACITY
