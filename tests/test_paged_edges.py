"""CPU checks at the edges of the paged calls: refusals of the remapping into new outputs."""
import ctypes as C

import pytest

from tests.test_paged import CAPACITY, INVALID, P, WORKSPACE, lib, pool  # noqa: F401  (lib: the library, a fixture)

at = lambda i: P + (i << 24)


@pytest.mark.parametrize("kw,code", [
    (dict(), None), (dict(kv_pages=None), INVALID), (dict(refs=None), INVALID), (dict(out_len=None), INVALID),
    (dict(out_tables=at(1)), INVALID), (dict(out_refs=at(5)), INVALID), (dict(n_before=-1), INVALID), (dict(parents=None, n_after=3), INVALID),
    (dict(n_after=1025), CAPACITY), (dict(ws=at(20) + 8), WORKSPACE), (dict(ws=None), WORKSPACE), (dict(ws_bytes=255), WORKSPACE),
])
def test_a_remap_into_new_outputs_refuses_what_the_other_refuses(lib, kw, code):  # noqa: F811
    a = dict(kv_pages=at(0), tables=at(1), out_tables=at(2), max_pages=8, n_before=2, n_after=2, seq_len=at(4), refs=at(5), out_refs=at(6),
             parents=at(7), room=None, out_len=at(8), out_free=at(9), ws=at(20), ws_bytes=1 << 30)
    a.update(kw)
    p = pool()
    if code is None:                                              # (in order: nothing here may launch it)
        a["ws_bytes"] = lib.poss_pages_remap_workspace_bytes(C.byref(p), 2, 2, 8) - 1
        code = WORKSPACE
    for f in (lib.poss_pages_remap, lib.poss_pages_remap_fresh):
        assert f(C.byref(p), *list(a.values()), None, None) == code


@pytest.mark.parametrize("kw", [dict(), dict(dtype=0), dict(page_slots=24), dict(head_dim=128), dict(head_dim=32)])
def test_attention_scratch_holds_the_parts_that_are_made_and_stays_small(lib, kw):  # noqa: F811
    """Parts are made where less than 592 blocks of 32 query rows would run: at most 64 for each, at most 592 + blocks in all.  Calls
    of more blocks make none, so that scratch is bounded however large the call is: by those 1183 parts of 32 rows, or by the
    tensor-core kernel's two partials of 256 rows for each of 160 CTAs and its plan."""
    p = pool(**kw)
    size = lambda b, r, hq, mp: lib.poss_paged_attention_workspace_bytes(C.byref(p), b, r, hq, mp)
    row = (p.head_dim + 2) * 4
    for hq in (2, 6, 16, 80):
        for batch in (1, 2, 5, 37, 150, 293, 294, 600, 1024):
            for rows in (1, 3, 33, 128):
                for mp in (1, 2, 9, 4000):
                    blocks = batch * 2 * -(-rows * (hq // 2) // 32)
                    parts = min(-(-592 // blocks), -(-mp * p.page_slots // 32), 64)
                    n = size(batch, rows, hq, mp)
                    assert n >= (blocks * parts * 32 * row if parts > 1 else 1)
                    assert n <= max(1183 * 32 * row, 160 * 2 * 256 * row + 8192) + 256


def test_the_module_of_the_calls_is_built_anew_for_another_torch(lib, monkeypatch):  # noqa: F811
    """It reaches into torch's C++ by layout: neither the build nor the package goes on with one built for another version."""
    import torch
    from paper_2506_03566_b200 import build, paged
    assert not build._calls_stale([])
    assert paged._calls().built_with_torch == build._torch_version()
    monkeypatch.setattr(torch, "__version__", "1.2.3")
    assert build._calls_stale([])
    monkeypatch.setattr(paged, "_module", None)
    with pytest.raises(ImportError, match="1.2.3.*build"):
        paged._calls()


@pytest.mark.parametrize("heads", [1 << 26, (1 << 31) - 2, 1 << 20])
def test_attention_counts_its_query_tiles_in_64_bits(lib, heads):  # noqa: F811
    """rows times query heads past 2^31 are more tiles than a launch has room for, and no small number of them."""
    a = [at(0), at(1), 8, 1, 128, heads, at(2), heads * 64, at(3), None, at(4), 1.0, at(5) + (1 << 50), at(90), 1 << 60, None, None]
    p = pool()
    assert lib.poss_paged_tree_attention(C.byref(p), 0, *a) == CAPACITY
    assert lib.poss_paged_attention_workspace_bytes(C.byref(p), 1, 128, heads, 8) >= 592 * 32 * 66 * 4
