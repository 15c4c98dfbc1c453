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
