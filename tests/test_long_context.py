"""CPU tests: the plain forms against one another, rotary frequencies, and refusals of the rotary, slot-weight, eviction and token-score
calls, which are decided on the host before a device is touched."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from tests import long_util as lu

FAKE = 1 << 20          # an aligned address that no call may follow


@pytest.fixture(scope="module")
def lib():
    from paper_2506_03566_b200 import build as b
    b.build()
    from paper_2506_03566_b200.binding import load_library
    return load_library()


def pool(layers=2, pages=64, heads=2, slots=16, d=64, dtype=1):
    from paper_2506_03566_b200.binding import poss_page_pool
    return C.byref(poss_page_pool(layers, pages, heads, slots, d, dtype))


@pytest.mark.parametrize("scaling,kw", [
    (None, {}), ("linear", {"factor": 4.0}), ("base", {"factor": 8.0}),
    ("bands", {"factor": 8.0, "low": 1.0, "high": 4.0, "original_len": 8192.0}),
    ("ramp", {"factor": 16.0, "low": 1.0, "high": 32.0, "original_len": 4096.0}),
    ("ramp", {"factor": 2.0, "low": 1.0, "high": 1.001, "original_len": 64.0}),
])
@pytest.mark.parametrize("rot_dim,theta", [(4, 10000.0), (24, 10000.0), (128, 500000.0)])
def test_frequencies(scaling, kw, rot_dim, theta):
    import paper_2506_03566_b200 as p
    got = p.poss_rotary_frequencies(rot_dim, theta, scaling, device="cpu", **kw)
    want = torch.tensor(lu.frequencies(rot_dim, theta, scaling, **kw), dtype=torch.float64)
    assert got.dtype == torch.float64 and torch.allclose(got, want, rtol=1e-12, atol=0)   # 64-bit powers and logarithms
    assert (got[1:] < got[:-1]).all() and got[0] <= 1.0
    if scaling in ("bands", "ramp"):
        plain = torch.tensor(lu.frequencies(rot_dim, theta), dtype=torch.float64)
        assert (got <= plain * (1 + 1e-12)).all() and (got >= plain / kw["factor"] * (1 - 1e-12)).all()


def test_frequency_refusals(lib):
    import paper_2506_03566_b200 as p
    out = (C.c_double * 256)()
    ok = [64, 10000.0, 0, 1.0, 1.0, 4.0, 100.0]
    assert lib.poss_rotary_frequencies(out, *ok) == 0
    assert lib.poss_rotary_frequencies(None, *ok) == 1
    for at, value, code in [(0, 63, 1), (0, 0, 1), (0, 514, 3), (1, 1.0, 1), (1, math.inf, 1), (1, math.nan, 1), (2, 5, 1), (2, -1, 1)]:
        a = list(ok)
        a[at] = value
        assert lib.poss_rotary_frequencies(out, *a) == code, (at, value)
    for scaling in (1, 2, 3, 4):
        for factor in (0.5, math.nan, math.inf):
            assert lib.poss_rotary_frequencies(out, 64, 10000.0, scaling, factor, 1.0, 4.0, 100.0) == 1
    for low, high, length in [(0.0, 4.0, 100.0), (4.0, 4.0, 100.0), (1.0, math.inf, 100.0), (1.0, 4.0, 0.0), (1.0, 4.0, math.nan)]:
        assert lib.poss_rotary_frequencies(out, 64, 10000.0, 3, 2.0, low, high, length) == 1
        assert lib.poss_rotary_frequencies(out, 64, 10000.0, 4, 2.0, low, high, length) == 1
    assert lib.poss_rotary_frequencies(out, 2, 10000.0, 2, 2.0, 1.0, 4.0, 100.0) == 1
    with pytest.raises(ValueError):
        p.poss_rotary_frequencies(64, 1e4, "other", device="cpu")
    with pytest.raises(ValueError):
        p.poss_rotary_frequencies(1024, 1e4, device="cpu")
    with pytest.raises(p.PossError):
        p.poss_rotary_frequencies(7, 1e4, device="cpu")


def refused(call, good, changes, done=0):
    """Every change of one argument (by place) gives its code; a `None` place: the whole call as it is must not get past the host."""
    for at, value, code in changes:
        a = list(good)
        a[at] = value
        assert call(*a) == code, (at, value)


def test_rotary_refusals(lib):
    # x, ld, out, ld_out, dtype, n, heads, d, positions, freq, rot, interleaved, magnitude, stream
    good = [FAKE, 512, FAKE + (1 << 24), 512, 1, 10, 8, 64, FAKE, FAKE, 64, 0, 1.0, None]
    refused(lib.poss_rotary, good, [
        (0, None, 1), (0, FAKE + 2, 1), (1, 511, 1), (1, 513, 1), (2, None, 1), (2, FAKE + 512, 1), (2, FAKE + 16, 1),
        (3, 504, 1), (4, 2, 1), (5, -1, 1), (5, 1 << 31, 3), (6, 0, 1), (7, 60, 2), (7, 0, 1), (8, None, 1), (9, None, 1),
        (10, 66, 1), (10, 63, 1), (10, 0, 1), (12, math.nan, 1), (12, math.inf, 1)])
    assert lib.poss_rotary(*[0 if i == 5 else a for i, a in enumerate(good)]) == 0                  # no rows
    assert lib.poss_rotary(FAKE, 1024, FAKE + (1 << 24), 1024, 1, 10, 1, 1024, FAKE, FAKE, 514, 0, 1.0, None) == 3
    assert lib.poss_rotary(FAKE, 512, FAKE, 1024, 1, 10, 8, 64, FAKE, FAKE, 64, 0, 1.0, None) == 1  # in place, rows elsewhere


def test_append_rotary_refusals(lib):
    # pool, layer, pages, tables, max_pages, batch, rows, k, v, ld_kv, hq, q, ld_q, out_q, ld_out, prefix, n_rows, pos, freq, rot, il, mag
    far = FAKE + (1 << 30)
    good = [pool(), 0, FAKE, FAKE, 4, 2, 3, FAKE, FAKE, 128, 4, far, 256, far, 256, FAKE, None, None, FAKE, 64, 0, 1.0, None, None]
    refused(lib.poss_pages_append_rotary, good, [
        (0, None, 1), (0, pool(d=48), 2), (1, 2, 1), (1, -1, 1), (2, None, 1), (2, FAKE + 8, 1), (3, None, 1), (4, 0, 1), (5, -1, 1),
        (5, 1025, 3), (6, 65536, 3), (7, None, 1), (8, FAKE + 4, 1), (9, 120, 1), (9, 129, 1), (10, -1, 1), (11, None, 1),
        (12, 248, 1), (13, None, 1), (13, far + 16, 1), (13, FAKE, 1), (14, 264, 1), (15, None, 1), (18, None, 1), (19, 66, 1),
        (19, 3, 1), (21, math.nan, 1)])
    assert lib.poss_pages_append_rotary(*[0 if i == 5 else a for i, a in enumerate(good)]) == 0


def test_append_rotary_refuses_rows_that_meet(lib):
    """Queries that turn in place between keys and values of one projection may lie between their rows; no element is of two, and none lies
    in the pages."""
    es, d, ld = 2, 64, 12 * 64                                        # rows of 8 query heads, 2 of keys, 2 of values, apart as one projection
    x, pages = FAKE + (1 << 30), FAKE + (1 << 31)
    pool_bytes = 2 * 64 * 2 * 2 * 16 * d * es

    def call(q=x, k=x + 8 * d * es, v=x + 10 * d * es, out=None, ld_q=ld, ld_out=None, kv_pages=pages, heads=8):
        out, ld_out = q if out is None else out, ld_q if ld_out is None else ld_out
        return lib.poss_pages_append_rotary(pool(), 0, kv_pages, FAKE, 4, 2, 3, k, v, ld, heads, q, ld_q, out, ld_out, FAKE, None, None, FAKE, d,
                                            0, 1.0, None, None)

    head, row = d * es, ld * es
    for q, k, v in [(x, x + 7 * head, x + 10 * head), (x, x, x + 10 * head), (x, x + 8 * head, x + 7 * head),     # the last query heads
                    (x + 2 * head, x + head, x + 10 * head), (x, x + 8 * head - 16, x + 10 * head), (x + 10 * head, x + 5 * head, x + 4 * head),
                    (x, x + 8 * head, x + 11 * head),                 # the last value head is the next row's first query head
                    (x + row, x + 8 * head, x + 11 * head), (x, x + row + 7 * head, x + 10 * head), (x, x + 8 * head, x + 4 * row + 7 * head)]:
        assert call(q, k, v) == 1, (q - x, k - x, v - x)
    assert call(ld_q=8 * d) == 1                                      # in place, but other rows than theirs
    assert call(out=x + (1 << 20), k=x + (1 << 20) + 8 * head) == 1   # elsewhere: not between them
    far = x + (1 << 24)
    for other in ({"q": pages}, {"q": pages + pool_bytes - 16}, {"k": pages + 256}, {"v": pages + pool_bytes - 16}, {"q": far, "out": pages - 16},
                  {"q": pages - 5 * row, "out": far}, {"k": pages - 5 * row - 2 * head + 16}, {"heads": 0, "k": pages}):
        assert call(**other) == 1, other


def test_mass_refusals(lib):
    need = lib.poss_paged_attention_mass_workspace_bytes(pool(), 2, 3, 4, 4)
    assert need > lib.poss_paged_attention_workspace_bytes(pool(), 2, 3, 4, 4) > 0 and need % 256 == 0
    assert lib.poss_paged_attention_mass_workspace_bytes(pool(), 2, 129, 4, 4) == 0
    assert lib.poss_paged_attention_mass_workspace_bytes(pool(), 0, 3, 4, 4) == 0
    q, out, mass = FAKE + (1 << 30), FAKE + (1 << 31), FAKE + (1 << 32)
    # pool, layer, pages, mass, slots, tables, max_pages, batch, rows, hq, q, ld_q, prefix, n_rows, mask, weights, scale, out, ws, bytes
    good = [pool(), 0, FAKE, mass, 64, FAKE, 4, 2, 3, 4, q, 256, FAKE, None, FAKE, None, 0.1, out, FAKE, need, None, None]
    refused(lib.poss_paged_tree_attention_mass, good, [
        (0, None, 1), (1, 2, 1), (2, None, 1), (3, None, 1), (4, 63, 1), (5, None, 1), (6, 0, 1), (7, -1, 1), (7, 1025, 3), (8, 129, 3),
        (9, 3, 2), (10, None, 1), (10, mass, 1), (11, 255, 1), (12, None, 1), (14, None, 1), (15, mass, 1), (16, math.nan, 1),
        (17, None, 1), (17, mass + 16, 1), (17, q, 1), (18, None, 4), (18, FAKE + 128, 4), (19, need - 1, 4)])
    assert lib.poss_paged_tree_attention_mass(*[0 if i == 8 else a for i, a in enumerate(good)]) == 0


def test_evict_and_commit_refusals(lib):
    need = lib.poss_pages_evict_workspace_bytes(pool(), 2, 4)
    assert need >= 2 * 2 * 2 * 64 * 4 and need % 256 == 0
    assert lib.poss_pages_evict_workspace_bytes(pool(), 0, 4) == 0
    assert lib.poss_pages_evict_workspace_bytes(pool(d=48), 2, 4) == 0
    mass, o = FAKE + (1 << 32), FAKE + (1 << 31)
    # pool, pages, tables, max_pages, batch, mass, out_mass, slots, len, keep, first, recent, out_len, ws, bytes, status, stream
    good = [pool(), FAKE, FAKE, 4, 2, mass, mass, 64, FAKE, FAKE, 1, 2, o, FAKE, need, None, None]
    refused(lib.poss_pages_evict, good, [
        (0, None, 1), (1, None, 1), (1, FAKE + 8, 1), (2, None, 1), (3, 0, 1), (4, -1, 1), (4, 1025, 3), (5, None, 1), (6, None, 1),
        (6, mass + 64, 1), (7, 63, 1), (8, None, 1), (8, o + 4, 1), (9, None, 1), (9, o, 1), (12, mass + 4, 1), (10, -1, 1), (11, -1, 1), (12, None, 1),
        (13, None, 4), (13, FAKE + 64, 4), (14, need - 1, 4)])
    assert lib.poss_pages_evict(*[0 if i == 4 else a for i, a in enumerate(good)]) == 0
    # pool, pages, mass, slots, tables, max_pages, batch, prefix, path, accepted, out_len, status, stream
    good = [pool(), FAKE, mass, 64, FAKE, 4, 2, FAKE, FAKE, FAKE, o, None, None]
    refused(lib.poss_pages_compact_mass, good, [(0, None, 1), (2, None, 1), (2, o, 1), (3, 63, 1), (1, None, 1), (7, o, 1), (10, None, 1),
                                                (6, 1025, 3)])


def test_eviction_with_holders_refusals(lib):
    need = lib.poss_pages_evict_workspace_bytes(pool(), 2, 4)
    mass, o, refs = FAKE + (1 << 32), FAKE + (1 << 31), FAKE + (1 << 30)
    # pool, pages, tables, max_pages, batch, refs, mass, out_mass, slots, len, keep, first, recent, out_len, ws, bytes, status, stream
    good = [pool(), FAKE, FAKE, 4, 2, refs, mass, mass, 64, FAKE, FAKE, 1, 2, o, FAKE, need, None, None]
    refused(lib.poss_pages_evict_refs, good, [
        (0, None, 1), (1, None, 1), (2, None, 1), (3, 0, 1), (4, -1, 1), (4, 1025, 3), (5, o, 1), (5, o + 4 - 64 * 4, 1), (5, mass, 1),
        (6, None, 1), (7, None, 1), (7, refs + 4, 1), (8, 63, 1), (9, None, 1), (9, o, 1), (10, None, 1), (11, -1, 1), (12, -1, 1), (13, None, 1),
        (13, refs + 64 * 4 - 4, 1), (14, None, 4), (15, need - 1, 4)])
    assert lib.poss_pages_evict_refs(*[0 if i == 4 else a for i, a in enumerate(good)]) == 0


def test_token_score_refusals(lib):
    out = [FAKE + (i << 28) for i in range(1, 6)]
    # logits, ld, dtype, rows, vocab, temperature, tokens, rows_of, n, logp, lse, entropy, k, top, top_logp, stream
    good = [FAKE, 100, 1, 4, 100, 1.0, FAKE + 4096, None, 4, out[0], out[1], out[2], 3, out[3], out[4], None]
    refused(lib.poss_token_logprobs, good, [
        (0, None, 1), (0, FAKE + 1, 1), (1, 99, 1), (2, 2, 1), (3, -1, 1), (3, 0, 1), (3, (1 << 24) + 1, 3), (4, 0, 1), (5, 0.0, 1),
        (5, -1.0, 1), (5, math.nan, 1), (5, math.inf, 1), (5, 1e-39, 1), (6, None, 1), (8, -1, 1), (8, 5, 1), (9, None, 1), (9, FAKE, 1),
        (9, FAKE + 4096, 1), (10, out[0], 1), (11, FAKE + 64, 1), (12, 17, 3), (12, -1, 1), (13, None, 1), (14, out[3], 1)])
    assert lib.poss_token_logprobs(FAKE, 100, 1, 0, 100, 1.0, None, None, 0, None, None, None, 0, None, None, None) == 0


def test_lost_load_hook_refusals(lib):
    for spared, launches, code in [(-1, 1, 1), (1, -1, 1), (3, 0, 0), (0, 0, 0)]:
        assert lib.poss_debug_paged_lose_load_after(spared, launches) == code
    assert lib.poss_debug_paged_lose_load(-1) == 1 and lib.poss_debug_paged_lose_load(0) == 0


def test_plain_forms_agree():
    """The eviction's choice against a loop over ranks; the scores against torch's log-softmax."""
    rng = np.random.default_rng(0)
    for n, keep, first, recent in [(10, 4, 1, 1), (9, 9, 0, 0), (30, 10, 0, 10), (30, 10, 4, 0), (7, 0, 0, 0)]:
        m = np.round(rng.random(n), 1).astype(np.float32)
        got = lu.chosen(m, n, keep, first, recent)
        always = [i for i in range(n) if n <= keep or i < first or i >= n - recent]
        rest = sorted((i for i in range(n) if i not in always), key=lambda i: (-m[i], i))[:max(0, min(n, keep) - len(always))]
        assert list(got) == sorted(always + rest)
    x = torch.randn(3, 50, dtype=torch.float64)
    w = lu.scores(x, [1, 2, 3], None, 4, 0.7)
    ref = torch.log_softmax(x / float(np.float32(0.7)), -1)
    assert torch.allclose(w["logp"][0], ref[[0, 1, 2], [1, 2, 3]], rtol=1e-12)
    assert torch.allclose(w["entropy"][0], -(ref.exp() * ref).sum(-1), rtol=1e-12)
    assert torch.equal(w["top_tokens"].long(), torch.topk(x, 4).indices)
