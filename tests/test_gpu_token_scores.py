"""GPU tests of the token scores against their plain 64-bit form."""
import math

import numpy as np
import pytest
import torch

from tests import long_util as lu
from tests.test_gpu_paged import BF, F32, cu, i32, lib

pytestmark = pytest.mark.gpu


def run(x, tokens=None, token_rows=None, topk=0, temperature=1.0):
    return lib().poss_token_logprobs(x, None if tokens is None else i32(tokens), None if token_rows is None else i32(token_rows),
                                     topk=topk, temperature=temperature)


def check(x, tokens=None, token_rows=None, topk=0, temperature=1.0):
    g = x if x.is_cuda else x.cuda()
    got = run(g, tokens, token_rows, topk, temperature)
    lu.check_scores(got, lu.scores(x.cpu().double(), tokens, token_rows, topk, temperature))
    again = run(g, tokens, token_rows, topk, temperature)
    for k in got:
        assert torch.equal(got[k], again[k])                          # equal calls, equal bits
    return got


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 7), (5, 31), (1, 257), (61, 1000), (2, 8191), (3, 8193), (2, 32001), (1, 65536),
                                        (1, 128256), (9, 50257), (150, 16400), (300, 300)])
@pytest.mark.parametrize("topk,temperature", [(0, 1.0), (1, 0.3), (5, 1.0), (16, 2.5)])
def test_scores_match_the_plain_form(dtype, rows, vocab, topk, temperature):
    gen = torch.Generator().manual_seed(vocab + topk)
    x = (torch.randn(rows, vocab, generator=gen) * 3).to(dtype)       # (bf16: many equal ones at the top)
    tokens = torch.randint(0, vocab, (rows,), generator=gen).tolist()
    check(x, tokens, None, topk, temperature)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_tokens_of_any_rows(dtype):
    """A tree's nodes in their parents' rows, one row asked often, none, and places out of range."""
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(6, 999, generator=gen).to(dtype)
    tokens = [5, 6, 7, -1, 998, 999, 0, 1 << 30, 3, 3] + torch.randint(0, 999, (700,), generator=gen).tolist()
    rows = [-1, 0, 0, 1, 2, 2, 6, 3, 5, -7] + torch.randint(-1, 6, (700,), generator=gen).tolist()
    got = check(x, tokens, rows, 3)
    assert got["logp"][0] == 0 and got["logp"][3] == 0 and got["logp"][5] == -math.inf and got["logp"][6] == -math.inf
    check(x, [1, 2], None, 1)                                         # fewer tokens than rows
    assert run(x.cuda(), None, None, 2)["logp"].shape == (0,)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("vocab", [100, 4097, 40000])
def test_banned_and_extreme_logits(dtype, vocab):
    gen = torch.Generator().manual_seed(4)
    low = torch.finfo(dtype).min
    x = torch.randn(16, vocab, generator=gen).to(dtype)
    x[0] = -math.inf                                                  # all banned
    x[1] = -math.inf
    x[1, vocab - 3] = 2.0                                             # one left
    x[2, ::2] = -math.inf
    x[3, 1:] = low                                                    # masks of the type's lowest value
    x[4] = low                                                        # nothing else
    x[5, 7] = math.nan
    x[5, 9] = math.inf
    x[6] = math.nan
    x[7] = 1.5                                                        # all equal
    x[8] = torch.arange(vocab, dtype=torch.float32).to(dtype)         # rising: every step has new best ones
    x[9] = -torch.arange(vocab, dtype=torch.float32).to(dtype)
    x[10] = 0.0
    x[10, ::2] = -0.0                                                 # signed zeros are equal
    x[11] = 0.0
    x[11, vocab // 2] = torch.finfo(dtype).max
    x[12] = torch.finfo(dtype).max
    x[13] = -1e10
    x[13, 5] = 30.0
    x[14, :90] = 60.0                                                 # one far above many
    x[14, 50] = 400.0
    x[15] = x[15] * 1e-38                                             # denormal differences
    tokens = [0, vocab - 3, 1, 0, 3, 9, 0, 5, vocab - 1, 0, 1, vocab // 2, 7, 5, 50, 2]
    for k, t in ((16, 1.0), (3, 0.01), (1, 50.0)):
        check(x, tokens, None, k, t)
    check(x, [7] * 16, list(range(16)), 0, 1.0)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("vocab,ld,shift", [(5000, 5003, 0), (5001, 5001, 1), (5000, 5008, 3), (9, 12, 5), (3, 17, 2)])
def test_rows_that_lie_apart_and_start_anywhere(dtype, vocab, ld, shift):
    gen = torch.Generator().manual_seed(5)
    whole = torch.full((7 * ld + shift,), math.nan, dtype=dtype)
    x = whole[shift:shift + 7 * ld].view(7, ld)[:, :vocab]
    x.copy_(torch.randn(7, vocab, generator=gen))
    g = whole.cuda()[shift:shift + 7 * ld].view(7, ld)[:, :vocab]
    got = run(g, [1] * 7, None, 4)
    lu.check_scores(got, lu.scores(x.double(), [1] * 7, None, 4, 1.0))


def test_many_rows_replay_and_streams():
    gen = torch.Generator().manual_seed(6)
    x = torch.randn(700, 4000, generator=gen).to(BF)
    tokens = torch.randint(0, 4000, (700,), generator=gen).to(torch.int32)
    g, t = x.cuda(), tokens.cuda()
    want = lib().poss_token_logprobs(g, t, topk=2)
    lu.check_scores({k: v[:40] for k, v in want.items()}, lu.scores(x[:40].double(), tokens[:40].tolist(), None, 2, 1.0))
    out = {k: torch.zeros_like(v) for k, v in want.items()}
    work = g.clone()
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        lib().poss_token_logprobs(work, t, topk=2, out=out)
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(graph):
        lib().poss_token_logprobs(work, t, topk=2, out=out)
    work.copy_(g.flip(0))
    t.copy_(t.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(out[k], want[k].flip(0))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    res = []
    for s in (s1, s2):
        with torch.cuda.stream(s):
            res.append(lib().poss_token_logprobs(work, t, topk=2))
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(res[0][k], out[k]) and torch.equal(res[1][k], out[k])
    empty = lib().poss_token_logprobs(torch.zeros(0, 5, device="cuda"), topk=2)
    assert empty["top_tokens"].shape == (0, 2)


def test_scores_of_a_verified_tree():
    """Beside a target pass: its logits and its greedy tokens, the drafted tokens in their parents' rows."""
    import poss_synth as ps
    from paper_2506_03566_b200 import Poss, make_config
    cfg = ps.CONFIGS["t_fp32"]
    w = ps.make_weights(cfg, 7)
    P = Poss(make_config(cfg, cfg.prefix + 3 + cfg.tree_slots, 256), w)
    kv = P.new_target_kv()
    prompt = torch.from_numpy(ps.make_prompt(cfg, 7, 12)).cuda()
    P.poss_target_prefill(kv, 0, prompt)
    tokens, parents, depth = [3, 5, 7, 5, 2], [-1, 0, 0, 1, 3], [0, 1, 1, 2, 3]
    anc = np.zeros((1, 5, 5), bool)
    for r in range(5):
        j = r
        while j >= 0:
            anc[0, r, j] = True
            j = parents[j]
    from tests import paged_util as pg
    _, arg, logits = P.poss_target_forward(kv, 12, i32(tokens), i32(depth), cu(pg.pack(anc)[0]), 5, want_logits=True)
    got = lib().poss_token_logprobs(logits, i32(tokens), token_rows=i32(parents), topk=3)
    lu.check_scores(got, lu.scores(logits.cpu().double(), tokens, parents, 3, 1.0))
    assert torch.equal(got["top_tokens"][:, 0], arg) and got["logp"][0] == 0


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,vocab", [(302, 41003), (302, 24576), (12, 100001)])
def test_masked_vocabularies(dtype, rows, vocab):
    """Rows of several steps that begin with banned tokens or keep few: masks of -inf, of the type's lowest value and of plain numbers."""
    gen = torch.Generator().manual_seed(8)
    x = (torch.randn(rows, vocab, generator=gen) * 3).to(dtype)
    few = torch.rand(rows, vocab, generator=gen) < 0.001
    place = torch.arange(vocab)
    masks = [-math.inf, torch.finfo(dtype).min, -1e4, -1e9]
    for r in range(rows):
        v = masks[r // 8 % 4]
        kind = r % 8
        if kind == 0:
            x[r, :20000] = v                                          # whole steps of nothing
        elif kind == 1:
            x[r][~few[r]] = v
        elif kind == 2:
            x[r][place % 3 != 0] = v
        elif kind == 3:
            x[r][place % 4999 != 17] = v                              # fewer left than best ones are wanted, or hardly more
        elif kind == 4:
            x[r][place % 4999 != 17] = v                              # a few, and then a flood above some of them
            x[r, 9000:17500] = 0.25
        elif kind == 5:
            x[r] = (place // 8192).float()                            # steps that are equal in themselves, rising
        elif kind == 6:
            x[r] = -(place // 8192).float()
            x[r, vocab - 2:] = 0.0                                    # equal ones behind all steps
        else:
            x[r, 16400:] = v
            x[r, :3] = v
            x[r, vocab - 1] = 1.0
    tokens = torch.randint(0, vocab, (rows,), generator=gen).tolist()
    for k, t in ((1, 1.0), (10, 1.0), (16, 0.7)):
        check(x, tokens, None, k, t)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_no_token_is_none_in_any_row(dtype):
    """A token below 0 scores 0 in a row behind the last one too; a token in such a row is banned."""
    x = torch.randn(3, 50, generator=torch.Generator().manual_seed(5)).to(dtype)
    got = check(x, [-1, -5, 7, -1, 7, -1], [3, 1 << 30, 3, -1, -1, 2], 0)
    assert got["logp"].cpu().tolist() == [0, 0, -math.inf, 0, 0, 0]
