"""Paged caches, rotary positions, beam selection and token scores: the calls of poss_paged.h over torch tensors.

kv_pages [layers][pages][2][kv heads][page slots][head dim] (bf16 or fp32); tables int32 [sequences][max pages], -1 behind
a sequence's last page; refs int32 [pages]; mass fp32 [layers][sequences][kv heads][slots], the attention weight that each slot has
drawn (slots >= max pages x page slots; a fork takes its parent's: mass[:, parents]).  Everything lives on the current CUDA device and runs on its current stream.
`status` (optional) is a caller's int32 CUDA tensor of one element that the kernels raise (poss_paged.h); `workspace`
(optional) a caller's uint8 CUDA tensor, else scratch comes from torch for the call.

A call of these costs the GPU a few microseconds, so the tensors are checked and the outputs made in C++
(csrc/paged_calls.cpp): a ValueError names the tensor that is not as wanted, a PossError the library's status.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import POSS_BF16, POSS_FP32, POSS_MAX_ROTARY_DIM, PossError, load_library, poss_page_pool

_module = None


def _calls():
    """The module of csrc/paged_calls.cpp.  Raises if it is missing, or was built with another torch."""
    global _module
    if _module is None:
        load_library()
        try:
            from . import _paged_calls as module
        except ImportError as e:
            raise ImportError(f"_paged_calls not built ({e}); run python -m paper_2506_03566_b200.build") from e
        from .build import _torch_version
        if module.built_with_torch != _torch_version():
            raise ImportError(f"_paged_calls was built with torch {module.built_with_torch}, this is {_torch_version()}; run "
                              "python -m paper_2506_03566_b200.build")
        module.bind(PossError)
        _module = module
    return _module


def _pool_struct(kv_pages):
    layers, pages, two, heads, slots, d = kv_pages.shape
    if two != 2 or kv_pages.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"kv_pages: [layers][pages][2][kv heads][page slots][head dim] of bf16 or fp32 is wanted, got "
                         f"{kv_pages.dtype} {list(kv_pages.shape)}")
    return C.byref(poss_page_pool(layers, pages, heads, slots, d,
                                  POSS_BF16 if kv_pages.dtype is torch.bfloat16 else POSS_FP32))


def poss_paged_attention_workspace_bytes(kv_pages, batch, rows, n_q_heads, max_pages):
    """Bytes of the `workspace` of poss_paged_tree_attention on the current device."""
    return load_library().poss_paged_attention_workspace_bytes(_pool_struct(kv_pages), batch, rows, n_q_heads, max_pages)


def poss_pages_remap_workspace_bytes(kv_pages, n_before, n_after, max_pages):
    """Bytes of the `workspace` of poss_pages_remap."""
    return load_library().poss_pages_remap_workspace_bytes(_pool_struct(kv_pages), n_before, n_after, max_pages)


def poss_beam_select_workspace_bytes(batch, beams, vocab):
    """Bytes of the `workspace` of poss_beam_select."""
    return load_library().poss_beam_select_workspace_bytes(batch, beams, vocab)


_SCALINGS = {"linear": 1, "base": 2, "bands": 3, "ramp": 4}


def poss_rotary_frequencies(rot_dim, theta, scaling=None, factor=1.0, low=1.0, high=4.0, original_len=0.0, device="cuda"):
    """Radians per position of rot_dim / 2 pairs, float64: theta^(-2i / rot_dim), scaled for longer contexts by None, "linear", "base",
    "bands" or "ramp" (poss_paged.h).  The `freq` of poss_rotary and poss_pages_append_rotary."""
    if scaling is not None and scaling not in _SCALINGS:
        raise ValueError(f"scaling: None or one of {sorted(_SCALINGS)} is wanted, got {scaling!r}")
    if not isinstance(rot_dim, int) or not 2 <= rot_dim <= POSS_MAX_ROTARY_DIM:
        raise ValueError(f"rot_dim: an even number of 2 to {POSS_MAX_ROTARY_DIM} is wanted, got {rot_dim!r}")
    out = torch.empty(rot_dim // 2, dtype=torch.float64)
    code = load_library().poss_rotary_frequencies(out.data_ptr(), rot_dim, theta, _SCALINGS.get(scaling, 0), factor, low, high,
                                                  original_len)
    if code:
        raise PossError(code, "poss_rotary_frequencies")
    return out.to(device)


def poss_rotary(x, positions, freq, out=None, interleaved=False, magnitude=1.0):
    """Turns the first 2 * freq.numel() elements of every head of x [batch][rows][heads][d] by positions int32 [batch][rows]; pairs
    are the halves of that part, or with `interleaved` neighbours.  out may be x.  Returns out."""
    return _calls().rotary(x, positions, freq, out, interleaved, magnitude)


def poss_pages_append_rotary(k, v, kv_pages, layer, tables, prefix_len, freq, positions=None, q=None, out_q=None, interleaved=False,
                             magnitude=1.0, n_rows=None, status=None):
    """poss_pages_append with k turned as by poss_rotary (positions None: the rows' slots), and q [batch][rows][query heads][d] too.
    Returns the turned queries (out_q, which may be q), None without queries; their rows behind n_rows[b] are not written."""
    return _calls().append_rotary(k, v, kv_pages, layer, tables, prefix_len, freq, positions, q, out_q, interleaved, magnitude, n_rows,
                                  status)


def poss_pages_append(k, v, kv_pages, layer, tables, prefix_len, n_rows=None, status=None):
    """Writes k, v [batch][rows][kv heads][d] behind every sequence's first prefix_len[b] slots in layer `layer`."""
    _calls().append(k, v, kv_pages, layer, tables, prefix_len, n_rows, status)


def poss_paged_tree_attention(q, kv_pages, layer, tables, prefix_len, anc_mask, scale, n_rows=None, out=None,
                              workspace=None, status=None):
    """Tree-masked attention of q [batch][rows][query heads][d] over the pages of layer `layer`; anc_mask int64
    [batch][rows][ceil(rows/64)].  Returns out [batch][rows][query heads][d]; rows behind n_rows[b] are not written."""
    return _calls().attention(q, kv_pages, layer, tables, prefix_len, anc_mask, scale, n_rows, out, workspace, status)


def poss_paged_attention_mass_workspace_bytes(kv_pages, batch, rows, n_q_heads, max_pages):
    """Bytes of the `workspace` of poss_paged_tree_attention_mass on the current device."""
    return load_library().poss_paged_attention_mass_workspace_bytes(_pool_struct(kv_pages), batch, rows, n_q_heads, max_pages)


def poss_paged_tree_attention_mass(q, kv_pages, mass, layer, tables, prefix_len, anc_mask, scale, n_rows=None, row_weights=None,
                                   out=None, workspace=None, status=None):
    """poss_paged_tree_attention that also adds up, in mass[layer], the weight that every slot draws from the rows (times row_weights
    fp32 [batch][rows]): committed slots are added to, the rows' own slots are set.  Returns out."""
    return _calls().attention_mass(q, kv_pages, mass, layer, tables, prefix_len, anc_mask, scale, n_rows, row_weights, out, workspace,
                                   status)


def poss_pages_evict_workspace_bytes(kv_pages, batch, max_pages):
    """Bytes of the `workspace` of poss_pages_evict."""
    return load_library().poss_pages_evict_workspace_bytes(_pool_struct(kv_pages), batch, max_pages)


def poss_pages_evict(kv_pages, mass, tables, seq_len, keep, first=0, recent=0, out_mass=None, out_len=None, workspace=None, status=None,
                     refs=None):
    """Cuts every sequence to keep[b] slots (int32 [batch]): the first, the last and, of the others, those of greatest mass, for each
    layer and KV head; they move to the front in their order, their masses to out_mass (None: mass itself).  With the `refs` of
    poss_pages_remap a sequence that would write to a page with other holders (a fork, a pinned prefix behind `first`) keeps its slots and
    raises the status; without them the caller answers for it that there is none.  Returns the new lengths."""
    return _calls().evict(kv_pages, mass, tables, seq_len, keep, first, recent, out_mass, out_len, workspace, status, refs)


def poss_pages_compact(kv_pages, tables, prefix_len, path, n_accepted, out_len=None, status=None, mass=None):
    """Moves every sequence's accepted path behind its committed slots in all layers; path int32 [batch]
    [POSS_MAX_DEPTH + 1], n_accepted int32 [batch].  With `mass` the slots' weights go with them.  Returns the new lengths int32
    [batch]."""
    return _calls().compact(kv_pages, tables, prefix_len, path, n_accepted, out_len, status, mass)


def poss_pages_remap(kv_pages, tables, seq_len, refs, parents=None, room=None, out=None, workspace=None, status=None):
    """Replaces the sequences of `tables` by parents.numel() new ones (poss_paged.h).  Returns a dict of int32 tensors:
    tables, refs, seq_len, n_free (one element).  A negative n_free: that many pages were missing, the pool is unchanged and
    refs as before; tables and seq_len are then as they were in a caller's `out`, else without pages and slots (-1 and 0)."""
    return _calls().remap(kv_pages, tables, seq_len, refs, parents, room, out, workspace, status)


def poss_beam_select(logits, scores, finished=None, eos=-1, out=None, workspace=None):
    """One beam-search selection: logits [batch][beams][vocab] (fp32 or bf16), scores fp32 [batch][beams], finished int32
    [batch][beams].  Returns a dict of [batch][beams] tensors: tokens, parents, finished (int32) and scores (fp32)."""
    return _calls().beam_select(logits, scores, finished, eos, out, workspace)


def poss_token_logprobs(logits, tokens=None, token_rows=None, topk=0, temperature=1.0, out=None):
    """Scores of logits [rows][vocab] (fp32 or bf16, rows may lie apart) at a temperature.  Returns a dict of tensors: logp fp32 [n] of
    tokens int32 [n] in rows token_rows int32 [n] (None: token i in row i), lse and entropy fp32 [rows], top_tokens int32 and top_logp
    fp32 [rows][topk], best first."""
    return _calls().token_logprobs(logits, tokens, token_rows, topk, temperature, out)
