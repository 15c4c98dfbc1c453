"""Paged caches and beam selection: the calls of poss_paged.h over torch tensors.

kv_pages [layers][pages][2][kv heads][page slots][head dim] (bf16 or fp32); tables int32 [sequences][max pages], -1 behind
a sequence's last page; refs int32 [pages].  Everything lives on the current CUDA device and runs on its current stream.
`status` (optional) is a caller's int32 CUDA tensor of one element that the kernels raise (poss_paged.h); `workspace`
(optional) a caller's uint8 CUDA tensor, else scratch comes from torch for the call.

A call of these costs the GPU a few microseconds, so the tensors are checked and the outputs made in C++
(csrc/paged_calls.cpp): a ValueError names the tensor that is not as wanted, a PossError the library's status.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import POSS_BF16, POSS_FP32, PossError, load_library, poss_page_pool

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


def poss_pages_append(k, v, kv_pages, layer, tables, prefix_len, n_rows=None, status=None):
    """Writes k, v [batch][rows][kv heads][d] behind every sequence's first prefix_len[b] slots in layer `layer`."""
    _calls().append(k, v, kv_pages, layer, tables, prefix_len, n_rows, status)


def poss_paged_tree_attention(q, kv_pages, layer, tables, prefix_len, anc_mask, scale, n_rows=None, out=None,
                              workspace=None, status=None):
    """Tree-masked attention of q [batch][rows][query heads][d] over the pages of layer `layer`; anc_mask int64
    [batch][rows][ceil(rows/64)].  Returns out [batch][rows][query heads][d]; rows behind n_rows[b] are not written."""
    return _calls().attention(q, kv_pages, layer, tables, prefix_len, anc_mask, scale, n_rows, out, workspace, status)


def poss_pages_compact(kv_pages, tables, prefix_len, path, n_accepted, out_len=None, status=None):
    """Moves every sequence's accepted path behind its committed slots in all layers; path int32 [batch]
    [POSS_MAX_DEPTH + 1], n_accepted int32 [batch].  Returns the new lengths int32 [batch]."""
    return _calls().compact(kv_pages, tables, prefix_len, path, n_accepted, out_len, status)


def poss_pages_remap(kv_pages, tables, seq_len, refs, parents=None, room=None, out=None, workspace=None, status=None):
    """Replaces the sequences of `tables` by parents.numel() new ones (poss_paged.h).  Returns a dict of int32 tensors:
    tables, refs, seq_len, n_free (one element).  A negative n_free: that many pages were missing, the pool is unchanged and
    refs as before; tables and seq_len are then as they were in a caller's `out`, else without pages and slots (-1 and 0)."""
    return _calls().remap(kv_pages, tables, seq_len, refs, parents, room, out, workspace, status)


def poss_beam_select(logits, scores, finished=None, eos=-1, out=None, workspace=None):
    """One beam-search selection: logits [batch][beams][vocab] (fp32 or bf16), scores fp32 [batch][beams], finished int32
    [batch][beams].  Returns a dict of [batch][beams] tensors: tokens, parents, finished (int32) and scores (fp32)."""
    return _calls().beam_select(logits, scores, finished, eos, out, workspace)
