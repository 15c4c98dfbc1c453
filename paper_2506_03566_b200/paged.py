"""Paged caches and beam selection: the calls of poss_paged.h over torch tensors.  Argument marshalling only.

kv_pages [layers][pages][2][kv heads][page slots][head dim] (bf16 or fp32); tables int32 [sequences][max pages], -1 behind
a sequence's last page; refs int32 [pages].  Everything lives on the current CUDA device and runs on its current stream.
`status` (optional) is a caller's int32 CUDA tensor of one element that the kernels raise (poss_paged.h); `workspace`
(optional) a caller's uint8 CUDA tensor, else scratch comes from torch for the call.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from .binding import POSS_BF16, POSS_FP32, PossError, _check, load_library, poss_page_pool  # noqa: F401

_DTYPES = {torch.bfloat16: POSS_BF16, torch.float32: POSS_FP32}


def _arg(t, dtype, shape, name, device):
    """Address of a contiguous tensor of the given type and shape on the device of the call (None stays None)."""
    if t is None:
        return None
    if t.device != device or t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor {list(shape)} on {device} is wanted, got {t.dtype} "
                         f"{list(t.shape)} on {t.device}")
    return t.data_ptr()


@functools.lru_cache(maxsize=256)
def _pool_struct(shape, dtype):
    layers, pages, two, heads, slots, d = shape
    if two != 2 or dtype not in _DTYPES:
        raise ValueError(f"kv_pages: [layers][pages][2][kv heads][page slots][head dim] of bf16 or fp32 is wanted, got "
                         f"{dtype} {list(shape)}")
    return poss_page_pool(layers, pages, heads, slots, d, _DTYPES[dtype])


def _pool(kv_pages):
    if kv_pages.dim() != 6 or not kv_pages.is_cuda or not kv_pages.is_contiguous():
        raise ValueError("kv_pages: a contiguous CUDA tensor of six dimensions is wanted")
    dev = kv_pages.device
    if dev.index != torch.cuda.current_device():
        raise ValueError(f"kv_pages is on {dev}, the current device is cuda:{torch.cuda.current_device()}")
    return C.byref(_pool_struct(tuple(kv_pages.shape), kv_pages.dtype)), dev


def _stream(dev):
    return torch.cuda.current_stream(dev).cuda_stream


def _rows(t, name, heads, d, dtype, device):
    """Address and row stride of [batch][rows][heads][d] whose rows may lie apart (a slice of a fused projection)."""
    b, r = t.shape[0], t.shape[1]
    if t.device != device or t.dtype != dtype or tuple(t.shape[2:]) != (heads, d):
        raise ValueError(f"{name}: {dtype} [batch][rows][{heads}][{d}] on {device} is wanted, got {t.dtype} "
                         f"{list(t.shape)} on {t.device}")
    st = t.stride()
    ld = st[1] if r > 1 else (st[0] if b > 1 else heads * d)
    if st[3] != 1 and d > 1 or st[2] != d and heads > 1 or r > 1 and b > 1 and st[0] != r * ld or ld < heads * d:
        raise ValueError(f"{name}: heads contiguous and rows evenly apart are wanted, got strides {list(st)}")
    return t.data_ptr(), ld


def _scratch(workspace, nbytes, device):
    if workspace is None:
        return torch.empty(nbytes, dtype=torch.uint8, device=device)
    if workspace.device != device or workspace.dtype != torch.uint8 or not workspace.is_contiguous():
        raise ValueError(f"workspace: a contiguous uint8 tensor on {device} is wanted")
    return workspace


def poss_pages_append(k, v, kv_pages, layer, tables, prefix_len, n_rows=None, status=None):
    """Writes k, v [batch][rows][kv heads][d] behind every sequence's first prefix_len[b] slots in layer `layer`."""
    pool, dev = _pool(kv_pages)
    b, r = k.shape[0], k.shape[1]
    heads, d = kv_pages.shape[3], kv_pages.shape[5]
    i32 = torch.int32
    kp, ld = _rows(k, "k", heads, d, kv_pages.dtype, dev)
    vp, ldv = _rows(v, "v", heads, d, kv_pages.dtype, dev)
    if ldv != ld or v.shape != k.shape:
        raise ValueError("k and v: the same shape and the same strides are wanted")
    mp = tables.shape[1]
    _check(load_library().poss_pages_append(
        pool, layer, kv_pages.data_ptr(), _arg(tables, i32, (b, mp), "tables", dev), mp, b, r, kp, vp, ld,
        _arg(prefix_len, i32, (b,), "prefix_len", dev), _arg(n_rows, i32, (b,), "n_rows", dev),
        _arg(status, i32, (1,), "status", dev), _stream(dev)), "poss_pages_append")


def poss_paged_tree_attention(q, kv_pages, layer, tables, prefix_len, anc_mask, scale, n_rows=None, out=None,
                              workspace=None, status=None):
    """Tree-masked attention of q [batch][rows][query heads][d] over the pages of layer `layer`; anc_mask int64
    [batch][rows][ceil(rows/64)].  Returns out [batch][rows][query heads][d]; rows behind n_rows[b] are not written."""
    pool, dev = _pool(kv_pages)
    b, r, hq = q.shape[0], q.shape[1], q.shape[2]
    d = kv_pages.shape[5]
    i32 = torch.int32
    qp, ld = _rows(q, "q", hq, d, kv_pages.dtype, dev)
    if out is None:
        out = torch.empty((b, r, hq, d), dtype=q.dtype, device=dev)
    if b == 0 or r == 0:
        return out
    lib = load_library()
    mp = tables.shape[1]
    ws = _scratch(workspace, lib.poss_paged_attention_workspace_bytes(pool, b, r, hq, mp), dev)
    _check(lib.poss_paged_tree_attention(
        pool, layer, kv_pages.data_ptr(), _arg(tables, i32, (b, mp), "tables", dev), mp, b, r, hq, qp, ld,
        _arg(prefix_len, i32, (b,), "prefix_len", dev), _arg(n_rows, i32, (b,), "n_rows", dev),
        _arg(anc_mask, torch.int64, (b, r, (r + 63) // 64), "anc_mask", dev), scale,
        _arg(out, q.dtype, (b, r, hq, d), "out", dev), ws.data_ptr(), ws.numel(),
        _arg(status, i32, (1,), "status", dev), _stream(dev)), "poss_paged_tree_attention")
    return out


def poss_pages_compact(kv_pages, tables, prefix_len, path, n_accepted, out_len=None, status=None):
    """Moves every sequence's accepted path behind its committed slots in all layers; path int32 [batch]
    [POSS_MAX_DEPTH + 1], n_accepted int32 [batch].  Returns the new lengths int32 [batch]."""
    pool, dev = _pool(kv_pages)
    b, mp = tables.shape
    i32 = torch.int32
    if out_len is None:
        out_len = torch.empty(b, dtype=i32, device=dev)
    _check(load_library().poss_pages_compact(
        pool, kv_pages.data_ptr(), _arg(tables, i32, (b, mp), "tables", dev), mp, b,
        _arg(prefix_len, i32, (b,), "prefix_len", dev), _arg(path, i32, (b, 17), "path", dev),
        _arg(n_accepted, i32, (b,), "n_accepted", dev), _arg(out_len, i32, (b,), "out_len", dev),
        _arg(status, i32, (1,), "status", dev), _stream(dev)), "poss_pages_compact")
    return out_len


def poss_pages_remap(kv_pages, tables, seq_len, refs, parents=None, room=None, out=None, workspace=None, status=None):
    """Replaces the sequences of `tables` by parents.numel() new ones (poss_paged.h).  Returns a dict of int32 tensors:
    tables, refs, seq_len, n_free (one element; negative: that many pages were missing and nothing changed)."""
    pool, dev = _pool(kv_pages)
    n0, mp = tables.shape
    n1 = n0 if parents is None else parents.numel()
    i32 = torch.int32
    pages = kv_pages.shape[1]
    if out is None:
        out = {"tables": torch.empty((n1, mp), dtype=i32, device=dev), "refs": torch.empty(pages, dtype=i32, device=dev),
               "seq_len": torch.empty(n1, dtype=i32, device=dev), "n_free": torch.empty(1, dtype=i32, device=dev)}
    lib = load_library()
    ws = _scratch(workspace, lib.poss_pages_remap_workspace_bytes(pool, n0, n1, mp), dev)
    _check(lib.poss_pages_remap(
        pool, kv_pages.data_ptr(), _arg(tables, i32, (n0, mp), "tables", dev),
        _arg(out["tables"], i32, (n1, mp), "out tables", dev), mp, n0, n1, _arg(seq_len, i32, (n0,), "seq_len", dev),
        _arg(refs, i32, (pages,), "refs", dev), _arg(out["refs"], i32, (pages,), "out refs", dev),
        _arg(parents, i32, (n1,), "parents", dev), _arg(room, i32, (n1,), "room", dev),
        _arg(out["seq_len"], i32, (n1,), "out seq_len", dev), _arg(out["n_free"], i32, (1,), "n_free", dev),
        ws.data_ptr(), ws.numel(), _arg(status, i32, (1,), "status", dev), _stream(dev)), "poss_pages_remap")
    return out


def poss_beam_select(logits, scores, finished=None, eos=-1, out=None, workspace=None):
    """One beam-search selection: logits [batch][beams][vocab] (fp32 or bf16), scores fp32 [batch][beams], finished int32
    [batch][beams].  Returns a dict of [batch][beams] tensors: tokens, parents, finished (int32) and scores (fp32)."""
    if logits.dim() != 3 or logits.dtype not in _DTYPES or not logits.is_cuda:
        raise ValueError("logits: a CUDA tensor [batch][beams][vocab] of fp32 or bf16 is wanted")
    dev = logits.device
    if dev.index != torch.cuda.current_device():
        raise ValueError(f"logits is on {dev}, the current device is cuda:{torch.cuda.current_device()}")
    b, k, v = logits.shape
    i32, f32 = torch.int32, torch.float32
    if out is None:
        out = {"tokens": torch.empty((b, k), dtype=i32, device=dev), "parents": torch.empty((b, k), dtype=i32, device=dev),
               "scores": torch.empty((b, k), dtype=f32, device=dev), "finished": torch.empty((b, k), dtype=i32, device=dev)}
    lib = load_library()
    ws = _scratch(workspace, lib.poss_beam_select_workspace_bytes(b, k, v), dev)
    _check(lib.poss_beam_select(
        _arg(logits, logits.dtype, (b, k, v), "logits", dev), _DTYPES[logits.dtype], b, k, v,
        _arg(scores, f32, (b, k), "scores", dev), _arg(finished, i32, (b, k), "finished", dev), eos,
        _arg(out["tokens"], i32, (b, k), "tokens", dev), _arg(out["parents"], i32, (b, k), "parents", dev),
        _arg(out["scores"], f32, (b, k), "out scores", dev), _arg(out["finished"], i32, (b, k), "out finished", dev),
        ws.data_ptr(), ws.numel(), _stream(dev)), "poss_beam_select")
    return out
