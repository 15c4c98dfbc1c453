"""Paged caches and beam selection: the calls of poss_paged.h over torch tensors.  Argument marshalling only.

kv_pages [layers][pages][2][kv heads][page slots][head dim] (bf16 or fp32); tables int32 [sequences][max pages], -1 behind
a sequence's last page; refs int32 [pages].  Everything lives on the current CUDA device and runs on its current stream.
`status` (optional) is a caller's int32 CUDA tensor of one element that the kernels raise (poss_paged.h); `workspace`
(optional) a caller's uint8 CUDA tensor, else scratch comes from torch for the call.

A call of these costs the GPU a few microseconds, so the host's part is kept short: sizes are asked of the library once per
geometry, the stream is read as a raw handle.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from .binding import POSS_BF16, POSS_FP32, POSS_MAX_DEPTH, PossError, load_library, poss_page_pool

_DTYPES = {torch.bfloat16: POSS_BF16, torch.float32: POSS_FP32}
_I32, _F32, _I64, _U8 = torch.int32, torch.float32, torch.int64, torch.uint8
_raw_stream = torch._C._cuda_getCurrentRawStream          # of a device ordinal; 0.1 us (the stream object: 3 us)


def _wrong(t, dtype, shape, name, dev):
    if not isinstance(t, torch.Tensor):
        return ValueError(f"{name}: a CUDA tensor is wanted, got {type(t).__name__}")
    return ValueError(f"{name}: a contiguous {dtype} tensor {list(shape)} on cuda:{dev} is wanted, got {t.dtype} "
                      f"{list(t.shape)} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}")


def _arg(t, dtype, shape, name, dev):
    """Address of a contiguous tensor of the given type and shape on device `dev`."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise _wrong(t, dtype, shape, name, dev)
    return t.data_ptr()


def _opt(t, dtype, shape, name, dev):
    return None if t is None else _arg(t, dtype, shape, name, dev)


def _call(code, where):
    if code:
        raise PossError(code, where)


@functools.lru_cache(maxsize=256)
def _pool_struct(shape, dtype):
    layers, pages, two, heads, slots, d = shape
    if two != 2 or dtype not in _DTYPES:
        raise ValueError(f"kv_pages: [layers][pages][2][kv heads][page slots][head dim] of bf16 or fp32 is wanted, got "
                         f"{dtype} {list(shape)}")
    s = poss_page_pool(layers, pages, heads, slots, d, _DTYPES[dtype])
    return C.byref(s), heads, slots, d


def _device(t, name):
    dev = t.get_device()
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError(f"{name}: a tensor on the current device is wanted, got one on {t.device}")
    return dev


def _pool(kv_pages):
    if kv_pages.dim() != 6 or not kv_pages.is_contiguous():
        raise ValueError("kv_pages: a contiguous CUDA tensor of six dimensions is wanted")
    return _pool_struct(kv_pages.shape, kv_pages.dtype), _device(kv_pages, "kv_pages")


def _rows(t, name, heads, d, dtype, dev):
    """Address and row stride of [batch][rows][heads][d] whose rows may lie apart (a slice of a fused projection)."""
    b, r, h, e = t.shape
    if t.dtype is not dtype or h != heads or e != d or t.get_device() != dev:
        raise _wrong(t, dtype, (b, r, heads, d), name, dev)
    if t.is_contiguous():
        return t.data_ptr(), heads * d
    sb, ld, sh, se = t.stride()
    if r == 1:
        ld = sb if b > 1 else heads * d
    if se != 1 or (heads > 1 and sh != d) or (r > 1 and b > 1 and sb != r * ld) or ld < heads * d:
        raise ValueError(f"{name}: heads contiguous and rows evenly apart are wanted, got strides {list(t.stride())}")
    return t.data_ptr(), ld


def _scratch(workspace, nbytes, dev):
    if workspace is None:
        return torch.empty(nbytes, dtype=_U8, device=dev)
    if workspace.get_device() != dev or workspace.dtype is not _U8 or not workspace.is_contiguous():
        raise ValueError(f"workspace: a contiguous uint8 tensor on cuda:{dev} is wanted")
    return workspace


@functools.lru_cache(maxsize=1024)
def _attention_bytes(shape, dtype, dev, b, r, hq, mp):
    return load_library().poss_paged_attention_workspace_bytes(_pool_struct(shape, dtype)[0], b, r, hq, mp)


@functools.lru_cache(maxsize=1024)
def _remap_bytes(shape, dtype, n0, n1, mp):
    return load_library().poss_pages_remap_workspace_bytes(_pool_struct(shape, dtype)[0], n0, n1, mp)


@functools.lru_cache(maxsize=1024)
def _beam_bytes(b, k, v):
    return load_library().poss_beam_select_workspace_bytes(b, k, v)


def poss_paged_attention_workspace_bytes(kv_pages, batch, rows, n_q_heads, max_pages):
    """Bytes of the `workspace` of poss_paged_tree_attention."""
    _, dev = _pool(kv_pages)
    return _attention_bytes(kv_pages.shape, kv_pages.dtype, dev, batch, rows, n_q_heads, max_pages)


def poss_pages_remap_workspace_bytes(kv_pages, n_before, n_after, max_pages):
    """Bytes of the `workspace` of poss_pages_remap."""
    return _remap_bytes(kv_pages.shape, kv_pages.dtype, n_before, n_after, max_pages)


def poss_beam_select_workspace_bytes(batch, beams, vocab):
    """Bytes of the `workspace` of poss_beam_select."""
    return _beam_bytes(batch, beams, vocab)


def poss_pages_append(k, v, kv_pages, layer, tables, prefix_len, n_rows=None, status=None):
    """Writes k, v [batch][rows][kv heads][d] behind every sequence's first prefix_len[b] slots in layer `layer`."""
    (pool, heads, _, d), dev = _pool(kv_pages)
    b, r = k.shape[0], k.shape[1]
    kp, ld = _rows(k, "k", heads, d, kv_pages.dtype, dev)
    vp, ldv = _rows(v, "v", heads, d, kv_pages.dtype, dev)
    if ldv != ld or v.shape != k.shape:
        raise ValueError("k and v: the same shape and the same strides are wanted")
    mp = tables.shape[1]
    _call(load_library().poss_pages_append(
        pool, layer, kv_pages.data_ptr(), _arg(tables, _I32, (b, mp), "tables", dev), mp, b, r, kp, vp, ld,
        _arg(prefix_len, _I32, (b,), "prefix_len", dev), _opt(n_rows, _I32, (b,), "n_rows", dev),
        _opt(status, _I32, (1,), "status", dev), _raw_stream(dev)), "poss_pages_append")


def poss_paged_tree_attention(q, kv_pages, layer, tables, prefix_len, anc_mask, scale, n_rows=None, out=None,
                              workspace=None, status=None):
    """Tree-masked attention of q [batch][rows][query heads][d] over the pages of layer `layer`; anc_mask int64
    [batch][rows][ceil(rows/64)].  Returns out [batch][rows][query heads][d]; rows behind n_rows[b] are not written."""
    (pool, _, _, d), dev = _pool(kv_pages)
    b, r, hq = q.shape[0], q.shape[1], q.shape[2]
    dtype = kv_pages.dtype
    qp, ld = _rows(q, "q", hq, d, dtype, dev)
    if out is None:
        out = torch.empty((b, r, hq, d), dtype=dtype, device=dev)
    if b == 0 or r == 0:
        return out
    mp = tables.shape[1]
    ws = _scratch(workspace, _attention_bytes(kv_pages.shape, dtype, dev, b, r, hq, mp), dev)
    _call(load_library().poss_paged_tree_attention(
        pool, layer, kv_pages.data_ptr(), _arg(tables, _I32, (b, mp), "tables", dev), mp, b, r, hq, qp, ld,
        _arg(prefix_len, _I32, (b,), "prefix_len", dev), _opt(n_rows, _I32, (b,), "n_rows", dev),
        _arg(anc_mask, _I64, (b, r, (r + 63) // 64), "anc_mask", dev), scale, _arg(out, dtype, (b, r, hq, d), "out", dev),
        ws.data_ptr(), ws.numel(), _opt(status, _I32, (1,), "status", dev), _raw_stream(dev)),
        "poss_paged_tree_attention")
    return out


def poss_pages_compact(kv_pages, tables, prefix_len, path, n_accepted, out_len=None, status=None):
    """Moves every sequence's accepted path behind its committed slots in all layers; path int32 [batch]
    [POSS_MAX_DEPTH + 1], n_accepted int32 [batch].  Returns the new lengths int32 [batch]."""
    (pool, _, _, _), dev = _pool(kv_pages)
    b, mp = tables.shape
    pp = _arg(prefix_len, _I32, (b,), "prefix_len", dev)
    if out_len is None:
        out_len = torch.empty_like(prefix_len)
    _call(load_library().poss_pages_compact(
        pool, kv_pages.data_ptr(), _arg(tables, _I32, (b, mp), "tables", dev), mp, b, pp,
        _arg(path, _I32, (b, POSS_MAX_DEPTH + 1), "path", dev), _arg(n_accepted, _I32, (b,), "n_accepted", dev),
        _arg(out_len, _I32, (b,), "out_len", dev), _opt(status, _I32, (1,), "status", dev), _raw_stream(dev)),
        "poss_pages_compact")
    return out_len


def poss_pages_remap(kv_pages, tables, seq_len, refs, parents=None, room=None, out=None, workspace=None, status=None):
    """Replaces the sequences of `tables` by parents.numel() new ones (poss_paged.h).  Returns a dict of int32 tensors:
    tables, refs, seq_len, n_free (one element; negative: that many pages were missing and nothing changed)."""
    (pool, _, _, _), dev = _pool(kv_pages)
    n0, mp = tables.shape
    n1 = n0 if parents is None else parents.numel()
    pages = kv_pages.shape[1]
    tp = _arg(tables, _I32, (n0, mp), "tables", dev)
    rp = _arg(refs, _I32, (pages,), "refs", dev)
    if out is None:
        out = {"tables": torch.empty_like(tables) if n1 == n0 else tables.new_empty((n1, mp)),
               "refs": torch.empty_like(refs),
               "seq_len": torch.empty_like(seq_len if parents is None else parents), "n_free": refs.new_empty(1)}
    ws = _scratch(workspace, _remap_bytes(kv_pages.shape, kv_pages.dtype, n0, n1, mp), dev)
    _call(load_library().poss_pages_remap(
        pool, kv_pages.data_ptr(), tp, _arg(out["tables"], _I32, (n1, mp), "out tables", dev), mp, n0, n1,
        _arg(seq_len, _I32, (n0,), "seq_len", dev), rp, _arg(out["refs"], _I32, (pages,), "out refs", dev),
        _opt(parents, _I32, (n1,), "parents", dev), _opt(room, _I32, (n1,), "room", dev),
        _arg(out["seq_len"], _I32, (n1,), "out seq_len", dev), _arg(out["n_free"], _I32, (1,), "n_free", dev),
        ws.data_ptr(), ws.numel(), _opt(status, _I32, (1,), "status", dev), _raw_stream(dev)), "poss_pages_remap")
    return out


def poss_beam_select(logits, scores, finished=None, eos=-1, out=None, workspace=None):
    """One beam-search selection: logits [batch][beams][vocab] (fp32 or bf16), scores fp32 [batch][beams], finished int32
    [batch][beams].  Returns a dict of [batch][beams] tensors: tokens, parents, finished (int32) and scores (fp32)."""
    if logits.dim() != 3 or logits.dtype not in _DTYPES:
        raise ValueError("logits: a CUDA tensor [batch][beams][vocab] of fp32 or bf16 is wanted")
    dev = _device(logits, "logits")
    b, k, v = logits.shape
    shape = (b, k)
    sp = _arg(scores, _F32, shape, "scores", dev)
    if out is None:
        like = torch.empty_like
        out = {"tokens": like(scores, dtype=_I32), "parents": like(scores, dtype=_I32), "scores": like(scores),
               "finished": like(scores, dtype=_I32)}
    ws = _scratch(workspace, _beam_bytes(b, k, v), dev)
    _call(load_library().poss_beam_select(
        _arg(logits, logits.dtype, (b, k, v), "logits", dev), _DTYPES[logits.dtype], b, k, v, sp,
        _opt(finished, _I32, shape, "finished", dev), eos, _arg(out["tokens"], _I32, shape, "tokens", dev),
        _arg(out["parents"], _I32, shape, "parents", dev), _arg(out["scores"], _F32, shape, "out scores", dev),
        _arg(out["finished"], _I32, shape, "out finished", dev), ws.data_ptr(), ws.numel(), _raw_stream(dev)),
        "poss_beam_select")
    return out
