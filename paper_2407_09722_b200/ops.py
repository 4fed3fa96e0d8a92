"""Operators around a decoder that the caller runs: the binding of mtad_paged_append, mtad_paged_attention, mtad_paged_evict,
mtad_accept_chain and mtad_accept_chain_spd (see include/mtad.h for what each computes).

They take torch tensors, allocate what is not handed in (outputs, scratch) from torch's allocator on the stream they run on, and
enqueue on the current stream of the tensors' device unless `stream` says otherwise.  Argument errors raise MtadError with the library's
code, or ValueError where a tensor has the wrong device, type or layout.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import struct
from typing import Optional, Tuple

import torch

from . import binding as B

MTAD_BF16, MTAD_F16, MTAD_F32 = 0, 1, 2
_DTYPE = {torch.bfloat16: MTAD_BF16, torch.float16: MTAD_F16, torch.float32: MTAD_F32}


class PagedKV(C.Structure):
    _fields_ = [("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("table", C.c_void_p),
                ("page_stride", C.c_int64), ("head_stride", C.c_int64), ("slot_stride", C.c_int64), ("table_stride", C.c_int64),
                ("dtype", C.c_int32), ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("max_pages", C.c_int32)]


class PagedRows(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("lens", "n_rows", "pos", "q", "k", "v", "q_out", "status")] + \
               [(n, C.c_int64) for n in ("q_stride_seq", "q_stride_row", "q_stride_head", "kv_stride_seq", "kv_stride_row",
                                         "kv_stride_head", "out_stride_seq", "out_stride_row", "out_stride_head")] + \
               [(n, C.c_int32) for n in ("dtype", "batch", "rows", "n_q_heads")] + [("rope_base", C.c_float)]


class PagedAttn(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("lens", "n_rows", "q", "out", "lse", "weights", "status")] + \
               [(n, C.c_int64) for n in ("q_stride_seq", "q_stride_row", "q_stride_head", "out_stride_seq", "out_stride_row",
                                         "out_stride_head", "weights_stride_seq", "weights_stride_head")] + \
               [(n, C.c_int32) for n in ("batch", "rows", "n_q_heads", "window", "sinks", "max_len")] + [("scale", C.c_float)]


class PagedEviction(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("lens", "scores", "kept", "new_lens", "scores_out", "status")] + \
               [(n, C.c_int64) for n in ("scores_stride_seq", "scores_stride_head", "out_stride_seq", "out_stride_head")] + \
               [(n, C.c_int32) for n in ("batch", "max_len", "keep", "first", "recent")]


class AcceptRows(C.Structure):
    _fields_ = [("logits", C.c_void_p)] + \
               [(n, C.c_int64) for n in ("logits_stride_seq", "logits_stride_row", "draft_stride_seq", "draft_stride_row")] + \
               [(n, C.c_void_p) for n in ("draft_tok", "n_draft", "last_uniform")] + \
               [(n, C.c_int32) for n in ("dtype", "batch", "gamma", "vocab")] + [("temperature", C.c_float), ("draft_temperature", C.c_float)]


# The argument blocks above as the bytes that a call passes (packing them costs a fraction of filling a ctypes structure, and a call of
# a few microseconds on the device is bound by its host side).
_KV, _ROWS, _ATTN = struct.Struct("@3P4q6i"), struct.Struct("@8P9q4if4x"), struct.Struct("@7P8q6if4x")
_EVICT, _ACCEPT = struct.Struct("@6P4q5i4x"), struct.Struct("@P4q3P4i2f")
assert [x.size for x in (_KV, _ROWS, _ATTN, _EVICT, _ACCEPT)] == [C.sizeof(x) for x in (PagedKV, PagedRows, PagedAttn, PagedEviction, AcceptRows)]


class _Entry:
    """The entry points with their argument blocks as bytes."""

    def __init__(self):
        lib, P, Y, I = B.load_library(), C.c_void_p, C.c_char_p, C.c_int

        def entry(name, *args):
            return C.CFUNCTYPE(I, *args)((name, lib))

        self.append = entry("mtad_paged_append", Y, Y, P)
        self.attention_workspace = entry("mtad_paged_attention_workspace", Y, Y, P)
        self.attention = entry("mtad_paged_attention", Y, Y, P, C.c_size_t, P)
        self.evict = entry("mtad_paged_evict", Y, Y, P)
        self.accept_chain = entry("mtad_accept_chain", Y, P, C.c_float, P, P)
        self.accept_chain_spd = entry("mtad_accept_chain_spd", Y, P, P, P, P)
        self.cuda_error = entry("mtad_ops_cuda_error")


_entry: Optional[_Entry] = None


def _lib() -> _Entry:
    global _entry
    if _entry is None:
        _entry = _Entry()
    return _entry


def _check(rc: int, where: str):
    if rc != B.MTAD_OK:
        raise B.MtadError(rc, where, _lib().cuda_error() if rc == B.MTAD_E_CUDA else 0)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _ptr(t: Optional[torch.Tensor], dtype, device: int, shape, what: str) -> int:
    """Device pointer of an optional contiguous tensor of that type and shape, 0 for none."""
    if t is None:
        return 0
    if t.dtype != dtype or t.get_device() != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: expected {dtype} {tuple(shape)}, contiguous, on cuda:{device}; got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _on(device: int, stream) -> Tuple[int, Optional[contextlib.ExitStack]]:
    """The stream of a call and, where the device or the stream is not the current one, what makes it so (scratch and outputs are
    allocated on the stream that uses them)."""
    if device < 0:
        raise ValueError("the operators run on CUDA tensors only")
    if stream is None and device == torch._C._cuda_getDevice():
        return torch._C._cuda_getCurrentRawStream(device), None
    with contextlib.ExitStack() as stack:
        stack.enter_context(torch.cuda.device(device))
        if stream is not None:
            if not isinstance(stream, torch.cuda.Stream):
                stream = torch.cuda.ExternalStream(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream), device=device)
            stack.enter_context(torch.cuda.stream(stream))
        return torch._C._cuda_getCurrentRawStream(device), stack.pop_all()


def _pages(k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, batch: int):
    """The argument block of the pages, their device, (kv heads, head_dim), and the slots that a table row can hold."""
    shape, stride, dtype, device = k_pages.shape, k_pages.stride(), k_pages.dtype, k_pages.get_device()
    if len(shape) != 4 or v_pages.shape != shape or v_pages.stride() != stride or v_pages.dtype != dtype or v_pages.get_device() != device:
        raise ValueError("k_pages and v_pages: [pages, kv heads, slots of a page, head_dim], alike in shape, strides, type and device")
    if table.dim() != 2 or table.dtype != torch.int32 or table.get_device() != device or table.stride(1) != 1 or table.shape[0] < batch:
        raise ValueError("table: int32 [sequences, pages] on the pages' device, a row for every sequence, a row contiguous")
    if stride[3] != 1 or dtype not in _DTYPE:
        raise ValueError("pages hold rows of bf16 or fp16 that are contiguous")
    n, h, ps, hd = shape
    wide = table.shape[1]
    return (_KV.pack(k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), stride[0], stride[1], stride[2], max(table.stride(0), wide),
                     _DTYPE[dtype], n, ps, h, hd, wide), device, h, hd, wide * ps)


def _like(t: torch.Tensor) -> torch.Tensor:
    """Contiguous memory of t's shape."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _rows(t: torch.Tensor, what: str, lead, hd: int, device: int) -> Tuple[int, int, int]:
    """Strides of [sequences, rows, heads, head_dim] rows."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 4 or shape[:2] != lead or shape[3] != hd or stride[3] != 1 or t.get_device() != device:
        raise ValueError(f"{what}: [sequences, rows, heads, head_dim] with contiguous heads on the pages' device, got {tuple(shape)}")
    return stride[:3]


def paged_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                 table: torch.Tensor, lens: torch.Tensor, *, n_rows: Optional[torch.Tensor] = None,
                 pos: Optional[torch.Tensor] = None, rope_base: float = 0.0, q_out: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """New rows [sequences, rows, heads, head_dim] enter the cache at slots lens - rows .. lens - 1; returns the turned queries."""
    lead = k.shape[:2]
    b, r = lead if k.dim() == 4 else (0, 0)
    kv, dev, hkv, hd, _ = _pages(k_pages, v_pages, table, b)
    ks, dtype = _rows(k, "k", lead, hd, dev), k.dtype
    _need(_rows(v, "v", lead, hd, dev) == ks and v.shape == k.shape and v.dtype == dtype, "v: like k in shape, strides and type")
    _need(k.shape[2] == hkv and dtype in _DTYPE, "k: the pages' heads, bf16, fp16 or fp32")
    raw, on = _on(dev, stream)
    try:
        hq, qs, os_, qp, op = 0, (0, 0, 0), (0, 0, 0), 0, 0
        if q is not None:
            qs, hq, qp = _rows(q, "q", lead, hd, dev), q.shape[2], q.data_ptr()
            _need(q.dtype == dtype, "q: k's type")
            if q_out is None:
                q_out, os_ = k_pages.new_empty(q.shape), (r * hq * hd, hq * hd, hd)
            else:
                os_ = _rows(q_out, "q_out", lead, hd, dev)
                _need(q_out.dtype == k_pages.dtype and q_out.shape[2] == hq, "q_out: the pages' type, q's heads")
            op = q_out.data_ptr()
        one = (b,)
        a = _ROWS.pack(_ptr(lens, torch.int32, dev, one, "lens"), _ptr(n_rows, torch.int32, dev, one, "n_rows"),
                       _ptr(pos, torch.int32, dev, one, "pos"), qp, k.data_ptr(), v.data_ptr(), op,
                       _ptr(status, torch.int32, dev, one, "status"), *qs, *ks, *os_, _DTYPE[dtype], b, r, hq, rope_base)
        _check(_lib().append(kv, a, raw), "mtad_paged_append")
    finally:
        if on is not None:
            on.close()
    return q_out if q is not None else None


def paged_attention(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, *,
                    n_rows: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0, scale: float = 0.0,
                    weights: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, return_lse: bool = False, max_len: Optional[int] = None,
                    status: Optional[torch.Tensor] = None, stream=None):
    """Attention of the last rows of every sequence, q [sequences, rows, heads, head_dim], over its slots.  `weights` [sequences, kv
    heads, slots] fp32 accumulates the attention that each slot drew.  `max_len` (default: all that the table can hold) bounds
    the lengths: the tighter, the less scratch and the better the launch fits.  Returns the output, with return_lse also the
    log of the softmax sums [sequences, rows, heads]."""
    shape = q.shape
    lead = shape[:2]
    b, r, hq = shape[:3] if q.dim() == 4 else (0, 0, 0)
    kv, dev, hkv, hd, most = _pages(k_pages, v_pages, table, b)
    qs = _rows(q, "q", lead, hd, dev)
    _need(q.dtype == k_pages.dtype, "q: the pages' type")
    if max_len is None or max_len > most:
        max_len = most
    raw, on = _on(dev, stream)
    try:
        if out is None:
            out, os_ = _like(q), (r * hq * hd, hq * hd, hd)
        else:
            os_ = _rows(out, "out", lead, hd, dev)
            _need(out.dtype == q.dtype and out.shape[2] == hq and out.data_ptr() != q.data_ptr(), "out: like q, in memory of its own")
        if lse is not None:
            lp = _ptr(lse, torch.float32, dev, (b, r, hq), "lse")
        elif return_lse:
            lse = q.new_empty((b, r, hq), dtype=torch.float32)
            lp = lse.data_ptr()
        else:
            lp = 0
        ws, wp = (0, 0), 0
        if weights is not None:
            _need(weights.dim() == 3 and weights.shape[0] >= b and weights.shape[1] == hkv and weights.shape[2] >= max_len and
                  weights.stride(2) == 1 and weights.dtype == torch.float32 and weights.get_device() == dev,
                  "weights: fp32 [sequences, kv heads, a column for every slot below max_len] on the pages' device")
            ws, wp = weights.stride()[:2], weights.data_ptr()
        one = (b,)
        a = _ATTN.pack(_ptr(lens, torch.int32, dev, one, "lens"), _ptr(n_rows, torch.int32, dev, one, "n_rows"), q.data_ptr(),
                       out.data_ptr(), lp, wp,
                       _ptr(status, torch.int32, dev, one, "status"), *qs, *os_, *ws, b, r, hq, window, sinks, max_len, scale)
        lib, need = _lib(), C.c_size_t(0)
        _check(lib.attention_workspace(kv, a, C.addressof(need)), "mtad_paged_attention")
        size = need.value
        if size:
            scratch = q.new_empty(size, dtype=torch.uint8)
            _check(lib.attention(kv, a, scratch.data_ptr(), size, raw), "mtad_paged_attention")
        else:
            _check(lib.attention(kv, a, None, 0, raw), "mtad_paged_attention")
    finally:
        if on is not None:
            on.close()
    return (out, lse) if return_lse else out


def paged_evict(k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, scores: torch.Tensor, keep: int,
                *, first: int = 0, recent: int = 0, kept: Optional[torch.Tensor] = None, new_lens: Optional[torch.Tensor] = None,
                scores_out: Optional[torch.Tensor] = None, max_len: Optional[int] = None, status: Optional[torch.Tensor] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Cuts sequences longer than `keep` back to the first, the last and the best-scored slots of every KV head; returns the former
    slots [sequences, kv heads, keep] and the new lengths."""
    b = lens.shape[0] if lens.dim() == 1 else 0
    kv, dev, hkv, _, most = _pages(k_pages, v_pages, table, b)

    def columns(t, what, n):
        shape, stride = t.shape, t.stride()
        if len(shape) != 3 or shape[0] != b or shape[1] != hkv or shape[2] < n or stride[2] != 1 or t.dtype != torch.float32 or t.get_device() != dev:
            raise ValueError(f"{what}: fp32 [sequences, kv heads, at least {n} slots] on the pages' device")
        return stride[:2]

    max_len = min(most, scores.shape[2] if max_len is None and scores.dim() == 3 else max_len or 0)
    ss, os_ = columns(scores, "scores", max_len), (0, 0)
    if scores_out is not None:
        os_ = columns(scores_out, "scores_out", min(keep, max_len))
        _need(scores_out.data_ptr() != scores.data_ptr() or os_ == ss, "scores_out: scores itself, or memory of its own")
    raw, on = _on(dev, stream)
    try:
        one, places = (b,), (b, hkv, max(keep, 0))
        lens_at = _ptr(lens, torch.int32, dev, one, "lens")
        if kept is None:
            kept = lens.new_empty(places)
            kept_at = kept.data_ptr()
        else:
            kept_at = _ptr(kept, torch.int32, dev, places, "kept")
        if new_lens is None:
            new_lens = torch.empty_like(lens)
            new_at = new_lens.data_ptr()
        else:
            new_at = _ptr(new_lens, torch.int32, dev, one, "new_lens")
        a = _EVICT.pack(lens_at, scores.data_ptr(), kept_at, new_at, 0 if scores_out is None else scores_out.data_ptr(),
                        _ptr(status, torch.int32, dev, one, "status"), *ss, *os_, b, max_len, keep, first, recent)
        _check(_lib().evict(kv, a, raw), "mtad_paged_evict")
    finally:
        if on is not None:
            on.close()
    return kept, new_lens


def _accept(logits, draft_tok, last_uniform, out, n_draft, temperature, draft_rows=None, draft_temperature=1.0):
    shape, stride, dev, dtype = logits.shape, logits.stride(), logits.get_device(), logits.dtype
    _need(len(shape) == 3 and stride[2] == 1 and dtype in _DTYPE, "logits: [sequences, drafted tokens + 1, vocab]")
    b, r, v = shape
    _need(out.B == b and out.N == r - 1 and out.D == r - 1 and out.buf.get_device() == dev, "out: ResultBuffers(sequences, gamma, gamma)")
    ds = (0, 0, 0)
    if draft_rows is not None:
        ds = draft_rows.stride()
        _need(draft_rows.shape == (b, r - 1, v) and ds[2] == 1 and draft_rows.dtype == dtype and draft_rows.get_device() == dev,
              "draft_rows: [sequences, drafted tokens, vocab], the logits' type")
    _need(r == 1 or draft_tok is not None, "draft_tok: the drafted tokens")
    return _ACCEPT.pack(logits.data_ptr(), stride[0], stride[1], ds[0], ds[1], _ptr(draft_tok, torch.int32, dev, (b, r - 1), "draft_tok") if r > 1 else 0,
                        _ptr(n_draft, torch.int32, dev, (b,), "n_draft"), _ptr(last_uniform, torch.float32, dev, (b, v), "last_uniform"),
                        _DTYPE[dtype], b, r - 1, v, temperature, draft_temperature)


def accept_chain(logits: torch.Tensor, draft_tok: Optional[torch.Tensor], draft_logq: Optional[torch.Tensor], log_tau: float,
                 last_uniform: torch.Tensor, out: B.ResultBuffers, *, n_draft: Optional[torch.Tensor] = None,
                 temperature: float = 1.0, stream=None):
    """The joint-likelihood threshold rule on the target's rows [sequences, gamma + 1, vocab]; results go to `out`."""
    a, dev = _accept(logits, draft_tok, last_uniform, out, n_draft, temperature), logits.get_device()
    lq = _ptr(draft_logq, torch.float32, dev, (out.B, out.N), "draft_logq") if out.N else 0
    raw, on = _on(dev, stream)
    try:
        _check(_lib().accept_chain(a, lq, log_tau, C.addressof(out.struct), raw), "mtad_accept_chain")
    finally:
        if on is not None:
            on.close()


def accept_chain_spd(logits: torch.Tensor, draft_tok: torch.Tensor, draft_rows: torch.Tensor, accept_uniform: torch.Tensor,
                     last_uniform: torch.Tensor, out: B.ResultBuffers, *, n_draft: Optional[torch.Tensor] = None,
                     temperature: float = 1.0, draft_temperature: float = 1.0, stream=None):
    """The rule of vanilla speculative decoding on the target's rows and the auxiliary model's [sequences, gamma, vocab]."""
    a, dev = _accept(logits, draft_tok, last_uniform, out, n_draft, temperature, draft_rows, draft_temperature), logits.get_device()
    ua = _ptr(accept_uniform, torch.float32, dev, (out.B, out.N), "accept_uniform")
    raw, on = _on(dev, stream)
    try:
        _check(_lib().accept_chain_spd(a, draft_rows.data_ptr(), ua, C.addressof(out.struct), raw), "mtad_accept_chain_spd")
    finally:
        if on is not None:
            on.close()
