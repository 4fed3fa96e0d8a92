"""Operators around a decoder that the caller runs: the binding of mtad_paged_append, mtad_paged_attention, mtad_paged_evict,
mtad_accept_chain and mtad_accept_chain_spd (see include/mtad.h for what each computes).

They take torch tensors, allocate what is not handed in (outputs, scratch) from torch's allocator on the stream they run on, and
enqueue on the current stream of the tensors' device unless `stream` says otherwise.  Argument errors raise MtadError with the library's
code, or ValueError where a tensor has the wrong device, type or layout.
"""
from __future__ import annotations

import ctypes as C
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


_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = B.load_library()
        P, KV = C.c_void_p, C.POINTER(PagedKV)
        lib.mtad_paged_append.argtypes = [KV, C.POINTER(PagedRows), P]
        lib.mtad_paged_attention_workspace.argtypes = [KV, C.POINTER(PagedAttn), C.POINTER(C.c_size_t)]
        lib.mtad_paged_attention.argtypes = [KV, C.POINTER(PagedAttn), P, C.c_size_t, P]
        lib.mtad_paged_evict.argtypes = [KV, C.POINTER(PagedEviction), P]
        lib.mtad_accept_chain.argtypes = [C.POINTER(AcceptRows), P, C.c_float, C.POINTER(B.Result), P]
        lib.mtad_accept_chain_spd.argtypes = [C.POINTER(AcceptRows), P, P, C.POINTER(B.Result), P]
        _ready = lib
    return _ready


def _check(rc: int, where: str):
    if rc != B.MTAD_OK:
        raise B.MtadError(rc, where, _lib().mtad_ops_cuda_error() if rc == B.MTAD_E_CUDA else 0)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _dev(t: Optional[torch.Tensor], dtype, device, what: str, shape=None, contiguous: bool = True) -> Optional[int]:
    """Device pointer of an optional tensor of that type on that device."""
    if t is None:
        return None
    if t.dtype != dtype or t.device != device or (contiguous and not t.is_contiguous()) or (shape is not None and t.shape != shape):
        raise ValueError(f"{what}: expected {dtype} on {device}" + (f" of shape {tuple(shape)}" if shape is not None else "") +
                         (", contiguous" if contiguous else "") + f"; got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


class _On:
    """The device and the stream of a call; the device is made the current one where it is not, scratch belongs to the stream."""
    __slots__ = ("device", "stream", "_dev", "_st")

    def __init__(self, device: torch.device, stream):
        if device.type != "cuda":
            raise ValueError("the operators run on CUDA tensors only")
        self.device, self._dev, self._st = device, None, None
        if device.index != torch.cuda.current_device():
            self._dev = torch.cuda.device(device)
            self._dev.__enter__()
        if stream is None:
            self.stream = torch.cuda.current_stream(device).cuda_stream
        else:
            st = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(
                stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream), device=device)
            self._st = torch.cuda.stream(st)
            self._st.__enter__()
            self.stream = st.cuda_stream

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        if self._st is not None:
            self._st.__exit__(*exc)
        if self._dev is not None:
            self._dev.__exit__(*exc)
        return False


def _kv(k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor) -> PagedKV:
    if k_pages.dim() != 4 or v_pages.shape != k_pages.shape or v_pages.stride() != k_pages.stride() or v_pages.dtype != k_pages.dtype:
        raise ValueError("k_pages and v_pages: [pages, kv heads, slots of a page, head_dim], alike in shape, strides and type")
    if table.dim() != 2 or table.dtype != torch.int32 or table.device != k_pages.device or v_pages.device != k_pages.device:
        raise ValueError("table: int32 [sequences, pages] on the pages' device")
    (n, h, ps, hd), (sp, sh, ss, sd), (tb, te) = k_pages.shape, k_pages.stride(), table.stride()
    if sd != 1 or te != 1 or k_pages.dtype not in _DTYPE:
        raise ValueError("pages hold bf16 or fp16 rows that are contiguous, a table row is contiguous")
    return PagedKV(k_pages.data_ptr(), v_pages.data_ptr(), table.data_ptr(), sp, sh, ss,
                   tb if table.shape[0] > 1 else max(tb, table.shape[1]), _DTYPE[k_pages.dtype], n, ps, h, hd, table.shape[1])


def _rows(t: torch.Tensor, what: str, batch: int, rows: int, hd: int, device) -> Tuple[int, int, int]:
    if t.dim() != 4 or t.shape[0] != batch or t.shape[1] != rows or t.shape[3] != hd or t.stride(3) != 1 or t.device != device:
        raise ValueError(f"{what}: [sequences, rows, heads, head_dim] with contiguous heads on the pages' device, got {tuple(t.shape)}")
    return t.stride()[:3]


def paged_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                 table: torch.Tensor, lens: torch.Tensor, *, n_rows: Optional[torch.Tensor] = None,
                 pos: Optional[torch.Tensor] = None, rope_base: float = 0.0, q_out: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """New rows [sequences, rows, heads, head_dim] enter the cache at slots lens - rows .. lens - 1; returns the turned queries."""
    kv, dev = _kv(k_pages, v_pages, table), k_pages.device
    b, r, hkv, hd = k.shape if k.dim() == 4 else (0, 0, 0, 0)
    ks = _rows(k, "k", b, r, kv.head_dim, dev)
    _need(_rows(v, "v", b, r, hd, dev) == ks and v.shape == k.shape and v.dtype == k.dtype, "v: like k in shape, strides and type")
    _need(hkv == kv.n_kv_heads and k.dtype in _DTYPE and table.shape[0] >= b, "k: the pages' heads, a table row for every sequence")
    hq, qs, os_ = 0, (0, 0, 0), (0, 0, 0)
    with _On(dev, stream) as on:
        if q is not None:
            qs, hq = _rows(q, "q", b, r, hd, dev), q.shape[2]
            _need(q.dtype == k.dtype, "q: k's type")
            if q_out is None:
                q_out = torch.empty(b, r, hq, hd, dtype=k_pages.dtype, device=dev)
            os_ = _rows(q_out, "q_out", b, r, hd, dev)
            _need(q_out.dtype == k_pages.dtype and q_out.shape[2] == hq, "q_out: the pages' type, q's heads")
        one = (b,)
        a = PagedRows(_dev(lens, torch.int32, dev, "lens", one), _dev(n_rows, torch.int32, dev, "n_rows", one),
                      _dev(pos, torch.int32, dev, "pos", one), None if q is None else q.data_ptr(), k.data_ptr(), v.data_ptr(),
                      None if q is None else q_out.data_ptr(), _dev(status, torch.int32, dev, "status", one),
                      *qs, *ks, *os_, _DTYPE[k.dtype], b, r, hq, rope_base)
        _check(_lib().mtad_paged_append(kv, a, on.stream), "mtad_paged_append")
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
    kv, dev = _kv(k_pages, v_pages, table), k_pages.device
    b, r, hq, hd = q.shape if q.dim() == 4 else (0, 0, 0, 0)
    qs = _rows(q, "q", b, r, kv.head_dim, dev)
    _need(q.dtype == k_pages.dtype and table.shape[0] >= b, "q: the pages' type, a table row for every sequence")
    max_len = kv.max_pages * kv.page_size if max_len is None else min(max_len, kv.max_pages * kv.page_size)
    with _On(dev, stream) as on:
        if out is None:
            out = torch.empty(b, r, hq, hd, dtype=q.dtype, device=dev)
        os_ = _rows(out, "out", b, r, hd, dev)
        _need(out.dtype == q.dtype and out.shape[2] == hq and out.data_ptr() != q.data_ptr(), "out: like q, in memory of its own")
        if return_lse and lse is None:
            lse = torch.empty(b, r, hq, dtype=torch.float32, device=dev)
        ws = (0, 0)
        if weights is not None:
            _need(weights.dim() == 3 and weights.shape[0] >= b and weights.shape[1] == kv.n_kv_heads and weights.shape[2] >= max_len
                  and weights.stride(2) == 1, "weights: fp32 [sequences, kv heads, a column for every slot below max_len]")
            ws = weights.stride()[:2]
        one = (b,)
        a = PagedAttn(_dev(lens, torch.int32, dev, "lens", one), _dev(n_rows, torch.int32, dev, "n_rows", one), q.data_ptr(),
                      out.data_ptr(), _dev(lse, torch.float32, dev, "lse", (b, r, hq)),
                      _dev(weights, torch.float32, dev, "weights", None, False), _dev(status, torch.int32, dev, "status", one),
                      *qs, *os_, *ws, b, r, hq, window, sinks, max_len, scale)
        lib, need = _lib(), C.c_size_t(0)
        _check(lib.mtad_paged_attention_workspace(kv, a, need), "mtad_paged_attention")
        scratch = torch.empty(need.value, dtype=torch.uint8, device=dev) if need.value else None
        _check(lib.mtad_paged_attention(kv, a, None if scratch is None else scratch.data_ptr(), need.value, on.stream),
               "mtad_paged_attention")
    return (out, lse) if return_lse else out


def paged_evict(k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, scores: torch.Tensor, keep: int,
                *, first: int = 0, recent: int = 0, kept: Optional[torch.Tensor] = None, new_lens: Optional[torch.Tensor] = None,
                scores_out: Optional[torch.Tensor] = None, max_len: Optional[int] = None, status: Optional[torch.Tensor] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Cuts sequences longer than `keep` back to the first, the last and the best-scored slots of every KV head; returns the former
    slots [sequences, kv heads, keep] and the new lengths."""
    kv, dev = _kv(k_pages, v_pages, table), k_pages.device
    b = lens.shape[0] if lens.dim() == 1 else 0
    _need(scores.dim() == 3 and scores.shape[0] == b and scores.shape[1] == kv.n_kv_heads and scores.stride(2) == 1 and
          table.shape[0] >= b, "scores: fp32 [sequences, kv heads, slots], a table row for every sequence")
    max_len = min(kv.max_pages * kv.page_size, scores.shape[2] if max_len is None else max_len)
    _need(scores.shape[2] >= max_len, "scores: at least max_len slots")
    ss, os_ = scores.stride()[:2], (0, 0)
    if scores_out is not None:
        _need(scores_out.dim() == 3 and scores_out.shape[0] == b and scores_out.shape[1] == kv.n_kv_heads and
              scores_out.shape[2] >= min(keep, max_len) and scores_out.stride(2) == 1, "scores_out: fp32 [sequences, kv heads, at least keep]")
        os_ = scores_out.stride()[:2]
        _need(scores_out.data_ptr() != scores.data_ptr() or os_ == ss, "scores_out: scores itself, or memory of its own")
    with _On(dev, stream) as on:
        if kept is None:
            kept = torch.empty(b, kv.n_kv_heads, max(keep, 0), dtype=torch.int32, device=dev)
        if new_lens is None:
            new_lens = torch.empty(b, dtype=torch.int32, device=dev)
        one = (b,)
        a = PagedEviction(_dev(lens, torch.int32, dev, "lens", one), _dev(scores, torch.float32, dev, "scores", None, False),
                          _dev(kept, torch.int32, dev, "kept", (b, kv.n_kv_heads, max(keep, 0))),
                          _dev(new_lens, torch.int32, dev, "new_lens", one),
                          _dev(scores_out, torch.float32, dev, "scores_out", None, False),
                          _dev(status, torch.int32, dev, "status", one), *ss, *os_, b, max_len, keep, first, recent)
        _check(_lib().mtad_paged_evict(kv, a, on.stream), "mtad_paged_evict")
    return kept, new_lens


def _accept(logits, draft_tok, last_uniform, out, n_draft, temperature, draft_rows=None, draft_temperature=1.0):
    dev = logits.device
    _need(logits.dim() == 3 and logits.stride(2) == 1 and logits.dtype in _DTYPE, "logits: [sequences, drafted tokens + 1, vocab]")
    b, r, v = logits.shape
    _need(out.B == b and out.N == r - 1 and out.D == r - 1 and out.buf.device == dev, "out: ResultBuffers(sequences, gamma, gamma)")
    ds = (0, 0)
    if draft_rows is not None:
        _need(draft_rows.shape == (b, r - 1, v) and draft_rows.stride(2) == 1 and draft_rows.dtype == logits.dtype and
              draft_rows.device == dev, "draft_rows: [sequences, drafted tokens, vocab], the logits' type")
        ds = draft_rows.stride()[:2]
    _need(r == 1 or draft_tok is not None, "draft_tok: the drafted tokens")
    return AcceptRows(logits.data_ptr(), *logits.stride()[:2], *ds, _dev(draft_tok, torch.int32, dev, "draft_tok", (b, r - 1)) if r > 1 else None,
                      _dev(n_draft, torch.int32, dev, "n_draft", (b,)), _dev(last_uniform, torch.float32, dev, "last_uniform", (b, v)),
                      _DTYPE[logits.dtype], b, r - 1, v, temperature, draft_temperature)


def accept_chain(logits: torch.Tensor, draft_tok: Optional[torch.Tensor], draft_logq: Optional[torch.Tensor], log_tau: float,
                 last_uniform: torch.Tensor, out: B.ResultBuffers, *, n_draft: Optional[torch.Tensor] = None,
                 temperature: float = 1.0, stream=None):
    """The joint-likelihood threshold rule on the target's rows [sequences, gamma + 1, vocab]; results go to `out`."""
    with _On(logits.device, stream) as on:
        a = _accept(logits, draft_tok, last_uniform, out, n_draft, temperature)
        lq = _dev(draft_logq, torch.float32, logits.device, "draft_logq", (a.batch, a.gamma)) if a.gamma else None
        _check(_lib().mtad_accept_chain(a, lq, log_tau, out.struct, on.stream), "mtad_accept_chain")


def accept_chain_spd(logits: torch.Tensor, draft_tok: torch.Tensor, draft_rows: torch.Tensor, accept_uniform: torch.Tensor,
                     last_uniform: torch.Tensor, out: B.ResultBuffers, *, n_draft: Optional[torch.Tensor] = None,
                     temperature: float = 1.0, draft_temperature: float = 1.0, stream=None):
    """The rule of vanilla speculative decoding on the target's rows and the auxiliary model's [sequences, gamma, vocab]."""
    with _On(logits.device, stream) as on:
        a = _accept(logits, draft_tok, last_uniform, out, n_draft, temperature, draft_rows, draft_temperature)
        ua = _dev(accept_uniform, torch.float32, logits.device, "accept_uniform", (a.batch, a.gamma))
        _check(_lib().mtad_accept_chain_spd(a, draft_rows.data_ptr(), ua, out.struct, on.stream), "mtad_accept_chain_spd")
