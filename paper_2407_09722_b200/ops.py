"""Operators around a decoder that the caller runs: the tensor form of mtad_paged_append, mtad_paged_attention, mtad_paged_evict,
mtad_accept_chain and mtad_accept_chain_spd (see include/mtad.h for what each computes).

They take torch tensors, allocate what is not handed in (outputs, scratch) from torch's allocator on the stream they run on, and
enqueue on the current stream of the tensors' device unless `stream` says otherwise.  Argument errors raise MtadError with the library's
code, or ValueError where a tensor has the wrong device, type or layout.  They have no backward pass: inputs that require a gradient are
read, outputs do not.  The marshalling is compiled (csrc/ops_py.cpp).
"""
from __future__ import annotations

import ctypes as C
import importlib
import os
from typing import Optional, Tuple

import torch

from . import binding as B

_mod = None


def _ops():
    global _mod
    if _mod is None:
        B.load_library()
        if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_ops.so")):
            raise RuntimeError("_ops.so is missing: run `python -m paper_2407_09722_b200.build` first (there is no fallback path)")
        mod = importlib.import_module("._ops", __package__)
        if mod.torch_version != torch.__version__:
            raise RuntimeError(f"_ops.so was built for another torch ({mod.torch_version}): run `python -m paper_2407_09722_b200.build` again")
        _mod = mod
    return _mod


def _handle(stream) -> Optional[int]:
    return None if stream is None else stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _raise(rc: int, where: str):
    raise B.MtadError(rc, where, B.load_library().mtad_ops_cuda_error() if rc == B.MTAD_E_CUDA else 0)


def paged_append(q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                 table: torch.Tensor, lens: torch.Tensor, *, n_rows: Optional[torch.Tensor] = None,
                 pos: Optional[torch.Tensor] = None, rope_base: float = 0.0, q_out: Optional[torch.Tensor] = None,
                 status: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
    """New rows [sequences, rows, heads, head_dim] enter the cache at slots lens - rows .. lens - 1; returns the turned queries."""
    r = (_mod or _ops()).append(q, k, v, k_pages, v_pages, table, lens, n_rows, pos, rope_base, q_out, status,
                                None if stream is None else _handle(stream))
    if type(r) is int:
        _raise(r, "mtad_paged_append")
    return r if q_out is None or q is None else q_out


def paged_attention(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, *,
                    n_rows: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0, scale: float = 0.0,
                    weights: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                    lse: Optional[torch.Tensor] = None, return_lse: bool = False, max_len: Optional[int] = None,
                    status: Optional[torch.Tensor] = None, stream=None):
    """Attention of the last rows of every sequence, q [sequences, rows, heads, head_dim], over its slots.  `weights` [sequences, kv
    heads, slots] fp32 accumulates the attention that each slot drew (clear what lies behind a length that went down, before other
    tokens take those slots).  `max_len` (default: all that the table can hold) bounds
    the lengths: the tighter, the less scratch and the better the launch fits.  Returns the output, with return_lse also the
    log of the softmax sums [sequences, rows, heads]."""
    r = (_mod or _ops()).attention(q, k_pages, v_pages, table, lens, n_rows, window, sinks, scale, weights, out, lse, return_lse, max_len,
                                   status, None if stream is None else _handle(stream))
    if type(r) is int:
        _raise(r, "mtad_paged_attention")
    return r


def paged_evict(k_pages: torch.Tensor, v_pages: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, scores: torch.Tensor, keep: int,
                *, first: int = 0, recent: int = 0, kept: Optional[torch.Tensor] = None, new_lens: Optional[torch.Tensor] = None,
                scores_out: Optional[torch.Tensor] = None, max_len: Optional[int] = None, status: Optional[torch.Tensor] = None,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Cuts sequences longer than `keep` back to the first, the last and the best-scored slots of every KV head; returns the former
    slots [sequences, kv heads, keep] and the new lengths.  `scores_out`, which may be `scores`, gets the scores of what stays; its columns
    from the new lengths on are left as they were (of accumulated weights: clear them)."""
    r = (_mod or _ops()).evict(k_pages, v_pages, table, lens, scores, keep, first, recent, kept, new_lens, scores_out, max_len, status,
                               None if stream is None else _handle(stream))
    if type(r) is int:
        _raise(r, "mtad_paged_evict")
    return r


def _accept(where, logits, draft_tok, last_uniform, out, n_draft, temperature, stream, *rule):
    if logits.dim() != 3 or out.B != logits.shape[0] or out.N != logits.shape[1] - 1 or out.D != out.N or out.buf.device != logits.device:
        raise ValueError("logits [sequences, gamma + 1, vocab] with out = ResultBuffers(sequences, gamma, gamma) on their device")
    rc = (_mod or _ops()).accept(logits, draft_tok, last_uniform, n_draft, temperature, None if stream is None else _handle(stream),
                                 C.addressof(out.struct), *rule)
    if rc:
        _raise(rc, where)


def accept_chain(logits: torch.Tensor, draft_tok: Optional[torch.Tensor], draft_logq: Optional[torch.Tensor], log_tau: float,
                 last_uniform: torch.Tensor, out: B.ResultBuffers, *, n_draft: Optional[torch.Tensor] = None,
                 temperature: float = 1.0, stream=None):
    """The joint-likelihood threshold rule on the target's rows [sequences, gamma + 1, vocab]; results go to `out`
    (of its out_tok and out_lp the first n_out entries of a sequence)."""
    _accept("mtad_accept_chain", logits, draft_tok, last_uniform, out, n_draft, temperature, stream, draft_logq, log_tau)


def accept_chain_spd(logits: torch.Tensor, draft_tok: torch.Tensor, draft_rows: torch.Tensor, accept_uniform: torch.Tensor,
                     last_uniform: torch.Tensor, out: B.ResultBuffers, *, n_draft: Optional[torch.Tensor] = None,
                     temperature: float = 1.0, draft_temperature: float = 1.0, stream=None):
    """The rule of vanilla speculative decoding on the target's rows and the auxiliary model's [sequences, gamma, vocab]."""
    _accept("mtad_accept_chain_spd", logits, draft_tok, last_uniform, out, n_draft, temperature, stream, draft_rows, accept_uniform,
            draft_temperature)
