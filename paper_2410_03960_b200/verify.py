"""The operators of a verification step over drafted tokens, over torch CUDA tensors: plan_pages, qk_norm_rope (and its
gradient), tree_attention, token_logprobs (and its gradient).  include/swiftkv.h states what each computes.

Argument checks and marshalling only, done in csrc/verify_py.cpp (these calls sit in a serving loop; from Python they would cost
more than the smallest kernels).  Every call queues its work on `stream` (default: the current stream of the tensors' device) and
returns without synchronising; outputs and scratch that the caller does not bring are allocated on that stream, so that torch does
not hand their memory to another one too early.  No tokens or no rows: nothing is queued, and results are empty (gain gradients zero).  ValueError: tensors that do not fit together; SwiftKVError: what the library
refuses."""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional, Tuple

import torch

from .binding import SwiftKVError, _check, load_library

PAGE_ROWS = 128
_I32, _F32 = torch.int32, torch.float32
_EXT = None
_ADDRESSES = ("swiftkv_last_error", "swiftkv_plan_pages", "swiftkv_qk_norm_rope", "swiftkv_qk_norm_rope_bwd", "swiftkv_qk_norm_rope_bwd_scratch_bytes",
              "swiftkv_tree_attention", "swiftkv_tree_attention_scratch_bytes", "swiftkv_token_logprobs", "swiftkv_token_logprobs_bwd")


def _load():
    """The extension, bound to the library's functions; like the library it has no fallback."""
    global _EXT
    if _EXT is None:
        lib = load_library()
        path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_verify.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -m paper_2410_03960_b200.build`")
        try:
            from . import _verify
            built_for = getattr(_verify, "built_for_torch", "another version")
        except ImportError as e:
            raise RuntimeError(f"{path} does not load into torch {torch.__version__} (rebuild it with `python -m paper_2410_03960_b200.build --force`): {e}") from e
        if built_for != torch.__version__:
            raise RuntimeError(f"{path} was built for torch {built_for}, this is {torch.__version__}: rebuild it with `python -m paper_2410_03960_b200.build --force`")
        _verify.bind(SwiftKVError, {name: C.cast(getattr(lib, name), C.c_void_p).value for name in _ADDRESSES})
        _EXT = _verify
    return _EXT


class _On:
    """Makes `stream` torch's current stream (and its device the current one) for the length of a call."""

    def __init__(self, t: torch.Tensor, stream: torch.cuda.Stream):
        if not (isinstance(t, torch.Tensor) and t.is_cuda):
            raise ValueError("want CUDA tensors")
        if stream.device_index != t.get_device():
            raise ValueError("the stream belongs to another device than the tensors")
        self.context = torch.cuda.stream(stream)

    def __enter__(self):
        return self.context.__enter__()

    def __exit__(self, *exc):
        return self.context.__exit__(*exc)


def op_status(device=None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """swiftkv_op_status: synchronises the stream; raises SwiftKVError for what the stand-alone operators met on the device (default: the
    stream's, else the current one) since the last call."""
    index = None if device is None else torch.device(device).index
    if stream is not None:
        if index is not None and index != stream.device_index:
            raise ValueError("the stream belongs to another device")
        index = stream.device_index
    index = torch.cuda.current_device() if index is None else index
    with torch.cuda.device(index):
        _check(load_library().swiftkv_op_status((stream or torch.cuda.current_stream()).cuda_stream))


def plan_pages(n_past: torch.Tensor, n_new: torch.Tensor, n_owned: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor,
               n_free: torch.Tensor, max_tokens: Optional[int] = None, out: Optional[Dict[str, torch.Tensor]] = None,
               stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """swiftkv_plan_pages: cache rows of a step's new tokens.  All int32: n_past, n_new, n_owned [n_seqs], block_table
    [n_seqs, max_blocks], free_pages [capacity], n_free [1].  Returns (or fills, with out=) block_table, n_owned, n_free, cu_new,
    slot_map, positions and info; slot_map and positions have room for `max_tokens` new tokens (out given: their own length)."""
    if stream is not None:
        with _On(n_past, stream):
            return plan_pages(n_past, n_new, n_owned, block_table, free_pages, n_free, max_tokens, out)
    if out is None:
        if max_tokens is None:
            raise ValueError("max_tokens: the room of slot_map and positions must be given where out is not")
        n, dev = n_past.numel(), n_past.device
        make = lambda *shape: torch.empty(shape, dtype=_I32, device=dev)  # noqa: E731
        out = {"block_table": make(*block_table.shape), "n_owned": make(n), "n_free": make(1), "cu_new": make(n + 1), "slot_map": make(max_tokens),
               "positions": make(max_tokens), "info": make(4)}
    (_EXT or _load()).plan_pages(n_past, n_new, n_owned, block_table, free_pages, n_free, out["block_table"], out["n_owned"], out["n_free"], out["cu_new"],
                                 out["slot_map"], out["positions"], out["info"])
    return out


def rope_table(max_pos: int, head_dim: int, theta: float, device="cuda", stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """swiftkv_rope_table: (cos, sin) fp32 [max_pos, head_dim / 2]."""
    device = torch.device(device)
    dev = torch.device("cuda", torch.cuda.current_device() if device.index is None else device.index)
    if stream is not None and stream.device != dev:
        raise ValueError("the stream belongs to another device than the table")
    with torch.cuda.device(dev), torch.cuda.stream(stream):
        cos = torch.empty((max_pos, head_dim // 2), dtype=_F32, device=dev)
        sin = torch.empty_like(cos)
        _check(load_library().swiftkv_rope_table(cos.data_ptr(), sin.data_ptr(), max_pos, head_dim, float(theta), torch.cuda.current_stream().cuda_stream))
    return cos, sin


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor, *,
                 k_cache: torch.Tensor, v_cache: torch.Tensor, q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None,
                 eps: float = 1e-5, slot_map: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """swiftkv_qk_norm_rope: q [T, n_q, hd], k, v [T, n_kv, hd] (slices of wider rows are fine); k_cache, v_cache [rows, n_kv, hd] of
    q's type, or uint8 codes with k_scale, v_scale [rows]; positions, slot_map int32 [T].  Returns the rotated queries (q_out, which
    may be q); keys and values go to the cache rows."""
    if stream is not None:
        with _On(q, stream):
            return qk_norm_rope(q, k, v, positions, cos, sin, k_cache=k_cache, v_cache=v_cache, q_gain=q_gain, k_gain=k_gain, eps=eps, slot_map=slot_map,
                                k_scale=k_scale, v_scale=v_scale, q_out=q_out)
    return (_EXT or _load()).qk_norm_rope(q, k, v, positions, cos, sin, q_gain, k_gain, eps, slot_map, k_cache, v_cache, k_scale, v_scale, q_out)


def qk_norm_rope_bwd(dq: torch.Tensor, dk: torch.Tensor, q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, cos: torch.Tensor,
                     sin: torch.Tensor, *, q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, eps: float = 1e-5,
                     out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream: Optional[torch.cuda.Stream] = None):
    """swiftkv_qk_norm_rope_bwd: gradients of the rotated queries and keys (contiguous [T, heads, hd]) -> (dq, dk of the inputs, gain
    gradients fp32 [hd] or None).  out: two tensors for the first two (dq and dk themselves are fine)."""
    if stream is not None:
        with _On(q, stream):
            return qk_norm_rope_bwd(dq, dk, q, k, positions, cos, sin, q_gain=q_gain, k_gain=k_gain, eps=eps, out=out)
    o0, o1 = (None, None) if out is None else out
    return (_EXT or _load()).qk_norm_rope_bwd(dq, dk, q, k, positions, cos, sin, q_gain, k_gain, eps, o0, o1)


def tree_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, n_past: torch.Tensor, cu_new: torch.Tensor, max_new: int,
                   max_kv: int, *, block_table: Optional[torch.Tensor] = None, row0: Optional[torch.Tensor] = None,
                   tree_mask: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                   softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """swiftkv_tree_attention: q [T, n_q, hd]; k_cache, v_cache [rows, n_kv, hd] of q's type, or uint8 codes with k_scale, v_scale
    [rows]; n_past [n_seqs], cu_new [n_seqs + 1], block_table [n_seqs, max_blocks] or row0 [n_seqs], tree_mask [T, words], all int32.
    max_new / max_kv bound the new tokens and all tokens of any sequence.  Returns out [T, n_q, hd]; fills lse [T, n_q] if given."""
    if stream is not None:
        with _On(q, stream):
            return tree_attention(q, k_cache, v_cache, n_past, cu_new, max_new, max_kv, block_table=block_table, row0=row0, tree_mask=tree_mask, k_scale=k_scale,
                                  v_scale=v_scale, softmax_scale=softmax_scale, out=out, lse=lse)
    return (_EXT or _load()).tree_attention(q, k_cache, v_cache, n_past, cu_new, max_new, max_kv, block_table, row0, tree_mask, k_scale, v_scale, softmax_scale, out, lse)


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, *, top_k: int = 0, temperature: float = 1.0,
                   out: Optional[Dict[str, torch.Tensor]] = None, stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """swiftkv_token_logprobs: logits [rows, vocab] (rows may be slices of wider ones), targets int32 [rows].  Returns (or fills, with
    out=) logprob, entropy, lse fp32 [rows], and top_ids int32 / top_logprobs fp32 [rows, top_k] where top_k > 0."""
    if stream is not None:
        with _On(logits, stream):
            return token_logprobs(logits, targets, top_k=top_k, temperature=temperature, out=out)
    if out is None:
        rows, dev = logits.shape[0], logits.device
        out = {name: torch.empty(rows, dtype=_F32, device=dev) for name in ("logprob", "entropy", "lse")}
        if top_k > 0:
            out["top_ids"] = torch.empty((rows, top_k), dtype=_I32, device=dev)
            out["top_logprobs"] = torch.empty((rows, top_k), dtype=_F32, device=dev)
    (_EXT or _load()).token_logprobs(logits, targets, top_k, temperature, out["logprob"], out["entropy"], out["lse"], out.get("top_ids"), out.get("top_logprobs"))
    return out


def token_logprobs_bwd(logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, entropy: Optional[torch.Tensor], grad_logprob: torch.Tensor,
                       grad_entropy: Optional[torch.Tensor] = None, *, temperature: float = 1.0, out: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """swiftkv_token_logprobs_bwd: the gradient with respect to the logits, in their type (out: a tensor of their shape, the logits
    themselves included).  lse and entropy as token_logprobs gave them; entropy may be None where grad_entropy is."""
    if stream is not None:
        with _On(logits, stream):
            return token_logprobs_bwd(logits, targets, lse, entropy, grad_logprob, grad_entropy, temperature=temperature, out=out)
    return (_EXT or _load()).token_logprobs_bwd(logits, targets, lse, entropy, grad_logprob, grad_entropy, temperature, out)
