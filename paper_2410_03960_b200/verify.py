"""The operators of a verification step over drafted tokens, over torch CUDA tensors: plan_pages, qk_norm_rope (and its
gradient), tree_attention, token_logprobs (and its gradient).  include/swiftkv.h states what each computes.

Argument checks and marshalling only.  Every call queues its work on `stream` (default: the current stream of the tensors'
device) and returns without synchronising; outputs and scratch that the caller does not bring are allocated on that stream, so
that torch does not hand their memory to another one too early.  ValueError: tensors that do not fit together; SwiftKVError:
what the library refuses."""
from __future__ import annotations

from typing import Dict, Optional, Tuple

import torch

from .binding import DTYPE_FP8_E4M3, _DTYPE_CODE, _check, load_library

PAGE_ROWS = 128
_I32, _F32 = torch.int32, torch.float32


class _On:
    """Makes `device` current and `stream` torch's current stream for the length of a call (both only where they are not)."""

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream]):
        self.index = device.index
        self.stream = stream
        self.back = None
        self.context = None

    def __enter__(self) -> int:
        if torch.cuda.current_device() != self.index:
            self.back = torch.cuda.current_device()
            torch.cuda.set_device(self.index)
        try:
            if self.stream is not None:
                if self.stream.device_index != self.index:
                    raise ValueError("the stream belongs to another device than the tensors")
                self.context = torch.cuda.stream(self.stream)
                self.context.__enter__()
                return self.stream.cuda_stream
            return torch._C._cuda_getCurrentRawStream(self.index)
        except BaseException:
            self.__exit__()
            raise

    def __exit__(self, *exc):
        if self.context is not None:
            self.context.__exit__(None, None, None)
        if self.back is not None:
            torch.cuda.set_device(self.back)
        return False


def _want(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _vec(t: torch.Tensor, name: str, n: Optional[int], device: torch.device, dtype: torch.dtype = _I32) -> int:
    """A contiguous vector of `n` elements (None: any) on `device` -> its address."""
    if t.dtype is not dtype or t.dim() != 1 or (n is not None and t.numel() != n) or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: want a contiguous {dtype} vector{'' if n is None else f' of {n}'} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _tensor(t: torch.Tensor, name: str, shape: Tuple[int, ...], device: torch.device, dtype: torch.dtype) -> int:
    """A contiguous tensor of this shape -> its address."""
    if t.dtype is not dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: want a contiguous {dtype} tensor {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _heads(t: torch.Tensor, name: str, device: torch.device, dtype: torch.dtype) -> Tuple[int, int]:
    """[tokens, heads, head_dim] with whole heads side by side and any token stride -> (address, token stride)."""
    if t.dim() != 3 or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name}: want a {dtype} tensor [tokens, heads, head_dim] on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    n, h, d = t.shape
    s0, s1, s2 = t.stride()
    if (s2 != 1 and d > 1) or (s1 != d and h > 1):
        raise ValueError(f"{name}: the heads of a token must be contiguous (strides {t.stride()})")
    return t.data_ptr(), max(s0, h * d) if n <= 1 else s0


def _cuda(t: torch.Tensor, name: str) -> torch.device:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return t.device


def op_status(device=None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """swiftkv_op_status: synchronises the stream; raises SwiftKVError for what the stand-alone operators met on the device since the last call."""
    index = torch.cuda.current_device() if device is None else torch.device(device).index or 0
    with _On(torch.device("cuda", index), stream) as st:
        _check(load_library().swiftkv_op_status(st))


def plan_pages(n_past: torch.Tensor, n_new: torch.Tensor, n_owned: torch.Tensor, block_table: torch.Tensor, free_pages: torch.Tensor,
               n_free: torch.Tensor, max_tokens: Optional[int] = None, out: Optional[Dict[str, torch.Tensor]] = None,
               stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """swiftkv_plan_pages: cache rows of a step's new tokens.  All int32: n_past, n_new, n_owned [n_seqs], block_table
    [n_seqs, max_blocks], free_pages [capacity], n_free [1].  Returns (or fills, with out=) block_table, n_owned, n_free, cu_new,
    slot_map, positions and info; slot_map and positions have room for `max_tokens` new tokens (out given: their own length)."""
    dev = _cuda(n_past, "n_past")
    n = n_past.numel()
    _want(block_table.dim() == 2 and block_table.shape[0] == n, "block_table: want [n_seqs, max_blocks]")
    blocks = block_table.shape[1]
    args = (_vec(n_past, "n_past", n, dev), _vec(n_new, "n_new", n, dev), _vec(n_owned, "n_owned", n, dev), n,
            _tensor(block_table, "block_table", (n, blocks), dev, _I32), blocks, _vec(free_pages, "free_pages", None, dev), free_pages.numel(),
            _vec(n_free, "n_free", 1, dev))
    with _On(dev, stream) as st:
        if out is None:
            if max_tokens is None:
                raise ValueError("max_tokens: the room of slot_map and positions must be given where out is not")
            make = lambda *shape: torch.empty(shape, dtype=_I32, device=dev)  # noqa: E731
            out = {"block_table": make(n, blocks), "n_owned": make(n), "n_free": make(1), "cu_new": make(n + 1), "slot_map": make(max_tokens),
                   "positions": make(max_tokens), "info": make(4)}
        room = out["slot_map"].numel()
        _check(load_library().swiftkv_plan_pages(
            *args, _tensor(out["block_table"], "out block_table", (n, blocks), dev, _I32), _vec(out["n_owned"], "out n_owned", n, dev),
            _vec(out["n_free"], "out n_free", 1, dev), _vec(out["cu_new"], "out cu_new", n + 1, dev), _vec(out["slot_map"], "out slot_map", room, dev),
            _vec(out["positions"], "out positions", room, dev), room, _vec(out["info"], "out info", 4, dev), st))
    return out


def rope_table(max_pos: int, head_dim: int, theta: float, device="cuda", stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """swiftkv_rope_table: (cos, sin) fp32 [max_pos, head_dim / 2]."""
    device = torch.device(device)
    dev = torch.device("cuda", torch.cuda.current_device() if device.index is None else device.index)
    with _On(dev, stream) as st:
        cos = torch.empty((max_pos, head_dim // 2), dtype=_F32, device=dev)
        sin = torch.empty_like(cos)
        _check(load_library().swiftkv_rope_table(cos.data_ptr(), sin.data_ptr(), max_pos, head_dim, float(theta), st))
    return cos, sin


def _rope_common(q, k, positions, cos, sin, q_gain, k_gain):
    dev = _cuda(q, "q")
    dt = q.dtype
    code = _DTYPE_CODE.get(dt)
    _want(code is not None, f"q: {dt} is not supported")
    qp, qs = _heads(q, "q", dev, dt)
    kp, ks = _heads(k, "k", dev, dt)
    n, n_q, hd = q.shape
    n_kv = k.shape[1]
    _want(k.shape[0] == n and k.shape[2] == hd, "q and k must have the same tokens and head_dim")
    _want(cos.dim() == 2 and hd % 2 == 0, "cos, sin: want [max_pos, head_dim / 2]")
    max_pos = cos.shape[0]
    tables = (_vec(positions, "positions", n, dev), _tensor(cos, "cos", (max_pos, hd // 2), dev, _F32), _tensor(sin, "sin", (max_pos, hd // 2), dev, _F32), max_pos)
    gains = tuple(None if g is None else _vec(g, "gain", hd, dev, dt) for g in (q_gain, k_gain))
    return dev, dt, code, (qp, qs), (kp, ks), n, n_q, n_kv, hd, tables, gains


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, cos: torch.Tensor, sin: torch.Tensor, *,
                 k_cache: torch.Tensor, v_cache: torch.Tensor, q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None,
                 eps: float = 1e-5, slot_map: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """swiftkv_qk_norm_rope: q [T, n_q, hd], k, v [T, n_kv, hd] (slices of wider rows are fine); k_cache, v_cache [rows, n_kv, hd] of
    q's type, or uint8 codes with k_scale, v_scale [rows]; positions, slot_map int32 [T].  Returns the rotated queries (q_out, which
    may be q); keys and values go to the cache rows."""
    dev, dt, code, (qp, qs), (kp, ks), n, n_q, n_kv, hd, (pos, cp, sp, max_pos), (qg, kg) = _rope_common(q, k, positions, cos, sin, q_gain, k_gain)
    vp, vs = _heads(v, "v", dev, dt)
    _want(v.shape == k.shape, "v must have k's shape")
    fp8 = k_scale is not None or v_scale is not None
    _want(not fp8 or (k_scale is not None and v_scale is not None), "k_scale and v_scale go together")
    rows = k_cache.shape[0]
    cdt = torch.uint8 if fp8 else dt
    kc, vc = _tensor(k_cache, "k_cache", (rows, n_kv, hd), dev, cdt), _tensor(v_cache, "v_cache", (rows, n_kv, hd), dev, cdt)
    ksc, vsc = (_vec(k_scale, "k_scale", rows, dev, _F32), _vec(v_scale, "v_scale", rows, dev, _F32)) if fp8 else (None, None)
    slots = None if slot_map is None else _vec(slot_map, "slot_map", n, dev)
    with _On(dev, stream) as st:
        if q_out is None:
            q_out = torch.empty((n, n_q, hd), dtype=dt, device=dev)
        op, os = _heads(q_out, "q_out", dev, dt)
        _want(q_out.shape == q.shape, "q_out must have q's shape")
        _check(load_library().swiftkv_qk_norm_rope(qp, qs, kp, ks, vp, vs, code, n, n_q, n_kv, hd, qg, kg, eps, pos, cp, sp, max_pos, op, os, kc, vc,
                                                  ksc, vsc, rows, slots, st))
    return q_out


def qk_norm_rope_bwd(dq: torch.Tensor, dk: torch.Tensor, q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, cos: torch.Tensor,
                     sin: torch.Tensor, *, q_gain: Optional[torch.Tensor] = None, k_gain: Optional[torch.Tensor] = None, eps: float = 1e-5,
                     out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None, stream: Optional[torch.cuda.Stream] = None):
    """swiftkv_qk_norm_rope_bwd: gradients of the rotated queries and keys (contiguous [T, heads, hd]) -> (dq, dk of the inputs, gain
    gradients fp32 [hd] or None).  out: two tensors for the first two (dq and dk themselves are fine)."""
    dev, dt, code, (qp, qs), (kp, ks), n, n_q, n_kv, hd, (pos, cp, sp, max_pos), (qg, kg) = _rope_common(q, k, positions, cos, sin, q_gain, k_gain)
    dqp, dkp = _tensor(dq, "dq", (n, n_q, hd), dev, dt), _tensor(dk, "dk", (n, n_kv, hd), dev, dt)
    lib = load_library()
    with _On(dev, stream) as st:
        if out is None:
            out = (torch.empty((n, n_q, hd), dtype=dt, device=dev), torch.empty((n, n_kv, hd), dtype=dt, device=dev))
        o0, o1 = _tensor(out[0], "out[0]", (n, n_q, hd), dev, dt), _tensor(out[1], "out[1]", (n, n_kv, hd), dev, dt)
        dqg = None if qg is None else torch.empty(hd, dtype=_F32, device=dev)
        dkg = None if kg is None else torch.empty(hd, dtype=_F32, device=dev)
        nbytes = lib.swiftkv_qk_norm_rope_bwd_scratch_bytes(hd)
        scratch = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=dev)
        _check(lib.swiftkv_qk_norm_rope_bwd(dqp, dkp, qp, qs, kp, ks, code, n, n_q, n_kv, hd, qg, kg, eps, pos, cp, sp, max_pos, o0, o1,
                                            None if dqg is None else dqg.data_ptr(), None if dkg is None else dkg.data_ptr(), scratch.data_ptr(), nbytes, st))
    return out[0], out[1], dqg, dkg


def tree_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, n_past: torch.Tensor, cu_new: torch.Tensor, max_new: int,
                   max_kv: int, *, block_table: Optional[torch.Tensor] = None, row0: Optional[torch.Tensor] = None,
                   tree_mask: Optional[torch.Tensor] = None, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None,
                   softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """swiftkv_tree_attention: q [T, n_q, hd]; k_cache, v_cache [rows, n_kv, hd] of q's type, or uint8 codes with k_scale, v_scale
    [rows]; n_past [n_seqs], cu_new [n_seqs + 1], block_table [n_seqs, max_blocks] or row0 [n_seqs], tree_mask [T, words], all int32.
    max_new / max_kv bound the new tokens and all tokens of any sequence.  Returns out [T, n_q, hd]; fills lse [T, n_q] if given."""
    dev = _cuda(q, "q")
    dt = q.dtype
    code = _DTYPE_CODE.get(dt)
    _want(code is not None, f"q: {dt} is not supported")
    qp, qs = _heads(q, "q", dev, dt)
    t, n_q, hd = q.shape
    _want(k_cache.dim() == 3 and k_cache.shape[2] == hd, "k_cache: want [rows, n_kv, head_dim]")
    rows, n_kv = k_cache.shape[0], k_cache.shape[1]
    fp8 = k_scale is not None or v_scale is not None
    _want(not fp8 or (k_scale is not None and v_scale is not None), "k_scale and v_scale go together")
    cdt = torch.uint8 if fp8 else dt
    kc, vc = _tensor(k_cache, "k_cache", (rows, n_kv, hd), dev, cdt), _tensor(v_cache, "v_cache", (rows, n_kv, hd), dev, cdt)
    ksc, vsc = (_vec(k_scale, "k_scale", rows, dev, _F32), _vec(v_scale, "v_scale", rows, dev, _F32)) if fp8 else (None, None)
    n_seqs = n_past.numel()
    past, cu = _vec(n_past, "n_past", n_seqs, dev), _vec(cu_new, "cu_new", n_seqs + 1, dev)
    table, blocks, first, mask, words = None, 0, None, None, 0
    if block_table is not None:
        _want(block_table.dim() == 2, "block_table: want [n_seqs, max_blocks]")
        blocks = block_table.shape[1]
        table = _tensor(block_table, "block_table", (n_seqs, blocks), dev, _I32)
    if row0 is not None:
        first = _vec(row0, "row0", n_seqs, dev)
    if tree_mask is not None:
        _want(tree_mask.dim() == 2, "tree_mask: want [tokens, words]")
        words = tree_mask.shape[1]
        mask = _tensor(tree_mask, "tree_mask", (t, words), dev, _I32)
    lib = load_library()
    with _On(dev, stream) as st:
        if out is None:
            out = torch.empty((t, n_q, hd), dtype=dt, device=dev)
        op = _tensor(out, "out", (t, n_q, hd), dev, dt)
        lp = None if lse is None else _tensor(lse, "lse", (t, n_q), dev, _F32)
        nbytes = lib.swiftkv_tree_attention_scratch_bytes(t, max_kv, n_q, hd)
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
        _check(lib.swiftkv_tree_attention(qp, qs, code, kc, vc, DTYPE_FP8_E4M3 if fp8 else code, ksc, vsc, rows, table, blocks, first, past, cu, mask, words,
                                          op, lp, n_seqs, t, max_new, max_kv, n_q, n_kv, hd, softmax_scale, None if scratch is None else scratch.data_ptr(),
                                          nbytes, st))
    return out


def _logits(logits: torch.Tensor):
    dev = _cuda(logits, "logits")
    code = _DTYPE_CODE.get(logits.dtype)
    _want(code is not None, f"logits: {logits.dtype} is not supported")
    _want(logits.dim() == 2 and (logits.stride(1) == 1 or logits.shape[1] == 1), "logits: want [rows, vocab] with contiguous rows")
    rows, vocab = logits.shape
    return dev, code, rows, vocab, max(logits.stride(0), vocab) if rows <= 1 else logits.stride(0)


def token_logprobs(logits: torch.Tensor, targets: Optional[torch.Tensor] = None, *, top_k: int = 0, temperature: float = 1.0,
                   out: Optional[Dict[str, torch.Tensor]] = None, stream: Optional[torch.cuda.Stream] = None) -> Dict[str, torch.Tensor]:
    """swiftkv_token_logprobs: logits [rows, vocab] (rows may be slices of wider ones), targets int32 [rows].  Returns (or fills, with
    out=) logprob, entropy, lse fp32 [rows], and top_ids int32 / top_logprobs fp32 [rows, top_k] where top_k > 0."""
    dev, code, rows, vocab, stride = _logits(logits)
    tgt = None if targets is None else _vec(targets, "targets", rows, dev)
    with _On(dev, stream) as st:
        if out is None:
            out = {name: torch.empty(rows, dtype=_F32, device=dev) for name in ("logprob", "entropy", "lse")}
            if top_k > 0:
                out["top_ids"] = torch.empty((rows, top_k), dtype=_I32, device=dev)
                out["top_logprobs"] = torch.empty((rows, top_k), dtype=_F32, device=dev)
        ids, lps = None, None
        if top_k > 0:
            ids, lps = _tensor(out["top_ids"], "top_ids", (rows, top_k), dev, _I32), _tensor(out["top_logprobs"], "top_logprobs", (rows, top_k), dev, _F32)
        _check(load_library().swiftkv_token_logprobs(logits.data_ptr(), stride, code, tgt, rows, vocab, temperature, top_k,
                                                    _vec(out["logprob"], "logprob", rows, dev, _F32), _vec(out["entropy"], "entropy", rows, dev, _F32),
                                                    _vec(out["lse"], "lse", rows, dev, _F32), ids, lps, st))
    return out


def token_logprobs_bwd(logits: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, entropy: Optional[torch.Tensor], grad_logprob: torch.Tensor,
                       grad_entropy: Optional[torch.Tensor] = None, *, temperature: float = 1.0, out: Optional[torch.Tensor] = None,
                       stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """swiftkv_token_logprobs_bwd: the gradient with respect to the logits, in their type (out: a tensor of their shape, the logits
    themselves included).  lse and entropy as token_logprobs gave them; entropy may be None where grad_entropy is."""
    dev, code, rows, vocab, stride = _logits(logits)
    args = (_vec(targets, "targets", rows, dev), rows, vocab, temperature, _vec(lse, "lse", rows, dev, _F32),
            None if entropy is None else _vec(entropy, "entropy", rows, dev, _F32), _vec(grad_logprob, "grad_logprob", rows, dev, _F32),
            None if grad_entropy is None else _vec(grad_entropy, "grad_entropy", rows, dev, _F32))
    with _On(dev, stream) as st:
        if out is None:
            out = torch.empty((rows, vocab), dtype=logits.dtype, device=dev)
        odev, ocode, orows, ovocab, ostride = _logits(out)
        _want(odev == dev and ocode == code and orows == rows and ovocab == vocab, "out must have the logits' shape, type and device")
        _check(load_library().swiftkv_token_logprobs_bwd(logits.data_ptr(), stride, code, *args, out.data_ptr(), ostride, st))
    return out
