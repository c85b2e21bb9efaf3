"""Operators of a serving step: paged caches, rotary positions, attention with
a sliding window and sinks, sampled tokens.

A step of a cached decoder takes them in this order: plan_pages finds pages
and slots for the step's new tokens, rope_append turns their queries and keys
and writes keys and values to the slots (per layer), paged_attention reads
the cache (per layer), sample_tokens draws the next token of every request.
Each is one call of the C ABI (include/streambeam.h, which defines what it
computes) on torch's current stream of its tensors' device; nothing waits,
and every call can be captured into a graph. There are no backward passes.
"""
from __future__ import annotations

import math
import operator
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

from . import _native as N

_HALVES = {torch.bfloat16: N.SB_BF16, torch.float16: N.SB_F16}
_LOGITS = {torch.float32: N.SB_F32, **_HALVES}
_LAYOUTS = {"half": N.SB_ROPE_HALF, "interleaved": N.SB_ROPE_INTERLEAVED}


def _refuse(what):
    raise ValueError(what)


# The current stream's handle and the current device by torch's direct calls:
# the public ones build objects, 3 of a single-token call's 15 microseconds.
_raw_stream, _current = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _call(fn, where, i, *args):
    """fn(*args, stream) on device i and its current stream."""
    if i == _current():
        status = fn(*args, _raw_stream(i))
    else:
        with torch.cuda.device(i):
            status = fn(*args, _raw_stream(i))
    if status != N.SB_OK:
        msg = N.lib().sb_last_error(None)
        raise N.StreambeamError(status, where, msg.decode() if msg else "")


# The checks read each property of a tensor once: a read takes 0.1 us, a call
# with single tokens 10 to 15.
def _whole(t, name, dtype, i, shape):
    """A contiguous array of whole numbers or parameters."""
    if t.dtype != dtype or t.get_device() != i or t.shape != shape or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{i}")
    return t.data_ptr()


def _apart(t, name):
    """A tensor that is written: no two of its elements in one place."""
    if not t.is_contiguous():
        span = 1
        for stride, size in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n > 1):
            if stride < span:
                _refuse(f"{name} is written and its elements overlap")
            span = stride * (size - 1) + span
    return t


def _no_grad(*tensors):
    """Refuses what a backward pass, or a tangent of forward mode, would have to go
    through: inputs, and what is written (None: left out)."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                _refuse("there is no backward pass: call it under torch.no_grad()")
    if forward_ad._current_level >= 0:   # (a dual tensor does not require a gradient)
        for t in tensors:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                _refuse("there is no forward-mode derivative: unpack the dual tensors")


# Tells autograd that tensors were written: one that it has saved is then found
# to have changed, as with torch's own in-place operations. (0.2 us.)
_written = torch._C._increment_version


def _device(t, name):
    i = t.get_device() if t.is_cuda else -1
    if i < 0:
        _refuse(f"{name} must be on a GPU")
    return i


def _heads(t, name, dtype, i, tokens=None, dim=None):
    """Its shape and strides."""
    shape, strides = t.shape, t.stride()
    if len(shape) != 3 or t.dtype != dtype or t.get_device() != i or (strides[2] != 1 and shape[2] > 1):
        _refuse(f"{name} must be a {dtype} tensor [tokens, heads, head_dim] on cuda:{i} with contiguous heads")
    if dim is not None and (shape[0] != tokens or shape[2] != dim):
        _refuse(f"{name} has another number of tokens or another head_dim")
    return shape, strides


def _caches(k_cache, v_cache, dtype, i, heads, dim):
    """Their shape, and the strides of each."""
    shape, kc, vc = k_cache.shape, k_cache.stride(), v_cache.stride()
    for t, name, strides in ((k_cache, "k_cache", kc), (v_cache, "v_cache", vc)):
        if len(strides) != 4 or t.dtype != dtype or t.get_device() != i or strides[3] != 1:
            _refuse(f"{name} must be a {dtype} tensor [pages, page_size, heads, head_dim] on cuda:{i} with contiguous heads")
    if shape != v_cache.shape or shape[3] != dim or (heads is not None and shape[2] != heads):
        _refuse("the caches must have one shape, with the keys' heads and head_dim")
    return shape, kc, vc


def _table(t, i):
    """Its shape and row stride."""
    shape = t.shape
    if len(shape) != 2 or t.dtype != torch.int32 or t.get_device() != i or (shape[1] > 1 and t.stride(1) != 1):
        _refuse(f"table must be an int32 tensor [requests, max_pages] on cuda:{i} with contiguous rows")
    return shape, t.stride(0) if shape[0] > 1 else shape[1]


class PagePlan(NamedTuple):
    """What plan_pages found. lens and n_free are the new state: give them to
    the next call."""
    q_start: torch.Tensor     # [requests + 1] int32: request b's new tokens are rows q_start[b] .. q_start[b + 1]
    lens: torch.Tensor        # [requests] int32: tokens cached, the granted ones included
    granted: torch.Tensor     # [requests] int32: new tokens granted
    slots: torch.Tensor       # [token_cap] int64: cache slot of each new token, -1 behind the last
    positions: torch.Tensor   # [token_cap] int32: its position in its request, -1 behind the last
    n_free: torch.Tensor      # [1] int32: pages on the free list


def plan_pages(lens, add, free_list, n_free, table, *, page_size: int, token_cap: int, out: Optional[PagePlan] = None) -> PagePlan:
    """Pages, slots and positions of a step's new tokens, from the requests'
    lengths (sb_plan_pages).

    lens, add: int32 [requests], one at least (add: new tokens wanted, 0 none,
    negative releases the request); free_list: int32 [pages], its first n_free (int32
    [1]) entries free page ids; table: int32 [requests, max_pages]. table and
    free_list are updated in place, the rest of the new state is returned, in
    new tensors or in `out`'s, which may be lens and n_free themselves. token_cap:
    the most tokens a step takes."""
    i = _device(lens, "lens")
    (B, width), row = _table(table, i)
    try:
        cap = operator.index(token_cap)
    except TypeError:
        _refuse("token_cap must be a whole number")
    if free_list.dim() != 1:
        _refuse("free_list must have one dimension")
    if cap < 0:
        _refuse("token_cap must not be negative")
    _apart(table, "table")
    i32, i64 = torch.int32, torch.int64
    fresh = out is None
    if fresh:
        q_start, after, granted, left = torch.empty(3 * B + 2, dtype=i32, device=i).split_with_sizes((B + 1, B, B, 1))
        out = PagePlan(q_start, after, granted, torch.empty(cap, dtype=i64, device=i), torch.empty(cap, dtype=i32, device=i), left)
        at = q_start.data_ptr()
        to = at + 4 * (B + 1), at + 4 * (3 * B + 1), at, at + 4 * (2 * B + 1), out.slots.data_ptr(), out.positions.data_ptr()
    else:
        to = (_whole(out.lens, "out.lens", i32, i, (B,)), _whole(out.n_free, "out.n_free", i32, i, (1,)),
              _whole(out.q_start, "out.q_start", i32, i, (B + 1,)), _whole(out.granted, "out.granted", i32, i, (B,)),
              _whole(out.slots, "out.slots", i64, i, (cap,)), _whole(out.positions, "out.positions", i32, i, (cap,)))
    args = N.PLAN_ARGS.pack(
        N.PLAN_ARGS.size, _whole(lens, "lens", i32, i, (B,)), _whole(add, "add", i32, i, (B,)), _whole(n_free, "n_free", i32, i, (1,)),
        _whole(free_list, "free_list", i32, i, free_list.shape), table.data_ptr(), *to,
        row, B, free_list.shape[0], page_size, width, cap, 0)
    _call(N.lib().sb_plan_pages, "sb_plan_pages", i, args)
    _written((table, free_list) if fresh else (table, free_list, *out))
    return out


def rope_frequencies(rot_dim: int, *, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, original_length: int = 4096,
                     beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda"):
    """(inv_freq, mscale) of rotary positions over rot_dim values of a head.

    inv_freq[i] = base^(-2i / rot_dim) in float64. For contexts `factor` times
    as long as the original_length trained on, scaling "linear" divides all by
    the factor; "ntk" raises the base by factor^(rot_dim / (rot_dim - 2)), which
    keeps the fastest pair and slows the slowest by the factor; "parts" divides
    pairs that turn less than beta_slow times over original_length, keeps
    those that turn more than beta_fast times, blends between, and scales the
    rotated part by mscale = 1 + ln(factor) / 10 (the YaRN method)."""
    if rot_dim < 2 or rot_dim % 2 or not base > 1 or not factor >= 1:
        _refuse("rot_dim must be even and at least 2, base above 1, factor at least 1")
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    mscale = 1.0
    if scaling == "ntk":
        if rot_dim > 2:
            base = base * factor ** (rot_dim / (rot_dim - 2))
    elif scaling not in ("none", "linear", "parts"):
        _refuse(f"unknown scaling {scaling!r}")
    inv = base ** (-2.0 * i / rot_dim)
    if scaling == "linear":
        inv = inv / factor
    elif scaling == "parts":
        def pair_of(turns):   # the pair (as a real number) that turns so often over original_length
            return rot_dim * math.log(original_length / (2 * math.pi * turns)) / (2 * math.log(base))
        lo = max(math.floor(pair_of(beta_fast)), 0)
        hi = min(math.ceil(pair_of(beta_slow)), rot_dim - 1)   # (may lie behind the last pair, which is then slowed in part)
        slowed = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        inv = inv * (1 - slowed) + inv / factor * slowed
        mscale = 1.0 + 0.1 * math.log(factor)
    return inv.to(device), mscale


def rope_append(q, k, v, positions, slots, k_cache, v_cache, inv_freq, *, layout: str = "half", mscale: float = 1.0, out=None):
    """Rotated queries; rotated keys and the values go to their cache slots
    (sb_rope_append).

    q: [tokens, q_heads, head_dim], k, v: [tokens, kv_heads, head_dim], caches:
    [pages, page_size, kv_heads, head_dim], one type (bfloat16 or float16); of
    any strides that are multiples of 8, heads contiguous, at addresses that are
    multiples of 16. positions: int32
    [tokens], slots: int64 [tokens] (plan_pages gives both; tokens with slots
    outside the cache are skipped, those of the others have to be distinct);
    inv_freq: float64, one per pair
    (rope_frequencies). out: where the queries go, q itself for in place."""
    i, dtype = _device(q, "q"), q.dtype
    if dtype not in _HALVES:
        _refuse("q must be bfloat16 or float16")
    _no_grad(q, k, v, k_cache, v_cache, inv_freq, out)
    (T, Hq, D), qs = _heads(q, "q", dtype, i)
    (_, Hkv, _), ks = _heads(k, "k", dtype, i, T, D)
    (_, Hv, _), vs = _heads(v, "v", dtype, i, T, D)
    if Hv != Hkv:
        _refuse("k and v must have the same heads")
    (pages, page_size, _, _), kc, vc = _caches(k_cache, v_cache, dtype, i, Hkv, D)
    _apart(k_cache, "k_cache"), _apart(v_cache, "v_cache")
    if out is None:
        out = torch.empty((T, Hq, D), dtype=dtype, device=i)
        os_ = (Hq * D, D)
    else:
        (_, Ho, _), os_ = _heads(out, "out", dtype, i, T, D)
        if Ho != Hq:
            _refuse("out must have q's heads")
        _apart(out, "out")
    if layout not in _LAYOUTS:
        _refuse(f"unknown layout {layout!r}")
    if inv_freq.dim() != 1:
        _refuse("inv_freq must have one dimension")
    pairs = inv_freq.shape[0]
    args = N.ROPE_ARGS.pack(
        N.ROPE_ARGS.size, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(),
        _whole(positions, "positions", torch.int32, i, (T,)), _whole(slots, "slots", torch.int64, i, (T,)),
        _whole(inv_freq, "inv_freq", torch.float64, i, (pairs,)), qs[0], qs[1], ks[0], ks[1], vs[0], vs[1], os_[0], os_[1],
        kc[0], kc[1], kc[2], vc[0], vc[1], vc[2], T, Hq, Hkv, D, pairs, _LAYOUTS[layout], _HALVES[dtype], pages, page_size, mscale)
    _call(N.lib().sb_rope_append, "sb_rope_append", i, args)
    _written((k_cache, v_cache, out))
    return out


def paged_attention(q, k_cache, v_cache, table, lens, q_start, *, max_q: int, max_kv: int, window: int = 0, sinks: int = 0,
                    scale: Optional[float] = None, out=None):
    """Causal attention of a step's queries over their requests' paged caches
    (sb_paged_attention).

    q: [tokens, q_heads, head_dim] (rotated), caches: [pages, page_size, kv_heads,
    head_dim], one type (bfloat16 or float16), head_dim 64, 128 or 256, strides and
    addresses as in rope_append; table: int32 [requests, max_pages], one request at
    least; lens: int32 [requests], the new tokens included;
    q_start: int32 [requests + 1]. A query sees the last `window` positions up
    to its own and the request's first `sinks` (window 0: all up to its own).
    scale: 1 / sqrt(head_dim) by default. max_q, max_kv: upper bounds of a request's queries
    and of lens, for the choice of kernels only. Rows of the result behind
    the last request's are left as they are in `out` (undefined without it)."""
    i, dtype = _device(q, "q"), q.dtype
    if dtype not in _HALVES:
        _refuse("q must be bfloat16 or float16")
    _no_grad(q, k_cache, v_cache, out)
    (T, Hq, D), qs = _heads(q, "q", dtype, i)
    (pages, page_size, Hkv, _), kc, vc = _caches(k_cache, v_cache, dtype, i, None, D)
    (B, width), row = _table(table, i)
    if out is None:
        out = torch.empty((T, Hq, D), dtype=dtype, device=i)
        os_ = (Hq * D, D)
    else:
        (_, Ho, _), os_ = _heads(out, "out", dtype, i, T, D)
        if Ho != Hq:
            _refuse("out must have q's heads")
        _apart(out, "out")
    args = N.ATTENTION_ARGS.pack(
        N.ATTENTION_ARGS.size, q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), table.data_ptr(),
        _whole(lens, "lens", torch.int32, i, (B,)), _whole(q_start, "q_start", torch.int32, i, (B + 1,)), out.data_ptr(),
        qs[0], qs[1], os_[0], os_[1], kc[0], kc[1], kc[2], vc[0], vc[1], vc[2], row,
        T, B, Hq, Hkv, D, _HALVES[dtype], pages, page_size, width, window, sinks, max_q, max_kv,
        1.0 / math.sqrt(D) if scale is None else scale)
    L = N.lib()
    if i == _current():
        need = L.sb_attention_workspace(args)
    else:
        with torch.cuda.device(i):
            need = L.sb_attention_workspace(args)
    work = torch.empty(need, dtype=torch.uint8, device=i) if need > 0 else None   # (below 0: refused by the call itself)
    _call(L.sb_paged_attention, "sb_paged_attention", i, args, None if work is None else work.data_ptr(), max(need, 0))
    _written((out,))
    return out


def sample_tokens(logits, u, *, temperature=None, top_k=None, top_p=None, min_p=None, out=None):
    """(tokens int32 [rows], logprobs float32 [rows]): one token per row of
    logits, drawn with the given numbers (sb_sample_tokens).

    logits: [rows, vocab], float32, bfloat16 or float16, contiguous rows; u:
    float32 [rows] in [0, 1). temperature, top_p, min_p (float32) and top_k
    (int32): one per row, or None to leave that filter out (temperature: 1; 0
    takes the largest logit). logprobs: of the drawn token among the kept
    ones. out: (tokens, logprobs) to write to."""
    i = _device(logits, "logits")
    if logits.dim() != 2 or logits.dtype not in _LOGITS or (logits.shape[1] > 1 and logits.stride(1) != 1):
        _refuse("logits must be a float32, bfloat16 or float16 tensor [rows, vocab] with contiguous rows")
    _no_grad(logits, u, temperature, top_p, min_p, *(out or ()))
    R, V = logits.shape
    f32 = torch.float32
    if out is None:
        out = torch.empty(R, dtype=torch.int32, device=i), torch.empty(R, dtype=f32, device=i)
    tokens, logprobs = out
    args = N.SAMPLE_ARGS.pack(
        N.SAMPLE_ARGS.size, logits.data_ptr(), _whole(u, "u", f32, i, (R,)),
        0 if temperature is None else _whole(temperature, "temperature", f32, i, (R,)),
        0 if top_k is None else _whole(top_k, "top_k", torch.int32, i, (R,)),
        0 if top_p is None else _whole(top_p, "top_p", f32, i, (R,)),
        0 if min_p is None else _whole(min_p, "min_p", f32, i, (R,)), _whole(tokens, "out tokens", torch.int32, i, (R,)),
        _whole(logprobs, "out logprobs", f32, i, (R,)), logits.stride(0) if R > 1 else V, R, V, _LOGITS[logits.dtype], 0)
    L = N.lib()
    need = L.sb_sample_workspace(args)   # (below 0: refused by the call itself)
    work = torch.empty(need, dtype=torch.uint8, device=i) if need > 0 else None
    _call(L.sb_sample_tokens, "sb_sample_tokens", i, args, None if work is None else work.data_ptr(), max(need, 0))
    _written((tokens, logprobs))
    return tokens, logprobs
