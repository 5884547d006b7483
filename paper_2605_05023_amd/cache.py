"""The 8-bit block cache: planning, appending and attention (include/attn.h).

A server keeps the keys and values of its requests in a pool of blocks of 16 to
128 tokens, in 8-bit floating point with one scale per block and kv head
(`KVCache`, made by `new_cache`). One step of it:

    plan = cache_plan(cached_lens, new_lens, block_tables, free_blocks, num_free,
                      block_size=64, total_new=n)            # blocks and slots
    cache_append(cache, k, v, plan.slots)                    # new keys and values
    out, lse = cache_fwd(q, cache, block_tables, plan.seqlens_k, causal=True,
                         cu_seqlens_q=plan.cu_seqlens_q, max_seqlen_q=longest)

Lengths, tables and slots stay on the device, so a step can be captured into a
graph. Nothing here takes part in autograd.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional

import torch

from ._abi import (ATTN_BF16, ATTN_E4M3, ATTN_E5M2, ATTN_FLAG_LOG, ATTN_FLAG_VALIDATE, ATTN_FP32,
                   ATTN_MASK_CAUSAL, ATTN_MASK_NONE, ATTN_MASK_SLIDING_WINDOW, AttnCache,
                   AttnCacheAppendDesc, AttnCacheFwdDesc, AttnCachePlanDesc, check, load)

_DTYPES = {torch.bfloat16: ATTN_BF16, torch.float32: ATTN_FP32}
_FORMATS = {torch.float8_e4m3fn: ATTN_E4M3, torch.float8_e5m2: ATTN_E5M2}


_native = None  # native argument marshalling (binding/fast_cache.cpp), bound to libattn.so


def bind_native(fast, lib):
    global _native
    fast.bind_cache(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        lib.attn_cache_plan, lib.attn_cache_append, lib.attn_cache_fwd, lib.attn_cache_workspace_bytes)))
    _native = fast


def _marshal():
    if _native is None:
        from . import _load_native
        _load_native()
    return _native


class KVCache(NamedTuple):
    """A pool of blocks: a stored value x of K stands for x * k_scale[block, head]."""
    k: torch.Tensor        # [blocks, kv heads, block size, head dim], float8_e4m3fn or float8_e5m2
    v: torch.Tensor        # [blocks, kv heads, head dim, block size]: V is stored transposed
    k_scale: torch.Tensor  # [blocks, kv heads] fp32
    v_scale: torch.Tensor


class CachePlan(NamedTuple):
    slots: torch.Tensor         # [total_new] int64, -1: none
    cu_seqlens_q: torch.Tensor  # [batch + 1] int32
    seqlens_k: torch.Tensor     # [batch] int32
    num_free: torch.Tensor      # [1] int32: free blocks that are left


def new_cache(num_blocks: int, num_kv_heads: int, block_size: int, head_dim: int, *,
              dtype=torch.float8_e4m3fn, device="cuda") -> KVCache:
    """An empty pool."""
    def side(*shape):
        return torch.zeros((num_blocks, num_kv_heads) + shape, dtype=dtype, device=device)

    def scales():
        return torch.zeros((num_blocks, num_kv_heads), dtype=torch.float32, device=device)

    return KVCache(side(block_size, head_dim), side(head_dim, block_size), scales(), scales())


def _want(t, name, dtype, device, shape):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device:
        raise TypeError(f"{name} must be {dtype} on {device}")
    if len(shape) != t.dim() or any(w is not None and n != w for n, w in zip(t.shape, shape)):
        raise ValueError(f"{name} must be {['*' if w is None else w for w in shape]}, got "
                         f"{tuple(t.shape)}")


def _flat(t, name, dtype, device, n):
    _want(t, name, dtype, device, (n,))
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _expanded(t):
    return any(st == 0 and n > 1 for n, st in zip(t.shape, t.stride()))


def _table(t, device, batch):
    _want(t, "block_tables", torch.int32, device, (batch, None))
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError("rows of block_tables must be contiguous")
    if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError("rows of block_tables must not overlap")
    # (one row's stride may be anything)
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _flags(validate, log):
    return (ATTN_FLAG_VALIDATE if validate else 0) | (ATTN_FLAG_LOG if log else 0)


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream if device.type == "cuda" else 0


def make_cache(cache: KVCache) -> AttnCache:
    """The descriptor of a pool; every mismatch of its tensors raises."""
    k, v, k_scale, v_scale = cache
    if k.dtype not in _FORMATS:
        raise TypeError("the cache must be float8_e4m3fn or float8_e5m2")
    if k.dim() != 4:
        raise ValueError(f"cache.k must be [blocks, kv heads, block size, head dim], got {tuple(k.shape)}")
    n, h, b, d = k.shape
    _want(v, "cache.v", k.dtype, k.device, (n, h, d, b))
    for name, t in (("k_scale", k_scale), ("v_scale", v_scale)):
        _want(t, "cache." + name, torch.float32, k.device, (n, h))
        if (h > 1 and t.stride(1) != 1) or _expanded(t):
            raise ValueError(f"the heads of cache.{name} must be contiguous")
    for name, t in (("k", k), ("v", v)):
        if t.stride(3) != 1 or t.stride(2) != t.shape[3] or _expanded(t):
            raise ValueError(f"the blocks of cache.{name} must be contiguous")
    c = AttnCache.new()
    c.cache_dtype = _FORMATS[k.dtype]
    c.num_blocks, c.num_kv_heads, c.block_size, c.head_dim = n, h, b, d
    c.k, c.v, c.k_scale, c.v_scale = (t.data_ptr() for t in (k, v, k_scale, v_scale))
    if n > 1:  # (the stride of a single entry says nothing)
        c.stride_k_block, c.stride_v_block = k.stride(0), v.stride(0)
        c.stride_ks_block, c.stride_vs_block = k_scale.stride(0), v_scale.stride(0)
    if h > 1:
        c.stride_k_head, c.stride_v_head = k.stride(1), v.stride(1)
    return c


def _on_gpu(t, name):
    if not t.is_cuda:
        raise ValueError(f"{name} runs on the GPU only")


def cache_plan(cached_lens, new_lens, block_tables, free_blocks, num_free, *, block_size: int,
               total_new: int, log: bool = False) -> CachePlan:
    """Give the new tokens of a step their blocks and slots.

    cached_lens, new_lens: int32 [batch], tokens that each request holds and gets.
    block_tables: int32 [batch, width]; the entries of the new blocks are written in
    place. free_blocks: int32 [n] with *num_free (int32 [1]) blocks on it, taken
    from its end; the count that is left is returned, for the next step, and the
    list itself is not changed. total_new: at least the sum of new_lens. A request
    whose blocks are not there, or do not fit its row, is refused: its slots are -1
    and its seqlens_k stays its cached length.
    """
    if not log:
        res = (_native or _marshal()).cache_plan(cached_lens, new_lens, block_tables, free_blocks, num_free,
                                                 block_size, total_new)
        if res is not NotImplemented:
            return CachePlan._make(res)
    _on_gpu(block_tables, "cache_plan")
    d, plan = make_plan_desc(cached_lens, new_lens, block_tables, free_blocks, num_free,
                             block_size=block_size, total_new=total_new, log=log)
    with torch.cuda.device(block_tables.device):
        check(load().attn_cache_plan(ctypes.byref(d)))
    return plan


def make_plan_desc(cached_lens, new_lens, block_tables, free_blocks, num_free, *, block_size, total_new,
                   log=False):
    """(descriptor, the outputs it points to) of a cache_plan call."""
    dev = block_tables.device
    batch = cached_lens.numel()
    _flat(cached_lens, "cached_lens", torch.int32, dev, None)
    _flat(new_lens, "new_lens", torch.int32, dev, batch)
    _flat(free_blocks, "free_blocks", torch.int32, dev, None)
    _flat(num_free, "num_free", torch.int32, dev, 1)
    total_new = int(total_new)
    if total_new < 0:
        raise ValueError(f"total_new is {total_new}")
    d = AttnCachePlanDesc.new()
    d.stride_table = _table(block_tables, dev, batch)
    d.batch, d.block_size, d.table_width = batch, int(block_size), block_tables.shape[1]
    d.free_len, d.total_new, d.flags = free_blocks.numel(), total_new, _flags(False, log)
    i32 = dict(dtype=torch.int32, device=dev)
    plan = CachePlan(torch.empty(total_new, dtype=torch.int64, device=dev), torch.empty(batch + 1, **i32),
                     torch.empty(batch, **i32), torch.empty(1, **i32))
    d.cached_lens, d.new_lens = cached_lens.data_ptr(), new_lens.data_ptr()
    d.block_tables, d.free_blocks = block_tables.data_ptr(), free_blocks.data_ptr()
    d.num_free, d.num_free_out = num_free.data_ptr(), plan.num_free.data_ptr()
    d.slots, d.cu_seqlens_q = plan.slots.data_ptr(), plan.cu_seqlens_q.data_ptr()
    d.seqlens_k = plan.seqlens_k.data_ptr()
    d.stream = _stream(dev)
    return d, plan


def cache_append(cache: KVCache, k, v, slots, *, validate: bool = False, log: bool = False) -> None:
    """Write new keys and values into the cache, in place.

    k, v: [tokens, kv heads, head dim], bfloat16 or float32; slots: int64 [tokens],
    as cache_plan gives them (the tokens of a block together and ascending; -1 and
    other slots outside the pool are skipped). Scales are powers of two; where the
    new values of a block need a larger one, its earlier values are stored anew.
    `validate` checks the order of the slots on the host first.
    """
    if not (validate or log):
        if (_native or _marshal()).cache_append(cache, k, v, slots) is not NotImplemented:
            return
    _on_gpu(k, "cache_append")
    k, v = (t.contiguous() if _expanded(t) else t for t in (k, v))
    c, d = make_append_desc(cache, k, v, slots, validate=validate, log=log)
    with torch.cuda.device(k.device):
        check(load().attn_cache_append(k.data_ptr(), v.data_ptr(), ctypes.byref(c), ctypes.byref(d)))


def make_append_desc(cache, k, v, slots, *, validate=False, log=False):
    c = make_cache(cache)
    if k.dtype not in _DTYPES:
        raise TypeError("k and v must be bfloat16 or float32")
    dev = cache.k.device
    for name, t in (("k", k), ("v", v)):
        _want(t, name, k.dtype, dev, (None, c.num_kv_heads, c.head_dim))
        if t.stride(2) != 1 or _expanded(t):
            raise ValueError(f"head_dim must be the innermost, contiguous axis of {name}, and no axis "
                             "expanded")
    if k.shape != v.shape:
        raise ValueError(f"k {tuple(k.shape)} and v {tuple(v.shape)} differ")
    _flat(slots, "slots", torch.int64, dev, k.shape[0])
    d = AttnCacheAppendDesc.new()
    d.dtype, d.total_new, d.flags = _DTYPES[k.dtype], k.shape[0], _flags(validate, log)
    for name, t in (("k", k), ("v", v)):
        if t.shape[1] > 1:
            setattr(d, f"stride_{name}_h", t.stride(1))
        if t.shape[0] > 1:
            setattr(d, f"stride_{name}_s", t.stride(0))
    d.slots = slots.data_ptr()
    d.stream = _stream(dev)
    return c, d


def _lse_shape(q, packed):
    return (q.shape[1], q.shape[0]) if packed else tuple(q.shape[:3])


def cache_fwd(q, cache: KVCache, block_tables, seqlens_k, *, causal: bool = False, window=None,
              alibi_slopes=None, softcap: float = 0.0, scale: Optional[float] = None, cu_seqlens_q=None,
              max_seqlen_q=None, max_seqlen_k=None, out=None, lse=None, return_lse: bool = True,
              validate: bool = False, log: bool = False, schedule=None):
    """Softmax attention of new queries to the cached keys of their requests.

    q: [batch, heads, queries, head dim], or packed [tokens, heads, head dim] with
    cu_seqlens_q (int32 [batch + 1]) and max_seqlen_q. seqlens_k: int32 [batch], the
    keys of each request, its new ones included; query i of n stands at key
    position seqlens_k - n + i. block_tables: int32 [batch, width].
    Masks, score options and outputs are those of `fwd`; max_seqlen_k (default: what
    the tables hold) is the longest key length, by which the keys are split over
    workgroups. Expanded q (an axis of stride 0) is copied first. `schedule`, a dict
    of the descriptor's sched_* overrides ("kernel", "waves", "tiles", "splits"), is
    for tuning and tests.
    """
    if not (validate or log or schedule):
        res = (_native or _marshal()).cache_fwd(
            q, cache, block_tables, seqlens_k, causal, window, alibi_slopes, softcap, scale, cu_seqlens_q,
            max_seqlen_q, max_seqlen_k, out, lse, return_lse)
        if res is not NotImplemented:
            return res
    # options and arguments that the native marshalling does not take, and
    # everything that is an error
    _on_gpu(q, "cache_fwd")
    if _expanded(q):
        q = q.contiguous()
    packed = cu_seqlens_q is not None
    if out is None:
        out = torch.empty_like(q)
    if lse is None and return_lse:
        lse = torch.empty(_lse_shape(q, packed), dtype=torch.float32, device=q.device)
    c, d = make_fwd_desc(q, cache, block_tables, seqlens_k, out, lse, causal=causal, window=window,
                         alibi_slopes=alibi_slopes, softcap=softcap, scale=scale,
                         cu_seqlens_q=cu_seqlens_q, max_seqlen_q=max_seqlen_q,
                         max_seqlen_k=max_seqlen_k, validate=validate, log=log, schedule=schedule)
    lib = load()
    nbytes = lib.attn_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(d))
    ws = None
    if nbytes > 0:
        try:
            ws = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
        except torch.OutOfMemoryError:  # computed without the split
            nbytes = 0
    with torch.cuda.device(q.device):
        check(lib.attn_cache_fwd(q.data_ptr(), out.data_ptr(), lse.data_ptr() if lse is not None else None,
                                 ctypes.byref(c), ctypes.byref(d),
                                 ws.data_ptr() if ws is not None else None, max(nbytes, 0)), lib)
    return (out, lse) if return_lse else out


def make_fwd_desc(q, cache, block_tables, seqlens_k, out, lse=None, *, causal=False, window=None,
                  alibi_slopes=None, softcap=0.0, scale=None, cu_seqlens_q=None, max_seqlen_q=None,
                  max_seqlen_k=None, validate=False, log=False, schedule=None):
    c = make_cache(cache)
    dev, packed = cache.k.device, cu_seqlens_q is not None
    if q.dtype not in _DTYPES:
        raise TypeError("q must be bfloat16 or float32")
    shape = (None, None, c.head_dim) if packed else (None, None, None, c.head_dim)
    _want(q, "q", q.dtype, dev, shape)
    _want(out, "out", q.dtype, dev, tuple(q.shape))
    for name, t in (("q", q), ("out", out)):
        if t.stride(-1) != 1 or _expanded(t):
            raise ValueError(f"head_dim must be the innermost, contiguous axis of {name}, and no axis "
                             "expanded")
    hq = q.shape[1]
    if lse is not None:
        _want(lse, "lse", torch.float32, dev, _lse_shape(q, packed))
        if not lse.is_contiguous():
            raise ValueError("lse must be contiguous")
    if alibi_slopes is not None:
        _flat(alibi_slopes, "alibi_slopes", torch.float32, dev, hq)
    _flat(seqlens_k, "seqlens_k", torch.int32, dev, None)
    batch = seqlens_k.numel()
    d = AttnCacheFwdDesc.new()
    if packed:
        _flat(cu_seqlens_q, "cu_seqlens_q", torch.int32, dev, batch + 1)
        if max_seqlen_q is None:
            raise ValueError("packed queries need max_seqlen_q (no device readback)")
        d.max_seqlen_q, d.total_q = int(max_seqlen_q), q.shape[0]
        d.cu_seqlens_q = cu_seqlens_q.data_ptr()
    else:
        if q.shape[0] != batch:
            raise ValueError(f"q has batch {q.shape[0]}, seqlens_k {batch}")
        d.seqlen_q = q.shape[2]
    d.stride_table = _table(block_tables, dev, batch)
    d.dtype, d.batch, d.num_q_heads = _DTYPES[q.dtype], batch, hq
    d.table_width = block_tables.shape[1]
    if max_seqlen_k is not None and int(max_seqlen_k) < 0:
        raise ValueError(f"max_seqlen_k is {max_seqlen_k}")
    # (a caller's 0, no keys, must not become the descriptor's default)
    d.max_seqlen_k = 0 if max_seqlen_k is None else max(1, int(max_seqlen_k))
    d.block_tables, d.seqlens_k = block_tables.data_ptr(), seqlens_k.data_ptr()
    if alibi_slopes is not None:
        d.alibi_slopes = alibi_slopes.data_ptr()
    d.scale = float(scale) if scale is not None else 1.0 / math.sqrt(c.head_dim)
    d.softcap = float(softcap)
    d.window_left = d.window_right = -1
    if window is not None:
        d.mask_kind = ATTN_MASK_SLIDING_WINDOW
        d.window_left, d.window_right = int(window[0]), int(window[1])
    else:
        d.mask_kind = ATTN_MASK_CAUSAL if causal else ATTN_MASK_NONE
    d.flags = _flags(validate, log)
    for name, value in (schedule or {}).items():
        setattr(d, "sched_" + {"kernel": "kernel", "waves": "waves", "tiles": "tiles",
                               "splits": "splits"}[name], int(value))
    for name, t in (("q", q), ("o", out)):
        axes = dict(h=1, s=0) if packed else dict(b=0, h=1, s=2)
        for axis, i in axes.items():
            if t.shape[i] > 1:
                setattr(d, f"stride_{name}_{axis}", t.stride(i))
    d.stream = _stream(dev)
    return c, d
