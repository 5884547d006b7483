"""The 8-bit block cache: the C ABI's refusals and the binding's checks on the
CPU, and on the GPU every operator against its plain 64-bit form (cache_ref)
at the sizes, layouts and masks where it can go wrong."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import cache_ref as ref
import paper_2605_05023_amd as attn
from paper_2605_05023_amd import _abi, cache as cm

P = 0x10000  # dummy aligned pointer, never dereferenced
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "attn.h")


# ---- CPU: descriptors -----------------------------------------------------

@pytest.mark.parametrize("cls, name", [
    (_abi.AttnCache, "attn_cache"), (_abi.AttnCachePlanDesc, "attn_cache_plan_desc"),
    (_abi.AttnCacheAppendDesc, "attn_cache_append_desc"), (_abi.AttnCacheFwdDesc, "attn_cache_fwd_desc")])
def test_mirror_matches_header(tmp_path, cls, name):
    fields = [f[0] for f in cls._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(
        ["#include <stdio.h>", "#include <stddef.h>", f'#include "{HEADER}"', "int main(void) {",
         f'  printf("%zu\\n", sizeof({name}));'] +
        [f'  printf("%zu\\n", offsetof({name}, {f}));' for f in fields] + ["  return 0;", "}"]))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c11", str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True,
                                          text=True).stdout.split()]
    assert got == [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f in fields]


def pool(**over):
    c = _abi.AttnCache.new()
    c.cache_dtype, c.num_blocks, c.num_kv_heads, c.block_size, c.head_dim = 0, 10, 2, 64, 128
    c.k = c.v = c.k_scale = c.v_scale = P
    for k, v in over.items():
        setattr(c, k, v)
    return c


def plan_desc(**over):
    d = _abi.AttnCachePlanDesc.new()
    d.batch, d.block_size, d.table_width, d.free_len, d.total_new = 3, 64, 5, 10, 20
    for f in ("cached_lens", "new_lens", "block_tables", "free_blocks", "num_free", "slots", "cu_seqlens_q",
              "seqlens_k"):
        setattr(d, f, P)
    d.num_free_out = 2 * P
    for k, v in over.items():
        setattr(d, k, v)
    return d


def append_desc(**over):
    d = _abi.AttnCacheAppendDesc.new()
    d.dtype, d.total_new, d.slots = _abi.ATTN_BF16, 20, P
    for k, v in over.items():
        setattr(d, k, v)
    return d


def fwd_desc(packed=False, **over):
    d = _abi.AttnCacheFwdDesc.new()
    d.dtype, d.batch, d.num_q_heads, d.seqlen_q = _abi.ATTN_BF16, 3, 8, 4
    d.table_width, d.block_tables, d.seqlens_k = 5, P, P
    d.scale = 0.1
    d.window_left = d.window_right = -1
    if packed:
        d.cu_seqlens_q, d.max_seqlen_q, d.total_q = P, 4, 9
    for k, v in over.items():
        setattr(d, k, v)
    return d


POOL_BAD = [
    ("size", dict(struct_size=8), "ATTN_ERR_ABI"), ("format", dict(cache_dtype=2), "ATTN_ERR_UNSUPPORTED"),
    ("head dim", dict(head_dim=96), "ATTN_ERR_UNSUPPORTED"),
    ("block size", dict(block_size=48), "ATTN_ERR_UNSUPPORTED"),
    ("block size 8", dict(block_size=8), "ATTN_ERR_UNSUPPORTED"),
    ("no blocks", dict(num_blocks=0), "ATTN_ERR_BAD_SHAPE"),
    ("no heads", dict(num_kv_heads=0), "ATTN_ERR_BAD_SHAPE"),
    ("many heads", dict(num_kv_heads=65536), "ATTN_ERR_UNSUPPORTED"),
    ("block stride", dict(stride_k_block=2 * 64 * 128 + 8), "ATTN_ERR_ALIGNMENT"),
    ("blocks overlap", dict(stride_v_block=64 * 128), "ATTN_ERR_BAD_SHAPE"),
    ("heads overlap", dict(stride_k_head=64 * 64), "ATTN_ERR_BAD_SHAPE"),
    ("negative stride", dict(stride_v_head=-16), "ATTN_ERR_BAD_SHAPE"),
    ("scales overlap", dict(stride_ks_block=1), "ATTN_ERR_BAD_SHAPE"),
    ("no K", dict(k=None), "ATTN_ERR_NULL_PTR"), ("no V scale", dict(v_scale=None), "ATTN_ERR_NULL_PTR"),
    ("V alignment", dict(v=P + 8), "ATTN_ERR_ALIGNMENT"),
    ("scale alignment", dict(k_scale=P + 2), "ATTN_ERR_ALIGNMENT"),
]


@pytest.mark.parametrize("name, over, err", POOL_BAD, ids=[c[0] for c in POOL_BAD])
def test_pool_refusals(name, over, err):
    lib, c = attn.load(), pool(**over)
    want = _abi.STATUS_CODE[err]
    d = append_desc()
    assert lib.attn_cache_append(P, P, ctypes.byref(c), ctypes.byref(d)) == want
    f = fwd_desc()
    assert lib.attn_cache_fwd(P, P, P, ctypes.byref(c), ctypes.byref(f), None, 0) == want
    if err not in ("ATTN_ERR_NULL_PTR", "ATTN_ERR_ALIGNMENT") or "stride" in name:
        assert lib.attn_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(f)) == want


PLAN_BAD = [
    ("size", dict(struct_size=4), "ATTN_ERR_ABI"), ("block size", dict(block_size=100), "ATTN_ERR_UNSUPPORTED"),
    ("batch", dict(batch=-1), "ATTN_ERR_BAD_SHAPE"), ("width", dict(table_width=-1), "ATTN_ERR_BAD_SHAPE"),
    ("free list", dict(free_len=-1), "ATTN_ERR_BAD_SHAPE"),
    ("tokens", dict(total_new=-1), "ATTN_ERR_BAD_SHAPE"),
    ("too many tokens", dict(total_new=1 << 31), "ATTN_ERR_UNSUPPORTED"),
    ("rows overlap", dict(stride_table=4), "ATTN_ERR_BAD_SHAPE"),
    ("flags", dict(flags=_abi.ATTN_FLAG_VALIDATE), "ATTN_ERR_BAD_VARIANT"),
    ("no lengths", dict(new_lens=None), "ATTN_ERR_NULL_PTR"), ("no slots", dict(slots=None), "ATTN_ERR_NULL_PTR"),
    ("no table", dict(block_tables=None), "ATTN_ERR_NULL_PTR"),
    ("no free list", dict(free_blocks=None), "ATTN_ERR_NULL_PTR"),
    ("no count", dict(num_free=None), "ATTN_ERR_NULL_PTR"),
    ("count in place", dict(num_free_out=P), "ATTN_ERR_BAD_SHAPE"),
    ("slot alignment", dict(slots=P + 4), "ATTN_ERR_ALIGNMENT"),
    ("length alignment", dict(seqlens_k=P + 1), "ATTN_ERR_ALIGNMENT"),
]


@pytest.mark.parametrize("name, over, err", PLAN_BAD, ids=[c[0] for c in PLAN_BAD])
def test_plan_refusals(name, over, err):
    d = plan_desc(**over)
    assert attn.load().attn_cache_plan(ctypes.byref(d)) == _abi.STATUS_CODE[err]


APPEND_BAD = [
    ("size", dict(struct_size=4), "ATTN_ERR_ABI"), ("dtype", dict(dtype=2), "ATTN_ERR_UNSUPPORTED"),
    ("tokens", dict(total_new=-1), "ATTN_ERR_BAD_SHAPE"),
    ("too many tokens", dict(total_new=1 << 31), "ATTN_ERR_UNSUPPORTED"),
    ("stride", dict(stride_k_s=4), "ATTN_ERR_ALIGNMENT"), ("negative", dict(stride_v_h=-8), "ATTN_ERR_BAD_SHAPE"),
    ("flags", dict(flags=4), "ATTN_ERR_BAD_VARIANT"), ("no slots", dict(slots=None), "ATTN_ERR_NULL_PTR"),
    ("slots", dict(slots=P + 4), "ATTN_ERR_ALIGNMENT"),
]


@pytest.mark.parametrize("name, over, err", APPEND_BAD, ids=[c[0] for c in APPEND_BAD])
def test_append_refusals(name, over, err):
    lib, c, d = attn.load(), pool(), append_desc(**over)
    assert lib.attn_cache_append(P, P, ctypes.byref(c), ctypes.byref(d)) == _abi.STATUS_CODE[err]


def test_append_pointers_and_empty_calls():
    lib, c, d = attn.load(), pool(), append_desc()
    call = lambda k, v: lib.attn_cache_append(k, v, ctypes.byref(c), ctypes.byref(d))  # noqa: E731
    assert call(None, P) == call(P, None) == _abi.STATUS_CODE["ATTN_ERR_NULL_PTR"]
    assert call(P + 8, P) == _abi.STATUS_CODE["ATTN_ERR_ALIGNMENT"]
    assert lib.attn_cache_append(P, P, None, ctypes.byref(d)) == _abi.STATUS_CODE["ATTN_ERR_NULL_PTR"]
    assert lib.attn_cache_append(P, P, ctypes.byref(c), None) == _abi.STATUS_CODE["ATTN_ERR_NULL_PTR"]
    assert lib.attn_cache_plan(None) == _abi.STATUS_CODE["ATTN_ERR_NULL_PTR"]
    d.total_new = 0
    assert call(None, None) == 0


FWD_BAD = [
    ("size", dict(struct_size=4), "ATTN_ERR_ABI"), ("dtype", dict(dtype=2), "ATTN_ERR_UNSUPPORTED"),
    ("batch", dict(batch=-1), "ATTN_ERR_BAD_SHAPE"), ("groups", dict(num_q_heads=7), "ATTN_ERR_BAD_SHAPE"),
    ("no heads", dict(num_q_heads=0), "ATTN_ERR_BAD_SHAPE"),
    ("queries", dict(seqlen_q=-1), "ATTN_ERR_BAD_SHAPE"),
    ("prefix mask", dict(mask_kind=_abi.ATTN_MASK_PREFIX_LM), "ATTN_ERR_UNSUPPORTED"),
    ("segment mask", dict(mask_kind=_abi.ATTN_MASK_CAUSAL_BLOCKWISE), "ATTN_ERR_UNSUPPORTED"),
    ("mask", dict(mask_kind=7), "ATTN_ERR_BAD_VARIANT"),
    ("window", dict(mask_kind=2, window_left=-2), "ATTN_ERR_BAD_VARIANT"),
    ("scale", dict(scale=0.0), "ATTN_ERR_BAD_VARIANT"), ("scale nan", dict(scale=math.nan), "ATTN_ERR_BAD_VARIANT"),
    ("soft-cap", dict(softcap=-1.0), "ATTN_ERR_BAD_VARIANT"),
    ("soft-cap inf", dict(softcap=math.inf), "ATTN_ERR_BAD_VARIANT"),
    ("tiny soft-cap", dict(softcap=1e-40), "ATTN_ERR_BAD_VARIANT"),
    ("flags", dict(flags=8), "ATTN_ERR_BAD_VARIANT"), ("width", dict(table_width=-1), "ATTN_ERR_BAD_SHAPE"),
    ("max keys", dict(max_seqlen_k=-1), "ATTN_ERR_BAD_SHAPE"),
    ("table rows", dict(stride_table=4), "ATTN_ERR_BAD_SHAPE"),
    ("q stride", dict(stride_q_s=132), "ATTN_ERR_ALIGNMENT"), ("o stride", dict(stride_o_h=-128), "ATTN_ERR_BAD_SHAPE"),
    ("out overlaps", dict(stride_o_s=64), "ATTN_ERR_BAD_SHAPE"),
    ("no table", dict(block_tables=None), "ATTN_ERR_NULL_PTR"),
    ("no lengths", dict(seqlens_k=None), "ATTN_ERR_NULL_PTR"),
    ("slopes", dict(alibi_slopes=P + 2), "ATTN_ERR_ALIGNMENT"),
    ("rows", dict(seqlen_q=1 << 30), "ATTN_ERR_UNSUPPORTED"),
    ("table keys", dict(table_width=1 << 25), "ATTN_ERR_UNSUPPORTED"),
    ("schedule kernel", dict(sched_kernel=3), "ATTN_ERR_BAD_VARIANT"),
    ("schedule waves", dict(sched_waves=6), "ATTN_ERR_BAD_VARIANT"),
    ("schedule tiles", dict(sched_tiles=3), "ATTN_ERR_BAD_VARIANT"),
    ("schedule tiles, many", dict(sched_kernel=2, sched_tiles=1), "ATTN_ERR_BAD_VARIANT"),
    ("schedule splits", dict(sched_splits=65), "ATTN_ERR_BAD_VARIANT"),
]


@pytest.mark.parametrize("name, over, err", FWD_BAD, ids=[c[0] for c in FWD_BAD])
def test_fwd_refusals(name, over, err):
    lib, c, d = attn.load(), pool(), fwd_desc(**over)
    assert lib.attn_cache_fwd(P, P, P, ctypes.byref(c), ctypes.byref(d), None, 0) == _abi.STATUS_CODE[err]


def test_fwd_pointers_and_empty_calls():
    lib, c = attn.load(), pool()

    def call(d, q=P, o=P, lse=P, ws=None):
        return lib.attn_cache_fwd(q, o, lse, ctypes.byref(c), ctypes.byref(d), ws, 0)

    null, align = _abi.STATUS_CODE["ATTN_ERR_NULL_PTR"], _abi.STATUS_CODE["ATTN_ERR_ALIGNMENT"]
    assert call(fwd_desc(), q=None) == call(fwd_desc(), o=None) == null
    assert call(fwd_desc(), q=P + 8) == call(fwd_desc(), lse=P + 2) == call(fwd_desc(), ws=P + 8) == align
    assert lib.attn_cache_fwd(P, P, P, None, ctypes.byref(fwd_desc()), None, 0) == null
    bad = _abi.STATUS_CODE["ATTN_ERR_BAD_SHAPE"]
    assert call(fwd_desc(packed=True, max_seqlen_q=-1)) == call(fwd_desc(packed=True, total_q=-1)) == bad
    for d in (fwd_desc(batch=0), fwd_desc(seqlen_q=0), fwd_desc(packed=True, max_seqlen_q=0),
              fwd_desc(packed=True, total_q=0)):
        assert call(d) == 0
        assert lib.attn_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(d)) == 0


def test_workspace_is_bounded():
    """No more than a quarter of q, out, K and V, or 256 MiB."""
    lib = attn.load()
    for batch, hq, hkv, sq, width in ((1, 32, 8, 1, 4000), (64, 128, 8, 1, 2000), (2, 8, 8, 500, 1000),
                                      (1, 64, 8, 4096, 1000), (300, 8, 8, 3, 100)):
        c = pool(num_kv_heads=hkv, num_blocks=batch * width)
        d = fwd_desc(batch=batch, num_q_heads=hq, seqlen_q=sq, table_width=width)
        n = lib.attn_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(d))
        moved = 2 * 128 * (batch * sq * hq * 2 + batch * width * 64 * hkv)
        assert 0 <= n <= max(moved // 4, 256 << 20)
    # one decode row of a long context is split, one of a short context is not
    d = fwd_desc(batch=1, seqlen_q=1, table_width=1000)
    c = pool(num_blocks=1000)
    assert lib.attn_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(d)) > 0
    d.max_seqlen_k = 100
    assert lib.attn_cache_workspace_bytes(ctypes.byref(c), ctypes.byref(d)) == 0


# ---- CPU: the binding -----------------------------------------------------

def cpu_cache(**over):
    c = attn.new_cache(6, 2, 16, 64, device="cpu")._asdict()
    c.update(over)
    return attn.KVCache(**c)


def T(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def I(*values):
    return torch.tensor(values, dtype=torch.int32)


CACHE_BAD = [
    dict(k=T(6, 2, 16, 64)), dict(v=T(6, 2, 16, 64).to(torch.float8_e4m3fn)),
    dict(v=T(6, 2, 64, 16).to(torch.float8_e5m2)), dict(k_scale=T(6, 2)),
    dict(v_scale=T(6, 3, dtype=torch.float32)), dict(k_scale=T(2, 6, dtype=torch.float32).t()),
    dict(k_scale=T(1, 2, dtype=torch.float32).expand(6, 2)),
    dict(k=T(6, 2, 64, 16).to(torch.float8_e4m3fn).transpose(2, 3)),
    dict(k=T(6, 2, 16, 128).to(torch.float8_e4m3fn)[..., :64]),
]


@pytest.mark.parametrize("over", CACHE_BAD, ids=[str(i) for i in range(len(CACHE_BAD))])
def test_binding_checks_the_cache(over):
    with pytest.raises((TypeError, ValueError)):
        cm.make_cache(cpu_cache(**over))


def test_binding_describes_views_of_a_pool():
    big = torch.zeros(6, 3, 2, 16, 64, dtype=torch.float8_e4m3fn)
    c = cm.make_cache(cpu_cache(k=big[:, 1]))
    assert (c.stride_k_block, c.stride_k_head, c.k) == (3 * 2 * 16 * 64, 16 * 64, big[:, 1].data_ptr())
    s = torch.zeros(6, 5)
    assert cm.make_cache(cpu_cache(k_scale=s[:, 1:3])).stride_ks_block == 5


APPEND_ARGS = [
    dict(k=T(5, 2, 64, dtype=torch.float16)), dict(v=T(5, 2, 64, dtype=torch.float32)), dict(k=T(4, 2, 64)),
    dict(k=T(5, 3, 64)), dict(k=T(5, 2, 128)), dict(k=T(5, 64, 2).transpose(1, 2)),
    dict(slots=torch.zeros(5, dtype=torch.int32)), dict(slots=torch.zeros(4, dtype=torch.int64)),
    dict(slots=torch.zeros(10, dtype=torch.int64)[::2]),
]


@pytest.mark.parametrize("over", APPEND_ARGS, ids=[str(i) for i in range(len(APPEND_ARGS))])
def test_binding_checks_append(over):
    a = dict(k=T(5, 2, 64), v=T(5, 2, 64), slots=torch.zeros(5, dtype=torch.int64))
    cm.make_append_desc(cpu_cache(), **a)
    a.update(over)
    with pytest.raises((TypeError, ValueError)):
        cm.make_append_desc(cpu_cache(), **a)


PLAN_ARGS = [
    dict(cached_lens=torch.zeros(3, dtype=torch.int64)), dict(new_lens=I(1, 2)), dict(num_free=I(1, 2)),
    dict(block_tables=torch.zeros(2, 4, dtype=torch.int32)), dict(block_tables=torch.zeros(3, 4)),
    dict(block_tables=torch.zeros(4, 3, dtype=torch.int32).t()),
    dict(block_tables=torch.zeros(1, 4, dtype=torch.int32).expand(3, 4)),
    dict(free_blocks=torch.zeros(8, dtype=torch.int32)[::2]), dict(total_new=-1),
]


@pytest.mark.parametrize("over", PLAN_ARGS, ids=[str(i) for i in range(len(PLAN_ARGS))])
def test_binding_checks_plan(over):
    a = dict(cached_lens=I(1, 2, 3), new_lens=I(1, 1, 1), block_tables=torch.zeros(3, 4, dtype=torch.int32),
             free_blocks=I(4, 5), num_free=I(2), block_size=16, total_new=3)
    cm.make_plan_desc(**a)
    a.update(over)
    with pytest.raises((TypeError, ValueError)):
        cm.make_plan_desc(**a)


FWD_ARGS = [
    dict(q=T(3, 4, 1, 64, dtype=torch.float16)), dict(q=T(3, 4, 1, 128)), dict(q=T(3, 4, 64)), dict(q=T(2, 4, 1, 64)),
    dict(out=T(3, 4, 2, 64)), dict(out=T(3, 4, 1, 64, dtype=torch.float32)),
    dict(out=T(1, 4, 1, 64).expand(3, 4, 1, 64)), dict(lse=T(3, 4, 2, dtype=torch.float32)),
    dict(lse=T(3, 4, 1)), dict(block_tables=torch.zeros(2, 4, dtype=torch.int32)),
    dict(seqlens_k=torch.zeros(3, dtype=torch.int64)), dict(alibi_slopes=T(3, dtype=torch.float32)),
    dict(cu_seqlens_q=I(0, 1, 2, 3)), dict(max_seqlen_k=-1),
]


@pytest.mark.parametrize("over", FWD_ARGS, ids=[str(i) for i in range(len(FWD_ARGS))])
def test_binding_checks_fwd(over):
    a = dict(q=T(3, 4, 1, 64), block_tables=torch.zeros(3, 4, dtype=torch.int32), seqlens_k=I(1, 2, 3))
    cm.make_fwd_desc(cache=cpu_cache(), out=torch.empty_like(a["q"]), **a)
    a.update(over)
    with pytest.raises((TypeError, ValueError)):
        cm.make_fwd_desc(cache=cpu_cache(), **{"out": torch.empty_like(a["q"]), **a})


def test_binding_packed_needs_max_seqlen_q():
    a = dict(q=T(5, 4, 64), cache=cpu_cache(), block_tables=torch.zeros(3, 4, dtype=torch.int32),
             seqlens_k=I(1, 2, 3), out=T(5, 4, 64), cu_seqlens_q=I(0, 1, 2, 5))
    with pytest.raises(ValueError):
        cm.make_fwd_desc(**a)
    _, d = cm.make_fwd_desc(max_seqlen_q=3, **a)
    assert (d.total_q, d.max_seqlen_q, d.batch, d.max_seqlen_k) == (5, 3, 3, 0)


def test_cpu_tensors_are_refused():
    with pytest.raises(ValueError):
        attn.cache_fwd(T(3, 4, 1, 64), cpu_cache(), torch.zeros(3, 4, dtype=torch.int32), I(1, 2, 3))
    with pytest.raises(ValueError):
        attn.cache_append(cpu_cache(), T(5, 2, 64), T(5, 2, 64), torch.zeros(5, dtype=torch.int64))
    with pytest.raises(ValueError):
        attn.cache_plan(I(1), I(1), torch.zeros(1, 4, dtype=torch.int32), I(1), I(1), block_size=16, total_new=1)


def test_reference_rounds_like_the_formats():
    """The test's own rounding against torch's conversions (both formats, every binade)."""
    g = torch.Generator().manual_seed(0)
    for fmt in ("e4m3", "e5m2"):
        x = torch.randn(20000, generator=g) * torch.exp2(torch.randint(-20, 9, (20000,), generator=g).float())
        x = x.clamp(-ref.MAX[fmt], ref.MAX[fmt])
        assert torch.equal(ref.round8(x, fmt), ref.decode(x.to(ref.F8[fmt]), fmt))
    assert ref.scale_for(448.0, "e4m3") == 1.0 and ref.scale_for(448.1, "e4m3") == 2.0
    assert ref.scale_for(0.0, "e5m2") == 2.0 ** -120
