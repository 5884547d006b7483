"""The 8-bit block cache on the GPU: each operator against its plain 64-bit
form, and the steps of a server that uses them together."""
import ctypes
import math
import random

import pytest
import torch

import cache_ref as ref
import paper_2605_05023_amd as attn
from gpu_util import log
from paper_2605_05023_amd import _abi, cache as cm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator().manual_seed(seed)


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def bytes_equal(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ---- plan -----------------------------------------------------------------

def check_plan(cached, new, bs, *, width=None, free=None, num_free=None, total=None, seed=0):
    g = gen(seed)
    held = [ref.cdiv(c, bs) for c in cached]
    need = sum(ref.cdiv(c + n, bs) - ref.cdiv(c, bs) for c, n in zip(cached, new))
    width = max([ref.cdiv(c + n, bs) for c, n in zip(cached, new)] + [1]) if width is None else width
    pool = torch.randperm(sum(held) + need + 7, generator=g).tolist()
    table, at = [], 0
    for h in held:
        row = [-1] * width
        row[:min(h, width)] = pool[at:at + min(h, width)]
        at += h
        table.append(row)
    free = pool[at:] if free is None else free
    num_free = len(free) if num_free is None else num_free
    total = sum(new) if total is None else total
    # a row stride larger than the width, guarded
    dev_table = torch.full((max(len(cached), 1), width + 3), -77, dtype=torch.int32, device=DEV)
    view = dev_table[:len(cached), :width]
    if cached:
        view.copy_(torch.tensor(table, dtype=torch.int32))
    p = attn.cache_plan(i32(cached), i32(new), view, i32(free), i32([num_free]), block_size=bs, total_new=total)
    want = ref.plan(cached, new, table, free, num_free, bs, total)
    assert view.cpu().tolist() == want[0]
    assert (dev_table[:, width:] == -77).all()
    assert p.slots.cpu().tolist() == want[1]
    assert p.cu_seqlens_q.cpu().tolist() == want[2]
    assert p.seqlens_k.cpu().tolist() == want[3]
    assert p.num_free.item() == want[4]


@pytest.mark.parametrize("bs", [16, 32, 64, 128])
@pytest.mark.parametrize("batch", [1, 2, 63, 64, 65, 300])
def test_plan_decode(batch, bs):
    rng = random.Random(batch * bs)
    check_plan([rng.randrange(0, 700) for _ in range(batch)], [1] * batch, bs, seed=batch)


@pytest.mark.parametrize("seed", range(8))
def test_plan_ragged(seed):
    rng = random.Random(seed)
    batch = rng.choice([1, 5, 64, 130, 1000])
    bs = rng.choice([16, 32, 64, 128])
    new = [rng.choice([0, 1, rng.randrange(0, 300)]) for _ in range(batch)]
    cached = [rng.choice([0, bs, bs - 1, rng.randrange(0, 900)]) for _ in range(batch)]
    check_plan(cached, new, bs, seed=seed, total=sum(new) + rng.choice([0, 1, 500]))


def test_plan_long_prompts():
    check_plan([0, 17, 5], [100003, 0, 33000], 16)


@pytest.mark.parametrize("num_free", [0, 1, 2, 3, 5, 8, 9, 200, -4, 10000])
def test_plan_runs_out_of_blocks(num_free):
    """A request that does not fit leaves its blocks to nobody; one that needs none is granted."""
    check_plan([0, 16, 3, 30, 100, 0], [40, 1, 5, 60, 0, 16], 16, free=list(range(100, 109)), num_free=num_free)
    rng = random.Random(num_free)
    cached = [rng.randrange(0, 100) for _ in range(200)]
    check_plan(cached, [rng.randrange(0, 20) for _ in range(200)], 16, num_free=num_free)


def test_plan_rows_that_do_not_fit():
    check_plan([10, 60, 64, 0], [10, 4, 1, 200], 16, width=4)
    check_plan([10, 0], [3, 3], 16, width=1, free=[9], num_free=1)


def test_plan_empty_calls():
    check_plan([], [], 64)
    check_plan([], [], 64, total=5)
    check_plan([0, 0, 0], [0, 0, 0], 64)
    check_plan([0], [1], 64, free=[], num_free=0)


def test_plan_missing_blocks_and_short_totals():
    """A token in a block whose entry is negative has no slot; tokens past total_new are not written."""
    table = torch.tensor([[-1, 5], [4, -1]], dtype=torch.int32, device=DEV)
    guard = torch.full((20,), -9, dtype=torch.int64, device=DEV)
    p = attn.cache_plan(i32([20, 3]), i32([2, 3]), table, i32([8]), i32([1]), block_size=16, total_new=5)
    assert p.slots.tolist() == [5 * 16 + 4, 5 * 16 + 5, 4 * 16 + 3, 4 * 16 + 4, 4 * 16 + 5]
    table[0, 1] = -1
    p = attn.cache_plan(i32([20, 3]), i32([2, 3]), table, i32([8]), i32([1]), block_size=16, total_new=5)
    assert p.slots.tolist() == [-1, -1, 4 * 16 + 3, 4 * 16 + 4, 4 * 16 + 5]
    d, plan = cm.make_plan_desc(i32([20, 3]), i32([2, 3]), table, i32([8]), i32([1]), block_size=16, total_new=3)
    d.slots = guard.data_ptr()
    _abi.check(attn.load().attn_cache_plan(ctypes.byref(d)))
    assert guard.tolist() == [-1, -1, 4 * 16 + 3] + [-9] * 17


# ---- append ---------------------------------------------------------------

def slots_of(runs, bs):
    """[(block, first place, tokens)] -> slots; block None: tokens without a slot."""
    out = []
    for b, place, n in runs:
        out += [-1] * n if b is None else [b * bs + place + i for i in range(n)]
    return out


def check_append(fmt, dt, d, hkv, bs, runs, *, blocks=12, seed=0, grow=1.0, x=None, transform=None):
    g = gen(seed)
    k, v, ks, vs = ref.make_pool(g, blocks, hkv, bs, d, fmt)
    slots = slots_of(runs, bs)
    n = len(slots)
    if x is None:
        x = [(torch.randn(n, hkv, d, generator=g) * torch.exp(torch.randn(n, hkv, 1, generator=g)) * grow)
             .to(ref.DT[dt]) for _ in range(2)]
    want = [ref.append(ref.decode(data, fmt), s, y, slots, bs, fmt, last)
            for data, s, y, last in ((k, ks, x[0], False), (v, vs, x[1], True))]
    cache = attn.KVCache(*(t.to(DEV) for t in (k, v, ks, vs)))
    kd, vd = (t.to(DEV) for t in x)
    if transform:
        cache, kd, vd = transform(cache, kd, vd)
    attn.cache_append(cache, kd, vd, torch.tensor(slots, dtype=torch.int64, device=DEV), validate=True)
    for got, scale, (values, s) in ((cache.k, cache.k_scale, want[0]), (cache.v, cache.v_scale, want[1])):
        assert torch.equal(scale.cpu().double(), s)
        a = ref.decode(got.contiguous(), fmt)
        same = (a == values) | (torch.isnan(a) & torch.isnan(values))
        assert same.all(), f"{int((~same).sum())} of {same.numel()} values differ"
    return cache


RUNS = {
    "one token": [(3, 0, 1)],
    "one token later": [(3, 15, 1)],
    "whole block": [(3, 0, 16)],
    "decode": [(b, (5 * b) % 16, 1) for b in (7, 2, 0, 11, 4, 9)],
    "prompt": [(5, 3, 13), (1, 0, 16), (8, 0, 16), (0, 0, 9)],
    "holes": [(None, 0, 2), (4, 7, 3), (None, 0, 1), (6, 0, 1), (None, 0, 30), (10, 1, 15)],
    "many": [(b, b % 3, 5) for b in range(12)],
}


@pytest.mark.parametrize("grow", [0.01, 1.0, 300.0], ids=["small", "like", "growing"])
@pytest.mark.parametrize("runs", RUNS.values(), ids=RUNS.keys())
@pytest.mark.parametrize("fmt, dt, d, hkv", [("e4m3", "bf16", 128, 2), ("e5m2", "fp32", 64, 3),
                                             ("e4m3", "fp32", 128, 1), ("e5m2", "bf16", 64, 2)])
def test_append(fmt, dt, d, hkv, runs, grow):
    """The stored bytes and scales are those of the definition, exactly."""
    check_append(fmt, dt, d, hkv, 16, runs, grow=grow)


@pytest.mark.parametrize("bs", [32, 64, 128])
@pytest.mark.parametrize("grow", [1.0, 300.0])
def test_append_larger_blocks(bs, grow):
    runs = [(2, 0, bs), (7, bs - 1, 1), (1, 17, 3), (9, 5, bs - 5), (0, 0, 1), (4, 15, 2), (11, 0, bs - 1)]
    check_append("e4m3", "bf16", 128, 3, bs, runs, grow=grow)
    check_append("e5m2", "fp32", 64, 2, bs, runs[::-1], grow=grow, seed=1)


def test_append_many_tokens():
    """Groups of 16 tokens a workgroup (a prompt's call), with runs of every length."""
    rng = random.Random(0)
    runs, blocks = [], list(range(300))
    rng.shuffle(blocks)
    for b in blocks:
        place = rng.choice([0, 0, rng.randrange(32)])
        runs.append((b, place, rng.choice([32 - place, rng.randint(1, 32 - place)])))
    check_append("e4m3", "bf16", 64, 8, 32, runs, blocks=300)


def test_append_strides_and_views():
    """A layer of a pool that holds several, and k, v as views of one projection."""
    def transform(c, k, v):
        n, h, b, d = c.k.shape
        big = torch.zeros(n, 3, h, b, d, dtype=torch.uint8, device=DEV).view(c.k.dtype)
        big_v = torch.zeros(n, 3, h, d, b, dtype=torch.uint8, device=DEV).view(c.k.dtype)
        scales = torch.full((n, 2, 2 * h), -5.0, device=DEV)
        big.view(torch.uint8)[:, 1] = c.k.view(torch.uint8)
        big_v.view(torch.uint8)[:, 2] = c.v.view(torch.uint8)
        scales[:, 0, :h], scales[:, 1, h:] = c.k_scale, c.v_scale
        qkv = torch.zeros(k.shape[0], 3 * h, d, dtype=k.dtype, device=DEV)
        qkv[:, h:2 * h], qkv[:, 2 * h:] = k, v
        view = attn.KVCache(big[:, 1], big_v[:, 2], scales[:, 0, :h], scales[:, 1, h:])
        transform.others = lambda: (big.view(torch.uint8)[:, ::2].any() | big_v.view(torch.uint8)[:, :2].any() |
                                    (scales[:, 0, h:] != -5).any())
        return view, qkv[:, h:2 * h], qkv[:, 2 * h:]

    check_append("e4m3", "bf16", 128, 2, 16, RUNS["prompt"], grow=30.0, transform=transform)
    assert not transform.others()


def test_append_odd_values():
    """Infinities become the largest value, NaN stays, neither sets the scale; zeros; subnormals;
    the largest and smallest magnitudes; an amax exactly at and just above a power's reach."""
    d, bs = 64, 16
    for fmt, dt in (("e4m3", "fp32"), ("e5m2", "fp32"), ("e4m3", "bf16"), ("e5m2", "bf16")):
        t = torch.zeros(9, 1, d)
        t[0, 0, :3] = torch.tensor([math.inf, -math.inf, math.nan])
        t[0, 0, 3:8] = torch.tensor([1.0, -2.5, 0.1, 1e-3, -0.0])
        t[2, 0] = 3.0e38 * torch.linspace(-1, 1, d)
        t[3, 0] = 1e-38 * torch.linspace(-1, 1, d)
        t[4, 0] = 1e-42
        t[5, 0, 0] = ref.MAX[fmt] * 4
        t[6, 0, 0] = ref.MAX[fmt] * 4 * (1 + 2.0 ** -7)
        t[7, 0] = torch.linspace(-1, 1, d) ** 9
        t[8, 0] = math.nan
        runs = [(b, 0, 1) for b in range(9)]
        x = [t.to(ref.DT[dt]), t.flip(0).to(ref.DT[dt])]
        check_append(fmt, dt, d, 1, bs, runs, x=x)
        check_append(fmt, dt, d, 1, bs, [(b, 3, 1) for b in range(9)], x=x, seed=2)


def test_append_validate_refuses_disorder():
    cache = attn.new_cache(6, 2, 16, 64)
    x = torch.randn(4, 2, 64, device=DEV).bfloat16()
    for slots in ([0, 1, 3, 4], [5, 4, 16, 17], [0, 16, 1, 2], [3, 3, 16, 17], [0, -1, 1, 2]):
        with pytest.raises(attn.AttnError):
            attn.cache_append(cache, x, x, torch.tensor(slots, device=DEV), validate=True)
    assert not cache.k.view(torch.uint8).any() and not cache.k_scale.any()
    attn.cache_append(cache, x, x, torch.tensor([15, 16, 17, 96], device=DEV), validate=True)  # 96: outside
    attn.cache_append(cache, x[:0], x[:0], torch.zeros(0, dtype=torch.int64, device=DEV))


# ---- attention ------------------------------------------------------------

def check_rows(name, o, l, want, dt):
    """out and lse of one request against (out, lse, error bounds, sum of p |v|)."""
    w, lse, err, lerr, mass = want
    # bf16: P and O are rounded once each, by half a step of 2^-8 relative
    tol = err * 2 + (2.0 ** -8 * (mass * (1 + 2.0 ** -7) + w.abs()) if dt == "bf16" else 2.0 ** -23 * w.abs())
    # P times V's scale may be lost below 2^-126: up to 57344 2^-126 for each of 2^10 keys
    bad = ~((o.double() - w).abs() <= tol + 2.0 ** -100)
    assert not bad.any(), f"{name}: out off by {float(((o.double() - w).abs() / tol.clamp(min=1e-30)).max()):.3g} bounds"
    if l is not None:
        fine = lse > -math.inf
        assert torch.equal(l > -math.inf, fine), name
        off = (l.double() - lse).abs()[fine]
        assert (off <= 2 * lerr[fine]).all(), f"{name}: lse off by {float((off / lerr[fine]).max()):.3g} bounds"


def attention_case(fmt="e4m3", dt="bf16", d=128, hq=8, hkv=2, bs=64, lens=((1, 700),), packed=True, seed=0,
                   causal=True, window=None, softcap=0.0, alibi=False, width=None, spoiled=True, qscale=1.0,
                   bad=()):
    """Inputs of a call: lens are (queries, keys); `bad`: (request, table column, entry) put into the tables."""
    g = gen(seed)
    table, count, _ = ref.make_tables(g, [lk for _, lk in lens], bs, width)
    k, v, ks, vs = ref.make_pool(g, count, hkv, bs, d, fmt)
    if spoiled:
        ref.spoil(k, v, ks, vs, table, [lk for _, lk in lens], bs)
    n = [a for a, _ in lens]
    q = (torch.randn(sum(n), hq, d, generator=g) * qscale).to(ref.DT[dt])
    for r, c, e in bad:
        table[r, c] = e
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]) if alibi else None
    return dict(fmt=fmt, dt=dt, bs=bs, lens=lens, packed=packed, q=q, table=table, pool=(k, v, ks, vs), hkv=hkv,
                opt=dict(causal=causal, window=window, softcap=softcap), slopes=slopes)


def run_case(c, *, max_q=None, max_k=None, ws=True, lib=None, **extra):
    """(out, lse) on the CPU, in packed rows."""
    lens, packed = c["lens"], c["packed"]
    cu = [0]
    for a, _ in lens:
        cu.append(cu[-1] + a)
    q = c["q"].to(DEV)
    kw = dict(c["opt"], max_seqlen_k=max_k, alibi_slopes=None if c["slopes"] is None else c["slopes"].to(DEV))
    if packed:
        kw.update(cu_seqlens_q=i32(cu), max_seqlen_q=max(a for a, _ in lens) if max_q is None else max_q)
    else:
        q = q.view(len(lens), lens[0][0], *q.shape[1:]).transpose(1, 2).contiguous()
    cache = attn.KVCache(*(t.to(DEV) for t in c["pool"]))
    args = (q, cache, c["table"].to(DEV), i32([lk for _, lk in lens]))
    if ws and lib is None:
        out, lse = attn.cache_fwd(*args, **kw, **extra)
    else:  # the C ABI itself: another library, or no workspace
        lib = lib or attn.load()
        out = torch.empty_like(q)
        lse = torch.empty(cm._lse_shape(q, packed), device=DEV)
        cd, d = cm.make_fwd_desc(q, cache, args[2], args[3], out, lse, **kw, **extra)
        nb = lib.attn_cache_workspace_bytes(ctypes.byref(cd), ctypes.byref(d)) if ws else 0
        w = torch.empty(max(nb, 16), dtype=torch.uint8, device=DEV)
        _abi.check(lib.attn_cache_fwd(q.data_ptr(), out.data_ptr(), lse.data_ptr(), ctypes.byref(cd),
                                      ctypes.byref(d), w.data_ptr() if nb else None, nb), lib)
    torch.cuda.synchronize()
    if packed:
        return out.cpu(), lse.cpu().t()
    return out.cpu().transpose(1, 2).flatten(0, 1), lse.cpu().transpose(1, 2).flatten(0, 1)


def schedules(c):
    """The kernels that a call may take: the library's choice and each of them."""
    fp32, d = c["dt"] == "fp32", c["q"].shape[-1]
    two = 1 if fp32 else 2
    yield None
    yield dict(kernel=1, waves=4, tiles=1)
    yield dict(kernel=1, waves=8, tiles=two, splits=3)
    yield dict(kernel=2, waves=4)
    yield dict(kernel=2, waves=4 if d == 64 else 8, splits=2)


def check_case(c, scheds=None, **how):
    got = []
    for sched in scheds or ([None] if "lib" in how else schedules(c)):
        out, lse = run_case(c, schedule=sched, **how)
        assert bool(torch.isfinite(out.float()).all()), sched
        got.append((sched, out, lse))
    k, v, ks, vs = c["pool"]
    kd, vd = ref.decode(k, c["fmt"]), ref.decode(v, c["fmt"])
    at, held = 0, c["table"].shape[1] * c["bs"]
    group = c["q"].shape[1] // c["hkv"]
    for r, (n, lk) in enumerate(c["lens"]):
        keys = min(lk, held)
        kk, there = ref.dense(kd, ks, c["table"][r], keys, c["bs"])
        vv, _ = ref.dense(vd, vs, c["table"][r], keys, c["bs"], True)
        kk[:, ~there], vv[:, ~there] = 0.0, 0.0
        want = ref.attention(c["q"][at:at + n], kk, vv, lk, group=group, slopes=c["slopes"], there=there, **c["opt"])
        for sched, out, lse in got:
            check_rows(f"request {r} ({n} x {lk}), schedule {sched}", out[at:at + n], lse[at:at + n], want, c["dt"])
        at += n


SHAPES = [("e4m3", "bf16", 128, 8, 2, 64), ("e5m2", "bf16", 64, 12, 4, 16), ("e4m3", "fp32", 64, 4, 4, 32),
          ("e5m2", "fp32", 128, 8, 1, 128), ("e4m3", "bf16", 64, 48, 2, 128), ("e4m3", "bf16", 128, 3, 3, 16)]
IDS = ["-".join(map(str, s)) for s in SHAPES]


def shaped(s, **more):
    return attention_case(**dict(zip(("fmt", "dt", "d", "hq", "hkv", "bs"), s)), **more)


@pytest.mark.parametrize("s", SHAPES, ids=IDS)
def test_decode_lengths(s):
    """One query against 1 key, tile edges, and long odd lengths; a request without keys."""
    lens = [(1, n) for n in (1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 0, 2049)]
    check_case(shaped(s, lens=lens, causal=False))
    check_case(shaped(s, lens=lens, packed=False, seed=1), max_k=2049)


@pytest.mark.parametrize("s", SHAPES, ids=IDS)
def test_few_and_many_queries(s):
    """Packed requests of 0 to some hundred queries; more queries than keys (rows without any)."""
    lens = [(3, 70), (0, 10), (17, 17), (1, 300), (129, 200), (5, 2), (64, 64), (33, 0), (300, 431)]
    check_case(shaped(s, lens=lens, seed=2))
    check_case(shaped(s, lens=[(5, 77), (5, 1), (5, 600)], packed=False, seed=3))
    check_case(shaped(s, lens=[(1, 5), (2, 100), (0, 50), (4, 333)], causal=False, seed=4))


@pytest.mark.parametrize("s", SHAPES, ids=IDS)
@pytest.mark.parametrize("window", [(0, 0), (5, 0), (63, 0), (100, 7), (-1, 3), (20, -1), (2, 300)])
def test_windows(s, window):
    lens = [(1, 500), (4, 131), (1, 3), (70, 260), (6, 4)]
    check_case(shaped(s, lens=lens, window=window, seed=5))
    check_case(shaped(s, lens=lens[:3], window=window, seed=6))


@pytest.mark.parametrize("s", SHAPES, ids=IDS)
@pytest.mark.parametrize("softcap, alibi", [(50.0, False), (0.0, True), (5.0, True), (1e4, False)])
def test_score_options(s, softcap, alibi):
    check_case(shaped(s, lens=[(1, 400), (3, 77), (90, 190), (2, 1)], softcap=softcap, alibi=alibi, qscale=2.0, seed=7))
    check_case(shaped(s, lens=[(1, 400), (3, 77)], softcap=softcap, alibi=alibi, window=(50, 2), seed=8))


@pytest.mark.parametrize("s", SHAPES[:4], ids=IDS[:4])
def test_key_splits(s):
    """Long keys over few requests, split over workgroups or (without a workspace) not."""
    c = shaped(s, lens=[(1, 9001), (1, 40), (2, 5000)], seed=9)
    check_case(c)
    check_case(c, ws=False)
    check_case(shaped(s, lens=[(40, 6000), (33, 100)], seed=10))
    check_case(shaped(s, lens=[(1, 9001), (1, 512)], window=(4000, 0), seed=11))


def test_longer_than_told():
    """max_seqlen_k only sizes the splits."""
    c = attention_case(lens=[(1, 9001), (1, 100)], seed=12)
    check_case(c, max_k=3000)
    check_case(c, max_k=0)


@pytest.mark.parametrize("batch", [40, 64, 65])
def test_longest_first(batch):
    """More workgroups than fit the chip at once, whole requests each (up to 64 of them in the
    order of their lengths): equal lengths, none, one token, and many."""
    rng = random.Random(batch)
    lens = [(1, rng.choice([0, 1, 5, 5, 70, rng.randint(1, 400)])) for _ in range(batch)]
    few = attention_case(d=64, hq=8, hkv=8, bs=16, lens=lens, seed=60)
    many = attention_case(d=64, hq=32, hkv=8, bs=16, lens=[(rng.choice([0, 1, 33]), lk) for _, lk in lens], seed=61)
    check_case(few, [dict(kernel=1, waves=8, tiles=1, splits=1), dict(kernel=1, waves=4, tiles=1, splits=1)])
    check_case(many, [dict(kernel=2, waves=4, splits=1)])


@pytest.mark.parametrize("n", [1, 40])
def test_tables(n):
    """Entries outside the pool hide their keys; so does the end of a narrow table."""
    check_case(attention_case(bs=16, lens=[(n, 200), (n, 90)], bad=[(0, 3, -1), (0, 12, 99999), (1, 0, -2 ** 31)], seed=13))
    check_case(attention_case(bs=64, lens=[(n, 300), (n, 700)], bad=[(0, 1, 2 ** 31 - 1)], seed=14))
    check_case(attention_case(bs=32, lens=[(n, 300), (n, 60)], width=4, seed=15))
    check_case(attention_case(bs=16, lens=[(n, 100), (n, 17)], bad=[(r, c, -1) for r in (0, 1) for c in range(7) if c < 7 - 5 * r], seed=16))


def test_freed_blocks_behind_a_window():
    """Blocks that no row's window reaches may be given back, and hold anything."""
    c = attention_case(bs=16, lens=[(2, 400), (1, 333)], window=(40, 0), seed=17)
    k, v, ks, vs = c["pool"]
    for r, lk in ((0, 400), (1, 333)):
        for col in range((lk - 2 - 40) // 16):
            b = int(c["table"][r, col])
            k.view(torch.uint8)[b], v.view(torch.uint8)[b], ks[b], vs[b] = 0x7F, 0x7F, math.nan, math.nan
    check_case(c, validate=True)


@pytest.mark.parametrize("n", [1, 40])
def test_scales_of_zero_and_far_apart(n):
    """A block whose scale is 0 holds zeros; neighbours may differ by many powers of two."""
    for dt in ("bf16", "fp32"):
        c = attention_case(dt=dt, bs=16, lens=[(n, 300), (n, 90)], hq=4, seed=21)
        k, v, ks, vs = c["pool"]
        for i, f in ((1, 0.0), (3, 2.0 ** -20), (7, 8.0)):
            ks[c["table"][0, i]] *= f
        for i, f in ((2, 0.0), (4, 2.0 ** -30), (9, 2.0 ** 20), (11, 0.0)):
            vs[c["table"][0, i]] *= f
        ks[c["table"][1, 0]] = 0.0
        check_case(c)
        check_case(dict(c, opt=dict(c["opt"], softcap=20.0)))


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("to", [2.0 ** -120, 2.0 ** -78, 2.0 ** -140, 2.0 ** -149])
def test_v_scales_near_the_smallest(n, to):
    """Keys whose V is all but nothing weigh in the row sum as any other: V's scale at the least
    that append writes, and below fp32's normal numbers."""
    for dt in ("bf16", "fp32"):
        c = attention_case(dt=dt, bs=16, lens=[(n, 900), (n, 90)], hq=4, seed=22)
        vs = c["pool"][3]
        for i in range(50):
            if i % 8:
                vs[c["table"][0, i]] = to
        vs[c["table"][1]] = to
        check_case(c)


def test_validate_refuses():
    def call(c, **kw):
        with pytest.raises(attn.AttnError):
            run_case(c, validate=True, **kw)

    good = dict(bs=16, lens=[(1, 100), (2, 30)])
    run_case(attention_case(**good), validate=True)
    call(attention_case(**good, bad=[(0, 6, 1000)]))
    call(attention_case(**good, bad=[(1, 0, -1)]))
    call(attention_case(**good, width=3))
    call(attention_case(**good), max_q=1)


def test_strides_guards_and_rows_behind():
    """q and out as views, a cache that is a layer of a larger pool; rows behind the last request
    and everything around the output keep their bytes; two runs give the same bits."""
    c = attention_case(lens=[(1, 300), (3, 100)], hq=8, seed=18)
    want, lse_want = run_case(c)
    k, v, ks, vs = (t.to(DEV) for t in c["pool"])
    n, h, b, d = k.shape
    big = torch.full((n, 2, h, b, d), 0x7F, dtype=torch.uint8, device=DEV)
    big[:, 1] = k.view(torch.uint8)
    cache = attn.KVCache(big.view(k.dtype)[:, 1], v, ks, vs)
    qkv = torch.randn(9, 20, 128, device=DEV).bfloat16()
    qkv[:4, 4:12] = c["q"].to(DEV)
    guard = torch.full((9, 10, 128), 7.0, device=DEV).bfloat16()
    lse = torch.full((8, 9), 7.0, device=DEV)
    attn.cache_fwd(qkv[:, 4:12], cache, c["table"].to(DEV), i32([300, 100]), causal=True,
                   cu_seqlens_q=i32([0, 1, 4]), max_seqlen_q=3, out=guard[:, 1:9], lse=lse)
    assert bytes_equal(guard[:4, 1:9].cpu(), want) and torch.equal(lse[:, :4].t().cpu(), lse_want)
    assert (guard[4:] == 7).all() and (guard[:, 0] == 7).all() and (guard[:, 9] == 7).all() and (lse[:, 4:] == 7).all()
    # heads before tokens, an expanded q, no lse
    q4 = torch.randn(1, 1, 2, 128, device=DEV).bfloat16().expand(2, 8, 2, 128)
    kw = dict(causal=True)
    a = attn.cache_fwd(q4, cache, c["table"].to(DEV), i32([300, 100]), return_lse=False, **kw)
    o = torch.empty(2, 2, 8, 128, device=DEV, dtype=torch.bfloat16).transpose(1, 2)
    attn.cache_fwd(q4.contiguous(), attn.KVCache(k, v, ks, vs), c["table"].to(DEV), i32([300, 100]), out=o, **kw)
    assert bytes_equal(a, o)


def test_empty_calls():
    cache = attn.new_cache(2, 2, 16, 64)
    table = torch.zeros(0, 3, dtype=torch.int32, device=DEV)
    out, lse = attn.cache_fwd(torch.zeros(0, 4, 1, 64, device=DEV), cache, table, i32([]))
    assert out.shape == (0, 4, 1, 64) and lse.shape == (0, 4, 1)
    out, lse = attn.cache_fwd(torch.zeros(0, 4, 64, device=DEV), cache, torch.zeros(2, 3, dtype=torch.int32, device=DEV),
                              i32([4, 5]), cu_seqlens_q=i32([0, 0, 0]), max_seqlen_q=3)
    assert out.numel() == 0
    # a table without columns: no key is there
    out, lse = attn.cache_fwd(torch.ones(2, 4, 3, 64, device=DEV), cache, torch.zeros(2, 0, dtype=torch.int32, device=DEV),
                              i32([4, 0]))
    assert not out.any() and (lse == -math.inf).all()


def test_nan_reaches_the_rows_that_see_it():
    c = attention_case(lens=[(1, 200)], hq=2, hkv=2, seed=19, spoiled=False)
    k, v, ks, vs = c["pool"]
    k.view(torch.uint8)[int(c["table"][0, 1]), 0, 5] = 0x7F
    for sched in schedules(c):
        out, lse = run_case(c, schedule=sched)
        assert torch.isnan(out[0, 0].float()).all() and torch.isnan(lse[0, 0])
        assert torch.isfinite(out[0, 1].float()).all() and torch.isfinite(lse[0, 1])


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_large_queries(dt):
    """Queries of 2^104, the largest whose products with any stored values stay finite, against
    keys small enough to keep the scores in range."""
    c = attention_case(dt=dt, d=128, hq=2, hkv=1, lens=[(2, 90)], seed=62)
    c["pool"][2].mul_(2.0 ** -104)
    c["q"] = c["q"].clamp(-1, 1) * 2.0 ** 104
    check_case(c)


def test_captured_split_call():
    """A split call and its workspace in two graphs, replayed in turn with new queries."""
    c = attention_case(lens=[(1, 9001), (1, 3000)], seed=63)
    cache = attn.KVCache(*(t.to(DEV) for t in c["pool"]))
    q, table, lens, cu = c["q"].to(DEV), c["table"].to(DEV), i32([9001, 3000]), i32([0, 1, 2])
    kw = dict(causal=True, cu_seqlens_q=cu, max_seqlen_q=1)
    attn.cache_fwd(q, cache, table, lens, **kw)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(attn.cache_fwd(q, cache, table, lens, **kw))
        graphs.append(g)
    for step in range(4):
        q.copy_(torch.randn(q.shape, generator=gen(step)))
        want = attn.cache_fwd(q, cache, table, lens, **kw)
        for g, (o, l) in zip(graphs, outs):
            g.replay()
            assert bytes_equal(o, want[0]) and torch.equal(l, want[1])


def test_far_pages():
    """Blocks whose bytes lie beyond 2^31 and 2^32 from the pool's start."""
    blocks, hkv, bs, d = 70000, 4, 128, 128
    cache = attn.new_cache(blocks, hkv, bs, d)
    pages = [69999, 33000, 1]
    x = torch.randn(3 * bs, hkv, d, generator=gen(20)).bfloat16()
    y = torch.randn(3 * bs, hkv, d, generator=gen(21)).bfloat16()
    slots = slots_of([(p, 0, bs) for p in pages], bs)
    attn.cache_append(cache, x.to(DEV), y.to(DEV), torch.tensor(slots, device=DEV))
    table = torch.tensor([pages], dtype=torch.int32)
    q = torch.randn(2, 8, d, generator=gen(22)).bfloat16()
    small = attn.KVCache(*(t[torch.tensor(pages, device=DEV)] if t.dtype == torch.float32 else
                           t.view(torch.uint8)[torch.tensor(pages, device=DEV)].view(t.dtype) for t in cache))
    kw = dict(causal=True, cu_seqlens_q=i32([0, 2]), max_seqlen_q=2)
    a = attn.cache_fwd(q.to(DEV), cache, table.to(DEV), i32([3 * bs - 5]), **kw)
    b = attn.cache_fwd(q.to(DEV), small, i32([[0, 1, 2]]), i32([3 * bs - 5]), **kw)
    assert bytes_equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.isfinite(a[0].float()).all() and a[0].any()
    values, s = ref.append(torch.zeros(3, hkv, bs, d, dtype=torch.float64), torch.zeros(3, hkv), x,
                           slots_of([(i, 0, bs) for i in range(3)], bs), bs, "e4m3")
    assert torch.equal(ref.decode(small.k, "e4m3"), values) and torch.equal(small.k_scale.cpu().double(), s)


@pytest.mark.parametrize("seed", range(30))
def test_random(seed):
    rng = random.Random(1000 + seed)
    d, bs = rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    hkv = rng.choice([1, 2, 3, 8])
    group = rng.choice([1, 2, 3, 4, 7, 16])
    few = rng.random() < 0.5
    lens = [(rng.randint(0, 4) if few else rng.randint(0, 150), rng.choice([0, 1, rng.randint(1, 300), rng.randint(1, 1500)]))
            for _ in range(rng.randint(1, 6))]
    lens.append((1, 50))
    opt = rng.choice([dict(causal=True), dict(causal=False), dict(window=(rng.randint(0, 200), 0)),
                      dict(window=(rng.randint(-1, 99), rng.randint(-1, 99)))])
    c = attention_case(fmt=rng.choice(["e4m3", "e5m2"]), dt=rng.choice(["bf16", "bf16", "fp32"]), d=d, hq=hkv * group,
                       hkv=hkv, bs=bs, lens=lens, seed=seed, softcap=rng.choice([0.0, 0.0, 30.0]),
                       alibi=rng.random() < 0.3, qscale=rng.choice([0.3, 1.0, 3.0]), **opt)
    check_case(c, ws=rng.random() < 0.7)


# ---- together -------------------------------------------------------------

class Server:
    """Requests over one pool, beside their tokens' keys and values as the cache holds them."""

    def __init__(self, batch, *, bs=16, hkv=2, hq=8, d=64, fmt="e4m3", blocks=40, width=12, seed=0):
        self.bs, self.hq, self.hkv, self.d, self.fmt = bs, hq, hkv, d, fmt
        self.cache = attn.new_cache(blocks, hkv, bs, d, dtype=ref.F8[fmt])
        self.table = torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
        self.free, self.num_free = i32(list(range(blocks))[::-1]), i32([blocks])
        self.lens = i32([0] * batch)
        self.g = gen(seed)

    def tokens(self, n):
        return [torch.randn(n, h, self.d, generator=self.g).bfloat16().to(DEV) for h in (self.hq, self.hkv, self.hkv)]

    def step(self, new, q, k, v, max_q):
        p = attn.cache_plan(self.lens, new, self.table, self.free, self.num_free, block_size=self.bs,
                            total_new=k.shape[0])
        attn.cache_append(self.cache, k, v, p.slots)
        out, lse = attn.cache_fwd(q, self.cache, self.table, p.seqlens_k, causal=True,
                                  cu_seqlens_q=p.cu_seqlens_q, max_seqlen_q=max_q)
        return p, out, lse

    def check(self, before, new, q, k, v, plan, out, lse, table, cache):
        """The step from the state before it (table, cache values and scales on the CPU)."""
        want = ref.plan(self.lens_before, new, table, self.free.tolist(), before, self.bs, k.shape[0])
        assert self.table.cpu().tolist() == want[0] and plan.slots.tolist() == want[1]
        assert plan.seqlens_k.tolist() == want[3] and plan.num_free.item() == want[4]
        sides = []
        for data, scale, x, last, got, gs in ((cache[0], cache[2], k, False, self.cache.k, self.cache.k_scale),
                                              (cache[1], cache[3], v, True, self.cache.v, self.cache.v_scale)):
            values, s = ref.append(data, scale, x.cpu(), want[1], self.bs, self.fmt, last)
            assert torch.equal(ref.decode(got, self.fmt), values) and torch.equal(gs.cpu().double(), s)
            sides.append((values, s))
        for r, n in enumerate(new):
            a, lk = want[2][r], want[3][r]
            kk, there = ref.dense(*sides[0], want[0][r], lk, self.bs)
            vv, _ = ref.dense(*sides[1], want[0][r], lk, self.bs, True)
            rows = ref.attention(q[a:a + n].cpu(), kk, vv, lk, group=self.hq // self.hkv, causal=True, there=there)
            check_rows(f"request {r}", out[a:a + n].cpu(), lse.t()[a:a + n].cpu(), rows, "bf16")

    def snapshot(self):
        self.lens_before = self.lens.tolist()
        k, v, ks, vs = self.cache
        return (self.num_free.item(), self.table.cpu().tolist(),
                (ref.decode(k, self.fmt), ref.decode(v, self.fmt), ks.cpu(), vs.cpu()))


def test_steps_of_a_server():
    """Prompts, decode steps, a late request, one that finds no block, and reuse of its blocks."""
    s = Server(4)
    for new in ([20, 0, 33, 1], [1, 7, 1, 1], [1, 1, 1, 1], [40, 1, 0, 1], [1, 1, 1, 100], [1, 1, 1, 1],
                [0, 200, 3, 1], [12, 1, 1, 15]):
        q, k, v = s.tokens(sum(new))
        num_free, table, cache = s.snapshot()
        plan, out, lse = s.step(i32(new), q, k, v, max(new))
        s.check(num_free, new, q, k, v, plan, out, lse, table, cache)
        s.lens, s.num_free = plan.seqlens_k, plan.num_free


def test_captured_decode_step():
    """A decode step recorded once and replayed over growing requests, beside eager work."""
    s = Server(3, blocks=30, seed=1)
    q, k, v = s.tokens(30)
    plan, _, _ = s.step(i32([17, 3, 10]), q, k, v, 17)
    s.lens, s.num_free = plan.seqlens_k.clone(), plan.num_free.clone()
    one = i32([1, 1, 1])
    q, k, v = s.tokens(3)
    s.step(one, q, k, v, 1)  # (loads the kernels; writes the slots that the first replay writes)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan, out, lse = s.step(one, q, k, v, 1)
        s.lens.copy_(plan.seqlens_k)
        s.num_free.copy_(plan.num_free)
    for step in range(20):
        for x, y in zip((q, k, v), s.tokens(3)):
            x.copy_(y)
        before = s.snapshot()
        graph.replay()
        torch.cuda.synchronize()
        s.check(before[0], [1, 1, 1], q, k, v, plan, out, lse, before[1], before[2])
        torch.zeros(1 << 20, device=DEV).sum().item()
    assert s.lens.tolist() == [37, 23, 30]


def test_two_streams():
    """Calls on two streams, with splits and workspaces of their own, give the bits of calls alone."""
    cases = [attention_case(lens=[(1, 7001), (1, 300)], seed=30 + i, d=(64, 128)[i]) for i in range(2)]
    alone = [run_case(c) for c in cases]
    ins = []
    for c in cases:
        ins.append((c["q"].to(DEV), attn.KVCache(*(t.to(DEV) for t in c["pool"])), c["table"].to(DEV),
                    i32([lk for _, lk in c["lens"]])))
    streams = [torch.cuda.Stream() for _ in cases]
    cu = i32([0, 1, 2])
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(attn.cache_fwd(*ins[i], causal=True, cu_seqlens_q=cu, max_seqlen_q=1))
    torch.cuda.synchronize()
    for i in range(2):
        for o, l in got[i]:
            assert bytes_equal(o.cpu(), alone[i][0]) and torch.equal(l.cpu().t(), alone[i][1])


def test_poisoned_lds():
    """Bit for bit the outputs of a build that fills LDS with all-ones bytes first."""
    import os
    path = os.path.join(os.path.dirname(_abi.LIB_PATH), "libattn_poison.so")
    lib = _abi.load(path)
    for c in (attention_case(lens=[(1, 300), (2, 5000), (1, 1)], seed=40),
              attention_case(lens=[(40, 300), (90, 100)], seed=41, dt="fp32", d=64),
              attention_case(lens=[(40, 300), (90, 100)], seed=41),
              attention_case(lens=[(1, 64)], seed=42, d=64, fmt="e5m2", bs=16)):
        for sched in schedules(c):
            a, b = run_case(c, schedule=sched), run_case(c, lib=lib, schedule=sched)
            assert bytes_equal(a[0], b[0]) and torch.equal(a[1], b[1])
    log("attention ok")
    for runs in (RUNS["prompt"], RUNS["decode"]):
        got = []
        for which in (attn.load(), lib):
            cache = attn.KVCache(*(t.to(DEV) for t in ref.make_pool(gen(43), 12, 2, 16, 128, "e4m3")))
            slots = torch.tensor(slots_of(runs, 16), device=DEV)
            x = torch.randn(slots.numel(), 2, 128, generator=gen(44)).bfloat16().to(DEV) * 9
            cd, d = cm.make_append_desc(cache, x, x, slots)
            _abi.check(which.attn_cache_append(x.data_ptr(), x.data_ptr(), ctypes.byref(cd), ctypes.byref(d)), which)
            d, plan = cm.make_plan_desc(i32([3, 70]), i32([40, 1]), i32([[0, 1, 2], [3, 4, 5]]), i32([7, 8, 9]), i32([3]),
                                        block_size=32, total_new=45)
            _abi.check(which.attn_cache_plan(ctypes.byref(d)), which)
            got.append([*cache, *plan])
        assert all(bytes_equal(a, b) for a, b in zip(*got))


# ---- native marshalling ---------------------------------------------------

def test_native_marshalling_takes_the_calls():
    """Ordinary calls go through binding/fast_cache.cpp and give the Python path's bits; the rest is
    left to that path."""
    native = attn._load_native()
    c = attention_case(lens=[(1, 900), (2, 70)], alibi=True, seed=50)
    cache = attn.KVCache(*(t.to(DEV) for t in c["pool"]))
    q, table, lens, cu = c["q"].to(DEV), c["table"].to(DEV), i32([900, 70]), i32([0, 1, 3])
    slopes = c["slopes"].to(DEV)
    args = [q, cache, table, lens, True, (300, 0), slopes, 30, None, cu, 2, None, None, None, True]
    got = native.cache_fwd(*args)
    kw = dict(window=(300, 0), alibi_slopes=slopes, softcap=30, cu_seqlens_q=cu, max_seqlen_q=2)
    want = attn.cache_fwd(q, cache, table, lens, log=True, **kw)  # log: the Python path
    assert bytes_equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert bytes_equal(native.cache_fwd(*args[:-1], False), want[0])
    out, lse = torch.empty_like(q), torch.empty_like(want[1])
    res = native.cache_fwd(*args[:12], out, lse, True)
    assert res[0] is out and res[1] is lse and bytes_equal(out, want[0])

    x = torch.randn(3, 2, 128, device=DEV).bfloat16()
    slots = torch.tensor([0, 64, 65], device=DEV)
    caches = [attn.KVCache(*(t.clone() for t in cache)) for _ in range(2)]
    assert native.cache_append(caches[0], x, x, slots) is None
    attn.cache_append(caches[1], x, x, slots, log=True)
    assert all(bytes_equal(a, b) for a, b in zip(*caches))
    lens = [i32([900, 70]), i32([30, 5]), table.clone(), i32([3, 2, 1]), i32([3])]
    a = native.cache_plan(*lens, 64, 40)
    b = attn.cache_plan(*lens, block_size=64, total_new=40, log=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))

    # not for it
    assert native.cache_fwd(q.half(), *args[1:]) is NotImplemented
    assert native.cache_fwd(*args[:2], table.long(), *args[3:]) is NotImplemented
    assert native.cache_fwd(q, (cache.k, cache.v), *args[2:]) is NotImplemented
    assert native.cache_append(caches[0], x.cpu(), x, slots) is NotImplemented
    assert native.cache_plan(*lens, 48, 40) is NotImplemented
    for bad in (dict(softcap=-1.0), dict(window=(-3, 0)), dict(max_seqlen_q=None)):
        with pytest.raises((attn.AttnError, ValueError)):
            attn.cache_fwd(q, cache, table, i32([900, 70]), **{**kw, **bad})
    with pytest.raises(attn.AttnError):
        attn.cache_plan(*lens, block_size=48, total_new=40)
    with pytest.raises(ValueError):
        attn.cache_append(caches[0], x.cpu(), x, slots)


def test_a_failed_launch_is_raised_once():
    native = attn._load_native()
    lib, calls = attn.load(), []
    failing = ctypes.CFUNCTYPE(ctypes.c_int, *[ctypes.c_void_p] * 4)(lambda *a: calls.append(1) or -7)
    addr = [ctypes.cast(f, ctypes.c_void_p).value for f in
            (lib.attn_cache_plan, failing, lib.attn_cache_fwd, lib.attn_cache_workspace_bytes)]
    cache = attn.new_cache(2, 2, 16, 64)
    x = torch.randn(1, 2, 64, device=DEV)
    native.bind_cache(*addr)
    try:
        with pytest.raises(attn.AttnError) as e:
            attn.cache_append(cache, x, x, torch.zeros(1, dtype=torch.int64, device=DEV))
    finally:
        attn._load_native()
    assert e.value.status == -7 and len(calls) == 1
