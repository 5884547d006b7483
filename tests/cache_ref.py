"""Plain 64-bit forms of the 8-bit block cache's operators, from their
definitions (include/attn.h), and the inputs of their tests. Nothing here uses
the library."""
import math

import numpy as np
import torch

F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
MAX = {"e4m3": 448.0, "e5m2": 57344.0}
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def cdiv(a, b):
    return -(-a // b)


def code_values(fmt):
    """The value of each of the 256 codes of a format, by its definition."""
    ebits, mbits, bias = (4, 3, 7) if fmt == "e4m3" else (5, 2, 15)
    out = np.empty(256)
    for code in range(256):
        e, m = code >> mbits & ((1 << ebits) - 1), code & ((1 << mbits) - 1)
        x = m * 2.0 ** (1 - bias - mbits) if e == 0 else (1 + m / (1 << mbits)) * 2.0 ** (e - bias)
        if fmt == "e4m3" and e == 15 and m == 7:
            x = math.nan
        if fmt == "e5m2" and e == 31:
            x = math.inf if m == 0 else math.nan
        out[code] = -x if code & 128 else x
    return out


def decode(t, fmt):
    """Values of an 8-bit tensor in float64."""
    return torch.from_numpy(code_values(fmt)[t.cpu().view(torch.uint8).numpy()])


def round8(x, fmt):
    """float64 values to the format: nearest even, limited to +-MAX, NaN kept."""
    mbits, emin = (3, -6) if fmt == "e4m3" else (2, -14)
    x = torch.as_tensor(x, dtype=torch.float64)
    _, e = torch.frexp(torch.where(torch.isfinite(x), x, 1.0))
    ulp = torch.exp2((e - 1).clamp(min=emin).double() - mbits)
    y = torch.where(torch.isfinite(x), torch.round(x / ulp) * ulp, x)
    return y.clamp(-MAX[fmt], MAX[fmt])


def scale_for(amax, fmt):
    """The smallest 2^e, e >= -120, with amax <= MAX 2^e."""
    e = -120
    while amax > MAX[fmt] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def plan(cached, new, table, free, num_free, bs, total):
    """(table, slots, cu, seqlens, num_free) by walking the requests."""
    table = [list(map(int, r)) for r in table]
    width = len(table[0]) if table else 0
    avail = min(max(int(num_free), 0), len(free))
    asked = taken = 0
    slots, cu, lens = [], [0], []
    for r, (c, n) in enumerate(zip(cached, new)):
        first, last = cdiv(c, bs), cdiv(c + n, bs)
        need = last - first if last <= width else 0
        granted = last <= width and (need == 0 or asked + need <= avail)
        if granted:
            for u in range(need):
                table[r][first + u] = int(free[avail - 1 - asked - u])
            if need:
                taken = asked + need
        asked += need
        for t in range(n):
            block = table[r][(c + t) // bs] if granted else -1
            slots.append(block * bs + (c + t) % bs if block >= 0 else -1)
        cu.append(cu[-1] + n)
        lens.append(c + n if granted else c)
    slots = (slots + [-1] * total)[:total]
    return table, slots, cu, lens, avail - taken


def append(values, scale, x, slots, bs, fmt, tokens_last=False):
    """New values and scales of K (or V, `tokens_last`): values [blocks, H, bs, D] are
    the stored ones in float64, x [T, H, D]."""
    values, scale = values.clone(), scale.double().clone()
    x = x.double()
    if tokens_last:
        values = values.transpose(2, 3)
    n, t = len(slots), 0
    while t < n:
        s = slots[t]
        if s < 0 or s >= values.shape[0] * bs:
            t += 1
            continue
        end = t + 1
        while end < n and slots[end] >= 0 and slots[end] // bs == s // bs:
            end += 1
        b, place = s // bs, s % bs
        for h in range(values.shape[1]):
            rows = x[t:end, h]
            a = rows[torch.isfinite(rows)].abs()
            now = scale_for(float(a.max()) if a.numel() else 0.0, fmt)
            if place > 0:
                old = float(scale[b, h])
                now = max(now, old)
                if now > old:
                    values[b, h, :place] = round8(values[b, h, :place] * (old / now), fmt)
            values[b, h, place:place + end - t] = round8(rows / now, fmt)
            scale[b, h] = now
        t = end
    return (values.transpose(2, 3).contiguous() if tokens_last else values), scale


def attention(q, kv, vv, lk, *, group, causal=False, window=None, softcap=0.0, slopes=None, scale=None,
              there=None):
    """One request in float64: q [n, Hq, D]; kv, vv [Hkv, keys, D], the values that the table
    holds (perhaps fewer than lk); `there`: keys that are visible at all. Returns (out, lse,
    bound of out's error in fp32 arithmetic, bound of lse's, sum of p |v|)."""
    n, hq, d = q.shape
    keys = kv.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    ip = torch.arange(n, dtype=torch.float64)[:, None] + (lk - n)
    j = torch.arange(keys, dtype=torch.float64)[None, :]
    seen = (j < lk).expand(n, keys).clone()
    if there is not None:
        seen &= there[None, :]
    if window is not None:
        if window[0] >= 0:
            seen &= ip - j <= window[0]
        if window[1] >= 0:
            seen &= j - ip <= window[1]
    elif causal:
        seen &= j <= ip
    out, err, mass = (torch.zeros(n, hq, d, dtype=torch.float64) for _ in range(3))
    lse, lerr = torch.full((n, hq), -math.inf, dtype=torch.float64), torch.zeros(n, hq, dtype=torch.float64)
    if keys == 0:
        return out, lse, err, lerr, mass
    eps = 2.0 ** -24
    for h in range(hq):
        k = torch.where(seen.any(0)[:, None], kv[h // group], 0.0)
        v = torch.where(seen.any(0)[:, None], vv[h // group], 0.0)
        qh = q[:, h].double()
        s = qh @ k.t() * scale
        # rounding of a score, in natural units: D products and their sums, three further
        # factors, the exponential (of a base-2 score, twice its relative error)
        off = eps * (d + 16) * (qh.abs() @ k.abs().t() * scale)
        if softcap:
            s = softcap * torch.tanh(s / softcap)
            # 1 - 2 / (1 + e^2y) from an exponential and a reciprocal, 1 ulp each about 1/2
            off = off + 8 * eps * softcap
        if slopes is not None:
            bias = float(slopes[h]) * (ip - j).abs()
            s = s - bias
            off = off + 4 * eps * bias
        s = s.masked_fill(~seen, -math.inf)
        m = s.amax(1, keepdim=True)
        m = torch.where(m == -math.inf, 0.0, m)
        p = torch.exp(s - m)
        total = p.sum(1, keepdim=True)
        p = p / torch.where(total > 0, total, 1.0)
        off = torch.where(seen, off + eps * (keys + 16 + 4 * (s - m).abs().masked_fill(~seen, 0.0)), 0.0)
        out[:, h] = p @ v
        mass[:, h] = p @ v.abs()
        w = p * off
        err[:, h] = w @ v.abs() + out[:, h].abs() * w.sum(1, keepdim=True) + 1e-30
        lse[:, h] = torch.where(total > 0, m + torch.log(total), -math.inf)[:, 0]
        lerr[:, h] = w.sum(1) + 8 * eps * (lse[:, h].abs().masked_fill(total[:, 0] == 0, 0.0) + 1)
    return out, lse, err, lerr, mass


def dense(cache_values, scale, table, keys, bs, tokens_last=False):
    """[Hkv, keys, D] that a request's table row stands for, and which keys are there at all."""
    n, h = cache_values.shape[:2]
    d = cache_values.shape[2] if tokens_last else cache_values.shape[3]
    out = torch.zeros(h, keys, d, dtype=torch.float64)
    there = torch.zeros(keys, dtype=torch.bool)
    for i in range(min(cdiv(keys, bs), len(table))):
        b = int(table[i])
        if not 0 <= b < n:
            continue
        m = min(bs, keys - i * bs)
        page = cache_values[b] * scale[b].double()[:, None, None]
        page = page.transpose(1, 2) if tokens_last else page
        out[:, i * bs:i * bs + m] = page[:, :m]
        there[i * bs:i * bs + m] = True
    return out, there


def make_pool(g, blocks, hkv, bs, d, fmt, scale=1.0):
    """Random finite codes under scales that are no powers of two."""
    finite = torch.from_numpy(np.flatnonzero(np.isfinite(code_values(fmt))).astype(np.uint8))
    # values of about unit variance: codes near 1 / s of the format
    def side(*shape):
        x = torch.randn((blocks, hkv) + shape, generator=g)
        s = 4.5 / MAX[fmt] * torch.exp(0.5 * torch.randn((blocks, hkv), generator=g)) * scale
        codes = (x * scale / s[:, :, None, None]).clamp(-MAX[fmt], MAX[fmt]).to(F8[fmt])
        # some of every code
        pick = torch.rand(x.shape, generator=g) < 0.01
        some = finite[torch.randint(len(finite), x.shape, generator=g)]
        return torch.where(pick, some, codes.view(torch.uint8)).view(F8[fmt]), s

    k, ks = side(bs, d)
    v, vs = side(d, bs)
    return k, v, ks, vs


def make_tables(g, lens, bs, width=None, spare=3):
    """Tables of requests with `lens` keys in a shuffled pool: (table, blocks, unused blocks)."""
    held = [cdiv(n, bs) for n in lens]
    width = max(held, default=0) if width is None else width
    count = sum(held) + spare
    perm = torch.randperm(count, generator=g).int()
    table = torch.full((len(lens), max(width, 1)), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(held):
        m = min(n, width)
        table[r, :m] = perm[at:at + m]
        at += n
    return table, count, perm[at:].clone()


def spoil(k, v, ks, vs, table, lens, bs):
    """NaN in every byte that no request's tokens fill, and in the scales of unused blocks."""
    used = torch.zeros(k.shape[0], bs, dtype=torch.bool)
    for r, n in enumerate(lens):
        for i in range(cdiv(n, bs)):
            if i < table.shape[1] and 0 <= int(table[r, i]) < k.shape[0]:
                used[int(table[r, i]), :min(bs, n - i * bs)] = True
    k.view(torch.uint8).transpose(1, 2)[~used] = 0x7F
    v.view(torch.uint8).permute(0, 3, 1, 2)[~used] = 0xFF
    ks[~used.any(1)] = math.nan
    vs[~used.any(1)] = math.inf
