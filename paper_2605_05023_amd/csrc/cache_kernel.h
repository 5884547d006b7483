// cache_kernel.h -- softmax attention to an 8-bit block cache: the kernel that
// cache_fwd_*.hip instantiate.
//
// A wavefront takes 64 consecutive keys at a time against MT tiles of 16 flat
// rows (row f of a kv group: query f / group of head f % group, so K and V are
// read once for all the heads that use them), entirely in registers:
//  * S^T = K Q^T with v_mfma_f32_16x16x32_bf16. Row m of product tile t stands
//    for key 16 (m / 4) + 4 t + m % 4 of the 64, so that the sixteen scores a
//    lane holds of a row (lanes r, r + 16, r + 32, r + 48 share row r) belong to
//    sixteen consecutive keys, 16 g on for g = lane / 16: one page, one scale.
//    The head dim is taken in the order of the loads: a lane's 16 bytes feed two
//    products.
//  * O^T = V^T P^T: those sixteen keys are, as they stand, the lane's share of the
//    B operand, and V, stored transposed, gives the A operand in one 16-byte
//    load per 16 dims. No value of K, V or P passes through LDS or another lane.
//  * 8-bit values become bf16 exactly (both formats have fewer mantissa bits);
//    the scale of a block multiplies the score, that of V the probability,
//    both in fp32. For fp32 calls q and P are split into three bf16 terms (24
//    bits), each with products of its own into the same sums.
// The four or eight wavefronts of a workgroup take every WAVES-th chunk of 64 keys
// and are merged through LDS, and the keys are split over workgroups (cache_many.h:
// many rows). Eight shorten the chain of chunks of a lone request; four fit three
// times to a CU where there is work for all.
// Bound by memory where the batch is large: 32 requests of up to 8192 keys at 32/8
// heads 63-66 us (4.2 TB/s), 2 of 100003 at 128/8 heads 78-82 us (5.1 TB/s); by the
// latency of length, table, K and V one after another where it is small: one request
// 8.8 us a call, 6.4 of them the host's.
#pragma once

#include "cache_params.h"
#include "kernel_params.h"
#include "score_mods.h"

namespace attn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int NT = 256, kWaves = 4;  // (the combine kernel)
constexpr int kChunk = 64;  // keys a wavefront takes at a time

// A row tile of one kv group and the keys its rows see.
struct RowTile {
    int b, hkv, f0, nflat;   // nflat: flat rows of the kv group
    int64_t qrow0;           // packed: first row of the request
    int64_t lk, lq;          // lengths that place the queries on the key axis
    int64_t kend;            // keys the table holds
};

// Visible keys [lo, hi) of query qi (hi <= lo: none).
__device__ __forceinline__ void row_keys(const CacheFwdParams& p, const RowTile& t, int64_t qi, int64_t* lo,
                                         int64_t* hi)
{
    const int64_t ip = qi + t.lk - t.lq;
    *lo = p.wl < 0 ? 0 : max(ip - p.wl, (int64_t)0);
    *hi = p.wr < 0 ? t.kend : min(t.kend, ip + p.wr + 1);
}

// false: a tile without rows.
__device__ __forceinline__ bool row_tile(const CacheFwdParams& p, uint32_t g, uint32_t rt, RowTile* t)
{
    t->b = (int)fast_div(g, p.div_hkv);
    t->hkv = (int)g - t->b * p.pool.hkv;
    t->qrow0 = 0;
    t->lq = p.seqlen_q;
    if (p.cu_q) {
        // (limits for prefix sums that are none: no row outside q and out)
        t->qrow0 = min(max((int64_t)p.cu_q[t->b], (int64_t)0), p.total_q);
        t->lq = max(min((int64_t)p.cu_q[t->b + 1], p.total_q) - t->qrow0, (int64_t)0);
    }
    t->lk = max(p.seqlens[t->b], 0);
    t->kend = min(t->lk, (int64_t)p.width << p.pool.bshift);
    t->nflat = (int)(t->lq * p.div_group.d);
    t->f0 = (int)rt * p.tile_rows;
    return t->f0 < t->nflat;
}

// Chunks [c0, c1) that rows [f0, f0 + n) of the tile see.
__device__ __forceinline__ void tile_chunks(const CacheFwdParams& p, const RowTile& t, int f0, int n, int* c0,
                                            int* c1)
{
    const int q0 = (int)fast_div((uint32_t)f0, p.div_group);
    const int q1 = (int)fast_div((uint32_t)min(f0 + n, t.nflat) - 1u, p.div_group);
    int64_t lo, hi, none;
    row_keys(p, t, q0, &lo, &none);
    row_keys(p, t, q1, &none, &hi);
    *c0 = (int)(lo / kChunk);
    *c1 = hi > lo ? (int)((hi + kChunk - 1) / kChunk) : *c0;
}

__device__ __forceinline__ int split_size(const CacheFwdParams& p, int chunks)
{
    return max(p.split_chunks, (chunks + p.splits - 1) / p.splits);
}

// The request of rank n by its number of keys, longest first (batch <= 64).
__device__ __forceinline__ uint32_t nth_longest(const CacheFwdParams& p, uint32_t n)
{
    const int lane = threadIdx.x & 63, mine = lane < p.batch ? max(p.seqlens[lane], 0) : -1;
    uint32_t rank = 0;
    for (int j = 0; j < p.batch; ++j) {
        const int other = __builtin_amdgcn_readlane(mine, j);
        rank += other > mine || (other == mine && j < lane);
    }
    return (uint32_t)__builtin_ctzll(__builtin_amdgcn_ballot_w64(rank == n && lane < p.batch));
}

// Work item -> (kv group, row tile): the row tiles of a group follow one another
// and, when the groups are a multiple of eight, on one XCD (ids are dealt
// round-robin over the 8 XCDs), so that they meet in its L2. The last ones, which
// see the most keys under a causal mask, come first, and (by_length) the requests
// with the most keys: the workgroups that are left at the end are short ones.
__device__ __forceinline__ void work_item(const CacheFwdParams& p, uint32_t id, uint32_t* g, uint32_t* rt)
{
    const uint32_t groups = (uint32_t)(p.batch * p.pool.hkv), nrt = (uint32_t)p.row_tiles;
    if (groups % 8 == 0) {
        const uint32_t k = id >> 3;
        *rt = k % nrt;
        *g = (id & 7) + 8 * (k / nrt);
    } else {
        *rt = id % nrt;
        *g = id / nrt;
    }
    *rt = nrt - 1 - *rt;
    if (p.by_length) {
        const uint32_t n = fast_div(*g, p.div_hkv), h = *g - n * (uint32_t)p.pool.hkv;
        *g = nth_longest(p, n) * (uint32_t)p.pool.hkv + h;
    }
}

template <bool E5M2, bool HI>
__device__ __forceinline__ bf16x2 to_bf16(uint32_t w)
{
    if constexpr (E5M2) return __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, HI);
    else return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI);
}

template <bool E5M2>
__device__ __forceinline__ bf16x8 to_bf16x8(uint32_t a, uint32_t b)
{
    const bf16x2 w0 = to_bf16<E5M2, false>(a), w1 = to_bf16<E5M2, true>(a);
    const bf16x2 w2 = to_bf16<E5M2, false>(b), w3 = to_bf16<E5M2, true>(b);
    return bf16x8{w0[0], w0[1], w1[0], w1[1], w2[0], w2[1], w3[0], w3[1]};
}

// Maximum and sum over the lanes that share a row (lane mod 16), without LDS:
// each swap leaves the two halves (of 16, then 32 lanes) side by side.
template <class F>
__device__ __forceinline__ float over_row(float x, F f)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x);
    const auto p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    const uint32_t c = __builtin_bit_cast(
        uint32_t, f(__builtin_bit_cast(float, (uint32_t)p[0]), __builtin_bit_cast(float, (uint32_t)p[1])));
    const auto q = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    return f(__builtin_bit_cast(float, (uint32_t)q[0]), __builtin_bit_cast(float, (uint32_t)q[1]));
}
__device__ __forceinline__ float row_max(float x)
{
    return over_row(x, [](float a, float b) { return __builtin_fmaxf(a, b); });
}
__device__ __forceinline__ float row_sum(float x)
{
    return over_row(x, [](float a, float b) { return a + b; });
}

// Eight elements of q as NS bf16 terms.
template <class T, int NS>
__device__ __forceinline__ void load_q(const T* s, bf16x8 (&q)[NS])
{
    if constexpr (NS == 1) {
        q[0] = *reinterpret_cast<const bf16x8*>(s);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = s[e];
            const __bf16 a = (__bf16)x, b = (__bf16)(x - (float)a);
            q[0][e] = a;
            q[1][e] = b;
            q[2][e] = (__bf16)(x - (float)a - (float)b);
        }
    }
}

// Wait for q here: a loop that may begin with its loads in flight waits for all
// loads, those for the next chunk included, wherever it uses q.
template <int MT, int KS, int NS>
__device__ __forceinline__ void arrived(const bf16x8 (&q)[MT][KS][NS])
{
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int n = 0; n < NS; ++n) asm volatile("" ::"v"(q[m][k][n]));
}

// w as NS bf16 terms, element j of each.
template <int NS>
__device__ __forceinline__ void split_p(float w, bf16x8 (&p)[NS], int j)
{
    const __bf16 a = (__bf16)w;
    p[0][j] = a;
    if constexpr (NS == 3) {
        const __bf16 b = (__bf16)(w - (float)a);
        p[1][j] = b;
        p[2][j] = (__bf16)(w - (float)a - (float)b);
    }
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Score options, one instantiation each: ALiBi alone, the soft-cap in either
// form (with ALiBi, whose slopes are then 0 where there are none).
enum : int { kModsNone = 0, kModsAlibi = 1, kModsCapShort = 2, kModsCapExact = 3 };

// What the softmax of one 16-row tile needs of the chunk: scores s of this lane's
// sixteen keys (from `key` on) under the scales ks and vs of their block.
struct ChunkScales {
    float ks, vs;        // 0 without a block
    float lvs, ivs;      // log2 and inverse of vs (of 1 where it is tiny)
    bool tiny;           // vs is 0, or so small that P vs would leave the normal numbers
    int key, page;       // first key; its block, -1: none
    bool whole;          // every row of the wavefront sees all 64 keys, and no vs is tiny
};

__device__ __forceinline__ ChunkScales chunk_scales(float ks, float vs, int key, int page, bool inside)
{
    ChunkScales c;  // (a page that is not there: scales of 0 in place of block 0's)
    c.ks = page < 0 ? 0.0f : ks;
    c.vs = page < 0 ? 0.0f : vs;
    c.tiny = !(c.vs >= 0x1p-80f);
    const float v = c.tiny ? 1.0f : vs;
    c.lvs = __builtin_amdgcn_logf(v);
    c.ivs = __builtin_amdgcn_rcpf(v);
    c.key = key;
    c.page = page;
    c.whole = inside && __builtin_amdgcn_ballot_w64(c.tiny) == 0;
    return c;
}

// One online-softmax step of a row tile, in two parts.
// softmax_max: score options and mask on s in place, then the running maximum.
// O and the sum are rescaled only where a maximum grows by more than 8 (P stays
// below 2^8, whose bf16 has the same relative error). Returns the factor that
// makes the scores of s.
template <int DT, int MODS>
__device__ __forceinline__ float softmax_max(const CacheFwdParams& p, f32x4 (&s)[4], const ChunkScales& c,
                                             int jlo, int jhi, int ip, float slope, float& mx, float& sum,
                                             f32x4 (&acc)[DT])
{
    float factor = c.ks * p.scale_u;
    if constexpr (MODS != kModsNone) {
        const float from = (float)(ip - c.key);
        // the short form's error, 1e-4 at most (score_mods.h), is far below that of bf16
        const float pre = c.ks * (MODS == kModsCapShort ? p.cap_pre2 : p.cap_pre);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            float x = s[j / 4][j % 4];
            if constexpr (MODS == kModsCapShort) x = softcap_short_u(x, pre, p.cap_post);
            else if constexpr (MODS == kModsCapExact) x = softcap_u(x, pre, p.cap_post);
            else x *= factor;
            s[j / 4][j % 4] = __builtin_fmaf(slope, __builtin_fabsf(from - (float)j), x);
        }
        factor = 1.0f;
    }
    if (!c.whole) {
        asm volatile("");  // a branch: most chunks are whole, and the selects are as long as the rest
        const int lo = jlo - c.key, hi = c.page < 0 ? 0 : jhi - c.key;
        // (a scale of 0: its scores are 0, not 0 * -inf)
        const bool zero = factor == 0.0f;
        factor = zero ? 1.0f : factor;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float x = zero ? 0.0f : s[j / 4][j % 4];
            s[j / 4][j % 4] = j >= lo && j < hi ? x : -__builtin_inff();
        }
    }
    auto x = [&](int j) { return s[j / 4][j % 4]; };
    float top = x(0);
#pragma unroll
    for (int j = 1; j < 15; j += 2) top = __builtin_fmaxf(__builtin_fmaxf(top, x(j)), x(j + 1));
    const float now = row_max(__builtin_fmaxf(top, x(15)) * factor);
    if (__builtin_amdgcn_ballot_w64(now > mx + 8.0f)) {
        const float to = __builtin_fmaxf(mx, now);
        // (a row without a key so far: nothing to scale, and not 2^(inf - inf))
        const float keep = to == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(mx - to);
        mx = to;
        sum *= keep;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[d] *= keep;
    }
    return factor;
}

// softmax_exp: P times V's scale as NS bf16 terms, the B operand of the P V
// products: 2^(score - maximum) and vs are one exponential, of an FMA with the
// score's factor. This lane's share of the row sum takes P without vs.
template <int NS>
__device__ __forceinline__ void softmax_exp(const f32x4 (&s)[4], const ChunkScales& c, float factor, float mx,
                                            float& sum, bf16x8 (&pf)[2][NS])
{
    const float shift = c.lvs - (mx == -__builtin_inff() ? 0.0f : mx);
    float add[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j / 4][j % 4], factor, shift));
        add[j % 4] += e;
        split_p<NS>(e, pf[j / 8], j % 8);
    }
    sum = __builtin_fmaf((add[0] + add[1]) + (add[2] + add[3]), c.ivs, sum);
}

// Where V's scale is tiny (that of a block of zeros is 2^-120), softmax_exp left it
// out, so that the row sum has all of P, and it comes in here. P vs below fp32's
// normal numbers may be lost.
template <int MT, int NS>
__device__ __forceinline__ void scale_tiny(const ChunkScales& c, bf16x8 (&pf)[MT][2][NS])
{
    if (!c.whole && c.tiny) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float x = 0.0f;
#pragma unroll
                    for (int n = NS - 1; n >= 0; --n) x += (float)pf[m][k][n][e];
                    split_p<NS>(x * c.vs, pf[m][k], e);
                }
    }
}

// The bytes of dword i of a lane's sixteen keys that lie in [lo, hi).
__device__ __forceinline__ uint32_t byte_mask(int i, int lo, int hi)
{
    const int a = min(max(lo - 4 * i, 0), 4), b = min(max(hi - 4 * i, 0), 4);
    const uint32_t below_b = b == 4 ? ~0u : (1u << (8 * b)) - 1u;
    const uint32_t below_a = a == 4 ? ~0u : (1u << (8 * a)) - 1u;
    return below_b & ~below_a;
}

// Where a row's O, row sum and maximum go: to the output, or to the partials of
// a split, which are in the order of the LSE.
template <int D, class T>
struct Writer {
    const CacheFwdParams& p;
    const RowTile& t;
    int64_t part;  // first partial row of the split, or -1

    // Query and head of flat row f, and its row of the LSE.
    __device__ __forceinline__ void place(int f, int* qi, int64_t* h) const
    {
        *qi = (int)fast_div((uint32_t)f, p.div_group);
        *h = t.hkv * (int)p.div_group.d + (f - *qi * (int)p.div_group.d);
    }
    __device__ __forceinline__ int64_t lse_row(int f) const
    {
        int qi;
        int64_t h;
        place(f, &qi, &h);
        return p.cu_q ? h * p.total_q + t.qrow0 + qi : ((int64_t)t.b * p.hq + h) * p.seqlen_q + qi;
    }
    __device__ __forceinline__ void scalars(int f, float m, float l) const
    {
        const int64_t row = lse_row(f);
        if (part >= 0) {
            p.ws_ml[2 * (part + row)] = m;
            p.ws_ml[2 * (part + row) + 1] = l;
        } else if (p.lse) {
            p.lse[row] = l == 0.0f ? -__builtin_inff() : (m + __builtin_log2f(l)) * kLn2;
        }
    }
    __device__ __forceinline__ float factor(float l) const  // (a NaN sum reaches O)
    {
        return part >= 0 ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
    }
    // Four dims from d on.
    __device__ __forceinline__ void out(int f, int d, f32x4 x) const
    {
        if (part >= 0) {
            *reinterpret_cast<f32x4*>(p.ws_o + (part + lse_row(f)) * D + d) = x;
            return;
        }
        int qi;
        int64_t h;
        place(f, &qi, &h);
        T* dst = static_cast<T*>(p.o) + (p.cu_q ? t.qrow0 + qi : qi) * p.so_s + h * p.so_h +
                 (p.cu_q ? 0 : t.b * p.so_b) + d;
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<bf16x4*>(dst) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
        else
            *reinterpret_cast<f32x4*>(dst) = x;
    }
};

// T: element of q and out.
template <int D, class T, bool E5M2, int MT, int MODS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void cache_fwd_kernel(CacheFwdParams p)
{
    constexpr int NS = sizeof(T) == 2 ? 1 : 3;  // bf16 terms of q and P
    constexpr int WR = 16 * MT;                 // rows of a wavefront
    constexpr int KS = D / 32, DT = D / 16;     // products along the head dim, tiles of it
    constexpr int HV = D / 64;                  // 16-byte loads of a key row per lane
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4;

    uint32_t group, rt;
    work_item(p, blockIdx.x, &group, &rt);
    RowTile t;
    if (!row_tile(p, group, rt, &t)) return;  // whole workgroup
    int c0, c1;
    tile_chunks(p, t, t.f0, p.tile_rows, &c0, &c1);
    const int sp = blockIdx.y, per = split_size(p, c1 - c0);
    const bool split = c1 - c0 > per;
    if (sp > 0 && c0 + sp * per >= c1) return;  // whole workgroup
    c0 += sp * per;
    c1 = min(c1, c0 + per);
    const Writer<D, T> write{p, t, split ? sp * p.ws_rows : (int64_t)-1};

    // keys that any, and that every row sees
    int lo_any, hi_any, lo_all, hi_all;
    {
        int64_t a, b, c, d;
        row_keys(p, t, (int)fast_div((uint32_t)t.f0, p.div_group), &a, &d);
        row_keys(p, t, (int)fast_div((uint32_t)min(t.f0 + WR, t.nflat) - 1u, p.div_group), &c, &b);
        lo_any = (int)min(a, t.kend);
        hi_any = (int)max(b, (int64_t)0);
        lo_all = (int)min(c, t.kend);
        hi_all = (int)max(d, (int64_t)0);
    }

    // q: lane holds dims 64 h + 16 g + 8 e .. + 7 of its row for product 2 h + e
    bf16x8 qf[MT][KS][NS];
    int jlo[MT], jhi[MT], ip[MT];
    float slope[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int f = min(t.f0 + 16 * m + r, t.nflat - 1);
        const int qi = (int)fast_div((uint32_t)f, p.div_group);
        const int64_t h = t.hkv * (int)p.div_group.d + (f - qi * (int)p.div_group.d);
        int64_t a, b;
        row_keys(p, t, qi, &a, &b);
        jlo[m] = (int)min(a, t.kend);
        jhi[m] = (int)max(b, (int64_t)0);
        ip[m] = (int)(qi + t.lk - t.lq);
        slope[m] = MODS != kModsNone && p.slopes ? -p.slopes[h] * kLog2e : 0.0f;
        const T* src = static_cast<const T*>(p.q) + (p.cu_q ? t.qrow0 + qi : qi) * p.sq_s + h * p.sq_h +
                       (p.cu_q ? 0 : t.b * p.sq_b) + 16 * g;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            load_q<T, NS>(src + 64 * (k / 2) + 8 * (k % 2), qf[m][k]);
        }
    }

    f32x4 acc[MT][DT];
    float mx[MT], sum[MT];  // running maximum of the row; this lane's share of the sum
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        mx[m] = -__builtin_inff();
        sum[m] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[m][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    const int bshift = p.pool.bshift, bs1 = (1 << bshift) - 1;
    const int32_t* table = p.table + t.b * p.stride_table;
    // The table entries of a chunk's keys are read one chunk ahead, without a
    // branch (a column past the end is the last one); which of them count is
    // decided when they are used: -1 where no row sees any of the 16 keys from
    // key16 on, or the entry is none of a block.
    int entry_k = -1, entry_v = -1;
    auto fetch = [&](int c) __attribute__((always_inline)) {
        entry_k = table[min((c * kChunk + 16 * (r >> 2)) >> bshift, p.width - 1)];
        entry_v = table[min((c * kChunk + 16 * g) >> bshift, p.width - 1)];
    };
    auto page_of = [&](int key16, int entry) __attribute__((always_inline)) -> int {
        return key16 < hi_any && key16 + 16 > lo_any && (uint32_t)entry < (uint32_t)p.pool.num_blocks ? entry
                                                                                                      : -1;
    };
    if (c0 + wave < c1) fetch(c0 + wave);
    arrived(qf);
    for (int c = c0 + wave; c < c1; c += WAVES) {
        const int base = c * kChunk, key_k = base + 16 * (r >> 2), key_v = base + 16 * g;
        const int page_k = page_of(key_k, entry_k), page_v = page_of(key_v, entry_v);
        fetch(c + WAVES);
        // (a page that is not there: block 0 is read and masked out)
        const uint8_t* kp = p.pool.k + (int64_t)max(page_k, 0) * p.pool.sk_b + t.hkv * p.pool.sk_h +
                            ((key_k & bs1) + (r & 3)) * D + 16 * g;
        const uint8_t* vp = p.pool.v + (int64_t)max(page_v, 0) * p.pool.sv_b + t.hkv * p.pool.sv_h +
                            (r << bshift) + (key_v & bs1);
        u32x4 kw[4][HV], vw[DT];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int h = 0; h < HV; ++h) kw[u][h] = *reinterpret_cast<const u32x4*>(kp + 4 * u * D + 64 * h);
        const float ks = p.pool.k_scale[max(page_v, 0) * p.pool.sks_b + t.hkv];
        const float vs = p.pool.v_scale[max(page_v, 0) * p.pool.svs_b + t.hkv];
#pragma unroll
        for (int d = 0; d < DT; ++d) vw[d] = *reinterpret_cast<const u32x4*>(vp + (d << (4 + bshift)));

        f32x4 s[MT][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
            for (int m = 0; m < MT; ++m) s[m][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const bf16x8 a = to_bf16x8<E5M2>(kw[u][k / 2][2 * (k % 2)], kw[u][k / 2][2 * (k % 2) + 1]);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = NS - 1; n >= 0; --n) s[m][u] = mfma(a, qf[m][k][n], s[m][u]);
            }
        }

        const ChunkScales cs =
            chunk_scales(ks, vs, key_v, page_v, base >= lo_all && base + kChunk <= hi_all);
        if (!cs.whole) {
            // bytes of V that no row sees weigh 0, whatever they hold
            const int lo = min(max(lo_any - key_v, 0), 16);
            const int hi = page_v < 0 ? 0 : min(max(hi_any - key_v, 0), 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t keep = byte_mask(i, lo, hi);
#pragma unroll
                for (int d = 0; d < DT; ++d) vw[d][i] &= keep;
            }
        }

        bf16x8 pf[MT][2][NS];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const float factor =
                softmax_max<DT, MODS>(p, s[m], cs, jlo[m], jhi[m], ip[m], slope[m], mx[m], sum[m], acc[m]);
            softmax_exp<NS>(s[m], cs, factor, mx[m], sum[m], pf[m]);
        }
        scale_tiny<MT, NS>(cs, pf);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bf16x8 a = to_bf16x8<E5M2>(vw[d][2 * k], vw[d][2 * k + 1]);
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = NS - 1; n >= 0; --n) acc[m][d] = mfma(a, pf[m][k][n], acc[m][d]);
            }
    }

#pragma unroll
    for (int m = 0; m < MT; ++m) sum[m] = row_sum(sum[m]);
    // merge the wavefronts: every row's O, maximum and sum through LDS (rows of
    // D + 4 floats: the lanes of a quarter wave write 16 rows to other banks)
    constexpr int LD = D + 4;
    __shared__ __attribute__((aligned(16))) float lo_[WAVES][WR * LD];
    __shared__ float lml[WAVES][WR][2];
    if constexpr (kLdsPoison) {
        for (int i = threadIdx.x; i < WAVES * WR * LD; i += 64 * WAVES)
            (&lo_[0][0])[i] = __builtin_bit_cast(float, ~0u);
        for (int i = threadIdx.x; i < WAVES * WR * 2; i += 64 * WAVES)
            (&lml[0][0][0])[i] = __builtin_bit_cast(float, ~0u);
        __syncthreads();
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if (g == 0) {
            lml[wave][16 * m + r][0] = mx[m];
            lml[wave][16 * m + r][1] = sum[m];
        }
#pragma unroll
        for (int d = 0; d < DT; ++d)
            *reinterpret_cast<f32x4*>(&lo_[wave][(16 * m + r) * LD + 16 * d + 4 * g]) = acc[m][d];
    }
    __syncthreads();
    constexpr int COLS = D / 4;
    for (int i = threadIdx.x; i < WR * COLS; i += 64 * WAVES) {
        const int row = i / COLS, col = 4 * (i % COLS), f = t.f0 + row;
        if (f >= t.nflat) break;
        float top = -__builtin_inff(), l = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = __builtin_fmaxf(top, lml[w][row][0]);
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            // (no key seen by any: weight 1 of nothing)
            const float mw = lml[w][row][0];
            const float k = mw == top ? 1.0f : __builtin_amdgcn_exp2f(mw - top);
            l = __builtin_fmaf(lml[w][row][1], k, l);
            o += *reinterpret_cast<const f32x4*>(&lo_[w][row * LD + col]) * k;
        }
        if (col == 0) write.scalars(f, top, l);
        write.out(f, col, o * write.factor(l));
    }
}

}  // namespace
}  // namespace attn
