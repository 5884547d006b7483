// cache_many.h -- attention to the 8-bit block cache for many rows of a request
// (prompts, chunks of them): the kernel that cache_fwd_*.hip instantiate for
// more than 64 flat rows a kv head.
//
// Products, operand layouts and the treatment of scales are those of
// cache_kernel.h. What differs is who reads K and V: here the wavefronts of a
// workgroup (four, or eight for large calls) take row tiles of their own (16 MT
// rows each) against the same keys. Each chunk of 64 keys is loaded once per
// workgroup, 16 bytes a thread and load, converted to bf16 once (a wavefront that converted all of it for
// itself spent as many instructions on that as on the softmax) and staged in
// LDS, K as [key][dim] and V as [dim][key], two buffers, one barrier a chunk:
// the loads of the next chunk are in flight during the products of this one.
// The operands are read back with ds_read_b128. Their 16-byte pieces are stored
// under an XOR of the piece's index with bits of the row, such that the 16 rows
// that a quarter of a wavefront reads (and the rows it writes) lie in all 64
// banks.
// Per score: half a v_max3, an FMA, an exponential, an add and half a conversion.
// Bound by the issue of matrix and vector instructions under the power limit: 4096
// queries over 8192 keys, 32/8 heads of 128, 428 us (963 TFLOP/s, 80 % of a large
// library product's rate).
#pragma once

#include "cache_kernel.h"

namespace attn {
namespace {

// Swizzled byte offset of 16-byte piece c of row `row` in a staged tile.
template <int D>
__device__ __forceinline__ int k_piece(int row, int c)
{
    // the rows 16 (r / 4) + 4 u + r % 4, r = 0..15, of one operand
    const int x = D == 128 ? (row & 3) | (row >> 4 & 3) << 2 : (row >> 1 & 1) | (row >> 4 & 3) << 1;
    return row * (2 * D) + ((c ^ x) << 4);
}
__device__ __forceinline__ int v_piece(int row, int c)
{
    return row * 128 + ((c ^ (row >> 1 & 7)) << 4);
}

// Order of one set of products: four operand reads ahead, then one for every
// operand used (`uses` products each). The compiler's own order reads an operand
// one product before it is waited for: 4096 queries over 8192 keys 476 against
// 453 us.
template <int READS, int USES, int SET>
__device__ __forceinline__ void issue_order()
{
    __builtin_amdgcn_sched_group_barrier(0x100, 4, SET);
#pragma unroll
    for (int i = 0; i < READS - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, USES, SET);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, SET);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 4 * USES, SET);
}

template <int D, class T, bool E5M2, int MT, int MODS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void cache_many_kernel(CacheFwdParams p)
{
    constexpr int NS = sizeof(T) == 2 ? 1 : 3;
    constexpr int WR = 16 * MT, KS = D / 32, DT = D / 16;
    constexpr int THREADS = 64 * WAVES;
    constexpr int PIECES = D / (16 * WAVES);  // 16-byte loads of K (and of V) per thread and chunk
    static_assert(PIECES >= 1, "a piece for every thread");
    constexpr int TILE = kChunk * D * 2;      // bytes of a staged tile
    __shared__ __attribute__((aligned(1024))) char lds[2][2][TILE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    if constexpr (kLdsPoison) {
        for (int i = tid; i < 4 * TILE / 4; i += THREADS) reinterpret_cast<uint32_t*>(&lds[0][0][0])[i] = ~0u;
        __syncthreads();
    }

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

    // keys that any row of the workgroup, any and every row of the wavefront sees
    const int fw = t.f0 + wave * WR;
    const bool rows = fw < t.nflat;
    int lo_wg, hi_wg, lo_any = 0, hi_any = 0, lo_all = 0, hi_all = 0;
    {
        int64_t a, b, none;
        row_keys(p, t, (int)fast_div((uint32_t)t.f0, p.div_group), &a, &none);
        row_keys(p, t, (int)fast_div((uint32_t)min(t.f0 + p.tile_rows, t.nflat) - 1u, p.div_group), &none, &b);
        lo_wg = (int)min(a, t.kend);
        hi_wg = (int)max(b, (int64_t)0);
        if (rows) {
            int64_t c, d;
            row_keys(p, t, (int)fast_div((uint32_t)fw, p.div_group), &a, &d);
            row_keys(p, t, (int)fast_div((uint32_t)min(fw + WR, t.nflat) - 1u, p.div_group), &c, &b);
            lo_any = (int)min(a, t.kend);
            hi_any = (int)max(b, (int64_t)0);
            lo_all = (int)min(c, t.kend);
            hi_all = (int)max(d, (int64_t)0);
        }
    }

    // q: lane holds dims 32 k + 8 g .. + 7 of its row for product k
    bf16x8 qf[MT][KS][NS];
    int jlo[MT], jhi[MT], ip[MT];
    float slope[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int f = min(fw + 16 * m + r, t.nflat - 1);
        const int qi = (int)fast_div((uint32_t)f, p.div_group);
        const int64_t h = t.hkv * (int)p.div_group.d + (f - qi * (int)p.div_group.d);
        int64_t a, b;
        row_keys(p, t, qi, &a, &b);
        jlo[m] = (int)min(a, t.kend);
        jhi[m] = (int)max(b, (int64_t)0);
        ip[m] = (int)(qi + t.lk - t.lq);
        slope[m] = MODS != kModsNone && p.slopes ? -p.slopes[h] * kLog2e : 0.0f;
        const T* src = static_cast<const T*>(p.q) + (p.cu_q ? t.qrow0 + qi : qi) * p.sq_s + h * p.sq_h +
                       (p.cu_q ? 0 : t.b * p.sq_b) + 8 * g;
#pragma unroll
        for (int k = 0; k < KS; ++k) load_q<T, NS>(src + 32 * k, qf[m][k]);
    }

    f32x4 acc[MT][DT];
    float mx[MT], sum[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        mx[m] = -__builtin_inff();
        sum[m] = 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d) acc[m][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // Loads of one chunk. The table entries of its four groups of 16 keys (one where
    // blocks are larger) are read one chunk earlier, a lane the entry of group
    // lane % 4, without a branch (a column past the end is the last one).
    const int bshift = p.pool.bshift, bs1 = (1 << bshift) - 1;
    const int32_t* table = p.table + t.b * p.stride_table;
    const uint8_t* kbase = p.pool.k + t.hkv * p.pool.sk_h;
    const uint8_t* vbase = p.pool.v + t.hkv * p.pool.sv_h;
    struct Staged {
        u32x4 k[PIECES], v[PIECES];
        float ks, vs;
        int page_v;    // of this thread's pieces of V; -1: none
        int page_s;    // of the keys whose scores this lane holds
    };
    int entry = -1;
    auto fetch = [&](int c) __attribute__((always_inline)) {
        entry = table[min((c * kChunk + 16 * (lane & 3)) >> bshift, p.width - 1)];
    };
    auto load = [&](int c, Staged& s) __attribute__((always_inline)) {
        // -1 where no row of the workgroup sees any of the 16 keys, or the entry is
        // none of a block
        const int base = c * kChunk, mine = base + 16 * (lane & 3);
        const int page = mine < hi_wg && mine + 16 > lo_wg && (uint32_t)entry < (uint32_t)p.pool.num_blocks
                             ? entry
                             : -1;
        const int pages[4] = {__builtin_amdgcn_readlane(page, 0), __builtin_amdgcn_readlane(page, 1),
                              __builtin_amdgcn_readlane(page, 2), __builtin_amdgcn_readlane(page, 3)};
        fetch(c + 1);
        s.page_v = page;
        s.page_s = g & 2 ? g & 1 ? pages[3] : pages[2] : g & 1 ? pages[1] : pages[0];
        s.ks = p.pool.k_scale[max(s.page_s, 0) * p.pool.sks_b + t.hkv];
        s.vs = p.pool.v_scale[max(s.page_s, 0) * p.pool.svs_b + t.hkv];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            // (a wavefront's pieces of K lie in one group)
            const int piece = tid + THREADS * i, row = piece / (D / 16), col = piece % (D / 16);
            const int kg = D == 128 ? (WAVES / 2) * i + (wave >> 1) : wave;
            const int page_k = kg & 2 ? kg & 1 ? pages[3] : pages[2] : kg & 1 ? pages[1] : pages[0];
            s.k[i] = *reinterpret_cast<const u32x4*>(kbase + (int64_t)max(page_k, 0) * p.pool.sk_b +
                                                     ((base + row) & bs1) * D + 16 * col);
            const int d = piece >> 2;
            s.v[i] = *reinterpret_cast<const u32x4*>(vbase + (int64_t)max(page, 0) * p.pool.sv_b +
                                                     (d << bshift) + (mine & bs1));
        }
    };
    auto store = [&](int c, const Staged& s, char* k, char* v) __attribute__((always_inline)) {
        const int base = c * kChunk;
        // V of keys that no row of the workgroup sees weighs 0, whatever it holds
        const bool edge = base < lo_wg || base + kChunk > hi_wg || s.page_v < 0;
        const int key = base + 16 * (tid & 3);
        const int lo = min(max(lo_wg - key, 0), 16), hi = s.page_v < 0 ? 0 : min(max(hi_wg - key, 0), 16);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int piece = tid + THREADS * i, row = piece / (D / 16), col = piece % (D / 16), d = piece >> 2;
            u32x4 w = s.v[i];
            if (edge) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] &= byte_mask(e, lo, hi);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                *reinterpret_cast<bf16x8*>(k + k_piece<D>(row, 2 * col + e)) =
                    to_bf16x8<E5M2>(s.k[i][2 * e], s.k[i][2 * e + 1]);
                *reinterpret_cast<bf16x8*>(v + v_piece(d, 2 * (tid & 3) + e)) =
                    to_bf16x8<E5M2>(w[2 * e], w[2 * e + 1]);
            }
        }
    };

    Staged next;
    if (c0 < c1) {
        fetch(c0);
        load(c0, next);
        store(c0, next, lds[0][0], lds[0][1]);
    }
    __syncthreads();
    arrived(qf);
    for (int c = c0; c < c1; ++c) {
        const int base = c * kChunk, key = base + 16 * g;
        const float ks = next.ks, vs = next.vs;
        const int page = next.page_s;
        const bool more = c + 1 < c1;
        if (more) load(c + 1, next);
        const char* kt = lds[(c - c0) & 1][0];
        const char* vt = lds[(c - c0) & 1][1];
        if (base < hi_any && base + kChunk > lo_any) {
            f32x4 s[MT][4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
#pragma unroll
                for (int m = 0; m < MT; ++m) s[m][u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                const int row = 16 * (r >> 2) + 4 * u + (r & 3);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const bf16x8 a = *reinterpret_cast<const bf16x8*>(kt + k_piece<D>(row, 4 * k + g));
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int n = NS - 1; n >= 0; --n) s[m][u] = mfma(a, qf[m][k][n], s[m][u]);
                }
            }

            issue_order<4 * KS, MT * NS, 0>();
            const ChunkScales cs =
                chunk_scales(ks, vs, key, page, base >= lo_all && base + kChunk <= hi_all);
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
                    const bf16x8 a = *reinterpret_cast<const bf16x8*>(vt + v_piece(16 * d + r, 2 * g + k));
#pragma unroll
                    for (int m = 0; m < MT; ++m)
#pragma unroll
                        for (int n = NS - 1; n >= 0; --n) acc[m][d] = mfma(a, pf[m][k][n], acc[m][d]);
                }
            issue_order<2 * DT, MT * NS, 1>();
        }
        if (more) store(c + 1, next, lds[(c + 1 - c0) & 1][0], lds[(c + 1 - c0) & 1][1]);
        __syncthreads();
    }

#pragma unroll
    for (int m = 0; m < MT; ++m) {
        sum[m] = row_sum(sum[m]);
        const int f = fw + 16 * m + r;
        if (f >= t.nflat) continue;
        const float inv = write.factor(sum[m]);
        if (g == 0) write.scalars(f, mx[m], sum[m]);
#pragma unroll
        for (int d = 0; d < DT; ++d) write.out(f, 16 * d + 4 * g, acc[m][d] * inv);
    }
}

}  // namespace
}  // namespace attn
