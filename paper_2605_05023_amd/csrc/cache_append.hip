// cache_append.hip -- new keys and values into the 8-bit block cache
// (attn_cache_append in include/attn.h states the rounding).
//
// The unit of work is a run: the new tokens of one block, for one head, of K or
// of V. Its scale needs the largest value of the run first, so a run belongs to
// one workgroup (or one wavefront), which reads its tokens twice, the second
// time through the caches. A workgroup looks at `group` consecutive tokens and
// takes the runs that start there. Where that is one or two (prompts) its four
// wavefronts share each; where it is more (decode steps, one token a run) every
// wavefront takes runs of its own. Powers of two as scales keep the growth of a
// block's scale exact: a stored value is only rounded again where it becomes
// subnormal. V is stored transposed, [head_dim][block_size]: a lane keeps one or
// two dims of 16 tokens and writes 16 bytes of each.
// Bound by memory: the values are read once from it and written as bytes.
#include "cache_params.h"
#include "fp8.h"
#include "kernel_params.h"

namespace attn {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256, kWaves = 4;

// One run and the share of this wavefront in it: wave `wid` of `nw`.
struct Run {
    int64_t token;
    int block, place, n;
    int wid, nw;
};

// x / s as IEEE division; a power of two by its exact inverse.
struct Divide {
    float s, inv;
    bool pow2;
    __device__ explicit Divide(float scale) : s(scale)
    {
        const uint32_t b = __builtin_bit_cast(uint32_t, scale);
        pow2 = (b & 0x7fffffu) == 0 && b != 0;
        inv = 1.0f / scale;
    }
    __device__ float operator()(float x) const { return pow2 ? x * inv : x / s; }
};

// Finite |x|, else 0.
__device__ __forceinline__ float finite_abs(float x)
{
    const float a = __builtin_fabsf(x);
    return a < __builtin_inff() ? a : 0.0f;
}

template <int D, class T, bool E5M2, bool VALUES>
__device__ __forceinline__ void append_run(const CacheAppendParams& p, int head, const Run& r, float* red)
{
    using F = Fp8<E5M2>;
    constexpr int EPL = 16 / sizeof(T);         // elements per 16-byte load
    constexpr int LPT = D / EPL, TPI = 64 / LPT;  // lanes per token, tokens side by side
    const int lane = threadIdx.x & 63, bs = 1 << p.pool.bshift;
    const T* x = static_cast<const T*>(p.x[VALUES]) + head * p.sx_h[VALUES] + r.token * p.sx_s[VALUES];
    const int64_t ss = p.sx_s[VALUES];

    // the largest finite value of the run
    float amax = 0.0f;
    {
        typedef T vec __attribute__((ext_vector_type(EPL)));
        const T* src = x + (lane % LPT) * EPL;
#pragma unroll 4
        for (int j = r.wid * TPI + lane / LPT; j < r.n; j += r.nw * TPI) {
            const vec v = *reinterpret_cast<const vec*>(src + j * ss);
#pragma unroll
            for (int e = 0; e < EPL; ++e) amax = __builtin_fmaxf(amax, finite_abs((float)v[e]));
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) amax = __builtin_fmaxf(amax, __shfl_xor(amax, d));
        if (r.nw > 1) {
            if (lane == 0) red[r.wid] = amax;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) amax = __builtin_fmaxf(amax, red[w]);
        }
    }
    float* scale = VALUES ? p.pool.v_scale + r.block * p.pool.svs_b + head
                          : p.pool.k_scale + r.block * p.pool.sks_b + head;
    const float before = r.place > 0 ? *scale : 0.0f;
    const float now = __builtin_fmaxf(before, F::scale_for(amax));
    const bool grown = r.place > 0 && now > before;
    const float again = before / now;
    const Divide div(now);
    if (r.nw > 1) __syncthreads();  // every wave has read the scale and `red`
    if (r.wid == 0 && lane == 0) *scale = now;

    if constexpr (!VALUES) {
        uint8_t* page = p.pool.k + r.block * p.pool.sk_b + head * p.pool.sk_h;
        if (grown) {  // earlier tokens: place * D bytes
            for (int i = (r.wid * 64 + lane) * 16; i < r.place * D; i += r.nw * 64 * 16) {
                u32x4 w = *reinterpret_cast<u32x4*>(page + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a, b, c, d;
                    F::template unpack<0>(w[e], &a, &b);
                    F::template unpack<1>(w[e], &c, &d);
                    w[e] = F::pack(a * again, b * again, c * again, d * again);
                }
                *reinterpret_cast<u32x4*>(page + i) = w;
            }
        }
        typedef T vec __attribute__((ext_vector_type(EPL)));
        const int col = (lane % LPT) * EPL;
#pragma unroll 4
        for (int j = r.wid * TPI + lane / LPT; j < r.n; j += r.nw * TPI) {
            const vec v = *reinterpret_cast<const vec*>(x + col + j * ss);
            uint32_t w[EPL / 4];
#pragma unroll
            for (int e = 0; e < EPL / 4; ++e)
                w[e] = F::pack(div((float)v[4 * e]), div((float)v[4 * e + 1]), div((float)v[4 * e + 2]),
                               div((float)v[4 * e + 3]));
            uint8_t* dst = page + (r.place + j) * D + col;
            if constexpr (EPL == 8) *reinterpret_cast<u32x2*>(dst) = u32x2{w[0], w[1]};
            else *reinterpret_cast<uint32_t*>(dst) = w[0];
        }
    } else {
        // segments of 16 places: those with new tokens, and the earlier ones where
        // the scale grew
        constexpr int DPL = D / 64;  // dims per lane
        typedef T vec __attribute__((ext_vector_type(DPL)));
        uint8_t* page = p.pool.v + r.block * p.pool.sv_b + head * p.pool.sv_h;
        const int end = r.place + r.n;
        const int seg0 = grown ? 0 : r.place >> 4, seg1 = (end + 15) >> 4;
        for (int seg = seg0 + r.wid; seg < seg1; seg += r.nw) {
            const int base = seg * 16, lo = max(r.place - base, 0), hi = min(end - base, 16);
            uint8_t* dst = page + lane * DPL * bs + base;
            float f[DPL][16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const bool in = j >= lo && j < hi;
                vec v = {};
                if (in) v = *reinterpret_cast<const vec*>(x + lane * DPL + (base + j - r.place) * ss);
#pragma unroll
                for (int e = 0; e < DPL; ++e) f[e][j] = (float)v[e];
            }
            const bool whole = lo == 0 && hi == 16, old = grown && lo > 0;
#pragma unroll
            for (int e = 0; e < DPL; ++e) {
                u32x4 w, was = {};
                if (old) was = *reinterpret_cast<const u32x4*>(dst + e * bs);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    w[q] = F::pack(div(f[e][4 * q]), div(f[e][4 * q + 1]), div(f[e][4 * q + 2]),
                                   div(f[e][4 * q + 3]));
                    if (old) {
                        // the run's bytes of w, the earlier ones scaled down; those behind
                        // the run keep their value
                        float a, b, c, d;
                        F::template unpack<0>(was[q], &a, &b);
                        F::template unpack<1>(was[q], &c, &d);
                        const uint32_t kept = F::pack(a * again, b * again, c * again, d * again);
                        uint32_t y = 0;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int j = 4 * q + i;
                            const uint32_t s = j < lo ? kept : j < hi ? w[q] : was[q];
                            y |= s & (0xffu << (8 * i));
                        }
                        w[q] = y;
                    }
                }
                if (whole || old) {
                    *reinterpret_cast<u32x4*>(dst + e * bs) = w;
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (j >= lo && j < hi) dst[e * bs + j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
                }
            }
        }
    }
}

template <int D, class T, bool E5M2>
__global__ __launch_bounds__(NT) void cache_append_kernel(CacheAppendParams p)
{
    __shared__ float red[kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bshift = p.pool.bshift, bs = 1 << bshift;
    if constexpr (kLdsPoison) {
        if (threadIdx.x < kWaves) red[threadIdx.x] = __builtin_bit_cast(float, ~0u);
        __syncthreads();
    }
    const int head = blockIdx.y;
    const int64_t t0 = (int64_t)blockIdx.x * p.group;

    // A token starts a run when the one before it lies in another block.
    auto block_of = [&](int64_t t) -> int64_t {
        if (t < 0 || t >= p.total_new) return -1;
        const int64_t s = p.slots[t];
        return s >= 0 && s < p.num_slots ? s >> bshift : -1;
    };
    bool lead = false;
    if (lane < p.group) {
        const int64_t b = block_of(t0 + lane);
        lead = b >= 0 && b != block_of(t0 + lane - 1);
    }
    uint64_t leads = __builtin_amdgcn_ballot_w64(lead);
    const bool shared = __builtin_popcountll(leads) <= 2;  // (the same in every wavefront)
    for (int i = 0; leads; ++i) {
        const int at = __builtin_ctzll(leads);
        leads &= leads - 1;
        if (!shared && (i & 3) != wave) continue;
        Run r;
        r.token = t0 + at;
        const int64_t slot = p.slots[r.token];
        r.block = (int)(slot >> bshift);
        r.place = (int)(slot & (bs - 1));
        // tokens of the run: up to the first of another block, or the block's end
        r.n = 0;
        for (int j0 = 0; j0 < bs; j0 += 64) {
            const uint64_t in = __builtin_amdgcn_ballot_w64(block_of(r.token + j0 + lane) == r.block);
            const int got = ~in ? __builtin_ctzll(~in) : 64;
            r.n += got;
            if (got < 64) break;
        }
        r.n = min(r.n, bs - r.place);
        r.wid = shared ? wave : 0;
        r.nw = shared ? kWaves : 1;
        if (blockIdx.z == 0) append_run<D, T, E5M2, false>(p, head, r, red);
        else append_run<D, T, E5M2, true>(p, head, r, red);
    }
}

template <int D, class T>
hipError_t launch(const CacheAppendParams& p, bool e5m2, hipStream_t stream)
{
    const dim3 grid((unsigned)((p.total_new + p.group - 1) / p.group), (unsigned)p.pool.hkv, 2);
    if (e5m2) hipLaunchKernelGGL((cache_append_kernel<D, T, true>), grid, dim3(NT), 0, stream, p);
    else hipLaunchKernelGGL((cache_append_kernel<D, T, false>), grid, dim3(NT), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheAppendParams& p, int head_dim, bool e5m2, bool fp32,
                               hipStream_t stream)
{
    if (head_dim == 128)
        return fp32 ? launch<128, float>(p, e5m2, stream) : launch<128, __bf16>(p, e5m2, stream);
    return fp32 ? launch<64, float>(p, e5m2, stream) : launch<64, __bf16>(p, e5m2, stream);
}

}  // namespace attn
