// cache_append.hip -- new keys and values into the 8-bit block cache
// (attn_cache_append in include/attn.h states the rounding).
//
// The unit of work is a run: the new tokens of one block, for one head, of K or
// of V. Its scale needs the largest value of the run first, so a run belongs to
// one workgroup (or one wavefront). A workgroup looks at `group` consecutive
// tokens and takes the runs that start there. Where that is one or two (prompts)
// its four wavefronts share each; where it is more (decode steps, one token a
// run) every wavefront takes runs of its own. A wavefront takes segments of 16
// places, keeps the first one's values in registers between the maximum and the
// rounding (only runs of more than 16 places a wavefront are read twice), and
// reads the slots of all tokens that matter to it at once: two round trips to
// memory, the slots, then values and old scale.
// Powers of two as scales keep the growth of a block's scale exact: a stored
// value is only rounded again where it becomes subnormal. V is stored
// transposed, [head_dim][block_size]: a lane keeps one or two dims of a segment
// and writes 16 bytes of each.
// Bound by its stores: the values are read once and written as bytes. Prompts of
// 18000 tokens, 8 heads of 128: 36 us (K alone 15, V 19; a copy of the bytes 24.5);
// a decode step of 256 requests 8.8 us (K alone 4.9, V, whose bytes of one token lie
// a row apart, 8.0).
#include <type_traits>

#include "cache_params.h"
#include "fp8.h"
#include "kernel_params.h"

namespace attn {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int NT = 256, kWaves = 4;

// One run and the share of this wavefront in it: wave `wid` of `nw`.
struct Run {
    int64_t token;
    int block, place, n;
    int wid, nw;
};

// Values over a scale, rounded. `plain`: the scale is a power of two, so that
// its inverse is exact, and the values are finite, so that no quotient is above
// the format's largest value. Otherwise the quotient by the inverse is
// corrected by its remainder (to the nearest float, or within an ulp of it) and
// limited.
struct Divide {
    float s, inv;
    bool plain;
    __device__ Divide(float scale, bool finite) : s(scale)
    {
        const uint32_t b = __builtin_bit_cast(uint32_t, scale);
        plain = (b & 0x7fffffu) == 0 && finite;
        inv = 1.0f / scale;
    }
    template <class F, bool PLAIN>
    __device__ __forceinline__ float quotient(float x) const
    {
        const float y = x * inv;
        if constexpr (PLAIN) return y;
        // (NaN passes the comparison)
        const float z = __builtin_fmaf(__builtin_fmaf(-y, s, x), inv, y);
        return __builtin_fabsf(y) > F::kMax ? __builtin_copysignf(F::kMax, y) : z;
    }
    template <class F, bool PLAIN>
    __device__ __forceinline__ uint32_t pack(float a, float b, float c, float d) const
    {
        return F::round(quotient<F, PLAIN>(a), quotient<F, PLAIN>(b), quotient<F, PLAIN>(c),
                        quotient<F, PLAIN>(d));
    }
};

// Maximum over the wavefront, without LDS: rotations within rows of 16 lanes,
// then swaps of rows and halves.
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, true));  // row_ror:8
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x122, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x121, 0xf, 0xf, true));
    const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max((uint32_t)p[0], (uint32_t)p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max((uint32_t)q[0], (uint32_t)q[1]);
}

// Finite |x|, else 0.
__device__ __forceinline__ float finite_abs(float x)
{
    const float a = __builtin_fabsf(x);
    return a < __builtin_inff() ? a : 0.0f;
}

// The largest |x| as bits, which order like the values (infinities and NaN
// above all): of two bf16 at a time, or of one fp32.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int N>
__device__ __forceinline__ uint32_t max_bits(const __bf16 __attribute__((ext_vector_type(N))) x, uint32_t m)
{
    if constexpr (N == 1) {
        return max(m, (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[0]) & 0x7fffu);
    } else {
        typedef uint32_t words __attribute__((ext_vector_type(N / 2)));
        const words w = __builtin_bit_cast(words, x);
        u16x2 y = __builtin_bit_cast(u16x2, m);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint32_t e = w[i] & 0x7fff7fffu;
            y = __builtin_elementwise_max(y, __builtin_bit_cast(u16x2, e));
        }
        return __builtin_bit_cast(uint32_t, y);
    }
}
template <int N>
__device__ __forceinline__ uint32_t max_bits(const float __attribute__((ext_vector_type(N))) x, uint32_t m)
{
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, __builtin_bit_cast(uint32_t, (float)x[i]) & 0x7fffffffu);
    return m;
}
// The float that the maximum stands for; +inf or NaN: not all were finite.
template <class T>
__device__ __forceinline__ float bits_value(uint32_t m)
{
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, m);
    else return __builtin_bit_cast(float, max(m & 0xffffu, m >> 16) << 16);
}

// Four stored values times f.
template <class F>
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float f)
{
    float a, b, c, d;
    F::template unpack<0>(w, &a, &b);
    F::template unpack<1>(w, &c, &d);
    return F::pack(a * f, b * f, c * f, d * f);
}

// A segment's new values. K: 16 bytes a lane, LPT lanes a token, TPI tokens side
// by side; V: the lane's dims of each token.
template <int D, class T, bool VALUES>
struct Segment {
    static constexpr int EPL = VALUES ? D / 64 : 16 / (int)sizeof(T);  // elements per load
    static constexpr int LPT = D / EPL, TPI = 64 / LPT, LOADS = 16 / TPI;
    typedef T vec __attribute__((ext_vector_type(EPL)));
    vec v[LOADS];

    // Token of load i, as a place of the segment; first element of the lane.
    static __device__ __forceinline__ int place(int i, int lane) { return i * TPI + lane / LPT; }
    static __device__ __forceinline__ int dim(int lane) { return lane % LPT * EPL; }

    // x: element 0 of place 0. Places outside [lo, hi) get a copy of the nearest
    // one, which changes no maximum and is not stored; without any: zeros.
    __device__ __forceinline__ void load(const T* x, int64_t stride, int lo, int hi, int lane)
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) v[i] = vec{};
        if (lo >= hi) return;  // (the same in every lane)
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            v[i] = *reinterpret_cast<const vec*>(x + min(max(place(i, lane), lo), hi - 1) * stride + dim(lane));
    }
    __device__ __forceinline__ uint32_t bits(uint32_t m) const
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) m = max_bits(v[i], m);
        return m;
    }
    __device__ __forceinline__ float finite_amax() const
    {
        float a = 0.0f;
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
#pragma unroll
            for (int e = 0; e < EPL; ++e) a = __builtin_fmaxf(a, finite_abs((float)v[i][e]));
        return a;
    }
};

// Places [lo, hi) of segment `seg` of K into the block.
template <int D, class T, class F, bool PLAIN>
__device__ __forceinline__ void store(const Segment<D, T, false>& s, uint8_t* page, int, int seg, int lo, int hi,
                                      const Divide& div, bool, float, int lane)
{
    using S = Segment<D, T, false>;
#pragma unroll
    for (int i = 0; i < S::LOADS; ++i) {
        const int j = S::place(i, lane);
        if (j < lo || j >= hi) continue;
        uint8_t* dst = page + (16 * seg + j) * D + S::dim(lane);
        uint32_t w[S::EPL / 4];
#pragma unroll
        for (int e = 0; e < S::EPL / 4; ++e)
            w[e] = div.pack<F, PLAIN>((float)s.v[i][4 * e], (float)s.v[i][4 * e + 1], (float)s.v[i][4 * e + 2],
                               (float)s.v[i][4 * e + 3]);
        if constexpr (S::EPL == 8) *reinterpret_cast<u32x2*>(dst) = u32x2{w[0], w[1]};
        else *reinterpret_cast<uint32_t*>(dst) = w[0];
    }
}

// The same of V. A segment that also holds earlier places (below lo) is written
// whole where the scale grew: those scaled down, the places behind the run as
// they are.
template <int D, class T, class F, bool PLAIN>
__device__ __forceinline__ void store(const Segment<D, T, true>& s, uint8_t* page, int bshift, int seg, int lo,
                                      int hi, const Divide& div, bool grown, float again, int lane)
{
    using S = Segment<D, T, true>;
    const bool whole = lo == 0 && hi == 16, old = grown && lo > 0;
    uint8_t* dst = page + (S::dim(lane) << bshift) + 16 * seg;
#pragma unroll
    for (int e = 0; e < S::EPL; ++e) {
        u32x4 w, was = {};
        uint8_t* d = dst + (e << bshift);
        if (old) was = *reinterpret_cast<const u32x4*>(d);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            w[q] = div.pack<F, PLAIN>((float)s.v[4 * q][e], (float)s.v[4 * q + 1][e], (float)s.v[4 * q + 2][e],
                               (float)s.v[4 * q + 3][e]);
            if (old) {
                const uint32_t kept = rescaled<F>(was[q], again);
                uint32_t y = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = 4 * q + i;
                    y |= (j < lo ? kept : j < hi ? w[q] : was[q]) & (0xffu << (8 * i));
                }
                w[q] = y;
            }
        }
        if (whole || old) {
            *reinterpret_cast<u32x4*>(d) = w;
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (j >= lo && j < hi) d[j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
        }
    }
}

template <int D, class T, bool E5M2, bool VALUES>
__device__ __forceinline__ void append_run(const CacheAppendParams& p, int head, const Run& r, uint32_t* red)
{
    using F = Fp8<E5M2>;
    const int lane = threadIdx.x & 63, bshift = p.pool.bshift;
    const int64_t ss = p.sx_s[VALUES];
    const T* x = static_cast<const T*>(p.x[VALUES]) + head * p.sx_h[VALUES] + r.token * ss;
    float* scale = VALUES ? p.pool.v_scale + r.block * p.pool.svs_b + head
                          : p.pool.k_scale + r.block * p.pool.sks_b + head;
    const int end = r.place + r.n, seg0 = r.place >> 4, seg1 = (end + 15) >> 4, mine = seg0 + r.wid;
    auto lo_of = [&](int seg) { return max(r.place - 16 * seg, 0); };
    auto hi_of = [&](int seg) { return min(end - 16 * seg, 16); };
    auto load = [&](Segment<D, T, VALUES>& s, int seg) __attribute__((always_inline)) {
        s.load(x + (16 * seg - r.place) * ss, ss, lo_of(seg), hi_of(seg), lane);
    };

    // the largest finite value of the run
    auto over_run = [&](float x) __attribute__((always_inline)) {
        uint32_t a = __builtin_bit_cast(uint32_t, x);  // (>= 0: ordered as its bits are)
        a = wave_max(a);
        if (r.nw > 1) {
            if (lane == 0) red[r.wid] = a;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) a = max(a, red[w]);
            __syncthreads();  // every wavefront has read `red` (and the scale, above)
        }
        return __builtin_bit_cast(float, a);
    };
    Segment<D, T, VALUES> first;
    load(first, mine);  // (past the run's last segment: no place)
    uint32_t bits = first.bits(0);
    for (int seg = mine + r.nw; seg < seg1; seg += r.nw) {
        Segment<D, T, VALUES> more;
        load(more, seg);
        bits = more.bits(bits);
    }
    const float stored = r.place > 0 ? *scale : 0.0f;
    float amax = over_run(bits_value<T>(bits));
    const bool finite = amax < __builtin_inff();
    if (!finite) {  // an infinity or a NaN among them: over again without those
        amax = first.finite_amax();
        for (int seg = mine + r.nw; seg < seg1; seg += r.nw) {
            Segment<D, T, VALUES> more;
            load(more, seg);
            amax = __builtin_fmaxf(amax, more.finite_amax());
        }
        amax = over_run(amax);
    }
    const float now = __builtin_fmaxf(stored, F::scale_for(amax));
    const bool grown = r.place > 0 && now > stored;
    const float again = stored / now;
    const Divide div(now, finite);
    if (r.wid == 0 && lane == 0) *scale = now;

    uint8_t* page = VALUES ? p.pool.v + r.block * p.pool.sv_b + head * p.pool.sv_h
                           : p.pool.k + r.block * p.pool.sk_b + head * p.pool.sk_h;
    if (grown) {
        // the earlier tokens: K's rows before the run, V's segments before its first
        const int pieces = VALUES ? seg0 * D : r.place * (D / 16);
        for (int i = r.wid * 64 + lane; i < pieces; i += r.nw * 64) {
            uint8_t* at = VALUES ? page + ((i % D) << bshift) + 16 * (i / D) : page + 16 * i;
            u32x4 w = *reinterpret_cast<u32x4*>(at);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = rescaled<F>(w[e], again);
            *reinterpret_cast<u32x4*>(at) = w;
        }
    }
    auto put = [&](auto plain) __attribute__((always_inline)) {
        for (int seg = mine; seg < seg1; seg += r.nw) {
            if (seg != mine) load(first, seg);
            store<D, T, F, decltype(plain)::value>(first, page, bshift, seg, lo_of(seg), hi_of(seg), div, grown,
                                                   again, lane);
        }
    };
    if (div.plain) put(std::true_type{});
    else put(std::false_type{});
}

template <int D, class T, bool E5M2>
__global__ __launch_bounds__(NT) void cache_append_kernel(CacheAppendParams p)
{
    __shared__ uint32_t red[kWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bshift = p.pool.bshift, bs = 1 << bshift;
    if constexpr (kLdsPoison) {
        if (threadIdx.x < kWaves) red[threadIdx.x] = ~0u;
        __syncthreads();
    }
    // (the heads of a group of tokens side by side: they read neighbouring rows)
    const int head = (int)(blockIdx.x % (uint32_t)p.pool.hkv);
    const int64_t t0 = (int64_t)(blockIdx.x / (uint32_t)p.pool.hkv) * p.group;

    // The slots of 192 tokens from the group's first on, and of the one before
    // each: a token starts a run (or ends one) when the one before it lies in
    // another block. A run that starts among the group's, 64 at most, ends
    // within them, as blocks hold 128 tokens at most.
    constexpr int kSpan = 3;
    int64_t slot[kSpan], prev[kSpan];
#pragma unroll
    for (int i = 0; i < kSpan; ++i) {
        const int64_t t = t0 + 64 * i + lane, last = p.total_new - 1;
        const int64_t s = p.slots[min(t, last)], q = p.slots[min(max(t - 1, (int64_t)0), last)];
        slot[i] = t <= last ? s : -1;
        prev[i] = t > 0 && t - 1 <= last ? q : -1;
    }
    auto block_of = [&](int64_t s) { return s >= 0 && s < p.num_slots ? s >> bshift : (int64_t)-1; };
    uint64_t edge[kSpan], leads = 0;
#pragma unroll
    for (int i = 0; i < kSpan; ++i) {
        const bool differs = block_of(slot[i]) != block_of(prev[i]);
        edge[i] = __builtin_amdgcn_ballot_w64(differs);
        if (i == 0) leads = __builtin_amdgcn_ballot_w64(differs && block_of(slot[0]) >= 0 && lane < p.group);
    }
    // (the group's very first token may go on with a run of the group before)
    const bool shared = __builtin_popcountll(leads) <= 2;  // (the same in every wavefront)
    for (int i = 0; leads; ++i) {
        const int at = __builtin_ctzll(leads);
        leads &= leads - 1;
        if (!shared && (i & 3) != wave) continue;
        Run r;
        r.token = t0 + at;
        const int64_t s = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)slot[0], at) |
                          (int64_t)__builtin_amdgcn_readlane((int)(slot[0] >> 32), at) << 32;
        r.block = (int)(s >> bshift);
        r.place = (int)(s & (bs - 1));
        // the next edge, or the block's end
        const uint64_t after = at < 63 ? edge[0] >> (at + 1) : 0;
        r.n = after        ? 1 + __builtin_ctzll(after)
              : edge[1] ? 64 - at + __builtin_ctzll(edge[1])
              : edge[2] ? 128 - at + __builtin_ctzll(edge[2])
                           : bs;
        r.n = min(r.n, bs - r.place);
        r.wid = shared ? wave : 0;
        r.nw = shared ? kWaves : 1;
        if (blockIdx.y == 0) append_run<D, T, E5M2, false>(p, head, r, red);
        else append_run<D, T, E5M2, true>(p, head, r, red);
    }
}

template <int D, class T>
hipError_t launch(const CacheAppendParams& p, bool e5m2, hipStream_t stream)
{
    const dim3 grid((unsigned)((p.total_new + p.group - 1) / p.group * p.pool.hkv), 2);
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
