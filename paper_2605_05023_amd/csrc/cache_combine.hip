// cache_combine.hip -- add up the partial results of row tiles whose keys were
// split over workgroups (cache_kernel.h): with m the largest running maximum of
// a row's partials and w_s = 2^(m_s - m), O = sum w_s O_s / sum w_s l_s and
// LSE = (m + log2 sum w_s l_s) ln 2. One wavefront per row: 16-byte pieces of
// O, D / 4 lanes side by side, the splits 256 / D apart. It finds the splits of
// its row tile as the attention kernel did; a tile that was not split is
// written already. Bound by the latency of its loads, or memory where the
// partials are many (106 MB 33 us).
#include "cache_kernel.h"

namespace attn {
namespace {

template <int D, class T>
__global__ __launch_bounds__(NT) void cache_combine_kernel(CacheFwdParams p)
{
    constexpr int COLS = D / 4, PAR = 64 / COLS, BATCH = 8;
    const int lane = threadIdx.x & 63;
    uint32_t group, rt;
    work_item(p, blockIdx.x, &group, &rt);
    RowTile t;
    if (!row_tile(p, group, rt, &t)) return;
    const int row = (int)blockIdx.y * kWaves + (int)(threadIdx.x >> 6), f = t.f0 + row;
    if (row >= p.tile_rows || f >= t.nflat) return;
    int c0, c1;
    tile_chunks(p, t, t.f0, p.tile_rows, &c0, &c1);
    const int per = split_size(p, c1 - c0);
    if (c1 - c0 <= per) return;
    const int n = (c1 - c0 + per - 1) / per;
    const Writer<D, T> write{p, t, -1};
    const int64_t part = write.lse_row(f);
    const int col = 4 * (lane % COLS), par = lane / COLS;

    // the splits' scalars, one per lane (no more than 64 splits)
    float m = -__builtin_inff(), l = 0.0f;
    if (lane < n) {
        m = p.ws_ml[2 * (part + lane * p.ws_rows)];
        l = p.ws_ml[2 * (part + lane * p.ws_rows) + 1];
    }
    float top = m;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, d));
    const float w = m == top ? 1.0f : __builtin_amdgcn_exp2f(m - top);
    l *= w;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    const float* src = p.ws_o + part * D + col;
    for (int s0 = 0; s0 < n; s0 += BATCH * PAR) {
        f32x4 x[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int s = min(s0 + u * PAR + par, n - 1);
            x[u] = *reinterpret_cast<const f32x4*>(src + s * p.ws_rows * D);
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int s = s0 + u * PAR + par;
            const float ws = __shfl(w, s & 63);
            if (s < n) acc += x[u] * ws;
        }
    }
#pragma unroll
    for (int d = COLS; d < 64; d <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], d);
    if (lane == 0) write.scalars(f, top, l);
    if (par == 0) write.out(f, col, acc * write.factor(l));
}

template <int D>
hipError_t launch(const CacheFwdParams& p, bool fp32, hipStream_t stream)
{
    const dim3 grid((unsigned)(p.batch * p.pool.hkv) * (unsigned)p.row_tiles,
                    (unsigned)((p.tile_rows + kWaves - 1) / kWaves));
    if (fp32) hipLaunchKernelGGL((cache_combine_kernel<D, float>), grid, dim3(NT), 0, stream, p);
    else hipLaunchKernelGGL((cache_combine_kernel<D, __bf16>), grid, dim3(NT), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_combine(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream)
{
    return kind.head_dim == 128 ? launch<128>(p, kind.fp32, stream) : launch<64>(p, kind.fp32, stream);
}

}  // namespace attn
