// cache_launch.h -- the instantiations of cache_fwd_kernel for one head dim.
#pragma once

#include "cache_kernel.h"
#include "cache_many.h"

namespace attn {
namespace {

// 16-row tiles per wavefront of cache_many_kernel: the most that leave two
// wavefronts a SIMD their registers (the three terms of fp32 q take 3/4 of one's).
template <class T>
constexpr int kManyTiles = sizeof(T) == 2 ? 2 : 1;

template <int D, class T, bool E5M2, bool MODS>
hipError_t launch_rows(const CacheFwdParams& p, bool many, hipStream_t stream)
{
    const dim3 grid((unsigned)(p.batch * p.pool.hkv) * (unsigned)p.row_tiles, (unsigned)p.splits);
    if (many)
        hipLaunchKernelGGL((cache_many_kernel<D, T, E5M2, kManyTiles<T>, MODS>), grid, dim3(NT), 0, stream, p);
    else
        hipLaunchKernelGGL((cache_fwd_kernel<D, T, E5M2, 1, MODS>), grid, dim3(NT), 0, stream, p);
    return hipGetLastError();
}

template <int D, class T, bool E5M2>
hipError_t launch_mods(const CacheFwdParams& p, bool many, hipStream_t stream)
{
    return p.slopes || p.cap_post != 0.0f ? launch_rows<D, T, E5M2, true>(p, many, stream)
                                          : launch_rows<D, T, E5M2, false>(p, many, stream);
}

template <int D>
hipError_t launch_head_dim(const CacheFwdParams& p, const CacheFwdKind& k, hipStream_t stream)
{
    if (k.fp32)
        return k.e5m2 ? launch_mods<D, float, true>(p, k.many_rows, stream)
                      : launch_mods<D, float, false>(p, k.many_rows, stream);
    return k.e5m2 ? launch_mods<D, __bf16, true>(p, k.many_rows, stream)
                  : launch_mods<D, __bf16, false>(p, k.many_rows, stream);
}

}  // namespace
}  // namespace attn
