// cache_launch.h -- the instantiations of the attention kernels for one head dim.
#pragma once

#include "cache_kernel.h"
#include "cache_many.h"

namespace attn {
namespace {

template <int D, class T, bool E5M2, int MODS>
hipError_t launch_rows(const CacheFwdParams& p, const CacheFwdKind& k, hipStream_t stream)
{
    // (the three terms of fp32 q leave registers for one row tile)
    constexpr int TWO = sizeof(T) == 2 ? 2 : 1;
    const dim3 grid((unsigned)(p.batch * p.pool.hkv) * (unsigned)p.row_tiles, (unsigned)p.splits);
    const dim3 block(64 * k.waves);
    if (k.many_rows && D == 128 && k.waves == 8)
        hipLaunchKernelGGL((cache_many_kernel<128, T, E5M2, TWO, MODS, 8>), grid, block, 0, stream, p);
    else if (k.many_rows)
        hipLaunchKernelGGL((cache_many_kernel<D, T, E5M2, TWO, MODS, 4>), grid, block, 0, stream, p);
    else if (k.waves == 8 && k.tiles == 1)
        hipLaunchKernelGGL((cache_fwd_kernel<D, T, E5M2, 1, MODS, 8>), grid, block, 0, stream, p);
    else if (k.waves == 8)
        hipLaunchKernelGGL((cache_fwd_kernel<D, T, E5M2, TWO, MODS, 8>), grid, block, 0, stream, p);
    else if (k.tiles == 1)
        hipLaunchKernelGGL((cache_fwd_kernel<D, T, E5M2, 1, MODS, 4>), grid, block, 0, stream, p);
    else
        hipLaunchKernelGGL((cache_fwd_kernel<D, T, E5M2, TWO, MODS, 4>), grid, block, 0, stream, p);
    return hipGetLastError();
}

template <int D, class T, bool E5M2>
hipError_t launch_mods(const CacheFwdParams& p, const CacheFwdKind& k, hipStream_t stream)
{
    if (p.softcap > 0.0f)
        return sizeof(T) == 2 && p.softcap <= kCapShortMax
                   ? launch_rows<D, T, E5M2, sizeof(T) == 2 ? kModsCapShort : kModsCapExact>(p, k, stream)
                   : launch_rows<D, T, E5M2, kModsCapExact>(p, k, stream);
    return p.slopes ? launch_rows<D, T, E5M2, kModsAlibi>(p, k, stream)
                    : launch_rows<D, T, E5M2, kModsNone>(p, k, stream);
}

template <int D, bool E5M2>
hipError_t launch_type(const CacheFwdParams& p, const CacheFwdKind& k, hipStream_t stream)
{
    return k.fp32 ? launch_mods<D, float, E5M2>(p, k, stream) : launch_mods<D, __bf16, E5M2>(p, k, stream);
}

}  // namespace
}  // namespace attn
