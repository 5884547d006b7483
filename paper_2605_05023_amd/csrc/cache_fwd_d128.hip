// cache_fwd_d128.hip -- attention to the 8-bit block cache, head dim 128, and
// the dispatch over head dims.
#include "cache_launch.h"

namespace attn {

hipError_t launch_cache_fwd_d128(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream)
{
    return launch_head_dim<128>(p, kind, stream);
}

int cache_tile_rows(const CacheFwdKind& kind)
{
    return !kind.many_rows ? 16 : kWaves * 16 * (kind.fp32 ? kManyTiles<float> : kManyTiles<__bf16>);
}

hipError_t launch_cache_fwd(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream)
{
    return kind.head_dim == 128 ? launch_cache_fwd_d128(p, kind, stream)
                                : launch_cache_fwd_d64(p, kind, stream);
}

}  // namespace attn
