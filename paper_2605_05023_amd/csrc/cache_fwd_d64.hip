// cache_fwd_d64.hip -- attention to the 8-bit block cache, head dim 64.
#include "cache_launch.h"

namespace attn {

hipError_t launch_cache_fwd_d64(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream)
{
    return launch_head_dim<64>(p, kind, stream);
}

}  // namespace attn
