// cache_fwd_e4m3_d64.hip -- attention to a block cache in e4m3, head dim 64.
#include "cache_launch.h"

namespace attn {

hipError_t launch_cache_fwd_e4m3_d64(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream)
{
    return launch_type<64, false>(p, kind, stream);
}

}  // namespace attn
