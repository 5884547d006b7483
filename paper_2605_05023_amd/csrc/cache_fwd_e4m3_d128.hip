// cache_fwd_e4m3_d128.hip -- attention to a block cache in e4m3, head dim 128.
#include "cache_launch.h"

namespace attn {

hipError_t launch_cache_fwd_e4m3_d128(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream)
{
    return launch_type<128, false>(p, kind, stream);
}

}  // namespace attn
