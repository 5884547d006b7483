// cache_fwd_e5m2_d128.hip -- attention to a block cache in e5m2, head dim 128.
#include "cache_launch.h"

namespace attn {

hipError_t launch_cache_fwd_e5m2_d128(const CacheFwdParams& p, const CacheFwdKind& kind, hipStream_t stream)
{
    return launch_type<128, true>(p, kind, stream);
}

}  // namespace attn
