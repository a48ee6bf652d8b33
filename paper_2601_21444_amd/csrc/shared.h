// Device/host declarations of the attention behind shared prefixes (internal; the public ABI is include/apbv_shared.h).
#pragma once
#include "cache.h"
#include "shared_validation.h"

namespace apbv {

struct SharedParams {
  CacheAttnParams prefix, own;       // the groups over their prefixes, the requests over their own keys
};
apbv_status launch_shared_short(const SharedParams& p, const SharedPlan& plan, int head_dim, hipStream_t stream);      // shared_short.hip
apbv_status launch_shared_attention(const SharedParams& p, const SharedPlan& plan, int head_dim, hipStream_t stream);

}  // namespace apbv
