// The attention kernels with modified scores: tanh cap, bias by distance, and a
// span of keys for every row (attn_kernels.h, MOD). They are a translation unit
// of their own, and the plain kernels have none of their arguments.

#include <hip/hip_runtime.h>

#include "attn_kernels.h"

namespace aug {

aug_status attn_scored(const AttnCall& call, float softcap, const float* slopes) {
  ScoreArgs a{};
  fill_args(call, a);
  if (plan_has_spans(*call.info))
    a.row_span = reinterpret_cast<const int2*>(static_cast<const char*>(call.plan_dev) + spans_offset(*call.info));
  a.slopes = slopes;
  if (softcap > 0.f) {
    a.cap_in = 2.f / softcap;
    a.cap_out = -2.f * softcap * kLog2e;
  }
  return dispatch<true>(call, a);
}

}  // namespace aug
