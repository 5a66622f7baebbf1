// One checked attention call, as the entry points hand it to the kernels'
// translation units.
#pragma once

#include <cstdint>

#include "aug.h"

namespace aug {

struct AttnCall {
  const aug_attn_shape* shape;
  const aug_attn_plan_info* info;
  void* plan_dev;
  const void* q;
  const void* k_cache;
  const void* v_cache;
  const float* k_scale;
  const float* v_scale;
  const int32_t* block_ids;
  int32_t num_pool_blocks;
  void* out;
  void* workspace;
  void* stream;
};

// The launch with modified scores (attn_scored.hip): softcap 0 for no cap,
// slopes NULL for no bias; a plan with row spans brings its mask.
aug_status attn_scored(const AttnCall& call, float softcap, const float* slopes);

}  // namespace aug
