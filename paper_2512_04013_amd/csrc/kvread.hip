// Rows of the paged cache read back out in the format that the append takes:
// f32 and bf16 rows as they are, fp8 and 4-bit ones decoded to bf16.
//
// A lane makes 16 bytes of one output row (8 bf16 or 4 floats); lanes of a wave
// cover consecutive pieces of consecutive rows, so stores are whole lines. A
// row's slot is one 8-byte load, the same for the lanes of the row. HBM-bound:
// the cache row in, the decoded row out. 16 fp8 requests, 31k rows of 64/8 heads:
// 38.6 us, 5.0 TB/s in and out (a large copy reaches 4.8), 52.7 with one piece a lane.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "aug.h"
#include "checks.h"
#include "plan_format.h"
#include "status.h"

namespace {

using aug::kBlock;

constexpr int kThreads = 256;

struct ReadArgs {
  const char* cache[2];      // K, V
  const float* scale[2];
  char* out[2];
  const int64_t* slots;
  int64_t pieces;            // 16-byte pieces of each output
  int64_t num_slots;         // of the pool
  int32_t hkv;
};

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2_t{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}

// Pieces that a lane makes, a workgroup's width apart: their slots, then their
// cache words, are on their way together.
constexpr int kPieces = 4;

template <int KV, int D>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a) {
  constexpr int PPR = D * (KV == AUG_F32 ? 4 : 2) / 16;      // pieces of one row and head
  const int is_v = blockIdx.y;
  const char* cache = a.cache[is_v];
  const int64_t first = static_cast<int64_t>(blockIdx.x) * (kThreads * kPieces) + threadIdx.x;
  int64_t slot[kPieces];
  int kvh[kPieces];
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    const int64_t i = first + u * kThreads;
    slot[u] = -1;
    if (i < a.pieces) {
      const uint32_t head_row = static_cast<uint32_t>(i / PPR);     // below 2^31
      kvh[u] = static_cast<int>(head_row % a.hkv);
      slot[u] = a.slots[head_row / a.hkv];
    }
  }
  uint4 w[kPieces];
  float scale[kPieces];
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    w[u] = uint4{0u, 0u, 0u, 0u};
    scale[u] = 0.f;
    if (static_cast<uint64_t>(slot[u]) >= static_cast<uint64_t>(a.num_slots)) continue;
    const int64_t block = slot[u] / kBlock;
    const int t = static_cast<int>(slot[u] % kBlock);
    const int piece = static_cast<int>((first + u * kThreads) % PPR);
    if constexpr (KV == AUG_MXFP4) {
      const char* base = cache + block * a.hkv * aug::kMxCell;
      const char* codes = base + kvh[u] * aug::kMxCodes;
      const char* scales = base + a.hkv * aug::kMxCodes + kvh[u] * aug::kMxScales;
      codes += is_v ? 256 * (t >> 2) + 16 * piece + 4 * (t & 3) : 64 * t + 4 * piece;
      scales += is_v ? 4 * (piece & ~3) + t : 4 * t + (piece >> 2);      // group piece / 4
      w[u].x = *reinterpret_cast<const uint32_t*>(codes);
      scale[u] = __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint8_t*>(scales)) << 23);
    } else if constexpr (KV == AUG_FP8_E4M3FN) {
      const uint2 c = *reinterpret_cast<const uint2*>(cache + (((block * a.hkv + kvh[u]) * kBlock + t) * D + 8 * piece));
      w[u].x = c.x;
      w[u].y = c.y;
      scale[u] = a.scale[is_v][block * a.hkv + kvh[u]];
    } else {
      w[u] = *reinterpret_cast<const uint4*>(cache + ((((block * a.hkv + kvh[u]) * kBlock + t) * PPR + piece) << 4));
    }
  }
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    const int64_t i = first + u * kThreads;
    if (i >= a.pieces) return;
    uint4 o = w[u];
    const float s = scale[u];
    if constexpr (KV == AUG_MXFP4) {
      o = uint4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u].x, s, 0)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u].x, s, 1)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u].x, s, 2)),
                __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[u].x, s, 3))};
    } else if constexpr (KV == AUG_FP8_E4M3FN) {
      const auto p0 = __builtin_amdgcn_cvt_pk_f32_fp8(w[u].x, false), p1 = __builtin_amdgcn_cvt_pk_f32_fp8(w[u].x, true);
      const auto p2 = __builtin_amdgcn_cvt_pk_f32_fp8(w[u].y, false), p3 = __builtin_amdgcn_cvt_pk_f32_fp8(w[u].y, true);
      o = uint4{bf16_pair(p0[0] * s, p0[1] * s), bf16_pair(p1[0] * s, p1[1] * s), bf16_pair(p2[0] * s, p2[1] * s),
                bf16_pair(p3[0] * s, p3[1] * s)};
    }
    *reinterpret_cast<uint4*>(a.out[is_v] + (i << 4)) = o;
  }
}

}  // namespace

extern "C" aug_status aug_kv_read(const aug_attn_shape* s, const void* k_cache, const void* v_cache, const float* k_scale,
                                  const float* v_scale, const int64_t* slots, int64_t n, int32_t num_pool_blocks,
                                  void* k_out, void* v_out, void* stream) {
  const char* who = "aug_kv_read";
  if (aug_status st = aug::check_shape(s, who); st != AUG_OK) return st;
  if (n < 0) return aug::fail(AUG_ERR_INVALID, "%s: %lld rows", who, (long long)n);
  if (num_pool_blocks < 1) return aug::fail(AUG_ERR_INVALID, "%s: empty pool", who);
  if (n > INT32_MAX / s->num_kv_heads)
    return aug::fail(AUG_ERR_UNSUPPORTED, "%s: %lld rows of %d heads", who, (long long)n, s->num_kv_heads);
  if (n == 0) return AUG_OK;
  if (!k_cache || !v_cache || !slots || !k_out || !v_out) return aug::fail(AUG_ERR_INVALID, "%s: NULL device pointer", who);
  const bool fp8 = s->kv_dtype == AUG_FP8_E4M3FN;
  if (fp8 && (!k_scale || !v_scale)) return aug::fail(AUG_ERR_INVALID, "%s: fp8 cache without scales", who);
  const auto bits = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if (((bits(k_cache) | bits(v_cache) | bits(k_out) | bits(v_out)) & 15) || (bits(slots) & 7))
    return aug::fail(AUG_ERR_INVALID, "%s: caches and rows must be 16-byte aligned, slots 8-byte aligned", who);

  ReadArgs a{};
  a.cache[0] = static_cast<const char*>(k_cache);
  a.cache[1] = static_cast<const char*>(v_cache);
  a.scale[0] = k_scale;
  a.scale[1] = v_scale;
  a.out[0] = static_cast<char*>(k_out);
  a.out[1] = static_cast<char*>(v_out);
  a.slots = slots;
  a.pieces = n * s->num_kv_heads * (s->head_dim * (s->kv_dtype == AUG_F32 ? 4 : 2) / 16);
  a.num_slots = static_cast<int64_t>(num_pool_blocks) * kBlock;
  a.hkv = s->num_kv_heads;
  const dim3 grid(static_cast<uint32_t>((a.pieces + kThreads * kPieces - 1) / (kThreads * kPieces)), 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define AUG_READ(KV, D) hipLaunchKernelGGL((read_kernel<KV, D>), grid, dim3(kThreads), 0, st, a)
  if (s->kv_dtype == AUG_MXFP4) AUG_READ(AUG_MXFP4, 128);
  else if (fp8) AUG_READ(AUG_FP8_E4M3FN, 128);
  else if (s->kv_dtype == AUG_BF16 && s->head_dim == 64) AUG_READ(AUG_BF16, 64);
  else if (s->kv_dtype == AUG_BF16) AUG_READ(AUG_BF16, 128);
  else if (s->head_dim == 64) AUG_READ(AUG_F32, 64);
  else AUG_READ(AUG_F32, 128);
#undef AUG_READ
  if (hipError_t e = hipGetLastError(); e != hipSuccess)
    return aug::fail(AUG_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return AUG_OK;
}
