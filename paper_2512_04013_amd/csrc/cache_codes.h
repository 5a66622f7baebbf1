// How new K/V values are written down in the fp8 and 4-bit caches: shared by the
// append of a planned batch and the append by slots (device code).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "plan_format.h"

namespace aug {

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2_t{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}

// E4M3FN code -> float, exact: exponent field 0 holds multiples of 2^-9,
// otherwise (1 + m/8) * 2^(e - 7).
__device__ __forceinline__ float fp8_value(uint32_t c) {
  const uint32_t e = (c >> 3) & 15u, m = c & 7u;
  const float mag = e == 0 ? static_cast<float>(m) * 0x1p-9f
                           : __uint_as_float(((e + 120u) << 23) | (m << 20));
  return (c & 0x80u) ? -mag : mag;
}

// Four floats -> four E4M3FN codes: round to nearest, ties to an even mantissa
// (the conversion instruction's own rounding, subnormals included); every
// magnitude from 448 up, and NaN, saturates to +-448; the sign of zero is kept.
__device__ __forceinline__ uint32_t fp8_codes(const float* y) {
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = fabsf(y[e]) < 448.f ? y[e] : copysignf(448.f, y[e]);
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true));
}

// x / s for many x by one s > 0. `fast` (s within 2^+-60): the correctly rounded
// reciprocal and two exact remainders give the correctly rounded quotient; a
// remainder that underflows belongs to a quotient below 2^-40, whose code is 0
// either way. Otherwise the plain division. Bounded by instructions on large
// appends: 8192 rows on the 64/8-head layer, 8 KV heads of 128 (33.6 MB of new
// rows and 16.8 of codes), took 19.6 us with a division and a code in plain
// operations per element and the maximum by shuffles, and take 11.75 (4.3 TB/s);
// 256 decode rows 5.27 / 4.04.
struct Divide {
  float s, inv;
  bool fast;
  __device__ explicit Divide(float d) : s(d), inv(1.f / d), fast(d >= 0x1p-60f && d <= 0x1p60f) {}
  __device__ __forceinline__ float operator()(float x) const {
    if (!fast) return x / s;
    float q = x * inv;
    q = fmaf(fmaf(-q, s, x), inv, q);
    q = fmaf(fmaf(-q, s, x), inv, q);
    return copysignf(q, x);      // a NaN keeps its sign too
  }
};

// Largest value over the wave, uniform: rotations within rows of 16 lanes, then
// one lane of each row.
template <int CTRL>
__device__ __forceinline__ float max_with(float v) {
  const int o = __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true);
  return fmaxf(v, __int_as_float(o));
}
__device__ __forceinline__ float wave_max(float v) {
  v = max_with<0x121>(max_with<0x122>(max_with<0x124>(max_with<0x128>(v))));   // row_ror
  float m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16 * i));
  return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

// New tokens of one (block, KV head) of an fp8 cache, head_dim 128, by one wave: `slots`
// has a bit for each slot that receives one, and lane l holds eight dims from 8 (l % 16) of
// slots l / 16 + 4p as x(p, 0 .. 7), zeros where the slot receives none. With slot 0 the
// block begins anew. Else the scale grows with the new tokens, and when it does the
// codes of the other slots below the highest new one are re-encoded.
template <typename X>
__device__ __forceinline__ void store_fp8_tokens(uint8_t* blk, float* scale, uint32_t slots, int lane, X&& x) {
  constexpr int D = 128, LPR = D / 8, RPP = 64 / LPR;
  const int col = (lane % LPR) * 8;
  const int t0 = lane / LPR;
  const bool fresh = slots & 1u;
  const float s_old = fresh ? 0.f : *scale;
  float amax = 0.f;
#pragma unroll
  for (int p = 0; p < kBlock / RPP; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x(p, e)));
  amax = wave_max(amax);

  const float need = amax / 448.f;
  float s = need;
  if (!fresh) {
    if (need > s_old) {
      const Divide by(need);
      const int top = 31 - __clz(slots);
      for (int t = t0; t < top; t += RPP) {
        if ((slots >> t) & 1u) continue;
        uint2* q = reinterpret_cast<uint2*>(blk + t * D + col);
        const uint2 c = *q;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = by(fp8_value(((e < 4 ? c.x : c.y) >> (8 * (e & 3))) & 0xFFu) * s_old);
        *q = uint2{fp8_codes(v), fp8_codes(v + 4)};
      }
    } else {
      s = s_old;
    }
  }
  const Divide by(s);
#pragma unroll
  for (int p = 0; p < kBlock / RPP; ++p) {
    const int t = t0 + p * RPP;
    if (!((slots >> t) & 1u)) continue;
    uint2 c{0u, 0u};
    if (s != 0.f) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = by(x(p, e));
      c = uint2{fp8_codes(v), fp8_codes(v + 4)};
    }
    *reinterpret_cast<uint2*>(blk + t * D + col) = c;
  }
  if (lane == 0) *scale = s;
}

// Eight dims from 8 * oct of one token into `slot` of a 4-bit cell (block points at the
// block's bytes, head_dim 128). A group of 32 dims is a quad of lanes, all of which call
// this: its maximum is two quad permutations away. The scale is a power of two (from
// the maximum's exponent field, one higher from 1.75 * 2^k on, where the largest
// element would otherwise lose more than an eighth to saturation), so dividing
// by it is exact and the only rounding is the conversion's, to nearest even.
__device__ __forceinline__ void store_fp4_octet(char* block, int hkv, int head, bool is_v, int slot, int oct, const float* x) {
  float amax = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
  amax = max_with<0x4E>(max_with<0xB1>(amax));       // over the quad: lanes ^ 1, ^ 2
  const int field = static_cast<int>((__float_as_uint(amax) + (1u << 21)) >> 23);
  const int byte = min(max(field - 2, 2), 252);
  const float s = __uint_as_float(static_cast<uint32_t>(byte) << 23);
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
  char* codes = block + head * kMxCodes;
  char* scales = block + hkv * kMxCodes + head * kMxScales;
  const int group = oct >> 2;
  const int at = is_v ? 256 * (slot >> 2) + 16 * oct + 4 * (slot & 3) : 64 * slot + 4 * oct;
  *reinterpret_cast<uint32_t*>(codes + at) = c;
  if ((oct & 3) == 0) scales[is_v ? 16 * group + slot : 4 * slot + group] = static_cast<char>(byte);
}

}  // namespace aug
