// Rotary positions: rows of queries and keys rotated, and new K/V rows rotated into
// slots of the paged cache.
//
// A lane takes an octet, eight neighbouring dims of one head: 16 lanes make a head of
// 128 dims and a wave four of them (eight of 64). All heads of a row turn by the same
// angles, so a wave works on one row (or a share of its heads) and makes the eight
// cosines and sines of its octet once: the angle in turns as a product in float64,
// of which rounding to the nearest quarter turn leaves at most an eighth, exactly enough
// for any position; then the Taylor series of sine and cosine up to a^9 and a^10 at
// |a| <= pi / 4 (off by less than 2e-9) in float32. The octet that an octet is paired with (half a rotary_dim
// away; an interleaved octet has its pairs within) is read by its own lane too, out of
// the same cache lines.
//
// fp8 caches share a scale per block, so there one wave takes all rows of a block, which
// follow one another in the call, for one KV head and K or V, as the append of a planned
// batch does. A wave looks for the blocks that begin among `window` rows: one where rows are
// few, 16 where they are many (a wave a row, of which 15 of 16 end at once: 143 us below).
//
// HBM-bound: rows in, rows and cache out. Two groups of heads have their loads on their
// way at once, which leaves four waves a SIMD beside the fp8 part (four groups: 10 us more
// below; rows and blocks in launches of their own, as much together). 8115 rows of 64/8
// heads of 128 into an fp8 cache: 98 us, 316 MB; the rows alone take 57 us and the blocks 33,
// as much instructions (angles, quotients, codes) as traffic; into a 4-bit cache 68 us, a bf16 one 75.
// 4004 rows of 8 + 2 fp32 heads in and out: 10 us.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "aug.h"
#include "cache_codes.h"
#include "checks.h"
#include "plan_format.h"
#include "status.h"

namespace {

using aug::kBlock;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// One of q, k, v: rows in, and where they go.
struct Rows {
  const char* in;
  char* out;               // rows, or the cache
  int64_t in_stride;       // bytes between rows
  int64_t out_stride;
  int32_t heads;
};

struct RopeArgs {
  Rows q, k, v;
  float* scale[2];         // of K and V (fp8)
  const int32_t* positions;
  const int64_t* slots;
  const int32_t* live_rows;   // how many of `rows` there are, NULL: all
  int64_t num_slots;       // of the pool
  int32_t rows;
  int32_t shares;          // waves that share a row's heads
  int32_t window;          // rows whose blocks a wave writes (fp8)
  int32_t rotary_dim;      // 0: nothing is rotated
  int32_t interleaved;
  float magnitude;
  double turns[64];
};

struct Octet { float x[8]; };

// An octet as it is in a row.
template <bool F32> struct Raw { uint4 w[F32 ? 2 : 1]; };
template <bool F32>
__device__ __forceinline__ Raw<F32> load_raw(const char* p) {
  Raw<F32> r;
  r.w[0] = reinterpret_cast<const uint4*>(p)[0];
  if constexpr (F32) r.w[1] = reinterpret_cast<const uint4*>(p)[1];
  return r;
}
template <bool F32>
__device__ __forceinline__ Octet octet_of(const Raw<F32>& r) {
  const uint4 w = r.w[0];
  if constexpr (F32) {
    const uint4 z = r.w[1];
    return Octet{{__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w), __uint_as_float(z.x),
                  __uint_as_float(z.y), __uint_as_float(z.z), __uint_as_float(z.w)}};
  }
  return Octet{{aug::bf16_lo(w.x), aug::bf16_hi(w.x), aug::bf16_lo(w.y), aug::bf16_hi(w.y), aug::bf16_lo(w.z),
                aug::bf16_hi(w.z), aug::bf16_lo(w.w), aug::bf16_hi(w.w)}};
}

// Rows are rounded to their type here, once.
template <bool F32>
__device__ __forceinline__ void store_octet(char* p, const Octet& o) {
  if constexpr (F32) {
    reinterpret_cast<float4*>(p)[0] = float4{o.x[0], o.x[1], o.x[2], o.x[3]};
    reinterpret_cast<float4*>(p)[1] = float4{o.x[4], o.x[5], o.x[6], o.x[7]};
  } else {
    *reinterpret_cast<uint4*>(p) = uint4{aug::bf16_pair(o.x[0], o.x[1]), aug::bf16_pair(o.x[2], o.x[3]),
                                         aug::bf16_pair(o.x[4], o.x[5]), aug::bf16_pair(o.x[6], o.x[7])};
  }
}

// The angles of an octet: cosine and sine for each of its dims, and which octet its
// partners stand in (0: its own).
struct Angles {
  float c[8], s[8];
  int partner;             // in octets
  bool turn;
};

__device__ __forceinline__ void sin_cos_turns(double t, float* s, float* c) {
  const double quarter = __builtin_rint(4.0 * t);
  const float a = static_cast<float>((t - 0.25 * quarter) * 6.283185307179586476925286766559);
  const float z = a * a;
  const float sn = a * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  // quarters modulo 4, of up to 2^42 of them
  const int k = static_cast<int>(quarter - 4.0 * __builtin_floor(0.25 * quarter));
  const float u = k & 1 ? cs : sn, w = k & 1 ? sn : cs;
  *s = k & 2 ? -u : u;
  *c = (k + 1) & 2 ? -w : w;
}

__device__ __forceinline__ int partner_of(const RopeArgs& a, int octet) {
  const int half = a.rotary_dim / 16;              // octets
  return a.interleaved || octet >= 2 * half ? 0 : octet >= half ? -half : half;
}

__device__ __forceinline__ Angles angles_of(const RopeArgs& a, int position, int octet) {
  Angles g;
  g.turn = 8 * octet < a.rotary_dim;
  g.partner = partner_of(a, octet);
  if (!g.turn) return g;
  const double pos = position;
  if (a.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float s, c;
      sin_cos_turns(pos * a.turns[4 * octet + i], &s, &c);
      g.c[2 * i] = g.c[2 * i + 1] = c * a.magnitude;
      g.s[2 * i] = -s * a.magnitude;
      g.s[2 * i + 1] = s * a.magnitude;
    }
  } else {
    const int half = a.rotary_dim / 16;            // octets
    const bool second = octet >= half;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float s, c;
      sin_cos_turns(pos * a.turns[8 * (second ? octet - half : octet) + i], &s, &c);
      g.c[i] = c * a.magnitude;
      g.s[i] = (second ? s : -s) * a.magnitude;
    }
  }
  return g;
}

// An octet turned; `y` is the one it is paired with, or itself.
template <bool F32>
__device__ __forceinline__ Octet turned(const Angles& g, bool turn, const Raw<F32>& x, const Raw<F32>& y) {
  Octet o = octet_of<F32>(x);
  if (!g.turn || !turn) return o;
  Octet other = octet_of<F32>(y);
  if (g.partner == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) other.x[i] = o.x[i ^ 1];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) o.x[i] = fmaf(o.x[i], g.c[i], other.x[i] * g.s[i]);
  return o;
}

// KV: the cache's format, or -1 for rows out.
template <int KV, int D, bool F32>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  constexpr int OCTETS = D / 8;              // lanes of a head
  constexpr int HEADS = 64 / OCTETS;         // of a wave at a time
  constexpr int EB = F32 ? 4 : 2;
  constexpr int U = 2;
  const int lane = threadIdx.x & 63;
  const int octet = lane % OCTETS, sub = lane / OCTETS;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row_units = static_cast<int64_t>(a.rows) * a.shares;
  const int rows = a.live_rows ? min(max(*a.live_rows, 0), a.rows) : a.rows;
  const Angles still{{}, {}, 0, false};

  if (unit < row_units) {
    const int row = static_cast<int>(unit / a.shares), share = static_cast<int>(unit % a.shares);
    if (row >= rows) return;
    const Angles g = a.rotary_dim ? angles_of(a, a.positions[row], octet) : still;
    const int nq = (a.q.heads + HEADS - 1) / HEADS, nk = (a.k.heads + HEADS - 1) / HEADS;
    const int nv = (a.v.heads + HEADS - 1) / HEADS;
    // groups of heads: q's, k's, v's (fp8 caches: q's alone)
    const int groups = KV == AUG_FP8_E4M3FN ? nq : nq + nk + nv;
    int64_t block = 0;
    int t = 0;
    bool ok = false;
    if constexpr (KV >= 0) {
      const int64_t slot = a.slots[row];
      ok = static_cast<uint64_t>(slot) < static_cast<uint64_t>(a.num_slots);
      block = slot / kBlock;
      t = static_cast<int>(slot % kBlock);
    }
    // the loads of U groups, then their stores: a group's own loads are before its stores, also in place
    for (int first = share; first < groups; first += U * a.shares) {
      Raw<F32> x[U], y[U];
      const auto of = [&](int u, bool& is_q, bool& is_v, int& head) -> const Rows& {
        const int i = first + u * a.shares;
        is_q = i < nq;
        is_v = i >= nq + nk;
        const Rows& r = is_q ? a.q : is_v ? a.v : a.k;
        head = i < groups ? (i - (is_q ? 0 : is_v ? nq + nk : nq)) * HEADS + sub : r.heads;
        return r;
      };
#pragma unroll
      for (int u = 0; u < U; ++u) {
        bool is_q, is_v;
        int head;
        const Rows& r = of(u, is_q, is_v, head);
        if (head >= r.heads) continue;
        const char* p = r.in + row * r.in_stride + (static_cast<int64_t>(head) * D + 8 * octet) * EB;
        x[u] = load_raw<F32>(p);
        y[u] = x[u];
        if (g.partner != 0 && !is_v) y[u] = load_raw<F32>(p + g.partner * (8 * EB));
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        bool is_q, is_v;
        int head;
        const Rows& r = of(u, is_q, is_v, head);
        if (head >= r.heads) continue;
        const Octet o = turned<F32>(g, !is_v, x[u], y[u]);
        if (is_q || KV < 0) {
          store_octet<F32>(r.out + row * r.out_stride + (static_cast<int64_t>(head) * D + 8 * octet) * EB, o);
        } else if (ok) {
          if constexpr (KV == AUG_MXFP4)
            aug::store_fp4_octet(r.out + block * r.heads * aug::kMxCell, r.heads, head, is_v, t, octet, o.x);
          else if constexpr (KV >= 0)
            store_octet<F32>(r.out + (((block * r.heads + head) * kBlock + t) * D + 8 * octet) * EB, o);
        }
      }
    }
    return;
  }

  if constexpr (KV == AUG_FP8_E4M3FN) {
    const int64_t u = unit - row_units;
    const int hkv = a.k.heads, windows = (rows + a.window - 1) / a.window;
    if (u >= static_cast<int64_t>(windows) * hkv * 2) return;
    const int row0 = static_cast<int>(u / (2 * hkv)) * a.window;
    const int head = static_cast<int>((u >> 1) % hkv);
    const bool is_v = u & 1;
    const auto in_pool = [&](int64_t x) { return static_cast<uint64_t>(x) < static_cast<uint64_t>(a.num_slots); };
    const int64_t mine = lane < a.window && row0 + lane < rows ? a.slots[row0 + lane] : -1;
    uint64_t live = __ballot(in_pool(mine));
    if (live == 0) return;
    // the block of the last row before these that goes anywhere: rows of it here are written with that one
    int64_t done = -1;
    for (int at = row0 - 1; at >= 0; at -= 64) {
      const int64_t x = at - lane >= 0 ? a.slots[at - lane] : -1;
      const uint64_t some = __ballot(in_pool(x));
      if (some == 0) continue;
      done = __shfl(static_cast<long long>(x / kBlock), __ffsll(static_cast<unsigned long long>(some)) - 1);
      break;
    }
    for (; live; live &= live - 1) {
      const int nth = __ffsll(static_cast<unsigned long long>(live)) - 1, row = row0 + nth;
      const int64_t block = __shfl(static_cast<long long>(mine / kBlock), nth);
      if (block == done) continue;
      done = block;
      // the rows of the block: lane t has one more than how far behind `row` that of slot t is
      int behind = 0;
      for (int at = row; at < rows; at += 64) {
        const int64_t x = at + lane < rows ? a.slots[at + lane] : -1;
        const uint64_t here = __ballot(in_pool(x) && x / kBlock == block), others = __ballot(in_pool(x) && x / kBlock != block);
        const uint64_t take = others ? here & ((others & -others) - 1) : here;      // up to the first of another block
        int found = 0;
        if ((take >> lane) & 1) found = at - row + lane + 1;
        found = __builtin_amdgcn_ds_permute(4 * ((take >> lane) & 1 ? static_cast<int>(x % kBlock) : lane < 16 ? 63 : lane), found);
        if (lane < kBlock && found) behind = found;
        if (others) break;
      }
      const uint32_t tokens = static_cast<uint32_t>(__ballot(behind > 0));
      const Rows& r = is_v ? a.v : a.k;
      constexpr int PASSES = kBlock / HEADS;
      const bool turn = a.rotary_dim && !is_v;
      Raw<F32> x[PASSES], y[PASSES];
      int position[PASSES];
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int from = __shfl(behind, sub + p * HEADS);
        x[p] = y[p] = Raw<F32>{};
        position[p] = 0;
        if (from) {
          const int64_t i = static_cast<int64_t>(row) + from - 1;
          const char* src = r.in + i * r.in_stride + (static_cast<int64_t>(head) * D + 8 * octet) * EB;
          x[p] = load_raw<F32>(src);
          if (turn) {
            position[p] = a.positions[i];
            y[p] = load_raw<F32>(src + partner_of(a, octet) * (8 * EB));
          }
        }
      }
      Octet o[PASSES];
#pragma unroll
      for (int p = 0; p < PASSES; ++p) o[p] = turn ? turned<F32>(angles_of(a, position[p], octet), true, x[p], y[p]) : octet_of<F32>(x[p]);
      const int64_t cell = block * hkv + head;
      aug::store_fp8_tokens(reinterpret_cast<uint8_t*>(r.out) + cell * kBlock * D, a.scale[is_v] + cell, tokens, lane,
                            [&](int p, int e) { return o[p].x[e]; });
    }
  }
}

// A buffer of rows: its pointer, its stride in elements, and the least it can be.
aug_status check_rows(const char* who, const char* name, const void* p, int64_t stride, int64_t least, int eb) {
  if (!p) return aug::fail(AUG_ERR_INVALID, "%s: %s is NULL", who, name);
  if ((reinterpret_cast<uintptr_t>(p) & 15) || (stride * eb) % 16)
    return aug::fail(AUG_ERR_INVALID, "%s: %s and its rows must be 16-byte aligned", who, name);
  if (stride < least || stride > (int64_t{1} << 40))
    return aug::fail(AUG_ERR_INVALID, "%s: rows of %s %lld elements apart (at least %lld)", who, name, (long long)stride,
                     (long long)least);
  return AUG_OK;
}

aug_status check_rope(const char* who, const aug_attn_shape* s, const aug_rope* rope, const int32_t* positions, RopeArgs* a) {
  if (!rope) return aug::fail(AUG_ERR_INVALID, "%s: rope is NULL", who);
  if (rope->rotary_dim < 16 || rope->rotary_dim > 128 || rope->rotary_dim % 16 || (rope->interleaved & ~1) || rope->reserved)
    return aug::fail(AUG_ERR_INVALID, "%s: rope is not one that aug_rope_init made", who);
  if (rope->rotary_dim > s->head_dim)
    return aug::fail(AUG_ERR_UNSUPPORTED, "%s: rotary_dim %d of heads of %d", who, rope->rotary_dim, s->head_dim);
  if (!positions) return aug::fail(AUG_ERR_INVALID, "%s: positions are NULL", who);
  a->rotary_dim = rope->rotary_dim;
  a->interleaved = rope->interleaved;
  a->magnitude = rope->magnitude;
  for (int i = 0; i < 64; ++i) a->turns[i] = rope->turns[i];
  a->positions = positions;
  return AUG_OK;
}

// Waves that share a row: enough of them to fill the card with few rows, one where
// there are many, so that a row's angles are made once.
int shares_of(int64_t rows, int groups) {
  const int64_t fill = 4096 / (rows > 0 ? rows : 1);
  return static_cast<int>(fill < 1 ? 1 : fill > groups ? groups : fill);
}

template <int KV>
aug_status launch(const char* who, const aug_attn_shape* s, RopeArgs& a, void* stream) {
  const int heads = 64 / (s->head_dim / 8);
  const auto groups_of = [&](const Rows& r) { return (r.heads + heads - 1) / heads; };
  const int groups = KV == AUG_FP8_E4M3FN ? groups_of(a.q) : groups_of(a.q) + groups_of(a.k) + groups_of(a.v);
  a.shares = groups ? shares_of(a.rows, groups) : 0;
  int64_t units = static_cast<int64_t>(a.rows) * a.shares;
  if (KV == AUG_FP8_E4M3FN) {
    const int64_t most = static_cast<int64_t>(a.rows) * a.k.heads * 2 / 8192;
    a.window = static_cast<int>(most < 1 ? 1 : most > kBlock ? kBlock : most);
    units += static_cast<int64_t>((a.rows + a.window - 1) / a.window) * a.k.heads * 2;
  }
  const int64_t grid = (units + kWaves - 1) / kWaves;
  if (grid > INT32_MAX) return aug::fail(AUG_ERR_UNSUPPORTED, "%s: %lld units", who, (long long)units);
  hipStream_t st = static_cast<hipStream_t>(stream);
#define AUG_ROPE(K, D, F32) hipLaunchKernelGGL((rope_kernel<K, D, F32>), dim3(grid), dim3(kThreads), 0, st, a)
  if constexpr (KV == AUG_MXFP4 || KV == AUG_FP8_E4M3FN) {
    AUG_ROPE(KV, 128, false);
  } else {
    const bool f32 = s->kv_dtype == AUG_F32;
    if (f32 && s->head_dim == 64) AUG_ROPE(KV, 64, true);
    else if (f32) AUG_ROPE(KV, 128, true);
    else if (s->head_dim == 64) AUG_ROPE(KV, 64, false);
    else AUG_ROPE(KV, 128, false);
  }
#undef AUG_ROPE
  if (hipError_t e = hipGetLastError(); e != hipSuccess)
    return aug::fail(AUG_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return AUG_OK;
}

}  // namespace

extern "C" aug_status aug_rope_rows(const aug_attn_shape* s, const aug_rope* rope, const int32_t* positions, int32_t rows,
                                    const void* q, int64_t q_stride, const void* k, int64_t k_stride, void* q_out,
                                    int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* stream) {
  const char* who = "aug_rope_rows";
  if (aug_status st = aug::check_shape(s, who); st != AUG_OK) return st;
  if (rows < 0) return aug::fail(AUG_ERR_INVALID, "%s: %d rows", who, rows);
  if (rows == 0) return AUG_OK;
  RopeArgs a{};
  if (aug_status st = check_rope(who, s, rope, positions, &a); st != AUG_OK) return st;
  const int eb = s->q_dtype == AUG_F32 ? 4 : 2;
  if ((!q != !q_out) || (!k != !k_out) || (!q && !k)) return aug::fail(AUG_ERR_INVALID, "%s: rows without output, or the reverse", who);
  const auto take = [&](Rows& r, const char* name, const void* in, int64_t in_stride, void* out, int64_t out_stride, int heads) {
    if (!in) return AUG_OK;
    const int64_t least = static_cast<int64_t>(heads) * s->head_dim;
    if (aug_status st = check_rows(who, name, in, in_stride, least, eb); st != AUG_OK) return st;
    if (aug_status st = check_rows(who, name, out, out_stride, least, eb); st != AUG_OK) return st;
    if (in == out && in_stride != out_stride) return aug::fail(AUG_ERR_INVALID, "%s: %s in place with another stride", who, name);
    r = Rows{static_cast<const char*>(in), static_cast<char*>(out), in_stride * eb, out_stride * eb, heads};
    return AUG_OK;
  };
  if (aug_status st = take(a.q, "q", q, q_stride, q_out, q_out_stride, s->num_q_heads); st != AUG_OK) return st;
  if (aug_status st = take(a.k, "k", k, k_stride, k_out, k_out_stride, s->num_kv_heads); st != AUG_OK) return st;
  a.rows = rows;
  return launch<-1>(who, s, a, stream);
}

extern "C" aug_status aug_rope_append(const aug_attn_shape* s, const aug_rope* rope, const int32_t* positions,
                                      const int64_t* slots, int32_t rows, const int32_t* live_rows, const void* q,
                                      int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride,
                                      void* k_cache, void* v_cache, float* k_scale, float* v_scale, int32_t num_pool_blocks,
                                      void* stream) {
  const char* who = "aug_rope_append";
  if (aug_status st = aug::check_shape(s, who); st != AUG_OK) return st;
  if (rows < 0) return aug::fail(AUG_ERR_INVALID, "%s: %d rows", who, rows);
  if (num_pool_blocks < 1) return aug::fail(AUG_ERR_INVALID, "%s: empty pool", who);
  if (rows == 0) return AUG_OK;
  RopeArgs a{};
  if (rope) {
    if (aug_status st = check_rope(who, s, rope, positions, &a); st != AUG_OK) return st;
  } else if (positions || q || q_out) {
    return aug::fail(AUG_ERR_INVALID, "%s: positions or queries without a rope", who);
  }
  if (!q != !q_out) return aug::fail(AUG_ERR_INVALID, "%s: queries without output, or the reverse", who);
  if (!slots || !k_cache || !v_cache) return aug::fail(AUG_ERR_INVALID, "%s: NULL device pointer", who);
  const bool fp8 = s->kv_dtype == AUG_FP8_E4M3FN;
  if (fp8 && (!k_scale || !v_scale)) return aug::fail(AUG_ERR_INVALID, "%s: fp8 cache without scales", who);
  const auto bits = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if (((bits(k_cache) | bits(v_cache)) & 15) || (bits(slots) & 7) || (bits(live_rows) & 3))
    return aug::fail(AUG_ERR_INVALID, "%s: caches must be 16-byte aligned, slots 8-byte and live_rows 4-byte aligned", who);
  const int eb = s->q_dtype == AUG_F32 ? 4 : 2;
  const int64_t least = static_cast<int64_t>(s->num_kv_heads) * s->head_dim;
  if (q) {
    const int64_t least_q = static_cast<int64_t>(s->num_q_heads) * s->head_dim;
    if (aug_status st = check_rows(who, "q", q, q_stride, least_q, eb); st != AUG_OK) return st;
    if (aug_status st = check_rows(who, "q_out", q_out, q_out_stride, least_q, eb); st != AUG_OK) return st;
    if (q == q_out && q_stride != q_out_stride) return aug::fail(AUG_ERR_INVALID, "%s: q in place with another stride", who);
    a.q = Rows{static_cast<const char*>(q), static_cast<char*>(q_out), q_stride * eb, q_out_stride * eb, s->num_q_heads};
  }
  if (aug_status st = check_rows(who, "k", k, k_stride, least, eb); st != AUG_OK) return st;
  if (aug_status st = check_rows(who, "v", v, v_stride, least, eb); st != AUG_OK) return st;
  a.k = Rows{static_cast<const char*>(k), static_cast<char*>(k_cache), k_stride * eb, 0, s->num_kv_heads};
  a.v = Rows{static_cast<const char*>(v), static_cast<char*>(v_cache), v_stride * eb, 0, s->num_kv_heads};
  a.scale[0] = k_scale;
  a.scale[1] = v_scale;
  a.slots = slots;
  a.live_rows = live_rows;
  a.num_slots = static_cast<int64_t>(num_pool_blocks) * kBlock;
  a.rows = rows;
  if (fp8) return launch<AUG_FP8_E4M3FN>(who, s, a, stream);
  if (s->kv_dtype == AUG_MXFP4) return launch<AUG_MXFP4>(who, s, a, stream);
  return launch<AUG_BF16>(who, s, a, stream);
}
