// Next tokens from logits: temperature, top-k, top-p, min-p, and the draw from a given
// uniform number.
//
// What is kept by top-k and top-p is a beginning of the order by falling logit (equal
// ones by rising index), so it is described by its last element: a logit, and the index
// up to which equal ones belong to it. A descent over the digits of the logit finds
// it: counts (or weights) of the elements that agree in the digits so far, by the
// next digit, summed from the largest digit down. The draw goes by index: sums of the
// kept weights of pieces of the row, a scan over the pieces, and the piece that the
// number falls into element by element.
//
// Weights are float64 exponentials as integers in units of 2^-s (aug.h): sums are exact, so
// they do not depend on the order in which threads come to add.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "aug.h"
#include "status.h"

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kPieces = 1024;       // at most, of a row
constexpr int kDigits = 256;

struct Rows {
  const void* logits;
  int64_t stride;
  int32_t vocab;
  int32_t fixed;             // s
  const float* uniform;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* tokens;
  float* probs;
};

// A logit as it counts: NaN is -infinity, -0 is 0.
__device__ __forceinline__ float clean(float x) { return fmaxf(x, -INFINITY) + 0.f; }

// Larger logits have larger keys.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

// exp((x - top) / temperature) for x <= top, off by a few 2^-52: 2^a = 2^n 2^f with |f| <= 1/2,
// and the Taylor series of e^(f ln 2) up to its twelfth power (the rest is below 2e-16).
struct Weight {
  double top, rate;          // rate: log2(e) / temperature
  float top_f;
  __device__ Weight(float t, float temperature) : top(t), rate(1.4426950408889634074 / static_cast<double>(temperature)), top_f(t) {}
  __device__ __forceinline__ double operator()(float x) const {
    if (x == top_f) return 1.0;              // infinite ones too
    const double a = fmax((static_cast<double>(x) - top) * rate, -200.0);
    const double n = __builtin_rint(a);
    const double z = (a - n) * 0.69314718055994530942;
    double e = 1.0 / 479001600.0;
    e = fma(e, z, 1.0 / 39916800.0);
    e = fma(e, z, 1.0 / 3628800.0);
    e = fma(e, z, 1.0 / 362880.0);
    e = fma(e, z, 1.0 / 40320.0);
    e = fma(e, z, 1.0 / 5040.0);
    e = fma(e, z, 1.0 / 720.0);
    e = fma(e, z, 1.0 / 120.0);
    e = fma(e, z, 1.0 / 24.0);
    e = fma(e, z, 1.0 / 6.0);
    e = fma(e, z, 0.5);
    e = fma(e, z, 1.0);
    e = fma(e, z, 1.0);
    return ldexp(e, static_cast<int>(n));
  }
};

// w * 2^s rounded to an integer: adding 2^52 leaves it in the mantissa.
__device__ __forceinline__ uint64_t fixed_of(double w, double unit) {
  return static_cast<uint64_t>(__double_as_longlong(fma(w, unit, 0x1p52))) & 0xFFFFFFFFFFFFFull;
}

// One row, read in pieces of whole 16-byte words (the first and last may be parts of one).
// Position p of the row's words is element p - shift.
template <bool F32>
struct Reader {
  static constexpr int VEC = F32 ? 4 : 8;
  static constexpr int STEP = 64 * VEC;      // elements of a wave's load
  const char* words;
  int shift, vocab, steps, pieces;           // steps of a piece
  __device__ Reader(const Rows& a, int64_t row) {
    const char* p = static_cast<const char*>(a.logits) + row * a.stride * (F32 ? 4 : 2);
    shift = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15) / (F32 ? 4 : 2);
    words = p - (reinterpret_cast<uintptr_t>(p) & 15);
    vocab = a.vocab;
    steps = ((vocab + shift + STEP - 1) / STEP + kPieces - 1) / kPieces;
    pieces = (vocab + shift + steps * STEP - 1) / (steps * STEP);
  }
  // the lane's elements of one step; what is none is -infinity
  __device__ __forceinline__ void load(int piece, int step, int lane, float (&x)[VEC], int* index) const {
    const int p = (piece * steps + step) * STEP + lane * VEC;
    *index = p - shift;
    if (p >= shift && p + VEC <= shift + vocab) {
      const uint4 w = *reinterpret_cast<const uint4*>(words + static_cast<int64_t>(p) * (F32 ? 4 : 2));
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
          x[i] = clean(__uint_as_float(u[i]));
        } else {
          x[2 * i] = clean(__uint_as_float(u[i] << 16));
          x[2 * i + 1] = clean(__uint_as_float(u[i] & 0xFFFF0000u));
        }
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      x[i] = -INFINITY;
      if (p + i < shift || p + i >= shift + vocab) continue;
      if constexpr (F32) x[i] = clean(reinterpret_cast<const float*>(words)[p + i]);
      else x[i] = clean(__uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(words)[p + i]) << 16));
    }
  }
};

template <typename T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
template <typename T>
__device__ __forceinline__ T wave_upto(T v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}

typedef unsigned long long u64;

struct Lds {
  u64 mass[kPieces];                 // digits' weights, then pieces' sums
  uint32_t count[kPieces];           // digits' counts, then pieces' counts
  u64 waves[kWaves];
  float top[kWaves];
  int index[kWaves];
  u64 found_before;
  int found;
  int tie;
};

// Over n values in the order of the threads (at most one each), the first at which their sum
// exceeds `target`: its number and the sum before it, for every thread; n where none does.
__device__ __forceinline__ int find_over(u64 v, int n, u64 target, Lds& s, u64* before) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const u64 upto = wave_upto(tid < n ? v : 0ull);
  __syncthreads();
  if (lane == 63) s.waves[wave] = upto;
  if (tid == 0) s.found = n;
  __syncthreads();
  u64 at = upto;
  for (int w = 0; w < wave; ++w) at += s.waves[w];
  if (tid < n && at > target && at - v <= target) {
    s.found = tid;
    s.found_before = at - v;
  }
  __syncthreads();
  *before = s.found_before;
  return s.found;
}

// The last element of a beginning of the order.
struct Cut {
  uint32_t key;          // elements above it are in
  uint32_t equal;        // and this many of those with it, lowest indices first
  u64 taken;             // elements of the beginning
  bool all_equal;        // all of those with it
};

// The shortest beginning with at least `target` elements (BY_MASS: weight) that are there.
template <bool F32, bool BY_MASS>
__device__ Cut descend(const Reader<F32>& in, const Weight& weight, double unit, u64 target, uint32_t from_key, Lds& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t prefix = 0;
  u64 above = 0, above_count = 0;     // of elements above the digits so far
  uint32_t equal = 0;
  for (int level = 0; level < 4; ++level) {
    const int low = 24 - 8 * level;
    __syncthreads();
    if (tid < kDigits) {
      s.mass[tid] = 0;
      s.count[tid] = 0;
    }
    __syncthreads();
    for (int piece = wave; piece < in.pieces; piece += kWaves)
      for (int step = 0; step < in.steps; ++step) {
        float x[Reader<F32>::VEC];
        int index;
        in.load(piece, step, lane, x, &index);
#pragma unroll
        for (int i = 0; i < Reader<F32>::VEC; ++i) {
          if (index + i < 0 || index + i >= in.vocab) continue;
          const uint32_t key = key_of(x[i]);
          if ((level > 0 && (key ^ prefix) >> (low + 8)) || key < from_key) continue;
          const int digit = (key >> low) & (kDigits - 1);
          atomicAdd(&s.count[digit], 1u);
          if constexpr (BY_MASS) atomicAdd(&s.mass[digit], static_cast<u64>(fixed_of(weight(x[i]), unit)));
        }
      }
    __syncthreads();
    // digits from the largest down: the first at which the sum reaches the target
    const int digit = kDigits - 1 - tid;
    const u64 n = tid < kDigits ? s.count[digit] : 0;
    const u64 v = BY_MASS && tid < kDigits ? s.mass[digit] : n;
    u64 before;
    const int at = find_over(v, kDigits, target - above - 1, s, &before);
    const u64 count_upto = wave_upto(n);
    __syncthreads();
    if (lane == 63) s.waves[wave] = count_upto;
    __syncthreads();
    if (tid == at) {
      u64 c = count_upto - n;
      for (int w = 0; w < wave; ++w) c += s.waves[w];
      s.found_before = c;
      s.index[0] = static_cast<int>(n);
    }
    __syncthreads();
    above += before;
    above_count += s.found_before;
    equal = static_cast<uint32_t>(s.index[0]);
    prefix |= static_cast<uint32_t>(kDigits - 1 - at) << low;
    __syncthreads();
  }
  Cut c;
  c.key = prefix;
  u64 need = target - above;
  if constexpr (BY_MASS) {
    const uint32_t b = prefix >> 31 ? prefix ^ 0x80000000u : ~prefix;
    const u64 each = fixed_of(weight(__uint_as_float(b)), unit);
    need = (need + each - 1) / each;
  }
  c.equal = static_cast<uint32_t>(need);
  c.taken = above_count + need;
  c.all_equal = need >= equal;
  return c;
}

template <bool F32>
__global__ __launch_bounds__(kThreads) void sample_kernel(Rows a) {
  __shared__ Lds s;
  constexpr int VEC = Reader<F32>::VEC;
  const int row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Reader<F32> in(a, row);
  const float temperature = a.temperature ? a.temperature[row] : 1.f;
  const int k = a.top_k ? a.top_k[row] : 0;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  const float min_p = a.min_p ? a.min_p[row] : 0.f;
  const double uniform = a.uniform[row];

  // the largest logit, the first of equal ones
  float top = -INFINITY;
  int at = INT32_MAX;
  for (int piece = wave; piece < in.pieces; piece += kWaves)
    for (int step = 0; step < in.steps; ++step) {
      float x[VEC];
      int index;
      in.load(piece, step, lane, x, &index);
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (x[i] > top) {
          top = x[i];
          at = index + i;
        }
    }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    const float o = __shfl_xor(top, d);
    const int oa = __shfl_xor(at, d);
    if (o > top || (o == top && oa < at)) {
      top = o;
      at = oa;
    }
  }
  if (lane == 0) {
    s.top[wave] = top;
    s.index[wave] = at;
  }
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    const float o = s.top[w];
    const int oa = s.index[w];
    if (o > top || (o == top && oa < at)) {
      top = o;
      at = oa;
    }
  }
  if (top == -INFINITY || !(temperature > 0.f) || k == 1 || p <= 0.f) {
    if (tid == 0) {
      a.tokens[row] = top == -INFINITY ? -1 : at;
      if (a.probs) a.probs[row] = top == -INFINITY ? 0.f : 1.f;
    }
    return;
  }

  const Weight weight(top, temperature);
  const double unit = ldexp(1.0, a.fixed);
  Cut cut{0u, 0u, ~0ull, true};
  if (k > 0 && k < in.vocab) cut = descend<F32, false>(in, weight, unit, static_cast<u64>(k), 0u, s);
  int tie = INT32_MAX;                    // the last index of those with the cut's logit
  // Sums over what is kept, by piece; with `ties`, counts of the elements at the cut.
  const auto keeps = [&](float x, int index) {
    const uint32_t key = key_of(x);
    return key > cut.key || (key == cut.key && index <= tie);
  };
  const auto resolve_ties = [&]() {
    tie = INT32_MAX;
    if (cut.all_equal) return;
    for (int piece = wave; piece < in.pieces; piece += kWaves) {
      uint32_t n = 0;
      for (int step = 0; step < in.steps; ++step) {
        float x[VEC];
        int index;
        in.load(piece, step, lane, x, &index);
#pragma unroll
        for (int i = 0; i < VEC; ++i) n += index + i >= 0 && index + i < in.vocab && key_of(x[i]) == cut.key;
      }
      n = wave_sum(n);
      if (lane == 0) s.count[piece] = n;
    }
    __syncthreads();
    u64 before;
    const int piece = find_over(tid < in.pieces ? s.count[tid] : 0u, in.pieces, cut.equal - 1, s, &before);
    if (wave == 0) {
      u64 seen = before;
      for (int step = 0; step < in.steps; ++step) {
        float x[VEC];
        int index;
        in.load(piece, step, lane, x, &index);
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) n += index + i >= 0 && index + i < in.vocab && key_of(x[i]) == cut.key;
        const uint32_t upto = wave_upto(n);
        u64 c = seen + upto - n;
#pragma unroll
        for (int i = 0; i < VEC; ++i)
          if (index + i >= 0 && index + i < in.vocab && key_of(x[i]) == cut.key && ++c == cut.equal) s.tie = index + i;
        seen += __shfl(upto, 63);
      }
    }
    __syncthreads();
    tie = s.tie;
  };
  const auto sums = [&](bool floor) {
    for (int piece = wave; piece < in.pieces; piece += kWaves) {
      u64 v = 0;
      for (int step = 0; step < in.steps; ++step) {
        float x[VEC];
        int index;
        in.load(piece, step, lane, x, &index);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if (!keeps(x[i], index + i)) continue;
          const double w = weight(x[i]);
          if (floor && min_p > 0.f && w < fmin(static_cast<double>(min_p), 1.0)) continue;
          v += fixed_of(w, unit);
        }
      }
      v = wave_sum(v);
      if (lane == 0) s.mass[piece] = v;
    }
    __syncthreads();
  };
  const auto total = [&]() {
    u64 v = wave_sum(tid < in.pieces ? s.mass[tid] : 0ull);
    __syncthreads();
    if (lane == 0) s.waves[wave] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < kWaves; ++w) v += s.waves[w];
    return v;
  };
  resolve_ties();
  if (p < 1.f) {
    sums(false);
    const u64 all = total();
    const double want = ceil(static_cast<double>(p) * static_cast<double>(all));
    u64 target = static_cast<u64>(want);
    target = target < 1 ? 1 : target > all ? all : target;
    const Cut by = descend<F32, true>(in, weight, unit, target, cut.key, s);
    if (by.taken < cut.taken) {
      cut = by;
      resolve_ties();
    }
  }
  sums(true);
  const u64 all = total();
  const double share = uniform * static_cast<double>(all);
  u64 target = share > 0.0 ? static_cast<u64>(share) : 0ull;
  if (target >= all) target = all - 1;
  u64 before;
  const int piece = find_over(tid < in.pieces ? s.mass[tid] : 0ull, in.pieces, target, s, &before);
  if (wave != 0) return;
  for (int step = 0; step < in.steps; ++step) {
    float x[VEC];
    int index;
    in.load(piece, step, lane, x, &index);
    u64 v[VEC], sum = 0;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      v[i] = 0;
      if (!keeps(x[i], index + i)) continue;
      const double w = weight(x[i]);
      if (!(min_p > 0.f && w < fmin(static_cast<double>(min_p), 1.0))) v[i] = fixed_of(w, unit);
      sum += v[i];
    }
    const u64 upto = wave_upto(sum);
    u64 c = before + upto - sum;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      if (c <= target && c + v[i] > target) {
        a.tokens[row] = index + i;
        if (a.probs) a.probs[row] = static_cast<float>(weight(x[i]) * unit / static_cast<double>(all));
      }
      c += v[i];
    }
    before += __shfl(upto, 63);
  }
}

}  // namespace

extern "C" aug_status aug_sample(const aug_sample_args* g, void* stream) {
  const char* who = "aug_sample";
  if (!g) return aug::fail(AUG_ERR_INVALID, "%s: arguments are NULL", who);
  if (g->reserved != 0) return aug::fail(AUG_ERR_INVALID, "%s: the reserved field must be zero", who);
  if (g->dtype != AUG_F32 && g->dtype != AUG_BF16) return aug::fail(AUG_ERR_INVALID, "%s: logits of dtype %d", who, g->dtype);
  if (g->rows < 0 || g->vocab < 1 || g->stride < g->vocab || g->stride > (int64_t{1} << 40))
    return aug::fail(AUG_ERR_INVALID, "%s: %d rows of %d logits, %lld apart", who, g->rows, g->vocab, (long long)g->stride);
  if (g->vocab > (1 << 20)) return aug::fail(AUG_ERR_UNSUPPORTED, "%s: a vocabulary of %d (supported: %d)", who, g->vocab, 1 << 20);
  if (g->rows == 0) return AUG_OK;
  if (!g->logits || !g->uniform || !g->tokens) return aug::fail(AUG_ERR_INVALID, "%s: NULL device pointer", who);
  if (reinterpret_cast<uintptr_t>(g->logits) & (g->dtype == AUG_F32 ? 3 : 1))
    return aug::fail(AUG_ERR_INVALID, "%s: logits must be aligned to their elements", who);
  int bits = 0;
  while ((1 << bits) < g->vocab) ++bits;
  const Rows a{g->logits, g->stride, g->vocab, 62 - bits < 51 ? 62 - bits : 51, g->uniform, g->temperature, g->top_k, g->top_p,
               g->min_p, g->tokens, g->probs};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (g->dtype == AUG_F32) hipLaunchKernelGGL((sample_kernel<true>), dim3(g->rows), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((sample_kernel<false>), dim3(g->rows), dim3(kThreads), 0, st, a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess)
    return aug::fail(AUG_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return AUG_OK;
}
