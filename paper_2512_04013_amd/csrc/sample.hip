// Next tokens from logits: temperature, top-k, top-p, min-p, and the draw from a given
// uniform number.
//
// What is kept by top-k and top-p is a beginning of the order by falling logit (equal
// ones by rising index), so it is described by its last element, the cut: a logit, and
// the index up to which equal ones belong to it. The draw goes by index.
//
// Weights are float64 exponentials as integers in units of 2^-s (aug.h): sums are exact, so
// they do not depend on the order in which threads come to add.
//
// A workgroup of 1024 threads takes a row and reads it in every pass, from the caches after the
// first (held in registers it spilled). The cut lies near the top of the row, so few elements
// need more than a comparison:
//
//  * top-k: at least k elements are not below the k-th largest of the maxima of groups of
//    elements (four groups a thread), which bins over the distance from the row's
//    largest logit bound from below. What is not below that goes on a list, is sorted by (logit,
//    index) and cut by top-k, top-p and min-p, and the draw is made on sums of the list by index.
//  * top-p alone: weights of all elements, by bins over the distance. If all up to the cut's bin
//    fit on the list only those of that bin are sorted; else the list has the bin alone, and sums of
//    the kept weights of pieces of the row, a scan over the pieces, and the piece that the
//    number falls into element by element make the draw.
//  * what this does not hold (more elements at the cut than the list has places, infinite
//    logits) takes a descent over the digits of the logit instead: counts or weights of the
//    elements that agree in the digits so far, by the next digit.
//
// One row of 32000 bf16 logits with top-k 50 and top-p: 10 us, of which reading the row is a
// fifth and the rest barriers and LDS round trips one behind the other. 64 rows of 50257 fp32 with
// top-p alone: 31 to 47 us by the logits, the time of the longest row; 9 of them for the largest logit, 17 for
// weights and the draw, as rows with a temperature alone need them (26 us), the rest for the list. 512 rows of
// 128000 bf16 with every setting: 103 us, bound by rows without top-k and their weights (40 vector instructions
// each, on one compute unit; a temperature alone 100 us, the largest logits 41). Digit by digit, 64 rows of 50257 take
// from 126 us (a temperature of 2^41) to 497 (equal logits with top-p, whose sums meet in one bin).

#include <hip/hip_runtime.h>

#include <cstdint>
#include <utility>

#include "aug.h"
#include "checks.h"
#include "status.h"

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kDigits = 256;
constexpr int kBins = 2 * kThreads;
constexpr int kBinBits = 11;
constexpr int kList = 2 * kThreads;
// pieces of a row: what one wave reads at once, at most (2^20 + 3) / 4 words of fp32
constexpr int kPieces = ((1 << 20) / 4 / kThreads + 1) * kWaves;

typedef unsigned long long u64;

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

// f(0), f(1), ... f(N - 1) with constants: arrays stay in registers however much f is.
template <typename F, int... I>
__device__ __forceinline__ void times(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void times(F&& f) {
  times(f, std::make_integer_sequence<int, N>{});
}

// Larger logits have larger keys; -0 has the key of 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
// Place in the order: earlier elements have larger ones. No element has 0.
__device__ __forceinline__ u64 place_of(float x, int index) {
  return (static_cast<u64>(key_of(x)) << 32) | static_cast<uint32_t>(~index);
}
__device__ __forceinline__ float logit_at(u64 place) {
  const uint32_t key = static_cast<uint32_t>(place >> 32);
  return __uint_as_float(key >> 31 ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ int index_at(u64 place) { return static_cast<int>(~static_cast<uint32_t>(place)); }

// exp((x - top) / temperature) for x <= top, off by less than 2^-51 (the largest weight is 1): with
// a = (x - top) log2(e) / temperature and m = 32 a rounded, 2^a = 2^(m >> 5) 2^((m & 31) / 32) 2^f with
// |f| <= 1 / 64, from a table of 2^(j / 32) and the Taylor series of e^(f ln 2) up to its sixth power. That
// one (2^-48.7 at most) is economized: with t = 64 f and Chebyshev's T6, t^6 is (48 t^4 - 18 t^2 + 1 + T6(t)) / 32,
// so all but 2^-52.7 of it goes into the coefficients of the fourth power and the second, for no
// instruction. Adding 1.5 * 2^52 rounds to an integer and leaves it in the low word. The table is
// 256 bytes of LDS, every bank once, so that its reads never wait for one another (128
// entries, with a shorter series, took twice as long), and -m is the element's bin below.
constexpr int kPowers = 32;
struct Weight {
  static constexpr double kRound = 6755399441055744.0;         // 1.5 * 2^52
  double top, rate;          // rate: log2(e) / temperature
  double unit;               // 2^s
  const u64* powers;         // LDS: 2^(j / 32), as bits
  int fixed_bits;            // s
  __device__ __forceinline__ Weight(float t, float temperature, int s, const u64* table)
      : top(t), rate(1.4426950408889634074 / static_cast<double>(temperature)), unit(ldexp(1.0, s)), powers(table), fixed_bits(s) {}
  // what is below 2^-100, -infinity and NaN count as that
  __device__ __forceinline__ double power_of(float x) const { return fmax((static_cast<double>(x) - top) * rate, -100.0); }
  // e^(f ln 2) and the bits of 2^(m / 32) times 2^up
  __device__ __forceinline__ double split(double a, int up, double* power, int* m) const {
    const double r = fma(a, 32.0, kRound);
    const double f = fma(r - kRound, -1.0 / 32.0, a);
    *m = static_cast<int>(__double_as_longlong(r));
    const u64 p = powers[*m & (kPowers - 1)];
    const int hi = static_cast<int>(p >> 32) + (((*m >> 5) + up) << 20);
    *power = __longlong_as_double(static_cast<long long>((static_cast<u64>(static_cast<uint32_t>(hi)) << 32) | static_cast<uint32_t>(p)));
    constexpr double c = 0.69314718055994530942, sixth = c * c * c * c * c * c / 720.0;
    double e = fma(f, c * c * c * c * c / 120.0, c * c * c * c / 24.0 + sixth * (48.0 / 32.0 / (64.0 * 64.0)));
    e = fma(e, f, c * c * c / 6.0);
    e = fma(e, f, c * c / 2.0 - sixth * (18.0 / 32.0 / (64.0 * 64.0 * 64.0 * 64.0)));
    e = fma(e, f, c);
    return fma(e, f, 1.0);
  }
  __device__ __forceinline__ double operator()(float x) const {
    double p;
    int m;
    const double e = split(power_of(x), 0, &p, &m);
    return e * p;
  }
  // In units of 2^-s: adding 2^52 leaves the rounded integer in the mantissa. *m: 32 times the
  // logarithm, rounded.
  __device__ __forceinline__ u64 fixed(float x, int* m) const {
    double p;
    const double e = split(power_of(x), fixed_bits, &p, m);
    return static_cast<u64>(__double_as_longlong(fma(e, p, 0x1p52))) & 0xFFFFFFFFFFFFFull;
  }
  __device__ __forceinline__ u64 fixed(float x) const {
    int m;
    return fixed(x, &m);
  }
  // the same, 0 below `floor`
  __device__ __forceinline__ u64 fixed_from(float x, u64 floor) const {
    const u64 v = fixed(x);
    return v < floor ? 0ull : v;
  }
  // the distance from the top in bins of 1 / 32 of a power
  __device__ __forceinline__ int bin(float x) const {
    return -static_cast<int>(__double_as_longlong(fma(power_of(x), 32.0, kRound)));
  }
  // a logit that none of bins 0 .. bin is below
  __device__ __forceinline__ float low(int bin) const {
    const double x = top - (bin + 0.51) / 32.0 / rate;
    return static_cast<float>(x - fabs(x) * 0x1p-22);
  }
};

// The largest of three, NaN where one of them is, quiet or signalling (v_maximum3_f32). v_max3_f32 will not
// do: it makes a quiet NaN of a signalling one, and the next passes over that and over all that was gathered before.
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(a, __builtin_elementwise_maximum(b, c));
}

// A row in 16-byte words, of which the first and last may be parts of one: thread t takes
// words t, t + kThreads, ... What is no element is -infinity; NaN stays, and is below everything
// in comparisons. Every pass reads the row, from the caches after the first.
template <bool F32>
struct Row {
  static constexpr int VEC = F32 ? 4 : 8;
  static constexpr uint32_t kNone = F32 ? 0xFF800000u : 0xFF80FF80u;
  const char* words;
  int shift, vocab, count, turns;         // element = position in the words - shift

  __device__ __forceinline__ Row(const Rows& a, int64_t row) {
    const char* p = static_cast<const char*>(a.logits) + row * a.stride * (F32 ? 4 : 2);
    shift = static_cast<int>(reinterpret_cast<uintptr_t>(p) & 15) / (F32 ? 4 : 2);
    words = p - (reinterpret_cast<uintptr_t>(p) & 15);
    vocab = a.vocab;
    count = (vocab + shift + VEC - 1) / VEC;
    turns = (count + kThreads - 1) / kThreads;
  }
  __device__ __forceinline__ int first(int w) const { return w * VEC - shift; }
  __device__ __forceinline__ uint4 word(int w) const {
    if (w * VEC >= shift && w * VEC + VEC <= shift + vocab) return *reinterpret_cast<const uint4*>(words + static_cast<int64_t>(w) * 16);
    // parts of it are no elements
    uint32_t u[4] = {kNone, kNone, kNone, kNone};
    times<VEC>([&](auto i) {
      const int p = w * VEC + i;
      if (p < shift || p >= shift + vocab) return;
      if constexpr (F32) {
        u[i] = reinterpret_cast<const uint32_t*>(words)[p];
      } else {
        const uint32_t h = reinterpret_cast<const uint16_t*>(words)[p];
        u[i / 2] = i & 1 ? (u[i / 2] & 0xFFFFu) | (h << 16) : (u[i / 2] & 0xFFFF0000u) | h;
      }
    });
    return uint4{u[0], u[1], u[2], u[3]};
  }
  __device__ static __forceinline__ void values(const uint4& w, float (&x)[VEC]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    times<4>([&](auto i) {
      if constexpr (F32) {
        x[i] = __uint_as_float(u[i]);
      } else {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
      }
    });
  }
  // NaN if `top` or an element is
  __device__ static __forceinline__ float largest(const uint4& w, float top) {
    float x[VEC];
    values(w, x);
    times<VEC / 2>([&](auto i) { top = max3(top, x[2 * i], x[2 * i + 1]); });
    return top;
  }
  // f(turn, word, part) of every word of the thread, four at a time, so that their loads are
  // on their way together; part is the word's number modulo four.
  template <typename F>
  __device__ __forceinline__ void by_words(F&& f) const {
    const int t = threadIdx.x;
    int turn = 0;
#pragma nounroll
    for (; turn + 5 < turns; turn += 4) {           // (not the last one, which may hold the row's end)
      uint4 u[4];
      times<4>([&](auto i) {
        const int w = (turn + i) * kThreads + t;
        u[i] = i == 0 && w == 0 ? word(0) : *reinterpret_cast<const uint4*>(words + static_cast<int64_t>(w) * 16);
      });
      times<4>([&](auto i) { f(turn + i, u[i], i); });
    }
#pragma nounroll
    for (; turn < turns; turn += 2) {
      const uint4 a = word(turn * kThreads + t), b = word((turn + 1) * kThreads + t);
      f(turn, a, std::integral_constant<int, 1>{});
      f(turn + 1, b, std::integral_constant<int, 2>{});
    }
  }
  // f(index, value) of the thread's elements from `low` up
  template <typename F>
  __device__ __forceinline__ void from(float low, F&& f) const {
    by_words([&](int turn, const uint4& u, auto) {
      if (!__any(!(largest(u, -INFINITY) < low))) return;      // (words with NaN are looked through)
      float x[VEC];
      values(u, x);
      const int index = first(turn * kThreads + static_cast<int>(threadIdx.x));
      times<VEC>([&](auto i) {
        if (x[i] >= low) f(index + i, x[i]);
      });
    });
  }
  // f(index, value) of all elements, and what is none, one by one, and end(turn) behind every word:
  // a loop of little code, for passes that do much for each
  template <typename F, typename E>
  __device__ __forceinline__ void each(F&& f, E&& end) const {
    uint4 next = word(threadIdx.x);
#pragma nounroll
    for (int turn = 0; turn < turns; ++turn) {
      uint4 u = next;
      next = word((turn + 1) * kThreads + threadIdx.x);
      int index = first(turn * kThreads + static_cast<int>(threadIdx.x));
#pragma nounroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t v = u.x;
        u = uint4{u.y, u.z, u.w, 0u};
        if constexpr (F32) {
          f(index++, __uint_as_float(v));
        } else {
          f(index++, __uint_as_float(v << 16));
          f(index++, __uint_as_float(v & 0xFFFF0000u));
        }
      }
      end(turn);
    }
  }
  // the largest of each of four groups of the thread's elements
  __device__ __forceinline__ void maxima(float (&top)[4]) const {
    times<4>([&](auto g) { top[g] = -INFINITY; });
    by_words([&](int, const uint4& u, auto part) { top[part] = largest(u, top[part]); });
    if (top[0] != top[0] || top[1] != top[1] || top[2] != top[2] || top[3] != top[3]) {
      // NaN: all in one group, one by one (64 rows of 50257 with fifty each: 17 us, without 13)
      float t = -INFINITY;
#pragma nounroll
      for (int turn = 0; turn < turns; ++turn) {
        float x[VEC];
        values(word(turn * kThreads + threadIdx.x), x);
        times<VEC>([&](auto i) {
          if (x[i] > t) t = x[i];
        });
      }
      top[0] = t;
      top[1] = top[2] = top[3] = -INFINITY;
    }
  }
  __device__ __forceinline__ bool is_element(int index) const { return index >= 0 && index < vocab; }
};

// ---- sums over lanes, waves and the workgroup ---------------------------------------------

template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp_add(u64 v) {
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(v >> 32), CTRL, ROWS, 0xF, false);
  return v + ((static_cast<u64>(hi) << 32) | lo);
}
// over the 16 lanes of a row up to this one, then over the wave
__device__ __forceinline__ u64 row_upto(u64 v) {
  return dpp_add<0x118, 0xF>(dpp_add<0x114, 0xF>(dpp_add<0x112, 0xF>(dpp_add<0x111, 0xF>(v))));   // row_shr 1, 2, 4, 8
}
__device__ __forceinline__ u64 wave_upto(u64 v) {
  return dpp_add<0x143, 0xC>(dpp_add<0x142, 0xA>(row_upto(v)));                                     // row_bcast 15, 31
}
__device__ __forceinline__ u64 lane_of(u64 v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), lane), hi = __builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane);
  return (static_cast<u64>(hi) << 32) | lo;
}
__device__ __forceinline__ u64 wave_sum(u64 v) { return lane_of(wave_upto(v), 63); }

struct Lds {
  u64 mass[kBins];                   // of bins or digits
  u64 list[kList];
  u64 piece[kPieces];                // sums of the pieces: 16 a turn
  uint32_t count[kBins];
  u64 powers[kPowers];
  u64 waves[2][kWaves];
  float top[kWaves];
  int index[kWaves];
  u64 found_before, other_before;
  int found, tie, listed;
};

// Sum over this thread and those before it, and over all. One barrier: consecutive calls alternate
// between the two BUFs.
template <int BUF>
__device__ __forceinline__ u64 block_upto(u64 v, Lds& s, u64* total) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const u64 upto = wave_upto(v);
  if (lane == 63) s.waves[BUF][wave] = upto;
  __syncthreads();
  const u64 w = row_upto(s.waves[BUF][lane & (kWaves - 1)]);
  *total = lane_of(w, kWaves - 1);
  return upto + (wave ? lane_of(w, wave - 1) : 0ull);
}
// Sum over all threads.
template <int BUF>
__device__ __forceinline__ u64 block_sum(u64 v, Lds& s) {
  u64 total;
  block_upto<BUF>(v, s, &total);
  return total;
}
// The first thread at which the sum of v exceeds `target`, and the sum before it; -1 if none.
__device__ __forceinline__ int find_over(u64 v, u64 target, Lds& s, u64* before) {
  if (threadIdx.x == 0) s.found = -1;
  u64 total;
  const u64 upto = block_upto<0>(v, s, &total);
  if (upto > target && upto - v <= target) {
    s.found = threadIdx.x;
    s.found_before = upto - v;
  }
  __syncthreads();
  const int found = s.found;
  *before = s.found_before;
  __syncthreads();
  return found;
}
// The piece at which the sum of the pieces exceeds `target`, and the sum before it.
__device__ __forceinline__ int find_piece(int turns, u64 target, Lds& s, u64* before) {
  const int tid = threadIdx.x;
  u64 v = 0;
  if (tid < turns) {
    times<kWaves>([&](auto w) { v += s.piece[tid * kWaves + w]; });
  }
  const int turn = max(find_over(v, target, s, before), 0);
  int piece = turn * kWaves;
  for (; piece < turn * kWaves + kWaves - 1 && *before + s.piece[piece] <= target; ++piece) *before += s.piece[piece];
  return piece;
}
// A wave's sum becomes a piece's.
__device__ __forceinline__ void set_piece(int turn, u64 v, Lds& s) {
  if (__any(v != 0)) v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) s.piece[turn * kWaves + (threadIdx.x >> 6)] = v;
}
// p of a sum, rounded up: at least 1, at most all.
__device__ __forceinline__ u64 share_of(float p, u64 all) {
  const u64 t = static_cast<u64>(ceil(static_cast<double>(p) * static_cast<double>(all)));
  return t < 1 ? 1 : t > all ? all : t;
}
// The number that the draw goes by: the first sum above it wins.
__device__ __forceinline__ u64 draw_of(double uniform, u64 all) {
  const double share = uniform * static_cast<double>(all);
  const u64 t = share > 0.0 ? static_cast<u64>(share) : 0ull;
  return t >= all ? all - 1 : t;
}

// ---- the cut by digits -----------------------------------------------------------------------

// The end of the shortest beginning of the order with at least `target` elements (BY_MASS:
// weight), that are there, looking no further than `last`; *taken: its elements.
template <bool BY_MASS, typename R, typename A>
__device__ __forceinline__ u64 descend(const R& in, const A& as, const Weight& weight, u64 target, u64 last, Lds& s, u64* taken) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t from = static_cast<uint32_t>(last >> 32);
  uint32_t prefix = 0;
  u64 above = 0, above_count = 0, equal = 0;      // of elements above the digits so far
  for (int level = 0; level < 4; ++level) {
    const int low = 24 - 8 * level;
    __syncthreads();
    if (tid < kDigits) {
      s.mass[tid] = 0;
      s.count[tid] = 0;
    }
    __syncthreads();
    in.each([&](int index, float x) {
      x = as(x != x ? -INFINITY : x);
      const uint32_t key = key_of(x);
      if (!in.is_element(index) || (level > 0 && (key ^ prefix) >> (low + 8)) || key < from) return;
      const int digit = (key >> low) & (kDigits - 1);
      atomicAdd(&s.count[digit], 1u);
      if constexpr (BY_MASS) atomicAdd(&s.mass[digit], weight.fixed(x));
    }, [](int) {});
    __syncthreads();
    // digits from the largest down: the first at which the sum reaches the target
    const int digit = kDigits - 1 - tid;
    const u64 n = tid < kDigits ? s.count[digit] : 0;
    const u64 v = BY_MASS && tid < kDigits ? s.mass[digit] : n;
    u64 before, total;
    const int at = max(find_over(v, target - above - 1, s, &before), 0);
    const u64 upto = block_upto<1>(n, s, &total);
    if (tid == at) {
      s.other_before = upto - n;
      s.index[0] = static_cast<int>(n);
    }
    __syncthreads();
    above += before;
    above_count += s.other_before;
    equal = static_cast<u64>(s.index[0]);
    prefix |= static_cast<uint32_t>(kDigits - 1 - at) << low;
  }
  u64 need = target - above;                      // of the elements with that key
  if constexpr (BY_MASS) {
    const u64 each = weight.fixed(logit_at(static_cast<u64>(prefix) << 32));
    need = each ? (need + each - 1) / each : equal;
  }
  *taken = above_count + need;
  if (need >= equal) return static_cast<u64>(prefix) << 32;
  // the index of the last of them
  __syncthreads();
  u64 c = 0;
  const auto is_equal = [&](int index, float x) { return in.is_element(index) && key_of(as(x != x ? -INFINITY : x)) == prefix; };
  in.each([&](int index, float x) { c += is_equal(index, x); },
          [&](int turn) {
            set_piece(turn, c, s);
            c = 0;
          });
  __syncthreads();
  u64 before;
  const int piece = find_piece(in.turns, need - 1, s, &before);
  if (wave == 0) {
    const int w = piece * 64 + lane, index = in.first(w);
    float x[R::VEC];
    R::values(in.word(w), x);
    u64 n = 0;
    times<R::VEC>([&](auto i) { n += is_equal(index + i, x[i]); });
    u64 at = before + wave_upto(n) - n;
    times<R::VEC>([&](auto i) {
      if (is_equal(index + i, x[i]) && ++at == need) s.tie = index + i;
    });
  }
  __syncthreads();
  return (static_cast<u64>(prefix) << 32) | static_cast<uint32_t>(~s.tie);
}

// ---- the list ----------------------------------------------------------------------------------

// Of the list, thread t holds elements list_pos(0) and list_pos(1): a wave has 128 in a row, its
// lanes the first 64 and the second.
__device__ __forceinline__ int list_pos(int i) { return 128 * (threadIdx.x >> 6) + 64 * i + (threadIdx.x & 63); }

// The value of lane ^ MASK.
template <int MASK>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  const int x = static_cast<int>(v);
  if constexpr (MASK == 1) return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, true);         // quad_perm
  if constexpr (MASK == 2) return __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, true);
  if constexpr (MASK == 4)                                                     // lane ^ 7, then ^ 3
    return __builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, true), 0x1B, 0xF, 0xF, true);
  if constexpr (MASK == 8) return __builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, true);        // row_ror:8
  if constexpr (MASK == 16) {
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? a[0] : a[1];
  }
  if constexpr (MASK == 32) {
    const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? a[0] : a[1];
  }
}
// the larger of two, or the smaller
__device__ __forceinline__ u64 pick(u64 a, u64 b, bool larger) { return (a < b) == larger ? b : a; }

// The list of n elements (in registers: v, 0 behind the last) sorted, largest first: bitonic. Pairs
// up to 32 apart are lanes of a wave, 64 apart a lane's own two, and wider ones meet in s.list.
__device__ __forceinline__ void sort_list(int n, u64 (&v)[2], Lds& s) {
  const int pos[2] = {list_pos(0), list_pos(1)};
  int size = 256;
  while (size < n) size <<= 1;
  const bool mine = __builtin_amdgcn_readfirstlane(pos[0]) < size;     // other waves have nothing
  const auto lanes = [&](auto gap, int run) {
    if (gap * 2 > run) return;
    times<2>([&](auto e) {
      const u64 other = (static_cast<u64>(lane_xor<gap>(static_cast<uint32_t>(v[e] >> 32))) << 32) | lane_xor<gap>(static_cast<uint32_t>(v[e]));
      v[e] = pick(v[e], other, ((pos[e] & gap) == 0) == ((pos[e] & run) == 0));
    });
  };
#pragma nounroll
  for (int run = 2; run <= size; run <<= 1) {
#pragma nounroll
    for (int gap = run >> 1; gap >= 128; gap >>= 1) {
      __syncthreads();
      if (mine) times<2>([&](auto e) { s.list[pos[e]] = v[e]; });
      __syncthreads();
      if (mine) times<2>([&](auto e) { v[e] = pick(v[e], s.list[pos[e] ^ gap], ((pos[e] & gap) == 0) == ((pos[e] & run) == 0)); });
    }
    if (!mine) continue;
    if (run >= 128) {
      const bool down = (pos[0] & run) == 0;
      const u64 a = pick(v[0], v[1], down), b = pick(v[0], v[1], !down);
      v[0] = a;
      v[1] = b;
    }
    lanes(std::integral_constant<int, 32>{}, run);
    lanes(std::integral_constant<int, 16>{}, run);
    lanes(std::integral_constant<int, 8>{}, run);
    lanes(std::integral_constant<int, 4>{}, run);
    lanes(std::integral_constant<int, 2>{}, run);
    lanes(std::integral_constant<int, 1>{}, run);
  }
}

// Sums of a thread's two over the list up to each.
template <int BUF>
__device__ __forceinline__ void list_upto(u64 a, u64 b, Lds& s, u64 (&upto)[2], u64* all) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  upto[0] = wave_upto(a);
  upto[1] = wave_upto(b) + lane_of(upto[0], 63);
  if (lane == 63) s.waves[BUF][wave] = upto[1];
  __syncthreads();
  const u64 w = row_upto(s.waves[BUF][lane & (kWaves - 1)]);
  *all = lane_of(w, kWaves - 1);
  const u64 before = wave ? lane_of(w, wave - 1) : 0ull;
  upto[0] += before;
  upto[1] += before;
}

// What the cut is made by. `skip`: weight of elements before the list's first.
struct Cut {
  int k;                  // elements of the list that top-k leaves, at most
  u64 target;             // weight that top-p asks for, 0: p of what k leaves
  u64 skip;
  float p;
};

// The list sorted and cut: how many of its elements top-k and top-p keep. The thread's places and
// their weights come back.
__device__ __forceinline__ int cut_list(int n, const Cut& cut, const Weight& weight, Lds& s, u64 (&place)[2], u64 (&w)[2]) {
  times<2>([&](auto i) { place[i] = list_pos(i) < n ? s.list[list_pos(i)] : 0; });
  sort_list(n, place, s);
  times<2>([&](auto i) { w[i] = place[i] ? weight.fixed(logit_at(place[i])) : 0; });
  int keep = min(n, cut.k);
  if (cut.p < 1.f) {
    u64 v[2], upto[2], all;
    times<2>([&](auto i) { v[i] = list_pos(i) < keep ? w[i] : 0; });
    list_upto<1>(v[0], v[1], s, upto, &all);
    const u64 target = (cut.target ? cut.target : share_of(cut.p, all)) - cut.skip;
    // the first sum that reaches it
    if (threadIdx.x == 0) s.tie = keep;
    __syncthreads();
    times<2>([&](auto i) {
      if (upto[i] >= target && upto[i] - v[i] < target) s.tie = list_pos(i) + 1;
    });
    __syncthreads();
    keep = min(keep, s.tie);
  }
  return keep;
}

__device__ __forceinline__ void write_token(const Rows& a, int row, int index, float x, u64 all, const Weight& weight) {
  a.tokens[row] = index;
  if (a.probs) a.probs[row] = static_cast<float>(weight(x) * weight.unit / static_cast<double>(all));
}

// The draw among two elements of each thread, of which those with a weight v are kept: sums of
// the weights by the index's upper eleven bits, and then by its lower ones in the bin that the number falls
// into (a sort by index and a scan took three times as long).
__device__ __forceinline__ void draw_by_index(const Rows& a, int row, double uniform, const Weight& weight, Lds& s, const u64 (&place)[2],
                                              const u64 (&v)[2]) {
  const int t = threadIdx.x, bits = 32 - __clz(a.vocab), shift = max(bits - kBinBits, 0);
  const auto find = [&](auto part, auto bin_of, double share, u64 target, u64* before) {
    __syncthreads();
    s.mass[2 * t] = s.mass[2 * t + 1] = 0;
    __syncthreads();
    times<2>([&](auto i) {
      const int bin = bin_of(index_at(place[i]));
      if (v[i] && bin >= 0) atomicAdd(&s.mass[bin], v[i]);
    });
    __syncthreads();
    const u64 w0 = s.mass[2 * t], w1 = s.mass[2 * t + 1];
    u64 all;
    const u64 upto = block_upto<part>(w0 + w1, s, &all);
    if (part == 0) target = draw_of(share, all);
    if (upto > target && upto - w0 - w1 <= target) {
      const bool second = upto - w1 <= target;
      s.found = 2 * t + second;
      s.found_before = upto - w1 - (second ? 0 : w0);
    }
    __syncthreads();
    *before = s.found_before;
    return std::pair<u64, u64>{all, target};
  };
  u64 before;
  const auto [all, target] = find(std::integral_constant<int, 0>{}, [&](int index) { return index >> shift; }, uniform, 0, &before);
  int index = s.found;
  if (shift > 0) {
    const int upper = index;
    u64 unused;
    find(std::integral_constant<int, 1>{}, [&](int x) { return x >> shift == upper ? x & ((1 << shift) - 1) : -1; }, 0.0, target - before, &unused);
    index = (upper << shift) + s.found;
  }
  times<2>([&](auto i) {
    if (v[i] && index_at(place[i]) == index) write_token(a, row, index, logit_at(place[i]), all, weight);
  });
}

// A value of each lane, largest first: bitonic.
__device__ __forceinline__ u64 sort_wave(u64 v) {
  const int lane = threadIdx.x & 63;
  times<6>([&](auto r) {
    times<r + 1>([&](auto g) {
      constexpr int run = 2 << r, gap = run >> (g + 1);
      const u64 other = (static_cast<u64>(lane_xor<gap>(static_cast<uint32_t>(v >> 32))) << 32) | lane_xor<gap>(static_cast<uint32_t>(v));
      v = pick(v, other, ((lane & gap) == 0) == ((lane & run) == 0));
    });
  });
  return v;
}
// Cut and draw of a list of up to 64 elements by the first wave, with no barrier: sorted, cut, sorted by
// index. 32000 logits with top-k 50: 11.9 us with the way below, 10.2 with this one.
__device__ __forceinline__ void finish_wave(const Rows& a, int row, int n, const Cut& cut, u64 floor, double uniform, const Weight& weight, Lds& s) {
  const int lane = threadIdx.x;
  if (lane >= 64) return;
  const u64 place = sort_wave(lane < n ? s.list[lane] : 0);
  const float x = logit_at(place);
  const u64 w = place ? weight.fixed(x) : 0;
  int keep = min(n, cut.k);
  if (cut.p < 1.f) {
    const u64 v = lane < keep ? w : 0, upto = wave_upto(v);
    const u64 target = cut.target ? cut.target : share_of(cut.p, lane_of(upto, 63));
    const u64 reached = __ballot(upto >= target && upto - v < target);      // the first sum that reaches it
    if (reached) keep = min(keep, static_cast<int>(__ffsll(reached)));
  }
  // by rising index: ~index above the lane that has the weight
  const u64 by_index = sort_wave(lane < keep ? (place << 32) | static_cast<uint32_t>(lane) : 0);
  const int from = static_cast<int>(by_index & 63);
  const u64 kept = __shfl(lane < keep && w >= floor ? w : 0, from);
  const float logit = __shfl(x, from);
  const u64 v = lane < keep ? kept : 0, upto = wave_upto(v);
  const u64 all = lane_of(upto, 63), target = draw_of(uniform, all);
  if (upto > target && upto - v <= target) write_token(a, row, index_at(by_index >> 32), logit, all, weight);
}

// Cut and draw of a list of up to 128 elements without sorting it: eight threads an element
// count the elements before it in the order and add their weights, sixteen others each; then the
// same over those before it by index that are kept. Half the time of two sorts.
__device__ __forceinline__ void finish_short(const Rows& a, int row, int n, const Cut& cut, u64 floor, double uniform, const Weight& weight, Lds& s) {
  constexpr int kShort = 128, kParts = kThreads / kShort, kEach = kShort / kParts;
  const int t = threadIdx.x, e = t & (kShort - 1), part = t / kShort;
  u64* before = s.mass + kShort;          // weights before each, in the order, then by index
  const u64 mine = e < n ? s.list[e] : 0;
  const float x = logit_at(mine);
  const u64 w = mine ? weight.fixed(x) : 0;
  if (part == 0) {
    s.list[e] = mine;
    s.mass[e] = w;
    before[e] = before[kShort + e] = 0;
    s.count[e] = 0;
  }
  __syncthreads();
  uint32_t rank = 0;
  u64 sum = 0;
#pragma unroll 4
  for (int j = part * kEach; j < part * kEach + kEach; ++j) {
    const bool first = s.list[j] > mine;
    rank += first;
    sum += first ? s.mass[j] : 0;
  }
  if (mine) {
    atomicAdd(&s.count[e], rank);
    atomicAdd(&before[e], sum);
  }
  __syncthreads();
  rank = s.count[e];
  sum = before[e];
  int keep = min(n, cut.k);
  if (cut.p < 1.f) {
    u64 target = cut.target;
    if (!target) {
      if (part == 0 && mine && static_cast<int>(rank) == keep - 1) s.found_before = sum + w;
      __syncthreads();
      target = share_of(cut.p, s.found_before);
    }
    if (part == 0 && mine && sum < target && sum + w >= target) s.tie = static_cast<int>(rank) + 1;
    __syncthreads();
    keep = min(keep, s.tie);
  }
  const u64 v = static_cast<int>(rank) < keep && w >= floor ? w : 0;
  if (part == 0) s.mass[e] = v;
  __syncthreads();
  sum = 0;
  u64 all = 0;
  const uint32_t index = ~static_cast<uint32_t>(mine);
#pragma unroll 4
  for (int j = part * kEach; j < part * kEach + kEach; ++j) {
    const u64 o = s.mass[j];
    sum += ~static_cast<uint32_t>(s.list[j]) < index ? o : 0;
    all += o;
  }
  if (mine) atomicAdd(&before[kShort + e], sum);
  if (e == 0) s.waves[0][part] = all;
  __syncthreads();
  all = 0;
  times<kParts>([&](auto i) { all += s.waves[0][i]; });
  const u64 target = draw_of(uniform, all);
  sum = before[kShort + e];
  if (part == 0 && v && sum <= target && sum + v > target) write_token(a, row, static_cast<int>(index), x, all, weight);
}

// An element comes on the list; more than it holds are counted.
__device__ __forceinline__ void put(int index, float x, Lds& s) {
  const int at = atomicAdd(&s.listed, 1);
  if (at < kList) s.list[at] = place_of(x, index);
}
template <typename R>
__device__ __forceinline__ int list_from(const R& in, float low, Lds& s) {
  in.from(low, [&](int index, float x) { put(index, x, s); });
  __syncthreads();
  return s.listed;
}

// The list of n elements cut, and the draw from it.
__device__ __forceinline__ void finish_list(const Rows& a, int row, int n, const Cut& cut, u64 floor, double uniform, const Weight& weight,
                                            Lds& s) {
  if (n <= 64) {
    finish_wave(a, row, n, cut, floor, uniform, weight, s);
  } else if (n <= 128) {
    finish_short(a, row, n, cut, floor, uniform, weight, s);
  } else {
    u64 place[2], w[2];
    const int keep = cut_list(n, cut, weight, s, place, w);
    times<2>([&](auto i) { w[i] = list_pos(i) < keep && w[i] >= floor ? w[i] : 0; });
    draw_by_index(a, row, uniform, weight, s, place, w);
  }
}

// What became of a row in the fast ways.
enum class Fast { kNot, kDrawn, kPieces };     // nothing done; done; pieces summed, `last` the end of what is kept

template <typename R>
__device__ __forceinline__ Fast fast_draw(const Rows& a, int row, const R& in, const float (&maxima)[4], const Weight& weight, int k,
                                          float p, u64 floor, double uniform, Lds& s, u64* last) {
  const int tid = threadIdx.x;
  Cut cut{kList, 0, 0, p};
  if (in.vocab <= kList) {
    if (tid == 0) s.listed = 0;
    __syncthreads();
    const int n = list_from(in, -3.402823466e38f, s);
    if (k > 0) cut.k = k;
    finish_list(a, row, n, cut, floor, uniform, weight, s);
    return Fast::kDrawn;
  }
  if (k > 0) {
    if (k > kList) return Fast::kNot;
    cut.k = k;
    // What is 64 powers below the top is in the last bin. Of the groups' maxima, if they are more than twice k: with k of G of them at the cut there
    // are about -G ln(1 - k / G) elements above it, 1.4 k for half. Else, and where elements are not
    // spread over the groups, of all elements.
    for (int pass = 2 * k <= min(in.count, 4 * kThreads) && k <= kList * 2 / 3 ? 0 : 1; pass < 2; ++pass) {
      __syncthreads();
      s.count[tid] = s.count[tid + kThreads] = 0;
      if (tid == 0) s.listed = 0;
      __syncthreads();
      const auto count = [&](float x) {
        if (x > -INFINITY) atomicAdd(&s.count[min(weight.bin(x), kBins - 1)], 1u);
      };
      if (pass == 0) {
        times<4>([&](auto g) { count(maxima[g]); });
      } else {
        in.each([&](int, float x) { count(x); }, [](int) {});
      }
      __syncthreads();
      const uint32_t c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1];
      u64 before;
      const int pair = find_over(static_cast<u64>(c0) + c1, static_cast<u64>(k - 1), s, &before);
      if (pair < 0) continue;
      const int bin = before + s.count[2 * pair] >= static_cast<u64>(k) ? 2 * pair : 2 * pair + 1;
      if (bin == kBins - 1) continue;
      const int n = list_from(in, weight.low(bin), s);
      if (n > kList) continue;
      finish_list(a, row, n, cut, floor, uniform, weight, s);
      return Fast::kDrawn;
    }
    return Fast::kNot;
  }

  // top-p alone. Adding up by bins in LDS costs a tenth of the pass.
  for (int i = tid; i < kBins; i += kThreads) {
    s.mass[i] = 0;
    s.count[i] = 0;
  }
  if (tid == 0) s.listed = 0;
  __syncthreads();
  u64 below = 0;
  in.each([&](int, float x) {
    int m;
    const u64 w = weight.fixed(x, &m);
    if (-m < kBins) {
      atomicAdd(&s.count[-m], 1u);
      atomicAdd(&s.mass[-m], w);
    } else {
      below += w;
    }
  }, [](int) {});
  __syncthreads();
  const uint32_t c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1];
  const u64 w0 = s.mass[2 * tid], w1 = s.mass[2 * tid + 1];
  u64 in_bins, counted;
  const u64 upto = block_upto<0>(w0 + w1, s, &in_bins);
  cut.target = share_of(p, block_sum<1>(below, s) + in_bins);
  if (cut.target > in_bins) return Fast::kNot;
  const u64 count_upto = block_upto<0>(static_cast<u64>(c0) + c1, s, &counted);
  if (upto >= cut.target && upto - w0 - w1 < cut.target) {
    const bool second = upto - w1 < cut.target;
    s.found = 2 * tid + second;
    s.found_before = upto - w1 - (second ? 0 : w0);
    s.other_before = count_upto - c1 - (second ? 0 : c0);
  }
  __syncthreads();
  const int bin = s.found;
  const u64 count_before = s.other_before;
  cut.skip = s.found_before;
  const uint32_t in_bin = s.count[bin];
  if (count_before + in_bin <= kList) {
    // all up to the bin's end
    cut.skip = 0;
    const u64 before = s.found_before;
    if (tid == 0) s.tie = 0;
    __syncthreads();
    in.from(weight.low(bin), [&](int index, float x) {
      const int b = weight.bin(x);
      if (b > bin) return;
      put(index, x, s);
      if (b < bin) return;
      const int at = atomicAdd(&s.tie, 1);
      if (at < 64) s.piece[at] = place_of(x, index);
    });
    __syncthreads();
    const int n = min(s.listed, kList);
    if (n <= 64 || in_bin > 64) {
      finish_list(a, row, n, cut, floor, uniform, weight, s);
      return Fast::kDrawn;
    }
    // the cut lies in the bin: its elements alone are sorted, by the first wave
    if (tid < 64) {
      const u64 place = sort_wave(tid < static_cast<int>(in_bin) ? s.piece[tid] : 0);
      const u64 w = place ? weight.fixed(logit_at(place)) : 0, sum = before + wave_upto(w);
      const int first = __ffsll(__ballot(sum >= cut.target && place)) - 1;
      const u64 end = lane_of(place, first < 0 ? static_cast<int>(in_bin) - 1 : first);
      if (tid == 0) s.other_before = end;
    }
    __syncthreads();
    const u64 end = s.other_before;
    u64 place[2], w[2];
    times<2>([&](auto i) {
      place[i] = list_pos(i) < n ? s.list[list_pos(i)] : 0;
      w[i] = place[i] >= end ? weight.fixed_from(logit_at(place[i]), floor) : 0;
    });
    draw_by_index(a, row, uniform, weight, s, place, w);
    return Fast::kDrawn;
  }
  if (in_bin > kList) return Fast::kNot;
  // the bin alone, and sums of what is above it
  u64 v = 0;
  in.each([&](int index, float x) {
    int m;
    const u64 w = weight.fixed(x, &m);
    v += -m < bin && w >= floor ? w : 0;
    if (-m == bin) put(index, x, s);
  }, [&](int turn) {
    set_piece(turn, v, s);
    v = 0;
  });
  __syncthreads();
  u64 place[2], w[2];
  const int keep = cut_list(min(s.listed, kList), cut, weight, s, place, w);
  times<2>([&](auto i) {
    if (list_pos(i) < keep && w[i] >= floor)
      atomicAdd(&s.piece[(index_at(place[i]) + in.shift) / (64 * R::VEC)], w[i]);
  });
  times<2>([&](auto i) {
    if (list_pos(i) == keep - 1) s.found_before = place[i];
  });
  __syncthreads();
  *last = s.found_before;
  __syncthreads();
  return Fast::kPieces;
}

// The row of a workgroup. More rows than there are compute units start one after another, and those
// that compute something for every element (no top-k) take up to five times as long as the others: they
// go first (512 rows of 128000, a third of them such: 140 us in the order they come). Each thread looks at one
// row, so more than 1024 start as they come (1024 rows of 32000: 88 us, 1025: 93).
__device__ __forceinline__ int row_of_block(const Rows& a, Lds& s) {
  const int b = blockIdx.x, rows = gridDim.x;
  if (rows <= 256 || rows > kThreads || !a.top_k) return b;
  const int t = threadIdx.x;
  bool slow = false;
  if (t < rows) {
    const int k = a.top_k[t];
    slow = (k <= 0 || k >= a.vocab) && (!a.temperature || a.temperature[t] > 0.f);
  }
  u64 count;
  const u64 upto = block_upto<1>(slow, s, &count);
  const int place = static_cast<int>(slow ? upto - 1 : count + t - upto);
  if (t < rows && place == b) s.found = t;
  __syncthreads();
  return s.found;
}

template <bool F32>
__global__ __launch_bounds__(kThreads) void sample_kernel(Rows a) {
  __shared__ Lds s;
  typedef Row<F32> R;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = row_of_block(a, s);
  const float temperature = a.temperature ? a.temperature[row] : 1.f;
  int k = a.top_k ? a.top_k[row] : 0;
  float p = a.top_p ? a.top_p[row] : 1.f;
  if (!(p < 1.f)) p = 1.f;
  const float min_p = a.min_p ? a.min_p[row] : 0.f;
  const double uniform = a.uniform[row];
  const R in(a, row);

  if (tid < kPowers) s.powers[tid] = static_cast<u64>(__double_as_longlong(exp2(static_cast<double>(tid) / kPowers)));
  float maxima[4];
  in.maxima(maxima);
  float top = fmaxf(fmaxf(maxima[0], maxima[1]), fmaxf(maxima[2], maxima[3]));
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if (lane == 0) s.top[wave] = top;
  __syncthreads();
  times<kWaves>([&](auto w) { top = fmaxf(top, s.top[w]); });
  if (top == -INFINITY) {
    if (tid == 0) {
      a.tokens[row] = -1;
      if (a.probs) a.probs[row] = 0.f;
    }
    return;
  }
  if (!(temperature > 0.f) || k == 1 || p <= 0.f) {
    int at = INT32_MAX;
    in.from(top, [&](int index, float) { at = min(at, index); });
#pragma unroll
    for (int d = 32; d; d >>= 1) at = min(at, __shfl_xor(at, d));
    if (lane == 0) s.index[wave] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < kWaves; ++w) at = min(at, s.index[w]);
      a.tokens[row] = at;
      if (a.probs) a.probs[row] = 1.f;
    }
    return;
  }
  if (k <= 0 || k >= in.vocab) k = 0;
  // infinite logits share the weight, and the others have none
  const bool endless = top == INFINITY;
  if (endless) top = 1.f;
  const auto as = [endless](float x) { return !endless ? x : x == INFINITY ? 1.f : -INFINITY; };

  const Weight weight(top, temperature, a.fixed, s.powers);
  // min-p as the least weight (what rounds to it is kept)
  const u64 floor = min_p > 0.f ? static_cast<u64>(__builtin_rint(fmin(static_cast<double>(min_p), 1.0) * weight.unit)) : 0;
  u64 last = 0;                 // elements at or before this place are kept: all
  // sums of what is kept, by piece
  const auto sum_up = [&](const auto& r, u64 least) {
    __syncthreads();
    u64 v = 0;
    r.each([&](int index, float x) {
      x = as(x);
      if (last == 0 || place_of(x, index) >= last) v += weight.fixed_from(x, least);
    }, [&](int turn) {
      set_piece(turn, v, s);
      v = 0;
    });
    __syncthreads();
  };
  const auto total = [&]() {
    u64 v = 0;
    for (int i = tid; i < in.turns * kWaves; i += kThreads) v += s.piece[i];
    return block_sum<0>(v, s);
  };
  if (k == 0 && p >= 1.f) {
    sum_up(in, floor);
  } else {
    // (a rate that float32 does not hold well leaves the bins without sense)
    const bool plain = !endless && temperature >= 0x1p-40f && temperature <= 0x1p40f;
    const Fast fast = plain ? fast_draw(a, row, in, maxima, weight, k, p, floor, uniform, s, &last) : Fast::kNot;
    if (fast == Fast::kDrawn) return;
    if (fast == Fast::kNot) {
      u64 taken = ~0ull, taken_p;
      if (k > 0) last = descend<false>(in, as, weight, static_cast<u64>(k), 0, s, &taken);
      if (p < 1.f) {
        sum_up(in, 0);
        const u64 by_p = descend<true>(in, as, weight, share_of(p, total()), last, s, &taken_p);
        if (taken_p < taken) last = by_p;
      }
      sum_up(in, floor);
    }
  }
  const u64 all = total();
  const u64 target = draw_of(uniform, all);
  u64 before;
  __syncthreads();
  const int piece = find_piece(in.turns, target, s, &before);
  if (wave != 0) return;
  const int w0 = piece * 64 + lane, index = in.first(w0);
  float x[R::VEC];
  R::values(in.word(w0), x);
  u64 v[R::VEC], sum = 0;
  times<R::VEC>([&](auto i) {
    x[i] = as(x[i]);
    v[i] = last == 0 || place_of(x[i], index + i) >= last ? weight.fixed_from(x[i], floor) : 0;
    sum += v[i];
  });
  u64 c = before + wave_upto(sum) - sum;
  times<R::VEC>([&](auto i) {
    if (c <= target && c + v[i] > target) {
      a.tokens[row] = index + i;
      if (a.probs) a.probs[row] = static_cast<float>(weight(x[i]) * weight.unit / static_cast<double>(all));
    }
    c += v[i];
  });
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
  // (a row's workgroup reads other rows' settings, and runs beside those that write)
  const int64_t n = g->rows, eb = g->dtype == AUG_F32 ? 4 : 2, most = int64_t{1} << 58;
  const int64_t reach = n - 1 <= most / g->stride ? (n - 1) * g->stride + g->vocab : most;
  const aug::Span read[] = {{"logits", g->logits, reach * eb}, {"uniform", g->uniform, 4 * n}, {"temperature", g->temperature, 4 * n},
                            {"top_k", g->top_k, 4 * n}, {"top_p", g->top_p, 4 * n}, {"min_p", g->min_p, 4 * n}};
  const aug::Span tokens{"tokens", g->tokens, 4 * n}, probs{"probs", g->probs, 4 * n};
  if (aug::overlap(tokens, probs)) return aug::fail(AUG_ERR_INVALID, "%s: tokens overlap probs", who);
  for (const aug::Span& r : read)
    if (aug::overlap(r, tokens) || aug::overlap(r, probs))
      return aug::fail(AUG_ERR_INVALID, "%s: tokens or probs overlap %s", who, r.name);
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
