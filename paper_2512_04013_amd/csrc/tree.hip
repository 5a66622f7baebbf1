// Attention of drafted tokens (trees of them) over the paged cache, with the lengths on
// the GPU.
//
// The n rows of a request and the G query heads of a KV head make n G query vectors
// that share one K/V stream: they are the columns of the products, and the stream is cut
// into spans of keys. A wave takes T tiles of 16 columns, 32 of them or 64. The four waves
// of a workgroup share out up to 128 columns (`wide` = 1, 2 or 4 groups of them) and the
// span's steps: with more columns fewer waves share the steps, and those with other columns
// find K and V in the caches. Per wave and step of two 16-token blocks (32 keys), with lane
// l = 16 g + j:
//   S^T[16 keys][16 columns] = K Q^T, D / 32 MFMAs 16x16x32 for each block and
//     tile. Lane l brings token j of the block and eight dims a step, the same
//     eight of K and Q.
//   The result gives lane l column j and keys 4g .. 4g + 3 of each block, which is the
//   B operand of a 16x16x32 MFMA over the 32 keys (slots 0 .. 3 of lane group g the
//   first block's, 4 .. 7 the second's): probabilities go on without any exchange.
//   O^T[D dims][16 columns] += V^T P^T, D / 16 MFMAs for 16 columns: row m of MFMA b is dim
//     (D / 16) m + b, so that a lane loads neighbouring dims of its tokens and regroups them.
// K and V operands are made once a step and used for all T tiles. The next step's K is asked
// for behind the products with this one's, its V behind those with this V: one set of
// registers holds them, which leaves room for two or three waves a SIMD (two sets took
// 60 registers more; with them and a branch at each product for tiles without columns, the
// cases below took 198, 308 and 460 us).
// Waves with the same columns are merged through LDS, spans by a second launch.
//
// 64 requests of 8 drafts behind about 2500 tokens, bf16, 32/8 heads: 181 us with the second
// launch (12 us), 890 MB of K and V at 5.4 TB/s while the kernel runs; its items start and end in
// two rounds. 128 requests of up to 16 drafts, fp8, 64/8 heads: 250 us, 882 MB, 111 GFLOP; 8
// requests of 64 drafts behind 16384 to 32768 tokens, fp4: 270 us, 233 GFLOP. Those two are bound by
// vector instructions (bf16 made of the codes, the softmax: 200 a step of 32 columns over fp8, 160
// over fp4, beside 32 MFMAs), which keep the SIMDs busy half of the time and overlap with the
// MFMAs (a quarter, a third) in part.
//
// fp32 caches: the same with 16x16x4 fp32 MFMAs, one block a step.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "attn_kernels.h"

namespace {

constexpr int kTreeWaves = 4;
constexpr int kTreeUnit = 128;         // keys: one step of four waves
constexpr int kTreeTarget = 1024;      // work items that a plan aims at: two rounds of two workgroups a compute unit
constexpr int kTreeMinSpan = 2;        // units
constexpr int kPlanThreads = 1024;

struct TreeHeader {                    // 64 bytes
  int32_t num_items;
  int32_t num_groups;
  int32_t hkv, group, tiles;           // what it was made for: heads,
  int32_t max_rows, max_blocks;        // and the batch
  int32_t reqs_drafts;                 // num_reqs and 2^16 max_draft
  int32_t reserved[8];
};
struct TreeItem {                      // 32 bytes
  int32_t req;
  int16_t kvh;
  int8_t tile;                         // of 16 T * wide columns
  int8_t wide;
  int32_t key_begin, key_end;
  int32_t q_row0, n_rows;              // of the request
  int32_t kv_len;
  int32_t part;                        // first of `wide` partial results, -1: the only span
};
struct TreeGroup {                     // 32 bytes: one item's columns over all spans
  int32_t q_row0, n_rows;
  int16_t kvh;
  int8_t tile;
  int8_t wide;
  int32_t part0, n_parts;              // those of a span follow those of the one before
  int32_t reserved[3];
};
static_assert(sizeof(TreeHeader) == 64 && sizeof(TreeItem) == 32 && sizeof(TreeGroup) == 32, "plan layout");

// num_reqs is up to 4096 and max_draft up to 64.
__host__ __device__ constexpr int32_t reqs_drafts_of(int num_reqs, int max_draft) { return num_reqs | (max_draft << 16); }

// What follows from a shape and the limits of a batch, on the host.
struct TreeSizes {
  int tiles, merge_tiles;              // of 16 columns: of a wave, of a group at most
  int64_t items, groups, parts;        // at most
  int64_t plan_bytes, workspace_bytes;
};

struct TreePlanArgs {
  const int32_t* q_start;
  const int32_t* kv_len;
  char* plan;
  int64_t items;                       // places for items: groups follow them
  int32_t num_reqs, max_rows, max_blocks, max_draft, hkv, group;
  int32_t tiles;                       // of 16 columns, of a wave
};

// Sum of v over the threads before this one.
template <typename T>
__device__ __forceinline__ T sum_before(T v, T* waves, T* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T upto = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  T before = upto - v, sum = 0;
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before += waves[w];
    sum += waves[w];
  }
  *total = sum;
  return before;
}

// Waves of a workgroup that have different columns, for a request's columns and a wave's tiles.
__host__ __device__ __forceinline__ int wide_for(int columns, int tiles) {
  const int waves = (columns + 16 * tiles - 1) / (16 * tiles), most = 8 / tiles;
  return waves <= 1 ? 1 : waves == 2 || most == 2 ? 2 : 4;
}

// One workgroup: spans that take equally long (keys x wide), long enough that about
// kTreeTarget items come out. With L units of keys, c / wide the span and items = sum of
// tiles x KV heads x ceil(L wide / c), c >= sum(tiles x KV heads x L x wide) / kTreeTarget gives at most
// kTreeTarget + requests x KV heads x tiles items, and at most 2 kTreeTarget of requests that
// are split (L wide > c, so ceil(L wide / c) < 2 L wide / c).
__global__ __launch_bounds__(kPlanThreads) void tree_plan_kernel(TreePlanArgs a) {
  extern __shared__ int32_t firsts[];                 // per request: first item, partial, group
  __shared__ unsigned long long waves64[kPlanThreads / 64];
  __shared__ int32_t waves[kPlanThreads / 64];
  const int n = a.num_reqs, tid = threadIdx.x;
  int32_t* first_item = firsts;                       // [n]
  int32_t* first_part = firsts + n;
  int32_t* first_group = firsts + 2 * n;
  int32_t* before = firsts + 3 * n;                   // [16 classes][rounds][waves]
  uint16_t* order = reinterpret_cast<uint16_t*>(before + 256 * ((n + kPlanThreads - 1) / kPlanThreads));
  struct Req { int32_t q0, rows, keys, units, tiles, wide; };
  const auto request = [&](int r) {
    Req q;
    q.q0 = min(max(a.q_start[r], 0), a.max_rows);
    q.rows = min(max(a.q_start[r + 1] - q.q0, 0), min(a.max_draft, a.max_rows - q.q0));
    q.keys = static_cast<int32_t>(min(static_cast<int64_t>(max(a.kv_len[r], 0)), static_cast<int64_t>(a.max_blocks) * kBlock));
    q.units = (q.keys + kTreeUnit - 1) / kTreeUnit;
    q.wide = wide_for(q.rows * a.group, a.tiles);
    q.tiles = (q.rows * a.group + 16 * a.tiles * q.wide - 1) / (16 * a.tiles * q.wide);
    return q;
  };
  const int per = (n + kPlanThreads - 1) / kPlanThreads;
  const int r0 = min(tid * per, n), r1 = min(r0 + per, n);

  // The span (x wide): an even share of the work, or up to twice that where rounding up makes more
  // items (1104 for two rounds of 512 took a third round: 460 us against 406).
  int32_t span = kTreeMinSpan;
  const auto length_of = [&](const Req& q) {
    // (units * wide is up to 2^19, span up to 2^21)
    const uint32_t s = max(static_cast<uint32_t>(q.units * q.wide + span - 1) / static_cast<uint32_t>(span), 1u);
    return max(static_cast<int>((q.units + s - 1) / s), 1);
  };
  const auto spans_of = [&](const Req& q) { const uint32_t l = length_of(q); return max(static_cast<int>((q.units + l - 1) / l), 1); };
  {
    unsigned long long work = 0, total;
    for (int r = r0; r < r1; ++r) {
      const Req q = request(r);
      work += static_cast<unsigned long long>(q.units) * q.tiles * q.wide * a.hkv;
    }
    sum_before(work, waves64, &total);
    // (no request is longer than 2^19)
    const int64_t even = min(static_cast<int64_t>((total + kTreeTarget - 1) / kTreeTarget), int64_t{1} << 20);
    span = max(span, static_cast<int32_t>(even));
    const int32_t most = 2 * span;
    for (int i = 0; i < 4; ++i) {
      int32_t items = 0, all;
      for (int r = r0; r < r1; ++r) {
        const Req q = request(r);
        items += q.tiles * a.hkv * spans_of(q);
      }
      sum_before(items, waves, &all);
      if (all <= kTreeTarget || span >= most) break;
      const int64_t longer = static_cast<int64_t>(span) * (all + kTreeTarget) / (2 * kTreeTarget);
      span = static_cast<int32_t>(min(static_cast<int64_t>(most), max(static_cast<int64_t>(span) + 1, longer)));
    }
  }
  // Requests with the longest items first: those behind fill the gaps at the end (198 us against 182,
  // 302 against 267, of lengths that differ). 16 classes of length (keys x wide), in each the requests' order.
  constexpr int kClasses = 16, kWaves = kPlanThreads / 64;
  const int lane = tid & 63, wave = tid >> 6, rounds = (n + kPlanThreads - 1) / kPlanThreads;
  const auto class_of = [&](const Req& q) {
    return kClasses - 1 - static_cast<int>(static_cast<uint32_t>(min(length_of(q) * q.wide, span)) * (kClasses - 1) / static_cast<uint32_t>(span));
  };
  for (int k = 0; k < rounds; ++k) {
    const int r = k * kPlanThreads + tid;
    const int mine = r < n ? class_of(request(r)) : -1;
    for (int c = 0; c < kClasses; ++c) {
      const int count = __popcll(__ballot(mine == c));
      if (lane == 0) before[(c * rounds + k) * kWaves + wave] = count;
    }
  }
  __syncthreads();
  {
    const int all = kClasses * rounds * kWaves, each = (all + kPlanThreads - 1) / kPlanThreads;
    int32_t sum = 0, unused;
    for (int i = 0; i < each; ++i) sum += tid * each + i < all ? before[tid * each + i] : 0;
    int32_t at = sum_before(sum, waves, &unused);
    for (int i = 0; i < each && tid * each + i < all; ++i) {
      const int32_t count = before[tid * each + i];
      before[tid * each + i] = at;
      at += count;
    }
  }
  __syncthreads();
  for (int k = 0; k < rounds; ++k) {
    const int r = k * kPlanThreads + tid;
    const int mine = r < n ? class_of(request(r)) : -1;
    for (int c = 0; c < kClasses; ++c) {
      const unsigned long long same = __ballot(mine == c);
      if (mine == c) order[before[(c * rounds + k) * kWaves + wave] + __popcll(same & ((1ull << lane) - 1))] = static_cast<uint16_t>(r);
    }
  }
  __syncthreads();
  int32_t items = 0, parts = 0, groups = 0;
  for (int p = r0; p < r1; ++p) {
    const Req q = request(order[p]);
    const int s = spans_of(q), columns = q.tiles * a.hkv;
    items += columns * s;
    parts += s > 1 ? columns * q.wide * s : 0;
    groups += s > 1 ? columns : 0;
  }
  int32_t num_items, num_parts, num_groups;
  int32_t item = sum_before(items, waves, &num_items);
  int32_t part = sum_before(parts, waves, &num_parts);
  int32_t group = sum_before(groups, waves, &num_groups);
  for (int p = r0; p < r1; ++p) {
    const Req q = request(order[p]);
    const int s = spans_of(q), columns = q.tiles * a.hkv;
    first_item[p] = item;
    first_part[p] = part;
    first_group[p] = group;
    item += columns * s;
    part += s > 1 ? columns * q.wide * s : 0;
    group += s > 1 ? columns : 0;
  }
  if (tid == 0)
    *reinterpret_cast<TreeHeader*>(a.plan) = TreeHeader{num_items,  num_groups,   a.hkv, a.group, a.tiles,
                                                        a.max_rows, a.max_blocks, reqs_drafts_of(n, a.max_draft), {}};
  __syncthreads();
  TreeItem* out = reinterpret_cast<TreeItem*>(a.plan + sizeof(TreeHeader));
  TreeGroup* group_out = reinterpret_cast<TreeGroup*>(out + a.items);
  for (int i = tid; i < num_items; i += kPlanThreads) {
    int lo = 0, hi = n - 1;                           // the last place whose first item is not behind i
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (first_item[mid] <= i) lo = mid; else hi = mid - 1;
    }
    const int req = order[lo];
    const Req q = request(req);
    const int s = spans_of(q), length = length_of(q) * kTreeUnit;
    const int local = i - first_item[lo];
    const int tile = local % q.tiles, at = local / q.tiles % s, kvh = local / (q.tiles * s);
    const int column = kvh * q.tiles + tile;
    TreeItem it;
    it.req = req;
    it.kvh = static_cast<int16_t>(kvh);
    it.tile = static_cast<int8_t>(tile);
    it.wide = static_cast<int8_t>(q.wide);
    it.key_begin = at * length;
    it.key_end = min(it.key_begin + length, q.keys);
    it.q_row0 = q.q0;
    it.n_rows = q.rows;
    it.kv_len = q.keys;
    it.part = s > 1 ? first_part[lo] + (column * s + at) * q.wide : -1;
    out[i] = it;
    if (s > 1 && at == 0)
      group_out[first_group[lo] + column] =
          TreeGroup{q.q0, q.rows, it.kvh, it.tile, it.wide, it.part, s, {}};
  }
}

// ---------------------------------------------------------------------------

struct TreeArgs {
  const char* plan;
  const void* q;
  const char* k_cache;
  const char* v_cache;
  const float* k_scale;
  const float* v_scale;
  const int32_t* block_table;
  const uint64_t* seen;
  void* out;
  float* partials;
  int64_t items;
  int32_t max_blocks, num_pool_blocks, hq, hkv;
  int32_t max_rows, reqs_drafts;
  int32_t group_log2;
  int32_t max_groups, merge_tiles;     // tiles of a group, at most
  float scale_log2;
};

__device__ __forceinline__ int64_t tree_cell(const TreeArgs& a, int bid, int kvh) { return static_cast<int64_t>(bid) * a.hkv + kvh; }

// A block's K and V of a lane, and what the products take of them.
template <int KVT, int D> struct TreeKv;
template <int D> struct TreeKv<KV_BF16, D> {
  using v_t = std::conditional_t<D == 128, uint4, uint2>;
  struct K { uint4 x[D / 32]; float scale = 1.f; };
  struct V { v_t x[4]; float scale = 1.f; };
  static constexpr int EB = 2;
  __device__ static constexpr int k_dim(int s, int g) { return 32 * s + 8 * g; }
  __device__ static void load(const TreeArgs& a, int bid, int kvh, int j, int g, K& b) {
    const char* k = a.k_cache + tree_cell(a, bid, kvh) * (kBlock * D * EB) + static_cast<uint32_t>(j * D * EB + 16 * g);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) b.x[i] = *reinterpret_cast<const uint4*>(k + 64 * i);
  }
  __device__ static void load(const TreeArgs& a, int bid, int kvh, int j, int g, V& b) {
    const char* v = a.v_cache + tree_cell(a, bid, kvh) * (kBlock * D * EB) + static_cast<uint32_t>((4 * g * D + D / 16 * j) * EB);
#pragma unroll
    for (int t = 0; t < 4; ++t) b.x[t] = *reinterpret_cast<const v_t*>(v + t * D * EB);
  }
  __device__ static uint4 k_operand(const K& b, int s) { return b.x[s]; }
  __device__ static void drop(V& b, int t) { b.x[t] = v_t{}; }
  // dims 2i and 2i + 1 of the lane's, over the keys of both blocks
  __device__ static void v_operands(const V& b0, const V& b1, int i, uint4& even, uint4& odd) {
    const auto word = [&](const V& b, int t) { return reinterpret_cast<const uint32_t*>(&b.x[t])[i]; };
    const auto pair = [&](uint32_t which) {
      return uint4{__builtin_amdgcn_perm(word(b0, 1), word(b0, 0), which), __builtin_amdgcn_perm(word(b0, 3), word(b0, 2), which),
                   __builtin_amdgcn_perm(word(b1, 1), word(b1, 0), which), __builtin_amdgcn_perm(word(b1, 3), word(b1, 2), which)};
    };
    even = pair(0x05040100u);
    odd = pair(0x07060302u);
  }
};
template <> struct TreeKv<KV_FP8, 128> {
  struct K { uint4 x[2]; float scale; };
  struct V { uint2 x[4]; float scale; };
  static constexpr int D = 128;
  __device__ static constexpr int k_dim(int s, int g) { return 64 * (s >> 1) + 16 * g + 8 * (s & 1); }
  __device__ static void load(const TreeArgs& a, int bid, int kvh, int j, int g, K& b) {
    const int64_t cell = tree_cell(a, bid, kvh);
    const char* k = a.k_cache + cell * (kBlock * D) + static_cast<uint32_t>(j * D + 16 * g);
    b.x[0] = *reinterpret_cast<const uint4*>(k);
    b.x[1] = *reinterpret_cast<const uint4*>(k + 64);
    b.scale = load_uniform(a.k_scale + cell);
  }
  __device__ static void load(const TreeArgs& a, int bid, int kvh, int j, int g, V& b) {
    const int64_t cell = tree_cell(a, bid, kvh);
    const char* v = a.v_cache + cell * (kBlock * D) + static_cast<uint32_t>(4 * g * D + 8 * j);
#pragma unroll
    for (int t = 0; t < 4; ++t) b.x[t] = *reinterpret_cast<const uint2*>(v + t * D);
    b.scale = load_uniform(a.v_scale + cell);
  }
  __device__ static uint4 k_operand(const K& b, int s) {
    const uint4& w = b.x[s >> 1];
    const uint32_t lo = (s & 1) ? w.z : w.x, hi = (s & 1) ? w.w : w.y;
    return uint4{fp8x2_to_bf16x2<false>(lo), fp8x2_to_bf16x2<true>(lo), fp8x2_to_bf16x2<false>(hi), fp8x2_to_bf16x2<true>(hi)};
  }
  __device__ static void drop(V& b, int t) { b.x[t] = uint2{0u, 0u}; }
  __device__ static void v_operands(const V& b0, const V& b1, int i, uint4& even, uint4& odd) {
    // bytes of dims 2i and 2i + 1 of two tokens side by side: a byte pair converts to the
    // bf16 pair of one dim
    const auto word = [&](const V& b, int t) { return i & 2 ? b.x[t].y : b.x[t].x; };
    const uint32_t which = i & 1 ? 0x07030602u : 0x05010400u;
    const uint32_t a01 = __builtin_amdgcn_perm(word(b0, 1), word(b0, 0), which), a23 = __builtin_amdgcn_perm(word(b0, 3), word(b0, 2), which);
    const uint32_t c01 = __builtin_amdgcn_perm(word(b1, 1), word(b1, 0), which), c23 = __builtin_amdgcn_perm(word(b1, 3), word(b1, 2), which);
    even = uint4{fp8x2_to_bf16x2<false>(a01), fp8x2_to_bf16x2<false>(a23), fp8x2_to_bf16x2<false>(c01), fp8x2_to_bf16x2<false>(c23)};
    odd = uint4{fp8x2_to_bf16x2<true>(a01), fp8x2_to_bf16x2<true>(a23), fp8x2_to_bf16x2<true>(c01), fp8x2_to_bf16x2<true>(c23)};
  }
};
template <> struct TreeKv<KV_FP4, 128> {
  struct K { uint4 x; uint32_t e; float scale = 1.f; };
  struct V { uint4 x; uint32_t e; float scale = 1.f; };
  __device__ static constexpr int k_dim(int s, int g) { return 32 * g + 8 * s; }
  // a block's codes of all heads, then their scales
  __device__ static const char* codes(const TreeArgs& a, const char* cache, int bid, int kvh) {
    return cache + (static_cast<int64_t>(bid) * a.hkv * aug::kMxCell + kvh * aug::kMxCodes);
  }
  __device__ static const char* scales(const TreeArgs& a, const char* cache, int bid, int kvh) {
    return cache + (static_cast<int64_t>(bid) * a.hkv * aug::kMxCell + (a.hkv * aug::kMxCodes + kvh * aug::kMxScales));
  }
  __device__ static void load(const TreeArgs& a, int bid, int kvh, int j, int g, K& b) {
    b.x = *reinterpret_cast<const uint4*>(codes(a, a.k_cache, bid, kvh) + static_cast<uint32_t>(64 * j + 16 * g));
    b.e = *reinterpret_cast<const uint8_t*>(scales(a, a.k_cache, bid, kvh) + static_cast<uint32_t>(4 * j + g));
  }
  __device__ static void load(const TreeArgs& a, int bid, int kvh, int j, int g, V& b) {
    b.x = *reinterpret_cast<const uint4*>(codes(a, a.v_cache, bid, kvh) + static_cast<uint32_t>(256 * g + 16 * j));
    b.e = *reinterpret_cast<const uint32_t*>(scales(a, a.v_cache, bid, kvh) + static_cast<uint32_t>(16 * (j >> 2) + 4 * g));
  }
  __device__ static uint4 k_operand(const K& b, int s) {
    const uint32_t w = s == 0 ? b.x.x : s == 1 ? b.x.y : s == 2 ? b.x.z : b.x.w;
    return fp4x8_to_bf16x8(w, fp4_scale(b.e, 0));
  }
  // value and scale (255 stands for NaN) zero
  __device__ static void drop(V& b, int t) {
    (t == 0 ? b.x.x : t == 1 ? b.x.y : t == 2 ? b.x.z : b.x.w) = 0u;
    b.e &= ~(0xFFu << (8 * t));
  }
  template <int E>
  __device__ static void decode(const V& b, uint32_t (&x)[4]) {
    const uint32_t w[4] = {b.x.x, b.x.y, b.x.z, b.x.w};
#pragma unroll
    for (int t = 0; t < 4; ++t)
      x[t] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[t], fp4_scale(b.e, t), E));
  }
  __device__ static void v_operands(const V& b0, const V& b1, int i, uint4& even, uint4& odd) {
    uint32_t x[4], y[4];
    switch (i) {
      case 0: decode<0>(b0, x); decode<0>(b1, y); break;
      case 1: decode<1>(b0, x); decode<1>(b1, y); break;
      case 2: decode<2>(b0, x); decode<2>(b1, y); break;
      default: decode<3>(b0, x); decode<3>(b1, y); break;
    }
    const auto pair = [&](uint32_t which) {
      return uint4{__builtin_amdgcn_perm(x[1], x[0], which), __builtin_amdgcn_perm(x[3], x[2], which),
                   __builtin_amdgcn_perm(y[1], y[0], which), __builtin_amdgcn_perm(y[3], y[2], which)};
    };
    even = pair(0x05040100u);
    odd = pair(0x07060302u);
  }
};

constexpr int tree_row(int D) { return D + 4; }      // floats of a wave's result of one column in LDS
constexpr int tree_merge_floats(int D) { return kTreeWaves * 16 * tree_row(D); }
constexpr int64_t tree_partial_floats(int D, int tiles) { return int64_t{16} * tiles * (D + 2); }

// A tile of 16 columns is written: out (bf16 or fp32), or its part of the item's partial.
// Thread `tid` takes D / 16 dims of column tid / 16.
template <int D, bool F32>
__device__ __forceinline__ void tree_store(const TreeArgs& a, int q_row0, int n_rows, int kvh, int column, int dim, const float* o) {
  const int row = column >> a.group_log2, head = column & ((1 << a.group_log2) - 1);
  if (row >= n_rows) return;
  const int64_t at = (static_cast<int64_t>(q_row0 + row) * a.hq + (kvh << a.group_log2) + head) * D + dim;
  constexpr int N = D / 16;
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at + i) = float4{o[i], o[i + 1], o[i + 2], o[i + 3]};
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at + i) = uint2{pack_bf16(o[i], o[i + 1]), pack_bf16(o[i + 2], o[i + 3])};
  }
}

// The results of tile t of a group's columns (lds: o[D], maximum and sum of each wave and
// column) of the waves that have them, group, group + wide, ..., joined, and stored as the result or as
// the item's partial.
template <int D, int T, bool F32>
__device__ __forceinline__ void tree_join(const TreeArgs& a, const TreeItem& it, int group, int t, const float* lds, int tid) {
  constexpr int ROW = tree_row(D), N = D / 16;
  const int c = tid >> 4, dim = N * (tid & 15);
  float m = kNegBig;
  for (int w = group; w < kTreeWaves; w += it.wide) m = fmaxf(m, lds[(w * 16 + c) * ROW + D]);
  float l = 0.f, o[N] = {};
  for (int w = group; w < kTreeWaves; w += it.wide) {
    const float* p = lds + (w * 16 + c) * ROW;
    const float f = __builtin_amdgcn_exp2f(p[D] - m);
    l = fmaf(f, p[D + 1], l);
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = fmaf(f, p[dim + i], o[i]);
  }
  if (it.part < 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = over_sum(o[i], l);
    tree_store<D, F32>(a, it.q_row0, it.n_rows, it.kvh, ((it.tile * it.wide + group) * T + t) * 16 + c, dim, o);
    return;
  }
  if (((((it.tile * it.wide + group) * T + t) * 16 + c) >> a.group_log2) >= it.n_rows) return;
  float* part = a.partials + (it.part + group) * tree_partial_floats(D, T);
  float* dst = part + (16 * t + c) * D + dim;
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(dst + i) = float4{o[i], o[i + 1], o[i + 2], o[i + 3]};
  if ((tid & 15) == 0) {
    part[16 * T * D + 16 * t + c] = m;
    part[16 * T * (D + 1) + 16 * t + c] = l;
  }
}

// Items and groups of the plan; none where it was made for other heads, tiles or sizes of the batch, whose
// items lie outside this launch's arrays.
__device__ __forceinline__ int2 tree_counts(const TreeArgs& a, int tiles) {
  typedef int32_t words_t __attribute__((ext_vector_type(8)));
  const words_t h = load_uniform(reinterpret_cast<const words_t*>(a.plan));
  const bool mine = h[2] == a.hkv && h[3] == 1 << a.group_log2 && h[4] == tiles && h[5] == a.max_rows && h[6] == a.max_blocks &&
                    h[7] == a.reqs_drafts;
  return mine ? int2{h[0], h[1]} : int2{0, 0};
}

__device__ __forceinline__ TreeItem load_tree_item(const TreeItem* p) {
  typedef int32_t words_t __attribute__((ext_vector_type(8)));
  const words_t raw = load_uniform(reinterpret_cast<const words_t*>(p));
  TreeItem it;
  __builtin_memcpy(&it, &raw, sizeof(it));
  return it;
}

// The columns of a lane: query operand addresses and masks.
struct TreeColumn {
  bool live;
  int64_t q;              // elements before the query vector
  uint64_t seen;
};
__device__ __forceinline__ TreeColumn tree_column(const TreeArgs& a, const TreeItem& it, int column, int D) {
  TreeColumn c;
  const int row = column >> a.group_log2, head = column & ((1 << a.group_log2) - 1);
  c.live = row < it.n_rows;
  c.q = (static_cast<int64_t>(it.q_row0 + row) * a.hq + (it.kvh << a.group_log2) + head) * D;
  c.seen = c.live ? a.seen[it.q_row0 + row] : 0;
  return c;
}
// Drafts that some column of the wave sees.
__device__ __forceinline__ uint64_t seen_by_any(uint64_t m) {
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) m |= static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(m), d));
  return m;
}

// Two or three waves a SIMD, as the registers allow.
template <int KVT, int D, int T>
__global__ __launch_bounds__(kThreads, T == 4 || (KVT == KV_BF16 && D == 128) ? 2 : 3) void tree_kernel(TreeArgs a) {
  using KV = TreeKv<KVT, D>;
  constexpr int KS = D / 32, NB = D / 16;
  constexpr bool FP8 = KVT == KV_FP8;
  constexpr bool PAIRS = KVT == KV_BF16;               // probabilities as two bf16
  constexpr int kQuery = 8 * KS * 64;                  // 16-byte query operands
  constexpr int kLds = kQuery * 16 > tree_merge_floats(D) * 4 ? kQuery * 16 : tree_merge_floats(D) * 4;
  __shared__ __align__(16) char lds[kLds];
  const int items = tree_counts(a, T).x;
  const TreeItem it = load_tree_item(reinterpret_cast<const TreeItem*>(a.plan + sizeof(TreeHeader)) + blockIdx.x);
  if (static_cast<int>(blockIdx.x) >= items) return;
  const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int base = it.kv_len - it.n_rows;              // tokens before the drafts

  // the wave's columns, and its share of the steps
  const int group = wave & (it.wide - 1), turn = wave / it.wide, turns = kTreeWaves / it.wide;
  const int columns = (it.n_rows << a.group_log2) - (it.tile * it.wide + group) * 16 * T;    // from the wave's first on
  const int blk0 = it.key_begin / kBlock;
  const int nblk = (it.key_end - it.key_begin + kBlock - 1) / kBlock;
  const int32_t* table = a.block_table + static_cast<int64_t>(it.req) * a.max_blocks + blk0;
  int next[2];
  const auto ids = [&](int bi) {
#pragma unroll
    for (int i = 0; i < 2; ++i) next[i] = bi + i < nblk ? load_uniform(table + bi + i) : -1;
  };
  const auto usable = [&](int bid) { return static_cast<uint32_t>(bid) < static_cast<uint32_t>(a.num_pool_blocks); };
  // A block that is none (past the span, or outside the pool) loads the pool's first one
  // and counts for nothing.
  const auto in_pool = [&](int bid) { return usable(bid) ? bid : 0; };
  typename KV::K k[2];
  typename KV::V v[2];
  int bid[2];
  const int step = 2 * turns;
  int bi = columns > 0 ? 2 * turn : nblk;
  ids(bi);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    KV::load(a, in_pool(next[i]), it.kvh, j, g, k[i]);
    KV::load(a, in_pool(next[i]), it.kvh, j, g, v[i]);
    bid[i] = next[i];
  }
  ids(bi + step);

  // the queries, once for the waves that have them
  uint64_t seen[T], any = 0;
  uint4* query = reinterpret_cast<uint4*>(lds) + group * T * KS * 64;
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const TreeColumn c = tree_column(a, it, ((it.tile * it.wide + group) * T + t) * 16 + j, D);
    seen[t] = c.seen;
    any |= c.seen;
    if (t % turns != turn % T) continue;
#pragma unroll
    for (int s = 0; s < KS; ++s)
      query[(t * KS + s) * 64 + lane] =
          c.live ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + c.q + KV::k_dim(s, g)) : uint4{0u, 0u, 0u, 0u};
  }
  any = seen_by_any(any);
  __syncthreads();

  const float sc = a.scale_log2;
  float m_run[T], l_run[T];
  f32x4_t oacc[T][NB];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    m_run[t] = kNegBig;
    l_run[t] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) oacc[t][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  int lane_of_query = lane;
  const auto compute = [&](auto tiles, int bi, int bi_next) __attribute__((always_inline)) {
    constexpr int N = decltype(tiles)::value;            // tiles that have columns
    asm volatile("" : "+v"(lane_of_query));           // the operands stay in LDS
    const int tok0 = (blk0 + bi) * kBlock;
    const bool ok[2] = {usable(bid[0]), usable(bid[1])};
    const bool full = ok[0] && ok[1] && tok0 + 2 * kBlock <= min(it.key_end, base);
    f32x4_t sacc[N][2];
#pragma unroll
    for (int t = 0; t < N; ++t) sacc[t][0] = sacc[t][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const bf16x8_t k0 = as_bf16x8(KV::k_operand(k[0], s)), k1 = as_bf16x8(KV::k_operand(k[1], s));
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const bf16x8_t qop = as_bf16x8(query[(t * KS + s) * 64 + lane_of_query]);
        sacc[t][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qop, sacc[t][0], 0, 0, 0);
        sacc[t][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qop, sacc[t][1], 0, 0, 0);
      }
    }
    float coef[2] = {sc, sc};
    if constexpr (FP8) {
      coef[0] *= k[0].scale;
      coef[1] *= k[1].scale;
      if ((__float_as_int(k[0].scale) | __float_as_int(k[1].scale)) < 0) {      // below, the largest score is that of the largest product
#pragma unroll
        for (int t = 0; t < N; ++t) {
          sacc[t][0] *= coef[0];
          sacc[t][1] *= coef[1];
        }
        coef[0] = coef[1] = 1.f;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // the next blocks' K is on its way from here on
#pragma unroll
    for (int i = 0; i < 2; ++i) KV::load(a, in_pool(next[i]), it.kvh, j, g, k[i]);
    __builtin_amdgcn_sched_barrier(0);
    float vlog[2] = {0.f, 0.f}, vinv[2] = {1.f, 1.f};
    if constexpr (FP8) {
      // a block's V scale enters each probability through its log2 and leaves the row sum
      // through its reciprocal (a zero scale is taken as 2^-100; one that is not finite belongs
      // to a block that nothing sees)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float vs = fminf(fmaxf(v[i].scale, 0x1p-100f), 0x1p100f);
        vlog[i] = __builtin_amdgcn_logf(vs);
        vinv[i] = __builtin_amdgcn_rcpf(vs);
      }
    }
    const auto visible = [&](int r, uint64_t mask) {
      const int tok = tok0 + kBlock * (r >> 2) + 4 * g + (r & 3);
      return ok[r >> 2] && tok < it.key_end && (tok < base || ((mask >> ((tok - base) & 63)) & 1));
    };
    uint32_t hidden = 0;                                 // bit 8 t + r: tile t does not see the lane's key r
    if (!full) {
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        if (!visible(r, any)) KV::drop(v[r >> 2], r & 3);      // zero, so 0 * value never meets NaN
#pragma unroll
        for (int t = 0; t < N; ++t)
          if (!visible(r, seen[t])) {
            sacc[t][r >> 2][r & 3] = -INFINITY;
            hidden |= 1u << (8 * t + r);
          }
      }
    }
    // scores in powers of two: the products are scaled where they are used
    float top[N];
    bool moved = false;
#pragma unroll
    for (int t = 0; t < N; ++t) {
      const auto top4 = [](f32x4_t x) { return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])); };
      top[t] = FP8 ? fmaxf(top4(sacc[t][0]) * coef[0], top4(sacc[t][1]) * coef[1]) : fmaxf(top4(sacc[t][0]), top4(sacc[t][1])) * sc;
      moved |= top[t] > m_run[t] + kRescaleSlack;
    }
    if (__any(moved)) {
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const float mn = fmaxf(m_run[t], group4_max(top[t]));
        const float alpha = __builtin_amdgcn_exp2f(m_run[t] - mn);
        l_run[t] *= alpha;
#pragma unroll
        for (int b = 0; b < NB; ++b) oacc[t][b] *= alpha;
        m_run[t] = mn;
      }
    }
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float bias = FP8 ? vlog[i] - m_run[t] : -m_run[t];
#pragma unroll
        for (int r = 0; r < 4; ++r) sacc[t][i][r] = __builtin_amdgcn_exp2f(fmaf(sacc[t][i][r], coef[i], bias));
      }
    if (!full) {                                         // also where a scale is zero or not finite
#pragma unroll
      for (int t = 0; t < N; ++t)
#pragma unroll
        for (int r = 0; r < 8; ++r) sacc[t][r >> 2][r & 3] = (hidden >> (8 * t + r)) & 1 ? 0.f : sacc[t][r >> 2][r & 3];
    }
    // Probabilities become operands. Over bf16 caches each is two bf16, the second what the first leaves (2^-16 together):
    // the results' own rounding is then all that shows, and its products hide behind the loads (64 requests of 8 drafts,
    // 183 us with and without; 8 of 64 drafts, 64/8 heads, 1218 for 1202; at most, 16 of 64 drafts with heads of 64, 181
    // for 159). Over codes, which are off by 2^-4 and more themselves, each is one (2^-8): two take 282 us for 258 (fp8)
    // and 403 for 279 (4 bits).
    bf16x8_t pop[N], rest[N];
#pragma unroll
    for (int t = 0; t < N; ++t) {
      uint32_t pp[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) pp[r] = pack_bf16(sacc[t][r >> 1][2 * (r & 1)], sacc[t][r >> 1][2 * (r & 1) + 1]);
      if constexpr (PAIRS) {
        uint32_t w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          w[r] = pack_bf16(sacc[t][r >> 1][2 * (r & 1)] - __uint_as_float(pp[r] << 16),
                           sacc[t][r >> 1][2 * (r & 1) + 1] - __uint_as_float(pp[r] & 0xFFFF0000u));
        rest[t] = as_bf16x8(uint4{w[0], w[1], w[2], w[3]});
        l_run[t] += ((sacc[t][0][0] + sacc[t][0][1]) + (sacc[t][0][2] + sacc[t][0][3])) +
                    ((sacc[t][1][0] + sacc[t][1][1]) + (sacc[t][1][2] + sacc[t][1][3]));
      } else {
        // exactly the packed probabilities
        const float s0 = dot2_bf16(pp[1], kBf16PairOne, dot2_bf16(pp[0], kBf16PairOne, 0.f));
        const float s1 = dot2_bf16(pp[3], kBf16PairOne, dot2_bf16(pp[2], kBf16PairOne, 0.f));
        l_run[t] = FP8 ? fmaf(s0, vinv[0], fmaf(s1, vinv[1], l_run[t])) : l_run[t] + (s0 + s1);
      }
      pop[t] = as_bf16x8(uint4{pp[0], pp[1], pp[2], pp[3]});
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < NB / 2; ++i) {
      uint4 even, odd;
      KV::v_operands(v[0], v[1], i, even, odd);
#pragma unroll
      for (int t = 0; t < N; ++t) {
        oacc[t][2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(even), pop[t], oacc[t][2 * i], 0, 0, 0);
        oacc[t][2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(odd), pop[t], oacc[t][2 * i + 1], 0, 0, 0);
        if constexpr (PAIRS) {
          oacc[t][2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(even), rest[t], oacc[t][2 * i], 0, 0, 0);
          oacc[t][2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(odd), rest[t], oacc[t][2 * i + 1], 0, 0, 0);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      KV::load(a, in_pool(next[i]), it.kvh, j, g, v[i]);
      bid[i] = next[i];
    }
    ids(bi_next);
  };
  const auto all_steps = [&](auto tiles) __attribute__((always_inline)) {
    for (; bi < nblk; bi += step) compute(tiles, bi, bi + 2 * step);
  };
  if (T == 2 || columns <= 32) all_steps(std::integral_constant<int, 2>{});
  else all_steps(std::integral_constant<int, T>{});

  float* merge = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int t = 0; t < T; ++t) {
    __syncthreads();                                   // the queries, or the tile before, have been read
    const float l = group4_sum(l_run[t]);
    float* dst = merge + (wave * 16 + j) * tree_row(D);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int b = 0; b < NB; b += 4)
        *reinterpret_cast<float4*>(dst + NB * (4 * g + r) + b) =
            float4{oacc[t][b][r], oacc[t][b + 1][r], oacc[t][b + 2][r], oacc[t][b + 3][r]};
    if (g == 0) {
      dst[D] = m_run[t];
      dst[D + 1] = l;
    }
    __syncthreads();
    for (int g2 = 0; g2 < it.wide; ++g2) tree_join<D, T, false>(a, it, g2, t, merge, threadIdx.x);
  }
}

// fp32: one block a step, 16x16x4 MFMAs. Lane l brings four dims 16i + 4g .. of K and Q
// a load, one of which a step takes; and of V tokens 4g .. 4g + 3, one a step.
template <int D>
__global__ __launch_bounds__(kThreads, 2) void tree_kernel_f32(TreeArgs a) {
  constexpr int KS = D / 16, NB = D / 16, T = 2;
  constexpr int kQuery = kTreeWaves * T * KS * 64;
  constexpr int kLds = kQuery * 16 > tree_merge_floats(D) * 4 ? kQuery * 16 : tree_merge_floats(D) * 4;
  __shared__ __align__(16) char lds[kLds];
  if (static_cast<int>(blockIdx.x) >= tree_counts(a, 2).x) return;
  const TreeItem it = load_tree_item(reinterpret_cast<const TreeItem*>(a.plan + sizeof(TreeHeader)) + blockIdx.x);
  const int lane = threadIdx.x & 63, j = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int base = it.kv_len - it.n_rows;

  // the wave's columns, and its share of the steps
  const int group = wave & (it.wide - 1), turn = wave / it.wide, turns = kTreeWaves / it.wide;
  const int columns = (it.n_rows << a.group_log2) - (it.tile * it.wide + group) * 16 * T;    // from the wave's first on
  uint64_t seen[T], any = 0;
  float4* query = reinterpret_cast<float4*>(lds) + wave * T * KS * 64;
#pragma unroll
  for (int t = 0; t < T; ++t) {
    const TreeColumn c = tree_column(a, it, ((it.tile * it.wide + group) * T + t) * 16 + j, D);
    seen[t] = c.seen;
    any |= c.seen;
#pragma unroll
    for (int s = 0; s < KS; ++s)
      query[(t * KS + s) * 64 + lane] =
          c.live ? *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + c.q + 16 * s + 4 * g) : float4{0.f, 0.f, 0.f, 0.f};
  }
  any = seen_by_any(any);

  float m_run[T], l_run[T];
  f32x4_t oacc[T][NB];
#pragma unroll
  for (int t = 0; t < T; ++t) {
    m_run[t] = kNegBig;
    l_run[t] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b) oacc[t][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int blk0 = it.key_begin / kBlock;
  const int nblk = (it.key_end - it.key_begin + kBlock - 1) / kBlock;
  const int32_t* table = a.block_table + static_cast<int64_t>(it.req) * a.max_blocks + blk0;
  for (int bi = columns > 0 ? turn : nblk; bi < nblk; bi += turns) {
    const int bid = load_uniform(table + bi);
    if (static_cast<uint32_t>(bid) >= static_cast<uint32_t>(a.num_pool_blocks)) continue;
    const int64_t cell = static_cast<int64_t>(bid) * a.hkv + it.kvh;
    const int tok0 = (blk0 + bi) * kBlock;
    const float* kp = reinterpret_cast<const float*>(a.k_cache) + (cell * kBlock + j) * D + 4 * g;
    const float* vp = reinterpret_cast<const float*>(a.v_cache) + (cell * kBlock + 4 * g) * D + NB * j;
    float k[KS][4], v[4][NB];
#pragma unroll
    for (int s = 0; s < KS; ++s) __builtin_memcpy(k[s], reinterpret_cast<const float4*>(kp + 16 * s), 16);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int b = 0; b < NB; b += 4) __builtin_memcpy(&v[r][b], reinterpret_cast<const float4*>(vp + r * D + b), 16);
    const bool full = tok0 + kBlock <= min(it.key_end, base);
    const auto visible = [&](int r, uint64_t mask) {
      const int tok = tok0 + 4 * g + r;
      return tok < it.key_end && (tok < base || ((mask >> ((tok - base) & 63)) & 1));
    };
    if (!full) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (!visible(r, any)) {
#pragma unroll
          for (int b = 0; b < NB; ++b) v[r][b] = 0.f;
        }
    }
#pragma unroll
    for (int t = 0; t < T; ++t) {
      if (16 * t >= columns) break;
      f32x4_t sacc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const float4 q4 = query[(t * KS + s) * 64 + lane];
        const float q[4] = {q4.x, q4.y, q4.z, q4.w};
#pragma unroll
        for (int c = 0; c < 4; ++c) sacc = __builtin_amdgcn_mfma_f32_16x16x4f32(k[s][c], q[c], sacc, 0, 0, 0);
      }
      float sv[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) sv[r] = full || visible(r, seen[t]) ? sacc[r] * a.scale_log2 : -INFINITY;
      const float mn = fmaxf(m_run[t], group4_max(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3]))));
      if (__any(mn > m_run[t] + kRescaleSlack)) {
        const float alpha = __builtin_amdgcn_exp2f(m_run[t] - mn);
        l_run[t] *= alpha;
#pragma unroll
        for (int b = 0; b < NB; ++b) oacc[t][b] *= alpha;
        m_run[t] = mn;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(sv[r] - m_run[t]);
        l_run[t] += p;
#pragma unroll
        for (int b = 0; b < NB; ++b) oacc[t][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][b], p, oacc[t][b], 0, 0, 0);
      }
    }
  }

  float* merge = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int t = 0; t < T; ++t) {
    __syncthreads();
    const float l = group4_sum(l_run[t]);
    float* dst = merge + (wave * 16 + j) * tree_row(D);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int b = 0; b < NB; b += 4)
        *reinterpret_cast<float4*>(dst + NB * (4 * g + r) + b) =
            float4{oacc[t][b][r], oacc[t][b + 1][r], oacc[t][b + 2][r], oacc[t][b + 3][r]};
    if (g == 0) {
      dst[D] = m_run[t];
      dst[D + 1] = l;
    }
    __syncthreads();
    for (int g2 = 0; g2 < it.wide; ++g2) tree_join<D, T, true>(a, it, g2, t, merge, threadIdx.x);
  }
}

// The spans of 16 columns joined by log-sum-exp, in their order.
template <int D, int T, bool F32>
__global__ __launch_bounds__(kThreads) void tree_merge_kernel(TreeArgs a) {
  constexpr int N = D / 16, U = 8;                      // spans whose loads are on their way at once
  const int groups = tree_counts(a, T).y;
  const TreeGroup* all = reinterpret_cast<const TreeGroup*>(a.plan + sizeof(TreeHeader) + a.items * sizeof(TreeItem));
  for (int at = blockIdx.x; at < a.max_groups * a.merge_tiles; at += gridDim.x) {
    const int t = at % a.merge_tiles;
    typedef int32_t words_t __attribute__((ext_vector_type(8)));
    const words_t raw = load_uniform(reinterpret_cast<const words_t*>(all + at / a.merge_tiles));
    if (at >= groups * a.merge_tiles) break;
    TreeGroup gr;
    __builtin_memcpy(&gr, &raw, sizeof(gr));
    const int c = 16 * (t % T) + (threadIdx.x >> 4), dim = N * (threadIdx.x & 15);
    const int column = (gr.tile * gr.wide * T + t) * 16 + (threadIdx.x >> 4);
    if (t >= gr.wide * T || (column >> a.group_log2) >= gr.n_rows) continue;
    const float* part = a.partials + (gr.part0 + t / T) * tree_partial_floats(D, T);
    const int64_t stride = gr.wide * tree_partial_floats(D, T);
    float m = kNegBig, l = 0.f, o[N] = {};
    for (int s = 0; s < gr.n_parts; s += U) {
      float ms[U], ls[U];
      float4 x[U][N / 4];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        ms[u] = kNegBig;
        ls[u] = 0.f;
#pragma unroll
        for (int i = 0; i < N / 4; ++i) x[u][i] = float4{0.f, 0.f, 0.f, 0.f};
        if (s + u < gr.n_parts) {
          const float* p = part + (s + u) * stride;
          ms[u] = p[16 * T * D + c];
          ls[u] = p[16 * T * (D + 1) + c];
#pragma unroll
          for (int i = 0; i < N / 4; ++i) x[u][i] = *reinterpret_cast<const float4*>(p + c * D + dim + 4 * i);
        }
      }
      float mn = m;
#pragma unroll
      for (int u = 0; u < U; ++u) mn = fmaxf(mn, ms[u]);
      const float f0 = __builtin_amdgcn_exp2f(m - mn);
      l *= f0;
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] *= f0;
      m = mn;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float f = __builtin_amdgcn_exp2f(ms[u] - mn);
        l = fmaf(f, ls[u], l);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
          o[4 * i] = fmaf(f, x[u][i].x, o[4 * i]);
          o[4 * i + 1] = fmaf(f, x[u][i].y, o[4 * i + 1]);
          o[4 * i + 2] = fmaf(f, x[u][i].z, o[4 * i + 2]);
          o[4 * i + 3] = fmaf(f, x[u][i].w, o[4 * i + 3]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = over_sum(o[i], l);
    tree_store<D, F32>(a, gr.q_row0, gr.n_rows, gr.kvh, column, dim, o);
  }
}

// ---------------------------------------------------------------------------

aug_status tree_sizes(const char* who, const aug_attn_shape* s, const aug_tree_batch* b, TreeSizes* z) {
  if (aug_status st = aug::check_shape(s, who); st != AUG_OK) return st;
  if (!b) return aug::fail(AUG_ERR_INVALID, "%s: batch is NULL", who);
  if (b->num_reqs < 0 || b->max_rows < 0 || b->max_blocks < 1)
    return aug::fail(AUG_ERR_INVALID, "%s: %d requests, %d rows, %d columns", who, b->num_reqs, b->max_rows, b->max_blocks);
  if (b->max_draft < 1 || b->max_draft > AUG_MAX_DRAFT)
    return aug::fail(AUG_ERR_INVALID, "%s: max_draft %d (1 to %d)", who, b->max_draft, AUG_MAX_DRAFT);
  if (b->num_reqs > AUG_STEP_MAX_REQS || b->max_blocks > (1 << 20))
    return aug::fail(AUG_ERR_UNSUPPORTED, "%s: %d requests of up to %d blocks (supported: %d, %d)", who, b->num_reqs,
                     b->max_blocks, AUG_STEP_MAX_REQS, 1 << 20);
  const int columns = b->max_draft * (s->num_q_heads / s->num_kv_heads);
  // items that no split makes: a request's columns in tiles (of the widest that it can have, or of 32
  // or 64 if they are fewer)
  const int64_t whole = static_cast<int64_t>(b->num_reqs) * s->num_kv_heads * ((columns + 127) / 128);
  z->items = kTreeTarget + whole;
  z->groups = whole < kTreeTarget ? whole : kTreeTarget;
  const int64_t split = z->items < 2 * kTreeTarget ? z->items : 2 * kTreeTarget;
  // 64 columns a wave: fp4 operands, which cost most to make and fit (310 us with 32, 280 with 64);
  // over fp8 they need more registers than there are (268 us, 32 columns 260)
  z->tiles = columns > 32 && s->kv_dtype == AUG_MXFP4 ? 4 : 2;
  z->parts = split * wide_for(columns, z->tiles);
  // tables too narrow for any request to be split: nothing to merge
  const int64_t units = (static_cast<int64_t>(b->max_blocks) * kBlock + kTreeUnit - 1) / kTreeUnit;
  if (units == 1 || units * wide_for(columns, z->tiles) <= kTreeMinSpan) z->groups = z->parts = 0;
  z->merge_tiles = columns < 128 ? (columns + 15) / 16 : 8;
  if (z->items > (1 << 24))
    return aug::fail(AUG_ERR_UNSUPPORTED, "%s: up to %lld work items", who, (long long)z->items);
  z->plan_bytes = sizeof(TreeHeader) + z->items * sizeof(TreeItem) + z->groups * sizeof(TreeGroup);
  z->workspace_bytes = 16 + z->parts * tree_partial_floats(s->head_dim, z->tiles) * 4;
  return AUG_OK;
}

template <int KVT, int D>
void launch_tree(const TreeArgs& a, const TreeSizes& z, hipStream_t st) {
  const int64_t tiles = z.groups * z.merge_tiles;
  const dim3 merge(static_cast<uint32_t>(tiles < 2048 ? tiles : 2048));
  if constexpr (KVT == KV_F32) {
    hipLaunchKernelGGL((tree_kernel_f32<D>), dim3(z.items), dim3(kThreads), 0, st, a);
    if (tiles) hipLaunchKernelGGL((tree_merge_kernel<D, 2, true>), merge, dim3(kThreads), 0, st, a);
  } else if (z.tiles == 2) {
    hipLaunchKernelGGL((tree_kernel<KVT, D, 2>), dim3(z.items), dim3(kThreads), 0, st, a);
    if (tiles) hipLaunchKernelGGL((tree_merge_kernel<D, 2, false>), merge, dim3(kThreads), 0, st, a);
  } else if constexpr (KVT == KV_FP4) {
    hipLaunchKernelGGL((tree_kernel<KVT, D, 4>), dim3(z.items), dim3(kThreads), 0, st, a);
    if (tiles) hipLaunchKernelGGL((tree_merge_kernel<D, 4, false>), merge, dim3(kThreads), 0, st, a);
  }
}

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) & 15; }

}  // namespace

extern "C" aug_status aug_tree_plan_size(const aug_attn_shape* s, const aug_tree_batch* b, size_t* plan_bytes,
                                         size_t* workspace_bytes) {
  const char* who = "aug_tree_plan_size";
  TreeSizes z;
  if (aug_status st = tree_sizes(who, s, b, &z); st != AUG_OK) return st;
  if (!plan_bytes || !workspace_bytes) return aug::fail(AUG_ERR_INVALID, "%s: NULL pointer", who);
  *plan_bytes = static_cast<size_t>(z.plan_bytes);
  *workspace_bytes = static_cast<size_t>(z.workspace_bytes);
  return AUG_OK;
}

extern "C" aug_status aug_tree_plan(const aug_attn_shape* s, const aug_tree_batch* b, void* plan_dev, size_t plan_bytes,
                                    void* stream) {
  const char* who = "aug_tree_plan";
  TreeSizes z;
  if (aug_status st = tree_sizes(who, s, b, &z); st != AUG_OK) return st;
  if (b->num_reqs == 0 || b->max_rows == 0) return AUG_OK;
  if (!b->q_start || !b->kv_len || !plan_dev) return aug::fail(AUG_ERR_INVALID, "%s: NULL device pointer", who);
  if (misaligned(plan_dev)) return aug::fail(AUG_ERR_INVALID, "%s: the plan must be 16-byte aligned", who);
  if (plan_bytes < static_cast<size_t>(z.plan_bytes))
    return aug::fail(AUG_ERR_NO_SPACE, "%s: plan %zu < %lld bytes", who, plan_bytes, (long long)z.plan_bytes);
  const TreePlanArgs a{b->q_start, b->kv_len, static_cast<char*>(plan_dev), z.items, b->num_reqs, b->max_rows, b->max_blocks,
                       b->max_draft, s->num_kv_heads, s->num_q_heads / s->num_kv_heads, z.tiles};
  const uint32_t lds = (3u * b->num_reqs + 256u * ((b->num_reqs + kPlanThreads - 1) / kPlanThreads)) * sizeof(int32_t) + b->num_reqs * sizeof(uint16_t);
  hipLaunchKernelGGL(tree_plan_kernel, dim3(1), dim3(kPlanThreads), lds, static_cast<hipStream_t>(stream), a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess)
    return aug::fail(AUG_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return AUG_OK;
}

extern "C" aug_status aug_attn_tree(const aug_attn_shape* s, const aug_tree_batch* b, const void* plan_dev, const void* q,
                                    const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                                    int32_t num_pool_blocks, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  const char* who = "aug_attn_tree";
  TreeSizes z;
  if (aug_status st = tree_sizes(who, s, b, &z); st != AUG_OK) return st;
  if (num_pool_blocks < 1) return aug::fail(AUG_ERR_INVALID, "%s: empty pool", who);
  if (b->num_reqs == 0 || b->max_rows == 0) return AUG_OK;
  if (!plan_dev || !q || !k_cache || !v_cache || !b->block_table || !b->seen || !out)
    return aug::fail(AUG_ERR_INVALID, "%s: NULL device pointer", who);
  if (s->kv_dtype == AUG_FP8_E4M3FN && (!k_scale || !v_scale))
    return aug::fail(AUG_ERR_INVALID, "%s: fp8 KV needs k_scale and v_scale", who);
  if (misaligned(plan_dev) || misaligned(q) || misaligned(k_cache) || misaligned(v_cache) || misaligned(out) || misaligned(workspace))
    return aug::fail(AUG_ERR_INVALID, "%s: plan, rows, caches and workspace must be 16-byte aligned", who);
  if (!workspace || workspace_bytes < static_cast<size_t>(z.workspace_bytes))
    return aug::fail(AUG_ERR_NO_SPACE, "%s: workspace %zu < %lld bytes", who, workspace_bytes, (long long)z.workspace_bytes);
  // out may be q: a column's queries are read by the one item that has it, or by its spans, before it is written
  const int64_t bytes = static_cast<int64_t>(b->max_rows) * s->num_q_heads * s->head_dim * (s->q_dtype == AUG_F32 ? 4 : 2);
  if (q != out && aug::overlap({"q", q, bytes}, {"out", out, bytes}))
    return aug::fail(AUG_ERR_INVALID, "%s: q and out overlap and are not the same", who);
  TreeArgs a{};
  a.plan = static_cast<const char*>(plan_dev);
  a.q = q;
  a.k_cache = static_cast<const char*>(k_cache);
  a.v_cache = static_cast<const char*>(v_cache);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.block_table = b->block_table;
  a.seen = b->seen;
  a.out = out;
  a.partials = static_cast<float*>(workspace);
  a.items = z.items;
  a.merge_tiles = z.merge_tiles;
  a.max_groups = static_cast<int32_t>(z.groups);
  a.max_blocks = b->max_blocks;
  a.max_rows = b->max_rows;
  a.reqs_drafts = reqs_drafts_of(b->num_reqs, b->max_draft);
  a.num_pool_blocks = num_pool_blocks;
  a.hq = s->num_q_heads;
  a.hkv = s->num_kv_heads;
  a.group_log2 = __builtin_ctz(static_cast<unsigned>(s->num_q_heads / s->num_kv_heads));
  a.scale_log2 = s->softmax_scale * kLog2e;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (s->kv_dtype == AUG_F32 && s->head_dim == 64) launch_tree<KV_F32, 64>(a, z, st);
  else if (s->kv_dtype == AUG_F32) launch_tree<KV_F32, 128>(a, z, st);
  else if (s->kv_dtype == AUG_BF16 && s->head_dim == 64) launch_tree<KV_BF16, 64>(a, z, st);
  else if (s->kv_dtype == AUG_BF16) launch_tree<KV_BF16, 128>(a, z, st);
  else if (s->kv_dtype == AUG_FP8_E4M3FN) launch_tree<KV_FP8, 128>(a, z, st);
  else launch_tree<KV_FP4, 128>(a, z, st);
  if (hipError_t e = hipGetLastError(); e != hipSuccess)
    return aug::fail(AUG_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return AUG_OK;
}
