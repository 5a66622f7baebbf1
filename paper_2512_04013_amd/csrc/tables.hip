// The tables of a step whose lengths are on the GPU: blocks given back and taken,
// row offsets, positions, slots and draft masks.
//
// Everything about requests follows from prefix sums over them: of rows (q_start), of
// blocks that come back and of blocks that are asked for. With `count` free blocks
// before the call and `back` coming back, block k to come back goes to place
// count + back - 1 - k of the stack, and block k to be taken comes from that place:
// for k < back it is the one that came back as k-th, read where its request held
// it, so nothing that one workgroup writes is read by another.
//
// One launch: every workgroup makes all sums for itself (12 bytes a request, from L2) and
// then takes its share of the blocks that come back, of those that are taken, and of the
// rows; whose a block or row is, is looked up in the sums. What the sums were made from
// (held, free_count, and kv_len, which may be the array of context lengths) is overwritten by the
// workgroup that finishes last, when all others have read it.
//
// Bound by the chain of loads: lengths, sums, table or stack, stores. 64 requests of 8 drafts:
// 6.3 us; 2000 of up to 32, 11.7 (with a workgroup a request, its rows behind its blocks: 42).

#include <hip/hip_runtime.h>

#include <cstdint>

#include "aug.h"
#include "checks.h"
#include "plan_format.h"
#include "status.h"

namespace {

using aug::kBlock;

constexpr int kEach = 4;               // requests of a thread, at most
constexpr int kFew = 1024;             // requests up to which a workgroup has kFew / kEach threads

// Sums of a and b over the threads before this one, in place; totals. Two barriers.
template <int THREADS>
__device__ __forceinline__ void sums_before(uint64_t& a, uint64_t& b, uint64_t* waves, uint64_t* a_total, uint64_t* b_total) {
  constexpr int W = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t x = a, y = b;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t ox = __shfl_up(static_cast<unsigned long long>(x), d), oy = __shfl_up(static_cast<unsigned long long>(y), d);
    if (lane >= d) {
      x += ox;
      y += oy;
    }
  }
  __syncthreads();
  if (lane == 63) {
    waves[wave] = x;
    waves[W + wave] = y;
  }
  __syncthreads();
  a = x - a;
  b = y - b;
  *a_total = *b_total = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    if (w < wave) {
      a += waves[w];
      b += waves[W + w];
    }
    *a_total += waves[w];
    *b_total += waves[W + w];
  }
}

__device__ __forceinline__ uint32_t cut(uint64_t v) { return v > ~0u ? ~0u : static_cast<uint32_t>(v); }

// The last of n ascending values that is not above x; values[0] is not.
__device__ __forceinline__ int last_not_above(const uint32_t* values, int n, uint32_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (values[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

struct Request {
  int32_t ctx, rows, held, need;
  bool valid;
};

__device__ __forceinline__ Request load_request(const aug_step_tables_args& a, int r) {
  Request q;
  const int32_t n = a.q_len[r];
  q.ctx = a.ctx_len[r];
  q.held = a.held[r];
  q.rows = max(n, 0);
  const int64_t end = static_cast<int64_t>(q.ctx) + n;
  const int64_t need = (end + kBlock - 1) / kBlock;
  q.valid = q.ctx >= 0 && n >= 0 && need <= a.max_blocks && q.held >= 0 && q.held <= a.max_blocks &&
            (a.max_draft == 0 || n <= a.max_draft);
  q.need = q.valid ? static_cast<int32_t>(need) : 0;
  return q;
}

// LDS, per request: first row (cut to max_rows), blocks that came back before it,
// blocks asked for before it.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void tables_kernel(aug_step_tables_args a) {
  extern __shared__ uint32_t lds[];
  __shared__ uint64_t waves[2 * (THREADS / 64)];
  __shared__ int32_t last;
  const int n = a.num_reqs, tid = threadIdx.x;
  uint32_t* start = lds;              // [n + 1]
  uint32_t* back_before = lds + n + 1;
  uint32_t* asked_before = lds + 2 * n + 1;
  const int per = (n + THREADS - 1) / THREADS;
  const int r0 = min(tid * per, n), r1 = min(r0 + per, n);
  const uint32_t cap = static_cast<uint32_t>(a.max_rows);
  const int32_t count0 = min(max(*a.free_count, 0), a.num_pool_blocks);

  Request mine[kEach];
  uint64_t at = 0, unused = 0, rows_sum, unused_sum;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    mine[i] = r0 + i < r1 ? load_request(a, r0 + i) : Request{};
    at += mine[i].rows;
  }
  sums_before<THREADS>(at, unused, waves, &rows_sum, &unused_sum);
  const int32_t rows_total = static_cast<int32_t>(rows_sum < cap ? rows_sum : cap);
  uint64_t back = 0, ask = 0, back_sum, ask_sum;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (r0 + i >= r1) break;
    const uint32_t first = static_cast<uint32_t>(at < cap ? at : cap);
    start[r0 + i] = first;
    at += mine[i].rows;
    mine[i].valid = mine[i].valid && static_cast<uint64_t>(first) + mine[i].rows <= cap;
    back += mine[i].valid ? max(mine[i].held - mine[i].need, 0) : 0;
    ask += mine[i].valid ? max(mine[i].need - mine[i].held, 0) : 0;
  }
  if (tid == 0) start[n] = rows_total;
  sums_before<THREADS>(back, ask, waves, &back_sum, &ask_sum);
  const uint32_t back_total = cut(back_sum);
  // blocks on the stack once all have come back
  const uint32_t avail = static_cast<uint32_t>(min(count0 + back_sum, static_cast<uint64_t>(a.num_pool_blocks)));
  uint32_t taken = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    if (r0 + i >= r1) break;
    back_before[r0 + i] = cut(back);
    asked_before[r0 + i] = cut(ask);
    back += mine[i].valid ? max(mine[i].held - mine[i].need, 0) : 0;
    const uint32_t take = mine[i].valid ? max(mine[i].need - mine[i].held, 0) : 0;
    ask += take;
    if (take > 0 && ask <= avail) taken = static_cast<uint32_t>(ask);
  }
  // the last request that got blocks got all that were asked for up to it
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) taken = max(taken, static_cast<uint32_t>(__shfl_xor(taken, d)));
  __syncthreads();
  if ((tid & 63) == 0) waves[tid >> 6] = taken;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) taken = max(taken, static_cast<uint32_t>(waves[w]));

  const auto outcome = [&](int r, const Request& q) {
    if (!q.valid || static_cast<uint64_t>(start[r]) + q.rows > cap) return AUG_STEP_INVALID;
    return q.need > q.held && static_cast<uint64_t>(asked_before[r]) + (q.need - q.held) > avail ? AUG_STEP_NO_BLOCKS : AUG_STEP_OK;
  };
  const auto table_of = [&](int r) { return a.block_table + static_cast<int64_t>(r) * a.max_blocks; };
  const auto place_of = [&](uint32_t nth) { return static_cast<int64_t>(count0) + back_total - 1 - nth; };
  const auto in_stack = [&](int64_t place) { return place >= 0 && place < a.num_pool_blocks; };
  // the block that came back as nth
  const auto given = [&](uint32_t nth) {
    const int r = last_not_above(back_before, n, nth);
    const int64_t col = static_cast<int64_t>(load_request(a, r).need) + (nth - back_before[r]);
    return col < a.max_blocks ? table_of(r)[col] : -1;
  };
  // the block that is taken as nth
  const auto block = [&](uint32_t nth) {
    if (nth < back_total) return given(nth);
    const int64_t place = place_of(nth);
    return in_stack(place) ? a.free_ids[place] : -1;
  };
  // the block of a column that the request has from now on
  const auto column = [&](int r, const Request& q, int64_t col) {
    return col < q.held ? table_of(r)[col] : block(asked_before[r] + static_cast<uint32_t>(col - q.held));
  };

  const uint32_t threads = gridDim.x * THREADS, thread = blockIdx.x * THREADS + tid;
  for (uint64_t nth = thread; nth < back_total; nth += threads) {
    const int64_t place = place_of(static_cast<uint32_t>(nth));
    if (in_stack(place)) a.free_ids[place] = given(static_cast<uint32_t>(nth));
  }
  for (uint64_t nth = thread; nth < taken; nth += threads) {
    const int r = last_not_above(asked_before, n, static_cast<uint32_t>(nth));
    const int64_t col = static_cast<int64_t>(a.held[r]) + static_cast<uint32_t>(nth - asked_before[r]);
    if (col < a.max_blocks) table_of(r)[col] = block(static_cast<uint32_t>(nth));
  }
  for (uint32_t r = thread; r < static_cast<uint32_t>(n); r += threads) {
    const Request q = load_request(a, r);
    const aug_step_state st = outcome(r, q);
    a.q_start[r] = static_cast<int32_t>(start[r]);
    a.state[r] = st;
  }
  if (thread == 0) a.q_start[n] = rows_total;

  if (a.max_draft == 0) {
    for (uint32_t i = thread; i < static_cast<uint32_t>(rows_total); i += threads) {
      const int r = last_not_above(start, n, i);
      const Request q = load_request(a, r);
      const bool ok = outcome(r, q) == AUG_STEP_OK;
      const int64_t token = static_cast<int64_t>(q.ctx) + (i - start[r]);
      a.slots[i] = ok ? static_cast<int64_t>(column(r, q, token / kBlock)) * kBlock + token % kBlock : -1;
      a.positions[i] = ok ? static_cast<int32_t>(token) : 0;
    }
  } else {
    // a wave a request: lane i has its row i
    const int lane = tid & 63;
    for (int r = static_cast<int>(thread >> 6); r < n; r += static_cast<int>(threads >> 6)) {
      const Request q = load_request(a, r);
      const bool ok = outcome(r, q) == AUG_STEP_OK;
      const int first = static_cast<int>(start[r]), rows = static_cast<int>(start[r + 1]) - first;
      if (!ok) {                                       // may be more rows than a wave has lanes
        for (int i = lane; i < rows; i += 64) {
          a.slots[first + i] = -1;
          a.seen[first + i] = 0;
          a.positions[first + i] = 0;
        }
        continue;
      }
      // Row i sees itself and what its parent sees. Six rounds of looking twice as
      // far up reach the root of any path of 64.
      int up = lane - 1;
      if (a.parents) up = lane < rows ? a.parents[first + lane] : -1;
      if (up < 0 || up >= lane) up = -1;
      uint64_t m = 1ull << lane;
#pragma unroll
      for (int d = 0; d < 6; ++d) {
        const int from = max(up, 0);
        const uint64_t om = static_cast<uint64_t>(__shfl(static_cast<unsigned long long>(m), from));
        const int ou = __shfl(up, from);
        if (up >= 0) {
          m |= om;
          up = ou;
        }
      }
      if (lane >= rows) continue;
      const int64_t token = static_cast<int64_t>(q.ctx) + lane;
      a.slots[first + lane] = static_cast<int64_t>(column(r, q, token / kBlock)) * kBlock + token % kBlock;
      a.seen[first + lane] = m;
      a.positions[first + lane] = q.ctx + __popcll(m) - 1;
    }
  }

  __syncthreads();
  if (tid == 0) {
    int32_t* done = static_cast<int32_t*>(a.scratch);
    last = __hip_atomic_fetch_add(done, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<int32_t>(gridDim.x) - 1;
    if (last) __hip_atomic_store(done, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return;
  for (int r = tid; r < n; r += THREADS) {
    const Request q = load_request(a, r);
    const bool ok = outcome(r, q) == AUG_STEP_OK;
    a.kv_len[r] = ok ? q.ctx + q.rows : 0;
    if (ok) a.held[r] = q.need;
  }
  if (tid == 0) *a.free_count = static_cast<int32_t>(avail - taken);
}

// Enough workgroups for a wave a request, or a thread a row, up to one a compute unit.
template <int THREADS>
void launch(const aug_step_tables_args& t, hipStream_t st) {
  const int64_t threads = t.max_draft > 0 ? int64_t{64} * t.num_reqs : t.max_rows > t.num_reqs ? t.max_rows : t.num_reqs;
  const int64_t groups = (threads + THREADS - 1) / THREADS;
  const uint32_t lds = (3u * t.num_reqs + 1) * sizeof(uint32_t);
  hipLaunchKernelGGL((tables_kernel<THREADS>), dim3(static_cast<uint32_t>(groups < 256 ? groups : 256)), dim3(THREADS), lds, st, t);
}

}  // namespace

extern "C" aug_status aug_step_tables(const aug_step_tables_args* t, void* stream) {
  const char* who = "aug_step_tables";
  if (!t) return aug::fail(AUG_ERR_INVALID, "%s: arguments are NULL", who);
  if (t->reserved != 0) return aug::fail(AUG_ERR_INVALID, "%s: the reserved field must be zero", who);
  if (t->num_reqs < 0 || t->max_rows < 0 || t->max_rows == INT32_MAX || t->max_blocks < 1 || t->num_pool_blocks < 1)
    return aug::fail(AUG_ERR_INVALID, "%s: %d requests, %d rows, %d columns, %d blocks", who, t->num_reqs, t->max_rows,
                     t->max_blocks, t->num_pool_blocks);
  if (t->max_draft < 0 || t->max_draft > AUG_MAX_DRAFT)
    return aug::fail(AUG_ERR_INVALID, "%s: max_draft %d (0 to %d)", who, t->max_draft, AUG_MAX_DRAFT);
  if (t->num_reqs > AUG_STEP_MAX_REQS || t->max_blocks > (1 << 20))
    return aug::fail(AUG_ERR_UNSUPPORTED, "%s: %d requests of up to %d blocks (supported: %d, %d)", who, t->num_reqs,
                     t->max_blocks, AUG_STEP_MAX_REQS, 1 << 20);
  if (t->max_draft == 0 && (t->parents || t->seen))
    return aug::fail(AUG_ERR_INVALID, "%s: parents and masks need max_draft", who);
  if (t->num_reqs == 0) return AUG_OK;
  if (!t->ctx_len || !t->q_len || !t->block_table || !t->held || !t->free_ids || !t->free_count || !t->q_start ||
      !t->kv_len || !t->state || !t->scratch)
    return aug::fail(AUG_ERR_INVALID, "%s: NULL device pointer", who);
  if (t->max_rows > 0 && (!t->positions || !t->slots || (t->max_draft > 0 && !t->seen)))
    return aug::fail(AUG_ERR_INVALID, "%s: NULL device pointer", who);
  const int64_t reqs = t->num_reqs, rows = t->max_rows;
  const aug::Span read[] = {{"ctx_len", t->ctx_len, 4 * reqs}, {"q_len", t->q_len, 4 * reqs}, {"parents", t->parents, 4 * rows}};
  const aug::Span written[] = {{"block_table", t->block_table, 4 * reqs * t->max_blocks}, {"held", t->held, 4 * reqs},
                          {"free_ids", t->free_ids, int64_t{4} * t->num_pool_blocks}, {"free_count", t->free_count, 4},
                          {"q_start", t->q_start, 4 * (reqs + 1)}, {"kv_len", t->kv_len, 4 * reqs}, {"state", t->state, 4 * reqs},
                          {"positions", t->positions, 4 * rows}, {"slots", t->slots, 8 * rows}, {"seen", t->seen, 8 * rows},
                          {"scratch", t->scratch, AUG_STEP_SCRATCH_BYTES}};
  for (const aug::Span& r : read)
    for (const aug::Span& w : written) {
      const bool same = &r == read && w.p == t->kv_len && r.p == w.p;      // kv_len is written behind the last read
      if (aug::overlap(r, w) && !same) return aug::fail(AUG_ERR_INVALID, "%s: %s overlaps %s", who, r.name, w.name);
    }
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (t->num_reqs <= kFew) launch<kFew / kEach>(*t, st);
  else launch<AUG_STEP_MAX_REQS / kEach>(*t, st);
  if (hipError_t e = hipGetLastError(); e != hipSuccess)
    return aug::fail(AUG_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return AUG_OK;
}
