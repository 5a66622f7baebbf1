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
// One launch: every workgroup makes all sums for itself (12 bytes a request, from L2)
// and then writes its own requests' blocks and rows. What the sums were made from
// (held, free_count) is overwritten by the workgroup that finishes last, when all
// others have read it.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "aug.h"
#include "plan_format.h"
#include "status.h"

namespace {

using aug::kBlock;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

// Sum of v over the threads before this one; *total over all of them. Two barriers.
__device__ __forceinline__ uint32_t block_before(uint32_t v, uint32_t* waves, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t upto = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  uint32_t before = upto - v, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += waves[w];
    sum += waves[w];
  }
  *total = sum;
  return before;
}

// Sums stay below 2^32: rows are cut to max_rows + 1 each and saturate, blocks are at most
// 4096 * 2^20 - 1 (a request that asks for 2^20 of a table of 2^20 holds none).
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return a + b < a ? ~0u : a + b; }

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
// blocks asked for up to and with it.
__global__ __launch_bounds__(kThreads) void tables_kernel(aug_step_tables_args a) {
  extern __shared__ uint32_t lds[];
  __shared__ uint32_t waves[kWaves];
  __shared__ int32_t last;
  const int n = a.num_reqs, tid = threadIdx.x;
  uint32_t* start = lds;              // [n + 1]
  uint32_t* back_before = lds + n + 1;
  uint32_t* asked = lds + 2 * n + 1;
  const int per = (n + kThreads - 1) / kThreads;
  const int r0 = min(tid * per, n), r1 = min(r0 + per, n);
  const uint32_t cap = static_cast<uint32_t>(a.max_rows);
  const int32_t count0 = min(max(*a.free_count, 0), a.num_pool_blocks);

  uint32_t rows = 0;
  for (int r = r0; r < r1; ++r) {
    const uint32_t q = min(static_cast<uint32_t>(max(a.q_len[r], 0)), cap + 1);
    rows = min(rows + q, cap + 1);   // at most 2^32 - 1, as cap < 2^31
  }
  // 256 sums of up to 2^31 would not fit: they are scanned a half at a time
  uint32_t high_total, low_total;
  const uint32_t high = block_before(rows >> 16, waves, &high_total);
  const uint32_t low = block_before(rows & 0xFFFFu, waves, &low_total);
  const auto joined = [&](uint32_t h, uint32_t l) {
    const uint64_t s = (static_cast<uint64_t>(h) << 16) + l;
    return static_cast<uint32_t>(s > cap + 1ull ? cap + 1ull : s);
  };
  uint32_t at = joined(high, low);
  const uint32_t rows_total = min(joined(high_total, low_total), cap);
  uint32_t back = 0, ask = 0;
  for (int r = r0; r < r1; ++r) {
    const Request q = load_request(a, r);
    start[r] = min(at, cap);
    at = min(at + min(static_cast<uint32_t>(q.rows), cap + 1), cap + 1);
    const bool valid = q.valid && start[r] + static_cast<uint32_t>(q.rows) <= cap;
    back += valid ? max(q.held - q.need, 0) : 0;
    ask = add_sat(ask, valid ? max(q.need - q.held, 0) : 0);
  }
  if (tid == 0) start[n] = rows_total;
  uint32_t back_total, ask_high, ask_low;
  uint32_t b = block_before(back, waves, &back_total);
  const uint32_t ah = block_before(ask >> 16, waves, &ask_high);
  const uint32_t al = block_before(ask & 0xFFFFu, waves, &ask_low);
  const uint64_t before = (static_cast<uint64_t>(ah) << 16) + al;
  uint32_t k = before > ~0u ? ~0u : static_cast<uint32_t>(before);
  // blocks on the stack once all have come back
  const uint32_t avail = min(static_cast<uint32_t>(count0) + back_total, static_cast<uint32_t>(a.num_pool_blocks));
  uint32_t taken = 0;
  for (int r = r0; r < r1; ++r) {
    const Request q = load_request(a, r);
    const bool valid = q.valid && start[r] + static_cast<uint32_t>(q.rows) <= cap;
    back_before[r] = b;
    b += valid ? max(q.held - q.need, 0) : 0;
    const uint32_t take = valid ? max(q.need - q.held, 0) : 0;
    k = add_sat(k, take);
    asked[r] = k;
    if (take > 0 && k <= avail) taken = k;
  }
  // the last request that got blocks got all that were asked for up to it
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) taken = max(taken, static_cast<uint32_t>(__shfl_xor(taken, d)));
  __syncthreads();
  if ((tid & 63) == 0) waves[tid >> 6] = taken;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) taken = max(taken, waves[w]);

  const auto outcome = [&](int r, const Request& q) {
    if (!q.valid || start[r] + static_cast<uint32_t>(q.rows) > cap) return AUG_STEP_INVALID;
    return q.need > q.held && asked[r] > avail ? AUG_STEP_NO_BLOCKS : AUG_STEP_OK;
  };

  for (int r = blockIdx.x; r < n; r += gridDim.x) {
    const Request q = load_request(a, r);
    const aug_step_state st = outcome(r, q);
    int32_t* table = a.block_table + static_cast<int64_t>(r) * a.max_blocks;
    if (st == AUG_STEP_OK) {
      for (int j = q.need + tid; j < q.held; j += kThreads) {
        const int64_t place = static_cast<int64_t>(count0) + back_total - 1 - (back_before[r] + (j - q.need));
        if (place >= 0 && place < a.num_pool_blocks) a.free_ids[place] = table[j];
      }
      for (int j = q.held + tid; j < q.need; j += kThreads) {
        const uint32_t nth = asked[r] - (q.need - q.held) + (j - q.held);
        if (nth < back_total) {
          // the request that gave it back: the last one with back_before <= nth that gave any
          int lo = 0, hi = n - 1;
          while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (back_before[mid] <= nth) lo = mid; else hi = mid - 1;
          }
          const Request from = load_request(a, lo);
          const int64_t col = static_cast<int64_t>(from.need) + (nth - back_before[lo]);
          table[j] = col < a.max_blocks ? a.block_table[static_cast<int64_t>(lo) * a.max_blocks + col] : -1;
        } else {
          const int64_t place = static_cast<int64_t>(count0) + back_total - 1 - nth;
          table[j] = place >= 0 && place < a.num_pool_blocks ? a.free_ids[place] : -1;
        }
      }
    }
    const int32_t first = static_cast<int32_t>(start[r]), next = static_cast<int32_t>(start[r + 1]);
    if (tid == 0) {
      a.q_start[r] = first;
      a.kv_len[r] = st == AUG_STEP_OK ? q.ctx + q.rows : 0;
      a.state[r] = st;
    }
    __syncthreads();      // the table's new entries
    const int rows_here = next - first;
    for (int i = tid; i < rows_here; i += kThreads) {
      const int64_t token = static_cast<int64_t>(q.ctx) + i;
      a.slots[first + i] = st == AUG_STEP_OK ? static_cast<int64_t>(table[token / kBlock]) * kBlock + token % kBlock : -1;
      if (a.max_draft == 0) a.positions[first + i] = st == AUG_STEP_OK ? q.ctx + i : 0;
    }
    if (a.max_draft > 0) {
      if (st != AUG_STEP_OK) {
        for (int i = tid; i < rows_here; i += kThreads) {
          a.seen[first + i] = 0;
          a.positions[first + i] = 0;
        }
      } else if (tid < 64) {
        // Row `tid` sees itself and what its parent sees. Six rounds of looking twice as
        // far up reach the root of any path of 64.
        int up = tid - 1;
        if (a.parents) up = tid < rows_here ? a.parents[first + tid] : -1;
        if (up < 0 || up >= tid) up = -1;
        uint64_t m = 1ull << tid;
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
        if (tid < rows_here) {
          a.seen[first + tid] = m;
          a.positions[first + tid] = q.ctx + __popcll(m) - 1;
        }
      }
    }
  }
  if (blockIdx.x == 0 && tid == 0) a.q_start[n] = static_cast<int32_t>(rows_total);

  __syncthreads();
  if (tid == 0) {
    int32_t* done = static_cast<int32_t*>(a.scratch);
    last = __hip_atomic_fetch_add(done, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == static_cast<int32_t>(gridDim.x) - 1;
    if (last) __hip_atomic_store(done, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return;
  for (int r = tid; r < n; r += kThreads) {
    const Request q = load_request(a, r);
    if (outcome(r, q) == AUG_STEP_OK) a.held[r] = q.need;
  }
  if (tid == 0) *a.free_count = static_cast<int32_t>(avail - taken);
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
  const uint32_t lds = (3u * t->num_reqs + 1) * sizeof(uint32_t);
  const int grid = t->num_reqs < 1024 ? t->num_reqs : 1024;
  hipLaunchKernelGGL(tables_kernel, dim3(grid), dim3(kThreads), lds, static_cast<hipStream_t>(stream), *t);
  if (hipError_t e = hipGetLastError(); e != hipSuccess)
    return aug::fail(AUG_ERR_HIP, "%s: launch failed: %s", who, hipGetErrorString(e));
  return AUG_OK;
}
