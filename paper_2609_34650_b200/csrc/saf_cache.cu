// Plan of a step on a paged cache: pages by length, rows, slots, positions and ancestor sets of the new tokens.
//
// need = ceil((ctx + new) / page); requests give pages back beyond it and pop what they lack.  Three sums over the requests (rows,
// pages asked for, pages given back) place everything else, so every block forms them for itself, from the same inputs, and
// takes its share of the rows and pages.  Popped page number k is entry total-1-k of the stack on which the given pages lie; that
// entry is looked up where it comes from (the old stack, or the table of the request that gives it), so no block waits for another's
// writes.  Counts and held pages, which a caller may update in place, are written by the last block to have read them.
// Latency bounds it: one launch, three scans.
#include "ptx.cuh"
#include "saf_internal.h"

#include <algorithm>

namespace saf {
namespace {

constexpr int PLAN_THREADS = 256;
constexpr int PLAN_WARPS = PLAN_THREADS / 32;

// Exclusive sum of v over the block's threads; *total gets the sum.  `red`: PLAN_WARPS + 1 words.
__device__ __forceinline__ long long block_scan(long long v, long long* red, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 31) red[warp] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < PLAN_WARPS; ++w) {
    const long long s = red[w];
    if (w < warp) before += s;
    all += s;
  }
  *total = all;
  return before + x - v;
}

// First r with a[r] > x (a: inclusive sums, not decreasing); n if none.
__device__ __forceinline__ int upper(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] > x) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

__global__ void __launch_bounds__(PLAN_THREADS) saf_cache_plan_kernel(CachePlanParams p) {
  extern __shared__ int sm[];
  __shared__ long long red[PLAN_WARPS];
  __shared__ long long taken_s;
  __shared__ int last_s;
  const int R = p.R, N = p.N;
  int* s_end = sm;                  // rows up to and with request r, at most N
  int* s_ctx = sm + R;
  int* s_held = sm + 2 * R;
  int* s_need = sm + 3 * R;
  int* s_grow = sm + 4 * R;         // inclusive sum of pages asked for
  int* s_give = sm + 5 * R;         // inclusive sum of pages given back
  int* s_flag = sm + 6 * R;         // bit 0: cannot be served as given, bit 1: more new tokens than a tree may have
  pdl_wait();
  pdl_launch_dependents();
  const int per = (R + PLAN_THREADS - 1) / PLAN_THREADS;
  const int r0 = min(R, static_cast<int>(threadIdx.x) * per), r1 = min(R, r0 + per);
  long long sum = 0, total;
  for (int r = r0; r < r1; ++r) sum += max(p.new_lens[r], 0);
  long long end = block_scan(sum, red, &total);
  long long asked = 0, given = 0;
  for (int r = r0; r < r1; ++r) {
    const int ctx = p.ctx_lens[r], nw = p.new_lens[r];
    const int held = min(max(p.held_in[r], 0), p.max_pages);
    end += max(nw, 0);
    const long long need = (static_cast<long long>(max(ctx, 0)) + max(nw, 0) + p.page_size - 1) / p.page_size;
    const bool wide = p.parents && nw > 64;
    const bool bad = ctx < 0 || nw < 0 || need > p.max_pages || (end > N && nw > 0) || wide;
    const int want = bad ? held : static_cast<int>(need);
    s_end[r] = static_cast<int>(min(end, static_cast<long long>(N)));
    s_ctx[r] = max(ctx, 0);
    s_held[r] = held;
    s_need[r] = want;
    s_flag[r] = (bad ? 1 : 0) | (wide ? 2 : 0);
    asked += max(want - held, 0);
    given += max(held - want, 0);
  }
  // (both sums are below 2^31: R * max_pages is)
  long long both = block_scan((asked << 32) | given, red, &total);
  const int count = min(max(*p.free_count_in, 0), p.n_pages);
  const int give_all = static_cast<int>(total & 0xffffffffll);
  const int stock = min(count + give_all, p.n_pages);      // (a sound state never holds more than n_pages)
  int grow_c = static_cast<int>(both >> 32), give_c = static_cast<int>(both & 0xffffffffll);
  if (threadIdx.x == 0) taken_s = 0;
  __syncthreads();
  int mine = 0;
  for (int r = r0; r < r1; ++r) {
    const int d = s_need[r] - s_held[r];
    grow_c += max(d, 0);
    give_c += max(-d, 0);
    s_grow[r] = grow_c;
    s_give[r] = give_c;
    if (d > 0 && grow_c <= stock) mine = grow_c;           // served: those whose sum still fits, a prefix of those that ask
  }
  if (mine) atomicMax(&taken_s, static_cast<long long>(mine));
  __syncthreads();
  const int taken = static_cast<int>(taken_s);
  const int left = stock - taken;
  // entry x of the stack with the given pages on top
  auto stack = [&](int x) -> int {
    if (x < count) return p.free_list[x];
    const int g = x - count, r = upper(s_give, R, g);
    if (r >= R) return 0;
    const int before = r ? s_give[r - 1] : 0;
    return p.block_table[static_cast<long long>(r) * p.max_pages + s_need[r] + (g - before)];
  };
  auto ok = [&](int r) { return !(s_flag[r] & 1) && (s_need[r] <= s_held[r] || s_grow[r] <= stock); };
  const int tid = blockIdx.x * PLAN_THREADS + threadIdx.x, nthr = gridDim.x * PLAN_THREADS;
  for (int k = tid; k < taken; k += nthr) {
    const int r = upper(s_grow, R, k);
    const int at = s_held[r] + k - (r ? s_grow[r - 1] : 0);
    p.block_table[static_cast<long long>(r) * p.max_pages + at] = stack(stock - 1 - k);
  }
  for (int x = count + tid; x < left; x += nthr) p.free_list[x] = stack(x);
  for (int r = tid; r < R; r += nthr) {
    const int nw = max(p.new_lens[r], 0);
    const bool fine = ok(r);
    p.new_offsets[r + 1] = s_end[r];
    p.kv_lens[r] = fine ? s_ctx[r] + nw : 0;
    p.missing[r] = (s_flag[r] & 1) ? -1 : fine ? 0 : s_need[r] - s_held[r];
  }
  if (tid == 0) p.new_offsets[0] = 0;
  const int rows = s_end[R - 1];
  for (int n = tid; n < N; n += nthr) {
    int slot = -1, pos = 0;
    if (n < rows) {
      const int r = upper(s_end, R, n);
      const int i = n - (r ? s_end[r - 1] : 0);
      const int at = s_ctx[r] + i;
      pos = at;
      if (ok(r)) {
        const int col = at / p.page_size;
        const int page = col < s_held[r] ? p.block_table[static_cast<long long>(r) * p.max_pages + col]
                                         : stack(stock - 1 - ((r ? s_grow[r - 1] : 0) + col - s_held[r]));
        slot = page * p.page_size + at - col * p.page_size;
      }
    }
    p.slots[n] = slot;
    if (!p.parents || n >= rows) {
      p.positions[n] = pos;
      if (p.parents) p.tree_masks[n] = 0;
    }
  }
  if (p.parents) {
    // A warp a request, two tokens a lane: sets and parents doubled six times reach 64 levels.
    const int lane = threadIdx.x & 31;
    for (int r = tid >> 5; r < R; r += nthr >> 5) {
      const int a = r ? s_end[r - 1] : 0, n = s_end[r] - a;
      if (s_flag[r] & 2) {
        for (int i = lane; i < n; i += 32) {
          p.positions[a + i] = s_ctx[r];
          p.tree_masks[a + i] = 0;
        }
        continue;
      }
      unsigned long long set[2];
      int up[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = lane + 32 * k;
        set[k] = 1ull << i;
        up[k] = i < n ? p.parents[a + i] : -1;
        if (up[k] < 0 || up[k] >= i) up[k] = -1;
      }
      for (int level = 0; level < 6; ++level) {
        unsigned long long nset[2];
        int nup[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int src = up[k] & 31;
          const unsigned long long lo = __shfl_sync(0xffffffffu, set[0], src), hi = __shfl_sync(0xffffffffu, set[1], src);
          const int ulo = __shfl_sync(0xffffffffu, up[0], src), uhi = __shfl_sync(0xffffffffu, up[1], src);
          nset[k] = up[k] < 0 ? set[k] : set[k] | (up[k] < 32 ? lo : hi);
          nup[k] = up[k] < 0 ? -1 : up[k] < 32 ? ulo : uhi;
        }
        set[0] = nset[0]; set[1] = nset[1];
        up[0] = nup[0]; up[1] = nup[1];
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int i = lane + 32 * k;
        if (i < n) {
          p.tree_masks[a + i] = set[k];
          p.positions[a + i] = s_ctx[r] + __popcll(set[k]) - 1;
        }
      }
    }
  }
  // everything that reads held_in and free_count_in has done so
  __syncthreads();
  if (threadIdx.x == 0) last_s = gridDim.x == 1 ? 1 : atomicAdd(p.arrived, 1) == static_cast<int>(gridDim.x) - 1;
  __syncthreads();
  if (!last_s) return;
  for (int r = threadIdx.x; r < R; r += PLAN_THREADS) p.held_out[r] = ok(r) ? s_need[r] : s_held[r];
  if (threadIdx.x == 0) {
    *p.free_count_out = left;
    if (gridDim.x > 1) *p.arrived = 0;
  }
}

}  // namespace

cudaError_t launch_cache_plan(const CachePlanParams& p, int num_sms, cudaStream_t st) {
  // a thread for each row, a warp for each drafted tree (256 trees of up to 32 tokens: 7.4 us; 2048 rows or 64 trees a block of 512 threads 12.6)
  const long long by_rows = (static_cast<long long>(p.N) + PLAN_THREADS - 1) / PLAN_THREADS, by_trees = p.parents ? (p.R + PLAN_WARPS - 1) / PLAN_WARPS : 1;
  const int grid = static_cast<int>(std::min<long long>(num_sms, std::max(by_rows, by_trees)));
  const size_t smem = static_cast<size_t>(7) * p.R * sizeof(int);
  if (smem > 40 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(saf_cache_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(PDL_REST, saf_cache_plan_kernel, grid, PLAN_THREADS, smem, st, p);
}

}  // namespace saf
