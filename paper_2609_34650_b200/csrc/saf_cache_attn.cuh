// What the kernels of the attention over a paged cache share: the line of all tiles and its cutting into runs, and the joining of
// units that lie in several runs.
#pragma once
#include <algorithm>
#include <cuda_bf16.h>

#include "ptx.cuh"
#include "saf_internal.h"

namespace saf {
namespace {

// Scores, maxima and references are kept in powers of 16: log16(e) is below one, so that every finite fp32 score stays finite (alpha + rho of keys
// that mask may be the type's lowest value), and a score in powers of two is four times as many, without rounding.
constexpr float LOG16E = 1.4426950408889634f / 4, LN2 = 0.6931471805599453f;
__device__ __forceinline__ float ex16(float x) { return ex2_approx(4.0f * x); }
__device__ __forceinline__ float natural_lse(float m, float l) { return fmaf(m, 4.0f * LN2, log2f(l) * LN2); }

// Where a run stands: a unit, and its place on the line of all tiles.
struct Unit {
  int start;                        // of the unit's first tile on the line
  int r, hk, rt;                    // request, cached head, row tile
  int first, many, len;             // the request's first row, rows that are computed, tokens in its cache that rows may see
  int ctx;                          // tokens that were cached before the step: place of the first new one
  int tiles, row_tiles, pitch;      // (pitch: places that a unit takes, 0: its tiles)
};

__device__ __forceinline__ bool has_keys(const CacheAttnParams& p, int hk) { return (p.with_keys[hk >> 5] >> (hk & 31)) & 1; }

template <int KT, int ROWS>
__device__ __forceinline__ void set_request(const CacheAttnParams& p, Unit& u, int first, int last, int len) {
  // New tokens that no row can see, behind the 64th or the last row (nor more of them than that before the cache begins), are left out.
  u.first = min(max(first, 0), p.N);
  const int n = max(last, u.first) - u.first, there = min(n, p.N - u.first);
  u.many = min(there, p.max_new);
  u.len = min(max(len, 0), p.max_len);
  u.ctx = max(u.len - n, -64);
  u.len = max(min(u.len, u.ctx + min(there, 64)), 0);
  u.row_tiles = ROWS <= 16 ? (u.many * p.kv_group + ROWS - 1) / ROWS : (u.many + p.tile_tokens - 1) / p.tile_tokens;
  u.tiles = max((u.len + KT - 1) / KT, 1);                    // (a request without keys still gets its zeros)
}
template <int KT, int ROWS>
__device__ __forceinline__ void load_request(const CacheAttnParams& p, Unit& u) {
  set_request<KT, ROWS>(p, u, p.new_offsets[u.r], p.new_offsets[u.r + 1], p.kv_lens[u.r]);
}
// Places on the line that a unit takes behind its tiles, for what it costs besides: 128-row units begin and end slowly, and their last
// tiles, with masks, take two to three times the others' time (24 trees of up to 32 tokens on contexts of up to 8192: the slowest block took
// 1.8 times the mean without).
template <int ROWS>
constexpr int EXTRA = ROWS > 16 ? 6 : 0;
// The next unit that has rows; u.r = p.R behind the last.
template <int KT, int ROWS>
__device__ __forceinline__ void next_unit(const CacheAttnParams& p, Unit& u) {
  u.start += u.pitch ? u.pitch : u.tiles + EXTRA<ROWS>;
  if (++u.rt < u.row_tiles) return;
  u.rt = 0;
  if (++u.hk >= p.heads_cached) {
    u.hk = 0;
    do {
      if (++u.r >= p.R) return;
      load_request<KT, ROWS>(p, u);
    } while (u.many == 0);
  }
}
// First tile of the unit at or behind place x, and at most all of them.
__device__ __forceinline__ int tile_at(const Unit& u, int x) { return min(max(x - u.start, 0), u.tiles); }
// `total` places in `runs` runs: the first `more` of them have one place more than the others.
struct Cut {
  int total, runs, each, more;
  __device__ __forceinline__ int start(int id) const { return id >= runs ? total : each * id + min(id, more); }
  __device__ __forceinline__ int run_of(int x) const {
    const int big = more * (each + 1);
    return x < big ? x / (each + 1) : more + (x - big) / each;
  }
};

// x / group for x < 2^16
__device__ __forceinline__ int by_group(const CacheAttnParams& p, int x) { return p.kv_group == 1 ? x : static_cast<int>(__umulhi(x, p.group_magic)); }

// A part of a unit's result: rows x D sums, then maxima, then sums of weights; whole 16-byte words, so that parts lie side by side.
__host__ __device__ constexpr int part_size(int max_rows, int D) { return (max_rows * (D + 2) + 3) / 4 * 4; }
// What it belongs to:
struct Part {
  int start, last;                  // of the unit's first and last tile (start < 0: none)
  int first, many, rt, hk;
};

// Rows of a unit, and new token and query head (of the group) of one.  Units of up to 16 rows take them as they come, token by
// token; the 128-row ones take whole tokens, head by head, so that a warp's rows are mostly one head's.
template <int ROWS>
__device__ __forceinline__ int unit_rows(const CacheAttnParams& p, int many, int rt) {
  return ROWS <= 16 ? min(ROWS, many * p.kv_group - rt * ROWS) : min(p.tile_tokens, many - rt * p.tile_tokens) * p.kv_group;
}
template <int ROWS>
__device__ __forceinline__ void row_at(const CacheAttnParams& p, int many, int rt, int row, int& token, int& head) {
  if (ROWS <= 16) {
    const int at = rt * ROWS + row;
    token = by_group(p, at);
    head = at - token * p.kv_group;
  } else {
    const int tokens = min(p.tile_tokens, many - rt * p.tile_tokens);
    head = row / tokens;
    token = rt * p.tile_tokens + row - head * tokens;
  }
}

template <int ROWS>
__device__ __forceinline__ void write_row(const CacheAttnParams& p, const Part& u, int row, int f, float4 x, float m, float l) {
  int i, hg;
  row_at<ROWS>(p, u.many, u.rt, row, i, hg);
  const int n = u.first + i, h = u.hk * p.kv_group + hg;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;               // (NaN stays NaN)
  const int64_t o = n * p.o_strides[0] + h * p.o_strides[1] + f;
  if (p.o_f32) {
    *reinterpret_cast<float4*>(static_cast<float*>(p.O) + o) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
  } else {
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.O) + o) = make_uint2(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv));
  }
  if (f == 0 && p.LSE) {
    const bool frozen = (p.frozen[h >> 5] >> (h & 31)) & 1;
    p.LSE[static_cast<int64_t>(n) * p.H + h] = frozen ? 0.0f : l == 0.0f ? -INFINITY : natural_lse(m, l);
  }
}

// Joins `members` parts, in order, on `nthr` threads of which this is number `tid`: to the outputs, or (dst) to one part.  A thread takes
// ITEMS times four features side by side, and AHEAD parts at a time, so that their loads are under way together; more than a few
// of both is no faster, because this code is met cold and every instruction of it has to be fetched.
template <int D, int ROWS, bool GLOBAL, int ITEMS, int AHEAD, typename At>
__device__ __forceinline__ void join(const CacheAttnParams& p, const Part& u, int max_rows, int members, At at, float* dst, int tid, int nthr) {
  const int items = unit_rows<ROWS>(p, u.many, u.rt) * (D / 4);
#pragma unroll 1
  for (int e0 = tid; e0 < items; e0 += ITEMS * nthr) {
    float m[ITEMS], l[ITEMS];
    float4 x[ITEMS];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      m[k] = -INFINITY;
      l[k] = 0.0f;
      x[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
#pragma unroll 1
    for (int i0 = 0; i0 < members; i0 += AHEAD) {
      float ms[ITEMS][AHEAD], ls[ITEMS][AHEAD];
      float4 v[ITEMS][AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const float* s = at(min(i0 + i, members - 1));
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
          const int e = e0 + k * nthr, row = e / (D / 4), f = (e - row * (D / 4)) * 4;
          const float* q = s + max_rows * D + row;
          ms[k][i] = -INFINITY;
          ls[k][i] = 0.0f;
          v[k][i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (i0 + i < members && e < items) {
            ms[k][i] = GLOBAL ? __ldcg(q) : *q;
            ls[k][i] = GLOBAL ? __ldcg(q + max_rows) : q[max_rows];
            v[k][i] = GLOBAL ? __ldcg(reinterpret_cast<const float4*>(s + row * D + f)) : *reinterpret_cast<const float4*>(s + row * D + f);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < ITEMS; ++k) {
        float top = m[k];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) top = fmaxf(top, ms[k][i]);
        const float base = top == -INFINITY ? 0.0f : top;
        const float c = ex16(m[k] - base);
        m[k] = top;
        l[k] *= c;
        x[k].x *= c; x[k].y *= c; x[k].z *= c; x[k].w *= c;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          const float w = ex16(ms[k][i] - base);             // (absent: 0, of zeros)
          l[k] += w * ls[k][i];
          x[k].x += w * v[k][i].x; x[k].y += w * v[k][i].y; x[k].z += w * v[k][i].z; x[k].w += w * v[k][i].w;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int e = e0 + k * nthr, row = e / (D / 4), f = (e - row * (D / 4)) * 4;
      if (e >= items) continue;
      if (dst) {
        *reinterpret_cast<float4*>(dst + row * D + f) = x[k];
        if (f == 0) {
          dst[max_rows * D + row] = m[k];
          dst[max_rows * (D + 1) + row] = l[k];
        }
      } else {
        write_row<ROWS>(p, u, row, f, x[k], m[k], l[k]);
      }
    }
  }
}

// The line of all tiles and where run number `run` of this block's RUNS begins: place x0, in unit u; the run ends before x1 (x0 = x1:
// it is empty, and u is not set).  Called by a block of W warps; smem: 16 R + 4 bytes that may be written over behind the next
// barrier.  SINGLE: tiles a run up to which a block takes a whole unit where there are no more units than blocks.
template <int KT, int ROWS, int W, int RUNS, int SINGLE>
__device__ __forceinline__ void place_run(const CacheAttnParams& p, uint8_t* smem, int (&red)[3][W], int run, Cut& cut, int& x0, int& x1, Unit& u) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // inclusive sums over each warp's requests, a warp for every 32 as far as there are warps (the others issue nothing meanwhile)
  int* sums = reinterpret_cast<int*>(smem);
  int* usums = sums + p.R;                                   // of units
  int* firsts = usums + p.R;                                 // [R + 1] and [R]: as in new_offsets and kv_lens
  int* lens = firsts + p.R + 1;
  const int Hk = p.heads_cached, scanning = min(W, (p.R + 31) >> 5), per = (p.R + 32 * scanning - 1) / (32 * scanning);
  if (warp < scanning) {
    const int r0 = min(static_cast<int>(threadIdx.x) * per, p.R), r1 = min(r0 + per, p.R);
    int cost = 0, units = 0, longest = 0;
    for (int r = r0; r < r1; ++r) {
      Unit u;
      const int first = p.new_offsets[r], last = p.new_offsets[r + 1], len = p.kv_lens[r];
      firsts[r] = first;
      if (r == p.R - 1) firsts[p.R] = last;
      lens[r] = len;
      set_request<KT, ROWS>(p, u, first, last, len);
      cost += u.row_tiles * Hk * (u.tiles + EXTRA<ROWS>);
      units += u.row_tiles * Hk;
      if (u.many > 0) longest = max(longest, u.tiles);
      sums[r] = cost;
      usums[r] = units;
    }
    int c = cost, n = units;
#pragma unroll 1
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, c, d), z = __shfl_up_sync(0xffffffffu, n, d);
      if (lane >= d) {
        c += y;
        n += z;
      }
    }
    longest = __reduce_max_sync(0xffffffffu, longest);
    if (lane == 31) {
      red[0][warp] = c;
      red[1][warp] = n;
      red[2][warp] = longest;
    }
    for (int r = r0; r < r1; ++r) {
      sums[r] += c - cost;
      usums[r] += n - units;
    }
  }
  __syncthreads();
  cut = Cut{0, 0, 0, 0};
  int pitch = 0;                                             // places from one unit to the next, 0: its tiles
  int chunk_sum = lane < scanning ? red[0][lane] : 0;
  {
    const int chunk_units = lane < scanning ? red[1][lane] : 0;
    const int units = __reduce_add_sync(0xffffffffu, chunk_units);
    const int longest = __reduce_max_sync(0xffffffffu, lane < scanning ? red[2][lane] : 0);
    if (units <= static_cast<int>(gridDim.x) && longest <= SINGLE * RUNS) {
      // Few short units: a block each, so that no unit's parts meet through L2.
      cut.each = (longest + RUNS - 1) / RUNS;
      pitch = cut.each * RUNS;
      cut.total = units * pitch;
      cut.runs = units * RUNS;
      chunk_sum = chunk_units * pitch;
    } else {
      // runs of two tiles at least; 128-row units, whose parts are large, not into more of them than joining is worth: a part takes the
      // block that joins about as long as a tile its own, so that the square root of the tiles is the best number of either (one tree of
      // 32 tokens on 8192 cached ones, 32 heads on 8: 112 us in 37 parts a unit, 60 in 12)
      cut.total = __reduce_add_sync(0xffffffffu, chunk_sum);
      const int least = ROWS <= 16 ? 2 : max(2, static_cast<int>(sqrtf(static_cast<float>(longest))));
      cut.runs = max(1, min(static_cast<int>(gridDim.x) * RUNS, (cut.total - 1) / least + 1));
      cut.each = cut.total / cut.runs;
      cut.more = cut.total - cut.each * cut.runs;
    }
  }
  x0 = cut.start(blockIdx.x * RUNS + run);
  x1 = cut.start(blockIdx.x * RUNS + run + 1);
  u.r = p.R;
  u.pitch = pitch;
  if (x0 < x1) {
    int chunk_end = chunk_sum;
#pragma unroll 1
    for (int d = 1; d < W; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, chunk_end, d);
      if (lane >= d) chunk_end += y;
    }
    const int chunk = __ffs(__ballot_sync(0xffffffffu, chunk_end > x0)) - 1;   // (x0 is below the total: there is one)
    const int off = __shfl_sync(0xffffffffu, chunk_end - chunk_sum, chunk);
    auto sum = [&](int r) { return off + (pitch ? usums[r] * pitch : sums[r]); };
    int lo = chunk * 32 * per, hi = min(lo + 32 * per, p.R) - 1;
    const int base = lo;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (sum(mid) > x0) hi = mid;
      else lo = mid + 1;
    }
    u.r = lo;
    u.start = lo > base ? sum(lo - 1) : off;
    set_request<KT, ROWS>(p, u, firsts[lo], firsts[lo + 1], lens[lo]);
    const int step = pitch ? pitch : u.tiles + EXTRA<ROWS>, at = (x0 - u.start) / step;   // number of the unit within its request
    u.hk = u.row_tiles == 1 ? at : at / u.row_tiles;
    u.rt = at - u.hk * u.row_tiles;
    u.start += at * step;
  }
}

}  // namespace
}  // namespace saf
