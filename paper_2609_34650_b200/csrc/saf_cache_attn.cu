// Attention of a step's new tokens over a paged cache, ordinary and frozen heads side by side.
//
//   O_i = sum_j e^{s_ij} V_j / sum_j e^{s_ij} over the keys j that row i sees; s_ij = scale q_i k_j (ordinary head) or
//   alpha(p_j) + rho(p_i - p_j) (frozen head), running maximum and sum in fp32, in powers of two.
//
// Every key and value is read once for all rows that share it, so DRAM bounds the call unless it is a short one.  A unit is one request,
// one cached head and up to 16 of its rows (new token, query head of the group); its keys come in tiles of 16.  The units' tiles, laid end to end
// and weighed by what they read (2 for keys and values, 1 where all heads of a group are frozen and only values are read), are cut
// into equal runs, one for each warp of the grid: no run is longer than another whatever the lengths are, and a single long request fills
// the GPU like many short ones.  A warp streams its run on its own: it fetches tiles by TMA into a ring of its own, multiplies with
// 16-row matrix instructions (rows that are not there are zeros: with up to 16 rows a tile costs 32 instructions of 4096 multiply-adds' worth for 8 KB, about
// a fifth of the tensor cores' time at DRAM speed), and meets other warps only when the run is over, to join what is left of
// units that were cut: in shared memory within a block, through L2 between blocks, where the block that arrives last joins the parts in order.
#include "ptx.cuh"
#include "saf_internal.h"

#include <algorithm>
#include <cuda_bf16.h>

namespace saf {
namespace {

constexpr int KT = 16;              // keys of a tile: one step of the second product
constexpr int ROWS = 16;            // rows of a unit
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <int D>
struct Cfg {
  static constexpr int HALVES = D == 64 ? 1 : 2;              // 64-feature boxes of a tile row (96: zero-filled to 128)
  static constexpr int TILE = HALVES * KT * 128;              // bytes of a key or value tile
  static constexpr int STAGE = 2 * TILE;
  static constexpr int WARPS = D == 64 ? 16 : 8;              // so that a ring of three stages a warp takes 192 KB
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// c += a b: a 16 rows x 16, b 16 x 8 columns
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Where a run stands: a unit, and its place on the line of all tiles.
struct Unit {
  long long start;                  // of the unit's first tile on the line
  int r, hk, rt;                    // request, cached head, row tile
  int first, many, len;             // the request's first row, rows that are computed, tokens in its cache
  int tiles, row_tiles, weight;
};

__device__ __forceinline__ int weight_of(const CacheAttnParams& p, int hk) { return ((p.with_keys[hk >> 5] >> (hk & 31)) & 1) + 1; }

__device__ __forceinline__ void load_request(const CacheAttnParams& p, Unit& u) {
  u.first = min(max(p.new_offsets[u.r], 0), p.N);
  const int last = min(p.new_offsets[u.r + 1], p.N);
  u.many = min(max(last - u.first, 0), p.max_new);
  u.len = min(max(p.kv_lens[u.r], 0), p.max_len);
  u.row_tiles = (u.many * p.kv_group + ROWS - 1) / ROWS;
  u.tiles = max((u.len + KT - 1) / KT, 1);                    // (a request without keys still gets its zeros)
}
// The next unit that has rows; u.r = p.R behind the last.
__device__ __forceinline__ void next_unit(const CacheAttnParams& p, Unit& u) {
  u.start += static_cast<long long>(u.weight) * u.tiles;
  if (++u.rt < u.row_tiles) return;
  u.rt = 0;
  if (++u.hk >= p.H / p.kv_group) {
    u.hk = 0;
    do {
      if (++u.r >= p.R) return;
      load_request(p, u);
    } while (u.many == 0);
  }
  u.weight = weight_of(p, u.hk);
}
// First tile of the unit at or behind place x, and at most all of them.
__device__ __forceinline__ int tile_at(const Unit& u, long long x) {
  const long long d = x - u.start;
  if (d <= 0) return 0;
  return static_cast<int>(min((d + u.weight - 1) / u.weight, static_cast<long long>(u.tiles)));
}

// A part of a unit's result: rows x D sums, then maxima, then sums of weights; whole 16-byte words, so that parts lie side by side.
__host__ __device__ constexpr int part_size(int max_rows, int D) { return (max_rows * (D + 2) + 3) / 4 * 4; }
// What it belongs to:
struct Part {
  long long start, last;            // of the unit's first and last tile (start < 0: none)
  int first, many, rt, hk;
};

template <int D>
__device__ __forceinline__ void write_row(const CacheAttnParams& p, const Part& u, int row, int f, float4 x, float m, float l) {
  const int g = p.kv_group, at = u.rt * ROWS + row, n = u.first + at / g, h = u.hk * g + at % g;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;               // (NaN stays NaN)
  const int64_t o = n * p.o_strides[0] + h * p.o_strides[1] + f;
  if (p.o_f32) {
    *reinterpret_cast<float4*>(static_cast<float*>(p.O) + o) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
  } else {
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.O) + o) = make_uint2(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv));
  }
  if (f == 0 && p.LSE) {
    const bool frozen = (p.frozen[h >> 5] >> (h & 31)) & 1;
    p.LSE[static_cast<int64_t>(n) * p.H + h] = frozen ? 0.0f : l == 0.0f ? -INFINITY : (m + log2f(l)) * LN2;
  }
}

// Joins `members` parts, in order, on `nthr` threads of which this is number `tid`: to the outputs, or (dst) to one part.
template <int D, bool GLOBAL, typename At>
__device__ __forceinline__ void join(const CacheAttnParams& p, const Part& u, int max_rows, int members, At at, float* dst, int tid, int nthr) {
  const int rows = min(ROWS, u.many * p.kv_group - u.rt * ROWS);
  for (int e = tid; e < rows * (D / 4); e += nthr) {
    const int row = e / (D / 4), f = (e - row * (D / 4)) * 4;
    float m = -INFINITY, l = 0.0f;
    for (int i = 0; i < members; ++i) {
      const float* s = at(i) + max_rows * D + row;
      m = fmaxf(m, GLOBAL ? __ldcg(s) : *s);
    }
    const float base = m == -INFINITY ? 0.0f : m;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int i = 0; i < members; ++i) {
      const float* s = at(i);
      const float* q = s + max_rows * D + row;
      const float4 v = GLOBAL ? __ldcg(reinterpret_cast<const float4*>(s + row * D + f)) : *reinterpret_cast<const float4*>(s + row * D + f);
      const float w = ex2_approx((GLOBAL ? __ldcg(q) : *q) - base);
      l += w * (GLOBAL ? __ldcg(q + max_rows) : q[max_rows]);
      x.x += w * v.x; x.y += w * v.y; x.z += w * v.z; x.w += w * v.w;
    }
    if (dst) {
      *reinterpret_cast<float4*>(dst + row * D + f) = x;
      if (f == 0) {
        dst[max_rows * D + row] = m;
        dst[max_rows * (D + 1) + row] = l;
      }
    } else {
      write_row<D>(p, u, row, f, x, m, l);
    }
  }
}

template <int D, bool EXACT>
__global__ void __launch_bounds__(32 * Cfg<D>::WARPS, 1)
saf_cache_attn_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const __grid_constant__ CacheAttnParams p) {
  constexpr int W = Cfg<D>::WARPS, TILE = Cfg<D>::TILE, STAGE = Cfg<D>::STAGE, HALVES = Cfg<D>::HALVES, NT = 32 * W;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int stages = p.stages, max_rows = p.max_rows, part_floats = part_size(max_rows, D);
  // [warps][stages] tiles, then a part of each warp's run; at the run's end its ring holds a second one
  float* parts = reinterpret_cast<float*>(smem + W * stages * STAGE);
  __shared__ uint64_t full[W][4];
  __shared__ Part meta[W][2];
  __shared__ long long red[W];
  __shared__ int abort_s, arrived_s[2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) abort_s = 0;
  if (lane < stages) mbar_init(&full[warp][lane], 1);
  if (lane < 2) meta[warp][lane].start = -1;
  mbar_fence_init();
  if (threadIdx.x == 0) {
    tma_prefetch_desc(&mk);
    tma_prefetch_desc(&mv);
  }
  pdl_wait();
  pdl_launch_dependents();

  // ---- the line of all tiles: inclusive sums over the requests (in the ring's memory, before it is used)
  long long* sums = reinterpret_cast<long long*>(smem);
  const int Hk = p.H / p.kv_group;
  const int per = (p.R + NT - 1) / NT, r0 = min(static_cast<int>(threadIdx.x) * per, p.R), r1 = min(r0 + per, p.R);
  long long cost = 0;
  for (int r = r0; r < r1; ++r) {
    Unit u;
    u.r = r;
    load_request(p, u);
    cost += static_cast<long long>(u.row_tiles) * u.tiles * p.head_weights;
    sums[r] = cost;
  }
  long long scan = cost;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += y;
  }
  if (lane == 31) red[warp] = scan;
  __syncthreads();
  long long before = scan - cost, total = 0;
  for (int w = 0; w < W; ++w) {
    const long long s = red[w];
    if (w < warp) before += s;
    total += s;
  }
  for (int r = r0; r < r1; ++r) sums[r] += before;
  __syncthreads();
  // runs of at least two whole tiles
  const long long runs = max(1ll, min(static_cast<long long>(gridDim.x) * W, (total + 3) / 4));
  auto run_start = [&](long long id) { return total * min(id, runs) / runs; };
  const long long x0 = run_start(static_cast<long long>(blockIdx.x) * W + warp), x1 = run_start(static_cast<long long>(blockIdx.x) * W + warp + 1);
  const long long b0 = run_start(static_cast<long long>(blockIdx.x) * W), b1 = run_start(static_cast<long long>(blockIdx.x + 1) * W);
  if (b0 >= b1) return;
  Unit u;
  u.r = p.R;
  if (x0 < x1) {
    int lo = 0, hi = p.R;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (sums[mid] > x0) hi = mid;
      else lo = mid + 1;
    }
    u.r = lo;                                               // (x0 < total: there is one)
    u.start = lo ? sums[lo - 1] : 0;
    load_request(p, u);
    u.hk = 0;
    u.rt = 0;
    u.weight = weight_of(p, 0);
    while (u.start + static_cast<long long>(u.weight) * u.tiles * u.row_tiles <= x0) {
      u.start += static_cast<long long>(u.weight) * u.tiles * u.row_tiles;
      u.weight = weight_of(p, ++u.hk);
    }
    const long long skip = (x0 - u.start) / (static_cast<long long>(u.weight) * u.tiles);
    u.rt = static_cast<int>(skip);
    u.start += skip * u.weight * u.tiles;
  }
  __syncthreads();                                          // the sums have been read: the ring may be filled

  uint8_t* ring = smem + warp * stages * STAGE;
  const uint32_t ring_s = smem_u32(ring);
  const WaitCtx wc{&abort_s, p.status, p.wait_limit_ns};
  const int g = p.kv_group, gid = lane >> 2, t2 = (lane & 3) * 2;

  // ---- the fetching end of the run: up to `stages` tiles ahead of the multiplying one
  Unit fu = u;
  int ft = 0, fend = 0, pages_at = 0, page_ids = 0, filled = 0;
  bool fmore = x0 < x1;
  auto load_pages = [&](int tile) {                          // lane l: page of tile + l
    pages_at = tile;
    const int t = tile + lane;
    int id = 0;
    if (t < fu.tiles && t * KT < p.max_len) id = p.block_table[static_cast<int64_t>(fu.r) * p.max_pages + t * KT / p.page_size];
    page_ids = min(max(id, 0), p.n_pages - 1);
  };
  auto enter = [&]() {                                       // false: the unit has no tile in the run
    ft = tile_at(fu, x0);
    fend = tile_at(fu, x1);
    return ft < fend;
  };
  auto advance = [&]() {                                     // to the next unit with a tile in the run
    do {
      next_unit(p, fu);
      if (fu.r >= p.R || fu.start >= x1) {
        fmore = false;
        return;
      }
    } while (!enter());
    load_pages(ft);
  };
  if (fmore) {
    if (enter()) load_pages(ft);
    else advance();
  }
  auto fetch = [&]() {
    if (!fmore) return;
    const int stage = filled % stages;
    if (ft - pages_at >= 32) load_pages(ft);
    const int page = __shfl_sync(0xffffffffu, page_ids, ft - pages_at);
    const int slot = (ft * KT) % p.page_size;
    const bool keys = fu.weight == 2;
    if (lane == 0) {
      uint8_t* dst = ring + stage * STAGE;
      uint64_t* bar = &full[warp][stage];
      mbar_expect_tx(bar, keys ? STAGE : TILE);
#pragma unroll
      for (int h = 0; h < HALVES; ++h) {
        if (keys) tma_load_4d(dst + h * KT * 128, &mk, bar, 64 * h, slot, fu.hk, page);
        tma_load_4d(dst + TILE + h * KT * 128, &mv, bar, 64 * h, slot, fu.hk, page);
      }
    }
    ++filled;
    if (++ft >= fend) advance();
  };
  for (int s = 0; s < stages; ++s) fetch();

  // ---- the multiplying end
  int used = 0, n_parts = 0;
  bool alive = true;
  while (alive && u.r < p.R && u.start < x1) {
    const int t_begin = tile_at(u, x0), t_end = tile_at(u, x1);
    if (t_begin >= t_end) {
      next_unit(p, u);
      continue;
    }
    const int ctx = u.len - u.many, rows = min(ROWS, u.many * g - u.rt * ROWS);
    // this thread's two rows
    int pos[2];
    bool there[2], frozen[2];
    unsigned long long mask[2];
    const float* arow[2];
    const float* rrow[2];
    int64_t qoff[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = gid + 8 * k;
      there[k] = row < rows;
      const int at = there[k] ? u.rt * ROWS + row : u.rt * ROWS;
      const int i = at / g, h = u.hk * g + at % g, n = u.first + i;
      frozen[k] = (p.frozen[h >> 5] >> (h & 31)) & 1;
      mask[k] = p.masks ? p.masks[n] : (2ull << i) - 1;      // (i = 63: all)
      pos[k] = frozen[k] ? (p.positions ? min(max(p.positions[n], 0), p.Tp - 1) : max(ctx + i, 0)) : 0;
      arow[k] = p.alpha + static_cast<int64_t>(h) * p.Tp;
      rrow[k] = p.rho + static_cast<int64_t>(h) * p.Tp;
      qoff[k] = n * p.q_strides[0] + h * p.q_strides[1];
      if (!there[k]) frozen[k] = false;
    }
    const bool any_frozen = __any_sync(0xffffffffu, frozen[0] || frozen[1]);
    const bool keys = u.weight == 2;
    uint32_t q[D / 16][4];
    if (keys) {
      const __nv_bfloat16* Q = static_cast<const __nv_bfloat16*>(p.q);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = e & 1;
          q[ks][e] = there[k] && !frozen[k] ? *reinterpret_cast<const uint32_t*>(Q + qoff[k] + ks * 16 + (e >> 1) * 8 + t2) : 0u;
        }
    }
    float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int f = 0; f < D / 8; ++f)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[f][e] = 0.0f;

    for (int t = t_begin; t < t_end; ++t) {
      const int stage = used % stages;
      const uint32_t ks_addr = ring_s + stage * STAGE, vs_addr = ks_addr + TILE;
      const int j0 = t * KT;
      const bool tail = j0 + KT > ctx;
      // frozen rows: this thread's preferences, fetched while the tile is waited for
      float fs[2][4];
      if (any_frozen) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = j0 + (e >> 1) * 8 + t2 + (e & 1), back = j - ctx;
            fs[k][e] = -INFINITY;
            if (frozen[k] && j < u.len) {
              const int pj = back < 0 || !p.positions ? j : min(max(p.positions[u.first + back], 0), p.Tp - 1);
              if (pj <= pos[k]) fs[k][e] = (arow[k][pj] + rrow[k][pos[k] - pj]) * LOG2E;
            }
          }
      }
      if (!mbar_wait_warp_compact(&full[warp][stage], (used / stages) & 1, wc, 90)) {
        alive = false;
        break;
      }
      float s[2][4];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[k][e] = 0.0f;
      if (keys) {
        // s[nt][2 k + e]: row gid + 8 k, key 8 nt + t2 + e
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          uint32_t b[4];
          const int row = ((lane >> 4) << 3) + (lane & 7), chunk = (ks & 3) * 2 + ((lane >> 3) & 1);
          ldsm4(ks_addr + (ks >> 2) * (KT * 128) + row * 128 + ((chunk ^ (row & 7)) << 4), b);
          mma16816(s[0], q[ks], b[0], b[1]);
          mma16816(s[1], q[ks], b[2], b[3]);
        }
      }
      float top[2] = {m[0], m[1]};
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = e >> 1;
          float x = frozen[k] ? fs[k][nt * 2 + (e & 1)] : s[nt][e] * p.scale_log2;
          if (tail) {
            const int j = j0 + nt * 8 + t2 + (e & 1), back = j - ctx;
            if (j >= u.len || (back >= 0 && !((mask[k] >> back) & 1))) x = -INFINITY;
          }
          if (!there[k]) x = -INFINITY;
          s[nt][e] = x;
          top[k] = fmaxf(top[k], x);
        }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 1));
        top[k] = fmaxf(top[k], __shfl_xor_sync(0xffffffffu, top[k], 2));
      }
      if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float c = top[k] == -INFINITY ? 1.0f : ex2_approx(m[k] - top[k]);
          m[k] = top[k];
          l[k] *= c;
#pragma unroll
          for (int f = 0; f < D / 8; ++f) {
            o[f][2 * k] *= c;
            o[f][2 * k + 1] *= c;
          }
        }
      }
      const float base[2] = {m[0] == -INFINITY ? 0.0f : m[0], m[1] == -INFINITY ? 0.0f : m[1]};
#pragma unroll
      for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = e >> 1;
          s[nt][e] = ex2_approx(s[nt][e] - base[k]);
          l[k] += s[nt][e];
        }
      if (tail) {
        // values behind the last key are whatever the page held, and a value that some rows do not see may be NaN or infinite: both
        // are zeroed for the product, the second kind added by hand to the rows that see it
        bool wild = false;
        for (int c = lane; c < KT * HALVES * 8; c += 32) {
          const int row = c & (KT - 1), rest = c >> 4;
          const uint32_t addr = vs_addr + (rest >> 3) * (KT * 128) + row * 128 + (((rest & 7) ^ (row & 7)) << 4);
          uint32_t w[4];
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
          if (j0 + row >= u.len) {
            st_shared_v4w(addr, 0, 0, 0, 0);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) wild |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
          }
        }
        __syncwarp();
        if (__any_sync(0xffffffffu, wild)) {
          for (int key = 0; key < KT; ++key) {
            const int src = (lane & ~3) | ((key & 7) >> 1);
            float w[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float a = (key & 1) ? s[0][2 * k + 1] : s[0][2 * k], b = (key & 1) ? s[1][2 * k + 1] : s[1][2 * k];
              w[k] = __shfl_sync(0xffffffffu, key < 8 ? a : b, src);
            }
#pragma unroll
            for (int f = 0; f < D / 8; ++f) {
              const uint32_t addr = vs_addr + (f >> 3) * (KT * 128) + key * 128 + (((f & 7) ^ (key & 7)) << 4) + t2 * 2;
              uint32_t v;
              asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
              const bool lo = (v & 0x7f80u) == 0x7f80u, hi = (v & 0x7f800000u) == 0x7f800000u;
              if (lo || hi) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  if (w[k] == 0.0f) continue;
                  if (lo) o[f][2 * k] += w[k] * __uint_as_float(v << 16);
                  if (hi) o[f][2 * k + 1] += w[k] * __uint_as_float(v & 0xffff0000u);
                }
              }
            }
          }
          __syncwarp();
          for (int c = lane; c < KT * HALVES * 32; c += 32) {   // (every word of the tile, wherever the swizzle put it)
            const uint32_t addr = vs_addr + c * 4;
            uint32_t v;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
            if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
            if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
          }
          __syncwarp();
        }
      }
      // second product.  EXACT (fp32 output): weights as three bf16 terms, 24 bits; else rounded to bf16 once (the output is, too)
      uint32_t a[EXACT ? 3 : 1][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {                           // a[e]: row gid + 8 (e & 1), keys 8 (e >> 1) + t2, + 1
        float lo = s[e >> 1][2 * (e & 1)], hi = s[e >> 1][2 * (e & 1) + 1];
#pragma unroll
        for (int i = 0; i < (EXACT ? 3 : 1); ++i) {
          a[i][e] = pack_bf16x2(lo, hi);
          lo -= __uint_as_float(a[i][e] << 16);
          hi -= __uint_as_float(a[i][e] & 0xffff0000u);
        }
      }
#pragma unroll
      for (int fb = 0; fb < D / 16; ++fb) {
        uint32_t b[4];
        const int row = (((lane >> 3) & 1) << 3) + (lane & 7), chunk = (fb & 3) * 2 + (lane >> 4);
        ldsm4t(vs_addr + (fb >> 2) * (KT * 128) + row * 128 + ((chunk ^ (row & 7)) << 4), b);
#pragma unroll
        for (int i = 0; i < (EXACT ? 3 : 1); ++i) {
          mma16816(o[2 * fb], a[i], b[0], b[1]);
          mma16816(o[2 * fb + 1], a[i], b[2], b[3]);
        }
      }
      if (tail) fence_proxy_async_smem();                     // (the tile may have been written to: before it is fetched over)
      __syncwarp();
      ++used;
      fetch();
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 1);
      l[k] += __shfl_xor_sync(0xffffffffu, l[k], 2);
    }
    const Part me{u.start, u.start + static_cast<long long>(u.weight) * (u.tiles - 1), u.first, u.many, u.rt, u.hk};
    if (!alive) {
      // given up: the copies in flight end before the block does (a bounded wait again), nothing is joined
      for (int i = used; i < filled; ++i)
        for (int spin = 0; spin < 100000 && !mbar_try_wait(&full[warp][i % stages], (i / stages) & 1); ++spin) {
        }
    } else if (t_begin == 0 && t_end == u.tiles) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // pairs of lanes put four features together
#pragma unroll
        for (int f = 0; f < D / 8; ++f) {
          const float a = o[f][2 * k], b = o[f][2 * k + 1];
          const float c = __shfl_xor_sync(0xffffffffu, a, 1), d = __shfl_xor_sync(0xffffffffu, b, 1);
          if (there[k] && (lane & 1) == 0) write_row<D>(p, me, gid + 8 * k, f * 8 + t2, make_float4(a, b, c, d), m[k], l[k]);
        }
      }
    } else {
      // the part of a unit that goes on elsewhere: at most two a run, the second when nothing more is fetched
      float* dst = n_parts == 0 ? parts + warp * part_floats : reinterpret_cast<float*>(ring);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int row = gid + 8 * k;
        if (there[k]) {
#pragma unroll
          for (int f = 0; f < D / 8; ++f) *reinterpret_cast<float2*>(dst + row * D + f * 8 + t2) = make_float2(o[f][2 * k], o[f][2 * k + 1]);
          if ((lane & 3) == 0) {
            dst[max_rows * D + row] = m[k];
            dst[max_rows * (D + 1) + row] = l[k];
          }
        }
      }
      if (lane == 0) meta[warp][n_parts] = me;
      ++n_parts;
    }
    next_unit(p, u);
  }
  // ---- what is left of cut units, in the order of the runs
  __syncthreads();
  auto part_of = [&](int i) { return (i & 1) ? reinterpret_cast<const float*>(smem + (i >> 1) * stages * STAGE) : parts + (i >> 1) * part_floats; };
  const Part* flat = &meta[0][0];
  auto block_of = [&](long long x) { return static_cast<int>(((x + 1) * runs - 1) / total / W); };
  int group = 0, n_open = 0;
  int open[2];
  for (int i = 0; i < 2 * W;) {
    if (flat[i].start < 0) {
      ++i;
      continue;
    }
    int members = 1, nexti = i + 1;
    int idx_last = i;
    for (; nexti < 2 * W; ++nexti) {
      if (flat[nexti].start < 0) continue;
      if (flat[nexti].start != flat[i].start) break;
      ++members;
      idx_last = nexti;
    }
    const Part unit = flat[i];
    // (members are the parts in [i, idx_last] that are there)
    auto member = [&](int k) {
      int at = i;
      for (int c = 0;; ++at) {
        if (flat[at].start < 0) continue;
        if (c++ == k) break;
      }
      return part_of(at);
    };
    (void)idx_last;
    const int c_first = block_of(unit.start), c_last = block_of(unit.last);
    if (c_first == c_last) {
      if (group % W == warp) join<D, false>(p, unit, max_rows, members, member, nullptr, lane, 32);
      ++group;
    } else {
      float* dst = p.workspace + (static_cast<int64_t>(blockIdx.x) * 2 + (b0 >= unit.start ? 0 : 1)) * part_floats;
      join<D, false>(p, unit, max_rows, members, member, dst, threadIdx.x, NT);
      if (n_open < 2) open[n_open++] = i;
    }
    i = nexti;
  }
  if (n_open == 0) return;
  __threadfence();
  __syncthreads();
  if (threadIdx.x < n_open) {
    const Part& unit = flat[open[threadIdx.x]];
    const int c_first = block_of(unit.start), c_last = block_of(unit.last);
    int* counter = p.counters + c_first;
    const int before_me = atomicAdd(counter, 1);
    arrived_s[threadIdx.x] = before_me == c_last - c_first;
    if (before_me == c_last - c_first) *counter = 0;
    __threadfence();
  }
  __syncthreads();
  for (int k = 0; k < n_open; ++k) {
    if (!arrived_s[k]) continue;
    const Part unit = flat[open[k]];
    const int c_first = block_of(unit.start), c_last = block_of(unit.last);
    auto member = [&](int i) {
      const int c = c_first + i;
      return p.workspace + (static_cast<int64_t>(c) * 2 + (run_start(static_cast<long long>(c) * W) >= unit.start ? 0 : 1)) * part_floats;
    };
    join<D, true>(p, unit, max_rows, c_last - c_first + 1, member, nullptr, threadIdx.x, NT);
  }
}

template <int D>
cudaError_t launch(const CUtensorMap& mk, const CUtensorMap& mv, CacheAttnParams& p, int num_sms, cudaStream_t st) {
  constexpr int W = Cfg<D>::WARPS;
  const size_t parts = static_cast<size_t>(W) * part_size(p.max_rows, D) * sizeof(float);
  p.stages = static_cast<int>(std::min<size_t>(4, (224 * 1024 - parts) / (static_cast<size_t>(W) * Cfg<D>::STAGE)));
  const size_t smem = static_cast<size_t>(W) * p.stages * Cfg<D>::STAGE + parts + 1024;
  auto kernel = p.o_f32 ? saf_cache_attn_kernel<D, true> : saf_cache_attn_kernel<D, false>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  return launch_pdl(PDL_REST, kernel, num_sms, 32 * W, smem, st, mk, mv, p);
}

}  // namespace

int cache_attn_rows(int max_new, int kv_group) { return std::min(ROWS, max_new * kv_group); }
size_t cache_attn_workspace(int max_rows, int D, int num_sms) { return static_cast<size_t>(num_sms) * 2 * part_size(max_rows, D) * sizeof(float); }

cudaError_t launch_cache_attn(const CUtensorMap& mk, const CUtensorMap& mv, CacheAttnParams& p, int num_sms, cudaStream_t st) {
  if (p.D == 64) return launch<64>(mk, mv, p, num_sms, st);
  if (p.D == 96) return launch<96>(mk, mv, p, num_sms, st);
  return launch<128>(mk, mv, p, num_sms, st);
}

}  // namespace saf
