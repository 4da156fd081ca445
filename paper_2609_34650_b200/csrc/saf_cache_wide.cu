// Attention of a step's new tokens over a paged cache where many rows share a key: drafted trees and chains on grouped heads.
//
// The mathematics is saf_cache_attn.cu's.  A unit here is one request, one cached head and up to 128 rows (whole new tokens with all
// query heads of the group, head by head), its tiles 64 keys, and a block takes one run of the line of all tiles.  With 16 rows
// a unit, 128 rows would read the cache eight times out of L2 and issue the 16-row instructions as often; on tcgen05 a tile takes
// the tensor core about 500 clk, whatever the rows, of the 1400 that DRAM needs for its 32 KB (head dimension 128).  The scores of a tile are
// formed while the one before is in its softmax (two places in TMEM; tiles of 128 keys, for which there is only one, took 7500 clk
// each in a chain of scores, softmax and second product), and two blocks an SM fill each other's waits.
//
// Per block (256 threads): warps 0-3 compute, a thread a row (= TMEM lane; two threads a row spilled 700 bytes at the registers that
// leaves), warps 4 and 5 fetch pages of keys and of values by TMA (a thread issues a copy in about 300 clk, and pages of 16 tokens
// take 12 a tile), warp 6 issues the MMAs and owns TMEM, warp 7 fetches bands.  TMEM columns [0,64) and [64,128) S (fp32) of even and odd tiles, then their
// weights (bf16 pairs) in the first half of each, [128,256) O.  Frozen rows replace their scores by alpha + rho out of a band that is
// copied in ahead: 64 preferences of keys and 192 of distances for each of up to FZ frozen heads (up to twice as many
// in one place instead of two); with more of them, or positions that are not near the tokens' places, they take them from global memory.
//
// 24 trees of up to 32 tokens on up to 8192 cached ones, 32 heads on 8, a third of them frozen: 137 us = 3.1 TB/s, 107 us without frozen
// heads.  In the second a tile and block takes 2740 clk, DRAM's rate for two blocks; the rest is the units' ends (12000 clk until the first
// scores, behind loads already in flight, 9000 for the last product and the part) and the joins (25000).
#include "saf_cache_attn.cuh"

namespace saf {
namespace {

constexpr int ROWS = 128, KT = 64, W = 8, NT = 32 * W, FZ = 6, BAND = 256;
constexpr int SINGLE_TILES = 16;    // tiles up to which a block takes a whole unit where there are no more units than blocks
constexpr int BLOCKS = CACHE_BLOCKS;

template <int D>
struct Cfg {
  static constexpr int PANELS = D == 64 ? 1 : 2;             // 64 features: 128-byte rows, one swizzle atom
  static constexpr int PANEL = KT * 128;
  static constexpr int TILE = PANELS * PANEL;
  static constexpr int ST = D == 64 ? 4 : 2;                 // tiles of keys, and of values, in shared memory
  static constexpr int OFF_Q = 0, OFF_K = PANELS * 128 * 128, OFF_V = OFF_K + ST * TILE, OFF_TAB = OFF_V + ST * TILE;
  // words: bands [2][FZ][BAND], keys' places in a band [2][64], positions of new tokens [64]
  static constexpr int TAB = 2 * FZ * BAND + 128 + 64;
  static constexpr int SMEM = OFF_TAB + TAB * 4 + 1024;
};

enum WideSite { SITE_K_EMPTY = 111, SITE_V_EMPTY, SITE_Q_FULL, SITE_K_FULL, SITE_P_FULL, SITE_V_FULL, SITE_O_FREE, SITE_S_FULL, SITE_PV_DONE, SITE_BAND_EMPTY, SITE_BAND_FULL };

// 4 bytes, or zeros
__device__ __forceinline__ void copy4(uint32_t dst, const float* src, bool in) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ float ld_shared_f(uint32_t addr) {
  float x;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(addr) : "memory");
  return x;
}
__device__ __forceinline__ bool wild16(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

// Scores of frozen rows without a band, from global memory: written over what the score MMA left.
__device__ __noinline__ void slow_scores(const CacheAttnParams& p, const Unit& w, int ctx, int t, int h, int pos, bool keys, bool frozen, uint32_t t_s,
                                         const int* newpos) {
  const int64_t head = static_cast<int64_t>(h) * p.Tp;
  for (int cc = 0; cc < KT / 16; ++cc) {
    uint32_t r[16];
    if (keys) {
      tmem_ld16(t_s + 16 * cc, r);
      tmem_wait_ld();
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int j = t * KT + 16 * cc + e, back = j - ctx;
      float x = keys ? __uint_as_float(r[e]) : 0.0f;
      if (frozen) {
        const int pj = back < 0 ? j : j < w.len ? newpos[back] : 0x7fffffff;
        x = pj <= pos ? p.alpha[head + pj] + p.rho[head + pos - pj] : -INFINITY;
      }
      r[e] = __float_as_uint(x);
    }
    tmem_st16(t_s + 16 * cc, r);
  }
  tmem_wait_st();
}

// Values behind the last key are whatever was there, and those from key `from` on, which not every row sees, may be NaN or infinite:
// both are zeroed for the product; true if there were any of the second kind (they are added to the rows that see them at the end).
template <int D>
__device__ __noinline__ bool clean_values(int br, int j0, int from, int len, uint32_t vs, int tid) {
  constexpr int PANELS = Cfg<D>::PANELS;
  bool wild = false;
  for (int c = tid; c < Cfg<D>::TILE / 16; c += 128) {
    const int box = c / (8 * br * PANELS), j = j0 + box * br + ((c >> 3) & (br - 1));
    if (j < from) continue;
    const uint32_t addr = vs + c * 16;
    uint32_t w[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
    if (j >= len) {
      st_shared_v4w(addr, 0, 0, 0, 0);
    } else if (wild16(w[0]) || wild16(w[1]) || wild16(w[2]) || wild16(w[3])) {
      wild = true;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if ((w[k] & 0x7f80u) == 0x7f80u) w[k] &= 0xffff0000u;
        if ((w[k] & 0x7f800000u) == 0x7f800000u) w[k] &= 0xffffu;
      }
      st_shared_v4w(addr, w[0], w[1], w[2], w[3]);
    }
  }
  return wild;
}

// New tokens of the unit's request whose keys rows may see (those that are not computed too); up to 64, and they have rows.
__device__ __forceinline__ int new_keys(const CacheAttnParams& p, const Unit& w) { return min(w.len - w.ctx, p.N - w.first); }

// Whether and how a unit's frozen rows go by bands; by a whole warp, the same for all.  A band serves a row whose position is at most 63 past the
// unit's first, and a key whose position is at most 63 from its tile's first slot: a cached key's is its place; a new token's, whichever of the
// request's it is, has to lie between the first new place and its own, as positions by place or by depth do.  (Out of line, once for both kinds of warps that ask: 24 trees 137 us, 141
// inlined.)
struct BandPlan {
  int n_frozen, pmin, span;
  bool fast, ahead;                 // by bands; in two places in turn
};
__device__ __noinline__ BandPlan plan_band(const CacheAttnParams& p, const Unit& w) {
  BandPlan b{0, 0, 0, false, false};
  for (int c = 0; c < p.kv_group; ++c) {
    const int hk = w.hk * p.kv_group + c;
    b.n_frozen += (p.frozen[hk >> 5] >> (hk & 31)) & 1;
  }
  if (b.n_frozen == 0) return b;
  const int ctx = w.ctx, fresh = new_keys(p, w), t0 = w.rt * p.tile_tokens, t1 = min(t0 + p.tile_tokens, w.many);
  int lo = 0x7fffffff, hi = 0;
  bool near = ctx >= 0;
#pragma unroll
  for (int c = threadIdx.x & 31; c < 64; c += 32) {
    if (c >= fresh) continue;
    const int x = p.positions ? min(max(p.positions[w.first + c], 0), p.Tp - 1) : max(ctx + c, 0);
    near &= x >= ctx && x <= ctx + c;
    if (c >= t0 && c < t1) {
      lo = min(lo, x);
      hi = max(hi, x);
    }
  }
  b.pmin = __reduce_min_sync(0xffffffffu, lo);
  b.span = __reduce_max_sync(0xffffffffu, hi) - b.pmin;
  b.fast = b.n_frozen <= 2 * FZ && b.span < 64 && __all_sync(0xffffffffu, near);
  b.ahead = b.fast && b.n_frozen <= FZ;
  return b;
}

// The block's part of a unit that lies in several blocks is complete (a barrier lies between its writes and this call, by one thread):
// whether it is the last.
__device__ __forceinline__ int arrive(const CacheAttnParams& p, const Cut& cut, const Part& unit) {
  const int first = cut.run_of(unit.start), last = cut.run_of(unit.last);
  __threadfence();
  const bool end = atomicAdd(p.counters + first, 1) == last - first;
  if (end) p.counters[first] = 0;
  __threadfence();
  return end;
}

template <int D>
__global__ void __launch_bounds__(NT, BLOCKS)
saf_cache_wide_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const __grid_constant__ CacheAttnParams p) {
  using C = Cfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ uint64_t k_full[4], k_empty[4], v_full[4], v_empty[4], q_full, s_full[2], p_full, pv_done, o_free, band_full[2], band_empty[2];
  __shared__ Part open_unit[2];                              // units that go on in other blocks: the run's first, its last
  __shared__ Unit work[3];                                   // what the compute warps are at, in turn; the run's first
  __shared__ Cut cut_s;
  __shared__ int red[3][W], arrived_s[2], range_s[2][2], abort_s, wild_s;
  __shared__ uint32_t tmem_slot;
  float* bands = reinterpret_cast<float*>(smem + C::OFF_TAB);
  int* places = reinterpret_cast<int*>(bands + 2 * FZ * BAND);
  int* newpos = places + 128;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const WaitCtx wc{&abort_s, p.status, p.wait_limit_ns};
  if (tid == 0) {
    abort_s = 0;
    open_unit[0].start = open_unit[1].start = -1;
    arrived_s[0] = arrived_s[1] = -1;
    for (int s = 0; s < 2; ++s) {
      mbar_init(&s_full[s], 1);
      mbar_init(&band_full[s], 64);                          // (each lane's copies, and each lane)
      mbar_init(&band_empty[s], 4);
    }
    for (int s = 0; s < C::ST; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&k_empty[s], 1);
      mbar_init(&v_full[s], p.selftest_drop_load && blockIdx.x == 1 && s == 0 ? 2 : 1);
      mbar_init(&v_empty[s], 1);
    }
    mbar_init(&q_full, 4);                                   // (one arrival per compute warp)
    mbar_init(&p_full, 4);
    mbar_init(&pv_done, 1);
    mbar_init(&o_free, 4);
    mbar_fence_init();
    tma_prefetch_desc(&mk);
    tma_prefetch_desc(&mv);
  }
  if (warp == 6) {
    tmem_alloc(&tmem_slot, 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_wait();
  pdl_launch_dependents();

  Unit u;
  int x0, x1;
  {
    Cut cut;
    place_run<KT, ROWS, W, 1, SINGLE_TILES>(p, smem, red, 0, cut, x0, x1, u);
    if (tid == 0) {
      cut_s = cut;
      work[1] = work[2] = u;
    }
  }
  __syncthreads();                                           // the sums have been read: tiles may be fetched over them
  auto slot_of = [&](int block, int start) {
    return p.workspace + (static_cast<int64_t>(block) * 2 + (cut_s.start(block) >= start ? 0 : 1)) * part_size(p.max_rows, D);
  };
  const int g = p.kv_group;

  if (x0 >= x1) {
  } else if (warp == 4 || warp == 5) {
    // ---------------------------------------------------------------- pages of keys (warp 4) and of values
    const bool values = warp == 5;
    uint64_t* full = values ? v_full : k_full;
    uint64_t* empty = values ? v_empty : k_empty;
    const CUtensorMap* map = values ? &mv : &mk;
    uint8_t* ring = smem + (values ? C::OFF_V : C::OFF_K);
    const int br = p.box_rows;
    const int split = values && D == 128 ? 1 : C::PANELS;    // copies of a box (values at 128: both halves at once)
    uint32_t count = 0;
    bool ok = true;
    for (; ok && u.r < p.R && u.start < x1; next_unit<KT, ROWS>(p, u)) {
      const int tb = tile_at(u, x0), te = tile_at(u, x1);
      if (!values && !has_keys(p, u.hk)) continue;
      constexpr int CH = KT / 16;
      int ids = 0, ids_at = tb - 32 / CH;
      for (int t = tb; t < te; ++t, ++count) {
        if (t - ids_at >= 32 / CH) {                         // lane l: page of the 16 keys number CH t + l
          ids_at = t;
          const int c = t * CH + lane;
          int id = 0;
          if (c * 16 < max(u.len, 1)) id = p.block_table[static_cast<int64_t>(u.r) * p.max_pages + (p.page_shift >= 0 ? c >> p.page_shift : c / (p.page_size >> 4))];
          ids = min(max(id, 0), p.n_pages - 1);
        }
        const int boxes = min(KT / br, (max(u.len, 1) - t * KT + br - 1) / br);   // (those with keys in them)
        const int s = count % C::ST;
        ok = mbar_wait_warp_compact(&empty[s], ((count / C::ST) & 1) ^ 1, wc, values ? SITE_V_EMPTY : SITE_K_EMPTY);
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(&full[s], boxes * br * 128 * C::PANELS);
        uint8_t* dst = ring + s * C::TILE;
        for (int x = 0; x < boxes * split; ++x) {
          const int c = split == 2 ? x >> 1 : x, pn = split == 2 ? x & 1 : 0;
          const int page = __shfl_sync(0xffffffffu, ids, (t - ids_at) * CH + c * (br >> 4)), at = t * KT + c * br;
          const int slot = p.page_shift >= 0 ? at & (p.page_size - 1) : at % p.page_size;
          // keys: panels of KT rows; values: box after box, its panels one after the other
          if (lane == 0) tma_load_5d(dst + (values ? (c * C::PANELS + pn) * br * 128 : pn * C::PANEL + c * br * 128), map, &full[s], 64 * pn, slot, 0, u.hk, page);
        }
        __syncwarp();
      }
    }
  } else if (warp == 6) {
    // ---------------------------------------------------------------- MMAs: the whole warp walks, an elected lane issues
    const bool leader = elect_one() != 0;
    const uint32_t sb = smem_u32(smem);
    constexpr uint32_t idesc_s = umma_idesc_bf16(128, KT, 0, 0), idesc_o = umma_idesc_bf16(128, D, 0, 1);
    const uint64_t d_kmaj = umma_smem_desc(sb, 16, 1024, UMMA_LAYOUT_SW128), d_mn = umma_smem_desc(sb, p.box_rows * 128, 1024, UMMA_LAYOUT_SW128);
    const uint32_t lo_k = desc_lo(d_kmaj), hi_k = desc_hi(d_kmaj), lo_m = desc_lo(d_mn), hi_m = desc_hi(d_mn);
    uint32_t nq = 0, nk = 0, count = 0, nitem = 0;           // count: tiles whose second product has been issued
    bool ok = true;
    const int br = p.box_rows;
    for (; ok && u.r < p.R && u.start < x1; next_unit<KT, ROWS>(p, u)) {
      const int tb = tile_at(u, x0), te = tile_at(u, x1);
      if (tb >= te) continue;
      const bool keys = has_keys(p, u.hk);
      // scores of the `ahead`-th tile from the one whose second product comes next, into the place of its parity: the weights that were
      // there have been read by a product issued before
      auto scores = [&](uint32_t tile) {
        if (keys) {
          const int s = nk % C::ST;
          ok = mbar_wait_warp_compact(&k_full[s], (nk / C::ST) & 1, wc, SITE_K_FULL);
          if (!ok) return;
          ++nk;
          tc_fence_after();
          if (leader) {
#pragma unroll
            for (int kc = 0; kc < D / 16; ++kc)
              umma_ss2(tmem + KT * (tile & 1), lo_k + ((C::OFF_Q + (kc >> 2) * 128 * 128 + (kc & 3) * 32) >> 4), hi_k,
                       lo_k + ((C::OFF_K + s * C::TILE + (kc >> 2) * C::PANEL + (kc & 3) * 32) >> 4), hi_k, idesc_s, kc > 0);
            umma_commit(&k_empty[s]);
          }
          __syncwarp();
        }
        if (leader) umma_commit(&s_full[tile & 1]);          // (without keys too: one phase a tile)
        __syncwarp();
      };
      if (keys) {
        ok = mbar_wait_warp_compact(&q_full, nq & 1, wc, SITE_Q_FULL);
        if (!ok) break;
        ++nq;
      }
      scores(count);
      for (int t = tb; t < te && ok; ++t) {
        if (t + 1 < te) scores(count + 1);
        if (!ok) break;
        ok = mbar_wait_warp_compact(&p_full, count & 1, wc, SITE_P_FULL);
        if (!ok) break;
        const int s = count % C::ST;
        ok = mbar_wait_warp_compact(&v_full[s], (count / C::ST) & 1, wc, SITE_V_FULL);
        if (!ok) break;
        if (t == tb) {
          ok = mbar_wait_warp_compact(&o_free, (nitem & 1) ^ 1, wc, SITE_O_FREE);
          if (!ok) break;
        }
        tc_fence_after();
        if (leader) {
#pragma unroll
          for (int kc = 0; kc < KT / 16; ++kc)
            umma_ts2(tmem + 128, tmem + KT * (count & 1) + 8 * kc,
                     lo_m + ((C::OFF_V + s * C::TILE + ((kc * 16 / br) * C::PANELS * br + kc * 16 % br) * 128) >> 4), hi_m, idesc_o, kc > 0 || t > tb ? 1u : 0u);
          umma_commit(&v_empty[s]);
          umma_commit(&pv_done);
        }
        __syncwarp();
        ++count;
      }
      ++nitem;
    }
  } else if (warp == 7) {
    // ---------------------------------------------------------------- bands.  A tile's: alpha of its keys' positions, then rho of distances
    // pmin - (j0 + KT - 1) and up (what lies outside the vectors belongs to keys that are not seen)
    uint32_t used[2] = {0, 0};
    bool ok = true;
    for (; ok && u.r < p.R && u.start < x1; next_unit<KT, ROWS>(p, u)) {
      const int tb = tile_at(u, x0), te = tile_at(u, x1);
      if (tb >= te) continue;
      const int ctx = u.ctx;
      const BandPlan b = plan_band(p, u);
      if (!b.fast) continue;
      for (int s = 0; s < 2 && ok; ++s) ok = mbar_wait_warp_compact(&band_empty[s], (used[s] & 1) ^ 1, wc, SITE_BAND_EMPTY);
      for (int t = tb; t < te && ok; ++t) {
        const int buf = b.ahead ? (t - tb) & 1 : 0, j0 = t * KT;
        ok = mbar_wait_warp_compact(&band_empty[buf], (used[buf] & 1) ^ 1, wc, SITE_BAND_EMPTY);
        if (!ok) break;
        ++used[buf];
        int at[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int y = lane + 32 * i, j = j0 + y;
          at[i] = j < ctx ? j : j >= u.len ? -1 : p.positions ? min(max(p.positions[u.first + j - ctx], 0), p.Tp - 1) : j;
          if (j0 + KT > ctx) places[buf * KT + y] = 4 * (at[i] < 0 ? y : at[i] - j0);   // (new tokens lie at their positions)
        }
        uint32_t dst = smem_u32(bands + buf * FZ * BAND + lane);
        const int d0 = b.pmin - j0 - (KT - 1) + lane;
        int seen = 0;
        for (int c = 0; c < g; ++c) {
          const int hk = u.hk * g + c;
          if (!((p.frozen[hk >> 5] >> (hk & 31)) & 1)) continue;
          const int64_t head = static_cast<int64_t>(hk) * p.Tp;
#pragma unroll
          for (int i = 0; i < 2; ++i) copy4(dst + 128 * i, p.alpha + head + max(at[i], 0), at[i] >= 0);
#pragma unroll
          for (int i = 0; i < 6; ++i) {
            const int d = d0 + 32 * i;
            const bool in = d >= 0 && d < p.Tp;
            copy4(dst + 256 + 128 * i, p.rho + head + (in ? d : 0), in);
          }
          dst += BAND * 4;
          if (++seen == b.n_frozen) break;
        }
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&band_full[buf])) : "memory");
        mbar_arrive(&band_full[buf]);
      }
    }
    // (copies in flight land before the block ends)
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    // ---------------------------------------------------------------- softmax
    const uint32_t t_s = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    uint32_t count = 0, band0 = 0, band1 = 0;                // tiles so far; bands, in either place
    bool ok = true;
    // (a warp whose wait was abandoned walks on, without storing, until all four leave together)
    for (uint32_t k = 0;; ++k) {
      if (tid == 0) {
        Unit v = work[(k & 1) ^ 1];
        if (k > 0) next_unit<KT, ROWS>(p, v);
        while (v.r < p.R && v.start < x1 && tile_at(v, x0) >= tile_at(v, x1)) next_unit<KT, ROWS>(p, v);
        const bool more = v.r < p.R && v.start < x1;
        work[k & 1] = v;
        range_s[k & 1][0] = more ? tile_at(v, x0) : 0;
        range_s[k & 1][1] = more ? tile_at(v, x1) : -1;
      }
      if (named_bar_or(5, 128, !ok)) break;
      if (tid == 0 && k == 1 && open_unit[0].start >= 0) arrived_s[0] = arrive(p, cut_s, open_unit[0]);   // (the first unit's part is complete)
      const int tb = range_s[k & 1][0], te = range_s[k & 1][1];
      if (te < 0) break;
      const Unit& w = work[k & 1];
      const int ctx = w.ctx, fresh = new_keys(p, w), rows = unit_rows<ROWS>(p, w.many, w.rt);
      const bool keys = has_keys(p, w.hk), there = tid < rows, idle = warp * 32 >= rows;
      int i, hg;
      row_at<ROWS>(p, w.many, w.rt, there ? tid : 0, i, hg);
      const int h = w.hk * g + hg, n = w.first + i;
      const bool frozen = (p.frozen[h >> 5] >> (h & 31)) & 1;
      unsigned long long mask = !there ? 0 : p.masks ? p.masks[n] : (2ull << i) - 1;
      if (fresh < 64) mask &= (1ull << fresh) - 1;
      if (keys) {
        // queries of ordinary rows, zeros elsewhere, as the swizzled tile that TMA would leave
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q) + static_cast<int64_t>(n) * p.q_strides[0] + h * p.q_strides[1];
        const uint32_t base = smem_u32(smem) + C::OFF_Q + tid * 128;   // (panels of 128 rows)
        uint4 x[D / 8];
#pragma unroll
        for (int c = 0; c < D / 8; ++c) x[c] = there && !frozen ? *reinterpret_cast<const uint4*>(q + c * 8) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int c = 0; c < D / 8; ++c) st_shared_v4w(base + (c >> 3) * 128 * 128 + (((c & 7) ^ (tid & 7)) << 4), x[c].x, x[c].y, x[c].z, x[c].w);
        fence_proxy_async_smem();
        warp_arrive(&q_full);
      }
      if (tid == 0) wild_s = 0;
      if (tid < fresh) newpos[tid] = p.positions ? min(max(p.positions[w.first + tid], 0), max(p.Tp - 1, 0)) : max(ctx + tid, 0);
      named_bar_sync(6, 128);
      const BandPlan plan = plan_band(p, w);
      const bool fast = plan.fast;
      const int from = plan.n_frozen > 0 ? min(ctx, plan.pmin + 1) : ctx;   // first key that some row does not see
      bool any_frozen = false;
      uint32_t band_at = 0;                                  // this row's band: alpha of key 0
      int rho_at = 0;                                        // from there to rho of that key
      int pos = 0;
      if (plan.n_frozen > 0) {
        pos = newpos[i];
        if (frozen && (p.positions || p.masks)) {            // (new tokens behind the row's position are not seen)
          for (int c = 0; c < fresh; ++c)
            if (newpos[c] > pos) mask &= ~(1ull << c);
        }
        int slot = 0;                                        // frozen heads of the group before this one
        for (int c = 0; c < hg; ++c) slot += (p.frozen[(w.hk * g + c) >> 5] >> ((w.hk * g + c) & 31)) & 1;
        if (!frozen) slot = 0;
        band_at = smem_u32(bands + min(slot, 2 * FZ - 1) * BAND);
        rho_at = (KT + min(max(pos - plan.pmin, 0), 63) + KT - 1) * 4;
        any_frozen = __any_sync(0xffffffffu, frozen && there);
      }
      const bool read = !fast || (keys && !__all_sync(0xffffffffu, frozen || !there));   // scores out of TMEM
      const float cf = frozen ? LOG16E : p.scale_log16;       // from scores to powers of 16
      float m_ref = -INFINITY, l = 0.0f;
      float factor = cf, offset = 0.0f;                       // a weight is 2^(factor score + offset); to begin with, finite for finite scores
      float limit = -INFINITY;                                // of that exponent, beyond which the reference moves
      for (int t = tb; t < te; ++t, ++count) {
        const bool plain = (t + 1) * KT <= ctx;               // all of its keys were cached before the step
        const int buf = plan.ahead ? (t - tb) & 1 : 0;
        if (fast && !mbar_wait_warp_compact(&band_full[buf], (buf ? band1 : band0) & 1, wc, SITE_BAND_FULL)) ok = false;
        const uint32_t t_p = t_s + KT * (count & 1);
        if (!mbar_wait_warp_compact(&s_full[count & 1], (count >> 1) & 1, wc, SITE_S_FULL)) ok = false;
        tc_fence_after();
        bool waited = t == tb;                                // for the product before this one
        if (!idle) {
          if (any_frozen && !fast) slow_scores(p, w, ctx, t, h, pos, keys, frozen, t_p, newpos);
          // 16 scores at a time, in little code (32 at a time took 152 us where this takes 139, 24 trees with a third of the heads frozen: the
          // loop over tiles has to stay in the instruction cache), and each once: the weights refer to a power of 16 that stays where it is until a
          // score passes it by 2^8, and then goes 2^8 to 2^12 beyond the score, so that what was formed before is moved by an exact factor.
          // From 2^27 powers of 16 on, either way, the next smaller score counts for nothing, but rounding the reference moves it by powers of two
          // (keys masked by a low value, when a row sees no others yet): there the reference is the score as it came, and only
          // scores that equal it have weight.
          uint64_t sum = 0;                                   // two sums
#pragma unroll 1
          for (int c = 0; c < KT / 16; ++c) {
            uint32_t r[16];
            if (read) {
              tmem_ld16(t_p + 16 * c, r);
              tmem_wait_ld();
            }
            if (any_frozen && fast) {
              const uint32_t a = band_at + buf * (FZ * BAND * 4) + 64 * c;
              float x[16], y[16];
#pragma unroll
              for (int e = 0; e < 16; e += 4) ld_shared_v4f(a + 4 * e, x[e], x[e + 1], x[e + 2], x[e + 3]);
              if (plain) {
#pragma unroll
                for (int e = 0; e < 16; ++e) y[e] = ld_shared_f(a + rho_at - 128 * c - 4 * e);
              } else {
                const uint32_t pl = smem_u32(places + buf * KT + 16 * c);
#pragma unroll
                for (int e = 0; e < 16; e += 4) ld_shared_v4f(pl + 4 * e, y[e], y[e + 1], y[e + 2], y[e + 3]);
#pragma unroll
                for (int e = 0; e < 16; ++e) y[e] = ld_shared_f(a - 64 * c + rho_at - __float_as_int(y[e]));
              }
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if (frozen) r[e] = __float_as_uint(x[e] + y[e]);
            }
            if (!plain) {
              // which keys the row sees
              const int rel = ctx - (t * KT + 16 * c);
              const uint32_t sees = rel >= 16 ? ~0u : rel > 0 ? ((1u << rel) - 1) | (static_cast<uint32_t>(mask) << rel) : rel > -64 ? static_cast<uint32_t>(mask >> -rel) : 0u;
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if (!((sees >> e) & 1)) r[e] = 0xff800000u;
            }
            float top = -INFINITY, top1 = -INFINITY;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              top = max3(top, __uint_as_float(r[e]), __uint_as_float(r[e + 1]));
              top1 = max3(top1, __uint_as_float(r[e + 2]), __uint_as_float(r[e + 3]));
            }
            top = fmaxf(top, top1);
            const bool need = fmaf(top, factor, offset) > limit;
            if (__any_sync(0xffffffffu, need)) {
              const float at = __fmul_rn(top, cf);
              const bool far = fabsf(at) >= 134217728.0f;
              const float to = far ? at : ceilf(at) + 2.0f, d = 4.0f * (m_ref - to);
              const float f = !need ? 1.0f : !far && d >= -126.0f ? __int_as_float((127 + static_cast<int>(d)) << 23) : 0.0f;
              if (need) {
                m_ref = to;
                factor = far ? __int_as_float(__float_as_int(4.0f * cf) & 0x7f800000) : 4.0f * cf;   // (a power of two: no rounding)
                offset = -(far ? top * factor : 4.0f * to);
                limit = 8.0f;
              }
              l *= f;
              sum = mul2(sum, pk2(f, f));
              if (!waited && !mbar_wait_warp_compact(&pv_done, (count & 1) ^ 1, wc, SITE_PV_DONE)) ok = false;
              waited = true;
              tc_fence_after();
              tmem_wait_st();
              if (t > tb) {
#pragma unroll 1
                for (int cc = 0; cc < D; cc += 8) {
                  uint32_t x[8];
                  tmem_ld8(t_s + 128 + cc, x);
                  tmem_wait_ld();
#pragma unroll
                  for (int e = 0; e < 8; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * f);
                  tmem_st8(t_s + 128 + cc, x);
                }
              }
#pragma unroll 1
              for (int cc = 0; cc < 8 * c; cc += 8) {         // weights of this tile's first keys
                uint32_t x[8];
                tmem_ld8(t_p + cc, x);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = pack_bf16x2(__uint_as_float(x[e] << 16) * f, __uint_as_float(x[e] & 0xffff0000u) * f);
                tmem_st8(t_p + cc, x);
              }
            }
            const uint64_t cf2 = pk2(factor, factor), neg2 = pk2(offset, offset);
            uint32_t pk[8];                                   // (weights take the place of scores that have been read)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float a0, a1;
              upk2(fma2(pk2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])), cf2, neg2), a0, a1);
              a0 = ex2_approx(a0);
              a1 = ex2_approx(a1);
              sum = add2(sum, pk2(a0, a1));
              pk[e] = pack_bf16x2(a0, a1);
            }
            tmem_st8(t_p + 8 * c, pk);
          }
          float l0, l1;
          upk2(sum, l0, l1);
          l += l0 + l1;
        }
        if (fast) {                                           // (the band has been read)
          warp_arrive(&band_empty[buf]);
          if (buf) ++band1;
          else ++band0;
        }
        if (!waited && !mbar_wait_warp_compact(&pv_done, (count & 1) ^ 1, wc, SITE_PV_DONE)) ok = false;   // (each phase is waited for in turn)
        if ((t + 1) * KT > from) {
          if (!mbar_wait_warp_compact(&v_full[count % C::ST], (count / C::ST) & 1, wc, SITE_V_FULL)) ok = false;
          if (clean_values<D>(p.box_rows, t * KT, from, w.len, smem_u32(smem) + C::OFF_V + (count % C::ST) * C::TILE, tid)) wild_s = 1;
          fence_proxy_async_smem();
        }
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(&p_full);
      }
      if (!mbar_wait_warp_compact(&pv_done, (count & 1) ^ 1, wc, SITE_PV_DONE)) ok = false;   // (behind it all four warps have set wild_s)
      tc_fence_after();
      const bool whole = tb == 0 && te == w.tiles;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;          // (NaN stays NaN)
      float* part = slot_of(blockIdx.x, w.start);
      if (!idle) {
#pragma unroll 1
        for (int f0 = 0; f0 < D; f0 += 32) {
          uint32_t r[32];
          __syncwarp();
          tmem_ld32(t_s + 128 + f0, r);
          tmem_wait_ld();
          if (wild_s && there) {
            for (int j = max(max(tb * KT, from), 0); j < min(te * KT, w.len); ++j) {
              if (j < ctx ? frozen && j > pos : !((mask >> (j - ctx)) & 1)) continue;
              const int page = min(max(p.block_table[static_cast<int64_t>(w.r) * p.max_pages + j / p.page_size], 0), p.n_pages - 1);
              const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v) + page * p.v_strides[0] + w.hk * p.v_strides[1] + (j % p.page_size) * p.v_strides[2] + f0;
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                const float x = __bfloat162float(v[e]);
                if (!isfinite(x)) r[e] = __float_as_uint(__uint_as_float(r[e]) + x);
              }
            }
          }
          // a warp's 32 rows by way of its share of the queries' place, so that a store covers whole lines (row by row they took 20000 clk a
          // part)
          const uint32_t stage = smem_u32(smem) + C::OFF_Q + warp * 4096;
          if (whole) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
              st_shared_v4w(stage + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4), pack_bf16x2(__uint_as_float(r[8 * c]) * inv, __uint_as_float(r[8 * c + 1]) * inv),
                            pack_bf16x2(__uint_as_float(r[8 * c + 2]) * inv, __uint_as_float(r[8 * c + 3]) * inv),
                            pack_bf16x2(__uint_as_float(r[8 * c + 4]) * inv, __uint_as_float(r[8 * c + 5]) * inv),
                            pack_bf16x2(__uint_as_float(r[8 * c + 6]) * inv, __uint_as_float(r[8 * c + 7]) * inv));
            __syncwarp();
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int row = c * 8 + (lane >> 2), q = lane & 3;
              const long long off = __shfl_sync(0xffffffffu, static_cast<long long>(n) * p.o_strides[0] + h * p.o_strides[1], row);
              float4 x;
              ld_shared_v4f(stage + row * 64 + ((q ^ ((row >> 1) & 3)) << 4), x.x, x.y, x.z, x.w);
              if (warp * 32 + row < rows && ok) *reinterpret_cast<float4*>(static_cast<__nv_bfloat16*>(p.O) + off + f0 + 8 * q) = x;
            }
          } else {
#pragma unroll
            for (int c = 0; c < 8; ++c) st_shared_v4w(stage + lane * 128 + ((c ^ (lane & 7)) << 4), r[4 * c], r[4 * c + 1], r[4 * c + 2], r[4 * c + 3]);
            __syncwarp();
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const int row = c * 4 + (lane >> 3), q = lane & 7;
              float4 x;
              ld_shared_v4f(stage + row * 128 + ((q ^ (row & 7)) << 4), x.x, x.y, x.z, x.w);
              if (warp * 32 + row < rows && ok) *reinterpret_cast<float4*>(part + (warp * 32 + row) * D + f0 + 4 * q) = x;
            }
          }
        }
      }
      if (there && ok) {
        if (!whole) {
          part[p.max_rows * D + tid] = m_ref;
          part[p.max_rows * (D + 1) + tid] = l;
        } else if (p.LSE) {
          p.LSE[static_cast<int64_t>(n) * p.H + h] = frozen ? 0.0f : l == 0.0f ? -INFINITY : natural_lse(m_ref, l);
        }
      }
      if (!whole && tid == 0) open_unit[x0 >= w.start ? 0 : 1] = Part{w.start, w.start + w.tiles - 1, w.first, w.many, w.rt, w.hk};
      tc_fence_before();
      warp_arrive(&o_free);
    }
  }

  // ------------------------------------------------------------------ teardown; then units that lie in several blocks
  __syncwarp();
  if (abort_s) {
    // a wait gave up: copies and MMAs in flight land before the block's memory is released, and what it did not come to is reported
    // all the same, so that the counters end at zero
    for (int k = 0; k < 64; ++k) __nanosleep(20000);
    if (tid == 0 && x0 < x1) {
      for (Unit v = work[2]; v.r < p.R && v.start < x1; next_unit<KT, ROWS>(p, v)) {
        const int tb = tile_at(v, x0), te = tile_at(v, x1);
        if (tb < te && te - tb < v.tiles) open_unit[x0 >= v.start ? 0 : 1] = Part{v.start, v.start + v.tiles - 1, v.first, v.many, v.rt, v.hk};
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 6) tmem_dealloc(tmem, 256);
  if (open_unit[0].start < 0 && open_unit[1].start < 0) return;
  if (tid < 2 && open_unit[tid].start >= 0 && arrived_s[tid] < 0) arrived_s[tid] = arrive(p, cut_s, open_unit[tid]);
  __syncthreads();
  // (a run's first unit has mostly been reported long before, so that its other blocks join it and this one its last)
  for (int k = 0; k < 2; ++k) {
    const Part unit = open_unit[k];
    if (unit.start < 0 || arrived_s[k] != 1) continue;
    const int first = cut_s.run_of(unit.start), last = cut_s.run_of(unit.last);
    __threadfence();
    join<D, ROWS, true, 8, 1>(p, unit, p.max_rows, last - first + 1, [&](int i) { return slot_of(first + i, unit.start); }, nullptr, tid, NT);
  }
}

template <int D>
cudaError_t launch(const CUtensorMap& mk, const CUtensorMap& mv, const CacheAttnParams& p, int num_sms, cudaStream_t st) {
  static SmemLimit limit;
  const cudaError_t e = raise_smem(saf_cache_wide_kernel<D>, Cfg<D>::SMEM, limit);
  if (e != cudaSuccess) return e;
  return launch_pdl(PDL_REST, saf_cache_wide_kernel<D>, BLOCKS * num_sms, NT, Cfg<D>::SMEM, st, mk, mv, p);
}

}  // namespace

CacheAttnForm cache_wide_form(int max_new, int kv_group, int D, int page_size, int max_len) {
  CacheAttnForm f;
  f.wide = true;
  f.tile_tokens = ROWS / kv_group;
  f.max_rows = std::min(max_new, f.tile_tokens) * kv_group;
  f.halves_k = 1;
  f.halves_v = D == 128 ? 2 : 1;
  f.box_rows = 16;
  while (f.box_rows < KT && page_size % (2 * f.box_rows) == 0) f.box_rows *= 2;
  f.tiles = static_cast<int64_t>((max_new - 1) / f.tile_tokens + 1) * ((max_len - 1) / KT + 1 + EXTRA<128>);
  return f;
}

size_t cache_wide_workspace(int num_sms) { return sizeof(float) * 2 * BLOCKS * num_sms * part_size(ROWS, 128); }

cudaError_t launch_cache_wide(const CUtensorMap& mk, const CUtensorMap& mv, const CacheAttnParams& p, int num_sms, cudaStream_t st) {
  if (p.D == 64) return launch<64>(mk, mv, p, num_sms, st);
  if (p.D == 96) return launch<96>(mk, mv, p, num_sms, st);
  return launch<128>(mk, mv, p, num_sms, st);
}

}  // namespace saf
