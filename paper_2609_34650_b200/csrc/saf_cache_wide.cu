// Attention of a step's new tokens over a paged cache where many rows share a key: drafted trees and chains on grouped heads.
//
// The mathematics is saf_cache_attn.cu's.  A unit here is one request, one cached head and up to 128 rows (whole new tokens with all
// query heads of the group, head by head), its tiles 128 keys, and a block takes one run of the line of all tiles.  With 16 rows
// a unit, 128 rows would read the cache eight times out of L2 and issue the 16-row instructions as often; on tcgen05 a tile takes
// the tensor core about 1000 clk, whatever the rows, of the 2800 that DRAM needs for its 64 KB (head dimension 128).  Two blocks an SM, so that one's
// chain of scores, softmax and second product runs while the other's waits.
//
// Per block (320 threads): warps 0-7 compute, warp 8 fetches pages by TMA, warp 9 issues the MMAs and owns TMEM.  Two compute threads
// share a row (= TMEM lane), each with 64 keys of a tile; TMEM columns [0,128) S (fp32), then weights (bf16 pairs in [0,32) and
// [64,96)), [128,256) O.  Frozen rows replace their scores by alpha + rho out of a band that is copied in one tile ahead: 128
// preferences of keys and 256 of distances for each of up to FZ frozen heads; other tiles (those that hold new tokens, more
// frozen heads, positions far apart) take them from global memory in a pass of their own.
#include "saf_cache_attn.cuh"

namespace saf {
namespace {

constexpr int ROWS = 128, KT = 128, W = 10, NT = 32 * W, FZ = 4;
constexpr int SINGLE_TILES = 8;     // tiles up to which a block takes a whole unit where there are no more units than blocks
constexpr int BLOCKS = 2;           // blocks an SM

template <int D>
struct Cfg {
  static constexpr int PANELS = D == 64 ? 1 : 2;             // 64 features: 128-byte rows, one swizzle atom
  static constexpr int PANEL = KT * 128;
  static constexpr int TILE = PANELS * PANEL;
  static constexpr int ST = D == 64 ? 2 : 1;                 // tiles of keys, and of values, in shared memory
  static constexpr int OFF_Q = 0, OFF_K = TILE, OFF_V = OFF_K + ST * TILE, OFF_TAB = OFF_V + ST * TILE;
  // floats: bands [2][FZ][384], row maxima [2][2][128], row sums [2][128]; ints: positions of new tokens [64], frozen heads [FZ]
  static constexpr int TAB = 2 * FZ * 384 + 512 + 256 + 64 + FZ;
  static constexpr int SMEM = OFF_TAB + TAB * 4 + 1024;
  static constexpr int HALF = D == 64 ? 32 : 64;             // output features of a compute thread
};

enum WideSite { SITE_K_EMPTY = 111, SITE_V_EMPTY, SITE_Q_FULL, SITE_K_FULL, SITE_P_FULL, SITE_V_FULL, SITE_O_FREE, SITE_S_FULL, SITE_PV_DONE };

__device__ __forceinline__ void copy4(uint32_t dst, const float* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ bool wild16(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

template <int D>
__global__ void __launch_bounds__(NT, BLOCKS)
saf_cache_wide_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const __grid_constant__ CacheAttnParams p) {
  using C = Cfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], q_full, s_full, p_full, pv_done, o_free;
  __shared__ Part open_unit[2];                              // units that go on in other blocks: the run's first, its last
  __shared__ int red[3][W], arrived_s[2], abort_s, wild_s, frozen_s;
  __shared__ uint32_t tmem_slot;
  float* bands = reinterpret_cast<float*>(smem + C::OFF_TAB);
  float* xch = bands + 2 * FZ * 384;                         // [tile parity][half][row]
  float* lx = xch + 512;                                     // [half][row]
  int* newpos = reinterpret_cast<int*>(lx + 256);
  int* fheads = newpos + 64;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const WaitCtx wc{&abort_s, p.status, p.wait_limit_ns};
  if (tid == 0) {
    abort_s = 0;
    open_unit[0].start = open_unit[1].start = -1;
    for (int s = 0; s < 2; ++s) {
      mbar_init(&k_full[s], 1);
      mbar_init(&k_empty[s], 1);
      mbar_init(&v_full[s], 1);
      mbar_init(&v_empty[s], 1);
    }
    mbar_init(&q_full, 8);                                   // (one arrival per compute warp)
    mbar_init(&s_full, 1);
    mbar_init(&p_full, 8);
    mbar_init(&pv_done, 1);
    mbar_init(&o_free, 8);
    mbar_fence_init();
    tma_prefetch_desc(&mk);
    tma_prefetch_desc(&mv);
  }
  if (warp == 9) {
    tmem_alloc(&tmem_slot, 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_wait();
  pdl_launch_dependents();

  Cut cut;
  Unit u;
  int x0, x1;
  place_run<KT, ROWS, W, 1, SINGLE_TILES>(p, smem, red, 0, cut, x0, x1, u);
  __syncthreads();                                           // the sums have been read: tiles may be fetched over them
  const int part_floats = part_size(p.max_rows, D), g = p.kv_group;
  auto slot_of = [&](int block, const Part& unit) {
    return p.workspace + (static_cast<int64_t>(block) * 2 + (cut.start(block) >= unit.start ? 0 : 1)) * part_floats;
  };

  if (x0 >= x1) {
  } else if (warp == 8) {
    // ---------------------------------------------------------------- pages
    uint32_t nk = 0, nv = 0;
    bool ok = true;
    const int br = p.box_rows;
    for (; ok && u.r < p.R && u.start < x1; next_unit<KT, ROWS>(p, u)) {
      const int tb = tile_at(u, x0), te = tile_at(u, x1);
      const bool keys = has_keys(p, u.hk);
      int ids = 0, ids_at = tb - 4;
      for (int t = tb; t < te && ok; ++t) {
        if (t - ids_at >= 4) {                               // lane l: page of the 16 keys number 8 t + l
          ids_at = t;
          const int c = t * 8 + lane;
          int id = 0;
          if (c * 16 < max(u.len, 1)) id = p.block_table[static_cast<int64_t>(u.r) * p.max_pages + (p.page_shift >= 0 ? c >> p.page_shift : c / (p.page_size >> 4))];
          ids = min(max(id, 0), p.n_pages - 1);
        }
        const int boxes = min(KT / br, (max(u.len, 1) - t * KT + br - 1) / br);   // (those with keys in them)
        for (int half = keys ? 0 : 1; half < 2 && ok; ++half) {
          uint32_t& n = half ? nv : nk;
          const int s = n % C::ST;
          uint64_t* full = half ? &v_full[s] : &k_full[s];
          ok = mbar_wait_warp(half ? &v_empty[s] : &k_empty[s], ((n / C::ST) & 1) ^ 1, wc, half ? SITE_V_EMPTY : SITE_K_EMPTY);
          if (!ok) break;
          ++n;
          if (lane == 0) mbar_expect_tx(full, boxes * br * 128 * C::PANELS);
          uint8_t* dst = smem + (half ? C::OFF_V : C::OFF_K) + s * C::TILE;
          for (int c = 0; c < boxes; ++c) {
            const int page = __shfl_sync(0xffffffffu, ids, (t - ids_at) * 8 + c * (br >> 4)), at = t * KT + c * br;
            const int slot = p.page_shift >= 0 ? at & (p.page_size - 1) : at % p.page_size;
            if (lane == 0)
#pragma unroll
              for (int pn = 0; pn < C::PANELS; ++pn) tma_load_5d(dst + pn * C::PANEL + c * br * 128, half ? &mv : &mk, full, 64 * pn, slot, 0, u.hk, page);
          }
          __syncwarp();
        }
      }
    }
  } else if (warp == 9) {
    // ---------------------------------------------------------------- MMAs: the whole warp walks, an elected lane issues
    const bool leader = elect_one() != 0;
    const uint32_t sb = smem_u32(smem);
    constexpr uint32_t idesc_s = umma_idesc_bf16(128, 128, 0, 0), idesc_o = umma_idesc_bf16(128, D, 0, 1);
    const uint64_t d_kmaj = umma_smem_desc(sb, 16, 1024, UMMA_LAYOUT_SW128), d_mn = umma_smem_desc(sb, C::PANEL, 1024, UMMA_LAYOUT_SW128);
    const uint32_t lo_k = desc_lo(d_kmaj), hi_k = desc_hi(d_kmaj), lo_m = desc_lo(d_mn), hi_m = desc_hi(d_mn);
    uint32_t nq = 0, nk = 0, nv = 0, np = 0, nitem = 0;
    bool ok = true;
    for (; ok && u.r < p.R && u.start < x1; next_unit<KT, ROWS>(p, u)) {
      const int tb = tile_at(u, x0), te = tile_at(u, x1);
      if (tb >= te) continue;
      const bool keys = has_keys(p, u.hk);
      if (keys) {
        ok = mbar_wait_warp(&q_full, nq & 1, wc, SITE_Q_FULL);
        if (!ok) break;
        ++nq;
      }
      for (int t = tb; t < te && ok; ++t) {
        if (keys) {
          const int s = nk % C::ST;
          ok = mbar_wait_warp(&k_full[s], (nk / C::ST) & 1, wc, SITE_K_FULL);
          if (!ok) break;
          ++nk;
          tc_fence_after();
          if (leader) {
#pragma unroll
            for (int kc = 0; kc < D / 16; ++kc) {
              const uint32_t off = ((kc >> 2) * C::PANEL + (kc & 3) * 32) >> 4;
              umma_ss2(tmem, lo_k + (C::OFF_Q >> 4) + off, hi_k, lo_k + ((C::OFF_K + s * C::TILE) >> 4) + off, hi_k, idesc_s, kc > 0);
            }
            umma_commit(&s_full);
            umma_commit(&k_empty[s]);
          }
          __syncwarp();
        }
        ok = mbar_wait_warp(&p_full, np & 1, wc, SITE_P_FULL);
        if (!ok) break;
        ++np;
        const int s = nv % C::ST;
        ok = mbar_wait_warp(&v_full[s], (nv / C::ST) & 1, wc, SITE_V_FULL);
        if (!ok) break;
        ++nv;
        if (t == tb) {
          ok = mbar_wait_warp(&o_free, (nitem & 1) ^ 1, wc, SITE_O_FREE);
          if (!ok) break;
        }
        tc_fence_after();
        if (leader) {
#pragma unroll
          for (int kc = 0; kc < 8; ++kc)                      // (bf16 pairs: keys 0-63 in columns [0,32), keys 64-127 in [64,96))
            umma_ts2(tmem + 128, tmem + 8 * kc + (kc >= 4 ? 32u : 0u), lo_m + ((C::OFF_V + s * C::TILE) >> 4) + 128 * kc, hi_m, idesc_o, kc > 0 || t > tb ? 1u : 0u);
          umma_commit(&v_empty[s]);
          umma_commit(&pv_done);
        }
        __syncwarp();
      }
      ++nitem;
    }
  } else {
    // ---------------------------------------------------------------- softmax
    const int hh = warp >> 2, rowl = (warp & 3) * 32 + lane, pair_bar = 1 + (warp & 3);
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lane_base + 64 * hh, t_o = tmem + lane_base + 128 + C::HALF * hh;
    uint32_t ns = 0, npv = 0, nv = 0;
    bool ok = true;
    // (a warp whose wait was abandoned walks on, without storing, until all eight leave together)
    for (; u.r < p.R && u.start < x1; next_unit<KT, ROWS>(p, u)) {
      const int tb = tile_at(u, x0), te = tile_at(u, x1);
      if (tb >= te) continue;
      if (named_bar_or(5, 256, !ok)) break;
      const int rows = unit_rows<ROWS>(p, u.many, u.rt), ctx = u.len - u.many, tokens = rows / g;
      const bool keys = has_keys(p, u.hk), there = rowl < rows;
      int i, hg;
      row_at<ROWS>(p, u.many, u.rt, there ? rowl : 0, i, hg);
      const int h = u.hk * g + hg, n = u.first + i;
      const bool frozen = (p.frozen[h >> 5] >> (h & 31)) & 1;
      const unsigned long long mask = !there ? 0 : p.masks ? p.masks[n] : (2ull << i) - 1;
      if (keys) {
        // queries of ordinary rows, zeros elsewhere, as the swizzled tile that TMA would leave
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q) + static_cast<int64_t>(n) * p.q_strides[0] + h * p.q_strides[1];
        constexpr int CH = D == 64 ? 4 : 8;
        uint4 x[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int f = (hh * CH + c) * 8;
          x[c] = there && !frozen && f < D ? *reinterpret_cast<const uint4*>(q + f) : make_uint4(0, 0, 0, 0);
        }
        const uint32_t base = smem_u32(smem) + C::OFF_Q + (D == 64 ? 0 : hh * C::PANEL) + rowl * 128;
#pragma unroll
        for (int c = 0; c < CH; ++c) st_shared_v4w(base + ((((D == 64 ? hh * CH : 0) + c) ^ (rowl & 7)) << 4), x[c].x, x[c].y, x[c].z, x[c].w);
        fence_proxy_async_smem();
        warp_arrive(&q_full);
      }
      // frozen heads of the group, positions of the new tokens
      if (tid == 0) {
        int count = 0;
        for (int k = 0; k < g; ++k) {
          const int hk = u.hk * g + k;
          if ((p.frozen[hk >> 5] >> (hk & 31)) & 1) {
            if (count < FZ) fheads[count] = hk;
            ++count;
          }
        }
        frozen_s = count;
        wild_s = 0;
      }
      if (tid < u.many) newpos[tid] = p.positions ? min(max(p.positions[u.first + tid], 0), max(p.Tp - 1, 0)) : ctx + tid;
      named_bar_sync(6, 256);
      const int n_frozen = frozen_s;
      int pos = 0, pmin = 0, span = 0, fslot = 0;
      bool fast = false;
      if (n_frozen > 0) {
        pos = max(newpos[i], 0);
        int lo = 0x7fffffff, hi = 0;
        for (int k = lane; k < tokens; k += 32) {
          const int x = max(newpos[u.rt * p.tile_tokens + k], 0);
          lo = min(lo, x);
          hi = max(hi, x);
        }
        pmin = __reduce_min_sync(0xffffffffu, lo);
        span = __reduce_max_sync(0xffffffffu, hi) - pmin;
        fast = n_frozen <= FZ && pmin >= ctx && span < 128;
        for (int k = 0; k < min(n_frozen, FZ); ++k)
          if (fheads[k] == h) fslot = k;
      }
      const bool any_frozen = __any_sync(0xffffffffu, frozen && there);
      const float cf = frozen ? 1.0f : p.scale_log2;          // (frozen scores are formed in powers of two)
      const float* arow = p.alpha + static_cast<int64_t>(h) * p.Tp;
      const float* rrow = p.rho + static_cast<int64_t>(h) * p.Tp;
      // a tile's band: alpha of its keys, rho of distances pmin - (j0 + 127) and up
      auto fetch_band = [&](int t) {
        const int j0 = t * KT;
        for (int x = tid; x < n_frozen * 384; x += 256) {
          const int s = x / 384, y = x - s * 384;
          const int64_t head = static_cast<int64_t>(fheads[s]) * p.Tp;
          const uint32_t dst = smem_u32(bands + ((t & 1) * FZ + s) * 384 + y);
          if (y < 128) copy4(dst, p.alpha + head + j0 + y);
          else if (y - 128 <= span + 127) copy4(dst, p.rho + head + pmin - j0 - 127 + (y - 128));
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
      auto plain_tile = [&](int t) { return (t + 1) * KT <= ctx; };   // all of its keys were cached before the step
      if (fast && plain_tile(tb)) fetch_band(tb);
      float m_ref = -INFINITY, l = 0.0f;
      for (int t = tb; t < te; ++t) {
        const int j0 = t * KT;
        const bool plain = plain_tile(t);
        if (fast && plain) {
          asm volatile("cp.async.wait_all;" ::: "memory");
          named_bar_sync(6, 256);                             // (the band of this tile is there, that of the one before has been read)
          if (t + 1 < te && plain_tile(t + 1)) fetch_band(t + 1);
        }
        if (keys) {
          if (!mbar_wait_warp(&s_full, ns & 1, wc, SITE_S_FULL)) ok = false;
          ++ns;
        }
        if (t > tb) {
          if (!mbar_wait_warp(&pv_done, npv & 1, wc, SITE_PV_DONE)) ok = false;
          ++npv;
        }
        tc_fence_after();
        if (!plain || (any_frozen && !fast)) {
          // scores that need looking at one by one go back to where they came from
#pragma unroll 1
          for (int cc = 0; cc < 4; ++cc) {
            uint32_t r[16];
            if (keys) {
              tmem_ld16(t_s + 16 * cc, r);
              tmem_wait_ld();
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const int j = j0 + 64 * hh + 16 * cc + e, back = j - ctx;
              const bool sees = j < u.len && (back < 0 || ((mask >> back) & 1));
              float x = keys ? __uint_as_float(r[e]) : 0.0f;
              if (frozen && sees) {
                const int pj = back < 0 ? j : newpos[back];
                x = pj <= pos ? (arow[pj] + rrow[pos - pj]) * LOG2E : -INFINITY;
              }
              r[e] = __float_as_uint(sees ? x : -INFINITY);
            }
            tmem_st16(t_s + 16 * cc, r);
          }
          tmem_wait_st();
        }
        uint32_t r0[32], r1[32];
        if (keys || !plain || !fast) {
          tmem_ld32(t_s, r0);
          tmem_ld32(t_s + 32, r1);
          tmem_wait_ld();
        }
        if (any_frozen && fast && plain) {
          const float* a = bands + ((t & 1) * FZ + fslot) * 384 + 64 * hh;
          const float* b = bands + ((t & 1) * FZ + fslot) * 384 + 128 + min(max(pos - pmin, 0), 127) + 127 - 64 * hh;
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float4 a0 = *reinterpret_cast<const float4*>(a + e), a1 = *reinterpret_cast<const float4*>(a + 32 + e);
            const float v0[4] = {a0.x, a0.y, a0.z, a0.w}, v1[4] = {a1.x, a1.y, a1.z, a1.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float s0 = (v0[k] + b[-e - k]) * LOG2E, s1 = (v1[k] + b[-32 - e - k]) * LOG2E;
              if (frozen) {
                r0[e + k] = __float_as_uint(s0);
                r1[e + k] = __float_as_uint(s1);
              }
            }
          }
        }
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          mx0 = max3(mx0, __uint_as_float(r0[e]), __uint_as_float(r0[e + 1]));
          mx1 = max3(mx1, __uint_as_float(r1[e]), __uint_as_float(r1[e + 1]));
        }
        float mx = fmaxf(mx0, mx1);
        float* xs = xch + (t & 1) * 256;
        xs[hh * 128 + rowl] = mx;
        named_bar_sync(pair_bar, 64);
        mx = fmaxf(mx, xs[(hh ^ 1) * 128 + rowl]);
        // the reference follows the maximum where that has grown by more than 2^8
        const float m_new = fmaxf(m_ref, mx * cf);
        const bool need = m_new - m_ref > 8.0f;               // (from -inf: always; -inf to -inf: NaN, no)
        if (t == tb) {
          m_ref = m_new;
        } else if (__any_sync(0xffffffffu, need)) {
          const float f = need ? ex2_approx(m_ref - m_new) : 1.0f;
          l *= f;
          if (need) m_ref = m_new;
#pragma unroll
          for (int cc = 0; cc < C::HALF / 16; ++cc) {
            uint32_t r[16];
            tmem_ld16(t_o + 16 * cc, r);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * f);
            tmem_st16(t_o + 16 * cc, r);
          }
        }
        const float neg_m = m_ref == -INFINITY ? 0.0f : -m_ref;
        float l0 = 0.0f, l1 = 0.0f;
        uint32_t pk[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float a0 = ex2_approx(fmaf(__uint_as_float(r0[2 * e]), cf, neg_m)), a1 = ex2_approx(fmaf(__uint_as_float(r0[2 * e + 1]), cf, neg_m));
          l0 += a0 + a1;
          pk[e] = pack_bf16x2(a0, a1);
        }
        tmem_st16(t_s, pk);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float a0 = ex2_approx(fmaf(__uint_as_float(r1[2 * e]), cf, neg_m)), a1 = ex2_approx(fmaf(__uint_as_float(r1[2 * e + 1]), cf, neg_m));
          l1 += a0 + a1;
          pk[e] = pack_bf16x2(a0, a1);
        }
        tmem_st16(t_s + 16, pk);
        l += l0 + l1;
        if (!plain) {
          // values behind the last key are whatever was there, and those of new tokens, which not every row sees, may be NaN or
          // infinite: both are zeroed for the product, the second kind added to the rows that see it at the end
          if (!mbar_wait_warp(&v_full[nv % C::ST], (nv / C::ST) & 1, wc, SITE_V_FULL)) ok = false;
          const uint32_t vs = smem_u32(smem) + C::OFF_V + (nv % C::ST) * C::TILE;
          bool wild = false;
          for (int c = tid; c < C::TILE / 16; c += 256) {
            const int j = j0 + ((c >> 3) & (KT - 1));
            if (j < ctx) continue;
            const uint32_t addr = vs + c * 16;
            uint32_t w[4];
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
            if (j >= u.len) {
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
          if (wild) wild_s = 1;
          fence_proxy_async_smem();
        }
        ++nv;
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(&p_full);
      }
      lx[hh * 128 + rowl] = l;
      named_bar_sync(6, 256);
      l += lx[(hh ^ 1) * 128 + rowl];
      if (!mbar_wait_warp(&pv_done, npv & 1, wc, SITE_PV_DONE)) ok = false;
      ++npv;
      tc_fence_after();
      const Part me{u.start, u.start + u.tiles - 1, u.first, u.many, u.rt, u.hk};
      const bool whole = tb == 0 && te == u.tiles;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;          // (NaN stays NaN)
      float* part = slot_of(blockIdx.x, me);
#pragma unroll
      for (int cc = 0; cc < C::HALF / 32; ++cc) {
        const int f0 = C::HALF * hh + 32 * cc;
        if (f0 >= D) break;
        uint32_t r[32];
        __syncwarp();
        tmem_ld32(t_o + 32 * cc, r);
        tmem_wait_ld();
        if (wild_s && there) {
          for (int back = max(tb * KT - ctx, 0); back < u.many && ctx + back < min(te * KT, u.len); ++back) {
            if (ctx + back < 0 || !((mask >> back) & 1) || (frozen && newpos[back] > pos)) continue;
            const int j = ctx + back;
            const int page = min(max(p.block_table[static_cast<int64_t>(u.r) * p.max_pages + j / p.page_size], 0), p.n_pages - 1);
            const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v) + page * p.v_strides[0] + u.hk * p.v_strides[1] + (j % p.page_size) * p.v_strides[2] + f0;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float x = __bfloat162float(v[e]);
              if (!isfinite(x)) r[e] = __float_as_uint(__uint_as_float(r[e]) + x);
            }
          }
        }
        if (there && ok && whole) {
          __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.O) + static_cast<int64_t>(n) * p.o_strides[0] + h * p.o_strides[1] + f0;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint4 x;
            x.x = pack_bf16x2(__uint_as_float(r[8 * k]) * inv, __uint_as_float(r[8 * k + 1]) * inv);
            x.y = pack_bf16x2(__uint_as_float(r[8 * k + 2]) * inv, __uint_as_float(r[8 * k + 3]) * inv);
            x.z = pack_bf16x2(__uint_as_float(r[8 * k + 4]) * inv, __uint_as_float(r[8 * k + 5]) * inv);
            x.w = pack_bf16x2(__uint_as_float(r[8 * k + 6]) * inv, __uint_as_float(r[8 * k + 7]) * inv);
            *reinterpret_cast<uint4*>(o + 8 * k) = x;
          }
        } else if (there && ok) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            *reinterpret_cast<float4*>(part + rowl * D + f0 + 4 * k) =
                make_float4(__uint_as_float(r[4 * k]), __uint_as_float(r[4 * k + 1]), __uint_as_float(r[4 * k + 2]), __uint_as_float(r[4 * k + 3]));
        }
      }
      if (hh == 0 && there && ok) {
        if (!whole) {
          part[p.max_rows * D + rowl] = m_ref;
          part[p.max_rows * (D + 1) + rowl] = l;
        } else if (p.LSE) {
          p.LSE[static_cast<int64_t>(n) * p.H + h] = frozen ? 0.0f : l == 0.0f ? -INFINITY : (m_ref + log2f(l)) * LN2;
        }
      }
      if (!whole && tid == 0) open_unit[x0 >= u.start ? 0 : 1] = me;
      tc_fence_before();
      warp_arrive(&o_free);
    }
  }

  // ------------------------------------------------------------------ teardown; then units that lie in several blocks
  __syncwarp();
  if (abort_s) {
    // a wait gave up: copies and MMAs in flight land before the block's memory is released
    for (int k = 0; k < 64; ++k) __nanosleep(20000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 9) tmem_dealloc(tmem, 256);
  if (open_unit[0].start < 0 && open_unit[1].start < 0) return;
  if (tid < 2 && open_unit[tid].start >= 0) {
    const Part& unit = open_unit[tid];
    const int first = cut.run_of(unit.start), last = cut.run_of(unit.last);
    __threadfence();                                          // (the block's parts, which the barrier put before this)
    const bool end = atomicAdd(p.counters + first, 1) == last - first;
    if (end) p.counters[first] = 0;
    arrived_s[tid] = end;
    __threadfence();
  }
  __syncthreads();
  for (int k = 0; k < 2; ++k) {
    const Part unit = open_unit[k];
    if (unit.start < 0 || !arrived_s[k]) continue;
    const int first = cut.run_of(unit.start), last = cut.run_of(unit.last);
    join<D, ROWS, true>(p, unit, p.max_rows, last - first + 1, [&](int i) { return slot_of(first + i, unit); }, nullptr, tid, NT);
  }
}

template <int D>
cudaError_t launch(const CUtensorMap& mk, const CUtensorMap& mv, const CacheAttnParams& p, int num_sms, cudaStream_t st) {
  const cudaError_t e = cudaFuncSetAttribute(saf_cache_wide_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::SMEM);
  if (e != cudaSuccess) return e;
  return launch_pdl(PDL_REST, saf_cache_wide_kernel<D>, BLOCKS * num_sms, NT, Cfg<D>::SMEM, st, mk, mv, p);
}

}  // namespace

CacheAttnForm cache_wide_form(int max_new, int kv_group, int D, int page_size, int max_len, int num_sms) {
  CacheAttnForm f;
  f.wide = true;
  f.tile_tokens = ROWS / kv_group;
  f.max_rows = std::min(max_new, f.tile_tokens) * kv_group;
  f.halves = 1;
  f.box_rows = 16;
  while (f.box_rows < KT && page_size % (2 * f.box_rows) == 0) f.box_rows *= 2;
  f.blocks = BLOCKS * num_sms;
  f.parts = 2 * f.blocks;
  f.part_bytes = part_size(f.max_rows, D) * sizeof(float);
  f.tiles = static_cast<int64_t>((max_new - 1) / f.tile_tokens + 1) * ((max_len - 1) / KT + 1);
  return f;
}

cudaError_t launch_cache_wide(const CUtensorMap& mk, const CUtensorMap& mv, const CacheAttnParams& p, int num_sms, cudaStream_t st) {
  if (p.D == 64) return launch<64>(mk, mv, p, num_sms, st);
  if (p.D == 96) return launch<96>(mk, mv, p, num_sms, st);
  return launch<128>(mk, mv, p, num_sms, st);
}

}  // namespace saf
