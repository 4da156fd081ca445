// Attention of a step's new tokens over a paged cache, ordinary and frozen heads side by side.
//
//   O_i = sum_j e^{s_ij} V_j / sum_j e^{s_ij} over the keys j that row i sees; s_ij = scale q_i k_j (ordinary head) or
//   alpha(p_j) + rho(p_i - p_j) (frozen head), running maximum and sum in fp32, in powers of 16.
//
// Every key and value is read once for up to 16 rows that share it, so DRAM bounds a step of few rows unless it is a short one.  A unit is one request,
// one cached head and up to 8 or 16 of its rows (new token, query head of the group); its keys come in tiles of 4 KB, 32 keys at
// head dimension 64 and 16 above.  The units' tiles, laid end to end, are cut into equal runs, one for each warp of the grid: no run is longer than
// another whatever the lengths are, and a single long request fills the GPU like many short ones.  A warp streams its run on its
// own: it fetches tiles by TMA into a ring of its own, and meets other warps only when the run is over, to join what is left of
// units that were cut: in shared memory within a block, through L2 between blocks, where the block that arrives last joins the parts in order.
// The products are taken transposed, S^T = K Q^T and O^T = V^T P^T, so that keys and features fill the 16-row side of the matrix
// instructions and the few rows of a step their 8-column side (with rows on the 16-row side the kernel issued twice the
// instructions, which bound it at 550 a tile of 16 keys).
// 16 requests of up to 32768 tokens, 32 heads on 8 of 128: 187 us = 5.9 TB/s, 90 % of a large copy's rate.  32 requests of up to 4096, 12 heads of 64:
// 45 us = 4.0 TB/s, of which 8 us pass before the first tile and 9 in the joins.
#include "saf_cache_attn.cuh"

namespace saf {
namespace {

constexpr int TILE = 4096, STAGE = 2 * TILE;   // a tile of keys or values; both
constexpr int MAX_STAGES = 4;
constexpr int SINGLE_TILES = 4;     // tiles a warp up to which a block takes a whole unit where there are no more units than blocks

template <int D, int NB>
struct Cfg {
  static constexpr int HALVES = D == 64 ? 1 : 2;              // 64-feature halves of a tile (96: zero-filled to 128)
  static constexpr int BOXES = D == 96 ? 2 : 1;               // copies that bring them
  static constexpr int KT = TILE / (HALVES * 128);            // keys of a tile
  static constexpr int WARPS = NB == 1 ? 12 : 8;              // what the registers allow: 168 a thread for 8 rows, 255 for 16
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

// 8 x 8 elements of 16 bits, a pair of a row in each lane, transposed
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <int D, int NB, bool EXACT>
__global__ void __launch_bounds__(32 * Cfg<D, NB>::WARPS, 1)
saf_cache_attn_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const __grid_constant__ CacheAttnParams p) {
  constexpr int HALVES = Cfg<D, NB>::HALVES, BOXES = Cfg<D, NB>::BOXES, KT = Cfg<D, NB>::KT, SUB = KT / 16, W = Cfg<D, NB>::WARPS, NT = 32 * W, ROWS = 8 * NB;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const int stages = p.stages, max_rows = p.max_rows, part_floats = part_size(max_rows, D);
  // [warps][stages] tiles, then a part of each warp's run; at the run's end its ring holds a second one
  auto part_at = [&](int w, int k) -> float* {
    if (k == 1) return reinterpret_cast<float*>(smem + w * stages * STAGE);
    if (!p.parts_in_smem) return p.workspace + (static_cast<int64_t>(gridDim.x) * 2 + static_cast<int64_t>(blockIdx.x) * W + w) * part_floats;
    return reinterpret_cast<float*>(smem + W * stages * STAGE) + w * part_floats;
  };
  __shared__ uint64_t full[W][MAX_STAGES];
  __shared__ Part open_unit[2];                              // units that go on in other blocks: the block's first, its last
  __shared__ int red[3][W], arrived_s[2], abort_s;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) abort_s = 0;
  if (lane < stages) mbar_init(&full[warp][lane], p.selftest_drop_load && blockIdx.x == 1 && warp + lane == 0 ? 2 : 1);
  if (threadIdx.x < 2) open_unit[threadIdx.x].start = -1;
  mbar_fence_init();
  if (threadIdx.x == 0) {
    tma_prefetch_desc(&mk);
    tma_prefetch_desc(&mv);
  }
  pdl_wait();
  pdl_launch_dependents();

  // ---- this warp's run (the ring's memory is not used yet)
  Cut cut;
  Unit u;
  int x0, x1;
  place_run<KT, ROWS, W, W, SINGLE_TILES>(p, smem, red, warp, cut, x0, x1, u);
  const int run0 = blockIdx.x * W, b0 = cut.start(run0), b1 = cut.start(run0 + W);   // the block's runs
  if (b0 >= b1) return;
  __syncthreads();                                          // the sums have been read: the ring may be filled

  uint8_t* ring = smem + warp * stages * STAGE;
  const uint32_t ring_s = smem_u32(ring);
  const WaitCtx wc{&abort_s, p.status, p.wait_limit_ns};
  const int g = p.kv_group, gid = lane >> 2, t2 = (lane & 3) * 2;

  // ---- the fetching end of the run: up to `stages` tiles ahead of the multiplying one
  Unit fu = u;
  int ft = 0, fend = 0, pages_at = 0, page_ids = 0, fstage = 0, ahead = 0, fslot = 0;   // ahead: tiles fetched and not yet used
  bool fmore = x0 < x1;                                     // (a run may still have no tile, behind the end of a unit that has a block to itself)
  auto load_pages = [&](int tile) {                          // lane l: page of the 16 keys number tile * SUB + l
    pages_at = tile;
    const int c = tile * SUB + lane;
    int id = 0;
    if (c * 16 < max(fu.len, 1)) id = p.block_table[static_cast<int64_t>(fu.r) * p.max_pages + (p.page_shift >= 0 ? c >> p.page_shift : c / (p.page_size >> 4))];
    page_ids = min(max(id, 0), p.n_pages - 1);
  };
  auto enter = [&]() {                                       // false: the unit has no tile in the run
    ft = tile_at(fu, x0);
    fend = tile_at(fu, x1);
    return ft < fend;
  };
  auto advance = [&]() {                                     // to the next unit with a tile in the run
    do {
      next_unit<KT, ROWS>(p, fu);
      if (fu.r >= p.R || fu.start >= x1) {
        fmore = false;
        return;
      }
    } while (!enter());
    load_pages(ft);
    fslot = p.page_shift >= 0 ? (ft * KT) & (p.page_size - 1) : ft * KT % p.page_size;
  };
  if (fmore) {
    if (enter()) {
      load_pages(ft);
      fslot = p.page_shift >= 0 ? (ft * KT) & (p.page_size - 1) : ft * KT % p.page_size;
    } else {
      advance();
    }
  }
  auto fetch = [&]() {
    if (!fmore) return;
    if (ft - pages_at >= 32 / SUB) load_pages(ft);
    int page[SUB];
#pragma unroll
    for (int c = 0; c < SUB; ++c) page[c] = __shfl_sync(0xffffffffu, page_ids, (ft - pages_at) * SUB + c);
    const bool keys = has_keys(p, fu.hk);
    if (lane == 0) {
      uint8_t* dst = ring + fstage * STAGE;
      uint64_t* bar = &full[warp][fstage];
      // (32 keys: one box where pages hold whole ones, else two, the second only if there are keys in it)
      const bool two = SUB == 2 && p.box_rows == 16 && ft * KT + 16 < fu.len;
      const int bytes = (two ? 32 : p.box_rows) * 128 * HALVES;
      mbar_expect_tx(bar, keys ? 2 * bytes : bytes);
#pragma unroll
      for (int h = 0; h < BOXES; ++h) {
        if (keys) tma_load_5d(dst + h * 2048, &mk, bar, 64 * h, fslot, 0, fu.hk, page[0]);
        tma_load_5d(dst + TILE + h * 2048, &mv, bar, 64 * h, fslot, 0, fu.hk, page[0]);
      }
      if (two) {
        const int at = fslot + 16 == p.page_size ? 0 : fslot + 16;
        if (keys) tma_load_5d(dst + 2048, &mk, bar, 0, at, 0, fu.hk, page[SUB - 1]);
        tma_load_5d(dst + TILE + 2048, &mv, bar, 0, at, 0, fu.hk, page[SUB - 1]);
      }
    }
    fstage = fstage + 1 == stages ? 0 : fstage + 1;
    ++ahead;
    fslot += KT;
    while (fslot >= p.page_size) fslot -= p.page_size;
    if (++ft >= fend) advance();
  };
  bool primed = false;

  // ---- the multiplying end
  int stage = 0;
  uint32_t phase = 0;
  bool alive = true;
  Part lead{-1, 0, 0, 0, 0, 0};                              // a unit within the block whose parts this warp joins
  // who joins a cut unit: the warp in whose run it begins, or, if it lies in several blocks, all of the block
  auto is_open = [&]() { return u.start < b0 || u.start + u.tiles > b1; };
  auto note_open = [&]() {                                   // (each warp of the unit writes the same)
    if (lane == 0) open_unit[b0 >= u.start ? 0 : 1] = Part{u.start, u.start + u.tiles - 1, u.first, u.many, u.rt, u.hk};
  };
  while (u.r < p.R && u.start < x1) {
    const int t_begin = tile_at(u, x0), t_end = tile_at(u, x1);
    if (t_begin >= t_end || !alive) {                        // (given up: what is left of the run is still reported, so that the counters end at zero)
      if (t_begin < t_end && is_open()) note_open();
      next_unit<KT, ROWS>(p, u);
      continue;
    }
    const int ctx = u.ctx, rows = min(ROWS, u.many * g - u.rt * ROWS);
    const bool keys = has_keys(p, u.hk);
    // queries, as columns: column gid of each block of eight rows
    uint32_t q[NB][D / 16][2];
    if (keys) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int at = u.rt * ROWS + min(8 * b + gid, rows - 1), i = by_group(p, at), h = u.hk * g + at - i * g;
        const bool use = 8 * b + gid < rows && !((p.frozen[h >> 5] >> (h & 31)) & 1);
        const __nv_bfloat16* Q = static_cast<const __nv_bfloat16*>(p.q) + static_cast<int64_t>(u.first + i) * p.q_strides[0] + h * p.q_strides[1] + t2;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
          for (int e = 0; e < 2; ++e) q[b][ks][e] = use ? *reinterpret_cast<const uint32_t*>(Q + ks * 16 + e * 8) : 0u;
      }
    }
    if (!primed) {                                            // (here, so that the queries and the first pages are fetched side by side)
      primed = true;
      for (int s = 0; s < stages; ++s) fetch();
    }
    // scores and weights: rows 8 b + t2 + e, keys gid and gid + 8 of each 16
    int pos[NB][2];
    bool frozen[NB][2];
    unsigned long long mask[NB][2];                            // of the new tokens that a row sees; a row that is not there sees nothing
    const float* arow[NB][2];
    const float* rrow[NB][2];
    bool any = false;
    int first_frozen = ROWS;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = 8 * b + t2 + e, at = u.rt * ROWS + min(row, rows - 1), i = by_group(p, at), h = u.hk * g + at - i * g, n = u.first + i;
        frozen[b][e] = (p.frozen[h >> 5] >> (h & 31)) & 1;
        any |= frozen[b][e];
        if (frozen[b][e]) first_frozen = min(first_frozen, min(row, rows - 1));
        mask[b][e] = p.masks ? p.masks[n] : (2ull << i) - 1;   // (i = 63: all)
        pos[b][e] = frozen[b][e] ? (p.positions ? min(max(p.positions[n], 0), p.Tp - 1) : max(ctx + i, 0)) : 0;
        arow[b][e] = p.alpha + static_cast<int64_t>(h) * p.Tp;
        rrow[b][e] = p.rho + static_cast<int64_t>(h) * p.Tp;
      }
    const bool any_frozen = __any_sync(0xffffffffu, any);
    int from = ctx;                                            // first key that some row does not see
    if (any_frozen) {
      int lowest = 0x7fffffff;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (frozen[b][e]) lowest = min(lowest, pos[b][e]);
      lowest = __reduce_min_sync(0xffffffffu, lowest);
      if (lowest < ctx) from = lowest + 1;
      // rows of ordinary heads look where the unit's first frozen row looks, so that their loads cost nothing
      const int first_row = __reduce_min_sync(0xffffffffu, first_frozen);
      const int at = u.rt * ROWS + first_row, i = by_group(p, at), h = u.hk * g + at - i * g, n = u.first + i;
      const int ps = p.positions ? min(max(p.positions[n], 0), p.Tp - 1) : max(ctx + i, 0);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (!frozen[b][e]) {
            arow[b][e] = p.alpha + static_cast<int64_t>(h) * p.Tp;
            rrow[b][e] = p.rho + static_cast<int64_t>(h) * p.Tp;
            pos[b][e] = ps;
          }
    }
    float o[NB][D / 16][4], m[NB][2], l[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int f = 0; f < D / 16; ++f)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[b][f][e] = 0.0f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[b][e] = -INFINITY;
        l[b][e] = 0.0f;
      }
    }
    // frozen rows: this thread's preferences of a tile, fetched while the tile before is worked on (index: block, 16 keys, key half, row)
    constexpr int NP = NB * SUB * 4;
    float fa[NP], fr[NP];
    auto prefer = [&](int t) {
      if ((t + 1) * KT <= ctx) {                               // every key cached before the step: no branches, loads side by side
#pragma unroll
        for (int x = 0; x < NP; ++x) {
          const int b = x / (SUB * 4), e = x & 1, j = t * KT + x / 4 % SUB * 16 + ((x >> 1) & 1) * 8 + gid;
          fa[x] = arow[b][e][j];
          fr[x] = rrow[b][e][max(pos[b][e] - j, 0)];
          if (pos[b][e] < j) fa[x] = -INFINITY;
        }
      } else {
#pragma unroll
        for (int x = 0; x < NP; ++x) {
          const int b = x / (SUB * 4), e = x & 1, j = t * KT + x / 4 % SUB * 16 + ((x >> 1) & 1) * 8 + gid, back = j - ctx;
          fa[x] = -INFINITY;
          fr[x] = 0.0f;
          if (j < u.len) {
            const int pj = back < 0 || !p.positions ? j : min(max(p.positions[u.first + back], 0), p.Tp - 1);
            if (pj <= pos[b][e]) {
              fa[x] = arow[b][e][pj];
              fr[x] = rrow[b][e][pos[b][e] - pj];
            }
          }
        }
      }
    };
    if (any_frozen) prefer(t_begin);
    for (int t = t_begin; t < t_end; ++t) {
      const uint32_t ks_addr = ring_s + stage * STAGE, vs_addr = ks_addr + TILE;
      const int j0 = t * KT;
      const bool tail = j0 + KT > ctx, unseen = j0 + KT > from;
      if (!mbar_wait_warp_compact(&full[warp][stage], phase, wc, 90)) {
        alive = false;
        break;
      }
      // s[b][sub][2 half + e]: key 16 sub + 8 half + gid, row 8 b + t2 + e
      float s[NB][SUB][4];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[b][sub][e] = 0.0f;
      if (keys) {
        float s2[NB][4];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) s2[b][e] = 0.0f;
        const int row = (((lane >> 3) & 1) << 3) + (lane & 7);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
          for (int sub = 0; sub < SUB; ++sub) {
            uint32_t a[4];
            ldsm4(ks_addr + (ks >> 2) * 2048 + (sub * 16 + row) * 128 + ((((ks & 3) * 2 + (lane >> 4)) ^ (row & 7)) << 4), a);
#pragma unroll
            for (int b = 0; b < NB; ++b) {                     // (16 keys: two chains of products)
              if (SUB == 1 && (ks & 1)) mma16816(s2[b], a, q[b][ks][0], q[b][ks][1]);
              else mma16816(s[b][sub], a, q[b][ks][0], q[b][ks][1]);
            }
          }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[b][sub][e] = __fmul_rn(SUB == 1 ? s[b][sub][e] + s2[b][e] : s[b][sub][e], p.scale_log16);
      }
      if (any_frozen) {
#pragma unroll
        for (int x = 0; x < NP; ++x) {
          const int b = x / (SUB * 4), sub = x / 4 % SUB;
          if (frozen[b][x & 1]) s[b][sub][x & 3] = __fmul_rn(fa[x] + fr[x], LOG16E);
        }
        if (t + 1 < t_end) prefer(t + 1);
      }
      if (tail) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = j0 + sub * 16 + (e >> 1) * 8 + gid, back = j - ctx;
              if (j >= u.len || (back >= 0 && !((mask[b][e & 1] >> back) & 1))) s[b][sub][e] = -INFINITY;
            }
      }
      float top[NB][2];
      bool grown = false;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = m[b][e];
#pragma unroll
          for (int sub = 0; sub < SUB; ++sub) x = max3(x, s[b][sub][e], s[b][sub][2 + e]);
          top[b][e] = x;
          grown |= x > m[b][e];
        }
      // the maximum is only looked for across the lanes where a lane found a larger one
      if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = top[b][e];
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            const float c = x == -INFINITY ? 1.0f : ex16(m[b][e] - x);
            m[b][e] = x;
            l[b][e] *= c;
#pragma unroll
            for (int f = 0; f < D / 16; ++f) {
              o[b][f][e] *= c;
              o[b][f][2 + e] *= c;
            }
          }
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float base = m[b][e] == -INFINITY ? 0.0f : m[b][e];
#pragma unroll
          for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const float x = ex16(__fsub_rn(s[b][sub][2 * half + e], base));   // (rounded scores: alike ones differ by nothing)
              s[b][sub][2 * half + e] = x;
              l[b][e] += x;
            }
        }
      if (unseen) {
        // values behind the last key are whatever the page held, and a value that some rows do not see may be NaN or infinite: both
        // are zeroed for the product, the second kind added by hand to the rows that see it
        bool wild = false;
        for (int c = lane; c < TILE / 16; c += 32) {
          const int row = (c >> 3) & (KT - 1);
          const uint32_t addr = vs_addr + c * 16;             // (the swizzle moves 16-byte words within a row)
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
#pragma unroll
          for (int sub = 0; sub < SUB; ++sub)
            for (int key = 0; key < 16; ++key) {
              const int src = ((key & 7) << 2) | (lane & 3), row = sub * 16 + key;
              float w[NB][2];
#pragma unroll
              for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int e = 0; e < 2; ++e) w[b][e] = __shfl_sync(0xffffffffu, key < 8 ? s[b][sub][e] : s[b][sub][2 + e], src);
#pragma unroll
              for (int f = 0; f < D / 8; ++f) {
                const uint32_t addr = vs_addr + (f >> 3) * 2048 + row * 128 + (((f & 7) ^ (row & 7)) << 4) + gid * 2;
                uint16_t v;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
                if ((v & 0x7f80u) == 0x7f80u) {
#pragma unroll
                  for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                      if (w[b][e] != 0.0f) o[b][f >> 1][(f & 1) * 2 + e] += w[b][e] * __uint_as_float(static_cast<uint32_t>(v) << 16);
                }
              }
            }
          __syncwarp();
          for (int c = lane; c < TILE / 4; c += 32) {
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
      const int key = ((lane >> 4) << 3) + (lane & 7);
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub) {
        uint32_t w[NB][EXACT ? 3 : 1][2];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float lo = s[b][sub][2 * half], hi = s[b][sub][2 * half + 1];
#pragma unroll
            for (int i = 0; i < (EXACT ? 3 : 1); ++i) {
              const uint32_t x = pack_bf16x2(lo, hi);
              lo -= __uint_as_float(x << 16);
              hi -= __uint_as_float(x & 0xffff0000u);
              w[b][i][half] = transpose8(x);
            }
          }
#pragma unroll
        for (int f = 0; f < D / 16; ++f) {
          uint32_t a[4];
          ldsm4t(vs_addr + (f >> 2) * 2048 + (sub * 16 + key) * 128 + ((((f & 3) * 2 + ((lane >> 3) & 1)) ^ (key & 7)) << 4), a);
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < (EXACT ? 3 : 1); ++i) mma16816(o[b][f], a, w[b][i][0], w[b][i][1]);
        }
      }
      if (unseen) fence_proxy_async_smem();                    // (the tile may have been written to: before it is fetched over)
      __syncwarp();
      --ahead;
      if (++stage == stages) {
        stage = 0;
        phase ^= 1;
      }
      fetch();
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[b][e] += __shfl_xor_sync(0xffffffffu, l[b][e], d);
    if (!alive) {
      // given up: the copies in flight end before the block does (a bounded wait again), nothing is joined
      for (; ahead > 0; --ahead) {
        for (int spin = 0; spin < 100000 && !mbar_try_wait(&full[warp][stage], phase); ++spin) {
        }
        if (++stage == stages) {
          stage = 0;
          phase ^= 1;
        }
      }
      continue;
    }
    if (t_begin == 0 && t_end == u.tiles) {
      // pairs of lanes exchange, the one taking the even row, the other the odd one, two features each
      const int odd = gid & 1;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int row = 8 * b + t2 + odd, at = u.rt * ROWS + row, i = by_group(p, at), n = u.first + i, h = u.hk * g + at - i * g;
        const float ls = odd ? l[b][1] : l[b][0], ms = odd ? m[b][1] : m[b][0], inv = ls == 0.0f ? 0.0f : 1.0f / ls;
        const int64_t off = static_cast<int64_t>(n) * p.o_strides[0] + h * p.o_strides[1] + (gid & ~1);
#pragma unroll
        for (int f = 0; f < D / 8; ++f) {
          const float lo = o[b][f >> 1][(f & 1) * 2], hi = o[b][f >> 1][(f & 1) * 2 + 1];
          const float got = __shfl_xor_sync(0xffffffffu, odd ? lo : hi, 4);
          const float x = (odd ? got : lo) * inv, y = (odd ? hi : got) * inv;
          if (row < rows) {
            if (p.o_f32) *reinterpret_cast<float2*>(static_cast<float*>(p.O) + off + f * 8) = make_float2(x, y);
            else *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.O) + off + f * 8) = pack_bf16x2(x, y);
          }
        }
        if (row < rows && gid < 2 && p.LSE) {
          const bool fz = (p.frozen[h >> 5] >> (h & 31)) & 1;
          p.LSE[static_cast<int64_t>(n) * p.H + h] = fz ? 0.0f : ls == 0.0f ? -INFINITY : natural_lse(ms, ls);
        }
      }
    } else {
      // the part of a unit that goes on elsewhere: at most two a run, the second when nothing more is fetched
      const int k = x0 >= u.start ? 0 : 1;                     // the run's first unit or a later one, which is its last
      float* dst = part_at(warp, k);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = 8 * b + t2 + e;
          if (row < rows) {
#pragma unroll
            for (int f = 0; f < D / 8; ++f) dst[row * D + f * 8 + gid] = o[b][f >> 1][(f & 1) * 2 + e];
            if (gid == 0) {
              dst[max_rows * D + row] = m[b][e];
              dst[max_rows * (D + 1) + row] = l[b][e];
            }
          }
        }
      if (is_open()) note_open();
      else if (t_begin == 0) lead = Part{u.start, u.start + u.tiles - 1, u.first, u.many, u.rt, u.hk};
    }
    next_unit<KT, ROWS>(p, u);
  }
  // ---- what is left of cut units, in the order of the runs.  A run's part of a unit lies in its first place if the unit began at or
  // before the run, else in its second; a block's likewise.
  __syncthreads();
  auto part_of = [&](int w, const Part& unit) -> const float* { return part_at(w, cut.start(run0 + w) >= unit.start ? 0 : 1); };
  auto slot_of = [&](int block, const Part& unit) {
    return p.workspace + (static_cast<int64_t>(block) * 2 + (cut.start(block * W) >= unit.start ? 0 : 1)) * part_floats;
  };
  for (int k = 0; k < 2; ++k) {
    const Part unit = open_unit[k];
    if (unit.start < 0) continue;
    const int w0 = unit.start <= b0 ? 0 : cut.run_of(unit.start) - run0;
    const int w1 = unit.last >= b1 ? W - 1 : cut.run_of(unit.last) - run0;
    join<D, ROWS, false, 1, 2>(p, unit, max_rows, w1 - w0 + 1, [&](int i) { return part_of(w0 + i, unit); }, slot_of(blockIdx.x, unit), threadIdx.x, NT);
  }
  const bool any_open = open_unit[0].start >= 0 || open_unit[1].start >= 0;
  int c_first = 0, c_last = 0;
  if (any_open) {
    __syncthreads();
    if (threadIdx.x < 2 && open_unit[threadIdx.x].start >= 0) {
      const Part& unit = open_unit[threadIdx.x];
      c_first = cut.run_of(unit.start) / W;
      c_last = cut.run_of(unit.last) / W;
      __threadfence();                                        // (the block's parts, which the barrier put before this)
      int* counter = p.counters + c_first;
      const bool last = atomicAdd(counter, 1) == c_last - c_first;
      if (last) *counter = 0;
      arrived_s[threadIdx.x] = last;
      __threadfence();
    }
  }
  if (lead.start >= 0) {
    const int members = cut.run_of(lead.last) - run0 - warp + 1;
    join<D, ROWS, false, 1, 2>(p, lead, max_rows, members, [&](int i) { return part_of(warp + i, lead); }, nullptr, lane, 32);
  }
  if (!any_open) return;
  __syncthreads();
  for (int k = 0; k < 2; ++k) {
    const Part unit = open_unit[k];
    if (unit.start < 0 || !arrived_s[k]) continue;
    c_first = cut.run_of(unit.start) / W;
    c_last = cut.run_of(unit.last) / W;
    join<D, ROWS, true, 1, 4>(p, unit, max_rows, c_last - c_first + 1, [&](int i) { return slot_of(c_first + i, unit); }, nullptr, threadIdx.x, NT);
  }
}

template <int D, int NB>
cudaError_t launch(const CUtensorMap& mk, const CUtensorMap& mv, CacheAttnParams& p, int num_sms, cudaStream_t st) {
  constexpr int W = Cfg<D, NB>::WARPS;
  // two stages a warp at least; the parts of the runs' first units where there is room, else in the workspace
  const size_t room = 222 * 1024, ring = static_cast<size_t>(W) * STAGE;
  size_t parts = static_cast<size_t>(W) * part_size(p.max_rows, D) * sizeof(float);
  p.parts_in_smem = parts + 2 * ring <= room;
  if (!p.parts_in_smem) parts = 0;
  p.stages = static_cast<int>(std::min<size_t>(MAX_STAGES, (room - parts) / ring));
  const size_t smem = p.stages * ring + parts + 1024;
  auto kernel = p.o_f32 ? saf_cache_attn_kernel<D, NB, true> : saf_cache_attn_kernel<D, NB, false>;
  static SmemLimit limits[2];
  const cudaError_t e = raise_smem(kernel, static_cast<int>(room) + 1024, limits[p.o_f32 ? 1 : 0]);
  if (e != cudaSuccess) return e;
  return launch_pdl(PDL_REST, kernel, num_sms, 32 * W, smem, st, mk, mv, p);
}
template <int D>
cudaError_t launch(const CUtensorMap& mk, const CUtensorMap& mv, CacheAttnParams& p, int num_sms, cudaStream_t st) {
  if (p.max_rows <= 8) return launch<D, 1>(mk, mv, p, num_sms, st);
  return launch<D, 2>(mk, mv, p, num_sms, st);
}

}  // namespace

CacheAttnForm cache_attn_form(int max_new, int kv_group, int D, int page_size, int max_len, bool o_f32) {
  const int rows = max_new * kv_group;
  // Units of 128 rows from 32 rows at head dimension 128, 43 at 96 and 64 at 64 on, where the two cross (us, this form / the wide one, 24 trees
  // on up to 8192 cached tokens, head dimension 128: 20 rows 95 / 122, 32 rows 131 / 124, 64 rows 225 / 137; 64: 48 rows 56 / 67, 64 rows
  // 70 / 67; 8 chains at 96: 32 rows 72 / 77, 48 rows 99 / 82).  The rule goes by the bound on new tokens, which the launch knows, not by the rows
  // that a step turns out to have.  fp32 output needs weights of 24 bits, three terms: at head dimension 128 the wide form's two blocks an SM leave
  // no TMEM columns for them; at 96 and 64, where 32 and 64 are free, it has not been written.
  if (rows * D >= 4096 && kv_group <= 128 && !o_f32) return cache_wide_form(max_new, kv_group, D, page_size, max_len);
  CacheAttnForm f;
  f.wide = false;
  f.tile_tokens = 0;
  f.max_rows = std::min(16, rows);
  f.halves_k = f.halves_v = D == 128 ? 2 : 1;
  f.box_rows = D == 64 && page_size % 32 == 0 ? 32 : 16;
  const int unit = rows <= 8 ? 8 : 16, keys = D == 64 ? 32 : 16;
  f.tiles = static_cast<int64_t>((rows - 1) / unit + 1) * ((max_len - 1) / keys + 1);
  return f;
}

// (two parts a block, and one a warp where shared memory has no room for them)
size_t cache_attn_workspace(int num_sms) {
  return std::max(sizeof(float) * (2 + Cfg<64, 1>::WARPS) * num_sms * part_size(16, 128), cache_wide_workspace(num_sms));
}

cudaError_t launch_cache_attn(const CUtensorMap& mk, const CUtensorMap& mv, CacheAttnParams& p, int num_sms, cudaStream_t st) {
  if (p.D == 64) return launch<64>(mk, mv, p, num_sms, st);
  if (p.D == 96) return launch<96>(mk, mv, p, num_sms, st);
  return launch<128>(mk, mv, p, num_sms, st);
}

}  // namespace saf
