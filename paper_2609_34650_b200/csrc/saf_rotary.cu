// Rotary positions on queries and keys, forward and backward, and the write of a step's new tokens into a paged cache.
//
// A pair (a, b) of a head's features becomes m (a cos t - b sin t, b cos t + a sin t), t = position * freq, in fp32, rounded once;
// backward the same with -t.  Every element is read and written once: DRAM bounds all but the smallest calls.  A block takes a
// few tokens with all their heads: its cosines and sines are formed once, in shared memory, and the heads stream past them.
// The angle in turns is formed and reduced in fp64: at position 10^6 an fp32 product would be off by up to 0.03 of a radian.
#include "ptx.cuh"
#include "saf_internal.h"

#include <algorithm>
#include <cuda_bf16.h>

namespace saf {
namespace {

constexpr int ROT_THREADS = 256;
constexpr int ROT_BLOCKS = 4;       // blocks an SM
constexpr int ROT_TOKENS = 16;      // tokens of a tile at most

__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  uint4 u;
  u.x = pack_bf16x2(x[0], x[1]);
  u.y = pack_bf16x2(x[2], x[3]);
  u.z = pack_bf16x2(x[4], x[5]);
  u.w = pack_bf16x2(x[6], x[7]);
  *reinterpret_cast<uint4*>(p) = u;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ void from_f32(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_f32(float* p, float x) { *p = x; }

// A chunk is two vectors of VEC features of one head: VEC pairs below rot_dim, copied features behind it.  VEC = 8 where the
// halves are whole 8-vectors, else 1.  A thread keeps its chunk (and so its place in the table) and walks rows = (token, head).  Four
// blocks an SM with a row in flight for each thread (forward and backward of 8 x 12 x 4096 x 64: 94 us = 5.3 TB/s; 32768 x 40 heads x 128, 124 us =
// 5.4; prompts of 31000 tokens into a cache 104 us = 5.4) are as fast as three with two or four rows, and faster than blocks that come and go (98, 129, 127).
template <typename TI, typename TO, int VEC>
__global__ void __launch_bounds__(ROT_THREADS, ROT_BLOCKS) saf_rotary_kernel(const __grid_constant__ RotaryParams p) {
  extern __shared__ float2 tables[];                      // [2][tokens of a tile][rot_dim / 2]: (m cos, m sin)
  // element offsets of a token in the five tensors: q, k, v, outputs of q and k (cached step: k's place in its pool), v's place
  __shared__ long long off_s[2][ROT_TOKENS][6];
  __shared__ int skip_s[2][ROT_TOKENS];
  pdl_wait();
  pdl_launch_dependents();
  const int half = p.rot_dim >> 1, TT = p.block_tokens, tiles = (p.tokens - 1) / TT + 1;
  // what a tile of tokens needs, in one of two places: the next tile's is made while others stream this one
  auto prepare = [&](int tile, int buf) {
    const int tok0 = tile * TT, ntok = min(TT, p.tokens - tok0);
    if (static_cast<int>(threadIdx.x) < ntok) {
      const int n = tok0 + threadIdx.x;
      const long long b = n / p.T, t = n - static_cast<int>(b) * p.T;
      long long* o = off_s[buf][threadIdx.x];
      o[0] = b * p.q_strides[0] + t * p.q_strides[2];
      o[1] = b * p.k_strides[0] + t * p.k_strides[2];
      o[2] = t * p.vn_strides[0];
      o[3] = b * p.qo_strides[0] + t * p.qo_strides[2];
      bool skip = false;
      if (p.slots) {
        const int slot = p.slots[n];
        skip = static_cast<unsigned>(slot) >= static_cast<unsigned>(p.n_slots);
        const long long page = skip ? 0 : slot / p.page_size, place = skip ? 0 : slot - page * p.page_size;
        o[4] = page * p.ko_strides[0] + place * p.ko_strides[2];
        o[5] = page * p.vo_strides[0] + place * p.vo_strides[2];
      } else {
        o[4] = b * p.ko_strides[0] + t * p.ko_strides[2];
        o[5] = 0;
      }
      skip_s[buf][threadIdx.x] = skip;
    }
    float2* table = tables + buf * TT * half;
    for (int e = threadIdx.x; e < ntok * half; e += ROT_THREADS) {
      const int tk = e / half, i = e - tk * half;
      const int n = tok0 + tk;
      const int pos = p.positions ? p.positions[n] : n % p.T;
      double turns = static_cast<double>(pos) * (p.freqs[i] * 0.15915494309189535);
      turns -= rint(turns);
      float s, c;
      sincospif(2.0f * static_cast<float>(turns), &s, &c);
      table[e] = make_float2(c * p.mscale, (p.backward ? -s : s) * p.mscale);
    }
  };
  const int chunks = p.D / (2 * VEC), rot_chunks = half / VEC;
  const int subs = ROT_THREADS / chunks;                   // rows that the block handles side by side
  const int chunk = threadIdx.x % chunks, sub = threadIdx.x / chunks;
  const bool turning = chunk < rot_chunks;
  int o0, o1;                                              // features of the chunk's two vectors
  if (!turning) {
    o0 = p.rot_dim + (chunk - rot_chunks) * 2 * VEC;
    o1 = o0 + VEC;
  } else if (p.interleaved) {
    o0 = chunk * 2 * VEC;
    o1 = o0 + VEC;
  } else {
    o0 = chunk * VEC;
    o1 = half + o0;
  }
  const int heads = p.Hq + p.Hk + p.Hv;
  const int step_t = subs / heads, step_h = subs - step_t * heads;
  // a row's source and destination
  auto find = [&](const long long* o, int head, const TI*& src, TO*& dst) {
    if (head < p.Hq) {
      src = static_cast<const TI*>(p.q) + o[0] + head * p.q_strides[1];
      dst = static_cast<TO*>(p.q_out) + o[3] + head * p.qo_strides[1];
    } else if (head < p.Hq + p.Hk) {
      const int hk = head - p.Hq;
      src = static_cast<const TI*>(p.k) + o[1] + hk * p.k_strides[1];
      dst = static_cast<TO*>(p.k_out) + o[4] + hk * p.ko_strides[1];
    } else {                                               // (new values of a cached step: copied)
      const int hv = head - p.Hq - p.Hk;
      src = static_cast<const TI*>(p.v) + o[2] + hv * p.vn_strides[1];
      dst = static_cast<TO*>(p.v_out) + o[5] + hv * p.vo_strides[1];
    }
  };
  const int tk0 = sub / heads, head0 = sub - tk0 * heads;
  prepare(blockIdx.x, 0);
  for (int tile = blockIdx.x, buf = 0; tile < tiles; tile += gridDim.x, buf ^= 1) {
    __syncthreads();
    const int ntok = min(TT, p.tokens - tile * TT);
    const float2* table = tables + buf * TT * half;
    int tk = sub < subs ? tk0 : ntok, head = head0;
    while (tk < ntok) {
      if (!skip_s[buf][tk]) {
        const TI* src;
        TO* dst;
        find(off_s[buf][tk], head, src, dst);
        const bool turn = turning && head < p.Hq + p.Hk;
        if constexpr (VEC == 8) {
          float a[8], c[8];
          load8(src + o0, a);
          load8(src + o1, c);
          if (turn) {
            const float4* cs = reinterpret_cast<const float4*>(table + tk * half + chunk * 8);
            float x[16];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float4 u = cs[i];
              x[4 * i] = u.x; x[4 * i + 1] = u.y; x[4 * i + 2] = u.z; x[4 * i + 3] = u.w;
            }
            if (p.interleaved) {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float a0 = a[2 * i], a1 = a[2 * i + 1], c0 = c[2 * i], c1 = c[2 * i + 1];
                a[2 * i] = a0 * x[2 * i] - a1 * x[2 * i + 1];
                a[2 * i + 1] = a1 * x[2 * i] + a0 * x[2 * i + 1];
                c[2 * i] = c0 * x[8 + 2 * i] - c1 * x[8 + 2 * i + 1];
                c[2 * i + 1] = c1 * x[8 + 2 * i] + c0 * x[8 + 2 * i + 1];
              }
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float a0 = a[i], c0 = c[i];
                a[i] = a0 * x[2 * i] - c0 * x[2 * i + 1];
                c[i] = c0 * x[2 * i] + a0 * x[2 * i + 1];
              }
            }
          }
          store8(dst + o0, a);
          store8(dst + o1, c);
        } else {
          float a = to_f32(src[o0]), c = to_f32(src[o1]);
          if (turn) {
            const float2 u = table[tk * half + chunk];
            const float a0 = a;
            a = a0 * u.x - c * u.y;
            c = c * u.x + a0 * u.y;
          }
          from_f32(dst + o0, a);
          from_f32(dst + o1, c);
        }
      }
      tk += step_t;
      head += step_h;
      if (head >= heads) {
        head -= heads;
        ++tk;
      }
    }
    if (tile + gridDim.x < tiles) prepare(tile + gridDim.x, buf ^ 1);
  }
}

template <typename TI, typename TO>
cudaError_t launch(const RotaryParams& p, int grid, size_t smem, cudaStream_t st) {
  // halves of whole 8-vectors, or single features
  if (p.rot_dim % 16 == 0 && p.D % 16 == 0) return launch_pdl(PDL_REST, saf_rotary_kernel<TI, TO, 8>, grid, ROT_THREADS, smem, st, p);
  return launch_pdl(PDL_REST, saf_rotary_kernel<TI, TO, 1>, grid, ROT_THREADS, smem, st, p);
}

}  // namespace

cudaError_t launch_rotary(RotaryParams& p, bool in_f32, bool out_f32, int num_sms, cudaStream_t st) {
  // tiles of tokens whose table takes up to 8 KB (two of them), on as many blocks as run at once, of a size that gives every
  // block the same number (32768 tokens on 592 blocks in tiles of 16 were 4 rounds for 3.5: 102 us for 93)
  const int most = std::max(1, std::min(ROT_TOKENS, 8192 / std::max(4 * p.rot_dim, 1))), blocks = ROT_BLOCKS * num_sms;
  const int rounds = (p.tokens - 1) / (blocks * most) + 1;
  p.block_tokens = (p.tokens - 1) / (blocks * rounds) + 1;
  const int grid = std::min(blocks, (p.tokens - 1) / p.block_tokens + 1);
  const size_t smem = static_cast<size_t>(2) * p.block_tokens * (p.rot_dim / 2) * sizeof(float2);
  if (in_f32) return out_f32 ? launch<float, float>(p, grid, smem, st) : launch<float, __nv_bfloat16>(p, grid, smem, st);
  return out_f32 ? launch<__nv_bfloat16, float>(p, grid, smem, st) : launch<__nv_bfloat16, __nv_bfloat16>(p, grid, smem, st);
}

}  // namespace saf
