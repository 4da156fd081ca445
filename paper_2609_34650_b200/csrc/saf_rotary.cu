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
// halves are whole 8-vectors, else 1.  A thread keeps its chunk (and so its place in the table) and walks rows = (token, head).
template <typename TI, typename TO, int VEC>
__global__ void __launch_bounds__(ROT_THREADS) saf_rotary_kernel(RotaryParams p) {
  extern __shared__ float2 table[];                       // [tokens of the block][rot_dim / 2]: (m cos, m sin)
  pdl_wait();
  pdl_launch_dependents();
  const int half = p.rot_dim >> 1;
  const int tok0 = blockIdx.x * p.block_tokens;
  const int ntok = min(p.block_tokens, p.tokens - tok0);
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
  __syncthreads();
  const int chunks = p.D / (2 * VEC), rot_chunks = half / VEC;
  const int subs = ROT_THREADS / chunks;                   // rows that the block handles side by side
  const int chunk = threadIdx.x % chunks, sub = threadIdx.x / chunks;
  if (sub >= subs) return;
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
  int tk = sub / heads, head = sub - tk * heads;
  const int step_t = subs / heads, step_h = subs - step_t * heads;
  while (tk < ntok) {
    const int n = tok0 + tk;
    const long long b = n / p.T, t = n - static_cast<int>(b) * p.T;
    const TI* src;
    TO* dst;
    bool turn = turning;
    bool skip = false;
    long long page = 0, place = 0;
    if (p.slots) {
      const int slot = p.slots[n];
      skip = static_cast<unsigned>(slot) >= static_cast<unsigned>(p.n_slots);
      page = skip ? 0 : slot / p.page_size;
      place = skip ? 0 : slot - page * p.page_size;
    }
    if (head < p.Hq) {
      src = static_cast<const TI*>(p.q) + b * p.q_strides[0] + head * p.q_strides[1] + t * p.q_strides[2];
      dst = static_cast<TO*>(p.q_out) + b * p.qo_strides[0] + head * p.qo_strides[1] + t * p.qo_strides[2];
    } else if (head < p.Hq + p.Hk) {
      const int hk = head - p.Hq;
      src = static_cast<const TI*>(p.k) + b * p.k_strides[0] + hk * p.k_strides[1] + t * p.k_strides[2];
      dst = p.slots ? static_cast<TO*>(p.k_out) + page * p.ko_strides[0] + hk * p.ko_strides[1] + place * p.ko_strides[2]
                    : static_cast<TO*>(p.k_out) + b * p.ko_strides[0] + hk * p.ko_strides[1] + t * p.ko_strides[2];
    } else {                                               // (new values of a cached step: copied)
      const int hv = head - p.Hq - p.Hk;
      src = static_cast<const TI*>(p.v) + hv * p.vn_strides[1] + t * p.vn_strides[0];
      dst = static_cast<TO*>(p.v_out) + page * p.vo_strides[0] + hv * p.vo_strides[1] + place * p.vo_strides[2];
      turn = false;
    }
    if (!skip) {
      const float2* row = table + tk * half;
      if constexpr (VEC == 8) {
        float a[8], c[8];
        load8(src + o0, a);
        load8(src + o1, c);
        if (turn) {
          const float4* cs = reinterpret_cast<const float4*>(row + chunk * 8);
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
          const float2 u = row[chunk];
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
}

template <typename TI, typename TO>
cudaError_t launch(const RotaryParams& p, int grid, size_t smem, cudaStream_t st) {
  // halves of whole 8-vectors, or single features
  if (p.rot_dim % 16 == 0 && p.D % 16 == 0) return launch_pdl(PDL_REST, saf_rotary_kernel<TI, TO, 8>, grid, ROT_THREADS, smem, st, p);
  return launch_pdl(PDL_REST, saf_rotary_kernel<TI, TO, 1>, grid, ROT_THREADS, smem, st, p);
}

}  // namespace

cudaError_t launch_rotary(RotaryParams& p, bool in_f32, bool out_f32, int num_sms, cudaStream_t st) {
  // up to 16 tokens a block (the table: up to 32 KB), as few as give every SM eight blocks
  p.block_tokens = std::min(16, std::max(1, p.tokens / (8 * num_sms)));
  const int grid = (p.tokens - 1) / p.block_tokens + 1;
  const size_t smem = static_cast<size_t>(p.block_tokens) * (p.rot_dim / 2) * sizeof(float2);
  if (in_f32) return out_f32 ? launch<float, float>(p, grid, smem, st) : launch<float, __nv_bfloat16>(p, grid, smem, st);
  return out_f32 ? launch<__nv_bfloat16, float>(p, grid, smem, st) : launch<__nv_bfloat16, __nv_bfloat16>(p, grid, smem, st);
}

}  // namespace saf
