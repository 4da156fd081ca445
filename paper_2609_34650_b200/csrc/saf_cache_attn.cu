// Attention of a step's new tokens over a paged cache, ordinary and frozen heads side by side.
//
//   O_i = sum_j e^{s_ij} V_j / sum_j e^{s_ij} over the keys j that row i sees; s_ij = scale q_i k_j (ordinary head) or
//   alpha(p_j) + rho(p_i - p_j) (frozen head), running maximum and sum in fp32.
//
// One block per (row, head): a warp takes every fourth key, its lanes the features; the four partial results are joined in shared memory.
#include "ptx.cuh"
#include "saf_internal.h"

#include <cuda_bf16.h>

namespace saf {
namespace {

constexpr int WARPS = 4;

template <int D>
__global__ void __launch_bounds__(32 * WARPS) saf_cache_attn_kernel(CacheAttnParams p) {
  constexpr int F = D / 32;
  __shared__ float s_m[WARPS], s_l[WARPS], s_o[WARPS][D];
  const int n = blockIdx.y, h = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int r = 0;
  while (r < p.R && p.new_offsets[r + 1] <= n) ++r;
  if (r == p.R) return;
  const int first = max(p.new_offsets[r], 0), i = n - first;
  if (i < 0 || i >= p.max_new) return;
  const int many = min(min(p.new_offsets[r + 1], p.N) - first, p.max_new);
  const int len = min(max(p.kv_lens[r], 0), p.max_len), ctx = len - many;
  const bool frozen = (p.frozen[h >> 5] >> (h & 31)) & 1;
  const int hk = h / p.kv_group;
  auto position = [&](int place) { return p.positions ? min(max(p.positions[first + place], 0), p.Tp - 1) : ctx + place; };
  const int pos = frozen ? position(i) : 0;
  const unsigned long long mask = p.masks ? p.masks[n] : 0;
  float q[F], o[F];
#pragma unroll
  for (int f = 0; f < F; ++f) {
    q[f] = frozen ? 0.0f : __bfloat162float(static_cast<const __nv_bfloat16*>(p.q)[n * p.q_strides[0] + h * p.q_strides[1] + f * 32 + lane]);
    o[f] = 0.0f;
  }
  float m = -INFINITY, l = 0.0f;
  for (int j = warp; j < len; j += WARPS) {
    const int back = j - ctx;
    if (back >= 0 && !(p.masks ? back < 64 && ((mask >> back) & 1) : back <= i)) continue;
    const int page = min(max(p.block_table[static_cast<long long>(r) * p.max_pages + j / p.page_size], 0), p.n_pages - 1);
    const int slot = j % p.page_size;
    float s;
    if (frozen) {
      const int pj = back >= 0 ? position(back) : j;
      if (pj > pos) continue;
      s = (p.alpha[static_cast<long long>(h) * p.Tp + pj] + p.rho[static_cast<long long>(h) * p.Tp + pos - pj]) * 1.4426950408889634f;
    } else {
      const __nv_bfloat16* k = static_cast<const __nv_bfloat16*>(p.k) + page * p.k_strides[0] + hk * p.k_strides[1] + slot * p.k_strides[2];
      s = 0.0f;
#pragma unroll
      for (int f = 0; f < F; ++f) s += q[f] * __bfloat162float(k[f * 32 + lane]);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
      s *= p.scale_log2;
    }
    const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v) + page * p.v_strides[0] + hk * p.v_strides[1] + slot * p.v_strides[2];
    const float nm = fmaxf(m, s), base = nm == -INFINITY ? 0.0f : nm;
    const float w = exp2f(s - base), c = exp2f(m - base);
    l = l * c + w;
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] = o[f] * c + w * __bfloat162float(v[f * 32 + lane]);
    m = nm;
  }
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
#pragma unroll
  for (int f = 0; f < F; ++f) s_o[warp][f * 32 + lane] = o[f];
  __syncthreads();
  m = -INFINITY;
  for (int w = 0; w < WARPS; ++w) m = fmaxf(m, s_m[w]);
  const float base = m == -INFINITY ? 0.0f : m;
  l = 0.0f;
  for (int w = 0; w < WARPS; ++w) l += s_l[w] * exp2f(s_m[w] - base);
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  for (int f = threadIdx.x; f < D; f += 32 * WARPS) {
    float x = 0.0f;
    for (int w = 0; w < WARPS; ++w) x += s_o[w][f] * exp2f(s_m[w] - base);
    x *= inv;
    const int64_t at = n * p.o_strides[0] + h * p.o_strides[1] + f;
    if (p.o_f32) static_cast<float*>(p.O)[at] = x;
    else static_cast<__nv_bfloat16*>(p.O)[at] = __float2bfloat16_rn(x);
  }
  if (threadIdx.x == 0 && p.LSE) p.LSE[static_cast<long long>(n) * p.H + h] = frozen ? 0.0f : (base + log2f(l)) * 0.6931471805599453f;
}

}  // namespace

cudaError_t launch_cache_attn(const CacheAttnParams& p, int num_sms, cudaStream_t st) {
  const dim3 grid(p.H, p.N);
  if (p.D == 64) saf_cache_attn_kernel<64><<<grid, 32 * WARPS, 0, st>>>(p);
  else if (p.D == 96) saf_cache_attn_kernel<96><<<grid, 32 * WARPS, 0, st>>>(p);
  else saf_cache_attn_kernel<128><<<grid, 32 * WARPS, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace saf
