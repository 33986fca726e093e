// Product of int8 rows: t [M, N] = bf16(a_scale[m] w_scale[n] sum_k A[m, k] W[n, k]), A [M, K] and W [N, K] int8 row-major, a scale
// for each token and each channel, with the epilogues of the bf16 product (GELU, column blocks, the residual's sum).  The sums
// are int32 and exact, so any grouping of K gives the same bits.
#pragma once

#include "gemm_tcgen05.cuh"
#include "q8_rows.cuh"

namespace ovggt {

struct GemmQ8Args {
  GemmArgs o;                          // M, N, K and the epilogue
  const int8_t *a, *w;
  const float *a_scale, *w_scale;
};
constexpr int kQ8MaxK = 131056;        // (128 * 128 * K stays below 2^31)

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight sums of row m, columns [n, n + 8), finished and stored.
__device__ __forceinline__ void q8_finish8(const GemmQ8Args& P, int m, int n, const int* acc) {
  const float as = P.a_scale[m];
  const float4 s0 = *reinterpret_cast<const float4*>(P.w_scale + n), s1 = *reinterpret_cast<const float4*>(P.w_scale + n + 4);
  const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16((float)acc[2 * e] * as * s[2 * e], (float)acc[2 * e + 1] * as * s[2 * e + 1]);
  if (P.o.gelu)
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = pack_bf16(gelu(__uint_as_float(w[e] << 16)), gelu(__uint_as_float(w[e] & 0xFFFF0000u)));
  const uint4 t = make_uint4(w[0], w[1], w[2], w[3]);
  if (P.o.residual != nullptr)
    gemm_store8<true>(P.o, m, n, t, *reinterpret_cast<const uint4*>(P.o.residual + (size_t)m * P.o.N + n));
  else
    gemm_store8<false>(P.o, m, n, t, make_uint4(0u, 0u, 0u, 0u));
}

// Few tokens: a CTA takes 16 channels and 8 GROUPS tokens, its eight warps every eighth 64 columns of K, whose sums they add up in
// shared memory.  A lane reads 16 bytes of a row: which of a product's columns they are does not matter as long as both
// operands agree.
template <int GROUPS>
__global__ void __launch_bounds__(256) k_linear_q8_few(const GemmQ8Args P) {
  constexpr int kTokens = 8 * GROUPS;
  __shared__ int part[8][kTokens][16 + 1];
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int M = P.o.M, N = P.o.N, K = P.o.K, n0 = (int)blockIdx.x * 16, m0 = (int)blockIdx.y * kTokens;
  int c[GROUPS][4];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) c[i][0] = c[i][1] = c[i][2] = c[i][3] = 0;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  const int8_t* w0 = P.w + (size_t)(n0 + g) * K;
  const int8_t* w1 = w0 + (size_t)8 * K;
#pragma unroll 2
  for (int k = warp * 64 + 16 * t; k - 16 * t < K; k += 512) {
    const bool in = k < K;
    const uint4 u = in && n0 + g < N ? ld_nc(reinterpret_cast<const uint4*>(w0 + k)) : zero;
    const uint4 v = in && n0 + 8 + g < N ? ld_nc(reinterpret_cast<const uint4*>(w1 + k)) : zero;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const int m = m0 + 8 * i + g;
      const uint4 x = in && m < M ? *reinterpret_cast<const uint4*>(P.a + (size_t)m * K + k) : zero;
      mma_s8(c[i], u.x, v.x, u.y, v.y, x.x, x.y);
      mma_s8(c[i], u.z, v.z, u.w, v.w, x.z, x.w);
    }
  }
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {                     // (rows: channels g, g + 8; columns: tokens 2 t, 2 t + 1)
    part[warp][8 * i + 2 * t][g] = c[i][0];
    part[warp][8 * i + 2 * t + 1][g] = c[i][1];
    part[warp][8 * i + 2 * t][g + 8] = c[i][2];
    part[warp][8 * i + 2 * t + 1][g + 8] = c[i][3];
  }
  __syncthreads();
  if (threadIdx.x < 2 * kTokens) {
    const int m = threadIdx.x >> 1, n = (threadIdx.x & 1) * 8;
    if (m0 + m < M && n0 + n < N) {
      int acc[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        acc[e] = 0;
#pragma unroll
        for (int w = 0; w < 8; ++w) acc[e] += part[w][m][n + e];
      }
      q8_finish8(P, m0 + m, n0 + n, acc);
    }
  }
}

static inline int gemm_q8_launch(const GemmQ8Args& P, cudaStream_t st) {
  const int M = P.o.M, groups = M <= 8 ? 1 : (M <= 16 ? 2 : 4);
  const auto kernel = groups == 1 ? k_linear_q8_few<1> : (groups == 2 ? k_linear_q8_few<2> : k_linear_q8_few<4>);
  const cudaError_t e = launch_dependent(kernel, dim3((P.o.N + 15) / 16, (M + 8 * groups - 1) / (8 * groups)), 256, 1, 0, st, true, P);
  if (e != cudaSuccess) { g_attn_last_error = (int)e; return OVGGT_ERR_CUDA; }
  return OVGGT_OK;
}

}  // namespace ovggt
