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

__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n .reg .b64 ra, rb, rd;\n mov.b64 ra, {%2, %3};\n mov.b64 rb, {%4, %5};\n mul.rn.f32x2 rd, ra, rb;\n mov.b64 {%0, %1}, rd;\n}\n"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// max(x, 0), NaN for NaN
__device__ __forceinline__ float positive(float x) {
  float y;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(x));
  return y;
}
// x Phi(x) of a pair of bf16 values, rounded to bf16: max(x, 0) - n Phi(-n) with n = |x|, at most 9 (where n Phi(-n) is 1e-18), and log2 Phi(t) as a
// polynomial of degree 8 on [-9, 0] in u = 1 + 2 t / 9 (through a weighted fit at Chebyshev nodes; relative error of the result before its
// rounding, over all bf16 values above -9, 8.7e-6).  One way for all values, 21 instructions a pair: by error functions below -3, as the bf16
// product does for the sake of its bits, 10992 x 4096 x 1024 with values of deviation 3 takes 82 us instead of 58.
__device__ __forceinline__ uint32_t gelu_near(uint32_t w) {
  const float2 x = make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  const float2 t = make_float2(fmaxf(-fabsf(x.x), -9.0f), fmaxf(-fabsf(x.y), -9.0f));
  const float2 u = fma2(t, make_float2(0.2222222222f, 0.2222222222f), make_float2(1.0f, 1.0f));
  constexpr float k[9] = {-18.167024612426758f, 30.540971755981445f, -14.040131568908691f, 0.30345144867897034f, 0.16877345740795135f,
                          0.09042360633611679f, 0.054782647639513016f, 0.036208659410476685f, 0.01254955492913723f};
  float2 q = make_float2(k[8], k[8]);
#pragma unroll
  for (int i = 7; i >= 0; --i) q = fma2(q, u, make_float2(k[i], k[i]));
  const float2 r = fma2(t, make_float2(ex2(q.x), ex2(q.y)), make_float2(positive(x.x), positive(x.y)));
  return pack_bf16(r.x, r.y);
}

// gemm_store8 with the column block found by comparing, not by a division (a fifth of this epilogue's instructions).
template <bool RES>
__device__ __forceinline__ void q8_store8(const GemmArgs& P, int m, int n, const uint4& t, const uint4& r) {
  if (P.out[0] != nullptr) {
    const bool second = n >= P.part, third = (unsigned)n >= 2u * (unsigned)P.part;       // (8 columns lie in one part: its width is a multiple of 8)
    __nv_bfloat16* o = third ? P.out[2] : (second ? P.out[1] : P.out[0]);
    *reinterpret_cast<uint4*>(o + (size_t)m * P.part + (n - (third ? 2 * P.part : (second ? P.part : 0)))) = t;
  }
  if constexpr (RES) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&t);
    const uint32_t* rw = reinterpret_cast<const uint32_t*>(&r);
    uint4 s;
    uint32_t* sw = reinterpret_cast<uint32_t*>(&s);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 v = add2(make_float2(__uint_as_float(rw[e] << 16), __uint_as_float(rw[e] & 0xFFFF0000u)),
                            make_float2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xFFFF0000u)));
      sw[e] = pack_bf16(v.x, v.y);
    }
    *reinterpret_cast<uint4*>(P.sum + (size_t)m * P.N + n) = s;
  }
}

// Eight sums of row m, columns [n, n + 8), finished and stored.
__device__ __forceinline__ void q8_finish8(const GemmQ8Args& P, int m, int n, const int* acc) {
  const float as = P.a_scale[m];
  const float4 s0 = *reinterpret_cast<const float4*>(P.w_scale + n), s1 = *reinterpret_cast<const float4*>(P.w_scale + n + 4);
  const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = pack_bf16((float)acc[2 * e] * as * s[2 * e], (float)acc[2 * e + 1] * as * s[2 * e + 1]);
  if (P.o.gelu) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = gelu_near(w[e]);
  }
  const uint4 t = make_uint4(w[0], w[1], w[2], w[3]);
  if (P.o.residual != nullptr)
    q8_store8<true>(P.o, m, n, t, *reinterpret_cast<const uint4*>(P.o.residual + (size_t)m * P.o.N + n));
  else
    q8_store8<false>(P.o, m, n, t, make_uint4(0u, 0u, 0u, 0u));
}

template <int COUNT>
struct Q8Steps {
  static constexpr int value = COUNT;
};

// Few tokens: a CTA takes 16 channels and 8 GROUPS tokens, its eight warps every eighth 64 columns of K, whose sums they add up in
// shared memory.  A lane reads 16 bytes of a row: which of a product's columns they are does not matter as long as both
// operands agree.  Bound by the time that a warp's loads take: where all CTAs run at once (ONE_WAVE, two to an SM) a warp has those of four
// steps in flight, elsewhere those of two, and four CTAs share an SM.  Measured: 1 x 4096 x 1024 2.5 us, 16 x 1024 x 4096 3.9,
// 32 x 1024 x 4096 4.7 (in four CTAs to an SM 5.6 and 8.7), 16 x 4096 x 4096 5.2 (7.8); in several waves 8 x 16384 x 1024 5.1 (with four steps and
// two CTAs 6.7), 1 x 16384 x 4096 8.3 (10.9).
template <int GROUPS, bool ONE_WAVE>
__global__ void __launch_bounds__(256, ONE_WAVE ? 2 : 4) k_linear_q8_few(const GemmQ8Args P) {
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
  const auto steps = [&](int k, auto count) {            // (all of the steps' loads first)
    constexpr int kSteps = decltype(count)::value;
    uint4 u[kSteps], v[kSteps], x[kSteps][GROUPS];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const int at = k + 512 * j + 16 * t;
      const bool in = at < K;
      u[j] = in && n0 + g < N ? __ldcg(reinterpret_cast<const uint4*>(w0 + at)) : zero;
      v[j] = in && n0 + 8 + g < N ? __ldcg(reinterpret_cast<const uint4*>(w1 + at)) : zero;
#pragma unroll
      for (int i = 0; i < GROUPS; ++i)
        x[j][i] = in && m0 + 8 * i + g < M ? *reinterpret_cast<const uint4*>(P.a + (size_t)(m0 + 8 * i + g) * K + at) : zero;
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        mma_s8(c[i], u[j].x, v[j].x, u[j].y, v[j].y, x[j][i].x, x[j][i].y);
        mma_s8(c[i], u[j].z, v[j].z, u[j].w, v[j].w, x[j][i].z, x[j][i].w);
      }
    }
  };
  long k = warp * 64;                                    // of the warp: the limits below are the same for its lanes
  if constexpr (ONE_WAVE) {
    for (; k + 1536 < K; k += 2048) steps((int)k, Q8Steps<4>{});
  }
  for (; k < K; k += 1024) steps((int)k, Q8Steps<2>{});
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

// ---------------------------------------------------------------- many tokens: tcgen05
//
// A persistent CTA per SM takes tiles of 128 tokens x BN channels (256, 128 or 64) in turn.  K in steps of 128: A [128, 128] and W [BN, 128], both
// K-major in 128-byte swizzled rows as they lie in memory, 32 columns of K an MMA, int32 sums in BN of 2 BN TMEM columns: while the epilogue
// warps take one tile's sums, the MMAs of the next tile run.
//   warps 0-15  epilogue: 32 tokens and a quarter of the channels each, 32 channels (of 64 wide tiles 16) at a time, through 2 KB of shared memory
//               (of 64 wide tiles 1) into whole sectors, by a bulk copy where a block of 32 channels has one output and no residual
//   warp 16     TMA producer; warp 17 allocates tensor memory and issues the MMAs
// Every wait is bounded, as in the bf16 product.  Measured: 10992 x 4096 x 1024 42 us, 2200 TOPS (with GELU 48), 10992 x 1024 x 4096 with a residual 47,
// 1041 x 4096 x 1024 with GELU 9.1, 1041 x 1024 x 4096 with a residual 10.8, 8192^3 391 (2810 TOPS).  The main loop alone runs at 3300 TOPS; what
// bounds the first is the epilogue beside it: its arithmetic, and results that share L2 with the 48 KB a step that tiles take in (by the
// threads' own stores 43 and 51 us).
constexpr int kQ8K = 128, kQ8ATile = 128 * kQ8K;
__host__ __device__ constexpr int q8_stage_bytes(int bn) { return kQ8ATile + bn * kQ8K; }
__host__ __device__ constexpr int q8_stages(int bn) { return bn == 256 ? 4 : (bn == 128 ? 6 : 8); }
__host__ __device__ constexpr int q8_chunk(int bn) { return bn >= 128 ? 32 : 16; }        // channels of a warp at a time
__host__ __device__ constexpr int q8_staging(int bn) { return kGemmEpilogueWarps * 32 * q8_chunk(bn) * 2; }
constexpr int kQ8MaxStages = 8;

struct Q8Barriers {
  unsigned long long full[kQ8MaxStages], empty[kQ8MaxStages], acc_full[2], acc_empty[2], drain;
  uint32_t tmem_base;
  int abort_flag;
};
__host__ __device__ constexpr size_t q8_smem_bytes(int bn) {
  return (size_t)q8_stages(bn) * q8_stage_bytes(bn) + q8_staging(bn) + sizeof(Q8Barriers) + 64;
}

// Instruction descriptor: int8 x int8 -> int32, both K-major, M = 128.
__host__ __device__ constexpr uint32_t idesc_s8(int n) { return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24); }

__device__ __forceinline__ void mma_ss_s8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc),
      "r"(idesc), "r"(acc)
      : "memory");
}

// A warp's 32 tokens (from row0) and quarter of a tile's channels (from col0): its sums from tensor memory (t_row) to where the caller wants
// them, by way of its part of the staging; free() once the last of the sums has been read.
template <int BN, bool GELU, bool RES, bool BULK, typename Free>
__device__ __forceinline__ void q8_epilogue(const GemmQ8Args& P, const CUtensorMap* out, uint32_t t_row, int row0, int col0, uint4* stage, Free free) {
  constexpr int kCols = BN / 4, kChunk = q8_chunk(BN), kUnits = kChunk / 8;   // a warp's channels, those of a round, their 16-byte units
  const int lane = threadIdx.x & 31;
  const float as = row0 + lane < P.o.M ? P.a_scale[row0 + lane] : 0.0f;
#pragma unroll 1
  for (int c = 0; c < kCols; c += kChunk) {
    const int col = col0 + c;
    uint4 res[RES ? kUnits : 1];
    if constexpr (RES) {
#pragma unroll
      for (int i = 0; i < kUnits; ++i) {
        const int r = row0 + (lane + 32 * i) / kUnits, n = col + (lane + 32 * i) % kUnits * 8;
        if (r < P.o.M && n < P.o.N) res[i] = *reinterpret_cast<const uint4*>(P.o.residual + (size_t)r * P.o.N + n);
      }
    }
#pragma unroll
    for (int h = 0; h < kChunk; h += 16) {
      uint32_t o[16];
      float4 ws[4];
      tmem_ld16(t_row + c + h, o);
      if constexpr (BULK)
        if (h == 0) {                                    // the staging's last contents have been read
          asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          __syncwarp();
        }
#pragma unroll
      for (int e = 0; e < 4; ++e) {                      // (N a multiple of 8: scales past it are not read)
        const int n = col + h + 4 * e;
        ws[e] = n < P.o.N ? *reinterpret_cast<const float4*>(P.w_scale + n) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      tmem_wait_ld();
      if (c + kChunk >= kCols && h + 16 >= kChunk) {     // the last of this tile's sums: the buffer is free
        tc_fence_before();
        if (lane == 0) free();
      }
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 x = mul2(mul2(make_float2((float)(int)o[4 * e], (float)(int)o[4 * e + 1]), make_float2(as, as)), make_float2(ws[e].x, ws[e].y));
        const float2 y = mul2(mul2(make_float2((float)(int)o[4 * e + 2], (float)(int)o[4 * e + 3]), make_float2(as, as)), make_float2(ws[e].z, ws[e].w));
        w[2 * e] = pack_bf16(x.x, x.y);
        w[2 * e + 1] = pack_bf16(y.x, y.y);
      }
      if constexpr (GELU) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = gelu_near(w[e]);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u)
        stage[lane * kUnits + ((h / 8 + u) ^ (BULK ? lane >> 1 & 3 : lane & (kUnits - 1)))] = make_uint4(w[4 * u], w[4 * u + 1], w[4 * u + 2], w[4 * u + 3]);
    }
    if constexpr (BULK) {                                // (rows and columns past the last are not written)
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0 && row0 < P.o.M && col < P.o.N) {
        const int i = (col >= P.o.part) + ((unsigned)col >= 2u * (unsigned)P.o.part);
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(out + i), "r"(col - i * P.o.part), "r"(row0),
                     "r"(smem_u32(stage))
                     : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      }
      continue;
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int r = (lane + 32 * i) / kUnits, u = (lane + 32 * i) % kUnits;
      if (row0 + r < P.o.M && col + u * 8 < P.o.N)
        q8_store8<RES>(P.o, row0 + r, col + u * 8, stage[r * kUnits + (u ^ (r & (kUnits - 1)))], res[RES ? i : 0]);
    }
    __syncwarp();
  }
}

// GELU and the residual's sum in instances of their own.
struct OutMaps { CUtensorMap m[3]; };
template <int BN, bool GELU, bool RES, bool BULK>
__global__ void __launch_bounds__(kGemmThreads, 1)
k_linear_q8_tcgen05(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ OutMaps tm_out,
                    const __grid_constant__ GemmQ8Args P) {
  constexpr int kStages = q8_stages(BN), kStage = q8_stage_bytes(BN);
  constexpr int kProducer = kGemmEpilogueWarps, kIssuer = kGemmEpilogueWarps + 1;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* staging = smem + kStages * kStage;
  Q8Barriers* B = reinterpret_cast<Q8Barriers*>(staging + q8_staging(BN));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int k_tiles = (P.o.K + kQ8K - 1) / kQ8K, tiles_m = (P.o.M + 127) / 128, tiles_n = (P.o.N + BN - 1) / BN;
  const int tiles = tiles_m * tiles_n;
  const bool aligned = (smem_u32(smem) & 1023u) == 0;
  if (!aligned && threadIdx.x == 0) report_status(P.o.status, OVGGT_ERR_DEVICE_STATUS);
  pdl_trigger();

  if (warp == kProducer && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_a) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_w) : "memory");
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&B->full[s], 1);
      mbar_init(&B->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&B->acc_full[b], 1);
      mbar_init(&B->acc_empty[b], kGemmEpilogueWarps);
    }
    mbar_init(&B->drain, 1);
    B->abort_flag = aligned ? 0 : 1;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    // the weights of its first tile, into L2 while the kernel before drains: a share of them with the CTAs of the same channels
    if ((int)blockIdx.x < tiles)
      for (int kt = (int)blockIdx.x % tiles_m; kt < k_tiles; kt += tiles_m) tma_prefetch_2d(&tm_w, kt * (kQ8K / 2), (int)blockIdx.x / tiles_m * BN);
  }
  if (warp == kIssuer) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&B->tmem_base)), "r"((uint32_t)(2 * BN)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)&B->tmem_base;
  pdl_wait();

  bool ok = aligned;
  if (warp == kProducer) {
    // ------------------------------------------------ TMA producer
    if (lane == 0) {
      int issued = 0;
      for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x) {
        const int m0 = tile % tiles_m * 128, n0 = tile / tiles_m * BN;
        for (int kt = 0; kt < k_tiles; ++kt, ++issued) {
          const int s = issued % kStages;
          if (issued >= kStages) ok = mbar_wait(&B->empty[s], (uint32_t)(issued / kStages - 1) & 1u, B, P.o.status);
          if (!ok) break;
          unsigned char* st = smem + s * kStage;
          mbar_expect_tx(&B->full[s], kStage);
          tma_load_2d(st, &tm_a, kt * (kQ8K / 2), m0, &B->full[s]);
          tma_load_2d(st + kQ8ATile, &tm_w, kt * (kQ8K / 2), n0, &B->full[s]);
        }
      }
      if (!ok)   // leave no bulk copy in flight into this CTA's shared memory
        for (int i = max(0, issued - kStages); i < issued; ++i)
          mbar_wait(&B->full[i % kStages], (uint32_t)(i / kStages) & 1u, B, P.o.status);
    }
    __syncwarp();
  } else if (warp == kIssuer) {
    // ------------------------------------------------ MMA issuer (whole warp in step, one elected lane issues)
    const bool leader = elect_one();
    const uint32_t tm = __reduce_or_sync(0xFFFFFFFFu, tmem);
    constexpr uint32_t idesc = idesc_s8(BN);
    auto wait_all = [&](void* bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, B, P.o.status)) != 0; };
    int it = 0, j = 0;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x, ++j) {
      const int buf = j & 1;
      if (j >= 2) ok = wait_all(&B->acc_empty[buf], (uint32_t)(j / 2 - 1) & 1u);
      if (!ok) break;
      tc_fence_after();
      for (int kt = 0; kt < k_tiles; ++kt, ++it) {
        const int s = it % kStages;
        ok = wait_all(&B->full[s], (uint32_t)(it / kStages) & 1u);
        if (!ok) break;
        tc_fence_after();
        const uint64_t da = smem_desc_sw128(smem_u32(smem + s * kStage)), dw = smem_desc_sw128(smem_u32(smem + s * kStage + kQ8ATile));
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < kQ8K / 32; ++kk)
            mma_ss_s8(tm + buf * BN, da + (uint64_t)(kk * 2), dw + (uint64_t)(kk * 2), idesc, (kt > 0 || kk > 0));
          tc_commit(&B->empty[s]);
          if (kt + 1 == k_tiles) tc_commit(&B->acc_full[buf]);
        }
      }
    }
    if (aligned) {
      if (leader) tc_commit(&B->drain);               // every issued MMA finishes before TMEM is freed
      wait_all(&B->drain, 0);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------ epilogue
    const int quad = warp & 3, side = warp >> 2;
    uint4* stage = reinterpret_cast<uint4*>(staging) + warp * 32 * (q8_chunk(BN) / 8);
    int j = 0;
    for (int tile = blockIdx.x; tile < tiles && ok; tile += gridDim.x, ++j) {
      const int buf = j & 1;
      ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->acc_full[buf], (uint32_t)(j / 2) & 1u, B, P.o.status)) != 0;
      if (!ok) break;
      tc_fence_after();
      q8_epilogue<BN, GELU, RES, BULK>(P, tm_out.m, tmem + ((uint32_t)(quad * 32) << 16) + buf * BN + side * (BN / 4), tile % tiles_m * 128 + quad * 32,
                                 tile / tiles_m * BN + side * (BN / 4), stage, [&]() { mbar_arrive(&B->acc_empty[buf]); });
    }
    if (BULK && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");   // (written before the CTA ends)
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kIssuer) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)(2 * BN)) : "memory");
  }
}

// [rows, C] bf16 row-major; box = 32 columns x 32 rows, 64-byte swizzle.
static inline int make_out_map(CUtensorMap* map, const void* base, int rows, int C) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return OVGGT_ERR_CUDA;
  cuuint64_t dims[2] = {(cuuint64_t)C, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)C * 2};
  cuuint32_t box[2] = {32, 32}, estr[2] = {1, 1};
  const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                        CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    g_attn_last_error = (int)r;
    return OVGGT_ERR_CUDA;
  }
  return OVGGT_OK;
}

template <int BN>
static inline int q8_tcgen05_launch(const GemmQ8Args& P, cudaStream_t st) {
  CUtensorMap ta, tw;
  // (128 int8 columns as 64 of two bytes: the copies move bits)
  int rc = make_rows_map(&ta, P.a, P.o.M, P.o.K / 2, 128);
  if (rc) return rc;
  rc = make_rows_map(&tw, P.w, P.o.N, P.o.K / 2, BN);
  if (rc) return rc;
  const bool gelu = P.o.gelu != 0, res = P.o.residual != nullptr;
  // results by bulk copies where no block of 32 channels lies in two of the outputs
  bool bulk = false;
  OutMaps out = {};
  auto kernel = gelu ? (res ? k_linear_q8_tcgen05<BN, true, true, false> : k_linear_q8_tcgen05<BN, true, false, false>)
                     : (res ? k_linear_q8_tcgen05<BN, false, true, false> : k_linear_q8_tcgen05<BN, false, false, false>);
  if constexpr (BN >= 128) {
    bulk = !res && (P.o.part == P.o.N || P.o.part % 32 == 0);
    if (bulk) kernel = gelu ? k_linear_q8_tcgen05<BN, true, false, true> : k_linear_q8_tcgen05<BN, false, false, true>;
    for (int i = 0; bulk && i < 3 && P.o.out[i] != nullptr; ++i) {
      rc = make_out_map(&out.m[i], P.o.out[i], P.o.M, P.o.part);
      if (rc) return rc;
    }
  }
  static std::atomic<uint64_t> smem_set[6];
  cudaError_t e = allow_smem(kernel, q8_smem_bytes(BN), smem_set[bulk ? 4 + gelu : 2 * gelu + res]);
  const long tiles = (long)((P.o.M + 127) / 128) * ((P.o.N + BN - 1) / BN);
  if (tiles > 0x7FFF0000) return OVGGT_ERR_UNSUPPORTED;
  if (e == cudaSuccess) e = launch_dependent(kernel, dim3((unsigned)std::min(tiles, 148l)), kGemmThreads, 1, q8_smem_bytes(BN), st, true, ta, tw, out, P);
  if (e != cudaSuccess) { g_attn_last_error = (int)e; return OVGGT_ERR_CUDA; }
  return OVGGT_OK;
}

// The few-token kernel is taken for up to 16 tokens and wherever its CTAs run at once, two to an SM: 128 x 1024 x 1024 3.8 us (by tiles 4.7),
// 64 x 1024 x 4096 6.5 (9.6), 128 x 1024 x 4096 7.2 (9.3), but in two waves 64 x 4096 x 1024 6.3 (4.6), 128 x 2048 x 4096 13.4 (9.5).
constexpr int kQ8OneWave = 296;

// Tile width, from a model in nanoseconds fitted to 718 to 10992 tokens, 768 to 4096 channels and columns: set-up and last epilogue, waves
// over 148 SMs as long as their steps of 128 columns, and what is left of an epilogue between two tiles.  1374 x 4096 x 1024 takes 15.2, 12.9
// and 14.8 us with tiles of 256, 128 and 64 channels, 1374 x 1024 x 4096 16.6, 12.5 and 17.6, 10992 x 4096 x 1024 58, 60 and 87.
inline int q8_tile_width(int M, int N, int K) {
  const long tiles_m = (M + 127) / 128, steps = (K + kQ8K - 1) / kQ8K;
  auto ns = [&](int bn, long step, long set_up, long between) {
    const long waves = (tiles_m * ((N + bn - 1) / bn) + 147) / 148;
    return set_up + waves * steps * step + (waves - 1) * between;
  };
  const long wide = ns(256, 400, 7600, 1200), middle = ns(128, 270, 5000, 700), narrow = ns(64, 250, 4000, 200);
  return wide <= middle && wide <= narrow ? 256 : (middle <= narrow ? 128 : 64);
}

static inline int gemm_q8_launch(const GemmQ8Args& P, cudaStream_t st) {
  const int M = P.o.M, groups = M <= 8 ? 1 : (M <= 16 ? 2 : 4);
  const long ctas = (long)((P.o.N + 15) / 16) * ((M + 8 * groups - 1) / (8 * groups));
  const bool one_wave = ctas <= kQ8OneWave;
  if (M > 16 && !one_wave) {
    const int bn = q8_tile_width(M, P.o.N, P.o.K);
    return bn == 256 ? q8_tcgen05_launch<256>(P, st) : (bn == 128 ? q8_tcgen05_launch<128>(P, st) : q8_tcgen05_launch<64>(P, st));
  }
  const auto kernel = groups == 1 ? (one_wave ? k_linear_q8_few<1, true> : k_linear_q8_few<1, false>)
                                  : (groups == 4 ? k_linear_q8_few<4, true> : (one_wave ? k_linear_q8_few<2, true> : k_linear_q8_few<2, false>));
  const cudaError_t e = launch_dependent(kernel, dim3((P.o.N + 15) / 16, (M + 8 * groups - 1) / (8 * groups)), 256, 1, 0, st, true, P);
  if (e != cudaSuccess) { g_attn_last_error = (int)e; return OVGGT_ERR_CUDA; }
  return OVGGT_OK;
}

}  // namespace ovggt
