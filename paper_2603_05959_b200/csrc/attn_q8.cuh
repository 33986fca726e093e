// Attention over an 8-bit cache: out = softmax(Q K^T / 8) V per head over the live rows of each sequence, head_dim 64; zero
// where no row is live.  Query heads h of a key head's group read that head; `rows` below are (token, query head of the group).
#pragma once

#include <cooperative_groups.h>

#include "gemm_q8.cuh"

namespace ovggt {

struct AttnQ8Args {
  const __nv_bfloat16* q;              // [seqs, M, H, 64]
  const int8_t *kq, *vq;               // [seqs, cap, HK, 64]
  const uint8_t *kx, *vx;              // [seqs, HK, cap]
  const int* lens;                     // [seqs] or nullptr: cap
  const uint8_t* live;                 // [seqs, cap] or nullptr
  __nv_bfloat16* out;
  int seqs, M, H, HK, cap, group, q_tiles;
  int* status;
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 bytes into shared memory behind the thread's back; zeros where `in` is false.
__device__ __forceinline__ void copy16(void* dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&d);
}
// Two int8, in the low bytes of the halves of x, as a pair of bf16, exact: 128 + the low seven bits, less 128 or, of a negative one, 256.
// (x: the bytes in halves whose high bytes are 0x43)
__device__ __forceinline__ uint32_t int8_to_bf16x2(uint32_t x) { return sub_bf16x2(x & 0xFF7FFF7Fu, x & 0xFF80FF80u); }

// ---------------------------------------------------------------- few rows: the cache streams through, once per 8, 16 or 32 rows
//
// Bound by the cache's bytes.  A warp takes tiles of 32 cached rows by itself, with three of them on their way in its own stages
// (no barrier in the loop); a cluster of CTAs shares a sequence and head, and its parts are joined through distributed shared
// memory: no scratch memory, no second launch.
//   scores  by int8 MMAs on the cached bytes as they are.  A row of Q is taken as whole numbers of 15 bits, q = 2^(e - 13) (256 hi + lo), two int8
//           operands: exact for elements down to 2^-6 of the row's largest, to 2^-14 of it for the rest.  With at
//           most 8 rows hi and lo are the two halves of one operand of 16 rows.
//   P V     by bf16 MMAs: the cached bytes are exact in bf16, their row's power of two goes into P.  With at most 8 rows P is
//           the sum of two bf16 numbers, the halves of the operand again; otherwise it is rounded to one (2^-9).
// Which cached row or column an operand's row or column stands for is free, so each lane takes 16 bytes of a K row and 8
// bytes of a V row at once.
constexpr int kFewWarps = 8, kFewStages = 3, kFewKeys = 32;
constexpr int kFewX = 2 * kFewKeys * 64;                 // of a stage: K, V, then the exponents of K and V and the mask, 32 bytes each
constexpr int kFewStage = kFewX + 128;
__host__ __device__ constexpr int few_smem_bytes(int rows) { return kFewWarps * kFewStages * kFewStage + rows * (64 + 2) * 4; }
static_assert(kFewStages * kFewStage >= 32 * (64 + 2) * 4, "a warp's result does not fit its stages");

template <int ROWS>
__global__ void __launch_bounds__(kFewWarps * 32) k_attn_q8_few(const AttnQ8Args P) {
  namespace cg = cooperative_groups;
  constexpr bool PACK = ROWS == 8;
  constexpr int T = PACK ? 1 : ROWS / 16;                // operands of 16 rows
  constexpr int R = PACK ? 1 : 2;                        // rows of an operand a thread holds scores of
  extern __shared__ __align__(1024) unsigned char smem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long long job = blockIdx.x / S;
  const int hk = (int)(job % P.HK), qt = (int)(job / P.HK % P.q_tiles), seq = (int)(job / P.HK / P.q_tiles);
  const int rows = P.M * P.group, row0 = qt * ROWS;
  pdl_trigger();
  pdl_wait();
  const int len = min(P.cap, max(0, P.lens != nullptr ? P.lens[seq] : P.cap));
  const int tiles = (len + kFewKeys - 1) / kFewKeys;
  auto q_at = [&](int r) {                               // (row r is token r / group, head r % group of this group)
    const int m = r / P.group;
    return (((size_t)seq * P.M + m) * P.H + (size_t)hk * P.group + (r - m * P.group)) * 64;
  };

  // ---- the operands of Q: [tile][0: hi (or hi and lo), 1: lo][32 columns][register]
  uint32_t qa[T][PACK ? 1 : 2][2][4];
  float f[T][R];                                         // a score in log2 units is f x the whole numbers' product x 2^(kx - 127)
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int half = 0; half < R; ++half) {
      const int r = row0 + 16 * i + 8 * half + g;
      float x[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = 0.0f;
      if (r < rows) {
        const uint4* p = reinterpret_cast<const uint4*>(P.q + q_at(r) + 16 * t);
        unpack<kBF16>(p[0], x);
        unpack<kBF16>(p[1], x + 8);
      }
      uint32_t most = 0;
#pragma unroll
      for (int e = 0; e < 16; ++e) most = max(most, __float_as_uint(x[e]) & 0x7FFFFFFFu);
      most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
      most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
      const int e2 = (int)(most >> 23) - 127, up = 13 - e2;
      const bool finite = most < 0x7F800000u, some = finite && most >= 0x00800000u;
      const float u0 = some ? __int_as_float((up / 2 + 127) << 23) : 0.0f, u1 = some ? __int_as_float((up - up / 2 + 127) << 23) : 0.0f;
      // log2(e) / 8 2^(e - 13) 2^-6: cached values are 2^(x - 133)
      f[i][half] = some ? ldexpf(1.4426950408889634f * 0.125f, e2 - 19) : (finite ? 0.0f : __int_as_float(0x7FC00000));
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        int hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int z = some ? __float2int_rn(x[4 * w + e] * u0 * u1) : 0;
          hi[e] = (z + 128) >> 8;
          lo[e] = z - hi[e] * 256;
        }
        const uint32_t ph = (hi[0] & 255) | (hi[1] & 255) << 8 | (hi[2] & 255) << 16 | (uint32_t)hi[3] << 24;
        const uint32_t pl = (lo[0] & 255) | (lo[1] & 255) << 8 | (lo[2] & 255) << 16 | (uint32_t)lo[3] << 24;
        // word w: columns 16 t + 4 w on: k-step w / 2, its first or second half; register of the operand: + 1 for rows 8 to 15
        if constexpr (PACK) {
          qa[i][0][w >> 1][(w & 1) * 2] = ph;
          qa[i][0][w >> 1][(w & 1) * 2 + 1] = pl;
        } else {
          qa[i][0][w >> 1][(w & 1) * 2 + half] = ph;
          qa[i][1][w >> 1][(w & 1) * 2 + half] = pl;
        }
      }
    }

  // ---- the cache, tile by tile
  unsigned char* stages = smem + warp * kFewStages * kFewStage;
  const size_t pitch = (size_t)P.HK * 64, base = ((size_t)seq * P.cap * P.HK + hk) * 64, xbase = ((size_t)seq * P.HK + hk) * P.cap;
  const int first = rank * kFewWarps + warp, stride = S * kFewWarps;
  auto request = [&](int tile, int stage) {
    if (tile < tiles) {
      unsigned char* s = stages + stage * kFewStage;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 8 * i + g, row = tile * kFewKeys + key, from = min(row, len - 1);
        const bool in = row < len;
        // K rows lie so that the two of a lane's adjacent scores are four apart; V rows 2 and 3 of four have their halves exchanged
        copy16(s + ((key & ~7) + (key & 3) * 2 + (key >> 2 & 1)) * 64 + t * 16, P.kq + base + (size_t)from * pitch + t * 16, in);
        copy16(s + 2048 + key * 64 + (t ^ (key & 2)) * 16, P.vq + base + (size_t)from * pitch + t * 16, in);
      }
      if (lane < 6 && (lane < 4 || P.live != nullptr)) {
        const int which = lane >> 1, row = tile * kFewKeys + (lane & 1) * 16;
        const uint8_t* src = which == 0 ? P.kx + xbase : (which == 1 ? P.vx + xbase : P.live + (size_t)seq * P.cap);
        copy16(s + kFewX + lane * 16, src + min(row, P.cap - 16), row < P.cap);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float m[T][R], l[T][R], o[T][8][4];
#pragma unroll
  for (int i = 0; i < T; ++i) {
#pragma unroll
    for (int r = 0; r < R; ++r) m[i][r] = -INFINITY, l[i][r] = 0.0f;
#pragma unroll
    for (int d = 0; d < 8; ++d) o[i][d][0] = o[i][d][1] = o[i][d][2] = o[i][d][3] = 0.0f;
  }
#pragma unroll
  for (int s = 0; s < kFewStages - 1; ++s) request(first + s * stride, s);
  int stage = 0;
#pragma unroll 1
  for (int tile = first; tile < tiles; tile += stride) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 2) : "memory");
    __syncwarp();                                        // this tile has arrived, and all lanes are done with the one before
    request(tile + (kFewStages - 1) * stride, stage == 0 ? kFewStages - 1 : stage - 1);
    const unsigned char* s = stages + stage * kFewStage;
    stage = stage + 1 == kFewStages ? 0 : stage + 1;

    float sc[T][R][8], vs[8];                            // scores of keys 8 b + t (even entries) and 8 b + t + 4
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const uint4 kw = *reinterpret_cast<const uint4*>(s + (8 * b + g) * 64 + t * 16);
      float ks[2];
      bool in[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int key = 8 * b + t + 4 * e;
        in[e] = tile * kFewKeys + key < len && (P.live == nullptr || s[kFewX + 64 + key] != 0);
        ks[e] = __int_as_float((int)s[kFewX + key] << 23);     // (255: infinity, which a block of zeros makes NaN)
        vs[2 * b + e] = in[e] ? q8_step(s[kFewX + 32 + key]) : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < T; ++i) {
        int c[4] = {0, 0, 0, 0};
        mma_s8(c, qa[i][0][0][0], qa[i][0][0][1], qa[i][0][0][2], qa[i][0][0][3], kw.x, kw.y);
        mma_s8(c, qa[i][0][1][0], qa[i][0][1][1], qa[i][0][1][2], qa[i][0][1][3], kw.z, kw.w);
        if constexpr (PACK) {
#pragma unroll
          for (int e = 0; e < 2; ++e) sc[i][0][2 * b + e] = in[e] ? (float)(c[e] * 256 + c[e + 2]) * (f[i][0] * ks[e]) : -INFINITY;
        } else {
          int d[4] = {0, 0, 0, 0};
          mma_s8(d, qa[i][1][0][0], qa[i][1][0][1], qa[i][1][0][2], qa[i][1][0][3], kw.x, kw.y);
          mma_s8(d, qa[i][1][1][0], qa[i][1][1][1], qa[i][1][1][2], qa[i][1][1][3], kw.z, kw.w);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              sc[i][r][2 * b + e] = in[e] ? (float)(c[2 * r + e] * 256 + d[2 * r + e]) * (f[i][r] * ks[e]) : -INFINITY;
        }
      }
    }
    // the running maximum moves only when it is outgrown by 2^8
    float top[T][R];
    bool grown = false;
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float x = sc[i][r][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) x = fmaxf(x, sc[i][r][e]);
        x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 1));
        top[i][r] = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 2));
        grown |= top[i][r] > m[i][r] + kRescaleThreshold;
      }
    if (__any_sync(0xFFFFFFFFu, grown)) {
#pragma unroll
      for (int i = 0; i < T; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float mn = fmaxf(m[i][r], top[i][r]), corr = m[i][r] == mn ? 1.0f : ex2(m[i][r] - mn);
          m[i][r] = mn;
          l[i][r] *= corr;
#pragma unroll
          for (int d = 0; d < 8; ++d)
            if constexpr (PACK) {
#pragma unroll
              for (int e = 0; e < 4; ++e) o[i][d][e] *= corr;
            } else {
              o[i][d][2 * r] *= corr;
              o[i][d][2 * r + 1] *= corr;
            }
        }
    }
    uint32_t pa[T][2][4];                                // P of 16 keys as an operand
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float ref = m[i][r] == -INFINITY ? 0.0f : m[i][r];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const float p0 = ex2(sc[i][r][2 * b] - ref), p1 = ex2(sc[i][r][2 * b + 1] - ref);
          l[i][r] += p0 + p1;
          const float w0 = p0 * vs[2 * b], w1 = p1 * vs[2 * b + 1];
          const uint32_t hi = pack_bf16(w0, w1);
          pa[i][b >> 1][(b & 1) * 2 + r] = hi;
          if constexpr (PACK) pa[i][b >> 1][(b & 1) * 2 + 1] = pack_bf16(w0 - __uint_as_float(hi << 16), w1 - __uint_as_float(hi & 0xFFFF0000u));
        }
      }
#pragma unroll
    for (int b = 0; b < 2; ++b) {                        // 16 keys: 16 b + t, + 4, + 8, + 12
      uint2 v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = 16 * b + t + 4 * e;
        v[e] = *reinterpret_cast<const uint2*>(s + 2048 + key * 64 + (((g >> 1) ^ (t & 2)) * 16) + (g & 1) * 8);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {             // four columns: pairs of keys side by side, then one column of both a register
        uint32_t w[2][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t x = half ? v[2 * e].y : v[2 * e].x, y = half ? v[2 * e + 1].y : v[2 * e + 1].x;
          w[e][0] = __byte_perm(x, y, 0x5140);
          w[e][1] = __byte_perm(x, y, 0x7362);
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const int sel = d & 1 ? 0x4342 : 0x4140;       // (byte 4: 0x43)
          const uint32_t b0 = int8_to_bf16x2(__byte_perm(w[0][d >> 1], 0x43434343u, sel)), b1 = int8_to_bf16x2(__byte_perm(w[1][d >> 1], 0x43434343u, sel));
#pragma unroll
          for (int i = 0; i < T; ++i) mma_bf16(o[i][4 * half + d], pa[i][b][0], pa[i][b][1], pa[i][b][2], pa[i][b][3], b0, b1);
        }
      }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncwarp();

  // ---- a warp's result into its stages: O [ROWS][64], the maxima, the sums
  float* mine = reinterpret_cast<float*>(stages);
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float x = l[i][r];
      x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
      x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
      const int row = 16 * i + 8 * r + g;
      if (t == 0) mine[ROWS * 64 + row] = m[i][r], mine[ROWS * 65 + row] = x;
#pragma unroll
      for (int e = 0; e < 2; ++e)                        // (column n of an MMA is 8 n + d)
#pragma unroll
        for (int d = 0; d < 8; d += 4) {
          float4 y;
          float* z = &y.x;
#pragma unroll
          for (int q = 0; q < 4; ++q) z[q] = PACK ? o[i][d + q][e] + o[i][d + q][e + 2] : o[i][d + q][2 * r + e];
          *reinterpret_cast<float4*>(mine + row * 64 + 16 * t + 8 * e + d) = y;
        }
    }
  __syncthreads();
  // ---- the CTA's, then the cluster's: out = sum O_i 2^(m_i - m) / sum l_i 2^(m_i - m) over the parts in order
  auto weight = [](float mi, float mx) { return mi == mx ? 1.0f : exp2f(mi - mx); };   // (both -inf: nothing was live)
  float* whole = reinterpret_cast<float*>(smem + kFewWarps * kFewStages * kFewStage);
  constexpr int kPart = kFewStages * kFewStage / 4;
  for (int u = threadIdx.x; u < ROWS * 16; u += kFewWarps * 32) {
    const int row = u >> 4, c4 = u & 15;
    const float* parts = reinterpret_cast<const float*>(smem);
    float mx = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) mx = fmaxf(mx, parts[w * kPart + ROWS * 64 + row]);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float k = weight(parts[w * kPart + ROWS * 64 + row], mx);
      const float4 x = *reinterpret_cast<const float4*>(parts + w * kPart + row * 64 + 4 * c4);
      sum = fmaf(k, parts[w * kPart + ROWS * 65 + row], sum);
      a.x = fmaf(k, x.x, a.x); a.y = fmaf(k, x.y, a.y); a.z = fmaf(k, x.z, a.z); a.w = fmaf(k, x.w, a.w);
    }
    *reinterpret_cast<float4*>(whole + row * 64 + 4 * c4) = a;
    if (c4 == 0) whole[ROWS * 64 + row] = mx, whole[ROWS * 65 + row] = sum;
  }
  if (S > 1) cluster.sync(); else __syncthreads();
  for (int u = rank * kFewWarps * 32 + threadIdx.x; u < ROWS * 16; u += S * kFewWarps * 32) {
    const int row = u >> 4, c4 = u & 15;
    if (row0 + row >= rows) continue;
    float mx = -INFINITY, sum = 0.0f;
    for (int s = 0; s < S; ++s) mx = fmaxf(mx, cluster.map_shared_rank(whole, s)[ROWS * 64 + row]);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < S; ++s) {
      const float* part = cluster.map_shared_rank(whole, s);
      const float k = weight(part[ROWS * 64 + row], mx);
      const float4 x = *reinterpret_cast<const float4*>(part + row * 64 + 4 * c4);
      sum = fmaf(k, part[ROWS * 65 + row], sum);
      a.x = fmaf(k, x.x, a.x); a.y = fmaf(k, x.y, a.y); a.z = fmaf(k, x.z, a.z); a.w = fmaf(k, x.w, a.w);
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    *reinterpret_cast<uint2*>(P.out + q_at(row0 + row) + 4 * c4) = make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
  }
  if (S > 1) cluster.sync();                             // (nobody leaves while its part is being read)
}

static inline int attn_q8_launch(AttnQ8Args P, cudaStream_t st) {
  const int rows = P.M * P.group, tile = rows <= 8 ? 8 : (rows <= 16 ? 16 : 32);
  P.q_tiles = (rows + tile - 1) / tile;
  const long long jobs = (long long)P.seqs * P.HK * P.q_tiles;
  // CTAs that share a head: as many as fill the SMs twice, while a warp has a tile to take
  int S = 1;
  while (S < 8 && jobs * S * 2 <= 2 * 148 && S * 2 * kFewWarps * kFewKeys <= P.cap) S *= 2;
  if (jobs * S > 0x7FFFFFFF) return OVGGT_ERR_UNSUPPORTED;
  const auto kernel = tile == 8 ? k_attn_q8_few<8> : (tile == 16 ? k_attn_q8_few<16> : k_attn_q8_few<32>);
  static std::atomic<uint64_t> smem_set[3];
  cudaError_t e = allow_smem(kernel, few_smem_bytes(tile), smem_set[tile == 8 ? 0 : (tile == 16 ? 1 : 2)]);
  if (e == cudaSuccess) e = launch_dependent(kernel, dim3((unsigned)(jobs * S)), kFewWarps * 32, S, few_smem_bytes(tile), st, true, P);
  if (e != cudaSuccess) { g_attn_last_error = (int)e; return OVGGT_ERR_CUDA; }
  return OVGGT_OK;
}

}  // namespace ovggt
