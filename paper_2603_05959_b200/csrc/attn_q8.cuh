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

// ---------------------------------------------------------------- many rows: tcgen05, the cache widened on its way into shared memory
//
// The bf16 attention's scheme (see attn_tcgen05.cuh: halves of 96 cached rows with a buffer of scores each, so that the MMAs of one half run
// under the softmax of the other) for two tiles of 128 rows a CTA, whose K and V tiles six warps read as int8 and write as bf16 planes, once
// for both: q 2^(x - 133) is exact in bf16, so the operands are what the cache stands for.  A plane costs 2.5 instructions an element,
// shared by 256 rows; a pass of its own that writes bf16 planes to memory would move 5 bytes an element instead of one.
//   warps 0-7    softmax, four a tile, one thread a row; the running maximum moves when it is outgrown by 2^8 and O is rescaled then
//   warps 8, 9   MMA issuers, one a tile; warp 8 allocates tensor memory (2 x 256 columns)
//   warps 10-15  K and V: copied to shared memory two tiles ahead, widened there
// The cached rows of a sequence and head are shared out over a cluster of CTAs, whose parts are joined through distributed shared memory.
// Every wait is bounded; on expiry the CTA records OVGGT_ERR_TIMEOUT and leaves through the common teardown.
constexpr int kManyThreads = 512, kManyConverters = 192, kManyRows = 2 * kBM;
constexpr int kManyRegsSoftmax = 200, kManyRegsOther = 56;
static_assert(256 * kManyRegsSoftmax + 256 * kManyRegsOther <= kManyThreads * kRegsLaunch, "register pool of the CTA exceeded");
constexpr int kManyPitch = kHD + 4;                      // floats between the rows of O in shared memory

struct ManyBarriers {
  unsigned long long k_full[kKVStages], k_empty[kKVStages], v_full[kKVStages], v_empty[kKVStages];
  unsigned long long s_full[2][2], p_full[2][2], pv_done[2], o_full[2], drain[2];   // by row tile
  uint32_t tmem_base;
  int abort_flag;
};
constexpr int kManyRaw = 3, kManyRawStage = 2 * kBN * kHD;   // stages of K and V tiles as they lie in the cache; O, maxima and sums come to lie over them
constexpr int kManyO = 2 * kQBytes + 2 * kKVStages * kTileBytes;
constexpr int kManyBar = kManyO + kManyRaw * kManyRawStage;
static_assert(kManyRows * (kManyPitch + 2) * 4 <= kManyRaw * kManyRawStage, "a CTA's result does not fit the tiles it lies over");
constexpr int kManySmem = kManyBar + (int)sizeof(ManyBarriers);

// 2^(x - 133) as a pair of bf16; NaN for 255.
__device__ __forceinline__ uint32_t q8_step_bf16x2(uint32_t x) { return (x == 255u ? 0x7FFFu : (max(x, 6u) - 6u) << 7) * 0x00010001u; }
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 d = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&d);
}
// 16 int8 of columns [16 c, 16 c + 16) of row r, times step -> the same place of a swizzled bf16 tile.
__device__ __forceinline__ void store_widened(unsigned char* tile, int r, int c, const uint4& w, uint32_t step) {
  const uint32_t in[4] = {w.x, w.y, w.z, w.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    o[2 * i] = mul_bf16x2(int8_to_bf16x2(__byte_perm(in[i], 0x43434343u, 0x4140)), step);
    o[2 * i + 1] = mul_bf16x2(int8_to_bf16x2(__byte_perm(in[i], 0x43434343u, 0x4342)), step);
  }
  unsigned char* p = tile + r * 128;
  *reinterpret_cast<uint4*>(p + (((2 * c) ^ (r & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
  *reinterpret_cast<uint4*>(p + (((2 * c + 1) ^ (r & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
}

__global__ void __launch_bounds__(kManyThreads, 1) k_attn_q8_many(const __grid_constant__ AttnQ8Args P) {
  namespace cg = cooperative_groups;
  extern __shared__ __align__(1024) unsigned char smem[];
  cg::cluster_group cluster = cg::this_cluster();
  const int S = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const bool aligned = (smem_u32(smem) & 1023u) == 0;    // the 128-byte swizzle needs 1024-byte aligned tiles
  if (!aligned && threadIdx.x == 0) report_status(P.status, OVGGT_ERR_DEVICE_STATUS);
  unsigned char* sQ = smem;
  unsigned char* sK = sQ + 2 * kQBytes;
  unsigned char* sV = sK + kKVStages * kTileBytes;
  unsigned char* sRaw = smem + kManyO;
  float* sO = reinterpret_cast<float*>(sRaw);            // [256][kManyPitch], then maxima [256], sums [256], once every tile has been widened
  ManyBarriers* B = reinterpret_cast<ManyBarriers*>(smem + kManyBar);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long job = blockIdx.x / S;
  const int hk = (int)(job % P.HK), qt = (int)(job / P.HK % P.q_tiles), seq = (int)(job / P.HK / P.q_tiles);
  const int rows = P.M * P.group, row0 = qt * kManyRows, n_q = min(2, (rows - row0 + kBM - 1) / kBM);   // row tiles of this CTA
  auto q_at = [&](int r) {                               // (row r is token r / group, head r % group of this group)
    const int m = r / P.group;
    return (((size_t)seq * P.M + m) * P.H + (size_t)hk * P.group + (r - m * P.group)) * kHD;
  };
  pdl_trigger();

  if (threadIdx.x == 0) {
    for (int s = 0; s < kKVStages; ++s) {
      mbar_init(&B->k_full[s], kManyConverters);
      mbar_init(&B->v_full[s], kManyConverters);
      mbar_init(&B->k_empty[s], n_q);
      mbar_init(&B->v_empty[s], n_q);
    }
    for (int i = 0; i < 2; ++i) {
      for (int hf = 0; hf < 2; ++hf) {
        mbar_init(&B->s_full[i][hf], 1);
        mbar_init(&B->p_full[i][hf], 128);
      }
      mbar_init(&B->pv_done[i], 1);
      mbar_init(&B->o_full[i], 1);
      mbar_init(&B->drain[i], 1);
    }
    B->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&B->tmem_base)), "r"((uint32_t)(2 * kTmemCols)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  const int len = min(P.cap, max(0, P.lens != nullptr ? P.lens[seq] : P.cap));
  const int tiles_total = (len + kBN - 1) / kBN;
  const int t_begin = (int)((long long)rank * tiles_total / S), n_tiles = aligned ? (int)((long long)(rank + 1) * tiles_total / S) - t_begin : 0;
  {                                                      // Q: 256 rows x 8 groups of 8 columns, rows past the last zero
    constexpr int kPer = kManyRows * 8 / kManyThreads;
    uint4 x[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int idx = threadIdx.x + i * kManyThreads, r = row0 + (idx >> 3);
      x[i] = r < rows ? *reinterpret_cast<const uint4*>(P.q + q_at(r) + (idx & 7) * 8) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int idx = threadIdx.x + i * kManyThreads, r = idx >> 3;
      *reinterpret_cast<uint4*>(sQ + r * 128 + (((idx & 7) ^ (r & 7)) << 4)) = x[i];
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)&B->tmem_base;
  // Every warp of the cluster meets here at the end, each in its own branch: what follows a change of registers stays in it.
  auto sync_all = [&]() {
    __syncwarp();
    if (S > 1) cluster.sync(); else asm volatile("barrier.sync.aligned 0;" ::: "memory");
  };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kManyRegsOther));
    if (warp < 10) {
      // ------------------------------------------------ MMA issuers, in the bf16 attention's order:
      // QK(0,0) QK(0,1) | PV(0,0) QK(1,0) PV(0,1) QK(1,1) | PV(1,0) QK(2,0) ...
      const int i = warp - 8;
      if (i < n_q && n_tiles > 0) {
        const bool leader = elect_one();
        const uint32_t tm = __reduce_or_sync(0xFFFFFFFFu, tmem) + i * kTmemCols;
        constexpr uint32_t idesc_qk = idesc_bf16(kHalf, false), idesc_pv = idesc_bf16(kHD, true);
        const uint64_t dq = smem_desc_sw128(smem_u32(sQ + i * kQBytes));
        auto wait_all = [&](void* bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, B, P.status)) != 0; };
        auto issue_qk = [&](int st, int hf) {
          const uint64_t dk = smem_desc_sw128(smem_u32(sK + st * kTileBytes + hf * (kTileBytes / 2)));
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < kHD / 16; ++kk) mma_ss(tm + kColS + hf * kHalf, dq + (uint64_t)(kk * 2), dk + (uint64_t)(kk * 2), idesc_qk, kk > 0);
            tc_commit(&B->s_full[i][hf]);
            if (hf == 1) tc_commit(&B->k_empty[st]);
          }
        };
        bool ok = wait_all(&B->k_full[0], 0);
        if (ok) {
          tc_fence_after();
          issue_qk(0, 0);
          issue_qk(0, 1);
        }
        for (int it = 0; it < n_tiles && ok; ++it) {
          const int s = it % kKVStages, s1 = (it + 1) % kKVStages;
          const uint32_t ph = (uint32_t)(it / kKVStages) & 1u, ph1 = (uint32_t)((it + 1) / kKVStages) & 1u;
          const bool more = it + 1 < n_tiles;
          ok = wait_all(&B->v_full[s], ph);
          if (!ok) break;
          const uint64_t dv = smem_desc_sw128(smem_u32(sV + s * kTileBytes));
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            ok = wait_all(&B->p_full[i][hf], (uint32_t)it & 1u);
            if (!ok) break;
            tc_fence_after();
            if (leader) {
#pragma unroll
              for (int kk = 0; kk < kHalf / 16; ++kk)
                mma_ts(tm + kColO, tm + kColS + hf * kHalf + kk * 8, dv + (uint64_t)((hf * (kHalf / 16) + kk) * 128), idesc_pv, (it > 0 || hf > 0 || kk > 0));
              if (hf == 1) tc_commit(&B->v_empty[s]);
              if (!more && hf == 0) tc_commit(&B->pv_done[i]);   // (the last half has no later score MMA to tell it by)
            }
            if (more) {
              if (hf == 0) {
                ok = wait_all(&B->k_full[s1], ph1);
                if (!ok) break;
                tc_fence_after();
              }
              issue_qk(s1, hf);
            }
          }
        }
        if (ok) {
          if (leader) tc_commit(&B->o_full[i]);
          wait_all(&B->o_full[i], 0);
        } else {
          if (leader) tc_commit(&B->drain[i]);           // let every issued MMA finish before TMEM is freed
          wait_all(&B->drain[i], 0);
        }
      }
      __syncwarp();
    } else if (n_tiles > 0) {
      // ------------------------------------------------ K and V
      // A thread has four adjacent rows of a tile, 16 columns of each, and reads back what it copied itself: no barrier between the copy
      // and the widening.  (Two threads next to each other take their rows in another order: their stores go to different banks.)
      const int ct = (int)threadIdx.x - 320, c = ct & 3, g = ct >> 2;
      const size_t pitch = (size_t)P.HK * kHD, base = ((size_t)seq * P.cap * P.HK + hk) * kHD + c * 16, xbase = ((size_t)seq * P.HK + hk) * P.cap;
      auto request = [&](int t) {
        if (t < n_tiles) {
          unsigned char* raw = sRaw + (t % kManyRaw) * kManyRawStage + ct * 16;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = (t_begin + t) * kBN + 4 * g + (i ^ (g & 1));
            const size_t at = base + (size_t)min(r, len - 1) * pitch;
            copy16(raw + i * (kManyConverters * 16), P.kq + at, r < len);
            copy16(raw + (4 + i) * (kManyConverters * 16), P.vq + at, r < len);
          }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
      struct Bytes { uint32_t k, v, live; };               // of the four rows
      auto bytes_of = [&](int t) {
        const int r = (t_begin + t) * kBN + 4 * g;         // (the capacity is a multiple of 16)
        Bytes b = {0u, 0u, 0xFFFFFFFFu};
        if (t < n_tiles && r < len) {
          b.k = __ldg(reinterpret_cast<const uint32_t*>(P.kx + xbase + r));
          b.v = __ldg(reinterpret_cast<const uint32_t*>(P.vx + xbase + r));
          if (P.live != nullptr) b.live = __ldg(reinterpret_cast<const uint32_t*>(P.live + (size_t)seq * P.cap + r));
        }
        return b;
      };
      auto widen = [&](bool values, int t, const Bytes& b, unsigned char* tiles) {
        const unsigned char* raw = sRaw + (t % kManyRaw) * kManyRawStage + (values ? 4 : 0) * (kManyConverters * 16) + ct * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int e = i ^ (g & 1), r = 4 * g + e;
          uint32_t x = b.k >> (8 * e) & 255u;
          // a row that is masked counts for nothing; one whose key is not finite makes the result NaN whatever its weight came out as
          if (values) x = (b.live >> (8 * e) & 255u) == 0u ? 0u : (x == 255u ? 255u : b.v >> (8 * e) & 255u);
          if ((t_begin + t) * kBN + r >= len) x = 0u;
          store_widened(tiles + t % kKVStages * kTileBytes, r, c, *reinterpret_cast<const uint4*>(raw + i * (kManyConverters * 16)), q8_step_bf16x2(x));
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      };
#pragma unroll
      for (int t = 0; t < kManyRaw - 1; ++t) request(t);
      Bytes next = bytes_of(0);
#pragma unroll 1
      for (int t = 0; t < n_tiles; ++t) {
        const Bytes b = next;
        next = bytes_of(t + 1);
        request(t + kManyRaw - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(kManyRaw - 1) : "memory");
        const int s = t % kKVStages;
        const uint32_t ph = (uint32_t)(t / kKVStages - 1) & 1u;
        if (t >= kKVStages && !mbar_wait(&B->k_empty[s], ph, B, P.status)) break;
        widen(false, t, b, sK);
        mbar_arrive(&B->k_full[s]);
        if (t >= kKVStages && !mbar_wait(&B->v_empty[s], ph, B, P.status)) break;
        widen(true, t, b, sV);
        mbar_arrive(&B->v_full[s]);
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      __syncwarp();
    }
    // ---- teardown: the softmax warps join the parts
    tc_fence_before();
    sync_all();
    if (warp == 8) {
      tc_fence_after();
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)(2 * kTmemCols)) : "memory");
    }
    if (S > 1) sync_all();
  } else {
    // ------------------------------------------------ softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegsSoftmax));
    const int i = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t t_row = tmem + i * kTmemCols + ((uint32_t)((warp & 3) * 32) << 16);
    const float c = 1.4426950408889634f * 0.125f;        // log2(e) / sqrt(64)
    float m = -INFINITY, l = 0.0f;
    bool ok = true, seen = false;                        // seen: some row is live
    for (int idx = 0; idx < 2 * n_tiles && ok && i < n_q; ++idx) {                // idx = 2 * tile + half
      const int it = idx >> 1, hf = idx & 1, col0 = (t_begin + it) * kBN + hf * kHalf;
      uint32_t mask[kHalf / 32];
      bool whole = P.live == nullptr && col0 + kHalf <= len;
      if (!whole) {
        whole = true;
#pragma unroll
        for (int j = 0; j < kHalf / 32; ++j) {
          const int r = col0 + 32 * j + lane;
          mask[j] = __ballot_sync(0xFFFFFFFFu, r < len && (P.live == nullptr || P.live[(size_t)seq * P.cap + r] != 0));
          whole = whole && mask[j] == 0xFFFFFFFFu;
          seen = seen || mask[j] != 0u;
        }
      } else {
        seen = true;
      }
      ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->s_full[i][hf], (uint32_t)it & 1u, B, P.status)) != 0;
      if (!ok) break;
      tc_fence_after();
      uint32_t s[kHalf];
      auto load_scores = [&]() {
#pragma unroll
        for (int j = 0; j < kHalf / 32; ++j) tmem_ld32(t_row + kColS + hf * kHalf + j * 32, s + j * 32);
        tmem_wait_ld();
        if (!whole) {
#pragma unroll
          for (int j = 0; j < kHalf; ++j)
            if (!(mask[j >> 5] >> (j & 31) & 1u)) s[j] = 0xFF800000u;
        }
      };
      // p = 2^(s c - reference) on pairs, packed to bf16 over the front of s[]; returns the row's sum of p and its largest raw score
      auto exp_pass = [&](auto track, float& raw) -> float {
        const float ref = m == -INFINITY ? 0.0f : m;
        const float2 c2 = make_float2(c, c), nm2 = make_float2(-ref, -ref);
        float2 acc[4];
        float m4[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          acc[q] = make_float2(0.0f, 0.0f);
          m4[q] = -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < kHalf; j += 2) {
          const float s0 = __uint_as_float(s[j]), s1 = __uint_as_float(s[j + 1]);
          if constexpr (decltype(track)::value) m4[(j >> 1) & 3] = max3(m4[(j >> 1) & 3], s0, s1);
          const float2 x = fma2(make_float2(s0, s1), c2, nm2);
          const float2 p = pair_on_fma_pipes(j >> 1) ? ex2_poly2<true>(x) : make_float2(ex2(x.x), ex2(x.y));
          acc[(j >> 1) & 3] = add2(acc[(j >> 1) & 3], p);
          s[j >> 1] = pack_bf16(p.x, p.y);
        }
        raw = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
        const float2 t = add2(add2(acc[0], acc[1]), add2(acc[2], acc[3]));
        return t.x + t.y;
      };
      load_scores();
      float add, raw;
      if (idx == 0) {
        // the first half fixes the reference: its maximum has to be known before any exponential
        float m4[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          m4[q] = fmaxf(__uint_as_float(s[24 * q]), __uint_as_float(s[24 * q + 1]));
#pragma unroll
          for (int j = 2; j < 24; j += 2) m4[q] = max3(m4[q], __uint_as_float(s[24 * q + j]), __uint_as_float(s[24 * q + j + 1]));
        }
        static_assert(kHalf == 96, "four chains of 24");
        m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * c;
        add = exp_pass(std::false_type{}, raw);
      } else {
        add = exp_pass(std::true_type{}, raw);
        const float mx = raw * c;
        const bool grow = mx - m > kRescaleThreshold;    // (also from nothing live to something)
        if (__any_sync(0xFFFFFFFFu, grow)) {
          // O may still be accumulating the half before: the scores of the next half, issued behind it, tell; or the last one's own barrier
          ok = idx + 1 < 2 * n_tiles ? mbar_wait(&B->s_full[i][hf ^ 1], (uint32_t)((idx + 1) >> 1) & 1u, B, P.status)
                                     : mbar_wait(&B->pv_done[i], 0, B, P.status);
          ok = __all_sync(0xFFFFFFFFu, ok) != 0;
          if (!ok) break;
          tc_fence_after();
          const float a = grow ? ex2(m - mx) : 1.0f;
          if (grow) {
            m = mx;
            l *= a;
          }
          uint32_t o[16];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            tmem_ld16(t_row + kColO + j * 16, o);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * a);
            tmem_st16(t_row + kColO + j * 16, o);
          }
          load_scores();
          add = exp_pass(std::false_type{}, raw);
        }
      }
      l += add;
      tmem_st32(t_row + kColS + hf * kHalf, s);
      tmem_st16(t_row + kColS + hf * kHalf + 32, s + 32);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(&B->p_full[i][hf]);
    }
    if (i < n_q) {
      float* o_row = sO + (i * kBM + row) * kManyPitch;
      if (n_tiles > 0 && ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->o_full[i], 0, B, P.status)) != 0;
      tc_fence_after();
      uint32_t o[32];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (n_tiles > 0 && ok) {
          tmem_ld32(t_row + kColO + j * 32, o);
          tmem_wait_ld();
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          *reinterpret_cast<uint4*>(o_row + 32 * j + 4 * e) = n_tiles > 0 && ok ? make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]) : make_uint4(0u, 0u, 0u, 0u);
      }
      // live rows, but no score that is a number, or one that is infinite
      if ((seen && m == -INFINITY) || m == INFINITY) l = __int_as_float(0x7FC00000);
      sO[kManyRows * kManyPitch + i * kBM + row] = m;
      sO[kManyRows * (kManyPitch + 1) + i * kBM + row] = seen ? l : 0.0f;
    }
    // ---- the cluster's parts in order, a share of the rows each
    tc_fence_before();
    sync_all();
    const int valid = min(kManyRows, rows - row0);
    for (int u = rank * 256 + threadIdx.x; u < valid * 16; u += S * 256) {
      const int r = u >> 4, c4 = u & 15;
      float mx = -INFINITY, sum = 0.0f;
      for (int s = 0; s < S; ++s) mx = fmaxf(mx, cluster.map_shared_rank(sO, s)[kManyRows * kManyPitch + r]);
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s = 0; s < S; ++s) {
        const float* part = cluster.map_shared_rank(sO, s);
        const float mi = part[kManyRows * kManyPitch + r], k = mi == mx ? 1.0f : exp2f(mi - mx);
        const float4 x = *reinterpret_cast<const float4*>(part + r * kManyPitch + 4 * c4);
        sum = fmaf(k, part[kManyRows * (kManyPitch + 1) + r], sum);
        a.x = fmaf(k, x.x, a.x); a.y = fmaf(k, x.y, a.y); a.z = fmaf(k, x.z, a.z); a.w = fmaf(k, x.w, a.w);
      }
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      *reinterpret_cast<uint2*>(P.out + q_at(row0 + r) + 4 * c4) = make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
    }
    if (S > 1) sync_all();                               // (nobody leaves while its part is being read)
  }
}

// CTAs that share the cached rows: waves over 148 SMs, each as long as its tiles of 192 rows and three more (set-up, joining).
inline int many_parts(long long jobs, int cap) {
  const int tiles = (cap + kBN - 1) / kBN;
  int best = 1;
  long long best_cost = -1;
  for (int s = 1; s <= 8 && s <= tiles; ++s) {
    const long long cost = (jobs * s + 147) / 148 * ((tiles + s - 1) / s + 3);
    if (best_cost < 0 || cost < best_cost) best_cost = cost, best = s;
  }
  return best;
}

constexpr int kManyFrom = 65;          // rows from which that kernel is taken

static inline int attn_q8_launch(AttnQ8Args P, cudaStream_t st) {
  const int rows = P.M * P.group;
  if (rows >= kManyFrom) {
    P.q_tiles = (rows + kManyRows - 1) / kManyRows;
    const long long jobs = (long long)P.seqs * P.HK * P.q_tiles;
    const int S = many_parts(jobs, P.cap);
    if (jobs * S > 0x7FFFFFFF) return OVGGT_ERR_UNSUPPORTED;
    static std::atomic<uint64_t> smem_many;
    cudaError_t e = allow_smem(k_attn_q8_many, kManySmem, smem_many);
    if (e == cudaSuccess) e = launch_dependent(k_attn_q8_many, dim3((unsigned)(jobs * S)), kManyThreads, S, kManySmem, st, true, P);
    if (e != cudaSuccess) { g_attn_last_error = (int)e; return OVGGT_ERR_CUDA; }
    return OVGGT_OK;
  }
  const int tile = rows <= 8 ? 8 : (rows <= 16 ? 16 : 32);
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
