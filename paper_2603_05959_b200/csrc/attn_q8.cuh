// Attention over an 8-bit cache: out = softmax(Q K^T / 8) V per head over the live rows of each sequence, head_dim 64; zero
// where no row is live.  Query heads h of a key head's group read that head; `rows` below are (token, query head of the group).
#pragma once

#include "gemm_q8.cuh"

namespace ovggt {

struct AttnQ8Args {
  const __nv_bfloat16* q;              // [seqs, M, H, 64]
  const int8_t *kq, *vq;               // [seqs, cap, HK, 64]
  const uint8_t *kx, *vx;              // [seqs, HK, cap]
  const int* lens;                     // [seqs] or nullptr: cap
  const uint8_t* live;                 // [seqs, cap] or nullptr
  __nv_bfloat16* out;                  // [seqs, M, H, 64]      (parts == 1)
  float* o_part;                       // un-normalised results of the parts of the cached rows: [parts, seqs * M, H * 64]
  float2* ml_part;                     // (reference maximum in log2 units, row sum): [parts, seqs * M, H]
  int seqs, M, H, HK, cap, group, q_tiles, parts;
  int* status;
};

// What stands for a part without live rows: a maximum below every other's, so that it weighs nothing beside a part that has some, and
// a sum that makes the result zero where no part has.
constexpr float kDeadMax = -3.4e38f, kDeadSum = 1.0f;

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first product of a sum that begins at `on`.
__device__ __forceinline__ void mma_s8_on(int (&c)[4], uint32_t on, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(on));
}
__device__ __forceinline__ void mma_u8s8(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Byte c of each of four words, in order, in word c.
__device__ __forceinline__ void transpose4(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t (&o)[4]) {
  const uint32_t ab = __byte_perm(a, b, 0x5140), cd = __byte_perm(c, d, 0x5140), ab2 = __byte_perm(a, b, 0x7362), cd2 = __byte_perm(c, d, 0x7362);
  o[0] = __byte_perm(ab, cd, 0x5410);
  o[1] = __byte_perm(ab, cd, 0x7632);
  o[2] = __byte_perm(ab2, cd2, 0x5410);
  o[3] = __byte_perm(ab2, cd2, 0x7632);
}
// 16 bytes into shared memory behind the thread's back; zeros where `in` is false.
__device__ __forceinline__ void copy16(void* dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 d = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&d);
}
// Two int8, the low bytes of the halves of x, as a pair of bf16, exact: 128 + the low seven bits, less 128 or, of a negative one, 256.
__device__ __forceinline__ uint32_t int8_to_bf16x2(uint32_t x) { return sub_bf16x2((x & 0x007F007Fu) | 0x43004300u, (x & 0x00800080u) | 0x43004300u); }

// ---------------------------------------------------------------- few rows: the cache streams through, once per 8, 16 or 32 rows
//
// What bounds it: the cache's bytes (the copies alone take 10 of 20 us of one row over 32768), and beside them the arithmetic on them, chains of
// copy, MMA, exponentials and MMA that a dozen warps an SM do not cover.  A warp takes tiles of 32 cached rows by itself, with three of them on their way in its own stages
// (no barrier in the loop); the warps' results are joined through shared memory, those of the CTAs that share a sequence and head (parts) by
// the bf16 attention's merge kernel.
//   scores  from queries that keep every bit.  With at most 8 rows by int8 MMAs on the cached bytes as they are: a row of Q is taken as whole
//           numbers of 31 bits in units of 2^-29 of its largest power of two, four int8 operands in the halves of two; where that would not
//           be exact (a row with elements below 2^-22 of its largest), and with more rows, by bf16 MMAs on Q itself and the cached bytes
//           made bf16.  (One row over 32768, 16 heads: 20.0 us, by bf16 MMAs 22.0; two operands' 15 bits took 18.4 and lost a row's small elements.)
//   P V     with at most 8 rows by int8 MMAs too: a weight p 2^(x - 133) as a whole number of 31 bits, 2^-28 of a reference that follows the largest
//           weight, four unsigned bytes in the halves of two operands; the cached bytes of four rows are only put side by side.  The int32 sums
//           are exact and go into fp32 when the reference moves.  With more rows, where that many sums do not fit the registers, by bf16 MMAs: the
//           cached bytes are exact in bf16, a weight is rounded to it (2^-8).
// Which cached row or column an operand's row or column stands for is free, so each lane takes 16 bytes of a K row and 8
// bytes of a V row at once.
// An SM holds as many warps as their registers leave without spilling (with queries of 15 bits four tokens over up to 16384 rows by 16 warps 28 us, by
// 12 25, now 29; 16 rows over 2048 8.6 and 7.9, now 8.0; 32 rows over 8192 by 12 warps 16.5, by 8 13.7, now 14.3), in one CTA or in two or three smaller ones (see attn_q8_plan).
__host__ __device__ constexpr int few_warps(int rows) { return rows == 32 ? 8 : 12; }
constexpr int kFewStages = 3, kFewKeys = 32;
constexpr int kFewX = 2 * kFewKeys * 64;                 // of a stage: K, V, then the exponents of K and V and the mask, 32 bytes each
constexpr int kFewStage = kFewX + 128;
constexpr int kFewTable = kFewKeys * 16;                 // of a warp: (step of K, 0 or -inf under the mask, step of V) for each row of its tile
__host__ __device__ constexpr int few_smem_bytes(int warps) { return warps * (kFewStages * kFewStage + kFewTable); }
static_assert(kFewStages * kFewStage >= 32 * (64 + 2) * 4, "a warp's result does not fit its stages");

template <int ROWS, int kFewWarps>
__global__ void __launch_bounds__(kFewWarps * 32, few_warps(ROWS) / kFewWarps) k_attn_q8_few(const AttnQ8Args P) {
  constexpr bool PACK = ROWS == 8;
  constexpr int T = PACK ? 1 : ROWS / 16;                // operands of 16 rows
  constexpr int R = PACK ? 1 : 2;                        // rows of an operand a thread holds scores of
  extern __shared__ __align__(1024) unsigned char smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int hk = (int)(blockIdx.x % P.HK), qt = (int)(blockIdx.x / P.HK % P.q_tiles), rest = (int)(blockIdx.x / P.HK / P.q_tiles);
  const int part = rest % P.parts, seq = rest / P.parts;
  const int rows = P.M * P.group, row0 = qt * ROWS;
  pdl_trigger();
  pdl_wait();
  const int len = min(P.cap, max(0, P.lens != nullptr ? P.lens[seq] : P.cap));
  const int tiles = (len + kFewKeys - 1) / kFewKeys;
  auto q_at = [&](int r) {                               // (row r is token r / group, head r % group of this group)
    const int m = r / P.group;
    return (((size_t)seq * P.M + m) * P.H + (size_t)hk * P.group + (r - m * P.group)) * 64;
  };

  // ---- the cache, tile by tile
  unsigned char* stages = smem + warp * kFewStages * kFewStage;
  const size_t pitch = (size_t)P.HK * 64, base = ((size_t)seq * P.cap * P.HK + hk) * 64, xbase = ((size_t)seq * P.HK + hk) * P.cap;
  const int first = part * kFewWarps + warp, stride = P.parts * kFewWarps;
  float4* table = reinterpret_cast<float4*>(smem + kFewWarps * kFewStages * kFewStage + warp * kFewTable);
  const int8_t* k_lane = P.kq + base + (size_t)g * pitch + t * 16;            // this lane's part of the cache's first row and every eighth after it
  const int8_t* v_lane = P.vq + base + (size_t)g * pitch + t * 16;
  // K rows lie so that the two of a lane's adjacent scores are four apart; V rows 2 and 3 of four have their halves exchanged.
  const int k_to = ((g & 3) * 2 + (g >> 2)) * 64 + t * 16, v_to = 2048 + g * 64 + (t ^ (g & 2)) * 16;
  const uint8_t* x_lane = nullptr;                       // lanes 0 to 5: sixteen bytes of the exponents and the mask
  if (lane < 4 || (lane < 6 && P.live != nullptr))
    x_lane = (lane < 2 ? P.kx + xbase : (lane < 4 ? P.vx + xbase : P.live + (size_t)seq * P.cap)) + (lane & 1) * 16;
  auto request = [&](int tile, int stage) {
    if (tile < tiles) {
      unsigned char* s = stages + stage * kFewStage;
      const int row0 = tile * kFewKeys;
      const size_t at = (size_t)row0 * pitch;
      if (row0 + kFewKeys <= len) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          copy16(s + k_to + i * 512, k_lane + at + i * 8 * pitch, true);
          copy16(s + v_to + i * 512, v_lane + at + i * 8 * pitch, true);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool in = row0 + 8 * i + g < len;
          const size_t from = in ? at + i * 8 * pitch : 0;
          copy16(s + k_to + i * 512, in ? k_lane + from : P.kq, in);
          copy16(s + v_to + i * 512, in ? v_lane + from : P.vq, in);
        }
      }
      // (the capacity is a multiple of 16)
      if (x_lane != nullptr && row0 + (lane & 1) * 16 < P.cap) copy16(s + kFewX + lane * 16, x_lane + row0, true);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < kFewStages - 1; ++s) request(first + s * stride, s);

  // ---- the operands of Q: of a row the 16 columns of which this lane reads K, two by two as K's bytes come apart, times the power of two
  // that brings the row's largest near one (a query may have any size, and the products' sums are fp32)
  // [four of its columns]: row g, (row g + 8,) columns 0 and 2 of them, then 1 and 3; or the four bytes of all four columns, from the highest
  uint32_t qa[T][4][PACK ? 4 : 2 * R];
  float f[T][R];                                         // a score in log2 units is f x the product with the whole numbers x 2^(kx - 127)
  bool odd[T][R];                                        // a query that is not finite: its result is not a number
  bool wide = false;                                     // of this warp's rows: some element is below 2^-22 of its row's largest
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = row0 + 16 * i + 8 * r + g;
      uint4 x[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
      if (row < rows) {
        const uint4* p = reinterpret_cast<const uint4*>(P.q + q_at(row) + 16 * t);
        x[0] = p[0];
        x[1] = p[1];
      }
      uint32_t* w = &x[0].x;
      uint32_t most = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) most = max(most, max(w[e] << 16 & 0x7FFFFFFFu, w[e] & 0x7FFF0000u));
      most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
      most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
      odd[i][r] = most >= 0x7F800000u;
      const int e2 = min(max((int)(most >> 23) - 127, -100), 126);            // (down to 2^-100 and no further: f stays normal)
      const uint32_t scale = odd[i][r] ? 0u : (uint32_t)(127 - e2) << 7 | (uint32_t)(127 - e2) << 23;
      f[i][r] = 1.4426950408889634f * 0.125f * __int_as_float((e2 - 6 + 127) << 23);       // (2^-6: cached values are 2^(x - 133))
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = odd[i][r] ? 0u : mul_bf16x2(w[j], scale);
      if constexpr (PACK) {
        // (now in units of 2^-29: whole numbers of 31 bits as long as no element is below 2^-22)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint32_t a = w[j] << 16 & 0x7FFFFFFFu, b = w[j] & 0x7FFF0000u;
          wide |= (a != 0u && a < 0x34800000u) || (b != 0u && b < 0x34800000u);
        }
        wide = __any_sync(0xFFFFFFFFu, wide) != 0;
        if (wide) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            qa[0][j][0] = __byte_perm(w[2 * j], w[2 * j + 1], 0x5410);
            qa[0][j][1] = __byte_perm(w[2 * j], w[2 * j + 1], 0x7632);
            qa[0][j][2] = qa[0][j][3] = 0u;
          }
        } else {
          f[0][0] *= 0.03125f;                           // (the highest byte counts 2^24 units)
#pragma unroll
          for (int j = 0; j < 4; ++j) {                  // four columns: their bytes, from the highest, each rounded so that what is left fits a signed byte
            uint32_t plane[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t half = w[2 * j + (e >> 1)];
              int z = __float2int_rn(__uint_as_float(e & 1 ? half & 0xFFFF0000u : half << 16) * 536870912.0f);
#pragma unroll
              for (int b = 3; b >= 0; --b) {
                const int low = (int)(int8_t)z;
                plane[b] |= ((uint32_t)low & 255u) << 8 * e;
                z = (z - low) >> 8;
              }
            }
#pragma unroll
            for (int b = 0; b < 4; ++b) qa[0][j][b] = plane[b];
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          qa[i][j][r] = __byte_perm(w[2 * j], w[2 * j + 1], 0x5410);
          qa[i][j][R + r] = __byte_perm(w[2 * j], w[2 * j + 1], 0x7632);
        }
      }
    }

  float m[T][R], l[T][R], o[T][8][4];                    // O: with at most 8 rows two columns a register pair, [0] and [1]
  int c1[PACK ? 8 : 1][4], c2[PACK ? 8 : 1][4], since = 0;   // what the int8 MMAs have summed up since O was last brought up to date, in how many tiles
  float mv = -INFINITY;                                  // log2 of the reference weight times step, over 2^m (the scores themselves may be far from zero)
#pragma unroll
  for (int d = 0; d < (PACK ? 8 : 1); ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) c1[d][e] = c2[d][e] = 0;
  auto take_sums = [&](float scale) {                    // O = (O + sums) scale
#pragma unroll
    for (int d = 0; d < (PACK ? 8 : 1); ++d) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float hi = fmaf((float)c1[d][e], 256.0f, (float)c1[d][e + 2]), lo = fmaf((float)c2[d][e], 256.0f, (float)c2[d][e + 2]);
        o[0][d][e] = (o[0][d][e] + fmaf(hi, 65536.0f, lo)) * scale;
        c1[d][e] = c1[d][e + 2] = c2[d][e] = c2[d][e + 2] = 0;
      }
    }
    since = 0;
  };
  constexpr float kUnits = 28.0f, kRoom = 3.0f;          // a reference weight is 2^28 units; another is at most 2^3 of it
  constexpr int kSumsMost = 2000;                        // tiles: 64000 x 255 x 127 is below 2^31
  // With more rows O is in units of 2^(xv - 133), so that a weight times a value's step is a number bf16 holds whatever the values' size: xv is
  // the largest exponent seen, or up to 2^4 below it.
  int xv = 7;
  constexpr int kRoomX = 4;
#pragma unroll
  for (int i = 0; i < T; ++i) {
#pragma unroll
    for (int r = 0; r < R; ++r) m[i][r] = -INFINITY, l[i][r] = 0.0f;
#pragma unroll
    for (int d = 0; d < 8; ++d) o[i][d][0] = o[i][d][1] = o[i][d][2] = o[i][d][3] = 0.0f;
  }
  auto stream = [&](auto by_bytes) {                     // the loop over this warp's tiles
    constexpr bool kBytes = decltype(by_bytes)::value;   // Q by its bytes
    int stage = 0;
#pragma unroll 1
    for (int tile = first; tile < tiles; tile += stride) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 2) : "memory");
      __syncwarp();                                      // this tile has arrived, and all lanes are done with the one before
      request(tile + (kFewStages - 1) * stride, stage == 0 ? kFewStages - 1 : stage - 1);
      const unsigned char* s = stages + stage * kFewStage;
      stage = stage + 1 == kFewStages ? 0 : stage + 1;

      {                                                  // a lane a row: what its scores and its weight are multiplied with
        const bool in = tile * kFewKeys + lane < len && (P.live == nullptr || s[kFewX + 64 + lane] != 0);
        // (255: infinity, which a block of zeros makes NaN)
        const uint32_t vx = s[kFewX + 32 + lane];
        const float ks = __int_as_float((int)s[kFewX + lane] << 23);
        if constexpr (PACK)                              // (the exponent of the value's step; a value that is not finite takes its score with it)
          table[lane] = in ? make_float4(ks, vx == 255u ? __int_as_float(0x7FC00000) : 0.0f, (float)((int)vx - 133), 0.0f) : make_float4(0.0f, -INFINITY, 0.0f, 0.0f);
        else {
          const int most = in && vx != 255u ? (int)vx : 0;
          if (__any_sync(0xFFFFFFFFu, most > xv + kRoomX)) {
            const int to = __reduce_max_sync(0xFFFFFFFFu, most);
            const float down = to - xv > 126 ? 0.0f : __int_as_float((127 - (to - xv)) << 23);
            xv = to;
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
              for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][d][e] *= down;
          }
          const float vs = vx == 255u ? __int_as_float(0x7FC00000) : __int_as_float(max((int)vx - xv + 127, 0) << 23);
          table[lane] = in ? make_float4(ks, 0.0f, vs, 0.0f) : make_float4(0.0f, -INFINITY, 0.0f, 0.0f);
        }
      }
      __syncwarp();
      float sc[T][R][8], vs[8];                          // scores of keys 8 b + t (even entries) and 8 b + t + 4
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const uint4 kw = *reinterpret_cast<const uint4*>(s + (8 * b + g) * 64 + t * 16);
        float4 x[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[e] = table[8 * b + t + 4 * e];
          vs[2 * b + e] = x[e].z;
        }
        if constexpr (kBytes) {
          // (sums of at most 2^20 in size, on top of 1.5 2^23: read as fp32 they need no conversion)
          constexpr uint32_t kMagic = 0x4B400000u;
          int c[4], d[4];
          mma_s8_on(c, kMagic, qa[0][0][0], qa[0][0][1], qa[0][1][0], qa[0][1][1], kw.x, kw.y);
          mma_s8(c, qa[0][2][0], qa[0][2][1], qa[0][3][0], qa[0][3][1], kw.z, kw.w);
          mma_s8_on(d, kMagic, qa[0][0][2], qa[0][0][3], qa[0][1][2], qa[0][1][3], kw.x, kw.y);
          mma_s8(d, qa[0][2][2], qa[0][2][3], qa[0][3][2], qa[0][3][3], kw.z, kw.w);
          const float2 back = make_float2(-12582912.0f, -12582912.0f), down = make_float2(0.00390625f, 0.00390625f);
          float2 y = add2(make_float2(__int_as_float(d[2]), __int_as_float(d[3])), back);
          y = fma2(y, down, add2(make_float2(__int_as_float(d[0]), __int_as_float(d[1])), back));
          y = fma2(y, down, add2(make_float2(__int_as_float(c[2]), __int_as_float(c[3])), back));
          y = fma2(y, down, add2(make_float2(__int_as_float(c[0]), __int_as_float(c[1])), back));
          sc[0][0][2 * b] = fmaf(y.x, f[0][0] * x[0].x, x[0].y);
          sc[0][0][2 * b + 1] = fmaf(y.y, f[0][0] * x[1].x, x[1].y);
        } else {
          float c[T][4];
#pragma unroll
          for (int i = 0; i < T; ++i) c[i][0] = c[i][1] = c[i][2] = c[i][3] = 0.0f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {                  // four bytes of a key: columns 0 and 2, 1 and 3
            const uint32_t four = j == 0 ? kw.x : (j == 1 ? kw.y : (j == 2 ? kw.z : kw.w));
            const uint32_t b0 = int8_to_bf16x2(four), b1 = int8_to_bf16x2(four >> 8);
#pragma unroll
            for (int i = 0; i < T; ++i) mma_bf16(c[i], qa[i][j][0], PACK ? 0u : qa[i][j][1], qa[i][j][R], PACK ? 0u : qa[i][j][2 * R - 1], b0, b1);
          }
#pragma unroll
          for (int i = 0; i < T; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
              for (int e = 0; e < 2; ++e) sc[i][r][2 * b + e] = fmaf(c[i][2 * r + e], f[i][r] * x[e].x, x[e].y);
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
      auto top_weight = [&](float x) {                   // of the tile, over 2^x
        const float ref = x == -INFINITY ? 0.0f : x;
        float y = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) y = fmaxf(y, sc[0][0][e] - ref + vs[e]);
        y = fmaxf(y, __shfl_xor_sync(0xFFFFFFFFu, y, 1));
        return fmaxf(y, __shfl_xor_sync(0xFFFFFFFFu, y, 2));
      };
      if constexpr (PACK) {
        const float topv = top_weight(m[0][0]);
        grown |= topv > mv + kRoom || since >= kSumsMost;
      }
      if (__any_sync(0xFFFFFFFFu, grown)) {
        if constexpr (PACK) {
          const float to = fmaxf(m[0][0], top[0][0]);
          if (m[0][0] != to) mv += m[0][0] - to;         // (both are -inf before the first live row)
          const float mn = fmaxf(mv, top_weight(to));
          if (since > 0) take_sums(mv == mn ? 1.0f : ex2(mv - mn));
          mv = mn;
        }
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float mn = fmaxf(m[i][r], top[i][r]), corr = m[i][r] == mn ? 1.0f : ex2(m[i][r] - mn);
            m[i][r] = mn;
            l[i][r] *= corr;
            if constexpr (!PACK) {
#pragma unroll
              for (int d = 0; d < 8; ++d) {
                o[i][d][2 * r] *= corr;
                o[i][d][2 * r + 1] *= corr;
              }
            }
          }
      }
      if constexpr (PACK) {
        const float ref = m[0][0] == -INFINITY ? 0.0f : m[0][0], up = kUnits - (mv == -INFINITY ? 0.0f : mv);
        const float2 back = make_float2(-ref, -ref), up2 = make_float2(up, up);
        float2 sum = make_float2(0.0f, 0.0f);
        uint32_t w[8];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const float2 d = add2(make_float2(sc[0][0][2 * b], sc[0][0][2 * b + 1]), back), y = add2(add2(d, make_float2(vs[2 * b], vs[2 * b + 1])), up2);
          sum = add2(sum, make_float2(ex2(d.x), ex2(d.y)));
          w[2 * b] = __float2uint_rn(ex2(y.x));
          w[2 * b + 1] = __float2uint_rn(ex2(y.y));
        }
        l[0][0] += sum.x + sum.y;
        // operands: row g the top byte of the weights (a1) or the second lowest (a2), row g + 8 the byte below; 4 k's a register
        uint32_t a1[4], a2[4], x[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          transpose4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3], x);
          a1[2 * h] = x[3];
          a1[2 * h + 1] = x[2];
          a2[2 * h] = x[1];
          a2[2 * h + 1] = x[0];
        }
        uint2 v[8];                                      // rows t, t + 4, ...: the order of the weights
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const uint2*>(s + 2048 + (t + 4 * e) * 64 + (((g >> 1) ^ (t & 2)) * 16) + (g & 1) * 8);
#pragma unroll
        for (int half = 0; half < 2; ++half) {           // four columns
          uint32_t b0[4], b1[4];
          transpose4(half ? v[0].y : v[0].x, half ? v[1].y : v[1].x, half ? v[2].y : v[2].x, half ? v[3].y : v[3].x, b0);
          transpose4(half ? v[4].y : v[4].x, half ? v[5].y : v[5].x, half ? v[6].y : v[6].x, half ? v[7].y : v[7].x, b1);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            mma_u8s8(c1[4 * half + d], a1, b0[d], b1[d]);
            mma_u8s8(c2[4 * half + d], a2, b0[d], b1[d]);
          }
        }
        ++since;                                         // (the same in every lane)
      } else {
        uint32_t pa[T][2][4];                                // P of 16 keys as an operand
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float ref = m[i][r] == -INFINITY ? 0.0f : m[i][r];
            const float2 back = make_float2(-ref, -ref);
            float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const float2 d = add2(make_float2(sc[i][r][2 * b], sc[i][r][2 * b + 1]), back), p = make_float2(ex2(d.x), ex2(d.y));
              sum = add2(sum, p);
              const float w0 = p.x * vs[2 * b], w1 = p.y * vs[2 * b + 1];
              pa[i][b >> 1][(b & 1) * 2 + r] = pack_bf16(w0, w1);
            }
            l[i][r] += sum.x + sum.y;
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
              w[e][0] = __byte_perm(x, y, 0x5410);           // columns 0 and 1 of both, then 2 and 3
              w[e][1] = __byte_perm(x, y, 0x7632);
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) {
              const uint32_t b0 = int8_to_bf16x2(w[0][d >> 1] >> (d & 1) * 8), b1 = int8_to_bf16x2(w[1][d >> 1] >> (d & 1) * 8);
#pragma unroll
              for (int i = 0; i < T; ++i) mma_bf16(o[i][4 * half + d], pa[i][b][0], pa[i][b][1], pa[i][b][2], pa[i][b][3], b0, b1);
            }
          }
        }
      }
    }
  };
  if constexpr (PACK) {                                  // (loops of their own: with the choice inside one, a tenth slower)
    if (wide) stream(std::false_type{});
    else stream(std::true_type{});
  } else {
    stream(std::false_type{});
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncwarp();

  // ---- a warp's result into its stages: O [ROWS][64], the maxima, the sums
  float* mine = reinterpret_cast<float*>(stages);
  if constexpr (PACK) {                                  // (2^(mv - 28) by halves: a value's step may be 2^-126, and with the units' 2^-28 their product is no fp32 number)
    const float half = mv == -INFINITY ? 0.0f : ex2(0.5f * mv);
    take_sums(half * 3.725290298461914e-09f);
#pragma unroll
    for (int d = 0; d < 8; ++d) o[0][d][0] *= half, o[0][d][1] *= half;
  } else {
    const float units = __int_as_float((xv - 6) << 23);
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int d = 0; d < 8; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][d][e] *= units;
  }
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float x = l[i][r];
      x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
      x += __shfl_xor_sync(0xFFFFFFFFu, x, 2);
      if (odd[i][r] && m[i][r] != -INFINITY) x = __int_as_float(0x7FC00000);
      const int row = 16 * i + 8 * r + g;
      if (t == 0) mine[ROWS * 64 + row] = m[i][r], mine[ROWS * 65 + row] = x;
#pragma unroll
      for (int e = 0; e < 2; ++e)                        // (column n of an MMA is 8 n + d)
#pragma unroll
        for (int d = 0; d < 8; d += 4) {
          float4 y;
          float* z = &y.x;
#pragma unroll
          for (int q = 0; q < 4; ++q) z[q] = o[i][d + q][2 * r + e];
          *reinterpret_cast<float4*>(mine + row * 64 + 16 * t + 8 * e + d) = y;
        }
    }
  __syncthreads();
  // ---- the CTA's: sum O_i 2^(m_i - m), sum l_i 2^(m_i - m) over its warps in order
  constexpr int kPart = kFewStages * kFewStage / 4;
  for (int u = threadIdx.x; u < ROWS * 16; u += kFewWarps * 32) {
    const int row = u >> 4, c4 = u & 15;
    if (row0 + row >= rows) break;
    const float* parts = reinterpret_cast<const float*>(smem);
    float mx = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) mx = fmaxf(mx, parts[w * kPart + ROWS * 64 + row]);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kFewWarps; ++w) {
      const float mi = parts[w * kPart + ROWS * 64 + row], k = mi == mx ? 1.0f : exp2f(mi - mx);   // (both -inf: nothing was live)
      const float4 x = *reinterpret_cast<const float4*>(parts + w * kPart + row * 64 + 4 * c4);
      sum = fmaf(k, parts[w * kPart + ROWS * 65 + row], sum);
      a.x = fmaf(k, x.x, a.x); a.y = fmaf(k, x.y, a.y); a.z = fmaf(k, x.z, a.z); a.w = fmaf(k, x.w, a.w);
    }
    const size_t at = q_at(row0 + row);
    if (P.parts == 1) {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      *reinterpret_cast<uint2*>(P.out + at + 4 * c4) = make_uint2(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv));
    } else {
      const size_t to = (size_t)part * P.seqs * P.M * P.H * 64 + at;
      *reinterpret_cast<float4*>(P.o_part + to + 4 * c4) = a;
      if (c4 == 0) P.ml_part[to / 64] = make_float2(mx == -INFINITY ? kDeadMax : mx, sum == 0.0f ? kDeadSum : sum);
    }
  }
}

// ---------------------------------------------------------------- many rows: tcgen05 over bf16 planes
//
// From some tiles of queries on (see attn_q8_by_planes), widening the cache once, into bf16 planes in scratch memory, costs less than each tile's
// doing it: a plane takes some 3 instructions an element and 5 bytes of traffic, most of it in L2 (17758 rows of 16 heads: 22 us, 26 from memory, beside 128 of
// attention and merge for 11 tiles of queries; widened on the way into shared memory, once for two tiles, the same attention took 250 us: the
// widening warps share the issue slots with the softmax).  The planes are what the cache stands for: q 2^(x - 133) is exact in bf16.
constexpr size_t kPlanesAtOnce = (size_t)128 << 20;      // bytes of planes up to which sequences are taken together: what stays in L2
constexpr size_t kPlanesMost = (size_t)2 << 30;          // beyond which the few-row kernel takes any number of rows

// 2^(x - 133) as a pair of bf16; NaN for 255.
__device__ __forceinline__ uint32_t q8_step_bf16x2(uint32_t x) { return (x == 255u ? 0x7FFFu : (max(x, 6u) - 6u) << 7) * 0x00010001u; }

// Where the live rows of each 64 of a sequence go among its live rows, and how many there are: they lie without gaps in the planes, so
// the attention's loop knows no mask.  One CTA a sequence.
constexpr int kWidenRows = 64;
struct LiveArgs {
  const int* lens;
  const uint8_t* live;
  int *first, *count;                  // [seqs, blocks], [seqs]
  int cap, blocks;
};
__device__ __forceinline__ int q8_length(const int* lens, int seq, int cap) { return lens != nullptr ? min(cap, max(0, lens[seq])) : cap; }
// A 64-row block's mask: bit r for row 64 block + r.
__device__ __forceinline__ unsigned long long live_bits(const uint8_t* live, int len, int row0) {
  unsigned long long bits = 0;
#pragma unroll
  for (int i = 0; i < kWidenRows / 16; ++i)
    if (row0 + 16 * i < len) {                           // (the capacity is a multiple of 16)
      const uint4 u = *reinterpret_cast<const uint4*>(live + row0 + 16 * i);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t top = __vcmpne4(w[e], 0u) & 0x08040201u, nibble = (top | top >> 8 | top >> 16 | top >> 24) & 15u;
        bits |= (unsigned long long)nibble << (16 * i + 4 * e);
      }
    }
  const int left = len - row0;
  return left >= kWidenRows ? bits : (left <= 0 ? 0ull : bits & ((1ull << left) - 1ull));
}
__global__ void __launch_bounds__(1024) k_live_rows(const LiveArgs P) {
  __shared__ int sh[32];
  pdl_trigger();
  pdl_wait();
  const int seq = blockIdx.x, len = q8_length(P.lens, seq, P.cap);
  const uint8_t* live = P.live + (size_t)seq * P.cap;
  int before = 0;
  for (int b0 = 0; b0 < P.blocks; b0 += 1024) {
    const int b = b0 + (int)threadIdx.x;
    int total;
    const int at = block_excl_scan_int(b < P.blocks ? __popcll(live_bits(live, len, b * kWidenRows)) : 0, sh, &total);
    if (b < P.blocks) P.first[(size_t)seq * P.blocks + b] = before + at;
    before += total;
  }
  if (threadIdx.x == 0) P.count[seq] = before;
}

struct WidenArgs {
  const uint4 *kq, *vq;                // [seqs, cap, HK * 64] int8
  const uint8_t *kx, *vx;
  const int* lens;
  const uint8_t* live;
  const int *first, *count;            // of the live rows, where there is a mask
  uint4 *k, *v;                        // [seqs, rows, HK * 64] bf16
  unsigned* norms;                     // [seqs, rows / 64, HK]: the bits of the largest squared norm of a key of these rows
  int cap, HK, rows;                   // rows: the capacity up to whole tiles
};

// A CTA takes 64 rows of four heads, sixteen elements a thread at a time, their exponents by way of shared memory: all of a thread's loads are
// on their way at once (17758 rows of 16 heads: 23.6 us with all heads in a CTA).  Behind the last row, up to the end of its tile, come zeros.  A value
// whose key is not finite becomes NaN with it: that makes the result NaN whatever its weight comes out as.
constexpr int kWidenHeads = 4, kWidenUnits = kWidenRows * kWidenHeads * 4 / 256;   // heads of a CTA, units of a thread
__global__ void __launch_bounds__(256) k_widen_q8(const WidenArgs P) {
  __shared__ uint8_t from[kWidenRows];                   // the live rows of this block, in order
  __shared__ __align__(16) uint8_t sx[kWidenHeads][kWidenRows];
  __shared__ unsigned top[kWidenHeads];
  pdl_trigger();
  const int seq = blockIdx.y, side = blockIdx.z & 1, h0 = (int)(blockIdx.z >> 1) * kWidenHeads, row0 = (int)blockIdx.x * kWidenRows;
  const int heads = min(kWidenHeads, P.HK - h0), units = heads * 4;               // of a row here
  const size_t pitch = (size_t)P.HK * 4;                 // 16-byte words of a cached row
  if (threadIdx.x < kWidenHeads) top[threadIdx.x] = 0u;
  pdl_wait();
  const int len = q8_length(P.lens, seq, P.cap);
  const int have = max(0, min(kWidenRows, len - row0));
  int n = have, to = row0, count = len;
  if (P.live != nullptr) {
    count = P.count[seq];
    if (threadIdx.x >= 224) {
      const unsigned long long bits = live_bits(P.live + (size_t)seq * P.cap, len, row0);
      for (int r = threadIdx.x - 224; r < kWidenRows; r += 32)
        if (bits >> r & 1ull) from[__popcll(bits & ((1ull << r) - 1ull))] = (uint8_t)r;
    }
    to = P.first[(size_t)seq * gridDim.x + blockIdx.x];
    n = (blockIdx.x + 1 < gridDim.x ? P.first[(size_t)seq * gridDim.x + blockIdx.x + 1] : count) - to;
    __syncthreads();
  }
  const int all = n * units;
  const uint4* src = (side == 0 ? P.kq : P.vq) + ((size_t)seq * P.cap + row0) * pitch + h0 * 4;
  uint4 w[kWidenUnits];
#pragma unroll
  for (int j = 0; j < kWidenUnits; ++j) {
    const int u = threadIdx.x + 256 * j, i = u / units;
    if (u < all) w[j] = __ldcg(src + (P.live != nullptr ? from[i] : i) * pitch + (u - i * units));
  }
  if ((int)threadIdx.x < units) {                        // (16 rows at a time: the capacity is a multiple of 16)
    const int h = threadIdx.x >> 2, r = (threadIdx.x & 3) * 16;
    if (r < have) {
      const size_t at = ((size_t)seq * P.HK + h0 + h) * P.cap + row0 + r;
      uint4 x = *reinterpret_cast<const uint4*>(P.kx + at);
      if (side == 1) {
        const uint4 y = *reinterpret_cast<const uint4*>(P.vx + at);
        x.x = y.x | __vcmpeq4(x.x, 0xFFFFFFFFu);
        x.y = y.y | __vcmpeq4(x.y, 0xFFFFFFFFu);
        x.z = y.z | __vcmpeq4(x.z, 0xFFFFFFFFu);
        x.w = y.w | __vcmpeq4(x.w, 0xFFFFFFFFu);
      }
      *reinterpret_cast<uint4*>(&sx[h][r]) = x;
    }
  }
  __syncthreads();
  uint4* dst = (side == 0 ? P.k : P.v) + (size_t)seq * P.rows * pitch * 2 + h0 * 8;
#pragma unroll
  for (int j = 0; j < kWidenUnits; ++j) {
    const int u = threadIdx.x + 256 * j, i = u / units, part = u - i * units;
    if (u < all) {
      const uint32_t x = sx[part >> 2][P.live != nullptr ? from[i] : i], step = q8_step_bf16x2(x), in[4] = {w[j].x, w[j].y, w[j].z, w[j].w};
      uint32_t o[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[2 * e] = mul_bf16x2(int8_to_bf16x2(__byte_perm(in[e], 0u, 0x4140)), step);
        o[2 * e + 1] = mul_bf16x2(int8_to_bf16x2(__byte_perm(in[e], 0u, 0x4342)), step);
      }
      uint4* d = dst + (size_t)(to + i) * pitch * 2 + 2 * part;
      d[0] = make_uint4(o[0], o[1], o[2], o[3]);
      d[1] = make_uint4(o[4], o[5], o[6], o[7]);
      if (side == 0) {                                   // (four lanes have a key of a head: whole numbers of at most 64 x 127^2)
        int n2 = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) n2 = __dp4a((int)in[e], (int)in[e], n2);
        const unsigned quad = 15u << (threadIdx.x & 28);
        n2 += __shfl_xor_sync(quad, n2, 1);
        n2 += __shfl_xor_sync(quad, n2, 2);
        const float f = q8_step(x);
        if ((part & 3) == 0) atomicMax(&top[part >> 2], __float_as_uint((float)n2 * f * f) & 0x7FFFFFFFu);
      }
    }
  }
  if (side == 0) {
    __syncthreads();
    if ((int)threadIdx.x < heads) P.norms[((size_t)seq * gridDim.x + blockIdx.x) * P.HK + h0 + threadIdx.x] = top[threadIdx.x];
  }
  // this CTA's share of the zeros: rows [row0, row0 + 64) of the planes
  const int z0 = max(row0, count), z1 = min(row0 + kWidenRows, (count + kBN - 1) / kBN * kBN);
  for (int u = threadIdx.x; u < (z1 - z0) * units * 2; u += 256) {
    const int i = u / (units * 2);
    dst[(size_t)(z0 + i) * pitch * 2 + (u - i * units * 2)] = make_uint4(0u, 0u, 0u, 0u);
  }
}

// The bf16 attention's scheme (see attn_tcgen05.cuh: the same warps, tiles, halves and order of MMAs, two CTAs an SM) with lengths that are
// read here, sequences and shared heads, and sequences without a live row.
constexpr int kManyBar = kQBytes + 2 * kKVStages * kTileBytes;
constexpr int kManySmem = kManyBar + (int)sizeof(AttnBarriers) + 64;

// What a CTA takes: a tile of rows, a key head, a part of the cached rows, a sequence.
struct Place {
  int row0, hk, part, seq;
  __device__ __forceinline__ Place(const AttnQ8Args& P, unsigned block) {
    const unsigned a = block / P.q_tiles, b = a / P.HK;
    row0 = (int)(block - a * P.q_tiles) * kBM;
    hk = (int)(a - b * P.HK);
    seq = (int)(b / P.parts);
    part = (int)(b - (unsigned)seq * P.parts);
  }
  // Where row r lies in q and out: it is token r / group, head r % group of this group.
  __device__ __forceinline__ size_t q(const AttnQ8Args& P, int r) const {
    const int m = r / P.group;
    return (((size_t)seq * P.M + m) * P.H + (size_t)hk * P.group + (r - m * P.group)) * kHD;
  }
};

__global__ void __launch_bounds__(kAttnThreads, kCtasPerSm)
k_attn_q8_many(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ AttnQ8Args P, const int* counts, const unsigned* norms, const int plane_rows) {
  extern __shared__ __align__(1024) unsigned char smem[];
  if (smem_u32(smem) & 1023u) {                          // the 128-byte swizzle needs 1024-byte aligned tiles
    if (threadIdx.x == 0) report_status(P.status, OVGGT_ERR_DEVICE_STATUS);
    return;
  }
  unsigned char* sQ = smem;
  unsigned char* sK = sQ + kQBytes;
  unsigned char* sV = sK + kKVStages * kTileBytes;
  AttnBarriers* B = reinterpret_cast<AttnBarriers*>(smem + kManyBar);
  unsigned* top = reinterpret_cast<unsigned*>(B + 1);    // [8]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Place at0(P, blockIdx.x);
  const int hk = at0.hk, part = at0.part, seq = at0.seq;
  pdl_trigger();
  if (warp == 4 && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_v) : "memory");
    for (int hf = 0; hf < 2; ++hf) {
      mbar_init(&B->s_full[hf], 1);
      mbar_init(&B->p_full[hf], 128);
    }
    mbar_init(&B->pv_done, 1);
    mbar_init(&B->o_full, 1);
    mbar_init(&B->drain, 1);
    for (int s = 0; s < kKVStages; ++s) {
      mbar_init(&B->k_full[s], 1);
      mbar_init(&B->k_empty[s], 1);
      mbar_init(&B->v_empty[s], 1);
      mbar_init(&B->v_full[s], 1);
    }
    B->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 5) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&B->tmem_base)), "r"((uint32_t)kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  const int len = counts != nullptr ? counts[seq] : q8_length(P.lens, seq, P.cap);      // live rows
  const int tiles_total = (len + kBN - 1) / kBN;
  const int t_begin = (int)((long long)part * tiles_total / P.parts), n_tiles = (int)((long long)(part + 1) * tiles_total / P.parts) - t_begin;
  // What the first tiles need is requested at once: K and V by the producer's thread, the queries (128 rows x 8 groups of 8 columns, rows
  // past the last zero) and the norms of this head's keys by all.
  const int plane_row = seq * plane_rows + t_begin * kBN;
  if (warp == 4 && lane == 0 && n_tiles > 0) {
    mbar_expect_tx(&B->k_full[0], kTileBytes);
    tma_load_2d(sK, &tm_k, hk * kHD, plane_row, &B->k_full[0]);
    mbar_expect_tx(&B->v_full[0], kTileBytes);
    tma_load_2d(sV, &tm_v, hk * kHD, plane_row, &B->v_full[0]);
  }
  {
    constexpr int kPer = kBM * 8 / kAttnThreads;
    uint4 x[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int idx = threadIdx.x + i * kAttnThreads, r = at0.row0 + (idx >> 3);
      x[i] = r < P.M * P.group ? *reinterpret_cast<const uint4*>(P.q + at0.q(P, r) + (idx & 7) * 8) : make_uint4(0u, 0u, 0u, 0u);
    }
    unsigned most = 0u;
    const int blocks = (q8_length(P.lens, seq, P.cap) + kWidenRows - 1) / kWidenRows;
    for (int b = threadIdx.x; b < blocks; b += kAttnThreads) most = max(most, norms[((size_t)seq * (plane_rows / kWidenRows) + b) * P.HK + hk]);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int idx = threadIdx.x + i * kAttnThreads, r = idx >> 3;
      *reinterpret_cast<uint4*>(sQ + r * 128 + (((idx & 7) ^ (r & 7)) << 4)) = x[i];
    }
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    if (lane == 0) top[warp] = most;
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *(volatile uint32_t*)&B->tmem_base;

  if (warp >= 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsOther));
    if (warp == 4) {
      // ------------------------------------------------ TMA producer
      if (lane == 0) {
        int issued_k = min(n_tiles, 1), issued_v = issued_k;                    // (the first tile's are under way)
        bool ok = true;
        for (int it = 1; it < n_tiles && ok; ++it) {
          const int s = it % kKVStages, row = plane_row + it * kBN;
          const uint32_t ph = (uint32_t)(it / kKVStages - 1) & 1u;
          if (it >= kKVStages) ok = mbar_wait(&B->k_empty[s], ph, B, P.status);
          if (!ok) break;
          mbar_expect_tx(&B->k_full[s], kTileBytes);
          tma_load_2d(sK + s * kTileBytes, &tm_k, hk * kHD, row, &B->k_full[s]);
          ++issued_k;
          if (it >= kKVStages) ok = mbar_wait(&B->v_empty[s], ph, B, P.status);
          if (!ok) break;
          mbar_expect_tx(&B->v_full[s], kTileBytes);
          tma_load_2d(sV + s * kTileBytes, &tm_v, hk * kHD, row, &B->v_full[s]);
          ++issued_v;
        }
        if (!ok) {
          // leave no bulk copy in flight into this CTA's shared memory
          for (int i = max(0, issued_k - kKVStages); i < issued_k; ++i)
            mbar_wait(&B->k_full[i % kKVStages], (uint32_t)(i / kKVStages) & 1u, B, P.status);
          for (int i = max(0, issued_v - kKVStages); i < issued_v; ++i)
            mbar_wait(&B->v_full[i % kKVStages], (uint32_t)(i / kKVStages) & 1u, B, P.status);
        }
      }
      __syncwarp();
    } else if (warp == 5 && n_tiles > 0) {
      // ------------------------------------------------ MMA issuer, in the bf16 attention's order:
      // QK(0,0) QK(0,1) | PV(0,0) QK(1,0) PV(0,1) QK(1,1) | PV(1,0) QK(2,0) ...
      const bool leader = elect_one();
      const uint32_t tm = __reduce_or_sync(0xFFFFFFFFu, tmem);
      constexpr uint32_t idesc_qk = idesc_bf16(kHalf, false), idesc_pv = idesc_bf16(kHD, true);
      const uint64_t dq = smem_desc_sw128(smem_u32(sQ));
      auto wait_all = [&](void* bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, mbar_wait(bar, parity, B, P.status)) != 0; };
      auto issue_qk = [&](int st, int hf) {
        const uint64_t dk = smem_desc_sw128(smem_u32(sK + st * kTileBytes + hf * (kTileBytes / 2)));
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < kHD / 16; ++kk) mma_ss(tm + kColS + hf * kHalf, dq + (uint64_t)(kk * 2), dk + (uint64_t)(kk * 2), idesc_qk, kk > 0);
          tc_commit(&B->s_full[hf]);
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
          ok = wait_all(&B->p_full[hf], (uint32_t)it & 1u);
          if (!ok) break;
          tc_fence_after();
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < kHalf / 16; ++kk)
              mma_ts(tm + kColO, tm + kColS + hf * kHalf + kk * 8, dv + (uint64_t)((hf * (kHalf / 16) + kk) * 128), idesc_pv, (it > 0 || hf > 0 || kk > 0));
            if (hf == 1) tc_commit(&B->v_empty[s]);
            if (!more && hf == 0) tc_commit(&B->pv_done);    // (the last half has no later score MMA to tell it by)
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
        if (leader) tc_commit(&B->o_full);
        wait_all(&B->o_full, 0);
      } else {
        if (leader) tc_commit(&B->drain);                // let every issued MMA finish before TMEM is freed
        wait_all(&B->drain, 0);
      }
      __syncwarp();
    }
  } else {
    // ------------------------------------------------ softmax and epilogue, one thread a row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    const int row = warp * 32 + lane;
    const uint32_t t_row = tmem + ((uint32_t)(warp * 32) << 16);
    const float c = 1.4426950408889634f * 0.125f;        // log2(e) / sqrt(64)
    float m = -INFINITY, l = 0.0f;
    bool ok = true;
    // Upper bound of this row's logits in log2 units, |q| |k|_max log2(e) / 8, for the fixed reference (see attn_tcgen05.cuh).
    float bound;
    bool fixed_ref = false, in_range = false, odd;       // odd: a query that is not finite, whose result is NaN anyhow; it does not decide for its warp
    {
      const float kmax2 = __uint_as_float(max(max(max(top[0], top[1]), max(top[2], top[3])), max(max(top[4], top[5]), max(top[6], top[7]))));
      float qn2 = 0.0f, zero = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint4 u = *reinterpret_cast<const uint4*>(sQ + row * 128 + ((j ^ (row & 7)) << 4));
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float lo = __uint_as_float(w[e] << 16), hi = __uint_as_float(w[e] & 0xFFFF0000u);
          qn2 = fmaf(lo, lo, qn2);
          qn2 = fmaf(hi, hi, qn2);
          zero = fmaf(lo, 0.0f, fmaf(hi, 0.0f, zero));
        }
      }
      bound = sqrtf(qn2 * kmax2) * c;
      odd = !(zero == 0.0f);
    }
    int idx = 0, left = min(len - t_begin * kBN, n_tiles * kBN);   // idx = 2 * tile + half; live rows from there on
    for (; ok && ((idx & 1) != 0 || left > 0); ++idx, left -= kHalf) {
      const int it = idx >> 1, hf = idx & 1;
      // (every wait result is made warp-uniform before the warp meets an .aligned tensor-memory instruction)
      ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->s_full[hf], (uint32_t)it & 1u, B, P.status)) != 0;
      if (!ok) break;
      tc_fence_after();
      uint32_t s[kHalf];
      auto load_scores = [&]() {
#pragma unroll
        for (int j = 0; j < kHalf / 32; ++j) tmem_ld32(t_row + kColS + hf * kHalf + j * 32, s + j * 32);
        tmem_wait_ld();
        if (left < kHalf) {
#pragma unroll
          for (int j = 0; j < kHalf; ++j)
            if (j >= left) s[j] = 0xFF800000u;           // -inf on columns past the last row
        }
      };
      // p = 2^(s c - reference) on pairs, packed to bf16 over the front of s[]; returns the row's sum of p and its largest raw score
      auto exp_pass = [&](auto track, auto clamp, float& raw) -> float {
        const float2 c2 = make_float2(c, c), nm2 = make_float2(-m, -m);
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
          const float2 p = pair_on_fma_pipes(j >> 1) ? ex2_poly2<decltype(clamp)::value>(x) : make_float2(ex2(x.x), ex2(x.y));
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
        constexpr int kChain = kHalf / 4;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          m4[q] = fmaxf(__uint_as_float(s[kChain * q]), __uint_as_float(s[kChain * q + 1]));
#pragma unroll
          for (int j = 2; j < kChain; j += 2) m4[q] = max3(m4[q], __uint_as_float(s[kChain * q + j]), __uint_as_float(s[kChain * q + j + 1]));
        }
        m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * c;
        // the bound as the reference, a whole number of powers of two above what was seen, where it is not absurdly far above
        fixed_ref = __all_sync(0xFFFFFFFFu, odd || (bound >= m && bound - m <= kFixedRefMaxGap)) != 0;
        if (fixed_ref && !odd) m += ceilf(bound - m);
        in_range = fixed_ref && __all_sync(0xFFFFFFFFu, odd || bound + m <= -1.0f - kPolyLowest) != 0;
        add = exp_pass(std::false_type{}, std::true_type{}, raw);
      } else if (fixed_ref) {
        add = in_range && left >= kHalf ? exp_pass(std::false_type{}, std::false_type{}, raw) : exp_pass(std::false_type{}, std::true_type{}, raw);
      } else {
        add = exp_pass(std::true_type{}, std::true_type{}, raw);
        const float mx = raw * c;
        const bool grow = mx - m > kRescaleThreshold;
        if (__any_sync(0xFFFFFFFFu, grow)) {
          // O may still be accumulating the half before: the scores of the next half, issued behind it, tell; or the last one's own barrier
          ok = hf == 0 || left > kHalf ? mbar_wait(&B->s_full[hf ^ 1], (uint32_t)((idx + 1) >> 1) & 1u, B, P.status)
                                     : mbar_wait(&B->pv_done, 0, B, P.status);
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
          add = exp_pass(std::false_type{}, std::true_type{}, raw);
        }
      }
      l += add;
      tmem_st32(t_row + kColS + hf * kHalf, s);
      tmem_st16(t_row + kColS + hf * kHalf + 32, s + 32);
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(&B->p_full[hf]);
    }
    const bool seen = idx > 0;
    if (seen && ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&B->o_full, 0, B, P.status)) != 0;
    if (ok) {
      tc_fence_after();
      // (a tile's first half has a live row: a maximum of -inf is one of scores that are not numbers, and an infinite one makes NaN too)
      if (seen && fabsf(m) == INFINITY) l = __int_as_float(0x7FC00000);
      const bool one = P.parts == 1;
      const float inv = !seen ? 0.0f : (one ? 1.0f / l : 1.0f);
      // By way of the operand tiles, which are free now: a thread has a row, but a warp stores whole lines of it.
      unsigned char* stage = sK + warp * 32 * kOutRow;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t o[32];
        if (seen) {
          tmem_ld32(t_row + kColO + j * 32, o);
          tmem_wait_ld();
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = seen ? __float_as_uint(__uint_as_float(o[e]) * inv) : 0u;
        uint4* dst = reinterpret_cast<uint4*>(stage + lane * kOutRow);
        if (one) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float* f = reinterpret_cast<const float*>(o) + 8 * e;
            dst[4 * j + e] = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
          }
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) dst[8 * j + e] = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        }
      }
      __syncwarp();
      unsigned block = blockIdx.x;
      asm volatile("" : "+r"(block));                    // (taken apart again: nothing of it is kept through the loop)
      const Place at1(P, block);
      // (a lane's row of the result, in rows of a head; -1 past the last)
      const int mine = at1.row0 + row < P.M * P.group ? (int)(at1.q(P, at1.row0 + row) / kHD) : -1;
      const size_t shift = (size_t)at1.part * P.seqs * P.M * P.H;
      auto store = [&](auto lanes, unsigned char* to) {  // lanes: 16-byte words of a row
        constexpr int kLanes = decltype(lanes)::value;
        const int sub = lane % kLanes, r0 = lane / kLanes;
        const unsigned char* from = stage + r0 * kOutRow + sub * 16;
#pragma unroll
        for (int i = 0; i < kLanes; i += 8) {
          uint4 w[8];
          int at[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            w[e] = *reinterpret_cast<const uint4*>(from + (i + e) * (32 / kLanes) * kOutRow);
            at[e] = __shfl_sync(0xFFFFFFFFu, mine, r0 + (i + e) * (32 / kLanes));
          }
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (at[e] >= 0) *reinterpret_cast<uint4*>(to + (size_t)at[e] * (kLanes * 16) + sub * 16) = w[e];
        }
      };
      if (one) {
        store(std::integral_constant<int, 8>{}, reinterpret_cast<unsigned char*>(P.out));
      } else {
        store(std::integral_constant<int, 16>{}, reinterpret_cast<unsigned char*>(P.o_part + shift * kHD));
        if (mine >= 0) P.ml_part[shift + mine] = seen ? make_float2(fmaxf(m, kDeadMax), l) : make_float2(kDeadMax, kDeadSum);
      }
    }
  }

  // ------------------------------------------------ teardown
  tc_fence_before();
  __syncthreads();
  if (warp == 5) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kTmemCols) : "memory");
  }
}

// ---------------------------------------------------------------- host side

// Whether a call goes by way of planes, from its time in picoseconds: streaming the cache costs 5 us and 45 ps a cached row, head and 32
// rows of queries; the planes 11 us, 118 ps a cached row and head, and 25 ps more for each 128 rows of queries after the first.  Fitted to 96 to
// 512 rows over 512 to 32768 of 16 heads, with queries of 15 bits where they stream.  Now 64 x 8192 21.3 us against 26.5, 96 x 8192 26.8 against 26.7, 128 x 8192
// 34.0 against 27.1, 256 x 2048 19.2 against 20.0, 256 x 8192 55.7 against 30.9, 512 x 2048 32.2 against 21.9.
inline bool attn_q8_by_planes(long long cached, long long rows) {      // cached rows times heads, over all sequences
  const double x = (double)cached;
  return 5e6 + 45.0 * x * (double)((rows + 31) / 32) > 11e6 + x * (118.0 + 25.0 * (double)((rows - 1) / kBM));
}

// How a call is cut: rows a CTA takes (8, 16, 32: the few-row kernel, by so many warps; 128), parts of the cached rows, sequences at once.
struct AttnQ8Plan {
  int tile, warps, q_tiles, parts, seqs, plane_rows;
  size_t planes, o_part, ml_part, bytes;   // of scratch: K and V planes, the parts' results, where the live rows go and the norms; all
};
inline AttnQ8Plan attn_q8_plan(int seqs, int M, int H, int HK, int cap) {
  AttnQ8Plan A = {};
  const long long rows = (long long)M * (H / HK);
  A.plane_rows = (cap + kBN - 1) / kBN * kBN;
  const size_t one = (size_t)A.plane_rows * HK * kHD * 4;
  if (one <= kPlanesMost && attn_q8_by_planes((long long)seqs * HK * cap, rows)) {
    A.tile = kBM;
    A.seqs = (int)std::max<size_t>(1, std::min<size_t>(seqs, kPlanesAtOnce / one));
    A.planes = one * A.seqs;
    A.q_tiles = (int)((rows + kBM - 1) / kBM);
    // waves of CTAs over 2 x 148 places, each as long as its tiles and two more (set-up, epilogue), a merge one tile more
    const int tiles = A.plane_rows / kBN;
    const long long jobs = (long long)A.seqs * HK * A.q_tiles;
    long long best = -1;
    for (int s = 1; s <= kMaxSplits && s <= tiles; ++s) {
      const long long cost = (jobs * s + 295) / 296 * ((tiles + s - 1) / s + 2) + (s > 1 ? 1 : 0);
      if (best < 0 || cost < best) best = cost, A.parts = s;
    }
  } else {
    A.tile = rows <= 8 ? 8 : (rows <= 16 ? 16 : 32);
    A.seqs = seqs;
    A.q_tiles = (int)((rows + A.tile - 1) / A.tile);
    // Warps a CTA and parts, by a model of the time in 10 ns: waves of CTAs over 148 SMs, each as long as a warp's tiles of 32 cached rows (a last
    // one shorter, which has the SMs to itself) and its set-up and end, which smaller CTAs hide under one another's work, and a merge.  Fitted to 16 to 1024 sequences times heads over 256 to 32768 rows: 16 x
    // 32768 by 12 warps 20 us, by 6 21, by 4 27; 80 x 8192 21, 21 and 19; 256 x 2048 21, 17.6 and 20; 1024 x 2048 71, 59 and 54.  (480 x 8192
    // takes 99 us as chosen, 84 by 4: the constants are those of queries of 15 bits, whose tiles took a tenth less.)
    const long long jobs = (long long)seqs * HK * A.q_tiles, tiles = (cap + kFewKeys - 1) / kFewKeys;
    const int whole = few_warps(A.tile), step = A.tile == 8 ? 115 : (A.tile == 16 ? 168 : 157);
    long long best = -1;
    for (int per_sm = 1; per_sm <= (whole == 12 ? 3 : 2); ++per_sm)
      for (int parts = 1; parts <= kMaxSplits; ++parts) {
        const int warps = whole / per_sm, ends = per_sm == 1 ? 230 : (per_sm == 2 ? 130 : 90);
        if (parts > 1 && (long long)(parts - 1) * warps >= tiles) break;       // (each part's first warp has a tile)
        const long long places = 148 * per_sm, full = jobs * parts / places, rest = jobs * parts % places;
        const long long a_warp = (tiles + (long long)parts * warps - 1) / ((long long)parts * warps) * step;
        const long long cost = full * (a_warp + ends) + (rest ? a_warp * std::max(places * (full ? 45 : 90) / 100, rest) / places + ends : 0) + (parts > 1 ? 200 + 20 * parts : 0);
        if (best < 0 || cost < best) best = cost, A.parts = parts, A.warps = warps;
      }
  }
  A.o_part = A.parts == 1 ? 0 : (size_t)A.parts * A.seqs * M * H * kHD * 4;
  A.ml_part = A.parts == 1 ? 0 : (size_t)A.parts * A.seqs * M * H * 8;
  A.bytes = A.planes + A.o_part + A.ml_part + (A.planes ? (size_t)A.seqs * (A.plane_rows / kWidenRows * (1 + HK) + 1) * 4 : 0);
  return A;
}

static inline int attn_q8_launch(AttnQ8Args P, void* scratch, cudaStream_t st, int* launches) {
  const AttnQ8Plan A = attn_q8_plan(P.seqs, P.M, P.H, P.HK, P.cap);
  const int all = P.seqs;
  P.q_tiles = A.q_tiles;
  P.parts = A.parts;
  P.o_part = reinterpret_cast<float*>(static_cast<char*>(scratch) + A.planes);
  P.ml_part = reinterpret_cast<float2*>(static_cast<char*>(scratch) + A.planes + A.o_part);
  const size_t q_seq = (size_t)P.M * P.H * kHD, rows_seq = (size_t)P.cap * P.HK * kHD, x_seq = (size_t)P.HK * P.cap;
  *launches = 0;
  for (int s0 = 0; s0 < all; s0 += A.seqs) {
    P.seqs = std::min(A.seqs, all - s0);
    const long long ctas = (long long)P.seqs * P.HK * P.q_tiles * P.parts;
    if (ctas > 0x7FFFFFFF) return OVGGT_ERR_UNSUPPORTED;
    cudaError_t e;
    if (A.tile == kBM) {
      char* planes = static_cast<char*>(scratch);
      const size_t side = A.planes / 2;
      const int blocks = A.plane_rows / kWidenRows;
      int* first = reinterpret_cast<int*>(planes + A.planes + A.o_part + A.ml_part);
      int* counts = P.live ? first + (size_t)A.seqs * blocks : nullptr;
      unsigned* norms = reinterpret_cast<unsigned*>(first + (size_t)A.seqs * (blocks + 1));
      const WidenArgs W = {reinterpret_cast<const uint4*>(P.kq), reinterpret_cast<const uint4*>(P.vq), P.kx, P.vx, P.lens, P.live, first, counts,
                           reinterpret_cast<uint4*>(planes), reinterpret_cast<uint4*>(planes + side), norms, P.cap, P.HK, A.plane_rows};
      CUtensorMap tk, tv;
      int rc = make_rows_map(&tk, planes, P.seqs * A.plane_rows, P.HK * kHD, kBN);
      if (rc) return rc;
      rc = make_rows_map(&tv, planes + side, P.seqs * A.plane_rows, P.HK * kHD, kBN);
      if (rc) return rc;
      e = cudaSuccess;
      if (P.live) {
        e = launch_dependent(k_live_rows, dim3(P.seqs), 1024, 1, 0, st, true, LiveArgs{P.lens, P.live, first, counts, P.cap, blocks});
        *launches += 1;
      }
      if (e == cudaSuccess) e = launch_dependent(k_widen_q8, dim3(blocks, P.seqs, (P.HK + kWidenHeads - 1) / kWidenHeads * 2), 256, 1, 0, st, true, W);
      static std::atomic<uint64_t> smem_many;
      if (e == cudaSuccess) e = allow_smem(k_attn_q8_many, kManySmem, smem_many);
      if (e == cudaSuccess) e = launch_dependent(k_attn_q8_many, dim3((unsigned)ctas), kAttnThreads, 1, kManySmem, st, true, tk, tv, P, (const int*)counts, (const unsigned*)norms, A.plane_rows);
      *launches += 2;
    } else {
      const auto launch = [&](auto kernel, std::atomic<uint64_t>& smem_set) {
        const int smem = few_smem_bytes(A.warps);
        const cudaError_t set = allow_smem(kernel, smem, smem_set);
        return set != cudaSuccess ? set : launch_dependent(kernel, dim3((unsigned)ctas), A.warps * 32, 1, smem, st, true, P);
      };
      static std::atomic<uint64_t> smem_few[8];
      if (A.tile == 8) e = A.warps == 12 ? launch(k_attn_q8_few<8, 12>, smem_few[0]) : (A.warps == 6 ? launch(k_attn_q8_few<8, 6>, smem_few[1]) : launch(k_attn_q8_few<8, 4>, smem_few[2]));
      else if (A.tile == 16) e = A.warps == 12 ? launch(k_attn_q8_few<16, 12>, smem_few[3]) : (A.warps == 6 ? launch(k_attn_q8_few<16, 6>, smem_few[4]) : launch(k_attn_q8_few<16, 4>, smem_few[5]));
      else e = A.warps == 8 ? launch(k_attn_q8_few<32, 8>, smem_few[6]) : launch(k_attn_q8_few<32, 4>, smem_few[7]);
      *launches += 1;
    }
    if (e != cudaSuccess) { g_attn_last_error = (int)e; return OVGGT_ERR_CUDA; }
    if (P.parts > 1) {
      const int rc = attn_merge_launch<__nv_bfloat16>(P.o_part, P.ml_part, P.seqs * P.M, P.H, P.parts, P.out, nullptr, st);
      if (rc) return rc;
      *launches += 1;
    }
    P.q += A.seqs * q_seq;
    P.out += A.seqs * q_seq;
    P.kq += A.seqs * rows_seq;
    P.vq += A.seqs * rows_seq;
    P.kx += A.seqs * x_seq;
    P.vx += A.seqs * x_seq;
    if (P.lens) P.lens += A.seqs;
    if (P.live) P.live += (size_t)A.seqs * P.cap;
  }
  return OVGGT_OK;
}

}  // namespace ovggt
