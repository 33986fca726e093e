// Rows in 8 bits: quantising rows behind a residual sum and a norm, and keys and values into and out of an 8-bit cache.
#pragma once

#include "attn_tcgen05.cuh"

namespace ovggt {

// Four floats, whole numbers of at most 127 in size after rounding, as int8 (round to nearest, ties to even): adding 1.5 * 2^23
// leaves the whole number's two's complement in the low byte.
__device__ __forceinline__ uint32_t pack_int8(float a, float b, float c, float d) {
  const float magic = 12582912.0f;
  const uint32_t x = __float_as_uint(a + magic), y = __float_as_uint(b + magic), z = __float_as_uint(c + magic), w = __float_as_uint(d + magic);
  return __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
}

// ---------------------------------------------------------------- rows to int8 with a scale each

// One row is h = x + residual (rounded to the rows' type and stored), y = its norm, scale = max |y| / 127, q = round(y / scale).
// The row stays in registers between its three reductions (mean, squares, maximum), so x and the residual are read once.
struct NormQ8Args {
  const uint4 *x, *residual, *weight, *bias;   // rows of C elements; residual, weight, bias may be nullptr
  uint4* sum;                                  // h, or nullptr
  uint2* q;
  float* scale;
  int rows, C, kind;
  float eps;
};

template <int DT>
__device__ __forceinline__ void load8(const uint4* p, size_t unit, float* f) {   // eight elements
  if constexpr (DT == kBF16) {
    unpack<DT>(p[unit], f);
  } else {
    unpack<DT>(p[2 * unit], f);
    unpack<DT>(p[2 * unit + 1], f + 4);
  }
}

// A value over the THREADS threads that hold a row: a butterfly, then the warps' results in order.
template <int THREADS, typename Op>
__device__ __forceinline__ float row_reduce(float x, float* sh, Op op) {
#pragma unroll
  for (int o = (THREADS < 32 ? THREADS : 32) / 2; o > 0; o >>= 1) x = op(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  if constexpr (THREADS > 32) {
    __syncthreads();                                     // (the scratch of the reduction before has been read)
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    x = sh[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) x = op(x, sh[w]);
  }
  return x;
}

// Four groups of eight elements a thread, whatever the row's width: 8 to 512 threads a row, several rows a CTA where they are less than
// 128.  All loads, the weight's among them, are requested before the first reduction.  What bounds it is memory (10992 x 1024 bf16 with a
// residual: 79 MB in 15.8 us, 5.0 TB/s; 12.9 where they still are in L2), of a single row the trip to it: with one to four groups a thread, a warp up to 1024 columns and a CTA beyond, and weights
// read where they are needed, 60000 x 256 took 23.6 us instead of 18.1, 4000 x 8192 59 instead of 40 and one row of 1024 3.5 instead of 2.4.
// PLAIN: neither a residual nor a norm, in instances with registers for no more (10992 x 4096: 25.2 us, without them 29.8).
constexpr int kNormUnits = 4;
__host__ __device__ constexpr int norm_cta(int threads) { return threads < 128 ? (threads == 64 ? 64 : 128) : threads; }
template <int DT, int THREADS, bool PLAIN>
__global__ void __launch_bounds__(norm_cta(THREADS)) k_norm_q8(const NormQ8Args P) {
  __shared__ float sh[16];
  constexpr int U = kNormUnits, kWords = DT == kBF16 ? 1 : 2;                 // 16-byte words of a group
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x % THREADS;
  const long long row = (long long)blockIdx.x * (norm_cta(THREADS) / THREADS) + threadIdx.x / THREADS;
  const bool in = THREADS > 32 || row < P.rows;          // (a warp's rows go through its shuffles together)
  const int units = P.C / 8;
  const size_t u0 = (size_t)row * units;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  constexpr int V = PLAIN ? 1 : U;
  uint4 x[U][kWords], r[V][kWords], w[V][kWords];
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
      const int u = tid + i * THREADS;
      const bool here = in && u < units;
      x[i][j] = here ? P.x[(u0 + u) * kWords + j] : zero;
      if constexpr (!PLAIN) {
        r[i][j] = here && P.residual != nullptr ? P.residual[(u0 + u) * kWords + j] : zero;
        w[i][j] = u < units && P.weight != nullptr ? P.weight[(size_t)u * kWords + j] : zero;
      }
    }
  auto eight = [](const uint4 (&v)[kWords], float* f) {
    unpack<DT>(v[0], f);
    if constexpr (DT != kBF16) unpack<DT>(v[kWords - 1], f + 4);
  };
  float y[U][8];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    eight(x[i], y[i]);
    if (!PLAIN && P.residual != nullptr) {
      float b[8];
      eight(r[PLAIN ? 0 : i], b);
      uint4 s[kWords];
      if constexpr (DT == kBF16) {
        uint32_t* o = reinterpret_cast<uint32_t*>(s);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = pack_bf16(y[i][2 * e] + b[2 * e], y[i][2 * e + 1] + b[2 * e + 1]);
      } else {
        float* o = reinterpret_cast<float*>(s);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = y[i][e] + b[e];
      }
      eight(s, y[i]);                                    // (the norm is that of the stored sum)
      const int u = tid + i * THREADS;
      if (P.sum != nullptr && in && u < units) {
#pragma unroll
        for (int j = 0; j < kWords; ++j) P.sum[(u0 + u) * kWords + j] = s[j];
      }
    }
  }
  const auto add = [](float a, float b) { return a + b; };
  if (!PLAIN && P.kind != OVGGT_NORM_NONE) {
    float eps = P.eps;
    const auto sum = [&]() {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s += y[i][e];
      return row_reduce<THREADS>(s, sh, add);
    };
    const auto squares = [&]() {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(y[i][e], y[i][e], s);
      return row_reduce<THREADS>(s, sh, add);
    };
    // A row whose sum or squares leave fp32's range is taken times a power of two, and eps with it.  (The norm does not change; a row's threads all
    // have its sums, a warp's rows go through the shuffles together.)
    const auto rescale = [&](float by) {
      if (THREADS <= 32 ? __all_sync(0xFFFFFFFFu, by == 1.0f) != 0 : by == 1.0f) return false;
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) y[i][e] *= by;
      eps = eps * by * by;
      return true;
    };
    constexpr float kDown = 8.271806125530277e-25f, kUp = 1.2676506002282294e30f;        // 2^-80, 2^100
    if (P.kind == OVGGT_NORM_LAYER) {
      float s = sum();
      if (rescale(fabsf(s) < INFINITY ? 1.0f : kDown)) s = sum();
      const float mean = s / (float)P.C;
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (tid + i * THREADS < units) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[i][e] -= mean;
        }
    }
    float s = squares();
    // (below 2^-90 and above 2^-80: what s lacks does not show beside eps)
    if (rescale(!(s < INFINITY) ? kDown : (s < 8.077935669463161e-28f && eps < 8.271806125530277e-25f ? kUp : 1.0f))) s = squares();
    const float rstd = 1.0f / sqrtf(s / (float)P.C + eps);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = tid + i * THREADS;
      float g[8];
      eight(w[PLAIN ? 0 : i], g);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[i][e] *= P.weight != nullptr ? rstd * g[e] : rstd;
      if (P.bias != nullptr && u < units) {
        load8<DT>(P.bias, u, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[i][e] += g[e];
      }
    }
  }
  // The maximum of the magnitudes' bits, which order as the magnitudes do, infinities and NaN on top.
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < U; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(y[i][e]) & 0x7FFFFFFFu);
  most = __float_as_uint(row_reduce<THREADS>(__uint_as_float(most), sh, [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }));
  // A row with a value that is not finite gets a scale that is not a number, and products of it are none; a row of
  // nothing but (almost) zeros a scale of 0: down to 2^-119 maximum / 127 is a normal number, and 127 / maximum one of fp32's.
  const float amax = __uint_as_float(most);
  const bool finite = most < 0x7F800000u, some = finite && amax >= 1.504632769052528e-36f;
  const float inv = some ? 127.0f / amax : 0.0f;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int u = tid + i * THREADS;
    if (in && u < units) {
      float z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = some ? fminf(fmaxf(y[i][e] * inv, -127.0f), 127.0f) : 0.0f;
      P.q[u0 + u] = make_uint2(pack_int8(z[0], z[1], z[2], z[3]), pack_int8(z[4], z[5], z[6], z[7]));
    }
  }
  if (tid == 0 && in) P.scale[row] = some ? amax / 127.0f : (finite ? 0.0f : __int_as_float(0x7FC00000));
}

constexpr int kNormMaxC = 512 * kNormUnits * 8;

template <int DT>
static inline cudaError_t norm_q8_launch(const NormQ8Args& P, cudaStream_t st) {
  const int threads = (P.C / 8 + kNormUnits - 1) / kNormUnits;
  const bool plain = P.kind == OVGGT_NORM_NONE && P.residual == nullptr;
  const auto launch = [&](auto t) {
    constexpr int T = decltype(t)::value, kRows = norm_cta(T) / T;
    return launch_dependent(plain ? k_norm_q8<DT, T, true> : k_norm_q8<DT, T, false>, dim3((P.rows + kRows - 1) / kRows), norm_cta(T), 1, 0, st, true, P);
  };
  if (threads <= 8) return launch(std::integral_constant<int, 8>{});
  if (threads <= 16) return launch(std::integral_constant<int, 16>{});
  if (threads <= 32) return launch(std::integral_constant<int, 32>{});
  if (threads <= 64) return launch(std::integral_constant<int, 64>{});
  if (threads <= 128) return launch(std::integral_constant<int, 128>{});
  if (threads <= 256) return launch(std::integral_constant<int, 256>{});
  return launch(std::integral_constant<int, 512>{});
}

// ---------------------------------------------------------------- an 8-bit cache: rows in, rows out

// A block is the 64 columns of one row and head.  With 2^e the largest power of two that its largest magnitude reaches (e at least
// -120, whose step 2^(6 - e) is the last that fp32 holds), the cache has q = round(x 2^(6 - e)), at most 127 in size, and the byte e + 127.  The
// values q 2^(e - 6) are exact in bf16, so reading back rounds nothing and writing back what was read gives the same
// bytes.  A block that is not finite is the byte 255, and reads as NaN.
constexpr int kQ8Lowest = -120;

struct StoreQ8Args {
  const uint4* src[2];                 // keys, values [seqs, M, C]
  uint2* q[2];                         // int8 [seqs, cap, C]
  uint8_t* x[2];                       // [seqs, H, cap]
  const int* start;                    // [seqs] or nullptr
  int seqs, M, H, cap;
};

// Eight lanes a block, eight elements each.
template <int DT>
__global__ void __launch_bounds__(256) k_store_q8(const StoreQ8Args P) {
  pdl_trigger();
  pdl_wait();
  const long long at = (long long)blockIdx.x * 256 + threadIdx.x, unit = at >> 3, per_row = P.H;
  const long long row = unit / per_row;
  const int h = (int)(unit - row * per_row), part = (int)(at & 7), side = blockIdx.y;
  const bool in = row < (long long)P.seqs * P.M;
  const int seq = in ? (int)(row / P.M) : 0, j = in ? (int)(row - (long long)seq * P.M) : 0;
  const long long to = in ? (P.start != nullptr ? (long long)P.start[seq] : 0) + j : -1;
  const bool keep = in && (P.start == nullptr || P.start[seq] >= 0) && to < P.cap;
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = 0.0f;
  if (keep) load8<DT>((side == 0 ? P.src[0] : P.src[1]), (size_t)at, f);
  uint32_t most = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(f[e]) & 0x7FFFFFFFu);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
  if (!keep) return;
  const bool finite = most < 0x7F800000u;
  const int e = max((int)(most >> 23) - 127, kQ8Lowest);
  const float step = __int_as_float((6 - e + 127) << 23);
  float z[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) z[i] = finite ? fminf(fmaxf(f[i] * step, -127.0f), 127.0f) : 0.0f;
  (side == 0 ? P.q[0] : P.q[1])[(((size_t)seq * P.cap + to) * P.H + h) * 8 + part] = make_uint2(pack_int8(z[0], z[1], z[2], z[3]), pack_int8(z[4], z[5], z[6], z[7]));
  if (part == 0) (side == 0 ? P.x[0] : P.x[1])[((size_t)seq * P.H + h) * P.cap + to] = finite ? (uint8_t)(e + 127) : (uint8_t)255;
}

struct LoadQ8Args {
  const void* q[2];
  const uint8_t* x[2];
  void* dst[2];                        // [seqs, n, C]
  int first, n, H, cap;
};

// 2^(x - 133), the step of a block whose exponent byte is x; NaN for 255.
__device__ __forceinline__ float q8_step(uint32_t x) { return x == 255u ? __int_as_float(0x7FC00000) : __int_as_float((int)(max(x, 6u) - 6u) << 23); }
// Byte i of a word of int8 as fp32, exact.
template <int I>
__device__ __forceinline__ float int8_at(uint32_t flipped) {   // (flipped: the word ^ 0x80808080)
  return __uint_as_float(__byte_perm(flipped, 0x4B000000u, 0x7440 + I)) - 8388736.0f;
}

// Bound by memory.  Whole lines both ways: four groups of 16 bytes of output a thread, a CTA's width apart; stores that leave L2 first, since what
// is read back is as a rule larger than it.  17758 rows of 16 heads: bf16 23 us (4.7 TB/s), fp32 37.8 (4.8).  With the cache in L2 17.6 and 30.4; so measured
// with ordinary stores 20.8 and 36.4, with 16 elements a thread side by side 19.8 and 41.7, with eight groups a thread 21.3 and 31.0.
constexpr int kLoadGroups = 4;
template <int DT>
__global__ void __launch_bounds__(256) k_load_q8(const LoadQ8Args P) {
  constexpr int E = VecOf<DT>::n, kWords = E / 4;        // elements of a group, its words of int8
  pdl_trigger();
  pdl_wait();
  const int seq = blockIdx.y, side = blockIdx.z;
  const unsigned per_row = (unsigned)P.H * (64 / E), all = (unsigned)P.n * per_row, g0 = blockIdx.x * (256u * kLoadGroups) + threadIdx.x;
  const uint32_t* q = reinterpret_cast<const uint32_t*>(side == 0 ? P.q[0] : P.q[1]) + ((size_t)seq * P.cap + P.first) * P.H * 16;
  const uint8_t* xs = (side == 0 ? P.x[0] : P.x[1]) + (size_t)seq * P.H * P.cap + P.first;
  uint4* d = static_cast<uint4*>(side == 0 ? P.dst[0] : P.dst[1]) + (size_t)seq * all;
  uint32_t w[kLoadGroups][kWords], x[kLoadGroups];
#pragma unroll
  for (int j = 0; j < kLoadGroups; ++j) {
    const unsigned g = g0 + 256u * j;
    if (g < all) {
      if constexpr (kWords == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(q + (size_t)g * 2);
        w[j][0] = v.x, w[j][kWords - 1] = v.y;
      } else {
        w[j][0] = q[g];
      }
      const unsigned row = g / per_row;
      x[j] = xs[(size_t)((g - row * per_row) / (64 / E)) * P.cap + row];
    }
  }
#pragma unroll
  for (int j = 0; j < kLoadGroups; ++j) {
    const unsigned g = g0 + 256u * j;
    if (g < all) {
      const float step = q8_step(x[j]);
      float f[E];
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const uint32_t u = w[j][i] ^ 0x80808080u;
        f[4 * i] = int8_at<0>(u) * step;
        f[4 * i + 1] = int8_at<1>(u) * step;
        f[4 * i + 2] = int8_at<2>(u) * step;
        f[4 * i + 3] = int8_at<3>(u) * step;
      }
      if constexpr (DT == kBF16) {
        __stcs(d + g, make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[E - 4], f[E - 3]), pack_bf16(f[E - 2], f[E - 1])));
      } else {
        __stcs(d + g, make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])));
      }
    }
  }
}

}  // namespace ovggt
