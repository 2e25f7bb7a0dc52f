// Codes of 8-bit floating point with a power of two per block of 128 (sr_quantize_f8), of a matrix and of its
// transpose in one pass.
//
// A workgroup takes a tile of 128 x 128: thread (g, l) holds rows 8 g .. 8 g + 7, channels 8 l .. 8 l + 7.  A row's
// block is then 16 neighbouring lanes, a column's the 16 values of g, and eight codes of a column are eight consecutive
// bytes of the transpose, which leaves through LDS in whole rows.  Bound by memory.
#include "block_ops.h"

namespace sr {

namespace {

constexpr int kPitch = 136;   // bytes of a row of the transposed tile in LDS

struct QuantF8 {
  int M, N;
  const void* x;
  int64_t ldx;
  uint8_t *q, *e, *qt, *et;
};

SR_DEV uint32_t dpp_max16(uint32_t m) {   // over 16 neighbouring lanes
  auto over = [&](auto ctl) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, decltype(ctl)::value, 0xF, 0xF, false));
  };
  over(IC<0xB1>{});
  over(IC<0x4E>{});
  over(IC<0x141>{});
  over(IC<0x140>{});
  return m;
}

template <typename T, bool TILE>
__global__ __launch_bounds__(256) void quantize_f8_kernel(QuantF8 a, int vec) {
  __shared__ __attribute__((aligned(16))) uint8_t tr[128 * kPitch];
  __shared__ uint32_t top[4][128];
  __shared__ __attribute__((aligned(16))) uint8_t ex[128];
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4, wave = wave_index();
  const int tiles_n = (a.N + 127) / 128, tm = (int)(blockIdx.x / (unsigned)tiles_n), tn = (int)(blockIdx.x - (unsigned)tm * (unsigned)tiles_n);
  const int m0 = tm * 128, n0 = tn * 128, n = n0 + 8 * l;
  const int64_t Np = (int64_t)tiles_n * 128, Mp = (int64_t)(a.M + 127) / 128 * 128;
  const int64_t Mr = (int64_t)(a.M + 15) / 16 * 16, Nr = (int64_t)(a.N + 15) / 16 * 16;

  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int m = m0 + 8 * g + i;
    const T* p = (const T*)a.x + (int64_t)m * a.ldx + n;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    if (m < a.M) {
      if (vec && n + 8 <= a.N) {
        if constexpr (sizeof(T) == 2) {
          const i32x4 w = *reinterpret_cast<const i32x4*>(p);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[i][2 * j] = __uint_as_float((uint32_t)w[j] << 16);
            v[i][2 * j + 1] = __uint_as_float((uint32_t)w[j] & 0xFFFF0000u);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const f32x4 w = *reinterpret_cast<const f32x4*>(p + 4 * j);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][4 * j + k] = w[k];
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (n + j < a.N) v[i][j] = to_f32<T>(p[j]);
      }
    }
  }

  uint32_t big[8];   // of the tile's block, or of each row's
  if constexpr (TILE) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
    m = dpp_max16(m);
    if (l == 0) top[0][g] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) m = max(m, top[0][k]);
#pragma unroll
    for (int i = 0; i < 8; ++i) big[i] = m;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
      big[i] = dpp_max16(m);
    }
  }
  if (a.q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int m = m0 + 8 * g + i;
      const uint32_t E = f8_exponent(big[i]);
      const float inv = f8_inverse(big[i], E);
      float c[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = f8_clamp(v[i][j] * inv);
      if (m < a.M) {
        i32x2 w;
        w[0] = (int)f8_code4(c[0], c[1], c[2], c[3]);
        w[1] = (int)f8_code4(c[4], c[5], c[6], c[7]);
        *reinterpret_cast<i32x2*>(a.q + m * Np + n) = w;
        if (l == 0) a.e[tn * Mr + m] = (uint8_t)E;
      }
    }
  }
  if (!a.qt) return;

  uint32_t colbig[8];
  if constexpr (TILE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) colbig[j] = big[0];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
      auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);   // the four g of a wave
      m = max(r[0], r[1]);
      r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
      m = max(r[0], r[1]);
      if ((threadIdx.x & 63) < 16) top[wave][8 * l + j] = m;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = 8 * l + j;
      colbig[j] = max(max(top[0][c], top[1][c]), max(top[2][c], top[3][c]));
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t E = f8_exponent(colbig[j]);
    const float inv = f8_inverse(colbig[j], E);
    float c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = f8_clamp(v[i][j] * inv);
    i32x2 w;
    w[0] = (int)f8_code4(c[0], c[1], c[2], c[3]);
    w[1] = (int)f8_code4(c[4], c[5], c[6], c[7]);
    *reinterpret_cast<i32x2*>(tr + (8 * l + j) * kPitch + 8 * g) = w;
    if (g == 0) ex[8 * l + j] = (uint8_t)E;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) {   // 16 lanes a row, eight bytes each
    const int r = g + 16 * k;
    if (n0 + r < a.N)
      *reinterpret_cast<i32x2*>(a.qt + (n0 + r) * Mp + m0 + 8 * l) = *reinterpret_cast<const i32x2*>(tr + r * kPitch + 8 * l);
  }
  if (threadIdx.x < 128 && n0 + (int)threadIdx.x < a.N) a.et[tm * Nr + n0 + threadIdx.x] = ex[threadIdx.x];
}

template <typename T>
hipError_t run(int kind, const QuantF8& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.M + 127) / 128) * (unsigned)((a.N + 127) / 128));
  const int vec = ((uintptr_t)a.x & 15) == 0 && a.ldx * sizeof(T) % 16 == 0;
  if (kind == SR_F8_TILE) SR_LAUNCH((quantize_f8_kernel<T, true>), grid, dim3(256), 0, st, a, vec);
  else SR_LAUNCH((quantize_f8_kernel<T, false>), grid, dim3(256), 0, st, a, vec);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_f8(int kind, int dtype, int M, int N, const void* x, int64_t ldx, uint8_t* q, uint8_t* e,
                              uint8_t* qt, uint8_t* et, hipStream_t st) {
  const QuantF8 a = {M, N, x, ldx, q, e, qt, et};
  return dtype == kBF16 ? run<bf16_t>(kind, a, st) : run<float>(kind, a, st);
}

}  // namespace sr
