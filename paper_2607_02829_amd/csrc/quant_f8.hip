// Codes of 8-bit floating point with a power of two per block of 128 (sr_quantize_f8), of a matrix and of its
// transpose in one pass.
//
// A workgroup takes a tile of 128 x 128: thread (g, l) holds rows 8 g .. 8 g + 7, channels 8 l .. 8 l + 7, as they lie in
// memory.  A row's block is then 16 neighbouring lanes, a column's the 16 values of g, and eight codes of a column are eight
// consecutive bytes of the transpose, which leaves through LDS in whole rows.  Magnitudes are compared as bit patterns
// (pairs of bf16 at once).  Bound by memory.
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

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Eight values of a row in memory's order, W words of them; magnitudes by word (two values of bf16, or one), the larger of two
// words by value, and as the bits of an fp32: of a word's larger value (wide), or of column j (column).
template <typename T>
struct Row8;
template <>
struct Row8<bf16_t> {
  static constexpr int W = 4;   // words
  uint32_t w[4];
  SR_DEV void load(const bf16_t* p) {
    const i32x4 r = load16(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (uint32_t)r[j];
  }
  SR_DEV void set(int j, bf16_t v) { w[j / 2] |= (uint32_t)v << (16 * (j & 1)); }
  SR_DEV float at(int j) const { return __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16); }
  static SR_DEV uint32_t mag(uint32_t v) { return v & 0x7FFF7FFFu; }
  static SR_DEV uint32_t top(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
  }
  static SR_DEV uint32_t wide(uint32_t m) { return max(m & 0xFFFF0000u, m << 16); }          // of both values of a word
  static SR_DEV uint32_t column(const uint32_t* m, int j) { return j & 1 ? m[j / 2] & 0xFFFF0000u : m[j / 2] << 16; }
};
template <>
struct Row8<float> {
  static constexpr int W = 8;
  uint32_t w[8];
  SR_DEV void load(const float* p) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const i32x4 r = load16(p + 4 * k);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * k + j] = (uint32_t)r[j];
    }
  }
  SR_DEV void set(int j, float v) { w[j] = __float_as_uint(v); }
  SR_DEV float at(int j) const { return __uint_as_float(w[j]); }
  static SR_DEV uint32_t mag(uint32_t v) { return v & 0x7FFFFFFFu; }
  static SR_DEV uint32_t top(uint32_t a, uint32_t b) { return max(a, b); }
  static SR_DEV uint32_t wide(uint32_t m) { return m; }
  static SR_DEV uint32_t column(const uint32_t* m, int j) { return m[j]; }
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

// Codes of eight values, of one block or of one each; in a tile at the matrix's edge `left` of them are its own.
SR_DEV i32x2 codes8(const float (&v)[8], const float (&inv)[8], bool clamps, bool edge, int left) {
  float c[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) c[j] = v[j] * inv[j];
  if (clamps) {   // blocks past 1.75 * 2^127 alone can pass 448
#pragma unroll
    for (int j = 0; j < 8; ++j) c[j] = f8_clamp(c[j]);
  }
  i32x2 w;
  w[0] = (int)f8_code4(c[0], c[1], c[2], c[3]);
  w[1] = (int)f8_code4(c[4], c[5], c[6], c[7]);
  if (edge) {
    w[0] = (int)f8_first((uint32_t)w[0], left);
    w[1] = (int)f8_first((uint32_t)w[1], left - 4);
  }
  return w;
}

template <typename T, bool TILE, bool ROWS, bool COLS>
__global__ __launch_bounds__(256) void quantize_f8_kernel(QuantF8 a) {
  typedef Row8<T> R;
  __shared__ __attribute__((aligned(16))) uint8_t tr[COLS ? 128 * kPitch : 16];
  __shared__ uint32_t top[4][COLS ? 128 : 16];
  __shared__ __attribute__((aligned(16))) uint8_t ex[128];
  const int l = threadIdx.x & 15, g = threadIdx.x >> 4, wave = wave_index();
  const int tiles_n = (a.N + 127) / 128, tm = (int)(blockIdx.x / (unsigned)tiles_n), tn = (int)(blockIdx.x - (unsigned)tm * (unsigned)tiles_n);
  const int m0 = tm * 128, n0 = tn * 128, n = n0 + 8 * l;
  const int64_t Np = (int64_t)tiles_n * 128, Mp = (int64_t)(a.M + 127) / 128 * 128;
  const int64_t Mr = (int64_t)(a.M + 15) / 16 * 16, Nr = (int64_t)(a.N + 15) / 16 * 16;

  R v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int m = m0 + 8 * g + i;
    const T* p = (const T*)a.x + (int64_t)m * a.ldx + n;
#pragma unroll
    for (int j = 0; j < R::W; ++j) v[i].w[j] = 0;
    if (m < a.M) {
      if (n + 8 <= a.N) {
        v[i].load(p);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (n + j < a.N) v[i].set(j, p[j]);
      }
    }
  }

  uint32_t tile_top = 0;
  if constexpr (TILE) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < R::W; ++j) m = R::top(m, R::mag(v[i].w[j]));
    m = dpp_max16(R::wide(m));
    if (l == 0) top[0][g] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) m = max(m, top[0][k]);
    tile_top = m;
    if constexpr (COLS) __syncthreads();
  }
  if constexpr (ROWS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int m = m0 + 8 * g + i;
      uint32_t big = tile_top;
      if constexpr (!TILE) {
        uint32_t t = R::mag(v[i].w[0]);
#pragma unroll
        for (int j = 1; j < R::W; ++j) t = R::top(t, R::mag(v[i].w[j]));
        big = dpp_max16(R::wide(t));
      }
      const uint32_t E = f8_exponent(big);
      const float s = f8_inverse(big, E);
      float c[8], inv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        c[j] = v[i].at(j);
        inv[j] = s;
      }
      if (m < a.M) {
        *reinterpret_cast<i32x2*>(a.q + m * Np + n) = codes8(c, inv, E == 246u, n0 + 128 > a.N, a.N - n);
        if (l == 0) a.e[tn * Mr + m] = (uint8_t)E;
      }
    }
  }
  if constexpr (COLS) {
    uint32_t colmax[R::W];
    if constexpr (!TILE) {
#pragma unroll
      for (int j = 0; j < R::W; ++j) {
        uint32_t m = R::mag(v[0].w[j]);
#pragma unroll
        for (int i = 1; i < 8; ++i) m = R::top(m, R::mag(v[i].w[j]));
        auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);   // the four g of a wave
        m = R::top(r[0], r[1]);
        r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
        m = R::top(r[0], r[1]);
        if ((threadIdx.x & 63) < 16) top[wave][R::W * l + j] = m;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < R::W; ++j) {
        const int c = R::W * l + j;
        colmax[j] = R::top(R::top(top[0][c], top[1][c]), R::top(top[2][c], top[3][c]));
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t big = TILE ? tile_top : R::column(colmax, j), E = f8_exponent(big);
      const float s = f8_inverse(big, E);
      float c[8], inv[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        c[i] = v[i].at(j);
        inv[i] = s;
      }
      *reinterpret_cast<i32x2*>(tr + (8 * l + j) * kPitch + 8 * g) = codes8(c, inv, E == 246u, m0 + 128 > a.M, a.M - (m0 + 8 * g));
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
}

template <typename T, bool TILE>
hipError_t run(const QuantF8& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.M + 127) / 128) * (unsigned)((a.N + 127) / 128));
  if (!a.qt) SR_LAUNCH((quantize_f8_kernel<T, TILE, true, false>), grid, dim3(256), 0, st, a);
  else if (!a.q) SR_LAUNCH((quantize_f8_kernel<T, TILE, false, true>), grid, dim3(256), 0, st, a);
  else SR_LAUNCH((quantize_f8_kernel<T, TILE, true, true>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_f8(int kind, int dtype, int M, int N, const void* x, int64_t ldx, uint8_t* q, uint8_t* e,
                              uint8_t* qt, uint8_t* et, hipStream_t st) {
  const QuantF8 a = {M, N, x, ldx, q, e, qt, et};
  if (kind == SR_F8_TILE) return dtype == kBF16 ? run<bf16_t, true>(a, st) : run<float, true>(a, st);
  return dtype == kBF16 ? run<bf16_t, false>(a, st) : run<float, false>(a, st);
}

}  // namespace sr
