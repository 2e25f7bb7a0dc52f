// Eight-bit activations: rows of the storage type to signed 8-bit codes and back.
//
// SR_Q8_ROW (operands of the int8 products; one fp32 scale per row, a = max |x| of the row):
//   q = nearest integer to 127 x / a, halves to the even one, of the exact quotient;  scale = a / 127.
// SR_Q8_BLOCK (what a forward keeps for its backward; a power of two per 32 channels):
//   e = the smallest integer with max |x| <= 127 2^e inside [-126, 121], kept as the byte e + 127;
//   q = nearest integer to x 2^-e, halves to even, within +-127.  The value q 2^e has at most seven
//   significant bits, so it is exact in bf16 and fp32: what reads a checkpoint rounds nothing.
//
// Both are bound by memory: 3 bytes per bf16 element (5 per fp32 one) each way.
#include "common.h"
#include "epilogue.h"
#include "quant8.h"
#include "sr_internal.h"

namespace sr {

namespace {

constexpr uint32_t kInfBits = 0x7F800000u;

SR_DEV uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Eight consecutive elements as fp32.
SR_DEV void load8(const bf16_t* p, float v[8]) {
  const i32x4 w = *reinterpret_cast<const i32x4*>(p);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float((uint32_t)w[j] << 16);
    v[2 * j + 1] = __uint_as_float((uint32_t)w[j] & 0xFFFF0000u);
  }
}
SR_DEV void load8(const float* p, float v[8]) {
  const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = a[j];
    v[4 + j] = b[j];
  }
}
SR_DEV void store8(bf16_t* p, const float v[8]) {
  i32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = (int)f2bf2(v[2 * j], v[2 * j + 1]);
  *reinterpret_cast<i32x4*>(p) = w;
}
SR_DEV void store8(float* p, const float v[8]) {
  f32x4 a, b;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    a[j] = v[j];
    b[j] = v[4 + j];
  }
  reinterpret_cast<f32x4*>(p)[0] = a;
  reinterpret_cast<f32x4*>(p)[1] = b;
}

// Largest value of each group of LPR (32 or 64) lanes, without LDS round trips (as wave_max).
template <int CTRL>
SR_DEV uint32_t dppu(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
template <int LPR>
SR_DEV uint32_t lanes_umax(uint32_t v) {
  v = max(v, dppu<0xB1>(v));
  v = max(v, dppu<0x4E>(v));
  v = max(v, dppu<0x141>(v));
  v = max(v, dppu<0x140>(v));
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max((uint32_t)r[0], (uint32_t)r[1]);
  if constexpr (LPR == 64) {
    const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = max((uint32_t)h[0], (uint32_t)h[1]);
  }
  return v;
}

// Adding 1.5 2^23 to |v| < 2^22 rounds v to an integer (halves to even), whose two's complement
// is then in the low bits of the sum.
constexpr float kMagic = 12582912.0f;
SR_DEV uint32_t low_bytes(float a, float b, float c, float d) {
  return (__float_as_uint(a) & 0xFFu) | (__float_as_uint(b) & 0xFFu) << 8 | (__float_as_uint(c) & 0xFFu) << 16 |
         __float_as_uint(d) << 24;
}

// 127 x / a to the nearest integer for the elements of one row; x and a are first scaled by the power of two that
// brings a into [0.5, 1).
//  bf16: 127 x is exact in fp32 and the quotient, corrected once, is within an ulp; a quotient that is no tie
//    lies more than 2^-18 from every tie (both sides are multiples of 2^-16 over a), and a tie is hit exactly.
//  fp32: x (127 / a) is within 3e-5 of the quotient, which decides the code unless it lies that near a tie; the few
//    waves that see such an element take the quotient in fp64, where 127 x is exact and the distance at least 2^-33.
template <typename T>
struct RowCode;
template <>
struct RowCode<bf16_t> {
  float a, inv;
  int ex;
  SR_DEV explicit RowCode(float amax) {
    ex = __builtin_amdgcn_frexp_expf(amax);
    a = __builtin_amdgcn_ldexpf(amax, -ex);
    inv = __fdiv_rn(1.0f, a);
  }
  SR_DEV void codes(float v[8]) const {   // in: elements, out: kMagic + code
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float t = 127.0f * __builtin_amdgcn_ldexpf(v[j], -ex);
      const float u = t * inv;
      v[j] = __fadd_rn(fmaf(fmaf(-u, a, t), inv, u), kMagic);
    }
  }
};
template <>
struct RowCode<float> {
  float a, inv;
  int ex;
  SR_DEV explicit RowCode(float amax) {
    ex = __builtin_amdgcn_frexp_expf(amax);
    a = __builtin_amdgcn_ldexpf(amax, -ex);
    inv = __fdiv_rn(127.0f, a);
  }
  SR_DEV void codes(float v[8]) const {
    float x[8], far = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j] = __builtin_amdgcn_ldexpf(v[j], -ex);
      const float u = x[j] * inv;
      v[j] = __fadd_rn(u, kMagic);
      far = fmaxf(far, fabsf(u - __fsub_rn(v[j], kMagic)));
    }
    if (__any(far > 0.5f - 4e-5f)) {
      const double ad = a, id = 1.0 / ad;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double t = 127.0 * (double)x[j], u = t * id;
        v[j] = __fadd_rn((float)__builtin_rint(fma(fma(-u, ad, t), id, u)), kMagic);
      }
    }
  }
};

// One row on LPR lanes (a part of a wave, a wave, or the workgroup), C chunks of eight elements per lane, which
// stay in registers between the maximum and the codes; C = 0: rows of any length, read twice.
// us for M x N, bf16 and fp32, against a wave per row that reads it twice: 16200 x 4096 56 and 93 -> 37 and 60,
// 16200 x 1024 11.8 and 17.8 -> 11.0 and 14.3, 16200 x 256 6.5 and 8.3 -> 4.4 and 5.9, 1024 x 4096 7.0 and 9.7 -> 4.3 and 6.2.
template <typename T, int LPR, int C>
__global__ __launch_bounds__(256) void quant_rows_kernel(const T* __restrict__ x, int M, int N, int8_t* __restrict__ q,
                                                         float* __restrict__ scale) {
  const int row = blockIdx.x * (256 / LPR) + (int)threadIdx.x / LPR, lane = threadIdx.x % LPR;
  const bool in = row < M;
  const T* xr = x + (size_t)row * N;
  float v[C > 0 ? C : 1][8];
  uint32_t m = 0;
  auto top = [&](const float w[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, abs_bits(w[j]));
  };
  if constexpr (C > 0) {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int c = (lane + i * LPR) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
      if (in && c < N) load8(xr + c, v[i]);
    }
#pragma unroll
    for (int i = 0; i < C; ++i) top(v[i]);
  } else if (in) {
    for (int c = lane * 8; c < N; c += LPR * 8) {
      load8(xr + c, v[0]);
      top(v[0]);
    }
  }
  m = lanes_umax<(LPR < 64 ? LPR : 64)>(m);
  if constexpr (LPR > 64) {
    __shared__ uint32_t red[LPR / 64];
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < LPR / 64; ++k) m = max(m, red[k]);
  }
  const bool ok = m < kInfBits;   // the order of magnitudes is that of the bits, NaN above Inf
  const float amax = __uint_as_float(m);
  if (in && lane == 0) scale[row] = ok ? __fdiv_rn(amax, 127.0f) : __uint_as_float(0x7FC00000u);
  const RowCode<T> rc(ok && m ? amax : 1.0f);
  auto put = [&](int c, float w[8]) {
    rc.codes(w);
    i32x2 b;
    b[0] = ok ? (int)low_bytes(w[0], w[1], w[2], w[3]) : 0;
    b[1] = ok ? (int)low_bytes(w[4], w[5], w[6], w[7]) : 0;
    if (in && c < N) *reinterpret_cast<i32x2*>(q + (size_t)row * N + c) = b;
  };
  if constexpr (C > 0) {
#pragma unroll
    for (int i = 0; i < C; ++i) put((lane + i * LPR) * 8, v[i]);
  } else if (in) {
    for (int c = lane * 8; c < N; c += LPR * 8) {
      load8(xr + c, v[0]);
      put(c, v[0]);
    }
  }
}

// LayerNorm and the codes of its rows: one wave per row, C chunks of eight channels per lane; mean, variance and
// maximum from registers, in fp32.
template <typename T, int C>
__global__ __launch_bounds__(256) void ln_quant_kernel(const float* __restrict__ x, const T* __restrict__ gamma,
                                                       const T* __restrict__ beta, const float* __restrict__ mod,
                                                       int mod_off, int M, int S, int D, float eps,
                                                       int8_t* __restrict__ q, float* __restrict__ scale) {
  const int row = blockIdx.x * 4 + wave_index(), lane = threadIdx.x & 63;
  if (row >= M) return;
  const float* shift = mod ? mod + (size_t)(row / S) * 6 * D + mod_off : nullptr;
  float v[C][8], sum = 0.f;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = (lane + i * 64) * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    if (c < D) load8(x + (size_t)row * D + c, v[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += v[i][j];
  }
  const float mean = wave_sum(sum) / (float)D;
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < C; ++i)
    if ((lane + i * 64) * 8 < D) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] -= mean;
        sq = fmaf(v[i][j], v[i][j], sq);
      }
    }
  const float rstd = rsqrtf(wave_sum(sq) / (float)D + eps);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = (lane + i * 64) * 8;
    if (c < D) {
      float w[8], b[8];
      if (mod) {
        load8(shift + D + c, w);
        load8(shift + c, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] += 1.0f;
      } else {
        load8(gamma + c, w);
        load8(beta + c, b);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] = fmaf(v[i][j] * rstd, w[j], b[j]);
        m = max(m, abs_bits(v[i][j]));
      }
    }
  }
  m = lanes_umax<64>(m);
  const bool ok = m < kInfBits;
  const float amax = __uint_as_float(m);
  if (lane == 0) scale[row] = ok ? __fdiv_rn(amax, 127.0f) : __uint_as_float(0x7FC00000u);
  const RowCode<float> rc(ok && m ? amax : 1.0f);
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = (lane + i * 64) * 8;
    rc.codes(v[i]);
    i32x2 b;
    b[0] = ok ? (int)low_bytes(v[i][0], v[i][1], v[i][2], v[i][3]) : 0;
    b[1] = ok ? (int)low_bytes(v[i][4], v[i][5], v[i][6], v[i][7]) : 0;
    if (c < D) *reinterpret_cast<i32x2*>(q + (size_t)row * D + c) = b;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void dequant_rows_kernel(const int8_t* __restrict__ q, const float* __restrict__ scale,
                                                           size_t n8, int N8, T* __restrict__ x) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n8) return;
  const i32x2 w = reinterpret_cast<const i32x2*>(q)[i];
  const float s = scale[i / (size_t)N8];
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)((uint32_t)w[j >> 2] >> (8 * (j & 3))) * s;
  store8(x + i * 8, v);
}

// Eight elements per lane, four lanes per block of 32 channels.
template <typename T>
SR_DEV void quant_block8(const T* __restrict__ x, size_t i, int8_t* __restrict__ q, uint8_t* __restrict__ e) {
  float v[8];
  load8(x + i * 8, v);
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[j]));
  m = max(m, dppu<0xB1>(m));   // the four lanes of a block: pairs, then quads
  m = max(m, dppu<0x4E>(m));
  const uint32_t E = block_exponent(m);
  const float inv = __uint_as_float((254u - min(E, 253u)) << 23);   // 2^-e
#pragma unroll
  for (int j = 0; j < 8; ++j)   // the upper limit is met only by a block whose 2^e is at its largest
    v[j] = __builtin_amdgcn_fmed3f(fmaf(v[j], inv, kMagic), kMagic - 127.0f, kMagic + 127.0f);
  i32x2 w;
  w[0] = E == 255u ? 0 : (int)low_bytes(v[0], v[1], v[2], v[3]);
  w[1] = E == 255u ? 0 : (int)low_bytes(v[4], v[5], v[6], v[7]);
  reinterpret_cast<i32x2*>(q)[i] = w;
  if ((threadIdx.x & 3) == 0) e[i >> 2] = (uint8_t)E;
}

template <typename T>
SR_DEV void dequant_block8(const int8_t* __restrict__ q, const uint8_t* __restrict__ e, size_t i, T* __restrict__ x) {
  const i32x2 w = reinterpret_cast<const i32x2*>(q)[i];
  const float s = block_scale(e[i >> 2]);
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)((uint32_t)w[j >> 2] >> (8 * (j & 3))) * s;
  store8(x + i * 8, v);
}

template <typename T, bool QUANT>
__global__ __launch_bounds__(256) void blocks8_kernel(T* __restrict__ x, size_t n8, int8_t* __restrict__ q,
                                                      uint8_t* __restrict__ e) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n8) return;   // n8 is a multiple of 8: the four lanes of a block leave together
  if constexpr (QUANT) quant_block8<T>(x, i, q, e);
  else dequant_block8<T>(q, e, i, x);
}

template <typename T>
__global__ __launch_bounds__(256) void gelu_kept_kernel(Kept8 z, size_t n8, T* __restrict__ gz) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n8) return;
  const i32x2 w = reinterpret_cast<const i32x2*>(z.q)[i];
  const float s = block_scale(z.e[i >> 2]);
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j)
    v[j] = gelu_f<gelu_deg<T>()>((float)(int8_t)((uint32_t)w[j >> 2] >> (8 * (j & 3))) * s);
  store8(gz + i * 8, v);
}

// Job j takes the workgroups [first[j], first[j + 1]).
struct Q8Jobs {
  Q8Job job[kMaxQ8Jobs];
  int first[kMaxQ8Jobs + 1];
};
template <bool QUANT>
__global__ __launch_bounds__(256) void q8_jobs_kernel(Q8Jobs js) {
  int j = 0;
  while (j + 1 < kMaxQ8Jobs && (int)blockIdx.x >= js.first[j + 1]) ++j;
  const Q8Job& b = js.job[j];
  const size_t i = (size_t)((int)blockIdx.x - js.first[j]) * 256 + threadIdx.x;
  if (i >= b.n / 8) return;
  if (b.dtype == kBF16) {
    if constexpr (QUANT) quant_block8<bf16_t>((const bf16_t*)b.x, i, b.q, b.e);
    else dequant_block8<bf16_t>(b.q, b.e, i, (bf16_t*)b.x);
  } else {
    if constexpr (QUANT) quant_block8<float>((const float*)b.x, i, b.q, b.e);
    else dequant_block8<float>(b.q, b.e, i, (float*)b.x);
  }
}

template <typename T>
hipError_t quant(int kind, int M, int N, const void* x, int8_t* q, void* scale, hipStream_t st) {
  if (kind == SR_Q8_ROW) {
    auto rows = [&](auto lpr, auto c) {
      constexpr int LPR = decltype(lpr)::value, C = decltype(c)::value;
      SR_LAUNCH((quant_rows_kernel<T, LPR, C>), dim3((unsigned)(((size_t)M * LPR + 255) / 256)), dim3(256), 0, st,
                (const T*)x, M, N, q, (float*)scale);
    };
    if (N <= 256) rows(IC<32>{}, IC<1>{});
    else if (N <= 512) rows(IC<64>{}, IC<1>{});
    else if (N <= 1024) rows(IC<64>{}, IC<2>{});
    else if (N <= 2048) rows(IC<256>{}, IC<1>{});
    else if (N <= 4096) rows(IC<256>{}, IC<2>{});
    else if (N <= 8192) rows(IC<256>{}, IC<4>{});
    else rows(IC<256>{}, IC<0>{});
  } else {
    const size_t n8 = (size_t)M * N / 8;
    SR_LAUNCH((blocks8_kernel<T, true>), dim3((unsigned)((n8 + 255) / 256)), dim3(256), 0, st, (T*)const_cast<void*>(x),
              n8, q, (uint8_t*)scale);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t dequant(int kind, int M, int N, const int8_t* q, const void* scale, void* x, hipStream_t st) {
  const size_t n8 = (size_t)M * N / 8;
  const dim3 grid((unsigned)((n8 + 255) / 256));
  if (kind == SR_Q8_ROW)
    SR_LAUNCH(dequant_rows_kernel<T>, grid, dim3(256), 0, st, q, (const float*)scale, n8, N / 8, (T*)x);
  else
    SR_LAUNCH((blocks8_kernel<T, false>), grid, dim3(256), 0, st, (T*)x, n8, const_cast<int8_t*>(q),
              (uint8_t*)const_cast<void*>(scale));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_q8_jobs(const Q8Job* jobs, int njobs, bool quantize, hipStream_t st) {
  if (njobs > kMaxQ8Jobs) return hipErrorInvalidValue;
  Q8Jobs js{};
  int blocks = 0;
  for (int j = 0; j < njobs; ++j) {
    js.job[j] = jobs[j];
    js.first[j] = blocks;
    blocks += (int)((jobs[j].n / 8 + 255) / 256);
  }
  if (blocks == 0) return hipSuccess;
  for (int j = njobs; j <= kMaxQ8Jobs; ++j) js.first[j] = blocks;
  if (quantize) SR_LAUNCH(q8_jobs_kernel<true>, dim3((unsigned)blocks), dim3(256), 0, st, js);
  else SR_LAUNCH(q8_jobs_kernel<false>, dim3((unsigned)blocks), dim3(256), 0, st, js);
  return hipGetLastError();
}

hipError_t launch_gelu_kept(int dtype, const Kept8& z, void* gz, size_t n, hipStream_t st) {
  const size_t n8 = n / 8;
  const dim3 grid((unsigned)((n8 + 255) / 256));
  if (dtype == kBF16) SR_LAUNCH(gelu_kept_kernel<bf16_t>, grid, dim3(256), 0, st, z, n8, (bf16_t*)gz);
  else SR_LAUNCH(gelu_kept_kernel<float>, grid, dim3(256), 0, st, z, n8, (float*)gz);
  return hipGetLastError();
}

template <typename T>
static hipError_t ln_quant(const float* x, const void* gamma, const void* beta, const float* mod, int mod_off, int M, int S,
                           int D, float eps, int8_t* q, float* scale, hipStream_t st) {
  auto rows = [&](auto c) {
    SR_LAUNCH((ln_quant_kernel<T, decltype(c)::value>), dim3((unsigned)((M + 3) / 4)), dim3(256), 0, st, x,
              (const T*)gamma, (const T*)beta, mod, mod_off, M, S, D, eps, q, scale);
  };
  if (D <= 512) rows(IC<1>{});
  else if (D <= 1024) rows(IC<2>{});
  else if (D <= 2048) rows(IC<4>{});
  else return hipErrorInvalidValue;
  return hipGetLastError();
}
hipError_t launch_ln_quant(int dtype, const float* x, const void* gamma, const void* beta, const float* mod, int mod_off,
                           int M, int S, int D, float eps, int8_t* q, float* scale, hipStream_t st) {
  return dtype == kBF16 ? ln_quant<bf16_t>(x, gamma, beta, mod, mod_off, M, S, D, eps, q, scale, st)
                        : ln_quant<float>(x, gamma, beta, mod, mod_off, M, S, D, eps, q, scale, st);
}

hipError_t launch_quantize8(int kind, int dtype, int M, int N, const void* x, int8_t* q, void* scale, hipStream_t st) {
  return dtype == kBF16 ? quant<bf16_t>(kind, M, N, x, q, scale, st) : quant<float>(kind, M, N, x, q, scale, st);
}
hipError_t launch_dequantize8(int kind, int dtype, int M, int N, const int8_t* q, const void* scale, void* x,
                              hipStream_t st) {
  return dtype == kBF16 ? dequant<bf16_t>(kind, M, N, q, scale, x, st) : dequant<float>(kind, M, N, q, scale, x, st);
}

}  // namespace sr
