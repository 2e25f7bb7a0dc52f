// Products of 8-bit floating point with a power of two per block of 128 (sr_linear_f8).
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes the codes as they are and a power of two per lane (its row, its 32 values of k)
// as an exponent byte, so blocks of 128 cost no instruction of their own.  Its sums are fp32, but of eight products that
// it adds at a time it drops what lies 14 bits below the largest: 1.5e-5 of the results' deviation, a hundredth of a
// bf16 result's rounding.  So bf16 results come from it, and fp32 results from products in bf16, which holds codes times their powers of two
// exactly (v_cvt_scalef32_pk_bf16_fp8), at half its rate.
#include "block_ops.h"
#include "epilogue.h"

namespace sr {

namespace {

typedef __attribute__((__vector_size__(8 * sizeof(int)))) int i32x8;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight codes times 2^e as bf16 (exact).
SR_DEV bf16x8 decode8(int lo, int hi, float scale) {
  union {
    bf16x2 h[4];
    bf16x8 v;
  } u;
  u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false);
  u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true);
  u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false);
  u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
  return u.v;
}

// 32 x 32 products of one wave, fragments straight from memory.
template <typename T>
__global__ __launch_bounds__(64) void linear_f8_kernel(LinearF8 a) {
  const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
  const int tn = (a.N + 31) / 32, m0 = (int)(blockIdx.x / (unsigned)tn) * 32, n0 = (int)(blockIdx.x % (unsigned)tn) * 32;
  const int kb = (a.K + 127) / 128;
  const uint32_t Kp = 128u * kb, Mr = (uint32_t)((a.M + 15) / 16 * 16), Nr = (uint32_t)((a.N + 15) / 16 * 16);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq, (uint32_t)a.M * Kp), rw = make_rsrc(a.wq, (uint32_t)a.N * Kp);
  const __amdgpu_buffer_rsrc_t rex = make_rsrc(a.xe, Mr * kb), rew = make_rsrc(a.we, Nr * kb);
  f32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  for (int b = 0; b < kb; ++b) {
    const int ex = __builtin_amdgcn_raw_buffer_load_b8(rex, b * Mr + m0 + r, 0, 0);
    const int ew = __builtin_amdgcn_raw_buffer_load_b8(rew, b * Nr + n0 + r, 0, 0);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      i32x8 x, w;
      const uint32_t ox = (uint32_t)(m0 + r) * Kp + 128 * b + 64 * s + 32 * h, ow = (uint32_t)(n0 + r) * Kp + 128 * b + 64 * s + 32 * h;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const i32x4 tx = buf_load16(rx, ox + 16 * k), tw = buf_load16(rw, ow + 16 * k);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[4 * k + i] = tx[i];
          w[4 * k + i] = tw[i];
        }
      }
      if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, w, acc, 0, 0, 0, ex, 0, ew);
      } else {
        const float sx = __uint_as_float((uint32_t)ex << 23), sw = __uint_as_float((uint32_t)ew << 23);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode8(x[2 * k], x[2 * k + 1], sx), decode8(w[2 * k], w[2 * k + 1], sw),
                                                        acc, 0, 0, 0);
      }
    }
  }
  const int n = n0 + r;
  if (n >= a.N) return;
  const float bias = a.bias ? to_f32<T>(((const T*)a.bias)[n]) : 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {   // register i: row 8 (i / 4) + 4 h + i % 4, column lane % 32
    const int m = m0 + 8 * (i >> 2) + 4 * h + (i & 3);
    if (m < a.M) {
      float v = acc[i] + bias;
      if (a.act == SR_ACT_GELU) v = gelu_lim(v);
      ((T*)a.y)[(size_t)m * a.N + n] = from_f32<T>(v);
    }
  }
}

}  // namespace

size_t linear_f8_scratch(int, int, int) { return 0; }

hipError_t launch_linear_f8(int dtype, const LinearF8& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.N + 31) / 32) * (unsigned)((a.M + 31) / 32));
  if (dtype == kBF16) SR_LAUNCH((linear_f8_kernel<bf16_t>), grid, dim3(64), 0, st, a);
  else SR_LAUNCH((linear_f8_kernel<float>), grid, dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace sr
