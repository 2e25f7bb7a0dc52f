// The eight-bit operators (quant8.hip, linear8.hip, wgrad8.hip): launchers and the checkpoint format.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/sr.h"
#include "common.h"
#include "sr_internal.h"

namespace sr {

constexpr int kQBlock = 32;   // channels that share an exponent

// Exponent byte of a block whose largest magnitude has the bits m: the smallest e with
// |x| <= 127 2^e.  127 2^e has the mantissa 0x7E0000, so a mantissa above it carries into the
// exponent.  255 for a block with an Inf or NaN; 1 <= e + 127 <= 248 otherwise, so that 127 2^e stays
// finite and 2^e and 2^-e are normal.
SR_DEV uint32_t block_exponent(uint32_t m) {
  const int E = (int)((m + 0x1FFFFu) >> 23) - 6;
  return m >= 0x7F800000u ? 255u : (uint32_t)min(max(E, 1), 248);
}
// 2^e of an exponent byte; NaN for 255 (a block with an Inf or NaN reads back as NaN).
SR_DEV float block_scale(uint32_t E) { return __uint_as_float(E == 255u ? 0x7FC00000u : E << 23); }

hipError_t launch_quantize8(int kind, int dtype, int M, int N, const void* x, int8_t* q, void* scale, hipStream_t st);
hipError_t launch_dequantize8(int kind, int dtype, int M, int N, const int8_t* q, const void* scale, void* x,
                              hipStream_t st);

// SR_Q8_BLOCK of up to kMaxQ8Jobs tensors in one launch, with the values of single calls.
struct Q8Job {
  void* x = nullptr;   // n elements of the type, a multiple of 64
  int dtype = 0;
  size_t n = 0;
  int8_t* q = nullptr;
  uint8_t* e = nullptr;
};
constexpr int kMaxQ8Jobs = 6;
hipError_t launch_q8_jobs(const Q8Job* jobs, int njobs, bool quantize, hipStream_t st);

// gz = GELU(z) of the pre-activation kept in 8 bits, n elements: launch_gelu of the value restored.
hipError_t launch_gelu_kept(int dtype, const Kept8& z, void* gz, size_t n, hipStream_t st);

// LayerNorm of the fp32 rows x [M, D] (affine, or modulated by mod as in launch_ln_fwd; D <= 2048) to SR_Q8_ROW
// codes in one pass.
hipError_t launch_ln_quant(int dtype, const float* x, const void* gamma, const void* beta, const float* mod, int mod_off,
                           int M, int S, int D, float eps, int8_t* q, float* scale, hipStream_t st);

// y = act(xs_m ws_n sum_k xq_mk wq_nk + bias_n);  with kActResid out = resid + gate_b (the value before act), fp32
constexpr int kActResid = 2;
struct Linear8 {
  int M = 0, N = 0, K = 0;
  const int8_t *xq = nullptr, *wq = nullptr;
  const float *xs = nullptr, *ws = nullptr;
  const void* bias = nullptr;   // storage type, or null
  void* y = nullptr;            // storage type (not with kActResid)
  int act = SR_ACT_NONE;
  const float* resid = nullptr;   // [M, N]
  const float* gate = nullptr;    // per sample (S rows each), gate[b * gate_stride + n], or null
  int gate_stride = 0, S = 1;
  float* out = nullptr;           // [M, N], may not be resid
};
hipError_t launch_linear8(int dtype, const Linear8& a, hipStream_t st);

// dw[n, k] = sum_m dy[m, n] xhat[m, k] and db[n] = sum_m dy[m, n] (db may be null), xhat the
// SR_Q8_BLOCK values of xq and xe.
struct Wgrad8 {
  int M = 0, N = 0, K = 0;
  const void* dy = nullptr;
  const int8_t* xq = nullptr;
  const uint8_t* xe = nullptr;
  float *dw = nullptr, *db = nullptr, *scratch = nullptr;
};
size_t wgrad8_scratch(int dtype, int M, int N, int K);   // bytes; with N = K not less for more of M
hipError_t launch_wgrad8(int dtype, const Wgrad8& a, hipStream_t st);

}  // namespace sr
