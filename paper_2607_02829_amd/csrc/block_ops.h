// Launchers of the operators that blocks of single calls are put together from: rotary positions, dropout, the
// residual step with its norms, and linear layers on 8-bit floating point.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/sr.h"
#include "common.h"
#include "drop.h"
#include "sr_internal.h"

namespace sr {

// Results of this many bytes and more, in rows of whole lines, are stored past the caches (non-temporal) by the kernels that come back to
// what they have read: the products, whose operands other workgroups read again, and the residual step, whose backward reads x1
// and y again.  us, past and in the caches, with the call that reads the results (sr_quantize_f8, or the residual step):
//   8-bit codes, 16200 x 4096 x 1024 124.5 and 131.0, with GELU 140 and 152, 16200 x 1024 x 4096 100.1 and 100.8
//   residual step, both directions, 8 x 512 x 1024 50.2 and 49.4 (without readers 33.5 and 36.5), 16200 x 1024 132.0 and 132.7
// Partial lines lose: 16200 x 1030 x 1024 56.6 and 52.7, the residual step of 16200 x 1023 175 and 168.  So do kernels that read everything
// once and have nothing to keep in the caches; there the reader pays more than the call gains: rotary of 65536 x 1024 88.6 and 84.9
// (alone 47.2 and 50.9), dropout of 16200 x 1024 added to a residual 30.0 and 28.1 (alone 15.3 and 17.7).
constexpr int64_t kStreamBytes = 4 << 20;
SR_DEV bool past_caches(int64_t rows, int64_t cols, int elt) { return cols * elt % 128 == 0 && rows * cols * elt >= kStreamBytes; }
// Runs of 8 and 16 bytes that start at any element: global accesses need no more alignment than that here, so rows of odd
// lengths take the same wide accesses (16200 x 4093 dropout of whole rows 103 -> 55 us, 8192 x 1023 x 1000 on 8-bit codes with theirs 34 -> 26).
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef int i32x2_any __attribute__((ext_vector_type(2), aligned(2), may_alias));
SR_DEV i32x4 load16(const void* p) { return __builtin_bit_cast(i32x4, *(const i32x4_any*)p); }
SR_DEV i32x2 load8(const void* p) { return __builtin_bit_cast(i32x2, *(const i32x2_any*)p); }
SR_DEV void store16(void* p, i32x4 v, bool past = false) {
  if (past) {   // between the two empty statements, or the compiler makes one plain store of both branches
    asm volatile("" ::: "memory");
    __builtin_nontemporal_store(__builtin_bit_cast(i32x4_any, v), (i32x4_any*)p);
    asm volatile("" ::: "memory");
  } else {
    *(i32x4_any*)p = __builtin_bit_cast(i32x4_any, v);
  }
}
SR_DEV void store8(void* p, i32x2 v) { *(i32x2_any*)p = __builtin_bit_cast(i32x2_any, v); }

constexpr int kMaxRotPairs = 128;   // head dims up to 256
// Largest angle: its rounding in 64 bits is 2^-8 there, and the quarter turns in it are still counted to 2^-7 (turn_of).
constexpr double kMaxRotAngle = 0x1p45;
struct Rotary {
  int B = 0, S = 0, heads = 0, hd = 0;
  int axes = 1, grid[3] = {1, 1, 1}, first[4] = {0, 0, 0, 0};   // axis a owns pairs first[a] .. first[a + 1] - 1
  int neighbours = 0, inverse = 0, idx_shared = 0;
  double origin[3] = {0, 0, 0}, step[3] = {1, 1, 1};
  double freq[kMaxRotPairs];
  const void* x = nullptr;
  void* y = nullptr;
  const int32_t* idx = nullptr;
  int64_t ldx = 0, ldy = 0;
};
hipError_t launch_rotary(int dtype, const Rotary& a, hipStream_t st);

struct Dropout {
  int64_t M = 0, N = 0;
  const void *x = nullptr, *resid = nullptr;
  void* y = nullptr;
  DropArgs drop;
};
hipError_t launch_dropout(int dtype, const Dropout& a, hipStream_t st);

struct ResidualNorm {
  int B = 0, S = 0, D = 0;
  int norm = 0, post = 0;
  float eps = 0.f;
  int64_t mod_stride = 0;
  DropArgs drop;
  sr_residual_norm_params w = {};
  const void *x = nullptr, *y = nullptr;   // backward: x is the forward's x1
  void *x1 = nullptr, *u = nullptr;
  uint8_t *uq = nullptr, *ue = nullptr;
  float* stats = nullptr;
  const void *dx1 = nullptr, *du = nullptr;
  void *dx = nullptr, *dy = nullptr;
  sr_residual_norm_grads g = {};
  float* part = nullptr;
};
constexpr int kMaxNormD = 8192;
size_t residual_norm_need(int B, int S, int D);      // bytes that the backward of these sizes uses
size_t residual_norm_scratch(int B, int S, int D);   // bytes for these sizes and all smaller ones
hipError_t launch_residual_norm_fwd(int dtype, int stream_dtype, const ResidualNorm& a, hipStream_t st);
hipError_t launch_residual_norm_bwd(int dtype, int stream_dtype, const ResidualNorm& a, hipStream_t st);

// ---- 8-bit floating point

constexpr int kF8Block = 128;
inline int64_t f8_cols(int64_t c) { return (c + 127) / 128 * 128; }
inline int64_t f8_rows(int64_t r) { return (r + 15) / 16 * 16; }
// Exponent byte of a block whose largest magnitude has the bits m: 448 2^e has the mantissa 0x600000, so a larger one
// carries into the exponent.  1 <= e + 127 <= 246, so that 2^e and 2^-e are normal and 448 2^e is finite.
SR_DEV uint32_t f8_exponent(uint32_t m) {
  const int E = (int)((m + 0x1FFFFFu) >> 23) - 8;
  return m >= 0x7F800000u ? 127u : (uint32_t)min(max(E, 1), 246);
}
// 2^-e of an exponent byte (exact), NaN for a block with an Inf or NaN, which makes all of its codes NaN.
SR_DEV float f8_inverse(uint32_t m, uint32_t E) { return __uint_as_float(m >= 0x7F800000u ? 0x7FC00000u : (254u - E) << 23); }
// Codes of four values that 2^-e has been multiplied into.
SR_DEV uint32_t f8_code4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// The first n of four codes, zeros behind them: in a block with an Inf or NaN the values past a row's end would be NaN too.
SR_DEV uint32_t f8_first(uint32_t w, int n) { return n >= 4 ? w : n <= 0 ? 0u : w & ((1u << (8 * n)) - 1u); }
SR_DEV float f8_clamp(float v) { return __builtin_isnan(v) ? v : fminf(fmaxf(v, -448.f), 448.f); }

hipError_t launch_quantize_f8(int kind, int dtype, int M, int N, const void* x, int64_t ldx, uint8_t* q, uint8_t* e,
                              uint8_t* qt, uint8_t* et, hipStream_t st);

struct LinearF8 {
  int M = 0, N = 0, K = 0;
  const uint8_t *xq = nullptr, *xe = nullptr, *wq = nullptr, *we = nullptr;
  const void* bias = nullptr;
  void* y = nullptr;
  int act = SR_ACT_NONE;
  float* scratch = nullptr;
};
size_t linear_f8_need(int M, int N, int K);      // bytes that a product of these sizes uses
size_t linear_f8_scratch(int M, int N, int K);   // bytes for these sizes and all smaller ones
hipError_t launch_linear_f8(int dtype, const LinearF8& a, hipStream_t st);

}  // namespace sr
