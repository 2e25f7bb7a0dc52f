// Linear layer on 8-bit integers: y[m, n] = act(xs[m] ws[n] sum_k xq[m, k] wq[n, k] + bias[n]).
//
// The products are summed exactly in int32 (127^2 K < 2^31 for every K that the call takes); the sum
// is then rounded to fp32 once, scaled, and rounded once to the storage type.
#include "common.h"
#include "epilogue.h"
#include "quant8.h"
#include "sr_internal.h"

namespace sr {

namespace {

typedef __attribute__((__vector_size__(16 * sizeof(int)))) int i32x16;

template <typename T>
SR_DEV float finish(const Linear8& a, int m, int n, int acc) {
  float v = (float)acc * a.xs[m] * a.ws[n];
  if (a.bias) v += to_f32<T>(((const T*)a.bias)[n]);
  return a.act == SR_ACT_GELU ? gelu_f<gelu_deg<T>()>(v) : v;
}

// One wave per 32 x 32 tile of y, operands straight from memory: lane l holds 16 k values of row
// (or output channel) l % 32, k = 16 (l / 32) .. of each 32.  Rows past the end read zeros.
template <typename T>
__global__ __launch_bounds__(64) void linear8_kernel(Linear8 a) {
  const int lane = threadIdx.x, r = lane & 31, h = lane >> 5;
  const int m0 = blockIdx.y * 32, n0 = blockIdx.x * 32;
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq, (uint32_t)a.M * (uint32_t)a.K);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wq, (uint32_t)a.N * (uint32_t)a.K);
  const uint32_t ox = (uint32_t)(m0 + r) * (uint32_t)a.K + 16u * h, ow = (uint32_t)(n0 + r) * (uint32_t)a.K + 16u * h;
  i32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0;
  for (int k = 0; k < a.K; k += 32)
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(buf_load16(rx, ox + k), buf_load16(rw, ow + k), acc, 0, 0, 0);
  const int n = n0 + r;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int m = m0 + 8 * (i >> 2) + 4 * h + (i & 3);
    if (m < a.M && n < a.N) ((T*)a.y)[(size_t)m * a.N + n] = from_f32<T>(finish<T>(a, m, n, acc[i]));
  }
}

}  // namespace

hipError_t launch_linear8(int dtype, const Linear8& a, hipStream_t st) {
  const dim3 grid((unsigned)((a.N + 31) / 32), (unsigned)((a.M + 31) / 32));
  if (dtype == kBF16) SR_LAUNCH(linear8_kernel<bf16_t>, grid, dim3(64), 0, st, a);
  else SR_LAUNCH(linear8_kernel<float>, grid, dim3(64), 0, st, a);
  return hipGetLastError();
}

}  // namespace sr
