// Weight and bias gradient of a linear layer from the 8-bit checkpoint of its input:
//   dw[n, k] = sum_m dy[m, n] xhat[m, k],   db[n] = sum_m dy[m, n],   xhat = q 2^e (SR_Q8_BLOCK).
#include "common.h"
#include "quant8.h"
#include "sr_internal.h"

namespace sr {

namespace {

// 64 x 64 tiles of dw in fp32, 16 tokens at a time through LDS; the tiles of the first column of
// tiles also sum db.
template <typename T>
__global__ __launch_bounds__(256) void wgrad8_kernel(Wgrad8 a) {
  __shared__ float sy[16][64], sx[16][64];
  const int n0 = blockIdx.y * 64, k0 = blockIdx.x * 64, t = threadIdx.x;
  const int tn = (t >> 4) * 4, tk = (t & 15) * 4;
  float acc[4][4] = {}, sum = 0.f;
  for (int m0 = 0; m0 < a.M; m0 += 16) {
    for (int i = t; i < 1024; i += 256) {
      const int m = m0 + (i >> 6), c = i & 63;
      const bool in = m < a.M;
      sy[i >> 6][c] = in && n0 + c < a.N ? to_f32<T>(((const T*)a.dy)[(size_t)m * a.N + n0 + c]) : 0.f;
      const size_t o = (size_t)m * a.K + k0 + c;
      sx[i >> 6][c] = in ? (float)a.xq[o] * block_scale(a.xe[o / kQBlock]) : 0.f;
    }
    __syncthreads();
#pragma unroll 4
    for (int m = 0; m < 16; ++m) {
      const f32x4 y = *reinterpret_cast<const f32x4*>(&sy[m][tn]), x = *reinterpret_cast<const f32x4*>(&sx[m][tk]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(y[i], x[j], acc[i][j]);
      if (t < 64) sum += sy[m][t];
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n0 + tn + i < a.N) {
      const f32x4 v = {acc[i][0], acc[i][1], acc[i][2], acc[i][3]};
      *reinterpret_cast<f32x4*>(a.dw + (size_t)(n0 + tn + i) * a.K + k0 + tk) = v;
    }
  if (a.db && blockIdx.x == 0 && t < 64 && n0 + t < a.N) a.db[n0 + t] = sum;
}

}  // namespace

size_t wgrad8_scratch(int, int, int, int) { return 0; }

hipError_t launch_wgrad8(int dtype, const Wgrad8& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.K / 64), (unsigned)((a.N + 63) / 64));
  if (dtype == kBF16) SR_LAUNCH(wgrad8_kernel<bf16_t>, grid, dim3(256), 0, st, a);
  else SR_LAUNCH(wgrad8_kernel<float>, grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace sr
