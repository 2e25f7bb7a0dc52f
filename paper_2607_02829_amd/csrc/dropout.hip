// Dropout with draws from a counter (sr_dropout): y = resid + keep x factor, the mask formed where it is used.
//
// Bound by memory; the generator costs two 64-bit products a word of four draws, under the loads.
#include <algorithm>

#include "block_ops.h"

namespace sr {

namespace {

constexpr int kThreads = 256;

template <typename T>
struct Eight {
  float v[8];
  SR_DEV void load(const T* p) {
    if constexpr (sizeof(T) == 2) {
      const i32x4 w = load16(p);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float((uint32_t)w[j] << 16);
        v[2 * j + 1] = __uint_as_float((uint32_t)w[j] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const f32x4 w = __builtin_bit_cast(f32x4, load16(p + 4 * j));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * j + i] = w[i];
      }
    }
  }
  SR_DEV void store(T* p) const {
    if constexpr (sizeof(T) == 2) {
      i32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = (int)f2bf2(v[2 * j], v[2 * j + 1]);
      store16(p, w);
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        store16(p + 4 * j, __builtin_bit_cast(i32x4, f32x4{v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]}));
    }
  }
};

// One draw per element: the tensor as one run of M N elements, eight to a thread and step.
template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(Dropout a) {
  const int64_t n = a.M * a.N, whole = n / 8;
  const uint64_t key = drop_key(a.drop), e0 = a.drop.first_row * (uint64_t)a.N;
  const T *x = (const T*)a.x, *r = (const T*)a.resid;
  T* y = (T*)a.y;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < whole; i += (int64_t)gridDim.x * kThreads) {
    Eight<T> v, w;
    v.load(x + 8 * i);
    if (r) w.load(r + 8 * i);
    const uint32_t keep = drop_keep8(key, e0 + 8 * (uint64_t)i, a.drop.thresh);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float t = keep >> j & 1u ? v.v[j] * a.drop.factor : 0.f;
      v.v[j] = r ? w.v[j] + t : t;
    }
    v.store(y + 8 * i);
  }
  const int64_t i = 8 * whole + threadIdx.x;
  if (blockIdx.x == 0 && i < n) {
    float t = drop_keep1(key, e0 + (uint64_t)i, a.drop.thresh) ? to_f32<T>(x[i]) * a.drop.factor : 0.f;
    if (r) t += to_f32<T>(r[i]);
    y[i] = from_f32<T>(t);
  }
}

// One draw per group of rows: a wave takes a row; of a dropped one x is not read.
template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_rows_kernel(Dropout a) {
  const uint64_t key = drop_key(a.drop);
  const int lane = threadIdx.x & 63;
  const int64_t step = (int64_t)gridDim.x * (kThreads / 64);
  for (int64_t row = (int64_t)blockIdx.x * (kThreads / 64) + wave_index(); row < a.M; row += step) {
    const bool keep = drop_keep1(key, (a.drop.first_row + (uint64_t)row) / (uint64_t)a.drop.group, a.drop.thresh);
    const T *x = (const T*)a.x + row * a.N, *r = a.resid ? (const T*)a.resid + row * a.N : nullptr;
    T* y = (T*)a.y + row * a.N;
    const int64_t whole = a.N / 8 * 8;
    for (int64_t c = 8 * lane; c < whole; c += 512) {
      Eight<T> v, w;
      if (keep) v.load(x + c);
      if (r) w.load(r + c);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float t = keep ? v.v[j] * a.drop.factor : 0.f;
        v.v[j] = r ? w.v[j] + t : t;
      }
      v.store(y + c);
    }
    for (int64_t c = whole + lane; c < a.N; c += 64) {
      const float t = keep ? to_f32<T>(x[c]) * a.drop.factor : 0.f;
      y[c] = from_f32<T>(r ? to_f32<T>(r[c]) + t : t);
    }
  }
}

template <typename T>
hipError_t run(const Dropout& a, hipStream_t st) {
  if (a.drop.group) {
    const int64_t wgs = std::min<int64_t>((a.M + 3) / 4, 1 << 16);
    SR_LAUNCH((dropout_rows_kernel<T>), dim3((unsigned)wgs), dim3(kThreads), 0, st, a);
  } else {
    const int64_t wgs = std::min<int64_t>(std::max<int64_t>((a.M * a.N / 8 + kThreads - 1) / kThreads, 1), 1 << 16);
    SR_LAUNCH((dropout_kernel<T>), dim3((unsigned)wgs), dim3(kThreads), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int dtype, const Dropout& a, hipStream_t st) {
  return dtype == kBF16 ? run<bf16_t>(a, st) : run<float>(a, st);
}

}  // namespace sr
