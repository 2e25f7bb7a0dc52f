// Rotary positions: every head of a row turns its channel pairs by the angles of the row's token (sr_rotary).
//
// A workgroup takes the rows of a few tokens.  Its threads first issue the loads of their channels, then form the
// cosines and sines of all pairs of these tokens (in LDS, once for all heads), then turn and store.  The angle is a
// 64-bit product, reduced to a quarter turn in 64 bits (a coordinate of 10^6 keeps 2^-33 of a turn), so that
// 32-bit polynomials of |r| <= pi/4 finish it to the rounding of fp32.
#include <algorithm>

#include "block_ops.h"

namespace sr {

namespace {

// (cos t, sin t): r = t - k pi/2 with pi/2 in two parts, Taylor polynomials of cos r and sin r, then the quadrant.  The first
// terms left out are 2^-32 of the cosine and 2^-28 of the sine at pi/4.  |t| <= kMaxRotAngle: k is the nearest number of quarter turns but
// for the rounding of t 2/pi, at most 2^-7 of one there, so |r| stays below 0.80; past 2^53 quarter turns r would be anything.
SR_DEV float2 turn_of(double t) {
  const double k = rint(t * 0.63661977236758134308);
  const double rd = fma(-k, 6.123233995736766036e-17, fma(-k, 1.57079632679489655800, t));
  const float r = (float)rd, z = r * r;
  float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(s, z, 8.3333333e-3f);
  s = fmaf(s, z, -1.6666667e-1f);
  s = fmaf(s * z, r, r);
  float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(c, z, -1.3888889e-3f);
  c = fmaf(c, z, 4.1666667e-2f);
  c = fmaf(c, z, -0.5f);
  c = fmaf(c, z, 1.0f);
  const int q = (int)(k - 4.0 * floor(k * 0.25));
  const float a = q & 1 ? s : c, b = q & 1 ? c : s;
  return float2{(q == 1 || q == 2) ? -a : a, q >= 2 ? -b : b};
}

constexpr int kThreads = 256, kUnroll = 2, kTokens = 16;   // 65536 x 1024 with two units a thread 50.8 us, four 52.7

// 16 bytes of channels.
template <typename T>
struct Vec16 {
  static constexpr int V = 16 / (int)sizeof(T);
  T v[V];
};

// What is left of i after whole d's, and their number; magic = ceil(2^32 / d), exact for i d < 2^32.
SR_DEV uint32_t quotient(uint32_t i, uint32_t magic, uint32_t d) { return d == 1 ? i : __umulhi(i, magic); }

struct Units {
  uint32_t tokens;    // of a workgroup, kTokens at most
  uint32_t per_head, per_token, rot;   // units of a head and of a row; those of a head that turn
  uint32_t magic_head, magic_token, magic_pairs;
};

// PAIRED: a unit turns V pairs, of channels c0 .. and c1 ..; otherwise V / 2 pairs of neighbours in V channels.  With
// WHOLE the last unit of a head's turning channels, and of those that do not turn, ends at the last of them; without, it may
// have fewer (16384 rows of 9 heads of 110 channels: 15 us, without 27).
template <typename T, bool PAIRED, bool WHOLE>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Rotary a, Units un) {
  extern __shared__ float2 cs[];   // [tokens][P]
  __shared__ double place[kTokens][3];
  typedef Vec16<T> Vec;
  constexpr int V = Vec::V;
  const int P = a.first[3];
  const int64_t rows = (int64_t)a.B * a.S, row0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (int64_t)un.tokens;
  const uint32_t n = un.tokens * un.per_token;
  auto get = [&](Vec& v, const T* p, int count) {
    if (WHOLE || count == V) {
      v = __builtin_bit_cast(Vec, load16(p));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v.v[j] = j < count ? p[j] : T{};
    }
  };
  auto put = [&](T* p, const Vec& v, int count) {
    if (WHOLE || count == V) {
      store16(p, __builtin_bit_cast(i32x4, v));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (j < count) p[j] = v.v[j];
    }
  };
  bool first = true;
  for (uint32_t base = 0; base < n || first; base += kThreads * kUnroll) {
    Vec lo[kUnroll], hi[kUnroll];
    int64_t oy[kUnroll];
    int count[kUnroll], at[kUnroll];   // channels of the unit (of one side, PAIRED); first pair in cs, -1: they do not turn, -2: nothing
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const uint32_t i = base + threadIdx.x + kThreads * k;
      const uint32_t t = quotient(i, un.magic_token, un.per_token), r = i - t * un.per_token;
      const uint32_t h = quotient(r, un.magic_head, un.per_head), u = r - h * un.per_head;
      at[k] = -2;
      if (i < n && row0 + t < rows) {
        int c0;
        if (u < un.rot) {
          constexpr int n_pairs = PAIRED ? V : V / 2;
          int p = (int)u * n_pairs;
          if (WHOLE) p = min(p, P - n_pairs);
          at[k] = (int)t * P + p;
          c0 = PAIRED ? p : 2 * p;
          count[k] = WHOLE ? V : min(V, PAIRED ? P - p : 2 * (P - p));
        } else {
          at[k] = -1;
          c0 = 2 * P + (int)(u - un.rot) * V;
          if (WHOLE) c0 = min(c0, a.hd - V);
          count[k] = WHOLE ? V : min(V, a.hd - c0);
        }
        const T* xp = (const T*)a.x + (row0 + t) * a.ldx + (int64_t)h * a.hd + c0;
        oy[k] = (row0 + t) * a.ldy + (int64_t)h * a.hd + c0;
        get(lo[k], xp, count[k]);
        if (PAIRED && at[k] >= 0) get(hi[k], xp + P, count[k]);
      }
    }
    if (first) {
      // the tokens' coordinates, then the turns of all their pairs
      if (threadIdx.x < un.tokens && row0 + threadIdx.x < rows) {
        const uint32_t row = (uint32_t)(row0 + threadIdx.x), b = row / (uint32_t)a.S, s = row - b * (uint32_t)a.S;
        uint32_t l = a.idx ? (uint32_t)a.idx[(size_t)(a.idx_shared ? 0 : b) * a.S + s] : s;
#pragma unroll
        for (int ax = 2; ax >= 0; --ax) {   // axes that there are not have one place
          const uint32_t g = (uint32_t)a.grid[ax], q = ax > 0 ? l / g : 0u;
          place[threadIdx.x][ax] = fma(a.step[ax], (double)(l - q * g), a.origin[ax]);
          l = q;
        }
      }
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < un.tokens * (uint32_t)P; i += kThreads) {
        const uint32_t t = quotient(i, un.magic_pairs, (uint32_t)P);
        const int p = (int)(i - t * (uint32_t)P), ax = (p >= a.first[1]) + (p >= a.first[2]);
        float2 c = turn_of(place[t][ax] * a.freq[p]);
        if (a.inverse) c.y = -c.y;
        cs[i] = c;
      }
      __syncthreads();
      first = false;
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      if (at[k] == -2) continue;
      T* yp = (T*)a.y + oy[k];
      if (at[k] >= 0) {
        if constexpr (PAIRED) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            if (!WHOLE && j >= count[k]) break;
            const float2 c = cs[at[k] + j];
            const float x0 = to_f32<T>(lo[k].v[j]), x1 = to_f32<T>(hi[k].v[j]);
            lo[k].v[j] = from_f32<T>(fmaf(x0, c.x, -x1 * c.y));
            hi[k].v[j] = from_f32<T>(fmaf(x1, c.x, x0 * c.y));
          }
          put(yp + P, hi[k], count[k]);
        } else {
#pragma unroll
          for (int j = 0; j < V / 2; ++j) {
            if (!WHOLE && 2 * j >= count[k]) break;
            const float2 c = cs[at[k] + j];
            const float x0 = to_f32<T>(lo[k].v[2 * j]), x1 = to_f32<T>(lo[k].v[2 * j + 1]);
            lo[k].v[2 * j] = from_f32<T>(fmaf(x0, c.x, -x1 * c.y));
            lo[k].v[2 * j + 1] = from_f32<T>(fmaf(x1, c.x, x0 * c.y));
          }
        }
      }
      put(yp, lo[k], count[k]);
    }
  }
}

template <typename T, bool PAIRED>
hipError_t run(const Rotary& a, hipStream_t st) {
  constexpr int V = Vec16<T>::V;
  const int P = a.first[3], turning = PAIRED ? P : 2 * P, rest = a.hd - 2 * P;
  Units un;
  un.rot = (uint32_t)((turning + V - 1) / V);
  const bool copies = a.x != a.y;   // in place the channels that do not turn stay
  un.per_head = un.rot + (copies ? (uint32_t)((rest + V - 1) / V) : 0);
  un.per_token = un.per_head * (uint32_t)a.heads;
  if (un.per_token == 0) return hipSuccess;
  // about kUnroll units a thread
  un.tokens = std::min((uint32_t)kTokens, std::max(1u, kThreads * kUnroll / un.per_token));
  un.magic_head = (uint32_t)(((1ull << 32) + un.per_head - 1) / un.per_head);
  un.magic_pairs = P ? (uint32_t)(((1ull << 32) + P - 1) / P) : 0;
  un.magic_token = (uint32_t)(((1ull << 32) + un.per_token - 1) / un.per_token);
  const int64_t rows = (int64_t)a.B * a.S, wgs = (rows + un.tokens - 1) / un.tokens;
  constexpr int64_t kMaxX = 1 << 22;   // 256 threads each: a launch counts threads along x in 32 bits
  const dim3 grid((unsigned)std::min(wgs, kMaxX), (unsigned)((wgs + kMaxX - 1) / kMaxX));
  const uint32_t lds = (uint32_t)(un.tokens * P * sizeof(float2));
  // a last unit that lies back over its neighbour stores the same values twice, which in place it may not
  const bool whole = copies ? (turning == 0 || turning >= V) && (rest == 0 || rest >= V) : turning % V == 0;
  if (whole) SR_LAUNCH((rotary_kernel<T, PAIRED, true>), grid, dim3(kThreads), lds, st, a, un);
  else SR_LAUNCH((rotary_kernel<T, PAIRED, false>), grid, dim3(kThreads), lds, st, a, un);
  return hipGetLastError();
}

template <typename T>
hipError_t run_type(const Rotary& a, hipStream_t st) {
  return a.neighbours ? run<T, false>(a, st) : run<T, true>(a, st);
}

}  // namespace

hipError_t launch_rotary(int dtype, const Rotary& a, hipStream_t st) {
  return dtype == kBF16 ? run_type<bf16_t>(a, st) : run_type<float>(a, st);
}

}  // namespace sr
