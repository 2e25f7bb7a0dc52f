// The residual step between two branches (sr_residual_norm_fwd / _bwd): norm of the branch output, dropout, gate and
// residual scale, the sum, and the next branch's norm, in one pass over the rows per direction.
//
// A row lives in the registers of a team of LPR lanes, NV runs of eight channels each, so every tensor is read once and the
// deviations are summed from values whose mean is already taken off.  The backward keeps four column sums per
// channel in registers while its team walks the rows of one sample:
//   S1 = sum du,  S2 = sum du v,  S3 = sum d,  S4 = sum d n     v = Norm(x1), n = Norm(y) (or y), d = keep f (dx1 + ..)
// All parameters' gradients are combinations of these per sample (a second launch adds the workgroups' parts up in a
// fixed order):  dshift = S1, dscale = pre_w S2 + pre_b S1, dpre_w = sum_b (1 + scale) S2, dpre_b likewise of S1,
// with t = post_w S4 + post_b S3:  dgate = res_scale t, dres_scale = sum_b gate t, dpost_w = sum_b gate res_scale S4,
// dpost_b likewise of S3.
#include <algorithm>

#include "block_ops.h"

namespace sr {

namespace {

// Eight channels c .. c + 7 of a row of D as fp32; `fill` past the row, where the row is absent (!on) or p is NULL.
// vec: every such run starts on 16 bytes and lies inside the row or past it.
template <typename T>
SR_DEV void get8(const T* p, int c, int D, bool vec, bool on, float fill, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = fill;
  if (!on || !p || c >= D) return;
  p += c;
  if (!vec) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < D) v[j] = to_f32<T>(p[j]);
  } else if constexpr (sizeof(T) == 2) {
    const i32x4 w = *reinterpret_cast<const i32x4*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float((uint32_t)w[j] << 16);
      v[2 * j + 1] = __uint_as_float((uint32_t)w[j] & 0xFFFF0000u);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const f32x4 w = *reinterpret_cast<const f32x4*>(p + 4 * j);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * j + i] = w[i];
    }
  }
}
template <typename T>
SR_DEV void put8(T* p, int c, int D, bool vec, const float (&v)[8]) {
  if (c >= D) return;
  p += c;
  if (!vec) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < D) p[j] = from_f32<T>(v[j]);
  } else if constexpr (sizeof(T) == 2) {
    i32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (int)f2bf2(v[2 * j], v[2 * j + 1]);
    *reinterpret_cast<i32x4*>(p) = w;
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j)
      *reinterpret_cast<f32x4*>(p + 4 * j) = f32x4{v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
  }
}

// Sums over the LPR lanes of a team (16, 32 or 64 neighbouring lanes, or whole waves).
template <int LPR>
SR_DEV float lanes_sum(float v) {
  if constexpr (LPR >= 64) return wave_sum(v);
  v += dppf<0xB1>(v);
  v += dppf<0x4E>(v);
  v += dppf<0x141>(v);
  v += dppf<0x140>(v);
  if constexpr (LPR == 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

template <int LPR>
constexpr int threads_of() {
  return LPR > 256 ? LPR : 256;
}

// Two sums at once over a team.  Teams of several waves meet in LDS: the slots alternate, so that one barrier a sum
// is enough (a slot is written again only behind the other one's barrier).
template <int LPR>
struct TeamSum {
  static constexpr int W = LPR / 64;   // waves of a team (0: less than one)
  float (*slot)[2][16];
  int parity = 0;
  SR_DEV void operator()(float& a, float& b) {
    a = lanes_sum<LPR>(a);
    b = lanes_sum<LPR>(b);
    if constexpr (W > 1) {
      const int wave = wave_index(), first = wave / W * W;
      slot[parity][0][wave] = a;
      slot[parity][1][wave] = b;
      __syncthreads();
      a = b = 0.f;
#pragma unroll
      for (int k = 0; k < W; ++k) {
        a += slot[parity][0][first + k];
        b += slot[parity][1][first + k];
      }
      parity ^= 1;
    }
  }
  SR_DEV void operator()(float& a) {
    float b = 0.f;
    (*this)(a, b);
  }
};

// z -> Norm(z) in place, with the row's mean and reciprocal deviation; channels past D come out as zeros.
template <int LPR, int NV>
SR_DEV void norm_row(float (&z)[NV][8], const int (&c)[NV], int D, bool layer, float eps, TeamSum<LPR>& sum, float& mean,
                     float& rstd) {
  mean = 0.f;
  if (layer) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s += z[i][j];
    sum(s);
    mean = s / (float)D;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) z[i][j] = c[i] + j < D ? z[i][j] - mean : 0.f;
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) q = fmaf(z[i][j], z[i][j], q);
  sum(q);
  rstd = 1.0f / sqrtf(q / (float)D + eps);
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) z[i][j] *= rstd;
}

// Bit j: channel c + j of the row keeps its value.
SR_DEV uint32_t keep_of(const DropArgs& d, uint64_t key, int64_t row, int D, int c) {
  const uint64_t r = d.first_row + (uint64_t)row;
  if (d.group) return drop_keep1(key, r / (uint64_t)d.group, d.thresh) ? 0xFFu : 0u;
  return drop_keep8(key, r * (uint64_t)D + (uint64_t)c, d.thresh);
}

struct Flags {
  bool vec;      // rows of every tensor and the parameters start on 16 bytes
  bool modvec;   // gate, shift and scale too
};

template <typename T, typename X, int LPR, int NV>
__global__ __launch_bounds__(threads_of<LPR>()) void residual_norm_fwd_kernel(ResidualNorm a, Flags f) {
  constexpr int NT = threads_of<LPR>(), TEAMS = NT / LPR;
  __shared__ float slots[2][2][16];
  TeamSum<LPR> sum{slots};
  const int t = threadIdx.x % LPR, team = threadIdx.x / LPR, D = a.D;
  const int64_t M = (int64_t)a.B * a.S;
  const bool layer = a.norm == SR_NORM_LAYER, drops = a.y && a.drop.thresh;
  const uint64_t key = drops ? drop_key(a.drop) : 0;
  int c[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) c[i] = (i * LPR + t) * 8;

  for (int64_t row0 = (int64_t)blockIdx.x * TEAMS; row0 < M; row0 += (int64_t)gridDim.x * TEAMS) {
    const int64_t row = row0 + team;
    const bool on = row < M;
    const int64_t b = on ? row / a.S : 0;
    float x[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) get8<X>((const X*)a.x + row * D, c[i], D, f.vec, on, 0.f, x[i]);
    if (a.y) {
      float n[NV][8];
#pragma unroll
      for (int i = 0; i < NV; ++i) get8<T>((const T*)a.y + row * D, c[i], D, f.vec, on, 0.f, n[i]);
      if (a.post) {
        float mean, rstd;
        norm_row<LPR, NV>(n, c, D, layer, a.eps, sum, mean, rstd);
        if (a.stats && on && t == 0) {
          a.stats[row] = mean;
          a.stats[M + row] = rstd;
        }
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float w[8], bias[8], rs[8], g[8];
        get8<T>((const T*)a.w.post_w, c[i], D, f.vec, a.post, 1.f, w);
        get8<T>((const T*)a.w.post_b, c[i], D, f.vec, a.post, 0.f, bias);
        get8<T>((const T*)a.w.res_scale, c[i], D, f.vec, true, 1.f, rs);
        get8<float>(a.w.gate ? a.w.gate + b * a.mod_stride : nullptr, c[i], D, f.modvec, true, 1.f, g);
        const uint32_t keep = drops ? keep_of(a.drop, key, row, D, c[i]) : 0xFFu;
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float v = fmaf(n[i][j], w[j], bias[j]);
          v = keep >> j & 1u ? v * a.drop.factor : 0.f;
          o[j] = fmaf(g[j] * rs[j], v, x[i][j]);
        }
        if (on) put8<X>((X*)a.x1 + row * D, c[i], D, f.vec, o);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = c[i] + j < D ? to_f32<X>(from_f32<X>(o[j])) : 0.f;   // the next norm's input is what is kept
      }
    }
    if (!a.u && !a.uq) continue;
    float mean, rstd;
    norm_row<LPR, NV>(x, c, D, layer, a.eps, sum, mean, rstd);
    if (a.stats && on && t == 0) {
      a.stats[2 * M + row] = mean;
      a.stats[3 * M + row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float w[8], bias[8], sc[8], sh[8], o[8];
      get8<T>((const T*)a.w.pre_w, c[i], D, f.vec, true, 1.f, w);
      get8<T>((const T*)a.w.pre_b, c[i], D, f.vec, true, 0.f, bias);
      get8<float>(a.w.scale ? a.w.scale + b * a.mod_stride : nullptr, c[i], D, f.modvec, true, 0.f, sc);
      get8<float>(a.w.shift ? a.w.shift + b * a.mod_stride : nullptr, c[i], D, f.modvec, true, 0.f, sh);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = fmaf(fmaf(x[i][j], w[j], bias[j]), 1.f + sc[j], sh[j]);
      if (a.u && on) put8<T>((T*)a.u + row * D, c[i], D, f.vec, o);
      if (a.uq) {   // blocks of 128 channels: 16 neighbouring lanes
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (c[i] + j >= D) o[j] = 0.f;
          m = max(m, __float_as_uint(o[j]) & 0x7FFFFFFFu);
        }
        auto over = [&](auto ctl) {
          m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, decltype(ctl)::value, 0xF, 0xF, false));
        };
        over(IC<0xB1>{});
        over(IC<0x4E>{});
        over(IC<0x141>{});
        over(IC<0x140>{});
        const uint32_t E = f8_exponent(m);
        const float inv = f8_inverse(m, E);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = f8_clamp(o[j] * inv);
        const int Dp = (D + 127) / 128 * 128;
        if (on && c[i] < Dp) {
          i32x2 q;
          q[0] = (int)f8_code4(o[0], o[1], o[2], o[3]);
          q[1] = (int)f8_code4(o[4], o[5], o[6], o[7]);
          *reinterpret_cast<i32x2*>(a.uq + row * Dp + c[i]) = q;
          if ((t & 15) == 0) a.ue[(int64_t)(c[i] / 128) * ((M + 15) / 16 * 16) + row] = (uint8_t)E;
        }
      }
    }
  }
}

// Workgroup (b, k): rows k R .. of sample b; its part of the four column sums at part[((b chunks + k) 4 + i) D].
template <typename T, typename X, int LPR, int NV>
__global__ __launch_bounds__(threads_of<LPR>()) void residual_norm_bwd_kernel(ResidualNorm a, Flags f, int chunks) {
  constexpr int NT = threads_of<LPR>(), TEAMS = NT / LPR, COLS = LPR * NV * 8;
  __shared__ float slots[2][2][16];
  __shared__ float cols[TEAMS > 1 ? TEAMS : 1][TEAMS > 1 ? COLS : 1];
  TeamSum<LPR> sum{slots};
  const int t = threadIdx.x % LPR, team = threadIdx.x / LPR, D = a.D;
  const int64_t M = (int64_t)a.B * a.S;
  const int b = (int)(blockIdx.x / (unsigned)chunks), k = (int)(blockIdx.x - (unsigned)b * (unsigned)chunks);
  const int R = (a.S + chunks - 1) / chunks, s0 = (int)min((long)k * R, (long)a.S), s1 = min(a.S - s0, R) + s0;
  const bool layer = a.norm == SR_NORM_LAYER, drops = a.y && a.drop.thresh;
  const uint64_t key = drops ? drop_key(a.drop) : 0;
  const float rD = 1.0f / (float)D;
  int c[NV];
  float acc[4][NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    c[i] = (i * LPR + t) * 8;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[q][i][j] = 0.f;
  }

  for (int sb = s0; sb < s1; sb += TEAMS) {
    const int s = sb + team;
    const bool on = s < s1;
    const int64_t row = (int64_t)b * a.S + (on ? s : s0);
    float dx[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) get8<X>((const X*)a.dx1 + (a.dx1 ? row * D : 0), c[i], D, f.vec, on, 0.f, dx[i]);
    if (a.du) {
      float v[NV][8], g[NV][8], c1 = 0.f, c2 = 0.f;
      const float mean = layer ? a.stats[2 * M + row] : 0.f, rstd = a.stats[3 * M + row];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        float w[8], sc[8];
        get8<X>((const X*)a.x + row * D, c[i], D, f.vec, on, mean, v[i]);
        get8<T>((const T*)a.du + row * D, c[i], D, f.vec, on, 0.f, g[i]);
        get8<T>((const T*)a.w.pre_w, c[i], D, f.vec, true, 1.f, w);
        get8<float>(a.w.scale ? a.w.scale + b * a.mod_stride : nullptr, c[i], D, f.modvec, true, 0.f, sc);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[i][j] = (v[i][j] - mean) * rstd;
          acc[0][i][j] += g[i][j];
          acc[1][i][j] = on ? fmaf(g[i][j], v[i][j], acc[1][i][j]) : acc[1][i][j];
          g[i][j] *= (1.f + sc[j]) * w[j];
          c1 += g[i][j];
          c2 = fmaf(g[i][j], v[i][j], c2);
        }
      }
      sum(c1, c2);
      c1 = layer ? c1 * rD : 0.f;
      c2 *= rD;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dx[i][j] = fmaf(rstd, g[i][j] - fmaf(v[i][j], c2, c1), dx[i][j]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (on) put8<X>((X*)a.dx + row * D, c[i], D, f.vec, dx[i]);
    if (!a.y) continue;
    float n[NV][8], g[NV][8], c1 = 0.f, c2 = 0.f, mean = 0.f, rstd = 1.f;
    if (a.post) {
      if (layer) mean = a.stats[row];
      rstd = a.stats[M + row];
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float w[8], rs[8], gt[8];
      get8<T>((const T*)a.y + row * D, c[i], D, f.vec, on, mean, n[i]);
      get8<T>((const T*)a.w.post_w, c[i], D, f.vec, a.post, 1.f, w);
      get8<T>((const T*)a.w.res_scale, c[i], D, f.vec, true, 1.f, rs);
      get8<float>(a.w.gate ? a.w.gate + b * a.mod_stride : nullptr, c[i], D, f.modvec, true, 1.f, gt);
      const uint32_t keep = drops ? keep_of(a.drop, key, row, D, c[i]) : 0xFFu;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        n[i][j] = (n[i][j] - mean) * rstd;
        const float d = on && c[i] + j < D && (keep >> j & 1u) ? dx[i][j] * a.drop.factor : 0.f;
        acc[2][i][j] += d;
        // a dropped value does not count, not even a NaN
        acc[3][i][j] = on && (keep >> j & 1u) ? fmaf(d, n[i][j], acc[3][i][j]) : acc[3][i][j];
        g[i][j] = d * (gt[j] * rs[j]) * w[j];
        c1 += g[i][j];
        c2 = fmaf(g[i][j], n[i][j], c2);
      }
    }
    if (a.post) {
      sum(c1, c2);
      c1 = layer ? c1 * rD : 0.f;
      c2 *= rD;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) g[i][j] = rstd * (g[i][j] - fmaf(n[i][j], c2, c1));
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (on) put8<T>((T*)a.dy + row * D, c[i], D, f.vec, g[i]);
  }

  float* part = a.part + (size_t)blockIdx.x * 4 * D;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (TEAMS == 1) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c[i] + j < D) part[(size_t)q * D + c[i] + j] = acc[q][i][j];
    } else {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) cols[team][c[i] + j] = acc[q][i][j];
      __syncthreads();
      for (int d = threadIdx.x; d < D; d += NT) {
        float s = 0.f;
#pragma unroll
        for (int k2 = 0; k2 < TEAMS; ++k2) s += cols[k2][d];
        part[(size_t)q * D + d] = s;
      }
    }
  }
}

// The workgroups' parts to the gradients.  A workgroup takes 32 channels and one of the two pairs of sums: thread (g, d)
// adds the parts g, g + 8, .. of channel d, the eight groups meet in LDS, and the first one goes on with the sample.
template <typename T>
__global__ __launch_bounds__(256) void residual_norm_grads_kernel(ResidualNorm a, int chunks) {
  constexpr int G = 8;
  __shared__ float sm[2][G][32];
  const int dl = threadIdx.x & 31, g = threadIdx.x >> 5, D = a.D, d = blockIdx.x * 32 + dl, pair = blockIdx.y;
  const bool in = d < D;
  auto w = [&](const void* p, float fill) { return p && in ? to_f32<T>(((const T*)p)[d]) : fill; };
  const float pre_w = w(a.w.pre_w, 1.f), pre_b = w(a.w.pre_b, 0.f), rs = w(a.w.res_scale, 1.f);
  const float post_w = w(a.post ? a.w.post_w : nullptr, 1.f), post_b = w(a.post ? a.w.post_b : nullptr, 0.f);
  float tw = 0.f, tb = 0.f, tr = 0.f;
  for (int b = 0; b < a.B; ++b) {
    float s0 = 0.f, s1 = 0.f;
    if (in)
      for (int k = g; k < chunks; k += G) {
        const float* p = a.part + (((size_t)b * chunks + k) * 4 + 2 * pair) * D + d;
        s0 += p[0];
        s1 += p[D];
      }
    sm[0][g][dl] = s0;
    sm[1][g][dl] = s1;
    __syncthreads();
    if (g == 0 && in) {
      s0 = s1 = 0.f;
#pragma unroll
      for (int k = 0; k < G; ++k) {
        s0 += sm[0][k][dl];
        s1 += sm[1][k][dl];
      }
      const size_t o = (size_t)b * D + d, om = (size_t)b * a.mod_stride + d;
      if (pair == 0) {
        const float sc = 1.f + (a.w.scale ? a.w.scale[om] : 0.f);
        if (a.g.shift) a.g.shift[o] = s0;
        if (a.g.scale) a.g.scale[o] = fmaf(pre_w, s1, pre_b * s0);
        tb = fmaf(sc, s0, tb);
        tw = fmaf(sc, s1, tw);
      } else {
        const float gt = a.w.gate ? a.w.gate[om] : 1.f, v = fmaf(post_w, s1, post_b * s0);
        if (a.g.gate) a.g.gate[o] = rs * v;
        tr = fmaf(gt, v, tr);
        tb = fmaf(gt * rs, s0, tb);
        tw = fmaf(gt * rs, s1, tw);
      }
    }
    __syncthreads();
  }
  if (g == 0 && in) {
    if (pair == 0) {
      if (a.g.pre_w) a.g.pre_w[d] = tw;
      if (a.g.pre_b) a.g.pre_b[d] = tb;
    } else {
      if (a.g.post_w) a.g.post_w[d] = a.post ? tw : 0.f;
      if (a.g.post_b) a.g.post_b[d] = a.post ? tb : 0.f;
      if (a.g.res_scale) a.g.res_scale[d] = tr;
    }
  }
}

int lanes_of(int D) { return D <= 128 ? 16 : D <= 256 ? 32 : D <= 1024 ? 64 : D <= 2048 ? 128 : D <= 4096 ? 256 : 512; }

// Workgroups of the backward per sample: about 1024 in all, four rows or more to a team.
int chunks_of(int B, int S, int D) {
  const int lpr = lanes_of(D), teams = (lpr > 256 ? lpr : 256) / lpr;
  const int64_t most = std::max<int64_t>(1, ((int64_t)S + 4 * teams - 1) / (4 * teams));
  return (int)std::min<int64_t>(most, std::max<int64_t>(1, 1024 / B));
}

Flags flags_of(const ResidualNorm& a) {
  auto al = [](const void* p) { return ((uintptr_t)p & 15) == 0; };
  Flags f;
  f.vec = a.D % 8 == 0;   // the tensors themselves start on 16 bytes
  f.modvec = f.vec && al(a.w.gate) && al(a.w.shift) && al(a.w.scale) && a.mod_stride % 4 == 0;
  return f;
}

template <typename T, typename X, int LPR, int NV>
hipError_t run_rows(const ResidualNorm& a, bool bwd, hipStream_t st) {
  constexpr int NT = threads_of<LPR>(), TEAMS = NT / LPR;
  if (!bwd) {
    const int64_t M = (int64_t)a.B * a.S, wgs = std::min<int64_t>((M + TEAMS - 1) / TEAMS, 1 << 16);
    SR_LAUNCH((residual_norm_fwd_kernel<T, X, LPR, NV>), dim3((unsigned)wgs), dim3(NT), 0, st, a, flags_of(a));
  } else {
    const int chunks = chunks_of(a.B, a.S, a.D);
    SR_LAUNCH((residual_norm_bwd_kernel<T, X, LPR, NV>), dim3((unsigned)a.B * (unsigned)chunks), dim3(NT), 0, st, a,
              flags_of(a), chunks);
  }
  return hipGetLastError();
}

template <typename T, typename X>
hipError_t run(const ResidualNorm& a, bool bwd, hipStream_t st) {
  switch (lanes_of(a.D)) {
    case 16: return run_rows<T, X, 16, 1>(a, bwd, st);
    case 32: return run_rows<T, X, 32, 1>(a, bwd, st);
    case 64: return a.D <= 512 ? run_rows<T, X, 64, 1>(a, bwd, st) : run_rows<T, X, 64, 2>(a, bwd, st);
    case 128: return run_rows<T, X, 128, 2>(a, bwd, st);
    case 256: return run_rows<T, X, 256, 2>(a, bwd, st);
    default: return run_rows<T, X, 512, 2>(a, bwd, st);
  }
}

hipError_t run_types(int dtype, int stream_dtype, const ResidualNorm& a, bool bwd, hipStream_t st) {
  if (dtype == kF32) return run<float, float>(a, bwd, st);
  return stream_dtype == kF32 ? run<bf16_t, float>(a, bwd, st) : run<bf16_t, bf16_t>(a, bwd, st);
}

}  // namespace

size_t residual_norm_scratch(int B, int S, int D) { return (size_t)B * chunks_of(B, S, D) * 4 * D * sizeof(float); }

hipError_t launch_residual_norm_fwd(int dtype, int stream_dtype, const ResidualNorm& a, hipStream_t st) {
  return run_types(dtype, stream_dtype, a, false, st);
}

hipError_t launch_residual_norm_bwd(int dtype, int stream_dtype, const ResidualNorm& a, hipStream_t st) {
  hipError_t e = run_types(dtype, stream_dtype, a, true, st);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)((a.D + 31) / 32), 2);
  const int chunks = chunks_of(a.B, a.S, a.D);
  if (dtype == kBF16) SR_LAUNCH((residual_norm_grads_kernel<bf16_t>), grid, dim3(256), 0, st, a, chunks);
  else SR_LAUNCH((residual_norm_grads_kernel<float>), grid, dim3(256), 0, st, a, chunks);
  return hipGetLastError();
}

}  // namespace sr
