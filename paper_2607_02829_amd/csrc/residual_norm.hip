// The residual step between two branches (sr_residual_norm_fwd / _bwd): norm of the branch output, dropout, gate and
// residual scale, the sum, and the next branch's norm, in one pass over the rows per direction.
//
// A row lives in the registers of a team of LPR lanes, NV runs of four channels each, so every tensor is read once and the
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

// Rows of a tensor as a raw buffer: the rows of a workgroup's teams from `row` on, `rows` of them.  What lies past them, or
// past a row (kPast), reads as zero and is not written, so neither needs a branch; a NULL tensor has no rows.
constexpr uint32_t kPast = 0x20000000u;   // in elements: 2^30 bytes or 2^31
template <typename T>
SR_DEV __amdgpu_buffer_rsrc_t rows_of(const void* p, int64_t row, int rows, int D) {
  return make_rsrc((const T*)p + row * D, p ? (uint32_t)rows * (uint32_t)D * (uint32_t)sizeof(T) : 0u);
}

// How a row is cut into runs of four channels.  kWhole: D is a multiple of four.  kShifted: the last run starts at D - 4
// instead, so that every load is whole (buffer accesses need no alignment here); its first channels belong to the run
// before, count there and are left out here.  kSingle: D < 4, channel by channel.
enum Cut { kWhole, kShifted, kSingle };

// A thread's runs: offset from a workgroup's first row (kPast: none), first channel, and which of the four are its own.
template <int LPR, int NV, int CUT>
struct Place {
  uint32_t off[NV];
  int t, D;
  uint32_t row;
  SR_DEV Place(int t_, int team, int D_) : t(t_), D(D_), row((uint32_t)(team * D_)) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int k = natural(i);
      off[i] = k < D ? row + (uint32_t)(CUT == kShifted ? min(k, D - 4) : k) : kPast;
    }
  }
  SR_DEV int natural(int i) const { return (i * LPR + t) * 4; }
  SR_DEV uint32_t c(int i) const { return off[i] - row; }   // D or more where there is none
  SR_DEV int lo(int i) const { return CUT == kShifted ? natural(i) - (int)c(i) : 0; }
  SR_DEV int hi(int i) const { return CUT == kSingle ? D - natural(i) : 4; }
  SR_DEV bool own(int i, int j) const {
    if constexpr (CUT == kWhole) return off[i] < kPast;
    if constexpr (CUT == kShifted) return off[i] < kPast && j >= lo(i);
    return j < hi(i);
  }
};

// Four channels as they lie in memory, so that they can be on their way while the row before is computed.
template <typename T, int CUT>
struct Four;
template <int CUT>
struct Four<float, CUT> {
  f32x4 r;
  SR_DEV void load(__amdgpu_buffer_rsrc_t b, uint32_t off, int hi) {
    if constexpr (CUT != kSingle) {
      r = __builtin_bit_cast(f32x4, buf_load16(b, off * 4));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        r[j] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(b, (j < hi ? off + j : kPast) * 4, 0, 0));
    }
  }
  SR_DEV void fill(float v) { r = f32x4{v, v, v, v}; }
  SR_DEV float at(int j) const { return r[j]; }
};
template <int CUT>
struct Four<bf16_t, CUT> {
  i32x2 r;
  SR_DEV void load(__amdgpu_buffer_rsrc_t b, uint32_t off, int hi) {
    if constexpr (CUT != kSingle) {
      r = buf_load8(b, off * 2);
    } else {
      uint32_t h[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        h[j] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(b, (j < hi ? off + j : kPast) * 2, 0, 0);
      r = i32x2{(int)(h[0] | h[1] << 16), (int)(h[2] | h[3] << 16)};
    }
  }
  SR_DEV void fill(float v) {
    const int f = (int)f2bf2(v, v);
    r = i32x2{f, f};
  }
  SR_DEV float at(int j) const { return __uint_as_float(j & 1 ? (uint32_t)r[j / 2] & 0xFFFF0000u : (uint32_t)r[j / 2] << 16); }
};
// past: past the caches.
constexpr int kPastCaches = 2;   // the buffer instructions' non-temporal bit
template <typename T, int CUT>
SR_DEV void put4(__amdgpu_buffer_rsrc_t b, uint32_t off, int lo, int hi, const float (&v)[4], bool past = false) {
  if (CUT == kWhole || (CUT == kShifted && lo == 0)) {
    if constexpr (sizeof(T) == 2) {
      const i32x2 w = {(int)f2bf2(v[0], v[1]), (int)f2bf2(v[2], v[3])};
      if (past) __builtin_amdgcn_raw_buffer_store_b64(w, b, off * 2, 0, kPastCaches);
      else __builtin_amdgcn_raw_buffer_store_b64(w, b, off * 2, 0, 0);
    } else {
      const i32x4 w = __builtin_bit_cast(i32x4, f32x4{v[0], v[1], v[2], v[3]});
      if (past) __builtin_amdgcn_raw_buffer_store_b128(w, b, off * 4, 0, kPastCaches);
      else __builtin_amdgcn_raw_buffer_store_b128(w, b, off * 4, 0, 0);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t o = (j >= lo && j < hi ? off + j : kPast) * (uint32_t)sizeof(T);
      if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16((short)f2bf(v[j]), b, o, 0, 0);
      else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(int, v[j]), b, o, 0, 0);
    }
  }
}
// A parameter's channels ([D], or a sample's row of it), `fill` where it is NULL.
template <typename T, int CUT>
SR_DEV Four<T, CUT> param4(const void* p, int D, uint32_t c, int hi, float fill) {
  Four<T, CUT> v;
  if (p) v.load(rows_of<T>(p, 0, 1, D), c, hi);
  else v.fill(fill);
  return v;
}

// Sums over the LPR lanes of a team (32 neighbouring lanes, or whole waves).
template <int LPR>
SR_DEV float lanes_sum(float v) {
  if constexpr (LPR >= 64) return wave_sum(v);
  v += dppf<0xB1>(v);
  v += dppf<0x4E>(v);
  v += dppf<0x141>(v);
  v += dppf<0x140>(v);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Threads of a workgroup.  The backward's holds twice as many teams of up to a wave, whose column sums leave as one part (16200 x
// 1024 with the join 72.7 -> 70.5 us); teams of several waves meet at barriers, where more of them wait for each other (4 x 1000 x
// 4096: 76 us, with twice as many 89).
constexpr int fwd_threads(int lpr) { return lpr > 256 ? lpr : 256; }
constexpr int bwd_threads(int lpr) { return lpr <= 64 || lpr > 256 ? 512 : 256; }

// N sums at once over a team, of the sum of a thread's runs: the runs that lie CL lanes apart are added up first, in their order
// (add_run), then the lanes of a wave, then the waves.  CL follows D alone, so a row has the same sums, bit for bit, on a team of CL lanes with NV
// runs and on one with a lane for every run (NV = 1), whose runs meet in LDS.  Several waves meet there too: the slots
// alternate, so that one barrier a sum is enough (a slot is written again only behind the other one's barrier).
constexpr int lanes_apart(int lpr, int nv) { return nv > 1 || lpr <= 64 ? lpr : lpr == 512 ? 128 : 64; }
SR_DEV void add_run(float& all, int i, float run) { all = i ? all + run : run; }
template <int LPR, int NV>
struct TeamSum {
  static constexpr int CL = lanes_apart(LPR, NV), W = LPR / 64;   // waves of a team (0: less than one)
  static constexpr int SLOTS = CL < LPR ? 512 : 16;
  float (*slot)[2][SLOTS];
  int team, parity = 0;
  template <int N>
  SR_DEV void operator()(float (&q)[N]) {
    if constexpr (CL < LPR) {
      const int t = threadIdx.x % LPR;
#pragma unroll
      for (int n = 0; n < N; ++n) slot[parity][n][team * LPR + t] = q[n];
      __syncthreads();
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float* at = slot[parity][n] + team * LPR + (t & 63);
        q[n] = 0.f;
#pragma unroll
        for (int w = 0; w < CL / 64; ++w) {
          float s = at[64 * w];
#pragma unroll
          for (int i = 1; i < LPR / CL; ++i) s += at[64 * w + CL * i];
          q[n] += wave_sum(s);
        }
      }
      parity ^= 1;
    } else {
#pragma unroll
      for (int n = 0; n < N; ++n) q[n] = lanes_sum<LPR>(q[n]);
      if constexpr (W > 1) {
        const int wave = wave_index(), first = wave / W * W;
#pragma unroll
        for (int n = 0; n < N; ++n) slot[parity][n][wave] = q[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
          q[n] = 0.f;
#pragma unroll
          for (int k = 0; k < W; ++k) q[n] += slot[parity][n][first + k];
        }
        parity ^= 1;
      }
    }
  }
};

// z -> Norm(z) in place, with the row's mean and reciprocal deviation; channels past D come out as zeros.
template <int LPR, int NV, int CUT>
SR_DEV void norm_row(float (&z)[NV][4], const Place<LPR, NV, CUT>& at, float rD, bool layer, float eps, TeamSum<LPR, NV>& sum,
                     float& mean, float& rstd) {
#pragma clang fp contract(off)
  mean = 0.f;
  if (layer) {
    float s[1];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float r = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) r += z[i][j];
      add_run(s[0], i, r);
    }
    sum(s);
    mean = s[0] * rD;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) z[i][j] = at.own(i, j) ? z[i][j] - mean : 0.f;
  }
  float q[1];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float r = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) r = fmaf(z[i][j], z[i][j], r);
    add_run(q[0], i, r);
  }
  sum(q);
  rstd = 1.0f / sqrtf(fmaf(q[0], rD, eps));
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) z[i][j] *= rstd;
}

// Rows of part k of a sample's S, cut into `chunks` parts.  Unsigned: S and the parts' number pass 2^31 together, and so does the
// row that a team is to take next.  (chunks - 1) R < S + chunks stays below 2^32.
struct Rows {
  uint32_t begin, end;
};
SR_DEV Rows rows_of_part(int S, int chunks, int k) {
  const uint32_t n = (uint32_t)S, R = (n + (uint32_t)chunks - 1) / (uint32_t)chunks, begin = min((uint32_t)k * R, n);
  return {begin, begin + min(n - begin, R)};
}

// Bit j: channel c + j of the row keeps its value.
SR_DEV uint32_t keep_of(const DropArgs& d, uint64_t key, int64_t row, int D, int c) {
  const uint64_t r = d.first_row + (uint64_t)row;
  if (d.group) return drop_keep1(key, r / (uint64_t)d.group, d.thresh) ? 0xFu : 0u;
  return drop_keep4(key, r * (uint64_t)D + (uint64_t)c, d.thresh);
}

// Workgroup (b, k): rows k R .. of sample b, a team every TEAMS-th of them; the next row's values are on their way while
// one is computed.  A sample's parameters become one factor and one summand per channel and norm:
//   x1 = x + keep (n w1 + b1),  w1 = f gate res_scale post_w, b1 alike;   u = v w2 + b2,  w2 = (1 + scale) pre_w, ..
template <typename T, typename X, int LPR, int NV, int CUT>
__global__ __launch_bounds__(fwd_threads(LPR)) void residual_norm_fwd_kernel(ResidualNorm a, int chunks) {
#pragma clang fp contract(off)   // a row's bits do not depend on the team that takes it: every fma is written out
  constexpr int NT = fwd_threads(LPR), TEAMS = NT / LPR;
  __shared__ float slots[2][2][TeamSum<LPR, NV>::SLOTS];
  const int t = threadIdx.x % LPR, team = LPR < 64 ? (int)threadIdx.x / LPR : wave_index() / (LPR / 64 > 0 ? LPR / 64 : 1), D = a.D;
  TeamSum<LPR, NV> sum{slots, team};
  const int64_t M = (int64_t)a.B * a.S;
  const int b = (int)(blockIdx.x / (unsigned)chunks), k = (int)(blockIdx.x - (unsigned)b * (unsigned)chunks);
  const Rows mine = rows_of_part(a.S, chunks, k);
  const uint32_t s0 = mine.begin, s1 = mine.end;
  const bool layer = a.norm == SR_NORM_LAYER, drops = a.y && a.drop.thresh, next = a.u || a.uq;
  // x1 stays in the caches where a backward is to read it (16200 x 1024, both directions: 96 us, with x1 past them 103; forward alone 41, 38)
  const bool past = CUT == kWhole && past_caches(M, D, sizeof(T)), past_x1 = past && !a.stats;
  const float rD = 1.0f / (float)D;
  const Place<LPR, NV, CUT> at(t, team, D);
  Four<X, CUT> xr[NV];
  Four<T, CUT> yr[NV];
  auto load = [&](uint32_t sb) {
    const int rows = (int)min((uint32_t)TEAMS, s1 - sb);
    const int64_t row0 = (int64_t)b * a.S + sb;
    const __amdgpu_buffer_rsrc_t bx = rows_of<X>(a.x, row0, rows, D), by = rows_of<T>(a.y, row0, rows, D);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      xr[i].load(bx, at.off[i], at.hi(i));
      yr[i].load(by, at.off[i], at.hi(i));
    }
  };
  if (s0 < s1) load(s0);
  const uint64_t key = drops ? drop_key(a.drop) : 0;
  float w1[NV][4], b1[NV][4], w2[NV][4], b2[NV][4];
  {
    auto mod = [&](const float* p) { return p ? p + b * a.mod_stride : nullptr; };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t c = at.c(i);
      const int left = at.hi(i);
      const Four<T, CUT> pw = param4<T, CUT>(a.post ? a.w.post_w : nullptr, D, c, left, 1.f);
      const Four<T, CUT> pb = param4<T, CUT>(a.post ? a.w.post_b : nullptr, D, c, left, 0.f);
      const Four<T, CUT> rs = param4<T, CUT>(a.w.res_scale, D, c, left, 1.f);
      const Four<T, CUT> nw = param4<T, CUT>(a.w.pre_w, D, c, left, 1.f), nb = param4<T, CUT>(a.w.pre_b, D, c, left, 0.f);
      const Four<float, CUT> g = param4<float, CUT>(mod(a.w.gate), D, c, left, 1.f);
      const Four<float, CUT> sc = param4<float, CUT>(mod(a.w.scale), D, c, left, 0.f);
      const Four<float, CUT> sh = param4<float, CUT>(mod(a.w.shift), D, c, left, 0.f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float ga = g.at(j) * rs.at(j) * a.drop.factor;
        w1[i][j] = ga * pw.at(j);
        b1[i][j] = ga * pb.at(j);
        w2[i][j] = (1.f + sc.at(j)) * nw.at(j);
        b2[i][j] = fmaf(1.f + sc.at(j), nb.at(j), sh.at(j));
      }
    }
  }

  for (uint32_t sb = s0; sb < s1; sb += TEAMS) {
    const int rows = (int)min((uint32_t)TEAMS, s1 - sb);
    const int64_t row0 = (int64_t)b * a.S + sb, row = row0 + team;
    const bool on = team < rows;
    float x[NV][4], n[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i][j] = CUT != kShifted || at.own(i, j) ? xr[i].at(j) : 0.f;
        n[i][j] = CUT != kShifted || at.own(i, j) ? yr[i].at(j) : 0.f;
      }
    if (sb + TEAMS < s1) load(sb + TEAMS);
    if (a.y) {
      if (a.post) {
        float mean, rstd;
        norm_row(n, at, rD, layer, a.eps, sum, mean, rstd);
        if (a.stats && on && t == 0) {
          a.stats[row] = mean;
          a.stats[M + row] = rstd;
        }
      }
      const __amdgpu_buffer_rsrc_t bx1 = rows_of<X>(a.x1, row0, rows, D);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const uint32_t keep = drops ? keep_of(a.drop, key, row, D, (int)at.c(i)) : 0xFu;
        float o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = x[i][j] + (keep >> j & 1u ? fmaf(n[i][j], w1[i][j], b1[i][j]) : 0.f);
        put4<X, CUT>(bx1, at.off[i], at.lo(i), at.hi(i), o, past_x1);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[i][j] = at.own(i, j) ? to_f32<X>(from_f32<X>(o[j])) : 0.f;   // the next norm's input is what is kept
      }
    }
    if (!next) continue;
    float mean, rstd;
    norm_row(x, at, rD, layer, a.eps, sum, mean, rstd);
    if (a.stats && on && t == 0) {
      a.stats[2 * M + row] = mean;
      a.stats[3 * M + row] = rstd;
    }
    const __amdgpu_buffer_rsrc_t bu = rows_of<T>(a.u, row0, rows, D);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = fmaf(x[i][j], w2[i][j], b2[i][j]);
      put4<T, CUT>(bu, at.off[i], at.lo(i), at.hi(i), o, past);
      if (a.uq) {   // blocks of 128 channels: 32 neighbouring lanes
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (!at.own(i, j)) o[j] = 0.f;
          m = max(m, __float_as_uint(o[j]) & 0x7FFFFFFFu);
        }
        auto over = [&](auto ctl) {
          m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, decltype(ctl)::value, 0xF, 0xF, false));
        };
        over(IC<0xB1>{});
        over(IC<0x4E>{});
        over(IC<0x141>{});
        over(IC<0x140>{});
        const auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
        m = max(r[0], r[1]);
        const uint32_t E = f8_exponent(m);
        const float inv = at.off[i] < kPast ? f8_inverse(m, E) : 0.f;   // codes past D are zeros in any block
        const int Dp = (D + 127) / 128 * 128, ch = (i * LPR + t) * 4;
        if (on && ch < Dp) {
          uint32_t q = f8_code4(f8_clamp(o[0] * inv), f8_clamp(o[1] * inv), f8_clamp(o[2] * inv), f8_clamp(o[3] * inv));
          if (CUT == kShifted && ch < D) q >>= 8 * at.lo(i);
          if constexpr (CUT == kSingle) q = f8_first(q, D - ch);
          *reinterpret_cast<uint32_t*>(a.uq + row * Dp + ch) = q;
          if ((t & 31) == 0) a.ue[(int64_t)(ch / 128) * ((M + 15) / 16 * 16) + row] = (uint8_t)E;
        }
      }
    }
  }
}

// Workgroup (b, k): rows k R .. of sample b; its part of the four column sums at part[((b chunks + k) 4 + i) D].  As in
// the forward the next row is on its way while a row is computed.  Rows and channels that are not there read as zeros in
// every tensor and statistic, and add nothing.
template <typename T, typename X, int LPR, int NV, int CUT>
__global__ __launch_bounds__(bwd_threads(LPR), 2) void residual_norm_bwd_kernel(ResidualNorm a, int chunks) {
#pragma clang fp contract(off)   // as in the forward
  constexpr int NT = bwd_threads(LPR), TEAMS = NT / LPR, COLS = LPR * NV * 4;
  __shared__ float slots[2][2][TeamSum<LPR, NV>::SLOTS];
  __shared__ __attribute__((aligned(16))) float cols[TEAMS > 1 ? TEAMS : 1][TEAMS > 1 ? COLS : 4];
  const int t = threadIdx.x % LPR, team = LPR < 64 ? (int)threadIdx.x / LPR : wave_index() / (LPR / 64 > 0 ? LPR / 64 : 1), D = a.D;
  TeamSum<LPR, NV> sum{slots, team};
  const int64_t M = (int64_t)a.B * a.S;
  const int b = (int)(blockIdx.x / (unsigned)chunks), k = (int)(blockIdx.x - (unsigned)b * (unsigned)chunks);
  const Rows mine = rows_of_part(a.S, chunks, k);
  const uint32_t s0 = mine.begin, s1 = mine.end;
  const bool layer = a.norm == SR_NORM_LAYER, drops = a.y && a.drop.thresh;
  const bool past = CUT == kWhole && past_caches(M, D, sizeof(T));
  const uint64_t key = drops ? drop_key(a.drop) : 0;
  const float rD = 1.0f / (float)D;
  const Place<LPR, NV, CUT> at(t, team, D);
  float acc[4][NV][4], wpre[NV][4], wpost[NV][4];   // sums; (1 + scale) pre_w and gate res_scale post_w of the sample
  {
    const float *scale = a.w.scale ? a.w.scale + b * a.mod_stride : nullptr, *gate = a.w.gate ? a.w.gate + b * a.mod_stride : nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Four<T, CUT> pw = param4<T, CUT>(a.w.pre_w, D, at.c(i), at.hi(i), 1.f), rs = param4<T, CUT>(a.w.res_scale, D, at.c(i), at.hi(i), 1.f);
      const Four<T, CUT> ow = param4<T, CUT>(a.post ? a.w.post_w : nullptr, D, at.c(i), at.hi(i), 1.f);
      const Four<float, CUT> sc = param4<float, CUT>(scale, D, at.c(i), at.hi(i), 0.f), gt = param4<float, CUT>(gate, D, at.c(i), at.hi(i), 1.f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        wpre[i][j] = (1.f + sc.at(j)) * pw.at(j);
        wpost[i][j] = gt.at(j) * rs.at(j) * ow.at(j);
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[q][i][j] = 0.f;
      }
    }
  }
  Four<X, CUT> dxr[NV], xr[NV];
  Four<T, CUT> dur[NV], yr[NV];
  float mx, rx, my, ry;   // the row's statistics
  const bool has_y = a.y && a.post;
  auto load = [&](uint32_t sb) {
    const int rows = (int)min((uint32_t)TEAMS, s1 - sb);
    const int64_t row0 = (int64_t)b * a.S + sb;
    const __amdgpu_buffer_rsrc_t bdx = rows_of<X>(a.dx1, row0, rows, D), bx = rows_of<X>(a.du ? a.x : nullptr, row0, rows, D);
    const __amdgpu_buffer_rsrc_t bdu = rows_of<T>(a.du, row0, rows, D);
    auto stat = [&](int q, bool has) {
      return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rows_of<float>(has ? a.stats + q * M : nullptr, row0, rows, 1), (uint32_t)team * 4, 0, 0));
    };
    mx = stat(2, a.du && layer);
    rx = stat(3, a.du);
    my = stat(0, has_y && layer);
    ry = stat(1, has_y);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      xr[i].load(bx, at.off[i], at.hi(i));
      dur[i].load(bdu, at.off[i], at.hi(i));
      dxr[i].load(bdx, at.off[i], at.hi(i));
    }
  };
  auto load_y = [&](uint32_t sb) {   // read half a row later than the others, so its registers are free that much longer
    const __amdgpu_buffer_rsrc_t by = rows_of<T>(a.y, (int64_t)b * a.S + sb, (int)min((uint32_t)TEAMS, s1 - sb), D);
#pragma unroll
    for (int i = 0; i < NV; ++i) yr[i].load(by, at.off[i], at.hi(i));
  };
  if (s0 < s1) {
    load(s0);
    load_y(s0);
  }

  for (uint32_t sb = s0; sb < s1; sb += TEAMS) {
    const int rows = (int)min((uint32_t)TEAMS, s1 - sb);
    const int64_t row0 = (int64_t)b * a.S + sb;
    float dx[NV][4], v[NV][4], g[NV][4];
    const float rstd = rx, pmean = my, prstd = a.post ? ry : 1.f;
    float c[2];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        dx[i][j] = dxr[i].at(j);
        v[i][j] = (xr[i].at(j) - mx) * rx;
        g[i][j] = CUT != kShifted || at.own(i, j) ? dur[i].at(j) : 0.f;
      }
    }
    if (sb + TEAMS < s1) load(sb + TEAMS);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float r0 = 0.f, r1 = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        acc[0][i][j] += g[i][j];
        acc[1][i][j] = fmaf(g[i][j], v[i][j], acc[1][i][j]);
        g[i][j] *= wpre[i][j];
        r0 += g[i][j];
        r1 = fmaf(g[i][j], v[i][j], r1);
      }
      add_run(c[0], i, r0);
      add_run(c[1], i, r1);
    }
    sum(c);
    float c1 = layer ? c[0] * rD : 0.f, c2 = c[1] * rD;
    const __amdgpu_buffer_rsrc_t bdx = rows_of<X>(a.dx, row0, rows, D);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) dx[i][j] = fmaf(rstd, g[i][j] - fmaf(v[i][j], c2, c1), dx[i][j]);
      put4<X, CUT>(bdx, at.off[i], at.lo(i), at.hi(i), dx[i], past);
    }
    if (!a.y) continue;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const uint32_t keep = drops ? keep_of(a.drop, key, row0 + team, D, (int)at.c(i)) : 0xFu;
      float r0 = 0.f, r1 = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool in = team < rows && at.own(i, j) && (keep >> j & 1u);
        const float d = in ? dx[i][j] * a.drop.factor : 0.f;
        const float n = (yr[i].at(j) - pmean) * prstd;
        v[i][j] = n;
        acc[2][i][j] += d;
        acc[3][i][j] = in ? fmaf(d, n, acc[3][i][j]) : acc[3][i][j];   // a dropped value does not count, not even a NaN
        g[i][j] = d * wpost[i][j];
        r0 += g[i][j];
        r1 = fmaf(g[i][j], n, r1);
      }
      add_run(c[0], i, r0);
      add_run(c[1], i, r1);
    }
    if (sb + TEAMS < s1) load_y(sb + TEAMS);
    if (a.post) {
      sum(c);
      c1 = layer ? c[0] * rD : 0.f;
      c2 = c[1] * rD;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) g[i][j] = prstd * (g[i][j] - fmaf(v[i][j], c2, c1));
    }
    const __amdgpu_buffer_rsrc_t bdy = rows_of<T>(a.dy, row0, rows, D);
#pragma unroll
    for (int i = 0; i < NV; ++i) put4<T, CUT>(bdy, at.off[i], at.lo(i), at.hi(i), g[i], past);
  }

  float* part = a.part + (size_t)blockIdx.x * 4 * D;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (TEAMS == 1) {
#pragma unroll
      for (int i = 0; i < NV; ++i) put4<float, CUT>(rows_of<float>(part, q, 1, D), at.c(i), at.lo(i), at.hi(i), acc[q][i]);
    } else {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)   // natural order: a shifted run's own channels follow the run before
          if (CUT != kShifted) cols[team][(i * LPR + t) * 4 + j] = acc[q][i][j];
          else if (at.own(i, j)) cols[team][at.c(i) + j] = acc[q][i][j];
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

// The workgroups' parts to the gradients.  A workgroup takes kCols channels and one of the two pairs of sums, kGroups
// samples at a time: its kGroups groups of threads share the samples (G to a sample, thread (g, d) adds the parts g, g + G, .. of channel d),
// meet in LDS, and one group per sample goes on with it; the parameters' sums over the samples follow in their order.
constexpr int kCols = 32, kGroups = 1024 / kCols;
template <typename T>
__global__ __launch_bounds__(1024) void residual_norm_grads_kernel(ResidualNorm a, int chunks) {
  __shared__ float sm[2][kGroups][kCols + 1], cb[3][kGroups][kCols + 1];
  const int dl = threadIdx.x % kCols, grp = threadIdx.x / kCols, D = a.D, d = blockIdx.x * kCols + dl, pair = blockIdx.y;
  const bool in = d < D;
  auto w = [&](const void* p, float fill) { return p && in ? to_f32<T>(((const T*)p)[d]) : fill; };
  const float pre_w = w(a.w.pre_w, 1.f), pre_b = w(a.w.pre_b, 0.f), rs = w(a.w.res_scale, 1.f);
  const float post_w = w(a.post ? a.w.post_w : nullptr, 1.f), post_b = w(a.post ? a.w.post_b : nullptr, 0.f);
  float tw = 0.f, tb = 0.f, tr = 0.f;
  for (int b0 = 0; b0 < a.B; b0 += kGroups) {
    const int nb = min(a.B - b0, kGroups);
    int G = kGroups;   // groups of a sample: the largest power of two that gives every sample one
    while (G * nb > kGroups) G >>= 1;
    const int bl = grp / G, g = grp - bl * G;
    float s0 = 0.f, s1 = 0.f;
    if (in && bl < nb) {
      const float* p = a.part + ((size_t)(b0 + bl) * chunks * 4 + 2 * pair) * D + d;
#pragma unroll 8
      for (int k = g; k < chunks; k += G) {
        s0 += p[(size_t)k * 4 * D];
        s1 += p[(size_t)k * 4 * D + D];
      }
    }
    sm[0][grp][dl] = s0;
    sm[1][grp][dl] = s1;
    __syncthreads();
    if (grp < nb && in) {
      s0 = s1 = 0.f;
      for (int k = 0; k < G; ++k) {
        s0 += sm[0][grp * G + k][dl];
        s1 += sm[1][grp * G + k][dl];
      }
      const size_t o = (size_t)(b0 + grp) * D + d, om = (size_t)(b0 + grp) * a.mod_stride + d;
      if (pair == 0) {
        const float sc = 1.f + (a.w.scale ? a.w.scale[om] : 0.f);
        if (a.g.shift) a.g.shift[o] = s0;
        if (a.g.scale) a.g.scale[o] = fmaf(pre_w, s1, pre_b * s0);
        cb[0][grp][dl] = sc * s0;
        cb[1][grp][dl] = sc * s1;
      } else {
        const float gt = a.w.gate ? a.w.gate[om] : 1.f, v = fmaf(post_w, s1, post_b * s0);
        if (a.g.gate) a.g.gate[o] = rs * v;
        cb[0][grp][dl] = gt * rs * s0;
        cb[1][grp][dl] = gt * rs * s1;
        cb[2][grp][dl] = gt * v;
      }
    }
    __syncthreads();
    if (grp == 0 && in)
      for (int k = 0; k < nb; ++k) {
        tb += cb[0][k][dl];
        tw += cb[1][k][dl];
        if (pair) tr += cb[2][k][dl];
      }
  }
  if (grp == 0 && in) {
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

// Lanes of a row.  Few rows of up to 2048 channels take as many as have a run of four channels: each row has a CU of its own, and
// what counts is the length of a wave's instructions.  us of a kernel in a graph, forward and backward with its join, a lane for every
// run against four or fewer runs a lane:
//   1024 channels: 1 row 3.0 + 6.7 (4.6 + 11.2), 256 rows 3.5 + 10.0 (5.2 + 12.2), 257 4.3 + 10.4 (5.2 + 12.2), 512 4.6 + 11.1 (5.5 + 13.1),
//   1024 5.5 + 13.9 (5.9 + 15.4), 2048 7.3 + 16.5 (8.7 + 16.8);  512: 256 rows 3.4 + 9.0 (3.7 + 9.0), 384 3.4 + 9.9 (3.8 + 9.3), 2048
//   5.4 + 13.8 (5.6 + 12.3);  2048: 256 rows 4.5 + 11.8 (5.4 + 14.8), 512 6.0 + 13.7 (5.9 + 16.4).
// The border is where a CU has one row; 513 to 1024 channels would still gain at eight times as many rows.
constexpr int kFewRows = 256;
int lanes_of(int64_t M, int D) {
  if (M <= kFewRows && D > 256 && D <= 2048) return D <= 512 ? 128 : D <= 1024 ? 256 : 512;
  return D <= 128 ? 32 : D <= 1024 ? 64 : D <= 2048 ? 128 : D <= 4096 ? 256 : 512;
}

// Workgroups per sample, so that there are about `wgs` of them: in the backward 512 threads per CU, all that its registers leave room for; in the forward, where three fit,
// a little more (16200 x 1024: 768 42.3 us, 1024 41.0, 1536 42.0).
int chunks_of(int B, int S, int D, int threads, int wgs) {
  const int64_t M = (int64_t)B * S;
  const int teams = threads / lanes_of(M, D);
  // rows of a team: two at least once every CU has a workgroup, so that one loads under the other (8 x 512 x 1024 forward 14.1 -> 12.1 us)
  const int64_t rows = std::max<int64_t>(M > 256 * teams ? 2 : 1, (M + (int64_t)wgs * teams - 1) / ((int64_t)wgs * teams));
  return (int)((S + rows * teams - 1) / (rows * teams));
}
int fwd_chunks(int B, int S, int D) { return chunks_of(B, S, D, fwd_threads(lanes_of((int64_t)B * S, D)), 1024); }
int bwd_chunks(int B, int S, int D) {
  const int threads = bwd_threads(lanes_of((int64_t)B * S, D));
  return chunks_of(B, S, D, threads, 512 * 256 / threads);
}

template <typename T, typename X, int LPR, int NV, int CUT>
hipError_t run_rows(const ResidualNorm& a, bool bwd, hipStream_t st) {
  const int chunks = bwd ? bwd_chunks(a.B, a.S, a.D) : fwd_chunks(a.B, a.S, a.D);
  const dim3 grid((unsigned)a.B * (unsigned)chunks);
  if (bwd) SR_LAUNCH((residual_norm_bwd_kernel<T, X, LPR, NV, CUT>), grid, dim3(bwd_threads(LPR)), 0, st, a, chunks);
  else SR_LAUNCH((residual_norm_fwd_kernel<T, X, LPR, NV, CUT>), grid, dim3(fwd_threads(LPR)), 0, st, a, chunks);
  return hipGetLastError();
}

template <typename T, typename X, int LPR, int CUT>
hipError_t run_runs(const ResidualNorm& a, bool bwd, hipStream_t st) {   // one where few rows have a lane for each; three where they hold the row
  if constexpr (LPR > 64) {
    if (a.D <= 4 * LPR) return run_rows<T, X, LPR, 1, CUT>(a, bwd, st);
  }
  return a.D <= 12 * LPR ? run_rows<T, X, LPR, 3, CUT>(a, bwd, st) : run_rows<T, X, LPR, 4, CUT>(a, bwd, st);
}
template <typename T, typename X, int CUT>
hipError_t run_width(const ResidualNorm& a, bool bwd, hipStream_t st) {
  switch (lanes_of((int64_t)a.B * a.S, a.D)) {
    case 32: return run_rows<T, X, 32, 1, CUT>(a, bwd, st);
    case 64:
      if (a.D <= 256) return run_rows<T, X, 64, 1, CUT>(a, bwd, st);
      return a.D <= 512 ? run_rows<T, X, 64, 2, CUT>(a, bwd, st) : run_runs<T, X, 64, CUT>(a, bwd, st);
    case 128: return run_runs<T, X, 128, CUT>(a, bwd, st);
    case 256: return run_runs<T, X, 256, CUT>(a, bwd, st);
    default: return run_runs<T, X, 512, CUT>(a, bwd, st);
  }
}
template <typename T, typename X>
hipError_t run(const ResidualNorm& a, bool bwd, hipStream_t st) {
  if (a.D < 4) return run_rows<T, X, 32, 1, kSingle>(a, bwd, st);
  return a.D % 4 == 0 ? run_width<T, X, kWhole>(a, bwd, st) : run_width<T, X, kShifted>(a, bwd, st);
}

hipError_t run_types(int dtype, int stream_dtype, const ResidualNorm& a, bool bwd, hipStream_t st) {
  if (dtype == kF32) return run<float, float>(a, bwd, st);
  return stream_dtype == kF32 ? run<bf16_t, float>(a, bwd, st) : run<bf16_t, bf16_t>(a, bwd, st);
}

}  // namespace

size_t residual_norm_need(int B, int S, int D) { return (size_t)B * bwd_chunks(B, S, D) * 4 * D * sizeof(float); }

// The most that a call of this many samples, rows and channels or fewer needs (more rows take fewer lanes each, and then fewer
// workgroups).  Of W workgroups aimed at (chunks_of; 512 from 1025 channels on, and where few rows take more lanes, but these are 256 rows at
// most), a sample has (W - 1) / B + 1 at most, and no more than rows / T of whole teams.
size_t residual_norm_scratch(int B, int S, int D) {
  const int64_t W = D <= 1024 ? 256 : 512, T = D <= 128 ? 16 : D <= 256 ? 8 : 1;
  const int64_t parts = std::max<int64_t>(B, std::min(B * ((S + T - 1) / T), std::min<int64_t>(B, W) + W - 1));
  return (size_t)parts * 4 * D * sizeof(float);
}

hipError_t launch_residual_norm_fwd(int dtype, int stream_dtype, const ResidualNorm& a, hipStream_t st) {
  return run_types(dtype, stream_dtype, a, false, st);
}

hipError_t launch_residual_norm_bwd(int dtype, int stream_dtype, const ResidualNorm& a, hipStream_t st) {
  hipError_t e = run_types(dtype, stream_dtype, a, true, st);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)((a.D + kCols - 1) / kCols), 2);
  const int chunks = bwd_chunks(a.B, a.S, a.D);
  if (dtype == kBF16) SR_LAUNCH((residual_norm_grads_kernel<bf16_t>), grid, dim3(1024), 0, st, a, chunks);
  else SR_LAUNCH((residual_norm_grads_kernel<float>), grid, dim3(1024), 0, st, a, chunks);
  return hipGetLastError();
}

}  // namespace sr
