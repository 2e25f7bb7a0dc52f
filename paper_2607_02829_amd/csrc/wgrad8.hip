// Weight and bias gradient of a linear layer from the 8-bit checkpoint of its input:
//   dw[n, k] = sum_m dy[m, n] xhat[m, k],   db[n] = sum_m dy[m, n],   xhat = q 2^e (SR_Q8_BLOCK).
//
// xhat is exact in bf16, so bf16 gradients take one product of v_mfma_f32_32x32x16_bf16 per term, exact before
// the fp32 sum.  fp32 gradients are cut into three bf16 parts of eight significant bits each, dy = hi + mid + lo
// without a remainder (of values under 2^-117 the bits below 2^-133 are left out), and take three products per term: a
// third of the bf16 rate, which is five times that of the fp32 matrix instructions.
//
// Both operands are token-major and the sum runs over tokens.  A workgroup takes 64 tokens at a time: each
// thread loads 16-byte pieces of dy and of the codes into registers, two tiles ahead, turns codes (and fp32
// gradients) into bf16 and writes them to one of two LDS stages while the other is multiplied; fragments come
// out of the transposing LDS reads.  The codes are a byte each on their way from memory and are decoded once per
// workgroup.  Few output tiles are cut over tokens into planes that a second launch adds in order.
//
// What bounds it: at 16200 x 1024 x 4096 the matrix pipes are busy 46 % of the time, the LDS 46 % and the vector
// units 28 %; a wave issues in order, so fragment reads, decoding and writes are placed between its products
// (256 x 128 tiles 177 us with the writes before the products, 157 so).  A call takes 148 us, 8 of them the planes'
// sum: 0.92 PFLOP/s.
#include <algorithm>

#include "common.h"
#include "quant8.h"
#include "sr_internal.h"
#include "tiles.h"

namespace sr {

namespace {

constexpr int TM = 64;   // tokens per tile

// LDS tile of TM token rows of R values: the 16-byte chunk c of row m at position c ^ rowswz(m), so that
// the four rows that a transposing read touches lie in different banks.
template <int R>
SR_DEV int rowswz(int m) {
  return R >= 128 ? (m & 3) << 2 : R == 64 ? ((m >> 1) & 1) << 2 : 0;
}

// The upper halves of two fp32 values as a pair of bf16 (truncated).
SR_DEV uint32_t upper2(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
SR_DEV float truncated(float v) { return __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); }

// Eight gradients of one token in flight: raw[0 ..) and their P bf16 parts.
template <typename T>
struct Grad8;
template <>
struct Grad8<bf16_t> {
  static constexpr int P = 1;
  i32x4 raw;
  SR_DEV void load(__amdgpu_buffer_rsrc_t r, uint32_t off) { raw = buf_load16(r, off); }
  SR_DEV void parts(i32x4 p[P]) const { p[0] = raw; }
  SR_DEV void add(float* s) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s[2 * j] += __uint_as_float((uint32_t)raw[j] << 16);
      s[2 * j + 1] += __uint_as_float((uint32_t)raw[j] & 0xFFFF0000u);
    }
  }
};
template <>
struct Grad8<float> {
  static constexpr int P = 3;
  i32x4 raw[2];
  SR_DEV void load(__amdgpu_buffer_rsrc_t r, uint32_t off) {
    raw[0] = buf_load16(r, off);
    raw[1] = buf_load16(r, off + 16);
  }
  SR_DEV float at(int j) const { return __int_as_float(raw[j >> 2][j & 3]); }
  // truncation leaves an exact remainder of the bits below, 24 = 8 + 8 + 8; none of an infinity, which would be NaN
  SR_DEV static float rest(float v) {
    const float t = truncated(v);
    return v == t ? 0.f : v - t;
  }
  SR_DEV void parts(i32x4 p[P]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = at(2 * j), b = at(2 * j + 1);
      const float ra = rest(a), rb = rest(b);
      p[0][j] = (int)upper2(a, b);
      p[1][j] = (int)upper2(ra, rb);
      p[2][j] = (int)upper2(ra - truncated(ra), rb - truncated(rb));
    }
  }
  SR_DEV void add(float* s) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] += at(j);
  }
};

// BN x BK tile of dw on KG groups of WN x WK waves, each with a part of the run's tokens and LDS stages of its own;
// the groups' sums meet in LDS.
template <typename T, int BN, int BK, int WN, int WK, int KG, int OCC>
__global__ __launch_bounds__(64 * WN * WK * KG, OCC) void wgrad8_kernel(Wgrad8 a, int tiles_n, int tiles_k, int per_split) {
  constexpr int NT = 64 * WN * WK, P = Grad8<T>::P;
  constexpr int NI = BN / (32 * WN), KJ = BK / (32 * WK);
  constexpr int STAGE = TM * (P * BN + BK);                        // bf16 elements: the parts of dy, then xhat
  constexpr int GR = NT / (BN / 8), GL = TM / GR;                  // dy: rows per round of loads, rounds
  constexpr int XR = NT / (BK / 16), XL = TM / XR;                 // codes
  static_assert(GL * GR == TM && XL * XR == TM, "whole rounds of loads");
  __shared__ __attribute__((aligned(1024))) bf16_t smem[KG * 2 * STAGE];
  const int grp = KG == 1 ? 0 : wave_index() / (WN * WK), wave = KG == 1 ? wave_index() : wave_index() % (WN * WK);
  const int tid = KG == 1 ? (int)threadIdx.x : (int)threadIdx.x % NT, lane = threadIdx.x & 63, h = lane >> 5;
  const int wn = wave / WK, wk = wave % WK;
  bf16_t* const stages = smem + grp * 2 * STAGE;
  int tn, tk, split;
  tile_coords(blockIdx.x, gridDim.x, tiles_n, tiles_k, tn, tk, split);
  const int n0 = tn * BN, k0 = tk * BK, mrun = split * per_split, mend = min(a.M, mrun + per_split);
  const int ntile = mrun < mend ? (mend - mrun + KG * TM - 1) / (KG * TM) : 0;   // per group; past the last token zeros
  const int mbeg = mrun + grp * ntile * TM;
  const __amdgpu_buffer_rsrc_t ry = make_rsrc(a.dy, (uint32_t)((size_t)a.M * a.N * sizeof(T)));
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq, (uint32_t)((size_t)a.M * a.K));
  const __amdgpu_buffer_rsrc_t re = make_rsrc(a.xe, (uint32_t)((size_t)a.M * (a.K / kQBlock)));

  // this thread's pieces: dy chunk gc of rows gr + i GR, codes 16 xc .. of rows xr + i XR
  const int gc = tid % (BN / 8), gr = tid / (BN / 8);
  const int xc = tid % (BK / 16), xr = tid / (BK / 16);
  const bool gin = n0 + gc * 8 < a.N, xin = k0 + xc * 16 < a.K;
  // pieces of a tile: GL of dy, then XL of codes, which are written in two halves; two tiles of them in flight
  constexpr int NP = GL + XL, NWR = GL + 2 * XL;
  Grad8<T> g[2][GL];
  i32x4 xv[2][XL];
  uint32_t xe[2][XL];
  // byte offsets of the next tile's pieces.  Rows past the last token lie past the operands and read zeros, as do the
  // offsets from 2^31 of channels past the last; tiles past the last read rows that nothing uses.
  uint32_t go[GL], xo[XL], eo[XL];
#pragma unroll
  for (int i = 0; i < GL; ++i)
    go[i] = gin ? ((uint32_t)(mbeg + gr + i * GR) * (uint32_t)a.N + (uint32_t)(n0 + gc * 8)) * (uint32_t)sizeof(T) : 0x80000000u;
#pragma unroll
  for (int i = 0; i < XL; ++i) {
    const uint32_t m = (uint32_t)(mbeg + xr + i * XR), k = (uint32_t)(k0 + xc * 16);
    xo[i] = xin ? m * (uint32_t)a.K + k : 0x80000000u;
    eo[i] = xin ? m * (uint32_t)(a.K / kQBlock) + k / kQBlock : 0x80000000u;
  }
  const uint32_t gstep = gin ? (uint32_t)(TM * sizeof(T)) * (uint32_t)a.N : 0u, xstep = xin ? (uint32_t)(TM * a.K) : 0u;
  auto load = [&](auto bv, auto pv) {
    constexpr int B = decltype(bv)::value, p = decltype(pv)::value;
    if constexpr (p < GL) {
      g[B][p].load(ry, go[p]);
      go[p] += gstep;
    } else {
      constexpr int i = p - GL;
      xv[B][i] = buf_load16(rx, xo[i]);
      xe[B][i] = __builtin_amdgcn_raw_buffer_load_b8(re, eo[i], 0, 0);
      xo[i] += xstep;
      eo[i] += xstep / kQBlock;
    }
  };
  const bool want_db = a.db && tk == 0;
  float dbv[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  auto write = [&](auto bv, auto wv, bf16_t* st, bool used) {
    constexpr int B = decltype(bv)::value, w = decltype(wv)::value;
    if constexpr (w < GL) {
      const int m = gr + w * GR;
      i32x4 p[P];
      g[B][w].parts(p);
#pragma unroll
      for (int q = 0; q < P; ++q)
        *reinterpret_cast<i32x4*>(st + q * TM * BN + m * BN + ((gc ^ rowswz<BN>(m)) << 3)) = p[q];
      if (want_db && used) g[B][w].add(dbv);
    } else {
      constexpr int i = (w - GL) / 2, c = (w - GL) % 2;
      const int m = xr + i * XR;
      const float s = block_scale(xe[B][i]);
      i32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int b = xv[B][i][2 * c + (j >> 1)] >> (16 * (j & 1));
        v[j] = (int)f2bf2((float)(int8_t)b * s, (float)(int8_t)(b >> 8) * s);
      }
      *reinterpret_cast<i32x4*>(st + P * TM * BN + m * BK + (((2 * xc + c) ^ rowswz<BK>(m)) << 3)) = v;
    }
  };

  // fragment of columns cb .. cb + 31 (lane: column lane % 32) at tokens 16 ks + 8 h .. + 7: two reads of four tokens
  const int fm = 8 * (lane >> 5) + ((lane & 15) >> 2), fc = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  auto frag = [&](const bf16_t* tile, auto rc, int cb, int ks) {
    constexpr int R = decltype(rc)::value;
    const int c = cb + fc;
    const bf16_t* p = tile + (16 * ks + fm) * R + (((c >> 3) ^ rowswz<R>(fm)) << 3) + (c & 7);
    i32x4 v;
    const i32x2 lo = __builtin_bit_cast(i32x2, ds_tr(p)), hi = __builtin_bit_cast(i32x2, ds_tr(p + 4 * R));
    v[0] = lo[0]; v[1] = lo[1]; v[2] = hi[0]; v[3] = hi[1];
    return __builtin_bit_cast(bf16x8, v);
  };
  f32x16 acc[NI][KJ];
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < KJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  static_for<NP>([&](auto p) { load(IC<0>{}, p); });
  static_for<NP>([&](auto p) { load(IC<1>{}, p); });
  static_for<NWR>([&](auto w) { write(IC<0>{}, w, stages, true); });
  static_for<NP>([&](auto p) { load(IC<0>{}, p); });
  // tile t, whose stage has parity S: its products, with the pieces of tile t + 1 written and those of t + 3
  // fetched in between
  constexpr int KS = TM / 16;
  auto body = [&](int t, auto sidx) {
    constexpr int S = decltype(sidx)::value;
    const bf16_t* st = stages + S * STAGE;
    bf16_t* next = stages + (1 - S) * STAGE;
    __syncthreads();   // tile t is written, and every wave is done with the other stage
    // fragments of k-step ks: the KJ of xhat, then the NI of each part of dy
    bf16x8 fx[2][KJ], fg[2][P * NI];
    auto read = [&](auto ksv, auto fv) {
      constexpr int ks = decltype(ksv)::value, f = decltype(fv)::value;
      if constexpr (f < KJ) fx[ks & 1][f] = frag(st + P * TM * BN, IC<BK>{}, wk * (BK / WK) + 32 * f, ks);
      else fg[ks & 1][f - KJ] = frag(st + (f - KJ) / NI * TM * BN, IC<BN>{}, wn * (BN / WN) + 32 * ((f - KJ) % NI), ks);
    };
    constexpr int NF = KJ + P * NI, NX = P * NI * KJ, SLOTS = KS * NX;
    static_for<NF>([&](auto f) { read(IC<0>{}, f); });
    static_for<KS>([&](auto ksv) {
      constexpr int ks = decltype(ksv)::value;
      static_for<NX>([&](auto xv_) {
        constexpr int X = decltype(xv_)::value, qi = X / KJ, j = X % KJ, Y = ks * NX + X;
        acc[qi % NI][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fg[ks & 1][qi], fx[ks & 1][j], acc[qi % NI][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        // under this product: a share of the next k-step's fragment reads, of the next tile's writes and of the loads
        if constexpr (ks + 1 < KS) {
          constexpr int F0 = X * NF / NX, F1 = (X + 1) * NF / NX;
          static_for<F1 - F0>([&](auto f) { read(IC<ks + 1>{}, IC<F0 + decltype(f)::value>{}); });
        }
        constexpr int W0 = Y * NWR / SLOTS, W1 = (Y + 1) * NWR / SLOTS;
        static_for<W1 - W0>([&](auto wv) {
          constexpr int w = W0 + decltype(wv)::value;
          write(IC<1 - S>{}, IC<w>{}, next, t + 1 < ntile);
          if constexpr (w < GL) load(IC<1 - S>{}, IC<w>{});
          else if constexpr ((w - GL) % 2 == 1) load(IC<1 - S>{}, IC<GL + (w - GL) / 2>{});
        });
        __builtin_amdgcn_sched_barrier(0);
      });
    });
  };
  // whole pairs in the loop: a way around the second body would make the waits on the first one's loads those of
  // the shorter way, with one tile in flight instead of two
  int t = 0;
  for (; t + 1 < ntile; t += 2) {
    body(t, IC<0>{});
    body(t + 1, IC<1>{});
  }
  if (t < ntile) body(t, IC<0>{});

  if constexpr (KG > 1) {   // the groups' sums, in order
    float* red = reinterpret_cast<float*>(smem);
    constexpr int TILE = NI * KJ * 16 * NT;
    static_assert(TILE * 4 * (KG - 1) <= (int)sizeof(smem), "sums fit the stages");
    __syncthreads();
    if (grp > 0) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < KJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) red[(grp - 1) * TILE + ((i * KJ + j) * 16 + r) * NT + tid] = acc[i][j][r];
    }
    __syncthreads();
    if (grp == 0) {
#pragma unroll
      for (int g = 0; g < KG - 1; ++g)
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
          for (int j = 0; j < KJ; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] += red[g * TILE + ((i * KJ + j) * 16 + r) * NT + tid];
    }
  }
  const bool cut = per_split < a.M;
  float* dw = cut ? a.scratch + (size_t)split * a.N * a.K : a.dw;
#pragma unroll
  for (int i = 0; i < NI; ++i)
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      const int k = k0 + wk * (BK / WK) + 32 * j + (lane & 31);
      if (grp > 0) break;
#pragma unroll
      for (int r = 0; r < 16; ++r) {   // register r: row 8 (r/4) + 4 h + r%4
        const int n = n0 + wn * (BN / WN) + 32 * i + 8 * (r >> 2) + 4 * h + (r & 3);
        if (n < a.N && k < a.K) dw[(size_t)n * a.K + k] = acc[i][j][r];
      }
    }
  if (want_db) {   // the threads of one chunk, in row order
    __syncthreads();
    float* red = reinterpret_cast<float*>(smem);   // [KG * GR][BN]
#pragma unroll
    for (int e = 0; e < 8; ++e) red[(grp * GR + gr) * BN + gc * 8 + e] = dbv[e];
    __syncthreads();
    for (int c = threadIdx.x; c < BN; c += KG * NT) {
      float s = 0.f;
      for (int r = 0; r < KG * GR; ++r) s += red[r * BN + c];
      const int n = n0 + c;
      if (n < a.N) (cut ? a.scratch + (size_t)gridDim.x / (tiles_n * tiles_k) * a.N * a.K + (size_t)split * a.N : a.db)[n] = s;
    }
  }
}

// The planes of a cut sum, in order: four values of dw per thread, then those of db; four planes are fetched at
// once.  One wave per workgroup, so that a small gradient spreads over the CUs.
__global__ __launch_bounds__(64) void wgrad8_sum_kernel(const float* __restrict__ part, int splits, size_t n4, size_t b4,
                                                        float* __restrict__ dw, float* __restrict__ db) {
  const size_t i = (size_t)blockIdx.x * 64 + threadIdx.x;
  if (i >= n4 + b4) return;
  const bool w = i < n4;
  const f32x4* p = reinterpret_cast<const f32x4*>(part) + (w ? i : (size_t)splits * n4 + (i - n4));
  const size_t step = w ? n4 : b4;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  int z = 0;
  for (; z + 4 <= splits; z += 4) {
    f32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = p[(size_t)(z + u) * step];
#pragma unroll
    for (int u = 0; u < 4; ++u) s += v[u];
  }
  for (; z < splits; ++z) s += p[(size_t)z * step];
  (w ? reinterpret_cast<f32x4*>(dw)[i] : reinterpret_cast<f32x4*>(db)[i - n4]) = s;
}

// Tile of dw and runs over tokens, by the size of dw in tiles of 128 x 128 (u) and the tokens.  us on bf16 for
// M x N x K (tokens, rows and columns of dw), /runs:
//   64 x 64 for a small dw or few tokens, on two groups of four waves up to a tile per CU:  1024 x 1024 x 1024 9.1
//     (one group 11.0; 128 x 128 14.0), 2048 x 1024 x 1024 13.3 (17.4; /2 18.6), 512 x 512 x 512 6.1 (6.7), and past
//     it two workgroups per CU:  1024 x 2048 x 1024 12.6 (two groups 14.8).  4096 x 512 x 512 /4 12.5 (/3 13.6), fp32
//     2048 x 1024 x 512 /2 18 (/1 22).
//   128 x 128 on eight waves:  8192 x 1024 x 1024 /4 32 (64 x 64 37), 2048 x 1024 x 4096 /1 26.9 (38; 256 x 128 33),
//     4096 x 2048 x 1024 /2 32 (36);  four waves of 64 x 64 each are behind.  fp32 gradients, three products a term,
//     reach it with fewer tokens: 4096 x 1024 x 1024 /4 37 (64 x 64 41).
//   256 x 128 where it costs less:  16200 x 1024 x 4096 /2 147 (169), 2048 x 4096 x 2048 /1 41 (46),
//     16200 x 1536 x 1024 /5 65 (77);  128 x 256 has twice the codes to decode per thread
// n runs cost rounds of workgroups x (tokens of a run x what a workgroup takes for a token + 3 us), and, where the sum
// is cut, a launch and the planes' way through the caches; 2 us more for 256 x 128's first and last tiles.  More
// tokens take more runs (their factor falls with n, the rest grows) and larger tiles, so for a square dw the scratch
// for more tokens is never less.  Over 286 sizes and types this is 1 % behind the fastest on average.
enum Shape { k64x64, k128x128, k256x128 };

struct Plan {
  int shape, splits, per_split, tiles_n, tiles_k, groups;
};
Plan plan(int dtype, int M, int N, int K) {
  const long u = (long)N * K >> 14;
  const bool bf = dtype == kBF16;
  auto tiled = [&](int shape, int bn, int bk) {
    Plan p;
    p.shape = shape;
    p.tiles_n = (N + bn - 1) / bn;
    p.tiles_k = (K + bk - 1) / bk;
    p.splits = p.groups = 1;
    return p;
  };
  // the runs of at least `least` tokens that cost least, token us per token of a workgroup; returns the cost
  auto cut = [&](Plan& p, double token, long least) {
    const long t = (long)p.tiles_n * p.tiles_k, most = std::clamp(M / least, 1l, 32l);
    double best = 0;
    for (long n = 1; n <= most; ++n) {
      const double rounds = (double)((t * n + 255) / 256);
      const double us = rounds * (M * token / n + 3) + (n > 1 ? 4 + 1e-6 * n * N * K : 0);
      if (n == 1 || us < best) best = us, p.splits = (int)n;
    }
    return best;
  };
  Plan p;
  if (std::min(N, K) > 64 && (u > 128 || (u > 64 ? M >= (bf ? 2560 : 1408)
                                                 : M >= (bf ? 4608 : 2560) && u * M >= (bf ? 224 : 104) << 10))) {
    p = tiled(k128x128, 128, 128);
    const double us = cut(p, bf ? 0.0105 : 0.025, bf ? 256 : 128);
    if (bf) {
      Plan w = tiled(k256x128, 256, 128);
      if (cut(w, 0.0155, 256) + 2 < us) p = w;
    }
  } else {
    p = tiled(k64x64, 64, 64);
    if ((long)p.tiles_n * p.tiles_k <= 256 && M >= 256) {
      p.groups = 2;
      cut(p, bf ? 0.0041 : 0.0088, 192);
    }
  }
  const int unit = TM * p.groups;
  p.per_split = ((M + p.splits - 1) / p.splits + unit - 1) / unit * unit;
  return p;
}

template <typename T, int BN, int BK, int WN, int WK, int KG, int OCC>
hipError_t run(const Wgrad8& a, const Plan& p, hipStream_t st) {
  const int n = p.splits > 1 ? (a.M + p.per_split - 1) / p.per_split : 1;
  SR_LAUNCH((wgrad8_kernel<T, BN, BK, WN, WK, KG, OCC>), dim3((unsigned)(p.tiles_n * p.tiles_k * n)),
            dim3(64 * WN * WK * KG), 0, st, a, p.tiles_n, p.tiles_k, n > 1 ? p.per_split : a.M);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || n == 1) return e;
  const size_t n4 = (size_t)a.N * a.K / 4, b4 = a.db ? (size_t)a.N / 4 : 0;
  SR_LAUNCH(wgrad8_sum_kernel, dim3((unsigned)((n4 + b4 + 63) / 64)), dim3(64), 0, st, a.scratch, n, n4, b4, a.dw,
            a.db);
  return hipGetLastError();
}

template <typename T>
hipError_t dispatch(const Wgrad8& a, const Plan& p, hipStream_t st) {
  constexpr bool F = sizeof(T) == 4;   // three parts of dy fill the LDS of a workgroup per CU
  switch (p.shape) {
    case k64x64:
      return p.groups == 2 ? run<T, 64, 64, 2, 2, 2, 2>(a, p, st) : run<T, 64, 64, 2, 2, 1, 2>(a, p, st);
    case k128x128: return run<T, 128, 128, 2, 4, 1, F ? 1 : 2>(a, p, st);
    case k256x128:
      if constexpr (!F) return run<T, 256, 128, 4, 2, 1, 1>(a, p, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace

size_t wgrad8_scratch(int dtype, int M, int N, int K) {
  const Plan p = plan(dtype, M, N, K);
  return p.splits > 1 ? (size_t)p.splits * ((size_t)N * K + N) * 4 : 0;
}

hipError_t launch_wgrad8(int dtype, const Wgrad8& a, hipStream_t st) {
  const Plan p = plan(dtype, a.M, a.N, a.K);
  return dtype == kBF16 ? dispatch<bf16_t>(a, p, st) : dispatch<float>(a, p, st);
}

}  // namespace sr
