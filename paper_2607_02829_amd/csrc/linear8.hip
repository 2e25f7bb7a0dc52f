// Linear layer on 8-bit integers: y[m, n] = act(xs[m] ws[n] sum_k xq[m, k] wq[n, k] + bias[n]).
//
// The products are summed exactly in int32 (127^2 K < 2^31 for every K that the call takes), so how a
// sum is cut over instructions, waves and tiles changes no bit; it is then rounded to fp32 once, scaled,
// and rounded once to the storage type.  Every variant finishes its sums with the same operations
// (finish4), so a token's result does not depend on its batch.
#include "common.h"
#include "epilogue.h"
#include "quant8.h"
#include "sr_internal.h"
#include "tiles.h"

namespace sr {

namespace {

typedef __attribute__((__vector_size__(16 * sizeof(int)))) int i32x16;

// Columns n .. n + 3: the channels' scales and bias.
struct Cols {
  f32x4 ws, bias;
};
template <typename T>
SR_DEV f32x4 load4(const void* p, size_t o) {
  if constexpr (sizeof(T) == 4) {
    return *reinterpret_cast<const f32x4*>((const float*)p + o);
  } else {
    const i32x2 w = *reinterpret_cast<const i32x2*>((const bf16_t*)p + o);
    return f32x4{__uint_as_float((uint32_t)w[0] << 16), __uint_as_float((uint32_t)w[0] & 0xFFFF0000u),
                 __uint_as_float((uint32_t)w[1] << 16), __uint_as_float((uint32_t)w[1] & 0xFFFF0000u)};
  }
}
template <typename T>
SR_DEV void store4(void* p, size_t o, f32x4 v) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>((float*)p + o) = v;
  } else {
    i32x2 w;
    w[0] = (int)f2bf2(v[0], v[1]);
    w[1] = (int)f2bf2(v[2], v[3]);
    *reinterpret_cast<i32x2*>((bf16_t*)p + o) = w;
  }
}
template <typename T>
SR_DEV Cols load_cols(const Linear8& a, int n) {
  Cols c;
  c.ws = load4<float>(a.ws, n);
  c.bias = a.bias ? load4<T>(a.bias, n) : f32x4{0.f, 0.f, 0.f, 0.f};
  return c;
}
// Type of what a tile stages, and the store of columns n .. n + 3 of row m.
template <int ACT, typename T>
struct OutOf { typedef T type; };
template <typename T>
struct OutOf<kActResid, T> { typedef float type; };
template <int ACT, typename T>
SR_DEV void put4(const Linear8& a, int m, int n, f32x4 v) {
  const size_t o = (size_t)m * a.N + n;
  if constexpr (ACT == kActResid) {
    if (a.gate) v *= *reinterpret_cast<const f32x4*>(a.gate + (size_t)(m / a.S) * a.gate_stride + n);
    *reinterpret_cast<f32x4*>(a.out + o) = *reinterpret_cast<const f32x4*>(a.resid + o) + v;
  } else {
    store4<T>(a.y, o, v);
  }
}
// z Phi(z) as max(z, 0) - |z| Phi(-|z|): an operation fewer than z times Phi(z), with the limits at the infinities
// (a finite |z| times a Phi of 0).  Phi is fp32's fit for bf16 results too, so that they are the exact GELU rounded
// once: the shorter fit, four instructions an element fewer, puts 0.23 % of them a step away (2e-5 with this one) and
// takes 115 instead of 120 us with the tokens' codes at 16200 x 4096 x 1024.  The vector units are what the layer with
// GELU waits for: 23 instructions an element, two of them at a quarter of the rate, issuing in 51 % of the time there,
// with the matrix pipes at 28 %.
SR_DEV float gelu8(float z) {
  return fmaf(-fminf(fabsf(z), 3.4028234663852886e38f), half_erfc_of<9>(z, z * z), fmaxf(z, 0.f));
}
template <int ACT>
SR_DEV f32x4 finish4(float xs, const Cols& c, i32x4 acc) {
  f32x4 v;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[q] = fmaf((float)acc[q] * xs, c.ws[q], c.bias[q]);
    if constexpr (ACT == SR_ACT_GELU) v[q] = gelu8(v[q]);
  }
  return v;
}

// ---------------------------------------------------------------- tiles through LDS

// Operand tile of R rows x KB bytes (64 or 128): row r at KB r, its 16-byte chunks at positions c ^ bswz(r), so
// that the 16 rows of a fragment read's quarter wave cover the 64 banks once.  It is filled by whole 1 KB blocks,
// straight from memory (buffer_load ... lds): lane l lands at byte 16 l of its block and fetches the chunk that
// the swizzle places there.
template <int KB>
SR_DEV int bswz(int r) {
  return (r / (256 / KB)) & (KB / 16 - 1);
}
template <int KB, int BPW>
struct Fill {
  uint32_t off[BPW];
  uint32_t upper = 0;   // bit i: load i fetches the second 64 bytes of the tile
  SR_DEV void init(int r0, int K, int lane, int wid) {
    constexpr int CH = KB / 16, RPB = 64 / CH;
#pragma unroll
    for (int i = 0; i < BPW; ++i) {
      const int row = (wid * BPW + i) * RPB + lane / CH, c = (lane % CH) ^ bswz<KB>(row);
      off[i] = (uint32_t)(r0 + row) * (uint32_t)K + (uint32_t)(c * 16);
      upper |= (uint32_t)(c >> 2) << i;
    }
  }
};
// delta: the tile's byte offset in a row, or 2^31 past the last tile, which keeps the count of fills in flight
// uniform: those of rows of the operand then lie past its end and read zeros.  (A row past the operand's last
// one may wrap into the operand; what it holds reaches no output that is stored.)
template <int BPW>
SR_DEV void fill_tile(const uint32_t* off, __amdgpu_buffer_rsrc_t rs, char* lds, int wid, uint32_t delta) {
#pragma unroll
  for (int i = 0; i < BPW; ++i)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr_t*)(lds + (wid * BPW + i) * 1024), 16, off[i] + delta, 0, 0, 0);
}
// A tile of which the row has the first 64 bytes only: what would be the second half reads zeros.
template <int BPW>
SR_DEV void fill_half(const uint32_t* off, uint32_t upper, __amdgpu_buffer_rsrc_t rs, char* lds, int wid, uint32_t delta) {
#pragma unroll
  for (int i = 0; i < BPW; ++i)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr_t*)(lds + (wid * BPW + i) * 1024), 16,
                                             off[i] + (upper >> i & 1u ? 0x80000000u : delta), 0, 0, 0);
}

// BM x BN workgroup tile on WM x WN waves, each MI x NJ tiles of v_mfma_i32_32x32x32_i8; KG such groups of
// waves share the tile, each with a run of the k range and LDS stages of its own.  NST stages; fills run
// NST - 1 k-tiles ahead; fragment reads are explicit (lds_read16), so none waits for a fill it does not need.
// Per k-tile: a k-step's products with the next one's fragment reads under them; before the last k-step's the wait
// for the next tile's fill and the barrier, after which this tile's stage is filled anew and the next tile's first
// fragments are read.  OCC workgroups per CU.
template <int BM, int BN, int KB, int WM, int WN, int KG, int NST, int OCC, int ACT, typename T>
__global__ __launch_bounds__(64 * WM * WN * KG, OCC) void linear8_tile_kernel(Linear8 a, int tiles_m, int tiles_n) {
  constexpr int NW = WM * WN, NT = 64 * NW * KG;
  constexpr int MI = BM / (32 * WM), NJ = BN / (32 * WN);
  constexpr int SB = (BM + BN) * KB;               // bytes of a stage: the token tile, then the weight tile
  constexpr int RPB = 1024 / KB, APW = BM / RPB / NW, BPW = BN / RPB / NW, LPT = APW + BPW, KS = KB / 32;
  static_assert(MI * 32 * WM == BM && NJ * 32 * WN == BN && APW * RPB * NW == BM && BPW * RPB * NW == BN, "whole tiles");
  static_assert(NST >= 2 && NST <= 4 && (NST - 1) * LPT < 64 && MI + NJ < 16, "counter ranges");
  __shared__ __attribute__((aligned(1024))) char smem[KG * NST * SB];
  __shared__ __attribute__((aligned(16))) float sc[KG == 1 ? 2 * BN : 4];   // the tile's channel scales, then its biases

  const int lane = threadIdx.x & 63, wave = wave_index();
  const int grp = wave / NW, wid = wave % NW;
  const int wm = wid / WN, wn = wid % WN, h = lane >> 5;
  int tm, tn, split;
  tile_coords(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn, split);
  const int m0 = tm * BM, n0 = tn * BN;
  const int all = (a.K + KB - 1) / KB, ntile = (all + KG - 1) / KG;   // every group runs ntile, the missing ones on zeros
  const int t0 = grp * ntile, nmine = min(ntile, all - t0);
  const __amdgpu_buffer_rsrc_t ra = make_rsrc(a.xq, (uint32_t)a.M * (uint32_t)a.K);
  const __amdgpu_buffer_rsrc_t rb = make_rsrc(a.wq, (uint32_t)a.N * (uint32_t)a.K);

  if constexpr (KG == 1) {
    for (int i = threadIdx.x; i < BN; i += NT) {
      const bool in = n0 + i < a.N;
      sc[i] = in ? a.ws[n0 + i] : 0.f;
      sc[BN + i] = in && a.bias ? to_f32<T>(((const T*)a.bias)[n0 + i]) : 0.f;
    }
  }
  i32x16 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;

  Fill<KB, APW> fla;
  Fill<KB, BPW> flb;
  fla.init(m0, a.K, lane, wid);
  flb.init(n0, a.K, lane, wid);
  auto fill = [&](int t, int s) {
    char* st = smem + (grp * NST + s) * SB;
    const int k0 = (t0 + t) * KB;
    const uint32_t delta = t < nmine ? (uint32_t)k0 : 0x80000000u;
    if (KB > 64 && t < nmine && k0 + KB > a.K) {
      fill_half<APW>(fla.off, fla.upper, ra, st, wid, delta);
      fill_half<BPW>(flb.off, flb.upper, rb, st + BM * KB, wid, delta);
    } else {
      fill_tile<APW>(fla.off, ra, st, wid, delta);
      fill_tile<BPW>(flb.off, rb, st + BM * KB, wid, delta);
    }
  };
  // fragment of rows r .. r + 31 at k-step ks: lane's row r + lane % 32, chunk 2 ks + lane / 32; rows 16 apart
  // share the swizzle
  const uint32_t sbase = lds_addr(smem) + (uint32_t)(grp * NST * SB);
  uint32_t fa[KS], fb[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    const int r = lane & 31, c = ((2 * ks + h) ^ bswz<KB>(r)) * 16;
    fa[ks] = sbase + (uint32_t)((wm * (BM / WM) + r) * KB + c);
    fb[ks] = sbase + (uint32_t)(BM * KB + (wn * (BN / WN) + r) * KB + c);
  }
  i32x4 ua[2][MI], ub[2][NJ];
  // fragment F of k-step ks of stage S: the MI token fragments, then the NJ weight fragments
  auto read1 = [&](auto sidx, auto ksv, auto fv) {
    constexpr int S = decltype(sidx)::value, ks = decltype(ksv)::value, F = decltype(fv)::value;
    if constexpr (F < MI) ua[ks & 1][F] = rd16<S * SB + F * 32 * KB>(fa[ks]);
    else ub[ks & 1][F - MI] = rd16<S * SB + (F - MI) * 32 * KB>(fb[ks]);
  };
  auto settle = [&](int ks) {
#pragma unroll
    for (int i = 0; i < MI; ++i) pin(ua[ks & 1][i]);
#pragma unroll
    for (int j = 0; j < NJ; ++j) pin(ub[ks & 1][j]);
  };
  // the products of one k-step, with issue(X) after product X: what it issues goes out under the products
  auto mfmas = [&](auto ksv, auto&& issue) {
    constexpr int ks = decltype(ksv)::value & 1;
    static_for<MI * NJ>([&](auto x) {
      constexpr int i = decltype(x)::value / NJ, j = decltype(x)::value % NJ;
      acc[i][j] = KG == 1 ? __builtin_amdgcn_mfma_i32_32x32x32_i8(ub[ks][j], ua[ks][i], acc[i][j], 0, 0, 0)
                          : __builtin_amdgcn_mfma_i32_32x32x32_i8(ua[ks][i], ub[ks][j], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      issue(x);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // the share of NF fragment reads that goes out after product X of NX
  constexpr int NF = MI + NJ, NX = MI * NJ;

  static_for<NST>([&](auto s) { fill(s.value, s.value); });
  wait_vm_lgkm0<(NST - 1) * LPT>();
  lds_barrier();
  static_for<NF>([&](auto f) { read1(IC<0>{}, IC<0>{}, f); });
  auto body = [&](int t, auto sidx) {
    constexpr int S = decltype(sidx)::value;
    static_for<KS - 1>([&](auto ksv) {
      constexpr int ks = decltype(ksv)::value;
      lgkm_wait<0>();
      settle(ks);
      __builtin_amdgcn_sched_barrier(0);
      mfmas(ksv, [&](auto x) {
        constexpr int X = decltype(x)::value, F0 = X * NF / NX, F1 = (X + 1) * NF / NX;
        static_for<F1 - F0>([&](auto f) { read1(sidx, IC<ks + 1>{}, IC<F0 + decltype(f)::value>{}); });
      });
    });
    // the next tile is resident (its fill is the oldest in flight), and every wave is done with this one's stage
    wait_vm_lgkm0<(NST - 2) * LPT>();
    lds_barrier();
    settle(KS - 1);
    __builtin_amdgcn_sched_barrier(0);
    mfmas(IC<KS - 1>{}, [&](auto x) {   // reads of the next tile: unused past the last one
      constexpr int X = decltype(x)::value, F0 = X * NF / NX, F1 = (X + 1) * NF / NX;
      static_for<F1 - F0>([&](auto f) { read1(IC<(S + 1) % NST>{}, IC<0>{}, IC<F0 + decltype(f)::value>{}); });
      if constexpr (X == (NX > 1 ? 1 : 0)) fill(t + NST, S);
    });
  };
  for (int t = 0; t < ntile; t += NST)
    static_for<NST>([&](auto s) {
      if (s.value == 0 || t + s.value < ntile) body(t + s.value, s);
    });
  // the last body's reads and fills land before their registers and stages are used again
  lgkm_wait<0>();
  settle(0);
  wait_vm_lgkm0<0>();
  __syncthreads();

  if constexpr (KG == 1) {
    // one group: the weight is the first operand, so that a lane has four consecutive channels of one token in each
    // register quad (register r: channel 8 (r/4) + 4 h + r%4, token lane % 32) and finishes them where they are.  The
    // results go through LDS, IPP blocks of every wave row at a time, so that memory sees whole rows of the tile
    // (16200 x 4096 x 1024: 105 us in 32-byte pieces from the registers, 95 in rows).
    typedef typename OutOf<ACT, T>::type O;
    constexpr int E = sizeof(O), LDB = BN * E + 16, PR = 32 * WM;
    constexpr int FIT = NST * SB / (PR * LDB), IPP = FIT >= MI ? MI : FIT >= 2 && MI % 2 == 0 ? 2 : 1;
    static_assert(IPP * PR * LDB <= NST * SB && MI % IPP == 0, "staging fits the stages");
    constexpr int CPR = BN * E / 16, NB = IPP * PR * CPR / NT;
    static_assert(NB * NT == IPP * PR * CPR, "whole rounds");
#pragma unroll
    for (int p = 0; p < MI; p += IPP) {
      if (p) __syncthreads();
#pragma unroll
      for (int i = 0; i < IPP; ++i) {
        const int m = m0 + wm * (BM / WM) + 32 * (p + i) + (lane & 31);
        const float xs = m < a.M ? a.xs[m] : 0.f;
        char* row = smem + ((i * WM + wm) * 32 + (lane & 31)) * LDB;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int nb = wn * (BN / WN) + 32 * j;
          f32x4 v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const Cols c = {*reinterpret_cast<const f32x4*>(sc + nb + 8 * q + 4 * h),
                            *reinterpret_cast<const f32x4*>(sc + BN + nb + 8 * q + 4 * h)};
            v[q] = finish4<ACT>(xs, c, i32x4{acc[p + i][j][4 * q], acc[p + i][j][4 * q + 1], acc[p + i][j][4 * q + 2],
                                                acc[p + i][j][4 * q + 3]});
            store4<O>(row, nb + 8 * q + 4 * h, v[q]);
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int c = threadIdx.x + NT * b, lr = c / CPR, col = c % CPR * (16 / E), blk = lr >> 5;
        const int m = m0 + blk % WM * (BM / WM) + 32 * (p + blk / WM) + (lr & 31), n = n0 + col;
        if (m < a.M && n < a.N) {
          const i32x4 w = *reinterpret_cast<const i32x4*>(smem + lr * LDB + col * E);
          if constexpr (ACT == kActResid) put4<ACT, T>(a, m, n, __builtin_bit_cast(f32x4, w));
          else *reinterpret_cast<i32x4*>((T*)a.y + (size_t)m * a.N + n) = w;
        }
      }
    }
  } else {
    // more groups: MI passes of PR rows.  Pass p stages block p of every wave row in LDS, one plane per group; each
    // thread then finishes NB chunks of four columns (register r: row 8 (r/4) + 4 h + r%4, column lane % 32)
    int* stg = reinterpret_cast<int*>(smem);
    constexpr int PR = 32 * WM, LD = BN + 8, CPR = BN / 4, NB = (PR * CPR + NT - 1) / NT;
    static_assert(NT % CPR == 0 && (NB * NT == PR * CPR || NB == 1), "a thread's chunks share their columns");
    static_assert(KG * PR * LD * 4 <= KG * NST * SB, "staging fits the stages");
    const bool active = PR * CPR >= NT || (int)threadIdx.x < PR * CPR;
    const int c4 = (threadIdx.x % CPR) * 4, n = n0 + c4;
    const bool ok = active && n < a.N;
    auto row_of = [&](int p, int q) {
      const int lr = (threadIdx.x + NT * q) / CPR;
      return m0 + (lr >> 5) * (BM / WM) + p * 32 + (lr & 31);
    };
    Cols cols{};
    if (ok) cols = load_cols<T>(a, n);
    float xs[MI][NB];
#pragma unroll
    for (int p = 0; p < MI; ++p)
#pragma unroll
      for (int q = 0; q < NB; ++q) {
        const int m = row_of(p, q);
        xs[p][q] = m < a.M && ok ? a.xs[m] : 0.f;
      }
#pragma unroll
    for (int p = 0; p < MI; ++p) {
      if (p) __syncthreads();
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          stg[(grp * PR + wm * 32 + 8 * (r >> 2) + 4 * h + (r & 3)) * LD + wn * (BN / WN) + j * 32 + (lane & 31)] =
              acc[p][j][r];
      __syncthreads();
#pragma unroll
      for (int q = 0; q < NB; ++q) {
        const int lr = (threadIdx.x + NT * q) / CPR, m = row_of(p, q);
        if (m < a.M && ok) {
          i32x4 v = *reinterpret_cast<const i32x4*>(stg + lr * LD + c4);
#pragma unroll
          for (int g = 1; g < KG; ++g) v += *reinterpret_cast<const i32x4*>(stg + (g * PR + lr) * LD + c4);
          put4<ACT, T>(a, m, n, finish4<ACT>(xs[p][q], cols, v));
        }
      }
    }
  }
}

// ---------------------------------------------------------------- few tokens

// R x R tile on W waves that share the k range, fragments straight from memory (lane: row lane % R, 16 bytes of k):
// with few tiles a launch is as long as its slowest chain of loads, and here a wave has its next eight k-steps in
// flight at once.  The waves' sums meet in LDS.
template <int R, int W, int ACT, typename T>
__global__ __launch_bounds__(64 * W) void linear8_few_kernel(Linear8 a) {
  static_assert(R == 16, "register layout of the 16 x 16 product");
  constexpr int STEP = 64, U = 8;
  __shared__ int stg[W][R][R + 4];
  const int lane = threadIdx.x & 63, wave = wave_index(), r = lane % R, h = lane / R;
  const int m0 = blockIdx.y * R, n0 = blockIdx.x * R;
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq, (uint32_t)a.M * (uint32_t)a.K);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wq, (uint32_t)a.N * (uint32_t)a.K);
  const uint32_t ox = (uint32_t)(m0 + r) * (uint32_t)a.K + 16u * h, ow = (uint32_t)(n0 + r) * (uint32_t)a.K + 16u * h;
  const int steps = a.K / STEP, per = (steps + W - 1) / W, s1 = min(steps, (wave + 1) * per);
  i32x4 acc = {0, 0, 0, 0};
  for (int s = wave * per; s < s1; s += U) {
    i32x4 x[U], w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {   // past the run's end: beyond the operands, zeros
      const uint32_t k = s + u < s1 ? (uint32_t)((s + u) * STEP) : 0x80000000u;
      x[u] = buf_load16(rx, ox + k);
      w[u] = buf_load16(rw, ow + k);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[u], w[u], acc, 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) stg[wave][4 * h + i][r] = acc[i];   // register i: row 4 h + i, column r
  __syncthreads();
  constexpr int CPR = R / 4;
  if ((int)threadIdx.x < R * CPR) {
    const int lr = threadIdx.x / CPR, c4 = threadIdx.x % CPR * 4, m = m0 + lr, n = n0 + c4;
    if (m < a.M && n < a.N) {
      i32x4 v = *reinterpret_cast<const i32x4*>(&stg[0][lr][c4]);
#pragma unroll
      for (int g = 1; g < W; ++g) v += *reinterpret_cast<const i32x4*>(&stg[g][lr][c4]);
      put4<ACT, T>(a, m, n, finish4<ACT>(a.xs[m], load_cols<T>(a, n), v));
    }
  }
}

// ---------------------------------------------------------------- dispatch

enum Shape { kFew16, k32x32g8, k64x64g2, k64x128, k128x128, k128x128x2, k256x128x2, k256x256 };

template <int BM, int BN, int KB, int WM, int WN, int KG, int NST, int OCC, int ACT, typename T>
hipError_t run_tile(const Linear8& a, hipStream_t st) {
  const int tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  SR_LAUNCH((linear8_tile_kernel<BM, BN, KB, WM, WN, KG, NST, OCC, ACT, T>), dim3((unsigned)(tm * tn)),
            dim3(64 * WM * WN * KG), 0, st, a, tm, tn);
  return hipGetLastError();
}
template <int R, int W, int ACT, typename T>
hipError_t run_few(const Linear8& a, hipStream_t st) {
  SR_LAUNCH((linear8_few_kernel<R, W, ACT, T>), dim3((unsigned)((a.N + R - 1) / R), (unsigned)((a.M + R - 1) / R)),
            dim3(64 * W), 0, st, a);
  return hipGetLastError();
}

template <int ACT, typename T>
hipError_t run_shape(int shape, const Linear8& a, hipStream_t st) {
  switch (shape) {
    case kFew16:   // longer rows on more waves (1 x 1024 x 8192 7.2 -> 6.5 us; x 4096 4.6, 4.4; x 2048 3.4, 3.8)
      return a.K > 2048 ? run_few<16, 8, ACT, T>(a, st) : run_few<16, 4, ACT, T>(a, st);
    case k32x32g8: return run_tile<32, 32, 64, 1, 1, 8, 4, 1, ACT, T>(a, st);
    case k64x64g2:
      // longer rows in whole lines (512 x 1024 x 4096 12.0 -> 10.8 us; 1024 x 512 x 2048 6.9, 7.7)
      return a.K > 2048 ? run_tile<64, 64, 128, 2, 2, 2, 4, 1, ACT, T>(a, st)
                        : run_tile<64, 64, 64, 2, 2, 2, 4, 1, ACT, T>(a, st);
    case k64x128: return run_tile<64, 128, 128, 2, 4, 1, 4, 1, ACT, T>(a, st);
    case k128x128: return run_tile<128, 128, 128, 2, 4, 1, 4, 1, ACT, T>(a, st);
    case k128x128x2: return run_tile<128, 128, 128, 2, 4, 1, 2, 2, ACT, T>(a, st);
    case k256x128x2:
      if constexpr (ACT == SR_ACT_GELU) return run_tile<256, 128, 64, 2, 2, 1, 3, 2, ACT, T>(a, st);
      else break;
    case k256x256: return run_tile<256, 256, 128, 2, 4, 1, 2, 1, ACT, T>(a, st);
  }
  return hipErrorInvalidValue;
}

// The smallest tile whose grid is one round of workgroups on the 256 CUs; past one round of 128 x 128 those, two
// workgroups per CU (one's epilogue under the other's products), or with long rows 256 x 256, once its own grid is most
// of a round.  us, bf16, M x N x K:
//   fragments straight from memory, up to one 16 x 16 tile per CU, of long rows with few tokens (or as much work in
//   more, shorter tiles):  1 x 4096 x 1024 3.3 (32 x 32 in eight groups 4.0), 64 x 1024 x 1024 3.2 (3.8), 1 x 1024 x 4096
//   4.4 (5.6), 16 x 4096 x 4096 7.2 (8.7), 64 x 1024 x 8192 9.4 (10.2), 128 x 1536 x 64 2.5 (64 x 64 3.3);  past it
//   100 x 1024 x 1024 4.2 (3.8), 128 x 1024 x 4096 9.2 (6.7), 100 x 512 x 8192 9.2 (8.6)
//   32 x 32, eight groups of waves:  128 x 1024 x 4096 6.7 (64 x 64 9.1);  x 256 3.6 (3.4)
//   64 x 64, two groups:  1024 x 1024 x 1024 6.2 (64 x 128 7.3);  64 x 128:  2048 x 1024 x 1024 7.7 (8.7, 128 x 128 9.7)
//   128 x 128, four stages, one workgroup per CU:  4050 x 1024 x 4096 22.9 (two 26.1);  with shorter rows two
//   workgroups are level or ahead: 4050 x 1024 x 1024 10.7 (10.3), 16200 x 256 x 1024 12.3 (14.4), 4083 x 1024 x 256 6.4
//   (6.8), fp32 8.6 (8.9).  Smaller tiles of four stages are behind where 128 x 128 is one round or just under it, which
//   leaves the second slot of every CU empty:  4050 x 1024 x 1024 64 x 128 12.8, 64 x 64 15.2;  4083 x 1024 x 256 8.4,
//   9.4, fp32 10.1, 10.1;  2500 x 1024 x 1024 11.4, 11.6 (9.7)
//   256 x 256:  16200 x 4096 x 1024 95 (106), 16200 x 1024 x 4096 67 (80), 16200 x 2048 x 512 36 (32);  with half a
//   round of them 8192 x 1024 x 4096 45 (42);  with GELU, whose vector work wants the second workgroup,
//   16200 x 2048 x 2048 93 (97), 8192 x 4096 x 1024 66 (62)
//   256 x 128 of 64-byte stages, two workgroups per CU, with GELU from two rounds of them:  16200 x 4096 x 1024 123
//   (128 x 128 126, 256 x 256 130), 8192 x 4096 x 1024 62.1 (62.1), 4050 x 4096 x 1024 34.8 (34.4)
// Elsewhere tiles of 256 x 128, and sixteen waves, lie within 4 % of these.
int pick_shape(const Linear8& a) {
  auto tiles = [&](int bm, int bn) { return (long)((a.M + bm - 1) / bm) * ((a.N + bn - 1) / bn); };
  const long t16 = tiles(16, 16);
  if ((t16 <= 256 && (a.K <= 4096 || a.M <= 64)) || (a.K <= 1024 && t16 * a.K <= 1 << 17)) return kFew16;
  if (a.K >= 512 && tiles(32, 32) <= 256) return k32x32g8;
  if (tiles(64, 64) <= 256) return k64x64g2;
  if (tiles(64, 128) <= 256) return k64x128;
  if (a.K >= 2048 && tiles(128, 128) <= 256) return k128x128;
  const bool gelu = a.act == SR_ACT_GELU;
  if (a.K >= (gelu ? 2048 : 1024) && tiles(256, 256) >= 200) return k256x256;
  return gelu && tiles(256, 128) >= 1024 ? k256x128x2 : k128x128x2;
}

template <typename T>
hipError_t run(int shape, const Linear8& a, hipStream_t st) {
  switch (a.act) {
    case SR_ACT_NONE: return run_shape<SR_ACT_NONE, T>(shape, a, st);
    case SR_ACT_GELU: return run_shape<SR_ACT_GELU, T>(shape, a, st);
    case kActResid: return run_shape<kActResid, T>(shape, a, st);
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_linear8(int dtype, const Linear8& a, hipStream_t st) {
  const int shape = pick_shape(a);
  return dtype == kBF16 ? run<bf16_t>(shape, a, st) : run<float>(shape, a, st);
}

}  // namespace sr
