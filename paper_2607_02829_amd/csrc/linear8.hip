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

constexpr int KB = 64;   // bytes (and channels) of k in an operand tile: K is a multiple of it

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
template <int ACT, typename T>
SR_DEV f32x4 finish4(float xs, const Cols& c, i32x4 acc) {
  f32x4 v;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    v[q] = fmaf((float)acc[q] * xs, c.ws[q], c.bias[q]);
    if constexpr (ACT == SR_ACT_GELU) v[q] = gelu_f<gelu_deg<T>()>(v[q]);
  }
  return v;
}

// ---------------------------------------------------------------- tiles through LDS

// Operand tile of R rows x KB bytes: row r at 64 r, its four 16-byte chunks at positions c ^ (r / 4) % 4,
// so that the 16 rows of a fragment read's quarter wave cover the 64 banks once.  It is filled by whole 1 KB
// blocks of 16 rows, straight from memory (buffer_load ... lds): lane l lands at byte 16 l of its block
// and fetches the chunk that the swizzle places there.
SR_DEV int bswz(int r) { return (r >> 2) & 3; }
template <int BPW>
SR_DEV void fill_offsets(uint32_t* off, int r0, int K, int lane, int wid) {
#pragma unroll
  for (int i = 0; i < BPW; ++i) {
    const int row = (wid * BPW + i) * 16 + (lane >> 2);
    off[i] = (uint32_t)(r0 + row) * (uint32_t)K + (uint32_t)(((lane & 3) ^ bswz(row)) * 16);
  }
}
// delta: the tile's byte offset in a row, or 2^31 past the last tile, which keeps the count of fills in flight
// uniform: those of rows of the operand then lie past its end and read zeros.  (A row past the operand's last
// one may wrap into the operand; what it holds reaches no output that is stored.)
template <int BPW>
SR_DEV void fill_tile(const uint32_t* off, __amdgpu_buffer_rsrc_t rs, char* lds, int wid, uint32_t delta) {
#pragma unroll
  for (int i = 0; i < BPW; ++i)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_ptr_t*)(lds + (wid * BPW + i) * 1024), 16, off[i] + delta, 0, 0,
                                             0);
}

// BM x BN workgroup tile on WM x WN waves, each MI x NJ tiles of v_mfma_i32_32x32x32_i8; KG such groups of
// waves share the tile, each with a run of the k range and LDS stages of its own.  NST stages; fills run
// NST - 1 k-tiles ahead; fragment reads are explicit (lds_read16), so none waits for a fill it does not need.
// Per k-tile: the second half's fragments are read, the first half multiplied; then the wait for the next tile's
// fill and the barrier, after which this tile's stage is filled anew and the next tile's first fragments are read
// under the second half's products.  OCC workgroups per CU.
template <int BM, int BN, int WM, int WN, int KG, int NST, int OCC, int ACT, typename T>
__global__ __launch_bounds__(64 * WM * WN * KG, OCC) void linear8_tile_kernel(Linear8 a, int tiles_m, int tiles_n) {
  constexpr int NW = WM * WN, NT = 64 * NW * KG;
  constexpr int MI = BM / (32 * WM), NJ = BN / (32 * WN);
  constexpr int SB = (BM + BN) * KB;               // bytes of a stage: the token tile, then the weight tile
  constexpr int APW = BM / 16 / NW, BPW = BN / 16 / NW, LPT = APW + BPW;
  static_assert(MI * 32 * WM == BM && NJ * 32 * WN == BN && APW * 16 * NW == BM && BPW * 16 * NW == BN, "whole tiles");
  static_assert(NST >= 2 && NST <= 4 && (NST - 1) * LPT < 64 && MI + NJ < 16, "counter ranges");
  __shared__ __attribute__((aligned(1024))) char smem[KG * NST * SB];

  const int lane = threadIdx.x & 63, wave = wave_index();
  const int grp = wave / NW, wid = wave % NW;
  const int wm = wid / WN, wn = wid % WN, h = lane >> 5;
  int tm, tn, split;
  tile_coords(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn, split);
  const int m0 = tm * BM, n0 = tn * BN;
  const int all = a.K / KB, ntile = (all + KG - 1) / KG;   // every group runs ntile, the missing ones on zeros
  const int t0 = grp * ntile, nmine = min(ntile, all - t0);
  const __amdgpu_buffer_rsrc_t ra = make_rsrc(a.xq, (uint32_t)a.M * (uint32_t)a.K);
  const __amdgpu_buffer_rsrc_t rb = make_rsrc(a.wq, (uint32_t)a.N * (uint32_t)a.K);

  i32x16 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0;

  uint32_t offa[APW], offb[BPW];
  fill_offsets<APW>(offa, m0, a.K, lane, wid);
  fill_offsets<BPW>(offb, n0, a.K, lane, wid);
  auto fill = [&](int t, int s) {
    char* st = smem + (grp * NST + s) * SB;
    const uint32_t delta = t < nmine ? (uint32_t)((t0 + t) * KB) : 0x80000000u;
    fill_tile<APW>(offa, ra, st, wid, delta);
    fill_tile<BPW>(offb, rb, st + BM * KB, wid, delta);
  };
  // fragment of rows r .. r + 31 at k-step ks: lane's row r + lane % 32, chunk 2 ks + lane / 32; rows 16 apart
  // share the swizzle
  const uint32_t sbase = lds_addr(smem) + (uint32_t)(grp * NST * SB);
  uint32_t fa[2], fb[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    const int r = lane & 31, c = ((2 * ks + h) ^ bswz(r)) * 16;
    fa[ks] = sbase + (uint32_t)((wm * (BM / WM) + r) * KB + c);
    fb[ks] = sbase + (uint32_t)(BM * KB + (wn * (BN / WN) + r) * KB + c);
  }
  i32x4 ua[2][MI], ub[2][NJ];
  auto read = [&](auto sidx, auto ksv) {
    constexpr int S = decltype(sidx)::value, ks = decltype(ksv)::value;
    static_for<MI>([&](auto i) { ua[ks][i.value] = rd16<S * SB + i.value * 32 * KB>(fa[ks]); });
    static_for<NJ>([&](auto j) { ub[ks][j.value] = rd16<S * SB + j.value * 32 * KB>(fb[ks]); });
  };
  auto settle = [&](int ks) {
#pragma unroll
    for (int i = 0; i < MI; ++i) pin(ua[ks][i]);
#pragma unroll
    for (int j = 0; j < NJ; ++j) pin(ub[ks][j]);
  };
  auto mfmas = [&](int ks) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        acc[i][j] = KG == 1 ? __builtin_amdgcn_mfma_i32_32x32x32_i8(ub[ks][j], ua[ks][i], acc[i][j], 0, 0, 0)
                            : __builtin_amdgcn_mfma_i32_32x32x32_i8(ua[ks][i], ub[ks][j], acc[i][j], 0, 0, 0);
  };

  static_for<NST>([&](auto s) { fill(s.value, s.value); });
  wait_vm_lgkm0<(NST - 1) * LPT>();
  lds_barrier();
  read(IC<0>{}, IC<0>{});
  auto body = [&](int t, auto sidx) {
    constexpr int S = decltype(sidx)::value;
    read(sidx, IC<1>{});
    lgkm_wait<MI + NJ>();   // the first half's fragments, read one step earlier, have arrived
    settle(0);
    __builtin_amdgcn_sched_barrier(0);
    mfmas(0);
    __builtin_amdgcn_sched_barrier(0);
    // the next tile is resident (its fill is the oldest in flight), and every wave is done with this one's stage
    wait_vm_lgkm0<(NST - 2) * LPT>();
    lds_barrier();
    settle(1);
    fill(t + NST, S);
    read(IC<(S + 1) % NST>{}, IC<0>{});   // unused past the last tile
    __builtin_amdgcn_sched_barrier(0);
    mfmas(1);
    __builtin_amdgcn_sched_barrier(0);
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
    // register quad (register r: channel 8 (r/4) + 4 h + r%4, token lane % 32) and finishes them where they are
    float* sc = reinterpret_cast<float*>(smem);   // the tile's channel scales, then its biases
    for (int i = threadIdx.x; i < BN; i += NT) {
      const bool in = n0 + i < a.N;
      sc[i] = in ? a.ws[n0 + i] : 0.f;
      sc[BN + i] = in && a.bias ? to_f32<T>(((const T*)a.bias)[n0 + i]) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int nb = wn * (BN / WN) + 32 * j;
      Cols cols[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        cols[q].ws = *reinterpret_cast<const f32x4*>(sc + nb + 8 * q + 4 * h);
        cols[q].bias = *reinterpret_cast<const f32x4*>(sc + BN + nb + 8 * q + 4 * h);
      }
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int m = m0 + wm * (BM / WM) + 32 * i + (lane & 31);
        const float xs = m < a.M ? a.xs[m] : 0.f;
        f32x4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          v[q] = finish4<ACT, T>(xs, cols[q], i32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                                                    acc[i][j][4 * q + 3]});
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int n = n0 + nb + 8 * q + 4 * h;
            if (m < a.M && n < a.N) store4<float>(a.y, (size_t)m * a.N + n, v[q]);
          }
        } else {
          // the halves of the wave trade quads: each lane stores eight consecutive channels
#pragma unroll
          for (int q = 0; q < 4; q += 2) {
            i32x4 w;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const auto r = __builtin_amdgcn_permlane32_swap(f2bf2(v[q][2 * e], v[q][2 * e + 1]),
                                                              f2bf2(v[q + 1][2 * e], v[q + 1][2 * e + 1]), false, false);
              w[e] = (int)r[0];
              w[2 + e] = (int)r[1];
            }
            const int n = n0 + nb + 8 * q + 8 * h;
            if (m < a.M && n < a.N) *reinterpret_cast<i32x4*>((bf16_t*)a.y + (size_t)m * a.N + n) = w;
          }
        }
      }
    }
    return;
  }

  // more groups: epilogue in MI passes of PR rows: pass p stages block p of every wave row in LDS, one plane per group; each
  // thread then finishes NB chunks of four columns (register r of a 32 x 32 tile: row 8 (r/4) + 4 h + r%4, column
  // lane % 32)
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
        store4<T>(a.y, (size_t)m * a.N + n, finish4<ACT, T>(xs[p][q], cols, v));
      }
    }
  }
}

// ---------------------------------------------------------------- few tokens

// R x R tile (16 or 32) on W waves that share the k range, fragments straight from memory: with few tiles a
// launch is as long as its slowest chain of loads, and here a wave's whole run is in flight at once (8 k-steps
// of 64 bytes at R = 16, 32 at R = 32, then the next 8).  The waves' sums meet in LDS.
template <int R, int W, int ACT, typename T>
__global__ __launch_bounds__(64 * W) void linear8_few_kernel(Linear8 a) {
  constexpr int STEP = R == 16 ? 64 : 32, U = 8, NR = R * R / 64;
  typedef __attribute__((__vector_size__(NR * sizeof(int)))) int accv;
  __shared__ int stg[W][R][R + 4];
  const int lane = threadIdx.x & 63, wave = wave_index(), r = lane % R, h = lane / R;
  const int m0 = blockIdx.y * R, n0 = blockIdx.x * R;
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq, (uint32_t)a.M * (uint32_t)a.K);
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wq, (uint32_t)a.N * (uint32_t)a.K);
  const uint32_t ox = (uint32_t)(m0 + r) * (uint32_t)a.K + 16u * h, ow = (uint32_t)(n0 + r) * (uint32_t)a.K + 16u * h;
  const int steps = a.K / STEP, per = (steps + W - 1) / W, s1 = min(steps, (wave + 1) * per);
  accv acc = {};
  for (int s = wave * per; s < s1; s += U) {
    i32x4 x[U], w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {   // past the run's end: beyond the operands, zeros
      const uint32_t k = s + u < s1 ? (uint32_t)((s + u) * STEP) : 0x80000000u;
      x[u] = buf_load16(rx, ox + k);
      w[u] = buf_load16(rw, ow + k);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (R == 16) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(x[u], w[u], acc, 0, 0, 0);
      else acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(x[u], w[u], acc, 0, 0, 0);
    }
  }
  // register i: row 8 (i/4) + 4 h + i%4 at R = 32, 4 h + i at R = 16; column r
#pragma unroll
  for (int i = 0; i < NR; ++i) stg[wave][R == 16 ? 4 * h + i : 8 * (i >> 2) + 4 * h + (i & 3)][r] = acc[i];
  __syncthreads();
  constexpr int CPR = R / 4;
  for (int c = threadIdx.x; c < R * CPR; c += 64 * W) {
    const int lr = c / CPR, c4 = c % CPR * 4, m = m0 + lr, n = n0 + c4;
    if (m >= a.M || n >= a.N) continue;
    i32x4 v = *reinterpret_cast<const i32x4*>(&stg[0][lr][c4]);
#pragma unroll
    for (int g = 1; g < W; ++g) v += *reinterpret_cast<const i32x4*>(&stg[g][lr][c4]);
    store4<T>(a.y, (size_t)m * a.N + n, finish4<ACT, T>(a.xs[m], load_cols<T>(a, n), v));
  }
}

// ---------------------------------------------------------------- dispatch

enum Shape { kFew16, kFew32, k32x32g8, k64x64g2, k64x128, k128x128, k256x128, k256x256 };

template <int BM, int BN, int WM, int WN, int KG, int NST, int OCC, int ACT, typename T>
hipError_t run_tile(const Linear8& a, hipStream_t st) {
  const int tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  SR_LAUNCH((linear8_tile_kernel<BM, BN, WM, WN, KG, NST, OCC, ACT, T>), dim3((unsigned)(tm * tn)),
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
    case kFew16: return a.K > 1024 ? run_few<16, 16, ACT, T>(a, st) : run_few<16, 4, ACT, T>(a, st);
    case kFew32: return a.K > 1024 ? run_few<32, 16, ACT, T>(a, st) : run_few<32, 4, ACT, T>(a, st);
    case k32x32g8: return run_tile<32, 32, 1, 1, 8, 4, 1, ACT, T>(a, st);
    case k64x64g2: return run_tile<64, 64, 2, 2, 2, 4, 1, ACT, T>(a, st);
    case k64x128: return run_tile<64, 128, 2, 2, 1, 4, 1, ACT, T>(a, st);
    case k128x128: return run_tile<128, 128, 2, 2, 1, 4, 2, ACT, T>(a, st);
    case k256x128: return run_tile<256, 128, 2, 2, 1, 3, 2, ACT, T>(a, st);
    case k256x256: return run_tile<256, 256, 2, 4, 1, 4, 1, ACT, T>(a, st);
  }
  return hipErrorInvalidValue;
}

int pick_shape(const Linear8& a) {
  auto tiles = [&](int bm, int bn) { return (long)((a.M + bm - 1) / bm) * ((a.N + bn - 1) / bn); };
  if (tiles(32, 32) <= 512) return tiles(16, 16) <= 512 ? kFew16 : kFew32;
  if (tiles(64, 64) <= 256) return k64x64g2;
  if (tiles(64, 128) <= 256) return k64x128;
  if (tiles(128, 128) <= 512) return k128x128;
  return k256x128;
}

template <typename T>
hipError_t run(int shape, const Linear8& a, hipStream_t st) {
  return a.act == SR_ACT_GELU ? run_shape<SR_ACT_GELU, T>(shape, a, st) : run_shape<SR_ACT_NONE, T>(shape, a, st);
}

}  // namespace

hipError_t launch_linear8(int dtype, const Linear8& a, hipStream_t st) {
  const int shape = pick_shape(a);
  return dtype == kBF16 ? run<bf16_t>(shape, a, st) : run<float>(shape, a, st);
}

}  // namespace sr
