// Products of 8-bit floating point with a power of two per block of 128 (sr_linear_f8).
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes the codes as they are and a power of two per lane (its row, its 32 values of k)
// as an exponent byte, so blocks of 128 cost no instruction of their own.  Its sums are fp32, but of eight products that
// it adds at a time it drops what lies 14 bits below the largest: 1.5e-5 of the results' deviation, a hundredth of a
// bf16 result's rounding.  So bf16 results come from it, and fp32 results from products in bf16, which holds codes times
// their powers of two exactly (v_cvt_scalef32_pk_bf16_fp8; 2^-9 of a code times 2^-124 is bf16's smallest number, and in the two
// lower exponents a block can have, values round to its multiples), at half its rate.
//
// Which tile, group or run a product belongs to follows the sizes alone, and every sum has a fixed order.
#include <algorithm>

#include "block_ops.h"
#include "epilogue.h"
#include "tiles.h"

namespace sr {

namespace {

typedef __attribute__((__vector_size__(8 * sizeof(int)))) int i32x8;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight codes times 2^e as bf16 (exact down to e = -124).
SR_DEV bf16x8 decode8(int lo, int hi, float scale) {
  union {
    bf16x2 h[4];
    bf16x8 v;
  } u;
  u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false);
  u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true);
  u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false);
  u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
  return u.v;
}
SR_DEV float scale_of(int e) { return __uint_as_float((uint32_t)e << 23); }

// Explicit LDS read of one byte (see common.h).
template <int OFF>
SR_DEV int rd_u8(uint32_t a) {
  constexpr int HI = OFF & ~0xFFFF;
  int v;
  asm volatile("ds_read_u8 %0, %1 offset:%2" : "=v"(v) : "v"(a + HI), "i"(OFF - HI));
  return v;
}

template <typename T>
SR_DEV float bias_at(const LinearF8& a, int n) {
  return a.bias && n < a.N ? to_f32<T>(((const T*)a.bias)[n]) : 0.f;
}
// Phi is fp32's fit for bf16 results too, so that they are the exact GELU of the sum rounded once: the shorter fit puts 0.23 to 0.5 % of them a
// step away (this one 2e-5) and takes 96.7 instead of 99.0 us at 16200 x 4096 x 1024, 27.7 instead of 29.1 at
// 4050.  ACT is a constant, so that the elements of a lane interleave (16200 x 4096 x 1024: with a branch each 109 us, without 105).
template <int ACT>
SR_DEV float finish(float acc, float bias) {
  const float v = acc + bias;
  return ACT == SR_ACT_GELU ? gelu_lim(v) : v;
}
template <typename O>
SR_DEV void store4(char* p, f32x4 v) {
  if constexpr (sizeof(O) == 4) {
    store16(p, __builtin_bit_cast(i32x4, v));
  } else {
    i32x2 w;
    w[0] = (int)f2bf2(v[0], v[1]);
    w[1] = (int)f2bf2(v[2], v[3]);
    store8(p, w);
  }
}

// ---------------------------------------------------------------- tiles through LDS

// Operand tile of R rows x KB bytes (64 or 128): row r at KB r, its 16-byte chunks at positions c ^ swz(r), so that the 16
// rows of a fragment read's quarter wave cover the 64 banks once.  It is filled by whole 1 KB blocks, straight from memory
// (buffer_load ... lds): lane l lands at byte 16 l of its block and fetches the chunk that the swizzle places there.
template <int KB>
SR_DEV int swz(int r) {
  return (r / (256 / KB)) & (KB / 16 - 1);
}
template <int KB, int BPW>
struct Fill {
  uint32_t off[BPW];
  SR_DEV void init(int r0, uint32_t Kp, int lane, int wid) {
    constexpr int CH = KB / 16, RPB = 64 / CH;
#pragma unroll
    for (int i = 0; i < BPW; ++i) {
      const int row = (wid * BPW + i) * RPB + lane / CH, c = (lane % CH) ^ swz<KB>(row);
      off[i] = (uint32_t)(r0 + row) * Kp + (uint32_t)(c * 16);
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

// BM x BN workgroup tile on WM x WN waves, each MI x NJ tiles of 32 x 32; KG such groups of waves share the tile, each
// with a run of the k range and LDS stages of its own.  NST stages; fills run NST - 1 k-tiles ahead; a wave's exponent bytes,
// which lie side by side in memory, come with them.  Fragment reads are explicit (rd16), so none waits for a
// fill it does not need.  Per k-tile: a k-step's products with the next one's fragment reads under them; before the last
// k-step's the wait for the next tile's fill and the barrier, after which this tile's stage is filled anew and the next
// tile's first fragments are read.  OCC workgroups per CU.  T float: products in bf16, of 32 values of k in a k-step.
template <int BM, int BN, int KB, int WM, int WN, int KG, int NST, int OCC, typename T>
__global__ __launch_bounds__(64 * WM * WN * KG, OCC) void linear_f8_tile_kernel(LinearF8 a, int tiles_m, int tiles_n, int splits) {
  constexpr bool WIDE = sizeof(T) == 4;
  constexpr bool GELU = BM * BN < 256 * 256;   // tiles of 256 x 256 have no registers to spare for it
  constexpr int NW = WM * WN, NT = 64 * NW * KG;
  constexpr int MI = BM / (32 * WM), NJ = BN / (32 * WN);
  constexpr int SB = (BM + BN) * KB;               // bytes of a stage: the token tile, then the weight tile
  constexpr int RPB = 1024 / KB, APW = BM / RPB / NW, BPW = BN / RPB / NW, LPT = APW + BPW + 2;
  constexpr int RPF = WIDE ? 1 : 2, KS = KB / 32 / RPF;   // fragment reads of a k-step, k-steps of a tile
  constexpr int EX = KG * NST * SB;                // the waves' exponents: 256 bytes of rows, 256 of channels, per stage
  static_assert(MI * 32 * WM == BM && NJ * 32 * WN == BN && APW * RPB * NW == BM && BPW * RPB * NW == BN, "whole tiles");
  constexpr int PH = NST * KS % 2 ? 2 * NST : NST;   // k-tiles after which stage and set of fragments recur
  static_assert(NST >= 2 && NST <= 4 && (NST - 1) * LPT < 64 && MI * 32 <= 256 && NJ * 32 <= 256, "counter ranges");
  __shared__ __attribute__((aligned(1024))) char smem[EX + NW * KG * NST * 512];
  __shared__ __attribute__((aligned(16))) float bias[BN];

  const int lane = threadIdx.x & 63, wave = wave_index();
  const int grp = wave / NW, wid = wave % NW;
  const int wm = wid / WN, wn = wid % WN, h = lane >> 5;
  int tm, tn, split;
  tile_coords(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn, split);
  const int m0 = tm * BM, n0 = tn * BN;
  constexpr int TPB = kF8Block / KB;   // k-tiles of a block
  const int kb = (a.K + kF8Block - 1) / kF8Block, per = (kb + splits - 1) / splits * TPB;
  const int k0 = min(split * per, kb * TPB), all = min(per, kb * TPB - k0);   // k-tiles of this run
  const int ntile = (per + KG - 1) / KG;                          // every group runs ntile, the missing ones on zeros
  const int t0 = k0 + grp * ntile, nmine = min(ntile, k0 + all - t0);
  const uint32_t Kp = (uint32_t)kb * kF8Block, Mr = (uint32_t)(a.M + 15) / 16 * 16, Nr = (uint32_t)(a.N + 15) / 16 * 16;
  const __amdgpu_buffer_rsrc_t ra = make_rsrc(a.xq, (uint32_t)a.M * Kp);
  const __amdgpu_buffer_rsrc_t rb = make_rsrc(a.wq, (uint32_t)a.N * Kp);
  const __amdgpu_buffer_rsrc_t rea = make_rsrc(a.xe, Mr * (uint32_t)kb);
  const __amdgpu_buffer_rsrc_t reb = make_rsrc(a.we, Nr * (uint32_t)kb);

  for (int i = threadIdx.x; i < BN; i += NT) bias[i] = splits == 1 ? bias_at<T>(a, n0 + i) : 0.f;
  f32x16 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  Fill<KB, APW> fla;
  Fill<KB, BPW> flb;
  fla.init(m0, Kp, lane, wid);
  flb.init(n0, Kp, lane, wid);
  const uint32_t oea = (uint32_t)(m0 + wm * (BM / WM) + 4 * lane), oeb = (uint32_t)(n0 + wn * (BN / WN) + 4 * lane);
  auto fill = [&](int t, int s) {
    char* st = smem + (grp * NST + s) * SB;
    char* se = smem + EX + (wave * NST + s) * 512;
    const bool in = t < nmine;
    const uint32_t kt = (uint32_t)(t0 + t), delta = in ? kt * KB : 0x80000000u;
    fill_tile<APW>(fla.off, ra, st, wid, delta);
    fill_tile<BPW>(flb.off, rb, st + BM * KB, wid, delta);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rea, (lds_ptr_t*)se, 4, in ? oea + kt / TPB * Mr : 0x80000000u, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(reb, (lds_ptr_t*)(se + 256), 4, in ? oeb + kt / TPB * Nr : 0x80000000u, 0, 0, 0);
  };
  // fragment of rows r .. r + 31, chunk pair c4: lane's row r + lane % 32, chunk 2 c4 + lane / 32; rows 16 apart share
  // the swizzle
  const uint32_t sbase = lds_addr(smem) + (uint32_t)(grp * NST * SB);
  const uint32_t ebase = lds_addr(smem) + (uint32_t)(EX + wave * NST * 512 + (lane & 31));
  uint32_t fa[KB / 32], fb[KB / 32];
#pragma unroll
  for (int c4 = 0; c4 < KB / 32; ++c4) {
    const int r = lane & 31, c = ((2 * c4 + h) ^ swz<KB>(r)) * 16;
    fa[c4] = sbase + (uint32_t)((wm * (BM / WM) + r) * KB + c);
    fb[c4] = sbase + (uint32_t)(BM * KB + (wn * (BN / WN) + r) * KB + c);
  }
  i32x4 ua[2][MI][RPF], ub[2][NJ][RPF];
  int ea[MI], eb[NJ], na[MI], nb[NJ];   // exponents of this tile's rows and channels, and of the next one's
  constexpr int NF = (MI + NJ) * RPF;
  // read F of k-step ks of stage S: the MI token fragments, then the NJ weight fragments
  auto read1 = [&](auto sidx, auto ksv, auto fv) {
    constexpr int G = decltype(sidx)::value, S = G % NST, ks = decltype(ksv)::value, F = decltype(fv)::value / RPF, p = decltype(fv)::value % RPF;
    constexpr int Q = (G * KS + ks) & 1;
    if constexpr (F < MI) ua[Q][F][p] = rd16<S * SB + F * 32 * KB>(fa[ks * RPF + p]);
    else ub[Q][F - MI][p] = rd16<S * SB + (F - MI) * 32 * KB>(fb[ks * RPF + p]);
  };
  auto read_ex = [&](auto sidx, auto fv) {
    constexpr int S = decltype(sidx)::value % NST, F = decltype(fv)::value;
    if constexpr (F < MI) na[F] = rd_u8<S * 512 + F * 32>(ebase);
    else nb[F - MI] = rd_u8<S * 512 + 256 + (F - MI) * 32>(ebase);
  };
  auto settle = [&](auto q) {
    constexpr int Q = decltype(q)::value;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int p = 0; p < RPF; ++p) pin(ua[Q][i][p]);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int p = 0; p < RPF; ++p) pin(ub[Q][j][p]);
  };
  auto settle_ex = [&]() {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      pin(na[i]);
      ea[i] = na[i];
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      pin(nb[j]);
      eb[j] = nb[j];
    }
  };
  // the products of one k-step, with issue(X) after product X: what it issues goes out under the products
  constexpr int NX = MI * NJ * (WIDE ? 2 : 1);
  auto mfmas = [&](auto qv, auto&& issue) {
    constexpr int Q = decltype(qv)::value;
    if constexpr (!WIDE) {
      static_for<MI * NJ>([&](auto x) {
        constexpr int i = decltype(x)::value / NJ, j = decltype(x)::value % NJ;
        const i32x8 xa = __builtin_shufflevector(ua[Q][i][0], ua[Q][i][RPF - 1], 0, 1, 2, 3, 4, 5, 6, 7);
        const i32x8 xb = __builtin_shufflevector(ub[Q][j][0], ub[Q][j][RPF - 1], 0, 1, 2, 3, 4, 5, 6, 7);
        acc[i][j] = KG == 1 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xb, xa, acc[i][j], 0, 0, 0, eb[j], 0, ea[i])
                            : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xa, xb, acc[i][j], 0, 0, 0, ea[i], 0, eb[j]);
        __builtin_amdgcn_sched_barrier(0);
        issue(x);
        __builtin_amdgcn_sched_barrier(0);
      });
    } else {
      static_for<2>([&](auto hv) {   // 16 values of k each
        constexpr int q = decltype(hv)::value;
        bf16x8 da[MI], db[NJ];
#pragma unroll
        for (int i = 0; i < MI; ++i) da[i] = decode8(ua[Q][i][0][2 * q], ua[Q][i][0][2 * q + 1], scale_of(ea[i]));
#pragma unroll
        for (int j = 0; j < NJ; ++j) db[j] = decode8(ub[Q][j][0][2 * q], ub[Q][j][0][2 * q + 1], scale_of(eb[j]));
        static_for<MI * NJ>([&](auto x) {
          constexpr int i = decltype(x)::value / NJ, j = decltype(x)::value % NJ;
          acc[i][j] = KG == 1 ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(db[j], da[i], acc[i][j], 0, 0, 0)
                              : __builtin_amdgcn_mfma_f32_32x32x16_bf16(da[i], db[j], acc[i][j], 0, 0, 0);
          issue(IC<q * MI * NJ + decltype(x)::value>{});
        });
      });
    }
  };

  static_for<NST>([&](auto s) { fill(s.value, s.value); });
  wait_vm_lgkm0<(NST - 1) * LPT>();
  lds_barrier();
  static_for<NF>([&](auto f) { read1(IC<0>{}, IC<0>{}, f); });
  static_for<MI + NJ>([&](auto f) { read_ex(IC<0>{}, f); });
  auto body = [&](int t, auto sidx) {
    constexpr int G = decltype(sidx)::value, S = G % NST;
    static_for<KS - 1>([&](auto ksv) {
      constexpr int ks = decltype(ksv)::value;
      constexpr int Q = (G * KS + ks) & 1;
      lgkm_wait<0>();
      settle(IC<Q>{});
      if constexpr (ks == 0) settle_ex();
      __builtin_amdgcn_sched_barrier(0);
      mfmas(IC<Q>{}, [&](auto x) {
        constexpr int X = decltype(x)::value, F0 = X * NF / NX, F1 = (X + 1) * NF / NX;
        static_for<F1 - F0>([&](auto f) { read1(sidx, IC<ks + 1>{}, IC<F0 + decltype(f)::value>{}); });
      });
    });
    // the next tile is resident (its fill is the oldest in flight), and every wave is done with this one's stage
    wait_vm_lgkm0<(NST - 2) * LPT>();
    lds_barrier();
    constexpr int Q = (G * KS + KS - 1) & 1;
    settle(IC<Q>{});
    if constexpr (KS == 1) settle_ex();
    __builtin_amdgcn_sched_barrier(0);
    mfmas(IC<Q>{}, [&](auto x) {   // reads of the next tile: unused past the last one
      constexpr int X = decltype(x)::value, NA = NF + MI + NJ, F0 = X * NA / NX, F1 = (X + 1) * NA / NX;
      static_for<F1 - F0>([&](auto f) {
        constexpr int F = F0 + decltype(f)::value;
        if constexpr (F < NF) read1(IC<(G + 1) % PH>{}, IC<0>{}, IC<F>{});
        else read_ex(IC<(G + 1) % PH>{}, IC<F - NF>{});
      });
      if constexpr (X == (NX > 1 ? 1 : 0)) fill(t + NST, S);
    });
  };
  for (int t = 0; t < ntile; t += PH)
    static_for<PH>([&](auto s) {
      if (s.value == 0 || t + s.value < ntile) body(t + s.value, s);
    });
  // the last body's reads and fills land before their registers and stages are used again
  lgkm_wait<0>();
  settle(IC<0>{});
  settle(IC<1>{});
  settle_ex();
  wait_vm_lgkm0<0>();
  __syncthreads();

  // Results, as O: the storage type, or fp32 sums of a run (whose bias is zero).
  auto write = [&](auto otype, void* dst, auto actv) {
    typedef decltype(otype) O;
    constexpr int ACT = decltype(actv)::value;
    O* out = (O*)dst;
    const bool past = splits == 1 && past_caches(a.M, a.N, sizeof(O));
    if constexpr (KG == 1) {
      // one group: the weight is the first operand, so that a lane has four consecutive channels of one token in each
      // register quad (register r: channel 8 (r/4) + 4 h + r%4, token lane % 32).  The results go through LDS, IPP blocks of
      // every wave row at a time, so that memory sees whole rows of the tile.
      constexpr int E = sizeof(O), LDB = BN * E + 16, PR = 32 * WM;
      constexpr int FIT = EX / (PR * LDB), IPP = FIT >= MI ? MI : FIT >= 2 && MI % 2 == 0 ? 2 : 1;
      static_assert(IPP * PR * LDB <= EX && MI % IPP == 0, "staging fits the stages");
      constexpr int CPR = BN * E / 16, NB = IPP * PR * CPR / NT;
      static_assert(NB * NT == IPP * PR * CPR, "whole rounds");
#pragma unroll
      for (int p = 0; p < MI; p += IPP) {
        if (p) __syncthreads();
#pragma unroll
        for (int i = 0; i < IPP; ++i) {
          char* row = smem + ((i * WM + wm) * 32 + (lane & 31)) * LDB;
#pragma unroll
          for (int j = 0; j < NJ; ++j) {
            const int nb0 = wn * (BN / WN) + 32 * j;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4 b = *reinterpret_cast<const f32x4*>(bias + nb0 + 8 * q + 4 * h);
              f32x4 v;
#pragma unroll
              for (int r = 0; r < 4; ++r) v[r] = finish<ACT>(acc[p + i][j][4 * q + r], b[r]);
              store4<O>(row + (nb0 + 8 * q + 4 * h) * E, v);
            }
          }
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const int c = threadIdx.x + NT * b, lr = c / CPR, col = c % CPR * (16 / E), blk = lr >> 5;
          const int m = m0 + blk % WM * (BM / WM) + 32 * (p + blk / WM) + (lr & 31), n = n0 + col;
          if (m < a.M && n < a.N) {
            const char* s = smem + lr * LDB + col * E;
            O* o = out + (size_t)m * a.N + n;
            if (n + 16 / E <= a.N) {
              store16(o, *reinterpret_cast<const i32x4*>(s), past);
            } else {
#pragma unroll
              for (int r = 0; r < 16 / E; ++r)
                if (n + r < a.N) o[r] = reinterpret_cast<const O*>(s)[r];
            }
          }
        }
      }
    } else {
      // more groups: MI passes of PR rows.  Pass p stages block p of every wave row in LDS, one plane per group; each
      // thread then adds up NB chunks of four columns (register r: row 8 (r/4) + 4 h + r%4, column lane % 32)
      float* stg = reinterpret_cast<float*>(smem);
      constexpr int PR = 32 * WM, LD = BN + 8, CPR = BN / 4, NB = (PR * CPR + NT - 1) / NT;
      static_assert(KG * PR * LD * 4 <= EX, "staging fits the stages");
#pragma unroll
      for (int p = 0; p < MI; ++p) {
        if (p) __syncthreads();
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            stg[(grp * PR + wm * 32 + 8 * (r >> 2) + 4 * h + (r & 3)) * LD + wn * (BN / WN) + j * 32 + (lane & 31)] = acc[p][j][r];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < NB; ++q) {
          const int c = threadIdx.x + NT * q, lr = c / CPR, c4 = c % CPR * 4;
          const int m = m0 + (lr >> 5) * (BM / WM) + p * 32 + (lr & 31), n = n0 + c4;
          if (lr < PR && m < a.M && n < a.N) {
            f32x4 v = *reinterpret_cast<const f32x4*>(stg + lr * LD + c4);
#pragma unroll
            for (int g = 1; g < KG; ++g) v += *reinterpret_cast<const f32x4*>(stg + (g * PR + lr) * LD + c4);
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = finish<ACT>(v[r], bias[c4 + r]);
            O* o = out + (size_t)m * a.N + n;
            if (n + 4 <= a.N) {
              store4<O>((char*)o, v);
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (n + r < a.N) o[r] = from_f32<O>(v[r]);
            }
          }
        }
      }
    }
  };
  if (splits > 1) write(float{}, a.scratch + (size_t)split * a.M * a.N, IC<SR_ACT_NONE>{});
  else if (!GELU || a.act == SR_ACT_NONE) write(T{}, a.y, IC<SR_ACT_NONE>{});
  else if constexpr (GELU) write(T{}, a.y, IC<SR_ACT_GELU>{});
}

// The sums of `splits` runs, in order, finished.
template <typename T>
__global__ __launch_bounds__(256) void linear_f8_join_kernel(LinearF8 a, int splits) {
  const int64_t n = (int64_t)a.M * a.N;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    float v = a.scratch[i];
    for (int s = 1; s < splits; ++s) v += a.scratch[s * n + i];
    const float b = bias_at<T>(a, (int)(i % a.N));
    ((T*)a.y)[i] = from_f32<T>(a.act == SR_ACT_GELU ? finish<SR_ACT_GELU>(v, b) : finish<SR_ACT_NONE>(v, b));
  }
}

// ---------------------------------------------------------------- few tokens

// 16 x 16 tile on W waves that share the k range, fragments straight from memory (lane: row lane % 16, 32 bytes of k):
// with few tiles a launch is as long as its slowest chain of loads, and here a wave has its next U blocks in flight at
// once.  The waves' sums meet in LDS.
template <int W, typename T>
__global__ __launch_bounds__(64 * W) void linear_f8_few_kernel(LinearF8 a) {
  constexpr int U = 4;
  __shared__ float stg[W][16][20];
  const int lane = threadIdx.x & 63, wave = wave_index(), r = lane & 15, h = lane >> 4;
  const int tiles_n = (a.N + 15) / 16;
  const int m0 = (int)(blockIdx.x / (unsigned)tiles_n) * 16, n0 = (int)(blockIdx.x % (unsigned)tiles_n) * 16;
  const int kb = (a.K + kF8Block - 1) / kF8Block, per = (kb + W - 1) / W, b1 = min(kb, (wave + 1) * per);
  const uint32_t Kp = (uint32_t)kb * kF8Block, Mr = (uint32_t)(a.M + 15) / 16 * 16, Nr = (uint32_t)(a.N + 15) / 16 * 16;
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.xq, (uint32_t)a.M * Kp), rw = make_rsrc(a.wq, (uint32_t)a.N * Kp);
  const __amdgpu_buffer_rsrc_t rex = make_rsrc(a.xe, Mr * (uint32_t)kb), rew = make_rsrc(a.we, Nr * (uint32_t)kb);
  const uint32_t ox = (uint32_t)(m0 + r) * Kp + 32u * h, ow = (uint32_t)(n0 + r) * Kp + 32u * h;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int b = wave * per; b < b1; b += U) {
    i32x4 x[U][2], w[U][2];
    int ex[U], ew[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {   // past the run's end: beyond the operands, zeros
      const bool in = b + u < b1;
      const uint32_t k = in ? (uint32_t)(b + u) * kF8Block : 0x80000000u;
      ex[u] = __builtin_amdgcn_raw_buffer_load_b8(rex, in ? (uint32_t)(b + u) * Mr + m0 + r : 0x80000000u, 0, 0);
      ew[u] = __builtin_amdgcn_raw_buffer_load_b8(rew, in ? (uint32_t)(b + u) * Nr + n0 + r : 0x80000000u, 0, 0);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        x[u][p] = buf_load16(rx, ox + k + 16u * p);
        w[u][p] = buf_load16(rw, ow + k + 16u * p);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_shufflevector(x[u][0], x[u][1], 0, 1, 2, 3, 4, 5, 6, 7),
                                                               __builtin_shufflevector(w[u][0], w[u][1], 0, 1, 2, 3, 4, 5, 6, 7),
                                                               acc, 0, 0, 0, ex[u], 0, ew[u]);
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              decode8(x[u][q >> 1][2 * (q & 1)], x[u][q >> 1][2 * (q & 1) + 1], scale_of(ex[u])),
              decode8(w[u][q >> 1][2 * (q & 1)], w[u][q >> 1][2 * (q & 1) + 1], scale_of(ew[u])), acc, 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) stg[wave][4 * h + i][r] = acc[i];   // register i: row 4 h + i, column r
  __syncthreads();
  for (int i = threadIdx.x; i < 256; i += 64 * W) {
    const int lr = i >> 4, lc = i & 15, m = m0 + lr, n = n0 + lc;
    if (m < a.M && n < a.N) {
      float v = stg[0][lr][lc];
#pragma unroll
      for (int g = 1; g < W; ++g) v += stg[g][lr][lc];
      const float b = bias_at<T>(a, n);
      ((T*)a.y)[(size_t)m * a.N + n] = from_f32<T>(a.act == SR_ACT_GELU ? finish<SR_ACT_GELU>(v, b) : finish<SR_ACT_NONE>(v, b));
    }
  }
}

// ---------------------------------------------------------------- dispatch

enum Shape { kFew, k32, k64, k64x128, k128, k128x2, k256x128, k256 };
struct Plan {
  Shape shape;
  int splits;
};

int64_t tiles_of(int M, int N, int bm, int bn) { return ((int64_t)(M + bm - 1) / bm) * ((N + bn - 1) / bn); }

// The smallest tile whose grid is one round of workgroups on the 256 CUs, past it those that read LDS least; long rows
// with few tiles are cut into runs.  The borders between are where a grid no longer is one round, and numbers of blocks of k picked where two
// shapes met; over 240 sizes of 1 to 16384 tokens, 16 to 4096 channels and 64 to 16384 of k, the shape that it picks is 1.3 % (bf16)
// and 0.9 % (fp32) behind the fastest of all on average, 9 and 7 % at the 95th of a hundred, 21 % at most (91 x 210 x 5071).  us, M x N x K, bf16 results (fp32 where it says so, with two or four groups of waves that
// share the tile, since decoding for 64 x 64 per wave costs least):
//   fragments straight from memory, up to one 16 x 16 tile per CU:  1 x 4096 x 1024 3.5 (32 x 32 in eight groups 4.5),
//   1 x 1024 x 4096 4.3 (5.9), 64 x 1024 x 1024 3.8 (4.3);  past it 128 x 1024 x 4096 9.3 (6.1)
//   32 x 32, eight groups:  128 x 1024 x 4096 6.1 (64 x 64 9.1), fp32 512 x 512 x 4096 8.0 (11.1), 276 x 256 x 4083 7.0 (9.4);
//   in four runs 256 x 256 x 16200 11.4 (one 19.5), in six 64 x 64 x 16200 9.4 (15.3)
//   64 x 64:  1024 x 1024 x 1024 5.5 (64 x 128 6.2, 128 x 128 7.7);  fp32 1024 x 1024 x 4050 14.8 (128 x 128 in two runs 21.2), in four
//   runs 256 x 1024 x 16200 18.5 (32 x 32 20.4)
//   64 x 128:  2048 x 1024 x 1024 6.5 (64 x 64 7.6, 128 x 128 8.0), 2013 x 1024 x 256 4.9 (5.1)
//   128 x 128, four stages:  4050 x 1024 x 1024 9.3 (two workgroups per CU 10.1);  4083 x 1024 x 256 6.4 (5.8);  fp32, two
//   groups, 1024 x 4096 x 16200 109 (256 x 128 in two runs 117, two workgroups 122), 4096 x 1024 x 4050 34 (39); in four runs
//   1024 x 1024 x 16200 39 (64 x 64 49, one run 101)
//   256 x 128:  8192 x 1024 x 1024 13.9 (128 x 128 14.6, 256 x 256 18.9)
//   256 x 256:  16200 x 4096 x 1024 80 (86), 16200 x 1024 x 4096 57 (67), 4050 x 4096 x 1024 23.7 (24.5);  with GELU or fp32 results two
//   workgroups of 256 x 128 in three stages of 64 bytes: 16200 x 4096 x 1024 with GELU 97 - 100 (128 x 128 110), fp32 122 (256 x 256 130)
Plan plan_of(int M, int N, int K) {
  auto tiles = [&](int bm, int bn) { return tiles_of(M, N, bm, bn); };
  const int kb = (K + kF8Block - 1) / kF8Block;
  const int64_t t16 = tiles(16, 16), t32 = tiles(32, 32), t64 = tiles(64, 64), t128 = tiles(128, 128);
  // runs of a row: as many as fill the CUs, of 20 blocks or more
  auto runs = [&](int64_t t) { return (int)std::max<int64_t>(1, std::min<int64_t>(256 / t, kb / 20)); };
  if (t16 <= 256 && kb <= 64 && (kb <= 32 || M <= 64)) return {kFew, 1};
  if (t32 <= 256 && kb >= 4 && (t32 <= 128 || kb < 64)) return {k32, runs(t32)};
  if (t64 <= 256 && (kb < 96 || t128 < 32)) return {k64, runs(t64)};
  if (kb < 96 && tiles(64, 128) <= 256) return {k64x128, 1};
  if (t128 <= 256) return {kb >= 4 ? k128 : k128x2, runs(t128)};
  if (kb >= 8 && tiles(256, 128) <= 256) return {k256x128, 1};
  if (kb >= 8 && tiles(256, 256) >= 200) return {k256, 1};
  return {k128x2, 1};
}

template <int BM, int BN, int KB, int WM, int WN, int KG, int NST, int OCC, typename T>
hipError_t run_tile(const LinearF8& a, int splits, hipStream_t st) {
  const int tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  SR_LAUNCH((linear_f8_tile_kernel<BM, BN, KB, WM, WN, KG, NST, OCC, T>), dim3((unsigned)tm * (unsigned)tn * (unsigned)splits),
            dim3(64 * WM * WN * KG), 0, st, a, tm, tn, splits);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  const int64_t wgs = std::min<int64_t>(((int64_t)a.M * a.N + 255) / 256, 4096);
  SR_LAUNCH((linear_f8_join_kernel<T>), dim3((unsigned)wgs), dim3(256), 0, st, a, splits);
  return hipGetLastError();
}
template <typename T>
hipError_t run(const LinearF8& a, hipStream_t st) {
  constexpr bool WIDE = sizeof(T) == 4;
  const Plan p = plan_of(a.M, a.N, a.K);
  const int s = p.splits;
  switch (p.shape) {
    case kFew: {   // more waves than blocks of a row would have nothing to do, but cost nothing (1 x 4096 x 1024: four 4.2, eight 3.5 us)
      SR_LAUNCH((linear_f8_few_kernel<8, T>), dim3((unsigned)tiles_of(a.M, a.N, 16, 16)), dim3(512), 0, st, a);
      return hipGetLastError();
    }
    case k32: return run_tile<32, 32, 128, 1, 1, 8, 2, 1, T>(a, s, st);
    case k64:   // longer rows in more stages, or groups (512 x 1024 x 4096 13.2 -> 9.9 us; x 1024 5.1, 5.4)
      if (a.K <= 2048) return run_tile<64, 64, 128, 2, 2, 2, 2, 2, T>(a, s, st);
      if constexpr (WIDE) return run_tile<64, 64, 128, 2, 2, 4, 2, 1, T>(a, s, st);
      else return run_tile<64, 64, 128, 2, 2, 2, 4, 1, T>(a, s, st);
    case k64x128: return run_tile<64, 128, 128, 2, 4, 1, 4, 1, T>(a, s, st);
    case k128:
      if constexpr (WIDE) return run_tile<128, 128, 128, 2, 2, 2, 2, 1, T>(a, s, st);
      else return run_tile<128, 128, 128, 2, 4, 1, 4, 1, T>(a, s, st);
    case k128x2: return run_tile<128, 128, 128, 2, 4, 1, 2, 2, T>(a, s, st);
    case k256x128: return run_tile<256, 128, 128, 4, 2, 1, 3, 1, T>(a, s, st);
    case k256:
      // decoding and GELU are vector work, under which a second workgroup's products run
      if (WIDE || a.act == SR_ACT_GELU) return run_tile<256, 128, 64, 2, 2, 1, 3, 2, T>(a, s, st);
      if constexpr (!WIDE) return run_tile<256, 256, 128, 2, 4, 1, 2, 1, T>(a, s, st);
      break;
  }
  return hipErrorInvalidValue;
}

}  // namespace

size_t linear_f8_need(int M, int N, int K) {
  const Plan p = plan_of(M, N, K);
  return p.splits == 1 ? 0 : (size_t)p.splits * M * N * sizeof(float);
}

// The most that a product of these sizes or smaller ones needs (more tiles leave fewer runs, and none past a tile per CU): runs of 20
// blocks or more, on 256 tiles at most with all runs, of 32 x 32 up to 128 of these and of 128 x 128 at most beyond.
size_t linear_f8_scratch(int M, int N, int K) {
  const int64_t runs = (K + kF8Block - 1) / kF8Block / 20, side = tiles_of(M, N, 32, 32) <= 128 ? 32 : 128;
  return runs < 2 ? 0 : (size_t)std::min(runs * M * N, 256 * side * side) * sizeof(float);
}

hipError_t launch_linear_f8(int dtype, const LinearF8& a, hipStream_t st) {
  return dtype == kBF16 ? run<bf16_t>(a, st) : run<float>(a, st);
}

}  // namespace sr
