// Dropout's draws (sr_drop): a bit per value from a counter, the same wherever it is asked for.
#pragma once
#include <math.h>

#include "../../include/sr.h"
#include "common.h"

namespace sr {

constexpr uint64_t kDropGamma = 0x9E3779B97F4A7C15ull;

SR_DEV uint64_t drop_mix(uint64_t z) {   // SplitMix64's output function
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

struct DropArgs {
  uint64_t seed = 0, step = 0, first_row = 0;
  const uint64_t* step_dev = nullptr;
  uint32_t thresh = 0;   // a draw below it is dropped; 0: none is
  float factor = 1.f;    // of the kept values
  int group = 0;
};
inline DropArgs drop_args(const sr_drop& d) {
  DropArgs a;
  a.seed = d.seed; a.step = d.step; a.first_row = d.first_row; a.step_dev = d.step_dev; a.group = d.group;
  a.thresh = (uint32_t)lrint((double)d.p * 65536.0);
  a.factor = a.thresh < 65536u ? (float)(65536.0 / (65536.0 - a.thresh)) : 0.f;
  return a;
}

// The key of a call: wave-uniform, so scalar instructions form it.
SR_DEV uint64_t drop_key(const DropArgs& a) {
  const uint64_t step = a.step + (a.step_dev ? *a.step_dev : 0ull);
  return drop_mix(a.seed + (step + 1ull) * kDropGamma);
}
SR_DEV uint64_t drop_word(uint64_t key, uint64_t w) { return drop_mix(key + (w + 1ull) * kDropGamma); }
// A word is taken apart in halves of 32 bits: a 64-bit shift by a lane's own amount is not safe here in every register (the
// build's scan of the assembly has the case).
SR_DEV bool drop_keep1(uint64_t key, uint64_t e, uint32_t thresh) {
  const uint64_t v = drop_word(key, e >> 2);
  uint32_t lo = (uint32_t)v, hi = (uint32_t)(v >> 32);
  asm("" : "+v"(lo), "+v"(hi));   // or the compiler makes the choice such a shift again
  const uint32_t w = e & 2 ? hi : lo;
  return ((e & 1 ? w >> 16 : w) & 0xFFFFu) >= thresh;
}
// n words of 32 bits from draw e on, of n + 2 that start at a multiple of four draws.
template <int n>
SR_DEV void drop_align(uint32_t (&w)[n + 2], uint64_t e) {
  if (e & 2) {
#pragma unroll
    for (int j = 0; j <= n; ++j) w[j] = w[j + 1];
  }
  if (e & 1) {
#pragma unroll
    for (int j = 0; j < n; ++j) w[j] = __builtin_amdgcn_alignbit(w[j + 1], w[j], 16);
  }
}
// Bit j: draw e + j is kept, j = 0 .. 3.  One word of the generator where e is a multiple of four, else two.
SR_DEV uint32_t drop_keep4(uint64_t key, uint64_t e, uint32_t thresh) {
  const uint64_t v = drop_word(key, e >> 2);
  uint32_t w[4] = {(uint32_t)v, (uint32_t)(v >> 32), 0, 0};
  if (e & 3) {
    const uint64_t top = drop_word(key, (e >> 2) + 1);
    w[2] = (uint32_t)top;
    w[3] = (uint32_t)(top >> 32);
    drop_align<2>(w, e);
  }
  uint32_t keep = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    keep |= (uint32_t)((w[j] & 0xFFFFu) >= thresh) << (2 * j);
    keep |= (uint32_t)((w[j] >> 16) >= thresh) << (2 * j + 1);
  }
  return keep;
}
// Bit j: draw e + j is kept, j = 0 .. 7.  Two words of the generator where e is a multiple of four, else three.
SR_DEV uint32_t drop_keep8(uint64_t key, uint64_t e, uint32_t thresh) {
  const uint64_t lo = drop_word(key, e >> 2), hi = drop_word(key, (e >> 2) + 1);
  uint32_t w[6] = {(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32), 0, 0};
  if (e & 3) {
    const uint64_t top = drop_word(key, (e >> 2) + 2);
    w[4] = (uint32_t)top;
    w[5] = (uint32_t)(top >> 32);
    drop_align<4>(w, e);
  }
  uint32_t keep = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    keep |= (uint32_t)((w[j] & 0xFFFFu) >= thresh) << (2 * j);
    keep |= (uint32_t)((w[j] >> 16) >= thresh) << (2 * j + 1);
  }
  return keep;
}

}  // namespace sr
