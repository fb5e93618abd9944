// The rules that choose kernels and launch shapes of the int8 product by sizes (plain C++; vnm_spmm_i8*.hip).
#pragma once
#include <stdint.h>

namespace vnm {

// What one launch of the many-token kernels takes: 65535 workgroups in y and 2^32 threads (the product's workgroups have 512 at
// most: tiles of 128 tokens in x, groups of 4 or 8 row blocks in y); more goes in ranges, one launch each.
constexpr int64_t kI8GridY = 65535, kI8GridTiles = 1 << 22, kI8GridRows = 4 * kI8GridY;

// A launch shape of the few-token kernel: 32-row tiles and tokens per workgroup, waves that cut K between them.
struct I8FewShape { int tiles, tokens, waves; };

// Estimated time, in us, of the few-token kernel: workgroups come in rounds of 256, one per compute unit; a round has a fixed part
// (first loads, sums over the waves, stores) and a part per K step, set by the loads that a wave issues (weights: 4 or 5 per
// step; activations: tokens x M / 64) and the byte permutations (two per block for M > 8).  Fitted to 4096 x 4096 at M = 5 and 16,
// 11008 x 4096 and 2304 x 768 at M = 8, 1 to 2048 tokens, four waves; estimated / measured: 4096 x 4096, M = 5, 16 tokens
// 5.5 / 7.0, 512 tokens at 16 per workgroup 50 / 45, at 32 34 / 31, at 32 on two tiles 23.3 / 20.6.  Over 60 random products
// the choice costs 4 % against the fastest of all shapes in the mean.
inline double i8_few_us(I8FewShape s, int64_t T, int64_t R64, int64_t S, int M) {
  const double fixed = s.tiles == 2 ? 1.5 : s.tokens == 32 ? 1.2 : 0.9;
  const double step = s.tiles == 2 ? (0.048 + 0.0046 * M) * (M > 8 ? 1.27 : 1.0) : s.tokens == 32 ? (M > 8 ? 0.112 : 0.053) : M > 8 ? 0.06 : 0.04;
  const int64_t groups = (T + s.tokens - 1) / s.tokens, wgs = (s.tiles == 2 ? R64 : 2 * R64) * groups;
  return 2.5 + (double)((wgs + 255) / 256) * (fixed + step * (double)S);
}
inline I8FewShape i8_few_shape(int64_t T, int64_t R64, int64_t S, int M) {
  // Eight waves where K is long and half of the compute units would be idle: 4096 x 11008, M = 5 at 1 / 16 tokens 7.6 / 9.0 us
  // with eight, 8.6 / 12.4 with four; 4096 x 4096 (52 steps), which keeps four, 5.2 / 5.9 and 5.4 / 7.0.
  const int waves = S >= 96 && 2 * R64 <= 128 ? 8 : 4;
  // Groups of four tokens where all of their workgroups run at once: 176 x 5416, M = 5, 8 tokens 5.6 us, in one group of 16 6.3;
  // 144 x 2424, M = 4, 25 tokens 4.7 and 4.8
  if (T <= 4 || (T <= 32 && 2 * R64 * ((T + 3) / 4) <= 256)) return {1, 4, waves};
  if (T <= 16) return {1, 16, waves};
  I8FewShape best = {1, 16, waves};
  const I8FewShape others[] = {{1, 32, waves}, {2, 32, 4}};
  for (const I8FewShape& s : others)
    if (i8_few_us(s, T, R64, S, M) < i8_few_us(best, T, R64, S, M)) best = s;
  return best;
}

// Workgroups of 8 row blocks (otherwise 4, cutting K in two): where more than half of the compute units get one
inline bool i8_staged_wide(int64_t tiles, int64_t R64) { return R64 >= 8 && tiles * ((R64 + 7) / 8) > 128; }
// Estimated time of staging and product: launches, prologue and store; bytes staged; K steps of each round.  4096 x 4096, M = 5,
// estimated / measured: 256 tokens 25.5 / 25.3, 700 26.4 / 27.5, 4096 46.4 / 48.2.
inline double i8_staged_us(int64_t T, int64_t R64, int64_t in, int64_t S) {
  const int64_t tiles = (T + 127) / 128;
  const bool wide = i8_staged_wide(tiles, R64);
  const int64_t wgs = tiles * (wide ? (R64 + 7) / 8 : (R64 + 3) / 4), steps = wide ? S : (S + 1) / 2;
  return 12.0 + (double)(T * in) * 5e-7 + (double)((wgs + 255) / 256) * (double)steps * 0.5;
}
inline bool i8_takes_few(int64_t T, int64_t R64, int64_t in, int64_t S, int M) {
  if (T <= 128) return true;
  if (T > 4 * 65535) return false;                          // (its grid)
  return i8_few_us(i8_few_shape(T, R64, S, M), T, R64, S, M) < i8_staged_us(T, R64, in, S);
}

}  // namespace vnm
