// Host-side choices that the plans of the two-model losses (kd_api.hip) and of the one-head losses (kd_head_api.hip) share.
#pragma once
#include "kd_launch.h"

namespace kd {

inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Vocabulary chunk of the backward pass.  The [T_pad, V_c] bf16 staging buffer of dL/dz_s is written by the gradient
// kernel and read back by both products; it should stay in the 256 MB last-level cache together with the operands, but every chunk also
// costs the ends of three launches and re-reads and re-writes the fp32 sums of grad_h_s.
//  - From 4096 tokens on 16384 columns, halved until the staging buffer is within 512 MiB (at least 1024).  Against 8192 columns, means of
//    steps with all tokens and with a tenth masked, 59 sizes, FKL and JSD, T = 4190 .. 16384, V = 54032 .. 151936: 0.966 of the time where
//    the buffer stays in the cache (up to 6656 tokens; 12 sizes, 0.90 .. 0.99), beyond 0.971 with up to 6144 elements contracted for a
//    logit (13 sizes, 0.93 .. 1.00) and 0.991 with more (34 sizes, 0.966 .. 1.013), whose products hide a chunk's ends best.  What a size
//    gains or loses follows the rounds of workgroups: T = 8192, H = 8192 / 2048, V = 128256 38.4 -> 37.0 ms with all tokens, 34.7 -> 34.9
//    with a tenth masked, two teachers, H = 4096 + 2048 / 1024, V = 151936 36.3 -> 34.7; fp32, T = 16384, H = 2048 / 1024, V = 32000
//    15.9 -> 16.0.  (The rounds as priced below would take 16384 at every one of the 59.)  12288 columns: 0.970, 0.991, 0.993.
//    Past 512 MiB wider chunks lose (T = 32768, H = 5120 / 4096, JSD 262.6 -> 265.4).  (At 4096 tokens 24576 columns, 201 MB, measured 11.72
//    against 12.25 ms without a mask on an earlier state; tests/test_abi_host.py holds that size to 16384 columns.)
//  - Below, up to 208 MiB (201 MB still stays in the cache), and the width decides how full the last rounds of
//    workgroups are: the candidates (multiples of the tile heights) are priced by the rounds of the gradient kernel,
//    with all tokens and with an eighth of them masked, and of the grad_W_s product.  Measured steps: T = 3584 10.60 ms
//    with 24576 columns against 10.78 with 16384; T = 2048 6.03 with 49152 against 6.25 with 32768; T = 1024 3.28 with
//    98304 against 3.34 with 65536.
// `logit_k`: elements contracted for one logit of every model of the call (each teacher with the student again).
inline int64_t choose_chunk(const Problem& q, int64_t v_all, int64_t logit_k) {
  if (q.T_pad >= 4096) {
    int64_t vc = 16384;
    while (vc > 1024 && (int64_t)q.T_pad * vc * 2 > (512ll << 20)) vc >>= 1;
    return vc;
  }
  const int64_t step = 1536, most = (208ll << 20) / (2 * q.T_pad);      // a multiple of 192, 256 and 128
  if (most >= v_all) return v_all;
  const int tile_m = q.strip ? 192 : kTileM, masked_tt = (q.n_tt * 7 + 7) / 8;
  // (the grad_W_s tile that covers H_s cheapest, whatever the width; priced by each width's own, grad_W_tile, a twelfth of the widths
  // below 4096 tokens change, for the worse as often as for the better: T = 1764, H = 576, V = 151936 1.59 -> 1.68 ms, T = 2880,
  // H = 512 / 192 1.63 -> 1.57)
  int64_t gw_rows = 256;
  auto cover = [&](int64_t rows) { return (q.H_s + rows - 1) / rows * (rows + 48); };
  for (int64_t rows : {192, 128}) if (cover(rows) < cover(gw_rows)) gw_rows = rows;
  const int64_t m_tiles = (q.H_s + gw_rows - 1) / gw_rows;
  // multiply-adds of one workgroup: a logit tile, a grad_W_s tile, and what a chunk costs besides (three launches
  // and the sums of grad_h_s: 20 us and 8 bytes per element at 5 TB/s, at 2.6e12 a second)
  const double logit = (double)tile_m * kTileN * (double)logit_k;
  const double gw = (double)gw_rows * 256. * q.T_pad;
  const double fixed = 52e6 + (double)q.T * q.H_s * 4.2;
  auto cost = [&](int64_t width) {
    const int64_t n = (width + tile_m - 1) / tile_m;
    auto rounds = [&](int64_t tiles) { return (double)((tiles + q.n_cu - 1) / q.n_cu); };
    return logit * 0.5 * (rounds(n * q.n_tt) + rounds(n * masked_tt)) + gw * rounds((width + 255) / 256 * m_tiles) + fixed;
  };
  int64_t best = step;
  double best_cost = 1e300;
  for (int64_t vc = step; vc <= most; vc += step) {
    const int64_t full = q.V / vc, rest = q.V - full * vc;
    const double c = (double)full * cost(vc) + (rest > 0 ? cost(rest) : 0.);
    if (c <= best_cost) { best_cost = c; best = vc; }
  }
  return best;
}

// Tile and split-K of the grad_h_s product: the tiles of every chunk are rounds of n_cu workgroups, each of so many k-steps of 64
// columns (the last chunk has those of the first, in fewer parts); 1.47, 1.19, 0.85, 0.62 us a k-step for 256, 192, 128, 64 hidden
// rows (1.43 PFLOP/s down to 0.85); where the chunk of dz and of the head is more than the last-level cache keeps, the smaller tiles,
// which have less in flight, take longer; 1.7 us a tile to start and 8.5 us per 256 rows to write its sums, 24 us with reading
// them where there are several chunks; and every part is read once more at the end of the call (3.4 TB/s).  The mean of all tokens and
// of an eighth of them masked, as in choose_chunk.  Fitted to 516 sizes, T = 100 .. 16384, H_s = 128 .. 4096, both head orders, each
// with up to 18 tiles and splits (product and gradh_finish), and 180 more: 0.6 % behind the best one of each on average (2.5 % and more
// with the last chunk and the cache left out).  T = 4096, H_s = 1024, V = 151936 128 rows x 2 parts 1123 us a call, 256 x 4 1213; T = 1024 256 x 16 353 us,
// 128 x 8 372, 128 x 16 312; T = 512 256 x 32 142 us, 128 x 16 159.
// `products`: so many that are summed, each with parts of its own (GradHPairs).
inline void plan_grad_h(Problem& q, bool lean, int products = 1) {
  const int first_width = (int)(q.V < q.V_c ? q.V : q.V_c), steps_first = (first_width + 63) / 64;
  const int full_chunks = q.V / first_width, last_width = q.V - full_chunks * first_width;
  double least = 1e300;
  int sk = 1;
  for (int rows = lean ? 128 : 256; rows >= 64; rows -= 64) {
    if (q.w_hv_inplace && q.V > (1 << 23) && rows > 128) continue;              // (32-bit offsets: rows of 2 V bytes)
    const int i = rows / 64 - 1;
    const double in_cache[] = {0.62, 0.85, 1.19, 1.47}, from_memory[] = {0.82, 0.98, 1.26, 1.47};
    const double ends = 1.7 + rows / 256. * (q.V > q.V_c ? 24. : 8.5);
    const int64_t h_tiles = (q.H_s + rows - 1) / rows * products, tiles = h_tiles * q.n_tt, masked_tiles = h_tiles * ((q.n_tt * 7 + 7) / 8);
    auto rounds = [&](int64_t n) { return (double)((n + q.n_cu - 1) / q.n_cu); };
    for (int s = 1; s <= 32 && (s == 1 || q.V_c / s >= 512) && s <= steps_first; ++s) {
      if (lean && s > 1 && s * tiles > q.n_cu) break;
      const int steps = (steps_first + s - 1) / s;
      auto chunk = [&](int width) {
        const int n = (width + 63) / 64, parts = (n + steps - 1) / steps;
        const double step = 2. * width * (double)(q.T_pad + q.H_s) > 240e6 ? from_memory[i] : in_cache[i];
        return 0.5 * (rounds(tiles * parts) + rounds(masked_tiles * parts)) * ((steps < n ? steps : n) * step + ends);
      };
      const double t = full_chunks * chunk(first_width) + (last_width > 0 ? chunk(last_width) : 0.) +
                       (double)((steps_first + steps - 1) / steps) * q.T * q.H_s * products * 1.17e-6;
      if (t < least) { least = t; q.gh_rows = rows; sk = s; }
    }
  }
  q.ksteps_h = (steps_first + sk - 1) / sk;
  q.n_ksplit_h = (steps_first + q.ksteps_h - 1) / q.ksteps_h;   // every part is written by the first chunk
}

}  // namespace kd
