// Which kernel form computes a block-scaled E4M3 product. Host code without any device's, so that the choice can be
// looked at for any size.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace xs {
namespace f8 {

constexpr uint32_t kNone = 1u << 30;   // an offset past every buffer of the split form; twice it does not wrap

enum Form { kSplit12, kSplit21, kSplit22, kSplit24, kSplit44, kLow, kDeep, kMid, kBig };

// The cheapest form by a model of its time in us, from M, N, K and the CU count (n_seg > 0: grouped, with
// exponential segment lengths, n / (1 - exp(-rows n / M)) row blocks of n segments). A split form takes its rounds of
// workgroups, each a start and a join that grow with its outputs, and its rows of K bytes at the rate of a
// CU's memory path; tiles take K / 128 blocks a round, of one 256 x 256, up to two 128 x 128 or one tile of four
// stages a CU. Weights past the caches (grouped products that touch over 100 MB) come more slowly. Measured, us,
// split 1x2 / 2x4 / 4x4, 64 x 128 and 128 x 128 of four stages, 128- and 256-tiles, N = 4096, K = 7168:
//   M = 24  8.4 / 12.0 / 16.8 / 25 / 24 / 37 / 71        M = 128  26 / 13.3 / 18.1 / 25.6 / 27.8 / 42 / 71
//   M = 512  93 / 46 / 35 / 27.2 / 28.3 / 43 / 74        M = 1024  - / 86 / 67 / 52 / 35.7 / 44 / -
//   M = 2048  - / 171 / 131 / 101 / 71 / 62 / 82         M = 4093  - / - / - / 198 / 146 / 134 / 105
//   K = 1024: M = 512  - / 16.3 / 12.6 / 8.3 / 9.2 / 11.1 / -
// 32 segments with SwiGLU: 64 rows in all  137 / 128 / 137 / 127 / 129 / 143 / 178; 1024  342 / 211 / 197 / 170 /
// 163 / 159 / 189; 8192  - / 909 / 701 / 496 / 371 / 346 / 323.
inline Form choose_form(double cus, int M, int N, int K, int64_t ldb_s, int n_seg, bool swiglu, bool f32) {
  const bool grouped = n_seg > 0;
  if (!grouped) n_seg = 1;
  const double nk = K / 128, n_out = swiglu ? N / 2 : N;
  const double segs = std::min(n_seg, M);
  const auto blocks = [&](int rows) {
    return segs > 1 ? std::ceil(segs / (1 - std::exp(-rows * segs / M))) : std::ceil(static_cast<double>(M) / rows);
  };
  const bool far = segs * N * K > 100e6 && grouped;
  double best = 1e300;
  Form form = kMid;
  const auto offer = [&](Form f, double us) {
    if (us < best) {
      best = us;
      form = f;
    }
  };
  // offsets of the split form's buffers stay below kNone, its column blocks (of 16 or more, 256 threads) in a
  // grid's first dimension of 2^32 - 1 threads, its row blocks in the second
  if ((n_out / 128 + 1) * ldb_s * 4 < kNone && N < (1 << 28)) {
    constexpr int forms[5][2] = {{1, 2}, {2, 1}, {2, 2}, {2, 4}, {4, 4}};
    const double rate = f32 ? 55e3 : far ? 47e3 : 70e3;
    for (int f = 0; f < 5; ++f) {
      const int rows = 16 * forms[f][0], cols = 16 * forms[f][1];
      if ((swiglu && f == kSplit21) || static_cast<double>(M) / rows + n_seg > 65535) continue;   // gate and up take two blocks
      const double wgs = blocks(rows) * std::ceil(N / static_cast<double>(cols));
      const double idle = (static_cast<double>(M) / rows + n_seg) * std::ceil(N / static_cast<double>(cols)) - wgs;
      offer(static_cast<Form>(f), 2 + (grouped ? 0.5 * std::max(0.0, idle) / cus : 0) + std::ceil(wgs / cus) * (1.45 + 5.5e-4 * rows * cols + (rows + cols) * static_cast<double>(K) / rate));
    }
  }
  const auto tiles = [&](int bm, int bn) { return blocks(bm) * std::ceil(N / static_cast<double>(bn)); };
  const double mid = tiles(128, 128), rest = std::fmod(mid, 2 * cus) / cus;
  const double part = rest == 0 ? 0 : rest <= 1 ? 0.62 : 0.62 + 0.48 * (rest - 1);
  offer(kMid, 6 + nk * (std::floor(mid / (2 * cus)) * 1.1 + part) * (f32 ? 1.75 : far ? 1.2 : 1));
  if (!f32) {                                            // exact sums do not fit its registers
    // one tile a CU at a time; grouped, a round's end is not the same for all, half a round lost on the average
    const auto lone = [&](Form f, int rows, double start, double per, double full, double far_per) {
      const double nt = std::ceil(N / 128.);
      double us = 0;
      if (segs > 1) {
        const double x = segs / (1 - std::exp(-rows * segs / M)) * nt / cus, rounds = x <= 1.05 ? 1 : x + 0.5;
        us = start + nk * (far ? far_per : full) * rounds + 5 * (rounds - 1);
      } else {
        const double x = blocks(rows) * nt / cus, whole = std::floor(x), rest = x - whole;
        us = start + nk * (whole * full + (rest == 0 ? 0 : per + (full - per) * std::max(0., 2 * rest - 1))) + 5 * (std::ceil(x) - 1);
      }
      offer(f, us);
    };
    lone(kLow, 64, 5.2, 0.37, 0.395, 0.56);
    lone(kDeep, 128, 6.3, 0.38, 0.51, 0.62);
    const double big = tiles(256, 256), left = std::fmod(big, cus) / cus;
    offer(kBig, 6 + nk * (std::floor(big / cus) * 1.85 + (left == 0 ? 0 : 1.25 + 0.6 * left)));
  }
  return form;
}

}  // namespace f8
}  // namespace xs
