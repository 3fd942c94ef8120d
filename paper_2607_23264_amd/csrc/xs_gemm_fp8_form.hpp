// Which kernel form computes a block-scaled E4M3 product. Host code without any device's, so that the choice can be
// looked at for any size.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace xs {
namespace f8 {

constexpr uint32_t kNone = 1u << 30;   // an offset past every buffer of the split form; twice it does not wrap

enum Form { kSplit12, kSplit22, kSplit24, kSplit44, kLow, kDeep, kMid, kBig };

// The cheapest form by a model of its time in us, from M, N, K and the CU count (n_seg > 0: grouped, with
// exponential segment lengths, n / (1 - exp(-rows n / M)) row blocks of n segments). A split form takes its rounds of
// workgroups, each a start and a join that grow with its outputs, and its rows of K bytes at the rate of a
// CU's memory path; tiles take K / 128 blocks a round, of one 256 x 256, up to two 128 x 128 or one tile of four
// stages a CU. Weights past the caches (grouped products that touch over 100 MB) come more slowly. Measured, us,
// split 1x2 / 2x2 / 2x4 / 4x4, 64 x 128 and 128 x 128 of four stages, 128- and 256-tiles, N = 4096, K = 7168:
//   M = 24  8.0 / 8.9 / 11.6 / 16.2 / 23 / 22 / 36 / 52      M = 64  13.8 / 9.8 / 12.3 / 18.0 / 25 / 23 / 37 / 53
//   M = 128  25.5 / 17.7 / 12.7 / 17.5 / 25 / 27 / 48 / 55   M = 256  48 / 32 / 23 / 18.0 / 25 / 27 / 45 / 76
//   M = 512  92 / 62 / 44 / 34 / 26.6 / 27.7 / 43 / 75       M = 1024  180 / 122 / 85 / 66 / 49 / 33.8 / 44 / 76
//   M = 2048  - / - / - / 134 / 100 / 64 / 62 / 82           M = 4093  - / - / - / 259 / 195 / 131 / 123 / 102
//   K = 1024: M = 512  - / - / 16.3 / 12.6 / 8.3 / 9.2 / 11.1 / -
// Scales by rows on both sides cost more in each form and leave the order nearly as it is, so the model has no term
// for them (the worst choice seen: 2048 rows 80 for 72):
//   M = 24  9.0 / 10.4 / 15.0 / 18.0 / 27 / 26 / 40 / 66     M = 128  29.7 / 20.1 / 15.4 / 20.3 / 32 / 38 / 50 / 68
//   M = 512  110 / 72 / 54 / 39.5 / 32.6 / 37.1 / 46 / 98    M = 1024  216 / 142 / 106 / 77 / 62 / 41.7 / 46 / 98
//   M = 2048  - / - / - / 157 / 122 / 80 / 72 / 102          M = 4093  - / - / - / 309 / 245 / 163 / 143 / 122
//   fp32 results (split forms, 128-tiles)  M = 128  30.7 / 21.4 / 16.1 / 22.4 / 68   M = 512  115 / 77 / 58 / 44.5 / 67
//   M = 1024  224 / 150 / 112 / 87 / 68
// 32 segments with SwiGLU: 64 rows in all  142 / 147 / 130 / 141 / 127 / 129 / 142 / 177; 1024  370 / 281 / 214 / 202 / 169 /
// 162 / 158 / 188; 8192  - / - / 909 / 701 / 492 / 362 / 337 / 315. Where the
// model took a 2x1 form (96 x 1360 x 1024 6.7, 160 x 816 x 4096 6.8) 2x2 takes the same: there is none.
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
    constexpr int forms[4][2] = {{1, 2}, {2, 2}, {2, 4}, {4, 4}};
    const double rate = f32 ? 55e3 : far ? 47e3 : 70e3;
    for (int f = 0; f < 4; ++f) {
      const int rows = 16 * forms[f][0], cols = 16 * forms[f][1];
      if (static_cast<double>(M) / rows + n_seg > 65535) continue;
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
