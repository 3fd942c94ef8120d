// Block-scaled E4M3 GEMM core for gfx950: C = A B^T where block b of 128 K elements of row m of A has
// the fp32 scale sa[m][b], and of row n of B sb[n][b] (1 x 128 blocks) or sb[n / 128][b] (128 x 128):
//
//   c[m][n] = sum_b sa[m][b] sb[.][b] sum_{k in block b} a[m][k] b[n][k]
//
// One v_mfma_f32_16x16x128_f8f6f4 is one block of 16 x 16 outputs; its sum goes into the fp32
// accumulators with the scales by vector multiply-adds, which run beside the matrix pipe. The weight
// fragment is the first operand, so a lane holds one output row and four consecutive columns, and the
// two scales of a 128 x 128 weight block and a row are one factor per lane.
//
// The 8-bit matrix instructions (this one and the 16x16x32 form alike) add the products of eight
// consecutive K elements aligned to the largest of them and cut below 2^-13 of its exponent, then
// accumulate in fp32 (measured: beside 2^16, 2^3 counts and 2^2 does not within a group; in another group
// 2^-7 does). A block's sum is off by at most 8 2^-13 of each group's largest product, for random
// operands by 1.3e-5 of the result: a hundredth of the rounding of a bf16 result. An fp32 result takes the
// EXACT form: the codes become bf16 (exactly) and go through v_mfma_f32_16x16x32_bf16, whose sums are
// fp32 (1e-8), at half the matrix rate.
//
// LDS: two stages of one K block, A rows then B rows of 128 bytes (16-byte piece c of row r at c ^ ((r >>
// 1) & 7): the 16 rows of a fragment read hit 16 distinct bank groups), and two buffers of scales, each
// the 16 bytes of four blocks per row. All arrive by direct global -> LDS loads.
#pragma once
#include "xs_gemm.hpp"

namespace xs {
namespace f8 {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i_ __attribute__((ext_vector_type(4)));

// The 32 codes of a fragment as bf16: four operands of v_mfma_f32_16x16x32_bf16.
struct Wide {
  bf16x8 k[4];
};
__device__ __forceinline__ Wide widen(v8i v) {
  Wide r;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    union {
      bf16x8 all;
      bf16x2_t two[4];
    } u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u.two[2 * h] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<unsigned>(v[2 * q + h]), 1.f, false);
      u.two[2 * h + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<unsigned>(v[2 * q + h]), 1.f, true);
    }
    r.k[q] = u.all;
  }
  return r;
}

// The sum over one K block of 16 x 16 outputs.
__device__ __forceinline__ f32x4 block_sum(const v8i& b, const v8i& a) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
}
__device__ __forceinline__ f32x4 block_sum(const Wide& b, const Wide& a) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int q = 0; q < 4; ++q) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.k[q], a.k[q], s, 0, 0, 0);
  return s;
}
__device__ __forceinline__ void as_operand(v8i v, v8i& out) { out = v; }
__device__ __forceinline__ void as_operand(v8i v, Wide& out) { out = widen(v); }

template <int BM_, int BN_, int WM_, int WN_>
struct Tile {
  static constexpr int kBM = BM_, kBN = BN_, kWM = WM_, kWN = WN_;
  static constexpr int kWaves = WM_ * WN_, kThreads = kWaves * 64;
  static constexpr int kMI = BM_ / WM_ / 16, kNJ = BN_ / WN_ / 16;
  static constexpr int kALoads = BM_ / 8 / kWaves, kBLoads = BN_ / 8 / kWaves;   // 8 rows a load
  static constexpr int kSLoads = (BM_ + BN_) / 64 / kWaves;                      // 64 rows' scales a load
  static constexpr int kStage = (BM_ + BN_) * 128, kScales = (BM_ + BN_) * 16;
  static constexpr int kPitch = (BN_ + 8) * 2;                                   // staged bf16 output row
  static constexpr int kOperands = 2 * kStage + 2 * kScales, kOut = BM_ * kPitch;
  static constexpr int kLds = kOperands > kOut ? kOperands : kOut;
  typedef f32x4 Acc[kMI][kNJ];
};

// One output tile: A rows [0, rows), B rows through b_row_map (rows past b_end read row b_end - 1).
struct Product {
  const uint8_t* a;
  int64_t lda;
  const float* a_s;
  int64_t lda_s;
  int rows;
  const uint8_t* b;
  int64_t ldb;
  const float* b_s;
  int64_t ldb_s;
  int n0, b_end, half, K;
};

template <class T, bool ROW, bool SWIGLU, bool EXACT>
__device__ __forceinline__ void mainloop(const Product& p, typename T::Acc& acc, char* lds) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = w / T::kWN, wn = w % T::kWN;
  const int nk = p.K / 128;
  const auto b_row = [&](int r) { return min(b_row_map(r, p.n0, p.half, SWIGLU), p.b_end - 1); };
  // load i of wave w fills rows 8 (kWaves i + w) .. + 7: lane -> row lane / 8, physical piece lane % 8
  uint32_t oa[T::kALoads], ob[T::kBLoads], os[T::kSLoads];
  const int lr = lane >> 3, lp = lane & 7;
#pragma unroll
  for (int i = 0; i < T::kALoads; ++i) {
    const int r = 8 * (T::kWaves * i + w) + lr;
    oa[i] = static_cast<uint32_t>(min(r, p.rows - 1) * p.lda + ((lp ^ ((r >> 1) & 7)) << 4));
  }
#pragma unroll
  for (int i = 0; i < T::kBLoads; ++i) {
    const int r = 8 * (T::kWaves * i + w) + lr;
    ob[i] = static_cast<uint32_t>(b_row(r) * p.ldb + ((lp ^ ((r >> 1) & 7)) << 4));
  }
  // scale load i of wave w: rows 64 (kWaves i + w) .. + 63 of A, then of B
  const char* sbase[T::kSLoads];
#pragma unroll
  for (int i = 0; i < T::kSLoads; ++i) {
    const int r0 = 64 * (T::kWaves * i + w);
    if (r0 < T::kBM) {
      sbase[i] = reinterpret_cast<const char*>(p.a_s);
      os[i] = static_cast<uint32_t>(min(r0 + lane, p.rows - 1) * p.lda_s * 4);
    } else {
      const int n = b_row(r0 - T::kBM + lane);
      sbase[i] = reinterpret_cast<const char*>(p.b_s);
      os[i] = static_cast<uint32_t>((ROW ? n : n / 128) * p.ldb_s * 4);
    }
  }
  char* const scales = lds + 2 * T::kStage;
  const auto issue = [&](int kt) {
    char* const st = lds + (kt & 1) * T::kStage;
    const char* const a = reinterpret_cast<const char*>(p.a) + static_cast<int64_t>(kt) * 128;
    const char* const b = reinterpret_cast<const char*>(p.b) + static_cast<int64_t>(kt) * 128;
#pragma unroll
    for (int i = 0; i < T::kALoads; ++i)
      __builtin_amdgcn_global_load_lds((glob_void*)(a + oa[i]), (lds_void*)(st + (T::kWaves * i + w) * 1024), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < T::kBLoads; ++i)
      __builtin_amdgcn_global_load_lds((glob_void*)(b + ob[i]),
                                       (lds_void*)(st + T::kBM * 128 + (T::kWaves * i + w) * 1024), 16, 0, 0);
  };
  const auto issue_scales = [&](int g) {
#pragma unroll
    for (int i = 0; i < T::kSLoads; ++i)
      __builtin_amdgcn_global_load_lds((glob_void*)(sbase[i] + static_cast<int64_t>(g) * 16 + os[i]),
                                       (lds_void*)(scales + (g & 1) * T::kScales + (T::kWaves * i + w) * 1024), 16, 0, 0);
  };
  const int l16 = lane & 15, g4 = lane >> 4, swz = (l16 >> 1) & 7;
  const int ar = wm * T::kMI * 16 + l16, br = wn * T::kNJ * 16 + l16;
  const auto frag = [&](const char* rows, int r) {
    const v4i_ lo = *reinterpret_cast<const v4i_*>(rows + r * 128 + ((g4 ^ swz) << 4));
    const v4i_ hi = *reinterpret_cast<const v4i_*>(rows + r * 128 + (((g4 + 4) ^ swz) << 4));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
#pragma unroll
  for (int i = 0; i < T::kMI; ++i)
#pragma unroll
    for (int j = 0; j < T::kNJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  issue(0);
  issue_scales(0);
  wait_vm0();
  __builtin_amdgcn_s_barrier();
  for (int kt = 0; kt < nk; ++kt) {
    if (kt + 1 < nk) issue(kt + 1);
    if ((kt & 3) == 0 && kt + 4 < nk) issue_scales((kt >> 2) + 1);
    const char* const st = lds + (kt & 1) * T::kStage;
    const char* const sc = scales + ((kt >> 2) & 1) * T::kScales + (kt & 3) * 4;
    std::conditional_t<EXACT, Wide, v8i> bf[T::kNJ], af;
#pragma unroll
    for (int j = 0; j < T::kNJ; ++j) as_operand(frag(st + T::kBM * 128, br + 16 * j), bf[j]);
    float sb[ROW ? T::kNJ : (SWIGLU ? 2 : 1)][ROW ? 4 : 1];
    if constexpr (ROW) {
#pragma unroll
      for (int j = 0; j < T::kNJ; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          sb[j][c] = *reinterpret_cast<const float*>(sc + (T::kBM + wn * T::kNJ * 16 + 16 * j + 4 * g4 + c) * 16);
    } else {
      sb[0][0] = *reinterpret_cast<const float*>(sc + (T::kBM + wn * T::kNJ * 16) * 16);
      if constexpr (SWIGLU) sb[1][0] = *reinterpret_cast<const float*>(sc + (T::kBM + wn * T::kNJ * 16 + 32) * 16);
    }
#pragma unroll
    for (int i = 0; i < T::kMI; ++i) {
      as_operand(frag(st, ar + 16 * i), af);
      const float sa = *reinterpret_cast<const float*>(sc + (ar + 16 * i) * 16);
#pragma unroll
      for (int j = 0; j < T::kNJ; ++j) {
        const f32x4 v = block_sum(bf[j], af);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if constexpr (ROW) acc[i][j][c] = __builtin_fmaf(v[c] * sb[j][c], sa, acc[i][j][c]);
          else acc[i][j][c] = __builtin_fmaf(v[c], sa * sb[SWIGLU ? (j >> 1) & 1 : 0][0], acc[i][j][c]);
        }
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0): the next stage has landed, this one is read
    __builtin_amdgcn_s_barrier();
  }
}

}  // namespace f8
}  // namespace xs
