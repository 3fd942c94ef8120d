// GEMM and grouped GEMM on block-scaled E4M3 (xs_gemm_fp8.hpp).
#include <algorithm>

#include "xs_gemm_fp8.hpp"

namespace xs {
namespace f8 {

// Both products are lists of row segments, each with its own weight: the plain one has one segment.
struct GemmArgs {
  const uint8_t* a;
  int64_t lda;
  const float* a_s;
  int64_t lda_s;
  const uint8_t* b;
  int64_t ldb, b_seg;          // bytes between rows and between segments' weights
  const float* b_s;
  int64_t ldb_s, b_s_seg;      // floats
  char* c;
  int64_t ldc;                 // elements
  int M, N, K;
  const int* seg_off;          // null: one segment, all M rows
  const int* seg_rows;
  int n_seg;
  int* status;
};

// Work index t -> (segment, row block, column tile): segments in order, within one the row blocks
// vary fastest (neighbouring tiles share the weight's columns). Every wave scans the segments itself.
struct Where {
  int seg, m0, rows, nb;
};
template <int BM>
__device__ __forceinline__ bool find_tile(const GemmArgs& p, int64_t t, int nt, Where& at) {
  if (!p.seg_off) {
    const int blocks = (p.M + BM - 1) / BM;
    const int mb = static_cast<int>(t % blocks);
    at = Where{0, mb * BM, min(BM, p.M - mb * BM), static_cast<int>(t / blocks)};
    return at.nb < nt;
  }
  const int lane = threadIdx.x & 63;
  int64_t base = 0;
  for (int s0 = 0; s0 < p.n_seg; s0 += 64) {
    const int sg = s0 + lane;
    int r = 0, o = 0;
    if (sg < p.n_seg) {
      r = p.seg_rows[sg];
      o = p.seg_off[sg];
      if (r < 0 || o < 0 || static_cast<int64_t>(o) + r > p.M) {
        if (r != 0) set_status(p.status, XS_EBADINPUT);
        r = 0;
      }
    }
    const int64_t tiles = static_cast<int64_t>((static_cast<int64_t>(r) + BM - 1) / BM) * nt;
    int64_t incl = tiles;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int64_t v = __shfl_up(incl, off);
      if (lane >= off) incl += v;
    }
    const unsigned long long hit = __ballot(t < base + incl);
    if (hit) {
      const int l = __ffsll(static_cast<long long>(hit)) - 1;
      const int rows = __shfl(r, l), off = __shfl(o, l);
      const int64_t local = t - (base + __shfl(incl, l) - __shfl(tiles, l));
      const int blocks = (rows + BM - 1) / BM;
      const int mb = static_cast<int>(local % blocks);
      at.seg = __builtin_amdgcn_readfirstlane(s0 + l);
      at.m0 = __builtin_amdgcn_readfirstlane(off + mb * BM);
      at.rows = __builtin_amdgcn_readfirstlane(min(BM, rows - mb * BM));
      at.nb = __builtin_amdgcn_readfirstlane(static_cast<int>(local / blocks));
      return true;
    }
    base += __shfl(incl, 63);
  }
  return false;
}

template <class T, bool ROW, bool SWIGLU, bool F32>
__global__ __launch_bounds__(T::kThreads) void gemm_kernel(GemmArgs p) {
  __shared__ __attribute__((aligned(16))) char lds[T::kLds];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = w / T::kWN, wn = w % T::kWN;
  constexpr int kCols = SWIGLU ? T::kBN / 2 : T::kBN;           // output columns of a tile
  const int n_out = SWIGLU ? p.N / 2 : p.N;
  const int nt = (n_out + kCols - 1) / kCols;
  Where at;
  for (int64_t t = blockIdx.x; find_tile<T::kBM>(p, t, nt, at); t += gridDim.x) {
    const int n0 = at.nb * kCols;
    const Product q{p.a + at.m0 * p.lda, p.lda, p.a_s + at.m0 * p.lda_s, p.lda_s, at.rows,
                    p.b + at.seg * p.b_seg, p.ldb, p.b_s + at.seg * p.b_s_seg, p.ldb_s, n0, p.N, p.N / 2, p.K};
    typename T::Acc acc;
    mainloop<T, ROW, SWIGLU, F32>(q, acc, lds);
    const int row0 = wm * T::kMI * 16 + (lane & 15), col0 = wn * T::kNJ * 16 + 4 * (lane >> 4);
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < T::kMI; ++i)
#pragma unroll
        for (int j = 0; j < T::kNJ; ++j) {
          const int r = row0 + 16 * i, n = n0 + col0 + 16 * j;
          if (r < at.rows && n < p.N)
            *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(p.c) + (at.m0 + r) * p.ldc + n) = acc[i][j];
        }
    } else {
#pragma unroll
      for (int i = 0; i < T::kMI; ++i)
#pragma unroll
        for (int j = 0; j < T::kNJ; ++j) {
          if constexpr (SWIGLU) {
            // blocks j and j + 2 of a wave are the gate and up rows of the same columns
            static_assert(T::kNJ % 4 == 0, "");
            if (j & 2) continue;
            float h[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float g = acc[i][j][c];
              h[c] = g * __builtin_amdgcn_rcpf(1.f + __expf(-g)) * acc[i][j + 2][c];
            }
            const int col = wn * T::kNJ * 8 + 16 * ((j >> 2) * 2 + (j & 1)) + 4 * (lane >> 4);
            *reinterpret_cast<uint2*>(lds + (row0 + 16 * i) * T::kPitch + col * 2) =
                make_uint2(pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3]));
          } else {
            const f32x4 v = acc[i][j];
            *reinterpret_cast<uint2*>(lds + (row0 + 16 * i) * T::kPitch + (col0 + 16 * j) * 2) =
                make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
          }
        }
      __syncthreads();
      constexpr int kPieces = kCols / 8, kRowsPass = T::kThreads / kPieces;
      const int pc = tid % kPieces;
      if (n0 + pc * 8 < n_out) {
        char* const dst = p.c + (at.m0 * p.ldc + n0 + pc * 8) * 2;
#pragma unroll 4
        for (int r = tid / kPieces; r < at.rows; r += kRowsPass)
          *reinterpret_cast<u32x4*>(dst + r * p.ldc * 2) = *reinterpret_cast<const u32x4*>(lds + r * T::kPitch + pc * 16);
      }
      lds_barrier();
    }
  }
}

}  // namespace f8
}  // namespace xs

using namespace xs;

namespace xs_host {
int persistent_grid(int max_producers);
}  // namespace xs_host

namespace {

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

typedef f8::Tile<128, 128, 2, 2> Mid;

template <class T, bool ROW, bool SWIGLU, bool F32>
int launch(const f8::GemmArgs& p, hipStream_t st) {
  const int cols = SWIGLU ? T::kBN / 2 : T::kBN;
  const int64_t nt = ((SWIGLU ? p.N / 2 : p.N) + cols - 1) / cols;
  const int64_t blocks = (static_cast<int64_t>(p.M) + T::kBM - 1) / T::kBM + (p.seg_off ? p.n_seg : 0);
  const int grid = static_cast<int>(std::min<int64_t>(blocks * nt, 2 * xs_host::persistent_grid(0)));
  hipLaunchKernelGGL((f8::gemm_kernel<T, ROW, SWIGLU, F32>), dim3(grid), dim3(T::kThreads), 0, st, p);
  return xs_host::launch_status();
}

// Byte offsets inside a tile are 32-bit: up to 256 rows of at most 2^22 bytes.
constexpr int64_t kMaxRow = int64_t(1) << 22;

int operand_ok(const void* codes, int64_t ld, const float* scales, int64_t ld_s, int32_t K) {
  if (!codes || !scales) return XS_EINVAL;
  if (ld < K || ld_s < K / 128) return XS_EINVAL;
  if (ld % 16 || ld_s % 4 || !aligned_to(codes, 16) || !aligned_to(scales, 16)) return XS_EINVAL;
  return ld > kMaxRow || ld_s > kMaxRow / 4 ? XS_EUNSUPPORTED : XS_OK;
}

}  // namespace

extern "C" int xs_gemm_fp8(const void* a, int64_t lda, const float* a_scales, int64_t lda_s, const void* b, int64_t ldb,
                           const float* b_scales, int64_t ldb_s, int32_t b_block, void* c, int64_t ldc, int32_t c_type,
                           int32_t M, int32_t N, int32_t K, void* stream) {
  if (!c || M < 0 || N <= 0 || K <= 0 || (b_block != XS_BLOCK_ROW && b_block != XS_BLOCK_TILE) ||
      (c_type != XS_TYPE_BF16 && c_type != XS_TYPE_F32))
    return XS_EINVAL;
  if (N % 8 || K % 128 || N > (1 << 30)) return XS_EUNSUPPORTED;
  int rc = operand_ok(a, lda, a_scales, lda_s, K);
  if (!rc) rc = operand_ok(b, ldb, b_scales, ldb_s, K);
  if (rc) return rc;
  if (ldc < N || ldc % 8 || !aligned_to(c, 16)) return XS_EINVAL;
  if (M == 0) return XS_OK;
  const f8::GemmArgs p{static_cast<const uint8_t*>(a), lda, a_scales, lda_s, static_cast<const uint8_t*>(b), ldb, 0,
                       b_scales, ldb_s, 0, static_cast<char*>(c), ldc, M, N, K, nullptr, nullptr, 1, nullptr};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (b_block == XS_BLOCK_ROW)
    return c_type == XS_TYPE_F32 ? launch<Mid, true, false, true>(p, st) : launch<Mid, true, false, false>(p, st);
  return c_type == XS_TYPE_F32 ? launch<Mid, false, false, true>(p, st) : launch<Mid, false, false, false>(p, st);
}

extern "C" int xs_grouped_gemm_fp8(const void* a, int64_t lda, const float* a_scales, int64_t lda_s, int32_t M,
                                   const int32_t* seg_offsets, const int32_t* seg_rows, int32_t n_seg, const void* b,
                                   const float* b_scales, int64_t ldb_s, int32_t N, int32_t K, void* c, int64_t ldc,
                                   int32_t epilogue, int32_t* dev_status, void* stream) {
  if (!c || !seg_offsets || !seg_rows || M < 0 || n_seg < 0 || n_seg > 1024 || N <= 0 || K <= 0 ||
      (epilogue != XS_EPI_STORE && epilogue != XS_EPI_SWIGLU))
    return XS_EINVAL;
  const bool swiglu = epilogue == XS_EPI_SWIGLU;
  const int n_out = swiglu ? N / 2 : N;
  if (K % 128 || N % (swiglu ? 256 : 8) || N > (1 << 30)) return XS_EUNSUPPORTED;
  int rc = operand_ok(a, lda, a_scales, lda_s, K);
  if (!rc) rc = operand_ok(b, K, b_scales, ldb_s, K);
  if (rc) return rc;
  if (ldc < n_out || ldc % 8 || !aligned_to(c, 16)) return XS_EINVAL;
  if (M == 0 || n_seg == 0) return XS_OK;
  const f8::GemmArgs p{static_cast<const uint8_t*>(a), lda, a_scales, lda_s, static_cast<const uint8_t*>(b), K,
                       static_cast<int64_t>(N) * K, b_scales, ldb_s, static_cast<int64_t>((N + 127) / 128) * ldb_s,
                       static_cast<char*>(c), ldc, M, N, K, seg_offsets, seg_rows, n_seg, dev_status};
  hipStream_t st = static_cast<hipStream_t>(stream);
  return swiglu ? launch<Mid, false, true, false>(p, st) : launch<Mid, false, false, false>(p, st);
}
