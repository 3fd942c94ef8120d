// GEMM and grouped GEMM on block-scaled E4M3 (xs_gemm_fp8.hpp).
#include <algorithm>

#include "xs_gemm_fp8.hpp"
#include "xs_gemm_fp8_form.hpp"

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
  int one_each;                // one tile per workgroup, not a persistent grid
};

// Work index t -> (segment, row block, column tile): segments in order; within one, groups of eight row
// blocks, the row blocks of a group varying fastest (32 consecutive tiles, one XCD's, are then 8 x 4: twelve
// operand panels for its L2). Every wave scans the segments itself. more: there is, or may be, a tile t + step.
struct Where {
  int seg, m0, rows, nb;
  bool more;
};
constexpr int kGroupRows = 8, kRun = 32;
constexpr int64_t kNoTile = int64_t(1) << 50;
__device__ __forceinline__ void in_groups(int64_t t, int blocks, int nt, int* mb, int* nb) {
  const int64_t per = static_cast<int64_t>(kGroupRows) * nt;
  const int first = static_cast<int>(t / per) * kGroupRows, local = static_cast<int>(t % per);
  const int gm = min(kGroupRows, blocks - first);
  *mb = first + local % gm;
  *nb = local / gm;
}
template <int BM>
__device__ __forceinline__ bool find_tile(const GemmArgs& p, int64_t t, int64_t step, int nt, Where& at) {
  if (!p.seg_off) {
    const int blocks = static_cast<int>((static_cast<int64_t>(p.M) + BM - 1) / BM);
    if (t >= static_cast<int64_t>(blocks) * nt) return false;
    int mb, nb;
    in_groups(t, blocks, nt, &mb, &nb);
    at = Where{0, mb * BM, min(BM, p.M - mb * BM), nb, t + step < static_cast<int64_t>(blocks) * nt};
    return true;
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
      const int blocks = static_cast<int>((static_cast<int64_t>(rows) + BM - 1) / BM);
      int mb, nb;
      in_groups(local, blocks, nt, &mb, &nb);
      at.seg = __builtin_amdgcn_readfirstlane(s0 + l);
      at.m0 = __builtin_amdgcn_readfirstlane(off + mb * BM);
      at.rows = __builtin_amdgcn_readfirstlane(min(BM, rows - mb * BM));
      at.nb = __builtin_amdgcn_readfirstlane(nb);
      at.more = s0 + 64 < p.n_seg || __ballot(t + step < base + incl);
      return true;
    }
    base += __shfl(incl, 63);
  }
  return false;
}

template <class T, bool ROW, bool SWIGLU, bool F32>
__global__ __launch_bounds__(T::kThreads, 2) void gemm_kernel(GemmArgs p) {
  __shared__ __attribute__((aligned(16))) char lds[T::kLds];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = w / T::kWN, wn = w % T::kWN;
  constexpr int kCols = SWIGLU ? T::kBN / 2 : T::kBN;           // output columns of a tile
  const int n_out = SWIGLU ? p.N / 2 : p.N;
  const int nt = (n_out + kCols - 1) / kCols;
  Where at;
  // Consecutive workgroups go to different XCDs: each XCD takes runs of consecutive tiles, of the grid's eighth
  // or (one tile per workgroup) of kRun. 128-tiles come two to a CU, and a last round of one to a CU is quicker,
  // which dealing a tile to each workgroup as it starts makes use of (7 tiles per CU: 262 us persistent, 238
  // so); the 256-tiles' workgroups gain nothing by it.
  const int G = gridDim.x, b = blockIdx.x;
  int64_t t = G % 8 ? b : (b % 8) * (G / 8) + b / 8;
  if (p.one_each) t = (static_cast<int64_t>(b / 8 / kRun) * 8 + b % 8) * kRun + b / 8 % kRun;
  const int64_t step = p.one_each ? kNoTile : G;
  for (; find_tile<T::kBM>(p, t, step, nt, at); t += step) {
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

// The kernel's only argument, read where this stands from where the launch put it.
template <class A>
__device__ __forceinline__ A kernel_args() {
  typedef const uint32_t __attribute__((address_space(4))) Constant;
  int zero;
  asm volatile("s_mov_b32 %0, 0" : "=s"(zero));
  Constant* const p = (Constant*)__builtin_amdgcn_kernarg_segment_ptr() + zero;
  struct Words {
    uint32_t w[sizeof(A) / 4];
  } words;
#pragma unroll
  for (unsigned i = 0; i < sizeof(A) / 4; ++i) words.w[i] = p[i];
  return __builtin_bit_cast(A, words);
}

// Products with few output tiles: a workgroup takes 16 NB rows and 16 NJ columns and splits the K blocks
// over its four waves, whose scaled fp32 sums meet in LDS once and are added in wave order. Each wave
// stages its own blocks (one 128-byte line of every row, and the rows' scales) kDepth deep in a slice of
// LDS of its own, by direct loads, and needs no barrier until the end. SWIGLU: columns y < NJ / 2 are the
// gate's, the others the same columns of up. GROUPED: segments that overlap have more row blocks than the grid was
// sized for, and a workgroup goes on to a second one. Arguments and lanes' offsets are made anew for each: held over the
// loop they spill, 137 us for 134 (32 segments, 128 rows of 4096 x 7168) and 4.8 for 4.5 (4 segments of 768 x 1792).
template <int NB, int NJ, int kDepth, bool ROW, bool SWIGLU, bool F32, bool GROUPED>
__global__ __launch_bounds__(256) void split_kernel(GemmArgs args) {
  constexpr int kWaves = 4, kRows = 16 * NB, kCols = 16 * NJ, kPitch = kCols + 4;
  constexpr int kPiece = (kRows + kCols) * 128 + 512;      // B rows, A rows, 64 scales of A, 64 of B
  constexpr int kLoads = 2 * (NB + NJ) + 2;
  constexpr int kStage = kWaves * kDepth * kPiece, kRed = kWaves * kRows * kPitch * 4;
  constexpr int kHalf = SWIGLU ? kCols / 2 : kCols;        // output columns of the workgroup
  __shared__ __attribute__((aligned(16))) char smem[kStage > kRed ? kStage : kRed];
  for (int64_t t = blockIdx.y;; t += gridDim.y) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const GemmArgs p = GROUPED ? kernel_args<GemmArgs>() : args;
    Where at;
    if (!find_tile<kRows>(p, t, gridDim.y, 1, at)) return;  // the whole workgroup
    const int lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * kHalf, n_out = SWIGLU ? p.N / 2 : p.N;
    const int rows = at.rows, cols = min(kHalf, n_out - n0);
    lds_char* const lds = (lds_char*)smem + w * kDepth * kPiece;
    const uint8_t* const b = p.b + at.seg * p.b_seg;
    const float* const b_s = p.b_s + at.seg * p.b_s_seg;
    const int nk = p.K / 128;
    const auto span = [&](int64_t rows_, int64_t ld, int64_t last) { return static_cast<uint32_t>((rows_ - 1) * ld + last); };
    const v4i ra = buffer_rsrc(p.a + at.m0 * p.lda, span(rows, p.lda, p.K));
    const v4i rb = buffer_rsrc(b + n0 * p.ldb, span(cols, p.ldb, p.K));
    const v4i rb2 = buffer_rsrc(b + (n0 + (SWIGLU ? n_out : 0)) * p.ldb, span(cols, p.ldb, p.K));
    const v4i rsa = buffer_rsrc(p.a_s + at.m0 * p.lda_s, span(rows, p.lda_s * 4, nk * 4));
    // scales of B: one per column, or of the workgroup's 128 x 128 block (and of up's)
    const int sb_rows = ROW ? cols : 1;
    const v4i rsb = buffer_rsrc(b_s + (ROW ? n0 : n0 / 128) * p.ldb_s,
                                span(SWIGLU ? n_out / 128 + 1 : sb_rows, p.ldb_s * 4, nk * 4));
    // load n of an operand fills its rows 8 n .. + 7 of a piece; past the buffers' ends nothing is fetched
    uint32_t oa[2 * NB], ob[2 * NJ];
    const int lr = lane >> 3, lp = lane & 7;
#pragma unroll
    for (int n = 0; n < 2 * NB; ++n) oa[n] = static_cast<uint32_t>((8 * n + lr) * p.lda + ((lp ^ ((4 * n + (lr >> 1)) & 7)) << 4));
#pragma unroll
    for (int n = 0; n < 2 * NJ; ++n) {
      const int r = SWIGLU && n >= NJ ? 8 * (n - NJ) : 8 * n;
      ob[n] = static_cast<uint32_t>((r + lr) * p.ldb + ((lp ^ ((4 * n + (lr >> 1)) & 7)) << 4));
    }
    const uint32_t osa = lane < kRows ? static_cast<uint32_t>(lane * p.lda_s * 4) : kNone;
    uint32_t osb = kNone;
    if (ROW ? lane < kCols : lane < (SWIGLU ? 2 : 1)) osb = static_cast<uint32_t>((SWIGLU ? lane * (n_out / 128) : lane) * p.ldb_s * 4);
    const int k0 = nk * w / kWaves, k1 = nk * (w + 1) / kWaves;   // this wave's blocks
    f32x4 acc[NB][NJ];
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
      for (int y = 0; y < NJ; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
    // block k into slot s; past the wave's range every lane points past the buffers, so the number of loads
    // in flight stays the same
    const auto load = [&](int s, int k) {
      const uint32_t kb = k < k1 ? static_cast<uint32_t>(k) * 128u : kNone, ks = k < k1 ? static_cast<uint32_t>(k) * 4u : kNone;
      lds_char* const at_ = lds + s * kPiece;
#pragma unroll
      for (int n = 0; n < 2 * NJ; ++n) load_lds16(SWIGLU && n >= NJ ? rb2 : rb, ob[n] + kb, at_ + n * 1024);
#pragma unroll
      for (int n = 0; n < 2 * NB; ++n) load_lds16(ra, oa[n] + kb, at_ + kCols * 128 + n * 1024);
      load_lds4(rsa, osa + ks, at_ + (kRows + kCols) * 128);
      load_lds4(rsb, osb + ks, at_ + (kRows + kCols) * 128 + 256);
    };
    const int swz = (i >> 1) & 7;
    typedef __attribute__((address_space(3))) v4i_ lds_v4i;
    typedef __attribute__((address_space(3))) float lds_float;
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    const auto frag = [&](const lds_char* row) {
      const v4i_ lo = *(const lds_v4i*)(row + ((g ^ swz) << 4)), hi = *(const lds_v4i*)(row + (((g + 4) ^ swz) << 4));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
#pragma unroll
    for (int s = 0; s < kDepth; ++s) load(s, k0 + s);
    for (int k = k0; k < k1; k += kDepth) {
#pragma unroll
      for (int s = 0; s < kDepth; ++s) {
        if (k + s >= k1) break;
        wait_vm<(kDepth - 1) * kLoads>();                    // block k + s has landed
        const lds_char* const at_ = lds + s * kPiece;
        const lds_char* const sc = at_ + (kRows + kCols) * 128;
        v8i bc[NJ], ac[NB];
        float sa[NB];
        f32x4 sb[ROW ? NJ : 1];
#pragma unroll
        for (int y = 0; y < NJ; ++y) bc[y] = frag(at_ + (16 * y + i) * 128);
#pragma unroll
        for (int x = 0; x < NB; ++x) {
          ac[x] = frag(at_ + (kCols + 16 * x + i) * 128);
          sa[x] = *(const lds_float*)(sc + (16 * x + i) * 4);
        }
        if constexpr (ROW) {
#pragma unroll
          for (int y = 0; y < NJ; ++y) sb[y] = *(const lds_f32x4*)(sc + 256 + (16 * y + 4 * g) * 4);
        } else {
          sb[0][0] = *(const lds_float*)(sc + 256);
          sb[0][1] = SWIGLU ? *(const lds_float*)(sc + 260) : 0.f;
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);                  // lgkmcnt(0): the slot has been read
        asm volatile("" ::: "memory");
        load(s, k + s + kDepth);
        std::conditional_t<F32, Wide, v8i> bf[NJ], af;
#pragma unroll
        for (int y = 0; y < NJ; ++y) as_operand(bc[y], bf[y]);
#pragma unroll
        for (int x = 0; x < NB; ++x) {
          as_operand(ac[x], af);
#pragma unroll
          for (int y = 0; y < NJ; ++y) {
            const f32x4 v = block_sum(bf[y], af);
            const float f = ROW ? sa[x] : sa[x] * sb[0][SWIGLU && y >= NJ / 2 ? 1 : 0];
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[x][y][c] = __builtin_fmaf(ROW ? v[c] * sb[y][c] : v[c], f, acc[x][y][c]);
          }
        }
      }
    }
    wait_vm<0>();
    __syncthreads();                                         // no load is in flight: the LDS is free
    float* const red = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int x = 0; x < NB; ++x)
#pragma unroll
      for (int y = 0; y < NJ; ++y)
        *reinterpret_cast<f32x4*>(red + (w * kRows + 16 * x + i) * kPitch + 16 * y + 4 * g) = acc[x][y];
    __syncthreads();
    const auto sum = [&](int r, int c) {
      f32x4 v = *reinterpret_cast<const f32x4*>(red + r * kPitch + c);
#pragma unroll
      for (int x = 1; x < kWaves; ++x) v += *reinterpret_cast<const f32x4*>(red + (x * kRows + r) * kPitch + c);
      return v;
    };
    for (int u = tid; u < rows * (kHalf / 4); u += 256) {
      const int r = u / (kHalf / 4), c = 4 * (u % (kHalf / 4));
      if (n0 + c >= n_out) continue;
      f32x4 v = sum(r, c);
      if constexpr (SWIGLU) {
        const f32x4 up = sum(r, c + kHalf);
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = v[q] * __builtin_amdgcn_rcpf(1.f + __expf(-v[q])) * up[q];
      }
      const int64_t to = (at.m0 + r) * p.ldc + n0 + c;
      if constexpr (F32) *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(p.c) + to) = v;
      else *reinterpret_cast<uint2*>(p.c + to * 2) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
    if (!GROUPED || !at.more) return;
    __syncthreads();                                         // the sums have been read: the LDS is free
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

typedef f8::Tile<256, 256, 2, 4> Big;
typedef f8::Tile<128, 128, 2, 2> Mid;
// For tiles that have a CU to themselves: four stages, since a K block's products (0.2 us) are much shorter than a
// load's way (1024 x 4096 x 7168: 43.5 us with two stages, 35.7; 512 rows 43.4, in 64 x 128 27.2).
typedef f8::Tile<128, 128, 4, 2, 4> Deep;
typedef f8::Tile<64, 128, 2, 2, 4> Low;

template <int NB, int NJ, int kDepth, bool ROW, bool SWIGLU, bool F32>
int launch_split(const f8::GemmArgs& p, hipStream_t st) {
  const int cols = SWIGLU ? 8 * NJ : 16 * NJ, n_out = SWIGLU ? p.N / 2 : p.N;
  const int64_t blocks = (static_cast<int64_t>(p.M) + 16 * NB - 1) / (16 * NB) + (p.seg_off ? p.n_seg : 0);
  const dim3 grid((n_out + cols - 1) / cols, static_cast<unsigned>(blocks));
  if constexpr (!SWIGLU)
    if (!p.seg_off) {
      hipLaunchKernelGGL((f8::split_kernel<NB, NJ, kDepth, ROW, SWIGLU, F32, false>), grid, dim3(256), 0, st, p);
      return xs_host::launch_status();
    }
  if constexpr (!ROW && !F32) hipLaunchKernelGGL((f8::split_kernel<NB, NJ, kDepth, ROW, SWIGLU, F32, true>), grid, dim3(256), 0, st, p);
  return xs_host::launch_status();
}

template <class T, bool ROW, bool SWIGLU, bool F32>
int launch_tiles(f8::GemmArgs p, int per_cu, hipStream_t st) {
  const int cols = SWIGLU ? T::kBN / 2 : T::kBN;
  const int64_t nt = ((SWIGLU ? p.N / 2 : p.N) + cols - 1) / cols;
  const int64_t blocks = (static_cast<int64_t>(p.M) + T::kBM - 1) / T::kBM + (p.seg_off ? p.n_seg : 0);
  const int64_t runs = (blocks * nt + 8 * f8::kRun - 1) / (8 * f8::kRun) * (8 * f8::kRun);
  p.one_each = per_cu > 1 && !p.seg_off && runs < (1 << 22);
  const int grid = static_cast<int>(p.one_each ? runs : std::min<int64_t>(blocks * nt, static_cast<int64_t>(per_cu) * xs_host::persistent_grid(0)));
  hipLaunchKernelGGL((f8::gemm_kernel<T, ROW, SWIGLU, F32>), dim3(grid), dim3(T::kThreads), 0, st, p);
  return xs_host::launch_status();
}

template <bool ROW, bool SWIGLU, bool F32>
int launch(const f8::GemmArgs& p, hipStream_t st) {
  using namespace f8;
  switch (choose_form(xs_host::persistent_grid(0), p.M, p.N, p.K, p.ldb_s, p.seg_off ? p.n_seg : 0, SWIGLU, F32)) {
    case kSplit12: return launch_split<1, 2, 4, ROW, SWIGLU, F32>(p, st);
    case kSplit22: return launch_split<2, 2, 3, ROW, SWIGLU, F32>(p, st);
    case kSplit24: return launch_split<2, 4, 2, ROW, SWIGLU, F32>(p, st);
    case kSplit44: return launch_split<4, 4, 2, ROW, SWIGLU, F32>(p, st);
    case kLow:
      if constexpr (!F32) return launch_tiles<Low, ROW, SWIGLU, F32>(p, 1, st);
    case kDeep:
      if constexpr (!F32) return launch_tiles<Deep, ROW, SWIGLU, F32>(p, 1, st);
    case kMid: return launch_tiles<Mid, ROW, SWIGLU, F32>(p, 2, st);
    case kBig:
      if constexpr (!F32) return launch_tiles<Big, ROW, SWIGLU, F32>(p, 1, st);
  }
  return launch_tiles<Mid, ROW, SWIGLU, F32>(p, 2, st);
}

// Byte offsets inside a tile are 32-bit: up to 256 rows of at most 2^22 bytes.
constexpr int64_t kMaxRow = int64_t(1) << 22, kMaxSpan = 0x7FFFFF00;

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
                       b_scales, ldb_s, 0, static_cast<char*>(c), ldc, M, N, K, nullptr, nullptr, 1, nullptr, 0};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (b_block == XS_BLOCK_ROW)
    return c_type == XS_TYPE_F32 ? launch<true, false, true>(p, st) : launch<true, false, false>(p, st);
  return c_type == XS_TYPE_F32 ? launch<false, false, true>(p, st) : launch<false, false, false>(p, st);
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
  // a tile's gate and up rows in one buffer range
  if (swiglu && ((n_out + 128) * static_cast<int64_t>(K) > kMaxSpan || (n_out / 128 + 1) * ldb_s * 4 > kMaxSpan)) return XS_EUNSUPPORTED;
  if (ldc < n_out || ldc % 8 || !aligned_to(c, 16)) return XS_EINVAL;
  if (M == 0 || n_seg == 0) return XS_OK;
  const f8::GemmArgs p{static_cast<const uint8_t*>(a), lda, a_scales, lda_s, static_cast<const uint8_t*>(b), K,
                       static_cast<int64_t>(N) * K, b_scales, ldb_s, static_cast<int64_t>((N + 127) / 128) * ldb_s,
                       static_cast<char*>(c), ldc, M, N, K, seg_offsets, seg_rows, n_seg, dev_status, 0};
  hipStream_t st = static_cast<hipStream_t>(stream);
  return swiglu ? launch<false, true, false>(p, st) : launch<false, false, false>(p, st);
}
