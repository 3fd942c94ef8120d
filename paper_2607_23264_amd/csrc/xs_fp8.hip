// E4M3 with one fp32 scale per block of 128 (its arithmetic: xs_fp8.hpp): the quantizers, and SwiGLU with an
// 8-bit result and an 8-bit checkpoint.
#include <algorithm>

#include "xs_common.hpp"
#include "xs_fp8.hpp"

namespace xs {
namespace f8 {

constexpr u32x4 kZero4 = {0, 0, 0, 0};

// ------------------------------------------------------------------------------ 1 x 128 along rows
// Sixteen lanes per block, one 16-byte piece of eight values each. 16,381 rows of 7168: 68.4 us, a copy's rate.
__global__ __launch_bounds__(256) void quantize_rows_kernel(const uint16_t* __restrict__ x, int64_t ldx, int64_t rows,
                                                            int cols, uint8_t* __restrict__ codes, int64_t ldc,
                                                            float* __restrict__ scales, int64_t lds) {
  const int blocks = (cols + 127) / 128, sub = threadIdx.x & 15;
  const int64_t i = block_number() * 16 + (threadIdx.x >> 4);
  const bool live = i < rows * blocks;
  const int64_t r = i / blocks;
  const int b = static_cast<int>(i - r * blocks), col = b * 128 + sub * 8;
  u32x4 raw = kZero4;
  if (live && col < cols) raw = *reinterpret_cast<const u32x4*>(x + r * ldx + col);
  const Scale s = scale_of(amax_f32(max16_packed(amax8(raw))));
  if (live) {
    *reinterpret_cast<uint2*>(codes + r * ldc + col) = codes8(raw, s);
    if (sub == 0) scales[r * lds + b] = s.s;
  }
}

// ------------------------------------------------------------------------------ 128 x 128 regions
// One workgroup per 128 x 128 region of x, read once: the blocks along the rows (ROWS), along the
// columns (COLS, written transposed), or the region as one block (TILE), in either orientation.
// Thread (rg = tid / 16, cg = tid % 16) has rows 8 rg .. + 7 and columns 8 cg .. + 7: a row of the
// region is 16 lanes' pieces (256 contiguous bytes), and a column's eight values in a thread are eight
// consecutive codes of the transposed row. Those go through LDS ([128 columns][128 codes], pitch
// kPitchT) so that the stores are whole 128-byte rows. Each scale's two divisions are one lane's work:
// every thread taking its own eight rows' and eight columns' held 260 registers and took 301 us where
// this takes 102 (16,381 rows of 7168 both ways: 4.7 TB/s, a copy's rate being 5.2).
constexpr int kPitchT = 144;
// Regions in order: 32 row blocks of a column block, then the next column block, so that the 128-byte
// pieces of a transposed row are written together; each XCD (consecutive workgroups go to different ones)
// takes four consecutive row blocks, whose scales of a column are neighbours. Measured with 16 / 32 / 64 /
// 128 row blocks (16,384 rows of 7168): transposed 87.0 / 77.8 / 76.0 / 73.9 us, both ways 109.1 / 105.2 /
// 107.6 / 107.0, tiles both ways 100.0 / 94.6 / 97.4 / 96.8, tiles alone 68.1 / 68.2 / 70.4 / 72.6; with
// consecutive row blocks on different XCDs 78.6, 105.6, 96.9, 68.5.
constexpr int kGroupR = 32;
struct RegionArgs {
  const uint16_t* x;
  int64_t ldx;
  int64_t rows;
  int cols, col_blocks;
  uint8_t* codes;
  int64_t ldc;
  float* scales;
  int64_t lds;
  uint8_t* codes_t;
  int64_t ldc_t;
  float* scales_t;
  int64_t lds_t;
};

template <bool TILE, bool ROWS, bool COLS>
__global__ __launch_bounds__(256, 4) void quantize_region_kernel(RegionArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t tr[COLS ? 128 * kPitchT : 16];
  __shared__ __attribute__((aligned(16))) uint32_t red[4][64];     // per wave: column maxima (packed pairs)
  __shared__ __attribute__((aligned(16))) float2 col_s[COLS && !TILE ? 128 : 1];
  const int tid = threadIdx.x, w = tid >> 6, rg = tid >> 4, cg = tid & 15;
  const int64_t id = block_number(), per_group = static_cast<int64_t>(kGroupR) * a.col_blocks;
  const int64_t first = id / per_group * kGroupR, in = id % per_group;
  const int64_t left = (a.rows + 127) / 128 - first;
  if (left <= 0) return;                            // the whole workgroup (surplus of the grid)
  const int gm = static_cast<int>(min(left, static_cast<int64_t>(kGroupR)));
  const int cb = static_cast<int>(in / gm);
  const int64_t rb = first + (gm == kGroupR ? in % 8 * (kGroupR / 8) + in / 8 % (kGroupR / 8) : in % gm);
  if (cb >= a.col_blocks) return;
  const int64_t row0 = rb * 128;
  const int col = cb * 128 + cg * 8;
  const int rows = static_cast<int>(min(a.rows - row0, static_cast<int64_t>(128)));
  const uint16_t* const x = a.x + row0 * a.ldx + col;
  u32x4 raw[8];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    raw[p] = kZero4;
    if (8 * rg + p < rows && col < a.cols) raw[p] = *reinterpret_cast<const u32x4*>(x + (8 * rg + p) * a.ldx);
  }
  Scale tile{};
  if constexpr (TILE) {
    uint32_t v = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) v = max2(v, amax8(raw[p]));
    v = max16_packed(v);
    if (cg == 0) red[w][rg & 3] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) v = max2(v, red[i >> 2][i & 3]);
    tile = scale_of(amax_f32(v));
  } else if constexpr (COLS) {
    // the columns' maxima: over the thread's rows, the wave's four row groups, the four waves
    uint32_t cm[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      cm[i] = 0;
#pragma unroll
      for (int p = 0; p < 8; ++p) cm[i] = max2(cm[i], mag2(raw[p][i]));
      cm[i] = max2(cm[i], static_cast<uint32_t>(__shfl_xor(static_cast<int>(cm[i]), 16)));
      cm[i] = max2(cm[i], static_cast<uint32_t>(__shfl_xor(static_cast<int>(cm[i]), 32)));
    }
    if ((tid & 63) < 16) *reinterpret_cast<u32x4*>(&red[w][cg * 4]) = u32x4{cm[0], cm[1], cm[2], cm[3]};
    __syncthreads();
    // one thread a column: a scale and its reciprocal are two divisions
    if (tid < 128) {
      uint32_t v = red[0][tid >> 1];
#pragma unroll
      for (int ww = 1; ww < 4; ++ww) v = max2(v, red[ww][tid >> 1]);
      const Scale s = scale_of(tid & 1 ? v & 0xFFFF0000u : v << 16);
      col_s[tid] = make_float2(s.s, s.inv);
      if (cb * 128 + tid < a.cols) a.scales_t[static_cast<int64_t>(cb * 128 + tid) * a.lds_t + rb] = s.s;
    }
  }
  if constexpr (ROWS) {
    // a row's maximum is known to its sixteen lanes: lane p takes row p's divisions
    Scale mine{};
    if constexpr (!TILE) {
      uint32_t v = 0;
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        const uint32_t m = max16_packed(amax8(raw[p]));
        v = (cg & 7) == p ? m : v;
      }
      mine = scale_of(amax_f32(v));
      if (cg < 8 && 8 * rg + cg < rows) a.scales[(row0 + 8 * rg + cg) * a.lds + cb] = mine.s;
    }
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const Scale s = TILE ? tile : scale_from(__shfl(mine.s, p, 16), __shfl(mine.inv, p, 16));
      if (8 * rg + p < rows) *reinterpret_cast<uint2*>(a.codes + (row0 + 8 * rg + p) * a.ldc + col) = codes8(raw[p], s);
    }
    if (TILE && tid == 0) a.scales[rb * a.lds + cb] = tile.s;
  }
  if constexpr (COLS) {
    if constexpr (!TILE) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Scale s = tile;
        if constexpr (!TILE) {
          const float2 c = col_s[8 * cg + 2 * i + h];
          s = scale_from(c.x, c.y);
        }
        float v[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) v[p] = h ? bf_hi(raw[p][i]) : bf_lo(raw[p][i]);
        *reinterpret_cast<uint2*>(tr + (8 * cg + 2 * i + h) * kPitchT + 8 * rg) =
            make_uint2(codes4(v[0], v[1], v[2], v[3], s), codes4(v[4], v[5], v[6], v[7], s));
      }
    }
    if (TILE && tid == 0) a.scales_t[static_cast<int64_t>(cb) * a.lds_t + rb] = tile.s;
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int c = p * 32 + (tid >> 3), pc = tid & 7;
      if (cb * 128 + c < a.cols)
        *reinterpret_cast<u32x4*>(a.codes_t + static_cast<int64_t>(cb * 128 + c) * a.ldc_t + row0 + pc * 16) =
            *reinterpret_cast<const u32x4*>(tr + c * kPitchT + pc * 16);
    }
  }
}

// ------------------------------------------------------------------------------ SwiGLU
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.f + __expf(-g)); }

__device__ __forceinline__ void unpack8(u32x4 r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[2 * i] = bf_lo(r[i]), v[2 * i + 1] = bf_hi(r[i]);
}

struct SwigluArgs {
  const uint16_t* gu;
  int64_t ld_gu;
  int64_t rows;
  int I;
  uint8_t* h;
  int64_t ld_h;
  float* h_s;
  int64_t ld_hs;
  uint8_t* ck;
  int64_t ld_ck;
  float* ck_s;
  int64_t ld_cks;
};

// h = silu(g) u in fp32, its blocks of 128 columns quantized; with KEEP the gate and up values too, each
// in its own blocks. Sixteen lanes per block of h, eight columns each. 32,768 x 2048 with KEEP: 93-97 us, memory (a copy's
// rate) and vector issue (90 % of slots) at once. The sigmoid by the reciprocal unit is off by up to an fp32 unit more than a
// division; the codes' error against 64 bits is that of fp32 divisions all the same (2.4e-4; 2.2e-4 with silu as a
// quotient of one rounding, which took 4.6 % longer).
template <bool KEEP>
__global__ __launch_bounds__(256) void swiglu_fp8_kernel(SwigluArgs a) {
  const int blocks = a.I / 128;
  const int64_t i = block_number() * 16 + (threadIdx.x >> 4);
  const int sub = threadIdx.x & 15;
  const bool live = i < a.rows * blocks;
  const int64_t r = live ? i / blocks : 0;
  const int b = live ? static_cast<int>(i - r * blocks) : 0;
  const int col = b * 128 + sub * 8;
  const uint16_t* const row = a.gu + r * a.ld_gu;
  const u32x4 graw = *reinterpret_cast<const u32x4*>(row + col);
  const u32x4 uraw = *reinterpret_cast<const u32x4*>(row + a.I + col);
  float g[8], u[8];
  unpack8(graw, g);
  unpack8(uraw, u);
  uint32_t amax = 0;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    g[c] = g[c] * sigmoid(g[c]) * u[c];
    amax = max(amax, __float_as_uint(g[c]) & 0x7FFFFFFFu);
  }
  const Scale s = scale_of(max16(amax));
  const uint2 hc = make_uint2(codes4(g[0], g[1], g[2], g[3], s), codes4(g[4], g[5], g[6], g[7], s));
  if (live) {
    *reinterpret_cast<uint2*>(a.h + r * a.ld_h + col) = hc;
    if (sub == 0) a.h_s[r * a.ld_hs + b] = s.s;
  }
  if constexpr (KEEP) {
    const Scale sg = scale_of(amax_f32(max16_packed(amax8(graw))));
    const Scale su = scale_of(amax_f32(max16_packed(amax8(uraw))));
    const uint2 gc = codes8(graw, sg), uc = codes8(uraw, su);
    if (live) {
      *reinterpret_cast<uint2*>(a.ck + r * a.ld_ck + col) = gc;
      *reinterpret_cast<uint2*>(a.ck + r * a.ld_ck + a.I + col) = uc;
      if (sub == 0) {
        a.ck_s[r * a.ld_cks + b] = sg.s;
        a.ck_s[r * a.ld_cks + blocks + b] = su.s;
      }
    }
  }
}

struct SwigluGradArgs {
  const uint8_t* ck;
  int64_t ld_ck;
  const float* ck_s;
  int64_t ld_cks;
  const uint16_t* dh;
  int64_t ld_dh;
  int64_t rows;
  int I;
  uint16_t* dgu;
  int64_t ld_dgu;
  uint16_t* h;
  int64_t ld_h;
};

__device__ __forceinline__ void values8(uint2 c, float s, float (&v)[8]) {
  typedef float f32x2_ __attribute__((ext_vector_type(2)));
  const f32x2_ a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c.x), false), b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c.x), true);
  const f32x2_ d = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c.y), false), e = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(c.y), true);
  v[0] = a[0] * s, v[1] = a[1] * s, v[2] = b[0] * s, v[3] = b[1] * s;
  v[4] = d[0] * s, v[5] = d[1] * s, v[6] = e[0] * s, v[7] = e[1] * s;
}

__device__ __forceinline__ u32x4 pack8(const float (&v)[8]) {
  return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

// dg = dh u sig (1 + g (1 - sig)), du = dh g sig and, with H, h = g sig u, from the checkpoint's g and u. Bound by memory:
// 32,768 x 2048 with H 120 us, 5.6 TB/s.
template <bool H>
__global__ __launch_bounds__(256) void swiglu_fp8_grad_kernel(SwigluGradArgs a) {
  const int pieces = a.I / 8;
  const int64_t i = block_number() * 256 + threadIdx.x;
  if (i >= a.rows * pieces) return;
  const int64_t r = i / pieces;
  const int col = static_cast<int>(i - r * pieces) * 8;
  const uint2 gc = *reinterpret_cast<const uint2*>(a.ck + r * a.ld_ck + col);
  const uint2 uc = *reinterpret_cast<const uint2*>(a.ck + r * a.ld_ck + a.I + col);
  const u32x4 draw = *reinterpret_cast<const u32x4*>(a.dh + r * a.ld_dh + col);
  const float* const sc = a.ck_s + r * a.ld_cks + col / 128;
  float g[8], u[8], d[8], dg[8], du[8], h[8];
  values8(gc, sc[0], g);
  values8(uc, sc[a.I / 128], u);
  unpack8(draw, d);
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const float sig = sigmoid(g[c]), act = g[c] * sig;
    h[c] = act * u[c];
    du[c] = d[c] * act;
    dg[c] = d[c] * u[c] * sig * (1.f + g[c] * (1.f - sig));
  }
  *reinterpret_cast<u32x4*>(a.dgu + r * a.ld_dgu + col) = pack8(dg);
  *reinterpret_cast<u32x4*>(a.dgu + r * a.ld_dgu + a.I + col) = pack8(du);
  if constexpr (H) *reinterpret_cast<u32x4*>(a.h + r * a.ld_h + col) = pack8(h);
}

}  // namespace f8
}  // namespace xs

using namespace xs;

namespace {

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int64_t kMaxRows = int64_t(1) << 37;

// A quantized output: codes in rows of whole blocks, scales in rows of at least one per block.
int codes_ok(const void* codes, int64_t ld, const float* scales, int64_t ld_s, int64_t cols) {
  const int64_t blocks = (cols + 127) / 128;
  if (!codes || !scales || ld < blocks * 128 || ld_s < blocks) return XS_EINVAL;
  if (ld % 16 || ld_s % 4 || !aligned_to(codes, 16) || !aligned_to(scales, 16)) return XS_EINVAL;
  return XS_OK;
}

int quantize_ok(const void* x, int64_t rows, int32_t cols, int64_t ldx, const void* codes, int64_t ld_codes,
                const float* scales, int64_t ld_scales, const void* codes_t, int64_t ld_codes_t, const float* scales_t,
                int64_t ld_scales_t) {
  if (!x || rows < 0 || cols <= 0 || (!codes && !codes_t)) return XS_EINVAL;
  if (cols % 8) return XS_EUNSUPPORTED;
  if (ldx < cols || ldx % 8 || !aligned_to(x, 16)) return XS_EINVAL;
  if (cols > (1 << 30) || rows > kMaxRows || (rows + 127) / 128 * ((cols + 127) / 128) > xs_host::kMaxBlocks) return XS_EUNSUPPORTED;
  if (!codes != !scales || !codes_t != !scales_t) return XS_EINVAL;
  if (codes)
    if (int rc = codes_ok(codes, ld_codes, scales, ld_scales, cols)) return rc;
  if (codes_t)
    if (int rc = codes_ok(codes_t, ld_codes_t, scales_t, ld_scales_t, rows)) return rc;
  return XS_OK;
}

template <bool TILE>
int launch_regions(const f8::RegionArgs& a, hipStream_t st) {
  const dim3 grid = xs_host::grid_of((a.rows + 127) / 128 * a.col_blocks);
  if (a.codes && a.codes_t) hipLaunchKernelGGL((f8::quantize_region_kernel<TILE, true, true>), grid, dim3(256), 0, st, a);
  else if (a.codes_t) hipLaunchKernelGGL((f8::quantize_region_kernel<TILE, false, true>), grid, dim3(256), 0, st, a);
  else if constexpr (TILE) hipLaunchKernelGGL((f8::quantize_region_kernel<true, true, false>), grid, dim3(256), 0, st, a);
  return xs_host::launch_status();
}

}  // namespace

extern "C" int xs_quantize_fp8(const void* x, int64_t rows, int32_t cols, int64_t ldx, void* codes, int64_t ld_codes,
                               float* scales, int64_t ld_scales, void* codes_t, int64_t ld_codes_t, float* scales_t,
                               int64_t ld_scales_t, void* stream) {
  int rc = quantize_ok(x, rows, cols, ldx, codes, ld_codes, scales, ld_scales, codes_t, ld_codes_t, scales_t, ld_scales_t);
  if (rc) return rc;
  if (rows == 0) return XS_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (!codes_t) {
    const int64_t groups = (rows * ((cols + 127) / 128) + 15) / 16;
    if (groups > xs_host::kMaxBlocks) return XS_EUNSUPPORTED;
    hipLaunchKernelGGL(f8::quantize_rows_kernel, xs_host::grid_of(groups), dim3(256), 0, st,
                       static_cast<const uint16_t*>(x), ldx, rows, cols, static_cast<uint8_t*>(codes), ld_codes, scales, ld_scales);
    return xs_host::launch_status();
  }
  return launch_regions<false>(f8::RegionArgs{static_cast<const uint16_t*>(x), ldx, rows, cols, (cols + 127) / 128, static_cast<uint8_t*>(codes),
                                              ld_codes, scales, ld_scales, static_cast<uint8_t*>(codes_t), ld_codes_t,
                                              scales_t, ld_scales_t}, st);
}

extern "C" int xs_quantize_fp8_tile(const void* x, int64_t rows, int32_t cols, int64_t ldx, void* codes, int64_t ld_codes,
                                    float* scales, int64_t ld_scales, void* codes_t, int64_t ld_codes_t, float* scales_t,
                                    int64_t ld_scales_t, void* stream) {
  int rc = quantize_ok(x, rows, cols, ldx, codes, ld_codes, scales, ld_scales, codes_t, ld_codes_t, scales_t, ld_scales_t);
  if (rc) return rc;
  if (rows == 0) return XS_OK;
  return launch_regions<true>(f8::RegionArgs{static_cast<const uint16_t*>(x), ldx, rows, cols, (cols + 127) / 128, static_cast<uint8_t*>(codes),
                                             ld_codes, scales, ld_scales, static_cast<uint8_t*>(codes_t), ld_codes_t,
                                             scales_t, ld_scales_t}, static_cast<hipStream_t>(stream));
}

extern "C" int xs_swiglu_fp8(const void* gu, int64_t ld_gu, int64_t rows, int32_t I, void* h_codes, int64_t ld_h,
                             float* h_scales, int64_t ld_hs, void* ck_codes, int64_t ld_ck, float* ck_scales, int64_t ld_cks,
                             void* stream) {
  if (!gu || rows < 0 || I <= 0) return XS_EINVAL;
  if (I % 128 || I > (1 << 29)) return XS_EUNSUPPORTED;
  if (ld_gu < 2 * static_cast<int64_t>(I) || ld_gu % 8 || !aligned_to(gu, 16) || !ck_codes != !ck_scales) return XS_EINVAL;
  int rc = codes_ok(h_codes, ld_h, h_scales, ld_hs, I);
  if (!rc && ck_codes) rc = codes_ok(ck_codes, ld_ck, ck_scales, ld_cks, 2 * static_cast<int64_t>(I));
  if (rc) return rc;
  if (rows == 0) return XS_OK;
  if (rows > kMaxRows || (rows * (I / 128) + 15) / 16 > xs_host::kMaxBlocks) return XS_EUNSUPPORTED;
  const f8::SwigluArgs a{static_cast<const uint16_t*>(gu), ld_gu, rows, I, static_cast<uint8_t*>(h_codes), ld_h, h_scales, ld_hs,
                         static_cast<uint8_t*>(ck_codes), ld_ck, ck_scales, ld_cks};
  const dim3 grid = xs_host::grid_of((rows * (I / 128) + 15) / 16);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (ck_codes) hipLaunchKernelGGL((f8::swiglu_fp8_kernel<true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((f8::swiglu_fp8_kernel<false>), grid, dim3(256), 0, st, a);
  return xs_host::launch_status();
}

extern "C" int xs_swiglu_fp8_backward(const void* ck_codes, int64_t ld_ck, const float* ck_scales, int64_t ld_cks,
                                      const void* dh, int64_t ld_dh, int64_t rows, int32_t I, void* d_gu, int64_t ld_dgu, void* h,
                                      int64_t ld_h, void* stream) {
  if (!dh || !d_gu || rows < 0 || I <= 0) return XS_EINVAL;
  if (I % 128 || I > (1 << 29)) return XS_EUNSUPPORTED;
  int rc = codes_ok(ck_codes, ld_ck, ck_scales, ld_cks, 2 * static_cast<int64_t>(I));
  if (rc) return rc;
  if (ld_dh < I || ld_dh % 8 || !aligned_to(dh, 16) || ld_dgu < 2 * static_cast<int64_t>(I) || ld_dgu % 8 || !aligned_to(d_gu, 16))
    return XS_EINVAL;
  if (h && (ld_h < I || ld_h % 8 || !aligned_to(h, 16))) return XS_EINVAL;
  if (rows == 0) return XS_OK;
  if (rows > kMaxRows || (rows * (I / 128) + 15) / 16 > xs_host::kMaxBlocks) return XS_EUNSUPPORTED;
  const f8::SwigluGradArgs a{static_cast<const uint8_t*>(ck_codes), ld_ck, ck_scales, ld_cks, static_cast<const uint16_t*>(dh), ld_dh,
                             rows, I, static_cast<uint16_t*>(d_gu), ld_dgu, static_cast<uint16_t*>(h), ld_h};
  const dim3 grid = xs_host::grid_of((rows * (I / 8) + 255) / 256);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (h) hipLaunchKernelGGL((f8::swiglu_fp8_grad_kernel<true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((f8::swiglu_fp8_grad_kernel<false>), grid, dim3(256), 0, st, a);
  return xs_host::launch_status();
}
