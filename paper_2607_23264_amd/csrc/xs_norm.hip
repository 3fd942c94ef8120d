// Root-mean-square norm of a residual stream, with an E4M3 result, and its gradients.
//
//   h = bf16(x + r)          y_c = h_c w_c i,  i = (sum_c h_c^2 / n + eps)^(-1/2)
//   u_c = h_c i              dh_c = i (g_c - u_c sum_c g_c u_c / n) + (the gradient that h has besides),  g_c = dy_c w_c
//                            dw_c = sum over rows of dy_c u_c
//
// h is rounded before the norm, so that the gradient, which starts from the h that was kept, is the gradient of
// what was computed, and needs nothing else from the forward pass: the two row sums of the gradient
// (h^2 and g h) come from the same read. Everything after h is fp32, rounded once.
//
// A row is NT threads' pieces of eight values (16 bytes), held in registers from the one read to the
// write; sixteen lanes hold a block of 128 and take its scale.
//
// Bound by memory: 16,381 x 7168 with the residual, bf16 and E4M3 results 197 us, 5.4 TB/s (a large copy: 4.9), its gradients 189 us, 5.0 TB/s, and 4.8 to
// add dw up; 24 rows 4.3 us, a chain of two loads, a sum and a store.
#include <cfloat>
#include <cmath>

#include "xs_common.hpp"
#include "xs_fp8.hpp"

namespace xs {
namespace norm {

constexpr u32x4 kZero4 = {0, 0, 0, 0};

struct Args {
  const uint16_t *x, *r;
  int64_t ldx, ldr;
  const void* w;
  int w32;
  float eps;
  int64_t rows;
  int cols;
  uint16_t *h, *y;
  int64_t ldh, ldy;
  uint8_t* codes;
  int64_t ldc;
  float* scales;
  int64_t lds;
};

struct GradArgs {
  const uint16_t *dy, *dh, *h;
  int64_t lddy, lddh, ldh;
  const void* w;
  int w32;
  float eps;
  int64_t rows;
  int cols;
  uint16_t* dx;
  int64_t lddx;
  float* part;          // [workgroups][cols], or NULL
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Eight weights of columns col .. + 7 as fp32. The compiler keeps every piece's address, two registers each, over a loop of rows; unless HELD it
// gets an offset from the scalar address anew. (Gradients of 16,381 x 7168: held 208 us, anew 193; a wave a row, 8000 x 2048: 39.1 and 41.4.)
struct W8 {
  float v[8];
};
template <bool HELD>
__device__ __forceinline__ W8 weights8(const void* w, int w32, int col) {
  W8 o;
  uint32_t at = static_cast<uint32_t>(col);
  if constexpr (!HELD) asm volatile("" : "+v"(at));
  if (w32) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(static_cast<const char*>(w) + at * 4);
    const f32x4 b = *reinterpret_cast<const f32x4*>(static_cast<const char*>(w) + at * 4 + 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o.v[e] = a[e];
      o.v[4 + e] = b[e];
    }
  } else {
    const u32x4 a = *reinterpret_cast<const u32x4*>(static_cast<const char*>(w) + at * 2);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o.v[2 * e] = bf_lo(a[e]);
      o.v[2 * e + 1] = bf_hi(a[e]);
    }
  }
  return o;
}

// Sums of one value (or two) over the NT threads of a row; RP rows to a workgroup.
template <int NT>
__device__ __forceinline__ float row_sum(float v, float* red, int row) {
  v = wave_sum(v);
  if constexpr (NT == 64) return v;
  constexpr int NW = NT / 64;
  const int w = (threadIdx.x % NT) >> 6;
  if ((threadIdx.x & 63) == 0) red[row * NW + w] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) v += red[row * NW + i];
  return v;
}

// The power of two that a row's values are multiplied with before they are squared: 1, unless the sum ss of their squares has left fp32's range.
// 2^-80 where it is infinite (a value of 2^56 or more; the largest are below 2^48 then), 2^80 where the mean and eps are below 2^-80, so
// that squares which fp32 does not hold may weigh in it (values below 2^-32, then below 2^48).
__device__ __forceinline__ float unit_of(float ss, float n, float eps) {
  return !(ss <= FLT_MAX) ? 0x1p-80f : ss < 0x1p-80f * n && eps < 0x1p-80f ? 0x1p80f : 1.f;
}

// EARLY: the weights are read with the row, not behind its sum (few rows, where a kernel's time is its chain of loads).
template <int NT, int NP, int RP, bool EARLY>
__global__ __launch_bounds__(NT * RP) void norm_kernel(Args a) {
  __shared__ float red[NT > 64 ? RP * NT / 64 : 1];
  const int in = threadIdx.x / NT, t = threadIdx.x % NT;
  const int64_t row = block_number() * RP + in;
  const bool live = row < a.rows;
  if (NT > 64 && block_number() * RP >= a.rows) return;      // the whole workgroup (surplus of the grid)
  u32x4 h[NP];
  W8 early[EARLY ? NP : 1];
  float ss = 0.f;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int col = (p * NT + t) * 8;
    h[p] = kZero4;
    if (live && col < a.cols) {
      h[p] = *reinterpret_cast<const u32x4*>(a.x + row * a.ldx + col);
      if constexpr (EARLY) early[p] = weights8<false>(a.w, a.w32, col);
      if (a.r) {
        const u32x4 r = *reinterpret_cast<const u32x4*>(a.r + row * a.ldr + col);
#pragma unroll
        for (int e = 0; e < 4; ++e) h[p][e] = pack_bf16x2(bf_lo(h[p][e]) + bf_lo(r[e]), bf_hi(h[p][e]) + bf_hi(r[e]));
      }
      if (a.h) *reinterpret_cast<u32x4*>(a.h + row * a.ldh + col) = h[p];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) ss = __builtin_fmaf(bf_lo(h[p][e]), bf_lo(h[p][e]), __builtin_fmaf(bf_hi(h[p][e]), bf_hi(h[p][e]), ss));
  }
  const float n = static_cast<float>(a.cols);
  ss = row_sum<NT>(ss, red, in);
  const float k = unit_of(ss, n, a.eps);
  if (k != 1.f) {            // the same in the whole row, which is a wave or the workgroup
    if (NT > 64) __syncthreads();                 // the first sums have been read
    ss = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float h0 = bf_lo(h[p][e]) * k, h1 = bf_hi(h[p][e]) * k;
        ss = __builtin_fmaf(h0, h0, __builtin_fmaf(h1, h1, ss));
      }
    ss = row_sum<NT>(ss, red, in);
  }
  const float inv = k / sqrtf(ss / n + a.eps * k * k);
  const int padded = (a.cols + 127) & ~127;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int col = (p * NT + t) * 8;
    float y[8] = {};
    if (col < a.cols) {
      const W8 w = EARLY ? early[EARLY ? p : 0] : weights8<false>(a.w, a.w32, col);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        y[2 * e] = bf_lo(h[p][e]) * inv * w.v[2 * e];
        y[2 * e + 1] = bf_hi(h[p][e]) * inv * w.v[2 * e + 1];
      }
      if (live && a.y) {
        const u32x4 o = {pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7])};
        *reinterpret_cast<u32x4*>(a.y + row * a.ldy + col) = o;
      }
    }
    if (a.codes) {
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(y[e]) & 0x7FFFFFFFu);
      const f8::Scale s = f8::scale_of(f8::max16(top));
      if (live && col < padded) {
        *reinterpret_cast<uint2*>(a.codes + row * a.ldc + col) = make_uint2(f8::codes4(y[0], y[1], y[2], y[3], s), f8::codes4(y[4], y[5], y[6], y[7], s));
        if ((t & 15) == 0) a.scales[row * a.lds + (col >> 7)] = s.s;
      }
    }
  }
}

// A workgroup takes rows in turn, RP at a time, and keeps the sums of dw of its columns in registers; they are
// joined over the workgroup in LDS and over the workgroups by sum_kernel, in a fixed order.
template <int NT, int NP, int RP>
__global__ __launch_bounds__(NT * RP) void norm_grad_kernel(GradArgs a) {
  __shared__ float red[2][NT > 64 ? RP * NT / 64 : 1];
  __shared__ __attribute__((aligned(16))) float join[RP > 1 ? NT * 8 : 4];
  const int in = threadIdx.x / NT, t = threadIdx.x % NT;
  float dw[NP][8];
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[p][e] = 0.f;
  const float n = static_cast<float>(a.cols);
  for (int64_t base = static_cast<int64_t>(blockIdx.x) * RP; base < a.rows; base += static_cast<int64_t>(gridDim.x) * RP) {
    const int64_t row = base + in;
    const bool live = row < a.rows;
    u32x4 h[NP], dy[NP], dh[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int col = (p * NT + t) * 8;
      h[p] = dy[p] = dh[p] = kZero4;
      if (live && col < a.cols) {
        h[p] = *reinterpret_cast<const u32x4*>(a.h + row * a.ldh + col);
        dy[p] = *reinterpret_cast<const u32x4*>(a.dy + row * a.lddy + col);
        if (a.dh) dh[p] = *reinterpret_cast<const u32x4*>(a.dh + row * a.lddh + col);
      }
    }
    float ss = 0.f, sg = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int col = (p * NT + t) * 8;
      if (col < a.cols) {
        const W8 w = weights8<NT == 64>(a.w, a.w32, col);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float h0 = bf_lo(h[p][e]), h1 = bf_hi(h[p][e]);
          ss = __builtin_fmaf(h0, h0, __builtin_fmaf(h1, h1, ss));
          sg = __builtin_fmaf(bf_lo(dy[p][e]) * w.v[2 * e], h0, __builtin_fmaf(bf_hi(dy[p][e]) * w.v[2 * e + 1], h1, sg));
        }
      }
    }
    if (NT > 64) __syncthreads();                  // the last row's sums have been read
    ss = row_sum<NT>(ss, red[0], in);
    sg = row_sum<NT>(sg, red[1], in);
    const float k = unit_of(ss, n, a.eps);
    bool again = k != 1.f;
    if constexpr (NT > 64 && RP > 1) {             // of any of the workgroup's rows
#pragma unroll
      for (int r = 0; r < RP; ++r) {
        float other = 0.f;
#pragma unroll
        for (int i = 0; i < NT / 64; ++i) other += red[0][r * (NT / 64) + i];
        again |= unit_of(other, n, a.eps) != 1.f;
      }
    }
    if (again) {
      ss = sg = 0.f;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int col = (p * NT + t) * 8;
        if (col < a.cols) {
          const W8 w = weights8<NT == 64>(a.w, a.w32, col);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float h0 = bf_lo(h[p][e]) * k, h1 = bf_hi(h[p][e]) * k;
            ss = __builtin_fmaf(h0, h0, __builtin_fmaf(h1, h1, ss));
            sg = __builtin_fmaf(bf_lo(dy[p][e]) * w.v[2 * e], h0, __builtin_fmaf(bf_hi(dy[p][e]) * w.v[2 * e + 1], h1, sg));
          }
        }
      }
      if (NT > 64) __syncthreads();                // the first sums have been read
      ss = row_sum<NT>(ss, red[0], in);
      sg = row_sum<NT>(sg, red[1], in);
    }
    const float root = 1.f / sqrtf(ss / n + a.eps * k * k), inv = k * root;
    const float c = sg * root / n * inv;            // of h, inside the brackets: u sum(g u) / n = h i (sg i) / n
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int col = (p * NT + t) * 8;
      if (col >= a.cols) continue;
      const W8 w = weights8<NT == 64>(a.w, a.w32, col);
      u32x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float h0 = bf_lo(h[p][e]), h1 = bf_hi(h[p][e]), y0 = bf_lo(dy[p][e]), y1 = bf_hi(dy[p][e]);
        o[e] = pack_bf16x2(__builtin_fmaf(inv, __builtin_fmaf(-h0, c, y0 * w.v[2 * e]), bf_lo(dh[p][e])),
                           __builtin_fmaf(inv, __builtin_fmaf(-h1, c, y1 * w.v[2 * e + 1]), bf_hi(dh[p][e])));
        if (live) {
          dw[p][2 * e] = __builtin_fmaf(y0, h0 * inv, dw[p][2 * e]);
          dw[p][2 * e + 1] = __builtin_fmaf(y1, h1 * inv, dw[p][2 * e + 1]);
        }
      }
      if (live) *reinterpret_cast<u32x4*>(a.dx + row * a.lddx + col) = o;
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int col = (p * NT + t) * 8;
    if constexpr (RP > 1) {
      for (int r = 1; r < RP; ++r) {
        __syncthreads();
        if (in == r)
#pragma unroll
          for (int e = 0; e < 8; ++e) join[e * NT + t] = dw[p][e];
        __syncthreads();
        if (in == 0)
#pragma unroll
          for (int e = 0; e < 8; ++e) dw[p][e] += join[e * NT + t];
      }
    }
    if (in == 0 && col < a.cols) {
      float* const o = a.part + static_cast<int64_t>(blockIdx.x) * a.cols + col;
      *reinterpret_cast<f32x4*>(o) = f32x4{dw[p][0], dw[p][1], dw[p][2], dw[p][3]};
      *reinterpret_cast<f32x4*>(o + 4) = f32x4{dw[p][4], dw[p][5], dw[p][6], dw[p][7]};
    }
  }
}

// dw[c] = sum over n parts: sixteen threads of a workgroup have four columns each, 64 groups of threads every 64th part, eight of
// them on their way at once.
__global__ __launch_bounds__(1024) void sum_kernel(const float* __restrict__ part, int n, int cols, float* __restrict__ dw) {
  __shared__ __attribute__((aligned(16))) f32x4 red[16][16];
  const int q = threadIdx.x & 15, g = threadIdx.x >> 4, col = (blockIdx.x * 16 + q) * 4;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (col < cols)
    for (int i = g; i < n; i += 8 * 64) {
      f32x4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const f32x4*>(part + static_cast<int64_t>(min(i + 64 * u, n - 1)) * cols + col);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (i + 64 * u < n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] += v[u][e];
    }
#pragma unroll
  for (int d = 16; d < 64; d <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += __shfl_xor(s[e], d);
  if ((threadIdx.x & 63) < 16) red[threadIdx.x >> 6][q] = s;
  __syncthreads();
  if (g || col >= cols) return;
#pragma unroll
  for (int w = 1; w < 16; ++w)
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += red[w][q][e];
  *reinterpret_cast<f32x4*>(dw + col) = s;
}

constexpr int kMaxCols = 32768;

}  // namespace norm
}  // namespace xs

using namespace xs;

namespace {

bool lies_at(const void* p, int64_t ld, int32_t cols, int64_t rows) {     // a bf16 matrix of 16-byte pieces; NULL if it has no rows
  return (p || rows == 0) && !(reinterpret_cast<uintptr_t>(p) & 15) && ld >= cols && ld % 8 == 0 && ld < (int64_t(1) << 40);
}

int norm_ok(const void* w, int32_t wt, float eps, int64_t rows, int32_t cols) {
  if (!w || (reinterpret_cast<uintptr_t>(w) & 15) || (wt != XS_TYPE_BF16 && wt != XS_TYPE_F32)) return XS_EINVAL;
  if (!(eps >= 0.f) || !std::isfinite(eps) || rows < 0 || cols < 1) return XS_EINVAL;
  if (cols % 8 || cols > norm::kMaxCols || rows >= (int64_t(1) << 31)) return XS_EUNSUPPORTED;
  return XS_OK;
}

// Workgroups of the gradient, a function of the shape and the device alone (the order of dw's sum).
int grad_groups(int64_t rows, int32_t cols) {
  const int rp = cols <= 2048 ? 4 : cols <= 8192 ? 2 : 1;
  const int64_t most = (rows + rp - 1) / rp, want = 2 * int64_t(xs_host::num_cus());
  return static_cast<int>(most < want ? most : want);
}

template <template <int, int, int> class L, class A>
void by_columns(const A& a, hipStream_t st) {
  const int pieces = a.cols / 8 + (a.cols % 8 != 0);
  // a wave a row up to 2048 columns, 256 threads up to 8192
  if (pieces <= 64) L<64, 1, 4>::go(a, st);
  else if (pieces <= 128) L<64, 2, 4>::go(a, st);
  else if (pieces <= 256) L<64, 4, 4>::go(a, st);
  else if (pieces <= 512) L<256, 2, 2>::go(a, st);
  else if (pieces <= 768) L<256, 3, 2>::go(a, st);
  else if (pieces <= 1024) L<256, 4, 2>::go(a, st);
  else if (pieces <= 2048) L<1024, 2, 1>::go(a, st);
  else L<1024, 4, 1>::go(a, st);
}

template <int NT, int NP, int RP>
struct Forward {
  static void go(const norm::Args& a, hipStream_t st) {
    constexpr int rp = NT == 64 ? RP : 1;
    hipLaunchKernelGGL((norm::norm_kernel<NT, NP, rp, false>), xs_host::grid_of((a.rows + rp - 1) / rp), dim3(NT * rp), 0, st, a);
  }
};
// Few rows: as many threads a row as it has pieces.
template <int NT, int NP>
void forward_few(const norm::Args& a, hipStream_t st) {
  hipLaunchKernelGGL((norm::norm_kernel<NT, NP, 1, true>), xs_host::grid_of(a.rows), dim3(NT), 0, st, a);
}
template <int NT, int NP, int RP>
struct Backward {
  static void go(const norm::GradArgs& a, hipStream_t st) {
    hipLaunchKernelGGL((norm::norm_grad_kernel<NT, NP, RP>), dim3(grad_groups(a.rows, a.cols)), dim3(NT * RP), 0, st, a);
  }
};

}  // namespace

extern "C" int xs_rmsnorm(const void* x, int64_t ldx, const void* residual, int64_t ld_res, const void* weight,
                          int32_t weight_type, float eps, int64_t rows, int32_t cols, void* h, int64_t ld_h, void* y,
                          int64_t ld_y, void* codes, int64_t ld_codes, float* scales, int64_t ld_scales, void* stream) {
  if (int rc = norm_ok(weight, weight_type, eps, rows, cols)) return rc;
  if (!lies_at(x, ldx, cols, rows) || (residual && !lies_at(residual, ld_res, cols, rows)) || (h && !lies_at(h, ld_h, cols, rows)) ||
      (y && !lies_at(y, ld_y, cols, rows)) || (!y && !codes && rows) || (!codes != !scales))
    return XS_EINVAL;
  if (codes) {
    const int blocks = (cols + 127) / 128;
    if ((reinterpret_cast<uintptr_t>(codes) & 15) || (reinterpret_cast<uintptr_t>(scales) & 15) || ld_codes < blocks * 128 ||
        ld_codes % 16 || ld_scales < blocks || ld_scales % 4 || ld_codes >= (int64_t(1) << 40) || ld_scales >= (int64_t(1) << 40))
      return XS_EINVAL;
  }
  // a result in the place of an input: rows lie where the input's rows do
  const auto shifted = [](const void* o, int64_t ldo, const void* i, int64_t ldi) { return o && o == i && ldo != ldi; };
  if (shifted(h, ld_h, x, ldx) || shifted(h, ld_h, residual, ld_res) || shifted(y, ld_y, x, ldx) || shifted(y, ld_y, residual, ld_res))
    return XS_EINVAL;
  if (h && h == y) return XS_EINVAL;
  if (rows == 0) return XS_OK;
  const norm::Args a{static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(residual), ldx, ld_res, weight,
                     weight_type == XS_TYPE_F32, eps, rows, cols, static_cast<uint16_t*>(h), static_cast<uint16_t*>(y), ld_h, ld_y,
                     static_cast<uint8_t*>(codes), ld_codes, scales, ld_scales};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (rows > xs_host::num_cus()) by_columns<Forward>(a, st);
  else if (cols <= 512) forward_few<64, 1>(a, st);
  else if (cols <= 2048) forward_few<256, 1>(a, st);
  else if (cols <= 8192) forward_few<1024, 1>(a, st);
  else if (cols <= 16384) forward_few<1024, 2>(a, st);
  else forward_few<1024, 4>(a, st);
  return xs_host::launch_status();
}

extern "C" int xs_rmsnorm_backward_workspace_bytes(int64_t rows, int32_t cols, int64_t* bytes) {
  if (!bytes || rows < 0 || cols < 1) return XS_EINVAL;
  if (cols % 8 || cols > norm::kMaxCols || rows >= (int64_t(1) << 31)) return XS_EUNSUPPORTED;
  *bytes = static_cast<int64_t>(grad_groups(rows, cols)) * cols * 4;
  return XS_OK;
}

extern "C" int xs_rmsnorm_backward(const void* dy, int64_t ld_dy, const void* dh, int64_t ld_dh, const void* h, int64_t ld_h,
                                   const void* weight, int32_t weight_type, float eps, int64_t rows, int32_t cols, void* dx,
                                   int64_t ld_dx, float* d_weight, void* workspace, int64_t workspace_bytes, void* stream) {
  if (int rc = norm_ok(weight, weight_type, eps, rows, cols)) return rc;
  if (!lies_at(dy, ld_dy, cols, rows) || (dh && !lies_at(dh, ld_dh, cols, rows)) || !lies_at(h, ld_h, cols, rows) || !lies_at(dx, ld_dx, cols, rows) ||
      (reinterpret_cast<uintptr_t>(d_weight) & 15))
    return XS_EINVAL;
  const auto shifted = [=](const void* i, int64_t ldi) { return dx && dx == i && ld_dx != ldi; };
  if (shifted(dy, ld_dy) || shifted(dh, ld_dh) || shifted(h, ld_h)) return XS_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int groups = grad_groups(rows, cols);
  if (d_weight && groups) {
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15) || workspace_bytes < static_cast<int64_t>(groups) * cols * 4)
      return XS_EWORKSPACE;
  }
  if (rows) {
    const norm::GradArgs a{static_cast<const uint16_t*>(dy), static_cast<const uint16_t*>(dh), static_cast<const uint16_t*>(h),
                           ld_dy, ld_dh, ld_h, weight, weight_type == XS_TYPE_F32, eps, rows, cols, static_cast<uint16_t*>(dx), ld_dx,
                           d_weight ? static_cast<float*>(workspace) : nullptr};
    by_columns<Backward>(a, st);
    if (xs_host::launch_status()) return XS_EHIP;
  }
  if (!d_weight) return XS_OK;
  hipLaunchKernelGGL(norm::sum_kernel, dim3((cols + 63) / 64), dim3(1024), 0, st, static_cast<const float*>(workspace), groups, cols, d_weight);
  return xs_host::launch_status();
}
