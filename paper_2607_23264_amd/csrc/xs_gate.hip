// Routing gates: softmax or sigmoid scores, a bias that only the selection sees, groups of experts,
// top-k, renormalized and scaled weights; and the gradient of the weights in the logits.
//
//   s_e = 1 / (1 + exp(-l_e))  or  exp(l_e - m) / sum_f exp(l_f - m)          (0 where l_e = -inf)
//   key_e = s_e + b_e          group score = the largest key, or the sum of the two largest
//   w_j = scale s_j            or, renormalized, scale s_j / S with S = sum_i s_i over the k chosen
//
// Gradient, g_j = dL/dw_j:  ds_j = scale g_j, or scale (g_j - sum_i g_i s_i / S) / S;
//   sigmoid  dl_e = sum_{j: e_j = e} ds_j s_e (1 - s_e)
//   softmax  dl_e = s_e (sum_{j: e_j = e} ds_j - sum_j ds_j s_j)   (renormalized: the second sum is 0)
#include <algorithm>
#include <cmath>

#include "xs_common.hpp"

namespace xs {

struct GateArgs {
  const void* logits;
  int64_t ld;
  const float* bias;
  int T, E, k, score, n_group, topk_group, top2, renorm;
  float scale;
  int* idx;
  float* w;
};

template <typename LT>
__device__ __forceinline__ float load_logit(const void* row, int e) {
  if constexpr (sizeof(LT) == 2) return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(row)[e]) << 16);
  else return static_cast<const float*>(row)[e];
}

template <typename LT>
__device__ __forceinline__ const char* logit_row(const void* logits, int64_t ld, int64_t t) {
  return static_cast<const char*>(logits) + t * ld * static_cast<int64_t>(sizeof(LT));
}

// Keys are finite: a masked expert (logit -inf or NaN, key NaN or below) has the lowest, one outside
// the chosen groups -inf.
constexpr double kMaskedKey = -3.4028234663852886e38;
__device__ __forceinline__ double finite_key(double key, bool masked) {
  return masked || !(key > kMaskedKey) ? kMaskedKey : fmin(key, -kMaskedKey);
}

// One wave per token, everything in 64 bits: any E, k and groups.
template <typename LT>
__global__ __launch_bounds__(256) void gate_wave_kernel(GateArgs g) {
  extern __shared__ double gate_keys[];   // [4][E]
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t t = block_number() * 4 + w;
  if (t >= g.T) return;                   // whole waves; there is no barrier below
  double* const key = gate_keys + w * g.E;
  const char* const row = logit_row<LT>(g.logits, g.ld, t);
  const int E = g.E;
  float m = -INFINITY;
  double sum = 0.;
  if (g.score == XS_SCORE_SOFTMAX) {
    for (int e = lane; e < E; e += 64) m = fmaxf(m, load_logit<LT>(row, e));
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
    for (int e = lane; e < E; e += 64) {
      const float l = load_logit<LT>(row, e);
      if (l != -INFINITY) sum += exp(static_cast<double>(l) - static_cast<double>(m));
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
  }
  const auto score = [&](float l) -> double {
    if (l == -INFINITY) return 0.;
    if (g.score == XS_SCORE_SIGMOID) return 1. / (1. + exp(-static_cast<double>(l)));
    return exp(static_cast<double>(l) - static_cast<double>(m)) / sum;
  };
  // without a bias the logits have the scores' order, and no rounding
  const bool by_logit = !g.bias && (g.n_group == 1 || !g.top2);
  for (int e = lane; e < E; e += 64) {
    const float l = load_logit<LT>(row, e);
    double v = by_logit ? static_cast<double>(l) : score(l);
    if (g.bias) v += static_cast<double>(g.bias[e]);
    key[e] = finite_key(v, l == -INFINITY || l != l);
  }
  __builtin_amdgcn_wave_barrier();
  const auto best = [&](double& bv, int& bi) {   // over the wave; ties to the lower index
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      const double ov = __shfl_xor(bv, off);
      const int oi = __shfl_xor(bi, off);
      if (ov > bv || (ov == bv && oi < bi)) {
        bv = ov;
        bi = oi;
      }
    }
  };
  const int Eg = E / g.n_group;
  if (g.n_group > 1) {
    // lane = group: its two largest keys
    double gs = -INFINITY;
    if (lane < g.n_group) {
      double a = -INFINITY, b = -INFINITY;
      for (int i = 0; i < Eg; ++i) {
        const double v = key[lane * Eg + i];
        if (v > a) {
          b = a;
          a = v;
        } else if (v > b) {
          b = v;
        }
      }
      gs = g.top2 && b > kMaskedKey ? a + b : a;
    }
    bool kept = false;
    double left = gs;
    for (int j = 0; j < g.topk_group; ++j) {
      double bv = left;
      int bi = lane < g.n_group && !kept ? lane : 64 + lane;
      best(bv, bi);
      if (bi == lane) {
        kept = true;
        left = -INFINITY;
      }
    }
    const unsigned long long keep = __ballot(kept);
    for (int e = lane; e < E; e += 64)
      if (!((keep >> (e / Eg)) & 1ull)) key[e] = -INFINITY;
  }
  __builtin_amdgcn_wave_barrier();
  int my_idx = 0;
  double my_s = 0.;
  for (int j = 0; j < g.k; ++j) {
    double bv = -INFINITY;
    int bi = 0x7fffffff;
    for (int e = lane; e < E; e += 64) {
      const double v = key[e];
      if (v > bv) {
        bv = v;
        bi = e;
      }
    }
    best(bv, bi);
    if ((bi & 63) == lane) key[bi] = -INFINITY;
    if (lane == j) {
      my_idx = bi;
      my_s = score(load_logit<LT>(row, bi));
    }
  }
  if (g.renorm) {
    double total = lane < g.k ? my_s : 0.;
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) total += __shfl_xor(total, off);
    my_s = total == 0. ? 0. : my_s / total;
  }
  if (lane < g.k) {
    g.idx[t * g.k + lane] = my_idx;
    g.w[t * g.k + lane] = static_cast<float>(my_s * g.scale);
  }
}

struct GateGradArgs {
  const void* logits;
  int64_t ld;
  int T, E, k, score, renorm;
  float scale;
  const int* idx;
  const float* d_w;
  void* d_logits;
  int64_t ld_d;
  int* status;
};

template <int LPT>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int off = LPT / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  return v;
}
template <int LPT>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int off = LPT / 2; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off));
  return v;
}

// LPT lanes per token; lane `sub` has the experts 4 LPT q + 4 sub + c (q < NQ, c < 4), a vector load or
// store for each q where rows are aligned. Slot j of a token is lane j % LPT's (slots j and, with more
// slots than lanes, none: k <= LPT). The row's logits are read for softmax only; the chosen experts'
// are read one by one for sigmoid. Every lane adds the k slots to its own experts in ascending j, so
// an expert that is listed twice gets both terms and the order of the sum is fixed.
template <typename LT, int LPT, int NQ, bool VEC>
__global__ __launch_bounds__(256) void gate_grad_kernel(GateGradArgs g) {
  const int sub = threadIdx.x % LPT;
  const int64_t t_raw = block_number() * (256 / LPT) + threadIdx.x / LPT;
  const bool live = t_raw < g.T;
  const int64_t t = live ? t_raw : g.T - 1;   // every lane takes part in the sums
  const char* const row = logit_row<LT>(g.logits, g.ld, t);
  const bool softmax = g.score == XS_SCORE_SOFTMAX;
  int e_j = -1;
  float gj = 0.f, l_j = -INFINITY;
  if (sub < g.k) {
    e_j = g.idx[t * g.k + sub];
    if (e_j < 0 || e_j >= g.E) {
      set_status(g.status, XS_EBADINPUT);
      e_j = -1;
    } else {
      gj = g.d_w[t * g.k + sub] * g.scale;
      l_j = load_logit<LT>(row, e_j);
    }
  }
  float v[4 * NQ];
  float m = -INFINITY, inv = 0.f;
  if (softmax) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int e = 4 * LPT * q + 4 * sub;
      if constexpr (VEC) {
        if (e < g.E) {
          if constexpr (sizeof(LT) == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(row + e * 2);
            v[4 * q] = bf_lo(x.x), v[4 * q + 1] = bf_hi(x.x), v[4 * q + 2] = bf_lo(x.y), v[4 * q + 3] = bf_hi(x.y);
          } else {
            const f32x4 x = *reinterpret_cast<const f32x4*>(row + e * 4);
#pragma unroll
            for (int c = 0; c < 4; ++c) v[4 * q + c] = x[c];
          }
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) v[4 * q + c] = -INFINITY;
        }
      } else {
#pragma unroll
        for (int c = 0; c < 4; ++c) v[4 * q + c] = e + c < g.E ? load_logit<LT>(row, e + c) : -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < 4 * NQ; ++i) m = fmaxf(m, v[i]);
    m = lanes_max<LPT>(m);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * NQ; ++i) {
      v[i] = v[i] == -INFINITY ? 0.f : expf(v[i] - m);
      s += v[i];
    }
    s = lanes_sum<LPT>(s);
    inv = s == 0.f ? 0.f : 1.f / s;        // a row that is masked whole has no gradient
  }
  float s_j = 0.f;
  if (l_j != -INFINITY) s_j = softmax ? expf(l_j - m) * inv : 1.f / (1.f + expf(-l_j));
  float ds = gj;
  if (g.renorm) {
    const float S = lanes_sum<LPT>(s_j);
    const float dot = lanes_sum<LPT>(gj * s_j);
    ds = S == 0.f ? 0.f : (gj - dot / S) / S;
  }
  // softmax: the part that every expert of the row gets; the renormalized weights' is zero
  const float shared = softmax && !g.renorm ? lanes_sum<LPT>(ds * s_j) : 0.f;
  const float add = softmax ? ds : ds * s_j * (1.f - s_j);
  float d[4 * NQ];
#pragma unroll
  for (int i = 0; i < 4 * NQ; ++i) d[i] = 0.f;
  for (int j = 0; j < g.k; ++j) {
    const int e = __shfl(e_j, j, LPT);
    const float a = __shfl(add, j, LPT);
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) d[4 * q + c] += e == 4 * LPT * q + 4 * sub + c ? a : 0.f;
  }
  if (softmax) {
#pragma unroll
    for (int i = 0; i < 4 * NQ; ++i) d[i] = v[i] * inv * (d[i] - shared);
  }
  if (!live) return;
  char* const out = static_cast<char*>(g.d_logits) + t * g.ld_d * static_cast<int64_t>(sizeof(LT));
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int e = 4 * LPT * q + 4 * sub;
    if constexpr (VEC) {
      if (e < g.E) {
        if constexpr (sizeof(LT) == 2)
          *reinterpret_cast<uint2*>(out + e * 2) =
              make_uint2(pack_bf16x2(d[4 * q], d[4 * q + 1]), pack_bf16x2(d[4 * q + 2], d[4 * q + 3]));
        else
          *reinterpret_cast<f32x4*>(out + e * 4) = f32x4{d[4 * q], d[4 * q + 1], d[4 * q + 2], d[4 * q + 3]};
      }
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (e + c < g.E) {
          if constexpr (sizeof(LT) == 2) reinterpret_cast<uint16_t*>(out)[e + c] = static_cast<uint16_t>(f2bf(d[4 * q + c]));
          else reinterpret_cast<float*>(out)[e + c] = d[4 * q + c];
        }
    }
  }
}

}  // namespace xs

using namespace xs;

namespace {

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int gate_ok(const xs_gate* g, const void* logits, int64_t ld, int32_t T) {
  if (!g || !logits || T < 0 || g->reserved != 0) return XS_EINVAL;
  if (g->E < 1 || g->E > 1024 || g->k < 1 || g->k > g->E || g->k > 32 || ld < g->E) return XS_EINVAL;
  if (g->score != XS_SCORE_SOFTMAX && g->score != XS_SCORE_SIGMOID) return XS_EINVAL;
  if (g->logits_type != XS_TYPE_BF16 && g->logits_type != XS_TYPE_F32) return XS_EINVAL;
  if (g->group_score != XS_GROUP_MAX && g->group_score != XS_GROUP_TOP2) return XS_EINVAL;
  if (g->n_group < 1 || g->n_group > 64 || g->E % g->n_group || g->topk_group < 1 || g->topk_group > g->n_group)
    return XS_EINVAL;
  if (g->k > g->topk_group * (g->E / g->n_group)) return XS_EINVAL;
  if (!std::isfinite(g->scale)) return XS_EINVAL;
  const int64_t size = g->logits_type == XS_TYPE_BF16 ? 2 : 4;
  if (ld > (int64_t(1) << 40) || !aligned_to(logits, size) || !aligned_to(g->bias, 4)) return XS_EINVAL;
  return XS_OK;
}

template <typename LT, int LPT, int NQ>
void launch_grad(const GateGradArgs& a, bool vec, hipStream_t st) {
  const int per = 256 / LPT;
  const dim3 grid = xs_host::grid_of((static_cast<int64_t>(a.T) + per - 1) / per);
  if (vec) hipLaunchKernelGGL((gate_grad_kernel<LT, LPT, NQ, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((gate_grad_kernel<LT, LPT, NQ, false>), grid, dim3(256), 0, st, a);
}

template <typename LT>
void launch_grad(const GateGradArgs& a, hipStream_t st) {
  const uintptr_t piece = 4 * sizeof(LT);
  const bool vec = a.E % 4 == 0 && a.ld % 4 == 0 && a.ld_d % 4 == 0 && aligned_to(a.logits, piece) && aligned_to(a.d_logits, piece);
  if (a.E <= 256 && a.k <= 16) {
    if (a.E <= 64) launch_grad<LT, 16, 1>(a, vec, st);
    else if (a.E <= 128) launch_grad<LT, 16, 2>(a, vec, st);
    else launch_grad<LT, 16, 4>(a, vec, st);
  } else if (a.E <= 512) {
    launch_grad<LT, 64, 2>(a, vec, st);
  } else {
    launch_grad<LT, 64, 4>(a, vec, st);
  }
}

}  // namespace

extern "C" int xs_route_gate(const xs_gate* g, const void* logits, int64_t ld, int32_t T, int32_t* topk_idx,
                             float* topk_w, void* stream) {
  int rc = gate_ok(g, logits, ld, T);
  if (rc) return rc;
  if (!topk_idx || !topk_w) return XS_EINVAL;
  if (T == 0) return XS_OK;
  const GateArgs a{logits, ld, g->bias, T, g->E, g->k, g->score, g->n_group, g->topk_group,
                   g->group_score == XS_GROUP_TOP2, g->renormalize != 0, g->scale, topk_idx, topk_w};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid = xs_host::grid_of((static_cast<int64_t>(T) + 3) / 4);
  const size_t lds = 4 * sizeof(double) * g->E;
  if (g->logits_type == XS_TYPE_BF16) hipLaunchKernelGGL((gate_wave_kernel<uint16_t>), grid, dim3(256), lds, st, a);
  else hipLaunchKernelGGL((gate_wave_kernel<float>), grid, dim3(256), lds, st, a);
  return xs_host::launch_status();
}

extern "C" int xs_route_gate_backward(const xs_gate* g, const void* logits, int64_t ld, int32_t T, const int32_t* topk_idx,
                                      const float* d_topk_w, void* d_logits, int64_t ld_d, int32_t* dev_status,
                                      void* stream) {
  int rc = gate_ok(g, logits, ld, T);
  if (rc) return rc;
  if (!topk_idx || !d_topk_w || !d_logits || ld_d < g->E || ld_d > (int64_t(1) << 40)) return XS_EINVAL;
  if (!aligned_to(d_logits, g->logits_type == XS_TYPE_BF16 ? 2 : 4)) return XS_EINVAL;
  if (T == 0) return XS_OK;
  const GateGradArgs a{logits, ld, T, g->E, g->k, g->score, g->renormalize != 0, g->scale, topk_idx, d_topk_w,
                       d_logits, ld_d, dev_status};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (g->logits_type == XS_TYPE_BF16) launch_grad<uint16_t>(a, st);
  else launch_grad<float>(a, st);
  return xs_host::launch_status();
}
