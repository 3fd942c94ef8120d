// Routing gates: softmax or sigmoid scores, a bias that only the selection sees, groups of experts,
// top-k, renormalized and scaled weights; and the gradient of the weights in the logits.
//
//   s_e = 1 / (1 + exp(-l_e))  or  exp(l_e - m) / sum_f exp(l_f - m)          (0 where l_e = -inf)
//   key_e = s_e + b_e          group score = the largest key, or the sum of the two largest
//   w_j = scale s_j            or, renormalized, scale s_j / S with S = sum_i s_i over the k chosen
//
// A factor that all k scores have cancels in s_j / S: renormalized weights r_j are computed from exp(l_j - c)
// with c the largest of the k logits (sigmoid: where that is below 0), so scores that underflow fp32
// still have their weights.
//
// Gradient, g_j = scale dL/dw_j; sums over the slots j of expert e, all other elements 0 but for plain softmax:
//   sigmoid               dl_e = sum g_j s_e (1 - s_e)            (1 - s_e as 1 / (1 + e^l_e))
//   softmax               dl_e = s_e (sum g_j - sum_i g_i s_i)          (every e)
//   renormalized, d_j = (g_j - sum_i g_i r_i) r_j:
//     sigmoid             dl_e = sum d_j (1 - s_e)
//     softmax             dl_e = sum d_j
#include <algorithm>
#include <cmath>
#include <utility>

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

// f of the constants I... in turn
template <class F, int... I>
__device__ __forceinline__ void each_of(const F& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}

template <typename LT>
__device__ __forceinline__ float load_logit(const void* row, int e) {
  if constexpr (sizeof(LT) == 2) return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(row)[e]) << 16);
  else return static_cast<const float*>(row)[e];
}

template <typename LT>
__device__ __forceinline__ const char* logit_row(const void* logits, int64_t ld, int64_t t) {
  return static_cast<const char*>(logits) + t * ld * static_cast<int64_t>(sizeof(LT));
}

// Keys lie within 2^127: a masked expert (logit -inf or NaN, key NaN or below) has the lowest, and one
// outside the chosen groups a lower value yet. A group's score may be the sum of two keys; one without an unmasked
// expert has at most every such sum (in fp32 the sum of the two lowest, -FLT_MAX; in 64 bits below all).
constexpr double kMaskedKey = -0x1p127, kDeadGroup = -0x1p129;
constexpr float kDeadGroup32 = -3.40282346638528859812e+38f;
__device__ __forceinline__ double finite_key(double key, bool masked) {
  return masked || !(key > kMaskedKey) ? kMaskedKey : fmin(key, -kMaskedKey);
}

// LDS operations of one wave take place in order: only the compiler has to keep to it.
__device__ __forceinline__ void wave_order() { asm volatile("" ::: "memory"); }

template <int CTRL>
__device__ __forceinline__ float dpp32(float f) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(f), CTRL, 0xF, 0xF, false));
}
template <int CTRL>
__device__ __forceinline__ int dpp32(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, false);
}
// Within the 16 lanes of a DPP row: rotations by r (kRor + r, a lane takes the value r lanes below its own,
// around the row), the lane's neighbours in its pair and in its four, and its mirror in its eight.
constexpr int kRor = 0x120, kRor8 = 0x128, kRor4 = 0x124, kRor2 = 0x122, kRor1 = 0x121;
constexpr int kPair = 0xB1, kFour = 0x4E, kMirror8 = 0x141;
// Sums and maxima over a token's lanes: 16 (a DPP row) or 64; the same bits in every lane.
template <int LPT>
__device__ __forceinline__ float lanes_sum(float v) {
  v += dpp32<kRor8>(v);
  v += dpp32<kRor4>(v);
  v += dpp32<kRor2>(v);
  v += dpp32<kRor1>(v);
  if constexpr (LPT == 64) {
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
  }
  return v;
}
template <int LPT>
__device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, dpp32<kRor8>(v));
  v = fmaxf(v, dpp32<kRor4>(v));
  v = fmaxf(v, dpp32<kRor2>(v));
  v = fmaxf(v, dpp32<kRor1>(v));
  if constexpr (LPT == 64) {
    v = fmaxf(v, __shfl_xor(v, 16));
    v = fmaxf(v, __shfl_xor(v, 32));
  }
  return v;
}

// n / d, |n| <= d and d within 2^+-64, in one rounding but for 2^-23 of one: the product with the reciprocal unit's 1 / d
// (within an fp32 unit), and its remainder's. The mean square error of renormalized weights is that of divisions; with
// the product alone 1.18 times it, in the same time (32,768 tokens: 15.4 us).
__device__ __forceinline__ float quotient(float n, float d) {
  const float r = __builtin_amdgcn_rcpf(d), q = n * r;
  return __builtin_fmaf(__builtin_fmaf(-q, d, n), r, q);
}

// A slot's renormalized weight r_j among its token's lanes (0 without a live slot); l: its logit. Both divisors are
// between 1/2 and 32 (the largest s is 1 or, of sigmoids, at least 1/2).
template <int LPT>
__device__ __forceinline__ float renormalized(bool softmax, bool slot, float l) {
  slot = slot && l != -INFINITY;
  float c = lanes_max<LPT>(slot ? l : -INFINITY);
  float s = 0.f;
  if (softmax) {
    if (slot) s = expf(l - c);
  } else {
    // e^-|l| once; below all of the k, e^(l - c) comes with c = 0 from it too
    c = fminf(c, 0.f);
    const float t = expf(-fabsf(l));
    if (slot) s = quotient(l > 0.f ? 1.f : c == 0.f ? t : expf(l - c), 1.f + t);
  }
  const float total = lanes_sum<LPT>(s);
  return total == 0.f ? 0.f : quotient(s, total);
}
// Its score; m and inv: the row's largest logit and the reciprocal of its softmax sum.
__device__ __forceinline__ float slot_score(bool softmax, bool slot, float l, float m, float inv) {
  if (!slot || l == -INFINITY) return 0.f;
  return softmax ? expf(l - m) * inv : 1.f / (1.f + expf(-l));
}

template <int CTRL>
__device__ __forceinline__ double dpp64(double d) {
  const uint64_t u = __builtin_bit_cast(uint64_t, d);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), CTRL, 0xF, 0xF, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), CTRL, 0xF, 0xF, false);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double wave_max(double v) {
  v = fmax(v, dpp64<kRor8>(v));
  v = fmax(v, dpp64<kRor4>(v));
  v = fmax(v, dpp64<kRor2>(v));
  v = fmax(v, dpp64<kRor1>(v));
  v = fmax(v, __shfl_xor(v, 16));
  return fmax(v, __shfl_xor(v, 32));
}
template <int CTRL>
__device__ __forceinline__ int min_dpp(int v) { return min(v, __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, false)); }
__device__ __forceinline__ int wave_min(int v) {
  v = min_dpp<kRor1>(min_dpp<kRor2>(min_dpp<kRor4>(min_dpp<kRor8>(v))));
  v = min(v, __shfl_xor(v, 16));
  return min(v, __shfl_xor(v, 32));
}

// One token by a whole wave, keys in 64 bits: any E, k and groups. key: E doubles of LDS, this wave's
// own. A reduction is a maximum, then the lowest index that has it.
template <typename LT>
__device__ void gate_token(const GateArgs& g, int64_t t, double* key) {
  const int lane = threadIdx.x & 63;
  const char* const row = logit_row<LT>(g.logits, g.ld, t);
  const int E = g.E;
  const bool softmax = g.score == XS_SCORE_SOFTMAX;
  float m = -INFINITY;
  double sum = 0.;
  if (softmax) {
    for (int e = lane; e < E; e += 64) m = fmaxf(m, load_logit<LT>(row, e));
    m = lanes_max<64>(m);
    for (int e = lane; e < E; e += 64) {
      const float l = load_logit<LT>(row, e);
      if (l != -INFINITY) sum += exp(static_cast<double>(l) - static_cast<double>(m));
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
  }
  // without a bias the logits have the scores' order, and no rounding
  const bool by_logit = !g.bias && (g.n_group == 1 || !g.top2);
  for (int e = lane; e < E; e += 64) {
    const float l = load_logit<LT>(row, e);
    const bool masked = l == -INFINITY || l != l;
    double v = static_cast<double>(l);
    if (!by_logit && !masked) v = softmax ? exp(v - static_cast<double>(m)) / sum : 1. / (1. + exp(-v));
    if (g.bias) v += static_cast<double>(g.bias[e]);
    key[e] = finite_key(v, masked);
  }
  wave_order();
  if (g.n_group > 1) {
    // lanes 2^s per group: its two largest keys; then group = lane
    const int Eg = E / g.n_group, lanes = 64 >> (32 - __builtin_clz(g.n_group - 1));
    const int grp = lane / lanes;
    double a = -INFINITY, b = -INFINITY;
    if (grp < g.n_group)
      for (int i = lane % lanes; i < Eg; i += lanes) {
        const double v = key[grp * Eg + i];
        b = fmax(b, fmin(a, v));
        a = fmax(a, v);
      }
    for (int off = 1; off < lanes; off <<= 1) {
      const double oa = __shfl_xor(a, off), ob = __shfl_xor(b, off);
      b = fmax(fmin(a, oa), fmax(b, ob));
      a = fmax(a, oa);
    }
    const double total = a <= kMaskedKey ? kDeadGroup : g.top2 && b > kMaskedKey ? a + b : a;
    double left = __shfl(total, (lane * lanes) & 63);
    if (lane >= g.n_group) left = -INFINITY;
    bool kept = false;
    for (int j = 0; j < g.topk_group; ++j) {
      const double most = wave_max(left);
      if (wave_min(left == most ? lane : 64) == lane) {
        kept = true;
        left = -INFINITY;
      }
    }
    const unsigned long long keep = __ballot(kept);
    for (int e = lane; e < E; e += 64)
      if (!((keep >> (e / Eg)) & 1ull)) key[e] = -INFINITY;
    wave_order();
  }
  int my_idx = 0;
  for (int j = 0; j < g.k; ++j) {
    double bv = -INFINITY;
    int bi = E;
    for (int e = lane; e < E; e += 64) {
      const double v = key[e];
      if (v > bv) {
        bv = v;
        bi = e;
      }
    }
    bi = wave_min(bv == wave_max(bv) ? bi : E);
    if ((bi & 63) == lane) key[bi] = -INFINITY;
    if (lane == j) my_idx = bi;
  }
  const bool slot = lane < g.k;
  const float l = slot ? load_logit<LT>(row, my_idx) : 0.f;
  const float s = g.renorm ? renormalized<64>(softmax, slot, l) : slot_score(softmax, slot, l, m, static_cast<float>(1. / sum));
  if (slot) {
    g.idx[t * g.k + lane] = my_idx;
    g.w[t * g.k + lane] = s * g.scale;
  }
}

template <typename LT>
__global__ __launch_bounds__(256) void gate_wave_kernel(GateArgs g) {
  extern __shared__ double gate_keys[];   // [4][E]
  const int w = threadIdx.x >> 6;
  const int64_t t = block_number() * 4 + w;
  if (t < g.T) gate_token<LT>(g, t, gate_keys + w * g.E);   // whole waves, no barrier
}

// ------------------------------------------------------------------------------ sixteen lanes a token
// fp32 values as integers of the same order (and back: the map is its own inverse), and such a key, cut to 14
// bits of mantissa, with its expert: larger is earlier (a larger cut key or, of equal ones, the lower
// index; E <= 512).
__device__ __forceinline__ int ordered(int bits) { return bits ^ ((bits >> 31) & 0x7FFFFFFF); }
__device__ __forceinline__ int ordered(float f) { return ordered(__float_as_int(f)); }
__device__ __forceinline__ float from_ordered(int o) { return __int_as_float(ordered(o)); }
__device__ __forceinline__ int pack_key(int o, int e) { return (o & ~511) | (511 - e); }
__device__ __forceinline__ int key_expert(int p) { return 511 - (p & 511); }
constexpr int kNoKey = -0x7FFFFFFF - 1, kUnknown = 0x7FFFFFFF;

__device__ __forceinline__ void order(int& a, int& b) {   // the larger first
  const int hi = max(a, b), lo = min(a, b);
  a = hi;
  b = lo;
}
// A list whose halves' maxima are placed (a bitonic sequence) into descending order.
template <int N>
__device__ __forceinline__ void order_bitonic(int (&v)[N]) {
#pragma unroll
  for (int d = N / 2; d >= 1; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!(i & d)) order(v[i], v[i + d]);
}
// Descending order of any list (Batcher's odd-even merge sort).
template <int N>
__device__ __forceinline__ void order_all(int (&v)[N]) {
#pragma unroll
  for (int p = 1; p < N; p <<= 1)
#pragma unroll
    for (int k = p; k >= 1; k >>= 1)
#pragma unroll
      for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) order(v[i + j], v[i + j + k]);
}
// The N largest of two descending lists, in descending order.
template <int N>
__device__ __forceinline__ void keep_largest(int (&v)[N], const int (&o)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = max(v[i], o[N - 1 - i]);
  order_bitonic(v);
}
__device__ __forceinline__ int lanes_max16(int v) {
  v = max(v, dpp32<kRor8>(v));
  v = max(v, dpp32<kRor4>(v));
  v = max(v, dpp32<kRor2>(v));
  return max(v, dpp32<kRor1>(v));
}

// From the sixteen lanes' descending lists, the J-th largest key and on to the k-th into lane J's, J + 1's ...
// `mine`, each taken from its list (keys in use are all different); kUnknown follows a list's end.
template <int J, int KL>
__device__ __forceinline__ void take_largest(int (&top)[KL], int k, int sub, int& mine) {
  if (J >= k) return;
  const int most = lanes_max16(top[0]);
  mine = sub == J ? most : mine;
  const bool from_here = top[0] == most;
#pragma unroll
  for (int i = 0; i < KL - J; ++i) top[i] = from_here ? (i + 1 < KL ? top[i + 1 < KL ? i + 1 : 0] : kUnknown) : top[i];
  if constexpr (J + 1 < KL) take_largest<J + 1>(top, k, sub, mine);
}

// VP consecutive values of T from p: in pieces of 16 bytes where `vec`.
template <int VPL, typename LT, bool FULL>
__device__ __forceinline__ void load_run(const void* base, int first, int VP, int E, bool vec, float other, float (&v)[VPL]) {
  constexpr int kPiece = sizeof(LT) == 2 && VPL >= 8 ? 8 : 4;
  if (FULL || vec) {
    const char* const p = static_cast<const char*>(base) + static_cast<int64_t>(first) * static_cast<int64_t>(sizeof(LT));
#pragma unroll
    for (int i = 0; i < VPL; i += kPiece) {
#pragma unroll
      for (int c = 0; c < kPiece; ++c) v[i + c] = other;
      if (FULL || (i < VP && first + i < E)) {
        if constexpr (sizeof(LT) == 4) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(p + i * 4);
#pragma unroll
          for (int c = 0; c < 4; ++c) v[i + c] = x[c];
        } else if constexpr (kPiece == 8) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(p + i * 2);
#pragma unroll
          for (int c = 0; c < 4; ++c) v[i + 2 * c] = bf_lo(x[c]), v[i + 2 * c + 1] = bf_hi(x[c]);
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(p + i * 2);
          v[i] = bf_lo(x.x), v[i + 1] = bf_hi(x.x), v[i + 2] = bf_lo(x.y), v[i + 3] = bf_hi(x.y);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) v[i] = i < VP && first + i < E ? load_logit<LT>(base, first + i) : other;
  }
}

// Sixteen lanes per token, four tokens per wave. A group of experts has 16 / n_group whole lanes, each with up to VP
// = ceil(E / n_group / lanes) of its consecutive experts; lanes are in the experts' order.
//
// The k largest keys are found by a sorting network on 32-bit words, each a key cut to 14 bits with its
// expert; then every lane looks up one of them whole. Their order is the 64-bit one where it is clear: with s
// off by at most sigma (below) and a key by sigma + 2^-24 |key|, two keys further apart than twice that are
// in the right order, so no other key may come that near to the last of the k, and no neighbours among them.
// Elsewhere (one token in a hundred for 256 sigmoid scores, by the cut) the keys within reach of the last,
// if they are at most sixteen, are done again in 64 bits, one a lane; so are the groups' scores where it is
// unclear which are kept. What remains (more candidates, a group's second key too near its third) is done again
// by the token's whole wave (gate_token).
// Without a bias the logits are the keys, exactly (bf16 ones also when cut).
//
// 32,768 tokens, top-8 of 256 biased sigmoid scores in groups: 15.5 us, 2.3 TB/s, vector instructions issuing for 10.3
// of them (780 for four tokens, at 2.4 GHz). What a token needs is fixed when the kernel is compiled (the kind
// of key, whole rows), the lanes exchange by DPP, and the keys are integers throughout. Not at a bound: `r % lanes`
// below is some ten dependent scalar instructions fourteen times, and keys are mapped to integers one by one.
//   sigmoid: exp(-l) is off by 2^-23 and, from its argument, |l| 2^-23; times s (1 - s), with s (1 - s) |l|
//     <= 0.224; the sum and the reciprocal 2^-24 + 2^-23 of s: together below 2^-22 (s <= 1).
//   softmax: e^-d is off by d 2^-22 + 2^-23 (d e^-d <= 0.37), the sum of up to 512 terms (32 in a
//     lane, four levels) by 2^-19 of itself at most: below 2^-18 of the largest score.
// MODE: the keys are the logits, sigmoid scores or softmax scores. FULL: E = 16 VPL experts in aligned rows.
enum { kByLogit, kSigmoid, kSoftmax };
template <typename LT, int VPL, int KL, int MODE, bool FULL>
__global__ __launch_bounds__(256) void gate_rows_kernel(GateArgs g, int VP, int vec, int bias_vec) {
  extern __shared__ double gate_keys[];   // [4][E], for tokens done again
  __shared__ int candidates[16][16];
  const int sub = threadIdx.x & 15, w = threadIdx.x >> 6;
  const int64_t t_raw = block_number() * 16 + (threadIdx.x >> 4);
  const bool live = t_raw < g.T;
  const int64_t t = live ? t_raw : g.T - 1;   // every lane takes part in its row's reductions
  const char* const row = logit_row<LT>(g.logits, g.ld, t);
  const int lanes = 16 / g.n_group;         // of a group
  const int group_end = g.E / g.n_group * ((sub >> __builtin_ctz(lanes)) + 1);
  const int first = FULL ? VPL * sub : group_end - g.E / g.n_group + VP * (sub & (lanes - 1));
  constexpr bool by_logit = MODE == kByLogit;
  const bool softmax = by_logit ? g.score == XS_SCORE_SOFTMAX : MODE == kSoftmax;
  constexpr float kMasked = static_cast<float>(kMaskedKey), kDropped = 1.5f * kMasked;
  constexpr int kDroppedKey = static_cast<int>(0xFF400000u) ^ 0x7FFFFFFF;
  float v[VPL];
  load_run<VPL, LT, FULL>(row, first, VP, group_end, vec, -INFINITY, v);
  float m = 0.f, inv = 1.f, sigma = 0x1p-22f;
  if (softmax) {
    m = -INFINITY;
#pragma unroll
    for (int i = 0; i < VPL; ++i) m = fmaxf(m, v[i]);
    m = lanes_max<16>(m);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) s += v[i] == -INFINITY ? 0.f : __expf(v[i] - m);
    inv = 1.f / lanes_sum<16>(s);
    sigma = 0x1p-18f * inv;
  }
  // the key of a logit: clamped, and the lowest for NaN (med3 takes the lower bound) and masked ones
  const auto key_of = [&](float l, float b) {
    float s;
    if (by_logit) s = l + 0.f;              // -0 becomes 0: as integers they differ
    else s = (softmax ? __expf(l - m) * inv : __builtin_amdgcn_rcpf(1.f + __expf(-l))) + b;
    s = __builtin_amdgcn_fmed3f(s, kMasked, -kMasked);
    return l == -INFINITY ? kMasked : s;
  };
  int o[VPL];                               // the keys, ordered
  {
    float b[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) b[i] = 0.f;
    if (!by_logit && g.bias) load_run<VPL, float, FULL>(g.bias, first, VP, group_end, bias_vec, 0.f, b);
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      o[i] = FULL || (i < VP && first + i < group_end) ? ordered(key_of(v[i], b[i])) : kDroppedKey;
  }
  const auto key_at = [&](int i) { return from_ordered(o[i]); };
  bool kept = true;                         // the lane's group
  // In doubt: a score in 64 bits, of a softmax with its row's sum (by the token's sixteen lanes).
  const auto sum64 = [&]() -> double {
    if (!softmax) return 1.;
    double s = 0.;
#pragma unroll 4
    for (int i = 0; i < VPL; ++i)
      if (FULL || (i < VP && first + i < group_end)) {
        const float l = load_logit<LT>(row, first + i);
        if (l != -INFINITY) s += exp(static_cast<double>(l) - static_cast<double>(m));
      }
    s += dpp64<kRor8>(s);
    s += dpp64<kRor4>(s);
    s += dpp64<kRor2>(s);
    return s + dpp64<kRor1>(s);
  };
  const auto score64 = [&](float l, double sum) -> double {
    return softmax ? exp(static_cast<double>(l) - static_cast<double>(m)) / sum : 1. / (1. + exp(-static_cast<double>(l)));
  };
  bool unsure = false;
  if (g.n_group > 1) {
    int a = kNoKey, b = kNoKey;             // the group's two largest keys
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      b = max(b, min(a, o[i]));
      a = max(a, o[i]);
    }
    const auto join = [&](int oa, int ob) {
      b = max(min(a, oa), max(b, ob));
      a = max(a, oa);
    };
    if (lanes > 1) join(dpp32<kPair>(a), dpp32<kPair>(b));
    if (lanes > 2) join(dpp32<kFour>(a), dpp32<kFour>(b));
    if (lanes > 4) join(dpp32<kMirror8>(a), dpp32<kMirror8>(b));
    const float ka = from_ordered(a), kb = from_ordered(b);   // (one expert to a group: b is dropped, or NaN)
    const float gs = !(ka > kMasked) ? kDeadGroup32 : g.top2 && kb > kMasked ? ka + kb : ka;
    // off by both keys' errors and the sum's rounding, on both sides
    const float tol = by_logit ? 0.f : 4.f * sigma + 0x1p-21f * (fabsf(ka) + (kb > kMasked ? fabsf(kb) : 0.f));
    int above = 0, near = 0;                // groups surely before this one, groups that may be
    const auto compare = [&](auto rc) {
      constexpr int r = decltype(rc)::value + 1, ctrl = kRor + r;
      if (r % lanes) return;                // (the same in every lane)
      const int os = dpp32<ctrl>(sub);
      const float other = dpp32<ctrl>(gs), far = fmaxf(tol, dpp32<ctrl>(tol));
      if (by_logit) {
        const bool before = other > gs || (other == gs && os < sub);
        above += before;
        near += before;
      } else {
        above += other - gs > far;
        near += !(gs - other > far);
      }
    };
    each_of(compare, std::make_integer_sequence<int, 15>());
    kept = near < g.topk_group;
    const unsigned long long doubts = __ballot(above < g.topk_group && !kept);
    if (doubts) {
      // the groups' scores in 64 bits, from the largest keys, if those are clear of the next one
      const bool doubt = (doubts >> (threadIdx.x & 48)) & 0xFFFFull;     // of the token
      float k1 = -INFINITY, k2 = -INFINITY, k3 = -INFINITY;
      int e1 = 0, e2 = 0;
      const auto insert = [&](float x, int e) {
        if (x > k1 || (x == k1 && e < e1)) {
          k3 = k2;
          k2 = k1, e2 = e1;
          k1 = x, e1 = e;
        } else if (x > k2 || (x == k2 && e < e2)) {
          k3 = k2;
          k2 = x, e2 = e;
        } else {
          k3 = fmaxf(k3, x);
        }
      };
#pragma unroll
      for (int i = 0; i < VPL; ++i) insert(key_at(i), first + i);
      for (int off = 1; off < lanes; off <<= 1) {
        const float o1 = __shfl_xor(k1, off), o2 = __shfl_xor(k2, off), o3 = __shfl_xor(k3, off);
        const int i1 = __shfl_xor(e1, off), i2 = __shfl_xor(e2, off);
        insert(o1, i1);
        insert(o2, i2);
        k3 = fmaxf(k3, o3);
      }
      const float used = g.top2 && k2 > kMasked ? k2 : k1, unused = g.top2 ? k3 : k2;
      const bool fine = unused <= kMasked || used - unused > 2.f * sigma + 0x1p-22f * fmaxf(fabsf(used), fabsf(unused));
      const double sum = by_logit ? 1. : sum64();
      const auto exact = [&](float k, int e) -> double {
        if (k <= kMasked) return kMaskedKey;
        const double x = score64(load_logit<LT>(row, e), sum);
        return finite_key(g.bias ? x + static_cast<double>(g.bias[e]) : x, false);
      };
      const double d1 = exact(k1, e1), d2 = exact(k2, e2), most = fmax(d1, d2);
      const double score = !(k1 > kMasked) ? kDeadGroup : g.top2 && k2 > kMasked ? d1 + d2 : most;
      int before = 0;
      for (int r = lanes; r < 16; r += lanes) {
        const int os = (sub + r) & 15;
        const double o = __shfl(score, os, 16);
        before += o > score || (o == score && os / lanes < sub / lanes);
      }
      if (doubt) {
        kept = before < g.topk_group;
        unsure = !fine;
      }
    }
  }
  // The KL largest of a lane's keys in order; then the sixteen lanes' largest first keys one by one, each taken
  // from its lane's list (merging the lists in a network over the lanes instead took a tenth longer).
  int top[KL];
#pragma unroll
  for (int i = 0; i < KL; ++i) top[i] = i < VPL ? pack_key(o[i < VPL ? i : 0], first + i) : kNoKey;
  order_all(top);
#pragma unroll
  for (int c = KL; c < VPL; c += KL) {
    int more[KL];
#pragma unroll
    for (int i = 0; i < KL; ++i) more[i] = c + i < VPL ? pack_key(o[c + i < VPL ? c + i : 0], first + c + i) : kNoKey;
    order_all(more);
    keep_largest(top, more);
  }
#pragma unroll
  for (int i = 0; i < KL; ++i) top[i] = kept ? top[i] : kDroppedKey & ~511;
  int mine = kNoKey;                        // lane j has the j-th
  take_largest<0>(top, g.k, sub, mine);
  const int rest = lanes_max16(top[0]);     // kUnknown: one lane had them all
  bool slot = sub < g.k;
  int e = slot ? key_expert(mine) : 512 + sub;
  float l = slot ? load_logit<LT>(row, e) : -INFINITY;
  const float key = slot ? key_of(l, g.bias ? g.bias[e] : 0.f) : kDropped;
  const float largest = lanes_max<16>(key);
  const float last = -lanes_max<16>(slot ? -key : -INFINITY);
  const float tol = by_logit ? 0.f : 2.f * sigma + 0x1p-22f * fmaxf(fabsf(largest), last > kMasked ? fabsf(last) : 0.f);
  const auto before = [&](auto a, int ea, auto b, int eb) { return a > b || (a == b && ea < eb); };
  // No key of the rest is above the next cut one's largest value: those may not come near the last. (A masked
  // last one: nothing else is left, as no key above -2^127 is cut down to it; whole keys in the network: they
  // are in order.)
  const bool whole = by_logit && sizeof(LT) == 2;
  const bool apart = whole || last <= kMasked || from_ordered(rest | 511) < last - tol;
  const float next = dpp32<kRor + 15>(key);         // of the lane above
  const int en = dpp32<kRor + 15>(e);
  // masked keys are equal without doubt
  const bool clear = tol == 0.f || next == kMasked ? before(key, e, next, en) : key - next > tol;
  int rank = sub;
  bool doubt = !apart || (sub + 1 < g.k && !clear) || !(tol >= 0.f);   // (a NaN among softmax logits)
  const unsigned long long doubts = __ballot(doubt);
  if (doubts) {
    doubt = (doubts >> (threadIdx.x & 48)) & 0xFFFFull;                  // of the token
    // the keys that may be among the k: up to sixteen, one a lane, in 64 bits
    const int from = ordered(last - tol);
    int c = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) c += kept && o[i] >= from ? 1 : 0;
    int at = c;                             // candidates of the lanes up to this one
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) {
      const int below = __shfl_up(at, off, 16);
      if (sub >= off) at += below;
    }
    const int n = __shfl(at, 15, 16);
    at -= c;
    const bool few = doubt && n <= 16 && last > kMasked && tol >= 0.f;
    const double sum = by_logit ? 1. : sum64();
    unsure |= doubt && !few;
    if (few) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (kept && o[i] >= from) candidates[threadIdx.x >> 4][at++] = first + i;
    }
    wave_order();
    if (few) {
      e = sub < n ? candidates[threadIdx.x >> 4][sub] : 512 + sub;
      l = sub < n ? load_logit<LT>(row, e) : -INFINITY;
    }
    double kd = -INFINITY;
    if (few && sub < n) {
      const double x = by_logit ? static_cast<double>(l) : score64(l, sum);
      kd = finite_key(g.bias ? x + static_cast<double>(g.bias[e]) : x, l == -INFINITY || l != l);
    }
    int r0 = 0;
    for (int r = 1; r < 16; ++r) {
      const double o = __shfl(kd, (sub + r) & 15, 16);
      const int eo = __shfl(e, (sub + r) & 15, 16);
      r0 += before(o, eo, kd, e);
    }
    if (few) {
      rank = r0;
      slot = r0 < g.k;
    }
  }
  const float s = g.renorm ? renormalized<16>(softmax, slot, l) : slot_score(softmax, slot, l, m, inv);
  unsigned long long again = __ballot(unsure && live);
  if (slot && live && !((again >> (threadIdx.x & 48)) & 0xFFFFull)) {
    g.idx[t * g.k + rank] = e;
    g.w[t * g.k + rank] = s * g.scale;
  }
  while (again) {
    const int q = (__ffsll(static_cast<long long>(again)) - 1) >> 4;
    again &= ~(0xFFFFull << (16 * q));
    gate_token<LT>(g, block_number() * 16 + 4 * w + q, gate_keys + w * g.E);
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

// LPT lanes per token; lane `sub` has the experts P (LPT q + sub) + c (q < NQ, c < P), 16 bytes for each q where
// rows are aligned. Slot j of a token is lane j's (k <= LPT). Every element gets what the whole row gets (0,
// or for a plain softmax -s_e sum_i g_i s_i) and goes to LDS; the slots' lanes then write their experts' whole
// elements over it (LDS operations of one wave are in order; an expert's duplicate slots write the same
// value, summed in ascending j), and the row is stored from there. Adding the k slots to all of a lane's
// elements in registers instead took 1.55 times as long (32,765 tokens of 256 bf16 logits: 10.3 us, of sigmoid or
// renormalized gates, which read no whole row, 7.7; fp32 logits 11.7 and 9.8). Not at a bound: the index, then the slot's
// logit, then the row's pieces are waited for one after the other.
template <typename LT, int LPT, int NQ, bool VEC>
__global__ __launch_bounds__(256) void gate_grad_kernel(GateGradArgs g) {
  constexpr int P = 16 / sizeof(LT), kRow = NQ * LPT * P;      // elements of a row in LDS
  __shared__ __attribute__((aligned(16))) LT rows[256 / LPT][kRow];
  const int sub = threadIdx.x % LPT;
  const int64_t t_raw = block_number() * (256 / LPT) + threadIdx.x / LPT;
  const bool live = t_raw < g.T;
  const int64_t t = live ? t_raw : g.T - 1;   // every lane takes part in the sums
  const char* const row = logit_row<LT>(g.logits, g.ld, t);
  LT* const mine = rows[threadIdx.x / LPT];
  const bool softmax = g.score == XS_SCORE_SOFTMAX, whole = softmax && !g.renorm;
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
  float v[P * NQ];
  float m = -INFINITY, inv = 0.f;
  if (whole) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int e = P * (LPT * q + sub);
#pragma unroll
      for (int c = 0; c < P; ++c) v[P * q + c] = -INFINITY;
      if constexpr (VEC) {
        if (e < g.E) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(row + e * static_cast<int>(sizeof(LT)));
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if constexpr (P == 8) v[P * q + 2 * c] = bf_lo(x[c]), v[P * q + 2 * c + 1] = bf_hi(x[c]);
            else v[P * q + c] = __uint_as_float(x[c]);
          }
        }
      } else {
#pragma unroll
        for (int c = 0; c < P; ++c)
          if (e + c < g.E) v[P * q + c] = load_logit<LT>(row, e + c);
      }
    }
#pragma unroll
    for (int i = 0; i < P * NQ; ++i) m = fmaxf(m, v[i]);
    m = lanes_max<LPT>(m);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < P * NQ; ++i) {
      v[i] = v[i] == -INFINITY ? 0.f : __expf(v[i] - m);
      s += v[i];
    }
    s = lanes_sum<LPT>(s);
    inv = s == 0.f ? 0.f : 1.f / s;        // a row that is masked whole has no gradient
  }
  // of a slot: its own term, and (whole) its expert's score and what every element gets by its score
  float add, s_j = 0.f, shared = 0.f;
  // 1 - s of a sigmoid as 1 / (1 + e^l): the difference loses a score near 1 (6 % of the slope at l = 16, all from 17 on)
  const float rest = softmax ? 1.f : 1.f / (1.f + expf(l_j));
  if (g.renorm) {
    const float r = renormalized<LPT>(softmax, e_j >= 0, l_j);
    add = (gj - lanes_sum<LPT>(gj * r)) * r * rest;
  } else {
    s_j = slot_score(softmax, e_j >= 0, l_j, m, inv);
    if (softmax) shared = lanes_sum<LPT>(gj * s_j);
    add = softmax ? gj : gj * s_j * rest;
  }
  float sum = 0.f;                          // over the slots of the same expert
  for (int j = 0; j < g.k; ++j) {
    const int e = __shfl(e_j, j, LPT);
    const float a = __shfl(add, j, LPT);
    sum += e == e_j ? a : 0.f;
  }
  const float all = -shared * inv;
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    float d[P];
#pragma unroll
    for (int c = 0; c < P; ++c) d[c] = whole ? v[P * q + c] * all : 0.f;
    u32x4 x;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if constexpr (P == 8) x[c] = pack_bf16x2(d[2 * c], d[2 * c + 1]);
      else x[c] = __float_as_uint(d[c]);
    }
    *reinterpret_cast<u32x4*>(mine + P * (LPT * q + sub)) = x;
  }
  wave_order();
  if (e_j >= 0) {
    const float d = whole ? s_j * (sum - shared) : sum;
    if constexpr (P == 8) mine[e_j] = static_cast<LT>(f2bf(d));
    else mine[e_j] = d;
  }
  wave_order();
  if (!live) return;
  char* const out = static_cast<char*>(g.d_logits) + t * g.ld_d * static_cast<int64_t>(sizeof(LT));
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const int e = P * (LPT * q + sub);
    if constexpr (VEC) {
      if (e < g.E) *reinterpret_cast<u32x4*>(out + e * static_cast<int>(sizeof(LT))) = *reinterpret_cast<const u32x4*>(mine + e);
    } else {
#pragma unroll
      for (int c = 0; c < P; ++c)
        if (e + c < g.E) reinterpret_cast<LT*>(out)[e + c] = mine[e + c];
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

template <typename LT, int VPL, int KL, int MODE>
void launch_rows(const GateArgs& a, size_t lds, hipStream_t st) {
  const int lanes = 16 / a.n_group, Eg = a.E / a.n_group, VP = (Eg + lanes - 1) / lanes;
  constexpr int kPiece = sizeof(LT) == 2 && VPL >= 8 ? 8 : 4;
  // whole pieces: of each lane's run, and (the last lane's) of the group
  const int vec = VP % kPiece == 0 && Eg % kPiece == 0 && a.ld % kPiece == 0 && aligned_to(a.logits, kPiece * sizeof(LT));
  const int bias_vec = VP % 4 == 0 && Eg % 4 == 0 && aligned_to(a.bias, 16);
  const dim3 grid = xs_host::grid_of((static_cast<int64_t>(a.T) + 15) / 16);
  if (a.E == 16 * VPL && vec && bias_vec)
    hipLaunchKernelGGL((gate_rows_kernel<LT, VPL, KL, MODE, true>), grid, dim3(256), lds, st, a, VP, vec, bias_vec);
  else hipLaunchKernelGGL((gate_rows_kernel<LT, VPL, KL, MODE, false>), grid, dim3(256), lds, st, a, VP, vec, bias_vec);
}

template <typename LT, int VPL, int MODE>
void launch_rows(const GateArgs& a, size_t lds, hipStream_t st) {
  if (a.k <= 8) launch_rows<LT, VPL, 8, MODE>(a, lds, st);
  else launch_rows<LT, VPL, 16, MODE>(a, lds, st);
}

template <typename LT, int VPL>
void launch_rows(const GateArgs& a, size_t lds, hipStream_t st) {
  if (!a.bias && (a.n_group == 1 || !a.top2)) launch_rows<LT, VPL, kByLogit>(a, lds, st);
  else if (a.score == XS_SCORE_SOFTMAX) launch_rows<LT, VPL, kSoftmax>(a, lds, st);
  else launch_rows<LT, VPL, kSigmoid>(a, lds, st);
}

template <typename LT>
void launch_rows(const GateArgs& a, size_t lds, hipStream_t st) {
  const int lanes = 16 / a.n_group, VP = (a.E / a.n_group + lanes - 1) / lanes;
  if (VP <= 4) launch_rows<LT, 4>(a, lds, st);
  else if (VP <= 8) launch_rows<LT, 8>(a, lds, st);
  else if (VP <= 16) launch_rows<LT, 16>(a, lds, st);
  else launch_rows<LT, 32>(a, lds, st);
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
  constexpr int P = 16 / sizeof(LT);
  const bool vec = a.E % P == 0 && a.ld % P == 0 && a.ld_d % P == 0 && aligned_to(a.logits, 16) && aligned_to(a.d_logits, 16);
  if (a.E <= 256 && a.k <= 16) {
    if (a.E <= 16 * P) launch_grad<LT, 16, 1>(a, vec, st);
    else if (a.E <= 32 * P) launch_grad<LT, 16, 2>(a, vec, st);
    else launch_grad<LT, 16, 4>(a, vec, st);     // fp32 logits only
  } else if (a.E <= 64 * P) {
    launch_grad<LT, 64, 1>(a, vec, st);
  } else if (a.E <= 128 * P) {
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
  const size_t lds = 4 * sizeof(double) * g->E;
  // Sixteen lanes per token where each lane has at most 32 consecutive experts and groups are whole lanes;
  // one wave per token otherwise (32,768 tokens, top-8 of 256 in groups: 15.5 us against 120; 16,384, top-4 of 60 in
  // 4 groups: 8.4 against 18).
  if (a.E <= 512 && a.k <= 16 && 16 % a.n_group == 0) {
    if (g->logits_type == XS_TYPE_BF16) launch_rows<uint16_t>(a, lds, st);
    else launch_rows<float>(a, lds, st);
    return xs_host::launch_status();
  }
  const dim3 grid = xs_host::grid_of((static_cast<int64_t>(T) + 3) / 4);
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
  if (!aligned_to(d_logits, g->logits_type == XS_TYPE_BF16 ? 2 : 4) || (d_logits == logits && ld_d != ld)) return XS_EINVAL;
  if (T == 0) return XS_OK;
  const GateGradArgs a{logits, ld, T, g->E, g->k, g->score, g->renormalize != 0, g->scale, topk_idx, d_topk_w,
                       d_logits, ld_d, dev_status};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (g->logits_type == XS_TYPE_BF16) launch_grad<uint16_t>(a, st);
  else launch_grad<float>(a, st);
  return xs_host::launch_status();
}
