// Counts and balance loss of a router over packed sequences, and the loss's gradient in the logits.
//
//   p_te = softmax(l_t)_e, or s_te / sum_f s_tf of the sigmoid scores s      (shares: they sum to 1)
//   f_se = E counts_se / (k T_s)      P_se = sum over the sequence's tokens of p_te / T_s
//   L_s = alpha sum_e f_se P_se
//   dl_te = p_te (c_e - sum_f c_f p_tf) [(1 - s_te) for sigmoid scores],  c_e = alpha dL_s f_se / T_s
// (counts have no gradient; f is 1 for every expert of a balanced router, and L_s alpha.)
//
// A token is LPT lanes with EPL experts each, a lane's experts V consecutive ones at a time. Every lane keeps the
// sums of its experts over its tokens in registers, so that the only exchange between lanes is a token's
// maximum and sum; a workgroup joins them in LDS and leaves one row of sums and counts. finish_kernel adds a sequence's rows
// in a fixed order, 64 experts to a workgroup, and the last of a sequence's workgroups adds their shares of the loss.
//
// 32,768 tokens of 256 experts, fp32: 10 us (35 MB, which a copy moves in 7.1) and 6.5 to finish, a chain of loads through memory; gradient, bf16: 16 us for 50 MB
// (10.3): waves wait for their token's loads 75% of the time, vector units are busy 26%.
#include <cmath>

#include "xs_common.hpp"
#include "xs_packed.hpp"

namespace xs {
namespace balance {

struct Args {
  const void* logits;
  int64_t ld;
  const int* idx;
  const int32_t* start;     // [n_seq + 1], or NULL: one sequence of T tokens
  int T, E, k, n_seq, sigmoid, chunk, tiles;
  float alpha;
  int width;                // E up to a multiple of four
  float* part;              // [tiles][width] sums of shares
  int* part_n;              // [tiles][width] counts
  float* terms;             // [n_seq][16] shares of the loss
  int* done;                // [n_seq] workgroups that have left theirs
  int* counts;              // [n_seq][E]
  float* mean;              // [n_seq][E]
  float* loss;              // [n_seq]
  int32_t* status;
};

struct GradArgs {
  const void* logits;
  int64_t ld;
  const int32_t* start;
  int T, E, k, n_seq, sigmoid, chunk;
  float alpha;
  const int* counts;
  const float* d_loss;
  const void* d_add;
  int64_t ld_add;
  void* d;
  int64_t ld_d;
  int32_t* status;
};

template <typename A>
__device__ __forceinline__ bool find(const A& a, int t, PackedTile* out) {
  if (a.start) return packed_tile(a.start, a.n_seq, a.T, a.chunk, t, out, a.status);
  *out = PackedTile{0, t, 0, a.T};
  return static_cast<int64_t>(t) * a.chunk < a.T;
}

template <int LPT>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int d = LPT / 2; d; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
template <int LPT>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int d = LPT / 2; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}

// Expert of a lane's value i, lane sub of its token.
template <int V, int LPT>
__device__ __forceinline__ int expert_of(int sub, int i) { return (sub + i / V * LPT) * V + i % V; }

// A token's values, `fill` where there is no expert.
template <typename LT, int V, int LPT, int EPL>
__device__ __forceinline__ void load_row(const void* m, int64_t at, int E, int sub, float fill, float (&l)[EPL]) {
  const LT* const row = static_cast<const LT*>(m) + at;
#pragma unroll
  for (int i = 0; i < EPL; i += V) {
    const int e = expert_of<V, LPT>(sub, i);
    if constexpr (V == 1) {
      l[i] = fill;
      if (e < E) {
        if constexpr (sizeof(LT) == 2) l[i] = __uint_as_float(static_cast<uint32_t>(row[e]) << 16);
        else l[i] = row[e];
      }
    } else if (e < E) {                 // the vectors of V = 4 need E % 4 == 0
      if constexpr (sizeof(LT) == 2) {
        const uint2 r = *reinterpret_cast<const uint2*>(row + e);
        l[i] = bf_lo(r.x), l[i + 1] = bf_hi(r.x), l[i + 2] = bf_lo(r.y), l[i + 3] = bf_hi(r.y);
      } else {
        const f32x4 r = *reinterpret_cast<const f32x4*>(row + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) l[i + j] = r[j];
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) l[i + j] = fill;
    }
  }
}

// Logits x to shares p and, for sigmoid scores, rest = 1 - s (as 1 / (1 + e^x), which a score near 1 does not cancel).
// Scores below 2^-126 come out as 0 (the reciprocal does not give smaller numbers). Where a token's sum to less than 2^-64 each is e^x but for 2^-64
// of it, and the shares are those of a softmax.
template <int LPT, int EPL, bool REST>
__device__ __forceinline__ void shares(bool sigmoid, const float (&x)[EPL], float (&p)[EPL], float (&rest)[REST ? EPL : 1]) {
  constexpr float kLog2e = 1.4426950408889634f;
  float total = 0.f;
  // e^(x - the token's largest x) into p, and their sum
  auto exponentials = [&] {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < EPL; ++i) top = fmaxf(top, x[i]);
    top = lanes_max<LPT>(top);
    if (top == -INFINITY) top = 0.f;          // every expert masked: all shares 0
    total = 0.f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      p[i] = __builtin_amdgcn_exp2f((x[i] - top) * kLog2e);
      total += p[i];
    }
    total = lanes_sum<LPT>(total);
  };
  if (sigmoid) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      // the reciprocal of one unit in the last place, which is what exp2 has too: a quotient takes ten instructions
      p[i] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-x[i] * kLog2e));
      if constexpr (REST) rest[i] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x[i] * kLog2e));
      total += p[i];
    }
    total = lanes_sum<LPT>(total);
    if (total < 0x1p-64f) exponentials();      // the same in all lanes of the token
  } else {
    exponentials();
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int i = 0; i < EPL; ++i) p[i] *= inv;
}

template <typename LT, int V, int LPT, int EPL>
__global__ __launch_bounds__(256) void sums_kernel(Args a) {
  constexpr int kGroups = 256 / LPT, kCols = LPT * EPL;
  __shared__ float sums[kGroups * kCols];
  __shared__ int hist[kCols];
  const int tid = threadIdx.x, sub = tid % LPT, grp = tid / LPT;
  for (int64_t i = block_number() * 256 + tid; i < a.n_seq; i += static_cast<int64_t>(gridDim.x) * gridDim.y * 256) a.done[i] = 0;
  PackedTile s;
  if (block_number() >= a.tiles || !find(a, static_cast<int>(block_number()), &s)) return;
  const int first = s.tile * a.chunk, n = min(a.chunk, s.rows - first);
  const int64_t t0 = static_cast<int64_t>(s.start) + first;
  // a token's logits are on their way while the token before is worked on
  float next[EPL], acc[EPL];
  load_row<LT, V, LPT, EPL>(a.logits, (t0 + min(grp, n - 1)) * a.ld, a.E, sub, -INFINITY, next);
  for (int e = tid; e < kCols; e += 256) hist[e] = 0;
  __syncthreads();
  for (int64_t i = tid; i < static_cast<int64_t>(n) * a.k; i += 256) {
    const int e = a.idx[t0 * a.k + i];
    if (e < 0 || e >= a.E) set_status(a.status, XS_EBADINPUT);
    else atomicAdd(&hist[e], 1);
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) acc[i] = 0.f;
  for (int t = grp; t < n; t += kGroups) {
    float x[EPL], p[EPL], none[1];
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = next[i];
    load_row<LT, V, LPT, EPL>(a.logits, (t0 + min(t + kGroups, n - 1)) * a.ld, a.E, sub, -INFINITY, next);
    shares<LPT, EPL, false>(a.sigmoid, x, p, none);
#pragma unroll
    for (int i = 0; i < EPL; ++i) acc[i] += p[i];
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) sums[grp * kCols + expert_of<V, LPT>(sub, i)] = acc[i];
  __syncthreads();
  const int64_t row = block_number() * a.width;
  for (int e = tid; e < a.E; e += 256) {
    float v = 0.f;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) v += sums[g * kCols + e];
    a.part[row + e] = v;
    a.part_n[row + e] = hist[e];
  }
}

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 64 experts of a sequence: 16 lanes have four each, NT / 16 groups of lanes the tiles' rows in turn. (All experts in one workgroup, without the
// count of workgroups, is no faster: 7.4 us against 6.9 for eight sequences of 32768 tokens, the longest of which has 180 tiles.)
template <int NT>
__global__ __launch_bounds__(NT) void finish_kernel(Args a) {
  constexpr int kGroups = NT / 16, kAhead = 8;
  __shared__ __attribute__((aligned(16))) f32x4 sums[NT / 64][16];
  __shared__ __attribute__((aligned(16))) i32x4 hist[NT / 64][16];
  const int tid = threadIdx.x, blocks = (a.E + 63) / 64;
  const int64_t id = block_number();
  const int s = static_cast<int>(id / blocks), b = static_cast<int>(id - static_cast<int64_t>(s) * blocks);
  if (s >= a.n_seq) return;
  int first = 0, rows = a.T;                           // the sequence's first tile and tokens
  if (a.start) {
    int before = 0;
    for (int s0 = 0; s0 <= s; s0 += 64) {
      const int i = s0 + (tid & 63);
      int len = 0;
      if (i < a.n_seq) {
        const int lo = a.start[i], hi = a.start[i + 1];
        len = lo < 0 || hi < lo || hi > a.T ? 0 : hi - lo;
      }
      const int tiles = static_cast<int>((static_cast<int64_t>(len) + a.chunk - 1) / a.chunk), upto = wave_scan(tiles);
      if (s < s0 + 64) {
        rows = __builtin_amdgcn_readlane(len, s - s0);
        first = before + __builtin_amdgcn_readlane(upto, s - s0) - __builtin_amdgcn_readlane(tiles, s - s0);
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  int tiles = static_cast<int>((static_cast<int64_t>(rows) + a.chunk - 1) / a.chunk);
  tiles = min(tiles, max(0, a.tiles - first));         // sequences that overlap have more tiles than the workspace holds
  const int q = tid & 15, g = tid >> 4, e = b * 64 + 4 * q;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  i32x4 c = {0, 0, 0, 0};
  if (e < a.width) {
    const int64_t base = static_cast<int64_t>(first) * a.width + e;
    for (int i = g; i < tiles; i += kAhead * kGroups) {
      f32x4 vs[kAhead];
      i32x4 cs[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int64_t at = base + static_cast<int64_t>(min(i + u * kGroups, tiles - 1)) * a.width;
        vs[u] = *reinterpret_cast<const f32x4*>(a.part + at);
        cs[u] = *reinterpret_cast<const i32x4*>(a.part_n + at);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i + u * kGroups < tiles) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            v[j] += vs[u][j];
            c[j] += cs[u][j];
          }
        }
    }
  }
#pragma unroll
  for (int d = 16; d < 64; d <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] += __shfl_xor(v[j], d);
      c[j] += __shfl_xor(c[j], d);
    }
  if ((tid & 63) < 16) {
    sums[tid >> 6][q] = v;
    hist[tid >> 6][q] = c;
  }
  __syncthreads();
  if (tid >= 64) return;
  const int x = b * 64 + tid;
  float term = 0.f;
  if (x < a.E) {
    float sum = 0.f;
    int n = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      sum += reinterpret_cast<const float*>(sums[w])[tid];
      n += reinterpret_cast<const int*>(hist[w])[tid];
    }
    const float tokens = static_cast<float>(rows > 0 ? rows : 1), mean = sum / tokens;
    a.counts[static_cast<int64_t>(s) * a.E + x] = n;
    a.mean[static_cast<int64_t>(s) * a.E + x] = mean;
    term = static_cast<float>(n) / (static_cast<float>(a.k) * tokens) * mean;
  }
  term = lanes_sum<64>(term);
  if (tid) return;
  if (blocks > 1) {
    float* const terms = a.terms + static_cast<int64_t>(s) * 16;
    // the term has reached memory before the count says so; a release would write the whole L2 back
    store_through4(terms + b, __float_as_uint(term));
    wait_vm<0>();
    if (__hip_atomic_fetch_add(a.done + s, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != blocks - 1) return;
    term = 0.f;
    for (int i = 0; i < blocks; ++i) term += __hip_atomic_load(terms + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  a.loss[s] = a.alpha * static_cast<float>(a.E) * term;
}

template <typename LT, int V, int LPT, int EPL>
__global__ __launch_bounds__(256) void grad_kernel(GradArgs a) {
  constexpr int kGroups = 256 / LPT;
  PackedTile s;
  if (!find(a, static_cast<int>(block_number()), &s)) return;
  const int tid = threadIdx.x, sub = tid % LPT, grp = tid / LPT;
  const int first = s.tile * a.chunk, n = min(a.chunk, s.rows - first);
  const int64_t t0 = static_cast<int64_t>(s.start) + first;
  const float rows = static_cast<float>(s.rows);
  const float unit = a.alpha * static_cast<float>(a.E) / static_cast<float>(a.k) / rows * a.d_loss[s.seq] / rows;
  float c[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = expert_of<V, LPT>(sub, i);
    c[i] = e < a.E ? unit * static_cast<float>(a.counts[static_cast<int64_t>(s.seq) * a.E + e]) : 0.f;
  }
  for (int t = grp; t < n; t += kGroups) {
    float x[EPL], p[EPL], rest[EPL], add[EPL];
    load_row<LT, V, LPT, EPL>(a.logits, (t0 + t) * a.ld, a.E, sub, -INFINITY, x);
    load_row<LT, V, LPT, EPL>(a.d_add, (t0 + t) * a.ld_add, a.d_add ? a.E : 0, sub, 0.f, add);
    shares<LPT, EPL, true>(a.sigmoid, x, p, rest);
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) dot = __builtin_fmaf(c[i], p[i], dot);
    dot = lanes_sum<LPT>(dot);
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      float d = p[i] * (c[i] - dot);
      if (a.sigmoid) d *= rest[i];
      p[i] = add[i] + d;
    }
    LT* const out = static_cast<LT*>(a.d) + (t0 + t) * a.ld_d;
#pragma unroll
    for (int i = 0; i < EPL; i += V) {
      const int e = expert_of<V, LPT>(sub, i);
      if (e >= a.E) continue;
      if constexpr (V == 1) {
        if constexpr (sizeof(LT) == 2) out[e] = static_cast<uint16_t>(f2bf(p[i]));
        else out[e] = p[i];
      } else if constexpr (sizeof(LT) == 2) {
        *reinterpret_cast<uint2*>(out + e) = make_uint2(pack_bf16x2(p[i], p[i + 1]), pack_bf16x2(p[i + 2], p[i + 3]));
      } else {
        *reinterpret_cast<f32x4*>(out + e) = f32x4{p[i], p[i + 1], p[i + 2], p[i + 3]};
      }
    }
  }
}

constexpr int kMaxSeq = 1 << 16;

}  // namespace balance
}  // namespace xs

using namespace xs;

namespace {

// Tokens per workgroup, 16 at least, from the shape and the device alone: the chip's CUs twice over for the sums, whose every workgroup
// leaves a row; four times for the gradient (32765 tokens of 256 experts: 20.5 us with two, 16.9 with four, 21 with eight).
int chunk_of(int32_t T, int times = 2) {
  const int64_t groups = times * int64_t(xs_host::num_cus());
  const int64_t c = groups > 0 ? (T + groups - 1) / groups : 64;
  return static_cast<int>(c < 16 ? 16 : (c + 15) / 16 * 16);
}

int64_t width_of(int32_t E) { return (E + 3) / 4 * 4; }
int64_t tiles_of(int32_t T, int32_t n_seq, int chunk) {
  const int64_t n = packed_tiles_bound(T, n_seq, 1, chunk);
  return n > 0 ? n : 1;
}

int64_t workspace_of(int32_t T, int32_t E, int32_t n_seq) { return tiles_of(T, n_seq, chunk_of(T)) * width_of(E) * 8 + int64_t(n_seq) * 17 * 4; }

int balance_ok(const xs_gate* g, const void* logits, int64_t ld, int32_t T, const int32_t* start, int32_t n_seq, float alpha) {
  if (!g || (!logits && T) || g->E < 1 || g->E > 1024 || g->k < 1 || g->k > g->E || g->k > 32 || g->reserved != 0) return XS_EINVAL;
  if (g->score != XS_SCORE_SOFTMAX && g->score != XS_SCORE_SIGMOID) return XS_EINVAL;
  if (g->logits_type != XS_TYPE_BF16 && g->logits_type != XS_TYPE_F32) return XS_EINVAL;
  if (T < 0 || ld < g->E || ld > (int64_t(1) << 40) || !std::isfinite(alpha)) return XS_EINVAL;
  if (reinterpret_cast<uintptr_t>(logits) & (g->logits_type == XS_TYPE_BF16 ? 1 : 3)) return XS_EINVAL;
  if (n_seq < 1 || n_seq > balance::kMaxSeq || (!start && n_seq != 1)) return XS_EINVAL;
  if (T > INT32_MAX - 64) return XS_EUNSUPPORTED;
  return XS_OK;
}

bool vectors(const void* p, int64_t ld, int32_t E, int size) {      // rows of four values at a time
  return !p || (E % 4 == 0 && ld % 4 == 0 && !(reinterpret_cast<uintptr_t>(p) & (4 * size - 1)));
}

template <typename LT, int V>
void launch_sums(const balance::Args& a, dim3 grid, hipStream_t st) {
  if (a.E <= 64) hipLaunchKernelGGL((balance::sums_kernel<LT, V, 16, 4>), grid, dim3(256), 0, st, a);
  else if (a.E <= 256) hipLaunchKernelGGL((balance::sums_kernel<LT, V, 16, 16>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((balance::sums_kernel<LT, V, 64, 16>), grid, dim3(256), 0, st, a);
}

template <typename LT, int V>
void launch_grad(const balance::GradArgs& a, dim3 grid, hipStream_t st) {
  if (a.E <= 64) hipLaunchKernelGGL((balance::grad_kernel<LT, V, 16, 4>), grid, dim3(256), 0, st, a);
  else if (a.E <= 256) hipLaunchKernelGGL((balance::grad_kernel<LT, V, 16, 16>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((balance::grad_kernel<LT, V, 64, 16>), grid, dim3(256), 0, st, a);
}

}  // namespace

extern "C" int xs_balance_loss_workspace_bytes(int32_t T, int32_t E, int32_t n_seq, int64_t* bytes) {
  if (!bytes || T < 0 || E < 1 || E > 1024 || n_seq < 1 || n_seq > balance::kMaxSeq) return XS_EINVAL;
  if (T > INT32_MAX - 64) return XS_EUNSUPPORTED;
  *bytes = workspace_of(T, E, n_seq);
  return XS_OK;
}

extern "C" int xs_balance_loss(const xs_gate* g, const void* logits, int64_t ld, int32_t T, const int32_t* topk_idx,
                               const int32_t* seq_start, int32_t n_seq, float alpha, int32_t* counts, float* mean_share, float* loss,
                               void* workspace, int64_t workspace_bytes, int32_t* dev_status, void* stream) {
  if (int rc = balance_ok(g, logits, ld, T, seq_start, n_seq, alpha)) return rc;
  if ((!topk_idx && T) || !counts || !mean_share || !loss) return XS_EINVAL;
  const int64_t tiles = tiles_of(T, n_seq, chunk_of(T));
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15) || workspace_bytes < workspace_of(T, g->E, n_seq)) return XS_EWORKSPACE;
  balance::Args a{logits, ld, topk_idx, seq_start, T, g->E, g->k, n_seq, g->score == XS_SCORE_SIGMOID, chunk_of(T), static_cast<int>(tiles), alpha,
                  static_cast<int>(width_of(g->E)), static_cast<float*>(workspace), nullptr, nullptr, nullptr, counts, mean_share, loss, dev_status};
  a.part_n = reinterpret_cast<int*>(a.part + tiles * a.width);
  a.terms = reinterpret_cast<float*>(a.part_n + tiles * a.width);
  a.done = reinterpret_cast<int*>(a.terms + int64_t(n_seq) * 16);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid = xs_host::grid_of(tiles);
  const bool v4 = vectors(logits, ld, g->E, g->logits_type == XS_TYPE_BF16 ? 2 : 4);
  if (g->logits_type == XS_TYPE_BF16) v4 ? launch_sums<uint16_t, 4>(a, grid, st) : launch_sums<uint16_t, 1>(a, grid, st);
  else v4 ? launch_sums<float, 4>(a, grid, st) : launch_sums<float, 1>(a, grid, st);
  if (xs_host::launch_status()) return XS_EHIP;
  const dim3 parts = xs_host::grid_of(int64_t(n_seq) * ((g->E + 63) / 64));
  if (tiles > 16 * int64_t(n_seq)) hipLaunchKernelGGL(balance::finish_kernel<1024>, parts, dim3(1024), 0, st, a);
  else hipLaunchKernelGGL(balance::finish_kernel<256>, parts, dim3(256), 0, st, a);
  return xs_host::launch_status();
}

extern "C" int xs_balance_loss_backward(const xs_gate* g, const void* logits, int64_t ld, int32_t T, const int32_t* seq_start,
                                        int32_t n_seq, float alpha, const int32_t* counts, const float* d_loss, const void* d_add,
                                        int64_t ld_add, void* d_logits, int64_t ld_d, int32_t* dev_status, void* stream) {
  if (int rc = balance_ok(g, logits, ld, T, seq_start, n_seq, alpha)) return rc;
  const int size = g->logits_type == XS_TYPE_BF16 ? 2 : 4;
  const auto lies = [=](const void* p, int64_t l) {
    return l >= g->E && l <= (int64_t(1) << 40) && !(reinterpret_cast<uintptr_t>(p) & (size - 1));
  };
  if (!counts || !d_loss || (!d_logits && T) || !lies(d_logits, ld_d) || (d_add && !lies(d_add, ld_add))) return XS_EINVAL;
  if (T == 0) return XS_OK;
  if ((d_logits == logits && ld_d != ld) || (d_logits == d_add && ld_d != ld_add)) return XS_EINVAL;
  const balance::GradArgs a{logits, ld, seq_start, T, g->E, g->k, n_seq, g->score == XS_SCORE_SIGMOID, chunk_of(T, 4), alpha, counts,
                            d_loss, d_add, ld_add, d_logits, ld_d, dev_status};
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid = xs_host::grid_of(tiles_of(T, n_seq, a.chunk));
  const bool v4 = vectors(logits, ld, g->E, size) && vectors(d_add, ld_add, g->E, size) && vectors(d_logits, ld_d, g->E, size);
  if (g->logits_type == XS_TYPE_BF16) v4 ? launch_grad<uint16_t, 4>(a, grid, st) : launch_grad<uint16_t, 1>(a, grid, st);
  else v4 ? launch_grad<float, 4>(a, grid, st) : launch_grad<float, 1>(a, grid, st);
  return xs_host::launch_status();
}
