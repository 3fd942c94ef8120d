// Causal attention of packed sequences with grouped heads, over prompts and over a cache, and its gradients.
//
//   s_ij = scale q_i . k_j for the keys j that row i sees      o_i = sum_j exp(s_ij - lse_i) v_j
//   P_ij = exp(s_ij - lse_i)      delta_i = do_i . o_i      dS_ij = P_ij (do_i . v_j - delta_i)
//   dq_i = scale sum_j dS_ij k_j      dk_j = scale sum_i dS_ij q_i      dv_j = sum_i P_ij do_i
//
// The rows of a sequence and a key head are its queries times the G query heads that read that key head,
// row r = query r / G, head r % G: one new token of a request is G rows, not one, and all heads of a group take
// a tile of keys from LDS once. A row's mask is one number, how many keys it sees.
//
// Every product is the 32 x 32 x 16 matrix instruction in the transposed form, so that a lane's accumulators
// belong to one row (forward, dq) or one key (dk, dv): its B operand is held in registers for the whole
// loop, its A operand comes from tiles in LDS, by rows (16 bytes a lane) or by columns (gfx950's transposing
// read), and a result in registers becomes the next product's B operand with two half swaps for
// 16 keys or rows.
//
// Forward, four forms (form_of chooses): rows_kernel, a workgroup 128 rows over all keys that they see; wide_kernel, the same with the
// keys dealt out evenly where such tiles do not fill the chip; narrow_kernel, a few rows a sequence, each wave its share of all keys; short_kernel,
// 32 rows a workgroup with the keys shared out among its waves: short caches, few or short prompts. Gradients: dq_kernel by rows, dkv_kernel by keys, each recomputing P;
// dq_short_kernel and dkv_short_kernel for few or short prompts.
//
// LDS tiles are rows of 2 D bytes in pieces of 16; row r keeps its piece p at p ^ swz(r). A read by rows takes one
// piece of 16 consecutive rows at a time, a read by columns four pieces of four consecutive rows; swz
// spreads a tile's reads over all banks, also where the gradients read one tile both ways.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "xs_common.hpp"
#include "xs_packed.hpp"

namespace xs {
namespace pattn {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
typedef float f32x2_t __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// a row's running maximum is raised (and its sums rescaled) only when a block's maximum exceeds it by more than
// this many powers of two; until then probabilities stay <= 2^8
constexpr float kRescaleSlack = 8.f;

// One of q, k, v, ...: where row t of head h lies, in bytes.
struct Mat {
  char* p;
  int64_t row, head;
};
__device__ __forceinline__ char* at(const Mat& m, int64_t row, int head) { return m.p + row * m.row + head * m.head; }

struct Args {
  Mat q, k, v, o, d_o, dq, dk, dv;
  const int32_t *q_start, *k_start, *k_rows;
  int n_seq, H, Hkv, G, Tq, Tk, causal, max_k;
  int shift;             // log2 G, or -1
  int cus;
  float scale, scale_log2e;
  float* lse;            // [H][Tq]
  float *delta, *lse2;   // [H][Tq] (gradients): do . o, lse in powers of two
  float* part_o;         // parts: two slots of each range
  float* part_ml;        // their rows' maxima and sums
  int32_t* status;
};

// a / b of what is not negative and the same in all lanes: mostly it fits 32 bits, and a division of 64 takes four times as long.
__device__ __forceinline__ int64_t quot(int64_t a, int64_t b) {
  if ((a | b) >> 32) return a / b;
  return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
}

struct Seq {
  int q0, nq, k0, nk;       // its first query and their number, its first key and theirs
};

// The query of row r.
__device__ __forceinline__ int query_of(const Args& a, int r) { return a.shift >= 0 ? r >> a.shift : r / a.G; }
// How many keys row r of a sequence sees.
__device__ __forceinline__ int sees(const Args& a, int r, int nq, int nk) {
  return a.causal ? min(max(nk - nq + query_of(a, r) + 1, 0), nk) : nk;
}
// Where row r of a sequence and key head lies in q, o, ...
__device__ __forceinline__ char* row_at(const Args& a, const Mat& m, const Seq& s, int kvh, int r) {
  const int qi = query_of(a, r);
  return at(m, s.q0 + qi, kvh * a.G + (r - qi * a.G));
}

// A lane's value, taken where it stands: what follows from it does not hold registers over a loop before.
__device__ __forceinline__ int here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// How a tile is read.
enum Way { kRows, kCols, kBoth };

template <int D>
struct Geo {
  static constexpr int kRow = 2 * D, kPieces = D / 8, kRowsPerLoad = 1024 / kRow, kSteps = D / 16, kBlocks = D / 32;
  // D = 128: a row is all banks; by rows, 16 consecutive rows need distinct values, by columns four consecutive
  // rows distinct upper bits. D = 64: two rows are all banks; the same for rows with the same low bit.
  static __device__ __forceinline__ int swz(Way way, int r) {
    if (way == kRows) return D == 128 ? r & 15 : r >> 1 & 7;
    if (way == kCols) return D == 128 ? (r & 3) << 2 : (r >> 1 & 1) << 2;
    return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
  }
};

// A tile of NR rows into LDS by NW waves (wave w of them), straight from memory; rows past `left` are zeros.
template <int D, int NR, int NW, Way WAY>
struct Loader {
  using G = Geo<D>;
  static constexpr int kLoads = NR / (G::kRowsPerLoad * NW), kStep = G::kRowsPerLoad * NW;
  static_assert(kLoads * kStep == NR);
  static constexpr int kVar = kStep >= 16 ? 1 : 16 / kStep;     // loads until the swizzles repeat
  uint32_t off[kVar];
  uint32_t row_bytes;
  __device__ __forceinline__ Loader(int w, int lane, int64_t row) : row_bytes(static_cast<uint32_t>(row)) {
#pragma unroll
    for (int i = 0; i < kVar; ++i) {
      const int r = G::kRowsPerLoad * (NW * i + w) + lane / G::kPieces;
      off[i] = static_cast<uint32_t>(r) * row_bytes + (((lane % G::kPieces) ^ G::swz(WAY, r)) << 4);
    }
  }
  __device__ __forceinline__ void issue(const char* base, int left, lds_char* dst, int w) const {
    const int n = min(left, NR);
    const v4i rs = buffer_rsrc(base, n > 0 ? (n - 1) * row_bytes + G::kRow : 0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      load_lds16(rs, off[i % kVar] + static_cast<uint32_t>(i / kVar * kVar * kStep) * row_bytes, dst + (NW * i + w) * 1024);
  }
};

// A lane's addresses of its fragments in a tile, by rows: row lane % 32 (+ 32 b), piece 2 kk + lane / 32; the pieces'
// upper bits are toggled over the first's.
template <int D, Way WAY>
struct RowReads {
  int first;
  __device__ __forceinline__ explicit RowReads(int lane) {
    const int r = lane & 31, up = lane >> 5;
    first = r * Geo<D>::kRow + ((up ^ Geo<D>::swz(WAY, r)) << 4);
  }
  __device__ __forceinline__ int at(int kk) const { return first ^ kk << 5; }
  __device__ __forceinline__ RowReads fresh() const {
    RowReads r(*this);
    r.first = here(first);
    return r;
  }
};
// By columns: key or row 16 s (+ 4 hf), column block db. Where the swizzle does not change over four rows the second
// address is the first and a constant.
template <int D, Way WAY>
struct ColReads {
  static constexpr int kHalves = WAY == kBoth ? 2 : 1;
  int first[kHalves];
  __device__ __forceinline__ explicit ColReads(int lane) {
    const int grp = lane >> 4, j = lane & 15, d = 16 * (grp & 1) + 4 * (j & 3);
#pragma unroll
    for (int hf = 0; hf < kHalves; ++hf) {
      const int k = 8 * (grp >> 1) + (j >> 2) + 4 * hf;
      first[hf] = k * Geo<D>::kRow + (((d >> 3) ^ Geo<D>::swz(WAY, k)) << 4) + (d >> 2 & 1) * 8;
    }
  }
  __device__ __forceinline__ int at(int hf, int db) const { return first[hf] ^ db << 6; }
  __device__ __forceinline__ ColReads fresh() const {
    ColReads r(*this);
#pragma unroll
    for (int hf = 0; hf < kHalves; ++hf) r.first[hf] = here(first[hf]);
    return r;
  }
};

// N matrix instructions, mul(i, operand), whose LDS reads are issued AHEAD instructions before them. Left to itself the
// compiler reads one operand, waits for it and multiplies. FIRST: the wave goes before the others of its SIMD, whose softmax fills the
// matrix unit's time (heads of 128: rows 550 -> 530 us, dq 322 -> 306; of 64 2% slower).
template <int N, int AHEAD, bool FIRST, class Read, class Mul>
__device__ __forceinline__ void fed(const Read& read, const Mul& mul) {
  decltype(read(0)) buf[AHEAD + 1];
  if constexpr (FIRST) __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) buf[i] = read(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i + AHEAD < N) buf[(i + AHEAD) % (AHEAD + 1)] = read(i + AHEAD);
    __builtin_amdgcn_sched_barrier(0);
    mul(i, buf[i % (AHEAD + 1)]);
    __builtin_amdgcn_sched_barrier(0);
  }
  if constexpr (FIRST) __builtin_amdgcn_s_setprio(0);
}

template <int D, Way WAY>
__device__ __forceinline__ bf16x8 row_operand(const lds_char* tile, int b, const RowReads<D, WAY>& rd, int kk) {
  return *(const lds_bf16x8*)(tile + b * 32 * Geo<D>::kRow + rd.at(kk));
}
template <int D, Way WAY>
__device__ __forceinline__ bf16x8 col_operand(const lds_char* tile, int s, const ColReads<D, WAY>& rd, int db) {
  constexpr int kLast = ColReads<D, WAY>::kHalves - 1, kNext = kLast ? 0 : 4 * Geo<D>::kRow;
  const s16x4 r0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + 16 * s * Geo<D>::kRow + rd.at(0, db)));
  const s16x4 r1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + 16 * s * Geo<D>::kRow + kNext + rd.at(kLast, db)));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(r0, r1, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ void zero(f32x16& v) {
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] = 0.f;
}
__device__ __forceinline__ void mma(f32x16& acc, bf16x8 a, bf16x8 b) { acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0); }

// acc[row of the tile][lane's column] = tile rows 32 b .. + 31 times the held fragments
template <int D, Way WAY>
__device__ __forceinline__ f32x16 rows_product(const lds_char* tile, int b, const RowReads<D, WAY>& rd, const bf16x8 (&frag)[D / 16]) {
  f32x16 acc;
  zero(acc);
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) mma(acc, row_operand<D>(tile, b, rd, kk), frag[kk]);
  return acc;
}

// Accumulator entry e of a 32-row block is row 8 (e / 4) + 4 (lane / 32) + e % 4.
__device__ __forceinline__ int entry_row(int e, int up) { return 8 * (e >> 2) + 4 * up + (e & 3); }

// The packed pairs of a 32-row block as the B operands of its two steps of 16 rows: the lower half needs rows
// +0 .. 7, the upper half +8 .. 15.
__device__ __forceinline__ bf16x8 operand(const uint32_t (&pk)[8], int half) {
  const int o = 4 * half;
  const auto x = __builtin_amdgcn_permlane32_swap(pk[o], pk[o + 2], false, false);
  const auto y = __builtin_amdgcn_permlane32_swap(pk[o + 1], pk[o + 3], false, false);
  const u32x4 v = {x[0], y[0], x[1], y[1]};
  return __builtin_bit_cast(bf16x8, v);
}

// The two halves of a wave hold two halves of a row's keys; both results through one two-element vector (a bit
// cast of each on its own was compiled to read the first twice).
__device__ __forceinline__ f32x2_t both_halves(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const u32x2 t = {r[0], r[1]};
  return __builtin_bit_cast(f32x2_t, t);
}
__device__ __forceinline__ float max_halves(float x) {
  const f32x2_t h = both_halves(x);
  return fmaxf(h.x, h.y);
}
__device__ __forceinline__ float add_halves(float x) {
  const f32x2_t h = both_halves(x);
  return h.x + h.y;
}

template <int D>
__device__ __forceinline__ void load_frags(const char* row, bf16x8 (&f)[D / 16]) {
  const int up = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) f[kk] = *reinterpret_cast<const bf16x8*>(row + 32 * kk + 16 * up);
}

// 8 consecutive columns of a lane's row from the pieces of four that the two halves of a wave hold: the lower half gets the
// first 8, the upper half the next.
__device__ __forceinline__ u32x4 columns8(u32x2 first, u32x2 next) {
  const auto x = __builtin_amdgcn_permlane32_swap(first[0], next[0], false, false);
  const auto y = __builtin_amdgcn_permlane32_swap(first[1], next[1], false, false);
  return u32x4{x[0], y[0], x[1], y[1]};
}
__device__ __forceinline__ u32x2 four(const f32x16& v, int g, float c) {
  return u32x2{pack_bf16x2(v[4 * g] * c, v[4 * g + 1] * c), pack_bf16x2(v[4 * g + 2] * c, v[4 * g + 3] * c)};
}

// Accumulators, times c, as bf16: each lane its row (or key), all lanes together; where `live`.
template <int D>
__device__ __forceinline__ void store_row(char* row, const f32x16 (&acc)[D / 32], float c, bool live) {
  const int up = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      const u32x4 v = columns8(four(acc[db], g, c), four(acc[db], g + 1, c));
      if (live) *reinterpret_cast<u32x4*>(row + (32 * db + 8 * (g + up)) * 2) = v;
    }
}

// The same through LDS (32 rows of 2 D bytes, the wave's own), whole rows at a time: row(i) says where row i goes, NULL: nowhere.
// A store by lanes' rows touches 32 cache lines, 16 of them for a wave took as long as one and a half tiles of 64 keys.
template <int D, class Row>
__device__ __forceinline__ void store_rows(lds_char* mine, const f32x16 (&acc)[D / 32], float c, const Row& row) {
  using G = Geo<D>;
  const int lane = here(threadIdx.x & 63), i = lane & 31, up = lane >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *(lds_u32x2*)(mine + i * G::kRow + (((4 * db + g) ^ G::swz(kRows, i)) << 4) + up * 8) = four(acc[db], g, c);
#pragma unroll
  for (int t = 0; t < 32 / G::kRowsPerLoad; ++t) {
    const int r = t * G::kRowsPerLoad + lane / G::kPieces, p = lane % G::kPieces;
    const bf16x8 v = *(const lds_bf16x8*)(mine + r * G::kRow + ((p ^ G::swz(kRows, r)) << 4));
    char* const dst = row(r);
    if (dst) *reinterpret_cast<bf16x8*>(dst + 16 * p) = v;
  }
}

// A row's softmax so far: maximum (in powers of two, scaled) and sum. The maximum starts at the lowest finite
// value, so that keys a row does not see (score -inf) weigh 0 also before the first that it sees.
template <int D>
struct Soft {
  float m, l;
  f32x16 o[D / 32];
  __device__ __forceinline__ void clear() {
    m = -FLT_MAX;
    l = 0.f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
  }
  // NB blocks of 32 keys, scores s, to probabilities (packed bf16); the sum takes them unrounded: it gives
  // lse too, and a rounding of 2^-9 in it would be lse's error for rows with few keys.
  template <int NB>
  __device__ __forceinline__ void take(f32x16 (&s)[NB], float scale_log2e, uint32_t (&pk)[NB][8]) {
    float mx = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[b][e]);
    const float mxs = max_halves(mx) * scale_log2e;
    if (__builtin_amdgcn_ballot_w64(mxs > m + kRescaleSlack)) {    // wave-uniform
      const float m_new = fmaxf(m, mxs), corr = __builtin_amdgcn_exp2f(m - m_new);
      l *= corr;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] *= corr;
      m = m_new;
    }
    float rs = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][2 * e], scale_log2e, -m));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][2 * e + 1], scale_log2e, -m));
        rs += p0 + p1;
        pk[b][e] = pack_bf16x2(p0, p1);
      }
    l += add_halves(rs);
  }
  __device__ __forceinline__ float inverse() const { return l == 0.f ? 0.f : 1.f / l; }
  __device__ __forceinline__ float lse() const { return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2; }
};

// Scores of keys that the lane's row does not see become -inf.
__device__ __forceinline__ void hide(f32x16& s, int key0, int lim, int up) {
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (key0 + entry_row(e, up) >= lim) s[e] = -INFINITY;
}

__device__ __forceinline__ int64_t lane64(int64_t v, int l) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), l), hi = __builtin_amdgcn_readlane(static_cast<int>(v >> 32), l);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ Seq lane_seq(const Seq& s, int l) {
  return Seq{__builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.nq, l), __builtin_amdgcn_readlane(s.k0, l), __builtin_amdgcn_readlane(s.nk, l)};
}

// Sequence i; without queries and keys (and with the error noted) if they do not lie in q and k, and where there is none.
__device__ __forceinline__ Seq seq_of(const Args& a, int i) {
  if (i >= a.n_seq) return Seq{0, 0, 0, 0};
  const int q0 = a.q_start[i], q1 = a.q_start[i + 1], k0 = a.k_start[i], nk = a.k_rows ? a.k_rows[i] : a.k_start[i + 1] - k0;
  if (q0 < 0 || q1 < q0 || q1 > a.Tq || k0 < 0 || nk < 0 || nk > a.max_k || k0 > a.Tk - nk) {
    set_status(a.status, XS_EBADINPUT);
    return Seq{0, 0, 0, 0};
  }
  return Seq{q0, q1 - q0, k0, nk};
}

// The workgroup's tile of PER rows (or keys) of a sequence and key head, key heads side by side; false past the last. Every wave finds it
// by itself, 64 sequences a step, all that it has to know of one in a lane and on its way at once.
template <int PER, bool KEYS = false>
__device__ __forceinline__ bool tile_of(const Args& a, Seq* s, int* kvh, int* tile) {
  const int64_t id = block_number(), t = quot(id, a.Hkv);
  *kvh = static_cast<int>(id - t * a.Hkv);
  int left = static_cast<int>(t);
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    const Seq mine = seq_of(a, s0 + (threadIdx.x & 63));
    const int n = static_cast<int>((static_cast<int64_t>(KEYS ? mine.nk : mine.nq * a.G) + PER - 1) / PER), upto = wave_scan(n);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(upto > left);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      *s = lane_seq(mine, l);
      *tile = left - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
      return true;
    }
    left -= __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// ------------------------------------------------------------------------------ many rows
// The rows [r0, end) of a sequence and key head (128 at most, four waves of 32) over the key tiles [jb, je) of 64. LDS: two K
// slots and one V slot. Per tile t: S from K slot t % 2, a barrier, K tile t + 2 into that slot; the softmax; V tile
// t waited for and a barrier; O from the V slot; K tile t + 1 waited for, a barrier, V tile t + 1 into the V slot.
//
// Measured: 16384 tokens, 8 heads of 128: 497 us, 1105 TFLOP/s; 16381 in 12 prompts, 32 heads over 8: 443 us, 1058. Three waves share a SIMD; matrix units are busy
// 59% of cycles at the 1.75 GHz that the power limit leaves, vector units 61% (exp takes 40% of that), LDS 30%: no unit is full, what is missing is
// overlap within a SIMD (a library's plain product of 8192^3 runs at 1430 TFLOP/s here). 168 registers hold three waves without spills only
// with addresses made anew in the loop.
//
// NG = 2: eight waves, each four of them every second tile in slots of their own; join_groups adds the second's sums to the first's: for few long tiles,
// where a wave is alone on its SIMD (one prompt of 2000 tokens, 8 heads: 46.7 -> 35.7 us).
constexpr int kKeys = 64;      // of a tile
template <int D, int AHEAD, int NG>
__device__ __forceinline__ void rows_unit(const Args& a, lds_char* lds, const Seq& s, int kvh, int r0, int end, int jb, int je, Soft<D>& f) {
  constexpr int kTile = kKeys * Geo<D>::kRow, kLoads = Loader<D, kKeys, 4, kRows>::kLoads;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3, first = jb + (wave >> 2);
  const int n = (je - jb + NG - 1) / NG;                                           // tiles first + NG t; the second group's last may be tile je
  const int whole = min(max((sees(a, r0, s.nq, s.nk) / kKeys - first + NG - 1) / NG, 0), NG == 1 ? n : (je - first + 1) / 2);   // those that every row sees whole
  const int r = min(r0 + 32 * w + (lane & 31), end - 1), lim = NG == 1 ? sees(a, r, s.nq, s.nk) : min(sees(a, r, s.nq, s.nk), je * kKeys);
  const char* const kp = at(a.k, s.k0, kvh);
  const char* const vp = at(a.v, s.k0, kvh);
  lds += (wave >> 2) * 3 * kTile;
  lds_char* const vs = lds + 2 * kTile;
  const Loader<D, kKeys, 4, kRows> lk(w, lane, a.k.row);
  const Loader<D, kKeys, 4, kCols> lv(w, lane, a.v.row);
  // What follows from these is made anew where it is used: kept over the loop it spills, and a reload waits for all the tiles
  // in flight.
  const RowReads<D, kRows> rows(lane);
  const ColReads<D, kCols> cols(lane);
  auto issue_k = [&](int t) {
    const int key = (first + NG * t) * kKeys;
    lk.issue(kp + key * a.k.row, s.nk - key, lds + (t & 1) * kTile, w);
  };
  auto issue_v = [&](int t) {
    const int key = (first + NG * t) * kKeys;
    lv.issue(vp + key * a.v.row, s.nk - key, vs, w);
  };
  bf16x8 qf[D / 16];
  f.clear();
  if (n > 0) {
    issue_k(0);
    issue_v(0);
    if (n > 1) issue_k(1);
    // behind the tiles: 32 rows' pieces are 32 cache lines an instruction
    load_frags<D>(row_at(a, a.q, s, kvh, r), qf);
    wait_vm<0>();
    asm volatile("s_barrier" ::: "memory");
  }
  auto step = [&](int t, auto masked) {
    lds_char* const ks = lds + (t & 1) * kTile;
    const RowReads<D, kRows> rr = rows.fresh();
    f32x16 sc[2];
    zero(sc[0]);
    zero(sc[1]);
    fed<D / 8, AHEAD, D == 128>([&](int i) { return row_operand<D>(ks, i & 1, rr, i >> 1); }, [&](int i, bf16x8 v) { mma(sc[i & 1], v, qf[i >> 1]); });
    // every wave is done with K slot t % 2: K tile t + 2 goes there
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const bool k2 = t + 2 < n;
    if (k2) issue_k(t + 2);
    if constexpr (masked) {
      const int key = (first + NG * t) * kKeys;
      hide(sc[0], key, lim, here(lane) >> 5);
      hide(sc[1], key + 32, lim, here(lane) >> 5);
    }
    uint32_t pk[2][8];
    f.take(sc, a.scale_log2e, pk);
    // V tile t has landed in every wave's share (only K tile t + 2 may still be in flight)
    if (k2) wait_vm<kLoads>(); else wait_vm<0>();
    asm volatile("s_barrier" ::: "memory");
    const ColReads<D, kCols> rc = cols.fresh();
    const bf16x8 p[4] = {operand(pk[0], 0), operand(pk[0], 1), operand(pk[1], 0), operand(pk[1], 1)};
    fed<D / 8, AHEAD, D == 128>([&](int i) { return col_operand<D>(vs, i / (D / 32), rc, i % (D / 32)); },
                                [&](int i, bf16x8 v) { mma(f.o[i % (D / 32)], v, p[i / (D / 32)]); });
    if (t + 1 < n) {
      // K tile t + 1 has landed in every wave's share, and no wave reads the V slot any more
      if (k2) wait_vm<kLoads>(); else wait_vm<0>();
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      issue_v(t + 1);
    }
  };
  // The groups are one barrier apart: one's softmax goes with the other's products.
  if (NG == 2 && n > 0 && wave >= 4) asm volatile("s_barrier" ::: "memory");
  int t = 0;
  for (; t < whole; ++t) step(t, std::false_type());
  for (; t < n; ++t) step(t, std::true_type());
  if (NG == 2 && n > 0 && wave < 4) asm volatile("s_barrier" ::: "memory");
}

// The sums of waves 4 to 7 into those of waves 0 to 3, through LDS that nobody reads any more behind the barrier (4 D 128 bytes and 2048).
template <int D>
__device__ __forceinline__ void join_groups(lds_char* lds, Soft<D>& f) {
  typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
  typedef __attribute__((address_space(3))) f32x2_t lds_f32x2;
  const int lane = here(threadIdx.x & 63), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3;
  lds_char* const o = lds + w * D * 128 + lane * 16;
  lds_char* const ml = lds + 4 * D * 128 + (w * 64 + lane) * 8;
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  if (wave >= 4) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(lds_f32x4*)(o + (db * 4 + g) * 1024) = f32x4{f.o[db][4 * g], f.o[db][4 * g + 1], f.o[db][4 * g + 2], f.o[db][4 * g + 3]};
    *(lds_f32x2*)ml = f32x2_t{f.m, f.l};
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  if (wave >= 4) return;
  const f32x2_t other = *(const lds_f32x2*)ml;
  const float m = fmaxf(f.m, other.x), was = __builtin_amdgcn_exp2f(f.m - m), is = __builtin_amdgcn_exp2f(other.x - m);
  f.m = m;
  f.l = __builtin_fmaf(other.y, is, f.l * was);
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 v = *(const lds_f32x4*)(o + (db * 4 + g) * 1024);
#pragma unroll
      for (int e = 0; e < 4; ++e) f.o[db][4 * g + e] = __builtin_fmaf(v[e], is, f.o[db][4 * g + e] * was);
    }
}

// 32 rows of a sequence and key head from r0 are done, those before `end` of them; `mine`: LDS of the wave's own for whole rows, or NULL.
template <int D>
__device__ __forceinline__ void finish(const Args& a, const Seq& s, int kvh, int r0, int end, const Soft<D>& f, lds_char* mine = nullptr) {
  const int lane = here(threadIdx.x & 63), r = r0 + (lane & 31), qi = query_of(a, min(r, end - 1)), h = kvh * a.G + (min(r, end - 1) - qi * a.G);
  if (mine) store_rows<D>(mine, f.o, f.inverse(), [&](int i) { return r0 + i < end ? row_at(a, a.o, s, kvh, r0 + i) : nullptr; });
  else store_row<D>(at(a.o, s.q0 + qi, h), f.o, f.inverse(), r < end);
  if (a.lse && lane < 32 && r < end) a.lse[static_cast<int64_t>(h) * a.Tq + s.q0 + qi] = f.lse();
}

// A row's part over some of its keys: its sums relative to its maximum, and that with the sum of the weights.
template <int D>
__device__ __forceinline__ void leave_part(const Args& a, int64_t at, const Soft<D>& f) {
  const int up = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(a.part_o + at * D + 32 * db + 8 * g + 4 * up) =
          f32x4{f.o[db][4 * g], f.o[db][4 * g + 1], f.o[db][4 * g + 2], f.o[db][4 * g + 3]};
  if (up == 0) *reinterpret_cast<f32x2_t*>(a.part_ml + at * 2) = f32x2_t{f.m, f.l};
}

// The same of all 128 rows of a workgroup's slot, each lane's accumulators in its own pieces: whole lines. Without a tile only that the
// weights' sum is 0.
template <int D>
__device__ __forceinline__ void leave_whole(const Args& a, int64_t slot, const Soft<D>& f, bool any) {
  const int lane = here(threadIdx.x & 63), w = threadIdx.x >> 6;
  f32x4* const part = reinterpret_cast<f32x4*>(a.part_o) + (slot * 4 + w) * (D * 8) + lane;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; any && g < 4; ++g) part[(db * 4 + g) * 64] = f32x4{f.o[db][4 * g], f.o[db][4 * g + 1], f.o[db][4 * g + 2], f.o[db][4 * g + 3]};
  if (lane < 32) *reinterpret_cast<f32x2_t*>(a.part_ml + (slot * 128 + 32 * w + lane) * 2) = f32x2_t{f.m, f.l};
}

template <int D, int NG>
__global__ __launch_bounds__(256 * NG, NG == 2 ? (D == 128 ? 2 : 4) : (D == 128 ? 3 : 4)) void rows_kernel(Args a) {
  __shared__ __attribute__((aligned(16))) char lds[NG * 3 * kKeys * Geo<D>::kRow];
  Seq s;
  int kvh, tile;
  if (!tile_of<128>(a, &s, &kvh, &tile)) return;
  const int R = s.nq * a.G, r0 = ((R + 127) / 128 - 1 - tile) * 128, end = min(r0 + 128, R);       // the longest rows first
  Soft<D> f;
  rows_unit<D, 2, NG>(a, (lds_char*)lds, s, kvh, r0, end, 0, (sees(a, end - 1, s.nq, s.nk) + kKeys - 1) / kKeys, f);
  if constexpr (NG == 2) join_groups<D>((lds_char*)lds, f);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // no wave reads the K slots any more, or what the others have left of this one's sums
  if (w < 4 && r0 + 32 * w < end) finish<D>(a, s, kvh, r0 + 32 * w, end, f, (lds_char*)lds + w * (NG == 2 ? D * 128 : 32 * Geo<D>::kRow));
}

// ------------------------------------------------------------------------------ keys dealt out
// Where the rows alone do not fill the chip their keys are dealt out too: all work is laid end to end, as units of rows
// of one key head times the keys these see, and cut into ranges of the same length, wherever units begin and
// end. A unit that lies in one range is finished there; of the others each range leaves a part: in its slot 0 of
// the unit that it begins in or with, in slot 1 of one that begins later. A second launch adds them in order.
//
// Wide units, for sequences of many rows: as many queries as make 128 rows at most, in keys, behind them kStart keys for
// what a unit takes besides its tiles (chunks of 61 tokens over 7 caches, some of them short: 45 us without). A workgroup a range: it takes the
// tiles of 64 keys that begin in it. Measured: those chunks, 32 heads over 8, 7900 keys: 23 to 24 us, 10 of them a workgroup's start and end, and 10 to join; the
// parts are 28 MB written and read, as much as the caches.
struct Wide {
  static constexpr int kStart = 256;
  static constexpr int kLeast = 384;          // of a range (256 to 768 measured: the parts against the ranges)
  static __device__ __forceinline__ int queries(const Args& a) { return a.G < 128 ? a.shift >= 0 ? 128 >> a.shift : 128 / a.G : 1; }
  static __device__ __forceinline__ int units(const Args& a, const Seq& s) { return (s.nq + queries(a) - 1) / queries(a); }
  // length of the units before unit b: the keys that its last query sees, one where that sees none, and kStart
  static __device__ __forceinline__ int64_t before(const Args& a, const Seq& s, int b) {
    if (!a.causal) return static_cast<int64_t>(b) * (max(1, s.nk) + kStart);
    const int n = queries(a), off = s.nk - s.nq, full = min(b, units(a, s) - 1);
    const int none = off < 0 ? min(full, -off / n) : 0;
    int64_t v = static_cast<int64_t>(b) * kStart + none + static_cast<int64_t>(full - none) * off + n * ((static_cast<int64_t>(full) * (full + 1) - static_cast<int64_t>(none) * (none + 1)) / 2);
    if (b > full) v += max(1, s.nk);
    return v;
  }
  static __device__ __forceinline__ int64_t of_head(const Args& a, const Seq& s) { return before(a, s, units(a, s)); }
  static __device__ __forceinline__ int64_t work(const Args& a, const Seq& s) { return s.nq > 0 ? of_head(a, s) * a.Hkv : 0; }
  static __device__ __forceinline__ int64_t length(int64_t total, int64_t n) { return max(static_cast<int64_t>(kLeast), quot(total + n - 1, n)); }
};

// Narrow units, for a few rows: 32 of them, in tiles of 32 keys, a wave a range. Up to four key heads are side by side: waves of
// one workgroup take the same tiles of theirs, which lie side by side in memory too where a token's heads do. Bound by memory: 32 requests, 39,400
// keys of 8 heads, 162 MB: 31 to 35 us, 4.6 to 5.3 TB/s (a large copy: 4.9), and 6.5 to join.
struct Narrow {
  static constexpr int kRows = 32;
  static constexpr int kLeast = 2;             // tiles of a range (1 to 8 measured: with 1 the join takes longer than the ranges)
  static __device__ __forceinline__ int tiles(const Seq& s) { return max(1, (s.nk + 31) >> 5); }
  static __device__ __forceinline__ int side(const Args& a) { return a.Hkv % 4 == 0 ? 4 : a.Hkv % 2 == 0 ? 2 : 1; }
  static __device__ __forceinline__ int64_t work(const Args& a, const Seq& s) {
    return static_cast<int64_t>((s.nq * a.G + 31) / 32) * (a.Hkv / side(a)) * tiles(s);
  }
  static __device__ __forceinline__ int64_t length(int64_t total, int64_t n) { return max(static_cast<int64_t>(kLeast), quot(total + n - 1, n)); }
  static __device__ __forceinline__ void row(const Args& a, const Seq& s, int64_t x, int* kvh, int* r, int* i, int64_t* u0) {
    const int b = static_cast<int>(quot(x, 32 * static_cast<int64_t>(a.Hkv))), n = min(32, s.nq * a.G - 32 * b);
    const int in = static_cast<int>(x - static_cast<int64_t>(b) * 32 * a.Hkv);
    *kvh = in / n;
    *i = in - *kvh * n;
    *r = 32 * b + *i;
    *u0 = (static_cast<int64_t>(b) * (a.Hkv / side(a)) + *kvh / side(a)) * tiles(s);
  }
};

// The sequences laid end to end, one a lane, 64 at a time; the first 64 are kept.
template <class U>
struct Line {
  Seq mine;
  int64_t n, upto, total;
  __device__ __forceinline__ explicit Line(const Args& a) {
    const int lane = threadIdx.x & 63;
    mine = seq_of(a, lane);
    n = U::work(a, mine);
    upto = wave_scan(n);
    total = lane64(upto, 63);
    for (int s0 = 64; s0 < a.n_seq; s0 += 64) total += lane64(wave_scan(U::work(a, seq_of(a, s0 + lane))), 63);
  }
  // The sequence in which u (less than total) lies, and u's place in it.
  __device__ __forceinline__ Seq find(const Args& a, int64_t u, int64_t* in) const {
    Seq m = mine;
    int64_t nn = n, up = upto;
    for (int s0 = 0;;) {
      const uint64_t hit = __builtin_amdgcn_ballot_w64(up > u);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        *in = u - lane64(up - nn, l);
        return lane_seq(m, l);
      }
      u -= lane64(up, 63);
      s0 += 64;
      m = seq_of(a, s0 + (threadIdx.x & 63));
      nn = U::work(a, m);
      up = wave_scan(nn);
    }
  }
};

// The range of workgroup b of n, of `used` ranges that are not empty: those side by side lie on one XCD, whose L2 then holds what they
// share, and every XCD has as many.
__device__ __forceinline__ int64_t range_of_block(int b, int n, int64_t used) {
  if (n % 8) return b;
  const int64_t each = (used + 7) / 8;
  return b / 8 < each ? b % 8 * each + b / 8 : used;
}

template <int D>
__global__ __launch_bounds__(256, 2) void wide_kernel(Args a) {
  __shared__ __attribute__((aligned(16))) char lds[3 * kKeys * Geo<D>::kRow];
  const Line<Wide> line(a);
  const int64_t per = Wide::length(line.total, gridDim.x), W = range_of_block(blockIdx.x, gridDim.x, quot(line.total + per - 1, per));
  const int64_t begin = W * per, end = min(begin + per, line.total);
  for (int64_t u = begin; u < end;) {
    int64_t in;
    const Seq s = line.find(a, u, &in);
    const int64_t head = Wide::of_head(a, s);
    const int kvh = static_cast<int>(quot(in, head));
    in -= kvh * head;
    int lo = 0, hi = Wide::units(a, s) - 1;                     // the unit with before(unit) <= in < before(unit + 1)
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (Wide::before(a, s, mid + 1) > in) hi = mid;
      else lo = mid + 1;
    }
    const int64_t b0 = Wide::before(a, s, lo), b1 = Wide::before(a, s, lo + 1);
    const int first = static_cast<int>(in - b0), last = static_cast<int>(min(b1 - b0, first + (end - u)));
    const int rows = Wide::queries(a) * a.G, r0 = lo * rows, r_end = min(r0 + rows, s.nq * a.G);
    Soft<D> f;
    // the last unit's reads of these slots are done
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int jb = (first + kKeys - 1) / kKeys, je = (min(last, sees(a, r_end - 1, s.nq, s.nk)) + kKeys - 1) / kKeys;
    rows_unit<D, 4, 1>(a, (lds_char*)lds, s, kvh, r0, r_end, jb, je, f);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (first != 0 || last != b1 - b0) leave_whole<D>(a, W * 2 + (u > begin), f, jb < je);
    else if (r0 + 32 * w < r_end) finish<D>(a, s, kvh, r0 + 32 * w, r_end, f, (lds_char*)lds + w * 32 * Geo<D>::kRow);
    u += last - first;
  }
}

// A wave's key tiles [first, stop), every step-th, of 32 rows. It has a slot of K and one of V to itself and waits for
// nobody: K tile j + 1 is on its way from the time the scores are there, V tile j + 1 from the end of the second product.
template <int D>
__device__ __forceinline__ void narrow_unit(const Args& a, lds_char* mine, const Seq& s, int kvh, int r0, int first, int stop, int step, Soft<D>& f) {
  using Lk = Loader<D, 32, 1, kRows>;
  using Lv = Loader<D, 32, 1, kCols>;
  constexpr int kTile = 32 * Geo<D>::kRow;
  const int lane = threadIdx.x & 63, R = s.nq * a.G, r = min(r0 + (lane & 31), R - 1);
  const int lim = sees(a, r, s.nq, s.nk), all = sees(a, r0, s.nq, s.nk);
  const char* const kp = at(a.k, s.k0, kvh);
  const char* const vp = at(a.v, s.k0, kvh);
  lds_char* const vs = mine + kTile;
  const Lk lk(0, lane, a.k.row);
  const Lv lv(0, lane, a.v.row);
  auto issue_k = [&](int j) { lk.issue(kp + static_cast<int64_t>(j) * 32 * a.k.row, s.nk - j * 32, mine, 0); };
  auto issue_v = [&](int j) { lv.issue(vp + static_cast<int64_t>(j) * 32 * a.v.row, s.nk - j * 32, vs, 0); };
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");            // the last unit's reads of these slots are done
  if (first < stop) {
    issue_k(first);
    issue_v(first);
  }
  bf16x8 qf[D / 16];
  load_frags<D>(row_at(a, a.q, s, kvh, r), qf);
  const RowReads<D, kRows> rr(lane);
  const ColReads<D, kCols> rc(lane);
  f.clear();
  for (int j = first; j < stop; j += step) {
    const bool more = j + step < stop;
    wait_vm<Lv::kLoads>();                                       // K tile j (V tile j may still be in flight)
    f32x16 sc[1];
    zero(sc[0]);
    fed<D / 16, 4, D == 128>([&](int i) { return row_operand<D>(mine, 0, rr, i); }, [&](int i, bf16x8 v) { mma(sc[0], v, qf[i]); });
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) issue_k(j + step);
    if (j * 32 + 32 > all) hide(sc[0], j * 32, lim, lane >> 5);
    uint32_t pk[1][8];
    f.take(sc, a.scale_log2e, pk);
    if (more) wait_vm<Lk::kLoads>(); else wait_vm<0>();          // V tile j
    const bf16x8 p[2] = {operand(pk[0], 0), operand(pk[0], 1)};
    fed<D / 16, 4, D == 128>([&](int i) { return col_operand<D>(vs, i / (D / 32), rc, i % (D / 32)); },
                    [&](int i, bf16x8 v) { mma(f.o[i % (D / 32)], v, p[i / (D / 32)]); });
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) issue_v(j + step);
  }
}

template <int D>
__global__ __launch_bounds__(256, 2) void narrow_kernel(Args a) {
  __shared__ __attribute__((aligned(16))) char lds[4 * 2 * 32 * Geo<D>::kRow];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), side = Narrow::side(a), sub = wv % side;
  lds_char* const mine = (lds_char*)lds + wv * 2 * 32 * Geo<D>::kRow;
  const Line<Narrow> line(a);
  const int64_t W = static_cast<int64_t>(blockIdx.x) * (4 / side) + wv / side;
  const int64_t per = Narrow::length(line.total, static_cast<int64_t>(gridDim.x) * (4 / side)), begin = W * per, end = min(begin + per, line.total);
  for (int64_t u = begin; u < end;) {
    int64_t in;
    const Seq s = line.find(a, u, &in);
    const int L = Narrow::tiles(s);
    const int64_t unit = quot(in, L);
    const int64_t block = quot(unit, a.Hkv / side);
    const int first = static_cast<int>(in - unit * L), last = static_cast<int>(min(static_cast<int64_t>(L), first + (end - u)));
    const int kvh = static_cast<int>(unit - block * (a.Hkv / side)) * side + sub, r0 = static_cast<int>(block) * 32, R = s.nq * a.G;
    Soft<D> f;
    narrow_unit<D>(a, mine, s, kvh, r0, first, min(last, (sees(a, min(r0 + 31, R - 1), s.nq, s.nk) + 31) / 32), 1, f);
    const int i = here(threadIdx.x & 31);
    if (first == 0 && last == L) finish<D>(a, s, kvh, r0, R, f);
    else if (r0 + i < R) leave_part<D>(a, ((W * side + sub) * 2 + (u > begin)) * Narrow::kRows + i, f);
    u += last - first;
  }
}

// The b-th of all things, `things(s)` in sequence s: its sequence, its number there, and U's work before the sequence and in all.
// False past the last.
template <class U, class Things>
__device__ __forceinline__ bool locate(const Args& a, const Things& things, int64_t b, Seq* s, int64_t* in, int64_t* before, int64_t* total) {
  bool found = false;
  *total = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    const Seq mine = seq_of(a, s0 + (threadIdx.x & 63));
    const int64_t work = U::work(a, mine), w_upto = wave_scan(work), n = things(mine), upto = wave_scan(n);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(upto > b);
    if (!found && hit) {
      const int l = __builtin_ctzll(hit);
      found = true;
      *in = b - lane64(upto - n, l);
      *before = *total + lane64(w_upto - work, l);
      *s = lane_seq(mine, l);
    } else if (!found) {
      b -= lane64(upto, 63);
    }
    *total += lane64(w_upto, 63);
  }
  return found;
}

__device__ __forceinline__ void store_joined(const Args& a, const Seq& s, int kvh, int r, int col, const f32x4& o, float top, float sum) {
  const int qi = query_of(a, r), h = kvh * a.G + (r - qi * a.G);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  *reinterpret_cast<u32x2*>(at(a.o, s.q0 + qi, h) + col * 2) = u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
  if (a.lse && col == 0) a.lse[static_cast<int64_t>(h) * a.Tq + s.q0 + qi] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Wide units: a wave takes 32 rows' 32 columns over the parts in turn, its lanes as they left them.
template <int D>
__global__ __launch_bounds__(256) void join_wide_kernel(Args a, int64_t ranges) {
  const int lane = threadIdx.x & 63, up = lane >> 5;
  const int64_t id = block_number() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = static_cast<int>(id % (D / 8)), w = part / (D / 32), db = part % (D / 32);
  Seq s;
  int64_t in, before, total;
  if (!locate<Wide>(a, [&](const Seq& x) { return static_cast<int64_t>(Wide::units(a, x)) * a.Hkv; }, id / (D / 8), &s, &in, &before, &total)) return;
  const int units = Wide::units(a, s), kvh = static_cast<int>(quot(in, units)), b = static_cast<int>(in - static_cast<int64_t>(kvh) * units);
  const int per_unit = Wide::queries(a) * a.G, r0 = b * per_unit + 32 * w, end = min(b * per_unit + per_unit, s.nq * a.G);
  if (r0 >= end) return;
  before += kvh * Wide::of_head(a, s);
  const int64_t u0 = before + Wide::before(a, s, b), u1 = before + Wide::before(a, s, b + 1);
  const int64_t per = Wide::length(total, ranges), w0 = quot(u0, per), w1 = quot(u1 - 1, per);
  if (w0 == w1) return;                                       // finished by its range
  float top = -FLT_MAX, sum = 0.f;
  f32x4 o[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) o[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int64_t x = w0; x <= w1; ++x) {
    const int64_t slot = x * 2 + (x == w0 && u0 > w0 * per);
    const f32x4* const from = reinterpret_cast<const f32x4*>(a.part_o) + ((slot * 4 + w) * (D / 32) + db) * 256 + lane;
    const f32x2_t ml = *reinterpret_cast<const f32x2_t*>(a.part_ml + (slot * 128 + 32 * w + (lane & 31)) * 2);
    f32x4 v[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      v[g] = from[g * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[g][e] = ml.y == 0.f ? 0.f : v[g][e];       // not written
    }
    const float m = fmaxf(top, ml.x), was = __builtin_amdgcn_exp2f(top - m), is = __builtin_amdgcn_exp2f(ml.x - m);
    top = m;
    sum = __builtin_fmaf(ml.y, is, sum * was);
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[g][e] = __builtin_fmaf(v[g][e], is, o[g][e] * was);
  }
  const int r = min(r0 + (lane & 31), end - 1), qi = query_of(a, r), h = kvh * a.G + (r - qi * a.G);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  char* const to = at(a.o, s.q0 + qi, h) + 64 * db;
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    const auto pack = [&](const f32x4& v) { return u32x2{pack_bf16x2(v[0] * inv, v[1] * inv), pack_bf16x2(v[2] * inv, v[3] * inv)}; };
    const u32x4 v = columns8(pack(o[g]), pack(o[g + 1]));
    if (r0 + (lane & 31) < end) *reinterpret_cast<u32x4*>(to + 16 * (g + up)) = v;
  }
  if (a.lse && db == 0 && lane < 32 && r0 + lane < end)
    a.lse[static_cast<int64_t>(h) * a.Tq + s.q0 + qi] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Narrow units: a workgroup a row, D / 4 lanes a part, 16 parts at once in each wave (a request's next token has a few rows, and their
// parts are many).
// Where the rows are many, and most of them finished, a wave a row (60 sequences of 30 tokens, 8 heads: 29 us otherwise).
template <int D, bool WAVE>
__global__ __launch_bounds__(256) void join_narrow_kernel(Args a, int64_t ranges) {
  constexpr int kLanes = D / 4, kParts = 64 / kLanes, kOnce = 16 / kParts;
  __shared__ __attribute__((aligned(16))) f32x4 waves[4][kLanes];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), side = Narrow::side(a);
  Seq s;
  int64_t in, before, total;
  if (!locate<Narrow>(a, [&](const Seq& x) { return static_cast<int64_t>(x.nq) * a.H; },
                      WAVE ? block_number() * 4 + wv : block_number(), &s, &in, &before, &total))
    return;
  int kvh, r, i;
  int64_t u0;
  Narrow::row(a, s, in, &kvh, &r, &i, &u0);
  u0 += before;
  const int64_t per = Narrow::length(total, ranges), w0 = quot(u0, per), w1 = quot(u0 + Narrow::tiles(s) - 1, per);
  if (w0 == w1) return;                                       // finished by its range
  const auto part = [&](int64_t w) { return ((w * side + kvh % side) * 2 + (w == w0 && u0 > w0 * per)) * Narrow::kRows + i; };
  const auto weight = [&](int64_t w) {                        // maximum and sum of part w, none past the last
    return w <= w1 ? *reinterpret_cast<const f32x2_t*>(a.part_ml + part(w) * 2) : f32x2_t{-FLT_MAX, 0.f};
  };
  float top = -FLT_MAX;
  for (int64_t w = w0; w <= w1; w += 64) top = fmaxf(top, weight(w + lane).x);
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  float sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const int grp = lane / kLanes, col = lane % kLanes * 4;
  for (int64_t w = w0; w <= w1; w += 64) {
    const f32x2_t ml = weight(w + lane);
    const float c = w + lane <= w1 ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
    sum = __builtin_fmaf(ml.y, c, sum);
    const int n = static_cast<int>(min(w1 - w + 1, static_cast<int64_t>(64)));
    for (int p = WAVE ? 0 : 16 * wv; p < n; p += WAVE ? 16 : 64) {
      f32x4 v[kOnce];
#pragma unroll
      for (int q = 0; q < kOnce; ++q) v[q] = *reinterpret_cast<const f32x4*>(a.part_o + part(w + min(p + q * kParts + grp, n - 1)) * D + col);
#pragma unroll
      for (int q = 0; q < kOnce; ++q) {
        const float cq = __shfl(c, p + q * kParts + grp);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(v[q][e], cq, o[e]);
      }
    }
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
#pragma unroll
  for (int d = kLanes; d < 64; d <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], d);
  if constexpr (!WAVE) {
    if (grp == 0) waves[wv][lane] = o;
    __syncthreads();
    if (wv) return;
  }
  if (grp) return;
  if constexpr (!WAVE) {
#pragma unroll
    for (int w = 1; w < 4; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += waves[w][lane][e];
  }
  store_joined(a, s, kvh, r, col, o, top, sum);
}

// Short caches and prompts: a workgroup a narrow unit, its eight waves each an eighth of the key tiles, added up in LDS: no second launch. One request's next token
// over 80 keys: 4 us, a chain of dependent loads (starts, keys, result); 1024 keys 9.6.
template <int D>
__global__ __launch_bounds__(512, 2) void short_kernel(Args a) {
  constexpr int kMine = 2 * 32 * Geo<D>::kRow;                  // a wave's slots: also 32 rows of D sums
  __shared__ __attribute__((aligned(16))) char lds[8 * kMine];
  __shared__ f32x2_t ml[8][32];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, up = lane >> 5;
  Seq s;
  int kvh, tile;
  if (!tile_of<32>(a, &s, &kvh, &tile)) return;
  const int R = s.nq * a.G, r0 = tile * 32, tiles = (sees(a, min(r0 + 31, R - 1), s.nq, s.nk) + 31) / 32;
  Soft<D> f;
  narrow_unit<D>(a, (lds_char*)lds + wv * kMine, s, kvh, r0, wv, tiles, 8, f);
  const int waves = min(8, max(1, tiles)), rows = min(32, R - r0);
  if (waves == 1) {
    if (wv == 0) finish<D>(a, s, kvh, r0, R, f);
    return;
  }
  // row i of a wave's sums: pieces of four columns, piece p at p ^ i
  if (wv < waves) {
    const int i = lane & 31;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(lds + wv * kMine + i * D * 4 + (((8 * db + 2 * g + up) ^ i % (D / 4)) << 4)) =
            f32x4{f.o[db][4 * g], f.o[db][4 * g + 1], f.o[db][4 * g + 2], f.o[db][4 * g + 3]};
    if (up == 0) ml[wv][i] = f32x2_t{f.m, f.l};
  }
  __syncthreads();
  constexpr int kLanes = D / 4;
  const int col = threadIdx.x % kLanes;
  for (int i = threadIdx.x / kLanes; i < rows; i += 512 / kLanes) {
    float top = -FLT_MAX, sum = 0.f;
    for (int w = 0; w < waves; ++w) top = fmaxf(top, ml[w][i].x);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < waves; ++w) {
      const float c = __builtin_amdgcn_exp2f(ml[w][i].x - top);
      sum = __builtin_fmaf(ml[w][i].y, c, sum);
      const f32x4 v = *reinterpret_cast<const f32x4*>(lds + w * kMine + i * D * 4 + ((col ^ i % kLanes) << 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(v[e], c, o[e]);
    }
    store_joined(a, s, kvh, r0 + i, 4 * col, o, top, sum);
  }
}

// ------------------------------------------------------------------------------ gradients
// dq: as rows_kernel, with a second product (V times the row's do) and dS in place of the probabilities, K and V tiles in two slots each, one
// barrier a tile. It computes delta for its rows and leaves it, and lse in powers of two, for the kernel below. 8192 tokens in 4 documents, 32 heads over 8: 282 to
// 301 us, 1010 to 1075 TFLOP/s; matrix units busy 55% of cycles at 1.8 GHz, vector units 43%.
//
// delta = do . o takes o's roundings (of the probabilities and of o itself) to every dS of the row alike, a
// relative error of dq and dk of about 0.0023 / sqrt(keys that share the weight): nothing beside the 0.0017 that dS's own
// rounding gives where a row sees many keys, and the larger part where it sees ten. Tiles that see at most
// kExactTiles tiles of keys therefore take delta = sum_j P_ij (do_i . v_j) in a pass before.
constexpr int kExactTiles = 4;
template <int D, int NG>
__global__ __launch_bounds__(256 * NG, 2) void dq_kernel(Args a) {
  using G = Geo<D>;
  constexpr int kBKV = 64, kTile = kBKV * G::kRow;
  __shared__ __attribute__((aligned(16))) char lds_raw[NG * 4 * kTile];
  __shared__ float deltas[NG][128];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3, group = wave >> 2, up = lane >> 5;
  lds_char* const lds = (lds_char*)lds_raw + group * 4 * kTile;
  Seq s;
  int kvh, tile;
  if (!tile_of<128>(a, &s, &kvh, &tile)) return;
  const int nq = s.nq, nk = s.nk, R = nq * a.G, r0 = ((R + 127) / 128 - 1 - tile) * 128, end = min(r0 + 128, R);
  const int nkv = (sees(a, end - 1, nq, nk) + kBKV - 1) / kBKV, n = (nkv + NG - 1) / NG;      // the group's tiles are group + NG t
  const int w0 = r0 + 32 * w;
  const int all = w0 < R ? sees(a, w0, nq, nk) : 0, any = w0 < R ? sees(a, min(w0 + 31, R - 1), nq, nk) : 0;
  const int r = min(w0 + (lane & 31), R - 1), qi = query_of(a, r), h = kvh * a.G + (r - qi * a.G), lim = sees(a, r, nq, nk);
  const RowReads<D, kBoth> rk(lane);
  const ColReads<D, kBoth> ck(lane);
  const RowReads<D, kRows> rv(lane);
  const Loader<D, kBKV, 4, kBoth> lk(w, lane, a.k.row);
  const Loader<D, kBKV, 4, kRows> lv(w, lane, a.v.row);
  const char* const kp = at(a.k, s.k0, kvh);
  const char* const vp = at(a.v, s.k0, kvh);
  auto issue = [&](int t, int slot) {
    const int key = (group + NG * t) * kBKV;
    lk.issue(kp + key * a.k.row, nk - key, lds + slot * kTile, w);
    lv.issue(vp + key * a.v.row, nk - key, lds + (2 + slot) * kTile, w);
  };
  if (n > 0) issue(0, 0);
  bf16x8 qf[D / 16], df[D / 16];
  load_frags<D>(at(a.q, s.q0 + qi, h), qf);
  load_frags<D>(at(a.d_o, s.q0 + qi, h), df);
  const int64_t stat = static_cast<int64_t>(h) * a.Tq + s.q0 + qi;
  const float lse2 = lim > 0 ? a.lse[stat] * kLog2e : 0.f;
  int slot = 0;
  // a tile has landed in every wave's share, and no wave reads the tile before it any more; then `next` is loaded
  auto turn = [&](int next) {
    wait_vm<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    slot ^= 1;
    if (next < n) issue(next, slot);
  };
  float delta = 0.f;
  if (nkv <= kExactTiles) {
    for (int t = 0; t < n; ++t) {
      turn(t + 1 < n ? t + 1 : 0);
      const int key = (group + NG * t) * kBKV;
#pragma unroll 1
      for (int b = 0; b < 2 && key + 32 * b < any; ++b) {
        f32x16 sc = rows_product<D>(lds + (slot ^ 1) * kTile, b, rk, qf);
        const f32x16 dp = rows_product<D>(lds + (2 + (slot ^ 1)) * kTile, b, rv, df);
        hide(sc, key + 32 * b, lim, up);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          delta = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], a.scale_log2e, -lse2)), dp[e], delta);
      }
    }
    delta = add_halves(delta);
    if constexpr (NG == 2) {
      if (up == 0) deltas[group][32 * w + lane] = delta;
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      delta = deltas[0][32 * w + (lane & 31)] + deltas[1][32 * w + (lane & 31)];
    }
  } else {
    bf16x8 of[D / 16];
    load_frags<D>(at(a.o, s.q0 + qi, h), of);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = __builtin_fmaf(static_cast<float>(df[kk][e]), static_cast<float>(of[kk][e]), delta);
    delta = add_halves(delta);
  }
  f32x16 acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;
  for (int t = 0; t < n; ++t) {
    turn(t + 1);
    const int key = (group + NG * t) * kBKV;
    if (key >= any) continue;                                // wave-uniform
    lds_char* const ks = lds + (slot ^ 1) * kTile;
    lds_char* const vs = lds + (2 + (slot ^ 1)) * kTile;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x16 sc, dp;
      zero(sc);
      zero(dp);
      fed<D / 8, 2, D == 128>([&](int i) { return i & 1 ? row_operand<D>(vs, b, rv, i >> 1) : row_operand<D>(ks, b, rk, i >> 1); },
                     [&](int i, bf16x8 v) { mma(i & 1 ? dp : sc, v, i & 1 ? df[i >> 1] : qf[i >> 1]); });
      if (key + 32 * b + 32 > all) hide(sc, key + 32 * b, lim, up);
      uint32_t pk[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[2 * e], a.scale_log2e, -lse2));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[2 * e + 1], a.scale_log2e, -lse2));
        pk[e] = pack_bf16x2(p0 * (dp[2 * e] - delta), p1 * (dp[2 * e + 1] - delta));
      }
      const bf16x8 ds[2] = {operand(pk, 0), operand(pk, 1)};
      fed<D / 16, 2, D == 128>([&](int i) { return col_operand<D>(ks, 2 * b + i / (D / 32), ck, i % (D / 32)); },
                      [&](int i, bf16x8 v) { mma(acc[i % (D / 32)], v, ds[i / (D / 32)]); });
    }
  }
  if (group == 0 && up == 0 && w0 + lane < R) {
    a.delta[stat] = delta;
    a.lse2[stat] = lse2;
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // no wave reads the tiles any more
  lds_char* const mine = (lds_char*)lds_raw + w * D * 128;
  if constexpr (NG == 2) {
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    if (group)
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(lds_f32x4*)(mine + ((db * 4 + g) * 64 + lane) * 16) = f32x4{acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]};
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (group) return;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 v = *(const lds_f32x4*)(mine + ((db * 4 + g) * 64 + lane) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[db][4 * g + e] += v[e];
      }
  }
  if (w0 < end) store_rows<D>(mine, acc, a.scale, [&](int i) { return w0 + i < end ? row_at(a, a.dq, s, kvh, w0 + i) : nullptr; });
}

// dq of few or short prompts, as short_kernel: a workgroup 32 rows, its eight waves each every eighth tile of 32 keys in a slot of K and one of V
// of their own, their sums added up in LDS. Rows that see at most 256 keys have one tile a wave, so that delta from P and dP takes no second pass.
// One prompt, 8 heads: 100 tokens 8 us, 1000 16, 2000 36 (by rows 11, 26, 43); a chain of dependent steps: two loads, two products, two barriers and a store take 7.
template <int D>
__global__ __launch_bounds__(512, 2) void dq_short_kernel(Args a) {
  using G = Geo<D>;
  using Lk = Loader<D, 32, 1, kBoth>;
  using Lv = Loader<D, 32, 1, kRows>;
  constexpr int kTile = 32 * G::kRow, kMine = 2 * kTile;        // a wave's slots: also 32 rows of D sums
  __shared__ __attribute__((aligned(16))) char lds[8 * kMine];
  __shared__ float deltas[8][32];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, up = lane >> 5;
  lds_char* const ks = (lds_char*)lds + wv * kMine;
  lds_char* const vs = ks + kTile;
  Seq s;
  int kvh, tile;
  if (!tile_of<32>(a, &s, &kvh, &tile)) return;
  const int R = s.nq * a.G, r0 = tile * 32, rows = min(32, R - r0), any = sees(a, r0 + rows - 1, s.nq, s.nk), all = sees(a, r0, s.nq, s.nk);
  const int tiles = (any + 31) / 32, r = min(r0 + (lane & 31), R - 1), qi = query_of(a, r), h = kvh * a.G + (r - qi * a.G), lim = sees(a, r, s.nq, s.nk);
  const char* const kp = at(a.k, s.k0, kvh);
  const char* const vp = at(a.v, s.k0, kvh);
  const Lk lk(0, lane, a.k.row);
  const Lv lv(0, lane, a.v.row);
  auto issue_k = [&](int j) { lk.issue(kp + static_cast<int64_t>(j) * 32 * a.k.row, s.nk - j * 32, ks, 0); };
  auto issue_v = [&](int j) { lv.issue(vp + static_cast<int64_t>(j) * 32 * a.v.row, s.nk - j * 32, vs, 0); };
  if (wv < tiles) {
    issue_k(wv);
    issue_v(wv);
  }
  bf16x8 qf[D / 16], df[D / 16];
  load_frags<D>(at(a.q, s.q0 + qi, h), qf);
  load_frags<D>(at(a.d_o, s.q0 + qi, h), df);
  const int64_t stat = static_cast<int64_t>(h) * a.Tq + s.q0 + qi;
  const float lse2 = lim > 0 ? a.lse[stat] * kLog2e : 0.f;
  const RowReads<D, kBoth> rk(lane);
  const ColReads<D, kBoth> ck(lane);
  const RowReads<D, kRows> rv(lane);
  f32x16 sc, dp, acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) zero(acc[db]);
  float delta = 0.f;
  // P of tile j into sc, and dP
  auto scores = [&](int j) {
    wait_vm<0>();
    zero(sc);
    zero(dp);
    fed<D / 8, 4, D == 128>([&](int i) { return i & 1 ? row_operand<D>(vs, 0, rv, i >> 1) : row_operand<D>(ks, 0, rk, i >> 1); },
                            [&](int i, bf16x8 v) { mma(i & 1 ? dp : sc, v, i & 1 ? df[i >> 1] : qf[i >> 1]); });
    if (j * 32 + 32 > all) hide(sc, j * 32, lim, up);
#pragma unroll
    for (int e = 0; e < 16; ++e) sc[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], a.scale_log2e, -lse2));
  };
  auto product = [&] {
    uint32_t pk[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) pk[e] = pack_bf16x2(sc[2 * e] * (dp[2 * e] - delta), sc[2 * e + 1] * (dp[2 * e + 1] - delta));
    const bf16x8 ds[2] = {operand(pk, 0), operand(pk, 1)};
    fed<D / 16, 4, D == 128>([&](int i) { return col_operand<D>(ks, i / (D / 32), ck, i % (D / 32)); },
                             [&](int i, bf16x8 v) { mma(acc[i % (D / 32)], v, ds[i / (D / 32)]); });
  };
  if (tiles <= 8) {
    if (wv < tiles) {
      scores(wv);
#pragma unroll
      for (int e = 0; e < 16; ++e) delta = __builtin_fmaf(sc[e], dp[e], delta);
      delta = add_halves(delta);
    }
    if (up == 0) deltas[wv][lane] = delta;
    __syncthreads();
    delta = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) delta += deltas[w][lane & 31];
    if (wv < tiles) product();
  } else {
    bf16x8 of[D / 16];
    load_frags<D>(at(a.o, s.q0 + qi, h), of);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = __builtin_fmaf(static_cast<float>(df[kk][e]), static_cast<float>(of[kk][e]), delta);
    delta = add_halves(delta);
    for (int j = wv; j < tiles; j += 8) {
      scores(j);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // V tile j has been read
      if (j + 8 < tiles) issue_v(j + 8);
      product();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (j + 8 < tiles) issue_k(j + 8);
    }
  }
  if (wv == 0 && lane < rows) {
    a.delta[stat] = delta;
    a.lse2[stat] = lse2;
  }
  // as in short_kernel
  const int waves = min(8, max(1, tiles));
  if (wv < waves) {
    const int i = lane & 31;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(lds + wv * kMine + i * D * 4 + (((8 * db + 2 * g + up) ^ i % (D / 4)) << 4)) =
            f32x4{acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]};
  }
  __syncthreads();
  constexpr int kLanes = D / 4;
  const int col = threadIdx.x % kLanes;
  for (int i = threadIdx.x / kLanes; i < rows; i += 512 / kLanes) {
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < waves; ++w) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(lds + w * kMine + i * D * 4 + ((col ^ i % kLanes) << 4));
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += v[e];
    }
    *reinterpret_cast<u32x2*>(row_at(a, a.dq, s, kvh, r0 + i) + col * 8) =
        u32x2{pack_bf16x2(o[0] * a.scale, o[1] * a.scale), pack_bf16x2(o[2] * a.scale, o[3] * a.scale)};
  }
}

// dk and dv: a workgroup holds 32 NW keys of a key head (NW waves of 32), their K and V fragments beside both
// results' accumulators in registers, and streams the rows that see them, 32 queries of one head at a time with do,
// lse and delta, two blocks ahead in three LDS slots. Two waves share a SIMD's registers: kStash of V's fragments lie in
// LDS. Queries past the end of the sequence are zeros with lse 0: P = 1, but do = 0 and dS = 1 (0 - 0).
//
// The same 8192 tokens: 390 to 417 us, 970 to 1035 TFLOP/s, and 28 to join (60 to 130 MB of parts). Matrix units are busy 48% of cycles, vector units 36%, LDS 34%: both waves of
// a SIMD wait at the same barrier. One wave a SIMD with all its registers, a block's products between the next one's softmax: 684 us, some 630 instructions a
// block at five cycles each; the softmax put between this kernel's own products: 495 us against 447 then.
//
// The first keys of a sequence have G times as many rows as it has queries, the last ones hardly any, and there are few key
// heads: key tiles dealt one to a workgroup leave the chip waiting for the longest (8192 tokens in 4 sequences, 32 heads
// over 8: 904 us). So the blocks of all key tiles, laid end to end, are dealt out evenly: workgroup W takes the blocks [W per,
// (W + 1) per). A key tile that lies in one range is finished there, of
// the others each workgroup leaves a part, in its slot 0 for the tile that its range begins in or with, in slot 1 for one that
// begins later; dkv_join_kernel adds them up in order.
constexpr int kTileStart = 3;    // what a key tile takes besides its blocks, in blocks: its length is theirs and these, which come first
constexpr int kLeast = 5;
// Length of a range: all dealt out over n workgroups, but kLeast + 4 at least (with less the parts take longer than the ranges are shorter), or as
// much as gives every CU one, kLeast at least (two documents of 300 and 200 tokens, 4 heads: 32 blocks 78 us, 8 27.6, 4 18; one of 17
// tokens: a tile each of 4 key heads in one range 20.5, in four 8).
__device__ __forceinline__ int64_t range_length(const Args& a, int64_t total, int64_t n) {
  return max(min(max(quot(total + a.cus - 1, a.cus), static_cast<int64_t>(kLeast)), static_cast<int64_t>(kLeast + 4)), quot(total + n - 1, n));
}

struct KeyTile {
  Seq s;
  int kvh, tile, per_head;      // key tile; blocks of 32 queries that see it
  int64_t place, blocks;        // the place searched for in the tile; its blocks of all heads of the group, behind kTileStart
};

// Blocks of one query head in a sequence's tiles of 32 NW keys before tile j: those whose first key every query sees have all
// ceil(nq / 32) (one where there is none: such keys' zeros are still written), from there on every tile has NW less.
template <int NW>
__device__ __forceinline__ int64_t blocks_before(const Args& a, const Seq& s, int64_t j) {
  const int64_t f = max(1, (s.nq + 31) / 32), c = (s.nk + 31) / 32, off = s.nk - s.nq;
  if (!a.causal) return j * f;
  const int64_t full = off > 0 ? (off + 32 * NW - 1) / (32 * NW) : 0;
  return j <= full ? j * f : full * f + (j - full) * c - NW / 2 * (j * (j - 1) - full * (full - 1));
}

__device__ __forceinline__ Seq key_seq(const Args& a, int s) {
  Seq x{0, 0, 0, 0};
  if (s >= a.n_seq) return x;
  const int q0 = a.q_start[s], q1 = a.q_start[s + 1], k0 = a.k_start[s], k1 = a.k_start[s + 1];
  if (q0 < 0 || q1 < q0 || q1 > a.Tq || k0 < 0 || k1 < k0 || k1 > a.Tk || k1 - k0 > a.max_k) {
    set_status(a.status, XS_EBADINPUT);
    return x;
  }
  return Seq{q0, q1 - q0, k0, k1 - k0};
}
template <int NW>
__device__ __forceinline__ int key_tiles(const Seq& s) { return (s.nk + 32 * NW - 1) / (32 * NW); }
// Length of a key head's tiles before tile j: their blocks of all heads of the group, and kTileStart for each.
template <int NW>
__device__ __forceinline__ int64_t length_before(const Args& a, const Seq& s, int64_t j) { return blocks_before<NW>(a, s, j) * a.G + j * kTileStart; }
template <int NW>
__device__ __forceinline__ int64_t length_of(const Args& a, const Seq& s) { return length_before<NW>(a, s, key_tiles<NW>(s)) * a.Hkv; }

template <int NW>
__device__ __forceinline__ int64_t whole_length(const Args& a) {
  int64_t total = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) total += lane64(wave_scan(length_of<NW>(a, key_seq(a, s0 + (threadIdx.x & 63)))), 63);
  return total;
}


// The key tile that place u of all lies in; u is less than the whole length.
template <int NW>
__device__ __forceinline__ void key_tile_at(const Args& a, int64_t u, KeyTile* out) {
  int64_t before = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    const Seq mine = key_seq(a, s0 + (threadIdx.x & 63));
    const int64_t n = length_of<NW>(a, mine), upto = wave_scan(n);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(before + upto > u);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      out->s = lane_seq(mine, l);
      const int tiles = key_tiles<NW>(out->s);
      const int64_t head = length_before<NW>(a, out->s, tiles), in = u - before - lane64(upto - n, l);
      out->kvh = static_cast<int>(quot(in, head));
      const int64_t x = in - out->kvh * head;
      int lo = 0, hi = tiles - 1;                               // the tile with before(tile) <= x < before(tile + 1)
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (length_before<NW>(a, out->s, mid + 1) > x) hi = mid;
        else lo = mid + 1;
      }
      out->tile = lo;
      out->per_head = static_cast<int>(blocks_before<NW>(a, out->s, lo + 1) - blocks_before<NW>(a, out->s, lo));
      out->blocks = static_cast<int64_t>(out->per_head) * a.G;
      out->place = x - length_before<NW>(a, out->s, lo);
      return;
    }
    before += lane64(upto, 63);
  }
}

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, D == 128 ? 8 / NW : 12 / NW) void dkv_kernel(Args a) {
  using G = Geo<D>;
  constexpr int kBQ = 32, kTile = kBQ * G::kRow, kStages = 3, kStash = D == 128 ? 6 : 0;
  constexpr int kLoads = 2 * Loader<D, kBQ, NW, kBoth>::kLoads;                 // of a stage, a wave's (without lse and delta)
  __shared__ __attribute__((aligned(16))) char lds_raw[2 * kStages * kTile + 2 * kStages * kBQ * 4 + NW * kStash * 1024];
  lds_char* const lds = (lds_char*)lds_raw;
  lds_char* const stats = lds + 2 * kStages * kTile;                           // lse and delta of each stage
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const RowReads<D, kBoth> rows(lane);
  const ColReads<D, kBoth> cols(lane);
  const Loader<D, kBQ, NW, kBoth> lq(w, lane, a.q.row), ld(w, lane, a.d_o.row);
  lds_char* const stash = stats + 2 * kStages * kBQ * 4 + w * kStash * 1024;
  const int64_t total = whole_length<NW>(a), per = range_length(a, total, gridDim.x);
  const int64_t W = range_of_block(blockIdx.x, gridDim.x, quot(total + per - 1, per)), begin = W * per, end = min(begin + per, total);
  for (int64_t u = begin; u < end;) {
    KeyTile x;
    key_tile_at<NW>(a, u, &x);
    const int64_t from = max(x.place - kTileStart, static_cast<int64_t>(0)), step = min(x.blocks + kTileStart - x.place, end - u);
    const int n = static_cast<int>(x.place + step - kTileStart - from);       // blocks [from, from + n) of the tile
    if (n <= 0) {
      u += step;
      continue;
    }
    const int nq = x.s.nq, nk = x.s.nk, key0 = x.tile * 32 * NW, kw = key0 + 32 * w, off = nk - nq;
    const int first = a.causal ? max(0, key0 - off) : 0;       // the first query that sees one of these keys
    // the next block to load: its head in the group, first query and stage
    const int lg = static_cast<int>(quot(from, x.per_head));
    int lt = first + static_cast<int>(from - static_cast<int64_t>(lg) * x.per_head) * kBQ, lst = 0;
    int t = lt, st = 0;
    const char *pq = at(a.q, x.s.q0 + lt, x.kvh * a.G + lg), *pd = at(a.d_o, x.s.q0 + lt, x.kvh * a.G + lg);
    const float* ps = (w ? a.delta : a.lse2) + static_cast<int64_t>(x.kvh * a.G + lg) * a.Tq + x.s.q0 + lt;
    auto issue = [&] {
      lq.issue(pq, nq - lt, lds + 2 * lst * kTile, w);
      ld.issue(pd, nq - lt, lds + (2 * lst + 1) * kTile, w);
      // waves 0 and 1: the lower half's lanes fetch the 32 rows' numbers
      if (w < 2 && (here(lane) & 32) == 0) load_lds4(buffer_rsrc(ps, min(nq - lt, kBQ) * 4), here(lane) * 4, stats + (2 * lst + w) * kBQ * 4);
      lt += kBQ;
      if (lt < nq) {
        pq += kBQ * a.q.row;
        pd += kBQ * a.d_o.row;
        ps += kBQ;
      } else {                                                 // the next head's first query
        pq += a.q.head - (lt - kBQ - first) * a.q.row;
        pd += a.d_o.head - (lt - kBQ - first) * a.d_o.row;
        ps += a.Tq - (lt - kBQ - first);
        lt = first;
      }
      lst = lst + 1 == kStages ? 0 : lst + 1;
    };
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // the slots of the tile before have been read
    const bool some = nq > 0;
    if (some) issue();
    if (some && n > 1) issue();
    bf16x8 kf[D / 16], vf[D / 16];
    {
      const int kc = min(kw + (lane & 31), nk - 1);
      load_frags<D>(at(a.k, x.s.k0 + kc, x.kvh), kf);
      load_frags<D>(at(a.v, x.s.k0 + kc, x.kvh), vf);
      wait_vm<0>();                                            // here, or the loop waits for them, and so for the blocks in flight
    }
#pragma unroll
    for (int kk = 0; kk < kStash; ++kk) *(lds_bf16x8*)(stash + kk * 1024 + lane * 16) = vf[kk];
    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) dk[db][e] = dv[db][e] = 0.f;
    for (int i = 0; some && i < n; ++i) {
      // block i has landed in every wave's share (of block i + 1 nothing need have), and no wave reads block i - 1 any more
      if (i + 1 < n) wait_vm<kLoads>(); else wait_vm<0>();
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      if (i + 2 < n) issue();
      if (!a.causal || t + 31 + off >= kw) {                   // wave-uniform
        lds_char* const qs = lds + 2 * st * kTile;
        lds_char* const ds = qs + kTile;
        const int ln = here(lane);
        const RowReads<D, kBoth> rr = rows.fresh();
        f32x16 sc, dp;
        zero(sc);
        zero(dp);
        struct Pair {
          bf16x8 a, b;
        };
        fed<D / 8, 2, D == 128>([&](int i) {
                        Pair p;
                        p.a = row_operand<D>(i < D / 16 ? qs : ds, 0, rr, i % (D / 16));
                        const int kk = i - D / 16;
                        p.b = kk < 0 ? kf[i] : kk < kStash ? *(const lds_bf16x8*)(stash + kk * 1024 + ln * 16) : vf[kk];
                        return p;
                      },
                      [&](int i, const Pair& p) { mma(i < D / 16 ? sc : dp, p.a, p.b); });
        if (a.causal && t + off < kw + 31) {
          const int key = kw + (ln & 31);
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (t + entry_row(e, ln >> 5) + off < key) sc[e] = -INFINITY;
        }
        uint32_t pp[8], pd[8];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
          const lds_char* const at4 = stats + 2 * st * kBQ * 4 + (8 * g + 4 * (ln >> 5)) * 4;
          const f32x4 ls = *(const lds_f32x4*)at4, de = *(const lds_f32x4*)(at4 + kBQ * 4);
          float p[4], d[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * g + e], a.scale_log2e, -ls[e]));
            d[e] = p[e] * (dp[4 * g + e] - de[e]);
          }
          pp[2 * g] = pack_bf16x2(p[0], p[1]);
          pp[2 * g + 1] = pack_bf16x2(p[2], p[3]);
          pd[2 * g] = pack_bf16x2(d[0], d[1]);
          pd[2 * g + 1] = pack_bf16x2(d[2], d[3]);
        }
        const ColReads<D, kBoth> rc = cols.fresh();
        const bf16x8 po[2] = {operand(pp, 0), operand(pp, 1)}, so[2] = {operand(pd, 0), operand(pd, 1)};
        constexpr int kB = D / 32;                             // instruction i: 16 rows i / (2 kB), of dv, then dk, its block
        fed<4 * kB, 2, D == 128>([&](int i) { return col_operand<D>(i / kB % 2 ? qs : ds, i / (2 * kB), rc, i % kB); },
                       [&](int i, bf16x8 v) {
                         if (i / kB % 2) mma(dk[i % kB], v, so[i / (2 * kB)]);
                         else mma(dv[i % kB], v, po[i / (2 * kB)]);
                       });
      }
      t += kBQ;
      if (t >= nq) t = first;
      st = st + 1 == kStages ? 0 : st + 1;
    }
    const int key = kw + here(lane & 31);
    if (n == x.blocks) {
      const int kc = min(key, nk - 1);
      store_row<D>(at(a.dk, x.s.k0 + kc, x.kvh), dk, a.scale, key < nk);
      store_row<D>(at(a.dv, x.s.k0 + kc, x.kvh), dv, 1.f, key < nk);
    } else {
      f32x4* const part = reinterpret_cast<f32x4*>(a.part_o) + ((W * 2 + (u > begin)) * NW + w) * (D * 16) + here(lane);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          part[(db * 4 + g) * 64] = f32x4{dk[db][4 * g], dk[db][4 * g + 1], dk[db][4 * g + 2], dk[db][4 * g + 3]};
          part[(D / 8 + db * 4 + g) * 64] = f32x4{dv[db][4 * g], dv[db][4 * g + 1], dv[db][4 * g + 2], dv[db][4 * g + 3]};
        }
    }
    u += step;
  }
}

// A wave adds 32 columns of 32 keys' dk and dv over the parts, in the order of the ranges.
template <int D, int NW>
__global__ __launch_bounds__(256) void dkv_join_kernel(Args a, int n_ranges) {
  constexpr int kPieces = NW * (D / 32);              // waves of a key tile
  const int lane = threadIdx.x & 63, up = lane >> 5;
  const int64_t id = block_number() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int piece = static_cast<int>(id % kPieces), w = piece / (D / 32), db = piece % (D / 32);
  const int64_t number = quot(id / kPieces, a.Hkv);
  const int kvh = static_cast<int>(id / kPieces - number * a.Hkv);
  int64_t t = number, blocks = 0, total = 0;
  Seq s{0, 0, 0, 0};
  bool found = false;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    const Seq mine = key_seq(a, s0 + lane);
    const int64_t tiles = key_tiles<NW>(mine), upto = wave_scan(tiles), n = length_of<NW>(a, mine), n_upto = wave_scan(n);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(upto > t);
    if (!found && hit) {
      const int l = __builtin_ctzll(hit);
      found = true;
      s = lane_seq(mine, l);
      t -= lane64(upto - tiles, l);
      blocks = total + lane64(n_upto - n, l);
    } else if (!found) {
      t -= lane64(upto, 63);
    }
    total += lane64(n_upto, 63);
  }
  if (!found) return;
  const int64_t per = range_length(a, total, n_ranges);
  const int64_t u0 = blocks + kvh * length_before<NW>(a, s, key_tiles<NW>(s)) + length_before<NW>(a, s, t);
  const int64_t u1 = u0 + length_before<NW>(a, s, t + 1) - length_before<NW>(a, s, t);
  const int64_t w0 = quot(u0, per), w_first = quot(u0 + kTileStart, per), w1 = quot(u1 - 1, per);     // the first with blocks of it: w_first
  if (w_first == w1) return;                          // finished by its workgroup
  f32x4 dk[4], dv[4];
#pragma unroll
  for (int g = 0; g < 4; ++g) dk[g] = dv[g] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int64_t W = w_first; W <= w1; W += 4) {         // four parts on their way at once
    f32x4 k4[4][4], v4[4][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t x = min(W + q, w1);
      const f32x4* const part = reinterpret_cast<const f32x4*>(a.part_o) + ((x * 2 + (x == w0 && u0 > w0 * per)) * NW + w) * (D * 16) + db * 256 + lane;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        k4[q][g] = part[g * 64];
        v4[q][g] = part[D * 8 + g * 64];
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (W + q <= w1)
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            dk[g][e] += k4[q][g][e];
            dv[g][e] += v4[q][g][e];
          }
  }
  const int key = static_cast<int>(t) * 32 * NW + 32 * w + (lane & 31), kc = min(key, s.nk - 1);
  const auto pack = [](const f32x4& v, float c) { return u32x2{pack_bf16x2(v[0] * c, v[1] * c), pack_bf16x2(v[2] * c, v[3] * c)}; };
  char* const to_k = at(a.dk, s.k0 + kc, kvh) + 64 * db + 16 * up;
  char* const to_v = at(a.dv, s.k0 + kc, kvh) + 64 * db + 16 * up;
#pragma unroll
  for (int g = 0; g < 4; g += 2) {
    const u32x4 k = columns8(pack(dk[g], a.scale), pack(dk[g + 1], a.scale)), v = columns8(pack(dv[g], 1.f), pack(dv[g + 1], 1.f));
    if (key < s.nk) {
      *reinterpret_cast<u32x4*>(to_k + 16 * g) = k;
      *reinterpret_cast<u32x4*>(to_v + 16 * g) = v;
    }
  }
}

// dk and dv of few or short prompts: a workgroup 32 keys of a key head, its eight waves each every eighth block of 32 queries of a head that sees them, in
// slots of their own; their sums are added up in LDS, dk first, then dv: no parts, no second launch. K's and V's fragments, the same for all waves, lie in LDS: with K's in registers 25 of them spilled, 24 us for 16.
// One prompt, 8 heads: 100 tokens 6.5 us, 1000 16, 3000 64; about 1.8 us a block of a wave.
template <int D>
__global__ __launch_bounds__(512, 2) void dkv_short_kernel(Args a) {
  using G = Geo<D>;
  using L = Loader<D, 32, 1, kBoth>;
  typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
  constexpr int kTile = 32 * G::kRow, kMine = 2 * kTile, kB = D / 32;
  __shared__ __attribute__((aligned(16))) char lds[8 * kMine + 2 * kTile + 8 * 256];
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, up = lane >> 5;
  lds_char* const qs = (lds_char*)lds + wv * kMine;
  lds_char* const ds = qs + kTile;
  lds_char* const vs = (lds_char*)lds + 8 * kMine;
  lds_char* const stats = vs + 2 * kTile + wv * 256;           // lse and delta of the block's rows
  Seq s;
  int kvh, tile;
  if (!tile_of<32, true>(a, &s, &kvh, &tile)) return;
  const int key0 = tile * 32, keys = min(32, s.nk - key0), off = s.nk - s.nq, first = a.causal ? max(0, key0 - off) : 0;
  const int per_head = (max(0, s.nq - first) + 31) / 32;
  const int64_t blocks = static_cast<int64_t>(per_head) * a.G;
  const L lq(0, lane, a.q.row), ld(0, lane, a.d_o.row);
  // block b: queries t .. + 31 of head h
  auto place = [&](int64_t b, int* h, int* t) {
    const int g = static_cast<int>(quot(b, per_head));
    *h = kvh * a.G + g;
    *t = first + static_cast<int>(b - static_cast<int64_t>(g) * per_head) * 32;
  };
  auto issue_q = [&](int64_t b) {
    int h, t;
    place(b, &h, &t);
    lq.issue(at(a.q, s.q0 + t, h), s.nq - t, qs, 0);
    if (up == 0) {
      const int64_t stat = static_cast<int64_t>(h) * a.Tq + s.q0 + t;
      load_lds4(buffer_rsrc(a.lse2 + stat, min(s.nq - t, 32) * 4), lane * 4, stats);
      load_lds4(buffer_rsrc(a.delta + stat, min(s.nq - t, 32) * 4), lane * 4, stats + 128);
    }
  };
  auto issue_d = [&](int64_t b) {
    int h, t;
    place(b, &h, &t);
    ld.issue(at(a.d_o, s.q0 + t, h), s.nq - t, ds, 0);
  };
  if (wv < blocks) {
    issue_q(wv);
    issue_d(wv);
  }
  // fragments of 16 columns, K's first: a wave one of each
  if (wv < D / 16) {
    const int kc = s.k0 + key0 + min(lane & 31, keys - 1);
    const bf16x8 k = *reinterpret_cast<const bf16x8*>(at(a.k, kc, kvh) + 32 * wv + 16 * up), v = *reinterpret_cast<const bf16x8*>(at(a.v, kc, kvh) + 32 * wv + 16 * up);
    *(lds_bf16x8*)(vs + wv * 1024 + lane * 16) = k;
    *(lds_bf16x8*)(vs + kTile + wv * 1024 + lane * 16) = v;
  }
  __syncthreads();
  const RowReads<D, kBoth> rr(lane);
  const ColReads<D, kBoth> rc(lane);
  f32x16 dk[kB], dv[kB];
#pragma unroll
  for (int db = 0; db < kB; ++db) {
    zero(dk[db]);
    zero(dv[db]);
  }
  for (int64_t b = wv; b < blocks; b += 8) {
    int h, t;
    place(b, &h, &t);
    wait_vm<0>();
    f32x16 sc, dp;
    zero(sc);
    zero(dp);
    struct Pair {
      bf16x8 a, b;
    };
    fed<D / 8, 2, D == 128>([&](int i) {
                              Pair p;
                              p.a = row_operand<D>(i < D / 16 ? qs : ds, 0, rr, i % (D / 16));
                              p.b = *(const lds_bf16x8*)(vs + i * 1024 + lane * 16);
                              return p;
                            },
                            [&](int i, const Pair& p) { mma(i < D / 16 ? sc : dp, p.a, p.b); });
    if (a.causal && t + off < key0 + 31) {
      const int edge = key0 + (lane & 31) - off - t;           // rows before it do not see the lane's key
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (entry_row(e, up) < edge) sc[e] = -INFINITY;
    }
    uint32_t pp[8], pd[8];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 ls = *(const lds_f32x4*)(stats + (8 * g + 4 * up) * 4), de = *(const lds_f32x4*)(stats + 128 + (8 * g + 4 * up) * 4);
      float p[4], d[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * g + e], a.scale_log2e, -ls[e]));
        d[e] = p[e] * (dp[4 * g + e] - de[e]);
      }
      pp[2 * g] = pack_bf16x2(p[0], p[1]);
      pp[2 * g + 1] = pack_bf16x2(p[2], p[3]);
      pd[2 * g] = pack_bf16x2(d[0], d[1]);
      pd[2 * g + 1] = pack_bf16x2(d[2], d[3]);
    }
    const bf16x8 po[2] = {operand(pp, 0), operand(pp, 1)};
    fed<2 * kB, 2, D == 128>([&](int i) { return col_operand<D>(ds, i / kB, rc, i % kB); }, [&](int i, bf16x8 v) { mma(dv[i % kB], v, po[i / kB]); });
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // do has been read
    if (b + 8 < blocks) issue_d(b + 8);
    const bf16x8 so[2] = {operand(pd, 0), operand(pd, 1)};
    fed<2 * kB, 2, D == 128>([&](int i) { return col_operand<D>(qs, i / kB, rc, i % kB); }, [&](int i, bf16x8 v) { mma(dk[i % kB], v, so[i / kB]); });
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (b + 8 < blocks) issue_q(b + 8);
  }
  const int waves = static_cast<int>(min(static_cast<int64_t>(8), max(static_cast<int64_t>(1), blocks)));
  constexpr int kLanes = D / 4;
  const int col = threadIdx.x % kLanes;
  auto sum = [&](const f32x16(&acc)[kB], const Mat& to, float c) {
    if (wv < waves) {
      const int i = lane & 31;
#pragma unroll
      for (int db = 0; db < kB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4*>(lds + wv * kMine + i * D * 4 + (((8 * db + 2 * g + up) ^ i % kLanes) << 4)) =
              f32x4{acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]};
    }
    __syncthreads();
    for (int i = threadIdx.x / kLanes; i < keys; i += 512 / kLanes) {
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      for (int w = 0; w < waves; ++w) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(lds + w * kMine + i * D * 4 + ((col ^ i % kLanes) << 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += v[e];
      }
      *reinterpret_cast<u32x2*>(at(to, s.k0 + key0 + i, kvh) + col * 8) = u32x2{pack_bf16x2(o[0] * c, o[1] * c), pack_bf16x2(o[2] * c, o[3] * c)};
    }
  };
  sum(dk, a.dk, a.scale);
  __syncthreads();
  sum(dv, a.dv, 1.f);
}

constexpr int kMaxSeq = 1 << 16;

}  // namespace pattn
}  // namespace xs

using namespace xs;

namespace {

bool aligned16(const void* p) { return !(reinterpret_cast<uintptr_t>(p) & 15); }

// A tensor of `heads` heads of D values, strides in elements; it may be NULL if it has no rows.
int lies(const void* p, int64_t row, int64_t head, int heads, int D, int rows) {
  if ((!p && rows) || !aligned16(p) || row < D || row % 8 || (heads > 1 && (head < D || head % 8 || head >= (int64_t(1) << 40)))) return XS_EINVAL;
  return row > (1 << 23) ? XS_EUNSUPPORTED : XS_OK;
}

pattn::Mat mat(const void* p, int64_t row, int64_t head) { return pattn::Mat{const_cast<char*>(static_cast<const char*>(p)), 2 * row, 2 * head}; }

int check(const xs_attn_packed* A, pattn::Args* a) {
  if (!A || A->n_seq < 1 || A->n_seq > pattn::kMaxSeq || A->heads < 1 || A->kv_heads < 1 || A->heads % A->kv_heads || A->head_dim < 1 ||
      A->Tq < 0 || A->Tk < 0 || A->max_k < 0 || A->max_k > A->Tk || !(A->scale >= 0.f) || !std::isfinite(A->scale) || A->reserved ||
      !A->q_start || !A->k_start)
    return XS_EINVAL;
  const int D = A->head_dim;
  int rc = lies(A->q, A->q_row, A->q_head, A->heads, D, A->Tq);
  for (const int r : {lies(A->k, A->k_row, A->k_head, A->kv_heads, D, A->Tk), lies(A->v, A->v_row, A->v_head, A->kv_heads, D, A->Tk),
                      lies(A->o, A->o_row, A->o_head, A->heads, D, A->Tq)})
    if (rc != XS_EINVAL && r) rc = r;
  if (rc == XS_EINVAL) return rc;
  if (rc || (D != 64 && D != 128) || static_cast<int64_t>(A->Tq) * (A->heads / A->kv_heads) >= (1 << 30) || A->Tk > (1 << 30) || A->heads > (1 << 16) ||
      static_cast<int64_t>(A->Tq) * A->heads >= (int64_t(1) << 34) || static_cast<int64_t>(A->Tk) * A->kv_heads >= (int64_t(1) << 38))
    return XS_EUNSUPPORTED;
  a->q = mat(A->q, A->q_row, A->q_head);
  a->k = mat(A->k, A->k_row, A->k_head);
  a->v = mat(A->v, A->v_row, A->v_head);
  a->o = mat(A->o, A->o_row, A->o_head);
  a->q_start = A->q_start;
  a->k_start = A->k_start;
  a->k_rows = A->k_rows;
  a->n_seq = A->n_seq;
  a->H = A->heads;
  a->Hkv = A->kv_heads;
  a->G = A->heads / A->kv_heads;
  a->shift = a->G & (a->G - 1) ? -1 : __builtin_ctz(a->G);
  a->cus = xs_host::num_cus();
  a->Tq = A->Tq;
  a->Tk = A->Tk;
  a->causal = A->causal != 0;
  a->max_k = A->max_k ? A->max_k : A->Tk;
  a->scale = A->scale > 0.f ? A->scale : 1.f / std::sqrt(static_cast<float>(D));
  a->scale_log2e = a->scale * pattn::kLog2e;
  a->lse = A->lse;
  return XS_OK;
}

// How many keys a long sequence has, as far as the host knows: a prompt's about twice their average, a cache is taken to be full. (max_k only lowers it:
// one long prompt among many short ones is taken for a short one, and its tiles follow each other in a few workgroups.)
int64_t long_keys(const pattn::Args& a) { return a.k_rows ? a.max_k : std::min<int64_t>(a.max_k, 2 * int64_t(a.Tk) / a.n_seq); }
int64_t row_tiles(const pattn::Args& a) { return packed_tiles_bound(a.Tq, a.n_seq, a.G, 128) * a.Hkv; }
// Eight waves a tile of rows where the tiles are few and long (one prompt of 1000 tokens, 8 heads: rows 25.6 -> 21.5 us, dq 28.9 -> 25.6;
// 5500 tokens in three, heads of 64: 51 -> 39, 54 -> 41; short ones lose: twenty of 200, 12 -> 16; as do many: 3000 tokens, 32 heads, 86 -> 103).
bool pairs(const pattn::Args& a) { return long_keys(a) > 768 && 2 * row_tiles(a) <= 3 * int64_t(xs_host::num_cus()); }

// Eight waves for 32 rows where these fill the chip once, twice if they are long: an eighth of the keys each (one prompt, us by rows or dealt out and so:
// 8 heads of 100 tokens 8.1 and 5.6, 512: 15.6 and 9.8, 1000: 21.3 and 11.7, 2000: 36 and 27; one head of 5000 33 and 26; four of 250, 10 heads: 11.3
// and 10.3, 12 heads: 11.4 and 12.5, the limit between them leaves 10 heads, 350 units, by rows; two of 1000, 8 heads: 22 both; 128 tokens over a cache of 4000, 8 heads: 25 and 22).
bool few_units(const pattn::Args& a) {
  const int64_t units = packed_tiles_bound(a.Tq, a.n_seq, a.G, 32) * a.Hkv, cus = xs_host::num_cus(), keys = long_keys(a);
  return keys <= 4096 && (3 * units <= 4 * cus || (keys > 768 && units <= 2 * cus));
}

// Which kernels a forward call takes, from what the host knows.
enum class Form { kRows, kWide, kNarrow, kShort };
Form form_of(const pattn::Args& a) {
  // Few rows a sequence: one launch up to 1024 keys (8 units of 1024 keys 9.6 us, in two 11.4 and the time between; 256 22.0 and 29.8; of 2048
  // keys 13.3 and 11.7).
  if (static_cast<int64_t>(a.Tq) * a.G <= 32ll * a.n_seq) return long_keys(a) <= 1024 ? Form::kShort : Form::kNarrow;
  if (few_units(a)) return Form::kShort;
  // Where the tiles of 128 rows are too few for their length the keys are dealt out too. One prompt, us by rows and dealt out (two launches): 8 heads of 4000
  // tokens 65.5 and 64.3, 8000: 184 and 164, 16384: 509 and 598; 16 heads of 2000: 39 and 47, 4000: 95 and 101.
  const int64_t tiles = row_tiles(a), cus = xs_host::num_cus(), keys = long_keys(a);
  return keys <= 1024 || tiles > 2 * cus || tiles * 4000 > cus * keys || a.G > 128 ? Form::kRows : Form::kWide;
}

// Ranges of a call whose keys are dealt out: two workgroups a CU, of narrow units each wave's.
int64_t ranges_of(const pattn::Args& a, Form f) {
  return 2 * int64_t(xs_host::num_cus()) * (f == Form::kWide ? 1 : a.Hkv % 4 == 0 ? 1 : a.Hkv % 2 == 0 ? 2 : 4);
}
// Rows of parts: two slots of each of its waves' 32 rows.
int64_t part_rows(Form f) { return f == Form::kWide || f == Form::kNarrow ? 2 * int64_t(xs_host::num_cus()) * 4 * 2 * 32 : 0; }
int64_t part_bytes(const pattn::Args& a, int D) { return a.Tq ? part_rows(form_of(a)) * (D + 2) * 4 : 0; }

template <int D>
int forward(pattn::Args a, void* ws, int64_t bytes, hipStream_t st) {
  const Form f = form_of(a);
  if (f == Form::kRows) {
    if (pairs(a)) hipLaunchKernelGGL((pattn::rows_kernel<D, 2>), xs_host::grid_of(row_tiles(a)), dim3(512), 0, st, a);
    else hipLaunchKernelGGL((pattn::rows_kernel<D, 1>), xs_host::grid_of(row_tiles(a)), dim3(256), 0, st, a);
    return xs_host::launch_status();
  }
  if (f == Form::kShort) {
    hipLaunchKernelGGL((pattn::short_kernel<D>), xs_host::grid_of(packed_tiles_bound(a.Tq, a.n_seq, a.G, 32) * a.Hkv), dim3(512), 0, st, a);
    return xs_host::launch_status();
  }
  if (!ws || !aligned16(ws) || bytes < part_bytes(a, D)) return XS_EWORKSPACE;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = a.part_o + part_rows(f) * D;
  const dim3 grid(2 * xs_host::num_cus());
  if (f == Form::kWide) {
    hipLaunchKernelGGL((pattn::wide_kernel<D>), grid, dim3(256), 0, st, a);
    if (xs_host::launch_status()) return XS_EHIP;
    const int64_t units = packed_tiles_bound(a.Tq, a.n_seq, 1, a.G < 128 ? 128 / a.G : 1) * a.Hkv;
    hipLaunchKernelGGL((pattn::join_wide_kernel<D>), xs_host::grid_of(D / 32 * units), dim3(256), 0, st, a, ranges_of(a, f));
  } else {
    hipLaunchKernelGGL((pattn::narrow_kernel<D>), grid, dim3(256), 0, st, a);
    if (xs_host::launch_status()) return XS_EHIP;
    const int64_t rows = static_cast<int64_t>(a.Tq) * a.H;
    if (rows <= 2048) hipLaunchKernelGGL((pattn::join_narrow_kernel<D, false>), xs_host::grid_of(rows), dim3(256), 0, st, a, ranges_of(a, f));
    else hipLaunchKernelGGL((pattn::join_narrow_kernel<D, true>), xs_host::grid_of((rows + 3) / 4), dim3(256), 0, st, a, ranges_of(a, f));
  }
  return xs_host::launch_status();
}

// dk and dv by 32 keys a workgroup, unless the first keys' rows are too many for one or there are units enough to share out longer tiles (us with the join,
// and so; heads of 128: one prompt of 100 tokens, 8 heads: 18.7 and 6.5, 1000: 36.9 and 16, 3000: 77 and 64; two of 1500: 57 and 45; forty of 100: 36 and 34; 32 heads
// over 8, ten of 100 tokens 30 and 21, 1000: 53 and 38; 8 heads over 2, 2000: 56 and 61; heads of 64, 1000 tokens: 24 and 10).
bool few_keys(const pattn::Args& a) {
  return a.Tk && long_keys(a) * a.G <= 4096 && packed_tiles_bound(a.Tk, a.n_seq, 1, 32) * a.Hkv <= 4 * int64_t(xs_host::num_cus());
}
// Waves of a dkv_kernel workgroup: eight (256 keys, half the rows' traffic) for sequences of 512 keys and more on average, four
// for shorter ones and for heads of 64, where a block of 32 rows is four waves' loads.
template <int D>
int dkv_waves(const pattn::Args& a) { return D == 128 && a.Tk / a.n_seq >= 512 ? 8 : 4; }
template <int D>
int64_t key_tiles_bound(const pattn::Args& a) { return packed_tiles_bound(a.Tk, a.n_seq, 1, 32 * dkv_waves<D>(a)) * a.Hkv; }
// Its workgroups: as many as the chip holds, fewer where the shortest ranges need fewer.
template <int D>
int dkv_ranges(const pattn::Args& a) {
  const int64_t most = (key_tiles_bound<D>(a) * (static_cast<int64_t>(a.G) * (a.Tq / 32 + 1) + pattn::kTileStart) + pattn::kLeast - 1) / pattn::kLeast;
  return static_cast<int>(std::min<int64_t>(most, (D == 128 ? 8 : 12) / dkv_waves<D>(a) * int64_t(xs_host::num_cus())));
}
// delta and lse of every row
int64_t stats_bytes(const pattn::Args& a) { return (static_cast<int64_t>(a.H) * a.Tq * 8 + 255) / 256 * 256; }
template <int D>
int64_t grad_bytes(const pattn::Args& a) { return stats_bytes(a) + (few_keys(a) ? 0 : dkv_ranges<D>(a)) * int64_t(2 * 2 * 32 * D * 4) * dkv_waves<D>(a); }

template <int D, int NW>
int dkv(const pattn::Args& a, int ranges, hipStream_t st) {
  hipLaunchKernelGGL((pattn::dkv_kernel<D, NW>), dim3(ranges), dim3(64 * NW), 0, st, a);
  if (xs_host::launch_status()) return XS_EHIP;
  hipLaunchKernelGGL((pattn::dkv_join_kernel<D, NW>), xs_host::grid_of(key_tiles_bound<D>(a) * (NW * (D / 32) / 4)), dim3(256), 0, st, a, ranges);
  return xs_host::launch_status();
}

template <int D>
int backward(pattn::Args a, void* ws, int64_t bytes, hipStream_t st) {
  const int64_t need = grad_bytes<D>(a);
  if (need && (!ws || !aligned16(ws) || bytes < need)) return XS_EWORKSPACE;
  a.delta = static_cast<float*>(ws);
  a.lse2 = a.delta + static_cast<int64_t>(a.H) * a.Tq;
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + stats_bytes(a));
  if (a.Tq) {
    if (few_units(a))
      hipLaunchKernelGGL((pattn::dq_short_kernel<D>), xs_host::grid_of(packed_tiles_bound(a.Tq, a.n_seq, a.G, 32) * a.Hkv), dim3(512), 0, st, a);
    else if (pairs(a)) hipLaunchKernelGGL((pattn::dq_kernel<D, 2>), xs_host::grid_of(row_tiles(a)), dim3(512), 0, st, a);
    else hipLaunchKernelGGL((pattn::dq_kernel<D, 1>), xs_host::grid_of(row_tiles(a)), dim3(256), 0, st, a);
    if (xs_host::launch_status()) return XS_EHIP;
  }
  if (few_keys(a)) {
    hipLaunchKernelGGL((pattn::dkv_short_kernel<D>), xs_host::grid_of(packed_tiles_bound(a.Tk, a.n_seq, 1, 32) * a.Hkv), dim3(512), 0, st, a);
    return xs_host::launch_status();
  }
  const int ranges = dkv_ranges<D>(a);
  if (!ranges) return XS_OK;
  if constexpr (D == 128)
    if (dkv_waves<D>(a) == 8) return dkv<D, 8>(a, ranges, st);
  return dkv<D, 4>(a, ranges, st);
}

}  // namespace

extern "C" int xs_attention_packed_workspace_bytes(const xs_attn_packed* A, int64_t* bytes) {
  pattn::Args a{};
  if (!bytes) return XS_EINVAL;
  if (int rc = check(A, &a)) return rc;
  *bytes = part_bytes(a, A->head_dim);
  return XS_OK;
}

extern "C" int xs_attention_packed(const xs_attn_packed* A, void* workspace, int64_t workspace_bytes, int32_t* dev_status, void* stream) {
  pattn::Args a{};
  if (int rc = check(A, &a)) return rc;
  if (a.Tq == 0) return XS_OK;
  a.status = dev_status;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return A->head_dim == 128 ? forward<128>(a, workspace, workspace_bytes, st) : forward<64>(a, workspace, workspace_bytes, st);
}

extern "C" int xs_attention_packed_backward_workspace_bytes(const xs_attn_packed* A, int64_t* bytes) {
  pattn::Args a{};
  if (!bytes) return XS_EINVAL;
  if (int rc = check(A, &a)) return rc;
  *bytes = A->head_dim == 128 ? grad_bytes<128>(a) : grad_bytes<64>(a);
  return XS_OK;
}

extern "C" int xs_attention_packed_backward(const xs_attn_packed* A, const xs_attn_grads* g, void* workspace, int64_t workspace_bytes,
                                            int32_t* dev_status, void* stream) {
  pattn::Args a{};
  if (int rc = check(A, &a)) return rc;
  if (!g || (!a.lse && a.Tq)) return XS_EINVAL;
  const int D = A->head_dim;
  bool unsupported = a.k_rows != nullptr;
  for (const int r : {lies(g->d_o, g->do_row, g->do_head, a.H, D, a.Tq), lies(g->dq, g->dq_row, g->dq_head, a.H, D, a.Tq),
                      lies(g->dk, g->dk_row, g->dk_head, a.Hkv, D, a.Tk), lies(g->dv, g->dv_row, g->dv_head, a.Hkv, D, a.Tk)}) {
    if (r == XS_EINVAL) return r;
    unsupported |= r != XS_OK;
  }
  if (unsupported) return XS_EUNSUPPORTED;
  a.d_o = mat(g->d_o, g->do_row, g->do_head);
  a.dq = mat(g->dq, g->dq_row, g->dq_head);
  a.dk = mat(g->dk, g->dk_row, g->dk_head);
  a.dv = mat(g->dv, g->dv_row, g->dv_head);
  a.status = dev_status;
  hipStream_t st = static_cast<hipStream_t>(stream);
  return D == 128 ? backward<128>(a, workspace, workspace_bytes, st) : backward<64>(a, workspace, workspace_bytes, st);
}
