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
  float scale, scale_log2e;
  float* lse;            // [H][Tq]
  float* delta;          // [H][Tq] (gradients)
  float* part_o;         // [waves][2][32][D] (split); dkv_kernel's parts
  float* part_ml;        // [waves][2][32][2]
  int32_t* status;
};

// The keys of a sequence; false (with the error noted) if they do not lie in k.
__device__ __forceinline__ bool keys_of(const Args& a, int seq, int* k0, int* m) {
  const int s = a.k_start[seq];
  const int n = a.k_rows ? a.k_rows[seq] : a.k_start[seq + 1] - s;
  if (s < 0 || n < 0 || n > a.max_k || s > a.Tk - n) {
    set_status(a.status, XS_EBADINPUT);
    return false;
  }
  *k0 = s;
  *m = n;
  return true;
}

// How many keys row r of a sequence sees.
__device__ __forceinline__ int sees(const Args& a, int r, int nq, int nk) {
  return a.causal ? min(max(nk - nq + r / a.G + 1, 0), nk) : nk;
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
};

// N matrix instructions, mul(i, operand), whose LDS reads are issued AHEAD instructions before them. Left to itself the
// compiler reads one operand, waits for it and multiplies.
template <int N, int AHEAD, class Read, class Mul>
__device__ __forceinline__ void fed(const Read& read, const Mul& mul) {
  decltype(read(0)) buf[AHEAD + 1];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) buf[i] = read(i);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i + AHEAD < N) buf[(i + AHEAD) % (AHEAD + 1)] = read(i + AHEAD);
    __builtin_amdgcn_sched_barrier(0);
    mul(i, buf[i % (AHEAD + 1)]);
    __builtin_amdgcn_sched_barrier(0);
  }
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

// acc[column of the tile][lane's column] += sum over 16 rows of the tile, from row 16 s
template <int D, Way WAY>
__device__ __forceinline__ void cols_product(const lds_char* tile, int s, const ColReads<D, WAY>& rd, bf16x8 b, f32x16 (&acc)[D / 32]) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db) mma(acc[db], col_operand<D>(tile, s, rd, db), b);
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

// A lane's row (or key) of accumulators, times c, as bf16 to `row`.
template <int D>
__device__ __forceinline__ void store_row(char* row, const f32x16 (&acc)[D / 32], float c) {
  const int up = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const u32x2 v = {pack_bf16x2(acc[db][4 * g] * c, acc[db][4 * g + 1] * c), pack_bf16x2(acc[db][4 * g + 2] * c, acc[db][4 * g + 3] * c)};
      *reinterpret_cast<u32x2*>(row + (32 * db + 8 * g + 4 * up) * 2) = v;
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

// ------------------------------------------------------------------------------ many rows
// A workgroup takes 128 rows (four waves of 32) and streams the keys they see in tiles of 64. LDS: two K slots
// and one V slot. Per tile j: S from K slot j % 2, a barrier, K tile j + 2 into that slot; the softmax; V tile
// j waited for and a barrier; O from the V slot; K tile j + 1 waited for, a barrier, V tile j + 1 into the V slot.
template <int D>
__global__ __launch_bounds__(256, D == 128 ? 3 : 4) void rows_kernel(Args a) {
  using G = Geo<D>;
  constexpr int kBKV = 64, kTile = kBKV * G::kRow, kLoads = Loader<D, kBKV, 4, kRows>::kLoads;
  __shared__ __attribute__((aligned(16))) char lds_raw[3 * kTile];
  lds_char* const lds = (lds_char*)lds_raw;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), up = lane >> 5;
  const int64_t id = block_number();
  const int kvh = static_cast<int>(id % a.Hkv);
  PackedTile s;
  int k0, nk;
  if (!packed_tile(a.q_start, a.n_seq, a.Tq, a.G, 128, static_cast<int>(id / a.Hkv), &s, a.status) || !keys_of(a, s.seq, &k0, &nk)) return;
  k0 = __builtin_amdgcn_readfirstlane(k0);
  nk = __builtin_amdgcn_readfirstlane(nk);
  const int nq = s.rows, R = nq * a.G;
  const int r0 = ((R + 127) / 128 - 1 - s.tile) * 128;       // the longest rows first
  const int nkv = (sees(a, min(r0 + 127, R - 1), nq, nk) + kBKV - 1) / kBKV;
  const int w0 = r0 + 32 * w;
  const int whole = min(sees(a, r0, nq, nk) / kBKV, nkv);   // tiles that every row sees whole
  const int r = min(w0 + (lane & 31), R - 1), lim = sees(a, r, nq, nk);
  bf16x8 qf[D / 16];
  load_frags<D>(at(a.q, s.start + r / a.G, kvh * a.G + r % a.G), qf);
  const char* const kp = at(a.k, k0, kvh);
  const char* const vp = at(a.v, k0, kvh);
  lds_char* const vs = lds + 2 * kTile;
  // Every lane's addresses are made anew where they are used: kept over the loop they spill, and a reload waits for all
  // the tiles in flight.
  auto issue_k = [&](int j) {
    Loader<D, kBKV, 4, kRows>(w, here(lane), a.k.row).issue(kp + static_cast<int64_t>(j) * kBKV * a.k.row, nk - j * kBKV, lds + (j & 1) * kTile, w);
  };
  auto issue_v = [&](int j) {
    Loader<D, kBKV, 4, kCols>(w, here(lane), a.v.row).issue(vp + static_cast<int64_t>(j) * kBKV * a.v.row, nk - j * kBKV, vs, w);
  };
  Soft<D> f;
  f.clear();
  if (nkv > 0) {
    issue_k(0);
    issue_v(0);
    if (nkv > 1) issue_k(1);
    wait_vm<0>();
    asm volatile("s_barrier" ::: "memory");
  }
  auto step = [&](int j, auto masked) {
    lds_char* const ks = lds + (j & 1) * kTile;
    const RowReads<D, kRows> rr(here(lane));
    f32x16 sc[2] = {rows_product<D>(ks, 0, rr, qf), rows_product<D>(ks, 1, rr, qf)};
    // every wave is done with K slot j % 2: K tile j + 2 goes there
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const bool k2 = j + 2 < nkv;
    if (k2) issue_k(j + 2);
    if constexpr (masked) {
      hide(sc[0], j * kBKV, lim, here(lane) >> 5);
      hide(sc[1], j * kBKV + 32, lim, here(lane) >> 5);
    }
    uint32_t pk[2][8];
    f.take(sc, a.scale_log2e, pk);
    // V tile j has landed in every wave's share (only K tile j + 2 may still be in flight)
    if (k2) wait_vm<kLoads>(); else wait_vm<0>();
    asm volatile("s_barrier" ::: "memory");
    const ColReads<D, kCols> rc(here(lane));
#pragma unroll
    for (int st = 0; st < 4; ++st) cols_product<D>(vs, st, rc, operand(pk[st >> 1], st & 1), f.o);
    if (j + 1 < nkv) {
      // K tile j + 1 has landed in every wave's share, and no wave reads the V slot any more
      if (k2) wait_vm<kLoads>(); else wait_vm<0>();
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      issue_v(j + 1);
    }
  };
  for (int j = 0; j < whole; ++j) step(j, std::false_type());
  for (int j = whole; j < nkv; ++j) step(j, std::true_type());
  const int rl = w0 + here(lane & 31);
  if (rl >= R) return;
  const int qi = rl / a.G, h = kvh * a.G + (rl - qi * a.G);
  store_row<D>(at(a.o, s.start + qi, h), f.o, f.inverse());
  if (a.lse && up == 0) a.lse[static_cast<int64_t>(h) * a.Tq + s.start + qi] = f.lse();
}

// ------------------------------------------------------------------------------ few rows
// Few rows over many keys: what counts is how fast the chip reads K and V, so the keys are dealt out evenly
// over all waves. The work is units (sequence, 32 rows, key head) of L = ceil(m / 32) key tiles each, laid end
// to end; wave W of NW takes the tiles [W per, (W + 1) per), per = ceil(total / NW), wherever units
// begin and end. A unit that lies in one wave's range is finished there; of the others each wave leaves a
// part (sums relative to its maximum): in its slot 0 for the unit that its range begins in or with, in slot 1 for
// one that begins later. join_kernel adds them up in order. A wave has its own two slots of K and V and waits for
// nobody.
struct Unit {
  int seq, q0, nq, k0, nk, L, first, kvh, r0;
};

// What a sequence has to do: false if it is skipped.
__device__ __forceinline__ int64_t units_of(const Args& a, int s, int* q0, int* nq, int* k0, int* nk) {
  *q0 = *nq = *k0 = *nk = 0;
  if (s >= a.n_seq) return 0;
  const int lo = a.q_start[s], hi = a.q_start[s + 1];
  if (lo < 0 || hi < lo || hi > a.Tq) {
    set_status(a.status, XS_EBADINPUT);
    return 0;
  }
  if (hi == lo || !keys_of(a, s, k0, nk)) return 0;
  *q0 = lo;
  *nq = hi - lo;
  return static_cast<int64_t>((static_cast<int64_t>(*nq) * a.G + 31) / 32) * a.Hkv;
}
__device__ __forceinline__ int tiles_of(int nk) { return nk > 0 ? static_cast<int>((static_cast<int64_t>(nk) + 31) / 32) : 1; }

__device__ __forceinline__ int64_t scan64(int64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t u = __shfl_up(v, d);
    if (lane >= d) v += u;
  }
  return v;
}
__device__ __forceinline__ int64_t lane64(int64_t v, int l) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(v), l), hi = __builtin_amdgcn_readlane(static_cast<int>(v >> 32), l);
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

__device__ __forceinline__ int64_t all_tiles(const Args& a) {
  int64_t total = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    int q0, nq, k0, nk;
    const int64_t u = units_of(a, s0 + (threadIdx.x & 63), &q0, &nq, &k0, &nk);
    total += lane64(scan64(u * tiles_of(nk)), 63);
  }
  return total;
}

// The unit that tile u of all lies in; u is less than their number.
__device__ __forceinline__ void unit_at(const Args& a, int64_t u, Unit* out) {
  int64_t before = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    int q0, nq, k0, nk;
    const int64_t tiles = units_of(a, s0 + (threadIdx.x & 63), &q0, &nq, &k0, &nk) * tiles_of(nk), upto = scan64(tiles);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(before + upto > u);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      out->seq = s0 + l;
      out->q0 = __builtin_amdgcn_readlane(q0, l);
      out->nq = __builtin_amdgcn_readlane(nq, l);
      out->k0 = __builtin_amdgcn_readlane(k0, l);
      out->nk = __builtin_amdgcn_readlane(nk, l);
      out->L = tiles_of(out->nk);
      const int64_t in = u - before - lane64(upto - tiles, l), unit = in / out->L;
      out->first = static_cast<int>(in - unit * out->L);
      out->kvh = static_cast<int>(unit % a.Hkv);
      out->r0 = static_cast<int>(unit / a.Hkv) * 32;
      return;
    }
    before += lane64(upto, 63);
  }
}

template <int D>
__global__ __launch_bounds__(256) void split_kernel(Args a) {
  using G = Geo<D>;
  constexpr int kTile = 32 * G::kRow;
  __shared__ __attribute__((aligned(16))) char lds_raw[16 * kTile];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), up = lane >> 5;
  lds_char* const mine = (lds_char*)lds_raw + wv * 4 * kTile;       // K 0, K 1, V 0, V 1
  const int64_t W = static_cast<int64_t>(blockIdx.x) * 4 + wv, NW = static_cast<int64_t>(gridDim.x) * 4;
  const int64_t total = all_tiles(a), per = (total + NW - 1) / NW, end = min(W * per + per, total);
  const RowReads<D, kRows> rr(lane);
  const ColReads<D, kCols> rc(lane);
  const Loader<D, 32, 1, kRows> lk(0, lane, a.k.row);
  const Loader<D, 32, 1, kCols> lv(0, lane, a.v.row);
  Soft<D> f;
  for (int64_t u = W * per; u < end;) {
    Unit x;
    unit_at(a, u, &x);
    const int last = static_cast<int>(min(static_cast<int64_t>(x.L), x.first + (end - u)));
    const int R = x.nq * a.G, rl = x.r0 + (lane & 31), r = min(rl, R - 1), qi = r / a.G, h = x.kvh * a.G + (r - qi * a.G);
    const int lim = sees(a, r, x.nq, x.nk), all = sees(a, x.r0, x.nq, x.nk), any = sees(a, min(x.r0 + 31, R - 1), x.nq, x.nk);
    const int stop = min(last, (any + 31) / 32);
    const char* const kp = at(a.k, x.k0, x.kvh);
    const char* const vp = at(a.v, x.k0, x.kvh);
    auto issue = [&](int j) {
      lk.issue(kp + static_cast<int64_t>(j) * 32 * a.k.row, x.nk - j * 32, mine + (j & 1) * kTile, 0);
      lv.issue(vp + static_cast<int64_t>(j) * 32 * a.v.row, x.nk - j * 32, mine + (2 + (j & 1)) * kTile, 0);
    };
    // the last unit's reads of these slots are done
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (x.first < stop) issue(x.first);
    bf16x8 qf[D / 16];
    load_frags<D>(at(a.q, x.q0 + qi, h), qf);
    f.clear();
    for (int j = x.first; j < stop; ++j) {
      wait_vm<0>();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // tile j - 1 has been read
      if (j + 1 < stop) issue(j + 1);
      f32x16 sc[1] = {rows_product<D>(mine + (j & 1) * kTile, 0, rr, qf)};
      if (j * 32 + 32 > all) hide(sc[0], j * 32, lim, up);
      uint32_t pk[1][8];
      f.take(sc, a.scale_log2e, pk);
      cols_product<D>(mine + (2 + (j & 1)) * kTile, 0, rc, operand(pk[0], 0), f.o);
      cols_product<D>(mine + (2 + (j & 1)) * kTile, 1, rc, operand(pk[0], 1), f.o);
    }
    if (rl < R) {
      if (x.first == 0 && last == x.L) {
        store_row<D>(at(a.o, x.q0 + qi, h), f.o, f.inverse());
        if (a.lse && up == 0) a.lse[static_cast<int64_t>(h) * a.Tq + x.q0 + qi] = f.lse();
      } else {
        const int64_t slot = (W * 2 + (u > W * per)) * 32 + (lane & 31);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(a.part_o + slot * D + 32 * db + 8 * g + 4 * up) =
                f32x4{f.o[db][4 * g], f.o[db][4 * g + 1], f.o[db][4 * g + 2], f.o[db][4 * g + 3]};
        if (up == 0) *reinterpret_cast<f32x2_t*>(a.part_ml + slot * 2) = f32x2_t{f.m, f.l};
      }
    }
    u += last - x.first;
  }
}

// One workgroup a unit, a wave a row at a time.
template <int D>
__global__ __launch_bounds__(256) void join_kernel(Args a, int64_t NW) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int64_t id = block_number(), total = all_tiles(a), per = (total + NW - 1) / NW;
  // the id-th unit and its first tile
  int64_t units = 0, tiles = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    int q0, nq, k0, nk;
    const int64_t n = units_of(a, s0 + lane, &q0, &nq, &k0, &nk), upto = scan64(n), t = n * tiles_of(nk), t_upto = scan64(t);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(units + upto > id);
    if (!hit) {
      units += lane64(upto, 63);
      tiles += lane64(t_upto, 63);
      continue;
    }
    const int l = __builtin_ctzll(hit);
    q0 = __builtin_amdgcn_readlane(q0, l);
    nq = __builtin_amdgcn_readlane(nq, l);
    const int L = tiles_of(__builtin_amdgcn_readlane(nk, l));
    const int64_t in = id - units - lane64(upto - n, l), u0 = tiles + lane64(t_upto - t, l) + in * L;
    const int64_t w0 = u0 / per, w1 = (u0 + L - 1) / per;
    if (w0 == w1) return;                                   // finished by its wave
    const int kvh = static_cast<int>(in % a.Hkv), r0 = static_cast<int>(in / a.Hkv) * 32;
    const int n_rows = min(32, nq * a.G - r0);
    for (int i = wv; i < n_rows; i += 4) {
      const auto slot = [&](int64_t w) { return (w * 2 + (w == w0 && u0 > w0 * per)) * 32 + i; };
      float top = -FLT_MAX;
      for (int64_t w = w0; w <= w1; ++w) top = fmaxf(top, a.part_ml[slot(w) * 2]);
      float sum = 0.f, o[D / 64] = {};
      for (int64_t w = w0; w <= w1; ++w) {
        const f32x2_t ml = *reinterpret_cast<const f32x2_t*>(a.part_ml + slot(w) * 2);
        const float c = __builtin_amdgcn_exp2f(ml.x - top);
        sum = __builtin_fmaf(ml.y, c, sum);
#pragma unroll
        for (int d = 0; d < D / 64; ++d) o[d] = __builtin_fmaf(a.part_o[slot(w) * D + lane * (D / 64) + d], c, o[d]);
      }
      const int r = r0 + i, qi = r / a.G, h = kvh * a.G + (r - qi * a.G);
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      char* const out = at(a.o, q0 + qi, h);
      if constexpr (D == 128) reinterpret_cast<uint32_t*>(out)[lane] = pack_bf16x2(o[0] * inv, o[1] * inv);
      else reinterpret_cast<uint16_t*>(out)[lane] = static_cast<uint16_t>(f2bf(o[0] * inv));
      if (a.lse && lane == 0)
        a.lse[static_cast<int64_t>(h) * a.Tq + q0 + qi] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
    return;
  }
}

// ------------------------------------------------------------------------------ gradients
// dq: as rows_kernel, with a second product (V times the row's do) and dS in place of the probabilities. It
// computes delta for its rows and leaves it for the kernel below.
//
// delta = do . o takes o's roundings (of the probabilities and of o itself) to every dS of the row alike, a
// relative error of dq and dk of about 0.0023 / sqrt(keys that share the weight): nothing beside the 0.0017 that dS's own
// rounding gives where a row sees many keys, and the larger part where it sees ten. Tiles that see at most
// kExactTiles tiles of keys therefore take delta = sum_j P_ij (do_i . v_j) in a pass before.
constexpr int kExactTiles = 4;
template <int D>
__global__ __launch_bounds__(256, 2) void dq_kernel(Args a) {
  using G = Geo<D>;
  constexpr int kBKV = 64, kTile = kBKV * G::kRow;
  __shared__ __attribute__((aligned(16))) char lds_raw[4 * kTile];
  lds_char* const lds = (lds_char*)lds_raw;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), up = lane >> 5;
  const int64_t id = block_number();
  const int kvh = static_cast<int>(id % a.Hkv);
  PackedTile s;
  int k0, nk;
  if (!packed_tile(a.q_start, a.n_seq, a.Tq, a.G, 128, static_cast<int>(id / a.Hkv), &s, a.status) || !keys_of(a, s.seq, &k0, &nk)) return;
  k0 = __builtin_amdgcn_readfirstlane(k0);
  nk = __builtin_amdgcn_readfirstlane(nk);
  const int nq = s.rows, R = nq * a.G;
  const int r0 = ((R + 127) / 128 - 1 - s.tile) * 128;
  const int nkv = (sees(a, min(r0 + 127, R - 1), nq, nk) + kBKV - 1) / kBKV;
  const int w0 = r0 + 32 * w;
  const int all = w0 < R ? sees(a, w0, nq, nk) : 0, any = w0 < R ? sees(a, min(w0 + 31, R - 1), nq, nk) : 0;
  const int r = min(w0 + (lane & 31), R - 1), qi = r / a.G, h = kvh * a.G + (r - qi * a.G), lim = sees(a, r, nq, nk);
  const RowReads<D, kBoth> rk(lane);
  const ColReads<D, kBoth> ck(lane);
  const RowReads<D, kRows> rv(lane);
  const Loader<D, kBKV, 4, kBoth> lk(w, lane, a.k.row);
  const Loader<D, kBKV, 4, kRows> lv(w, lane, a.v.row);
  const char* const kp = at(a.k, k0, kvh);
  const char* const vp = at(a.v, k0, kvh);
  auto issue = [&](int j, int slot) {
    lk.issue(kp + static_cast<int64_t>(j) * kBKV * a.k.row, nk - j * kBKV, lds + slot * kTile, w);
    lv.issue(vp + static_cast<int64_t>(j) * kBKV * a.v.row, nk - j * kBKV, lds + (2 + slot) * kTile, w);
  };
  if (nkv > 0) issue(0, 0);
  bf16x8 qf[D / 16], df[D / 16];
  load_frags<D>(at(a.q, s.start + qi, h), qf);
  load_frags<D>(at(a.d_o, s.start + qi, h), df);
  const int64_t stat = static_cast<int64_t>(h) * a.Tq + s.start + qi;
  const float lse2 = lim > 0 ? a.lse[stat] * kLog2e : 0.f;
  int slot = 0;
  // tile j has landed in every wave's share, and no wave reads the tile before it any more; then `next` is loaded
  auto turn = [&](int next) {
    wait_vm<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    slot ^= 1;
    if (next < nkv) issue(next, slot);
  };
  float delta = 0.f;
  if (nkv <= kExactTiles) {
    for (int j = 0; j < nkv; ++j) {
      turn(j + 1 < nkv ? j + 1 : 0);
#pragma unroll 1
      for (int b = 0; b < 2 && j * kBKV + 32 * b < any; ++b) {
        f32x16 sc = rows_product<D>(lds + (slot ^ 1) * kTile, b, rk, qf);
        const f32x16 dp = rows_product<D>(lds + (2 + (slot ^ 1)) * kTile, b, rv, df);
        hide(sc, j * kBKV + 32 * b, lim, up);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          delta = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(sc[e], a.scale_log2e, -lse2)), dp[e], delta);
      }
    }
  } else {
    bf16x8 of[D / 16];
    load_frags<D>(at(a.o, s.start + qi, h), of);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = __builtin_fmaf(static_cast<float>(df[kk][e]), static_cast<float>(of[kk][e]), delta);
  }
  delta = add_halves(delta);
  f32x16 acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[db][e] = 0.f;
  for (int j = 0; j < nkv; ++j) {
    turn(j + 1);
    if (j * kBKV >= any) continue;                           // wave-uniform
    lds_char* const ks = lds + (slot ^ 1) * kTile;
    lds_char* const vs = lds + (2 + (slot ^ 1)) * kTile;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x16 sc = rows_product<D>(ks, b, rk, qf);
      const f32x16 dp = rows_product<D>(vs, b, rv, df);
      if (j * kBKV + 32 * b + 32 > all) hide(sc, j * kBKV + 32 * b, lim, up);
      uint32_t pk[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[2 * e], a.scale_log2e, -lse2));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[2 * e + 1], a.scale_log2e, -lse2));
        pk[e] = pack_bf16x2(p0 * (dp[2 * e] - delta), p1 * (dp[2 * e + 1] - delta));
      }
      cols_product<D>(ks, 2 * b, ck, operand(pk, 0), acc);
      cols_product<D>(ks, 2 * b + 1, ck, operand(pk, 1), acc);
    }
  }
  if (w0 + (lane & 31) >= R) return;
  if (up == 0) a.delta[stat] = delta;
  store_row<D>(at(a.dq, s.start + qi, h), acc, a.scale);
}

// dk and dv: a workgroup holds 32 NW keys of a key head (NW waves of 32), their K and V fragments beside both
// results' accumulators in registers, and streams the rows that see them, 32 queries of one head at a time with do,
// lse and delta, two blocks ahead in three LDS slots. Two waves share a SIMD's registers: kStash of V's fragments lie in
// LDS. Queries past the end of the sequence are zeros with lse 0: P = 1, but do = 0 and dS = 1 (0 - 0).
//
// The first keys of a sequence have G times as many rows as it has queries, the last ones hardly any, and there are few key
// heads: key tiles dealt one to a workgroup leave the chip waiting for the longest (8192 tokens in 4 sequences, 32 heads
// over 8: 904 us). So the blocks of all key tiles, laid end to end, are dealt out evenly: workgroup W takes the blocks [W per,
// (W + 1) per), per = ceil(total / workgroups) but at least kLeast. A key tile that lies in one range is finished there, of
// the others each workgroup leaves a part, in its slot 0 for the tile that its range begins in or with, in slot 1 for one that
// begins later; dkv_join_kernel adds them up in order.
constexpr int kLeast = 16;

struct KeySeq {
  int q0, nq, k0, nk;
};
struct KeyTile {
  KeySeq s;
  int kvh, tile, per_head;      // key tile; blocks of 32 queries that see it
  int64_t first, blocks;        // the block searched for, of the tile's
};

// Blocks of one query head in a sequence's tiles of 32 NW keys before tile j: those whose first key every query sees have all
// ceil(nq / 32) (one where there is none: such keys' zeros are still written), from there on every tile has NW less.
template <int NW>
__device__ __forceinline__ int64_t blocks_before(const Args& a, const KeySeq& s, int64_t j) {
  const int64_t f = max(1, (s.nq + 31) / 32), c = (s.nk + 31) / 32, off = s.nk - s.nq;
  if (!a.causal) return j * f;
  const int64_t full = off > 0 ? (off + 32 * NW - 1) / (32 * NW) : 0;
  return j <= full ? j * f : full * f + (j - full) * c - NW / 2 * (j * (j - 1) - full * (full - 1));
}

__device__ __forceinline__ KeySeq key_seq(const Args& a, int s) {
  KeySeq x{0, 0, 0, 0};
  if (s >= a.n_seq) return x;
  const int q0 = a.q_start[s], q1 = a.q_start[s + 1], k0 = a.k_start[s], k1 = a.k_start[s + 1];
  if (q0 < 0 || q1 < q0 || q1 > a.Tq || k0 < 0 || k1 < k0 || k1 > a.Tk || k1 - k0 > a.max_k) {
    set_status(a.status, XS_EBADINPUT);
    return x;
  }
  return KeySeq{q0, q1 - q0, k0, k1 - k0};
}
template <int NW>
__device__ __forceinline__ int key_tiles(const KeySeq& s) { return (s.nk + 32 * NW - 1) / (32 * NW); }
template <int NW>
__device__ __forceinline__ int64_t blocks_of(const Args& a, const KeySeq& s) { return blocks_before<NW>(a, s, key_tiles<NW>(s)) * a.H; }

template <int NW>
__device__ __forceinline__ int64_t all_blocks(const Args& a) {
  int64_t total = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) total += lane64(scan64(blocks_of<NW>(a, key_seq(a, s0 + (threadIdx.x & 63)))), 63);
  return total;
}

__device__ __forceinline__ KeySeq lane_seq(const KeySeq& s, int l) {
  return KeySeq{__builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.nq, l), __builtin_amdgcn_readlane(s.k0, l),
                __builtin_amdgcn_readlane(s.nk, l)};
}

// The key tile that block u of all lies in; u is less than their number.
template <int NW>
__device__ __forceinline__ void key_tile_at(const Args& a, int64_t u, KeyTile* out) {
  int64_t before = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    const KeySeq mine = key_seq(a, s0 + (threadIdx.x & 63));
    const int64_t n = blocks_of<NW>(a, mine), upto = scan64(n);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(before + upto > u);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      out->s = lane_seq(mine, l);
      const int tiles = key_tiles<NW>(out->s);
      const int64_t head = blocks_before<NW>(a, out->s, tiles) * a.G, in = u - before - lane64(upto - n, l);
      out->kvh = static_cast<int>(in / head);
      const int64_t x = in - out->kvh * head;
      int lo = 0, hi = tiles - 1;                               // the tile with before(tile) G <= x < before(tile + 1) G
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (blocks_before<NW>(a, out->s, mid + 1) * a.G > x) hi = mid;
        else lo = mid + 1;
      }
      const int64_t b0 = blocks_before<NW>(a, out->s, lo);
      out->tile = lo;
      out->per_head = static_cast<int>(blocks_before<NW>(a, out->s, lo + 1) - b0);
      out->blocks = static_cast<int64_t>(out->per_head) * a.G;
      out->first = x - b0 * a.G;
      return;
    }
    before += lane64(upto, 63);
  }
}

// Workgroups that have blocks to do lie side by side on one XCD, whose L2 then holds their rows.
__device__ __forceinline__ int64_t range_of_block(int b, int n) { return n % 8 ? b : static_cast<int64_t>(b % 8) * (n / 8) + b / 8; }

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, D == 128 ? 8 / NW : 12 / NW) void dkv_kernel(Args a) {
  using G = Geo<D>;
  constexpr int kBQ = 32, kTile = kBQ * G::kRow, kStages = 3, kStash = D == 128 ? 6 : 0;
  constexpr int kLoads = 2 * Loader<D, kBQ, NW, kBoth>::kLoads;                 // of a stage, a wave's (without lse and delta)
  __shared__ __attribute__((aligned(16))) char lds_raw[2 * kStages * kTile + 2 * kStages * kBQ * 4 + NW * kStash * 1024];
  lds_char* const lds = (lds_char*)lds_raw;
  lds_char* const stats = lds + 2 * kStages * kTile;                           // lse and delta of each stage
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  lds_char* const stash = stats + 2 * kStages * kBQ * 4 + w * kStash * 1024;
  const int64_t total = all_blocks<NW>(a), per = max(static_cast<int64_t>(kLeast), (total + gridDim.x - 1) / gridDim.x);
  const int64_t W = range_of_block(blockIdx.x, gridDim.x), begin = W * per, end = min(begin + per, total);
  for (int64_t u = begin; u < end;) {
    KeyTile x;
    key_tile_at<NW>(a, u, &x);
    const int n = static_cast<int>(min(x.blocks - x.first, end - u));
    const int nq = x.s.nq, nk = x.s.nk, key0 = x.tile * 32 * NW, kw = key0 + 32 * w, off = nk - nq;
    const int first = a.causal ? max(0, key0 - off) : 0;       // the first query that sees one of these keys
    // the next block to load: its head in the group, first query and stage
    int lg = static_cast<int>(x.first / x.per_head), lt = first + static_cast<int>(x.first - static_cast<int64_t>(lg) * x.per_head) * kBQ, lst = 0;
    int t = lt, st = 0;
    auto issue = [&] {
      const int h = x.kvh * a.G + lg;
      const Loader<D, kBQ, NW, kBoth> lq(w, here(lane), a.q.row), ld(w, here(lane), a.d_o.row);
      lq.issue(at(a.q, x.s.q0 + lt, h), nq - lt, lds + 2 * lst * kTile, w);
      ld.issue(at(a.d_o, x.s.q0 + lt, h), nq - lt, lds + (2 * lst + 1) * kTile, w);
      if (w < 2) {                                             // the lower half's lanes fetch the 32 rows' numbers
        const float* const src = (w ? a.delta : a.lse) + static_cast<int64_t>(h) * a.Tq + x.s.q0 + lt;
        if ((here(lane) & 32) == 0) load_lds4(buffer_rsrc(src, min(nq - lt, kBQ) * 4), here(lane) * 4, stats + (2 * lst + w) * kBQ * 4);
      }
      lt += kBQ;
      if (lt >= nq) {
        lt = first;
        ++lg;
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
        const RowReads<D, kBoth> rr(ln);
        f32x16 sc, dp;
        zero(sc);
        zero(dp);
        struct Pair {
          bf16x8 a, b;
        };
        fed<D / 8, 2>([&](int i) {
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
            p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[4 * g + e], a.scale_log2e, -ls[e] * kLog2e));
            d[e] = p[e] * (dp[4 * g + e] - de[e]);
          }
          pp[2 * g] = pack_bf16x2(p[0], p[1]);
          pp[2 * g + 1] = pack_bf16x2(p[2], p[3]);
          pd[2 * g] = pack_bf16x2(d[0], d[1]);
          pd[2 * g + 1] = pack_bf16x2(d[2], d[3]);
        }
        const ColReads<D, kBoth> rc(ln);
        const bf16x8 po[2] = {operand(pp, 0), operand(pp, 1)}, so[2] = {operand(pd, 0), operand(pd, 1)};
        constexpr int kB = D / 32;                             // instruction i: 16 rows i / (2 kB), of dv, then dk, its block
        fed<4 * kB, 2>([&](int i) { return col_operand<D>(i / kB % 2 ? qs : ds, i / (2 * kB), rc, i % kB); },
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
      if (key < nk) {
        store_row<D>(at(a.dk, x.s.k0 + key, x.kvh), dk, a.scale);
        store_row<D>(at(a.dv, x.s.k0 + key, x.kvh), dv, 1.f);
      }
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
    u += n;
  }
}

// One workgroup a key tile: its parts, each wave its 32 keys', in the order of the ranges.
template <int D, int NW>
__global__ __launch_bounds__(64 * NW) void dkv_join_kernel(Args a, int n_ranges) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t id = block_number(), total = all_blocks<NW>(a), per = max(static_cast<int64_t>(kLeast), (total + n_ranges - 1) / n_ranges);
  const int kvh = static_cast<int>(id % a.Hkv);
  int64_t t = id / a.Hkv, blocks = 0;                 // the tile's number, counted over the sequences
  for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
    const KeySeq mine = key_seq(a, s0 + lane);
    const int64_t tiles = key_tiles<NW>(mine), upto = scan64(tiles), n = blocks_of<NW>(a, mine), n_upto = scan64(n);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(upto > t);
    if (!hit) {
      t -= lane64(upto, 63);
      blocks += lane64(n_upto, 63);
      continue;
    }
    const int l = __builtin_ctzll(hit);
    const KeySeq s = lane_seq(mine, l);
    const int64_t tile = t - lane64(upto - tiles, l), b0 = blocks_before<NW>(a, s, tile), b1 = blocks_before<NW>(a, s, tile + 1);
    const int64_t head = blocks + lane64(n_upto - n, l) + kvh * blocks_before<NW>(a, s, key_tiles<NW>(s)) * a.G;
    const int64_t u0 = head + b0 * a.G, u1 = head + b1 * a.G, w0 = u0 / per, w1 = (u1 - 1) / per;
    if (w0 == w1) return;                             // finished by its workgroup
    f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) dk[db][e] = dv[db][e] = 0.f;
    for (int64_t W = w0; W <= w1; ++W) {
      const f32x4* const part = reinterpret_cast<const f32x4*>(a.part_o) + ((W * 2 + (W == w0 && u0 > w0 * per)) * NW + w) * (D * 16) + lane;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x4 k4 = part[(db * 4 + g) * 64], v4 = part[(D / 8 + db * 4 + g) * 64];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            dk[db][4 * g + e] += k4[e];
            dv[db][4 * g + e] += v4[e];
          }
        }
    }
    const int key = static_cast<int>(tile) * 32 * NW + 32 * w + (lane & 31);
    if (key >= s.nk) return;
    store_row<D>(at(a.dk, s.k0 + key, kvh), dk, a.scale);
    store_row<D>(at(a.dv, s.k0 + key, kvh), dv, 1.f);
    return;
  }
}

constexpr int kMaxSeq = 1 << 16;

}  // namespace pattn
}  // namespace xs

using namespace xs;

namespace {

bool aligned16(const void* p) { return !(reinterpret_cast<uintptr_t>(p) & 15); }

// A tensor of `heads` heads of D values, strides in elements.
int lies(const void* p, int64_t row, int64_t head, int heads, int D) {
  if (!p || !aligned16(p) || row < D || row % 8 || (heads > 1 && (head < D || head % 8 || head >= (int64_t(1) << 40)))) return XS_EINVAL;
  return row > (1 << 23) ? XS_EUNSUPPORTED : XS_OK;
}

pattn::Mat mat(const void* p, int64_t row, int64_t head) { return pattn::Mat{const_cast<char*>(static_cast<const char*>(p)), 2 * row, 2 * head}; }

int check(const xs_attn_packed* A, pattn::Args* a) {
  if (!A || A->n_seq < 1 || A->n_seq > pattn::kMaxSeq || A->heads < 1 || A->kv_heads < 1 || A->heads % A->kv_heads || A->head_dim < 1 ||
      A->Tq < 0 || A->Tk < 0 || A->max_k < 0 || A->max_k > A->Tk || !(A->scale >= 0.f) || !std::isfinite(A->scale) || A->reserved ||
      !A->q_start || !A->k_start)
    return XS_EINVAL;
  const int D = A->head_dim;
  int rc = lies(A->q, A->q_row, A->q_head, A->heads, D);
  for (const int r : {lies(A->k, A->k_row, A->k_head, A->kv_heads, D), lies(A->v, A->v_row, A->v_head, A->kv_heads, D),
                      lies(A->o, A->o_row, A->o_head, A->heads, D)})
    if (rc != XS_EINVAL && r) rc = r;
  if (rc == XS_EINVAL) return rc;
  if (rc || (D != 64 && D != 128) || static_cast<int64_t>(A->Tq) * (A->heads / A->kv_heads) >= (1 << 30) || A->Tk > (1 << 30))
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
  a->Tq = A->Tq;
  a->Tk = A->Tk;
  a->causal = A->causal != 0;
  a->max_k = A->max_k ? A->max_k : A->Tk;
  a->scale = A->scale > 0.f ? A->scale : 1.f / std::sqrt(static_cast<float>(D));
  a->scale_log2e = a->scale * pattn::kLog2e;
  a->lse = A->lse;
  return XS_OK;
}

// Few rows: on average at most 32 a sequence and key head, or 128-row tiles that leave CUs without one.
bool few_rows(const pattn::Args& a) {
  const int64_t rows = static_cast<int64_t>(a.Tq) * a.G;
  return rows <= 32ll * a.n_seq || packed_tiles_bound(a.Tq, a.n_seq, a.G, 128) * a.Hkv <= xs_host::num_cus();
}

template <int D>
int64_t split_bytes() { return static_cast<int64_t>(xs_host::num_cus()) * 4 * 2 * 32 * (D + 2) * 4; }

template <int D>
int forward(pattn::Args a, void* ws, int64_t bytes, hipStream_t st) {
  if (few_rows(a)) {
    if (!ws || !aligned16(ws) || bytes < split_bytes<D>()) return XS_EWORKSPACE;
    const int cus = xs_host::num_cus();
    a.part_o = static_cast<float*>(ws);
    a.part_ml = a.part_o + static_cast<int64_t>(cus) * 4 * 2 * 32 * D;
    hipLaunchKernelGGL((pattn::split_kernel<D>), dim3(cus), dim3(256), 0, st, a);
    if (xs_host::launch_status()) return XS_EHIP;
    const int64_t units = packed_tiles_bound(a.Tq, a.n_seq, a.G, 32) * a.Hkv;
    hipLaunchKernelGGL((pattn::join_kernel<D>), xs_host::grid_of(units), dim3(256), 0, st, a, static_cast<int64_t>(cus) * 4);
  } else {
    const int64_t tiles = packed_tiles_bound(a.Tq, a.n_seq, a.G, 128) * a.Hkv;
    hipLaunchKernelGGL((pattn::rows_kernel<D>), xs_host::grid_of(tiles), dim3(256), 0, st, a);
  }
  return xs_host::launch_status();
}

// Waves of a dkv_kernel workgroup: eight (256 keys, half the rows' traffic) for sequences of 512 keys and more on average, four
// for shorter ones and for heads of 64, where a block of 32 rows is four waves' loads.
template <int D>
int dkv_waves(const pattn::Args& a) { return D == 128 && a.Tk / a.n_seq >= 512 ? 8 : 4; }
template <int D>
int64_t key_tiles_bound(const pattn::Args& a) { return packed_tiles_bound(a.Tk, a.n_seq, 1, 32 * dkv_waves<D>(a)) * a.Hkv; }
// Its workgroups: as many as the chip holds, fewer where there cannot be kLeast blocks for each.
template <int D>
int dkv_ranges(const pattn::Args& a) {
  const int64_t most = (key_tiles_bound<D>(a) * a.G * (a.Tq / 32 + 1) + pattn::kLeast - 1) / pattn::kLeast;
  return static_cast<int>(std::min<int64_t>(most, (D == 128 ? 8 : 12) / dkv_waves<D>(a) * int64_t(xs_host::num_cus())));
}
int64_t delta_bytes(const pattn::Args& a) { return (static_cast<int64_t>(a.H) * a.Tq * 4 + 255) / 256 * 256; }
template <int D>
int64_t grad_bytes(const pattn::Args& a) { return delta_bytes(a) + dkv_ranges<D>(a) * int64_t(2 * 2 * 32 * D * 4) * dkv_waves<D>(a); }

template <int D, int NW>
int dkv(const pattn::Args& a, int ranges, hipStream_t st) {
  hipLaunchKernelGGL((pattn::dkv_kernel<D, NW>), dim3(ranges), dim3(64 * NW), 0, st, a);
  if (xs_host::launch_status()) return XS_EHIP;
  hipLaunchKernelGGL((pattn::dkv_join_kernel<D, NW>), xs_host::grid_of(key_tiles_bound<D>(a)), dim3(64 * NW), 0, st, a, ranges);
  return xs_host::launch_status();
}

template <int D>
int backward(pattn::Args a, void* ws, int64_t bytes, hipStream_t st) {
  const int64_t need = grad_bytes<D>(a);
  if (need && (!ws || !aligned16(ws) || bytes < need)) return XS_EWORKSPACE;
  a.delta = static_cast<float*>(ws);
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + delta_bytes(a));
  if (a.Tq) {
    hipLaunchKernelGGL((pattn::dq_kernel<D>), xs_host::grid_of(packed_tiles_bound(a.Tq, a.n_seq, a.G, 128) * a.Hkv), dim3(256), 0, st, a);
    if (xs_host::launch_status()) return XS_EHIP;
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
  *bytes = a.Tq == 0 || !few_rows(a) ? 0 : A->head_dim == 128 ? split_bytes<128>() : split_bytes<64>();
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
  if (!g || !a.lse) return XS_EINVAL;
  const int D = A->head_dim;
  bool unsupported = a.k_rows != nullptr;
  for (const int r : {lies(g->d_o, g->do_row, g->do_head, a.H, D), lies(g->dq, g->dq_row, g->dq_head, a.H, D),
                      lies(g->dk, g->dk_row, g->dk_head, a.Hkv, D), lies(g->dv, g->dv_row, g->dv_head, a.Hkv, D)}) {
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
