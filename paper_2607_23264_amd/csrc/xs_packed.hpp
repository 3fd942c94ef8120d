// Tiles of packed sequences: sequence s has the rows [start[s], start[s + 1]) of a tensor.
#pragma once
#include "xs_common.hpp"

namespace xs {

struct PackedTile {
  int seq;      // its sequence
  int tile;     // its number in the sequence
  int start;    // the sequence's first row
  int rows;     // and its number of rows
};

// Inclusive sum over the wave's lanes: within rows of 16, then each row's last value to the rows behind it. Lanes without a
// source add 0. (With __shfl_up, which goes through LDS, a scan is six round trips of about 100 cycles.)
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp0(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int64_t add_dpp(int64_t v) {
  const uint32_t lo = dpp0<CTRL, ROWS>(static_cast<int>(v)), hi = dpp0<CTRL, ROWS>(static_cast<int>(v >> 32));
  return v + static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int add_dpp(int v) { return v + dpp0<CTRL, ROWS>(v); }
template <class T>
__device__ __forceinline__ T wave_scan(T v) {
  v = add_dpp<0x111>(v);            // row_shr 1, 2, 4, 8
  v = add_dpp<0x112>(v);
  v = add_dpp<0x114>(v);
  v = add_dpp<0x118>(v);
  v = add_dpp<0x142, 0xa>(v);       // row_bcast 15 to rows 1 and 3
  return add_dpp<0x143, 0xc>(v);    // row_bcast 31 to rows 2 and 3
}

// The t-th tile of all sequences, ceil(rows / per) of each; false past the last. A sequence that does not
// lie in [0, T) sets XS_EBADINPUT and has no tiles. Every wave of a workgroup finds it by itself: 64 sequences a
// step, one a lane, which are two loads and a scan (n_seq <= 64), and no launch before that lists the tiles.
__device__ __forceinline__ bool packed_tile(const int32_t* __restrict__ start, int n_seq, int T, int per, int t,
                                            PackedTile* out, int32_t* status) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int s0 = 0; s0 < n_seq; s0 += 64) {
    const int s = s0 + lane;
    int a = 0, b = 0;
    if (s < n_seq) {
      a = start[s];
      b = start[s + 1];
    }
    if (a < 0 || b < a || b > T) {
      set_status(status, XS_EBADINPUT);
      b = a;
    }
    const int tiles = static_cast<int>((static_cast<int64_t>(b - a) + per - 1) / per);
    const int upto = wave_scan(tiles);
    const uint64_t hit = __builtin_amdgcn_ballot_w64(before + upto > t);
    if (hit) {
      const int at = __builtin_ctzll(hit);
      out->seq = s0 + at;
      out->start = __builtin_amdgcn_readlane(a, at);
      out->rows = __builtin_amdgcn_readlane(b, at) - out->start;
      out->tile = t - (before + __builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(tiles, at));
      return true;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// At least as many tiles as sequences of T rows together have, `mult` rows of tiles to a row and `per` to a tile.
inline __host__ int64_t packed_tiles_bound(int64_t T, int64_t n_seq, int64_t mult, int64_t per) {
  const int64_t whole = T * mult / per + n_seq;
  return whole < T * mult ? whole : T * mult;
}

}  // namespace xs
