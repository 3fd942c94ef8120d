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

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(v, d);
    if (lane >= d) v += up;
  }
  return v;
}

// The t-th tile of all sequences, ceil(rows mult / per) of each; false past the last. A sequence that does not
// lie in [0, T) sets XS_EBADINPUT and has no tiles. Every wave of a workgroup finds it by itself: 64 sequences a
// step, one a lane, which are two loads and a scan (n_seq <= 64), and no launch before that lists the tiles.
__device__ __forceinline__ bool packed_tile(const int32_t* __restrict__ start, int n_seq, int T, int mult, int per, int t,
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
    const int tiles = static_cast<int>((static_cast<int64_t>(b - a) * mult + per - 1) / per);
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

// At least as many tiles as packed_tile finds, from what the host knows.
inline __host__ int64_t packed_tiles_bound(int64_t T, int64_t n_seq, int64_t mult, int64_t per) {
  const int64_t whole = T * mult / per + n_seq;
  return whole < T * mult ? whole : T * mult;
}

}  // namespace xs
