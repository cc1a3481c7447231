// segments.h -- the rows of a product of experts: consecutive segments of one
// matrix, one for each expert, of any lengths (zero included).
//
// Their ends are device data (a routing plan), so a launch cannot be sized by
// them: rows / T + min(n + 1, rows) tiles of T rows are the most that n
// segments and the rows behind the last one can have (each but its last tile is
// whole), and every workgroup finds its tile among those there are.  All lanes
// of a wave take part: lane l holds the segment c + l of a chunk of 64, one
// scan over the lanes gives the tiles before each, and a ballot the one that
// holds the tile.  With up to 63 experts that is one pair of loads and six
// adds; a kernel of its own for a table of tiles would cost a launch (3 us).
//
// Nothing read here can lead a kernel out of its buffers: ends are clamped to
// the matrix, and a segment whose end comes before its beginning is empty.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fastbfp {

enum { kSegNone = 0, kSegRows = 1, kSegK = 2 };

struct Segments {
  const int32_t* offsets;  // n + 1 ends: segment e is [offsets[e], offsets[e + 1])
  int n;                   // segments (experts)
  int rows;                // of the matrix: those from offsets[n] on belong to no segment
};
struct NoSegments {};
template <int SEG> struct SegArg { typedef Segments type; };
template <> struct SegArg<kSegNone> { typedef NoSegments type; };

inline int64_t most_segment_tiles(const Segments& s, int tile) {
  return s.rows / tile + (s.rows < s.n + 1 ? s.rows : s.n + 1);
}

#if defined(__HIPCC__)
// The sum of v over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int v) {
  const int lane = __lane_id();
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(v, d);
    if (lane >= d) v += u;
  }
  return v;
}

// Lane l's segment of the chunk at c (index n: the rows behind the last one):
// its rows and tiles of T.
template <int T>
__device__ __forceinline__ void chunk_segment(const Segments& s, int c, int& lo, int& hi, int& tiles) {
  const int i = c + (int)__lane_id();
  lo = i <= s.n ? min(max(s.offsets[i], 0), s.rows) : s.rows;
  hi = i < s.n ? min(max(s.offsets[i + 1], 0), s.rows) : s.rows;
  tiles = max(hi - lo + T - 1, 0) / T;
}

// Tiles of T rows of all segments and of the rows behind them.
template <int T>
__device__ __forceinline__ int segment_tiles(const Segments& s) {
  int total = 0;
  for (int c = 0; c <= s.n; c += 64) {
    int lo, hi, tiles;
    chunk_segment<T>(s, c, lo, hi, tiles);
    total += __builtin_amdgcn_readlane(wave_scan(tiles), 63);
  }
  return total;
}

struct Segment {
  int index;  // n: the rows behind the last segment; -1: there is no such tile
  int first;  // the tile's first row
  int end;    // the segment's end
};

// Where tile t lies.
template <int T>
__device__ __forceinline__ Segment find_segment(const Segments& s, int t) {
  int before = 0;
  for (int c = 0; c <= s.n; c += 64) {
    int lo, hi, tiles;
    chunk_segment<T>(s, c, lo, hi, tiles);
    const int upto = before + wave_scan(tiles);
    const uint64_t past = __ballot(upto > t);
    if (past) {
      const int l = __builtin_amdgcn_readfirstlane((int)__builtin_ctzll(past));
      return Segment{c + l,
                     __builtin_amdgcn_readlane(lo, l) + (t - __builtin_amdgcn_readlane(upto - tiles, l)) * T,
                     __builtin_amdgcn_readlane(hi, l)};
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return Segment{-1, 0, 0};
}
#endif

}  // namespace fastbfp
