// What the attention kernels share: parameters, a problem's rows and limits, how its keys are cut
// into tiles and splits, and the running softmax of a lane's row.
//
// Rows.  The G query heads of a problem are stacked token by token: row rr is token rr / G, head
// rr % G, so that a tile of rows covers few tokens and its rows see nearly the same candidates.
//
// Keys.  A tile is KT consecutive rows of the cache or of the chunk, never of both; tiles of the
// cache come first.  Rows past a part's last one are read as that one again and masked.  The
// tiles a tile of rows sees are dealt out to `splits` workgroups, `span` tiles each at least;
// what they have is joined by attend_join.
#pragma once

#include "score_common.h"

namespace finch {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

struct AttendParams {
  const finch_attention* descs;
  int32_t n;            // problems
  int32_t group;        // G
  int32_t rows_lo, rows_hi;  // problems with as many stacked rows are this launch's
  int32_t row_tiles;    // of the problem with the most rows
  int32_t splits;       // most workgroups on one tile of rows
  int32_t span;         // tiles of keys a split has at least (but the last)
  int32_t block_shift;  // log2 of the rows per power of two of an 8-bit cache
  float scale_log2;     // log2(e) / sqrt(d_k)
  float* part;          // [n][row_tiles][splits][rows of a tile][D] sums of weighted values ...
  float2* part_ml;      // ... and [n][row_tiles][splits][rows of a tile] (reference, sum of weights)
};

// rows and keys of a tile
constexpr int kRowsTile = 32, kRowsKeys = 32, kRowsWaves = 4;    // attend_rows
constexpr int kF32Tile = 16, kF32Keys = 16, kF32Waves = 4;       // attend_rows_f32
constexpr int kTilesRows = 256, kTilesKeys = 64, kTilesWaves = 8;  // attend_tiles

__device__ __forceinline__ finch_attention load_attention(const finch_attention* p) {
  typedef const __attribute__((address_space(4))) unsigned long long* words;
  struct Raw {
    unsigned long long w[sizeof(finch_attention) / 8];
  } raw;
  static_assert(sizeof(Raw) == sizeof(finch_attention), "descriptors are whole 8-byte words");
  const words src = (words)(unsigned long long)p;
#pragma unroll
  for (unsigned i = 0; i < sizeof(finch_attention) / 8; ++i) raw.w[i] = src[i];
  return __builtin_bit_cast(finch_attention, raw);
}

// A problem as a tile of rows meets it.
struct Seen {
  finch_attention d;
  int m;        // rows of the chunk that are there
  int R;        // stacked rows
  int group;
  __device__ __forceinline__ Seen(const AttendParams& prm, int p) : d(load_attention(prm.descs + p)), group(prm.group) {
    m = d.m;
    if (d.m_live) m = min(m, max(0, uni(*as_global<int>(d.m_live))));
    R = d.n_que * group;
  }
  // whether row r0 is this launch's
  __device__ __forceinline__ bool has(const AttendParams& prm, int r0) const { return R >= prm.rows_lo && R <= prm.rows_hi && r0 < R; }
  // candidates that stacked row rr sees
  __device__ __forceinline__ int limit(int rr) const {
    const int all = d.c + m;
    return d.causal ? max(0, min(all, all - d.n_que + rr / group + 1)) : all;
  }
};

// The tiles of keys of rows [r0, r0 + rows) and the part of them that split s has.
struct Share {
  int cache_tiles, tiles;  // all that the rows see
  int active;              // splits with any
  int first, last;         // this split's
  __device__ __forceinline__ Share(const AttendParams& prm, const Seen& pb, int r0, int rows, int kt, int s) {
    const int lim = pb.limit(min(r0 + rows, pb.R) - 1);
    cache_tiles = (min(lim, pb.d.c) + kt - 1) / kt;
    tiles = cache_tiles + (max(lim - pb.d.c, 0) + kt - 1) / kt;
    active = max(1, min(prm.splits, (tiles + prm.span - 1) / prm.span));
    const int per = (tiles + active - 1) / active;
    first = min(s * per, tiles);
    last = min(first + per, tiles);
  }
};

// The value of the lane 32 further on (or back).
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// Weights may stand up to 2^kSlack above the reference before it is moved: sums stay far
// inside fp32 and bf16, and most tiles need no rescaling of what has been summed.
constexpr float kSlack = 8.f;

inline __device__ float from_log2(float x) { return x * 0.6931471805599453f; }

}  // namespace finch
