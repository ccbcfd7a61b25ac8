// What the attention kernels share: parameters, a problem's rows and limits, how its keys are cut
// into tiles and splits, and the running softmax of a lane's row.
//
// Rows.  The G query heads of a problem are stacked token by token: row rr is token rr / G, head
// rr % G, so that a tile of rows covers few tokens and its rows see nearly the same candidates.
//
// Keys.  A tile is KT consecutive rows of the cache or of the chunk, never of both; tiles of the
// cache come first.  Rows past a part's last one are read as that one again and masked.  The
// tiles a tile of rows sees are dealt out to `splits` workgroups, `span` tiles each at most;
// what they have is joined by attend_join.
//
// Workgroups.  A launch has as many as there are pieces of work: its problems lie in runs of neighbours in the batch that
// have as many tiles of rows and of keys, and each run's workgroups follow those of the run before.
#pragma once

#include "score_common.h"

namespace finch {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

// Tiles of rows top, top - 1, .. (`levels` of them) of `count` problems from `problem` on, each by `splits` workgroups (some of a
// run that stands for unlike problems have nothing to do).
struct AttendRun {
  int32_t problem, count, top, levels;
  int32_t splits;
  int32_t slot;         // where the run's partial results begin (splits > 1)
};
// (The table goes along as kernel arguments: with 64, 2 KB in all, a single token's call that is waited for took 21 to 33 us,
// 21 with 32, and batches of 64 and 128 tokens 222 and 233 us in place of 216 and 232.)
constexpr int kMostRuns = 32;

struct AttendParams {
  const finch_attention* descs;
  int32_t group;        // G
  int32_t rows_lo, rows_hi;  // problems with as many stacked rows are this launch's
  int32_t most_splits;  // of a run
  int32_t span;         // tiles of keys a split has at most
  int32_t block_shift;  // log2 of the rows per power of two of an 8-bit cache
  float scale_log2;     // log2(e) / sqrt(d_k)
  float* part;          // [slots][rows of a tile][D] sums of weighted values: `splits` slots one after the other for each tile of rows ...
  float2* part_ml;      // ... and [slots][rows of a tile] (reference, sum of weights)
  int32_t* meet;        // a counter per slot, at zero between launches: the last split to come joins a tile's; null: attend_join
  int32_t base;         // number of the launch's first workgroup
  int32_t runs;
  AttendRun one;             // the only run, beside what a workgroup reads first anyway; or, with more of them:
  int32_t start[kMostRuns];  // a run's first workgroup
  AttendRun run[kMostRuns];
};

// The run of workgroup w, whose number in it w becomes.
__host__ __device__ __forceinline__ AttendRun run_of(const AttendParams& prm, int& w) {
  AttendRun r = prm.one;
#ifdef __HIP_DEVICE_COMPILE__
  // (now and together: left to itself the compiler fetches each where it is used, one round trip after the other)
  asm("" : "+s"(r.problem), "+s"(r.count), "+s"(r.top), "+s"(r.levels), "+s"(r.splits), "+s"(r.slot)
      : "s"(prm.descs), "s"(prm.runs), "s"(prm.group), "s"(prm.rows_lo), "s"(prm.rows_hi), "s"(prm.span));
#endif
  if (prm.runs > 1) {
    int e = 0;
#ifdef __HIP_DEVICE_COMPILE__
    static_assert(kMostRuns <= 64, "a run a lane");
    const int lane = threadIdx.x & 63;
    e = uni(static_cast<int>(__popcll(__ballot(lane < prm.runs && prm.start[lane] <= w))) - 1);
#else
    while (e + 1 < prm.runs && prm.start[e + 1] <= w) ++e;
#endif
    r = prm.run[e];
    w -= prm.start[e];
  }
  return r;
}

// What workgroup w has.
struct AttendPiece {
  int p, rt;            // problem, tile of rows
  int split, splits;
  int slot;             // of the tile's first split
};
__host__ __device__ __forceinline__ AttendPiece piece_of(const AttendParams& prm, int w) {
  const AttendRun r = run_of(prm, w);
  const int tiles = r.count * r.levels, split = w / tiles, t = w - split * tiles, level = t / r.count;
  AttendPiece x;
  x.p = r.problem + t - level * r.count;
  x.rt = r.top - level;
  x.split = split;
  x.splits = r.splits;
  x.slot = r.slot + t * r.splits;
  return x;
}

// rows and keys of a tile
constexpr int kRowsTile = 32, kRowsKeys = 32, kRowsWaves = 4;    // attend_rows
constexpr int kRows16 = 16;                                      // attend_rows16 (keys and waves as above)
constexpr int kF32Tile = 16, kF32Keys = 16, kF32Waves = 4;       // attend_rows_f32
constexpr int kJoinThreads = 256;
// From as many splits on, a launch of its own joins them in any call, a row a workgroup where those are few: 4 rows in 32 splits 10.2 us
// and 11.3 if the last split to come did it, 32 rows in 64 splits 36 and 56.  Below, the last split does (5 splits: 8.3 us, 9.4 by a
// launch), or in a captured call a launch that sums in the same order.  A single row is summed in the same order either way, and joined
// by the last split however many there are (128: 21.3 us, 21.7 by a launch).
constexpr int kJoinApart = 16;
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
  __device__ __forceinline__ Share(const AttendParams& prm, const Seen& pb, int r0, int rows, int kt, int s, int splits) {
    const int lim = pb.limit(min(r0 + rows, pb.R) - 1);
    cache_tiles = (min(lim, pb.d.c) + kt - 1) / kt;
    tiles = cache_tiles + (max(lim - pb.d.c, 0) + kt - 1) / kt;
    active = max(1, min(splits, (tiles + prm.span - 1) / prm.span));
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

// How far weights may stand above the reference (log2) before it is moved: the sums of 2^24 of them stay far
// inside fp32.
constexpr float kSlack = 16.f;

__device__ __forceinline__ float from_log2(float x) { return x * 0.6931471805599453f; }

// What a workgroup hands to another one in the same launch goes past the caches of its own part of the chip.
__device__ __forceinline__ void to_others(void* p, f32x2 x) {
  __hip_atomic_store(static_cast<unsigned long long*>(p), __builtin_bit_cast(unsigned long long, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void to_others(float* p, f32x4 x) {
  to_others(p, f32x2{x[0], x[1]});
  to_others(p + 2, f32x2{x[2], x[3]});
}
__device__ __forceinline__ f32x2 from_others(const void* p) {
  return __builtin_bit_cast(f32x2, __hip_atomic_load(static_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Whether this workgroup is the last of `all` to come here, with everything they have handed over in place; called by
// the whole workgroup.  Nobody waits for anybody.  The counter is back at zero afterwards.
__device__ __forceinline__ bool last_to_come(int32_t* counter, int all, int tid) {
  __shared__ int before;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this thread's stores have arrived
  __syncthreads();
  if (tid == 0) before = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (before != all - 1) return false;
  if (tid == 0) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}

// Joins the splits of rows [first, first + n) of a tile that starts with stacked row r0, by a workgroup of kJoinThreads; at0: where
// the tile's results begin.  A thread takes four channels of a row in every `groups`-th split, with a running reference, and the
// groups are joined in LDS: few rows in many splits are read by all threads at once (131000 keys of one request in 125
// splits took 60 us with the splits of a row behind each other).  The order of the sums depends on sizes alone: there are as
// many groups as for a workgroup that joins `together` >= n rows, of which this one may have a part (HANDED: all).
template <int D, bool BF16, bool HANDED>
__device__ __forceinline__ void join_splits(const AttendParams& prm, const Seen& pb, int active, size_t at0, int tile_rows, int r0, int first, int n,
                                            int together, float* other, int tid) {
  const auto at_once = [](int rows) {
    int per = kJoinThreads / (D / 4);
    while (per > 1 && per / 2 >= rows) per >>= 1;
    return per;
  };
  const int per = at_once(n), items = per * (D / 4), groups = kJoinThreads / ((HANDED ? per : at_once(together)) * (D / 4));
  const int g = tid / items, it = tid % items, pc = it % (D / 4);
  for (int b = 0; b < n; b += per) {
    const int row = first + b + it / (D / 4), rr = r0 + row;
    const bool there = b + it / (D / 4) < n && g < groups;
    const float2* ml = prm.part_ml + at0 + row;
    const float* o = prm.part + (at0 + row) * D + 4 * pc;
    float ref = -kInf, total = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    const auto add = [&](float r, float z, f32x4 y) {
      const float to = fmaxf(ref, r), from = to == -kInf ? 0.f : to;
      const float f0 = fast_exp2(ref - from), f1 = fast_exp2(r - from);
      total = fmaf(total, f0, z * f1);  // (written out: every kernel that joins has the same roundings)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(sum[e], f0, y[e] * f1);
      ref = to;
    };
    if (there) {
      constexpr int kBatch = 8;  // splits whose loads are under way together
      for (int s0 = g; s0 < active; s0 += kBatch * groups) {
        f32x2 w[kBatch];
        f32x4 y[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
          const int s = s0 + i * groups;
          const size_t at = static_cast<size_t>(s < active ? s : s0) * tile_rows;
          if (HANDED) {
            w[i] = from_others(ml + at);
            const f32x2 lo = from_others(o + at * D), hi = from_others(o + at * D + 2);
            y[i] = f32x4{lo[0], lo[1], hi[0], hi[1]};
          } else {
            w[i] = *as_global<f32x2>(ml + at);
            y[i] = *as_global<f32x4>(o + at * D);
          }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) add(s0 + i * groups < active ? w[i][0] : -kInf, w[i][1], y[i]);
      }
    }
    if (groups > 1) {
      __syncthreads();
      float* mine = other + tid * 6;
      mine[0] = ref;
      mine[1] = total;
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[2 + e] = sum[e];
      __syncthreads();
      if (g == 0) {
        for (int k = 1; k < groups; ++k) {
          const float* x = mine + k * items * 6;
          add(x[0], x[1], f32x4{x[2], x[3], x[4], x[5]});
        }
      }
    }
    if (g > 0 || !there) continue;
    const float inv = total > 0.f ? 1.f / total : 0.f;
    const int tok = rr / pb.group, head = rr % pb.group;
    const long long to = tok * pb.d.out_row + head * pb.d.out_head + 4 * pc;
    if (BF16) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = static_cast<__bf16>(sum[e] * inv);
      *as_global_mut<bf16x4>(static_cast<char*>(pb.d.out) + 2 * to) = y;
    } else {
      *as_global_mut<f32x4>(static_cast<char*>(pb.d.out) + 4 * to) = f32x4{sum[0] * inv, sum[1] * inv, sum[2] * inv, sum[3] * inv};
    }
    if (pb.d.lse && pc == 0) as_global_mut<float>(pb.d.lse)[head * pb.d.n_que + tok] = total > 0.f ? from_log2(ref + fast_log2(total)) : -kInf;
  }
}

}  // namespace finch
