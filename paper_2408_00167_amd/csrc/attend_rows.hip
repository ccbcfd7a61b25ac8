// Attention of few rows over many keys, bf16: out = softmax(Q K^T / sqrt(d)) V for 32 stacked rows
// a workgroup, each of whose four waves takes tiles of 32 keys of its own through the whole
// calculation with a running softmax; the waves' results are joined in LDS, those of several
// workgroups on the same rows by attend_join.  A generated token's pass is bound by the bytes of
// the cache, so every row of K and V is read from HBM once, straight into registers.
//
// S^T = K Q^T is one chain of v_mfma_f32_32x32x16_bf16 per tile: K rows are the A operand as they
// lie in memory, and a lane ends up with 16 keys of one row, whose maximum and sum are the
// lane's own but for one exchange with the lane 32 further on.  O^T = V^T P^T takes exactly those
// weights as its B operand if the 16 keys of a step are numbered as the lanes hold them (lane half h:
// keys 4h..4h+3 and 8+4h..8+4h+3), and V^T as the A operand: V goes through 8 KB of LDS of the
// wave's own and comes out transposed by ds_read_b64_tr_b16.  Pieces of 16 bytes are swapped
// by row so that neither side of that meets bank conflicts.  In O^T a lane has one row, so moving
// the softmax's reference is a multiplication by one number a lane.
//
// K of the next tile is under way while the softmax runs, V of the next tile during P V.
#include <algorithm>

#include "attend.h"
#include "attend_bf16.h"

namespace finch {

namespace {

// Lane (t, h) takes of key t, for the pair of k-steps u, channels 32u + 16h .. +15: 16 bytes of e4m3 or two pieces
// of bf16.  (Any order of the channels will do, as long as Q is read in the same.)
template <int D, bool E8>
__device__ __forceinline__ void load_k(Tile<D, E8>& t, const Part& a, int key0, int shift, int lane) {
  const int key = min(key0 + (lane & 31), a.n - 1);
  const FINCH_GLOBAL u32x4* rp = as_global<u32x4>(a.k + key * a.row + (lane >> 5) * (E8 ? 16 : 32));
  if (E8) {
#pragma unroll
    for (int u = 0; u < D / 32; ++u) t.k[u] = rp[2 * u];
    t.ks = as_global<unsigned char>(a.ks)[key >> shift];
  } else {
#pragma unroll
    for (int u = 0; u < D / 32; ++u) {
      t.k[2 * u] = rp[4 * u];
      t.k[(2 * u + 1) % Tile<D, E8>::kPieces] = rp[4 * u + 1];
    }
  }
}

// Tiles first, first + step, ... below last of one part (or, for bf16, of both one after the other).
template <int D, bool E8>
__device__ __forceinline__ void stream(Rows<D>& st, const bf16x8 (&q)[D / 16], const Part& cache, const Part& chunk, int cache_tiles,
                                       int first, int last, int step, int lim, int lim_all, float scale, int shift, char* lds, int lane) {
  if (first >= last) return;
  const int h = lane >> 5;
  Tile<D, E8> t;
  const auto part = [&](int i) -> Part { return i < cache_tiles ? cache : chunk; };
  const auto key0 = [&](int i) { return (i < cache_tiles ? i : i - cache_tiles) * kRowsKeys; };
  int off[D / 32];
  v_offsets<D>(off, lane);
  load_k<D, E8>(t, part(first), key0(first), shift, lane);
  load_v<D, E8>(t, part(first), key0(first), shift, lane);
  for (int i = first; i < last; i += step) {
    const int next = i + step < last ? i + step : i;  // (the last one again: a branch would hide how many loads are pending)
    f32x16 s = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < D / 32; ++u) {
      bf16x8 a, b;
      if (E8) {
        a = widen(t.k[u][0], t.k[u][1], t.ks);
        b = widen(t.k[u][2], t.k[u][3], t.ks);
      } else {
        a = __builtin_bit_cast(bf16x8, t.k[2 * u]);
        b = __builtin_bit_cast(bf16x8, t.k[(2 * u + 1) % Tile<D, E8>::kPieces]);
      }
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[2 * u], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, q[2 * u + 1], s, 0, 0, 0);
    }
    load_k<D, E8>(t, part(next), key0(next), shift, lane);
    // keys past the part's end or the row's limit; lim_all: what every row of the tile sees
    const int base = key0(i), off_c = i < cache_tiles ? 0 : cache.n;
    if (base + kRowsKeys > min(lim_all - off_c, part(i).n)) {
      const int left = min(lim - off_c, part(i).n) - base;
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = acc_key(v, h) < left ? s[v] : -kInf;
    }
    bf16x8 pf[2];
    weigh<D, 1>(st, &s, pf, scale);
    v_to_lds<D, E8>(t, lds, lane);
    load_v<D, E8>(t, part(next), key0(next), shift, lane);
    add_values<D, 1>(st, pf, lds, off);
  }
}

}  // namespace

template <int D, bool EIGHT>
__global__ __launch_bounds__(64 * kRowsWaves, 2) void attend_rows(AttendParams prm) {
  // V of the waves' tiles; later three quarters of every wave's O^T
  constexpr int kQuarter = D / 8;  // values of O^T a wave ends up with, per lane
  __shared__ __align__(16) char lds[kRowsWaves * 3 * kQuarter * 64 * 4];
  __shared__ float ml[2][kRowsWaves][kRowsTile];
  static_assert(sizeof(lds) >= kRowsWaves * kRowsKeys * D * 2, "V tiles of all waves");
  const AttendPiece piece = piece_of(prm, prm.base + blockIdx.x);
  const int split = piece.split;
  const Seen pb(prm, piece.p);
  const int r0 = piece.rt * kRowsTile;
  if (!pb.has(prm, r0)) return;
  const Share sh(prm, pb, r0, kRowsTile, kRowsKeys, split, piece.splits);
  if (split >= sh.active) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), h = lane >> 5;
  const int row = lane & 31, rr = min(r0 + row, pb.R - 1), tok = rr / pb.group, head = rr % pb.group;
  bf16x8 q[D / 16];
  {
    const FINCH_GLOBAL u32x4* qp = as_global<u32x4>(static_cast<const char*>(pb.d.q) + (tok * pb.d.q_row + head * pb.d.q_head) * 2 + 32 * h);
#pragma unroll
    for (int u = 0; u < D / 32; ++u) {
      q[2 * u] = __builtin_bit_cast(bf16x8, qp[4 * u]);
      q[2 * u + 1] = __builtin_bit_cast(bf16x8, qp[4 * u + 1]);
    }
  }
  const bool eight = EIGHT && pb.d.k_scale != nullptr;
  const Part cache = {static_cast<const char*>(pb.d.k_cache), static_cast<const char*>(pb.d.v_cache), pb.d.cache_row * (eight ? 1 : 2), pb.d.c,
                      pb.d.k_scale, pb.d.v_scale};
  const Part chunk = {static_cast<const char*>(pb.d.k_chunk), static_cast<const char*>(pb.d.v_chunk), pb.d.chunk_row * 2, pb.m, nullptr, nullptr};
  Rows<D> st;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) st.o[db][v] = 0.f;
  const int lim = pb.limit(rr), lim_all = pb.limit(r0);
  char* mine = lds + wave * (kRowsKeys * D * 2);
  int first = sh.first + wave;
  if (EIGHT && eight) {
    const int end = min(sh.last, sh.cache_tiles);
    stream<D, true>(st, q, cache, chunk, sh.cache_tiles, first, end, kRowsWaves, lim, lim_all, prm.scale_log2, prm.block_shift, mine, lane);
    first = max(first, first + (end - first + kRowsWaves - 1) / kRowsWaves * kRowsWaves);
  }
  stream<D, false>(st, q, cache, chunk, sh.cache_tiles, first, sh.last, kRowsWaves, lim, lim_all, prm.scale_log2, prm.block_shift, mine, lane);

  // join the waves: wave w ends up with values kQuarter * w .. of every lane's O^T
  st.sum += other_half(st.sum);
  if (h == 0) {
    ml[0][wave][row] = st.ref;
    ml[1][wave][row] = st.sum;
  }
  __syncthreads();
  float top = ml[0][0][row];
#pragma unroll
  for (int w = 1; w < kRowsWaves; ++w) top = fmaxf(top, ml[0][w][row]);
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < kRowsWaves; ++w) total += top == -kInf ? 0.f : ml[1][w][row] * fast_exp2(ml[0][w][row] - top);
  const float f = st.ref == -kInf ? 0.f : fast_exp2(st.ref - top);
  float* ex = reinterpret_cast<float*>(lds);
  float own[kQuarter];
#pragma unroll
  for (int w = 0; w < kRowsWaves; ++w) {
    float* to = ex + (w * 3 + (wave < w ? wave : wave - 1)) * kQuarter * 64 + lane;
#pragma unroll
    for (int x = 0; x < kQuarter; ++x) {
      const int v = w * kQuarter + x;
      const float val = st.o[v >> 4][v & 15] * f;
      if (w == wave) {
        own[x] = val;
      } else {
        to[x * 64] = val;
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kQuarter; ++x) {
    const float* from = ex + wave * 3 * kQuarter * 64 + x * 64 + lane;
#pragma unroll
    for (int w = 0; w < 3; ++w) own[x] += from[w * kQuarter * 64];
  }
  const bool there = r0 + row < pb.R;
  if (sh.active == 1) {
    if (!there) return;
    const float inv = total > 0.f ? 1.f / total : 0.f;
    char* to = static_cast<char*>(pb.d.out) + (tok * pb.d.out_row + head * pb.d.out_head) * 2;
#pragma unroll
    for (int x = 0; x < kQuarter; x += 4) {
      const int v = wave * kQuarter + x, d = 32 * (v >> 4) + 8 * ((v & 15) >> 2) + 4 * h;
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = static_cast<__bf16>(own[x + e] * inv);
      *as_global_mut<bf16x4>(to + 2 * d) = y;
    }
    if (pb.d.lse && wave == 0 && h == 0)
      as_global_mut<float>(pb.d.lse)[head * pb.d.n_que + tok] = total > 0.f ? from_log2(top + fast_log2(total)) : -kInf;
  } else {
    const size_t at = static_cast<size_t>(piece.slot + split) * kRowsTile + row;
    if (there) {
#pragma unroll
      for (int x = 0; x < kQuarter; x += 4) {
        const int v = wave * kQuarter + x, d = 32 * (v >> 4) + 8 * ((v & 15) >> 2) + 4 * h;
        to_others(prm.part + at * D + d, f32x4{own[x], own[x + 1], own[x + 2], own[x + 3]});
      }
      if (wave == 0 && h == 0) to_others(prm.part_ml + at, f32x2{top, total});
    }
    if (prm.meet && last_to_come(prm.meet + piece.slot, sh.active, tid))
      join_splits<D, true, true>(prm, pb, sh.active, at - row - static_cast<size_t>(split) * kRowsTile, kRowsTile, r0, 0, min(kRowsTile, pb.R - r0),
                                 min(kRowsTile, pb.R - r0), ex, tid);
  }
}

// Joins the splits of `per` rows of a tile of rows (see join_splits).
template <int D, bool BF16>
__global__ __launch_bounds__(kJoinThreads) void attend_join(int tile_rows, int tile_keys, int per, int chunks, AttendParams prm) {
  __shared__ float other[kJoinThreads * 6];
  // (a run here has `chunks` workgroups for each tile of rows, problems fastest, and last the last tiles of rows, which may have few: 300 rows
  // of 4 problems on 9000 keys 31.3 us in all, 32.5 the other way round)
  int w = blockIdx.x;
  const AttendRun r = run_of(prm, w);
  const int back = w / (r.count * chunks), at = w - back * r.count * chunks, ch = at / r.count, i = at - ch * r.count, level = r.levels - 1 - back;
  const Seen pb(prm, r.problem + i);
  const int r0 = (r.top - level) * tile_rows;
  if (!pb.has(prm, r0 + ch * per)) return;
  const Share sh(prm, pb, r0, tile_rows, tile_keys, 0, r.splits);
  if (sh.active == 1) return;
  const int rows = min(tile_rows, pb.R - r0), mine = min(per, rows - ch * per);
  join_splits<D, BF16, false>(prm, pb, sh.active, static_cast<size_t>(r.slot + (level * r.count + i) * r.splits) * tile_rows, tile_rows, r0, ch * per, mine,
                              prm.most_splits < kJoinApart ? rows : mine, other, threadIdx.x);
}

hipError_t launch_attend_rows(int head_dim, bool eight, const AttendParams& p, int workgroups, hipStream_t s) {
  const dim3 grid(workgroups), block(64 * kRowsWaves);
  if (head_dim == 128 && eight) {
    hipLaunchKernelGGL((attend_rows<128, true>), grid, block, 0, s, p);
  } else if (head_dim == 128) {
    hipLaunchKernelGGL((attend_rows<128, false>), grid, block, 0, s, p);
  } else if (eight) {
    hipLaunchKernelGGL((attend_rows<64, true>), grid, block, 0, s, p);
  } else {
    hipLaunchKernelGGL((attend_rows<64, false>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

hipError_t launch_attend_join(int head_dim, bool bf16, int tile_rows, int tile_keys, int rows_max, int problems, int tiles, AttendParams& p, hipStream_t s) {
  const int per = p.most_splits >= kJoinApart && static_cast<int64_t>(problems) * rows_max <= 2048 ? 1 : 8;
  const int chunks = (std::min(rows_max, tile_rows) + per - 1) / per;  // of a tile of rows
  for (int i = 0; i < p.runs; ++i) p.start[i] *= chunks;
  const dim3 grid(tiles * chunks), block(kJoinThreads);
  if (head_dim == 128 && bf16) {
    hipLaunchKernelGGL((attend_join<128, true>), grid, block, 0, s, tile_rows, tile_keys, per, chunks, p);
  } else if (head_dim == 128) {
    hipLaunchKernelGGL((attend_join<128, false>), grid, block, 0, s, tile_rows, tile_keys, per, chunks, p);
  } else if (bf16) {
    hipLaunchKernelGGL((attend_join<64, true>), grid, block, 0, s, tile_rows, tile_keys, per, chunks, p);
  } else {
    hipLaunchKernelGGL((attend_join<64, false>), grid, block, 0, s, tile_rows, tile_keys, per, chunks, p);
  }
  return hipGetLastError();
}

}  // namespace finch
