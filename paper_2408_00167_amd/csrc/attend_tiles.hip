// Attention of many rows, bf16: 256 stacked rows a workgroup, 32 for each of its eight waves, which walk
// the keys together in tiles of 64.  K and V of a tile lie in LDS, where all waves read them, in two buffers each; what
// comes next is on its way from memory to registers meanwhile.  The calculation of a wave is that of attend_rows: S^T = K Q^T, a
// running softmax of a lane's own row, O^T = V^T P^T.  Rows, splits and joins are those of attend_common.h; the tiles
// with the most keys start first.
//
// A tile costs a wave as many cycles of the matrix pipe (32 products) as of the vector unit (32 exponentials a lane and what
// belongs to them), so the two waves of a SIMD take turns: the first four waves make their products - S of the next
// tile and P V of this one - while the others weigh, and the other way round, with a barrier at each change.  All
// eight in step left both pipes idle half of the time (4096 rows of 32 heads on 1364 kept rows of 8: 235 us).
#include "attend.h"
#include "attend_bf16.h"

namespace finch {

namespace {

constexpr int kThreads = 64 * kTilesWaves;

// A tile of K or of V between memory and LDS: this thread's 16-byte pieces, of bf16 or of e4m3.
template <int D>
struct Staged {
  static constexpr int kMine = kTilesKeys * (D / 8) / kThreads, kMine8 = (kMine + 1) / 2;
  u32x4 x[kMine];
  unsigned e[kMine8];
};

// Row r of a tile in LDS starts with piece r & 15 (& 7) of K, so that 16 (8) rows read side by side are clear of each other;
// V as swap_of says.
template <int D, bool V>
__device__ __forceinline__ int swap_in(int r) {
  return V ? swap_of<D>(r) : r & (D / 8 - 1);
}

// MAY: the rows may be e4m3 (`eight`); then all loads are made for either kind, and some of them for nothing: a branch around
// loads makes the wave wait for them where it ends (96 rows on 10000 keys of 128 heads in 8 bits: 160 us, 255 with one).
template <int D, bool MAY>
__device__ __forceinline__ void fetch(Staged<D>& t, bool eight, const char* rows, long long row, int n, const unsigned char* exps, int key0, int shift,
                                      int tid) {
  constexpr int kPer = D / 8;  // pieces of a row of bf16; e4m3: half
  const int per = MAY && eight ? kPer / 2 : kPer, log_per = MAY && eight ? __builtin_ctz(kPer / 2) : __builtin_ctz(kPer);
#pragma unroll
  for (int i = 0; i < Staged<D>::kMine; ++i) {
    const int id = i * kThreads + tid, key = min(key0 + min(id >> log_per, kTilesKeys - 1), n - 1);
    t.x[i] = as_global<u32x4>(rows + key * row)[id & (per - 1)];
    if (MAY && i < Staged<D>::kMine8) t.e[i] = as_global<unsigned char>(eight ? exps : reinterpret_cast<const unsigned char*>(rows))[eight ? key >> shift : 0];
  }
}

template <int D, bool E8, bool V>
__device__ __forceinline__ void store(const Staged<D>& t, char* lds, int tid) {
  constexpr int kPer = D / (E8 ? 16 : 8);
#pragma unroll
  for (int i = 0; i < (E8 ? Staged<D>::kMine8 : Staged<D>::kMine); ++i) {
    const int id = i * kThreads + tid, r = id / kPer, pc = id % kPer;
    if (kPer * kTilesKeys < kThreads && r >= kTilesKeys) return;
    char* to = lds + r * (2 * D);
    if (E8) {
      *reinterpret_cast<bf16x8*>(to + ((2 * pc) ^ swap_in<D, V>(r)) * 16) = widen(t.x[i][0], t.x[i][1], t.e[i]);
      *reinterpret_cast<bf16x8*>(to + ((2 * pc + 1) ^ swap_in<D, V>(r)) * 16) = widen(t.x[i][2], t.x[i][3], t.e[i]);
    } else {
      *reinterpret_cast<u32x4*>(to + (pc ^ swap_in<D, V>(r)) * 16) = t.x[i];
    }
  }
}

}  // namespace

template <int D, bool EIGHT>
__global__ __launch_bounds__(kThreads, 2) void attend_tiles(AttendParams prm) {
  constexpr int kBuf = kTilesKeys * D * 2;
  extern __shared__ __align__(16) char lds[];  // two tiles of K, two of V
  const AttendPiece piece = piece_of(prm, prm.base + blockIdx.x);
  const int split = piece.split;
  const Seen pb(prm, piece.p);
  const int r0 = piece.rt * kTilesRows;
  if (!pb.has(prm, r0)) return;
  const Share sh(prm, pb, r0, kTilesRows, kTilesKeys, split, piece.splits);
  if (split >= sh.active) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), h = lane >> 5;
  const int w0 = r0 + wave * 32, row = lane & 31, rr = min(w0 + row, pb.R - 1), tok = rr / pb.group, head = rr % pb.group;
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
  // what the row, the first and the last row of the wave see
  const int lim = pb.limit(rr), lim_all = uni(pb.limit(min(w0, pb.R - 1))), lim_any = uni(pb.limit(min(w0 + 31, pb.R - 1)));
  int voff[D / 32], koff[D / 16];
  v_offsets<D>(voff, lane);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) koff[s] = row * (2 * D) + ((4 * (s >> 1) + 2 * h + (s & 1)) ^ swap_in<D, false>(row)) * 16;
  // tiles are numbered from the split's first on; the wave sees the first `mine` of them
  const int all = sh.last - sh.first, late = wave >> 2;
  const int seen = (min(lim_any, cache.n) + kTilesKeys - 1) / kTilesKeys + (max(lim_any - cache.n, 0) + kTilesKeys - 1) / kTilesKeys;
  const int mine = w0 < pb.R ? min(seen - sh.first, all) : 0;
  char* const lds_v = lds + 2 * kBuf;
  Staged<D> tk, tv;
  const auto get = [&](Staged<D>& t, int j, bool v) {
    if (j >= all) return;
    const int i = sh.first + j;
    const bool in_cache = i < sh.cache_tiles;
    const Part& a = in_cache ? cache : chunk;
    fetch<D, EIGHT>(t, EIGHT && eight && in_cache, v ? a.v : a.k, a.row, a.n, v ? cache.vs : cache.ks, (in_cache ? i : i - sh.cache_tiles) * kTilesKeys,
                    prm.block_shift, tid);
  };
  const auto put_k = [&](int j) {
    if (j >= all) return;
    if (EIGHT && eight && sh.first + j < sh.cache_tiles) {
      store<D, true, false>(tk, lds + (j & 1) * kBuf, tid);
    } else {
      store<D, false, false>(tk, lds + (j & 1) * kBuf, tid);
    }
  };
  const auto put_v = [&](int j) {
    if (j >= all) return;
    if (EIGHT && eight && sh.first + j < sh.cache_tiles) {
      store<D, true, true>(tv, lds_v + (j & 1) * kBuf, tid);
    } else {
      store<D, false, true>(tv, lds_v + (j & 1) * kBuf, tid);
    }
  };
  f32x16 s[2];
  bf16x8 pf[4];
  const auto logits = [&](int j) {
    if (j >= mine) return;
    const char* buf = lds + (j & 1) * kBuf;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[kb][v] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      const bf16x8 k0 = *reinterpret_cast<const bf16x8*>(buf + koff[c]);
      const bf16x8 k1 = *reinterpret_cast<const bf16x8*>(buf + koff[c] + 32 * (2 * D));
      s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0, q[c], s[0], 0, 0, 0);
      s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k1, q[c], s[1], 0, 0, 0);
    }
  };
  const auto weights = [&](int j) {
    if (j >= mine) return;
    const int i = sh.first + j;
    const bool in_cache = i < sh.cache_tiles;
    const int base = (in_cache ? i : i - sh.cache_tiles) * kTilesKeys, before = in_cache ? 0 : cache.n, n = in_cache ? cache.n : pb.m;
    if (base + kTilesKeys > min(lim_all - before, n)) {
      const int left = min(lim - before, n) - base;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v) s[kb][v] = 32 * kb + acc_key(v, h) < left ? s[kb][v] : -kInf;
    }
    weigh<D, 2>(st, s, pf, prm.scale_log2);
  };
  get(tk, 0, false);
  get(tv, 0, true);
  put_k(0);
  put_v(0);
  get(tk, 1, false);
  put_k(1);
  __syncthreads();
  get(tk, 2, false);
  get(tv, 1, true);
  logits(0);
  weights(0);
  __syncthreads();
  // From here on the late waves are one turn behind the others.  In turn 2j the first ones make the products with K of tile j + 1
  // and V of tile j, in turn 2j + 1 the late ones do.  K of tile j + 2 and V of tile j + 1 go to the buffers of tiles j and
  // j - 1, which were read last in turn 2j - 1: the late waves' part in turn 2j, the others' in turn 2j + 1.
  if (late) {
    put_k(2);
    put_v(1);
    get(tk, 3, false);
    get(tv, 2, true);
    __syncthreads();
  }
  for (int j = 0; j < all; ++j) {
    __builtin_amdgcn_s_setprio(1);
    logits(j + 1);
    if (j < mine) add_values<D, 2>(st, pf, lds_v + (j & 1) * kBuf, voff);
    __builtin_amdgcn_s_setprio(0);
    __syncthreads();
    put_k(j + 2 + late);
    put_v(j + 1 + late);
    get(tk, j + 3 + late, false);
    get(tv, j + 2 + late, true);
    weights(j + 1);
    __syncthreads();
  }
  if (!late) __syncthreads();
  if (w0 + row >= pb.R) return;
  const float total = st.sum + other_half(st.sum);
  const bool whole = sh.active == 1;
  if (whole) {
    const float inv = total > 0.f ? 1.f / total : 0.f;
    char* to = static_cast<char*>(pb.d.out) + (tok * pb.d.out_row + head * pb.d.out_head) * 2;
#pragma unroll
    for (int v = 0; v < D / 2; v += 4) {
      const int d = 32 * (v >> 4) + 8 * ((v & 15) >> 2) + 4 * h;
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = static_cast<__bf16>(st.o[v >> 4][(v & 15) + e] * inv);
      *as_global_mut<bf16x4>(to + 2 * d) = y;
    }
    if (pb.d.lse && h == 0)
      as_global_mut<float>(pb.d.lse)[head * pb.d.n_que + tok] = total > 0.f ? from_log2(st.ref + fast_log2(total)) : -kInf;
  } else {
    const size_t at = static_cast<size_t>(piece.slot + split) * kTilesRows + wave * 32 + row;
    float* to = prm.part + at * D;
#pragma unroll
    for (int v = 0; v < D / 2; v += 4) {
      const int d = 32 * (v >> 4) + 8 * ((v & 15) >> 2) + 4 * h;
      *as_global_mut<f32x4>(to + d) = f32x4{st.o[v >> 4][v & 15], st.o[v >> 4][(v & 15) + 1], st.o[v >> 4][(v & 15) + 2], st.o[v >> 4][(v & 15) + 3]};
    }
    if (h == 0) *as_global_mut<f32x2>(prm.part_ml + at) = f32x2{st.ref, total};
  }
}

hipError_t set_max_lds_attend() {
  constexpr int kMost = 2 * 2 * kTilesKeys * 128 * 2;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(attend_tiles<128, true>), hipFuncAttributeMaxDynamicSharedMemorySize, kMost);
  if (e == hipSuccess) e = hipFuncSetAttribute(reinterpret_cast<const void*>(attend_tiles<128, false>), hipFuncAttributeMaxDynamicSharedMemorySize, kMost);
  return e;
}

hipError_t launch_attend_tiles(int head_dim, bool eight, const AttendParams& p, int workgroups, hipStream_t s) {
  const dim3 grid(workgroups), block(kThreads);
  const size_t lds = 2 * 2 * static_cast<size_t>(kTilesKeys) * head_dim * 2;
  if (head_dim == 128 && eight) {
    hipLaunchKernelGGL((attend_tiles<128, true>), grid, block, lds, s, p);
  } else if (head_dim == 128) {
    hipLaunchKernelGGL((attend_tiles<128, false>), grid, block, lds, s, p);
  } else if (eight) {
    hipLaunchKernelGGL((attend_tiles<64, true>), grid, block, lds, s, p);
  } else {
    hipLaunchKernelGGL((attend_tiles<64, false>), grid, block, lds, s, p);
  }
  return hipGetLastError();
}

}  // namespace finch
