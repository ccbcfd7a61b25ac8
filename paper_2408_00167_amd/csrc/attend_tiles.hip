// Attention of many rows, bf16: 256 stacked rows a workgroup, 32 for each of its eight waves, which walk
// the keys together in tiles of 64.  K and V of a tile lie in LDS, where all waves read them; the next
// tile is on its way from memory to registers meanwhile and goes to a second pair of buffers behind the products, so
// that there is one barrier a tile.  The calculation of a wave is that of attend_rows: S^T = K Q^T, a
// running softmax of a lane's own row, O^T = V^T P^T.  Rows, splits and joins are those of attend_common.h; the tiles
// with the most keys start first.
#include "attend.h"
#include "attend_bf16.h"

namespace finch {

namespace {

constexpr int kThreads = 64 * kTilesWaves;

// A tile of K and V between memory and LDS: this thread's pieces.
template <int D>
struct Staged {
  static constexpr int kMine = kTilesKeys * (D / 8) / kThreads;  // 16-byte pieces of bf16, of K and of V
  u32x4 k[kMine], v[kMine];
  unsigned ks, vs;
};

// Row r of a tile in LDS starts with piece r & 15 (& 7) of K, so that 16 (8) rows read side by side are clear of each other.
template <int D>
__device__ __forceinline__ int k_swap(int r) {
  return r & (D / 8 - 1);
}

template <int D, bool E8>
__device__ __forceinline__ void fetch(Staged<D>& t, const Part& a, int key0, int shift, int tid) {
  if (E8) {
    constexpr int kPer = D / 16;  // pieces of 16 e4m3 numbers
    const int key = min(key0 + min(tid / kPer, kTilesKeys - 1), a.n - 1);
    t.k[0] = as_global<u32x4>(a.k + key * a.row)[tid % kPer];
    t.v[0] = as_global<u32x4>(a.v + key * a.row)[tid % kPer];
    t.ks = as_global<unsigned char>(a.ks)[key >> shift];
    t.vs = as_global<unsigned char>(a.vs)[key >> shift];
  } else {
    constexpr int kPer = D / 8;
#pragma unroll
    for (int i = 0; i < Staged<D>::kMine; ++i) {
      const int id = i * kThreads + tid, key = min(key0 + id / kPer, a.n - 1);
      t.k[i] = as_global<u32x4>(a.k + key * a.row)[id % kPer];
      t.v[i] = as_global<u32x4>(a.v + key * a.row)[id % kPer];
    }
  }
}

template <int D, bool E8>
__device__ __forceinline__ void store(const Staged<D>& t, char* lds_k, char* lds_v, int tid) {
  if (E8) {
    constexpr int kPer = D / 16;
    const int r = tid / kPer, pc = 2 * (tid % kPer);
    if (kPer * kTilesKeys < kThreads && r >= kTilesKeys) return;
    char* k = lds_k + r * (2 * D);
    char* v = lds_v + r * (2 * D);
    *reinterpret_cast<bf16x8*>(k + (pc ^ k_swap<D>(r)) * 16) = widen(t.k[0][0], t.k[0][1], t.ks);
    *reinterpret_cast<bf16x8*>(k + ((pc + 1) ^ k_swap<D>(r)) * 16) = widen(t.k[0][2], t.k[0][3], t.ks);
    *reinterpret_cast<bf16x8*>(v + (pc ^ swap_of<D>(r)) * 16) = widen(t.v[0][0], t.v[0][1], t.vs);
    *reinterpret_cast<bf16x8*>(v + ((pc + 1) ^ swap_of<D>(r)) * 16) = widen(t.v[0][2], t.v[0][3], t.vs);
  } else {
    constexpr int kPer = D / 8;
#pragma unroll
    for (int i = 0; i < Staged<D>::kMine; ++i) {
      const int id = i * kThreads + tid, r = id / kPer, pc = id % kPer;
      *reinterpret_cast<u32x4*>(lds_k + r * (2 * D) + (pc ^ k_swap<D>(r)) * 16) = t.k[i];
      *reinterpret_cast<u32x4*>(lds_v + r * (2 * D) + (pc ^ swap_of<D>(r)) * 16) = t.v[i];
    }
  }
}

}  // namespace

template <int D, bool EIGHT>
__global__ __launch_bounds__(kThreads, 2) void attend_tiles(AttendParams prm) {
  constexpr int kBuf = kTilesKeys * D * 2;
  extern __shared__ __align__(16) char lds[];  // [2][K, V]
  const int p = blockIdx.x % prm.n, rest = blockIdx.x / prm.n, rt = prm.row_tiles - 1 - rest % prm.row_tiles, split = rest / prm.row_tiles;
  const Seen pb(prm, p);
  const int r0 = rt * kTilesRows;
  if (!pb.has(prm, r0)) return;
  const Share sh(prm, pb, r0, kTilesRows, kTilesKeys, split);
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
  const bool idle = w0 >= pb.R;
  int voff[D / 32], koff[D / 16];
  v_offsets<D>(voff, lane);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) koff[s] = row * (2 * D) + ((4 * (s >> 1) + 2 * h + (s & 1)) ^ k_swap<D>(row)) * 16;
  Staged<D> t;
  const auto get = [&](int i) {
    if (EIGHT && eight && i < sh.cache_tiles) {
      fetch<D, true>(t, cache, i * kTilesKeys, prm.block_shift, tid);
    } else {
      const bool in_cache = i < sh.cache_tiles;
      fetch<D, false>(t, in_cache ? cache : chunk, (in_cache ? i : i - sh.cache_tiles) * kTilesKeys, 0, tid);
    }
  };
  const auto put = [&](int i, char* buf) {
    if (EIGHT && eight && i < sh.cache_tiles) {
      store<D, true>(t, buf, buf + kBuf, tid);
    } else {
      store<D, false>(t, buf, buf + kBuf, tid);
    }
  };
  if (sh.first < sh.last) {
    get(sh.first);
    put(sh.first, lds);
  }
  __syncthreads();
  for (int i = sh.first; i < sh.last; ++i) {
    char* buf = lds + ((i - sh.first) & 1) * (2 * kBuf);
    if (i + 1 < sh.last) get(i + 1);
    const bool in_cache = i < sh.cache_tiles;
    const int base = (in_cache ? i : i - sh.cache_tiles) * kTilesKeys, before = in_cache ? 0 : cache.n, n = in_cache ? cache.n : pb.m;
    if (!idle && base < lim_any - before) {
      f32x16 s[2];
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
      if (base + kTilesKeys > min(lim_all - before, n)) {
        const int left = min(lim - before, n) - base;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int v = 0; v < 16; ++v) s[kb][v] = 32 * kb + acc_key(v, h) < left ? s[kb][v] : -kInf;
      }
      weigh<D, 2>(st, s, prm.scale_log2);
      add_values<D, 2>(st, s, buf + kBuf, voff);
    }
    if (i + 1 < sh.last) put(i + 1, lds + ((i + 1 - sh.first) & 1) * (2 * kBuf));
    __syncthreads();
  }
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
    const size_t at = ((static_cast<size_t>(p) * prm.row_tiles + rt) * prm.splits + split) * kTilesRows + wave * 32 + row;
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

hipError_t launch_attend_tiles(int head_dim, bool eight, const AttendParams& p, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(p.n) * p.row_tiles * p.splits), block(kThreads);
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
