// Attention of at most 16 stacked rows over many keys, bf16: a generated token of up to 16 heads on one KV head.  As
// attend_rows, with products of 16 rows (v_mfma_f32_16x16x32_bf16): half the registers for queries and results, half the exponentials,
// half of what the waves and splits join.  Bound by the cache's bytes like that one where caches are long; 64 problems of 1000 keys 13.8 -> 12.8 us, in
// 8 bits 11.5 -> 10.4.  (Registers for three workgroups a compute unit in place of two: some of them spilled, 128 requests in 8 bits 238 -> 261 us.)
//
// S^T = K Q^T leaves in lane (row, part) the keys 4 part .. 4 part + 3 of its row, of either block of 16 keys; numbered like that
// they are one B operand of 32 keys for O^T = V^T P^T.
#include "attend.h"
#include "attend_bf16.h"

namespace finch {

namespace {

// Lane (t, part) takes of keys t and 16 + t, for the pair of k-steps u, channels 64u + 16 part .. +15: 16 bytes of e4m3 or two
// pieces of bf16.
template <int D, bool E8>
__device__ __forceinline__ void load_k16(Tile<D, E8>& t, unsigned (&ks)[2], const Part& a, int key0, int shift, int lane) {
  constexpr int kPairs = D / 64;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const int key = min(key0 + 16 * kb + (lane & 15), a.n - 1);
    const FINCH_GLOBAL u32x4* rp = as_global<u32x4>(a.k + key * a.row + (lane >> 4) * (E8 ? 16 : 32));
    if (E8) {
#pragma unroll
      for (int u = 0; u < kPairs; ++u) t.k[kb * kPairs + u] = rp[4 * u];
      ks[kb] = as_global<unsigned char>(a.ks)[key >> shift];
    } else {
#pragma unroll
      for (int u = 0; u < kPairs; ++u) {
        t.k[(kb * kPairs + u) * 2 % Tile<D, E8>::kPieces] = rp[8 * u];
        t.k[((kb * kPairs + u) * 2 + 1) % Tile<D, E8>::kPieces] = rp[8 * u + 1];
      }
    }
  }
}

template <int D>
struct Rows16 {
  float ref = -kInf, sum = 0.f;
  f32x4 o[D / 16];
};

__device__ __forceinline__ float most_of_parts(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, other_half(x));
}

// weigh, for 32 keys against a lane's row of 16.
template <int D>
__device__ __forceinline__ void weigh16(Rows16<D>& st, const f32x4 (&s)[2], bf16x8& pf, float scale) {
  float all;
  const auto pass = [&](float ref) {
    float part[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      const float w = fast_exp2(fmaf(s[v >> 2][v & 3], scale, -ref));
      part[v & 1] += w;
      pf[v] = static_cast<__bf16>(w);
    }
    all = part[0] + part[1];
  };
  bool move = __any(st.ref == -kInf);
  if (!move) {
    pass(st.ref);
    move = __any(!(all <= __builtin_exp2f(kSlack)));
  }
  if (move) {
    float mx = s[0][0];
#pragma unroll
    for (int v = 1; v < 8; ++v) mx = fmaxf(mx, s[v >> 2][v & 3]);
    const float ref = fmaxf(st.ref, most_of_parts(mx) * scale);
    const float f = st.ref == -kInf ? 0.f : fast_exp2(st.ref - ref);
    st.ref = ref;
    st.sum *= f;
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) st.o[db][i] *= f;
    pass(ref == -kInf ? 0.f : ref);
  }
  st.sum += all;
}

template <int D, bool E8>
__device__ __forceinline__ void stream16(Rows16<D>& st, const bf16x8 (&q)[D / 32], const Part& cache, const Part& chunk, int cache_tiles,
                                         int first, int last, int step, int lim, int lim_all, float scale, int shift, char* lds, int lane) {
  if (first >= last) return;
  constexpr int kPairs = D / 64;
  const int part_of = lane >> 4;
  Tile<D, E8> t;
  unsigned ks[2];
  const auto part = [&](int i) -> Part { return i < cache_tiles ? cache : chunk; };
  const auto key0 = [&](int i) { return (i < cache_tiles ? i : i - cache_tiles) * kRowsKeys; };
  // where a lane reads V^T: keys 4 part + (lane & 15) / 4 of a block of 16, columns of its 16-lane group
  const int vkey = 4 * part_of + ((lane & 15) >> 2), vpc = (lane & 3) >> 1;
  load_k16<D, E8>(t, ks, part(first), key0(first), shift, lane);
  load_v<D, E8>(t, part(first), key0(first), shift, lane);
  for (int i = first; i < last; i += step) {
    const int next = i + step < last ? i + step : i;  // (the last one again: a branch would hide how many loads are pending)
    f32x4 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      s[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < kPairs; ++u) {
        bf16x8 a, b;
        if (E8) {
          const u32x4 raw = t.k[kb * kPairs + u];
          a = widen(raw[0], raw[1], ks[kb]);
          b = widen(raw[2], raw[3], ks[kb]);
        } else {
          a = __builtin_bit_cast(bf16x8, t.k[(kb * kPairs + u) * 2 % Tile<D, E8>::kPieces]);
          b = __builtin_bit_cast(bf16x8, t.k[((kb * kPairs + u) * 2 + 1) % Tile<D, E8>::kPieces]);
        }
        s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[2 * u], s[kb], 0, 0, 0);
        s[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, q[2 * u + 1], s[kb], 0, 0, 0);
      }
    }
    load_k16<D, E8>(t, ks, part(next), key0(next), shift, lane);
    const int base = key0(i), off_c = i < cache_tiles ? 0 : cache.n;
    if (base + kRowsKeys > min(lim_all - off_c, part(i).n)) {
      const int left = min(lim - off_c, part(i).n) - base;
#pragma unroll
      for (int v = 0; v < 8; ++v) s[v >> 2][v & 3] = 16 * (v >> 2) + 4 * part_of + (v & 3) < left ? s[v >> 2][v & 3] : -kInf;
    }
    bf16x8 pf;
    weigh16<D>(st, s, pf, scale);
    v_to_lds<D, E8>(t, lds, lane);
    load_v<D, E8>(t, part(next), key0(next), shift, lane);
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      const char* at = lds + vkey * (2 * D) + ((2 * db + vpc) ^ swap_of<D>(vkey)) * 16 + 8 * (lane & 1);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)(at));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)(at + 16 * (2 * D)));
      const s16x8 a = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      st.o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), pf, st.o[db], 0, 0, 0);
    }
  }
}

}  // namespace

template <int D, bool EIGHT>
__global__ __launch_bounds__(64 * kRowsWaves, D == 128 ? 2 : 3) void attend_rows16(AttendParams prm) {
  // V of the waves' tiles; later three quarters of every wave's O^T
  constexpr int kQuarter = D / 16;  // values of O^T a wave ends up with, per lane
  __shared__ __align__(16) char lds[kRowsWaves * kRowsKeys * D * 2];
  __shared__ float ml[2][kRowsWaves][kRows16];
  static_assert(sizeof(lds) >= kRowsWaves * 3 * kQuarter * 64 * 4 && sizeof(lds) >= kJoinThreads * 24, "O^T, join_splits");
  const AttendPiece piece = piece_of(prm, prm.base + blockIdx.x);  // (one tile of rows a problem)
  const int split = piece.split;
  const Seen pb(prm, piece.p);
  if (!pb.has(prm, 0)) return;
  const Share sh(prm, pb, 0, kRows16, kRowsKeys, split, piece.splits);
  if (split >= sh.active) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), part = lane >> 4;
  const int row = lane & 15, rr = min(row, pb.R - 1), tok = rr / pb.group, head = rr % pb.group;
  bf16x8 q[D / 32];
  {
    const FINCH_GLOBAL u32x4* qp = as_global<u32x4>(static_cast<const char*>(pb.d.q) + (tok * pb.d.q_row + head * pb.d.q_head) * 2 + 32 * part);
#pragma unroll
    for (int u = 0; u < D / 64; ++u) {
      q[2 * u] = __builtin_bit_cast(bf16x8, qp[8 * u]);
      q[2 * u + 1] = __builtin_bit_cast(bf16x8, qp[8 * u + 1]);
    }
  }
  const bool eight = EIGHT && pb.d.k_scale != nullptr;
  const Part cache = {static_cast<const char*>(pb.d.k_cache), static_cast<const char*>(pb.d.v_cache), pb.d.cache_row * (eight ? 1 : 2), pb.d.c,
                      pb.d.k_scale, pb.d.v_scale};
  const Part chunk = {static_cast<const char*>(pb.d.k_chunk), static_cast<const char*>(pb.d.v_chunk), pb.d.chunk_row * 2, pb.m, nullptr, nullptr};
  Rows16<D> st;
#pragma unroll
  for (int db = 0; db < D / 16; ++db) st.o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int lim = pb.limit(rr), lim_all = pb.limit(0);
  char* mine = lds + wave * (kRowsKeys * D * 2);
  int first = sh.first + wave;
  if (EIGHT && eight) {
    const int end = min(sh.last, sh.cache_tiles);
    stream16<D, true>(st, q, cache, chunk, sh.cache_tiles, first, end, kRowsWaves, lim, lim_all, prm.scale_log2, prm.block_shift, mine, lane);
    first = max(first, first + (end - first + kRowsWaves - 1) / kRowsWaves * kRowsWaves);
  }
  stream16<D, false>(st, q, cache, chunk, sh.cache_tiles, first, sh.last, kRowsWaves, lim, lim_all, prm.scale_log2, prm.block_shift, mine, lane);

  // join the waves: wave w ends up with values kQuarter * w .. of every lane's O^T
  st.sum += __shfl_xor(st.sum, 16);
  st.sum += other_half(st.sum);
  if (part == 0) {
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
      const float val = st.o[v >> 2][v & 3] * f;
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
  const bool there = row < pb.R;
  if (sh.active == 1) {
    if (!there) return;
    const float inv = total > 0.f ? 1.f / total : 0.f;
    char* to = static_cast<char*>(pb.d.out) + (tok * pb.d.out_row + head * pb.d.out_head) * 2;
#pragma unroll
    for (int x = 0; x < kQuarter; x += 4) {
      const int d = 16 * ((wave * kQuarter + x) >> 2) + 4 * part;
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = static_cast<__bf16>(own[x + e] * inv);
      *as_global_mut<bf16x4>(to + 2 * d) = y;
    }
    if (pb.d.lse && wave == 0 && part == 0)
      as_global_mut<float>(pb.d.lse)[head * pb.d.n_que + tok] = total > 0.f ? from_log2(top + fast_log2(total)) : -kInf;
  } else {
    const size_t at = static_cast<size_t>(piece.slot + split) * kRows16 + row;
    if (there) {
#pragma unroll
      for (int x = 0; x < kQuarter; x += 4)
        to_others(prm.part + at * D + 16 * ((wave * kQuarter + x) >> 2) + 4 * part, f32x4{own[x], own[x + 1], own[x + 2], own[x + 3]});
      if (wave == 0 && part == 0) to_others(prm.part_ml + at, f32x2{top, total});
    }
    if (prm.meet && last_to_come(prm.meet + piece.slot, sh.active, tid))
      join_splits<D, true, true>(prm, pb, sh.active, at - row - static_cast<size_t>(split) * kRows16, kRows16, 0, 0, pb.R, pb.R, ex, tid);
  }
}

hipError_t launch_attend_rows16(int head_dim, bool eight, const AttendParams& p, int workgroups, hipStream_t s) {
  const dim3 grid(workgroups), block(64 * kRowsWaves);
  if (head_dim == 128 && eight) {
    hipLaunchKernelGGL((attend_rows16<128, true>), grid, block, 0, s, p);
  } else if (head_dim == 128) {
    hipLaunchKernelGGL((attend_rows16<128, false>), grid, block, 0, s, p);
  } else if (eight) {
    hipLaunchKernelGGL((attend_rows16<64, true>), grid, block, 0, s, p);
  } else {
    hipLaunchKernelGGL((attend_rows16<64, false>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace finch
