// Attention of fp32 rows: 16 stacked rows a workgroup, each of whose four waves takes tiles of 16 keys of
// its own.  Both products are v_mfma_f32_16x16x4_f32.  S^T = K Q^T leaves in lane (row, part) the
// keys 4 part .. 4 part + 3 of its row; O^T = V^T P^T takes them as they lie, step i with the
// keys 4 part + i, and reads V from memory as its A operand, 16 channels of four keys at a time.
#include "attend.h"

namespace finch {

template <int D>
__global__ __launch_bounds__(64 * kF32Waves) void attend_rows_f32(AttendParams prm) {
  constexpr int kPieces = D / 16, kVals = D / 4, kQuarter = kVals / kF32Waves;
  __shared__ float ex[kF32Waves * 3 * kQuarter * 64];
  static_assert(kF32Waves * 3 * kQuarter * 64 >= kJoinThreads * 6, "join_splits");
  __shared__ float ml[2][kF32Waves][kF32Tile];
  const AttendPiece piece = piece_of(prm, prm.base + blockIdx.x);
  const int split = piece.split;
  const Seen pb(prm, piece.p);
  const int r0 = piece.rt * kF32Tile;
  if (!pb.has(prm, r0)) return;
  const Share sh(prm, pb, r0, kF32Tile, kF32Keys, split, piece.splits);
  if (split >= sh.active) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), row = lane & 15, part = lane >> 4;
  const int rr = min(r0 + row, pb.R - 1), tok = rr / pb.group, head = rr % pb.group;
  // k-element `part` of step s is channel part * D/4 + s, on both sides
  u32x4 q[kPieces];
  {
    const FINCH_GLOBAL u32x4* qp = as_global<u32x4>(static_cast<const char*>(pb.d.q) + (tok * pb.d.q_row + head * pb.d.q_head) * 4) + part * kPieces;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) q[i] = qp[i];
  }
  const int lim = pb.limit(rr);
  float ref = -kInf, sum = 0.f;
  f32x4 o[D / 16];
#pragma unroll
  for (int db = 0; db < D / 16; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int t = sh.first + wave; t < sh.last; t += kF32Waves) {
    const bool in_cache = t < sh.cache_tiles;
    const int base = (in_cache ? t : t - sh.cache_tiles) * kF32Keys, n = in_cache ? pb.d.c : pb.m;
    const long long stride = (in_cache ? pb.d.cache_row : pb.d.chunk_row) * 4;
    const char* kb = static_cast<const char*>(in_cache ? pb.d.k_cache : pb.d.k_chunk);
    const char* vb = static_cast<const char*>(in_cache ? pb.d.v_cache : pb.d.v_chunk);
    const FINCH_GLOBAL u32x4* kp = as_global<u32x4>(kb + min(base + row, n - 1) * stride) + part * kPieces;
    u32x4 k[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) k[i] = kp[i];
    float v[4][D / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const FINCH_GLOBAL float* vp = as_global<float>(vb + min(base + 4 * part + i, n - 1) * stride) + row;
#pragma unroll
      for (int db = 0; db < D / 16; ++db) v[i][db] = vp[16 * db];
    }
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
    for (int s = 0; s < D / 4; s += 2) {
      s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[s >> 2][s & 3]), __uint_as_float(q[s >> 2][s & 3]), s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[s >> 2][(s & 3) + 1]), __uint_as_float(q[s >> 2][(s & 3) + 1]), s1, 0, 0, 0);
    }
    const int left = min(lim - (in_cache ? 0 : pb.d.c), n) - base;
    float w[4], mx = -kInf;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = 4 * part + i < left ? s0[i] + s1[i] : -kInf;
      mx = fmaxf(mx, w[i]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32)) * prm.scale_log2;
    if (__any(mx > ref + kSlack)) {
      const float to = fmaxf(ref, mx), f = ref == -kInf ? 0.f : fast_exp2(ref - to);
      ref = to;
      sum *= f;
#pragma unroll
      for (int db = 0; db < D / 16; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[db][i] *= f;
    }
    const float at = ref == -kInf ? 0.f : ref;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = fast_exp2(fmaf(w[i], prm.scale_log2, -at));
      sum += w[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int db = 0; db < D / 16; ++db) o[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i][db], w[i], o[db], 0, 0, 0);
  }
  // join the waves: wave w ends up with values kQuarter * w .. of every lane's O^T
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if (part == 0) {
    ml[0][wave][row] = ref;
    ml[1][wave][row] = sum;
  }
  __syncthreads();
  float top = ml[0][0][row];
#pragma unroll
  for (int w = 1; w < kF32Waves; ++w) top = fmaxf(top, ml[0][w][row]);
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < kF32Waves; ++w) total += top == -kInf ? 0.f : ml[1][w][row] * fast_exp2(ml[0][w][row] - top);
  const float f = ref == -kInf ? 0.f : fast_exp2(ref - top);
  float own[kQuarter];
#pragma unroll
  for (int w = 0; w < kF32Waves; ++w) {
    float* to = ex + (w * 3 + (wave < w ? wave : wave - 1)) * kQuarter * 64 + lane;
#pragma unroll
    for (int x = 0; x < kQuarter; ++x) {
      const int v = w * kQuarter + x;
      const float val = o[v >> 2][v & 3] * f;
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
  const bool there = r0 + row < pb.R, whole = sh.active == 1;
  const size_t at = static_cast<size_t>(piece.slot + split) * kF32Tile + row;
  if (there) {
    const float inv = total > 0.f ? 1.f / total : 0.f;
    float* to = static_cast<float*>(pb.d.out) + tok * pb.d.out_row + head * pb.d.out_head;
#pragma unroll
    for (int x = 0; x < kQuarter; x += 4) {
      const int d = 16 * ((wave * kQuarter + x) >> 2) + 4 * part;
      if (whole) {
        *as_global_mut<f32x4>(to + d) = f32x4{own[x] * inv, own[x + 1] * inv, own[x + 2] * inv, own[x + 3] * inv};
      } else {
        to_others(prm.part + at * D + d, f32x4{own[x], own[x + 1], own[x + 2], own[x + 3]});
      }
    }
    if (wave == 0 && part == 0) {
      if (!whole) {
        to_others(prm.part_ml + at, f32x2{top, total});
      } else if (pb.d.lse) {
        as_global_mut<float>(pb.d.lse)[head * pb.d.n_que + tok] = total > 0.f ? from_log2(top + fast_log2(total)) : -kInf;
      }
    }
  }
  if (!whole && prm.meet && last_to_come(prm.meet + piece.slot, sh.active, tid))
    join_splits<D, false, true>(prm, pb, sh.active, at - row - static_cast<size_t>(split) * kF32Tile, kF32Tile, r0, 0, min(kF32Tile, pb.R - r0),
                                  min(kF32Tile, pb.R - r0), ex, tid);
}

hipError_t launch_attend_rows_f32(int head_dim, const AttendParams& p, int workgroups, hipStream_t s) {
  const dim3 grid(workgroups), block(64 * kF32Waves);
  if (head_dim == 128) {
    hipLaunchKernelGGL((attend_rows_f32<128>), grid, block, 0, s, p);
  } else {
    hipLaunchKernelGGL((attend_rows_f32<64>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace finch
