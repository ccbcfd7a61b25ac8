// What the bf16 attention kernels share: where rows lie, e4m3 to bf16, the running softmax of a lane's row,
// V^T out of LDS.
#pragma once

#include "attend_common.h"

namespace finch {

typedef __attribute__((address_space(3))) s16x4* lds_tr;

// rows of K or V in memory
struct Part {
  const char* k;
  const char* v;
  long long row;  // bytes
  int n;          // rows
  const unsigned char* ks;
  const unsigned char* vs;
};

// 8 e4m3 numbers times 2^(e - 127) as bf16: exact, one instruction for two.
__device__ __forceinline__ bf16x8 widen(unsigned lo, unsigned hi, unsigned e) {
  const float f = __uint_as_float(e << 23);
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Which piece of row r takes the place of piece 0 in LDS: rows 0..7 (0..3 with 64 channels) differ by two pieces.
template <int D>
__device__ __forceinline__ int swap_of(int r) {
  return 2 * (r & (D == 128 ? 7 : 3));
}

// A tile of 32 keys in a wave's registers: 16-byte pieces of K as the kernel's products take them, and of V as they lie in memory.
template <int D, bool E8>
struct Tile {
  static constexpr int kPieces = D / (E8 ? 32 : 16);  // 16-byte pieces a lane has of K, and of V
  u32x4 k[kPieces], v[kPieces];
  unsigned ks, vs[kPieces];
};

template <int D, bool E8>
__device__ __forceinline__ void load_v(Tile<D, E8>& t, const Part& a, int key0, int shift, int lane) {
  constexpr int kPer = D / (E8 ? 16 : 8);  // pieces of a row
#pragma unroll
  for (int i = 0; i < Tile<D, E8>::kPieces; ++i) {
    const int id = i * 64 + lane, key = min(key0 + id / kPer, a.n - 1);
    t.v[i] = as_global<u32x4>(a.v + key * a.row)[id % kPer];
    if (E8) t.vs[i] = as_global<unsigned char>(a.vs)[key >> shift];
  }
}

template <int D, bool E8>
__device__ __forceinline__ void v_to_lds(const Tile<D, E8>& t, char* lds, int lane) {
  constexpr int kPer = D / (E8 ? 16 : 8);
#pragma unroll
  for (int i = 0; i < Tile<D, E8>::kPieces; ++i) {
    const int id = i * 64 + lane, r = id / kPer, pc = id % kPer;
    char* row = lds + r * (2 * D);
    if (E8) {
      *reinterpret_cast<bf16x8*>(row + ((2 * pc) ^ swap_of<D>(r)) * 16) = widen(t.v[i][0], t.v[i][1], t.vs[i]);
      *reinterpret_cast<bf16x8*>(row + ((2 * pc + 1) ^ swap_of<D>(r)) * 16) = widen(t.v[i][2], t.v[i][3], t.vs[i]);
    } else {
      *reinterpret_cast<u32x4*>(row + (pc ^ swap_of<D>(r)) * 16) = t.v[i];
    }
  }
}

// The rows' state in a lane: reference (log2 domain), sum of the lane's weights, O^T.
template <int D>
struct Rows {
  float ref = -kInf, sum = 0.f;
  f32x16 o[D / 32];
};

// Logits of one row against NB blocks of 32 keys become weights, as the B operands of steps of 16 keys, and their sum goes to the
// lane's.  Weights are rounded once, to the bf16 that products with bf16 values take (the sum has them unrounded): over long rows outputs are
// off by 0.0023 of their norm, 0.0017 with weights of 32 bits, which is the output's own rounding; a product with what the rounding drops
// would be half as many again.  The reference only has to keep the weights in range, and neither fp32 nor bf16 lose
// anything for weights far above one: it is taken from the row's first tile and moved only when a tile's sum in some lane passes
// 2^kSlack, so that most tiles need no maximum.
template <int D, int NB>
__device__ __forceinline__ void weigh(Rows<D>& st, const f32x16* s, bf16x8* pf, float scale) {
  float part[4];
  const auto pass = [&](float ref) {
#pragma unroll
    for (int i = 0; i < 4; ++i) part[i] = 0.f;
#pragma unroll
    for (int b = 0; b < 2 * NB; ++b)
#pragma unroll
      for (int v = 0; v < 8; ++v) {
        const float w = fast_exp2(fmaf(s[b >> 1][8 * (b & 1) + v], scale, -ref));
        part[v & 3] += w;
        pf[b][v] = static_cast<__bf16>(w);
      }
    part[0] = (part[0] + part[1]) + (part[2] + part[3]);
  };
  bool move = __any(st.ref == -kInf);
  if (!move) {
    pass(st.ref);
    move = __any(!(part[0] <= __builtin_exp2f(kSlack)));
  }
  if (move) {
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[kb][v]);
    mx = fmaxf(mx, other_half(mx)) * scale;
    const float ref = fmaxf(st.ref, mx);
    const float f = st.ref == -kInf ? 0.f : fast_exp2(st.ref - ref);
    st.ref = ref;
    st.sum *= f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) st.o[db][v] *= f;
    pass(ref == -kInf ? 0.f : ref);
  }
  st.sum += part[0];
}

// Where a lane reads V^T in LDS: keys 4h + (lane & 15) / 4 of a step of 16, columns of its 16-lane group.
template <int D>
__device__ __forceinline__ void v_offsets(int (&off)[D / 32], int lane) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    const int key = 4 * (lane >> 5) + ((lane & 15) >> 2), pc = 4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    off[db] = key * (2 * D) + (pc ^ swap_of<D>(key)) * 16 + 8 * (lane & 1);
  }
}

// O^T += V^T P^T for NB blocks of 32 keys.
template <int D, int NB>
__device__ __forceinline__ void add_values(Rows<D>& st, const bf16x8* pf, const char* lds, const int (&off)[D / 32]) {
#pragma unroll
  for (int b = 0; b < 2 * NB; ++b) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)(lds + off[db] + (16 * b) * (2 * D)));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)(lds + off[db] + (16 * b + 8) * (2 * D)));
      const s16x8 a = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      st.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), pf[b], st.o[db], 0, 0, 0);
    }
  }
}

}  // namespace finch
