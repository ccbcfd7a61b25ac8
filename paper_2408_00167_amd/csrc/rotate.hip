// From a layer's projections to the rows that scoring and attention read: norm per head, rotary
// embedding, placing (finch_rotate).  Every element is read once and written once; the kernel is
// bound by those bytes.
//
// A workgroup takes a few tokens of one request with all their heads: sine and cosine of a token's
// pairs are computed once (angles reduced in fp64) and shared through LDS.  A thread takes two 16-byte
// pieces of a head, chosen so that it holds both sides of its pairs in either pairing, in turn one
// of the queries', the keys' and the values' heads; the norm's sum goes over the 4, 8 or 16 lanes
// that hold a head.
#include "attend.h"
#include "reposition_common.h"

namespace finch {

namespace {

constexpr int kRotateThreads = 256;

struct RotateParams {
  const finch_rows* descs;
  int32_t group, tokens;  // G; tokens of a workgroup
  int32_t chunks;         // workgroups of the longest request
  finch_rotary how;
};

__device__ __forceinline__ finch_rows load_rows(const finch_rows* p) {
  typedef const __attribute__((address_space(4))) unsigned long long* words;
  struct Raw {
    unsigned long long w[sizeof(finch_rows) / 8];
  } raw;
  static_assert(sizeof(Raw) == sizeof(finch_rows), "descriptors are whole 8-byte words");
  const words src = (words)(unsigned long long)p;
#pragma unroll
  for (unsigned i = 0; i < sizeof(finch_rows) / 8; ++i) raw.w[i] = src[i];
  return __builtin_bit_cast(finch_rows, raw);
}

}  // namespace

template <int D, int E>  // E: elements of a piece
__global__ __launch_bounds__(kRotateThreads) void rotate_rows(RotateParams prm) {
  constexpr int kPieces = D / E, kItems = kPieces / 2;  // of a head: pieces, and pairs of them
  constexpr int kTokens = 4;
  __shared__ float2 turns[kTokens][D / 2];  // (cos, sin), with the gain
  const int p = blockIdx.x / prm.chunks;
  const finch_rows d = load_rows(prm.descs + p);
  const int t0 = (blockIdx.x - p * prm.chunks) * prm.tokens;
  if (t0 >= d.n) return;
  const int nt = min(prm.tokens, d.n - t0), tid = threadIdx.x;
  const bool turning = prm.how.pairing != FINCH_ROPE_OFF;
  const int pairs = turning ? prm.how.dims / 2 : 0;
  for (int i = tid; i < nt * pairs; i += kRotateThreads) {
    const int t = i / pairs, u = i - t * pairs;
    const int at = d.pos ? as_global<int>(d.pos)[t0 + t] : d.pos0 + t0 + t;
    float c, s;
    turn(as_global<double>(prm.how.freq)[u], at, c, s);
    turns[t][u] = make_float2(c * prm.how.gain, s * prm.how.gain);
  }
  __syncthreads();
  // this thread's two pieces of every head it takes (kItems divides the workgroup's size)
  const int j = tid % kItems, turned = turning ? prm.how.dims / E : 0;  // pieces that are rotated, an even number
  const bool rot = j < turned / 2;
  const int pa = rot ? j : turned + 2 * (j - turned / 2), pc = rot ? j + turned / 2 : pa + 1;
  const int hq = d.q ? d.kv_heads * prm.group : 0, hk = d.k ? d.kv_heads : 0, hv = d.v ? d.kv_heads : 0;
  const int heads = hq + hk + hv;
  for (int i = tid / kItems; i < nt * heads; i += kRotateThreads / kItems) {
    const int t = i / heads, hh = i - t * heads, tok = t0 + t;
    const char *src;
    char* dst;
    const void* weight = nullptr;
    bool value = false;
    int row = tok;
    if (hh < hq) {
      src = static_cast<const char*>(d.q) + (tok * d.q_row + hh * d.q_head) * (16 / E);
      dst = static_cast<char*>(d.q_out) + (tok * d.q_out_row + hh * d.q_out_head) * (16 / E);
      weight = prm.how.q_norm;
    } else {
      if (d.slot) {
        row = as_global<int>(d.slot)[tok];
        if (row < 0 || row >= d.slots) row = -1;
      }
      if (hh < hq + hk) {
        const int g = hh - hq;
        src = static_cast<const char*>(d.k) + (tok * d.k_row + g * d.k_head) * (16 / E);
        dst = static_cast<char*>(d.k_out) + (row * d.k_out_row + g * d.k_out_head) * (16 / E);
        weight = prm.how.k_norm;
      } else {
        const int g = hh - hq - hk;
        src = static_cast<const char*>(d.v) + (tok * d.v_row + g * d.v_head) * (16 / E);
        dst = static_cast<char*>(d.v_out) + (row * d.v_out_row + g * d.v_out_head) * (16 / E);
        value = true;
      }
    }
    u32x4 a = as_global<u32x4>(src)[pa], b = as_global<u32x4>(src)[pc];
    if (!value) {
      float x[E], y[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        x[e] = piece_get<E>(a, e);
        y[e] = piece_get<E>(b, e);
      }
      if (weight) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) sq += x[e] * x[e] + y[e] * y[e];
#pragma unroll
        for (int o = 1; o < kItems; o <<= 1) sq += __shfl_xor(sq, o);
        const float f = 1.f / sqrtf(sq * (1.f / D) + prm.how.eps);
        const u32x4 wa = as_global<u32x4>(weight)[pa], wb = as_global<u32x4>(weight)[pc];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          x[e] *= f * piece_get<E>(wa, e);
          y[e] *= f * piece_get<E>(wb, e);
        }
      }
      if (rot && prm.how.pairing == FINCH_ROPE_HALF) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float2 cs = turns[t][E * j + e];
          const float u = x[e], w = y[e];
          x[e] = u * cs.x - w * cs.y;
          y[e] = w * cs.x + u * cs.y;
        }
      } else if (rot) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 ca = turns[t][(E * pa + e) / 2], cb = turns[t][(E * pc + e) / 2];
          const float u = x[e], w = x[e + 1], m = y[e], n = y[e + 1];
          x[e] = u * ca.x - w * ca.y;
          x[e + 1] = w * ca.x + u * ca.y;
          y[e] = m * cb.x - n * cb.y;
          y[e + 1] = n * cb.x + m * cb.y;
        }
      }
      // (what neither the norm nor the rotation has touched goes through bit for bit)
      if (weight || rot) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          piece_set<E>(a, e, x[e]);
          piece_set<E>(b, e, y[e]);
        }
      }
    }
    if (row >= 0) {
      as_global_mut<u32x4>(dst)[pa] = a;
      as_global_mut<u32x4>(dst)[pc] = b;
    }
  }
}

hipError_t launch_rotate(int head_dim, bool bf16, const finch_rotary& how, const finch_rows* descs, int n, int group, int n_max,
                         hipStream_t s) {
  if (n == 0 || n_max == 0) return hipSuccess;
  RotateParams p;
  p.group = group;
  p.how = how;
  p.tokens = n_max >= 4 ? 4 : 1;
  p.chunks = (n_max + p.tokens - 1) / p.tokens;
  // (a launch has fewer than 2^32 threads: enormous batches go in several)
  const int per_launch = (1 << 23) / p.chunks > 0 ? (1 << 23) / p.chunks : 1;
  for (int first = 0; first < n; first += per_launch) {
    p.descs = descs + first;
    const dim3 grid(static_cast<unsigned>(p.chunks) * static_cast<unsigned>(n - first < per_launch ? n - first : per_launch)), block(kRotateThreads);
    if (bf16 && head_dim == 128) {
      hipLaunchKernelGGL((rotate_rows<128, 8>), grid, block, 0, s, p);
    } else if (bf16) {
      hipLaunchKernelGGL((rotate_rows<64, 8>), grid, block, 0, s, p);
    } else if (head_dim == 128) {
      hipLaunchKernelGGL((rotate_rows<128, 4>), grid, block, 0, s, p);
    } else {
      hipLaunchKernelGGL((rotate_rows<64, 4>), grid, block, 0, s, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace finch
