// The compressed cache in 8 bits (finch_quantize): per block of rows of one head the smallest power of
// two with max|x| <= 448 * 2^e, and the e4m3 numbers nearest to x / 2^e.  One pass over the rows: a
// workgroup holds a block of K (or V) in registers from the maximum to the conversion, so
// the kernel moves each element in once and out once and is bound by that.
#include "attend.h"
#include "reposition_common.h"

namespace finch {

namespace {

constexpr int kQuantThreads = 256;

}  // namespace

// B: rows of a block; E: elements of a 16-byte piece.
template <int D, int E, int B>
__global__ __launch_bounds__(kQuantThreads) void quantize_blocks(const finch_quantization* descs, int chunks) {
  constexpr int kPer = D / E, kMine = B * kPer / kQuantThreads > 0 ? B * kPer / kQuantThreads : 1;
  __shared__ unsigned tops[kQuantThreads / 64];
  const int p = blockIdx.x / (2 * chunks), rest = blockIdx.x - p * 2 * chunks, b = rest >> 1;
  const bool val = rest & 1;
  const finch_quantization d = descs[p];
  if (b * B >= d.n) return;
  const int tid = threadIdx.x, rows = min(B, d.n - b * B);
  const char* src = static_cast<const char*>(val ? d.v : d.k) + static_cast<long long>(b) * B * d.in_row * (16 / E);
  u32x4 x[kMine];
  unsigned top = 0;  // bits of the largest |x|: ordered like the numbers
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int id = i * kQuantThreads + tid, r = id / kPer;
    x[i] = u32x4{0, 0, 0, 0};
    if (r < rows) x[i] = as_global<u32x4>(src + r * d.in_row * (16 / E))[id % kPer];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (E == 4) {
        top = max(top, x[i][w] & 0x7FFFFFFFu);
      } else {
        top = max(top, max(x[i][w] & 0x7FFF0000u, (x[i][w] & 0x7FFFu) << 16));
      }
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) top = max(top, static_cast<unsigned>(__shfl_xor(static_cast<int>(top), o)));
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQuantThreads / 64; ++w) top = max(top, tops[w]);
  // 448 = 1.75 * 2^8: one power more where the largest number's fraction is above 1.75.  (Numbers below the
  // normal ones are far under 2^-100 * 448.)
  int e = static_cast<int>(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = top == 0 ? 0 : max(e, -100);
  const float f = __uint_as_float(static_cast<unsigned>(127 - e) << 23);
  unsigned char* dst = (val ? d.v_out : d.k_out) + static_cast<long long>(b) * B * d.out_row;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int id = i * kQuantThreads + tid, r = id / kPer;
    if (r < rows) {
      unsigned w[E / 4];
#pragma unroll
      for (int o = 0; o < E / 4; ++o) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(piece_get<E>(x[i], 4 * o) * f, piece_get<E>(x[i], 4 * o + 1) * f, 0, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(piece_get<E>(x[i], 4 * o + 2) * f, piece_get<E>(x[i], 4 * o + 3) * f, v, true);
        w[o] = static_cast<unsigned>(v);
      }
      FINCH_GLOBAL unsigned* to = as_global_mut<unsigned>(dst + r * d.out_row + (id % kPer) * E);
      if (E == 8) {
        typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
        *reinterpret_cast<FINCH_GLOBAL u32x2*>(to) = u32x2{w[0], w[E / 4 - 1]};
      } else {
        to[0] = w[0];
      }
    }
  }
  if (tid == 0) as_global_mut<unsigned char>(val ? d.v_scale : d.k_scale)[b] = static_cast<unsigned char>(e + 127);
}

namespace {

template <int D, int E>
hipError_t launch_blocks(const finch_quantization* descs, int n, int n_max, int block, hipStream_t s) {
  const int chunks = (n_max + block - 1) / block;
  const int per_launch = (1 << 22) / chunks > 0 ? (1 << 22) / chunks : 1;
  for (int first = 0; first < n; first += per_launch) {
    const int some = n - first < per_launch ? n - first : per_launch;
    const dim3 grid(2u * static_cast<unsigned>(chunks) * static_cast<unsigned>(some)), threads(kQuantThreads);
    if (block == 16) {
      hipLaunchKernelGGL((quantize_blocks<D, E, 16>), grid, threads, 0, s, descs + first, chunks);
    } else if (block == 32) {
      hipLaunchKernelGGL((quantize_blocks<D, E, 32>), grid, threads, 0, s, descs + first, chunks);
    } else if (block == 64) {
      hipLaunchKernelGGL((quantize_blocks<D, E, 64>), grid, threads, 0, s, descs + first, chunks);
    } else {
      hipLaunchKernelGGL((quantize_blocks<D, E, 128>), grid, threads, 0, s, descs + first, chunks);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_quantize(int head_dim, bool bf16, const finch_quantization* descs, int n, int n_max, int block, hipStream_t s) {
  if (n == 0 || n_max == 0) return hipSuccess;
  if (bf16) return head_dim == 128 ? launch_blocks<128, 8>(descs, n, n_max, block, s) : launch_blocks<64, 8>(descs, n, n_max, block, s);
  return head_dim == 128 ? launch_blocks<128, 4>(descs, n, n_max, block, s) : launch_blocks<64, 4>(descs, n, n_max, block, s);
}

}  // namespace finch
