// Dense projections in 8-bit integers (gfx950):  y[t][c] = (sum_j q[t][j] w[c][j]) * q_scale[t] * w_scale[c].
//
// The products are summed in int32 on the matrix cores, exactly, so the order of the sum does not show in the result.
// v_mfma_i32_16x16x64_i8: lane l of a wave holds row (l % 16), k = 16 (l / 16) .. +15 of the first operand and column
// (l % 16), same k, of the second; it receives D[4 (l / 16) + i][l % 16], i = 0..3.  The channels are the rows of D here
// and the tokens its columns: a lane then holds four consecutive channels of one token and stores them with one access.
#include "device_common.h"
#include "q8.h"

namespace sgmv {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4 mfma_i8(const uint4& a, const uint4& b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// Per-projection pointers of a launch (passed by value as a kernel argument).
struct DenseTable {
  const int8_t* w[kDenseMostProjections];
  const float* w_scales[kDenseMostProjections];
  uint16_t* y[kDenseMostProjections];
  int h_out[kDenseMostProjections];
  int first[kDenseMostProjections + 1];  // channel blocks before each projection, and all of them
};

// Sixteen bytes of a row at k, zeros from h_in on (k and h_in are multiples of 8).
__device__ __forceinline__ uint4 load_row16(const int8_t* row, int k, int h_in) {
  uint2 lo = make_uint2(0, 0), hi = lo;
  if (k < h_in) lo = *reinterpret_cast<const uint2*>(row + k);
  if (k + 8 < h_in) hi = *reinterpret_cast<const uint2*>(row + k + 8);
  return make_uint4(lo.x, lo.y, hi.x, hi.y);
}

// Four channels of a token, scaled and rounded once.
template <class DT>
__device__ __forceinline__ uint2 finish4(i32x4 sum, float q_scale, const float* w_scales) {
  float r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = (float)sum[i] * q_scale * w_scales[i];
    // the compiler would make the last product and the conversion to binary16 one instruction where it sees both, here
    // or there: held apart, all kernels and both types round the same way
    asm("" : "+v"(r[i]));
  }
  return make_uint2(pack2<DT>(r[0], r[1]), pack2<DT>(r[2], r[3]));
}

// 64 tokens x 64 channels per workgroup of four waves, each 32 x 32; 64 bytes of k per step through LDS.
// grid = (channel blocks of all projections, token blocks)
template <class DT>
__global__ __launch_bounds__(256) void dense_q8_tile_kernel(DenseTable t, const int8_t* __restrict__ q,
                                                            const float* __restrict__ q_scales, int n_tokens, int h_in, int n_proj) {
  __shared__ uint4 lds_w[64 * 5], lds_q[64 * 5];  // rows of 64 bytes at a stride of 80
  int p = 0;
  while (p + 1 < n_proj && (int)blockIdx.x >= t.first[p + 1]) ++p;
  const int channels = t.h_out[p], c0 = ((int)blockIdx.x - t.first[p]) * 64, t0 = (int)blockIdx.y * 64;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = threadIdx.x >> 2, piece = threadIdx.x & 3;
  // rows past the end repeat the last one: nothing of them is stored
  const int8_t* w_row = t.w[p] + (size_t)min(c0 + row, channels - 1) * h_in;
  const int8_t* q_row = q + (size_t)min(t0 + row, n_tokens - 1) * h_in;
  const int wc = (wave & 1) * 32, wt = (wave >> 1) * 32;
  i32x4 acc[2][2] = {};
  for (int k = 0; k < h_in; k += 64) {
    const uint4 a = load_row16(w_row, k + piece * 16, h_in), b = load_row16(q_row, k + piece * 16, h_in);
    __syncthreads();
    lds_w[row * 5 + piece] = a;
    lds_q[row * 5 + piece] = b;
    __syncthreads();
    uint4 fa[2], fb[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      fa[i] = lds_w[(wc + i * 16 + (lane & 15)) * 5 + (lane >> 4)];
      fb[i] = lds_q[(wt + i * 16 + (lane & 15)) * 5 + (lane >> 4)];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = mfma_i8(fa[i], fb[j], acc[i][j]);
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int token = t0 + wt + j * 16 + (lane & 15);
    if (token >= n_tokens) continue;
    const float s = q_scales[token];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = c0 + wc + i * 16 + (lane >> 4) * 4;
      if (c < channels)  // widths are multiples of 8: four channels are in or out together
        *reinterpret_cast<uint2*>(t.y[p] + (size_t)token * channels + c) = finish4<DT>(acc[i][j], s, t.w_scales[p] + c);
    }
  }
}

// Channel blocks of `width` channels of all projections.
int fill_table(DenseTable* t, const DenseArgs& a, int width) {
  t->first[0] = 0;
  for (int i = 0; i < a.n_proj; ++i) {
    t->w[i] = a.w[i];
    t->w_scales[i] = a.w_scales[i];
    t->y[i] = static_cast<uint16_t*>(a.y[i]);
    t->h_out[i] = a.h_out[i];
    t->first[i + 1] = t->first[i] + (a.h_out[i] + width - 1) / width;
  }
  return t->first[a.n_proj];
}

template <class DT>
hipError_t launch_typed(const DenseArgs& a, hipStream_t st) {
  DenseTable t = {};
  const dim3 grid((unsigned)fill_table(&t, a, 64), (unsigned)((a.n_tokens + 63) / 64));
  dense_q8_tile_kernel<DT><<<grid, 256, 0, st>>>(t, a.q, a.q_scales, a.n_tokens, a.h_in, a.n_proj);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dense(const DenseArgs& a, hipStream_t st) {
  return a.bf16 ? launch_typed<BF16>(a, st) : launch_typed<F16>(a, st);
}

}  // namespace sgmv
