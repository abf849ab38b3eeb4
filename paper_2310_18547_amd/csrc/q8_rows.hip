// Row kernels of the 8-bit backbone (gfx950): rms norm with the residual's addition, silu(gate) * up, and plain rows,
// each with an 8-bit output and a scale per row, the first two with a 16-bit output as well.
//
//   norm      s = x + residual;  v = s * rsqrt(mean(s^2) + eps) * weight
//   silu      v = gate / (1 + exp(-gate)) * up
//   quantize  v = x
//   8 bits    top = max |v|;  scale = top / 127;  q = v * (1 / top * 127), rounded to the nearest even
//
// All of it is fp32 between the 16-bit loads and the stores.  A row is read once, kept in registers, reduced (in the norm
// twice: the sum of squares, then the maximum of the normed values) and written.
//
// The maximum is taken of the bit patterns of |v| as unsigned integers, which puts infinities above every number and NaN
// above those: one comparison against the infinity's pattern tells a row that holds something not finite.
//
// Bound by memory (replays over more than 1 GB of inputs and outputs, so that no cache serves them; a copy of 1 GiB reaches 5.1 TB/s):
// 4814 rows of 8192 with residual, sum and both outputs 65 us (5.5 TB/s), silu of 2900 rows of 13824 53 us (5.3), 8190 rows of 4096
// into 8 bits 21 us (4.8; 16380 rows 37 us, 5.5).  A single row by the launch (a norm 3.6 us), some hundred rows, all of them resident
// at once, by one chain of launch, loads, reductions and stores (577 rows of 5128 7.5 us).
#include "device_common.h"
#include "q8.h"

namespace sgmv {

namespace {

constexpr uint32_t kInfBits = 0x7F800000u;

// A sum or a maximum over the workgroup, in every thread.
template <class V, class Join>
__device__ __forceinline__ V reduce_row(V v, V* of_waves, Join join) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = join(v, (V)__shfl_xor(v, m));
  const int waves = blockDim.x >> 6;
  if (waves == 1) return v;
  if ((threadIdx.x & 63) == 0) of_waves[threadIdx.x >> 6] = v;
  __syncthreads();
  v = of_waves[0];
  for (int w = 1; w < waves; ++w) v = join(v, of_waves[w]);
  return v;
}

// One workgroup per row, CHUNKS pieces of eight values to a thread.  grid = rows.
template <class DT, RowsKind KIND, int CHUNKS>
__global__ __launch_bounds__(1024) void rows_q8_kernel(const uint16_t* x, const uint16_t* other,
                                                       const uint16_t* __restrict__ weight, uint16_t* sum_out, uint16_t* out,
                                                       int8_t* q, float* q_scales, int h, float eps) {
  __shared__ float sums[2][16];
  __shared__ uint32_t tops[16];
  const size_t base = (size_t)blockIdx.x * (size_t)h;
  float v[CHUNKS][8];
  uint4 a[CHUNKS], b[CHUNKS];
  uint4 g[KIND == kRowsNorm ? CHUNKS : 1];  // the norm's weights, 16 bits each
  // everything is loaded before anything is stored: outputs may lie where inputs do
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int at = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
    a[c] = b[c] = make_uint4(0, 0, 0, 0);
    if constexpr (KIND == kRowsNorm) g[c] = a[c];
    if (at < h) {
      a[c] = load128(x + base + at);
      if (KIND == kRowsSiluMul || (KIND == kRowsNorm && other != nullptr)) b[c] = load128(other + base + at);
      if constexpr (KIND == kRowsNorm) g[c] = load128(weight + at);
    }
  }
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int at = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
    unpack8<DT>(a[c], v[c]);
    float t[8];
    unpack8<DT>(b[c], t);
    if constexpr (KIND == kRowsNorm) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] += t[i];  // without a residual: + 0
    } else if constexpr (KIND == kRowsSiluMul) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // (1 + exp(-gate)) / 256: the reciprocal instruction gives zero for results under 2^-126, that of 1 + exp(88) is one
        const float d = fmaf(__expf(-v[c][i]), 0x1p-8f, 0x1p-8f);
        v[c][i] = __builtin_amdgcn_rcpf(d) * 0x1p-8f * v[c][i] * t[i];
      }
    }
    if (KIND == kRowsNorm && sum_out != nullptr && at < h)
      store128(sum_out + base + at, make_uint4(pack2<DT>(v[c][0], v[c][1]), pack2<DT>(v[c][2], v[c][3]), pack2<DT>(v[c][4], v[c][5]),
                                               pack2<DT>(v[c][6], v[c][7])));
  }
  if constexpr (KIND == kRowsNorm) {
    auto squares = [&](float* of_waves) {
      float sum = 0.0f;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[c][i] * v[c][i];
      return reduce_row(sum, of_waves, [](float a, float b) { return a + b; });
    };
    const float per = 1.0f / (float)h;
    float mean = squares(sums[0]) * per + eps;
    if (!(mean >= 0x1p-100f && mean < __uint_as_float(kInfBits))) {
      // Values past about 1e18, whose squares leave fp32's range: the row times 2^-80, which the norm does not change by (what
      // is not finite itself stays so).  Values under about 1e-15 next to an eps that does not cover them: times 2^80, as squares
      // lose bits from 2^-126 on (an error of 2^-150 each, nothing next to 2^-100), and are zero below 2^-150.
      const float by = mean < 1.0f ? 0x1p80f : 0x1p-80f;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= by;
      mean = squares(sums[1]) * per + eps * by * by;
    }
    const float inv = rsqrtf(mean);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      float w[8];
      unpack8<DT>(g[c], w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[c][i] = v[c][i] * inv * w[i];
    }
  }
  if (q != nullptr) {
    uint32_t top = 0;  // zeros stand behind the row's end (or NaN, 0 * inv, where inv is infinite and so the row not finite)
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[c][i]) & 0x7FFFFFFFu);
    top = reduce_row(top, tops, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
    const bool finite = top < kInfBits;
    const float peak = __uint_as_float(top);
    if (threadIdx.x == 0) q_scales[blockIdx.x] = finite ? peak / 127.0f : __uint_as_float(0x7FC00000u);
    // 1 / peak leaves fp32's range for the smallest peaks: those rows are made larger first
    const float up = peak < 0x1p-60f ? 0x1p64f : 1.0f;
    const float factor = finite && top != 0 ? 1.0f / (peak * up) * 127.0f : 0.0f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int at = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
      if (at >= h) break;
      uint32_t packed[2] = {0, 0};
      if (finite) {
#pragma unroll
        for (int i = 0; i < 8; ++i) packed[i >> 2] |= ((uint32_t)(int)rintf(v[c][i] * up * factor) & 0xFFu) << (8 * (i & 3));
      }
      *reinterpret_cast<uint2*>(q + base + at) = make_uint2(packed[0], packed[1]);
    }
  }
  if (KIND != kRowsQuantize && out != nullptr) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int at = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
      if (at >= h) break;
      store128(out + base + at, make_uint4(pack2<DT>(v[c][0], v[c][1]), pack2<DT>(v[c][2], v[c][3]), pack2<DT>(v[c][4], v[c][5]),
                                           pack2<DT>(v[c][6], v[c][7])));
    }
  }
}

template <class DT, RowsKind KIND>
hipError_t launch_kind(const RowsArgs& a, hipStream_t st) {
  // Pieces of a row to a thread: two from 4096 wide on, or in large batches from 1024 wide on, one below; four where two are not
  // enough.  One / two / four pieces, us: norm, 4096 wide, 64 rows 4.1 / 4.1 / 4.8, 512 rows 6.8 / 6.4 / 7.6, 8192 rows
  // 58.4 / 57.2 / 58.9; 8192 wide, 768 rows 16.6 / 13.7 / 13.6, 2048 rows 33.7 / 31.4 / 32.4; 2048 wide, 512 rows 4.9 / 5.1 / 6.0,
  // 8192 rows 30.6 / 30.4 / 31.0; plain rows, 4096 wide, 8192 rows 21.0 / 16.9 / 16.9, 1024 wide 7.3 / 6.4 / 6.8; 512 wide, 16384
  // rows 7.0 / 7.2 / 8.1.
  const int pieces = a.h / 8;
  const int chunks = pieces > 2048 ? 4 : pieces >= 512 || (pieces >= 128 && a.n_tokens >= 2048) ? 2 : 1;
  const int threads = ((pieces + chunks - 1) / chunks + 63) / 64 * 64;
  auto launch = [&](auto kernel) -> hipError_t {
    auto at = [](auto* p, size_t offset) { return p == nullptr ? nullptr : p + offset; };
    // a launch takes fewer than 2^32 threads
    const int most = (1 << 30) / threads;
    for (int first = 0; first < a.n_tokens;) {
      const int rows = a.n_tokens - first < most ? a.n_tokens - first : most;
      const size_t offset = (size_t)first * a.h;
      kernel<<<(unsigned)rows, threads, 0, st>>>(at(static_cast<const uint16_t*>(a.x), offset), at(static_cast<const uint16_t*>(a.other), offset),
                                                 static_cast<const uint16_t*>(a.weight), at(static_cast<uint16_t*>(a.sum), offset),
                                                 at(static_cast<uint16_t*>(a.out), offset), at(a.q, offset), at(a.q_scales, (size_t)first),
                                                 a.h, a.eps);
      const hipError_t err = hipGetLastError();
      if (err != hipSuccess) return err;
      first += rows;
    }
    return hipSuccess;
  };
  switch (chunks) {
    case 1: return launch(rows_q8_kernel<DT, KIND, 1>);
    case 2: return launch(rows_q8_kernel<DT, KIND, 2>);
    default: return launch(rows_q8_kernel<DT, KIND, 4>);
  }
}

template <class DT>
hipError_t launch_typed(const RowsArgs& a, hipStream_t st) {
  switch (a.kind) {
    case kRowsNorm: return launch_kind<DT, kRowsNorm>(a, st);
    case kRowsSiluMul: return launch_kind<DT, kRowsSiluMul>(a, st);
    default: return launch_kind<DT, kRowsQuantize>(a, st);
  }
}

}  // namespace

hipError_t launch_rows(const RowsArgs& a, hipStream_t st) {
  return a.bf16 ? launch_typed<BF16>(a, st) : launch_typed<F16>(a, st);
}

}  // namespace sgmv
