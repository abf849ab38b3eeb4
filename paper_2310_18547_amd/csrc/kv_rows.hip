// Rows into and out of the paged 4-bit cache (gfx950).
//
//   rotation  a' = a cos - b sin,  b' = b cos + a sin   of the pairs of the first rope_dim values, then rounded to 16 bits
//   4 bits    m = min x;  s = (max x - m) / 15, rounded to 16 bits;  c = (x - m) / s, rounded to the nearest even, in [0, 15]
//   back      c * s + m
//
// A head of a row is head_dim / 8 lanes of eight values: one 128-bit load, the reductions within these lanes, one 32-bit store of
// codes.  Every product and sum is rounded to fp32 by itself (no fused multiply-add), so that a code next to the border of two does
// not depend on how the compiler joins operations.
#include "device_common.h"
#include "kv.h"

namespace sgmv {

namespace {

constexpr uint32_t kInfBits = 0x7F800000u;

// A slot's tile of a head, and its position in it.
struct TilePlace {
  uint8_t* tile;
  int pos;
};
template <int D>
__device__ __forceinline__ TilePlace tile_of(const KvPlace& at, uint32_t slot, int head) {
  const uint32_t page = slot >> at.page_shift, pos = slot & ((1u << at.page_shift) - 1);
  const size_t tiles = (size_t)((1u << at.page_shift) / kTilePositions);
  return {at.layer + page * at.page_stride + (head * tiles + pos / kTilePositions) * tile_bytes(D), (int)(pos % kTilePositions)};
}
template <int D>
__device__ __forceinline__ uint32_t* codes_at(const TilePlace& p, bool of_v, int lane) {
  return reinterpret_cast<uint32_t*>(p.tile + (of_v ? 8 * D + (p.pos >> 2) * 2 * D + lane * 16 + (p.pos & 3) * 4 : p.pos * (D / 2) + lane * 4));
}
template <int D>
__device__ __forceinline__ uint32_t* params_at(const TilePlace& p, bool of_v) {
  return reinterpret_cast<uint32_t*>(p.tile + 16 * D + (of_v ? 64 : 0) + p.pos * 4);
}

// A lane's eight values of a head rotated; `partner` holds those of the lane that has the pairs' other halves.
template <bool ADJACENT>
__device__ __forceinline__ void rotate(float (&x)[8], const float (&partner)[8], const float* row, int dim, int lane) {
#pragma clang fp contract(off)
  const int half = dim >> 1;
  if (ADJACENT) {
    if (lane * 8 >= dim) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float c = row[lane * 4 + i], s = row[half + lane * 4 + i], a = x[2 * i], b = x[2 * i + 1];
      const float ac = a * c, bs = b * s, bc = b * c, as = a * s;
      x[2 * i] = ac - bs;
      x[2 * i + 1] = bc + as;
    }
    return;
  }
  if (lane * 8 >= dim) return;
  const bool second = lane * 8 >= half;
  const int first = lane * 8 - (second ? half : 0);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = row[first + i], s = row[half + first + i];
    const float own = x[i] * c, other = partner[i] * s;
    x[i] = second ? own + other : own - other;
  }
}

template <class DT>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]), pack2<DT>(x[4], x[5]), pack2<DT>(x[6], x[7]));
}

// One head's row in 4 bits, from all its lanes.
template <class DT, int D>
__device__ __forceinline__ void quantize_row(const float (&x)[8], const TilePlace& p, bool of_v, int lane) {
#pragma clang fp contract(off)
  float low = x[0], high = x[0];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    low = fminf(low, x[i]);
    high = fmaxf(high, x[i]);
    top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int m = 1; m < D / 8; m <<= 1) {
    low = fminf(low, __shfl_xor(low, m));
    high = fmaxf(high, __shfl_xor(high, m));
    top = max(top, (uint32_t)__shfl_xor((int)top, m));
  }
  low += 0.0f;  // of -0 and +0 the latter, whichever lane had it
  const float span = high - low;
  const bool finite = top < kInfBits && __float_as_uint(span) < kInfBits;
  const uint32_t scale_bits = finite ? encode1<DT>(span / 15.0f) : 0x7FFFu;  // a NaN of either type
  const float scale = decode1<DT>((uint16_t)scale_bits);
  uint32_t codes = 0;
  if (finite && scale > 0.0f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) codes |= (uint32_t)fminf(rintf((x[i] - low) / scale), 15.0f) << (4 * i);
  }
  *codes_at<D>(p, of_v, lane) = codes;
  if (lane == 0) *params_at<D>(p, of_v) = scale_bits | (finite ? encode1<DT>(low) << 16 : 0u);
}

// D / 8 lanes to a head of a row: query heads, then those of k, then those of v.  grid.x = items / items of a workgroup.
template <class DT, int D, bool ADJACENT>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a, int first_row, int last_row) {
  constexpr int LANES = D / 8, ITEMS = 256 / LANES;
  const int lane = threadIdx.x % LANES;
  const uint32_t units = a.n_heads + 2 * a.at.n_kv_heads;
  const uint32_t item = blockIdx.x * ITEMS + threadIdx.x / LANES;
  const uint32_t row = item / units;
  const int unit = item - row * units;
  const long long t = (long long)first_row + row;
  if (t >= last_row) return;
  const float* turn = nullptr;
  if (a.rope != nullptr) {
    const int pos = a.positions[t];
    if (pos < 0 || pos >= a.rope_rows) return;
    turn = a.rope + (size_t)pos * a.rope_dim;
  }
  const int head = unit - a.n_heads;
  const bool of_q = head < 0, of_v = head >= a.at.n_kv_heads;
  const uint16_t* from = of_q ? a.q + t * a.q_stride + unit * D : of_v ? a.v + t * a.kv_stride + (head - a.at.n_kv_heads) * D : a.k + t * a.kv_stride + head * D;
  float x[8];
  unpack8<DT>(load128(from + lane * 8), x);
  if (turn != nullptr && !of_v) {
    float partner[8] = {};
    if (!ADJACENT) {
      const int half = a.rope_dim / 16;
      const int at = (threadIdx.x & 63) + (lane < half ? half : lane < 2 * half ? -half : 0);
#pragma unroll
      for (int i = 0; i < 8; ++i) partner[i] = __shfl(x[i], at);
    }
    rotate<ADJACENT>(x, partner, turn, a.rope_dim, lane);
    const uint4 rounded = pack8<DT>(x);
    if (of_q) store128(a.q_out + t * a.q_out_stride + unit * D + lane * 8, rounded);
    unpack8<DT>(rounded, x);
  }
  if (of_q) return;
  const uint32_t slot = (uint32_t)a.slots[t];
  if (slot >= a.at.n_slots) return;
  quantize_row<DT, D>(x, tile_of<D>(a.at, slot, of_v ? head - a.at.n_kv_heads : head), of_v, lane);
}

// The rows of k, then those of v, of all heads.
template <class DT, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadArgs a, int first_row, int last_row) {
#pragma clang fp contract(off)
  constexpr int LANES = D / 8, ITEMS = 256 / LANES;
  const int lane = threadIdx.x % LANES;
  const uint32_t units = 2 * a.at.n_kv_heads;
  const uint32_t item = blockIdx.x * ITEMS + threadIdx.x / LANES;
  const uint32_t row = item / units;
  const int unit = item - row * units;
  const long long t = (long long)first_row + row;
  if (t >= last_row) return;
  const uint32_t slot = (uint32_t)a.slots[t];
  const bool of_v = unit >= a.at.n_kv_heads;
  const int head = of_v ? unit - a.at.n_kv_heads : unit;
  uint16_t* to = of_v ? a.v : a.k;
  if (to == nullptr || slot >= a.at.n_slots) return;
  const TilePlace p = tile_of<D>(a.at, slot, head);
  const uint32_t codes = *codes_at<D>(p, of_v, lane), params = *params_at<D>(p, of_v);
  float scale, low, x[8];
  unpack2<DT>(params, scale, low);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)(codes >> (4 * i) & 15u) * scale + low;
  store128(to + t * a.kv_stride + head * D + lane * 8, pack8<DT>(x));
}

// Launches of fewer than 2^30 threads each, over ranges of rows.
template <class F>
hipError_t by_rows(int n_rows, int units, int items, F launch) {
  const long long most = ((1LL << 30) / 256 * items) / units;
  for (long long first = 0; first < n_rows; first += most) {
    const long long rows = n_rows - first < most ? n_rows - first : most;
    launch((unsigned)((rows * units + items - 1) / items), (int)first, (int)(first + rows));
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

template <class DT, int D>
hipError_t append_typed(const KvAppendArgs& a, hipStream_t st) {
  return by_rows(a.n_tokens, a.n_heads + 2 * a.at.n_kv_heads, 256 / (D / 8), [&](unsigned blocks, int first, int last) {
    if (a.adjacent)
      kv_append_kernel<DT, D, true><<<blocks, 256, 0, st>>>(a, first, last);
    else
      kv_append_kernel<DT, D, false><<<blocks, 256, 0, st>>>(a, first, last);
  });
}

template <class DT, int D>
hipError_t read_typed(const KvReadArgs& a, hipStream_t st) {
  return by_rows(a.n_rows, 2 * a.at.n_kv_heads, 256 / (D / 8),
                 [&](unsigned blocks, int first, int last) { kv_read_kernel<DT, D><<<blocks, 256, 0, st>>>(a, first, last); });
}

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs& a, hipStream_t st) {
  if (a.bf16) return a.at.head_dim == 64 ? append_typed<BF16, 64>(a, st) : append_typed<BF16, 128>(a, st);
  return a.at.head_dim == 64 ? append_typed<F16, 64>(a, st) : append_typed<F16, 128>(a, st);
}

hipError_t launch_kv_read(const KvReadArgs& a, hipStream_t st) {
  if (a.bf16) return a.at.head_dim == 64 ? read_typed<BF16, 64>(a, st) : read_typed<BF16, 128>(a, st);
  return a.at.head_dim == 64 ? read_typed<F16, 64>(a, st) : read_typed<F16, 128>(a, st);
}

}  // namespace sgmv
