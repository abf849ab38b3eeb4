// Rows into and out of the paged 4-bit cache (gfx950).
//
//   rotation  a' = a cos - b sin,  b' = b cos + a sin   of the pairs of the first rope_dim values, then rounded to 16 bits
//   4 bits    m = min x;  s = (max x - m) / 15, rounded to 16 bits;  c = (x - m) / s, rounded to the nearest even, in [0, 15]
//   back      c * s + m
//
// A head of a row is head_dim / 8 lanes of eight values: one 128-bit load, the reductions within these lanes, one 32-bit store of
// codes.  Every product and sum of the rotation is rounded to fp32 by itself (no fused multiply-add) and quotients are correctly rounded, so
// that a code next to the border of two does not depend on how the compiler joins operations.
//
// Bound by memory: 4184 rows of 64 query and 8 cache heads, 158 MB there and back, 32 us (4.9 TB/s; a copy of 1 GiB reaches 5.1; 36 us with loads that stay in
// the caches, 47 where the lanes of a head load its cosines and sines each time, with divisions); their rows back 7.2 us; one row of 96
// heads 4.2 us, its launch.
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
  if (scale > 0x1p-60f && scale < 0x1p60f) {  // not of a NaN
    // quotients by the correctly rounded reciprocal and two steps of the remainder, which leave them correctly rounded (Markstein): five
    // instructions to a value, a division is a dozen
    const float inverse = 1.0f / scale;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = x[i] - low;
      float q = t * inverse;
      q = fmaf(fmaf(-q, scale, t), inverse, q);
      q = fmaf(fmaf(-q, scale, t), inverse, q);
      codes |= (uint32_t)fminf(rintf(q), 15.0f) << (4 * i);
    }
  } else if (scale > 0.0f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) codes |= (uint32_t)fminf(rintf((x[i] - low) / scale), 15.0f) << (4 * i);
  }
  *codes_at<D>(p, of_v, lane) = codes;
  if (lane == 0) *params_at<D>(p, of_v) = scale_bits | (finite ? encode1<DT>(low) << 16 : 0u);
}

// The words of the lane that holds the other halves of this lane's pairs, `half` lanes away.
template <int D>
__device__ __forceinline__ uint4 other_halves(const uint4& w, int half, int lane_of_head) {
  if (D == 128 && half == 8) {  // all of a row of sixteen lanes: turned by eight
    auto turn = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, true); };
    return make_uint4(turn(w.x), turn(w.y), turn(w.z), turn(w.w));
  }
  const int from = (threadIdx.x & 63) + (lane_of_head < half ? half : lane_of_head < 2 * half ? -half : 0);
  return make_uint4(__shfl(w.x, from), __shfl(w.y, from), __shfl(w.z, from), __shfl(w.w, from));
}

// A wave to a row and `per` of its heads (query heads, then those of k, then those of v), D / 8 lanes to a head: the row's cosines and sines are
// loaded once.  The four rows of a workgroup write the same lines of v's codes where they follow one another in the cache.
// grid = (rows / 4, heads / per).
template <class DT, int D, bool ADJACENT>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a, int first_row, int last_row, int per) {
#pragma clang fp contract(off)
  constexpr int LANES = D / 8, GROUPS = 64 / LANES, AHEAD = 3;
  const int lane = threadIdx.x & (LANES - 1), group = (threadIdx.x & 63) / LANES;
  const long long t = (long long)first_row + blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (t >= last_row) return;
  const int begin = blockIdx.y * per, end = min(begin + per, a.n_heads + 2 * a.at.n_kv_heads);
  const uint32_t slot = (uint32_t)a.slots[t];
  // cosine and sine of each of the lane's values; of the pair's second half the sine is negative
  float cosine[8], sine[8];
  bool turned = false;
  if (a.rope != nullptr) {
    const int pos = a.positions[t];
    if (pos < 0 || pos >= a.rope_rows) return;
    const int half = a.rope_dim >> 1;
    const float* row = a.rope + (size_t)pos * a.rope_dim;
    turned = lane * 8 < a.rope_dim;
    if (turned && ADJACENT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        cosine[2 * i] = cosine[2 * i + 1] = row[lane * 4 + i];
        sine[2 * i] = row[half + lane * 4 + i];
        sine[2 * i + 1] = -sine[2 * i];
      }
    } else if (turned) {
      const bool second = lane * 8 >= half;
      const int first = lane * 8 - (second ? half : 0);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        cosine[i] = row[first + i];
        sine[i] = second ? -row[half + first + i] : row[half + first + i];
      }
    }
  }
  const uint16_t* q_row = a.q + t * a.q_stride + lane * 8;
  const uint16_t* k_row = a.k + t * a.kv_stride + lane * 8;
  const uint16_t* v_row = a.v + t * a.kv_stride + lane * 8;
  for (int base = begin; base < end; base += GROUPS * AHEAD) {
    uint4 words[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int unit = base + k * GROUPS + group, head = unit - a.n_heads;
      words[k] = make_uint4(0, 0, 0, 0);
      if (unit < end)
        words[k] = load128_stream(head < 0 ? q_row + unit * D : head < a.at.n_kv_heads ? k_row + head * D : v_row + (head - a.at.n_kv_heads) * D);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int unit = base + k * GROUPS + group, head = unit - a.n_heads;
      if (base + k * GROUPS >= end) break;
      const bool of_q = head < 0, of_v = head >= a.at.n_kv_heads;
      float x[8];
      unpack8<DT>(words[k], x);
      if (a.rope != nullptr && base + k * GROUPS < a.n_heads + a.at.n_kv_heads) {
        uint4 rounded = words[k];
        float other[8];
        if (ADJACENT) {
#pragma unroll
          for (int i = 0; i < 8; ++i) other[i] = x[i ^ 1];
        } else {
          unpack8<DT>(other_halves<D>(words[k], a.rope_dim >> 4, lane), other);
        }
        if (turned && !of_v) {
          // a cos - b sin and b cos + a sin: products and sums rounded one by one
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float own = x[i] * cosine[i], rest = other[i] * sine[i];
            x[i] = own - rest;
          }
          rounded = pack8<DT>(x);
        }
        if (of_q) store128(a.q_out + t * a.q_out_stride + unit * D + lane * 8, rounded);
        unpack8<DT>(rounded, x);
      }
      if (!of_q && unit < end && slot < a.at.n_slots)
        quantize_row<DT, D>(x, tile_of<D>(a.at, slot, of_v ? head - a.at.n_kv_heads : head), of_v, lane);
    }
  }
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
  constexpr int GROUPS = 64 / (D / 8);
  const int units = a.n_heads + 2 * a.at.n_kv_heads;
  // heads to a wave: as few as there are lanes for in a small batch, else so many that the launch has 128 waves to a unit (4184 rows of 80 heads, 16 / 32 / 64 /
  // 128 / 256 / 512 waves: 40 / 40 / 38 / 36 / 38 / 43 us)
  const int iterations = (units + GROUPS - 1) / GROUPS;
  const long long waves = 128LL * compute_units();
  long long parts = a.n_tokens >= waves ? 1 : waves / a.n_tokens;
  parts = parts < iterations ? parts : iterations;
  const int per = (int)((iterations + parts - 1) / parts) * GROUPS;
  const unsigned columns = (unsigned)((units + per - 1) / per);
  const long long most = (1LL << 21) / columns > 0 ? (1LL << 21) / columns * 4 : 4;  // rows of a launch of at most 2^29 threads
  for (long long first = 0; first < a.n_tokens; first += most) {
    const long long rows = a.n_tokens - first < most ? a.n_tokens - first : most;
    const dim3 grid((unsigned)((rows + 3) / 4), columns);
    if (a.adjacent)
      kv_append_kernel<DT, D, true><<<grid, 256, 0, st>>>(a, (int)first, (int)(first + rows), per);
    else
      kv_append_kernel<DT, D, false><<<grid, 256, 0, st>>>(a, (int)first, (int)(first + rows), per);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
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
