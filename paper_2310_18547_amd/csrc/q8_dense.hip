// Dense projections in 8-bit integers (gfx950):  y[t][c] = (sum_j q[t][j] w[c][j]) * q_scale[t] * w_scale[c].
//
// The products are summed in int32 on the matrix cores, exactly, so the order of the sum does not show in the result.
// v_mfma_i32_16x16x64_i8: lane l of a wave holds row (l % 16), k = 16 (l / 16) .. +15 of the first operand and column
// (l % 16), same k, of the second; it receives D[4 (l / 16) + i][l % 16], i = 0..3.  The channels are the rows of D here
// and the tokens its columns: a lane then holds four consecutive channels of one token and stores them with one access.
#include <atomic>

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
  int before[kDenseMostProjections];     // channels before each projection
};
struct DenseShape {
  int n_tokens, h_in, n_proj;
  int token_tiles;   // tile kernels
  int splits;        // workgroups that divide the sum of a tile among themselves; from two on they leave it in `partials`
  int all_channels;  // of all projections
  int* partials;
};

// Sixteen bytes of a row at k, zeros from h_in on (k and h_in are multiples of 8).
__device__ __forceinline__ uint4 load_row16(const int8_t* row, int k, int h_in) {
  uint2 lo = make_uint2(0, 0), hi = lo;
  if (k < h_in) lo = *reinterpret_cast<const uint2*>(row + k);
  if (k + 8 < h_in) hi = *reinterpret_cast<const uint2*>(row + k + 8);
  return make_uint4(lo.x, lo.y, hi.x, hi.y);
}

__host__ __device__ inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

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

// N loads, each of sixteen bytes of every lane from `from` + the lane's own offset + a common one into 1024 consecutive bytes of
// LDS, the first to `to` and each STRIDE bytes behind the one before.  In assembly because the compiler, which cannot tell the
// places of the ring apart, waits for every such load in front of every LDS read; arrive() does the waiting.  The loads write no
// register but m0, which nothing else here uses.  The five wait states (s_nop 4) are those that a load needs behind a vector
// instruction that has written one of its scalar operands, which the compiler does not see to in front of assembly.
template <int N, int STRIDE>
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t from, const uint32_t (&lane_off)[N], uint32_t uniform_off, const int8_t* to) {
  const uint32_t at = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(const __attribute__((address_space(3))) int8_t*)to);
  uniform_off = (uint32_t)__builtin_amdgcn_readfirstlane((int)uniform_off);
#pragma unroll
  for (int i = 0; i + 1 < N; i += 2)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds\n\t"
                 "s_add_u32 m0, m0, %5\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %2, %3 offen lds" ::"s"(at + i * STRIDE), "v"(lane_off[i]), "s"(from),
                 "s"(uniform_off), "v"(lane_off[i + 1]), "n"(STRIDE)
                 : "memory", "scc");
  if constexpr (N % 2 != 0)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(at + (N - 1) * STRIDE), "v"(lane_off[N - 1]),
                 "s"(from), "s"(uniform_off)
                 : "memory");
}
// Waits until all but this many of the wave's loads have arrived and its LDS reads are done, then for the other waves.
template <int LEFT>
__device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// A tile of WC x WT waves: WC * NC * 16 channels of WT * NT * 16 tokens, k in steps of 128 bytes (a cache line of every row) that go from
// memory to a ring of DEPTH places in LDS without passing through registers, and from there to the matrix cores.
template <int NC, int NT, int WC, int WT, int DEPTH>
struct DenseTile {
  static constexpr int kWaves = WC * WT, kThreads = 64 * kWaves;
  static constexpr int kChannels = WC * NC * 16, kTokens = WT * NT * 16, kRows = kChannels + kTokens;
  static constexpr int kPlace = kRows * 128, kLds = DEPTH * kPlace;
  // of a wave and step, each eight rows of eight pieces of sixteen bytes
  static constexpr int kLoadsW = kChannels / 8 / kWaves, kLoadsQ = kTokens / 8 / kWaves, kLoads = kLoadsW + kLoadsQ;
  static_assert(kChannels % (8 * kWaves) == 0 && kTokens % (8 * kWaves) == 0, "whole loads");

  // A wave's fragments in LDS: fragment f, row r of the wave's channels is row (r / 4) 4 NC + 4 f + r % 4, so that a lane,
  // which receives rows 4 (l / 16) + i of every fragment, holds 4 NC consecutive channels; the tokens' fragments are
  // rows of sixteen.
  static __device__ __forceinline__ int w_row(int f, int r) { return (r >> 2) * (4 * NC) + f * 4 + (r & 3); }
  // The banks hold 256 bytes, two rows.  The pieces of a row are permuted by what tells the sixteen rows apart that a
  // fragment's read touches at once, so that these lie in different banks (the counter of bank conflicts stays at zero).
  static __device__ __forceinline__ int w_swizzle(int row) { return ((row / (4 * NC) & 3) << 1) | (row >> 1 & 1); }
  static __device__ __forceinline__ int q_swizzle(int row) { return row >> 1 & 7; }
};

// What a wave of a tile kernel works on, and its ways between memory, LDS and registers.
template <class T, int NC, int NT, int WC>
struct DenseWork {
  int lane, wave, channels, c0, t0, last_w, last_q, h_in, n_tokens;
  int split, first, steps;  // of the divided sum: which part, its first step, its whole steps
  bool rest;                // whether the shorter step behind the last whole one is this part's
  const int8_t *w, *x, *my_w, *my_q;
  int8_t* lds;
  int piece_w, piece_q, p;
  __amdgpu_buffer_rsrc_t from_w, from_q;
  uint32_t off_w[T::kLoadsW], off_q[T::kLoadsQ];  // of this lane's piece of a row, from w and x at k = 0

  __device__ __forceinline__ DenseWork(const DenseTable& t, const int8_t* q, const DenseShape& shape, int8_t* lds_)
      : h_in(shape.h_in), n_tokens(shape.n_tokens), lds(lds_) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    // Workgroups are dealt to the XCDs round-robin: every XCD gets a contiguous run of tiles, which go through kGroup token
    // tiles for every channel tile, so that those that run together share rows of both kinds in the XCD's cache.
    constexpr int kGroup = 4;
    int id = (int)blockIdx.x;
    const int total = (int)gridDim.x, each = total / 8, more = total % 8, xcd = id % 8;
    id = xcd * each + min(xcd, more) + id / 8;
    const int tiles = t.first[shape.n_proj] * shape.token_tiles;
    split = id / tiles;
    id -= split * tiles;
    const int per_group = kGroup * t.first[shape.n_proj], group = id / per_group, in_group = id % per_group;
    const int rows_here = min(kGroup, shape.token_tiles - group * kGroup);
    const int token_tile = group * kGroup + in_group % rows_here, channel_tile = in_group / rows_here;
    const int all = h_in / 128;
    first = (int)((long long)all * split / shape.splits);
    steps = (int)((long long)all * (split + 1) / shape.splits) - first;
    rest = split + 1 == shape.splits && h_in % 128 != 0;
    p = 0;
    while (p + 1 < shape.n_proj && channel_tile >= t.first[p + 1]) ++p;
    channels = t.h_out[p];
    c0 = (channel_tile - t.first[p]) * T::kChannels;
    t0 = token_tile * T::kTokens;
    w = t.w[p] + (size_t)c0 * h_in;
    x = q + (size_t)t0 * h_in;
    from_w = make_uniform_buffer(w + (size_t)first * 128, 0x7FFFFFFF);
    from_q = make_uniform_buffer(x + (size_t)first * 128, 0x7FFFFFFF);
    last_w = channels - 1 - c0;  // rows past these repeat them: nothing of them is stored
    last_q = n_tokens - 1 - t0;
    const int piece = lane & 7;
#pragma unroll
    for (int i = 0; i < T::kLoadsW; ++i) {
      const int row = (i * T::kWaves + wave) * 8 + (lane >> 3);
      off_w[i] = (uint32_t)min(row, last_w) * (uint32_t)h_in + (uint32_t)((piece ^ T::w_swizzle(row)) * 16);
    }
#pragma unroll
    for (int i = 0; i < T::kLoadsQ; ++i) {
      const int row = (i * T::kWaves + wave) * 8 + (lane >> 3);
      off_q[i] = (uint32_t)min(row, last_q) * (uint32_t)h_in + (uint32_t)((piece ^ T::q_swizzle(row)) * 16);
    }
    const int rw = wave % WC * NC * 16 + T::w_row(0, lane & 15), rq = wave / WC * NT * 16 + (lane & 15);
    my_w = lds + rw * 128;
    my_q = lds + (T::kChannels + rq) * 128;
    piece_w = ((lane >> 4) ^ T::w_swizzle(rw)) * 16;  // a fragment further on changes no bit that the permutation looks at
    piece_q = ((lane >> 4) ^ T::q_swizzle(rq)) * 16;
  }
  // All of a step into the ring.
  __device__ __forceinline__ void fetch(int step, int place) const {
    load_to_lds<T::kLoadsW, T::kWaves * 1024>(from_w, off_w, (uint32_t)step * 128u, lds + place + wave * 1024);
    load_to_lds<T::kLoadsQ, T::kWaves * 1024>(from_q, off_q, (uint32_t)step * 128u, lds + place + T::kChannels * 128 + wave * 1024);
  }
  // The shorter step at the end into the first place, through registers: zeros behind the rows' ends.
  __device__ __forceinline__ void fetch_rest() const {
    const int k0 = h_in / 128 * 128;
    __syncthreads();
    for (int i = threadIdx.x; i < T::kRows * 8; i += T::kThreads) {
      const int r = i >> 3, piece = i & 7;
      const bool is_w = r < T::kChannels;
      const int row = is_w ? r : r - T::kChannels;
      const int8_t* from = is_w ? w + (size_t)min(row, last_w) * h_in : x + (size_t)min(row, last_q) * h_in;
      *reinterpret_cast<uint4*>(lds + r * 128 + (piece ^ (is_w ? T::w_swizzle(row) : T::q_swizzle(row))) * 16) =
          load_row16(from, k0 + piece * 16, h_in);
    }
    __syncthreads();
  }
  // This wave's fragments of 64 bytes of k, the first or the second of a step.
  __device__ __forceinline__ void read(int place, int half, uint4 (&fw)[NC], uint4 (&fq)[NT]) const {
#pragma unroll
    for (int i = 0; i < NC; ++i) fw[i] = *reinterpret_cast<const uint4*>(my_w + place + i * 512 + (piece_w ^ (half * 64)));
#pragma unroll
    for (int j = 0; j < NT; ++j) fq[j] = *reinterpret_cast<const uint4*>(my_q + place + j * 2048 + (piece_q ^ (half * 64)));
  }
  // y, or the partial sums where several workgroups divide the sum ([split][token][channel of all projections]).
  template <class DT>
  __device__ __forceinline__ void store(const DenseTable& t, const float* q_scales, const DenseShape& shape, const i32x4 (&acc)[NC][NT]) const {
    const int c = c0 + wave % WC * NC * 16 + (lane >> 4) * (4 * NC);  // of this lane's 4 NC channels
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int token = t0 + (wave / WC * NT + j) * 16 + (lane & 15);
      if (token >= n_tokens) continue;
      if (shape.splits > 1) {
        int* part = shape.partials + ((size_t)split * n_tokens + token) * shape.all_channels + t.before[p] + c;
#pragma unroll
        for (int i = 0; i < NC; ++i)
          if (c + 4 * i < channels) *reinterpret_cast<i32x4*>(part + 4 * i) = acc[i][j];
        continue;
      }
      const float s = q_scales[token];
      uint16_t* y = t.y[p] + (size_t)token * channels;
#pragma unroll
      for (int i = 0; i < NC; i += 2)
        if (c + 4 * i < channels) {  // widths are multiples of 8: eight channels are in or out together
          const uint2 lo = finish4<DT>(acc[i][j], s, t.w_scales[p] + c + 4 * i),
                      hi = finish4<DT>(acc[i + 1][j], s, t.w_scales[p] + c + 4 * i + 4);
          store128(y + c + 4 * i, make_uint4(lo.x, lo.y, hi.x, hi.y));
        }
    }
  }
};

template <int NC, int NT>
__device__ __forceinline__ void multiply(const uint4 (&fw)[NC], const uint4 (&fq)[NT], i32x4 (&acc)[NC][NT]) {
#pragma unroll
  for (int i = 0; i < NC; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = mfma_i8(fw[i], fq[j], acc[i][j]);
}

// The kernel for large tiles.  A step is four products, of one half of a wave's channels with one half of its tokens each.  In
// front of a product the half that it is the first to need is read from LDS, and a quarter of the step after next is fetched
// into the place that the product before was the last to read: what is fetched has seven products' time to arrive.
// PONG: eight waves in two groups, one of each to every SIMD, half a product apart: while one group multiplies, the other reads
// and fetches (8192 tokens, 8192 -> 8192: 438 us, 2500 TOPS at 1.9 GHz, the matrix cores busy 64 % of the time: bound by power, as
// a library's product is, 462 us at 1.6 GHz).  Else several workgroups share a compute unit and fill each other's gaps.
// grid = tiles (channel tiles of all projections times token tiles)
template <class DT, int NC, int NT, int WC, int WT, bool PONG>
__global__ __launch_bounds__(64 * WC * WT, 2) void dense_q8_large_kernel(DenseTable t, const int8_t* __restrict__ q,
                                                                        const float* __restrict__ q_scales, DenseShape shape) {
  using T = DenseTile<NC, NT, WC, WT, 2>;
  constexpr int kLoadsW = T::kLoadsW / 2, kLoadsQ = T::kLoadsQ / 2;  // of a half
  static_assert(T::kLoadsW % 2 == 0 && T::kLoadsQ % 2 == 0 && NC % 4 == 0 && NT % 2 == 0, "whole loads of half the rows");
  static_assert(T::kWaves * 8 % (2 * NC) == 0 && T::kWaves * 8 % (8 * NT) == 0, "loads of a half lie evenly");
  extern __shared__ __align__(1024) int8_t lds[];
  const DenseWork<T, NC, NT, WC> work(t, q, shape, lds);
  // row j of a half: the first or second NC / 2 fragments of every wave's channels, NT / 2 of its tokens
  auto w_half_row = [](int half, int j) { return j / (2 * NC) * (4 * NC) + half * (2 * NC) + j % (2 * NC); };
  auto q_half_row = [](int half, int j) { return j / (8 * NT) * (16 * NT) + half * (8 * NT) + j % (8 * NT); };
  uint32_t off_w[2][kLoadsW], off_q[2][kLoadsQ];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
#pragma unroll
    for (int i = 0; i < kLoadsW; ++i) {
      const int row = w_half_row(half, (i * T::kWaves + work.wave) * 8 + (work.lane >> 3));
      off_w[half][i] = (uint32_t)min(row, work.last_w) * (uint32_t)shape.h_in + (uint32_t)(((work.lane & 7) ^ T::w_swizzle(row)) * 16);
    }
#pragma unroll
    for (int i = 0; i < kLoadsQ; ++i) {
      const int row = q_half_row(half, (i * T::kWaves + work.wave) * 8 + (work.lane >> 3));
      off_q[half][i] = (uint32_t)min(row, work.last_q) * (uint32_t)shape.h_in + (uint32_t)(((work.lane & 7) ^ T::q_swizzle(row)) * 16);
    }
  }
  auto fetch_w = [&](int step, int half) {
    // a load further on is kWaves * 8 rows of the half, twice as many of the tile
    load_to_lds<kLoadsW, T::kWaves * 2048>(work.from_w, off_w[half], (uint32_t)step * 128u,
                                           lds + (step & 1) * T::kPlace + w_half_row(half, work.wave * 8) * 128);
  };
  auto fetch_q = [&](int step, int half) {
    load_to_lds<kLoadsQ, T::kWaves * 2048>(work.from_q, off_q[half], (uint32_t)step * 128u,
                                           lds + (step & 1) * T::kPlace + (T::kChannels + q_half_row(half, work.wave * 8)) * 128);
  };
  i32x4 acc[NC][NT] = {};
  uint4 fw[2][NC / 2], fq[2][2][NT / 2];
  auto read_w = [&](int place, int half) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < NC / 2; ++i)
        fw[s][i] = *reinterpret_cast<const uint4*>(work.my_w + place * T::kPlace + (half * (NC / 2) + i) * 512 + (work.piece_w ^ (s * 64)));
  };
  auto read_q = [&](int place, int half) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < NT / 2; ++i)
        fq[half][s][i] = *reinterpret_cast<const uint4*>(work.my_q + place * T::kPlace + (half * (NT / 2) + i) * 2048 + (work.piece_q ^ (s * 64)));
  };
  auto product = [&](int half_w, int half_q) {
    __builtin_amdgcn_sched_barrier(0);
    if (PONG) __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < NC / 2; ++i)
#pragma unroll
        for (int j = 0; j < NT / 2; ++j) {
          i32x4& a = acc[half_w * (NC / 2) + i][half_q * (NT / 2) + j];
          a = mfma_i8(fw[s][i], fq[half_q][s][j], a);
        }
    if (PONG) __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    if (PONG) asm volatile("s_barrier" ::: "memory");
  };
  constexpr int kLeft = 3 * (kLoadsW + kLoadsQ);  // fetched after what the next product needs
#define DENSE_PRODUCT(READ, FETCH, MORE, HALF_W, HALF_Q) \
  do {                                                   \
    READ;                                                \
    if (MORE) {                                          \
      FETCH;                                             \
      arrive<kLeft>();                                   \
    } else {                                             \
      arrive<0>();                                       \
    }                                                    \
    product(HALF_W, HALF_Q);                             \
  } while (0)
  const int steps = work.steps;
  if (steps > 0) {
    // even steps begin with the tokens' first half, odd ones with the second, which is read during the step before
    fetch_q(0, 0);
    fetch_w(0, 0);
    fetch_q(0, 1);
    fetch_w(0, 1);
    if (steps > 1) {
      fetch_q(1, 1);
      fetch_w(1, 0);
      fetch_q(1, 0);
      fetch_w(1, 1);
      arrive<2 * (kLoadsW + kLoadsQ)>();
    } else {
      arrive<0>();
    }
    read_q(0, 0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // read by all: the first product fetches into its place
    if (PONG && work.wave >= T::kWaves / 2) asm volatile("s_barrier" ::: "memory");
    int step = 0;
    for (; step + 1 < steps; step += 2) {
      const bool more = step + 2 < steps, yet_more = step + 3 < steps;
      DENSE_PRODUCT(read_w(0, 0), fetch_q(step + 2, 0), more, 0, 0);
      DENSE_PRODUCT(read_q(0, 1), fetch_w(step + 2, 0), more, 0, 1);
      DENSE_PRODUCT(read_w(0, 1), fetch_q(step + 2, 1), more, 1, 1);
      DENSE_PRODUCT(read_q(1, 1), fetch_w(step + 2, 1), more, 1, 0);
      DENSE_PRODUCT(read_w(1, 0), fetch_q(step + 3, 1), yet_more, 0, 1);
      DENSE_PRODUCT(read_q(1, 0), fetch_w(step + 3, 0), yet_more, 0, 0);
      DENSE_PRODUCT(read_w(1, 1), fetch_q(step + 3, 0), yet_more, 1, 0);
      DENSE_PRODUCT(if (more) read_q(0, 0), fetch_w(step + 3, 1), yet_more, 1, 1);
    }
    if (step < steps) {
      DENSE_PRODUCT(read_w(0, 0), , false, 0, 0);
      DENSE_PRODUCT(read_q(0, 1), , false, 0, 1);
      DENSE_PRODUCT(read_w(0, 1), , false, 1, 1);
      DENSE_PRODUCT(, , false, 1, 0);
    }
    if (PONG && work.wave < T::kWaves / 2) asm volatile("s_barrier" ::: "memory");
  }
#undef DENSE_PRODUCT
  if (work.rest) {
    work.fetch_rest();
    read_q(0, 0);
    read_q(0, 1);
    read_w(0, 0);
    product(0, 0);
    product(0, 1);
    read_w(0, 1);
    product(1, 0);
    product(1, 1);
  }
  work.template store<DT>(t, q_scales, shape, acc);
}

// The kernel for smaller tiles.  The fetches alone of 1024 tokens, 4096 -> 4096, take 19 of its 26 us, and some 100 to 190 clocks go
// around a step's barrier.  What bounds the fetches is not known: of 517 tokens, 4096 -> 4096 + 2 x 1024 (23 to 25 us), the tiles take in
// 252 MB, of which three quarters come from the L2s.  While half a step's products run, the other half's or the next step's
// fragments go from LDS to registers and a later step's pieces from memory to LDS; one barrier a step.
// grid = tiles (channel tiles of all projections times token tiles)
template <class DT, int NC, int NT, int WC, int WT, int DEPTH>
__global__ __launch_bounds__(64 * WC * WT, 2) void dense_q8_small_kernel(DenseTable t, const int8_t* __restrict__ q,
                                                                        const float* __restrict__ q_scales, DenseShape shape) {
  using T = DenseTile<NC, NT, WC, WT, DEPTH>;
  static_assert(DEPTH >= 3 && (DEPTH - 2) * T::kLoads <= 63, "what the wait for loads can count");
  extern __shared__ __align__(1024) int8_t lds[];
  const DenseWork<T, NC, NT, WC> work(t, q, shape, lds);
  i32x4 acc[NC][NT] = {};
  uint4 fw[2][NC], fq[2][NT];
  auto after = [](int place) { return place + T::kPlace == T::kLds ? 0 : place + T::kPlace; };
  const int steps = work.steps;
  if (steps > 0) {
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d)
      if (d < steps) work.fetch(d, d * T::kPlace);
    if (steps >= DEPTH - 1)
      arrive<(DEPTH - 2) * T::kLoads>();
    else
      arrive<0>();
    work.read(0, 0, fw[0], fq[0]);
    int place = 0, free = T::kLds - T::kPlace;  // where the step lies, and where the step before did
    for (int step = 0; step < steps; ++step) {
      // the next step has arrived, and everybody has read the one before
      if (step + DEPTH - 1 <= steps)
        arrive<(DEPTH - 3) * T::kLoads>();
      else
        arrive<0>();
      work.read(place, 1, fw[1], fq[1]);
      if (step + DEPTH - 1 < steps) work.fetch(step + DEPTH - 1, free);
      multiply(fw[0], fq[0], acc);
      place = after(place);
      free = after(free);
      if (step + 1 < steps) work.read(place, 0, fw[0], fq[0]);
      multiply(fw[1], fq[1], acc);
    }
  }
  if (work.rest) {
    work.fetch_rest();
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      work.read(0, half, fw[half], fq[half]);
      multiply(fw[half], fq[half], acc);
    }
  }
  work.template store<DT>(t, q_scales, shape, acc);
}

// The kernel for few tokens.  A workgroup computes 16 CH channels of up to 16 NT tokens; its WAVES waves divide k among
// themselves in chunks of 128 bytes (a cache line of every row).  A wave's chunks go from memory to a ring of DEPTH places in
// LDS that is its own, eight rows to a load, and from there to the matrix cores: no registers are held by what is in flight,
// and no wave waits for another until their sums meet at the end.  Wide blocks are for batches whose narrower ones would take a
// second round of workgroups: 64 tokens, 5120 -> 2 x 13824 (128 channels, 216 workgroups) 35 to 37 us, with 32 to 96 channels 40 and more;
// 8192 -> 28672 47 to 50 us (4.8 to 5.1 TB/s) against 53.  One token, 4096 -> 3 x 4096 12.0 us, 64 tokens, 4096 -> 2 x 11008 23 us
// (weights from memory in all of these).  Memory bounds the widest; of lines that its L2 does not hold a compute unit takes in some
// 40 bytes a nanosecond, which bounds one token.  64 tokens, 2 x 11008, reach neither (4.0 TB/s; 28 bytes a nanosecond and unit).
// grid = (channel blocks of all projections, token blocks)
template <int CH, int NT, int WAVES, int DEPTH>
struct DenseFew {
  static constexpr int kPlace = (CH + NT) * 16 * 128;  // bytes of a chunk
  static constexpr int kRing = WAVES * DEPTH * kPlace, kSums = WAVES * CH * NT * 1024;
  static constexpr int kLds = kRing > kSums ? kRing : kSums;
};
template <class DT, int CH, int NT, int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void dense_q8_few_kernel(DenseTable t, const int8_t* __restrict__ q,
                                                                  const float* __restrict__ q_scales, DenseShape shape) {
  using T = DenseFew<CH, NT, WAVES, DEPTH>;
  const int n_tokens = shape.n_tokens, h_in = shape.h_in;
  extern __shared__ __align__(1024) int8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  int p = 0;
  while (p + 1 < shape.n_proj && (int)blockIdx.x >= t.first[p + 1]) ++p;
  const int channels = t.h_out[p], c0 = ((int)blockIdx.x - t.first[p]) * (16 * CH), t0 = (int)blockIdx.y * (16 * NT);
  const int8_t* w = t.w[p] + (size_t)c0 * h_in;
  const int8_t* x = q + (size_t)t0 * h_in;
  const __amdgpu_buffer_rsrc_t from_w = make_uniform_buffer(w, 0x7FFFFFFF), from_q = make_uniform_buffer(x, 0x7FFFFFFF);
  const int last_w = channels - 1 - c0, last_q = n_tokens - 1 - t0;  // rows past these repeat them: nothing of them is stored
  // the sixteen-byte pieces of a row are permuted in LDS so that the sixteen rows a fragment's read touches lie in different banks
  uint32_t off_w[2 * CH], off_q[2 * NT];
#pragma unroll
  for (int i = 0; i < 2 * CH; ++i) {
    const int row = i * 8 + (lane >> 3);
    off_w[i] = (uint32_t)min(row, last_w) * (uint32_t)h_in + (uint32_t)(((lane & 7) ^ (row >> 1 & 7)) * 16);
  }
#pragma unroll
  for (int i = 0; i < 2 * NT; ++i) {
    const int row = i * 8 + (lane >> 3);
    off_q[i] = (uint32_t)min(row, last_q) * (uint32_t)h_in + (uint32_t)(((lane & 7) ^ (row >> 1 & 7)) * 16);
  }
  int8_t* ring = lds + wave * (DEPTH * T::kPlace);
  const int chunks = h_in / 128;
  // The sum begins somewhere else in every workgroup: rows 4096 bytes apart would have all of them read from the same memory
  // channels at once (4096 wide: one token, 3 x 4096 12.9 -> 11.8 us, 64 tokens, 2 x 11008 23.3 -> 22.3; 5120 and 8192 wide as without).
  const int begin = chunks > 0 ? (int)(blockIdx.x * 11u % (unsigned)chunks) : 0;
  auto fetch = [&](int chunk, int place) {
    chunk += begin;
    if (chunk >= chunks) chunk -= chunks;
    int8_t* to = ring + place * T::kPlace;
    load_to_lds<2 * CH, 1024>(from_w, off_w, (uint32_t)chunk * 128u, to);
    load_to_lds<2 * NT, 1024>(from_q, off_q, (uint32_t)chunk * 128u, to + CH * 2048);
  };
  i32x4 acc[CH][NT] = {};
  const int piece = ((lane >> 4) ^ (lane >> 1 & 7)) * 16;
  const int8_t* mine = ring + (lane & 15) * 128;
  auto multiply = [&](int place) {
    uint4 a[2][CH], b[2][NT];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int i = 0; i < CH; ++i) a[s][i] = *reinterpret_cast<const uint4*>(mine + place * T::kPlace + i * 2048 + (piece ^ (s * 64)));
#pragma unroll
      for (int j = 0; j < NT; ++j) b[s][j] = *reinterpret_cast<const uint4*>(mine + place * T::kPlace + (CH + j) * 2048 + (piece ^ (s * 64)));
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = mfma_i8(a[s][i], b[s][j], acc[i][j]);
  };
  constexpr int kLoads = 2 * (CH + NT);
  static_assert(kLoads * (DEPTH - 1) <= 63, "what the wait for loads can count");
  int fetched = wave;  // the chunk to fetch next
#pragma unroll
  for (int d = 0; d < DEPTH; ++d, fetched += WAVES)
    if (fetched < chunks) fetch(fetched, d);
  for (int c = wave; c < chunks; c += DEPTH * WAVES) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      if (c + d * WAVES >= chunks) break;
      // the chunks behind this one may still be on their way; near the end there are fewer of them
      if (c + (d + DEPTH - 1) * WAVES < chunks)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads * (DEPTH - 1)) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      multiply(d);
      if (fetched < chunks) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // its place has been read
        fetch(fetched, d);
      }
      fetched += WAVES;
    }
  }
  // what is left of k, by the waves that had a chunk less
  const int left = (h_in - chunks * 128 + 63) / 64;  // steps
  for (int s = (wave - chunks % WAVES + WAVES) % WAVES; s < left; s += WAVES) {
    const int at = chunks * 128 + s * 64 + (lane >> 4) * 16;
    uint4 a[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) a[i] = load_row16(w + (size_t)min(i * 16 + (lane & 15), last_w) * h_in, at, h_in);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const uint4 b = load_row16(x + (size_t)min(j * 16 + (lane & 15), last_q) * h_in, at, h_in);
#pragma unroll
      for (int i = 0; i < CH; ++i) acc[i][j] = mfma_i8(a[i], b, acc[i][j]);
    }
  }
  __syncthreads();
  i32x4* sums = reinterpret_cast<i32x4*>(lds);  // [wave][fragment][lane]
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) sums[(wave * CH * NT + i * NT + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (int e = threadIdx.x; e < CH * NT * 64; e += 64 * WAVES) {
    const int l = e & 63, i = (e >> 6) / NT, j = (e >> 6) % NT;
    const int token = t0 + j * 16 + (l & 15), ch = c0 + i * 16 + (l >> 4) * 4;
    if (token >= n_tokens || ch >= channels) continue;  // widths are multiples of 8: four channels are in or out together
    i32x4 s = sums[e];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) s += sums[v * CH * NT * 64 + e];
    *reinterpret_cast<uint2*>(t.y[p] + (size_t)token * channels + ch) = finish4<DT>(s, q_scales[token], t.w_scales[p] + ch);
  }
}

// Eight channels of a token: the parts of a divided sum added up, and y.  grid = (eights of channels / 256, tokens)
template <class DT>
__global__ __launch_bounds__(256) void dense_q8_join_kernel(DenseTable t, const float* __restrict__ q_scales, DenseShape shape) {
  const int column = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 8, token = (int)blockIdx.y;
  if (column >= shape.all_channels) return;
  int p = 0;
  while (p + 1 < shape.n_proj && column >= t.before[p + 1]) ++p;
  const int c = column - t.before[p];
  i32x4 lo = {}, hi = {};
  for (int s = 0; s < shape.splits; ++s) {
    const i32x4* part = reinterpret_cast<const i32x4*>(shape.partials + ((size_t)s * shape.n_tokens + token) * shape.all_channels + column);
    lo += part[0];
    hi += part[1];
  }
  const float s = q_scales[token];
  const uint2 a = finish4<DT>(lo, s, t.w_scales[p] + c), b = finish4<DT>(hi, s, t.w_scales[p] + c + 4);
  store128(t.y[p] + (size_t)token * t.h_out[p] + c, make_uint4(a.x, a.y, b.x, b.y));
}

// Channel blocks of `width` channels of all projections.
DenseTable fill_table(const DenseArgs& a, int width) {
  DenseTable t = {};
  for (int i = 0; i < a.n_proj; ++i) {
    t.w[i] = a.w[i];
    t.w_scales[i] = a.w_scales[i];
    t.y[i] = static_cast<uint16_t*>(a.y[i]);
    t.h_out[i] = a.h_out[i];
    t.first[i + 1] = t.first[i] + ceil_div(a.h_out[i], width);
    if (i > 0) t.before[i] = t.before[i - 1] + a.h_out[i - 1];
  }
  return t;
}

// LDS beyond 64 KiB per workgroup has to be enabled per kernel, once per device.
constexpr int kMostDevices = 64;
hipError_t allow_lds(const void* kernel, int bytes, std::atomic<bool>* allowed) {
  if (bytes <= 64 * 1024) return hipSuccess;
  int dev = 0;
  hipError_t err = hipGetDevice(&dev);
  if (err != hipSuccess) return err;
  if (dev < 0 || dev >= kMostDevices) return hipErrorInvalidDevice;
  if (allowed[dev].load(std::memory_order_acquire)) return hipSuccess;
  err = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (err == hipSuccess) allowed[dev].store(true, std::memory_order_release);
  return err;
}

template <class T, class DT, class Kernel>
hipError_t launch_tiles(Kernel kernel, std::atomic<bool>* allowed, const DenseArgs& a, const DensePlan& plan, hipStream_t st) {
  const hipError_t err = allow_lds(reinterpret_cast<const void*>(kernel), T::kLds, allowed);
  if (err != hipSuccess) return err;
  const DenseTable t = fill_table(a, T::kChannels);
  const DenseShape shape = {a.n_tokens, a.h_in, a.n_proj, ceil_div(a.n_tokens, T::kTokens), plan.splits,
                            t.before[a.n_proj - 1] + a.h_out[a.n_proj - 1], static_cast<int*>(a.workspace)};
  kernel<<<(unsigned)(t.first[a.n_proj] * shape.token_tiles * plan.splits), T::kThreads, T::kLds, st>>>(t, a.q, a.q_scales, shape);
  const hipError_t launched = hipGetLastError();
  if (launched != hipSuccess || plan.splits == 1) return launched;
  const dim3 grid((unsigned)ceil_div(shape.all_channels, 8 * 256), (unsigned)a.n_tokens);
  dense_q8_join_kernel<DT><<<grid, 256, 0, st>>>(t, a.q_scales, shape);
  return hipGetLastError();
}
template <class DT, int NC, int NT, int WC, int WT, bool PONG>
hipError_t launch_large(const DenseArgs& a, const DensePlan& plan, hipStream_t st) {
  static std::atomic<bool> allowed[kMostDevices];
  return launch_tiles<DenseTile<NC, NT, WC, WT, 2>, DT>(dense_q8_large_kernel<DT, NC, NT, WC, WT, PONG>, allowed, a, plan, st);
}
template <class DT, int NC, int NT, int WC, int WT, int DEPTH>
hipError_t launch_small(const DenseArgs& a, const DensePlan& plan, hipStream_t st) {
  static std::atomic<bool> allowed[kMostDevices];
  return launch_tiles<DenseTile<NC, NT, WC, WT, DEPTH>, DT>(dense_q8_small_kernel<DT, NC, NT, WC, WT, DEPTH>, allowed, a, plan, st);
}
template <class DT, int CH, int NT, int WAVES, int DEPTH>
hipError_t launch_few(const DenseArgs& a, hipStream_t st) {
  using T = DenseFew<CH, NT, WAVES, DEPTH>;
  static std::atomic<bool> allowed[kMostDevices];
  auto kernel = dense_q8_few_kernel<DT, CH, NT, WAVES, DEPTH>;
  const hipError_t err = allow_lds(reinterpret_cast<const void*>(kernel), T::kLds, allowed);
  if (err != hipSuccess) return err;
  const DenseTable t = fill_table(a, 16 * CH);
  const DenseShape shape = {a.n_tokens, a.h_in, a.n_proj, 0, 1, 0, nullptr};
  kernel<<<dim3((unsigned)t.first[a.n_proj], (unsigned)ceil_div(a.n_tokens, 16 * NT)), 64 * WAVES, T::kLds, st>>>(t, a.q, a.q_scales, shape);
  return hipGetLastError();
}

// The kernels, and what the choice among them goes by: the time of a call is estimated for every one of them and the
// shortest taken.  The figures below are fits to graph replays of 48 shapes (1 to 4814 tokens, h_in 1024 to 13824, outputs
// of 1024 to 28672, weights from HBM), with every kernel each, before the few-token kernels' sums began at different places and
// before there was one of 128 channels: of these shapes the kernel chosen took 1.5 % more time than the best of them on average, 10 % at
// worst.  That is no bound for others: the estimates hold no fixed time of a launch, and none for units that the one round of a
// launch leaves idle (300 tokens, 2048 -> 2 x 5504 takes tiles of 128 x 256 on 172 of 256 units and 22.8 us, where 18.8 are possible).
struct DenseKernel {
  int channels, tokens, threads, lds;
  // Few tokens, 0: a compute unit takes in 40 bytes of w and x a nanosecond, and the workgroups of a launch run in rounds of one to
  // each unit.  Tiles: microseconds of a step of 128 bytes of k while a unit has one workgroup at most, and of each
  // round of one workgroup to each unit from the second on.
  float one, more;
  // How much longer it takes where rows do not begin on cache lines (h_in no multiple of 128: a piece of a row then lies on two).
  float askew;
};
template <int NC, int NT, int WC, int WT, int DEPTH>
constexpr DenseKernel tile_of(float one, float more, float askew) {
  using T = DenseTile<NC, NT, WC, WT, DEPTH>;
  return {T::kChannels, T::kTokens, T::kThreads, T::kLds, one, more, askew};
}
template <int CH, int NT, int WAVES, int DEPTH>
constexpr DenseKernel few_of() {
  return {16 * CH, 16 * NT, 64 * WAVES, DenseFew<CH, NT, WAVES, DEPTH>::kLds, 0.0f, 0.0f, 1.2f};
}
// In the order of launch_typed's cases.
constexpr DenseKernel kKernels[] = {
    few_of<1, 1, 16, 2>(), few_of<2, 1, 8, 2>(), few_of<4, 1, 4, 2>(), few_of<2, 2, 8, 2>(), few_of<3, 2, 4, 2>(), few_of<2, 3, 4, 2>(),
    few_of<6, 4, 4, 2>(), few_of<8, 4, 3, 2>(),
    tile_of<2, 1, 2, 2, 6>(0.26f, 0.22f, 1.27f),  // 64 x 32
    tile_of<2, 1, 2, 4, 6>(0.33f, 0.33f, 1.27f),  // 64 x 64
    tile_of<2, 2, 2, 4, 5>(0.47f, 0.50f, 1.27f),  // 64 x 128
    tile_of<4, 2, 2, 4, 5>(0.72f, 0.67f, 1.27f),  // 128 x 128, eight waves
    tile_of<4, 4, 2, 2, 2>(0.77f, 0.58f, 1.27f),  // 128 x 128, four waves, two workgroups to a unit
    tile_of<4, 4, 2, 4, 2>(1.08f, 1.10f, 1.15f),  // 128 x 256
    tile_of<8, 4, 2, 4, 2>(1.60f, 1.78f, 1.15f),  // 256 x 256
};
constexpr int kFewKernels = 8, kSmallKernels = 4;  // the rest are the large ones
constexpr int kFewMostTokens = 128;

template <class DT>
hipError_t launch_typed(const DenseArgs& a, const DensePlan& plan, hipStream_t st) {
  switch (plan.kernel) {
    case 0: return launch_few<DT, 1, 1, 16, 2>(a, st);
    case 1: return launch_few<DT, 2, 1, 8, 2>(a, st);
    case 2: return launch_few<DT, 4, 1, 4, 2>(a, st);
    case 3: return launch_few<DT, 2, 2, 8, 2>(a, st);
    case 4: return launch_few<DT, 3, 2, 4, 2>(a, st);
    case 5: return launch_few<DT, 2, 3, 4, 2>(a, st);
    case 6: return launch_few<DT, 6, 4, 4, 2>(a, st);
    case 7: return launch_few<DT, 8, 4, 3, 2>(a, st);
    case 8: return launch_small<DT, 2, 1, 2, 2, 6>(a, plan, st);
    case 9: return launch_small<DT, 2, 1, 2, 4, 6>(a, plan, st);
    case 10: return launch_small<DT, 2, 2, 2, 4, 5>(a, plan, st);
    case 11: return launch_small<DT, 4, 2, 2, 4, 5>(a, plan, st);
    case 12: return launch_large<DT, 4, 4, 2, 2, false>(a, plan, st);
    case 13: return launch_large<DT, 4, 4, 2, 4, true>(a, plan, st);
    default: return launch_large<DT, 8, 4, 2, 4, true>(a, plan, st);
  }
}

}  // namespace

void plan_dense(const DenseArgs& a, int units, DensePlan* plan) {
  constexpr long long kMostThreads = 0xFFFFFFFFLL;  // of a launch
  double weights = 0.0, channels = 0.0;  // bytes of w; channels of all projections
  for (int i = 0; i < a.n_proj; ++i) channels += a.h_out[i];
  weights = channels * a.h_in;
  const int all = a.h_in / 128;  // whole steps
  double best = 0.0;
  plan->kernel = -1;
  // One launch; where no kernel's threads fit into one, the tokens in ranges, a launch each.  A token block of the largest tiles
  // fits into a launch whatever the number of channels, so there is always a choice.
  for (int ranges = 0; ranges < 2 && plan->kernel < 0; ++ranges)
    for (int k = 0; k < (int)(sizeof kKernels / sizeof kKernels[0]); ++k) {
      const DenseKernel& kernel = kKernels[k];
      const bool few = k < kFewKernels;
      if (few && a.n_tokens > kFewMostTokens) continue;
      long long blocks = 0;
      for (int i = 0; i < a.n_proj; ++i) blocks += ceil_div(a.h_out[i], kernel.channels);
      const long long token_blocks = ceil_div(a.n_tokens, kernel.tokens), range = kMostThreads / (blocks * kernel.threads);
      if (ranges == 0 ? token_blocks > range : range == 0) continue;
      for (int splits = 1; splits <= 8; ++splits) {
        if (splits > 1) {
          // parts of eight steps and more, 4 bytes of partial sums written and read per value and part
          if (few || all < 8 * splits || a.n_tokens > 65535 || 4.0 * splits * a.n_tokens * channels > (double)a.workspace_bytes) break;
          if (token_blocks * splits > range) break;
        }
        const long long groups = blocks * token_blocks * splits;
        const double rounds = (double)((groups + units - 1) / units), askew = a.h_in % 128 != 0 ? kernel.askew : 1.0;
        double us;
        if (few) {
          const double unit = askew * rounds * (kernel.channels + kernel.tokens) * a.h_in / 40e3;
          // weights that later token blocks read again come from the cache behind the L2s
          const double memory = weights * (1.0 + 0.2 * (double)(token_blocks - 1)) / 5.4e6;
          us = unit > memory ? unit : memory;
          if (kernel.threads > 512 && rounds > 1.0) us *= 1.1;  // sixteen waves only where one workgroup to a unit is all there is
        } else {
          const double steps = (double)ceil_div(all, splits) + (a.h_in % 128 != 0);
          const double unit = askew * steps * (rounds > 1.0 ? rounds * kernel.more : kernel.one), memory = weights / 5.0e6;
          us = unit > memory ? unit : memory;
          if (splits > 1) us += 3.0 + 8.0 * splits * a.n_tokens * channels / 4e6;  // the second launch
        }
        if (plan->kernel < 0 || us < best) {
          best = us;
          plan->kernel = k;
          plan->family = few ? kDenseFew : k < kFewKernels + kSmallKernels ? kDenseSmall : kDenseLarge;
          plan->splits = splits;
          plan->workgroups = groups;
          plan->lds = kernel.lds;
          plan->tokens = token_blocks > range ? (int)range * kernel.tokens : a.n_tokens;
        }
      }
    }
}

hipError_t launch_dense(const DenseArgs& a, const DensePlan& plan, hipStream_t st) {
  DenseArgs part = a;
  for (int first = 0; first < a.n_tokens; first += part.n_tokens) {
    part.n_tokens = a.n_tokens - first < plan.tokens ? a.n_tokens - first : plan.tokens;
    part.q = a.q + (size_t)first * a.h_in;
    part.q_scales = a.q_scales + first;
    for (int i = 0; i < a.n_proj; ++i) part.y[i] = static_cast<uint16_t*>(a.y[i]) + (size_t)first * a.h_out[i];
    const hipError_t err = a.bf16 ? launch_typed<BF16>(part, plan, st) : launch_typed<F16>(part, plan, st);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace sgmv
