// Attention over the paged 4-bit cache (gfx950).
//
//   x_p = scale q . k_p,   w_p = exp(x_p - max x),   out = sum w_p v_p / sum w_p      over the visible positions p
//   with k_p = s c + m (codes c of 4 bits, scale and minimum of the position):
//   q . k_p = s (sum_j q_j c_j) + m sum_j q_j,       sum_p w_p v_p = sum_p (w_p s_p) c_p + sum_p w_p m_p
//
// so the codes go to the matrix cores as they are, and scales and minima touch scores and weights alone.  A code c
// masked out of its word is the binary16 number c * 2^-24 (or, one nibble higher, 16 c * 2^-24), exactly: the matrix cores take
// these as they take any other, five instructions make eight operands of a word, and the powers of two go into q and out.
//
// Columns are rows x query heads of one cache head's group; sixteen of them make a tile.  S^T = K q^T has positions as rows, so a lane
// receives four positions of its column, and the weights of these are the second operand of out^T = V^T w^T for the very same lane
// if v's four positions stand there as the contraction index: nothing passes through LDS on the way.  The tiles of the cache hold
// v in pieces of four positions x eight values for this: a lane's 128-bit load.
#include "device_common.h"
#include "kv.h"
#include "mfma.h"

namespace sgmv {

namespace {

// Below every score, and what a column's maximum is before it has seen one.
constexpr float kLowest = -3.0e38f;
// Weights times v's scales are brought below 2^12 by a power of two: binary16 then has all of its 11 bits down to 2^-26 of the largest.
constexpr int kWeightTop = 12;

template <int D>
__device__ __forceinline__ uint4 unpack_k(uint32_t w) {
  const uint32_t h = w >> 8;
  return make_uint4(w & 0x000F000Fu, w & 0x00F000F0u, h & 0x000F000Fu, h & 0x00F000F0u);
}

// 2^n for any n; what fp32 cannot hold is 0 or infinity.
__device__ __forceinline__ float power_of_two(int n) { return ldexpf(1.0f, n); }

__device__ __forceinline__ int clamp_int(int v, int low, int high) { return v < low ? low : v > high ? high : v; }

// The request of a column tile: request i starts at tile q_starts[i] * group / columns + i.  64 of them looked at at once.
__device__ __forceinline__ int request_of(const AttentionArgs& a, int columns_log2, int tile) {
  int low = 0, high = a.n_reqs;
  const int lane = threadIdx.x & 63;
  while (high - low > 1) {
    const int step = (high - low + 63) >> 6;
    const int i = low + lane * step;
    bool at_or_before = false;
    if (i < high) at_or_before = (int)(((long long)clamp_int(a.q_starts[i], 0, a.n_tokens) * a.group) >> columns_log2) + i <= tile;
    const int count = __popcll(__ballot(at_or_before));
    if (count == 0) return 0;
    low += (count - 1) * step;
    high = high < low + step ? high : low + step;
  }
  return __builtin_amdgcn_readfirstlane(low);
}

// A tile's part of the batch.
struct Tile {
  int request, first_row, rows;  // of the request
  int first_column, columns;     // of the tile; all of the request's
  int kv_len;
};
__device__ __forceinline__ bool tile_of_batch(const AttentionArgs& a, int columns_log2, int tile, Tile& t) {
  t.request = request_of(a, columns_log2, tile);
  t.first_row = clamp_int(a.q_starts[t.request], 0, a.n_tokens);
  t.rows = clamp_int(a.q_starts[t.request + 1], t.first_row, a.n_tokens) - t.first_row;
  const int before = (int)(((long long)t.first_row * a.group) >> columns_log2) + t.request;
  t.columns = t.rows * a.group;
  if (tile < before || ((long long)(tile - before) << columns_log2) >= t.columns) return false;
  t.first_column = (tile - before) << columns_log2;
  t.kv_len = clamp_int(a.kv_lens[t.request], 0, a.table_width << a.at.page_shift);
  return true;
}

// Positions [low, high) that a row of the request sees.
struct Span {
  int low, high;
};
__device__ __forceinline__ Span seen_by(const AttentionArgs& a, const Tile& t, int row) {
  const int pos = t.kv_len - t.rows + row;
  const int high = a.causal ? clamp_int(pos + 1, 0, t.kv_len) : t.kv_len;
  const int low = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  return {low, high};
}

// Codes, scales and minima of two tiles of the cache, as a wave holds them.  Lane = 16 g + i: k's codes of position i, a quarter g of
// its values; v's codes of positions 4 g .. 4 g + 3, eight values from 8 i on (a head of 64: from 8 (i % 8) on); scales and minima of
// positions 4 g .. 4 g + 3.
template <int D>
struct Step {
  uint32_t k[2][D / 32];
  uint4 v[2], k_params[2], v_params[2];
  bool there[2];
};
template <int D>
__device__ __forceinline__ void load_step(const AttentionArgs& a, const int32_t* table, size_t head_offset, int step, int last_tile, int lane, Step<D>& s) {
  const int g = lane >> 4, i = lane & 15;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // tiles behind the last position are not looked up: the last one again, all of it hidden
    const int tile = step * 2 + h < last_tile ? step * 2 + h : last_tile;
    const int pos = tile * kTilePositions;
    const int page = __builtin_amdgcn_readfirstlane(table[pos >> a.at.page_shift]);
    s.there[h] = page >= 0 && page < a.n_pages;
    const uint8_t* at = a.at.layer + (size_t)(s.there[h] ? page : 0) * a.at.page_stride + head_offset +
                        (size_t)((pos & ((1 << a.at.page_shift) - 1)) / kTilePositions) * tile_bytes(D);
    const uint8_t* k = at + i * (D / 2) + g * (D / 8);
    if constexpr (D == 128) {
      const uint4 w = load128(k);
      s.k[h][0] = w.x, s.k[h][1] = w.y, s.k[h][2] = w.z, s.k[h][3] = w.w;
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(k);
      s.k[h][0] = w.x, s.k[h][1] = w.y;
    }
    s.v[h] = load128(at + 8 * D + g * (2 * D) + (D == 128 ? i : i & 7) * 16);
    s.k_params[h] = load128(at + 16 * D + g * 16);
    s.v_params[h] = load128(at + 16 * D + 64 + g * 16);
  }
}

// q of one column as the second operand of S^T = K q^T, times a power of two that brings its largest value to between 2^13 and 2^14;
// the values that meet a nibble at 16 times its worth are a sixteenth.
template <int D>
struct Query {
  uint4 parts[D / 32];
  float sum;     // of the scaled values, times 2^-24 like the codes
  float factor;  // from scores to powers of two
};
template <class DT, int D>
__device__ __forceinline__ void load_query(const AttentionArgs& a, const uint16_t* q, bool live, int lane, Query<D>& out) {
  const int g = lane >> 4;
  float x[D / 4];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    float part[8] = {};
    if (live) unpack8<DT>(load128(q + g * (D / 4) + c * 8), part);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[c * 8 + i] = part[i];
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < D / 4; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  // 2^up times a value of exponent 13 - up; not finite, or 2^100 and more: the column is NaN
  const bool fits = top < 0x71800000u;
  const int up = fits ? 13 - ((int)(top >> 23) - 127) : 0;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < D / 4; ++i) {
    x[i] = fits ? ldexpf(x[i], up) : 0.0f;
    sum += x[i];
  }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  out.sum = sum * 0x1p-24f;
  out.factor = fits ? ldexpf(a.scale * 1.44269504088896341f, 24 - up) : __uint_as_float(0x7FC00000u);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    const float* v = x + c * 8;
    out.parts[c] = make_uint4(pack2<F16>(v[0], v[4]), pack2<F16>(v[1] * 0.0625f, v[5] * 0.0625f), pack2<F16>(v[2], v[6]),
                              pack2<F16>(v[3] * 0.0625f, v[7] * 0.0625f));
  }
}

// Codes of v of 32 positions as first operands of out^T = V^T w^T: of output tile j, row i of which is value 8 i + j of a head of
// 128 and 8 (i % 8) + 4 (i / 8) + j of one of 64, j odd at 16 times their worth.
template <int D>
__device__ __forceinline__ void unpack_v(const uint4 (&v)[2], int lane, uint4 (&out)[D / 16]) {
  const uint32_t pairs[4][2] = {{v[0].x, v[0].y}, {v[0].z, v[0].w}, {v[1].x, v[1].y}, {v[1].z, v[1].w}};
  uint32_t w[D / 16][4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    // halves of the words of two positions side by side
    const uint32_t own = D == 128 || (lane & 8) == 0 ? 0x05040100u : 0x07060302u;
#pragma unroll
    for (int h = 0; h < D / 64; ++h) {
      const uint32_t both = __builtin_amdgcn_perm(pairs[e][1], pairs[e][0], h == 0 ? own : 0x07060302u), up = both >> 8;
      w[h * 4][e] = both & 0x000F000Fu;
      w[h * 4 + 1][e] = both & 0x00F000F0u;
      w[h * 4 + 2][e] = up & 0x000F000Fu;
      w[h * 4 + 3][e] = up & 0x00F000F0u;
    }
  }
#pragma unroll
  for (int j = 0; j < D / 16; ++j) out[j] = make_uint4(w[j][0], w[j][1], w[j][2], w[j][3]);
}
// First of the values whose row 4 g + i of tile j a lane receives: value_of + j.
template <int D>
__device__ __forceinline__ int value_of(int row) {
  return D == 128 ? 8 * row : 8 * (row & 7) + 4 * (row >> 3);
}

// A column's softmax so far, in its lanes (each has a quarter of the positions' sums).
struct Column {
  float top;       // maximum of the scores in units of the column, the same in all of its lanes
  float sum;       // of the weights
  float minima;    // of the weights times v's minima
};

// Scores, weights and weighted values of 32 positions for one tile of sixteen columns.
template <class DT, int D>
__device__ __forceinline__ void attend_step(const Step<D>& s, const uint4 (&v_codes)[D / 16], const Query<D>& q, int first_pos, bool all_visible,
                                            Span span, int lane, float v_unit, Column& col, f32x4 (&acc)[D / 16]) {
  const int g = lane >> 4;
  float x[8], v_scale[8], v_min[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 dots = {};
#pragma unroll
    for (int c = 0; c < D / 32; ++c) dots = mfma16x16x32<F16>(unpack_k<D>(s.k[h][c]), q.parts[c], dots);
    const uint32_t kp[4] = {s.k_params[h].x, s.k_params[h].y, s.k_params[h].z, s.k_params[h].w};
    const uint32_t vp[4] = {s.v_params[h].x, s.v_params[h].y, s.v_params[h].z, s.v_params[h].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float scale, low;
      unpack2<DT>(kp[i], scale, low);
      x[h * 4 + i] = fmaf(dots[i], scale, low * q.sum);
      unpack2<DT>(vp[i], v_scale[h * 4 + i], v_min[h * 4 + i]);
    }
  }
  uint32_t visible = 0xFFu;
  if (!all_visible) {
    visible = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int pos = first_pos + (e >> 2) * kTilePositions + g * 4 + (e & 3);
      const bool sees = pos >= span.low && pos < span.high && s.there[e >> 2];
      visible |= (uint32_t)sees << e;
      if (!sees) x[e] = kLowest, v_min[e] = 0.0f, v_scale[e] = 0.0f;
    }
  }
  float top = col.top;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e]);
  top = fmaxf(top, __shfl_xor(top, 16));
  top = fmaxf(top, __shfl_xor(top, 32));
  if (__any(top > col.top)) {
    const float shrink = __builtin_amdgcn_exp2f((col.top - top) * q.factor);
    col.sum *= shrink;
    col.minima *= shrink;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) acc[j] *= shrink;
    col.top = top;
  }
  const float base = col.top * q.factor;
  float w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    w[e] = __builtin_amdgcn_exp2f(fmaf(x[e], q.factor, -base));
    if (!all_visible && !(visible >> e & 1u)) w[e] = 0.0f;
    col.sum += w[e];
    col.minima = fmaf(w[e], v_min[e], col.minima);
    w[e] *= v_scale[e] * v_unit;
  }
  uint32_t high[4], low[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    high[e] = pack2<F16>(w[2 * e], w[2 * e + 1]);
    if constexpr (std::is_same_v<DT, F16>) {
      float a, b;
      unpack2<F16>(high[e], a, b);
      low[e] = pack2<F16>(w[2 * e] - a, w[2 * e + 1] - b);
    }
  }
  const uint4 weights = make_uint4(high[0], high[1], high[2], high[3]);
#pragma unroll
  for (int j = 0; j < D / 16; ++j) acc[j] = mfma16x16x32<F16>(v_codes[j], weights, acc[j]);
  if constexpr (std::is_same_v<DT, F16>) {
    const uint4 rest = make_uint4(low[0], low[1], low[2], low[3]);
#pragma unroll
    for (int j = 0; j < D / 16; ++j) acc[j] = mfma16x16x32<F16>(v_codes[j], rest, acc[j]);
  }
}

// v's scales are brought below 2^kWeightTop by a power of two of the wave's, which falls when a larger scale comes.  True if it fell; `by`: by
// what the sums so far have to be multiplied.
template <class DT, int D>
__device__ __forceinline__ bool fit_scales(const Step<D>& s, int first_pos, bool all_visible, Span seen, int lane, float& limit, float& unit, float& by) {
  float top = 0.0f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t vp[4] = {s.v_params[h].x, s.v_params[h].y, s.v_params[h].z, s.v_params[h].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float scale, low;
      unpack2<DT>(vp[i], scale, low);
      if (!all_visible) {  // what nobody sees may hold anything
        const int pos = first_pos + h * kTilePositions + (lane >> 4) * 4 + i;
        if (pos < seen.low || pos >= seen.high || !s.there[h]) scale = 0.0f;
      }
      top = scale < __uint_as_float(0x7F800000u) ? fmaxf(top, scale) : top;
    }
  }
  if (!__any(top > limit)) return false;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
  const int exponent = (int)(__float_as_uint(top) >> 23) - 127 + 1;  // top < 2^exponent
  const int up = min(kWeightTop - exponent, 100);
  const float to = power_of_two(up);
  by = to / unit;
  unit = to;
  limit = power_of_two(kWeightTop - up);
  return true;
}

// Sixteen columns of one cache head: the four waves take steps of 32 positions in turn and meet in LDS.  grid = (cache heads x tiles, slices).
template <class DT, int D>
__global__ __launch_bounds__(256) void attention_few_kernel(AttentionArgs a, int first_tile) {
  __shared__ float sums[4][16][D + 4];
  __shared__ float4 stats[4][16];  // maximum in powers of two, sum of weights, of weights times minima
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, c = lane & 15;
  const int head = blockIdx.x % a.at.n_kv_heads, tile = first_tile + blockIdx.x / a.at.n_kv_heads, slice = blockIdx.y;
  Tile t;
  if (!tile_of_batch(a, 4, tile, t)) return;
  const int column = t.first_column + c;
  const bool live = column < t.columns;
  const int row = live ? column / a.group : 0;
  const int q_head = head * a.group + (live ? column - row * a.group : 0);
  const int last_column = min(t.first_column + 15, t.columns - 1);
  const Span first = seen_by(a, t, t.first_column / a.group), last = seen_by(a, t, last_column / a.group);
  const Span span = live ? seen_by(a, t, row) : Span{first.low, last.high};
  // steps of this slice, then this wave's of them
  const int from = first.low / kStepPositions;
  const int steps = last.high > first.low ? (last.high + kStepPositions - 1) / kStepPositions - from : 0;
  const int per = max(a.slice_steps, (steps + a.slices - 1) / a.slices);
  const int begin = from + min(steps, slice * per), end = from + min(steps, (slice + 1) * per);

  Query<D> q;
  const long long at = t.first_row + row;
  load_query<DT, D>(a, a.q + at * a.q_stride + q_head * D, live, lane, q);
  Column col = {kLowest, 0.0f, 0.0f};
  f32x4 acc[D / 16] = {};
  float limit = 0.0f, unit = power_of_two(100);
  const int32_t* table = a.tables + (size_t)t.request * a.table_width;
  const size_t head_offset = (size_t)head * ((1u << a.at.page_shift) / kTilePositions) * tile_bytes(D);
  const int last_tile = (last.high - 1) / kTilePositions;
  for (int s = begin + wave; s < end; s += 4) {
    Step<D> step;
    load_step<D>(a, table, head_offset, s, last_tile, lane, step);
    const int pos = s * kStepPositions;
    const bool all_visible = pos >= last.low && pos + kStepPositions <= first.high && step.there[0] && step.there[1];
    float by;
    if (fit_scales<DT, D>(step, pos, all_visible, Span{first.low, last.high}, lane, limit, unit, by)) {
#pragma unroll
      for (int j = 0; j < D / 16; ++j) acc[j] *= by;
    }
    uint4 v_codes[D / 16];
    unpack_v<D>(step.v, lane, v_codes);
    attend_step<DT, D>(step, v_codes, q, pos, all_visible, span, lane, unit, col, acc);
  }
  col.sum += __shfl_xor(col.sum, 16);
  col.sum += __shfl_xor(col.sum, 32);
  col.minima += __shfl_xor(col.minima, 16);
  col.minima += __shfl_xor(col.minima, 32);
  if (live) {
    const float back = 1.0f / unit;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int j = 0; j < D / 16; ++j) sums[wave][c][value_of<D>(4 * g + i) + j] = acc[j][i] * (j & 1 ? 0x1p20f : 0x1p24f) * back;
    }
    if (g == 0) stats[wave][c] = make_float4(col.top == kLowest ? kLowest : col.top * q.factor, col.sum, col.minima, 0.0f);
  }
  __syncthreads();
  // sixteen threads to a column
  const int mine = threadIdx.x >> 4, part = threadIdx.x & 15;
  if (t.first_column + mine >= t.columns) return;
  float top = kLowest;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, stats[w][mine].x);
  float weight[4], sum = 0.0f, minima = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    weight[w] = __builtin_amdgcn_exp2f(stats[w][mine].x - top);
    sum += weight[w] * stats[w][mine].y;
    minima += weight[w] * stats[w][mine].z;
  }
  const int my_row = (t.first_column + mine) / a.group, my_head = head * a.group + (t.first_column + mine) - my_row * a.group;
  const long long out_row = t.first_row + my_row;
  constexpr int PER = D / 16;
  float v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    v[i] = minima;
#pragma unroll
    for (int w = 0; w < 4; ++w) v[i] = fmaf(weight[w], sums[w][mine][part * PER + i], v[i]);
  }
  if (a.slices > 1) {
    const size_t to = ((size_t)out_row * a.n_heads + my_head) * a.slices + slice;
#pragma unroll
    for (int i = 0; i < PER; i += 4) *reinterpret_cast<float4*>(a.sums + to * D + part * PER + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    if (part == 0) a.tops[to] = make_float2(top, sum);
    return;
  }
  const float inverse = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint32_t packed[PER / 2];
#pragma unroll
  for (int i = 0; i < PER; i += 2) packed[i / 2] = pack2<DT>(sum == 0.0f ? 0.0f : v[i] * inverse, sum == 0.0f ? 0.0f : v[i + 1] * inverse);
  uint32_t* to = reinterpret_cast<uint32_t*>(a.out + out_row * a.out_stride + my_head * D + part * PER);
#pragma unroll
  for (int i = 0; i < PER / 2; ++i) to[i] = packed[i];
  if (a.lse != nullptr && part == 0)
    a.lse[out_row * a.n_heads + my_head] = sum == 0.0f ? -__uint_as_float(0x7F800000u) : (top + log2f(sum)) * 0.693147180559945309f;
}

// Joins the slices of a row's head, a wave each.  grid = rows x heads / 4.
template <class DT, int D>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a, long long first) {
  const long long item = first + (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (item >= (long long)a.n_tokens * a.n_heads) return;
  const int row = (int)(item / a.n_heads), head = (int)(item - (long long)row * a.n_heads);
  if (row < a.q_starts[0] || row >= a.q_starts[a.n_reqs]) return;
  const float2* tops = a.tops + item * a.slices;
  float top = kLowest;
  for (int z = lane; z < a.slices; z += 64) top = fmaxf(top, tops[z].x);
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
  constexpr int PER = D / 64;
  float v[PER] = {}, sum = 0.0f;
  for (int z = 0; z < a.slices; ++z) {
    const float2 p = tops[z];
    if (p.y == 0.0f) continue;  // a slice without positions
    const float w = __builtin_amdgcn_exp2f(p.x - top);
    sum += w * p.y;
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = fmaf(w, a.sums[(item * a.slices + z) * D + lane * PER + i], v[i]);
  }
  const float inverse = 1.0f / sum;
  uint16_t* to = a.out + (long long)row * a.out_stride + head * D + lane * PER;
#pragma unroll
  for (int i = 0; i < PER; ++i) to[i] = (uint16_t)encode1<DT>(sum == 0.0f ? 0.0f : v[i] * inverse);
  if (a.lse != nullptr && lane == 0)
    a.lse[item] = sum == 0.0f ? -__uint_as_float(0x7F800000u) : (top + log2f(sum)) * 0.693147180559945309f;
}

template <class DT, int D>
hipError_t few_typed(const AttentionArgs& a, hipStream_t st) {
  const long long tiles = attention_tiles(a.n_tokens, a.group, a.n_reqs, kFewColumns);
  // fewer than 2^31 threads to a launch
  const long long share = (1LL << 30) / 256 / a.slices / a.at.n_kv_heads, most = share > 0 ? share : 1;
  for (long long first = 0; first < tiles; first += most) {
    const long long n = tiles - first < most ? tiles - first : most;
    attention_few_kernel<DT, D><<<dim3((unsigned)(n * a.at.n_kv_heads), (unsigned)a.slices), 256, 0, st>>>(a, (int)first);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

template <class DT, int D>
hipError_t join_typed(const AttentionArgs& a, hipStream_t st) {
  const long long items = (long long)a.n_tokens * a.n_heads, most = 1LL << 24;
  for (long long first = 0; first < items; first += most) {
    const long long n = items - first < most ? items - first : most;
    attention_join_kernel<DT, D><<<(unsigned)((n + 3) / 4), 256, 0, st>>>(a, first);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_attention_few(const AttentionArgs& a, hipStream_t st) {
  if (a.bf16) return a.at.head_dim == 64 ? few_typed<BF16, 64>(a, st) : few_typed<BF16, 128>(a, st);
  return a.at.head_dim == 64 ? few_typed<F16, 64>(a, st) : few_typed<F16, 128>(a, st);
}

hipError_t launch_attention_join(const AttentionArgs& a, hipStream_t st) {
  if (a.bf16) return a.at.head_dim == 64 ? join_typed<BF16, 64>(a, st) : join_typed<BF16, 128>(a, st);
  return a.at.head_dim == 64 ? join_typed<F16, 64>(a, st) : join_typed<F16, 128>(a, st);
}

}  // namespace sgmv
