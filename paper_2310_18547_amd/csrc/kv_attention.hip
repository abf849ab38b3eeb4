// Attention over the paged 4-bit cache (gfx950).
//
//   x_p = scale q . k_p,   w_p = exp(x_p - max x),   out = sum w_p v_p / sum w_p      over the visible positions p
//   with k_p = s c + m (codes c of 4 bits, scale and minimum of the position):
//   q . k_p = s (sum_j q_j c_j) + m sum_j q_j,       sum_p w_p v_p = sum_p (w_p s_p) c_p + sum_p w_p m_p
//
// so the codes go to the matrix cores as they are, and scales and minima touch scores and weights alone.  A code c in bits 4 to 7 of
// a half word, everything else masked out, is the binary16 number 16 c * 2^-24, exactly: seven instructions make eight operands of
// a word.  (Those cores cut products with numbers below 2^-14 off at a fixed place: of codes in bits 0 to 3 the sum of 32 products is
// off by 2^-21.8 of their size on average, always downwards, of bits 4 to 7 by a sixteenth of that.)
//
// Sums of many positive w s c that nearly cancel against the minima would lose what is left of them: v's odd positions are taken from
// their largest value down, v = (m + 15 s) - s (15 - c), which costs an inversion of their words, so that terms of both signs add up.
//
// Columns are rows x query heads of one cache head's group; sixteen of them make a tile.  S^T = K q^T has positions as rows, so a lane
// receives four positions of its column, and the weights of these are the second operand of out^T = V^T w^T for the very same lane
// if v's four positions stand there as the contraction index: nothing passes through LDS on the way.  The tiles of the cache hold
// v in pieces of four positions x eight values for this: a lane's 128-bit load.  Scales and minima: sixteen lanes need those of eight
// positions of k and of v, sixteen pairs; each lane loads and decodes one, and the others read it from its lane as they multiply.
#include "device_common.h"
#include "kv.h"
#include "mfma.h"

namespace sgmv {

namespace {

// Below every score, and what a column's maximum is before it has seen one.
constexpr float kLowest = -3.0e38f;
// The weights are 2^unit larger than their definition, so that the largest one times the largest scale of v stays below 2^11 (binary16 has
// all of its 11 bits down to 2^-25 of that), and below 2^15 while a column's maximum is up to 2^4 behind.  Minima count as scales of 2^-60
// of their size, so that 2^30 positions' stay below 2^105 in sum where v is constant, and with neither the weights themselves below 2^124.
constexpr int kWeightTop = 11, kMostUnit = 90;
constexpr float kMinimum = 0x1p-60f;
constexpr float kBehind = 4.0f;
// Maxima beyond it (in powers of two) are taken off the scores themselves: as part of a base they would be rounded, by 2^-8 here, by 2^7 at
// scores of 2^31, which rows of binary16 have, and a weight of 1 would be worth nothing, or no number.  Such a column goes through raise() at every
// step, so that the others' steps know nothing of it (a branch in them took 4 %).
constexpr float kFar = 0x1p16f;
// What a weight of 1 is worth at least, in powers of two, where parts of a column meet, and exactly in those of a far one, which would not meet as
// equals with units of their own.  From here to kMostUnit fp32 holds the sums of both; a unit is as low as -114 next to the largest scales.
constexpr int kLeastUnit = -20;
// What a sum is multiplied by in one go, of as many powers of two as a unit may fall by at once.
constexpr int kMostFall = 100;

// Codes of a word's halves as binary16 operands of 2^-20 each: values n and n + 4 of part n.
__device__ __forceinline__ uint4 unpack_codes(uint32_t w) {
  constexpr uint32_t kMask = 0x00F000F0u;
  return make_uint4(w << 4 & kMask, w & kMask, w >> 4 & kMask, w >> 8 & kMask);
}

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

// The lane whose bit is the n-th that is set.
__device__ __forceinline__ int nth_bit(unsigned long long bits, int n) {
  const int lane = threadIdx.x & 63, before = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(bits >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)bits, 0));
  return __builtin_ctzll(__ballot((bits >> lane & 1) && before == n) | 1ULL << 63);
}

// The n-th of the requests, long ones first: sixty-four of them at a time in eight classes of their lengths next to the longest that the
// caller expects.  The last workgroups of a launch are then short ones, and no long one is left running alone behind the others.
__device__ __forceinline__ int request_by_length(const AttentionArgs& a, int n) {
  const int lane = threadIdx.x & 63, first = n & ~63, i = first + lane;
  int of = -1;
  if (i < a.n_reqs) {
    const int len = a.kv_lens[i];
    of = min((int)((float)(a.window > 0 ? min(len, a.window) : len) * a.classes), 7);
    of = max(of, 0);
  }
  int rank = n - first;
  unsigned long long same = 0;
  for (int k = 7; k >= 0; --k) {
    same = __ballot(of == k);
    const int count = __popcll(same);
    if (rank < count) break;
    rank -= count;
  }
  return first + nth_bit(same, rank);
}
// That request's columns from 0 on; false where it has none.
__device__ __forceinline__ bool whole_request(const AttentionArgs& a, int request, Tile& t) {
  t.request = request;
  t.first_row = clamp_int(a.q_starts[request], 0, a.n_tokens);
  t.rows = clamp_int(a.q_starts[request + 1], t.first_row, a.n_tokens) - t.first_row;
  t.columns = t.rows * a.group;
  t.first_column = 0;
  t.kv_len = clamp_int(a.kv_lens[request], 0, a.table_width << a.at.page_shift);
  return t.rows > 0;
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

// Two tiles of the cache, as a wave holds them.  Lane = 16 g + i: k's codes of position i, a quarter g of its values; v's codes of positions
// 4 g .. 4 g + 3, eight values from 8 i on (a head of 64: from 8 (i % 8) on); of the sixteen pairs (scale, minimum) that the lanes
// 16 g .. 16 g + 15 use (positions 4 g .. 4 g + 3 of both tiles, k's, then v's) the i-th.
template <int D>
struct Held {
  uint32_t k[2][D / 32];
  uint4 v[2];
  uint32_t pair;
};

// A request's pages of one cache head, and the two tiles of a step in them.
struct Pages {
  const __attribute__((address_space(4))) int32_t* table;
  const uint8_t* head;
  int last_tile;
};
struct Place {
  const uint8_t* first;
  const uint8_t* second;
  uint32_t there;  // a bit each
};
// The pages of a step's tiles.  Tiles behind the last position are not looked up: the last one again, all of it hidden.
struct Looked {
  int first, second;
};
__device__ __forceinline__ Looked look_up(const AttentionArgs& a, const Pages& p, int step) {
  const int tiles_log2 = a.at.page_shift - 4;
  return {p.table[min(step * 2, p.last_tile) >> tiles_log2], p.table[min(step * 2 + 1, p.last_tile) >> tiles_log2]};
}
template <int D>
__device__ __forceinline__ const uint8_t* find_tile(const AttentionArgs& a, const Pages& p, int tile, int page, bool& there) {
  tile = min(tile, p.last_tile);
  const int tiles_log2 = a.at.page_shift - 4;
  there = page >= 0 && page < a.n_pages;
  return p.head + (size_t)(uint32_t)(there ? page : 0) * a.at.page_stride + (uint32_t)(tile & ((1 << tiles_log2) - 1)) * (uint32_t)tile_bytes(D);
}
template <int D>
__device__ __forceinline__ Place place_of(const AttentionArgs& a, const Pages& p, int step, const Looked& pages) {
  bool one, two;
  const uint8_t* first = find_tile<D>(a, p, step * 2, pages.first, one);
  const uint8_t* second = find_tile<D>(a, p, step * 2 + 1, pages.second, two);
  return {first, second, (one ? 1u : 0u) | (two ? 2u : 0u)};
}
// A lane's offsets in a tile.
template <int D>
struct Lane {
  uint32_t k, v, pair;
  bool second;  // its pair lies in the second tile
};
template <int D>
__device__ __forceinline__ Lane<D> offsets_of(int lane) {
  const uint32_t g = (uint32_t)lane >> 4, i = (uint32_t)lane & 15;
  return {i * (D / 2) + g * (D / 8), 8 * D + g * (2 * D) + (D == 128 ? i : i & 7) * 16, 16 * D + (i & 8) * 8 + g * 16 + (i & 3) * 4, (i & 4) != 0};
}
// ONCE: nobody else reads these tiles, so they pass the caches by (few columns: 64 requests of 512 to 2048 positions 80 -> 75 us, 131 000 positions 37 -> 35;
// but tiles of prompts, which meet there: 84 -> 89).
template <int D, bool ONCE>
__device__ __forceinline__ void load_k(const Place& at, const Lane<D>& lane, Held<D>& s) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const __amdgpu_buffer_rsrc_t tile = make_buffer(h ? at.second : at.first, tile_bytes(D));
    if constexpr (D == 128) {
      const uint4 w = buffer_load128<ONCE ? kNonTemporal : 0>(tile, lane.k);
      s.k[h][0] = w.x, s.k[h][1] = w.y, s.k[h][2] = w.z, s.k[h][3] = w.w;
    } else {
      const uint2 w = buffer_load64_at<ONCE ? kNonTemporal : 0>(tile, lane.k, 0);
      s.k[h][0] = w.x, s.k[h][1] = w.y;
    }
  }
  const uint8_t *first = at.first, *second = at.second;
  s.pair = *reinterpret_cast<const uint32_t*>((lane.second ? second : first) + (size_t)lane.pair);
}
template <int D, bool ONCE>
__device__ __forceinline__ void load_v(const Place& at, const Lane<D>& lane, Held<D>& s) {
#pragma unroll
  for (int h = 0; h < 2; ++h) s.v[h] = buffer_load128<ONCE ? kNonTemporal : 0>(make_buffer(h ? at.second : at.first, tile_bytes(D)), lane.v);
}

// The value of the i-th of a lane's sixteen neighbours.
template <int I>
__device__ __forceinline__ float of_lane(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x150 + I, 0xF, 0xF, true));
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Two values as binary16, to the nearest even.
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, h2));
}

// q of one column as the second operand of S^T = K q^T, times a power of two that brings its largest value to between 2^13 and 2^14.
template <int D>
struct Query {
  uint4 parts[D / 32];
  float sum;     // of the scaled values, times 2^-20 like the codes
  float factor;  // from scores to powers of two
};
template <class DT, int D>
__device__ __forceinline__ void load_query(const AttentionArgs& a, const uint16_t* q, bool live, int lane, Query<D>& out) {
  const int g = lane >> 4;
  uint4 x[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c) x[c] = live ? load128(q + g * (D / 4) + c * 8) : make_uint4(0, 0, 0, 0);
  // the largest magnitude, as a pattern
  u16x2 most = {0, 0};
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    const uint32_t words[4] = {x[c].x, x[c].y, x[c].z, x[c].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, words[i] & 0x7FFF7FFFu));
  }
  uint32_t top = max((uint32_t)most.x, (uint32_t)most.y);
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  const float largest = decode1<DT>((uint16_t)top);
  const int up = 13 - ((int)(__float_as_uint(largest) >> 23) - 127);
  float sum = 0.0f;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    float v[8];
    unpack8<DT>(x[c], v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = ldexpf(v[i], up);
      sum += v[i];
    }
    out.parts[c] = make_uint4(pack_half(v[0], v[4]), pack_half(v[1], v[5]), pack_half(v[2], v[6]), pack_half(v[3], v[7]));
  }
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  out.sum = sum * 0x1p-20f;
  // (the power of two first: a scale near fp32's largest goes with small queries.  Not zero: times the -infinity of a hidden position that would be NaN)
  const float factor = ldexpf(a.scale, 20 - up) * 1.44269504088896341f;
  // not finite, or 2^100 and more, with the scale 2^120 and more: the column is NaN, whatever its operands
  const bool fits = largest < 0x1p100f && factor < __uint_as_float(0x7F800000u);
  out.factor = fits ? fmaxf(factor, 0x1p-126f) : __uint_as_float(0x7FC00000u);
}

// First of the values whose row 4 g + i of output tile j a lane receives: value_of + j.
template <int D>
__device__ __forceinline__ int value_of(int row) {
  return D == 128 ? 8 * row : 8 * (row & 7) + 4 * (row >> 3);
}

// A wave's columns: NT tiles of sixteen, a column's softmax in the four lanes that hold it (a quarter of the positions' sums each).
template <int D, int NT>
struct Columns {
  Query<D> q[NT];
  Span span[NT];     // of the lane's column
  Span some, all;    // positions that some column of the wave sees, and that all do
  float top[NT];     // maximum of the scores, up to kBehind of it behind, the same in all lanes of a column
  float bar[NT];     // scores above it raise the maximum
  float base[NT];    // 2^base: what a weight of 1 is worth (next to the maximum, where that is far)
  float sum[NT];     // of the weights
  float minima[NT];  // of the weights times v's minima
  f32x4 acc[NT][D / 16];  // of the weights times v's codes and scales, times 2^-20
  int unit;
  float limit;       // scales and minima of v above it (Scores::size) lower the unit; infinity in lanes that hold k's
};
template <int D, int NT>
__device__ __forceinline__ void start_columns(Columns<D, NT>& c, int lane) {
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    c.top[n] = c.bar[n] = kLowest;
    c.base[n] = c.sum[n] = c.minima[n] = 0.0f;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) c.acc[n][j] = f32x4{};
  }
  c.unit = kMostUnit;
  c.limit = lane & 8 ? 0.0f : __uint_as_float(0x7F800000u);
}

// What a step's scores are, and the scales and minima of its positions (a lane's own, see Held).
template <int NT>
struct Scores {
  float x[NT][8], highest[NT];
  uint32_t sees[NT];  // a bit for every position that the column sees
  float scale, low, size;  // size: what the weights are to fit
  bool above;         // of a bar or a limit: raise() is due
};
template <int D, int NT>
__device__ __forceinline__ bool is_far(const Columns<D, NT>& c, int n) {
  return fabsf(c.top[n] * c.q[n].factor) > kFar;
}

// Raises the columns' maxima to those of this step's scores and lowers the unit to its scales; takes maxima that are far off the scores.
template <int D, int NT>
__device__ __forceinline__ void raise(Columns<D, NT>& c, Scores<NT>& r, int lane) {
  float s = lane & 8 ? r.size : 0.0f;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) s = fmaxf(s, __shfl_xor(s, m));
  const int fits = min(kWeightTop - ((int)(__float_as_uint(s) >> 23) - 126), kMostUnit);  // s < 2^(kWeightTop - fits)
  const int unit = min(c.unit, fits);
  const int fall = c.unit - unit;
  const float by = ldexpf(1.0f, -min(fall, kMostFall));
  c.unit = unit;
  if (lane & 8) c.limit = ldexpf(1.0f, kWeightTop - unit);
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float top = fmaxf(r.highest[n], __shfl_xor(r.highest[n], 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    top = fmaxf(top, c.top[n]);
    // A column that has seen nothing yet stays as it began, whatever its neighbours raise: the first score that it sees has to raise it (kBehind
    // of a factor of 2^-126 would put the bar above any), and kLowest times the factor is no base to subtract from the score of a hidden page.
    const bool blind = top == kLowest;
    const float shrink = blind ? 1.0f : __builtin_amdgcn_exp2f((c.top[n] - top) * c.q[n].factor) * by;
    c.top[n] = top;
    const bool far = !blind && is_far(c, n);
    c.bar[n] = blind ? kLowest : far ? -__uint_as_float(0x7F800000u) : top + kBehind / c.q[n].factor;
    c.base[n] = blind ? 0.0f : fmaf(far ? 0.0f : top, c.q[n].factor, -(float)unit);
    if (__any(far)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) r.x[n][e] -= far ? top : 0.0f;
    }
    c.sum[n] *= shrink;
    c.minima[n] *= shrink;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) c.acc[n][j] *= shrink;
  }
  if (__any(fall > kMostFall)) {  // from values of nothing to 2^20 and more: what is left of the power of two would be 0 as one factor
    const float rest = ldexpf(1.0f, kMostFall - fall);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      c.sum[n] *= rest;
      c.minima[n] *= rest;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) c.acc[n][j] *= rest;
    }
  }
}

// Scores of the 32 positions whose keys are in `s`.  MASKED: some column does not see all of them, or a tile is not `there`.
template <class DT, int D, int NT, bool MASKED>
__device__ __forceinline__ void score_step(const Held<D>& s, int first_pos, uint32_t there, int lane, const Columns<D, NT>& c, Scores<NT>& r) {
  const int g = lane >> 4, i = lane & 15;
  // this lane's pair; v's odd positions from the top down
  unpack2<DT>(s.pair, r.scale, r.low);
  if (MASKED) {  // what nobody sees may hold anything
    const int pos = first_pos + (i & 4) * 4 + g * 4 + (i & 3);
    if (pos < c.some.low || pos >= c.some.high || !(there >> (i >> 2 & 1) & 1u)) r.scale = r.low = 0.0f;
  }
  r.size = fmaxf(r.scale, fabsf(r.low) * kMinimum);
  const bool down = (i & 9) == 9;
  r.low = fmaf(r.scale, down ? 15.0f : 0.0f, r.low);
  r.scale = down ? -r.scale : r.scale;

  f32x4 dots[NT][2] = {};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int w = 0; w < D / 32; ++w) {
      const uint4 codes = unpack_codes(s.k[h][w]);
#pragma unroll
      for (int n = 0; n < NT; ++n) dots[n][h] = mfma16x16x32<F16>(codes, c.q[n].parts[w], dots[n][h]);
    }
#pragma unroll
  for (int n = 0; n < NT; ++n) r.highest[n] = kLowest, r.sees[n] = 0;
  auto score = [&](auto which) {
    constexpr int E = decltype(which)::value;
    const float ks = of_lane<E>(r.scale), km = of_lane<E>(r.low);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float x = fmaf(dots[n][E >> 2][E & 3], ks, km * c.q[n].sum);
      if (MASKED) {
        const int pos = first_pos + (E >> 2) * kTilePositions + g * 4 + (E & 3);
        const bool visible = pos >= c.span[n].low && pos < c.span[n].high && (there >> (E >> 2) & 1u);
        r.sees[n] |= (uint32_t)visible << E;
        x = visible ? x : kLowest;
      }
      r.x[n][E] = x;
      r.highest[n] = fmaxf(r.highest[n], x);
    }
  };
  score(std::integral_constant<int, 0>{}), score(std::integral_constant<int, 1>{}), score(std::integral_constant<int, 2>{});
  score(std::integral_constant<int, 3>{}), score(std::integral_constant<int, 4>{}), score(std::integral_constant<int, 5>{});
  score(std::integral_constant<int, 6>{}), score(std::integral_constant<int, 7>{});
  if (!MASKED && there != 3) {  // a page that is not of the cache
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!(there >> (e >> 2) & 1u)) r.x[n][e] = -__uint_as_float(0x7F800000u);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      r.highest[n] = r.x[n][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) r.highest[n] = fmaxf(r.highest[n], r.x[n][e]);
    }
    if (!(there >> (i >> 2 & 1) & 1u)) r.scale = r.low = r.size = 0.0f;
  }
  r.above = r.size > c.limit;
#pragma unroll
  for (int n = 0; n < NT; ++n) r.above |= r.highest[n] > c.bar[n];
}

// v's codes of two positions side by side, halves of their words; odd positions from the top down.
template <int D>
struct Beside {
  uint32_t codes[D / 64][4];
};
template <int D>
__device__ __forceinline__ void put_beside(const Held<D>& s, int lane, Beside<D>& b) {
  const uint32_t pairs[4][2] = {{s.v[0].x, ~s.v[0].y}, {s.v[0].z, ~s.v[0].w}, {s.v[1].x, ~s.v[1].y}, {s.v[1].z, ~s.v[1].w}};
  const uint32_t own = D == 128 || (lane & 8) == 0 ? 0x05040100u : 0x07060302u;
#pragma unroll
  for (int h = 0; h < D / 64; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) b.codes[h][e] = __builtin_amdgcn_perm(pairs[e][1], pairs[e][0], h == 0 ? own : 0x07060302u);
}

// Weights of a step and the weighted values.
template <class DT, int D, int NT, bool MASKED>
__device__ __forceinline__ void weigh_step(const Beside<D>& v, Scores<NT>& r, Columns<D, NT>& c) {
  // Weights times scales as one binary16 number are off by up to 2^-11 of their size: an eighth of a bfloat16 result's own rounding (errors against 64 bits
  // 0.0017 to 0.0018, with the rest as a second part 0.0017; single tokens take 1 to 3 % longer with it, two prompts of 4095 rows 16 %, 834 -> 969 us),
  // and as much as a binary16 result's, which has the second part.
  constexpr bool kTwoParts = std::is_same_v<DT, F16>;
  uint32_t high[NT][4], rest[NT][4];
  auto weigh = [&](auto which) {
    constexpr int E = decltype(which)::value;
    const float vs = of_lane<8 + E>(r.scale), vm = of_lane<8 + E>(r.low);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const bool visible = !MASKED || (r.sees[n] >> E & 1u);
      const float w = visible ? __builtin_amdgcn_exp2f(fmaf(r.x[n][E], c.q[n].factor, -c.base[n])) : 0.0f;
      c.sum[n] += w;
      c.minima[n] = fmaf(w, visible ? vm : 0.0f, c.minima[n]);
      r.x[n][E] = w * (visible ? vs : 0.0f);
      if constexpr (E & 1) {
        high[n][E / 2] = pack_half(r.x[n][E - 1], r.x[n][E]);
        if constexpr (kTwoParts) {
          float a, b;
          unpack2<F16>(high[n][E / 2], a, b);
          rest[n][E / 2] = pack_half(r.x[n][E - 1] - a, r.x[n][E] - b);
        }
      }
    }
  };
  weigh(std::integral_constant<int, 0>{}), weigh(std::integral_constant<int, 1>{}), weigh(std::integral_constant<int, 2>{});
  weigh(std::integral_constant<int, 3>{}), weigh(std::integral_constant<int, 4>{}), weigh(std::integral_constant<int, 5>{});
  weigh(std::integral_constant<int, 6>{}), weigh(std::integral_constant<int, 7>{});

  // v's codes as first operands of out^T = V^T w^T: row i of output tile j is value 8 i + j of a head of 128, 8 (i % 8) + 4 (i / 8) + j of
  // one of 64
#pragma unroll
  for (int h = 0; h < D / 64; ++h) {
    uint4 parts[4];  // of a pair of positions each: tiles 4 h .. 4 h + 3
#pragma unroll
    for (int e = 0; e < 4; ++e) parts[e] = unpack_codes(v.codes[h][e]);
    const uint4 codes[4] = {make_uint4(parts[0].x, parts[1].x, parts[2].x, parts[3].x), make_uint4(parts[0].y, parts[1].y, parts[2].y, parts[3].y),
                            make_uint4(parts[0].z, parts[1].z, parts[2].z, parts[3].z), make_uint4(parts[0].w, parts[1].w, parts[2].w, parts[3].w)};
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const uint4 weights = make_uint4(high[n][0], high[n][1], high[n][2], high[n][3]);
#pragma unroll
      for (int j = 0; j < 4; ++j) c.acc[n][h * 4 + j] = mfma16x16x32<F16>(codes[j], weights, c.acc[n][h * 4 + j]);
      if constexpr (kTwoParts) {
        const uint4 more = make_uint4(rest[n][0], rest[n][1], rest[n][2], rest[n][3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) c.acc[n][h * 4 + j] = mfma16x16x32<F16>(codes[j], more, c.acc[n][h * 4 + j]);
      }
    }
  }
}

// The next step's keys and values are loaded as soon as the scores are there and the values' words put beside one another, a whole step of weights ahead: the
// compiler left to itself moves them behind it (2 to 9 % slower).
template <class DT, int D, int NT, bool ONCE>
__device__ __forceinline__ void attend_steps(const AttentionArgs& a, const Pages& p, int begin, int end, int stride_log2, int lane, Columns<D, NT>& c) {
  if (begin >= end) return;
  const Lane<D> offsets = offsets_of<D>(lane);
  // of the wave's steps, begin + (n << stride_log2), those from the head'th to the tail'th are seen whole by all columns; the others come first
  const int stride = 1 << stride_log2, count = (end - begin + stride - 1) >> stride_log2;
  auto steps_before = [&](int step) { return clamp_int((step - begin + stride - 1) >> stride_log2, 0, count); };
  const int head = steps_before((c.all.low + kStepPositions - 1) / kStepPositions), tail = max(steps_before(c.all.high / kStepPositions), head);
  const int ends = head + count - tail;
  // (behind the last one that one again: what is loaded ahead of nothing comes from a cache)
  auto step_at = [&](int n) {
    n = min(n, count - 1);
    return begin + ((n < head ? n : n < ends ? n - head + tail : n - ends + head) << stride_log2);
  };
  Held<D> held;
  // pages are looked up two steps ahead of their use: a scalar load's wait is for all of them
  Looked pages = look_up(a, p, step_at(1));
  Place at = place_of<D>(a, p, step_at(0), look_up(a, p, step_at(0))), next;
  load_k<D, ONCE>(at, offsets, held);
  load_v<D, ONCE>(at, offsets, held);
  next = place_of<D>(a, p, step_at(1), pages);
  pages = look_up(a, p, step_at(2));
  int n = 0;
  auto on = [&] {
    ++n;
    at = next;
    next = place_of<D>(a, p, step_at(n + 1), pages);
    pages = look_up(a, p, step_at(n + 2));
  };
  Scores<NT> r;
  Beside<D> beside;
  auto ahead = [&] {
    put_beside<D>(held, lane, beside);
    load_k<D, ONCE>(next, offsets, held);
    load_v<D, ONCE>(next, offsets, held);
    __builtin_amdgcn_sched_barrier(0);
  };
  while (n < ends) {
    score_step<DT, D, NT, true>(held, step_at(n) * kStepPositions, at.there, lane, c, r);
    ahead();
    if (__any(r.above)) raise<D, NT>(c, r, lane);
    weigh_step<DT, D, NT, true>(beside, r, c);
    on();
  }
  while (n < count) {
    // raise() stands outside of the inner loop, and the step is begun again for it: inside, the sums would be copied at every step
    score_step<DT, D, NT, false>(held, 0, at.there, lane, c, r);
    if (__any(r.above)) raise<D, NT>(c, r, lane);
    for (;;) {
      ahead();
      weigh_step<DT, D, NT, false>(beside, r, c);
      on();
      if (n >= count) break;
      score_step<DT, D, NT, false>(held, 0, at.there, lane, c, r);
      if (__any(r.above)) break;
    }
  }
}

// Steps [begin, end) of a slice.  `whole`: the first slice has all of the tile's, so its result is the rows', and not a part to be joined.
struct Steps {
  int begin, end;
  bool whole;
};
__device__ __forceinline__ Steps steps_of_slice(const AttentionArgs& a, const Tile& t, int columns, int slice) {
  const Span lowest = seen_by(a, t, t.first_column / a.group), highest = seen_by(a, t, (t.first_column + columns - 1) / a.group);
  const int from = lowest.low / kStepPositions;
  const int steps = highest.high > lowest.low ? (highest.high + kStepPositions - 1) / kStepPositions - from : 0;
  const int per = max(a.slice_steps, (steps + a.slices - 1) / a.slices);
  return {from + min(steps, slice * per), from + min(steps, (slice + 1) * per), steps <= per};
}

// A wave's columns, from column `first` of the request on, and those of the slice's steps that they look at.
template <class DT, int D, int NT>
__device__ __forceinline__ Steps load_columns(const AttentionArgs& a, const Tile& t, int first, int head, const Steps& slice, int lane, Columns<D, NT>& c, Pages& p) {
  start_columns<D, NT>(c, lane);
  const int last_column = min(first + 16 * NT, t.columns) - 1;
  const Span lowest = seen_by(a, t, first / a.group), highest = seen_by(a, t, last_column / a.group);
  c.some = {lowest.low, highest.high};
  c.all = {highest.low, lowest.high};
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int column = first + n * 16 + (lane & 15);
    const bool live = column < t.columns;
    const int row = live ? column / a.group : 0, of_group = live ? column - row * a.group : 0;
    c.span[n] = live ? seen_by(a, t, row) : c.some;
    load_query<DT, D>(a, a.q + (long long)(t.first_row + row) * a.q_stride + (head * a.group + of_group) * D, live, lane, c.q[n]);
  }
  p.table = (const __attribute__((address_space(4))) int32_t*)(a.tables + (size_t)t.request * a.table_width);
  p.head = a.at.layer + (size_t)head * ((1u << a.at.page_shift) / kTilePositions) * tile_bytes(D);
  p.last_tile = (c.some.high - 1) / kTilePositions;
  const int end = c.some.high > c.some.low ? (c.some.high + kStepPositions - 1) / kStepPositions : 0;
  return {max(slice.begin, c.some.low / kStepPositions), min(slice.end, end), slice.whole};
}

// Sums of a column over its four lanes.
__device__ __forceinline__ float of_column(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// (The sum's exponent meets the base before its logarithm does: of the two, up to 90 each, little may be left.)
__device__ __forceinline__ float log_sum(float base, float sum) {
  const float exponent = (float)__builtin_amdgcn_frexp_expf(sum), rest = log2f(__builtin_amdgcn_frexp_mantf(sum));
  return sum == 0.0f ? -__uint_as_float(0x7F800000u) : (base + exponent + rest) * 0.693147180559945309f;
}

// What the sum of a row's first slice is where that slice has been written as the row's result.
constexpr float kWritten = -1.0f;

// Values of a column from `value` on, unnormalised, into the result (whole) or into the slice's part.
template <class DT, int D, int N>
__device__ __forceinline__ void put_values(const AttentionArgs& a, bool whole, long long row, int q_head, int slice, int value, const float (&v)[N], float sum) {
  if (!whole) {
    if (sum == 0.0f) return;  // the join passes such parts by
    const size_t part = ((size_t)row * a.n_heads + q_head) * a.slices + slice;
#pragma unroll
    for (int k = 0; k < N; k += 4) *reinterpret_cast<float4*>(a.sums + part * D + value + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
    return;
  }
  const float inverse = 1.0f / sum;
  uint2* to = reinterpret_cast<uint2*>(a.out + row * a.out_stride + q_head * D + value);
#pragma unroll
  for (int k = 0; k < N; k += 4) {
    float w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = sum == 0.0f ? 0.0f : v[k + e] * inverse;
    to[k / 4] = make_uint2(pack2<DT>(w[0], w[1]), pack2<DT>(w[2], w[3]));
  }
}
__device__ __forceinline__ void put_sum(const AttentionArgs& a, bool whole, long long row, int q_head, int slice, float base, float sum) {
  const size_t item = (size_t)row * a.n_heads + q_head;
  if (whole && a.lse != nullptr) a.lse[item] = log_sum(base, sum);
  if (a.slices > 1) a.tops[item * a.slices + slice] = make_float2(base, whole ? kWritten : sum);
}

// What the waves of a workgroup that share columns hand to one another.
template <int D, int NT>
struct Shared {
  float sums[4][16 * NT][D + 4];
  float4 stats[4][16 * NT];  // worth of a weight of 1 in powers of two, sum of weights, of weights times minima
};

// A tile's columns.  The four waves are 2^groups_log2 groups, of which each takes 16 NT columns; the waves of a group take the steps in turn and meet in
// LDS.  HEADS (groups_log2 is 2): every wave takes all columns of a head of its own, from `first_head` on.
template <class DT, int D, int NT, bool HEADS, bool ONCE>
__device__ __forceinline__ void attend_tile(const AttentionArgs& a, const Tile& t, int columns, int first_head, int groups_log2, int slice, Shared<D, NT>& shared) {
  constexpr int PER = 16 * NT;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, i = lane & 15;
  const int group = wave & ((1 << groups_log2) - 1);
  const int first = HEADS ? t.first_column : t.first_column + group * PER, head = HEADS ? first_head + group : first_head;
  const Steps of_slice = steps_of_slice(a, t, columns, slice);
  if (of_slice.whole && slice > 0) return;
  Columns<D, NT> c;
  if (HEADS ? head < a.at.n_kv_heads : first < t.columns) {
    Pages p;
    const Steps steps = load_columns<DT, D, NT>(a, t, first, head, of_slice, lane, c, p);
    attend_steps<DT, D, NT, ONCE>(a, p, steps.begin + (wave >> groups_log2), steps.end, 2 - groups_log2, lane, c);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      // a query without a factor (see load_query): by what is its to see, not by what its steps' products made of it
      const bool moved = c.unit < kLeastUnit || is_far(c, n);
      const float worth = moved ? ldexpf(1.0f, kLeastUnit - c.unit) : 1.0f;
      const float sum = isnan(c.q[n].factor) ? (c.span[n].high > c.span[n].low ? c.q[n].factor : 0.0f) : of_column(c.sum[n]) * worth;
      const float minima = of_column(c.minima[n]) * worth;
      const float base = sum == 0.0f ? kLowest : moved ? fmaf(c.top[n], c.q[n].factor, -(float)kLeastUnit) : c.base[n];
      const int column = first + n * 16 + i;
      if (column >= t.columns) continue;
      const int row = column / a.group, q_head = head * a.group + column - row * a.group;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int value = value_of<D>(4 * g + r);
        float v[D / 16];
#pragma unroll
        for (int j = 0; j < D / 16; ++j) v[j] = c.acc[n][j][r] * (worth * 0x1p20f);
        if (groups_log2 < 2) {
#pragma unroll
          for (int j = 0; j < D / 16; ++j) shared.sums[wave][n * 16 + i][value + j] = v[j];
        } else {
#pragma unroll
          for (int j = 0; j < D / 16; ++j) v[j] += minima;
          put_values<DT, D>(a, of_slice.whole, t.first_row + row, q_head, slice, value, v, sum);
        }
      }
      if (g != 0) continue;
      if (groups_log2 < 2)
        shared.stats[wave][n * 16 + i] = make_float4(base, sum, minima, 0.0f);
      else
        put_sum(a, of_slice.whole, t.first_row + row, q_head, slice, base, sum);
    }
  }
  if (HEADS || groups_log2 == 2) return;
  __syncthreads();
  // sixteen threads to a column
  const int waves = 4 >> groups_log2, part = threadIdx.x & 15;
  for (int j = threadIdx.x >> 4; j < columns; j += 16) {
    const int from = j / PER, at = j % PER;
    float base = kLowest;
    for (int w = 0; w < waves; ++w) base = fmaxf(base, shared.stats[(w << groups_log2) + from][at].x);
    float sum = 0.0f, minima = 0.0f, v[D / 16] = {};
    for (int w = 0; w < waves; ++w) {
      const int of = (w << groups_log2) + from;
      const float4 stat = shared.stats[of][at];
      const float weight = __builtin_amdgcn_exp2f(stat.x - base);
      sum = fmaf(weight, stat.y, sum);
      minima = fmaf(weight, stat.z, minima);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) v[k] = fmaf(weight, shared.sums[of][at][part * (D / 16) + k], v[k]);
    }
#pragma unroll
    for (int k = 0; k < D / 16; ++k) v[k] += minima;
    const int column = t.first_column + j, row = column / a.group, q_head = first_head * a.group + column - row * a.group;
    put_values<DT, D>(a, of_slice.whole, t.first_row + row, q_head, slice, part * (D / 16), v, sum);
    if (part == 0) put_sum(a, of_slice.whole, t.first_row + row, q_head, slice, base, sum);
  }
}

// Most requests of a batch whose tiles are ordered by their work.
constexpr int kMostOrdered = 512;
struct Ordered {
  int first_row[kMostOrdered + 1], kv_len[kMostOrdered];
};
// The n-th of `tiles` tiles, those with many steps to a wave first: 128 at a time, from the last ones on, in eight classes next to the longest of these.
// False where it holds no rows.  `per_wave`: columns of a wave.
__device__ __forceinline__ bool tile_by_work(const AttentionArgs& a, int columns_log2, int per_wave, int tiles, int n, Ordered& o, Tile& t) {
  const int lane = threadIdx.x & 63;
  for (int i = threadIdx.x; i <= a.n_reqs; i += 256) {
    o.first_row[i] = clamp_int(a.q_starts[i], 0, a.n_tokens);
    if (i < a.n_reqs) o.kv_len[i] = clamp_int(a.kv_lens[i], 0, a.table_width << a.at.page_shift);
  }
  __syncthreads();
  auto tiles_before = [&](int i) { return (int)(((long long)o.first_row[i] * a.group) >> columns_log2) + i; };
  const int end = tiles - (n & ~127), first = end > 128 ? end - 128 : 0;
  int of[2], request[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int tile = first + k * 64 + lane;
    int low = 0, high = a.n_reqs - 1;  // the last request that starts at this tile or before it
    while (low < high) {
      const int mid = (low + high + 1) >> 1;
      if (tiles_before(mid) <= tile)
        low = mid;
      else
        high = mid - 1;
    }
    const int rows = max(o.first_row[low + 1] - o.first_row[low], 0), columns = rows * a.group, column = (tile - tiles_before(low)) << columns_log2;
    const int last_row = (min(column + (1 << columns_log2), columns) - 1) / a.group;
    const int sees = a.causal ? clamp_int(o.kv_len[low] - rows + last_row + 1, 0, o.kv_len[low]) : o.kv_len[low];
    // waves that share the columns share the steps
    const int live = columns - column, of_wave = (a.window > 0 ? min(sees, a.window) : sees) >> (live <= per_wave ? 2 : live <= 2 * per_wave ? 1 : 0);
    of[k] = tile >= end ? -1 : column < 0 || column >= columns ? 0 : of_wave;
    request[k] = low;
  }
  int most = max(of[0], of[1]);
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) most = max(most, __shfl_xor(most, m));
  const float classes = 8.0f / (float)(most + 1);
#pragma unroll
  for (int k = 0; k < 2; ++k) of[k] = of[k] < 0 ? -1 : min((int)((float)of[k] * classes), 7);
  int rank = n & 127;
  unsigned long long one = 0, two = 0;
  for (int c = 7; c >= 0; --c) {
    one = __ballot(of[0] == c), two = __ballot(of[1] == c);
    const int count = __popcll(one) + __popcll(two);
    if (rank < count) break;
    rank -= count;
  }
  const int in_one = __popcll(one);
  const bool second = rank >= in_one;
  const int at = nth_bit(second ? two : one, second ? rank - in_one : rank), tile = first + at + (second ? 64 : 0);
  t.request = __builtin_amdgcn_readlane(second ? request[1] : request[0], at);
  // the same in all lanes, and in scalar registers from here on
  t.first_row = __builtin_amdgcn_readfirstlane(o.first_row[t.request]);
  t.rows = max(__builtin_amdgcn_readfirstlane(o.first_row[t.request + 1]) - t.first_row, 0);
  t.columns = t.rows * a.group;
  t.kv_len = __builtin_amdgcn_readfirstlane(o.kv_len[t.request]);
  const int before = (int)(((long long)t.first_row * a.group) >> columns_log2) + t.request;
  if (tile < before || ((long long)(tile - before) << columns_log2) >= t.columns) return false;
  t.first_column = (tile - before) << columns_log2;
  return true;
}

// Up to 64 NT columns of one cache head (2^columns_log2; 2^7 where NT is 2).  grid = (cache heads x tiles, slices).
//
// Bound by the vector units, busy for 81 % of the time of two prompts of 4095 rows (the matrix cores for 29 %): a step of 32 positions takes a wave with 32
// columns some 320 instructions besides its 32 products, 126 of them for the codes of k and v whatever its columns.  8000 rows of 32 heads, 8 of the
// cache, bfloat16 714 us (734 TFLOP/s), binary16, whose weights are two parts, 825 to 835; those two prompts, 64 heads, 8 of the cache, 834.  Four tiles of sixteen
// columns to a wave would halve the codes' part: their 256 registers and more to a lane leave one wave to a SIMD, 2100 us.  Codes unpacked once for the
// four waves, through LDS: a quarter fewer instructions, 877 us where this took 848, for a barrier a step.
template <class DT, int D, int NT>
__global__ __launch_bounds__(256, NT == 1 ? 3 : 2) void attention_many_kernel(AttentionArgs a, int first_tile, int tiles) {
  const int log2 = NT == 1 ? a.columns_log2 : 7;
  __shared__ Shared<D, NT> shared;
  __shared__ Ordered ordered;
  const int head = blockIdx.x % a.at.n_kv_heads, n = (int)(blockIdx.x / a.at.n_kv_heads), slice = blockIdx.y;
  Tile t;
  if (a.ordered) {
    if (!tile_by_work(a, log2, 16 * NT, tiles, n, ordered, t)) return;
  } else if (!tile_of_batch(a, log2, first_tile + tiles - 1 - n, t)) {
    return;
  }
  const int columns = min(t.columns - t.first_column, 1 << log2);
  if (NT > 1 && columns <= 16)
    attend_tile<DT, D, 1, false, false>(a, t, columns, head, 0, slice, reinterpret_cast<Shared<D, 1>&>(shared));
  else
    attend_tile<DT, D, NT, false, false>(a, t, columns, head, columns <= 16 * NT ? 0 : columns <= 32 * NT ? 1 : 2, slice, shared);
}

// Requests of up to sixteen columns (more than the hint said: sixteen after sixteen), 2^HEADS_LOG2 cache heads to a workgroup.
// grid = (cache heads / that x requests, slices).
//
// Bound by memory: 64 requests of 2048 positions, 32 heads, 571 MB, 98 us (5.9 TB/s, as a read of 1 GiB), of 512 to 2048 73 us (5.2; the last long ones are
// alone), of 512 28.9; one of 130 000 positions, 8 heads, in 64 slices 29 us and 5 for their join.  Three waves to a SIMD: four (128 registers)
// spill, two with two steps held at once are 3 % slower.
template <class DT, int D, int HEADS_LOG2>
__global__ __launch_bounds__(256, 3) void attention_few_kernel(AttentionArgs a, int first_request) {
  __shared__ Shared<D, 1> shared;
  const int blocks = (a.at.n_kv_heads + (1 << HEADS_LOG2) - 1) >> HEADS_LOG2, head = (int)(blockIdx.x % blocks) << HEADS_LOG2;
  const int request = request_by_length(a, first_request + (int)(blockIdx.x / blocks)), slice = blockIdx.y;
  Tile t;
  if (!whole_request(a, request, t)) return;
  for (; t.first_column < t.columns; t.first_column += kFewColumns) {
    attend_tile<DT, D, 1, (HEADS_LOG2 > 0), true>(a, t, min(t.columns - t.first_column, kFewColumns), head, HEADS_LOG2, slice, shared);
    __syncthreads();
  }
}

// Joins the slices of rows' heads that are in parts: D / 4 threads take four values each, GROUPS such sets of threads the slices of one head in turn
// (few rows, many slices) or, with one, a head each.  grid = rows x heads / (256 / (GROUPS D / 4)).
template <class DT, int D, int GROUPS>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a, long long first) {
  constexpr int THREADS = D / 4, ITEMS = 256 / (THREADS * GROUPS);
  __shared__ float4 parts[GROUPS][THREADS];
  __shared__ float sums[GROUPS];
  const int part = threadIdx.x % THREADS, group = threadIdx.x / THREADS % GROUPS;
  const long long item = first + (long long)blockIdx.x * ITEMS + threadIdx.x / (THREADS * GROUPS);
  if (item >= (long long)a.n_tokens * a.n_heads) return;
  const int row = (int)(item / a.n_heads), head = (int)(item - (long long)row * a.n_heads);
  if (row < a.q_starts[0] || row >= a.q_starts[a.n_reqs]) return;
  const float2* tops = a.tops + item * a.slices;
  if (tops[0].y == kWritten) return;
  float top = kLowest;
  for (int z = part; z < a.slices; z += THREADS) top = fmaxf(top, tops[z].x);
#pragma unroll
  for (int m = 1; m < THREADS; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  float sum = 0.0f;
#pragma unroll 4
  for (int z = group; z < a.slices; z += GROUPS) {
    const float2 of = tops[z];
    if (of.y == 0.0f) continue;  // a slice that sees nothing: no values are there
    const float4 x = *reinterpret_cast<const float4*>(a.sums + (item * a.slices + z) * D + part * 4);
    const float w = __builtin_amdgcn_exp2f(of.x - top);
    sum = fmaf(w, of.y, sum);
    v.x = fmaf(w, x.x, v.x), v.y = fmaf(w, x.y, v.y), v.z = fmaf(w, x.z, v.z), v.w = fmaf(w, x.w, v.w);
  }
  if (GROUPS > 1) {
    parts[group][part] = v;
    if (part == 0) sums[group] = sum;
    __syncthreads();
    if (group != 0) return;
    for (int k = 1; k < GROUPS; ++k) {
      const float4 x = parts[k][part];
      v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
      sum += sums[k];
    }
  }
  const float inverse = 1.0f / sum;
  const bool none = sum == 0.0f;
  *reinterpret_cast<uint2*>(a.out + (long long)row * a.out_stride + head * D + part * 4) =
      make_uint2(none ? 0 : pack2<DT>(v.x * inverse, v.y * inverse), none ? 0 : pack2<DT>(v.z * inverse, v.w * inverse));
  if (a.lse != nullptr && part == 0) a.lse[item] = log_sum(top, sum);
}

// Launches over ranges of tiles, fewer than 2^31 threads each.
template <class F>
hipError_t by_tiles(const AttentionArgs& a, F launch) {
  const long long tiles = a.few ? a.n_reqs : attention_tiles(a.n_tokens, a.group, a.n_reqs, 1 << a.columns_log2);
  const int blocks = a.few ? (a.at.n_kv_heads + (1 << a.heads_log2) - 1) >> a.heads_log2 : a.at.n_kv_heads;
  // whole sixty-fours of requests
  const long long share = (1LL << 30) / 256 / a.slices / blocks & ~63LL, most = share > 0 ? share : 64;
  for (long long first = 0; first < tiles; first += most) {
    const long long n = tiles - first < most ? tiles - first : most;
    launch(dim3((unsigned)(n * blocks), (unsigned)a.slices), (int)first, (int)n);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

template <class DT, int D>
hipError_t columns_typed(AttentionArgs a, hipStream_t st) {
  // In the order of their work where the launch goes through the chip a few times at most (eight prompts of up to 1024 rows, 32 heads, 1376 workgroups: 101 -> 86 us; two of
  // 4095 rows, 4104 workgroups: 848 -> 882); of one request the last tiles are the ones with most work anyway.
  a.ordered = a.n_reqs > 1 && a.n_reqs <= kMostOrdered;
  const long long groups = attention_tiles(a.n_tokens, a.group, a.n_reqs, 1 << a.columns_log2) * a.at.n_kv_heads * a.slices;
  a.ordered = a.ordered && groups > 2LL * compute_units() && groups <= 8LL * compute_units();
  return by_tiles(a, [&](dim3 grid, int first, int n) {
    if (a.few && a.heads_log2 == 0)
      attention_few_kernel<DT, D, 0><<<grid, 256, 0, st>>>(a, first);
    else if (a.few)
      attention_few_kernel<DT, D, 2><<<grid, 256, 0, st>>>(a, first);
    else if (1 << a.columns_log2 < kManyColumns)
      attention_many_kernel<DT, D, 1><<<grid, 256, 0, st>>>(a, first, n);
    else
      attention_many_kernel<DT, D, 2><<<grid, 256, 0, st>>>(a, first, n);
  });
}

template <class DT, int D>
hipError_t join_typed(const AttentionArgs& a, hipStream_t st) {
  constexpr int kAll = 256 / (D / 4);
  // a workgroup to a head while these are few; with many, one after the other has enough to load
  const bool few = (long long)a.n_tokens * a.n_heads <= 4096;
  const long long items = (long long)a.n_tokens * a.n_heads, most = 1LL << 22;
  for (long long first = 0; first < items; first += most) {
    const long long n = items - first < most ? items - first : most;
    if (few)
      attention_join_kernel<DT, D, kAll><<<(unsigned)n, 256, 0, st>>>(a, first);
    else
      attention_join_kernel<DT, D, 1><<<(unsigned)((n + kAll - 1) / kAll), 256, 0, st>>>(a, first);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_attention(const AttentionArgs& a, hipStream_t st) {
  if (a.bf16) return a.at.head_dim == 64 ? columns_typed<BF16, 64>(a, st) : columns_typed<BF16, 128>(a, st);
  return a.at.head_dim == 64 ? columns_typed<F16, 64>(a, st) : columns_typed<F16, 128>(a, st);
}

hipError_t launch_attention_join(const AttentionArgs& a, hipStream_t st) {
  if (a.bf16) return a.at.head_dim == 64 ? join_typed<BF16, 64>(a, st) : join_typed<BF16, 128>(a, st);
  return a.at.head_dim == 64 ? join_typed<F16, 64>(a, st) : join_typed<F16, 128>(a, st);
}

}  // namespace sgmv
