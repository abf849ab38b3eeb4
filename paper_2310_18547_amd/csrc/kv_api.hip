// C ABI of the paged 4-bit cache and attention over it: argument checks and dispatch (include/sgmv.h, last but one section).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sgmv.h"
#include "kv.h"
#include "launch.h"
#include "spans.h"

namespace {

using namespace sgmv;

// Most heads, and most positions that a request's block table covers.
constexpr int kMostHeads = 1 << 16, kMostPositions = 1 << 30;
// Most parts of a request's positions.
constexpr int kMostSlices = 256;
int check_cache(const sgmv_kv_cache* c) {
  if (c == nullptr) return SGMV_ERR_NULL;
  if (c->dtype != SGMV_F16 && c->dtype != SGMV_BF16) return SGMV_ERR_UNSUPPORTED;
  if (c->n_kv_heads <= 0 || c->num_layers <= 0 || c->n_pages <= 0 || c->page_size <= 0 || c->head_dim <= 0) return SGMV_ERR_SHAPE;
  if (c->head_dim != 64 && c->head_dim != 128) return SGMV_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)) != 0) return SGMV_ERR_UNSUPPORTED;
  if (c->n_kv_heads > kMostHeads || (long long)c->n_pages * c->page_size > INT32_MAX) return SGMV_ERR_UNSUPPORTED;
  return SGMV_OK;
}

size_t head_bytes(const sgmv_kv_cache* c) { return (size_t)(c->page_size / kTilePositions) * tile_bytes(c->head_dim); }
size_t page_bytes(const sgmv_kv_cache* c) { return head_bytes(c) * (size_t)c->n_kv_heads * (size_t)c->num_layers; }
size_t page_stride(const sgmv_kv_cache* c) { return c->page_stride == 0 ? page_bytes(c) : c->page_stride; }
Span pages_of(const sgmv_kv_cache* c) { return {c->pages, page_stride(c) * (size_t)(c->n_pages - 1) + page_bytes(c)}; }

// A call that reads or writes a layer's rows.
int check_pages(const sgmv_kv_cache* c, int32_t layer_idx) {
  if (layer_idx < 0 || layer_idx >= c->num_layers) return SGMV_ERR_RANGE;
  if (c->page_stride != 0 && (c->page_stride < page_bytes(c) || c->page_stride > SIZE_MAX / 4 / (size_t)c->n_pages)) return SGMV_ERR_SHAPE;
  if (c->pages == nullptr) return SGMV_ERR_NULL;
  return aligned(c->pages, 16) && c->page_stride % 16 == 0 ? SGMV_OK : SGMV_ERR_ALIGN;
}

int shift_of(int32_t page_size) { return __builtin_ctz((unsigned)page_size); }

KvPlace place_of(const sgmv_kv_cache* c, int32_t layer_idx) {
  return {c->head_dim, c->n_kv_heads, shift_of(c->page_size), (uint32_t)c->n_pages * (uint32_t)c->page_size, page_stride(c),
          static_cast<uint8_t*>(c->pages) + (size_t)layer_idx * head_bytes(c) * (size_t)c->n_kv_heads};
}

int check_batch(const sgmv_kv_cache* c, const sgmv_kv_batch* b) {
  if (b == nullptr) return SGMV_ERR_NULL;
  if (b->n_reqs < 0 || b->n_tokens < 0 || b->table_width < 0 || b->max_q_len < 0 || b->max_kv_len < 0) return SGMV_ERR_SHAPE;
  if ((long long)b->table_width * c->page_size > kMostPositions || b->n_reqs > kMostPositions || b->n_tokens > kMostPositions) return SGMV_ERR_UNSUPPORTED;
  return SGMV_OK;
}

// 16-bit rows of a call: `row` bytes at every `stride` bytes; none where `at` is nullptr.
struct Rows {
  const void* at;
  size_t n, row, stride;
};
Span span_of(const Rows& r) { return {r.at, r.n == 0 ? 0 : (r.n - 1) * r.stride + r.row}; }
// Rows at the same stride may lie between one another, as the parts of one wider row do.
bool overlap(const Rows& a, const Rows& b) {
  if (!overlap(span_of(a), span_of(b))) return false;
  if (a.stride != b.stride) return true;
  const uintptr_t from = reinterpret_cast<uintptr_t>(a.at), to = reinterpret_cast<uintptr_t>(b.at);
  const size_t apart = from <= to ? (to - from) % a.stride : a.stride - 1 - (from - to - 1) % a.stride;  // of b's row from the a's row before it
  return apart < a.row || apart + b.row > a.stride;
}
int check_stride(int64_t stride, long long values, int32_t n) {
  if (stride < values || stride > INT64_MAX / 4 / (n > 0 ? n : 1)) return SGMV_ERR_SHAPE;
  return stride % 8 == 0 ? SGMV_OK : SGMV_ERR_SHAPE;
}
Rows rows_of(const void* at, int32_t n, long long values, int64_t stride) { return {at, (size_t)n, (size_t)(2 * values), (size_t)(2 * stride)}; }
bool overlap(const Rows& a, const Span& b) { return overlap(span_of(a), b); }

// What an attention call and its plan refuse alike; `*nothing`: the call has nothing to do.
int check_attention(const sgmv_kv_cache* c, const sgmv_kv_batch* b, int32_t n_heads, const void* workspace, size_t workspace_bytes, bool* nothing) {
  *nothing = true;
  int rc = check_cache(c);
  if (rc == SGMV_OK) rc = check_batch(c, b);
  if (rc != SGMV_OK) return rc;
  if (n_heads <= 0 || n_heads % c->n_kv_heads != 0 || workspace_bytes > SIZE_MAX / 2) return SGMV_ERR_SHAPE;
  if (n_heads > kMostHeads || (long long)b->n_tokens * n_heads > INT32_MAX) return SGMV_ERR_UNSUPPORTED;
  *nothing = b->n_reqs == 0 || b->n_tokens == 0;
  return aligned(workspace, 256) ? SGMV_OK : SGMV_ERR_ALIGN;
}

struct AttentionPlan {
  bool few;
  int columns_log2, heads_log2, slices, slice_steps;
  long long workgroups;
};
size_t slice_bytes(const sgmv_kv_cache* c, const sgmv_kv_batch* b, int32_t n_heads) {
  return (size_t)b->n_tokens * (size_t)n_heads * (4 * (size_t)c->head_dim + 8);
}
// Time of an attention launch in us, to choose the kernel, the tiles and the slices by.
//
// Few columns: one, two and three workgroups to a unit take 1.2, 1.6 and 2.4 us for a step of 32 positions (the loads; 131 000 positions in 48, 64 and
// 96 slices: 1.5, 1.8, 2.4), a workgroup's lookups, queries and end 4 us (64 requests of 512 to 2048 positions, 32 heads, take two thirds more in
// six slices than whole), and a batch's last round is half empty.
// Tiles: 1.1 us a step and 4 us around them while tiles are few (1.15 and 6 where a wave has 32 columns), 1.4 (1.6) and 6.5 us where they queue
// for units.  300 rows, 32 heads, in tiles of 16 / 32 / 64 / 128: 10 / 11 / 15 / 19 us; 600 and 600 rows 36 / 32 / 28 / 35; 8 prompts of up to 1024
// 127 / 101 / 104 / 85; 453 rows next to 64 single tokens, 8 heads shared by 4 each, 36 / 30 / 26 / 32.
// A join takes 3 us and its sums' way there and back at 4 TB/s.
struct Estimate {
  double rows, heads, tile_bytes, units;
  double join(int slices) const { return slices > 1 ? 3.0 + rows * heads * slices * tile_bytes / 2 / 4e6 : 0.0; }
  // `groups` workgroups of a slice, of at most `steps` steps to a wave
  double few(double groups, double steps, double mean_steps, int slices) const {
    const double total = groups * slices, slots = 3 * units;
    const int waves = total >= slots ? 3 : (int)((total + units - 1) / units);
    const double step = waves == 1 ? 1.2 : waves == 2 ? 1.6 : 2.4;
    const double longest = (double)(long long)(steps + 0.999) * step + 4.0;
    const double all = total > slots ? (total / slots + 0.5) * (mean_steps * step + 4.0) : 0.0;
    return 1.5 + (longest > all ? longest : all) + join(slices);
  }
  // `steps` of all tiles together
  double many(int columns, double groups, double steps, double all_steps, int slices) const {
    const bool wide = columns == kManyColumns;
    const double total = groups * slices, slots = (wide ? 2 : 3) * units;
    const double longest = (double)(long long)(steps + 0.999) * (wide ? 1.15 : 1.1) + (wide ? 6.0 : 4.0);
    const double all = total > slots ? (total / slots + 0.4) * (all_steps / groups * (wide ? 1.6 : 1.4) + 6.5) : 0.0;
    return 1.5 + (longest > all ? longest : all) + join(slices);
  }
};
// `room`: bytes of workspace.
AttentionPlan plan_attention(const sgmv_kv_cache* c, const sgmv_kv_batch* b, int32_t n_heads, int32_t window, size_t room) {
  const long long group = n_heads / c->n_kv_heads, covered = (long long)b->table_width * c->page_size;
  const long long rows = b->max_q_len > 0 ? (b->max_q_len < b->n_tokens ? b->max_q_len : b->n_tokens) : (b->n_tokens + b->n_reqs - 1LL) / b->n_reqs;
  long long longest = b->max_kv_len > 0 && b->max_kv_len < covered ? b->max_kv_len : covered;
  if (window > 0 && longest > window + rows) longest = window + rows;
  const long long steps = longest > 0 ? (longest + kStepPositions - 1) / kStepPositions : 1;
  const long long fit = (long long)(room / slice_bytes(c, b, n_heads)), most = fit < 1 ? 1 : fit < kMostSlices ? fit : kMostSlices;
  Estimate e = {};
  e.rows = b->n_tokens;
  e.heads = n_heads;
  e.tile_bytes = tile_bytes(c->head_dim);
  e.units = compute_units();
  AttentionPlan p = {};
  p.few = rows * group <= kFewColumns;
  double best = 0;
  static const int kSlices[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256};
  const double seen = (double)steps - (double)(rows < longest ? rows : longest) / (2 * kStepPositions);  // by an average row
  // Requests with the most rows, if the others have one each (over 0.6 of the longest context on average).  Prompts next to single tokens are taken for new ones, shorter than the longest context, unless
  // that is much longer than a prompt (a part of a long one may then stand at its end, and slices that nobody needs cost less than one
  // workgroup that goes through all of it).
  const long long more = b->n_tokens - b->n_reqs, full = rows > 1 ? (more + rows - 2) / (rows - 1) : b->n_reqs;
  const long long prompts = full < 1 ? 1 : full < b->n_reqs ? full : b->n_reqs, others = b->n_reqs - prompts;
  const bool fresh = prompts <= b->n_reqs / 2 && longest <= 6 * rows;
  const double prompt_steps = fresh ? (double)((rows + kStepPositions - 1) / kStepPositions) : (double)steps, prompt_mean = fresh ? prompt_steps / 2 : seen;
  for (int log2 = 4; log2 <= (p.few ? 4 : 7); ++log2) {
    const int columns = 1 << log2;
    // tiles of requests that all have the most rows, or of the whole batch if that is less
    const long long all = p.few ? b->n_reqs : attention_tiles(b->n_tokens, (int)group, b->n_reqs, columns);
    const long long busiest = b->n_reqs * ((rows * group + columns - 1) / columns), tiles = all < busiest ? all : busiest;
    const long long per_wave = columns == kManyColumns ? 32 : 16;
    auto share_of = [&](long long live) { return live <= per_wave ? 4 : live <= 2 * per_wave ? 2 : 1; };
    const int share = share_of(rows * group < columns ? rows * group : columns), other_share = share_of(group < columns ? group : columns);
    const long long of_prompts = tiles > others ? tiles - others : 0;
    const double groups = (double)(tiles * c->n_kv_heads);
    for (const int slices : kSlices) {
      if (slices > most || (slices > 1 && slices * share > steps)) break;
      double us;
      if (p.few) {
        us = e.few(groups, (double)steps / slices / share, seen / slices / share, slices);
      } else {
        const double one = prompt_steps / share, other = others > 0 ? (double)steps / other_share : 0.0;
        us = e.many(columns, groups, (one > other ? one : other) / slices, (double)c->n_kv_heads * ((double)of_prompts * prompt_mean / share + (double)others * other * 0.6) / slices, slices);
      }
      if (best > 0 && us >= best) continue;
      best = us;
      p.columns_log2 = log2;
      p.slices = slices;
      p.slice_steps = (int)((steps + slices - 1) / slices);
      p.workgroups = all * c->n_kv_heads * slices;
    }
  }
  // A wave to a head saves its waves' common start and end where there are heads enough and all contexts are short (64 requests of 32 heads, a head to a
  // workgroup / to a wave: 128 positions 20.7 / 13.1 us, 512 37.2 / 31.8, 768 47.4 / 44.2; but 100 to 1000 39 / 45, 512 to 2048 73 / 87, where the
  // longest are left running; all some 5 % less since).
  if (p.few && p.slices == 1 && steps <= 20 && b->n_reqs * (long long)c->n_kv_heads >= 6LL * compute_units()) {
    p.heads_log2 = 2;
    p.workgroups = b->n_reqs * ((c->n_kv_heads + 3LL) / 4);
  }
  return p;
}

}  // namespace

extern "C" {

size_t sgmv_kv_page_bytes(const sgmv_kv_cache* c) { return check_cache(c) == SGMV_OK ? page_bytes(c) : 0; }

int sgmv_kv_assign(const sgmv_kv_cache* c, const sgmv_kv_batch* b, const int32_t* new_lens, const int32_t* old_lens, int32_t* free_pages,
                   const int32_t* free_count, int32_t* free_count_out, int32_t* status, void* stream) {
  int rc = check_cache(c);
  if (rc == SGMV_OK) rc = check_batch(c, b);
  if (rc != SGMV_OK || b->n_reqs == 0) return rc;
  if (new_lens == nullptr || old_lens == nullptr || free_pages == nullptr || free_count == nullptr || free_count_out == nullptr || status == nullptr) return SGMV_ERR_NULL;
  if (b->q_starts == nullptr || b->kv_lens == nullptr || (b->tables == nullptr && b->table_width > 0)) return SGMV_ERR_NULL;
  if (b->n_tokens > 0 && (b->slots == nullptr || b->positions == nullptr)) return SGMV_ERR_NULL;
  const size_t reqs = 4 * (size_t)b->n_reqs, tokens = 4 * (size_t)b->n_tokens;
  const Span written[] = {{b->q_starts, reqs + 4}, {b->kv_lens, reqs}, {b->tables, reqs * (size_t)b->table_width}, {b->slots, tokens},
                          {b->positions, tokens}, {free_pages, 4 * (size_t)c->n_pages}, {free_count_out, 4}, {status, 8}};
  const Span read[] = {{new_lens, reqs}, {old_lens, reqs}, {free_count, 4}};
  for (const Span& s : written)
    if (!aligned(s.at, 4)) return SGMV_ERR_ALIGN;
  for (const Span& s : read)
    if (!aligned(s.at, 4)) return SGMV_ERR_ALIGN;
  for (int i = 0; i < 8; ++i) {
    for (int j = 0; j < i; ++j)
      if (overlap(written[i], written[j])) return SGMV_ERR_SHAPE;
    for (int j = 0; j < 3; ++j) {
      const bool in_place = written[i].at == read[j].at && ((i == 1 && j == 1) || (i == 6 && j == 2));
      if (overlap(written[i], read[j]) && !in_place) return SGMV_ERR_SHAPE;
    }
  }
  const KvAssignArgs a = {shift_of(c->page_size), c->n_pages, b->n_reqs, b->n_tokens, b->table_width, new_lens, old_lens, free_pages, free_count,
                          free_count_out, b->q_starts, b->kv_lens, b->tables, b->slots, b->positions, status};
  return launch_kv_assign(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SGMV_OK : SGMV_ERR_LAUNCH;
}

int sgmv_kv_append_q4(const sgmv_kv_cache* c, const sgmv_kv_batch* b, int32_t layer_idx, void* q_out, const void* q, const void* k, const void* v,
                      int32_t n_heads, int64_t q_out_stride, int64_t q_stride, int64_t kv_stride, const sgmv_rope* rope, void* stream) {
  int rc = check_cache(c);
  if (rc == SGMV_OK) rc = check_batch(c, b);
  if (rc == SGMV_OK) rc = check_pages(c, layer_idx);
  if (rc != SGMV_OK) return rc;
  const int32_t n = b->n_tokens;
  const long long q_values = (long long)n_heads * c->head_dim, kv_values = (long long)c->n_kv_heads * c->head_dim;
  if ((q_out == nullptr) != (q == nullptr)) return SGMV_ERR_NULL;
  if (q != nullptr) {
    if (n_heads <= 0 || rope == nullptr) return SGMV_ERR_SHAPE;
    if (n_heads > kMostHeads) return SGMV_ERR_UNSUPPORTED;
    rc = check_stride(q_stride, q_values, n);
    if (rc == SGMV_OK) rc = check_stride(q_out_stride, q_values, n);
    if (rc != SGMV_OK) return rc;
  }
  rc = check_stride(kv_stride, kv_values, n);
  if (rc != SGMV_OK) return rc;
  if (rope != nullptr) {
    if (rope->rows < 0 || rope->dim <= 0) return SGMV_ERR_SHAPE;
    if (rope->dim % 16 != 0 || rope->dim > c->head_dim) return SGMV_ERR_UNSUPPORTED;
  }
  if (n == 0 || b->n_reqs == 0) return SGMV_OK;
  if (k == nullptr || v == nullptr || b->slots == nullptr) return SGMV_ERR_NULL;
  if (rope != nullptr && (rope->table == nullptr || b->positions == nullptr)) return SGMV_ERR_NULL;
  if (!aligned(q_out, 16) || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(b->slots, 4)) return SGMV_ERR_ALIGN;
  if (rope != nullptr && (!aligned(rope->table, 4) || !aligned(b->positions, 4))) return SGMV_ERR_ALIGN;
  const Rows out = rows_of(q_out, n, q_values, q_out_stride), qs = rows_of(q, n, q_values, q_stride), ks = rows_of(k, n, kv_values, kv_stride),
             vs = rows_of(v, n, kv_values, kv_stride);
  const Span pages = pages_of(c), slots = {b->slots, 4 * (size_t)n}, positions = {rope == nullptr ? nullptr : b->positions, 4 * (size_t)n},
             table = {rope == nullptr ? nullptr : rope->table, rope == nullptr ? 0 : 4 * (size_t)rope->rows * (size_t)rope->dim};
  if (overlap(out, pages) || overlap(qs, pages) || overlap(ks, pages) || overlap(vs, pages) || overlap(slots, pages) || overlap(positions, pages) ||
      overlap(table, pages))
    return SGMV_ERR_SHAPE;
  const bool in_place = q_out == q && q_out_stride == q_stride;
  if ((overlap(out, qs) && !in_place) || overlap(out, ks) || overlap(out, vs) || overlap(out, slots) || overlap(out, positions) || overlap(out, table))
    return SGMV_ERR_SHAPE;
  KvAppendArgs a = {};
  a.bf16 = c->dtype == SGMV_BF16;
  a.at = place_of(c, layer_idx);
  a.n_tokens = n;
  a.n_heads = q == nullptr ? 0 : n_heads;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.q_out_stride = q_out_stride;
  a.q_stride = q_stride;
  a.kv_stride = kv_stride;
  a.slots = b->slots;
  if (rope != nullptr) {
    a.positions = b->positions;
    a.rope = rope->table;
    a.rope_rows = rope->rows;
    a.rope_dim = rope->dim;
    a.adjacent = rope->adjacent != 0;
  }
  return launch_kv_append(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SGMV_OK : SGMV_ERR_LAUNCH;
}

int sgmv_kv_read_q4(const sgmv_kv_cache* c, int32_t layer_idx, void* k, void* v, int64_t kv_stride, const int32_t* slots, int32_t n_rows, void* stream) {
  int rc = check_cache(c);
  if (rc == SGMV_OK) rc = check_pages(c, layer_idx);
  if (rc != SGMV_OK) return rc;
  if (n_rows < 0) return SGMV_ERR_SHAPE;
  if (n_rows > kMostPositions) return SGMV_ERR_UNSUPPORTED;
  const long long values = (long long)c->n_kv_heads * c->head_dim;
  rc = check_stride(kv_stride, values, n_rows);
  if (rc != SGMV_OK || n_rows == 0) return rc;
  if ((k == nullptr && v == nullptr) || slots == nullptr) return SGMV_ERR_NULL;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4)) return SGMV_ERR_ALIGN;
  const Rows ks = rows_of(k, n_rows, values, kv_stride), vs = rows_of(v, n_rows, values, kv_stride);
  const Span at = {slots, 4 * (size_t)n_rows}, pages = pages_of(c);
  if (overlap(ks, vs) || overlap(ks, at) || overlap(vs, at) || overlap(ks, pages) || overlap(vs, pages)) return SGMV_ERR_SHAPE;
  const KvReadArgs a = {c->dtype == SGMV_BF16, place_of(c, layer_idx), n_rows, static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), kv_stride, slots};
  return launch_kv_read(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SGMV_OK : SGMV_ERR_LAUNCH;
}

int sgmv_attention_q4(const sgmv_kv_cache* c, const sgmv_kv_batch* b, int32_t layer_idx, void* out, float* lse, const void* q, int32_t n_heads,
                      int64_t out_stride, int64_t q_stride, float scale, int32_t causal, int32_t window, void* workspace, size_t workspace_bytes,
                      void* stream) {
  bool nothing = false;
  int rc = check_attention(c, b, n_heads, workspace, workspace_bytes, &nothing);
  if (rc == SGMV_OK) rc = check_pages(c, layer_idx);
  if (rc != SGMV_OK) return rc;
  if (!(scale > 0.0f) || !(scale < __builtin_inff())) return SGMV_ERR_UNSUPPORTED;
  if (window < 0) return SGMV_ERR_SHAPE;
  const long long values = (long long)n_heads * c->head_dim;
  rc = check_stride(out_stride, values, b->n_tokens);
  if (rc == SGMV_OK) rc = check_stride(q_stride, values, b->n_tokens);
  if (rc != SGMV_OK || nothing) return rc;
  if (out == nullptr || q == nullptr || b->q_starts == nullptr || b->kv_lens == nullptr || (b->tables == nullptr && b->table_width > 0)) return SGMV_ERR_NULL;
  if (!aligned(out, 16) || !aligned(q, 16)) return SGMV_ERR_ALIGN;
  const int32_t n = b->n_tokens;
  const size_t reqs = 4 * (size_t)b->n_reqs;
  const Span read[] = {{b->q_starts, reqs + 4}, {b->kv_lens, reqs}, {b->tables, reqs * (size_t)b->table_width}, pages_of(c)};
  if (!aligned(lse, 4) || !aligned(b->q_starts, 4) || !aligned(b->kv_lens, 4) || !aligned(b->tables, 4)) return SGMV_ERR_ALIGN;
  const AttentionPlan plan = plan_attention(c, b, n_heads, window, workspace == nullptr ? 0 : workspace_bytes);
  const size_t partials = plan.slices > 1 ? slice_bytes(c, b, n_heads) * (size_t)plan.slices : 0;
  const Rows outs = rows_of(out, n, values, out_stride), qs = rows_of(q, n, values, q_stride);
  const Span sums = {lse, 4 * (size_t)n * (size_t)n_heads}, scratch = {partials > 0 ? workspace : nullptr, partials};
  if (overlap(outs, qs) || overlap(outs, sums) || overlap(outs, scratch) || overlap(qs, sums) || overlap(qs, scratch) || overlap(sums, scratch)) return SGMV_ERR_SHAPE;
  for (const Span& s : read)
    if (overlap(outs, s) || overlap(sums, s) || overlap(scratch, s)) return SGMV_ERR_SHAPE;
  AttentionArgs a = {};
  a.bf16 = c->dtype == SGMV_BF16;
  a.at = place_of(c, layer_idx);
  a.n_pages = c->n_pages;
  a.n_heads = n_heads;
  a.group = n_heads / c->n_kv_heads;
  a.n_reqs = b->n_reqs;
  a.n_tokens = n;
  a.table_width = b->table_width;
  a.causal = causal != 0;
  a.window = window;
  a.scale = scale;
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.q = static_cast<const uint16_t*>(q);
  a.out_stride = out_stride;
  a.q_stride = q_stride;
  a.q_starts = b->q_starts;
  a.kv_lens = b->kv_lens;
  a.tables = b->tables;
  a.few = plan.few;
  a.columns_log2 = plan.columns_log2;
  a.heads_log2 = plan.heads_log2;
  const long long covered = (long long)b->table_width * c->page_size, hint = b->max_kv_len > 0 && b->max_kv_len < covered ? b->max_kv_len : covered;
  a.classes = 8.0f / (float)(window > 0 && window < hint ? window : hint + 1);
  a.slices = plan.slices;
  a.slice_steps = plan.slice_steps;
  a.sums = static_cast<float*>(workspace);
  a.tops = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + (size_t)n * n_heads * plan.slices * 4 * c->head_dim);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t err = launch_attention(a, st);
  if (err == hipSuccess && plan.slices > 1) err = launch_attention_join(a, st);
  return err == hipSuccess ? SGMV_OK : SGMV_ERR_LAUNCH;
}

size_t sgmv_attention_workspace_bytes(const sgmv_kv_cache* c, const sgmv_kv_batch* b, int32_t n_heads, int32_t window) {
  bool nothing = false;
  if (window < 0 || check_attention(c, b, n_heads, nullptr, 0, &nothing) != SGMV_OK || nothing) return 0;
  const AttentionPlan plan = plan_attention(c, b, n_heads, window, SIZE_MAX / 2);
  return plan.slices > 1 ? slice_bytes(c, b, n_heads) * (size_t)plan.slices : 0;
}

int sgmv_plan_attention_q4(const sgmv_kv_cache* c, const sgmv_kv_batch* b, int32_t n_heads, int32_t window, const void* workspace,
                           size_t workspace_bytes, sgmv_plan* plan) {
  if (plan == nullptr) return SGMV_ERR_NULL;
  *plan = sgmv_plan{};
  bool nothing = false;
  const int rc = check_attention(c, b, n_heads, workspace, workspace_bytes, &nothing);
  if (rc != SGMV_OK) return rc;
  if (window < 0) return SGMV_ERR_SHAPE;
  if (nothing) return rc;
  const AttentionPlan p = plan_attention(c, b, n_heads, window, workspace == nullptr ? 0 : workspace_bytes);
  plan->kernel = p.few ? SGMV_KERNEL_ATTENTION_FEW : SGMV_KERNEL_ATTENTION_MANY;
  plan->launches = p.slices > 1 ? 2 : 1;
  plan->slices = p.slices;
  plan->workgroups = p.workgroups > INT32_MAX ? INT32_MAX : (int32_t)p.workgroups;
  return SGMV_OK;
}

}  // extern "C"
