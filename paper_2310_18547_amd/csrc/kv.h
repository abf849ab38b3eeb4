// Host-side launch descriptors of the paged 4-bit cache's kernels (kv_assign.hip, kv_rows.hip, kv_attention.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sgmv {

// Positions of a tile of the cache (one head): codes of k, codes of v, (scale, minimum) of k and of v for every position.
constexpr int kTilePositions = 16;
__host__ __device__ constexpr int tile_bytes(int head_dim) { return 16 * head_dim + 128; }

struct KvAssignArgs {
  int page_shift, n_pages, n_reqs, n_tokens, table_width;
  const int32_t* new_lens;
  const int32_t* old_lens;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* free_count_out;
  int32_t* q_starts;
  int32_t* kv_lens;
  int32_t* tables;
  int32_t* slots;
  int32_t* positions;
  int32_t* status;
};
hipError_t launch_kv_assign(const KvAssignArgs& a, hipStream_t st);

// Where the rows of a layer lie in the pages.
struct KvPlace {
  int head_dim, n_kv_heads, page_shift;
  uint32_t n_slots;          // n_pages << page_shift
  size_t page_stride;        // bytes
  uint8_t* layer;            // pages + the layer's offset in a page
};
struct KvAppendArgs {
  bool bf16;
  KvPlace at;
  int n_tokens, n_heads;     // n_heads 0: q is not rotated
  uint16_t* q_out;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  long long q_out_stride, q_stride, kv_stride;
  const int32_t* slots;
  const int32_t* positions;
  const float* rope;         // nullptr: nothing is rotated
  int rope_rows, rope_dim;
  bool adjacent;
};
hipError_t launch_kv_append(const KvAppendArgs& a, hipStream_t st);

struct KvReadArgs {
  bool bf16;
  KvPlace at;
  int n_rows;
  uint16_t* k;               // either may be nullptr
  uint16_t* v;
  long long kv_stride;
  const int32_t* slots;
};
hipError_t launch_kv_read(const KvReadArgs& a, hipStream_t st);

// Columns of an attention workgroup's tile: rows x query heads of one cache head's group, row by row; of all of a request, or of a tile of the batch at most.
constexpr int kFewColumns = 16, kManyColumns = 128;
// Positions of one step of a wave.
constexpr int kStepPositions = 32;
struct AttentionArgs {
  bool bf16;
  KvPlace at;
  int n_pages;
  int n_heads, group, n_reqs, n_tokens, table_width;
  int causal, window;
  float scale;
  bool few;                  // whole requests, kFewColumns at a time; else tiles of the batch
  int columns_log2;          // of a tile, 4 to 7
  int heads_log2;            // few: cache heads of a workgroup, one (whose steps its waves share) or 2^2 (a wave each)
  uint16_t* out;
  float* lse;
  const uint16_t* q;
  long long out_stride, q_stride;
  const int32_t* q_starts;
  const int32_t* kv_lens;
  const int32_t* tables;
  float classes;             // classes of lengths for a position (request_by_length)
  bool ordered;              // tiles by their work (tile_by_work), set at launch
  int slices;                // parts of a tile's positions (workgroups), joined by a second launch where there are several
  int slice_steps;           // steps of a slice at least
  float* sums;               // slices > 1: [n_tokens][n_heads][slices][head_dim] unnormalised, then ...
  float2* tops;              // ... {maximum in powers of two, sum} of each
};
hipError_t launch_attention(const AttentionArgs& a, hipStream_t st);
hipError_t launch_attention_join(const AttentionArgs& a, hipStream_t st);

// Tiles of so many columns: a request's may start in the middle of one of the batch's, so each adds one.
inline long long attention_tiles(long long n_tokens, int group, int n_reqs, int columns) { return n_tokens * group / columns + n_reqs; }

}  // namespace sgmv
