// Host-side launch descriptors of the 8-bit backbone kernels (q8_rows.hip, q8_dense.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sgmv {

// Widest row that one workgroup of the row kernels holds in registers: 1024 threads, four chunks of eight values each.
constexpr int kRowsMostWidth = 1024 * 4 * 8;
// Widest input of a dense projection: 128 * 128 * h_in stays below 2^31.
constexpr int kDenseMostHin = 131064;
// Most tokens, and widest output of a projection: rows and channels, all projections' together, are 32-bit numbers.
constexpr int kDenseMostTokens = 1 << 30, kDenseMostHout = 1 << 27;
// Most values of y in all: the workgroups of every kernel's tiles, padded to whole tiles of each projection, are a 32-bit number.
constexpr long long kDenseMostValues = 1LL << 38;
// Most projections of one sgmv_dense_q8 call.
constexpr int kDenseMostProjections = 8;

enum RowsKind { kRowsNorm, kRowsSiluMul, kRowsQuantize };

struct RowsArgs {
  RowsKind kind;
  bool bf16;
  int n_tokens, h;
  float eps;
  const void* x;         // rows; the gate of kRowsSiluMul
  const void* other;     // residual of kRowsNorm (may be nullptr), up of kRowsSiluMul
  const void* weight;    // kRowsNorm
  void* sum;             // kRowsNorm, may be nullptr
  void* out;             // 16-bit result, may be nullptr
  int8_t* q;             // 8-bit result with its scales, both or neither
  float* q_scales;
};
hipError_t launch_rows(const RowsArgs& a, hipStream_t st);

struct DenseArgs {
  bool bf16;
  int n_tokens, h_in, n_proj;
  const int8_t* q;
  const float* q_scales;
  int h_out[kDenseMostProjections];
  const int8_t* w[kDenseMostProjections];
  const float* w_scales[kDenseMostProjections];
  void* y[kDenseMostProjections];
  void* workspace;       // may be nullptr
  size_t workspace_bytes;
};
enum DenseFamily { kDenseFew, kDenseSmall, kDenseLarge };
struct DensePlan {
  int kernel;            // of q8_dense.hip's table
  DenseFamily family;
  int splits;            // workgroups that divide a tile's sum; from two on a second launch joins the parts
  long long workgroups;  // of all launches
  int tokens;            // of a launch, whole tiles; all of them but for batches beyond the threads of one launch
  int lds;               // bytes per workgroup
};
// The kernel for a call on a device of that many compute units; pure host arithmetic.
void plan_dense(const DenseArgs& a, int units, DensePlan* plan);
hipError_t launch_dense(const DenseArgs& a, const DensePlan& plan, hipStream_t st);

}  // namespace sgmv
