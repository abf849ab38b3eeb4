// Pages, block tables, slots and positions of a step from the requests' lengths (gfx950).
//
//   held_i = ceil(old_i / P);  a request that is over pushes its held_i pages, in the requests' order;  then request i pops
//   need_i = ceil((old_i + new_i) / P) - held_i pages off the top;  q_starts are the prefix sums of new
//   row t of request i:  position old_i + t - q_starts_i,  slot = page * P + position % P
//
// One workgroup takes the requests 1024 at a time: totals first, as a step is refused as a whole, then prefix sums of rows, pushed
// and needed pages.  Its rows follow in the same launch, or in one of their own where there are many.
#include "device_common.h"
#include "kv.h"

#include "../../include/sgmv.h"

namespace sgmv {

namespace {

constexpr int kThreads = 1024;
// Rows that the first launch's one workgroup takes itself.
constexpr int kRowsOfOne = 4096;

struct Need {
  int rows, pushed, needed;
};

// A request's part of the step; `flags` gets what is wrong with it.
__device__ __forceinline__ Need need_of(const KvAssignArgs& a, int i, int& flags) {
  const int old = a.old_lens[i], fresh = a.new_lens[i];
  const long long most = (long long)a.table_width << a.page_shift;
  if (old < 0 || old > most || fresh < -1) {
    flags |= SGMV_KV_LENGTHS;
    return {0, 0, 0};
  }
  const int mask = (1 << a.page_shift) - 1;
  const int held = (int)(((long long)old + mask) >> a.page_shift);
  if (fresh < 0) return {0, held, 0};
  const long long len = (long long)old + fresh;
  if (len > most) {
    flags |= SGMV_KV_TABLE;
    return {0, 0, 0};
  }
  return {fresh, 0, (int)((len + mask) >> a.page_shift) - held};
}

// Sum over the workgroup, in every thread; `of_waves` has a place per wave.
__device__ __forceinline__ long long total_of(long long v, long long* of_waves) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) of_waves[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < kThreads / 64; ++w) v += of_waves[w];
  return v;
}

// Sum over the threads before this one; `total` gets all of it.
__device__ __forceinline__ int before_of(int v, int* of_waves, int& total) {
  const int lane = threadIdx.x & 63;
  int sum = v;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int o = __shfl_up(sum, m);
    if (lane >= m) sum += o;
  }
  __syncthreads();
  if (lane == 63) of_waves[threadIdx.x >> 6] = sum;
  __syncthreads();
  int front = 0;
  total = 0;
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < (int)(threadIdx.x >> 6)) front += of_waves[w];
    total += of_waves[w];
  }
  return front + sum - v;
}

// Slot and position of a row; q_starts, kv_lens and tables are this step's.
__device__ __forceinline__ void place_row(const KvAssignArgs& a, int t) {
  int slot = -1, pos = -1;
  if (t < a.q_starts[a.n_reqs]) {
    int low = 0, high = a.n_reqs - 1;  // the first request that ends behind t
    while (low < high) {
      const int mid = (low + high) >> 1;
      if (a.q_starts[mid + 1] > t)
        high = mid;
      else
        low = mid + 1;
    }
    pos = a.kv_lens[low] - (a.q_starts[low + 1] - t);
    const int page = a.tables[(size_t)low * a.table_width + (pos >> a.page_shift)];
    if (page >= 0 && page < a.n_pages)
      slot = (page << a.page_shift) | (pos & ((1 << a.page_shift) - 1));
    else
      atomicOr(a.status, SGMV_KV_PAGE), atomicOr(a.status + 1, SGMV_KV_PAGE);
  }
  a.slots[t] = slot;
  a.positions[t] = pos;
}

// write(request, column + j, place, j), j < n, for every lane's request: a few by the lane itself, many by the whole wave.
template <class F>
__device__ __forceinline__ void for_each_of(int n, int request, int column, int place, F write) {
  if (n <= 4)
    for (int j = 0; j < n; ++j) write(request, column + j, place, j);
  for (unsigned long long many = __ballot(n > 4); many != 0; many &= many - 1) {
    const int from = __builtin_ctzll(many);
    const int count = __shfl(n, from), r = __shfl(request, from), c = __shfl(column, from), at = __shfl(place, from);
    for (int j = threadIdx.x & 63; j < count; j += 64) write(r, c + j, at, j);
  }
}

__global__ __launch_bounds__(kThreads) void kv_assign_kernel(KvAssignArgs a, int own_rows) {
  __shared__ long long sums[kThreads / 64];
  __shared__ int parts[3][kThreads / 64];
  const int tid = threadIdx.x;
  long long rows = 0, pushed = 0, needed = 0;
  int flags = 0;
  for (int i = tid; i < a.n_reqs; i += kThreads) {
    const Need n = need_of(a, i, flags);
    rows += n.rows, pushed += n.pushed, needed += n.needed;
  }
  const int free_count = *a.free_count;
  rows = total_of(rows, sums), pushed = total_of(pushed, sums), needed = total_of(needed, sums);
  if (free_count < 0 || free_count + pushed > a.n_pages)
    flags |= SGMV_KV_LENGTHS;
  else if (needed > free_count + pushed)
    flags |= SGMV_KV_NO_PAGES;
  if (rows > a.n_tokens) flags |= SGMV_KV_ROWS;
  int all = 0;
  for (int bit = 1; bit <= SGMV_KV_LENGTHS; bit <<= 1)
    if (__syncthreads_or(flags & bit)) all |= bit;
  if (tid == 0) {
    a.status[0] = all;
    a.status[1] |= all;
    *a.free_count_out = all ? free_count : free_count + (int)(pushed - needed);
    a.q_starts[0] = 0;
  }
  if (all) {
    for (int i = tid; i < a.n_reqs; i += kThreads) {
      a.kv_lens[i] = a.old_lens[i];
      a.q_starts[i + 1] = 0;
    }
    for (int t = tid; t < own_rows; t += kThreads) a.slots[t] = a.positions[t] = -1;
    return;
  }
  if (pushed > 0) {
    int at = free_count;
    for (int base = 0; base < a.n_reqs; base += kThreads) {
      const int i = base + tid;
      const int n = i < a.n_reqs ? need_of(a, i, flags).pushed : 0;
      int total;
      const int to = at + before_of(n, parts[0], total);
      for_each_of(n, i, 0, to, [&](int r, int column, int place, int j) {
        a.free_pages[place + j] = a.tables[(size_t)r * a.table_width + column];
      });
      at += total;
    }
    __syncthreads();
  }
  int row = 0, top = free_count + (int)pushed;
  for (int base = 0; base < a.n_reqs; base += kThreads) {
    const int i = base + tid;
    const Need n = i < a.n_reqs ? need_of(a, i, flags) : Need{0, 0, 0};
    int total_rows, total_pages;
    const int start = row + before_of(n.rows, parts[1], total_rows);
    const int from = top - 1 - before_of(n.needed, parts[2], total_pages);
    int len = 0;
    if (i < a.n_reqs) {
      const int old = a.old_lens[i];
      len = a.new_lens[i] < 0 ? 0 : old + n.rows;
      a.q_starts[i + 1] = start + n.rows;
      a.kv_lens[i] = len;
    }
    // the request's last pages, from the first new one on
    const int mask = (1 << a.page_shift) - 1, held = ((len + mask) >> a.page_shift) - n.needed;
    for_each_of(n.needed, i, held, from, [&](int r, int column, int place, int j) {
      a.tables[(size_t)r * a.table_width + column] = a.free_pages[place - j];
    });
    row += total_rows;
    top -= total_pages;
  }
  __syncthreads();
  for (int t = tid; t < own_rows; t += kThreads) place_row(a, t);
}

__global__ __launch_bounds__(256) void kv_rows_kernel(KvAssignArgs a) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t < a.n_tokens) place_row(a, t);
}

}  // namespace

hipError_t launch_kv_assign(const KvAssignArgs& a, hipStream_t st) {
  const int own_rows = a.n_tokens <= kRowsOfOne ? a.n_tokens : 0;
  kv_assign_kernel<<<1, kThreads, 0, st>>>(a, own_rows);
  hipError_t err = hipGetLastError();
  if (err == hipSuccess && own_rows < a.n_tokens) {
    kv_rows_kernel<<<(unsigned)((a.n_tokens + 255LL) / 256), 256, 0, st>>>(a);
    err = hipGetLastError();
  }
  return err;
}

}  // namespace sgmv
