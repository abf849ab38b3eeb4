// Pages, block tables, slots and positions of a step from the requests' lengths (gfx950).
//
//   held_i = ceil(old_i / P);  a request that is over pushes its held_i pages, in the requests' order;  then request i pops
//   need_i = ceil((old_i + new_i) / P) - held_i pages off the top;  q_starts are the prefix sums of new
//   row t of request i:  position old_i + t - q_starts_i,  slot = page * P + position % P
//
// One workgroup.  A step is refused as a whole, so totals come first, then prefix sums of rows, pushed and needed pages; up to 4096 requests get
// both from one scan and one barrier (more go through it in turns).  The prefix sums stay in LDS, and every pushed page, needed page and
// row finds its request there by bisection: a thread each, whether one request has them all or every one has one.  Sums saturate:
// lengths may be anything.
//
// Bound by two round trips to memory behind one another (lengths, then table and stack) and the bisections in LDS: 64 requests with a row each and three
// that are over 4.6 us, 1060 requests with 23 000 rows, 7600 pages pushed 13.8 us and 4.8 for the rows (17 and 35 where waves went through requests one
// after the other, with and without a launch for the rows).
#include "device_common.h"
#include "kv.h"

#include "../../include/sgmv.h"

namespace sgmv {

namespace {

constexpr int kThreads = 1024;
// Rows that the first launch's one workgroup writes itself.
constexpr int kRowsOfOne = 4096;

struct Need {
  uint32_t rows, pushed, needed;
};

// A request's part of the step; `flags` gets what is wrong with it.
__device__ __forceinline__ Need need_of(const KvAssignArgs& a, int i, int& flags, int& old) {
  old = a.old_lens[i];
  const int fresh = a.new_lens[i];
  const long long most = (long long)a.table_width << a.page_shift;
  if (old < 0 || old > most || fresh < -1) {
    flags |= SGMV_KV_LENGTHS;
    return {0, 0, 0};
  }
  const int mask = (1 << a.page_shift) - 1;
  const int held = (int)(((long long)old + mask) >> a.page_shift);
  if (fresh < 0) return {0, (uint32_t)held, 0};
  const long long len = (long long)old + fresh;
  if (len > most) {
    flags |= SGMV_KV_TABLE;
    return {0, 0, 0};
  }
  return {(uint32_t)fresh, 0, (uint32_t)((len + mask) >> a.page_shift) - (uint32_t)held};
}

__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Sums over a wave's lanes up to this one.
__device__ __forceinline__ uint32_t scan_wave(uint32_t v) {
  auto from = [](uint32_t x, auto ctrl, auto rows) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xF, false); };
  using all = std::integral_constant<int, 0xF>;
  v = plus(v, from(v, std::integral_constant<int, 0x111>{}, all{}));  // one, two, four and eight lanes down in a row of sixteen
  v = plus(v, from(v, std::integral_constant<int, 0x112>{}, all{}));
  v = plus(v, from(v, std::integral_constant<int, 0x114>{}, all{}));
  v = plus(v, from(v, std::integral_constant<int, 0x118>{}, all{}));
  v = plus(v, from(v, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{}));  // rows 0 and 2 into 1 and 3
  return plus(v, from(v, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{}));  // the lower half into the upper one
}

// The prefix sums of a turn's requests, and their positions so far.
template <int ITEMS>
struct Turn {
  static constexpr int kMost = kThreads * ITEMS;
  uint32_t rows[kMost + 1], pushed[kMost + 1], needed[kMost + 1];
  int old[kMost];
  Need waves[kThreads / 64];
  int wave_flags[kThreads / 64];
};

// The last of `n` prefix sums that is not above j: the request that j belongs to.
__device__ __forceinline__ int owner_of(const uint32_t* sums, int n, uint32_t j) {
  int low = 0, high = n - 1;
  while (low < high) {
    const int mid = (low + high + 1) >> 1;
    if (sums[mid] <= j)
      low = mid;
    else
      high = mid - 1;
  }
  return low;
}

// Requests base .. base + count - 1 into LDS, ITEMS to a thread; their totals, and what is wrong with any of them.
template <int ITEMS>
__device__ __forceinline__ Need scan_turn(const KvAssignArgs& a, int base, int count, bool again, Turn<ITEMS>& turn, int& flags) {
  const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, first = threadIdx.x * ITEMS;
  Need n[ITEMS], mine = {0, 0, 0};
  int old[ITEMS], wrong = 0;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    n[k] = {0, 0, 0};
    old[k] = 0;
    if (first + k < count) n[k] = need_of(a, base + first + k, wrong, old[k]);
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) mine = {plus(mine.rows, n[k].rows), plus(mine.pushed, n[k].pushed), plus(mine.needed, n[k].needed)};
  const Need to = {scan_wave(mine.rows), scan_wave(mine.pushed), scan_wave(mine.needed)};
  wrong = (__any(wrong & SGMV_KV_LENGTHS) ? SGMV_KV_LENGTHS : 0) | (__any(wrong & SGMV_KV_TABLE) ? SGMV_KV_TABLE : 0);
  if (base > 0 || again) __syncthreads();  // the turn before is done with the arrays
  if ((threadIdx.x & 63) == 63) {
    turn.waves[wave] = to;
    turn.wave_flags[wave] = wrong;
  }
  __syncthreads();
  Need before = {to.rows - mine.rows, to.pushed - mine.pushed, to.needed - mine.needed}, total = {0, 0, 0};
  for (int w = 0; w < waves; ++w) {
    const Need x = turn.waves[w];
    if (w < wave) before = {plus(before.rows, x.rows), plus(before.pushed, x.pushed), plus(before.needed, x.needed)};
    total = {plus(total.rows, x.rows), plus(total.pushed, x.pushed), plus(total.needed, x.needed)};
    flags |= turn.wave_flags[w];
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    if (first + k < count) {
      turn.rows[first + k] = before.rows;
      turn.pushed[first + k] = before.pushed;
      turn.needed[first + k] = before.needed;
      turn.old[first + k] = old[k];
    }
    before = {plus(before.rows, n[k].rows), plus(before.pushed, n[k].pushed), plus(before.needed, n[k].needed)};
    if (first + k == count - 1) turn.rows[count] = before.rows, turn.pushed[count] = before.pushed, turn.needed[count] = before.needed;
  }
  return total;
}

__device__ __forceinline__ void put_row(const KvAssignArgs& a, int t, int pos, int page) {
  int slot = -1;
  if (page >= 0 && page < a.n_pages)
    slot = (page << a.page_shift) | (pos & ((1 << a.page_shift) - 1));
  else
    atomicOr(a.status, SGMV_KV_PAGE), atomicOr(a.status + 1, SGMV_KV_PAGE);
  a.slots[t] = slot;
  a.positions[t] = pos;
}

// own_rows: rows of the batch that this launch writes, all or none.
template <int ITEMS>
__global__ __launch_bounds__(kThreads) void kv_assign_kernel(KvAssignArgs a, int own_rows) {
  __shared__ Turn<ITEMS> turn;
  const int tid = threadIdx.x, threads = blockDim.x, at_once = threads * ITEMS, free_count = *a.free_count, seen = a.status[1];
  int wrong = 0;
  Need total = {0, 0, 0};
  for (int base = 0; base < a.n_reqs; base += at_once) {
    const Need x = scan_turn<ITEMS>(a, base, min(at_once, a.n_reqs - base), false, turn, wrong);
    total = {plus(total.rows, x.rows), plus(total.pushed, x.pushed), plus(total.needed, x.needed)};
  }
  const long long stacked = (long long)free_count + total.pushed;
  if (free_count < 0 || stacked > a.n_pages)
    wrong |= SGMV_KV_LENGTHS;
  else if (total.needed > stacked)
    wrong |= SGMV_KV_NO_PAGES;
  if (total.rows > (uint32_t)a.n_tokens) wrong |= SGMV_KV_ROWS;
  if (tid == 0) {
    a.status[0] = wrong;
    a.status[1] = seen | wrong;
    *a.free_count_out = wrong ? free_count : (int)(stacked - total.needed);
    a.q_starts[0] = 0;
  }
  if (wrong) {
    for (int i = tid; i < a.n_reqs; i += threads) {
      a.kv_lens[i] = a.old_lens[i];
      a.q_starts[i + 1] = 0;
    }
    for (int t = tid; t < own_rows; t += threads) a.slots[t] = a.positions[t] = -1;
    return;
  }
  for (int t = (int)total.rows + tid; t < own_rows; t += threads) a.slots[t] = a.positions[t] = -1;
  const bool turns = a.n_reqs > at_once;
  __syncthreads();
  if (total.pushed > 0) {
    int to = free_count;
    for (int base = 0; base < a.n_reqs; base += at_once) {
      const int count = min(at_once, a.n_reqs - base);
      if (turns) {
        scan_turn<ITEMS>(a, base, count, true, turn, wrong);
        __syncthreads();
      }
      const uint32_t pushed = turn.pushed[count];
      for (uint32_t j = tid; j < pushed; j += threads) {
        const int r = owner_of(turn.pushed, count, j);
        a.free_pages[to + (int)j] = a.tables[(size_t)(base + r) * a.table_width + (j - turn.pushed[r])];
      }
      to += (int)pushed;
    }
    __syncthreads();
  }
  const int mask = (1 << a.page_shift) - 1;
  int row = 0, top = (int)stacked - 1;
  for (int base = 0; base < a.n_reqs; base += at_once) {
    const int count = min(at_once, a.n_reqs - base);
    if (turns) {
      scan_turn<ITEMS>(a, base, count, true, turn, wrong);
      __syncthreads();
    }
    const uint32_t rows = turn.rows[count], needed = turn.needed[count];
    for (uint32_t j = tid; j < needed; j += threads) {
      const int r = owner_of(turn.needed, count, j), held = (turn.old[r] + mask) >> a.page_shift;
      a.tables[(size_t)(base + r) * a.table_width + held + (j - turn.needed[r])] = a.free_pages[top - (int)j];
    }
    for (int i = tid; i < count; i += threads) {
      const uint32_t fresh = turn.rows[i + 1] - turn.rows[i];
      a.q_starts[base + i + 1] = row + (int)turn.rows[i + 1];
      a.kv_lens[base + i] = turn.pushed[i + 1] != turn.pushed[i] ? 0 : turn.old[i] + (int)fresh;
    }
    if (own_rows > 0) {
      for (uint32_t t = tid; t < rows; t += threads) {
        const int r = owner_of(turn.rows, count, t), pos = turn.old[r] + (int)(t - turn.rows[r]), column = pos >> a.page_shift;
        const int held = (turn.old[r] + mask) >> a.page_shift;
        const int page = column < held ? a.tables[(size_t)(base + r) * a.table_width + column] : a.free_pages[top - (int)turn.needed[r] - (column - held)];
        put_row(a, row + (int)t, pos, page);
      }
    }
    row += (int)rows;
    top -= (int)needed;
  }
}

// The rows of a batch with many; q_starts, kv_lens and tables are this step's.
__global__ __launch_bounds__(256) void kv_rows_kernel(KvAssignArgs a) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= a.n_tokens) return;
  if (t >= a.q_starts[a.n_reqs]) {
    a.slots[t] = a.positions[t] = -1;
    return;
  }
  int low = 0, high = a.n_reqs - 1;  // the first request that ends behind t
  while (low < high) {
    const int mid = (low + high) >> 1;
    if (a.q_starts[mid + 1] > t)
      high = mid;
    else
      low = mid + 1;
  }
  const int pos = a.kv_lens[low] - (a.q_starts[low + 1] - t);
  put_row(a, t, pos, a.tables[(size_t)low * a.table_width + (pos >> a.page_shift)]);
}

}  // namespace

hipError_t launch_kv_assign(const KvAssignArgs& a, hipStream_t st) {
  // many rows: a launch of their own
  const int own_rows = a.n_tokens <= kRowsOfOne ? a.n_tokens : 0;
  const int most = a.n_reqs > own_rows ? a.n_reqs : own_rows, threads = most >= kThreads ? kThreads : (most + 63) / 64 * 64;
  if (a.n_reqs <= kThreads)
    kv_assign_kernel<1><<<1, threads, 0, st>>>(a, own_rows);
  else
    kv_assign_kernel<4><<<1, kThreads, 0, st>>>(a, own_rows);
  hipError_t err = hipGetLastError();
  if (err == hipSuccess && own_rows < a.n_tokens) {
    kv_rows_kernel<<<(unsigned)((a.n_tokens + 255LL) / 256), 256, 0, st>>>(a);
    err = hipGetLastError();
  }
  return err;
}

}  // namespace sgmv
