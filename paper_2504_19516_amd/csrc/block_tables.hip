// Block tables and places of a step's new rows, made on the GPU from the requests' lengths (Section 3.5.1's paged cache).
//
// Request i holds c_i tokens in ceil(c_i / 16) pages and gets a_i more. It needs ceil((c_i + a_i) / 16) - ceil(c_i / 16) pages, which
// come off the top of the stack of free pages in the requests' order; row start_i + t of the step (start: exclusive sum of a) is the
// request's token c_i + t, in page table[i][(c_i + t) / 16], slot (c_i + t) % 16.
//
// Bound by latency: a few KB in, 12 bytes a row out. One launch: every workgroup scans all lengths for itself (they are in L2; 4096
// requests are 32 KB) and then writes the rows that are its own, so nothing is handed from one workgroup to another. A step that cannot
// be had is known to every workgroup alike, before anything is written. 256 requests of one new token each take 3.6 us, 8393 rows of 208
// requests 7.2 (0.1 MB; the scan and, row by row, a binary search in LDS).
#include "device_ops.h"

namespace sts {
namespace {

constexpr int BT_THREADS = 256, BT_ROWS = 1024;       // rows of a workgroup

__device__ __forceinline__ int pages_of(int tokens) { return (int)(((unsigned)tokens + OP_PAGE - 1) / OP_PAGE); }

// Exclusive sum of v over the workgroup's threads, and the total.
__device__ __forceinline__ long long block_scan(long long v, long long* waves, long long* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) waves[wave] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < BT_THREADS / 64; w++) {
    if (w < wave) before += waves[w];
    all += waves[w];
  }
  __syncthreads();
  *total = all;
  return before + x - v;
}

__global__ void __launch_bounds__(BT_THREADS) block_tables_kernel(sts_block_tables a) {
  extern __shared__ int lds[];
  __shared__ long long waves[BT_THREADS / 64];
  __shared__ int flags;                                // 1: a length out of range, 2: a table row too short
  const int n = a.n_requests, tid = threadIdx.x;
  int *start = lds, *first = lds + n, *cached = lds + 2 * n;      // rows and pages taken before request i, its cached tokens
  if (tid == 0) flags = 0;
  __syncthreads();
  int mine = 0;
  for (int i = tid; i < n; i += BT_THREADS) {
    const int c = a.cached[i], add = a.added[i];
    const bool bad = c < 0 || add < 0 || c > 0x7FFFFFFF - OP_PAGE - add;
    if (bad) mine |= 1;
    else if (add > 0 && pages_of(c + add) > a.max_pages) mine |= 2;
    cached[i] = c;
    start[i] = bad ? 0 : add;
    first[i] = bad ? 0 : pages_of(c + add) - pages_of(c);
  }
  if (mine) atomicOr(&flags, mine);
  __syncthreads();
  // a thread's contiguous share of the requests, then the shares
  const int per = (n + BT_THREADS - 1) / BT_THREADS, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  long long rows = 0, pages = 0, all_rows, all_pages;
  for (int i = i0; i < i1; i++) { rows += start[i]; pages += first[i]; }
  rows = block_scan(rows, waves, &all_rows);
  pages = block_scan(pages, waves, &all_pages);
  const int n_free = *a.n_free;
  int status = STS_OK;
  if ((flags & 1) || n_free < 0 || n_free > a.free_capacity) status = STS_EINVAL;
  else if ((flags & 2) || all_pages > n_free || all_rows > a.max_rows) status = STS_ENOMEM;
  for (int i = i0; i < i1; i++) {
    const int r = start[i], p = first[i];
    start[i] = (int)rows; first[i] = (int)pages;
    rows += r; pages += p;
    if (blockIdx.x == 0) {
      a.row_starts[i] = status ? 0 : start[i];
      a.lens[i] = status ? cached[i] : cached[i] + r;
    }
  }
  __syncthreads();
  const int total = status ? 0 : (int)all_rows;
  if (blockIdx.x == 0 && tid == 0) {
    a.row_starts[n] = total;
    *a.n_free_left = status ? n_free : n_free - (int)all_pages;
    *a.status = status;
  }
  const int top = n_free - (int)all_pages, end = min(a.max_rows, ((int)blockIdx.x + 1) * BT_ROWS);
  for (int row = blockIdx.x * BT_ROWS + tid; row < end; row += BT_THREADS) {
    if (row >= total) { a.places[row] = -1; continue; }
    int lo = 0, hi = n;                                // the last request that starts at or before the row
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= row) lo = mid; else hi = mid;
    }
    const int c = cached[lo], pos = c + row - start[lo], at = pos / OP_PAGE, held = pages_of(c);
    int* entry = a.tables + (long long)lo * a.table_stride + at;
    int page;
    if (at < held) page = *entry;
    else {
      page = a.free_pages[top + first[lo] + at - held];
      if (pos % OP_PAGE == 0) *entry = page;           // every new page begins with a new row
    }
    a.requests[row] = lo;
    a.positions[row] = pos;
    a.places[row] = (unsigned)page < 0x7FFFFFFFu / OP_PAGE ? page * OP_PAGE + pos % OP_PAGE : -1;
  }
}

}  // namespace
}  // namespace sts

using namespace sts;

extern "C" int sts_op_block_tables(const sts_block_tables* a, void* stream) {
  if (!a || a->n_requests < 0 || a->n_requests > OP_MAX_REQUESTS || a->max_pages < 0 || a->max_rows < 0 || a->max_rows > (1 << 30) || a->free_capacity < 0 || a->table_stride < a->max_pages) return STS_EINVAL;
  if (!a->n_free || !a->n_free_left || !a->status || !a->row_starts) return STS_EINVAL;
  if (a->n_requests > 0 && (!a->cached || !a->added || !a->lens || (a->max_pages > 0 && !a->tables))) return STS_EINVAL;
  if (a->max_rows > 0 && (!a->requests || !a->positions || !a->places)) return STS_EINVAL;
  if (a->free_capacity > 0 && !a->free_pages) return STS_EINVAL;
  if (a->n_free_left == a->n_free || a->lens == a->cached || a->lens == a->added) return STS_EINVAL;      // read by workgroups that start late
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  const unsigned grid = a->max_rows <= BT_ROWS ? 1 : (a->max_rows + (unsigned)BT_ROWS - 1) / BT_ROWS;
  return op_result(launch(block_tables_kernel, dim3(grid), dim3(BT_THREADS), (size_t)a->n_requests * 3 * sizeof(int), s, *a));
}
