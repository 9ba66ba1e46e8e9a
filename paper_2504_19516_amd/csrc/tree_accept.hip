// What a verified tree of drafted tokens leaves: the path that the target agrees with, and its K and V rows where the next step expects them.
//
// Path: node 0, then the first child of the last node whose token is the target's choice behind that node. A wave keeps a request's nodes in registers, four a
// lane; a step of the path is a comparison and a ballot.
//
// Rows: the path's j-th node n_j lies at token cached + n_j and goes to cached + j, in all layers. n_j >= j and n_j ascend, so a row's new place is read by
// nobody after it; a wave (one head of one request in one layer) takes the rows in order, four at a time, all loaded before any is stored. K rows move 16 bytes a lane, V^T
// columns an element a lane, since a page's 16 tokens lie side by side.
//
// Pages behind the path go back onto the stack of free ones, in the requests' order: one workgroup, a scan of their numbers.
//
// Bound by latency: lengths, path, table, rows, one behind the other: one request's 32 layers 4 us, its path 2.4. Many requests are bound by the V columns: a column of 128 elements
// is a store of two bytes into each of 128 sectors of a page (64 requests, 8 layers, two rows each: 12.8 us for 8 MB of rows, whose columns reach into pages of up to 72 MB, read and written).
#include "device_ops.h"

namespace sts {
namespace {

constexpr int TA_NODES = 256, TA_LAYERS = 256, TA_THREADS = 256;
constexpr int TA_ROWS = 4;                             // rows of a wave under way

// Rows of a request; none where row_starts is out of range.
__device__ __forceinline__ int nodes_of(const int* row_starts, int request, int max_rows, int* first) {
  *first = row_starts[request];
  const int end = row_starts[request + 1];
  return *first < 0 || end < *first || end > max_rows ? 0 : end - *first;
}

__global__ void __launch_bounds__(256) tree_accept_kernel(sts_tree_accept a) {
  const int request = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (request >= a.n_requests) return;
  int first;
  const int nodes = nodes_of(a.row_starts, request, a.max_rows, &first);
  constexpr int PER = TA_NODES / 64;
  int parent[PER], token[PER], chosen[PER];
#pragma unroll
  for (int u = 0; u < PER; u++) {
    const int j = u * 64 + lane;
    const bool here = j < nodes;
    parent[u] = here ? a.parents[first + j] : -2;
    token[u] = here ? a.tokens[first + j] : 0;
    chosen[u] = here ? a.chosen[first + j] : 0;
  }
  int count = 0, next = -1;
  if (nodes > 0 && nodes <= TA_NODES && __builtin_amdgcn_readfirstlane(parent[0]) == -1) {
    for (int at = 0; at >= 0;) {                       // ascends
      if (lane == 0) a.path[first + count] = at;
      count++;
      next = 0;
#pragma unroll
      for (int u = 0; u < PER; u++)
        if (at >> 6 == u) next = __builtin_amdgcn_readlane(chosen[u], at & 63);
      int child = -1;
#pragma unroll
      for (int u = PER - 1; u >= 0; u--) {
        const unsigned long long fit = __ballot(parent[u] == at && token[u] == next && u * 64 + lane > at && u * 64 + lane < nodes);
        if (fit) child = u * 64 + __builtin_ctzll(fit);
      }
      at = child;
    }
  }
  for (int j = count + lane; j < nodes; j += 64) a.path[first + j] = -1;
  if (lane == 0) {
    a.counts[request] = count;
    a.lens[request] = (int)((unsigned)a.cached[request] + (unsigned)count);
    a.next_token[request] = next;
  }
}

// Pages behind the paths, back onto the stack of free ones. One workgroup: a thread has neighbouring requests.
__global__ void __launch_bounds__(TA_THREADS) tree_release_kernel(sts_tree_accept a) {
  __shared__ long long waves[TA_THREADS / 64];         // row_starts out of order may name a row in many requests: sums of 64 bits
  const int n = a.n_requests, tid = threadIdx.x, per = (n + TA_THREADS - 1) / TA_THREADS, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  auto pages_of = [](int tokens) { return (tokens + OP_PAGE - 1) / OP_PAGE; };
  // of a request: the first page behind its path, and how many the nodes' rows had
  auto behind = [&](int i, int* page) {
    int first;
    // lens may have taken the place of cached by now
    const int nodes = nodes_of(a.row_starts, i, a.max_rows, &first), count = a.counts[i], c = (int)((unsigned)a.lens[i] - (unsigned)count);
    *page = 0;
    if (c < 0 || c > a.max_pages * (long long)OP_PAGE - nodes) return 0;
    *page = pages_of(c + count);
    return pages_of(c + nodes) - *page;
  };
  long long sum = 0;
  int page;
  for (int i = i0; i < i1; i++) sum += behind(i, &page);
  long long x = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long y = __shfl_up(x, o, 64);
    if ((tid & 63) >= o) x += y;
  }
  if ((tid & 63) == 63) waves[tid >> 6] = x;
  const int free = *a.n_free;
  __syncthreads();
  long long at = x - sum, total = 0;
#pragma unroll
  for (int w = 0; w < TA_THREADS / 64; w++) {
    if (w < tid >> 6) at += waves[w];
    total += waves[w];
  }
  if (free < 0 || free > a.free_capacity - total) return;
  for (int i = i0; i < i1; i++) {
    const int m = behind(i, &page);
    for (int e = 0; e < m; e++) a.free_pages[free + at++] = a.tables[i * a.table_stride + page + e];
  }
  if (tid == 0) *a.n_free = free + (int)total;
}

struct CompactCall { sts_tree_compact a; void* pools[TA_LAYERS]; };

template <int D>
__global__ void __launch_bounds__(256) tree_compact_kernel(CompactCall c) {
  const sts_tree_compact& a = c.a;
  const int at = blockIdx.x * 4 + (threadIdx.x >> 6), request = at / a.n_kv, head = at % a.n_kv, lane = threadIdx.x & 63;
  if (request >= a.n_requests) return;
  int first;
  const int nodes = nodes_of(a.row_starts, request, a.max_rows, &first), count = min(a.counts[request], min(nodes, TA_NODES));
  const long long cached = a.cached[request];
  if (cached < 0) return;
  const int* table = a.tables + request * a.table_stride;
  auto place = [&](int node) {                         // page * 16 + slot, -1: not in the pool
    if (node < 0 || node >= nodes || (cached + node) / OP_PAGE >= a.max_pages) return -1ll;
    const int page = table[(cached + node) / OP_PAGE];
    return (unsigned)page < (unsigned)a.pool_pages ? page * (long long)OP_PAGE + (cached + node) % OP_PAGE : -1ll;
  };
  typedef unsigned short u16;
  u16* pool = reinterpret_cast<u16*>(c.pools[blockIdx.y]);
  auto rows = [&](long long p) { return pool + ((p / OP_PAGE) * a.n_kv + head) * (2 * OP_PAGE * D); };
  constexpr int CPR = D / 8, VPL = D / 64;             // 16-byte chunks of a K row; elements of a V column a lane
  for (int j0 = 0; j0 < count; j0 += 64) {             // 64 rows' places, one a lane
    const int j = j0 + lane, node = j < count ? a.path[first + j] : -1;
    const long long dst = place(j), src = place(node);              // on the way together
    const bool moves = node > j && src >= 0 && dst >= 0;
    unsigned long long left = __ballot(moves);
    while (left) {                                     // the next rows that move, four at most
      u32x4 k[TA_ROWS];
      u16 v[TA_ROWS][VPL];
      long long to[TA_ROWS];
      int n = 0;
#pragma unroll
      for (int i = 0; i < TA_ROWS; i++) {
        if (!left) break;
        const int l = __builtin_ctzll(left);
        left &= left - 1;
        const long long p = __shfl(src, l, 64);
        to[i] = __shfl(dst, l, 64);
        const u16* from = rows(p);
        if (lane < CPR) k[i] = *reinterpret_cast<const u32x4*>(from + p % OP_PAGE * D + lane * 8);
#pragma unroll
        for (int e = 0; e < VPL; e++) v[i][e] = from[OP_PAGE * D + (e * 64 + lane) * OP_PAGE + p % OP_PAGE];
        n++;
      }
      wait_vmem<0>();                                  // all are in registers before the first is stored
      __asm__ volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < TA_ROWS; i++) {
        if (i >= n) break;
        u16* there = rows(to[i]);
        if (lane < CPR) *reinterpret_cast<u32x4*>(there + to[i] % OP_PAGE * D + lane * 8) = k[i];
#pragma unroll
        for (int e = 0; e < VPL; e++) there[OP_PAGE * D + (e * 64 + lane) * OP_PAGE + to[i] % OP_PAGE] = v[i][e];
      }
    }
  }
}

}  // namespace
}  // namespace sts

using namespace sts;

extern "C" int sts_op_tree_accept(const sts_tree_accept* a, void* stream) {
  // rows as sts_op_block_tables makes them: a wave's steps over a request's path stay within 32 bits
  if (!a || a->n_requests < 0 || a->n_requests > OP_MAX_REQUESTS || a->max_rows < 0 || a->max_rows > (1 << 30)) return STS_EINVAL;
  if (a->n_requests == 0) return STS_OK;
  if (!a->cached || !a->row_starts || !a->lens || !a->counts || !a->next_token) return STS_EINVAL;
  if (a->max_rows > 0 && (!a->parents || !a->tokens || !a->chosen || !a->path)) return STS_EINVAL;
  if (a->tables && (!a->free_pages || !a->n_free || a->max_pages < 0 || a->max_pages > (1 << 26) || a->free_capacity < 0 || a->table_stride < a->max_pages)) return STS_EINVAL;
  // What is written is read by other waves or by the second kernel: arrays of their own, but for lens in place of cached, and a path in place of the rows that its own wave has read.
  const bool rows = a->max_rows > 0, pages = a->tables != nullptr;
  const void* written[] = {a->lens, a->counts, a->next_token, rows ? a->path : nullptr, pages ? a->free_pages : nullptr, pages ? a->n_free : nullptr};
  const void* read[] = {a->row_starts, a->cached, a->tables, rows ? a->parents : nullptr, rows ? a->tokens : nullptr, rows ? a->chosen : nullptr};
  for (int i = 0; i < 6; i++)
    for (int j = 0; j < 6 && written[i]; j++) {
      if (j > i && written[i] == written[j]) return STS_EINVAL;
      if (written[i] == read[j] && !(i == 0 && j == 1) && !(i == 3 && j >= 3)) return STS_EINVAL;
    }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  hipError_t e = launch(tree_accept_kernel, dim3((a->n_requests + 3) / 4), dim3(256), 0, s, *a);
  if (e == hipSuccess && a->tables) e = launch(tree_release_kernel, dim3(1), dim3(TA_THREADS), 0, s, *a);
  return op_result(e);
}

extern "C" int sts_op_tree_compact(const sts_tree_compact* a, void* const* pools, int32_t n_layers, void* stream) {
  if (!a || a->n_requests < 0 || a->n_requests > OP_MAX_REQUESTS || a->max_rows < 0 || a->n_kv < 1 || a->n_kv > 256 || (a->d != 64 && a->d != 128) || a->pool_pages < 0 || a->max_pages < 0 ||
      a->max_pages > (1 << 26) || a->table_stride < a->max_pages || n_layers < 0 || n_layers > TA_LAYERS) return STS_EINVAL;
  if (a->n_requests == 0 || a->max_rows == 0 || n_layers == 0) return STS_OK;
  if (!a->cached || !a->row_starts || !a->counts || !a->path || (a->max_pages > 0 && !a->tables) || !pools) return STS_EINVAL;
  CompactCall c{};
  c.a = *a;
  for (int i = 0; i < n_layers; i++) {
    if (!pools[i] || !aligned(pools[i], 16)) return STS_EINVAL;
    c.pools[i] = pools[i];
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  const dim3 grid((unsigned)(((int64_t)a->n_requests * a->n_kv + 3) / 4), (unsigned)n_layers);
  return op_result(a->d == 128 ? launch(tree_compact_kernel<128>, grid, dim3(256), 0, s, c) : launch(tree_compact_kernel<64>, grid, dim3(256), 0, s, c));
}
