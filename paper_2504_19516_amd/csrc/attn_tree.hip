// Attention of drafted tokens over a paged cache: a request brings up to 256 nodes, each of which attends to the request's cached tokens, to its
// ancestors among the nodes, and to itself (a chain is the tree whose nodes have one child each).
//
//   o_i = sum_t p_t v_t / l,   p_t = 2^(scale log2(e) q_i . k_t - m),   l = sum_t p_t,   over t < c and t = c + j, j on the path to node i
//
// computed in parts of the token range, each with its own maximum m, that a second kernel joins:
//   m = max m_j,  l = sum l_j 2^(m_j - m),  o = sum o_j 2^(m_j - m) / l
//
// The rows of a KV head are a request's nodes times its query heads: they are cut into tiles of up to 128, and a tile over all the request's pages is a
// segment. Up to 32 rows (narrow) a wave takes pages by itself; beyond that (wide) the waves of a workgroup share the pages through LDS. A KV element read serves
// all rows of a tile, so few rows are bound by memory, and from some 230 rows (the card's operations a byte) the matrix cores are what bounds.
//
// The plan, made once a step on the device, does three things: it follows the parents up (each round doubles how far) and keeps for every node a bit
// for each token of the pages that hold nodes; it writes the nodes' positions; and it lays the segments of each kind end to end (pages, and the start and end of
// a segment counted as pages) and cuts each line into equal shares, one for each workgroup or wave. Piece p of segment s lies in share k: s + k is its number and
// (first row) + (rows of a share's tile) * k the place of its partial result, both without a further scan.
//
// Measured, 32 query and 8 KV heads of 128 in bf16, or 64 and 8 in fp16; us of the plan (once a step), and of products and join (each layer), medians under a trace:
//   one tree of 26 nodes on 1500 tokens, 6 MB of pages a layer     6   13   4    latency: table, pages, one to three tiles, partial results, one behind the other
//   64 chains of 5 on 1100 tokens (spread), 322 MB                 8   65   8    4.95 TB/s in the products: memory
//   16 trees of 64 on 4096 tokens (spread), 270 MB                10  143  15    0.48 PFLOP/s; without the trace 129, 0.53 and 0.8 with the second numbers': see run_wide
//   six trees of up to 33 on 14000 tokens, 64 heads, 238 MB        8   69  12    memory for the small trees (3.6 TB/s), matrix cores and exponentials for the large
#include <algorithm>

#include "attn_parts.h"

namespace sts {
namespace {

constexpr int AT_ROWS = 32;                     // rows of a narrow segment: columns of a product
constexpr int AT_TILE = 128;                    // rows of a wide one, at most
constexpr int AT_SLOTS = 512;                   // workgroups of a launch: two on each CU
constexpr int AT_NODES = 256;                   // of a request
constexpr int AT_MASK = 32;                     // 16-bit words of a row's mask, one for each page from the first that holds a node: up to 17 are used
constexpr int AT_MAX_ROWS = 1 << 16;
constexpr int AT_PLAN_THREADS = 512;
constexpr int AT_JOIN_ROWS = 1024;              // up to so many (row, head) pairs four waves join each, beyond it a run of lanes
constexpr int AT_JOIN_BATCH = 4;                // parts of a run under way
// Start and end of a wide and of a narrow segment, and the smallest shares beyond them, in pages; what a page of a wide segment takes a workgroup, in
// pages of a narrow one. Wide start and least share 8 and 4 / 4 and 4 / 6 and 2 / 4 and 2: one tree on 1500 tokens (four layers) 70 / - / 73 / 73 us, 16 trees (two) 287 / 288 / 287 / 287, six
// of the larger shape (two) 161 / 162 / 160 / 159. Narrow least share 4 / 12: a request of two nodes on 420 tokens 17 / 20. Wide weight 1.25 / 2: level.
constexpr int AT_WIDE_START = 8, AT_NARROW_START = 2, AT_WIDE_LEAST = 4, AT_NARROW_LEAST = 4;
constexpr float AT_WIDE_WEIGHT = 1.25f;
// Pages up to which segments are neither cut nor strung together where there is a workgroup or wave for each: none / 8 / 16, us: four trees of six nodes behind two tokens (64 heads, one layer)
// 26.7 / 18.2 / 18.2, 25 requests of two nodes on 76 tokens (two layers) 25.0 / 21.7 / 21.7, four chains of 16 on 129 (two) 37.2 / 37.6 / 33.2, one of 7 on 45 (two) 28.7 / 30.6 / 30.6.
constexpr int AT_APART = 16;

// A piece of a segment: rows row0 .. row0 + rows - 1 (node row * heads of a group + head) over the pages [pg0, pg1) of a request's table. part: number of its
// first row's partial result, -1: it finishes its rows.
struct Item { int row0, rows, request, pg0, pg1, part, cached, len; };
// Items of a wave: the first, and next .. end - 1; none if its rows are 0. The four of a workgroup with wide ones (whose last tile may have few rows) have the same.
struct Range { Item first; int next, end, wide, pad; };
// Where a node row's partial results are: head h of a group in base + h + j * step, j < count. One: its one piece finishes it. count -1: gives NaN.
struct Parts { int base, count, step, pad; };
struct Header {
  unsigned long long tag;                        // sizes_tag() of the batch that the plan was made for
  int rows;                                      // node rows; -1: row_starts out of order
  int pad;
};
struct Plan {
  Header* header;
  Range* ranges;                                 // [slots][4]
  Item* items;
  Parts* parts;                                  // [max_rows]
  int* nodes;                                    // [max_rows]: 0: the row is no node
  unsigned short* masks;                         // [max_rows][AT_MASK]: a bit for each token of a page
  f32x2* stats;                                  // [partial row][kv head]: maximum (log2 units), sum
  float* outs;                                   // [partial row][kv head][d]
};

int slots_of(int n_kv) { return std::max(1, AT_SLOTS / n_kv); }
// tiles: of whole nodes, and for each request one that is not full
int64_t max_segments(int n, int max_rows, int heads) { return (int64_t)max_rows / (AT_TILE / heads) + n; }
int64_t max_items(int n, int max_rows, int n_q, int n_kv) { return max_segments(n, max_rows, n_q / n_kv) + 4 * slots_of(n_kv); }
int64_t max_part_rows(int max_rows, int n_q, int n_kv) { return (int64_t)2 * max_rows * (n_q / n_kv) + (int64_t)slots_of(n_kv) * AT_TILE; }

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
// The workspace's parts behind each other; returns its size.
size_t lay_out(unsigned char* base, int n, int max_rows, int n_q, int n_kv, int d, Plan* p) {
  size_t at = 0;
  auto take = [&](size_t bytes) { unsigned char* q = base + at; at += up256(bytes); return q; };
  const size_t rows = (size_t)max_part_rows(max_rows, n_q, n_kv) * n_kv;
  Plan q;
  q.header = reinterpret_cast<Header*>(take(sizeof(Header)));
  q.ranges = reinterpret_cast<Range*>(take(slots_of(n_kv) * 4 * sizeof(Range)));
  q.items = reinterpret_cast<Item*>(take(max_items(n, max_rows, n_q, n_kv) * sizeof(Item)));
  q.parts = reinterpret_cast<Parts*>(take(max_rows * sizeof(Parts)));
  q.nodes = reinterpret_cast<int*>(take(max_rows * sizeof(int)));
  q.masks = reinterpret_cast<unsigned short*>(take((size_t)max_rows * AT_MASK * sizeof(unsigned short)));
  q.stats = reinterpret_cast<f32x2*>(take(rows * sizeof(f32x2)));
  q.outs = reinterpret_cast<float*>(take(rows * d * sizeof(float)));
  if (p) *p = q;
  return at;
}

// The sizes on which the indexes of a plan's users depend, never 0. A workspace without a plan of the batch's sizes gives NaN: nothing in it is followed.
unsigned long long sizes_tag(const sts_tree_batch& b) {
  unsigned long long t = 2;
  for (int32_t x : {b.n_requests, b.max_rows, b.n_q, b.n_kv, b.d, b.max_pages}) t = t * 0x9E3779B97F4A7C15ull + (uint32_t)x;
  return t << 1 | 1;
}

// ---- the plan: workgroup 0 deals the pages out, workgroup 1 + i makes the masks of request i
struct PlanCall { unsigned long long tag; int n, max_rows, heads, slots, max_pages; const int *cached, *row_starts, *parents; int* positions; Plan plan; };

// Exclusive sums over the workgroup's threads, and the totals, of N values.
template <int N>
__device__ __forceinline__ void plan_scan(int (&v)[N], int (&total)[N], int (*waves)[AT_PLAN_THREADS / 64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x[N];
#pragma unroll
  for (int i = 0; i < N; i++) {
    x[i] = wave_sums_up(v[i]);
    if (lane == 63) waves[i][wave] = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; i++) {
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < AT_PLAN_THREADS / 64; w++) {
      const int y = waves[i][w];
      before += w < wave ? y : 0;
      all += y;
    }
    total[i] = all;
    v[i] = before + x[i] - v[i];
  }
  __syncthreads();
}

// Whether request i's rows and lengths are in range (row_starts as a whole may still be out of order).
__device__ __forceinline__ bool request_ok(const PlanCall& c, int cached, int first, int end) {
  return first >= 0 && end >= first && end <= c.max_rows && end - first <= AT_NODES && cached >= 0 && cached <= c.max_pages * (long long)OP_PAGE - (end - first);
}

__device__ void deal_out(const PlanCall& c) {
  constexpr int N = OP_MAX_REQUESTS;
  // by request: first row; places on the lines of wide and narrow segments; the first wide and narrow segment (2^16 rows of 32 heads are 2^14 tiles and one for each
  // request); tiles (none of one that is not computed) and nodes of a tile
  __shared__ int start[N + 1], line_at[2][N + 1], cached[N], waves[4][AT_PLAN_THREADS / 64];
  __shared__ unsigned short seg0[2][N + 1], tiles_of[N], nodes_of[N];
  __shared__ int longest_of_all;
  const int n = c.n, tid = threadIdx.x;
  bool malformed = false;
  for (int i = tid; i <= n; i += AT_PLAN_THREADS) {
    const int s = c.row_starts[i];
    malformed |= s < 0 || s > c.max_rows || (i == 0 && s != 0) || (i < n && s > c.row_starts[i + 1]);
    start[i] = s;
    if (i < n) cached[i] = c.cached[i];
  }
  const bool ordered = !__syncthreads_or(malformed);
  struct Shape { int rows, pages, per, tiles, kind; };
  auto shape = [&](int i) {
    const int nodes = start[i + 1] - start[i], rows = nodes * c.heads;
    return Shape{rows, (cached[i] + nodes + OP_PAGE - 1) / OP_PAGE, nodes_of[i] * c.heads, tiles_of[i], rows <= AT_ROWS};
  };
  const int per = (n + AT_PLAN_THREADS - 1) / AT_PLAN_THREADS, r0 = min(n, tid * per), r1 = min(n, r0 + per);
  int sums[4] = {0, 0, 0, 0}, all[4], longest = 0;      // cost and segments, wide and narrow
  if (tid == 0) longest_of_all = 0;
  const int most = AT_TILE / c.heads;            // nodes of a tile; a request's tiles have alike numbers of them
  for (int i = r0; i < r1; i++) {
    const int nodes = start[i + 1] - start[i];
    int tiles = 0, of_tile = 1;
    if (ordered && nodes > 0 && request_ok(c, cached[i], start[i], start[i + 1])) {
      tiles = (nodes + most - 1) / most;
      of_tile = (nodes + tiles - 1) / tiles;
      tiles = (nodes + of_tile - 1) / of_tile;
    }
    tiles_of[i] = (unsigned short)tiles;
    nodes_of[i] = (unsigned short)of_tile;
    if (tiles == 0) continue;
    const Shape s = shape(i);
    sums[s.kind] += tiles * (s.pages + (s.kind ? AT_NARROW_START : AT_WIDE_START));
    sums[2 + s.kind] += tiles;
    longest = max(longest, s.pages);
  }
  __syncthreads();
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) longest = max(longest, __shfl_xor(longest, o, 64));
  if ((tid & 63) == 0) atomicMax(&longest_of_all, longest);
  plan_scan(sums, all, waves);
  longest = longest_of_all;
  // Short segments that all find a workgroup or wave of their own: each is as long on its line as a share.
  const bool apart = longest <= AT_APART && all[2] + (all[3] + 3) / 4 <= c.slots;
  const float wide_work = AT_WIDE_WEIGHT * all[0];
  int wide = all[0] == 0 ? 0 : (int)(c.slots * (wide_work / (wide_work + all[1])) + 0.5f);
  wide = apart ? all[2] : min(max(wide, (int)(all[0] > 0)), c.slots - (all[1] > 0));
  const int narrow = 4 * (c.slots - wide);
  auto line = [&](int total, int count, int start, int least, int granule) {
    const int share = apart ? start + longest : max((total + max(count, 1) - 1) / max(count, 1), start + least);
    return Line{share, start, granule, 1.f / (float)share};
  };
  const Line lines[2] = {line(all[0], wide, AT_WIDE_START, AT_WIDE_LEAST, 4), line(all[1], narrow, AT_NARROW_START, AT_NARROW_LEAST, 2)};
  auto tile_cost = [&](const Shape& s) { return (apart ? longest : s.pages) + (s.kind ? AT_NARROW_START : AT_WIDE_START); };
  if (apart) {
    sums[0] = sums[2] * lines[0].share; sums[1] = sums[3] * lines[1].share;
    all[0] = all[2] * lines[0].share; all[1] = all[3] * lines[1].share;
  }
  const int narrow_part = c.max_rows * c.heads + wide * AT_TILE;
  if (tid == 0) {
    *c.plan.header = Header{c.tag, ordered ? start[n] : -1, 0};
    line_at[0][n] = all[0]; line_at[1][n] = all[1];
  }
  for (int i = r0; i < r1; i++) {
    const Shape s = shape(i);
    line_at[0][i] = sums[0]; line_at[1][i] = sums[1];
    seg0[0][i] = (unsigned short)sums[2]; seg0[1][i] = (unsigned short)sums[3];
    if (s.tiles == 0) continue;
    sums[s.kind] += s.tiles * tile_cost(s);
    sums[2 + s.kind] += s.tiles;
  }
  __syncthreads();
  for (int row = tid; row < (ordered ? start[n] : 0); row += AT_PLAN_THREADS) {
    const int i = last_up_to(start, n, row);
    const Shape s = shape(i);
    Parts p{0, -1, 0, 0};
    if (s.tiles > 0) {
      const Line& l = lines[s.kind];
      const int at = line_at[s.kind][i] + (row - start[i]) / nodes_of[i] * tile_cost(s);
      p.step = s.kind ? AT_ROWS : AT_TILE;
      p.count = l.pieces(at, s.pages);
      p.base = (s.kind ? narrow_part : 0) + row * c.heads + p.step * l.first(at, s.pages);
    }
    c.plan.parts[row] = p;
  }
  // The items of a share, by a thread of its own. Neighbouring narrow shares go to different workgroups.
  for (int j = tid; j < wide + narrow; j += AT_PLAN_THREADS) {
    const int kind = j >= wide, k = kind ? j - wide : j;
    const Line& l = lines[kind];
    const int begin = k * l.share, end = begin + l.share;
    Range r{};
    r.wide = !kind;
    if (begin < all[kind]) {
      int i = last_up_to(line_at[kind], n, begin);                // has tiles there: the last of several at one place
      Shape s = shape(i);
      int t = (begin - line_at[kind][i]) / tile_cost(s);
      for (int from_at = line_at[kind][i] + t * tile_cost(s); from_at < end;) {
        const int from = begin > from_at ? l.up_to(from_at, s.pages, k - 1) : 0, to = l.up_to(from_at, s.pages, k);
        if (from < to) {
          const int item = (kind ? all[2] + wide : 0) + seg0[kind][i] + t + k, v0 = start[i] * c.heads + t * s.per;
          const bool done = to - from == s.pages;
          const Item it{v0, min(s.per, s.rows - t * s.per), i, from, to, done ? -1 : kind ? narrow_part + v0 + AT_ROWS * k : v0 + AT_TILE * k, cached[i], cached[i] + start[i + 1] - start[i]};
          if (r.first.rows == 0) {
            r.first = it;
            r.next = r.end = item + 1;
          } else {
            c.plan.items[item] = it;
            r.end = item + 1;
          }
        }
        from_at += tile_cost(s);
        if (++t < s.tiles) continue;
        do i++; while (i < n && line_at[kind][i + 1] == line_at[kind][i]);
        if (i == n) break;
        s = shape(i);
        t = 0;
      }
    }
    if (kind) {
      const int others = c.slots - wide;
      c.plan.ranges[(wide + k % others) * 4 + k / others] = r;
    } else {
      for (int w = 0; w < 4; w++) c.plan.ranges[k * 4 + w] = r;
    }
  }
}

__device__ void follow_parents(const PlanCall& c, int request) {
  __shared__ unsigned up[2][AT_NODES][8];        // ancestors and the node itself
  __shared__ short jump[2][AT_NODES];            // an ancestor further and further up, -1: none
  __shared__ unsigned char lost[2][AT_NODES];    // no node, or below one that is none
  const int first = c.row_starts[request], end = c.row_starts[request + 1], cached = c.cached[request], tid = threadIdx.x;
  if (first < 0 || end <= first || end > c.max_rows) return;
  const bool ok = request_ok(c, cached, first, end);
  if (!ok) {
    for (int row = first + tid; row < end; row += AT_PLAN_THREADS) {
      c.plan.nodes[row] = 1;
      if (c.positions) c.positions[row] = -1;
    }
    return;
  }
  // two threads a node, four words each
  const int nodes = end - first, i = tid >> 1, w0 = (tid & 1) * 4;
  if (i < nodes) {
    const int p = c.parents[first + i];
    const bool none = p < -1 || p >= i;
#pragma unroll
    for (int w = 0; w < 4; w++) up[0][i][w0 + w] = i >> 5 == w0 + w ? 1u << (i & 31) : 0u;
    if (w0 == 0) { jump[0][i] = (short)(none ? -1 : p); lost[0][i] = none; }
  }
  int now = 0;
  for (int reach = 1; reach < nodes; reach <<= 1, now ^= 1) {
    __syncthreads();
    const int j = i < nodes ? jump[now][i] : -1;
    if (!__syncthreads_or(j >= 0)) break;
    if (i < nodes) {
#pragma unroll
      for (int w = 0; w < 4; w++) up[now ^ 1][i][w0 + w] = up[now][i][w0 + w] | (j >= 0 ? up[now][j][w0 + w] : 0u);
      if (w0 == 0) {
        jump[now ^ 1][i] = j >= 0 ? jump[now][j] : (short)-1;
        lost[now ^ 1][i] = lost[now][i] | (j >= 0 ? lost[now][j] : (unsigned char)0);
      }
    }
  }
  __syncthreads();
  if (i >= nodes) return;
  const bool node = !lost[now][i];
  if (w0 == 0) {
    int depth = -1;
#pragma unroll
    for (int w = 0; w < 8; w++) depth += __popc(up[now][i][w]);
    if (c.positions) c.positions[first + i] = node ? cached + depth : -1;
    c.plan.nodes[first + i] = node;
  }
  // Bits of the tokens from the page of the first node on: those before it belong to the context. Words of two pages.
  const int shift = cached % OP_PAGE;
  unsigned* to = reinterpret_cast<unsigned*>(c.plan.masks + (size_t)(first + i) * AT_MASK);
  for (int w = tid & 1; w < 9; w += 2) {
    const unsigned here = w < 8 ? up[now][i][w] : 0u, before = w > 0 ? up[now][i][w - 1] : ~0u;
    to[w] = !node ? 0u : shift ? here << shift | before >> (32 - shift) : here;
  }
}

__global__ void __launch_bounds__(AT_PLAN_THREADS) attn_tree_plan_kernel(PlanCall c) {
  if (blockIdx.x == 0) deal_out(c);
  else follow_parents(c, blockIdx.x - 1);
}

// ---- the products
template <typename T>
struct TreeCall {
  const T* q; long long q_stride; const T* pool; T* out; long long out_stride; float* lse;
  const int* tables; long long table_stride;
  int max_rows, n, n_q, n_kv, heads, pool_pages;
  float scale_log2e;
  bool q_vec, out_vec;                           // rows can be loaded 16 bytes, stored 8 bytes at a time
  unsigned long long tag;                        // what the plan's header has to hold
  Plan plan;
};

// What a row sees of an item's pages.
struct Seen {
  const unsigned short* masks;
  int row, first, end;                           // node row, the page of the first node, the item's last page + 1
  __device__ __forceinline__ unsigned page(int pg) const { return pg >= end ? 0u : pg < first ? 0xFFFFu : masks[row * AT_MASK + pg - first]; }
};
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// Eight elements as the products may take them, those that are no numbers as 0: an exponent of ones carries into the sign's place. True if there were some.
template <typename T>
__device__ __forceinline__ bool without_odd(u32x4& x) {
  constexpr unsigned EXP = std::is_same<T, f16>::value ? 0x7C007C00u : 0x7F807F80u, ONE = std::is_same<T, f16>::value ? 0x04000400u : 0x00800080u;
  unsigned any = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const unsigned odd = ((x[i] & EXP) + ONE) >> 15 & 0x00010001u;
    x[i] &= ~(odd * 0xFFFFu);
    any |= odd;
  }
  return any != 0;
}
// Adds what those elements of V bring to the rows that see them, where the wave has stored its rows (first, .. of the item's): another branch's infinity must
// not become 0 * inf in a row that does not see it. p > 0 times an infinity or NaN is that. Seldom. The item's pages from pg0 on; `table`: of the whole request.
template <typename T, int D>
__device__ __forceinline__ void add_odd(const TreeCall<T>& c, const Item& it, int first, int rows, int pg0, const int* table, int kvh) {
  wait_vmem<0>();
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
  const int lane = threadIdx.x & 63;
#pragma unroll 1
  for (int t = pg0 * OP_PAGE; t < min(it.len, it.pg1 * OP_PAGE); t++) {
    const int page = table[t / OP_PAGE];
    if ((unsigned)page >= (unsigned)c.pool_pages) continue;
    const T* v = c.pool + ((size_t)page * c.n_kv + kvh) * 2 * OP_PAGE * D + OP_PAGE * D + t % OP_PAGE;
#pragma unroll 1
    for (int i = lane; i < rows * D; i += 64) {
      const int r = first + i / D, d = i % D, row = (it.row0 + r) / c.heads, head = kvh * c.heads + (it.row0 + r) % c.heads;
      const float x = (float)v[d * OP_PAGE];
      if (finite(x) || !(Seen{c.plan.masks, row, it.cached / OP_PAGE, it.pg1}.page(t / OP_PAGE) >> (t % OP_PAGE) & 1)) continue;
      if (it.part >= 0) {
        c.plan.outs[((size_t)(it.part + r) * c.n_kv + kvh) * D + d] += x;
      } else {
        T* to = c.out + (long long)row * c.out_stride + head * D + d;
        *to = (T)((float)*to + x);
      }
    }
  }
}

template <int D>
constexpr int attn_tree_lds() { return AS_LDS_BASE + 4 * 2 * 2 * 16 * D * 2; }   // two blocks of K for each wave; two tiles of K and V^T; 128 rows of output

// A lane's four elements of a row, 4 d-elements in a row, rounded once.
template <typename T>
__device__ __forceinline__ void store4(T* to, f32x4 x, float f, bool vec) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 v;
#pragma unroll
  for (int e = 0; e < 4; e++) v[e] = (T)(x[e] * f);
  if (vec) *reinterpret_cast<T4*>(to) = v;
  else
#pragma unroll
    for (int e = 0; e < 4; e++) to[e] = v[e];
}

// ---- narrow items, one wave: blocks of two pages (32 tokens), K rows global -> LDS without passing through registers, V^T straight into the registers of
// its product, both two blocks ahead, with the waits of attn_decode.hip, which explains the order of the tokens. Nobody else reads the pages:
// non-temporal.
template <typename T, int D>
__device__ __forceinline__ void run_narrow(unsigned char* smem, const TreeCall<T>& c, const Item& it, int kvh) {
  typedef typename Mfma<T>::V V;
  constexpr int KSTEPS = D / 16, DB = D / 32;
  constexpr int ROWB = D * 2, CPR = D / 8, RPI = 64 / CPR, IPP = 16 / RPI;   // K row bytes, 16-byte chunks, rows per load, loads per page
  constexpr int PAGE_KB = 16 * ROWB, STAGE = 2 * PAGE_KB;
  constexpr int LOADS = 2 * IPP + 2 * DB;            // loads of a block: K to LDS, V^T to registers
  const int tid = fresh(threadIdx.x), lane = tid & 63, l32 = lane & 31, lh = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int npg = it.pg1 - it.pg0, nblk = (npg + 1) >> 1;
  const int* table = c.tables + (long long)it.request * c.table_stride + it.pg0;
  const size_t head_elems = (size_t)2 * OP_PAGE * D;
  // Page numbers, 64 of them one per lane, and the next 64; past the end the last page again (fetched, left out). One outside the pool
  // is not followed: page 0 is read for it, and the rows come out as NaN.
  bool bad = false, odd = false;
  auto load_pages = [&](int window) {
    const int page = table[min(window * 64 + lane, npg - 1)];
    const bool out = (unsigned)page >= (unsigned)c.pool_pages;
    bad |= out;
    return out ? 0 : page;
  };
  int window = 0, pages_now = load_pages(0), pages_next = npg > 64 ? load_pages(1) : 0;
  auto page_base = [&](int i) -> const T* {           // windows are asked for in order
    const int j = __builtin_amdgcn_readfirstlane(min(i, npg - 1));
    if ((j >> 6) > window) { window++; pages_now = pages_next; pages_next = load_pages(window + 1); }
    const int page = __builtin_amdgcn_readlane(pages_now, j & 63);
    return c.pool + ((size_t)page * c.n_kv + kvh) * head_elems;
  };
  auto swz = [](int row) { return D == 128 ? (row & 15) : ((row >> 1) & 7); };
  unsigned char* kbuf = smem + AS_LDS_BASE + wv * 2 * STAGE;
  int ksrc[IPP];
#pragma unroll
  for (int j = 0; j < IPP; j++) {
    const int row = j * RPI + lane / CPR;
    ksrc[j] = row * D + ((lane % CPR) ^ swz(row)) * 8;
  }
  const T* base[2];                                   // the two pages of the block fetched last
  auto issue_k = [&](int b, int stage) {
#pragma unroll
    for (int u = 0; u < 2; u++) {
      base[u] = page_base(2 * b + u);
#pragma unroll
      for (int j = 0; j < IPP; j++) load_to_lds16_nt(base[u] + ksrc[j], kbuf + stage * STAGE + u * PAGE_KB + j * 1024);
    }
  };
  auto load_v = [&](u32x4 (&vr)[2][DB]) {
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int bb = 0; bb < DB; bb++) vr[u][bb] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base[u] + (size_t)16 * D + (bb * 32 + l32) * 16 + lh * 8));
  };

  // Q^T operand: column l32 is row l32 of the item
  V qf[KSTEPS];
  const int vrow = it.row0 + min(l32, it.rows - 1), row = vrow / c.heads, head = kvh * c.heads + vrow % c.heads;
  const Seen seen{c.plan.masks, row, it.cached / OP_PAGE, it.pg1};
  const int mixed = min(max(it.cached / OP_PAGE - it.pg0, 0), npg) >> 1;         // the first block that is not two pages of context of the item's
  {
    const T* q = c.q + (long long)row * c.q_stride + head * D + lh * 8;
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++) {
      if (c.q_vec) qf[kk] = *reinterpret_cast<const V*>(q + kk * 16);
      else
#pragma unroll
        for (int e = 0; e < 8; e++) qf[kk][e] = q[kk * 16 + e];
    }
  }
  const int tok = (l32 & 3) | (((l32 >> 3) & 1) << 2) | (((l32 >> 2) & 1) << 3);
  const int krow = (l32 >> 4) * PAGE_KB + tok * ROWB;
  int kslot[KSTEPS];
#pragma unroll
  for (int kk = 0; kk < KSTEPS; kk++) kslot[kk] = krow + ((2 * kk + lh) ^ swz(tok)) * 16;

  f32x16 o[DB];
#pragma unroll
  for (int bb = 0; bb < DB; bb++)
#pragma unroll
    for (int r = 0; r < 16; r++) o[bb][r] = 0.f;
  float m_ref = -INFINITY, l_run = 0.f;

  auto scores = [&](int stage, f32x16& s) {
    const unsigned char* kst = kbuf + stage * STAGE;
#pragma unroll
    for (int r = 0; r < 16; r++) s[r] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++) s = Mfma<T>::mul(*reinterpret_cast<const V*>(kst + kslot[kk]), qf[kk], s);
  };
  auto softmax_pv = [&](int b, f32x16& s, u32x4 (&vr)[2][DB]) {
    if (b >= mixed) {                                 // wave-uniform
      const int pg = it.pg0 + 2 * b;
      const unsigned see = seen.page(pg) >> (8 * lh) & 0xFF | (seen.page(pg + 1) >> (8 * lh) & 0xFF) << 8;
#pragma unroll
      for (int r = 0; r < 16; r++)                    // register r: page r >> 3 of the pair, token 8 * half + (r & 7)
        if (!(see >> r & 1)) s[r] = -INFINITY;
#pragma unroll
      for (int u = 0; u < 2; u++)                     // what lies behind the nodes may be anything: 0 * V must be 0
#pragma unroll
        for (int bb = 0; bb < DB; bb++) odd |= without_odd<T>(vr[u][bb]);
    }
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 16; r++) mx = fmaxf(mx, s[r]);
    mx = half_swap_max_f(mx);
    if (__any(mx > m_ref)) {                         // wave-uniform
      const float m_new = fmaxf(m_ref, mx);
      const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_ref - m_new) * c.scale_log2e);
      m_ref = m_new;
      l_run *= corr;
#pragma unroll
      for (int bb = 0; bb < DB; bb++)
#pragma unroll
        for (int r = 0; r < 16; r++) o[bb][r] *= corr;
    }
    const float nm = m_ref == -INFINITY ? 0.f : fmaf(-m_ref, c.scale_log2e, AS_LIFT<T>);
    float rs = 0.f;
#pragma unroll
    for (int r = 0; r < 16; r++) {
      const float p = __builtin_amdgcn_exp2f(fmaf(s[r], c.scale_log2e, nm));
      s[r] = p;
      rs += p;
    }
    l_run += rs;
#pragma unroll
    for (int u = 0; u < 2; u++) {
      V pb, pr;
      in_two(s, 8 * u, pb, pr);
#pragma unroll
      for (int bb = 0; bb < DB; bb++) o[bb] = Mfma<T>::mul(__builtin_bit_cast(V, vr[u][bb]), pb, o[bb]);
#pragma unroll
      for (int bb = 0; bb < DB; bb++) o[bb] = Mfma<T>::mul(__builtin_bit_cast(V, vr[u][bb]), pr, o[bb]);
    }
  };
  auto fence = [] { __asm__ volatile("" ::: "memory"); __builtin_amdgcn_sched_barrier(0); };
  u32x4 va[2][DB], vb[2][DB];
  auto step = [&](int i, int stage, u32x4 (&vr)[2][DB]) {
    if (i + 1 < nblk) wait_vmem<LOADS>(); else wait_vmem<0>();
    fence();
    f32x16 s;
    scores(stage, s);
    if (i + 2 < nblk) {
      __builtin_amdgcn_s_waitcnt(0xC07F);            // lgkmcnt(0): every K operand of this block has been read
      fence();
      issue_k(i + 2, stage);
    }
    softmax_pv(i, s, vr);
    if (i + 2 < nblk) load_v(vr);
  };
  issue_k(0, 0); load_v(va);
  if (nblk > 1) { issue_k(1, 1); load_v(vb); }
  for (int i = 0; i < nblk; i += 2) {
    step(i, 0, va);
    if (i + 1 < nblk) step(i + 1, 1, vb);
  }
  l_run += __shfl_xor(l_run, 32, 64);
  if (__any(bad)) l_run = NAN;

  // a lane has four elements in a row of its row's output, 32 bb + 8 r4 + 4 lh
  if (l32 < it.rows) {
    const float m2 = fmaf(m_ref, c.scale_log2e, -AS_LIFT<T>);
    auto four = [&](int bb, int r4) { return f32x4{o[bb][4 * r4], o[bb][4 * r4 + 1], o[bb][4 * r4 + 2], o[bb][4 * r4 + 3]}; };
    if (it.part < 0) {
      T* out = c.out + (long long)row * c.out_stride + head * D + 4 * lh;
      const float f = 1.f / ((1.f + AS_EXTRA<T>) * l_run);
#pragma unroll
      for (int bb = 0; bb < DB; bb++)
#pragma unroll
        for (int r4 = 0; r4 < 4; r4++) store4(out + bb * 32 + 8 * r4, four(bb, r4), f, c.out_vec);
      if (lh == 0 && c.lse) c.lse[(long long)row * c.n_q + head] = LN2 * (m2 + __builtin_amdgcn_logf(l_run));
    } else {
      const size_t at = (size_t)(it.part + l32) * c.n_kv + kvh;
      float* out = c.plan.outs + at * D + 4 * lh;
#pragma unroll
      for (int bb = 0; bb < DB; bb++)
#pragma unroll
        for (int r4 = 0; r4 < 4; r4++) *reinterpret_cast<f32x4*>(out + bb * 32 + 8 * r4) = four(bb, r4);
      if (lh == 0) c.plan.stats[at] = f32x2{m2, l_run};
    }
  }
  if (__any(odd)) add_odd<T, D>(c, it, 0, it.rows, it.pg0 + 2 * mixed, table - it.pg0, kvh);
}

// ---- wide items, a workgroup: tiles of four pages go global -> LDS, two stages deep, a page a wave. KB = 2: every wave takes 32 rows over all the pages;
// KB = 1 (up to 64 rows, a last tile's few ones too): waves w and w + 2 take the same 32 rows over two of each tile's pages, and join what they have at the end. Products, order of the tokens and softmax
// as in attn_prefill.hip, whose queries lie in a row where these come from any node.
// What bounds 128 rows: of 16 trees' cycles matrix instructions take 46 % and vector instructions 43 %, and on these cards the two hardly overlap, whatever their order: the next tile's
// first product between this one's exponentials, instruction by instruction, was level (298 and 300 us a step of two layers), as was reading K up to four steps ahead, or the first product
// at a higher priority. The tiles of a request read its pages each for itself (530 MB a layer past L2 where K and V are 270): eight waves on 256 rows read them once and took 280 instead of
// 301 us here, but 205 instead of 173 with six trees of different sizes and 79 instead of 70 with one tree.
// KB = 1 instead of 2 for 33 to 64 rows: three chains of 16 on 161 tokens (two layers) 46 -> 39 us, on 3214 tokens 71 -> 60.
template <typename T, int D, int KB>
__device__ __forceinline__ void run_wide(unsigned char* smem, const TreeCall<T>& c, const Item& it, int kvh) {
  typedef typename Mfma<T>::V V;
  constexpr int KSTEPS = D / 16, DB = D / 32;
  constexpr int ROWB = D * 2, CPR = D / 8, RPI = 64 / CPR, IPP = 16 / RPI;     // K row bytes, 16-byte chunks, rows per load, loads per page
  constexpr int PAGE = 16 * ROWB, TILE = 4 * PAGE, STAGE = 2 * TILE;           // bytes of a K (or V^T) page, tile; of a stage
  const int tid = fresh(threadIdx.x), lane = tid & 63, l32 = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int npg = it.pg1 - it.pg0, tiles = (npg + 3) >> 2;
  const int* table = c.tables + (long long)it.request * c.table_stride + it.pg0;
  const int block = KB == 2 ? wave : wave & 1, my_pages = KB == 2 ? 0 : wave & 2;       // of 32 rows; the wave's first page of a tile
  const int my_rows = min(it.rows - block * 32, 32);                           // none or fewer: the wave only fetches

  // This wave's page of tile kt; past the last page that page again, whose products are left out.
  bool bad = false, odd = false;
  const size_t page_stride = (size_t)c.n_kv * 2 * OP_PAGE * D;
  const T* pool_h = c.pool + (size_t)kvh * 2 * OP_PAGE * D;
  auto page_id = [&](int kt) {
    const int page = table[min(kt * 4 + wave, npg - 1)];
    const bool out = (unsigned)page >= (unsigned)c.pool_pages;
    bad |= out;
    return out ? 0 : page;
  };
  int next_page = page_id(0);
  const int page1 = page_id(1);
  V qf[KSTEPS];
  const int vrow = it.row0 + min(block * 32 + l32, it.rows - 1);
  const Seen seen{c.plan.masks, vrow / c.heads, it.cached / OP_PAGE, it.pg1};
  {
    const T* q = c.q + (long long)(vrow / c.heads) * c.q_stride + (kvh * c.heads + vrow % c.heads) * D + 8 * lh;
#pragma unroll
    for (int j = 0; j < KSTEPS; j++) {
      if (c.q_vec) qf[j] = *reinterpret_cast<const V*>(q + 16 * j);
      else
#pragma unroll
        for (int e = 0; e < 8; e++) qf[j][e] = q[16 * j + e];
    }
  }
  unsigned k_off[IPP];
#pragma unroll
  for (int j = 0; j < IPP; j++) {
    const int row = j * RPI + lane / CPR, swz = D == 128 ? row : (row >> 1) & 7;
    k_off[j] = (unsigned)row * ROWB + (unsigned)((lane % CPR) ^ swz) * 16u;
  }
  unsigned char* arena = smem + AS_LDS_BASE;
  auto issue = [&](int stage, int page) {
    const T* pb = pool_h + (size_t)__builtin_amdgcn_readfirstlane(page) * page_stride;
    unsigned char* dst = arena + stage * STAGE + wave * PAGE;
#pragma unroll
    for (int j = 0; j < IPP; j++) lds_dma16(pb, k_off[j], dst + j * 1024);
#pragma unroll
    for (int j = 0; j < IPP; j++) lds_dma16(pb + (size_t)16 * D, (unsigned)(j * 1024 + lane * 16), dst + TILE + j * 1024);
  };
  const int tok = (l32 & 3) | (((l32 >> 3) & 1) << 2) | (((l32 >> 2) & 1) << 3);
  const int k_row = my_pages * PAGE + (l32 >> 4) * PAGE + tok * ROWB;
  int k_slot[KSTEPS];
#pragma unroll
  for (int j = 0; j < KSTEPS; j++) k_slot[j] = k_row + ((2 * j + lh) ^ (D == 128 ? tok : (tok >> 1) & 7)) * 16;
  const int v_lane = TILE + my_pages * PAGE + l32 * 32 + lh * 16;              // V^T operand: d row l32 of a 32-row block, tokens 8 lh .. of a page

  f32x16 o[DB];
#pragma unroll
  for (int b = 0; b < DB; b++)
#pragma unroll
    for (int r = 0; r < 16; r++) o[b][r] = 0.f;
  float m_ref = -INFINITY, l_run = 0.f;
  const int mixed = max(min(it.cached / OP_PAGE, it.pg1) - it.pg0, 0) >> 2;    // the first tile that is not four pages of context of the item's
  issue(0, next_page);
  next_page = page1;
  auto tile = [&](int kt) {
    const unsigned char* st = arena + (kt & 1) * STAGE;
    unsigned see[KB];                                      // a bit for each of a lane's scores
    if (kt >= mixed)                                       // wave-uniform, as below
#pragma unroll
      for (int kb = 0; kb < KB; kb++) {
        const int pg = it.pg0 + kt * 4 + my_pages + 2 * kb;
        see[kb] = seen.page(pg) >> (8 * lh) & 0xFF | (seen.page(pg + 1) >> (8 * lh) & 0xFF) << 8;
      }
    f32x16 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; kb++)
#pragma unroll
      for (int r = 0; r < 16; r++) s[kb][r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
    {
      V kf[2][KB];
#pragma unroll
      for (int kb = 0; kb < KB; kb++) kf[0][kb] = *reinterpret_cast<const V*>(st + kb * 2 * PAGE + k_slot[0]);
#pragma unroll
      for (int j = 0; j < KSTEPS; j++) {
        const int a = j & 1, b = a ^ 1;
        if (j + 1 < KSTEPS) {
#pragma unroll
          for (int kb = 0; kb < KB; kb++) kf[b][kb] = *reinterpret_cast<const V*>(st + kb * 2 * PAGE + k_slot[j + 1]);
        }
#pragma unroll
        for (int kb = 0; kb < KB; kb++) s[kb] = Mfma<T>::mul(kf[a][kb], qf[j], s[kb]);
      }
      __builtin_amdgcn_sched_group_barrier(0x100, KB, 0);
#pragma unroll
      for (int j = 0; j + 1 < KSTEPS; j++) {
        __builtin_amdgcn_sched_group_barrier(0x100, KB, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, KB, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, KB, 0);
    }
    V vf[2][DB];                                           // first V^T operands: in flight during the softmax arithmetic
#pragma unroll
    for (int b = 0; b < DB; b++) vf[0][b] = *reinterpret_cast<const V*>(st + v_lane + b * 1024);
    if (kt >= mixed)
#pragma unroll
      for (int kb = 0; kb < KB; kb++)
#pragma unroll
        for (int r = 0; r < 16; r++)
          if (!(see[kb] >> r & 1)) s[kb][r] = -INFINITY;
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KB; kb++)
#pragma unroll
      for (int r = 0; r < 16; r++) mx = fmaxf(mx, s[kb][r]);
    mx = half_swap_max_f(mx);
    // The reference moves when a score has outgrown it by 2^8, by which probabilities and their sums may then exceed 1: two numbers of the type, and 32 bits,
    // hold them as well there.
    if (__any((mx - m_ref) * c.scale_log2e > AS_RISE)) {                       // wave-uniform
      const float m_new = fmaxf(m_ref, mx);
      const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m_ref - m_new) * c.scale_log2e);
      m_ref = m_new;
      l_run *= corr;
#pragma unroll
      for (int b = 0; b < DB; b++)
#pragma unroll
        for (int r = 0; r < 16; r++) o[b][r] *= corr;
    }
    const float nm = (m_ref == -INFINITY) ? 0.f : fmaf(-m_ref, c.scale_log2e, AS_LIFT<T>);
    float rs = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; kb++)
#pragma unroll
      for (int r = 0; r < 16; r++) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[kb][r], c.scale_log2e, nm));
        s[kb][r] = p;
        rs += p;
      }
    l_run += rs;                                                               // this half's keys; halves are added at the end
#pragma unroll
    for (int g = 0; g < 2 * KB; g++) {
      const int a = g & 1, b2 = a ^ 1;
      if (g + 1 < 2 * KB) {
#pragma unroll
        for (int b = 0; b < DB; b++) vf[b2][b] = *reinterpret_cast<const V*>(st + v_lane + (g + 1) * PAGE + b * 1024);
      }
      V pb, pr;
      in_two(s[g >> 1], 8 * (g & 1), pb, pr);
#pragma unroll
      for (int b = 0; b < DB; b++) o[b] = Mfma<T>::mul(vf[a][b], pb, o[b]);
#pragma unroll
      for (int b = 0; b < DB; b++) o[b] = Mfma<T>::mul(vf[a][b], pr, o[b]);
    }
#pragma unroll
    for (int g = 0; g + 1 < 2 * KB; g++) {
      __builtin_amdgcn_sched_group_barrier(0x100, DB, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 2 * DB, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 2 * DB, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  for (int kt = 0; kt < tiles; kt++) {
    wait_vmem<0>();                                        // every wave waits for its own page, and nobody reads the other stage any more
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
    if (kt + 1 < tiles) {
      issue((kt + 1) & 1, next_page);
      next_page = page_id(kt + 2);
    }
    if (kt >= mixed) {                                     // what lies behind the nodes may be anything: 0 * V must be 0
      bool here = false;
      unsigned char* vt = arena + (kt & 1) * STAGE + TILE;
      for (int i = tid; i < TILE / 16; i += 256) {
        u32x4 x = *reinterpret_cast<const u32x4*>(vt + i * 16);
        if (!without_odd<T>(x)) continue;
        here = true;
        *reinterpret_cast<u32x4*>(vt + i * 16) = x;
      }
      odd |= __syncthreads_or(here);
    }
    if (my_rows > 0) tile(kt);                             // wave-uniform
  }
  l_run += __shfl_xor(l_run, 32, 64);
  if (__syncthreads_or(bad)) l_run = NAN;                // LDS now takes the output
  // whole rows through LDS: 16-byte chunks, swizzled by row
  constexpr int OROWB = D * 4, OCPR = OROWB / 16, ORPI = 64 / OCPR;
  unsigned char* buf = arena + block * 32 * OROWB;
  auto slot = [&](int row, int chunk) { return reinterpret_cast<f32x4*>(buf + row * OROWB + (chunk ^ (row % 16)) * 16); };
  f32x2* other = reinterpret_cast<f32x2*>(arena + 2 * 32 * OROWB) + block * 32;         // KB = 1: maximum and sum of the waves of the second pages
  const int lane2 = fresh(tid & 63), r32 = lane2 & 31, rh = lane2 >> 5;
  if (KB == 1) {
    if (my_pages != 0 && my_rows > 0) {
#pragma unroll
      for (int b = 0; b < DB; b++)
#pragma unroll
        for (int r4 = 0; r4 < 4; r4++) *slot(r32, b * 8 + 2 * r4 + rh) = f32x4{o[b][4 * r4], o[b][4 * r4 + 1], o[b][4 * r4 + 2], o[b][4 * r4 + 3]};
      if (rh == 0) other[r32] = f32x2{m_ref, l_run};
    }
    __syncthreads();
    if (my_pages == 0 && my_rows > 0) {
      const f32x2 st = other[r32];
      const float m = fmaxf(m_ref, st[0]);
      const float fa = m_ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_ref - m) * c.scale_log2e), fb = st[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((st[0] - m) * c.scale_log2e);
      // an empty side's sum is 0, or NaN for a page that is none
      l_run = (m_ref == -INFINITY ? l_run : l_run * fa) + (st[0] == -INFINITY ? st[1] : st[1] * fb);
      m_ref = m;
#pragma unroll
      for (int b = 0; b < DB; b++)
#pragma unroll
        for (int r4 = 0; r4 < 4; r4++) {
          const f32x4 x = *slot(r32, b * 8 + 2 * r4 + rh);
#pragma unroll
          for (int e = 0; e < 4; e++) o[b][4 * r4 + e] = o[b][4 * r4 + e] * fa + x[e] * fb;
        }
    }
  }
  if (my_rows > 0 && my_pages == 0) {
#pragma unroll
    for (int b = 0; b < DB; b++)
#pragma unroll
      for (int r4 = 0; r4 < 4; r4++) *slot(r32, b * 8 + 2 * r4 + rh) = f32x4{o[b][4 * r4], o[b][4 * r4 + 1], o[b][4 * r4 + 2], o[b][4 * r4 + 3]};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int r0 = lane2 / OCPR, ch = lane2 % OCPR;
    const float m2 = fmaf(m_ref, c.scale_log2e, -AS_LIFT<T>), f = 1.f / ((1.f + AS_EXTRA<T>) * l_run);
#pragma unroll
    for (int i = 0; i < 32 / ORPI; i++) {
      const int r = i * ORPI + r0;
      const f32x4 x = *slot(r, ch);
      const float fr = __shfl(f, r, 64);
      if (r >= my_rows) continue;
      if (it.part < 0) {
        const int v = it.row0 + block * 32 + r;
        store4(c.out + (long long)(v / c.heads) * c.out_stride + (kvh * c.heads + v % c.heads) * D + ch * 4, x, fr, c.out_vec);
      } else {
        *reinterpret_cast<f32x4*>(c.plan.outs + ((size_t)(it.part + block * 32 + r) * c.n_kv + kvh) * D + ch * 4) = x;
      }
    }
    if (lane2 < my_rows) {
      if (it.part >= 0) c.plan.stats[(size_t)(it.part + block * 32 + lane2) * c.n_kv + kvh] = f32x2{m2, l_run};
      else if (c.lse) {
        const int v = it.row0 + block * 32 + lane2;
        c.lse[(long long)(v / c.heads) * c.n_q + kvh * c.heads + v % c.heads] = LN2 * (m2 + __builtin_amdgcn_logf(l_run));
      }
    }
    if (odd) add_odd<T, D>(c, it, block * 32, my_rows, it.pg0 + 4 * mixed, table - it.pg0, kvh);
  }
  __syncthreads();                                       // before the next item's K lands there
}

template <typename T, int D>
__global__ void __launch_bounds__(256, 2) attn_tree_kernel(TreeCall<T> c) {
  __shared__ __align__(16) unsigned char smem[attn_tree_lds<D>()];
  // With 8 KV heads a head's workgroups are all on one XCD: the tiles of a request find each other's pages in its L2.
  const int slot = blockIdx.x / c.n_kv, kvh = blockIdx.x % c.n_kv;
  const Range& r = c.plan.ranges[slot * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)];
  auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  auto take = [&](const Item& x) { return Item{scalar(x.row0), scalar(x.rows), scalar(x.request), scalar(x.pg0), scalar(x.pg1), scalar(x.part), scalar(x.cached), scalar(x.len)}; };
  Item it = take(r.first);
  const int next = scalar(r.next), end = scalar(r.end), wide = scalar(r.wide);
  if (c.plan.header->tag != c.tag || it.rows == 0) return;
  for (int i = next;; i++) {
    if (!wide) run_narrow<T, D>(smem, c, it, kvh);
    else if (it.rows > 2 * AT_ROWS) run_wide<T, D, 2>(smem, c, it, kvh);
    else run_wide<T, D, 1>(smem, c, it, kvh);
    if (i >= end) break;
    it = take(c.plan.items[i]);
  }
}

// Where the partial results of a (row, query head) are.
struct Pieces { int count, base, step; bool bad, done; };          // done: finished by its one piece, or behind the last row
template <typename T>
__device__ __forceinline__ Pieces pieces_of(const TreeCall<T>& c, int row, int h) {
  const Header hd = *c.plan.header;
  const Parts p = c.plan.parts[row];                     // whatever they hold where there is no plan
  const int node = c.plan.nodes[row];
  if (hd.tag != c.tag || hd.rows < 0) return Pieces{0, 0, 0, true, false};
  if (row >= hd.rows) return Pieces{0, 0, 0, false, true};
  if (p.count < 0) return Pieces{0, 0, 0, true, false};
  return Pieces{node ? p.count : 0, p.base + h, p.step, false, node && p.count == 1};
}
// A lane's four elements from e4 on; lse by the lane of the first.
template <typename T, int D>
__device__ __forceinline__ void finish_row(const TreeCall<T>& c, int row, int head, int e4, const Pieces& p, float m, float l, f32x4 o) {
  const bool none = p.count == 0;                        // no node: zeros, and the logarithm of an empty sum
  const f32x4 x = p.bad ? f32x4{NAN, NAN, NAN, NAN} : none ? f32x4{0.f, 0.f, 0.f, 0.f} : o;
  store4(c.out + (long long)row * c.out_stride + head * D + e4, x, none ? 1.f : 1.f / ((1.f + AS_EXTRA<T>) * l), c.out_vec);
  if (e4 == 0 && c.lse) c.lse[(long long)row * c.n_q + head] = p.bad ? NAN : none ? -INFINITY : LN2 * (m + __builtin_amdgcn_logf(l));
}

// Joins the partial results of a (row, query head), where there are few of these: four waves each, a lane four elements of every 1024 / D-th part.
template <typename T, int D>
__global__ void __launch_bounds__(256) attn_tree_join_few_kernel(TreeCall<T> c) {
  constexpr int LANES = D / 4, WAVES = 4, APART = 64 / LANES * WAVES;       // lanes of a part, parts side by side
  __shared__ f32x4 sums[WAVES][LANES];
  __shared__ f32x2 ls[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x / c.n_q, head = blockIdx.x % c.n_q, kvh = head / c.heads;
  const Pieces p = pieces_of(c, row, head % c.heads);
  if (p.done) return;
  auto row_of = [&](int j) { return (size_t)(p.base + j * p.step) * c.n_kv + kvh; };
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](float m1, float l1, f32x4 o1) {         // another part's maximum, sum (0 of one without scores above -inf, or NaN) and output
    const float now = fmaxf(m, m1), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now), f1 = m1 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m1 - now);
    l = (m == -INFINITY ? l : l * f) + (m1 == -INFINITY ? l1 : l1 * f1);
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] = o[e] * f + o1[e] * f1;
    m = now;
  };
  const int first = wave * (64 / LANES) + lane / LANES, e4 = lane % LANES * 4;
  for (int j0 = first; j0 < p.count; j0 += AT_JOIN_BATCH * APART) {
    f32x2 st[AT_JOIN_BATCH];
    f32x4 x[AT_JOIN_BATCH];
#pragma unroll
    for (int u = 0; u < AT_JOIN_BATCH; u++) {
      const size_t part = row_of(min(j0 + u * APART, p.count - 1));
      st[u] = c.plan.stats[part];
      x[u] = *reinterpret_cast<const f32x4*>(c.plan.outs + part * D + e4);
    }
#pragma unroll
    for (int u = 0; u < AT_JOIN_BATCH; u++)
      if (j0 + u * APART < p.count) add(st[u][0], st[u][1], x[u]);
  }
#pragma unroll
  for (int s = LANES; s < 64; s <<= 1) add(__shfl_xor(m, s, 64), __shfl_xor(l, s, 64), f32x4{__shfl_xor(o[0], s, 64), __shfl_xor(o[1], s, 64), __shfl_xor(o[2], s, 64), __shfl_xor(o[3], s, 64)});
  if (lane < LANES) sums[wave][lane] = o;
  if (lane == 0) ls[wave] = f32x2{m, l};
  __syncthreads();
  if (wave > 0 || lane >= LANES) return;
#pragma unroll
  for (int w = 1; w < WAVES; w++) add(ls[w][0], ls[w][1], sums[w][lane]);
  finish_row<T, D>(c, row, head, e4, p, m, l, o);
}

// Joins the partial results of many: a run of D / 4 lanes each, which take the parts in order, their statistics as many at a time as there are lanes.
template <typename T, int D>
__global__ void __launch_bounds__(256) attn_tree_join_kernel(TreeCall<T> c) {
  constexpr int LANES = D / 4, RUNS = 256 / LANES;
  const int lane = threadIdx.x % LANES, at = (int)(blockIdx.y * gridDim.x + blockIdx.x) * RUNS + threadIdx.x / LANES;
  if (at >= c.max_rows * c.n_q) return;
  const int row = at / c.n_q, head = at % c.n_q, kvh = head / c.heads;
  const Pieces p = pieces_of(c, row, head % c.heads);
  if (p.done) return;
  auto row_of = [&](int j) { return (size_t)(p.base + j * p.step) * c.n_kv + kvh; };
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f}, x[AT_JOIN_BATCH];
  auto fetch = [&](int j) {                              // past the last the last again, which counts for nothing
#pragma unroll
    for (int u = 0; u < AT_JOIN_BATCH; u++) x[u] = *reinterpret_cast<const f32x4*>(c.plan.outs + row_of(min(j + u, p.count - 1)) * D + lane * 4);
  };
  if (p.count > 0) fetch(0);
  for (int j0 = 0; j0 < p.count; j0 += LANES) {
    const f32x2 st = j0 + lane < p.count ? c.plan.stats[row_of(j0 + lane)] : f32x2{-INFINITY, 0.f};
    float now = st[0];
#pragma unroll
    for (int s = 1; s < LANES; s <<= 1) now = fmaxf(now, __shfl_xor(now, s, 64));
    now = fmaxf(now, m);
    if (now > m) {                                       // the same for the run
      const float f = __builtin_amdgcn_exp2f(m - now);
      l *= f;
#pragma unroll
      for (int e = 0; e < 4; e++) o[e] *= f;
      m = now;
    }
    const float w = st[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[0] - m);
    float z = st[0] == -INFINITY ? st[1] : st[1] * w;            // 0 of a part without scores above -inf, or NaN
#pragma unroll
    for (int s = 1; s < LANES; s <<= 1) z += __shfl_xor(z, s, 64);
    l += z;
    const int n = min(LANES, p.count - j0);
    for (int j = 0; j < n; j += AT_JOIN_BATCH) {
      if (j0 + j > 0) fetch(j0 + j);
#pragma unroll
      for (int u = 0; u < AT_JOIN_BATCH; u++) {
        const float wj = __shfl(w, j + u, LANES);
        if (j + u < n)
#pragma unroll
          for (int e = 0; e < 4; e++) o[e] += x[u][e] * wj;
      }
    }
  }
  finish_row<T, D>(c, row, head, lane * 4, p, m, l, o);
}

template <typename T, int D>
hipError_t launch_attn(hipStream_t s, const TreeCall<T>& c) {
  hipError_t e = launch(attn_tree_kernel<T, D>, dim3(slots_of(c.n_kv) * c.n_kv), dim3(256), 0, s, c);
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)c.max_rows * c.n_q;
  if (rows <= AT_JOIN_ROWS) return launch(attn_tree_join_few_kernel<T, D>, dim3((unsigned)rows), dim3(256), 0, s, c);
  // a launch's x ends below 2^32 threads: the most rows of the most heads are 2^34
  constexpr int RUNS = 256 / (D / 4);
  const unsigned groups = (unsigned)((rows + RUNS - 1) / RUNS), x = std::min(groups, 1u << 20);
  return launch(attn_tree_join_kernel<T, D>, dim3(x, (groups + x - 1) / x), dim3(256), 0, s, c);
}

bool sizes_ok(int n, int max_rows, int n_q, int n_kv, int d) {
  return n >= 0 && n <= OP_MAX_REQUESTS && max_rows >= 0 && max_rows <= AT_MAX_ROWS && n_kv >= 1 && n_kv <= AT_SLOTS / 2 && n_q >= n_kv && n_q % n_kv == 0 && n_q / n_kv <= AT_ROWS &&
         (d == 64 || d == 128);
}
// The batch's description, without what a call of one layer adds.
int check_batch(const sts_tree_batch* b, Plan* plan) {
  if (!b || (b->dtype != STS_BF16 && b->dtype != STS_F16) || !sizes_ok(b->n_requests, b->max_rows, b->n_q, b->n_kv, b->d)) return STS_EINVAL;
  if (b->pool_pages < 0 || b->max_pages < 0 || b->max_pages > (1 << 26) || b->table_stride < b->max_pages) return STS_EINVAL;
  // the lines' lengths stay within 32 bits
  if (max_segments(b->n_requests, b->max_rows, b->n_q / b->n_kv) * (b->max_pages + (int64_t)AT_WIDE_START) > (1 << 30)) return STS_EINVAL;
  if (b->n_requests == 0 || b->max_rows == 0) return STS_OK;
  if (!b->cached || !b->row_starts || !b->parents || (b->max_pages > 0 && !b->tables)) return STS_EINVAL;
  if (b->positions && (b->positions == b->parents || b->positions == b->cached || b->positions == b->row_starts)) return STS_EINVAL;      // read by workgroups that start late
  if (!b->workspace || !aligned(b->workspace, 256)) return STS_EINVAL;
  if ((int64_t)lay_out(reinterpret_cast<unsigned char*>(b->workspace), b->n_requests, b->max_rows, b->n_q, b->n_kv, b->d, plan) > b->workspace_bytes) return STS_EINVAL;
  return STS_OK;
}

template <typename T>
int attn_tree(const sts_tree_batch* b, const Plan& plan, const void* q, int64_t q_stride, const void* pool, void* out, int64_t out_stride, float* lse, float scale, hipStream_t s) {
  const bool q_vec = aligned(q, 16) && q_stride % 8 == 0, out_vec = aligned(out, 8) && out_stride % 4 == 0;
  const TreeCall<T> c{reinterpret_cast<const T*>(q), q_stride, reinterpret_cast<const T*>(pool), reinterpret_cast<T*>(out), out_stride, lse, b->tables, b->table_stride,
                      b->max_rows, b->n_requests, b->n_q, b->n_kv, b->n_q / b->n_kv, b->pool_pages, scale * LOG2E, q_vec, out_vec, sizes_tag(*b), plan};
  return op_result(b->d == 128 ? launch_attn<T, 128>(s, c) : launch_attn<T, 64>(s, c));
}

}  // namespace
}  // namespace sts

using namespace sts;

extern "C" int64_t sts_attn_tree_workspace(int32_t n_requests, int32_t max_rows, int32_t n_q, int32_t n_kv, int32_t d) {
  if (!sizes_ok(n_requests, max_rows, n_q, n_kv, d)) return -1;
  return (int64_t)lay_out(nullptr, n_requests, max_rows, n_q, n_kv, d, nullptr);
}

extern "C" int sts_op_attn_tree_plan(const sts_tree_batch* b, void* stream) {
  Plan plan{};
  const int rc = check_batch(b, &plan);
  if (rc != STS_OK || b->n_requests == 0 || b->max_rows == 0) return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  const PlanCall c{sizes_tag(*b), b->n_requests, b->max_rows, b->n_q / b->n_kv, slots_of(b->n_kv), b->max_pages, b->cached, b->row_starts, b->parents, b->positions, plan};
  return op_result(launch(attn_tree_plan_kernel, dim3(1 + b->n_requests), dim3(AT_PLAN_THREADS), 0, s, c));
}

extern "C" int sts_op_attn_tree(const sts_tree_batch* b, const void* q, int64_t q_stride, const void* pool, void* out, int64_t out_stride, float* lse, float scale, void* stream) {
  Plan plan{};
  const int rc = check_batch(b, &plan);
  if (rc != STS_OK || b->n_requests == 0 || b->max_rows == 0) return rc;
  const int64_t row = (int64_t)b->n_q * b->d;
  if (!q || !out || !aligned(q, 2) || !aligned(out, 2) || !pool || !aligned(pool, 16) || b->pool_pages < 1 || (b->max_rows > 1 && (q_stride < row || out_stride < row))) return STS_EINVAL;
  if (!(scale >= 0.f) || scale > 1e30f) return STS_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  const float sc = scale == 0.f ? 1.f / sqrtf((float)b->d) : scale;
  return b->dtype == STS_BF16 ? attn_tree<bf16>(b, plan, q, q_stride, pool, out, out_stride, lse, sc, s) : attn_tree<f16>(b, plan, q, q_stride, pool, out, out_stride, lse, sc, s);
}
