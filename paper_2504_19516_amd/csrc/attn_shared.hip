// Decode attention for requests that share the beginning of their contexts (Section 3.5.1's pages in several block tables): a
// group's shared pages are read once for all its requests, every request's own pages once for it.
//
//   o_r = sum_t p_t v_t / l,   p_t = 2^(scale log2(e) q_r . k_t - m),   l = sum_t p_t,   over the tokens t < len_r
//
// computed in parts of the token range, each with its own maximum m, that a second kernel joins:
//   m = max m_j,  l = sum l_j 2^(m_j - m),  o = sum o_j 2^(m_j - m) / l
//
// A segment is a token range with the rows that read it: the shared pages of a group with a tile of its requests, or the own pages of
// one request. A request brings n_q / n_kv rows (the query heads of a KV head) to the products, so a tile of shared pages fills the matrix
// cores' columns that a single request leaves empty. There are two kinds:
//   - up to 32 rows (narrow): one wave takes pages by itself, bound by memory;
//   - up to 128 rows (wide): the four waves of a workgroup take 32 rows each and share the pages through LDS, bound by the matrix cores
//     and by the exponentials beside them.
// The plan, made once a step on the device from the lengths, divides the workgroups of a KV head between the kinds in proportion to their
// work, lays each kind's segments end to end (pages, and the start and end of a segment counted as pages) and cuts each line into equal
// shares, one for each workgroup or wave: a long context is shared by many, short ones are strung together.
//
// Measured, bf16, 32 query and 8 KV heads of 128; us of the plan (once a step), and of products and join (each layer):
//   8 requests on 1031 shared tokens, 6 MB of pages a layer     7    8   4    latency
//   64 requests on 2048 shared tokens, 100 MB                    8   24   5    4.2 TB/s in the products: memory
//   256 requests on a document of 8192 tokens, 187 MB           12   89  10    2.1 TB/s and 0.39 PFLOP/s at once (0.59 with the second numbers): matrix cores and exponentials
// (medians under a trace; on another card the document's products were 94)
// (read by every request for itself, the document alone would be 8.6 GB a layer).
#include <algorithm>

#include "device_ops.h"

namespace sts {
namespace {

constexpr int AS_ROWS = 32;                     // rows of a narrow segment: columns of a product
constexpr int AS_TILE = 128;                    // rows of a wide one
constexpr int AS_SLOTS = 512;                   // workgroups of a launch: two on each CU
constexpr int AS_PLAN_THREADS = 512;
// Up to so many (request, head) pairs four waves join each, beyond it one: products and join of 16 requests on 8192 tokens (512 pairs) 22.3 us with four and
// 23.7 with one, of 128 on 2048 (4096 pairs) 29.5 and 25.4. In between it is the parts that count, which the host does not know: 24 requests of
// several long prompts (1536 pairs, a step of two layers) 61 and 63, 64 requests on 2048 tokens (2048 pairs, four layers) 126 and 119.
constexpr int AS_JOIN_ROWS = 1024;
// Start and end of a wide and of a narrow segment, and the smallest shares beyond them, in pages; what a page of a wide segment takes a
// workgroup, in pages of a narrow one. Products and join of 40 requests on 1000 tokens / of 96 in four groups on 4096 (64 heads) / a step of 256 on one document (two layers):
// 16.2 / 58 / 187 us as here; wide start and least share of 16 and 8 pages 19.9 / 58 / 184; wide weight 1: 16.4 / 60 / 189, 1.6: 16.3 / 57 /
// 179 (but 128 requests on 2048 tokens 27.6 for 25.4); narrow least share of 2: 17.0 / 59 / 186, 8: 19.3 / 58 / 187 (a single request of 8192 tokens 17.0, 16.5 and 16.0 with 2, 4 and 8;
// a step of 8 requests on 1000 tokens, four layers, 54.4, 56.1 and 62.5).
// Where the line of narrow segments costs AS_LONG pages or more for each segment of the batch (wide ones and those without pages count too) and AS_LONG_SHARE pages or more for
// each wave, its shares are not below AS_LONG_LEAST: fewer partial results and joins for a longer way of each wave. 64 requests on 2048 tokens (four layers) 126 ->
// 119 us, the larger shape's groups (two) 67 -> 63, 8 requests of 2000 tokens 20.0 -> 19.5; with 12 pages 123, 65 and 22.1. Where waves have less to do, it is slower: 2 requests of 3000
// tokens 12.0 -> 14.6.
constexpr int AS_WIDE_START = 8, AS_NARROW_START = 2, AS_WIDE_LEAST = 4, AS_NARROW_LEAST = 4, AS_LONG = 16, AS_LONG_SHARE = 3, AS_LONG_LEAST = 8;
constexpr float AS_WIDE_WEIGHT = 1.25f, AS_RISE = 8.f;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// A piece of a segment: rows row0 .. row0 + rows - 1 (request * heads of a group + head) over the pages [pg0, pg1) of a request's
// table, tokens from len on left out. part: number of its first row's partial result, -1: it finishes its rows. once: nobody else reads the pages.
struct Item { int row0, rows, request, pg0, pg1, len, part, once; };
struct Range { Item first; int next, end, pad[2]; };              // items of a wave: the first, and next .. end - 1; none if its rows are 0. The four of a workgroup with wide ones have the same
// Where a request's partial results are: head h in p_part + j * p_step + h, j < p_count, and s_part + j * heads + h, j < s_count.
// done: its one piece finishes it. len < 0: its length is out of range.
struct Parts { int p_part, p_step, p_count, s_part, s_count, len, done, pad; };
struct Plan {
  unsigned long long* sizes;                     // sizes_tag() of the batch that it was made for
  Range* ranges;                                 // [slots][4]
  Item* items;
  Parts* parts;                                  // [n_requests]
  f32x2* stats;                                  // [partial row][kv head]: maximum (log2 units), sum
  float* outs;                                   // [partial row][kv head][d]
};

int slots_of(int n_kv) { return std::max(1, AS_SLOTS / n_kv); }
// A segment is one piece, and one more for every share that ends in it; shares are a workgroup's of 128 rows or a wave's of 32.
int max_items(int n, int n_kv) { return 2 * n + 4 * slots_of(n_kv); }
int64_t max_part_rows(int n, int n_q, int n_kv) { return (int64_t)2 * n * (n_q / n_kv) + (int64_t)slots_of(n_kv) * AS_TILE; }

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
// The workspace's parts behind each other; returns its size.
size_t lay_out(unsigned char* base, int n, int n_q, int n_kv, int d, Plan* p) {
  size_t at = 0;
  auto take = [&](size_t bytes) { unsigned char* q = base + at; at += up256(bytes); return q; };
  const size_t rows = (size_t)max_part_rows(n, n_q, n_kv) * n_kv;
  Plan q;
  q.sizes = reinterpret_cast<unsigned long long*>(take(sizeof(unsigned long long)));
  q.ranges = reinterpret_cast<Range*>(take(slots_of(n_kv) * 4 * sizeof(Range)));
  q.items = reinterpret_cast<Item*>(take(max_items(n, n_kv) * sizeof(Item)));
  q.parts = reinterpret_cast<Parts*>(take(n * sizeof(Parts)));
  q.stats = reinterpret_cast<f32x2*>(take(rows * sizeof(f32x2)));
  q.outs = reinterpret_cast<float*>(take(rows * d * sizeof(float)));
  if (p) *p = q;
  return at;
}

// The sizes on which the indexes of a plan's users depend, never 0. A workspace without a plan of the batch's sizes gives NaN: nothing in it is followed.
unsigned long long sizes_tag(const sts_attn_batch& b) {
  unsigned long long t = 1;
  for (int32_t x : {b.n_requests, b.n_q, b.n_kv, b.d, b.max_pages}) t = t * 0x9E3779B97F4A7C15ull + (uint32_t)x;
  return t << 1 | 1;
}

// ---- the plan: one workgroup
// wide_requests: of a wide tile, and 2^20 over it, rounded up: quotients of numbers up to 4223 by it are exact, as 4223 * 128 < 2^20
struct PlanCall { unsigned long long tag; int n, groups, heads, slots, max_pages, wide_requests; unsigned wide_inverse; const int *lens, *group_starts, *shared_lens; Plan plan; };

// The sum of a wave's values up to each lane's: within rows of 16 lanes, then the rows before.
__device__ __forceinline__ int wave_sums_up(int x) {
  auto moved = [&](auto ctrl, auto rows) { return __builtin_amdgcn_update_dpp(0, x, decltype(ctrl)::value, decltype(rows)::value, 0xF, false); };
  using std::integral_constant;
  const integral_constant<int, 0xF> all;
  x += moved(integral_constant<int, 0x111>{}, all);              // from 1, 2, 4, 8 lanes below
  x += moved(integral_constant<int, 0x112>{}, all);
  x += moved(integral_constant<int, 0x114>{}, all);
  x += moved(integral_constant<int, 0x118>{}, all);
  x += moved(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});      // rows 1 and 3: the last lane of the row before
  x += moved(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});      // rows 2 and 3: lane 31
  return x;
}

// Exclusive sums over the workgroup's threads, and the totals, of N values.
template <int N>
__device__ __forceinline__ void plan_scan(int (&v)[N], int (&total)[N], int (*waves)[AS_PLAN_THREADS / 64]) {
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
    for (int w = 0; w < AS_PLAN_THREADS / 64; w++) {
      const int y = waves[i][w];
      before += w < wave ? y : 0;
      all += y;
    }
    total[i] = all;
    v[i] = before + x[i] - v[i];
  }
  __syncthreads();
}

// A line of segments cut into shares. A segment lies from `at` on: its start, then its pages. Where a share ends in it, it is cut at a whole
// block of pages; of the shares that it lies in, the first and the last may get none of them. Shares are longer than a start and a
// block, so those in between get some.
struct Line {
  int share, start, granule;
  float inverse;
  __device__ __forceinline__ int share_of(int at) const {
    int k = (int)((float)at * inverse);
    while (k * share > at) k--;
    while ((k + 1) * share <= at) k++;
    return k;
  }
  // pages of the segment that lie in the shares up to k
  __device__ __forceinline__ int up_to(int at, int pages, int k) const {
    const int room = (k + 1) * share - at - start;
    return room >= pages ? pages : max(room, 0) & ~(granule - 1);
  }
  // the first share that has pages of a segment of some, and how many have
  __device__ __forceinline__ int first(int at, int pages) const {
    const int k = share_of(at);
    return k + (up_to(at, pages, k) == 0);
  }
  __device__ __forceinline__ int pieces(int at, int pages) const {
    if (pages == 0) return 0;
    const int last = share_of(at + start + pages - 1), k0 = first(at, pages);
    return last - k0 + (last == k0 || up_to(at, pages, last - 1) < pages);
  }
};

// The last of count ascending values at or before x (the first is).
template <typename I>
__device__ __forceinline__ int last_up_to(const I* list, int count, int x) {
  int lo = 0, hi = count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((int)list[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(AS_PLAN_THREADS) attn_shared_plan_kernel(PlanCall c) {
  constexpr int N = OP_MAX_REQUESTS;
  // by group: first request, shared pages, first tile; by tile: place on the line of wide segments; by segment: place on the line of narrow
  // ones, first item, first partial row
  __shared__ unsigned short start[N + 1], tile0[N + 1], item0[2 * N + 1];
  __shared__ int lens[N], pages[N], wide_at[N + 1], narrow_at[2 * N + 1], part0[2 * N], waves[2][AS_PLAN_THREADS / 64];
  const int n = c.n, groups = c.groups, tid = threadIdx.x;
  if (tid == 0) *c.plan.sizes = c.tag;
  // groups whose starts do not lead from 0 to n in order are left aside: every request then reads all its pages for itself
  bool malformed = false;
  for (int g = tid; groups > 0 && g <= groups; g += AS_PLAN_THREADS) {
    const int s = c.group_starts[g];
    const bool ok = s >= 0 && s <= n && (g > 0 || s == 0) && (g < groups ? s <= c.group_starts[g + 1] : s == n);
    start[g] = (unsigned short)(ok ? s : 0);
    malformed |= !ok;
    if (g < groups) pages[g] = max(c.shared_lens[g], 0) / OP_PAGE;
  }
  for (int i = tid; i < n; i += AS_PLAN_THREADS) {               // -1: longer than its table, or negative
    const int l = c.lens[i];
    lens[i] = l < 0 || l > c.max_pages * (long long)OP_PAGE ? -1 : l;
  }
  const bool shares = !__syncthreads_or(malformed) && groups > 0;
  // a group shares what its shortest member holds in whole pages
  if (shares)
    for (int i = tid; i < n; i += AS_PLAN_THREADS) {
      int* p = &pages[last_up_to(start, groups, i)];
      const int held = max(lens[i], 0) / OP_PAGE;
      if (*reinterpret_cast<volatile int*>(p) > held) atomicMin(p, held);      // seldom: the caller knows what they share
    }
  __syncthreads();
  // requests of a tile: a group that fills more than the columns of one product takes wide ones
  auto per_tile = [&](int members) { return members * c.heads > AS_ROWS ? c.wide_requests : AS_TILE; };
  auto tiles_of = [&](int g) {
    const int members = start[g + 1] - start[g];
    return pages[g] == 0 ? 0 : members * c.heads > AS_ROWS ? (int)((members + c.wide_requests - 1) * (unsigned long long)c.wide_inverse >> 20) : 1;
  };
  const int gper = (groups + AS_PLAN_THREADS - 1) / AS_PLAN_THREADS, g0 = min(groups, tid * gper), g1 = min(groups, g0 + gper);
  int tiles[1] = {0}, all_tiles[1];
  for (int g = g0; g < g1; g++) {
    if (!shares || start[g + 1] - start[g] < 2) pages[g] = 0;
    tiles[0] += tiles_of(g);
  }
  plan_scan(tiles, all_tiles, waves);
  for (int g = g0; g < g1; g++) {
    tile0[g] = (unsigned short)tiles[0];
    tiles[0] += tiles_of(g);
  }
  __syncthreads();

  // segments: the tiles, then the requests' own pages
  const int T = all_tiles[0], segments = T + n;
  struct Tile { int group, request, rows; };          // its first request
  auto tile = [&](int s) {
    const int g = last_up_to(tile0, groups, s);                   // the last of several with that first tile: it has tiles
    const int per = per_tile(start[g + 1] - start[g]), r0 = start[g] + (s - tile0[g]) * per;
    return Tile{g, r0, min(per, start[g + 1] - r0) * c.heads};
  };
  auto rows_of = [&](int s) { return s < T ? tile(s).rows : c.heads; };
  auto held_pages = [&](int r) { return (max(lens[r], 0) + OP_PAGE - 1) / OP_PAGE; };
  auto cost_of = [&](int pages, int kind) { return pages > 0 ? pages + (kind ? AS_NARROW_START : AS_WIDE_START) : 0; };
  const int per = (segments + AS_PLAN_THREADS - 1) / AS_PLAN_THREADS, s0 = min(segments, tid * per), s1 = min(segments, s0 + per);
  int cost[2] = {0, 0}, all_cost[2];             // wide, narrow
  int rows = c.heads;                            // of the thread's last segment
  for (int s = s0; s < s1; s++) {
    int seg_pages;
    if (s < T) {
      const Tile t = tile(s);
      rows = t.rows; seg_pages = pages[t.group];
    } else {
      rows = c.heads; seg_pages = held_pages(s - T) - (shares ? pages[last_up_to(start, groups, s - T)] : 0);
    }
    part0[s] = seg_pages;                        // for now
    cost[rows <= AS_ROWS] += cost_of(seg_pages, rows <= AS_ROWS);
  }
  plan_scan(cost, all_cost, waves);
  const float wide_work = AS_WIDE_WEIGHT * all_cost[0];
  int wide = all_cost[0] == 0 ? 0 : (int)(c.slots * (wide_work / (wide_work + all_cost[1])) + 0.5f);
  wide = min(max(wide, (int)(all_cost[0] > 0)), c.slots - (all_cost[1] > 0));
  const int narrow = 4 * (c.slots - wide);
  auto line = [&](int total, int count, int start, int least, int granule) {
    const int share = max((total + max(count, 1) - 1) / max(count, 1), start + least);
    return Line{share, start, granule, 1.f / (float)share};
  };
  const int narrow_least = all_cost[1] < AS_LONG * segments || all_cost[1] < AS_LONG_SHARE * narrow ? AS_NARROW_LEAST : AS_LONG_LEAST;
  const Line lines[2] = {line(all_cost[0], wide, AS_WIDE_START, AS_WIDE_LEAST, 4), line(all_cost[1], narrow, AS_NARROW_START, narrow_least, 2)};
  int sums[2] = {0, 0}, all[2], at[2] = {cost[0], cost[1]};        // items (narrow ones in the upper half), partial rows
  int pieces = 0;                                // of the thread's last segment
  for (int s = s0; s < s1; s++) {
    if (per > 1) rows = rows_of(s);
    const int kind = rows <= AS_ROWS;
    pieces = lines[kind].pieces(at[kind], part0[s]);
    at[kind] += cost_of(part0[s], kind);
    sums[0] += kind ? pieces << 16 : pieces;
    sums[1] += pieces * rows;
  }
  plan_scan(sums, all, waves);
  at[0] = cost[0]; at[1] = cost[1];
  for (int s = s0; s < s1; s++) {
    if (per > 1) rows = rows_of(s);
    const int kind = rows <= AS_ROWS, seg_pages = part0[s];
    if (per > 1) pieces = lines[kind].pieces(at[kind], seg_pages);
    if (s < T) wide_at[s] = at[0];
    narrow_at[s] = at[1];
    item0[s] = (unsigned short)(kind ? (all[0] & 0xFFFF) + (sums[0] >> 16) : sums[0] & 0xFFFF);      // wide ones first
    part0[s] = sums[1];
    if (s >= T) {
      const int r = s - T;
      const bool alone = seg_pages == held_pages(r);              // shares nothing
      Parts* p = c.plan.parts + r;
      p->s_part = sums[1]; p->s_count = pieces; p->len = lens[r]; p->done = pieces == 1 && alone;
      if (alone) p->p_count = 0;
    } else {
      Parts* p = c.plan.parts + tile(s).request;
      for (int i = 0; i < rows; i += c.heads, p++) { p->p_part = sums[1] + i; p->p_step = rows; p->p_count = pieces; }
    }
    at[kind] += cost_of(seg_pages, kind);
    sums[0] += kind ? pieces << 16 : pieces;
    sums[1] += pieces * rows;
  }
  if (tid == 0) { wide_at[T] = all_cost[0]; narrow_at[segments] = all_cost[1]; }
  __syncthreads();
  // The items of a share, by a thread of its own. Neighbouring narrow shares go to different workgroups.
  for (int i = tid; i < wide + narrow; i += AS_PLAN_THREADS) {
    const int kind = i >= wide, k = kind ? i - wide : i, *places = kind ? narrow_at : wide_at, count_of = kind ? segments : T;
    const Line& l = lines[kind];
    const int begin = k * l.share, end = begin + l.share;
    Range r{};
    if (begin < all_cost[kind]) {
      for (int s = last_up_to(places, count_of, begin), from_at = places[s], to_at; s < count_of && from_at < end; s++, from_at = to_at) {
        to_at = places[s + 1];
        const int seg_pages = to_at - from_at - l.start;          // no more than 0: of the other kind, or without pages
        const int from = begin > from_at ? l.up_to(from_at, seg_pages, k - 1) : 0, to = l.up_to(from_at, seg_pages, k);
        if (from >= to) continue;
        const int piece = from == 0 ? 0 : k - l.first(from_at, seg_pages), item = item0[s] + piece;
        Item it;
        if (s < T) {
          const Tile t = tile(s);
          it = Item{t.request * c.heads, t.rows, start[t.group], from, to, seg_pages * OP_PAGE, part0[s] + piece * t.rows, 0};
        } else {
          const int q = s - T, held = held_pages(q), pg0 = held - seg_pages;
          const bool done = pg0 == 0 && to - from == held;        // a request without a shared part whose pages are all here
          it = Item{q * c.heads, c.heads, q, pg0 + from, pg0 + to, lens[q], done ? -1 : part0[s] + piece * c.heads, 1};
        }
        if (r.end == 0) {
          r.first = it;
          r.next = item + 1;
        } else {
          c.plan.items[item] = it;
        }
        r.end = item + 1;
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

// ---- the products
template <typename T> struct Mfma;
template <> struct Mfma<bf16> {
  typedef bf16x8 V;
  static __device__ __forceinline__ f32x16 mul(V a, V b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<f16> {
  typedef f16x8 V;
  static __device__ __forceinline__ f32x16 mul(V a, V b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

template <typename T>
struct AttnCall {
  const T* q; long long q_stride; const T* pool; T* out; long long out_stride; float* lse;
  const int* tables; long long table_stride;
  int n, n_q, n_kv, heads, pool_pages;
  float scale_log2e;
  bool q_vec, out_vec;                           // rows can be loaded 16 bytes, stored 8 bytes at a time
  unsigned long long tag;                        // what plan.sizes has to hold
  Plan plan;
};

// Eight probabilities for the second product, each in two numbers of the type: p without what the type drops, and p (1 + e) less that, which is above 0
// wherever p is, so that a V of infinity gives infinity and not inf - inf or 0 * inf. With u for half a step of the type (bf16 2^-8, fp16 2^-11) their sum is
// within 2 u (2 u + e) of p (1 + e); what reads the sums takes the factor out, and the
// output is rounded once, at the end: as far from 64 bits as that leaves any output. One number each, for half the second products, left outputs 1.04 to 1.11
// times as far and took, us a pass then / now: 8 requests on 1031 tokens (four layers) 54.9 / 56.0, 64 on 2048 (four) 116 / 119, 256 on 8192 (two) 164 / 186 (on
// another card 172 / 196), the larger shape's groups (two) 61 / 63.
// fp16 ends at 2^-24: its probabilities are lifted by 2^7, as far as AS_RISE leaves room for, and are held to 2^-31 of the reference's (the second number is above 0
// from 2^-22 on).
template <typename T> constexpr float AS_EXTRA = std::is_same<T, f16>::value ? 0x1p-9f : 0x1p-18f;            // e
template <typename T> constexpr float AS_LIFT = std::is_same<T, f16>::value ? 7.f : 0.f;                       // exponent
__device__ __forceinline__ void in_two(const f32x16& p, int at, bf16x8& first, bf16x8& rest) {
  u32x4 f;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const unsigned a = __float_as_uint(p[at + e]), b = __float_as_uint(p[at + e + 1]);
    f[e / 2] = __builtin_amdgcn_perm(b, a, 0x07060302);              // the upper halves
    rest[e] = (bf16)fmaf(p[at + e], 1.f + AS_EXTRA<bf16>, -__uint_as_float(a & 0xFFFF0000u));
    rest[e + 1] = (bf16)fmaf(p[at + e + 1], 1.f + AS_EXTRA<bf16>, -__uint_as_float(b & 0xFFFF0000u));
  }
  first = __builtin_bit_cast(bf16x8, f);
}
__device__ __forceinline__ void in_two(const f32x16& p, int at, f16x8& first, f16x8& rest) {
  typedef f16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const f16x2 f = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(p[at + e], p[at + e + 1]));
    const f16x2 r = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(fmaf(p[at + e], 1.f + AS_EXTRA<f16>, -(float)f[0]), fmaf(p[at + e + 1], 1.f + AS_EXTRA<f16>, -(float)f[1])));
    first[e] = f[0]; first[e + 1] = f[1];
    rest[e] = r[0]; rest[e + 1] = r[1];
  }
}

__device__ __forceinline__ float half_swap_max_f(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A value that the compiler derives nothing from earlier on: addresses made from it are not kept in registers over a whole loop of items.
__device__ __forceinline__ int fresh(int x) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(x));
#endif
  return x;
}

constexpr int AS_LDS_BASE = 1024;                // buffers filled by direct-to-LDS loads stay clear of address 0
template <int D>
constexpr int attn_shared_lds() { return AS_LDS_BASE + 4 * 2 * 2 * 16 * D * 2; }   // two blocks of K for each wave; two tiles of K and V^T; 128 rows of output

// ---- narrow items, one wave: blocks of two pages (32 tokens), K rows global -> LDS without passing through registers, V^T straight into the
// registers of its product, both two blocks ahead, with the waits of attn_decode.hip, which explains the order of the tokens.
// ONCE: pages that nobody else reads are fetched with the non-temporal hint.
template <typename T, int D, bool ONCE>
__device__ __forceinline__ void run_narrow(unsigned char* smem, const AttnCall<T>& c, const Item& it, int kvh) {
  typedef typename Mfma<T>::V V;
  constexpr int KSTEPS = D / 16, DB = D / 32;
  constexpr int ROWB = D * 2, CPR = D / 8, RPI = 64 / CPR, IPP = 16 / RPI;   // K row bytes, 16-byte chunks, rows per load, loads per page
  constexpr int PAGE_KB = 16 * ROWB, STAGE = 2 * PAGE_KB;
  constexpr int LOADS = 2 * IPP + 2 * DB;            // loads of a block: K to LDS, V^T to registers
  const int tid = fresh(threadIdx.x), lane = tid & 63, l32 = lane & 31, lh = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int npg = it.pg1 - it.pg0, nblk = (npg + 1) >> 1;
  const int nt = min(it.len, it.pg1 * OP_PAGE) - it.pg0 * OP_PAGE;           // tokens
  const int* table = c.tables + (long long)it.request * c.table_stride + it.pg0;
  const size_t head_elems = (size_t)2 * OP_PAGE * D;
  // Page numbers, 64 of them one per lane, and the next 64; past the end the last page again (fetched, left out). One outside the pool
  // is not followed: page 0 is read for it, and the rows come out as NaN.
  bool bad = false;
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
      for (int j = 0; j < IPP; j++) {
        unsigned char* to = kbuf + stage * STAGE + u * PAGE_KB + j * 1024;
        if constexpr (ONCE) load_to_lds16_nt(base[u] + ksrc[j], to); else load_to_lds16(base[u] + ksrc[j], to);
      }
    }
  };
  auto load_v = [&](u32x4 (&vr)[2][DB]) {
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int bb = 0; bb < DB; bb++) {
        const u32x4* from = reinterpret_cast<const u32x4*>(base[u] + (size_t)16 * D + (bb * 32 + l32) * 16 + lh * 8);
        if constexpr (ONCE) vr[u][bb] = __builtin_nontemporal_load(from); else vr[u][bb] = *from;
      }
  };

  // Q^T operand: column l32 is row l32 of the item
  V qf[KSTEPS];
  const int vrow = it.row0 + min(l32, it.rows - 1), request = vrow / c.heads, head = kvh * c.heads + vrow % c.heads;
  {
    const T* q = c.q + (long long)request * c.q_stride + head * D + lh * 8;
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
    const int t_base = b * 32 + 8 * lh;               // register r: page r >> 3 of the pair, token 8 * half + (r & 7)
    if (b * 32 + 32 > nt) {                           // wave-uniform: some tokens of the block are left out
#pragma unroll
      for (int r = 0; r < 16; r++)
        if (t_base + (r >> 3) * 16 + (r & 7) >= nt) s[r] = -INFINITY;
      // what lies in a page behind the context may be anything, NaN included: 0 * V must be 0
#pragma unroll
      for (int u = 0; u < 2; u++)
#pragma unroll
        for (int bb = 0; bb < DB; bb++) {
          V v = __builtin_bit_cast(V, vr[u][bb]);
#pragma unroll
          for (int e = 0; e < 8; e++)
            if (t_base + u * 16 + e >= nt) v[e] = (T)0.f;
          vr[u][bb] = __builtin_bit_cast(u32x4, v);
        }
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
    if (it.part < 0) {
      T* out = c.out + (long long)request * c.out_stride + head * D + 4 * lh;
      const float f = 1.f / ((1.f + AS_EXTRA<T>) * l_run);
#pragma unroll
      for (int bb = 0; bb < DB; bb++)
#pragma unroll
        for (int r4 = 0; r4 < 4; r4++) {
          typedef T T4 __attribute__((ext_vector_type(4)));
          T4 v;
#pragma unroll
          for (int e = 0; e < 4; e++) v[e] = (T)(o[bb][4 * r4 + e] * f);
          T* to = out + bb * 32 + 8 * r4;
          if (c.out_vec) *reinterpret_cast<T4*>(to) = v;
          else
#pragma unroll
            for (int e = 0; e < 4; e++) to[e] = v[e];
        }
      if (lh == 0 && c.lse) c.lse[(long long)request * c.n_q + head] = LN2 * (m2 + __builtin_amdgcn_logf(l_run));
    } else {
      const size_t row = (size_t)(it.part + l32) * c.n_kv + kvh;
      float* out = c.plan.outs + row * D + 4 * lh;
#pragma unroll
      for (int bb = 0; bb < DB; bb++)
#pragma unroll
        for (int r4 = 0; r4 < 4; r4++) *reinterpret_cast<f32x4*>(out + bb * 32 + 8 * r4) = f32x4{o[bb][4 * r4], o[bb][4 * r4 + 1], o[bb][4 * r4 + 2], o[bb][4 * r4 + 3]};
      if (lh == 0) c.plan.stats[row] = f32x2{m2, l_run};
    }
  }
}

// ---- wide items, a workgroup: every wave takes 32 rows over all the pages. Tiles of four pages go global -> LDS, two stages deep, a page
// a wave; products, order of the tokens and softmax as in attn_prefill.hip, whose queries lie in a row where these come from any request.

template <typename T, int D>
__device__ __forceinline__ void run_wide(unsigned char* smem, const AttnCall<T>& c, const Item& it, int kvh) {
  typedef typename Mfma<T>::V V;
  constexpr int KSTEPS = D / 16, DB = D / 32;
  constexpr int ROWB = D * 2, CPR = D / 8, RPI = 64 / CPR, IPP = 16 / RPI;     // K row bytes, 16-byte chunks, rows per load, loads per page
  constexpr int PAGE = 16 * ROWB, TILE = 4 * PAGE, STAGE = 2 * TILE;           // bytes of a K (or V^T) page, tile; of a stage
  const int tid = fresh(threadIdx.x), lane = tid & 63, l32 = lane & 31, lh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int npg = it.pg1 - it.pg0, tiles = (npg + 3) >> 2;
  const int* table = c.tables + (long long)it.request * c.table_stride + it.pg0;
  const int my_rows = min(it.rows - wave * 32, 32);                            // none or fewer: the wave only fetches

  V qf[KSTEPS];
  {
    const int v = it.row0 + min(wave * 32 + l32, it.rows - 1);
    const T* q = c.q + (long long)(v / c.heads) * c.q_stride + (kvh * c.heads + v % c.heads) * D + 8 * lh;
#pragma unroll
    for (int j = 0; j < KSTEPS; j++) {
      if (c.q_vec) qf[j] = *reinterpret_cast<const V*>(q + 16 * j);
      else
#pragma unroll
        for (int e = 0; e < 8; e++) qf[j][e] = q[16 * j + e];
    }
  }
  // This wave's page of tile kt; past the last page that page again, whose products are left out.
  bool bad = false;
  const size_t page_stride = (size_t)c.n_kv * 2 * OP_PAGE * D;
  const T* pool_h = c.pool + (size_t)kvh * 2 * OP_PAGE * D;
  auto page_id = [&](int kt) {
    const int page = table[min(kt * 4 + wave, npg - 1)];
    const bool out = (unsigned)page >= (unsigned)c.pool_pages;
    bad |= out;
    return out ? 0 : page;
  };
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
  const int k_row = (l32 >> 4) * PAGE + tok * ROWB;
  int k_slot[KSTEPS];
#pragma unroll
  for (int j = 0; j < KSTEPS; j++) k_slot[j] = k_row + ((2 * j + lh) ^ (D == 128 ? tok : (tok >> 1) & 7)) * 16;
  const int v_lane = TILE + l32 * 32 + lh * 16;          // V^T operand: d row l32 of a 32-row block, tokens 8 lh .. of a page

  f32x16 o[DB];
#pragma unroll
  for (int b = 0; b < DB; b++)
#pragma unroll
    for (int r = 0; r < 16; r++) o[b][r] = 0.f;
  float m_ref = -INFINITY, l_run = 0.f;
  issue(0, page_id(0));
  int next_page = page_id(1);
  auto tile = [&](int kt, auto whole) {
    const unsigned char* st = arena + (kt & 1) * STAGE;
    const int here = decltype(whole)::value ? 4 : npg - kt * 4;                // pages of the tile
    f32x16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; kb++)
#pragma unroll
      for (int r = 0; r < 16; r++) s[kb][r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
    {
      V kf[2][2];
#pragma unroll
      for (int kb = 0; kb < 2; kb++) kf[0][kb] = *reinterpret_cast<const V*>(st + kb * 2 * PAGE + k_slot[0]);
#pragma unroll
      for (int j = 0; j < KSTEPS; j++) {
        const int a = j & 1, b = a ^ 1;
        if (j + 1 < KSTEPS) {
#pragma unroll
          for (int kb = 0; kb < 2; kb++) kf[b][kb] = *reinterpret_cast<const V*>(st + kb * 2 * PAGE + k_slot[j + 1]);
        }
#pragma unroll
        for (int kb = 0; kb < 2; kb++) s[kb] = Mfma<T>::mul(kf[a][kb], qf[j], s[kb]);
      }
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
      for (int j = 0; j + 1 < KSTEPS; j++) {
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
    }
    V vf[2][DB];                                           // first V^T operands: in flight during the softmax arithmetic
#pragma unroll
    for (int b = 0; b < DB; b++) vf[0][b] = *reinterpret_cast<const V*>(st + v_lane + b * 1024);
    if constexpr (!decltype(whole)::value) {
#pragma unroll
      for (int kb = 0; kb < 2; kb++)
#pragma unroll
        for (int r = 0; r < 16; r++)
          if (2 * kb + (r >> 3) >= here) s[kb][r] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; kb++)
#pragma unroll
      for (int r = 0; r < 16; r++) mx = fmaxf(mx, s[kb][r]);
    mx = half_swap_max_f(mx);
    // The reference moves when a score has outgrown it by 2^8, by which probabilities and their sums may then exceed 1: two numbers of the type, and 32 bits, hold
    // them as well there. Following every new maximum, 256 requests on 8192 tokens (two layers) took 193 instead of 186 us, with outputs as near to 64 bits.
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
    for (int kb = 0; kb < 2; kb++)
#pragma unroll
      for (int r = 0; r < 16; r++) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[kb][r], c.scale_log2e, nm));
        s[kb][r] = p;
        rs += p;
      }
    l_run += rs;                                                               // this half's keys; halves are added at the end
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const int a = g & 1, b2 = a ^ 1;
      if (g + 1 < 4) {
#pragma unroll
        for (int b = 0; b < DB; b++) vf[b2][b] = *reinterpret_cast<const V*>(st + v_lane + (g + 1) * PAGE + b * 1024);
      }
      V pb, pr;
      in_two(s[g >> 1], 8 * (g & 1), pb, pr);
      if (decltype(whole)::value || g < here) {
#pragma unroll
        for (int b = 0; b < DB; b++) o[b] = Mfma<T>::mul(vf[a][b], pb, o[b]);
#pragma unroll
        for (int b = 0; b < DB; b++) o[b] = Mfma<T>::mul(vf[a][b], pr, o[b]);
      }
    }
    if constexpr (decltype(whole)::value) {
#pragma unroll
      for (int g = 0; g + 1 < 4; g++) {
        __builtin_amdgcn_sched_group_barrier(0x100, DB, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 2 * DB, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 2 * DB, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto landed = [&](int kt) {                              // every wave waits for its own page, and nobody reads the other stage any more
    wait_vmem<0>();
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
    if (kt + 1 < tiles) {
      issue((kt + 1) & 1, next_page);
      next_page = page_id(kt + 2);
    }
  };
  const int whole = npg >> 2;
  for (int kt = 0; kt < whole; kt++) {
    landed(kt);
    if (my_rows > 0) tile(kt, std::true_type{});           // wave-uniform
  }
  if (whole < tiles) {
    landed(whole);
    if (my_rows > 0) tile(whole, std::false_type{});
  }
  l_run += __shfl_xor(l_run, 32, 64);
  if (__syncthreads_or(bad)) l_run = NAN;                // LDS now takes the output
  if (my_rows > 0) {
    // whole rows through LDS: 16-byte chunks, swizzled by row
    constexpr int OROWB = D * 4, OCPR = OROWB / 16, ORPI = 64 / OCPR;
    unsigned char* buf = arena + wave * 32 * OROWB;
    const int lane = fresh(tid & 63), l32 = lane & 31, lh = lane >> 5;
#pragma unroll
    for (int b = 0; b < DB; b++)
#pragma unroll
      for (int r4 = 0; r4 < 4; r4++)
        *reinterpret_cast<f32x4*>(buf + l32 * OROWB + ((b * 8 + 2 * r4 + lh) ^ (l32 % 16)) * 16) = f32x4{o[b][4 * r4], o[b][4 * r4 + 1], o[b][4 * r4 + 2], o[b][4 * r4 + 3]};
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int r0 = lane / OCPR, ch = lane % OCPR, part = it.part + wave * 32;
#pragma unroll
    for (int i = 0; i < 32 / ORPI; i++) {
      const int r = i * ORPI + r0;
      const f32x4 v = *reinterpret_cast<const f32x4*>(buf + r * OROWB + (ch ^ (r % 16)) * 16);
      if (r < my_rows) *reinterpret_cast<f32x4*>(c.plan.outs + ((size_t)(part + r) * c.n_kv + kvh) * D + ch * 4) = v;
    }
    if (lane < my_rows) c.plan.stats[(size_t)(part + lane) * c.n_kv + kvh] = f32x2{fmaf(m_ref, c.scale_log2e, -AS_LIFT<T>), l_run};
  }
  __syncthreads();                                       // before the next item's K lands there
}

template <typename T, int D>
__global__ void __launch_bounds__(256, 2) attn_shared_kernel(AttnCall<T> c) {
  __shared__ __align__(16) unsigned char smem[attn_shared_lds<D>()];
  // With 8 KV heads a head's workgroups are all on one XCD: the tiles of a prefix find each other's pages in its L2.
  const int slot = blockIdx.x / c.n_kv, kvh = blockIdx.x % c.n_kv;
  const Range r = c.plan.ranges[slot * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)];
  if (*c.plan.sizes != c.tag || r.first.rows == 0) return;
  Item it = r.first;
  for (int i = r.next;; i++) {
    if (it.rows > AS_ROWS) run_wide<T, D>(smem, c, it, kvh);
    else if (it.once) run_narrow<T, D, true>(smem, c, it, kvh);
    else run_narrow<T, D, false>(smem, c, it, kvh);
    if (i >= r.end) break;
    it = c.plan.items[i];
  }
}

// Joins the partial results of a (request, query head): WAVES waves each, a lane four elements of every 256 / D-th part (of a wave's share).
template <typename T, int D, int WAVES>
__global__ void __launch_bounds__(256) attn_shared_join_kernel(AttnCall<T> c) {
  constexpr int LANES = D / 4, APART = 64 / LANES * WAVES;       // lanes of a part, parts side by side
  __shared__ f32x4 sums[WAVES > 1 ? WAVES : 1][LANES];
  __shared__ float ls[WAVES];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = WAVES > 1 ? blockIdx.x : blockIdx.x * 4 + wave;
  if (at >= c.n * c.n_q) return;
  const int r = at / c.n_q, head = at % c.n_q, kvh = head / c.heads, h = head % c.heads;
  Parts p = c.plan.parts[r];
  if (*c.plan.sizes != c.tag) p = Parts{0, 0, 0, 0, 0, -1, 0, 0};
  if (p.done) return;
  const int count = p.len < 0 ? 0 : p.p_count + p.s_count;
  auto row_of = [&](int j) { return (size_t)((j < p.p_count ? p.p_part + j * p.p_step : p.s_part + (j - p.p_count) * c.heads) + h) * c.n_kv + kvh; };
  float m = -INFINITY;
  for (int j = lane; j < count; j += 64) m = fmaxf(m, c.plan.stats[row_of(j)][0]);
  m = wave_max(m);
  float l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const int first = (WAVES > 1 ? wave * (64 / LANES) : 0) + lane / LANES, e4 = lane % LANES * 4;
#pragma unroll 4
  for (int j = first; j < count; j += APART) {
    const size_t row = row_of(j);
    const f32x2 st = c.plan.stats[row];
    const f32x4 x = *reinterpret_cast<const f32x4*>(c.plan.outs + row * D + e4);
    const float w = st[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[0] - m);
    l += st[0] == -INFINITY ? st[1] : st[1] * w;                 // 0 of a part without scores above -inf, or NaN
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] += x[e] * w;
  }
#pragma unroll
  for (int s = LANES; s < 64; s <<= 1) {
    l += __shfl_xor(l, s, 64);
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] += __shfl_xor(o[e], s, 64);
  }
  if constexpr (WAVES > 1) {
    if (lane < LANES) sums[wave][lane] = o;
    if (lane == 0) ls[wave] = l;
    __syncthreads();
    if (wave > 0) return;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; w++) l += ls[w];
    if (lane < LANES) {
      o = sums[0][lane];
#pragma unroll
      for (int w = 1; w < WAVES; w++)
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] += sums[w][lane][e];
    }
  }
  if (lane < LANES) {
    T* out = c.out + (long long)r * c.out_stride + head * D + e4;
    const bool none = p.len == 0;                      // nothing to attend to: zeros, and the logarithm of an empty sum
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 v;
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = (T)(p.len < 0 ? NAN : none ? 0.f : o[e] / ((1.f + AS_EXTRA<T>) * l));
    if (c.out_vec) *reinterpret_cast<T4*>(out) = v;
    else
#pragma unroll
      for (int e = 0; e < 4; e++) out[e] = v[e];
    if (lane == 0 && c.lse) c.lse[(long long)r * c.n_q + head] = p.len < 0 ? NAN : none ? -INFINITY : LN2 * (m + __builtin_amdgcn_logf(l));
  }
}

template <typename T, int D>
hipError_t launch_attn(hipStream_t s, const AttnCall<T>& c) {
  hipError_t e = launch(attn_shared_kernel<T, D>, dim3(slots_of(c.n_kv) * c.n_kv), dim3(256), 0, s, c);
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)c.n * c.n_q;
  if (rows <= AS_JOIN_ROWS) return launch(attn_shared_join_kernel<T, D, 4>, dim3((unsigned)rows), dim3(256), 0, s, c);
  return launch(attn_shared_join_kernel<T, D, 1>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, c);
}

bool sizes_ok(int n, int n_q, int n_kv, int d) {
  return n >= 0 && n <= OP_MAX_REQUESTS && n_kv >= 1 && n_kv <= AS_SLOTS / 2 && n_q >= n_kv && n_q % n_kv == 0 && n_q / n_kv <= AS_ROWS && (d == 64 || d == 128);
}
// The batch's description, without what a call of one layer adds.
int check_batch(const sts_attn_batch* b, Plan* plan) {
  if (!b || (b->dtype != STS_BF16 && b->dtype != STS_F16) || !sizes_ok(b->n_requests, b->n_q, b->n_kv, b->d)) return STS_EINVAL;
  if (b->n_groups < 0 || b->n_groups > b->n_requests || b->pool_pages < 0 || b->max_pages < 0 || b->max_pages > (1 << 26) || (int64_t)b->n_requests * b->max_pages > (1 << 28) || b->table_stride < b->max_pages) return STS_EINVAL;
  if (b->n_requests == 0) return STS_OK;
  if (!b->lens || (b->max_pages > 0 && !b->tables) || (b->n_groups > 0 && (!b->group_starts || !b->shared_lens))) return STS_EINVAL;
  if (!b->workspace || !aligned(b->workspace, 256)) return STS_EINVAL;
  if ((int64_t)lay_out(reinterpret_cast<unsigned char*>(b->workspace), b->n_requests, b->n_q, b->n_kv, b->d, plan) > b->workspace_bytes) return STS_EINVAL;
  return STS_OK;
}

}  // namespace
}  // namespace sts

using namespace sts;

extern "C" int64_t sts_attn_shared_workspace(int32_t n_requests, int32_t n_q, int32_t n_kv, int32_t d) {
  if (!sizes_ok(n_requests, n_q, n_kv, d)) return -1;
  return (int64_t)lay_out(nullptr, n_requests, n_q, n_kv, d, nullptr);
}

extern "C" int sts_op_attn_shared_plan(const sts_attn_batch* b, void* stream) {
  Plan plan{};
  const int rc = check_batch(b, &plan);
  if (rc != STS_OK || b->n_requests == 0) return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  const int n = b->n_requests, slots = slots_of(b->n_kv);
  const int heads = b->n_q / b->n_kv, wide_requests = AS_TILE / heads;
  const PlanCall c{sizes_tag(*b), n, b->n_groups, heads, slots, b->max_pages, wide_requests, ((1u << 20) + wide_requests - 1) / wide_requests, b->lens, b->group_starts, b->shared_lens, plan};
  return op_result(launch(attn_shared_plan_kernel, dim3(1), dim3(AS_PLAN_THREADS), 0, s, c));
}

template <typename T>
static int attn_shared(const sts_attn_batch* b, const Plan& plan, const void* q, int64_t q_stride, const void* pool, void* out, int64_t out_stride, float* lse, float scale, hipStream_t s) {
  const bool q_vec = aligned(q, 16) && q_stride % 8 == 0, out_vec = aligned(out, 8) && out_stride % 4 == 0;
  const AttnCall<T> c{reinterpret_cast<const T*>(q), q_stride, reinterpret_cast<const T*>(pool), reinterpret_cast<T*>(out), out_stride, lse, b->tables, b->table_stride,
                      b->n_requests, b->n_q, b->n_kv, b->n_q / b->n_kv, b->pool_pages, scale * LOG2E, q_vec, out_vec, sizes_tag(*b), plan};
  return op_result(b->d == 128 ? launch_attn<T, 128>(s, c) : launch_attn<T, 64>(s, c));
}

extern "C" int sts_op_attn_shared(const sts_attn_batch* b, const void* q, int64_t q_stride, const void* pool, void* out, int64_t out_stride, float* lse, float scale, void* stream) {
  Plan plan{};
  const int rc = check_batch(b, &plan);
  if (rc != STS_OK || b->n_requests == 0) return rc;
  const int64_t row = (int64_t)b->n_q * b->d;
  if (!q || !out || !aligned(q, 2) || !aligned(out, 2) || !pool || !aligned(pool, 16) || b->pool_pages < 1 || (b->n_requests > 1 && (q_stride < row || out_stride < row))) return STS_EINVAL;
  if (!(scale >= 0.f) || scale > 1e30f) return STS_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  const float sc = scale == 0.f ? 1.f / sqrtf((float)b->d) : scale;
  return b->dtype == STS_BF16 ? attn_shared<bf16>(b, plan, q, q_stride, pool, out, out_stride, lse, sc, s) : attn_shared<f16>(b, plan, q, q_stride, pool, out, out_stride, lse, sc, s);
}
