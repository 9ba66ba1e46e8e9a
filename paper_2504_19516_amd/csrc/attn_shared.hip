// Decode attention for requests that share the beginning of their contexts (Section 3.5.1's pages in several block tables): a
// group's shared pages are read once for all its requests, every request's own pages once for it.
//
//   o_r = sum_t p_t v_t / l,   p_t = 2^(scale log2(e) q_r . k_t - m),   l = sum_t p_t,   over the tokens t < len_r
//
// computed in parts of the token range, each with its own maximum m, that a second kernel joins:
//   m = max m_j,  l = sum l_j 2^(m_j - m),  o = sum o_j 2^(m_j - m) / l
//
// A segment is a token range with the rows that read it: the shared pages of a group with a tile of its requests, or the own pages of
// one request. A request brings n_q / n_kv rows (the query heads of a KV head) to the products, so a tile of shared pages fills the matrix cores'
// columns that a single request leaves empty. The plan, made once a step on the device from the lengths, lays the segments of a KV
// head end to end, weighs them (pages, and the start and end of a segment), and cuts the line into equal shares, one for each workgroup
// of a KV head: a long context is shared by many workgroups, short ones are strung together in one.
//
// A workgroup's 4 waves take blocks of two pages (32 tokens) in turns, K rows global -> LDS without passing through registers, V^T
// straight into the registers of its product, both two blocks ahead, as attn_decode.hip does and explains; the rows of the block's
// product are here any (request, head) pairs instead of the heads of one request. The waves' partial results meet in LDS.
#include <algorithm>

#include "device_ops.h"

namespace sts {
namespace {

constexpr int AS_ROWS = 32;                     // rows of a segment: columns of a product
constexpr int AS_SLOTS = 512;                   // workgroups of a launch: two on each CU
constexpr int AS_PLAN_THREADS = 1024;
// Weights: a page read, and the start and end of a segment, in sixteenths of a page.
constexpr int AS_PAGE_COST = 16, AS_START_COST = 96, AS_MIN_SHARE = AS_START_COST + 8 * AS_PAGE_COST;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// A piece of a segment: rows row0 .. row0 + rows - 1 (request * heads of a group + head) over the pages [pg0, pg1) of a request's
// table, tokens from len on left out. part: number of its first row's partial result, -1: it finishes its rows.
struct Item { int row0, rows, request, pg0, pg1, len, part, slot; };
// Where a request's partial results are: head h in p_part + j * p_step + h, j < p_count, and s_part + j * heads + h, j < s_count.
// done: its one piece finishes it. len < 0: its length is out of range.
struct Parts { int p_part, p_step, p_count, s_part, s_count, len, done, pad; };
struct Plan {
  int* slot_first;                               // [slots + 1]: first item of each
  Item* items;
  Parts* parts;                                  // [n_requests]
  f32x2* stats;                                  // [partial row][kv head]: maximum (log2 units), sum
  float* outs;                                   // [partial row][kv head][d]
};

int slots_of(int n_kv) { return std::max(1, AS_SLOTS / n_kv); }
int max_items(int n, int n_kv) { return 2 * n + slots_of(n_kv); }           // pieces: one a segment and one a cut
int64_t max_part_rows(int n, int n_q, int n_kv) { return (int64_t)2 * n * (n_q / n_kv) + (int64_t)slots_of(n_kv) * AS_ROWS; }

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
// The workspace's parts behind each other; returns its size.
size_t lay_out(unsigned char* base, int n, int n_q, int n_kv, int d, Plan* p) {
  size_t at = 0;
  auto take = [&](size_t bytes) { unsigned char* q = base + at; at += up256(bytes); return q; };
  const size_t rows = (size_t)max_part_rows(n, n_q, n_kv) * n_kv;
  Plan q;
  q.slot_first = reinterpret_cast<int*>(take((slots_of(n_kv) + 1) * sizeof(int)));
  q.items = reinterpret_cast<Item*>(take(max_items(n, n_kv) * sizeof(Item)));
  q.parts = reinterpret_cast<Parts*>(take(n * sizeof(Parts)));
  q.stats = reinterpret_cast<f32x2*>(take(rows * sizeof(f32x2)));
  q.outs = reinterpret_cast<float*>(take(rows * d * sizeof(float)));
  if (p) *p = q;
  return at;
}

// ---- the plan: one workgroup
struct PlanCall { int n, groups, heads, slots, max_pages; const int *lens, *group_starts, *shared_lens; Plan plan; };

// Exclusive sums over the workgroup's threads, and the totals.
__device__ __forceinline__ long long plan_scan(long long v, long long* waves, long long* total) {
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
  for (int w = 0; w < AS_PLAN_THREADS / 64; w++) {
    if (w < wave) before += waves[w];
    all += waves[w];
  }
  __syncthreads();
  *total = all;
  return before + x - v;
}

__global__ void __launch_bounds__(AS_PLAN_THREADS) attn_shared_plan_kernel(PlanCall c) {
  extern __shared__ int lds[];
  __shared__ long long waves[AS_PLAN_THREADS / 64];
  __shared__ int malformed;
  const int n = c.n, tid = threadIdx.x, per_tile = AS_ROWS / c.heads;        // requests of a tile
  int *start = lds, *pages = start + n + 1, *tile0 = pages + n;              // by group: first request, shared pages, first tile
  int* slot_at = tile0 + n + 1;                  // [slots + 1]
  if (tid == 0) malformed = 0;
  __syncthreads();
  // groups whose starts do not lead from 0 to n in order are left aside: every request then reads all its pages for itself
  const int groups = c.groups;
  for (int g = tid; groups > 0 && g <= groups; g += AS_PLAN_THREADS) {
    const int s = c.group_starts[g];
    start[g] = s;
    const bool ok = s >= 0 && s <= n && (g > 0 || s == 0) && (g < groups ? s <= c.group_starts[g + 1] : s == n);
    if (!ok) malformed = 1;
    if (g < groups) pages[g] = max(c.shared_lens[g], 0) / OP_PAGE;
  }
  auto len = [&](int r) {                        // -1: longer than its table, or negative
    const int l = c.lens[r];
    return l < 0 || l > c.max_pages * (long long)OP_PAGE ? -1 : l;
  };
  __syncthreads();
  const bool shares = groups > 0 && !malformed;
  auto group_of = [&](int r) {
    int lo = 0, hi = groups;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= r) lo = mid; else hi = mid;
    }
    return lo;
  };
  // a group shares what its shortest member holds in whole pages
  if (shares)
    for (int i = tid; i < n; i += AS_PLAN_THREADS) atomicMin(&pages[group_of(i)], max(len(i), 0) / OP_PAGE);
  __syncthreads();
  // tiles of each group
  const int gper = (groups + AS_PLAN_THREADS - 1) / AS_PLAN_THREADS, g0 = min(groups, tid * gper), g1 = min(groups, g0 + gper);
  long long tiles = 0, all_tiles = 0;
  for (int g = g0; g < g1; g++) {
    if (!shares || start[g + 1] - start[g] < 2) pages[g] = 0;
    tiles += pages[g] > 0 ? (start[g + 1] - start[g] + per_tile - 1) / per_tile : 0;
  }
  tiles = plan_scan(tiles, waves, &all_tiles);
  for (int g = g0; g < g1; g++) {
    tile0[g] = (int)tiles;
    tiles += pages[g] > 0 ? (start[g + 1] - start[g] + per_tile - 1) / per_tile : 0;
  }
  if (tid == 0) tile0[groups] = (int)all_tiles;
  for (int k = tid; k <= c.slots; k += AS_PLAN_THREADS) slot_at[k] = 0x7FFFFFFF;
  __syncthreads();

  // segments: the tiles, then the requests' own pages
  const int T = (int)all_tiles, segments = T + n;
  struct Segment { int row0, rows, request, pg0, pg1, len; };
  auto segment = [&](int s) {
    Segment x;
    if (s < T) {
      int lo = 0, hi = groups;                   // the last group whose first tile is at or before s; it has tiles
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (tile0[mid] <= s) lo = mid; else hi = mid;
      }
      const int r0 = start[lo] + (s - tile0[lo]) * per_tile;
      x = {r0 * c.heads, min(per_tile, start[lo + 1] - r0) * c.heads, start[lo], 0, pages[lo], pages[lo] * OP_PAGE};
    } else {
      const int r = s - T, l = max(len(r), 0);
      x = {r * c.heads, c.heads, r, shares ? pages[group_of(r)] : 0, (l + OP_PAGE - 1) / OP_PAGE, l};
    }
    return x;
  };
  auto cost_of = [&](const Segment& x) { return x.pg1 > x.pg0 ? AS_START_COST + (long long)(x.pg1 - x.pg0) * AS_PAGE_COST : 0; };
  const int per = (segments + AS_PLAN_THREADS - 1) / AS_PLAN_THREADS, s0 = min(segments, tid * per), s1 = min(segments, s0 + per);
  long long cost = 0, all_cost;
  for (int s = s0; s < s1; s++) cost += cost_of(segment(s));
  const long long cost0 = plan_scan(cost, waves, &all_cost);
  const long long share = max((all_cost + c.slots - 1) / c.slots, (long long)AS_MIN_SHARE);
  // f(slot, first page, last page) for the pieces of a segment that lies from `at` on the line
  auto pieces = [&](const Segment& x, long long at, auto f) {
    const long long end = at + cost_of(x);
    if (end == at) return;
    int from = x.pg0;
    for (long long k = at / share; from < x.pg1; k++) {
      const long long cut = (k + 1) * share;     // pages up to the end of slot k, whole blocks of two
      const long long up = (cut - at - AS_START_COST) / AS_PAGE_COST;
      int to = cut >= end ? x.pg1 : x.pg0 + (int)max(up, 0ll) / 2 * 2;
      to = min(max(to, from), x.pg1);
      if (to > from) f((int)k, from, to);
      from = to;
    }
  };
  long long at = cost0, count = 0, rows = 0, all_items, all_rows;
  for (int s = s0; s < s1; s++) {
    const Segment x = segment(s);
    pieces(x, at, [&](int, int, int) { count++; rows += x.rows; });
    at += cost_of(x);
  }
  count = plan_scan(count, waves, &all_items);
  rows = plan_scan(rows, waves, &all_rows);
  at = cost0;
  for (int s = s0; s < s1; s++) {
    const Segment x = segment(s);
    int mine = 0;
    pieces(x, at, [&](int, int, int) { mine++; });
    const bool own = s >= T;
    const bool done = own && mine == 1 && x.pg0 == 0;
    const int part = (int)rows;
    pieces(x, at, [&](int slot, int from, int to) {
      c.plan.items[count] = Item{x.row0, x.rows, x.request, from, to, x.len, done ? -1 : (int)rows, slot};
      atomicMin(&slot_at[slot], (int)count);
      count++;
      rows += x.rows;
    });
    if (own) {
      Parts* p = c.plan.parts + x.request;
      p->s_part = part; p->s_count = mine; p->len = len(x.request); p->done = done;
      if (x.pg0 == 0) p->p_count = 0;
    } else {
      for (int i = 0; i < x.rows; i += c.heads) {
        Parts* p = c.plan.parts + (x.row0 + i) / c.heads;
        p->p_part = part + i; p->p_step = x.rows; p->p_count = mine;
      }
    }
    at += cost_of(x);
  }
  __syncthreads();
  // a slot without items begins where the next one does
  for (int k = tid; k <= c.slots; k += AS_PLAN_THREADS) {
    int j = k;
    while (j < c.slots && slot_at[j] == 0x7FFFFFFF) j++;
    c.plan.slot_first[k] = j < c.slots ? slot_at[j] : (int)all_items;
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
  bool q_vec;                                    // q's rows can be loaded 16 bytes at a time
  Plan plan;
};

__device__ __forceinline__ float half_swap_max_f(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

constexpr int AS_LDS_BASE = 1024;                // buffers filled by direct-to-LDS loads stay clear of address 0
template <int D>
constexpr int attn_shared_lds() { return AS_LDS_BASE + std::max(4 * 2 * 2 * 16 * D * 2, 4 * AS_ROWS * (D + 2) * 4); }

template <typename T, int D>
__device__ __forceinline__ void run_item(unsigned char* smem, const AttnCall<T>& c, const Item& it, int kvh) {
  typedef typename Mfma<T>::V V;
  constexpr int KSTEPS = D / 16, DB = D / 32;
  constexpr int ROWB = D * 2, CPR = D / 8, RPI = 64 / CPR, IPP = 16 / RPI;   // K row bytes, 16-byte chunks, rows per load, loads per page
  constexpr int PAGE_KB = 16 * ROWB, STAGE = 2 * PAGE_KB;
  constexpr int LOADS = 2 * IPP + 2 * DB;            // loads of a block: K to LDS, V^T to registers
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, lh = lane >> 5;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int npg = it.pg1 - it.pg0, nblk = (npg + 1) >> 1;
  const int nt = min(it.len, it.pg1 * OP_PAGE) - it.pg0 * OP_PAGE;           // tokens
  const int* table = c.tables + (long long)it.request * c.table_stride + it.pg0;
  const size_t head_elems = (size_t)2 * OP_PAGE * D;
  // Page numbers, 64 of them one per lane, and the next 64; past the end the last page again (fetched, left out). One outside the pool
  // is not followed: page 0 is read for it, and the rows come out as NaN.
  bool bad = false;
  auto load_pages = [&](int window) {
    const int page = npg > 0 ? table[min(window * 64 + lane, npg - 1)] : 0;
    const bool out = (unsigned)page >= (unsigned)c.pool_pages;
    bad |= out;
    return out ? 0 : page;
  };
  int window = 0, pages_now = load_pages(0), pages_next = load_pages(1);
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
      for (int j = 0; j < IPP; j++) load_to_lds16(base[u] + ksrc[j], kbuf + stage * STAGE + u * PAGE_KB + j * 1024);
    }
  };
  auto load_v = [&](u32x4 (&vr)[2][DB]) {
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
      for (int bb = 0; bb < DB; bb++) vr[u][bb] = *reinterpret_cast<const u32x4*>(base[u] + (size_t)16 * D + (bb * 32 + l32) * 16 + lh * 8);
  };

  // Q^T operand: column l32 is row l32 of the item
  V qf[KSTEPS];
  const int vrow = it.row0 + min(l32, it.rows - 1);
  {
    const T* q = c.q + (long long)(vrow / c.heads) * c.q_stride + (kvh * c.heads + vrow % c.heads) * D + lh * 8;
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
    const bool tail = b * 32 + 32 > nt;               // wave-uniform: some tokens of the block are left out
    if (tail) {
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
    const float nm = m_ref == -INFINITY ? 0.f : -m_ref * c.scale_log2e;
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
      V pb;
#pragma unroll
      for (int e = 0; e < 8; e++) pb[e] = (T)s[8 * u + e];
#pragma unroll
      for (int bb = 0; bb < DB; bb++) o[bb] = Mfma<T>::mul(__builtin_bit_cast(V, vr[u][bb]), pb, o[bb]);
    }
  };
  auto fence = [] { __asm__ volatile("" ::: "memory"); __builtin_amdgcn_sched_barrier(0); };
  u32x4 va[2][DB], vb[2][DB];
  const int nmine = wv < nblk ? (nblk - wv + 3) >> 2 : 0;
  auto step = [&](int i, int stage, u32x4 (&vr)[2][DB]) {
    const int b = wv + 4 * i;
    if (i + 1 < nmine) wait_vmem<LOADS>(); else wait_vmem<0>();
    fence();
    f32x16 s;
    scores(stage, s);
    if (i + 2 < nmine) {
      __builtin_amdgcn_s_waitcnt(0xC07F);            // lgkmcnt(0): every K operand of this block has been read
      fence();
      issue_k(b + 8, stage);
    }
    softmax_pv(b, s, vr);
    if (i + 2 < nmine) load_v(vr);
  };
  if (nmine > 0) {
    issue_k(wv, 0); load_v(va);
    if (nmine > 1) { issue_k(wv + 4, 1); load_v(vb); }
    for (int i = 0; i < nmine; i += 2) {
      step(i, 0, va);
      if (i + 1 < nmine) step(i + 1, 1, vb);
    }
  }
  l_run += __shfl_xor(l_run, 32, 64);
  if (__any(bad)) l_run = NAN;

  // ---- the four waves' results meet in LDS (the K buffers are free once every wave is past its loop)
  __syncthreads();
  float* sm = reinterpret_cast<float*>(smem + AS_LDS_BASE);              // [4][rows] maxima, then sums, in log2 units
  float* sl = sm + 4 * AS_ROWS;
  float* red = sl + 4 * AS_ROWS;                                         // [4][rows][D]
  const int rows = it.rows;
  const float m2 = m_ref * c.scale_log2e;
  if (lane < 32) { sm[wv * AS_ROWS + lane] = m2; sl[wv * AS_ROWS + lane] = l_run; }
  __syncthreads();
  auto max_of = [&](int g) { return fmaxf(fmaxf(sm[g], sm[AS_ROWS + g]), fmaxf(sm[2 * AS_ROWS + g], sm[3 * AS_ROWS + g])); };
  auto sum_of = [&](int g, float mall) {
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; w++) {
      const float m = sm[w * AS_ROWS + g], x = sl[w * AS_ROWS + g];
      l += m == -INFINITY ? x : x * __builtin_amdgcn_exp2f(m - mall);    // 0 of a wave without scores above -inf, or NaN
    }
    return l;
  };
  if (l32 < rows) {
    const float mall = max_of(l32), f = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m2 - mall);
#pragma unroll
    for (int bb = 0; bb < DB; bb++)
#pragma unroll
      for (int r = 0; r < 16; r++) red[(wv * AS_ROWS + l32) * D + bb * 32 + 8 * (r >> 2) + 4 * lh + (r & 3)] = o[bb][r] * f;
  }
  __syncthreads();
  for (int i = tid; i < rows * D; i += 256) {
    const int g = i / D, e = i % D;
    const float sum = red[i] + red[AS_ROWS * D + i] + red[2 * AS_ROWS * D + i] + red[3 * AS_ROWS * D + i];
    if (it.part < 0) {
      const float mall = max_of(g), l = sum_of(g, mall);
      const int v = it.row0 + g, r = v / c.heads, h = kvh * c.heads + v % c.heads;
      c.out[(long long)r * c.out_stride + h * D + e] = (T)(sum / l);
      if (e == 0 && c.lse) c.lse[(long long)r * c.n_q + h] = LN2 * (mall + __builtin_amdgcn_logf(l));
    } else {
      c.plan.outs[((size_t)(it.part + g) * c.n_kv + kvh) * D + e] = sum;
    }
  }
  if (it.part >= 0 && tid < rows) {
    const float mall = max_of(tid);
    c.plan.stats[(size_t)(it.part + tid) * c.n_kv + kvh] = f32x2{mall, sum_of(tid, mall)};
  }
  __syncthreads();                                   // before the next item's K lands there
}

template <typename T, int D>
__global__ void __launch_bounds__(256, 2) attn_shared_kernel(AttnCall<T> c) {
  __shared__ __align__(16) unsigned char smem[attn_shared_lds<D>()];
  const int slot = blockIdx.x / c.n_kv, kvh = blockIdx.x % c.n_kv;
  const int first = c.plan.slot_first[slot], end = c.plan.slot_first[slot + 1];
  for (int i = first; i < end; i++) run_item<T, D>(smem, c, c.plan.items[i], kvh);
}

// Joins the partial results of a (request, query head): a wave each, d / 64 elements a lane.
template <typename T, int D>
__global__ void __launch_bounds__(256) attn_shared_join_kernel(AttnCall<T> c) {
  constexpr int PER = D / 64;
  const int lane = threadIdx.x & 63, at = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= c.n * c.n_q) return;
  const int r = at / c.n_q, head = at % c.n_q, kvh = head / c.heads, h = head % c.heads;
  const Parts p = c.plan.parts[r];
  if (p.done && p.len >= 0) return;
  const int count = p.len < 0 ? 0 : p.p_count + p.s_count;
  auto row_of = [&](int j) { return (size_t)((j < p.p_count ? p.p_part + j * p.p_step : p.s_part + (j - p.p_count) * c.heads) + h) * c.n_kv + kvh; };
  float m = -INFINITY;
  for (int j = lane; j < count; j += 64) m = fmaxf(m, c.plan.stats[row_of(j)][0]);
  m = wave_max(m);
  float l = 0.f, o[PER];
#pragma unroll
  for (int e = 0; e < PER; e++) o[e] = 0.f;
#pragma unroll 4
  for (int j = 0; j < count; j++) {
    const size_t row = row_of(j);
    const f32x2 st = c.plan.stats[row];
    const float w = st[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[0] - m);
    l += st[0] == -INFINITY ? st[1] : st[1] * w;
#pragma unroll
    for (int e = 0; e < PER; e++) o[e] += c.plan.outs[row * D + lane * PER + e] * w;
  }
  T* out = c.out + (long long)r * c.out_stride + head * D + lane * PER;
  const bool none = p.len == 0;                      // nothing to attend to: zeros, and the logarithm of an empty sum
#pragma unroll
  for (int e = 0; e < PER; e++) out[e] = (T)(p.len < 0 ? NAN : none ? 0.f : o[e] / l);
  if (lane == 0 && c.lse) c.lse[(long long)r * c.n_q + head] = p.len < 0 ? NAN : none ? -INFINITY : LN2 * (m + __builtin_amdgcn_logf(l));
}

template <typename T, int D>
hipError_t launch_attn(hipStream_t s, const AttnCall<T>& c) {
  hipError_t e = launch(attn_shared_kernel<T, D>, dim3(slots_of(c.n_kv) * c.n_kv), dim3(256), 0, s, c);
  if (e == hipSuccess) e = launch(attn_shared_join_kernel<T, D>, dim3((unsigned)(((int64_t)c.n * c.n_q + 3) / 4)), dim3(256), 0, s, c);
  return e;
}

bool sizes_ok(int n, int n_q, int n_kv, int d) {
  return n >= 0 && n <= OP_MAX_REQUESTS && n_kv >= 1 && n_kv <= AS_SLOTS && n_q >= n_kv && n_q % n_kv == 0 && n_q / n_kv <= AS_ROWS && (d == 64 || d == 128);
}
// The batch's description, without what a call of one layer adds.
int check_batch(const sts_attn_batch* b, Plan* plan) {
  if (!b || (b->dtype != STS_BF16 && b->dtype != STS_F16) || !sizes_ok(b->n_requests, b->n_q, b->n_kv, b->d)) return STS_EINVAL;
  if (b->n_groups < 0 || b->n_groups > b->n_requests || b->pool_pages < 0 || b->max_pages < 0 || b->max_pages > (1 << 26) || b->table_stride < b->max_pages) return STS_EINVAL;
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
  const PlanCall c{n, b->n_groups, b->n_q / b->n_kv, slots, b->max_pages, b->lens, b->group_starts, b->shared_lens, plan};
  return op_result(launch(attn_shared_plan_kernel, dim3(1), dim3(AS_PLAN_THREADS), (size_t)(3 * n + 2 + slots + 1) * sizeof(int), s, c));
}

template <typename T>
static int attn_shared(const sts_attn_batch* b, const Plan& plan, const void* q, int64_t q_stride, const void* pool, void* out, int64_t out_stride, float* lse, float scale, hipStream_t s) {
  const bool q_vec = aligned(q, 16) && q_stride % 8 == 0;
  const AttnCall<T> c{reinterpret_cast<const T*>(q), q_stride, reinterpret_cast<const T*>(pool), reinterpret_cast<T*>(out), out_stride, lse, b->tables, b->table_stride,
                      b->n_requests, b->n_q, b->n_kv, b->n_q / b->n_kv, b->pool_pages, scale * LOG2E, q_vec, plan};
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
