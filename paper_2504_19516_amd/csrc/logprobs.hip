// Log probabilities of given tokens, with the entropy of each row, the token's rank and the most likely alternatives.
//
// With m = max x, Z = sum e^(x - m), S = sum (x - m) e^(x - m) of a row of logits x:
//   log p(t) = x_t - (m + ln Z),   entropy = ln Z - S / Z,   rank(t) = #{j : x_j > x_t, or x_j = x_t and j < t}
// and the top k in that same order (value descending, then index ascending).
//
// One pass over the logits, in units of log2: y = x log2(e) - M, with M = m log2(e) as it rounds, is one fused multiply-add, p = 2^y.
// M stands in for m to the end, so its rounding cancels. A maximum beyond 2^100 (a row masked throughout with the type's lowest value)
// would leave fp32's range there: it takes y = x - m, which is 0 or below -2^77. Every lane keeps its own running maximum, sum and weighted
// sum, and they meet once at the end. A row is cut into parts (one workgroup each) when there are few rows; a second kernel joins the parts.
//
// Top k: while the row streams by, each lane only notes the largest element of every group of its own (32 elements or more) in LDS. The largest
// of the four waves' lanes i, for each i, are 64 different elements, so the k-th largest of them bounds the k-th best from below (of all 256
// lanes it bounded it a little better, and took more time than that saved: one row 13.1 us for 12.4, 1000 rows of 4000 10.7 for 9.7). Few groups
// reach the bound (some k), and their elements are read again, compared with it, and sorted by compare-exchanges between lanes. Where more
// elements reach the bound than the buffer holds (rows of equal values), the waves go through the part again, each with a sorted list of its 64
// best, and compare value and index with its k-th.
//
// Bound by memory: 2048 rows of 128256 bf16 logits take 103 us with one alternative (5.1 TB/s), 112 with 20. One row of fp32 takes 8 us and 4.5
// for the join of its 16 parts: one batch a wave, then latencies (the bound, the groups read again, the sort) and the fetch of code that runs
// once: with the elements before and behind the aligned vectors handled in every load instead of by one lane each, it took 2 us more, and 2048
// rows 11. The form that tested every element as it came, with a buffer of candidates in the loop, took 140 us with one alternative, 230 with 20.
#include <algorithm>

#include "device_ops.h"

namespace sts {
namespace {

constexpr int LP_THREADS = 256, LP_WAVES = LP_THREADS / 64;
constexpr int LP_ELEMS = 32;                    // elements of a lane and batch
constexpr int LP_MAX_K = 32, LP_MAX_PARTS = 16;
constexpr int LP_SLOTS = 8;                     // groups of a lane
constexpr int LP_BUFFER = 256;                  // candidates of a part
constexpr int LP_WORKGROUPS = 1024;             // wanted: four a CU, see logprob_parts
constexpr float LOG2E = 1.4426950408889634f;
constexpr double LN2 = 0.69314718055994530942;

// Sums of a part of a row; above: elements that stand before the token.
struct RowSums { float m, z, s; int above; };
__device__ __forceinline__ bool beyond(float m) { return !(fabsf(m) < 0x1p100f) && m != -INFINITY; }
// (a - b) log2(e), as the sums over y refer to it; b >= a. Bounded: 2^ of it is 0 anyway, and 0 times it has to be 0.
__device__ __forceinline__ float log2_diff(float a, float b) {
#pragma clang fp contract(off)
  return fmaxf(beyond(a) || beyond(b) ? (a - b) * LOG2E : a * LOG2E - b * LOG2E, -0x1p100f);
}

// An element's place in the order, larger = earlier: value (-0 as 0, NaN as -inf), then the lower index. 0: no element.
__device__ __forceinline__ unsigned value_key(float x) {
  const unsigned b = __float_as_uint(x == x ? x + 0.f : -INFINITY);
  return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(unsigned k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ unsigned long long order_key(float x, int index) { return (unsigned long long)value_key(x) << 32 | (unsigned)~index; }

__device__ __forceinline__ void join_sums(RowSums& a, const RowSums& b) {
  const float m = fmaxf(a.m, b.m), ma = m == -INFINITY ? 0.f : log2_diff(a.m, m), mb = m == -INFINITY ? 0.f : log2_diff(b.m, m);
  const float fa = __builtin_amdgcn_exp2f(ma), fb = __builtin_amdgcn_exp2f(mb);      // 0 for a side that has seen nothing but -inf
  // sum (y - shift) p = s + (old - new) z
  a.s = fa * (a.s + (a.m == -INFINITY ? 0.f : ma * a.z)) + fb * (b.s + (b.m == -INFINITY ? 0.f : mb * b.z));
  a.z = fa * a.z + fb * b.z;
  a.m = m;
  a.above += b.above;
}

// Exchange with the lane whose number differs in one bit, without a trip through LDS.
template <int M>
__device__ __forceinline__ unsigned xor_lane(unsigned v) {
  auto dpp = [](unsigned x, auto ctrl) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, true); };
  if constexpr (M == 1) return dpp(v, std::integral_constant<int, 0xB1>{});
  if constexpr (M == 2) return dpp(v, std::integral_constant<int, 0x4E>{});
  if constexpr (M == 4) return dpp(dpp(v, std::integral_constant<int, 0x141>{}), std::integral_constant<int, 0x1B>{});     // 7 - i, then i ^ 3
  if constexpr (M == 8) return dpp(v, std::integral_constant<int, 0x128>{});                                              // turned by 8 of 16
  if constexpr (M == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  if constexpr (M == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return threadIdx.x & 32 ? r[0] : r[1];
  }
}
template <int M> __device__ __forceinline__ float xor_lane(float v) { return __uint_as_float(xor_lane<M>(__float_as_uint(v))); }
template <int M> __device__ __forceinline__ unsigned long long xor_lane(unsigned long long v) {
  return (unsigned long long)xor_lane<M>((unsigned)(v >> 32)) << 32 | xor_lane<M>((unsigned)v);
}
template <typename T, typename F>
__device__ __forceinline__ T all_lanes(T v, F f) {
  v = f(v, xor_lane<1>(v)); v = f(v, xor_lane<2>(v)); v = f(v, xor_lane<4>(v));
  v = f(v, xor_lane<8>(v)); v = f(v, xor_lane<16>(v)); v = f(v, xor_lane<32>(v));
  return v;
}
// One step of a sorting network: lanes M apart keep the larger key in the lane where `larger` holds.
template <int M>
__device__ __forceinline__ void exchange(unsigned long long& key, bool larger) {
  const unsigned long long other = xor_lane<M>(key);
  if ((other > key) == larger) key = other;
}
// A bitonic run of 64 keys into descending order.
__device__ __forceinline__ void settle(unsigned long long& key) {
  const int lane = threadIdx.x & 63;
  exchange<32>(key, !(lane & 32)); exchange<16>(key, !(lane & 16)); exchange<8>(key, !(lane & 8));
  exchange<4>(key, !(lane & 4)); exchange<2>(key, !(lane & 2)); exchange<1>(key, !(lane & 1));
}
// 64 keys into ascending order.
__device__ __forceinline__ void sort_up(unsigned long long& key) {
  const int lane = threadIdx.x & 63;
  auto up = [&](int size) { return (lane & size) == 0; };          // this lane's run of `size` goes up
#define STEP(size, m) exchange<m>(key, ((lane & m) != 0) == up(size))
  STEP(2, 1);
  STEP(4, 2); STEP(4, 1);
  STEP(8, 4); STEP(8, 2); STEP(8, 1);
  STEP(16, 8); STEP(16, 4); STEP(16, 2); STEP(16, 1);
  STEP(32, 16); STEP(32, 8); STEP(32, 4); STEP(32, 2); STEP(32, 1);
  STEP(64, 32); STEP(64, 16); STEP(64, 8); STEP(64, 4); STEP(64, 2); STEP(64, 1);
#undef STEP
}
// The 64 best of a descending list and of 64 further keys, in descending order.
__device__ __forceinline__ void merge_64(unsigned long long& best, unsigned long long more) {
  sort_up(more);
  best = more > best ? more : best;
  settle(best);
}
// The 32 best of `n` descending lists of 32 keys each, in descending order (lanes 0 to 31).
__device__ __forceinline__ unsigned long long merge_lists(const unsigned long long (*lists)[LP_MAX_K], int n) {
  const int lane = threadIdx.x & 63;
  unsigned long long key = lane < 32 ? lists[0][lane] : 0;
  for (int i = 1; i < n; i++) {
    if (lane >= 32) key = lists[i][63 - lane];
    settle(key);
  }
  return key;
}

struct LogprobsCall {
  sts_logprobs a;
  int parts, width;                             // of a row, and elements of a part
  RowSums* sums;                                // [rows][parts]
  unsigned long long* keys;                     // [rows][parts][top_k]
};

// What is written for a row once its sums are whole. For one thread.
struct RowResult { double ref, lz; float entropy; bool none; };
__device__ __forceinline__ RowResult finish_sums(const RowSums& t) {
  RowResult r;
  r.none = t.m == -INFINITY && t.z == 0.f;       // nothing but -inf
  r.ref = beyond(t.m) ? (double)t.m : (double)t.m + LN2 * ((double)(t.m * LOG2E) - (double)t.m * (double)LOG2E);      // m, and what M was rounded by
  r.lz = log((double)t.z);
  r.entropy = r.none ? 0.f : (float)(r.lz - LN2 * ((double)t.s / (double)t.z));
  return r;
}
__device__ __forceinline__ float logprob_of(float x, const RowResult& r) { return r.none ? -INFINITY : (float)((double)x - r.ref - r.lz); }

// tok, x: the given token and its logit (NaN if there is none).
__device__ __forceinline__ void write_row(const sts_logprobs& a, int row, const RowSums& t, const RowResult& r, int tok, float x) {
  const bool given = tok >= 0 && tok < a.vocab;
  if (a.logprob) a.logprob[row] = given ? logprob_of(x, r) : NAN;
  if (a.rank) a.rank[row] = x != x ? -1 : x == -INFINITY ? tok + t.above : t.above;
  if (a.entropy) a.entropy[row] = r.entropy;
  if (a.lse) a.lse[row] = r.none ? -INFINITY : (float)(r.ref + r.lz);
}
__device__ __forceinline__ void write_top(const sts_logprobs& a, int row, int at, unsigned long long key, const RowResult& r) {
  const long long i = (long long)row * a.top_k + at;
  if (a.top_token) a.top_token[i] = (int)~(unsigned)key;
  if (a.top_logprob) a.top_logprob[i] = logprob_of(key_value((unsigned)(key >> 32)), r);
}

__device__ __forceinline__ float below(float x) {                 // the next value below
  return x == 0.f ? -__uint_as_float(1u) : key_value(value_key(x) - 1);
}
__device__ __forceinline__ void lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wave's 64 best of every fourth load of a part's vectors, and of one more key a lane (0: none), in descending order, with a buffer of its own
// of 64 + 64 E keys.
template <typename T, typename L>
__device__ unsigned long long second_pass(unsigned long long* buffer, int n_vecs, int a0, int k, unsigned long long more, L load) {
  constexpr int E = 16 / sizeof(T);
  const int lane = threadIdx.x & 63;
  unsigned long long best = 0, least = 0;        // the list, and its k-th key: what is not above it is not among the k best
  int count = 0;
  merge_64(best, more);
  for (int q = threadIdx.x; q - lane < n_vecs; q += LP_THREADS) {
    const vec16<T> v = load(q);
#pragma unroll
    for (int e = 0; e < E; e++) {
      const unsigned long long key = order_key((float)v[e], a0 + q * E + e);
      const bool pass = key > least && q < n_vecs;
      const unsigned long long mask = __ballot(pass);
      if (pass) buffer[count + __popcll(mask & ((1ull << lane) - 1))] = key;
      count += __popcll(mask);
    }
    lds_fence();
    while (count >= 64) {
      count -= 64;
      merge_64(best, buffer[count + lane]);
      least = (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(best >> 32), k - 1) << 32 | (unsigned)__builtin_amdgcn_readlane((int)best, k - 1);
    }
    lds_fence();
  }
  merge_64(best, lane < count ? buffer[lane] : 0);
  return best;
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS, 5) logprobs_kernel(LogprobsCall c) {
  constexpr int E = 16 / sizeof(T), VECS = LP_ELEMS / E, BATCH = 64 * VECS;
  typedef vec16<T> V;
  const sts_logprobs& a = c.a;
  constexpr int SECOND = 64 + 64 * E;            // keys that a wave's buffer holds in the second pass: almost a list, and what a load may pass on
  union Scratch {
    struct { unsigned long long buffer[LP_BUFFER]; float group_max[LP_SLOTS][LP_THREADS], lane_maxima[LP_THREADS]; } first;
    unsigned long long second[LP_WAVES][SECOND];
    char none;
  };
  __shared__ __align__(16) unsigned char scratch[TOP ? sizeof(Scratch) : 16];
  __shared__ unsigned long long lists[TOP ? LP_WAVES : 1][LP_MAX_K];
  auto& first = reinterpret_cast<Scratch*>(scratch)->first;
  __shared__ RowSums wave_sums[LP_WAVES];
  __shared__ int candidates;
  const int row = blockIdx.y, part = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const T* x = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride;
  const int i0 = part * c.width, i1 = min(a.vocab, i0 + c.width), k = TOP ? a.top_k : 0;
  // vectors at 16-byte addresses, from element a0 to a1; the fewer than 2 E elements around them go to the first wave's lanes
  const int a0 = min(i1, i0 + (int)(-reinterpret_cast<uintptr_t>(x + i0) % 16 / sizeof(T))), n_vecs = (i1 - a0) / E, a1 = a0 + n_vecs * E;
  auto load = [&](int q) {
    V v;
    if (q < n_vecs) v = *reinterpret_cast<const V*>(x + a0 + q * E);
    else {
#pragma unroll
      for (int e = 0; e < E; e++) v[e] = (T)-INFINITY;
    }
    return v;
  };
  V raw[VECS];
  auto fetch = [&](int b) {
#pragma unroll
    for (int j = 0; j < VECS; j++) raw[j] = load(b + j * 64 + lane);
  };
  fetch(wave * BATCH);
  const bool edge = tid < (a0 - i0) + (i1 - a1);
  const int edge_at = tid < a0 - i0 ? i0 + tid : a1 + tid - (a0 - i0);
  const float edge_x = edge ? (float)x[edge_at] : -INFINITY;
  const int tok = a.tokens ? a.tokens[row] : -1;
  const float xt = tok >= 0 && tok < a.vocab ? (float)x[tok] : NAN;
  // an element stands before the token if it is above xt -- or, at a lower index, above `loose`, the next value below. A token of -inf:
  // its rank is its index plus the elements above -inf behind it
  const float loose = xt != xt ? NAN : xt == -INFINITY ? INFINITY : below(xt);
  if (TOP && tid == 0) candidates = 0;

  RowSums t{-INFINITY, 0.f, 0.f, 0};
  auto raise = [&](float mx) {                   // the lane's maximum
    if (mx > t.m) {
      const float shift = log2_diff(t.m, mx), f = __builtin_amdgcn_exp2f(shift);
      t.s = t.z == 0.f ? 0.f : f * (t.s + shift * t.z);
      t.z *= f;
      t.m = mx;
    }
  };
  float scale, ref;
  auto refer = [&] {
    const bool far = beyond(t.m);                // there other values are 2^77 and more away: x - m is as good as any multiple of it
    scale = far ? 1.f : LOG2E; ref = t.m == -INFINITY ? 0.f : t.m * scale;
  };
  auto add = [&](float x1) {
    const float y = fmaf(x1, scale, -ref), p = __builtin_amdgcn_exp2f(y);
    t.z += p;
    t.s = fmaf(p, fmaxf(y, -200.f), t.s);        // p is 0 there; -inf * 0 is not
  };
  raise(edge_x);
  refer();
  add(edge_x);
  int above = __popcll(__ballot(edge && edge_x > (edge_at < tok ? loose : xt)));         // wave-uniform
  float lane_max = edge_x, slot_max = -INFINITY;
  // batches of a wave, and of a group
  const int batches = max(0, (n_vecs - wave * BATCH + LP_WAVES * BATCH - 1) / (LP_WAVES * BATCH)), span = (batches + LP_SLOTS - 1) / LP_SLOTS;
  int slot = 0, in_slot = 0;
  for (int i = 0, b = wave * BATCH; i < batches; i++, b += LP_WAVES * BATCH) {
    float v[VECS][E], mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < VECS; j++)
#pragma unroll
      for (int e = 0; e < E; e++) {
        v[j][e] = (float)raw[j][e];
        mx = fmaxf(mx, v[j][e]);
      }
    if (i + 1 < batches) fetch(b + LP_WAVES * BATCH);
    raise(mx);
    refer();
#pragma unroll
    for (int j = 0; j < VECS; j++) {
      // a vector lies before the token or behind it; the one around it counts as behind (mended below)
      const float limit = a0 + (b + j * 64 + lane + 1) * E <= tok ? loose : xt;
#pragma unroll
      for (int e = 0; e < E; e++) {
        add(v[j][e]);
        above += __popcll(__ballot(v[j][e] > limit));
      }
    }
    if constexpr (TOP) {
      slot_max = fmaxf(slot_max, mx);
      if (++in_slot == span || i + 1 == batches) {
        first.group_max[slot++][tid] = slot_max;
        lane_max = fmaxf(lane_max, slot_max);
        slot_max = -INFINITY;
        in_slot = 0;
      }
    }
  }
  // the elements before the token in its own vector
  if (wave == 0 && tok >= a0 && tok < a1) {
    const int at = a0 + (tok - a0) / E * E + lane;
    const float xe = at < tok ? (float)x[at] : NAN;
    above += __popcll(__ballot(xe > loose)) - __popcll(__ballot(xe > xt));
  }
  // ---- the lanes' sums, the waves' sums and lists
  const float m = all_lanes(t.m, [](float p, float q) { return fmaxf(p, q); });
  const float shift = t.m == -INFINITY ? 0.f : log2_diff(t.m, m), f = t.m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(shift);      // a lane without a maximum has sums of 0, or NaN
  t.s = f * (t.s + (t.z == 0.f ? 0.f : shift * t.z));
  t.s = all_lanes(t.s, [](float p, float q) { return p + q; });
  t.z = all_lanes(t.z * f, [](float p, float q) { return p + q; });
  t.m = m;
  t.above = above;
  if (lane == 0) wave_sums[wave] = t;
  unsigned long long best = 0;                   // a descending list, a key a lane
  if constexpr (TOP) {
    first.lane_maxima[tid] = lane_max;
    __syncthreads();
    // the k-th largest of the 64, its upper 16 bits; none where fewer than k have seen anything above -inf
    float largest = first.lane_maxima[lane];
#pragma unroll
    for (int w = 1; w < LP_WAVES; w++) largest = fmaxf(largest, first.lane_maxima[w * 64 + lane]);
    const unsigned key = value_key(largest);
    unsigned kth = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; bit--) {
      const unsigned cand = kth | 1u << bit;
      if ((int)__popcll(__ballot(key >= cand)) >= k) kth = cand;
    }
    const bool open = kth <= value_key(-INFINITY);
    float bound = open ? -INFINITY : below(key_value(kth));
    // Without a bound everything above -inf is a candidate, and the part's first 64 elements: among them are 32 of -inf, or more than k others
    auto append = [&](float xe, int at) {
      const int n = atomicAdd(&candidates, 1);
      if (n < LP_BUFFER) first.buffer[n] = order_key(xe, at);
    };
    if (edge && (edge_x > bound || (open && edge_at < i0 + 64))) append(edge_x, edge_at);
    unsigned hits = 0;
    for (int g = 0; g < slot; g++) hits |= (unsigned)(first.group_max[g][tid] > bound || (open && g == 0 && tid * E < 64)) << g;
    while (hits) {                               // lanes apart: their groups
      const int g = __builtin_ctz(hits);
      hits &= hits - 1;
      for (int i = g * span; i < min(batches, (g + 1) * span); i++) {
        const int b = wave * BATCH + i * LP_WAVES * BATCH;
        V again[VECS];
#pragma unroll
        for (int j = 0; j < VECS; j++) again[j] = load(b + j * 64 + lane);
        unsigned found = 0;                      // bit j E + e
#pragma unroll
        for (int j = 0; j < VECS; j++)
#pragma unroll
          for (int e = 0; e < E; e++) found |= (unsigned)((float)again[j][e] > bound) << (j * E + e);
        if (open && i == 0 && tid * E < 64) found |= (1u << E) - 1;             // the first load's
        while (found) {                          // few: their values again, from L1
          const int q = b + __builtin_ctz(found) / E * 64 + lane, at = a0 + q * E + __builtin_ctz(found) % E;
          found &= found - 1;
          if (q >= n_vecs) continue;
          const float xe = (float)x[at];
          if (xe > bound || at < i0 + 64) append(xe, at);
        }
      }
    }
    __syncthreads();
    const int n = candidates;
    if (n <= LP_BUFFER) {
      if (wave != 0) return;
      for (int i = 0; i < n; i += 64) merge_64(best, i + lane < n ? first.buffer[i + lane] : 0);
    } else {
      __syncthreads();                           // the second pass takes the scratch over
      best = second_pass<T>(reinterpret_cast<Scratch*>(scratch)->second[wave], n_vecs, a0, k, edge ? order_key(edge_x, edge_at) : 0, load);
      if (lane < LP_MAX_K) lists[wave][lane] = best;
      __syncthreads();
      if (wave != 0) return;
      best = merge_lists(lists, LP_WAVES);
    }
  } else {
    __syncthreads();
    if (wave != 0) return;
  }
  t = wave_sums[0];
#pragma unroll
  for (int w = 1; w < LP_WAVES; w++) join_sums(t, wave_sums[w]);
  if (c.parts == 1) {
    const RowResult r = finish_sums(t);
    if (lane == 0) write_row(a, row, t, r, tok, xt);
    if constexpr (TOP) if (lane < k) write_top(a, row, lane, best, r);
  } else {
    const long long at = (long long)row * c.parts + part;
    if (lane == 0) c.sums[at] = t;
    if constexpr (TOP) if (lane < k) c.keys[at * k + lane] = best;
  }
}

// Joins the parts of a row.
template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS) logprobs_join_kernel(LogprobsCall c) {
  static_assert(LP_MAX_PARTS == 4 * LP_WAVES, "four parts a wave");
  __shared__ unsigned long long lists[TOP ? LP_MAX_PARTS : 1][LP_MAX_K], quarters[TOP ? LP_WAVES : 1][LP_MAX_K];
  const sts_logprobs& a = c.a;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = a.top_k;
  const int tok = a.tokens ? a.tokens[row] : -1;
  const float xt = tok >= 0 && tok < a.vocab ? (float)reinterpret_cast<const T*>(a.logits)[(long long)row * a.row_stride + tok] : NAN;
  RowSums t{-INFINITY, 0.f, 0.f, 0};
  if (wave == 0 && lane < c.parts) t = c.sums[(long long)row * c.parts + lane];
  unsigned long long best = 0;
  if constexpr (TOP) {
    for (int i = tid; i < LP_MAX_PARTS * LP_MAX_K; i += LP_THREADS) {
      const int p = i / LP_MAX_K, j = i % LP_MAX_K;
      lists[p][j] = p < c.parts && j < k ? c.keys[((long long)row * c.parts + p) * k + j] : 0;
    }
    __syncthreads();
    best = merge_lists(lists + 4 * wave, 4);
    if (lane < LP_MAX_K) quarters[wave][lane] = best;
    __syncthreads();
  }
  if (wave != 0) return;
#pragma unroll
  for (int o = LP_MAX_PARTS / 2; o > 0; o >>= 1) join_sums(t, RowSums{__shfl_xor(t.m, o, 64), __shfl_xor(t.z, o, 64), __shfl_xor(t.s, o, 64), __shfl_xor(t.above, o, 64)});
  t = RowSums{__shfl(t.m, 0, 64), __shfl(t.z, 0, 64), __shfl(t.s, 0, 64), __shfl(t.above, 0, 64)};
  const RowResult r = finish_sums(t);
  if (lane == 0) write_row(a, row, t, r, tok, xt);
  if constexpr (TOP) {
    best = merge_lists(quarters, LP_WAVES);
    if (lane < k) write_top(a, row, lane, best, r);
  }
}

// Parts of a row: enough workgroups for four per CU, none shorter than a batch of each of its waves. Wanting 512 / 1024 / 2048 workgroups, 64
// rows of 128256 fp32 logits with 5 alternatives took 16.9 / 17.7 / 17.7 us, 200 rows 30.4 / 29.1 / 30.7, the join among them.
int logprob_parts(int rows, int vocab) {
  constexpr int batch = LP_WAVES * 64 * LP_ELEMS;
  return std::max(1, std::min({(vocab + batch - 1) / batch, (LP_WORKGROUPS + rows - 1) / rows, LP_MAX_PARTS}));
}
size_t workspace_of(int rows, int parts, int k) { return parts == 1 ? 0 : (size_t)rows * parts * (sizeof(RowSums) + (size_t)k * sizeof(unsigned long long)); }

template <typename T>
hipError_t launch_logprobs(hipStream_t s, const LogprobsCall& c) {
  const dim3 grid(c.parts, c.a.rows);
  hipError_t e = c.a.top_k > 0 ? launch(logprobs_kernel<T, true>, grid, dim3(LP_THREADS), 0, s, c) : launch(logprobs_kernel<T, false>, grid, dim3(LP_THREADS), 0, s, c);
  if (e != hipSuccess || c.parts == 1) return e;
  const dim3 rows(c.a.rows);
  e = c.a.top_k > 0 ? launch(logprobs_join_kernel<T, true>, rows, dim3(LP_THREADS), 0, s, c) : launch(logprobs_join_kernel<T, false>, rows, dim3(LP_THREADS), 0, s, c);
  return e;
}

}  // namespace
}  // namespace sts

using namespace sts;

extern "C" int64_t sts_op_logprobs_workspace(int32_t dtype, int32_t rows, int32_t vocab, int32_t top_k) {
  if (dtype < STS_F32 || dtype > STS_F16 || rows < 0 || rows > 65535 || vocab < 1 || vocab > (1 << 30) || top_k < 0 || top_k > LP_MAX_K) return -1;
  return rows == 0 ? 0 : (int64_t)workspace_of(rows, logprob_parts(rows, vocab), top_k);
}

extern "C" int sts_op_logprobs(const sts_logprobs* a, void* stream) {
  if (!a || a->dtype < STS_F32 || a->dtype > STS_F16 || a->rows < 0 || a->rows > 65535 || a->vocab < 1 || a->vocab > (1 << 30) || a->top_k < 0 || a->top_k > LP_MAX_K || a->top_k > a->vocab) return STS_EINVAL;
  if (a->rows == 0) return STS_OK;
  const size_t size = dtype_bytes(a->dtype);
  if (!a->logits || !aligned(a->logits, size) || (a->rows > 1 && a->row_stride < a->vocab)) return STS_EINVAL;
  if (!a->tokens && (a->logprob || a->rank)) return STS_EINVAL;
  if ((a->top_logprob || a->top_token) && a->top_k == 0) return STS_EINVAL;
  LogprobsCall c{*a, logprob_parts(a->rows, a->vocab), 0, nullptr, nullptr};
  c.width = (a->vocab + c.parts - 1) / c.parts;
  const size_t need = workspace_of(a->rows, c.parts, a->top_k);
  if (need > 0 && (!a->workspace || !aligned(a->workspace, 16) || a->workspace_bytes < (int64_t)need)) return STS_EINVAL;
  c.sums = reinterpret_cast<RowSums*>(a->workspace);
  c.keys = reinterpret_cast<unsigned long long*>(c.sums + (size_t)a->rows * c.parts);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  const hipError_t e = a->dtype == STS_F32 ? launch_logprobs<float>(s, c) : a->dtype == STS_BF16 ? launch_logprobs<bf16>(s, c) : launch_logprobs<f16>(s, c);
  return op_result(e);
}
