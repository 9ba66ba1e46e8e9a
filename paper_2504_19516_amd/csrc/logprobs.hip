// Log probabilities of given tokens, with the entropy of each row, the token's rank and the most likely alternatives.
//
// With m = max x, Z = sum e^(x - m), S = sum (x - m) e^(x - m) of a row of logits x:
//   log p(t) = x_t - (m + ln Z),   entropy = ln Z - S / Z,   rank(t) = #{j : x_j > x_t, or x_j = x_t and j < t}
// and the top k in that same order (value descending, then index ascending).
//
// One pass over the logits, in units of log2: y = x log2(e) - M, with M = m log2(e) as it rounds, is one fused multiply-add, p = 2^y.
// M stands in for m to the end, so its rounding cancels. Logits beyond 2^100 (a row masked throughout with the type's lowest value)
// would leave fp32's range there: they take y = (x - m) log2(e). Every lane keeps its own running maximum, sum and weighted sum, and
// they meet once at the end. A row is cut into parts (one workgroup each) when there are few rows;
// a second kernel joins the parts.
//
// Top k: a wave keeps a bound below which nothing can be among its k best, and passes elements above it on to a list in LDS. The bound
// comes from the lanes' running maxima, which are there anyway: they are different elements, so the k-th largest of the 64 is a lower
// bound of the wave's k-th best. Some k (1 + ln n) elements of a row in random order pass. A full list is cut to its k best, which
// makes the bound exact; from then on equals do not pass, because a wave goes through its elements in ascending order. So no order of
// the logits and no number of equal ones makes a wave pass on more than a list per batch of its lanes' elements.
#include <algorithm>

#include "device_ops.h"

namespace sts {
namespace {

constexpr int LP_THREADS = 256, LP_WAVES = LP_THREADS / 64;
constexpr int LP_VECS = 8;                      // 16-byte vectors of a lane and batch
constexpr int LP_LIST = 256;                    // entries of a wave's list
constexpr int LP_MAX_K = 32, LP_MAX_PARTS = 16;
constexpr float LOG2E = 1.4426950408889634f;
constexpr double LN2 = 0.69314718055994530942;

// Sums of a part of a row; above: elements that stand before the token.
struct RowSums { float m, z, s; int above; };
__device__ __forceinline__ bool beyond(float m) { return !(fabsf(m) < 0x1p100f) && m != -INFINITY; }
// (a - b) log2(e), as the sums over y refer to it; b >= a
__device__ __forceinline__ float log2_diff(float a, float b) {
#pragma clang fp contract(off)
  return beyond(a) || beyond(b) ? (a - b) * LOG2E : a * LOG2E - b * LOG2E;
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

// The k largest of `count` keys in LDS, in their order, to the front of the list. For one wave. Keys differ from each other.
__device__ __forceinline__ void keep_best(unsigned long long* list, int count, int k) {
  const int lane = threadIdx.x & 63;
  constexpr int PER = LP_LIST / 64;
  unsigned long long mine[PER];
  int before[PER];
#pragma unroll
  for (int j = 0; j < PER; j++) {
    mine[j] = lane + 64 * j < count ? list[lane + 64 * j] : 0;
    before[j] = 0;
  }
  for (int i = 0; i < count; i++) {
    const unsigned long long other = list[i];
#pragma unroll
    for (int j = 0; j < PER; j++) before[j] += other > mine[j];
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int j = 0; j < PER; j++)
    if (lane + 64 * j < count && before[j] < k) list[before[j]] = mine[j];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
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

template <typename T>
__device__ __forceinline__ void write_row(const sts_logprobs& a, int row, const RowSums& t) {
  const RowResult r = finish_sums(t);
  const int tok = a.tokens ? a.tokens[row] : -1;
  const bool given = tok >= 0 && tok < a.vocab;
  const float x = given ? (float)reinterpret_cast<const T*>(a.logits)[(long long)row * a.row_stride + tok] : NAN;
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

template <typename T, bool TOP>
__global__ void __launch_bounds__(LP_THREADS) logprobs_kernel(LogprobsCall c) {
  constexpr int E = 16 / sizeof(T);
  typedef vec16<T> V;
  const sts_logprobs& a = c.a;
  __shared__ unsigned long long lists[TOP ? LP_WAVES : 1][TOP ? LP_LIST : 1];
  __shared__ RowSums wave_sums[LP_WAVES];
  __shared__ int counts[LP_WAVES];
  const int row = blockIdx.y, part = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const T* x = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride;
  const int i0 = part * c.width, i1 = min(a.vocab, i0 + c.width), k = TOP ? a.top_k : 0;
  // vectors lie at 16-byte addresses: the first may begin before the part
  const int lead = (int)(reinterpret_cast<uintptr_t>(x + i0) % 16 / sizeof(T));
  const int base = i0 - lead;
  const int tok = a.tokens ? a.tokens[row] : -1;
  const float xt = tok >= 0 && tok < a.vocab ? (float)x[tok] : NAN;
  // an element stands before the token if it is above `strict` -- or, at a lower index, above `loose`, the next value below. A token of
  // -inf: its rank is its index plus the elements above -inf behind it
  const float strict = xt;
  float loose = key_value(value_key(xt) - 1);
  if (xt == 0.f) loose = -__uint_as_float(1u);
  if (xt == -INFINITY) loose = INFINITY;
  if (xt != xt) loose = NAN;

  RowSums t{-INFINITY, 0.f, 0.f, 0};
  float lane_max = -INFINITY;                    // of the wave's elements so far
  float bound = -INFINITY;                       // elements above it are passed on
  bool open = TOP;                               // there is no bound yet: all are
  int count = 0, above = 0;                      // wave-uniform
  unsigned long long* list = lists[TOP ? wave : 0];

  const int n_vecs = (i1 - base + E - 1) / E;
  constexpr int BATCH = 64 * LP_VECS;
  for (int b = wave * BATCH; b < n_vecs; b += LP_WAVES * BATCH) {
    float v[LP_VECS][E];
#pragma unroll
    for (int j = 0; j < LP_VECS; j++) {
      const int q = b + j * 64 + lane, at = base + q * E;
      if (at >= i0 && at + E <= i1) {
        const V w = *reinterpret_cast<const V*>(x + at);
#pragma unroll
        for (int e = 0; e < E; e++) v[j][e] = (float)w[e];
      } else {
#pragma unroll
        for (int e = 0; e < E; e++) v[j][e] = at + e >= i0 && at + e < i1 ? (float)x[at + e] : -INFINITY;
      }
    }
    float top[LP_VECS], mx = -INFINITY;
#pragma unroll
    for (int j = 0; j < LP_VECS; j++) {
      top[j] = v[j][0];
#pragma unroll
      for (int e = 1; e < E; e++) top[j] = fmaxf(top[j], v[j][e]);
      mx = fmaxf(mx, top[j]);
    }
    // ---- sums
    if (mx > t.m) {
      const float shift = log2_diff(t.m, mx), f = __builtin_amdgcn_exp2f(shift);
      t.s = t.z == 0.f ? 0.f : f * (t.s + shift * t.z);
      t.z *= f;
      t.m = mx;
    }
    auto add = [&](auto y_of) {
#pragma unroll
      for (int j = 0; j < LP_VECS; j++)
#pragma unroll
        for (int e = 0; e < E; e++) {
          const float y = y_of(v[j][e]), p = __builtin_amdgcn_exp2f(y);
          t.z += p;
          t.s = fmaf(p, fmaxf(y, -200.f), t.s);  // p is 0 there; -inf * 0 is not
        }
    };
    if (!__any(beyond(t.m))) {
      const float ref = t.m == -INFINITY ? 0.f : t.m * LOG2E;
      add([&](float x) { return fmaf(x, LOG2E, -ref); });
    } else {
      const float ref = t.m == -INFINITY ? 0.f : t.m, big = t.m * LOG2E;
      const bool far = beyond(t.m);
      add([&](float x) { return far ? (x - ref) * LOG2E : t.m == -INFINITY ? x : fmaf(x, LOG2E, -big); });
    }
    // ---- elements before the token
#pragma unroll
    for (int j = 0; j < LP_VECS; j++) {
      const int at = base + (b + j * 64 + lane) * E;
      const bool all_before = at + E <= tok, all_behind = at >= tok;
#pragma unroll
      for (int e = 0; e < E; e++) {
        const float limit = all_before || (!all_behind && at + e < tok) ? loose : strict;
        above += __popcll(__ballot(v[j][e] > limit));
      }
    }
    // ---- candidates
    if constexpr (TOP) {
      lane_max = fmaxf(lane_max, mx);
      {
        // the k-th largest of the lanes' maxima, its upper 16 bits
        const unsigned mk = value_key(lane_max);
        unsigned kth = 0;
#pragma unroll
        for (int bit = 31; bit >= 16; bit--) {
          const unsigned cand = kth | 1u << bit;
          if (__popcll(__ballot(mk >= cand)) >= k) kth = cand;
        }
        if (kth > value_key(-INFINITY)) {
          const float at_least = key_value(kth), below = at_least == 0.f ? -__uint_as_float(1u) : key_value(kth - 1);
          bound = open ? below : fmaxf(bound, below);
          open = false;
        }
      }
#pragma unroll
      for (int j = 0; j < LP_VECS; j++) {
        if (!__any(open || top[j] > bound)) continue;
        const int at = base + (b + j * 64 + lane) * E;
        bool cut = false;
        for (int e = 0; e < E; e++) {
          float xe = v[j][0];
#pragma unroll
          for (int u = 1; u < E; u++) xe = e == u ? v[j][u] : xe;
          const bool pass = (open || xe > bound) && at + e >= i0 && at + e < i1;
          const unsigned long long mask = __ballot(pass);
          if (mask == 0) continue;
          const int more = __popcll(mask);
          if (count + more > LP_LIST) {
            keep_best(list, count, k);
            count = k;
            cut = true;
          }
          if (pass) list[count + __popcll(mask & ((1ull << lane) - 1))] = order_key(xe, at + e);
          count += more;
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          __builtin_amdgcn_wave_barrier();
        }
        if (cut || count > LP_LIST - 128) {
          // the bound becomes the k-th best: everything up to this vector is in, and what comes has higher indices
          keep_best(list, count, k);
          count = min(count, k);
          if (count < k) continue;
          bound = key_value((unsigned)(list[k - 1] >> 32));
          open = false;
        }
      }
    }
  }
  t.above = 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    RowSums u{__shfl_xor(t.m, o, 64), __shfl_xor(t.z, o, 64), __shfl_xor(t.s, o, 64), 0};
    join_sums(t, u);
  }
  if constexpr (TOP) {
    keep_best(list, count, k);
    count = min(count, k);
  }
  if (lane == 0) {
    t.above = above;
    wave_sums[wave] = t;
    counts[wave] = count;
  }
  __syncthreads();
  if (tid >= 64) return;
  t = wave_sums[0];
#pragma unroll
  for (int w = 1; w < LP_WAVES; w++) join_sums(t, wave_sums[w]);
  int n = counts[0];
  if constexpr (TOP) {
    for (int w = 1; w < LP_WAVES; w++) {
      const unsigned long long key = lane < counts[w] ? lists[w][lane] : 0;
      if (lane < counts[w]) lists[0][n + lane] = key;
      n += counts[w];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    keep_best(lists[0], n, k);
    n = min(n, k);
  }
  if (c.parts == 1) {
    if (lane == 0) write_row<T>(a, row, t);
    if constexpr (TOP) {
      const RowResult r = finish_sums(t);
      if (lane < k) write_top(a, row, lane, lists[0][lane], r);
    }
  } else {
    const long long at = (long long)row * c.parts + part;
    if (lane == 0) c.sums[at] = t;
    if constexpr (TOP) if (lane < k) c.keys[at * k + lane] = lane < n ? lists[0][lane] : 0;
  }
}

// Joins the parts of a row.
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_join_kernel(LogprobsCall c) {
  __shared__ unsigned long long keys[LP_MAX_PARTS * LP_MAX_K];
  const sts_logprobs& a = c.a;
  const int row = blockIdx.x, tid = threadIdx.x, n = c.parts * a.top_k;
  for (int i = tid; i < n; i += LP_THREADS) keys[i] = c.keys[(long long)row * n + i];
  RowSums t = c.sums[(long long)row * c.parts];
  for (int p = 1; p < c.parts; p++) join_sums(t, c.sums[(long long)row * c.parts + p]);
  if (tid == 0) write_row<T>(a, row, t);
  if (n == 0) return;
  const RowResult r = finish_sums(t);
  __syncthreads();
  for (int i = tid; i < n; i += LP_THREADS) {
    const unsigned long long mine = keys[i];
    int before = 0;
    for (int j = 0; j < n; j++) before += keys[j] > mine;
    if (mine != 0 && before < a.top_k) write_top(a, row, before, mine, r);
  }
}

// Parts of a row: enough workgroups for four per CU, none shorter than a batch of each of its waves.
int logprob_parts(int rows, int vocab, int bytes) {
  const int batch = LP_WAVES * 64 * LP_VECS * (16 / bytes);
  return std::max(1, std::min({(vocab + batch - 1) / batch, (1024 + rows - 1) / rows, LP_MAX_PARTS}));
}
size_t workspace_of(int rows, int parts, int k) { return parts == 1 ? 0 : (size_t)rows * parts * (sizeof(RowSums) + (size_t)k * sizeof(unsigned long long)); }

template <typename T>
hipError_t launch_logprobs(hipStream_t s, const LogprobsCall& c) {
  const dim3 grid(c.parts, c.a.rows);
  hipError_t e = c.a.top_k > 0 ? launch(logprobs_kernel<T, true>, grid, dim3(LP_THREADS), 0, s, c) : launch(logprobs_kernel<T, false>, grid, dim3(LP_THREADS), 0, s, c);
  if (e == hipSuccess && c.parts > 1) e = launch(logprobs_join_kernel<T>, dim3(c.a.rows), dim3(LP_THREADS), 0, s, c);
  return e;
}

}  // namespace
}  // namespace sts

using namespace sts;

extern "C" int64_t sts_op_logprobs_workspace(int32_t dtype, int32_t rows, int32_t vocab, int32_t top_k) {
  if (dtype < STS_F32 || dtype > STS_F16 || rows < 0 || vocab < 1 || top_k < 0 || top_k > LP_MAX_K) return -1;
  return rows == 0 ? 0 : (int64_t)workspace_of(rows, logprob_parts(rows, vocab, (int)dtype_bytes(dtype)), top_k);
}

extern "C" int sts_op_logprobs(const sts_logprobs* a, void* stream) {
  if (!a || a->dtype < STS_F32 || a->dtype > STS_F16 || a->rows < 0 || a->rows > 65535 || a->vocab < 1 || a->vocab > (1 << 30) || a->top_k < 0 || a->top_k > LP_MAX_K || a->top_k > a->vocab) return STS_EINVAL;
  if (a->rows == 0) return STS_OK;
  const size_t size = dtype_bytes(a->dtype);
  if (!a->logits || !aligned(a->logits, size) || (a->rows > 1 && a->row_stride < a->vocab)) return STS_EINVAL;
  if (!a->tokens && (a->logprob || a->rank)) return STS_EINVAL;
  if ((a->top_logprob || a->top_token) && a->top_k == 0) return STS_EINVAL;
  LogprobsCall c{*a, logprob_parts(a->rows, a->vocab, (int)size), 0, nullptr, nullptr};
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
