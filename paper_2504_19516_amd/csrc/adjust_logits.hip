// Logits before a token is chosen: penalties for tokens that were there, biases, masks of a grammar.
//
//   y = x / r or x r (x > 0 or not), where the token stands in prompt or output;  y -= f n + (n > 0) w;  y += b;  -inf where ruled out
//
// with n the token's count in the output. A workgroup takes a part of the vocabulary for some rows in a row: it counts the history's tokens of its part in LDS, once for
// all rows of a request. One bit for each token tells whether anything may apply to it, eight more on which of the rows' paths it is (how often is counted where that is so:
// seldom); of the others nothing is computed, and in place they are not even read: a group of neighbouring elements goes to memory only where it changes, and without being read
// where all of it is ruled out. The arithmetic is in 64 bits, rounded once, to the type: it runs for a few thousand elements of a row.
//
// Bound by memory where rows are copied (320 rows of 128256 in 32 bits, chains of five on histories of 1500: 83 us, a copy of as many bytes 68; without the arithmetic of what changes some 12
// less, the rest is histories that are read and counted while little else is under way), by latency for a few rows (one row 6.5 us: descriptions, history, LDS, elements, one behind the
// other) and for masks in place (256 rows of 16 bits, half of them masked, 30 MB: 12.5 us). Stores past the caches took 85 instead of 87 us on rows that change, but the log
// probabilities that read them next took longer: 124 instead of 119 for both.
#include <algorithm>
#include <cmath>

#include "device_ops.h"

namespace sts {
namespace {

// Figures of the constants: rows that change, in 32 bits unless stated, with histories of up to 2000 tokens and 8 biases a request; runs differ by up to 2 %.
// "24 calls" is the geometric mean of 24 calls with penalties or biases, of all sizes and types.
// 256 / 512 / 1024 threads: 320 rows in chains of five 86 / 88 / 112 us, 702 rows of 56507 in chains of three 103 / 96 / 132, 256 single rows of 16 bits 81 / 94 / 153, 24 calls 12.3 / 11.5 / 12.7.
constexpr int AL_THREADS = 512, AL_NODES = 256;
// Groups of elements of a thread under way. 2 / 4 / 8: 320 rows 88 / 88 / 103 us, 702 rows 95 / 96 / 115, one row 6.2 / 6.4 / 7.0, 24 calls 11.1 / 11.5 / 12.5: 2 would do as well, and gain some 0.3 us of the small ones.
constexpr int AL_BATCH = 4;
constexpr int AL_ROWS = 8;                             // rows of a workgroup, at most: a bit each
// Tokens of a part, fewer where that leaves fewer workgroups than these. Parts of 2048 / 4096 / 8192: 320 rows 97 / 88 / 86 us, 702 rows of 56507 111 / 96 / 102, 38 chains of 15 and 10586 tokens of vocabulary
// 44 / 38 / 48, 256 single rows of 16 bits 147 / 94 / 82 (each part counts the history for itself), 24 calls 12.3 / 11.5 / 11.3. 256 / 512 / 1024 workgroups: 24 calls 11.5 / 11.0 / 11.4, the large ones level.
constexpr int AL_PART = 4096, AL_LEAST = 1024, AL_WORKGROUPS = 256;
constexpr unsigned AL_PROMPT = 1u << 31;               // beside the count of the output

constexpr int AL_MASK_THREADS = 256, AL_MASK_BATCH = 4;       // groups of a thread: 4 / 8 / 16, 256 rows, half of them masked, 13.4 / 18.5 / 17.5 us, 1000 of 32000, all masked, 19 / 22 / 22

struct AdjustCall {
  sts_adjust_logits a;
  int part, rows_per;                                  // tokens of a part (a multiple of 32), rows of a workgroup
  bool in_place, tokens_vec;                           // tokens can be loaded 16 bytes at a time
  bool parts_first;                                    // the launch's x counts parts, not workgroups' rows
  __device__ __forceinline__ int first_token() const { return (parts_first ? blockIdx.x : blockIdx.y) * part; }
  __device__ __forceinline__ int first_row() const { return (parts_first ? blockIdx.y : blockIdx.x) * rows_per; }
};

// A group of elements, 16 bytes that may begin at any element: rows of odd lengths lie one behind the other as often as aligned ones (702 rows of 56507 in 32 bits 87 us so,
// 147 an element at a time).
template <typename T, int E> struct Group {
  typedef T V __attribute__((ext_vector_type(E)));
  typedef V InMemory __attribute__((aligned(sizeof(T))));
};
// Up to E elements of a row, those behind its end left out.
template <typename T, int E>
__device__ __forceinline__ void load_group(typename Group<T, E>::V& x, const T* from, int left) {
  if (left < E) {
#pragma unroll
    for (int e = 0; e < E; e++)
      if (e < left) x[e] = from[e];
  } else {
    x = *reinterpret_cast<const typename Group<T, E>::InMemory*>(from);
  }
}
template <typename T, int E>
__device__ __forceinline__ void store_group(T* to, typename Group<T, E>::V x, unsigned out, int left) {      // out: elements that are ruled out
#pragma unroll
  for (int e = 0; e < E; e++)
    if (out >> e & 1) x[e] = (T)-INFINITY;
  if (left < E) {
#pragma unroll
    for (int e = 0; e < E; e++)
      if (e < left) to[e] = x[e];
  } else {
    *reinterpret_cast<typename Group<T, E>::InMemory*>(to) = x;
  }
}

// Rows to which nothing but their masks applies: a part of a row a workgroup.
template <typename T, int E>
__global__ void __launch_bounds__(AL_MASK_THREADS) mask_logits_kernel(AdjustCall c) {
  typedef typename Group<T, E>::V V;
  const sts_adjust_logits& a = c.a;
  const int row = c.first_row(), lo = c.first_token(), size = min(a.vocab - lo, c.part), m = a.masks ? a.mask_rows[row] : -1;
  const bool masked = (unsigned)m < (unsigned)a.n_masks;
  if (c.in_place && !masked) return;
  const T* from = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride + lo;
  T* to = reinterpret_cast<T*>(a.out) + (long long)row * a.out_stride + lo;
  const unsigned* mask = a.masks + (masked ? m * a.mask_stride + lo / 32 : 0);
  constexpr unsigned ALL = (1u << E) - 1;
  V x[AL_MASK_BATCH];
  unsigned out[AL_MASK_BATCH];
  auto at = [&](int u) { return ((int)threadIdx.x + u * AL_MASK_THREADS) * E; };
#pragma unroll
  for (int u = 0; u < AL_MASK_BATCH; u++) out[u] = masked && at(u) < size ? ~mask[at(u) >> 5] >> (at(u) & 31) & ALL : 0u;
#pragma unroll
  for (int u = 0; u < AL_MASK_BATCH; u++)
    if (at(u) < size && out[u] != ALL && (out[u] || !c.in_place)) load_group<T, E>(x[u], from + at(u), size - at(u));
#pragma unroll
  for (int u = 0; u < AL_MASK_BATCH; u++)
    if (at(u) < size && (out[u] || !c.in_place)) store_group<T, E>(to + at(u), x[u], out[u], size - at(u));
}

template <typename T, int E>
__global__ void __launch_bounds__(AL_THREADS) adjust_logits_kernel(AdjustCall c) {
  typedef typename Group<T, E>::V V;
  extern __shared__ unsigned lds[];
  __shared__ short parents[AL_NODES];
  __shared__ int drafted[AL_NODES], mask_of[AL_ROWS];
  const sts_adjust_logits& a = c.a;
  const int tid = threadIdx.x, lo = c.first_token(), size = min(a.vocab - lo, c.part);
  const bool counted = a.tokens || a.drafted;
  // a bit for each token that something applies to; counts; the bias' entry + 1, 0 without one; a bit for each of the rows on whose path a token is
  unsigned *touched = lds, *count = lds + c.part / 32, *bias = count + (counted ? c.part : 0), *on_path = bias + (a.bias_tokens ? c.part : 0);
  const int words = c.part / 32 + (counted ? c.part : 0) + (a.bias_tokens ? c.part : 0) + (a.drafted ? c.part / 4 : 0);
  auto clear = [&] {
    for (int i = tid; i < words / 4; i += AL_THREADS) reinterpret_cast<u32x4*>(lds)[i] = u32x4{0u, 0u, 0u, 0u};
  };
  auto mark = [&](int t) { atomicOr(&touched[t >> 5], 1u << (t & 31)); };
  auto request_of = [&](int row) {
    const int r = a.requests ? a.requests[row] : row;
    return (unsigned)r < (unsigned)a.n_requests ? r : -1;
  };
  const int end = min(a.rows, c.first_row() + c.rows_per);
  const int lane = tid & 63;
  for (int row0 = c.first_row(), rows; row0 < end; row0 += rows) {
    // the next rows of one request
    const int mine = row0 + lane < end ? request_of(row0 + lane) : -2, request = __builtin_amdgcn_readfirstlane(mine);
    rows = __builtin_ctzll(~__ballot(mine == request) | 1ull << AL_ROWS);
    // A thread's groups, neighbours of neighbouring threads', the rows one behind the other: four under way, the first ones of a copy from here on
    struct At { int row, t; };
    auto next = [&](At at) {
      if (++at.row == rows) { at.row = 0; at.t += AL_THREADS * E; }
      return at;
    };
    V x[AL_BATCH];
    At at{0, tid * E}, ats[AL_BATCH];
    auto load = [&](V& x, const At& at) {
      load_group<T, E>(x, reinterpret_cast<const T*>(a.logits) + (long long)(row0 + at.row) * a.row_stride + lo + at.t, size - at.t);
    };
    auto begin = [&] {
#pragma unroll
      for (int u = 0; u < AL_BATCH; u++) {
        ats[u] = at;
        at = next(at);
        if (!c.in_place && ats[u].t < size) load(x[u], ats[u]);
      }
    };
    begin();
    // what there is of the request: on the way together
    const bool some = request >= 0;
    const int held = some && a.tokens ? a.lens[request] : 0, prompt = some && a.tokens && a.prompt_lens ? a.prompt_lens[request] : 0;
    const int bias0 = some && a.bias_tokens ? a.bias_starts[request] : 0, bias1 = some && a.bias_tokens ? a.bias_starts[request + 1] : 0;
    const int first = some && a.drafted ? a.row_starts[request] : 0, behind = some && a.drafted ? a.row_starts[request + 1] : 0;
    const float r = some && a.repetition ? a.repetition[request] : 1.f, f = some && a.frequency ? a.frequency[request] : 0.f, w = some && a.presence ? a.presence[request] : 0.f;
    __syncthreads();                                   // nobody reads the rows before any more
    if (tid < rows) mask_of[tid] = a.masks ? a.mask_rows[row0 + tid] : -1;
    clear();
    const int nodes = first >= 0 && behind >= first && behind <= a.rows ? min(behind - first, AL_NODES) : 0;
    if (tid < nodes) {
      const int p = a.parents[first + tid];
      parents[tid] = (short)(p >= 0 && p < tid ? p : -1);
      drafted[tid] = a.drafted[first + tid];
    }
    __syncthreads();
    if (held > 0) {
      const int* tokens = a.tokens + (long long)request * a.token_stride;
      // up to 2^31 - 1 tokens: an index that the next step takes past them is still a number of 32 bits without a sign
      const unsigned len = (unsigned)min((long long)held, (long long)a.token_stride);
      auto one = [&](int t, unsigned i) {
        t = (int)((unsigned)t - (unsigned)lo);
        if ((unsigned)t >= (unsigned)size) return;
        if ((int)i < prompt) atomicOr(&count[t], AL_PROMPT); else atomicAdd(&count[t], 1u);
        mark(t);
      };
      unsigned i = 0;
      if (c.tokens_vec) {
        const unsigned whole = len / 4;
#pragma unroll 4
        for (unsigned v = tid; v < whole; v += AL_THREADS) {
          const i32x4 t = reinterpret_cast<const i32x4*>(tokens)[v];
#pragma unroll
          for (int e = 0; e < 4; e++) one(t[e], 4 * v + e);
        }
        i = whole * 4;
      }
      for (i += tid; i < len; i += AL_THREADS) one(tokens[i], i);
    }
    // both ends of the request's entries within the list before anything is added to them: counted from 0, as an end may be any number
    const unsigned bias_first = min(max(bias0, 0), a.n_biases), bias_count = max(min(max(bias1, 0), a.n_biases) - (int)bias_first, 0);
    for (unsigned i = tid; i < bias_count; i += AL_THREADS) {
      const int t = (int)((unsigned)a.bias_tokens[bias_first + i] - (unsigned)lo);
      if ((unsigned)t >= (unsigned)size) continue;
      atomicMax(&bias[t], bias_first + i + 1);
      mark(t);
    }
    if (tid < rows && row0 + tid >= first && row0 + tid < first + nodes)       // a thread for each row's path
      for (int j = row0 + tid - first; j >= 0; j = parents[j]) {
        const int t = (int)((unsigned)drafted[j] - (unsigned)lo);
        if ((unsigned)t >= (unsigned)size) continue;
        atomicOr(&on_path[t >> 2], 1u << (t % 4 * 8 + tid));
        mark(t);
      }
    __syncthreads();
    const double inverse = 1.0 / r;
    constexpr unsigned ALL = (1u << E) - 1;
    auto changed = [&](T x, int t, int row) {          // an element that something may apply to, but for the mask
      unsigned n = counted ? count[t] : 0u;
      if (a.drafted && on_path[t >> 2] >> (t % 4 * 8 + row) & 1)
        for (int j = row0 + row - first; j >= 0; j = parents[j]) n += drafted[j] == t + lo;
      const unsigned b = a.bias_tokens ? bias[t] : 0u;
      if (n == 0 && b == 0) return x;                  // on another row's path
      double y = (float)x;
      if (n) y *= y > 0.0 ? inverse : (double)r;
      if (n & ~AL_PROMPT) y -= (double)f * (n & ~AL_PROMPT) + w;
      if (b) y += a.bias_values[b - 1];
      return (T)y;                                     // one rounding, from 64 bits to the type
    };
    auto group = [&](const At& at) {                   // bits of its elements: something may apply; ruled out
      const int m = __builtin_amdgcn_readfirstlane(mask_of[at.row]);
      const unsigned apply = touched[at.t >> 5] >> (at.t & 31) & ALL;
      return u32x2{apply, (unsigned)m < (unsigned)a.n_masks ? ~a.masks[(long long)m * a.mask_stride + ((lo + at.t) >> 5)] >> (at.t & 31) & ALL : 0u};
    };
    while (ats[0].t < size) {
      u32x2 bits[AL_BATCH];
#pragma unroll
      for (int u = 0; u < AL_BATCH; u++) bits[u] = ats[u].t < size ? group(ats[u]) : u32x2{0u, 0u};
      if (c.in_place)                                  // only what changes, and is not ruled out as a whole
#pragma unroll
        for (int u = 0; u < AL_BATCH; u++)
          if ((bits[u][0] | bits[u][1]) && bits[u][1] != ALL) load(x[u], ats[u]);
#pragma unroll
      for (int u = 0; u < AL_BATCH; u++) {
        const int t = ats[u].t, row = ats[u].row;
        const unsigned apply = bits[u][0], out = bits[u][1];
        if (t >= size || (c.in_place && !(apply | out))) continue;
        const unsigned ours = apply & ~out;
        if (ours)
#pragma unroll
          for (int e = 0; e < E; e++)
            if (ours >> e & 1) x[u][e] = changed(x[u][e], t + e, row);
        store_group<T, E>(reinterpret_cast<T*>(a.out) + (long long)(row0 + row) * a.out_stride + lo + t, x[u], out, size - t);
      }
      begin();
    }
  }
}

template <typename T>
hipError_t launch_adjust(hipStream_t s, const AdjustCall& c0) {
  constexpr int E = 16 / sizeof(T);
  AdjustCall c = c0;
  const sts_adjust_logits& a = c.a;
  auto parts = [&] { return ((int64_t)a.vocab + c.part - 1) / c.part; };
  auto groups = [&] { return ((int64_t)a.rows + c.rows_per - 1) / c.rows_per; };
  auto workgroups = [&] { return parts() * groups(); };
  // All rows' first parts first: a text's tokens have low numbers more often than others, and what takes longest had better not begin last. The launch's y ends
  // at 65535.
  auto grid = [&] {
    c.parts_first = parts() > 65535;
    return c.parts_first ? dim3((unsigned)parts(), (unsigned)groups()) : dim3((unsigned)groups(), (unsigned)parts());
  };
  const bool counted = a.tokens || a.drafted;
  c.rows_per = 1;
  if (!counted && !a.bias_tokens) {
    c.part = AL_MASK_BATCH * AL_MASK_THREADS * E;
    while (c.part > AL_LEAST && workgroups() < AL_WORKGROUPS) c.part /= 2;
    const dim3 g = grid();
    return launch(mask_logits_kernel<T, E>, g, dim3(AL_MASK_THREADS), 0, s, c);
  }
  c.part = AL_PART;
  if (a.drafted && a.n_requests > 0) {                 // equal shares of a request's rows, where they have alike numbers
    const int mean = std::max(1, (a.rows + a.n_requests / 2) / a.n_requests), shares = (mean + AL_ROWS - 1) / AL_ROWS;
    c.rows_per = (mean + shares - 1) / shares;
    while (c.rows_per > 1 && workgroups() < AL_WORKGROUPS) c.rows_per = (c.rows_per + 1) / 2;
  }
  while (c.part > AL_LEAST && workgroups() < AL_WORKGROUPS) c.part /= 2;
  const size_t lds = ((size_t)c.part / 32 + (counted ? c.part : 0) + (a.bias_tokens ? c.part : 0) + (a.drafted ? c.part / 4 : 0)) * sizeof(unsigned);
  const dim3 g = grid();
  return launch(adjust_logits_kernel<T, E>, g, dim3(AL_THREADS), lds, s, c);
}
}  // namespace
}  // namespace sts

using namespace sts;

extern "C" int sts_op_adjust_logits(const sts_adjust_logits* a, void* stream) {
  if (!a || a->dtype < STS_F32 || a->dtype > STS_F16 || a->rows < 0 || a->rows > 65535 || a->vocab < 1 || a->vocab > (1 << 30) || a->n_requests < 0 || a->n_biases < 0 || a->n_masks < 0) return STS_EINVAL;
  if (a->rows == 0) return STS_OK;
  const size_t size = dtype_bytes(a->dtype);
  if (!a->logits || !a->out || !aligned(a->logits, size) || !aligned(a->out, size)) return STS_EINVAL;
  if (a->rows > 1 && (a->row_stride < a->vocab || a->out_stride < a->vocab)) return STS_EINVAL;
  const bool in_place = a->logits == a->out;
  if (in_place && a->rows > 1 && a->row_stride != a->out_stride) return STS_EINVAL;
  if (!a->requests && a->n_requests < a->rows && (a->tokens || a->drafted || a->bias_tokens)) return STS_EINVAL;      // rows without a request
  if (a->tokens && (!a->lens || a->token_stride < 0)) return STS_EINVAL;
  if (a->drafted && (!a->row_starts || !a->parents)) return STS_EINVAL;
  if ((a->repetition || a->frequency || a->presence || a->prompt_lens) && !a->tokens && !a->drafted) return STS_EINVAL;                 // penalties for nothing
  if (a->bias_tokens ? !a->bias_starts || !a->bias_values : a->n_biases > 0) return STS_EINVAL;
  if (a->masks ? !a->mask_rows || a->mask_stride < (a->vocab + (int64_t)31) / 32 : a->n_masks > 0) return STS_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  const AdjustCall c{*a, 1, 1, in_place, a->tokens && aligned(a->tokens, 16) && a->token_stride % 4 == 0, false};
  return op_result(a->dtype == STS_F32 ? launch_adjust<float>(s, c) : a->dtype == STS_BF16 ? launch_adjust<bf16>(s, c) : launch_adjust<f16>(s, c));
}
