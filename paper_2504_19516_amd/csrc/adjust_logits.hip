// Logits before a token is chosen: penalties for tokens that were there, biases, masks of a grammar.
//
//   y = x / r or x r (x > 0 or not), where the token stands in prompt or output;  y -= f n + (n > 0) w;  y += b;  -inf where ruled out
//
// with n the token's count in the output. A workgroup takes a part of the vocabulary for some rows in a row: it counts the history's tokens of its part in LDS, once for
// all rows of a request, and adds and takes off again the few tokens of each drafted node's path. One bit for each token tells whether anything applies to it; of the
// others nothing is computed, and in place they are not even read: a group of neighbouring elements goes to memory only where it changes, and without being read
// where all of it is ruled out.
//
// Bound by memory where rows are copied, by latency for a few rows (history, LDS, elements one behind the other). The arithmetic is in 64 bits, rounded once to 32 and to the type: it
// runs for the tokens that something applies to, a few thousand of a row.
#include <algorithm>
#include <cmath>

#include "device_ops.h"

namespace sts {
namespace {

constexpr int AL_THREADS = 256, AL_NODES = 256;
constexpr int AL_BATCH = 4;                            // groups of elements of a thread under way
constexpr int AL_ROWS = 8;                             // rows of a workgroup, at most: a bit each
constexpr int AL_PART = 4096, AL_LEAST = 1024, AL_WORKGROUPS = 1024;       // tokens of a part, fewer where there are fewer workgroups than that
constexpr unsigned AL_PROMPT = 1u << 31;               // beside the count of the output

struct AdjustCall {
  sts_adjust_logits a;
  int part, rows_per;                                  // tokens of a part (a multiple of 32), rows of a workgroup
  bool in_place, tokens_vec;                           // tokens can be loaded 16 bytes at a time
};

// E: elements of a group, in aligned vectors
template <typename T, int E>
__global__ void __launch_bounds__(AL_THREADS) adjust_logits_kernel(AdjustCall c) {
  typedef T V __attribute__((ext_vector_type(E)));
  extern __shared__ unsigned lds[];
  __shared__ short parents[AL_NODES];
  __shared__ int drafted[AL_NODES], mask_of[AL_ROWS];
  const sts_adjust_logits& a = c.a;
  const int tid = threadIdx.x, lo = blockIdx.y * c.part, size = min(a.vocab - lo, c.part);
  const bool counted = a.tokens || a.drafted, any = counted || a.bias_tokens;
  // a bit for each token that something applies to; counts; the bias' entry + 1, 0 without one; a bit for each of the rows on whose path a token is
  unsigned *touched = lds, *count = lds + c.part / 32, *bias = count + (counted ? c.part : 0), *on_path = bias + (a.bias_tokens ? c.part : 0);
  const int words = c.part / 32 + (counted ? c.part : 0) + (a.bias_tokens ? c.part : 0) + (a.drafted ? c.part / 4 : 0);
  auto mark = [&](int t) { atomicOr(&touched[t >> 5], 1u << (t & 31)); };
  auto request_of = [&](int row) {
    const int r = a.requests ? a.requests[row] : row;
    return (unsigned)r < (unsigned)a.n_requests ? r : -1;
  };
  const int end = min(a.rows, ((int)blockIdx.x + 1) * c.rows_per);
  for (int row0 = blockIdx.x * c.rows_per, row1; row0 < end; row0 = row1) {
    // the next rows of one request
    const int request = request_of(row0);
    row1 = row0 + 1;
    while (row1 < end && request_of(row1) == request) row1++;
    const int rows = row1 - row0;
    int first = 0, nodes = 0;
    __syncthreads();                                   // nobody reads the rows before any more
    if (tid < rows) mask_of[tid] = a.masks ? a.mask_rows[row0 + tid] : -1;
    if (!any) __syncthreads();
    if (any) {
      for (int i = tid; i < words; i += AL_THREADS) lds[i] = 0;
      if (a.drafted && request >= 0) {
        first = a.row_starts[request];
        const int behind = a.row_starts[request + 1];
        nodes = first >= 0 && behind >= first && behind <= a.rows ? min(behind - first, AL_NODES) : 0;
        if (tid < nodes) {
          const int p = a.parents[first + tid];
          parents[tid] = (short)(p >= 0 && p < tid ? p : -1);
          drafted[tid] = a.drafted[first + tid];
        }
      }
      __syncthreads();
      if (request >= 0 && a.tokens) {
        const int* tokens = a.tokens + (long long)request * a.token_stride;
        const int len = (int)min((long long)a.lens[request], (long long)a.token_stride), prompt = a.prompt_lens ? a.prompt_lens[request] : 0;
        auto one = [&](int t, int i) {
          t -= lo;
          if ((unsigned)t >= (unsigned)size) return;
          if (i < prompt) atomicOr(&count[t], AL_PROMPT); else atomicAdd(&count[t], 1u);
          mark(t);
        };
        int i = 0;
        if (c.tokens_vec) {
          const int whole = max(len, 0) / 4;
#pragma unroll 4
          for (int v = tid; v < whole; v += AL_THREADS) {
            const i32x4 t = reinterpret_cast<const i32x4*>(tokens)[v];
#pragma unroll
            for (int e = 0; e < 4; e++) one(t[e], 4 * v + e);
          }
          i = whole * 4;
        }
        for (i += tid; i < len; i += AL_THREADS) one(tokens[i], i);
      }
      if (request >= 0 && a.bias_tokens) {
        const int behind = min(a.bias_starts[request + 1], a.n_biases);
        for (int i = max(a.bias_starts[request], 0) + tid; i < behind; i += AL_THREADS) {
          const int t = a.bias_tokens[i] - lo;
          if ((unsigned)t >= (unsigned)size) continue;
          atomicMax(&bias[t], (unsigned)i + 1);
          mark(t);
        }
      }
      if (tid < rows && row0 + tid >= first && row0 + tid < first + nodes)       // a thread for each row's path
        for (int j = row0 + tid - first; j >= 0; j = parents[j]) {
          const int t = drafted[j] - lo;
          if ((unsigned)t >= (unsigned)size) continue;
          atomicOr(&on_path[t >> 2], 1u << (t % 4 * 8 + tid));
          mark(t);
        }
      __syncthreads();
    }
    const double r = request >= 0 && a.repetition ? a.repetition[request] : 1.f, f = request >= 0 && a.frequency ? a.frequency[request] : 0.f, w = request >= 0 && a.presence ? a.presence[request] : 0.f;
    const double inverse = 1.0 / r;
    constexpr unsigned ALL = (1u << E) - 1;
    auto changed = [&](T x, int t, int row) {          // an element that something may apply to, but for the mask
      unsigned n = counted ? count[t] : 0u;
      if (a.drafted && on_path[t >> 2] >> (t % 4 * 8 + row) & 1)
        for (int j = row0 + row - first; j >= 0; j = parents[j]) n += drafted[j] == t + lo;
      const unsigned b = a.bias_tokens ? bias[t] : 0u;
      if (n == 0 && b == 0) return x;                  // on another row's path
      double y = (float)x;
      if (n) y *= y > 0.0 ? inverse : r;
      if (n & ~AL_PROMPT) y -= f * (n & ~AL_PROMPT) + w;
      if (b) y += a.bias_values[b - 1];
      return (T)(float)y;
    };
    // A thread's groups, neighbours of neighbouring threads', the rows one behind the other: four under way
    struct At { int row, t; };
    auto next = [&](At at) {
      if (++at.row == rows) { at.row = 0; at.t += AL_THREADS * E; }
      return at;
    };
    auto group = [&](const At& at) {                   // bits of its elements: something may apply; ruled out
      const int m = __builtin_amdgcn_readfirstlane(mask_of[at.row]);
      const unsigned apply = any ? touched[at.t >> 5] >> (at.t & 31) & ALL : 0u;
      return u32x2{apply, (unsigned)m < (unsigned)a.n_masks ? ~a.masks[(long long)m * a.mask_stride + ((lo + at.t) >> 5)] >> (at.t & 31) & ALL : 0u};
    };
    auto load = [&](V& x, const At& at) {
      const T* from = reinterpret_cast<const T*>(a.logits) + (long long)(row0 + at.row) * a.row_stride + lo + at.t;
      if (E > 1 && at.t + E > size) {
#pragma unroll
        for (int e = 0; e < E; e++)
          if (at.t + e < size) x[e] = from[e];
      } else {
        x = *reinterpret_cast<const V*>(from);
      }
    };
    At at{0, tid * E};
    while (at.t < size) {
      V x[AL_BATCH];
      u32x2 bits[AL_BATCH];
      At ats[AL_BATCH];
#pragma unroll
      for (int u = 0; u < AL_BATCH; u++) {
        ats[u] = at;
        at = next(at);
      }
      if (!c.in_place)
#pragma unroll
        for (int u = 0; u < AL_BATCH; u++)
          if (ats[u].t < size) load(x[u], ats[u]);
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
#pragma unroll
        for (int e = 0; e < E; e++)
          if (out >> e & 1) x[u][e] = (T)-INFINITY;
        T* to = reinterpret_cast<T*>(a.out) + (long long)(row0 + row) * a.out_stride + lo + t;
        if (E > 1 && t + E > size) {
#pragma unroll
          for (int e = 0; e < E; e++)
            if (t + e < size) to[e] = x[u][e];
        } else {
          *reinterpret_cast<V*>(to) = x[u];
        }
      }
    }
  }
}

template <typename T, int E>
hipError_t launch_adjust(hipStream_t s, const AdjustCall& c) {
  const bool counted = c.a.tokens || c.a.drafted;
  const size_t lds = ((size_t)c.part / 32 + (counted ? c.part : 0) + (c.a.bias_tokens ? c.part : 0) + (c.a.drafted ? c.part / 4 : 0)) * sizeof(unsigned);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(adjust_logits_kernel<T, E>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const dim3 grid((c.a.rows + c.rows_per - 1) / c.rows_per, (unsigned)(((int64_t)c.a.vocab + c.part - 1) / c.part));
  return launch(adjust_logits_kernel<T, E>, grid, dim3(AL_THREADS), lds, s, c);
}
template <typename T>
hipError_t launch_adjust(hipStream_t s, const AdjustCall& c) {
  constexpr int E = 16 / sizeof(T);
  auto fits = [&](const void* p, int64_t stride) { return aligned(p, 16) && (stride % E == 0 || c.a.rows == 1); };
  return fits(c.a.logits, c.a.row_stride) && fits(c.a.out, c.a.out_stride) ? launch_adjust<T, E>(s, c) : launch_adjust<T, 1>(s, c);
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
  const int rows_per = a->drafted ? AL_ROWS : 1;
  const int64_t blocks = (a->rows + rows_per - 1) / rows_per;
  int part = AL_PART;
  while (part > AL_LEAST && blocks * ((a->vocab + (int64_t)part - 1) / part) < AL_WORKGROUPS) part /= 2;
  const AdjustCall c{*a, part, rows_per, in_place, a->tokens && aligned(a->tokens, 16) && a->token_stride % 4 == 0};
  return op_result(a->dtype == STS_F32 ? launch_adjust<float>(s, c) : a->dtype == STS_BF16 ? launch_adjust<bf16>(s, c) : launch_adjust<f16>(s, c));
}
