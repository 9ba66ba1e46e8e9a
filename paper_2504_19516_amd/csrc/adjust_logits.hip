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
constexpr unsigned AL_PROMPT = 1u << 31;               // beside the count of the output

struct AdjustCall {
  sts_adjust_logits a;
  int part, rows_per;                                  // tokens of a part (a multiple of 32), rows of a workgroup
  bool in_place;
};

// E: elements of a group, in aligned vectors
template <typename T, int E>
__global__ void __launch_bounds__(AL_THREADS) adjust_logits_kernel(AdjustCall c) {
  typedef T V __attribute__((ext_vector_type(E)));
  extern __shared__ unsigned lds[];
  __shared__ short parents[AL_NODES];
  __shared__ int drafted[AL_NODES];
  const sts_adjust_logits& a = c.a;
  const int tid = threadIdx.x, lo = blockIdx.y * c.part, hi = min(a.vocab, lo + c.part);
  const bool counted = a.tokens || a.drafted, any = counted || a.bias_tokens;
  unsigned *touched = lds, *count = lds + c.part / 32, *bias = count + (counted ? c.part : 0);      // bias: the entry's number + 1, 0 without one
  const int words = c.part / 32 + (counted ? c.part : 0) + (a.bias_tokens ? c.part : 0);
  auto mark = [&](int t) { atomicOr(&touched[t >> 5], 1u << (t & 31)); };
  int built = -2, first = 0, nodes = 0;
  const int row0 = blockIdx.x * c.rows_per, row1 = min(a.rows, row0 + c.rows_per);
  for (int row = row0; row < row1; row++) {
    int request = a.requests ? a.requests[row] : row;
    if ((unsigned)request >= (unsigned)a.n_requests) request = -1;
    int node = -1;
    if (any) {
      __syncthreads();                                 // nobody reads the row before any more
      if (request != built) {
        built = request;
        nodes = 0;
        for (int i = tid; i < words; i += AL_THREADS) lds[i] = 0;
        __syncthreads();
        if (request >= 0) {
          if (a.tokens) {
            const int* tokens = a.tokens + (long long)request * a.token_stride;
            const int len = min((long long)a.lens[request], (long long)a.token_stride), prompt = a.prompt_lens ? a.prompt_lens[request] : 0;
#pragma unroll 4
            for (int i = tid; i < len; i += AL_THREADS) {
              const int t = tokens[i];
              if (t < lo || t >= hi) continue;
              if (i < prompt) atomicOr(&count[t - lo], AL_PROMPT); else atomicAdd(&count[t - lo], 1u);
              mark(t - lo);
            }
          }
          if (a.bias_tokens) {
            const int end = min(a.bias_starts[request + 1], a.n_biases);
            for (int i = max(a.bias_starts[request], 0) + tid; i < end; i += AL_THREADS) {
              const int t = a.bias_tokens[i];
              if (t < lo || t >= hi) continue;
              atomicMax(&bias[t - lo], (unsigned)i + 1);
              mark(t - lo);
            }
          }
          if (a.drafted) {
            first = a.row_starts[request];
            const int end = a.row_starts[request + 1];
            nodes = first >= 0 && end >= first && end <= a.rows ? min(end - first, AL_NODES) : 0;
            if (tid < nodes) {
              const int p = a.parents[first + tid];
              parents[tid] = (short)(p >= 0 && p < tid ? p : -1);
              drafted[tid] = a.drafted[first + tid];
            }
          }
        }
        __syncthreads();
      }
      if (nodes > 0 && row >= first && row < first + nodes) node = row - first;
    }
    // the path's tokens of this part: they come, and go again behind the row
    auto path = [&](unsigned by) {
      for (int j = node; j >= 0; j = parents[j]) {
        const int t = drafted[j];
        if (t < lo || t >= hi) continue;
        atomicAdd(&count[t - lo], by);
        mark(t - lo);
      }
    };
    if (node >= 0) {                                   // the same for all of the workgroup
      if (tid == 0) path(1u);
      __syncthreads();
    }
    const double r = request >= 0 && a.repetition ? a.repetition[request] : 1.f, f = request >= 0 && a.frequency ? a.frequency[request] : 0.f, w = request >= 0 && a.presence ? a.presence[request] : 0.f;
    const int m = a.masks ? a.mask_rows[row] : -1;
    const unsigned* mask = (unsigned)m < (unsigned)a.n_masks ? a.masks + (long long)m * a.mask_stride + lo / 32 : nullptr;
    const T* from = reinterpret_cast<const T*>(a.logits) + (long long)row * a.row_stride + lo;
    T* to = reinterpret_cast<T*>(a.out) + (long long)row * a.out_stride + lo;
    constexpr unsigned ALL = E == 32 ? ~0u : (1u << E) - 1;
    auto changed = [&](T x, int t) {                   // an element that something applies to, but for the mask
      const unsigned n = counted ? count[t] : 0u, b = a.bias_tokens ? bias[t] : 0u;
      if (n == 0 && b == 0) return x;                  // a path's token that went
      double y = (float)x;
      if (n) y = y > 0.0 ? y / r : y * r;
      if (n & ~AL_PROMPT) y -= f * (n & ~AL_PROMPT) + w;
      if (b) y += a.bias_values[b - 1];
      return (T)(float)y;
    };
    const int groups = (hi - lo + E - 1) / E;
    for (int g0 = tid; g0 < groups; g0 += AL_BATCH * AL_THREADS) {
      V x[AL_BATCH];
      unsigned apply[AL_BATCH], out[AL_BATCH];         // bits of the group's elements: something applies, ruled out
#pragma unroll
      for (int u = 0; u < AL_BATCH; u++) {
        const int t = (g0 + u * AL_THREADS) * E;
        if (t >= hi - lo) break;
        apply[u] = any ? touched[t >> 5] >> (t & 31) & ALL : 0u;
        out[u] = mask ? ~mask[t >> 5] >> (t & 31) & ALL : 0u;
        const bool reads = out[u] != ALL && (!c.in_place || (apply[u] | out[u]));
        if (E > 1 && t + E > hi - lo) {
#pragma unroll
          for (int e = 0; e < E; e++)
            if (reads && t + e < hi - lo) x[u][e] = from[t + e];
        } else if (reads) {
          x[u] = *reinterpret_cast<const V*>(from + t);
        }
      }
#pragma unroll
      for (int u = 0; u < AL_BATCH; u++) {
        const int t = (g0 + u * AL_THREADS) * E;
        if (t >= hi - lo) break;
        if (c.in_place && !(apply[u] | out[u])) continue;
        if (apply[u] & ~out[u])
#pragma unroll
          for (int e = 0; e < E; e++)
            if ((apply[u] & ~out[u]) >> e & 1) x[u][e] = changed(x[u][e], t + e);
#pragma unroll
        for (int e = 0; e < E; e++)
          if (out[u] >> e & 1) x[u][e] = (T)-INFINITY;
        if (E > 1 && t + E > hi - lo) {
#pragma unroll
          for (int e = 0; e < E; e++)
            if (t + e < hi - lo) to[t + e] = x[u][e];
        } else {
          *reinterpret_cast<V*>(to + t) = x[u];
        }
      }
    }
    if (node >= 0) {
      __syncthreads();
      if (tid == 0) path(~0u);                         // less 1
    }
  }
}

template <typename T, int E>
hipError_t launch_adjust(hipStream_t s, const AdjustCall& c) {
  const bool counted = c.a.tokens || c.a.drafted;
  const size_t lds = ((size_t)c.part / 32 + (counted ? c.part : 0) + (c.a.bias_tokens ? c.part : 0)) * sizeof(unsigned);
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
  const AdjustCall c{*a, 8192, a->drafted ? 8 : 1, in_place};
  return op_result(a->dtype == STS_F32 ? launch_adjust<float>(s, c) : a->dtype == STS_BF16 ? launch_adjust<bf16>(s, c) : launch_adjust<f16>(s, c));
}
