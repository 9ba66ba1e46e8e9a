// Rotary positions of Q and K rows, and the append of K and V rows to their pages.
//
// Pair i of a head's first R elements -- (i, i + R/2), or (2i, 2i + 1) interleaved -- turns by the angle position * f_i, where f_i is
// theta^(-2i/R) scaled for long contexts (rope_turns below); elements from R on pass. One pass: rows are read once and written once, to
// q_out, to k_out and to the pool's pages [K: 16 x d | V^T: d x 16].
//
// Angles: f_i / 2 pi is kept as a 64-bit binary fraction of a turn, so position * f_i modulo one turn is one 64-bit product that drops
// whole turns exactly: the angle of position 2^20 is as good as that of position 1 (fp32 products are off by 0.06 radians there). The
// host makes the fractions in 64 bits and hands them over as a kernel argument; a workgroup computes its rows' cosines and sines once
// and keeps them in LDS for all heads.
//
// Bound by memory for prefills and by latency for decodes.
#include <cmath>

#include "device_ops.h"

namespace sts {
namespace {

constexpr int RP_THREADS = 256, RP_MAX_PAIRS = 128;   // head elements that turn: up to 256

struct RopeTurns { uint64_t step[RP_MAX_PAIRS]; };    // pair i: 2^64 * f_i / 2 pi, modulo 2^64

// Radians a token of each pair; false for a description out of range.
bool rope_frequencies(const sts_rope& r, double* f) {
  if (r.rotary_dim < 2 || r.rotary_dim % 2 || r.rotary_dim > 2 * RP_MAX_PAIRS || !(r.theta > 0.f) || !std::isfinite(r.theta) || !std::isfinite(r.magnitude) || r.magnitude < 0.f) return false;
  if (r.interleaved != 0 && r.interleaved != 1) return false;
  const int R = r.rotary_dim, pairs = R / 2;
  const double theta = r.theta, factor = r.factor, low = r.low, high = r.high, len = r.original_len, two_pi = 6.283185307179586476925;
  if (r.scaling != STS_ROPE_PLAIN && !(factor > 0.0 && std::isfinite(factor))) return false;
  double base = theta, lo = 0.0, hi = 0.0;
  switch (r.scaling) {
    case STS_ROPE_PLAIN: case STS_ROPE_LINEAR: break;
    case STS_ROPE_BASE:
      if (R < 4) return false;                        // the slowest pair is the only one
      base = theta * std::pow(factor, R / (R - 2.0));
      break;
    case STS_ROPE_BANDS:
      if (r.original_len < 1 || !(low > 0.0) || !(high > low) || !std::isfinite(high)) return false;
      break;
    case STS_ROPE_RAMP: {
      if (r.original_len < 1 || !(low > 0.0) || !(high >= low) || !std::isfinite(high) || !(theta > 1.0)) return false;
      auto pair = [&](double beta) { return R * std::log(len / (beta * two_pi)) / (2.0 * std::log(theta)); };
      lo = std::max(std::floor(pair(high)), 0.0);
      hi = std::min(std::ceil(pair(low)), R - 1.0);
      break;
    }
    default: return false;
  }
  for (int i = 0; i < pairs; i++) {
    const double w = std::pow(base, -2.0 * i / R), slow = w / factor;
    double share = 1.0;                               // of the unscaled angle
    if (r.scaling == STS_ROPE_LINEAR) share = 0.0;
    if (r.scaling == STS_ROPE_BANDS) share = std::min(std::max((len * w / two_pi - low) / (high - low), 0.0), 1.0);
    if (r.scaling == STS_ROPE_RAMP) share = 1.0 - std::min(std::max((i - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
    f[i] = share == 1.0 ? w : slow + (w - slow) * share;
    if (!std::isfinite(f[i])) return false;
  }
  return true;
}

bool rope_turns(const sts_rope& r, RopeTurns* t) {
  double f[RP_MAX_PAIRS];
  if (!rope_frequencies(r, f)) return false;
  for (int i = 0; i < RP_MAX_PAIRS; i++) {
    long double turns = i < r.rotary_dim / 2 ? f[i] / 6.283185307179586476925286766559L : 0.0L;
    turns -= std::floor(turns);
    const long double scaled = std::ldexp(turns, 64);
    t->step[i] = scaled >= 18446744073709551615.0L ? 0 : (uint64_t)scaled;
  }
  return true;
}

struct RopeCall {
  sts_rope_rows a;
  int pairs, interleaved;
  float magnitude;
};

template <typename T> __device__ __forceinline__ float to_f(T x) { return (float)x; }

// ROWS: rows of a workgroup. VEC: 8 elements (4 of fp32) at a time; needs aligned rows and pairs that come in whole vectors.
template <typename T, int ROWS, bool VEC>
__global__ void __launch_bounds__(RP_THREADS) rope_kernel(RopeCall c, RopeTurns turns) {
  constexpr int E = 16 / sizeof(T);
  const sts_rope_rows& a = c.a;
  extern __shared__ float trig[];                      // [ROWS][pairs][cosine, sine]
  const int row0 = blockIdx.x * ROWS, rows = min(ROWS, a.rows - row0), tid = threadIdx.x;
  const int d = a.d, P = c.pairs, R = 2 * P;
  for (int i = tid; i < rows * P; i += RP_THREADS) {
    const int r = i / P, p = i % P;
    const uint64_t phase = (uint64_t)(int64_t)a.positions[row0 + r] * turns.step[p];
    float s, co;
    sincospif((float)(int)(phase >> 32) * 0x1p-31f, &s, &co);          // the top 32 bits, as a signed fraction of a half turn
    trig[2 * i] = co * c.magnitude;
    trig[2 * i + 1] = s * c.magnitude;
  }
  __syncthreads();
  // this workgroup's share of the heads (the launch splits them over y)
  const int qh0 = (int)((long long)a.n_q * blockIdx.y / gridDim.y), qh1 = (int)((long long)a.n_q * (blockIdx.y + 1) / gridDim.y);
  const int kh0 = (int)((long long)a.n_kv * blockIdx.y / gridDim.y), kh1 = (int)((long long)a.n_kv * (blockIdx.y + 1) / gridDim.y);
  const size_t head_elems = (size_t)2 * OP_PAGE * d;
  auto place_of = [&](int r) -> int {                  // -1: not appended
    if (!a.pool) return -1;
    const int p = a.places[row0 + r];
    return p >= 0 && p / OP_PAGE < a.pool_pages ? p : -1;
  };
  auto page_head = [&](int place, int h) { return reinterpret_cast<T*>(a.pool) + ((size_t)(place / OP_PAGE) * a.n_kv + h) * head_elems; };
  // One head's row from src to up to two destinations: a pair (of vectors) or a passing element (vector) at a time.
  auto turn = [&](const T* src, T* to, T* to2, const float* tr, int task) {
    if constexpr (VEC) {
      typedef vec16<T> V;
      auto put = [&](int at, const V& v) {
        if (to) *reinterpret_cast<V*>(to + at) = v;
        if (to2) *reinterpret_cast<V*>(to2 + at) = v;
      };
      if (c.interleaved) {
        V v = *reinterpret_cast<const V*>(src + task * E);
        if (task * E < R) {
#pragma unroll
          for (int e = 0; e < E; e += 2) {
            const float* t = tr + task * E + e;
            float u, w;
            rotate_pair((float)v[e], (float)v[e + 1], t[0], t[1], &u, &w);
            v[e] = (T)u; v[e + 1] = (T)w;
          }
        }
        put(task * E, v);
      } else if (task * E < P) {
        V x = *reinterpret_cast<const V*>(src + task * E), y = *reinterpret_cast<const V*>(src + P + task * E);
#pragma unroll
        for (int e = 0; e < E; e++) {
          const float* t = tr + 2 * (task * E + e);
          float u, w;
          rotate_pair((float)x[e], (float)y[e], t[0], t[1], &u, &w);
          x[e] = (T)u; y[e] = (T)w;
        }
        put(task * E, x);
        put(P + task * E, y);
      } else {
        const int at = R + (task - P / E) * E;
        put(at, *reinterpret_cast<const V*>(src + at));
      }
    } else {
      auto put = [&](int at, T v) {
        if (to) to[at] = v;
        if (to2) to2[at] = v;
      };
      if (task < P) {
        const int i = c.interleaved ? 2 * task : task, j = c.interleaved ? i + 1 : i + P;
        float u, w;
        rotate_pair((float)src[i], (float)src[j], tr[2 * task], tr[2 * task + 1], &u, &w);
        put(i, (T)u);
        put(j, (T)w);
      } else {
        put(R + task - P, src[R + task - P]);
      }
    }
  };
  const int tasks = VEC ? (c.interleaved ? d / E : P / E + (d - R) / E) : P + d - R;     // of a head's row
  const int q_tasks = (qh1 - qh0) * tasks, k_tasks = (kh1 - kh0) * tasks;
  for (int i = tid; i < rows * q_tasks; i += RP_THREADS) {
    const int r = i / q_tasks, h = qh0 + i % q_tasks / tasks;
    turn(reinterpret_cast<const T*>(a.q) + (row0 + r) * a.q_stride + h * d, reinterpret_cast<T*>(a.q_out) + (row0 + r) * a.q_out_stride + h * d, nullptr, trig + 2 * P * r,
         i % tasks);
  }
  for (int i = tid; i < rows * k_tasks; i += RP_THREADS) {
    const int r = i / k_tasks, h = kh0 + i % k_tasks / tasks, place = place_of(r);
    T* to = a.k_out ? reinterpret_cast<T*>(a.k_out) + (row0 + r) * a.k_out_stride + h * d : nullptr;
    T* page = place < 0 ? nullptr : page_head(place, h) + (place % OP_PAGE) * d;
    if (to || page) turn(reinterpret_cast<const T*>(a.k) + (row0 + r) * a.k_stride + h * d, to, page, trig + 2 * P * r, i % tasks);
  }
  if (!a.pool) return;
  for (int i = tid; i < rows * (kh1 - kh0) * d; i += RP_THREADS) {
    const int r = i / ((kh1 - kh0) * d), h = kh0 + i / d % (kh1 - kh0), e = i % d, place = place_of(r);
    if (place >= 0) page_head(place, h)[OP_PAGE * d + e * OP_PAGE + place % OP_PAGE] = reinterpret_cast<const T*>(a.v)[(row0 + r) * a.v_stride + h * d + e];
  }
}

template <typename T, bool VEC>
hipError_t launch_rope(hipStream_t s, const RopeCall& c, const RopeTurns& t) {
  constexpr int ROWS = 4;
  const int heads = std::max(c.a.n_q, c.a.n_kv);
  const int split = std::max(1, std::min(heads / 8, 4));
  return launch(rope_kernel<T, ROWS, VEC>, dim3((c.a.rows + ROWS - 1) / ROWS, split), dim3(RP_THREADS), (size_t)ROWS * c.pairs * 8, s, c, t);
}
template <typename T>
hipError_t launch_rope(hipStream_t s, const RopeCall& c, const RopeTurns& t) {
  constexpr int E = 16 / sizeof(T);
  const sts_rope_rows& a = c.a;
  auto rows_fit = [&](const void* p, int64_t stride) { return !p || (aligned(p, 16) && stride % E == 0); };
  const bool vec = a.d % E == 0 && (c.interleaved ? 2 * c.pairs % E == 0 : c.pairs % E == 0) && rows_fit(a.q, a.q_stride) && rows_fit(a.q_out, a.q_out_stride) &&
                   rows_fit(a.k, a.k_stride) && rows_fit(a.k_out, a.k_out_stride) && rows_fit(a.pool, 0);
  return vec ? launch_rope<T, true>(s, c, t) : launch_rope<T, false>(s, c, t);
}

}  // namespace
}  // namespace sts

using namespace sts;

extern "C" int sts_rope_frequencies(const sts_rope* rope, double* out) {
  if (!rope || !out || !rope_frequencies(*rope, out)) return STS_EINVAL;
  return STS_OK;
}

extern "C" int sts_op_rope(const sts_rope* rope, const sts_rope_rows* a, void* stream) {
  RopeTurns turns;
  if (!rope || !a || !rope_turns(*rope, &turns)) return STS_EINVAL;
  if (a->dtype < STS_F32 || a->dtype > STS_F16 || a->rows < 0 || a->n_q < 0 || a->n_kv < 0 || a->d < rope->rotary_dim || a->d > 1024 || a->n_q > 4096 || a->n_kv > 4096) return STS_EINVAL;
  if (a->n_q > 0 && (!a->q || !a->q_out)) return STS_EINVAL;
  if (a->n_kv > 0 && (!a->k || (!a->k_out && !a->pool))) return STS_EINVAL;
  if (a->pool && (a->n_kv < 1 || !a->v || !a->places || a->dtype == STS_F32 || (a->d != 64 && a->d != 128) || a->pool_pages < 0)) return STS_EINVAL;
  // rows lie one behind the other; only a row turned in place may be read and written
  const int64_t q_row = (int64_t)a->n_q * a->d, k_row = (int64_t)a->n_kv * a->d;
  if (a->rows > 1 && ((a->n_q > 0 && (a->q_stride < q_row || a->q_out_stride < q_row)) || (a->n_kv > 0 && (a->k_stride < k_row || (a->k_out && a->k_out_stride < k_row) ||
      (a->pool && a->v_stride < k_row))))) return STS_EINVAL;
  if ((a->q && a->q == a->q_out && a->q_stride != a->q_out_stride) || (a->k && a->k == a->k_out && a->k_stride != a->k_out_stride)) return STS_EINVAL;
  if (a->rows == 0 || (a->n_q == 0 && a->n_kv == 0)) return STS_OK;
  if (!a->positions) return STS_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  const RopeCall c{*a, rope->rotary_dim / 2, rope->interleaved, rope->magnitude == 0.f ? 1.f : rope->magnitude};
  const hipError_t e = a->dtype == STS_F32 ? launch_rope<float>(s, c, turns) : a->dtype == STS_BF16 ? launch_rope<bf16>(s, c, turns) : launch_rope<f16>(s, c, turns);
  return op_result(e);
}
