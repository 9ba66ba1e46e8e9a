// Rotary positions of Q and K rows, and the append of K and V rows to their pages; the same behind a norm of each head.
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
// Norms of heads: y = x / sqrt(mean(x^2) + eps) * gain before the rotation, in 32 bits. A head's row is then a run of neighbouring lanes (a power of two of them; those
// beyond its vectors hold none), which add up their squares; the rows are still read once. Rows that do not come in vectors take a wave each and are read twice. The norms
// hide behind memory: the prefill below takes 38 to 41 us with them again and again on the same rows, 48 on rows that change (46.7 without norms); 130 rows 5.5 us.
//
// Bound by memory for prefills (8192 rows of 32 + 8 heads of 128: 201 MB in 44 us, 4.6 TB/s, where a plain copy takes 38), by latency for decodes
// (64 rows 4 us). V columns stored 1 KB in a row by neighbouring lanes, both halves of a page at once, were level.
#include <algorithm>
#include <cmath>

#include "device_ops.h"

namespace sts {
namespace {

constexpr int RP_THREADS = 256, RP_MAX_PAIRS = 128;   // head elements that turn: up to 256
// Rows from which a workgroup takes a page's 16 (its V then leaves in whole 32-byte columns); below it takes one, 32 heads at a time. 300
// rows of 32 + 8 heads 6.1 us with one row a workgroup, 5.6 with 16, but 6.6 and 7.6 of as many requests; 1000 rows 11.2 and 7.6, 12.6 and 12.3.
constexpr int RP_PAGE_ROWS = 512, RP_HEADS = 32;
// Workgroups wanted of launches with 16 rows each, in up to eight parts of their rotations and of their V: 512 / 1024 / 2048 wanted, 8192 rows took
// 45 / 44 / 44 us, with neighbours as pairs 52 / 44 / 45.
constexpr int RP_WORKGROUPS = 1024, RP_PARTS = 8;

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
  // one power, then products: 128 of them are off by 128 roundings at most, and a call for a few rows would else wait for the host
  const double ratio = std::pow(base, -2.0 / R);
  double w = 1.0;
  for (int i = 0; i < pairs; i++, w *= ratio) {
    const double slow = w / factor;
    double share = 1.0;                               // of the unscaled angle
    if (r.scaling == STS_ROPE_LINEAR) share = 0.0;
    if (r.scaling == STS_ROPE_BANDS) share = std::min(std::max((len * w / two_pi - low) / (high - low), 0.0), 1.0);
    if (r.scaling == STS_ROPE_RAMP) share = 1.0 - std::min(std::max((i - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
    f[i] = share == 1.0 ? w : slow + (w - slow) * share;
    if (!(f[i] < 1e15)) return false;                 // not a finite number of turns that leaves a fraction
  }
  return true;
}

bool rope_turns(const sts_rope& r, RopeTurns* t) {
  double f[RP_MAX_PAIRS];
  if (!rope_frequencies(r, f)) return false;
  for (int i = 0; i < r.rotary_dim / 2; i++) {
    double turns = f[i] * 0.15915494309189533577;
    if (turns >= 1.0) turns -= std::floor(turns);
    t->step[i] = (uint64_t)(turns * 18446744073709551616.0);
  }
  return true;
}

constexpr int RP_NORM_D = 512;                        // elements of a head that is normed
struct HeadNorms { const void *q_gain, *k_gain; int dtype, lanes; float eps, offset; };      // lanes: of a head's row

struct RopeCall {
  sts_rope_rows a;
  int pairs, interleaved, turn_parts;
  bool v_vec;                                    // V's rows and the pages can be moved 16 bytes at a time
  float magnitude;
};

// Cosine and sine of a fraction of a turn (2^-32 each): the nearest quarter turn and what is left, at most pi / 4, by their series up to
// t^10 and t^9, which end 2e-9 from the functions.
__device__ __forceinline__ f32x2 cos_sin(unsigned turn) {
  const unsigned quarter = (turn + 0x20000000u) >> 30;
  const float t = (float)(int)(turn - (quarter << 30)) * 1.4629180792671596e-9f, q = t * t;       // 2 pi / 2^32
  const float s = t * fmaf(q, fmaf(q, fmaf(q, fmaf(q, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
  const float c = fmaf(q, fmaf(q, fmaf(q, fmaf(q, fmaf(q, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
  return f32x2{(quarter + 1) & 2 ? -x : x, quarter & 2 ? -y : y};
}

template <typename T, int N> struct VecOf { typedef T type __attribute__((ext_vector_type(N))); };
template <typename T> struct VecOf<T, 1> { typedef T type; };

__device__ __forceinline__ float gain_at(const void* gain, int dtype, int e) {
  return !gain ? 1.f : dtype == STS_F32 ? reinterpret_cast<const float*>(gain)[e] : dtype == STS_BF16 ? (float)reinterpret_cast<const bf16*>(gain)[e] : (float)reinterpret_cast<const f16*>(gain)[e];
}
// The sum over runs of `lanes` neighbouring lanes.
__device__ __forceinline__ float run_sum(float x, int lanes) {
  for (int s = 1; s < lanes; s <<= 1) x += __shfl_xor(x, s, 64);
  return x;
}

// ROWS: rows of a workgroup (1, or a page's 16). E: elements at a time, in aligned vectors; pairs come in whole vectors. N: HeadNorms, or none.
template <typename T, int ROWS, int E, typename... N>
__global__ void __launch_bounds__(RP_THREADS) rope_kernel(RopeCall c, RopeTurns turns, N... norms) {
  constexpr bool VEC = E > 1, NORM = sizeof...(N) > 0;
  typedef typename VecOf<T, E>::type V;
  const sts_rope_rows& a = c.a;
  __shared__ f32x2 trig[ROWS * RP_MAX_PAIRS];          // [row][pair]: cosine, sine
  __shared__ int places[ROWS];
  const int row0 = blockIdx.x * ROWS, rows = min(ROWS, a.rows - row0), tid = threadIdx.x;
  const int d = a.d, P = c.pairs, R = 2 * P;
  // The launch's y: parts of the rotations first, then of the heads whose V is appended.
  const bool turns_rows = (int)blockIdx.y < c.turn_parts;
  if (tid < ROWS) {                                    // -1: not appended
    const int p = a.pool && tid < rows ? a.places[row0 + tid] : -1;
    places[tid] = p >= 0 && p / OP_PAGE < a.pool_pages ? p : -1;
  }
  const size_t head_elems = (size_t)2 * OP_PAGE * d;
  auto page_head = [&](int place, int h) { return reinterpret_cast<T*>(a.pool) + ((size_t)(place / OP_PAGE) * a.n_kv + h) * head_elems; };
  if (turns_rows) {
    // Tasks of a head's row: a pair (of vectors), or one vector of neighbours or of elements that pass. The workgroup's part of all of them
    const int pair_tasks = !VEC ? P : c.interleaved ? d / E : P / E, tasks = !VEC ? P + d - R : c.interleaved ? pair_tasks : pair_tasks + (d - R) / E;
    int lanes = 1;                                     // of a head's row; whole ones are then a workgroup's
    if constexpr (NORM) lanes = (norms.lanes, ...);
    const int of_row = (a.n_q + a.n_kv) * (NORM ? lanes : tasks);
    const long long units = (long long)rows * (NORM ? a.n_q + a.n_kv : of_row);
    const int t0 = (int)(units * blockIdx.y / c.turn_parts) * lanes, t1 = (int)(units * (blockIdx.y + 1) / c.turn_parts) * lanes;
    const int r_first = t0 / of_row, r_end = (t1 + of_row - 1) / of_row;
    for (int i = tid + r_first * P; i < r_end * P; i += RP_THREADS) {
      const int r = ROWS == 1 ? 0 : i / P, p = i - r * P;
      const uint64_t phase = (uint64_t)(int64_t)a.positions[row0 + r] * turns.step[p];
      const f32x2 cs = cos_sin((unsigned)(phase >> 32));
      trig[i] = f32x2{cs[0] * c.magnitude, cs[1] * c.magnitude};
    }
    __shared__ float gains[2][NORM ? RP_NORM_D : 1];
    if constexpr (NORM) {
      const HeadNorms n = (norms, ...);
      for (int e = tid; e < d; e += RP_THREADS) {
        gains[0][e] = n.q_gain ? gain_at(n.q_gain, n.dtype, e) + n.offset : 1.f;
        gains[1][e] = n.k_gain ? gain_at(n.k_gain, n.dtype, e) + n.offset : 1.f;
      }
    }
    auto root = [&](float squares) {
      float eps = 0.f;
      if constexpr (NORM) eps = (norms.eps, ...);
      return __builtin_amdgcn_rsqf(squares / (float)d + eps);
    };
    struct Task { int r, h, task; };                   // heads from n_q on are K's
    auto task_of = [&](int t) {
      const int r = ROWS == 1 ? 0 : t / of_row, q = t - r * of_row, h = q / (NORM ? lanes : tasks);
      return Task{r, h, q - h * (NORM ? lanes : tasks)};
    };
    auto source = [&](const Task& k) {
      return k.h < a.n_q ? reinterpret_cast<const T*>(a.q) + (row0 + k.r) * a.q_stride + k.h * d : reinterpret_cast<const T*>(a.k) + (row0 + k.r) * a.k_stride + (k.h - a.n_q) * d;
    };
    struct Targets { T *row, *page; bool to_row, to_page; };           // pointers by value: through memory they would be generic ones
    auto targets = [&](const Task& k) {
      const bool q = k.h < a.n_q;
      const int h = q ? 0 : k.h - a.n_q, p = q ? -1 : places[k.r];
      T* row = q ? reinterpret_cast<T*>(a.q_out) + (row0 + k.r) * a.q_out_stride + k.h * d : reinterpret_cast<T*>(a.k_out) + (row0 + k.r) * a.k_out_stride + h * d;
      return Targets{row, page_head(max(p, 0), h) + max(p, 0) % OP_PAGE * d, q || a.k_out, p >= 0};
    };
    if constexpr (VEC) {
      constexpr int DEPTH = ROWS == 1 ? 1 : 2;         // tasks of a thread under way: 8192 rows 44.4 / 44.0 / 48.4 us with 1 / 2 / 4
      V x[DEPTH], y[DEPTH];
      Task k[DEPTH];
      auto is_pair = [&](const Task& q) { return !c.interleaved && q.task < pair_tasks; };
      auto place_in = [&](const Task& q) { return c.interleaved || q.task < pair_tasks ? q.task * E : R + (q.task - pair_tasks) * E; };
      auto load = [&](int t) {
#pragma unroll
        for (int u = 0; u < DEPTH; u++) {
          if (t + u * RP_THREADS >= t1) break;
          k[u] = task_of(t + u * RP_THREADS);
          if constexpr (NORM) {
            if (k[u].task >= tasks) continue;          // a lane beyond the vectors
          }
          const T* src = source(k[u]) + place_in(k[u]);
          x[u] = *reinterpret_cast<const V*>(src);
          if (is_pair(k[u])) y[u] = *reinterpret_cast<const V*>(src + P);
        }
      };
      load(t0 + tid);                                  // on the way while the angles are made
      __syncthreads();
      for (int t = t0 + tid; t < t1; t += DEPTH * RP_THREADS) {
        if (t != t0 + tid) load(t);
#pragma unroll
        for (int u = 0; u < DEPTH; u++) {
          if (t + u * RP_THREADS >= t1) break;
          const Targets to = targets(k[u]);
          const f32x2* tr = trig + k[u].r * P;
          const int at = place_in(k[u]);
          if constexpr (NORM) {
            const bool pair = is_pair(k[u]), here = k[u].task < tasks;
            float v[E], w[E], squares = 0.f;
#pragma unroll
            for (int e = 0; e < E; e++) {
              v[e] = (float)x[u][e]; w[e] = (float)y[u][e];
              squares += here ? v[e] * v[e] + (pair ? w[e] * w[e] : 0.f) : 0.f;
            }
            const float f = root(run_sum(squares, lanes));
            if (!here) continue;
            const float* g = gains[k[u].h >= a.n_q] + at;
#pragma unroll
            for (int e = 0; e < E; e++) v[e] = v[e] * f * g[e];
            if (pair) {
#pragma unroll
              for (int e = 0; e < E; e++) {
                w[e] = w[e] * f * g[P + e];
                const f32x2 cs = tr[at + e];
                float p, q;
                rotate_pair(v[e], w[e], cs[0], cs[1], &p, &q);
                x[u][e] = (T)p; y[u][e] = (T)q;
              }
              if (to.to_row) *reinterpret_cast<V*>(to.row + at + P) = y[u];
              if (to.to_page) *reinterpret_cast<V*>(to.page + at + P) = y[u];
            } else if (at < R) {
#pragma unroll
              for (int e = 0; e < E; e += 2) {
                const f32x2 cs = tr[(at + e) / 2];
                float p, q;
                rotate_pair(v[e], v[e + 1], cs[0], cs[1], &p, &q);
                x[u][e] = (T)p; x[u][e + 1] = (T)q;
              }
            } else {
#pragma unroll
              for (int e = 0; e < E; e++) x[u][e] = (T)v[e];
            }
          } else if (is_pair(k[u])) {
#pragma unroll
            for (int e = 0; e < E; e++) {
              float v, w;
              const f32x2 cs = tr[at + e];
              rotate_pair((float)x[u][e], (float)y[u][e], cs[0], cs[1], &v, &w);
              x[u][e] = (T)v; y[u][e] = (T)w;
            }
            if (to.to_row) *reinterpret_cast<V*>(to.row + at + P) = y[u];
            if (to.to_page) *reinterpret_cast<V*>(to.page + at + P) = y[u];
          } else if (at < R) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
              float v, w;
              const f32x2 cs = tr[(at + e) / 2];
              rotate_pair((float)x[u][e], (float)x[u][e + 1], cs[0], cs[1], &v, &w);
              x[u][e] = (T)v; x[u][e + 1] = (T)w;
            }
          }
          if (to.to_row) *reinterpret_cast<V*>(to.row + at) = x[u];
          if (to.to_page) *reinterpret_cast<V*>(to.page + at) = x[u];
        }
      }
    } else if constexpr (NORM) {                       // 64 lanes a head's row
      __syncthreads();
      const int lane = tid & 63;
      for (int t = t0 + tid; t < t1; t += RP_THREADS) {
        Task k = task_of(t);
        const T* src = source(k);
        const Targets to = targets(k);
        const float* g = gains[k.h >= a.n_q];
        float squares = 0.f;
        for (int e = lane; e < d; e += 64) squares += (float)src[e] * (float)src[e];
        const float f = root(run_sum(squares, 64));
        auto put = [&](int e, float v) {
          if (to.to_row) to.row[e] = (T)v;
          if (to.to_page) to.page[e] = (T)v;
        };
        for (k.task = lane; k.task < tasks; k.task += 64) {
          if (k.task < P) {
            const int e = c.interleaved ? 2 * k.task : k.task, w = c.interleaved ? e + 1 : e + P;
            const f32x2 cs = trig[k.r * P + k.task];
            float p, q;
            rotate_pair((float)src[e] * f * g[e], (float)src[w] * f * g[w], cs[0], cs[1], &p, &q);
            put(e, p);
            put(w, q);
          } else {
            const int e = R + k.task - P;
            put(e, (float)src[e] * f * g[e]);
          }
        }
      }
    } else {
      __syncthreads();
      for (int t = t0 + tid; t < t1; t += RP_THREADS) {
        const Task k = task_of(t);
        const T* src = source(k);
        const Targets to = targets(k);
        auto put = [&](int e, T v) {
          if (to.to_row) to.row[e] = v;
          if (to.to_page) to.page[e] = v;
        };
        if (k.task < P) {
          const int e = c.interleaved ? 2 * k.task : k.task, f = c.interleaved ? e + 1 : e + P;
          const f32x2 cs = trig[k.r * P + k.task];
          float v, w;
          rotate_pair((float)src[e], (float)src[f], cs[0], cs[1], &v, &w);
          put(e, (T)v);
          put(f, (T)w);
        } else {
          put(R + k.task - P, src[R + k.task - P]);
        }
      }
    }
    return;
  }
  const int v_part = blockIdx.y - c.turn_parts, v_parts = gridDim.y - c.turn_parts;
  const int kh0 = a.n_kv * v_part / v_parts, k_heads = a.n_kv * (v_part + 1) / v_parts - kh0;
  __syncthreads();
  // V, transposed inside the page
  if (ROWS == OP_PAGE && sizeof(T) == 2 && c.v_vec) {
    typedef typename VecOf<T, 16 / sizeof(T)>::type V;
    // Runs of rows in neighbouring slots of a page: the workgroup stores those that begin in its 16 rows, to their end, so that a page's 32 bytes
    // of a column are written by one workgroup whatever slot a prompt begins in (a page shared by two of them took a third longer: its
    // lines go to memory twice, in parts, from two L2s).
    constexpr int SPAN = 2 * OP_PAGE;
    __shared__ __align__(16) T tile[ROWS == OP_PAGE ? SPAN : 1][128 + 8];
    typedef T T4 __attribute__((ext_vector_type(4)));
    // places of the rows from the first on, one a lane (-1: not appended, or behind the last row), and where runs and halves of pages begin
    const int lane = tid & 63, at = row0 + lane;
    auto place_at = [&](int r) {
      const int p = r >= 0 && r < a.rows ? a.places[r] : -1;
      return p >= 0 && p / OP_PAGE < a.pool_pages ? p : -1;
    };
    const int mine = lane < SPAN ? place_at(at) : -1, before = lane < SPAN ? place_at(at - 1) : -1;
    const unsigned runs = (unsigned)__ballot(mine < 0 || mine % OP_PAGE == 0 || mine != before + 1), halves = runs | (unsigned)__ballot(mine % 8 == 0);
    auto place = [&](int r) { return __builtin_amdgcn_readlane(mine, r); };
    const int first = min(__builtin_ctz(runs | 1u << OP_PAGE), rows);
    const int end = first == rows ? rows : rows < ROWS ? rows : OP_PAGE + __builtin_ctz(runs >> OP_PAGE | 1u << (OP_PAGE - 1));
    const int at_once = 128 / d, col = tid & 127, half = __builtin_amdgcn_readfirstlane(tid >> 7) * 8, my_h = col / d, e = col - my_h * d;
    const int in_r = tid >> 4, in_col = (tid & 15) * 8;           // a vector of the tile, and one 16 rows on
    V next[2];
    auto fetch = [&](int h) {
      const int hh = min(h + in_col / d, k_heads - 1);
#pragma unroll
      for (int u = 0; u < 2; u++)
        if (first + in_r + 16 * u < end)
          next[u] = *reinterpret_cast<const V*>(reinterpret_cast<const T*>(a.v) + (row0 + first + in_r + 16 * u) * a.v_stride + (kh0 + hh) * d + in_col % d);
    };
    fetch(0);
    for (int h = 0; h < k_heads; h += at_once) {
      __syncthreads();
#pragma unroll
      for (int u = 0; u < 2; u++)
        if (first + in_r + 16 * u < end) *reinterpret_cast<V*>(&tile[in_r + 16 * u][in_col]) = next[u];
      if (h + at_once < k_heads) fetch(h + at_once);
      __syncthreads();
      if (h + my_h >= k_heads) continue;
      for (int r = first; r < end;) {                             // wave-uniform: the slots of this half of a page, eight or four together where they can be
        const int p = place(r);
        if (p < 0 || p % OP_PAGE / 8 * 8 != half) { r++; continue; }
        const int run = min(r + 1 < SPAN ? __builtin_ctzll((unsigned long long)(halves >> (r + 1)) | 1ull << 32) + 1 : 1, end - r);
        T* to = page_head(p, kh0 + h + my_h) + OP_PAGE * d + e * OP_PAGE + p % OP_PAGE;
        if (run == 8) {
          V v;
#pragma unroll
          for (int u = 0; u < 16 / (int)sizeof(T); u++) v[u] = tile[r - first + u][col];
          *reinterpret_cast<V*>(to) = v;
          r += 8;
        } else if (p % 4 == 0 && run >= 4) {
          T4 v;
#pragma unroll
          for (int u = 0; u < 4; u++) v[u] = tile[r - first + u][col];
          *reinterpret_cast<T4*>(to) = v;
          r += 4;
        } else {
          *to = tile[r - first][col];
          r++;
        }
      }
    }
  } else {
    for (int i = tid; i < rows * k_heads * d; i += RP_THREADS) {
      const int r = ROWS == 1 ? 0 : i / (k_heads * d), h = i / d % k_heads, e = i % d, p = places[r];
      if (p >= 0) page_head(p, kh0 + h)[OP_PAGE * d + e * OP_PAGE + p % OP_PAGE] = reinterpret_cast<const T*>(a.v)[(row0 + r) * a.v_stride + (kh0 + h) * d + e];
    }
  }
}

template <typename T, int ROWS, int E, typename... N>
hipError_t launch_rows(hipStream_t s, const RopeCall& c, const RopeTurns& t, const N&... norms) {
  const int blocks = (c.a.rows + ROWS - 1) / ROWS, heads = c.a.n_q + c.a.n_kv;
  RopeCall call = c;
  call.turn_parts = ROWS == 1 ? (heads + RP_HEADS - 1) / RP_HEADS : std::max(1, std::min({(RP_WORKGROUPS + blocks - 1) / blocks, heads, RP_PARTS}));
  const int v_parts = !c.a.pool ? 0 : ROWS == 1 ? 1 : std::max(1, std::min({(RP_WORKGROUPS + blocks - 1) / blocks / 2, c.a.n_kv, RP_PARTS}));
  return launch(rope_kernel<T, ROWS, E, N...>, dim3(blocks, call.turn_parts + v_parts), dim3(RP_THREADS), 0, s, call, t, norms...);
}
template <typename T, int E, typename... N>
hipError_t launch_vectors(hipStream_t s, const RopeCall& c, const RopeTurns& t, const N&... norms) {
  return c.a.rows < RP_PAGE_ROWS ? launch_rows<T, 1, E>(s, c, t, norms...) : launch_rows<T, OP_PAGE, E>(s, c, t, norms...);
}
// Lanes of a head's row in vectors of e elements: a power of two
int norm_lanes(const RopeCall& c, int e) {
  const int R = 2 * c.pairs, vectors = c.interleaved ? c.a.d / e : c.pairs / e + (c.a.d - R) / e;
  int lanes = 1;
  while (lanes < vectors) lanes *= 2;
  return lanes;
}
template <typename T, typename... N>
hipError_t launch_rope(hipStream_t s, const RopeCall& c0, const RopeTurns& t, N... norms) {
  RopeCall c = c0;
  const sts_rope_rows& a = c.a;
  auto rows_fit = [&](const void* p, int64_t stride, int e) { return !p || (aligned(p, e * sizeof(T)) && stride % e == 0); };
  // whole vectors of e elements: heads, pairs and rows
  auto fits = [&](int e) {
    bool lanes = true;
    if constexpr (sizeof...(N) > 0) lanes = ((norms.lanes = norm_lanes(c, e)), ...) <= 64;
    return lanes && a.d % e == 0 && (c.interleaved ? 2 * c.pairs : c.pairs) % e == 0 && rows_fit(a.q, a.q_stride, e) && rows_fit(a.q_out, a.q_out_stride, e) && rows_fit(a.k, a.k_stride, e) &&
           rows_fit(a.k_out, a.k_out_stride, e) && rows_fit(a.pool, 0, e);
  };
  c.v_vec = a.pool && sizeof(T) == 2 && aligned(a.pool, 16) && rows_fit(a.v, a.v_stride, 8);
  if (fits(16 / sizeof(T))) return launch_vectors<T, 16 / sizeof(T)>(s, c, t, norms...);
  if (sizeof(T) == 2 && fits(4)) return launch_vectors<T, 4>(s, c, t, norms...);
  if constexpr (sizeof...(N) > 0) ((norms.lanes = 64), ...);
  return launch_vectors<T, 1>(s, c, t, norms...);
}

// sts_op_rope, with the norms of the heads or none.
template <typename... N>
int rope_rows(const sts_rope* rope, const sts_rope_rows* a, void* stream, const N&... norms) {
  RopeTurns turns;
  if (!rope || !a || !rope_turns(*rope, &turns)) return STS_EINVAL;
  if (a->dtype < STS_F32 || a->dtype > STS_F16 || a->rows < 0 || a->rows > (1 << 27) || a->n_q < 0 || a->n_kv < 0 || a->d < rope->rotary_dim || a->d > 1024 || a->n_q > 4096 || a->n_kv > 4096) return STS_EINVAL;
  if (a->n_q > 0 && (!a->q || !a->q_out)) return STS_EINVAL;
  if (a->n_kv > 0 && (!a->k || (!a->k_out && !a->pool))) return STS_EINVAL;
  if (a->pool && (a->n_kv < 1 || !a->v || !a->places || a->dtype == STS_F32 || (a->d != 64 && a->d != 128) || a->pool_pages < 0)) return STS_EINVAL;
  // rows lie one behind the other; only a row turned in place may be read and written
  const int64_t q_row = (int64_t)a->n_q * a->d, k_row = (int64_t)a->n_kv * a->d;
  if (a->rows > 1 && ((a->n_q > 0 && (a->q_stride < q_row || a->q_out_stride < q_row)) || (a->n_kv > 0 && (a->k_stride < k_row || (a->k_out && a->k_out_stride < k_row) ||
      (a->pool && a->v_stride < k_row))))) return STS_EINVAL;
  auto elements = [&](const void* p) { return aligned(p, dtype_bytes(a->dtype)); };
  if ((a->n_q > 0 && !(elements(a->q) && elements(a->q_out))) || (a->n_kv > 0 && !(elements(a->k) && elements(a->k_out))) || (a->pool && !(elements(a->v) && elements(a->pool)))) return STS_EINVAL;
  if ((a->q && a->q == a->q_out && a->q_stride != a->q_out_stride) || (a->k && a->k == a->k_out && a->k_stride != a->k_out_stride)) return STS_EINVAL;
  if (a->rows == 0 || (a->n_q == 0 && a->n_kv == 0)) return STS_OK;
  if (!a->positions) return STS_EINVAL;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  OnStreamDevice dev(s);
  if (dev.error() != hipSuccess) return op_result(dev.error());
  sts_rope_rows rows = *a;
  if (rows.n_q == 0) rows.q = nullptr, rows.q_out = nullptr;
  if (rows.n_kv == 0) rows.k = nullptr, rows.k_out = nullptr;
  const RopeCall c{rows, rope->rotary_dim / 2, rope->interleaved, 0, false, rope->magnitude == 0.f ? 1.f : rope->magnitude};
  const hipError_t e = a->dtype == STS_F32 ? launch_rope<float>(s, c, turns, norms...) : a->dtype == STS_BF16 ? launch_rope<bf16>(s, c, turns, norms...) : launch_rope<f16>(s, c, turns, norms...);
  return op_result(e);
}

}  // namespace
}  // namespace sts

using namespace sts;

extern "C" int sts_rope_frequencies(const sts_rope* rope, double* out) {
  if (!rope || !out || !rope_frequencies(*rope, out)) return STS_EINVAL;
  return STS_OK;
}

extern "C" int sts_op_rope(const sts_rope* rope, const sts_rope_rows* a, void* stream) { return rope_rows(rope, a, stream); }

extern "C" int sts_op_norm_rope(const sts_head_norm* norm, const sts_rope* rope, const sts_rope_rows* a, void* stream) {
  if (!norm || !a || norm->dtype < STS_F32 || norm->dtype > STS_F16 || (norm->offset_one != 0 && norm->offset_one != 1) || !(norm->eps >= 0.f) || !std::isfinite(norm->eps) || a->d > RP_NORM_D) return STS_EINVAL;
  // of heads that are none nothing is read, their gains neither
  const void *q_gain = a->n_q > 0 ? norm->q_gain : nullptr, *k_gain = a->n_kv > 0 ? norm->k_gain : nullptr;
  if (!aligned(q_gain, dtype_bytes(norm->dtype)) || !aligned(k_gain, dtype_bytes(norm->dtype))) return STS_EINVAL;
  return rope_rows(rope, a, stream, HeadNorms{q_gain, k_gain, norm->dtype, 0, norm->eps, norm->offset_one ? 1.f : 0.f});
}
