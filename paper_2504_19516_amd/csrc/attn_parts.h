// What the attention kernels on the caller's pages share: the matrix instructions of their types, probabilities in two numbers of the type, lines of
// segments cut into shares.
#pragma once
#include "device_ops.h"

namespace sts {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float AS_RISE = 8.f;                   // how far scores may outgrow the reference of their exponentials, in powers of two
constexpr int AS_LDS_BASE = 1024;                // buffers filled by direct-to-LDS loads stay clear of address 0

template <typename T> struct Mfma;
template <> struct Mfma<bf16> {
  typedef bf16x8 V;
  static __device__ __forceinline__ f32x16 mul(V a, V b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<f16> {
  typedef f16x8 V;
  static __device__ __forceinline__ f32x16 mul(V a, V b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
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

}  // namespace sts
