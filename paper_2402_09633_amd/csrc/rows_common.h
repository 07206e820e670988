// Device helpers of the row operators (rows.hip, linear.hip): rows of fp32,
// bf16 or fp16 read eight values at a time, their rounding to 8 bits, and the
// group of a workgroup's rows.
#pragma once

#include "device_common.h"

namespace gnn {
namespace {

typedef int32_t i4 __attribute__((ext_vector_type(4)));
typedef int32_t i16v __attribute__((ext_vector_type(16)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// Types of row elements, as GNN_FP32, GNN_BF16, GNN_F16 and GNN_INT8.
constexpr int T_F32 = 0, T_BF16 = 1, T_F16 = 2, T_I8 = 3;
template <int T>
struct Elem;
template <>
struct Elem<T_F32> {
  typedef float type;
};
template <>
struct Elem<T_BF16> {
  typedef __bf16 type;
};
template <>
struct Elem<T_F16> {
  typedef _Float16 type;
};
template <>
struct Elem<T_I8> {
  typedef int8_t type;
};
template <int T>
using elem_t = typename Elem<T>::type;

typedef int8_t c8 __attribute__((ext_vector_type(8)));

// Eight elements as they lie in memory.  Rows start at any element, so the
// load claims no more alignment than an element has (the hardware takes
// 16-byte loads from any address).
template <int T>
struct Raw8 {
  typedef elem_t<T> vec __attribute__((ext_vector_type(8)));
  vec v;
};

// Elements k .. k + 7 of a row.  ONCE: they are not read again, and need no
// place in the caches.
template <int T, bool ONCE = false>
__device__ __forceinline__ Raw8<T> load8(const elem_t<T> *row, int k) {
  typedef typename Raw8<T>::vec loose __attribute__((aligned(sizeof(elem_t<T>))));
  Raw8<T> r;
  if constexpr (ONCE)
    r.v = __builtin_nontemporal_load((const loose *)(row + k));
  else
    r.v = *(const loose *)(row + k);
  return r;
}

// The same of a row of K, with zeros from K on, which is not read past: from K
// >= 8 on, the row's last eight elements moved down by as many as lie before k.
template <int T, bool ONCE = false>
__device__ __forceinline__ Raw8<T> load8_end(const elem_t<T> *row, int k, int K) {
  if (K < 8) {  // the same for all lanes
    Raw8<T> r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r.v[j] = k + j < K ? row[k + j] : (elem_t<T>)0;
    return r;
  }
  const int at = min(k, K - 8), d = min(k - at, 8);
  Raw8<T> r = load8<T, ONCE>(row, at);
  if constexpr (T == T_I8) {
    const uint64_t v = __builtin_bit_cast(uint64_t, r.v);
    const uint64_t m = d < 8 ? v >> (8 * d) : 0;
    r.v = __builtin_bit_cast(typename Raw8<T>::vec, m);
  } else {
    if constexpr (T == T_F32) {
#pragma unroll
      for (int b = 1; b <= 8; b *= 2)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float up = j + b < 8 ? r.v[j + b] : 0.f;
          r.v[j] = d & b ? up : r.v[j];
        }
    } else {
      u4 w = __builtin_bit_cast(u4, r.v);
#pragma unroll
      for (int b = 1; b <= 4; b *= 2)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t up = j + b < 4 ? w[j + b] : 0u;
          w[j] = d & (2 * b) ? up : w[j];
        }
      const uint32_t odd = 16 * (d & 1);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w[j] = (uint32_t)((((uint64_t)(j < 3 ? w[j + 1] : 0u) << 32) | w[j]) >> odd);
      r.v = __builtin_bit_cast(typename Raw8<T>::vec, w);
    }
  }
  return r;
}

template <int T>
__device__ __forceinline__ f8 to_f32(const Raw8<T> &r) {
  if constexpr (T == T_F32) return r.v;
  return __builtin_convertvector(r.v, f8);
}

// ---- rows to 8 bits ----
// A row's scale is s = fl32(max |x| / 127) and its values are the whole
// numbers nearest to x / s (ties to even); s = 0 where that is below the
// smallest normal number (such a row counts as zero), NaN where the row holds
// an infinity or a NaN (its values are then 0, and what is computed from them
// NaN).
// The bits of |x| order as |x| does, infinities and NaN above all numbers: the
// largest of eight is taken as whole numbers, of 16-bit types two at a time.
typedef uint16_t s2 __attribute__((ext_vector_type(2)));
template <int T>
__device__ __forceinline__ uint32_t max_bits(const Raw8<T> &r, uint32_t m) {
  if constexpr (T == T_F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(r.v[j]) & 0x7fffffffu);
  } else {
    const u4 w = __builtin_bit_cast(u4, r.v);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      m = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(
                                           __builtin_bit_cast(s2, m),
                                           __builtin_bit_cast(s2, w[j] & 0x7fff7fffu)));
  }
  return m;
}

// The value that max_bits found.
template <int T>
__device__ __forceinline__ float top_of(uint32_t m) {
  if constexpr (T == T_F32) {
    return __uint_as_float(m);
  } else {
    const uint16_t h = (uint16_t)max(m & 0xffffu, m >> 16);
    return (float)__builtin_bit_cast(elem_t<T>, h);
  }
}

// The largest value of L = 2^i neighbouring lanes, in all of them.
__device__ __forceinline__ float lanes_max(float v, int L) {
  uint32_t m = __float_as_uint(v);
  auto step = [&](uint32_t o) { m = max(m, o); };
  if (L >= 2) step(__builtin_amdgcn_mov_dpp(m, 0xb1, 0xf, 0xf, true));   // lane ^ 1
  if (L >= 4) step(__builtin_amdgcn_mov_dpp(m, 0x4e, 0xf, 0xf, true));   // lane ^ 2
  if (L >= 8) step(__builtin_amdgcn_mov_dpp(m, 0x141, 0xf, 0xf, true));  // 7 - lane of 8
  if (L >= 16) step(__builtin_amdgcn_mov_dpp(m, 0x140, 0xf, 0xf, true)); // 15 - lane of 16
  if (L >= 32) step((uint32_t)__shfl_xor((int)m, 16));
  if (L >= 64) step((uint32_t)__shfl_xor((int)m, 32));
  return __uint_as_float(m);
}

__device__ __forceinline__ float quant_scale(float top) {
  if (!(__float_as_uint(top) < 0x7f800000u)) return __uint_as_float(0x7fc00000u);
  const float s = top / 127.f;
  return s < 1.17549435e-38f ? 0.f : s;
}

// What a row of type T is multiplied by, so that one fused multiply-add rounds
// x / s exactly (adding 1.5 * 2^23 rounds to a whole number, ties to even, whose
// two's complement is the sum's low byte).
//
// 16-bit types.  With c = top / 127 and s = c (1 + d), |d| <= 2^-24, a quotient
// x / c is exactly half way between two whole numbers, or at least 1 / (2 * 2047
// * 127) > 1.9e-6 of itself away from there (x and top are whole multiples of
// one number, below 2^11 but for powers of two).  In the second case x / s and
// x * f, for f within 2^-23 of 1 / c, lie on the same side.  In the first the
// sign of d says where x / s lies, and f is taken on that side of 1 / c.  Where
// d = 0 the quotient is a true tie: the whole numbers that a factor below and
// one above 1 / c lead to are then its neighbours, and half their sum rounds to
// the even one (without a tie they are the same).
//
// fp32.  Factors one step below and above 1 / s round alike unless x / s is next
// to a half.  Then half the sum h of what they lead to, a and b, is that half, and
// x - h s says on which side x / s lies.  It is formed as 2 (x - a s) + (a - b) s:
// both steps are exact in fp32 (multiples of the smaller of ulp(x) and ulp(s), at
// most s), also for the smallest scales, half of whose last place is no fp32 number.
struct Quant {
  float s, lo, hi;
  bool zero, tie;
};

__device__ __forceinline__ float step_up(float x, int by) {  // x > 0
  return __uint_as_float(__float_as_uint(x) + (uint32_t)by);
}

template <int T>
__device__ __forceinline__ Quant quant_of(float top) {
  Quant q;
  q.s = quant_scale(top);
  q.zero = !(q.s > 0.f);
  q.tie = false;
  if constexpr (T == T_F32) {
    const float inv = 1.f / q.s;
    q.lo = step_up(inv, -1);
    q.hi = step_up(inv, 1);
  } else {
    const float d = __builtin_fmaf(q.s, 127.f, -top);
    const float f = 127.f / top, e = __builtin_fmaf(f, top, -127.f);
    const float below = e >= 0.f ? step_up(f, -1) : f, above = e <= 0.f ? step_up(f, 1) : f;
    q.lo = d >= 0.f ? below : above;
    q.hi = above;
    q.tie = d == 0.f;
  }
  return q;
}

constexpr float ROUND_MAGIC = 12582912.f;

// The low bytes of eight sums.
__device__ __forceinline__ u2 pack_bytes(const float (&t)[8]) {
  u2 q;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(t[4 * h + 1]),
                                              __float_as_uint(t[4 * h]), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(t[4 * h + 3]),
                                              __float_as_uint(t[4 * h + 2]), 0x04000c0cu);
    q[h] = lo | hi;
  }
  return q;
}

template <int T>
__device__ __forceinline__ u2 quantize8(const f8 &x, const Quant &z) {
  float t[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) t[j] = __builtin_fmaf(x[j], z.lo, ROUND_MAGIC);
  u2 q = pack_bytes(t);
  if constexpr (T == T_F32) {
    float u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = __builtin_fmaf(x[j], z.hi, ROUND_MAGIC);
    const u2 p = pack_bytes(u);
    if (((p[0] ^ q[0]) | (p[1] ^ q[1])) != 0 || z.zero) {
      asm volatile("");  // a branch, not selected values: it is hardly ever taken
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = t[j] - ROUND_MAGIC, b = u[j] - ROUND_MAGIC;
        const float h = 0.5f * (a + b);
        const float r = __builtin_fmaf(2.f, __builtin_fmaf(-a, z.s, x[j]), (a - b) * z.s);
        t[j] = (h + (r == 0.f ? 0.f : __builtin_copysignf(0.25f, r))) + ROUND_MAGIC;
      }
      q = pack_bytes(t);
      if (z.zero) q = u2{0u, 0u};
    }
  } else if (z.tie || z.zero) {
    asm volatile("");
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float u = __builtin_fmaf(x[j], z.hi, ROUND_MAGIC);
      t[j] = 0.5f * ((t[j] - ROUND_MAGIC) + (u - ROUND_MAGIC)) + ROUND_MAGIC;
    }
    q = pack_bytes(t);
    if (z.zero) q = u2{0u, 0u};
  }
  return q;
}

// launch() with more than 64 KiB of dynamic LDS allowed.
template <typename... P, typename... A>
hipError_t launch_lds(void (*k)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t stream,
                      A &&...args) {
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void *)k,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  return launch(k, grid, block, lds, stream, std::forward<A>(args)...);
}

// ---- groups ----
// Rows group_off[g] .. group_off[g + 1] - 1 of the (ordered) rows form group
// g.  Tiles of PM rows are numbered so that every group's first tile follows
// from its offset alone: group g owns the tile numbers from off[g] / PM + g up
// to the next group's, which are at least as many as it has tiles (a number
// past its last tile has no rows).  A wave finds the group of a number with
// two steps of 64 comparisons.  Offsets are clamped into [0, n_rows], so that
// no value of theirs leads out of range.
struct TileRows {
  int32_t g, r0, r1;  // group, first row, end of the group's rows
};

__device__ __forceinline__ TileRows find_tile(const int32_t *__restrict__ off, int32_t G,
                                              int32_t n_rows, int32_t tile, int32_t PM) {
  if (!off) return TileRows{0, tile * PM, n_rows};
  const int lane = threadIdx.x & 63;
  auto at = [&](int32_t g) { return min(max(off[min(g, G)], 0), n_rows); };
  int32_t base = 0;
  const int32_t step = (G + 63) / 64;
  if (step > 1) {
    const int32_t g = lane * step;
    const uint64_t m = __ballot(g < G && at(g) / PM + g <= tile);
    base = (max((int)__popcll(m), 1) - 1) * step;
  }
  // the last of up to 64 groups from base on whose first number is <= tile
  const int32_t g = base + lane;
  const bool in = lane < (step > 1 ? step : 64) && g < G;
  const int32_t first = at(g), end = at(g + 1);
  const uint64_t m = __ballot(in && first / PM + g <= tile);
  const int32_t n = __popcll(m);
  if (n == 0) return TileRows{0, 0, 0};
  const int32_t gg = base + n - 1;
  const int32_t lo = __builtin_amdgcn_readlane(first, n - 1),
                hi = __builtin_amdgcn_readlane(end, n - 1);
  const int64_t r0 = lo + (int64_t)(tile - (lo / PM + gg)) * PM;
  if (r0 < lo || r0 >= hi) return TileRows{gg, 0, 0};
  return TileRows{gg, (int32_t)r0, hi};
}

}  // namespace
}  // namespace gnn
