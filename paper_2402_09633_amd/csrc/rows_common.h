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

// Elements k .. k + 7 of a row of K; zeros from K on, which is not read past.
template <int T>
__device__ __forceinline__ Raw8<T> load8(const elem_t<T> *row, int k, int K) {
  Raw8<T> r;
  if (k + 8 <= K) {
    __builtin_memcpy(&r.v, row + k, sizeof r.v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) r.v[j] = k + j < K ? row[k + j] : (elem_t<T>)0;
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
__device__ __forceinline__ float max_abs8(const f8 &x, float m) {
  // the bits of |x| order as x does, infinities and NaN above all numbers
#pragma unroll
  for (int j = 0; j < 8; ++j)
    m = __uint_as_float(max(__float_as_uint(m), __float_as_uint(x[j]) & 0x7fffffffu));
  return m;
}

__device__ __forceinline__ float quant_scale(float top) {
  if (!(__float_as_uint(top) < 0x7f800000u)) return __uint_as_float(0x7fc00000u);
  const float s = top / 127.f;
  return s < 1.17549435e-38f ? 0.f : s;
}

// The factor that quantize8 multiplies by: 1 / s, 0 where the values are 0.
__device__ __forceinline__ float quant_inv(float s) { return s > 0.f ? 1.f / s : 0.f; }

// t = x * inv is within 1.5 * 2^-24 * 127 < 1.2e-5 of x / s.  Where its
// distance from the nearest whole number is not within that of a half, the
// nearest whole number is the one of x / s.  Otherwise x - t s decides, which
// is exact in fp32 (a multiple of the smaller of ulp(x) and ulp(s), below s).
__device__ __forceinline__ float quant_exact(float x, float s, float inv) {
  float t = rintf(x * inv);
  const float r2 = 2.f * __builtin_fmaf(-t, s, x);
  const float dir = r2 > 0.f ? 1.f : -1.f;
  const bool odd = t - 2.f * truncf(0.5f * t) != 0.f;
  if (fabsf(r2) > s || (fabsf(r2) == s && odd)) t += dir;
  return t;
}

// Eight values to bytes.  Adding 1.5 * 2^23 rounds to a whole number (to
// nearest, ties to even) whose two's complement is the sum's low byte.
__device__ __forceinline__ u2 quantize8(const f8 &x, float s, float inv) {
  constexpr float MAGIC = 12582912.f;
  float t[8], far = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    t[j] = __builtin_fmaf(x[j], inv, MAGIC);
    const float r = __builtin_fmaf(x[j], inv, -(t[j] - MAGIC));
    far = fmaxf(far, fabsf(r));
  }
  if (far > 0.5f - 2e-5f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = quant_exact(x[j], s, inv) + MAGIC;
  }
  u2 q;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(t[4 * h + 1]),
                                              __float_as_uint(t[4 * h]), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(t[4 * h + 3]),
                                              __float_as_uint(t[4 * h + 2]), 0x04000c0cu);
    q[h] = inv == 0.f ? 0u : lo | hi;
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
  auto at = [&](int32_t g) { return min(max(off[g], 0), n_rows); };
  int32_t base = 0, step = (G + 63) / 64;
  if (step > 1) {
    const int32_t g = lane * step;
    const uint64_t m = __ballot(g < G && at(min(g, G - 1)) / PM + g <= tile);
    base = (max((int)__popcll(m), 1) - 1) * step;
  }
  // the last of up to 64 groups from base on whose first number is <= tile
  const int32_t g = base + lane;
  const bool in = lane < (step > 1 ? step : 64) && g < G;
  const uint64_t m = __ballot(in && at(min(g, G - 1)) / PM + g <= tile);
  const int32_t n = __popcll(m);
  if (n == 0) return TileRows{0, 0, 0};
  const int32_t gg = base + n - 1;
  const int32_t lo = at(gg), hi = at(gg + 1);
  const int64_t r0 = lo + (int64_t)(tile - (lo / PM + gg)) * PM;
  if (r0 < lo || r0 >= hi) return TileRows{gg, 0, 0};
  return TileRows{gg, (int32_t)r0, hi};
}

}  // namespace
}  // namespace gnn
