// Layer norm of rows, its gradients, and the column sums that parameter
// gradients end with.
//
// A row's values stay in registers between the reductions: L lanes of a wave
// hold a row of up to 2048 (C units of eight each), a workgroup of 512 a wider
// one.  The mean, and then its error and the sum of squares around it, are two
// passes over the registers, so that a large mean costs no digits.
//
// Bound by memory: x is read and y written once forward; x and dy read and dx
// written backward, whose parameter gradients stay in registers until a workgroup
// has done all its rows.  1000513 x 128 fp32 205 us forward (5.0 TB/s), 309 backward
// (5.0 TB/s) and 7 for joining 1024 workgroups' sums; 8192 x 8192 bf16 62, 91 (4.4
// TB/s) and 7; 20011 x 391 of a 396 table fp16 15, 17 and 5.5 (2.1 TB/s: rows that
// start anywhere, whose 16-byte accesses cross lines, and a quarter of the lanes idle).
#include "rows_common.h"

namespace gnn {
namespace {

constexpr int LN_WAVES = 4, LN_WIDE = 512;

template <int T>
__device__ __forceinline__ void store8(elem_t<T> *row, int k, int K, const f8 &v) {
  typedef typename Raw8<T>::vec vec;
  typedef vec loose __attribute__((aligned(sizeof(elem_t<T>))));
  const vec r = __builtin_convertvector(v, vec);
  if (k + 8 <= K) {
    *(loose *)(row + k) = r;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (k + j < K) row[k + j] = r[j];
  }
}

template <int T, bool FULL>
__device__ __forceinline__ f8 values8(const elem_t<T> *row, int k, int K) {
  return to_f32<T>(FULL ? load8<T>(row, k) : load8_end<T>(row, k, K));
}

// Sums of V values over the lanes of a row: L lanes of a wave, or the workgroup
// (WIDE; `turn` says which half of `part` is free).
template <int V, bool WIDE>
__device__ __forceinline__ void row_sum(float (&v)[V], int L, float (*part)[LN_WIDE / 64][2],
                                        int &turn) {
  for (int o = 1; o < (WIDE ? 64 : L); o *= 2)
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] += __shfl_xor(v[i], o);
  if constexpr (WIDE) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < V; ++i) part[turn][wave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < LN_WIDE / 64; ++w) v[i] += part[turn][w][i];
    }
    turn ^= 1;
  }
}

template <bool WIDE>
struct RowOf {
  int64_t first, step;  // this lane's rows
  int u0, L;            // its first unit, units to the next one
  __device__ __forceinline__ explicit RowOf(int lanes) {
    if constexpr (WIDE) {
      L = LN_WIDE;
      u0 = threadIdx.x;
      first = blockIdx.x;
      step = gridDim.x;
    } else {
      L = lanes;
      const int lane = threadIdx.x & 63, per = 64 / L;
      u0 = lane % L;
      first = ((int64_t)blockIdx.x * LN_WAVES + (threadIdx.x >> 6)) * per + lane / L;
      step = (int64_t)gridDim.x * LN_WAVES * per;
    }
  }
};

template <int T, int C, bool WIDE, bool FULL>
__global__ __launch_bounds__(WIDE ? LN_WIDE : 64 * LN_WAVES) void layer_norm(LayerNormArgs a,
                                                                             int lanes) {
  __shared__ float part[2][LN_WIDE / 64][2];
  int turn = 0;
  const RowOf<WIDE> at(lanes);
  const int K = a.width;
  const float inv = 1.f / (float)K;
  f8 gamma[C], beta[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int k = 8 * (at.u0 + at.L * c);
    gamma[c] = values8<T_F32, FULL>(a.gamma, k, K);
    beta[c] = values8<T_F32, FULL>(a.beta, k, K);
  }
  // every lane of a wave goes round as often as its first: they add together
  const int64_t lead = WIDE ? at.first : at.first - (threadIdx.x & 63) / at.L;
  for (int64_t r0 = lead; r0 < a.n; r0 += at.step) {
    const int64_t r = r0 + (at.first - lead);
    const bool in = r < a.n;
    const elem_t<T> *row = (const elem_t<T> *)a.x + (in ? r : a.n - 1) * a.x_stride;
    f8 x[C];
    float s[1] = {0.f};
#pragma unroll
    for (int c = 0; c < C; ++c) x[c] = values8<T, FULL>(row, 8 * (at.u0 + at.L * c), K);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) s[0] += x[c][j];
    row_sum<1, WIDE>(s, at.L, part, turn);
    const float first = s[0] / (float)K;
    float t[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = x[c][j] - first;
        x[c][j] = d;
        const float e = FULL || 8 * (at.u0 + at.L * c) + j < K ? d : 0.f;
        t[0] += e * e;
        t[1] += e;
      }
    row_sum<2, WIDE>(t, at.L, part, turn);
    // The sum's roundings leave `first` off by some last places; the deviations' own mean
    // says by how much.  So a constant row deviates by nothing.
    const float off = t[1] * inv, mean = first + off, shift = mean - first;
    const float rstd = 1.f / sqrtf(fmaxf(t[0] * inv - off * off, 0.f) + a.eps);
    if (!in) continue;
    elem_t<T> *y = (elem_t<T> *)a.y + r * a.y_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      f8 v;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = (x[c][j] - shift) * rstd * gamma[c][j] + beta[c][j];
      store8<T>(y, 8 * (at.u0 + at.L * c), K, v);
    }
    if (at.u0 == 0 && a.mean) {
      a.mean[r] = mean;
      a.rstd[r] = rstd;
    }
  }
}

// dx = r (g - mean g - xh mean(g xh)), g = dy gamma, and this workgroup's part
// of dgamma = sum dy xh and dbeta = sum dy, which its lanes hold for their
// columns over all their rows.
template <int T, int C, bool WIDE, bool FULL>
__global__ __launch_bounds__(WIDE ? LN_WIDE : 64 * LN_WAVES) void layer_norm_backward(
    LayerNormArgs a, int lanes) {
  __shared__ float part[2][LN_WIDE / 64][2];
  extern __shared__ __attribute__((aligned(16))) float sums[];  // [LN_WAVES][2][width up to 8]
  int turn = 0;
  const RowOf<WIDE> at(lanes);
  const int K = a.width;
  const float inv = 1.f / (float)K;
  f8 gamma[C], dgamma[C], dbeta[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    gamma[c] = values8<T_F32, FULL>(a.gamma, 8 * (at.u0 + at.L * c), K);
    dgamma[c] = dbeta[c] = f8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  }
  const int64_t lead = WIDE ? at.first : at.first - (threadIdx.x & 63) / at.L;
  for (int64_t r0 = lead; r0 < a.n; r0 += at.step) {
    const int64_t r = r0 + (at.first - lead);
    const bool in = r < a.n;
    const int64_t rr = in ? r : a.n - 1;
    const elem_t<T> *xr = (const elem_t<T> *)a.x + rr * a.x_stride;
    const elem_t<T> *dr = (const elem_t<T> *)a.dy + rr * a.dy_stride;
    const float mean = a.mean[rr], rstd = a.rstd[rr];
    f8 x[C], d[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int k = 8 * (at.u0 + at.L * c);
      x[c] = values8<T, FULL>(xr, k, K);
      d[c] = values8<T, FULL>(dr, k, K);
    }
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float xh = (x[c][j] - mean) * rstd, g = d[c][j] * gamma[c][j];
        x[c][j] = xh;
        if (in) {  // d is zero past the row's end
          dgamma[c][j] += FULL || 8 * (at.u0 + at.L * c) + j < K ? d[c][j] * xh : 0.f;
          dbeta[c][j] += d[c][j];
        }
        s[0] += g;
        s[1] += FULL || 8 * (at.u0 + at.L * c) + j < K ? g * xh : 0.f;
        d[c][j] = g;
      }
    row_sum<2, WIDE>(s, at.L, part, turn);
    if (!in) continue;
    const float m0 = s[0] * inv, m1 = s[1] * inv;
    elem_t<T> *dx = (elem_t<T> *)a.dx + r * a.dx_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      f8 v;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = rstd * (d[c][j] - m0 - x[c][j] * m1);
      store8<T>(dx, 8 * (at.u0 + at.L * c), K, v);
    }
  }
  float *out = a.part + (int64_t)blockIdx.x * 2 * K;
  if constexpr (WIDE) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int k = 8 * (at.u0 + at.L * c);
      store8<T_F32>(out, k, K, dgamma[c]);
      store8<T_F32>(out + K, k, K, dbeta[c]);
    }
  } else {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, pad = (K + 7) & ~7;
#pragma unroll
    for (int c = 0; c < C; ++c) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        for (int o = at.L; o < 64; o *= 2) {
          dgamma[c][j] += __shfl_xor(dgamma[c][j], o);
          dbeta[c][j] += __shfl_xor(dbeta[c][j], o);
        }
      const int k = 8 * (at.u0 + at.L * c);
      if (lane < at.L && k < K) {
        *(f8 *)(sums + (wave * 2) * pad + k) = dgamma[c];
        *(f8 *)(sums + (wave * 2 + 1) * pad + k) = dbeta[c];
      }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * K; k += 64 * LN_WAVES) {
      const int at0 = k < K ? k : pad + k - K;
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < LN_WAVES; ++w) v += sums[w * 2 * pad + at0];
      out[k] = v;
    }
  }
}

// ---- column sums ----
// Rows to at most SUM_PARTS rows of partial sums: L lanes hold a row's units, as
// above, and go down the table; blockIdx.y takes 512 columns each.
constexpr int SUM_PARTS = 512, SUM_DIRECT = 1024;

template <int T>
__global__ __launch_bounds__(64 * LN_WAVES) void column_parts(SumArgs a, int L) {
  __shared__ __attribute__((aligned(16))) float sums[LN_WAVES][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = 64 / L;
  const int k = 8 * (blockIdx.y * 64 + lane % L);
  f8 s = f8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (k < a.width) {
    const int64_t step = (int64_t)gridDim.x * LN_WAVES * per;
#pragma unroll 4
    for (int64_t r = ((int64_t)blockIdx.x * LN_WAVES + wave) * per + lane / L; r < a.n; r += step) {
      const elem_t<T> *row = (const elem_t<T> *)a.x + r * a.x_stride;
      s += to_f32<T>(k + 8 <= a.width ? load8<T>(row, k) : load8_end<T>(row, k, a.width));
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    for (int o = L; o < 64; o *= 2) s[j] += __shfl_xor(s[j], o);
  if (lane < L) *(f8 *)&sums[wave][8 * lane] = s;
  __syncthreads();
  for (int i = threadIdx.x; i < 8 * L; i += 64 * LN_WAVES) {
    const int c = blockIdx.y * 512 + i;
    if (c >= a.width) break;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < LN_WAVES; ++w) v += sums[w][i];
    a.part[(int64_t)blockIdx.x * a.width + c] = v;
  }
}

// Sums of n rows of partial sums, sixteen rows at a time to a workgroup.
__global__ __launch_bounds__(1024) void column_join(SumArgs a, const float *part, int64_t n) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < a.width) {
#pragma unroll 8
    for (int64_t r = wave; r < n; r += 16) s += part[r * a.width + c];
  }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave || c >= a.width) return;
  s = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) s += sums[w][lane];
  const int which = c < a.split ? 0 : 1, at = which ? c - a.skip : c;
  if (at < 0 || at >= a.split || !a.y[which]) return;
  if (a.y_type == T_F32)
    ((float *)a.y[which])[at] = s;
  else if (a.y_type == T_BF16)
    ((__bf16 *)a.y[which])[at] = (__bf16)s;
  else
    ((_Float16 *)a.y[which])[at] = (_Float16)s;
}

int lanes_of(int units) {
  int L = 1;
  while (L < units && L < 64) L *= 2;
  return L;
}

struct LnShape {
  bool wide, full;
  int C, L;
};
LnShape ln_shape(int width) {
  const int units = (width + 7) / 8;
  LnShape s;
  s.wide = units > 256;
  s.L = s.wide ? LN_WIDE : lanes_of(units);
  s.C = 1;
  while (s.L * s.C < units) s.C *= 2;
  s.full = s.L * s.C * 8 == width;
  return s;
}

template <int T, int C, bool WIDE, bool FULL>
hipError_t ln_go(const LayerNormArgs &a, int L, bool backward, hipStream_t stream) {
  const dim3 block(WIDE ? LN_WIDE : 64 * LN_WAVES);
  if (backward) {
    const size_t lds = WIDE ? 0 : (size_t)LN_WAVES * 2 * ((a.width + 7) & ~7) * 4;
    return launch_lds(layer_norm_backward<T, C, WIDE, FULL>,
                      dim3((unsigned)layer_norm_parts(a.n, a.width)), block, lds, stream, a, L);
  }
  const int64_t rows = WIDE ? 1 : LN_WAVES * (64 / L);
  // four rows to a wave before there are more than 1024 workgroups: gamma and beta
  // are loaded once for all of them
  const int64_t all = (a.n + rows - 1) / rows;
  const int64_t grid =
      WIDE ? std::min<int64_t>(all, 1024)
           : std::min<int64_t>(all, std::min<int64_t>(4096, std::max<int64_t>(1024, all / 4)));
  return launch(layer_norm<T, C, WIDE, FULL>, dim3((unsigned)grid), block, 0, stream, a, L);
}

template <int T, bool WIDE, bool FULL>
hipError_t ln_c(const LayerNormArgs &a, const LnShape &s, bool backward, hipStream_t stream) {
  if (s.C == 1) return ln_go<T, 1, WIDE, FULL>(a, s.L, backward, stream);
  if (s.C == 2) return ln_go<T, 2, WIDE, FULL>(a, s.L, backward, stream);
  return ln_go<T, 4, WIDE, FULL>(a, s.L, backward, stream);
}

template <int T>
hipError_t ln_t(const LayerNormArgs &a, bool backward, hipStream_t stream) {
  const LnShape s = ln_shape(a.width);
  if (s.wide)
    return s.full ? ln_c<T, true, true>(a, s, backward, stream)
                  : ln_c<T, true, false>(a, s, backward, stream);
  return s.full ? ln_c<T, false, true>(a, s, backward, stream)
                : ln_c<T, false, false>(a, s, backward, stream);
}

hipError_t ln(const LayerNormArgs &a, bool backward, hipStream_t stream) {
  if (a.type == T_F32) return ln_t<T_F32>(a, backward, stream);
  if (a.type == T_BF16) return ln_t<T_BF16>(a, backward, stream);
  return ln_t<T_F16>(a, backward, stream);
}

}  // namespace

// Workgroups of the backward pass: as many as the chip holds, so that few
// partial sums are written.
int64_t layer_norm_parts(int64_t n, int32_t width) {
  const LnShape s = ln_shape(width);
  const int64_t rows = s.wide ? 1 : LN_WAVES * (64 / s.L);
  return std::min<int64_t>((n + rows - 1) / rows, s.wide ? 512 : 1024);
}

hipError_t launch_layer_norm(const LayerNormArgs &a, hipStream_t stream) {
  return ln(a, false, stream);
}
hipError_t launch_layer_norm_backward(const LayerNormArgs &a, hipStream_t stream) {
  return ln(a, true, stream);
}

namespace {
// Rows of partial sums that are written first: none of up to SUM_DIRECT rows that lie as
// such do (fp32, without gaps).
int64_t colsum_parts(int64_t n, int32_t width, bool as_parts) {
  if (n == 0 || (as_parts && n <= SUM_DIRECT)) return 0;
  const int64_t rows = LN_WAVES * (64 / lanes_of((width + 7) / 8)) * 4;
  return std::min<int64_t>((n + rows - 1) / rows, SUM_PARTS);
}
}  // namespace

size_t colsum_scratch(int64_t n, int32_t width, bool as_parts) {
  return (size_t)colsum_parts(n, width, as_parts) * width * 4;
}

hipError_t launch_colsum(const SumArgs &a, hipStream_t stream) {
  const float *part = (const float *)a.x;
  int64_t n = a.n;
  if (const int64_t parts = colsum_parts(n, a.width, a.x_type == T_F32 && a.x_stride == a.width)) {
    const int L = lanes_of((a.width + 7) / 8);
    const dim3 grid((unsigned)parts, (unsigned)((a.width + 511) / 512));
    const dim3 block(64 * LN_WAVES);
    const hipError_t e = a.x_type == T_F32    ? launch(column_parts<T_F32>, grid, block, 0, stream, a, L)
                         : a.x_type == T_BF16 ? launch(column_parts<T_BF16>, grid, block, 0, stream, a, L)
                                              : launch(column_parts<T_F16>, grid, block, 0, stream, a, L);
    if (e != hipSuccess) return e;
    part = a.part;
    n = grid.x;
  }
  return launch(column_join, dim3((unsigned)((a.width + 63) / 64)), dim3(1024), 0, stream, a, part, n);
}

}  // namespace gnn
