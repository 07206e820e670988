// The global norm of many tensors, and their scaling.  Both read everything
// once, so HBM bounds them; a list of tensors goes with the launch's arguments,
// and every workgroup takes CLIP_TILE elements of one of them.  302M bf16 elements in
// 192 tensors, 341 us a call; under a profiler, which slows them, squares 146 us (4.1
// TB/s), the norm 6 and scaling 213 (5.7 TB/s, some of it from the last-level cache).
#include "rows_common.h"

namespace gnn {
namespace {

// The tensor of workgroup b: the last whose first tile is <= b (a tensor
// without elements has none).
__device__ __forceinline__ int tensor_of(const ClipList &l, int32_t b) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int i = 0; i < CLIP_LIST; i += 64) {
    const int at = i + lane;
    n += (int)__popcll(__ballot(at < l.count && l.tile[min(at, CLIP_LIST)] <= b));
  }
  return __builtin_amdgcn_readfirstlane(n - 1);
}

// Squares are formed and added in 64 bits: no gradient of 32 bits over- or
// underflows there, and memory is slower all the same.
template <int T>
__device__ __forceinline__ double squares_of(const void *p, int64_t first, int64_t n) {
  const elem_t<T> *x = (const elem_t<T> *)p;
  double s = 0.0;
#pragma unroll 4
  for (int i = 0; i < CLIP_TILE / 2048; ++i) {
    const int64_t k = first + (i * 256 + (int)threadIdx.x) * 8;
    if (k + 8 <= n) {
      const f8 v = to_f32<T>(load8<T>(x + k, 0));
#pragma unroll
      for (int j = 0; j < 8; ++j) s = __builtin_fma((double)v[j], (double)v[j], s);
    } else {
      for (int64_t q = k; q < n; ++q) {
        const double v = (double)(float)x[q];
        s = __builtin_fma(v, v, s);
      }
    }
  }
  return s;
}

__device__ __forceinline__ double block_sum(double s, double *part, int waves) {
#pragma unroll
  for (int o = 1; o < 64; o *= 2) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  s = part[0];
  for (int w = 1; w < waves; ++w) s += part[w];
  return s;
}

__global__ __launch_bounds__(256) void clip_squares(ClipList l, double *out) {
  __shared__ double part[4];
  const int t = tensor_of(l, blockIdx.x);
  const int64_t first = (int64_t)((int32_t)blockIdx.x - l.tile[t]) * CLIP_TILE;
  double s;
  if (l.type[t] == T_F32)
    s = squares_of<T_F32>(l.x[t], first, l.n[t]);
  else if (l.type[t] == T_BF16)
    s = squares_of<T_BF16>(l.x[t], first, l.n[t]);
  else
    s = squares_of<T_F16>(l.x[t], first, l.n[t]);
  s = block_sum(s, part, 4);
  if (threadIdx.x == 0) out[blockIdx.x] = s;
}

__global__ __launch_bounds__(1024) void clip_norm(const double *in, int64_t n, float max_norm,
                                                  float *norm, float *scale) {
  __shared__ double part[16];
  double s = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += in[i];
  s = block_sum(s, part, 16);
  if (threadIdx.x) return;
  const float v = (float)sqrt(s), c = max_norm / (v + 1e-6f);
  *norm = v;
  *scale = c > 1.f ? 1.f : c;  // a NaN stays one
}

template <int T>
__device__ __forceinline__ void scale_tile(const void *from, void *to, int64_t first, int64_t n,
                                           float c) {
  typedef typename Raw8<T>::vec vec;
  typedef vec loose __attribute__((aligned(sizeof(elem_t<T>))));
  const elem_t<T> *x = (const elem_t<T> *)from;
  elem_t<T> *y = (elem_t<T> *)to;
#pragma unroll 4
  for (int i = 0; i < CLIP_TILE / 2048; ++i) {
    const int64_t k = first + (i * 256 + (int)threadIdx.x) * 8;
    if (k + 8 <= n) {
      f8 v = to_f32<T>(load8<T>(x + k, 0));
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= c;
      *(loose *)(y + k) = __builtin_convertvector(v, vec);
    } else {
      for (int64_t q = k; q < n; ++q) y[q] = (elem_t<T>)((float)x[q] * c);
    }
  }
}

// Last tiles first: what the sum of squares read last is still in the caches.
__global__ __launch_bounds__(256) void clip_scale(ClipList l, const float *scale) {
  const int32_t b = (int32_t)(gridDim.x - 1 - blockIdx.x);
  const int t = tensor_of(l, b);
  const int64_t first = (int64_t)(b - l.tile[t]) * CLIP_TILE;
  const float c = *scale;
  if (l.type[t] == T_F32)
    scale_tile<T_F32>(l.x[t], l.y[t], first, l.n[t], c);
  else if (l.type[t] == T_BF16)
    scale_tile<T_BF16>(l.x[t], l.y[t], first, l.n[t], c);
  else
    scale_tile<T_F16>(l.x[t], l.y[t], first, l.n[t], c);
}

}  // namespace

hipError_t launch_squares(const ClipList &l, double *part, hipStream_t stream) {
  return launch(clip_squares, dim3((unsigned)l.tile[l.count]), dim3(256), 0, stream, l, part);
}

hipError_t launch_norm_scale(const double *part, int64_t n, float max_norm, float *norm,
                             float *scale, hipStream_t stream) {
  return launch(clip_norm, dim3(1), dim3(1024), 0, stream, part, n, max_norm, norm, scale);
}

hipError_t launch_scale(const ClipList &l, const float *scale, hipStream_t stream) {
  return launch(clip_scale, dim3((unsigned)l.tile[l.count]), dim3(256), 0, stream, l, scale);
}

}  // namespace gnn
