// Row operators that feed the linear layers (linear.hip): rows rounded to 8
// bits with a scale each, and rows put in the order of their groups.
#include <type_traits>

#include "rows_common.h"

namespace gnn {
namespace {

// ---- rows to 8 bits ----
// One pass over the rows: L lanes hold a row (C units of eight elements
// each), form its largest absolute value and round the values they hold.
// Bound by memory: x is read and q written once; 1000513 x 128 fp32 110 us, 5.9
// TB/s.
constexpr int Q_WAVES = 4;
constexpr int Q_GRID = 1 << 20;  // most workgroups in a dimension of a launch

__device__ __forceinline__ void store_q8(int8_t *row, int k, int K, const u2 &q) {
  if (k <= K - 8) {
    __builtin_memcpy(row + k, &q, 8);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < K - k) row[k + j] = (int8_t)(q[j / 4] >> (8 * (j % 4)));
  }
}

template <int XT, int C, bool FULL>
__global__ __launch_bounds__(64 * Q_WAVES) void quantize_rows(QuantArgs a, int L) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = 64 / L, sub = lane / L, u0 = lane % L;
  const int64_t wg = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const int64_t r = (wg * Q_WAVES + wave) * per + sub;
  if (r >= a.n) return;
  const int width = a.pad ? a.pad : a.K;
  const elem_t<XT> *row = (const elem_t<XT> *)a.x + r * a.x_stride;
  Raw8<XT> raw[C];
#pragma unroll
  for (int c = 0; c < C; ++c)
    raw[c] = FULL ? load8<XT>(row, 8 * (u0 + L * c)) : load8_end<XT>(row, 8 * (u0 + L * c), a.K);
  uint32_t bits = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) bits = max_bits<XT>(raw[c], bits);
  const Quant z = quant_of<XT>(lanes_max(top_of<XT>(bits), L));
  if (u0 == 0) a.scales[r] = z.s;
  int8_t *q = a.q + r * a.q_stride;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const u2 v = quantize8<XT>(to_f32<XT>(raw[c]), z);
    if (FULL)
      __builtin_memcpy(q + 8 * (u0 + L * c), &v, 8);
    else
      store_q8(q, 8 * (u0 + L * c), width, v);
  }
  for (int u = u0 + L * C; 8 * u < width; u += L) store_q8(q, 8 * u, width, u2{0u, 0u});
}

// Rows too wide for a wave's registers: a workgroup to a row, which is read
// twice (the second time from the caches).  The step past the end of the widest
// rows (to 2^31 - 1) is no 32-bit number.
template <int XT>
__global__ __launch_bounds__(64 * Q_WAVES) void quantize_wide(QuantArgs a) {
  __shared__ float part[Q_WAVES];
  const int tid = threadIdx.x;
  const int width = a.pad ? a.pad : a.K;
  for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
    const elem_t<XT> *row = (const elem_t<XT> *)a.x + r * a.x_stride;
    uint32_t bits = 0;
    for (int64_t k = 8 * tid; k < a.K; k += 8 * 64 * Q_WAVES)
      bits = max_bits<XT>(load8_end<XT>(row, (int)k, a.K), bits);
    float top = lanes_max(top_of<XT>(bits), 64);
    __syncthreads();  // part has been read for the row before
    if ((tid & 63) == 0) part[tid >> 6] = top;
    __syncthreads();
    for (int w = 0; w < Q_WAVES; ++w)
      top = __uint_as_float(max(__float_as_uint(top), __float_as_uint(part[w])));
    const Quant z = quant_of<XT>(top);
    if (tid == 0) a.scales[r] = z.s;
    int8_t *q = a.q + r * a.q_stride;
    for (int64_t k = 8 * tid; k < width; k += 8 * 64 * Q_WAVES)
      store_q8(q, (int)k, width, quantize8<XT>(to_f32<XT>(load8_end<XT>(row, (int)k, a.K)), z));
  }
}

template <int XT>
hipError_t quantize_t(const QuantArgs &a, hipStream_t stream) {
  const int units = (int)(((int64_t)a.K + 7) / 8);
  const dim3 block(64 * Q_WAVES);
  if (units > 512)
    return launch(quantize_wide<XT>, dim3((uint32_t)(a.n < Q_GRID ? a.n : Q_GRID)), block, 0,
                  stream, a);
  int L = 16;
  while (L / 2 >= units) L /= 2;
  while (8 * L < units) L *= 2;
  const int C = (units + L - 1) / L;
  const int64_t rows = (int64_t)Q_WAVES * (64 / L);
  // A dimension of a launch has fewer than 2^32 threads, which 2^28 rows of 16 to a
  // workgroup reach: a second one behind the first Q_GRID workgroups.  (A loop over
  // the rows kept a partial row's comparisons in scalar registers, 82 vector
  // registers in place of 51: 100000 x 1152 bf16 77 us -> 90.)
  const int64_t wgs = (a.n + rows - 1) / rows;
  const dim3 grid((uint32_t)(wgs < Q_GRID ? wgs : Q_GRID), (uint32_t)((wgs + Q_GRID - 1) / Q_GRID));
  auto go = [&](auto n) {
    constexpr int CC = decltype(n)::value;
    if (a.K == 8 * CC * L) return launch(quantize_rows<XT, CC, true>, grid, block, 0, stream, a, L);
    return launch(quantize_rows<XT, CC, false>, grid, block, 0, stream, a, L);
  };
  if (C <= 1) return go(std::integral_constant<int, 1>());
  if (C <= 2) return go(std::integral_constant<int, 2>());
  if (C <= 3) return go(std::integral_constant<int, 3>());
  if (C <= 4) return go(std::integral_constant<int, 4>());
  if (C <= 6) return go(std::integral_constant<int, 6>());
  return go(std::integral_constant<int, 8>());
}

// ---- rows in another type ----
// A thread to eight elements; zeros from K up to the padded width.
template <int XT, int YT>
__global__ __launch_bounds__(256) void convert_rows(ConvertArgs a) {
  const int units = a.pad / 8;
  const int64_t all = a.n * units;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all;
       i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / units;
    const int k = (int)(i - r * units) * 8;
    const Raw8<XT> x = load8_end<XT>((const elem_t<XT> *)a.x + r * a.x_stride, k, a.K);
    Raw8<YT> y;
    if constexpr (XT == YT)
      y = x;
    else
      y.v = __builtin_convertvector(to_f32<XT>(x), typename Raw8<YT>::vec);
    __builtin_memcpy((elem_t<YT> *)a.y + i * 8, &y.v, sizeof y.v);
  }
}

template <int XT>
hipError_t convert_t(const ConvertArgs &a, hipStream_t stream) {
  const int64_t wgs = (a.n * (a.pad / 8) + 255) / 256;
  const dim3 grid((uint32_t)(wgs < (1 << 20) ? wgs : 1 << 20)), block(256);
  if constexpr (XT == T_I8) {
    return launch(convert_rows<T_I8, T_I8>, grid, block, 0, stream, a);
  } else {
    if (a.y_type == T_BF16) return launch(convert_rows<XT, T_BF16>, grid, block, 0, stream, a);
    return launch(convert_rows<XT, T_F16>, grid, block, 0, stream, a);
  }
}

// ---- LayerNorm and ReLU of hidden rows ----
// A wave to a row: mean, then variance of the centred values, both in fp32
// from registers (C units of eight a lane; rows of up to 4096).
template <int YT, int C>
__device__ __forceinline__ void norm_row(const NormArgs &a, int64_t p, int lane) {
  int32_t g = 0;
  if (a.ids) g = clamp_idx(a.ids[clamp_idx(a.order[p], (int32_t)a.n)], a.G);
  const float *row = a.x + p * a.H, *gm = a.gamma + (int64_t)g * a.H,
              *bt = a.beta + (int64_t)g * a.H;
  f8 x[C];
  float s = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    x[c] = load8_end<T_F32>(row, 8 * (lane + 64 * c), a.H).v;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += x[c][j];
  }
  for (int m = 32; m; m /= 2) s += __shfl_xor(s, m);
  const float mean = s / a.H;
  float var = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[c][j] = 8 * (lane + 64 * c) + j < a.H ? x[c][j] - mean : 0.f;
      var += x[c][j] * x[c][j];
    }
  for (int m = 32; m; m /= 2) var += __shfl_xor(var, m);
  const float rstd = ln_rstd(var / a.H + a.eps);
  uint32_t bits = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int k = 8 * (lane + 64 * c);
    const f8 gg = load8_end<T_F32>(gm, k, a.H).v, bb = load8_end<T_F32>(bt, k, a.H).v;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = x[c][j] * rstd * gg[j] + bb[j];
      x[c][j] = v < 0.f ? 0.f : v;  // a NaN stays one
    }
    bits = max_bits<T_F32>(Raw8<T_F32>{x[c]}, bits);
  }
  elem_t<YT> *y = (elem_t<YT> *)a.y + p * a.H;
  if constexpr (YT == T_I8) {
    const Quant z = quant_of<T_F32>(lanes_max(top_of<T_F32>(bits), 64));
    if (lane == 0) a.scales[p] = z.s;
#pragma unroll
    for (int c = 0; c < C; ++c)
      store_q8(y, 8 * (lane + 64 * c), a.H, quantize8<T_F32>(x[c], z));
  } else {
    typedef elem_t<YT> vec __attribute__((ext_vector_type(8)));
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int k = 8 * (lane + 64 * c);
      const vec o = __builtin_convertvector(x[c], vec);
      if (k + 8 <= a.H) {
        __builtin_memcpy(y + k, &o, sizeof o);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (k + j < a.H) y[k + j] = o[j];
      }
    }
  }
}

template <int YT, int C>
__global__ __launch_bounds__(64 * Q_WAVES) void norm_rows(NormArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = a.n_in ? min((int64_t)max(*a.n_in, 0), a.n) : a.n;
  for (int64_t p = (int64_t)blockIdx.x * Q_WAVES + wave; p < n; p += (int64_t)gridDim.x * Q_WAVES)
    norm_row<YT, C>(a, p, lane);
}

template <int YT>
hipError_t norm_t(const NormArgs &a, hipStream_t stream) {
  const int64_t wgs = (a.n + Q_WAVES - 1) / Q_WAVES;
  const dim3 grid((uint32_t)(wgs < (1 << 20) ? wgs : 1 << 20)), block(64 * Q_WAVES);
  const int units = (a.H + 7) / 8;
  if (units <= 64) return launch(norm_rows<YT, 1>, grid, block, 0, stream, a);
  if (units <= 128) return launch(norm_rows<YT, 2>, grid, block, 0, stream, a);
  if (units <= 256) return launch(norm_rows<YT, 4>, grid, block, 0, stream, a);
  return launch(norm_rows<YT, 8>, grid, block, 0, stream, a);
}

// ---- rows in the order of their groups ----
// A stable counting sort of the group ids.  Every tile of rows counts its
// ids (group_count), and places its rows behind those of lower groups and of
// earlier tiles (group_place); ids outside [0, G) form one more group, G, that
// comes last.  In a tile every wave owns a run of consecutive rows and counters
// of its own: the lanes of a step that hold the same id are found with one
// ballot per bit of the id, so there are no atomics and the order is the
// input's.  Reads the ids twice, writes the order once; bound by the latency of
// its launches (2000 rows 7 us, 1000513 rows in 16 groups 14).
//
// How the tiles' counts become places: with few of them (G + 1 times the tiles
// at most GROUP_DIRECT) every tile sums them itself; else
// one more launch (group_scan) leaves each tile's place and the groups' totals.
constexpr int64_t GROUP_DIRECT = 16384;

__device__ __forceinline__ int32_t group_of(int32_t id, int32_t G) {
  return (uint32_t)id < (uint32_t)G ? id : G;
}

// Lanes with this lane's id, of those with ok.
__device__ __forceinline__ uint64_t same_id(int32_t id, int bits, bool ok) {
  uint64_t m = __ballot(ok);
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((id >> b) & 1);
    m &= (id >> b) & 1 ? set : ~set;
  }
  return m;
}

// This wave's ids of its run, and their counts added to cnt[0 .. G].
template <int STEPS>
__device__ __forceinline__ void count_run(const GroupArgs &a, int64_t r0, int bits, int32_t *cnt,
                                          int32_t (&id)[STEPS]) {
  const int lane = threadIdx.x & 63;
  const uint64_t lt = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    const int64_t r = r0 + s * 64 + lane;
    id[s] = r < a.n ? group_of(a.ids[r], a.G) : 0;
  }
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    if (r0 + s * 64 >= a.n) break;
    const bool ok = r0 + s * 64 + lane < a.n;
    const uint64_t m = same_id(id[s], bits, ok);
    if (ok && (m & lt) == 0) cnt[id[s]] += __popcll(m);
  }
}

// counts[0 .. G][tile]
template <int WAVES, int STEPS>
__global__ __launch_bounds__(64 * WAVES) void group_count(GroupArgs a, int bits) {
  extern __shared__ int32_t cnt[];  // [WAVES][G + 1]
  const int tid = threadIdx.x, wave = tid >> 6, W = a.G + 1;
  for (int i = tid; i < WAVES * W; i += 64 * WAVES) cnt[i] = 0;
  __syncthreads();
  int32_t id[STEPS];
  count_run(a, ((int64_t)blockIdx.x * WAVES + wave) * (STEPS * 64), bits, cnt + wave * W, id);
  __syncthreads();
  for (int g = tid; g < W; g += 64 * WAVES) {
    int32_t c = 0;
    for (int w = 0; w < WAVES; ++w) c += cnt[w * W + g];
    a.counts[(int64_t)g * gridDim.x + blockIdx.x] = c;
  }
}

// counts[g][tile] -> the sum over the tiles before; counts[G + 1][g] = the sum
// over all.  A wave to a group.
__global__ __launch_bounds__(256) void group_scan(int32_t *counts, int W, int tiles) {
  const int lane = threadIdx.x & 63, g = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (g >= W) return;
  int32_t *c = counts + (int64_t)g * tiles, carry = 0;
  for (int t0 = 0; t0 < tiles; t0 += 64) {
    const int32_t v = t0 + lane < tiles ? c[t0 + lane] : 0;
    int32_t inc = v;
    for (int m = 1; m < 64; m *= 2) {
      const int32_t u = __shfl_up(inc, m);
      if (lane >= m) inc += u;
    }
    if (t0 + lane < tiles) c[t0 + lane] = carry + inc - v;
    carry += __shfl(inc, 63);
  }
  if (lane == 0) counts[(int64_t)W * tiles + g] = carry;
}

template <int WAVES, int STEPS>
__global__ __launch_bounds__(64 * WAVES) void group_place(GroupArgs a, int bits, int tiles,
                                                          bool scanned) {
  extern __shared__ int32_t lds[];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, W = a.G + 1;
  int32_t *cnt = lds;               // [WAVES][W]: counts, then where a wave's rows go
  int32_t *total = cnt + WAVES * W;  // [W] rows of a group
  int32_t *before = total + W;       // [W] those of earlier tiles
  __shared__ int32_t wsum[WAVES];
  const int tile = blockIdx.x;
  for (int i = tid; i < WAVES * W; i += 64 * WAVES) cnt[i] = 0;
  __syncthreads();
  int32_t id[STEPS];
  const int64_t r0 = ((int64_t)tile * WAVES + wave) * (STEPS * 64);
  count_run(a, r0, bits, cnt + wave * W, id);
  if (scanned) {
    for (int g = tid; g < W; g += 64 * WAVES) {
      total[g] = a.counts[(int64_t)W * tiles + g];
      before[g] = a.counts[(int64_t)g * tiles + tile];
    }
  } else if (tiles > 1) {
    // L lanes to a group, up to four tiles to a lane where that is enough
    int L = 1;
    while (L < 64 && 4 * L < tiles) L *= 2;
    for (int g = tid / L; g < W; g += 64 * WAVES / L) {
      int32_t all = 0, prev = 0;
      for (int t = tid % L; t < tiles; t += L) {
        const int32_t c = a.counts[(int64_t)g * tiles + t];
        all += c;
        if (t < tile) prev += c;
      }
      for (int m = L / 2; m; m /= 2) {
        all += __shfl_xor(all, m);
        prev += __shfl_xor(prev, m);
      }
      if (tid % L == 0) {
        total[g] = all;
        before[g] = prev;
      }
    }
  }
  __syncthreads();
  // a wave's first place in group g: behind the lower groups, the earlier
  // tiles and the earlier waves
  int32_t carry = 0;
  for (int g0 = 0; g0 < W; g0 += 64 * WAVES) {
    const int g = g0 + tid;
    int32_t all = 0;
    if (g < W) {
      if (tiles > 1) {
        all = total[g];
      } else {
        for (int w = 0; w < WAVES; ++w) all += cnt[w * W + g];
      }
    }
    int32_t inc = all;  // inclusive sum over the groups of this round
    for (int m = 1; m < 64; m *= 2) {
      const int32_t v = __shfl_up(inc, m);
      if (lane >= m) inc += v;
    }
    if (g0 > 0) __syncthreads();
    if (lane == 63) wsum[wave] = inc;
    __syncthreads();
    int32_t first = carry + inc - all;
    for (int w = 0; w < WAVES; ++w) {
      first += w < wave ? wsum[w] : 0;
      carry += wsum[w];
    }
    if (g < W) {
      if (tile == 0) a.offsets[g] = first;
      int32_t at = first + (tiles > 1 ? before[g] : 0);
      for (int w = 0; w < WAVES; ++w) {
        const int32_t c = cnt[w * W + g];
        cnt[w * W + g] = at;
        at += c;
      }
    }
  }
  __syncthreads();
  const uint64_t lt = ((uint64_t)1 << lane) - 1;
  int32_t *mine = cnt + wave * W;
#pragma unroll
  for (int s = 0; s < STEPS; ++s) {
    if (r0 + s * 64 >= a.n) break;
    const bool ok = r0 + s * 64 + lane < a.n;
    const uint64_t m = same_id(id[s], bits, ok);
    const int32_t at = mine[id[s]];
    if (ok) a.order[at + __popcll(m & lt)] = (int32_t)(r0 + s * 64 + lane);
    if (ok && (m & lt) == 0) mine[id[s]] = at + __popcll(m);
  }
}

// Rows of a tile: one tile of up to 8192 rows, tiles of 4096 beyond (4 waves
// with longer runs where 16 waves' counters would not fit in 64 KiB of LDS).
constexpr int G_TILE = 4096, G_WIDE = 900;

int64_t group_tiles(int64_t n, int32_t G) {
  return n <= (G < G_WIDE ? 2 * G_TILE : G_TILE) ? 1 : (n + G_TILE - 1) / G_TILE;
}

template <int WAVES, int STEPS>
hipError_t group_t(const GroupArgs &a, int tiles, hipStream_t stream) {
  int bits = 0;
  while ((a.G >> bits) != 0) ++bits;  // ids 0 .. G
  const int W = a.G + 1;
  const dim3 block(64 * WAVES);
  const bool scanned = (int64_t)tiles * W > GROUP_DIRECT && tiles > 1;
  hipError_t e = hipSuccess;
  if (tiles > 1)
    e = launch_lds(group_count<WAVES, STEPS>, dim3(tiles), block, (size_t)WAVES * W * 4, stream, a,
                   bits);
  if (e == hipSuccess && scanned)
    e = launch(group_scan, dim3((W + 3) / 4), dim3(256), 0, stream, a.counts, W, tiles);
  if (e != hipSuccess) return e;
  return launch_lds(group_place<WAVES, STEPS>, dim3(tiles), block, (size_t)(WAVES + 2) * W * 4,
                    stream, a, bits, tiles, scanned);
}

}  // namespace

hipError_t launch_quantize(const QuantArgs &a, hipStream_t stream) {
  if (a.x_type == T_F32) return quantize_t<T_F32>(a, stream);
  if (a.x_type == T_BF16) return quantize_t<T_BF16>(a, stream);
  return quantize_t<T_F16>(a, stream);
}

hipError_t launch_convert(const ConvertArgs &a, hipStream_t stream) {
  if (a.x_type == T_F32) return convert_t<T_F32>(a, stream);
  if (a.x_type == T_BF16) return convert_t<T_BF16>(a, stream);
  if (a.x_type == T_F16) return convert_t<T_F16>(a, stream);
  return convert_t<T_I8>(a, stream);
}

hipError_t launch_norm(const NormArgs &a, hipStream_t stream) {
  if (a.y_type == T_I8) return norm_t<T_I8>(a, stream);
  if (a.y_type == T_BF16) return norm_t<T_BF16>(a, stream);
  return norm_t<T_F16>(a, stream);
}

size_t group_scratch_bytes(int64_t n, int32_t G) {
  const int64_t tiles = group_tiles(n, G);
  return tiles > 1 ? (size_t)(tiles + 1) * (G + 1) * 4 : 0;
}

hipError_t launch_group(const GroupArgs &a, hipStream_t stream) {
  const int tiles = (int)group_tiles(a.n, a.G);
  if (a.G >= G_WIDE) return group_t<4, G_TILE / 256>(a, tiles, stream);
  if (tiles > 1) return group_t<16, G_TILE / 1024>(a, tiles, stream);
  if (a.n <= 2048) return group_t<16, 2>(a, 1, stream);
  return group_t<16, 2 * G_TILE / 1024>(a, 1, stream);
}

}  // namespace gnn
