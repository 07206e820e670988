// Linear layers of wide and per-region networks: y = W_g x + b_g for the rows
// of every group g, with weights of 8 bits (one scale for each output channel,
// rows rounded to 8 bits with a scale of their own) or of 16.
//
//   8 bits:  y[m][n] = xs[m] ws[n] sum_k q(x)[m][k] q(W)[n][k] + b[n]
//   16 bits: y[m][n] = sum_k t(x[m][k]) t(W[n][k]) + b[n]
//
// with the sums in int32 (exact) and fp32.
#include <type_traits>

#include "rows_common.h"

namespace gnn {
namespace {

constexpr int WAVES = 8;
constexpr int CHUNK = 4096;        // most bytes of a row staged at a time
constexpr int HALF = 78 * 1024;    // LDS of a tile of more than 32 rows: two fit on a CU
constexpr int LDS_PAD = 16;  // bytes between staged rows: 16-byte slots of 8 rows differ

template <int WT>
struct Mma {
  typedef f16v acc;
};
template <>
struct Mma<T_I8> {
  typedef i16v acc;
};

// 32 rows x 32 output channels over 32 bytes of a row: lane l supplies 16
// bytes of row l % 32 and of channel l % 32 from byte 16 (l / 32) on, and holds
// channel l % 32 of the rows 8 (v / 4) + 4 (l / 32) + v % 4, v = 0 .. 15.
template <int WT>
__device__ __forceinline__ void mma(typename Mma<WT>::acc &c, const i4 &x, const i4 &w) {
  if constexpr (WT == T_I8)
    c = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, w, c, 0, 0, 0);
  else if constexpr (WT == T_BF16)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, x),
                                                __builtin_bit_cast(bf8, w), c, 0, 0, 0);
  else
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, x), __builtin_bit_cast(h8, w),
                                               c, 0, 0, 0);
}

// Stages PM rows of a tile in LDS as the products read them, bytes
// [0, chunk) of a row from element k0 on.  L lanes hold a row, C units of eight
// elements each (unit u0 + L c), so that a wave takes 64 / L rows at a time:
// with QUANT the row's scale is formed from the same registers, and what it
// costs is shared by the rows that the lanes work on at once.  FULL: kn = 8 L C.
template <int WT, int XT, bool QUANT, int C, bool FULL>
__device__ __forceinline__ void stage_rows(const LinearArgs &a, const int32_t *rows, float *scale,
                                           unsigned char *lds, int pitch, int PM, int k0, int kn,
                                           int L) {
  typedef typename std::conditional<WT == T_I8, u2, u4>::type unit;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = 64 / L;
  const int sub = lane / L, u0 = lane % L;
  const int cap = (int)(pitch - LDS_PAD) / (int)sizeof(unit);  // units a staged row holds
  for (int r = wave * per + sub; r < PM; r += WAVES * per) {
    Raw8<XT> raw[C];
    const elem_t<XT> *row = (const elem_t<XT> *)a.x + (int64_t)rows[r] * a.x_stride + k0;
#pragma unroll
    for (int c = 0; c < C; ++c)
      raw[c] = FULL ? load8_full<XT>(row, 8 * (u0 + L * c)) : load8<XT>(row, 8 * (u0 + L * c), kn);
    Quant z;
    if constexpr (QUANT) {
      uint32_t bits = 0;
#pragma unroll
      for (int c = 0; c < C; ++c) bits = max_bits<XT>(raw[c], bits);
      z = quant_of<XT>(lanes_max(top_of<XT>(bits), L));
      if (u0 == 0) scale[r] = z.s;
    }
    unsigned char *out = lds + r * pitch;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int u = u0 + L * c;
      unit q;
      if constexpr (XT == WT)
        q = __builtin_bit_cast(unit, raw[c].v);
      else if constexpr (WT == T_I8)
        q = quantize8<XT>(to_f32<XT>(raw[c]), z);
      else if constexpr (WT == T_BF16)
        q = __builtin_bit_cast(unit, __builtin_convertvector(to_f32<XT>(raw[c]), bf8));
      else
        q = __builtin_bit_cast(unit, __builtin_convertvector(to_f32<XT>(raw[c]), h8));
      if (FULL || u < cap) *(unit *)(out + u * (int)sizeof(unit)) = q;
    }
    // units past the last lane's: zeros up to the staged width
    for (int u = u0 + L * C; u < cap; u += L) *(unit *)(out + u * (int)sizeof(unit)) = unit{};
  }
}

// Lanes to a row and units to a lane: 16 lanes where eight units each are
// enough (a row's loads then span whole cache lines, and four rows share the
// instructions that form their scales), more for wider rows, fewer for rows of
// less than 16 units.  MAXU: the most units that a staged row of the calling
// kernel can have.
template <int WT, int XT, bool QUANT, int MAXU>
__device__ __forceinline__ void stage(const LinearArgs &a, const int32_t *rows, float *scale,
                                      unsigned char *lds, int pitch, int PM, int k0, int kn) {
  const int units = (kn + 7) / 8;
  int L = 16;
  while (L / 2 >= units) L /= 2;
  while (8 * L < units) L *= 2;
  const int C = (units + L - 1) / L;
  auto go = [&](auto n) {
    constexpr int CC = decltype(n)::value;
    if (kn == 8 * CC * L)
      stage_rows<WT, XT, QUANT, CC, true>(a, rows, scale, lds, pitch, PM, k0, kn, L);
    else
      stage_rows<WT, XT, QUANT, CC, false>(a, rows, scale, lds, pitch, PM, k0, kn, L);
  };
  if (C <= 1) {
    go(std::integral_constant<int, 1>());
  } else if (C <= 2) {
    go(std::integral_constant<int, 2>());
  } else if (C <= 3) {
    go(std::integral_constant<int, 3>());
  } else if (C <= 4) {
    go(std::integral_constant<int, 4>());
  } else if (C <= 6) {
    if constexpr (MAXU > 64) go(std::integral_constant<int, 6>());
  } else {
    if constexpr (MAXU > 96) go(std::integral_constant<int, 8>());
  }
}

// Stores one block of 32 rows x 32 channels (v in the accumulators' order).
// fp32 rows are stored 32 lanes to a row's 128 bytes.  Of 16-bit rows, two
// neighbouring lanes exchange halves, so that the even lane stores both
// channels of one row and the odd lane both of the next: 64 bytes of a row to
// a store of 16 lanes.  row_at: element offsets of the block's rows in y;
// left: how many of them there are; ch: this lane's channel.  FULL: 32 rows,
// 32 channels.
template <int T, bool FULL>
__device__ __forceinline__ void store_block(const LinearArgs &a, const f16v &v,
                                            const int64_t *row_at, int left, int ch) {
  const int lane = threadIdx.x & 63, hh = lane >> 5;
  // the row comparisons are made here each time: kept over the channel loop,
  // their masks would not fit in the scalar registers
  if constexpr (!FULL) asm volatile("" : "+v"(left));
  if constexpr (T == T_F32) {
    float *y = (float *)a.y + ch;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = 8 * (i / 4) + 4 * hh + i % 4;
      if (FULL || (r < left && ch < a.N)) y[row_at[r]] = v[i];
    }
  } else {
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef elem_t<T> vec __attribute__((ext_vector_type(2)));
    const int odd = lane & 1;
    // bytes of (neighbour, mine): the even lane takes the first row's two
    // halves in channel order, the odd lane the second row's
    const uint32_t sel = odd ? 0x03020706u : 0x05040100u;
    const int c0 = ch - odd;
    elem_t<T> *y = (elem_t<T> *)a.y + c0;
    row_at += 4 * hh + odd;
    left -= 4 * hh + odd;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const uint32_t mine =
          __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{v[i], v[i + 1]}, vec));
      const uint32_t other = __builtin_amdgcn_mov_dpp(mine, 0xb1, 0xf, 0xf, true);  // lane ^ 1
      const uint32_t out = __builtin_amdgcn_perm(other, mine, sel);
      const int r = 8 * (i / 4) + i % 4;
      if (FULL || (r < left && c0 + 1 < a.N))
        __builtin_memcpy(y + row_at[r], &out, 4);
      else if (r < left && c0 < a.N)
        y[row_at[r]] = __builtin_bit_cast(vec, out)[0];
    }
  }
}

// One row tile (PM = 32 RB rows of one group) by all waves: the rows are
// staged once (MULTI: chunk by chunk, where they do not fit), the weights come
// from the caches in fragment order.  A wave takes RBW of the tile's RB row
// blocks and one block of 32 channels at a time.
template <int WT, int XT, int RB, int RBW, bool MULTI>
__global__ __launch_bounds__(64 * WAVES, 4) void linear_panel(LinearArgs a) {
  constexpr int PM = 32 * RB;
  constexpr int WR = RB / RBW, WN = WAVES / WR;  // waves by row blocks and by channel blocks
  typedef typename Mma<WT>::acc acc_t;
  constexpr bool QUANT = WT == T_I8 && XT != T_I8;
  constexpr int MAXU = (RB > 1 ? HALF / PM - LDS_PAD : CHUNK) / (WT == T_I8 ? 8 : 16);
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ int32_t rows[PM];
  __shared__ int64_t row_at[PM];  // where a row lies in y
  __shared__ float scale[PM];
  const int bid = xcd_remap(blockIdx.x, gridDim.x);
  const int tile = bid / a.nsplit, split = bid % a.nsplit;
  const TileRows t = find_tile(a.off, a.G, a.n, tile, PM);
  if (t.r0 >= t.r1) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int nrow = min(PM, t.r1 - t.r0);
  if (tid < PM) {
    const int p = t.r0 + min(tid, nrow - 1);
    const int r = a.order ? clamp_idx(a.order[p], a.n) : p;
    rows[tid] = r;
    row_at[tid] = (a.y_order ? clamp_idx(a.y_order[p], a.n) : p) * a.y_stride;
    if (WT == T_I8 && !QUANT) scale[tid] = a.xs[r];
  }
  const int pitch = a.chunk + LDS_PAD;
  constexpr int esz = WT == T_I8 ? 1 : 2;
  const int steps = a.chunk / 32;  // of a chunk
  const int nchunk = MULTI ? (a.S + steps - 1) / steps : 1;
  const int ntile = (a.NB + WN - 1) / WN;
  const int col = lane & 31, hh = lane >> 5;
  const int rb0 = (wave % WR) * RBW;
  const unsigned char *xl = smem + (rb0 * 32 + col) * pitch + hh * 16;
  __syncthreads();
  if constexpr (!MULTI) {
    stage<WT, XT, QUANT, MAXU>(a, rows, scale, smem, pitch, PM, 0, a.K);
    __syncthreads();
  }
  for (int nt = split; nt < ntile; nt += a.nsplit) {
    const int nb = nt * WN + wave / WR;
    const bool live = nb < a.NB;
    acc_t acc[RBW];
#pragma unroll
    for (int r = 0; r < RBW; ++r)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[r][v] = 0;
    const i4 *wf = (const i4 *)a.w + ((int64_t)t.g * a.NB + min(nb, a.NB - 1)) * a.S * 64 + lane;
    for (int ch = 0; ch < nchunk; ++ch) {
      if constexpr (MULTI) {
        const int k0 = ch * (a.chunk / esz);
        __syncthreads();
        stage<WT, XT, false, MAXU>(a, rows, scale, smem, pitch, PM, k0, min(a.K - k0, a.chunk / esz));
        __syncthreads();
      }
      if (!live) continue;
      const int s1 = MULTI ? min(steps, a.S - ch * steps) : a.S;
      const i4 *wc = MULTI ? wf + ch * steps * 64 : wf;
      i4 w[2] = {wc[0], wc[64]};
      for (int s = 0; s < s1; s += 2) {
        const int sn = min(s + 2, s1 - 2);  // the next two steps' weights, in flight meanwhile
        const i4 n0 = wc[sn * 64], n1 = wc[sn * 64 + 64];
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          i4 x[RBW];
#pragma unroll
          for (int r = 0; r < RBW; ++r)
            x[r] = *(const i4 *)(xl + r * 32 * pitch + (s + d) * 32);
#pragma unroll
          for (int r = 0; r < RBW; ++r) mma<WT>(acc[r], x[r], w[d]);
        }
        w[0] = n0;
        w[1] = n1;
      }
    }
    if (!live) continue;
    const int ch = nb * 32 + col;
    const float bias = a.bias[(int64_t)t.g * a.NB * 32 + ch];
    const float ws = WT == T_I8 ? a.ws[(int64_t)t.g * a.NB * 32 + ch] : 1.f;
#pragma unroll
    for (int r = 0; r < RBW; ++r) {
      const int r0 = (rb0 + r) * 32;
      if (r0 >= nrow) break;
      f16v v;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (WT == T_I8)
          v[i] = __builtin_fmaf((float)acc[r][i] * ws, scale[r0 + 8 * (i / 4) + 4 * hh + i % 4],
                                bias);
        else
          v[i] = acc[r][i] + bias;
      }
      auto store = [&](auto type) {
        constexpr int T = decltype(type)::value;
        if (nrow - r0 >= 32 && nb * 32 + 32 <= a.N)
          store_block<T, true>(a, v, row_at + r0, 32, ch);
        else
          store_block<T, false>(a, v, row_at + r0, nrow - r0, ch);
      };
      if (a.y_type == T_F32)
        store(std::integral_constant<int, T_F32>());
      else if (a.y_type == T_BF16)
        store(std::integral_constant<int, T_BF16>());
      else
        store(std::integral_constant<int, T_F16>());
    }
  }
}

// Weight fragments of one block of 32 channels of one group: [S][64][16
// bytes], lane l holding channel l % 32 from byte 16 (l / 32) of the step on.
template <int WT>
__global__ __launch_bounds__(256) void linear_layout(const float *__restrict__ blob, LinearArgs a,
                                                     unsigned char *w, float *ws, float *bias) {
  const int nb = blockIdx.x, g = blockIdx.y, tid = threadIdx.x;
  const float *W = blob + (int64_t)g * ((int64_t)a.N * a.K + a.N);
  const float *bs = W + (int64_t)a.N * a.K;
  const int row = tid / 8, part = tid % 8;
  const int n = nb * 32 + row;
  __shared__ float sc[32];  // largest absolute value of a channel
  if constexpr (WT == T_I8) {
    uint32_t top = 0;
    if (n < a.N)
      for (int k = part; k < a.K; k += 8)
        top = max(top, __float_as_uint(W[(int64_t)n * a.K + k]) & 0x7fffffffu);
    for (int m = 4; m; m /= 2) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    if (part == 0) {
      sc[row] = __uint_as_float(top);
      ws[((int64_t)g * a.NB + nb) * 32 + row] = quant_scale(sc[row]);
    }
    __syncthreads();
  }
  if (tid < 32)
    bias[((int64_t)g * a.NB + nb) * 32 + tid] = nb * 32 + tid < a.N ? bs[nb * 32 + tid] : 0.f;
  unsigned char *out = w + ((int64_t)g * a.NB + nb) * a.S * 1024;
  constexpr int PER = WT == T_I8 ? 16 : 8;  // elements of 16 bytes
  for (int i = tid; i < a.S * 64; i += 256) {
    const int ln = i & 63, s = i >> 6;
    const int ch = ln % 32, c = nb * 32 + ch;
    const int k0 = (2 * s + ln / 32) * PER;
    f8 v[PER / 8];
#pragma unroll
    for (int h = 0; h < PER / 8; ++h)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = k0 + 8 * h + j;
        v[h][j] = c < a.N && k < a.K ? W[(int64_t)c * a.K + k] : 0.f;
      }
    u4 q;
    if constexpr (WT == T_I8) {
      const Quant z = quant_of<T_F32>(sc[ch]);
      const u2 lo = quantize8<T_F32>(v[0], z), hi = quantize8<T_F32>(v[PER / 8 - 1], z);
      q = u4{lo[0], lo[1], hi[0], hi[1]};
    } else if constexpr (WT == T_BF16) {
      q = __builtin_bit_cast(u4, __builtin_convertvector(v[0], bf8));
    } else {
      q = __builtin_bit_cast(u4, __builtin_convertvector(v[0], h8));
    }
    *(u4 *)(out + (int64_t)i * 16) = q;
  }
}

// What a launch of the row panels needs: RB row blocks to a tile, RBW to a
// wave, rows staged whole or in chunks.
struct Plan {
  int RB, RBW;
  bool multi;
  int64_t tiles;
};

template <int WT, int XT, int RB, int RBW, bool MULTI>
hipError_t panel(const LinearArgs &a, const Plan &p, hipStream_t stream) {
  const size_t lds = (size_t)32 * RB * (a.chunk + LDS_PAD);
  return launch_lds(linear_panel<WT, XT, RB, RBW, MULTI>, dim3((uint32_t)(p.tiles * a.nsplit)),
                    dim3(64 * WAVES), lds, stream, a);
}

template <int WT, int XT>
hipError_t panel_rows(const LinearArgs &a, const Plan &p, hipStream_t stream) {
  if (p.multi) {
    if constexpr (WT != T_I8 || XT == T_I8) return panel<WT, XT, 1, 1, true>(a, p, stream);
    return hipErrorInvalidValue;  // such rows are rounded beforehand
  }
  if (p.RB == 4) {
    if (p.RBW == 4) return panel<WT, XT, 4, 4, false>(a, p, stream);
    if (p.RBW == 2) return panel<WT, XT, 4, 2, false>(a, p, stream);
    return panel<WT, XT, 4, 1, false>(a, p, stream);
  }
  if (p.RB == 2) {
    if (p.RBW == 2) return panel<WT, XT, 2, 2, false>(a, p, stream);
    return panel<WT, XT, 2, 1, false>(a, p, stream);
  }
  return panel<WT, XT, 1, 1, false>(a, p, stream);
}

}  // namespace

int32_t linear_steps(int32_t K, int w_type) {
  const int per = w_type == T_I8 ? 64 : 32;  // elements of two steps
  return 2 * ((K + per - 1) / per);
}

size_t linear_frag_bytes(int32_t K, int32_t N, int32_t G, int w_type) {
  return (size_t)G * ((N + 31) / 32) * linear_steps(K, w_type) * 1024;
}

hipError_t launch_linear_layout(const float *blob, const LinearArgs &a, void *w, float *ws,
                                float *bias, hipStream_t stream) {
  const dim3 grid(a.NB, a.G);
  if (a.w_type == T_I8)
    return launch(linear_layout<T_I8>, grid, dim3(256), 0, stream, blob, a, (unsigned char *)w, ws,
                  bias);
  if (a.w_type == T_BF16)
    return launch(linear_layout<T_BF16>, grid, dim3(256), 0, stream, blob, a, (unsigned char *)w,
                  ws, bias);
  return launch(linear_layout<T_F16>, grid, dim3(256), 0, stream, blob, a, (unsigned char *)w, ws,
                bias);
}

bool linear_needs_rows8(const LinearArgs &a) { return a.S * 32 > CHUNK; }

hipError_t launch_linear(const LinearArgs &args, int n_cu, hipStream_t stream) {
  LinearArgs a = args;
  // The rows of a tile stay in LDS: 128 of them where two workgroups' fit on a
  // CU, fewer of wide ones and where there are too few tiles to fill the CUs.
  Plan p;
  const int row_bytes = a.S * 32;
  p.multi = row_bytes > CHUNK;
  a.chunk = p.multi ? CHUNK / 2 : row_bytes;
  auto tiles = [&](int RB) {
    const int64_t PM = 32 * RB;
    return a.off ? a.n / PM + a.G : (a.n + PM - 1) / PM;
  };
  p.RB = p.multi ? 1 : 4;
  while (p.RB > 1 && (32 * p.RB * (a.chunk + LDS_PAD) > HALF || a.n / (32 * p.RB) < 2 * n_cu))
    p.RB /= 2;
  p.tiles = tiles(p.RB);
  // Few channel blocks: the waves share out a tile's row blocks as well.
  p.RBW = p.RB;
  while (p.RBW > 1 && a.NB <= WAVES / (p.RB / p.RBW) / 2) p.RBW /= 2;
  const int WN = WAVES / (p.RB / p.RBW);
  const int ntile = (a.NB + WN - 1) / WN;
  a.nsplit = (int)((2 * n_cu + p.tiles - 1) / p.tiles);
  if (a.nsplit > ntile) a.nsplit = ntile;
  if (a.w_type == T_I8) {
    if (a.x_type == T_I8) return panel_rows<T_I8, T_I8>(a, p, stream);
    if (a.x_type == T_F32) return panel_rows<T_I8, T_F32>(a, p, stream);
    if (a.x_type == T_BF16) return panel_rows<T_I8, T_BF16>(a, p, stream);
    return panel_rows<T_I8, T_F16>(a, p, stream);
  }
  if (a.w_type == T_BF16) {
    if (a.x_type == T_F32) return panel_rows<T_BF16, T_F32>(a, p, stream);
    if (a.x_type == T_BF16) return panel_rows<T_BF16, T_BF16>(a, p, stream);
    return panel_rows<T_BF16, T_F16>(a, p, stream);
  }
  if (a.x_type == T_F32) return panel_rows<T_F16, T_F32>(a, p, stream);
  if (a.x_type == T_BF16) return panel_rows<T_F16, T_BF16>(a, p, stream);
  return panel_rows<T_F16, T_F16>(a, p, stream);
}

}  // namespace gnn
