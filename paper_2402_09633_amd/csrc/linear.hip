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
constexpr int CHUNK = 4096;      // most bytes of a row staged at a time
constexpr int HALF = 78 * 1024;  // LDS of a tile of more than 32 rows: two fit on a CU
constexpr int LDS_PAD = 16;      // bytes between staged rows: 16-byte slots of 8 rows differ

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

// Stages the n rows of a tile in LDS as the products read them, bytes
// [0, chunk) of a row from element k0 on.  L lanes hold a row, C units of eight
// elements each (unit u0 + L c), so that a wave takes 64 / L rows at a time:
// with QUANT the row's scale is formed from the same registers, and what it
// costs is shared by the rows that the lanes work on at once.  B such passes are
// loaded before the first is used.
template <int WT, int XT, bool QUANT, int C, int B, int NW, int RB>
__device__ __forceinline__ void stage_rows(const LinearArgs &a, const int32_t *rows, float *scale,
                                           unsigned char *lds, int pitch, int n, int k0, int kn,
                                           int L) {
  const bool full = kn == 8 * L * C;
  // Rows of large calls pass the caches by, so that the weights stay there (300000
  // x 512 -> 512 8-bit 187 us -> 174); fp32 rows, which take two loads to a cache
  // line, do not (1000513 x 384 -> 128: 358 and 382), nor those of small calls,
  // where several workgroups read a row (64 x 1024 -> 1024, 64 groups: 16.5, 18.3).
  constexpr bool ONCE = XT != T_F32 && RB > 1;
  constexpr int SURE = C >= 6 ? C - 2 : C - 1;  // units of a lane that end inside the row
  typedef typename std::conditional<WT == T_I8, u2, u4>::type unit;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = 64 / L;
  const int sub = lane / L, u0 = lane % L;
  const int cap = (int)(pitch - LDS_PAD) / (int)sizeof(unit);  // units a staged row holds
  for (int rb = wave * per + sub; rb < n; rb += NW * per * B) {
    Raw8<XT> raw[B][C];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int r = min(rb + b * NW * per, n - 1);
      const elem_t<XT> *row = (const elem_t<XT> *)a.x + (int64_t)rows[r] * a.x_stride + k0;
#pragma unroll
      for (int c = 0; c < C; ++c)
        raw[b][c] = c < SURE || full ? load8<XT, ONCE>(row, 8 * (u0 + L * c))
                                     : load8_end<XT, ONCE>(row, 8 * (u0 + L * c), kn);
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int r = rb + b * NW * per;
      if (r >= n) break;
      Quant z;
      if constexpr (QUANT) {
        uint32_t bits = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) bits = max_bits<XT>(raw[b][c], bits);
        z = quant_of<XT>(lanes_max(top_of<XT>(bits), L));
        if (u0 == 0) scale[r] = z.s;
      }
      unsigned char *out = lds + r * pitch;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int u = u0 + L * c;
        unit q;
        if constexpr (XT == WT)
          q = __builtin_bit_cast(unit, raw[b][c].v);
        else if constexpr (WT == T_I8)
          q = quantize8<XT>(to_f32<XT>(raw[b][c]), z);
        else if constexpr (WT == T_BF16)
          q = __builtin_bit_cast(unit, __builtin_convertvector(to_f32<XT>(raw[b][c]), bf8));
        else
          q = __builtin_bit_cast(unit, __builtin_convertvector(to_f32<XT>(raw[b][c]), h8));
        if (full || u < cap) *(unit *)(out + u * (int)sizeof(unit)) = q;
      }
      // units past the last lane's: zeros up to the staged width
      for (int u = u0 + L * C; u < cap; u += L) *(unit *)(out + u * (int)sizeof(unit)) = unit{};
    }
  }
}

// Lanes to a row and units to a lane: 16 lanes where eight units each are
// enough (a row's loads then span whole cache lines, and four rows share the
// instructions that form their scales), more for wider rows, fewer for rows of
// less than 16 units.  MAXU: the most units that a staged row of the calling
// kernel can have; RB: its tiles' row blocks.
template <int WT, int XT, bool QUANT, int MAXU, int RB, int NW>
__device__ __forceinline__ void stage(const LinearArgs &a, const int32_t *rows, float *scale,
                                      unsigned char *lds, int pitch, int n, int k0, int kn) {
  const int units = (kn + 7) / 8;
  int L = 16;
  while (L / 2 >= units) L /= 2;
  while (8 * L < units) L *= 2;
  const int C = (units + L - 1) / L;
  auto go = [&](auto nc) {
    constexpr int CC = decltype(nc)::value;
    // passes in flight: the tile's (at 16 lanes to a row), or as many as 64
    // registers hold
    constexpr int fit = 64 / (CC * (XT == T_F32 ? 8 : XT == T_I8 ? 2 : 4));
    constexpr int all = RB * 8 / NW;
    constexpr int B = all < fit ? all : fit >= 4 ? 4 : fit >= 2 ? 2 : 1;
    stage_rows<WT, XT, QUANT, CC, B, NW, RB>(a, rows, scale, lds, pitch, n, k0, kn, L);
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

// The epilogue of one block: scales and bias, rounding, store.
template <int WT>
__device__ __forceinline__ void finish_block(const LinearArgs &a,
                                             const typename Mma<WT>::acc &acc, const float *scale,
                                             const int64_t *row_at, int left, int ch, float ws,
                                             float bias) {
  const int hh = (threadIdx.x & 63) >> 5;
  f16v v;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if constexpr (WT == T_I8)
      v[i] = __builtin_fmaf((float)acc[i] * ws, scale[8 * (i / 4) + 4 * hh + i % 4], bias);
    else
      v[i] = acc[i] + bias;
  }
  auto store = [&](auto type) {
    constexpr int T = decltype(type)::value;
    if (left >= 32 && (ch | 31) < a.N)
      store_block<T, true>(a, v, row_at, 32, ch);
    else
      store_block<T, false>(a, v, row_at, left, ch);
  };
  if (a.y_type == T_F32)
    store(std::integral_constant<int, T_F32>());
  else if (a.y_type == T_BF16)
    store(std::integral_constant<int, T_BF16>());
  else
    store(std::integral_constant<int, T_F16>());
}

// How rows are staged: whole; in chunks, where they do not fit; or whole and
// narrow, 32 to a tile, in few enough registers for three workgroups to a CU
// (20011 x 391 -> 259 8-bit 18.7 us without, 15.8 with; rows past narrow_bytes
// lose by it, 3000 x 1024 -> 1024 13.3 and 18.4; fp32 rows to 8 bits take the
// registers of two).
enum { WHOLE, CHUNKS, NARROW };
constexpr int narrow_bytes(int w_type) { return w_type == T_I8 ? 768 : 1024; }

// One row tile (PM = 32 RB rows of one group) by all waves: the rows are
// staged once (CHUNKS: piece by piece), the weights come
// from the caches in fragment order, RING steps of them in flight.  A wave takes
// the tile's RB row blocks and one block of 32 channels at a time.  WK waves
// share the steps of a block (few rows: a call is then bound by how long the
// weights take, and all waves fetch them); their sums are added in LDS, in the
// waves' order.
//
// Bound by HBM: a row is read and an output written once.  1000513 x 384 -> 128
// 8-bit from fp32 rows 346 us, 5.2 TB/s, the rate of a large copy; 300000 x 512 ->
// 512 8-bit from bf16 165 us, 3.7 TB/s, the products' 33 us of matrix time and the
// weights' way from L2 (256 KB to a tile) not all covered.
template <int WT, int XT, int RB, int WK, int NW, int MODE>
__global__ __launch_bounds__(64 * NW, RB > 1           ? 4
                                     : MODE != NARROW ? 2
                                     : WT == T_I8 && XT == T_F32 ? 4 : 6) void linear_panel(
    LinearArgs a) {
  constexpr bool MULTI = MODE == CHUNKS;
  constexpr int PM = 32 * RB, RING = RB == 1 && MODE != NARROW ? 8 : 4;
  constexpr int WN = NW / WK;  // channel blocks at a time
  static_assert(WK == 1 || (RB == 1 && WK == NW), "one block to a workgroup");
  typedef typename Mma<WT>::acc acc_t;
  constexpr bool QUANT = WT == T_I8 && XT != T_I8;
  constexpr int MAXU = (RB > 1           ? HALF / PM - LDS_PAD
                        : MODE == NARROW ? narrow_bytes(WT)
                                         : CHUNK) /
                       (WT == T_I8 ? 8 : 16);
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
  const int pitch = a.chunk + LDS_PAD;
  constexpr int esz = WT == T_I8 ? 1 : 2;
  const int steps = a.chunk / 32;  // of a chunk
  const int nchunk = MULTI ? (a.S + steps - 1) / steps : 1;
  const int ntile = (a.NB + WN - 1) / WN;
  const int col = lane & 31, hh = lane >> 5;
  const int wk = WK > 1 ? wave : 0;
  const unsigned char *xl = smem + col * pitch + hh * 16;
  i4 w[RING];
  auto block_of = [&](int nt) { return nt * WN + (WK > 1 ? 0 : wave); };
  auto weights_of = [&](int nb) {
    return (const i4 *)a.w + ((int64_t)t.g * a.NB + min(nb, a.NB - 1)) * a.S * 64 + lane;
  };
  // this wave's steps of a chunk of n
  auto first = [&](int n) { return WK > 1 ? n * wk / WK : 0; };
  auto fill = [&](const i4 *wf, int s0, int s1) {
#pragma unroll
    for (int d = 0; d < RING; ++d) w[d] = wf[max(min(s0 + d, s1 - 1), 0) * 64];
  };
  const int n0 = MULTI ? min(steps, a.S) : a.S;
  fill(weights_of(block_of(split)), first(n0), WK > 1 ? n0 * (wk + 1) / WK : n0);
  if (tid < nrow) {
    const int p = t.r0 + tid;
    const int r = a.order ? clamp_idx(a.order[p], a.n) : p;
    rows[tid] = r;
    row_at[tid] = (a.y_order ? clamp_idx(a.y_order[p], a.n) : p) * a.y_stride;
    if (WT == T_I8 && !QUANT) scale[tid] = a.xs[r];
  }
  __syncthreads();
  if constexpr (!MULTI) {
    stage<WT, XT, QUANT, MAXU, RB, NW>(a, rows, scale, smem, pitch, nrow, 0, a.K);
    __syncthreads();
  }
  for (int nt = split; nt < ntile; nt += a.nsplit) {
    const int nb = block_of(nt);
    const bool live = nb < a.NB;
    acc_t acc[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[r][v] = 0;
    const i4 *wf = weights_of(nb);
    const int64_t cw = ((int64_t)t.g * a.NB + min(nb, a.NB - 1)) * 32 + col;
    const float bias = a.bias[cw], ws = WT == T_I8 ? a.ws[cw] : 1.f;
    for (int ch = 0; ch < nchunk; ++ch) {
      const int n = MULTI ? min(steps, a.S - ch * steps) : a.S;
      const int s0 = first(n), s1 = WK > 1 ? n * (wk + 1) / WK : n;
      const i4 *wc = MULTI ? wf + ch * steps * 64 : wf;
      if (ch > 0 || (RB == 1 && nt > split)) fill(wc, s0, s1);
      if constexpr (MULTI) {
        const int k0 = ch * (a.chunk / esz);
        __syncthreads();
        stage<WT, XT, false, MAXU, RB, NW>(a, rows, scale, smem, pitch, nrow, k0,
                                           min(a.K - k0, a.chunk / esz));
        __syncthreads();
      }
      if (!live) continue;
      auto step = [&](int s, int d) {
        i4 x[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) x[r] = *(const i4 *)(xl + r * 32 * pitch + (s + d) * 32);
#pragma unroll
        for (int r = 0; r < RB; ++r) mma<WT>(acc[r], x[r], w[d]);
      };
      if constexpr (RB > 1) {
        // a row's steps are a multiple of RING: behind the last come the next
        // block's first ones, ahead of this block's stores (loads and stores are
        // counted together, in order)
        const i4 *wn = nt + a.nsplit < ntile ? weights_of(block_of(nt + a.nsplit)) : nullptr;
        for (int s = 0; s < s1; s += RING) {
          const i4 *wl = s + RING < s1 ? wc + (s + RING) * 64 : wn;
#pragma unroll
          for (int d = 0; d < RING; ++d) {
            step(s, d);
            if (wl) w[d] = wl[d * 64];
          }
        }
      } else {
        for (int s = s0; s < s1; s += RING) {
#pragma unroll
          for (int d = 0; d < RING; ++d) {
            if (s + d >= s1) break;
            step(s, d);
            w[d] = wc[min(s + d + RING, s1 - 1) * 64];
          }
        }
      }
    }
    if constexpr (WK > 1) {
      // the staged rows have been read: their place takes the waves' sums
      typedef decltype(acc[0][0] + acc[0][0]) val;
      typedef val val4 __attribute__((ext_vector_type(4)));
      val4 *part = (val4 *)smem;  // [wave][v / 4][lane]
      __syncthreads();
#pragma unroll
      for (int q = 0; q < 4; ++q)
        part[(wave * 4 + q) * 64 + lane] =
            val4{acc[0][4 * q], acc[0][4 * q + 1], acc[0][4 * q + 2], acc[0][4 * q + 3]};
      __syncthreads();
      if (wave > 0) return;  // one block to a workgroup: nothing is left
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        val4 sum = part[q * 64 + lane];
        for (int k = 1; k < WK; ++k) sum += part[(k * 4 + q) * 64 + lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[0][4 * q + j] = sum[j];
      }
    }
    if (!live) continue;
    const int ch = nb * 32 + col;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      const int r0 = r * 32;
      if (r0 >= nrow) break;
      finish_block<WT>(a, acc[r], scale + r0, row_at + r0, nrow - r0, ch, ws, bias);
    }
  }
}

// ---- tiles for wide layers ----
// Where a row does not fit beside its neighbours in LDS, the matrix cores bound
// the layer, and every byte has to be used often once it is on the CU: tiles of
// 64 TR rows x 256 channels, eight waves of 32 TR x 64.  The rows (already in
// the weights' type, whole chunks of 16 bytes) go through LDS, 128 bytes of each
// at a time and two such stages in turn; a wave's weights come from the caches
// into registers, in fragment order.  While a stage is multiplied, the next one's
// weights and the rows of the one after it are in flight.  16384 x 4096 -> 4096 in
// 8 bits: 270 us, 2.0 POP/s; 8192 cubed in bf16 910 us, 1.2 PFLOP/s.
constexpr int T_STEPS = 4;                // steps of 32 bytes in a stage
constexpr int T_BYTES = 32 * T_STEPS;     // of a row
constexpr int T_CH = 8;                   // channel blocks of a tile

template <int WT, int TR>
__global__ __launch_bounds__(64 * WAVES, 2) void linear_tiled(LinearArgs a) {
  constexpr int PM = 64 * TR;             // rows of a tile
  constexpr int LOADS = PM / (8 * WAVES);  // 16-byte loads of a lane a stage
  typedef typename Mma<WT>::acc acc_t;
  __shared__ __align__(16) unsigned char xs[2][PM * T_BYTES];
  __shared__ int64_t row_at[PM];
  __shared__ float scale[PM];
  const int ntile = (a.NB + T_CH - 1) / T_CH;
  const int bid = xcd_remap(blockIdx.x, gridDim.x);
  // eight row tiles side by side go through the channels together, so that they
  // share the weights in an XCD's cache, and the channels the rows
  const int tiles = gridDim.x / ntile, band = 8 * ntile;
  const int b0 = bid / band * 8, wide = min(8, tiles - b0);
  const int tile = b0 + bid % band % wide, nt = bid % band / wide;
  const TileRows t = find_tile(a.off, a.G, a.n, tile, PM);
  if (t.r0 >= t.r1) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int nrow = min(PM, t.r1 - t.r0);
  auto row_of = [&](int i) {
    const int p = t.r0 + min(i, nrow - 1);
    return a.order ? clamp_idx(a.order[p], a.n) : p;
  };
  for (int i = tid; i < PM; i += 64 * WAVES) {
    const int p = t.r0 + min(i, nrow - 1);
    row_at[i] = (a.y_order ? clamp_idx(a.y_order[p], a.n) : p) * a.y_stride;
    if (WT == T_I8) scale[i] = a.xs[row_of(i)];
  }
  // A wave's load takes 8 rows of 128 bytes; the 16-byte chunk c of row r lies
  // at place c ^ (r % 8), so that 8 lanes of a product's read (8 rows, one chunk)
  // lie in 8 different places.  Rows r and r + 8 still meet; c ^ (r / 2 % 8), where
  // 16 rows do not, took the same time (300 and 308 us at 16384 x 4096 -> 4096).
  const int c = (lane & 7) ^ (lane >> 3);
  constexpr int esz = WT == T_I8 ? 1 : 2;
  const unsigned char *src[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i)
    src[i] = (const unsigned char *)a.x +
             (int64_t)row_of((i * WAVES + wave) * 8 + (lane >> 3)) * a.x_stride * esz;
  const int bytes = a.K * esz;  // whole chunks of 16; zeros behind them
  auto load = [&](i4(&r)[LOADS], int st) {
    const int at = st * T_BYTES + c * 16;
    const int from = at < bytes ? at : 0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) __builtin_memcpy(&r[i], src[i] + from, 16);
  };
  auto put = [&](const i4(&r)[LOADS], int buf, int st) {
    const bool in = st * T_BYTES + c * 16 < bytes;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      *(i4 *)(xs[buf] + (i * WAVES + wave) * 1024 + lane * 16) = in ? r[i] : i4{0, 0, 0, 0};
  };
  const int wr = wave & 1, wc = wave >> 1;
  const int nb0 = nt * T_CH + wc * 2;
  const i4 *wf[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    wf[i] = (const i4 *)a.w + ((int64_t)t.g * a.NB + min(nb0 + i, a.NB - 1)) * a.S * 64 + lane;
  i4 w[T_STEPS][2];
  auto weights = [&](int s, int st) {
#pragma unroll
    for (int i = 0; i < 2; ++i) w[s][i] = wf[i][min(st * T_STEPS + s, a.S - 1) * 64];
  };
  acc_t acc[2][TR];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int r = 0; r < TR; ++r)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][r][v] = 0;
  const int col = lane & 31, hh = lane >> 5;
  // A step's products, with the next step's rows on their way from LDS, and
  // behind them the same step's weights of the next stage.
  auto multiply = [&](int buf, int st) {
    const unsigned char *x0 = xs[buf] + (wr * TR * 32 + col) * T_BYTES;
    i4 x[2][TR];
    auto read = [&](int s) {
#pragma unroll
      for (int r = 0; r < TR; ++r)
        x[s & 1][r] = *(const i4 *)(x0 + r * 32 * T_BYTES + (((2 * s + hh) ^ (col & 7)) * 16));
    };
    read(0);
#pragma unroll
    for (int s = 0; s < T_STEPS; ++s) {
      if (s + 1 < T_STEPS) read(s + 1);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < TR; ++r) mma<WT>(acc[i][r], x[s & 1][r], w[s][i]);
      weights(s, st + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const int stages = a.S / T_STEPS;
  i4 rows[LOADS];
  load(rows, 0);
#pragma unroll
  for (int s = 0; s < T_STEPS; ++s) weights(s, 0);
  put(rows, 0, 0);
  load(rows, 1);
  __syncthreads();
  int st = 0;
  for (; st + 1 < stages; st += 2) {
    put(rows, 1, st + 1);
    load(rows, st + 2);
    multiply(0, st);
    __syncthreads();
    put(rows, 0, st + 2);
    load(rows, st + 3);
    multiply(1, st + 1);
    __syncthreads();
  }
  if (st < stages) {
    multiply(0, st);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (nb0 + i >= a.NB) break;
    const int ch = (nb0 + i) * 32 + col;
    const float bias = a.bias[(int64_t)t.g * a.NB * 32 + ch];
    const float ws = WT == T_I8 ? a.ws[(int64_t)t.g * a.NB * 32 + ch] : 1.f;
#pragma unroll
    for (int r = 0; r < TR; ++r) {
      const int r0 = (wr * TR + r) * 32;
      if (r0 >= nrow) break;
      finish_block<WT>(a, acc[i][r], scale + r0, row_at + r0, nrow - r0, ch, ws, bias);
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

template <int WT, int XT, int RB, int WK, int NW, int MODE>
hipError_t panel(const LinearArgs &a, const LinearPlan &p, hipStream_t stream) {
  size_t lds = (size_t)32 * RB * (a.chunk + LDS_PAD);
  if (WK > 1 && lds < 4096 * NW) lds = 4096 * NW;
  return launch_lds(linear_panel<WT, XT, RB, WK, NW, MODE>,
                    dim3((uint32_t)(p.tiles * a.nsplit)), dim3(64 * NW), lds, stream, a);
}

template <int WT, int XT>
hipError_t panel_rows(const LinearArgs &a, const LinearPlan &p, hipStream_t stream) {
  if (p.multi) {
    if constexpr (WT != T_I8 || XT == T_I8) {
      if (p.split) return panel<WT, XT, 1, 8, 8, CHUNKS>(a, p, stream);
      return panel<WT, XT, 1, 1, 8, CHUNKS>(a, p, stream);
    }
    return hipErrorInvalidValue;  // such rows are rounded beforehand
  }
  if (p.RB == 4) {
    if (p.NW == 8) return panel<WT, XT, 4, 1, 8, WHOLE>(a, p, stream);
    return panel<WT, XT, 4, 1, 4, WHOLE>(a, p, stream);
  }
  if (p.RB == 2) {
    if (p.NW == 8) return panel<WT, XT, 2, 1, 8, WHOLE>(a, p, stream);
    return panel<WT, XT, 2, 1, 4, WHOLE>(a, p, stream);
  }
  if (p.split) return panel<WT, XT, 1, 8, 8, WHOLE>(a, p, stream);
  if (p.narrow) return panel<WT, XT, 1, 1, 8, NARROW>(a, p, stream);
  return panel<WT, XT, 1, 1, 8, WHOLE>(a, p, stream);
}

template <int WT>
hipError_t tiled(const LinearArgs &a, int TR, hipStream_t stream) {
  const int64_t PM = 64 * TR, tiles = a.off ? a.n / PM + a.G : (a.n + PM - 1) / PM;
  const dim3 grid((uint32_t)(tiles * ((a.NB + T_CH - 1) / T_CH))), block(64 * WAVES);
  if (TR == 4) return launch(linear_tiled<WT, 4>, grid, block, 0, stream, a);
  return launch(linear_tiled<WT, 2>, grid, block, 0, stream, a);
}

}  // namespace

int32_t linear_steps(int32_t K, int w_type) {
  const int per = w_type == T_I8 ? 128 : 64;  // elements of four steps
  return 4 * ((K + per - 1) / per);
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

// Whether the tiles for wide layers take a call of n rows, and with how many
// row blocks to a wave (0: the row panels do).  extra: its rows would be rounded
// to 8 bits for the tiles alone, the panels take them as they are.  Measured
// (panels : tiles, us, bf16 rows and outputs where no type is given):
//  - rows up to 1 KB: 100000 x 512 -> 512 bf16 88 : 90, 300000 x 128 -> 128 bf16
//    42 : 54; past it 100000 x 640 -> 640 163 : 134, 1024 -> 256 113 : 80,
//    2048 -> 512 399 : 258
//  - 8-bit layers whose rows come as floats pay for a pass over the rows first
//    (in the tiles' times): 100000 x 1024 -> 1024 197 : 243, 2048 -> 512 237 : 272,
//    but 30000 x 1024 -> 2048 144 : 117, 8000 x 1024 -> 4096 81 : 62; where 64 of
//    their rows fit a panel the pass does not pay, 100000 x 1024 -> 1056 200 : 253,
//    1152 -> 1056 225 : 275, fp32 34000 x 1024 -> 1300 140 : 145 (34000 x 1024 ->
//    4096 loses by it, 263 : 240)
//  - few tiles leave CUs idle: 1000 x 4096 -> 512 bf16 33 : 47, 300 x 4096 -> 4096
//    44 : 49, 4000 x 2048 -> 2048 79 : 41; 32 groups of 312 rows x 1024 -> 1024
//    43 : 47 with the rows in the last-level cache and 47 : 42 without, of 937
//    126 : 104
//  - 256 rows to a tile where that gives every CU one: 16384 x 4096 -> 4096 8-bit
//    rows 277, with 128 rows 305; 2048 x 4096 -> 4096 56 and 44
static int tiled_rows(const LinearArgs &a, bool extra, int64_t n, int n_cu) {
  const int ntile = (a.NB + T_CH - 1) / T_CH;
  if (a.S * 32 < (extra ? 1024 : 1025) || a.NB <= (extra ? 32 : 4)) return 0;
  if (extra && n / 64 >= 2 * n_cu && 64 * (a.S * 32 + LDS_PAD) <= HALF) return 0;
  if (n / a.G < 512 || n / 128 * ntile < n_cu / 2) return 0;
  return n / 256 * ntile >= n_cu ? 4 : 2;
}

LinearPlan linear_plan(const LinearArgs &a, int n_cu) {
  // The decision is made once, for the rows as the caller has them, and holds for
  // the launch after they were converted.
  const bool rounds = a.w_type == T_I8 && a.x_type != T_I8;
  const bool panels = a.w_type == T_I8 ? !rounds || a.S * 32 <= CHUNK
                                       : a.x_type == T_F32 || a.x_type == a.w_type;
  LinearPlan p;
  p.tile = tiled_rows(a, rounds && panels, a.n, n_cu);
  if (p.tile) {
    p.convert = a.x_type != a.w_type || a.K * type_bytes(a.w_type) % 16 != 0;
    return p;
  }
  p.convert = !panels;
  // The rows of a tile stay in LDS: 128 of them where two workgroups' fit on a
  // CU, fewer of wide ones and where there are too few tiles to fill the CUs.
  // Layers of up to four channel blocks keep four waves busy: smaller workgroups,
  // and more of them to a CU (300000 x 128 -> 128 bf16 37 us with four waves, 44
  // with eight; 1000513 x 384 -> 128 f16 272 and 298).  Wider ones take eight
  // (300000 x 512 -> 512 8-bit 187 us, 201 with four waves and 64 rows).
  const int row_bytes = a.S * 32;
  p.multi = row_bytes > CHUNK;
  p.chunk = p.multi ? CHUNK / 2 : row_bytes;
  p.NW = a.NB <= 4 ? 4 : WAVES;
  const int room = p.NW == WAVES ? HALF : HALF / 2;
  // Output rows that do not start on 64 bytes share cache sectors between two
  // blocks' stores, which have to meet in L2: long ones do better with 64 rows to a
  // tile, whose output stays there (bf16 184899 x 64 -> 1537 244 : 198 us, fp32 out
  // -> 769 210 : 166, 100000 x 256 -> 1000 8-bit 84 : 79; short ones and whole
  // sectors lose by it, -> 513 71 : 73, -> 1536 138 : 144).
  const int64_t ysz = type_bytes(a.y_type);
  const bool torn = ((uintptr_t)a.y % 64 || a.y_stride * ysz % 64) && a.N * ysz > 1536;
  p.RB = p.multi ? 1 : torn ? 2 : 4;
  while (p.RB > 1 && (32 * p.RB * (p.chunk + LDS_PAD) > (p.RB == 4 ? room : HALF) ||
                      a.n / (32 * p.RB) < 2 * n_cu))
    p.RB /= 2;
  if (p.RB == 1) p.NW = WAVES;
  const int64_t PM = 32 * p.RB;
  p.tiles = a.off ? a.n / PM + a.G : (a.n + PM - 1) / PM;
  // No more blocks than CUs, or one to a tile: all waves to each.  Measured (eight
  // blocks to a workgroup : one, us): 1 x 4096 -> 4096 bf16 29.7 : 13.1, 64 x 4096
  // -> 4096 8-bit 22.3 : 15.2; with more blocks the rows are staged too often, 300 x
  // 1024 -> 1024 8-bit 8.3 : 11.4, 1000 x 1024 -> 1024 bf16 10.1 : 17.6.
  p.split = p.RB == 1 && (p.tiles * a.NB <= n_cu || a.NB == 1) && a.S >= 2 * WAVES;
  p.narrow = p.RB == 1 && !p.multi && !p.split && row_bytes <= narrow_bytes(a.w_type);
  const int WN = p.split ? 1 : p.NW;
  const int ntile = (a.NB + WN - 1) / WN;
  p.nsplit = (int)((2 * n_cu + p.tiles - 1) / p.tiles);
  if (p.nsplit > ntile || p.split) p.nsplit = ntile;
  return p;
}

hipError_t launch_linear(const LinearArgs &args, const LinearPlan &p, hipStream_t stream) {
  LinearArgs a = args;
  if (p.tile) {
    if (a.w_type == T_I8) return tiled<T_I8>(a, p.tile, stream);
    if (a.w_type == T_BF16) return tiled<T_BF16>(a, p.tile, stream);
    return tiled<T_F16>(a, p.tile, stream);
  }
  a.chunk = p.chunk;
  a.nsplit = p.nsplit;
  if (a.w_type == T_I8) {
    if (a.x_type == T_I8) return panel_rows<T_I8, T_I8>(a, p, stream);
    if (a.x_type == T_F32) return panel_rows<T_I8, T_F32>(a, p, stream);
    if (a.x_type == T_BF16) return panel_rows<T_I8, T_BF16>(a, p, stream);
    return panel_rows<T_I8, T_F16>(a, p, stream);
  }
  if (a.w_type == T_BF16) {
    if (a.x_type == T_F32) return panel_rows<T_BF16, T_F32>(a, p, stream);
    return panel_rows<T_BF16, T_BF16>(a, p, stream);
  }
  if (a.x_type == T_F32) return panel_rows<T_F16, T_F32>(a, p, stream);
  return panel_rows<T_F16, T_F16>(a, p, stream);
}

}  // namespace gnn
