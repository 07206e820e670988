// The products of a gated feed-forward block and of its gradients: rows x
// through gate and up weights, h = act(g) u, and down; backward, the gradients
// of g and u, of the rows and of the weights.
//
// Every product is C[m][n] = sum_k A(m, k) B(n, k) in tiles of 16-bit numbers
// on the matrix cores, sums in fp32.  An operand lies either with k contiguous
// ([m][k], rows of a table) or with k outermost ([k][m]: the weights of the
// backward pass, and everything of the weights' gradients, whose k are the
// rows).  The former goes to the matrix cores by 16-byte LDS reads, the latter
// by LDS reads that transpose 4 x 16 numbers: no operand is transposed in memory.
#include "rows_common.h"

namespace gnn {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef short s4v __attribute__((ext_vector_type(4)));
typedef short s8v __attribute__((ext_vector_type(8)));

typedef __attribute__((address_space(3))) unsigned char lds_byte;

constexpr int BK = 64;                  // k of a stage: 128 bytes of a row
constexpr uint32_t OUTSIDE = 1u << 31;  // a buffer offset that is out of range: reads zeros

template <int T>
__device__ __forceinline__ f4 mfma16(const s8v &a, const s8v &b, const f4 &c) {
  if constexpr (T == T_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a),
                                                   __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a),
                                                  __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// ---- activations ----
// act(g) and its derivative.  gelu is g Phi(g); 1 - erf(z) for z >= 0 is taken
// as t P(t) exp(-z^2), t = 1 / (1 + 0.3275911 z) (Abramowitz and Stegun, 7.1.26;
// off by at most 1.5e-7, a hundredth of a 16-bit number's last place at 1).
template <bool SLOPE>
__device__ __forceinline__ float activate(int act, float g, float *slope) {
  if (act == ACT_RELU) {
    if (SLOPE) *slope = g > 0.f ? 1.f : 0.f;
    return g > 0.f || g != g ? g : 0.f;
  }
  if (act == ACT_GELU) {
    const float z = fabsf(g) * 0.70710678118654752f;
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3275911f * z);
    const float e = __expf(-z * z);
    const float p = t * (0.254829592f +
                         t * (-0.284496736f +
                              t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
    const float tail = 0.5f * p * e;  // Phi(-|g|)
    const float phi = g >= 0.f ? 1.f - tail : tail;
    if (SLOPE) *slope = phi + g * (e * 0.39894228040143268f);
    return g * phi;
  }
  const float s = __builtin_amdgcn_rcpf(1.f + __expf(-g));
  if (act == ACT_SIGMOID) {
    if (SLOPE) *slope = s * (1.f - s);
    return s;
  }
  if (SLOPE) *slope = s * (1.f + g * (1.f - s));
  return g * s;
}

// ---- memory to LDS ----
// The next stage's numbers go to LDS without passing registers, 16 bytes a lane
// and 1 KB a wave's load.  The load is written in assembly because the compiler
// would let every LDS read wait for it; the stage's own wait stands before the
// barrier that ends a stage.
__device__ __forceinline__ i4 buffer_of(const void *p) {
  const uint64_t a = (uint64_t)p;
  return i4{(int32_t)a, (int32_t)(a >> 32), (int32_t)OUTSIDE, 0x00020000};
}
__device__ __forceinline__ void load_lds(uint32_t lds, uint32_t off, const i4 &buf) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(off), "s"(buf)
               : "memory");
}
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// One operand's part of a stage: R (m or n) by BK.
//
// k contiguous: rows of 128 bytes, whose eight 16-byte pieces are exchanged by
// the row's number, piece c of row r at c ^ (r & 7), so that the 16 rows that a
// read touches spread over all banks.
// k outermost: BK rows of R numbers, whose 32-byte units are exchanged by f(k): a
// transposing read takes one unit from each of eight k at a time (k & 3 and k >> 3
// & 1 differ), which then lie in different banks; of R = 64 two rows fill the
// banks, and their place tells k & 1 apart.
template <int R>
__device__ __forceinline__ int unit_of(int k) {
  return R == 64 ? ((k >> 1) & 1) | ((k >> 3) & 1) << 1 : (k & 3) | ((k >> 3) & 1) << 2;
}
template <int R, int NW, bool KS>
struct Staged {
  static constexpr int WIDTH = R, BYTES = R * BK * 2, LOADS = BYTES / 1024 / NW;
  uint32_t off[LOADS];  // a lane's offsets from the stage's first element

  // ext: how many of the R lie in the operand (a multiple of 8 with KS)
  __device__ __forceinline__ void init(int wave, int lane, int64_t ld, int32_t ext) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int q = wave * LOADS + i;
      if constexpr (!KS) {
        const int row = 8 * q + (lane >> 3), c = (lane & 7) ^ (lane >> 3);
        off[i] = row < ext ? (uint32_t)(row * (int32_t)ld * 2 + c * 16) : OUTSIDE;
      } else {
        const int at = q * 1024 + lane * 16, k = at / (R * 2), p = at % (R * 2);
        const int col = (((p >> 5) ^ unit_of<R>(k)) << 4) + ((p >> 4) & 1) * 8;
        off[i] = col < ext ? (uint32_t)(k * (int32_t)ld * 2 + col * 2) : OUTSIDE;
      }
    }
  }

  // left: how many k there are from the stage's first on
  __device__ __forceinline__ void issue(uint32_t lds, const i4 &buf, int wave, int lane,
                                        int32_t left) const {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) issue1(i, lds, buf, wave, lane, left);
  }
  __device__ __forceinline__ void issue1(int i, uint32_t lds, const i4 &buf, int wave, int lane,
                                         int32_t left) const {
    uint32_t o = off[i];
    if (left < BK) {
      const int k = KS ? ((wave * LOADS + i) * 1024 + lane * 16) / (R * 2)
                       : ((lane & 7) ^ (lane >> 3)) * 8;
      if (k >= left) o = OUTSIDE;
    }
    load_lds(lds + (wave * LOADS + i) * 1024, o, buf);
  }
};

// A lane's operand of the MFMA: of block b (16 m or n) from `first` on, k = 32 s +
// 8 (lane / 16) .. + 7.
template <int R, bool KS>
struct Frag {
  uint32_t at;
  int x;
  __device__ __forceinline__ void init(int first, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (!KS) {
      at = (first + i) * 128;
      x = g ^ (i & 7);
    } else {
      const int k = g * 8 + (i >> 2);
      at = k * (R * 2) + (((first >> 4) ^ unit_of<R>(k)) << 5) + (i & 3) * 8;
      x = 0;
    }
  }
  __device__ __forceinline__ s8v load(uint32_t lds, int b, int s) const {
    if constexpr (!KS) {
      typedef __attribute__((address_space(3))) s8v *p8;
      return *(p8)(uintptr_t)(lds + at + b * 2048 + ((x ^ (s * 4)) << 4));
    } else {
      typedef __attribute__((address_space(3))) s4v *p4;
      const uint32_t p = lds + (at ^ (b << 5)) + s * (32 * R * 2);
      const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)p);
      const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)(p + 4 * R * 2));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
};

// Four neighbouring 16-bit numbers, those below n stored.
template <int T>
__device__ __forceinline__ void store4(elem_t<T> *p, const f4 &v, int32_t n, bool whole) {
  typedef elem_t<T> e4 __attribute__((ext_vector_type(4)));
  const e4 r = __builtin_convertvector(v, e4);
  if (whole && n >= 4) {
    *(e4 *)p = r;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[j] = r[j];
  }
}

template <int T>
__device__ __forceinline__ f4 load4(const elem_t<T> *p, int32_t n) {
  f4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = p && j < n ? (float)p[j] : 0.f;
  return v;
}

// ---- the product ----
// WM x WN waves, each with MI x NI blocks of 16 x 16.  The n are the MFMA's
// first operand, so that a lane holds four neighbouring n of one m.
// GATE and GRAD: B is the gate's and the up projection's rows in turn, 16 NI / 2 of
// each to a wave, so that a wave has g and u of the same elements.  GRAD goes on
// with dh = dy Wd (k outermost) of these elements in registers of its own: dh is
// never rounded, nor in memory.
template <int T, int WM, int WN, int MI, int NI, bool AKS, bool BKS, int EPI>
__global__ __launch_bounds__(64 * WM * WN, 2) void gated_product(ProductArgs a) {
  constexpr int NW = WM * WN, TM = WM * MI * 16, TN = WN * NI * 16;
  constexpr bool DUAL = EPI == EPI_GATE || EPI == EPI_GRAD;
  constexpr int CN = DUAL ? TN / 2 : TN;  // columns of C in a tile
  typedef Staged<TM, NW, AKS> SA;
  typedef Staged<TN, NW, BKS> SB;
  constexpr int STAGE = SA::BYTES + SB::BYTES;
  typedef elem_t<T> E;
  extern __shared__ __attribute__((aligned(1024))) unsigned char shared[];
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_byte *)shared;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // Tiles in bands of 8 m tiles, column by column within a band; a compute die
  // (and its L2) gets a contiguous range of them.
  const int64_t per = (int64_t)a.mt * a.nt;
  int64_t t = xcd_remap(blockIdx.x, gridDim.x);
  const int32_t split = (int32_t)(t / per);
  t -= split * per;
  const int64_t band = t / (8 * (int64_t)a.nt), in = t - band * 8 * a.nt;
  const int32_t bm = (int32_t)min((int64_t)8, a.mt - band * 8);
  const int32_t tm = (int32_t)(band * 8 + in % bm), tn = (int32_t)(in / bm);
  const int64_t m0 = (int64_t)tm * TM;
  const int32_t n0 = tn * CN;

  SA sa;
  SB sb;
  // the third product's operands
  typedef Staged<EPI == EPI_GRAD ? CN : 128, NW, true> SD;
  static_assert(SD::BYTES <= SB::BYTES || EPI != EPI_GRAD, "its stages take the others' place");
  SA sy;
  SD sd;
  if constexpr (EPI == EPI_GRAD) {
    sy.init(wave, lane, a.lda2, (int32_t)min((int64_t)TM, a.M - m0));
    sd.init(wave, lane, a.ldb2, min(CN, a.N - n0));
  }
  sa.init(wave, lane, a.lda, (int32_t)min((int64_t)TM, a.M - m0));
  if constexpr (DUAL) {
    // stage row r: part (r / U) & 1 of column n0 + r / (2 U) * U + r % U
    constexpr int U = NI * 8;
#pragma unroll
    for (int i = 0; i < SB::LOADS; ++i) {
      const int row = 8 * (wave * SB::LOADS + i) + (lane >> 3), c = (lane & 7) ^ (lane >> 3);
      const int col = row / (2 * U) * U + row % U;
      sb.off[i] = n0 + col < a.N ? (uint32_t)(col * (int32_t)a.ldb * 2 + c * 16) : OUTSIDE;
    }
  } else {
    sb.init(wave, lane, a.ldb, min(TN, a.N - n0));
  }

  const int32_t seg_steps = (a.K + BK - 1) / BK;
  const int32_t steps = EPI == EPI_GRAD ? seg_steps + (a.K2 + BK - 1) / BK : seg_steps * a.segs;
  const int32_t first = (int32_t)min((int64_t)steps, (int64_t)split * a.split_steps);
  const int32_t end = (int32_t)min((int64_t)steps, (int64_t)first + a.split_steps);

  auto issue = [&](int32_t step, int buf) {
    const int32_t seg = step >= seg_steps ? 1 : 0, k = (step - seg * seg_steps) * BK;
    const int32_t left = a.K - k;
    const uint32_t to = lds + buf * STAGE;
    if constexpr (EPI == EPI_GRAD) {
      if (seg) {
        sy.issue(to, buffer_of((const E *)a.a[1] + m0 * a.lda2 + k), wave, lane, a.K2 - k);
        sd.issue(to + SA::BYTES, buffer_of((const E *)a.b2 + k * a.ldb2 + n0), wave, lane,
                 a.K2 - k);
        return;
      }
    }
    const E *pa = (const E *)a.a[seg] + (AKS ? k * a.lda + m0 : m0 * a.lda + k);
    sa.issue(to, buffer_of(pa), wave, lane, left);
    if constexpr (DUAL) {
      const i4 g = buffer_of((const E *)a.b[0] + n0 * a.ldb + k);
      const i4 u = buffer_of((const E *)a.b[1] + n0 * a.ldb + k);
#pragma unroll
      for (int i = 0; i < SB::LOADS; ++i) {
        const bool up = (8 * (wave * SB::LOADS + i) / (NI * 8)) & 1;
        sb.issue1(i, to + SA::BYTES, up ? u : g, wave, lane, left);
      }
    } else {
      const E *pb = (const E *)a.b[seg] + (BKS ? k * a.ldb + n0 : n0 * a.ldb + k);
      sb.issue(to + SA::BYTES, buffer_of(pb), wave, lane, left);
    }
  };

  const int wm = wave / WN, wn = wave % WN;
  Frag<TM, AKS> fa;
  Frag<TN, BKS> fb;
  fa.init(wm * MI * 16, lane);
  fb.init(wn * NI * 16, lane);
  f4 acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

  constexpr int HN = NI / 2;
  f4 third[EPI == EPI_GRAD ? MI : 1][EPI == EPI_GRAD ? HN : 1];
  const int32_t end1 = EPI == EPI_GRAD ? seg_steps : end;
  if (first < end) issue(first, 0);
  for (int32_t step = first; step < end1; ++step) {
    const int buf = (step - first) & 1;
    stage_barrier();
    if (step + 1 < end) issue(step + 1, buf ^ 1);
    const uint32_t la = lds + buf * STAGE, lb = la + SA::BYTES;
#pragma unroll
    for (int s = 0; s < BK / 32; ++s) {
      s8v xb[NI], xa[MI];
#pragma unroll
      for (int j = 0; j < NI; ++j) xb[j] = fb.load(lb, j, s);
#pragma unroll
      for (int i = 0; i < MI; ++i) xa[i] = fa.load(la, i, s);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = mfma16<T>(xb[j], xa[i], acc[i][j]);
    }
  }
  if constexpr (EPI == EPI_GRAD) {
    Frag<SD::WIDTH, true> fd;
    fd.init(wn * HN * 16, lane);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < HN; ++j) third[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    for (int32_t step = end1; step < end; ++step) {
      const int buf = step & 1;
      stage_barrier();
      if (step + 1 < end) issue(step + 1, buf ^ 1);
      const uint32_t la = lds + buf * STAGE, lb = la + SA::BYTES;
#pragma unroll
      for (int s = 0; s < BK / 32; ++s) {
        s8v xb[HN], xa[MI];
#pragma unroll
        for (int j = 0; j < HN; ++j) xb[j] = fd.load(lb, j, s);
#pragma unroll
        for (int i = 0; i < MI; ++i) xa[i] = fa.load(la, i, s);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < HN; ++j) third[i][j] = mfma16<T>(xb[j], xa[i], third[i][j]);
      }
    }
  }

  // A lane's part of block (i, j): row mrow(i), columns 4 (lane / 16) .. + 3 of
  // the block's.
  const int li = lane & 15, lg = lane >> 4;
  const int64_t mw = m0 + wm * MI * 16 + li;
  if constexpr (DUAL) {
    const int32_t c0 = n0 + wn * HN * 16 + lg * 4;
    f4 bg[HN], bu[HN], sg[HN], su[HN];
#pragma unroll
    for (int j = 0; j < HN; ++j) {
      const int32_t c = c0 + j * 16;
      bg[j] = load4<T>((const E *)a.bias[0] ? (const E *)a.bias[0] + c : nullptr, a.N - c);
      bu[j] = load4<T>((const E *)a.bias[1] ? (const E *)a.bias[1] + c : nullptr, a.N - c);
      sg[j] = su[j] = f4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int64_t m = mw + i * 16;
#pragma unroll
      for (int j = 0; j < HN; ++j) {
        const int32_t c = c0 + j * 16;
        if (m < a.M && c < a.ldc) {  // ldc: N and its padding, in which everything is zero
          const f4 g = acc[i][j] + bg[j], u = acc[i][j + HN] + bu[j];
          E *ph = (E *)a.c + m * a.ldc + c;
          f4 h;
          if constexpr (EPI == EPI_GATE) {
#pragma unroll
            for (int v = 0; v < 4; ++v) h[v] = activate<false>(a.act, g[v], nullptr) * u[v];
            store4<T>(ph, h, 4, true);
          } else {
            const f4 dh = third[i][j];
            f4 dg, du;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              float slope;
              const float s = activate<true>(a.act, g[v], &slope);
              h[v] = s * u[v];
              dg[v] = dh[v] * u[v] * slope;
              du[v] = dh[v] * s;
            }
            sg[j] += dg;
            su[j] += du;
            E *pd = (E *)a.c2 + m * 2 * a.ldc + c;
            store4<T>(ph, h, 4, true);
            store4<T>(pd, dg, 4, true);
            store4<T>(pd + a.ldc, du, 4, true);
          }
        }
      }
    }
    // Column sums of dg and du over the wave's rows (the biases' gradients),
    // from the numbers before they are rounded.
    if (EPI == EPI_GRAD && a.sums) {
      float *ps = a.sums + ((int64_t)tm * WM + wm) * 2 * a.ldc;
#pragma unroll
      for (int j = 0; j < HN; ++j) {
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
          for (int o = 1; o < 16; o *= 2) {
            sg[j][v] += __shfl_xor(sg[j][v], o);
            su[j][v] += __shfl_xor(su[j][v], o);
          }
        const int32_t c = c0 + j * 16;
        if (li == 0 && c < a.ldc) {
          *(f4 *)(ps + c) = sg[j];
          *(f4 *)(ps + a.ldc + c) = su[j];
        }
      }
    }
  } else if constexpr (EPI == EPI_PART) {
    float *part = (float *)a.c + (int64_t)split * a.M * a.ldc;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int64_t m = mw + i * 16;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int32_t c = n0 + wn * NI * 16 + j * 16 + lg * 4;
        if (m < a.M && c < a.ldc) *(f4 *)(part + m * a.ldc + c) = acc[i][j];
      }
    }
  } else {
    const bool whole = a.ldc % 4 == 0 && ((uintptr_t)a.c | (uintptr_t)a.c2) % 8 == 0;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int32_t c = n0 + wn * NI * 16 + j * 16 + lg * 4;
      const f4 b = load4<T>((const E *)a.bias[0] ? (const E *)a.bias[0] + c : nullptr, a.N - c);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int64_t m = mw + i * 16;
        const bool one = m < a.c_rows;
        const int64_t r = one ? m : m - a.c_rows;
        if (m < a.M && r < a.c_valid)
          store4<T>((one ? (E *)a.c : (E *)a.c2) + r * a.ldc + c, acc[i][j] + b, a.N - c, whole);
      }
    }
  }
}

// ---- few rows ----
// Up to 16 MB rows: every weight is read once, from memory straight into the
// MFMA's registers, and there is nothing else to wait for.  A workgroup takes 16
// columns (of gate and of up alike, GATE), its waves a share of the k each; their
// sums meet in LDS.  k of a step go to the lanes in a different order than in
// memory, the same for both operands, so that the four lanes of a row read 128
// neighbouring bytes.
template <int T, int MB, int NW, bool GATE>
__global__ __launch_bounds__(64 * NW) void gated_few(ProductArgs a) {
  typedef elem_t<T> E;
  constexpr int NB = GATE ? 2 : 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int32_t n0 = blockIdx.x * 16;
  const E *pa[MB], *pb[NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
    pa[i] = (const E *)a.a[0] + min((int64_t)(i * 16 + li), a.M - 1) * a.lda;
#pragma unroll
  for (int j = 0; j < NB; ++j) pb[j] = (const E *)a.b[j] + (int64_t)min(n0 + li, a.N - 1) * a.ldb;
  f4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
  const int32_t whole = a.K / BK;
  auto step = [&](int32_t k, bool end) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int32_t kk = k + lg * 16 + s * 8;
      Raw8<T> xb[NB], xa[MB];
#pragma unroll
      for (int j = 0; j < NB; ++j)
        xb[j] = end ? load8_end<T>(pb[j], kk, a.K) : load8<T>(pb[j], kk);
#pragma unroll
      for (int i = 0; i < MB; ++i)
        xa[i] = end ? load8_end<T>(pa[i], kk, a.K) : load8<T>(pa[i], kk);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
          acc[i][j] = mfma16<T>(__builtin_bit_cast(s8v, xb[j].v), __builtin_bit_cast(s8v, xa[i].v),
                                acc[i][j]);
    }
  };
  int32_t st = wave;
#pragma unroll 4
  for (; st < whole; st += NW) step(st * BK, false);
  if (st == whole && a.K % BK) step(st * BK, true);

  __shared__ f4 sum[NW][MB * NB][64];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) sum[wave][i * NB + j][lane] = acc[i][j];
  __syncthreads();
  for (int i = wave; i < MB; i += NW) {
    f4 v[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      v[j] = sum[0][i * NB + j][lane];
      for (int w = 1; w < NW; ++w) v[j] += sum[w][i * NB + j][lane];
    }
    const int64_t m = i * 16 + li;
    const int32_t c = n0 + lg * 4;
#pragma unroll
    for (int j = 0; j < NB; ++j)
      v[j] += load4<T>((const E *)a.bias[j] ? (const E *)a.bias[j] + c : nullptr, a.N - c);
    if (m >= a.M) continue;
    if constexpr (GATE) {
      f4 h;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        h[q] = c + q < a.N ? activate<false>(a.act, v[0][q], nullptr) * v[1][q] : 0.f;
      if (c < a.ldc) store4<T>((E *)a.c + m * a.ldc + c, h, 4, true);
    } else {
      store4<T>((E *)a.c + m * a.ldc + c, v[0], a.N - c,
                a.ldc % 4 == 0 && (uintptr_t)a.c % 8 == 0);
    }
  }
}

// Sums of the parts of a product whose k were shared out: part [splits][M][ldp]
// to 16-bit rows, those from c_rows on to c2.
template <int T>
__global__ __launch_bounds__(256) void join_parts(JoinArgs a) {
  typedef elem_t<T> E;
  const int64_t quads = a.ldp / 4, total = a.M * quads;
  for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < total;
       q += (int64_t)gridDim.x * 256) {
    const int64_t m = q / quads;
    const int32_t c = (int32_t)(q - m * quads) * 4;
    const bool one = m < a.c_rows;
    const int64_t r = one ? m : m - a.c_rows;
    if (r >= a.c_valid) continue;
    const float *p = a.part + m * a.ldp + c;
    f4 v = f4{0.f, 0.f, 0.f, 0.f};
    for (int32_t s = 0; s < a.splits; ++s) v += *(const f4 *)(p + s * a.M * a.ldp);
    store4<T>((one ? (E *)a.c : (E *)a.c2) + r * a.ldc + c, v, a.N - c, false);
  }
}

template <int T, int WM, int WN, int MI, int NI, bool AKS, bool BKS, int EPI>
hipError_t product_go(const ProductArgs &in, hipStream_t stream) {
  ProductArgs a = in;
  constexpr int TM = WM * MI * 16, TN = WN * NI * 16;
  constexpr int CN = EPI == EPI_GATE || EPI == EPI_GRAD ? TN / 2 : TN;
  a.mt = (int32_t)((a.M + TM - 1) / TM);
  a.nt = (a.N + CN - 1) / CN;
  const int64_t grid = (int64_t)a.mt * a.nt * a.splits;
  if (grid * 64 * WM * WN >= (int64_t)1 << 32) return hipErrorInvalidConfiguration;
  return launch_lds(gated_product<T, WM, WN, MI, NI, AKS, BKS, EPI>, dim3((unsigned)grid),
                    dim3(64 * WM * WN), (TM + TN) * BK * 2 * 2, stream, a);
}

template <int T, bool AKS, bool BKS, int EPI>
hipError_t product_tile(const ProductArgs &a, int tile, hipStream_t stream) {
  if (tile == TILE_256) return product_go<T, 2, 4, 8, 4, AKS, BKS, EPI>(a, stream);
  if (tile == TILE_256x128) return product_go<T, 4, 2, 4, 4, AKS, BKS, EPI>(a, stream);
  return product_go<T, 2, 2, 4, 4, AKS, BKS, EPI>(a, stream);
}

template <int T>
hipError_t product_t(const ProductArgs &a, int kind, int tile, hipStream_t stream) {
  switch (kind) {
    case PRODUCT_GATE: return product_tile<T, false, false, EPI_GATE>(a, tile, stream);
    case PRODUCT_GRAD: return product_tile<T, false, false, EPI_GRAD>(a, tile, stream);
    case PRODUCT_DOWN: return product_tile<T, false, false, EPI_ROWS>(a, tile, stream);
    case PRODUCT_ROWS: return product_tile<T, false, true, EPI_ROWS>(a, tile, stream);
    default:
      if (a.splits > 1) return product_tile<T, true, true, EPI_PART>(a, tile, stream);
      return product_tile<T, true, true, EPI_ROWS>(a, tile, stream);
  }
}

template <int T, bool GATE>
hipError_t few_t(const ProductArgs &a, hipStream_t stream) {
  const dim3 grid((a.N + 15) / 16);
  constexpr int NW = GATE ? 8 : 16;
  switch ((a.M + 15) / 16) {
    case 1: return launch(gated_few<T, 1, NW, GATE>, grid, dim3(64 * NW), 0, stream, a);
    case 2: return launch(gated_few<T, 2, 8, GATE>, grid, dim3(512), 0, stream, a);
    case 3: return launch(gated_few<T, 3, 8, GATE>, grid, dim3(512), 0, stream, a);
    default: return launch(gated_few<T, 4, 8, GATE>, grid, dim3(512), 0, stream, a);
  }
}

}  // namespace

// The tile of a product and into how many parts its k go.
ProductPlan product_plan(int kind, int64_t M, int64_t N, int64_t K, int n_cu) {
  ProductPlan p;
  const bool dual = kind == PRODUCT_GATE || kind == PRODUCT_GRAD;
  auto tiles = [&](int64_t tm, int64_t tn) {
    if (dual) tn /= 2;
    return ((M + tm - 1) / tm) * ((N + tn - 1) / tn);
  };
  const int64_t wide = dual ? 2 * N : N;
  if (wide > 128 && M > 128 && (tiles(256, 256) >= n_cu || kind == PRODUCT_WEIGHTS))
    p.tile = TILE_256;
  else if (M > 128 && (tiles(256, 128) >= n_cu || kind == PRODUCT_WEIGHTS))
    p.tile = TILE_256x128;
  else
    p.tile = TILE_128;
  const int64_t tm = p.tile == TILE_128 ? 128 : 256, tn = p.tile == TILE_256 ? 256 : 128;
  if (kind == PRODUCT_WEIGHTS) {
    // as many parts as fill the chip, of eight stages at least
    const int64_t steps = (K + BK - 1) / BK, n = tiles(tm, tn);
    const int64_t fill = p.tile == TILE_128 ? 2 * (int64_t)n_cu : n_cu;
    int64_t s = std::min(fill / n, steps / 8);
    if (s < 1) s = 1;
    p.split_steps = (int32_t)std::max<int64_t>(1, (steps + s - 1) / s);
    p.splits = (int32_t)std::max<int64_t>(1, (steps + p.split_steps - 1) / p.split_steps);
  } else {
    p.splits = 1;
    p.split_steps = INT32_MAX;
  }
  return p;
}

hipError_t launch_product(const ProductArgs &a, int kind, int type, int tile, hipStream_t stream) {
  return type == T_BF16 ? product_t<T_BF16>(a, kind, tile, stream)
                        : product_t<T_F16>(a, kind, tile, stream);
}

hipError_t launch_few(const ProductArgs &a, bool gate, int type, hipStream_t stream) {
  if (type == T_BF16) return gate ? few_t<T_BF16, true>(a, stream) : few_t<T_BF16, false>(a, stream);
  return gate ? few_t<T_F16, true>(a, stream) : few_t<T_F16, false>(a, stream);
}

hipError_t launch_join(const JoinArgs &a, int type, hipStream_t stream) {
  const int64_t quads = a.M * (a.ldp / 4);
  const dim3 grid((unsigned)std::min<int64_t>((quads + 255) / 256, 4096));
  return type == T_BF16 ? launch(join_parts<T_BF16>, grid, dim3(256), 0, stream, a)
                        : launch(join_parts<T_F16>, grid, dim3(256), 0, stream, a);
}

}  // namespace gnn
