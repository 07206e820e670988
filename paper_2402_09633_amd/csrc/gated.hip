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
#include <type_traits>
#include <utility>

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
// off by at most 1.5e-7, a 6000th of the last place of an fp16 number next to 1).
template <int act, bool SLOPE>
__device__ __forceinline__ float activate(float g, float *slope) {
  if constexpr (act == ACT_RELU) {
    if (SLOPE) *slope = g > 0.f ? 1.f : 0.f;
    return g > 0.f || g != g ? g : 0.f;
  }
  if constexpr (act == ACT_GELU && !SLOPE) {
    // g Phi(g) = max(g, 0) - |g| Phi(-|g|)
    const float t = __builtin_amdgcn_rcpf(1.f + 0.23164188f * fabsf(g));
    const float e = __builtin_amdgcn_exp2f(g * g * -0.72134752f);
    const float p = t * (0.127414796f +
                         t * (-0.142248368f +
                              t * (0.7107068705f + t * (-0.7265760135f + t * 0.5307027145f))));
    // (the product has vanished long before 100, and an infinite g shall not undo that)
    return __builtin_fmaf(-fminf(fabsf(g), 100.f), p * e, 0.5f * (g + fabsf(g)));
  }
  if constexpr (act == ACT_GELU) {
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
  if constexpr (act == ACT_SIGMOID) {
    if (SLOPE) *slope = s * (1.f - s);
    return s;
  }
  if (SLOPE) *slope = s * (1.f + g * (1.f - s));
  return g * s;
}

// f with the activation as a constant: one branch for all elements, between which
// the instructions of several then overlap.
template <typename F>
__host__ __device__ __forceinline__ auto with_activation(int act, F &&f) {
  switch (act) {
    case ACT_GELU: return f(std::integral_constant<int, ACT_GELU>{});
    case ACT_SIGMOID: return f(std::integral_constant<int, ACT_SIGMOID>{});
    case ACT_RELU: return f(std::integral_constant<int, ACT_RELU>{});
    default: return f(std::integral_constant<int, ACT_SILU>{});
  }
}

// ---- memory to LDS ----
// The next stage's numbers go to LDS without passing registers, 16 bytes a lane
// and 1 KB a wave's load.  The load is written in assembly because the compiler
// would let every LDS read wait for it; the stage's own wait stands before the
// barrier that ends a stage.
// `on` false: nothing lies in range, so that a load only clears its place.
__device__ __forceinline__ i4 buffer_of(const void *p, bool on) {
  const uint64_t a = (uint64_t)p;
  return i4{(int32_t)a, (int32_t)(a >> 32) & 0xffff, on ? (int32_t)OUTSIDE : 0, 0x00020000};
}
__device__ __forceinline__ void load_lds(uint32_t lds, uint32_t off, const i4 &buf) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(off), "s"(buf)
               : "memory", "m0");
}
// All but the last N loads of this wave have come, and all waves are here.
template <int N>
__device__ __forceinline__ void stage_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
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

  // Load i of a stage from whose first k on there are `left`.
  __device__ __forceinline__ uint32_t from(int i, int wave, int lane, int32_t left) const {
    const int k = KS ? ((wave * LOADS + i) * 1024 + lane * 16) / (R * 2)
                     : ((lane & 7) ^ (lane >> 3)) * 8;
    return k < left ? off[i] : OUTSIDE;
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

// Sixteen values of each of 16 neighbouring lanes: lane i's result is the sum of
// value i over the 16.  Every step trades half of the values that are left.
__device__ __forceinline__ float sums16(const float (&v)[16]) {
  const int li = threadIdx.x & 15;
  float w[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) w[j] = v[j];
  auto step = [&](auto half, auto ctrl) {
    constexpr int H = half.value;
    const bool up = li & H;
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const float mine = up ? w[j + H] : w[j], theirs = up ? w[j] : w[j + H];
      w[j] = mine + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(theirs), ctrl.value,
                                                             0xf, 0xf, true));
    }
  };
  step(std::integral_constant<int, 8>{}, std::integral_constant<int, 0x140>{});  // 15 - lane of 16
  step(std::integral_constant<int, 4>{}, std::integral_constant<int, 0x141>{});  // 7 - lane of 8
  step(std::integral_constant<int, 2>{}, std::integral_constant<int, 0x4e>{});   // lane ^ 2
  step(std::integral_constant<int, 1>{}, std::integral_constant<int, 0xb1>{});   // lane ^ 1
  return w[0];
}

// What rounding v to 16 bits leaves (nothing where that is no number).
template <int T>
__device__ __forceinline__ f4 rest4(const f4 &v) {
  typedef elem_t<T> e4 __attribute__((ext_vector_type(4)));
  const f4 hi = __builtin_convertvector(__builtin_convertvector(v, e4), f4);
  f4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = fabsf(hi[j]) < INFINITY ? v[j] - hi[j] : 0.f;
  return r;
}

// ---- the range of fp16 gradients ----
// h and the gradients of g and u go on in 16 bits, and fp16 numbers below 2^-14 lose
// digits: with dy near 1e-5 the weights' gradients of 256 -> 512 -> 256 were off by 4e-3
// of themselves, 19 times what rounding them costs.  So the backward pass keeps them
// times a power of two each, the largest with which none can leave the range and never
// below 1, and its products take it out again, in fp32 and exactly.  By the
// Cauchy-Schwarz inequality, with the largest sum of squares of a row of each table,
//   |dh| <= |dy| sqrt(sum over n of max over h of Wd[n][h]^2)
//   |g| <= |x| |Wg| + |bg|, |u| <= |x| |Wu| + |bu|, |du| <= |dh| |act(g)|
//   |dg| <= 1.13 |dh| |u|, |h| <= |act(g)| |u|; |act(g)| <= |g|, sigmoid's <= 1.
// For random rows and weights these bounds are 2^3 to 2^11 times the largest number,
// which leaves more digits below it than fp16 has.
// Elements that are no numbers are left out: what they reach is none either.
//
// Bound by memory: everything is read once.  A workgroup takes rows of one table and
// leaves its part of one of the SIZES numbers (of x, dy, gate, up, down, the biases);
// tables that the products cannot read as they lie are copied on the way, as
// pack_tables does for bf16.  300000 x 128 -> 256 -> 128: 34 us of 549 forward and
// backward (4.5 TB/s); 8192 x 2048 -> 8192 -> 2048 31 (5.4 TB/s); 48 x 256 -> 1024 -> 256
// 6.6; 4097 x 391 -> 1031 -> 259, copies among it, 12 (copies alone 5.3).
template <int T>
__global__ __launch_bounds__(1024) void gated_sizes(SizeArgs a) {
  typedef elem_t<T> E;
  typedef typename Raw8<T>::vec e8;
  constexpr int NW = 16, ROWS = 4, LOADS = 4;  // on their way at once
  __shared__ float parts[NW];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int t = 0;
  while (t + 1 < SIZES && (int)blockIdx.x >= a.first[t + 1]) ++t;
  const int64_t n = (int)blockIdx.x < a.first[SIZES] ? a.rows[t] : 0;
  const int32_t K = a.width[t];
  const bool top = t >= SIZE_DOWN;  // the largest number of a row, not its sum of squares
  int L = 1;                        // lanes to a row
  while (L < 64 && 8 * L < K) L *= 2;
  const int64_t step = (int64_t)(a.first[t + 1] - a.first[t]) * NW * (64 / L);
  const E *x = (const E *)a.x[t];
  E *copy = (E *)a.y[t];
  const int64_t pitch = (K + 7) & ~7;
  auto add = [&](float s, const Raw8<T> &raw) {
    float p = 0.f;
    if (top) {
      p = top_of<T>(max_bits<T>(raw, 0));
      p *= p;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) p = __builtin_fmaf((float)raw.v[j], (float)raw.v[j], p);
    }
    if (!(p < INFINITY)) {  // an element is no number: a branch that is hardly ever taken
      asm volatile("");
      p = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = (float)raw.v[j], m = fabsf(v) < INFINITY ? v : 0.f;
        p = top ? fmaxf(p, m * m) : __builtin_fmaf(m, m, p);
      }
    }
    return top ? fmaxf(s, p) : s + p;
  };
  auto over_row = [&](float s) {
    for (int o = 1; o < L; o *= 2) {
      const float w = __shfl_xor(s, o);
      s = top ? fmaxf(s, w) : s + w;
    }
    return s;
  };
  float most = 0.f;
  // every lane of a wave goes round as often as its first: they add together
  int64_t r0 = ((int64_t)((int)blockIdx.x - a.first[t]) * NW + wave) * (64 / L);
  auto row_done = [&](int64_t r, float s) {
    s = over_row(s);
    if (t != SIZE_DOWN)
      most = fmaxf(most, s);
    else if (r < n && lane % L == 0)
      most += s;
  };
  if (K <= 512) {  // a row is one load of its lanes: four rows at a time
    const int k = 8 * (lane % L);
    for (; r0 < n; r0 += ROWS * step) {
      Raw8<T> raw[ROWS];
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int64_t r = r0 + i * step + lane / L;
        const E *row = x + min(r, n - 1) * a.stride[t];
        raw[i] = k + 8 <= K ? load8<T>(row, k) : load8_end<T>(row, k, K);
      }
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int64_t r = r0 + i * step + lane / L;
        if (copy && r < n && k < K) *(e8 *)(copy + r * pitch + k) = raw[i].v;
        row_done(r, add(0.f, raw[i]));
      }
    }
  } else {  // four loads of a row at a time
    for (; r0 < n; r0 += step) {
      const E *row = x + r0 * a.stride[t];
      float s = 0.f;
      for (int k0 = 8 * lane; k0 < K; k0 += LOADS * 512) {
        Raw8<T> raw[LOADS];
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int k = k0 + i * 512;
          raw[i] = k + 8 <= K ? load8<T>(row, k) : load8_end<T>(row, k, K);
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int k = k0 + i * 512;
          if (copy && k < K) *(e8 *)(copy + r0 * pitch + k) = raw[i].v;
          s = add(s, raw[i]);
        }
      }
      row_done(r0, s);
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const float w = __shfl_xor(most, o);
    most = t == SIZE_DOWN ? most + w : fmaxf(most, w);
  }
  if (lane == 0) parts[wave] = most;
  __syncthreads();
  if (threadIdx.x < SIZES) {
    float v = parts[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) v = t == SIZE_DOWN ? v + parts[w] : fmaxf(v, parts[w]);
    a.part[threadIdx.x * SIZE_PARTS + blockIdx.x] = (int)threadIdx.x == t ? v : 0.f;
  }
}

// What the gradients of g and u, and h, are multiplied by, from gated_sizes' parts.
struct GradScales {
  float grad, h;
};
__device__ __forceinline__ GradScales grad_scales(const float *part, int act) {
  static_assert(SIZE_PARTS == 4 * 64, "four parts to a lane");
  const int lane = threadIdx.x & 63;
  float v[SIZES];
#pragma unroll
  for (int q = 0; q < SIZES; ++q) {
    const f4 p = ((const f4 *)(part + q * SIZE_PARTS))[lane];
    v[q] = q == SIZE_DOWN ? (p[0] + p[1]) + (p[2] + p[3])
                          : fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3]));
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2)
#pragma unroll
    for (int q = 0; q < SIZES; ++q) {
      const float w = __shfl_xor(v[q], o);
      v[q] = q == SIZE_DOWN ? v[q] + w : fmaxf(v[q], w);
    }
  const float dh = sqrtf(v[1]) * sqrtf(v[4]);
  const float u = sqrtf(v[0]) * sqrtf(v[3]) + sqrtf(v[6]);
  const float s = act == ACT_SIGMOID ? 1.f : sqrtf(v[0]) * sqrtf(v[2]) + sqrtf(v[5]);
  // 65504 / 1.05: the sums of up to 16384 products and squares are off by less than that
  auto scale = [](float most) {
    const float q = fminf(62384.f / most, 0x1p40f);
    const float two = __uint_as_float(__float_as_uint(q) & 0x7f800000u);
    return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(two > 1.f ? two : 1.f)));
  };
  return GradScales{scale(dh * fmaxf(1.13f * u, s)), scale(s * u)};
}

// ---- the product ----
// Half a stage (k of one MFMA) of a wave's blocks, while the operands of the next
// half come from LDS and, in every second half, a stage from memory: loads stand
// between the MFMAs in the order in which they are written here, so that the
// matrix cores never wait for a run of them.
template <int N, typename F, int... Q>
__device__ __forceinline__ void each(F &&f, std::integer_sequence<int, Q...>) {
  (f(std::integral_constant<int, Q>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F &&f) {
  each<N>(f, std::make_integer_sequence<int, N>{});
}

template <int T, int MI, int NI, int D, typename LA, typename LB, typename DMA>
__device__ __forceinline__ void half_stage(f4 (&acc)[MI][NI], const s8v (&xa)[MI],
                                           const s8v (&xb)[NI], s8v (&ya)[MI], s8v (&yb)[NI],
                                           LA &&load_a, LB &&load_b, DMA &&dma) {
  constexpr int MF = MI * NI, R = MI + NI;
  each<MF>([&](auto at) {
    constexpr int q = at.value, i = q % MI, j = q / MI;
    // reads in the order in which the MFMAs need them, done by three quarters
    constexpr int r0 = (4 * R * q + 3 * MF - 1) / (3 * MF), r1 = (4 * R * (q + 1) + 3 * MF - 1) / (3 * MF);
    each<(r1 < R ? r1 : R) - (r0 < R ? r0 : R)>([&](auto n) {
      constexpr int r = r0 + n.value;
      if constexpr (r == 0)
        yb[0] = load_b(0);
      else if constexpr (r <= MI)
        ya[r - 1] = load_a(r - 1);
      else
        yb[r - MI] = load_b(r - MI);
    });
    constexpr int d0 = (D * q + MF - 1) / MF, d1 = (D * (q + 1) + MF - 1) / MF;
    each<d1 - d0>([&](auto n) { dma(d0 + n.value); });
    acc[i][j] = mfma16<T>(xb[j], xa[i], acc[i][j]);
    if constexpr (d1 > d0 || (r1 > r0 && r0 < R)) __builtin_amdgcn_sched_barrier(0);
  });
}

// WM x WN waves, each with MI x NI blocks of 16 x 16.  The n are the MFMA's
// first operand, so that a lane holds four neighbouring n of one m.  S stages lie
// in LDS; a stage's place is filled again as soon as its second half is in
// registers, so that memory has S - 1/2 stages' time.  Where two waves share a SIMD
// and their sums leave no room for two halves' operands (!AHEAD), a half's operands
// are read just before it, and the other wave's MFMAs cover that.
// GATE and GRAD: B is the gate's and the up projection's rows in turn, 16 NI / 2 of
// each to a wave, so that a wave has g and u of the same elements.  GRAD goes on
// with dh = dy Wd (k outermost) of these elements in registers of its own: dh is
// never rounded, nor in memory.
// ACT: GRAD's activation; its sums leave no registers for a choice among four.
template <int T, int WM, int WN, int MI, int NI, int S, bool AKS, bool BKS, int EPI, int ACT>
__global__ __launch_bounds__(64 * WM * WN, WM * WN == 4 && (MI * NI > 16 || S > 2) ? 1 : 2) void
gated_product(ProductArgs a) {
  constexpr int NW = WM * WN, TM = WM * MI * 16, TN = WN * NI * 16;
  constexpr bool DUAL = EPI == EPI_GATE || EPI == EPI_GRAD;
  constexpr int CN = DUAL ? TN / 2 : TN;  // columns of C in a tile
  typedef Staged<TM, NW, AKS> SA;
  typedef Staged<TN, NW, BKS> SB;
  constexpr int STAGE = SA::BYTES + SB::BYTES;
  typedef elem_t<T> E;
  // WEIGHTS of tiles whose sums leave room: also sums of A over k, by MFMAs with ones
  constexpr bool SUMS = AKS && MI * NI <= 16;
  constexpr bool LO = EPI == EPI_GRAD && MI * NI <= 8;  // the tile that few rows take
  constexpr bool AHEAD = !(NW == 8 && MI * NI >= 32 && EPI == EPI_GRAD);
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

  GradScales scales{1.f, 1.f};
  if constexpr (T == T_F16 && EPI == EPI_GRAD) {
    scales = grad_scales(a.sizes, ACT);
    if (blockIdx.x == 0 && threadIdx.x == 0) {  // for the products that follow
      a.scales[0] = 1.f / scales.grad;
      a.scales[1] = 1.f / scales.h;
    }
    // here, where no other registers are taken
    asm volatile("" : "+s"(scales.grad), "+s"(scales.h));
  }

  const int32_t seg_steps = (a.K + BK - 1) / BK;
  const int32_t steps = EPI == EPI_GRAD ? seg_steps + (a.K2 + BK - 1) / BK : seg_steps * a.segs;
  const int32_t first = (int32_t)min((int64_t)steps, (int64_t)split * a.split_steps);
  const int32_t end = (int32_t)min((int64_t)steps, (int64_t)first + a.split_steps);

  // A stage on its way.
  struct Coming {
    i4 a, b, b2;
    int32_t left;
    uint32_t to;
    bool second;  // of GRAD's third product
  };
  constexpr int LOADS = SA::LOADS + SB::LOADS;
  auto coming = [&](int32_t step, uint32_t to) {
    Coming c;
    const bool on = step < end;
    const int32_t seg = (step >= seg_steps) + (EPI != EPI_GRAD && step >= 2 * seg_steps) +
                        (EPI != EPI_GRAD && step >= 3 * seg_steps);
    const int32_t k = (step - seg * seg_steps) * BK;
    c.to = to;
    c.second = EPI == EPI_GRAD && seg > 0;
    c.left = (c.second ? a.K2 : a.K) - k;
    const E *pa = (const E *)a.a[seg], *pb = (const E *)a.b[DUAL ? 0 : seg];
    const int64_t lda = c.second ? a.lda2 : a.lda;
    c.a = buffer_of(pa + (AKS ? k * lda + m0 : m0 * lda + k), on);
    c.b = buffer_of(pb + (BKS ? k * a.ldb + n0 : n0 * a.ldb + k), on);
    if constexpr (DUAL) c.b2 = buffer_of((const E *)a.b[1] + n0 * a.ldb + k, on);
    if (EPI == EPI_GRAD && c.second) c.b = buffer_of((const E *)a.b2 + k * a.ldb2 + n0, on);
    return c;
  };
  auto load = [&](int i, const Coming &c) {
    if (i < SA::LOADS) {
      uint32_t o = sa.from(i, wave, lane, c.left);
      if constexpr (EPI == EPI_GRAD) o = c.second ? sy.from(i, wave, lane, c.left) : o;
      load_lds(c.to + (wave * SA::LOADS + i) * 1024, o, c.a);
      return;
    }
    i -= SA::LOADS;
    uint32_t o = sb.from(i, wave, lane, c.left);
    if constexpr (DUAL) {
      const bool up = (8 * (wave * SB::LOADS + i) / (NI * 8)) & 1;
      const i4 buf = up && !c.second ? c.b2 : c.b;
      int32_t at = wave * SB::LOADS + i;
      if constexpr (EPI == EPI_GRAD) {
        // the third product's part is smaller: the loads left over clear the rest
        if (i < SD::LOADS) {
          o = c.second ? sd.from(i, wave, lane, c.left) : o;
          at = c.second ? wave * SD::LOADS + i : at;
        } else {
          o = c.second ? OUTSIDE : o;
          at = c.second ? NW * SD::LOADS + wave * (SB::LOADS - SD::LOADS) + i - SD::LOADS : at;
        }
      }
      load_lds(c.to + SA::BYTES + at * 1024, o, buf);
    } else {
      load_lds(c.to + SA::BYTES + (wave * SB::LOADS + i) * 1024, o, c.b);
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

  f4 over_k[SUMS ? MI : 1];
  const bool sums = SUMS && a.sums && tn == 0 && wn == 0;
  typedef E e8v __attribute__((ext_vector_type(8)));
  const s8v ones = __builtin_bit_cast(s8v, e8v{1, 1, 1, 1, 1, 1, 1, 1});
#pragma unroll
  for (f4 &v : over_k) v = f4{0.f, 0.f, 0.f, 0.f};
  auto add_up = [&](const s8v(&xa)[MI]) {
    if constexpr (SUMS)
      if (sums)
#pragma unroll
        for (int i = 0; i < MI; ++i) over_k[i] = mfma16<T>(ones, xa[i], over_k[i]);
  };
  constexpr int HN = NI / 2;
  f4 third[EPI == EPI_GRAD ? MI : 1][EPI == EPI_GRAD ? HN : 1];
  if (first < end) {
    uint32_t now = lds;  // the stage that is multiplied
    auto after = [&](uint32_t p) { return p + STAGE == lds + S * STAGE ? lds : p + STAGE; };
#pragma unroll
    for (int i = 0; i < (AHEAD ? S : S - 1); ++i) {
      const Coming c = coming(first + i, lds + i * STAGE);
#pragma unroll
      for (int d = 0; d < LOADS; ++d) load(d, c);
    }
    if constexpr (AHEAD) stage_barrier<(S - 1) * LOADS>();
    auto stages = [&](auto &sum, auto &fb, int32_t from, int32_t to) {
      constexpr int N = sizeof(sum[0]) / sizeof(f4);
      if constexpr (!AHEAD) {
        for (int32_t step = from; step < to; ++step) {
          stage_barrier<(S - 2) * LOADS>();
          const uint32_t last = now == lds ? lds + (S - 1) * STAGE : now - STAGE;
          const Coming c = coming(step + S - 1, last);
#pragma unroll
          for (int d = 0; d < LOADS; ++d) load(d, c);
#pragma unroll
          for (int s = 0; s < BK / 32; ++s) {
            s8v xa[MI], xb[N];
#pragma unroll
            for (int j = 0; j < N; ++j) xb[j] = fb.load(now + SA::BYTES, j, s);
#pragma unroll
            for (int i = 0; i < MI; ++i) xa[i] = fa.load(now, i, s);
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
              for (int j = 0; j < N; ++j) sum[i][j] = mfma16<T>(xb[j], xa[i], sum[i][j]);
          }
          now = after(now);
        }
        return;
      }
      s8v xa[MI], ya[MI], xb[N], yb[N];
#pragma unroll
      for (int j = 0; j < N; ++j) xb[j] = fb.load(now + SA::BYTES, j, 0);
#pragma unroll
      for (int i = 0; i < MI; ++i) xa[i] = fa.load(now, i, 0);
      for (int32_t step = from; step < to; ++step) {
        const uint32_t next = after(now);
        half_stage<T, MI, N, 0>(
            sum, xa, xb, ya, yb, [&](int i) { return fa.load(now, i, 1); },
            [&](int j) { return fb.load(now + SA::BYTES, j, 1); }, [](int) {});
        add_up(xa);
        stage_barrier<(S - 2) * LOADS>();
        const Coming c = coming(step + S, now);
        // after the last of these stages, what is read here is not used
        half_stage<T, MI, N, LOADS>(
            sum, ya, yb, xa, xb, [&](int i) { return fa.load(next, i, 0); },
            [&](int j) { return fb.load(next + SA::BYTES, j, 0); }, [&](int d) { load(d, c); });
        add_up(ya);
        now = next;
      }
    };
    if constexpr (EPI == EPI_GRAD) {
      Frag<SD::WIDTH, true> fd;
      fd.init(wn * HN * 16, lane);
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < HN; ++j) third[i][j] = f4{0.f, 0.f, 0.f, 0.f};
      stages(acc, fb, 0, seg_steps);
      stages(third, fd, seg_steps, end);
    } else {
      stages(acc, fb, first, end);
    }
    stage_barrier<0>();  // no load is under way when the workgroup ends
  }

  // A lane's part of block (i, j): row mrow(i), columns 4 (lane / 16) .. + 3 of
  // the block's.
  const int li = lane & 15, lg = lane >> 4;
  const int64_t mw = m0 + wm * MI * 16 + li;
  if constexpr (SUMS) {
    if (sums && lg == 0)
#pragma unroll
      for (int i = 0; i < MI; ++i)
        if (mw + i * 16 < a.M) a.sums[split * a.M + mw + i * 16] = over_k[i][0];
  }
  if constexpr (DUAL) {
    const int32_t c0 = n0 + wn * HN * 16 + lg * 4;
    f4 bg[HN], bu[HN];
    float over_m[16];  // GRAD: dg, then du of the lane's columns, over its rows
    static_assert(EPI != EPI_GRAD || HN == 2, "sums16");
#pragma unroll
    for (float &v : over_m) v = 0.f;
#pragma unroll
    for (int j = 0; j < HN; ++j) {
      const int32_t c = c0 + j * 16;
      bg[j] = load4<T>((const E *)a.bias[0] ? (const E *)a.bias[0] + c : nullptr, a.N - c);
      bu[j] = load4<T>((const E *)a.bias[1] ? (const E *)a.bias[1] + c : nullptr, a.N - c);
    }
    auto elements = [&](auto which) {
      constexpr int A = which.value;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int64_t m = mw + i * 16;
#pragma unroll
        for (int j = 0; j < HN; ++j) {
          const int32_t c = c0 + j * 16;
          if (m < a.M && c < a.ldc) {  // ldc: N and its padding, in which everything is zero
            const f4 g = acc[i][j] + bg[j], u = acc[i][j + HN] + bu[j];
            const int64_t times = LO && a.lo ? 2 : 1;
            E *ph = (E *)a.c + m * times * a.ldc + c;
            f4 h;
            if constexpr (EPI == EPI_GATE) {
#pragma unroll
              for (int v = 0; v < 4; ++v) h[v] = activate<A, false>(g[v], nullptr) * u[v];
              store4<T>(ph, h, 4, true);
            } else {
              const f4 dh = third[i][j];
              f4 dg, du;
#pragma unroll
              for (int v = 0; v < 4; ++v) {
                float slope;
                const float s = activate<A, true>(g[v], &slope);
                h[v] = s * u[v];
                dg[v] = dh[v] * u[v] * slope;
                du[v] = dh[v] * s;
                over_m[j * 4 + v] += dg[v];
                over_m[8 + j * 4 + v] += du[v];
              }
              if constexpr (T == T_F16) {
                h *= scales.h;
                dg *= scales.grad;
                du *= scales.grad;
              }
              E *pd = (E *)a.c2 + m * times * 2 * a.ldc + c;
              store4<T>(ph, h, 4, true);
              store4<T>(pd, dg, 4, true);
              store4<T>(pd + a.ldc, du, 4, true);
              if (LO && a.lo) {
                store4<T>(ph + a.ldc, rest4<T>(h), 4, true);
                store4<T>(pd + 2 * a.ldc, rest4<T>(dg), 4, true);
                store4<T>(pd + 3 * a.ldc, rest4<T>(du), 4, true);
              }
            }
          }
        }
      }
    };
    if constexpr (EPI == EPI_GRAD)
      elements(std::integral_constant<int, ACT>{});
    else
      with_activation(a.act, elements);
    // Sums over the wave's rows (for the biases' gradients), from the numbers before
    // they are rounded.
    if (EPI == EPI_GRAD && a.sums) {
      const float v = sums16(over_m);
      const int32_t c = n0 + wn * HN * 16 + ((li >> 2) & 1) * 16 + lg * 4 + (li & 3);
      if (c < a.ldc)
        a.sums[((int64_t)tm * WM + wm) * 2 * a.ldc + (li >> 3) * a.ldc + c] = v;
    }
  } else if constexpr (EPI == EPI_PART) {
    const float scale = T == T_F16 && a.scale ? *a.scale : 1.f;
    float *part = (float *)a.c + (int64_t)split * a.M * a.ldc;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int64_t m = mw + i * 16;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int32_t c = n0 + wn * NI * 16 + j * 16 + lg * 4;
        if (m < a.M && c < a.ldc) *(f4 *)(part + m * a.ldc + c) = acc[i][j] * scale;
      }
    }
  } else {
    const bool whole = a.ldc % 4 == 0 && ((uintptr_t)a.c | (uintptr_t)a.c2) % 8 == 0;
    const float scale = T == T_F16 && BKS && a.scale ? *a.scale : 1.f;
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
          store4<T>((one ? (E *)a.c : (E *)a.c2) + r * a.ldc + c,
                    (T == T_F16 && BKS ? acc[i][j] * scale : acc[i][j]) + b, a.N - c, whole);
      }
    }
  }
}

// ---- narrow blocks in one pass ----
// Rows of up to 128 elements in and out: what lies between them stays in registers.
// A wave keeps its 16 MI rows of x and its sums of y, and goes through the hidden
// elements 32 at a time, whose weights (32 rows of gate and of up, 32 columns of
// down) come to LDS a step ahead.  A lane's sums of g and u are, for one row, four
// neighbouring hidden elements of either block of 16; their products in 16 bits
// are the eight k that the MFMA of the down projection wants of a lane, if Wd's
// are read in the same order (4 lg + j and 16 + 4 lg + j).
//
// GRAD: dh from the rows of dy, which a wave keeps too, then h, dg and du, which go to
// memory for the weights' gradients, and dx from dg and du as y from h; Wd, Wg and
// Wu are read from the same places by transposing reads.
//
// Bound by the activation's instructions (half of the issue slots of 300000 x 128 ->
// 512 -> 128 bf16 gelu; MFMAs a fifth); GRAD also by the rows that it writes, 2.3 GB
// for 1000513 x 128 -> 256 -> 128.  Workgroups of four waves, three to a CU (GRAD: two)
// run out of step and cover one another's waits: 188 us for the former, 240 with two,
// 278 with one of eight waves, 411 through the products above.  GRAD of the latter
// takes 700, the products 1093.
constexpr int THIN_WAVES = 4, THIN_HIDDEN = 2048;
constexpr int thin_stages(bool grad) { return grad ? 3 : 2; }

// KS, NS: 32s of elements of x and of y (2 or 4).
template <int T, int MI, int KS, int NS, bool GRAD, int ACT>
__global__ __launch_bounds__(64 * THIN_WAVES, GRAD ? 2 : 3) void gated_thin(ProductArgs a) {
  constexpr int STAGES = thin_stages(GRAD);
  typedef elem_t<T> E;
  typedef E e4 __attribute__((ext_vector_type(4)));
  typedef typename Raw8<T>::vec e8;
  typedef __attribute__((address_space(3))) s8v *p8;
  typedef __attribute__((address_space(3))) s4v *p4;
  constexpr int NW = THIN_WAVES;
  constexpr int ROW = KS * 64;  // bytes of a gate or up row in LDS
  constexpr int UP = 32 * ROW, DOWN = 2 * UP, STAGE = DOWN + 8192;
  constexpr int LG = DOWN / 1024 / NW, LD = 8 / NW, LOADS = LG + LD;  // loads of a wave
  constexpr int OUT = GRAD ? 2 * KS : 2 * NS;  // blocks of 16 of dx or y
  extern __shared__ __attribute__((aligned(1024))) unsigned char shared[];
  const uint32_t lds = (uint32_t)(uintptr_t)(lds_byte *)shared;
  const uint32_t bias = lds + STAGES * STAGE;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int32_t steps = (a.N + 31) / 32;  // N: hidden elements, K2: columns of y

  // biases of gate and up as they are, [2][steps * 32], zeros where there are none
  for (int32_t i = threadIdx.x; i < 2 * 32 * steps; i += 64 * NW) {
    const int32_t p = i >= 32 * steps, h = i - p * 32 * steps;
    const E *b = (const E *)a.bias[p];
    ((__attribute__((address_space(3))) E *)(uintptr_t)bias)[i] = b && h < a.N ? b[h] : (E)0.f;
  }

  // A wave's loads: gate and up rows of ROW bytes, then rows of down of 64 bytes.
  // Their 16-byte pieces are exchanged by the row's number so that the eight rows
  // that a read touches at a time, or the eight pairs of pieces that a transposing
  // one does, lie in different banks.
  auto swap_k = [](int r) { return KS == 4 ? (r & 7) << 1 : ((r >> 1) & 3) << 1; };
  auto swap_d = [](int r) { return (r >> 2) & 3; };
  uint32_t off[LOADS];
  int32_t at[LOADS];  // hidden element of the load's lane, from the step's first
#pragma unroll
  for (int i = 0; i < LG; ++i) {
    const int p = (wave * LG + i) * 1024 + lane * 16, r = p / ROW, c = (p % ROW / 16) ^ swap_k(r);
    at[i] = r % 32;
    off[i] = c * 8 < a.K ? (uint32_t)((r % 32) * (int32_t)a.ldb * 2 + c * 16) : OUTSIDE;
  }
#pragma unroll
  for (int i = 0; i < LD; ++i) {
    const int p = (wave * LD + i) * 1024 + lane * 16, r = p / 64, c = (p % 64 / 16) ^ swap_d(r);
    at[LG + i] = c * 8;
    off[LG + i] = r < a.K2 ? (uint32_t)(r * (int32_t)a.ldb2 * 2 + c * 16) : OUTSIDE;
  }
  auto issue = [&](int32_t step, uint32_t to) {
    const bool on = step < steps;
    const int32_t left = a.N - step * 32;
#pragma unroll
    for (int i = 0; i < LG; ++i) {
      const bool up = (wave * LG + i) * 1024 >= UP;
      load_lds(to + (wave * LG + i) * 1024, at[i] < left ? off[i] : OUTSIDE,
               buffer_of((const E *)a.b[up ? 1 : 0] + (int64_t)step * 32 * a.ldb, on));
    }
#pragma unroll
    for (int i = 0; i < LD; ++i)
      load_lds(to + DOWN + (wave * LD + i) * 1024, at[LG + i] < left ? off[LG + i] : OUTSIDE,
               buffer_of((const E *)a.b2 + step * 32, on));
  };

  const int64_t m0 = ((int64_t)blockIdx.x * NW + wave) * (16 * MI) + li;
  auto rows = [&](const void *p, int64_t ld, int32_t width, auto &to) {
    constexpr int S = sizeof(to[0]) / sizeof(s8v);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const E *row = (const E *)p + min(m0 + i * 16, a.M - 1) * ld;
#pragma unroll
      for (int k = 0; k < S; ++k) {
        const int c = k * 32 + lg * 8;
        to[i][k] = __builtin_bit_cast(
            s8v, (width == S * 32 ? load8<T>(row, c) : load8_end<T>(row, c, width)).v);
      }
    }
  };
  s8v x[MI][KS], dy[MI][GRAD ? NS : 1];
  rows(a.a[0], a.lda, a.K, x);
  if constexpr (GRAD) rows(a.a[1], a.lda2, a.K2, dy);
  f4 y[MI][OUT];  // GRAD: dx
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int n = 0; n < OUT; ++n) y[i][n] = f4{0.f, 0.f, 0.f, 0.f};
  GradScales scales{1.f, 1.f};
  if constexpr (T == T_F16 && GRAD) {
    scales = grad_scales(a.sizes, ACT);
    if (blockIdx.x == 0 && threadIdx.x == 0) {  // for the products that follow
      a.scales[0] = 1.f / scales.grad;
      a.scales[1] = 1.f / scales.h;
    }
  }
  // the compiler's own loads are counted with the stages': none may be under way
  __syncthreads();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) issue(s, lds + s * STAGE);

  uint32_t now = lds;
  for (int32_t step = 0; step < steps; ++step) {
    // Loads come back in their order, so this stage is here when no more operations
    // are under way than the next ones have loads, whatever the stores do.
    stage_barrier<(STAGES - 2) * LOADS>();
    issue(step + STAGES - 1, now == lds ? lds + (STAGES - 1) * STAGE : now - STAGE);
    f4 sum[2][2][MI], dh[2][MI];  // g, u and dh of two blocks of 16 hidden elements
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const s4v raw = *(p4)(uintptr_t)(bias + 2 * (32 * (p * steps + step) + b * 16 + lg * 4));
        const f4 v = __builtin_convertvector(__builtin_bit_cast(e4, raw), f4);
#pragma unroll
        for (int i = 0; i < MI; ++i) sum[p][b][i] = v;
      }
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const s8v w = *(p8)(uintptr_t)(now + p * UP + (b * 16 + li) * ROW +
                                         (((k * 4 + lg) ^ swap_k(li)) << 4));
#pragma unroll
          for (int i = 0; i < MI; ++i) sum[p][b][i] = mfma16<T>(w, x[i][k], sum[p][b][i]);
        }
    // rows r .. r + 3, 16 columns from piece 2 b on, to a lane's column
    const int tr = li >> 2, tc = (li >> 1) & 1, tb = (li & 1) * 8;
    if constexpr (GRAD) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int i = 0; i < MI; ++i) dh[b][i] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NS; ++k) {
          const int r = k * 32 + lg * 8 + tr;
          const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)(
              now + DOWN + r * 64 + (((2 * b + tc) ^ swap_d(r)) << 4) + tb));
          const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)(
              now + DOWN + (r + 4) * 64 + (((2 * b + tc) ^ swap_d(r + 4)) << 4) + tb));
          const s8v w = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
          for (int i = 0; i < MI; ++i) dh[b][i] = mfma16<T>(w, dy[i][k], dh[b][i]);
        }
      }
    }
    s8v h[MI], dg[MI], du[MI];
    float over_m[16];  // dg, then du of the lane's columns, over its rows
#pragma unroll
    for (float &v : over_m) v = 0.f;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      f8 v, vg, vu;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float g = sum[0][j / 4][i][j % 4], u = sum[1][j / 4][i][j % 4];
        if constexpr (GRAD) {
          float slope;
          const float s = activate<ACT, true>(g, &slope), d = dh[j / 4][i][j % 4];
          v[j] = s * u;
          vg[j] = d * u * slope;
          vu[j] = d * s;
          if (m0 + i * 16 < a.M) {
            over_m[j] += vg[j];
            over_m[8 + j] += vu[j];
          }
        } else {
          v[j] = activate<ACT, false>(g, nullptr) * u;
        }
      }
      if constexpr (T == T_F16 && GRAD) {
        v *= scales.h;
        vg *= scales.grad;
        vu *= scales.grad;
      }
      h[i] = __builtin_bit_cast(s8v, __builtin_convertvector(v, e8));
      if constexpr (GRAD) {
        dg[i] = __builtin_bit_cast(s8v, __builtin_convertvector(vg, e8));
        du[i] = __builtin_bit_cast(s8v, __builtin_convertvector(vu, e8));
      }
    }
    if constexpr (GRAD) {
      // Lanes of odd lg trade with those before them, so that each has eight
      // neighbouring elements: 4 lg .. of the first 16 (even), of the second (odd).
      const int32_t c = step * 32 + (lg & 1) * 16 + (lg & 2) * 4;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int64_t m = m0 + i * 16;
        auto store = [&](const s8v &v, E *to) {
          u4 w = __builtin_bit_cast(u4, v);
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const auto t = __builtin_amdgcn_permlane16_swap(w[q], w[q + 2], false, false);
            w[q] = t[0];
            w[q + 2] = t[1];
          }
          if (m < a.M && c < a.ldc2) *(u4 *)(to + c) = w;
        };
        store(h[i], (E *)a.c2 + m * a.ldc2);
        store(dg[i], (E *)a.c3 + m * 2 * a.ldc2);
        store(du[i], (E *)a.c3 + m * 2 * a.ldc2 + a.ldc2);
      }
      if (a.sums) {
        const float v = sums16(over_m);
        const int32_t e = step * 32 + ((li >> 2) & 1) * 16 + lg * 4 + (li & 3);
        if (e < a.ldc2)
          a.sums[((int64_t)blockIdx.x * NW + wave) * 2 * a.ldc2 + (li >> 3) * a.ldc2 + e] = v;
      }
#pragma unroll
      for (int n = 0; n < OUT; ++n)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const int r = lg * 4 + tr;
          const uint32_t row = now + p * UP + r * ROW + (((2 * n + tc) ^ swap_k(r)) << 4) + tb;
          const s4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)row);
          // sixteen rows on, where the pieces are exchanged alike
          const s4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((p4)(uintptr_t)(row + 16 * ROW));
          const s8v w = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
          for (int i = 0; i < MI; ++i) y[i][n] = mfma16<T>(w, p ? du[i] : dg[i], y[i][n]);
        }
    } else {
#pragma unroll
      for (int n = 0; n < OUT; ++n) {
        const uint32_t row = now + DOWN + (n * 16 + li) * 64 + (lg & 1) * 8;
        const s4v lo = *(p4)(uintptr_t)(row + (((lg >> 1) ^ swap_d(li)) << 4));
        const s4v hi = *(p4)(uintptr_t)(row + (((2 + (lg >> 1)) ^ swap_d(li)) << 4));
        const s8v w = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int i = 0; i < MI; ++i) y[i][n] = mfma16<T>(w, h[i], y[i][n]);
      }
    }
    now = now + STAGE == bias ? lds : now + STAGE;
  }
  stage_barrier<0>();  // no load is under way when the workgroup ends

  const int32_t width = GRAD ? a.K : a.K2;
  const float undo = 1.f / scales.grad;
  const bool whole = a.ldc % 4 == 0 && (uintptr_t)a.c % 8 == 0;
#pragma unroll
  for (int n = 0; n < OUT; ++n) {
    const int32_t c = n * 16 + lg * 4;
    const f4 b = load4<T>(!GRAD && a.bias2 ? (const E *)a.bias2 + c : nullptr, width - c);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int64_t m = m0 + i * 16;
      if (m < a.M)
        store4<T>((E *)a.c + m * a.ldc + c, (T == T_F16 && GRAD ? y[i][n] * undo : y[i][n]) + b,
                  width - c, whole);
    }
  }
}

// ---- few rows ----
// Up to 16 MB rows: every weight is read once, from memory straight into the
// MFMA's registers, and there is nothing else to wait for.  A workgroup takes 16 NC
// columns (of gate and of up alike, GATE), its waves a share of the k each; their
// sums meet in LDS.  k of a step go to the lanes in a different order than in
// memory, the same for both operands, so that the four lanes of a row read 128
// neighbouring bytes.
//
// With up to 16 rows the errors of h's rounding do not average out over a result (2 x
// 36 -> 114 -> 4386 bf16: 1.6 times the error of rounding the exact result, where many
// rows have 1.4), and another operand costs nothing beside the weights: h goes on in
// two 16-bit numbers, the second what the first one's rounding left.  (48 rows of 2048
// -> 8192 -> 2048 would take 45.5 us so, 39.5 without.)
//
// The down projection has few columns and many k, so several workgroups (gridDim.y)
// share a column's k, and few_join adds up what they leave: 8192 -> 2048, one row,
// 12.3 us without.  (One kernel whose last workgroup adds up took 99: a fence
// between compute dies writes their caches back.)
template <int T, int MB, int NC, int NW, bool GATE>
__global__ __launch_bounds__(64 * NW) void gated_few(ProductArgs a) {
  typedef elem_t<T> E;
  constexpr int NB = GATE ? 2 * NC : NC;
  constexpr bool TWO = MB == 1;
  __shared__ f4 sum[NW][MB * NB][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int32_t n0 = blockIdx.x * 16 * NC;
  const E *pa[MB], *pb[NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
    pa[i] = (const E *)a.a[0] + min((int64_t)(i * 16 + li), a.M - 1) * a.lda;
#pragma unroll
  for (int j = 0; j < NB; ++j)
    pb[j] = (const E *)a.b[j / NC] + (int64_t)min(n0 + j % NC * 16 + li, a.N - 1) * a.ldb;
  f4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
  const int32_t whole = a.K / BK, step_k = NW * gridDim.y;
  auto step = [&](int32_t k, bool end) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int32_t kk = k + lg * 16 + s * 8;
      Raw8<T> xb[NB], xa[MB], xl[MB];
#pragma unroll
      for (int j = 0; j < NB; ++j)
        xb[j] = end ? load8_end<T>(pb[j], kk, a.K) : load8<T>(pb[j], kk);
#pragma unroll
      for (int i = 0; i < MB; ++i)
        xa[i] = end ? load8_end<T>(pa[i], kk, a.K) : load8<T>(pa[i], kk);
      if constexpr (TWO && !GATE)
#pragma unroll
        for (int i = 0; i < MB; ++i)
          xl[i] = end ? load8_end<T>(pa[i] + a.lo, kk, a.K) : load8<T>(pa[i] + a.lo, kk);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const s8v w = __builtin_bit_cast(s8v, xb[j].v);
          acc[i][j] = mfma16<T>(w, __builtin_bit_cast(s8v, xa[i].v), acc[i][j]);
          if constexpr (TWO && !GATE)
            acc[i][j] = mfma16<T>(w, __builtin_bit_cast(s8v, xl[i].v), acc[i][j]);
        }
    }
  };
  int32_t st = wave + NW * blockIdx.y;
#pragma unroll(MB == 1 ? 8 : 4)
  for (; st < whole; st += step_k) step(st * BK, false);
  if (st == whole && a.K % BK) step(st * BK, true);

#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) sum[wave][i * NB + j][lane] = acc[i][j];
  __syncthreads();
  if (!GATE && gridDim.y > 1) {
    f4 *mine = (f4 *)a.part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (MB * NB * 64);
    for (int q = wave; q < MB * NB; q += NW) {
      f4 v = sum[0][q][lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) v += sum[w][q][lane];
      mine[q * 64 + lane] = v;
    }
    return;
  }
  for (int q = wave; q < MB * NC; q += NW) {
    const int i = q / NC, j0 = q % NC;
    f4 v[GATE ? 2 : 1];
#pragma unroll
    for (int p = 0; p < (GATE ? 2 : 1); ++p) {
      const int at = i * NB + p * NC + j0;
      v[p] = sum[0][at][lane];
#pragma unroll
      for (int w = 1; w < NW; ++w) v[p] += sum[w][at][lane];
    }
    const int64_t m = i * 16 + li;
    const int32_t c = n0 + j0 * 16 + lg * 4;
#pragma unroll
    for (int p = 0; p < (GATE ? 2 : 1); ++p)
      v[p] += load4<T>((const E *)a.bias[p] ? (const E *)a.bias[p] + c : nullptr, a.N - c);
    if (m >= a.M) continue;
    if constexpr (GATE) {
      f4 h;
      with_activation(a.act, [&](auto act) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          h[e] = c + e < a.N ? activate<act.value, false>(v[0][e], nullptr) * v[1][e] : 0.f;
      });
      if (c < (TWO ? a.lo : a.ldc)) {
        store4<T>((E *)a.c + m * a.ldc + c, h, 4, true);
        if (TWO) store4<T>((E *)a.c + m * a.ldc + a.lo + c, rest4<T>(h), 4, true);
      }
    } else {
      store4<T>((E *)a.c + m * a.ldc + c, v[0], a.N - c,
                a.ldc % 4 == 0 && (uintptr_t)a.c % 8 == 0);
    }
  }
}

// A wave adds up one block of 16 x 16: `parts` sums of it, `blocks` blocks apart.
template <int T>
__global__ __launch_bounds__(64) void few_join(ProductArgs a, int32_t parts, int32_t mb,
                                               int32_t nc) {
  typedef elem_t<T> E;
  const int lane = threadIdx.x, blk = blockIdx.x, blocks = gridDim.x;
  f4 v = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int32_t y = 0; y < parts; ++y)
    v += ((const f4 *)a.part)[((int64_t)y * blocks + blk) * 64 + lane];
  // blocks lie as gated_few's workgroups have them: [column group][m][column]
  const int in = blk % (mb * nc);
  const int64_t m = in / nc * 16 + (lane & 15);
  const int32_t c = (blk / (mb * nc) * nc + in % nc) * 16 + (lane >> 4) * 4;
  if (m >= a.M) return;
  v += load4<T>((const E *)a.bias[0] ? (const E *)a.bias[0] + c : nullptr, a.N - c);
  store4<T>((E *)a.c + m * a.ldc + c, v, a.N - c, a.ldc % 4 == 0 && (uintptr_t)a.c % 8 == 0);
}

// Tables that the products cannot read as they lie (at odd addresses, or with rows
// of odd lengths) to aligned rows with zeros behind them, all in one launch (63 x 65
// -> 523 -> 8 bf16 forward and backward: 51 us; with a launch to each 10 more).  The
// backward pass of fp16 copies them in gated_sizes.
template <int T>
__global__ __launch_bounds__(256) void pack_tables(PackArgs a) {
  typedef elem_t<T> E;
  typedef typename Raw8<T>::vec e8;
  int t = 0;
  while (t + 1 < a.count && blockIdx.x >= (uint32_t)a.first[t + 1]) ++t;
  const int64_t units = (a.width[t] + 7) / 8, total = a.rows[t] * units;
  const int64_t blocks = a.first[t + 1] - a.first[t];
  for (int64_t u = (blockIdx.x - a.first[t]) * 256 + threadIdx.x; u < total; u += blocks * 256) {
    const int64_t r = u / units;
    const int k = (int)(u - r * units) * 8;
    const E *row = (const E *)a.x[t] + r * a.stride[t];
    const Raw8<T> v = k + 8 <= a.width[t] ? load8<T>(row, k) : load8_end<T>(row, k, a.width[t]);
    *(e8 *)((E *)a.y[t] + u * 8) = v.v;
  }
}

// Sums of the parts of a product whose k were shared out: part [splits][M][ldp]
// to 16-bit rows, those from c_rows on to c2.  Sixteen waves share the parts of 64
// quads of columns: 253 parts of 128 x 256 took 73 us with a thread to a quad.
template <int T>
__global__ __launch_bounds__(1024) void join_parts(JoinArgs a) {
  typedef elem_t<T> E;
  __shared__ f4 sum[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t quads = a.ldp / 4, total = a.M * quads;
  const int64_t q = (int64_t)blockIdx.x * 64 + lane;
  f4 v = f4{0.f, 0.f, 0.f, 0.f};
  if (q < total) {
    const f4 *p = (const f4 *)a.part + q;
#pragma unroll 4
    for (int32_t s = wave; s < a.splits; s += 16) v += p[s * total];
  }
  sum[wave][lane] = v;
  __syncthreads();
  const int64_t m = q / quads, r = m < a.c_rows ? m : m - a.c_rows;
  const int32_t c = (int32_t)(q - m * quads) * 4;
  if (wave || q >= total || r >= a.c_valid) return;
  const int n = min(a.splits, 16);
  for (int w = 1; w < n; ++w) v += sum[w][lane];
  store4<T>((m < a.c_rows ? (E *)a.c : (E *)a.c2) + r * a.ldc + c, v, a.N - c, false);
}

template <int T, int WM, int WN, int MI, int NI, int S, bool AKS, bool BKS, int EPI>
hipError_t product_go(const ProductArgs &in, hipStream_t stream) {
  ProductArgs a = in;
  constexpr int TM = WM * MI * 16, TN = WN * NI * 16;
  constexpr int CN = EPI == EPI_GATE || EPI == EPI_GRAD ? TN / 2 : TN;
  a.mt = (int32_t)((a.M + TM - 1) / TM);
  a.nt = (a.N + CN - 1) / CN;
  const int64_t grid = (int64_t)a.mt * a.nt * a.splits;
  if (grid * 64 * WM * WN >= (int64_t)1 << 32) return hipErrorInvalidConfiguration;
  auto go = [&](auto act) {
    return launch_lds(gated_product<T, WM, WN, MI, NI, S, AKS, BKS, EPI, act.value>,
                      dim3((unsigned)grid), dim3(64 * WM * WN), (TM + TN) * BK * 2 * S, stream, a);
  };
  if constexpr (EPI == EPI_GRAD)
    return with_activation(a.act, go);
  else
    return go(std::integral_constant<int, ACT_SILU>{});
}

template <int T, bool AKS, bool BKS, int EPI>
hipError_t product_tile(const ProductArgs &a, int tile, hipStream_t stream) {
  // Four waves of 128 x 128 read least from LDS, eight of 128 x 64 hide more.  Two
  // projections of 8192 x 2048 -> 8192 take 512 us with eight, 610 with four; the
  // gradients of their weights and rows, whose LDS reads are twice as many, 458 and
  // 452 with four, 580 and 534 with eight.  GRAD takes 890 to 1030 so (0.8 to 0.93
  // PFLOP/s, its operands read just before their use), 1105 in tiles of 256 x 128 with
  // operands ahead.
  if (tile == TILE_256) {
    if constexpr (EPI == EPI_ROWS && BKS)
      return product_go<T, 2, 2, 8, 8, 2, AKS, BKS, EPI>(a, stream);
    else
      return product_go<T, 2, 4, 8, 4, 2, AKS, BKS, EPI>(a, stream);
  }
  if (tile == TILE_256x128) return product_go<T, 4, 2, 4, 4, 3, AKS, BKS, EPI>(a, stream);
  if (tile == TILE_128) return product_go<T, 2, 2, 4, 4, 2, AKS, BKS, EPI>(a, stream);
  return product_go<T, 4, 2, 2, 4, 4, AKS, BKS, EPI>(a, stream);
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

template <int T, int KS, int NS, bool GRAD>
hipError_t thin_go(const ProductArgs &a, hipStream_t stream) {
  constexpr int MI = THIN_ROWS / 16 / THIN_WAVES;
  const size_t lds = thin_stages(GRAD) * (2 * 32 * KS * 64 + 8192) + (size_t)(a.N + 31) / 32 * 128;
  const dim3 grid((unsigned)((a.M + THIN_ROWS - 1) / THIN_ROWS)), block(64 * THIN_WAVES);
  return with_activation(a.act, [&](auto act) {
    return launch_lds(gated_thin<T, MI, KS, NS, GRAD, act.value>, grid, block, lds, stream, a);
  });
}

template <int T, bool GRAD>
hipError_t thin_t(const ProductArgs &a, hipStream_t stream) {
  if (a.K > 64)
    return a.K2 > 64 ? thin_go<T, 4, 4, GRAD>(a, stream) : thin_go<T, 4, 2, GRAD>(a, stream);
  return a.K2 > 64 ? thin_go<T, 2, 4, GRAD>(a, stream) : thin_go<T, 2, 2, GRAD>(a, stream);
}

template <int T, bool GATE, int MB, int NC>
hipError_t few_go(const ProductArgs &a, int splits, hipStream_t stream) {
  const int n = (a.N + 16 * NC - 1) / (16 * NC);
  constexpr int NW = MB == 1 && !GATE ? 16 : 8;
  const hipError_t e =
      launch(gated_few<T, MB, NC, NW, GATE>, dim3(n, splits), dim3(64 * NW), 0, stream, a);
  if (e != hipSuccess || splits == 1) return e;
  return launch(few_join<T>, dim3(n * MB * NC), dim3(64), 0, stream, a, splits, MB, NC);
}

template <int T, bool GATE>
hipError_t few_t(const ProductArgs &a, int splits, hipStream_t stream) {
  switch ((a.M + 15) / 16) {
    case 1: return few_go<T, GATE, 1, 1>(a, splits, stream);
    case 2: return few_go<T, GATE, 2, FEW_COLUMNS>(a, splits, stream);
    case 3: return few_go<T, GATE, 3, FEW_COLUMNS>(a, splits, stream);
    default: return few_go<T, GATE, 4, FEW_COLUMNS>(a, splits, stream);
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
  // The tile whose rounds over the chip take least; a round's cost is next to that of
  // two workgroups of 128 x 128 on a CU.  us of a forward / backward bf16 call by the
  // rule, and with 128 x 128, 256 x 128, 256 x 256 and four stages of 128 x 128 throughout
  // (one run of all; clocks of other runs differ by some percent):
  // 4097 x 391 -> 1031 -> 259     45 / 115   50 / 124  56 / 136  68 / 165  50 / 119
  // 8192 x 2048 -> 8192 -> 2048   702 / 1987 826 / 2535 732 / 2248 663 / 1981 945 / 2868
  // 1622 x 5084 -> 2893 -> 1191   159 / 485  216 / 560 210 / 537 219 / 503 191 / 550
  // 4096 x 1024 -> 4096 -> 1024   101 / 427  119 / 381 124 / 388 147 / 526 135 / 397
  // 1000 x 512 -> 2048 -> 512     32 / 110   36 / 126  43 / 138  64 / 206  32 / 113
  // 30000 x 256 -> 1024 -> 256    77 / 248   81 / 240  87 / 247  86 / 269  114 / 284
  // 6774 x 1056 -> 32 -> 960      24 / 57    23 / 64   27 / 70   40 / 108  25 / 61
  // 100000 x 160 -> 320 -> 160    90 / 258   86 / 246  100 / 253 87 / 257  124 / 293
  // 300 x 2048 -> 2048 -> 2048    38 / 99    49 / 119  54 / 129  87 / 227  39 / 103
  // The rule does not count what writing and joining parts costs, and loses by up to 12%
  // where that decides (the fourth row backward).
  static constexpr struct {
    int tile, tm, tn, to_cu;
    double cost;
  } all[] = {{TILE_256, 256, 256, 1, 1.6},
             {TILE_256x128, 256, 128, 1, 1.0},
             {TILE_128, 128, 128, 2, 1.0},
             {TILE_128_DEEP, 128, 128, 1, 0.6}};
  const int64_t steps = (K + BK - 1) / BK;
  double best = 0.0;
  for (const auto &t : all) {
    const int64_t n = tiles(t.tm, t.tn), slots = (int64_t)t.to_cu * n_cu;
    // the weights' gradients share out their k, and fill the chip that way
    const double rounds = kind == PRODUCT_WEIGHTS && n < slots
                              ? std::max((double)n / slots, 8.0 / std::max<int64_t>(steps, 8))
                              : (double)((n + slots - 1) / slots);
    if (best == 0.0 || rounds * t.cost < best) {
      best = rounds * t.cost;
      p.tile = t.tile;
    }
  }
  const bool small = p.tile == TILE_128 || p.tile == TILE_128_DEEP;
  const int64_t tm = small ? 128 : 256, tn = p.tile == TILE_256 ? 256 : 128;
  if (kind == PRODUCT_WEIGHTS) {
    // as many parts as fill the chip, of eight stages at least
    const int64_t n = tiles(tm, tn);
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

// Workgroups that share a column block's k: as many as fill the chip, of two
// steps to a wave at least.  Up to 16 rows a workgroup has 16 waves, and the sums'
// own launch pays for itself only where few have work (8192 -> 2048, one row: 11.2
// and 3.6 us shared, 12.3 alone; 48 rows 15.1 and 4.0, 31.8 alone).
int few_splits(int64_t M, int64_t N, int64_t K, int n_cu) {
  const int64_t n = few_blocks(M, N), steps = (K + BK - 1) / BK;
  if (M <= 16 && n >= n_cu / 4) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(2 * n_cu / n, steps / 16));
}

hipError_t launch_few(const ProductArgs &a, bool gate, int type, int splits, hipStream_t stream) {
  if (type == T_BF16)
    return gate ? few_t<T_BF16, true>(a, 1, stream) : few_t<T_BF16, false>(a, splits, stream);
  return gate ? few_t<T_F16, true>(a, 1, stream) : few_t<T_F16, false>(a, splits, stream);
}

bool thin_fits(int64_t M, int64_t K, int64_t H, int64_t N, int n_cu) {
  return K <= 128 && N <= 128 && H <= THIN_HIDDEN && (M + THIN_ROWS - 1) / THIN_ROWS >= n_cu;
}

hipError_t launch_thin(const ProductArgs &a, bool grad, int type, hipStream_t stream) {
  if (type == T_BF16)
    return grad ? thin_t<T_BF16, true>(a, stream) : thin_t<T_BF16, false>(a, stream);
  return grad ? thin_t<T_F16, true>(a, stream) : thin_t<T_F16, false>(a, stream);
}

hipError_t launch_pack(PackArgs a, int type, hipStream_t stream) {
  a.first[0] = 0;
  for (int t = 0; t < a.count; ++t) {
    const int64_t units = a.rows[t] * ((a.width[t] + 7) / 8);
    a.first[t + 1] = a.first[t] + (int32_t)std::min<int64_t>((units + 255) / 256, 8192);
  }
  if (a.first[a.count] == 0) return hipSuccess;
  const dim3 grid((unsigned)a.first[a.count]);
  return type == T_BF16 ? launch(pack_tables<T_BF16>, grid, dim3(256), 0, stream, a)
                        : launch(pack_tables<T_F16>, grid, dim3(256), 0, stream, a);
}

hipError_t launch_sizes(SizeArgs a, hipStream_t stream) {
  // workgroups by the bytes of a table, one at least, SIZE_PARTS at most in all; those
  // left over only clear their parts
  int64_t bytes[SIZES], all = 0, last = 0;
  for (int t = 0; t < SIZES; ++t) all += bytes[t] = a.rows[t] * a.width[t] * 2;
  for (int t = 0; t < SIZES; ++t) {
    a.first[t] = (int32_t)last;
    if (bytes[t] == 0) continue;
    const int64_t share = (SIZE_PARTS - SIZES) * (bytes[t] / 1024 + 1) / (all / 1024 + SIZES) + 1;
    last += std::min<int64_t>(share, SIZE_PARTS);
  }
  a.first[SIZES] = (int32_t)last;
  return launch(gated_sizes<T_F16>, dim3(SIZE_PARTS), dim3(1024), 0, stream, a);
}

int64_t thin_sum_rows(int64_t M) { return (M + THIN_ROWS - 1) / THIN_ROWS * THIN_WAVES; }

hipError_t launch_join(const JoinArgs &a, int type, hipStream_t stream) {
  const dim3 grid((unsigned)((a.M * (a.ldp / 4) + 63) / 64));
  return type == T_BF16 ? launch(join_parts<T_BF16>, grid, dim3(1024), 0, stream, a)
                        : launch(join_parts<T_F16>, grid, dim3(1024), 0, stream, a);
}

}  // namespace gnn
