// Device pieces of the matrix products: element types, activations, group lookup, matrix instructions, epilogue.
#pragma once

#include "tt_gemm.h"

#ifdef __HIPCC__
namespace ttg {

typedef __bf16 bf16;
typedef _Float16 f16;
template <class T> struct Vec;  // four and sixteen bytes' worth of elements, at any element's address
template <> struct Vec<float> { typedef float v4 __attribute__((ext_vector_type(4), aligned(4))); typedef v4 v16b; };
template <> struct Vec<bf16> {
  typedef unsigned short v4 __attribute__((ext_vector_type(4), aligned(2)));
  typedef unsigned short v16b __attribute__((ext_vector_type(8), aligned(2)));
};
template <> struct Vec<f16> {
  typedef unsigned short v4 __attribute__((ext_vector_type(4), aligned(2)));
  typedef unsigned short v16b __attribute__((ext_vector_type(8), aligned(2)));
};
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) { return __uint_as_float((unsigned)__builtin_bit_cast(unsigned short, x) << 16); }
__device__ __forceinline__ float to_f32(f16 x) { return (float)x; }
template <class T> __device__ __forceinline__ T from_f32(float x) { return (T)x; }  // to nearest, ties to even

// Four elements at p (any element's address); with `valid` < 4 only the first ones are touched.
template <class T> __device__ __forceinline__ void load4(const T *p, int valid, float v[4]) {
  if (valid >= 4) {
    const typename Vec<T>::v4 r = *reinterpret_cast<const typename Vec<T>::v4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) v[i] = r[i];
      else v[i] = to_f32(__builtin_bit_cast(T, (unsigned short)r[i]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < valid ? to_f32(p[i]) : 0.f;
  }
}
template <class T, bool STREAM = false> __device__ __forceinline__ void store4(T *p, int valid, const float v[4]) {  // STREAM: past the caches
  if (valid >= 4) {
    typename Vec<T>::v4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) r[i] = v[i];
      else r[i] = __builtin_bit_cast(unsigned short, from_f32<T>(v[i]));
    }
    if constexpr (STREAM) __builtin_nontemporal_store(r, reinterpret_cast<typename Vec<T>::v4 *>(p));
    else *reinterpret_cast<typename Vec<T>::v4 *>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < valid) p[i] = from_f32<T>(v[i]);
  }
}

template <class T, int C, bool STREAM = false> __device__ __forceinline__ void load_n(const T *p, int valid, float v[C]) {
  if constexpr (C == 8 && sizeof(T) == 2) {
    if (valid >= 8) {
      typename Vec<T>::v16b r;
      if constexpr (STREAM) r = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T>::v16b *>(p));
      else r = *reinterpret_cast<const typename Vec<T>::v16b *>(p);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = to_f32(__builtin_bit_cast(T, (unsigned short)r[i]));
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < C; i += 4) load4(p + i, valid - i, v + i);
}
template <class T, int C, bool STREAM = false> __device__ __forceinline__ void store_n(T *p, int valid, const float v[C]) {
  if constexpr (C == 8 && sizeof(T) == 2) {
    if (valid >= 8) {
      typename Vec<T>::v16b r;
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i] = __builtin_bit_cast(unsigned short, from_f32<T>(v[i]));
      if constexpr (STREAM) __builtin_nontemporal_store(r, reinterpret_cast<typename Vec<T>::v16b *>(p));
      else *reinterpret_cast<typename Vec<T>::v16b *>(p) = r;
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < C; i += 4) store4<T, STREAM>(p + i, valid - i, v + i);
}

// ---- activations ---------------------------------------------------------------------------------
// With the slope taken from the stored pre-activation: NaN passes through both, relu has slope 0 at 0.
__device__ __forceinline__ float act_value(float z, int act) {
  switch (act) {
    case TT_ACT_RELU: return z <= 0.f ? 0.f : z;
    case TT_ACT_GELU: return 0.5f * z * erfcf(z * -0.70710678118654752f);
    case TT_ACT_SILU: return z / (1.f + expf(-z));
    case TT_ACT_SIGMOID: return 1.f / (1.f + expf(-z));
    default: return z;
  }
}
__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case TT_ACT_RELU: return z <= 0.f ? 0.f : (z != z ? z : 1.f);
    case TT_ACT_GELU: {
      const float e = expf(-0.5f * z * z);  // 0 for large z: the product below must not be inf * 0
      return 0.5f * erfcf(z * -0.70710678118654752f) + (e == 0.f ? 0.f : z * e * 0.39894228040143268f);
    }
    case TT_ACT_SILU: {
      const float s = 1.f / (1.f + expf(-z));  // z s (1 - s), written so that an infinite z gives its limit
      const float t = 1.f / (1.f + expf(z));
      return s + (s == 0.f || t == 0.f ? 0.f : z * s * t);
    }
    case TT_ACT_SIGMOID: {
      const float s = 1.f / (1.f + expf(-z)), t = 1.f / (1.f + expf(z));
      return s * t;
    }
    default: return 1.f;
  }
}
// The same for results of 16 bits.  exp and the reciprocal are the hardware's (good to a few units of 2^-24).  On the negative
// side Phi(z) = exp(-z^2 / 2) t Q(t) with t = 1 / (1 + 0.3625 |z|) and a polynomial Q of degree 6, fitted to the least largest relative error over
// -14 <= z <= 0: 7.7e-7, with its own rounding 1.2e-6, half a percent of fp16's half step, however far out.  The rounding of z^2 / 2 adds
// z^2 2^-25, 1e-5 at z = -13; below -13.2 exp is 0.
__device__ __forceinline__ float fast_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }
__device__ __forceinline__ float fast_phi(float z, float e) {  // e = exp(-z^2 / 2)
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.3625f, 1.f));
  const float q = fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.0480627407f, -0.179741932f), 0.17510341f), 0.0296827701f), 0.139256611f), 0.142936407f), 0.144700376f);
  const float p = e * t * q;
  return z < 0.f ? p : 1.f - p;
}
template <class O, int C> __device__ __forceinline__ void act_of(float v[C], int act) {
  constexpr bool fast = sizeof(O) == 2;
  switch (act) {
    case TT_ACT_RELU:
#pragma unroll
      for (int i = 0; i < C; ++i) v[i] = act_value(v[i], TT_ACT_RELU);
      break;
    case TT_ACT_GELU:
#pragma unroll
      for (int i = 0; i < C; ++i) v[i] = fast ? v[i] * fast_phi(v[i], __expf(-0.5f * v[i] * v[i])) : act_value(v[i], TT_ACT_GELU);
      break;
    case TT_ACT_SILU:
#pragma unroll
      for (int i = 0; i < C; ++i) v[i] = fast ? v[i] * fast_sigmoid(v[i]) : act_value(v[i], TT_ACT_SILU);
      break;
    case TT_ACT_SIGMOID:
#pragma unroll
      for (int i = 0; i < C; ++i) v[i] = fast ? fast_sigmoid(v[i]) : act_value(v[i], TT_ACT_SIGMOID);
      break;
    default: break;
  }
}
template <class O> __device__ __forceinline__ float slope_of(float z, int act) {
  if constexpr (sizeof(O) == 4) return act_slope(z, act);
  switch (act) {
    case TT_ACT_GELU: {
      const float e = __expf(-0.5f * z * z);  // 0 for large z: the product below must not be inf * 0
      return fast_phi(z, e) + (e == 0.f ? 0.f : z * e * 0.39894228040143268f);
    }
    case TT_ACT_SILU: {
      const float s = fast_sigmoid(z), t = fast_sigmoid(-z);
      return s + (s == 0.f || t == 0.f ? 0.f : z * s * t);
    }
    case TT_ACT_SIGMOID: return fast_sigmoid(z) * fast_sigmoid(-z);
    default: return act_slope(z, act);
  }
}
// A stored pre-activation keeps its sign: one that would round to zero in half precision becomes the smallest number, so
// that relu's slope there is that of the exact value.
template <class T> __device__ __forceinline__ float keep_sign(float z) { return z; }
template <> __device__ __forceinline__ float keep_sign<f16>(float z) {
  return z != 0.f && fabsf(z) < 0x1p-24f ? copysignf(0x1p-24f, z) : z;
}

// ---- groups --------------------------------------------------------------------------------------
// Offsets come from the device unseen by the host.  Every use goes by the running maximum of the offsets, clamped to [0,
// rows]: groups never overlap and never leave the buffers, whatever the offsets hold.
__device__ __forceinline__ int wave_max_scan(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int t = __shfl_up(v, o, 64);
    if (lane >= o && t > v) v = t;
  }
  return v;
}
__device__ __forceinline__ int clamp_row(int64_t o, int rows) { return o < 0 ? 0 : (o > rows ? rows : (int)o); }

// Tile t of the row tiles of TM rows, counted group after group: its group and rows [lo, lo + count).  Returns the tiles there
// are; for t at or behind that, `lo` and `hi` are the first and the end of the rows that groups cover.
template <int TM>
__device__ __forceinline__ int find_tile(const int64_t *off, int groups, int rows, int t, int &group, int &lo, int &hi) {
  const int lane = threadIdx.x & 63;
  const int first = clamp_row(off[0], rows);
  int start = first, tiles = 0;
  for (int g0 = 0; g0 < groups; g0 += 64) {
    const int g = g0 + lane;
    int e = wave_max_scan(g < groups ? clamp_row(off[g + 1], rows) : 0);
    if (e < start) e = start;
    int b = __shfl_up(e, 1, 64);
    if (lane == 0) b = start;
    const int mine = g < groups ? (e - b + TM - 1) / TM : 0;
    const int incl = tt_wave_incl_scan(mine);
    const unsigned long long has = __ballot(t < tiles + incl);
    if (has) {
      const int l = __ffsll(has) - 1;
      group = g0 + l;
      lo = __shfl(b, l, 64) + (t - tiles - __shfl(incl - mine, l, 64)) * TM;
      hi = __shfl(e, l, 64);
      if (hi > lo + TM) hi = lo + TM;
      return 0x7fffffff;
    }
    tiles += __shfl(incl, 63, 64);
    start = __shfl(e, 63, 64);
  }
  group = -1;
  lo = first;
  hi = start;
  return tiles;
}

// Sums over a group's rows are cut into pieces: ceil(rows / chunk) of them, of equal size in whole steps of `bk`, at least one. Slot t of all
// the groups' pieces: its group (-1: there is no such slot) and rows [lo, hi), the group's number of pieces, and the slot's number
// among those of groups that have several, which is where its sums go.  With `t` < 0: the group that is number `group` of those that have
// several (-1: there is none), and its first slot's number.
__device__ __forceinline__ void find_slot(const int64_t *off, int groups, int rows, int chunk, int bk, int t, int &group, int &lo, int &hi, int &pieces, int &number) {
  const int lane = threadIdx.x & 63, asked = group;
  int start = clamp_row(off[0], rows), slots = 0, several = 0, cut = 0;
  group = -1;
  for (int g0 = 0; g0 < groups; g0 += 64) {
    const int g = g0 + lane;
    int e = wave_max_scan(g < groups ? clamp_row(off[g + 1], rows) : 0);
    if (e < start) e = start;
    int b = __shfl_up(e, 1, 64);
    if (lane == 0) b = start;
    int mine = g < groups ? (int)(((long long)e - b + chunk - 1) / chunk) : 0;
    if (g < groups && mine < 1) mine = 1;
    const int incl = tt_wave_incl_scan(mine), incl2 = tt_wave_incl_scan(mine > 1 ? mine : 0);
    const unsigned long long many = __ballot(mine > 1);
    const int rank = cut + __popcll(many & ((1ull << lane) - 1));
    const unsigned long long has = __ballot(t >= 0 ? t < slots + incl : mine > 1 && rank == asked);
    cut += __popcll(many);
    if (has) {
      const int l = __ffsll(has) - 1, first = slots + __shfl(incl - mine, l, 64);
      group = g0 + l;
      pieces = __shfl(mine, l, 64);
      const int nth = t >= 0 ? t - first : 0, from = __shfl(b, l, 64), to = __shfl(e, l, 64);
      number = several + __shfl(incl2 - (mine > 1 ? mine : 0), l, 64) + nth;
      const int steps = (to - from + bk - 1) / bk, per = (steps + pieces - 1) / pieces;
      const long long x = from + (long long)nth * per * bk, y = x + (long long)per * bk;
      lo = x < to ? (int)x : to;
      hi = y < to ? (int)y : to;
      return;
    }
    slots += __shfl(incl, 63, 64);
    several += __shfl(incl2, 63, 64);
    start = __shfl(e, 63, 64);
  }
}

// ---- matrix instructions -------------------------------------------------------------------------
typedef float f32x4 __attribute__((ext_vector_type(4)));
// D[16 x 16] += A[16 x 32] B[32 x 16]: lane l holds A[l % 16][8 (l / 16) + i], B[8 (l / 16) + i][l % 16], D[4 (l / 16) + i][l % 16]
__device__ __forceinline__ f32x4 mma(bf16, u16x8 a, u16x8 b, f32x4 c) {
  typedef __bf16 v8 __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f16, u16x8 a, u16x8 b, f32x4 c) {
  typedef _Float16 v8 __attribute__((ext_vector_type(8)));
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
}
// Transposing LDS read of 16-bit elements: in every 16 lanes, lane j's address is that of elements 4 (j % 4) .. + 3 of row j / 4,
// and lane c receives column c of the four rows.
__device__ __forceinline__ u16x4 lds_read_tr(const unsigned short *p) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(p)));
}

// ---- which tile ------------------------------------------------------------------------------------
struct Place {
  int z, lo, hi, n0;  // member / group; rows [lo, hi) of out; first column
  int k_lo, k_hi;     // values of K of this workgroup (stored rows in RAGGED_K)
};
// Workgroups go round the eight dies by their number; each die gets neighbouring tiles, and within them eight row tiles
// take a column tile together, so that what they read of both operands is in the die's L2.
// Of a symmetric result only the tiles with mt <= nt, n (n + 1) / 2 of them.
__device__ __forceinline__ void tile_order(unsigned t, unsigned m_tiles, unsigned n_tiles, bool symmetric, unsigned &mt, unsigned &nt) {
  const unsigned total = symmetric ? n_tiles * (n_tiles + 1) / 2 : m_tiles * n_tiles, per = total / 8, left = total % 8, die = t % 8;
  t = die * per + (die < left ? die : left) + t / 8;
  if (symmetric) {
    nt = (unsigned)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (nt * (nt + 1) / 2 > t) --nt;
    while ((nt + 1) * (nt + 2) / 2 <= t) ++nt;
    mt = t - nt * (nt + 1) / 2;
    return;
  }
  const unsigned band = t / (8 * n_tiles), rows = m_tiles - 8 * band < 8 ? m_tiles - 8 * band : 8, in = t - band * 8 * n_tiles;
  mt = 8 * band + in % rows;
  nt = in / rows;
}

// RAGGED_M: clears the rows that no group covers; `idx` of `n` workgroups that found no tile, for columns n0 .. n0 + width
template <class O> __device__ __forceinline__ void clear_rest(const TTGemm &g, int above, int covered, int idx, int n, int n0, int width) {
  const float zero[4] = {0.f, 0.f, 0.f, 0.f};
  const long long rest = (long long)above + g.M - covered;
  const int end = g.N < n0 + width ? g.N : n0 + width;
  for (long long r = (long long)idx * 4 + (threadIdx.x >> 6); r < rest; r += (long long)n * 4)
    for (int c = n0 + 4 * (threadIdx.x & 63); c < end; c += 256)
      store4((O *)g.out + (r < above ? r : r - above + covered) * g.ldo + c, end - c < 4 ? end - c : 4, zero);
}

// out[m][n .. n + C - 1] from C = 4 or 8 sums, of which `valid` columns exist.  `bias` and `res`: these columns' values where the caller
// has them already (null: they are read here).
template <class T, class O, int C, bool STREAM = false>
__device__ __forceinline__ void finish(const TTGemm &g, int z, int m, int n, int valid, float v[C], const float *bias = nullptr, const float *res = nullptr) {
  float t[C];
#pragma unroll
  for (int i = 0; i < C; ++i) v[i] *= g.alpha;
  if (bias) {
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] += bias[i];
  } else if (g.bias) {
    load_n<T, C>((const T *)g.bias + z * g.bias_step + n, valid, t);
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] += t[i];
  }
  if (g.pre) {
#pragma unroll
    for (int i = 0; i < C; ++i) t[i] = keep_sign<O>(v[i]);
    store_n<O, C, STREAM>((O *)g.pre + z * g.p_step + (long long)m * g.ldp + n, valid, t);
  }
  act_of<O, C>(v, g.act);
  if (res) {
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] = fmaf(g.beta, res[i], v[i]);
  } else if (g.res) {
    load_n<T, C>((const T *)g.res + z * g.r_step + (long long)m * g.ldr + n, valid, t);
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] = fmaf(g.beta, t[i], v[i]);
  }
  store_n<O, C, STREAM>((O *)g.out + z * g.o_step + (long long)m * g.ldo + n, valid, v);
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const long long b = __builtin_bit_cast(long long, v);
    const int lo = __shfl((int)b, (threadIdx.x & 63) ^ o, 64), hi = __shfl((int)(b >> 32), (threadIdx.x & 63) ^ o, 64);
    v += __builtin_bit_cast(double, ((long long)hi << 32) | (unsigned)lo);
  }
  return v;
}
// relu of an fp32 product (K-contiguous operands): v becomes alpha v + bias, and where rounding may have decided its sign, all 64 lanes form
// it again in 64 bits.  A sum of K products has about K roundings, each of at most 2^-24 of a partial sum, which is at most |a| |b| (2-norms of
// the two rows; squares_a and squares_b are theirs): as errors of either sign they come to sqrt(K) 2^-24 |a| |b|.  Below four times
// that v is formed again; measured errors of random operands are a thousandth of it.  (Operands beyond 2^+-60, whose squares leave the range,
// have all results formed again, or keep the sign that they have.)  At K = 128 one result in 40000, at 4096 one in 1200.
// 16384 x 128 -> 512 takes 26.9 us with relu, 24.8 without; 4096 x 4096 -> 1024 214 and 188.  Data of few values, whose sums cancel exactly, have
// more of them at a microsecond each: 0 and 1 by -1 and 1, 5 % of the first product's results, 222 us.  Four at a time by 16 lanes each take 107 there, but the
// products above 28.6 and 251.
// All lanes of the wavefront call it, with one z; `valid` <= 0: a lane without results.
template <int C>
__device__ __forceinline__ void settle_signs(const TTGemm &g, int z, int m, int n, int valid, float v[C], const float bias[C], float squares_a,
                                             const float squares_b[C]) {
  const int lane = threadIdx.x & 63;
  const float share = 16.f * 0x1p-48f * (float)g.K * squares_a;  // compared as squares
  unsigned near = 0;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    v[i] = g.alpha * v[i] + bias[i];
    near |= i < valid && v[i] * v[i] < share * squares_b[i] ? 1u << i : 0u;
  }
  for (unsigned long long lanes = __ballot(near != 0); lanes; lanes = __ballot(near != 0)) {
    const int l = __ffsll(lanes) - 1, which = __ffs(__shfl((int)near, l, 64)) - 1;
    const int row = __shfl(m, l, 64), col = __shfl(n, l, 64) + which;
    const float *a = (const float *)g.a + (g.mode == TT_GEMM_BATCH ? z * g.a_step : 0) + (long long)row * g.lda;
    const float *b = (const float *)g.b + z * g.b_step + (long long)col * g.ldb;
    double s = 0;
    for (int k = 4 * lane; k < g.K; k += 256) {
      float x[4], y[4];
      load4(a + k, g.K - k, x);
      load4(b + k, g.K - k, y);
#pragma unroll
      for (int i = 0; i < 4; ++i) s += (double)x[i] * y[i];
    }
    s = g.alpha * wave_sum64(s) + (g.bias ? ((const float *)g.bias)[z * g.bias_step + col] : 0.f);
    const float r = s != 0 && fabs(s) < 0x1p-149 ? (s < 0 ? -0x1p-149f : 0x1p-149f) : (float)s;
    if (lane == l) {
      near &= near - 1;
#pragma unroll
      for (int i = 0; i < C; ++i) v[i] = i == which ? r : v[i];
    }
  }
}

// The results of a wavefront, 16 FX x 16 FY of out from row m0 and column n0, rows below `end`.  The instruction leaves a lane
// four columns of a row, 8 bytes of a 16-bit row at a time; through 16 XB rows of LDS (`lds`: finish_floats of the wavefront's own) a lane
// gets eight, and what is read and written is whole lines of 128 bytes.  The loop over the rows is not unrolled: with all activations in it
// 16 times, the code is longer than the instruction cache.
// A product's description with its sums themselves as the result: a piece of a cut product.
__device__ __forceinline__ TTGemm as_piece(const TTGemm &g, float *piece) {
  TTGemm p = g;
  p.out = piece;
  p.ldo = g.N;
  p.o_step = 0;
  p.alpha = 1.f;
  p.bias = p.res = nullptr;
  p.pre = nullptr;
  p.act = TT_ACT_NONE;
  return p;
}
template <int FY, int XB> constexpr int finish_floats() { return 16 * XB * (16 * FY + 4); }
// STREAM (16-bit tiles of 256): results are written and the residual is read past the caches, which keep the operands instead (16384 x 4096
// x 4096 bf16 without residual 543 -> 423 us), and the residual is read four rows ahead: one at a time, its latency had each tile's end
// take as long as a quarter of its product.
// `squares_a` and `squares_b` (LDS, null: nothing is settled): of the wavefront's rows of A and of B, for settle_signs.
template <class T, class O, int FX, int FY, int XB, bool STREAM>
__device__ __forceinline__ void finish_tile(const TTGemm &g, int z, int m0, int end, int n0, const f32x4 (&acc)[FX][FY], float *lds, bool mirror = false,
                                            const float *squares_a = nullptr, const float *squares_b = nullptr) {
  constexpr int LD = 16 * FY + 4, PER = 2 * FY, ROWS = 64 / PER;  // lanes of a row, rows at a time
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15, c = 8 * (lane % PER), r = lane / PER;
  const int valid = g.N - n0 - c;
  float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (g.bias && valid > 0) load_n<T, 8>((const T *)g.bias + z * g.bias_step + n0 + c, valid, bias);
  float squares[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (squares_b) {
#pragma unroll
    for (int i = 0; i < 8; ++i) squares[i] = squares_b[c + i];
  }
  constexpr int AHEAD = 4;
  typename Vec<T>::v16b ahead[AHEAD];
  auto residual = [&](int row) {
    typename Vec<T>::v16b v = {};
    if (row < 16 * FX && m0 + row < end && valid >= 8)
      v = __builtin_nontemporal_load(reinterpret_cast<const typename Vec<T>::v16b *>((const T *)g.res + z * g.r_step + (long long)(m0 + row) * g.ldr + n0 + c));
    return v;
  };
  if constexpr (STREAM) {
    if (g.res) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) ahead[i] = residual(r + i * ROWS);
    }
  }
#pragma unroll
  for (int x0 = 0; x0 < FX; x0 += XB) {
#pragma unroll
    for (int x = 0; x < XB; ++x)
#pragma unroll
      for (int y = 0; y < FY; ++y) *reinterpret_cast<f32x4 *>(lds + (16 * x + j) * LD + 16 * y + 4 * q) = acc[x0 + x][y];
    tt_wave_lds_order();
    auto sums = [&](int row, float v[8]) {
      const f32x4 a = *reinterpret_cast<const f32x4 *>(lds + row * LD + c), b = *reinterpret_cast<const f32x4 *>(lds + row * LD + c + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[4 + i] = b[i];
      }
    };
    if (STREAM && g.res) {
      if constexpr (STREAM) {
#pragma unroll 1
        for (int row = r; row < 16 * XB; row += ROWS) {
          const int m = m0 + 16 * x0 + row;
          float v[8], res[8];
          sums(row, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) res[i] = to_f32(__builtin_bit_cast(T, (unsigned short)ahead[0][i]));
#pragma unroll
          for (int i = 0; i + 1 < AHEAD; ++i) ahead[i] = ahead[i + 1];
          ahead[AHEAD - 1] = residual(16 * x0 + row + AHEAD * ROWS);
          if (m < end && valid >= 8) finish<T, O, 8, true>(g, z, m, n0 + c, 8, v, bias, res);
          else if (m < end && valid > 0) finish<T, O, 8, true>(g, z, m, n0 + c, valid, v, bias);
        }
      }
    } else {
#pragma unroll 1
      for (int row = r; row < 16 * XB; row += ROWS) {
        const int m = m0 + 16 * x0 + row;
        float v[8];
        sums(row, v);
        if constexpr (std::is_same<T, float>::value && std::is_same<O, float>::value) {
          if (squares_a) {
            const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};  // (bias is in v)
            settle_signs<8>(g, z, m, n0 + c, m < end ? valid : 0, v, bias, squares_a[16 * x0 + row], squares);
            if (m < end && valid > 0) finish<T, O, 8, STREAM>(g, z, m, n0 + c, valid, v, none);
            continue;
          }
        }
        if (m < end && valid > 0) finish<T, O, 8, STREAM>(g, z, m, n0 + c, valid, v, bias);
      }
    }
    if (mirror) {  // the same results as rows n of columns m (only products without a bias)
#pragma unroll 1
      for (int e = lane; e < 16 * FY * 2 * XB; e += 64) {
        const int row = e / (2 * XB), col = 8 * (e % (2 * XB)), n = n0 + row, m = m0 + 16 * x0 + col;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = lds[(col + i) * LD + row];
        if (n < g.N && m < end) finish<T, O, 8>(g, z, n, m, end - m, v);
      }
    }
    tt_wave_lds_order();
  }
}

}  // namespace ttg
#endif
