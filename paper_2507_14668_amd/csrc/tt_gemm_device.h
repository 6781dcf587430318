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
template <class T> __device__ __forceinline__ void store4(T *p, int valid, const float v[4]) {
  if (valid >= 4) {
    typename Vec<T>::v4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) r[i] = v[i];
      else r[i] = __builtin_bit_cast(unsigned short, from_f32<T>(v[i]));
    }
    *reinterpret_cast<typename Vec<T>::v4 *>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < valid) p[i] = from_f32<T>(v[i]);
  }
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

// Rows [lo, hi) of group z (the whole wavefront calls it).
__device__ __forceinline__ void group_rows(const int64_t *off, int z, int rows, int &lo, int &hi) {
  const int lane = threadIdx.x & 63;
  int m = 0;
  for (int g = lane; g <= z; g += 64) {
    const int v = clamp_row(off[g], rows);
    if (v > m) m = v;
  }
  lo = __shfl(wave_max_scan(m), 63, 64);
  const int e = clamp_row(off[z + 1], rows);
  hi = e > lo ? e : lo;
}

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

}  // namespace ttg
#endif
