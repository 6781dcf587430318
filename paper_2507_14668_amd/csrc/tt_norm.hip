// Layer norm of rows and its gradients.
#include "tt_gemm_device.h"

namespace {
using namespace ttg;

struct Norm {  // of a call, by value to the kernels
  const void *x, *weight, *bias, *grad;
  void *out;     // y, or dx
  float *stats;  // [rows][2]
  float *partial;
  long long rows, ld_x, ld_out, ld_grad;
  int n;
  float eps;
};

// Sixteen bytes of a row: C elements, of which `valid` exist (zeros stand in for the others).
template <class T> struct Piece {
  static constexpr int C = 16 / sizeof(T);
  typename Vec<T>::v16b v;
  __device__ __forceinline__ void load(const T *p, int valid) {
    if (valid >= C) {
      v = *reinterpret_cast<const typename Vec<T>::v16b *>(p);
    } else {
#pragma unroll
      for (int i = 0; i < C; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = i < valid ? p[i] : 0.f;
        else v[i] = i < valid ? __builtin_bit_cast(unsigned short, p[i]) : (unsigned short)0;
      }
    }
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return v[i];
    else return to_f32(__builtin_bit_cast(T, (unsigned short)v[i]));
  }
  __device__ __forceinline__ void ones() {
#pragma unroll
    for (int i = 0; i < C; ++i) {
      if constexpr (sizeof(T) == 4) v[i] = 1.f;
      else v[i] = std::is_same<T, f16>::value ? 0x3c00 : 0x3f80;
    }
  }
  __device__ __forceinline__ void zeros() {
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] = 0;
  }
};

// The sums of a and b over the LANES threads of a row, the same bits in each.  `room`: float[2][8][2] of LDS, whose halves
// take turns, so that one barrier a sum is enough.
template <int LANES> __device__ __forceinline__ void row_sum(float &a, float &b, float *room, int &turn) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = (LANES < 64 ? LANES : 64) / 2; o > 0; o >>= 1) {
    a += __shfl(a, lane ^ o, 64);
    b += __shfl(b, lane ^ o, 64);
  }
  if constexpr (LANES > 64) {
    float *half = room + turn * 16;
    turn ^= 1;
    if (lane == 0) {
      half[2 * (threadIdx.x >> 6)] = a;
      half[2 * (threadIdx.x >> 6) + 1] = b;
    }
    __syncthreads();
    const int first = (int)(threadIdx.x / LANES) * (LANES / 64);
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) {
      a += half[2 * (first + w)];
      b += half[2 * (first + w) + 1];
    }
  }
}
// The largest of v over them; NaN does not count.
template <int LANES> __device__ __forceinline__ float row_largest(float v, float *room, int &turn) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = (LANES < 64 ? LANES : 64) / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl(v, lane ^ o, 64));
  if constexpr (LANES > 64) {
    float *half = room + turn * 16;
    turn ^= 1;
    if (lane == 0) half[threadIdx.x >> 6] = v;
    __syncthreads();
    const int first = (int)(threadIdx.x / LANES) * (LANES / 64);
    v = half[first];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) v = fmaxf(v, half[first + w]);
  }
  return v;
}
template <int LANES> constexpr int threads_of() { return LANES > 256 ? LANES : 256; }

// The mean of a row's sum is off by the rounding of that sum, in the size of its elements, which may be far above their spread: it is mended by the mean `off` of
// what it leaves of them, whose rounding is in the size of the spread, and the mean of the squares of that by off's.  A NaN stays one.
__device__ __forceinline__ float variance_of(float squares, float off) {
  const float v = fmaf(-off, off, squares);
  return v < 0.f ? 0.f : v;
}
// Whether a row's sums have left fp32's range, or its squares are so small that they lose bits that eps does not cover: the row is then taken again, times the power of two
// that makes its largest number (or the root of eps) about one.
__device__ __forceinline__ bool out_of_range(float variance, float eps) { return !(variance < 0x1p100f) || variance + eps < 0x1p-100f; }
__device__ __forceinline__ float scale_for(float largest, float eps) {
  const int e = (int)(__float_as_uint(fmaxf(largest, sqrtf(eps))) >> 23);  // of 1 127
  return __uint_as_float((unsigned)(254 - (e < 1 ? 1 : e > 253 ? 253 : e)) << 23);
}
// Large numbers that lie close together: the row as it is, whose deviations may be what eps is.
__device__ __forceinline__ void rescale(float &mean, float &rstd, float &scale, float variance, float eps) {
  if (!(scale < 1.f)) return;
  const float whole = variance / scale / scale + eps;
  if (!(whole < 0x1p100f)) return;
  mean /= scale;
  rstd = 1.f / sqrtf(whole);
  scale = 1.f;
}
// Of a row with deviations near the largest numbers, (x - mean) rstd with both halved twice: the difference may be twice as large as those.
struct Center {
  float q, mean, rstd;
  __device__ __forceinline__ Center(float m, float r) : q(r < 0x1p-100f ? 0.25f : 1.f), mean(q * m), rstd(r / q) {}
  __device__ __forceinline__ float of(float x) const { return fmaf(x, q, -mean) * rstd; }
};
// A row stays in the registers of LANES threads, NV pieces each: it is read once, and the variance is the mean of the squares of
// what is left after the mean.  weight and bias stay in registers over a workgroup's rows.  Bound by memory: 106496 rows of 128 in fp32 18.3 us
// (6.0 TB/s), 16384 of 4096 in bf16 52 (5.2), a large copy 5.1.
template <class T, int LANES, int NV> __global__ void __launch_bounds__(threads_of<LANES>()) k_norm_forward(Norm p) {
  constexpr int C = Piece<T>::C, GROUPS = threads_of<LANES>() / LANES;
  __shared__ float room[32];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  int turn = 0;
  Piece<T> w[NV], b[NV], x[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * LANES + lane) * C;
    if (p.weight) w[i].load((const T *)p.weight + c, p.n - c);
    else w[i].ones();
    if (p.bias) b[i].load((const T *)p.bias + c, p.n - c);
    else b[i].zeros();
  }
  const float inv = 1.f / (float)p.n;
  for (long long r0 = (long long)blockIdx.x * GROUPS; r0 < p.rows; r0 += (long long)gridDim.x * GROUPS) {
    const bool live = r0 + group < p.rows;
    const long long r = live ? r0 + group : p.rows - 1;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LANES + lane) * C;
      x[i].load((const T *)p.x + r * p.ld_x + c, p.n - c);
    }
    float scale = 1.f, mean, rstd, variance;  // of the row times scale
    for (int pass = 0;; ++pass) {
      float sum = 0.f, squares = 0.f, none = 0.f, off = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < C; ++e) sum = fmaf(x[i].at(e), scale, sum);
      row_sum<LANES>(sum, none, room, turn);
      const float about = sum * inv;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < C; ++e) {
          const float d = (i * LANES + lane) * C + e < p.n ? fmaf(x[i].at(e), scale, -about) : 0.f;
          squares = fmaf(d, d, squares);
          off += d;
        }
      row_sum<LANES>(squares, off, room, turn);
      off *= inv;
      variance = variance_of(squares * inv, off);
      mean = about + off;
      rstd = 1.f / sqrtf(variance + p.eps * scale * scale);
      const bool again = pass == 0 && out_of_range(variance, p.eps);
      if (!__ballot(again)) break;  // (the wavefront's other rows do the same once more)
      float largest = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < C; ++e) largest = fmaxf(largest, fabsf(x[i].at(e)));
      largest = row_largest<LANES>(largest, room, turn);
      if (again) scale = scale_for(largest, p.eps);
    }
    rescale(mean, rstd, scale, variance, p.eps);
    if (!live) continue;
    if (p.stats && lane == 0) {
      p.stats[2 * r] = mean / scale;
      p.stats[2 * r + 1] = rstd * scale;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LANES + lane) * C;
      float y[C];
#pragma unroll
      for (int e = 0; e < C; ++e) y[e] = fmaf(fmaf(x[i].at(e), scale, -mean) * rstd, w[i].at(e), b[i].at(e));
      if (c < p.n) store_n<T, C>((T *)p.out + r * p.ld_out + c, p.n - c, y);
    }
  }
}

// dx in one pass, and beside it the workgroup's share of dweight and dbias, summed over its rows in registers and written to
// partial[workgroup][2][n].  512 workgroups: 27.9 us (5.9 TB/s) and 90 us (4.5) for the rows above, and 4 for the joining of their shares.
template <class T, int LANES, int NV> __global__ void __launch_bounds__(threads_of<LANES>()) k_norm_backward(Norm p) {
  constexpr int C = Piece<T>::C, THREADS = threads_of<LANES>(), GROUPS = THREADS / LANES;
  __shared__ float room[32];
  __shared__ __align__(16) float shares[GROUPS > 1 ? THREADS * C : 4];
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  int turn = 0;
  Piece<T> w[NV], x[NV], g[NV];
  float dw[NV][C] = {}, db[NV][C] = {};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * LANES + lane) * C;
    if (p.weight) w[i].load((const T *)p.weight + c, p.n - c);
    else w[i].ones();
  }
  const float inv = 1.f / (float)p.n;
  for (long long r0 = (long long)blockIdx.x * GROUPS; r0 < p.rows; r0 += (long long)gridDim.x * GROUPS) {
    const bool live = r0 + group < p.rows;
    const long long r = live ? r0 + group : p.rows - 1;
    const float rstd = p.stats[2 * r + 1];
    const Center center(p.stats[2 * r], rstd);
    float s = 0.f, sx = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LANES + lane) * C;
      x[i].load((const T *)p.x + r * p.ld_x + c, p.n - c);
      g[i].load((const T *)p.grad + r * p.ld_grad + c, p.n - c);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < C; ++e) {
        const bool in = live && (i * LANES + lane) * C + e < p.n;
        const float ge = g[i].at(e), xh = center.of(x[i].at(e)), h = ge * w[i].at(e);
        s += in ? h : 0.f;
        sx += in ? h * xh : 0.f;
        dw[i][e] += in ? ge * xh : 0.f;
        db[i][e] += in ? ge : 0.f;
      }
    if (!p.out) continue;
    row_sum<LANES>(s, sx, room, turn);
    s *= inv;
    sx *= inv;
    if (!live) continue;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * LANES + lane) * C;
      float d[C];
#pragma unroll
      for (int e = 0; e < C; ++e) d[e] = rstd * (g[i].at(e) * w[i].at(e) - s - center.of(x[i].at(e)) * sx);
      if (c < p.n) store_n<T, C>((T *)p.out + r * p.ld_out + c, p.n - c, d);
    }
  }
  if (!p.partial) return;
  float *to = p.partial + (long long)blockIdx.x * 2 * p.n;
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const float(&mine)[C] = which ? db[i] : dw[i];
      if constexpr (GROUPS == 1) {
        const int c = (i * LANES + lane) * C;
        if (c < p.n) store_n<float, C>(to + (long long)which * p.n + c, p.n - c, mine);
      } else {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < C; ++e) shares[threadIdx.x * C + e] = mine[e];
        __syncthreads();
        for (int k = threadIdx.x; k < LANES * C; k += THREADS) {  // the groups in order
          const int c = i * LANES * C + k;
          float sum = 0.f;
#pragma unroll
          for (int o = 0; o < GROUPS; ++o) sum += shares[o * LANES * C + k];
          if (c < p.n) to[(long long)which * p.n + c] = sum;
        }
      }
    }
}

// Rows that do not fit the registers: read again for each step.
constexpr int WIDE = 512;
template <class T> __global__ void __launch_bounds__(WIDE) k_norm_forward_wide(Norm p) {
  constexpr int C = Piece<T>::C;
  __shared__ float room[32];
  int turn = 0;
  const float inv = 1.f / (float)p.n;
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T *x = (const T *)p.x + r * p.ld_x;
    float scale = 1.f, mean, rstd, variance;  // as above
    for (int pass = 0;; ++pass) {
      float sum = 0.f, squares = 0.f, none = 0.f, off = 0.f, largest = 0.f;
      for (int c = threadIdx.x * C; c < p.n; c += WIDE * C) {
        float v[C];
        load_n<T, C>(x + c, p.n - c, v);
#pragma unroll
        for (int e = 0; e < C; ++e) {
          sum = fmaf(v[e], scale, sum);
          largest = fmaxf(largest, fabsf(v[e]));
        }
      }
      row_sum<WIDE>(sum, none, room, turn);
      const float about = sum * inv;
      for (int c = threadIdx.x * C; c < p.n; c += WIDE * C) {
        float v[C];
        load_n<T, C>(x + c, p.n - c, v);
#pragma unroll
        for (int e = 0; e < C; ++e) {
          const float d = c + e < p.n ? fmaf(v[e], scale, -about) : 0.f;
          squares = fmaf(d, d, squares);
          off += d;
        }
      }
      row_sum<WIDE>(squares, off, room, turn);
      off *= inv;
      variance = variance_of(squares * inv, off);
      mean = about + off;
      rstd = 1.f / sqrtf(variance + p.eps * scale * scale);
      if (pass != 0 || !out_of_range(variance, p.eps)) break;
      scale = scale_for(row_largest<WIDE>(largest, room, turn), p.eps);
    }
    rescale(mean, rstd, scale, variance, p.eps);
    if (p.stats && threadIdx.x == 0) {
      p.stats[2 * r] = mean / scale;
      p.stats[2 * r + 1] = rstd * scale;
    }
    for (int c = threadIdx.x * C; c < p.n; c += WIDE * C) {
      float v[C], w[C], b[C];
      load_n<T, C>(x + c, p.n - c, v);
      if (p.weight) load_n<T, C>((const T *)p.weight + c, p.n - c, w);
      if (p.bias) load_n<T, C>((const T *)p.bias + c, p.n - c, b);
#pragma unroll
      for (int e = 0; e < C; ++e) v[e] = fmaf(fmaf(v[e], scale, -mean) * rstd, p.weight ? w[e] : 1.f, p.bias ? b[e] : 0.f);
      store_n<T, C>((T *)p.out + r * p.ld_out + c, p.n - c, v);
    }
  }
}
template <class T> __global__ void __launch_bounds__(WIDE) k_norm_backward_wide(Norm p) {
  constexpr int C = Piece<T>::C;
  __shared__ float room[32];
  int turn = 0;
  const float inv = 1.f / (float)p.n;
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T *x = (const T *)p.x + r * p.ld_x, *g = (const T *)p.grad + r * p.ld_grad;
    const float rstd = p.stats[2 * r + 1];
    const Center center(p.stats[2 * r], rstd);
    float s = 0.f, sx = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      for (int c = threadIdx.x * C; c < p.n; c += WIDE * C) {
        float v[C], h[C], w[C];
        load_n<T, C>(x + c, p.n - c, v);
        load_n<T, C>(g + c, p.n - c, h);
        if (p.weight) load_n<T, C>((const T *)p.weight + c, p.n - c, w);
#pragma unroll
        for (int e = 0; e < C; ++e) {
          v[e] = center.of(v[e]);
          h[e] *= p.weight ? w[e] : 1.f;
          if (pass == 0) {
            s += c + e < p.n ? h[e] : 0.f;
            sx += c + e < p.n ? h[e] * v[e] : 0.f;
          } else {
            v[e] = rstd * (h[e] - s - v[e] * sx);
          }
        }
        if (pass) store_n<T, C>((T *)p.out + r * p.ld_out + c, p.n - c, v);
      }
      if (pass == 0) {
        row_sum<WIDE>(s, sx, room, turn);
        s *= inv;
        sx *= inv;
      }
    }
  }
}
// partial[blockIdx.y][2][n] of rows blockIdx.y, + gridDim.y, ...; a thread has C columns
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_norm_columns_wide(Norm p) {
  constexpr int C = Piece<T>::C;
  const int c = (int)(blockIdx.x * TT_BLOCK + threadIdx.x) * C;
  if (c >= p.n) return;
  float dw[C] = {}, db[C] = {};
  for (long long r = blockIdx.y; r < p.rows; r += gridDim.y) {
    const Center center(p.stats[2 * r], p.stats[2 * r + 1]);
    float v[C], g[C];
    load_n<T, C>((const T *)p.x + r * p.ld_x + c, p.n - c, v);
    load_n<T, C>((const T *)p.grad + r * p.ld_grad + c, p.n - c, g);
#pragma unroll
    for (int e = 0; e < C; ++e) {
      dw[e] += g[e] * center.of(v[e]);
      db[e] += g[e];
    }
  }
  float *to = p.partial + (long long)blockIdx.y * 2 * p.n + c;
  store_n<float, C>(to, p.n - c, dw);
  store_n<float, C>(to + p.n, p.n - c, db);
}

// dweight and dbias: the shares in order of their numbers, in 16 runs that are then added in order.
constexpr int RUNS = 16, COLUMNS = 32;
template <class T> __global__ void __launch_bounds__(RUNS *COLUMNS) k_norm_join(const float *__restrict__ partial, int shares, int n, T *dw, T *db) {
  __shared__ float room[RUNS][COLUMNS];
  const int col = threadIdx.x % COLUMNS, run = threadIdx.x / COLUMNS;
  const long long c = (long long)blockIdx.x * COLUMNS + col;  // of 2 n
  const int per = (shares + RUNS - 1) / RUNS, first = run * per, end = first + per < shares ? first + per : shares;
  float s = 0.f;
  if (c < 2LL * n) {
#pragma unroll 8
    for (int i = first; i < end; ++i) s += partial[(long long)i * 2 * n + c];
  }
  room[run][col] = s;
  __syncthreads();
  if (run != 0 || c >= 2LL * n) return;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < RUNS; ++i) s += room[i][col];
  if (c < n) {
    if (dw) dw[c] = from_f32<T>(s);
  } else if (db) {
    db[c - n] = from_f32<T>(s);
  }
}

// ---- host ------------------------------------------------------------------------------------------
// Threads of a row: 16 up to two pieces each, 64 up to four, then 256 and 512.
struct Shape {
  int lanes, nv;  // lanes 0: the row does not fit
};
Shape shape_of(int dtype, int n) {
  const int pieces = tt_ceil_div(n, dtype == TT_F32 ? 4 : 8);
  Shape h = {0, 0};
  if (pieces <= 32) h = {16, pieces <= 16 ? 1 : 2};
  else if (pieces <= 256) h = {64, pieces <= 64 ? 1 : pieces <= 128 ? 2 : 4};
  else if (pieces <= 1024) h = {256, pieces <= 512 ? 2 : 4};
  else if (pieces <= 2048) h = {512, 4};
  return h;
}
int groups_of(const Shape &h) { return h.lanes ? (h.lanes > 256 ? 1 : 256 / h.lanes) : 1; }
// Workgroups whose shares of dweight and dbias are added; fixed by the sizes, so that the same sums come of it on any device.
int shares_of(const tt_norm *op) {
  const Shape h = shape_of(op->dtype, op->dim);
  const long long blocks = tt_ceil_div(op->rows, groups_of(h)), most = h.lanes ? 512 : 64;
  return (int)(blocks < most ? blocks : most);
}

tt_status check(const tt_norm *op) {
  if (!op || op->dtype < TT_F32 || op->dtype > TT_F16 || op->rows < 0 || !(op->eps >= 0.f) || op->eps == INFINITY) return TT_ERR_INVALID_ARG;
  if (op->dim < 1 || op->dim > TT_NORM_MAX_DIM || op->rows >= 2147483647LL) return TT_ERR_SHAPE;
  const int64_t ld[4] = {op->ld_x, op->ld_out, op->ld_grad, op->ld_dx};
  for (int i = 0; i < 4; ++i)
    if (ld[i] != 0 && (ld[i] < op->dim || ld[i] > ((int64_t)1 << 40))) return TT_ERR_SHAPE;
  return TT_OK;
}
bool aligned(const void *p, size_t size) { return ((uintptr_t)p & (size - 1)) == 0; }
long long step(int64_t ld, int dim) { return ld ? ld : dim; }

template <class T, int LANES, int NV> void launch_fit(const Norm &p, bool backward, int shares, hipStream_t s) {
  constexpr int THREADS = threads_of<LANES>(), GROUPS = THREADS / LANES;
  long long blocks = (p.rows + GROUPS - 1) / GROUPS;
  if (backward) {
    hipLaunchKernelGGL((k_norm_backward<T, LANES, NV>), dim3((unsigned)shares), dim3(THREADS), 0, s, p);
  } else {
    if (blocks > 2048) blocks = 2048;
    hipLaunchKernelGGL((k_norm_forward<T, LANES, NV>), dim3((unsigned)blocks), dim3(THREADS), 0, s, p);
  }
}
template <class T> tt_status launch(const Norm &p, const Shape &h, bool backward, int shares, hipStream_t s) {
  if (h.lanes == 16) h.nv == 1 ? launch_fit<T, 16, 1>(p, backward, shares, s) : launch_fit<T, 16, 2>(p, backward, shares, s);
  else if (h.lanes == 64) h.nv == 1 ? launch_fit<T, 64, 1>(p, backward, shares, s) : h.nv == 2 ? launch_fit<T, 64, 2>(p, backward, shares, s) : launch_fit<T, 64, 4>(p, backward, shares, s);
  else if (h.lanes == 256) h.nv == 2 ? launch_fit<T, 256, 2>(p, backward, shares, s) : launch_fit<T, 256, 4>(p, backward, shares, s);
  else if (h.lanes == 512) launch_fit<T, 512, 4>(p, backward, shares, s);
  else {
    const long long blocks = p.rows < 1024 ? p.rows : 1024;
    if (!backward) {
      hipLaunchKernelGGL(k_norm_forward_wide<T>, dim3((unsigned)blocks), dim3(WIDE), 0, s, p);
    } else {
      if (p.out) hipLaunchKernelGGL(k_norm_backward_wide<T>, dim3((unsigned)blocks), dim3(WIDE), 0, s, p);
      if (p.partial)
        hipLaunchKernelGGL(k_norm_columns_wide<T>, dim3((unsigned)tt_ceil_div(p.n, TT_BLOCK * Piece<T>::C), (unsigned)shares), dim3(TT_BLOCK), 0, s, p);
    }
  }
  return tt_launch_status();
}
template <class T> tt_status join(const float *partial, int shares, int n, void *dw, void *db, hipStream_t s) {
  hipLaunchKernelGGL(k_norm_join<T>, dim3((unsigned)tt_ceil_div(2LL * n, COLUMNS)), dim3(RUNS * COLUMNS), 0, s, partial, shares, n, (T *)dw, (T *)db);
  return tt_launch_status();
}

}  // namespace

extern "C" size_t tt_layer_norm_workspace_bytes(const tt_norm *op) {
  if (check(op) != TT_OK) return 0;
  return ((size_t)shares_of(op) * 2 * op->dim * 4 + 255) & ~(size_t)255;
}

extern "C" tt_status tt_layer_norm_forward(const tt_norm *op, const void *x, const void *weight, const void *bias, void *out, float *stats, void *stream) {
  const tt_status st = check(op);
  if (st != TT_OK) return st;
  if (op->rows == 0) return TT_OK;
  const size_t es = op->dtype == TT_F32 ? 4 : 2;
  if (!x || !out || !aligned(x, es) || !aligned(weight, es) || !aligned(bias, es) || !aligned(out, es) || !aligned(stats, 4)) return TT_ERR_INVALID_ARG;
  if (out == x || out == weight || out == bias || out == (void *)stats || (stats && (stats == x || stats == weight || stats == bias))) return TT_ERR_INVALID_ARG;
  Norm p = {x, weight, bias, nullptr, out, stats, nullptr, op->rows, step(op->ld_x, op->dim), step(op->ld_out, op->dim), 0, op->dim, op->eps};
  const Shape h = shape_of(op->dtype, op->dim);
  hipStream_t s = (hipStream_t)stream;
  return op->dtype == TT_F32    ? launch<float>(p, h, false, 0, s)
         : op->dtype == TT_BF16 ? launch<ttg::bf16>(p, h, false, 0, s)
                                : launch<ttg::f16>(p, h, false, 0, s);
}

extern "C" tt_status tt_layer_norm_backward(const tt_norm *op, const void *x, const void *weight, const float *stats, const void *grad_out, void *dx,
                                            void *dweight, void *dbias, void *workspace, size_t workspace_bytes, void *stream) {
  tt_status st = check(op);
  if (st != TT_OK) return st;
  if (!dx && !dweight && !dbias) return TT_OK;
  const bool some = op->rows > 0, sums = dweight || dbias;
  const size_t es = op->dtype == TT_F32 ? 4 : 2;
  if (some && (!x || !stats || !grad_out)) return TT_ERR_INVALID_ARG;
  const void *ptrs[7] = {x, weight, stats, grad_out, dx, dweight, dbias};
  for (int i = 0; i < 7; ++i) {
    if (!aligned(ptrs[i], i == 2 ? 4 : es)) return TT_ERR_INVALID_ARG;
    for (int j = 4; j < 7; ++j)
      if (i < j && ptrs[j] && ptrs[i] == ptrs[j]) return TT_ERR_INVALID_ARG;
  }
  const int shares = shares_of(op);
  if (sums && some && (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < (size_t)shares * 2 * op->dim * 4)) return TT_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  float *partial = sums ? (float *)workspace : nullptr;
  if (some && (dx || sums)) {
    Norm p = {x, weight, nullptr, grad_out, dx, const_cast<float *>(stats), partial, op->rows, step(op->ld_x, op->dim), step(op->ld_dx, op->dim),
              step(op->ld_grad, op->dim), op->dim, op->eps};
    const Shape h = shape_of(op->dtype, op->dim);
    st = op->dtype == TT_F32    ? launch<float>(p, h, true, shares, s)
         : op->dtype == TT_BF16 ? launch<ttg::bf16>(p, h, true, shares, s)
                                : launch<ttg::f16>(p, h, true, shares, s);
    if (st != TT_OK) return st;
  }
  if (!sums) return TT_OK;
  return op->dtype == TT_F32    ? join<float>(partial, some ? shares : 0, op->dim, dweight, dbias, s)
         : op->dtype == TT_BF16 ? join<ttg::bf16>(partial, some ? shares : 0, op->dim, dweight, dbias, s)
                                : join<ttg::f16>(partial, some ? shares : 0, op->dim, dweight, dbias, s);
}
