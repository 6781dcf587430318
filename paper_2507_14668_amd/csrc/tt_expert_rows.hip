// Rows to their experts and back: copies into the experts' order, weighted sums out of it, and the gradients.
#include "tt_gemm_device.h"

namespace {
using namespace ttg;

struct Deal {  // of a call, by value to the kernels
  const void *x, *y, *residual, *grad;
  const int32_t *slots, *sources;
  const float *weights;
  void *out, *dy;
  float *dweights;
  long long rows, places, ld_rows, ld_residual, ld_places, ld_dy;
  int n, k, zero_rest;
};

// Sixteen bytes of a row as they are; `valid` of its C elements exist.
template <class T> struct Chunk {
  static constexpr int C = 16 / sizeof(T);
  typename Vec<T>::v16b v;
  __device__ __forceinline__ void load(const T *p, int valid) {
    if (valid >= C) v = *reinterpret_cast<const typename Vec<T>::v16b *>(p);
    else {
#pragma unroll
      for (int i = 0; i < C; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = i < valid ? p[i] : 0.f;
        else v[i] = i < valid ? __builtin_bit_cast(unsigned short, p[i]) : (unsigned short)0;
      }
    }
  }
  __device__ __forceinline__ void store(T *p, int valid) const {
    if (valid >= C) *reinterpret_cast<typename Vec<T>::v16b *>(p) = v;
    else {
#pragma unroll
      for (int i = 0; i < C; ++i)
        if (i < valid) {
          if constexpr (sizeof(T) == 4) p[i] = v[i];
          else p[i] = __builtin_bit_cast(T, (unsigned short)v[i]);
        }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] = 0;
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return v[i];
    else return to_f32(__builtin_bit_cast(T, (unsigned short)v[i]));
  }
};

// LANES threads take a row.  The place of choice j, in all of them; -1 if there is none.
__device__ __forceinline__ int place_of(const Deal &p, long long r, int j) {
  const int s = p.slots[r * p.k + j];
  return s >= 0 && s < p.places ? s : -1;
}
__device__ __forceinline__ bool no_source(const Deal &p, long long place) {
  const int s = p.sources[place];
  return s < 0 || s >= p.places;
}

// Bound by memory: 16384 rows of 1024 in bf16 to four places each 33.9 us (5.0 TB/s).
// A row is read once and written to its places.  The places numbered row * k .. + k - 1 are looked after too: those without a
// source are cleared.
template <class T, int LANES> __global__ void __launch_bounds__(TT_BLOCK) k_rows(Deal p) {
  constexpr int C = Chunk<T>::C, GROUPS = TT_BLOCK / LANES;
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  for (long long r = (long long)blockIdx.x * GROUPS + group; r < p.rows; r += (long long)gridDim.x * GROUPS) {
    for (int c = lane * C; c < p.n; c += LANES * C) {
      Chunk<T> v;
      v.load((const T *)p.x + r * p.ld_rows + c, p.n - c);
      for (int j = 0; j < p.k; ++j) {
        const int s = place_of(p, r, j);
        if (s >= 0) v.store((T *)p.out + s * p.ld_places + c, p.n - c);
      }
      if (p.zero_rest) {
        v.zero();
        for (int j = 0; j < p.k; ++j)
          if (no_source(p, r * p.k + j)) v.store((T *)p.out + (r * p.k + j) * p.ld_places + c, p.n - c);
      }
    }
  }
}

// out = residual + sum of weight * y, fp32, the choices in order.  A lane has NV chunks of a row at a time (all of a row that they
// cover), so that its loads for several choices are under way together.  The rows above back: 46 us (4.3 TB/s; rows of 2 KB anywhere in memory).
template <class T, int LANES, int NV> __global__ void __launch_bounds__(TT_BLOCK) k_combine(Deal p) {
  constexpr int C = Chunk<T>::C, GROUPS = TT_BLOCK / LANES, WIDTH = LANES * C * NV;
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  for (long long r = (long long)blockIdx.x * GROUPS + group; r < p.rows; r += (long long)gridDim.x * GROUPS) {
    for (int c0 = lane * C; c0 < p.n; c0 += WIDTH) {
      float sum[NV][C] = {};
#pragma unroll 4
      for (int j = 0; j < p.k; ++j) {
        const int s = place_of(p, r, j);
        if (s < 0) continue;
        const float w = p.weights ? p.weights[r * p.k + j] : 1.f;
        Chunk<T> v[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i].load((const T *)p.y + s * p.ld_places + c0 + i * LANES * C, p.n - c0 - i * LANES * C);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
          for (int e = 0; e < C; ++e) sum[i][e] = fmaf(w, v[i].at(e), sum[i][e]);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = c0 + i * LANES * C;
        if (c >= p.n) break;
        if (p.residual) {
          Chunk<T> v;
          v.load((const T *)p.residual + r * p.ld_residual + c, p.n - c);
#pragma unroll
          for (int e = 0; e < C; ++e) sum[i][e] += v.at(e);
        }
        store_n<T, C>((T *)p.out + r * p.ld_rows + c, p.n - c, sum[i]);
      }
    }
  }
}

// dy = weight * grad in each place, dweight = <grad, y>.  With NV a row fits its lanes and its gradient is read once; without (0) it is read
// for every choice (70 us for the rows above, 57 with: 5.3 TB/s).
template <class T, int LANES, int NV> __global__ void __launch_bounds__(TT_BLOCK) k_combine_backward(Deal p) {
  constexpr int C = Chunk<T>::C, GROUPS = TT_BLOCK / LANES, N = NV ? NV : 1;
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
  for (long long r0 = (long long)blockIdx.x * GROUPS; r0 < p.rows; r0 += (long long)gridDim.x * GROUPS) {
    const bool live = r0 + group < p.rows;
    const long long r = live ? r0 + group : p.rows - 1;
    Chunk<T> g[N];
    if constexpr (NV != 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) g[i].load((const T *)p.grad + r * p.ld_rows + (i * LANES + lane) * C, p.n - (i * LANES + lane) * C);
    }
#pragma unroll 2
    for (int j = 0; j < p.k; ++j) {
      const int s = live ? place_of(p, r, j) : -1;
      const float w = s >= 0 && p.weights ? p.weights[r * p.k + j] : 1.f;
      const bool rest = live && p.dy && no_source(p, r * p.k + j);
      float dot = 0.f;
      for (int c0 = lane * C; c0 < p.n; c0 += LANES * C * N) {
        if (s >= 0) {
          if constexpr (NV == 0) g[0].load((const T *)p.grad + r * p.ld_rows + c0, p.n - c0);
          Chunk<T> v[N];
          if (p.dweights) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i].load((const T *)p.y + s * p.ld_places + c0 + i * LANES * C, p.n - c0 - i * LANES * C);
          }
          if (p.dy) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
              const int c = c0 + i * LANES * C;
              float d[C];
#pragma unroll
              for (int e = 0; e < C; ++e) d[e] = w * g[i].at(e);
              if (c < p.n) store_n<T, C>((T *)p.dy + s * p.ld_dy + c, p.n - c, d);
            }
          }
          if (p.dweights) {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
              for (int e = 0; e < C; ++e) dot = fmaf(g[i].at(e), v[i].at(e), dot);  // (zeros behind the row's end)
          }
        }
        if (rest) {
          Chunk<T> z;
          z.zero();
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int c = c0 + i * LANES * C;
            if (c < p.n) z.store((T *)p.dy + (r * p.k + j) * p.ld_dy + c, p.n - c);
          }
        }
      }
      if (p.dweights) {
#pragma unroll
        for (int o = LANES / 2; o > 0; o >>= 1) dot += __shfl(dot, (threadIdx.x & 63) ^ o, 64);
        if (live && lane == 0) p.dweights[r * p.k + j] = s >= 0 ? dot : 0.f;
      }
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------
const long long kMostPlaces = 2147483647LL - 2 * TT_DENSE_MAX_GROUPS;

tt_status check(const tt_deal *op) {
  if (!op || op->dtype < TT_F32 || op->dtype > TT_F16 || op->rows < 0) return TT_ERR_INVALID_ARG;
  if (op->dim < 1 || op->dim > TT_NORM_MAX_DIM || op->choices < 1 || op->choices > TT_ROUTE_MAX_CHOICES || op->rows >= kMostPlaces / op->choices)
    return TT_ERR_SHAPE;
  const int64_t ld[4] = {op->ld_rows, op->ld_residual, op->ld_places, op->ld_dy};
  for (int i = 0; i < 4; ++i)
    if (ld[i] != 0 && (ld[i] < op->dim || ld[i] > ((int64_t)1 << 40))) return TT_ERR_SHAPE;
  return TT_OK;
}
bool aligned(const void *p, size_t size) { return ((uintptr_t)p & (size - 1)) == 0; }
size_t elem(int dtype) { return dtype == TT_F32 ? 4 : 2; }
Deal describe(const tt_deal *op) {
  Deal p = {};
  p.rows = op->rows;
  p.places = op->rows * op->choices;
  p.ld_rows = op->ld_rows ? op->ld_rows : op->dim;
  p.ld_residual = op->ld_residual ? op->ld_residual : op->dim;
  p.ld_places = op->ld_places ? op->ld_places : op->dim;
  p.ld_dy = op->ld_dy ? op->ld_dy : op->dim;
  p.n = op->dim;
  p.k = op->choices;
  p.zero_rest = op->zero_rest;
  return p;
}
enum Which { ROWS, COMBINE, BACKWARD };
template <class T, int LANES, int NV> void launch_as(const Deal &p, Which which, hipStream_t s) {
  long long blocks = (p.rows + TT_BLOCK / LANES - 1) / (TT_BLOCK / LANES);
  if (blocks > 65536) blocks = 65536;
  const dim3 grid((unsigned)blocks), block(TT_BLOCK);
  if (which == ROWS) hipLaunchKernelGGL((k_rows<T, LANES>), grid, block, 0, s, p);
  else if (which == COMBINE) hipLaunchKernelGGL((k_combine<T, LANES, NV ? NV : 4>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((k_combine_backward<T, LANES, NV>), grid, block, 0, s, p);
}
template <class T> tt_status launch(const Deal &p, Which which, hipStream_t s) {
  const int chunks = tt_ceil_div(p.n, Chunk<T>::C);
  if (chunks <= 16) launch_as<T, 16, 1>(p, which, s);
  else if (chunks <= 32) launch_as<T, 16, 2>(p, which, s);
  else if (chunks <= 64) launch_as<T, 64, 1>(p, which, s);
  else if (chunks <= 128) launch_as<T, 64, 2>(p, which, s);
  else if (chunks <= 256) launch_as<T, 64, 4>(p, which, s);
  else launch_as<T, 64, 0>(p, which, s);
  return tt_launch_status();
}
tt_status launch(int dtype, const Deal &p, Which which, hipStream_t s) {
  return dtype == TT_F32 ? launch<float>(p, which, s) : dtype == TT_BF16 ? launch<ttg::bf16>(p, which, s) : launch<ttg::f16>(p, which, s);
}

}  // namespace

extern "C" tt_status tt_expert_rows(const tt_deal *op, const void *x, const int32_t *slots, const int32_t *sources, void *out, void *stream) {
  const tt_status st = check(op);
  if (st != TT_OK) return st;
  if (op->rows == 0) return TT_OK;
  const size_t es = elem(op->dtype);
  if (!x || !slots || !out || (op->zero_rest && !sources) || !aligned(x, es) || !aligned(out, es) || !aligned(slots, 4) || !aligned(sources, 4))
    return TT_ERR_INVALID_ARG;
  if (out == x || out == (const void *)slots || out == (const void *)sources) return TT_ERR_INVALID_ARG;
  Deal p = describe(op);
  p.x = x;
  p.slots = slots;
  p.sources = sources;
  p.out = out;
  return launch(op->dtype, p, ROWS, (hipStream_t)stream);
}

extern "C" tt_status tt_expert_combine(const tt_deal *op, const void *y, const int32_t *slots, const float *weights, const void *residual, void *out,
                                       void *stream) {
  const tt_status st = check(op);
  if (st != TT_OK) return st;
  if (op->rows == 0) return TT_OK;
  const size_t es = elem(op->dtype);
  if (!y || !slots || !out || !aligned(y, es) || !aligned(out, es) || !aligned(residual, es) || !aligned(slots, 4) || !aligned(weights, 4))
    return TT_ERR_INVALID_ARG;
  if (out == y || out == (const void *)slots || out == (const void *)weights) return TT_ERR_INVALID_ARG;
  Deal p = describe(op);
  if (out == residual && op->rows > 1 && p.ld_rows != p.ld_residual) return TT_ERR_INVALID_ARG;
  p.y = y;
  p.slots = slots;
  p.weights = weights;
  p.residual = residual;
  p.out = out;
  return launch(op->dtype, p, COMBINE, (hipStream_t)stream);
}

extern "C" tt_status tt_expert_combine_backward(const tt_deal *op, const void *y, const int32_t *slots, const int32_t *sources, const float *weights,
                                                const void *grad, void *dy, float *dweights, void *stream) {
  const tt_status st = check(op);
  if (st != TT_OK) return st;
  if (op->rows == 0 || (!dy && !dweights)) return TT_OK;
  const size_t es = elem(op->dtype);
  if ((dweights && !y) || !slots || !grad || (dy && !sources)) return TT_ERR_INVALID_ARG;
  const void *ptrs[7] = {y, slots, sources, weights, grad, dy, dweights};
  const size_t sizes[7] = {es, 4, 4, 4, es, es, 4};
  for (int i = 0; i < 7; ++i) {
    if (!aligned(ptrs[i], sizes[i])) return TT_ERR_INVALID_ARG;
    for (int j = 5; j < 7; ++j)
      if (i < j && ptrs[j] && ptrs[i] == ptrs[j]) return TT_ERR_INVALID_ARG;
  }
  Deal p = describe(op);
  p.y = y;
  p.slots = slots;
  p.sources = sources;
  p.weights = weights;
  p.grad = grad;
  p.dy = dy;
  p.dweights = dweights;
  return launch(op->dtype, p, BACKWARD, (hipStream_t)stream);
}
