// Softmax cross entropy of short rows (up to 128 elements of 16 bits): nothing of the size rows x classes is ever stored.
#include "tt_gemm_device.h"
#include "tt_loss.h"

namespace {
using namespace ttg;

// Three kernels of one build.  A wavefront holds 64 vectors (`held`) in its registers as one operand of the products, and a workgroup of four
// streams the others through LDS, 32 at a time, as the other:
//   STATS    held rows, streamed classes: running largest logit and sum of exponentials of each row
//   ROWS     held rows, streamed classes: dx^T += W^T P
//   CLASSES  held classes, streamed rows: dW^T += x^T P (and its sums: dbias)
// The first product's result S (streamed x held) leaves a lane four neighbouring streamed vectors of one held one, and the second product sums
// over the streamed ones: two tiles of 16 of P = exp(S - ..) are, as they lie in the registers, an operand of 32 terms, whose order 4 q + i | 16 +
// 4 q + i the transposing LDS reads of the other operand follow.  So P goes from matrix instruction to matrix instruction through exp and a
// rounding alone; it is never in memory.
// What is added to a logit comes for nothing: of the streamed vector (the class's bias, or a row's -lse) as the product's starting value, of the held
// one in the multiply-add before exp2.
// 512 registers of a SIMD's lane are two wavefronts of 256: 64 of the held operand, 128 of the sums, 32 of S.
constexpr int WAVES = 4, THREADS = 64 * WAVES, STEP = 32;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float RAISE = 13.f;  // P is formed 2^13 times its size: fp16's smallest numbers then are of 2^-37, and P stays below 2^14
enum Mode { STATS, ROWS, CLASSES };
constexpr int held_tiles(int KP, Mode mode) { return mode != STATS && KP == 128 ? 3 : 4; }  // of 16 vectors, of a wavefront

struct Args {
  const void *held, *streamed;
  const void *bias;          // [classes], nullable
  const float *lse, *weight; // of places
  const int32_t *label;
  const int64_t *offsets;
  void *out, *sums;          // CLASSES of one run: dW, dbias
  const float *back;
  float *parts;
  long long rows;
  int dim, classes, runs;
};

// 16-byte pieces of an LDS row are spread so that sixteen neighbouring rows at one piece, and eight at two neighbouring pieces (the transposing
// read), meet every bank once.
template <int KP> __device__ __forceinline__ int spread(int r) {
  if constexpr (KP == 128) return (r & 7) << 1 | (r >> 3 & 1);
  else return (r >> 1 & 3) << 1 | (r >> 3 & 1);  // (two rows of 128 bytes share the banks)
}
template <int KP> __device__ __forceinline__ u16x8 frag(const unsigned short *tile, int r0, int s) {  // rows r0 .. + 15, k = 32 s + 8 q + i
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15;
  return *reinterpret_cast<const u16x8 *>(tile + (r0 + j) * KP + (((4 * s + q) ^ spread<KP>(j)) << 3));
}
template <int KP> __device__ __forceinline__ u16x8 frag_across(const unsigned short *tile, int c0) {  // columns c0 .. + 15, rows 4 q + i | 16 + 4 q + i
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15, r = 4 * q + (j >> 2);
  const unsigned short *at = tile + r * KP + (((c0 >> 3) + ((j & 3) >> 1)) ^ spread<KP>(r)) * 8 + 4 * (j & 1);
  const u16x4 x = lds_read_tr(at), y = lds_read_tr(at + 16 * KP);
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
// Eight elements of a vector, zeros where there are none.
template <class T> __device__ __forceinline__ u16x8 load8(const T *p, int valid) {
  u16x8 v;
  if (valid >= 8) {
    const typename Vec<T>::v16b r = *reinterpret_cast<const typename Vec<T>::v16b *>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = r[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? __builtin_bit_cast(unsigned short, p[i]) : (unsigned short)0;
  }
  return v;
}

template <class T, int KP, Mode MODE, bool SHARES> __global__ void __launch_bounds__(THREADS, 2) k_narrow(Args a) {
  constexpr int KS = KP / 32, H = held_tiles(KP, MODE), HELD = 16 * H, D = KP / 16, PIECES = STEP * KP / 8 / THREADS;
  constexpr bool OUT = MODE != STATS, CLASS = MODE == CLASSES;
  __shared__ __align__(16) unsigned short tiles[2][STEP * KP];
  __shared__ __align__(16) float starts[2][STEP], shares[SHARES ? 2 : 1][SHARES ? STEP : 4];
  __shared__ int labels[CLASS ? 2 : 1][CLASS ? STEP : 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), q = lane >> 4, j = lane & 15;
  const long long places = a.offsets[1];
  const long long held_count = CLASS ? a.classes : places, streamed_count = CLASS ? places : a.classes;
  const long long h0 = (long long)blockIdx.x * (HELD * WAVES) + wave * HELD;
  if ((long long)blockIdx.x * (HELD * WAVES) >= held_count) return;  // (the whole workgroup)
  // this run's share of the streamed vectors, whole steps
  const long long steps = (streamed_count + STEP - 1) / STEP, per = (steps + a.runs - 1) / a.runs;
  const long long s0 = blockIdx.y * per * STEP, s1 = s0 + per * STEP < streamed_count ? s0 + per * STEP : streamed_count;
  // vectors of x are KP apart, padded with zeros; of W dim apart
  const int ld_held = CLASS ? a.dim : KP, ld_streamed = CLASS ? KP : a.dim, held_dim = ld_held, streamed_dim = ld_streamed;

  u16x8 held[H][KS];
  float constant[H];  // of the held vector, in units of log 2
#pragma unroll
  for (int x = 0; x < H; ++x) {
    const long long h = h0 + 16 * x + j;
    const bool in = h < held_count;
#pragma unroll
    for (int s = 0; s < KS; ++s) held[x][s] = load8((const T *)a.held + (in ? h : 0) * ld_held + 32 * s + 8 * q, in ? held_dim - 32 * s - 8 * q : 0);
    if constexpr (MODE == ROWS) constant[x] = (in ? -a.lse[h] * LOG2E : 0.f) + RAISE;
    else if constexpr (CLASS) constant[x] = (a.bias && in ? to_f32(((const T *)a.bias)[h]) * LOG2E : 0.f) + (SHARES ? 0.f : RAISE);
    else constant[x] = 3e38f;  // less the largest so far: below all
  }
  f32x4 acc[OUT ? D : 1][H] = {};  // [columns][held]
  float sums[H] = {};

  u16x8 next[PIECES];
  float start_next = 0.f, share_next = 0.f;
  int label_next = -1;
  auto fetch = [&](long long t) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int p = threadIdx.x + i * THREADS, r = p / (KP / 8), c = p % (KP / 8) * 8;
      const bool in = t + r < s1;
      next[i] = load8((const T *)a.streamed + (in ? t + r : 0) * ld_streamed + c, in ? streamed_dim - c : 0);
    }
    if (threadIdx.x < STEP) {
      const long long r = t + threadIdx.x;
      const bool in = r < s1;
      if constexpr (CLASS) {
        start_next = in ? -a.lse[r] : -INFINITY;
        label_next = in ? a.label[r] : -1;
        if constexpr (SHARES) share_next = in ? a.weight[r] : 0.f;
      } else {
        start_next = in ? (a.bias ? to_f32(((const T *)a.bias)[r]) : 0.f) : -INFINITY;
      }
    }
  };
  auto put = [&](int b) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int p = threadIdx.x + i * THREADS, r = p / (KP / 8), c8 = p % (KP / 8);
      *reinterpret_cast<u16x8 *>(tiles[b] + r * KP + ((c8 ^ spread<KP>(r & 15)) << 3)) = next[i];
    }
    if (threadIdx.x < STEP) {
      starts[b][threadIdx.x] = start_next;
      if constexpr (CLASS) labels[b][threadIdx.x] = label_next;
      if constexpr (SHARES) shares[b][threadIdx.x] = share_next;
    }
  };

  if (s0 < s1) {
    fetch(s0);
    put(0);
  }
  int b = 0;
  for (long long t = s0; t < s1; t += STEP, b ^= 1) {
    __syncthreads();  // this step's tile is whole, and nobody reads the other buffer any more
    const bool more = t + STEP < s1;
    if (more) fetch(t + STEP);
    const unsigned short *tile = tiles[b];
    bool hit = false;  // a label of these rows is among the wavefront's classes
    if constexpr (CLASS) hit = __ballot(lane < STEP && (unsigned)(labels[b][lane & 31] - (int)h0) < (unsigned)HELD) != 0;
    u16x8 P[OUT ? H : 1];
#pragma unroll
    for (int half = 0; half < 2; ++half) {  // 16 streamed vectors
      f32x4 S[H];
      const f32x4 from = *reinterpret_cast<const f32x4 *>(&starts[b][16 * half + 4 * q]);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const u16x8 f = frag<KP>(tile, 16 * half, s);
#pragma unroll
        for (int x = 0; x < H; ++x) S[x] = mma(T(), f, held[x][s], s ? S[x] : from);
      }
      if constexpr (MODE == STATS) {
#pragma unroll
        for (int x = 0; x < H; ++x) {
          const float top = fmaxf(fmaxf(S[x][0], S[x][1]), fmaxf(S[x][2], S[x][3]));
          // what exp2 gets stays below 16, so that the sum stays far from the range's end; seldom after the first steps
          const bool above = fmaf(top, LOG2E, constant[x]) > 16.f;
          if (__ballot(above)) {
            const float now = above ? -top * LOG2E : constant[x];
            sums[x] *= above ? __builtin_amdgcn_exp2f(now - constant[x]) : 1.f;
            constant[x] = now;
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) sums[x] += __builtin_amdgcn_exp2f(fmaf(S[x][i], LOG2E, constant[x]));
        }
      } else {
        __builtin_amdgcn_sched_barrier(0);
        f32x4 share;
        if constexpr (SHARES) share = *reinterpret_cast<const f32x4 *>(&shares[b][16 * half + 4 * q]);
#pragma unroll
        for (int x = 0; x < H; ++x) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            S[x][i] = __builtin_amdgcn_exp2f(fmaf(S[x][i], LOG2E, constant[x]));
            if constexpr (SHARES) S[x][i] *= share[i];
          }
          if constexpr (CLASS) {
            if (hit) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (labels[b][16 * half + 4 * q + i] == (int)(h0 + 16 * x + j)) S[x][i] -= SHARES ? share[i] : 8192.f;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) sums[x] += S[x][i];
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) P[x][4 * half + i] = __builtin_bit_cast(unsigned short, from_f32<T>(S[x][i]));
        }
      }
    }
    if constexpr (OUT) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int y = 0; y < D; ++y) {
        const u16x8 f = frag_across<KP>(tile, 16 * y);
#pragma unroll
        for (int x = 0; x < H; ++x) acc[y][x] = mma(T(), f, P[x], acc[y][x]);
      }
    }
    if (more) put(b ^ 1);
  }

  if constexpr (MODE == STATS) {
#pragma unroll
    for (int x = 0; x < H; ++x) {  // four lanes have a row's columns
      float2 mine = {-constant[x] * LN2, sums[x]};
      if (constant[x] == 3e38f) mine = {-INFINITY, sums[x]};  // nothing but -infinity (or NaN, which the sum has)
#pragma unroll
      for (int o = 16; o < 64; o *= 2) mine = join_stats(mine, float2{__shfl(mine.x, lane ^ o, 64), __shfl(mine.y, lane ^ o, 64)});
      const long long h = h0 + 16 * x + j;
      if (q == 0 && h < held_count) reinterpret_cast<float2 *>(a.parts)[blockIdx.y * a.rows + h] = mine;
    }
  } else {
#pragma unroll
    for (int x = 0; x < H; ++x) {
      const long long h = h0 + 16 * x + j;
      if constexpr (CLASS) {
        sums[x] += __shfl(sums[x], lane ^ 16, 64);
        sums[x] += __shfl(sums[x], lane ^ 32, 64);
      }
      if (h >= held_count) continue;
      if (CLASS && a.runs == 1) {
        const float back = *a.back;
#pragma unroll
        for (int y = 0; y < D; ++y) {
          const int c = 16 * y + 4 * q;
          float v[4] = {acc[y][x][0] * back, acc[y][x][1] * back, acc[y][x][2] * back, acc[y][x][3] * back};
          if (a.out && c < a.dim) store4((T *)a.out + h * a.dim + c, a.dim - c, v);
        }
        if (a.sums && q == 0) ((T *)a.sums)[h] = from_f32<T>(sums[x] * back);
      } else {
        constexpr int LD = CLASS ? KP + 4 : KP;
        float *to = a.parts + (blockIdx.y * (CLASS ? (long long)a.classes : a.rows) + h) * LD;
#pragma unroll
        for (int y = 0; y < D; ++y) *reinterpret_cast<f32x4 *>(to + 16 * y + 4 * q) = acc[y][x];
        if (CLASS && q == 0) to[KP] = sums[x];
      }
    }
  }
}

// z of each place's label, as a product of its own: 16 lanes a place
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_narrow_picked(TTNarrow n, float *picked) {
  const int lane = threadIdx.x % 16;
  const long long i = (long long)blockIdx.x * (TT_BLOCK / 16) + threadIdx.x / 16;
  const bool in = i < n.r.offsets[1];
  const int label = in ? n.r.label[i] : -1;
  float v[8] = {}, w[8] = {}, s = 0.f;
  const int left = label >= 0 ? n.dim - 8 * lane : 0;
  if (left > 0) {
    load_n<T, 8>((const T *)n.x + i * n.padded + 8 * lane, left, v);
    load_n<T, 8>((const T *)n.w + (long long)label * n.dim + 8 * lane, left, w);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(v[e], w[e], s);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) s += __shfl(s, (threadIdx.x & 63) ^ o, 64);
  if (in && lane == 0) picked[i] = s + (n.bias && label >= 0 ? to_f32(((const T *)n.bias)[label]) : 0.f);
}

// dx = share (sum of the runs' parts - W of the label), zeros in rows that do not count; four columns a thread
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_narrow_dx(TTNarrow n, int runs, const float *__restrict__ parts, T *dx, long long ld) {
  const int per = (n.dim + 3) / 4;
  for (long long e = (long long)blockIdx.x * TT_BLOCK + threadIdx.x; e < n.rows * per; e += (long long)gridDim.x * TT_BLOCK) {
    const long long r = e / per;
    const int c = (int)(e - r * per) * 4, at = n.r.at[r];
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (at >= 0) {
      f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
      for (int k = 0; k < runs; ++k) s += *reinterpret_cast<const f32x4 *>(parts + (k * n.rows + at) * n.padded + c);
      const int label = n.r.label[at];
      if (label >= 0) load4((const T *)n.w + (long long)label * n.dim + c, n.dim - c, v);
      const float share = n.r.share[at];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = share * (s[i] * 0x1p-13f - v[i]);
    }
    store4(dx + r * ld + c, n.dim - c, v);
  }
}
// dW and dbias of several runs of the rows
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_narrow_dw(TTNarrow n, int runs, const float *__restrict__ parts, T *dw, T *db) {
  const int per = (n.dim + 3) / 4 + 1, ld = n.padded + 4;
  const float back = *n.r.back;
  for (long long e = (long long)blockIdx.x * TT_BLOCK + threadIdx.x; e < (long long)n.classes * per; e += (long long)gridDim.x * TT_BLOCK) {
    const long long h = e / per;
    const int c = (int)(e - h * per) * 4;
    const bool sum = c >= n.dim;  // the last one: dbias
    if (sum ? !db : !dw) continue;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int k = 0; k < runs; ++k) {
      const float *p = parts + (k * (long long)n.classes + h) * ld + (sum ? n.padded : c);
      if (sum) s[0] += *p;
      else s += *reinterpret_cast<const f32x4 *>(p);
    }
    float v[4] = {s[0] * back, s[1] * back, s[2] * back, s[3] * back};
    if (sum) db[h] = from_f32<T>(v[0]);
    else store4(dw + h * n.dim + c, n.dim - c, v);
  }
}

// ---- host ------------------------------------------------------------------------------------------
Args args_of(const TTNarrow &n, bool classes) {
  Args a = {};
  a.held = classes ? n.w : n.x;
  a.streamed = classes ? n.x : n.w;
  a.bias = n.bias;
  a.lse = n.r.lse;
  a.weight = n.r.weight;
  a.label = n.r.label;
  a.offsets = n.r.offsets;
  a.back = n.r.back;
  a.rows = n.rows;
  a.dim = n.dim;
  a.classes = n.classes;
  return a;
}
template <class T, int KP> tt_status launch(Mode mode, bool shares, const Args &a, long long held, hipStream_t s) {
  const dim3 grid((unsigned)tt_ceil_div(held, 16 * held_tiles(KP, mode) * WAVES), (unsigned)a.runs), block(THREADS);
  if (mode == STATS) hipLaunchKernelGGL((k_narrow<T, KP, STATS, false>), grid, block, 0, s, a);
  else if (mode == ROWS) hipLaunchKernelGGL((k_narrow<T, KP, ROWS, false>), grid, block, 0, s, a);
  else if (shares) hipLaunchKernelGGL((k_narrow<T, KP, CLASSES, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_narrow<T, KP, CLASSES, false>), grid, block, 0, s, a);
  return tt_launch_status();
}
tt_status launch(const TTNarrow &n, Mode mode, bool shares, const Args &a, hipStream_t s) {
  const long long held = mode == CLASSES ? n.classes : n.rows;
  if (n.dtype == TT_BF16) return n.padded == 64 ? launch<ttg::bf16, 64>(mode, shares, a, held, s) : launch<ttg::bf16, 128>(mode, shares, a, held, s);
  return n.padded == 64 ? launch<ttg::f16, 64>(mode, shares, a, held, s) : launch<ttg::f16, 128>(mode, shares, a, held, s);
}
unsigned grid_of(long long items) {
  const long long blocks = (items + TT_BLOCK - 1) / TT_BLOCK;
  return (unsigned)(blocks < 1 ? 1 : blocks > 16384 ? 16384 : blocks);
}
int runs_of(long long held, long long streamed) {
  // about as many workgroups as two rounds of two on 256 compute units, eight steps at least in each
  const long long blocks = (held + 255) / 256, steps = (streamed + STEP - 1) / STEP;
  long long runs = 1024 / (blocks > 0 ? blocks : 1);
  if (runs > steps / 8) runs = steps / 8;
  if (runs > 256) runs = 256;
  return (int)(runs < 1 ? 1 : runs);
}

}  // namespace

#ifndef TT_LOSS_NARROW
#define TT_LOSS_NARROW 128
#endif
bool ttk_narrow_serves(int dtype, int dim) { return dtype != TT_F32 && dim <= TT_LOSS_NARROW; }
int ttk_narrow_padded(int dim) { return dim <= 64 ? 64 : 128; }
int ttk_narrow_runs(long long rows, int classes) { return runs_of(rows, classes); }
int ttk_narrow_row_runs(long long rows, int classes) { return runs_of(classes, rows); }

tt_status ttk_narrow_stats(const TTNarrow &n, float *stats, hipStream_t s) {
  Args a = args_of(n, false);
  a.parts = stats;
  a.runs = ttk_narrow_runs(n.rows, n.classes);
  return launch(n, STATS, false, a, s);
}
tt_status ttk_narrow_picked(const TTNarrow &n, float *picked, hipStream_t s) {
  const dim3 grid((unsigned)tt_ceil_div(n.rows, TT_BLOCK / 16)), block(TT_BLOCK);
  if (n.dtype == TT_BF16) hipLaunchKernelGGL(k_narrow_picked<ttg::bf16>, grid, block, 0, s, n, picked);
  else hipLaunchKernelGGL(k_narrow_picked<ttg::f16>, grid, block, 0, s, n, picked);
  return tt_launch_status();
}
tt_status ttk_narrow_dx(const TTNarrow &n, float *parts, void *dx, long long ld_dx, hipStream_t s) {
  Args a = args_of(n, false);
  a.parts = parts;
  a.runs = ttk_narrow_runs(n.rows, n.classes);
  const tt_status st = launch(n, ROWS, false, a, s);
  if (st != TT_OK) return st;
  const dim3 grid(grid_of(n.rows * ((n.dim + 3) / 4))), block(TT_BLOCK);
  const int runs = a.runs;
  if (n.dtype == TT_BF16) hipLaunchKernelGGL(k_narrow_dx<ttg::bf16>, grid, block, 0, s, n, runs, (const float *)parts, (ttg::bf16 *)dx, ld_dx);
  else hipLaunchKernelGGL(k_narrow_dx<ttg::f16>, grid, block, 0, s, n, runs, (const float *)parts, (ttg::f16 *)dx, ld_dx);
  return tt_launch_status();
}
tt_status ttk_narrow_dw(const TTNarrow &n, bool shares, float *parts, void *dw, void *dbias, hipStream_t s) {
  Args a = args_of(n, true);
  a.parts = parts;
  a.out = dw;
  a.sums = dbias;
  a.runs = ttk_narrow_row_runs(n.rows, n.classes);
  const tt_status st = launch(n, CLASSES, shares, a, s);
  if (st != TT_OK || a.runs == 1) return st;
  const dim3 grid(grid_of((long long)n.classes * ((n.dim + 3) / 4 + 1))), block(TT_BLOCK);
  const int runs = a.runs;
  if (n.dtype == TT_BF16) hipLaunchKernelGGL(k_narrow_dw<ttg::bf16>, grid, block, 0, s, n, runs, (const float *)parts, (ttg::bf16 *)dw, (ttg::bf16 *)dbias);
  else hipLaunchKernelGGL(k_narrow_dw<ttg::f16>, grid, block, 0, s, n, runs, (const float *)parts, (ttg::f16 *)dw, (ttg::f16 *)dbias);
  return tt_launch_status();
}
