// Softmax cross entropy of short rows (up to 128 elements): nothing of the size rows x classes is ever stored.
#include <float.h>

#include "tt_gemm_device.h"
#include "tt_loss.h"

namespace {
using namespace ttg;

// Three kernels of one build.  A wavefront holds 64 vectors (`held`) in its registers as one operand of the products, and a workgroup of four
// streams the others through LDS, 32 at a time, as the other:
//   STATS    held rows, streamed classes: running largest logit and sum of exponentials of each row, its label's apart
//   ROWS     held rows, streamed classes: dx^T += W^T P
//   CLASSES  held classes, streamed rows: dW^T += x^T P (and its sums: dbias)
// The first product's result S (streamed x held) leaves a lane four neighbouring streamed vectors of one held one, and the second product sums
// over the streamed ones: two tiles of 16 of P = exp(S - ..) are, as they lie in the registers, an operand of 32 terms, whose order 4 q + i | 16 +
// 4 q + i the transposing LDS reads of the other operand follow.  So P goes from matrix instruction to matrix instruction through exp and a
// rounding alone; it is never in memory.
// A class's bias is the product's starting value, in all three, so that all have the same bits of a logit.  What the row has (the reference of its statistics, or lse) is taken off
// before the difference is scaled for exp2: in one multiply-add with that it would be rounded in the size of the logits, and e to the power of that is what all probabilities
// are off by (14 % at logits of 2^20).
// fp32 operands come in PARTS = 3 planes of bf16 (tt_split_bf16), P is split as it is formed, and six of the nine products count, as in the other fp32
// products; what they redo with the fp32 instruction (numbers below 2^-100 in size, or near the range's end) has fewer bits here, or is NaN.
// 512 registers of a SIMD's lane are two wavefronts of 256: 48 of the held operand (three tiles of 16), 96 of the sums, 24 of S.
// Measured, 4096 rows (3686 count) of 128 in bf16 against 500001 classes: STATS 600 us, ROWS 803, CLASSES 844; with G stored in pieces and multiplied
// from there the training pass took 7129, now 2300.  The matrix cores are busy 34, 50 and 47 % of it, as much again goes to the exponentials and what is around
// them, and two wavefronts a SIMD do not hide the one behind the other; the clock falls to 2.2 GHz.  Four held tiles spill, a step of the
// other half prefetched into registers does too, and loads through registers instead of straight into LDS took 742, 964 and 1052.
constexpr int WAVES = 4, THREADS = 64 * WAVES, STEP = TT_LOSS_STEP;
constexpr float LOG2E = 1.4426950408889634f;
// In fp16 P is formed 2^13 times its size: the smallest numbers then are of 2^-37, and P stays below 2^14.  bf16 has the range, and sums that need theirs.
template <class T> constexpr float raise() { return std::is_same<T, f16>::value ? 13.f : 0.f; }
template <class T> constexpr float raised() { return std::is_same<T, f16>::value ? TT_LOSS_RAISE : 1.f; }
enum Mode { STATS, ROWS, CLASSES };
// of 16 vectors, of a wavefront: what fits the registers
__host__ __device__ constexpr int held_tiles(int KP, Mode mode, int parts) { return parts == 1 ? (mode != STATS && KP == 128 ? 3 : 4) : KP == 128 ? (mode == STATS ? 3 : 2) : (mode == STATS ? 4 : 3); }

// How a launch is cut, from the number of held vectors (which the host does not know where they are rows that count) and of workgroups that run at once:
// workgroup w has block w % blocks of the held vectors and run w / blocks of the streamed ones.  As many runs as fill the card once, or
// twice where that wastes less; `least` steps at least in each, since its parts are written and added at the end.  (The rows above: ROWS in 64 runs, two and a half
// rounds, 964 us, in 23, one round, 899.)
struct Cut {
  int blocks, runs;
};
struct Sizes {  // of a kernel's launches
  int tile, slots, least;
};
__host__ __device__ inline Cut cut_of(long long held, long long streamed, const Sizes &z) {
  const int tile = z.tile, slots = z.slots;
  const long long blocks = held < 1 ? 1 : (held + tile - 1) / tile, steps = (streamed + STEP - 1) / STEP;
  const long long one = slots / blocks, two = 2LL * slots / blocks;
  long long runs = 42 * one >= 20 * two ? one : two;
  if (runs > steps / z.least) runs = steps / z.least;
  return Cut{(int)blocks, (int)(runs < 1 ? 1 : runs)};
}
// Workgroups for any number of vectors up to these.
inline long long grid_for(long long held, long long streamed, const Sizes &z) {
  const long long blocks = held < 1 ? 1 : (held + z.tile - 1) / z.tile, most = blocks * ((streamed + z.least * STEP - 1) / (z.least * STEP));
  const long long twice = 2LL * z.slots < most ? 2LL * z.slots : most;
  return blocks > twice ? blocks : twice;
}
__host__ __device__ constexpr int tile_of(int KP, Mode mode, int parts) { return 16 * held_tiles(KP, mode, parts) * WAVES; }
// A step takes 0.4 us of a wavefront, of fp32 1.5; the statistics' parts are eight bytes a row.
__host__ __device__ constexpr Sizes sizes_of(int KP, Mode mode, int parts) {
  return Sizes{tile_of(KP, mode, parts), 256 * (mode == STATS && parts == 1 ? 3 : 2), parts == 3 ? (mode == STATS ? 2 : 3) : mode == STATS ? 4 : 8};
}

struct Args {
  const void *held, *streamed;
  const float *starts;       // of streamed vectors: the bias, or a row's -lse; -infinity behind the last one, whole steps
  const float *constants;    // of held vectors: a row's -lse, or the bias
  const float *weight;       // CLASSES with shares: of the rows, whole steps
  const int32_t *label;      // of the rows, whole steps
  const float *hot;          // of the rows: the label's softmax less one
  float *picked;             // STATS: of the rows
  const int64_t *offsets;
  void *out, *sums;          // CLASSES of one run: dW, dbias
  const float *back;
  float *parts;              // [workgroup][tile]...
  long long held_plane, streamed_plane;  // elements between the planes of fp32 operands
  int dim, classes;
};

typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;
// Waits for the wavefront's loads (into LDS too) and LDS reads.
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(7 << 4);
  asm volatile("" ::: "memory");
}

// 16-byte pieces of an LDS row are spread so that sixteen neighbouring rows at one piece, and eight at two neighbouring pieces (the transposing
// read), lie in banks of their own.  The hardware takes the lanes in another grouping: 44 % of the LDS cycles of STATS, which reads `frag` alone, and 31 % of those of the
// other two are conflicts still.
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

__device__ __forceinline__ f32x4 all_of(float v) { return f32x4{v, v, v, v}; }

// A step's LDS: the tile, then of its vectors `starts` and the shares.
template <int KP, int PARTS> constexpr int step_bytes() { return STEP * KP * 2 * PARTS + 2 * STEP * 4; }

// What a thread fetches of a step.  The tile's 16-byte pieces go from memory into LDS, lane after lane; which piece a lane fetches makes their order
// there.  A vector behind the last one is the last one again, with -infinity: its P is zero.
template <int KP, Mode MODE, bool SHARES, int PARTS> struct Fetcher {
  const unsigned short *streamed;
  long long plane;
  const float *starts, *weight;
  long long count;
  int row, wave, lane;
  unsigned offset;
  __device__ __forceinline__ void fetch(long long t, char *to) const {
    constexpr int PIECES = STEP * KP / 8 / THREADS, PLANE = STEP * KP * 2, TILE = PARTS * PLANE;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const long long r = t + row + i * (THREADS / (KP / 8));
      const unsigned short *from = streamed + (r < count ? r : count - 1) * KP + offset;
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
        __builtin_amdgcn_global_load_lds((GlobalPtr)(from + p * plane), (LdsPtr)(to + p * PLANE + (i * THREADS + wave * 64) * 16), 16, 0, 0);
    }
    if (lane < STEP) {  // a wavefront each
      if (wave == 0) __builtin_amdgcn_global_load_lds((GlobalPtr)(starts + t + lane), (LdsPtr)(to + TILE), 4, 0, 0);
      if constexpr (SHARES)
        if (wave == 1) __builtin_amdgcn_global_load_lds((GlobalPtr)(weight + t + lane), (LdsPtr)(to + TILE + STEP * 4), 4, 0, 0);
    }
  }
};

// A step, from `now`, while the next one (`ahead`; behind the last: none) is on its way to `next`.  (The buffers are separate to the compiler,
// which else has every read wait for the loads.)
// hit: a label of the rows is among the classes here, which few steps have; one branch, since what is on its two sides is not
// interleaved.  `label`: of the held rows, less the step's first class; CLASSES lane l's is row l's, less the first held class.
// STATS gives the label's logit out there, and leaves it out of its sums (row_of_loss).  The others have the label's softmax less one, which the loss says to its last bits (`hot`, of the held rows or, CLASSES,
// of the step's): where a row is nearly sure of its label, exp(z - lse) - 1 would be the rounding of lse.
template <class T, int KP, Mode MODE, bool SHARES, int PARTS, int H, int DO>
__device__ __forceinline__ void step_of(const char *__restrict__ now, char *__restrict__ next, const Fetcher<KP, MODE, SHARES, PARTS> &fetcher, long long ahead,
                                        long long end, bool hit, const int (&label)[MODE == CLASSES ? 1 : H], const float *hot, float *picked,
                                        const u16x8 (&held)[H][KP / 32][PARTS], float (&constant)[H], f32x4 (&acc)[DO][H], float (&sums)[H]) {
  constexpr int KS = KP / 32, D = KP / 16;
  constexpr bool OUT = MODE != STATS, CLASS = MODE == CLASSES;
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15;
  if (ahead < end) fetcher.fetch(ahead, next);
  const unsigned short *tile = reinterpret_cast<const unsigned short *>(now);
  const float *starts = reinterpret_cast<const float *>(now + STEP * KP * 2 * PARTS), *shares = starts + STEP;
  f32x4 S[2][H];
#pragma unroll
  for (int half = 0; half < 2; ++half) {  // 16 streamed vectors
    const f32x4 of_streamed = *reinterpret_cast<const f32x4 *>(starts + 16 * half + 4 * q);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u16x8 f[PARTS];
#pragma unroll
      for (int p = 0; p < PARTS; ++p) f[p] = frag<KP>(tile + p * STEP * KP, 16 * half, s);
      // the smallest terms first
#pragma unroll
      for (int d = PARTS - 1; d >= 0; --d)
#pragma unroll
        for (int p = 0; p <= d; ++p)
#pragma unroll
          for (int x = 0; x < H; ++x) S[half][x] = mma(T(), f[d - p], held[x][s][p], s || d != PARTS - 1 || p ? S[half][x] : CLASS ? all_of(constant[x]) : of_streamed);
    }
    if constexpr (MODE == STATS) {
      if (hit) {
#pragma unroll
        for (int x = 0; x < H; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (label[x] == 16 * half + 4 * q + i) {
              picked[16 * x + j] = S[half][x][i];
              S[half][x][i] = -INFINITY;
            }
      }
#pragma unroll
      for (int x = 0; x < H; ++x) {
        const float top = fmaxf(fmaxf(S[half][x][0], S[half][x][1]), fmaxf(S[half][x][2], S[half][x][3]));
        // what is added up stays below e^11, so that the sum stays far from the range's end; seldom after the first steps
        const bool above = top - constant[x] > 11.f;
        if (__ballot(above)) {
          const float now = above ? top : constant[x];
          const float by = above ? __builtin_amdgcn_exp2f((constant[x] - now) * LOG2E) : 1.f;
          sums[x] *= by;
          acc[0][x][0] *= by;
          constant[x] = now;
        }
        float e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f((S[half][x][i] - constant[x]) * LOG2E);
        sums[x] += (e[0] + e[1]) + (e[2] + e[3]);
      }
    } else {
#pragma unroll
      for (int x = 0; x < H; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) S[half][x][i] = __builtin_amdgcn_exp2f(fmaf(S[half][x][i] + (CLASS ? of_streamed[i] : constant[x]), LOG2E, SHARES ? 0.f : raise<T>()));
    }
  }
  if constexpr (OUT) {
    if (hit) {
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int x = 0; x < H; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int streamed = 16 * half + 4 * q + i;
            if (CLASS ? __shfl(label[0], streamed, 64) == 16 * x + j : label[CLASS ? 0 : x] == streamed)
              S[half][x][i] = hot[CLASS ? streamed : 16 * x + j] * (SHARES ? 1.f : raised<T>());
          }
    }
    u16x8 P[H][PARTS];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      f32x4 share = {1.f, 1.f, 1.f, 1.f};
      if constexpr (SHARES) share = *reinterpret_cast<const f32x4 *>(shares + 16 * half + 4 * q);
#pragma unroll
      for (int x = 0; x < H; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (SHARES) S[half][x][i] *= share[i];
          if constexpr (PARTS == 1) P[x][0][4 * half + i] = __builtin_bit_cast(unsigned short, from_f32<T>(S[half][x][i]));
          else if (i & 1) {
            unsigned part[3];
            tt_split_bf16(S[half][x][i - 1], S[half][x][i], part[0], part[1], part[2]);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
              P[x][p][4 * half + i - 1] = (unsigned short)part[p];
              P[x][p][4 * half + i] = (unsigned short)(part[p] >> 16);
            }
          }
        }
      if constexpr (CLASS) {
#pragma unroll
        for (int x = 0; x < H; ++x) sums[x] += (S[half][x][0] + S[half][x][1]) + (S[half][x][2] + S[half][x][3]);
      }
    }
#pragma unroll
    for (int y = 0; y < D; ++y) {
      u16x8 f[PARTS];
#pragma unroll
      for (int p = 0; p < PARTS; ++p) f[p] = frag_across<KP>(tile + p * STEP * KP, 16 * y);
#pragma unroll
      for (int d = PARTS - 1; d >= 0; --d)
#pragma unroll
        for (int p = 0; p <= d; ++p)
#pragma unroll
          for (int x = 0; x < H; ++x) acc[y][x] = mma(T(), f[d - p], P[x][p], acc[y][x]);
    }
  }
}

// Statistics of two sets of a row's logits: m, about the largest, and s, the sum of exp(logit - m).  (A NaN or +infinity among them makes s NaN.)
__device__ __forceinline__ float2 join_runs(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x), base = top == -INFINITY ? 0.f : top;
  return float2{top, a.y * __builtin_amdgcn_exp2f((a.x - base) * LOG2E) + b.y * __builtin_amdgcn_exp2f((b.x - base) * LOG2E)};
}

// T: of the products; O: of dW and dbias
template <class T, class O, int KP, Mode MODE, bool SHARES> __global__ void __launch_bounds__(THREADS, MODE == STATS && sizeof(O) == 2 ? 3 : 2) k_narrow(Args a) {
  constexpr int PARTS = sizeof(O) == 4 ? 3 : 1, KS = KP / 32, H = held_tiles(KP, MODE, PARTS), HELD = 16 * H, D = KP / 16;
  constexpr bool OUT = MODE != STATS, CLASS = MODE == CLASSES;
  constexpr int BYTES = step_bytes<KP, PARTS>(), GIVE = CLASS ? WAVES * 16 * (KP + 8) * 2 : 0;  // two steps, or what is given out through it
  __shared__ __align__(16) char lds[GIVE > 2 * BYTES ? GIVE : 2 * BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), q = lane >> 4, j = lane & 15;
  const long long places = a.offsets[1];
  const long long held_count = CLASS ? a.classes : places, streamed_count = CLASS ? places : a.classes;
  const Cut cut = cut_of(held_count, streamed_count, sizes_of(KP, MODE, PARTS));
  const int block = (int)(blockIdx.x % (unsigned)cut.blocks), run = (int)(blockIdx.x / (unsigned)cut.blocks);
  if (run >= cut.runs || held_count == 0) return;
  const long long h0 = (long long)block * tile_of(KP, MODE, PARTS) + wave * HELD;
  // this run's share of the streamed vectors, whole steps
  const long long steps = (streamed_count + STEP - 1) / STEP, per = (steps + cut.runs - 1) / cut.runs;
  const long long s0 = run * per * STEP, s1 = s0 + per * STEP < streamed_count ? s0 + per * STEP : streamed_count;

  u16x8 held[H][KS][PARTS];
  float constant[H];  // of the held vector
#pragma unroll
  for (int x = 0; x < H; ++x) {
    const long long h = h0 + 16 * x + j < held_count ? h0 + 16 * x + j : held_count - 1;  // (of vectors outside nothing is written)
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int p = 0; p < PARTS; ++p)
        held[x][s][p] = *reinterpret_cast<const u16x8 *>((const unsigned short *)a.held + p * a.held_plane + h * KP + 32 * s + 8 * q);
    constant[x] = MODE == STATS ? -FLT_MAX /* the largest so far, about: below all */ : a.constants[h];
  }
  f32x4 acc[OUT ? D : 1][H] = {};  // [columns][held]; STATS: [0] what sums were 16 steps ago and before (a chain of additions stays short)
  float sums[H] = {};

  const int row = (int)threadIdx.x / (KP / 8);
  const Fetcher<KP, MODE, SHARES, PARTS> fetcher = {(const unsigned short *)a.streamed, a.streamed_plane, a.starts, a.weight, streamed_count, row, wave, lane,
                                                ((threadIdx.x % (KP / 8)) ^ spread<KP>(row & 15)) * 8};
  // Labels are a step ahead of their use, in a register: of the held rows less the first class, or of the streamed rows less the first held class.
  int label[CLASS ? 1 : H] = {}, label_next = 0;
  if constexpr (!CLASS) {
#pragma unroll
    for (int x = 0; x < H; ++x) label[x] = h0 + 16 * x + j < held_count ? a.label[h0 + 16 * x + j] - (int)s0 : -1;
  }
  if (s0 < s1) {
    fetcher.fetch(s0, lds);
    if constexpr (CLASS) label_next = a.label[s0 + (lane & 31)];
    wait_loads();
  }
  int b = 0;
  for (long long t = s0; t < s1; t += STEP, b ^= 1) {
    __syncthreads();  // this step has landed, everyone's part of it, and nobody reads the other buffer any more
    bool hit = false;
    if constexpr (!CLASS) {
#pragma unroll
      for (int x = 0; x < H; ++x) hit |= (unsigned)label[x] < (unsigned)STEP;
    }
    if constexpr (CLASS) {
      label[0] = label_next - (int)h0;
      hit = (unsigned)label[0] < (unsigned)HELD;
      if (t + STEP < s1) label_next = a.label[t + STEP + (lane & 31)];
    }
    step_of<T, KP, MODE, SHARES, PARTS>(lds + b * BYTES, lds + (b ^ 1) * BYTES, fetcher, t + STEP, s1, __ballot(hit) != 0, label, CLASS ? a.hot + t : a.hot + h0, a.picked + h0, held, constant, acc, sums);
    if constexpr (!CLASS) {
#pragma unroll
      for (int x = 0; x < H; ++x) label[x] -= STEP;
    }
    if (MODE == STATS && ((t - s0) / STEP & 15) == 15) {
#pragma unroll
      for (int x = 0; x < H; ++x) {
        acc[0][x][0] += sums[x];
        sums[x] = 0.f;
      }
    }
    wait_loads();
  }

  const int first = wave * HELD;  // of the workgroup's tile
  if constexpr (MODE == STATS) {
#pragma unroll
    for (int x = 0; x < H; ++x) {  // four lanes have a row's columns
      sums[x] += acc[0][x][0];
      float2 mine = {sums[x] == 0.f ? -INFINITY : constant[x], sums[x]};  // (0: nothing but -infinity)
#pragma unroll
      for (int o = 16; o < 64; o *= 2) mine = join_runs(mine, float2{__shfl(mine.x, lane ^ o, 64), __shfl(mine.y, lane ^ o, 64)});
      if (q == 0) reinterpret_cast<float2 *>(a.parts)[(long long)blockIdx.x * tile_of(KP, MODE, PARTS) + first + 16 * x + j] = mine;
    }
  } else if (MODE == ROWS || cut.runs > 1) {
    constexpr int LD = CLASS ? KP + 4 : KP;
    float *to = a.parts + ((long long)blockIdx.x * tile_of(KP, MODE, PARTS) + first) * LD;
#pragma unroll
    for (int x = 0; x < H; ++x) {
#pragma unroll
      for (int y = 0; y < D; ++y) *reinterpret_cast<f32x4 *>(to + (16 * x + j) * LD + 16 * y + 4 * q) = acc[y][x];
      if constexpr (CLASS) {
        sums[x] += __shfl(sums[x], lane ^ 16, 64);
        sums[x] += __shfl(sums[x], lane ^ 32, 64);
        if (q == 0) to[(16 * x + j) * LD + KP] = sums[x];
      }
    }
  } else if constexpr (CLASS) {
    const float back = *a.back;
    // through LDS, 16 classes at a time, so that whole lines are written
    constexpr int LD = KP + 8, PER = KP / 8, ROWS_AT = 64 / PER;
    __syncthreads();  // nobody reads a step any more
    unsigned short *room = reinterpret_cast<unsigned short *>(lds) + wave * 16 * LD;
#pragma unroll
    for (int x = 0; x < H; ++x) {
      sums[x] += __shfl(sums[x], lane ^ 16, 64);
      sums[x] += __shfl(sums[x], lane ^ 32, 64);
      const long long h = h0 + 16 * x;
      if (a.sums && q == 0 && h + j < held_count) ((O *)a.sums)[h + j] = from_f32<O>(sums[x] * back);
      if (!a.out) continue;
      if constexpr (PARTS == 3) {  // 64 bytes of a row at a time as they are
#pragma unroll
        for (int y = 0; y < D; ++y) {
          const int c = 16 * y + 4 * q;
          const float v[4] = {acc[y][x][0] * back, acc[y][x][1] * back, acc[y][x][2] * back, acc[y][x][3] * back};
          if (h + j < held_count && c < a.dim) store4((float *)a.out + (h + j) * a.dim + c, a.dim - c, v);
        }
        continue;
      }
#pragma unroll
      for (int y = 0; y < D; ++y) {
        u16x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(unsigned short, from_f32<T>(acc[y][x][i] * back));
        *reinterpret_cast<u16x4 *>(room + j * LD + 16 * y + 4 * q) = v;
      }
      tt_wave_lds_order();
#pragma unroll
      for (int r = lane / PER; r < 16; r += ROWS_AT) {
        const int c = lane % PER * 8;
        const u16x8 v = *reinterpret_cast<const u16x8 *>(room + r * LD + c);
        if (h + r >= held_count || c >= a.dim) continue;
        T *to = (T *)a.out + (h + r) * a.dim + c;
        if (a.dim - c >= 8) {
          typename Vec<T>::v16b o;
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = v[i];
          *reinterpret_cast<typename Vec<T>::v16b *>(to) = o;
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i < a.dim - c) to[i] = __builtin_bit_cast(T, (unsigned short)v[i]);
        }
      }
      tt_wave_lds_order();
    }
  }
}

// Each place's statistics of all runs together, and what the row has of them: a wavefront a place.
__global__ void __launch_bounds__(TT_BLOCK) k_narrow_fold(TTNarrow n, const float2 *__restrict__ parts, Sizes z, const float *picked, float2 *each, float *loss) {
  const int lane = threadIdx.x & 63;
  const long long i = (long long)blockIdx.x * (TT_BLOCK / 64) + (threadIdx.x >> 6), places = n.r.offsets[1];
  if (i >= places) return;
  const Cut cut = cut_of(places, n.classes, z);
  const long long block = i / z.tile;
  float2 s = {-INFINITY, 0.f};
  for (int k = lane; k < cut.runs; k += 64) s = join_runs(s, parts[(k * (long long)cut.blocks + block) * z.tile + i % z.tile]);
#pragma unroll
  for (int o = 1; o < 64; o *= 2) s = join_runs(s, float2{__shfl(s.x, lane ^ o, 64), __shfl(s.y, lane ^ o, 64)});
  if (lane != 0) return;
  const int r = n.r.of[i];
  const float2 of = n.r.label[i] < 0 ? float2{NAN, NAN} : row_of_loss(s, picked[i]);
  each[r] = of;
  if (loss) loss[r] = of.y;
}

// The sums of the runs' parts of vectors, four columns a thread (the last four: the sums beside dW).  Up to eight runs: SEGMENTS vectors a workgroup, each by its own
// threads; more: one vector, the runs in SEGMENTS shares that are then added in order (in the threads of the first).
template <int KP> struct Summing {
  static constexpr int PER = KP / 4 + 1, SEGMENTS = TT_BLOCK / PER;
  __device__ static __forceinline__ bool together(const Cut &cut) { return cut.runs > 8; }
  // `vector`: the workgroup's, or its threads' own (-1: none); all threads of the workgroup call it
  __device__ static __forceinline__ f32x4 sum(const float *__restrict__ parts, int ld, const Cut &cut, int tile, long long vector, f32x4 *room) {
    const int c = (int)threadIdx.x % PER, seg = (int)threadIdx.x / PER, each = together(cut) ? (cut.runs + SEGMENTS - 1) / SEGMENTS : cut.runs;
    const int from = together(cut) ? seg * each : 0, end = from + each < cut.runs ? from + each : cut.runs;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (vector >= 0 && seg < SEGMENTS && 4 * c < ld) {
      const long long block = vector / tile;
#pragma unroll 4
      for (int k = from; k < end; ++k) s += *reinterpret_cast<const f32x4 *>(parts + ((k * (long long)cut.blocks + block) * tile + vector % tile) * ld + 4 * c);
    }
    if (!together(cut)) return s;
    __syncthreads();  // nobody reads the last vector's any more
    room[threadIdx.x] = s;
    __syncthreads();
    if (seg == 0) {
#pragma unroll
      for (int k = 1; k < SEGMENTS; ++k) s += room[k * PER + c];
    }
    return s;
  }
};
// dx = share times the sum, zeros in rows that do not count
template <class T, int KP> __global__ void __launch_bounds__(TT_BLOCK) k_narrow_dx(TTNarrow n, const float *__restrict__ parts, T *dx, long long ld) {
  typedef Summing<KP> S;
  constexpr Sizes z = sizes_of(KP, ROWS, sizeof(T) == 4 ? 3 : 1);
  __shared__ __align__(16) f32x4 room[TT_BLOCK];
  const Cut cut = cut_of(n.r.offsets[1], n.classes, z);
  const bool together = S::together(cut);
  const int c = 4 * ((int)threadIdx.x % S::PER), seg = (int)threadIdx.x / S::PER, many = together ? 1 : S::SEGMENTS;
  for (long long r0 = (long long)blockIdx.x * many; r0 < n.rows; r0 += (long long)gridDim.x * many) {
    const long long r = r0 + (together ? 0 : seg);
    const bool in = r < n.rows && seg < S::SEGMENTS;
    const int at = in ? n.r.at[r] : -1;
    f32x4 s = S::sum(parts, KP, cut, z.tile, at, room);
    if (!in || (together && seg != 0) || c >= n.dim || c >= KP) continue;
    if (at >= 0) s *= 1.f / raised<T>() * n.r.share[at];
    const float v[4] = {s[0], s[1], s[2], s[3]};
    store4(dx + r * ld + c, n.dim - c, v);
  }
}
// dW and dbias where the rows came in several runs
template <class T, int KP> __global__ void __launch_bounds__(TT_BLOCK) k_narrow_dw(TTNarrow n, const float *__restrict__ parts, T *dw, T *db) {
  typedef Summing<KP> S;
  constexpr Sizes z = sizes_of(KP, CLASSES, sizeof(T) == 4 ? 3 : 1);
  __shared__ __align__(16) f32x4 room[TT_BLOCK];
  const Cut cut = cut_of(n.classes, n.r.offsets[1], z);
  if (cut.runs == 1) return;  // the products' kernel has written them
  const bool together = S::together(cut);
  const float back = *n.r.back;
  const int c = 4 * ((int)threadIdx.x % S::PER), seg = (int)threadIdx.x / S::PER, many = together ? 1 : S::SEGMENTS;
  for (long long h0 = (long long)blockIdx.x * many; h0 < n.classes; h0 += (long long)gridDim.x * many) {
    const long long h = h0 + (together ? 0 : seg);
    const bool in = h < n.classes && seg < S::SEGMENTS;
    const f32x4 s = S::sum(parts, KP + 4, cut, z.tile, in ? h : -1, room) * back;
    if (!in || (together && seg != 0)) continue;
    const float v[4] = {s[0], s[1], s[2], s[3]};
    if (dw && c < n.dim && c < KP) store4(dw + h * n.dim + c, n.dim - c, v);
    if (db && c == KP) db[h] = from_f32<T>(v[0]);
  }
}

// What the kernels above take: vectors `padded` apart with zeros behind their ends (fp32: three planes of their parts), those at `of` of them if that
// is given, zeros behind the `there` that there are; and the classes' biases as numbers of 32 bits (-infinity behind the last one, whole steps).
template <class T> __global__ void __launch_bounds__(TT_BLOCK) k_narrow_take(const T *from, long long ld, const int32_t *of, const int64_t *there, long long count, int dim,
                                                                             unsigned short *to, int padded, const T *bias, float *starts) {
  const long long stride = (long long)gridDim.x * TT_BLOCK, some = there ? there[1] : count, whole = (count + STEP - 1) / STEP * STEP, plane = count * padded;
  if (starts)
    for (long long i = (long long)blockIdx.x * TT_BLOCK + threadIdx.x; i < whole; i += stride) starts[i] = i >= count ? -INFINITY : bias ? to_f32(bias[i]) : 0.f;
  if (!to) return;
  const int per = padded / 8;
  for (long long e = (long long)blockIdx.x * TT_BLOCK + threadIdx.x; e < count * per; e += stride) {
    const long long r = e / per;
    const int c = (int)(e - r * per) * 8;
    float v[8] = {};
    if (r < some) load_n<T, 8>(from + (of ? of[r] : r) * ld + c, dim - c, v);
    if constexpr (sizeof(T) == 2) {
      store_n<T, 8>((T *)to + r * padded + c, 8, v);
    } else {
      typedef unsigned u4 __attribute__((ext_vector_type(4)));
      u4 part[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        unsigned h, m, l;
        tt_split_bf16(v[2 * i], v[2 * i + 1], h, m, l);
        part[0][i] = h;
        part[1][i] = m;
        part[2][i] = l;
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) *reinterpret_cast<u4 *>(to + p * plane + r * padded + c) = part[p];
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------
Args args_of(const TTNarrow &n, bool classes) {
  Args a = {};
  const void *w = n.copy ? n.copy : n.w;
  a.held = classes ? w : n.x;
  a.streamed = classes ? n.x : w;
  a.starts = classes ? n.r.lse : n.starts;
  a.constants = classes ? n.starts : n.r.lse;
  a.weight = n.r.weight;
  a.label = n.r.label;
  a.hot = n.r.hot;
  a.offsets = n.r.offsets;
  a.back = n.r.back;
  a.held_plane = (classes ? (long long)n.classes : n.rows) * n.padded;
  a.streamed_plane = (classes ? n.rows : (long long)n.classes) * n.padded;
  a.dim = n.dim;
  a.classes = n.classes;
  return a;
}
int parts_of(const TTNarrow &n) { return n.dtype == TT_F32 ? 3 : 1; }
template <Mode MODE> Sizes sizes_for(const TTNarrow &n) { return sizes_of(n.padded, MODE, parts_of(n)); }
template <Mode MODE> int tile_for(const TTNarrow &n) { return sizes_for<MODE>(n).tile; }
template <Mode MODE> long long workgroups(const TTNarrow &n) {
  const long long held = MODE == CLASSES ? n.classes : n.rows, streamed = MODE == CLASSES ? n.rows : n.classes;
  return grid_for(held, streamed, sizes_for<MODE>(n));
}
template <class T, class O, int KP, Mode MODE> tt_status launch_as(const TTNarrow &n, bool shares, const Args &a, hipStream_t s) {
  const dim3 grid((unsigned)workgroups<MODE>(n)), block(THREADS);
  if constexpr (MODE == CLASSES) {
    if (shares) hipLaunchKernelGGL((k_narrow<T, O, KP, MODE, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_narrow<T, O, KP, MODE, false>), grid, block, 0, s, a);
  } else {
    hipLaunchKernelGGL((k_narrow<T, O, KP, MODE, false>), grid, block, 0, s, a);
  }
  return tt_launch_status();
}
template <class T, class O, Mode MODE> tt_status launch_padded(const TTNarrow &n, bool shares, const Args &a, hipStream_t s) {
  return n.padded == 64 ? launch_as<T, O, 64, MODE>(n, shares, a, s) : launch_as<T, O, 128, MODE>(n, shares, a, s);
}
template <Mode MODE> tt_status launch(const TTNarrow &n, bool shares, const Args &a, hipStream_t s) {
  if (workgroups<MODE>(n) > TT_MAX_WORKGROUPS) return TT_ERR_SHAPE;
  if (n.dtype == TT_F32) return launch_padded<ttg::bf16, float, MODE>(n, shares, a, s);
  return n.dtype == TT_BF16 ? launch_padded<ttg::bf16, ttg::bf16, MODE>(n, shares, a, s) : launch_padded<ttg::f16, ttg::f16, MODE>(n, shares, a, s);
}
#define TT_BY_TYPE(call, dtype, ...) \
  ((dtype) == TT_F32 ? call<float>(__VA_ARGS__) : (dtype) == TT_BF16 ? call<ttg::bf16>(__VA_ARGS__) : call<ttg::f16>(__VA_ARGS__))
unsigned grid_of(long long items) {
  const long long blocks = (items + TT_BLOCK - 1) / TT_BLOCK;
  return (unsigned)(blocks < 1 ? 1 : blocks > 16384 ? 16384 : blocks);
}
unsigned most_of(long long n) { return (unsigned)(n > 65536 ? 65536 : n); }
template <class T> tt_status finish_dx(const TTNarrow &n, const float *parts, void *dx, long long ld, hipStream_t s) {
  const dim3 grid(most_of(n.rows)), block(TT_BLOCK);
  if (n.padded == 64) hipLaunchKernelGGL((k_narrow_dx<T, 64>), grid, block, 0, s, n, parts, (T *)dx, ld);
  else hipLaunchKernelGGL((k_narrow_dx<T, 128>), grid, block, 0, s, n, parts, (T *)dx, ld);
  return tt_launch_status();
}
template <class T> tt_status finish_dw(const TTNarrow &n, const float *parts, void *dw, void *db, hipStream_t s) {
  const dim3 grid(most_of(n.classes)), block(TT_BLOCK);
  if (n.padded == 64) hipLaunchKernelGGL((k_narrow_dw<T, 64>), grid, block, 0, s, n, parts, (T *)dw, (T *)db);
  else hipLaunchKernelGGL((k_narrow_dw<T, 128>), grid, block, 0, s, n, parts, (T *)dw, (T *)db);
  return tt_launch_status();
}
template <class T> tt_status take(const TTNarrow &n, bool classes, hipStream_t s) {
  const long long count = classes ? n.classes : n.rows, ld = classes ? n.dim : n.ld;
  const T *from = (const T *)(classes ? n.w : n.of_call), *bias = classes ? (const T *)n.bias : nullptr;
  const int32_t *of = classes ? nullptr : n.r.of;
  const int64_t *there = classes ? nullptr : n.r.offsets;
  unsigned short *to = (unsigned short *)(classes ? n.copy : n.x);
  float *starts = classes ? n.starts : nullptr;
  const int dim = n.dim, padded = n.padded;
  hipLaunchKernelGGL(k_narrow_take<T>, dim3(grid_of(count * (to ? padded / 8 : 1))), dim3(TT_BLOCK), 0, s, from, ld, of, there, count, dim, to, padded, bias, starts);
  return tt_launch_status();
}
// Whether the classes are few enough for the rows to come in several runs (fewer rows that count never make it so).
bool several(const TTNarrow &n) { return workgroups<CLASSES>(n) > tt_ceil_div(n.classes, tile_for<CLASSES>(n)); }

}  // namespace

#ifndef TT_LOSS_NARROW
#define TT_LOSS_NARROW 128
#endif
bool ttk_narrow_serves(int dim) { return dim <= TT_LOSS_NARROW; }
int ttk_narrow_padded(int dim) { return dim <= 64 ? 64 : 128; }

size_t ttk_narrow_stats_bytes(const TTNarrow &n) { return (size_t)workgroups<STATS>(n) * tile_for<STATS>(n) * 8; }
size_t ttk_narrow_parts_bytes(const TTNarrow &n) {
  const size_t dx = (size_t)workgroups<ROWS>(n) * tile_for<ROWS>(n) * n.padded * 4;
  const size_t dw = several(n) ? (size_t)workgroups<CLASSES>(n) * tile_for<CLASSES>(n) * (n.padded + 4) * 4 : 0;
  return dx > dw ? dx : dw;
}

tt_status ttk_narrow_take(const TTNarrow &n, hipStream_t s) {
  const tt_status st = TT_BY_TYPE(take, n.dtype, n, false, s);
  return st == TT_OK ? TT_BY_TYPE(take, n.dtype, n, true, s) : st;
}
tt_status ttk_narrow_stats(const TTNarrow &n, float *stats, float *picked, float *each, float *loss, hipStream_t s) {
  Args a = args_of(n, false);
  a.parts = stats;
  a.picked = picked;
  const tt_status st = launch<STATS>(n, false, a, s);
  if (st != TT_OK) return st;
  const Sizes z = sizes_for<STATS>(n);
  hipLaunchKernelGGL(k_narrow_fold, dim3((unsigned)tt_ceil_div(n.rows, TT_BLOCK / 64)), dim3(TT_BLOCK), 0, s, n, (const float2 *)stats, z, (const float *)picked,
                     (float2 *)each, loss);
  return tt_launch_status();
}
tt_status ttk_narrow_dx(const TTNarrow &n, float *parts, void *dx, long long ld_dx, hipStream_t s) {
  Args a = args_of(n, false);
  a.parts = parts;
  const tt_status st = launch<ROWS>(n, false, a, s);
  return st == TT_OK ? TT_BY_TYPE(finish_dx, n.dtype, n, (const float *)parts, dx, ld_dx, s) : st;
}
tt_status ttk_narrow_dw(const TTNarrow &n, bool shares, float *parts, void *dw, void *dbias, hipStream_t s) {
  Args a = args_of(n, true);
  a.parts = parts;
  a.out = dw;
  a.sums = dbias;
  const tt_status st = launch<CLASSES>(n, shares, a, s);
  return st == TT_OK && several(n) ? TT_BY_TYPE(finish_dw, n.dtype, n, (const float *)parts, dw, dbias, s) : st;
}
