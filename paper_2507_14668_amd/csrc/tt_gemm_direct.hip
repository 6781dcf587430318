// Large 16-bit products: tiles of 256 x 256, operands straight from memory into LDS.
#include "tt_gemm_device.h"

namespace {
using namespace ttg;

// 256 x 256 of out per workgroup of eight wavefronts (128 x 64 each), in steps of 64 values of K through two buffers of 64 KB.  Every
// element is fetched once per tile and never passes through a register on its way to LDS: a tile of 128 x 128 through registers
// (tt_gemm.hip) is bound by LDS, whose reads and writes take longer than its matrix instructions.  A step has two halves: while one
// half's operands multiply, the next half's are read from LDS into the registers that fall free, and between the halves a step's buffer is
// handed to the loads of the step after the next, which have a whole step to land.
// A load puts 16 bytes a lane at consecutive places in LDS, so the order that spreads the reads over the banks is made
// by which 16 bytes each lane fetches.  Needs 16-byte aligned rows and a K (K-contiguous) or a number of rows (row-contiguous) that is
// a multiple of 8: pieces of 16 bytes are whole or outside.  Rows outside are read from a row inside (their results are not stored),
// values of K outside from a piece of zeros.
// Measured in bf16: 16384 x 4096 x 4096 426 us (1290 TFLOP/s; x W, both from rows 446, dz^T x 464), 8192^3 815 us (1350); the library's product
// without an epilogue 353 and 757.  With bias, gelu and residual the first takes 490: a tile's results are finished while nothing multiplies
// (one workgroup fills the LDS), and that is what bounds it now.  Tried and no faster: steps of 32 through four buffers (half lines of 128
// bytes for K-contiguous operands), touching lines of later steps so that they are in the L2.
constexpr int E = 256, BK = 64, THREADS = 512, OPERAND = E * BK;  // halves of an operand in a buffer
constexpr int STAGES = 2, PIECES = 4;                             // loads of a thread for an operand and step
__device__ __align__(16) unsigned short g_zeros[8];

typedef const __attribute__((address_space(1))) void *GlobalPtr;
typedef __attribute__((address_space(3))) void *LdsPtr;

// One operand's loads: a wavefront fills the pieces 64 (wave + 8 i) + lane of a buffer.
template <class T, bool KC> struct Loader {
  const T *base;         // of the next step
  unsigned off[PIECES];  // elements
  int k[PIECES];         // of the piece, within a step
  long long step;
  __device__ __forceinline__ void start(const T *tile, long long ld, int rows, int wave, int lane) {  // tile: row 0 of the tile at the first k
    base = tile;
    step = KC ? BK : (long long)BK * ld;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int p = 64 * (wave + 8 * i) + lane;
      if constexpr (KC) {
        const int r = p >> 3, k8 = (p & 7) ^ (r & 7);
        k[i] = 8 * k8;
        off[i] = (unsigned)((long long)(r < rows ? r : rows - 1) * ld + 8 * k8);
      } else {
        // blocks of four rows by 16 columns, 128 bytes that a transposing read takes whole; blocks of four rows after each other
        const int kr = 4 * (p >> 7) + ((p >> 1) & 3), c = 16 * ((p >> 3) & 15) + 8 * (p & 1);
        k[i] = kr;
        off[i] = (unsigned)(kr * ld + (c < rows ? c : 0));
      }
    }
  }
  __device__ __forceinline__ void load(unsigned short *lds, int wave, int left) {  // left: values of K from this step on
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const void *src = left >= BK || k[i] < left ? (const void *)(base + off[i]) : (const void *)g_zeros;
      __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)(lds + (wave + 8 * i) * 512), 16, 0, 0);
    }
    base += step;
  }
};

// eight elements of rows r0 .. + 15 at k = 32 s + 8 (lane / 16) + i
template <bool KC> __device__ __forceinline__ u16x8 frag(const unsigned short *lds, int r0, int s) {
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15;
  if constexpr (KC) return *reinterpret_cast<const u16x8 *>(lds + (r0 + j) * BK + (((4 * s + q) ^ (j & 7)) << 3));
  const unsigned short *at = lds + (8 * s + 2 * q) * 1024 + r0 * 4 + 4 * j;  // block [8 s + 2 q][r0 / 16], of 64 elements
  const u16x4 x = lds_read_tr(at), y = lds_read_tr(at + 1024);
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Waits until at most N of the wavefront's loads are under way (and no LDS read).
template <int N> __device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Half a step: its operands are in fa and fb; those of the next half (`s` of `next`) are read between the matrix instructions,
// each into the registers that are free by then.
template <class T, bool AKC, bool BKC>
__device__ __forceinline__ void half_step(const unsigned short *__restrict__ next, int s, int wm, int wn, bool sums, u16x8 (&fa)[8], u16x8 (&fb)[4],
                                          f32x4 (&acc)[8][4], f32x4 &rs) {
  u16x8 nb[4];
#pragma unroll
  for (int y = 0; y < 4; ++y) nb[y] = frag<BKC>(next + OPERAND, wn + 16 * y, s);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int x = 0; x < 8; ++x) {
#pragma unroll
    for (int y = 0; y < 4; ++y) acc[x][y] = mma(T(), fb[y], fa[x], acc[x][y]);
    if constexpr (!AKC) {
      if (sums) {  // row x of one result: ones in row x of the first operand
        unsigned short one = std::is_same<T, f16>::value ? 0x3c00 : 0x3f80;
        one = (threadIdx.x & 15) == x ? one : 0;
        rs = mma(T(), u16x8{one, one, one, one, one, one, one, one}, fa[x], rs);
      }
    }
    fa[x] = frag<AKC>(next, wm + 16 * x, s);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int y = 0; y < 4; ++y) fb[y] = nb[y];
}
// A step whose first half is in the registers and whose buffer is `now`; between its halves that buffer is free for the loads of the step
// after the next one, `next`, which has landed by then.  (The buffers are separate to the compiler too, which else has every
// read wait for all loads.)
template <class T, bool AKC, bool BKC>
__device__ __forceinline__ void step_of(unsigned short *__restrict__ now, const unsigned short *__restrict__ next, Loader<T, AKC> &la, Loader<T, BKC> &lb,
                                        int ahead, int wave, int wm, int wn, bool sums, u16x8 (&fa)[8], u16x8 (&fb)[4], f32x4 (&acc)[8][4], f32x4 &rs) {
  half_step<T, AKC, BKC>(now, 1, wm, wn, sums, fa, fb, acc, rs);
  wait_loads<0>();  // this wavefront's loads of the next step have landed, and its reads of this one are done
  barrier();        // ... everyone's
  la.load(now, wave, ahead);  // behind the last step: zeros
  lb.load(now + OPERAND, wave, ahead);
  half_step<T, AKC, BKC>(next, 0, wm, wn, sums, fa, fb, acc, rs);
}

// Sums of A's rows wm .. + 127 from memory, in the order of the steps above: for tiles where the one result that keeps all eight of a lane's
// sums is of no use (a NaN or an infinity times its zeros is NaN, in the sums of seven other rows).  Eight results of their own do not fit the
// registers beside the product, and such tiles are the exception; the bits of the other sums are the same either way.
template <class T> __device__ __forceinline__ void row_sums(const T *a, long long lda, int rows, int K, int wm, f32x4 (&rs)[8]) {
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15;
  const unsigned short one = std::is_same<T, f16>::value ? 0x3c00 : 0x3f80;
#pragma unroll 1
  for (int k0 = 0; k0 < K; k0 += 32) {
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const int c = wm + 16 * x + j;
      u16x8 v;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = k0 + 8 * q + i;
        v[i] = k < K && c < rows ? __builtin_bit_cast(unsigned short, a[k * lda + c]) : (unsigned short)0;
      }
      rs[x] = mma(T(), u16x8{one, one, one, one, one, one, one, one}, v, rs[x]);
    }
  }
}

template <class T, bool AKC, bool BKC> __global__ void __launch_bounds__(THREADS, 2) k_gemm_direct(TTGemm g, int m_tiles, int n_tiles, int chunk, float *partial) {
  __shared__ __align__(16) unsigned short lds[16 * finish_floats<4, 4>()];  // (more than two buffers take)
  static_assert(16 * finish_floats<4, 4>() >= STAGES * 2 * OPERAND, "LDS");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  unsigned mt, nt;
  tile_order(blockIdx.x, (unsigned)m_tiles, (unsigned)n_tiles, false, mt, nt);
  Place w;
  w.n0 = (int)nt * E;
  w.k_lo = 0;
  w.k_hi = g.K;
  float *piece = nullptr;
  if (g.mode == TT_GEMM_RAGGED_M) {
    const int there = find_tile<E>(g.offsets, g.batch, g.M, (int)mt, w.z, w.lo, w.hi);
    if (w.z < 0) {
      if (g.zero_rest) clear_rest<T>(g, w.lo, w.hi, (int)mt - there, m_tiles - there, w.n0, E);
      return;
    }
  } else {
    w.z = (int)blockIdx.y;
    w.lo = (int)mt * E;
    w.hi = g.M < w.lo + E ? g.M : w.lo + E;
    if (g.mode == TT_GEMM_RAGGED_K) {
      int pieces = 1, number = 0;
      find_slot(g.offsets, g.batch, g.K, chunk, BK, (int)blockIdx.y, w.z, w.k_lo, w.k_hi, pieces, number);
      if (w.z < 0) return;
      if (pieces > 1) piece = partial + (long long)__builtin_amdgcn_readfirstlane(number) * ttk_gemm_piece_floats(g);
    }
  }
  w.z = __builtin_amdgcn_readfirstlane(w.z);
  w.lo = __builtin_amdgcn_readfirstlane(w.lo);
  w.hi = __builtin_amdgcn_readfirstlane(w.hi);
  w.k_lo = __builtin_amdgcn_readfirstlane(w.k_lo);
  w.k_hi = __builtin_amdgcn_readfirstlane(w.k_hi);
  const T *a = (const T *)g.a + (g.mode == TT_GEMM_BATCH ? w.z * g.a_step : 0) + (AKC ? w.lo * g.lda + w.k_lo : w.k_lo * g.lda + w.lo);
  const T *b = (const T *)g.b + (g.mode != TT_GEMM_RAGGED_K ? w.z * g.b_step : 0) + (BKC ? w.n0 * g.ldb + w.k_lo : w.k_lo * g.ldb + w.n0);
  Loader<T, AKC> la;
  Loader<T, BKC> lb;
  la.start(a, g.lda, w.hi - w.lo, wave, lane);
  lb.start(b, g.ldb, g.N - w.n0 < E ? g.N - w.n0 : E, wave, lane);
  const int wm = (wave >> 2) * 128, wn = (wave & 3) * 64;
  f32x4 acc[8][4] = {};
  f32x4 rs = {};  // sums of A's rows, beside products over stored rows only: lane (q, j) has those of 16 (4 q + i) + j
  const bool sums = !AKC && g.rowsum && w.n0 == 0 && wn == 0;
  const int K = w.k_hi - w.k_lo;
  int ahead = K;  // values of K that are not yet asked for
  if (K > 0) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
      la.load(lds + i * 2 * OPERAND, wave, ahead);
      lb.load(lds + i * 2 * OPERAND + OPERAND, wave, ahead);
      ahead -= BK;
    }
    wait_loads<2 * PIECES>();
    barrier();
    u16x8 fa[8], fb[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) fb[y] = frag<BKC>(lds + OPERAND, wn + 16 * y, 0);
#pragma unroll
    for (int x = 0; x < 8; ++x) fa[x] = frag<AKC>(lds, wm + 16 * x, 0);
    int now = 0;
    for (int k0 = 0; k0 < K; k0 += BK) {
      step_of<T, AKC, BKC>(lds + now, lds + (now ^ (2 * OPERAND)), la, lb, ahead, wave, wm, wn, sums, fa, fb, acc, rs);
      ahead -= BK;
      now ^= 2 * OPERAND;
    }
    wait_loads<0>();  // the zeros too, before LDS is used for something else
  }
  auto give_sum = [&](int m, float v) {
    if (m >= w.hi) return;
    if (piece) piece[(long long)g.M * g.N + m] = v;
    else ((T *)g.rowsum)[w.z * g.rs_step + m] = from_f32<T>(v);
  };
  bool odd = false;  // a sum that is not finite, in any lane
  if constexpr (!AKC) {
    if (sums) {
#pragma unroll
      for (int i = 0; i < 4; ++i) odd |= lane < 32 && !(fabsf(rs[i]) < INFINITY);
      odd = __ballot(odd) != 0;
      if (!odd && lane < 32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) give_sum(w.lo + wm + 16 * (4 * (lane >> 4) + i) + (lane & 15), rs[i]);
      }
    }
  }
  __syncthreads();  // nobody reads the operands any more
  float *room = reinterpret_cast<float *>(lds) + wave * finish_floats<4, 4>();
  if constexpr (!AKC) {  // (only sums over stored rows are cut)
    if (piece) finish_tile<T, float, 8, 4, 4, false>(as_piece(g, piece), 0, w.lo + wm, w.hi, w.n0 + wn, acc, room);
    else finish_tile<T, T, 8, 4, 4, true>(g, w.z, w.lo + wm, w.hi, w.n0 + wn, acc, room);
    if (odd) {
      f32x4 whole[8] = {};
      row_sums<T>(a, g.lda, w.hi - w.lo, K, wm, whole);
#pragma unroll
      for (int x = 0; x < 8; ++x)
        if (lane < 16) give_sum(w.lo + wm + 16 * x + lane, whole[x][0]);
    }
  } else {
    finish_tile<T, T, 8, 4, 4, true>(g, w.z, w.lo + wm, w.hi, w.n0 + wn, acc, room);
  }
}

template <class T> tt_status launch(const TTGemm &g, void *partial, hipStream_t s) {
  const long long n_tiles = tt_ceil_div(g.N, E);
  const long long m_tiles = g.mode == TT_GEMM_RAGGED_M ? (long long)tt_ceil_div(g.M, E) + g.batch + 1 : tt_ceil_div(g.M, E);
  const int chunk = ttk_gemm_direct_chunk(g);
  const long long members = g.mode == TT_GEMM_RAGGED_M ? 1 : chunk ? (long long)tt_ceil_div(g.K, chunk) + g.batch : g.batch;
  if (m_tiles * n_tiles > TT_MAX_WORKGROUPS / 2 || m_tiles * n_tiles * members > TT_MAX_WORKGROUPS / 2 || members > 65535) return TT_ERR_SHAPE;
  if (chunk && !partial) return TT_ERR_WORKSPACE;
  const dim3 grid((unsigned)(m_tiles * n_tiles), (unsigned)members);
  const int mti = (int)m_tiles, nti = (int)n_tiles;
  float *part = (float *)partial;
  if (g.a_kc && g.b_kc) hipLaunchKernelGGL((k_gemm_direct<T, true, true>), grid, dim3(THREADS), 0, s, g, mti, nti, chunk, part);
  else if (g.a_kc) hipLaunchKernelGGL((k_gemm_direct<T, true, false>), grid, dim3(THREADS), 0, s, g, mti, nti, chunk, part);
  else hipLaunchKernelGGL((k_gemm_direct<T, false, false>), grid, dim3(THREADS), 0, s, g, mti, nti, chunk, part);
  const tt_status st = tt_launch_status();
  return st == TT_OK && chunk ? ttk_gemm_join_groups(g, chunk, BK, part, s) : st;
}

}  // namespace

// Tiles of 256 from which they are taken: a workgroup fills a compute unit, and fewer leave too many without.  bf16, these / tiles of 128
// and 64, us: 2048 x 2048 x 2048 (64 tiles) 52 / 46, 2048 x 4096 x 1024 (128) 33 / 32, 4096 x 2560 x 1024 (160) 35 / 52, 4096 x 4096 x 1024
// (256) 37 / 61; 64 weights of 1024 x 1024 over 32768 uneven rows 146 / 204.
#ifndef TT_GEMM_DIRECT_TILES
#define TT_GEMM_DIRECT_TILES 144
#endif
#ifndef TT_GEMM_DIRECT_LEAST
#define TT_GEMM_DIRECT_LEAST 128  // of a side of out
#endif
bool ttk_gemm_direct_serves(const TTGemm &g) {
  if (g.dtype == TT_F32 || g.out_dtype != g.dtype || g.symmetric) return false;
  const uintptr_t addresses = (uintptr_t)g.a | (uintptr_t)g.b;
  if ((addresses & 15) || ((g.lda | g.ldb | g.a_step | g.b_step) & 7)) return false;
  if (((g.a_kc || g.b_kc) && (g.K & 7)) || (!g.a_kc && (g.M & 7)) || (!g.b_kc && (g.N & 7))) return false;
  if (g.lda > (1 << 23) || g.ldb > (1 << 23)) return false;  // offsets within a tile are 32 bits
  // half a tile would be empty
  if ((g.mode != TT_GEMM_RAGGED_M && g.M <= TT_GEMM_DIRECT_LEAST) || (g.like_N ? g.like_N : g.N) <= TT_GEMM_DIRECT_LEAST) return false;
  const long long tiles = (long long)tt_ceil_div(g.M, E) * tt_ceil_div(g.like_N ? g.like_N : g.N, E) * (g.mode == TT_GEMM_RAGGED_M ? 1 : g.batch);
  return tiles >= TT_GEMM_DIRECT_TILES;
}

int ttk_gemm_direct_chunk(const TTGemm &g) { return g.mode == TT_GEMM_RAGGED_K ? ttk_gemm_chunk(g, E, BK, 64) : 0; }
size_t ttk_gemm_direct_bytes(const TTGemm &g) { return g.mode == TT_GEMM_RAGGED_K && g.dtype != TT_F32 ? ttk_gemm_chunk_bytes(g, ttk_gemm_direct_chunk(g)) : 0; }
tt_status ttk_gemm_direct(const TTGemm &g, void *partial, hipStream_t s) {
  return g.dtype == TT_BF16 ? launch<ttg::bf16>(g, partial, s) : launch<ttg::f16>(g, partial, s);
}
