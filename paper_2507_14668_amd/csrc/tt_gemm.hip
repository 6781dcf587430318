// Matrix products with an epilogue on the matrix cores (fp32, bf16, fp16 operands; fp32 sums).
#include "tt_gemm_device.h"

namespace {
using namespace ttg;

// ---- the general kernel ----------------------------------------------------------------------------
// 64 x 64 of out per workgroup, four wavefronts of 32 x 32, operands through registers into LDS: any size, any row step, any
// alignment down to the element's.  16 bytes of an operand per thread and step; elements outside are zeros.
// The product is formed as out^T (B's rows are the instruction's M side), so that a lane's four results are neighbours in a row of out.
constexpr int GT = 64;                                                // tile edge
template <class T> struct Geo { static constexpr int E = 16 / sizeof(T), TK = 4 * E; };  // elements in 16 bytes; K of a step
template <class T, bool KC> struct Lds {
  // [64 rows][TK + pad] or [TK][64 + pad]; pads keep rows 8- / 16-byte aligned and spread them over the banks
  static constexpr int LD = KC ? Geo<T>::TK + Geo<T>::E : GT + 8;
  static constexpr int SIZE = KC ? GT * LD : Geo<T>::TK * LD;
};

// 16 bytes of an operand: chunk `c` (0..255) of the step at k0.  row0, rows: first row of the tile and the rows there are.
template <class T, bool KC>
__device__ __forceinline__ typename Vec<T>::v16b load_chunk(const T *base, long long ld, int row0, int rows, int k0, int K, int c) {
  constexpr int E = Geo<T>::E;
  const int major = KC ? row0 + c / 4 : k0 + c / (GT / E), minor = KC ? k0 + (c % 4) * E : row0 + (c % (GT / E)) * E;
  const int nmajor = KC ? rows : K, nminor = KC ? K : rows;
  typename Vec<T>::v16b v;
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = 0;
  if (major >= nmajor || minor >= nminor) return v;
  const T *p = base + (long long)major * ld + minor;
  if (nminor - minor >= E) return *reinterpret_cast<const typename Vec<T>::v16b *>(p);
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (i < nminor - minor) {
      if constexpr (sizeof(T) == 4) v[i] = p[i];
      else v[i] = __builtin_bit_cast(unsigned short, p[i]);
    }
  return v;
}
template <class T, bool KC>
__device__ __forceinline__ void store_chunk(T *lds, typename Vec<T>::v16b v, int c) {
  constexpr int E = Geo<T>::E, LD = Lds<T, KC>::LD;
  const int o = KC ? (c / 4) * LD + (c % 4) * E : (c / (GT / E)) * LD + (c % (GT / E)) * E;
  typedef unsigned u4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<u4 *>(lds + o) = __builtin_bit_cast(u4, v);
}
// The lane's elements of the 16 rows at r0: k = 8 (lane / 16) + i (16-bit), or k = 4 (lane / 16) + j for four steps j (fp32)
template <class T, bool KC>
__device__ __forceinline__ u16x8 frag16(const T *lds, int r0) {
  constexpr int LD = Lds<T, KC>::LD;
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15;
  if constexpr (KC) return *reinterpret_cast<const u16x8 *>(lds + (r0 + j) * LD + 8 * q);
  const unsigned short *p = reinterpret_cast<const unsigned short *>(lds) + (8 * q + (j >> 2)) * LD + r0 + 4 * (j & 3);
  const u16x4 x = lds_read_tr(p), y = lds_read_tr(p + 4 * LD);
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <bool KC>
__device__ __forceinline__ f32x4 frag32(const float *lds, int r0) {
  constexpr int LD = Lds<float, KC>::LD;
  const int lane = threadIdx.x & 63, q = lane >> 4, j = lane & 15;
  if constexpr (KC) return *reinterpret_cast<const f32x4 *>(lds + (r0 + j) * LD + 4 * q);
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = lds[(4 * q + i) * LD + r0 + j];
  return v;
}

struct Tile {
  int z, lo, hi, n0, k_lo, k_hi;  // member / group; rows [lo, hi) of out; first column; stored rows of K (RAGGED_K), else [0, K)
};

// out[m][n .. n + 3] from four sums
template <class T, class O>
__device__ __forceinline__ void epilogue4(const TTGemm &g, int z, int m, int n, const f32x4 &acc) {
  const int valid = g.N - n < 4 ? g.N - n : 4;
  float v[4], t[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = g.alpha * acc[i];
  if (g.bias) {
    load4((const T *)g.bias + z * g.bias_step + n, valid, t);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += t[i];
  }
  if (g.pre) {
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = keep_sign<O>(v[i]);
    store4((O *)g.pre + z * g.p_step + (long long)m * g.ldp + n, valid, t);
  }
  if (g.act != TT_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = act_value(v[i], g.act);
  }
  if (g.res) {
    load4((const T *)g.res + z * g.r_step + (long long)m * g.ldr + n, valid, t);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += g.beta * t[i];
  }
  store4((O *)g.out + z * g.o_step + (long long)m * g.ldo + n, valid, v);
}

template <class T, class O, bool AKC, bool BKC>
__global__ void __launch_bounds__(TT_BLOCK) k_gemm(TTGemm g, int m_tiles, int n_tiles) {
  constexpr int TK = Geo<T>::TK;
  __shared__ __align__(16) T la[Lds<T, AKC>::SIZE];
  __shared__ __align__(16) T lb[Lds<T, BKC>::SIZE];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // column tiles fastest: workgroups in flight share rows of A
  const int n0 = (int)(blockIdx.x % (unsigned)n_tiles) * GT;
  const unsigned rest = blockIdx.x / (unsigned)n_tiles;
  int z, lo, hi, K = g.K, k_lo = 0;
  if (g.mode == TT_GEMM_RAGGED_M) {
    const int t = (int)rest, there = find_tile<GT>(g.offsets, g.batch, g.M, t, z, lo, hi);
    if (z < 0) {  // a tile behind the last one: the rows that no group covers are dealt to these
      if (!g.zero_rest) return;
      const int above = lo, below = g.M - hi, idx = t - there, n = m_tiles - there;
      const float zero[4] = {0.f, 0.f, 0.f, 0.f};
      const int nn = n0 + 4 * (tid & 15), valid = g.N - nn < 4 ? g.N - nn : 4;
      for (long long r = (long long)idx * 16 + (tid >> 4); r < (long long)above + below; r += (long long)n * 16)
        if (valid > 0) store4((O *)g.out + (r < above ? r : r - above + hi) * g.ldo + nn, valid, zero);
      return;
    }
  } else {
    z = (int)(rest / (unsigned)m_tiles);
    lo = (int)(rest % (unsigned)m_tiles) * GT;
    hi = g.M < lo + GT ? g.M : lo + GT;
    if (g.mode == TT_GEMM_RAGGED_K) {
      int k_hi;
      group_rows(g.offsets, z, g.K, k_lo, k_hi);
      K = k_hi - k_lo;
    }
  }
  const bool ragged_k = g.mode == TT_GEMM_RAGGED_K;
  const T *a = (const T *)g.a + (g.mode == TT_GEMM_BATCH ? z * g.a_step : ragged_k ? (long long)k_lo * g.lda : 0);
  const T *b = (const T *)g.b + (ragged_k ? (long long)k_lo * g.ldb : z * g.b_step);

  const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32, q = lane >> 4, j = lane & 15;
  f32x4 acc[2][2] = {}, rs[2] = {};  // [m][n]; sums of A's rows
  const bool sums = g.rowsum && n0 == 0;
  typename Vec<T>::v16b va = load_chunk<T, AKC>(a, g.lda, lo, hi, 0, K, tid), vb = load_chunk<T, BKC>(b, g.ldb, n0, g.N, 0, K, tid);
  for (int k0 = 0; k0 < K; k0 += TK) {
    __syncthreads();
    store_chunk<T, AKC>(la, va, tid);
    store_chunk<T, BKC>(lb, vb, tid);
    __syncthreads();
    if (k0 + TK < K) {
      va = load_chunk<T, AKC>(a, g.lda, lo, hi, k0 + TK, K, tid);
      vb = load_chunk<T, BKC>(b, g.ldb, n0, g.N, k0 + TK, K, tid);
    }
    if constexpr (sizeof(T) == 2) {
      u16x8 fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = frag16<T, AKC>(la, wm + 16 * i);
        fb[i] = frag16<T, BKC>(lb, wn + 16 * i);
      }
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) acc[x][y] = mma(T(), fb[y], fa[x], acc[x][y]);
      if (sums) {
        u16x8 ones;
#pragma unroll
        for (int i = 0; i < 8; ++i) ones[i] = __builtin_bit_cast(unsigned short, (T)1.f);
#pragma unroll
        for (int x = 0; x < 2; ++x) rs[x] = mma(T(), ones, fa[x], rs[x]);
      }
    } else {
      f32x4 fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = frag32<AKC>(la, wm + 16 * i);
        fb[i] = frag32<BKC>(lb, wn + 16 * i);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
          for (int y = 0; y < 2; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[y][i], fa[x][i], acc[x][y], 0, 0, 0);
          if (sums) rs[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(1.f, fa[x][i], rs[x], 0, 0, 0);
        }
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int m = lo + wm + 16 * x + j;
    if (m >= hi) continue;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int n = n0 + wn + 16 * y + 4 * q;
      if (n < g.N) epilogue4<T, O>(g, z, m, n, acc[x][y]);
    }
    if (sums && wn == 0 && q == 0) ((O *)g.rowsum)[z * g.rs_step + m] = from_f32<O>(rs[x][0]);
  }
}

template <class T, class O>
void launch_general(const TTGemm &g, unsigned blocks, int m_tiles, int n_tiles, hipStream_t s) {
  if (g.a_kc && g.b_kc)
    hipLaunchKernelGGL((k_gemm<T, O, true, true>), dim3(blocks), dim3(TT_BLOCK), 0, s, g, m_tiles, n_tiles);
  else if (g.a_kc)
    hipLaunchKernelGGL((k_gemm<T, O, true, false>), dim3(blocks), dim3(TT_BLOCK), 0, s, g, m_tiles, n_tiles);
  else
    hipLaunchKernelGGL((k_gemm<T, O, false, false>), dim3(blocks), dim3(TT_BLOCK), 0, s, g, m_tiles, n_tiles);
}

}  // namespace

tt_status ttk_gemm(const TTGemm &g, hipStream_t s) {
  if (g.M < 1 || g.N < 1 || g.batch < 1) return TT_OK;
  const long long n_tiles = tt_ceil_div(g.N, GT);
  // every group ends in at most one part tile; one more for the rows outside the groups
  const long long m_tiles = g.mode == TT_GEMM_RAGGED_M ? (long long)tt_ceil_div(g.M, GT) + g.batch + 1 : tt_ceil_div(g.M, GT);
  const long long members = g.mode == TT_GEMM_RAGGED_M ? 1 : g.batch;
  if (m_tiles * members > TT_MAX_WORKGROUPS || m_tiles * members * n_tiles > TT_MAX_WORKGROUPS) return TT_ERR_SHAPE;
  const unsigned blocks = (unsigned)(m_tiles * members * n_tiles);
  if (!g.a_kc && g.b_kc) return TT_ERR_INVALID_ARG;  // no caller needs it
  if (g.dtype == TT_F32 && g.out_dtype == TT_F32) launch_general<float, float>(g, blocks, (int)m_tiles, (int)n_tiles, s);
  else if (g.dtype == TT_F32 && g.out_dtype == TT_BF16) launch_general<float, ttg::bf16>(g, blocks, (int)m_tiles, (int)n_tiles, s);
  else if (g.dtype == TT_F32 && g.out_dtype == TT_F16) launch_general<float, ttg::f16>(g, blocks, (int)m_tiles, (int)n_tiles, s);
  else if (g.dtype == TT_BF16 && g.out_dtype == TT_BF16) launch_general<ttg::bf16, ttg::bf16>(g, blocks, (int)m_tiles, (int)n_tiles, s);
  else if (g.dtype == TT_F16 && g.out_dtype == TT_F16) launch_general<ttg::f16, ttg::f16>(g, blocks, (int)m_tiles, (int)n_tiles, s);
  else return TT_ERR_INVALID_ARG;
  return tt_launch_status();
}
