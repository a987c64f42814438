// Products with few columns to a group: decoding steps, and both halves of a low-rank adapter.
//
// Such a product reads its large operand once and does 2 n flop for every value of it, n columns: it is bound by memory
// (n <= 32: at most 64 flop for 4 bytes, where the chip has 33 FP32 flop on the matrix unit for every byte that a copy
// moves per second).  Splitting would add nothing, so the FP32 matrix instruction multiplies the values as they are:
// v_mfma_f32_16x16x4_f32, 16 rows and 16 columns, four of the depth.  The result is at least as exact as either mode's,
// values far from 1, infinities and NaN included.  What is arranged is the traffic:
//   * a block takes 16 rows (64 where rows are contiguous) and all the group's columns, its eight waves share the depth
//     between them, each taking every eighth stretch, so that the block reads runs of 2 KiB of every row; the eight sums
//     meet in LDS and are added in order.
//   * lane l of a wave has row and column l % 16 and takes a float4 of the depth at 4 (l / 16): element e of it is that
//     lane's part of instruction e, for either operand, so both are read 16 bytes at a time and need no rearrangement.
//   * two stretches are in flight in registers while a third one is multiplied.
#pragma once
#include "grouped_kernel.hpp"

namespace ecgemm {

typedef float narrow_acc_t __attribute__((ext_vector_type(4)));
constexpr int kNarrowWaves = 8, kNarrowThreads = 64 * kNarrowWaves;
constexpr int kNarrowColumns = 32;  // of one pass over the rows

// What one wave adds up: rows of S (FR blocks of 16) times columns of T (NF blocks of 16).  S(r, k) = s[k + r lds] (S_DEPTH) or
// s[r + k lds]; T(c, k) alike.  Which row lane l's element v of acc[f][.] belongs to: row_of.
template <bool S_DEPTH, bool T_DEPTH, int FR, int NF>
struct WaveProduct {
  static_assert(S_DEPTH || FR == 4, "rows contiguous: four rows a load");
  static constexpr int STRETCH = S_DEPTH && FR == 1 ? (T_DEPTH && NF == 1 ? 64 : 32) : 16;  // of the depth per step
  static constexpr int QUADS = STRETCH / 16;
  const float* s;
  const float* t;
  int64_t lds, ldt, K;
  int rows, cols;  // that exist, at least 1
  int lane;
  struct Values {
    float s[FR][QUADS][4], t[NF][QUADS][4];  // S_DEPTH: [row block][..][e]; else [u][..][e] of rows 4 (l % 16) + u
  };

  __device__ __forceinline__ static int row_of(int f, int v, int lane) { return S_DEPTH ? 16 * f + 4 * (lane >> 4) + v : 16 * (lane >> 4) + 4 * v + f; }

  __device__ __forceinline__ int64_t k_of(int64_t k0, int q) const { return k0 + 16 * q + 4 * (lane >> 4); }
  __device__ __forceinline__ int row(int f) const {
    const int r = S_DEPTH ? 16 * f + (lane & 15) : 4 * (lane & 15) + f;
    return r < rows ? r : rows - 1;
  }
  __device__ __forceinline__ int column(int n) const {
    const int c = 16 * n + (lane & 15);
    return c < cols ? c : cols - 1;
  }
  // the stretch from k0 on (the same for the wave), which lies inside the depth; rows contiguous: all 64 rows exist.  Buffer
  // loads: a scalar base, an offset per lane that never changes, and a scalar offset per load.
  __device__ __forceinline__ void fetch(Values& x, int64_t k0) const {
    const auto from_s = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(s + (S_DEPTH ? k0 : k0 * lds)), 0, -1, 0x00020000);
    const auto from_t = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(t + (T_DEPTH ? k0 : k0 * ldt)), 0, -1, 0x00020000);
    const int s_step = (int)(4 * lds), t_step = (int)(4 * ldt), quad = 4 * (lane >> 4);
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
      if constexpr (S_DEPTH) {
#pragma unroll
        for (int f = 0; f < FR; ++f) {
          const source4_t v = __builtin_bit_cast(source4_t, __builtin_amdgcn_raw_buffer_load_b128(from_s, (int)((row(f) * lds + quad) * 4) + 64 * q, 0, 0));
#pragma unroll
          for (int e = 0; e < 4; ++e) x.s[f][q][e] = v[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const source4_t v = __builtin_bit_cast(source4_t, __builtin_amdgcn_raw_buffer_load_b128(from_s, (int)((4 * (lane & 15) + quad * lds) * 4), (16 * q + e) * s_step, 0));
#pragma unroll
          for (int f = 0; f < FR; ++f) x.s[f][q][e] = v[f];
        }
      }
#pragma unroll
      for (int n = 0; n < NF; ++n) {
        if constexpr (T_DEPTH) {
          const source4_t v = __builtin_bit_cast(source4_t, __builtin_amdgcn_raw_buffer_load_b128(from_t, (int)((column(n) * ldt + quad) * 4) + 64 * q, 0, 0));
#pragma unroll
          for (int e = 0; e < 4; ++e) x.t[n][q][e] = v[e];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x.t[n][q][e] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from_t, (int)((column(n) + quad * ldt) * 4), (16 * q + e) * t_step, 0));
        }
      }
    }
  }
  // any stretch, value by value: zero behind the depth
  __device__ __forceinline__ void fetch_any(Values& x, int64_t k0) const {
#pragma unroll
    for (int q = 0; q < QUADS; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t k = k_of(k0, q) + e;
        const bool inside = k < K;
#pragma unroll
        for (int f = 0; f < FR; ++f) x.s[f][q][e] = inside ? s[S_DEPTH ? row(f) * lds + k : row(f) + k * lds] : 0.0f;
#pragma unroll
        for (int n = 0; n < NF; ++n) x.t[n][q][e] = inside ? t[T_DEPTH ? column(n) * ldt + k : column(n) + k * ldt] : 0.0f;
      }
  }
  __device__ __forceinline__ static void multiply(const Values& x, narrow_acc_t (&acc)[FR][NF]) {
#pragma unroll
    for (int q = 0; q < QUADS; ++q)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int f = 0; f < FR; ++f)
#pragma unroll
          for (int n = 0; n < NF; ++n) acc[f][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(x.s[f][q][e], x.t[n][q][e], acc[f][n], 0, 0, 0);
  }
  // adds stretches first, first + step, ... to acc (all in units of STRETCH)
  __device__ __forceinline__ void run(narrow_acc_t (&acc)[FR][NF], int64_t first, int64_t step) const {
    const int64_t whole = S_DEPTH || rows >= 64 ? K / STRETCH : 0, all = (K + STRETCH - 1) / STRETCH;
    int64_t i = first;
    if (i < whole) {
      Values x[2];
      fetch(x[0], i * STRETCH);
      if (i + step < whole) fetch(x[1], (i + step) * STRETCH);
      for (; i + 3 * step < whole; i += 2 * step) {
        multiply(x[0], acc);
        fetch(x[0], (i + 2 * step) * STRETCH);
        multiply(x[1], acc);
        fetch(x[1], (i + 3 * step) * STRETCH);
      }
      multiply(x[0], acc);
      i += step;
      if (i < whole) {
        multiply(x[1], acc);
        i += step;
      }
      if (i < whole) {
        fetch(x[0], i * STRETCH);
        multiply(x[0], acc);
        i += step;
      }
    }
    for (; i < all; i += step) {
      Values x;
      fetch_any(x, i * STRETCH);
      multiply(x, acc);
    }
  }
};

// The block's sums over the whole depth, in `sums`[column][row] (ROWS + 1 apart): all waves' partial sums in order.
template <bool S_DEPTH>
constexpr int narrow_rows() { return S_DEPTH ? 16 : 64; }
template <bool S_DEPTH>
struct NarrowSums {
  float of_wave[kNarrowWaves][kNarrowColumns][narrow_rows<S_DEPTH>() + 1];
};
template <bool S_DEPTH, bool T_DEPTH, int NF>
__device__ __forceinline__ void narrow_pass(const float* s, int64_t lds, int rows, const float* t, int64_t ldt, int cols, int64_t K,
                                            NarrowSums<S_DEPTH>& sums) {
  constexpr int FR = S_DEPTH ? 1 : 4;
  typedef WaveProduct<S_DEPTH, T_DEPTH, FR, NF> Product;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  narrow_acc_t acc[FR][NF];
#pragma unroll
  for (int f = 0; f < FR; ++f)
#pragma unroll
    for (int n = 0; n < NF; ++n) acc[f][n] = narrow_acc_t{0.0f, 0.0f, 0.0f, 0.0f};
  const Product product{s, t, lds, ldt, K, rows, cols, lane};
  product.run(acc, wave, kNarrowWaves);
#pragma unroll
  for (int f = 0; f < FR; ++f)
#pragma unroll
    for (int n = 0; n < NF; ++n)
#pragma unroll
      for (int v = 0; v < 4; ++v) sums.of_wave[wave][16 * n + (lane & 15)][Product::row_of(f, v, lane)] = acc[f][n][v];
}
// ends with a barrier; element (row, column) is then narrow_sum(...)
template <bool S_DEPTH, bool T_DEPTH>
__device__ __forceinline__ void narrow_block(const float* s, int64_t lds, int rows, const float* t, int64_t ldt, int cols, int64_t K,
                                             NarrowSums<S_DEPTH>& sums) {
  __syncthreads();  // the sums of the pass before have been read
  if (cols > 16) narrow_pass<S_DEPTH, T_DEPTH, 2>(s, lds, rows, t, ldt, cols, K, sums);
  else narrow_pass<S_DEPTH, T_DEPTH, 1>(s, lds, rows, t, ldt, cols, K, sums);
  __syncthreads();
}
template <bool S_DEPTH>
__device__ __forceinline__ float narrow_sum(const NarrowSums<S_DEPTH>& sums, int row, int column) {
  float c = 0.0f;
#pragma unroll
  for (int w = 0; w < kNarrowWaves; ++w) c += sums.of_wave[w][column][row];
  return c;
}

struct NarrowParams {
  const float* A;  // as in GroupedParams; A is the operand that is read once
  const float* B;
  int64_t lda, ldb, ldc, stride_a, M, N, K;
  const int64_t* offsets;  // null: one group of all columns
  int64_t groups;
  const int* index;
  int matrices;
  float alpha, beta;
  float* C;
  int row_blocks;
  int clear_outside;  // C = 0 in the columns of no group (blocks groups row_blocks .. of the grid)
  // adapters only (else U is null): C += scales[a] op(U_a) H(:, j) for the columns j of an adapter's groups
  const float* U;
  int64_t ldu, stride_u, rank;
  int u_depth;  // the rank is contiguous in U
  const float* H;
  int64_t ldh;
  const float* scales;
  const int64_t* adapter_offsets;
  int64_t adapter_groups;
};

// The adapter of each of `count` <= kNarrowColumns columns from `first` on, -1 for none; called by all threads, ends with a barrier.
__device__ __forceinline__ void find_adapters(const int64_t* offsets, int64_t groups, const int* index, int matrices, int64_t N, int64_t first,
                                              int count, int (&adapter)[kNarrowColumns], int threads) {
  if (threadIdx.x < kNarrowColumns) adapter[threadIdx.x] = -1;
  __syncthreads();
  for (int64_t g = threadIdx.x; g < groups; g += threads) {
    const int64_t begin = clamp_offset(offsets[g], 0, N), end = clamp_offset(offsets[g + 1], begin, N);
    if (begin < first + count && end > first && begin < end) {
      const int a = index[g];
      if (a >= 0 && a < matrices)
        for (int64_t j = begin > first ? begin : first; j < end && j < first + count; ++j) adapter[j - first] = a;
    }
  }
  __syncthreads();
}

// C(:, j) = alpha op(A_g) op(B)(:, j) + beta C(:, j) for the columns j of group g, at best a handful of them.  Block b: group
// b / row_blocks, rows narrow_rows (b % row_blocks) and on.
template <bool DEPTH_A, bool DEPTH_B>
__global__ void __launch_bounds__(kNarrowThreads, DEPTH_A && DEPTH_B ? 4 : 2) narrow_kernel(const NarrowParams p) {
  constexpr int ROWS = narrow_rows<DEPTH_A>();
  __shared__ NarrowSums<DEPTH_A> sums;
  __shared__ int adapter[kNarrowColumns];
  const int64_t group = blockIdx.x / (unsigned)p.row_blocks;
  const int64_t m0 = (int64_t)(blockIdx.x % (unsigned)p.row_blocks) * ROWS;
  const int rows = (int)(p.M - m0 < ROWS ? p.M - m0 : ROWS);
  int64_t begin = 0, end = p.N;
  int matrix = 0;
  if (p.offsets != nullptr) {
    if (group >= p.groups) {  // columns in no group, before the first one and behind the last
      const int64_t first = clamp_offset(uniform(p.offsets[0]), 0, p.N), last = clamp_offset(uniform(p.offsets[p.groups]), first, p.N);
      for (int64_t i = threadIdx.x; i < (first + p.N - last) * rows; i += kNarrowThreads) {
        const int64_t j = i / rows;
        p.C[m0 + i % rows + (j < first ? j : j - first + last) * p.ldc] = 0.0f;
      }
      return;
    }
    begin = clamp_offset(uniform(p.offsets[group]), 0, p.N), end = clamp_offset(uniform(p.offsets[group + 1]), begin, p.N);
    matrix = (int)group;
    if (p.index != nullptr) {
      matrix = uniform(p.index[group]);
      if (matrix < 0 || matrix >= p.matrices) matrix = -1;
    }
  }
  const float* a = p.A + matrix * p.stride_a + (DEPTH_A ? m0 * p.lda : m0);
  for (int64_t n0 = begin; n0 < end; n0 += kNarrowColumns) {
    const int cols = (int)(end - n0 < kNarrowColumns ? end - n0 : kNarrowColumns);
    if (p.U != nullptr) find_adapters(p.adapter_offsets, p.adapter_groups, p.index, p.matrices, p.N, n0, cols, adapter, kNarrowThreads);
    narrow_block<DEPTH_A, DEPTH_B>(a, p.lda, rows, p.B + (DEPTH_B ? n0 * p.ldb : n0), p.ldb, cols, matrix >= 0 ? p.K : 0, sums);
    for (int i = threadIdx.x; i < ROWS * cols; i += kNarrowThreads) {
      const int r = i % ROWS, c = i / ROWS;
      if (r >= rows) continue;
      float value = p.alpha * narrow_sum<DEPTH_A>(sums, r, c);
      if (p.U != nullptr && adapter[c] >= 0) {
        const float* u = p.U + adapter[c] * p.stride_u + (p.u_depth ? (m0 + r) * p.ldu : m0 + r);
        const float* h = p.H + (n0 + c) * p.ldh;
        const int64_t u_step = p.u_depth ? 1 : p.ldu;
        float added = 0.0f;
#pragma unroll 8
        for (int64_t q = 0; q < p.rank; ++q) added = __builtin_fmaf(u[q * u_step], h[q], added);
        value = __builtin_fmaf(p.scales != nullptr ? p.scales[adapter[c]] : 1.0f, added, value);
      }
      float* dst = p.C + m0 + r + (n0 + c) * p.ldc;
      *dst = p.beta != 0.0f ? __builtin_fmaf(p.beta, *dst, value) : value;
    }
  }
}

// The first half of the adapters for many columns: H = op(D_a) op(B), the other way round: the columns of B, read once, are
// the rows of the product, and the rank its columns.  A block takes 16 columns of B (64 where they are contiguous) whichever
// groups they belong to, one pass for each adapter among them, and writes zero where there is none.
struct AdapterDownParams {
  const float* B;
  const float* D;
  int64_t ldb, ldd, stride_d, N, K, rank;
  const int64_t* offsets;
  int64_t groups;
  const int* index;
  int matrices;
  float* H;
  int64_t ldh;
};
template <bool DEPTH_B, bool DEPTH_D>
__global__ void __launch_bounds__(kNarrowThreads, DEPTH_B && DEPTH_D ? 4 : 2) adapter_down_kernel(const AdapterDownParams p) {
  constexpr int ROWS = narrow_rows<DEPTH_B>();
  __shared__ NarrowSums<DEPTH_B> sums;
  __shared__ int adapter[2][kNarrowColumns];
  const int64_t j0 = (int64_t)blockIdx.x * ROWS;
  const int rows = (int)(p.N - j0 < ROWS ? p.N - j0 : ROWS);
  for (int half = 0; half < (ROWS + kNarrowColumns - 1) / kNarrowColumns; ++half)
    find_adapters(p.offsets, p.groups, p.index, p.matrices, p.N, j0 + half * kNarrowColumns, kNarrowColumns, adapter[half], kNarrowThreads);
  auto adapter_of = [&](int r) { return adapter[r / kNarrowColumns][r % kNarrowColumns]; };
  for (int i = threadIdx.x; i < rows * (int)p.rank; i += kNarrowThreads)
    if (adapter_of(i / (int)p.rank) < 0) p.H[i % (int)p.rank + (j0 + i / (int)p.rank) * p.ldh] = 0.0f;
  for (int first = 0; first < rows;) {
    const int a = uniform(adapter_of(first));
    int last = first + 1;  // a run of columns with the same adapter
    while (last < rows && uniform(adapter_of(last)) == a) ++last;
    if (a >= 0) {
      const float* s = p.B + (DEPTH_B ? (j0 + first) * p.ldb : j0 + first);
      for (int64_t q0 = 0; q0 < p.rank; q0 += kNarrowColumns) {
        const int cols = (int)(p.rank - q0 < kNarrowColumns ? p.rank - q0 : kNarrowColumns);
        narrow_block<DEPTH_B, DEPTH_D>(s, p.ldb, last - first, p.D + a * p.stride_d + (DEPTH_D ? q0 * p.ldd : q0), p.ldd, cols, p.K, sums);
        for (int i = threadIdx.x; i < (last - first) * cols; i += kNarrowThreads) {
          const int c = i % cols, r = i / cols;
          p.H[q0 + c + (j0 + first + r) * p.ldh] = narrow_sum<DEPTH_B>(sums, r, c);
        }
      }
    }
    first = last;
  }
}

// The second half: C = scales[a] op(U_a) H + beta C in every column, before the projection is added.  A block takes 256 rows
// of C and 32 columns, a wave 64 rows; the depth is the rank.  Bound by writing C (and by reading it, unless beta is zero).
struct AdapterUpParams {
  const float* U;
  const float* H;
  int64_t ldu, stride_u, ldh, ldc, M, N, rank;
  const int64_t* offsets;
  int64_t groups;
  const int* index;
  int matrices;
  const float* scales;
  float beta;
  float* C;
  int row_blocks;
};
template <bool DEPTH_U>
__global__ void __launch_bounds__(256) adapter_up_kernel(const AdapterUpParams p) {
  __shared__ int adapter[kNarrowColumns];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)(blockIdx.x / (unsigned)p.row_blocks) * kNarrowColumns;
  const int64_t m0 = (int64_t)(blockIdx.x % (unsigned)p.row_blocks) * 256 + 64 * wave;
  const int cols = (int)(p.N - n0 < kNarrowColumns ? p.N - n0 : kNarrowColumns);
  find_adapters(p.offsets, p.groups, p.index, p.matrices, p.N, n0, cols, adapter, 256);
  if (m0 >= p.M) return;
  const int rows = (int)(p.M - m0 < 64 ? p.M - m0 : 64);
  typedef WaveProduct<DEPTH_U, true, 4, 2> Product;
  narrow_acc_t result[4][2];
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int n = 0; n < 2; ++n) result[f][n] = narrow_acc_t{0.0f, 0.0f, 0.0f, 0.0f};
  for (int first = 0; first < cols;) {
    const int a = uniform(adapter[first]);
    int last = first + 1;
    while (last < cols && uniform(adapter[last]) == a) ++last;
    if (a >= 0) {
      narrow_acc_t acc[4][2];
#pragma unroll
      for (int f = 0; f < 4; ++f)
#pragma unroll
        for (int n = 0; n < 2; ++n) acc[f][n] = narrow_acc_t{0.0f, 0.0f, 0.0f, 0.0f};
      const Product product{p.U + a * p.stride_u + (DEPTH_U ? m0 * p.ldu : m0), p.H + n0 * p.ldh, p.ldu, p.ldh, p.rank, rows, cols, lane};
      product.run(acc, 0, 1);
      const float scale = p.scales != nullptr ? p.scales[a] : 1.0f;
      // (a column takes the sums of its own adapter; what the others made of it is not looked at)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int c = 16 * n + (lane & 15);
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
          for (int v = 0; v < 4; ++v) result[f][n][v] = c >= first && c < last ? scale * acc[f][n][v] : result[f][n][v];
      }
    }
    first = last;
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int c = 16 * n + (lane & 15);
    if (c >= cols) continue;
    float* dst = p.C + m0 + (n0 + c) * p.ldc;
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int r = Product::row_of(f, v, lane);
        if (r < rows) dst[r] = p.beta != 0.0f ? __builtin_fmaf(p.beta, dst[r], result[f][n][v]) : result[f][n][v];
      }
  }
}

}  // namespace ecgemm
