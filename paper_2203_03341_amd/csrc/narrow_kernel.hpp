// Products with few columns to a group: decoding steps, and both halves of a low-rank adapter.
//
// Such a product reads its large operand once and does 2 n flop for every value of it, n columns: it is bound by memory
// (n <= 32: at most 64 flop for 4 bytes, where the chip has 33 FP32 flop on the matrix unit for every byte that a copy
// moves per second).  Splitting would add nothing, so the FP32 matrix instruction multiplies the values as they are:
// v_mfma_f32_16x16x4_f32, 16 rows and 16 columns, four of the depth.  Values far from 1, infinities and NaN need no care.  An
// element is off by at most 2^-24 of its products' magnitudes for each of the products that one wave adds up: an eighth of the
// depth here, all of it in shallow_kernel.  What is arranged is the traffic:
//   * a block takes 16 rows (64 where rows are contiguous) and all the group's columns, its eight waves share the depth
//     between them, each taking every eighth stretch, so that the block reads runs of 1 KiB of every row; the eight sums
//     meet in LDS and are added in order.
//   * an instruction takes row and column l % 16 from lane l.  Loads in that order have neighbouring lanes in different rows,
//     and the memory path takes 16 bytes a cycle then instead of 64 (4096 x 4096 times 32 columns 27 us, three quarters of
//     them that): where its depth is contiguous, an operand is read along it, eight lanes a row, and changes lanes in a part
//     of LDS that is the wave's own.
//   * lane l's float4 at 4 (l / 16) of a quad of 16 k is its part of four instructions, for either operand.
//   * two stretches are in flight in registers while a third one is multiplied.
// Measured: 64 groups of 2 columns, 1536 x 2048 each, 130 us, 6.2 TB/s; one of 4096 x 4096 13.3 us with up to 16 columns, 16.0
// with 32; eight of 768 x 1024 with 16 columns together 6.8.
#pragma once
#include "grouped_kernel.hpp"

namespace ecgemm {

typedef float narrow_acc_t __attribute__((ext_vector_type(4)));
typedef float float4_any_t __attribute__((ext_vector_type(4), aligned(4)));
constexpr int kNarrowColumns = 32;  // of one pass over the rows; twice that in adapter_down_kernel

// What one wave adds up: rows of S (FR blocks of 16) times columns of T (NF blocks of 16).  S(r, k) = s[k + r lds] (S_DEPTH) or
// s[r + k lds]; T(c, k) alike.  Which row lane l's element v of acc[f][.] belongs to: row_of.
// STORES, rows contiguous: the lanes' rows are dealt so that the sums a store takes lie next to each other, at the cost of loads
// whose neighbours do not (for products whose result is larger than their operands).
template <bool S_DEPTH, bool T_DEPTH, int FR, int NF, bool STORES = false>
struct WaveProduct {
  static_assert(S_DEPTH || FR == 4, "rows contiguous: four rows a load");
  static_assert(NF == 1 || NF == 2 || NF == 4, "columns contiguous: one load");
  static constexpr int STRETCH = S_DEPTH && FR <= 2 ? 32 : 16;  // of the depth per step
  static constexpr int QUADS = STRETCH / 16;
  // the wave's part of LDS: 16 FR rows of S and 16 NF columns of T, whichever of them have their depth contiguous, PITCH apart
  static constexpr int LANES = STRETCH / 4, AT_ONCE = 64 / LANES, PITCH = STRETCH + 4;  // lanes per row, rows per load
  static constexpr int S_LOADS = FR * 16 / AT_ONCE, T_LOADS = NF * 16 / AT_ONCE;
  static constexpr int SPACE = (S_DEPTH ? 16 * FR * PITCH : 0) + (T_DEPTH ? 16 * NF * PITCH : 0);  // floats

  const float* s;
  const float* t;
  int64_t lds, ldt, K;
  int rows, cols;  // that exist, at least 1
  int lane;
  float* space;
  struct Values {
    float s[S_DEPTH ? S_LOADS : FR][S_DEPTH ? 1 : QUADS][4];  // S_DEPTH: as loaded; else [u][quad][e] of rows 4 (l % 16) + u
    float t[T_DEPTH ? T_LOADS : NF][T_DEPTH ? 1 : QUADS][4];
  };

  __device__ __forceinline__ static int row_of(int f, int v, int lane) {
    return S_DEPTH ? 16 * f + 4 * (lane >> 4) + v : STORES ? 16 * v + 4 * (lane >> 4) + f : 16 * (lane >> 4) + 4 * v + f;
  }
  // rows contiguous: the first of the four rows that this lane loads
  __device__ __forceinline__ int quad_row() const { return 4 * (STORES ? 4 * (lane & 3) + (lane >> 2 & 3) : lane & 15); }
  // which column lane l's part of acc[.][n] belongs to: where columns are contiguous, a load takes NF of them
  __device__ __forceinline__ static int column_of(int n, int lane) { return T_DEPTH ? 16 * n + (lane & 15) : NF * (lane & 15) + n; }
  __device__ __forceinline__ int loaded_row(int j) const { return AT_ONCE * j + lane / LANES; }
  __device__ __forceinline__ static int clamped(int i, int count) { return i < count ? i : count - 1; }

  // the stretch from k0 on (the same for the wave), which lies inside the depth; rows or columns contiguous: as many as whole
  // loads take (a lane whose own do not exist reads the last ones that do).  Buffer loads: a scalar base, an offset per lane that never changes, and a scalar offset per load.
  __device__ __forceinline__ void fetch(Values& x, int64_t k0) const {
    const auto from_s = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(s + (S_DEPTH ? k0 : k0 * lds)), 0, -1, 0x00020000);
    const auto from_t = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(t + (T_DEPTH ? k0 : k0 * ldt)), 0, -1, 0x00020000);
    const int s_step = (int)(4 * lds), t_step = (int)(4 * ldt), quad = 4 * (lane >> 4), k_here = 4 * (lane % LANES);
    if constexpr (S_DEPTH) {
#pragma unroll
      for (int j = 0; j < S_LOADS; ++j) {
        const source4_t v = __builtin_bit_cast(source4_t, __builtin_amdgcn_raw_buffer_load_b128(from_s, (int)((clamped(loaded_row(j), rows) * lds + k_here) * 4), 0, 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) x.s[j][0][e] = v[e];
      }
    } else {
      const int first = quad_row(), at = (int)(((first < rows ? first : rows - 4) + quad * lds) * 4);
#pragma unroll
      for (int i = 0; i < 4 * QUADS; ++i) {
        const source4_t v = __builtin_bit_cast(source4_t, __builtin_amdgcn_raw_buffer_load_b128(from_s, at, (16 * (i / 4) + i % 4) * s_step, 0));
#pragma unroll
        for (int f = 0; f < FR; ++f) x.s[f][i / 4][i % 4] = v[f];
      }
    }
    if constexpr (T_DEPTH) {
#pragma unroll
      for (int j = 0; j < T_LOADS; ++j) {
        const source4_t v = __builtin_bit_cast(source4_t, __builtin_amdgcn_raw_buffer_load_b128(from_t, (int)((clamped(loaded_row(j), cols) * ldt + k_here) * 4), 0, 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) x.t[j][0][e] = v[e];
      }
    } else {
      const int first = NF * (lane & 15), at = (int)(((first < cols ? first : cols - NF) + quad * ldt) * 4);
#pragma unroll
      for (int i = 0; i < 4 * QUADS; ++i) {
        const int by = (16 * (i / 4) + i % 4) * t_step;
        if constexpr (NF == 1) {
          x.t[0][i / 4][i % 4] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(from_t, at, by, 0));
        } else if constexpr (NF == 2) {
          typedef float float2_t __attribute__((ext_vector_type(2)));
          const float2_t v = __builtin_bit_cast(float2_t, __builtin_amdgcn_raw_buffer_load_b64(from_t, at, by, 0));
          x.t[0][i / 4][i % 4] = v[0], x.t[1][i / 4][i % 4] = v[1];
        } else {
          const source4_t v = __builtin_bit_cast(source4_t, __builtin_amdgcn_raw_buffer_load_b128(from_t, at, by, 0));
#pragma unroll
          for (int f = 0; f < 4; ++f) x.t[f][i / 4][i % 4] = v[f];
        }
      }
    }
  }
  // any stretch, value by value: zero behind the depth
  __device__ __forceinline__ void fetch_any(Values& x, int64_t k0) const {
#pragma unroll
    for (int i = 0; i < (S_DEPTH ? S_LOADS : FR * QUADS); ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t k = k0 + e + (S_DEPTH ? 4 * (lane % LANES) : 16 * (i % QUADS) + 4 * (lane >> 4));
        const int r = clamped(S_DEPTH ? loaded_row(i) : quad_row() + i / QUADS, rows);
        x.s[S_DEPTH ? i : i / QUADS][S_DEPTH ? 0 : i % QUADS][e] = k < K ? s[S_DEPTH ? r * lds + k : r + k * lds] : 0.0f;
      }
#pragma unroll
    for (int i = 0; i < (T_DEPTH ? T_LOADS : NF * QUADS); ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t k = k0 + e + (T_DEPTH ? 4 * (lane % LANES) : 16 * (i % QUADS) + 4 * (lane >> 4));
        const int c = clamped(T_DEPTH ? loaded_row(i) : column_of(i / QUADS, lane), cols);
        x.t[T_DEPTH ? i : i / QUADS][T_DEPTH ? 0 : i % QUADS][e] = k < K ? t[T_DEPTH ? c * ldt + k : c + k * ldt] : 0.0f;
      }
  }
  __device__ __forceinline__ void multiply(const Values& x, narrow_acc_t (&acc)[FR][NF]) const {
    float* const s_space = space;
    float* const t_space = space + (S_DEPTH ? 16 * FR * PITCH : 0);
    // (a wave's LDS instructions are carried out in order: nothing but the compiler has to be kept from changing it)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    if constexpr (S_DEPTH)
#pragma unroll
      for (int j = 0; j < S_LOADS; ++j) *reinterpret_cast<narrow_acc_t*>(s_space + loaded_row(j) * PITCH + 4 * (lane % LANES)) = narrow_acc_t{x.s[j][0][0], x.s[j][0][1], x.s[j][0][2], x.s[j][0][3]};
    if constexpr (T_DEPTH)
#pragma unroll
      for (int j = 0; j < T_LOADS; ++j) *reinterpret_cast<narrow_acc_t*>(t_space + loaded_row(j) * PITCH + 4 * (lane % LANES)) = narrow_acc_t{x.t[j][0][0], x.t[j][0][1], x.t[j][0][2], x.t[j][0][3]};
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int q = 0; q < QUADS; ++q) {
      narrow_acc_t from_s[FR], from_t[NF];
#pragma unroll
      for (int f = 0; f < FR; ++f) {
        if constexpr (S_DEPTH) from_s[f] = *reinterpret_cast<const narrow_acc_t*>(s_space + (16 * f + (lane & 15)) * PITCH + 16 * q + 4 * (lane >> 4));
        else from_s[f] = narrow_acc_t{x.s[f][q][0], x.s[f][q][1], x.s[f][q][2], x.s[f][q][3]};
      }
#pragma unroll
      for (int n = 0; n < NF; ++n) {
        if constexpr (T_DEPTH) from_t[n] = *reinterpret_cast<const narrow_acc_t*>(t_space + (16 * n + (lane & 15)) * PITCH + 16 * q + 4 * (lane >> 4));
        else from_t[n] = narrow_acc_t{x.t[n][q][0], x.t[n][q][1], x.t[n][q][2], x.t[n][q][3]};
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int f = 0; f < FR; ++f)
#pragma unroll
          for (int n = 0; n < NF; ++n) acc[f][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(from_s[f][e], from_t[n][e], acc[f][n], 0, 0, 0);
    }
  }
  // Adds stretches first, first + step, ... to acc (all in units of STRETCH).  `turn` of 2^32 of the way through the depth is
  // where it begins, going on from the front when it comes to the end: blocks that start together would otherwise all read
  // the same columns of rows that lie a power of two apart, from a few of the memory's channels.
  __device__ __forceinline__ void run(narrow_acc_t (&acc)[FR][NF], int64_t first, int64_t step, unsigned turn) const {
    const bool vectors = (S_DEPTH || rows % 4 == 0) && (T_DEPTH || cols % NF == 0);
    const int64_t whole = vectors ? K / STRETCH : 0, all = (K + STRETCH - 1) / STRETCH;
    const int64_t begin = (int64_t)(((uint64_t)turn * (uint64_t)whole) >> 32);
    auto k_at = [&](int64_t stretch) {
      const int64_t turned = stretch + begin;
      return (turned < whole ? turned : turned - whole) * STRETCH;
    };
    int64_t i = first;
    if (i < whole) {
      Values x[2];
      fetch(x[0], k_at(i));
      if (i + step < whole) fetch(x[1], k_at(i + step));
      for (; i + 3 * step < whole; i += 2 * step) {
        // (kept in this order: a product drawn in front of the loads behind it would wait for all that is in flight)
        multiply(x[0], acc);
        __builtin_amdgcn_sched_barrier(0);
        fetch(x[0], k_at(i + 2 * step));
        __builtin_amdgcn_sched_barrier(0);
        multiply(x[1], acc);
        __builtin_amdgcn_sched_barrier(0);
        fetch(x[1], k_at(i + 3 * step));
        __builtin_amdgcn_sched_barrier(0);
      }
      multiply(x[0], acc);
      i += step;
      if (i < whole) {
        multiply(x[1], acc);
        i += step;
      }
      if (i < whole) {
        fetch(x[0], k_at(i));
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
template <bool S_DEPTH, bool T_DEPTH, int FR, bool WIDE>
union NarrowSums {
  float space[kNarrowWaves][WaveProduct<S_DEPTH, T_DEPTH, FR, WIDE ? 4 : 2>::SPACE + 4];  // while the waves multiply
  float of_wave[kNarrowWaves][WIDE ? 2 * kNarrowColumns : kNarrowColumns][16 * FR + 1];
};
template <bool S_DEPTH, bool T_DEPTH, int FR, int NF, bool WIDE>
__device__ __forceinline__ void narrow_pass(const float* s, int64_t lds, int rows, const float* t, int64_t ldt, int cols, int64_t K,
                                            NarrowSums<S_DEPTH, T_DEPTH, FR, WIDE>& sums) {
  typedef WaveProduct<S_DEPTH, T_DEPTH, FR, NF> Product;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  narrow_acc_t acc[FR][NF];
#pragma unroll
  for (int f = 0; f < FR; ++f)
#pragma unroll
    for (int n = 0; n < NF; ++n) acc[f][n] = narrow_acc_t{0.0f, 0.0f, 0.0f, 0.0f};
  const Product product{s, t, lds, ldt, K, rows, cols, lane, sums.space[wave]};
  product.run(acc, wave, kNarrowWaves, blockIdx.x * 0x9E3779B1u);
  __syncthreads();  // every wave is through with its space
#pragma unroll
  for (int f = 0; f < FR; ++f)
#pragma unroll
    for (int n = 0; n < NF; ++n)
#pragma unroll
      for (int v = 0; v < 4; ++v) sums.of_wave[wave][Product::column_of(n, lane)][Product::row_of(f, v, lane)] = acc[f][n][v];
}
// ends with a barrier; element (row, column) is then narrow_sum(...)
template <bool S_DEPTH, bool T_DEPTH, int FR, bool WIDE>
__device__ __forceinline__ void narrow_block(const float* s, int64_t lds, int rows, const float* t, int64_t ldt, int cols, int64_t K,
                                             NarrowSums<S_DEPTH, T_DEPTH, FR, WIDE>& sums) {
  __syncthreads();  // the sums of the pass before have been read
  if (WIDE && cols > 32) narrow_pass<S_DEPTH, T_DEPTH, FR, WIDE ? 4 : 2, WIDE>(s, lds, rows, t, ldt, cols, K, sums);
  else if (cols > 16) narrow_pass<S_DEPTH, T_DEPTH, FR, 2, WIDE>(s, lds, rows, t, ldt, cols, K, sums);
  else narrow_pass<S_DEPTH, T_DEPTH, FR, 1, WIDE>(s, lds, rows, t, ldt, cols, K, sums);
  __syncthreads();
}
template <bool S_DEPTH, bool T_DEPTH, int FR, bool WIDE>
__device__ __forceinline__ float narrow_sum(const NarrowSums<S_DEPTH, T_DEPTH, FR, WIDE>& sums, int row, int column) {
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
    const int a = index[g];
    if (begin < first + count && end > first && begin < end) {
      if (a >= 0 && a < matrices)
        for (int64_t j = begin > first ? begin : first; j < end && j < first + count; ++j) adapter[j - first] = a;
    }
  }
  __syncthreads();
}

// C(:, j) = alpha op(A_g) op(B)(:, j) + beta C(:, j) for the columns j of group g, at best a handful of them.  Block b: group
// b / row_blocks, rows narrow_rows (b % row_blocks) and on.
template <bool DEPTH_A, bool DEPTH_B, int FR>
__global__ void __launch_bounds__(kNarrowThreads, DEPTH_A && FR == 1 ? 4 : 2) narrow_kernel(const NarrowParams p) {
  constexpr int ROWS = 16 * FR;
  __shared__ __attribute__((aligned(16))) NarrowSums<DEPTH_A, DEPTH_B, FR, false> sums;
  __shared__ int adapter[kNarrowColumns];
  const int64_t group = blockIdx.x / (unsigned)p.row_blocks;
  // (rows contiguous: a last block that is not whole is moved back to be whole, for its loads, and writes what is its own;
  // four groups of 99 rows, 40 columns, depth 4096: 36 us with its rows read one by one, 24 so)
  const int64_t m_block = (int64_t)(blockIdx.x % (unsigned)p.row_blocks) * ROWS;
  const int64_t m0 = !DEPTH_A && p.M >= ROWS && m_block > p.M - ROWS ? p.M - ROWS : m_block;
  const int rows = (int)(p.M - m0 < ROWS ? p.M - m0 : ROWS), skip = (int)(m_block - m0);
  // (the offsets are read once for the block: all its waves pass the same barriers, whatever happens to them meanwhile)
  __shared__ int64_t range[2];
  __shared__ int chosen;
  if (threadIdx.x == 0) {
    range[0] = 0, range[1] = p.N, chosen = 0;
    if (p.offsets != nullptr) {
      const int64_t first = group < p.groups ? group : 0, last = group < p.groups ? group + 1 : p.groups;
      range[0] = clamp_offset(p.offsets[first], 0, p.N);
      range[1] = clamp_offset(p.offsets[last], range[0], p.N);
      if (group < p.groups) {
        chosen = (int)group;
        if (p.index != nullptr) {
          const int index = p.index[group];
          chosen = index >= 0 && index < p.matrices ? index : -1;
        }
      }
    }
  }
  __syncthreads();
  const int64_t begin = uniform(range[0]), end = uniform(range[1]);
  const int matrix = uniform(chosen);
  if (p.offsets != nullptr && group >= p.groups) {  // columns in no group, before the first one and behind the last
    for (int64_t i = threadIdx.x; i < (begin + p.N - end) * rows; i += kNarrowThreads) {
      const int64_t j = i / rows;
      p.C[m0 + i % rows + (j < begin ? j : j - begin + end) * p.ldc] = 0.0f;
    }
    return;
  }
  const float* a = p.A + matrix * p.stride_a + (DEPTH_A ? m0 * p.lda : m0);
  for (int64_t n0 = begin; n0 < end; n0 += kNarrowColumns) {
    const int cols = (int)(end - n0 < kNarrowColumns ? end - n0 : kNarrowColumns);
    if (p.U != nullptr) {
      __syncthreads();  // the adapters of the columns before are no longer looked at
      find_adapters(p.adapter_offsets, p.adapter_groups, p.index, p.matrices, p.N, n0, cols, adapter, kNarrowThreads);
    }
    narrow_block<DEPTH_A, DEPTH_B, FR, false>(a, p.lda, rows, p.B + (DEPTH_B ? n0 * p.ldb : n0), p.ldb, cols, matrix >= 0 ? p.K : 0, sums);
    for (int i = threadIdx.x; i < ROWS * cols; i += kNarrowThreads) {
      const int r = i % ROWS, c = i / ROWS;
      if (r >= rows || r < skip) continue;
      float value = p.K > 0 ? p.alpha * narrow_sum(sums, r, c) : 0.0f;
      if (p.U != nullptr && adapter[c] >= 0) {
        const float* u = p.U + adapter[c] * p.stride_u + (p.u_depth ? (m0 + r) * p.ldu : m0 + r);
        const float* h = p.H + (n0 + c) * p.ldh;
        const int64_t u_step = p.u_depth ? 1 : p.ldu;
        float added = 0.0f;
        int64_t q = 0;
        if (p.u_depth) {
#pragma unroll 4
          for (; q + 4 <= p.rank; q += 4) {
            const float4_any_t u4 = *reinterpret_cast<const float4_any_t*>(u + q), h4 = *reinterpret_cast<const float4_any_t*>(h + q);
#pragma unroll
            for (int e = 0; e < 4; ++e) added = __builtin_fmaf(u4[e], h4[e], added);
          }
        }
#pragma unroll 8
        for (; q < p.rank; ++q) added = __builtin_fmaf(u[q * u_step], h[q], added);
        value = __builtin_fmaf(p.scales != nullptr ? p.scales[adapter[c]] : 1.0f, added, value);
      }
      float* dst = p.C + m0 + r + (n0 + c) * p.ldc;
      *dst = p.beta != 0.0f ? __builtin_fmaf(p.beta, *dst, value) : value;
    }
  }
}

// The first half of the adapters for many columns: H = op(D_a) op(B), the other way round: the columns of B, read once, are
// the rows of the product, and the rank its columns.  A block takes 16 columns of B (64 where they are contiguous) whichever
// groups they belong to, one pass for each adapter among them, and writes zero where there is none.  The passes are dealt to
// gridDim.y blocks: with one, the blocks where two requests meet take twice the time of the others.
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
template <bool DEPTH_B, bool DEPTH_D, int FR>
__global__ void __launch_bounds__(kNarrowThreads, 2) adapter_down_kernel(const AdapterDownParams p) {
  constexpr int ROWS = 16 * FR;
  __shared__ __attribute__((aligned(16))) NarrowSums<DEPTH_B, DEPTH_D, FR, DEPTH_B> sums;
  __shared__ int adapter[2][kNarrowColumns];
  const int64_t j0 = (int64_t)xcd_run_position(blockIdx.x, gridDim.x) * ROWS;  // (an adapter is read by few of the L2s)
  const int rows = (int)(p.N - j0 < ROWS ? p.N - j0 : ROWS);
  for (int half = 0; half < (ROWS + kNarrowColumns - 1) / kNarrowColumns; ++half)
    find_adapters(p.offsets, p.groups, p.index, p.matrices, p.N, j0 + half * kNarrowColumns, kNarrowColumns, adapter[half], kNarrowThreads);
  auto adapter_of = [&](int r) { return adapter[r / kNarrowColumns][r % kNarrowColumns]; };
  if (blockIdx.y == 0)
    for (int i = threadIdx.x; i < rows * (int)p.rank; i += kNarrowThreads)
      if (adapter_of(i / (int)p.rank) < 0) p.H[i % (int)p.rank + (j0 + i / (int)p.rank) * p.ldh] = 0.0f;
  unsigned run = 0;
  for (int first = 0; first < rows;) {
    const int a = uniform(adapter_of(first));
    int last = first + 1;  // a run of columns with the same adapter
    while (last < rows && uniform(adapter_of(last)) == a) ++last;
    if (a >= 0 && run++ % gridDim.y == blockIdx.y) {
      const float* s = p.B + (DEPTH_B ? (j0 + first) * p.ldb : j0 + first);
      constexpr int AT_ONCE = DEPTH_B ? 2 * kNarrowColumns : kNarrowColumns;
      for (int64_t q0 = 0; q0 < p.rank; q0 += AT_ONCE) {
        const int cols = (int)(p.rank - q0 < AT_ONCE ? p.rank - q0 : AT_ONCE);
        narrow_block<DEPTH_B, DEPTH_D, FR, DEPTH_B>(s, p.ldb, last - first, p.D + a * p.stride_d + (DEPTH_D ? q0 * p.ldd : q0), p.ldd, cols, p.K, sums);
        for (int i = threadIdx.x; i < (last - first) * cols; i += kNarrowThreads) {
          const int c = i % cols, r = i / cols;
          p.H[q0 + c + (j0 + first + r) * p.ldh] = narrow_sum(sums, r, c);
        }
      }
    }
    first = last;
  }
}

// The second half: C = scales[a] op(U_a) H + beta C in every column, before the projection is added.  A block takes 256 rows
// of C and 64 columns (8 where there are few to a request), a wave 64 rows, run by run of columns with the same adapter; the
// depth is the rank.  Bound by writing C (and by reading it, unless beta is zero).
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
template <bool DEPTH_U, int COLUMNS>
__global__ void __launch_bounds__(kAdapterUpThreads) adapter_up_kernel(const AdapterUpParams p) {
  __shared__ int adapter[(COLUMNS + kNarrowColumns - 1) / kNarrowColumns][kNarrowColumns];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)(blockIdx.x / (unsigned)p.row_blocks) * COLUMNS;
  const int64_t m0 = (int64_t)(blockIdx.x % (unsigned)p.row_blocks) * kAdapterUpRows + 64 * wave;
  const int cols = (int)(p.N - n0 < COLUMNS ? p.N - n0 : COLUMNS);
  for (int i = 0; i * kNarrowColumns < cols; ++i)
    find_adapters(p.offsets, p.groups, p.index, p.matrices, p.N, n0 + i * kNarrowColumns, kNarrowColumns, adapter[i], kAdapterUpThreads);
  if (m0 >= p.M) return;
  const int rows = (int)(p.M - m0 < 64 ? p.M - m0 : 64);
  auto adapter_of = [&](int c) { return uniform(adapter[c / kNarrowColumns][c % kNarrowColumns]); };
  constexpr int NF = (COLUMNS + 15) / 16;
  typedef WaveProduct<DEPTH_U, true, 4, NF> Product;
  __shared__ __attribute__((aligned(16))) float space[4][Product::SPACE];
  for (int first = 0; first < cols;) {
    const int a = adapter_of(first);
    int last = first + 1;  // a run of columns with the same adapter
    while (last < cols && adapter_of(last) == a) ++last;
    narrow_acc_t acc[4][NF];
#pragma unroll
    for (int f = 0; f < 4; ++f)
#pragma unroll
      for (int n = 0; n < NF; ++n) acc[f][n] = narrow_acc_t{0.0f, 0.0f, 0.0f, 0.0f};
    float scale = 0.0f;
    if (a >= 0) {
      const Product product{p.U + a * p.stride_u + (DEPTH_U ? m0 * p.ldu : m0), p.H + (n0 + first) * p.ldh, p.ldu, p.ldh, p.rank, rows, last - first, lane, space[wave]};
      product.run(acc, 0, 1, 0);
      scale = p.scales != nullptr ? p.scales[a] : 1.0f;
    }
#pragma unroll
    for (int n = 0; n < NF; ++n) {
      const int c = 16 * n + (lane & 15);
      if (first + c >= last) continue;
      float* dst = p.C + m0 + (n0 + first + c) * p.ldc;
      // four rows next to each other: elements v of one block, or (rows of U contiguous) element v of four
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float4_any_t value;
#pragma unroll
        for (int u = 0; u < 4; ++u) value[u] = scale * (DEPTH_U ? acc[i][n][u] : acc[u][n][i]);
        const int r = DEPTH_U ? Product::row_of(i, 0, lane) : Product::row_of(0, i, lane);
        if (rows == 64) {
          float4_any_t* at = reinterpret_cast<float4_any_t*>(dst + r);
          if (p.beta != 0.0f) {
            const float4_any_t before = *at;
#pragma unroll
            for (int u = 0; u < 4; ++u) value[u] = __builtin_fmaf(p.beta, before[u], value[u]);
          }
          *at = value;
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (r + u < rows) dst[r + u] = p.beta != 0.0f ? __builtin_fmaf(p.beta, dst[r + u], value[u]) : value[u];
        }
      }
    }
    first = last;
  }
}

// C_g = alpha op(A)(:, k's of g) op(B)(k's of g, :) + beta C_g where the groups are shallow: a few flop for every value of C,
// bound by writing it (and reading it, unless beta is zero).  A block takes 256 rows and 64 columns of C, a wave 64 rows, and
// leaves room for others on its unit, which hide each other's way to memory; a tile of grouped_kernel has the unit to itself and takes 5 us
// however shallow it is.
struct ShallowParams {
  const float* A;
  const float* B;
  int64_t lda, ldb, ldc, stride_c, M, N, K;
  const int64_t* offsets;
  float alpha, beta;
  float* C;
  int row_blocks, column_blocks;
};
template <bool DEPTH_A, bool DEPTH_B>
__global__ void __launch_bounds__(kShallowThreads) shallow_kernel(const ShallowParams p) {
  constexpr int NF = kShallowColumns / 16;
  typedef WaveProduct<DEPTH_A, DEPTH_B, 4, NF, true> Product;
  __shared__ __attribute__((aligned(16))) float space[4][Product::SPACE + 4];
  __shared__ int64_t range[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned blocks = (unsigned)p.row_blocks * (unsigned)p.column_blocks;
  const int64_t group = blockIdx.x / blocks;
  const unsigned block = blockIdx.x % blocks;
  if (threadIdx.x == 0) {
    range[0] = clamp_offset(p.offsets[group], 0, p.K);
    range[1] = clamp_offset(p.offsets[group + 1], range[0], p.K);
  }
  __syncthreads();
  const int64_t begin = uniform(range[0]), depth = uniform(range[1]) - begin;
  const int64_t m0 = (int64_t)(block % (unsigned)p.row_blocks) * kShallowRows + 64 * wave, n0 = (int64_t)(block / (unsigned)p.row_blocks) * kShallowColumns;
  if (m0 >= p.M) return;
  const int rows = (int)(p.M - m0 < 64 ? p.M - m0 : 64), cols = (int)(p.N - n0 < kShallowColumns ? p.N - n0 : kShallowColumns);
  narrow_acc_t acc[4][NF];
#pragma unroll
  for (int f = 0; f < 4; ++f)
#pragma unroll
    for (int n = 0; n < NF; ++n) acc[f][n] = narrow_acc_t{0.0f, 0.0f, 0.0f, 0.0f};
  if (depth > 0) {
    const Product product{p.A + (DEPTH_A ? m0 * p.lda + begin : m0 + begin * p.lda), p.B + (DEPTH_B ? n0 * p.ldb + begin : n0 + begin * p.ldb), p.lda,
                          p.ldb, depth, rows, cols, lane, space[wave]};
    product.run(acc, 0, 1, 0);
  }
  const float alpha = depth > 0 ? p.alpha : 0.0f;
  float* c = p.C + group * p.stride_c + m0 + n0 * p.ldc;
#pragma unroll
  for (int n = 0; n < NF; ++n) {
    const int column = Product::column_of(n, lane);
    if (column >= cols) continue;
    float* dst = c + column * p.ldc;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float4_any_t value;
#pragma unroll
      for (int u = 0; u < 4; ++u) value[u] = alpha * (DEPTH_A ? acc[i][n][u] : acc[u][n][i]);
      const int r = DEPTH_A ? Product::row_of(i, 0, lane) : Product::row_of(0, i, lane);
      if (rows == 64) {
        float4_any_t* at = reinterpret_cast<float4_any_t*>(dst + r);
        if (p.beta != 0.0f) {
          const float4_any_t before = *at;
#pragma unroll
          for (int u = 0; u < 4; ++u) value[u] = __builtin_fmaf(p.beta, before[u], value[u]);
        }
        *at = value;  // (past the caches 73 us instead of 58: 64 groups of one row, 1024 x 768)
      } else {
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (r + u < rows) dst[r + u] = p.beta != 0.0f ? __builtin_fmaf(p.beta, dst[r + u], value[u]) : value[u];
      }
    }
  }
}

}  // namespace ecgemm
