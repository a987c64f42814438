// Products in groups: the method's steps 1 to 5 on the caller's FP32 operands, one launch for all groups.  Where the groups
// lie is known to the GPU only: `offsets`, groups + 1 entries in device memory, not decreasing.
//
//   columns (a layer of experts)   C(:, j) = alpha op(A_g) op(B)(:, j) + beta C(:, j)     for offsets[g] <= j < offsets[g + 1]
//   depth (its weights' gradient)  C_g = alpha op(A)(:, k's of g) op(B)(k's of g, :) + beta C_g
//
// The arrangement of a block is wide_kernel's: a tile of 128 x 128, four waves that fetch FP32 values and split them and
// beside them four that multiply, 64 x 64 of the tile each, chunks of the depth in two LDS buffers, one barrier per chunk.
// What is different:
//   * the grid is persistent, a block per compute unit.  The number of tiles is known on the GPU only, so a grid of one
//     block per tile would have to be launched for the worst case; and while the multiplying waves write a tile the
//     splitting waves already fetch the next one, which hides the first loads and the epilogue behind each other.
//   * every block makes the table of the groups' tiles for itself, from the offsets, before its first tile (1 to 2 us, where
//     a launch of its own would cost 4).
//   * rows and columns are clamped to the group, so a tile may hold any number of columns from 1 to 128, and a group's depth
//     may be anything from nothing on.
//   * both modes: three BF16 parts take chunks of 32 (96 KiB of LDS), two FP16 parts chunks of 64 (128 KiB).
// Measured: 1.47 us a chunk of 64 in FP16 mode with all units busy, 4 us a tile for the rest; 4096 cubed as one group 373 us,
// 368 FP32-equivalent TFLOP/s (BF16 598), eight groups of 1024 columns, 4096 x 2048, 400.  60 % of the cycles are matrix
// instructions, at 1.7 GHz: the board is at its power cap.
#pragma once
#include "grouped_sizes.hpp"
#include "wide_kernel.hpp"

namespace ecgemm {

constexpr int kGroupedThreads = 512, kGroupedSplitWaves = 4;
constexpr int kGroupsPerLaunch = 1024;             // the table of the groups lies in LDS; more groups are more launches
constexpr int kGroupedTilesPerBlock = 1024;        // most tiles a block walks through (a byte of LDS per tile and wave)
constexpr int64_t kGroupedLargestLd = (int64_t)1 << 21;  // a chunk's values lie within 2^30 bytes of its first

constexpr int64_t kLargestRank = 1024;             // of an adapter

struct GroupedParams {
  const float* A;  // device, column-major
  const float* B;
  int64_t lda, ldb, ldc;
  int64_t stride_a;  // columns: from one group's A to the next one's; depth: 0
  int64_t stride_c;  // depth: from one group's C to the next one's; columns: 0
  int64_t M, N, K;   // columns: N is the number of columns of B and C; depth: K is the depth of A and B
  const int64_t* offsets;
  int groups;        // at most kGroupsPerLaunch
  int along_depth;   // 1: groups of the depth, 0: groups of columns
  int tiles_m, tiles_n;  // tiles_n: not for columns
  // ADAPTERS only: tiles are of all N columns and tiles_n counts them; group g's columns have scales[a] op(U_a) H added,
  // a = index[g] if that is one of `matrices` (scales may be null: 1); H is rank x N with the rank contiguous
  const int* index;
  int matrices;
  const float* scales;
  const float* U;
  int64_t ldu, stride_u, rank;
  const float* H;
  int64_t ldh;
  // slices > 1 (not ADAPTERS): every tile's depth is cut into that many items, whose sums go to partials[slice][tile][column][row]
  // of `partial_tiles` tiles a slice, for grouped_reduce_kernel to add up
  int slices;
  int64_t partial_tiles;
  float* partials;
  float prescale_a, prescale_b;  // powers of two applied before the split
  float out_scale;               // 1 / (prescale_a prescale_b)
  float alpha, beta;
  float* C;
};

// What one tile is: which part of the operands, and where its result goes.  The same for every lane.
struct GroupedItem {
  const float* a;  // &op(A)(first row of the tile, first k)
  const float* b;
  float* c;        // &C(first row, first column)
  int64_t K;       // depth, 0 for a group without any (columns: never)
  int rows, cols;  // of the tile that exist, at most 128
  int readable_rows, readable_cols;  // how many are in memory from the first one on, at most 128
  int m0, n0;      // adapters only: the tile's first row and column
  float* partial;  // sliced tiles only, else null: where its sums go, 128 rows apart
};

// the value of the first lane, for what is the same in all of them
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const unsigned low = (unsigned)__builtin_amdgcn_readfirstlane((int)v), high = (unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32));
  return (int64_t)(((uint64_t)high << 32) | low);
}
__device__ __forceinline__ const float* uniform(const float* v) { return reinterpret_cast<const float*>(uniform((int64_t)(uintptr_t)v)); }

// One operand of a tile, as WideOperand but for any number of rows and either mode.  A splitting thread t of 256 holds UNITS
// units of a row and an octet of the depth each:
//   !DEPTH (rows contiguous)   rows UNITS (t % (128 / UNITS)) + u, octet t / (128 / UNITS); load j: k = 8 octet + j of all rows
//   DEPTH (depth contiguous)   rows t / OCTETS + (256 / OCTETS) u, octet t % OCTETS; two 16-byte loads per unit
template <int METHOD, bool DEPTH>
struct GroupedOperand {
  static constexpr int KIND = split_kind_of(METHOD), NP = parts_of_split(KIND);
  static constexpr int K_STEPS = METHOD == kMethodFp16Split ? 4 : 2, CHUNK = 16 * K_STEPS, OCTETS = 2 * K_STEPS;
  static constexpr int UNITS = kGroupedTile * CHUNK / (8 * 256), VALUES = 8 * UNITS;
  static constexpr int REGION_BYTES = (kGroupedTile / 32) * K_STEPS * NP * 1024;
  typedef unsigned uint4_t __attribute__((ext_vector_type(4)));
  typedef float unit_rows_t __attribute__((ext_vector_type(UNITS), aligned(4)));
  typedef float float4_any_t __attribute__((ext_vector_type(4), aligned(4)));
  // (what went through uniform() is no longer known to be global memory, and would be read by FLAT instructions)
  typedef __attribute__((address_space(1))) unit_rows_t global_rows_t;
  typedef __attribute__((address_space(1))) float4_any_t global_float4_t;

  const float* first;  // &X(first row of the tile, first k), the same for the block
  int64_t ld, K;
  int row, octet;      // of this thread's unit 0
  int rows;            // DEPTH: rows that exist; else: rows in memory
  // !DEPTH, the same for the block: the last rows in memory are fewer than a load takes, so that lane reads the last ones that
  // fill one, `shift` rows earlier, and realign() moves them; or all of them are, and they are read one by one.  (Every tile
  // that straddles with its rows read one by one: eight gradients of 1001 x 2003 over 8192 262 us instead of 134.)
  bool straddles, tiny;
  int shift;
  unsigned lane_bytes[DEPTH ? UNITS : 1];
  float factor;

  // The place of a row within a half of 32 (see wide_lds_slot).  Where 16 lanes write at once they hold two rows of eight
  // octets each (chunks of 64), rows contiguous four rows apart: place_in_half sends those to different banks.  In chunks of 32
  // they hold four rows of four octets, or every other row of 32: bits 1 and 0 of the row become bits 3 and 2 of the place
  // for the one, and bit 4 joins bit 0 for the other.  (With place_in_half a third of the LDS cycles of a BF16 call were
  // conflicts.)
  __device__ __forceinline__ static int place_of(int r) {
    return K_STEPS == 4 ? place_in_half(r) : (r & 16) | (r & 2) << 2 | ((r ^ r >> 4) & 1) << 2 | (r & 8) >> 2 | (r & 4) >> 2;
  }
  __device__ __forceinline__ static int row_of_place(int q) {
    return K_STEPS == 4 ? row_at_place(q) : (q & 16) | (q & 8) >> 2 | ((q >> 2 ^ q >> 4) & 1) | (q & 2) << 2 | (q & 1) << 2;
  }
  __device__ __forceinline__ static int lds_slot(int row_block, int place, int octet) {
    return (row_block * K_STEPS + (octet >> 1)) * NP * 1024 + (octet & 1) * 512 + ((place + octet) & 31) * 16;
  }
  __device__ __forceinline__ int unit_row(int u) const { return DEPTH ? row + (256 / OCTETS) * u : row + u; }
  __device__ __forceinline__ int clamped_row(int u) const {
    const int r = unit_row(u);
    return r < rows ? r : rows - 1;
  }

  __device__ __forceinline__ void init(const float* first_, int64_t ld_, int64_t K_, int exist, int readable, float factor_, int t) {
    asm volatile("" : "+v"(t));  // (or everything made of it is worked out before the first tile and kept)
    // (a buffer load takes its base from scalar registers: where the compiler cannot tell that it is the same in all lanes, every
    // load becomes a loop over them)
    first = uniform(first_), ld = ld_, K = uniform(K_), factor = factor_;
    octet = DEPTH ? t % OCTETS : t / (kGroupedTile / UNITS);
    row = DEPTH ? t / OCTETS : UNITS * (t % (kGroupedTile / UNITS));
    rows = DEPTH ? exist : readable;
    tiny = !DEPTH && readable < UNITS;
    straddles = !DEPTH && !tiny && readable < kGroupedTile && readable % UNITS != 0;
    if constexpr (DEPTH) {
#pragma unroll
      for (int u = 0; u < UNITS; ++u) lane_bytes[u] = (unsigned)((clamped_row(u) * ld + 8 * octet) * 4);
    } else {
      const int start = row + UNITS <= rows ? row : rows >= UNITS ? rows - UNITS : 0;
      lane_bytes[0] = (unsigned)((8 * octet * ld + start) * 4);
      shift = row - start;
    }
  }

  // Loads FIRST .. FIRST + COUNT - 1 of chunk c, which lies inside the depth; not tiny.
  static constexpr int LOADS = DEPTH ? 2 * UNITS : 8;
  template <int FIRST = 0, int COUNT = LOADS>
  __device__ __forceinline__ void fetch(float (&x)[VALUES], int c) const {
    const float* chunk = first + (DEPTH ? (int64_t)c * CHUNK : (int64_t)c * CHUNK * ld);
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(chunk), 0, -1, 0x00020000);
    const unsigned step = (unsigned)(4 * ld);
#pragma unroll
    for (int j = FIRST; j < FIRST + COUNT; ++j) {
      if constexpr (DEPTH) {
        const source4_t v = __builtin_bit_cast(source4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer, (int)(lane_bytes[j >> 1] + (j & 1) * 16), 0, 0));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[8 * (j >> 1) + 4 * (j & 1) + e] = v[e];
      } else if constexpr (UNITS == 4) {
        const source4_t v = __builtin_bit_cast(source4_t, __builtin_amdgcn_raw_buffer_load_b128(buffer, (int)lane_bytes[0], (int)(j * step), 0));
#pragma unroll
        for (int u = 0; u < 4; ++u) x[8 * u + j] = v[u];
      } else {
        typedef float float2_t __attribute__((ext_vector_type(2)));
        const float2_t v = __builtin_bit_cast(float2_t, __builtin_amdgcn_raw_buffer_load_b64(buffer, (int)lane_bytes[0], (int)(j * step), 0));
#pragma unroll
        for (int u = 0; u < 2; ++u) x[8 * u + j] = v[u];
      }
    }
  }
  // Chunk c whatever it is: every address is inside the operand, complete() does the rest.  K >= 1.
  __device__ __forceinline__ void fetch_any(float (&x)[VALUES], int c) const {
    const int64_t k0 = (int64_t)c * CHUNK + 8 * octet;
    if constexpr (DEPTH) {
      if (K >= 4) {
#pragma unroll
        for (int j = 0; j < 2 * UNITS; ++j) {
          const int64_t k = k0 + 4 * (j & 1);
          const float4_any_t v = *(const global_float4_t*)(first + clamped_row(j >> 1) * ld + (k < K - 4 ? k : K - 4));
#pragma unroll
          for (int e = 0; e < 4; ++e) x[8 * (j >> 1) + 4 * (j & 1) + e] = v[e];
        }
      } else {
#pragma unroll
        for (int i = 0; i < VALUES; ++i) x[i] = load_global(first + clamped_row(i >> 3) * ld + (k0 + (i & 7) < K ? k0 + (i & 7) : K - 1));
      }
    } else {
      if (!tiny) {
        const int start = row + UNITS <= rows ? row : rows - UNITS;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const unit_rows_t v = *(const global_rows_t*)(first + start + (k0 + j < K ? k0 + j : K - 1) * ld);
#pragma unroll
          for (int u = 0; u < UNITS; ++u) x[8 * u + j] = v[u];
        }
      } else {
#pragma unroll
        for (int i = 0; i < VALUES; ++i) x[i] = load_global(first + clamped_row(i >> 3) + (k0 + (i & 7) < K ? k0 + (i & 7) : K - 1) * ld);
      }
    }
  }
  // k behind the depth counts as zero
  __device__ __forceinline__ void complete(float (&x)[VALUES], int c) const {
    const int64_t k0 = (int64_t)c * CHUNK + 8 * octet;
    if (DEPTH && K >= 4) {
#pragma unroll
      for (int j = 0; j < 2 * UNITS; ++j) {
        const int64_t k = k0 + 4 * (j & 1);
        float* at = &x[8 * (j >> 1) + 4 * (j & 1)];
        const source4_t y = shift_or_zero(source4_t{at[0], at[1], at[2], at[3]}, k - (k < K - 4 ? k : K - 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) at[e] = y[e];
      }
    } else {
#pragma unroll
      for (int i = 0; i < VALUES; ++i) x[i] = k0 + (i & 7) < K ? x[i] : 0.0f;
    }
  }

  // The rows of a lane that read earlier ones, in their places (rows that do not exist hold anything)
  __device__ __forceinline__ void realign(float (&x)[VALUES]) const {
    if constexpr (!DEPTH) {
      if (!straddles) return;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
#pragma unroll
          for (int d = 1; u + d < UNITS; ++d) x[8 * u + j] = shift == d ? x[8 * (u + d) + j] : x[8 * u + j];
    }
  }

  // The parts of unit u, by the short split without a test for the values it does not take (see wide_kernel).
  template <bool SCALED>
  __device__ __forceinline__ void convert(const float (&x)[VALUES], int u, uint4_t (&parts)[NP]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v0 = SCALED ? x[8 * u + 2 * e] * factor : x[8 * u + 2 * e], v1 = SCALED ? x[8 * u + 2 * e + 1] * factor : x[8 * u + 2 * e + 1];
      unsigned words[NP];
      FastSplit<KIND>::split2(v0, v1, v0 * 2048.0f, v1 * 2048.0f, words);
#pragma unroll
      for (int q = 0; q < NP; ++q) parts[q][e] = words[q];
    }
  }
  __device__ __forceinline__ void convert_with_care(const float (&x)[VALUES], int u, uint4_t (&parts)[NP]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      unsigned short even[NP], odd[NP];
      Splitter<KIND>::split(x[8 * u + 2 * e] * factor, even);
      Splitter<KIND>::split(x[8 * u + 2 * e + 1] * factor, odd);
#pragma unroll
      for (int q = 0; q < NP; ++q) parts[q][e] = (unsigned)even[q] | ((unsigned)odd[q] << 16);
    }
  }
  __device__ __forceinline__ void write(const uint4_t (&parts)[NP], int u, char* region) const {
    const int r = unit_row(u);
    char* at = region + lds_slot(r >> 5, place_of(r & 31), octet);
#pragma unroll
    for (int q = 0; q < NP; ++q) *reinterpret_cast<uint4_t*>(at + q * 1024) = parts[q];
  }
  // Splits units FIRST .. and writes their parts to `region`.  REFILL: chunk `next`, which lies inside the depth, is
  // requested into the registers as they become free.
  template <bool SCALED, bool REFILL, int FIRST>
  __device__ __forceinline__ void deposit(float (&x)[VALUES], char* region, int next) const {
    if constexpr (REFILL && DEPTH && FIRST > 0) {
      fetch<0, 2 * FIRST>(x, next);
      __builtin_amdgcn_sched_barrier(0);
    }
    static_for<UNITS - FIRST>([&](auto u_c) {
      constexpr int u = FIRST + decltype(u_c)::value;
      uint4_t parts[NP];
      convert<SCALED>(x, u, parts);
      write(parts, u, region);
      if constexpr (REFILL && DEPTH) {
        __builtin_amdgcn_sched_barrier(0);
        fetch<2 * u, 2>(x, next);
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    if constexpr (REFILL && !DEPTH) {
      __builtin_amdgcn_sched_barrier(0);
      fetch(x, next);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __device__ __forceinline__ void deposit_with_care(const float (&x)[VALUES], char* region) const {
    static_for<UNITS>([&](auto u_c) {
      constexpr int u = decltype(u_c)::value;
      uint4_t parts[NP];
      convert_with_care(x, u, parts);
      write(parts, u, region);
      __builtin_amdgcn_sched_barrier(0);
    });
  }
};

// The groups of a launch as a block keeps them: [begin, end) of each along the columns or the depth, and the number of
// 128-column tiles before it (columns only).  A block reads the offsets once: all its waves see the same ones, whatever
// happens to them meanwhile, and pass the same barriers.
struct GroupTable {
  int first_tile[kGroupsPerLaunch + 64];  // [groups] and everything behind it: the number of all tiles
  int begin[kGroupsPerLaunch], end[kGroupsPerLaunch];
};
// ADAPTERS: those of each group's columns.
struct AdapterTable {
  int adapter[kGroupsPerLaunch];  // -1: none
  float scale[kGroupsPerLaunch];
};
__device__ __forceinline__ int64_t clamp_offset(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }
// Called by all kGroupedThreads threads; ends with a barrier.  Offsets outside [0, N] (or K) or decreasing ones are
// clamped, so that no tile ever reaches beyond the operands (the caller holds N and K <= 2^31 - 1).
__device__ __forceinline__ void make_group_table(const GroupedParams& p, GroupTable& table, AdapterTable* adapters, int* wave_sums) {
  constexpr int PER_THREAD = kGroupsPerLaunch / kGroupedThreads;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  int tiles[PER_THREAD], sum = 0;
#pragma unroll
  for (int i = 0; i < PER_THREAD; ++i) {
    const int g = PER_THREAD * t + i;
    tiles[i] = 0;
    if (g < p.groups) {
      const int64_t most = p.along_depth ? p.K : p.N;
      const int64_t begin = clamp_offset(p.offsets[g], 0, most), end = clamp_offset(p.offsets[g + 1], begin, most);
      table.begin[g] = (int)begin, table.end[g] = (int)end;
      if (adapters != nullptr) {
        const int a = p.index[g], adapter = a >= 0 && a < p.matrices ? a : -1;
        adapters->adapter[g] = adapter;
        adapters->scale[g] = adapter >= 0 && p.scales != nullptr ? p.scales[adapter] : 1.0f;
      }
      tiles[i] = (int)grouped_tiles(end - begin);
    }
    sum += tiles[i];  // (at most 2 x 2^24)
  }
  // (decreasing offsets can make the sum of all of them larger than what 32 bits hold: 2^29 is beyond any sound one)
  auto add = [](int a, int b) { return a + b < (1 << 29) ? a + b : 1 << 29; };
  int upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int other = __shfl_up(upto, d, 64);
    if (lane >= d) upto = add(upto, other);
  }
  if (lane == 63) wave_sums[wave] = upto;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < wave; ++w) before = add(before, wave_sums[w]);
  int at = add(before, upto) - sum;
  at = at < 0 ? 0 : at;
#pragma unroll
  for (int i = 0; i < PER_THREAD; ++i) {
    table.first_tile[PER_THREAD * t + i] = at;
    at += tiles[i];
  }
  if (t == kGroupedThreads - 1) {
    for (int i = 0; i < 64; ++i) table.first_tile[kGroupsPerLaunch + i] = at;
  }
  __syncthreads();
}

// Item number `index`: the tile, and which slice of its depth.  Called by whole waves.
template <bool DEPTH_A, bool DEPTH_B, bool ADAPTERS, int CHUNK>
__device__ __forceinline__ GroupedItem grouped_item(const GroupedParams& p, const GroupTable& table, int index) {
  const int lane = threadIdx.x & 63;
  GroupedItem it;
  it.partial = nullptr;
  int slice = 0;
  if (!ADAPTERS && p.slices > 1) {
    const int tile = index / p.slices;
    slice = index - tile * p.slices;
    it.partial = p.partials + (slice * p.partial_tiles + tile) * (kGroupedTile * kGroupedTile);
    index = tile;
  }
  int group, tile_m, tile_n;
  if constexpr (ADAPTERS) {
    tile_coordinates(index, p.tiles_m, p.tiles_n, 4, 1, tile_m, tile_n);
    const int64_t m0 = (int64_t)tile_m * kGroupedTile, n0 = (int64_t)tile_n * kGroupedTile;
    it.a = p.A + (DEPTH_A ? m0 * p.lda : m0);
    it.b = p.B + (DEPTH_B ? n0 * p.ldb : n0);
    it.c = p.C + m0 + n0 * p.ldc;
    it.K = p.K;
    it.rows = it.readable_rows = (int)(p.M - m0 < kGroupedTile ? p.M - m0 : kGroupedTile);
    it.cols = it.readable_cols = (int)(p.N - n0 < kGroupedTile ? p.N - n0 : kGroupedTile);
    it.m0 = (int)m0, it.n0 = (int)n0;
  } else if (p.along_depth) {
    const int tiles = p.tiles_m * p.tiles_n;
    group = index / tiles;
    tile_coordinates(index - group * tiles, p.tiles_m, p.tiles_n, 4, 1, tile_m, tile_n);
    const int64_t begin = uniform(table.begin[group]), end = uniform(table.end[group]);
    const int64_t m0 = (int64_t)tile_m * kGroupedTile, n0 = (int64_t)tile_n * kGroupedTile;
    it.a = p.A + (DEPTH_A ? m0 * p.lda + begin : m0 + begin * p.lda);
    it.b = p.B + (DEPTH_B ? n0 * p.ldb + begin : n0 + begin * p.ldb);
    it.c = p.C + group * p.stride_c + m0 + n0 * p.ldc;
    it.K = end - begin;
    it.rows = it.readable_rows = (int)(p.M - m0 < kGroupedTile ? p.M - m0 : kGroupedTile);
    it.cols = it.readable_cols = (int)(p.N - n0 < kGroupedTile ? p.N - n0 : kGroupedTile);
  } else {
    // the last group that starts at or before this tile: 64 lanes look at every 64th entry, then at 64 entries
    const int column_tile = index / p.tiles_m;
    const int block = __popcll(__builtin_amdgcn_ballot_w64(lane < kGroupsPerLaunch / 64 && table.first_tile[64 * (lane & (kGroupsPerLaunch / 64 - 1))] <= column_tile)) - 1;
    group = 64 * block + __popcll(__builtin_amdgcn_ballot_w64(table.first_tile[64 * block + lane] <= column_tile)) - 1;
    group = group < p.groups ? group : p.groups - 1;
    const int begin = uniform(table.begin[group]), end = uniform(table.end[group]);
    const int first_tile = uniform(table.first_tile[group]);
    const int tiles_n = (int)grouped_tiles(end - begin);
    const int64_t within = index - (int64_t)first_tile * p.tiles_m;
    // (only offsets that decrease can bring a tile that does not exist: it has no columns and is passed over)
    tile_m = 0, tile_n = tiles_n;
    if (within < (int64_t)tiles_n * p.tiles_m) tile_coordinates((int)within, p.tiles_m, tiles_n, 4, 1, tile_m, tile_n);
    const int64_t m0 = (int64_t)tile_m * kGroupedTile, n0 = begin + (int64_t)tile_n * kGroupedTile;
    it.a = p.A + group * p.stride_a + (DEPTH_A ? m0 * p.lda : m0);
    it.b = p.B + (DEPTH_B ? n0 * p.ldb : n0);
    it.c = p.C + m0 + n0 * p.ldc;
    it.rows = it.readable_rows = (int)(p.M - m0 < kGroupedTile ? p.M - m0 : kGroupedTile);
    it.cols = (int)(end - n0 < kGroupedTile ? end - n0 : kGroupedTile);
    it.readable_cols = (int)(p.N - n0 < kGroupedTile ? p.N - n0 : kGroupedTile);
    it.K = it.cols > 0 ? p.K : 0;
  }
  if (!ADAPTERS && p.slices > 1) {
    const int64_t chunks = (it.K + CHUNK - 1) / CHUNK, per_slice = (chunks + p.slices - 1) / p.slices, begin = slice * per_slice * CHUNK;
    const int64_t left = it.K > begin ? it.K - begin : 0;
    if (left > 0) {
      it.a += DEPTH_A ? begin : begin * p.lda;
      it.b += DEPTH_B ? begin : begin * p.ldb;
    }
    it.K = left < per_slice * CHUNK ? left : per_slice * CHUNK;
  }
  return it;
}

// ADAPTERS: a projection of all columns, op(A) op(B), with low-rank adapters.  The groups that a tile's columns belong to add a
// chunk or two each to its depth: U_a's rows times H's columns, those of other groups taken as zero, times scale / alpha.  C is
// written once; a pass of its own over C for the adapters costs as much as writing it twice more (4096 cubed, rank 32, 65 us
// of 440 FP16).
template <int METHOD, bool DEPTH_A, bool DEPTH_B, bool SCALED, bool ADAPTERS>
__global__ void __launch_bounds__(kGroupedThreads, 1) grouped_kernel(const GroupedParams p) {
  static_assert(!ADAPTERS || (DEPTH_B && !SCALED), "H has its rank contiguous");
  constexpr int KIND = split_kind_of(METHOD), NP = parts_of_split(KIND), PRODUCTS = products_of(METHOD), ELEM = element_kind_of(METHOD);
  typedef GroupedOperand<METHOD, DEPTH_A> OperandA;
  typedef GroupedOperand<METHOD, DEPTH_B> OperandB;
  constexpr int K_STEPS = OperandA::K_STEPS, CHUNK = OperandA::CHUNK, VALUES = OperandA::VALUES;
  constexpr int REGION_BYTES = OperandA::REGION_BYTES, STAGE_BYTES = 2 * REGION_BYTES;
  typedef typename Mfma<ELEM>::frag_t frag_t;
  __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE_BYTES];
  __shared__ GroupTable table;
  __shared__ std::conditional_t<ADAPTERS, AdapterTable, char> adapter_space;
  AdapterTable* const adapter_table = reinterpret_cast<AdapterTable*>(&adapter_space);  // (ADAPTERS only)
  __shared__ int wave_sums[kGroupedThreads / 64];
  // Whether multiplying wave w left its part of the block's tile number i unwritten (below); any[w]: of any tile
  __shared__ __attribute__((aligned(4))) unsigned char not_finite[kGroupedTilesPerBlock][4];
  __shared__ int any_not_finite[4];

  const int t = threadIdx.x, lane = t & 63;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
  int items;
  if (p.along_depth) {
    make_group_table(p, table, nullptr, wave_sums);
    items = p.groups * p.tiles_m * p.tiles_n * p.slices;
  } else if (ADAPTERS) {
    make_group_table(p, table, adapter_table, wave_sums);
    items = p.tiles_m * p.tiles_n;
  } else {
    make_group_table(p, table, nullptr, wave_sums);
    const int64_t all = (int64_t)table.first_tile[kGroupsPerLaunch] * p.tiles_m * p.slices;
    // (more than the host has counted on there are only with offsets that decrease)
    const int64_t most = p.slices > 1 ? p.partial_tiles * p.slices : (int64_t)gridDim.x * kGroupedTilesPerBlock;
    items = uniform((int)(all < most ? all : most));
  }
  // Each XCD takes a contiguous run of every round of tiles, whose patch shares rows of A and columns of B in its L2.
  const int position = (int)xcd_run_position(blockIdx.x, gridDim.x), step_items = (int)gridDim.x;

  auto item_at = [&](int index) { return grouped_item<DEPTH_A, DEPTH_B, ADAPTERS, OperandA::CHUNK>(p, table, index); };
  auto chunks_of = [&](const GroupedItem& it) { return (int)((it.K + CHUNK - 1) / CHUNK); };

  // The adapters of a tile's columns, in the order of their groups: visit(group, first column, last column + 1).
  const int rank_chunks = ADAPTERS ? (int)((p.rank + CHUNK - 1) / CHUNK) : 0;
  auto for_adapters = [&](const GroupedItem& it, auto&& visit) {
    for (int base = 0; base < p.groups; base += 64) {
      const int g = base + lane;
      bool hit = false;
      if (g < p.groups) {
        const int begin = table.begin[g], end = table.end[g];
        hit = adapter_table->adapter[g] >= 0 && begin < end && begin < it.n0 + it.cols && end > it.n0;
      }
      for (uint64_t left = __builtin_amdgcn_ballot_w64(hit); left != 0; left &= left - 1) {
        const int at = base + __builtin_ctzll(left);
        const int lo = uniform(table.begin[at]) - it.n0, hi = uniform(table.end[at]) - it.n0;
        visit(at, lo > 0 ? lo : 0, hi < it.cols ? hi : it.cols);
      }
    }
  };
  auto adapters_of = [&](const GroupedItem& it) {
    int n = 0;
    for (int base = 0; base < p.groups; base += 64) {
      const int g = base + lane;
      n += __popcll(__builtin_amdgcn_ballot_w64(g < p.groups && adapter_table->adapter[g] >= 0 && table.begin[g] < table.end[g] && table.begin[g] < it.n0 + it.cols && table.end[g] > it.n0));
    }
    return n;
  };

  auto block_barrier = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // Every wave passes one barrier per chunk of every tile, and one more where a tile's chunks are odd in number, so that
  // every tile starts with buffer 0: a splitting wave after each chunk it has written, a multiplying wave before each chunk
  // it reads, having read the chunk before it to the end.  Chunk c of a tile lives in buffer c % 2.
  //
  // The short split's conversions saturate by a mode bit.  What it does not take, infinities, NaN and values next to the
  // format's end, leaves an infinity or a NaN among the parts, and with it in every element of the row or column of the tile.
  // So nothing is tested in the loop; a multiplying wave whose sums are not all finite writes none of them, and when the
  // block is through with its tiles it goes through those once more, with Splitter, and writes what was left out.
  if (wave < kGroupedSplitWaves) {
    if constexpr (METHOD == kMethodFp16Split) __builtin_amdgcn_s_setreg(1 | (23 << 6), 1);  // MODE.FP16_OVFL
    OperandA a;
    OperandB b;
    // The chunks of one group's adapter, from chunk `number` of the tile on.  A tile begins with those: their loads' way is
    // then covered like that of the projection's first chunk, which is requested before them, by what the multiplying
    // waves still have to do for the tile before (behind the projection they cost 7 us a tile).
    auto deposit_adapter = [&](const GroupedItem& it, int group, int lo, int hi, int& number, auto careful_c) {
      constexpr bool careful = decltype(careful_c)::value;
      const int adapter = uniform(adapter_table->adapter[group]);
      const float scale = adapter_table->scale[group];
      OperandA oa;
      OperandB ob;
      float va[VALUES], vb[VALUES];
      oa.init(p.U + adapter * p.stride_u + (DEPTH_A ? it.m0 * p.ldu : (int64_t)it.m0), p.ldu, p.rank, it.rows, it.readable_rows, 1.0f, t);
      ob.init(p.H + it.n0 * p.ldh, p.ldh, p.rank, it.cols, it.readable_cols, scale / p.alpha, t);
      for (int c = 0; c < rank_chunks; ++c, ++number) {
        char* stage = lds + (number & 1) * STAGE_BYTES;
        oa.fetch_any(va, c);
        oa.complete(va, c);
        oa.realign(va);
        if constexpr (careful) oa.deposit_with_care(va, stage);
        else oa.template deposit<false, false, 0>(va, stage, 0);
        __builtin_amdgcn_sched_barrier(0);
        ob.fetch_any(vb, c);
        ob.complete(vb, c);
        static_for<VALUES>([&](auto i_c) {
          constexpr int i = decltype(i_c)::value;
          const int r = ob.unit_row(i / 8);
          vb[i] = r >= lo && r < hi ? vb[i] : 0.0f;
        });
        if constexpr (careful) {
          ob.deposit_with_care(vb, stage + REGION_BYTES);
        } else {
          ob.template deposit<true, false, 0>(vb, stage + REGION_BYTES, 0);
        }
        block_barrier();
      }
    };
    for (int index = position; index < items; index += step_items) {
      const GroupedItem it = item_at(index);
      const int chunks = chunks_of(it);
      if (chunks == 0) continue;
      float xa[2][VALUES], xb[2][VALUES];
      a.init(it.a, p.lda, it.K, it.rows, it.readable_rows, p.prescale_a, t);
      b.init(it.b, p.ldb, it.K, it.cols, it.readable_cols, p.prescale_b, t);
      const int whole = a.tiny || b.tiny ? 0 : (int)(it.K / CHUNK);
      const int bulk = a.straddles || b.straddles ? 0 : whole;  // (the loop of whole chunks has no rows to move)
      auto request = [&](auto r_c, int c) {
        constexpr int r = decltype(r_c)::value;
        if (c < whole) a.fetch(xa[r], c), b.fetch(xb[r], c);
        else if (c < chunks) a.fetch_any(xa[r], c), b.fetch_any(xb[r], c);
      };
      request(std::integral_constant<int, 0>{}, 0);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (ADAPTERS) {
        int number = 0;
        for_adapters(it, [&](int group, int lo, int hi) { deposit_adapter(it, group, lo, hi, number, std::false_type{}); });
        if (number & 1) block_barrier();
      }
      request(std::integral_constant<int, 1>{}, 1);
      __builtin_amdgcn_sched_barrier(0);
      int c = 0;
      // the bulk of the depth: chunks that lie inside it, and so do those requested behind them
      typename OperandA::uint4_t ahead[NP];
      if (c + 4 <= bulk) a.template convert<SCALED>(xa[0], 0, ahead);
      for (; c + 4 <= bulk; c += 2) {
        static_for<2>([&](auto r_c) {
          constexpr int r = decltype(r_c)::value;
          a.write(ahead, 0, lds + r * STAGE_BYTES);
          a.template deposit<SCALED, true, 1>(xa[r], lds + r * STAGE_BYTES, c + r + 2);
          b.template deposit<SCALED, true, 0>(xb[r], lds + r * STAGE_BYTES + REGION_BYTES, c + r + 2);
          a.template convert<SCALED>(xa[r ^ 1], 0, ahead);
          block_barrier();
        });
      }
      for (; c < chunks; c += 2) {
        static_for<2>([&](auto r_c) {
          constexpr int r = decltype(r_c)::value;
          if (c + r < chunks) {
            if (c + r >= whole) a.complete(xa[r], c + r), b.complete(xb[r], c + r);
            a.realign(xa[r]), b.realign(xb[r]);
            a.template deposit<SCALED, false, 0>(xa[r], lds + r * STAGE_BYTES, 0);
            b.template deposit<SCALED, false, 0>(xb[r], lds + r * STAGE_BYTES + REGION_BYTES, 0);
            __builtin_amdgcn_sched_barrier(0);
            request(r_c, c + r + 2);
            block_barrier();
          }
        });
      }
      if (chunks & 1) block_barrier();
    }
    block_barrier();  // the multiplying waves' words are there
    if (uniform(any_not_finite[0] | any_not_finite[1] | any_not_finite[2] | any_not_finite[3]) == 0) return;
    int number = 0;
    for (int index = position; index < items; index += step_items, ++number) {
      if (uniform(*reinterpret_cast<const int*>(not_finite[number])) == 0) continue;
      const GroupedItem it = item_at(index);
      auto again = [&](auto&& adapter) {
        int number = 0;
        adapter(number);
        if (number & 1) block_barrier();
        a.init(it.a, p.lda, it.K, it.rows, it.readable_rows, p.prescale_a, t);
        b.init(it.b, p.ldb, it.K, it.cols, it.readable_cols, p.prescale_b, t);
        const int chunks = chunks_of(it);
        for (int c = 0; c < chunks; ++c) {
          float xa[VALUES], xb[VALUES];
          char* stage = lds + (c & 1) * STAGE_BYTES;
          a.fetch_any(xa, c), b.fetch_any(xb, c);
          a.complete(xa, c), b.complete(xb, c);
          a.realign(xa), b.realign(xb);
          a.deposit_with_care(xa, stage);
          b.deposit_with_care(xb, stage + REGION_BYTES);
          block_barrier();
        }
        if (chunks & 1) block_barrier();
      };
      if constexpr (ADAPTERS)
        for_adapters(it, [&](int group, int lo, int hi) { again([&](int& number) { deposit_adapter(it, group, lo, hi, number, std::true_type{}); }); });
      again([](int&) {});
    }
    return;
  }

  // ---- multiplying waves: rows wave_m 64 .. + 63 and columns wave_n 64 .. + 63 of the tile
  __builtin_amdgcn_s_setprio(2);
  const int wave_m = wave & 1, wave_n = (wave >> 1) & 1, which = wave - kGroupedSplitWaves;
  float16_t acc_main[2][2], acc_corr[2][2];
  int lane_off[K_STEPS];
#pragma unroll
  for (int ks = 0; ks < K_STEPS; ++ks) lane_off[ks] = OperandA::lds_slot(0, lane & 31, 2 * ks + (lane >> 5));
  frag_t fa[2][2][NP], fb[2][2][NP];
  constexpr int READS = 4 * NP, MFMAS = 4 * PRODUCTS;
  auto read_fragment = [&](auto set_c, auto r_c, const char* stage, int off) {
    constexpr int set = decltype(set_c)::value, r = decltype(r_c)::value, part = r / 4, place = r % 4;  // a0 b0 b1 a1 of part 0, b0 b1 a0 a1 of the others
    constexpr bool from_b = part == 0 ? (place == 1 || place == 2) : place < 2;
    constexpr int index = part == 0 ? (place >= 2 ? 1 : 0) : place & 1;
    if constexpr (from_b)
      fb[set][index][part] = *reinterpret_cast<const frag_t*>(stage + REGION_BYTES + (wave_n * 2 + index) * K_STEPS * NP * 1024 + part * 1024 + off);
    else
      fa[set][index][part] = *reinterpret_cast<const frag_t*>(stage + (wave_m * 2 + index) * K_STEPS * NP * 1024 + part * 1024 + off);
  };
  auto step = [&](auto set_c, const char* stage, int off) {
    constexpr int SET = decltype(set_c)::value;
    static_for<MFMAS>([&](auto m_c) {
      constexpr int m = decltype(m_c)::value;
      constexpr ProductTerm term = product_term(METHOD, m / 4);
      constexpr int i = (m % 4) / 2, j = m % 2;
      if constexpr (term.correction)
        acc_corr[i][j] = Mfma<ELEM>::run(fb[SET][j][term.qb], fa[SET][i][term.qa], acc_corr[i][j]);
      else
        acc_main[i][j] = Mfma<ELEM>::run(fb[SET][j][term.qb], fa[SET][i][term.qa], acc_main[i][j]);
      if constexpr (m < READS) read_fragment(std::integral_constant<int, SET ^ 1>{}, m_c, stage, off);
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // A tile's sums, main + correction, in acc_main; returns whether all of them are finite.  ADAPTERS: their chunks first.
  auto multiply = [&](int adapter_chunks, int own_chunks) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc_main[i][j][v] = 0.0f, acc_corr[i][j][v] = 0.0f;
    for (int part = ADAPTERS ? 0 : 1; part < 2; ++part) {
      const int chunks = part == 0 ? adapter_chunks : own_chunks;
      if (chunks == 0) continue;
      block_barrier();  // chunk 0 is there
      static_for<READS>([&](auto r_c) { read_fragment(std::integral_constant<int, 0>{}, r_c, lds, lane_off[0]); });
      auto steps_within = [&](const char* stage) {
        static_for<K_STEPS - 1>([&](auto ks_c) {
          constexpr int ks = decltype(ks_c)::value;
          step(std::integral_constant<int, ks & 1>{}, stage, lane_off[ks + 1]);
        });
      };
      auto chunk_and_next = [&](const char* stage, const char* next) {
        steps_within(stage);
        block_barrier();  // this chunk has been read to the end, the next one is there
        step(std::integral_constant<int, (K_STEPS - 1) & 1>{}, next, lane_off[0]);
      };
      int left = chunks - 1;
      for (; left >= 2; left -= 2) {
        chunk_and_next(lds, lds + STAGE_BYTES);
        chunk_and_next(lds + STAGE_BYTES, lds);
      }
      if (left == 1) chunk_and_next(lds, lds + STAGE_BYTES);
      const char* last = lds + ((chunks - 1) & 1) * STAGE_BYTES;
      steps_within(last);
      step(std::integral_constant<int, (K_STEPS - 1) & 1>{}, last, lane_off[0]);  // (what it reads is not used)
      if (chunks & 1) block_barrier();
    }
    float largest = 0.0f;
    constexpr float corr_scale = METHOD == kMethodFp16Split ? 0x1p-11f : 1.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          acc_main[i][j][v] = acc_main[i][j][v] + acc_corr[i][j][v] * corr_scale;
          largest = __builtin_elementwise_maximum(largest, __builtin_fabsf(acc_main[i][j][v]));
        }
    return __builtin_amdgcn_ballot_w64(!(largest <= 3.402823466e+38f)) == 0;
  };
  // a lane owns one row per 32 x 32 block; register v of it is the matrix instruction's column 8 (v / 4) + 4 (lane / 32) + v % 4
  // ADAPTERS: `columns` of the tile's columns, a bit each
  auto write_tile = [&](const GroupedItem& it, const uint64_t (&columns)[2]) {
    const float alpha = it.K > 0 ? p.alpha : 0.0f;  // (nothing to multiply: no infinity times zero)
    auto mine = [&](int c) { return c < it.cols && (!ADAPTERS || (columns[c >> 6] >> (c & 63) & 1) != 0); };
    // (the lane hidden from the optimizer: it would work out the columns' offsets before the first tile and keep them all)
    int lane_here = lane;
    asm volatile("" : "+v"(lane_here));
    const int tile_row = wave_m * 64 + OperandA::row_of_place(lane_here & 31);
    auto tile_column = [&](int j, int v) { return wave_n * 64 + j * 32 + OperandA::row_of_place(8 * (v / 4) + 4 * (lane_here >> 5) + v % 4); };
    auto store_all = [&](auto whole_c) {
      constexpr bool whole = decltype(whole_c)::value;
      if (it.partial != nullptr) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (whole || mine(tile_column(j, v))) store_partial(it.partial + tile_column(j, v) * kGroupedTile + tile_row + i * 32, acc_main[i][j][v]);
        return;
      }
      if (p.beta != 0.0f) {
        // (all that is added to is requested first, into the registers that the corrections have left, and without conditions:
        // a row or column that does not exist reads the last one that does)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = tile_row + i * 32;
          const float* from = it.c + (r < it.rows ? r : it.rows - 1);
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const int c = tile_column(j, v);
              acc_corr[i][j][v] = load_global(from + (whole || c < it.cols ? c : it.cols - 1) * p.ldc);
            }
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float* dst = it.c + tile_row + i * 32;
        if (tile_row + i * 32 >= it.rows) continue;
        if (p.beta != 0.0f) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (whole || mine(tile_column(j, v)))
                store_result(dst + tile_column(j, v) * p.ldc, scaled_sum(alpha, acc_main[i][j][v] * p.out_scale, p.beta, acc_corr[i][j][v]));
        } else {
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (whole || mine(tile_column(j, v))) store_result(dst + tile_column(j, v) * p.ldc, alpha * (acc_main[i][j][v] * p.out_scale));
        }
      }
    };
    if (it.cols <= 0) return;
    if (it.cols == kGroupedTile && (!ADAPTERS || (columns[0] & columns[1]) == ~0ull)) store_all(std::true_type{});
    else store_all(std::false_type{});
  };
  // (one loop for both passes, so that what they do is in the program once.  In the second one, a tile with adapters is made
  // once for each of them and once without any, and the columns concerned are written: an adapter that is not finite has
  // nothing to do with the columns of the others)
  for (int pass = 0;; ++pass) {
    int number = 0, left_out = 0;
    for (int index = position; index < items; index += step_items, ++number) {
      if (pass == 1 && uniform(*reinterpret_cast<const int*>(not_finite[number])) == 0) continue;
      const GroupedItem it = item_at(index);
      const int adapters = ADAPTERS ? adapters_of(it) : 0;
      uint64_t covered[2] = {0, 0};
      for (int turn = 0; turn <= (ADAPTERS && pass == 1 ? adapters : 0); ++turn) {
        uint64_t columns[2] = {~0ull, ~0ull};
        int adapter_chunks = 0;
        if constexpr (ADAPTERS) {
          if (pass == 0) {
            adapter_chunks = adapters * rank_chunks;
          } else if (turn < adapters) {
            adapter_chunks = rank_chunks;
            int at = 0;
            for_adapters(it, [&](int, int lo, int hi) {
              if (at++ != turn) return;
              auto below = [](int c, int word) { return c <= 64 * word ? 0ull : c >= 64 * word + 64 ? ~0ull : (1ull << (c - 64 * word)) - 1; };
#pragma unroll
              for (int w = 0; w < 2; ++w) columns[w] = below(hi, w) & ~below(lo, w), covered[w] |= columns[w];
            });
          } else {
            columns[0] = ~covered[0], columns[1] = ~covered[1];
          }
        }
        const bool finite = multiply(adapter_chunks, chunks_of(it));
        bool write = finite;
        if (pass == 0) {
          if (lane == 0) not_finite[number][which] = !finite;
          left_out |= !finite;
        } else {
          write = uniform((int)not_finite[number][which]) != 0;
        }
        if (write) write_tile(it, columns);
      }
    }
    if (pass == 1) return;
    if (lane == 0) any_not_finite[which] = left_out;
    block_barrier();
    if (uniform(any_not_finite[0] | any_not_finite[1] | any_not_finite[2] | any_not_finite[3]) == 0) return;  // the same for the block
  }
}

}  // namespace ecgemm
