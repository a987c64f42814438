// Host side of the grouped products (see "Grouped products" in include/ecgemm.h): argument checks and launches.  Part of
// ecgemm.hip, whose context, error and workspace helpers it uses.
#pragma once

namespace {

// The calls of this file run on the handle's device, whichever is current.
struct OnDeviceOf {
  int before = -1;
  hipError_t error = hipSuccess;
  explicit OnDeviceOf(ecgemm_handle_t h) {
    int now = 0;
    error = hipGetDevice(&now);
    if (error == hipSuccess && now != h->device) {
      error = hipSetDevice(h->device);
      if (error == hipSuccess) before = now;
    }
  }
  ~OnDeviceOf() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

typedef void (*grouped_fn_t)(GroupedParams);
template <int METHOD, bool SCALED>
grouped_fn_t grouped_kernel_of(bool depth_a, bool depth_b) {
  return depth_a ? (depth_b ? grouped_kernel<METHOD, true, true, SCALED, false> : grouped_kernel<METHOD, true, false, SCALED, false>)
                 : (depth_b ? grouped_kernel<METHOD, false, true, SCALED, false> : grouped_kernel<METHOD, false, false, SCALED, false>);
}

constexpr int64_t kGroupedMostTiles = 1 << 30;
// Most tiles that a call with groups of columns, or all that one with groups of the depth can have in one launch.
int64_t most_grouped_tiles(bool along_depth, int64_t groups, int64_t M, int64_t N) {
  const int64_t g = std::min<int64_t>(groups, kGroupsPerLaunch);
  return along_depth ? g * grouped_tiles(M) * grouped_tiles(N) : grouped_tiles(M) * (N / kGroupedTile + std::min(g, N));
}

// Slices of the depth: where the tiles are few, as many as fill the chip, 512 deep at least, and only if that saves more than
// the 7 us that adding them up takes, by the 0.95 us of a chunk of 64 in FP16 mode (1.5 in BF16 mode, which is cut by the same
// rule).  At most 256 tiles of partial sums: ECGEMM_GROUPED_WORKSPACE_BYTES.
int grouped_slices(int64_t tiles, int64_t depth) {
  const int64_t slices = std::min<int64_t>(kPlanComputeUnits / std::max<int64_t>(tiles, 1), std::min<int64_t>(depth / 512, 64));
  return slices >= 2 && depth / 64.0 * (1.0 - 1.0 / slices) * 0.95 > 8.0 ? (int)slices : 1;
}
static_assert((size_t)kPlanComputeUnits * kGroupedTile * kGroupedTile * sizeof(float) == ECGEMM_GROUPED_WORKSPACE_BYTES, "partial sums");

// Everything about the call is checked; gp.groups and what goes with it is filled in here.
ecgemm_status_t launch_grouped(ecgemm_handle_t h, ecgemm_mode_t mode, bool depth_a, bool depth_b, int64_t groups, GroupedParams gp) {
  const bool scaled = h->log2_scale_a != 0 || h->log2_scale_b != 0;
  gp.prescale_a = std::ldexp(1.0f, h->log2_scale_a);
  gp.prescale_b = std::ldexp(1.0f, h->log2_scale_b);
  gp.out_scale = std::ldexp(1.0f, -(h->log2_scale_a + h->log2_scale_b));
  gp.tiles_m = (int)grouped_tiles(gp.M);
  gp.tiles_n = gp.along_depth ? (int)grouped_tiles(gp.N) : 0;
  const grouped_fn_t kernel = mode == ECGEMM_MODE_FP16_SPLIT
                                  ? (scaled ? grouped_kernel_of<kMethodFp16Split, true>(depth_a, depth_b) : grouped_kernel_of<kMethodFp16Split, false>(depth_a, depth_b))
                                  : (scaled ? grouped_kernel_of<kMethodBf16Full, true>(depth_a, depth_b) : grouped_kernel_of<kMethodBf16Full, false>(depth_a, depth_b));
  const GroupedParams whole = gp;
  // The workspace for whichever launch needs most (all but the last one have as many groups as a launch takes), before the
  // first of them: a call that is refused leaves C as it was.
  const int64_t depth = gp.along_depth ? gp.K / groups : gp.K;  // of a group, all taken as equal
  size_t partial_bytes = 0;
  for (const int64_t n : {std::min<int64_t>(groups, kGroupsPerLaunch), (groups - 1) % kGroupsPerLaunch + 1}) {
    const int64_t tiles = most_grouped_tiles(gp.along_depth, n, gp.M, gp.N), slices = grouped_slices(tiles, depth);
    if (slices > 1) partial_bytes = std::max(partial_bytes, (size_t)(slices * tiles) * kGroupedTile * kGroupedTile * sizeof(float));
  }
  char* ws = nullptr;
  const ecgemm_status_t st = acquire_workspace(h, partial_bytes, &ws);
  if (st != ECGEMM_OK) return st;
  if (partial_bytes > 0) h->auto_choice = nullptr;  // (the workspace held it)
  for (int64_t first = 0; first < groups; first += kGroupsPerLaunch) {
    gp.groups = (int)std::min<int64_t>(groups - first, kGroupsPerLaunch);
    gp.offsets = whole.offsets + first;
    gp.A = whole.A + first * whole.stride_a;
    gp.C = whole.C + first * whole.stride_c;
    const int64_t tiles = most_grouped_tiles(gp.along_depth, gp.groups, gp.M, gp.N);
    gp.slices = grouped_slices(tiles, depth);
    gp.partial_tiles = tiles;
    gp.partials = gp.slices > 1 ? reinterpret_cast<float*>(ws) : nullptr;
    const int64_t items = tiles * gp.slices;
    const int64_t grid = std::max(std::min<int64_t>(items, h->compute_units), (items + kGroupedTilesPerBlock - 1) / kGroupedTilesPerBlock);
    void* args[] = {&gp};
    ECGEMM_HIP(h, hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)grid), dim3(kGroupedThreads), args, 0, h->stream));
    if (gp.slices > 1) {
      hipLaunchKernelGGL(grouped_reduce_kernel, dim3((unsigned)(16 * tiles)), dim3(kGroupedThreads), 0, h->stream, gp);
      ECGEMM_HIP(h, hipGetLastError());
    }
  }
  return ECGEMM_OK;
}

// The kernels for few columns to a group (narrow_kernel.hpp).
// H of adapters: by group below that many columns on average, else by columns of B.  Calls with M = 0, us, by group / by columns, B
// with the depth contiguous, requests of 1, 4, 8, 16 and 32 columns: D with the depth contiguous, K 4096, rank 16, 32 requests
// 10.2 / 65, 10.2 / 19, 10.2 / 11.7, 10.2 / 11.6, 14.1 / 12.3, K 2048, rank 64, 128 of them 11.1 / 99, 11.7 / 29, 14.3 / 18.6,
// 19.3 / 19.7, 21.0 / 26.9; D with the rank contiguous, 4096, 16, 32 24 / 60, 24 / 18, 24 / 10.9, 24 / 11.0, 39 / 11.5, 2048, 64, 128
// 15.9 / 91, 15.8 / 26.8, 15.8 / 17.6, 15.9 / 19.0, 24 / 28.  (B with the columns contiguous, D with the depth: 10 / 660, 9.9 / 177,
// 9.9 / 93, 9.9 / 51, 14.5 / 31: the rule is made for the other order.)
constexpr int64_t kAdapterDownMeanColumns = 8, kNarrowProjectionColumns = 64;
constexpr int64_t kShallowMeanDepth = 16, kShallowMeanDepthSlim = 64;
constexpr int64_t kAdapterOneLaunchDepth = 6144, kAdapterOneLaunchChunks = 8, kAdapterOneLaunchTiles = 128;

// Whether ecgemm_sgemm_grouped runs on narrow_kernel, by what either kernel is estimated to take (us), all groups taken as
// equal:
//   tiles: 6, and the larger of what their rounds over the chip take (0.95 a chunk of 64 in FP16 mode, 1.5 BF16; less by the
//   slices of the depth, which cost 7 to add up) and of reading A at 4.1 TB/s.
//   narrow: 4, and a pass over A for every 32 columns of a group, at 4.7 TB/s or, where there are too few blocks for that, at
//   what a block needs for the depth (2.9 per 1024; 9.3 where the rows are contiguous, and a block takes 64).
// Tiles without slices / narrow measured, FP16, A with the depth contiguous: M = K = 4096, one group of 32 columns 66.9 / 15.8, 64 67.9 /
// 29.5, 128 65.2 / 55.2; eight groups of 8 127 / 94, 32 130 / 113, 48 132 / 185; 64 groups, 1536 x 2048, of 8 192 / 139, 32
// 198 / 191, 48 202 / 306; eight, 768 x 1024, of 8 23.9 / 6.8, 96 26.4 / 22.9, 128 24.3 / 29.3; 4096 x 512 of 8 20.3 / 18.1, 32
// 21.7 / 25.5; four, 512 x 8192, of 96 122 / 74, 128 121 / 98; rows contiguous: 4096 x 4096, one of 32 72 / 42, 64 72 / 80; eight of
// 32 121 / 109, 64 124 / 197.  At worst 2048 x 2048, sixteen of 32, 55.5 / 60.6, which it takes narrow.
bool narrow_is_faster(bool depth_a, int64_t groups, int64_t M, int64_t N, int64_t K, ecgemm_mode_t mode) {
  const double bytes = 4.0 * groups * M * K, columns = (double)N / groups;
  if (columns > kGroupedTile) return false;  // (not measured)
  const double rounds = std::ceil((double)grouped_tiles(M) * groups * std::ceil(columns / kGroupedTile) / kPlanComputeUnits);
  const int slices = grouped_slices(most_grouped_tiles(false, groups, M, N), K);
  const double chunks = (K / 64.0) * (mode == ECGEMM_MODE_FP16_SPLIT ? 0.95 : 1.5) / slices;
  const double tiles_us = 6.0 + std::max(rounds * chunks, bytes / 4.1e6) + (slices > 1 ? 7.0 : 0.0);
  const double pass_us = std::max(bytes / 4.7e6, K / 1024.0 * (depth_a ? 2.9 : 9.3));
  return 4.0 + std::ceil(columns / kNarrowColumns) * pass_us < tiles_us;
}

// The same for a projection of few columns with adapters, by a pass over A for every 32 columns, and for what ecgemm_sgemm
// takes with 9 us for the adapters written before.  Calls narrow / the other way, us, A with the depth contiguous, 97 requests of
// a column, rank 16: 4096 x 4096 70 / 52, 1024 x 2048 39 / 30, 8192 x 2048 68 / 51; 64 of them narrow 44, 25, 41, 65 the other way
// 53, 30, 50.
bool narrow_projection_is_faster(bool depth_a, int64_t M, int64_t N, int64_t K, ecgemm_mode_t mode) {
  if (N > kNarrowProjectionColumns) return false;
  const Plan pl = make_plan(M, N, K, mode, ECGEMM_SHAPE_AUTO, kOneLaunchSliced);
  if (pl.shape == nullptr) return true;
  const double other_us = 9.0 + (pl.shape->fused ? one_launch_us(pl, K, mode) : split_first_us(pl, M, N, K, mode));
  const double pass_us = std::max(4.0 * M * K / 4.7e6, K / 1024.0 * (depth_a ? 2.9 : 9.3));
  return 4.0 + std::ceil((double)N / kNarrowColumns) * pass_us < other_us;
}

ecgemm_status_t launch_narrow(ecgemm_handle_t h, bool depth_a, bool depth_b, NarrowParams np) {
  const int64_t groups = np.offsets ? np.groups : 1;
  const int fr = narrow_fr(depth_a, groups, np.M, np.N / groups);
  np.row_blocks = (int)narrow_row_blocks(fr, np.M);
  void (*const kernel)(NarrowParams) = fr == 4   ? (depth_b ? narrow_kernel<false, true, 4> : narrow_kernel<false, false, 4>)
                                       : fr == 2 ? (depth_b ? narrow_kernel<true, true, 2> : narrow_kernel<true, false, 2>)
                                                 : (depth_b ? narrow_kernel<true, true, 1> : narrow_kernel<true, false, 1>);
  void* args[] = {&np};
  ECGEMM_HIP(h, hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)((groups + (np.clear_outside ? 1 : 0)) * np.row_blocks)),
                                dim3(kNarrowThreads), args, 0, h->stream));
  return ECGEMM_OK;
}

// Modes the grouped products run in: those of the method.
ecgemm_status_t check_grouped_mode(ecgemm_handle_t h, int mode, int position, const char* function) {
  if (!valid_mode_or_auto(mode)) return bad_arg(h, position, (std::string(function) + ": unknown mode").c_str());
  if (mode != ECGEMM_MODE_FP16_SPLIT && mode != ECGEMM_MODE_BF16_FULL)
    return fail(h, ECGEMM_ERR_UNSUPPORTED, std::string(function) + ": ECGEMM_MODE_FP16_SPLIT or ECGEMM_MODE_BF16_FULL", position);
  return ECGEMM_OK;
}
#define ECGEMM_ARG(h, bad, position, what) \
  do {                                     \
    if (bad) return bad_arg((h), (position), what); \
  } while (0)
bool bad_offsets(const int64_t* offsets) { return offsets == nullptr || (uintptr_t)offsets % 8 != 0; }

}  // namespace

extern "C" {

ecgemm_status_t ecgemm_sgemm_grouped(ecgemm_handle_t handle, ecgemm_op_t transA, ecgemm_op_t transB, int64_t groups, int64_t M,
                                     int64_t N, int64_t K, float alpha, const float* A, int64_t lda, int64_t strideA,
                                     const float* B, int64_t ldb, const int64_t* offsets, float beta, float* C, int64_t ldc,
                                     ecgemm_mode_t mode) {
  ecgemm_handle_t h = handle;
  if (!h) return ECGEMM_ERR_INVALID_ARG;
  ECGEMM_ARG(h, !valid_op(transA), 2, "ecgemm_sgemm_grouped: bad transA");
  ECGEMM_ARG(h, !valid_op(transB), 3, "ecgemm_sgemm_grouped: bad transB");
  ECGEMM_ARG(h, groups < 0, 4, "ecgemm_sgemm_grouped: negative number of groups");
  ECGEMM_ARG(h, M < 0, 5, "ecgemm_sgemm_grouped: negative M");
  ECGEMM_ARG(h, N < 0, 6, "ecgemm_sgemm_grouped: negative N");
  ECGEMM_ARG(h, K < 0, 7, "ecgemm_sgemm_grouped: negative K");
  const ecgemm_status_t st = check_grouped_mode(h, (int)mode, 18, "ecgemm_sgemm_grouped");
  if (st != ECGEMM_OK) return st;
  if (groups == 0 || M == 0 || N == 0) return ECGEMM_OK;
  ECGEMM_ARG(h, groups > INT_MAX, 4, "ecgemm_sgemm_grouped: too many groups");
  ECGEMM_ARG(h, M > INT_MAX, 5, "ecgemm_sgemm_grouped: M too large");
  ECGEMM_ARG(h, N > INT_MAX, 6, "ecgemm_sgemm_grouped: N too large");
  ECGEMM_ARG(h, most_grouped_tiles(false, groups, M, N) > kGroupedMostTiles, 5, "ecgemm_sgemm_grouped: M x N too large");
  ECGEMM_ARG(h, bad_offsets(offsets), 14, "ecgemm_sgemm_grouped: null or misaligned offsets");
  ECGEMM_ARG(h, !C, 16, "ecgemm_sgemm_grouped: C is null");
  ECGEMM_ARG(h, ldc < M, 17, "ecgemm_sgemm_grouped: ldc < M");
  if (alpha == 0.0f) K = 0;  // A and B are not read
  if (K > 0) {
    ECGEMM_ARG(h, K > INT_MAX, 7, "ecgemm_sgemm_grouped: K too large");
    ECGEMM_ARG(h, !A, 9, "ecgemm_sgemm_grouped: A is null");
    ECGEMM_ARG(h, lda < (transA == ECGEMM_OP_N ? M : K), 10, "ecgemm_sgemm_grouped: lda too small");
    ECGEMM_ARG(h, lda > kGroupedLargestLd, 10, "ecgemm_sgemm_grouped: lda beyond 2^21");
    ECGEMM_ARG(h, strideA < 0, 11, "ecgemm_sgemm_grouped: negative strideA");
    ECGEMM_ARG(h, !B, 12, "ecgemm_sgemm_grouped: B is null");
    ECGEMM_ARG(h, ldb < (transB == ECGEMM_OP_N ? K : N), 13, "ecgemm_sgemm_grouped: ldb too small");
    ECGEMM_ARG(h, ldb > kGroupedLargestLd, 13, "ecgemm_sgemm_grouped: ldb beyond 2^21");
  }
  const OnDeviceOf device(h);
  if (device.error != hipSuccess) return hip_fail(h, device.error, "hipSetDevice");
  if (narrow_is_faster(transA == ECGEMM_OP_T, groups, M, N, K, mode) && narrow_fits(transA == ECGEMM_OP_T, groups, M, N / groups, 0)) {
    NarrowParams np{};
    np.A = A, np.lda = lda, np.stride_a = strideA;
    np.B = B, np.ldb = ldb;
    np.C = C, np.ldc = ldc;
    np.M = M, np.N = N, np.K = K;
    np.offsets = offsets, np.groups = groups;
    np.alpha = alpha, np.beta = beta;
    return launch_narrow(h, transA == ECGEMM_OP_T, transB == ECGEMM_OP_N, np);
  }
  GroupedParams gp{};
  gp.A = A, gp.lda = lda, gp.stride_a = strideA;
  gp.B = B, gp.ldb = ldb;
  gp.C = C, gp.ldc = ldc;
  gp.M = M, gp.N = N, gp.K = K;
  gp.offsets = offsets;
  gp.alpha = alpha, gp.beta = beta;
  return launch_grouped(h, mode, transA == ECGEMM_OP_T, transB == ECGEMM_OP_N, groups, gp);
}

ecgemm_status_t ecgemm_sgemm_grouped_depth(ecgemm_handle_t handle, ecgemm_op_t transA, ecgemm_op_t transB, int64_t groups,
                                           int64_t M, int64_t N, int64_t K, float alpha, const float* A, int64_t lda,
                                           const float* B, int64_t ldb, const int64_t* offsets, float beta, float* C,
                                           int64_t ldc, int64_t strideC, ecgemm_mode_t mode) {
  ecgemm_handle_t h = handle;
  if (!h) return ECGEMM_ERR_INVALID_ARG;
  ECGEMM_ARG(h, !valid_op(transA), 2, "ecgemm_sgemm_grouped_depth: bad transA");
  ECGEMM_ARG(h, !valid_op(transB), 3, "ecgemm_sgemm_grouped_depth: bad transB");
  ECGEMM_ARG(h, groups < 0, 4, "ecgemm_sgemm_grouped_depth: negative number of groups");
  ECGEMM_ARG(h, M < 0, 5, "ecgemm_sgemm_grouped_depth: negative M");
  ECGEMM_ARG(h, N < 0, 6, "ecgemm_sgemm_grouped_depth: negative N");
  ECGEMM_ARG(h, K < 0, 7, "ecgemm_sgemm_grouped_depth: negative K");
  const ecgemm_status_t st = check_grouped_mode(h, (int)mode, 18, "ecgemm_sgemm_grouped_depth");
  if (st != ECGEMM_OK) return st;
  if (groups == 0 || M == 0 || N == 0) return ECGEMM_OK;
  ECGEMM_ARG(h, groups > INT_MAX, 4, "ecgemm_sgemm_grouped_depth: too many groups");
  ECGEMM_ARG(h, M > INT_MAX, 5, "ecgemm_sgemm_grouped_depth: M too large");
  ECGEMM_ARG(h, N > INT_MAX, 6, "ecgemm_sgemm_grouped_depth: N too large");
  // (each factor is below 2^25, so their product of at most 2^10 2^24 2^24 fits)
  ECGEMM_ARG(h, most_grouped_tiles(true, groups, M, N) > kGroupedMostTiles, 5, "ecgemm_sgemm_grouped_depth: groups x M x N too large");
  ECGEMM_ARG(h, bad_offsets(offsets), 13, "ecgemm_sgemm_grouped_depth: null or misaligned offsets");
  ECGEMM_ARG(h, !C, 15, "ecgemm_sgemm_grouped_depth: C is null");
  ECGEMM_ARG(h, ldc < M, 16, "ecgemm_sgemm_grouped_depth: ldc < M");
  ECGEMM_ARG(h, groups > 1 && strideC < (__int128)ldc * (N - 1) + M, 17, "ecgemm_sgemm_grouped_depth: the groups' C overlap");
  if (alpha == 0.0f) K = 0;
  if (K > 0) {
    ECGEMM_ARG(h, K > INT_MAX, 7, "ecgemm_sgemm_grouped_depth: K too large");
    ECGEMM_ARG(h, !A, 9, "ecgemm_sgemm_grouped_depth: A is null");
    ECGEMM_ARG(h, lda < (transA == ECGEMM_OP_N ? M : K), 10, "ecgemm_sgemm_grouped_depth: lda too small");
    ECGEMM_ARG(h, lda > kGroupedLargestLd, 10, "ecgemm_sgemm_grouped_depth: lda beyond 2^21");
    ECGEMM_ARG(h, !B, 11, "ecgemm_sgemm_grouped_depth: B is null");
    ECGEMM_ARG(h, ldb < (transB == ECGEMM_OP_N ? K : N), 12, "ecgemm_sgemm_grouped_depth: ldb too small");
    ECGEMM_ARG(h, ldb > kGroupedLargestLd, 12, "ecgemm_sgemm_grouped_depth: ldb beyond 2^21");
  }
  const OnDeviceOf device(h);
  if (device.error != hipSuccess) return hip_fail(h, device.error, "hipSetDevice");
  // Shallow groups, by their mean depth.  Tiles / shallow, us, FP16, groups of M x N: 64 of 1024 x 768, of depth 1 66 / 58, 16 66 /
  // 55, 32 66 / 63 and 97 / 112 with beta; 51 of 1792 x 1216, 1 146 / 110, 16 146 / 119, 32 146 / 158; 4 of 4096 x 4096, 1 86 / 60, 32 87 /
  // 77, 48 87 / 99; 11 of 320 x 1664, 16 16 / 13.6, 32 with beta 20 / 28.  One side of 64 or less, which a tile only half fills: 8 of
  // 64 x 4096, 1 10.1 / 5.9, 64 9.6 / 7.8, 128 10.3 / 11.7; 4096 x 64 alike.
  const int64_t shallow = M <= 64 || N <= 64 ? kShallowMeanDepthSlim : kShallowMeanDepth;
  if (K <= shallow * groups && shallow_fits(groups, M, N)) {
    ShallowParams sp{};
    sp.A = A, sp.lda = lda;
    sp.B = B, sp.ldb = ldb;
    sp.C = C, sp.ldc = ldc, sp.stride_c = strideC;
    sp.M = M, sp.N = N, sp.K = K;
    sp.offsets = offsets;
    sp.alpha = alpha, sp.beta = beta;
    sp.row_blocks = (int)shallow_row_blocks(M), sp.column_blocks = (int)shallow_column_blocks(N);
    static void (*const kernels[2][2])(ShallowParams) = {{shallow_kernel<false, false>, shallow_kernel<false, true>},
                                                         {shallow_kernel<true, false>, shallow_kernel<true, true>}};
    void* args[] = {&sp};
    ECGEMM_HIP(h, hipLaunchKernel(reinterpret_cast<const void*>(kernels[transA == ECGEMM_OP_T][transB == ECGEMM_OP_N]),
                                  dim3((unsigned)(groups * (shallow_row_blocks(M) * shallow_column_blocks(N)))), dim3(kShallowThreads), args, 0, h->stream));
    return ECGEMM_OK;
  }
  GroupedParams gp{};
  gp.A = A, gp.lda = lda;
  gp.B = B, gp.ldb = ldb;
  gp.C = C, gp.ldc = ldc, gp.stride_c = strideC;
  gp.M = M, gp.N = N, gp.K = K;
  gp.offsets = offsets;
  gp.along_depth = 1;
  gp.alpha = alpha, gp.beta = beta;
  return launch_grouped(h, mode, transA == ECGEMM_OP_T, transB == ECGEMM_OP_N, groups, gp);
}

ecgemm_status_t ecgemm_sgemm_adapters(ecgemm_handle_t handle, ecgemm_op_t transA, ecgemm_op_t transB, int64_t M, int64_t N,
                                      int64_t K, float alpha, const float* A, int64_t lda, const float* B, int64_t ldb,
                                      int64_t groups, const int64_t* offsets, const int32_t* index, int64_t adapters,
                                      int64_t rank, ecgemm_op_t transD, const float* D, int64_t ldd, int64_t strideD,
                                      ecgemm_op_t transU, const float* U, int64_t ldu, int64_t strideU, const float* scales,
                                      float* H, int64_t ldh, float beta, float* C, int64_t ldc, ecgemm_mode_t mode) {
  ecgemm_handle_t h = handle;
  if (!h) return ECGEMM_ERR_INVALID_ARG;
  ECGEMM_ARG(h, !valid_op(transA), 2, "ecgemm_sgemm_adapters: bad transA");
  ECGEMM_ARG(h, !valid_op(transB), 3, "ecgemm_sgemm_adapters: bad transB");
  ECGEMM_ARG(h, M < 0, 4, "ecgemm_sgemm_adapters: negative M");
  ECGEMM_ARG(h, N < 0, 5, "ecgemm_sgemm_adapters: negative N");
  ECGEMM_ARG(h, K < 0, 6, "ecgemm_sgemm_adapters: negative K");
  ECGEMM_ARG(h, groups < 0, 12, "ecgemm_sgemm_adapters: negative number of groups");
  ECGEMM_ARG(h, adapters < 0, 15, "ecgemm_sgemm_adapters: negative number of adapters");
  ECGEMM_ARG(h, rank < 0, 16, "ecgemm_sgemm_adapters: negative rank");
  ECGEMM_ARG(h, !valid_op(transD), 17, "ecgemm_sgemm_adapters: bad transD");
  ECGEMM_ARG(h, !valid_op(transU), 21, "ecgemm_sgemm_adapters: bad transU");
  ecgemm_status_t st = check_grouped_mode(h, (int)mode, 31, "ecgemm_sgemm_adapters");
  if (st != ECGEMM_OK) return st;
  if (N == 0) return ECGEMM_OK;
  ECGEMM_ARG(h, M > INT_MAX, 4, "ecgemm_sgemm_adapters: M too large");
  ECGEMM_ARG(h, N > INT_MAX, 5, "ecgemm_sgemm_adapters: N too large");
  ECGEMM_ARG(h, K > INT_MAX, 6, "ecgemm_sgemm_adapters: K too large");
  ECGEMM_ARG(h, groups > INT_MAX, 12, "ecgemm_sgemm_adapters: too many groups");
  ECGEMM_ARG(h, adapters > INT_MAX, 15, "ecgemm_sgemm_adapters: too many adapters");
  ECGEMM_ARG(h, rank > kLargestRank, 16, "ecgemm_sgemm_adapters: rank too large");
  ECGEMM_ARG(h, most_grouped_tiles(false, groups, M, N) > kGroupedMostTiles, 4, "ecgemm_sgemm_adapters: M x N too large");
  const bool any = groups > 0 && adapters > 0 && rank > 0;
  ECGEMM_ARG(h, any && bad_offsets(offsets), 13, "ecgemm_sgemm_adapters: null or misaligned offsets");
  ECGEMM_ARG(h, any && (!index || (uintptr_t)index % 4 != 0), 14, "ecgemm_sgemm_adapters: null or misaligned index");
  if (K > 0 && (any || alpha != 0.0f)) {
    ECGEMM_ARG(h, !B, 10, "ecgemm_sgemm_adapters: B is null");
    ECGEMM_ARG(h, ldb < (transB == ECGEMM_OP_N ? K : N), 11, "ecgemm_sgemm_adapters: ldb too small");
    ECGEMM_ARG(h, any && ldb > kGroupedLargestLd, 11, "ecgemm_sgemm_adapters: ldb beyond 2^21");
  }
  if (M > 0 && K > 0 && alpha != 0.0f) {
    ECGEMM_ARG(h, !A, 8, "ecgemm_sgemm_adapters: A is null");
    ECGEMM_ARG(h, lda < (transA == ECGEMM_OP_N ? M : K), 9, "ecgemm_sgemm_adapters: lda too small");
  }
  if (any && K > 0) {
    ECGEMM_ARG(h, !D, 18, "ecgemm_sgemm_adapters: D is null");
    ECGEMM_ARG(h, ldd < (transD == ECGEMM_OP_N ? rank : K), 19, "ecgemm_sgemm_adapters: ldd too small");
    ECGEMM_ARG(h, ldd > kGroupedLargestLd, 19, "ecgemm_sgemm_adapters: ldd beyond 2^21");
    ECGEMM_ARG(h, strideD < 0, 20, "ecgemm_sgemm_adapters: negative strideD");
  }
  if (any && M > 0) {
    ECGEMM_ARG(h, !U, 22, "ecgemm_sgemm_adapters: U is null");
    ECGEMM_ARG(h, ldu < (transU == ECGEMM_OP_N ? M : rank), 23, "ecgemm_sgemm_adapters: ldu too small");
    ECGEMM_ARG(h, ldu > kGroupedLargestLd, 23, "ecgemm_sgemm_adapters: ldu beyond 2^21");
    ECGEMM_ARG(h, strideU < 0, 24, "ecgemm_sgemm_adapters: negative strideU");
  }
  if (rank > 0) {
    ECGEMM_ARG(h, !H, 26, "ecgemm_sgemm_adapters: H is null");
    ECGEMM_ARG(h, ldh < rank, 27, "ecgemm_sgemm_adapters: ldh < rank");
    ECGEMM_ARG(h, ldh > kGroupedLargestLd, 27, "ecgemm_sgemm_adapters: ldh beyond 2^21");
  }
  if (M > 0) {
    ECGEMM_ARG(h, !C, 29, "ecgemm_sgemm_adapters: C is null");
    ECGEMM_ARG(h, ldc < M, 30, "ecgemm_sgemm_adapters: ldc < M");
  }
  const OnDeviceOf device(h);
  if (device.error != hipSuccess) return hip_fail(h, device.error, "hipSetDevice");
  const bool depth_b = transB == ECGEMM_OP_N, project = M > 0 && K > 0 && alpha != 0.0f;
  if (!any) {
    if (rank > 0) {  // H = 0
      const dim3 grid((unsigned)((rank + 255) / 256), (unsigned)std::min<int64_t>(N, 65535));
      hipLaunchKernelGGL(scale_c_kernel, grid, dim3(256), 0, h->stream, rank, N, 0.0f, H, ldh);
      ECGEMM_HIP(h, hipGetLastError());
    }
    if (M == 0) return ECGEMM_OK;
    return sgemm_common(h, transA, transB, M, N, K, alpha, A, lda, B, ldb, beta, C, ldc, mode, nullptr, nullptr, kWorkspaceOfHandle);
  }
  const bool narrow = project && lda <= kGroupedLargestLd && narrow_projection_is_faster(transA == ECGEMM_OP_T, M, N, K, mode) &&
                      narrow_fits(transA == ECGEMM_OP_T, 1, M, N, 0);
  // Projection and adapters in one launch, where both matrices and H are laid out alike (see grouped_kernel), there are tiles
  // enough for half the chip, no more than a few adapters meet in a tile, and the projection is not so deep that splitting
  // first outweighs two passes over C.  Whole calls so / with C written first and the projection added, us, FP16, M x N x K,
  // rank, groups: 4096^3, 16, 4 429 / 438, 64, 64 443 / 466; 4096 x 1024 x 4096, 16, 4 122 / 133, x 512 89 / 88, x 128 95 / 57; 1024 x
  // 2048 x 1024, 16, 4 43 / 51, x 512 37 / 33; 2048 x 6000 x 5120, 64, 4 452 / 524; 8192 x 4096 x 8192, 32, 4 1534 / 1480; BF16 4096^3,
  // 16, 4 610 / 665; 2049 x 1040 x 1500, 20, 61 76 / 100.
  const int64_t chunk = mode == ECGEMM_MODE_FP16_SPLIT ? 64 : 32, added_chunks = (1 + kGroupedTile * groups / N) * ((rank + chunk - 1) / chunk);
  const int64_t tiles = grouped_tiles(M) * grouped_tiles(N);
  const bool one_launch = project && !narrow && transA == transU && depth_b && groups <= kGroupsPerLaunch && lda <= kGroupedLargestLd &&
                          h->log2_scale_a == 0 && h->log2_scale_b == 0 && K <= kAdapterOneLaunchDepth && tiles >= kAdapterOneLaunchTiles && added_chunks <= kAdapterOneLaunchChunks &&
                          std::fabs(alpha) >= 0x1p-16f && std::fabs(alpha) <= 0x1p16f;  // (H is multiplied by scales / alpha)
  // The launches for H and for C before the projection, refused before the first of them where they cannot hold the call
  const bool narrow_down = N < kAdapterDownMeanColumns * groups && narrow_fits(transD == ECGEMM_OP_T, groups, rank, N / groups, 1);
  const int down_fr = narrow_fr(depth_b, 1, N, rank);
  ECGEMM_ARG(h, !narrow_down && !launchable(narrow_row_blocks(down_fr, N), kNarrowThreads), 5, "ecgemm_sgemm_adapters: N too large");
  const bool few = N < 2 * kAdapterUpColumnsShort * groups && launchable(adapter_up_blocks(M, N, kAdapterUpColumnsShort), kAdapterUpThreads);
  const int64_t up_blocks = adapter_up_blocks(M, N, few ? kAdapterUpColumnsShort : kAdapterUpColumns);
  ECGEMM_ARG(h, M > 0 && !narrow && !one_launch && !launchable(up_blocks, kAdapterUpThreads), 4, "ecgemm_sgemm_adapters: M x N too large");
  if (project && !narrow && !one_launch) {  // what the projection would refuse is refused before anything is enqueued
    st = check_sizes(h, M, N, K, mode, 4);
    if (st != ECGEMM_OK) return st;
    const Plan pl = make_plan(M, N, K, mode, h->shape, kOneLaunchSliced);
    if (!pl.shape) return no_plan(h, pl, "ecgemm_sgemm_adapters");
    char* ws = nullptr;
    st = acquire_workspace(h, pl.total_bytes, &ws);
    if (st != ECGEMM_OK) return st;
  }
  // H = op(D) op(B), zero in every column without an adapter: few columns to a group, the adapters are read once, else B is
  if (narrow_down) {
    NarrowParams down{};
    down.A = D, down.lda = ldd, down.stride_a = strideD;
    down.B = B, down.ldb = ldb;
    down.C = H, down.ldc = ldh;
    down.M = rank, down.N = N, down.K = K;
    down.offsets = offsets, down.groups = groups;
    down.index = index, down.matrices = (int)adapters;
    down.alpha = 1.0f, down.beta = 0.0f;
    down.clear_outside = 1;
    st = launch_narrow(h, transD == ECGEMM_OP_T, depth_b, down);
    if (st != ECGEMM_OK) return st;
  } else {
    AdapterDownParams down{};
    down.B = B, down.ldb = ldb;
    down.D = D, down.ldd = ldd, down.stride_d = strideD;
    down.N = N, down.K = K, down.rank = rank;
    down.offsets = offsets, down.groups = groups;
    down.index = index, down.matrices = (int)adapters;
    down.H = H, down.ldh = ldh;
    const bool depth_d = transD == ECGEMM_OP_T;
    void (*const kernel)(AdapterDownParams) = down_fr == 4 ? (depth_d ? adapter_down_kernel<false, true, 4> : adapter_down_kernel<false, false, 4>)
                                              : down_fr == 2
                                                  ? (depth_d ? adapter_down_kernel<true, true, 2> : adapter_down_kernel<true, false, 2>)
                                                  : (depth_d ? adapter_down_kernel<true, true, 1> : adapter_down_kernel<true, false, 1>);
    void* args[] = {&down};
    ECGEMM_HIP(h, hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)narrow_row_blocks(down_fr, N), groups > 1 ? 2 : 1),
                                  dim3(kNarrowThreads), args, 0, h->stream));
  }
  if (M == 0) return ECGEMM_OK;
  if (narrow) {
    // the projection reads its matrix once (and once more for every 32 columns), and adds the adapters to what it writes
    NarrowParams np{};
    np.A = A, np.lda = lda;
    np.B = B, np.ldb = ldb;
    np.C = C, np.ldc = ldc;
    np.M = M, np.N = N, np.K = K;
    np.alpha = alpha, np.beta = beta;
    np.U = U, np.ldu = ldu, np.stride_u = strideU, np.rank = rank, np.u_depth = transU == ECGEMM_OP_T;
    np.H = H, np.ldh = ldh, np.scales = scales;
    np.adapter_offsets = offsets, np.adapter_groups = groups, np.index = index, np.matrices = (int)adapters;
    return launch_narrow(h, transA == ECGEMM_OP_T, depth_b, np);
  }
  if (one_launch) {
    GroupedParams gp{};
    gp.A = A, gp.lda = lda;
    gp.B = B, gp.ldb = ldb;
    gp.C = C, gp.ldc = ldc;
    gp.M = M, gp.N = N, gp.K = K;
    gp.offsets = offsets, gp.groups = (int)groups;
    gp.index = index, gp.matrices = (int)adapters, gp.scales = scales;
    gp.tiles_m = (int)grouped_tiles(M), gp.tiles_n = (int)grouped_tiles(N);
    gp.U = U, gp.ldu = ldu, gp.stride_u = strideU, gp.rank = rank;
    gp.H = H, gp.ldh = ldh;
    gp.prescale_a = gp.prescale_b = gp.out_scale = 1.0f;
    gp.slices = 1;
    gp.alpha = alpha, gp.beta = beta;
    const bool depth_a = transA == ECGEMM_OP_T;
    const grouped_fn_t kernel = mode == ECGEMM_MODE_FP16_SPLIT
                                    ? (depth_a ? grouped_kernel<kMethodFp16Split, true, true, false, true> : grouped_kernel<kMethodFp16Split, false, true, false, true>)
                                    : (depth_a ? grouped_kernel<kMethodBf16Full, true, true, false, true> : grouped_kernel<kMethodBf16Full, false, true, false, true>);
    const int64_t grid = std::max(std::min<int64_t>(tiles, h->compute_units), (tiles + kGroupedTilesPerBlock - 1) / kGroupedTilesPerBlock);
    void* args[] = {&gp};
    ECGEMM_HIP(h, hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)grid), dim3(kGroupedThreads), args, 0, h->stream));
    return ECGEMM_OK;
  }
  // C = scales op(U) H + beta C first, which the projection adds to as it writes: it finds what it reads in the caches
  AdapterUpParams up{};
  up.U = U, up.ldu = ldu, up.stride_u = strideU;
  up.H = H, up.ldh = ldh;
  up.C = C, up.ldc = ldc;
  up.M = M, up.N = N, up.rank = rank;
  up.offsets = offsets, up.groups = groups;
  up.index = index, up.matrices = (int)adapters;
  up.scales = scales, up.beta = beta;
  up.row_blocks = (int)adapter_up_row_blocks(M);
  // Few columns to a request: a block's runs follow each other at 2 us each.  Calls with 64 / 8 columns a block, 128 requests of
  // a column, rank 16: 4096 x 4096 170 us / 53, 1024 x 2048 150 / 30; 512 of a column, 8192 x 2048, 198 / 108.
  void (*const up_kernel)(AdapterUpParams) =
      transU == ECGEMM_OP_T ? (few ? adapter_up_kernel<true, kAdapterUpColumnsShort> : adapter_up_kernel<true, kAdapterUpColumns>)
                            : (few ? adapter_up_kernel<false, kAdapterUpColumnsShort> : adapter_up_kernel<false, kAdapterUpColumns>);
  void* up_args[] = {&up};
  ECGEMM_HIP(h, hipLaunchKernel(reinterpret_cast<const void*>(up_kernel), dim3((unsigned)up_blocks), dim3(kAdapterUpThreads), up_args,
                                0, h->stream));
  if (!project) return ECGEMM_OK;
  return sgemm_common(h, transA, transB, M, N, K, alpha, A, lda, B, ldb, 1.0f, C, ldc, mode, nullptr, nullptr, kWorkspaceOfHandle);
}

}  // extern "C"
