// out[m, n] = (sum_k aq[m, k] bq[n, k]) s_a[m] s_b[n] of two 8-bit matrices (prism.h): the grouped GEMM's kernel without groups
// (grouped_gemm.h, DENSE).
//
// Four tiles (matmul_i8_plan.h); where they alone would leave compute units without one, the contraction of a tile is shared by several
// workgroups, which leave fp32 partial sums that a last kernel adds in their order.  Bound: large products by the power of the matrix
// cores (8192 x 8192 x 8192 423 us, 2600 Tops; all zeros 298 us), few rows by streaming the weights, small ones by the latency of
// their k-tiles.
#include "grouped_gemm.h"
#include "matmul_i8_plan.h"

namespace prism {
namespace {

using namespace mm8;

// out = sum of the splits' partial sums, in their order: four columns per thread.
__global__ __launch_bounds__(256) void reduce_dense_kernel(const float* __restrict__ part, int splits, int M, int N, void* out,
                                                           long long ldo, int f32) {
  const int pitch = (N + 3) / 4 * 4, quads = pitch / 4;
  const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (long long)M * quads) return;
  const int row = (int)(i / quads), n = (int)(i - (long long)row * quads) * 4;
  f32x4 v[kMaxSplits];
#pragma unroll
  for (int s = 0; s < kMaxSplits; ++s)
    if (s < splits) v[s] = *reinterpret_cast<const f32x4*>(part + ((size_t)s * M + row) * pitch + n);
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < kMaxSplits; ++s)
    if (s < splits) sum += v[s];
  gg::store_dense(out, ldo, f32, row, n, N, sum);
}

template <int BM, int BN, int BK, int STAGES, bool CAN_SPLIT>
prism_status launch_tiles(const gg::GemmArgs& g, hipStream_t st) {
  const long long items = (long long)ceil_div(g.c_rows, BM) * ceil_div(g.N, BN);
  const int per_xcd = (int)((items + gg::kXcds - 1) / gg::kXcds);
  if constexpr (CAN_SPLIT)
    if (g.dense_splits > 1) return gg::launch_gemm<BM, BN, 2, 2, BK, STAGES, false, true, false, false, false, true, true>(g, per_xcd, st);
  return gg::launch_gemm<BM, BN, 2, 2, BK, STAGES, false, false, false, false, false, true, true>(g, per_xcd, st);
}

}  // namespace

// A bound for every number of rows up to max_rows.
size_t matmul_i8_workspace_bytes(int max_rows, int N, int K) {
  (void)K;
  return align_up(std::min((size_t)kMaxSplits * max_rows * align_up(N, 4) * 4, kMaxPartialBytes) + 1, 256);
}

prism_status launch_matmul_i8(const void* a, const void* b, int M, int N, int K, void* out, long long ldo, int out_dtype,
                              void* workspace, hipStream_t st) {
  if (M == 0) return PRISM_OK;
  constexpr size_t kMaxOperandBytes = 0xFFFF0000ull;    // 32-bit offsets
  if (i8_elements(M, K) >= kMaxOperandBytes || i8_elements(N, K) >= kMaxOperandBytes) return PRISM_ERR_UNSUPPORTED;
  if ((long long)ceil_div(M, 64) * ceil_div(N, 64) >= (1LL << 30)) return PRISM_ERR_UNSUPPORTED;
  const Plan plan = plan_of(M, N, K);
  gg::GemmArgs g{};
  g.A = (const uint16_t*)a;
  g.Cpart = (float*)workspace;
  g.c_rows = M;
  g.a_bytes = (uint32_t)i8_elements(M, K);
  g.b_bytes = (uint32_t)i8_elements(N, K);
  g.K = (int)(i8_row_bytes(K) / 2);
  g.N = N;
  g.top_k = 1;
  g.a_tiled = g.b_tiled = 1;
  g.a_kstep = 1024;
  g.a_scale = (const float*)((const uint8_t*)a + i8_elements(M, K));
  g.a_scale_bytes = (uint32_t)M * 4;
  g.dense_b = b;
  g.dense_out = out;
  g.dense_ldo = ldo;
  g.dense_f32 = out_dtype == PRISM_F32;
  g.dense_splits = plan.splits;
  switch (plan.tile) {
    case Tile::k64x64: PRISM_TRY((launch_tiles<64, 64, 64, 4, true>(g, st))); break;
    case Tile::k64x128: PRISM_TRY((launch_tiles<64, 128, 64, 4, true>(g, st))); break;
    case Tile::k128x128: PRISM_TRY((launch_tiles<128, 128, 64, 4, true>(g, st))); break;
    case Tile::k256x256: PRISM_TRY((launch_tiles<256, 256, 32, 4, false>(g, st))); break;
    case Tile::kShort: PRISM_TRY((launch_tiles<128, 128, 32, 3, false>(g, st))); break;
  }
  if (plan.splits > 1) {
    const long long threads = (long long)M * (align_up(N, 4) / 4);
    hipLaunchKernelGGL(reduce_dense_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, (const float*)workspace,
                       plan.splits, M, N, out, ldo, g.dense_f32);
    PRISM_CHECK_LAUNCH();
  }
  return PRISM_OK;
}

}  // namespace prism
