// out[m, n] = (sum_k aq[m, k] bq[n, k]) s_a[m] s_b[n] of two 8-bit matrices (prism.h): the grouped GEMM's kernel without groups
// (grouped_gemm.h, DENSE).
//
// Few rows: the weights are streamed once, in 64 x 128 tiles, and the contraction of a tile is shared by several workgroups where
// the tiles alone would leave compute units without one; they leave fp32 partial sums that a last kernel adds in their order.
#include "grouped_gemm.h"

namespace prism {
namespace {

constexpr int kMaxSplits = 8;
constexpr int kWorkgroups = 256;      // one per CU
constexpr size_t kMaxPartialBytes = (size_t)64 << 20;

enum class Tile { kFew, kSquare, kLarge };
struct Plan {
  Tile tile;
  int splits;
};

constexpr int kFewRows = 64;
// What a tile's contraction costs to begin and end, in k-tiles of 64 bytes.
constexpr float kRoundKt = 14.f;

Plan plan_of(int M, int N, int K) {
  const int kt = (int)(i8_row_bytes(K) / 64);
  auto items = [&](int bm, int bn) { return (long long)ceil_div(M, bm) * ceil_div(N, bn); };
  if (M > kFewRows && items(256, 256) >= kWorkgroups) return Plan{kt >= 3 ? Tile::kLarge : Tile::kSquare, 1};
  const bool few = M <= kFewRows;
  const long long n = few ? items(64, 128) : items(128, 128);
  const int ring = few ? 7 : 6;       // k-tiles of 64 bytes that a split must have
  int best = 1;
  float cost = INFINITY;
  for (int s = 1; s <= kMaxSplits; ++s) {
    if (s > 1 && (kt / s < ring || (size_t)s * M * align_up(N, 4) * 4 > kMaxPartialBytes)) break;
    const float rounds = (float)((n * s + kWorkgroups - 1) / kWorkgroups);
    const float c = rounds * ((float)ceil_div(kt, s) + kRoundKt) + (s > 1 ? 12.f + 0.002f * (float)s * M * N / 4096.f : 0.f);
    if (c < cost) {
      cost = c;
      best = s;
    }
  }
  return Plan{few ? Tile::kFew : Tile::kSquare, best};
}

// out = sum of the splits' partial sums, in their order: four columns per thread.
__global__ __launch_bounds__(256) void reduce_dense_kernel(const float* __restrict__ part, int splits, int M, int N, void* out,
                                                           long long ldo, int f32, int vec) {
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
  gg::store_dense(out, ldo, f32, vec, row, n, N, sum);
}

template <int BM, int BN, int BK, int STAGES, bool STREAM_B, bool CAN_SPLIT = true>
prism_status launch_tiles(gg::GemmArgs& g, long long items, hipStream_t st) {
  const int per_xcd = (int)((items + gg::kXcds - 1) / gg::kXcds);
  if constexpr (CAN_SPLIT)
    if (g.dense_splits > 1) return gg::launch_gemm<BM, BN, 2, 2, BK, STAGES, false, true, STREAM_B, STREAM_B, false, true, true>(g, per_xcd, st);
  return gg::launch_gemm<BM, BN, 2, 2, BK, STAGES, false, false, STREAM_B, STREAM_B, false, true, true>(g, per_xcd, st);
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
  if ((long long)ceil_div(M, 64) * ceil_div(N, 128) >= (1LL << 30)) return PRISM_ERR_UNSUPPORTED;
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
  const int es = g.dense_f32 ? 4 : 2;
  g.dense_vec = ((uintptr_t)out & (4 * es - 1)) == 0 && ldo % 4 == 0;
  g.dense_splits = plan.splits;
  auto items = [&](int bm, int bn) { return (long long)ceil_div(M, bm) * ceil_div(N, bn); };
  switch (plan.tile) {
    case Tile::kFew:
      if (g.K / 32 >= 7) PRISM_TRY((launch_tiles<64, 128, 32, 8, true>(g, items(64, 128), st)));
      else PRISM_TRY((launch_tiles<64, 128, 32, 3, true, false>(g, items(64, 128), st)));
      break;
    case Tile::kSquare:
      if (g.K / 64 >= 3) PRISM_TRY((launch_tiles<128, 128, 64, 4, false>(g, items(128, 128), st)));
      else PRISM_TRY((launch_tiles<128, 128, 32, 3, false, false>(g, items(128, 128), st)));
      break;
    case Tile::kLarge:
      PRISM_TRY((launch_tiles<256, 256, 32, 4, false, false>(g, items(256, 256), st)));
      break;
  }
  if (plan.splits > 1) {
    const long long threads = (long long)M * (align_up(N, 4) / 4);
    hipLaunchKernelGGL(reduce_dense_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, (const float*)workspace,
                       plan.splits, M, N, out, ldo, g.dense_f32, g.dense_vec);
    PRISM_CHECK_LAUNCH();
  }
  return PRISM_OK;
}

}  // namespace prism
