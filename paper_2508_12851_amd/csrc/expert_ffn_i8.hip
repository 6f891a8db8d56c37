// The expert FFN of layers whose expert weights are 8-bit matrices (prism.h, PRISM_WEIGHTS_INT8).
//
//   xq, sx = tokens in 8 bits, a scale per token
//   h[r, f] = silu( (xq[tok(r)] . Wq_gate^e[f]) sx s_gate[f] ) * ( (xq[tok(r)] . Wq_up^e[f]) sx s_up[f] )
//   hq, sh = h in 8 bits, a scale per row
//   y[r, n] = (hq[r] . Wq_down^e[n]) sh[r] s_down[n]
//
// Four steps: tokens to 8 bits, gate/up product with silu(gate) * up in its epilogue (fp32), h to 8 bits, down product.  The scale of a
// row of h is known only once all its columns are, which are spread over the machine: hence the step between the products.
// The products are those of grouped_gemm.h in the tiles that bf16 weights take for as many bytes (ffn_paths.h).
#include "ffn_tiles.h"

namespace prism {
namespace {

template <typename C1, typename C2, bool SPLIT_DOWN, bool STREAM_B, bool ROTATE, bool WIDTHS>
prism_status run_i8_ffn(const prism_layer_desc& d, const void* x, const prism_expert_weights& w, const int32_t* local_src,
                        const int32_t* local_offsets, int T, void* y, const Workspace& ws, hipStream_t st,
                        void* const* stage_events, const int32_t** deferred_splits, bool schedules_built) {
  using gg::GemmArgs;
  const int A = T * d.top_k, rows = A + d.n_shared * T;
  const int k1 = contraction(d, d.hidden), k2 = contraction(d, d.ffn);
  // the k-tile ring of a workgroup must not be longer than its contraction slice
  if (k1 / C1::BK < C1::STAGES - 1 || k2 / C2::BK < C2::STAGES - 1) return PRISM_ERR_UNSUPPORTED;
  int32_t* const sched1 = ws.tiles;
  int32_t* const sched2 = ws.tiles + tile_table_ints(d, T);
  const FfnShapes f = shapes_of<C1, C2, SPLIT_DOWN, ROTATE, WIDTHS>(d, T);   // as ffn_schedule_shapes()
  constexpr bool kPrefill = !SPLIT_DOWN && C2::BM == 256;

  // Prefill tiles read 64 bytes of a row per k-tile, half a line of a gathered one: where a copy of the tokens in row order pays
  // for bf16 weights, they are quantised in row order into tiles (once per pick).  Other batches gather.
  const bool in_rows = kPrefill && pack_rows_pays(d, T);
  QuantizeArgs qx{};
  qx.src = x; qx.ld = d.hidden; qx.cols = d.hidden; qx.dst = ws.xq; qx.scale = ws.x_scale;
  qx.rows = T;
  if (in_rows) {
    qx.rows = rows;
    qx.tiled = 1;
    qx.places = ws.row_places;
    qx.local_src = local_src; qx.local_offsets = local_offsets;
    qx.E = d.n_experts; qx.A = A; qx.T = T; qx.top_k = d.top_k;
  }
  if (schedules_built) PRISM_TRY(launch_quantize(qx, PRISM_BF16, st));
  else PRISM_TRY(launch_quantize_tokens(d, qx, local_offsets, T, ws.tiles, st));
  trace(stage_events, PRISM_STAGE_DISPATCH, 1, st);   // counts as dispatch: its end is recorded anew

  GemmArgs g1{};
  g1.A = (const uint16_t*)ws.xq;
  g1.B0 = w.w_gate; g1.B1 = w.w_up; g1.SB0 = w.shared_w_gate; g1.SB1 = w.shared_w_up;
  g1.Cpart = (float*)ws.h;
  g1.sched = sched1;
  g1.b_bytes = (uint32_t)i8_elements(d.ffn, d.hidden);
  g1.K = k1; g1.N = d.ffn; g1.E = d.n_experts;
  g1.b_tiled = 1;
  g1.a_scale = ws.x_scale;
  g1.a_scale_bytes = (uint32_t)(in_rows ? rows : T) * 4;
  if (in_rows) {
    g1.a_bytes = (uint32_t)i8_elements(rows, d.hidden);
    g1.local_src = ws.row_places;
    g1.src_bytes = (uint32_t)rows * 4;
    g1.top_k = 1;
    g1.a_tiled = 1;
    g1.a_pitch = 64;
    g1.a_kstep = 1024;
  } else {
    g1.a_bytes = (uint32_t)((size_t)T * k1 * 2);
    g1.local_src = local_src;
    g1.src_bytes = (uint32_t)A * 4;
    g1.top_k = d.top_k;
    g1.a_pitch = (uint32_t)k1 * 2;
    g1.a_kstep = 64;
  }
  trace(stage_events, PRISM_STAGE_FFN_UP, 0, st);
  if constexpr (WIDTHS)
    PRISM_TRY((gg::launch_gemm_widths<C1::BM, C1::BN, C1::BK, C1::STAGES, kWideStages, true, false, true>(g1, st)));
  else
    PRISM_TRY((gg::launch_gemm<C1::BM, C1::BN, 2, 2, C1::BK, C1::STAGES, true, false, ROTATE, STREAM_B, false, true>(
        g1, gg::sched_capacity(d, T, C1::BM, f.nt1), st)));
  trace(stage_events, PRISM_STAGE_FFN_UP, 1, st);

  trace(stage_events, PRISM_STAGE_FFN_DOWN, 0, st);
  QuantizeArgs qh{};
  qh.src = ws.h; qh.ld = d.ffn; qh.cols = d.ffn; qh.dst = ws.hq; qh.scale = ws.h_scale;
  qh.rows = rows;
  qh.tiled = 1;
  qh.local_offsets = local_offsets;
  qh.E = d.n_experts; qh.A = A;
  PRISM_TRY(launch_quantize(qh, PRISM_F32, st));

  GemmArgs g2{};
  g2.A = (const uint16_t*)ws.hq;
  g2.B0 = w.w_down; g2.SB0 = w.shared_w_down;
  g2.C = (uint16_t*)y;
  g2.Cpart = SPLIT_DOWN ? ws.part : ws.slice_part;
  g2.c_rows = rows;
  g2.sched = sched2; g2.local_src = local_src;
  g2.a_bytes = (uint32_t)i8_elements(rows, d.ffn);
  g2.b_bytes = (uint32_t)i8_elements(d.hidden, d.ffn);
  g2.K = k2; g2.N = d.hidden; g2.top_k = d.top_k; g2.E = d.n_experts;
  g2.b_tiled = g2.a_tiled = 1;
  g2.a_pitch = (uint32_t)k2 * 2;
  g2.a_kstep = 1024;
  g2.a_scale = ws.h_scale;
  g2.a_scale_bytes = (uint32_t)rows * 4;
  const int32_t* n_splits = sched2 + 2;
  const int capacity2 = gg::sched_capacity(d, T, C2::BM, f.nt2);
  if constexpr (WIDTHS)
    PRISM_TRY((gg::launch_gemm_widths<C2::BM, C2::BN, C2::BK, C2::STAGES, kWideStages, false, SPLIT_DOWN, true>(g2, st)));
  else
    PRISM_TRY((gg::launch_gemm<C2::BM, C2::BN, 2, 2, C2::BK, C2::STAGES, false, SPLIT_DOWN, ROTATE, STREAM_B, false, true>(
        g2, capacity2, st)));
  if constexpr (kPrefill && C2::STAGES == 4) {   // (layers whose last round may be cut have long contractions)
    if (f.slice_kt2 > 0) {   // the cut last round: one slice entry per workgroup, fp32 partial tiles
      PRISM_TRY((gg::launch_gemm<C2::BM, C2::BN, 2, 2, C2::BK, C2::STAGES, false, false, false, false, true, true>(
          g2, capacity2, st)));
      PRISM_TRY(launch_sum_slices(d, sched2, capacity2, ws.slice_part, y, st));
    }
  }
  if (SPLIT_DOWN && deferred_splits != nullptr)
    *deferred_splits = n_splits;   // the caller's combine sums the slices itself
  else if (SPLIT_DOWN)
    PRISM_TRY(launch_reduce_splits(d, T, ws.part, local_offsets, n_splits, y, st));
  trace(stage_events, PRISM_STAGE_FFN_DOWN, 1, st);
  return PRISM_OK;
}

}  // namespace

prism_status launch_expert_ffn_i8(const prism_layer_desc& d, const void* x, const prism_expert_weights& w,
                                  const int32_t* local_src, const int32_t* local_offsets, int T, void* y, const Workspace& ws,
                                  hipStream_t st, void* const* stage_events, const int32_t** deferred_splits,
                                  bool schedules_built) {
  if (deferred_splits != nullptr) *deferred_splits = nullptr;
  if (T == 0) return PRISM_OK;
  return select_path(d, T, [&](auto path) {
    using P = decltype(path);
    return run_i8_ffn<typename P::C1, typename P::C2, P::kSplitDown, P::kStreamB, P::kRotate, P::kWidths>(
        d, x, w, local_src, local_offsets, T, y, ws, st, stage_events, deferred_splits, schedules_built);
  });
}

}  // namespace prism
