// The tile shapes of the expert FFN's paths (ffn_paths.h) on the matrix cores, for bf16 weights and, with the
// same bytes per k-tile, for 8-bit ones.
#ifndef PRISM_FFN_TILES_H_
#define PRISM_FFN_TILES_H_

#include "grouped_gemm.h"
#include "prism_internal.h"

namespace prism {
namespace {

template <int BM_, int BN_, int BK_, int STAGES_> struct TileCfg {
  static constexpr int BM = BM_, BN = BN_, BK = BK_, STAGES = STAGES_;
};

// Fixed cost of one round of items of a split down projection, as weight bytes a workgroup
// could have streamed meanwhile (first loads of the ring, epilogue, partial-tile stores): fitted
// to the times of a 32-token batch of the 4096 x 14336 layer run with 2 to 8 splits.
constexpr float kSplitRoundBytes = 14 * 8192.f;

// Wide tiles of a path with two widths (schedule.h, "Two widths"): ring of their own, fewest items.
constexpr int kWideStages = 3;
constexpr int kWideItemsUp = 150, kWideItemsDown = 48;

// What the schedule builders need to know about a path's two GEMMs (C1: gate/up, C2: down).
template <typename C1, typename C2, bool SPLIT_DOWN, bool ROTATE, bool WIDTHS>
FfnShapes shapes_of(const prism_layer_desc& d, int T) {
  FfnShapes f{};
  f.bm1 = C1::BM;
  f.nt1 = ceil_div(d.ffn, C1::BN / 2);     // GEMM1 tile: BN/2 gate rows + BN/2 up rows
  f.bm2 = C2::BM;
  f.nt2 = ceil_div(d.hidden, C2::BN);
  f.interleave = ROTATE;
  // prefill tiles: the down projection's last round may be cut along its contraction
  f.slice_kt2 = !SPLIT_DOWN && C2::BM == 256 && down_slicing_applies(d, T) ? contraction(d, d.ffn) / C2::BK : 0;
  if (SPLIT_DOWN) {
    f.split_kt2 = contraction(d, d.ffn) / C2::BK;
    f.split_min_kt2 = C2::STAGES - 1;      // a slice must be at least as long as the k-tile ring
    f.split_wgs2 = gg::gemm_wgs_per_xcd<C2::BM, C2::BN, 2, C2::BK, C2::STAGES, false, true>();
    const float kt_bytes = (float)(C2::BN * C2::BK * 2);   // weight bytes of one k-tile
    f.split_round_kt2 = kSplitRoundBytes / kt_bytes;
    // one more split: every row written once more as fp32 and read once more, shared by all workgroups
    f.split_row_kt2 = (float)d.hidden * 8.f / (float)(gg::kXcds * f.split_wgs2) / kt_bytes;
  }
  if (WIDTHS) {
    static_assert(!WIDTHS || (SPLIT_DOWN && ROTATE && kWideStages <= C1::STAGES && kWideStages <= C2::STAGES),
                  "the wide tiles' ring is no longer than the slices that the narrow ones allow");
    f.wide_nt1 = ceil_div(d.ffn, C1::BN);
    f.wide_nt2 = ceil_div(d.hidden, 2 * C2::BN);
    f.wide_items1 = kWideItemsUp;
    f.wide_items2 = kWideItemsDown;
  }
  return f;
}

// One tile path of the bf16 FFN: tile shapes of the two GEMMs, whether the down projection is
// split along its contraction, whether the weight loads are marked non-temporal, whether the items
// are dealt to the XCDs one by one with rotated contractions (grouped_gemm.h, ROTATE), whether the
// schedule may choose tiles twice as wide instead.
template <typename C1_, typename C2_, bool SPLIT_DOWN_, bool STREAM_B_, bool ROTATE_, bool WIDTHS_ = false> struct Path {
  using C1 = C1_;
  using C2 = C2_;
  static constexpr bool kSplitDown = SPLIT_DOWN_, kStreamB = STREAM_B_, kRotate = ROTATE_, kWidths = WIDTHS_;
};

// Calls fn(Path<...>{}) with the path that serves a bf16 batch of T tokens of layer d (ffn_paths.h).
template <typename Fn>
auto select_path(const prism_layer_desc& d, int T, Fn&& fn) {
  using Decode = TileCfg<64, 128, 64, 4>;
  using Square = TileCfg<128, 128, 64, 4>;
  using Wide = TileCfg<128, 256, 64, 3>;
  switch (ffn_path(d, T)) {
    case FfnPath::kDecodeTiled: return fn(Path<TileCfg<64, 128, 32, 8>, TileCfg<64, 128, 32, 8>, true, true, true>{});
    case FfnPath::kDecode: return fn(Path<Decode, Decode, true, true, true>{});
    case FfnPath::kDecodeShort: return fn(Path<TileCfg<64, 128, 32, 3>, TileCfg<64, 128, 32, 3>, true, true, true>{});
    case FfnPath::kStream: return fn(Path<Square, Square, true, true, true, true>{});
    case FfnPath::kSplitSquare: return fn(Path<Square, Square, true, false, false>{});
    case FfnPath::kSplitWide: return fn(Path<Wide, Wide, true, false, false>{});
    case FfnPath::kFewRows64: return fn(Path<Decode, Decode, false, true, false>{});
    case FfnPath::kFewRows128: return fn(Path<Wide, Square, false, false, false>{});
    case FfnPath::kPrefill: return fn(Path<TileCfg<256, 256, 32, 4>, TileCfg<256, 256, 32, 4>, false, false, false>{});
    default: return fn(Path<TileCfg<256, 256, 32, 3>, TileCfg<256, 256, 32, 3>, false, false, false>{});
  }
}

}  // namespace
}  // namespace prism
#endif  // PRISM_FFN_TILES_H_
