// Balance loss of a batch's routing and the backward pass of the router (prism.h, prism_balance_loss and
// prism_route_backward): what the activation counts f_n^l(e) of the paper's Sec. III-B are to a router that learns.
//
//   p[t, e]  = softmax(logits[t])             P[g, e] = mean of p[t, e] over the n tokens of group g that count
//   loss[g]  = E / (k n) sum_e counts[g, e] P[g, e]
//   d loss / d logits[t, e] = p[t, e] (u_e - sum_j u_j p[t, j]),   u_e = E counts[g, e] / (k n^2)
//
// A constant in all u_e drops out, so u is formed from E counts[e] - sum counts, a whole number: near an even spread the
// counts themselves would cancel to a small difference in fp32.
//
// Rows: a token's E logits lie on 2^n lanes with 4 consecutive experts each, so that a wavefront holds one row of 256
// experts or 64 rows of 4, and row sums are exchanges between lanes.  Both passes read the logits once: 65531 tokens of 256
// experts (67 MB) 17 us for the sums (3.9 TB/s) and 8 to add their 256 parts, 34 us for the gradient (3.9 TB/s in and out; a
// large copy reaches 4.8): the vector ALU, about 100 and 210 instructions a row, takes nearly as long as memory.  Below a few MB
// the launches' latency: 8192 tokens of 64 experts in 16 groups 9 + 5 us.
#include <type_traits>

#include "prism_internal.h"

namespace prism {
namespace {

constexpr int kThreads = 1024;          // of balance_kernel
constexpr int kFinishThreads = 1024;
constexpr int kBackThreads = 256;
constexpr int kMaxE = PRISM_MAX_EXPERTS;

struct RowArgs {
  const float* logits;        // [T, E]
  const int32_t* topk_idx;    // [T, k]
  const uint8_t* mask;        // [T] or NULL
  int T, E, k;
  int group;                  // tokens of a group
  int parts, part_rows;       // workgroups of a group and the tokens of each
  int first_wg;               // workgroups of the launches before this one
};

// Tokens [first, end) of this workgroup: of the workgroups of all launches, part w % parts of group w / parts.
struct Rows {
  int group, part, first, end;
};
__device__ __forceinline__ Rows rows_of(const RowArgs& a) {
  const int w = a.first_wg + blockIdx.x, g = w / a.parts, part = w % a.parts;
  const long long begin = (long long)g * a.group;     // (groups may be longer than the batch)
  const int stop = (int)min(begin + a.group, (long long)a.T);
  const int first = (int)min(begin + (long long)part * a.part_rows, (long long)stop);
  return Rows{g, part, first, (int)min((long long)first + a.part_rows, (long long)stop)};
}

// The sum (or maximum) over the LPR lanes of a row, in all of them.
template <int LPR, typename F> __device__ __forceinline__ float over_row(float v, F&& f) {
  if constexpr (LPR > 1) v = f(v, row_xor<1>(v));
  if constexpr (LPR > 2) v = f(v, row_xor<2>(v));
  if constexpr (LPR > 4) v = f(v, row_xor<4>(v));
  if constexpr (LPR > 8) v = f(v, row_xor<8>(v));
  if constexpr (LPR == 32) v = f(v, __shfl_xor(v, 16));
  if constexpr (LPR == 64) {                    // (the row is the wavefront: its four parts through scalar registers)
    auto part = [&](int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); };
    v = f(f(part(0), part(16)), f(part(32), part(48)));
  }
  return v;
}

// e^x for x <= 0 by the hardware's exp2, which is within 1 ulp: the product with log2 e is off by |x| 2^-24 of the result's value.
__device__ __forceinline__ float exp_neg(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ float add(float a, float b) { return a + b; }

// Sets of rows that a wavefront has in flight.
template <int LPR> constexpr int ahead_of = LPR >= 16 ? 4 : 2;
template <int LPR> constexpr int back_ahead_of = LPR >= 16 ? 2 : 1;

// The 4 logits of this lane; experts past the last one have -inf.
__device__ __forceinline__ f32x4 load_row(const RowArgs& a, int row, int e0) {
  const float* p = a.logits + (size_t)row * a.E + e0;
  f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
  if (e0 + 4 <= a.E) {
    v = reinterpret_cast<const Unaligned<f32x4, 4>*>(p)->v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e0 + i < a.E) v[i] = p[i];
  }
  return v;
}

// softmax over the lanes of a row, in place.  An expert at -inf has probability 0, and so have all of a row of nothing else.
template <int LPR> __device__ __forceinline__ void softmax_row(f32x4& v) {
  float m = over_row<LPR>(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), [](float x, float y) { return fmaxf(x, y); });
  if (m == -INFINITY) m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = exp_neg(v[i] - m);
  const float s = over_row<LPR>((v[0] + v[1]) + (v[2] + v[3]), add);
  const float inv = s > 0.f ? 1.0f / s : s;     // (a NaN stays one)
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] *= inv;
}

// A group's results from its sums: probs, loss and the counts.  sum_p of expert threadIdx.x, in 64 bits; all threads call it.
__device__ __forceinline__ void finish_group(int g, int E, int k, int n, int count, double sum_p, int32_t* counts, float* probs,
                                             int32_t* n_tokens, float* loss) {
  constexpr int kWaves = kMaxE / 64;
  __shared__ double s_term[kWaves];
  const int e = threadIdx.x;
  double term = 0.0;
  if (e < E) {
    const double p = n > 0 ? sum_p / n : 0.0;
    counts[(size_t)g * E + e] = count;
    probs[(size_t)g * E + e] = (float)p;
    term = (double)count * p;
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) term += __shfl_xor(term, off);
  if (e < kMaxE && (e & 63) == 0) s_term[e >> 6] = term;
  __syncthreads();
  if (e == 0) {
    term = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) term += s_term[w];
    n_tokens[g] = n;
    loss[g] = n > 0 ? (float)(term * E / ((double)k * n)) : 0.f;
  }
}

static_assert(kThreads >= kMaxE, "a thread per expert");

// What workgroups leave for one another.  Of the workgroups of balance_kernel: probabilities [kParts][E4], counts [kParts][E4] and
// tokens [kParts], with E4 = E rounded up to 4; of those of finish_kernel: their shares of a group's loss [kParts][kMaxPieces],
// and how many of a group's have left theirs [kParts].  (Groups that have parts are fewer than kParts.)
constexpr int kParts = 256;       // workgroups that share the tokens of a batch in balance_kernel, about
constexpr int kPieceLanes = 8;    // experts of a workgroup of finish_kernel, by fours
constexpr int kMaxPieces = kMaxE / 4 / kPieceLanes;
struct Partial {
  double* terms;
  float* probs;
  int* counts;
  int* n;
  unsigned* done;
  int E4;
};
size_t partial_bytes(int E) { return (size_t)kParts * (kMaxPieces * 8 + 2 * align_up(E, 4) * 4 + 2 * 4); }
Partial partial_of(void* base, int E) {
  const int E4 = (int)align_up(E, 4);
  double* const terms = (double*)base;
  float* const probs = (float*)(terms + kParts * kMaxPieces);
  int* const counts = (int*)probs + (size_t)kParts * E4;
  int* const n = counts + (size_t)kParts * E4;
  return Partial{terms, probs, counts, n, (unsigned*)n + kParts, E4};
}

// Sums over a part of a group's tokens.  parts == 1: the group's results; else partial sums for finish_kernel.  A lane adds the
// probabilities of its experts over kHeldRows rows in fp32 and these sums in 64 bits, so that their error does not grow with
// the number of tokens (1024 equal rows of a lane in one fp32 sum: off by up to 2^-16; 65536 tokens of 256 experts are 16 of a lane);
// the wavefronts' sums are added in their order; the counts are whole numbers, whose order does not matter.
constexpr int kHeldRows = 16;
template <int LPR>
__global__ __launch_bounds__(kThreads) void balance_kernel(const RowArgs a, const Partial partial, int32_t* __restrict__ counts,
                                                           float* __restrict__ probs, int32_t* __restrict__ n_tokens,
                                                           float* __restrict__ loss) {
  constexpr int kRows = 64 / LPR;           // rows a wavefront holds
  constexpr int kAhead = ahead_of<LPR>;     // ... and sets of them in flight
  static_assert(kHeldRows % kAhead == 0, "whole sets");
  constexpr int kWaves = kThreads / 64;
  __shared__ int s_counts[kMaxE], s_n;
  __shared__ f32x4 s_sum[kWaves][LPR];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const Rows r = rows_of(a);
  if (tid < kMaxE) s_counts[tid] = 0;
  if (tid == 0) s_n = 0;
  __syncthreads();
  int live_rows = 0;
  for (int row = r.first + tid; row < r.end; row += kThreads) {
    if (a.mask != nullptr && a.mask[row] == 0) continue;
    ++live_rows;
    int e[PRISM_MAX_TOPK];
#pragma unroll
    for (int j = 0; j < PRISM_MAX_TOPK; ++j) e[j] = j < a.k ? a.topk_idx[(size_t)row * a.k + j] : -1;
#pragma unroll
    for (int j = 0; j < PRISM_MAX_TOPK; ++j)
      if ((unsigned)e[j] < (unsigned)a.E) atomicAdd(&s_counts[e[j]], 1);
  }
  if (live_rows > 0) atomicAdd(&s_n, live_rows);
  const int e0 = (lane % LPR) * 4;
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  double earlier[4] = {0., 0., 0., 0.};
  int held = 0;                             // rows in sum
  for (int row0 = r.first + wave * kRows * kAhead; row0 < r.end; row0 += kWaves * kRows * kAhead) {
    f32x4 v[kAhead];
    bool live[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int row = row0 + u * kRows + lane / LPR;
      live[u] = row < r.end && (a.mask == nullptr || a.mask[row] != 0);
      v[u] = load_row(a, min(row, r.end - 1), e0);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      softmax_row<LPR>(v[u]);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += live[u] ? v[u][i] : 0.f;
    }
    held += kAhead;
    if (held == kHeldRows) {
#pragma unroll
      for (int i = 0; i < 4; ++i) earlier[i] += (double)sum[i];
      sum = f32x4{0.f, 0.f, 0.f, 0.f};
      held = 0;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = (float)(earlier[i] + (double)sum[i]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {             // the rows of the wavefront
    if constexpr (LPR <= 1) sum[i] += row_xor<1>(sum[i]);
    if constexpr (LPR <= 2) sum[i] += row_xor<2>(sum[i]);
    if constexpr (LPR <= 4) sum[i] += row_xor<4>(sum[i]);
    if constexpr (LPR <= 8) sum[i] += row_xor<8>(sum[i]);
    if constexpr (LPR <= 16) sum[i] += __shfl_xor(sum[i], 16);
    if constexpr (LPR <= 32) sum[i] += __shfl_xor(sum[i], 32);
  }
  if (lane < LPR) s_sum[wave][lane] = sum;
  __syncthreads();
  float total = 0.f;
  if (tid < a.E)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += s_sum[w][tid / 4][tid % 4];
  if (a.parts == 1) {
    finish_group(r.group, a.E, a.k, s_n, tid < kMaxE ? s_counts[tid] : 0, total, counts, probs, n_tokens, loss);
    return;
  }
  if (tid == 0) {
    partial.n[blockIdx.x] = s_n;
    if (r.part == 0) partial.done[r.group] = 0;
  }
  if (tid < partial.E4) {                   // (past E: zeros)
    partial.counts[(size_t)blockIdx.x * partial.E4 + tid] = s_counts[tid];
    partial.probs[(size_t)blockIdx.x * partial.E4 + tid] = total;
  }
}

// The parts of a group, added in 64 bits: thread (slice, 4 experts) the parts slice, slice + slices, ..., then the slices of a
// wavefront, then the wavefronts.  `pieces` workgroups of 4 * lanes experts each share a group (256 parts of 256 experts: 8 us by 8
// of them, 12 by one); the last of them to arrive adds their shares of the loss, in their order.
__global__ __launch_bounds__(kFinishThreads) void finish_kernel(const Partial partial, int E, int k, int parts, int lanes, int pieces,
                                                                int32_t* __restrict__ counts, float* __restrict__ probs,
                                                                int32_t* __restrict__ n_tokens, float* __restrict__ loss) {
  constexpr int kWaves = kFinishThreads / 64;
  __shared__ double s_sum[kWaves][kPieceLanes * 4];
  __shared__ int s_count[kWaves][kPieceLanes * 4], s_n[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = blockIdx.x / pieces, piece = blockIdx.x % pieces;
  const int first = piece * lanes * 4;
  const int slices = kFinishThreads / lanes, slice = tid / lanes, e0 = first + tid % lanes * 4;
  double sum[4] = {0., 0., 0., 0.};
  int count[4] = {0, 0, 0, 0}, n = 0;
#pragma unroll 8
  for (int p = slice; p < parts; p += slices) {
    const size_t at = (size_t)g * parts + p;
    n += partial.n[at];
    if (e0 < E) {
      const int4 c = *reinterpret_cast<const int4*>(partial.counts + at * partial.E4 + e0);
      const f32x4 v = *reinterpret_cast<const f32x4*>(partial.probs + at * partial.E4 + e0);
      count[0] += c.x; count[1] += c.y; count[2] += c.z; count[3] += c.w;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += (double)v[i];
    }
  }
  for (int off = lanes; off < 64; off <<= 1) {
    n += __shfl_xor(n, off);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[i] += __shfl_xor(sum[i], off);
      count[i] += __shfl_xor(count[i], off);
    }
  }
  if (lane < lanes)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s_sum[wave][lane * 4 + i] = sum[i];
      s_count[wave][lane * 4 + i] = count[i];
    }
  if (lane == 0) s_n[wave] = n;
  __syncthreads();
  if (wave != 0) return;
  static_assert(kPieceLanes * 4 <= 64, "a wavefront has a thread per expert of a piece");
  double total = 0.0;
  int c = 0;
  n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    n += s_n[w];
    if (tid < lanes * 4) {
      total += s_sum[w][tid];
      c += s_count[w][tid];
    }
  }
  const int e = first + tid;
  double term = 0.0;
  if (tid < lanes * 4 && e < E) {
    const double p = n > 0 ? total / n : 0.0;
    counts[(size_t)g * E + e] = c;
    probs[(size_t)g * E + e] = (float)p;
    term = (double)c * p;
  }
#pragma unroll
  for (int off = kPieceLanes * 2; off > 0; off >>= 1) term += __shfl_xor(term, off);
  if (tid != 0) return;
  if (pieces > 1) {
    double* const terms = partial.terms + (size_t)g * kMaxPieces;
    __hip_atomic_store(terms + piece, term, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__hip_atomic_fetch_add(partial.done + g, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) != (unsigned)pieces - 1) return;
    term = 0.0;
    for (int i = 0; i < pieces; ++i) term += __hip_atomic_load(terms + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  n_tokens[g] = n;
  loss[g] = n > 0 ? (float)(term * E / ((double)k * n)) : 0.f;
}

struct BackwardArgs {
  RowArgs r;
  const float* d_gate;        // [T, k] or NULL
  const int32_t* counts;      // [G, E], with n_tokens and d_loss; or all NULL
  const int32_t* n_tokens;
  const float* d_loss;
  float* d_logits;            // [T, E]
  int softmax_all;
};

// Slot j of a row's picks belongs to lane j % LPR of the row, register j / LPR; in rows of more than 16 lanes every 16 of them hold
// all slots.  What a pick adds to its expert reaches the lane that has the expert through LDS, where a wavefront has a float per
// expert of its rows (adding in the vector ALU, 8 slots to 4 experts per lane, took two fifths of the kernel's instructions).
template <int LPR> constexpr int slots_of = LPR >= PRISM_MAX_TOPK ? 1 : PRISM_MAX_TOPK / LPR;
template <int LPR> constexpr int slot_lanes_of = LPR > 16 ? 16 : LPR;

template <int LPR>
__global__ __launch_bounds__(kBackThreads) void route_backward_kernel(const BackwardArgs b) {
  constexpr int kRows = 64 / LPR, SL = slots_of<LPR>, kSlotLanes = slot_lanes_of<LPR>;
  constexpr int kAhead = back_ahead_of<LPR>, kWaves = kBackThreads / 64;
  const RowArgs& a = b.r;
  __shared__ __align__(16) float s_add[kWaves][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int in_row = lane % LPR, e0 = in_row * 4;
  const Rows r = rows_of(a);
  f32x4 u = {0.f, 0.f, 0.f, 0.f};           // d loss / d p of this lane's experts, up to a constant
  if (b.counts != nullptr) {
    const int n = b.n_tokens[r.group];
    int c[4] = {0, 0, 0, 0}, all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e0 + i < a.E) c[i] = b.counts[(size_t)r.group * a.E + e0 + i];
    all = c[0] + c[1] + c[2] + c[3];
#pragma unroll
    for (int off = 1; off < LPR; off <<= 1) all += __shfl_xor(all, off);
    const double f = n > 0 ? (double)b.d_loss[r.group] / ((double)a.k * n * n) : 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = (float)(f * (double)((long long)a.E * c[i] - all));
  }
  for (int row0 = r.first + wave * kRows * kAhead; row0 < r.end; row0 += kWaves * kRows * kAhead) {
    f32x4 v[kAhead];
    int idx[kAhead][SL];
    float dg[kAhead][SL], l[kAhead][SL];
    bool live[kAhead];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int row = min(row0 + s * kRows + lane / LPR, r.end - 1);
      live[s] = a.mask == nullptr || a.mask[row] != 0;
      v[s] = load_row(a, row, e0);
#pragma unroll
      for (int q = 0; q < SL; ++q) {
        const int j = in_row % kSlotLanes + q * LPR;
        idx[s][q] = -1;
        dg[s][q] = 0.f;
        if (b.d_gate != nullptr && j < a.k) {
          idx[s][q] = a.topk_idx[(size_t)row * a.k + j];
          if ((unsigned)idx[s][q] >= (unsigned)a.E) idx[s][q] = -1;
          else dg[s][q] = b.d_gate[(size_t)row * a.k + j];
        }
        l[s][q] = idx[s][q] >= 0 && !b.softmax_all ? a.logits[(size_t)row * a.E + idx[s][q]] : -INFINITY;
      }
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      softmax_row<LPR>(v[s]);
      // what the gates give: to u at a pick (softmax over all experts), or to the logit of a pick (over the picks)
      float t[SL];
      if (b.d_gate != nullptr && !b.softmax_all) {
        float m = -INFINITY;
#pragma unroll
        for (int q = 0; q < SL; ++q) m = fmaxf(m, l[s][q]);
        m = over_row<kSlotLanes>(m, [](float x, float y) { return fmaxf(x, y); });
        if (m == -INFINITY) m = 0.f;
        float sum = 0.f, dot = 0.f;
#pragma unroll
        for (int q = 0; q < SL; ++q) {
          t[q] = exp_neg(l[s][q] - m);
          sum += t[q];
          dot += t[q] * dg[s][q];
        }
        sum = over_row<kSlotLanes>(sum, add);
        dot = over_row<kSlotLanes>(dot, add);
        const float inv = sum > 0.f ? 1.0f / sum : sum;
#pragma unroll
        for (int q = 0; q < SL; ++q) t[q] = t[q] * inv * (dg[s][q] - dot * inv);
      } else {
#pragma unroll
        for (int q = 0; q < SL; ++q) t[q] = dg[s][q];
      }
      f32x4 g = {0.f, 0.f, 0.f, 0.f};       // of this lane's experts
      if (b.d_gate != nullptr) {
        float* const add_to = s_add[wave];
        *reinterpret_cast<f32x4*>(add_to + lane * 4) = f32x4{0.f, 0.f, 0.f, 0.f};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        // (one wavefront's additions, of one instruction or one after the other: an expert picked twice gets its sum in the same
        // order every time)
#pragma unroll
        for (int q = 0; q < SL; ++q)
          if (in_row < kSlotLanes && idx[s][q] >= 0)
            __hip_atomic_fetch_add(add_to + (lane - in_row) * 4 + idx[s][q], t[q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        g = *reinterpret_cast<const f32x4*>(add_to + lane * 4);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      f32x4 w = u;
      if (b.softmax_all) w += g;
      const float mean = over_row<LPR>((w[0] * v[s][0] + w[1] * v[s][1]) + (w[2] * v[s][2] + w[3] * v[s][3]), add);
      f32x4 d;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        d[i] = v[s][i] * (w[i] - mean);
        if (!b.softmax_all) d[i] += g[i];
        if (!live[s]) d[i] = 0.f;           // whatever the row holds
      }
      const int row = row0 + s * kRows + lane / LPR;
      if (row < r.end) {
        float* out = b.d_logits + (size_t)row * a.E + e0;
        if (e0 + 4 <= a.E) {
          reinterpret_cast<Unaligned<f32x4, 4>*>(out)->v = d;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (e0 + i < a.E) out[i] = d[i];
        }
      }
    }
  }
}

// Calls fn with the number of lanes a row takes (a power of two, 4 experts on each).
template <typename Fn> void with_lanes(int E, Fn&& fn) {
  if (E <= 4) fn(std::integral_constant<int, 1>{});
  else if (E <= 8) fn(std::integral_constant<int, 2>{});
  else if (E <= 16) fn(std::integral_constant<int, 4>{});
  else if (E <= 32) fn(std::integral_constant<int, 8>{});
  else if (E <= 64) fn(std::integral_constant<int, 16>{});
  else if (E <= 128) fn(std::integral_constant<int, 32>{});
  else fn(std::integral_constant<int, 64>{});
}

constexpr int kBackParts = 2048;  // of route_backward_kernel, about: it leaves no sums to be added
constexpr int kMaxGroups = PRISM_MAX_BALANCE_GROUPS;
constexpr int kMaxGrid = 1 << 21; // workgroups of a launch of balance_kernel: a grid has fewer than 2^32 threads
static_assert((long long)kMaxGrid * kThreads < 1LL << 32 && (long long)kMaxGroups * kBackThreads < 1LL << 32, "threads of a grid");

// The groups of a batch, and how many workgroups share one: at least one pass of rows each, and one workgroup for up to
// `few` passes (another pass takes less than the launch that adds the parts).
int split_groups(RowArgs* a, int group_tokens, int T, int most, int rows_per_pass, int few) {
  a->group = group_tokens > 0 ? group_tokens : std::max(T, 1);
  const int G = group_tokens > 0 ? (int)(((long long)T + group_tokens - 1) / group_tokens) : 1;
  const int rows = std::min(a->group, std::max(T, 1));
  const int wanted = std::max(1, most / std::max(G, 1));
  a->part_rows = std::max(ceil_div(rows, wanted), rows_per_pass);
  if (rows <= few * rows_per_pass) a->part_rows = rows;
  a->parts = ceil_div(rows, a->part_rows);
  return G;
}

}  // namespace

size_t balance_workspace_bytes(int E) { return align_up(partial_bytes(E), 256); }

prism_status launch_balance(const prism_layer_desc& d, const float* logits, const int32_t* topk_idx, const uint8_t* mask,
                            int group_tokens, int T, float* loss, int32_t* counts, float* probs, int32_t* n_tokens,
                            void* workspace, hipStream_t st) {
  if (T == 0 && group_tokens > 0) return PRISM_OK;    // no groups
  RowArgs a{logits, topk_idx, mask, T, d.n_experts, d.top_k, 0, 1, 0, 0};
  prism_status status = PRISM_OK;
  with_lanes(a.E, [&](auto lanes) {
    constexpr int LPR = decltype(lanes)::value;
    const int G = split_groups(&a, group_tokens, T, kParts, kThreads / LPR * ahead_of<LPR>, 4);
    if (G > kMaxGroups) {
      status = PRISM_ERR_UNSUPPORTED;
      return;
    }
    const Partial partial = partial_of(workspace, a.E);
    const int wgs = G * a.parts;            // (more than kParts of them: a group each)
    for (a.first_wg = 0; a.first_wg < wgs; a.first_wg += kMaxGrid)
      hipLaunchKernelGGL((balance_kernel<LPR>), dim3((unsigned)std::min(wgs - a.first_wg, kMaxGrid)), dim3(kThreads), 0, st, a, partial,
                         counts, probs, n_tokens, loss);
    if (a.parts > 1) {
      constexpr int kLanes = std::min(LPR, kPieceLanes);
      const int pieces = ceil_div(a.E, 4 * kLanes);
      hipLaunchKernelGGL(finish_kernel, dim3((unsigned)(G * pieces)), dim3(kFinishThreads), 0, st, partial, a.E, a.k, a.parts, kLanes,
                         pieces, counts, probs, n_tokens, loss);
    }
  });
  PRISM_TRY(status);
  PRISM_CHECK_LAUNCH();
  return PRISM_OK;
}

prism_status launch_route_backward(const prism_layer_desc& d, const float* logits, const int32_t* topk_idx, const uint8_t* mask,
                                   int group_tokens, int T, const int32_t* counts, const int32_t* n_tokens, const float* d_loss,
                                   const float* d_gate, float* d_logits, hipStream_t st) {
  if (T == 0) return PRISM_OK;
  BackwardArgs b{{logits, topk_idx, mask, T, d.n_experts, d.top_k, 0, 1, 0, 0}, d_gate, counts, n_tokens, d_loss, d_logits, d.gate_mode == PRISM_GATES_SOFTMAX_ALL};
  prism_status status = PRISM_OK;
  with_lanes(b.r.E, [&](auto lanes) {
    constexpr int LPR = decltype(lanes)::value;
    const int G = split_groups(&b.r, counts != nullptr ? group_tokens : 0, T, kBackParts, kBackThreads / LPR * back_ahead_of<LPR>, 1);
    if (G > kMaxGroups) {
      status = PRISM_ERR_UNSUPPORTED;
      return;
    }
    hipLaunchKernelGGL((route_backward_kernel<LPR>), dim3((unsigned)G * b.r.parts), dim3(kBackThreads), 0, st, b);
  });
  PRISM_TRY(status);
  PRISM_CHECK_LAUNCH();
  return PRISM_OK;
}

}  // namespace prism
