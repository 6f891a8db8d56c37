// Rows in 8 bits with a scale each (prism.h, "8-bit matrices"): activations of a product, weights as they are loaded, and
// the intermediate h of 8-bit experts.
//
//   scale = max |v| * (1 / 127), in fp32     q = the integer nearest to v / scale, ties to even, |q| <= 127
//
// q is that integer exactly: v / scale in fp32 is within one of it, and the remainder v - q scale, which fp32 holds
// without rounding (both are multiples of the smaller one's last place, and it is at most scale in magnitude), says which way.
// A value halfway between two integers is common, not rare: bf16 rows whose largest value has twice some element's
// digits put that element at 63.5.
//
// Bound by memory: a wavefront or a workgroup takes a row and holds it in registers between the maximum and the quotients
// (rows of more than 16384 elements are read again from there on).
#include <type_traits>

#include "grouped_gemm.h"

namespace prism {
namespace {

constexpr int kThreads = 256;                 // of pack_i8_kernel
constexpr int kElems = 8;                     // of a lane per pass
constexpr int kMaxGrid = 1 << 20;             // workgroups (a grid has fewer than 2^32 threads)

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// 8 elements of a row.  grow(m): m joined with the largest |v|; bits_of(m): that as the bits of a float, in which a NaN
// is larger than all numbers.
template <typename S> struct Chunk;
template <> struct Chunk<float> {
  typedef uint32_t Max;
  f32x4 a, b;
  __device__ void load(const float* p) {
    a = reinterpret_cast<const Unaligned<f32x4, 4>*>(p)[0].v;
    b = reinterpret_cast<const Unaligned<f32x4, 4>*>(p)[1].v;
  }
  __device__ void set(int i, float v) { (i < 4 ? a : b)[i & 3] = v; }
  __device__ __forceinline__ float get(int i) const { return (i < 4 ? a : b)[i & 3]; }
  __device__ __forceinline__ void grow(Max& m) const {
#pragma unroll
    for (int i = 0; i < kElems; ++i) m = max(m, __float_as_uint(get(i)) & 0x7fffffffu);
  }
  static __device__ __forceinline__ uint32_t bits_of(Max m) { return m; }
};
template <> struct Chunk<bf16_t> {
  typedef u16x2 Max;
  u32x4 a;
  __device__ void load(const bf16_t* p) { a = reinterpret_cast<const Unaligned<u32x4, 2>*>(p)->v; }
  __device__ void set(int i, bf16_t v) {
    const uint32_t w = a[i / 2], b = __builtin_bit_cast(uint16_t, v);
    a[i / 2] = i & 1 ? (w & 0xffffu) | b << 16 : (w & 0xffff0000u) | b;
  }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = a[i / 2];
    return i & 1 ? bf16_hi(w) : bf16_lo(w);
  }
  __device__ __forceinline__ void grow(Max& m) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, a[i] & 0x7fff7fffu));
  }
  static __device__ __forceinline__ uint32_t bits_of(Max m) { return (uint32_t)max(m.x, m.y) << 16; }
};

// Elements c .. c + 7 of a row of n, zeros past its end.
template <typename S> __device__ __forceinline__ Chunk<S> load_chunk(const S* row, int c, int n) {
  Chunk<S> v{};
  if (c + kElems <= n) {
    v.load(row + c);
  } else {
#pragma unroll
    for (int i = 0; i < kElems; ++i) v.set(i, c + i < n ? row[c + i] : (S)0.f);
  }
  return v;
}

// v / scale to the nearest integer, exactly.  scale and values are lifted where the reciprocal would not be finite.
struct Quotient {
  float scale, inverse, lift;
  __device__ explicit Quotient(float s) {
    lift = s < 0x1p-64f ? 0x1p64f : 1.f;
    scale = s * lift;
    inverse = 1.0f / scale;
  }
  __device__ __forceinline__ int exact(float v) const {
    v *= lift;
    float q = rintf(v * inverse);
    const float r2 = 2.f * fmaf(-q, scale, v);
    const bool odd = ((int)q & 1) != 0;
    if (r2 > scale || (r2 == scale && odd)) q += 1.f;
    else if (r2 < -scale || (r2 == -scale && odd)) q -= 1.f;
    return (int)fminf(fmaxf(q, -127.f), 127.f);
  }
};
// The 8 bytes of a chunk.  v * inverse is off by at most 127.5 * 2^-24 from the quotient (its factor's rounding; the product is
// not rounded before 1.5 * 2^23 is added, which leaves the integer in the low bits), so that only a chunk with a
// product within 10^-4 of a half needs the exact look: one in a hundred of random values.
constexpr float kRound = 12582912.f;
template <typename S> __device__ __forceinline__ uint2 quotients(const Chunk<S>& v, const Quotient& q) {
  uint32_t b[kElems];
  float far = 0.f;
#pragma unroll
  for (int i = 0; i < kElems; ++i) {
    const float x = v.get(i), t = fmaf(x, q.inverse, kRound);
    b[i] = __float_as_uint(t);
    far = fmaxf(far, fabsf(fmaf(x, q.inverse, kRound - t)));
  }
  if (far > 0.4999f || q.lift != 1.f) {
#pragma unroll
    for (int i = 0; i < kElems; ++i) b[i] = (uint32_t)q.exact(v.get(i));
  }
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    w[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x0c0c0400u), 0x05040100u);
  return uint2{w[0], w[1]};
}

// Byte of element c (a multiple of 8) of row r.
__device__ __forceinline__ size_t byte_of(int r, int c, size_t row_bytes, bool tiled) {
  return tiled ? ((size_t)(r >> 4) * (row_bytes / 64) + (c >> 6)) * 1024 + (r & 15) * 64 + (c & 63) : (size_t)r * row_bytes + c;
}

// Row r on LANES lanes (a wavefront, or a workgroup), `lane` of them this one.
template <typename S, int LANES, int HELD>
__device__ __forceinline__ void quantize_row(const QuantizeArgs& a, int r, int lane) {
  int from = r;
  if (a.local_offsets != nullptr) {
    if (r < a.A && (r < a.local_offsets[0] || r >= a.local_offsets[a.E])) return;   // holds no assignment
    if (a.local_src != nullptr) from = r < a.A ? a.local_src[r] / a.top_k : (r - a.A) % a.T;
  }
  const S* row = (const S*)a.src + (size_t)from * a.ld;
  const int row_bytes = (a.cols + kI8RowAlign - 1) / kI8RowAlign * kI8RowAlign;
  const int c0 = lane * kElems;
  constexpr int kPass = LANES * kElems;
  Chunk<S> held[HELD];
  typename Chunk<S>::Max grown{};
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (c0 + i * kPass < a.cols) held[i] = load_chunk<S>(row, c0 + i * kPass, a.cols);
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (c0 + i * kPass < a.cols) held[i].grow(grown);
  for (int c = c0 + HELD * kPass; c < a.cols; c += kPass) load_chunk<S>(row, c, a.cols).grow(grown);
  uint32_t m = Chunk<S>::bits_of(grown);
  m = max(m, (uint32_t)row_xor<1>((int)m));
  m = max(m, (uint32_t)row_xor<2>((int)m));
  m = max(m, (uint32_t)row_xor<4>((int)m));
  m = max(m, (uint32_t)row_xor<8>((int)m));
  m = max(m, (uint32_t)__shfl_xor((int)m, 16));
  m = max(m, (uint32_t)__shfl_xor((int)m, 32));
  if constexpr (LANES > 64) {
    __shared__ uint32_t s_max[LANES / 64];
    lds_barrier();                            // (the row before has been read)
    if ((lane & 63) == 0) s_max[lane >> 6] = m;
    lds_barrier();
    m = s_max[0];
#pragma unroll
    for (int w = 1; w < LANES / 64; ++w) m = max(m, s_max[w]);
  }
  const float scale = __uint_as_float(m) * (1.f / 127.f);
  if (lane == 0) {
    a.scale[r] = scale;
    if (a.places != nullptr) a.places[r] = (r >> 4) * (row_bytes / 64) * 16 + (r & 15);
  }
  // a row of zeros; of one that is not finite only the scale says so
  const bool zeros = !(scale > 0.f && scale < INFINITY);
  const Quotient q(zeros ? 1.f : scale);
  auto store = [&](int c, const Chunk<S>& v) {
    *reinterpret_cast<uint2*>(a.dst + byte_of(r, c, row_bytes, a.tiled)) = zeros || c >= a.cols ? uint2{0u, 0u} : quotients(v, q);
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (c0 + i * kPass < row_bytes) store(c0 + i * kPass, held[i]);
  for (int c = c0 + HELD * kPass; c < row_bytes; c += kPass) store(c, load_chunk<S>(row, c, a.cols));
}

// The 16 rows of a tile belong to workgroups that the hardware deals to one XCD (workgroups 8 apart), whose L2 joins their 64-byte
// pieces to whole lines: `per` workgroups a tile, of `wgs` in all (the last ones, too few for 8 tiles, in order).
__device__ __forceinline__ int same_xcd(int wg, int per, int wgs) {
  const int first = wg / (8 * per) * (8 * per), i = wg - first;
  return first + 8 * per <= wgs ? first + i % 8 * per + i / 8 : wg;
}
template <typename S, int LANES, int HELD>
__device__ __forceinline__ void quantize_rows(const QuantizeArgs& a, int wg, int wgs) {
  if constexpr (LANES == 64) {
    const int all = (a.rows + 3) / 4;
    for (int w = wg; w < all; w += wgs) {
      const int r = same_xcd(w, 4, all) * 4 + (threadIdx.x >> 6);
      if (r < a.rows) quantize_row<S, 64, HELD>(a, r, threadIdx.x & 63);
    }
  } else {
    for (int w = wg; w < a.rows; w += wgs) quantize_row<S, LANES, HELD>(a, same_xcd(w, 16, a.rows), threadIdx.x);
  }
}

template <typename S, int LANES, int HELD>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void quantize_kernel(const QuantizeArgs a) {
  quantize_rows<S, LANES, HELD>(a, blockIdx.x, gridDim.x);
}

// The tokens of an expert FFN, and the schedules of its two products: some workgroups more, where a launch of their own took 4 to 10 us.
constexpr int kScheduleParts = 4;             // workgroups that share the items of one schedule
template <int LANES, int HELD, bool WIDTHS>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void quantize_and_schedule_kernel(
    const QuantizeArgs a, const int32_t* __restrict__ local_offsets, int E, int S, int T, int A_total,
    const gg::sched_params_t<WIDTHS> p0, const gg::sched_params_t<WIDTHS> p1) {
  if (blockIdx.x < 2 * kScheduleParts) {
    const gg::sched_params_t<WIDTHS> p[1] = {blockIdx.x < kScheduleParts ? p0 : p1};
    gg::build_schedules_block<1, WIDTHS>(local_offsets, E, S, T, A_total, p, blockIdx.x % kScheduleParts, kScheduleParts);
  } else {
    quantize_rows<bf16_t, LANES, HELD>(a, blockIdx.x - 2 * kScheduleParts, gridDim.x - 2 * kScheduleParts);
  }
}

// Rows of bytes that are quantised already, into tiles: a row per workgroup.
__global__ __launch_bounds__(kThreads) void pack_i8_kernel(const int8_t* __restrict__ src, long long ld, const float* __restrict__ scale,
                                                           int rows, int cols, uint8_t* __restrict__ dst,
                                                           float* __restrict__ dst_scale) {
  const int row_bytes = (cols + kI8RowAlign - 1) / kI8RowAlign * kI8RowAlign;
  for (int r = blockIdx.x; r < rows; r += gridDim.x) {
    const int8_t* row = src + (size_t)r * ld;
    for (int c = threadIdx.x * 16; c < row_bytes; c += kThreads * 16) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (c + 16 <= cols) {
        v = reinterpret_cast<const Unaligned<u32x4, 1>*>(row + c)->v;
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c + i < cols) v[i / 4] |= (uint32_t)(uint8_t)row[c + i] << (8 * (i % 4));
      }
      *reinterpret_cast<u32x4*>(dst + byte_of(r, c, row_bytes, true)) = v;
    }
    if (threadIdx.x == 0) dst_scale[r] = scale[r];
  }
}

}  // namespace

namespace {
// Calls launch(lanes, held) with the lanes of a row: a wavefront where rows are many and it holds them; else as many as make one or two
// passes of it, and of long rows half as many once there are more than CUs.  Rows from HBM (every launch another copy, 1.5 GB of
// them), bytes in and out in TB/s (a large copy reaches 4.8): 28000 x 1408 fp32 by 64 lanes 4.8, by 256 3.9; 5001 x 2048 bf16 2.2 by
// either; 7000 x 4096 fp32 by 256 lanes 4.9, by 512 4.3, by 64 3.6; 7200 x 4096 bf16 3.3, 2.4, 2.5; 7200 x 14336 fp32 by 512 lanes 5.25, by
// 1024 4.5, by 256 5.1; 4096 x 14336 bf16 3.6, 2.6, 2.95.  Few rows, us: 600 x 2048 bf16 by 256 lanes 4.6, by 64 6.9; 32 x 14336 bf16 by 1024
// lanes 5.8, by 512 7.0; 128 x 4160 4.4 against 5.3, 128 x 14336 6.1 / 7.2, but 300 x 4160 6.8 / 5.8, 300 x 14336 10.6 / 9.7, 512 x 8192 8.8 / 7.6
// (fp32 rows alike).
constexpr int kManyLongRows = 256;
template <typename Fn> void with_row_lanes(const QuantizeArgs& a, Fn&& launch) {
  using std::integral_constant;
  if (a.cols <= 2048 && a.rows > 4096) launch(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  else if (a.cols <= 2048) launch(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (a.cols <= 4096) launch(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (a.rows > kManyLongRows) launch(integral_constant<int, 512>{}, integral_constant<int, 4>{});
  else launch(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}
unsigned workgroups(const QuantizeArgs& a, int lanes) { return (unsigned)std::min(ceil_div(a.rows, lanes == 64 ? 4 : 1), kMaxGrid); }
}  // namespace

prism_status launch_quantize(const QuantizeArgs& a, int src_dtype, hipStream_t st) {
  if (a.rows == 0) return PRISM_OK;
  auto of_type = [&](auto elem) {
    using S = decltype(elem);
    with_row_lanes(a, [&](auto lanes, auto held) {
      constexpr int L = decltype(lanes)::value, N = decltype(held)::value;
      const dim3 grid(workgroups(a, L)), block(L < 256 ? 256 : L);
      hipLaunchKernelGGL((quantize_kernel<S, L, N>), grid, block, 0, st, a);
    });
  };
  if (src_dtype == PRISM_F32) of_type(float{});
  else of_type(bf16_t{});
  PRISM_CHECK_LAUNCH();
  return PRISM_OK;
}

prism_status launch_quantize_tokens(const prism_layer_desc& d, const QuantizeArgs& a, const int32_t* local_offsets, int T,
                                    int32_t* tiles, hipStream_t st) {
  gg::WidthParams p0, p1;
  gg::ffn_sched_params(d, T, tiles, &p0, &p1);
  with_row_lanes(a, [&](auto lanes, auto held) {
    constexpr int L = decltype(lanes)::value, N = decltype(held)::value;
    const dim3 grid(workgroups(a, L) + 2 * kScheduleParts), block(L < 256 ? 256 : L);
    if (p0.wide_ntiles > 0)
      hipLaunchKernelGGL((quantize_and_schedule_kernel<L, N, true>), grid, block, 0, st, a, local_offsets, d.n_experts, d.n_shared, T,
                         T * d.top_k, p0, p1);
    else
      hipLaunchKernelGGL((quantize_and_schedule_kernel<L, N, false>), grid, block, 0, st, a, local_offsets, d.n_experts, d.n_shared, T,
                         T * d.top_k, p0, p1);
  });
  PRISM_CHECK_LAUNCH();
  return PRISM_OK;
}

prism_status launch_pack_i8(const int8_t* src, long long ld, const float* scale, int rows, int cols, void* dst, hipStream_t st) {
  hipLaunchKernelGGL(pack_i8_kernel, dim3((unsigned)std::min(rows, kMaxGrid)), dim3(kThreads), 0, st, src, ld, scale, rows, cols,
                     (uint8_t*)dst, (float*)((uint8_t*)dst + i8_elements(rows, cols)));
  PRISM_CHECK_LAUNCH();
  return PRISM_OK;
}

}  // namespace prism
