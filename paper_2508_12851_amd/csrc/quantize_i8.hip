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
// Bound by memory: a workgroup takes a row, holds up to 16384 elements in registers between the maximum and the quotients, and reads
// longer rows again.
#include <type_traits>

#include "prism_internal.h"

namespace prism {
namespace {

constexpr int kThreads = 256;
constexpr int kElems = 8;                     // of a thread per pass
constexpr int kHeld = 8;                      // passes whose elements stay in registers
constexpr int kMaxGrid = 1 << 20;             // workgroups (a grid has fewer than 2^32 threads)

template <typename S> struct Chunk;
template <> struct Chunk<float> {
  f32x4 a, b;
  __device__ void load(const float* p) {
    a = reinterpret_cast<const f32x4*>(p)[0];
    b = reinterpret_cast<const f32x4*>(p)[1];
  }
  __device__ void set(int i, float v) { (i < 4 ? a : b)[i & 3] = v; }
  __device__ float get(int i) const { return (i < 4 ? a : b)[i & 3]; }
};
template <> struct Chunk<bf16_t> {
  bf16x8 a;
  __device__ void load(const bf16_t* p) { a = *reinterpret_cast<const bf16x8*>(p); }
  __device__ void set(int i, bf16_t v) { a[i] = v; }
  __device__ float get(int i) const { return (float)a[i]; }
};

// Elements c .. c + 7 of a row of n, zeros past its end.
template <typename S, bool VEC> __device__ __forceinline__ Chunk<S> load_chunk(const S* row, int c, int n) {
  Chunk<S> v;
  if (VEC && c + kElems <= n) {
    v.load(row + c);
  } else {
#pragma unroll
    for (int i = 0; i < kElems; ++i) v.set(i, c + i < n ? row[c + i] : (S)0.f);
  }
  return v;
}

// |v| of the largest as its bits, in which a NaN is larger than all numbers.
template <typename S> __device__ __forceinline__ uint32_t grow(uint32_t m, const Chunk<S>& v) {
#pragma unroll
  for (int i = 0; i < kElems; ++i) m = max(m, __float_as_uint(v.get(i)) & 0x7fffffffu);
  return m;
}

struct Quotient {
  float scale, inverse, lift;     // scale and values are lifted where the reciprocal would not be finite
  __device__ explicit Quotient(float s) {
    lift = s < 0x1p-64f ? 0x1p64f : 1.f;
    scale = s * lift;
    inverse = 1.0f / scale;
  }
  __device__ __forceinline__ int operator()(float v) const {
    v *= lift;
    float q = rintf(v * inverse);
    const float r2 = 2.f * fmaf(-q, scale, v);
    const bool odd = ((int)q & 1) != 0;
    if (r2 > scale || (r2 == scale && odd)) q += 1.f;
    else if (r2 < -scale || (r2 == -scale && odd)) q -= 1.f;
    return (int)fminf(fmaxf(q, -127.f), 127.f);
  }
};
template <typename S> __device__ __forceinline__ uint2 quotients(const Chunk<S>& v, const Quotient& q) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    w[h] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[h] |= (uint32_t)(q(v.get(4 * h + i)) & 0xff) << (8 * i);
  }
  return uint2{w[0], w[1]};
}

// Byte of element c (a multiple of 8) of row r.
__device__ __forceinline__ size_t byte_of(int r, int c, size_t row_bytes, bool tiled) {
  return tiled ? ((size_t)(r >> 4) * (row_bytes / 64) + (c >> 6)) * 1024 + (r & 15) * 64 + (c & 63) : (size_t)r * row_bytes + c;
}

template <typename S, bool VEC> __device__ __forceinline__ void quantize_row(const QuantizeArgs& a, int r) {
  __shared__ uint32_t s_max[kThreads / 64];
  int from = r;
  if (a.local_offsets != nullptr) {
    if (r < a.A && (r < a.local_offsets[0] || r >= a.local_offsets[a.E])) return;   // holds no assignment
    if (a.local_src != nullptr) from = r < a.A ? a.local_src[r] / a.top_k : (r - a.A) % a.T;
  }
  const S* row = (const S*)a.src + (size_t)from * a.ld;
  const int row_bytes = (a.cols + kI8RowAlign - 1) / kI8RowAlign * kI8RowAlign;
  const int c0 = threadIdx.x * kElems;
  constexpr int kPass = kThreads * kElems;
  Chunk<S> held[kHeld];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (c0 + i * kPass < a.cols) held[i] = load_chunk<S, VEC>(row, c0 + i * kPass, a.cols);
#pragma unroll
  for (int i = 0; i < kHeld; ++i)
    if (c0 + i * kPass < a.cols) m = grow(m, held[i]);
  for (int c = c0 + kHeld * kPass; c < a.cols; c += kPass) m = grow(m, load_chunk<S, VEC>(row, c, a.cols));
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off));
  if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = m;
  __syncthreads();
  m = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
  const float scale = __uint_as_float(m) * (1.f / 127.f);
  if (threadIdx.x == 0) {
    a.scale[r] = scale;
    if (a.places != nullptr) a.places[r] = (r >> 4) * (row_bytes / 64) * 16 + (r & 15);
  }
  const Quotient q(scale > 0.f ? scale : 1.f);     // (a row of zeros; of one that is not finite only the scale says so)
  uint8_t* const dst = a.dst;
  auto store = [&](int c, const Chunk<S>& v) {
    *reinterpret_cast<uint2*>(dst + byte_of(r, c, row_bytes, a.tiled)) = scale > 0.f ? quotients(v, q) : uint2{0u, 0u};
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int c = c0 + i * kPass;
    if (c < a.cols) store(c, held[i]);
    else if (c < row_bytes) *reinterpret_cast<uint2*>(dst + byte_of(r, c, row_bytes, a.tiled)) = uint2{0u, 0u};
  }
  for (int c = c0 + kHeld * kPass; c < row_bytes; c += kPass) {
    if (c < a.cols) store(c, load_chunk<S, VEC>(row, c, a.cols));
    else *reinterpret_cast<uint2*>(dst + byte_of(r, c, row_bytes, a.tiled)) = uint2{0u, 0u};
  }
}

template <typename S, bool VEC> __global__ __launch_bounds__(kThreads) void quantize_kernel(const QuantizeArgs a) {
  for (int r = blockIdx.x; r < a.rows; r += gridDim.x) {
    quantize_row<S, VEC>(a, r);
    __syncthreads();                            // (the maxima are read)
  }
}

// Rows of bytes that are quantised already, into tiles: a row per workgroup.
__global__ __launch_bounds__(kThreads) void pack_i8_kernel(const int8_t* __restrict__ src, long long ld, const float* __restrict__ scale,
                                                           int rows, int cols, int vec, uint8_t* __restrict__ dst,
                                                           float* __restrict__ dst_scale) {
  const int row_bytes = (cols + kI8RowAlign - 1) / kI8RowAlign * kI8RowAlign;
  for (int r = blockIdx.x; r < rows; r += gridDim.x) {
    const int8_t* row = src + (size_t)r * ld;
    for (int c = threadIdx.x * 16; c < row_bytes; c += kThreads * 16) {
      uint4 v{0u, 0u, 0u, 0u};
      if (vec && c + 16 <= cols) {
        v = *reinterpret_cast<const uint4*>(row + c);
      } else {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
  #pragma unroll
        for (int i = 0; i < 16; ++i)
          if (c + i < cols) w[i / 4] |= (uint32_t)(uint8_t)row[c + i] << (8 * (i % 4));
        v = uint4{w[0], w[1], w[2], w[3]};
      }
      *reinterpret_cast<uint4*>(dst + byte_of(r, c, row_bytes, true)) = v;
    }
    if (threadIdx.x == 0) dst_scale[r] = scale[r];
  }
}

}  // namespace

prism_status launch_quantize(const QuantizeArgs& a, int src_dtype, hipStream_t st) {
  if (a.rows == 0) return PRISM_OK;
  auto launch = [&](auto elem) {
    using S = decltype(elem);
    const bool vec = ((uintptr_t)a.src & 15u) == 0 && a.ld * (long long)sizeof(S) % 16 == 0;
    if (vec) hipLaunchKernelGGL((quantize_kernel<S, true>), dim3((unsigned)std::min(a.rows, kMaxGrid)), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((quantize_kernel<S, false>), dim3((unsigned)std::min(a.rows, kMaxGrid)), dim3(kThreads), 0, st, a);
  };
  if (src_dtype == PRISM_F32) launch(float{});
  else launch(bf16_t{});
  PRISM_CHECK_LAUNCH();
  return PRISM_OK;
}

prism_status launch_pack_i8(const int8_t* src, long long ld, const float* scale, int rows, int cols, void* dst, hipStream_t st) {
  const int vec = ((uintptr_t)src & 15u) == 0 && ld % 16 == 0;
  hipLaunchKernelGGL(pack_i8_kernel, dim3((unsigned)std::min(rows, kMaxGrid)), dim3(kThreads), 0, st, src, ld, scale, rows, cols, vec, (uint8_t*)dst,
                     (float*)((uint8_t*)dst + i8_elements(rows, cols)));
  PRISM_CHECK_LAUNCH();
  return PRISM_OK;
}

}  // namespace prism
