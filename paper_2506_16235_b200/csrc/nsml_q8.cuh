// The q8 format: int8 codes, a row per token or output channel, and one float32 scale per row, a power of two.
//   scale = 2^e, e the smallest integer with amax 2^-e <= 127, held between -126 and 121
//   code  = clamp(rint(v / scale), +-127), half to even
// A power of two costs up to one of the eight bits against amax / 127, and buys that everything behind it is exact: the
// quotient, the restored value (eight significant bits are a bfloat16), and a scale that moves from one operand of a
// product to the other (the gradients' products sum over the axis that the scales belong to).
#pragma once

#include <cuda_bf16.h>

#include "nsml_common.cuh"

namespace nsml {
namespace q8 {

constexpr int kMinExp = -126, kMaxExp = 121;  // 127 * 2^121 is finite; from 2^-126 on a restored value is a normal number

// Scale of a row from the bits of its largest magnitude (NaN's bits are above infinity's): 0 for 0, NaN for NaN or infinity.
// inv: its reciprocal, exact; 0 where codes are to be 0.
__device__ __forceinline__ float scale_of(uint32_t amax_bits, float* inv) {
  if (amax_bits == 0 || amax_bits >= kInfKey) {
    *inv = 0.0f;
    return amax_bits == 0 ? 0.0f : __uint_as_float(0x7FC00000u);
  }
  // amax = 1.f * 2^(E - 127); 127 = 1.984375 * 2^6
  int e = (int)(amax_bits >> 23) - 127 - 6 + ((amax_bits & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);
  e = min(max(e, kMinExp), kMaxExp);
  *inv = __uint_as_float((uint32_t)(127 - e) << 23);
  return __uint_as_float((uint32_t)(127 + e) << 23);
}

// v is finite, or inv is 0 (codes of a row with NaN or infinity are 0)
__device__ __forceinline__ int code_of(float v, float inv) {
  const int c = inv == 0.0f ? 0 : __float2int_rn(__fmul_rn(v, inv));
  return max(-127, min(127, c));
}

__device__ __forceinline__ float restore(int code, float scale) { return __fmul_rn((float)code, scale); }

// ---- eight consecutive elements ---------------------------------------------------------------------------------------
template <int DTYPE>
struct Elem { using type = float; };
template <>
struct Elem<NSML_BF16> { using type = __nv_bfloat16; };

__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// Elements c .. c+7 of a row of `cols`; those past the end are 0.  vec: the row starts on a 16-byte boundary.
template <int DTYPE>
__device__ __forceinline__ void load8(const typename Elem<DTYPE>::type* row, int64_t c, int64_t cols, bool vec, float (&v)[8]) {
  if (vec && c + 8 <= cols) {
    if constexpr (DTYPE == NSML_F32) {
      const float4 a = *reinterpret_cast<const float4*>(row + c), b = *reinterpret_cast<const float4*>(row + c + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
      const uint4 a = *reinterpret_cast<const uint4*>(row + c);
      unpack2(a.x, v[0], v[1]); unpack2(a.y, v[2], v[3]);
      unpack2(a.z, v[4], v[5]); unpack2(a.w, v[6], v[7]);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? (float)row[c + i] : 0.0f;
}

template <int DTYPE>
__device__ __forceinline__ void store8(typename Elem<DTYPE>::type* row, int64_t c, int64_t cols, bool vec, const float (&v)[8]) {
  if (vec && c + 8 <= cols) {
    if constexpr (DTYPE == NSML_F32) {
      *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      *reinterpret_cast<uint4*>(row + c) = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < cols) row[c + i] = (typename Elem<DTYPE>::type)v[i];
}

// Eight codes; rows of codes start on 16-byte boundaries.  Nothing past `cols` is written.
__device__ __forceinline__ void store8_codes(int8_t* row, int64_t c, int64_t cols, const int (&q)[8]) {
  if (c + 8 <= cols) {
    uint2 w;
    w.x = (q[0] & 255) | (q[1] & 255) << 8 | (q[2] & 255) << 16 | q[3] << 24;
    w.y = (q[4] & 255) | (q[5] & 255) << 8 | (q[6] & 255) << 16 | q[7] << 24;
    *reinterpret_cast<uint2*>(row + c) = w;
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < cols) row[c + i] = (int8_t)q[i];
}

// Restored values of eight codes; those past the end are 0 (whatever the bytes behind the row hold).
__device__ __forceinline__ void load8_codes(const int8_t* row, int64_t c, int64_t cols, float scale, float (&v)[8]) {
  if (c >= cols) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    return;
  }
  // (c is a multiple of 8 and rows are a multiple of 16 bytes apart: the eight bytes are inside the row's own)
  const uint2 w = *reinterpret_cast<const uint2*>(row + c);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int code = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    v[i] = c + i < cols ? restore(code, scale) : 0.0f;
  }
}

// ---- sums over the THREADS threads that share a row (a warp, or the whole block) -----------------------------------------
template <int THREADS>
__device__ __forceinline__ double row_sum(double v, double* shared) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if constexpr (THREADS > 32) {
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) v += shared[w];
  }
  return v;
}

template <int THREADS>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* shared) {
  v = __reduce_max_sync(0xFFFFFFFFu, v);
  if constexpr (THREADS > 32) {
    __syncthreads();
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) v = max(v, shared[w]);
  }
  return v;
}

}  // namespace q8
}  // namespace nsml
