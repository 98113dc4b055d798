// The q8 format: int8 codes, a row per token or output channel, and one float32 scale per row, a power of two.
//   scale = 2^e, e the smallest integer with amax 2^-e <= 127, held between -126 and 121
//   code  = clamp(rint(v / scale), +-127), half to even
// A power of two costs up to one of the eight bits against amax / 127, and buys that everything behind it is exact: the
// quotient, the restored value (eight significant bits are a bfloat16), and a scale that moves from one operand of a
// product to the other (the gradients' products sum over the axis that the scales belong to).
#pragma once

#include <cuda_bf16.h>

#include "nsml_common.cuh"
#include "nsml_launch.h"

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

// Four codes of values times inv (exact: a power of two).  Adding 1.5 * 2^23 rounds to an integer, half to even, whose low
// byte is the code.  clamp: products may round to 128 (a scale held at 2^121), or the row is not finite (inv is 0: codes 0).
__device__ __forceinline__ bool needs_clamp(uint32_t amax_bits) { return amax_bits >= 0x7F7F0000u; }  // 127.5 * 2^121
template <bool CLAMP>
__device__ __forceinline__ uint32_t code_bits(float v, float inv) {
  if constexpr (CLAMP) {
    const int c = inv == 0.0f ? 0 : __float2int_rn(__fmul_rn(v, inv));
    return (uint32_t)max(-127, min(127, c));
  }
  return __float_as_uint(__fmaf_rn(v, inv, 12582912.0f));
}
template <bool CLAMP>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv) {
  return __byte_perm(__byte_perm(code_bits<CLAMP>(a, inv), code_bits<CLAMP>(b, inv), 0x0040),
                     __byte_perm(code_bits<CLAMP>(c, inv), code_bits<CLAMP>(d, inv), 0x0040), 0x5410);
}
template <bool CLAMP>
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float inv) {
  return make_uint2(codes4<CLAMP>(v[0], v[1], v[2], v[3], inv), codes4<CLAMP>(v[4], v[5], v[6], v[7], inv));
}
// largest magnitude so far; a NaN stays
__device__ __forceinline__ float top3(float top, float a, float b) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(top), "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float top8(float top, const float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; j += 2) top = top3(top, v[j], v[j + 1]);
  return top;
}

__device__ __forceinline__ float restore(int code, float scale) { return __fmul_rn((float)code, scale); }

// ---- eight consecutive elements ---------------------------------------------------------------------------------------
template <int DTYPE>
struct Elem { using type = float; using bits = uint32_t; };
template <>
struct Elem<NSML_BF16> { using type = __nv_bfloat16; using bits = uint16_t; };

__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// Eight elements of a row as they are in memory: chunk `i` of the thread that is number `lane` of a row's THREADS.
//   VEC      rows (and the width: a multiple of eight) are on 16-byte boundaries: eight consecutive elements, four registers
//            of bfloat16 or eight of float32
//   else     every THREADS-th element, so that a warp's loads of one element each are next to each other
//   APART    of those: a register each, so that they are waited for where they are used (putting two together waits where they
//            are loaded, but takes half the registers)
// Elements past the end are 0, and are not written.
template <bool VEC, int THREADS>
__device__ __forceinline__ unsigned int column(int lane, int i, int j) {  // (past the end of the widest row it passes 2^31)
  return VEC ? 8u * (lane + i * THREADS) + j : (8u * i + j) * THREADS + lane;
}
// whether chunk i of every thread lies past the end, or inside
template <int THREADS>
__device__ __forceinline__ bool outside(int i, int cols) { return 8u * i * THREADS >= (unsigned int)cols; }
template <int THREADS>
__device__ __forceinline__ bool inside(int i, int cols) { return 8u * i * THREADS + 8 * THREADS <= (unsigned int)cols; }

template <int DTYPE, bool VEC, bool APART = false>
struct Raw8 {
  static constexpr bool kPairs = (VEC || !APART) && DTYPE == NSML_BF16;
  uint32_t w[kPairs ? 4 : 8];
  __device__ __forceinline__ void widen(float (&v)[8]) const {
    if constexpr (kPairs) {
#pragma unroll
      for (int j = 0; j < 4; ++j) unpack2(w[j], v[2 * j], v[2 * j + 1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(DTYPE == NSML_F32 ? w[j] : w[j] << 16);
    }
  }
  __device__ __forceinline__ void round(const float (&v)[8]) {
    if constexpr (kPairs) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = pack2(v[2 * j], v[2 * j + 1]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = DTYPE == NSML_F32 ? __float_as_uint(v[j]) : (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v[j]));
    }
  }
  using Bits = typename Elem<DTYPE>::bits;
  template <int THREADS>
  __device__ __forceinline__ void load(const typename Elem<DTYPE>::type* row, int lane, int i, int cols) {
#pragma unroll
    for (uint32_t& x : w) x = 0;
    if constexpr (VEC) {
      if (column<VEC, THREADS>(lane, i, 0) >= (unsigned int)cols) return;
      const uint4* from = reinterpret_cast<const uint4*>(row + column<VEC, THREADS>(lane, i, 0));
      set(0, from[0]);
      if constexpr (!kPairs) set(4, from[1]);
    } else {
      const Bits* from = reinterpret_cast<const Bits*>(row) + lane;
      if (inside<THREADS>(i, cols)) {  // (the offsets are the instructions' own)
#pragma unroll
        for (int j = 0; j < 8; ++j) put(j, from[(8u * i + j) * THREADS]);
      } else if (!outside<THREADS>(i, cols)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) put(j, column<VEC, THREADS>(lane, i, j) < (unsigned int)cols ? (uint32_t)from[(8u * i + j) * THREADS] : 0u);
      }
    }
  }
  template <int THREADS>
  __device__ __forceinline__ void store(typename Elem<DTYPE>::type* row, int lane, int i, int cols) const {
    if constexpr (VEC) {
      if (column<VEC, THREADS>(lane, i, 0) >= (unsigned int)cols) return;
      uint4* to = reinterpret_cast<uint4*>(row + column<VEC, THREADS>(lane, i, 0));
      if constexpr (kPairs) {
        to[0] = make_uint4(w[0], w[1], w[2], w[3]);
      } else if (reinterpret_cast<uintptr_t>(to) % 32 == 0) {  // in one store: two of 16 bytes, 32 apart across the lanes, write half sectors
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
                     "r"(w[6]), "r"(w[7]) : "memory");
      } else {
        to[0] = make_uint4(w[0], w[1], w[2], w[3]);
        to[1] = make_uint4(w[4], w[5], w[6], w[7]);
      }
    } else {
      Bits* to = reinterpret_cast<Bits*>(row) + lane;
      if (inside<THREADS>(i, cols)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) to[(8u * i + j) * THREADS] = (Bits)bits(j);
      } else if (!outside<THREADS>(i, cols)) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (column<VEC, THREADS>(lane, i, j) < (unsigned int)cols) to[(8u * i + j) * THREADS] = (Bits)bits(j);
      }
    }
  }
  __device__ __forceinline__ void put(int j, uint32_t x) {
    if constexpr (kPairs) w[j / 2] = (j & 1) ? __byte_perm(w[j / 2], x, 0x5410) : x;
    else w[j] = x;
  }
  __device__ __forceinline__ uint32_t bits(int j) const {
    if constexpr (kPairs) return (j & 1) ? w[j / 2] >> 16 : w[j / 2];
    else return w[j];
  }
  __device__ __forceinline__ void set(int at, const uint4& x) {
    w[at] = x.x;
    w[at + 1] = x.y;
    w[at + 2] = x.z;
    w[at + 3] = x.w;
  }
};

template <int DTYPE, bool VEC, int THREADS>
__device__ __forceinline__ void load8(const typename Elem<DTYPE>::type* row, int lane, int i, int cols, float (&v)[8]) {
  Raw8<DTYPE, VEC> r;
  r.template load<THREADS>(row, lane, i, cols);
  r.widen(v);
}
template <int DTYPE, bool VEC, int THREADS>
__device__ __forceinline__ void store8(typename Elem<DTYPE>::type* row, int lane, int i, int cols, const float (&v)[8]) {
  Raw8<DTYPE, VEC> r;
  r.round(v);
  r.template store<THREADS>(row, lane, i, cols);
}

// The same for codes, whose rows are always on 16-byte boundaries.
template <bool VEC, int THREADS>
__device__ __forceinline__ void store8_codes(int8_t* row, int lane, int i, int cols, uint2 w) {
  if constexpr (VEC) {
    if (column<VEC, THREADS>(lane, i, 0) < (unsigned int)cols) *reinterpret_cast<uint2*>(row + column<VEC, THREADS>(lane, i, 0)) = w;
  } else {
    int8_t* to = row + lane;
    if (inside<THREADS>(i, cols)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) to[(8u * i + j) * THREADS] = (int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    } else if (!outside<THREADS>(i, cols)) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (column<VEC, THREADS>(lane, i, j) < (unsigned int)cols) to[(8u * i + j) * THREADS] = (int8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    }
  }
}
template <bool VEC, bool APART = false>
struct RawCodes8 {
  static constexpr bool kFours = VEC || !APART;
  uint32_t w[kFours ? 2 : 8];
  template <int THREADS>
  __device__ __forceinline__ void load(const int8_t* row, int lane, int i, int cols) {
#pragma unroll
    for (uint32_t& x : w) x = 0;
    if constexpr (VEC) {
      if (column<VEC, THREADS>(lane, i, 0) >= (unsigned int)cols) return;
      const uint2 x = *reinterpret_cast<const uint2*>(row + column<VEC, THREADS>(lane, i, 0));
      w[0] = x.x;
      w[1] = x.y;
    } else {
      const uint8_t* from = reinterpret_cast<const uint8_t*>(row) + lane;
      uint32_t b[8] = {};
      if (inside<THREADS>(i, cols)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = from[(8u * i + j) * THREADS];
      } else if (!outside<THREADS>(i, cols)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = column<VEC, THREADS>(lane, i, j) < (unsigned int)cols ? (uint32_t)from[(8u * i + j) * THREADS] : 0u;
      }
      if constexpr (kFours) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          w[j] = __byte_perm(__byte_perm(b[4 * j], b[4 * j + 1], 0x0040), __byte_perm(b[4 * j + 2], b[4 * j + 3], 0x0040), 0x5410);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = b[j];
      }
    }
  }
  // As numbers: the byte, moved up by 128, becomes the last one of 2^23 (whose unit is 1).
  __device__ __forceinline__ void numbers(float (&v)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t bits = kFours ? __byte_perm(w[kFours ? j / 4 : 0] ^ 0x80808080u, 0x4B000000u, 0x7540 | (j & 3)) : (w[kFours ? 0 : j] ^ 0x80u) | 0x4B000000u;
      v[j] = __fadd_rn(__uint_as_float(bits), -8388736.0f);
    }
  }
};

// whether a row's threads skip chunk i (VEC: empty ones are only skipped where they are loaded and stored)
template <bool VEC, int THREADS>
__device__ __forceinline__ bool empty(int i, int cols) { return !VEC && outside<THREADS>(i, cols); }

template <bool VEC, int THREADS>
__device__ __forceinline__ void load8_weight(const void* weight, bool bf16, int lane, int i, int cols, float (&w)[8]) {
  if (bf16) load8<NSML_BF16, VEC, THREADS>(static_cast<const __nv_bfloat16*>(weight), lane, i, cols, w);
  else load8<NSML_F32, VEC, THREADS>(static_cast<const float*>(weight), lane, i, cols, w);
}

template <int THREADS>
__device__ __forceinline__ int my_lane() { return threadIdx.x % THREADS; }

// ---- over the THREADS threads that share a row (part of a warp, a warp, or the whole block; then once per `shared`) --------
template <int THREADS>
__device__ __forceinline__ double row_sum(double v, double* shared) {
#pragma unroll
  for (int d = (THREADS < 32 ? THREADS : 32) / 2; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if constexpr (THREADS > 32) {
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) v += shared[w];
  }
  return v;
}

// bits of the largest magnitude (NaN's are above infinity's)
template <int THREADS>
__device__ __forceinline__ uint32_t row_top(float top, uint32_t* shared) {
  uint32_t v = __float_as_uint(top) & 0x7FFFFFFFu;
  if constexpr (THREADS < 32) {
#pragma unroll
    for (int d = THREADS / 2; d; d >>= 1) v = max(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
  } else {
    v = __reduce_max_sync(0xFFFFFFFFu, v);
  }
  if constexpr (THREADS > 32) {
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = shared[0];
#pragma unroll
    for (int w = 1; w < THREADS / 32; ++w) v = max(v, shared[w]);
  }
  return v;
}

// ---- arguments -----------------------------------------------------------------------------------------------------
inline bool rows16(const void* p, int64_t ld, int dtype) {
  return aligned(p, 16) && (ld * (dtype == NSML_F32 ? 4 : 2)) % 16 == 0;
}
inline bool valid_type(int dtype) { return dtype == NSML_F32 || dtype == NSML_BF16; }
inline bool valid_matrix(const void* p, int64_t rows, int64_t cols, int64_t ld, int dtype) {
  return p != nullptr && aligned(p, dtype == NSML_F32 ? 4 : 2) && (rows <= 1 || ld >= cols);
}
inline bool valid_codes(const void* p, int64_t rows, int64_t cols, int64_t ldq) {
  return p != nullptr && aligned(p, 16) && (rows <= 1 || (ldq >= cols && ldq % 16 == 0));
}
inline bool valid_sizes(int64_t rows, int64_t cols, int64_t max_cols) {
  return rows >= 0 && rows <= NSML_Q8_MAX_ROWS && cols >= 1 && cols <= max_cols;
}

}  // namespace q8
}  // namespace nsml
