// Row-wise operators of the q8 format (nsml_q8.cuh): storing and restoring an activation, the RMS norm with an 8-bit output
// and its gradient.  All of them stream: their floor is the bytes of their arguments.
#include <type_traits>

#include "nsml_launch.h"
#include "nsml_q8.cuh"

namespace nsml {
namespace q8 {

// A row is held in registers between its maximum and its codes: CHUNKS pieces of eight elements per thread, the threads of
// a row next to each other (16 bytes of bfloat16 each).  Rows of up to 2048 elements have a warp each (no block-wide step);
// wider ones a block.
constexpr int kWarpRows = 4;  // rows per block where a row has a warp

template <int THREADS>
__device__ __forceinline__ int64_t my_row() {
  if constexpr (THREADS == 32) return (int64_t)blockIdx.x * kWarpRows + (threadIdx.x >> 5);
  return blockIdx.x;
}
template <int THREADS>
__device__ __forceinline__ int my_lane() { return THREADS == 32 ? threadIdx.x & 31 : threadIdx.x; }

// ---- store -----------------------------------------------------------------------------------------------------------
template <int DTYPE, int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS == 32 ? 32 * kWarpRows : THREADS)
k_q8_pack(const typename Elem<DTYPE>::type* __restrict__ x, int64_t rows, int64_t cols, int64_t ldx, bool vec, int8_t* __restrict__ codes,
          int64_t ldq, float* __restrict__ scales) {
  __shared__ uint32_t shared[32];
  pdl_wait();
  pdl_launch_dependents();
  const int64_t row = my_row<THREADS>();
  if (row >= rows) return;
  const int lane = my_lane<THREADS>();
  const auto* from = x + row * ldx;
  float v[CHUNKS][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) load8<DTYPE>(from, 8 * (int64_t)(lane + i * THREADS), cols, vec, v[i]);
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
  // wider than the registers hold: read twice
  for (int64_t c = 8 * ((int64_t)lane + CHUNKS * THREADS); c < cols; c += 8 * THREADS) {
    float w[8];
    load8<DTYPE>(from, c, cols, vec, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(w[j]) & 0x7FFFFFFFu);
  }
  float inv;
  const float scale = scale_of(row_max<THREADS>(top, shared), &inv);
  if (lane == 0) scales[row] = scale;
  int8_t* to = codes + row * ldq;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    int q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = code_of(v[i][j], inv);
    store8_codes(to, 8 * (int64_t)(lane + i * THREADS), cols, q);
  }
  for (int64_t c = 8 * ((int64_t)lane + CHUNKS * THREADS); c < cols; c += 8 * THREADS) {
    float w[8];
    int q[8];
    load8<DTYPE>(from, c, cols, vec, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = code_of(w[j], inv);
    store8_codes(to, c, cols, q);
  }
}

// ---- restore ---------------------------------------------------------------------------------------------------------
template <int DTYPE>
__global__ void __launch_bounds__(256)
k_q8_unpack(const int8_t* __restrict__ codes, int64_t ldq, const float* __restrict__ scales, int64_t rows, int64_t cols,
            typename Elem<DTYPE>::type* __restrict__ out, int64_t ldo, bool vec) {
  pdl_wait();
  pdl_launch_dependents();
  const int64_t chunks = (cols + 7) / 8, total = rows * chunks;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t row = i / chunks, c = 8 * (i - row * chunks);
    float v[8];
    load8_codes(codes + row * ldq, c, cols, scales[row], v);
    store8<DTYPE>(out + row * ldo, c, cols, vec, v);
  }
}

// ---- RMS norm, 8-bit output --------------------------------------------------------------------------------------------
struct NormArgs {
  const void* x;
  const void* residual;  // may be null
  const void* weight;
  void* h;               // may be null
  int8_t* codes;
  float* scales;
  float* rstd;           // may be null
  int64_t rows, cols, ldx, ldr, ldh, ldq;
  float eps;
  bool vec_in, vec_h, vec_w, weight_bf16;
};

// h = rn(x + residual); rstd = 1/sqrt(sum h^2 / cols + eps): sum, quotient and root in 64 bits, rounded once, so that the
// codes do not depend on the order of the sum; y = (h rstd) weight; codes and scale of y.
template <int DTYPE, int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS == 32 ? 32 * kWarpRows : THREADS) k_q8_norm(const NormArgs a) {
  using T = typename Elem<DTYPE>::type;
  __shared__ double shared_sum[32];
  __shared__ uint32_t shared_max[32];
  pdl_wait();
  pdl_launch_dependents();
  const int64_t row = my_row<THREADS>();
  if (row >= a.rows) return;
  const int lane = my_lane<THREADS>();
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  float v[CHUNKS][8];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) load8<DTYPE>(x, 8 * (int64_t)(lane + i * THREADS), a.cols, a.vec_in, v[i]);
  if (a.residual != nullptr) {
    const T* r = static_cast<const T*>(a.residual) + row * a.ldr;
    float w[CHUNKS][8];
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) load8<DTYPE>(r, 8 * (int64_t)(lane + i * THREADS), a.cols, a.vec_in, w[i]);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = (float)(T)__fadd_rn(v[i][j], w[i][j]);
  }
  if (a.h != nullptr) {
    T* h = static_cast<T*>(a.h) + row * a.ldh;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) store8<DTYPE>(h, 8 * (int64_t)(lane + i * THREADS), a.cols, a.vec_h, v[i]);
  }
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) sum = __fma_rn((double)v[i][j], (double)v[i][j], sum);
  sum = row_sum<THREADS>(sum, shared_sum);
  const float rstd = (float)(1.0 / sqrt(sum / (double)a.cols + (double)a.eps));
  if (lane == 0 && a.rstd != nullptr) a.rstd[row] = rstd;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int64_t c = 8 * (int64_t)(lane + i * THREADS);
    float w[8];
    if (a.weight_bf16) load8<NSML_BF16>(static_cast<const __nv_bfloat16*>(a.weight), c, a.cols, a.vec_w, w);
    else load8<NSML_F32>(static_cast<const float*>(a.weight), c, a.cols, a.vec_w, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // (an element past the end is 0 whatever rstd is)
      v[i][j] = c + j < a.cols ? __fmul_rn(__fmul_rn(v[i][j], rstd), w[j]) : 0.0f;
      top = max(top, __float_as_uint(v[i][j]) & 0x7FFFFFFFu);
    }
  }
  float inv;
  const float scale = scale_of(row_max<THREADS>(top, shared_max), &inv);
  if (lane == 0) a.scales[row] = scale;
  int8_t* to = a.codes + row * a.ldq;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    int q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = code_of(v[i][j], inv);
    store8_codes(to, 8 * (int64_t)(lane + i * THREADS), a.cols, q);
  }
}

// ---- its gradient ------------------------------------------------------------------------------------------------------
struct NormGradArgs {
  const void* dy;
  const void* dh;       // may be null
  const void* h;        // rows as they are, or
  const int8_t* codes;  // their 8-bit checkpoint
  const float* scales;
  const float* rstd;
  const void* weight;
  void* dx;
  float* partial;       // [gridDim.x][cols]: every block's part of the weight's gradient
  int64_t rows, cols, ldy, lddh, ldh, ldq, lddx;
  bool vec, vec_w, weight_bf16;
};

// n = h rstd, g = dy weight, c = mean(g n): dx = rstd (g - n c) + dh, and dweight = sum over rows of dy n.  A block takes
// every gridDim.x-th row; a thread keeps its columns' part of dweight in registers, so that the sum's order depends on the
// sizes alone.
template <int DTYPE, bool PACKED, int THREADS, int CHUNKS>
__global__ void __launch_bounds__(THREADS) k_q8_norm_grad(const NormGradArgs a) {
  using T = typename Elem<DTYPE>::type;
  __shared__ double shared[32];
  pdl_wait();
  pdl_launch_dependents();
  float dw[CHUNKS][8], w[CHUNKS][8];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int64_t c = 8 * (int64_t)(threadIdx.x + i * THREADS);
    if (a.weight_bf16) load8<NSML_BF16>(static_cast<const __nv_bfloat16*>(a.weight), c, a.cols, a.vec_w, w[i]);
    else load8<NSML_F32>(static_cast<const float*>(a.weight), c, a.cols, a.vec_w, w[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
  }
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float rstd = a.rstd[row];
    float n[CHUNKS][8], g[CHUNKS][8];
    double dot = 0.0;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int64_t c = 8 * (int64_t)(threadIdx.x + i * THREADS);
      load8<DTYPE>(static_cast<const T*>(a.dy) + row * a.ldy, c, a.cols, a.vec, g[i]);
      if constexpr (PACKED) load8_codes(a.codes + row * a.ldq, c, a.cols, a.scales[row], n[i]);
      else load8<DTYPE>(static_cast<const T*>(a.h) + row * a.ldh, c, a.cols, a.vec, n[i]);
    }
    float part = 0.0f;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = 8 * (int64_t)(threadIdx.x + i * THREADS) + j < a.cols;
        n[i][j] = in ? __fmul_rn(n[i][j], rstd) : 0.0f;
        dw[i][j] = __fmaf_rn(g[i][j], n[i][j], dw[i][j]);
        g[i][j] = __fmul_rn(g[i][j], w[i][j]);
        part = __fmaf_rn(g[i][j], n[i][j], part);
      }
    dot = row_sum<THREADS>((double)part, shared);
    const float mean = (float)(dot / (double)a.cols);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int64_t c = 8 * (int64_t)(threadIdx.x + i * THREADS);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[i][j] = __fmul_rn(rstd, __fsub_rn(g[i][j], __fmul_rn(n[i][j], mean)));
      if (a.dh != nullptr) {
        float d[8];
        load8<DTYPE>(static_cast<const T*>(a.dh) + row * a.lddh, c, a.cols, a.vec, d);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[i][j] = __fadd_rn(g[i][j], d[j]);
      }
      store8<DTYPE>(static_cast<T*>(a.dx) + row * a.lddx, c, a.cols, a.vec, g[i]);
    }
  }
  if (a.partial != nullptr) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
      store8<NSML_F32>(a.partial + (int64_t)blockIdx.x * a.cols, 8 * (int64_t)(threadIdx.x + i * THREADS), a.cols, a.cols % 4 == 0, dw[i]);
  }
}

// dweight (+)= sum of the blocks' parts, in their order
__global__ void __launch_bounds__(1024) k_q8_norm_weight(const float* __restrict__ partial, int parts, int64_t cols, void* dweight,
                                                        bool bf16, bool zero_first) {
  __shared__ float sums[32][33];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  float s = 0.0f;
  if (c < cols)
    for (int p = warp; p < parts; p += 32) s = __fadd_rn(s, partial[(int64_t)p * cols + c]);
  sums[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= cols) return;
  s = 0.0f;
#pragma unroll
  for (int w = 0; w < 32; ++w) s = __fadd_rn(s, sums[w][lane]);
  if (bf16) {
    __nv_bfloat16* to = static_cast<__nv_bfloat16*>(dweight) + c;
    *to = __float2bfloat16_rn(zero_first ? s : __fadd_rn((float)*to, s));
  } else {
    float* to = static_cast<float*>(dweight) + c;
    *to = zero_first ? s : __fadd_rn(*to, s);
  }
}

static bool rows16(const void* p, int64_t ld, int dtype) {
  return aligned(p, 16) && (ld * (dtype == NSML_F32 ? 4 : 2)) % 16 == 0;
}
static bool valid_type(int dtype) { return dtype == NSML_F32 || dtype == NSML_BF16; }
static bool valid_matrix(const void* p, int64_t rows, int64_t cols, int64_t ld, int dtype) {
  return p != nullptr && aligned(p, dtype == NSML_F32 ? 4 : 2) && (rows <= 1 || ld >= cols);
}
static bool valid_codes(const void* p, int64_t rows, int64_t cols, int64_t ldq) {
  return p != nullptr && aligned(p, 16) && (rows <= 1 || (ldq >= cols && ldq % 16 == 0));
}
static bool valid_sizes(int64_t rows, int64_t cols, int64_t max_cols) {
  return rows >= 0 && rows <= NSML_Q8_MAX_ROWS && cols >= 1 && cols <= max_cols;
}

// The gradient of the norm: threads per block (a chunk of eight columns each, up to 8192 columns), and blocks: 2048 threads
// per SM of a B200, or a row each; also the height of the workspace's table.
static int grad_threads(int64_t cols) { return cols <= 1024 ? 128 : cols <= 2048 ? 256 : cols <= 4096 ? 512 : 1024; }
static int grad_blocks(int64_t rows, int64_t cols) {
  const int most = 148 * 2048 / grad_threads(cols);
  return rows < most ? (int)rows : most;
}

template <class Launch>
static int by_width(int64_t cols, Launch launch) {
  using std::integral_constant;
  if (cols <= 256) return launch(integral_constant<int, 32>{}, integral_constant<int, 1>{});
  if (cols <= 512) return launch(integral_constant<int, 32>{}, integral_constant<int, 2>{});
  if (cols <= 1024) return launch(integral_constant<int, 32>{}, integral_constant<int, 4>{});
  if (cols <= 2048) return launch(integral_constant<int, 32>{}, integral_constant<int, 8>{});
  if (cols <= 4096) return launch(integral_constant<int, 128>{}, integral_constant<int, 4>{});
  if (cols <= 8192) return launch(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  if (cols <= 16384) return launch(integral_constant<int, 512>{}, integral_constant<int, 4>{});
  return launch(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}
static unsigned int row_grid(int64_t rows, int threads) { return (unsigned int)(threads == 32 ? (rows + kWarpRows - 1) / kWarpRows : rows); }

template <int DTYPE>
static int pack_rows(const void* x, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes, int64_t ldq, float* scales, cudaStream_t st) {
  using T = typename Elem<DTYPE>::type;
  return by_width(cols, [&](auto threads, auto chunks) {
    constexpr int THREADS = threads, CHUNKS = chunks;
    LaunchScope scope(K_Q8_PACK, st);
    const cudaError_t e = launch_prio(k_q8_pack<DTYPE, THREADS, CHUNKS>, dim3(row_grid(rows, THREADS)), dim3(THREADS == 32 ? 32 * kWarpRows : THREADS),
                                      0, st, false, 0, false, true, static_cast<const T*>(x), rows, cols, ldx, rows16(x, ldx, DTYPE), codes, ldq, scales);
    return e == cudaSuccess ? NSML_OK : cuda_error();
  });
}

template <int DTYPE>
static int norm_rows(const NormArgs& a, cudaStream_t st) {
  return by_width(a.cols, [&](auto threads, auto chunks) {
    constexpr int THREADS = threads, CHUNKS = chunks;
    LaunchScope scope(K_Q8_NORM, st);
    const cudaError_t e = launch_prio(k_q8_norm<DTYPE, THREADS, CHUNKS>, dim3(row_grid(a.rows, THREADS)), dim3(THREADS == 32 ? 32 * kWarpRows : THREADS),
                                      0, st, false, 0, false, true, a);
    return e == cudaSuccess ? NSML_OK : cuda_error();
  });
}

template <int DTYPE, bool PACKED>
static int norm_grad_rows(const NormGradArgs& a, cudaStream_t st) {
  auto go = [&](auto threads, auto chunks) {
    constexpr int THREADS = threads, CHUNKS = chunks;
    LaunchScope scope(K_Q8_NORM_GRAD, st);
    const cudaError_t e = launch_prio(k_q8_norm_grad<DTYPE, PACKED, THREADS, CHUNKS>, dim3(grad_blocks(a.rows, a.cols)), dim3(THREADS), 0, st, false, 0, false, true, a);
    return e == cudaSuccess ? NSML_OK : cuda_error();
  };
  using std::integral_constant;
  if (a.cols <= 1024) return go(integral_constant<int, 128>{}, integral_constant<int, 1>{});
  if (a.cols <= 2048) return go(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  if (a.cols <= 4096) return go(integral_constant<int, 512>{}, integral_constant<int, 1>{});
  if (a.cols <= 8192) return go(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
  if (a.cols <= 16384) return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  return go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

}  // namespace q8
}  // namespace nsml

using namespace nsml;
using namespace nsml::q8;

extern "C" {

int64_t nsml_q8_row_bytes(int64_t cols) { return cols < 1 || cols > NSML_Q8_MAX_COLS ? 0 : (cols + 15) / 16 * 16; }

int nsml_q8_pack(const void* x, int64_t rows, int64_t cols, int64_t ldx, int dtype, int8_t* codes, int64_t ldq, float* scales, void* stream) {
  if (!valid_type(dtype) || !valid_sizes(rows, cols, NSML_Q8_MAX_COLS)) return NSML_ERR_ARG;
  if (rows == 0) return NSML_OK;
  if (!valid_matrix(x, rows, cols, ldx, dtype) || !valid_codes(codes, rows, cols, ldq) || scales == nullptr || !aligned(scales, 4)) return NSML_ERR_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return dtype == NSML_F32 ? pack_rows<NSML_F32>(x, rows, cols, ldx, codes, ldq, scales, st)
                           : pack_rows<NSML_BF16>(x, rows, cols, ldx, codes, ldq, scales, st);
}

int nsml_q8_unpack(const int8_t* codes, int64_t ldq, const float* scales, int64_t rows, int64_t cols, void* out, int64_t ldo, int dtype, void* stream) {
  if (!valid_type(dtype) || !valid_sizes(rows, cols, NSML_Q8_MAX_COLS)) return NSML_ERR_ARG;
  if (rows == 0) return NSML_OK;
  if (!valid_codes(codes, rows, cols, ldq) || scales == nullptr || !aligned(scales, 4) || !valid_matrix(out, rows, cols, ldo, dtype)) return NSML_ERR_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int64_t total = rows * ((cols + 7) / 8), blocks = (total + 255) / 256;
  const unsigned int grid = (unsigned int)(blocks < (1 << 30) ? blocks : (1 << 30));
  const bool vec = rows16(out, ldo, dtype);
  LaunchScope scope(K_Q8_UNPACK, st);
  const cudaError_t e = dtype == NSML_F32
      ? launch_prio(k_q8_unpack<NSML_F32>, dim3(grid), dim3(256), 0, st, false, 0, false, true, codes, ldq, scales, rows, cols, static_cast<float*>(out), ldo, vec)
      : launch_prio(k_q8_unpack<NSML_BF16>, dim3(grid), dim3(256), 0, st, false, 0, false, true, codes, ldq, scales, rows, cols, static_cast<__nv_bfloat16*>(out), ldo, vec);
  return e == cudaSuccess ? NSML_OK : cuda_error();
}

int nsml_q8_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, int64_t rows, int64_t cols, int dtype,
                     const void* weight, int weight_dtype, float eps, void* h, int64_t ldh, int8_t* codes, int64_t ldq,
                     float* scales, float* rstd, void* stream) {
  if (!valid_type(dtype) || !valid_type(weight_dtype) || !valid_sizes(rows, cols, NSML_Q8_MAX_NORM_COLS) || !(eps > 0.0f) || !(eps <= 3.4e38f))
    return NSML_ERR_ARG;
  if (rows == 0) return NSML_OK;
  if (!valid_matrix(x, rows, cols, ldx, dtype) || !valid_codes(codes, rows, cols, ldq) || scales == nullptr || !aligned(scales, 4)) return NSML_ERR_ARG;
  if (!valid_matrix(weight, 1, cols, cols, weight_dtype) || (residual != nullptr && !valid_matrix(residual, rows, cols, ldr, dtype)) ||
      (h != nullptr && !valid_matrix(h, rows, cols, ldh, dtype)) || (rstd != nullptr && !aligned(rstd, 4)))
    return NSML_ERR_ARG;
  NormArgs a = {};
  a.x = x; a.residual = residual; a.weight = weight; a.h = h; a.codes = codes; a.scales = scales; a.rstd = rstd;
  a.rows = rows; a.cols = cols; a.ldx = ldx; a.ldr = ldr; a.ldh = ldh; a.ldq = ldq; a.eps = eps;
  a.vec_in = rows16(x, ldx, dtype) && (residual == nullptr || rows16(residual, ldr, dtype));
  a.vec_h = rows16(h, ldh, dtype);
  a.vec_w = aligned(weight, 16);
  a.weight_bf16 = weight_dtype == NSML_BF16;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return dtype == NSML_F32 ? norm_rows<NSML_F32>(a, st) : norm_rows<NSML_BF16>(a, st);
}

size_t nsml_q8_rms_norm_backward_workspace_bytes(int64_t cols) {
  if (cols < 1 || cols > NSML_Q8_MAX_NORM_COLS) return 0;
  return align_up((size_t)grad_blocks(NSML_Q8_MAX_ROWS, cols) * (size_t)cols * 4, 256);
}

int nsml_q8_rms_norm_backward(const void* dy, int64_t ldy, const void* dh, int64_t lddh, const void* h, int64_t ldh,
                              const int8_t* codes, int64_t ldq, const float* scales, const float* rstd, int64_t rows,
                              int64_t cols, int dtype, const void* weight, int weight_dtype, void* dx, int64_t lddx,
                              void* dweight, int dweight_dtype, int zero_first, void* workspace, size_t workspace_bytes,
                              void* stream) {
  if (!valid_type(dtype) || !valid_type(weight_dtype) || !valid_type(dweight_dtype) || !valid_sizes(rows, cols, NSML_Q8_MAX_NORM_COLS)) return NSML_ERR_ARG;
  if ((h == nullptr) == (codes == nullptr) && rows > 0) return NSML_ERR_ARG;
  if (rows > 0) {
    if (!valid_matrix(dy, rows, cols, ldy, dtype) || !valid_matrix(dx, rows, cols, lddx, dtype) || rstd == nullptr || !aligned(rstd, 4)) return NSML_ERR_ARG;
    if (dh != nullptr && !valid_matrix(dh, rows, cols, lddh, dtype)) return NSML_ERR_ARG;
    if (h != nullptr && !valid_matrix(h, rows, cols, ldh, dtype)) return NSML_ERR_ARG;
    if (codes != nullptr && (!valid_codes(codes, rows, cols, ldq) || scales == nullptr || !aligned(scales, 4))) return NSML_ERR_ARG;
    if (!valid_matrix(weight, 1, cols, cols, weight_dtype)) return NSML_ERR_ARG;
  }
  if (dweight != nullptr) {
    if (!aligned(dweight, dweight_dtype == NSML_F32 ? 4 : 2) || workspace == nullptr || !aligned(workspace, 256)) return NSML_ERR_ARG;
    if (workspace_bytes < nsml_q8_rms_norm_backward_workspace_bytes(cols)) return NSML_ERR_CAPACITY;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (rows > 0) {
    NormGradArgs a = {};
    a.dy = dy; a.dh = dh; a.h = h; a.codes = codes; a.scales = scales; a.rstd = rstd; a.weight = weight; a.dx = dx;
    a.partial = dweight != nullptr ? static_cast<float*>(workspace) : nullptr;
    a.rows = rows; a.cols = cols; a.ldy = ldy; a.lddh = lddh; a.ldh = ldh; a.ldq = ldq; a.lddx = lddx;
    a.vec = rows16(dy, ldy, dtype) && rows16(dx, lddx, dtype) && (dh == nullptr || rows16(dh, lddh, dtype)) && (h == nullptr || rows16(h, ldh, dtype));
    a.vec_w = aligned(weight, 16);
    a.weight_bf16 = weight_dtype == NSML_BF16;
    const bool packed = codes != nullptr;
    const int rc = dtype == NSML_F32 ? (packed ? norm_grad_rows<NSML_F32, true>(a, st) : norm_grad_rows<NSML_F32, false>(a, st))
                                     : (packed ? norm_grad_rows<NSML_BF16, true>(a, st) : norm_grad_rows<NSML_BF16, false>(a, st));
    if (rc != NSML_OK) return rc;
  }
  if (dweight != nullptr) {
    LaunchScope scope(K_Q8_NORM_WEIGHT, st);
    const cudaError_t e = launch_prio(k_q8_norm_weight, dim3((unsigned int)((cols + 31) / 32)), dim3(1024), 0, st, false, 0, true, true,
                                      static_cast<const float*>(workspace), grad_blocks(rows, cols), cols, dweight,
                                      dweight_dtype == NSML_BF16, zero_first != 0);
    if (e != cudaSuccess) return cuda_error();
  }
  return NSML_OK;
}

}  // extern "C"
