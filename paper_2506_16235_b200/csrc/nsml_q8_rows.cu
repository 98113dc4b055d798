// Row-wise operators of the q8 format (nsml_q8.cuh): storing and restoring an activation, and the RMS norm with an 8-bit
// output.  All of them stream: their floor is the bytes of their arguments.
#include <type_traits>

#include "nsml_launch.h"
#include "nsml_q8.cuh"

namespace nsml {
namespace q8 {

// A row is held in registers between its maximum and its codes: four chunks of eight elements per thread, the threads of a
// row next to each other (16 bytes of bfloat16 each).  Rows of up to 1024 elements have a warp or a part of one (no block-wide
// step), wider ones a block.  What bounds these kernels is memory; what has to be right for that is enough loads in flight
// (norm of 16384 x 2048 bfloat16 with a residual: 37 us; eight chunks and a warp per row 55) and few instructions per
// element.  A line that every row of the GPU reads, such as the norm's weight, must come from L1: prefetching it there asked
// L2 for it every time, 34 us instead of 15 for 16384 x 768.
constexpr int kChunks = 4;
constexpr int kTeamThreads = 128;  // of a block whose warps have rows of their own

template <int THREADS>
__host__ __device__ constexpr int block_threads() { return THREADS <= 32 ? kTeamThreads : THREADS; }
template <int THREADS>
__device__ __forceinline__ int64_t my_row() {
  if constexpr (THREADS <= 32) return (int64_t)blockIdx.x * (kTeamThreads / THREADS) + threadIdx.x / THREADS;
  return blockIdx.x;
}

// ---- store -----------------------------------------------------------------------------------------------------------
// A maximum, then codes; one pass over memory for rows of up to 32768 elements.  16384 x 8192 bfloat16: 58 us, 6.9 TB/s;
// 8192 x 4096 float32 25 us.  Rows off 16-byte boundaries go element by element: 16383 x 2047 bfloat16 25 us (aligned 18).
template <int DTYPE, bool VEC, int THREADS>
__global__ void __launch_bounds__(block_threads<THREADS>())
k_q8_pack(const typename Elem<DTYPE>::type* __restrict__ x, int64_t rows, int cols, int64_t ldx, int8_t* __restrict__ codes, int64_t ldq,
          float* __restrict__ scales) {
  __shared__ uint32_t shared[32];
  pdl_wait();
  pdl_launch_dependents();
  const int64_t row = my_row<THREADS>();
  const int lane = my_lane<THREADS>(), end = row < rows ? cols : 0;  // (a row behind the last: nothing is read or written)
  const auto* from = x + row * ldx;
  Raw8<DTYPE, VEC> r[kChunks];
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < kChunks; ++i) r[i].template load<THREADS>(from, lane, i, end);
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    if (empty<VEC, THREADS>(i, cols)) break;
    float v[8];
    r[i].widen(v);
    top = top8(top, v);
  }
  // wider than the registers hold: read twice
  const int chunks = THREADS == 1024 ? (int)(((unsigned int)end + 8 * THREADS - 1) / (8 * THREADS)) : kChunks;
  for (int i = kChunks; i < chunks; ++i) {
    float v[8];
    load8<DTYPE, VEC, THREADS>(from, lane, i, end, v);
    top = top8(top, v);
  }
  float inv;
  const uint32_t amax = row_top<THREADS>(top, shared);
  const float scale = scale_of(amax, &inv);
  if (lane == 0 && row < rows) scales[row] = scale;
  int8_t* to = codes + row * ldq;
  const bool clamp = needs_clamp(amax);
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    if (empty<VEC, THREADS>(i, cols)) break;
    float v[8];
    r[i].widen(v);
    store8_codes<VEC, THREADS>(to, lane, i, end, clamp ? codes8<true>(v, inv) : codes8<false>(v, inv));
  }
  for (int i = kChunks; i < chunks; ++i) {
    float v[8];
    load8<DTYPE, VEC, THREADS>(from, lane, i, end, v);
    store8_codes<VEC, THREADS>(to, lane, i, end, clamp ? codes8<true>(v, inv) : codes8<false>(v, inv));
  }
}

// ---- restore ---------------------------------------------------------------------------------------------------------
// A block takes kSpan columns of a row; narrow rows several at a time.  16384 x 8192 to bfloat16: 61 us, 6.6 TB/s; to float32
// 16384 x 2048 27 us, 6.2 TB/s (a thread's 32 bytes in two stores of 16: 38 us).  Rows off 16-byte boundaries: 16383 x 2047 23
// and 36 us.
constexpr int kSpan = 8192;

template <int DTYPE, bool VEC, int THREADS>
__global__ void __launch_bounds__(block_threads<THREADS>())
k_q8_unpack(const int8_t* __restrict__ codes, int64_t ldq, const float* __restrict__ scales, int64_t rows, int cols,
            typename Elem<DTYPE>::type* __restrict__ out, int64_t ldo, unsigned int spans) {
  pdl_wait();
  pdl_launch_dependents();
  const unsigned int span = blockIdx.x % spans, group = blockIdx.x / spans;
  constexpr int kAtOnce = THREADS <= 32 ? kTeamThreads / THREADS : 1;
  const int64_t row = (int64_t)group * kAtOnce + (kAtOnce > 1 ? threadIdx.x / THREADS : 0);
  if (row >= rows) return;
  const int first = (int)span * kSpan, end = min(cols - first, kSpan), lane = my_lane<THREADS>();
  const float scale = scales[row];
  const int8_t* from = codes + row * ldq + first;
  auto* to = out + row * ldo + first;
  RawCodes8<VEC> q[kChunks];
#pragma unroll
  for (int i = 0; i < kChunks; ++i) q[i].template load<THREADS>(from, lane, i, end);
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    if (empty<VEC, THREADS>(i, end)) break;
    float v[8];
    q[i].numbers(v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], scale);
    store8<DTYPE, VEC, THREADS>(to, lane, i, end, v);
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
  int64_t rows, ldx, ldr, ldh, ldq;
  double inv_cols, eps;
  int cols;
  bool weight_bf16;
};

// 1/sqrt(v): two Newton steps in 64 bits on the float32 approximation (relative error 2^-22 -> 2^-43 -> a rounding or two of 64
// bits), where float32 holds v; v > 0, or NaN.  With one step a root next to a border between two float32 may be rounded to the
// wrong one.
__device__ __forceinline__ double reciprocal_root(double v) {
  if (!(v > 1e-30 && v < 1e30)) return 1.0 / sqrt(v);
  double y = (double)rsqrtf((float)v);
#pragma unroll
  for (int step = 0; step < 2; ++step) y = __fma_rn(0.5 * y, __fma_rn(-(v * y), y, 1.0), y);
  return y;
}

// h = rn(x + residual); rstd = 1/sqrt(sum h^2 / cols + eps): sum, quotient and root in 64 bits, rounded once, so that the
// codes do not depend on the order of the sum; y = (h rstd) weight; codes and scale of y.  16384 x 2048 bfloat16 with a residual:
// 37 us, 6.3 TB/s; without 22 us, where the conversions to 64 bits and the codes keep the issue slots as busy as the memory.
template <int DTYPE, bool VEC, int THREADS>
__global__ void __launch_bounds__(block_threads<THREADS>()) k_q8_norm(const NormArgs a) {
  using T = typename Elem<DTYPE>::type;
  __shared__ double shared_sum[32];
  __shared__ uint32_t shared_top[32];
  const int lane = my_lane<THREADS>();
  pdl_wait();
  pdl_launch_dependents();
  const int64_t row = my_row<THREADS>();
  const int end = row < a.rows ? a.cols : 0;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  Raw8<DTYPE, VEC> h[kChunks];
#pragma unroll
  for (int i = 0; i < kChunks; ++i) h[i].template load<THREADS>(x, lane, i, end);
  if (a.residual != nullptr) {
    const T* r = static_cast<const T*>(a.residual) + row * a.ldr;
    Raw8<DTYPE, VEC> w[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) w[i].template load<THREADS>(r, lane, i, end);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (empty<VEC, THREADS>(i, a.cols)) break;
      float p[8], q[8];
      h[i].widen(p);
      w[i].widen(q);
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = __fadd_rn(p[j], q[j]);
      h[i].round(p);
    }
  }
  if (a.h != nullptr) {
    T* to = static_cast<T*>(a.h) + row * a.ldh;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) h[i].template store<THREADS>(to, lane, i, end);
  }
  float y[kChunks][8];
  double sums[4] = {0.0, 0.0, 0.0, 0.0};  // (chains a quarter as long)
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    if (empty<VEC, THREADS>(i, a.cols)) break;
    h[i].widen(y[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[j & 3] = __fma_rn((double)y[i][j], (double)y[i][j], sums[j & 3]);
  }
  const double sum = row_sum<THREADS>((sums[0] + sums[1]) + (sums[2] + sums[3]), shared_sum);
  const float rstd = (float)reciprocal_root(sum * a.inv_cols + a.eps);
  if (lane == 0 && a.rstd != nullptr && row < a.rows) a.rstd[row] = rstd;
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {  // (elements past the end are 0, and NaN only where the row is not finite)
    if (empty<VEC, THREADS>(i, a.cols)) break;
    float w[8];
    load8_weight<VEC, THREADS>(a.weight, a.weight_bf16, lane, i, a.cols, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[i][j] = __fmul_rn(__fmul_rn(y[i][j], rstd), w[j]);
    top = top8(top, y[i]);
  }
  float inv;
  const uint32_t amax = row_top<THREADS>(top, shared_top);
  const float scale = scale_of(amax, &inv);
  if (lane == 0 && row < a.rows) a.scales[row] = scale;
  int8_t* to = a.codes + row * a.ldq;
  const bool clamp = needs_clamp(amax);
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    if (empty<VEC, THREADS>(i, a.cols)) break;
    store8_codes<VEC, THREADS>(to, lane, i, end, clamp ? codes8<true>(y[i], inv) : codes8<false>(y[i], inv));
  }
}

// Threads for a row of up to `cols` columns: 32 columns (four chunks) each.  MOST: no more of them than that.
template <int MOST = 1024, class Launch>
static int by_width(int64_t cols, Launch launch) {
  using std::integral_constant;
  if (cols <= 128) return launch(integral_constant<int, 4>{});
  if (cols <= 512) return launch(integral_constant<int, 16>{});
  if (cols <= 1024) return launch(integral_constant<int, 32>{});
  if (cols <= 2048) return launch(integral_constant<int, 64>{});
  if (cols <= 4096) return launch(integral_constant<int, 128>{});
  if (MOST <= 256 || cols <= 8192) return launch(integral_constant<int, 256>{});
  if constexpr (MOST > 256) {
    if (cols <= 16384) return launch(integral_constant<int, 512>{});
    return launch(integral_constant<int, 1024>{});
  }
}
template <int THREADS>
static dim3 row_grid(int64_t rows) {
  constexpr int at_once = THREADS <= 32 ? kTeamThreads / THREADS : 1;
  return dim3((unsigned int)((rows + at_once - 1) / at_once));
}

template <int DTYPE, bool VEC>
static int pack_rows(const void* x, int64_t rows, int64_t cols, int64_t ldx, int8_t* codes, int64_t ldq, float* scales, cudaStream_t st) {
  using T = typename Elem<DTYPE>::type;
  return by_width(cols, [&](auto threads) {
    constexpr int THREADS = threads;
    LaunchScope scope(K_Q8_PACK, st);
    const cudaError_t e = launch_in_stream(k_q8_pack<DTYPE, VEC, THREADS>, row_grid<THREADS>(rows), dim3(block_threads<THREADS>()), 0, st, 0,
                                      static_cast<const T*>(x), rows, (int)cols, ldx, codes, ldq, scales);
    return e == cudaSuccess ? NSML_OK : cuda_error();
  });
}

template <int DTYPE, bool VEC>
static int unpack_rows(const int8_t* codes, int64_t ldq, const float* scales, int64_t rows, int64_t cols, void* out, int64_t ldo, cudaStream_t st) {
  using T = typename Elem<DTYPE>::type;
  return by_width<kSpan / 32>(cols < kSpan ? cols : kSpan, [&](auto threads) {
    constexpr int THREADS = threads;
    const int64_t spans = (cols + kSpan - 1) / kSpan, blocks = spans * row_grid<THREADS>(rows).x;
    if (blocks > NSML_Q8_MAX_ROWS) return (int)NSML_ERR_ARG;
    LaunchScope scope(K_Q8_UNPACK, st);
    const cudaError_t e = launch_in_stream(k_q8_unpack<DTYPE, VEC, THREADS>, dim3((unsigned int)blocks), dim3(block_threads<THREADS>()), 0, st, 0,
                                      codes, ldq, scales, rows, (int)cols, static_cast<T*>(out), ldo, (unsigned int)spans);
    return e == cudaSuccess ? (int)NSML_OK : cuda_error();
  });
}

template <int DTYPE, bool VEC>
static int norm_rows(const NormArgs& a, cudaStream_t st) {
  return by_width(a.cols, [&](auto threads) {
    constexpr int THREADS = threads;
    LaunchScope scope(K_Q8_NORM, st);
    const cudaError_t e = launch_in_stream(k_q8_norm<DTYPE, VEC, THREADS>, row_grid<THREADS>(a.rows), dim3(block_threads<THREADS>()), 0, st, 0, a);
    return e == cudaSuccess ? NSML_OK : cuda_error();
  });
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
  const bool vec = cols % 8 == 0 && rows16(x, ldx, dtype);
  if (dtype == NSML_F32) return vec ? pack_rows<NSML_F32, true>(x, rows, cols, ldx, codes, ldq, scales, st) : pack_rows<NSML_F32, false>(x, rows, cols, ldx, codes, ldq, scales, st);
  return vec ? pack_rows<NSML_BF16, true>(x, rows, cols, ldx, codes, ldq, scales, st) : pack_rows<NSML_BF16, false>(x, rows, cols, ldx, codes, ldq, scales, st);
}

int nsml_q8_unpack(const int8_t* codes, int64_t ldq, const float* scales, int64_t rows, int64_t cols, void* out, int64_t ldo, int dtype, void* stream) {
  if (!valid_type(dtype) || !valid_sizes(rows, cols, NSML_Q8_MAX_COLS)) return NSML_ERR_ARG;
  if (rows == 0) return NSML_OK;
  if (!valid_codes(codes, rows, cols, ldq) || scales == nullptr || !aligned(scales, 4) || !valid_matrix(out, rows, cols, ldo, dtype)) return NSML_ERR_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool vec = cols % 8 == 0 && rows16(out, ldo, dtype);
  if (dtype == NSML_F32) return vec ? unpack_rows<NSML_F32, true>(codes, ldq, scales, rows, cols, out, ldo, st) : unpack_rows<NSML_F32, false>(codes, ldq, scales, rows, cols, out, ldo, st);
  return vec ? unpack_rows<NSML_BF16, true>(codes, ldq, scales, rows, cols, out, ldo, st) : unpack_rows<NSML_BF16, false>(codes, ldq, scales, rows, cols, out, ldo, st);
}

int nsml_q8_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ldr, int64_t rows, int64_t cols, int dtype,
                     const void* weight, int weight_dtype, double eps, void* h, int64_t ldh, int8_t* codes, int64_t ldq,
                     float* scales, float* rstd, void* stream) {
  if (!valid_type(dtype) || !valid_type(weight_dtype) || !valid_sizes(rows, cols, NSML_Q8_MAX_NORM_COLS) || !((float)eps > 0.0f) || !(eps <= 3.4e38))
    return NSML_ERR_ARG;
  if (rows == 0) return NSML_OK;
  if (!valid_matrix(x, rows, cols, ldx, dtype) || !valid_codes(codes, rows, cols, ldq) || scales == nullptr || !aligned(scales, 4)) return NSML_ERR_ARG;
  if (!valid_matrix(weight, 1, cols, cols, weight_dtype) || (residual != nullptr && !valid_matrix(residual, rows, cols, ldr, dtype)) ||
      (h != nullptr && !valid_matrix(h, rows, cols, ldh, dtype)) || (rstd != nullptr && !aligned(rstd, 4)))
    return NSML_ERR_ARG;
  NormArgs a = {};
  a.x = x; a.residual = residual; a.weight = weight; a.h = h; a.codes = codes; a.scales = scales; a.rstd = rstd;
  a.rows = rows; a.cols = (int)cols; a.inv_cols = 1.0 / (double)cols; a.ldx = ldx; a.ldr = ldr; a.ldh = ldh; a.ldq = ldq; a.eps = eps;
  a.weight_bf16 = weight_dtype == NSML_BF16;
  const bool vec = cols % 8 == 0 && rows16(x, ldx, dtype) && aligned(weight, 16) && (residual == nullptr || rows16(residual, ldr, dtype)) &&
                   (h == nullptr || rows16(h, ldh, dtype));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == NSML_F32) return vec ? norm_rows<NSML_F32, true>(a, st) : norm_rows<NSML_F32, false>(a, st);
  return vec ? norm_rows<NSML_BF16, true>(a, st) : norm_rows<NSML_BF16, false>(a, st);
}

}  // extern "C"
