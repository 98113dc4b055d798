// Gradient of the RMS norm with an 8-bit output (nsml_q8.cuh).  It streams: its floor is the bytes of its arguments.
#include <atomic>
#include <type_traits>

#include "nsml_launch.h"
#include "nsml_q8.cuh"

namespace nsml {
namespace q8 {

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
  int64_t rows, ldy, lddh, ldh, ldq, lddx;
  int cols;
  bool weight_bf16;
};

// n = h rstd, g = dy weight, c = mean(g n): dx = rstd (g - n c) + dh, and dweight = sum over rows of dy n, worked out as
//   p = dy h,  dweight += p rstd,  c = rstd mean(p weight),  dx = rstd (dy weight - h (rstd c)) + dh
// (few operations per element: the issue rate is near the memory's).  THREADS threads take a row, blocks of 256 threads several
// rows next to each other, and every so many-th row after them.  A thread's chunks of the next row are copied to its own places
// in shared memory meanwhile (asynchronous copies: no registers, and no barrier, since nobody else reads them); it reads them
// there twice and keeps its columns' part of dweight in registers.  The block's rows add theirs up in the end, so that the
// sum's order depends on the sizes alone.  16384 x 2048 bfloat16, rows in 8 bits and dh: 41 us with the weight's sum behind it
// (235 MB, 5.7 TB/s); from bfloat16 rows without dh 36 us.  Rows off 16-byte boundaries: 16383 x 2047 67 us.
constexpr int kGradBlock = 256;

template <int THREADS>
__host__ __device__ constexpr int grad_block() { return THREADS < kGradBlock ? kGradBlock : THREADS; }

template <class Raw>
__device__ __forceinline__ void forget(Raw& r) {  // the compiler is not to keep what it has worked out from r
#pragma unroll
  for (uint32_t& w : r.w) asm volatile("" : "+r"(w));
}

template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// Where a thread's chunks of the next row wait: two sets of dy, h (or codes) and dh; one where two do not fit, which is filled
// again as soon as a chunk has been read for the last time (7056 x 9680 float32 with dh 401 us without, 275 with).
template <int DTYPE, bool VEC, int THREADS, int CHUNKS>
struct GradStage {
  static constexpr int kPiece = sizeof(Raw8<DTYPE, true>);
  static constexpr size_t kSet = (size_t)3 * CHUNKS * kPiece * grad_block<THREADS>();
  static constexpr size_t kRoom = 200 * 1024 / (THREADS <= kGradBlock ? 2 : 1);  // (of two blocks, where an SM has two)
  static constexpr int kSets = !VEC || kSet > kRoom ? 0 : 2 * kSet <= kRoom ? 2 : 1;
  static constexpr bool kAhead = kSets != 0;
  static constexpr size_t kSum = THREADS < kGradBlock ? (size_t)kGradBlock * CHUNKS * 32 : 0;       // the rows' parts of dweight, in the end
  static constexpr size_t kSmem = kAhead ? kSets * kSet : kSum;
  static_assert(!kAhead || kSets * kSet >= kSum, "");
};

// KEEP: the weight has the rows' type, and a thread keeps its part in registers, as it is in memory (read from L1 for every row:
// 16384 x 2048 bfloat16 49 us instead of 36).
template <int DTYPE, bool PACKED, bool VEC, bool KEEP, int THREADS, int CHUNKS>
__global__ void __launch_bounds__(grad_block<THREADS>(), THREADS <= kGradBlock ? 2 : 1) k_q8_norm_grad(const NormGradArgs a) {
  using T = typename Elem<DTYPE>::type;
  using G = GradStage<DTYPE, VEC, THREADS, CHUNKS>;
  constexpr int kBlock = grad_block<THREADS>(), kTeams = kBlock / THREADS, kWarps = THREADS > 32 ? THREADS / 32 : 1;
  extern __shared__ uint4 stage[];
  __shared__ float shared[2][kTeams][kWarps];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = my_lane<THREADS>(), team = threadIdx.x / THREADS;
  const int64_t step = (int64_t)gridDim.x * kTeams;
  // (every team of a block makes the same turns: rows behind the last are zeros)
  const int64_t turns = (a.rows - (int64_t)blockIdx.x * kTeams + step - 1) / step;
  float dw[CHUNKS][8];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[i][j] = 0.0f;
  Raw8<DTYPE, VEC> weight[KEEP ? CHUNKS : 1];
  if constexpr (KEEP)
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) weight[i].template load<THREADS>(static_cast<const T*>(a.weight), lane, i, a.cols);
  auto weights = [&](int i, float (&w)[8]) {
    if constexpr (KEEP) weight[i].widen(w);
    else load8_weight<VEC, THREADS>(a.weight, a.weight_bf16, lane, i, a.cols, w);
  };
  const float inv_cols = 1.0f / (float)a.cols;
  int64_t row = (int64_t)blockIdx.x * kTeams + team;
  // this thread's chunk i of operand o (dy, h or codes, dh)
  auto place = [&](int set, int o, int i) {
    return reinterpret_cast<unsigned char*>(stage) + set * G::kSet + ((size_t)(o * CHUNKS + i) * kBlock + threadIdx.x) * G::kPiece;
  };
  auto chunk_ahead = [&](int set, int64_t at, int i) {
    const unsigned int c = column<VEC, THREADS>(lane, i, 0);
    if (at >= a.rows || c >= (unsigned int)a.cols) return;
    const T *dy = static_cast<const T*>(a.dy) + at * a.ldy, *h = static_cast<const T*>(a.h) + at * a.ldh, *dh = static_cast<const T*>(a.dh) + at * a.lddh;
#pragma unroll
    for (int k = 0; k < G::kPiece; k += 16) {
      copy_async<16>(place(set, 0, i) + k, reinterpret_cast<const char*>(dy + c) + k);
      if constexpr (!PACKED) copy_async<16>(place(set, 1, i) + k, reinterpret_cast<const char*>(h + c) + k);
      if (a.dh != nullptr) copy_async<16>(place(set, 2, i) + k, reinterpret_cast<const char*>(dh + c) + k);
    }
    if constexpr (PACKED) copy_async<8>(place(set, 1, i), a.codes + at * a.ldq + c);
  };
  auto ahead = [&](int set, int64_t at) {
    if constexpr (G::kAhead) {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) chunk_ahead(set, at, i);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
  };
  auto scalars = [&](int64_t at, float& rstd, float& factor) {  // factor: from what h holds to n (exact for a power of two)
    rstd = at < a.rows ? a.rstd[at] : 0.0f;
    factor = PACKED && at < a.rows ? a.scales[at] : 1.0f;
  };
  if constexpr (G::kAhead) {  // chunks past the end stay 0: no branches around them
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
      if (column<VEC, THREADS>(lane, i, 0) >= (unsigned int)a.cols)
        for (int k = 0; k < 3 * G::kSets * G::kPiece; k += 16) *reinterpret_cast<uint4*>(place(k / (3 * G::kPiece), k / G::kPiece % 3, i) + k % G::kPiece) = make_uint4(0, 0, 0, 0);
  }
  // rows that cannot be copied 16 bytes at a time: the next one is loaded into registers meanwhile, where they suffice
  constexpr bool kNext = !G::kAhead && THREADS <= 512;
  // the widest of them are read again (from L2) instead: several chunks of a row in registers are too many for 1024 threads
  // (7056 x 9681 bfloat16 with dh 600 us with four, 364 with two, 275 read again)
  constexpr bool kAgain = !G::kAhead && CHUNKS > 1 && THREADS == 1024;
  struct {
    Raw8<DTYPE, VEC, true> dy[CHUNKS], dh[CHUNKS], h[PACKED ? 1 : CHUNKS];
    RawCodes8<VEC, true> codes[PACKED ? CHUNKS : 1];
  } next;
  auto load = [&](int64_t at, auto& to) {
    const int end = at < a.rows ? a.cols : 0;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      to.dy[i].template load<THREADS>(static_cast<const T*>(a.dy) + at * a.ldy, lane, i, end);
      if constexpr (PACKED) to.codes[i].template load<THREADS>(a.codes + at * a.ldq, lane, i, end);
      else to.h[i].template load<THREADS>(static_cast<const T*>(a.h) + at * a.ldh, lane, i, end);
      if (a.dh != nullptr) to.dh[i].template load<THREADS>(static_cast<const T*>(a.dh) + at * a.lddh, lane, i, end);
    }
  };
  float rstd_next, factor_next;
  scalars(row, rstd_next, factor_next);
  ahead(0, row);
  if constexpr (kNext) load(row, next);
  for (int64_t turn = 0; turn < turns; ++turn, row += step) {
    const int sums_at = (int)(turn & 1), set = G::kSets == 2 ? sums_at : 0, end = row < a.rows ? a.cols : 0;
    const float rstd = rstd_next, factor = __fmul_rn(factor_next, rstd);
    Raw8<DTYPE, VEC, true> dy[CHUNKS], dh[CHUNKS], h[PACKED ? 1 : CHUNKS];
    RawCodes8<VEC, true> codes[PACKED ? CHUNKS : 1];
    if constexpr (G::kSets == 2) ahead(set ^ 1, row + step);
    scalars(row + step, rstd_next, factor_next);
    if constexpr (G::kAhead) {
      asm volatile("cp.async.wait_group %0;" ::"n"(G::kSets - 1) : "memory");
    } else if constexpr (!kAgain) {
      if constexpr (!kNext) load(row, next);
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        dy[i] = next.dy[i];
        dh[i] = next.dh[i];
        if constexpr (PACKED) codes[i] = next.codes[i];
        else h[i] = next.h[i];
      }
      if constexpr (kNext) load(row + step, next);
    }
    auto fetched = [&](int o, int i, const Raw8<DTYPE, VEC, true>& direct, float (&v)[8]) {
      if constexpr (kAgain) {
        const T* from = static_cast<const T*>(o == 0 ? a.dy : o == 1 ? a.h : a.dh) + row * (o == 0 ? a.ldy : o == 1 ? a.ldh : a.lddh);
        Raw8<DTYPE, VEC, true> x;
        x.template load<THREADS>(from, lane, i, end);
        x.widen(v);
      } else if constexpr (G::kAhead) {
        const uint4* p = reinterpret_cast<const uint4*>(place(set, o, i));
        Raw8<DTYPE, VEC> x;
        x.set(0, p[0]);
        if constexpr (DTYPE == NSML_F32) x.set(4, p[1]);
        x.widen(v);
      }
      else direct.widen(v);
    };
    auto kept = [&](int i, float (&v)[8]) {
      if constexpr (!PACKED) {
        fetched(1, i, h[i], v);
      } else {
        if constexpr (G::kAhead) {
          const uint2 x = *reinterpret_cast<const uint2*>(place(set, 1, i));
          codes[i].w[0] = x.x;
          codes[i].w[1] = x.y;
        } else if constexpr (kAgain) {
          codes[i].template load<THREADS>(a.codes + row * a.ldq, lane, i, end);
        }
        codes[i].numbers(v);
      }
    };
    float dot = 0.0f;
    if (row < a.rows)
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      if (empty<VEC, THREADS>(i, a.cols)) break;
      float v[8], d[8], w[8];
      weights(i, w);
      kept(i, v);
      fetched(0, i, dy[i], d);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float p = __fmul_rn(d[j], v[j]);
        dw[i][j] = __fmaf_rn(p, factor, dw[i][j]);
        dot = __fmaf_rn(p, w[j], dot);
      }
    }
#pragma unroll
    for (int d = (THREADS < 32 ? THREADS : 32) / 2; d; d >>= 1) dot = __fadd_rn(dot, __shfl_xor_sync(0xFFFFFFFFu, dot, d));
    if constexpr (THREADS > 32) {  // (two sets, so that one step of the row's warps per turn is enough)
      float* const sums = shared[sums_at][team];
      if ((threadIdx.x & 31) == 0) sums[lane >> 5] = dot;
      if constexpr (kTeams > 1) asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(THREADS) : "memory");
      else __syncthreads();
      dot = sums[0];
#pragma unroll
      for (int k = 1; k < kWarps; ++k) dot = __fadd_rn(dot, sums[k]);
    }
    if constexpr (!G::kAhead && !kAgain) {
#pragma unroll
      for (int i = 0; i < CHUNKS; ++i) {
        forget(dy[i]);
        if constexpr (PACKED) forget(codes[i]);
        else forget(h[i]);
      }
    }
    const float slope = -__fmul_rn(__fmul_rn(__fmul_rn(dot, factor), inv_cols), factor);  // -c, per unit of what h holds
    if (row < a.rows)
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      if (empty<VEC, THREADS>(i, a.cols)) break;
      float v[8], g[8], d[8], w[8];
      weights(i, w);
      kept(i, v);
      fetched(0, i, dy[i], g);
      if (a.dh != nullptr) fetched(2, i, dh[i], d);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float u = __fmaf_rn(v[j], slope, __fmul_rn(g[j], w[j]));
        g[j] = a.dh != nullptr ? __fmaf_rn(u, rstd, d[j]) : __fmul_rn(u, rstd);
      }
      store8<DTYPE, VEC, THREADS>(static_cast<T*>(a.dx) + row * a.lddx, lane, i, end, g);
      if constexpr (G::kSets == 1) chunk_ahead(0, row + step, i);  // (behind the store, which has used all that was read there)
    }
    if constexpr (G::kSets == 1) asm volatile("cp.async.commit_group;" ::: "memory");
  }
  if (a.partial == nullptr) return;
  float* const to = a.partial + (int64_t)blockIdx.x * a.cols;
  if constexpr (kTeams > 1) {
    float* const parts = reinterpret_cast<float*>(stage);
    __syncthreads();  // (nobody waits for or reads copies any more: the last ones are of rows behind the end, or done)
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) parts[team * (THREADS * CHUNKS * 8) + column<VEC, THREADS>(lane, i, j)] = dw[i][j];
    __syncthreads();
    for (int c = threadIdx.x; c < a.cols; c += kGradBlock) {
      float s = parts[c];
#pragma unroll
      for (int k = 1; k < kTeams; ++k) s = __fadd_rn(s, parts[k * (THREADS * CHUNKS * 8) + c]);
      to[c] = s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) store8<NSML_F32, VEC, THREADS>(to, lane, i, a.cols, dw[i]);
  }
}

// dweight (+)= sum of the blocks' parts, in their order.  A block has 32 columns, its warps every 32nd part: dependent reads
// bound it, 4-5 us behind the kernel above for 296 parts.
__global__ void __launch_bounds__(1024) k_q8_norm_weight(const float* __restrict__ partial, int parts, int64_t cols, void* dweight,
                                                        bool bf16, bool zero_first, int* status) {
  __shared__ float sums[32][33];
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = NSML_OK;
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

// The gradient of the norm: chunks per thread, threads per row (the fewest that hold it: aligned bfloat16 16384 x 768 with dh
// 18.5 us, with twice as many 27.2; 32768 x 255 17.8 and 29.4), and blocks: what a B200's 148 SMs hold; also the height of
// the workspace's table.
constexpr int kGradMostBlocks = 2 * 148;
constexpr size_t kGradTableAt = 256;  // (the status word comes first)
static constexpr int grad_chunks(int dtype, bool vec) { return vec ? (dtype == NSML_F32 ? 2 : 4) : 1; }
static int grad_threads(int64_t cols, int dtype, bool vec) {
  const int64_t each = 8 * grad_chunks(dtype, vec);
  int threads = 128 / (int)each;  // narrowest: 128 columns
  while (threads < 1024 && cols > each * threads) threads *= (threads < 16 ? 4 : 2);
  return threads;
}
static int grad_blocks(int64_t rows, int64_t cols, int dtype, bool vec) {
  const int threads = grad_threads(cols, dtype, vec), teams = threads < kGradBlock ? kGradBlock / threads : 1;
  const int64_t most = threads <= kGradBlock ? kGradMostBlocks : kGradMostBlocks / 2, need = (rows + teams - 1) / teams;
  return (int)(need < most ? need : most);
}

template <int DTYPE, bool PACKED, bool VEC, bool KEEP>
static int norm_grad_rows(const NormGradArgs& a, cudaStream_t st) {
  auto go = [&](auto threads, auto chunks) {
    constexpr int THREADS = threads, CHUNKS = chunks;
    constexpr size_t smem = GradStage<DTYPE, VEC, THREADS, CHUNKS>::kSmem;
    cudaError_t e = cudaSuccess;
    if constexpr (smem > 40 * 1024) {  // more than 48 KB have to be allowed, once per kernel and device
      static std::atomic<unsigned long long> allowed{0};
      int dev = 0;
      if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cuda_error();
      if ((allowed.load(std::memory_order_relaxed) >> dev & 1) == 0) {
        e = cudaFuncSetAttribute(k_q8_norm_grad<DTYPE, PACKED, VEC, KEEP, THREADS, CHUNKS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return cuda_error();
        allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
      }
    }
    LaunchScope scope(K_Q8_NORM_GRAD, st);
    e = launch_in_stream(k_q8_norm_grad<DTYPE, PACKED, VEC, KEEP, THREADS, CHUNKS>, dim3(grad_blocks(a.rows, a.cols, DTYPE, VEC)), dim3(grad_block<THREADS>()), smem, st,
                         0, a);
    return e == cudaSuccess ? NSML_OK : cuda_error();
  };
  using std::integral_constant;
  constexpr int C = grad_chunks(DTYPE, VEC), kLeast = 128 / (8 * C);  // 4, 8 or 16
  const int threads = grad_threads(a.cols, DTYPE, VEC);
  if (threads == 1024 && a.cols > 8192 * C) {
    if constexpr (C == 1)  // (four chunks do not fit into the registers)
      if (a.cols <= 16384) return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    return go(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
  }
  if (threads == kLeast) return go(integral_constant<int, kLeast>{}, integral_constant<int, C>{});
  switch (threads) {
    case 16: if constexpr (kLeast == 4) return go(integral_constant<int, 16>{}, integral_constant<int, C>{});
    case 32: return go(integral_constant<int, 32>{}, integral_constant<int, C>{});
    case 64: return go(integral_constant<int, 64>{}, integral_constant<int, C>{});
    case 128: return go(integral_constant<int, 128>{}, integral_constant<int, C>{});
    case 256: return go(integral_constant<int, 256>{}, integral_constant<int, C>{});
    case 512: return go(integral_constant<int, 512>{}, integral_constant<int, C>{});
    default: return go(integral_constant<int, 1024>{}, integral_constant<int, C>{});
  }
}

}  // namespace q8
}  // namespace nsml

using namespace nsml;
using namespace nsml::q8;

extern "C" {

size_t nsml_q8_rms_norm_backward_workspace_bytes(int64_t cols) {
  if (cols < 1 || cols > NSML_Q8_MAX_NORM_COLS) return 0;
  return kGradTableAt + align_up((size_t)kGradMostBlocks * (size_t)cols * 4, 256);  // (the same for every width, so that it never shrinks)
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
  float* const table = dweight != nullptr ? reinterpret_cast<float*>(static_cast<char*>(workspace) + kGradTableAt) : nullptr;
  const bool vec = cols % 8 == 0 && rows16(dy, ldy, dtype) && rows16(dx, lddx, dtype) && aligned(weight, 16) &&
                   (dh == nullptr || rows16(dh, lddh, dtype)) && (h == nullptr || rows16(h, ldh, dtype));
  if (rows > 0) {
    NormGradArgs a = {};
    a.dy = dy; a.dh = dh; a.h = h; a.codes = codes; a.scales = scales; a.rstd = rstd; a.weight = weight; a.dx = dx;
    a.partial = table;
    a.rows = rows; a.cols = (int)cols; a.ldy = ldy; a.lddh = lddh; a.ldh = ldh; a.ldq = ldq; a.lddx = lddx;
    a.weight_bf16 = weight_dtype == NSML_BF16;
    const bool packed = codes != nullptr;
    const bool keep = weight_dtype == dtype;
    auto by_flags = [&](auto type) {
      constexpr int DTYPE = type;
      using yes = std::true_type;
      using no = std::false_type;
      auto run = [&](auto p, auto v, auto k) { return norm_grad_rows<DTYPE, p, v, k>(a, st); };
      auto with_keep = [&](auto p, auto v) { return keep ? run(p, v, yes{}) : run(p, v, no{}); };
      auto with_vec = [&](auto p) { return vec ? with_keep(p, yes{}) : with_keep(p, no{}); };
      return packed ? with_vec(yes{}) : with_vec(no{});
    };
    const int rc = dtype == NSML_F32 ? by_flags(std::integral_constant<int, NSML_F32>{}) : by_flags(std::integral_constant<int, NSML_BF16>{});
    if (rc != NSML_OK) return rc;
  }
  if (dweight != nullptr) {
    LaunchScope scope(K_Q8_NORM_WEIGHT, st);
    const cudaError_t e = launch_in_stream(k_q8_norm_weight, dim3((unsigned int)((cols + 31) / 32)), dim3(1024), 0, st, 0,
                                           static_cast<const float*>(table), grad_blocks(rows, cols, dtype, vec), cols, dweight,
                                           dweight_dtype == NSML_BF16, zero_first != 0, static_cast<int*>(workspace));
    if (e != cudaSuccess) return cuda_error();
  }
  return NSML_OK;
}

}  // extern "C"
