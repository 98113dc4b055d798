// Product of a few tokens with 8-bit weights: out[m, n] = (sum_k a[m,k] b[n,k]) sa[m] sb[n], m <= kMaxTokens.  The weights have to be read
// once and nothing else counts, so no tensor cores: a warp takes kRows rows of the weights (so that the tokens' codes are
// read once per kRows of them), its lanes 16 codes each, and multiplies with four-way integer products.  One token, n = 8192,
// k = 2048 (17 MB): 5.0 us where L2 holds the weights, 7.5 from cold caches; n = k = 16384 (268 MB) 44 us, 6.1 TB/s.
#include <type_traits>

#include "nsml_launch.h"
#include "nsml_q8.cuh"
#include "nsml_q8_products.h"

namespace nsml {
namespace q8 {

constexpr int kRows = 4, kTokenWarps = 8;

// 16 codes at c; those from `end` on are 0
__device__ __forceinline__ uint4 load16(const int8_t* row, int c, int end) {
  if (c >= end) return make_uint4(0, 0, 0, 0);
  uint4 w = *reinterpret_cast<const uint4*>(row + c);  // (rows are a multiple of 16 bytes apart)
  if (end - c < 16) {
    uint32_t* p = &w.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int left = end - c - 4 * i;
      p[i] = left >= 4 ? p[i] : left <= 0 ? 0u : p[i] & (0xFFFFFFFFu >> (8 * (4 - left)));
    }
  }
  return w;
}

// M: tokens (those past m repeat the last one, and are not stored).  SPLIT: warps that share a row's sum.
template <int M, int SPLIT>
__global__ void __launch_bounds__(32 * kTokenWarps)
k_q8_tokens(const int8_t* __restrict__ a, int64_t lda, const float* __restrict__ sa, const int8_t* __restrict__ b, int64_t ldb,
            const float* __restrict__ sb, int m, int64_t n, int k, void* out, int64_t ldo, bool bf16, int* status) {
  __shared__ int shared[SPLIT > 1 ? kTokenWarps * kRows * M : 1];
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0) *status = NSML_OK;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % SPLIT;
  const int64_t row0 = ((int64_t)blockIdx.x * (kTokenWarps / SPLIT) + warp / SPLIT) * kRows;
  const int8_t* rows[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) rows[r] = b + min(row0 + r, n - 1) * ldb;
  int sum[kRows][M] = {};
#pragma unroll 2
  for (int c = 16 * (lane + 32 * part); c < k; c += 512 * SPLIT) {
    uint4 w[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) w[r] = __ldcs(reinterpret_cast<const uint4*>(rows[r] + c));  // (past k: times 0)
#pragma unroll
    for (int t = 0; t < M; ++t) {
      const uint4 x = load16(a + (int64_t)min(t, m - 1) * lda, c, k);
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        sum[r][t] = __dp4a((int)w[r].x, (int)x.x, sum[r][t]);
        sum[r][t] = __dp4a((int)w[r].y, (int)x.y, sum[r][t]);
        sum[r][t] = __dp4a((int)w[r].z, (int)x.z, sum[r][t]);
        sum[r][t] = __dp4a((int)w[r].w, (int)x.w, sum[r][t]);
      }
    }
  }
  int mine = 0;  // lane i keeps the sum of row i % kRows and token i / kRows
  static_assert(kRows * M <= 32, "");
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int t = 0; t < M; ++t) {
      const int s = __reduce_add_sync(0xFFFFFFFFu, sum[r][t]);
      if (lane == t * kRows + r) mine = s;
    }
  if constexpr (SPLIT > 1) {
    if (lane < kRows * M) shared[warp * (kRows * M) + lane] = mine;
    __syncthreads();
    if (part != 0) return;
#pragma unroll
    for (int p = 1; p < SPLIT; ++p)
      if (lane < kRows * M) mine += shared[(warp + p) * (kRows * M) + lane];
  }
  const int t = lane / kRows;
  const int64_t row = row0 + lane % kRows;
  if (t >= m || t >= M || row >= n) return;
  const float v = __fmul_rn(__fmul_rn((float)mine, sa[t]), sb[row]);
  if (bf16) static_cast<__nv_bfloat16*>(out)[t * ldo + row] = __float2bfloat16_rn(v);
  else static_cast<float*>(out)[t * ldo + row] = v;
}

int launch_tokens(const int8_t* a, int64_t lda, const float* sa, const int8_t* b, int64_t ldb, const float* sb, int m, int64_t n, int k, void* out,
                  int64_t ldo, bool bf16, int* status, cudaStream_t st) {
  using std::integral_constant;
  auto go = [&](auto tokens, auto split) {
    constexpr int M = tokens, SPLIT = split, per_block = kRows * kTokenWarps / SPLIT;
    LaunchScope scope(K_Q8_TOKENS, st);
    const cudaError_t e = launch_in_stream(k_q8_tokens<M, SPLIT>, dim3((unsigned int)((n + per_block - 1) / per_block)), dim3(32 * kTokenWarps), 0, st, 0,
                                           a, lda, sa, b, ldb, sb, m, n, k, out, ldo, bf16, status);
    return e == cudaSuccess ? NSML_OK : cuda_error();
  };
  // enough warps to have the memory busy (some 2000), but not so many that a lane has nothing to read (512 codes per warp)
  const int64_t groups = (n + kRows - 1) / kRows;
  const int split = groups >= 2048 || k <= 512 ? 1 : groups >= 512 || k <= 2048 ? 4 : 8;
  auto with_tokens = [&](auto s) {
    if (m == 1) return go(integral_constant<int, 1>{}, s);
    if (m == 2) return go(integral_constant<int, 2>{}, s);
    static_assert(kMaxTokens == 4, "");
    return go(integral_constant<int, 4>{}, s);
  };
  if (split == 1) return with_tokens(integral_constant<int, 1>{});
  if (split == 4) return with_tokens(integral_constant<int, 4>{});
  return with_tokens(integral_constant<int, 8>{});
}

}  // namespace q8
}  // namespace nsml
