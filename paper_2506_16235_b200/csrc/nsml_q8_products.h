// What the source files of the q8 products share.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace nsml {
namespace q8 {

// Products of so many tokens or fewer have a kernel of their own.  n = 8192, k = 2048 (from L2), one B200: 1 token 5.0 us (tensor cores
// 8.7), 4 6.9 (9.4), 8 10.0 (9.4), 16 34 (9.4).
constexpr int kMaxTokens = 4;

int launch_tokens(const int8_t* a, int64_t lda, const float* sa, const int8_t* b, int64_t ldb, const float* sb, int m, int64_t n, int k, void* out,
                  int64_t ldo, bool bf16, int* status, cudaStream_t st);

}  // namespace q8
}  // namespace nsml
