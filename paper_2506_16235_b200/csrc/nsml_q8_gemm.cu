// Matrix products of the q8 format on the tensor cores (tcgen05, accumulators in TMEM, operands by TMA).
//
//   kForward      out[m,n] = (sum_k a[m,k] b[n,k]) sa[m] sb[n]     int8 operands, 32-bit integer sums (exact)
//   kGradInput    dx[m,k]  = sum_n dy[m,n] (b[n,k] sb[n])          bfloat16 operands, float32 sums
//   kGradWeight   dw[n,k]  = sum_m dy[m,n] (a[m,k] sa[m])          the same, dy read across its rows
//
// In the gradients the codes' scale belongs to the axis of the sum, so it cannot wait for the epilogue: eight warps restore
// the codes to bfloat16 on their way from one shared-memory ring to another (exact for the scales that nsml_q8_pack makes).
// The restored matrix never exists in memory.
#include <cuda.h>

#include <mutex>

#include "nsml_launch.h"
#include "nsml_q8.cuh"

namespace nsml {
namespace q8 {

enum { kForward = 0, kGradInput = 1, kGradWeight = 2 };

constexpr int kTileM = 128;
constexpr unsigned long long kWaitNs = 2000000000ull;  // a wait gives up after two seconds

// ---- PTX ---------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xFFFFFFFF;\n selp.b32 %0, 1, 0, p;\n}" : "=r"(one));
  return one != 0;
}

__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
// false: the wait ran out (here or, as `failed` says, elsewhere in the block)
__device__ __noinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, volatile int* failed) {
  const unsigned long long from = now_ns();
  while (true) {
    for (int i = 0; i < 64; ++i)
      if (bar_try(bar, parity)) return true;
    if (*failed != 0 || now_ns() - from > kWaitNs) {
      *failed = 1;
      return false;
    }
  }
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* failed) {
  if (bar_try(bar, parity)) return true;
  return bar_wait_slow(bar, parity, failed);
}

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

template <int COLS>
__device__ __forceinline__ void tmem_alloc(uint32_t slot) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "n"(COLS) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
template <int COLS>
__device__ __forceinline__ void tmem_free(uint32_t addr) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(COLS));
}
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// the barrier is arrived at once all tensor work issued so far by this thread is done
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <int MODE>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
  if constexpr (MODE == kForward)
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
  else
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory");
}
// 32 columns of this warp's 32 lanes
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
      "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// ---- operand tiles -----------------------------------------------------------------------------------------------------
// Shared-memory descriptors of tiles with 128-byte swizzle.
//   sum axis along the 128 bytes of a row (kForward, the rows of dy in kGradInput): groups of 8 rows are 1024 bytes apart;
//     the next step along the sum is 32 bytes further
//   other axis along the 128 bytes: blocks of 64 columns x 64 rows of the sum, 8192 bytes each (leading offset), in
//     groups of 8 rows 1024 bytes apart; the next step along the sum (16 rows) is 2048 bytes further
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, uint32_t leading, uint32_t stride) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(leading >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
template <int MODE, int BN>
__host__ __device__ constexpr uint32_t mma_desc() {
  return (MODE == kForward ? (2u << 4 | 1u << 7 | 1u << 10)                                          // s32 += s8 * s8
                           : (1u << 4 | 1u << 7 | 1u << 10 | (MODE == kGradWeight ? 1u << 15 : 0u) | 1u << 16))  // f32 += bf16 * bf16
         | (uint32_t)(BN / 8) << 17 | (uint32_t)(kTileM / 16) << 24;
}

struct GemmArgs {
  int64_t rows, cols;         // of the result
  int steps;                  // blocks of the sum: 128 codes (kForward) or 64 products
  int64_t depth;              // length of the sum
  void* out;
  int64_t ldo;
  bool bf16, add, pair;       // pair: rows of the result start on even elements (two of them per store)
  const float* row_scale;     // kForward
  const float* col_scale;     // kForward
  const float* depth_scale;   // gradients
  int* status;
  int64_t tiles_m, tiles_n;
};

template <int MODE, int BN>
struct Shape {
  static constexpr int kA = kTileM * 128;                              // bytes of a stage: the first operand,
  static constexpr int kB = MODE == kForward ? BN * 128 : BN * 64;     // codes of the second
  static constexpr int kStage = kA + kB;
  static constexpr int kStages = 4;
  static constexpr int kWide = MODE == kForward ? 0 : BN * 128;        // a restored tile of the second operand
  static constexpr int kWides = 2;
  static constexpr int kThreads = MODE == kForward ? 256 : 512;
  static constexpr int kStaging = 4 * 32 * 33 * 4;                     // a warp's 32 x 32 results on their way out
  static constexpr int kRings = kStages * kStage + kWides * kWide;
  static constexpr size_t kSmem = 1024 + kRings + kStaging;
};

// The order of the tiles: columns of 16 tiles high, so that the tiles in flight share their operands in L2.
__device__ __forceinline__ void tile_at(int64_t t, int64_t tiles_m, int64_t tiles_n, int64_t& m, int64_t& n) {
  constexpr int64_t kGroup = 16;
  const int64_t per = kGroup * tiles_n, g = t / per, first = g * kGroup, high = min(kGroup, tiles_m - first), in = t - g * per;
  m = first + in % high;
  n = in / high;
}

// Codes to bfloat16, times a scale.  The low seven bits of a code go into 128.0 (whose unit is 1), the sign bit into a second
// 128.0 (which it makes 256.0): the difference is the code.  A scale that is a bfloat16 (every power of two from 2^-126 on,
// 0, NaN) is multiplied in bfloat16, rounded once; any other in float32, rounded again.
__device__ __forceinline__ uint32_t restore2(uint32_t pair, __nv_bfloat162 scale) {
  const uint32_t x = (pair & 0x007F007Fu) | 0x43004300u, y = (pair & 0x00800080u) | 0x43004300u;
  const __nv_bfloat162 d = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&y)), scale);
  return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ uint4 restore8(uint32_t w0, uint32_t w1, float scale) {
  const uint32_t b = __float_as_uint(scale);
  if ((b & 0xFFFFu) == 0) {
    const uint32_t twice = __byte_perm(b, 0, 0x3232);
    const __nv_bfloat162 s = *reinterpret_cast<const __nv_bfloat162*>(&twice);
    return make_uint4(restore2(__byte_perm(w0, 0, 0x4140), s), restore2(__byte_perm(w0, 0, 0x4342), s),
                      restore2(__byte_perm(w1, 0, 0x4140), s), restore2(__byte_perm(w1, 0, 0x4342), s));
  }
  auto two = [&](uint32_t w) { return pack2(restore((int8_t)w, scale), restore((int8_t)(w >> 8), scale)); };
  return make_uint4(two(w0), two(w0 >> 16), two(w1), two(w1 >> 16));
}

template <int MODE, int BN, bool SPLIT>
__global__ void __launch_bounds__(Shape<MODE, BN>::kThreads, 1)
k_q8_gemm(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const GemmArgs g) {
  using S = Shape<MODE, BN>;
  constexpr int kTmem = SPLIT ? BN : 2 * BN;
  extern __shared__ unsigned char raw[];
  __shared__ alignas(8) uint64_t bars[2 * S::kStages + 2 * S::kWides + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ int failed;
  const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
  const uint32_t wide = ring + S::kStages * S::kStage;
  unsigned char* const ring_ptr = raw + (ring - smem_addr(raw));
  const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, wide_full = empty + 8 * S::kStages,
                 wide_empty = wide_full + 8 * S::kWides, acc_full = wide_empty + 8 * S::kWides, acc_empty = acc_full + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t splits = 1, part = 0;
  if constexpr (SPLIT) {
    asm("mov.u32 %0, %cluster_nctarank;" : "=r"(splits));
    asm("mov.u32 %0, %cluster_ctarank;" : "=r"(part));
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      bar_init(full + 8 * i, 1);
      bar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < S::kWides; ++i) {
      bar_init(wide_full + 8 * i, 256);
      bar_init(wide_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(acc_full + 8 * i, 1);
      bar_init(acc_empty + 8 * i, 128);
    }
    failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) tmem_alloc<kTmem>(smem_addr(&tmem_slot));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0) *g.status = NSML_OK;

  const int64_t tiles = g.tiles_m * g.tiles_n, first = blockIdx.x / splits, stride = gridDim.x / splits;
  const int from = (int)((int64_t)g.steps * part / splits), to = (int)((int64_t)g.steps * (part + 1) / splits);

  if (warp == 0) {
    if (elect_one()) {  // ---- loads
      uint32_t it = 0;
      bool ok = true;
      for (int64_t t = first; ok && t < tiles; t += stride) {
        int64_t m, n;
        tile_at(t, g.tiles_m, g.tiles_n, m, n);
        for (int k = from; k < to; ++k, ++it) {
          const uint32_t s = it % S::kStages, bar = full + 8 * s, at = ring + s * S::kStage;
          if (!(ok = bar_wait(empty + 8 * s, (it / S::kStages + 1) & 1, &failed))) break;
          bar_expect(bar, S::kStage);
          if constexpr (MODE == kForward) {
            tma_load(at, &map_a, k * 128, (int)(m * kTileM), bar);
            tma_load(at + S::kA, &map_b, k * 128, (int)(n * BN), bar);
          } else {
            if constexpr (MODE == kGradInput) {
              tma_load(at, &map_a, k * 64, (int)(m * kTileM), bar);
            } else {
              tma_load(at, &map_a, (int)(m * kTileM), k * 64, bar);
              tma_load(at + S::kA / 2, &map_a, (int)(m * kTileM) + 64, k * 64, bar);
            }
            tma_load(at + S::kA, &map_b, (int)(n * BN), k * 64, bar);
          }
        }
      }
      // copies in flight land before the block's shared memory goes (after a failure too: each wait is bounded)
      if (!ok) {
        for (uint32_t back = 0; back < S::kStages && back < it; ++back) {
          const uint32_t i = it - 1 - back;
          const unsigned long long began = now_ns();
          while (!bar_try(full + 8 * (i % S::kStages), (i / S::kStages) & 1) && now_ns() - began < kWaitNs) {}
        }
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (elect_one()) {  // ---- products
      uint32_t it = 0, count = 0;
      bool ok = true;
      for (int64_t t = first; ok && t < tiles; t += stride, ++count) {
        const uint32_t buffer = SPLIT ? 0 : count & 1, acc = tmem + buffer * BN;
        if (!(ok = bar_wait(acc_empty + 8 * buffer, ((count >> 1) + 1) & 1, &failed))) break;
        tc_fence_after();
        for (int k = from; k < to; ++k, ++it) {
          const uint32_t s = it % S::kStages, at = ring + s * S::kStage, w = it % S::kWides;
          if (!(ok = bar_wait(full + 8 * s, (it / S::kStages) & 1, &failed))) break;
          if constexpr (MODE != kForward)
            if (!(ok = bar_wait(wide_full + 8 * w, (it / S::kWides) & 1, &failed))) break;
          tc_fence_after();
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint64_t a = MODE == kGradWeight ? tile_desc(at + j * 2048, 8192, 1024) : tile_desc(at + j * 32, 16, 1024);
            const uint64_t b = MODE == kForward ? tile_desc(at + S::kA + j * 32, 16, 1024) : tile_desc(wide + w * S::kWide + j * 2048, 8192, 1024);
            tc_mma<MODE>(acc, a, b, mma_desc<MODE, BN>(), k > from || j > 0);
          }
          tc_commit(empty + 8 * s);
          if constexpr (MODE != kForward) tc_commit(wide_empty + 8 * w);
        }
        if (ok) tc_commit(acc_full + 8 * buffer);
      }
    }
    __syncwarp();
  } else if (warp >= 4 && warp < 8) {  // ---- results
    const int quarter = warp - 4;
    uint32_t* const stage = reinterpret_cast<uint32_t*>(ring_ptr + S::kRings) + quarter * 32 * 33;
    uint32_t count = 0;
    for (int64_t t = first; t < tiles; t += stride, ++count) {
      const uint32_t buffer = SPLIT ? 0 : count & 1;
      if (!bar_wait(acc_full + 8 * buffer, (count >> 1) & 1, &failed)) break;
      tc_fence_after();
      int64_t m, n;
      tile_at(t, g.tiles_m, g.tiles_n, m, n);
      const int64_t row0 = m * kTileM + quarter * 32;
      const float my_scale = MODE == kForward && row0 + lane < g.rows ? g.row_scale[row0 + lane] : 0.0f;
#pragma unroll 1
      for (int c = 0; c < BN / 32; ++c) {
        uint32_t r[32];
        tmem_load32(tmem + buffer * BN + c * 32 + ((uint32_t)quarter << 21), r);
        if (c == BN / 32 - 1) {
          tc_fence_before();
          bar_arrive(acc_empty + 8 * buffer);
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) stage[lane * 33 + j] = r[j];
        __syncwarp();
        // half a warp per row, two columns per lane
        const int64_t col = n * BN + c * 32 + 2 * (lane & 15);
        float cs[2] = {0.0f, 0.0f};
        if constexpr (MODE == kForward) {
          if (col < g.cols) cs[0] = g.col_scale[col];
          if (col + 1 < g.cols) cs[1] = g.col_scale[col + 1];
        }
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
          const int rr = 2 * i + (lane >> 4);
          const int64_t row = row0 + rr;
          const uint32_t* from_stage = stage + rr * 33 + 2 * (lane & 15);
          float v[2];
          if constexpr (MODE == kForward) {
            const float rs = __shfl_sync(0xFFFFFFFFu, my_scale, rr);
            v[0] = __fmul_rn(__fmul_rn((float)(int)from_stage[0], rs), cs[0]);
            v[1] = __fmul_rn(__fmul_rn((float)(int)from_stage[1], rs), cs[1]);
          } else {
            v[0] = __uint_as_float(from_stage[0]);
            v[1] = __uint_as_float(from_stage[1]);
          }
          if (row >= g.rows || col >= g.cols) continue;
          if (g.bf16) {
            __nv_bfloat16* to_row = static_cast<__nv_bfloat16*>(g.out) + row * g.ldo + col;
            if (g.pair && col + 1 < g.cols) {
              if (g.add) {
                float a, b;
                unpack2(*reinterpret_cast<const uint32_t*>(to_row), a, b);
                v[0] = __fadd_rn(v[0], a);
                v[1] = __fadd_rn(v[1], b);
              }
              *reinterpret_cast<uint32_t*>(to_row) = pack2(v[0], v[1]);
            } else {
              for (int e = 0; e < 2 && col + e < g.cols; ++e)
                to_row[e] = __float2bfloat16_rn(g.add ? __fadd_rn(v[e], (float)to_row[e]) : v[e]);
            }
          } else {
            float* to_row = static_cast<float*>(g.out) + row * g.ldo + col;
            for (int e = 0; e < 2 && col + e < g.cols; ++e) to_row[e] = g.add ? __fadd_rn(v[e], to_row[e]) : v[e];
          }
        }
        __syncwarp();
      }
    }
  } else if (MODE != kForward && warp >= 8) {  // ---- codes to bfloat16
    if constexpr (MODE != kForward) {
      constexpr int kLanes = BN / 16, kRowsAtOnce = 32 / kLanes, kRounds = 8 / kRowsAtOnce;  // a warp: 8 rows of a tile
      const int sub = lane % kLanes, row = (warp - 8) * 8 + lane / kLanes;
      const int flip = (sub >> 2) & 1;  // lanes whose blocks of columns share banks write their halves in opposite order
      uint32_t it = 0;
      bool ok = true;
      for (int64_t t = first; ok && t < tiles; t += stride) {
        float scale[kRounds];
        auto fetch = [&](int k) {
#pragma unroll
          for (int i = 0; i < kRounds; ++i) {
            const int64_t at = (int64_t)k * 64 + row + i * kRowsAtOnce;
            scale[i] = k < to && at < g.depth ? g.depth_scale[at] : 0.0f;
          }
        };
        fetch(from);
        for (int k = from; k < to; ++k, ++it) {
          const uint32_t s = it % S::kStages, w = it % S::kWides;
          if (!(ok = bar_wait(wide_empty + 8 * w, (it / S::kWides + 1) & 1, &failed))) break;
          if (!(ok = bar_wait(full + 8 * s, (it / S::kStages) & 1, &failed))) break;
          const unsigned char* codes = ring_ptr + s * S::kStage + S::kA;
          unsigned char* dst = ring_ptr + S::kStages * S::kStage + w * S::kWide + (sub >> 2) * 8192;
#pragma unroll
          for (int i = 0; i < kRounds; ++i) {
            const int rr = row + i * kRowsAtOnce;
            const uint4 q = *reinterpret_cast<const uint4*>(codes + rr * BN + sub * 16);
            const uint4 o[2] = {restore8(q.x, q.y, scale[i]), restore8(q.z, q.w, scale[i])};
            unsigned char* line = dst + rr * 128;
            const int c0 = (sub & 3) * 2;
            *reinterpret_cast<uint4*>(line + (((c0 + flip) ^ (rr & 7)) << 4)) = flip ? o[1] : o[0];
            *reinterpret_cast<uint4*>(line + (((c0 + 1 - flip) ^ (rr & 7)) << 4)) = flip ? o[0] : o[1];
          }
          fence_async_shared();
          bar_arrive(wide_full + 8 * w);
          fetch(k + 1);
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 2) tmem_free<kTmem>(tmem);
  if (threadIdx.x == 0 && failed != 0) set_status(g.status, NSML_ERR_TIMEOUT);
}

// ---- host ----------------------------------------------------------------------------------------------------------------
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled encoder() {  // found in the driver, so that the library needs no link to it
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      p = nullptr;
    }
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

// rows x cols elements; boxes of box_cols x box_rows.  What lies outside reads as 0.
static bool tensor_map(CUtensorMap* map, const void* p, bool codes, int64_t rows, int64_t cols, int64_t ld, int box_cols, int box_rows, bool swizzle) {
  const int size = codes ? 1 : 2;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? ld : (cols * size + 15) / 16 * 16 / size) * size};  // (one row: any stride will do)
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return encoder()(map, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, step,
                   CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct GemmDevice {
  bool ready = false;
  int sms = 0;
};
static GemmDevice g_gemm_dev[64];
static std::mutex g_gemm_mutex;

template <int MODE, int BN, bool SPLIT>
static cudaError_t prepare_kernel() {
  return cudaFuncSetAttribute(k_q8_gemm<MODE, BN, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<MODE, BN>::kSmem);
}

static int gemm_device(int* sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cuda_error();
  std::lock_guard<std::mutex> lock(g_gemm_mutex);
  GemmDevice& d = g_gemm_dev[dev];
  if (!d.ready) {
    cudaError_t e = cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = prepare_kernel<kForward, 256, false>();
    if (e == cudaSuccess) e = prepare_kernel<kGradInput, 256, false>();
    if (e == cudaSuccess) e = prepare_kernel<kGradWeight, 256, false>();
    if (e != cudaSuccess || encoder() == nullptr) return cuda_error();
    d.ready = true;
  }
  *sms = d.sms;
  return NSML_OK;
}

template <int MODE, int BN, bool SPLIT>
static int launch_gemm(const CUtensorMap& map_a, const CUtensorMap& map_b, GemmArgs g, int sms, cudaStream_t st) {
  using S = Shape<MODE, BN>;
  g.tiles_m = (g.rows + kTileM - 1) / kTileM;
  g.tiles_n = (g.cols + BN - 1) / BN;
  const int64_t tiles = g.tiles_m * g.tiles_n;
  LaunchScope scope(K_Q8_GEMM, st);
  const cudaError_t e = launch_prio(k_q8_gemm<MODE, BN, SPLIT>, dim3((unsigned int)(tiles < sms ? tiles : sms)), dim3(S::kThreads), S::kSmem, st, false, 0,
                                    false, true, map_a, map_b, g);
  return e == cudaSuccess ? NSML_OK : cuda_error();
}

static bool valid_size(int64_t v) { return v >= 0 && v <= NSML_Q8_MAX_ROWS; }
static bool valid_codes(const void* p, int64_t rows, int64_t cols, int64_t ld) {
  return p != nullptr && aligned(p, 16) && (rows <= 1 || (ld >= cols && ld % 16 == 0 && ld < ((int64_t)1 << 40)));
}
static bool valid_gradient(const void* p, int64_t rows, int64_t cols, int64_t ld) {
  return p != nullptr && aligned(p, 16) && (rows <= 1 || (ld >= cols && ld % 8 == 0 && ld < ((int64_t)1 << 39)));
}
static int check_out(const void* out, int64_t rows, int64_t cols, int64_t ldo, int dtype, const void* workspace, size_t workspace_bytes) {
  if (dtype != NSML_F32 && dtype != NSML_BF16) return NSML_ERR_ARG;
  if (out == nullptr || !aligned(out, dtype == NSML_F32 ? 4 : 2) || (rows > 1 && ldo < cols)) return NSML_ERR_ARG;
  if (workspace == nullptr || !aligned(workspace, 256)) return NSML_ERR_ARG;
  return workspace_bytes < NSML_Q8_MATMUL_WORKSPACE_BYTES ? NSML_ERR_CAPACITY : NSML_OK;
}
static GemmArgs result(void* out, int64_t rows, int64_t cols, int64_t ldo, int dtype, bool add, void* workspace) {
  GemmArgs g = {};
  g.rows = rows;
  g.cols = cols;
  g.out = out;
  g.ldo = ldo;
  g.bf16 = dtype == NSML_BF16;
  g.add = add;
  g.pair = g.bf16 && aligned(out, 4) && (rows <= 1 || ldo % 2 == 0);
  g.status = static_cast<int*>(workspace);
  return g;
}

}  // namespace q8
}  // namespace nsml

using namespace nsml;
using namespace nsml::q8;

extern "C" {

int nsml_q8_matmul(const int8_t* a, int64_t lda, const float* a_scales, const int8_t* b, int64_t ldb, const float* b_scales, int64_t m,
                   int64_t n, int64_t k, void* out, int64_t ldo, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_size(m) || !valid_size(n) || n < 1 || k < 1 || k > NSML_Q8_MAX_DEPTH) return NSML_ERR_ARG;
  if (m == 0) return NSML_OK;
  if (!valid_codes(a, m, k, lda) || !valid_codes(b, n, k, ldb) || a_scales == nullptr || !aligned(a_scales, 4) || b_scales == nullptr || !aligned(b_scales, 4))
    return NSML_ERR_ARG;
  int rc = check_out(out, m, n, ldo, dtype, workspace, workspace_bytes);
  if (rc != NSML_OK) return rc;
  int sms = 0;
  if ((rc = gemm_device(&sms)) != NSML_OK) return rc;
  GemmArgs g = result(out, m, n, ldo, dtype, false, workspace);
  g.row_scale = a_scales;
  g.col_scale = b_scales;
  g.depth = k;
  g.steps = (int)((k + 127) / 128);
  CUtensorMap map_a, map_b;
  if (!tensor_map(&map_a, a, true, m, k, lda, 128, kTileM, true) || !tensor_map(&map_b, b, true, n, k, ldb, 128, 256, true)) return NSML_ERR_CUDA;
  return launch_gemm<kForward, 256, false>(map_a, map_b, g, sms, static_cast<cudaStream_t>(stream));
}

int nsml_q8_matmul_grad_input(const void* dy, int64_t ldy, const int8_t* b, int64_t ldb, const float* b_scales, int64_t m, int64_t n, int64_t k,
                              void* dx, int64_t lddx, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_size(m) || !valid_size(n) || !valid_size(k) || n < 1 || k < 1) return NSML_ERR_ARG;
  if (m == 0) return NSML_OK;
  if (!valid_gradient(dy, m, n, ldy) || !valid_codes(b, n, k, ldb) || b_scales == nullptr || !aligned(b_scales, 4)) return NSML_ERR_ARG;
  int rc = check_out(dx, m, k, lddx, dtype, workspace, workspace_bytes);
  if (rc != NSML_OK) return rc;
  int sms = 0;
  if ((rc = gemm_device(&sms)) != NSML_OK) return rc;
  GemmArgs g = result(dx, m, k, lddx, dtype, false, workspace);
  g.depth_scale = b_scales;
  g.depth = n;
  g.steps = (int)((n + 63) / 64);
  CUtensorMap map_a, map_b;
  if (!tensor_map(&map_a, dy, false, m, n, ldy, 64, kTileM, true) || !tensor_map(&map_b, b, true, n, k, ldb, 256, 64, false)) return NSML_ERR_CUDA;
  return launch_gemm<kGradInput, 256, false>(map_a, map_b, g, sms, static_cast<cudaStream_t>(stream));
}

int nsml_q8_matmul_grad_weight(const void* dy, int64_t ldy, const int8_t* a, int64_t lda, const float* a_scales, int64_t m, int64_t n, int64_t k,
                               void* dw, int64_t lddw, int dtype, int zero_first, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_size(m) || !valid_size(n) || !valid_size(k) || n < 1 || k < 1) return NSML_ERR_ARG;
  if (m > 0 && (!valid_gradient(dy, m, n, ldy) || !valid_codes(a, m, k, lda) || a_scales == nullptr || !aligned(a_scales, 4))) return NSML_ERR_ARG;
  int rc = check_out(dw, n, k, lddw, dtype, workspace, workspace_bytes);
  if (rc != NSML_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (m == 0) {  // an empty sum
    if (cudaMemsetAsync(workspace, 0, 256, st) != cudaSuccess) return cuda_error();
    const size_t size = dtype == NSML_F32 ? 4 : 2;
    if (zero_first && cudaMemset2DAsync(dw, (size_t)(n > 1 ? lddw : k) * size, 0, (size_t)k * size, (size_t)n, st) != cudaSuccess) return cuda_error();
    return NSML_OK;
  }
  int sms = 0;
  if ((rc = gemm_device(&sms)) != NSML_OK) return rc;
  GemmArgs g = result(dw, n, k, lddw, dtype, zero_first == 0, workspace);
  g.depth_scale = a_scales;
  g.depth = m;
  g.steps = (int)((m + 63) / 64);
  CUtensorMap map_a, map_b;
  if (!tensor_map(&map_a, dy, false, m, n, ldy, 64, 64, true) || !tensor_map(&map_b, a, true, m, k, lda, 256, 64, false)) return NSML_ERR_CUDA;
  return launch_gemm<kGradWeight, 256, false>(map_a, map_b, g, sms, st);
}

}  // extern "C"
