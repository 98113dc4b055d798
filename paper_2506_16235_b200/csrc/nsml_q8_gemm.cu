// Matrix products of the q8 format on the tensor cores (tcgen05, accumulators in TMEM, operands by TMA).
//
//   kForward      out[m,n] = (sum_k a[m,k] b[n,k]) sa[m] sb[n]     int8 operands, 32-bit integer sums (exact)
//   kGradInput    dx[m,k]  = sum_n dy[m,n] (b[n,k] sb[n])          bfloat16 operands, float32 sums
//   kGradWeight   dw[n,k]  = sum_m dy[m,n] (a[m,k] sa[m])          the same, dy read across its rows
//
// Large products are bound by the tensor cores and, a few milliseconds into a loop, by the board's power (clocks of 1.2 to
// 1.45 GHz).  8192 x 8192 x 2048 in a loop, one B200: kForward 100-111 us (2.5 to 2.7 10^15 operations per second; the library's
// 8-bit product 99-117), the gradients 227-257 us (1.1 to 1.2; the library's bfloat16 product 180-210).  The gradients' distance
// is the restoring of every code once per 256 rows of the result.  Small ones are bound by latency: 4.1 us for 16 x 64 x 64
// (gradients 5.1 and 6.0), a third of a microsecond per step of the sum.  Large results of short sums are bound by the warps that
// take them out: 8192 x 16384 x 128 to bfloat16 81 us (268 MB, 41 us of the memory's time).
//
// In the gradients the codes' scale belongs to the axis of the sum, so it cannot wait for the epilogue: eight warps restore
// the codes to bfloat16 on their way from one shared-memory ring to another (exact for the scales that nsml_q8_pack makes).
// The restored matrix never exists in memory.
//
// Two forms.  PAIR: two blocks on neighbouring SMs share a 256 x 256 tile (cta_group::2): each loads, and restores, one half
// of both operands, so that shared memory is read half as often per product and every code is restored once per 256 rows of
// the result.  Otherwise a block has a 128 x 128 tile, and the blocks of a cluster have parts of the sum each, which they
// exchange through their shared memories (distributed shared memory, added in the order of the parts): for results that are
// too small to fill the GPU.
//
// The tensor cores cut float32 sums off instead of rounding them (measured: a relative error of 3e-10 per product of a sum),
// so float32 results are summed in pieces of kPiece products, which are added with rounding: 4e-7 instead of 6e-6 for 16384
// products.  A bfloat16 result of the pairs' form is one sum (at most 2^22 products: 1.3e-3, less than its rounding).
#include <cuda.h>

#include <mutex>
#include <type_traits>

#include "nsml_launch.h"
#include "nsml_q8.cuh"
#include "nsml_q8_products.h"

namespace nsml {
namespace q8 {

enum { kForward = 0, kGradInput = 1, kGradWeight = 2 };

constexpr int kPiece = 2048;                           // products per piece of a float32 sum
constexpr int kStepsPerPiece = kPiece / 64;
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
// CLUSTER: arrivals of both blocks of a pair are waited for
template <bool CLUSTER>
__device__ __forceinline__ bool bar_try_at(uint32_t bar, uint32_t parity) {
  if constexpr (!CLUSTER) return bar_try(bar, parity);
  uint32_t done;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.b32 %0, 1, 0, p;\n}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
// false: the wait ran out (here or, as `failed` says, elsewhere in the block)
template <bool CLUSTER, unsigned long long LIMIT>
__device__ __noinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, volatile int* failed) {
  const unsigned long long from = now_ns();
  while (true) {
    for (int i = 0; i < 64; ++i)
      if (bar_try_at<CLUSTER>(bar, parity)) return true;
    if (*failed != 0 || now_ns() - from > LIMIT) {
      *failed = 1;
      return false;
    }
  }
}
// For one thread.
template <bool CLUSTER = false, unsigned long long LIMIT = kWaitNs>
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* failed) {
  return bar_try_at<CLUSTER>(bar, parity) || bar_wait_slow<CLUSTER, LIMIT>(bar, parity, failed);
}
// For a whole warp, which then goes on as one (tcgen05.ld and .st want all of its lanes): the lanes poll on their own, and one
// may give up just as the barrier completes for another, so they agree on what came of it.  False if any lane gave up.
template <unsigned long long LIMIT = kWaitNs>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* failed) {
  return __all_sync(0xFFFFFFFFu, bar_wait<false, LIMIT>(bar, parity, failed));
}
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {  // the same place in another block of the cluster
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// bar: an address from in_block.  What the arrival announces has been fenced already (a proxy fence, or the tensor cores'
// own): a release over the cluster would wait for all of the thread's memory once more (8192 x 8192 x 2048: 355 against 282 us).
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();  // (aligned: the warp's lanes arrive together, one that has been on its own among them)
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// PAIR: bar may be the other block's (an address from in_block)
template <bool PAIR>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
__device__ __forceinline__ void tma_load_1d(uint32_t dst, const CUtensorMap* map, int x, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.1d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2}], [%3];"
               ::"r"(dst), "l"(map), "r"(x), "r"(bar) : "memory");
}

template <bool PAIR, int COLS>
__device__ __forceinline__ void tmem_alloc(uint32_t slot) {
  if constexpr (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "n"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "n"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
}
template <bool PAIR, int COLS>
__device__ __forceinline__ void tmem_free(uint32_t addr) {
  if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(COLS));
  else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "n"(COLS));
}
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
// the barrier (of both blocks) is arrived at once all tensor work issued so far by this thread is done
template <bool PAIR>
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  if constexpr (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
#define NSML_TC_MMA(GROUP, KIND)                                                                                       \
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::" GROUP ".kind::" KIND              \
               " [%0], %1, %2, %3, p;\n}" ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"((uint32_t)add) : "memory")
template <int MODE, bool PAIR>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
  if constexpr (MODE == kForward && PAIR) NSML_TC_MMA("2", "i8");
  else if constexpr (MODE == kForward) NSML_TC_MMA("1", "i8");
  else if constexpr (PAIR) NSML_TC_MMA("2", "f16");
  else NSML_TC_MMA("1", "f16");
}
#undef NSML_TC_MMA
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

// ... and back
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, "
      "%21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr) : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
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
// types, axes (bits 15, 16: the other axis is the contiguous one) and shape of one multiplication
template <int MODE, bool PAIR>
__host__ __device__ constexpr uint32_t mma_desc() {
  return (MODE == kForward ? (2u << 4 | 1u << 7 | 1u << 10)                                                        // s32 += s8 * s8
                           : (1u << 4 | 1u << 7 | 1u << 10 | (MODE == kGradWeight ? 1u << 15 : 0u) | 1u << 16))  // f32 += bf16 * bf16
         | (PAIR ? 256u / 8 << 17 | 256u / 16 << 24 : 128u / 8 << 17 | 128u / 16 << 24);
}

struct GemmArgs {
  int64_t rows, cols;        // of the result
  int steps;                 // blocks of the sum: 128 codes (kForward) or 64 products
  int piece;                 // blocks per piece of the sum
  void* out;
  int64_t ldo;
  bool bf16, add, vec, even; // vec: rows of the result start on 16-byte boundaries; even: on 4-byte ones
  const float* row_scale;    // kForward
  const float* col_scale;    // kForward
  int scale_shift;           // gradients: where the first scale is in the tensor map's first four
  int* status;
  int64_t tiles_m, tiles_n;
};

// A block's share of a tile is 128 rows of the first operand and 128 of the second in both forms.
template <int MODE, bool PAIR>
struct Shape {
  static constexpr int kTile = PAIR ? 256 : 128;
  static constexpr int kStage = MODE == kForward ? 2 * 128 * 128 : 128 * 128;  // bytes of a stage: the first operand; kForward: both
  static constexpr int kStages = PAIR ? 5 : 6;
  // gradients: the second operand's codes with the scales of their rows (68 of them, so that 64 start anywhere), and restored
  static constexpr int kCode = MODE == kForward ? 0 : 128 * 64 + 384;
  static constexpr int kCodes = 4;
  static constexpr int kWide = MODE == kForward ? 0 : 128 * 128;
  static constexpr int kWides = 4;
  // warps that restore one step's codes, taking turns (8192 x 8192 x 2048: all eight at every step 550 us, four 414, two 357;
  // sixteen warps instead of eight no change)
  static constexpr int kTurn = 2, kTurns = 8 / kTurn;
  // every turn meets every phase of its slots of the rings (a wait tells a phase from the next one only, not from the one after)
  static_assert(kCodes % kTurns == 0 && kWides % kTurns == 0, "");
  static constexpr int kWideAt = kStages * kStage, kCodeAt = kWideAt + kWides * kWide, kRings = kCodeAt + kCodes * kCode;
  static constexpr int kOutWarps = 8;  // warps that take results out: a quarter of the rows and half of the columns each
  static constexpr int kFirstRestorer = 4 + kOutWarps, kThreads = 32 * kFirstRestorer + (MODE == kForward ? 0 : 256);
  // PAIR: staging of results on their way out.  Otherwise a block's part of the results takes the rings' place at the end,
  // rows of kRow floats.
  static constexpr int kOut = PAIR ? kOutWarps * (32 * 128 + (MODE == kForward ? 128 * 4 : 0)) : 0;
  static constexpr int kRow = 132;
  static_assert(PAIR || 128 * kRow * 4 <= kRings, "");
  // two accumulators, one is read while the other is filled; PAIR false: and the sum of the pieces so far
  static constexpr int kTmem = 512, kSum = 2 * kTile;
  static constexpr size_t kSmem = 1024 + kRings + kOut;
  static_assert(kSmem + 512 <= 227 * 1024, "");
};

// The order of the tiles: columns `high` tiles high, so that the 74 or so in flight are a block whose sides are alike and share
// their operands in L2 (8192 x 8192 x 2048 forward: 8 high 105 us, 16 high 115; the gradients the same with 4 to 24).
__device__ __forceinline__ void tile_at(int64_t t, int64_t high, int64_t tiles_m, int64_t tiles_n, int64_t& m, int64_t& n) {
  const int64_t per = high * tiles_n, g = t / per, first = g * high, rows = min(high, tiles_m - first), in = t - g * per;
  m = first + in % rows;
  n = in / rows;
}

// Codes to bfloat16, times a scale.  The low seven bits of a code go into 128.0 (whose unit is 1), the sign bit into a second
// 128.0 (which it makes 256.0): the difference is the code.  A scale that is a bfloat16 (every power of two from 2^-126 on,
// 0, NaN) is multiplied in bfloat16, rounded once; any other in float32, rounded again.
__device__ __forceinline__ uint32_t restore2(uint32_t pair, __nv_bfloat162 scale) {
  const uint32_t x = (pair & 0x007F007Fu) | 0x43004300u, y = (pair & 0x00800080u) | 0x43004300u;
  const __nv_bfloat162 d = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&y)), scale);
  return *reinterpret_cast<const uint32_t*>(&d);
}
template <bool IN_BF16>
__device__ __forceinline__ uint4 restore8(uint32_t w0, uint32_t w1, float scale) {
  if constexpr (IN_BF16) {
    const uint32_t twice = __byte_perm(__float_as_uint(scale), 0, 0x3232);
    const __nv_bfloat162 s = *reinterpret_cast<const __nv_bfloat162*>(&twice);
    return make_uint4(restore2(__byte_perm(w0, 0, 0x4140), s), restore2(__byte_perm(w0, 0, 0x4342), s),
                      restore2(__byte_perm(w1, 0, 0x4140), s), restore2(__byte_perm(w1, 0, 0x4342), s));
  } else {
    auto two = [&](uint32_t w) { return pack2(restore((int8_t)w, scale), restore((int8_t)(w >> 8), scale)); };
    return make_uint4(two(w0), two(w0 >> 16), two(w1), two(w1 >> 16));
  }
}

// ---- results out ---------------------------------------------------------------------------------------------------------
// One result, in float32, to its place; g.add or `add`: on top of what is there, with one addition.
__device__ __forceinline__ void put1(const GemmArgs& g, int64_t row, int64_t col, bool add, float v) {
  if (row >= g.rows || col >= g.cols) return;
  if (g.bf16) {
    __nv_bfloat16* to = static_cast<__nv_bfloat16*>(g.out) + row * g.ldo + col;
    *to = __float2bfloat16_rn(add ? __fadd_rn(v, (float)*to) : v);
  } else {
    float* to = static_cast<float*>(g.out) + row * g.ldo + col;
    *to = add ? __fadd_rn(v, *to) : v;
  }
}

// Four consecutive ones; the rows start on 16-byte boundaries (g.vec).
__device__ __forceinline__ void put4(const GemmArgs& g, int64_t row, int64_t col, bool add, const float (&v)[4]) {
  if (row >= g.rows || col >= g.cols) return;
  if (col + 4 > g.cols) {
#pragma unroll
    for (int i = 0; i < 4; ++i) put1(g, row, col + i, add, v[i]);
    return;
  }
  float4 o;
  if (g.bf16) {
    uint2* to = reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(g.out) + row * g.ldo + col);
    if (add) {
      const uint2 w = *to;
      unpack2(w.x, o.x, o.y);
      unpack2(w.y, o.z, o.w);
      *to = make_uint2(pack2(__fadd_rn(v[0], o.x), __fadd_rn(v[1], o.y)), pack2(__fadd_rn(v[2], o.z), __fadd_rn(v[3], o.w)));
    } else {
      *to = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
    }
  } else {
    float4* to = reinterpret_cast<float4*>(static_cast<float*>(g.out) + row * g.ldo + col);
    if (add) {
      o = *to;
      *to = make_float4(__fadd_rn(v[0], o.x), __fadd_rn(v[1], o.y), __fadd_rn(v[2], o.z), __fadd_rn(v[3], o.w));
    } else {
      *to = make_float4(v[0], v[1], v[2], v[3]);
    }
  }
}

// Results that nothing is added to leave L2 first, so that their lines are written as they fill up (8192 x 8192 x 128 in float32
// 69 us without, 56 with it; beside it, 32 rows in a row without a branch back: 13779 x 9100 x 100 in bfloat16 107 -> 94).
template <bool KEEP, class T>
__device__ __forceinline__ void store_out(T* to, T v) {
  if constexpr (KEEP) *to = v;
  else __stcs(to, v);
}

// Word `lane` of a row of 128 bytes that is staged in 16-byte pieces, swizzled.
__device__ __forceinline__ uint32_t staged(const unsigned char* stage, int rr, int lane) {
  return *reinterpret_cast<const uint32_t*>(stage + rr * 128 + (((lane >> 2) ^ (rr & 7)) << 4) + 4 * (lane & 3));
}
// Those of every row below `last`, and where they go.
template <class Put>
__device__ __forceinline__ void each_row(const unsigned char* stage, int lane, int last, unsigned char* to, int64_t pitch, Put put) {
#pragma unroll
  for (int rr = 0; rr < 32; ++rr, to += pitch) {
    const uint32_t w = staged(stage, rr, lane);
    if (rr < last) put(to, w);
  }
}

// The block of 32 x 32 float32 results on top of what is there, rows below `rows` and columns below `cols`; wide: all of them,
// and float32 rows on 16-byte boundaries.  What is there is fetched for all rows before the first one is stored (a load may not
// move past a store: row by row 1024 x 8192 x 2048 took 98 us instead of 51, in bfloat16 171 instead of 64, and 7487 x 385 x 10163,
// whose rows are off 16-byte boundaries, 275 instead of 127).  A function of its own, so that the rest has the registers.
template <class T>
__device__ __forceinline__ void add_rows(const unsigned char* stage, int lane, int last, unsigned char* to, int64_t pitch) {
  T old[32];
#pragma unroll
  for (int rr = 0; rr < 32; ++rr) old[rr] = rr < last ? *reinterpret_cast<const T*>(to + rr * pitch) : T(0.0f);
#pragma unroll
  for (int rr = 0; rr < 32; ++rr) {
    const float v = __fadd_rn(__uint_as_float(staged(stage, rr, lane)), (float)old[rr]);
    if (rr >= last) continue;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<T*>(to + rr * pitch) = __float2bfloat16_rn(v);
    else *reinterpret_cast<T*>(to + rr * pitch) = v;
  }
}
__device__ __noinline__ void add_out(const unsigned char* stage, int rows, int cols, unsigned char* to, int64_t pitch, bool bf16, bool wide) {
  const int lane = threadIdx.x & 31, last = lane < cols ? rows : 0;
  if (bf16) return add_rows<__nv_bfloat16>(stage, lane, last, to + 2 * lane, pitch);
  if (!wide) return add_rows<float>(stage, lane, last, to + 4 * lane, pitch);
  const int j = lane & 7;
  to += (lane >> 3) * pitch + 16 * j;
  float4 old[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) old[i] = *reinterpret_cast<const float4*>(to + 4 * i * pitch);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int rr = 4 * i + (lane >> 3);
    const float4 w = *reinterpret_cast<const float4*>(stage + rr * 128 + ((j ^ (rr & 7)) << 4));
    *reinterpret_cast<float4*>(to + 4 * i * pitch) = make_float4(__fadd_rn(w.x, old[i].x), __fadd_rn(w.y, old[i].y), __fadd_rn(w.z, old[i].z), __fadd_rn(w.w, old[i].w));
  }
}

// ADD (PAIR only): results may go on top of what is there, a piece of the sum on top of the one before it among them.
template <int MODE, bool PAIR, bool ADD>
__global__ void __launch_bounds__(Shape<MODE, PAIR>::kThreads, 1)
k_q8_gemm(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_scales,
          const GemmArgs g) {
  using S = Shape<MODE, PAIR>;
  extern __shared__ unsigned char raw[];
  __shared__ alignas(8) uint64_t bars[2 * (S::kStages + S::kCodes + S::kWides) + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ int failed;
  const uint32_t ring = (smem_addr(raw) + 1023) & ~1023u;
  unsigned char* const ring_ptr = raw + (ring - smem_addr(raw));
  // full: the operands that the tensor cores read from the stages have landed (PAIR: in both blocks; the first block's barrier
  // counts).  codes_full, codes_empty: this block's codes.  wide_full, acc_empty: arrivals of both blocks, at the first one's.
  const uint32_t full = smem_addr(bars), empty = full + 8 * S::kStages, codes_full = empty + 8 * S::kStages, codes_empty = codes_full + 8 * S::kCodes,
                 wide_full = codes_empty + 8 * S::kCodes, wide_empty = wide_full + 8 * S::kWides, acc_full = wide_empty + 8 * S::kWides,
                 acc_empty = acc_full + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t blocks, rank;
  asm("mov.u32 %0, %cluster_nctarank;" : "=r"(blocks));
  asm("mov.u32 %0, %cluster_ctarank;" : "=r"(rank));
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      bar_init(full + 8 * i, 1);
      bar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < S::kCodes; ++i) {
      bar_init(codes_full + 8 * i, 1);
      bar_init(codes_empty + 8 * i, S::kTurn);  // a warp each
    }
    for (int i = 0; i < S::kWides; ++i) {
      bar_init(wide_full + 8 * i, PAIR ? 2 * S::kTurn : S::kTurn);  // a warp each
      bar_init(wide_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(acc_full + 8 * i, 1);
      bar_init(acc_empty + 8 * i, PAIR ? 2 * S::kOutWarps : S::kOutWarps);
    }
    failed = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) tmem_alloc<PAIR, S::kTmem>(smem_addr(&tmem_slot));
  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_sync();  // the other block's barriers are there
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  if (threadIdx.x == 0) {
    prefetch_map(&map_a);
    prefetch_map(&map_b);
    if constexpr (MODE != kForward) prefetch_map(&map_scales);
  }
  pdl_wait();
  pdl_launch_dependents();
  if (blockIdx.x == 0 && threadIdx.x == 0) *g.status = NSML_OK;

  // PAIR: a cluster takes every so many-th tile.  Otherwise one tile, and this block a part of its sum.
  const int64_t tiles = g.tiles_m * g.tiles_n, clusters = gridDim.x / blocks, first = blockIdx.x / blocks;
  const int64_t high = PAIR ? 8 : 32, stride = PAIR ? clusters : tiles;
  const int from = PAIR ? 0 : (int)((int64_t)g.steps * rank / blocks), to = PAIR ? g.steps : (int)((int64_t)g.steps * (rank + 1) / blocks);

  // PAIR false: in the end a warp takes a row of the tile at a time, rows dealt out to the blocks.  Its scales are fetched now.
  [[maybe_unused]] const int dealt = (int)blocks * (S::kThreads / 32);  // from a warp's row to its next one
  [[maybe_unused]] int64_t tile_m = 0, col = 0;
  [[maybe_unused]] float cs[4] = {}, my_scale = 0.0f;
  if constexpr (!PAIR) {
    int64_t n;
    tile_at(first, high, g.tiles_m, g.tiles_n, tile_m, n);
    col = n * 128 + 4 * lane;
    if constexpr (MODE == kForward) {
#pragma unroll
      for (int i = 0; i < 4; ++i) cs[i] = col + i < g.cols ? g.col_scale[col + i] : 0.0f;
      const int rr = rank + blocks * warp + lane * dealt;  // (lane i: the scale of the warp's i-th row)
      if (rr < 128 && tile_m * 128 + rr < g.rows) my_scale = g.row_scale[tile_m * 128 + rr];
    }
  }

  if (warp == 0 || (MODE != kForward && warp == 3)) {
    if (elect_one()) {  // ---- loads: warp 0 what the tensor cores read, warp 3 codes
      uint32_t it = 0;
      bool ok = true;
      for (int64_t t = first; ok && t < tiles; t += stride) {
        int64_t m, n;
        tile_at(t, high, g.tiles_m, g.tiles_n, m, n);
        const int row = (int)(m * S::kTile + (PAIR ? rank * 128 : 0)), col = (int)(n * S::kTile + (PAIR ? rank * 128 : 0));
        if (MODE != kForward && warp == 3) {
          for (int k = from; k < to; ++k, ++it) {
            const uint32_t s = it % S::kCodes, at = ring + S::kCodeAt + s * S::kCode, bar = codes_full + 8 * s;
            if (!(ok = bar_wait(codes_empty + 8 * s, (it / S::kCodes + 1) & 1, &failed))) break;
            bar_expect(bar, 128 * 64 + 68 * 4);
            tma_load<false>(at, &map_b, col, k * 64, bar);
            tma_load_1d(at + 128 * 64, &map_scales, k * 64, bar);
          }
          continue;
        }
        for (int k = from; k < to; ++k, ++it) {
          const uint32_t s = it % S::kStages, at = ring + s * S::kStage;
          if (!(ok = bar_wait(empty + 8 * s, (it / S::kStages + 1) & 1, &failed))) break;
          const uint32_t bar = PAIR ? in_block(full + 8 * s, 0) : full + 8 * s;
          if (!PAIR || rank == 0) bar_expect(full + 8 * s, PAIR ? 2 * S::kStage : S::kStage);
          if constexpr (MODE == kForward) {
            tma_load<PAIR>(at, &map_a, k * 128, row, bar);
            tma_load<PAIR>(at + 128 * 128, &map_b, k * 128, col, bar);
          } else if constexpr (MODE == kGradInput) {
            tma_load<PAIR>(at, &map_a, k * 64, row, bar);
          } else {
            tma_load<PAIR>(at, &map_a, row, k * 64, bar);
            tma_load<PAIR>(at + 64 * 128, &map_a, row + 64, k * 64, bar);
          }
        }
      }
      if (!ok) {  // copies in flight land before the block's shared memory goes; this wait is bounded too
        const unsigned long long began = now_ns();
        while (now_ns() - began < kWaitNs / 100) {}
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if ((!PAIR || rank == 0) && elect_one()) {  // ---- products
      uint32_t it = 0, unit = 0;
      bool ok = true;
      for (int64_t t = first; ok && t < tiles; t += stride) {
        for (int piece = from; ok && piece < to; piece += g.piece, ++unit) {
          const uint32_t buffer = unit & 1, acc = tmem + buffer * S::kTile;
          if (!(ok = bar_wait<PAIR>(acc_empty + 8 * buffer, ((unit >> 1) + 1) & 1, &failed))) break;
          tc_fence_after();
          const int end = min(to, piece + g.piece);
          for (int k = piece; k < end; ++k, ++it) {
            const uint32_t s = it % S::kStages, at = ring + s * S::kStage, w = it % S::kWides, wide = ring + S::kWideAt + w * S::kWide;
            if (!(ok = bar_wait(full + 8 * s, (it / S::kStages) & 1, &failed))) break;
            if constexpr (MODE != kForward)
              if (!(ok = bar_wait<PAIR>(wide_full + 8 * w, (it / S::kWides) & 1, &failed))) break;
            tc_fence_after();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint64_t a = MODE == kGradWeight ? tile_desc(at + j * 2048, 8192, 1024) : tile_desc(at + j * 32, 16, 1024);
              const uint64_t b = MODE == kForward ? tile_desc(at + 128 * 128 + j * 32, 16, 1024) : tile_desc(wide + j * 2048, 8192, 1024);
              tc_mma<MODE, PAIR>(acc, a, b, mma_desc<MODE, PAIR>(), k > piece || j > 0);
            }
            tc_commit<PAIR>(empty + 8 * s);
            if constexpr (MODE != kForward) tc_commit<PAIR>(wide_empty + 8 * w);
          }
          if (ok) tc_commit<PAIR>(acc_full + 8 * buffer);
        }
      }
    }
    __syncwarp();
  } else if (warp >= 4 && warp < 4 + S::kOutWarps) {  // ---- results
    const int quarter = warp & 3;  // (a warp reaches the rows of TMEM that its number says)
    constexpr int kChunks = S::kTile / 32 * 4 / S::kOutWarps;  // of 32 columns
    const int first_chunk = (warp - 4) / 4 * kChunks;
    unsigned char* const out = ring_ptr + S::kRings;
    uint32_t unit = 0;
    bool ok = true;
    for (int64_t t = first; ok && t < tiles; t += stride) {
      int64_t m, n;
      tile_at(t, high, g.tiles_m, g.tiles_n, m, n);
      for (int piece = from; piece < to; piece += g.piece, ++unit) {
        const uint32_t buffer = unit & 1, acc = tmem + buffer * S::kTile + ((uint32_t)quarter << 21);
        if (!(ok = warp_wait(acc_full + 8 * buffer, (unit >> 1) & 1, &failed))) break;
        tc_fence_after();
        auto release = [&] {  // the accumulator has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            if constexpr (PAIR) bar_arrive_cluster(in_block(acc_empty + 8 * buffer, 0));
            else bar_arrive(acc_empty + 8 * buffer);
          }
          __syncwarp();  // (the next access to TMEM is the whole warp's again)
        };
        if constexpr (PAIR) {
          unsigned char* const stage = out + (warp - 4) * 4096;  // 32 rows of 128 bytes, pieces of 16 swizzled
          float* const scales = reinterpret_cast<float*>(out + S::kOutWarps * 4096) + (warp - 4) * 128;
          const int64_t row0 = m * 256 + rank * 128 + quarter * 32, col0 = n * 256 + first_chunk * 32;
          const bool add = ADD && (g.add || piece > from), packed = g.bf16 && !add;
          float rs = 0.0f;
          if constexpr (MODE == kForward) {
            rs = row0 + lane < g.rows ? g.row_scale[row0 + lane] : 0.0f;
            for (int i = lane; i < 32 * kChunks; i += 32) scales[i] = col0 + i < g.cols ? g.col_scale[col0 + i] : 0.0f;
            __syncwarp();
          }
#pragma unroll 1
          for (int c = 0; c < kChunks; ++c) {
            uint32_t r[32];
            tmem_load32(acc + (first_chunk + c) * 32, r);
            if (c == kChunks - 1) release();
            if constexpr (MODE == kForward) {
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                const float4 cs = *reinterpret_cast<const float4*>(scales + c * 32 + j);
                r[j] = __float_as_uint(__fmul_rn(__fmul_rn((float)(int)r[j], rs), cs.x));
                r[j + 1] = __float_as_uint(__fmul_rn(__fmul_rn((float)(int)r[j + 1], rs), cs.y));
                r[j + 2] = __float_as_uint(__fmul_rn(__fmul_rn((float)(int)r[j + 2], rs), cs.z));
                r[j + 3] = __float_as_uint(__fmul_rn(__fmul_rn((float)(int)r[j + 3], rs), cs.w));
              }
            }
            unsigned char* const line = stage + lane * 128;
            if (packed) {  // 64 columns of bfloat16 at a time
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                uint4 w;
                w.x = pack2(__uint_as_float(r[8 * j]), __uint_as_float(r[8 * j + 1]));
                w.y = pack2(__uint_as_float(r[8 * j + 2]), __uint_as_float(r[8 * j + 3]));
                w.z = pack2(__uint_as_float(r[8 * j + 4]), __uint_as_float(r[8 * j + 5]));
                w.w = pack2(__uint_as_float(r[8 * j + 6]), __uint_as_float(r[8 * j + 7]));
                *reinterpret_cast<uint4*>(line + (((j + 4 * (c & 1)) ^ (lane & 7)) << 4)) = w;
              }
              if ((c & 1) == 0) continue;
            } else {  // 32 columns of float32
#pragma unroll
              for (int j = 0; j < 8; ++j)
                *reinterpret_cast<uint4*>(line + ((j ^ (lane & 7)) << 4)) = make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
            }
            __syncwarp();
            // (addresses are worked out once per block of 32 rows: with a bound and a product for every store the results of
            // 13779 x 9100 from a sum of 9 took 151 us, those of 8192 x 8192 x 2048 a tenth of the whole)
            const int size = g.bf16 ? 2 : 4, width = packed ? 64 : 32;
            const int64_t block = col0 + (packed ? c >> 1 : c) * width;
            unsigned char* const corner = static_cast<unsigned char*>(g.out) + (row0 * g.ldo + block) * size;
            const int64_t pitch = g.ldo * size;
            const bool whole = g.vec && row0 + 32 <= g.rows && block + width <= g.cols;
            if (whole && !add) {  // 16 bytes per lane, four rows at a time
              unsigned char* to = corner + (lane >> 3) * pitch + 16 * (lane & 7);
#pragma unroll
              for (int i = 0; i < 8; ++i, to += 4 * pitch) {
                const int rr = 4 * i + (lane >> 3), j = lane & 7;
                store_out<ADD>(reinterpret_cast<uint4*>(to), *reinterpret_cast<const uint4*>(stage + rr * 128 + ((j ^ (rr & 7)) << 4)));
              }
            } else if (!add) {  // 4 bytes per lane, a row at a time: stores next to each other wherever the row starts
              const int64_t col = block + (packed ? 2 : 1) * lane;
              const int last = col < g.cols ? (int)min((int64_t)32, g.rows - row0) : 0;
              unsigned char* const to = corner + 4 * lane;
              if (!packed || (g.even && col + 2 <= g.cols)) {
                each_row(stage, lane, last, to, pitch, [](unsigned char* at, uint32_t w) { store_out<ADD>(reinterpret_cast<uint32_t*>(at), w); });
              } else {
                const bool two = col + 1 < g.cols;
                each_row(stage, lane, last, to, pitch, [&](unsigned char* at, uint32_t w) {
                  store_out<ADD>(reinterpret_cast<uint16_t*>(at), (uint16_t)w);
                  if (two) store_out<ADD>(reinterpret_cast<uint16_t*>(at) + 1, (uint16_t)(w >> 16));
                });
              }
            } else if constexpr (ADD) {  // on top of what is there
              add_out(stage, (int)min((int64_t)32, g.rows - row0), (int)min((int64_t)32, g.cols - block), corner, pitch, g.bf16, whole);
            }
            __syncwarp();
          }
        } else {  // the sum of the pieces stays in TMEM; in the end it is this block's part (integers, or float32)
          const bool last = piece + g.piece >= to;
          float* const line = reinterpret_cast<float*>(ring_ptr) + (quarter * 32 + lane) * S::kRow;
#pragma unroll 1
          for (int c = first_chunk; c < first_chunk + kChunks; ++c) {
            uint32_t r[32];
            tmem_load32(acc + c * 32, r);
            if (c == first_chunk + kChunks - 1) release();
            const uint32_t sum = tmem + S::kSum + ((uint32_t)quarter << 21) + c * 32;
            if (piece > from) {  // (never integers)
              uint32_t o[32];
              tmem_load32(sum, o);
#pragma unroll
              for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__fadd_rn(__uint_as_float(o[j]), __uint_as_float(r[j])));
            }
            if (!last) {
              tmem_store32(sum, r);
              continue;
            }
            // (all of the block's products are done, so nothing reads or fills the rings any more)
#pragma unroll
            for (int j = 0; j < 8; ++j) *reinterpret_cast<uint4*>(line + c * 32 + 4 * j) = make_uint4(r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
          }
        }
      }
    }
  } else if (MODE != kForward && warp >= S::kFirstRestorer) {  // ---- codes to bfloat16: the warps take turns at the steps, kTurn of them at one
    if constexpr (MODE != kForward) {
      constexpr int kTurn = S::kTurn, kTurns = S::kTurns, kRows = 64 / kTurn;
      const int sub = lane & 7, row = (warp - S::kFirstRestorer) % kTurn * kRows + (lane >> 3);
      const int flip = sub >> 2, c0 = (sub & 3) * 2;  // lanes whose blocks of columns share banks write their halves in opposite order
      const int64_t mine = first < tiles ? (tiles - first + stride - 1) / stride : 0, total = mine * (to - from);
      for (int64_t it = (warp - S::kFirstRestorer) / kTurn; it < total; it += kTurns) {
        const uint32_t s = (uint32_t)(it % S::kCodes), w = (uint32_t)(it % S::kWides);
        if (!warp_wait(codes_full + 8 * s, (uint32_t)(it / S::kCodes) & 1, &failed)) break;
        const unsigned char* codes = ring_ptr + S::kCodeAt + s * S::kCode;
        const float* scales = reinterpret_cast<const float*>(codes + 128 * 64) + g.scale_shift;
        unsigned char* dst = ring_ptr + S::kWideAt + w * S::kWide + (sub >> 2) * 8192;
        uint4 q[kRows / 4];
        float scale[kRows / 4];
        bool in_bf16 = true;
#pragma unroll
        for (int i = 0; i < kRows / 4; ++i) {
          const int rr = row + 4 * i;
          q[i] = *reinterpret_cast<const uint4*>(codes + rr * 128 + sub * 16);
          scale[i] = scales[rr];
          in_bf16 = in_bf16 && (__float_as_uint(scale[i]) & 0xFFFFu) == 0;
        }
        __syncwarp();
        if (lane == 0) bar_arrive(codes_empty + 8 * s);  // (they are in registers)
        if (!warp_wait(wide_empty + 8 * w, ((uint32_t)(it / S::kWides) & 1) ^ 1, &failed)) break;
        auto convert = [&](auto kind) {
#pragma unroll
          for (int i = 0; i < kRows / 4; ++i) {
            const int rr = row + 4 * i;
            const uint4 lo = restore8<kind>(q[i].x, q[i].y, scale[i]), hi = restore8<kind>(q[i].z, q[i].w, scale[i]);
            unsigned char* line = dst + rr * 128;
            *reinterpret_cast<uint4*>(line + (((c0 + flip) ^ (rr & 7)) << 4)) = flip ? hi : lo;
            *reinterpret_cast<uint4*>(line + (((c0 + 1 - flip) ^ (rr & 7)) << 4)) = flip ? lo : hi;
          }
        };
        if (__all_sync(0xFFFFFFFFu, in_bf16)) convert(std::true_type{});  // (one branch per step, so that its rows overlap)
        else convert(std::false_type{});
        fence_async_shared();
        __syncwarp();
        if (lane == 0) {
          if constexpr (PAIR) bar_arrive_cluster(in_block(wide_full + 8 * w, 0));
          else bar_arrive(wide_full + 8 * w);
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && failed != 0) set_status(g.status, NSML_ERR_TIMEOUT);
  cluster_sync();  // PAIR: neither block's memory is used by the other any more.  Otherwise: every block's part is complete
  tc_fence_after();
  if (warp == 2) tmem_free<PAIR, S::kTmem>(tmem);
  if constexpr (!PAIR) {
    const int last = (int)min((int64_t)128, g.rows - tile_m * 128);
    // (one row at a time: four at a time are more code, which is fetched for the first time here, and 1 us slower)
#pragma unroll 1
    for (int i = 0, rr = rank + blocks * warp; rr < last; ++i, rr += dealt) {
      uint32_t sum[4] = {0, 0, 0, 0};
      for (uint32_t p = 0; p < blocks; ++p) {
        uint32_t x[4];
        asm volatile("ld.shared::cluster.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                     : "r"(in_block(ring + (rr * S::kRow + 4 * lane) * 4, p)));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (MODE == kForward) sum[j] += x[j];
          else sum[j] = p == 0 ? x[j] : __float_as_uint(__fadd_rn(__uint_as_float(sum[j]), __uint_as_float(x[j])));
        }
      }
      const float rs = __shfl_sync(0xFFFFFFFFu, my_scale, i);
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v[j] = MODE == kForward ? __fmul_rn(__fmul_rn((float)(int)sum[j], rs), cs[j]) : __uint_as_float(sum[j]);
      if (g.vec) {
        put4(g, tile_m * 128 + rr, col, g.add, v);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) put1(g, tile_m * 128 + rr, col + j, g.add, v[j]);
      }
    }
    cluster_sync();  // no block leaves while another reads its part
  }
}

// The waits' limit reached on purpose: one warp, whose first `lanes` lanes wait for a barrier that nobody arrives at (a millisecond)
// and the others for one that is complete.  The lanes have to end up with one answer, and together.
__global__ void __launch_bounds__(32) k_q8_wait_probe(int lanes, int* status) {
  __shared__ alignas(8) uint64_t bars[2];
  __shared__ int failed;
  const uint32_t never = smem_addr(bars), done = never + 8;
  if (threadIdx.x == 0) {
    bar_init(never, 1);
    bar_init(done, 1);
    failed = 0;
    bar_arrive(done);
  }
  __syncwarp();
  const bool ok = warp_wait<1000000ull>((int)threadIdx.x < lanes ? never : done, 0, &failed);
  const uint32_t agreed = __ballot_sync(0xFFFFFFFFu, ok);
  if (threadIdx.x == 0) *status = agreed == 0 ? NSML_ERR_TIMEOUT : agreed == 0xFFFFFFFFu ? NSML_OK : NSML_ERR_INTERNAL;
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

// Encodes a map.  The driver wants a context for that, which a host thread that has made no other call does not have yet (a
// launch would bind the device's): the device is set, then.
template <class Encode>
static bool encoded(Encode encode) {
  CUresult r = encode();
  int dev = 0;
  if (r == CUDA_ERROR_INVALID_CONTEXT && cudaGetDevice(&dev) == cudaSuccess && cudaSetDevice(dev) == cudaSuccess) r = encode();
  return r == CUDA_SUCCESS;
}

// `count` scales, from the 16-byte boundary at or before them; boxes of 68.
static bool scales_map(CUtensorMap* map, const float* scales, int64_t count, int* shift) {
  *shift = (int)(reinterpret_cast<uintptr_t>(scales) % 16 / 4);
  const cuuint64_t dims[1] = {(cuuint64_t)(count + *shift)}, strides[1] = {0};
  const cuuint32_t box[1] = {68}, step[1] = {1};
  return encoded([&] {
    return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 1, const_cast<float*>(scales - *shift), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  });
}

// rows x cols elements; boxes of box_cols x box_rows.  What lies outside reads as 0.
static bool tensor_map(CUtensorMap* map, const void* p, bool codes, int64_t rows, int64_t cols, int64_t ld, int box_cols, int box_rows, bool swizzle) {
  const int size = codes ? 1 : 2;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)(rows > 1 ? ld : (cols * size + 15) / 16 * 16 / size) * size};  // (one row: any stride will do)
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return encoded([&] {
    return encoder()(map, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, step,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  });
}

struct GemmDevice {
  bool ready = false;
  int pairs[4] = {}, split[4] = {};  // resident clusters of 1, 2, 4, 8 blocks of the two forms (PAIR: of two)
};
static GemmDevice g_gemm_dev[64];
static std::mutex g_gemm_mutex;

// clusters[s]: how many clusters of 2^s blocks are resident at once (at most what all three modes have)
template <int MODE, bool PAIR, bool ADD = false>
static cudaError_t prepare_kernel(int* clusters) {
  cudaError_t e = cudaFuncSetAttribute(k_q8_gemm<MODE, PAIR, ADD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<MODE, PAIR>::kSmem);
  for (int s = 0; s <= 3 && e == cudaSuccess; ++s) {
    if (PAIR && s != 1) continue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1 << s);
    cfg.blockDim = dim3(Shape<MODE, PAIR>::kThreads);
    cfg.dynamicSmemBytes = Shape<MODE, PAIR>::kSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1 << s;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int c = 0;
    e = cudaOccupancyMaxActiveClusters(&c, k_q8_gemm<MODE, PAIR, ADD>, &cfg);
    if (e == cudaSuccess && c < 1) e = cudaErrorUnknown;
    if (clusters[s] == 0 || c < clusters[s]) clusters[s] = c;
  }
  return e;
}

static int gemm_device(const GemmDevice** out) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cuda_error();
  std::lock_guard<std::mutex> lock(g_gemm_mutex);
  GemmDevice& d = g_gemm_dev[dev];
  if (!d.ready) {
    cudaError_t e = prepare_kernel<kForward, true>(d.pairs);
    if (e == cudaSuccess) e = prepare_kernel<kGradInput, true>(d.pairs);
    if (e == cudaSuccess) e = prepare_kernel<kGradWeight, true>(d.pairs);
    if (e == cudaSuccess) e = prepare_kernel<kGradInput, true, true>(d.pairs);
    if (e == cudaSuccess) e = prepare_kernel<kGradWeight, true, true>(d.pairs);
    if (e == cudaSuccess) e = prepare_kernel<kForward, false>(d.split);
    if (e == cudaSuccess) e = prepare_kernel<kGradInput, false>(d.split);
    if (e == cudaSuccess) e = prepare_kernel<kGradWeight, false>(d.split);
    if (e != cudaSuccess || encoder() == nullptr) return cuda_error();
    d.ready = true;
  }
  *out = &d;
  return NSML_OK;
}

static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Which form: the one that is done first by a count of microseconds.  Measured on one B200, per call: a step of the sum takes
// about a third of a microsecond in both forms while it waits for loads (a step of a 256 x 256 tile on two SMs takes as long
// as one of a 128 x 128 tile on one), a wave of blocks six to seven besides its steps, the exchange of the parts one.
// Returns the blocks per tile that share the sum, or 0: PAIR.
static int choose_form(const GemmArgs& g, const GemmDevice& dev, double step_us) {
  double best = 7.0 + (double)up(up(g.rows, 256) * up(g.cols, 256), dev.pairs[1]) * (g.steps * step_us * 1.2 + 0.3);
  const int64_t tiles = up(g.rows, 128) * up(g.cols, 128);
  int form = 0;
  if (tiles > 4096) return form;
  for (int s = 0; s <= 3 && (1 << s) <= g.steps; ++s) {
    const double t = (double)up(tiles, dev.split[s]) * (6.0 + (s > 0 ? 1.0 : 0.0) + (double)up(g.steps, 1 << s) * step_us);
    if (t < best) {
      best = t;
      form = 1 << s;
    }
  }
  return form;
}

template <int MODE>
static int launch_gemm(const CUtensorMap& map_a, const CUtensorMap& map_b, const CUtensorMap& map_scales, GemmArgs g, const GemmDevice& dev, cudaStream_t st) {
  const int form = choose_form(g, dev, MODE == kForward ? 0.30 : 0.36);
  const int tile = form == 0 ? 256 : 128;
  if (MODE == kForward || (form == 0 && g.bf16)) g.piece = g.steps;  // (integers are exact)
  g.tiles_m = up(g.rows, tile);
  g.tiles_n = up(g.cols, tile);
  const int64_t tiles = g.tiles_m * g.tiles_n;
  LaunchScope scope(K_Q8_GEMM, st);
  cudaError_t e;
  if (form == 0) {
    using S = Shape<MODE, true>;
    auto* kernel = k_q8_gemm<MODE, true, false>;
    if constexpr (MODE != kForward)
      if (g.add || g.piece < g.steps) kernel = k_q8_gemm<MODE, true, true>;
    e = launch_in_stream(kernel, dim3((unsigned int)(2 * (tiles < dev.pairs[1] ? tiles : dev.pairs[1]))), dim3(S::kThreads), S::kSmem, st, 2, map_a, map_b,
                    map_scales, g);
  } else {
    using S = Shape<MODE, false>;
    e = launch_in_stream(k_q8_gemm<MODE, false, false>, dim3((unsigned int)(tiles * form)), dim3(S::kThreads), S::kSmem, st, (unsigned int)form,
                    map_a, map_b, map_scales, g);
  }
  return e == cudaSuccess ? NSML_OK : cuda_error();
}

static bool valid_size(int64_t v) { return v >= 0 && v <= NSML_Q8_MAX_ROWS; }
static bool valid_operand(const void* p, int64_t rows, int64_t cols, int64_t ld) {
  return valid_codes(p, rows, cols, ld) && (rows <= 1 || ld < ((int64_t)1 << 40));  // (the longest stride of a tensor map)
}
static bool valid_gradient(const void* p, int64_t rows, int64_t cols, int64_t ld) {
  return p != nullptr && aligned(p, 16) && (rows <= 1 || (ld >= cols && ld % 8 == 0 && ld < ((int64_t)1 << 39)));
}
// A call without tokens: nothing to compute, but the workspace's status is this call's.  (An address that CUDA does not know, as
// every one is on a machine without a device, is left alone.)
static int no_tokens(void* workspace, cudaStream_t st) {
  cudaPointerAttributes where;
  if (cudaPointerGetAttributes(&where, workspace) != cudaSuccess || where.type == cudaMemoryTypeUnregistered) {
    cudaGetLastError();
    return NSML_OK;
  }
  return cudaMemsetAsync(workspace, 0, NSML_Q8_MATMUL_WORKSPACE_BYTES, st) == cudaSuccess ? NSML_OK : cuda_error();
}
static int check_workspace(const void* workspace, size_t workspace_bytes) {
  if (workspace == nullptr || !aligned(workspace, 256)) return NSML_ERR_ARG;
  return workspace_bytes < NSML_Q8_MATMUL_WORKSPACE_BYTES ? NSML_ERR_CAPACITY : NSML_OK;
}
static int check_out(const void* out, int64_t rows, int64_t cols, int64_t ldo, int dtype, const void* workspace, size_t workspace_bytes) {
  if (dtype != NSML_F32 && dtype != NSML_BF16) return NSML_ERR_ARG;
  if (out == nullptr || !aligned(out, dtype == NSML_F32 ? 4 : 2) || (rows > 1 && ldo < cols)) return NSML_ERR_ARG;
  return check_workspace(workspace, workspace_bytes);
}
static GemmArgs result(void* out, int64_t rows, int64_t cols, int64_t ldo, int dtype, bool add, void* workspace) {
  GemmArgs g = {};
  g.rows = rows;
  g.cols = cols;
  g.out = out;
  g.ldo = ldo;
  g.bf16 = dtype == NSML_BF16;
  g.add = add;
  g.even = aligned(out, 4) && (rows <= 1 || !g.bf16 || ldo % 2 == 0);
  g.vec = aligned(out, 16) && (rows <= 1 || ldo % (g.bf16 ? 8 : 4) == 0);
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
  int rc = check_workspace(workspace, workspace_bytes);
  if (m == 0) return rc == NSML_OK ? no_tokens(workspace, static_cast<cudaStream_t>(stream)) : rc;
  if (!valid_operand(a, m, k, lda) || !valid_operand(b, n, k, ldb) || a_scales == nullptr || !aligned(a_scales, 4) || b_scales == nullptr || !aligned(b_scales, 4))
    return NSML_ERR_ARG;
  rc = check_out(out, m, n, ldo, dtype, workspace, workspace_bytes);
  if (rc != NSML_OK) return rc;
  if (m <= kMaxTokens)
    return launch_tokens(a, lda, a_scales, b, ldb, b_scales, (int)m, n, (int)k, out, ldo, dtype == NSML_BF16, static_cast<int*>(workspace),
                         static_cast<cudaStream_t>(stream));
  const GemmDevice* dev = nullptr;
  if ((rc = gemm_device(&dev)) != NSML_OK) return rc;
  GemmArgs g = result(out, m, n, ldo, dtype, false, workspace);
  g.row_scale = a_scales;
  g.col_scale = b_scales;
  g.steps = (int)((k + 127) / 128);
  CUtensorMap map_a, map_b;
  if (!tensor_map(&map_a, a, true, m, k, lda, 128, 128, true) || !tensor_map(&map_b, b, true, n, k, ldb, 128, 128, true)) return NSML_ERR_CUDA;
  return launch_gemm<kForward>(map_a, map_b, map_b, g, *dev, static_cast<cudaStream_t>(stream));
}

int nsml_q8_matmul_grad_input(const void* dy, int64_t ldy, const int8_t* b, int64_t ldb, const float* b_scales, int64_t m, int64_t n, int64_t k,
                              void* dx, int64_t lddx, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_size(m) || !valid_size(n) || !valid_size(k) || n < 1 || k < 1 || n > NSML_Q8_MAX_GRAD_DEPTH) return NSML_ERR_ARG;
  int rc = check_workspace(workspace, workspace_bytes);
  if (m == 0) return rc == NSML_OK ? no_tokens(workspace, static_cast<cudaStream_t>(stream)) : rc;
  if (!valid_gradient(dy, m, n, ldy) || !valid_operand(b, n, k, ldb) || b_scales == nullptr || !aligned(b_scales, 4)) return NSML_ERR_ARG;
  rc = check_out(dx, m, k, lddx, dtype, workspace, workspace_bytes);
  if (rc != NSML_OK) return rc;
  const GemmDevice* dev = nullptr;
  if ((rc = gemm_device(&dev)) != NSML_OK) return rc;
  GemmArgs g = result(dx, m, k, lddx, dtype, false, workspace);
  g.steps = (int)((n + 63) / 64);
  g.piece = kStepsPerPiece;
  CUtensorMap map_a, map_b, map_scales;
  if (!scales_map(&map_scales, b_scales, n, &g.scale_shift) || !tensor_map(&map_a, dy, false, m, n, ldy, 64, 128, true) || !tensor_map(&map_b, b, true, n, k, ldb, 128, 64, false)) return NSML_ERR_CUDA;
  return launch_gemm<kGradInput>(map_a, map_b, map_scales, g, *dev, static_cast<cudaStream_t>(stream));
}

int nsml_q8_matmul_grad_weight(const void* dy, int64_t ldy, const int8_t* a, int64_t lda, const float* a_scales, int64_t m, int64_t n, int64_t k,
                               void* dw, int64_t lddw, int dtype, int zero_first, void* workspace, size_t workspace_bytes, void* stream) {
  if (!valid_size(m) || !valid_size(n) || !valid_size(k) || n < 1 || k < 1 || m > NSML_Q8_MAX_GRAD_DEPTH) return NSML_ERR_ARG;
  if (m > 0 && (!valid_gradient(dy, m, n, ldy) || !valid_operand(a, m, k, lda) || a_scales == nullptr || !aligned(a_scales, 4))) return NSML_ERR_ARG;
  int rc = check_out(dw, n, k, lddw, dtype, workspace, workspace_bytes);
  if (rc != NSML_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (m == 0) {  // an empty sum
    if ((rc = no_tokens(workspace, st)) != NSML_OK) return rc;
    const size_t size = dtype == NSML_F32 ? 4 : 2;
    if (zero_first && cudaMemset2DAsync(dw, (size_t)(n > 1 ? lddw : k) * size, 0, (size_t)k * size, (size_t)n, st) != cudaSuccess) return cuda_error();
    return NSML_OK;
  }
  const GemmDevice* dev = nullptr;
  if ((rc = gemm_device(&dev)) != NSML_OK) return rc;
  GemmArgs g = result(dw, n, k, lddw, dtype, zero_first == 0, workspace);
  g.steps = (int)((m + 63) / 64);
  g.piece = kStepsPerPiece;
  CUtensorMap map_a, map_b, map_scales;
  if (!scales_map(&map_scales, a_scales, m, &g.scale_shift) || !tensor_map(&map_a, dy, false, m, n, ldy, 64, 64, true) || !tensor_map(&map_b, a, true, m, k, lda, 128, 64, false)) return NSML_ERR_CUDA;
  return launch_gemm<kGradWeight>(map_a, map_b, map_scales, g, *dev, st);
}

int nsml_selftest_q8_bounded_wait(void* workspace, size_t workspace_bytes, int lanes, void* stream) {
  if (workspace == nullptr || !aligned(workspace, 256) || lanes < 0 || lanes > 32) return NSML_ERR_ARG;
  if (workspace_bytes < NSML_Q8_MATMUL_WORKSPACE_BYTES) return NSML_ERR_CAPACITY;
  k_q8_wait_probe<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>(lanes, static_cast<int*>(workspace));
  return cudaGetLastError() == cudaSuccess ? NSML_OK : NSML_ERR_CUDA;
}

}  // extern "C"
