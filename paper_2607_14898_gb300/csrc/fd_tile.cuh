// What the attention kernels on 128 x 128 tiles share: 16-bit operands of either type, tile loads,
// products with a TMEM operand, and waits that give up.
#pragma once
#include "fd_internal.h"
#include "fd_ptx.cuh"

namespace fd {
namespace {

template <bool F16, int D>
struct Mma {
  // instruction descriptor: fp32 D, A and B fp16 (0) or bf16 (1), B MN-major for P V
  static __host__ __device__ constexpr uint32_t idesc(int n, bool b_mn) {
    return (1u << 4) | (F16 ? 0u : (1u << 7) | (1u << 10)) | (b_mn ? 1u << 16 : 0u) |
           (static_cast<uint32_t>(n >> 3) << 17) | (8u << 24);
  }
};

// 16-bit pairs of the cache's type
template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if constexpr (F16) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    return pack_bf16x2(lo, hi);
  }
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* m, uint32_t bar, int x,
                                            int y, int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
// 64 steps of K: A from TMEM (16 steps are 8 columns), B MN-major (16 steps are 2048 bytes)
__device__ __forceinline__ void mma4_ts_mn(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                           uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b32 a1, a2, a3;\n\t.reg .b64 b1, b2, b3;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 q, %4, %4;\n\t"
      "add.u32 a1, %1, 8;\n\tadd.u32 a2, %1, 16;\n\tadd.u32 a3, %1, 24;\n\t"
      "add.s64 b1, %2, 128;\n\tadd.s64 b2, %2, 256;\n\tadd.s64 b3, %2, 384;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, q;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, q;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, q;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// the same, issued by one lane of a converged warp
__device__ __forceinline__ void mma4_ts_mn_w(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q, e;\n\t.reg .b32 r, a1, a2, a3;\n\t.reg .b64 b1, b2, b3;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.eq.b32 q, %4, %4;\n\t"
      "add.u32 a1, %1, 8;\n\tadd.u32 a2, %1, 16;\n\tadd.u32 a3, %1, 24;\n\t"
      "add.s64 b1, %2, 128;\n\tadd.s64 b2, %2, 256;\n\tadd.s64 b3, %2, 384;\n\t"
      "elect.sync r|e, 0xffffffff;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a1], b1, %3, q;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a2], b2, %3, q;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a3], b3, %3, q;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// bytes (a multiple of 16) from 16-byte aligned memory, completing on `bar`
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
      "l"(src), "r"(bytes), "r"(bar)
      : "memory");
}
// MN-major operand in the 128-byte swizzle: 64 consecutive elements of the outer (M or N)
// dimension are one 128-byte row, 8 rows (8 steps of K) an atom of 1024 bytes; the stride
// between atoms along K is 1024 bytes, the leading offset the distance of the next 64 outer
// elements. 16 steps of K are 2048 bytes.
__device__ __forceinline__ uint64_t sdesc_mn_sw128(uint32_t saddr, uint32_t lead_bytes) {
  return static_cast<uint64_t>((saddr >> 4) & 0x3FFFu) |
         (static_cast<uint64_t>((lead_bytes >> 4) & 0x3FFFu) << 16) |
         (static_cast<uint64_t>(1024 >> 4) << 32) | (static_cast<uint64_t>(1) << 46) |
         (static_cast<uint64_t>(2) << 61);
}

// The waits of these kernels: at most kWaitLimitNs, like those of the library's other kernels (a wait that
// succeeds takes microseconds). One try is inline, the loop in a function of its own: with
// mbar_wait's 64-fold unrolled loop at every wait the attend kernel was 132 KB of code and a third
// of its issue slots went to instruction fetches (a third slower over the 480p chunk), and short
// loops inline cost as much in registers spilled around them. LIMIT is another only in the check of
// the waits themselves.
//
// Gives up after LIMIT, or soon after another wait of this launch (or an earlier one on the
// same status word) has given up (looked up every 64 tries: the word is a trip to L2 away); not so
// a drain, which waits for the CTA's own copies and products in flight.
template <unsigned long long LIMIT>
__device__ __noinline__ bool wait_more(uint32_t bar, uint32_t parity, int* err, int code, bool drain) {
  unsigned long long start = 0;
#pragma unroll 1
  for (unsigned n = 0; !mbar_try_wait(bar, parity); ++n) {
    if (n % 64 != 63) continue;
    const unsigned long long now = globaltimer();
    if (n == 63) start = now;
    if (now - start > LIMIT || (!drain && *reinterpret_cast<volatile int*>(err) != 0)) {
      atomicOr(err, code);
      return false;
    }
  }
  return true;
}
template <unsigned long long LIMIT = kWaitLimitNs>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, int* err, int code,
                                     bool drain = false) {
  return mbar_try_wait(bar, parity) || wait_more<LIMIT>(bar, parity, err, code, drain);
}
// For loops over several barriers that take whichever is through: whether to go on after a round
// that found none. rounds is 0 after one that did; every 1024 the time and the status word are looked at
// (32 bits of nanoseconds: they wrap after more than twice the limit).
template <unsigned long long LIMIT = kWaitLimitNs>
__device__ __forceinline__ bool poll_again(int& rounds, uint32_t& start, int* err, int code) {
  static_assert(LIMIT < 1ull << 31, "start wraps");
  if (++rounds % 1024 != 0) return true;
  const uint32_t now = static_cast<uint32_t>(globaltimer());
  if (rounds == 1024) start = now;
  if (now - start <= LIMIT && *reinterpret_cast<volatile int*>(err) == 0) return true;
  atomicOr(err, code);
  return false;
}
// The waits for a whole warp that stays together (tcgen05 loads and stores, which follow such
// waits, have to be executed by all its lanes at once): every decision is the warp's, so that its
// lanes never part. (Each instruction that only brings lanes together, or waits for a barrier that
// is through already, took 100 to 200 cycles of the attend kernel's softmax.)
template <unsigned long long LIMIT>
__device__ __noinline__ bool wait_more_warp(uint32_t bar, uint32_t parity, int* err, int code) {
  unsigned long long start = 0;
#pragma unroll 1
  for (unsigned n = 0; !__all_sync(0xffffffffu, mbar_try_wait(bar, parity)); ++n) {
    if (n % 64 != 63) continue;
    const unsigned long long now = globaltimer();
    if (n == 63) start = now;
    if (__any_sync(0xffffffffu,
                   now - start > LIMIT || *reinterpret_cast<volatile int*>(err) != 0)) {
      atomicOr(err, code);
      return false;
    }
  }
  return true;
}
template <unsigned long long LIMIT = kWaitLimitNs>
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, int* err, int code) {
  return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) ||
         wait_more_warp<LIMIT>(bar, parity, err, code);
}

// The end of a warp that issued products: none may be in flight when their operands' memory or TMEM is
// given back. (One barrier, used once; by every lane, so that the warp stays together.)
__device__ __forceinline__ void products_done(uint32_t bar, int* err) {
  mma_commit_w(bar);
  wait(bar, 0, err, ERR_WAIT_MMA, true);
  __syncwarp();
}

constexpr int kTile = 128;      // rows of a tile, slots of a block
constexpr int kSub = kTile * 128;  // bytes of 64 elements of 128 rows: one swizzled sub-tile

// Where 16 bytes, elements 8 chunk .. 8 chunk + 7 of a row, are in a tile of swizzled sub-tiles. A tile
// that goes to memory by TMA is put together there: a row is a thread's, and rows stored by threads
// take a cycle of the SM for every 32 bytes of each (4200 cycles at the end of every tile of 128 x 128).
__device__ __forceinline__ uint32_t tile_chunk(int row, int chunk) {
  return static_cast<uint32_t>((chunk >> 3) * kSub + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
}

// 4D map over 16-bit elements, strides in elements, boxes of 64 x b1 x b2 x 1
inline bool make_map(CUtensorMap* m, bool f16, const void* base, uint64_t d0, uint64_t d1, uint64_t d2,
              uint64_t d3, int64_t s1, int64_t s2, int64_t s3, uint32_t b1, uint32_t b2) {
  // a dimension of one entry never steps: its stride only has to be one that a map may have
  const uint64_t dims[4] = {d0, d1, d2, d3};
  const uint64_t strides[3] = {d1 > 1 ? static_cast<uint64_t>(s1) * 2 : 2 * d0,
                               d2 > 1 ? static_cast<uint64_t>(s2) * 2 : 2 * d0,
                               d3 > 1 ? static_cast<uint64_t>(s3) * 2 : 2 * d0};
  return tmap_16bit_4d(m, f16, base, dims, strides, b1, b2);
}

}  // namespace
}  // namespace fd
