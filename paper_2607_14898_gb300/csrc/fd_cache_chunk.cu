// Attention over a bounded cache, many rows (a chunk's or a prompt's queries): tensor cores, two
// passes over the scores.
//
//   attend   out = softmax(c q k^T) v by blocks of 256 slots with a running maximum and sum, and each
//            row's log2 of its sum of exponentials, lse
//   weigh    w_j = sum_r exp2(c q_r . k_j - lse_r): the scores again, transposed (a thread has a
//            slot and sums over rows), so that no probability is ever stored
//
// A tile is tile_tokens whole tokens with all `per` heads of the list's KV group: row r of tile
// i is row i * tile_rows + r of the list, token r / per, head r % per, loaded as one TMA box {64
// elements, per heads, tile_tokens tokens}. Rows past tile_rows in shared memory stay zero.
//
// Products: 4 rows used D flops for attend, 2 rows used D for weigh (bf16 or fp16 in, fp32
// accumulation in TMEM), and two exponentials for each score.
#include <algorithm>
#include <type_traits>

#include "fd_cache_attn.cuh"

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

// The waits of this file: at most kWaitLimitNs, like those of the library's other kernels (a wait that
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

// The waits above on a barrier that nothing arrives at, a warp: the word gets ERR_WAIT_CHECK when
// they give up, after a millisecond.
constexpr unsigned long long kCheckLimitNs = 1000000ull;
__global__ void __launch_bounds__(32) wait_check_kernel(int which, int* err) {
  __shared__ uint64_t never;
  const uint32_t bar = smem_u32(&never);
  if (threadIdx.x == 0) {
    mbar_init(bar, 1);
    fence_barrier_init();
  }
  __syncthreads();
  if (which == 0) {
    if (threadIdx.x == 0) wait<kCheckLimitNs>(bar, 0, err, ERR_WAIT_CHECK);
  } else if (which == 1) {
    if (threadIdx.x == 0) wait<kCheckLimitNs>(bar, 0, err, ERR_WAIT_CHECK, true);
  } else if (which == 2) {
    wait_warp<kCheckLimitNs>(bar, 0, err, ERR_WAIT_CHECK);
  } else if (threadIdx.x == 0) {
    int rounds = 0;
    uint32_t start = 0;
    while (!mbar_test_wait(bar, 0) &&
           poll_again<kCheckLimitNs>(rounds, start, err, ERR_WAIT_CHECK)) {
    }
  }
}

// 16 lanes of the warp's quarter and 16 columns in 16 x 8 fragments: of fragment j thread t gets
// columns 8 j + 2 (t % 4), + 1 of lane t / 4 (r[4 j], r[4 j + 1]) and of lane t / 4 + 8
__device__ __forceinline__ void tmem_ld_16x256b_x2(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7])
      : "r"(taddr));
}

// sum += x where a < b
__device__ __forceinline__ void add_if_less(float& sum, float x, uint32_t a, uint32_t b) {
  asm("{\n\t.reg .pred p;\n\tsetp.lt.u32 p, %2, %3;\n\t@p add.rn.f32 %0, %0, %1;\n\t}"
      : "+f"(sum)
      : "f"(x), "r"(a), "r"(b));
}

constexpr int kTile = 128;      // rows of a tile, slots of a block
constexpr int kSub = kTile * 128;  // bytes of 64 elements of 128 rows: one swizzled sub-tile

// ------------------------------------------------------------------------------ attend
//
// Persistent CTAs (one per SM), each with an equal run of the (tile, block of 256 slots) units,
// tile after tile: a segment is a tile's consecutive blocks. A tile that is cut between CTAs leaves
// partial results, which join_parts adds up in the order of the blocks.
//
// The softmax is the longest chain of a block (scores out of TMEM, maximum, exponentials, P into
// TMEM), so sixteen warps share it, four on every SM sub-partition: each of four groups of 128
// threads has a quarter of a block's slots, a row (TMEM lane) per thread. The row's running
// maximum is handed from quarter to quarter, which sets the groups a step apart: the exponentials
// of one run beside the loads, masks and maxima of the others.
//   warps 0-15    softmax: warps 4 q .. 4 q + 3 quarter q
//   warp 16       TMA: Q of the segment, K and V by half blocks (128 slots). K and V have a ring
//                 each, so that a half is fetched as soon as one has been used: two more are there
//                 or on their way meanwhile (D = 128, where 192 KB of them fit)
//   warps 17, 18  products: a thread issues one tcgen05.mma per 104 to 158 cycles whatever its
//                 size, so two of them share the work. D = 64: those of the block's first and
//                 second half, each half with a running maximum and an O of its own; D = 128: S of
//                 both halves, and P V into the one O that TMEM has room for.
//   warp 19       positions of each block, on the barrier of its scores; zeros for the values of
//                 empty slots (their probability is 0, but 0 times NaN is NaN)
// TMEM (512 columns): S 2 x 128, P 2 x 64 (two 16-bit values a column), O 2 x 64 or 128. S takes the
// next scores once the softmax has it in registers.
// Bound by the softmax's instruction issue (65 % of the slots at D = 128, 54 % at D = 64) with the
// round trips between its warps and the products; the tensor pipe is busy 59 % and 32 % of the time.
// 2 x 2001 queries of 32 heads of 128 over 8191 slots, fp16: 400 us, 1343 TFLOP/s; 1560 of 16 heads
// of 64 over 6240, bf16: 60 us, 664 TFLOP/s.
template <int D>
struct AttendCfg {
  static constexpr int kKeys = 256;
  static constexpr int kQBytes = kTile * D * 2;
  static constexpr int kHalfBytes = kTile * D * 2;  // K or V of half a block
  static constexpr int kSlots = D == 128 ? 3 : 6;   // of each ring; half 2 J + h is in slot (2 J + h) % kSlots
  static constexpr bool kTwoO = D == 64;
  // A parity tells a phase from its neighbours and no further, so whoever waits for a slot's
  // barrier has to wait for every phase of it: one thread waits for all halves, or (D = 64) one
  // for each half of the blocks, whose slots differ because the ring's length is even.
  static_assert(!kTwoO || kSlots % 2 == 0, "waiters");
  static constexpr int kOffK = kQBytes;
  static constexpr int kOffV = kOffK + kSlots * kHalfBytes;
  static constexpr int kOffPos = kOffV + kSlots * kHalfBytes;
  static constexpr int kOffMax = kOffPos + kKeys * 4;
  static constexpr int kOffBar = kOffMax + (kTwoO ? 4 : 1) * kTile * 4;  // D = 64: [half][m, l]
  static constexpr int kThreads = 640;  // five warps a sub-partition: 96 registers (six: 80)
  static constexpr uint32_t kColS = 0, kColP = 256, kColO = 384;
  // barriers: kSFull, kSRead of the halves, kPFull, kPv of the quarters, kMax of each of their
  // warps
  static constexpr int kQFull = 0, kQFree = 1, kKFull = 2, kKFree = kKFull + kSlots,
                       kVFull = kKFree + kSlots, kVFree = kVFull + kSlots,
                       kVReady = kVFree + kSlots, kSFull = kVReady + kSlots, kSRead = kSFull + 2,
                       kPFull = kSRead + 2, kPv = kPFull + 4, kMax = kPv + 4, kORead = kMax + 16,
                       kDone = kORead + 1, kBars = kDone + 2;
  static constexpr int kSmem = kOffBar + (kBars * 8 + 24 + 127) / 128 * 128;  // TMEM slot, largest positions
  static_assert(kSmem <= 227 * 1024, "shared memory");
};

// units [c W / parts, (c + 1) W / parts) of CTA c
struct Units {
  int64_t total;
  int parts;
  __host__ __device__ int64_t start(int c) const { return total * c / parts; }
  __host__ __device__ int owner(int64_t u) const {
    return static_cast<int>(((u + 1) * parts - 1) / total);
  }
};

// a walk over a CTA's units
struct Walk {
  int tile;              // over all lists
  int block, left, seg;  // left: units after this one
  bool first, last;      // of its segment
  __device__ Walk(const Units& w, int cta, int blocks) {
    const int64_t u = w.start(cta);
    left = static_cast<int>(w.start(cta + 1) - u) - 1;
    tile = static_cast<int>(u / blocks);
    block = static_cast<int>(u - static_cast<int64_t>(tile) * blocks);
    seg = 0;
    first = true;
    last = block == blocks - 1 || left == 0;
  }
  __device__ bool valid() const { return left >= 0; }
  __device__ void next(int blocks) {
    --left;
    first = ++block == blocks;
    if (first) {
      block = 0;
      ++tile;
      ++seg;
    }
    last = block == blocks - 1 || left <= 0;
  }
};

constexpr float kSlack = 8.f;  // log2 by which a row's maximum may grow before O is rescaled

template <bool F16, int D>
__global__ void __launch_bounds__(AttendCfg<D>::kThreads, 1)
    attend_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CacheAttn p) {
  using C = AttendCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem);
  const bool aligned = (base & 1023u) == 0;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kOffBar);
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * static_cast<uint32_t>(i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
  volatile uint32_t* pos_top = tmem_slot + 1;  // largest position of each half
  int32_t* pos_ring = reinterpret_cast<int32_t*>(smem + C::kOffPos);  // [256]
  // the rows' running maximum (D = 64: of each half); at a segment's end their sums
  volatile float* row_max = reinterpret_cast<volatile float*>(smem + C::kOffMax);
  const int blocks = p.attend_blocks;
  const Units units{static_cast<int64_t>(p.lists) * p.row_tiles * blocks, p.parts};

  // rows past tile_rows are never loaded
  for (int i = threadIdx.x; i < C::kQBytes / 16; i += C::kThreads)
    reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  if (threadIdx.x == 0) {
    if (!aligned) atomicOr(p.err, ERR_SMEM_ALIGN);
    mbar_init(bar(C::kQFull), 1);
    mbar_init(bar(C::kQFree), C::kTwoO ? 2 : 1);
    for (int i = 0; i < C::kSlots; ++i) {
      mbar_init(bar(C::kKFull + i), 1);
      mbar_init(bar(C::kKFree + i), 1);
      mbar_init(bar(C::kVFull + i), 1);
      mbar_init(bar(C::kVFree + i), 1);
      mbar_init(bar(C::kVReady + i), 1);
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(bar(C::kSFull + h), 2);  // scores, positions
      mbar_init(bar(C::kSRead + h), 256);
      mbar_init(bar(C::kDone + h), 1);
    }
    for (int q = 0; q < 4; ++q) {
      mbar_init(bar(C::kPFull + q), 128);
      mbar_init(bar(C::kPv + q), 1);
      for (int i = 0; i < 4; ++i) mbar_init(bar(C::kMax + 4 * q + i), 32);
    }
    mbar_init(bar(C::kORead), 512);
    fence_barrier_init();
  }
  grid_dep_wait();
  if (warp == 0) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (!aligned) {
    // nothing is loaded or computed; the status word says why
  } else if (warp == 16) {
    if (lane == 0) {
      prefetch_tmap(&tmQ);
      prefetch_tmap(&tmK);
      prefetch_tmap(&tmV);
      // the next half of K, or of V, as soon as its slot is free
      struct Next {
        Walk w;
        int half, slot;  // half: halves so far
        uint32_t phase;
        int stream, group;
      };
      const Walk w0(units, blockIdx.x, blocks);
      Next k{w0, 0, 0, 0, 0, 0}, v{w0, 0, 0, 0, 0, 0};
      auto load = [&](Next& n, const CUtensorMap* map, uint32_t to, int full) {
        const uint32_t b = bar(full + n.slot);
        mbar_expect_tx(b, C::kHalfBytes);
        for (int d = 0; d < D / 64; ++d)
          tma_load_4d(to + n.slot * C::kHalfBytes + d * kSub, map, b, 64 * d,
                      n.w.block * C::kKeys + (n.half & 1) * kTile, n.group, n.stream);
        if (++n.slot == C::kSlots) {
          n.slot = 0;
          n.phase ^= 1;
        }
        if (n.half++ & 1) n.w.next(blocks);
      };
      auto begins = [&](const Next& n) { return n.w.first && (n.half & 1) == 0; };
      auto locate = [&](Next& n) {
        const int lst = n.w.tile / p.row_tiles;
        n.stream = lst / p.groups;
        n.group = lst - n.stream * p.groups;
        return lst;
      };
      int segs = 0, idle = 0;
      uint32_t idle_since = 0;
      while (k.w.valid() || v.w.valid()) {
        bool moved = false;
        if (k.w.valid() && mbar_test_wait(bar(C::kKFree + k.slot), k.phase ^ 1) &&
            (!begins(k) || k.w.seg == 0 || mbar_test_wait(bar(C::kQFree), (k.w.seg - 1) & 1))) {
          if (begins(k)) {
            const int lst = locate(k);
            mbar_expect_tx(bar(C::kQFull), p.tile_rows * D * 2);
            for (int d = 0; d < D / 64; ++d)
              tma_load_4d(base + d * kSub, &tmQ, bar(C::kQFull), 64 * d, k.group * p.per,
                          (k.w.tile - lst * p.row_tiles) * p.tile_tokens, k.stream);
            segs = k.w.seg + 1;
          }
          load(k, &tmK, base + C::kOffK, C::kKFull);
          moved = true;
        }
        if (v.w.valid() && mbar_test_wait(bar(C::kVFree + v.slot), v.phase ^ 1)) {
          if (begins(v)) locate(v);
          load(v, &tmV, base + C::kOffV, C::kVFull);
          moved = true;
        }
        if (moved)
          idle = 0;
        else if (!poll_again(idle, idle_since, p.err, ERR_WAIT_MMA))
          break;
      }
      // nothing may be in flight when the CTA exits
      if (segs > 0) wait(bar(C::kQFull), (segs - 1) & 1, p.err, ERR_WAIT_TMA, true);
      for (int j = k.half - 1; j >= 0 && j >= k.half - C::kSlots; --j)
        wait(bar(C::kKFull + j % C::kSlots), (j / C::kSlots) & 1, p.err, ERR_WAIT_TMA, true);
      for (int j = v.half - 1; j >= 0 && j >= v.half - C::kSlots; --j)
        wait(bar(C::kVFull + j % C::kSlots), (j / C::kSlots) & 1, p.err, ERR_WAIT_TMA, true);
    }
  } else if (warp == 19) {
    // ---- positions, fetched a block ahead, and empty slots' values
    Walk w(units, blockIdx.x, blocks);  // at the block whose positions are fetched next
    const int count = w.left + 1;
    const int32_t* pos = p.pos;
    int32_t at[8];
    auto fetch = [&]() {
      if (!w.valid()) return;
      if (w.first) pos = p.pos + static_cast<int64_t>(w.tile / p.row_tiles) * p.capacity;
      const int slot0 = w.block * C::kKeys + lane;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        at[i] = slot0 + 32 * i < p.used ? __ldg(pos + slot0 + 32 * i) : -1;
      w.next(blocks);
    };
    auto through = [&](int b, uint32_t parity) {
      return __all_sync(0xffffffffu, mbar_test_wait(bar(b), parity)) != 0;
    };
    fetch();
    // blocks published and halves of V made ready so far
    int J = 0, n = 0, slot = 0, idle = 0;
    uint32_t phase = 0, idle_since = 0;
    // Bit i: this lane's slot 32 i + lane of the block published last is empty; above, those of the
    // blocks before it. (The softmax reads a block's scores after its part of the product before
    // last, so V is at most two blocks behind.)
    uint32_t holes = 0;
    while (n < 2 * count) {
      bool moved = false;
      // once the softmax is through with the positions and scores of the block before
      if (J < count && (J == 0 || (through(C::kSRead, (J - 1) & 1) &&
                                   through(C::kSRead + 1, (J - 1) & 1)))) {
        uint32_t top[2] = {0, 0};
        holes <<= 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          pos_ring[32 * i + lane] = at[i];
          top[i / 4] = max(top[i / 4], static_cast<uint32_t>(at[i]));
          holes |= at[i] < 0 ? 1u << i : 0u;
        }
        top[0] = __reduce_max_sync(0xffffffffu, top[0]);
        top[1] = __reduce_max_sync(0xffffffffu, top[1]);
        if (lane < 2) pos_top[lane] = lane ? top[1] : top[0];
        __syncwarp();
        if (lane < 2) mbar_arrive(bar(C::kSFull + lane));
        ++J;
        fetch();
        moved = true;
      }
      if (n < 2 * J && through(C::kVFull + slot, phase)) {
        const uint32_t mine = (holes >> (8 * (J - 1 - n / 2) + 4 * (n & 1))) & 15u;
        if (__any_sync(0xffffffffu, mine != 0)) {
#pragma unroll 1
          for (int r = 0; r < 4; ++r) {
            if (!((mine >> r) & 1u)) continue;
            uint4* row = reinterpret_cast<uint4*>(smem + C::kOffV + slot * C::kHalfBytes +
                                                  (32 * r + lane) * 128);
#pragma unroll
            for (int d = 0; d < D / 64; ++d)
#pragma unroll
              for (int c = 0; c < 8; ++c) row[d * (kSub / 16) + c] = make_uint4(0, 0, 0, 0);
          }
          fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::kVReady + slot));
        ++n;
        if (++slot == C::kSlots) {
          slot = 0;
          phase ^= 1;
        }
        moved = true;
      }
      if (moved)
        idle = 0;
      else if (!__all_sync(0xffffffffu, poll_again(idle, idle_since, p.err, ERR_WAIT_TMA)))
        break;
    }
  } else if (warp >= 17) {  // 17 and 18
    if (lane == 0) {
      constexpr uint32_t is = Mma<F16, D>::idesc(kTile, false), io = Mma<F16, D>::idesc(D, true);
      const uint32_t s_col = tmem + C::kColS, p_col = tmem + C::kColP, o_col = tmem + C::kColO;
      const uint64_t q0 = sdesc_k_sw128(base);
      // S of half h of the walk's block, number J, once Q and K are there
      auto scores = [&](int J, int h, const Walk& w) -> bool {
        const int i = 2 * J + h, s = i % C::kSlots;
        if (w.first && (C::kTwoO || h == 0) &&
            !wait(bar(C::kQFull), w.seg & 1, p.err, ERR_WAIT_TMA))
          return false;
        if (!wait(bar(C::kKFull + s), (i / C::kSlots) & 1, p.err, ERR_WAIT_TMA)) return false;
        tc_fence_after();
        const uint64_t k0 = sdesc_k_sw128(base + C::kOffK + s * C::kHalfBytes);
#pragma unroll
        for (int d = 0; d < D / 64; ++d)
          mma4_bf16_ss(s_col + 128u * h, q0 + static_cast<uint64_t>(d * (kSub >> 4)),
                       k0 + static_cast<uint64_t>(d * (kSub >> 4)), is, d > 0);
        mma_commit(bar(C::kSFull + h));
        mma_commit(bar(C::kKFree + s));
        if (w.last && (C::kTwoO || h == 1)) mma_commit(bar(C::kQFree));
        return true;
      };
      // P V of half h of block J into O (the half's own for D = 64), quarter after quarter
      auto values = [&](int J, int h, const Walk& w) -> bool {
        const int i = 2 * J + h, s = i % C::kSlots;
        if (!wait(bar(C::kVReady + s), (i / C::kSlots) & 1, p.err, ERR_WAIT_TMA)) return false;
        // the previous segment's O has been read
        if (w.first && w.seg > 0 && (C::kTwoO || h == 0) &&
            !wait(bar(C::kORead), (w.seg - 1) & 1, p.err, ERR_WAIT_EPI))
          return false;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int q = 2 * h + x;
          if (!wait(bar(C::kPFull + q), J & 1, p.err, ERR_WAIT_EPI)) return false;
          tc_fence_after();
          const uint64_t v0 =
              sdesc_mn_sw128(base + C::kOffV + s * C::kHalfBytes + x * (kSub / 2), kSub);
          const bool fresh = w.first && x == 0 && (C::kTwoO || h == 0);
          mma4_ts_mn(o_col + (C::kTwoO ? 64u * h : 0u), p_col + 32u * q, v0, io, !fresh);
          mma_commit(bar(C::kPv + q));
        }
        mma_commit(bar(C::kVFree + s));
        return true;
      };
      const int h = warp - 17;
      Walk w(units, blockIdx.x, blocks);
      bool ok = true;
      if (C::kTwoO) {
        ok = w.valid() && scores(0, h, w);
        for (int J = 0; w.valid() && ok; ++J) {
          const Walk here = w;
          w.next(blocks);
          if (w.valid())
            ok = wait(bar(C::kSRead + h), J & 1, p.err, ERR_WAIT_EPI) && scores(J + 1, h, w);
          ok = ok && values(J, h, here);
        }
      } else if (h == 0) {
        for (int J = 0; w.valid() && ok; w.next(blocks), ++J)
          for (int x = 0; x < 2 && ok; ++x)
            ok = (J == 0 || wait(bar(C::kSRead + x), (J - 1) & 1, p.err, ERR_WAIT_EPI)) &&
                 scores(J, x, w);
      } else {
        for (int J = 0; w.valid() && ok; w.next(blocks), ++J)
          ok = values(J, 0, w) && values(J, 1, w);
      }
      mma_commit(bar(C::kDone + h));
      wait(bar(C::kDone + h), 0, p.err, ERR_WAIT_MMA, true);
    }
  } else {
    // ---- softmax of quarter q of the blocks
    const int q = warp >> 2, h = q >> 1, lanes = warp & 3;
    const int row = lanes * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>(lanes * 32) << 16;
    const uint32_t s_col = tmem + lane_off + C::kColS + 64u * q;
    const uint32_t p_col = tmem + lane_off + C::kColP + 32u * q;
    const uint32_t o_col = tmem + lane_off + C::kColO;
    // the quarters that share an O and a running maximum: the one before this, in the same block
    // or (the first one) the last in the block before
    constexpr int kShare = C::kTwoO ? 2 : 4;
    const bool lead = q % kShare == 0;
    const int prev = lead ? q + kShare - 1 : q - 1;
    volatile float* const my_max = row_max + (C::kTwoO ? 2 * h * kTile : 0) + row;
    // (a per-thread copy: as a kernel parameter it cost the loops a fifth more instructions)
    const float c = __shfl_sync(0xffffffffu, p.scale_log2, 0);
    const uint64_t c2 = pack_f32x2(c, c);
    // A wait that gives up has set the status word, and every wait after it returns at once: the
    // warps go on to the end, since they have to meet at the segments' barriers.
    int J = 0;
    Walk w(units, blockIdx.x, blocks);  // at the segments' first blocks
    while (w.valid()) {
      // the segment's tile and this thread's row in it
      const int lst = w.tile / p.row_tiles, stream = lst / p.groups, group = lst - stream * p.groups;
      const int token = (w.tile - lst * p.row_tiles) * p.tile_tokens + row / p.per;
      const bool valid = row < p.tile_rows && token < p.n_q;
      const int qp = valid ? __ldg(p.q_pos + static_cast<int64_t>(stream) * p.n_q + token) : -1;
      // a slot is visible if its position, unsigned, is below this
      const uint32_t limit = qp < 0 ? 0u : static_cast<uint32_t>(qp) + 1u;
      // of the warp's rows (those that are none do not count: their results go nowhere)
      const uint32_t least = __reduce_min_sync(0xffffffffu, valid ? limit : 0x80000000u);
      const uint32_t most = __reduce_max_sync(0xffffffffu, limit);
      float m = -INFINITY, l = 0.f;
      const int count = min(blocks - w.block, w.left + 1), end = J + count;
      bool first = true;
#pragma unroll 1
      for (; J < end; ++J, first = false) {
        wait_warp(bar(C::kSFull + h), J & 1, p.err, ERR_WAIT_MMA);
        tc_fence_after();
        uint32_t sr[2][32];
#pragma unroll
        for (int i = 0; i < 2; ++i) tmem_ld_32x32b_x32(s_col + 32 * i, sr[i]);
        // The slots that this row sees. The rows of a warp differ in slots whose position is between
        // their limits, which are few: a warp's rows are a handful of tokens, next to each other as
        // a rule. Bit i of some_hidden: some row does not see all of slots 8 i to 8 i + 7.
        uint32_t seen[2] = {0xffffffffu, 0xffffffffu}, all[2] = {0xffffffffu, 0xffffffffu};
        if (pos_top[h] >= least) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t at =
                static_cast<uint32_t>(pos_ring[64 * q + 32 * i + lane]);
            all[i] = seen[i] = __ballot_sync(0xffffffffu, at < least);
            uint32_t todo = __ballot_sync(0xffffffffu, at < most) & ~seen[i];
#pragma unroll 1
            for (; todo != 0; todo &= todo - 1) {
              const int e = __ffs(todo) - 1;
              if (__shfl_sync(0xffffffffu, at, e) < limit) seen[i] |= 1u << e;
            }
          }
        }
        tmem_ld_wait();
        tc_fence_before();
        mbar_arrive(bar(C::kSRead + h));
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (all[i] != 0xffffffffu) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(seen[i] & (1u << e))) sr[i][e] = 0xff800000u;
          }
        float mx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t* x = sr[i / 2] + 16 * (i % 2);
          mx[i] = __uint_as_float(x[0]);
#pragma unroll
          for (int e = 1; e < 15; e += 2)
            mx[i] = fmax3(mx[i], __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
          mx[i] = fmaxf(mx[i], __uint_as_float(x[15]));
        }
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c;
        // the maximum that O stands for now
        const bool fresh = first && lead;  // O holds nothing yet
        float before = -INFINITY;
        if (!lead || J > 0) {
          wait_warp(bar(C::kMax + 4 * prev + lanes), (lead ? J - 1 : J) & 1, p.err, ERR_WAIT_EPI);
          if (!fresh) before = *my_max;
        }
        const bool grow = top > before + kSlack;
        const float now = grow ? top : before;
        const float off = now == -INFINITY ? 0.f : now;
        *my_max = now;
        mbar_arrive(bar(C::kMax + 4 * q + lanes));
        const float f = grow ? ex2_approx(before - off) : 1.f;  // of O
        l *= m == now ? 1.f : ex2_approx(m - off);
        m = now;
        const uint64_t off2 = pack_f32x2(-off, -off);
        uint64_t sum2[2] = {0, 0};
        // P in the cache's type, which the product with V takes (fp32 sums): 2^-9 (bf16) or 2^-12 (fp16) of
        // each p at most, the output by that share of sum p |v|, beside its own rounding of the same
        // size. The sums are of P unrounded, and weigh works its scores out for itself.
        uint32_t pk[2][16];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            uint64_t x;
            asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "r"(sr[i][e]), "r"(sr[i][e + 1]));
            asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(x) : "l"(x), "l"(c2), "l"(off2));
            float a, b;
            asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
            a = ex2_approx(a);
            b = ex2_approx(b);
            asm("add.rn.f32x2 %0, %0, %1;" : "+l"(sum2[e / 2 % 2]) : "l"(pack_f32x2(a, b)));
            pk[i][e / 2] = pack16<F16>(a, b);
          }
        // the previous block's product has read this quarter's P
        if (!first) wait_warp(bar(C::kPv + q), (J - 1) & 1, p.err, ERR_WAIT_MMA);
        if (!fresh && __any_sync(0xffffffffu, grow)) {
          // O as the products of all quarters before left it
          wait_warp(bar(C::kPv + prev), (lead ? J - 1 : J) & 1, p.err, ERR_WAIT_MMA);
          tc_fence_after();
#pragma unroll 1
          for (int d = 0; d < D; d += 16) {
            uint32_t o[16];
            const uint32_t at = o_col + (C::kTwoO ? 64u * h : 0u) + d;
            tmem_ld_32x32b_x16(at, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tmem_st_32x32b_x16(at, o);
          }
        }
        tc_fence_after();
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 2; ++i) tmem_st_32x32b_x16(p_col + 16 * i, pk[i]);
        {
          float a0, b0, a1, b1;
          asm("mov.b64 {%0, %1}, %2;" : "=f"(a0), "=f"(b0) : "l"(sum2[0]));
          asm("mov.b64 {%0, %1}, %2;" : "=f"(a1), "=f"(b1) : "l"(sum2[1]));
          l += (a0 + b0) + (a1 + b1);
        }
        tmem_st_wait();
        tc_fence_before();
        mbar_arrive(bar(C::kPFull + q));
      }

      // ---- the segment's result: this thread's quarter of the row's elements
#pragma unroll
      for (int i = 0; i < 4; ++i) wait_warp(bar(C::kPv + i), (J - 1) & 1, p.err, ERR_WAIT_MMA);
      tc_fence_after();
      // the sums on the last maximum, added up in the order of the quarters (named barriers of
      // the row's four warps between the steps)
      wait_warp(bar(C::kMax + 4 * (q / kShare * kShare + kShare - 1) + lanes), (J - 1) & 1, p.err,
                ERR_WAIT_EPI);
      const float last = *my_max;
      l *= m == last ? 1.f : ex2_approx(m - last);
      m = last;
      // (the warp together at each of them)
      auto meet = [&]() {
        __syncwarp();
        named_barrier(1 + lanes, 128);
      };
      meet();
      float all, f0 = 1.f, f1 = 1.f;
      if (C::kTwoO) {  // [half][m, l]: the halves on the larger maximum
        volatile float* const my_sum = my_max + kTile;
        if (lead) *my_sum = l;
        meet();
        if (!lead) *my_sum = *my_sum + l;
        meet();
        const float m0 = row_max[row], l0 = row_max[kTile + row];
        const float m1 = row_max[2 * kTile + row], l1 = row_max[3 * kTile + row];
        m = fmaxf(m0, m1);
        const float at = m == -INFINITY ? 0.f : m;
        f0 = ex2_approx(m0 - at);
        f1 = ex2_approx(m1 - at);
        all = fmaf(f0, l0, f1 * l1);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (q == i) *my_max = i == 0 ? l : *my_max + l;
          meet();
        }
        all = *my_max;
      }
      meet();  // read by all before the next segment writes
      const int64_t unit = static_cast<int64_t>(w.tile) * blocks;
      const bool whole = units.owner(unit) == units.owner(unit + blocks - 1);
      // a cut tile's part: the CTA's first segment (slot 0) unless the tile began in this CTA
      const int64_t part = static_cast<int64_t>(blockIdx.x) * 2 + (units.start(blockIdx.x) > unit ? 0 : 1);
      const float inv = all == 0.f ? 0.f : 1.f / all;
      uint16_t* out = static_cast<uint16_t*>(p.out) + stream * p.out_stream +
                      static_cast<int64_t>(token) * p.out_token +
                      static_cast<int64_t>(group * p.per + row % p.per) * p.out_head;
#pragma unroll
      for (int d0 = 0; d0 < D / 4; d0 += 16) {
        const int d = q * (D / 4) + d0;
        uint32_t o[16];
        __syncwarp();
        tmem_ld_32x32b_x16(o_col + d, o);
        if (C::kTwoO) {
          uint32_t o2[16];
          tmem_ld_32x32b_x16(o_col + 64 + d, o2);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e)
            o[e] = __float_as_uint(fmaf(f0, __uint_as_float(o[e]), f1 * __uint_as_float(o2[e])));
        } else {
          tmem_ld_wait();
        }
        if (whole && valid) {
#pragma unroll
          for (int e = 0; e < 16; e += 8) {
            uint4 v;
            v.x = pack16<F16>(__uint_as_float(o[e]) * inv, __uint_as_float(o[e + 1]) * inv);
            v.y = pack16<F16>(__uint_as_float(o[e + 2]) * inv, __uint_as_float(o[e + 3]) * inv);
            v.z = pack16<F16>(__uint_as_float(o[e + 4]) * inv, __uint_as_float(o[e + 5]) * inv);
            v.w = pack16<F16>(__uint_as_float(o[e + 6]) * inv, __uint_as_float(o[e + 7]) * inv);
            *reinterpret_cast<uint4*>(out + d + e) = v;
          }
        } else if (!whole) {
          uint4* po = reinterpret_cast<uint4*>(p.part_o) + part * (D / 4) * kTile + row;
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            po[(d + e) / 4 * kTile] = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
      }
      tc_fence_before();
      mbar_arrive(bar(C::kORead));
      if (q == 0) {
        if (!whole)
          p.part_ml[part * kTile + row] = make_float2(m, all);
        else if (row < p.tile_rows)
          p.lse[static_cast<int64_t>(w.tile) * p.tile_rows + row] =
              !valid || all == 0.f ? INFINITY : m + log2f(all);
      }
      w.left -= count;
      ++w.tile;
      w.block = 0;
    }
  }
  grid_dep_launch();
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// The cut tiles' parts added up: blockIdx.x + 1 = a CTA of attend, whose first unit may be where a
// tile was cut (the tile's first cut does the work), blockIdx.y = 4 elements of the head, a thread
// per row. Bound by latency (the maxima, then the parts): 10 us alone for the 480p chunk's 9.7 MB.
template <bool F16, int D>
__global__ void __launch_bounds__(kTile) join_parts_kernel(const __grid_constant__ CacheAttn p) {
  const int blocks = p.attend_blocks;
  const Units units{static_cast<int64_t>(p.lists) * p.row_tiles * blocks, p.parts};
  const int k = blockIdx.y, row = threadIdx.x;
  const int gt = static_cast<int>(units.start(blockIdx.x + 1) / blocks);  // tile over all lists
  const int lst = gt / p.row_tiles, tile = gt - lst * p.row_tiles;
  const int64_t unit = static_cast<int64_t>(gt) * blocks;
  const int lo = units.owner(unit), hi = units.owner(unit + blocks - 1);
  grid_dep_wait();  // (the divisions above are done while attend's last CTAs run)
  if (lo != hi && static_cast<int>(blockIdx.x) == lo) {
    // the tile is the last segment of its first CTA and the first of the others
    auto part_of = [&](int c) { return static_cast<int64_t>(c) * 2 + (c == lo ? 1 : 0); };
    float top = -INFINITY;
    for (int c = lo; c <= hi; ++c) top = fmaxf(top, __ldcg(p.part_ml + part_of(c) * kTile + row).x);
    const float off = top == -INFINITY ? 0.f : top;
    float l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = lo; c <= hi; ++c) {
      const int64_t part = part_of(c);
      const float2 ml = __ldcg(p.part_ml + part * kTile + row);
      const float4 o =
          __ldcg(reinterpret_cast<const float4*>(p.part_o) + (part * (D / 4) + k) * kTile + row);
      const float f = ex2_approx(ml.x - off);
      l = fmaf(f, ml.y, l);
      acc.x = fmaf(f, o.x, acc.x);
      acc.y = fmaf(f, o.y, acc.y);
      acc.z = fmaf(f, o.z, acc.z);
      acc.w = fmaf(f, o.w, acc.w);
    }
    const int stream = lst / p.groups, group = lst - stream * p.groups;
    const int token = tile * p.tile_tokens + row / p.per;
    const bool valid = row < p.tile_rows && token < p.n_q;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (valid) {
      uint16_t* out = static_cast<uint16_t*>(p.out) + stream * p.out_stream +
                      static_cast<int64_t>(token) * p.out_token +
                      static_cast<int64_t>(group * p.per + row % p.per) * p.out_head + 4 * k;
      *reinterpret_cast<uint2*>(out) = make_uint2(pack16<F16>(acc.x * inv, acc.y * inv),
                                                  pack16<F16>(acc.z * inv, acc.w * inv));
    }
    if (k == 0 && row < p.tile_rows)
      p.lse[static_cast<int64_t>(gt) * p.tile_rows + row] =
          !valid || l == 0.f ? INFINITY : off + log2f(l);
  }
  grid_dep_launch();
}

// ------------------------------------------------------------------------------ weigh
//
// A CTA has one block of 128 slots of one list and a run of the list's row tiles: S^T = K Q^T, K
// from shared memory all along, Q tiles through a ring; two groups of warps take the tiles in turn,
// each with its own accumulator in TMEM, and add exp2(c s - lse_r) over a tile's rows. Two CTAs
// fit an SM. Scores come out of TMEM in 16 x 8 fragments: a thread has 4 slots and every fourth
// pair of rows, so that a row's lse and limit, read from shared memory, serve 4 scores (with a slot
// a thread and all rows the reads were what bounded the kernel).
// Bound by the exponentials and the wait for the next scores: an accumulator is free when its group
// has read the last of it, and the other group's is all that runs meanwhile (TMEM holds two for
// each of the SM's two CTAs). Freeing them by halves of 64 rows with a product thread for each group was
// slower all the same (275 us for the prompt below, then at 249), and so was that thread alone (264).
// 2 x 2001 queries of 32 heads of 128 over 8191 slots: 240 us, 1119
// TFLOP/s; 1560 of 16 heads of 64 over 6240: 34 us, 586 TFLOP/s.
//   warps 0-3 / 4-7  even / odd tiles   warp 8  TMA   warp 9  products   warp 10  lse and limits
template <int D>
struct WeighCfg {
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kStages = D == 128 ? 2 : 4;
  static constexpr int kRowStages = 4;  // two for each of the accumulators
  static constexpr int kOffQ = kTileBytes;
  static constexpr int kOffRows = kOffQ + kStages * kTileBytes;    // lse, then limits, per stage
  static constexpr int kOffLow = kOffRows + kRowStages * kTile * 8;  // smallest limit per stage
  static constexpr int kOffSum = kOffLow + 64;                       // one group's sums
  static constexpr int kOffBar = kOffSum + kTile * 4;
  static constexpr int kSmem = kOffBar + 256;
  static constexpr int kThreads = 352;
  static constexpr int kKFull = 0, kQFull = 1, kQFree = kQFull + kStages,
                       kTFull = kQFree + kStages, kTFree = kTFull + 2, kDone = kTFree + 2,
                       kBars = kDone + 1;
  static_assert(kBars * 8 + 8 <= 256, "barriers");
  static_assert(2 * (kSmem + 1024) <= 227 * 1024, "two CTAs");
};

template <bool F16, int D>
__global__ void __launch_bounds__(WeighCfg<D>::kThreads, 2)
    weigh_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CacheAttn p) {
  using C = WeighCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem);
  const bool aligned = (base & 1023u) == 0;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kOffBar);
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * static_cast<uint32_t>(i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
  float* row_lse = reinterpret_cast<float*>(smem + C::kOffRows);
  uint32_t* row_lim = reinterpret_cast<uint32_t*>(row_lse + C::kRowStages * kTile);
  uint32_t* row_low = reinterpret_cast<uint32_t*>(smem + C::kOffLow);
  const int block = blockIdx.x, split = blockIdx.y, lst = blockIdx.z;
  const int stream = lst / p.groups, group = lst - stream * p.groups;
  const int first = static_cast<int>(static_cast<int64_t>(p.row_tiles) * split / p.row_splits);
  const int tiles =
      static_cast<int>(static_cast<int64_t>(p.row_tiles) * (split + 1) / p.row_splits) - first;

  for (int i = threadIdx.x; i < C::kStages * C::kTileBytes / 16; i += C::kThreads)
    reinterpret_cast<uint4*>(smem + C::kOffQ)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  if (threadIdx.x == 0) {
    if (!aligned) atomicOr(p.err, ERR_SMEM_ALIGN);
    mbar_init(bar(C::kKFull), 1);
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(bar(C::kQFull + i), 1);
      mbar_init(bar(C::kQFree + i), 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(bar(C::kTFull + x), 2);  // scores, rows
      mbar_init(bar(C::kTFree + x), 128);
    }
    mbar_init(bar(C::kDone), 1);
    fence_barrier_init();
  }
  grid_dep_wait();
  if (warp == 0) {
    tmem_alloc(smem_u32(tmem_slot), 256);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  // this thread's slot in the end
  float total = 0.f;
  const int key = block * kTile + (warp & 3) * 32 + (lane & 3) * 8 + (lane >> 2);
  const int64_t list_at = static_cast<int64_t>(lst) * p.capacity;
  if (!aligned) {
  } else if (warp == 8) {
    if (lane == 0) {
      prefetch_tmap(&tmQ);
      prefetch_tmap(&tmK);
      mbar_expect_tx(bar(C::kKFull), C::kTileBytes);
      for (int d = 0; d < D / 64; ++d)
        tma_load_4d(base + d * kSub, &tmK, bar(C::kKFull), 64 * d, block * kTile, group, stream);
      int i = 0;
      for (; i < tiles; ++i) {
        const int s = i % C::kStages;
        if (!wait(bar(C::kQFree + s), ((i / C::kStages) & 1) ^ 1, p.err, ERR_WAIT_MMA)) break;
        mbar_expect_tx(bar(C::kQFull + s), p.tile_rows * D * 2);
        for (int d = 0; d < D / 64; ++d)
          tma_load_4d(base + C::kOffQ + s * C::kTileBytes + d * kSub, &tmQ, bar(C::kQFull + s),
                      64 * d, group * p.per, (first + i) * p.tile_tokens, stream);
      }
      wait(bar(C::kKFull), 0, p.err, ERR_WAIT_TMA, true);
      for (int j = i - 1; j >= 0 && j >= i - C::kStages; --j)
        wait(bar(C::kQFull + j % C::kStages), (j / C::kStages) & 1, p.err, ERR_WAIT_TMA, true);
    }
  } else if (warp == 9) {
    if (lane == 0) {
      constexpr uint32_t idesc = Mma<F16, D>::idesc(kTile, false);
      const uint64_t k0 = sdesc_k_sw128(base);
      bool ok = wait(bar(C::kKFull), 0, p.err, ERR_WAIT_TMA);
      for (int i = 0; i < tiles && ok; ++i) {
        const int s = i % C::kStages, x = i & 1;
        ok = wait(bar(C::kTFree + x), ((i >> 1) & 1) ^ 1, p.err, ERR_WAIT_EPI) &&
             wait(bar(C::kQFull + s), (i / C::kStages) & 1, p.err, ERR_WAIT_TMA);
        if (!ok) break;
        tc_fence_after();
        const uint64_t q0 = sdesc_k_sw128(base + C::kOffQ + s * C::kTileBytes);
#pragma unroll
        for (int d = 0; d < D / 64; ++d) {
          const uint64_t at = static_cast<uint64_t>(d * (kSub >> 4));
          mma4_bf16_ss(tmem + 128u * x, k0 + at, q0 + at, idesc, d > 0);
        }
        mma_commit(bar(C::kTFull + x));
        mma_commit(bar(C::kQFree + s));
      }
      mma_commit(bar(C::kDone));
      wait(bar(C::kDone), 0, p.err, ERR_WAIT_MMA, true);
    }
  } else if (warp == 10) {
    bool ok = true;
    int token_of[4];  // within the tile
#pragma unroll
    for (int j = 0; j < 4; ++j) token_of[j] = (32 * j + lane) / p.per;
    const int32_t* q_pos = p.q_pos + static_cast<int64_t>(stream) * p.n_q;
    for (int i = 0; i < tiles && ok; ++i) {
      const int st = i % C::kRowStages;
      const int64_t at = (static_cast<int64_t>(lst) * p.row_tiles + first + i) * p.tile_rows;
      float lse[4];
      uint32_t lim[4], low = 0xffffffffu;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 32 * j + lane;
        const int token = (first + i) * p.tile_tokens + token_of[j];
        const bool in = r < p.tile_rows && token < p.n_q;
        lse[j] = in ? __ldcg(p.lse + at + r) : INFINITY;
        const int qp = in ? __ldg(q_pos + token) : -1;
        lim[j] = qp < 0 ? 0u : static_cast<uint32_t>(qp) + 1u;
        if (in) low = min(low, lim[j]);
      }
      low = __reduce_min_sync(0xffffffffu, low);
      ok = wait_warp(bar(C::kTFree + (i & 1)), ((i >> 1) & 1) ^ 1, p.err, ERR_WAIT_EPI);
      if (!ok) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        row_lse[st * kTile + 32 * j + lane] = -lse[j];
        row_lim[st * kTile + 32 * j + lane] = lim[j];
      }
      if (lane == 0) row_low[st] = low;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kTFull + (i & 1)));
    }
  } else if (warp < 8) {
    const int x = warp >> 2;
    const uint32_t col = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + 128u * x;
    // slot k of the four: lane 8 k + lane / 4 of the warp's quarter; an empty one's sum is not used
    uint32_t pos[4], top = 0;
    bool hole[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int slot = block * kTile + (warp & 3) * 32 + 8 * k + (lane >> 2);
      pos[k] = slot < p.used ? static_cast<uint32_t>(__ldg(p.pos + list_at + slot)) : 0xffffffffu;
      hole[k] = static_cast<int32_t>(pos[k]) < 0;
      top = max(top, hole[k] ? 0u : pos[k]);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    // (a per-thread copy: as a kernel parameter it cost the loops a fifth more instructions)
    const float c = __shfl_sync(0xffffffffu, p.scale_log2, 0);
    const uint64_t c2 = pack_f32x2(c, c);
    float totals[4] = {0.f, 0.f, 0.f, 0.f};
    bool ok = true;
    for (int i = x; i < tiles && ok; i += 2) {
      const int st = i % C::kRowStages;
      ok = wait_warp(bar(C::kTFull + x), (i >> 1) & 1, p.err, ERR_WAIT_MMA);
      if (!ok) break;
      tc_fence_after();
      uint32_t buf[2][2][8];  // a step of 16 rows ahead
      tmem_ld_16x256b_x2(col, buf[0][0]);
      tmem_ld_16x256b_x2(col + (16u << 16), buf[0][1]);
      uint64_t sum2[4] = {0, 0, 0, 0};  // even and odd rows
      float sum[4][2] = {};
      auto add = [&](auto masked) {
#pragma unroll
        for (int d = 0; d < kTile; d += 16) {
          uint32_t(&sr)[2][8] = buf[d / 16 % 2];  // slots 0 and 1, slots 2 and 3
          tmem_ld_wait();
          if (d + 16 < kTile) {
            tmem_ld_16x256b_x2(col + d + 16, buf[d / 16 % 2 ^ 1][0]);
            tmem_ld_16x256b_x2(col + (16u << 16) + d + 16, buf[d / 16 % 2 ^ 1][1]);
          } else {
            tc_fence_before();
            mbar_arrive(bar(C::kTFree + x));
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int at = st * kTile + d + 8 * j + 2 * (lane & 3);
            const uint64_t lse2 = *reinterpret_cast<const uint64_t*>(row_lse + at);  // negated
            uint2 lim;
            if constexpr (decltype(masked)::value) lim = *reinterpret_cast<const uint2*>(row_lim + at);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint64_t v;
              asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(sr[k / 2][4 * j + 2 * (k % 2)]),
                  "r"(sr[k / 2][4 * j + 2 * (k % 2) + 1]));
              asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(v), "l"(c2), "l"(lse2));
              float e0, e1;
              asm("mov.b64 {%0, %1}, %2;" : "=f"(e0), "=f"(e1) : "l"(v));
              e0 = ex2_approx(e0);
              e1 = ex2_approx(e1);
              if constexpr (decltype(masked)::value) {
                // (as predicated sums: with selects the integer pipe was the busiest)
                add_if_less(sum[k][0], e0, pos[k], lim.x);
                add_if_less(sum[k][1], e1, pos[k], lim.y);
              } else {
                asm("add.rn.f32x2 %0, %0, %1;" : "+l"(sum2[k]) : "l"(pack_f32x2(e0, e1)));
              }
            }
          }
        }
      };
      if (top < row_low[st]) add(std::false_type{});
      else add(std::true_type{});
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float s0, s1;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(s0), "=f"(s1) : "l"(sum2[k]));
        totals[k] += (s0 + sum[k][0]) + (s1 + sum[k][1]);
      }
    }
    // the four threads of a slot have shared out the rows; thread t keeps slot t % 4
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      totals[k] += __shfl_xor_sync(0xffffffffu, totals[k], 1);
      totals[k] += __shfl_xor_sync(0xffffffffu, totals[k], 2);
      if ((lane & 3) == k) total = hole[k] ? 0.f : totals[k];
    }
  }
  float* sums = reinterpret_cast<float*>(smem + C::kOffSum);
  if (warp >= 4 && warp < 8) sums[(warp & 3) * 32 + lane] = total;
  grid_dep_launch();
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, 256);
  }
  if (warp < 4 && key < p.used) {
    total += sums[warp * 32 + lane];
    if (p.row_splits > 1)
      p.part_w[(static_cast<int64_t>(split) * p.lists + lst) * p.used + key] = total;
    else
      p.weight_out[list_at + key] = fmaf(p.decay, p.weight[list_at + key], total);
  }
}

// The row splits' sums, in their order. (As a cluster whose first CTA adds up the others' sums out
// of their shared memory, weigh took 45 us for the 480p chunk: its CTAs only start when there is
// room for all three. Apart it takes 34, and this 6.)
__global__ void __launch_bounds__(256) sum_weights_kernel(const __grid_constant__ CacheAttn p) {
  const int64_t n = static_cast<int64_t>(p.lists) * p.used;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t lst = i / p.used, at = lst * p.capacity + (i - lst * p.used);
  grid_dep_wait();
  if (i < n) {
    float w = 0.f;
    for (int s = 0; s < p.row_splits; ++s) w += __ldcg(p.part_w + s * n + i);
    p.weight_out[at] = fmaf(p.decay, p.weight[at], w);
  }
  grid_dep_launch();
}

bool make_map(CUtensorMap* m, bool f16, const void* base, uint64_t d0, uint64_t d1, uint64_t d2,
              uint64_t d3, int64_t s1, int64_t s2, int64_t s3, uint32_t b1, uint32_t b2) {
  // a dimension of one entry never steps: its stride only has to be one that a map may have
  const uint64_t dims[4] = {d0, d1, d2, d3};
  const uint64_t strides[3] = {d1 > 1 ? static_cast<uint64_t>(s1) * 2 : 2 * d0,
                               d2 > 1 ? static_cast<uint64_t>(s2) * 2 : 2 * d0,
                               d3 > 1 ? static_cast<uint64_t>(s3) * 2 : 2 * d0};
  return tmap_16bit_4d(m, f16, base, dims, strides, b1, b2);
}

template <bool F16, int D>
cudaError_t launch_t(const CacheAttn& p, const fd_cache* c, cudaStream_t s) {
  using A = AttendCfg<D>;
  using W = WeighCfg<D>;
  int device = -1;
  if (const cudaError_t e = cudaGetDevice(&device); e != cudaSuccess) return e;
  static OncePerDevice smem;
  const cudaError_t attr = smem.run(device, [] {
    const cudaError_t e = cudaFuncSetAttribute(
        attend_kernel<F16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, A::kSmem);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(weigh_kernel<F16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                W::kSmem);
  });
  if (attr != cudaSuccess) return attr;
  CUtensorMap tq, tk, tv;
  if (!make_map(&tq, F16, p.q, D, p.heads, p.n_q, c->streams, p.q_head, p.q_token, p.q_stream,
                p.per, p.tile_tokens) ||
      !make_map(&tk, F16, p.k, D, p.used, p.groups, c->streams, p.slot_stride, p.group_stride,
                p.stream_stride, kTile, 1) ||
      !make_map(&tv, F16, p.v, D, p.used, p.groups, c->streams, p.slot_stride, p.group_stride,
                p.stream_stride, kTile, 1))
    return cudaErrorInvalidValue;
  cudaError_t e = launch_pdl(attend_kernel<F16, D>, dim3(p.parts), dim3(A::kThreads), A::kSmem, s,
                             tq, tk, tv, p);
  if (e == cudaSuccess && p.parts > 1)
    e = launch_pdl(join_parts_kernel<F16, D>, dim3(p.parts - 1, D / 4), dim3(kTile), 0, s, p);
  if (e != cudaSuccess || p.weight_out == nullptr) return e;
  e = launch_pdl(weigh_kernel<F16, D>, dim3(p.key_tiles, p.row_splits, p.lists), dim3(W::kThreads),
                 W::kSmem, s, tq, tk, p);
  if (e != cudaSuccess || p.row_splits == 1) return e;
  const int64_t n = static_cast<int64_t>(p.lists) * p.used;
  return launch_pdl(sum_weights_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0,
                    s, p);
}

}  // namespace

bool chunk_form(int rows, int used) { return rows > kMaxRows && used > 0; }

ChunkPlan chunk_plan(const fd_cache* c, int used, int per, int n_q) {
  ChunkPlan y{};
  const int64_t lists = static_cast<int64_t>(c->streams) * c->groups;
  y.tile_tokens = std::min(kTile / per, n_q);
  y.tile_rows = y.tile_tokens * per;
  y.row_tiles = (n_q + y.tile_tokens - 1) / y.tile_tokens;
  y.key_tiles = (used + kTile - 1) / kTile;
  y.attend_blocks = (used + 255) / 256;
  const int64_t units = lists * y.row_tiles * y.attend_blocks;
  // a CTA for every SM, of a block at least (100 queries of 16 heads over 1000 slots: 15 us; with
  // CTAs of 2 blocks at least 16, of 8 at least 27)
  y.parts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kSms, units)));
  // row splits: the fewest waves of two CTAs an SM, counted in tiles one after the other (480p
  // chunk: 3 splits 95 us, none 103; prompt of 2 x 2001 queries over 8191 slots: 2 or none the same)
  const int64_t ctas = lists * y.key_tiles;
  int64_t best = INT64_MAX;
  for (int r = 1; r <= 8 && r <= y.row_tiles; ++r) {
    const int64_t waves = (ctas * r + 2 * kSms - 1) / (2 * kSms);
    const int64_t cost = waves * ((y.row_tiles + r - 1) / r + 3) + (r > 1 ? 2 : 0);
    if (cost < best) {
      best = cost;
      y.row_splits = r;
    }
  }
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t at = 0;
  y.ml = at;
  at += up(static_cast<size_t>(y.parts) * 2 * kTile * 8);
  y.o = at;
  at += up(static_cast<size_t>(y.parts) * 2 * kTile * c->head_dim * 4);
  y.lse = at;
  at += up(static_cast<size_t>(lists) * y.row_tiles * y.tile_rows * 4);
  y.w = at;
  if (y.row_splits > 1) at += up(static_cast<size_t>(y.row_splits) * lists * used * 4);
  y.total = at;
  return y;
}

cudaError_t launch_chunk_wait_check(int which, int* err, cudaStream_t s) {
  wait_check_kernel<<<1, 32, 0, s>>>(which, err);
  return cudaGetLastError();
}

cudaError_t launch_chunk(const CacheAttn& p, const fd_cache* c, cudaStream_t s) {
  const bool f16 = c->dtype == FD_DTYPE_F16;
  if (c->head_dim == 64) return f16 ? launch_t<true, 64>(p, c, s) : launch_t<false, 64>(p, c, s);
  return f16 ? launch_t<true, 128>(p, c, s) : launch_t<false, 128>(p, c, s);
}

}  // namespace fd
