// Attention over a bounded cache, many rows (a chunk's or a prompt's queries): tensor cores, two
// passes over the scores.
//
//   attend   out = softmax(c q k^T) v by blocks of 128 slots with a running maximum and sum, and each
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
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
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

constexpr int kTile = 128;      // rows of a tile, slots of a block
constexpr int kSub = kTile * 128;  // bytes of 64 elements of 128 rows: one swizzled sub-tile

// ------------------------------------------------------------------------------ attend
//
// Persistent CTAs (one per SM), each with an equal run of the (tile pair, block) units, pair
// after pair: a segment is a pair's consecutive blocks. A pair that is cut between CTAs leaves
// partial results, which join_parts adds up in the order of the blocks.
//
// Per CTA two tiles, so that one tile's exponentials run while the tensor cores work for the other:
//   warps 0-3 / 4-7   softmax of tile 0 / 1, a row (TMEM lane) per thread
//   warp 8            TMA: Q of the segment, K and V blocks into a ring
//   warps 9 / 10      issue tile 0's / tile 1's products
//   warp 11           positions of each block, and zeros for the values of empty slots (their
//                     probability is 0, but 0 times NaN is NaN)
// TMEM (512 columns): S 2 x 128, O 2 x D, P (two 16-bit values a column) 2 x 64: for D = 64 beside S,
// for D = 128 over the first half of its own S, which then takes the next scores only
// after P V.
template <int D>
struct AttendCfg {
  static constexpr bool kAlias = D == 128;
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kSlots = D == 128 ? 4 : 8;  // ring of K, V, K, V, ..
  static constexpr int kPosStages = 4;
  static constexpr int kOffRing = 2 * kTileBytes;  // after the two Q tiles
  static constexpr int kOffPos = kOffRing + kSlots * kTileBytes;
  static constexpr int kOffTop = kOffPos + kPosStages * kTile * 4;  // largest position per stage
  static constexpr int kOffBar = kOffTop + 64;
  static constexpr int kSmem = kOffBar + 512;
  static constexpr int kThreads = 384;
  static constexpr uint32_t kColS = 0, kColP = kAlias ? 0 : 256, kColO = kAlias ? 256 : 384;
  static constexpr uint32_t kStepP = kAlias ? 128 : 64;
  // barriers
  static constexpr int kQFull = 0, kQFree = 1, kKvFull = 2, kKvFree = kKvFull + kSlots,
                       kVReady = kKvFree + kSlots, kSFull = kVReady + kSlots,
                       kSRead = kSFull + 2, kPFull = kSRead + 2, kPv = kPFull + 2,
                       kORead = kPv + 2, kPosFull = kORead + 2, kPosFree = kPosFull + kPosStages,
                       kDone = kPosFree + kPosStages, kBars = kDone + 2;
  static_assert(kBars * 8 + 8 <= 512, "barriers");
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
  int64_t pair;
  int block, left, seg;  // left: units after this one
  bool first, last;      // of its segment
  __device__ Walk(const Units& w, int cta, int blocks) {
    const int64_t u = w.start(cta);
    left = static_cast<int>(w.start(cta + 1) - u) - 1;
    pair = u / blocks;
    block = static_cast<int>(u - pair * blocks);
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
      ++pair;
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
  int32_t* pos_ring = reinterpret_cast<int32_t*>(smem + C::kOffPos);
  uint32_t* pos_top = reinterpret_cast<uint32_t*>(smem + C::kOffTop);
  const int blocks = p.key_tiles;
  const int pairs_list = (p.row_tiles + 1) / 2;
  const Units units{static_cast<int64_t>(p.lists) * pairs_list * blocks, p.parts};

  // rows past tile_rows are never loaded
  for (int i = threadIdx.x; i < 2 * C::kTileBytes / 16; i += C::kThreads)
    reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  if (threadIdx.x == 0) {
    if (!aligned) atomicOr(p.err, ERR_SMEM_ALIGN);
    mbar_init(bar(C::kQFull), 1);
    mbar_init(bar(C::kQFree), 2);
    for (int i = 0; i < C::kSlots; ++i) {
      mbar_init(bar(C::kKvFull + i), 1);
      mbar_init(bar(C::kKvFree + i), 2);
      mbar_init(bar(C::kVReady + i), 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(bar(C::kSFull + x), 1);
      mbar_init(bar(C::kSRead + x), 128);
      mbar_init(bar(C::kPFull + x), 128);
      mbar_init(bar(C::kPv + x), 1);
      mbar_init(bar(C::kORead + x), 128);
      mbar_init(bar(C::kDone + x), 1);
    }
    for (int i = 0; i < C::kPosStages; ++i) {
      mbar_init(bar(C::kPosFull + i), 1);
      mbar_init(bar(C::kPosFree + i), 8);
    }
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

  // tile x of a pair holds rows (an odd number of tiles leaves the last pair's second one empty)
  auto has_tile = [&](int64_t pair, int x) {
    return static_cast<int>(pair % pairs_list) * 2 + x < p.row_tiles;
  };
  if (!aligned) {
    // nothing is loaded or computed; the status word says why
  } else if (warp == 8) {
    if (lane == 0) {
      prefetch_tmap(&tmQ);
      prefetch_tmap(&tmK);
      prefetch_tmap(&tmV);
      int J = 0, segs = 0;
      bool ok = true;
      for (Walk w(units, blockIdx.x, blocks); w.valid() && ok; w.next(blocks), ++J) {
        const int lst = static_cast<int>(w.pair / pairs_list);
        const int stream = lst / p.groups, group = lst - stream * p.groups;
        if (w.first) {
          if (w.seg > 0 && !mbar_wait(bar(C::kQFree), (w.seg - 1) & 1, p.err, ERR_WAIT_MMA)) break;
          const int n = 1 + has_tile(w.pair, 1);
          mbar_expect_tx(bar(C::kQFull), n * p.tile_rows * D * 2);
          for (int x = 0; x < n; ++x)
            for (int d = 0; d < D / 64; ++d)
              tma_load_4d(base + x * C::kTileBytes + d * kSub, &tmQ, bar(C::kQFull), 64 * d,
                          group * p.per,
                          (static_cast<int>(w.pair % pairs_list) * 2 + x) * p.tile_tokens, stream);
          segs = w.seg + 1;
        }
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const int i = 2 * J + kv, s = i % C::kSlots;
          if (!mbar_wait(bar(C::kKvFree + s), ((i / C::kSlots) & 1) ^ 1, p.err, ERR_WAIT_MMA)) {
            ok = false;
            break;
          }
          mbar_expect_tx(bar(C::kKvFull + s), C::kTileBytes);
          for (int d = 0; d < D / 64; ++d)
            tma_load_4d(base + C::kOffRing + s * C::kTileBytes + d * kSub, kv ? &tmV : &tmK,
                        bar(C::kKvFull + s), 64 * d, w.block * kTile, group, stream);
        }
        if (!ok) {  // a K without its V: wait for what was started
          const int i = 2 * J, s = i % C::kSlots;
          mbar_wait(bar(C::kKvFull + s), (i / C::kSlots) & 1, p.err, ERR_WAIT_TMA);
        }
      }
      // nothing may be in flight when the CTA exits
      if (segs > 0) mbar_wait(bar(C::kQFull), (segs - 1) & 1, p.err, ERR_WAIT_TMA);
      for (int i = 2 * J - 1; i >= 0 && i >= 2 * J - C::kSlots; --i)
        mbar_wait(bar(C::kKvFull + i % C::kSlots), (i / C::kSlots) & 1, p.err, ERR_WAIT_TMA);
    }
  } else if (warp == 11) {
    // ---- positions and empty slots' values
    int J = 0;
    bool ok = true;
    for (Walk w(units, blockIdx.x, blocks); w.valid() && ok; w.next(blocks), ++J) {
      const int lst = static_cast<int>(w.pair / pairs_list);
      const int32_t* pos = p.pos + static_cast<int64_t>(lst) * p.capacity;
      int32_t v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int slot = w.block * kTile + 32 * i + lane;
        v[i] = slot < p.used ? __ldg(pos + slot) : -1;
      }
      const int st = J % C::kPosStages;
      ok = mbar_wait_warp(bar(C::kPosFree + st), ((J / C::kPosStages) & 1) ^ 1, p.err, ERR_WAIT_EPI);
      if (!ok) break;
      uint32_t top = 0;
      bool hole = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pos_ring[st * kTile + 32 * i + lane] = v[i];
        top = max(top, static_cast<uint32_t>(v[i]));
        hole |= v[i] < 0 && w.block * kTile + 32 * i + lane < p.used;
      }
      top = __reduce_max_sync(0xffffffffu, top);
      if (lane == 0) pos_top[st] = top;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kPosFull + st));
      const int i = 2 * J + 1, s = i % C::kSlots;
      ok = mbar_wait_warp(bar(C::kKvFull + s), (i / C::kSlots) & 1, p.err, ERR_WAIT_TMA);
      if (!ok) break;
      if (__any_sync(0xffffffffu, hole)) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (v[r] >= 0) continue;
          uint4* row = reinterpret_cast<uint4*>(smem + C::kOffRing + s * C::kTileBytes +
                                                (32 * r + lane) * 128);
#pragma unroll
          for (int d = 0; d < D / 64; ++d)
#pragma unroll
            for (int c = 0; c < 8; ++c) row[d * (kSub / 16) + c] = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kVReady + s));
    }
  } else if (warp >= 9) {
    // ---- products of tile x
    const int x = warp - 9;
    if (lane == 0) {
      constexpr uint32_t is = Mma<F16, D>::idesc(kTile, false), io = Mma<F16, D>::idesc(D, true);
      const uint32_t s_col = tmem + C::kColS + 128u * x;
      const uint32_t p_col = tmem + C::kColP + C::kStepP * x;
      const uint32_t o_col = tmem + C::kColO + static_cast<uint32_t>(D) * x;
      const uint64_t q0 = sdesc_k_sw128(base + x * C::kTileBytes);
      // scores of the walk's block (number J); leaves the K slot
      auto scores = [&](const Walk& w, int J) -> bool {
        if (w.first && !mbar_wait(bar(C::kQFull), w.seg & 1, p.err, ERR_WAIT_TMA)) return false;
        const int i = 2 * J, s = i % C::kSlots;
        if (!mbar_wait(bar(C::kKvFull + s), (i / C::kSlots) & 1, p.err, ERR_WAIT_TMA)) return false;
        if (!has_tile(w.pair, x)) {
          mbar_arrive(bar(C::kKvFree + s));
          if (w.last) mbar_arrive(bar(C::kQFree));
          return true;
        }
        tc_fence_after();
        const uint64_t k0 = sdesc_k_sw128(base + C::kOffRing + s * C::kTileBytes);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          const uint64_t at = static_cast<uint64_t>((d / 4) * (kSub >> 4) + (d % 4) * 2);
          mma_ss(s_col, q0 + at, k0 + at, is, d > 0);
        }
        mma_commit(bar(C::kSFull + x));
        mma_commit(bar(C::kKvFree + s));
        if (w.last) mma_commit(bar(C::kQFree));
        return true;
      };
      Walk w(units, blockIdx.x, blocks);
      // T: blocks of this tile so far, the phase of its own barriers (a pair without this tile
      // has none), E: segments that it has had
      int J = 0, T = 0, E = 0;
      bool ok = !w.valid() || scores(w, 0);
      for (; w.valid() && ok; ++J) {
        const Walk here = w;
        const bool mine = has_tile(here.pair, x);
        w.next(blocks);
        if (!C::kAlias && w.valid()) {
          // S is free once the softmax has read it
          if (mine) ok = mbar_wait(bar(C::kSRead + x), T & 1, p.err, ERR_WAIT_EPI);
          ok = ok && scores(w, J + 1);
          if (!ok) break;
        }
        const int i = 2 * J + 1, s = i % C::kSlots;
        ok = mbar_wait(bar(C::kVReady + s), (i / C::kSlots) & 1, p.err, ERR_WAIT_TMA);
        if (!ok) break;
        if (mine) {
          ok = mbar_wait(bar(C::kPFull + x), T & 1, p.err, ERR_WAIT_EPI);
          // the first product of a segment overwrites O
          if (ok && here.first && E > 0)
            ok = mbar_wait(bar(C::kORead + x), (E - 1) & 1, p.err, ERR_WAIT_EPI);
          if (!ok) break;
          tc_fence_after();
          const uint64_t v0 = sdesc_mn_sw128(base + C::kOffRing + s * C::kTileBytes, kSub);
#pragma unroll
          for (int k = 0; k < kTile / 16; ++k)
            mma_ts(o_col, p_col + 8u * k, v0 + static_cast<uint64_t>(k * (2048 >> 4)), io,
                   !here.first || k > 0);
          mma_commit(bar(C::kPv + x));
          mma_commit(bar(C::kKvFree + s));
          if (here.last) ++E;
          if (C::kAlias) ok = mbar_wait(bar(C::kPv + x), T & 1, p.err, ERR_WAIT_MMA);
          ++T;
        } else {
          mbar_arrive(bar(C::kKvFree + s));
        }
        if (C::kAlias && ok && w.valid()) ok = scores(w, J + 1);
      }
      mma_commit(bar(C::kDone + x));
      mbar_wait(bar(C::kDone + x), 0, p.err, ERR_WAIT_MMA);
    }
  } else {
    // ---- softmax of tile x
    const int x = warp >> 2, quarter = warp & 3;
    const int row = quarter * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t s_col = tmem + lane_off + C::kColS + 128u * x;
    const uint32_t p_col = tmem + lane_off + C::kColP + C::kStepP * x;
    const uint32_t o_col = tmem + lane_off + C::kColO + static_cast<uint32_t>(D) * x;
    const float c = p.scale_log2;
    float m = -INFINITY, l = 0.f;
    uint32_t limit = 0;  // a slot is visible if its position, unsigned, is below this
    int J = 0, T = 0;
    bool ok = true;
    for (Walk w(units, blockIdx.x, blocks); w.valid() && ok; w.next(blocks), ++J) {
      const int st = J % C::kPosStages;
      ok = mbar_wait_warp(bar(C::kPosFull + st), (J / C::kPosStages) & 1, p.err, ERR_WAIT_EPI);
      if (!ok) break;
      if (!has_tile(w.pair, x)) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::kPosFree + st));
        continue;
      }
      const int lst = static_cast<int>(w.pair / pairs_list);
      const int stream = lst / p.groups, group = lst - stream * p.groups;
      const int tile = static_cast<int>(w.pair % pairs_list) * 2 + x;
      const int token = tile * p.tile_tokens + row / p.per;
      const bool valid = row < p.tile_rows && token < p.n_q;
      if (w.first) {
        m = -INFINITY;
        l = 0.f;
        // (rows that are none see every entry: their results go nowhere, and they do not send the
        // warp through the masked path)
        const int qp = valid ? __ldg(p.q_pos + static_cast<int64_t>(stream) * p.n_q + token)
                             : 0x7fffffff;
        limit = qp < 0 ? 0u : static_cast<uint32_t>(qp) + 1u;
      }
      ok = mbar_wait_warp(bar(C::kSFull + x), T & 1, p.err, ERR_WAIT_MMA);
      if (!ok) break;
      tc_fence_after();
      uint32_t sr[4][32];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_ld_32x32b_x32(s_col + 32 * i, sr[i]);
      tmem_ld_wait();
      if (!C::kAlias) {
        tc_fence_before();
        mbar_arrive(bar(C::kSRead + x));
      }
      if (p.flip != 1.f) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            sr[i][e] = __float_as_uint(__uint_as_float(sr[i][e]) * p.flip);
      }
      if (!__all_sync(0xffffffffu, pos_top[st] < limit)) {
        const int4* ps = reinterpret_cast<const int4*>(pos_ring + st * kTile);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const int4 v = ps[8 * i + e / 4];
            if (static_cast<uint32_t>(v.x) >= limit) sr[i][e] = 0xff800000u;
            if (static_cast<uint32_t>(v.y) >= limit) sr[i][e + 1] = 0xff800000u;
            if (static_cast<uint32_t>(v.z) >= limit) sr[i][e + 2] = 0xff800000u;
            if (static_cast<uint32_t>(v.w) >= limit) sr[i][e + 3] = 0xff800000u;
          }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kPosFree + st));
      float mx[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mx[i] = __uint_as_float(sr[i][0]);
#pragma unroll
        for (int e = 1; e < 31; e += 2)
          mx[i] = fmax3(mx[i], __uint_as_float(sr[i][e]), __uint_as_float(sr[i][e + 1]));
        mx[i] = fmaxf(mx[i], __uint_as_float(sr[i][31]));
      }
      const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c;
      const bool grow = top > m + kSlack;
      const float now = grow ? top : m;
      const float off = now == -INFINITY ? 0.f : now;
      // O and P: the previous block's product is done
      if (!w.first) {
        ok = mbar_wait_warp(bar(C::kPv + x), (T - 1) & 1, p.err, ERR_WAIT_MMA);
        if (!ok) break;
        tc_fence_after();
        if (__any_sync(0xffffffffu, grow)) {
          const float f = grow ? ex2_approx(m - off) : 1.f;
          l *= f;
#pragma unroll 1
          for (int d = 0; d < D; d += 16) {
            uint32_t o[16];
            tmem_ld_32x32b_x16(o_col + d, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tmem_st_32x32b_x16(o_col + d, o);
          }
        }
      }
      m = now;
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t pk[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float a = ex2_approx(fmaf(__uint_as_float(sr[i][e]), c, -off));
          const float b = ex2_approx(fmaf(__uint_as_float(sr[i][e + 1]), c, -off));
          sum[e / 2 % 2] += a;
          sum[2 + e / 2 % 2] += b;
          pk[e / 2] = pack16<F16>(a, b);
        }
        tmem_st_32x32b_x16(p_col + 16 * i, pk);
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(bar(C::kPFull + x));
      ++T;
      if (!w.last) continue;

      // ---- the segment's result
      ok = mbar_wait_warp(bar(C::kPv + x), (T - 1) & 1, p.err, ERR_WAIT_MMA);
      if (!ok) break;
      tc_fence_after();
      const int lo = units.owner(w.pair * blocks), hi = units.owner(w.pair * blocks + blocks - 1);
      const bool whole = lo == hi;
      // a cut pair's part: the CTA's first segment (slot 0) unless the pair began in this CTA
      const int slot = units.start(blockIdx.x) > w.pair * blocks ? 0 : 1;
      const int64_t part = (static_cast<int64_t>(blockIdx.x) * 2 + slot) * 2 + x;
      const float inv = l > 0.f ? 1.f / l : 0.f;
      using T16 = uint16_t;
      T16* out = static_cast<T16*>(p.out) + stream * p.out_stream +
                 static_cast<int64_t>(token) * p.out_token +
                 static_cast<int64_t>(group * p.per + row % p.per) * p.out_head;
#pragma unroll
      for (int d = 0; d < D; d += 32) {
        uint32_t o[32];
        __syncwarp();
        tmem_ld_32x32b_x32(o_col + d, o);
        tmem_ld_wait();
        if (whole && valid) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
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
          for (int e = 0; e < 32; e += 4)
            po[(d + e) / 4 * kTile] = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
      }
      tc_fence_before();
      mbar_arrive(bar(C::kORead + x));
      if (!whole) {
        p.part_ml[part * kTile + row] = make_float2(m, l);
      } else if (row < p.tile_rows) {
        p.lse[(static_cast<int64_t>(lst) * p.row_tiles + tile) * p.tile_rows + row] =
            valid && l > 0.f ? m + log2f(l) : INFINITY;
      }
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

// The cut pairs' parts added up: blockIdx.x = (pair, tile of it), blockIdx.y = 4 elements of the
// head, a thread per row.
template <bool F16, int D>
__global__ void __launch_bounds__(kTile) join_parts_kernel(const __grid_constant__ CacheAttn p) {
  grid_dep_wait();
  const int blocks = p.key_tiles, pairs_list = (p.row_tiles + 1) / 2;
  const Units units{static_cast<int64_t>(p.lists) * pairs_list * blocks, p.parts};
  const int64_t pair = blockIdx.x >> 1;
  const int x = blockIdx.x & 1, k = blockIdx.y, row = threadIdx.x;
  const int lst = static_cast<int>(pair / pairs_list);
  const int tile = static_cast<int>(pair % pairs_list) * 2 + x;
  const int lo = units.owner(pair * blocks), hi = units.owner(pair * blocks + blocks - 1);
  if (lo != hi && tile < p.row_tiles) {
    auto part_of = [&](int c) {
      return (static_cast<int64_t>(c) * 2 + (units.start(c) > pair * blocks ? 0 : 1)) * 2 + x;
    };
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
    const float inv = l > 0.f ? 1.f / l : 0.f;
    if (valid) {
      uint16_t* out = static_cast<uint16_t*>(p.out) + stream * p.out_stream +
                      static_cast<int64_t>(token) * p.out_token +
                      static_cast<int64_t>(group * p.per + row % p.per) * p.out_head + 4 * k;
      *reinterpret_cast<uint2*>(out) = make_uint2(pack16<F16>(acc.x * inv, acc.y * inv),
                                                  pack16<F16>(acc.z * inv, acc.w * inv));
    }
    if (k == 0 && row < p.tile_rows)
      p.lse[(static_cast<int64_t>(lst) * p.row_tiles + tile) * p.tile_rows + row] =
          valid && l > 0.f ? top + log2f(l) : INFINITY;
  }
  grid_dep_launch();
}

// ------------------------------------------------------------------------------ weigh
//
// A CTA has one block of 128 slots of one list and a run of the list's row tiles: S^T = K Q^T, K
// from shared memory all along, Q tiles through a ring. A thread has one slot (TMEM lane) and
// adds exp2(c s - lse_r) over the tile's rows; two groups of warps take the tiles in turn, each
// with its own accumulator in TMEM. Two CTAs fit an SM.
//   warps 0-3 / 4-7  even / odd tiles   warp 8  TMA   warp 9  products   warp 10  lse and limits
template <int D>
struct WeighCfg {
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kStages = D == 128 ? 2 : 4;
  static constexpr int kRowStages = 4;
  static constexpr int kOffQ = kTileBytes;
  static constexpr int kOffRows = kOffQ + kStages * kTileBytes;    // lse, then limits, per stage
  static constexpr int kOffLow = kOffRows + kRowStages * kTile * 8;  // smallest limit per stage
  static constexpr int kOffSum = kOffLow + 64;                       // one group's sums
  static constexpr int kOffBar = kOffSum + kTile * 4;
  static constexpr int kSmem = kOffBar + 256;
  static constexpr int kThreads = 352;
  static constexpr int kKFull = 0, kQFull = 1, kQFree = kQFull + kStages,
                       kTFull = kQFree + kStages, kTFree = kTFull + 2, kRowFull = kTFree + 2,
                       kRowFree = kRowFull + kRowStages, kDone = kRowFree + kRowStages,
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
      mbar_init(bar(C::kTFull + x), 1);
      mbar_init(bar(C::kTFree + x), 128);
    }
    for (int i = 0; i < C::kRowStages; ++i) {
      mbar_init(bar(C::kRowFull + i), 1);
      mbar_init(bar(C::kRowFree + i), 4);
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

  float total = 0.f;
  const int key = block * kTile + (warp & 3) * 32 + lane;
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
        if (!mbar_wait(bar(C::kQFree + s), ((i / C::kStages) & 1) ^ 1, p.err, ERR_WAIT_MMA)) break;
        mbar_expect_tx(bar(C::kQFull + s), p.tile_rows * D * 2);
        for (int d = 0; d < D / 64; ++d)
          tma_load_4d(base + C::kOffQ + s * C::kTileBytes + d * kSub, &tmQ, bar(C::kQFull + s),
                      64 * d, group * p.per, (first + i) * p.tile_tokens, stream);
      }
      mbar_wait(bar(C::kKFull), 0, p.err, ERR_WAIT_TMA);
      for (int j = i - 1; j >= 0 && j >= i - C::kStages; --j)
        mbar_wait(bar(C::kQFull + j % C::kStages), (j / C::kStages) & 1, p.err, ERR_WAIT_TMA);
    }
  } else if (warp == 9) {
    if (lane == 0) {
      constexpr uint32_t idesc = Mma<F16, D>::idesc(kTile, false);
      const uint64_t k0 = sdesc_k_sw128(base);
      bool ok = mbar_wait(bar(C::kKFull), 0, p.err, ERR_WAIT_TMA);
      for (int i = 0; i < tiles && ok; ++i) {
        const int s = i % C::kStages, x = i & 1;
        ok = mbar_wait(bar(C::kTFree + x), ((i >> 1) & 1) ^ 1, p.err, ERR_WAIT_EPI) &&
             mbar_wait(bar(C::kQFull + s), (i / C::kStages) & 1, p.err, ERR_WAIT_TMA);
        if (!ok) break;
        tc_fence_after();
        const uint64_t q0 = sdesc_k_sw128(base + C::kOffQ + s * C::kTileBytes);
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          const uint64_t at = static_cast<uint64_t>((d / 4) * (kSub >> 4) + (d % 4) * 2);
          mma_ss(tmem + 128u * x, k0 + at, q0 + at, idesc, d > 0);
        }
        mma_commit(bar(C::kTFull + x));
        mma_commit(bar(C::kQFree + s));
      }
      mma_commit(bar(C::kDone));
      mbar_wait(bar(C::kDone), 0, p.err, ERR_WAIT_MMA);
    }
  } else if (warp == 10) {
    bool ok = true;
    for (int i = 0; i < tiles && ok; ++i) {
      const int st = i % C::kRowStages;
      const int64_t at = (static_cast<int64_t>(lst) * p.row_tiles + first + i) * p.tile_rows;
      float lse[4];
      uint32_t lim[4], low = 0xffffffffu;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 32 * j + lane;
        const int token = (first + i) * p.tile_tokens + r / p.per;
        const bool in = r < p.tile_rows && token < p.n_q;
        lse[j] = in ? __ldcg(p.lse + at + r) : INFINITY;
        const int qp = in ? __ldg(p.q_pos + static_cast<int64_t>(stream) * p.n_q + token) : -1;
        lim[j] = qp < 0 ? 0u : static_cast<uint32_t>(qp) + 1u;
        if (in) low = min(low, lim[j]);
      }
      low = __reduce_min_sync(0xffffffffu, low);
      ok = mbar_wait_warp(bar(C::kRowFree + st), ((i / C::kRowStages) & 1) ^ 1, p.err, ERR_WAIT_EPI);
      if (!ok) break;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        row_lse[st * kTile + 32 * j + lane] = lse[j];
        row_lim[st * kTile + 32 * j + lane] = lim[j];
      }
      if (lane == 0) row_low[st] = low;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kRowFull + st));
    }
  } else if (warp < 8) {
    const int x = warp >> 2;
    const uint32_t col = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + 128u * x;
    const uint32_t pos =
        key < p.used ? static_cast<uint32_t>(__ldg(p.pos + list_at + key)) : 0xffffffffu;
    const float c = p.scale_log2 * p.flip;  // flip 0: every score is 0
    bool ok = true;
    for (int i = x; i < tiles && ok; i += 2) {
      const int st = i % C::kRowStages;
      ok = mbar_wait_warp(bar(C::kRowFull + st), (i / C::kRowStages) & 1, p.err, ERR_WAIT_EPI) &&
           mbar_wait_warp(bar(C::kTFull + x), (i >> 1) & 1, p.err, ERR_WAIT_MMA);
      if (!ok) break;
      tc_fence_after();
      // an empty slot's sum is not used, so it does not matter here
      const bool all = __all_sync(0xffffffffu, pos < row_low[st] || static_cast<int32_t>(pos) < 0);
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < kTile; d += 32) {
        uint32_t sr[32];
        tmem_ld_32x32b_x32(col + d, sr);
        tmem_ld_wait();
        if (d == kTile - 32) {
          tc_fence_before();
          mbar_arrive(bar(C::kTFree + x));
        }
        const float4* ls = reinterpret_cast<const float4*>(row_lse + st * kTile + d);
        if (all) {
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float4 v = ls[e / 4];
            sum[0] += ex2_approx(fmaf(__uint_as_float(sr[e]), c, -v.x));
            sum[1] += ex2_approx(fmaf(__uint_as_float(sr[e + 1]), c, -v.y));
            sum[2] += ex2_approx(fmaf(__uint_as_float(sr[e + 2]), c, -v.z));
            sum[3] += ex2_approx(fmaf(__uint_as_float(sr[e + 3]), c, -v.w));
          }
        } else {
          const uint4* lm = reinterpret_cast<const uint4*>(row_lim + st * kTile + d);
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float4 v = ls[e / 4];
            const uint4 b = lm[e / 4];
            if (pos < b.x) sum[0] += ex2_approx(fmaf(__uint_as_float(sr[e]), c, -v.x));
            if (pos < b.y) sum[1] += ex2_approx(fmaf(__uint_as_float(sr[e + 1]), c, -v.y));
            if (pos < b.z) sum[2] += ex2_approx(fmaf(__uint_as_float(sr[e + 2]), c, -v.z));
            if (pos < b.w) sum[3] += ex2_approx(fmaf(__uint_as_float(sr[e + 3]), c, -v.w));
          }
        }
      }
      total += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kRowFree + st));
    }
    if (static_cast<int32_t>(pos) < 0) total = 0.f;
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

// the row splits' sums, in their order
__global__ void __launch_bounds__(256) sum_weights_kernel(const __grid_constant__ CacheAttn p) {
  grid_dep_wait();
  const int64_t n = static_cast<int64_t>(p.lists) * p.used;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i < n) {
    const int64_t lst = i / p.used, at = lst * p.capacity + (i - lst * p.used);
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
  static const cudaError_t attr = [] {
    const cudaError_t e = cudaFuncSetAttribute(
        attend_kernel<F16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, A::kSmem);
    if (e != cudaSuccess) return e;
    return cudaFuncSetAttribute(weigh_kernel<F16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                W::kSmem);
  }();
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
  const int pairs = p.lists * ((p.row_tiles + 1) / 2);
  // the pairs fall on whole CTAs only if the units divide evenly
  if (e == cudaSuccess && p.parts > 1)
    e = launch_pdl(join_parts_kernel<F16, D>, dim3(2 * pairs, D / 4), dim3(kTile), 0, s, p);
  if (e != cudaSuccess || p.weight_out == nullptr) return e;
  e = launch_pdl(weigh_kernel<F16, D>, dim3(p.key_tiles, p.row_splits, p.lists), dim3(W::kThreads),
                 W::kSmem, s, tq, tk, p);
  if (e != cudaSuccess || p.row_splits == 1) return e;
  const int64_t n = static_cast<int64_t>(p.lists) * p.used;
  return launch_pdl(sum_weights_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0,
                    s, p);
}

}  // namespace

bool chunk_form(int rows, int used) { return rows > 32 && used > 0; }

ChunkPlan chunk_plan(const fd_cache* c, int used, int per, int n_q) {
  ChunkPlan y{};
  const int64_t lists = static_cast<int64_t>(c->streams) * c->groups;
  y.tile_tokens = std::min(kTile / per, n_q);
  y.tile_rows = y.tile_tokens * per;
  y.row_tiles = (n_q + y.tile_tokens - 1) / y.tile_tokens;
  y.key_tiles = (used + kTile - 1) / kTile;
  const int64_t units = lists * ((y.row_tiles + 1) / 2) * y.key_tiles;
  // a CTA for every SM, of 4 blocks at least: its fixed cost is about that of 2 blocks
  y.parts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kSms, units / 4)));
  // row splits: the fewest waves of two CTAs an SM, counted in tiles one after the other
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
  at += up(static_cast<size_t>(y.parts) * 4 * kTile * 8);
  y.o = at;
  at += up(static_cast<size_t>(y.parts) * 4 * kTile * c->head_dim * 4);
  y.lse = at;
  at += up(static_cast<size_t>(lists) * y.row_tiles * y.tile_rows * 4);
  y.w = at;
  if (y.row_splits > 1) at += up(static_cast<size_t>(y.row_splits) * lists * used * 4);
  y.total = at;
  return y;
}

cudaError_t launch_chunk(const CacheAttn& p, const fd_cache* c, cudaStream_t s) {
  const bool f16 = c->dtype == FD_DTYPE_F16;
  if (c->head_dim == 64) return f16 ? launch_t<true, 64>(p, c, s) : launch_t<false, 64>(p, c, s);
  return f16 ? launch_t<true, 128>(p, c, s) : launch_t<false, 128>(p, c, s);
}

}  // namespace fd
