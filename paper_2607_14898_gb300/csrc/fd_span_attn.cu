// Attention in which every query sees a span of keys, forward (fd_op_span_attention):
//   s = scale q k^T within the span, lse = log sum exp s, out = exp(s - lse) v
// by blocks of 128 keys with a running maximum and sum, kept in fp32 with O in TMEM.
//
// Bound by the chain from a block's scores through their softmax to the product that waits for it, and by
// the softmax's instructions: heads of 64 (a clip of 4680 tokens) use 57 % of the issue slots and 39 % of the
// tensor cores, heads of 128 (4096 causal tokens) 43 % and 55 %. Measured, of the measured cuBLAS rate:
//   9360 queries in chunks of 1560, each sees up to 4; 16 heads of 64 on 4   201 us   892 TFLOP/s, 47 %
//   8191 packed causal tokens, 32 heads of 128 on 8                       187 us   914 TFLOP/s, 48 %
//   8191 queries, as many keys, every one seen, 32 heads of 128 on 8      721 us  1524 TFLOP/s, 81 %
//   1 query of 8 sequences, 49920 keys, 16 heads of 64 on 4               17.3 us  3.0 TB/s, 3 us to join parts
// Slower were: one block an SM with a row tile over blocks of 256 keys, by quarters (229 us for the first);
// blocks that stay and take one unit after another (5 to 20 %); no running maximum while sums stay small
// (222); four blocks an SM over 64 keys, a thread a row (246); no warp of its own for the zeros (199 instead
// of 187 for the second).
#include <algorithm>
#include <cmath>

#include "fd_span.cuh"

namespace fd {
namespace {

struct SpanFwd {
  SpanShape y;
  int parts;
  const int32_t* spans;
  float scale_log2;
  SpanRows out;
  float* lse;      // [heads][n_q]
  float* part_o;   // [group][row tile][part][128][D]
  float2* part_ml; // the same rows: running maximum (log2) and sum
  int* err;
};

// P is made as 2^Up exp(s - m), where m, the row's maximum (log2), may be Slack behind before O is rescaled.
// fp16 ends at 2^16 and has steps of 2^-24 below 2^-14: with 11 and 4 P stays below 2^15 and keeps its digits down
// to 2^-25 of the row's largest; smaller ones are off by 2^-36 of it each, those of all 2^24 keys by
// 2^-12. (Sums of exponentials and O have the factor alike; 8191 packed tokens take 187 us with or without it.)
// bf16 has fp32's range.
template <bool F16>
struct Lift {
  static constexpr float kUp = F16 ? 11.f : 0.f, kSlack = F16 ? 4.f : 8.f;
};

// A block has a row tile of a group and a run of the key blocks, of 128 keys, that any of its queries
// see. Two blocks share an SM (half of TMEM and of shared memory each), so that the softmax of one runs
// beside the products of the other, and its beginning and end beside the other's middle.
//   warps 0-7   softmax: two threads a row (TMEM lane), half of the block's keys each; the row's maximum
//               goes through shared memory
//   warp 8      TMA: Q, then K and V by blocks, through a ring each
//   warp 9      zeros for the values of keys that no query of the tile sees (their probability is 0, but
//               0 times NaN is NaN)
//   warp 10     products: S = Q K^T, O += P V
// TMEM (256 columns): S 128, O at the end. D = 64: P has 64 of its own, so that the next scores begin when
// the softmax has read the last. D = 128: each half's P takes the first columns of the scores it was made of; the
// next scores are issued after the product that reads P, by the same thread, and products run in
// their order.
template <int D>
struct FwdCfg {
  static constexpr int kThreads = 11 * 32;  // two blocks: six warps on a sub-partition, 80 registers
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr bool kOwnP = D == 64;
  static constexpr int kSlotsK = D == 64 ? 3 : 1, kSlotsV = D == 64 ? 2 : 1;
  static constexpr int kOffK = kTileBytes;
  static constexpr int kOffV = kOffK + kSlotsK * kTileBytes;
  static constexpr int kOffMax = kOffV + kSlotsV * kTileBytes;  // [2][half][row]
  static constexpr int kOffBar = kOffMax + 4 * kTile * 4;
  static constexpr int kQFull = 0, kKFull = 1, kKFree = kKFull + kSlotsK, kVFull = kKFree + kSlotsK,
                       kVFree = kVFull + kSlotsV, kVReady = kVFree + kSlotsV,
                       kSFull = kVReady + kSlotsV,
                       kSRead = kSFull + 1, kPFull = kSRead + 1, kPv = kPFull + 1,
                       kDone = kPv + 1, kBars = kDone + 1;
  static constexpr int kSmem = kOffBar + (kBars * 8 + 32 + 127) / 128 * 128;
  static constexpr uint32_t kColS = 0, kColP = kOwnP ? 128 : 0, kColO = 256 - D;
  static constexpr uint32_t kHalfP = kOwnP ? 32 : 64;  // columns from a half's P to the other's
  static_assert(kSmem + 1024 <= 114 * 1024, "shared memory of two blocks");
};

template <bool F16, int D>
__global__ void __launch_bounds__(FwdCfg<D>::kThreads, 2)
    span_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmO,
                    const __grid_constant__ SpanFwd p) {
  using C = FwdCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem);
  const bool aligned = (base & 1023u) == 0;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kOffBar);
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * static_cast<uint32_t>(i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
  volatile int* range = reinterpret_cast<volatile int*>(tmem_slot + 1);  // first key, blocks

  // (later tokens first: under a causal mask they see most)
  const int part = blockIdx.x % p.parts;
  const int tile = p.y.row_tiles - 1 - static_cast<int>(blockIdx.x) / p.parts;
  const int group = blockIdx.y;
  const int token0 = tile * p.y.tile_tokens;
  const int tokens = min(p.y.tile_tokens, p.y.n_q - token0);

  // rows past tile_rows are never loaded
  if (p.y.tile_rows < kTile) {
    for (int i = threadIdx.x; i < C::kTileBytes / 16; i += C::kThreads)
      reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    __syncthreads();  // before Q is loaded
  }
  if (threadIdx.x == 8 * 32) {
    if (!aligned) atomicOr(p.err, ERR_SMEM_ALIGN);
    prefetch_tmap(&tmQ);
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
    prefetch_tmap(&tmO);
    mbar_init(bar(C::kQFull), 1);
    for (int i = 0; i < C::kSlotsK; ++i) {
      mbar_init(bar(C::kKFull + i), 1);
      mbar_init(bar(C::kKFree + i), 1);
    }
    for (int i = 0; i < C::kSlotsV; ++i) {
      mbar_init(bar(C::kVFull + i), 1);
      mbar_init(bar(C::kVFree + i), 1);
      mbar_init(bar(C::kVReady + i), 1);
    }
    mbar_init(bar(C::kSFull), 1);
    mbar_init(bar(C::kSRead), 8);
    mbar_init(bar(C::kPFull), 8);
    mbar_init(bar(C::kPv), 1);
    mbar_init(bar(C::kDone), 1);
    fence_barrier_init();
  }
  grid_dep_wait();
  grid_dep_launch();
  int loads_k = 0, loads_v = 0;  // warp 8: so far
  // K or V of block n; waits for its slot after the first ones
  auto load = [&](int n, int first_key, const CUtensorMap* map, uint32_t to, int slots, int full, int free) {
    const int slot = n % slots;
    if (n >= slots && !wait(bar(free + slot), (n / slots - 1) & 1, p.err, ERR_WAIT_MMA)) return false;
    mbar_expect_tx(bar(full + slot), C::kTileBytes);
    for (int d = 0; d < D / 64; ++d)
      tma_load_4d(to + slot * C::kTileBytes + d * kSub, map, bar(full + slot), 64 * d, group,
                  first_key + n * kTile, 0);
    return true;
  };
  if (warp == 10) {
    tmem_alloc(smem_u32(tmem_slot), 256);
    tmem_relinquish();
  } else if (warp == 8) {
    if (lane == 0 && aligned) {
      mbar_expect_tx(bar(C::kQFull), p.y.tile_rows * D * 2);
      for (int d = 0; d < D / 64; ++d)
        tma_load_4d(base + d * kSub, &tmQ, bar(C::kQFull), 64 * d, group * p.y.per, token0, 0);
    }
    __syncwarp();
    // the keys that any query of the tile sees, and this block's part of them
    int lo = 0x7fffffff, hi = 0;
    for (int i = lane; i < tokens; i += 32) {
      const int2 s = span_of(p.spans, token0 + i, p.y.n_k);
      if (s.x < s.y) {
        lo = min(lo, s.x);
        hi = max(hi, s.y);
      }
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    const int key = hi > 0 ? lo / kTile * kTile : 0;
    const int n = (hi - key + kTile - 1) / kTile;
    const int first = static_cast<int>(static_cast<int64_t>(n) * part / p.parts);
    const int end = static_cast<int>(static_cast<int64_t>(n) * (part + 1) / p.parts);
    const int first_key = key + first * kTile, blocks = aligned ? end - first : 0;
    if (lane == 0) {
      range[0] = first_key;
      range[1] = blocks;
      // what there is room for, while the others get ready
      for (; loads_v < min(blocks, C::kSlotsV); ++loads_k, ++loads_v) {
        load(loads_k, first_key, &tmK, base + C::kOffK, C::kSlotsK, C::kKFull, C::kKFree);
        load(loads_v, first_key, &tmV, base + C::kOffV, C::kSlotsV, C::kVFull, C::kVFree);
      }
    }
  }
  // the softmax's rows
  const int token = token0 + ((warp & 3) * 32 + lane) / p.y.per;
  const bool valid = warp < 8 && (warp & 3) * 32 + lane < p.y.tile_rows && token < p.y.n_q;
  const int2 span = valid ? span_of(p.spans, token, p.y.n_k) : make_int2(0, 0);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int key_start = range[0], count = range[1];

  if (count == 0) {
    // nothing is seen: the softmax warps write that below, where Q may be on its way to (and nothing may be in
    // flight when the block exits)
    if (threadIdx.x < 8 * 32 && aligned) {
      wait(bar(C::kQFull), 0, p.err, ERR_WAIT_TMA, true);
      __syncwarp();
    }
  } else if (warp == 8) {
    if (lane == 0) {
      // K and V in turn, each when its slot is free (the scores of a block are through before its P V:
      // no K is kept waiting)
      int k = loads_k, v = loads_v;
      while (v < count && load(k, key_start, &tmK, base + C::kOffK, C::kSlotsK, C::kKFull, C::kKFree)) {
        ++k;
        if (!load(v, key_start, &tmV, base + C::kOffV, C::kSlotsV, C::kVFull, C::kVFree)) break;
        ++v;
      }
      // nothing may be in flight when the block exits
      wait(bar(C::kQFull), 0, p.err, ERR_WAIT_TMA, true);
      for (int j = max(0, k - C::kSlotsK); j < k; ++j)
        wait(bar(C::kKFull + j % C::kSlotsK), (j / C::kSlotsK) & 1, p.err, ERR_WAIT_TMA, true);
      for (int j = max(0, v - C::kSlotsV); j < v; ++j)
        wait(bar(C::kVFull + j % C::kSlotsV), (j / C::kSlotsV) & 1, p.err, ERR_WAIT_TMA, true);
    }
  } else if (warp == 9) {
    // ---- values of keys that nothing sees
    int2 spans[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      spans[i] = lane + 32 * i < tokens ? span_of(p.spans, token0 + lane + 32 * i, p.y.n_k)
                                       : make_int2(0, 0);
    for (int n = 0; n < count; ++n) {
      const int key0 = key_start + n * kTile, slot = n % C::kSlotsV;
      bool whole = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) whole |= spans[i].x <= key0 && spans[i].y >= key0 + kTile;
      uint32_t seen[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
      if (!__any_sync(0xffffffffu, whole)) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t mine = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) mine |= seen_word(spans[i], key0 + 32 * w);
          seen[w] = __reduce_or_sync(0xffffffffu, mine);
        }
      }
      if (!wait_warp(bar(C::kVFull + slot), (n / C::kSlotsV) & 1, p.err, ERR_WAIT_TMA)) break;
      if ((seen[0] & seen[1] & seen[2] & seen[3]) != 0xffffffffu) {
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
          const uint32_t there = w == 0 ? seen[0] : w == 1 ? seen[1] : w == 2 ? seen[2] : seen[3];
          if ((there >> lane) & 1u) continue;
          uint4* row = reinterpret_cast<uint4*>(smem + C::kOffV + slot * C::kTileBytes +
                                                (32 * w + lane) * 128);
#pragma unroll
          for (int d = 0; d < D / 64; ++d)
#pragma unroll
            for (int c = 0; c < 8; ++c) row[d * (kSub / 16) + c] = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kVReady + slot));
    }
  } else if (warp == 10) {
    constexpr uint32_t is = Mma<F16, D>::idesc(kTile, false), io = Mma<F16, D>::idesc(D, true);
    const uint64_t q0 = sdesc_k_sw128(base);
    auto scores = [&](int j) -> bool {
      const int slot = j % C::kSlotsK;
      if (!wait_warp(bar(C::kKFull + slot), (j / C::kSlotsK) & 1, p.err, ERR_WAIT_TMA)) return false;
      tc_fence_after();
      const uint64_t k0 = sdesc_k_sw128(base + C::kOffK + slot * C::kTileBytes);
#pragma unroll
      for (int d = 0; d < D / 64; ++d)
        mma4_bf16_ss_w(tmem + C::kColS, q0 + static_cast<uint64_t>(d * (kSub >> 4)),
                       k0 + static_cast<uint64_t>(d * (kSub >> 4)), is, d > 0);
      mma_commit_w(bar(C::kSFull));
      mma_commit_w(bar(C::kKFree + slot));
      return true;
    };
    bool ok = wait_warp(bar(C::kQFull), 0, p.err, ERR_WAIT_TMA) && scores(0);
    for (int j = 0; j < count && ok; ++j) {
      const int slot = j % C::kSlotsV;
      if (C::kOwnP && j + 1 < count)
        ok = wait_warp(bar(C::kSRead), j & 1, p.err, ERR_WAIT_EPI) && scores(j + 1);
      ok = ok && wait_warp(bar(C::kVReady + slot), (j / C::kSlotsV) & 1, p.err, ERR_WAIT_TMA) &&
           wait_warp(bar(C::kPFull), j & 1, p.err, ERR_WAIT_EPI);
      if (!ok) break;
      tc_fence_after();
      const uint32_t v = base + C::kOffV + slot * C::kTileBytes;
#pragma unroll
      for (int x = 0; x < 2; ++x)
        mma4_ts_mn_w(tmem + C::kColO, tmem + C::kColP + C::kHalfP * x, sdesc_mn_sw128(v + x * 64 * 128, kSub), io,
                     j > 0 || x > 0);
      mma_commit_w(bar(C::kPv));
      mma_commit_w(bar(C::kVFree + slot));
      if (!C::kOwnP && j + 1 < count) ok = scores(j + 1);
    }
    products_done(bar(C::kDone), p.err);
  }
  if (warp < 8) {
    // ---- softmax of half h of the blocks' keys
    const int h = warp >> 2, lanes = warp & 3;
    const int row = lanes * 32 + lane;
    const bool sees = span.x < span.y;
    // keys that all of the warp's rows see (rows that see none, or are none, are set right at the end)
    const int all_from = __reduce_max_sync(0xffffffffu, sees ? span.x : 0);
    const int all_to = __reduce_min_sync(0xffffffffu, sees ? span.y : 0x7fffffff);
    const uint32_t lane_off = static_cast<uint32_t>(lanes * 32) << 16;
    const uint32_t s_col = tmem + lane_off + C::kColS + 64u * h;
    const uint32_t p_col = tmem + lane_off + C::kColP + C::kHalfP * h;
    const uint32_t o_col = tmem + lane_off + C::kColO + D / 2 * h;
    volatile float* const tops = reinterpret_cast<volatile float*>(smem + C::kOffMax) + row;
    const float c = p.scale_log2;
    const uint64_t c2 = pack_f32x2(c, c);
    float m = -INFINITY, l = 0.f;
    // A wait that gives up has set the status word, and every wait after it returns at once: the warps
    // go on to the end. Warps without a row that sees any key (a tile of few queries has such) leave the
    // others their issue slots, which saves 2 us for the one query of 8 sequences; what is in their rows of
    // TMEM goes nowhere.
    const bool idle = !__any_sync(0xffffffffu, sees);
#pragma unroll 1
    for (int j = 0; j < count; ++j) {
      if (idle) {
        wait_warp(bar(C::kSFull), j & 1, p.err, ERR_WAIT_MMA);
        if (j > 0) wait_warp(bar(C::kPv), (j - 1) & 1, p.err, ERR_WAIT_MMA);
        if (lane == 0) {
          if (C::kOwnP) mbar_arrive(bar(C::kSRead));
          mbar_arrive(bar(C::kPFull));
        }
        continue;
      }
      const int key0 = key_start + j * kTile + 64 * h;
      const bool masked = key0 < all_from || key0 + 64 > all_to;
      wait_warp(bar(C::kSFull), j & 1, p.err, ERR_WAIT_MMA);
      tc_fence_after();
      // 32 scores at a time; the second 32 are fetched again for their exponentials
      uint32_t sr[32];
      auto hide = [&](int x) {
        if (masked) {
          __syncwarp();  // (not predicated: else the selections are made for every block)
          const uint32_t seen = seen_word(span, key0 + 32 * x);
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (!(seen & (1u << e))) sr[e] = 0xff800000u;
        }
      };
      float mx[2];
#pragma unroll
      for (int x = 1; x >= 0; --x) {
        tmem_ld_32x32b_x32(s_col + 32 * x, sr);
        tmem_ld_wait();
        hide(x);
        float a = __uint_as_float(sr[0]), b = __uint_as_float(sr[16]);
#pragma unroll
        for (int e = 1; e < 15; e += 2) {
          a = fmax3(a, __uint_as_float(sr[e]), __uint_as_float(sr[e + 1]));
          b = fmax3(b, __uint_as_float(sr[16 + e]), __uint_as_float(sr[17 + e]));
        }
        mx[x] = fmax3(fmaxf(a, b), __uint_as_float(sr[15]), __uint_as_float(sr[31]));
      }
      // the row's maximum over both halves
      float top = fmaxf(mx[0], mx[1]) * c;
      volatile float* const at = tops + (j & 1) * 2 * kTile;
      at[h * kTile] = top;
      named_barrier(1 + lanes, 64);
      top = fmaxf(top, at[(h ^ 1) * kTile]);
      const bool grow = top > m + Lift<F16>::kSlack;
      const float before = m;
      if (grow) m = top;
      const float off = m == -INFINITY ? 0.f : m;
      // the last product has read P, and O is as it left it
      if (j > 0) wait_warp(bar(C::kPv), (j - 1) & 1, p.err, ERR_WAIT_MMA);
      tc_fence_after();
      if (j > 0 && __any_sync(0xffffffffu, grow)) {
        const float f = grow ? ex2_approx(before - off) : 1.f;
        l *= f;
#pragma unroll 1
        for (int d = 0; d < D / 2; d += 16) {
          uint32_t o[16];
          tmem_ld_32x32b_x16(o_col + d, o);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
          tmem_st_32x32b_x16(o_col + d, o);
        }
      }
      const float lift = Lift<F16>::kUp - off;
      const uint64_t off2 = pack_f32x2(lift, lift);
      uint64_t sum2[2] = {0, 0};
      // P in the inputs' type, which the product with V takes: half a step of each, 2^-8 (bf16) or 2^-11
      // (fp16, down to 2^-25 of the row's largest) of it at most. The sums are of P unrounded.
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (x == 1) {
          tmem_ld_32x32b_x32(s_col + 32, sr);
          tmem_ld_wait();
          if (C::kOwnP) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(C::kSRead));
          }
          hide(1);
        }
        uint32_t pk[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float2 v = halves_of(fma2(pair_of(sr[e], sr[e + 1]), c2, off2));
          const float a = ex2_approx(v.x), b = ex2_approx(v.y);
          sum2[e / 2 % 2] = add2(sum2[e / 2 % 2], pack_f32x2(a, b));
          pk[e / 2] = pack16<F16>(a, b);
        }
        tmem_st_32x32b_x16(p_col + 16 * x, pk);
      }
      {
        const float2 a = halves_of(sum2[0]), b = halves_of(sum2[1]);
        l += (a.x + a.y) + (b.x + b.y);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kPFull));
    }

    // ---- the result: half of the row's elements a thread
    if (count > 0) wait_warp(bar(C::kPv), (count - 1) & 1, p.err, ERR_WAIT_MMA);
    tc_fence_after();
    volatile float* const at = tops + (count & 1) * 2 * kTile;
    at[h * kTile] = l;
    named_barrier(1 + lanes, 64);
    l = at[0] + at[kTile];
    if (!sees || count == 0) l = 0.f;
    if (l == 0.f) m = -INFINITY;
    const bool whole = p.parts == 1;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int head = group * p.y.per + row % p.y.per;
    const int64_t slot =
        ((static_cast<int64_t>(group) * p.y.row_tiles + tile) * p.parts + part) * kTile + row;
#pragma unroll 1
    for (int d = h * (D / 2); d < (h + 1) * (D / 2); d += 32) {
      uint32_t o[32];
      if (count > 0) {
        __syncwarp();
        tmem_ld_32x32b_x32(tmem + lane_off + C::kColO + d, o);
        tmem_ld_wait();
      }
      if (whole) {
        // into Q's place, which the last scores have read
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
          uint32_t v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[i] = l == 0.f ? 0u
                            : pack16<F16>(__uint_as_float(o[e + 2 * i]) * inv,
                                          __uint_as_float(o[e + 2 * i + 1]) * inv);
          *reinterpret_cast<uint4*>(smem + tile_chunk(row, (d + e) / 8)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
      } else if (valid && l != 0.f) {
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          *reinterpret_cast<uint4*>(p.part_o + slot * D + d + e) =
              make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      }
    }
    if (h == 0 && valid) {
      if (whole)
        p.lse[static_cast<int64_t>(head) * p.y.n_q + token] =
            l == 0.f ? -INFINITY : (m - Lift<F16>::kUp + log2f(l)) * kLn2;
      else
        p.part_ml[slot] = make_float2(m - Lift<F16>::kUp, l);
    }
    if (whole) {
      fence_proxy_async_smem();
      named_barrier(5, 256);
      if (threadIdx.x == 0 && aligned) {
        for (int d = 0; d < D / 64; ++d)
          tma_store_4d(&tmO, base + d * kSub, 64 * d, group * p.y.per, token0, 0);
        bulk_commit();
        bulk_wait_all();
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 10) {
    tc_fence_after();
    tmem_dealloc(tmem, 256);
  }
}

// A row's parts, added up: a block a row, 256 / (D / 4) of its threads' groups each every so many parts, whose
// sums are then added up in their order. (One thread an element walking over the parts took 13 us for
// 38 of them.)
template <bool F16, int D>
__global__ void __launch_bounds__(256) span_join_kernel(const __grid_constant__ SpanFwd p) {
  constexpr int kLanes = D / 4, kSlices = 256 / kLanes;
  __shared__ float4 sums[kSlices][kLanes];
  __shared__ float total[kSlices];
  __shared__ float most[8];
  grid_dep_wait();
  grid_dep_launch();
  const int token = blockIdx.x, head = blockIdx.y;
  const int group = head / p.y.per, tile = token / p.y.tile_tokens;
  const int row = (token - tile * p.y.tile_tokens) * p.y.per + head % p.y.per;
  const int64_t first = (static_cast<int64_t>(group) * p.y.row_tiles + tile) * p.parts * kTile + row;
  float m = -INFINITY;
  for (int c = threadIdx.x; c < p.parts; c += 256) m = fmaxf(m, __ldcg(p.part_ml + first + c * kTile).x);
#pragma unroll
  for (int i = 16; i; i >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, i));
  if ((threadIdx.x & 31) == 0) most[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, most[i]);
  const int lane = threadIdx.x % kLanes, slice = threadIdx.x / kLanes;
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int c = slice; c < p.parts; c += kSlices) {
    const int64_t at = first + c * kTile;
    const float2 x = __ldcg(p.part_ml + at);
    if (x.y == 0.f) continue;  // (nothing was seen, and nothing stored)
    const float4 a = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * D) + lane);
    const float f = ex2_approx(x.x - m);
    l = fmaf(f, x.y, l);
    o.x = fmaf(f, a.x, o.x);
    o.y = fmaf(f, a.y, o.y);
    o.z = fmaf(f, a.z, o.z);
    o.w = fmaf(f, a.w, o.w);
  }
  sums[slice][lane] = o;
  if (lane == 0) total[slice] = l;
  __syncthreads();
  if (threadIdx.x >= D) return;
  const int d = threadIdx.x;
  float sum = 0.f;
  l = 0.f;
#pragma unroll
  for (int i = 0; i < kSlices; ++i) {
    sum += reinterpret_cast<const float*>(sums[i])[d];
    l += total[i];
  }
  using T = typename std::conditional<F16, __half, __nv_bfloat16>::type;
  static_cast<T*>(p.out.p)[static_cast<int64_t>(token) * p.out.token +
                           static_cast<int64_t>(head) * p.out.head + d] = T(l == 0.f ? 0.f : sum / l);
  if (d == 0)
    p.lse[static_cast<int64_t>(head) * p.y.n_q + token] =
        l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Parts of every tile's key blocks: as many as fill the GPU (two blocks an SM) where there are few tiles,
// but 256 keys each at least where every key is seen, since joining the parts takes 3 us. (Spans are not known here: a
// query that sees 128 of 49920 keys has as many parts, nearly all of them empty, 8.4 us for 16 heads of 64 on 4; all
// of the keys 13.6.)
int fwd_parts(const SpanShape& y) {
  const int64_t units = static_cast<int64_t>(y.groups) * y.row_tiles;
  return static_cast<int>(
      std::max<int64_t>(1, std::min<int64_t>(y.key_blocks / 2, 2 * num_sms() / units)));
}

template <bool F16, int D>
cudaError_t launch_fwd(const SpanFwd& p, const SpanRows& q, const SpanRows& k, const SpanRows& v,
                       cudaStream_t s) {
  using C = FwdCfg<D>;
  CUtensorMap tmQ, tmK, tmV, tmO;
  if (!make_map(&tmO, F16, p.out.p, D, p.y.heads, p.y.n_q, 1, p.out.head, p.out.token, 0, p.y.per,
                p.y.tile_tokens) ||
      !make_map(&tmQ, F16, q.p, D, p.y.heads, p.y.n_q, 1, q.head, q.token, 0, p.y.per, p.y.tile_tokens) ||
      !make_map(&tmK, F16, k.p, D, p.y.groups, p.y.n_k, 1, k.head, k.token, 0, 1, kTile) ||
      !make_map(&tmV, F16, v.p, D, p.y.groups, p.y.n_k, 1, v.head, v.token, 0, 1, kTile))
    return cudaErrorInvalidValue;
  static OncePerDevice once;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess)
    e = once.run(dev, [&] {
      return cudaFuncSetAttribute(span_fwd_kernel<F16, D>,
                                  cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
    });
  if (e != cudaSuccess) return e;
  e = launch_pdl(span_fwd_kernel<F16, D>, dim3(p.y.row_tiles * p.parts, p.y.groups), dim3(C::kThreads),
                 C::kSmem, s, tmQ, tmK, tmV, tmO, p);
  if (e != cudaSuccess || p.parts == 1) return e;
  return launch_pdl(span_join_kernel<F16, D>, dim3(p.y.n_q, p.y.heads), dim3(256), 0, s, p);
}

// no keys: every query sees nothing
template <bool F16, int D>
__global__ void span_none_kernel(const __grid_constant__ SpanFwd p) {
  grid_dep_wait();
  const int64_t rows = static_cast<int64_t>(p.y.n_q) * p.y.heads;
  for (int64_t i = blockIdx.x; i < rows; i += gridDim.x) {
    const int64_t token = i / p.y.heads, head = i % p.y.heads;
    static_cast<uint16_t*>(p.out.p)[token * p.out.token + head * p.out.head + threadIdx.x] = 0;
    if (threadIdx.x == 0) p.lse[head * p.y.n_q + token] = -INFINITY;
  }
  grid_dep_launch();
}

template <bool F16, int D>
cudaError_t launch(const SpanFwd& p, const SpanRows& q, const SpanRows& k, const SpanRows& v,
                   cudaStream_t s) {
  if (p.y.n_k == 0)
    return launch_pdl(span_none_kernel<F16, D>, dim3(num_sms()), dim3(D), 0, s, p);
  return launch_fwd<F16, D>(p, q, k, v, s);
}

}  // namespace

size_t span_fwd_workspace_bytes(int n_q, int n_k, int heads, int groups, int head_dim) {
  if (n_q == 0 || n_k == 0) return 0;
  const SpanShape y = span_shape(n_q, n_k, heads, groups);
  const int parts = fwd_parts(y);
  if (parts == 1) return 0;
  return static_cast<size_t>(groups) * y.row_tiles * parts * kTile *
         (head_dim * sizeof(float) + sizeof(float2));
}

}  // namespace fd

extern "C" {

size_t fd_span_attention_workspace_bytes(const fd_span_attention* a, int backward) {
  if (!fd::span_valid(a)) return 0;
  return backward ? fd::span_bwd_workspace_bytes(a->n_q, a->n_k, a->heads, a->groups, a->head_dim)
                  : fd::span_fwd_workspace_bytes(a->n_q, a->n_k, a->heads, a->groups, a->head_dim);
}

fd_status fd_op_span_attention(const fd_span_attention* a, const void* q, int64_t q_token_stride,
                               int64_t q_head_stride, const void* k, int64_t k_token_stride,
                               int64_t k_head_stride, const void* v, int64_t v_token_stride,
                               int64_t v_head_stride, const int32_t* spans, void* out,
                               int64_t out_token_stride, int64_t out_head_stride, float* lse,
                               void* workspace, int* err_dev, void* stream) {
  if (!fd::span_valid(a)) return FD_ERR_INVALID_ARG;
  if (a->n_q == 0) return FD_OK;
  const fd::SpanRows qr{const_cast<void*>(q), q_token_stride, q_head_stride},
      kr{const_cast<void*>(k), k_token_stride, k_head_stride},
      vr{const_cast<void*>(v), v_token_stride, v_head_stride},
      outr{out, out_token_stride, out_head_stride};
  if (!fd::span_rows_ok(qr, a->n_q, a->heads, a->head_dim) ||
      !fd::span_out_ok(outr, a->n_q, a->heads, a->head_dim) ||
      (a->n_k > 0 && (!fd::span_rows_ok(kr, a->n_k, a->groups, a->head_dim) ||
                      !fd::span_rows_ok(vr, a->n_k, a->groups, a->head_dim))) ||
      !fd::span_ptr(spans, 8) || !fd::span_ptr(lse, 4) || !fd::span_ptr(err_dev, 4) ||
      fd::span_meets(outr, {q, k, v, spans, lse, workspace}))
    return FD_ERR_INVALID_ARG;
  const size_t need =
      fd::span_fwd_workspace_bytes(a->n_q, a->n_k, a->heads, a->groups, a->head_dim);
  if (need > 0 && !fd::span_ptr(workspace, 16)) return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  fd::SpanFwd p{};
  p.y = fd::span_shape(a->n_q, a->n_k, a->heads, a->groups);
  p.parts = a->n_k > 0 ? fd::fwd_parts(p.y) : 1;
  p.spans = spans;
  p.scale_log2 = a->scale * fd::kLog2e;
  p.out = outr;
  p.lse = lse;
  const int64_t rows = static_cast<int64_t>(p.y.groups) * p.y.row_tiles * p.parts * fd::kTile;
  p.part_o = static_cast<float*>(workspace);
  p.part_ml = need > 0 ? reinterpret_cast<float2*>(p.part_o + rows * a->head_dim) : nullptr;
  p.err = err_dev;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool f16 = a->dtype == FD_DTYPE_F16;
  const cudaError_t e =
      a->head_dim == 64
          ? (f16 ? fd::launch<true, 64>(p, qr, kr, vr, s) : fd::launch<false, 64>(p, qr, kr, vr, s))
          : (f16 ? fd::launch<true, 128>(p, qr, kr, vr, s) : fd::launch<false, 128>(p, qr, kr, vr, s));
  return e == cudaSuccess ? FD_OK : FD_ERR_CUDA;
}

}  // extern "C"
