// Attention in which every query sees a span of keys, forward (fd_op_span_attention):
//   s = scale q k^T within the span, lse = log sum exp s, out = exp(s - lse) v
// by blocks of 128 keys with a running maximum and sum, kept in fp32 with O in TMEM.
#include <algorithm>
#include <cmath>

#include "fd_span.cuh"

namespace fd {
namespace {

struct SpanFwd {
  SpanShape y;
  int pairs, parts;
  const int32_t* spans;
  float scale_log2;
  SpanRows out;
  float* lse;      // [heads][n_q]
  float* part_o;   // [group][pair][part][tile][128][D]
  float2* part_ml; // the same rows: running maximum (log2) and sum
  int* err;
};

constexpr float kSlack = 8.f;  // log2 by which a row's maximum may grow before O is rescaled

// A block has two row tiles of a group (a pair) and a run of the key blocks that any of their
// queries see.
//   warps 0 ..     softmax: D = 128: four warps a tile, a thread per row; D = 64: eight, half of a
//                  block's keys each, with a running maximum, a sum and an O of its own
//   next           TMA: Q of both tiles, then K and V by blocks through one ring
//   next           zeros for the values of keys that no query of the pair sees (their probability is
//                  0, but 0 times NaN is NaN)
//   last two       products of a tile each: S = Q K^T, O += P V
// TMEM: S of both tiles (P takes the first columns of what it was made of), then O.
template <int D>
struct FwdCfg {
  static constexpr int kHalves = D == 64 ? 2 : 1;
  static constexpr int kKeys = kTile / kHalves;  // of a softmax thread
  static constexpr int kSoftmax = 8 * kHalves;   // warps
  static constexpr int kThreads = (kSoftmax + 4) * 32;
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kSlots = D == 128 ? 5 : 10;
  static constexpr int kOffRing = 2 * kTileBytes;
  static constexpr int kOffMl = kOffRing + kSlots * kTileBytes;
  static constexpr int kOffBar = kOffMl + (kHalves == 2 ? 4 * kTile * 8 : 0);
  static constexpr int kQFull = 0, kFull = 1, kFree = kFull + kSlots, kReady = kFree + kSlots,
                       kSFull = kReady + kSlots, kPFull = kSFull + 2, kOFull = kPFull + 4,
                       kBars = kOFull + 2;
  static constexpr int kSmem = kOffBar + (kBars * 8 + 32 + 127) / 128 * 128;
  static constexpr uint32_t kColS = 0, kColO = 256;  // S of tile t at 128 t, O at 128 t (+ 64 half)
  static_assert(kSmem <= 227 * 1024, "shared memory");
  // the phase of kReady for item i of the ring: a slot has a V every kSlots items, or every second time
  static __device__ uint32_t ready_phase(int i) {
    return (kSlots % 2 ? i / (2 * kSlots) : i / kSlots) & 1;
  }
};

template <bool F16, int D>
__global__ void __launch_bounds__(FwdCfg<D>::kThreads, 1)
    span_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const __grid_constant__ SpanFwd p) {
  using C = FwdCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem);
  const bool aligned = (base & 1023u) == 0;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kOffBar);
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * static_cast<uint32_t>(i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
  volatile int* range = reinterpret_cast<volatile int*>(tmem_slot + 1);  // first block, blocks
  float2* ml = reinterpret_cast<float2*>(smem + C::kOffMl);              // [tile][half][row]

  // (later tokens first: under a causal mask they see most)
  const int part = blockIdx.x % p.parts;
  const int pair = p.pairs - 1 - static_cast<int>(blockIdx.x) / p.parts;
  const int group = blockIdx.y;
  const int token0 = pair * 2 * p.y.tile_tokens;
  const int tokens = min(2 * p.y.tile_tokens, p.y.n_q - token0);

  for (int i = threadIdx.x; i < 2 * C::kTileBytes / 16; i += C::kThreads)
    reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async_smem();
  if (threadIdx.x == 0) {
    if (!aligned) atomicOr(p.err, ERR_SMEM_ALIGN);
    mbar_init(bar(C::kQFull), 1);
    for (int i = 0; i < C::kSlots; ++i) {
      mbar_init(bar(C::kFull + i), 1);
      mbar_init(bar(C::kFree + i), 2);
      mbar_init(bar(C::kReady + i), 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(bar(C::kSFull + t), 1);
      mbar_init(bar(C::kOFull + t), 1);
      for (int h = 0; h < 2; ++h) mbar_init(bar(C::kPFull + 2 * t + h), 4);
    }
    fence_barrier_init();
  }
  grid_dep_wait();
  grid_dep_launch();
  if (warp == 0) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  } else if (warp == 1) {
    // the key blocks that any query of the pair sees, and this block's part of them
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
    const int b0 = hi > 0 ? lo / kTile : 0, n = hi > 0 ? (hi + kTile - 1) / kTile - b0 : 0;
    const int first = static_cast<int>(static_cast<int64_t>(n) * part / p.parts);
    const int end = static_cast<int>(static_cast<int64_t>(n) * (part + 1) / p.parts);
    if (lane == 0) {
      range[0] = b0 + first;
      range[1] = aligned ? end - first : 0;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int block0 = range[0], count = range[1];

  if (count == 0) {
    // nothing is seen: the softmax warps write that below
  } else if (warp == C::kSoftmax) {
    if (lane == 0) {
      prefetch_tmap(&tmQ);
      prefetch_tmap(&tmK);
      prefetch_tmap(&tmV);
      mbar_expect_tx(bar(C::kQFull), 2 * p.y.tile_rows * D * 2);
      for (int t = 0; t < 2; ++t)
        for (int d = 0; d < D / 64; ++d)
          tma_load_4d(base + t * C::kTileBytes + d * kSub, &tmQ, bar(C::kQFull), 64 * d,
                      group * p.y.per, token0 + t * p.y.tile_tokens, 0);
      int i = 0;  // K of block j is item 2 j of the ring, V item 2 j + 1
      for (; i < 2 * count; ++i) {
        const int slot = i % C::kSlots;
        if (i >= C::kSlots &&
            !wait(bar(C::kFree + slot), (i / C::kSlots - 1) & 1, p.err, ERR_WAIT_MMA))
          break;
        mbar_expect_tx(bar(C::kFull + slot), C::kTileBytes);
        for (int d = 0; d < D / 64; ++d)
          tma_load_4d(base + C::kOffRing + slot * C::kTileBytes + d * kSub, i & 1 ? &tmV : &tmK,
                      bar(C::kFull + slot), 64 * d, group, (block0 + i / 2) * kTile, 0);
      }
      // nothing may be in flight when the block exits
      wait(bar(C::kQFull), 0, p.err, ERR_WAIT_TMA, true);
      for (int j = max(0, i - C::kSlots); j < i; ++j)
        wait(bar(C::kFull + j % C::kSlots), (j / C::kSlots) & 1, p.err, ERR_WAIT_TMA, true);
    }
  } else if (warp == C::kSoftmax + 1) {
    // ---- values of keys that nothing sees
    int2 span[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      span[i] = lane + 32 * i < tokens ? span_of(p.spans, token0 + lane + 32 * i, p.y.n_k)
                                       : make_int2(0, 0);
    for (int j = 0; j < count; ++j) {
      const int key0 = (block0 + j) * kTile, item = 2 * j + 1, slot = item % C::kSlots;
      bool whole = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) whole |= span[i].x <= key0 && span[i].y >= key0 + kTile;
      uint32_t seen[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};
      if (!__any_sync(0xffffffffu, whole)) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t mine = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) mine |= seen_word(span[i], key0 + 32 * w);
          seen[w] = __reduce_or_sync(0xffffffffu, mine);
        }
      }
      // (K too: a parity tells a phase from its neighbours only, so none may be left out)
      const int before = item - 1;
      if (!wait_warp(bar(C::kFull + before % C::kSlots), (before / C::kSlots) & 1, p.err,
                     ERR_WAIT_TMA) ||
          !wait_warp(bar(C::kFull + slot), (item / C::kSlots) & 1, p.err, ERR_WAIT_TMA))
        break;
      if ((seen[0] & seen[1] & seen[2] & seen[3]) != 0xffffffffu) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if ((seen[w] >> lane) & 1u) continue;
          uint4* row = reinterpret_cast<uint4*>(smem + C::kOffRing + slot * C::kTileBytes +
                                                (32 * w + lane) * 128);
#pragma unroll
          for (int d = 0; d < D / 64; ++d)
#pragma unroll
            for (int c = 0; c < 8; ++c) row[d * (kSub / 16) + c] = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kReady + slot));
    }
  } else if (warp > C::kSoftmax + 1) {
    // ---- products of tile t. S of the next block goes where P of this one is: it is issued after
    // the product that reads P, by the same thread, and products run in their order.
    const int t = warp - C::kSoftmax - 2;
    if (lane == 0) {
      constexpr uint32_t is = Mma<F16, D>::idesc(kTile, false), io = Mma<F16, D>::idesc(D, true);
      const uint32_t s_col = tmem + C::kColS + 128u * t, o_col = tmem + C::kColO + 128u * t;
      const uint64_t q0 = sdesc_k_sw128(base + t * C::kTileBytes);
      auto scores = [&](int j) -> bool {
        const int item = 2 * j, slot = item % C::kSlots;
        if (!wait(bar(C::kFull + slot), (item / C::kSlots) & 1, p.err, ERR_WAIT_TMA)) return false;
        tc_fence_after();
        const uint64_t k0 = sdesc_k_sw128(base + C::kOffRing + slot * C::kTileBytes);
#pragma unroll
        for (int d = 0; d < D / 64; ++d)
          mma4_bf16_ss(s_col, q0 + static_cast<uint64_t>(d * (kSub >> 4)),
                       k0 + static_cast<uint64_t>(d * (kSub >> 4)), is, d > 0);
        mma_commit(bar(C::kSFull + t));
        mma_commit(bar(C::kFree + slot));
        return true;
      };
      bool ok = wait(bar(C::kQFull), 0, p.err, ERR_WAIT_TMA) && scores(0);
      for (int j = 0; j < count && ok; ++j) {
        const int item = 2 * j + 1, slot = item % C::kSlots;
        ok = wait(bar(C::kReady + slot), C::ready_phase(item), p.err, ERR_WAIT_TMA);
        const uint32_t v = base + C::kOffRing + slot * C::kTileBytes;
#pragma unroll
        for (int h = 0; h < C::kHalves; ++h) {
          ok = ok && wait(bar(C::kPFull + 2 * t + h), j & 1, p.err, ERR_WAIT_EPI);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int x = 0; x < C::kKeys / 64; ++x)
            mma4_ts_mn(o_col + 64u * h, s_col + 64u * h + 32u * x,
                       sdesc_mn_sw128(v + (h * C::kKeys + x * 64) * 128, kSub), io, j > 0 || x > 0);
        }
        if (!ok) break;
        mma_commit(bar(C::kFree + slot));
        if (j + 1 < count) ok = scores(j + 1);
      }
      mma_commit(bar(C::kOFull + t));
      wait(bar(C::kOFull + t), 0, p.err, ERR_WAIT_MMA, true);
    }
  }
  if (warp < C::kSoftmax) {
    // ---- softmax of half h of tile t
    const int t = warp / (4 * C::kHalves), h = (warp >> 2) % C::kHalves;
    const int row = (warp & 3) * 32 + lane;
    const int token = token0 + t * p.y.tile_tokens + row / p.y.per;
    const bool valid = row < p.y.tile_rows && token < p.y.n_q;
    const int2 span = valid ? span_of(p.spans, token, p.y.n_k) : make_int2(0, 0);
    const bool sees = span.x < span.y;
    // keys that all of the warp's rows see (rows that see none, or are none, are set right at the end)
    const int all_from = __reduce_max_sync(0xffffffffu, sees ? span.x : 0);
    const int all_to = __reduce_min_sync(0xffffffffu, sees ? span.y : 0x7fffffff);
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_col = tmem + lane_off + C::kColS + 128u * t + 64u * h;
    const uint32_t o_col = tmem + lane_off + C::kColO + 128u * t + 64u * h;
    const float c = p.scale_log2;
    const uint64_t c2 = pack_f32x2(c, c);
    float m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int j = 0; j < count; ++j) {
      const int key0 = (block0 + j) * kTile + h * C::kKeys;
      wait_warp(bar(C::kSFull + t), j & 1, p.err, ERR_WAIT_MMA);
      tc_fence_after();
      const bool masked = key0 < all_from || key0 + C::kKeys > all_to;
      // 64 scores at a time; those of 128 are fetched again for their exponentials
      uint32_t sr[2][32];
      auto fetch = [&](int x) {
#pragma unroll
        for (int i = 0; i < 2; ++i) tmem_ld_32x32b_x32(s_col + 64 * x + 32 * i, sr[i]);
        tmem_ld_wait();
        if (masked) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t seen = seen_word(span, key0 + 64 * x + 32 * i);
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(seen & (1u << e))) sr[i][e] = 0xff800000u;
          }
        }
      };
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int x = 0; x < C::kKeys / 64; ++x) {
        fetch(x);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 16; e += 2)
            mx[i] = fmax3(mx[i], __uint_as_float(sr[i / 2][16 * (i % 2) + e]),
                          __uint_as_float(sr[i / 2][16 * (i % 2) + e + 1]));
      }
      const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c;
      const bool grow = top > m + kSlack;
      if (j > 0 && __any_sync(0xffffffffu, grow)) {
        // O as the products of the blocks before left it: they came before these scores
        const float f = grow ? ex2_approx(m - top) : 1.f;
        l *= f;
#pragma unroll 1
        for (int d = 0; d < D; d += 32) {
          uint32_t o[32];
          tmem_ld_32x32b_x32(o_col + d, o);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
          tmem_st_32x32b_x32(o_col + d, o);
        }
      }
      if (grow) m = top;
      const float off = m == -INFINITY ? 0.f : m;
      const uint64_t off2 = pack_f32x2(-off, -off);
      uint64_t sum2[2] = {0, 0};
      // P in the inputs' type, which the product with V takes: 2^-9 (bf16) or 2^-12 (fp16) of each p at
      // most. The sums are of P unrounded.
#pragma unroll
      for (int x = 0; x < C::kKeys / 64; ++x) {
        if (C::kKeys > 64) fetch(x);
        uint32_t pk[2][16];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            uint64_t v;
            asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(sr[i][e]), "r"(sr[i][e + 1]));
            asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(v), "l"(c2), "l"(off2));
            float a, b;
            asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
            a = ex2_approx(a);
            b = ex2_approx(b);
            asm("add.rn.f32x2 %0, %0, %1;" : "+l"(sum2[e / 2 % 2]) : "l"(pack_f32x2(a, b)));
            pk[i][e / 2] = pack16<F16>(a, b);
          }
#pragma unroll
        for (int i = 0; i < 2; ++i) tmem_st_32x32b_x16(s_col + 32 * x + 16 * i, pk[i]);
      }
      {
        float a0, b0, a1, b1;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(a0), "=f"(b0) : "l"(sum2[0]));
        asm("mov.b64 {%0, %1}, %2;" : "=f"(a1), "=f"(b1) : "l"(sum2[1]));
        l += (a0 + b0) + (a1 + b1);
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kPFull + 2 * t + h));
    }
    if (count > 0) wait_warp(bar(C::kOFull + t), 0, p.err, ERR_WAIT_MMA);
    tc_fence_after();
    // the halves on the larger maximum
    float f0 = 1.f, f1 = 0.f;
    if (C::kHalves == 2) {
      ml[(2 * t + h) * kTile + row] = make_float2(m, l);
      named_barrier(1 + t, 256);
      const float2 a = ml[2 * t * kTile + row], b = ml[(2 * t + 1) * kTile + row];
      m = fmaxf(a.x, b.x);
      const float at = m == -INFINITY ? 0.f : m;
      f0 = ex2_approx(a.x - at);
      f1 = ex2_approx(b.x - at);
      l = fmaf(f0, a.y, f1 * b.y);
    }
    if (!sees || count == 0) l = 0.f, m = -INFINITY;
    const bool whole = p.parts == 1;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int head = group * p.y.per + row % p.y.per;
    uint16_t* out = static_cast<uint16_t*>(p.out.p) + static_cast<int64_t>(token) * p.out.token +
                    static_cast<int64_t>(head) * p.out.head;
    const int64_t slot =
        ((static_cast<int64_t>(group) * p.pairs + pair) * p.parts + part) * 2 * kTile + t * kTile + row;
    float* part_o = whole ? nullptr : p.part_o + slot * D;
#pragma unroll 1
    for (int d = h * (D / C::kHalves); d < (h + 1) * (D / C::kHalves); d += 32) {
      float o[32];
      if (count > 0) {
        uint32_t a[32];
        tmem_ld_32x32b_x32(tmem + lane_off + C::kColO + 128u * t + d, a);
        if (C::kHalves == 2) {
          uint32_t b[32];
          tmem_ld_32x32b_x32(tmem + lane_off + C::kColO + 128u * t + 64u + d, b);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e)
            o[e] = fmaf(f0, __uint_as_float(a[e]), f1 * __uint_as_float(b[e]));
        } else {
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(a[e]);
        }
      }
      if (!valid) continue;
      if (whole) {
#pragma unroll
        for (int e = 0; e < 32; e += 8) {
          uint32_t v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[i] = l == 0.f ? 0u : pack16<F16>(o[e + 2 * i] * inv, o[e + 2 * i + 1] * inv);
          *reinterpret_cast<uint4*>(out + d + e) = make_uint4(v[0], v[1], v[2], v[3]);
        }
      } else if (l != 0.f) {
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          *reinterpret_cast<float4*>(part_o + d + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      }
    }
    if (h == 0 && valid) {
      if (whole)
        p.lse[static_cast<int64_t>(head) * p.y.n_q + token] =
            l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      else
        p.part_ml[slot] = make_float2(m, l);
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// A row's parts, added up in their order: D threads a row.
template <bool F16, int D>
__global__ void __launch_bounds__(256) span_join_kernel(const __grid_constant__ SpanFwd p) {
  grid_dep_wait();
  grid_dep_launch();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * (256 / D) + threadIdx.x / D;
  const int d = threadIdx.x % D;
  if (i >= static_cast<int64_t>(p.y.n_q) * p.y.heads) return;
  const int token = static_cast<int>(i / p.y.heads), head = static_cast<int>(i % p.y.heads);
  const int group = head / p.y.per, tile = token / p.y.tile_tokens;
  const int row = (token - tile * p.y.tile_tokens) * p.y.per + head % p.y.per;
  const int64_t first = (static_cast<int64_t>(group) * p.pairs + tile / 2) * p.parts * 2 * kTile +
                        tile % 2 * kTile + row;
  float m = -INFINITY;
  for (int c = 0; c < p.parts; ++c) m = fmaxf(m, __ldcg(&p.part_ml[first + c * 2 * kTile].x));
  float l = 0.f, o = 0.f;
#pragma unroll 4
  for (int c = 0; c < p.parts; ++c) {
    const int64_t at = first + c * 2 * kTile;
    const float2 x = __ldcg(p.part_ml + at);
    if (x.y == 0.f) continue;
    const float f = ex2_approx(x.x - m);
    l = fmaf(f, x.y, l);
    o = fmaf(f, __ldcg(p.part_o + at * D + d), o);
  }
  using T = typename std::conditional<F16, __half, __nv_bfloat16>::type;
  static_cast<T*>(p.out.p)[static_cast<int64_t>(token) * p.out.token +
                           static_cast<int64_t>(head) * p.out.head + d] = T(l == 0.f ? 0.f : o / l);
  if (d == 0)
    p.lse[static_cast<int64_t>(head) * p.y.n_q + token] =
        l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Parts of every pair's key blocks: as many as fill the GPU where there are few pairs.
int fwd_parts(const SpanShape& y) {
  const int64_t units = static_cast<int64_t>(y.groups) * ((y.row_tiles + 1) / 2);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(y.key_blocks, num_sms() / units)));
}

template <bool F16, int D>
cudaError_t launch_fwd(const SpanFwd& p, const SpanRows& q, const SpanRows& k, const SpanRows& v,
                       cudaStream_t s) {
  using C = FwdCfg<D>;
  CUtensorMap tmQ, tmK, tmV;
  if (!make_map(&tmQ, F16, q.p, D, p.y.heads, p.y.n_q, 1, q.head, q.token, 0, p.y.per, p.y.tile_tokens) ||
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
  e = launch_pdl(span_fwd_kernel<F16, D>, dim3(p.pairs * p.parts, p.y.groups), dim3(C::kThreads),
                 C::kSmem, s, tmQ, tmK, tmV, p);
  if (e != cudaSuccess || p.parts == 1) return e;
  const int64_t rows = static_cast<int64_t>(p.y.n_q) * p.y.heads;
  return launch_pdl(span_join_kernel<F16, D>, dim3(static_cast<unsigned>((rows + 256 / D - 1) / (256 / D))),
                    dim3(256), 0, s, p);
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
  return static_cast<size_t>(groups) * ((y.row_tiles + 1) / 2) * parts * 2 * kTile *
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
      !fd::span_rows_ok(outr, a->n_q, a->heads, a->head_dim) ||
      (a->n_k > 0 && (!fd::span_rows_ok(kr, a->n_k, a->groups, a->head_dim) ||
                      !fd::span_rows_ok(vr, a->n_k, a->groups, a->head_dim))) ||
      !fd::span_ptr(spans, 8) || !fd::span_ptr(lse, 4) || !fd::span_ptr(err_dev, 4))
    return FD_ERR_INVALID_ARG;
  const size_t need =
      fd::span_fwd_workspace_bytes(a->n_q, a->n_k, a->heads, a->groups, a->head_dim);
  if (need > 0 && !fd::span_ptr(workspace, 16)) return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  fd::SpanFwd p{};
  p.y = fd::span_shape(a->n_q, a->n_k, a->heads, a->groups);
  p.pairs = (p.y.row_tiles + 1) / 2;
  p.parts = a->n_k > 0 ? fd::fwd_parts(p.y) : 1;
  p.spans = spans;
  p.scale_log2 = a->scale * fd::kLog2e;
  p.out = outr;
  p.lse = lse;
  const int64_t rows = static_cast<int64_t>(p.y.groups) * p.pairs * p.parts * 2 * fd::kTile;
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
