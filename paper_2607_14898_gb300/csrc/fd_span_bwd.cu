// Gradient of the attention in spans of keys (fd_op_span_attention_bwd). The probabilities are
// computed again from the log-sum-exp, tile by tile, and never stored:
//   P = exp(scale q k^T - lse),  delta = rowsum(dout o out),  dS = P (dout v^T - delta)
//   dv = P^T dout,  dk = scale dS^T q  (over the rows of a group's heads),  dq = scale dS k
//
//   span_rows   each row's lse and delta, each row tile's limits; in fp16 the sizes that dS is scaled by
//   span_grad   keys_block: dk and dv of 128 keys, a walk over the row tiles that see some of them
//               query_block: dq of a row tile, a walk over its key blocks
// Scores and dout v^T are computed twice, 7 products for the 5 that are needed, so that every sum stays
// in one block's TMEM: no atomics, the same bits every time.
//
// Bound by the chain from the scores through P and dS to the products that wait for them; all 7 products
// of the measured cuBLAS rate:
//   9360 queries in chunks of 1560, each sees up to 4; 16 heads of 64 on 4   522 us  1203 TFLOP/s, 64 %
//   8191 causal tokens, 32 heads of 128 on 8                    1177 to 1195 us  1633 TFLOP/s, 86 %
//   the same in fp16, whose scales cost a look at sizes in every block        560 us, 1297 us
// (a smaller clip: tensor cores 50 % busy, issue slots 58 %; fewer causal tokens: 66 % and 50 %). Dropped: X
// and Y read together, with dS told a step later (688 us to 1056 for the first).
#include <algorithm>
#include <cmath>

#include "fd_span.cuh"

namespace fd {
namespace {

struct SpanBwd {
  SpanShape y;
  int q_parts, k_parts;
  const int32_t* spans;
  float scale, scale_log2;
  SpanRows v, out, dout, dq, dk, dv;
  const float* lse;
  float* stat;    // [group][row tile] records of kRecord: see below
  int4* limits;   // of each row tile, those of its records
  // fp16: A = sum |dout_i| and A max |out_i| of each row, [group][row tile][128]; the largest of a token's heads behind
  // its span, [group][token]; those of a row tile, [group][row tile]; exponents (a byte) of each key's
  // max |v_i|, [group][key block][128], and the largest of a key block, [group][key block]
  float2* size_row;
  float4* size_token;
  float2* size_tile;
  uint8_t *v_exp, *v_most;
  float* part_q;  // [group][row tile][part][D / 4][128 rows] of four
  float* part_k;  // [group][key block][part][dk, dv][D / 4][128 keys] of four
  int* err;
};

// fp16 has few exponents: P goes into its product times 2^14, and dS times a power of two by which its bound
// |dS_tj| <= sum_i |dout_ti| (max |v_ji| + max |out_ti|) comes between 2^14 and 2^15: none is infinite, and small ones
// keep their digits down to 2^-28 of the bound. The bound is that of the row for dq, over the keys that it sees, and that
// of the key for dk, over the rows that see it (a lane has one row or key, and with it one scale): nothing of
// another sequence comes in. bf16 has fp32's range.
constexpr float kPUp = 16384.f;
constexpr float kPUpLog2 = 14.f;

// What a row tile's record holds, 16 bytes in line: -lse log2(e), -delta and the ends of the span (int) of
// each row, [4][128], then the tile's limits: {first key, end of the keys} that some query sees, {first, end}
// of those that all queries see which see any; the third is negative (~) where some query sees none, the fourth
// where some query sees one.
constexpr int kRecord = 4 * kTile + 4;

__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int i = 16; i; i >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, i));
  return x;
}

__device__ __forceinline__ float2 larger(float2 a, float2 b) {
  return make_float2(fmaxf(a.x, b.x), fmaxf(a.y, b.y));
}

// ------------------------------------------------------------------------------ rows
// The largest magnitude of eight numbers, and that of both halves of such a pair, as bits
__device__ __forceinline__ uint32_t top_of(const uint4& a) {
  const uint32_t m = 0x7fff7fffu;
  return __vmaxu2(__vmaxu2(a.x & m, a.y & m), __vmaxu2(a.z & m, a.w & m));
}
__device__ __forceinline__ float top_half(uint32_t x) {
  return __half2float(__ushort_as_half(static_cast<unsigned short>(max(x & 0xffffu, x >> 16))));
}

// The exponents of a key block's max |v_i|, D / 8 lanes a key (those of keys that nothing sees are not looked at).
template <int D>
__device__ __forceinline__ void key_sizes(const SpanBwd& p, int kb, int group) {
  constexpr int kLanes = D / 8;
  __shared__ uint32_t top[8];
  const int lane = threadIdx.x % kLanes;
  const int64_t block = static_cast<int64_t>(group) * p.y.key_blocks + kb;
  uint32_t most = 0;
#pragma unroll
  for (int row = threadIdx.x / kLanes; row < kTile; row += 256 / kLanes) {
    const int key = kb * kTile + row;
    uint32_t of_v = 0;
    if (key < p.y.n_k)
      of_v = top_of(__ldg(reinterpret_cast<const uint4*>(
          static_cast<const uint16_t*>(p.v.p) + key * p.v.token + group * p.v.head + lane * 8)));
#pragma unroll
    for (int i = kLanes / 2; i; i >>= 1) of_v = __vmaxu2(of_v, __shfl_xor_sync(0xffffffffu, of_v, i));
    const uint32_t e = __float_as_uint(top_half(of_v)) >> 23;
    if (lane == 0) p.v_exp[block * kTile + row] = static_cast<uint8_t>(e);
    most = max(most, e);
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if ((threadIdx.x & 31) == 0) top[threadIdx.x >> 5] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 0; i < 8; ++i) most = max(most, top[i]);
    p.v_most[block] = static_cast<uint8_t>(most);
  }
}

// D / 8 lanes a row. A row that sees nothing, or is none, gets P = 0 by an infinite lse.
template <bool F16, int D>
__global__ void __launch_bounds__(256) span_rows_kernel(const __grid_constant__ SpanBwd p) {
  constexpr int kLanes = D / 8;
  __shared__ float2 size[kTile];
  grid_dep_wait();
  grid_dep_launch();
  const int tile = blockIdx.x, group = blockIdx.y;
  const int lane = threadIdx.x % kLanes;
  if (F16 && tile >= p.y.row_tiles) {
    key_sizes<D>(p, tile - p.y.row_tiles, group);
    return;
  }
  const int token0 = tile * p.y.tile_tokens;
  float* stat = p.stat + (static_cast<int64_t>(group) * p.y.row_tiles + tile) * kRecord;
#pragma unroll
  for (int row = threadIdx.x / kLanes; row < kTile; row += 256 / kLanes) {
    const int token = token0 + row / p.y.per, head = group * p.y.per + row % p.y.per;
    const bool valid = row < p.y.tile_rows && token < p.y.n_q;
    const int2 span = valid ? span_of(p.spans, token, p.y.n_k) : make_int2(0, 0);
    const bool sees = span.x < span.y;
    float sum = 0.f, of_dout = 0.f;
    uint32_t of_out = 0;
    if (sees) {
      const uint4 a = __ldg(reinterpret_cast<const uint4*>(
          static_cast<const uint16_t*>(p.out.p) + token * p.out.token + head * p.out.head + lane * 8));
      const uint4 b = __ldg(reinterpret_cast<const uint4*>(
          static_cast<const uint16_t*>(p.dout.p) + token * p.dout.token + head * p.dout.head + lane * 8));
      const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
      if (F16) of_out = top_of(a);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float2 u, v;
        if (F16) {
          u = __half22float2(*reinterpret_cast<const __half2*>(&x[i]));
          v = __half22float2(*reinterpret_cast<const __half2*>(&y[i]));
          of_dout += fabsf(v.x) + fabsf(v.y);
        } else {
          u = make_float2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
          v = make_float2(__uint_as_float(y[i] << 16), __uint_as_float(y[i] & 0xffff0000u));
        }
        sum = fmaf(u.x, v.x, fmaf(u.y, v.y, sum));
      }
    }
#pragma unroll
    for (int i = kLanes / 2; i; i >>= 1) {
      sum += __shfl_xor_sync(0xffffffffu, sum, i);
      if (F16) {
        of_dout += __shfl_xor_sync(0xffffffffu, of_dout, i);
        of_out = __vmaxu2(of_out, __shfl_xor_sync(0xffffffffu, of_out, i));
      }
    }
    if (F16 && lane == 0) {
      const float2 both = make_float2(of_dout, of_dout * top_half(of_out));
      size[row] = both;
      p.size_row[(static_cast<int64_t>(group) * p.y.row_tiles + tile) * kTile + row] = both;
    }
    if (lane == 0) {
      const float l = sees ? __ldg(p.lse + static_cast<int64_t>(head) * p.y.n_q + token) : 0.f;
      stat[row] = sees ? fmaf(-l, kLog2e, F16 ? kPUpLog2 : 0.f) : -INFINITY;
      stat[kTile + row] = sees ? -sum : 0.f;
      reinterpret_cast<int*>(stat)[2 * kTile + row] = span.x;
      reinterpret_cast<int*>(stat)[3 * kTile + row] = span.y;
    }
  }
  if (F16) __syncthreads();
  if (threadIdx.x < 32) {
    int4 m = make_int4(0x7fffffff, 0, 0, 0x7fffffff);
    bool none = false, one = false;
    float2 most = make_float2(0.f, 0.f);  // of the tile
    for (int i = threadIdx.x; i < p.y.tile_tokens && token0 + i < p.y.n_q; i += 32) {
      const int2 s = span_of(p.spans, token0 + i, p.y.n_k);
      if (F16) {
        float2 of_token = make_float2(0.f, 0.f);
        for (int h = 0; h < p.y.per; ++h) of_token = larger(of_token, size[i * p.y.per + h]);
        p.size_token[static_cast<int64_t>(group) * p.y.n_q + token0 + i] =
            make_float4(__int_as_float(s.x), __int_as_float(s.y), of_token.x, of_token.y);
        most = larger(most, of_token);
      }
      if (s.x < s.y) {
        m.x = min(m.x, s.x);
        m.y = max(m.y, s.y);
        m.z = max(m.z, s.x);
        m.w = min(m.w, s.y);
        one |= s.x + 1 == s.y;
      } else {
        none = true;
      }
    }
    m.x = __reduce_min_sync(0xffffffffu, m.x);
    m.y = __reduce_max_sync(0xffffffffu, m.y);
    m.z = __reduce_max_sync(0xffffffffu, m.z);
    m.w = __reduce_min_sync(0xffffffffu, m.w);
    if (__any_sync(0xffffffffu, none)) m.z = ~m.z;
    if (__any_sync(0xffffffffu, one)) m.w = ~m.w;
    if (F16) most = make_float2(warp_max(most.x), warp_max(most.y));
    if (threadIdx.x == 0) {
      if (F16) p.size_tile[group * p.y.row_tiles + tile] = most;
      *reinterpret_cast<int4*>(stat + 4 * kTile) = m;
      if (group == 0) p.limits[tile] = m;
    }
  }
}

// The power of two that brings the bound of a lane's dS between 2^14 and 2^15, from its rows' sizes and the exponent
// of its keys' (1 where nothing is seen, or all is zero).
__device__ __forceinline__ float down_scale(float2 size, uint32_t v_exp) {
  // |v_i| < 2^(v_exp - 126)
  const float bound = size.x > 0.f ? fmaf(size.x, __uint_as_float((v_exp + 1) << 23), size.y) : 0.f;
  const uint32_t e = __float_as_uint(bound) >> 23;  // (of fp16 numbers: 79 to 167 unless it is zero)
  return e > 14u && e < 255u ? __uint_as_float((268u - e) << 23) : 1.f;
}

// ------------------------------------------------------------------------------ keys: dk and dv
// Lanes are keys and columns rows of the tile: X = K Q^T and Y = V dout^T into TMEM, P^T and dS^T
// from there back into TMEM as the first operands of dv += P^T dout and dk += dS^T q.
//   warps 0-15   P and dS: four groups of 128 threads (a key each), a quarter of a step's rows each
//   warps 16-19  products: X, Y, dv, dk (a warp issues one per 104 to 158 cycles); the last one loads K and
//                V, then q, dout and the rows' records by tiles, each when dk has gone into its place's
//                last tile (a twenty-first warp would leave 80 registers a thread, not 96)
// A step is a tile, or (D = 128, where TMEM has no room for more) half of one. (D = 64 in halves too, each
// with eight warps and a place in TMEM of its own so that their chains run apart: 577 us instead of 554 for the
// 480p clip's gradient.)
template <int D>
struct KeyCfg {
  static constexpr int kThreads = 20 * 32;
  static constexpr int kStep = D == 64 ? 128 : 64;  // rows of a step
  static constexpr int kSteps = kTile / kStep;      // of a tile
  static constexpr int kCols = kStep / 4;           // of a thread
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kStages = D == 64 ? 4 : 2;
  static constexpr int kStat = kRecord * 4;
  static constexpr int kOffV = kTileBytes;
  static constexpr int kOffRing = 2 * kTileBytes;  // q, dout of each stage
  static constexpr int kOffStat = kOffRing + kStages * 2 * kTileBytes;
  static constexpr int kOffBar = kOffStat + kStages * kStat;
  static constexpr int kKV = 0, kFull = 1, kFree = kFull + kStages, kReady = kFree + kStages,
                       kXFull = kReady + kStages, kYFull = kXFull + 1, kXRead = kYFull + 1,
                       kYRead = kXRead + 1, kPFull = kYRead + 1, kDsFull = kPFull + 1,
                       kPDone = kDsFull + 1, kDsDone = kPDone + 1, kDone = kDsDone + 1, kBars = kDone + 4;
  static constexpr int kOffSize = kOffBar + (kBars * 8 + 32 + 127) / 128 * 128;  // fp16: [16 warps][32 tokens]
  static constexpr int kOffAll = kOffSize + 16 * 32 * 16;  // [4][128]
  static constexpr int kSmem = kOffAll + 4 * kTile * 8;
  static constexpr uint32_t kColX = 0, kColY = kStep, kColP = 2 * kStep, kColDs = kColP + kStep / 2,
                            kColDv = 512 - 2 * D, kColDk = 512 - D;
  static_assert(kSmem <= 227 * 1024 && kColDs + kStep / 2 <= kColDv, "room");
};

template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t at, uint32_t (&r)[N]) {
  if constexpr (N == 32)
    tmem_ld_32x32b_x32(at, r);
  else
    tmem_ld_32x32b_x16(at, r);
}
template <int N>
__device__ __forceinline__ void tmem_st(uint32_t at, const uint32_t (&r)[N]) {
  if constexpr (N == 16)
    tmem_st_32x32b_x16(at, r);
  else
    tmem_st_32x32b_x8(at, r);
}

// 16 columns of an accumulator times f, columns d.. of a row: into a tile in shared memory (rows that are not
// `here` as zeros), or as floats to a part's place, [D / 4][128] of four.
template <bool F16>
__device__ __forceinline__ void leave16(uint32_t at, float f, bool here, uint8_t* tile, float4* part, int row,
                                        int d) {
  uint32_t a[16];
  tmem_ld_32x32b_x16(at, a);
  tmem_ld_wait();
  float o[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) o[e] = here ? __uint_as_float(a[e]) * f : 0.f;
  if (part == nullptr) {
#pragma unroll
    for (int e = 0; e < 16; e += 8)
      *reinterpret_cast<uint4*>(tile + tile_chunk(row, (d + e) / 8)) =
          make_uint4(pack16<F16>(o[e], o[e + 1]), pack16<F16>(o[e + 2], o[e + 3]),
                     pack16<F16>(o[e + 4], o[e + 5]), pack16<F16>(o[e + 6], o[e + 7]));
  } else {
#pragma unroll
    for (int e = 0; e < 16; e += 4)
      part[(d + e) / 4 * kTile + row] = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
  }
}
// the same of zeros
__device__ __forceinline__ void leave16_none(uint8_t* tile, float4* part, int row, int d) {
  if (part == nullptr) {
#pragma unroll
    for (int e = 0; e < 16; e += 8)
      *reinterpret_cast<uint4*>(tile + tile_chunk(row, (d + e) / 8)) = make_uint4(0, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 16; e += 4) part[(d + e) / 4 * kTile + row] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
}

// The largest sizes of the rows that see a thread's key (fp16), by warps 0-15: the four warps of a key share the
// tokens out, 32 at a time, and leave what they find in shared memory.
template <int D>
struct KeySizes {
  const SpanBwd& p;
  const int group, lane, q, at, key;  // at: the key's place in the block
  float4* const mine;
  float2* const all;  // [quarter][key]
  float2 size = make_float2(0.f, 0.f);

  __device__ __forceinline__ KeySizes(const SpanBwd& p, uint8_t* smem, int group, int key0)
      : p(p), group(group), lane(threadIdx.x & 31), q(threadIdx.x >> 7), at(threadIdx.x & 127), key(key0 + at),
        mine(reinterpret_cast<float4*>(smem + KeyCfg<D>::kOffSize) + (threadIdx.x >> 5) * 32),
        all(reinterpret_cast<float2*>(smem + KeyCfg<D>::kOffAll)) {}
  __device__ __forceinline__ float4 token(int t, int end) const {
    return t + lane < end ? __ldcg(p.size_token + static_cast<int64_t>(group) * p.y.n_q + t + lane)
                          : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void look_at(const float4& tokens, int count) {
    mine[lane] = tokens;
    __syncwarp();
#pragma unroll 1
    for (int i0 = 0; i0 < count; i0 += 8)
#pragma unroll
      for (int i = i0; i < i0 + 8; ++i) {
        const float4 x = mine[i];
        if (__float_as_int(x.x) <= key && key < __float_as_int(x.y))
          size = larger(size, make_float2(x.z, x.w));
      }
    __syncwarp();
  }
  // Row tiles [first, end), every fourth of them. A tile whose rows see all of the block's keys, or none, counts as a
  // whole; of the others every token is looked at, the next ones on their way meanwhile.
  __device__ __forceinline__ void look_at_tiles(int first, int end) {
    const int key0 = key - at, keys_end = min(key0 + kTile, p.y.n_k);
    float2 of_tiles = make_float2(0.f, 0.f);
    int held = 0;
    float4 x;
#pragma unroll 1
    for (int i0 = first + q; i0 < end; i0 += 128) {
      const int tile = i0 + 4 * lane;
      bool some = false;
      if (tile < end) {
        const int4 m = __ldcg(p.limits + tile);
        const float2 of_tile = __ldcg(p.size_tile + group * p.y.row_tiles + tile);
        if (m.x < keys_end && m.y > key0) {
          some = (m.z < 0 ? ~m.z : m.z) > key0 || (m.w < 0 ? ~m.w : m.w) < keys_end;
          if (!some) of_tiles = larger(of_tiles, of_tile);
        }
      }
#pragma unroll 1
      for (uint32_t left = __ballot_sync(0xffffffffu, some); left; left &= left - 1) {
        const int token0 = (i0 + 4 * (__ffs(left) - 1)) * p.y.tile_tokens;
        const int token1 = min(token0 + p.y.tile_tokens, p.y.n_q);
#pragma unroll 1
        for (int t = token0; t < token1; t += 32) {
          const float4 next = token(t, token1);
          if (held > 0) look_at(x, held);
          x = next;
          held = min(32, token1 - t);
        }
      }
    }
    if (held > 0) look_at(x, held);
    size = larger(size, make_float2(warp_max(of_tiles.x), warp_max(of_tiles.y)));
  }
  __device__ __forceinline__ void leave() const { all[q * kTile + at] = size; }
  // of all four, after a barrier
  __device__ __forceinline__ float2 found() const {
    return larger(larger(all[at], all[kTile + at]), larger(all[2 * kTile + at], all[3 * kTile + at]));
  }
};
// So few tokens are all looked at, while the limits of the tiles are on their way (2 sequences of 77 each, 6 heads of 64
// on 2: 17.4 us, by tiles 17.9).
constexpr int kFewTokens = 256;

template <bool F16, int D>
__device__ __forceinline__ void keys_block(const CUtensorMap& tmQ, const CUtensorMap& tmDo,
                                           const CUtensorMap& tmK, const CUtensorMap& tmV,
                                           const CUtensorMap& tmDk, const CUtensorMap& tmDv,
                                           const SpanBwd& p, int unit) {
  using C = KeyCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem);
  const bool aligned = (base & 1023u) == 0;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kOffBar);
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * static_cast<uint32_t>(i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
  int* range = reinterpret_cast<int*>(tmem_slot + 1);  // first row tile, the one past the last

  const int part = unit % p.k_parts, kb = unit / p.k_parts % p.y.key_blocks;
  const int group = unit / (p.k_parts * p.y.key_blocks);
  const int key0 = kb * kTile;

  // rows past tile_rows are never loaded
  if (p.y.tile_rows < kTile) {
    for (int i = threadIdx.x; i < C::kStages * 2 * C::kTileBytes / 16; i += C::kThreads)
      reinterpret_cast<uint4*>(smem + C::kOffRing)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  if (threadIdx.x == 19 * 32) {
    if (!aligned) atomicOr(p.err, ERR_SMEM_ALIGN);
    prefetch_tmap(&tmQ);
    prefetch_tmap(&tmDo);
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
    mbar_init(bar(C::kKV), 1);
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(bar(C::kFull + i), 1);
      mbar_init(bar(C::kFree + i), 2);
      mbar_init(bar(C::kReady + i), 1);
    }
    mbar_init(bar(C::kXFull), 1);
    mbar_init(bar(C::kYFull), 1);
    mbar_init(bar(C::kXRead), 16);
    mbar_init(bar(C::kYRead), 16);
    mbar_init(bar(C::kPFull), 16);
    mbar_init(bar(C::kDsFull), 16);
    mbar_init(bar(C::kPDone), 1);
    for (int i = 0; i < 4; ++i) mbar_init(bar(C::kDone + i), 1);
    mbar_init(bar(C::kDsDone), 1);
    fence_barrier_init();
    range[0] = 0x7fffffff;
    range[1] = 0;
  }
  grid_dep_wait();
  grid_dep_launch();
  if (warp == 0) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  } else if (threadIdx.x == 19 * 32 && aligned) {
    mbar_expect_tx(bar(C::kKV), 2 * C::kTileBytes);
    for (int d = 0; d < D / 64; ++d) {
      tma_load_4d(base + d * kSub, &tmK, bar(C::kKV), 64 * d, group, key0, 0);
      tma_load_4d(base + C::kOffV + d * kSub, &tmV, bar(C::kKV), 64 * d, group, key0, 0);
    }
  }
  __syncthreads();
  KeySizes<D> sizes(p, smem, group, key0);
  const bool few = p.y.n_q <= kFewTokens;
  uint32_t v_exp = 0;
  if (F16 && warp < 16)
    v_exp = __ldcg(p.v_exp + (static_cast<int64_t>(group) * p.y.key_blocks + kb) * kTile + sizes.at);
  {
    // the row tiles that see some of the keys: from the first to the last
    int first = 0x7fffffff, end = 0;
    float4 tokens[kFewTokens / 128];
    if (F16 && few && warp < 16) {
#pragma unroll
      for (int i = 0; i < kFewTokens / 128; ++i) tokens[i] = sizes.token((4 * i + sizes.q) * 32, p.y.n_q);
    }
    for (int i = threadIdx.x; i < p.y.row_tiles; i += C::kThreads) {
      const int4 m = __ldcg(p.limits + i);
      if (m.x < key0 + kTile && m.y > key0) {
        first = min(first, i);
        end = max(end, i + 1);
      }
    }
    first = __reduce_min_sync(0xffffffffu, first);
    end = __reduce_max_sync(0xffffffffu, end);
    if (lane == 0 && end > 0) {
      atomicMin(range, first);
      atomicMax(range + 1, end);
    }
    if (F16 && few && warp < 16) {
#pragma unroll
      for (int i = 0; i < kFewTokens / 128; ++i)
        sizes.look_at(tokens[i], min(32, p.y.n_q - (4 * i + sizes.q) * 32));
      sizes.leave();
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int n = aligned && range[1] > 0 ? range[1] - range[0] : 0;
  const int tile0 = range[0] + static_cast<int>(static_cast<int64_t>(n) * part / p.k_parts);
  const int count = static_cast<int>(static_cast<int64_t>(n) * (part + 1) / p.k_parts) -
                    static_cast<int>(static_cast<int64_t>(n) * part / p.k_parts);
  float ds_down = 1.f;  // the key's dS are kept times this
  if (F16 && warp < 16) {
    if (!few) {
      if (range[1] > 0) sizes.look_at_tiles(range[0], range[1]);  // (else the first one is the largest int)
      sizes.leave();
      named_barrier(1, 512);
    }
    ds_down = down_scale(sizes.found(), v_exp);
  }

  if (count == 0) {
    // no row sees any of the keys (which may be on their way to where zeros leave from; and nothing may be in flight
    // when the block exits)
    if (warp < 16 && aligned) {
      wait(bar(C::kKV), 0, p.err, ERR_WAIT_TMA, true);
      __syncwarp();
    }
  } else if (warp == 16 || warp == 17) {
    // ---- X = K Q^T (16), Y = V dout^T (17), and zeros for the rows of queries that see nothing:
    // their P and dS are 0, but 0 times NaN is NaN
    const bool y = warp == 17;
    constexpr uint32_t idesc = Mma<F16, D>::idesc(C::kStep, false);
    const uint64_t a0 = sdesc_k_sw128(base + (y ? C::kOffV : 0));
    const uint32_t col = tmem + (y ? C::kColY : C::kColX);
    bool ok = wait_warp(bar(C::kKV), 0, p.err, ERR_WAIT_TMA);
    for (int i = 0; i < count && ok; ++i) {
      const int st = i % C::kStages;
      ok = wait_warp(bar(C::kFull + st), (i / C::kStages) & 1, p.err, ERR_WAIT_TMA);
      if (!ok) break;
      const int off = C::kOffRing + st * 2 * C::kTileBytes + (y ? C::kTileBytes : 0);
      const int4 m = *reinterpret_cast<const int4*>(smem + C::kOffStat + st * C::kStat + 16 * kTile);
      if (m.z < 0) {  // some query sees nothing
        const int* ends = reinterpret_cast<const int*>(smem + C::kOffStat + st * C::kStat) + 2 * kTile;
#pragma unroll 1
        for (int r = lane; r < p.y.tile_rows; r += 32) {
          if (ends[r] < ends[kTile + r]) continue;
          uint4* row = reinterpret_cast<uint4*>(smem + off + r * 128);
#pragma unroll
          for (int d = 0; d < D / 64; ++d)
#pragma unroll
            for (int c = 0; c < 8; ++c) row[d * (kSub / 16) + c] = make_uint4(0, 0, 0, 0);
        }
        fence_proxy_async_smem();
        __syncwarp();
      }
      if (y && lane == 0) mbar_arrive(bar(C::kReady + st));
#pragma unroll
      for (int s = 0; s < C::kSteps; ++s) {
        const int k = i * C::kSteps + s;
        if (k > 0)
          ok = ok && wait_warp(bar(y ? C::kYRead : C::kXRead), (k - 1) & 1, p.err, ERR_WAIT_EPI);
        if (!ok) break;
        tc_fence_after();
        const uint64_t b0 = sdesc_k_sw128(base + off + s * C::kStep * 128);
#pragma unroll
        for (int d = 0; d < D / 64; ++d)
          mma4_bf16_ss_w(col, a0 + static_cast<uint64_t>(d * (kSub >> 4)),
                         b0 + static_cast<uint64_t>(d * (kSub >> 4)), idesc, d > 0);
        mma_commit_w(bar(y ? C::kYFull : C::kXFull));
      }
    }
    products_done(bar(C::kDone + (y ? 1 : 0)), p.err);
  } else if (warp >= 18) {
    // ---- dv += P^T dout (18), dk += dS^T q and the loads (19)
    const bool dk = warp == 19;
    constexpr uint32_t idesc = Mma<F16, D>::idesc(D, true);
    const uint32_t a = tmem + (dk ? C::kColDs : C::kColP), acc = tmem + (dk ? C::kColDk : C::kColDv);
    auto load = [&](int i) {
      const int st = i % C::kStages;
      const uint32_t b = bar(C::kFull + st), q = base + C::kOffRing + st * 2 * C::kTileBytes;
      mbar_expect_tx(b, 2 * p.y.tile_rows * D * 2 + C::kStat);
      const int token = (tile0 + i) * p.y.tile_tokens;
      for (int d = 0; d < D / 64; ++d) {
        tma_load_4d(q + d * kSub, &tmQ, b, 64 * d, group * p.y.per, token, 0);
        tma_load_4d(q + C::kTileBytes + d * kSub, &tmDo, b, 64 * d, group * p.y.per, token, 0);
      }
      bulk_load(base + C::kOffStat + st * C::kStat,
                p.stat + (static_cast<int64_t>(group) * p.y.row_tiles + tile0 + i) * kRecord, C::kStat, b);
    };
    int loaded = 0;
    if (dk) {
      if (lane == 0)
        for (int i = 0; i < min(count, C::kStages); ++i) load(i);
      loaded = min(count, C::kStages);
      __syncwarp();
    }
    bool ok = true;
    for (int i = 0; i < count && ok; ++i) {
      const int st = i % C::kStages;
      if (dk && i > 0 && loaded < count) {
        // the tile before is through: the next one to its place
        ok = wait_warp(bar(C::kFree + (i - 1) % C::kStages), ((i - 1) / C::kStages) & 1, p.err,
                       ERR_WAIT_MMA);
        if (!ok) break;
        if (lane == 0) load(loaded);
        __syncwarp();
        ++loaded;
      }
      // (dv does not depend on Y, which waits for dout; dk on both)
      ok = wait_warp(bar(C::kReady + st), (i / C::kStages) & 1, p.err, ERR_WAIT_TMA);
      const uint32_t b = base + C::kOffRing + st * 2 * C::kTileBytes + (dk ? 0 : C::kTileBytes);
#pragma unroll
      for (int s = 0; s < C::kSteps; ++s) {
        const int k = i * C::kSteps + s;
        ok = ok && wait_warp(bar(dk ? C::kDsFull : C::kPFull), k & 1, p.err, ERR_WAIT_EPI);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int x = 0; x < C::kStep / 64; ++x)
          mma4_ts_mn_w(acc, a + 32u * x, sdesc_mn_sw128(b + (s * C::kStep + x * 64) * 128, kSub), idesc,
                       k > 0 || x > 0);
        mma_commit_w(bar(dk ? C::kDsDone : C::kPDone));
      }
      if (ok) mma_commit_w(bar(C::kFree + st));
    }
    products_done(bar(C::kDone + (dk ? 3 : 2)), p.err);
    if (dk && lane == 0) {
      // nothing may be in flight when the block exits
      wait(bar(C::kKV), 0, p.err, ERR_WAIT_TMA, true);
      for (int j = max(0, loaded - C::kStages); j < loaded; ++j)
        wait(bar(C::kFull + j % C::kStages), (j / C::kStages) & 1, p.err, ERR_WAIT_TMA, true);
    }
  }
  if (warp < 16) {
    // ---- P^T and dS^T of a quarter of each step's rows
    const int q = warp >> 2, key = key0 + (warp & 3) * 32 + lane;
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t x_col = tmem + lane_off + C::kColX + C::kCols * q;
    const uint32_t y_col = tmem + lane_off + C::kColY + C::kCols * q;
    const uint32_t p_col = tmem + lane_off + C::kColP + C::kCols / 2 * q;
    const uint32_t ds_col = tmem + lane_off + C::kColDs + C::kCols / 2 * q;
    const uint64_t c2 = pack_f32x2(p.scale_log2, p.scale_log2);
    const float dn = F16 ? ds_down / kPUp : 1.f;
    const uint64_t down2 = pack_f32x2(dn, dn);
    int k = 0;
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      const int st = i % C::kStages;
      bool masked = false, one = false;
#pragma unroll 1
      for (int s = 0; s < C::kSteps; ++s, ++k) {
        const uint8_t* stat = smem + C::kOffStat + st * C::kStat + (s * C::kStep + q * C::kCols) * 4;
        wait_warp(bar(C::kXFull), k & 1, p.err, ERR_WAIT_MMA);
        tc_fence_after();
        uint32_t x[C::kCols];
        tmem_ld(x_col, x);
        if (s == 0) {
          // (a tile between others may see nothing of the block, or nothing at all)
          const int4 m = *reinterpret_cast<const int4*>(smem + C::kOffStat + st * C::kStat + 16 * kTile);
          masked = m.x > key0 || (m.z < 0 ? ~m.z : m.z) > key0 || (m.w < 0 ? ~m.w : m.w) < key0 + kTile;
          one = m.w < 0;
        }
        uint32_t seen = 0xffffffffu;  // bit c: the key is seen by row c of the quarter
        if (masked) {
          // (something that is not predicated, here and below: without it the selections were made for
          // every tile)
          __syncwarp();
          seen = 0;
#pragma unroll
          for (int c = 0; c < C::kCols; c += 4) {
            const int4 lo = *reinterpret_cast<const int4*>(stat + 2 * kTile * 4 + c * 4);
            const int4 hi = *reinterpret_cast<const int4*>(stat + 3 * kTile * 4 + c * 4);
            seen |= (lo.x <= key && key < hi.x ? 1u << c : 0u) |
                    (lo.y <= key && key < hi.y ? 2u << c : 0u) |
                    (lo.z <= key && key < hi.z ? 4u << c : 0u) |
                    (lo.w <= key && key < hi.w ? 8u << c : 0u);
          }
        }
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::kXRead));
        uint32_t y[C::kCols];
        auto read_y = [&]() {
          wait_warp(bar(C::kYFull), k & 1, p.err, ERR_WAIT_MMA);
          tc_fence_after();
          tmem_ld(y_col, y);
          tmem_ld_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::kYRead));
        };
        // (at once where there are registers for both)
        if (C::kCols == 16) read_y();
        uint32_t pk[C::kCols / 2];
#pragma unroll
        for (int c = 0; c < C::kCols; c += 4) {
          const ulonglong2 l = *reinterpret_cast<const ulonglong2*>(stat + c * 4);
          const float2 a = halves_of(fma2(pair_of(x[c], x[c + 1]), c2, l.x));
          const float2 b = halves_of(fma2(pair_of(x[c + 2], x[c + 3]), c2, l.y));
          x[c] = __float_as_uint(ex2_approx(a.x));
          x[c + 1] = __float_as_uint(ex2_approx(a.y));
          x[c + 2] = __float_as_uint(ex2_approx(b.x));
          x[c + 3] = __float_as_uint(ex2_approx(b.y));
        }
        if (masked) {
          __syncwarp();
#pragma unroll
          for (int c = 0; c < C::kCols; ++c)
            if (!(seen & (1u << c))) x[c] = 0;
        }
        // P and dS in the inputs' type, which the products take: half a step each, 2^-9 or 2^-12 of
        // their size; sums in fp32
#pragma unroll
        for (int c = 0; c < C::kCols; c += 2)
          pk[c / 2] = pack16<F16>(__uint_as_float(x[c]), __uint_as_float(x[c + 1]));
        if (k > 0) wait_warp(bar(C::kPDone), (k - 1) & 1, p.err, ERR_WAIT_MMA);
        tc_fence_after();
        tmem_st(p_col, pk);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::kPFull));
        if (C::kCols == 32) read_y();
#pragma unroll
        for (int c = 0; c < C::kCols; c += 4) {
          const ulonglong2 d = *reinterpret_cast<const ulonglong2*>(stat + kTile * 4 + c * 4);
          uint64_t a = pair_of(x[c], x[c + 1]), b = pair_of(x[c + 2], x[c + 3]);
          if (F16) {
            a = mul2(a, down2);
            b = mul2(b, down2);
          }
          const float2 u = halves_of(mul2(a, add2(pair_of(y[c], y[c + 1]), d.x)));
          const float2 v = halves_of(mul2(b, add2(pair_of(y[c + 2], y[c + 3]), d.y)));
          y[c] = __float_as_uint(u.x);
          y[c + 1] = __float_as_uint(u.y);
          y[c + 2] = __float_as_uint(v.x);
          y[c + 3] = __float_as_uint(v.y);
        }
        if (masked) {
          __syncwarp();
          // And where a row sees one key only: P is 1 whatever the scores, so dS is 0, not what rounding
          // leaves of a difference. (A loop: unrolled it took registers from every step, 535 us instead of
          // 520 for the 480p clip.)
          if (one) {
#pragma unroll 1
            for (int c = 0; c < C::kCols; c += 4) {
              const int4 lo = *reinterpret_cast<const int4*>(stat + 2 * kTile * 4 + c * 4);
              const int4 hi = *reinterpret_cast<const int4*>(stat + 3 * kTile * 4 + c * 4);
              const uint32_t four = (lo.x + 1 == hi.x ? 1u : 0u) | (lo.y + 1 == hi.y ? 2u : 0u) |
                                    (lo.z + 1 == hi.z ? 4u : 0u) | (lo.w + 1 == hi.w ? 8u : 0u);
              seen &= ~(four << c);
            }
          }
#pragma unroll
          for (int c = 0; c < C::kCols; ++c)
            if (!(seen & (1u << c))) y[c] = 0;
        }
#pragma unroll
        for (int c = 0; c < C::kCols; c += 2)
          pk[c / 2] = pack16<F16>(__uint_as_float(y[c]), __uint_as_float(y[c + 1]));
        if (k > 0) wait_warp(bar(C::kDsDone), (k - 1) & 1, p.err, ERR_WAIT_MMA);
        tc_fence_after();
        tmem_st(ds_col, pk);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::kDsFull));
      }
    }
    if (count > 0) {
      wait_warp(bar(C::kPDone), (k - 1) & 1, p.err, ERR_WAIT_MMA);
      wait_warp(bar(C::kDsDone), (k - 1) & 1, p.err, ERR_WAIT_MMA);
    }
    tc_fence_after();
    // dk goes through K's place in shared memory, dv through V's: the last products are through
    const int row = (warp & 3) * 32 + lane;
    const int64_t slot = ((static_cast<int64_t>(group) * p.y.key_blocks + kb) * p.k_parts + part) * 2;
    float4* part_k = p.k_parts > 1 ? reinterpret_cast<float4*>(p.part_k) + slot * (D / 4) * kTile : nullptr;
    float4* part_v = p.k_parts > 1 ? part_k + D / 4 * kTile : nullptr;
    const float fk = p.scale / ds_down, fv = F16 ? 1.f / kPUp : 1.f;
#pragma unroll 1
    for (int d = q * (D / 4); d < (q + 1) * (D / 4); d += 16) {
      if (count > 0) {
        leave16<F16>(tmem + lane_off + C::kColDk + d, fk, true, smem, part_k, row, d);
        leave16<F16>(tmem + lane_off + C::kColDv + d, fv, true, smem + C::kOffV, part_v, row, d);
      } else {
        leave16_none(smem, part_k, row, d);
        leave16_none(smem + C::kOffV, part_v, row, d);
      }
    }
    if (p.k_parts == 1) {
      fence_proxy_async_smem();
      named_barrier(1, 512);
      if (threadIdx.x == 0 && aligned) {
        for (int d = 0; d < D / 64; ++d) {
          tma_store_4d(&tmDk, base + d * kSub, 64 * d, group, key0, 0);
          tma_store_4d(&tmDv, base + C::kOffV + d * kSub, 64 * d, group, key0, 0);
        }
        bulk_commit();
        bulk_wait_all();
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------------------ queries: dq
// Lanes are rows of the tile and columns keys: X = q k^T, Y = dout v^T, dS back into TMEM as the first
// operand of dq += dS k.
//   warps 0-15   dS: four groups of 128 threads (a row each), a quarter of a block's keys each
//   warp 16      TMA: q and dout, then K and V by blocks
//   warps 17-19  products: X (and zeros for the keys that no query of the tile sees), Y, dq
template <int D>
struct QueryCfg {
  static constexpr int kThreads = 20 * 32;
  static constexpr int kTileBytes = kTile * D * 2;
  // V is through with when Y is, K when dq is: a ring each. (With one slot of both each, two of them for
  // D = 128, the loads were what a step waited for: 650 us for 8191 causal tokens of 32 heads.)
  static constexpr int kSlotsK = D == 64 ? 6 : 3, kSlotsV = D == 64 ? 5 : 2;
  static constexpr int kOffDo = kTileBytes;
  static constexpr int kOffK = 2 * kTileBytes;
  static constexpr int kOffV = kOffK + kSlotsK * kTileBytes;
  static constexpr int kOffBar = kOffV + kSlotsV * kTileBytes;
  static constexpr int kQ = 0, kKFull = 1, kKFree = kKFull + kSlotsK, kVFull = kKFree + kSlotsK,
                       kVFree = kVFull + kSlotsV, kXFull = kVFree + kSlotsV, kYFull = kXFull + 1,
                       kXRead = kYFull + 1, kYRead = kXRead + 1, kDsFull = kYRead + 1,
                       kDsDone = kDsFull + 1, kDone = kDsDone + 1, kBars = kDone + 3;
  static constexpr int kOffAll = kOffBar + (kBars * 8 + 32 + 127) / 128 * 128;  // fp16: [4][128]
  static constexpr int kSmem = kOffAll + 4 * kTile;
  static constexpr uint32_t kColX = 0, kColY = 128, kColDs = 256, kColDq = 384;
  static_assert(kSmem <= 227 * 1024, "shared memory");
};

// The largest exponent of max |v_i| among the keys that a thread's row sees (fp16), by warps 0-15: the four warps of
// a row share out 32 keys each of its first and of its last block, and the blocks between, which most rows of a
// warp have in common.
struct SeenKeys {
  int first, last;  // blocks
  int2 span;
  uint4 exps[4];              // of a quarter of the first block, of the last
  uint32_t all, before, behind;  // of the blocks that the warp's rows have in common, of those before and behind them

  // (Nothing waits for these loads here but the ends of the span. One for each place in line is enough
  // for most rows.)
  __device__ __forceinline__ void load(const SpanBwd& p, int group, const int* ends) {
    const int q = threadIdx.x >> 7, lane = threadIdx.x & 31;
    span = make_int2(__ldcg(ends), __ldcg(ends + kTile));
    const bool sees = span.x < span.y;
    first = sees ? span.x / kTile : 0;
    last = sees ? (span.y - 1) / kTile : 0;
    const int64_t block0 = static_cast<int64_t>(group) * p.y.key_blocks;
    const uint4* from = reinterpret_cast<const uint4*>(p.v_exp + block0 * kTile) + 2 * q;
    exps[0] = __ldcg(from + first * 8);
    exps[1] = __ldcg(from + first * 8 + 1);
    exps[2] = __ldcg(from + last * 8);
    exps[3] = __ldcg(from + last * 8 + 1);
    int lo = __reduce_max_sync(0xffffffffu, sees ? first + 1 : 0);
    int hi = __reduce_min_sync(0xffffffffu, sees ? last : 0x7fffffff);
    if (lo >= hi || hi == 0x7fffffff) lo = hi = 0;
    auto largest = [&](int b, int end, int step) {
      uint32_t x = b < end ? __ldcg(p.v_most + block0 + b) : 0u;
#pragma unroll 1
      for (b += step; b < end; b += step) x = max(x, static_cast<uint32_t>(__ldcg(p.v_most + block0 + b)));
      return x;
    };
    all = largest(lo + 32 * q + lane, hi, 128);
    before = largest(first + 1 + q, min(lo, last), 4);
    behind = largest(max(hi, first + 1) + q, last, 4);
  }
  __device__ __forceinline__ uint32_t found() const {
    const int q = threadIdx.x >> 7;
    const uint32_t most = max(__reduce_max_sync(0xffffffffu, all), max(before, behind));
    uint32_t four = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t seen = seen_word(span, (i < 2 ? first : last) * kTile + 32 * q) >> (i & 1) * 16;
      const uint32_t w[4] = {exps[i].x, exps[i].y, exps[i].z, exps[i].w};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t bits = seen >> 4 * c & 15u;
        four = __vmaxu4(four, w[c] & (bits * 0x00204081u & 0x01010101u) * 255u);  // a byte for every bit
      }
    }
    four = __vmaxu4(four, four >> 16);
    return max(most, __vmaxu4(four, four >> 8) & 255u);
  }
};

template <bool F16, int D>
__device__ __forceinline__ void query_block(const CUtensorMap& tmQ, const CUtensorMap& tmDo,
                                            const CUtensorMap& tmK, const CUtensorMap& tmV,
                                            const CUtensorMap& tmDq, const SpanBwd& p, int unit) {
  using C = QueryCfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = smem_u32(smem);
  const bool aligned = (base & 1023u) == 0;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kOffBar);
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * static_cast<uint32_t>(i); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);

  const int part = unit % p.q_parts;
  const int tile = p.y.row_tiles - 1 - unit / p.q_parts % p.y.row_tiles;
  const int group = unit / (p.q_parts * p.y.row_tiles);
  const int token0 = tile * p.y.tile_tokens;

  // rows past tile_rows are never loaded
  if (p.y.tile_rows < kTile) {
    for (int i = threadIdx.x; i < 2 * C::kTileBytes / 16; i += C::kThreads)
      reinterpret_cast<uint4*>(smem)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    __syncthreads();  // before q and dout are loaded
  }
  if (threadIdx.x == 16 * 32) {
    if (!aligned) atomicOr(p.err, ERR_SMEM_ALIGN);
    prefetch_tmap(&tmQ);
    prefetch_tmap(&tmDo);
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
    mbar_init(bar(C::kQ), 1);
    for (int i = 0; i < C::kSlotsK; ++i) {
      mbar_init(bar(C::kKFull + i), 1);
      mbar_init(bar(C::kKFree + i), 1);
    }
    for (int i = 0; i < C::kSlotsV; ++i) {
      mbar_init(bar(C::kVFull + i), 1);
      mbar_init(bar(C::kVFree + i), 1);
    }
    mbar_init(bar(C::kXFull), 1);
    mbar_init(bar(C::kYFull), 1);
    mbar_init(bar(C::kXRead), 16);
    mbar_init(bar(C::kYRead), 16);
    mbar_init(bar(C::kDsFull), 16);
    for (int i = 0; i < 3; ++i) mbar_init(bar(C::kDone + i), 1);
    mbar_init(bar(C::kDsDone), 1);
    fence_barrier_init();
  }
  grid_dep_wait();
  grid_dep_launch();
  if (warp == 0) {
    tmem_alloc(smem_u32(tmem_slot), 512);
    tmem_relinquish();
  }
  const int4 m = __ldcg(p.limits + tile);
  const int b0 = m.y > 0 ? m.x / kTile : 0;
  const int n = aligned && m.y > 0 ? (m.y + kTile - 1) / kTile - b0 : 0;
  const int block0 = b0 + static_cast<int>(static_cast<int64_t>(n) * part / p.q_parts);
  const int count = b0 + static_cast<int>(static_cast<int64_t>(n) * (part + 1) / p.q_parts) - block0;
  // K or V of block n; waits for its slot after the first ones
  auto load = [&](int n, const CUtensorMap* map, uint32_t to, int slots, int full, int free) {
    const int slot = n % slots;
    if (n >= slots && !wait(bar(free + slot), (n / slots - 1) & 1, p.err, ERR_WAIT_MMA)) return false;
    mbar_expect_tx(bar(full + slot), C::kTileBytes);
    for (int d = 0; d < D / 64; ++d)
      tma_load_4d(to + slot * C::kTileBytes + d * kSub, map, bar(full + slot), 64 * d, group,
                  (block0 + n) * kTile, 0);
    return true;
  };
  SeenKeys keys;
  if (F16 && warp < 16)
    keys.load(p, group, reinterpret_cast<const int*>(p.stat) + 2 * kTile + threadIdx.x % kTile +
                            (static_cast<int64_t>(group) * p.y.row_tiles + tile) * kRecord);
  int loads_k = 0, loads_v = 0;  // warp 16: so far
  if (threadIdx.x == 16 * 32 && count > 0) {  // what there is room for, while the others get ready
    mbar_expect_tx(bar(C::kQ), 2 * p.y.tile_rows * D * 2);
    for (int d = 0; d < D / 64; ++d) {
      tma_load_4d(base + d * kSub, &tmQ, bar(C::kQ), 64 * d, group * p.y.per, token0, 0);
      tma_load_4d(base + C::kOffDo + d * kSub, &tmDo, bar(C::kQ), 64 * d, group * p.y.per, token0, 0);
    }
    for (; loads_v < min(count, C::kSlotsV); ++loads_k, ++loads_v) {
      load(loads_k, &tmK, base + C::kOffK, C::kSlotsK, C::kKFull, C::kKFree);
      load(loads_v, &tmV, base + C::kOffV, C::kSlotsV, C::kVFull, C::kVFree);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (count == 0) {
    // no row sees any key
  } else if (warp == 16) {
    if (lane == 0) {
      // K and V in turn, each when its slot is free
      int k = loads_k, v = loads_v;
      while (v < count && load(k, &tmK, base + C::kOffK, C::kSlotsK, C::kKFull, C::kKFree)) {
        ++k;
        if (!load(v, &tmV, base + C::kOffV, C::kSlotsV, C::kVFull, C::kVFree)) break;
        ++v;
      }
      // nothing may be in flight when the block exits
      wait(bar(C::kQ), 0, p.err, ERR_WAIT_TMA, true);
      for (int j = max(0, k - C::kSlotsK); j < k; ++j)
        wait(bar(C::kKFull + j % C::kSlotsK), (j / C::kSlotsK) & 1, p.err, ERR_WAIT_TMA, true);
      for (int j = max(0, v - C::kSlotsV); j < v; ++j)
        wait(bar(C::kVFull + j % C::kSlotsV), (j / C::kSlotsV) & 1, p.err, ERR_WAIT_TMA, true);
    }
  } else if (warp == 17 || warp == 18) {
    // ---- X = q k^T (17), Y = dout v^T (18)
    const bool y = warp == 18;
    constexpr uint32_t idesc = Mma<F16, D>::idesc(kTile, false);
    const uint64_t a0 = sdesc_k_sw128(base + (y ? C::kOffDo : 0));
    const uint32_t col = tmem + (y ? C::kColY : C::kColX);
    int2 span[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = lane + 32 * i;
      span[i] = t < p.y.tile_tokens && token0 + t < p.y.n_q ? span_of(p.spans, token0 + t, p.y.n_k)
                                                           : make_int2(0, 0);
    }
    bool ok = wait_warp(bar(C::kQ), 0, p.err, ERR_WAIT_TMA);
    for (int i = 0; i < count && ok; ++i) {
      const int slots = y ? C::kSlotsV : C::kSlotsK, st = i % slots, key0 = (block0 + i) * kTile;
      ok = wait_warp(bar((y ? C::kVFull : C::kKFull) + st), (i / slots) & 1, p.err, ERR_WAIT_TMA);
      const int off = (y ? C::kOffV : C::kOffK) + st * C::kTileBytes;
      if (!y) {
        // zeros for K of keys that no query of the tile sees: their dS is 0, but 0 times NaN is NaN
        bool whole = false;
#pragma unroll
        for (int s = 0; s < 4; ++s) whole |= span[s].x <= key0 && span[s].y >= key0 + kTile;
        if (!__any_sync(0xffffffffu, whole)) {
          bool some = false;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            uint32_t mine = 0;
#pragma unroll
            for (int s = 0; s < 4; ++s) mine |= seen_word(span[s], key0 + 32 * w);
            const uint32_t seen = __reduce_or_sync(0xffffffffu, mine);
            some |= seen != 0xffffffffu;
            if ((seen >> lane) & 1u) continue;
            uint4* row = reinterpret_cast<uint4*>(smem + off + (32 * w + lane) * 128);
#pragma unroll
            for (int d = 0; d < D / 64; ++d)
#pragma unroll
              for (int c = 0; c < 8; ++c) row[d * (kSub / 16) + c] = make_uint4(0, 0, 0, 0);
          }
          if (some) fence_proxy_async_smem();
          __syncwarp();
        }
      }
      if (i > 0)
        ok = ok && wait_warp(bar(y ? C::kYRead : C::kXRead), (i - 1) & 1, p.err, ERR_WAIT_EPI);
      if (!ok) break;
      tc_fence_after();
      const uint64_t k0 = sdesc_k_sw128(base + off);
#pragma unroll
      for (int d = 0; d < D / 64; ++d)
        mma4_bf16_ss_w(col, a0 + static_cast<uint64_t>(d * (kSub >> 4)),
                       k0 + static_cast<uint64_t>(d * (kSub >> 4)), idesc, d > 0);
      mma_commit_w(bar(y ? C::kYFull : C::kXFull));
      if (y) mma_commit_w(bar(C::kVFree + st));
    }
    products_done(bar(C::kDone + (y ? 1 : 0)), p.err);
  } else if (warp == 19) {
    // ---- dq += dS k
    constexpr uint32_t idesc = Mma<F16, D>::idesc(D, true);
    bool ok = true;
    for (int i = 0; i < count && ok; ++i) {
      const int st = i % C::kSlotsK;
      ok = wait_warp(bar(C::kKFull + st), (i / C::kSlotsK) & 1, p.err, ERR_WAIT_TMA) &&
           wait_warp(bar(C::kDsFull), i & 1, p.err, ERR_WAIT_EPI);
      if (!ok) break;
      tc_fence_after();
      const uint32_t k = base + C::kOffK + st * C::kTileBytes;
#pragma unroll
      for (int x = 0; x < 2; ++x)
        mma4_ts_mn_w(tmem + C::kColDq, tmem + C::kColDs + 32u * x, sdesc_mn_sw128(k + x * 64 * 128, kSub),
                     idesc, i > 0 || x > 0);
      mma_commit_w(bar(C::kDsDone));
      mma_commit_w(bar(C::kKFree + st));
    }
    products_done(bar(C::kDone + 2), p.err);
  }
  if (warp < 16) {
    // ---- dS of a quarter of each block's keys
    const int q = warp >> 2, row = (warp & 3) * 32 + lane;
    const int64_t at = static_cast<int64_t>(group) * p.y.row_tiles + tile;
    const float* stat = p.stat + at * kRecord + row;
    const float neg_lse = __ldcg(stat), neg_delta = __ldcg(stat + kTile);
    const int2 span = make_int2(__ldcg(reinterpret_cast<const int*>(stat) + 2 * kTile),
                                __ldcg(reinterpret_cast<const int*>(stat) + 3 * kTile));
    const bool sees = span.x < span.y;
    float ds_down = 1.f;  // the row's dS are kept times this
    if (F16) {
      const float2 size = __ldcg(p.size_row + at * kTile + row);
      uint8_t* const v_exps = smem + C::kOffAll + row;  // by quarters
      v_exps[q * kTile] = static_cast<uint8_t>(keys.found());
      named_barrier(1, 512);
      ds_down = down_scale(size, max(max(v_exps[0], v_exps[kTile]), max(v_exps[2 * kTile], v_exps[3 * kTile])));
    }
    const int all_from = __reduce_max_sync(0xffffffffu, sees ? span.x : 0);
    const int all_to = __reduce_min_sync(0xffffffffu, sees ? span.y : 0x7fffffff);
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t x_col = tmem + lane_off + C::kColX + 32u * q;
    const uint32_t y_col = tmem + lane_off + C::kColY + 32u * q;
    const uint32_t ds_col = tmem + lane_off + C::kColDs + 16u * q;
    const uint64_t c2 = pack_f32x2(p.scale_log2, p.scale_log2), l2 = pack_f32x2(neg_lse, neg_lse),
                   d2 = pack_f32x2(neg_delta, neg_delta);
    const float dn = F16 ? ds_down / kPUp : 1.f;
    const uint64_t down2 = pack_f32x2(dn, dn);
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      const int key0 = (block0 + i) * kTile + 32 * q;
      const bool masked = key0 < all_from || key0 + 32 > all_to;
      wait_warp(bar(C::kXFull), i & 1, p.err, ERR_WAIT_MMA);
      tc_fence_after();
      uint32_t x[32], y[32];
      tmem_ld_32x32b_x32(x_col, x);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kXRead));
      wait_warp(bar(C::kYFull), i & 1, p.err, ERR_WAIT_MMA);
      tc_fence_after();
      tmem_ld_32x32b_x32(y_col, y);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kYRead));
#pragma unroll
      for (int c = 0; c < 32; c += 2) {
        const float2 a = halves_of(fma2(pair_of(x[c], x[c + 1]), c2, l2));
        x[c] = __float_as_uint(ex2_approx(a.x));
        x[c + 1] = __float_as_uint(ex2_approx(a.y));
      }
#pragma unroll
      for (int c = 0; c < 32; c += 2) {
        uint64_t a = pair_of(x[c], x[c + 1]);
        if (F16) a = mul2(a, down2);
        const float2 u = halves_of(mul2(a, add2(pair_of(y[c], y[c + 1]), d2)));
        y[c] = __float_as_uint(u.x);
        y[c + 1] = __float_as_uint(u.y);
      }
      if (masked) {
        __syncwarp();  // (as above)
        const uint32_t seen = span.y - span.x > 1 ? seen_word(span, key0) : 0u;
#pragma unroll
        for (int c = 0; c < 32; ++c)
          if (!(seen & (1u << c))) y[c] = 0;
      }
      uint32_t pk[16];
#pragma unroll
      for (int c = 0; c < 32; c += 2)
        pk[c / 2] = pack16<F16>(__uint_as_float(y[c]), __uint_as_float(y[c + 1]));
      if (i > 0) wait_warp(bar(C::kDsDone), (i - 1) & 1, p.err, ERR_WAIT_MMA);
      tc_fence_after();
      tmem_st_32x32b_x16(ds_col, pk);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::kDsFull));
    }
    if (count > 0) wait_warp(bar(C::kDsDone), (count - 1) & 1, p.err, ERR_WAIT_MMA);
    tc_fence_after();
    // dq goes through q's place in shared memory
    const int64_t slot = (static_cast<int64_t>(group) * p.y.row_tiles + tile) * p.q_parts + part;
    float4* part_q = p.q_parts > 1 ? reinterpret_cast<float4*>(p.part_q) + slot * (D / 4) * kTile : nullptr;
    const float f = p.scale / ds_down;
#pragma unroll 1
    for (int d = q * (D / 4); d < (q + 1) * (D / 4); d += 16) {
      if (count > 0)
        leave16<F16>(tmem + lane_off + C::kColDq + d, f, sees, smem, part_q, row, d);
      else
        leave16_none(smem, part_q, row, d);
    }
    if (p.q_parts == 1) {
      fence_proxy_async_smem();
      named_barrier(1, 512);
      if (threadIdx.x == 0 && aligned) {
        for (int d = 0; d < D / 64; ++d)
          tma_store_4d(&tmDq, base + d * kSub, 64 * d, group * p.y.per, token0, 0);
        bulk_commit();
        bulk_wait_all();
      }
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// The blocks of keys, which take longest, then those of queries: in one launch the second ones fill the end of
// the first.
template <bool F16, int D>
__global__ void __launch_bounds__(KeyCfg<D>::kThreads, 1)
    span_grad_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmDo,
                     const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const __grid_constant__ CUtensorMap tmDq, const __grid_constant__ CUtensorMap tmDk,
                     const __grid_constant__ CUtensorMap tmDv, const __grid_constant__ SpanBwd p) {
  static_assert(KeyCfg<D>::kThreads == QueryCfg<D>::kThreads, "one launch");
  const int keys = p.k_parts * p.y.key_blocks * p.y.groups;
  if (static_cast<int>(blockIdx.x) < keys)
    keys_block<F16, D>(tmQ, tmDo, tmK, tmV, tmDk, tmDv, p, blockIdx.x);
  else
    query_block<F16, D>(tmQ, tmDo, tmK, tmV, tmDq, p, static_cast<int>(blockIdx.x) - keys);
}

// ------------------------------------------------------------------------------ parts added up
// in their order: a block a tile, a thread per row (neighbours in a warp) and eight elements at a time
constexpr int kSumThreads = 4 * kTile;
template <bool F16, int D>
__global__ void __launch_bounds__(kSumThreads) span_sums_kernel(const __grid_constant__ SpanBwd p, int first) {
  grid_dep_wait();
  grid_dep_launch();
  const int row = threadIdx.x % kTile, which = first + blockIdx.y;  // dq, dk, dv
  const int tile = static_cast<int>(blockIdx.x) / p.y.groups, group = static_cast<int>(blockIdx.x) % p.y.groups;
  const float4* from;
  uint16_t* to;
  int parts;
  int64_t step = D / 4 * kTile;
  if (which == 0) {
    const int token = tile * p.y.tile_tokens + row / p.y.per, head = group * p.y.per + row % p.y.per;
    if (p.q_parts == 1 || tile >= p.y.row_tiles || row >= p.y.tile_rows || token >= p.y.n_q) return;
    parts = p.q_parts;
    from = reinterpret_cast<const float4*>(p.part_q) +
           (static_cast<int64_t>(group) * p.y.row_tiles + tile) * parts * step;
    to = static_cast<uint16_t*>(p.dq.p) + token * p.dq.token + head * p.dq.head;
  } else {
    const int key = tile * kTile + row;
    if (p.k_parts == 1 || tile >= p.y.key_blocks || key >= p.y.n_k) return;
    parts = p.k_parts;
    step *= 2;
    from = reinterpret_cast<const float4*>(p.part_k) +
           (static_cast<int64_t>(group) * p.y.key_blocks + tile) * parts * step + (which == 2 ? step / 2 : 0);
    const SpanRows& r = which == 2 ? p.dv : p.dk;
    to = static_cast<uint16_t*>(r.p) + key * r.token + group * r.head;
  }
#pragma unroll
  for (int d = threadIdx.x / kTile * 8; d < D; d += kSumThreads / kTile * 8) {
    const float4* at = from + d / 4 * kTile + row;
    float sum[8] = {};
#pragma unroll 4
    for (int c = 0; c < parts; ++c) {
      const float4 a = __ldcg(at + c * step), b = __ldcg(at + c * step + kTile);
      sum[0] += a.x, sum[1] += a.y, sum[2] += a.z, sum[3] += a.w;
      sum[4] += b.x, sum[5] += b.y, sum[6] += b.z, sum[7] += b.w;
    }
    *reinterpret_cast<uint4*>(to + d) =
        make_uint4(pack16<F16>(sum[0], sum[1]), pack16<F16>(sum[2], sum[3]),
                   pack16<F16>(sum[4], sum[5]), pack16<F16>(sum[6], sum[7]));
  }
}

// no keys, or no queries: what there is gets zeros
__global__ void span_zeros_kernel(SpanRows r, int tokens, int heads, int head_dim) {
  grid_dep_wait();
  const int64_t rows = static_cast<int64_t>(tokens) * heads;
  for (int64_t i = blockIdx.x; i < rows; i += gridDim.x)
    static_cast<uint16_t*>(r.p)[i / heads * r.token + i % heads * r.head + threadIdx.x] = 0;
  grid_dep_launch();
}

// Parts of a unit's walk over `steps` tiles: as many as give every SM a unit, but four tiles (4 us) each at
// least where every tile is walked (spans are not known here), since the sums of the parts take 3 us. (More parts of the keys' walks, four units an SM, even them out
// no better than the queries' units behind them do: 555 us instead of 519 for the 480p clip.)
int parts_for(int64_t units, int steps) {
  return static_cast<int>(
      std::max<int64_t>(1, std::min<int64_t>(steps / 4, (num_sms() + units - 1) / units)));
}

struct BwdPlan {
  int q_parts, k_parts;
  size_t stat, limits, size_row, size_token, size_tile, v_exp, v_most, part_q, part_k, total;  // byte offsets
};
BwdPlan bwd_plan(const SpanShape& y, int head_dim) {
  BwdPlan b{};
  b.q_parts = parts_for(static_cast<int64_t>(y.groups) * y.row_tiles, y.key_blocks);
  b.k_parts = parts_for(static_cast<int64_t>(y.groups) * y.key_blocks, y.row_tiles);
  const size_t tiles = static_cast<size_t>(y.groups) * y.row_tiles;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  b.stat = 0;
  b.limits = up(b.stat + tiles * kRecord * sizeof(float));
  // (for either type: the plan has none)
  b.size_row = b.limits + up(static_cast<size_t>(y.row_tiles) * sizeof(int4));
  b.size_token = b.size_row + up(tiles * kTile * sizeof(float2));
  b.size_tile = b.size_token + up(static_cast<size_t>(y.groups) * y.n_q * sizeof(float4));
  b.v_exp = b.size_tile + up(tiles * sizeof(float2));
  b.v_most = b.v_exp + up(static_cast<size_t>(y.groups) * y.key_blocks * kTile);
  b.part_q = b.v_most + up(static_cast<size_t>(y.groups) * y.key_blocks);
  b.part_k = b.part_q + (b.q_parts > 1 ? tiles * b.q_parts * kTile * head_dim * sizeof(float) : 0);
  b.total = b.part_k + (b.k_parts > 1 ? static_cast<size_t>(y.groups) * y.key_blocks * b.k_parts * 2 *
                                            kTile * head_dim * sizeof(float)
                                      : 0);
  return b;
}

template <bool F16, int D>
cudaError_t launch_bwd(const SpanBwd& p, const SpanRows& q, const SpanRows& k, const SpanRows& v,
                       cudaStream_t s) {
  CUtensorMap tmQ, tmDo, tmK, tmV, tmDq, tmDk, tmDv;
  if (!make_map(&tmQ, F16, q.p, D, p.y.heads, p.y.n_q, 1, q.head, q.token, 0, p.y.per, p.y.tile_tokens) ||
      !make_map(&tmDo, F16, p.dout.p, D, p.y.heads, p.y.n_q, 1, p.dout.head, p.dout.token, 0, p.y.per,
                p.y.tile_tokens) ||
      !make_map(&tmK, F16, k.p, D, p.y.groups, p.y.n_k, 1, k.head, k.token, 0, 1, kTile) ||
      !make_map(&tmV, F16, v.p, D, p.y.groups, p.y.n_k, 1, v.head, v.token, 0, 1, kTile) ||
      !make_map(&tmDq, F16, p.dq.p, D, p.y.heads, p.y.n_q, 1, p.dq.head, p.dq.token, 0, p.y.per,
                p.y.tile_tokens) ||
      !make_map(&tmDk, F16, p.dk.p, D, p.y.groups, p.y.n_k, 1, p.dk.head, p.dk.token, 0, 1, kTile) ||
      !make_map(&tmDv, F16, p.dv.p, D, p.y.groups, p.y.n_k, 1, p.dv.head, p.dv.token, 0, 1, kTile))
    return cudaErrorInvalidValue;
  constexpr int kSmem = std::max(KeyCfg<D>::kSmem, QueryCfg<D>::kSmem);
  static OncePerDevice once;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess)
    e = once.run(dev, [&] {
      return cudaFuncSetAttribute(span_grad_kernel<F16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                  kSmem);
    });
  if (e == cudaSuccess)
    e = launch_pdl(span_rows_kernel<F16, D>, dim3(p.y.row_tiles + (F16 ? p.y.key_blocks : 0), p.y.groups), dim3(256),
                   0, s, p);
  if (e == cudaSuccess)
    e = launch_pdl(span_grad_kernel<F16, D>,
                   dim3((p.y.key_blocks * p.k_parts + p.y.row_tiles * p.q_parts) * p.y.groups),
                   dim3(KeyCfg<D>::kThreads), kSmem, s, tmQ, tmDo, tmK, tmV, tmDq, tmDk, tmDv, p);
  if (e != cudaSuccess || (p.q_parts == 1 && p.k_parts == 1)) return e;
  const int64_t tiles = std::max(p.q_parts > 1 ? p.y.row_tiles : 0, p.k_parts > 1 ? p.y.key_blocks : 0);
  const int first = p.q_parts > 1 ? 0 : 1, end = p.k_parts > 1 ? 3 : 1;
  return launch_pdl(span_sums_kernel<F16, D>, dim3(static_cast<unsigned>(tiles * p.y.groups), end - first),
                    dim3(kSumThreads), 0, s, p, first);
}

}  // namespace

size_t span_bwd_workspace_bytes(int n_q, int n_k, int heads, int groups, int head_dim) {
  if (n_q == 0 || n_k == 0) return 0;
  return bwd_plan(span_shape(n_q, n_k, heads, groups), head_dim).total;
}

}  // namespace fd

extern "C" {

fd_status fd_op_span_attention_bwd(
    const fd_span_attention* a, const void* q, int64_t q_token_stride, int64_t q_head_stride,
    const void* k, int64_t k_token_stride, int64_t k_head_stride, const void* v,
    int64_t v_token_stride, int64_t v_head_stride, const int32_t* spans, const void* out,
    int64_t out_token_stride, int64_t out_head_stride, const float* lse, const void* dout,
    int64_t dout_token_stride, int64_t dout_head_stride, void* dq, int64_t dq_token_stride,
    int64_t dq_head_stride, void* dk, int64_t dk_token_stride, int64_t dk_head_stride, void* dv,
    int64_t dv_token_stride, int64_t dv_head_stride, void* workspace, int* err_dev, void* stream) {
  if (!fd::span_valid(a)) return FD_ERR_INVALID_ARG;
  if (a->n_q == 0 && a->n_k == 0) return FD_OK;
  const fd::SpanRows qr{const_cast<void*>(q), q_token_stride, q_head_stride},
      kr{const_cast<void*>(k), k_token_stride, k_head_stride},
      vr{const_cast<void*>(v), v_token_stride, v_head_stride};
  fd::SpanBwd p{};
  p.v = vr;
  p.out = {const_cast<void*>(out), out_token_stride, out_head_stride};
  p.dout = {const_cast<void*>(dout), dout_token_stride, dout_head_stride};
  p.dq = {dq, dq_token_stride, dq_head_stride};
  p.dk = {dk, dk_token_stride, dk_head_stride};
  p.dv = {dv, dv_token_stride, dv_head_stride};
  auto queries = [&](const fd::SpanRows& r) {
    return a->n_q == 0 || fd::span_rows_ok(r, a->n_q, a->heads, a->head_dim);
  };
  auto keys = [&](const fd::SpanRows& r) {
    return a->n_k == 0 || fd::span_rows_ok(r, a->n_k, a->groups, a->head_dim);
  };
  if (!queries(qr) || !queries(p.out) || !queries(p.dout) || !keys(kr) || !keys(vr) ||
      !fd::span_ptr(err_dev, 4))
    return FD_ERR_INVALID_ARG;
  if ((a->n_q > 0 && !fd::span_out_ok(p.dq, a->n_q, a->heads, a->head_dim)) ||
      (a->n_k > 0 && (!fd::span_out_ok(p.dk, a->n_k, a->groups, a->head_dim) ||
                      !fd::span_out_ok(p.dv, a->n_k, a->groups, a->head_dim))) ||
      fd::span_meets(p.dq, {q, k, v, spans, out, lse, dout, dk, dv, workspace}) ||
      fd::span_meets(p.dk, {q, k, v, spans, out, lse, dout, dv, workspace}) ||
      fd::span_meets(p.dv, {q, k, v, spans, out, lse, dout, workspace}))
    return FD_ERR_INVALID_ARG;
  if (a->n_q > 0 && a->n_k > 0 &&
      (!fd::span_ptr(spans, 8) || !fd::span_ptr(lse, 4) || !fd::span_ptr(workspace, 16)))
    return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (a->n_q == 0 || a->n_k == 0) {
    cudaError_t e = cudaSuccess;
    auto zeros = [&](const fd::SpanRows& r, int tokens, int heads) {
      if (tokens > 0 && e == cudaSuccess)
        e = fd::launch_pdl(fd::span_zeros_kernel, dim3(fd::num_sms()), dim3(a->head_dim), 0, s, r, tokens,
                           heads, a->head_dim);
    };
    zeros(p.dq, a->n_q, a->heads);
    zeros(p.dk, a->n_k, a->groups);
    zeros(p.dv, a->n_k, a->groups);
    return e == cudaSuccess ? FD_OK : FD_ERR_CUDA;
  }
  p.y = fd::span_shape(a->n_q, a->n_k, a->heads, a->groups);
  const fd::BwdPlan b = fd::bwd_plan(p.y, a->head_dim);
  p.q_parts = b.q_parts;
  p.k_parts = b.k_parts;
  p.spans = spans;
  p.scale = a->scale;
  p.scale_log2 = a->scale * fd::kLog2e;
  p.lse = lse;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.stat = reinterpret_cast<float*>(ws + b.stat);
  p.limits = reinterpret_cast<int4*>(ws + b.limits);
  p.size_row = reinterpret_cast<float2*>(ws + b.size_row);
  p.size_token = reinterpret_cast<float4*>(ws + b.size_token);
  p.size_tile = reinterpret_cast<float2*>(ws + b.size_tile);
  p.v_exp = ws + b.v_exp;
  p.v_most = ws + b.v_most;
  p.part_q = reinterpret_cast<float*>(ws + b.part_q);
  p.part_k = reinterpret_cast<float*>(ws + b.part_k);
  p.err = err_dev;
  const bool f16 = a->dtype == FD_DTYPE_F16;
  const cudaError_t e = a->head_dim == 64 ? (f16 ? fd::launch_bwd<true, 64>(p, qr, kr, vr, s)
                                                 : fd::launch_bwd<false, 64>(p, qr, kr, vr, s))
                                          : (f16 ? fd::launch_bwd<true, 128>(p, qr, kr, vr, s)
                                                 : fd::launch_bwd<false, 128>(p, qr, kr, vr, s));
  return e == cudaSuccess ? FD_OK : FD_ERR_CUDA;
}

}  // extern "C"
