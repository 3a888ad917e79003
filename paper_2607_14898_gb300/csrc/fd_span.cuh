// Attention in which every query sees a span of keys, and its gradient: what their kernels share
// (fd_span_attn.cu: forward, fd_span_bwd.cu: gradient).
//
// A row tile is tile_tokens whole tokens with the `per` heads of one KV group: row r of tile i is
// token i tile_tokens + r / per, head r % per, loaded as one TMA box {64 elements, per heads,
// tile_tokens tokens}; rows past tile_rows in shared memory stay zero. A key block is 128 keys.
#pragma once
#include <cuda_runtime.h>

#include <cmath>
#include <initializer_list>

#include "fd_once.h"
#include "fd_tile.cuh"
#include "flashdec_ops.h"

namespace fd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

constexpr int kMaxSpanTokens = 1 << 24;
constexpr int64_t kMaxSpanStride = 1ll << 38;  // elements (a tensor map's strides are below 2^40 bytes)
constexpr int64_t kMaxSpanRows = 1ll << 36;  // (a tile has 65 rows at least: fewer than 2^30 units)

struct SpanShape {
  int n_q, n_k, heads, groups, per;
  int tile_tokens, tile_rows, row_tiles, key_blocks;
};
struct SpanRows {  // element (token, head, i) at p[token token + head head + i]
  void* p;
  int64_t token, head;
};

inline SpanShape span_shape(int n_q, int n_k, int heads, int groups) {
  SpanShape y{n_q, n_k, heads, groups, heads / groups, 0, 0, 0, 0};
  y.tile_tokens = kTile / y.per;
  y.tile_rows = y.tile_tokens * y.per;
  y.row_tiles = (n_q + y.tile_tokens - 1) / y.tile_tokens;
  y.key_blocks = (n_k + kTile - 1) / kTile;
  return y;
}

// a token's span within [0, n_k); an empty one is (0, 0)
__device__ __forceinline__ int2 span_of(const int32_t* spans, int token, int n_k) {
  int2 s = __ldg(reinterpret_cast<const int2*>(spans) + token);
  s.x = max(s.x, 0);
  s.y = min(s.y, n_k);
  return s.x < s.y ? s : make_int2(0, 0);
}

// bits e of a word whose key first + e is within [lo, hi)
__device__ __forceinline__ uint32_t below(int n) {
  return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u;
}
__device__ __forceinline__ uint32_t seen_word(int2 span, int first) {
  return below(span.y - first) & ~below(span.x - first);
}

// ---- arguments of the calls
inline bool span_ptr(const void* p, uintptr_t align) {
  return p != nullptr && reinterpret_cast<uintptr_t>(p) % align == 0;
}
inline bool span_valid(const fd_span_attention* a) {
  return a != nullptr && a->n_q >= 0 && a->n_k >= 0 && a->groups >= 1 && a->heads >= a->groups &&
         a->heads % a->groups == 0 && a->heads / a->groups <= kTile && a->heads <= 65535 &&
         (a->head_dim == 64 || a->head_dim == 128) &&
         (a->dtype == FD_DTYPE_BF16 || a->dtype == FD_DTYPE_F16) && std::isfinite(a->scale * kLog2e) &&
         a->scale > 0.f && a->n_q <= kMaxSpanTokens && a->n_k <= kMaxSpanTokens &&
         static_cast<int64_t>(a->n_q) * a->heads <= kMaxSpanRows &&
         static_cast<int64_t>(a->n_k) * a->groups <= kMaxSpanRows;
}
inline bool span_rows_ok(const SpanRows& r, int tokens, int heads, int head_dim) {
  return span_ptr(r.p, 16) && r.token % 8 == 0 && r.head % 8 == 0 && r.token < kMaxSpanStride &&
         r.head < kMaxSpanStride &&
         (tokens == 1 || r.token >= head_dim) && (heads == 1 || r.head >= head_dim);
}
// rows that are written: no two share elements (a token's heads lie between tokens, or the other way round)
inline bool span_out_ok(const SpanRows& r, int tokens, int heads, int head_dim) {
  return span_rows_ok(r, tokens, heads, head_dim) &&
         (tokens == 1 || heads == 1 || r.token >= (heads - 1) * r.head + head_dim ||
          r.head >= (tokens - 1) * r.token + head_dim);
}
// whether what is written begins where one of the others does (other overlaps are the caller's to avoid)
inline bool span_meets(const SpanRows& r, std::initializer_list<const void*> others) {
  for (const void* p : others)
    if (r.p != nullptr && r.p == p) return true;
  return false;
}

}  // namespace

size_t span_fwd_workspace_bytes(int n_q, int n_k, int heads, int groups, int head_dim);
size_t span_bwd_workspace_bytes(int n_q, int n_k, int heads, int groups, int head_dim);

}  // namespace fd
