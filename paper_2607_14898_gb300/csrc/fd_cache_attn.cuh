// Shared by the two forms of the attention over a bounded cache: fd_cache_attn.cu (few rows) and
// fd_cache_chunk.cu (many rows).
#pragma once
#include "fd_internal.h"
#include "fd_once.h"
#include "fd_ptx.cuh"
#include "flashdec_ops.h"

namespace fd {

constexpr int kSms = 152;  // of the GPU that the library is built for
constexpr float kLog2e = 1.44269504088896341f;

// one launch's shapes, pointers and workspace
struct CacheAttn {
  int groups, heads, per;     // per: heads of a group
  int used, n_q, rows;        // rows = n_q * per
  int capacity;
  const void *k, *v;
  int64_t stream_stride, group_stride, slot_stride;
  const int32_t* pos;
  const float* weight;
  float* weight_out;
  const void* q;
  int64_t q_stream, q_token, q_head;
  const int32_t* q_pos;
  void* out;
  int64_t out_stream, out_token, out_head;
  float scale_log2, decay;
  int lists;                  // streams * groups
  int* err;
  // few rows: logits [lists][rows][pitch] (log2 domain, -inf where not visible), and per
  // (list, row, split) the maximum and sum, and the unnormalised output
  int splits, chunk;          // slots of a split
  int64_t logit_pitch;
  float* logits;
  float2* part_ml;            // [lists][splits][rows]; many rows: [ctas][2][128]
  float* part_o;              // [lists][splits][rows][D]; many rows: [ctas][2][D / 4][128] float4
  // many rows: tiles of whole tokens, tile_rows = tile_tokens * per <= 128 rows each
  int tile_tokens, tile_rows, row_tiles;
  int key_tiles;              // of 128 slots
  int attend_blocks;          // of 256 slots
  int parts;                  // CTAs of the attention
  int row_splits;             // of the weights
  float* lse;                 // [lists][row_tiles * tile_rows], log2; +inf: sees nothing
  float* part_w;              // [row_splits][lists][used], where row_splits > 1
};

template <bool F16>
struct Elem;
template <>
struct Elem<false> {
  using type = __nv_bfloat16;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16x2(lo, hi); }
};
template <>
struct Elem<true> {
  using type = __half;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
};


// whether a call runs on the many-rows form: a rule on its sizes, and its plan and workspace.
// Up to 32 rows a list (two tiles of 16) the few-rows form is ahead over long caches and behind over
// short ones, above it is behind. Device times in us, few / many rows, at 32 and 48 rows: 32 lists
// of 6240 slots, D = 64: 34 / 47 and 50 / 47; 4 such lists: 18.7 / 20.6 and 23.4 / 20.8; 16 lists of
// 65537, D = 128: 168 / 213 and 245 / 213; 32 lists of 1000, D = 64: 19.8 / 16.5 and 26 / 16.6.
constexpr int kMaxRows = 32;  // of the few-rows form
bool chunk_form(int rows, int used);
struct ChunkPlan {
  int tile_tokens, tile_rows, row_tiles, key_tiles, attend_blocks, parts, row_splits;
  size_t ml, o, lse, w, total;  // byte offsets
};
ChunkPlan chunk_plan(const fd_cache* c, int used, int per, int n_q);
cudaError_t launch_chunk(const CacheAttn& p, const fd_cache* c, cudaStream_t s);
// one of the many-rows form's waits (0 to 3) on a barrier that nothing arrives at
cudaError_t launch_chunk_wait_check(int which, int* err, cudaStream_t s);

}  // namespace fd
