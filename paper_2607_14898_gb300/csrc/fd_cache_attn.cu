// Attention over a cache of bounded size that also returns what weight each entry was given
// (fd_op_cache_attention): out = softmax(scale q k^T) v over the visible slots, and for every
// slot the sum over queries and heads of its probability.
//
// The rows of one list (a KV group of a stream) are its queries of all heads of the group: row
// r = t * per + i is token t, head group * per + i. A slot's weight needs the final maximum and
// sum of every row, which are known only when all slots have been seen, so there are two
// steps: scores (running maximum and sum, O) and join (weights, and O over the split parts).
#include <algorithm>
#include <cmath>

#include "fd_cache_attn.cuh"

namespace fd {

bool valid_cache(const fd_cache* c);  // fd_cache_evict.cu

namespace {

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
               "r"(valid ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
template <bool F16>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                          uint32_t b1) {
  if constexpr (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, "
                 "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, "
                 "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// ---------------------------------------------------------------- few rows: split over slots
//
// Bound by reading K and V once. A CTA takes up to 16 rows of one list and a run of slots; each of
// its warps streams its own tiles of keys and values (4 KB each) through a private ring in
// shared memory, so that no warp waits for another in the loop, and keeps its own running
// maximum, sum and O in registers. Products on mma.sync m16n8k16: with 16 rows at most a tile
// is 16 x 32 x 64, far below what a tcgen05 tile (128 rows) would be filled with, and K and V arrive
// slower than either unit could take them. One query of 2 streams, 32 heads on 8 groups of 128, over
// 65537 slots (537 MB): 89 us, 6.0 TB/s; with the join 97. One of 8 streams, 16 heads on 4 groups of
// 64, over 6240 (51 MB): 15.7 us with the join, of which two dependent launches and the first
// loads' way take half.
namespace few {
constexpr int kWarps = 4;
constexpr int kRows = 16;
constexpr int kStages = 3;
constexpr int kTileBytes = 4096;  // of keys, and of values
template <int D>
constexpr int kKeys = kTileBytes / (2 * D);  // of a tile: 32 (D = 64), 16 (D = 128)
constexpr int kStageBytes = 2 * kTileBytes + 128;                  // and the slots' positions
constexpr int kSmem = kWarps * kStages * kStageBytes;
}  // namespace few

// byte offset of 16-byte unit c of row r in a tile of rows of D 16-bit elements; units are
// permuted within 128 bytes so that the 8 rows of an ldmatrix hit different banks
template <int D>
__device__ __forceinline__ uint32_t tile_unit(int r, int c) {
  return static_cast<uint32_t>(r * (2 * D) + ((c ^ (r & 7)) << 4));
}

template <bool F16, int D>
__global__ void __launch_bounds__(few::kWarps * 32)
    few_rows_kernel(const __grid_constant__ CacheAttn p) {
  using namespace few;
  using T = typename Elem<F16>::type;
  constexpr int KT = kKeys<D>;
  constexpr int kUnits = D / 8;  // 16-byte units of a row
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = blockIdx.x, lst = blockIdx.z, row0 = blockIdx.y * kRows;
  const int stream = lst / p.groups, group = lst - stream * p.groups;
  const int begin = split * p.chunk;
  const int end = min(begin + p.chunk, p.used);
  const T* kb = static_cast<const T*>(p.k) + stream * p.stream_stride + group * p.group_stride;
  const T* vb = static_cast<const T*>(p.v) + stream * p.stream_stride + group * p.group_stride;
  const int32_t* pb = p.pos + static_cast<int64_t>(lst) * p.capacity;
  uint8_t* ring = smem + warp * kStages * kStageBytes;
  const uint32_t ring_s = smem_u32(ring);
  const int tiles = (end - begin + KT - 1) / KT;
  const int mine = tiles > warp ? (tiles - warp + kWarps - 1) / kWarps : 0;

  grid_dep_wait();
  grid_dep_launch();  // the join's blocks may be there, waiting, when the last of these is done
  // tile i of this warp into stage i % kStages
  auto fetch = [&](int i) {
    if (i < mine) {
      const int s0 = begin + (warp + i * kWarps) * KT;
      const uint32_t st = ring_s + (i % kStages) * kStageBytes;
#pragma unroll
      for (int u = lane; u < KT * kUnits; u += 32) {
        const int r = u / kUnits, c = u % kUnits;
        const bool in = s0 + r < end;
        const int64_t at = static_cast<int64_t>(in ? s0 + r : begin) * p.slot_stride + c * 8;
        cp_async_16(st + tile_unit<D>(r, c), kb + at, in);
        cp_async_16(st + kTileBytes + tile_unit<D>(r, c), vb + at, in);
      }
      if (lane < KT) {
        if (s0 + lane < end) cp_async_4(st + 2 * kTileBytes + 4 * lane, pb + s0 + lane);
        else reinterpret_cast<int32_t*>(ring + (i % kStages) * kStageBytes + 2 * kTileBytes)[lane] = -1;
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch(i);

  // Q fragments of the 16 rows, and what each of this thread's two rows may see
  uint32_t qf[D / 16][4];
  int qp[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int r = row0 + (lane >> 2) + 8 * x;
    const bool in = r < p.rows;
    const int t = in ? r / p.per : 0, h = group * p.per + (in ? r - t * p.per : 0);
    const T* q = static_cast<const T*>(p.q) + stream * p.q_stream + t * p.q_token + h * p.q_head;
    qp[x] = in ? p.q_pos[static_cast<int64_t>(stream) * p.n_q + t] : -1;
#pragma unroll
    for (int j = 0; j < D / 16; ++j)
#pragma unroll
      for (int y = 0; y < 2; ++y)
        qf[j][x + 2 * y] =
            in ? *reinterpret_cast<const uint32_t*>(q + 16 * j + 8 * y + 2 * (lane & 3)) : 0u;
  }

  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  float o[D / 8][4];
#pragma unroll
  for (int j = 0; j < D / 8; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[j][e] = 0.f;

  for (int i = 0; i < mine; ++i) {
    cp_async_wait<kStages - 2>();
    __syncwarp();
    fetch(i + kStages - 1);
    const int s0 = begin + (warp + i * kWarps) * KT;
    const uint32_t st = ring_s + (i % kStages) * kStageBytes;
    const int32_t* tp =
        reinterpret_cast<const int32_t*>(ring + (i % kStages) * kStageBytes + 2 * kTileBytes);
    // an empty slot's value must not reach the product: its probability is 0, but 0 times NaN is NaN
    const bool hole = lane < KT && tp[lane & (KT - 1)] < 0;
    if (__any_sync(0xffffffffu, hole)) {
      if (hole) {
#pragma unroll
        for (int c = 0; c < kUnits; ++c)
          *reinterpret_cast<uint4*>(ring + (i % kStages) * kStageBytes + kTileBytes +
                                    tile_unit<D>(lane, c)) = make_uint4(0, 0, 0, 0);
      }
      __syncwarp();
    }
    float s[KT / 8][4];
#pragma unroll
    for (int n = 0; n < KT / 8; ++n) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        // keys 8n .. 8n+7, elements 32 j .. 32 j + 31: matrices of 8 elements each
        uint32_t b[4];
        ldmatrix_x4(st + tile_unit<D>(8 * n + (lane & 7), 4 * j + (lane >> 3)), b);
        mma_16816<F16>(s[n], qf[2 * j], b[0], b[1]);
        mma_16816<F16>(s[n], qf[2 * j + 1], b[2], b[3]);
      }
    }
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < KT / 8; ++n) {
      const int2 ps = *reinterpret_cast<const int2*>(tp + 8 * n + 2 * (lane & 3));
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        s[n][2 * x] = ps.x >= 0 && ps.x <= qp[x] ? s[n][2 * x] * p.scale_log2 : -INFINITY;
        s[n][2 * x + 1] = ps.y >= 0 && ps.y <= qp[x] ? s[n][2 * x + 1] * p.scale_log2 : -INFINITY;
        top[x] = fmax3(top[x], s[n][2 * x], s[n][2 * x + 1]);
        const int r = row0 + (lane >> 2) + 8 * x;
        const int slot = s0 + 8 * n + 2 * (lane & 3);
        if (p.logits != nullptr && r < p.rows && slot < p.logit_pitch)
          *reinterpret_cast<float2*>(p.logits +
                                     (static_cast<int64_t>(lst) * p.rows + r) * p.logit_pitch + slot) =
              make_float2(s[n][2 * x], s[n][2 * x + 1]);
      }
    }
    float base[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 1));
      top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], 2));
      const float now = fmaxf(m[x], top[x]);
      base[x] = now == -INFINITY ? 0.f : now;  // a row that has seen nothing: exp2(-inf - 0) = 0
      const float f = ex2_approx(m[x] - base[x]);
      m[x] = now;
      l[x] *= f;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        o[j][2 * x] *= f;
        o[j][2 * x + 1] *= f;
      }
    }
#pragma unroll
    for (int n = 0; n < KT / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[n][e] = ex2_approx(s[n][e] - base[e >> 1]);
        l[e >> 1] += s[n][e];
      }
    // P goes to the cache's type for its product with V, since the tensor cores take 16-bit operands (sums are
    // fp32): every p is off by 2^-9 (bf16) or 2^-12 (fp16) of itself at most, the output by that share of
    // sum p |v|, beside its own rounding of the same size. l and the weights come from P unrounded.
#pragma unroll
    for (int kk = 0; kk < KT / 16; ++kk) {
      const uint32_t a[4] = {Elem<F16>::pack(s[2 * kk][0], s[2 * kk][1]),
                             Elem<F16>::pack(s[2 * kk][2], s[2 * kk][3]),
                             Elem<F16>::pack(s[2 * kk + 1][0], s[2 * kk + 1][1]),
                             Elem<F16>::pack(s[2 * kk + 1][2], s[2 * kk + 1][3])};
#pragma unroll
      for (int j = 0; j < D / 16; ++j) {
        // values of keys 16 kk .. +15, elements 16 j .. +15, transposed on the way
        uint32_t b[4];
        ldmatrix_x4_trans(st + kTileBytes +
                              tile_unit<D>(16 * kk + (lane & 15), 2 * j + (lane >> 4)),
                          b);
        mma_16816<F16>(o[2 * j], a, b[0], b[1]);
        mma_16816<F16>(o[2 * j + 1], a, b[2], b[3]);
      }
    }
    __syncwarp();
  }
  cp_async_wait<0>();
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
    l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
  }

  // ---- the warps' results into one: maximum and sum, then O
  __syncthreads();  // every warp is done with its ring
  float2* ml = reinterpret_cast<float2*>(smem);                              // [warps][16]
  float* po = reinterpret_cast<float*>(smem + kWarps * kRows * sizeof(float2));  // [warps][16][D]
  static_assert(kWarps * kRows * (8 + 4 * D) <= kSmem, "partial results fit the rings");
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int r = (lane >> 2) + 8 * x;
    if ((lane & 3) == 0) ml[warp * kRows + r] = make_float2(m[x], l[x]);
#pragma unroll
    for (int j = 0; j < D / 8; ++j)
      *reinterpret_cast<float2*>(po + (warp * kRows + r) * D + 8 * j + 2 * (lane & 3)) =
          make_float2(o[j][2 * x], o[j][2 * x + 1]);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < kRows * D; e += kWarps * 32) {
    const int r = e / D, d = e % D;
    if (row0 + r >= p.rows) break;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[w * kRows + r].x);
    const float off = top == -INFINITY ? 0.f : top;
    float sum = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float2 x = ml[w * kRows + r];
      const float f = ex2_approx(x.x - off);
      sum = fmaf(f, x.y, sum);
      acc = fmaf(f, po[(w * kRows + r) * D + d], acc);
    }
    const int64_t at = (static_cast<int64_t>(lst) * p.splits + split) * p.rows + row0 + r;
    p.part_o[at * D + d] = acc;
    if (d == 0) p.part_ml[at] = make_float2(top, sum);
  }
}

// Joins the split parts: a block per row for the output (the first out_blocks blocks of a list),
// four slots a thread for the weights (the rest). Every block works out the rows' log2 sums of
// exponentials for itself: there are kMaxRows rows at most, and a block has 1024 slots to use
// them on (with 256 the sums took longer than the slots: 23 us for 2 x 65537 slots of 8 groups, now 11).
constexpr int kJoinThreads = 256;
constexpr int kJoinSlots = 4 * kJoinThreads;

template <bool F16, int D>
__global__ void __launch_bounds__(kJoinThreads)
    join_kernel(const __grid_constant__ CacheAttn p, int out_blocks) {
  using T = typename Elem<F16>::type;
  const int lst = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int stream = lst / p.groups, group = lst - stream * p.groups;
  grid_dep_wait();
  grid_dep_launch();
  const float2* ml = p.part_ml + static_cast<int64_t>(lst) * p.splits * p.rows;
  // log2 of the row's sum of exponentials (+inf for a row that sees nothing: its weights are 0)
  auto row_lse = [&](int r) {
    float top = -INFINITY;
    for (int s = lane; s < p.splits; s += 32) top = fmaxf(top, ml[static_cast<int64_t>(s) * p.rows + r].x);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if (top == -INFINITY) top = 0.f;
    float sum = 0.f;
    for (int s = lane; s < p.splits; s += 32) {
      const float2 x = ml[static_cast<int64_t>(s) * p.rows + r];
      sum = fmaf(ex2_approx(x.x - top), x.y, sum);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    return sum == 0.f ? INFINITY : top + log2f(sum);
  };
  if (static_cast<int>(blockIdx.x) < out_blocks) {
    // a block per row: each warp adds up its share of the splits, then the block the warps' sums
    constexpr int kWarps = kJoinThreads / 32;
    __shared__ float part[kWarps][D];
    const int r = blockIdx.x;
    const float lse = row_lse(r);
    float acc[D / 32] = {};
#pragma unroll 4
    for (int s = warp; s < p.splits; s += kWarps) {
      const int64_t at = (static_cast<int64_t>(lst) * p.splits + s) * p.rows + r;
      const float f = ex2_approx(p.part_ml[at].x - lse);
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        const float2 x = *reinterpret_cast<const float2*>(p.part_o + at * D + 64 * j + 2 * lane);
        acc[2 * j] = fmaf(f, x.x, acc[2 * j]);
        acc[2 * j + 1] = fmaf(f, x.y, acc[2 * j + 1]);
      }
    }
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
      *reinterpret_cast<float2*>(&part[warp][64 * j + 2 * lane]) =
          make_float2(acc[2 * j], acc[2 * j + 1]);
    __syncthreads();
    if (threadIdx.x < D / 2) {
      const int d = 2 * threadIdx.x;
      float a = 0.f, b = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        a += part[w][d];
        b += part[w][d + 1];
      }
      const int t = r / p.per, h = group * p.per + r - t * p.per;
      T* out = static_cast<T*>(p.out) + stream * p.out_stream + t * p.out_token + h * p.out_head;
      *reinterpret_cast<uint32_t*>(out + d) = Elem<F16>::pack(a, b);
    }
  } else {
    const int slot = (blockIdx.x - out_blocks) * kJoinSlots + 4 * threadIdx.x;
    const int64_t at = static_cast<int64_t>(lst) * p.capacity + slot;
    __shared__ float lse[kMaxRows];
    float old[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) old[i] = slot + i < p.used ? p.weight[at + i] : 0.f;
    for (int r = warp; r < p.rows; r += kJoinThreads / 32) {
      const float x = row_lse(r);
      if (lane == 0) lse[r] = x;
    }
    __syncthreads();
    if (slot < p.used) {
      const float* row = p.logits + static_cast<int64_t>(lst) * p.rows * p.logit_pitch + slot;
      float w[4] = {};
#pragma unroll 4
      for (int r = 0; r < p.rows; ++r) {
        const float4 x = *reinterpret_cast<const float4*>(row + r * p.logit_pitch);
        const float l = lse[r];
        w[0] += ex2_approx(x.x - l);
        w[1] += ex2_approx(x.y - l);
        w[2] += ex2_approx(x.z - l);
        w[3] += ex2_approx(x.w - l);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (slot + i < p.used) p.weight_out[at + i] = fmaf(p.decay, old[i], w[i]);
    }
  }
}

// slots -> (splits, chunk): two CTAs for every SM over all lists and row tiles (16 lists of 65537
// slots, D = 128: one CTA 120 us, two 97, three 103; 32 lists of 6240, D = 64: 17.5, 15.7, 19.2), at
// least a tile for each warp of a CTA (4 lists of 1000 slots: 128 slots 5.6 us, 256 6.3, 64 5.5), runs of
// 32 slots so that the last split is not left with a small rest
void plan_few(int lists, int row_tiles, int used, int* splits, int* chunk) {
  const int64_t want = 2 * kSms / std::max<int64_t>(1, static_cast<int64_t>(lists) * row_tiles);
  int n = static_cast<int>(std::max<int64_t>(1, want));
  int c = std::max((used + n - 1) / n, 128);
  c = (c + 31) / 32 * 32;
  *chunk = c;
  *splits = (used + c - 1) / c;
}

struct Layout {
  int splits, chunk;
  int64_t logit_pitch;
  size_t logits, ml, o, total;  // byte offsets
};
Layout layout_of(const fd_cache* c, int used, int heads, int n_q) {
  Layout y{};
  const int64_t lists = static_cast<int64_t>(c->streams) * c->groups;
  const int64_t rows = static_cast<int64_t>(n_q) * (heads / c->groups);
  plan_few(static_cast<int>(lists), static_cast<int>((rows + few::kRows - 1) / few::kRows), used,
           &y.splits, &y.chunk);
  y.logit_pitch = (used + 3) / 4 * 4;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t at = 0;
  y.logits = at;
  at += up(static_cast<size_t>(lists * rows * y.logit_pitch) * 4);
  y.ml = at;
  at += up(static_cast<size_t>(lists * y.splits * rows) * 8);
  y.o = at;
  at += up(static_cast<size_t>(lists * y.splits * rows) * c->head_dim * 4);
  y.total = at;
  return y;
}

template <bool F16, int D>
cudaError_t launch_few(const CacheAttn& p, int lists, cudaStream_t s) {
  int device = -1;
  if (const cudaError_t e = cudaGetDevice(&device); e != cudaSuccess) return e;
  static OncePerDevice smem;
  const cudaError_t attr = smem.run(device, [] {
    return cudaFuncSetAttribute(few_rows_kernel<F16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                few::kSmem);
  });
  if (attr != cudaSuccess) return attr;
  if (p.rows > 0) {
    const dim3 grid(p.splits, (p.rows + few::kRows - 1) / few::kRows, lists);
    const cudaError_t e =
        launch_pdl(few_rows_kernel<F16, D>, grid, dim3(few::kWarps * 32), few::kSmem, s, p);
    if (e != cudaSuccess) return e;
  }
  const int out_blocks = p.rows;
  const int slot_blocks = p.weight_out ? (p.used + kJoinSlots - 1) / kJoinSlots : 0;
  return launch_pdl(join_kernel<F16, D>, dim3(out_blocks + slot_blocks, lists), dim3(kJoinThreads),
                    0, s, p, out_blocks);
}

bool valid_shape(const fd_cache* c, int used, int heads, int n_q) {
  if (!valid_cache(c) || used < 0 || used > c->capacity || n_q < 0 || n_q > (1 << 20)) return false;
  if (heads < c->groups || heads % c->groups || heads / c->groups > 128) return false;
  const int64_t lists = static_cast<int64_t>(c->streams) * c->groups;
  return lists <= 65535 && static_cast<int64_t>(n_q) * (heads / c->groups) <= 16ll * 65535;
}

bool ok_ptr(const void* x, uintptr_t a) {
  return x != nullptr && reinterpret_cast<uintptr_t>(x) % a == 0;
}

// rows that see nothing, where there is no slot at all
template <typename T>
__global__ void zero_rows_kernel(const __grid_constant__ CacheAttn p, int streams, int head_dim) {
  grid_dep_wait();
  const int64_t rows = static_cast<int64_t>(streams) * p.n_q * p.heads;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const int h = static_cast<int>(r % p.heads);
    const int64_t t = r / p.heads;
    T* o = static_cast<T*>(p.out) + t / p.n_q * p.out_stream + t % p.n_q * p.out_token +
           h * p.out_head;
    for (int d = threadIdx.x; d < head_dim; d += blockDim.x) o[d] = T(0.f);
  }
  grid_dep_launch();
}

template <bool F16, int D>
cudaError_t launch(const CacheAttn& p, const fd_cache* c, cudaStream_t s) {
  const int lists = c->streams * c->groups;
  if (p.used == 0)
    return launch_pdl(zero_rows_kernel<typename Elem<F16>::type>, dim3(kSms), dim3(D), 0, s, p,
                      c->streams, D);
  return launch_few<F16, D>(p, lists, s);
}

}  // namespace
}  // namespace fd

extern "C" {

size_t fd_cache_attention_workspace_bytes(const fd_cache* cache, int used, int heads, int n_q) {
  if (!fd::valid_shape(cache, used, heads, n_q)) return 0;
  if (cache->streams == 0 || used == 0 || n_q == 0) return 0;
  const int per = heads / cache->groups;
  return fd::chunk_form(n_q * per, used) ? fd::chunk_plan(cache, used, per, n_q).total
                                         : fd::layout_of(cache, used, heads, n_q).total;
}

fd_status fd_op_cache_attention(const fd_cache* cache, int used, int heads, int n_q,
                                const void* q, int64_t q_stream_stride, int64_t q_token_stride,
                                int64_t q_head_stride, const int32_t* q_pos, float scale,
                                float decay, void* out, int64_t out_stream_stride,
                                int64_t out_token_stride, int64_t out_head_stride,
                                float* weight_out, void* workspace, int* err_dev, void* stream) {
  if (!fd::valid_shape(cache, used, heads, n_q) || !std::isfinite(scale) || !(scale > 0.f) ||
      !std::isfinite(decay))
    return FD_ERR_INVALID_ARG;
  if (cache->streams == 0 || (n_q == 0 && (used == 0 || weight_out == nullptr))) return FD_OK;
  if (weight_out != nullptr && !fd::ok_ptr(weight_out, 4)) return FD_ERR_INVALID_ARG;
  if (n_q > 0) {
    if (!fd::ok_ptr(q, 16) || !fd::ok_ptr(out, 16) || !fd::ok_ptr(q_pos, 4) ||
        !fd::ok_ptr(err_dev, 4) || (used > 0 && !fd::ok_ptr(workspace, 16)))
      return FD_ERR_INVALID_ARG;
    // (rows that share elements would be written by several threads in out, and have no use in q)
    auto steps = [&](int64_t entries, int64_t stride) {
      return stride % 8 == 0 && (entries == 1 || stride >= cache->head_dim);
    };
    if (!steps(cache->streams, q_stream_stride) || !steps(n_q, q_token_stride) ||
        !steps(heads, q_head_stride) || !steps(cache->streams, out_stream_stride) ||
        !steps(n_q, out_token_stride) || !steps(heads, out_head_stride))
      return FD_ERR_INVALID_ARG;
  }
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  fd::CacheAttn p{};
  p.groups = cache->groups;
  p.heads = heads;
  p.per = heads / cache->groups;
  p.used = used;
  p.n_q = n_q;
  p.rows = n_q * p.per;
  p.capacity = cache->capacity;
  p.k = cache->k;
  p.v = cache->v;
  p.stream_stride = cache->stream_stride;
  p.group_stride = cache->group_stride;
  p.slot_stride = cache->slot_stride;
  p.pos = cache->pos;
  p.weight = cache->weight;
  p.weight_out = weight_out;
  p.q = q;
  p.q_stream = q_stream_stride;
  p.q_token = q_token_stride;
  p.q_head = q_head_stride;
  p.q_pos = q_pos;
  p.out = out;
  p.out_stream = out_stream_stride;
  p.out_token = out_token_stride;
  p.out_head = out_head_stride;
  p.scale_log2 = scale * fd::kLog2e;
  p.decay = decay;
  p.lists = cache->streams * cache->groups;
  p.err = err_dev;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  if (used > 0 && fd::chunk_form(p.rows, used)) {
    const fd::ChunkPlan y = fd::chunk_plan(cache, used, p.per, n_q);
    p.tile_tokens = y.tile_tokens;
    p.tile_rows = y.tile_rows;
    p.row_tiles = y.row_tiles;
    p.key_tiles = y.key_tiles;
    p.attend_blocks = y.attend_blocks;
    p.parts = y.parts;
    p.row_splits = y.row_splits;
    p.part_ml = reinterpret_cast<float2*>(ws + y.ml);
    p.part_o = reinterpret_cast<float*>(ws + y.o);
    p.lse = reinterpret_cast<float*>(ws + y.lse);
    p.part_w = reinterpret_cast<float*>(ws + y.w);
    return fd::launch_chunk(p, cache, static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? FD_OK
               : FD_ERR_CUDA;
  }
  if (used > 0 && n_q > 0) {
    const fd::Layout y = fd::layout_of(cache, used, heads, n_q);
    p.splits = y.splits;
    p.chunk = y.chunk;
    p.logit_pitch = y.logit_pitch;
    p.logits = weight_out ? reinterpret_cast<float*>(ws + y.logits) : nullptr;
    p.part_ml = reinterpret_cast<float2*>(ws + y.ml);
    p.part_o = reinterpret_cast<float*>(ws + y.o);
  }
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool f16 = cache->dtype == FD_DTYPE_F16;
  const cudaError_t e =
      cache->head_dim == 64
          ? (f16 ? fd::launch<true, 64>(p, cache, s) : fd::launch<false, 64>(p, cache, s))
          : (f16 ? fd::launch<true, 128>(p, cache, s) : fd::launch<false, 128>(p, cache, s));
  return e == cudaSuccess ? FD_OK : FD_ERR_CUDA;
}

fd_status fd_debug_cache_wait_timeout(int which, int* err_dev, void* stream) {
  if (which < 0 || which > 3 || !fd::ok_ptr(err_dev, 4)) return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  return fd::launch_chunk_wait_check(which, err_dev, static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? FD_OK
             : FD_ERR_CUDA;
}

}  // extern "C"
