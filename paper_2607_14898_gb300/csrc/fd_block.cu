// The join between two residual blocks and its gradient (fd_op_block_join, _bwd): the norm after a
// block, its gate and residual scale, the residual sum, and the norm before the next block.
//
//   n = b r_post,  r_post = (mean(b^2) + eps)^(-1/2)        (n = b without the norm after)
//   y = h + s gate n post
//   u = y r_pre pre,  r_pre = (mean(y^2) + eps)^(-1/2)
// Gradient, with m = y r_pre, g = du pre, y again from h and b (kept as they were or in 8 bits):
//   d = dy + r_pre (g - m mean(g m));  dh = d;  w = s d;  dgate = sum w n post
//   dpost = sum w gate n;  dpre = sum du m;  e = w gate post;  db = r_post (e - n mean(e n))
// (sums over the tokens; of a gate's tokens for dgate). All in fp32.
//
// Both are bound by memory: every row is read and written once, its sums taken while it is in
// registers.
#include <algorithm>
#include <cmath>

#include "fd_rows.cuh"
#include "flashdec_ops.h"

namespace fd {
namespace {

struct Join {
  int rows, width;
  const float *post, *pre, *gate;  // gate [ceil(rows / gate_rows)][width]
  int gate_rows;
  float scale, eps;
  const void *h, *b;
  int64_t h_stride, b_stride;
  void *y, *u;
  int64_t y_stride, u_stride;
  float *r_post, *r_pre;
  int8_t *h_codes, *b_codes;
  uint8_t *h_exps, *b_exps;
};

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int i = 16; i; i >>= 1) x += __shfl_xor_sync(0xffffffffu, x, i);
  return x;
}

template <int NV>
__device__ __forceinline__ void keep8(const float (&x)[NV][8], int row, int width, int unit0,
                                      int step, int8_t* codes, uint8_t* exps) {
  const int blocks = (width + kKeptBlock - 1) / kKeptBlock;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const uint32_t byte = kept_exponent(block_top(x[v]));
    const int unit = unit0 + v * step;
    if (unit >= width / 8) continue;
    *reinterpret_cast<uint2*>(codes + static_cast<int64_t>(row) * width + unit * 8) =
        kept_codes(x[v], byte);
    if (unit % 4 == 0) exps[static_cast<int64_t>(row) * blocks + unit / 4] = static_cast<uint8_t>(byte);
  }
}

// ------------------------------------------------------------------------------ forward
// NW warps a row, NV groups of eight elements a thread; with NW = 1 a block has four rows.
template <typename B, typename H, int NW, int NV>
__global__ void __launch_bounds__(NW == 1 ? 128 : NW * 32)
    join_kernel(const __grid_constant__ Join p) {
  __shared__ float part[2][NW == 1 ? 1 : NW];
  grid_dep_wait();
  grid_dep_launch();
  const int warp = threadIdx.x >> 5;
  const int row = NW == 1 ? blockIdx.x * 4 + warp : blockIdx.x;
  const int unit0 = NW == 1 ? threadIdx.x & 31 : threadIdx.x;
  constexpr int kStep = NW * 32;
  if (row >= p.rows) return;  // (whole warps, and no barrier with NW = 1)
  auto row_sum = [&](float x, int which) {
    x = warp_sum(x);
    if constexpr (NW > 1) {
      if ((threadIdx.x & 31) == 0) part[which][warp] = x;
      __syncthreads();
      x = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i) x += part[which][i];
    }
    return x;
  };
  float h[NV][8], b[NV][8];
  const int units = p.width / 8;
  {
    Raw8<H> hr[NV];
    Raw8<B> br[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int unit = unit0 + v * kStep;
      hr[v] = Raw8<H>{};
      br[v] = Raw8<B>{};
      if (unit < units) {
        hr[v] = load_raw(static_cast<const H*>(p.h) + row * p.h_stride + unit * 8);
        br[v] = load_raw(static_cast<const B*>(p.b) + row * p.b_stride + unit * 8);
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      widen(hr[v], h[v]);
      widen(br[v], b[v]);
    }
  }
  if (p.h_codes != nullptr) keep8(h, row, p.width, unit0, kStep, p.h_codes, p.h_exps);
  if (p.b_codes != nullptr) keep8(b, row, p.width, unit0, kStep, p.b_codes, p.b_exps);
  float r = 1.f;
  if (p.post != nullptr) {
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(b[v][i], b[v][i], sum);
    r = 1.f / sqrtf(row_sum(sum, 0) / static_cast<float>(p.width) + p.eps);
    if (p.r_post != nullptr && unit0 == 0) p.r_post[row] = r;
  }
  const float* gate =
      p.gate == nullptr ? nullptr : p.gate + static_cast<int64_t>(row / p.gate_rows) * p.width;
  float sum = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int unit = unit0 + v * kStep;
    if (unit >= units) continue;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = p.scale;
    if (gate != nullptr) {
      float g[8];
      load8(gate + unit * 8, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= g[i];
    }
    if (p.post != nullptr) {
      float g[8];
      load8(p.post + unit * 8, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) b[v][i] *= r * g[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[v][i] = fmaf(f[i], b[v][i], h[v][i]);
      sum = fmaf(h[v][i], h[v][i], sum);
    }
    store8(static_cast<H*>(p.y) + row * p.y_stride + unit * 8, h[v]);
  }
  if (p.pre == nullptr) return;
  r = 1.f / sqrtf(row_sum(sum, 1) / static_cast<float>(p.width) + p.eps);
  if (p.r_pre != nullptr && unit0 == 0) p.r_pre[row] = r;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int unit = unit0 + v * kStep;
    if (unit >= units) continue;
    float g[8];
    load8(p.pre + unit * 8, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[v][i] *= r * g[i];
    store8(static_cast<B*>(p.u) + row * p.u_stride + unit * 8, h[v]);
  }
}

template <typename B, typename H>
cudaError_t launch_join(const Join& p, cudaStream_t s) {
  const int units = p.width / 8;
  auto go = [&](auto kernel, int warps) {
    const int per_block = warps == 1 ? 4 : 1;
    return launch_pdl(kernel, dim3((p.rows + per_block - 1) / per_block),
                      dim3(warps == 1 ? 128 : warps * 32), 0, s, p);
  };
  // A warp has up to 1024 elements of a row, so that rows up to there need no barrier; few rows
  // are spread over more warps, for which a row is a shorter chain.
  const bool few = p.rows < 4 * num_sms();
  if (units <= 32) return go(join_kernel<B, H, 1, 1>, 1);
  if (units <= 64 && !few) return go(join_kernel<B, H, 1, 2>, 1);
  if (units <= 128) return few ? go(join_kernel<B, H, 4, 1>, 4) : go(join_kernel<B, H, 1, 4>, 1);
  if (units <= 256) return few ? go(join_kernel<B, H, 8, 1>, 8) : go(join_kernel<B, H, 2, 4>, 2);
  if (units <= 512) return few ? go(join_kernel<B, H, 16, 1>, 16) : go(join_kernel<B, H, 4, 4>, 4);
  return go(join_kernel<B, H, 8, 4>, 8);
}

// ------------------------------------------------------------------------------ gradient
// A block has the rows [rows c / grid, rows (c + 1) / grid) and a thread the same columns of all
// of them, so that the sums over tokens stay in registers: dpost, dpre, and dgate's of the present
// gate, which leaves when its last row is through: to dgate itself where all its rows were the
// block's, else to the block's first (it began in an earlier block) or last partial row. join_sums
// adds up the blocks' rows in their order: the same bits every time.
//
// A row takes one barrier: mean(e n) needs d, which needs mean(g m), but it is linear in it:
//   sum e n = s (sum (dy + r_pre g) q - r_pre mean(g m) sum m q),  q = gate post n.
struct JoinBwd {
  int rows, width;
  const float *post, *pre, *gate;
  int gate_rows;
  float scale;
  const void *dy, *du, *h, *b;
  int64_t dy_stride, du_stride, h_stride, b_stride;
  const uint8_t *h_exps, *b_exps;  // not null: h, b are codes
  const float *r_post, *r_pre;
  void *dh, *db;
  int64_t dh_stride, db_stride;
  float *d_post, *d_pre, *d_gate;
  float* part;  // [4][grid][width]: dpost, dpre, dgate's first and last
  int grid;
  int one_gate;  // every row has the same gate: dpost is the gate times dgate's sum
};

__host__ __device__ inline int first_row(int rows, int grid, int c) {
  return static_cast<int>(static_cast<int64_t>(rows) * c / grid);
}
// the block that has this row
__host__ __device__ inline int block_of(int rows, int grid, int row) {
  return static_cast<int>(((static_cast<int64_t>(row) + 1) * grid - 1) / rows);
}

template <typename B, typename H>
struct Inputs {
  Raw8<H> dy, h;
  Raw8<B> du, b;
  uint32_t h_byte, b_byte;
};

template <typename B, typename H, int NT, int NV>
__global__ void __launch_bounds__(NT) join_bwd_kernel(const __grid_constant__ JoinBwd p) {
  constexpr int NW = NT / 32;
  __shared__ float4 part[2][NW];
  grid_dep_wait();
  grid_dep_launch();
  const int units = p.width / 8, blocks = (p.width + kKeptBlock - 1) / kKeptBlock;
  const int row0 = first_row(p.rows, p.grid, blockIdx.x);
  const int row1 = first_row(p.rows, p.grid, blockIdx.x + 1);
  const float inv_width = 1.f / static_cast<float>(p.width);
  Inputs<B, H> in[NV];
  float next_post = 1.f, next_pre = 0.f;
  auto fetch = [&](int row) {
    if (p.post != nullptr) next_post = p.r_post[row];
    if (p.pre != nullptr) next_pre = p.r_pre[row];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int unit = threadIdx.x + v * NT;
      Inputs<B, H>& x = in[v];
      if (unit < units) {
        const int64_t at = unit * 8;
        if (p.dy != nullptr) x.dy = load_raw(static_cast<const H*>(p.dy) + row * p.dy_stride + at);
        if (p.pre != nullptr) {
          x.du = load_raw(static_cast<const B*>(p.du) + row * p.du_stride + at);
          if (p.h_exps != nullptr) {
            const uint2 c =
                *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(p.h) + row * p.h_stride + at);
            x.h.a.x = c.x;
            x.h.a.y = c.y;
            x.h_byte = p.h_exps[static_cast<int64_t>(row) * blocks + unit / 4];
          } else {
            x.h = load_raw(static_cast<const H*>(p.h) + row * p.h_stride + at);
          }
        }
        if (p.b_exps != nullptr) {
          const uint2 c =
              *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(p.b) + row * p.b_stride + at);
          x.b.a.x = c.x;
          x.b.a.y = c.y;
          x.b_byte = p.b_exps[static_cast<int64_t>(row) * blocks + unit / 4];
        } else {
          x.b = load_raw(static_cast<const B*>(p.b) + row * p.b_stride + at);
        }
      }
    }
  };
#pragma unroll
  for (int v = 0; v < NV; ++v) in[v] = Inputs<B, H>{};
  float s_post[NV][8], s_pre[NV][8], s_gate[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) s_post[v][i] = s_pre[v][i] = s_gate[v][i] = 0.f;
  const int64_t plane = static_cast<int64_t>(p.grid) * p.width;
  float* mine = p.part + static_cast<int64_t>(blockIdx.x) * p.width;
  int gate_at = p.gate != nullptr ? row0 / p.gate_rows : 0;
  // dgate's sum of the present gate leaves: with the gain where it is complete (the only gate's is
  // left to join_sums, which makes dpost of it too)
  auto leave = [&]() {
    const int64_t first = static_cast<int64_t>(gate_at) * p.gate_rows;
    const int64_t end = first + p.gate_rows;
    const bool whole = !p.one_gate && first >= row0 && (end < p.rows ? end : p.rows) <= row1;
    float* to = whole ? p.d_gate + static_cast<int64_t>(gate_at) * p.width
                      : mine + (first < row0 ? 2 : 3) * plane;
    if (whole && p.d_gate == nullptr) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int unit = threadIdx.x + v * NT;
      if (unit >= units) continue;
      if (whole && p.post != nullptr) {
        float g[8];
        load8(p.post + unit * 8, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) s_gate[v][i] *= g[i];
      }
      store8(to + unit * 8, s_gate[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) s_gate[v][i] = 0.f;
    }
  };
  if (row0 < row1) fetch(row0);
  for (int row = row0; row < row1; ++row) {
    if (p.gate != nullptr && row / p.gate_rows != gate_at) {
      leave();
      gate_at = row / p.gate_rows;
    }
    // into floats, and the next row's inputs on their way
    float n[NV][8], d[NV][8], m[NV][8], q[NV][8];
    const float r_post = next_post, r_pre = next_pre;
    float3 sum = make_float3(0.f, 0.f, 0.f);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Inputs<B, H>& x = in[v];
      const int unit = threadIdx.x + v * NT;
      const bool here = unit < units;
      if (p.b_exps != nullptr)
        kept_values(make_uint2(x.b.a.x, x.b.a.y), x.b_byte, n[v]);
      else
        widen(x.b, n[v]);
      widen(x.dy, d[v]);
      float post[8], g[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        n[v][i] *= r_post;
        q[v][i] = p.scale;
        post[i] = 1.f;
      }
      if (p.gate != nullptr && here) {
        load8(p.gate + static_cast<int64_t>(gate_at) * p.width + unit * 8, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) q[v][i] *= g[i];
      }
      if (p.post != nullptr && here) load8(p.post + unit * 8, post);
#pragma unroll
      for (int i = 0; i < 8; ++i) q[v][i] *= post[i];  // e = q d
      if (p.pre != nullptr) {
        float du[8], pre[8];
        if (p.h_exps != nullptr)
          kept_values(make_uint2(x.h.a.x, x.h.a.y), x.h_byte, m[v]);
        else
          widen(x.h, m[v]);
        widen(x.du, du);
#pragma unroll
        for (int i = 0; i < 8; ++i) pre[i] = 0.f;
        if (here) load8(p.pre + unit * 8, pre);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          m[v][i] = fmaf(q[v][i], n[v][i], m[v][i]) * r_pre;  // y r_pre
          s_pre[v][i] = fmaf(du[i], m[v][i], s_pre[v][i]);
          g[i] = du[i] * pre[i];
          sum.x = fmaf(g[i], m[v][i], sum.x);
          d[v][i] = fmaf(r_pre, g[i], d[v][i]);
          sum.z = fmaf(m[v][i], q[v][i] * n[v][i], sum.z);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum.y = fmaf(d[v][i], q[v][i] * n[v][i], sum.y);
    }
    if (row + 1 < row1) fetch(row + 1);
    sum.x = warp_sum(sum.x);
    sum.y = warp_sum(sum.y);
    sum.z = warp_sum(sum.z);
    if constexpr (NW > 1) {
      float4* to = part[row & 1];
      if ((threadIdx.x & 31) == 0) to[threadIdx.x >> 5] = make_float4(sum.x, sum.y, sum.z, 0.f);
      __syncthreads();
      sum = make_float3(0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        const float4 x = to[i];
        sum.x += x.x;
        sum.y += x.y;
        sum.z += x.z;
      }
    }
    const float mean_gm = r_pre * sum.x * inv_width;  // r_pre mean(g m)
    const float mean_en = p.post != nullptr ? (sum.y - mean_gm * sum.z) * inv_width : 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int unit = threadIdx.x + v * NT;
      if (unit >= units) continue;
      if (p.pre != nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[v][i] = fmaf(-mean_gm, m[v][i], d[v][i]);
      }
      if (p.dh != nullptr) store8(static_cast<H*>(p.dh) + row * p.dh_stride + unit * 8, d[v]);
      float db[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float wn = p.scale * d[v][i] * n[v][i];
        s_gate[v][i] += wn;
        db[i] = r_post * fmaf(-mean_en, n[v][i], q[v][i] * d[v][i]);
      }
      if (p.post != nullptr && !p.one_gate) {
        float g[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.f;
        if (p.gate != nullptr) load8(p.gate + static_cast<int64_t>(gate_at) * p.width + unit * 8, g);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          s_post[v][i] = fmaf(p.scale * d[v][i] * n[v][i], g[i], s_post[v][i]);
      }
      if (p.db != nullptr) store8(static_cast<B*>(p.db) + row * p.db_stride + unit * 8, db);
    }
  }
  if (row0 < row1 && p.gate != nullptr) leave();
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int unit = threadIdx.x + v * NT;
    if (unit >= units) continue;
    if (p.post != nullptr && !p.one_gate) store8(mine + unit * 8, s_post[v]);
    if (p.pre != nullptr) store8(mine + plane + unit * 8, s_pre[v]);
  }
}

// The blocks' partial rows added up in their order. Grid: (32 columns, what): 0 dpost, 1 dpre, then
// the gates that several blocks share, by the border between blocks c and c + 1 that is their first.
constexpr int kSumThreads = 512, kSumSlices = kSumThreads / 32;
__global__ void __launch_bounds__(kSumThreads) join_sums_kernel(const __grid_constant__ JoinBwd p) {
  __shared__ float part[kSumSlices][32];
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + lane;
  const int64_t plane = static_cast<int64_t>(p.grid) * p.width;
  // rows [c0, c1) of a plane; row c0 is another plane's where it is said to be
  auto total = [&](int which, int c0, int c1, int first_which) {
    float sum = 0.f;
    const int n = c1 - c0;
    const int a = c0 + n * slice / kSumSlices, e = c0 + n * (slice + 1) / kSumSlices;
    if (col < p.width) {
#pragma unroll 8
      for (int c = a; c < e; ++c)
        sum += p.part[(c == c0 ? first_which : which) * plane + static_cast<int64_t>(c) * p.width + col];
    }
    __syncthreads();
    part[slice][lane] = sum;
    __syncthreads();
    sum = 0.f;
    if (slice == 0) {
#pragma unroll
      for (int i = 0; i < kSumSlices; ++i) sum += part[i][lane];
    }
    return sum;
  };
  const bool out = slice == 0 && col < p.width;
  if (blockIdx.y == 0) {
    if (p.post == nullptr || p.one_gate || p.d_post == nullptr) return;
    const float sum = total(0, 0, p.grid, 0);
    if (out) p.d_post[col] = sum;
  } else if (blockIdx.y == 1) {
    if (p.pre == nullptr || p.d_pre == nullptr) return;
    const float sum = total(1, 0, p.grid, 1);
    if (out) p.d_pre[col] = sum;
  } else if (p.one_gate) {
    // the only gate: began in block 0
    const float sum = total(2, 0, p.grid, 3);
    if (!out) return;
    if (p.d_gate != nullptr) p.d_gate[col] = p.post != nullptr ? sum * p.post[col] : sum;
    if (p.post != nullptr && p.d_post != nullptr) p.d_post[col] = sum * p.gate[col];
  } else {
    if (p.d_gate == nullptr) return;
    for (int border = blockIdx.y - 2; border + 1 < p.grid; border += gridDim.y - 2) {
      const int row = first_row(p.rows, p.grid, border + 1);
      const int at = row / p.gate_rows, begin = at * p.gate_rows;
      if (begin == row || block_of(p.rows, p.grid, begin) != border) continue;
      const int64_t end = static_cast<int64_t>(begin) + p.gate_rows;
      const int last = static_cast<int>(end < p.rows ? end : p.rows) - 1;
      const float sum = total(2, border, block_of(p.rows, p.grid, last) + 1, 3);
      if (out)
        p.d_gate[static_cast<int64_t>(at) * p.width + col] =
            p.post != nullptr ? sum * p.post[col] : sum;
    }
  }
}

// threads for a row, and how many blocks of them an SM is given
int bwd_threads(int width) {
  const int units = width / 8;
  int t = 32;
  while (t < units && t < 512) t *= 2;
  return t;
}
int bwd_grid(int rows, int width) {
  const int t = bwd_threads(width);
  const int per_sm = std::max(1, std::min(16, 512 / t));
  return std::max(1, std::min(rows, num_sms() * per_sm));
}

template <typename B, typename H>
cudaError_t launch_join_bwd(const JoinBwd& p, cudaStream_t s) {
  const int t = bwd_threads(p.width);
  auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(p.grid), dim3(t), 0, s, p); };
  cudaError_t e = p.width > 4096 ? go(join_bwd_kernel<B, H, 512, 2>)
                  : t == 32      ? go(join_bwd_kernel<B, H, 32, 1>)
                  : t == 64      ? go(join_bwd_kernel<B, H, 64, 1>)
                  : t == 128     ? go(join_bwd_kernel<B, H, 128, 1>)
                  : t == 256     ? go(join_bwd_kernel<B, H, 256, 1>)
                                 : go(join_bwd_kernel<B, H, 512, 1>);
  if (e != cudaSuccess) return e;
  // (one gate's sum is one item; of several gates at most one begins before every border)
  const int gates = p.gate == nullptr ? 0 : p.one_gate ? 1 : std::min(p.grid - 1, 64);
  if (p.post == nullptr && p.pre == nullptr && gates == 0) return cudaSuccess;
  return launch_pdl(join_sums_kernel, dim3((p.width + 31) / 32, 2 + gates), dim3(kSumThreads), 0, s, p);
}

bool ok_ptr(const void* p, uintptr_t align) {
  return p != nullptr && reinterpret_cast<uintptr_t>(p) % align == 0;
}
// null, or aligned
bool ok_or_null(const void* p, uintptr_t align) { return reinterpret_cast<uintptr_t>(p) % align == 0; }

bool valid(const fd_block_join* j) {
  if (j == nullptr || j->rows < 0 || j->width < 8 || j->width % 8 != 0 || j->width > 8192)
    return false;
  if (j->dtype != FD_DTYPE_BF16 && j->dtype != FD_DTYPE_F16) return false;
  if (j->stream_dtype != FD_DTYPE_F32 && j->stream_dtype != j->dtype) return false;
  if (!std::isfinite(j->scale)) return false;
  if (j->gate != nullptr && j->gate_rows < 1) return false;
  return ok_or_null(j->post_gain, 16) && ok_or_null(j->pre_gain, 16) && ok_or_null(j->gate, 16);
}
// rows of a 16-byte aligned matrix
bool ok_rows(const fd_block_join* j, const void* p, int64_t stride) {
  return ok_ptr(p, 16) && stride % 8 == 0 && (j->rows == 1 || stride >= j->width);
}

}  // namespace
}  // namespace fd

extern "C" {

fd_status fd_op_block_join(const fd_block_join* j, const void* h, int64_t h_stride, const void* b,
                           int64_t b_stride, float eps, void* y, int64_t y_stride, void* u,
                           int64_t u_stride, float* r_post, float* r_pre, int8_t* h_codes,
                           uint8_t* h_exps, int8_t* b_codes, uint8_t* b_exps, void* stream) {
  if (!fd::valid(j) || !std::isfinite(eps) || !(eps >= 0.f)) return FD_ERR_INVALID_ARG;
  if (j->rows == 0) return FD_OK;
  if (!fd::ok_rows(j, h, h_stride) || !fd::ok_rows(j, b, b_stride) || !fd::ok_rows(j, y, y_stride))
    return FD_ERR_INVALID_ARG;
  if (j->pre_gain != nullptr ? !fd::ok_rows(j, u, u_stride) : u != nullptr) return FD_ERR_INVALID_ARG;
  if (!fd::ok_or_null(r_post, 4) || !fd::ok_or_null(r_pre, 4)) return FD_ERR_INVALID_ARG;
  if ((h_codes == nullptr) != (h_exps == nullptr) || (b_codes == nullptr) != (b_exps == nullptr) ||
      !fd::ok_or_null(h_codes, 8) || !fd::ok_or_null(b_codes, 8))
    return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  const fd::Join p{j->rows,  j->width, j->post_gain, j->pre_gain, j->gate,  j->gate_rows,
                   j->scale, eps,      h,            b,           h_stride, b_stride,
                   y,        u,        y_stride,     u_stride,    r_post,   r_pre,
                   h_codes,  b_codes,  h_exps,       b_exps};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool wide = j->stream_dtype == FD_DTYPE_F32;
  const cudaError_t e =
      j->dtype == FD_DTYPE_BF16
          ? (wide ? fd::launch_join<__nv_bfloat16, float>(p, s)
                  : fd::launch_join<__nv_bfloat16, __nv_bfloat16>(p, s))
          : (wide ? fd::launch_join<__half, float>(p, s) : fd::launch_join<__half, __half>(p, s));
  return e == cudaSuccess ? FD_OK : FD_ERR_CUDA;
}

size_t fd_block_join_bwd_workspace_bytes(int rows, int width) {
  if (rows < 1 || width < 8 || width % 8 != 0 || width > 8192) return 0;
  return static_cast<size_t>(4) * fd::bwd_grid(rows, width) * width * sizeof(float);
}

fd_status fd_op_block_join_bwd(const fd_block_join* j, const void* dy, int64_t dy_stride,
                               const void* du, int64_t du_stride, const void* h, int64_t h_stride,
                               const uint8_t* h_exps, const void* b, int64_t b_stride,
                               const uint8_t* b_exps, const float* r_post, const float* r_pre,
                               void* dh, int64_t dh_stride, void* db, int64_t db_stride,
                               float* d_post, float* d_pre, float* d_gate, void* workspace,
                               void* stream) {
  if (!fd::valid(j)) return FD_ERR_INVALID_ARG;
  auto kept_rows = [&](const void* p, int64_t stride, const uint8_t* exps) {
    return exps != nullptr ? fd::ok_ptr(p, 8) && stride == j->width : fd::ok_rows(j, p, stride);
  };
  const bool pre = j->pre_gain != nullptr, post = j->post_gain != nullptr, gate = j->gate != nullptr;
  if ((d_post != nullptr && !post) || (d_pre != nullptr && !pre) || (d_gate != nullptr && !gate) ||
      !fd::ok_or_null(d_post, 16) || !fd::ok_or_null(d_pre, 16) || !fd::ok_or_null(d_gate, 16))
    return FD_ERR_INVALID_ARG;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (j->rows == 0) {
    // sums over no tokens (a gate of no tokens has no rows)
    if (d_post == nullptr && d_pre == nullptr) return FD_OK;
    const fd_status st = fd::check_device();
    if (st != FD_OK) return st;
    const size_t bytes = static_cast<size_t>(j->width) * sizeof(float);
    if (d_post != nullptr && cudaMemsetAsync(d_post, 0, bytes, s) != cudaSuccess) return FD_ERR_CUDA;
    if (d_pre != nullptr && cudaMemsetAsync(d_pre, 0, bytes, s) != cudaSuccess) return FD_ERR_CUDA;
    return FD_OK;
  }
  if (dy != nullptr && !fd::ok_rows(j, dy, dy_stride)) return FD_ERR_INVALID_ARG;
  if (pre ? !fd::ok_rows(j, du, du_stride) || !fd::ok_ptr(r_pre, 4) || !kept_rows(h, h_stride, h_exps)
          : du != nullptr || dy == nullptr)
    return FD_ERR_INVALID_ARG;
  if (!kept_rows(b, b_stride, b_exps) || (post && !fd::ok_ptr(r_post, 4))) return FD_ERR_INVALID_ARG;
  if ((dh != nullptr && !fd::ok_rows(j, dh, dh_stride)) ||
      (db != nullptr && !fd::ok_rows(j, db, db_stride)) || !fd::ok_ptr(workspace, 16))
    return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  const fd::JoinBwd p{j->rows,    j->width,  j->post_gain, j->pre_gain, j->gate, j->gate_rows,
                      j->scale,   dy,        du,           h,           b,       dy_stride,
                      du_stride,  h_stride,  b_stride,     h_exps,      b_exps,  r_post,
                      r_pre,      dh,        db,           dh_stride,   db_stride, d_post,
                      d_pre,      d_gate,    static_cast<float*>(workspace),
                      fd::bwd_grid(j->rows, j->width),
                      gate && j->gate_rows >= j->rows ? 1 : 0};
  const bool wide = j->stream_dtype == FD_DTYPE_F32;
  const cudaError_t e =
      j->dtype == FD_DTYPE_BF16
          ? (wide ? fd::launch_join_bwd<__nv_bfloat16, float>(p, s)
                  : fd::launch_join_bwd<__nv_bfloat16, __nv_bfloat16>(p, s))
          : (wide ? fd::launch_join_bwd<__half, float>(p, s)
                  : fd::launch_join_bwd<__half, __half>(p, s));
  return e == cudaSuccess ? FD_OK : FD_ERR_CUDA;
}

}  // extern "C"
