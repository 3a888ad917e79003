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
// Every row is read and written once, its sums taken while it is in registers. Measured on inputs that are
// not in L2, of a plain copy's rate:
//   6240 x 1024, bf16 on fp32, both inputs kept in 8 bits: join      18.5 us  4.9 TB/s, 72 %
//     its gradient from 8 bits, a gate, two launches                  23.0 us  3.9 TB/s, 58 %
//   16001 x 4096, bf16, a gate for 1000 rows: gradient               137 us   5.8 TB/s, 85 %
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

// a row's elements as they lie in memory (and as floats) into their 8-bit form
template <typename T, int NV>
__device__ __forceinline__ void keep8(const Raw8<T> (&raw)[NV], const float (&x)[NV][8], int row, int width,
                                      int unit0, int step, int8_t* codes, uint8_t* exps) {
  const int blocks = (width + kKeptBlock - 1) / kKeptBlock;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const uint32_t byte = kept_exponent(block_top(raw[v]));
    const uint2 eight = kept_codes(x[v], byte);
    const int unit = unit0 + v * step;
    if (unit >= width / 8) continue;
    *reinterpret_cast<uint2*>(codes + static_cast<int64_t>(row) * width + unit * 8) = eight;
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
    if (p.h_codes != nullptr) keep8(hr, h, row, p.width, unit0, kStep, p.h_codes, p.h_exps);
    if (p.b_codes != nullptr) keep8(br, b, row, p.width, unit0, kStep, p.b_codes, p.b_exps);
  }
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
  // Up to 1024 elements a group of eight a thread (6240 x 1024: 18.3 us, two groups 19.4, four 22.8), past that
  // two (8000 x 4096: 78 us, one group 90). Few rows are spread over more warps, for which a row is a
  // shorter chain: 2048 elements, 300 rows 2.5 us instead of 2.7, 400 either way 3.0, 600 rows 5.1 instead of 4.4;
  // 2056 elements, 150 rows 2.4 instead of 2.5, 300 rows 3.5 instead of 2.9 (4096: 2.8 either way, 5.7 instead of 4.8).
  const int few_halves = units <= 256 ? 5 : 2;  // of a wave of a block an SM
  const bool few = 2 * static_cast<int64_t>(p.rows) <= few_halves * num_sms();
  if (units <= 32) return go(join_kernel<B, H, 1, 1>, 1);
  if (units <= 64) return go(join_kernel<B, H, 2, 1>, 2);
  if (units <= 128) return go(join_kernel<B, H, 4, 1>, 4);
  if (units <= 256) return few ? go(join_kernel<B, H, 8, 1>, 8) : go(join_kernel<B, H, 4, 2>, 4);
  if (units <= 512) return few ? go(join_kernel<B, H, 16, 1>, 16) : go(join_kernel<B, H, 8, 2>, 8);
  return go(join_kernel<B, H, 16, 2>, 16);
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

// A thread's eight columns of a row as they lie in memory, fetched a row ahead.
template <typename B, typename H>
struct Inputs {
  Raw8<H> dy, h;
  Raw8<B> du, b;
  uint32_t h_byte, b_byte;
};

// Bound by its instructions (pairs of fp32 throughout, gains and gate in registers while they stay the
// same): copies ahead into a ring in shared memory, three or four rows deep, made it slower (480p chunk 24.7 to 35
// us), fewer instructions faster.
// FORM: what there is, known beforehand where it is what training has, else looked up. (The branches for it, and
// three sums a row that were added up apart, cost 2 and 9 us of the two cases above; 8000 rows of 8192, which spill
// more for them, took 370 us instead of 242.)
enum Form { kSome, kAll, kAllKept };  // kAll: both norms, dy, dh and db; kAllKept: and both inputs in 8 bits
template <typename B, typename H, int NT, int NV, Form FORM>
__global__ void __launch_bounds__(NT) join_bwd_kernel(const __grid_constant__ JoinBwd p) {
  constexpr int NW = NT / 32;
  constexpr bool kKeep = NV == 1;  // gains stay in registers
  __shared__ float part[2][NW][4];
  grid_dep_wait();
  grid_dep_launch();
  const int units = p.width / 8, blocks = (p.width + kKeptBlock - 1) / kKeptBlock;
  const int row0 = first_row(p.rows, p.grid, blockIdx.x);
  const int row1 = first_row(p.rows, p.grid, blockIdx.x + 1);
  const float inv_width = 1.f / static_cast<float>(p.width);
  const int lane = threadIdx.x & 31;
  const bool pre = FORM != kSome || p.pre != nullptr, post = FORM != kSome || p.post != nullptr;
  const bool has_dy = FORM != kSome || p.dy != nullptr;
  const bool h_kept = FORM == kAllKept || (FORM == kSome && p.h_exps != nullptr);
  const bool b_kept = FORM == kAllKept || (FORM == kSome && p.b_exps != nullptr);
  Inputs<B, H> in[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) in[v] = Inputs<B, H>{};
  float next_post = 1.f, next_pre = 0.f;
  auto fetch = [&](int row) {
    if (post) next_post = p.r_post[row];
    if (pre) next_pre = p.r_pre[row];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int unit = threadIdx.x + v * NT;
      Inputs<B, H>& x = in[v];
      if (unit >= units) continue;
      auto codes = [&](const void* from, int64_t stride) {
        return *reinterpret_cast<const uint2*>(static_cast<const int8_t*>(from) + row * stride + unit * 8);
      };
      if (has_dy) x.dy = load_raw(static_cast<const H*>(p.dy) + row * p.dy_stride + unit * 8);
      if (pre) {
        x.du = load_raw(static_cast<const B*>(p.du) + row * p.du_stride + unit * 8);
        if (h_kept) {
          const uint2 c = codes(p.h, p.h_stride);
          x.h.a.x = c.x;
          x.h.a.y = c.y;
          x.h_byte = p.h_exps[static_cast<int64_t>(row) * blocks + unit / 4];
        } else {
          x.h = load_raw(static_cast<const H*>(p.h) + row * p.h_stride + unit * 8);
        }
      }
      if (b_kept) {
        const uint2 c = codes(p.b, p.b_stride);
        x.b.a.x = c.x;
        x.b.a.y = c.y;
        x.b_byte = p.b_exps[static_cast<int64_t>(row) * blocks + unit / 4];
      } else {
        x.b = load_raw(static_cast<const B*>(p.b) + row * p.b_stride + unit * 8);
      }
    }
  };
  // The row beyond the one fetched ahead goes into L2, which its loads then find it in: 16001 x 4096 in 137 us (four
  // rows ahead 141, none 153), 6240 x 1024 from 8 bits in 23.0 (24.6, 24.6).
  auto into_l2 = [&](int row) {
    auto line = [](const void* x) { asm volatile("prefetch.global.L2 [%0];" ::"l"(x)); };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int unit = threadIdx.x + v * NT;
      if (unit % 4 != 0 || unit >= units) continue;  // 64 bytes of 16-bit elements
      if (has_dy) line(static_cast<const H*>(p.dy) + row * p.dy_stride + unit * 8);
      if (pre) {
        line(static_cast<const B*>(p.du) + row * p.du_stride + unit * 8);
        line(static_cast<const char*>(p.h) + (row * p.h_stride + unit * 8) * (h_kept ? 1 : sizeof(H)));
      }
      line(static_cast<const char*>(p.b) + (row * p.b_stride + unit * 8) * (b_kept ? 1 : sizeof(B)));
    }
  };
  int gate_at = p.gate != nullptr ? row0 / p.gate_rows : 0;
  int64_t gate_end = p.gate != nullptr ? (static_cast<int64_t>(gate_at) + 1) * p.gate_rows : p.rows;
  // scale gate post of the present gate
  auto factors = [&](int unit) {
    Pairs q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q.v[i] = pack_f32x2(p.scale, p.scale);
    if (p.gate != nullptr) {
      const Pairs g = load8_2(p.gate + static_cast<int64_t>(gate_at) * p.width + unit * 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) q.v[i] = mul2(q.v[i], g.v[i]);
    }
    if (post) {
      const Pairs g = load8_2(p.post + unit * 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) q.v[i] = mul2(q.v[i], g.v[i]);
    }
    return q;
  };
  // sums over rows: du m; d n of the present gate; gate d n (times scale when they leave)
  Pairs s_pre[NV], s_gate[NV], s_post[NV], q_kept[NV], pre_kept[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int unit = threadIdx.x + v * NT;
    s_pre[v] = s_gate[v] = s_post[v] = q_kept[v] = pre_kept[v] = Pairs{};
    if (kKeep && unit < units) {
      q_kept[v] = factors(unit);
      if (pre) pre_kept[v] = load8_2(p.pre + unit * 8);
    }
  }
  const int64_t plane = static_cast<int64_t>(p.grid) * p.width;
  float* mine = p.part + static_cast<int64_t>(blockIdx.x) * p.width;
  // The present gate's sum leaves: into dpost's, and with the gain to dgate where it is complete (the
  // only gate's is left to join_sums, which makes dpost of it too).
  auto leave = [&]() {
    const int64_t first = gate_end - p.gate_rows;
    const bool whole = !p.one_gate && first >= row0 && (gate_end < p.rows ? gate_end : p.rows) <= row1;
    float* to = whole ? p.d_gate + static_cast<int64_t>(gate_at) * p.width
                      : mine + (first < row0 ? 2 : 3) * plane;
    if (whole && p.d_gate == nullptr) to = nullptr;
    const uint64_t scale2 = pack_f32x2(p.scale, p.scale);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int unit = threadIdx.x + v * NT;
      if (unit >= units) continue;
      const Pairs g = load8_2(p.gate + static_cast<int64_t>(gate_at) * p.width + unit * 8);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s_gate[v].v[i] = mul2(s_gate[v].v[i], scale2);
        s_post[v].v[i] = fma2(s_gate[v].v[i], g.v[i], s_post[v].v[i]);
      }
      if (whole && post) {
        const Pairs gain = load8_2(p.post + unit * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) s_gate[v].v[i] = mul2(s_gate[v].v[i], gain.v[i]);
      }
      if (to != nullptr) store8(to + unit * 8, s_gate[v]);
      s_gate[v] = Pairs{};
    }
  };
  if (row0 < row1) fetch(row0);
#pragma unroll 1
  for (int row = row0; row < row1; ++row) {
    if (row >= gate_end) {
      leave();
      gate_at = row / p.gate_rows;
      gate_end = (static_cast<int64_t>(gate_at) + 1) * p.gate_rows;
      if (kKeep && threadIdx.x < units) q_kept[0] = factors(threadIdx.x);
    }
    // into pairs, and the next row's inputs on their way
    Pairs n[NV], d[NV], m[NV];
    const float r_post = next_post, r_pre = next_pre;
    const uint64_t rpost2 = pack_f32x2(r_post, r_post), rpre2 = pack_f32x2(r_pre, r_pre);
    uint64_t sum_gm = 0, sum_dq = 0, sum_mq = 0;
    Pairs du[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Inputs<B, H>& x = in[v];
      n[v] = b_kept ? kept_values2(make_uint2(x.b.a.x, x.b.a.y), x.b_byte) : widen2(x.b);
      d[v] = widen2(x.dy);
      if (pre) {
        m[v] = h_kept ? kept_values2(make_uint2(x.h.a.x, x.h.a.y), x.h_byte) : widen2(x.h);
        du[v] = widen2(x.du);
      } else {
        m[v] = du[v] = Pairs{};
      }
    }
    if (row + 2 < row1) into_l2(row + 2);
    if (row + 1 < row1) fetch(row + 1);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int unit = threadIdx.x + v * NT;
      if (!kKeep && unit >= units) continue;  // (zeros add nothing: no branch)
      const Pairs q = kKeep ? q_kept[v] : factors(unit);
      Pairs qn;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        n[v].v[i] = mul2(n[v].v[i], rpost2);
        qn.v[i] = mul2(q.v[i], n[v].v[i]);
      }
      if (pre) {
        const Pairs gain = kKeep ? pre_kept[v] : load8_2(p.pre + unit * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          m[v].v[i] = mul2(add2(m[v].v[i], qn.v[i]), rpre2);  // y r_pre
          s_pre[v].v[i] = fma2(du[v].v[i], m[v].v[i], s_pre[v].v[i]);
          const uint64_t g = mul2(du[v].v[i], gain.v[i]);
          sum_gm = fma2(g, m[v].v[i], sum_gm);
          d[v].v[i] = fma2(rpre2, g, d[v].v[i]);
          sum_mq = fma2(m[v].v[i], qn.v[i], sum_mq);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) sum_dq = fma2(d[v].v[i], qn.v[i], sum_dq);
    }
    const float2 a = halves_of(sum_gm), b = halves_of(sum_dq), c = halves_of(sum_mq);
    // The three sums over the row, folded into one value a lane on the way: gm ends in lanes 0-7, mq in 8-15
    // and 24-31, dq in 16-23.
    float at;
    {
      const float gm = a.x + a.y, dq = b.x + b.y, mq = c.x + c.y;
      const bool upper = lane & 16, odd = lane & 8;
      const float x = (upper ? dq : gm) + __shfl_xor_sync(0xffffffffu, upper ? gm : dq, 16);
      const float y = mq + __shfl_xor_sync(0xffffffffu, mq, 16);
      at = (odd ? y : x) + __shfl_xor_sync(0xffffffffu, odd ? x : y, 8);
#pragma unroll
      for (int i = 4; i; i >>= 1) at += __shfl_xor_sync(0xffffffffu, at, i);
    }
    if constexpr (NW > 1) {
      float(*to)[4] = part[row & 1];
      if ((lane & 7) == 0) to[threadIdx.x >> 5][lane >> 3] = at;
      __syncthreads();
      at = to[lane & (NW < 8 ? NW - 1 : 7)][lane >> 3];
      if constexpr (NW > 8) at += to[8 + (lane & 7)][lane >> 3];
#pragma unroll
      for (int i = NW < 8 ? NW / 2 : 4; i; i >>= 1) at += __shfl_xor_sync(0xffffffffu, at, i);
    }
    const float3 sum = make_float3(__shfl_sync(0xffffffffu, at, 0), __shfl_sync(0xffffffffu, at, 16),
                                   __shfl_sync(0xffffffffu, at, 8));
    const float mean_gm = r_pre * sum.x * inv_width;  // r_pre mean(g m)
    const float mean_en = post ? (sum.y - mean_gm * sum.z) * inv_width : 0.f;
    const float en = -r_post * mean_en;
    const uint64_t gm2 = pack_f32x2(-mean_gm, -mean_gm), en2 = pack_f32x2(en, en);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int unit = threadIdx.x + v * NT;
      if (!kKeep && unit >= units) continue;
      const Pairs q = kKeep ? q_kept[v] : factors(unit);
      Pairs db;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (pre) d[v].v[i] = fma2(gm2, m[v].v[i], d[v].v[i]);
        s_gate[v].v[i] = fma2(d[v].v[i], n[v].v[i], s_gate[v].v[i]);
        db.v[i] = fma2(mul2(q.v[i], d[v].v[i]), rpost2, mul2(en2, n[v].v[i]));
      }
      if (unit < units && (FORM != kSome || p.dh != nullptr))
        store8(static_cast<H*>(p.dh) + row * p.dh_stride + unit * 8, d[v]);
      if (unit < units && (FORM != kSome || p.db != nullptr))
        store8(static_cast<B*>(p.db) + row * p.db_stride + unit * 8, db);
    }
  }
  if (row0 < row1 && p.gate != nullptr) leave();
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int unit = threadIdx.x + v * NT;
    if (unit >= units) continue;
    if (p.gate == nullptr) {  // no gate: dpost is the sum itself
#pragma unroll
      for (int i = 0; i < 4; ++i) s_post[v].v[i] = mul2(s_gate[v].v[i], pack_f32x2(p.scale, p.scale));
    }
    if (post && !p.one_gate) store8(mine + unit * 8, s_post[v]);
    if (pre) store8(mine + plane + unit * 8, s_pre[v]);
  }
}

// The blocks' partial rows added up, 32 columns a block, whose 32 warps share out the rows of what blockIdx.y
// says: dpost, dpre, then the gates that several blocks share: some at a time where there are fewer gates than
// blocks, `gate_slices` warps each, else (a gate then spans two or three blocks) 32 of the borders between
// blocks, a warp each.
constexpr int kSumThreads = 1024, kSumSlices = kSumThreads / 32;
__global__ void __launch_bounds__(kSumThreads)
    join_sums_kernel(const __grid_constant__ JoinBwd p, int gate_slices) {
  __shared__ float part[kSumSlices][33];
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + lane;
  const bool there = col < p.width;
  const int64_t plane = static_cast<int64_t>(p.grid) * p.width;
  const float* from = p.part + col;
  const int item = static_cast<int>(blockIdx.y) - 2;
  const int gates = p.gate == nullptr ? 0 : (p.rows + p.gate_rows - 1) / p.gate_rows;
  if (item >= 0 && gates > p.grid) {
    // the gate across the border between blocks c and c + 1, if it begins in block c
    const int c = item * kSumSlices + slice;
    if (c + 1 >= p.grid || !there || p.d_gate == nullptr) return;
    const int row = first_row(p.rows, p.grid, c + 1);
    const int at = row / p.gate_rows, begin = at * p.gate_rows;
    if (begin == row || block_of(p.rows, p.grid, begin) != c) return;
    const int64_t end = static_cast<int64_t>(begin) + p.gate_rows;
    const int last = block_of(p.rows, p.grid, static_cast<int>(end < p.rows ? end : p.rows) - 1);
    float sum = from[3 * plane + static_cast<int64_t>(c) * p.width];
    for (int i = c + 1; i <= last; ++i) sum += from[2 * plane + static_cast<int64_t>(i) * p.width];
    p.d_gate[static_cast<int64_t>(at) * p.width + col] = p.post != nullptr ? sum * p.post[col] : sum;
    return;
  }
  // blocks [c0, c1) of a plane, but block c0 of another where it is a gate's first
  const int slices = item < 0 ? kSumSlices : gate_slices;
  int which = blockIdx.y, first = blockIdx.y, c0 = 0, c1 = p.grid;
  int gate_at = 0;
  if (item < 0) {
    if (item == -1 ? p.d_pre == nullptr : p.d_post == nullptr || p.one_gate) return;
  } else {
    gate_at = (item * kSumSlices + slice) / slices;
    which = 2;
    first = 3;
    c1 = 0;
    if (gate_at < gates) {
      const int64_t begin = static_cast<int64_t>(gate_at) * p.gate_rows, end = begin + p.gate_rows;
      c0 = block_of(p.rows, p.grid, static_cast<int>(begin));
      c1 = block_of(p.rows, p.grid, static_cast<int>(end < p.rows ? end : p.rows) - 1) + 1;
    }
  }
  float sum = 0.f;
  if (there) {
    int c = c0 + slice % slices;
    if (c == c0 && c < c1) {
      sum = __ldcg(from + first * plane + static_cast<int64_t>(c) * p.width);
      c += slices;
    }
    const float* at = from + which * plane + static_cast<int64_t>(c) * p.width;
    const int64_t step = static_cast<int64_t>(slices) * p.width;
    int left = c < c1 ? (c1 - c + slices - 1) / slices : 0;
    for (; left >= 8; left -= 8, at += 8 * step) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __ldcg(at + i * step);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i];
    }
    float x[7];
#pragma unroll
    for (int i = 0; i < 7; ++i) x[i] = i < left ? __ldcg(at + i * step) : 0.f;
#pragma unroll
    for (int i = 0; i < 7; ++i) sum += x[i];
  }
  part[slice][lane] = sum;
  __syncthreads();
  // a warp for every column, a lane for every slice; a gate's slices are neighbours
  sum = part[lane][slice];
  for (int i = slices / 2; i; i >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, i);
  const int64_t at = blockIdx.x * 32 + slice;
  if (lane % slices != 0 || at >= p.width) return;
  if (item < 0) {
    (item == -1 ? p.d_pre : p.d_post)[at] = sum;
    return;
  }
  gate_at = (item * kSumSlices + lane) / slices;
  if (gate_at >= gates) return;
  const int64_t begin = static_cast<int64_t>(gate_at) * p.gate_rows, end = begin + p.gate_rows;
  const bool shared = p.one_gate || block_of(p.rows, p.grid, static_cast<int>(begin)) !=
                                        block_of(p.rows, p.grid, static_cast<int>(end < p.rows ? end : p.rows) - 1);
  // (a gate of one block alone has left from there)
  if (shared && p.d_gate != nullptr)
    p.d_gate[static_cast<int64_t>(gate_at) * p.width + at] = p.post != nullptr ? sum * p.post[at] : sum;
  // one gate: dpost is the gate times the sum without the gain
  if (p.one_gate && p.post != nullptr && p.d_post != nullptr) p.d_post[at] = sum * p.gate[at];
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
  const bool all = p.post != nullptr && p.pre != nullptr && p.dy != nullptr && p.dh != nullptr && p.db != nullptr;
  auto go = [&](auto some, auto as_they_are, auto kept) {
    const bool mixed = (p.h_exps == nullptr) != (p.b_exps == nullptr);
    return launch_pdl(!all || mixed ? some : p.h_exps != nullptr ? kept : as_they_are, dim3(p.grid),
                      dim3(t), 0, s, p);
  };
#define FD_FORMS(NT, NV) \
  go(join_bwd_kernel<B, H, NT, NV, kSome>, join_bwd_kernel<B, H, NT, NV, kAll>,  \
     join_bwd_kernel<B, H, NT, NV, kAllKept>)
  const cudaError_t e = p.width > 4096 ? FD_FORMS(512, 2)
                        : t == 32      ? FD_FORMS(32, 1)
                        : t == 64      ? FD_FORMS(64, 1)
                        : t == 128     ? FD_FORMS(128, 1)
                        : t == 256     ? FD_FORMS(256, 1)
                                       : FD_FORMS(512, 1);
#undef FD_FORMS
  if (e != cudaSuccess) return e;
  const int64_t gates =
      p.gate == nullptr ? 0 : (static_cast<int64_t>(p.rows) + p.gate_rows - 1) / p.gate_rows;
  // four partial rows a warp and gate, about
  int slices = kSumSlices, items = (p.grid - 1 + kSumSlices - 1) / kSumSlices;
  if (gates <= p.grid) {
    while (slices > 1 && static_cast<int64_t>(slices) * 2 * gates > p.grid) slices /= 2;
    items = static_cast<int>((gates * slices + kSumSlices - 1) / kSumSlices);
  }
  if (p.post == nullptr && p.pre == nullptr && gates == 0) return cudaSuccess;
  return launch_pdl(join_sums_kernel, dim3((p.width + 31) / 32, 2 + items), dim3(kSumThreads), 0, s, p, slices);
}

bool ok_ptr(const void* p, uintptr_t align) {
  return p != nullptr && reinterpret_cast<uintptr_t>(p) % align == 0;
}
// null, or aligned
bool ok_or_null(const void* p, uintptr_t align) { return reinterpret_cast<uintptr_t>(p) % align == 0; }

constexpr int kMaxRows = 1 << 30;  // (sums of rows and gate_rows, cut to rows, stay within 32 bits)
bool valid(const fd_block_join* j) {
  if (j == nullptr || j->rows < 0 || j->rows > kMaxRows || j->width < 8 || j->width % 8 != 0 || j->width > 8192)
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
// results that begin at the same address
bool meet(const void* a, const void* b) { return a != nullptr && a == b; }
// a result in the place of an input: of the same rows
bool ok_place(const void* to, int64_t to_stride, const void* from, int64_t from_stride) {
  return !meet(to, from) || to_stride == from_stride;
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
  if (fd::meet(y, u) || fd::meet(y, b) || fd::meet(u, h) || fd::meet(r_post, r_pre) ||
      fd::meet(h_codes, b_codes) || fd::meet(h_exps, b_exps) || !fd::ok_place(y, y_stride, h, h_stride) ||
      !fd::ok_place(u, u_stride, b, b_stride))
    return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  const fd::Join p{j->rows,  j->width, j->post_gain, j->pre_gain, j->gate,  std::min(j->gate_rows, j->rows),
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
  if (rows < 1 || rows > fd::kMaxRows || width < 8 || width % 8 != 0 || width > 8192) return 0;
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
  if (fd::meet(dh, db) || fd::meet(dh, du) || fd::meet(dh, b) || fd::meet(db, dy) || (pre && fd::meet(dh, h)) ||
      (pre && fd::meet(db, h)) || fd::meet(d_post, d_pre) || fd::meet(d_post, d_gate) ||
      fd::meet(d_pre, d_gate) || !fd::ok_place(dh, dh_stride, dy, dy_stride) ||
      !fd::ok_place(db, db_stride, du, du_stride) || (b_exps != nullptr && fd::meet(db, b)) ||
      !fd::ok_place(db, db_stride, b, b_stride))
    return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  const fd::JoinBwd p{j->rows,    j->width,  j->post_gain, j->pre_gain, j->gate, std::min(j->gate_rows, j->rows),
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
