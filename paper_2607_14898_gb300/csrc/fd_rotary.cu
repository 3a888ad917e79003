// Rotary positions as an operator of its own: queries and keys of T tokens turned by 1 to 3
// position axes, or their gradients turned back (fd_op_rotary).
//
// For pair (a, b) at frequency f (radians per position) and angle t = pos f:
//   a' = m (a cos t - b sin t),  b' = m (a sin t + b cos t);  the gradient has -t for t.
// The phase pos f / 2 pi is wanted modulo one turn only. f / 2 pi is kept as a 64-bit integer
// F in units of 2^-64 turns; pos F in wrapping 64-bit arithmetic is then the phase modulo one
// turn, exact in the product: what is left is the rounding of F (f as a double), |pos| f 2^-53, below
// 3e-7 rad for any int32 position, where fp32 pos * f is already 0.03 rad off at position 10^6.
// Its upper 32 bits, as a signed fraction of half a turn, go to sincospif where the outputs are fp32. For
// 16-bit outputs the hardware's sine and cosine do: at most 4.2e-7 off on [-pi, pi], 3e-7 more
// from the rounding of the angle and 1.8e-7 from the products, 9e-7 m (|a| + |b|) together, where the
// output's own rounding is 2^-9 (bf16) or 2^-12 of it (40001 x 40 heads below: 181 us with sincospif).
//
// Bound by memory: every element is read and written once. A thread owns one chunk (16 bytes
// of elements, with their 16 bytes of partners in the half layout) of one token and
// walks over some of the token's heads, so that the sines (14 to 50 instructions a pair) are
// computed once for them; the lanes of a head are neighbours, so accesses are whole lines. Up
// to kHeadsPerThread heads a thread once the launch fills the GPU, fewer for few tokens, where
// latency counts and a thread per (token, head, chunk) is the shortest chain. 40001 tokens of 40
// heads of 128 elements, 64 of them turned in halves (819 MB read and written): 155 us, 5.3 TB/s.
#include <algorithm>
#include <cmath>
#include <new>

#include "fd_internal.h"
#include "fd_ptx.cuh"
#include "flashdec_ops.h"

struct fd_rotary_s {
  fd_rotary_config cfg;
  uint64_t turn[128];  // 2^-64 turns per position of every pair
};

namespace fd {
namespace {

constexpr int kMaxPairs = 128;
constexpr int kThreads = 128, kMaxThreads = 256;  // a head has up to 254 chunks of one element
constexpr int kHeadsPerThread = 20;
constexpr int kVectors = 4;  // in flight a thread

struct RotaryParams {
  uint64_t turn[kMaxPairs];
  int axis_end[3];  // first pair past each axis
  int axes;
  int head_dim, rot_dim;
  int half;      // the half layout
  float sign;    // -1: gradient
  float amplitude;
  int tokens;
  const int32_t* pos;
  int q_heads, heads;  // heads: queries' and keys'
  const void* in[2];
  void* out[2];
  int64_t in_token[2], in_head[2], out_token[2], out_head[2];
  int copy_tail[2];    // elements past rot_dim have to be copied (the output is not the input)
  int lanes;           // chunks a head
  int rot_lanes;       // the first of them hold pairs
  int head_slots;      // threads that share a (token, chunk); slot s has heads s, s + slots, ..
};

template <int BYTES>
struct Raw;
template <>
struct Raw<16> { using type = uint4; };
template <>
struct Raw<8> { using type = uint2; };
template <>
struct Raw<4> { using type = uint32_t; };
template <>
struct Raw<2> { using type = uint16_t; };

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f(float x, float& y) { y = x; }
__device__ __forceinline__ void from_f(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_f(float x, __half& y) { y = __float2half_rn(x); }

// NV elements moved by one access
template <typename T, int NV>
union Vec {
  typename Raw<NV * sizeof(T)>::type raw;
  T e[NV];
  __device__ Vec() {}
};

template <typename T, int NV>
__device__ __forceinline__ Vec<T, NV> load_vec(const T* p) {
  Vec<T, NV> v;
  v.raw = *reinterpret_cast<const decltype(v.raw)*>(p);
  return v;
}
template <typename T, int NV>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, NV>& v) {
  *reinterpret_cast<decltype(Vec<T, NV>::raw)*>(p) = v.raw;
}

// A chunk of the half layout is two vectors of NV elements, rot_dim / 2 apart: NV pairs. A chunk
// of the interleaved layout is one vector, NV / 2 pairs (NV = 1: two single elements, one pair).
// Past rot_dim a chunk is one vector to copy.
template <int NV, bool HALF>
struct Chunk {
  static constexpr int kPairs = HALF ? NV : (NV > 1 ? NV / 2 : 1);
  static constexpr bool kTwo = HALF || NV == 1;  // two vectors
};
template <typename T, int NV, bool HALF>
__global__ void __launch_bounds__(kMaxThreads)
    rotary_kernel(const __grid_constant__ RotaryParams p) {
  constexpr int P = Chunk<NV, HALF>::kPairs;
  constexpr bool kTwo = Chunk<NV, HALF>::kTwo;
  const int per_block = blockDim.x / p.lanes;
  const int local = threadIdx.x / p.lanes;
  const int lane = threadIdx.x - local * p.lanes;
  const int64_t slot = static_cast<int64_t>(blockIdx.x) * per_block + local;
  grid_dep_wait();
  grid_dep_launch();
  if (local < per_block && slot < static_cast<int64_t>(p.tokens) * p.head_slots) {
    const int token = static_cast<int>(slot / p.head_slots);
    const int first = static_cast<int>(slot - static_cast<int64_t>(token) * p.head_slots);
    const bool turned = lane < p.rot_lanes;
    // element offsets of the chunk's vectors
    const int e0 = turned ? (HALF ? lane * P : lane * 2 * P)
                          : p.rot_dim + (lane - p.rot_lanes) * NV;
    const int e1 = HALF ? e0 + p.rot_dim / 2 : e0 + 1;
    float c[P], s[P];
    if (turned) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const int pair = lane * P + i;
        const int axis = (pair >= p.axis_end[0]) + (pair >= p.axis_end[1]);
        const int64_t pos = __ldg(p.pos + static_cast<int64_t>(token) * p.axes + axis);
        const uint64_t phase = static_cast<uint64_t>(pos) * p.turn[pair];
        const float half_turns = static_cast<float>(static_cast<int32_t>(phase >> 32)) * 0x1p-31f;
        // 16-bit outputs: the hardware's sine and cosine, 2^-21 off at most on [-pi, pi]
        if constexpr (sizeof(T) == 2) __sincosf(half_turns * 3.14159265358979f, &s[i], &c[i]);
        else sincospif(half_turns, &s[i], &c[i]);
        c[i] *= p.amplitude;
        s[i] *= p.amplitude * p.sign;
      }
    }
    const int step = p.head_slots;
    constexpr int U = kTwo ? kVectors / 2 : kVectors;  // heads whose loads are in flight
#pragma unroll 1
    for (int h0 = first; h0 < p.heads; h0 += U * step) {
      Vec<T, NV> x[U], y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * step;
        if (h >= p.heads) continue;
        const int w = h >= p.q_heads;
        const T* src = static_cast<const T*>(p.in[w]) + token * p.in_token[w] +
                       static_cast<int64_t>(w ? h - p.q_heads : h) * p.in_head[w];
        if (turned || p.copy_tail[w]) x[u] = load_vec<T, NV>(src + e0);
        if (kTwo && turned) y[u] = load_vec<T, NV>(src + e1);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * step;
        if (h >= p.heads) continue;
        const int w = h >= p.q_heads;
        T* dst = static_cast<T*>(p.out[w]) + token * p.out_token[w] +
                 static_cast<int64_t>(w ? h - p.q_heads : h) * p.out_head[w];
        if (!turned) {
          if (p.copy_tail[w]) store_vec<T, NV>(dst + e0, x[u]);
          continue;
        }
#pragma unroll
        for (int i = 0; i < P; ++i) {
          T& ea = kTwo ? x[u].e[i] : x[u].e[(2 * i) % NV];
          T& eb = kTwo ? y[u].e[i] : x[u].e[(2 * i + 1) % NV];
          const float a = to_f(ea), b = to_f(eb);
          from_f(a * c[i] - b * s[i], ea);
          from_f(a * s[i] + b * c[i], eb);
        }
        store_vec<T, NV>(dst + e0, x[u]);
        if (kTwo) store_vec<T, NV>(dst + e1, y[u]);
      }
    }
  }
}

template <typename T, int NV>
cudaError_t launch_nv(RotaryParams& p, int num_sms, cudaStream_t s) {
  p.rot_lanes = p.rot_dim / 2 / (p.half ? Chunk<NV, true>::kPairs : Chunk<NV, false>::kPairs);
  p.lanes = p.rot_lanes + (p.head_dim - p.rot_dim) / NV;
  // Heads a thread walks over: threads for 12 blocks on every SM come first, but 3 heads do while
  // there are 4 blocks. In us, with threads for 4 / 8 / 12 / 16 blocks: 4000 tokens of 40 heads
  // of 128 bf16 25 / 22 / 21 / 22; 24960 of 20 heads of 64 28 / 28 / 25 / 25; 1560 of them 3.6 (3
  // heads) / 5.0 / 5.0 / 5.0 (1 head). More than 20 heads: 40001 tokens of 40 heads 163, with 20 155,
  // with 8 164, with 1 353.
  const int64_t all = static_cast<int64_t>(p.tokens) * p.heads * p.lanes;
  const int64_t fill = static_cast<int64_t>(num_sms) * 4 * kThreads;
  const int64_t per = std::min<int64_t>(
      std::max<int64_t>({1, all / (3 * fill), std::min<int64_t>(3, all / fill)}), kHeadsPerThread);
  p.head_slots = (p.heads + static_cast<int>(per) - 1) / static_cast<int>(per);
  const int threads = p.lanes > kThreads ? kMaxThreads : kThreads;
  const int per_block = threads / p.lanes;
  const int64_t blocks = (static_cast<int64_t>(p.tokens) * p.head_slots + per_block - 1) / per_block;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks));
  return p.half ? launch_pdl(rotary_kernel<T, NV, true>, grid, dim3(threads), 0, s, p)
                : launch_pdl(rotary_kernel<T, NV, false>, grid, dim3(threads), 0, s, p);
}

// The widest access (16, 8 or 4 bytes, or one element) that divides the pairs and the tail and
// that every address of both tensors is a multiple of.
template <typename T>
cudaError_t launch_type(RotaryParams& p, int num_sms, cudaStream_t s) {
  uint64_t bits = 0;  // the or of all addresses and strides, in elements
  for (int w = 0; w < 2; ++w) {
    if (w == 1 && p.heads == p.q_heads) continue;
    bits |= reinterpret_cast<uintptr_t>(p.in[w]) / sizeof(T);
    bits |= reinterpret_cast<uintptr_t>(p.out[w]) / sizeof(T);
    bits |= static_cast<uint64_t>(p.in_token[w]) | static_cast<uint64_t>(p.in_head[w]) |
            static_cast<uint64_t>(p.out_token[w]) | static_cast<uint64_t>(p.out_head[w]);
  }
  bits |= static_cast<uint64_t>(p.half ? p.rot_dim / 2 : p.rot_dim) | static_cast<uint64_t>(p.head_dim - p.rot_dim);
  constexpr int kWide = 16 / sizeof(T);
  if (bits % kWide == 0) return launch_nv<T, kWide>(p, num_sms, s);
  if (kWide > 4 && bits % 4 == 0) return launch_nv<T, 4>(p, num_sms, s);
  if (bits % 2 == 0) return launch_nv<T, 2>(p, num_sms, s);
  return launch_nv<T, 1>(p, num_sms, s);
}

bool valid_rotary(const fd_rotary_config* c) {
  if (c == nullptr || c->head_dim < 2 || c->head_dim > 256 || c->rot_dim < 2 ||
      c->rot_dim > c->head_dim || c->rot_dim % 2 || c->axes < 1 || c->axes > 3)
    return false;
  if (c->layout != FD_ROTARY_INTERLEAVED && c->layout != FD_ROTARY_HALF) return false;
  if (c->scaling < FD_ROTARY_SCALE_NONE || c->scaling > FD_ROTARY_SCALE_BLEND) return false;
  int sum = 0;
  for (int a = 0; a < c->axes; ++a) {
    if (c->axis_dims[a] < 2 || c->axis_dims[a] > c->rot_dim || c->axis_dims[a] % 2) return false;
    sum += c->axis_dims[a];
  }
  if (sum != c->rot_dim || !std::isfinite(c->base) || !(c->base > 0.f) ||
      !std::isfinite(c->amplitude))
    return false;
  if (c->scaling != FD_ROTARY_SCALE_NONE && (!std::isfinite(c->factor) || !(c->factor > 0.f)))
    return false;
  if (c->scaling == FD_ROTARY_SCALE_BLEND &&
      (c->trained_len < 1 || !std::isfinite(c->fast_turns) || !std::isfinite(c->slow_turns) ||
       !(c->fast_turns > c->slow_turns)))
    return false;
  return true;
}

}  // namespace
}  // namespace fd

extern "C" {

fd_status fd_rotary_create(const fd_rotary_config* cfg, fd_rotary* out) {
  if (out == nullptr) return FD_ERR_INVALID_ARG;
  *out = nullptr;
  if (!fd::valid_rotary(cfg)) return FD_ERR_CONFIG;
  fd_rotary plan = new (std::nothrow) fd_rotary_s();
  if (plan == nullptr) return FD_ERR_OOM;
  plan->cfg = *cfg;
  constexpr double kTwoPi = 6.283185307179586476925;
  int pair = 0;
  for (int a = 0; a < cfg->axes; ++a) {
    const int d = cfg->axis_dims[a];
    double base = cfg->base;
    if (cfg->scaling == FD_ROTARY_SCALE_BASE && d > 2)
      base *= std::pow(static_cast<double>(cfg->factor), static_cast<double>(d) / (d - 2));
    for (int i = 0; i < d / 2; ++i, ++pair) {
      double f = std::pow(base, -2.0 * i / d);
      if (cfg->scaling == FD_ROTARY_SCALE_LINEAR) {
        f /= cfg->factor;
      } else if (cfg->scaling == FD_ROTARY_SCALE_BLEND) {
        const double n = cfg->trained_len * f / kTwoPi;
        double g = (n - cfg->slow_turns) / (static_cast<double>(cfg->fast_turns) - cfg->slow_turns);
        g = g < 0 ? 0 : (g > 1 ? 1 : g);
        f = g * f + (1 - g) * f / cfg->factor;
      }
      // turns per position modulo one, in 2^-64 turns (2^64 itself is a whole turn: 0)
      double turns = f / kTwoPi;
      turns -= std::floor(turns);
      const double scaled = std::nearbyint(turns * 0x1p64);
      plan->turn[pair] = scaled >= 0x1p64 ? 0 : static_cast<uint64_t>(scaled);
    }
  }
  *out = plan;
  return FD_OK;
}

fd_status fd_rotary_destroy(fd_rotary plan) {
  if (plan == nullptr) return FD_ERR_INVALID_ARG;
  delete plan;
  return FD_OK;
}

fd_status fd_op_rotary(fd_rotary plan, int backward, int dtype, int tokens,
                       const int32_t* positions, int q_heads, const void* q,
                       int64_t q_token_stride, int64_t q_head_stride, void* q_out,
                       int64_t q_out_token_stride, int64_t q_out_head_stride, int k_heads,
                       const void* k, int64_t k_token_stride, int64_t k_head_stride, void* k_out,
                       int64_t k_out_token_stride, int64_t k_out_head_stride, void* stream) {
  if (plan == nullptr || (backward != 0 && backward != 1) || tokens < 0 || q_heads < 0 ||
      k_heads < 0 || q_heads > 65536 || k_heads > 65536)
    return FD_ERR_INVALID_ARG;
  if (dtype != FD_DTYPE_F32 && dtype != FD_DTYPE_BF16 && dtype != FD_DTYPE_F16)
    return FD_ERR_INVALID_ARG;
  const uintptr_t esz = dtype == FD_DTYPE_F32 ? 4 : 2;
  auto bad = [&](const void* x) {
    return x == nullptr || reinterpret_cast<uintptr_t>(x) % esz != 0;
  };
  if (tokens == 0 || q_heads + k_heads == 0) return FD_OK;
  if (positions == nullptr || reinterpret_cast<uintptr_t>(positions) % 4) return FD_ERR_INVALID_ARG;
  if (q_heads > 0 && (bad(q) || bad(q_out))) return FD_ERR_INVALID_ARG;
  if (k_heads > 0 && (bad(k) || bad(k_out))) return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  const fd_rotary_config& c = plan->cfg;
  fd::RotaryParams p{};
  for (int i = 0; i < c.rot_dim / 2; ++i) p.turn[i] = plan->turn[i];
  p.axis_end[0] = c.axis_dims[0] / 2;
  p.axis_end[1] = c.axes > 1 ? p.axis_end[0] + c.axis_dims[1] / 2 : c.rot_dim / 2;
  p.axes = c.axes;
  p.head_dim = c.head_dim;
  p.rot_dim = c.rot_dim;
  p.half = c.layout == FD_ROTARY_HALF;
  p.sign = backward ? -1.f : 1.f;
  p.amplitude = c.amplitude;
  p.tokens = tokens;
  p.pos = positions;
  p.q_heads = q_heads;
  p.heads = q_heads + k_heads;
  p.in[0] = q; p.out[0] = q_out;
  p.in_token[0] = q_token_stride; p.in_head[0] = q_head_stride;
  p.out_token[0] = q_out_token_stride; p.out_head[0] = q_out_head_stride;
  p.in[1] = k; p.out[1] = k_out;
  p.in_token[1] = k_token_stride; p.in_head[1] = k_head_stride;
  p.out_token[1] = k_out_token_stride; p.out_head[1] = k_out_head_stride;
  for (int w = 0; w < 2; ++w)
    p.copy_tail[w] = p.in[w] != p.out[w] || p.in_token[w] != p.out_token[w] ||
                     p.in_head[w] != p.out_head[w];
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int sms = fd::num_sms();
  cudaError_t e = dtype == FD_DTYPE_F32    ? fd::launch_type<float>(p, sms, s)
                  : dtype == FD_DTYPE_BF16 ? fd::launch_type<__nv_bfloat16>(p, sms, s)
                                           : fd::launch_type<__half>(p, sms, s);
  return e == cudaSuccess ? FD_OK : FD_ERR_CUDA;
}

}  // extern "C"
