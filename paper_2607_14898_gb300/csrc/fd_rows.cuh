// Rows of activations for the kernels that work on them element by element (fd_block.cu,
// fd_checkpoint.cu): eight neighbours at once, as floats, and their 8-bit form.
#pragma once
#include "fd_internal.h"
#include "fd_ptx.cuh"

namespace fd {

// eight elements of a row as they lie in memory
template <typename T>
struct Raw8 {
  uint4 a;
};
template <>
struct Raw8<float> {
  uint4 a, b;
};

template <typename T>
__device__ __forceinline__ Raw8<T> load_raw(const T* p) {
  Raw8<T> r;
  r.a = *reinterpret_cast<const uint4*>(p);
  if constexpr (sizeof(T) == 4) r.b = *reinterpret_cast<const uint4*>(p + 4);
  return r;
}
__device__ __forceinline__ void widen(const Raw8<float>& r, float (&x)[8]) {
  x[0] = __uint_as_float(r.a.x), x[1] = __uint_as_float(r.a.y);
  x[2] = __uint_as_float(r.a.z), x[3] = __uint_as_float(r.a.w);
  x[4] = __uint_as_float(r.b.x), x[5] = __uint_as_float(r.b.y);
  x[6] = __uint_as_float(r.b.z), x[7] = __uint_as_float(r.b.w);
}
__device__ __forceinline__ void widen(const Raw8<__nv_bfloat16>& r, float (&x)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen(const Raw8<__half>& r, float (&x)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  widen(load_raw(p), x);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16) {
  return pack_bf16x2(lo, hi);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// rounded to nearest even
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(x[0], x[1], T()), pack2(x[2], x[3], T()),
                                              pack2(x[4], x[5], T()), pack2(x[6], x[7], T()));
  }
}

// ---- the 8-bit form: blocks of 32 neighbours of a row share a power of two, 2^E; E the smallest
// (-126 at least) that lets the largest magnitude fit into 127 steps, stored as E + 127, 255 for a
// block that holds an infinity or a NaN. The step being a power of two, codes are the same in
// every arithmetic and what they stand for is exact in fp32 and bf16.
constexpr int kKeptBlock = 32;

// the byte for the largest magnitude's bits
__device__ __forceinline__ uint32_t kept_exponent(uint32_t top_bits) {
  // top = 1.m 2^e is 64 (1.m) steps of 2^(e - 6): too many for 127 where 1.m > 127/64
  const uint32_t e = top_bits >> 23;
  if (e == 255u) return 255u;
  const int byte = static_cast<int>(e) - 6 + ((top_bits & 0x7fffffu) > 0x7e0000u);
  return static_cast<uint32_t>(byte < 1 ? 1 : byte);
}
// the codes of eight elements of the block, low byte first
__device__ __forceinline__ uint2 kept_codes(const float (&x)[8], uint32_t byte) {
  if (byte == 255u) return make_uint2(0u, 0u);
  const float per_step = __uint_as_float((254u - byte) << 23);  // 2^-E
  int c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    c[i] = __float2int_rn(x[i] * per_step);
    // 64 steps of 2^122 are 2^128: the largest floats stay finite
    if (byte >= 249u) c[i] = min(63, max(-63, c[i]));
  }
  auto four = [&](int i) {
    return __byte_perm(__byte_perm(c[i], c[i + 1], 0x0040), __byte_perm(c[i + 2], c[i + 3], 0x0040),
                       0x5410);
  };
  return make_uint2(four(0), four(4));
}
// what eight codes stand for (a byte of 255 makes the step infinite and the block NaN: 0 times it)
__device__ __forceinline__ void kept_values(uint2 codes, uint32_t byte, float (&x)[8]) {
  const float step = __uint_as_float(byte << 23);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = static_cast<float>(static_cast<int8_t>(codes.x >> (8 * i))) * step;
    x[4 + i] = static_cast<float>(static_cast<int8_t>(codes.y >> (8 * i))) * step;
  }
}
// the largest magnitude's bits over the four neighbouring lanes that hold a block (NaN above all)
__device__ __forceinline__ uint32_t block_top(const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  return max(top, __shfl_xor_sync(0xffffffffu, top, 2));
}

}  // namespace fd
