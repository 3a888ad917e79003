// Rows of activations for the kernels that work on them element by element (fd_block.cu,
// fd_checkpoint.cu): eight neighbours at once, as floats, and their 8-bit form.
#pragma once
#include <type_traits>

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

// as four pairs
struct Pairs {
  uint64_t v[4];
};
__device__ __forceinline__ Pairs pairs_of(const float (&x)[8]) {
  Pairs r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = pack_f32x2(x[2 * i], x[2 * i + 1]);
  return r;
}
template <typename T>
__device__ __forceinline__ Pairs widen2(const Raw8<T>& r) {
  float x[8];
  widen(r, x);
  return pairs_of(x);
}
template <typename T>
__device__ __forceinline__ Pairs load8_2(const T* p) {
  return widen2(load_raw(p));
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const Pairs& x) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 h = halves_of(x.v[i]);
    f[2 * i] = h.x;
    f[2 * i + 1] = h.y;
  }
  store8(p, f);
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
// The codes of eight elements of the block, low byte first; by a whole warp. x 2^-E + 1.5 2^23 is rounded to a
// whole number by the addition itself, ties to even, and its low byte is the code: no conversions, which
// run at a quarter of the additions' rate.
__device__ __forceinline__ uint2 kept_codes(const float (&x)[8], uint32_t byte) {
  const float per_step = __uint_as_float((254u - byte) << 23);  // 2^-E
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = __float_as_uint(fmaf(x[i], per_step, 12582912.f));
  auto four = [&](int i) {
    return __byte_perm(__byte_perm(c[i], c[i + 1], 0x0040), __byte_perm(c[i + 2], c[i + 3], 0x0040),
                       0x5410);
  };
  uint2 r = make_uint2(four(0), four(4));
  if (__any_sync(0xffffffffu, byte >= 249u)) {  // (rare, and not predicated)
    // 64 steps of 2^122 are 2^128: the largest floats stay finite
    if (byte >= 249u) {
      r.x = __vmins4(__vmaxs4(r.x, 0xc1c1c1c1u), 0x3f3f3f3fu);
      r.y = __vmins4(__vmaxs4(r.y, 0xc1c1c1c1u), 0x3f3f3f3fu);
    }
    if (byte == 255u) r = make_uint2(0u, 0u);
  }
  return r;
}
// What eight codes stand for: code + 128 goes into the last bits of 2^23, which is taken off again. (A
// byte of 255 makes the step infinite and the block NaN: 0 times it.)
__device__ __forceinline__ void kept_values(uint2 codes, uint32_t byte, float (&x)[8]) {
  const float step = __uint_as_float(byte << 23);
  const uint32_t w[2] = {codes.x ^ 0x80808080u, codes.y ^ 0x80808080u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    x[i] = (__uint_as_float(__byte_perm(w[i / 4], 0x4b000000u, 0x7650 + i % 4)) - 8388736.f) * step;
}
__device__ __forceinline__ Pairs kept_values2(uint2 codes, uint32_t byte) {
  const float step = __uint_as_float(byte << 23);
  const uint64_t step2 = pack_f32x2(step, step), base2 = pack_f32x2(-8388736.f, -8388736.f);
  const uint32_t w[2] = {codes.x ^ 0x80808080u, codes.y ^ 0x80808080u};
  Pairs r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r.v[i] = mul2(add2(pair_of(__byte_perm(w[i / 2], 0x4b000000u, 0x7650 + 2 * (i % 2)),
                               __byte_perm(w[i / 2], 0x4b000000u, 0x7651 + 2 * (i % 2))),
                       base2),
                  step2);
  return r;
}
// The largest magnitude's bits, as fp32's, over the four neighbouring lanes that hold a block (NaN above
// all); 16-bit elements are compared two by two as they lie in memory.
__device__ __forceinline__ uint32_t block_top(const Raw8<float>& r) {
  const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, w[i] & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  return max(top, __shfl_xor_sync(0xffffffffu, top, 2));
}
template <typename T>
__device__ __forceinline__ uint32_t block_top(const Raw8<T>& r) {
  const uint32_t m = 0x7fff7fffu;
  uint32_t top = __vmaxu2(__vmaxu2(r.a.x & m, r.a.y & m), __vmaxu2(r.a.z & m, r.a.w & m));
  top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
  top = max(top & 0xffffu, top >> 16);
  if constexpr (std::is_same<T, __half>::value)
    return __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(top))));
  else
    return top << 16;
}

}  // namespace fd
