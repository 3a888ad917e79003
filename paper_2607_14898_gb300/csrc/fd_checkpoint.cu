// Activations kept in 8 bits for the backward pass (fd_op_checkpoint_save / _load): the format is
// in fd_rows.cuh.
//
// Bound by memory: every element is read and written once, 1 + 1/32 byte of it in 8 bits.
#include <algorithm>

#include "fd_once.h"
#include "fd_rows.cuh"
#include "flashdec_ops.h"

namespace fd {
namespace {

constexpr int kThreads = 256;
constexpr int kPerThread = 4;                   // groups of eight elements in flight a thread
constexpr int kUnits = kThreads * kPerThread;   // of a block

// A block has `rows_of` rows by `units` groups of eight elements (whole blocks of 32, so that the
// four lanes of one are neighbours), at most kUnits together.
struct Plane {
  int rows, width;
  int units, rows_of;
  int padded;  // groups a row, those past its end too
};
Plane plane(int rows, int width) {
  Plane p{rows, width, 0, 0, (width + kKeptBlock - 1) / kKeptBlock * 4};
  p.units = std::min(p.padded, kUnits);
  p.rows_of = kUnits / p.units;
  return p;
}
dim3 grid_of(const Plane& p) {
  return dim3((p.rows + p.rows_of - 1) / p.rows_of, (p.padded + p.units - 1) / p.units);
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
    save_kernel(Plane p, const T* x, int64_t stride, int8_t* codes, uint8_t* exps) {
  grid_dep_wait();
  grid_dep_launch();
  Raw8<T> raw[kPerThread];
  int64_t row[kPerThread];
  int unit[kPerThread];
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    const int l = threadIdx.x + j * kThreads, r = l / p.units;
    row[j] = static_cast<int64_t>(blockIdx.x) * p.rows_of + r;
    unit[j] = static_cast<int>(blockIdx.y) * p.units + l - r * p.units;
    raw[j] = Raw8<T>{};
    if (r >= p.rows_of || row[j] >= p.rows || unit[j] >= p.padded) unit[j] = -1;
    if (unit[j] >= 0 && unit[j] < p.width / 8) raw[j] = load_raw(x + row[j] * stride + unit[j] * 8);
  }
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    float v[8];
    widen(raw[j], v);
    const uint32_t byte = kept_exponent(block_top(v));
    if (unit[j] < 0) continue;
    if (unit[j] < p.width / 8)
      *reinterpret_cast<uint2*>(codes + row[j] * p.width + unit[j] * 8) = kept_codes(v, byte);
    if (unit[j] % 4 == 0) exps[row[j] * (p.padded / 4) + unit[j] / 4] = static_cast<uint8_t>(byte);
  }
}

// fp16 has no room for what rounds up past its largest number: it stays there
template <typename T>
__device__ __forceinline__ void into_range(float (&x)[8]) {
  if constexpr (std::is_same<T, __half>::value) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (fabsf(x[i]) <= 65536.f) x[i] = fminf(fmaxf(x[i], -65504.f), 65504.f);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
    load_kernel(Plane p, const int8_t* codes, const uint8_t* exps, T* x, int64_t stride) {
  grid_dep_wait();
  grid_dep_launch();
  uint2 raw[kPerThread];
  uint32_t byte[kPerThread];
  T* to[kPerThread];
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    const int l = threadIdx.x + j * kThreads, r = l / p.units;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * p.rows_of + r;
    const int unit = static_cast<int>(blockIdx.y) * p.units + l - r * p.units;
    to[j] = nullptr;
    if (r < p.rows_of && row < p.rows && unit < p.width / 8) {
      raw[j] = *reinterpret_cast<const uint2*>(codes + row * p.width + unit * 8);
      byte[j] = exps[row * (p.padded / 4) + unit / 4];
      to[j] = x + row * stride + unit * 8;
    }
  }
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    if (to[j] == nullptr) continue;
    float v[8];
    kept_values(raw[j], byte[j], v);
    into_range<T>(v);
    store8(to[j], v);
  }
}

// Transposed: x[column][row]. A block turns 256 rows by 64 columns over in shared memory: codes are
// read by whole sectors of a row, and a column's values leave as aligned 16-byte stores. Columns begin
// at any address (rows may be odd), so a vector may reach over the tile's end: it is the tile's that has
// its first element, which has the next rows too for that. Only a column's own two ends are stored by
// elements. (Tiles of 128 x 128 that stored their ends by elements took 74 us for 16001 x 4096.)
constexpr int kTileRows = 256, kTileCols = 64;

template <typename T>
__global__ void __launch_bounds__(kThreads)
    load_transposed_kernel(int rows, int width, const int8_t* codes, const uint8_t* exps, T* x,
                           int64_t stride) {
  constexpr int kVec = 16 / sizeof(T);
  constexpr int kAll = kTileRows + 8;             // with the next tile's first rows
  constexpr int kPitch = kAll + 4 / sizeof(T);    // an odd number of 32-bit words
  extern __shared__ __align__(16) uint8_t smem[];
  T* tile = reinterpret_cast<T*>(smem);  // [column][row]
  grid_dep_wait();
  grid_dep_launch();
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kTileRows;
  const int col0 = blockIdx.y * kTileCols;
  const int blocks = (width + kKeptBlock - 1) / kKeptBlock;
  // lanes: 4 groups of eight columns (a sector) by 8 rows
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r_in = lane >> 2, u_in = lane & 3;
  constexpr int kRuns = kAll / 8 * (kTileCols / 32);  // 33 runs of 8 rows by 2 of 32 columns
  constexpr int kSteps = (kRuns + kThreads / 32 - 1) / (kThreads / 32);
  uint2 raw[kSteps];
  uint32_t byte[kSteps];
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const int step = j * (kThreads / 32) + warp;
    const int64_t row = row0 + (step >> 1) * 8 + r_in;
    const int col = col0 + (step & 1) * 32 + u_in * 8;
    raw[j] = make_uint2(0u, 0u);
    byte[j] = 1u;
    if (step < kRuns && row < rows && col < width) {
      raw[j] = __ldg(reinterpret_cast<const uint2*>(codes + row * width + col));
      byte[j] = __ldg(exps + row * blocks + col / kKeptBlock);
    }
  }
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const int step = j * (kThreads / 32) + warp;
    if (step >= kRuns) break;
    const int r = (step >> 1) * 8 + r_in, c = (step & 1) * 32 + u_in * 8;
    float v[8];
    kept_values(raw[j], byte[j], v);
    into_range<T>(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) tile[(c + i) * kPitch + r] = T(v[i]);
  }
  __syncthreads();
  // elements there are from row0 on, with those of the next tile that a vector may need
  const int count = static_cast<int>(min(static_cast<int64_t>(kAll), rows - row0));
  const int mine = min(kTileRows, count);
  const bool starts = blockIdx.x == 0;
  const int cols = min(kTileCols, width - col0);
  constexpr int kChunks = kTileRows / kVec;
  // lanes are neighbouring vectors of a column
  for (int it = threadIdx.x; it < cols * kChunks; it += kThreads) {
    const int c = it / kChunks, chunk = it % kChunks;
    T* column = x + static_cast<int64_t>(col0 + c) * stride + row0;
    const int lead =  // elements up to the first aligned address
        static_cast<int>((0 - reinterpret_cast<uintptr_t>(column) / sizeof(T)) % kVec);
    const int first = lead + chunk * kVec;
    const T* from = tile + c * kPitch;
    if (starts && chunk == 0)
      for (int e = 0; e < min(lead, count); ++e) column[e] = from[e];
    if (first >= mine) continue;
    if (first + kVec <= count) {
      uint4 v;
      if constexpr (sizeof(T) == 2) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(from) + (first >> 1);
        if (first & 1) {
          v.x = __funnelshift_r(w[0], w[1], 16);
          v.y = __funnelshift_r(w[1], w[2], 16);
          v.z = __funnelshift_r(w[2], w[3], 16);
          v.w = __funnelshift_r(w[3], w[4], 16);
        } else {
          v = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(from) + first;
        v = make_uint4(w[0], w[1], w[2], w[3]);
      }
      *reinterpret_cast<uint4*>(column + first) = v;
    } else {  // the column's end
      for (int e = first; e < count; ++e) column[e] = from[e];
    }
  }
}

template <typename T>
cudaError_t save_type(int rows, int width, const void* x, int64_t stride, int8_t* codes,
                      uint8_t* exps, cudaStream_t s) {
  const Plane p = plane(rows, width);
  return launch_pdl(save_kernel<T>, grid_of(p), dim3(kThreads), 0, s, p, static_cast<const T*>(x),
                    stride, codes, exps);
}

template <typename T>
cudaError_t load_type(bool transposed, int rows, int width, const int8_t* codes,
                      const uint8_t* exps, void* x, int64_t stride, cudaStream_t s) {
  if (!transposed) {
    const Plane p = plane(rows, width);
    return launch_pdl(load_kernel<T>, grid_of(p), dim3(kThreads), 0, s, p, codes, exps,
                      static_cast<T*>(x), stride);
  }
  constexpr size_t kSmem = kTileCols * (kTileRows + 8 + 4 / sizeof(T)) * sizeof(T);
  static OncePerDevice once;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess)
    e = once.run(dev, [&] {
      return cudaFuncSetAttribute(load_transposed_kernel<T>,
                                  cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    });
  if (e != cudaSuccess) return e;
  const dim3 grid((rows + kTileRows - 1) / kTileRows, (width + kTileCols - 1) / kTileCols);
  return launch_pdl(load_transposed_kernel<T>, grid, dim3(kThreads), kSmem, s, rows, width, codes,
                    exps, static_cast<T*>(x), stride);
}

bool ok_ptr(const void* p, uintptr_t align) {
  return p != nullptr && reinterpret_cast<uintptr_t>(p) % align == 0;
}
bool valid(int dtype, int rows, int width) {
  return (dtype == FD_DTYPE_F32 || dtype == FD_DTYPE_BF16 || dtype == FD_DTYPE_F16) && rows >= 0 &&
         width >= 8 && width % 8 == 0 && width <= 1 << 20;
}

}  // namespace
}  // namespace fd

extern "C" {

fd_status fd_op_checkpoint_save(int dtype, int rows, int width, const void* x, int64_t x_stride,
                                int8_t* codes, uint8_t* exps, void* stream) {
  if (!fd::valid(dtype, rows, width)) return FD_ERR_INVALID_ARG;
  if (rows == 0) return FD_OK;
  if (!fd::ok_ptr(x, 16) || !fd::ok_ptr(codes, 8) || exps == nullptr ||
      x_stride % 8 != 0)
    return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e =
      dtype == FD_DTYPE_F32    ? fd::save_type<float>(rows, width, x, x_stride, codes, exps, s)
      : dtype == FD_DTYPE_BF16 ? fd::save_type<__nv_bfloat16>(rows, width, x, x_stride, codes, exps, s)
                               : fd::save_type<__half>(rows, width, x, x_stride, codes, exps, s);
  return e == cudaSuccess ? FD_OK : FD_ERR_CUDA;
}

fd_status fd_op_checkpoint_load(int dtype, int transposed, int rows, int width,
                                const int8_t* codes, const uint8_t* exps, void* x,
                                int64_t x_stride, void* stream) {
  if (!fd::valid(dtype, rows, width) || (transposed != 0 && transposed != 1))
    return FD_ERR_INVALID_ARG;
  if (rows == 0) return FD_OK;
  const uintptr_t esz = dtype == FD_DTYPE_F32 ? 4 : 2;
  if (!fd::ok_ptr(codes, 8) || exps == nullptr) return FD_ERR_INVALID_ARG;
  if (transposed ? !fd::ok_ptr(x, esz) || x_stride < rows
                 : !fd::ok_ptr(x, 16) || x_stride % 8 != 0 || (rows > 1 && x_stride < width))
    return FD_ERR_INVALID_ARG;
  const fd_status st = fd::check_device();
  if (st != FD_OK) return st;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool t = transposed != 0;
  const cudaError_t e =
      dtype == FD_DTYPE_F32 ? fd::load_type<float>(t, rows, width, codes, exps, x, x_stride, s)
      : dtype == FD_DTYPE_BF16
          ? fd::load_type<__nv_bfloat16>(t, rows, width, codes, exps, x, x_stride, s)
          : fd::load_type<__half>(t, rows, width, codes, exps, x, x_stride, s);
  return e == cudaSuccess ? FD_OK : FD_ERR_CUDA;
}

}  // extern "C"
