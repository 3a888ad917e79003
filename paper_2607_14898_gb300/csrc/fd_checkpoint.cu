// Activations kept in 8 bits for the backward pass (fd_op_checkpoint_save / _load): the format is
// in fd_rows.cuh.
//
// Bound by memory: every element is read and written once, 1 + 1/32 byte of it in 8 bits. 6240 x 4096 of
// bf16 (not in L2) are saved in 14.8 us, 5.2 TB/s, 78 % of a plain copy's rate; divisions for a thread's places and
// one conversion an element cost 1 us more.
#include <algorithm>

#include "fd_once.h"
#include "fd_rows.cuh"
#include "flashdec_ops.h"

namespace fd {
namespace {

constexpr int kThreads = 256;
constexpr int kPerThread = 2;                   // groups of eight elements in flight a thread (4: 15.8 us, 1: 17.2)
constexpr int kUnits = kThreads * kPerThread;   // of a block

// A block has `rows_of` rows by `units` groups of eight elements (whole blocks of 32, so that the
// four lanes of one are neighbours), at most kUnits together.
struct Plane {
  int rows, width;
  int units, rows_of;
  int padded;  // groups a row, those past its end too
  int rows_on, units_on;  // from a thread's group to its next: so many rows and groups
};
// where a thread's group is in its block's plane (without a division for each)
struct Place {
  int row, unit;
  __device__ Place(const Plane& p) : row(threadIdx.x / p.units), unit(threadIdx.x - row * p.units) {}
  __device__ void next(const Plane& p) {
    row += p.rows_on;
    unit += p.units_on;
    if (unit >= p.units) {
      unit -= p.units;
      ++row;
    }
  }
};
Plane plane(int rows, int width) {
  Plane p{rows, width, 0, 0, (width + kKeptBlock - 1) / kKeptBlock * 4, 0, 0};
  p.units = std::min(p.padded, kUnits);
  p.rows_of = kUnits / p.units;
  p.rows_on = kThreads / p.units;
  p.units_on = kThreads % p.units;
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
  const int width8 = p.width / 8, unit0 = blockIdx.y * p.units;
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows_of;
  Place at(p);
#pragma unroll
  for (int j = 0; j < kPerThread; ++j, at.next(p)) {
    row[j] = row0 + at.row;
    unit[j] = unit0 + at.unit;
    raw[j] = Raw8<T>{};
    if (at.row >= p.rows_of || row[j] >= p.rows || unit[j] >= p.padded) unit[j] = -1;
    if (unit[j] >= 0 && unit[j] < width8) raw[j] = load_raw(x + row[j] * stride + unit[j] * 8);
  }
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    float v[8];
    widen(raw[j], v);
    const uint32_t byte = kept_exponent(block_top(raw[j]));
    const uint2 eight = kept_codes(v, byte);
    if (unit[j] < 0) continue;
    if (unit[j] < width8) *reinterpret_cast<uint2*>(codes + row[j] * p.width + unit[j] * 8) = eight;
    if (unit[j] % 4 == 0) exps[row[j] * (p.padded / 4) + unit[j] / 4] = static_cast<uint8_t>(byte);
  }
}

// fp16 has no room for what rounds up past its largest number, 64 steps of 2^10: it stays there. (Steps
// that large are rare: every other block is spared the comparisons.)
constexpr uint32_t kWideStep = 127u + 10u;  // the byte of 2^10
__device__ __forceinline__ float into_fp16(float x) {
  return fabsf(x) <= 65536.f ? fminf(fmaxf(x, -65504.f), 65504.f) : x;
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
    load_kernel(Plane p, const int8_t* codes, const uint8_t* exps, T* x, int64_t stride) {
  grid_dep_wait();
  grid_dep_launch();
  uint2 raw[kPerThread];
  uint32_t byte[kPerThread];
  T* to[kPerThread];
  Place at(p);
#pragma unroll
  for (int j = 0; j < kPerThread; ++j, at.next(p)) {
    const int64_t row = static_cast<int64_t>(blockIdx.x) * p.rows_of + at.row;
    const int unit = static_cast<int>(blockIdx.y) * p.units + at.unit;
    to[j] = nullptr;
    if (at.row < p.rows_of && row < p.rows && unit < p.width / 8) {
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
    if constexpr (std::is_same<T, __half>::value) {
      const uint32_t together = __activemask();
      if (__any_sync(together, byte[j] >= kWideStep)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = into_fp16(v[i]);
      }
    }
    store8(to[j], v);
  }
}

// Transposed: x[column][row]. A block turns 64 rows by 64 columns over in shared memory: codes are read by
// whole sectors of a row, two rows a thread (whose 16-bit values go into shared memory as one word), and a
// column's values leave as aligned 16-byte stores. Columns begin at any address (rows may be odd), so a
// vector may reach over the tile's end: it is the tile's that has its first element, which has the next
// rows too for that. Only a column's own two ends are stored by elements.
// 16001 x 4096 into fp16: 46 us, 4.3 TB/s, bound by the L1's way to memory (82 % busy: a store takes a cycle for
// every sector). With 256 threads 49 us, tiles of 128 rows 53 to 54, stores by whole sectors with the
// reads of shared memory free of conflicts 48.
constexpr int kTileRows = 64, kTileCols = 64, kTurners = 128;  // turners: threads of a block
static_assert(kTileCols == 64 && kTurners % 64 == 0, "two warps side by side have a tile's columns");

template <typename T>
__global__ void __launch_bounds__(kTurners)
    load_transposed_kernel(int rows, int width, const int8_t* codes, const uint8_t* exps, T* x,
                           int64_t stride) {
  constexpr int kVec = 16 / sizeof(T);
  constexpr int kAll = kTileRows + 16;            // with the next tile's first rows
  constexpr int kPitch = kAll + 4 / sizeof(T);    // an odd number of 32-bit words
  extern __shared__ __align__(16) uint8_t smem[];
  T* tile = reinterpret_cast<T*>(smem);  // [column][row]
  grid_dep_wait();
  grid_dep_launch();
  const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kTileRows;
  const int col0 = blockIdx.y * kTileCols;
  const int blocks = (width + kKeptBlock - 1) / kKeptBlock;
  // lanes: 4 groups of eight columns (a sector) by 8 pairs of rows; warps: runs of 16 rows by 32 columns
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int u_in = lane & 3;
  constexpr int kRuns = kAll / 16 * (kTileCols / 32);
  constexpr int kSteps = (kRuns + kTurners / 32 - 1) / (kTurners / 32);
  const int col = col0 + (warp & 1) * 32 + u_in * 8;  // (an even number of warps)
  const int64_t first_row = row0 + (warp >> 1) * 16 + (lane >> 2) * 2;
  const int8_t* from = codes + first_row * width + col;
  const uint8_t* exp_from = exps + first_row * blocks + col / kKeptBlock;
  constexpr int kRowStep = kTurners / 64 * 16;  // rows from a warp's run to its next
  uint2 raw[kSteps][2];
  uint32_t byte[kSteps][2];
#pragma unroll
  for (int j = 0; j < kSteps; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      raw[j][i] = make_uint2(0u, 0u);
      byte[j][i] = 1u;
      if (j * (kTurners / 32) + warp < kRuns && first_row + j * kRowStep + i < rows && col < width) {
        raw[j][i] = __ldg(reinterpret_cast<const uint2*>(from + static_cast<int64_t>(j * kRowStep + i) * width));
        byte[j][i] = __ldg(exp_from + static_cast<int64_t>(j * kRowStep + i) * blocks);
      }
    }
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    if (j * (kTurners / 32) + warp >= kRuns) break;
    const int r = (warp >> 1) * 16 + (lane >> 2) * 2 + j * kRowStep, c = (warp & 1) * 32 + u_in * 8;
    float v[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      kept_values(raw[j][i], byte[j][i], v[i]);
      if constexpr (std::is_same<T, __half>::value)
        if (__any_sync(0xffffffffu, byte[j][i] >= kWideStep)) {
#pragma unroll
          for (int k = 0; k < 8; ++k) v[i][k] = into_fp16(v[i][k]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      T* to = tile + (c + i) * kPitch + r;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint32_t*>(to) = pack2(v[0][i], v[1][i], T());
      } else {
        to[0] = v[0][i];
        to[1] = v[1][i];
      }
    }
  }
  __syncthreads();
  // elements there are from row0 on, with those of the next tile that a vector may need
  const int count = static_cast<int>(min(static_cast<int64_t>(kAll), rows - row0));
  const int mine = min(kTileRows, count);
  const bool starts = blockIdx.x == 0;
  const int cols = min(kTileCols, width - col0);
  constexpr int kChunks = kTileRows / kVec;
  constexpr int kColStep = kTurners / kChunks;
  // neighbouring threads have neighbouring vectors of a column
  const int chunk = threadIdx.x % kChunks;
  int c = threadIdx.x / kChunks;
  T* column = x + static_cast<int64_t>(col0 + c) * stride + row0;
  const T* in = tile + c * kPitch;
#pragma unroll 4
  for (; c < cols; c += kColStep, column += kColStep * stride, in += kColStep * kPitch) {
    const int lead =  // elements up to the first aligned address
        static_cast<int>((0u - static_cast<uint32_t>(reinterpret_cast<uintptr_t>(column)) / sizeof(T)) % kVec);
    const int first = lead + chunk * kVec;
    if (starts && chunk == 0)
      for (int e = 0; e < min(lead, count); ++e) column[e] = in[e];
    if (first + kVec <= count) {
      if (first >= mine) continue;
      uint4 v;
      if constexpr (sizeof(T) == 2) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(in) + (first >> 1);
        const uint32_t shift = (first & 1) * 16;
        const uint32_t a = w[0], b = w[1], d = w[2], e = w[3], f = w[4];
        v = make_uint4(__funnelshift_r(a, b, shift), __funnelshift_r(b, d, shift),
                       __funnelshift_r(d, e, shift), __funnelshift_r(e, f, shift));
      } else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(in) + first;
        v = make_uint4(w[0], w[1], w[2], w[3]);
      }
      *reinterpret_cast<uint4*>(column + first) = v;
    } else if (first < mine) {  // the column's end
      for (int e = first; e < count; ++e) column[e] = in[e];
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
  constexpr size_t kSmem = kTileCols * (kTileRows + 16 + 4 / sizeof(T)) * sizeof(T);
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
  return launch_pdl(load_transposed_kernel<T>, grid, dim3(kTurners), kSmem, s, rows, width, codes,
                    exps, static_cast<T*>(x), stride);
}

bool ok_ptr(const void* p, uintptr_t align) {
  return p != nullptr && reinterpret_cast<uintptr_t>(p) % align == 0;
}
bool valid(int dtype, int rows, int width) {
  return (dtype == FD_DTYPE_F32 || dtype == FD_DTYPE_BF16 || dtype == FD_DTYPE_F16) && rows >= 0 && rows <= 1 << 30 &&
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
