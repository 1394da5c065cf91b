// Activations put away in 8 bits and taken back (format: checkpoint.h).  Both are one
// pass over memory and bound by it: 8192 x 14336 in bf16 put away and taken back in 131 us
// (712 MB, 5.4 TB/s), 8191 x 2048 taken back in 10.6 us (4.8 TB/s).
#include "checkpoint.h"

#include <algorithm>

namespace trimmoe {

namespace {

constexpr int kThreads = 256;

template <typename T>
struct alignas(16) Vec8 {
  T e[8];
};

// the largest of the four lanes of a quad
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, false));  // lane ^ 1
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, false));  // lane ^ 2
}

// Rows of whole 8-value pieces, 16-byte aligned: four lanes a block of 32, so that every
// access is a whole load or store (a lane past the row's end holds zeros).
template <typename T>
__global__ __launch_bounds__(kThreads) void k_pack_vec(const T* x, int c, long n_quads, int8_t* codes,
                                                       uint8_t* scale) {
  const int blocks = (c + kPackBlock - 1) / kPackBlock;
  const long step = (long)gridDim.x * (kThreads / 4);
  for (long b = (long)blockIdx.x * (kThreads / 4) + (threadIdx.x >> 2); b < n_quads; b += step) {
    const long row = b / blocks;
    const int col = (int)(b - row * blocks) * kPackBlock + 8 * (threadIdx.x & 3);
    const bool in = col < c;
    Vec8<T> v = {};
    if (in) v = *reinterpret_cast<const Vec8<T>*>(x + row * c + col);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, abs_bits(to_f32<T>(v.e[i])));
    const uint32_t s = pack_scale(quad_max(top));
    union {
      int8_t q[8];
      uint2 w;
    } o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.q[i] = s == 255 ? 0 : pack_code(to_f32<T>(v.e[i]), s);
    if (in) *reinterpret_cast<uint2*>(codes + row * c + col) = o.w;
    if ((threadIdx.x & 3) == 0) scale[b] = (uint8_t)s;
  }
}

// any row length and alignment: a lane a value
template <typename T>
__global__ __launch_bounds__(kThreads) void k_pack_any(const T* x, int c, long n_blocks, int8_t* codes,
                                                       uint8_t* scale) {
  const int blocks = (c + kPackBlock - 1) / kPackBlock;
  const long step = (long)gridDim.x * (kThreads / kPackBlock);
  for (long b = (long)blockIdx.x * (kThreads / kPackBlock) + threadIdx.x / kPackBlock; b < n_blocks;
       b += step) {
    const long row = b / blocks;
    const int col = (int)(b - row * blocks) * kPackBlock + threadIdx.x % kPackBlock;
    const float v = col < c ? to_f32<T>(x[row * c + col]) : 0.f;
    uint32_t top = abs_bits(v);
#pragma unroll
    for (int o = kPackBlock / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    const uint32_t s = pack_scale(top);
    if (col < c) codes[row * c + col] = s == 255 ? 0 : pack_code(v, s);
    if (threadIdx.x % kPackBlock == 0) scale[b] = (uint8_t)s;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_unpack_vec(const int8_t* codes, const uint8_t* scale,
                                                         int c, long n_quads, T* x) {
  const int blocks = (c + kPackBlock - 1) / kPackBlock;
  const long step = (long)gridDim.x * (kThreads / 4);
  for (long b = (long)blockIdx.x * (kThreads / 4) + (threadIdx.x >> 2); b < n_quads; b += step) {
    const long row = b / blocks;
    const int col = (int)(b - row * blocks) * kPackBlock + 8 * (threadIdx.x & 3);
    if (col >= c) continue;
    union {
      int8_t q[8];
      uint2 w;
    } o;
    o.w = *reinterpret_cast<const uint2*>(codes + row * c + col);
    const uint32_t s = scale[b];
    Vec8<T> v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v.e[i] = from_f32<T>(pack_value(o.q[i], s));
    *reinterpret_cast<Vec8<T>*>(x + row * c + col) = v;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_unpack_any(const int8_t* codes, const uint8_t* scale,
                                                         int c, long n_blocks, T* x) {
  const int blocks = (c + kPackBlock - 1) / kPackBlock;
  const long step = (long)gridDim.x * (kThreads / kPackBlock);
  for (long b = (long)blockIdx.x * (kThreads / kPackBlock) + threadIdx.x / kPackBlock; b < n_blocks;
       b += step) {
    const long row = b / blocks;
    const int col = (int)(b - row * blocks) * kPackBlock + threadIdx.x % kPackBlock;
    if (col < c) x[row * c + col] = from_f32<T>(pack_value(codes[row * c + col], scale[b]));
  }
}

bool whole_pieces(int c, const void* x, const void* codes) {
  return c % 8 == 0 && ((uintptr_t)x & 15) == 0 && ((uintptr_t)codes & 7) == 0;
}

unsigned grid_of(long work) { return (unsigned)std::min<long>(std::max<long>(work, 1), 16384); }

template <typename T>
hipError_t pack(int n, int c, const T* x, int8_t* codes, uint8_t* scale, hipStream_t st) {
  const long b = (long)n * cdiv(c, kPackBlock);
  if (whole_pieces(c, x, codes))
    hipLaunchKernelGGL(k_pack_vec<T>, dim3(grid_of((b + 63) / 64)), dim3(kThreads), 0, st, x, c, b,
                       codes, scale);
  else
    hipLaunchKernelGGL(k_pack_any<T>, dim3(grid_of((b + 7) / 8)), dim3(kThreads), 0, st, x, c, b,
                       codes, scale);
  return hipGetLastError();
}

template <typename T>
hipError_t unpack(int n, int c, const int8_t* codes, const uint8_t* scale, T* x, hipStream_t st) {
  const long b = (long)n * cdiv(c, kPackBlock);
  if (whole_pieces(c, x, codes))
    hipLaunchKernelGGL(k_unpack_vec<T>, dim3(grid_of((b + 63) / 64)), dim3(kThreads), 0, st, codes,
                       scale, c, b, x);
  else
    hipLaunchKernelGGL(k_unpack_any<T>, dim3(grid_of((b + 7) / 8)), dim3(kThreads), 0, st, codes,
                       scale, c, b, x);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_checkpoint_pack(bool bf16, int n, int c, const void* x, int8_t* codes,
                                  uint8_t* scale, hipStream_t st) {
  if (n == 0) return hipSuccess;
  return bf16 ? pack(n, c, static_cast<const bf16_t*>(x), codes, scale, st)
              : pack(n, c, static_cast<const float*>(x), codes, scale, st);
}

hipError_t launch_checkpoint_unpack(bool bf16, int n, int c, const int8_t* codes,
                                    const uint8_t* scale, void* x, hipStream_t st) {
  if (n == 0) return hipSuccess;
  return bf16 ? unpack(n, c, codes, scale, static_cast<bf16_t*>(x), st)
              : unpack(n, c, codes, scale, static_cast<float*>(x), st);
}

}  // namespace trimmoe
