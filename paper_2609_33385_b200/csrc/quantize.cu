// Activations in front of a product of e4m3 codes: codes and one fp32 scale per row and 128 columns (block_scale.h), of
// bf16 rows or of silu(gate) * up of rows gate | up, in fp32 from the loads to the codes.
//
// HBM: 2 bytes read (4 with SwiGLU) and 1 written per element.  A half-warp holds a block, eight values (one
// 16-byte load) a lane, so that a block's maximum is four shuffles; a warp takes VECS times 256 columns of a row, its
// loads in flight together: four of them where there are rows enough to fill the GPU (16384 x 4096: 35.2 us, two 37.5), one where
// there are not (32 x 1024 with SwiGLU 1.9 us, four 2.6).
#include <algorithm>

#include "block_scale.h"
#include "kernels.h"
#include "row_args.h"

namespace oled {
namespace {

constexpr int kQuantWarps = 4;

template <bool SWIGLU, int VECS>
__global__ void __launch_bounds__(kQuantWarps * 32)
quantize_kernel(const uint16_t* __restrict__ x, int64_t x_stride, int64_t pieces, int pieces_per_row, int cols,
                uint8_t* __restrict__ codes, int64_t codes_stride, float* __restrict__ scales, int64_t scales_stride) {
  const int lane = threadIdx.x & 31;
  griddep_launch_dependents();
  griddep_wait();
  const int64_t piece = (int64_t)blockIdx.x * kQuantWarps + (threadIdx.x >> 5);
  if (piece >= pieces) return;
  const int64_t row = pieces_per_row == 1 ? piece : piece / pieces_per_row;
  const int c0 = (int)(piece - row * pieces_per_row) * (VECS * 256) + lane * 8;
  const uint16_t* src = x + row * x_stride + c0;
  uint4 a[VECS], b[SWIGLU ? VECS : 1];
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    a[i] = make_uint4(0u, 0u, 0u, 0u);
    if (SWIGLU) b[i] = a[i];
    if (c0 + i * 256 < cols) {  // (cols is a multiple of 16: a vector is whole or absent)
      a[i] = __ldcs(reinterpret_cast<const uint4*>(src + i * 256));
      if (SWIGLU) b[i] = __ldcs(reinterpret_cast<const uint4*>(src + cols + i * 256));
    }
  }
  if constexpr (SWIGLU) {
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      float v[8], u[8];
      unpack8(a[i], v);
      unpack8(b[i], u);
      // (The sigmoid's fast exponential and quotient are off by some 2^-21, the code by 2^-4: of 6.3 M codes 19 are on the other side of a rounding's
      // border from 64 bits, with expf() 17 and 8192 x 4096 in 35.0 us instead of 28.7, with an IEEE quotient too 12 and 42.8.)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __fdividef(v[j], 1.0f + __expf(-v[j])) * u[j];
      const uint32_t amax = amax_half_warp(amax8(v));
      const int c = c0 + i * 256;
      if (c < cols) {
        *reinterpret_cast<uint2*>(codes + row * codes_stride + c) = codes8(v, block_inverse(amax));
        if ((lane & 15) == 0) scales[row * scales_stride + c / kScaleBlock] = block_scale(amax);
      }
    }
  } else {
    // the blocks' largest magnitudes, two bf16 ones a word: their bits order like the values, and like fp32 ones with 16 zeros behind them
    uint32_t amax[VECS];
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      uint32_t big = __vmaxu2(__vmaxu2(a[i].x & 0x7fff7fffu, a[i].y & 0x7fff7fffu), __vmaxu2(a[i].z & 0x7fff7fffu, a[i].w & 0x7fff7fffu));
#pragma unroll
      for (int d = 8; d >= 1; d >>= 1) big = __vmaxu2(big, __shfl_xor_sync(0xffffffffu, big, d));
      amax[i] = max(max(big << 16, big & 0xffff0000u), kAmaxFloor);
    }
    // Lane i of a half-warp divides for its block i: quotients for every block in every lane were a third of the kernel's
    // instructions, which is what it was bound by (16384 x 4096: 35.2 us, now 32.0, as much as a copy).
    uint32_t mine = amax[0];
#pragma unroll
    for (int i = 1; i < VECS; ++i) mine = (lane & (VECS - 1)) == i ? amax[i] : mine;
    const float my_inverse = block_inverse(mine);
    {
      const int block = lane & 15, c = c0 - block * 8 + block * 256;  // (of the half-warp's blocks, 256 columns apart)
      if (block < VECS && c < cols) scales[row * scales_stride + c / kScaleBlock] = block_scale(mine);
    }
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const float inverse = __shfl_sync(0xffffffffu, my_inverse, (lane & 16) | i);
      float v[8];
      unpack8(a[i], v);
      const int c = c0 + i * 256;
      if (c < cols) *reinterpret_cast<uint2*>(codes + row * codes_stride + c) = codes8(v, inverse);
    }
  }
}

}  // namespace

cudaError_t launch_quantize(cudaStream_t st, const uint16_t* x, int64_t x_stride, int64_t rows, int cols, bool swiglu,
                            uint8_t* codes, int64_t codes_stride, float* scales, int64_t scales_stride) {
  // four vectors a lane once that still gives every SM sixteen warps
  const bool wide = rows * ((cols + 1023) / 1024) >= 148 * 16;
  const int width = wide ? 1024 : 256, per_row = (cols + width - 1) / width;
  const int64_t pieces = rows * per_row;
  const dim3 grid((unsigned)((pieces + kQuantWarps - 1) / kQuantWarps));
  const auto kernel = swiglu ? (wide ? quantize_kernel<true, 4> : quantize_kernel<true, 1>) : (wide ? quantize_kernel<false, 4> : quantize_kernel<false, 1>);
  return launch_pdl(kernel, grid, dim3(kQuantWarps * 32), 0, st, x, x_stride, pieces, per_row, cols, codes, codes_stride, scales, scales_stride);
}

}  // namespace oled

extern "C" int oled_quantize_blocks(const void* x, int64_t x_stride, int32_t rows, int32_t cols, int32_t swiglu,
                                       void* cuda_stream, void* codes, int64_t codes_stride, float* scales,
                                       int64_t scales_stride) {
  using namespace oled;
  const int64_t width = swiglu ? 2 * (int64_t)cols : (int64_t)cols;
  const int blocks = cols > 0 ? (cols + kScaleBlock - 1) / kScaleBlock : 0;
  if (rows < 0 || cols <= 0 || cols % 16 != 0 || cols > OLED_MAX_PRODUCT_K || (swiglu != 0 && swiglu != 1) || !stride_ok(x_stride, width) ||
      x_stride % 8 != 0 || !stride_ok(codes_stride, cols) || codes_stride % 16 != 0 || !stride_ok(scales_stride, blocks))
    return OLED_ERR_INVALID_ARG;
  if (rows == 0) return OLED_OK;
  if (!x || !codes || !scales || off_boundary(x, 16) || off_boundary(codes, 16) || off_boundary(scales, 4))
    return OLED_ERR_INVALID_ARG;
  const RowRange in{x, x_stride * 2, width * 2, rows}, out{codes, codes_stride, cols, rows}, sc{scales, scales_stride * 4, blocks * 4, rows};
  if (rows_overlap(in, out) || rows_overlap(in, sc) || rows_overlap(out, sc)) return OLED_ERR_INVALID_ARG;
  const cudaError_t err = launch_quantize(static_cast<cudaStream_t>(cuda_stream), static_cast<const uint16_t*>(x), x_stride, rows, cols,
                                          swiglu != 0, static_cast<uint8_t*>(codes), codes_stride, scales, scales_stride);
  return cudaGetLastError() == cudaSuccess && err == cudaSuccess ? OLED_OK : OLED_ERR_CUDA;
}
