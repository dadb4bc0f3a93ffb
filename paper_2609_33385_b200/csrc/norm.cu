// The norms around a block, with its gate and residual, in one pass over the rows:
//   z  = rms(y) * post_weight                        (without post_weight: z = y)
//   x' = x + residual_scale * gate * z               (without y: x' = x)
//   h  = rms(x') * pre_weight                        as bf16, and / or as e4m3 codes with a scale per 128 (block_scale.h)
//   rms(v) = v / sqrt(mean(v^2) + eps)
// Everything between the loads and the stores is fp32, and every output is rounded once: h is made from x' itself, not
// from its bf16 form.
//
// Bound by HBM (8 bytes an element where all is bf16; 16384 x 4096 with an fp32 stream 6.55 TB/s, as much as a copy).  A row stays in
// the registers of one CTA (of one warp up to 512 columns) between the two sums that it needs, eight consecutive values per
// thread and vector, so that sixteen lanes hold a block of 128.
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>

#include "block_scale.h"
#include "kernels.h"
#include "row_args.h"

namespace oled {
namespace {

struct NormArgs {
  const void* x;
  const uint16_t* y;
  const uint16_t* post;
  const uint16_t* gate;
  const uint16_t* pre;
  void* x_out;
  uint16_t* h;
  uint8_t* codes;
  float* scales;
  int64_t x_stride, y_stride, gate_stride, x_out_stride, h_stride, codes_stride, scales_stride;
  int tokens, hidden, gate_tokens;
  float eps, pre_eps, scale;
};

// Eight values at column c of a row, zeros behind its end, as they lie in memory.
struct Raw16 {
  uint4 p;
  __device__ __forceinline__ void values(float (&v)[8]) const { unpack8(p, v); }
};
struct Raw32 {
  uint4 p, q;
  __device__ __forceinline__ void values(float (&v)[8]) const {
    v[0] = __uint_as_float(p.x); v[1] = __uint_as_float(p.y); v[2] = __uint_as_float(p.z); v[3] = __uint_as_float(p.w);
    v[4] = __uint_as_float(q.x); v[5] = __uint_as_float(q.y); v[6] = __uint_as_float(q.z); v[7] = __uint_as_float(q.w);
  }
};
__device__ __forceinline__ Raw16 load8(const uint16_t* row, int c, int hidden) {
  Raw16 r{make_uint4(0u, 0u, 0u, 0u)};
  if (c < hidden) r.p = *reinterpret_cast<const uint4*>(row + c);
  return r;
}
__device__ __forceinline__ Raw32 load8(const float* row, int c, int hidden) {
  Raw32 r{make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
  if (c < hidden) {
    r.p = *reinterpret_cast<const uint4*>(row + c);
    r.q = *reinterpret_cast<const uint4*>(row + c + 4);
  }
  return r;
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void store8(uint16_t* row, int c, int hidden, const float (&v)[8]) {
  if (c < hidden)
    *reinterpret_cast<uint4*>(row + c) =
        make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* row, int c, int hidden, const float (&v)[8]) {
  if (c < hidden) {
    *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// The sum over the THREADS threads of a row (a warp, or the whole CTA), in every one of them.
template <int THREADS>
__device__ __forceinline__ float row_sum(float s, float* s_part) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  if (THREADS > 32) {
    constexpr int kWarps = THREADS / 32;
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += s_part[w];
  }
  return s;
}

// Rows of whole 16-byte vectors on 16-byte boundaries (codes: on 8-byte boundaries).
// R: the residual stream's type (uint16_t: bf16).  THREADS per row (32: four rows per CTA), V vectors per thread.  Two vectors
// were best wherever there are threads for it (16384 x 2048 bf16 with codes: 54 us, one vector 66, four 63).
// (an SM holds 1280 threads of fp32 rows, 48 registers each, and 1024 of bf16 rows, 64; 16384 x 4096 with 1024 fp32 threads 126.0 us
// instead of 122.7, with 768 bf16 ones 102 instead of 88)
template <typename R, int THREADS, int V>
__global__ void __launch_bounds__(THREADS == 32 ? 128 : THREADS, V > 2 ? 1 : (sizeof(R) == 4 ? 1280 : 1024) / (THREADS == 32 ? 128 : THREADS))
norm_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float s_part[2][THREADS / 32];
  constexpr int kRows = THREADS == 32 ? 4 : 1;
  const int lane_in_row = (int)threadIdx.x % THREADS, H = a.hidden;
  const int64_t t = (int64_t)blockIdx.x * kRows + (kRows > 1 ? threadIdx.x / THREADS : 0);
  griddep_launch_dependents();
  griddep_wait();
  if (t >= a.tokens) return;  // (whole warps, and only where no barrier follows)
  const R* const xr = static_cast<const R*>(a.x) + t * a.x_stride;
  const uint16_t* const yr = a.y + t * a.y_stride;
  const uint16_t* const gr = a.gate + (a.gate_tokens > 0 ? t / a.gate_tokens : 0) * a.gate_stride;
  // Everything that the row needs is requested before its first sum - the weights too where x is bf16 (16384 x 4096: 95.7 us,
  // with them 88.1); beside an fp32 x their registers cost more warps than that saves (122.6 us, with them 136.9).
  constexpr bool kEarly = sizeof(R) == 2;
  decltype(load8(xr, 0, 0)) x_raw[V];
  Raw16 y_raw[V], post[V], gate[V], pre[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (lane_in_row + i * THREADS) * 8;
    if (a.y != nullptr) y_raw[i] = load8(yr, c, H);
    x_raw[i] = load8(xr, c, H);
  }
  if (kEarly)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = (lane_in_row + i * THREADS) * 8;
      if (a.post != nullptr) post[i] = load8(a.post, c, H);
      if (a.gate != nullptr) gate[i] = load8(gr, c, H);
      if (a.pre != nullptr) pre[i] = load8(a.pre, c, H);
    }
  float v[V][8];
  if (a.y != nullptr) {
    float z[V][8], r = 1.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) y_raw[i].values(z[i]);
    if (a.post != nullptr) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fmaf(z[i][j], z[i][j], s);
      r = rsqrtf(row_sum<THREADS>(s, s_part[0]) / (float)H + a.eps);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float w[8];
      if (a.post != nullptr) {
        if (!kEarly) post[i] = load8(a.post, (lane_in_row + i * THREADS) * 8, H);
        post[i].values(w);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[i][j] = z[i][j] * r * w[j];
      }
      if (a.gate != nullptr) {
        if (!kEarly) gate[i] = load8(gr, (lane_in_row + i * THREADS) * 8, H);
        gate[i].values(w);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[i][j] *= w[j];
      }
      x_raw[i].values(v[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = fmaf(a.scale, z[i][j], v[i][j]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) x_raw[i].values(v[i]);
  }
  if (a.x_out != nullptr) {
    R* const xo = static_cast<R*>(a.x_out) + t * a.x_out_stride;
#pragma unroll
    for (int i = 0; i < V; ++i) store8(xo, (lane_in_row + i * THREADS) * 8, H, v[i]);
  }
  if (a.pre == nullptr) return;
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(v[i][j], v[i][j], s);
  const float r = rsqrtf(row_sum<THREADS>(s, s_part[1]) / (float)H + a.pre_eps);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = (lane_in_row + i * THREADS) * 8;
    float w[8];
    if (!kEarly) pre[i] = load8(a.pre, c, H);
    pre[i].values(w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = v[i][j] * r * w[j];
    if (a.h != nullptr) store8(a.h + t * a.h_stride, c, H, v[i]);
  }
  if (a.codes == nullptr) return;
  // lane i of a half-warp divides for its block i
  uint32_t amax[V], mine = 0u;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    amax[i] = amax_half_warp(amax8(v[i]));
    mine = i == 0 || (int)(threadIdx.x & (V - 1)) == i ? amax[i] : mine;
  }
  const float my_inverse = block_inverse(mine);
  const int half_lane = threadIdx.x & 15, c_mine = (lane_in_row - half_lane + half_lane * THREADS) * 8;
  if (half_lane < V && c_mine < H) a.scales[t * a.scales_stride + c_mine / kScaleBlock] = block_scale(mine);
  uint8_t* const cr = a.codes + t * a.codes_stride;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float inverse = __shfl_sync(0xffffffffu, my_inverse, (threadIdx.x & 16) | i);
    const int c = (lane_in_row + i * THREADS) * 8;
    if (c < H) *reinterpret_cast<uint2*>(cr + c) = codes8(v[i], inverse);
  }
}

// Any other rows: element by element, a warp's 32 next to each other, N per thread.  A block of 128 is then four warps'
// elements of one turn.  (Eight consecutive elements a thread, loaded one by one, took 168 us at
// 4099 x 3759 with both outputs, 16 of these 133, eight 66; the code of a row is run once, and fetching it counts.)
__device__ __forceinline__ float load1(const uint16_t* row, int c) { return __uint_as_float((uint32_t)row[c] << 16); }
__device__ __forceinline__ float load1(const float* row, int c) { return row[c]; }
__device__ __forceinline__ void store1(uint16_t* row, int c, float v) { row[c] = __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
__device__ __forceinline__ void store1(float* row, int c, float v) { row[c] = v; }

template <typename R, int THREADS, int N>
__global__ void __launch_bounds__(THREADS)
norm_odd_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float s_part[2][THREADS / 32];
  __shared__ uint32_t s_amax[N][THREADS / 32];
  const int H = a.hidden, tid = threadIdx.x;
  const int64_t t = blockIdx.x;
  griddep_launch_dependents();
  griddep_wait();
  const R* const xr = static_cast<const R*>(a.x) + t * a.x_stride;
  float v[N];
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = tid + i * THREADS < H ? load1(xr, tid + i * THREADS) : 0.0f;
  if (a.y != nullptr) {
    const uint16_t* const yr = a.y + t * a.y_stride;
    const uint16_t* const gr = a.gate + (a.gate_tokens > 0 ? t / a.gate_tokens : 0) * a.gate_stride;
    float z[N], r = 1.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = tid + i * THREADS < H ? load1(yr, tid + i * THREADS) : 0.0f;
    if (a.post != nullptr) {
      float s = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) s = fmaf(z[i], z[i], s);
      r = rsqrtf(row_sum<THREADS>(s, s_part[0]) / (float)H + a.eps);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = tid + i * THREADS;
      if (c >= H) continue;
      if (a.post != nullptr) z[i] = z[i] * r * load1(a.post, c);
      if (a.gate != nullptr) z[i] *= load1(gr, c);
      v[i] = fmaf(a.scale, z[i], v[i]);
    }
  }
  if (a.x_out != nullptr) {
    R* const xo = static_cast<R*>(a.x_out) + t * a.x_out_stride;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (tid + i * THREADS < H) store1(xo, tid + i * THREADS, v[i]);
  }
  if (a.pre == nullptr) return;
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) s = fmaf(v[i], v[i], s);
  const float r = rsqrtf(row_sum<THREADS>(s, s_part[1]) / (float)H + a.pre_eps);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = tid + i * THREADS;
    if (c < H) {
      v[i] = v[i] * r * load1(a.pre, c);
      if (a.h != nullptr) store1(a.h + t * a.h_stride, c, v[i]);
    }
    if (a.codes != nullptr) {
      const uint32_t big = __reduce_max_sync(0xffffffffu, c < H ? __float_as_uint(v[i]) & 0x7fffffffu : 0u);
      if ((tid & 31) == 0) s_amax[i][tid >> 5] = big;
    }
  }
  if (a.codes == nullptr) return;
  __syncthreads();
  uint8_t* const cr = a.codes + t * a.codes_stride;
  // lane i has the scale of the block that the warp's elements of turn i belong to
  static_assert(N <= 32, "a lane per turn");
  const int lane = tid & 31, turn = min(lane, N - 1), block = ((tid & ~127) + turn * THREADS) / kScaleBlock;
  const uint32_t* const four = &s_amax[turn][(tid >> 7) * 4];
  const uint32_t amax = max(max(max(four[0], four[1]), max(four[2], four[3])), kAmaxFloor);
  const float inverse = block_inverse(amax);
  if ((tid & 127) < N && block * kScaleBlock < H) a.scales[t * a.scales_stride + block] = block_scale(amax);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float f = __shfl_sync(0xffffffffu, inverse, i);
    const int c = tid + i * THREADS;
    if (c < H) cr[c] = (uint8_t)e4m3x2(__fmul_rn(v[i], f), 0.0f);
  }
}

template <typename R>
cudaError_t launch_norm_kind(cudaStream_t st, const NormArgs& a, bool vec) {
  const dim3 row((unsigned)a.tokens), rows4((unsigned)(((int64_t)a.tokens + 3) / 4));
  if (!vec) {
    if (a.hidden <= 512) return launch_pdl(norm_odd_kernel<R, 128, 4>, row, dim3(128), 0, st, a);
    if (a.hidden <= 2048) return launch_pdl(norm_odd_kernel<R, 256, 8>, row, dim3(256), 0, st, a);
    if (a.hidden <= 4096) return launch_pdl(norm_odd_kernel<R, 512, 8>, row, dim3(512), 0, st, a);
    if (a.hidden <= 8192) return launch_pdl(norm_odd_kernel<R, 1024, 8>, row, dim3(1024), 0, st, a);
    return launch_pdl(norm_odd_kernel<R, 1024, 16>, row, dim3(1024), 0, st, a);
  }
  if (a.hidden <= 256) return launch_pdl(norm_kernel<R, 32, 1>, rows4, dim3(128), 0, st, a);
  if (a.hidden <= 512) return launch_pdl(norm_kernel<R, 32, 2>, rows4, dim3(128), 0, st, a);
  if (a.hidden <= 1024) return launch_pdl(norm_kernel<R, 64, 2>, row, dim3(64), 0, st, a);
  if (a.hidden <= 2048) return launch_pdl(norm_kernel<R, 128, 2>, row, dim3(128), 0, st, a);
  if (a.hidden <= 4096) return launch_pdl(norm_kernel<R, 256, 2>, row, dim3(256), 0, st, a);
  if (a.hidden <= 8192) return launch_pdl(norm_kernel<R, 512, 2>, row, dim3(512), 0, st, a);
  return launch_pdl(norm_kernel<R, 512, 4>, row, dim3(512), 0, st, a);
}

}  // namespace

int norm_residual(const oled_norm_shape* shape, const void* x, const void* y, const void* post_weight, const void* gate,
                  const void* pre_weight, int32_t n_tokens, cudaStream_t st, void* x_out, void* h, void* h_codes, float* h_scales, float pre_eps) {
  if (!shape) return OLED_ERR_INVALID_ARG;
  const oled_norm_shape& s = *shape;
  const int H = s.hidden, blocks = (H + kScaleBlock - 1) / kScaleBlock;
  if (H <= 0 || H > 16384 || (s.residual != OLED_BF16 && s.residual != OLED_FP32) || s.gate_tokens < 0 || n_tokens < 0 ||
      !(s.eps > 0.0f) || !std::isfinite(s.eps) || !std::isfinite(s.residual_scale))
    return OLED_ERR_INVALID_ARG;
  if (n_tokens == 0) return OLED_OK;
  const int64_t item = s.residual == OLED_FP32 ? 4 : 2, T = n_tokens;
  if (!x || (!y && (post_weight || gate)) || ((h || h_codes) != (pre_weight != nullptr)) || ((h_codes != nullptr) != (h_scales != nullptr)) ||
      (!x_out && !h && !h_codes))
    return OLED_ERR_INVALID_ARG;
  if (!stride_ok(s.x_stride, H) || (y && !stride_ok(s.y_stride, H)) || (gate && !stride_ok(s.gate_stride, H)) ||
      (x_out && !stride_ok(s.x_out_stride, H)) || (h && !stride_ok(s.h_stride, H)) ||
      (h_codes && (!stride_ok(s.codes_stride, H) || !stride_ok(s.scales_stride, blocks))))
    return OLED_ERR_INVALID_ARG;
  if (off_boundary(x, item) || off_boundary(x_out, item) || off_boundary(y, 2) || off_boundary(post_weight, 2) || off_boundary(gate, 2) ||
      off_boundary(pre_weight, 2) || off_boundary(h, 2) || off_boundary(h_scales, 4))
    return OLED_ERR_INVALID_ARG;
  const int64_t gate_rows = s.gate_tokens > 0 ? (T + s.gate_tokens - 1) / s.gate_tokens : 1;
  const RowRange in[] = {{x, s.x_stride * item, H * item, T},       {y, s.y_stride * 2, H * 2, T}, {post_weight, H * 2, H * 2, 1},
                         {gate, s.gate_stride * 2, H * 2, gate_rows}, {pre_weight, H * 2, H * 2, 1}};
  const RowRange out[] = {{x_out, s.x_out_stride * item, H * item, T}, {h, s.h_stride * 2, H * 2, T},
                          {h_codes, s.codes_stride, H, T},             {h_scales, s.scales_stride * 4, blocks * 4, T}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < i; ++j)
      if (rows_overlap(out[i], out[j])) return OLED_ERR_INVALID_ARG;
    for (int j = 0; j < 5; ++j) {
      // an element of x or y is read by the thread that writes the same element of x_out or h, before it does
      if (out[i].p && (i == 0 || i == 1) && (j == 0 || j == 1) && same_rows(out[i], in[j])) continue;
      if (rows_overlap(out[i], in[j])) return OLED_ERR_INVALID_ARG;
    }
  }
  NormArgs a;
  a.x = x;
  a.y = static_cast<const uint16_t*>(y);
  a.post = static_cast<const uint16_t*>(post_weight);
  a.gate = static_cast<const uint16_t*>(gate);
  a.pre = static_cast<const uint16_t*>(pre_weight);
  a.x_out = x_out;
  a.h = static_cast<uint16_t*>(h);
  a.codes = static_cast<uint8_t*>(h_codes);
  a.scales = h_scales;
  a.x_stride = s.x_stride;
  a.y_stride = s.y_stride;
  a.gate_stride = s.gate_stride;
  a.x_out_stride = s.x_out_stride;
  a.h_stride = s.h_stride;
  a.codes_stride = s.codes_stride;
  a.scales_stride = s.scales_stride;
  a.tokens = n_tokens;
  a.hidden = H;
  a.gate_tokens = s.gate_tokens;
  a.eps = s.eps;
  a.pre_eps = pre_eps > 0.0f ? pre_eps : s.eps;
  a.scale = s.residual_scale;
  // 16-byte vectors where every row that is touched starts on a 16-byte boundary (codes: 8) and holds whole ones
  bool vec = H % 8 == 0;
  auto rows_ok = [&](const void* p, int64_t stride_bytes, uintptr_t align) {
    if (p != nullptr) vec = vec && !off_boundary(p, align) && stride_bytes % (int64_t)align == 0;
  };
  rows_ok(x, s.x_stride * item, 16);
  rows_ok(x_out, s.x_out_stride * item, 16);
  rows_ok(y, s.y_stride * 2, 16);
  rows_ok(gate, s.gate_stride * 2, 16);
  rows_ok(post_weight, 0, 16);
  rows_ok(pre_weight, 0, 16);
  rows_ok(h, s.h_stride * 2, 16);
  rows_ok(h_codes, s.codes_stride, 8);
  const cudaError_t err = s.residual == OLED_FP32 ? launch_norm_kind<float>(st, a, vec) : launch_norm_kind<uint16_t>(st, a, vec);
  return cudaGetLastError() == cudaSuccess && err == cudaSuccess ? OLED_OK : OLED_ERR_CUDA;
}

}  // namespace oled

extern "C" int oled_norm_residual(const oled_norm_shape* shape, const void* x, const void* y, const void* post_weight,
                                  const void* gate, const void* pre_weight, int32_t n_tokens, void* cuda_stream, void* x_out,
                                  void* h, void* h_codes, float* h_scales) {
  return oled::norm_residual(shape, x, y, post_weight, gate, pre_weight, n_tokens, static_cast<cudaStream_t>(cuda_stream), x_out, h,
                             h_codes, h_scales, 0.0f);
}
