// C[m, n] = sum_k A[m, k] B[n, k] (+ D[m, n]) of e4m3 codes with block scales (oled_matmul_blocks): one fp32 scale per row
// of A and 128 columns, one per 128 x 128 block of B.
//
// The scales change every 128 values of k, so a k-block's product is summed by the tensor cores alone (kind::f8f6f4, fp32 in
// tensor memory) and then added, times its two scales, to fp32 accumulators in registers: C = sum_b (sa sb)_b (A_b B_b^T).
// The scale of a row of A times that of the block of B is rounded once, the sums of k-blocks are fp32 fused multiply-adds.
//
// product_few_kernel: the weights are the MMA's M (128 rows, one block of scales), up to 128 rows of A its N, so that few
// tokens cost few columns.  What bounds it is the weights' way into shared memory; where the tiles are fewer than the SMs, a cluster of
// up to eight CTAs shares a tile's k-blocks and adds up through distributed shared memory, in the order of the k-blocks.
//
// product_pair_kernel: many rows.  A pair of CTAs computes 256 rows of A x 256 of B with M = 256 MMAs (cta_group::2): each CTA
// holds 128 rows of A and of the accumulators and half of the rows of B, 32 KB a k-block for 512 cycles of MMAs (one CTA alone
// on 128 x 256 would need 48 KB, more than an SM's share of L2 delivers in that time).  Here the rows of A are
// the accumulators' lanes, so that a thread's scale is one number per k-block.  Eight warps read a k-block's 128 x 256 products
// from tensor memory (two buffers) and add them to 128 registers a thread beside the next k-block's MMAs; results leave through shared memory as bulk tensor stores where rows of C are on 16-byte boundaries.
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "block_scale.h"
#include "kernels.h"
#include "row_args.h"
#include "sm100_ptx.h"

namespace oled {
namespace {

struct ProductArgs {
  const float* a_scale;
  const float* b_scale;
  const uint16_t* add;
  void* out;
  int64_t a_scale_stride, b_scale_stride, add_stride, out_stride;
  int m, n, k_blocks, out_fp32, vec, vec_add;  // vec: see store_four; vec_add: rows of D on 16-byte boundaries
};

// Four consecutive columns of a row of C.  vec: rows of C (and of D) start on boundaries of four elements.
__device__ __forceinline__ void store_four(const ProductArgs& p, int64_t row, int col, float (&v)[4], bool vec) {
  const uint16_t* const d = p.add != nullptr ? p.add + row * p.add_stride + col : nullptr;
  if (vec && col + 3 < p.n) {
    if (d != nullptr) {
      const uint2 w = *reinterpret_cast<const uint2*>(d);
      v[0] += __uint_as_float(w.x << 16);
      v[1] += __uint_as_float(w.x & 0xffff0000u);
      v[2] += __uint_as_float(w.y << 16);
      v[3] += __uint_as_float(w.y & 0xffff0000u);
    }
    if (p.out_fp32) {
      *reinterpret_cast<float4*>(static_cast<float*>(p.out) + row * p.out_stride + col) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
      const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + row * p.out_stride + col) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (col + j < p.n) {
      const float r = d != nullptr ? v[j] + __uint_as_float((uint32_t)d[j] << 16) : v[j];
      if (p.out_fp32) static_cast<float*>(p.out)[row * p.out_stride + col + j] = r;
      else static_cast<uint16_t*>(p.out)[row * p.out_stride + col + j] = __bfloat16_as_ushort(__float2bfloat16_rn(r));
    }
}
// Waits of these kernels are bounded like every other; there is no context to report to, so a tile whose wait ran out
// becomes NaN.
// (The warp stays converged: polling lane by lane cost 100 cycles more where the barrier was ready.)
__device__ __forceinline__ bool product_warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  unsigned long long t0 = 0;
  for (uint32_t it = 1; !__all_sync(0xffffffffu, mbar_try(bar, parity)); ++it) {
    if ((it & 1023u) == 0u) {
      const unsigned long long now = globaltimer();
      if (t0 == 0) t0 = now;
      if (now - t0 > kWaitLimitNs) *abort_flag = 1;
      if (__any_sync(0xffffffffu, *abort_flag != 0)) return false;
    }
  }
  return true;
}

// ---- few rows of A ---------------------------------------------------------------------------
constexpr int kFewStages = 8;   // at most
constexpr int kFewAccs = 4;     // k-blocks whose products wait in tensor memory
constexpr uint32_t kWTile = 128 * 128;
__host__ __device__ constexpr int few_epi_warps(int nt) { return nt > 64 ? 8 : 4; }

struct __align__(16) ProductFewCtl {
  unsigned long long full[kFewStages];
  unsigned long long empty[kFewStages];
  unsigned long long acc_full[kFewAccs];
  unsigned long long acc_empty[kFewAccs];
  uint32_t tmem_base;
  int abort;
};

__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A tile's columns (rows of A) are joined by the SPLIT CTAs of its cluster, NT / SPLIT each.  Every CTA sends its partial sums to where
// they are joined - `sums` there: [SPLIT senders][NT / SPLIT columns][128] - as soon as it has them: stores across the cluster are
// not waited for, loads were, and the CTAs then had to wait for one another a second time before they left (250 x 4096 x
// 2048: 10.5 us with loads).
template <int NT, int SPLIT, int COLS>
__device__ __forceinline__ void send_columns(const float (&acc)[COLS], uint32_t sums, int rank, int col0, int row) {
  constexpr int kShare = NT / SPLIT, kRun = COLS < kShare ? COLS : kShare;  // columns of the thread that go to one CTA
#pragma unroll
  for (int r = 0; r < COLS; r += kRun) {
    const int to = (col0 + r) / kShare;
    const uint32_t at = sums + (uint32_t)((rank * kShare + (col0 + r) % kShare) * 128 + row) * 4u;
    const uint32_t dst = SPLIT > 1 ? map_to_cta(at, (uint32_t)to) : at;
#pragma unroll
    for (int c = 0; c < kRun; ++c) {
      if (SPLIT > 1) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dst + (uint32_t)c * 512u), "f"(acc[r + c]) : "memory");
      else asm volatile("st.shared.f32 [%0], %1;" ::"r"(dst + (uint32_t)c * 512u), "f"(acc[r + c]) : "memory");
    }
  }
}
// The CTA's columns, the senders' parts added in order, a warp one column at a time and four of them requested together.
template <int NT, int SPLIT>
__device__ __forceinline__ void join_columns(const ProductArgs& p, const float* sums, int rank, int warp, int lane, int m0, int n0) {
  constexpr int kShare = NT / SPLIT, kEpi = few_epi_warps(NT), kTogether = SPLIT > 4 ? 2 : 4;
  const int n_cols = min(kShare, p.m - m0 - kShare * rank);
#pragma unroll 1
  for (int c = warp; c < n_cols; c += kEpi * kTogether) {
    float4 part[kTogether][SPLIT];
#pragma unroll
    for (int u = 0; u < kTogether; ++u)
#pragma unroll
      for (int s = 0; s < SPLIT; ++s)
        part[u][s] = *reinterpret_cast<const float4*>(sums + (s * kShare + min(c + u * kEpi, kShare - 1)) * 128 + lane * 4);
#pragma unroll
    for (int u = 0; u < kTogether; ++u) {
      if (c + u * kEpi >= n_cols) break;
      float v[4] = {part[u][0].x, part[u][0].y, part[u][0].z, part[u][0].w};
#pragma unroll
      for (int s = 1; s < SPLIT; ++s) {
        v[0] += part[u][s].x;
        v[1] += part[u][s].y;
        v[2] += part[u][s].z;
        v[3] += part[u][s].w;
      }
      store_four(p, m0 + kShare * rank + c + u * kEpi, n0 + lane * 4, v, p.vec != 0);
    }
  }
}

// blockIdx.x: tile of 128 rows of B x the SPLIT CTAs of a cluster, blockIdx.y: tile of NT rows of A.  Dynamic shared memory: control,
// [k-blocks of the CTA][NT] scales, then on a 1024-byte boundary the ring of `stages` (weight tile, rows of A), then the sums.
template <int NT, int SPLIT>
__global__ void __launch_bounds__((few_epi_warps(NT) + 2) * 32, 1)
product_few_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a,
                   const __grid_constant__ ProductArgs p, int stages) {
  constexpr int kEpi = few_epi_warps(NT), kProducer = kEpi, kMma = kEpi + 1;
  constexpr int kCols = NT / (kEpi / 4);  // columns of an epilogue warp
  constexpr uint32_t kStage = kWTile + NT * 128;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  ProductFewCtl* const ctl = reinterpret_cast<ProductFewCtl*>(smem_raw);
  float* const s_scale = reinterpret_cast<float*>(smem_raw + sizeof(ProductFewCtl));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = SPLIT > 1 ? (int)cluster_cta_rank() : 0;
  const int n_tile = (int)blockIdx.x / SPLIT, n0 = n_tile * 128, m0 = (int)blockIdx.y * NT;
  const int kb0 = (int)((int64_t)p.k_blocks * rank / SPLIT), kb1 = (int)((int64_t)p.k_blocks * (rank + 1) / SPLIT);
  const int kbs = kb1 - kb0;
  const uint32_t smem0 = smem_u32(smem_raw);
  const uint32_t ring = (smem_u32(s_scale) + (uint32_t)((p.k_blocks + SPLIT - 1) / SPLIT) * NT * 4u + 1023u) & ~1023u;
  const uint32_t sums = ring + (uint32_t)stages * kStage;
  volatile int* const abort_flag = &ctl->abort;
  const auto load = [&](int i, int stage) {
    const uint32_t bar = smem_u32(&ctl->full[stage]), dst = ring + (uint32_t)stage * kStage;
    mbar_expect_tx(bar, kStage);
    tma_load_2d(&map_b, dst, bar, (kb0 + i) * 128, n0);
    tma_load_2d(&map_a, dst + kWTile, bar, (kb0 + i) * 128, m0);
  };

  if (SPLIT > 1) cluster_arrive_relaxed();  // "this CTA runs": waited for before the first store into another one
  // Before the CTA's first barrier the first loads set out and tensor memory is taken.
  if (warp == kProducer) {
    if (lane == 0) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_b)) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_a)) : "memory");
      for (int s = 0; s < stages; ++s) {
        mbar_init(smem_u32(&ctl->full[s]), 1);
        mbar_init(smem_u32(&ctl->empty[s]), 1);
      }
      for (int s = 0; s < kFewAccs; ++s) {
        mbar_init(smem_u32(&ctl->acc_full[s]), 1);
        mbar_init(smem_u32(&ctl->acc_empty[s]), kEpi);
      }
      ctl->abort = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      griddep_wait();
      for (int i = 0; i < min(stages, kbs); ++i) load(i, i);
    }
    __syncwarp();
  } else if (warp == kMma) {
    // Tensor memory is taken only once the kernel in front has given its own back, the kernel behind starts only once every
    // CTA has its share, and nobody holds any while waiting for another CTA: no two can wait for each other's.
    griddep_wait();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                 "r"(kFewAccs * NT)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  } else {
    griddep_wait();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_launch_dependents();
  const uint32_t tmem = ctl->tmem_base;

  if (warp == kProducer) {
    bool ok = true;
    for (int i = stages; i < kbs && ok; ++i) {
      const int stage = i % stages;
      ok = product_warp_wait(smem_u32(&ctl->empty[stage]), ((uint32_t)(i / stages) & 1u) ^ 1u, abort_flag);
      if (ok && elect_one()) load(i, stage);
      __syncwarp();
    }
    if (!ok) {  // let copies already issued land before the CTA's shared memory is released
      const unsigned long long t0 = globaltimer();
      while (globaltimer() - t0 < 2000000ull) {
      }
    }
    if (SPLIT > 1) cluster_wait();
  } else if (warp == kMma) {
    const uint64_t w_desc0 = make_smem_desc(ring), x_desc0 = make_smem_desc(ring + kWTile);
    const uint32_t idesc = make_idesc_e4m3(NT);
    int stage = 0;
    uint32_t phase = 0;
    for (int i = 0; i < kbs; ++i) {
      const int buf = i % kFewAccs;
      if (i >= kFewAccs && !product_warp_wait(smem_u32(&ctl->acc_empty[buf]), ((uint32_t)(i / kFewAccs) & 1u) ^ 1u, abort_flag)) break;
      if (!product_warp_wait(smem_u32(&ctl->full[stage]), phase, abort_flag)) break;
      tc_fence_after();
      if (elect_one()) {
        const uint64_t off = (uint64_t)((uint32_t)stage * (kStage >> 4));
        const uint32_t d = tmem + (uint32_t)(buf * NT);
        tc_mma_desc<true, false>(d, w_desc0 + off, x_desc0 + off, idesc);
#pragma unroll
        for (int k = 1; k < 4; ++k) tc_mma_desc<true, true>(d, w_desc0 + off + k * 2, x_desc0 + off + k * 2, idesc);
        tc_commit(smem_u32(&ctl->acc_full[buf]));
        if (i + stages < kbs) tc_commit(smem_u32(&ctl->empty[stage]));
      }
      __syncwarp();
      if (++stage == stages) {
        stage = 0;
        phase ^= 1u;
      }
    }
    asm volatile("bar.sync 2, %0;" ::"n"((kEpi + 1) * 32) : "memory");  // the epilogue warps have read their last columns
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kFewAccs * NT) : "memory");
    if (SPLIT > 1) cluster_wait();
  } else {
    // scales of the CTA's k-blocks, those of A times that of B; zero behind the last row
    for (int i0 = threadIdx.x; i0 < kbs * NT; i0 += kEpi * 32 * 4) {
      float s[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * kEpi * 32, c = i / kbs, b = i - c * kbs;
        s[u] = i < kbs * NT && m0 + c < p.m ? __ldg(p.a_scale + (int64_t)(m0 + c) * p.a_scale_stride + kb0 + b) *
                                                  __ldg(p.b_scale + (int64_t)n_tile * p.b_scale_stride + kb0 + b)
                                            : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * kEpi * 32, c = i / kbs, b = i - c * kbs;
        if (i < kbs * NT) s_scale[b * NT + c] = s[u];
      }
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kEpi * 32) : "memory");
    const int quarter = warp & 3, c0 = (warp >> 2) * kCols;
    const uint32_t t_row = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)c0;
    float acc[kCols];
#pragma unroll
    for (int c = 0; c < kCols; ++c) acc[c] = 0.0f;
    bool ok = true;
    for (int i = 0; i < kbs && ok; ++i) {
      const int buf = i % kFewAccs;
      ok = product_warp_wait(smem_u32(&ctl->acc_full[buf]), (uint32_t)(i / kFewAccs) & 1u, abort_flag);
      if (!ok) break;
      tc_fence_after();
      constexpr int kPiece = kCols < 32 ? kCols : 32;
#pragma unroll
      for (int cc = 0; cc < kCols; cc += kPiece) {
        uint32_t v[kPiece / 16][16];
#pragma unroll
        for (int q = 0; q < kPiece / 16; ++q) tmem_ld16(t_row + (uint32_t)(buf * NT + cc + q * 16), v[q]);
        tmem_ld_wait();
        if (cc + kPiece == kCols) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&ctl->acc_empty[buf]));
        }
        const float4* const sc = reinterpret_cast<const float4*>(s_scale + i * NT + c0 + cc);
#pragma unroll
        for (int q = 0; q < kPiece / 4; ++q) {
          const float4 s = sc[q];
          acc[cc + 4 * q] = fmaf(__uint_as_float(v[q / 4][(4 * q) % 16]), s.x, acc[cc + 4 * q]);
          acc[cc + 4 * q + 1] = fmaf(__uint_as_float(v[q / 4][(4 * q + 1) % 16]), s.y, acc[cc + 4 * q + 1]);
          acc[cc + 4 * q + 2] = fmaf(__uint_as_float(v[q / 4][(4 * q + 2) % 16]), s.z, acc[cc + 4 * q + 2]);
          acc[cc + 4 * q + 3] = fmaf(__uint_as_float(v[q / 4][(4 * q + 3) % 16]), s.w, acc[cc + 4 * q + 3]);
        }
      }
    }
    tc_fence_before();
    asm volatile("bar.arrive 2, %0;" ::"n"((kEpi + 1) * 32) : "memory");
    if (!ok) {
#pragma unroll
      for (int c = 0; c < kCols; ++c) acc[c] = __int_as_float(0x7fffffff);
    }
    if (SPLIT > 1) cluster_wait();  // (every CTA runs)
    send_columns<NT, SPLIT>(acc, sums, rank, c0, quarter * 32 + lane);
  }
  __syncwarp();
  if (SPLIT > 1) {
    cluster_arrive();
    cluster_wait();  // everything has arrived, and nobody reads or writes another CTA's shared memory from here on
  } else {
    __syncthreads();
  }
  if (warp < kEpi) join_columns<NT, SPLIT>(p, reinterpret_cast<const float*>(smem_raw + (sums - smem0)), rank, warp, lane, m0, n0);
}

// ---- many rows of A: pairs of CTAs -------------------------------------------------------------
constexpr int kManyEpiWarps = 8, kManyProducer = 8, kManyMma = 9, kManyThreads = 12 * 32;
// Registers a thread: 168 at launch (12 warps), of which the third warpgroup gives to the two that accumulate.
constexpr int kManyRegs = 168, kManyFewRegs = 56, kManyEpiRegs = 224;
static_assert(4 * kManyFewRegs + 8 * kManyEpiRegs == 12 * kManyRegs, "what one warpgroup gives the others take");
// An SM has 65536: beside a CTA of this kernel there is room for 1024, less than any CTA takes that uses tensor memory (six warps and more).
static_assert(65536 - kManyThreads * kManyRegs < 6 * 32 * 16, "no second CTA with tensor memory on the SM");
constexpr int kManyStages = 4, kManyRows = 256, kManyCols = 256;  // of a pair's tile
constexpr uint32_t kManyStage = 2 * kWTile;
constexpr uint32_t kManyOut = 8192;  // staging of a warp's results: 32 rows x 128 bytes, twice

struct __align__(16) ProductManyCtl {
  unsigned long long full[kManyStages];   // in the first CTA: both CTAs' copies
  unsigned long long empty[kManyStages];  // in both
  unsigned long long acc_full[2];         // in both
  unsigned long long acc_empty[2];        // in the first CTA: the epilogue warps of both
  unsigned long long add_full[kManyEpiWarps];  // a warp's rows of D
  uint32_t tmem_base;
  int abort;
};
constexpr uint32_t kManySmem = 1024 + kManyStages * kManyStage + kManyEpiWarps * kManyOut + 1024;
static_assert(sizeof(ProductManyCtl) <= 1024, "control block");

// The tiles are dealt out in turn (tile t to pair t mod pairs), along a row of C first (the other way 1 % slower).
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kManyThreads, 1)
product_pair_kernel(const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a,
                    const __grid_constant__ CUtensorMap map_out, const __grid_constant__ CUtensorMap map_add,
                    const __grid_constant__ ProductArgs p, int bulk_out) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  ProductManyCtl* const ctl = reinterpret_cast<ProductManyCtl*>(smem_raw);
  const uint32_t ring = (smem_u32(smem_raw) + sizeof(ProductManyCtl) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_cta_rank();
  const int pair = (int)blockIdx.x >> 1, n_pairs = (int)gridDim.x >> 1;
  const int tiles_n = (p.n + kManyCols - 1) / kManyCols, tiles = (p.m + kManyRows - 1) / kManyRows * tiles_n;
  const int kbs = p.k_blocks;
  volatile int* const abort_flag = &ctl->abort;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kManyStages; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(smem_u32(&ctl->acc_full[s]), 1);
      mbar_init(smem_u32(&ctl->acc_empty[s]), 2 * kManyEpiWarps);
    }
    for (int s = 0; s < kManyEpiWarps; ++s) mbar_init(smem_u32(&ctl->add_full[s]), 1);
    ctl->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == kManyProducer && lane == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_b)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_a)) : "memory");
  }
  griddep_wait();
  // All of tensor memory: the registers leave no room on the SM for another CTA that takes any (shared memory would: product_few_kernel<16>
  // with one k-block needs 29 KB).  Were there one, it would be waited for and not the other way round: whoever holds tensor memory gives it
  // back without waiting for another kernel.
  if (warp == kManyMma) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  griddep_launch_dependents();
  const uint32_t tmem = ctl->tmem_base;
  const uint32_t full_on_first = map_to_cta(smem_u32(&ctl->full[0]), 0), acc_empty_on_first = map_to_cta(smem_u32(&ctl->acc_empty[0]), 0);

  if (warp >= kManyEpiWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kManyFewRegs));
  if (warp == kManyProducer) {
    bool ok = true;
    int stage = 0;
    uint32_t phase = 0;
    for (int tile = pair; tile < tiles && ok; tile += n_pairs) {
      const int row_a = (tile / tiles_n) * kManyRows + (int)rank * 128, row_b = (tile % tiles_n) * kManyCols + (int)rank * 128;
      for (int kb = 0; kb < kbs; ++kb) {
        ok = product_warp_wait(smem_u32(&ctl->empty[stage]), phase ^ 1u, abort_flag);
        if (!ok) break;
        if (elect_one()) {
          const uint32_t bar = full_on_first + (uint32_t)stage * 8u, dst = ring + (uint32_t)stage * kManyStage;
          if (rank == 0) mbar_expect_tx(smem_u32(&ctl->full[stage]), 2 * kManyStage);
          tma_load_2d_pair(&map_a, dst, bar, kb * 128, row_a);
          tma_load_2d_pair(&map_b, dst + kWTile, bar, kb * 128, row_b);
        }
        __syncwarp();
        if (++stage == kManyStages) {
          stage = 0;
          phase ^= 1u;
        }
      }
    }
    if (!ok) {  // let copies already issued land before the CTA's shared memory is released
      const unsigned long long t0 = globaltimer();
      while (globaltimer() - t0 < 2000000ull) {
      }
    }
  } else if (warp == kManyMma && rank == 0) {
    const uint64_t a_desc0 = make_smem_desc(ring), b_desc0 = make_smem_desc(ring + kWTile);
    const uint32_t idesc = make_idesc_pair_e4m3(kManyCols);
    bool ok = true;
    int stage = 0, buf = 0;
    uint32_t phase = 0, acc_phase = 0;
    for (int tile = pair; tile < tiles && ok; tile += n_pairs)
      for (int kb = 0; kb < kbs; ++kb) {
        ok = product_warp_wait(smem_u32(&ctl->full[stage]), phase, abort_flag) &&
             product_warp_wait(smem_u32(&ctl->acc_empty[buf]), acc_phase ^ 1u, abort_flag);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t off = (uint64_t)((uint32_t)stage * (kManyStage >> 4));
          const uint32_t d = tmem + (uint32_t)(buf * kManyCols);
          tc_mma_pair_e4m3<false>(d, a_desc0 + off, b_desc0 + off, idesc);
#pragma unroll
          for (int k = 1; k < 4; ++k) tc_mma_pair_e4m3<true>(d, a_desc0 + off + k * 2, b_desc0 + off + k * 2, idesc);
          tc_commit_pair(smem_u32(&ctl->acc_full[buf]), 3u);
          tc_commit_pair(smem_u32(&ctl->empty[stage]), 3u);
        }
        __syncwarp();
        if (++stage == kManyStages) {
          stage = 0;
          phase ^= 1u;
        }
        buf ^= 1;
        if (buf == 0) acc_phase ^= 1u;
      }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyEpiRegs));
    // warp w: lane quarter w mod 4, the block of 128 columns w / 4
    const int quarter = warp & 3, half = warp >> 2;
    const uint32_t t_row = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 128);
    const uint32_t stage_out = ring + kManyStages * kManyStage + (uint32_t)warp * kManyOut;
    bool ok = true, ready = false;
    int buf = 0;
    uint32_t acc_phase = 0, add_phase = 0;
    for (int tile = pair; tile < tiles; tile += n_pairs) {
      const int row = (tile / tiles_n) * kManyRows + (int)rank * 128 + quarter * 32 + lane;
      const int col0 = (tile % tiles_n) * kManyCols + half * 128;
      if (bulk_out && p.add != nullptr && lane == 0 && ok) {  // the tile's rows of D are fetched into the staging beside its products
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        const uint32_t bar = smem_u32(&ctl->add_full[warp]);
        mbar_expect_tx(bar, kManyOut);
        tma_load_2d(&map_add, stage_out, bar, col0, row);
        tma_load_2d(&map_add, stage_out + 4096u, bar, col0 + 64, row);
      }
      const float* const sa = p.a_scale + (int64_t)min(row, p.m - 1) * p.a_scale_stride;
      const float* const sb = p.b_scale + (int64_t)(min(col0, p.n - 1) / 128) * p.b_scale_stride;
      float acc[128];
#pragma unroll
      for (int c = 0; c < 128; ++c) acc[c] = 0.0f;
      // scales, fetched two k-blocks ahead (the shared memory leaves little L1: they come from L2)
      float s_a = __ldg(sa), s_b = __ldg(sb), next_a = __ldg(sa + min(1, kbs - 1)), next_b = __ldg(sb + min(1, kbs - 1));
      for (int kb = 0; kb < kbs && ok; ++kb) {
        const float s = s_a * s_b;
        s_a = next_a;
        s_b = next_b;
        next_a = __ldg(sa + min(kb + 2, kbs - 1));
        next_b = __ldg(sb + min(kb + 2, kbs - 1));
        // 64 columns, then 64: the buffer is handed back before its last ones are added, and the next one's barrier is asked
        // meanwhile (an answer takes 100 cycles even where it is yes)
        if (!ready) ok = product_warp_wait(smem_u32(&ctl->acc_full[buf]), acc_phase, abort_flag);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t v[64];
          tmem_ld64(t_row + (uint32_t)(buf * kManyCols + q * 64), v);
          tmem_ld_wait();
          if (q == 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster_relaxed(acc_empty_on_first + (uint32_t)buf * 8u);
            buf ^= 1;
            if (buf == 0) acc_phase ^= 1u;
            ready = mbar_test(smem_u32(&ctl->acc_full[buf]), acc_phase);
          }
#pragma unroll
          for (int c = 0; c < 64; ++c) acc[q * 64 + c] = fmaf(__uint_as_float(v[c]), s, acc[q * 64 + c]);
        }
        ready = __all_sync(0xffffffffu, ready);
      }
      if (!ok) {
#pragma unroll
        for (int c = 0; c < 128; ++c) acc[c] = __int_as_float(0x7fffffff);
      }
      if (bulk_out && p.add != nullptr) {
        ok = product_warp_wait(smem_u32(&ctl->add_full[warp]), add_phase, abort_flag) && ok;
        add_phase ^= 1u;
#pragma unroll
        for (int c = 0; c < 128; c += 8) {
          float w[8];
          unpack8(lds128(stage_out + (uint32_t)(c / 64) * 4096u + (uint32_t)lane * 128u + (uint32_t)((((c & 63) / 8) ^ (lane & 7)) * 16)), w);
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[c + j] += w[j];
        }
        __syncwarp();
      }
      if (bulk_out) {
        // rows of 128 bytes, 16-byte pieces where the 128-byte swizzle wants them; a piece of 64 bf16 or 32 fp32 columns at a time
        const int row0 = row - lane;
#pragma unroll
        for (int round = 0; round < 2; ++round) {  // of two pieces, the staging's two halves
          if (round == 1 && !p.out_fp32) break;
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the stores before have been read
          __syncwarp();
#pragma unroll
          for (int piece = 0; piece < 2; ++piece) {
            const uint32_t line = stage_out + (uint32_t)piece * 4096u + (uint32_t)lane * 128u;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              uint32_t w[4];
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                if (p.out_fp32) {
                  w[q] = __float_as_uint(acc[(round * 2 + piece) * 32 + j * 4 + q]);
                } else {
                  const __nv_bfloat162 h = __floats2bfloat162_rn(acc[piece * 64 + j * 8 + 2 * q], acc[piece * 64 + j * 8 + 2 * q + 1]);
                  w[q] = *reinterpret_cast<const uint32_t*>(&h);
                }
              }
              asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(line + (uint32_t)((j ^ (lane & 7)) * 16)), "r"(w[0]), "r"(w[1]),
                           "r"(w[2]), "r"(w[3])
                           : "memory");
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0 && row0 < p.m) {  // (rows and columns behind the end are left as they are)
#pragma unroll
            for (int piece = 0; piece < 2; ++piece) {
              const int col = col0 + (p.out_fp32 ? (round * 2 + piece) * 32 : piece * 64);
              if (col < p.n)
                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(&map_out),
                             "r"(stage_out + (uint32_t)piece * 4096u), "r"(col), "r"(row0)
                             : "memory");
            }
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        }
      } else {
        // rows of C anywhere: 64 fp32 columns at a time through the staging, then row by row, a warp's 32 elements next to each other
        // (stored by the lanes that hold them, 2352 x 687 x 2768 took 47 us, this way 19)
        const int row0 = row - lane;
#pragma unroll
        for (int round = 0; round < 2; ++round) {
          __syncwarp();
#pragma unroll
          for (int j = 0; j < 16; ++j)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(stage_out + (uint32_t)(j / 8) * 4096u + (uint32_t)lane * 128u +
                                                                         (uint32_t)(((j & 7) ^ (lane & 7)) * 16)),
                         "f"(acc[round * 64 + j * 4]), "f"(acc[round * 64 + j * 4 + 1]), "f"(acc[round * 64 + j * 4 + 2]),
                         "f"(acc[round * 64 + j * 4 + 3])
                         : "memory");
          __syncwarp();
          const float* const staged = reinterpret_cast<const float*>(smem_raw + (stage_out - smem_u32(smem_raw)));
#pragma unroll 1
          for (int i0 = 0; i0 < 64; i0 += 8) {
            float v[8], d[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int r = (i0 + u) >> 1, c = col0 + round * 64 + (u & 1) * 32 + lane;
              v[u] = staged[(u & 1) * 1024 + r * 32 + ((lane >> 2) ^ (r & 7)) * 4 + (lane & 3)];
              d[u] = 0.0f;
              if (p.add != nullptr && row0 + r < p.m && c < p.n)
                d[u] = __uint_as_float((uint32_t)p.add[(int64_t)(row0 + r) * p.add_stride + c] << 16);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int r = (i0 + u) >> 1, c = col0 + round * 64 + (u & 1) * 32 + lane;
              if (row0 + r < p.m && c < p.n) {
                if (p.out_fp32) static_cast<float*>(p.out)[(int64_t)(row0 + r) * p.out_stride + c] = v[u] + d[u];
                else
                  static_cast<uint16_t*>(p.out)[(int64_t)(row0 + r) * p.out_stride + c] = __bfloat16_as_ushort(__float2bfloat16_rn(v[u] + d[u]));
              }
            }
          }
        }
      }
    }
    if (bulk_out && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  // nobody leaves while the partner may still read this CTA's shared memory or arrive on its barriers
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == kManyMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

constexpr size_t kProductSmem = 222 * 1024;

bool byte_map(CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t stride, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
  const cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  return encode_tensor_map(m, 2, base, dims, strides, box, true);
}

// C or D in pieces of 32 rows x 128 bytes
bool rows_map(CUtensorMap* m, void* base, const ProductArgs& p, int64_t stride, bool fp32) {
  const cuuint64_t item = fp32 ? 4 : 2;
  const cuuint64_t dims[2] = {(cuuint64_t)p.n, (cuuint64_t)p.m}, strides[1] = {(cuuint64_t)stride * item};
  const cuuint32_t box[2] = {(cuuint32_t)(128 / item), 32};
  return encode_tensor_map(m, 2, base, dims, strides, box, false, false, fp32);
}

template <int NT, int SPLIT>
int launch_few_split(cudaStream_t st, const CUtensorMap& map_b, const CUtensorMap& map_a, const ProductArgs& p) {
  // (per device: the attribute belongs to the kernel of the current context)
  if (cudaFuncSetAttribute(product_few_kernel<NT, SPLIT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kProductSmem) != cudaSuccess)
    return OLED_ERR_CUDA;
  const int tiles_n = (p.n + 127) / 128, tiles_m = (p.m + NT - 1) / NT, kbs = (p.k_blocks + SPLIT - 1) / SPLIT;
  constexpr size_t kStage = kWTile + NT * 128;
  const size_t fixed = sizeof(ProductFewCtl) + (size_t)kbs * NT * 4 + (size_t)NT * 512 + 2048;
  const int stages = (int)std::min<size_t>({(size_t)kFewStages, (size_t)kbs, (kProductSmem - fixed) / kStage});
  const cudaError_t err = launch_cluster(product_few_kernel<NT, SPLIT>, dim3((unsigned)(tiles_n * SPLIT), (unsigned)tiles_m),
                                         dim3((few_epi_warps(NT) + 2) * 32), fixed + stages * kStage, st, SPLIT, map_b, map_a, p, stages);
  return err == cudaSuccess ? OLED_OK : OLED_ERR_CUDA;
}
template <int NT>
int launch_few(cudaStream_t st, const CUtensorMap& map_b, const CUtensorMap& map_a, const ProductArgs& p) {
  const int64_t tiles = (int64_t)((p.n + 127) / 128) * ((p.m + NT - 1) / NT);
  // as many CTAs to a tile as run at once: 74 clusters of two, 33 of four, 15 of eight (a GPC has 16 to 20 SMs, and an SM room for
  // one CTA; 128 x 128 t x 2048: t = 15 6.4 us, t = 16 in eights 10.7, in fours 6.5)
  int split = tiles <= 15 ? 8 : tiles <= 33 ? 4 : tiles <= 74 ? 2 : 1;
  while (split > p.k_blocks) split /= 2;
  switch (split) {
    case 1: return launch_few_split<NT, 1>(st, map_b, map_a, p);
    case 2: return launch_few_split<NT, 2>(st, map_b, map_a, p);
    case 4: return launch_few_split<NT, 4>(st, map_b, map_a, p);
    default: return launch_few_split<NT, 8>(st, map_b, map_a, p);
  }
}

int launch_pair(cudaStream_t st, const CUtensorMap& map_b, const CUtensorMap& map_a, const ProductArgs& p) {
  if (cudaFuncSetAttribute(product_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kManySmem) != cudaSuccess)
    return OLED_ERR_CUDA;
  const int64_t item = p.out_fp32 ? 4 : 2;
  CUtensorMap map_out = map_a, map_add = map_a;
  // (a bulk store writes whole 16-byte pieces, also of one that ends behind the last column)
  const bool bulk = !off_boundary(p.out, 16) && p.out_stride * item % 16 == 0 && p.n * item % 16 == 0 && (p.add == nullptr || p.vec_add);
  if (bulk && !rows_map(&map_out, p.out, p, p.out_stride, p.out_fp32)) return OLED_ERR_CUDA;
  if (bulk && p.add != nullptr && !rows_map(&map_add, const_cast<uint16_t*>(p.add), p, p.add_stride, false)) return OLED_ERR_CUDA;
  const int tiles = (p.m + kManyRows - 1) / kManyRows * ((p.n + kManyCols - 1) / kManyCols);
  const int pairs = std::min(tiles, 148 / 2);
  const cudaError_t err = launch_pdl(product_pair_kernel, dim3((unsigned)(2 * pairs)), dim3(kManyThreads), kManySmem, st, map_b, map_a, map_out, map_add, p,
                                     bulk ? 1 : 0);
  return err == cudaSuccess ? OLED_OK : OLED_ERR_CUDA;
}

}  // namespace

int matmul_blocks(const oled_product_shape* shape, const void* a, const float* a_scale, const void* b, const float* b_scale,
                     const void* add, int32_t m, cudaStream_t st, void* out) {
  if (!shape) return OLED_ERR_INVALID_ARG;
  const oled_product_shape& s = *shape;
  if (s.n <= 0 || s.n > (1 << 20) || s.k <= 0 || s.k > OLED_MAX_PRODUCT_K || s.k % 16 != 0 || (s.out != OLED_BF16 && s.out != OLED_FP32) || m < 0)
    return OLED_ERR_INVALID_ARG;
  const int kb = (s.k + 127) / 128, nb = (s.n + 127) / 128;
  if (!stride_ok(s.a_stride, s.k) || s.a_stride % 16 != 0 || !stride_ok(s.b_stride, s.k) || s.b_stride % 16 != 0 ||
      !stride_ok(s.a_scale_stride, kb) || !stride_ok(s.b_scale_stride, kb) || !stride_ok(s.out_stride, s.n) || (add && !stride_ok(s.add_stride, s.n)))
    return OLED_ERR_INVALID_ARG;
  if (m > OLED_MAX_ROUTE_TOKENS) return OLED_ERR_TOO_MANY_TOKENS;
  if (m == 0) return OLED_OK;
  const int64_t item = s.out == OLED_FP32 ? 4 : 2;
  if (!a || !a_scale || !b || !b_scale || !out || off_boundary(a, 16) || off_boundary(b, 16) || off_boundary(a_scale, 4) ||
      off_boundary(b_scale, 4) || off_boundary(add, 2) || off_boundary(out, item))
    return OLED_ERR_INVALID_ARG;
  {
    const RowRange o{out, s.out_stride * item, s.n * item, m}, d{add, s.add_stride * 2, (int64_t)s.n * 2, m};
    const RowRange in[] = {{a, s.a_stride, s.k, m}, {a_scale, s.a_scale_stride * 4, kb * 4, m}, {b, s.b_stride, s.k, s.n}, {b_scale, s.b_scale_stride * 4, kb * 4, nb}};
    for (const RowRange& r : in)
      if (rows_overlap(o, r)) return OLED_ERR_INVALID_ARG;
    if (!same_rows(o, d) && rows_overlap(o, d)) return OLED_ERR_INVALID_ARG;  // (in place: an element is read before it is written)
  }
  ProductArgs p;
  p.a_scale = a_scale;
  p.b_scale = b_scale;
  p.add = static_cast<const uint16_t*>(add);
  p.out = out;
  p.a_scale_stride = s.a_scale_stride;
  p.b_scale_stride = s.b_scale_stride;
  p.add_stride = s.add_stride;
  p.out_stride = s.out_stride;
  p.m = m;
  p.n = s.n;
  p.k_blocks = kb;
  p.out_fp32 = s.out == OLED_FP32;
  p.vec_add = !off_boundary(add, 16) && s.add_stride % 8 == 0;
  p.vec = !off_boundary(out, 4 * item) && s.out_stride % 4 == 0 && (!add || (!off_boundary(add, 8) && s.add_stride % 4 == 0));
  CUtensorMap map_a, map_b;
  // Many rows go to pairs of CTAs once their tiles fill the GPU.  Tiles of 128 x 128 in one wave are faster (512 x 1024 x 4096: 8.3 us, pairs
  // 17.0; 1000 x 2048 x 1024: 7.6 / 8.3) up to where they are not split and go through many k-blocks (512 x 4096 x 4096: 19.4 / 18.1),
  // in two waves slower (640 x 4096 x 2048: 20.8 / 11.6; 160 x 16384 x 1024: 12.9 / 8.4).  Up to 64 rows the weights count alone.
  const int64_t tiles = (int64_t)((m + 127) / 128) * nb;
  if (m > 64 && tiles > (kb <= 16 ? 148 : 74)) {
    if (!byte_map(&map_a, a, m, s.k, s.a_stride, 128) || !byte_map(&map_b, b, s.n, s.k, s.b_stride, 128)) return OLED_ERR_CUDA;
    const int rc = launch_pair(st, map_b, map_a, p);
    return cudaGetLastError() == cudaSuccess ? rc : OLED_ERR_CUDA;
  }
  const int nt = m <= 16 ? 16 : m <= 32 ? 32 : m <= 64 ? 64 : 128;
  if (!byte_map(&map_a, a, m, s.k, s.a_stride, nt) || !byte_map(&map_b, b, s.n, s.k, s.b_stride, 128)) return OLED_ERR_CUDA;
  int rc;
  switch (nt) {
    case 16: rc = launch_few<16>(st, map_b, map_a, p); break;
    case 32: rc = launch_few<32>(st, map_b, map_a, p); break;
    case 64: rc = launch_few<64>(st, map_b, map_a, p); break;
    default: rc = launch_few<128>(st, map_b, map_a, p); break;
  }
  return cudaGetLastError() == cudaSuccess ? rc : OLED_ERR_CUDA;
}

}  // namespace oled

extern "C" int oled_matmul_blocks(const oled_product_shape* shape, const void* a, const float* a_scale, const void* b,
                                     const float* b_scale, const void* add, int32_t m, void* cuda_stream, void* out) {
  return oled::matmul_blocks(shape, a, a_scale, b, b_scale, add, m, static_cast<cudaStream_t>(cuda_stream), out);
}
