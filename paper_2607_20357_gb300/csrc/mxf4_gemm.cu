// C[m, n] = f[m] * sum_k A[m, k] B[n, k] + R[m, n] for MXFP4 operands (mxf4.cuh)
// on the block-scaled tensor cores (tcgen05 kind::mxf4): codes and scales go
// from global to shared memory by TMA and bulk copies, the scales on to tensor
// memory by tcgen05.cp, and the accumulator (float32) is in tensor memory.
//
// Tile kernel: a CTA computes 128 rows of B by up to 256 rows of A (the rows of
// B, a weight's output channels, are the MMA's M: batches of a few rows then pay
// for 16 columns, not 128 rows), or, in a cluster of `split` CTAs, a share of
// that tile's K; the shares are added through distributed shared memory in the
// order of the CTAs, so that results do not depend on timing.
//
// No CTA waits for another while it holds tensor memory, so CTAs of several
// calls that share an SM cannot wait for each other in a circle.
#include <algorithm>

#include "mxf4.cuh"

namespace svl {

constexpr int kMxK = 256;          // values of K per stage: a 128-byte swizzled row of codes
constexpr int kMxW = 128;          // rows of B per tile (TMEM lanes)
constexpr int kMxXMax = 256;       // most rows of A per tile (TMEM columns)
constexpr int kMxWBytes = kMxW * 128;
constexpr int kMxWScales = 2 * kMxTileBytes;  // scales of 128 rows in a stage
constexpr int kMxMaxStages = 12;
constexpr int kMxGemmThreads = 224;  // warp 0 loads B, warp 6 A, warp 1 MMAs, warps 2-5 epilogue
constexpr int kMxBars = 1024;        // bytes of barriers behind the stages

struct Mxf4Params {
  CUtensorMap map_w, map_x;  // codes of B (boxes of 128 rows) and A (boxes of nt rows)
  Mxf4Gemm g;
  int nt;      // rows of A per tile, a multiple of 16
  int split;   // CTAs of a cluster, each with a share of K
  int stages, stage_bytes;
  int x_tiles;
  uint32_t tmem_cols;
};

// The launch's work of this CTA.
struct Mxf4Tile {
  int n0, m0;
  int s0, s1;  // stages of K
  int x_chunks;  // scale tiles of the A rows that exist in the tile (1 or 2)
};
SVL_DEVINL Mxf4Tile mxf4_tile(const Mxf4Params& p) {
  Mxf4Tile t;
  const int id = blockIdx.x / p.split, part = blockIdx.x - id * p.split;
  const int w = id / p.x_tiles;
  t.n0 = w * kMxW;
  t.m0 = (id - w * p.x_tiles) * p.nt;
  const int64_t all = (static_cast<int64_t>(p.g.K) + kMxK - 1) / kMxK;
  t.s0 = static_cast<int>(all * part / p.split);
  t.s1 = static_cast<int>(all * (part + 1) / p.split);
  t.x_chunks = min(p.nt, p.g.M - t.m0) > 128 ? 2 : 1;
  return t;
}

// Scale tiles (of 128 columns) in stage s.
SVL_DEVINL int stage_k_tiles(int K, int s) { return K - s * kMxK > 128 ? 2 : 1; }

// One thread loads B (OP 0), one A (OP 1). Stage: codes of B, codes of A, scales of
// B [k tile], scales of A [chunk of 128 rows][k tile].
template <int OP>
SVL_DEVINL void mx_producer(const Mxf4Params& p, uint8_t* stages, uint64_t* full, uint64_t* empty, volatile int* abort) {
  const Mxf4Tile t = mxf4_tile(p);
  const int64_t tiles = mxf4_scale_tiles(p.g.K);
  int slot = 0;
  uint32_t ph = 1;
  for (int s = t.s0; s < t.s1; ++s) {
    if (!mbar_wait(&empty[slot], ph, abort)) return mx_abort(abort, p.g.status);
    uint8_t* st = stages + slot * p.stage_bytes;
    const uint32_t sbytes = stage_k_tiles(p.g.K, s) * kMxTileBytes;
    if constexpr (OP == 0) {
      mbar_arrive_expect_tx(&full[slot], kMxWBytes + sbytes);
      tma_load_2d(st, &p.map_w, &full[slot], s * 128, t.n0);
      bulk_load(st + kMxWBytes + p.nt * 128, p.g.b_scale + ((t.n0 >> 7) * tiles + 2 * s) * kMxTileBytes, sbytes,
                &full[slot]);
    } else {
      mbar_arrive_expect_tx(&full[slot], p.nt * 128 + t.x_chunks * sbytes);
      tma_load_2d(st + kMxWBytes, &p.map_x, &full[slot], s * 128, t.m0);
      for (int c = 0; c < t.x_chunks; ++c)
        bulk_load(st + kMxWBytes + p.nt * 128 + (1 + c) * kMxWScales,
                  p.g.a_scale + (((t.m0 >> 7) + c) * tiles + 2 * s) * kMxTileBytes, sbytes, &full[slot]);
    }
    if (++slot == p.stages) {
      slot = 0;
      ph ^= 1;
    }
  }
}

SVL_DEVINL void mx_mma(const Mxf4Params& p, uint8_t* stages, uint64_t* full, uint64_t* empty, uint64_t* done,
                       uint32_t tmem, volatile int* abort) {
  const Mxf4Tile t = mxf4_tile(p);
  const uint32_t base = smem_u32(stages), scales = kMxWBytes + p.nt * 128;
  // scales in tensor memory behind the accumulator: B's two k tiles, then A's, each of four columns per 128 rows
  const uint32_t sw = tmem + p.nt, sx = sw + 8;
  const uint32_t id0 = idesc_mxf4(kMxW, p.nt, 0), id1 = idesc_mxf4(kMxW, p.nt, 1);
  int slot = 0;
  uint32_t ph = 0, accumulate = 0;
  for (int s = t.s0; s < t.s1; ++s) {
    if (!mbar_wait(&full[slot], ph, abort)) return mx_abort(abort, p.g.status);
    tc_fence_after();
    const uint32_t st = base + slot * p.stage_bytes;
    const int kt = stage_k_tiles(p.g.K, s);
    for (int j = 0; j < kt; ++j) {
      tc_copy_scales(sw + 4 * j, smem_desc_scales(st + scales + j * kMxTileBytes));
      for (int c = 0; c < t.x_chunks; ++c)
        tc_copy_scales(sx + 8 * j + 4 * c, smem_desc_scales(st + scales + (1 + c) * kMxWScales + j * kMxTileBytes));
    }
    const uint64_t dw = smem_desc_sw128(st), dx = smem_desc_sw128(st + kMxWBytes);
    // 64 values of K an instruction; none behind K's last block
    const int steps = min(4, (p.g.K - s * kMxK + 63) >> 6);
    for (int k = 0; k < steps; ++k) {
      const int j = k >> 1;
      tc_mma_mxf4(tmem, dw + 2 * k, dx + 2 * k, (k & 1) ? id1 : id0, sw + 4 * j, sx + 8 * j, accumulate);
      accumulate = 1;
    }
    tc_commit(&empty[slot]);
    if (++slot == p.stages) {
      slot = 0;
      ph ^= 1;
    }
  }
  tc_commit(done);
}

SVL_DEVINL float mx_residual(const Mxf4Gemm& g, int64_t at) {
  return g.f32 ? static_cast<const float*>(g.residual)[at] : __bfloat162float(static_cast<const __nv_bfloat16*>(g.residual)[at]);
}

// (one rounding: the product and the sum in float32, then C's type)
SVL_DEVINL void mx_store(const Mxf4Gemm& g, int m, int n, float v) {
  if (g.row_factor) v *= g.row_factor[m];
  if (g.residual) v += mx_residual(g, m * g.ld_residual + n);
  const int64_t at = m * g.ld_c + n;
  if (g.f32)
    static_cast<float*>(g.c)[at] = v;
  else
    static_cast<__nv_bfloat16*>(g.c)[at] = __float2bfloat16_rn(v);
}

__global__ void __launch_bounds__(kMxGemmThreads, 1) mxf4_tile_kernel(const __grid_constant__ Mxf4Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(stages + p.stages * p.stage_bytes);
  uint64_t* empty = full + kMxMaxStages;
  uint64_t* done = empty + kMxMaxStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(&full[i], 2);  // the two producers
      mbar_init(&empty[i], 1);
    }
    mbar_init(done, 1);
    *abort = 0;
    fence_barrier_init();
    fence_proxy_async();
    prefetch_tmap(&p.map_w);
    prefetch_tmap(&p.map_x);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, p.tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_begin(false);

  const Mxf4Tile t = mxf4_tile(p);
  float* part = reinterpret_cast<float*>(stages);  // [row of A][128 rows of B], over the stages when they are used up
  if (warp == 0) {
    if (elect_one()) mx_producer<0>(p, stages, full, empty, abort);
  } else if (warp == 6) {
    if (elect_one()) mx_producer<1>(p, stages, full, empty, abort);
  } else if (warp == 1) {
    if (elect_one()) mx_mma(p, stages, full, empty, done, tmem, abort);
  } else {
    const int q = warp & 3, r = q * 32 + lane;  // the lane quarter that this warp may read; its row of B
    const bool ok = mbar_wait(done, 0, abort);
    __syncwarp();
    if (!__all_sync(0xffffffffu, ok)) {
      mx_abort(abort, p.g.status);
    } else {
      tc_fence_after();
      for (int c0 = 0; c0 < p.nt; c0 += 32) {
        float v[32];
        tmem_ld32(tmem + (static_cast<uint32_t>(q * 32) << 16) + c0, v);
        const int cols = min(32, min(p.nt, p.g.M - t.m0) - c0);
        if (p.split > 1) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (j < cols) part[(c0 + j) * kMxW + r] = v[j];
        } else if (t.n0 + r < p.g.N) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (j < cols) mx_store(p.g, t.m0 + c0 + j, t.n0 + r, v[j]);
        }
      }
      tc_fence_before();
    }
  }
  __syncwarp();
  if (*abort) {
    // copies and MMAs already issued land before shared and tensor memory go
    const long long t0 = clock64();
    while (clock64() - t0 < 20000000LL) {
    }
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, p.tmem_cols);
  }
  if (p.split == 1) return;

  // the cluster's shares, added in the order of its CTAs; each CTA adds and stores a part of the tile
  cluster_sync();
  const int rank = static_cast<int>(cluster_rank());
  const int rows = min(p.nt, p.g.M - t.m0);
  for (int i = rank * kMxGemmThreads + threadIdx.x; i < rows * (kMxW / 4); i += p.split * kMxGemmThreads) {
    const int m = i / (kMxW / 4), r = (i - m * (kMxW / 4)) * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c = 0; c < p.split; ++c) {
      const float4 v = ld_cluster4(mapa_shared(part + m * kMxW + r, c));
      sum.x += v.x;
      sum.y += v.y;
      sum.z += v.z;
      sum.w += v.w;
    }
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (t.n0 + r + j < p.g.N) mx_store(p.g, t.m0 + m, t.n0 + r + j, v[j]);
  }
  __syncwarp();
  cluster_sync();  // the others have read this CTA's share
}

cudaError_t launch_mxf4_gemm(const Mxf4Gemm& g, cudaStream_t s) {
  #ifndef PAIR_MIN
#define PAIR_MIN 1024
#endif
  if (g.M >= PAIR_MIN) return launch_mxf4_pair(g, s);
  Mxf4Params p;
  p.g = g;
  p.nt = g.M <= kMxXMax ? (g.M + 15) / 16 * 16 : kMxXMax;
  p.x_tiles = (g.M - 1) / p.nt + 1;
  const int64_t w_tiles = (static_cast<int64_t>(g.N) + kMxW - 1) / kMxW, tiles = w_tiles * p.x_tiles;
  const int64_t k_stages = (static_cast<int64_t>(g.K) + kMxK - 1) / kMxK;
  p.split = 1;
  while (p.split < 8 && tiles * p.split * 2 <= 2 * g.num_sms && k_stages >= 4 * p.split) p.split *= 2;
  if (tiles * p.split > INT32_MAX) return cudaErrorInvalidValue;
  p.stage_bytes = kMxWBytes + p.nt * 128 + kMxWScales * (1 + (p.nt > 128 ? 2 : 1));
  // Batches of up to 64 rows stream their weights: two CTAs per SM, so that one loads while the other starts or ends.
  const int room = (p.nt <= 64 ? 113 * 1024 : 225 * 1024) - kMxBars - 1024;
  p.stages = std::min(kMxMaxStages, room / p.stage_bytes);
  p.tmem_cols = p.nt <= 64 ? 128 : 512;
  const uint64_t bytes = static_cast<uint64_t>(mxf4_row_bytes(g.K));
  if (!make_byte_map(&p.map_w, g.b, g.N, bytes, g.ld_b, kMxW) ||
      !make_byte_map(&p.map_x, g.a, g.M, bytes, g.ld_a, static_cast<uint32_t>(p.nt)))
    return cudaErrorInvalidValue;
  const int smem = p.stages * p.stage_bytes + kMxBars + 1024;
  // (the kernel's limit, not the call's: every call sets the same)
  cudaError_t e = cudaFuncSetAttribute(mxf4_tile_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 225 * 1024);
  if (e != cudaSuccess) return e;
  return launch_pdl_cluster(mxf4_tile_kernel, dim3(static_cast<unsigned>(tiles * p.split)), kMxGemmThreads, smem,
                            p.split, s, p);
}

}  // namespace svl
