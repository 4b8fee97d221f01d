// C[m, n] = f[m] * sum_k A[m, k] B[n, k] + R[m, n] for MXFP4 operands (mxf4.cuh)
// on the block-scaled tensor cores (tcgen05 kind::mxf4): codes and scales go
// from global to shared memory by TMA and bulk copies, the scales on to tensor
// memory by tcgen05.cp, and the accumulator (float32) is in tensor memory.
//
// This is the kernel for up to 128 rows of A; mxf4_pair.cu has the one for more. A
// CTA computes a tile of 128 rows of B by all rows of A. The rows of B, a weight's
// output channels, are the MMA's M and the rows of A its N: a batch of a few rows then
// pays for 16 columns, not for 128 rows. Clusters of up to eight CTAs share a
// tile's K. Each CTA adds up the shares of some of the columns, in the order of the
// CTAs, so that results do not depend on timing. Up to 32 columns travel as
// asynchronous stores into its shared memory, more by bulk copies from one CTA's to
// the other's (a cluster barrier on either side of plain loads took 2,800 of
// the 8,300 cycles of 1 x 4,096 x 4,096).
//
// No CTA waits for another that has not started (a cluster's CTAs start together),
// and two on an SM find tensor memory for both (256 columns at most), so CTAs of
// several calls that share an SM cannot wait in a circle.
#include <algorithm>

#include "mxf4.cuh"

namespace svl {

constexpr int kMxK = 256;  // values of K per stage: a 128-byte swizzled row of codes
constexpr int kMxW = 128;  // rows of B per tile (TMEM lanes)
constexpr int kMxWBytes = kMxW * 128;
constexpr int kMxWScales = 2 * kMxTileBytes;  // scales of 128 rows in a stage
constexpr int kMxMaxX = 128;    // most rows of A
constexpr int kMxStoredX = 32;  // ... whose shares are stored one by one
constexpr int kMxMaxStages = 12;
constexpr int kMxSmem = 225 * 1024;
constexpr int kMxLeastSmem = 76 * 1024;  // three of them do not fit an SM, nor do their registers
constexpr int kMxBars = 1024;            // bytes of barriers behind the stages
// warp 0 loads B's codes, 7 its scales, 6 A, 1 MMAs; all of them see to the results
constexpr int kMxGemmThreads = 256;

struct Mxf4Params {
  CUtensorMap w, x;  // codes of B (boxes of 128 rows) and A (boxes of nt rows)
  Mxf4Gemm g;
  int nt;         // rows of A, rounded up to a multiple of 16
  int log_split;  // CTAs of a cluster, each with a share of K
  int own;        // columns of the accumulator that a CTA adds up, a multiple of 4
  bool stored;    // shares go from CTA to CTA by stores, else by bulk copies
  bool wide;      // four results of a row at a time
  int stages, stage_bytes;
  int shares_at, bars_at;  // bytes from the stages' start
  uint32_t tmem_cols;
};

// The work of this CTA.
struct Mxf4Tile {
  int n0;      // its rows of B
  int part;    // its share of K
  int s0, s1;  // stages of K
};
SVL_DEVINL Mxf4Tile mxf4_tile(const Mxf4Params& p) {
  Mxf4Tile t;
  t.part = blockIdx.x & ((1 << p.log_split) - 1);
  t.n0 = static_cast<int>(blockIdx.x >> p.log_split) * kMxW;
  const int all = ((p.g.K - 1) >> 8) + 1;  // (at most 2^22)
  t.s0 = (all * t.part) >> p.log_split;
  t.s1 = (all * (t.part + 1)) >> p.log_split;
  return t;
}
static_assert(kMxK == 256, "stages of K");

// Scale tiles (of 128 columns) in stage s.
SVL_DEVINL int stage_k_tiles(int K, int s) { return K - s * kMxK > 128 ? 2 : 1; }

enum MxLoad : int { MX_W, MX_W_SCALES, MX_X };

// Three threads load. Stage: codes of B, codes of A, scales of B [k tile], scales of A [k tile].
template <MxLoad OP>
SVL_DEVINL void mx_producer(const Mxf4Params& p, const Mxf4Tile& t, uint8_t* stages, uint64_t* full, uint64_t* empty,
                            volatile int* abort) {
  const int64_t tiles = mxf4_scale_tiles(p.g.K);
  const int x_bytes = p.nt * 128;
  const uint8_t* scales = OP == MX_X ? p.g.a_scale
                                     : p.g.b_scale + (t.n0 >> 7) * tiles * kMxTileBytes;
  scales += static_cast<int64_t>(t.s0) * (2 * kMxTileBytes);
  int slot = 0;
  uint32_t ph = 1;
  pdl_wait();
  for (int s = t.s0; s < t.s1; ++s, scales += 2 * kMxTileBytes) {
    if (s - t.s0 >= p.stages && !mbar_wait(&empty[slot], ph, abort)) return mx_abort(abort, p.g.status);
    uint8_t* st = stages + slot * p.stage_bytes;
    if constexpr (OP == MX_W) {
      mbar_arrive_expect_tx(&full[slot], kMxWBytes);
      tma_load_2d(st, &p.w, &full[slot], s * 128, t.n0);
    } else {
      const uint32_t sbytes = stage_k_tiles(p.g.K, s) * kMxTileBytes;
      uint8_t* to = st + kMxWBytes + x_bytes;
      if constexpr (OP == MX_W_SCALES) {
        mbar_arrive_expect_tx(&full[slot], sbytes);
        bulk_load(to, scales, sbytes, &full[slot]);
      } else {
        mbar_arrive_expect_tx(&full[slot], x_bytes + sbytes);
        tma_load_2d(st + kMxWBytes, &p.x, &full[slot], s * 128, 0);
        bulk_load(to + kMxWScales, scales, sbytes, &full[slot]);
      }
    }
    if (++slot == p.stages) {
      slot = 0;
      ph ^= 1;
    }
  }
}

// One stage's copies of scales and MMAs, 64 values of K each (`steps` of them where
// the stage is not whole). `sw`, `sx`: tensor memory of B's and A's scales, four
// columns a k tile.
template <bool WHOLE>
SVL_DEVINL void mx_stage(uint32_t tmem, uint64_t dw, uint64_t dx, uint64_t ds, uint32_t sw, uint32_t sx, uint32_t id0,
                         uint32_t id1, uint32_t accumulate, int steps) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (!WHOLE && 2 * j >= steps) break;
    tc_copy_scales(sw + 4 * j, ds + j * (kMxTileBytes >> 4));
    tc_copy_scales(sx + 4 * j, ds + ((kMxWScales + j * kMxTileBytes) >> 4));
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (!WHOLE && k >= steps) break;
    tc_mma_mxf4(tmem, dw + 2 * k, dx + 2 * k, (k & 1) ? id1 : id0, sw + 4 * (k >> 1), sx + 4 * (k >> 1),
                k > 0 ? 1u : accumulate);
  }
}

SVL_DEVINL void mx_mma(const Mxf4Params& p, const Mxf4Tile& t, uint8_t* stages, uint64_t* full, uint64_t* empty,
                       uint64_t* done, uint32_t tmem, volatile int* abort) {
  uint32_t sw = tmem + p.nt;  // two sets of scales, used in turn, in tensor memory behind the accumulator
  const uint32_t id0 = idesc_mxf4(kMxW, p.nt, 0), id1 = idesc_mxf4(kMxW, p.nt, 1);
  const uint32_t base = smem_u32(stages);
  const uint64_t dw0 = smem_desc_sw128(base), dx0 = smem_desc_sw128(base + kMxWBytes);
  const uint64_t ds0 = smem_desc_scales(base + kMxWBytes + p.nt * 128);
  const uint32_t step = static_cast<uint32_t>(p.stage_bytes) >> 4;
  int slot = 0;
  uint32_t ph = 0, at = 0, odd = 0;
  for (int s = t.s0; s < t.s1; ++s) {
    if (!mbar_wait(&full[slot], ph, abort)) return mx_abort(abort, p.g.status);
    tc_fence_after();
    const uint32_t accumulate = s > t.s0, sx = sw + 8;
    const int left = p.g.K - s * kMxK;
    if (left >= kMxK)
      mx_stage<true>(tmem, dw0 + at, dx0 + at, ds0 + at, sw, sx, id0, id1, accumulate, 4);
    else  // none behind K's last block
      mx_stage<false>(tmem, dw0 + at, dx0 + at, ds0 + at, sw, sx, id0, id1, accumulate, (left + 63) >> 6);
    tc_commit(&empty[slot]);
    sw = odd ? sw - 16 : sw + 16;
    odd ^= 1;
    at += step;
    if (++slot == p.stages) {
      slot = 0;
      ph ^= 1;
      at = 0;
    }
  }
  tc_commit(done);
}

template <bool F32>
SVL_DEVINL float mx_load(const void* p, int64_t at) {
  return F32 ? static_cast<const float*>(p)[at] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
}
template <bool F32>
SVL_DEVINL void mx_store(void* p, int64_t at, float v) {
  if (F32)
    static_cast<float*>(p)[at] = v;
  else
    static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
}
// The factor and the sum with the residual in float32.
SVL_DEVINL float mx_result(float v, float factor, bool residual, float add) {
  v = __fmul_rn(v, factor);
  return residual ? __fadd_rn(v, add) : v;
}

// Results of rows m0 ... m0 + rows - 1 of A and 128 of B from n0 on: the shares of
// K, [share][row of A][128 rows of B], `stride` floats apart, are added in their
// order. A warp takes a row, four results a lane. What a batch of rows loads is
// requested before its first store, which might be to the residual.
template <bool F32, int SPLIT>
SVL_DEVINL void mx_results(const Mxf4Params& p, const float* shares, int stride, int m0, int rows, int n0) {
  constexpr int kWarps = kMxGemmThreads / 32, kBatch = SPLIT > 2 ? 2 : 4, kSize = F32 ? 4 : 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool resid = p.g.residual != nullptr;
  if (p.wide) {
    if (n0 + 4 * lane >= p.g.N) return;
    const int64_t row_c = kWarps * p.g.ld_c * kSize, row_r = kWarps * p.g.ld_residual * kSize;
    const int64_t m = m0 + warp;
    char* to = static_cast<char*>(p.g.c) + (m * p.g.ld_c + n0 + 4 * lane) * kSize;
    const char* from =
        resid ? static_cast<const char*>(p.g.residual) + (m * p.g.ld_residual + n0 + 4 * lane) * kSize : nullptr;
    const float* factors = p.g.row_factor ? p.g.row_factor + m : nullptr;
    const float4* sums = reinterpret_cast<const float4*>(shares + warp * kMxW) + lane;
    for (int r = warp; r < rows; r += kBatch * kWarps) {
      float4 v[kBatch];
      uint4 x[kBatch];
      float f[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        f[i] = 1.f;
        if (r + i * kWarps >= rows) break;
        if (factors) f[i] = factors[i * kWarps];
        if (resid) {
          if (F32) {
            x[i] = *reinterpret_cast<const uint4*>(from);
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(from);
            x[i].x = w.x, x[i].y = w.y;
          }
          from += row_r;
        }
        float4 w[SPLIT];
#pragma unroll
        for (int c = 0; c < SPLIT; ++c) w[c] = sums[(i * kWarps * kMxW + c * stride) / 4];
        v[i] = w[0];
#pragma unroll
        for (int c = 1; c < SPLIT; ++c) {
          v[i].x = __fadd_rn(v[i].x, w[c].x);
          v[i].y = __fadd_rn(v[i].y, w[c].y);
          v[i].z = __fadd_rn(v[i].z, w[c].z);
          v[i].w = __fadd_rn(v[i].w, w[c].w);
        }
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (r + i * kWarps >= rows) break;
        float add[4] = {0.f, 0.f, 0.f, 0.f};
        if (resid) {
          if (F32) {
            add[0] = __uint_as_float(x[i].x), add[1] = __uint_as_float(x[i].y);
            add[2] = __uint_as_float(x[i].z), add[3] = __uint_as_float(x[i].w);
          } else {
            const float2 lo = unpack_bf16x2(x[i].x), hi = unpack_bf16x2(x[i].y);
            add[0] = lo.x, add[1] = lo.y, add[2] = hi.x, add[3] = hi.y;
          }
        }
        const float o[4] = {mx_result(v[i].x, f[i], resid, add[0]), mx_result(v[i].y, f[i], resid, add[1]),
                            mx_result(v[i].z, f[i], resid, add[2]), mx_result(v[i].w, f[i], resid, add[3])};
        if (F32)
          *reinterpret_cast<float4*>(to) = make_float4(o[0], o[1], o[2], o[3]);
        else
          *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
        to += row_c;
      }
      sums += kBatch * kWarps * kMxW / 4;
      if (factors) factors += kBatch * kWarps;
    }
    return;
  }
  // rows of any alignment: consecutive lanes take consecutive columns
  for (int r = warp; r < rows; r += kWarps) {
    const int64_t m = m0 + r;
    const float f = p.g.row_factor ? p.g.row_factor[m] : 1.f;
    float add[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + lane + 32 * j;
      add[j] = resid && n < p.g.N ? mx_load<F32>(p.g.residual, m * p.g.ld_residual + n) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + lane + 32 * j;
      float v = shares[r * kMxW + lane + 32 * j];
#pragma unroll
      for (int c = 1; c < SPLIT; ++c) v = __fadd_rn(v, shares[c * stride + r * kMxW + lane + 32 * j]);
      if (n < p.g.N) mx_store<F32>(p.g.c, m * p.g.ld_c + n, mx_result(v, f, resid, add[j]));
    }
  }
}


template <bool F32>
__global__ void __launch_bounds__(kMxGemmThreads, 2) mxf4_tile_kernel(const __grid_constant__ Mxf4Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(stages + p.bars_at);
  uint64_t* empty = full + kMxMaxStages;
  uint64_t* done = empty + kMxMaxStages;
  uint64_t* free_bar = done + 1;        // the cluster's CTAs are through with their stages
  uint64_t* arrived = free_bar + 1;     // the shares for this CTA
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(arrived + 1);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const Mxf4Tile t = mxf4_tile(p);
  const int split = 1 << p.log_split;
  const int mine = max(0, min(p.own, p.g.M - t.part * p.own));  // the columns of this CTA that exist
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.stages; ++i) {
      mbar_init(&full[i], 3);  // the three producers
      mbar_init(&empty[i], 1);
    }
    mbar_init(done, 1);
    mbar_init(free_bar, split);
    mbar_init(arrived, 1);
    *abort = 0;
    fence_barrier_init();
    fence_proxy_async();
    if (split > 1) mbar_arrive_expect_tx(arrived, static_cast<uint32_t>((mine + 3) / 4 * split) * kMxW * 16);
  } else if (threadIdx.x == 64) {
    prefetch_tmap(&p.w);
    prefetch_tmap(&p.x);
  }
  __syncwarp();
  if (split > 1) cluster_arrive_relaxed();  // (the first warp behind its barriers' initialisation)
  if (warp == 1) {
    tmem_alloc(tmem_slot, p.tmem_cols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // Not before: the next kernel's CTAs, which keep their tensor memory until this kernel is complete, could take what
  // this CTA still has to get.
  pdl_trigger();

  if (warp == 0) {
    if (elect_one()) mx_producer<MX_W>(p, t, stages, full, empty, abort);
  } else if (warp == 7) {
    if (elect_one()) mx_producer<MX_W_SCALES>(p, t, stages, full, empty, abort);
  } else if (warp == 6) {
    if (elect_one()) mx_producer<MX_X>(p, t, stages, full, empty, abort);
  } else if (warp == 1) {
    if (elect_one()) mx_mma(p, t, stages, full, empty, done, tmem, abort);
  }
  __syncwarp();
  pdl_wait();
  bool ok = mbar_wait(done, 0, abort);
  __syncwarp();
  ok = __all_sync(0xffffffffu, ok);
  if (!ok) mx_abort(abort, p.g.status);
  tc_fence_after();
  if (split > 1) cluster_wait();  // every CTA has its barriers

  // The accumulator's lane quarters are for warps 2-5 and once more for 0, 1, 6 and 7, 32 columns in turn.
  const int q = warp & 3, r = q * 32 + lane, second = warp < 2 || warp > 5 ? 32 : 0;
  const uint32_t acc = tmem + (static_cast<uint32_t>(q * 32) << 16);
  float* shares = reinterpret_cast<float*>(stages + p.shares_at);  // [CTA][its columns][128 rows of B]
  if (p.stored) {
    if (ok && !second) {
      float v[kMxStoredX];
      tmem_ld32(acc, v);
      // [CTA][group of four columns][128 rows of B][4]
      int owner = 0, at = 0;  // of the group of columns, and its place there
      const int groups = p.own >> 2;
      uint32_t to = mapa_shared(shares, 0), bar = mapa_shared(arrived, 0);
#pragma unroll
      for (int j = 0; j < kMxStoredX; j += 4) {
        if (j < p.g.M) {
          st_async4(to + static_cast<uint32_t>(((t.part * groups + at) * kMxW + r) * 16), bar, v + j);
          if (++at == groups) {
            at = 0;
            ++owner;
            to = mapa_shared(shares, owner & (split - 1));
            bar = mapa_shared(arrived, owner & (split - 1));
          }
        }
      }
    }
    // this CTA's columns: a row of B a thread, four columns at a time
    const int b = threadIdx.x & 127, n = t.n0 + b;
    bool here = false;
    for (int g = (threadIdx.x >> 7) * 4; g < mine; g += 8) {
      const int64_t m = t.part * p.own + g;
      float add[4], factor[4], v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool there = g + i < mine && n < p.g.N;
        add[i] = p.g.residual && there ? mx_load<F32>(p.g.residual, (m + i) * p.g.ld_residual + n) : 0.f;
        factor[i] = p.g.row_factor && there ? p.g.row_factor[m + i] : 1.f;
      }
      if (!here && !(here = mbar_wait(arrived, 0, abort))) {
        mx_abort(abort, p.g.status);
        break;
      }
      const float4* from = reinterpret_cast<const float4*>(shares) + (g >> 2) * kMxW + b;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        if (c < split) {
          const float4 x = from[c * (p.own >> 2) * kMxW];
          v[0] = c ? __fadd_rn(v[0], x.x) : x.x;
          v[1] = c ? __fadd_rn(v[1], x.y) : x.y;
          v[2] = c ? __fadd_rn(v[2], x.z) : x.z;
          v[3] = c ? __fadd_rn(v[3], x.w) : x.w;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (g + i < mine && n < p.g.N)
          mx_store<F32>(p.g.c, (m + i) * p.g.ld_c + n, mx_result(v[i], factor[i], p.g.residual != nullptr, add[i]));
    }
    // (Stored shares have left their CTA, and where one adds up nothing, nothing is on its way there: it may end.)
  } else {
    // over the stages, which are used up: [column][128 rows of B]
    float* sums = reinterpret_cast<float*>(stages);
    if (split > 1 && ok && warp == 2 && lane < split) mbar_arrive_cluster_relaxed(mapa_shared(free_bar, lane));
    if (ok) {
      for (int c0 = second; c0 < p.g.M; c0 += 64) {
        float v[32];
        tmem_ld32(acc + c0, v);
        float* to = sums + c0 * kMxW + r;
#pragma unroll
        for (int j = 0; j < 32; j += 16)  // (p.nt is a multiple of 16)
          if (c0 + j < p.nt)
#pragma unroll
            for (int i = j; i < j + 16; ++i) to[i * kMxW] = v[i];
      }
    }
    if (split > 1) fence_proxy_async();  // generic-proxy writes, read by the copies
    __syncthreads();
    if (split > 1) {
      if (warp == 2) {
        const bool free = mbar_wait(free_bar, 0, abort);  // the others' stages are used up
        const int theirs = max(0, min(p.own, p.g.M - lane * p.own) + 3) & ~3;
        if (!free)
          mx_abort(abort, p.g.status);
        else if (lane < split && theirs > 0)
          bulk_to_cluster(mapa_shared(shares, lane) + t.part * p.own * (kMxW * 4), sums + lane * p.own * kMxW,
                          theirs * kMxW * 4, mapa_shared(arrived, lane));
        __syncwarp();
      }
      ok = mbar_wait(arrived, 0, abort);
      if (!ok) mx_abort(abort, p.g.status);
      __syncwarp();
      ok = __all_sync(0xffffffffu, ok);
    }
    if (ok) {
      const int m0 = t.part * p.own, stride = p.own * kMxW;
      switch (split) {
        case 1: mx_results<F32, 1>(p, sums, 0, 0, p.g.M, t.n0); break;
        case 2: mx_results<F32, 2>(p, shares, stride, m0, mine, t.n0); break;
        case 4: mx_results<F32, 4>(p, shares, stride, m0, mine, t.n0); break;
        default: mx_results<F32, 8>(p, shares, stride, m0, mine, t.n0); break;
      }
    }
    __syncwarp();
    if (split > 1) {
      cluster_arrive_relaxed();  // copies from this CTA's shared memory have been made where they have arrived
      cluster_wait();
    }
  }
  tc_fence_before();
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
}

cudaError_t launch_mxf4_gemm(const Mxf4Gemm& g, cudaStream_t s) {
  // More than 64 rows over a short K, where results take most of the time, and more than 96 over one that is not long
  // go to pairs, if one wave of them is enough: us here and there 100 x 5,120 x 256 3.9, 3.4; 128 x 4,096 x 4,096 8.0,
  // 7.7.
  const int k_stages = (g.K - 1) / kMxK + 1;
  if (g.M > kMxMaxX ||
      (((g.M > 64 && k_stages <= 4) || (g.M > 96 && k_stages <= 20)) && (g.N - 1) / 128 < mxf4_clusters(2)))
    return launch_mxf4_pair(g, s);
  Mxf4Params p;
  p.g = g;
  const int nt = (g.M + 15) / 16 * 16;
  const int64_t tiles = (static_cast<int64_t>(g.N) + kMxW - 1) / kMxW;
  p.nt = nt;
  // A cluster shares K while all clusters run at once, an SM to a CTA (up to 16 columns: half an SM), and K has
  // the stages to make up for the sums' way. us for at most 1, 2, 4 CTAs at 4,096 rows of B, K 4,096 (16 stages): 6.3,
  // 5.0, 4.7 for 1 row of A; 6.6, 6.0, 5.3 for 32; 6.8, 6.5, 6.8 for 48; 7.0, 6.9, 7.7 for 64; 7.4, 8.0, 8.2 for 96;
  // 8.0, 9.2, 9.6 for 128. K 2,048: 4.6, 4.0, 3.8; 4.9, 5.2, 4.5; 5.2, 5.9, 6.0; 5.4, 6.6, 6.9; 5.8, 7.2, 9.0; 6.2,
  // 8.3, 8.8. 3,584 and 18,944 (74 stages): 18.4, 11.1, 8.5; 18.6, 12.0, 9.1; 18.9, 12.5, 10.1; 19.0, 13.0, 10.4; 19.7,
  // 14.3, 11.7; 20.7, 15.7, 13.5. Where the rule is off: 96 by 2,048, K 8,192, 10.7, 9.0 (taken), 8.1.
  const int per_cta = nt <= kMxStoredX ? 2 : nt <= 64 ? 10 : 21;
  int split = 1;
  while (split < 8 && k_stages >= per_cta * split && tiles <= (nt <= 16 ? 2 : 1) * mxf4_clusters(2 * split)) split *= 2;
  p.log_split = split == 8 ? 3 : split == 4 ? 2 : split == 2 ? 1 : 0;
  p.own = (nt / split + 3) / 4 * 4;
  p.stage_bytes = kMxWBytes + nt * 128 + 2 * kMxWScales;
  p.stored = split > 1 && nt <= kMxStoredX;
  // Stored shares have room of their own, sums and copied shares lie over the stages. An SM has one CTA with all the
  // stages it can use, or two that need not run one after the other: 64 rows of A by 9,000 of B, K 4,096 (71 CTAs)
  // 8.1 us instead of 9.4 with half the stages, 72 by 22,016 (172 CTAs) 13.0 instead of 17.3.
  const int shares = split > 1 ? split * p.own * kMxW * 4 : 0, share_stages = (k_stages + split - 1) / split;
  const int fixed = kMxBars + 1024 + (p.stored ? shares : 0);
  const bool two = tiles > (split > 1 ? mxf4_clusters(split) : g.num_sms) &&
                   (kMxSmem / 2 - fixed) / p.stage_bytes >= std::min(share_stages, 2);
  const int room = ((two ? kMxSmem / 2 : kMxSmem) - fixed) / p.stage_bytes;
  p.stages = std::min(std::min(kMxMaxStages, share_stages), room);
  const int body = p.stages * p.stage_bytes;
  const int sums = split * p.own * kMxW * 4;
  p.shares_at = p.stored ? body : sums;
  p.bars_at = p.stored ? body + shares : std::max(body, sums + shares);
  const int size = g.f32 ? 4 : 2;
  auto fours = [&](const void* q, int64_t ld) { return !((reinterpret_cast<uintptr_t>(q) | (ld * size)) % (4 * size)); };
  p.wide = g.N % 4 == 0 && fours(g.c, g.ld_c) && (!g.residual || fours(g.residual, g.ld_residual));
  p.tmem_cols = 32;
  while (p.tmem_cols < static_cast<uint32_t>(nt + 32)) p.tmem_cols *= 2;
  const uint64_t bytes = static_cast<uint64_t>(mxf4_row_bytes(g.K));
  if (!make_byte_map(&p.w, g.b, g.N, bytes, g.ld_b, kMxW) ||
      !make_byte_map(&p.x, g.a, g.M, bytes, g.ld_a, static_cast<uint32_t>(nt)))
    return cudaErrorInvalidValue;
  const int smem = std::max(p.bars_at + kMxBars + 1024, kMxLeastSmem);
  void (*kernel)(Mxf4Params) = g.f32 ? mxf4_tile_kernel<true> : mxf4_tile_kernel<false>;
  static std::atomic<uint64_t> devices[2];
  cudaError_t e = mxf4_allow_smem(reinterpret_cast<const void*>(kernel), kMxSmem, &devices[g.f32]);
  if (e != cudaSuccess) return e;
  return launch_pdl_cluster(kernel, dim3(static_cast<unsigned>(tiles * split)), kMxGemmThreads, smem, split,
                            s, p);
}

}  // namespace svl
