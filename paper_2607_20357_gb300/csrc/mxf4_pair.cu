// The MXFP4 product (mxf4.cuh) for many rows: persistent pairs of CTAs, each
// with tiles of 256 rows of A (the MMA's M, 128 a CTA) by 256 rows of B.
//
// A pair issues one tcgen05.mma for both SMs, which read each other's half of B:
// per 64 columns of K an SM loads 8 KB of codes for 128 cycles of MMA, where a
// tile of 128 x 256 on one SM needs 12 KB.
//
// Tensor memory (512 columns a CTA) has two accumulators of 256 columns that
// overlap by as many as the scales take behind them: accumulator 0 is columns
// 0-255, accumulator 1 starts kOverlap columns before 256. The epilogue takes
// those columns first, then the next tile's MMAs start into the other
// accumulator while the rest is converted and stored.
//
// Barriers: full[s] (leader's: both CTAs' loads of stage s have landed), empty[s]
// (in both CTAs: the MMAs have read stage s), done (in both: a tile's MMAs are
// complete), taken (leader's: both epilogues have read the overlap, so the
// tile before is read altogether).
#include <algorithm>

#include "mxf4.cuh"

namespace svl {

constexpr int kPrK = 256;  // values of K per stage: a 128-byte swizzled row of codes
constexpr int kPrTile = 256;
constexpr int kPrCodes = 128 * 128;  // bytes of a CTA's rows of A, or of its half of B's
constexpr int kPrScalesA = 2 * kMxTileBytes;
constexpr int kPrScalesB = 4 * kMxTileBytes;
constexpr int kPrStageBytes = 2 * kPrCodes + kPrScalesA + kPrScalesB;
constexpr int kPrStages = 5;
constexpr int kPrChunk = 32 * 128;  // bytes of an epilogue chunk: 32 rows of 128 bytes
constexpr int kPrChunks = 3;        // buffers of a warp
constexpr int kPrSmem = 1024 + kPrStages * kPrStageBytes + 1024 + 4 * kPrChunks * kPrChunk;
constexpr int kPrThreads = 192;  // warp 0 loads, warp 1 MMAs (leader), warps 2-5 epilogue
constexpr int kPrSets = 2;       // sets of scales in tensor memory, used in turn
constexpr int kPrOverlap = 24 * kPrSets;
constexpr int kPrGroup = 8;  // tiles of rows that are walked together
static_assert(kPrSmem <= 232448, "shared memory per CTA");

struct Mxf4PairParams {
  CUtensorMap a, b, a_scale, b_scale, c, residual;
  Mxf4Gemm g;
  int m_tiles, n_tiles, tiles;
  bool tma;  // C and the residual go by TMA
};

struct PairTile {
  int m0, n0;
};
// Groups of kPrGroup row tiles, column tile by column tile: tiles that run at
// the same time share rows of both operands.
SVL_DEVINL PairTile pair_tile(const Mxf4PairParams& p, int t) {
  const int per = kPrGroup * p.n_tiles, g = t / per, r = t - g * per;
  const int height = min(kPrGroup, p.m_tiles - g * kPrGroup);
  PairTile ti;
  ti.m0 = (g * kPrGroup + r % height) * kPrTile;
  ti.n0 = r / height * kPrTile;
  return ti;
}

SVL_DEVINL int pair_stages(int K) { return (K - 1) / kPrK + 1; }

SVL_DEVINL void mx_pair_producer(const Mxf4PairParams& p, uint8_t* stages, uint64_t* full, uint64_t* empty,
                                 uint32_t rank, volatile int* abort) {
  const int n_stages = pair_stages(p.g.K);
  int s = 0;
  uint32_t ph = 1;
  auto next = [&]() {
    if (++s == kPrStages) {
      s = 0;
      ph ^= 1;
    }
  };
  for (int t = blockIdx.x >> 1; t < p.tiles; t += gridDim.x >> 1) {
    const PairTile ti = pair_tile(p, t);
    const int m0 = ti.m0 + static_cast<int>(rank) * 128, n0 = ti.n0 + static_cast<int>(rank) * 128;
    for (int k = 0; k < n_stages; ++k, next()) {
      if (!mbar_wait(&empty[s], ph, abort)) return mx_abort(abort, p.g.status);
      uint8_t* st = stages + s * kPrStageBytes;
      if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * kPrStageBytes);
      const uint32_t fb = mapa_shared(&full[s], 0);
      tma_load_2d_pair(st, &p.a, fb, k * 128, m0);
      tma_load_2d_pair(st + kPrCodes, &p.b, fb, k * 128, n0);
      tma_load_2d_pair(st + 2 * kPrCodes, &p.a_scale, fb, k * 256, m0 >> 7);
      tma_load_2d_pair(st + 2 * kPrCodes + kPrScalesA, &p.b_scale, fb, k * 256, ti.n0 >> 7);
    }
  }
  // the releases of the last stages (the leader's MMA commits) have arrived here
  for (int i = 0; i < kPrStages; ++i, next())
    if (!mbar_wait(&empty[s], ph, abort)) return mx_abort(abort, p.g.status);
}

SVL_DEVINL uint32_t pair_acc(uint32_t tmem, int it) { return tmem + ((it & 1) ? kPrTile - kPrOverlap : 0); }

SVL_DEVINL void mx_pair_mma(const Mxf4PairParams& p, uint8_t* stages, uint64_t* full, uint64_t* empty, uint64_t* done,
                            uint64_t* taken, uint32_t tmem, volatile int* abort) {
  const int n_stages = pair_stages(p.g.K);
  const uint32_t base = smem_u32(stages);
  constexpr uint32_t id0 = idesc_mxf4(kPrTile, kPrTile, 0), id1 = idesc_mxf4(kPrTile, kPrTile, 1);
  int s = 0, it = 0;
  uint32_t ph = 0, set = 0;
  for (int t = blockIdx.x >> 1; t < p.tiles; t += gridDim.x >> 1, ++it) {
    if (it > 0 && !mbar_wait(taken, (it - 1) & 1, abort)) return mx_abort(abort, p.g.status);
    tc_fence_after();
    const uint32_t d = pair_acc(tmem, it);
    uint32_t accumulate = 0;
    for (int k = 0; k < n_stages; ++k) {
      if (!mbar_wait(&full[s], ph, abort)) return mx_abort(abort, p.g.status);
      tc_fence_after();
      const uint32_t st = base + s * kPrStageBytes, sc = st + 2 * kPrCodes;
      // a set: A's two tiles of 128 columns (4 tensor memory columns each), then B's (8 each)
      const uint32_t sa = tmem + 512 - kPrOverlap + set * 24, sb = sa + 8;
      const int steps = min(4, (p.g.K - k * kPrK + 63) >> 6);  // 64 values of K an instruction
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        if (2 * j < steps) {
          tc_copy_scales_pair(sa + 4 * j, smem_desc_scales(sc + j * kMxTileBytes));
          tc_copy_scales_pair(sb + 8 * j, smem_desc_scales(sc + kPrScalesA + j * kMxTileBytes));
          tc_copy_scales_pair(sb + 8 * j + 4, smem_desc_scales(sc + kPrScalesA + (2 + j) * kMxTileBytes));
        }
      }
      const uint64_t da = smem_desc_sw128(st), db = smem_desc_sw128(st + kPrCodes);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i < steps) {
          tc_mma_mxf4_pair(d, da + 2 * i, db + 2 * i, (i & 1) ? id1 : id0, sa + 4 * (i >> 1), sb + 8 * (i >> 1),
                           accumulate);
          accumulate = 1;
        }
      }
      tc_commit_pair(&empty[s]);
      if (++s == kPrStages) {
        s = 0;
        ph ^= 1;
      }
      if (++set == kPrSets) set = 0;
    }
    tc_commit_pair(done);
  }
}

// The chunks of a warp, over all of its tiles: 128 bytes of 32 rows of C. In
// accumulator 1 they are taken from the left, in accumulator 0 from the right.
template <bool F32>
struct PairChunks {
  static constexpr int kCols = F32 ? 32 : 64;
  const Mxf4PairParams& p;
  int t, it, row0, quarter;  // tile, its number, the warp's first row, its rows' offset in the tile
  int n0, n, i;              // tile's first column, its chunks (0: no rows of the warp exist), the present one
  SVL_DEVINL PairChunks(const Mxf4PairParams& params, int offset) : p(params), quarter(offset) {
    t = blockIdx.x >> 1;
    it = 0;
    enter();
  }
  SVL_DEVINL void enter() {
    i = 0;
    n = 0;
    if (t >= p.tiles) return;
    const PairTile ti = pair_tile(p, t);
    row0 = ti.m0 + quarter;
    n0 = ti.n0;
    if (row0 < p.g.M) n = (min(kPrTile, p.g.N - n0) + kCols - 1) / kCols;
  }
  SVL_DEVINL void next_tile() {
    t += gridDim.x >> 1;
    ++it;
    enter();
  }
  // the next chunk there is, in this tile or a later one
  SVL_DEVINL void next_chunk() {
    ++i;
    settle();
  }
  SVL_DEVINL void settle() {
    while (i >= n && t < p.tiles) next_tile();
  }
  SVL_DEVINL bool more() const { return t < p.tiles; }
  SVL_DEVINL int column() const { return ((it & 1) ? i : n - 1 - i) * kCols; }
};

template <bool F32>
SVL_DEVINL void mx_pair_epilogue(const Mxf4PairParams& p, uint64_t* done, uint64_t* taken, uint64_t* loaded,
                                 uint32_t tmem, uint32_t rank, uint8_t* buffers, volatile int* abort) {
  constexpr int kCols = F32 ? 32 : 64;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q = warp & 3;
  uint8_t* mine = buffers + q * kPrChunks * kPrChunk;
  loaded += q * kPrChunks;
  const int offset = static_cast<int>(rank) * 128 + q * 32;
  const uint32_t release = mapa_shared(taken, 0);
  PairChunks<F32> ch(p, offset), ahead(p, offset);
  const bool resid = p.g.residual != nullptr;
  int buf = 0, ahead_buf = 0;  // buffers of the present chunk and of the one that is requested next
  uint32_t parity = 0;         // of each buffer's next wait
  auto request = [&]() {
    if (ahead.more()) {
      mbar_arrive_expect_tx(&loaded[ahead_buf], kPrChunk);
      tma_load_2d(mine + ahead_buf * kPrChunk, &p.residual, &loaded[ahead_buf], ahead.n0 + ahead.column(), ahead.row0);
      ahead_buf = ahead_buf == kPrChunks - 1 ? 0 : ahead_buf + 1;
      ahead.next_chunk();
    }
  };
  if (resid && p.tma) {
    ahead.settle();
    if (lane == 0) {
      request();
      request();
    }
  }
  for (; ch.more(); ch.next_tile()) {
    const int row = ch.row0 + lane;
    const float factor = p.g.row_factor && ch.n > 0 && row < p.g.M ? p.g.row_factor[row] : 1.f;
    const bool ok = mbar_wait(done, ch.it & 1, abort);
    __syncwarp();
    if (!__all_sync(0xffffffffu, ok)) return mx_abort(abort, p.g.status);
    tc_fence_after();
    const uint32_t acc = pair_acc(tmem, ch.it) + (static_cast<uint32_t>(q * 32) << 16);
    // chunks that hold the overlap: where the tile's columns end before it, there is nothing to wait for
    const int in_overlap =
        (ch.it & 1) ? (kPrOverlap + kCols - 1) / kCols : ch.n - (kPrTile - kPrOverlap) / kCols;
    if (ch.n == 0 || in_overlap <= 0) {
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_relaxed(release);
    }
    for (; ch.i < ch.n; ++ch.i) {
      float v[kCols];
      const int col = ch.column();
#pragma unroll
      for (int c = 0; c < kCols; c += 32) tmem_ld32(acc + col + c, v + c);
      if (ch.i + 1 == min(in_overlap, ch.n)) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(release);
      }
      if (p.tma) {
        uint8_t* slot0 = mine + buf * kPrChunk + lane * 128;
        if (resid) {
          const bool got = mbar_wait(&loaded[buf], (parity >> buf) & 1, abort);
          parity ^= 1u << buf;
          __syncwarp();
          if (!__all_sync(0xffffffffu, got)) return mx_abort(abort, p.g.status);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          // 16-byte piece c of the row, where the 128-byte swizzle has it
          uint4* slot = reinterpret_cast<uint4*>(slot0 + ((c ^ (lane & 7)) << 4));
          uint32_t o[4];
          uint4 x = make_uint4(0, 0, 0, 0);
          if (resid) x = *slot;
          const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if constexpr (F32) {
              float w = __fmul_rn(v[4 * c + k], factor);
              if (resid) w = __fadd_rn(w, __uint_as_float(xw[k]));
              o[k] = __float_as_uint(w);
            } else {
              float w0 = __fmul_rn(v[8 * c + 2 * k], factor), w1 = __fmul_rn(v[8 * c + 2 * k + 1], factor);
              if (resid) {
                const float2 f = unpack_bf16x2(xw[k]);
                w0 = __fadd_rn(w0, f.x);
                w1 = __fadd_rn(w1, f.y);
              }
              o[k] = pack_bf16x2(w0, w1);
            }
          }
          *slot = make_uint4(o[0], o[1], o[2], o[3]);
        }
        fence_proxy_async();  // generic-proxy writes, read by the TMA unit
        __syncwarp();
        if (lane == 0) {
          tma_store_2d(&p.c, mine + buf * kPrChunk, ch.n0 + col, ch.row0);
          bulk_commit();
          // a store's buffer is read before it is used again: by the chunk after the next two, or for its residual
          if (resid) {
            bulk_wait_read1();
            request();
          } else {
            bulk_wait_read2();
          }
        }
        __syncwarp();
        buf = buf == kPrChunks - 1 ? 0 : buf + 1;
      } else {
        // rows of any alignment: turned in shared memory, a row of the chunk by a warp's consecutive lanes
        float* turn = reinterpret_cast<float*>(mine);
#pragma unroll
        for (int c = 0; c < kCols; c += 32) {
#pragma unroll
          for (int j = 0; j < 32; ++j) turn[lane * 33 + j] = __fmul_rn(v[c + j], factor);
          __syncwarp();
          const int n = ch.n0 + col + c + lane;
          if (n < p.g.N) {
#pragma unroll 8
            for (int r = 0; r < 32; ++r) {
              const int64_t m = ch.row0 + r;
              if (m >= p.g.M) break;
              float w = turn[r * 33 + lane];
              if constexpr (F32) {
                if (resid) w = __fadd_rn(w, static_cast<const float*>(p.g.residual)[m * p.g.ld_residual + n]);
                static_cast<float*>(p.g.c)[m * p.g.ld_c + n] = w;
              } else {
                if (resid)
                  w = __fadd_rn(w, __bfloat162float(static_cast<const __nv_bfloat16*>(p.g.residual)[m * p.g.ld_residual + n]));
                static_cast<__nv_bfloat16*>(p.g.c)[m * p.g.ld_c + n] = __float2bfloat16_rn(w);
              }
            }
          }
          __syncwarp();
        }
      }
    }
  }
  if (lane == 0) bulk_wait0();  // this warp's stores are complete
}

template <bool F32>
__global__ void __launch_bounds__(kPrThreads, 1) mxf4_pair_kernel(const __grid_constant__ Mxf4PairParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(stages + kPrStages * kPrStageBytes);
  uint64_t* empty = full + kPrStages;
  uint64_t* done = empty + kPrStages;
  uint64_t* taken = done + 1;
  uint64_t* loaded = taken + 1;  // [4 warps][kPrChunks]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(loaded + 4 * kPrChunks);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const uint32_t rank = cluster_rank();
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);  // uniform over the warp
  if (threadIdx.x == 0) {
    for (int i = 0; i < kPrStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    mbar_init(done, 1);
    mbar_init(taken, 8);  // the epilogue warps of both CTAs
    for (int i = 0; i < 4 * kPrChunks; ++i) mbar_init(&loaded[i], 1);
    *abort = 0;
    fence_barrier_init();
    fence_proxy_async();
    prefetch_tmap(&p.a);
    prefetch_tmap(&p.b);
    prefetch_tmap(&p.a_scale);
    prefetch_tmap(&p.b_scale);
  }
  if (warp == 1) {
    tmem_alloc_pair(tmem_slot, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  cluster_sync();  // both CTAs' barriers exist before any load or arrive reaches them
  const uint32_t tmem = *tmem_slot;
  pdl_begin(false);

  if (warp == 0) {
    if (elect_one()) mx_pair_producer(p, stages, full, empty, rank, abort);
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) mx_pair_mma(p, stages, full, empty, done, taken, tmem, abort);
  } else {
    mx_pair_epilogue<F32>(p, done, taken, loaded, tmem, rank, stages + kPrStages * kPrStageBytes + 1024, abort);
  }

  __syncwarp();
  if (*abort) {
    // copies and MMAs already issued land before shared and tensor memory go
    const long long t0 = clock64();
    while (clock64() - t0 < 20000000LL) {
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // the peer is done with this CTA's barriers and tensor memory
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

cudaError_t launch_mxf4_pair(const Mxf4Gemm& g, cudaStream_t s) {
  Mxf4PairParams p;
  p.g = g;
  p.m_tiles = (g.M - 1) / kPrTile + 1;
  p.n_tiles = (g.N - 1) / kPrTile + 1;
  const int64_t tiles = static_cast<int64_t>(p.m_tiles) * p.n_tiles;
  if (tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
  p.tiles = static_cast<int>(tiles);
  const uint64_t bytes = static_cast<uint64_t>(mxf4_row_bytes(g.K));
  if (!make_byte_map(&p.a, g.a, g.M, bytes, g.ld_a, 128) || !make_byte_map(&p.b, g.b, g.N, bytes, g.ld_b, 128) ||
      !make_scale_map(&p.a_scale, g.a_scale, g.M, g.K, 1) || !make_scale_map(&p.b_scale, g.b_scale, g.N, g.K, 2))
    return cudaErrorInvalidValue;
  // Tensor stores want 16-byte rows; anything else goes by plain ones.
  p.tma = make_result_map(&p.c, g.c, g.f32, g.M, g.N, g.ld_c) &&
          (!g.residual || make_result_map(&p.residual, g.residual, g.f32, g.M, g.N, g.ld_residual));
  void (*kernel)(Mxf4PairParams) = g.f32 ? mxf4_pair_kernel<true> : mxf4_pair_kernel<false>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPrSmem);
  if (e != cudaSuccess) return e;
  const int pairs = static_cast<int>(std::min<int64_t>(tiles, std::max(1, g.num_sms / 2)));
  return launch_pdl_cluster(kernel, dim3(2 * pairs), kPrThreads, kPrSmem, 2, s, p);
}

}  // namespace svl
