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
// accumulator while the rest is converted and stored. Tiles of 128 rows of B,
// for products whose tiles of 256 would leave SMs without work, have two
// accumulators side by side.
//
// Barriers: full[s] (leader's: both CTAs' loads of stage s have landed), ready[i]
// (leader's: a stage's scales are in set i), empty[s] (in both CTAs: the MMAs have
// read stage s), done (in both: a tile's MMAs are complete), taken (leader's: both
// epilogues have read the overlap, so the tile before is read altogether).
//
// Where tiles are few, clusters of two or four pairs share a tile's K.
//
// What bounds tiles of 256: a stage of 256 columns of K takes 594 cycles. Its MMAs
// alone take 512 (65,536 operations a cycle and pair; 533 measured without loads), its
// loads almost as long (35 KB an SM; 478 measured with one MMA of four and no copies of
// scales), and the two do not overlap altogether. The MMA's form with 96 columns of K,
// which has a higher rate, was not measured. Tiles of 128 take 450 cycles a stage: their
// issue (some 50 cycles an MMA of a pair) and loads. 10,240 x 22,016 x 4,096 runs at 6.4
// PFLOP/s call after call, under the power cap, and at 6.9 for a moment.
#include <algorithm>
#include <atomic>

#include "mxf4.cuh"
#include "result_slots.cuh"

namespace svl {

constexpr int kPrK = 256;           // values of K per stage: a 128-byte swizzled row of codes
constexpr int kPrRows = 256;        // rows of A per tile
constexpr int kPrChunk = 32 * 128;  // bytes of an epilogue chunk: 32 rows of 128 bytes
constexpr int kPrOutWarps = 8;      // two for each quarter of the lanes, with every other chunk of columns
// warps 0 and 10 load A and B, warp 11 copies scales and warp 1 MMAs (both the leader's), 2-9 epilogue
constexpr int kPrThreads = 128 + 32 * kPrOutWarps;
constexpr int kPrGroup = 8;  // tiles of rows that are walked together
// The epilogue warps' second buffers are the end of the stages (behind shares of K, 96 KB at most), so many bytes
// in front of their first.
constexpr int kPrSecondBack = 1024 + kPrOutWarps * kPrChunk;

// COLS: rows of B per tile, 256 or 128
template <int COLS>
struct PairCfg {
  static constexpr int kCodesA = 128 * 128;        // bytes of a CTA's rows of A
  static constexpr int kCodesB = COLS / 2 * 128;   // of its half of B's
  static constexpr int kScalesA = 2 * kMxTileBytes;
  static constexpr int kScalesB = COLS / 128 * 2 * kMxTileBytes;
  static constexpr int kStageBytes = kCodesA + kCodesB + kScalesA + kScalesB;
  static constexpr int kStages = COLS == 256 ? 5 : 7;
  static constexpr int kSmem = 1024 + kStages * kStageBytes + 1024 + kPrOutWarps * kPrChunk;
  // tensor memory: sets of scales, used in turn, at the end; the second accumulator in front of them or of its own
  static constexpr bool kApart = COLS == 128;  // a thread of its own copies them there
  static constexpr int kSets = kApart ? 4 : 2;
  static constexpr int kSet = 8 + COLS / 16;
  static constexpr int kSecondAcc = COLS == 256 ? 512 - kSets * kSet - COLS : COLS;
  static constexpr int kOverlap = COLS - kSecondAcc;
  static_assert(kSmem <= 232448, "shared memory per CTA");
  static_assert(kStages * kStageBytes - kPrOutWarps * kPrChunk >= 96 * 1024, "second buffers");
};

struct Mxf4PairParams {
  CUtensorMap a, b, a_scale, b_scale, c, residual;
  Mxf4Gemm g;
  int m_tiles, n_tiles, tiles;
  int log_split;  // pairs of a cluster, each with a share of K
  bool tma;       // C and the residual go by TMA
};

// What is the same for all of a CTA's tiles.
struct PairPlace {
  int rank, part;       // in the pair; the pair in its cluster
  uint32_t leader;      // the leader's rank in the cluster
  int first, stride;    // tiles
  int s0, s1;           // stages of K
};
SVL_DEVINL PairPlace pair_place(const Mxf4PairParams& p) {
  PairPlace w;
  const int cr = static_cast<int>(cluster_rank()), all = (p.g.K - 1) / kPrK + 1;
  w.rank = cr & 1;
  w.part = cr >> 1;
  w.leader = static_cast<uint32_t>(cr & ~1);
  w.first = static_cast<int>(blockIdx.x >> (1 + p.log_split));
  w.stride = static_cast<int>(gridDim.x >> (1 + p.log_split));
  w.s0 = (all * w.part) >> p.log_split;
  w.s1 = (all * (w.part + 1)) >> p.log_split;
  return w;
}

struct PairTile {
  int m0, n0;
};
// Groups of kPrGroup row tiles, column tile by column tile: tiles that run at
// the same time share rows of both operands.
template <int COLS>
SVL_DEVINL PairTile pair_tile(const Mxf4PairParams& p, int t) {
  const int per = kPrGroup * p.n_tiles, g = t / per, r = t - g * per;
  const int height = max(1, min(kPrGroup, p.m_tiles - g * kPrGroup));  // (1: behind the last tile)
  PairTile ti;
  ti.m0 = (g * kPrGroup + r % height) * kPrRows;
  ti.n0 = r / height * COLS;
  return ti;
}

// One thread a CTA loads its rows of A (OP 0), one its half of B (OP 1), each with the scales.
template <int COLS, int OP>
SVL_DEVINL void mx_pair_producer(const Mxf4PairParams& p, const PairPlace& w, uint8_t* stages, uint64_t* full,
                                 uint64_t* empty, volatile int* abort) {
  using C = PairCfg<COLS>;
  int s = 0;
  uint32_t ph = 1;
  auto next = [&]() {
    if (++s == C::kStages) {
      s = 0;
      ph ^= 1;
    }
  };
  PairTile ti = pair_tile<COLS>(p, w.first);
  pdl_wait();
  for (int t = w.first; t < p.tiles; t += w.stride, ti = pair_tile<COLS>(p, t)) {
    const int m0 = ti.m0 + w.rank * 128, n0 = ti.n0 + w.rank * (COLS / 2);
    for (int k = w.s0; k < w.s1; ++k, next()) {
      if (!mbar_wait(&empty[s], ph, abort)) return mx_abort(abort, p.g.status);
      uint8_t* st = stages + s * C::kStageBytes;
      const uint32_t fb = mapa_shared(&full[s], w.leader);
      if constexpr (OP == 0) {
        if (w.rank == 0) mbar_arrive_expect_tx(&full[s], 2 * (C::kCodesA + C::kScalesA));
        tma_load_2d_pair(st, &p.a, fb, k * 128, m0);
        tma_load_2d_pair(st + C::kCodesA + C::kCodesB, &p.a_scale, fb, k * 256, m0 >> 7);
      } else {
        if (w.rank == 0) mbar_arrive_expect_tx(&full[s], 2 * (C::kCodesB + C::kScalesB));
        tma_load_2d_pair(st + C::kCodesA, &p.b, fb, k * 128, n0);
        tma_load_2d_pair(st + C::kCodesA + C::kCodesB + C::kScalesA, &p.b_scale, fb, k * 256, ti.n0 >> 7);
      }
    }
  }
  // the releases of the last stages (the leader's MMA commits) have arrived here
  for (int i = 0; i < C::kStages; ++i, next())
    if (!mbar_wait(&empty[s], ph, abort)) return mx_abort(abort, p.g.status);
}

template <int COLS>
SVL_DEVINL uint32_t pair_acc(uint32_t tmem, int it) {
  return tmem + ((it & 1) ? PairCfg<COLS>::kSecondAcc : 0);
}

// Copies a stage's scales (descriptor d) to a set in tensor memory: A's two tiles of
// 128 columns of K (4 tensor memory columns each), then B's (4 per 128 rows).
template <int COLS>
SVL_DEVINL void pair_copy_scales(uint64_t d, uint32_t sa, bool two) {
  const uint32_t sb = sa + 8;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (j == 0 || two) {
      tc_copy_scales_pair(sa + 4 * j, d + j * (kMxTileBytes >> 4));
#pragma unroll
      for (int c = 0; c < COLS / 128; ++c)
        tc_copy_scales_pair(sb + (COLS / 32) * j + 4 * c,
                            d + ((PairCfg<COLS>::kScalesA + (2 * c + j) * kMxTileBytes) >> 4));
    }
  }
}

// Tiles of 128 rows of B: a thread of its own copies the scales of each stage to the
// next of kSets sets, when the MMAs that read that set before are complete
// (their stage's release). The MMAs of a stage take half the time of a larger
// tile's, less than one thread needs to issue both (300 x 3,584 x 18,944 23.3 ->
// 19.9 us); with tiles of 256 the way over another thread costs more (26.0 -> 29.4).
template <int COLS>
SVL_DEVINL void mx_pair_scales(const Mxf4PairParams& p, const PairPlace& w, uint8_t* stages, uint64_t* full,
                               uint64_t* empty, uint64_t* ready, uint32_t tmem, volatile int* abort) {
  using C = PairCfg<COLS>;
  const uint64_t d0 = smem_desc_scales(smem_u32(stages) + C::kCodesA + C::kCodesB);
  int s = 0, set = 0, before = 0;  // stage, set, the stage that had the set before
  uint32_t ph = 0, before_ph = 0;
  int lead = C::kSets;             // sets that nothing has used yet
  for (int t = w.first; t < p.tiles; t += w.stride) {
    for (int k = w.s0; k < w.s1; ++k) {
      if (lead > 0) {
        --lead;
      } else {
        if (!mbar_wait(&empty[before], before_ph, abort)) return mx_abort(abort, p.g.status);
        if (++before == C::kStages) {
          before = 0;
          before_ph ^= 1;
        }
      }
      if (!mbar_wait(&full[s], ph, abort)) return mx_abort(abort, p.g.status);
      tc_fence_after();
      pair_copy_scales<COLS>(d0 + static_cast<uint32_t>(s * (C::kStageBytes >> 4)),
                             tmem + 512 - C::kSets * C::kSet + set * C::kSet, p.g.K - k * kPrK > 128);
      tc_commit_pair_here(&ready[set]);
      if (++s == C::kStages) {
        s = 0;
        ph ^= 1;
      }
      if (++set == C::kSets) set = 0;
    }
  }
}

// One thread of the leader issues the MMAs: when a stage's loads have landed, with
// its copies of scales in front, or when its scales are there (and so its codes,
// which their copies waited for).
template <int COLS>
SVL_DEVINL void mx_pair_mma(const Mxf4PairParams& p, const PairPlace& w, uint8_t* stages, uint64_t* full,
                            uint64_t* ready, uint64_t* empty, uint64_t* done, uint64_t* taken, uint32_t tmem,
                            volatile int* abort) {
  using C = PairCfg<COLS>;
  const uint32_t base = smem_u32(stages);
  const uint64_t da0 = smem_desc_sw128(base), db0 = smem_desc_sw128(base + C::kCodesA);
  const uint64_t ds0 = smem_desc_scales(base + C::kCodesA + C::kCodesB);
  constexpr uint32_t id0 = idesc_mxf4(kPrRows, COLS, 0), id1 = idesc_mxf4(kPrRows, COLS, 1);
  const uint16_t ctas = static_cast<uint16_t>(3u << w.leader);
  int s = 0, it = 0, set = 0;
  uint32_t ph = 0, set_ph = 0;
  for (int t = w.first; t < p.tiles; t += w.stride, ++it) {
    if (it > 0 && !mbar_wait(taken, (it - 1) & 1, abort)) return mx_abort(abort, p.g.status);
    tc_fence_after();
    const uint32_t d = pair_acc<COLS>(tmem, it);
    for (int k = w.s0; k < w.s1; ++k) {
      if (!(C::kApart ? mbar_wait(&ready[set], set_ph, abort) : mbar_wait(&full[s], ph, abort)))
        return mx_abort(abort, p.g.status);
      tc_fence_after();
      const uint32_t at = static_cast<uint32_t>(s * (C::kStageBytes >> 4));
      const uint32_t sa = tmem + 512 - C::kSets * C::kSet + set * C::kSet, sb = sa + 8;
      const uint64_t da = da0 + at, db = db0 + at;
      const int left = p.g.K - k * kPrK;
      if (!C::kApart) pair_copy_scales<COLS>(ds0 + at, sa, left > 128);
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // 64 values of K an instruction
        if (left > 64 * i)
          tc_mma_mxf4_pair(d, da + 2 * i, db + 2 * i, (i & 1) ? id1 : id0, sa + 4 * (i >> 1), sb + (COLS / 32) * (i >> 1),
                           i > 0 || k > w.s0);
      }
      tc_commit_pair(&empty[s], ctas);
      if (++s == C::kStages) {
        s = 0;
        ph ^= 1;
      }
      if (++set == C::kSets) {
        set = 0;
        set_ph ^= 1;
      }
    }
    tc_commit_pair(done, ctas);
  }
}

// The chunks of a warp, over all of its tiles: 128 bytes of 32 rows of C, every
// other of a tile's. In accumulator 1 they are taken from the left, in accumulator
// 0 from the right. Where K is shared (one tile a cluster), a CTA has the columns
// that it adds up.
template <bool F32, int COLS>
struct PairChunks {
  static constexpr int kCols = F32 ? 32 : 64;
  const Mxf4PairParams& p;
  const PairPlace& w;
  int t, it, row0, offset, half;  // tile, its number, the warp's first row, its rows' offset in the tile, first chunk
  int n0, n, i;                   // tile's first column, its chunks (0: no rows of the warp exist), the present one
  SVL_DEVINL PairChunks(const Mxf4PairParams& params, const PairPlace& place, int rows_at, int first)
      : p(params), w(place), t(place.first), it(0), offset(rows_at), half(first) {
    enter();
  }
  SVL_DEVINL void enter() {
    i = half;
    n = 0;
    if (t >= p.tiles) return;
    const PairTile ti = pair_tile<COLS>(p, t);
    row0 = ti.m0 + offset;
    const int width = COLS >> p.log_split;
    n0 = ti.n0 + w.part * width;
    if (row0 < p.g.M) n = (max(0, min(width, p.g.N - n0)) + kCols - 1) / kCols;
  }
  SVL_DEVINL void next_tile() {
    t += w.stride;
    ++it;
    enter();
  }
  // to a chunk that there is, in this tile or a later one
  SVL_DEVINL void settle() {
    while (i >= n && t < p.tiles) next_tile();
  }
  SVL_DEVINL bool more() const { return t < p.tiles; }
  SVL_DEVINL int column() const { return ((it & 1) ? i : n - 1 - i) * kCols; }
};

// A warp's results on their way out: its buffer in shared memory, and the next
// chunk of the residual, requested when the buffer is free. In the CTA's last tile
// the stages are used up, and a second buffer in their place takes every other
// chunk, the first one too (a store holds its buffer for some 900 cycles).
template <bool F32, int COLS>
struct PairOut {
  static constexpr int kCols = F32 ? 32 : 64;
  const Mxf4PairParams& p;
  uint8_t* own;
  uint64_t* loaded;  // [2]
  PairChunks<F32, COLS> ahead;
  volatile int* abort;
  uint32_t parity = 0;  // of each buffer's next wait
  ResultSlots slots;
  SVL_DEVINL PairOut(const Mxf4PairParams& params, const PairChunks<F32, COLS>& chunks, uint8_t* first, uint64_t* bars,
                     volatile int* flag)
      : p(params), own(first), loaded(bars), ahead(chunks), abort(flag) {
    if (p.g.residual && p.tma && (threadIdx.x & 31) == 0) request(0);
  }
  SVL_DEVINL uint8_t* buffer(int b) const { return own - b * kPrSecondBack; }
  SVL_DEVINL void request(int b) {
    ahead.settle();
    if (!ahead.more()) return;
    mbar_arrive_expect_tx(&loaded[b], kPrChunk);
    tma_load_2d(buffer(b), &p.residual, &loaded[b], ahead.n0 + ahead.column(), ahead.row0);
    ahead.i += 2;
  }
  // The last tile's MMAs are complete.
  SVL_DEVINL void enter_last() {
    slots.enter_last(p.g.residual != nullptr);
    if (p.g.residual && p.tma && (threadIdx.x & 31) == 0) request(1);
  }
  // The chunk from column n0 and row row0 on: the factor and the sum with the
  // residual in float32, one rounding to C's type.
  SVL_DEVINL bool chunk(const float* v, float factor, int n0, int row0) {
    const int lane = threadIdx.x & 31;
    const bool resid = p.g.residual != nullptr;
    if (p.tma) {
      const int slot = slots.slot;
      uint8_t* const at = buffer(slot);
      if (resid) {
        const bool got = mbar_wait(&loaded[slot], (parity >> slot) & 1, abort);
        parity ^= 1u << slot;
        __syncwarp();
        if (!__all_sync(0xffffffffu, got)) return false;
      } else {
        if (lane == 0) {  // the store before (in the last tile, the one before that) has read the buffer
          if (slots.unread())
            bulk_wait_read1();
          else
            bulk_wait_read0();
        }
        __syncwarp();
      }
      uint8_t* slot0 = at + lane * 128;
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
            float y = __fmul_rn(v[4 * c + k], factor);
            if (resid) y = __fadd_rn(y, __uint_as_float(xw[k]));
            o[k] = __float_as_uint(y);
          } else {
            float y0 = __fmul_rn(v[8 * c + 2 * k], factor), y1 = __fmul_rn(v[8 * c + 2 * k + 1], factor);
            if (resid) {
              const float2 f = unpack_bf16x2(xw[k]);
              y0 = __fadd_rn(y0, f.x);
              y1 = __fadd_rn(y1, f.y);
            }
            o[k] = pack_bf16x2(y0, y1);
          }
        }
        *slot = make_uint4(o[0], o[1], o[2], o[3]);
      }
      fence_proxy_async();  // generic-proxy writes, read by the TMA unit
      __syncwarp();
      if (lane == 0) {
        tma_store_2d(&p.c, at, n0, row0);
        bulk_commit();
        if (resid) {
          bulk_wait_read0();
          request(slot);
        }
      }
      slots.stored();
      return true;
    }
    // rows of any alignment: turned in shared memory, a row of the chunk by a warp's consecutive lanes
    float* turn = reinterpret_cast<float*>(own);
#pragma unroll
    for (int c = 0; c < kCols; c += 32) {
#pragma unroll
      for (int j = 0; j < 32; ++j) turn[lane * 32 + (j ^ lane)] = __fmul_rn(v[c + j], factor);
      __syncwarp();
      const int n = n0 + c + lane;
      if (n < p.g.N) {
        // (eight rows' residuals are requested before the first of them is stored over)
        for (int r0 = 0; r0 < 32; r0 += 8) {
          float y[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const int64_t m = row0 + r0 + r;
            y[r] = 0.f;
            if (resid && m < p.g.M)
              y[r] = F32 ? static_cast<const float*>(p.g.residual)[m * p.g.ld_residual + n]
                         : __bfloat162float(static_cast<const __nv_bfloat16*>(p.g.residual)[m * p.g.ld_residual + n]);
          }
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const int64_t m = row0 + r0 + r;
            if (m >= p.g.M) break;
            float x = turn[(r0 + r) * 32 + (lane ^ (r0 + r))];
            if (resid) x = __fadd_rn(x, y[r]);
            if constexpr (F32)
              static_cast<float*>(p.g.c)[m * p.g.ld_c + n] = x;
            else
              static_cast<__nv_bfloat16*>(p.g.c)[m * p.g.ld_c + n] = __float2bfloat16_rn(x);
          }
        }
      }
      __syncwarp();
    }
    return true;
  }
};

// Where a warp reads the accumulators, and its chunks.
struct PairWarp {
  int lane, q, half;  // quarter of the lanes, first chunk
  SVL_DEVINL PairWarp() : lane(threadIdx.x & 31), q((threadIdx.x >> 5) & 3), half((threadIdx.x - 64) >> 7) {}
  SVL_DEVINL int index() const { return q * 2 + half; }
  SVL_DEVINL uint32_t lanes() const { return static_cast<uint32_t>(q * 32) << 16; }
};

// A warp has read what the next MMAs write over: its reads of tensor memory are
// complete, and the fence keeps them in front of the arrival, which orders nothing else.
SVL_DEVINL void hand_over(uint32_t taken, int lane) {
  tc_fence_before();
  __syncwarp();
  if (lane == 0) mbar_arrive_cluster_relaxed(taken);
}

template <bool F32, int COLS>
SVL_DEVINL void mx_pair_epilogue(const Mxf4PairParams& p, const PairPlace& w, uint64_t* done, uint64_t* taken,
                                 uint64_t* loaded, uint32_t tmem, uint8_t* buffers, volatile int* abort) {
  using C = PairCfg<COLS>;
  constexpr int kCols = F32 ? 32 : 64;
  const PairWarp me;
  const uint32_t release = mapa_shared(taken, w.leader);
  PairChunks<F32, COLS> ch(p, w, w.rank * 128 + me.q * 32, me.half);
  pdl_wait();
  PairOut<F32, COLS> out(p, ch, buffers + me.index() * kPrChunk, loaded + 2 * me.index(), abort);
  for (; ch.more(); ch.next_tile()) {
    const int row = ch.row0 + me.lane;
    const float factor = p.g.row_factor && ch.n > 0 && row < p.g.M ? p.g.row_factor[row] : 1.f;
    const bool ok = mbar_wait(done, ch.it & 1, abort);
    __syncwarp();
    if (!__all_sync(0xffffffffu, ok)) return mx_abort(abort, p.g.status);
    tc_fence_after();
    const bool last = ch.t + w.stride >= p.tiles;
    if (last) out.enter_last();
    const uint32_t acc = pair_acc<COLS>(tmem, ch.it) + me.lanes();
    // Chunks that hold the overlap come first; a warp hands over when it has read the last of its own. (Where the
    // tile's columns end before the overlap, there is none.) Behind the last tile nothing waits for an arrival, and the
    // leader, to whose shared memory it goes, might have ended.
    const int in_overlap = min(
        ch.n, (ch.it & 1) ? (C::kOverlap + kCols - 1) / kCols : ch.n - (COLS - C::kOverlap) / kCols);
    bool handed = last || ch.i >= in_overlap;
    if (handed && !last) hand_over(release, me.lane);  // (for its reads of the tile before)
    for (; ch.i < ch.n; ch.i += 2) {
      float v[kCols];
      const int col = ch.column();
#pragma unroll
      for (int c = 0; c < kCols; c += 32) tmem_ld32(acc + col + c, v + c);
      if (!handed && ch.i + 2 >= in_overlap) {
        hand_over(release, me.lane);
        handed = true;
      }
      if (!out.chunk(v, factor, ch.n0 + col, ch.row0)) return mx_abort(abort, p.g.status);
    }
  }
  if (me.lane == 0) bulk_wait0();  // this warp's stores are complete
}

// The same where a cluster's pairs share a tile's K: each CTA sends the columns
// that others add up to them, over the stages, which are used up everywhere
// (`free_bar`), and adds what arrives to its own, in the order of the others.
// Layout: [the others in order][group of four columns][128 rows][4].
template <bool F32, int COLS>
SVL_DEVINL void mx_pair_shares(const Mxf4PairParams& p, const PairPlace& w, uint64_t* done, uint64_t* free_bar,
                               uint64_t* arrived, uint64_t* loaded, uint32_t tmem, uint8_t* stages, uint8_t* buffers,
                               volatile int* abort) {
  constexpr int kCols = F32 ? 32 : 64;
  const PairWarp me;
  const int split = 1 << p.log_split, width = COLS >> p.log_split;
  const int share = (width / 4) * 128 * 16;  // bytes
  PairChunks<F32, COLS> ch(p, w, w.rank * 128 + me.q * 32, me.half);
  pdl_wait();
  PairOut<F32, COLS> out(p, ch, buffers + me.index() * kPrChunk, loaded + 2 * me.index(), abort);
  const bool rows = ch.row0 < p.g.M;  // of this warp, which the other pairs' warps with the same place have too
  const float factor = p.g.row_factor && ch.row0 + me.lane < p.g.M ? p.g.row_factor[ch.row0 + me.lane] : 1.f;
  bool ok = mbar_wait(done, 0, abort);
  __syncwarp();
  ok = __all_sync(0xffffffffu, ok);
  if (ok) {
    out.enter_last();
    if (me.index() == 0 && me.lane < split) mbar_arrive_cluster_relaxed(mapa_shared(free_bar, 2 * me.lane + w.rank));
    ok = mbar_wait(free_bar, 0, abort);
    __syncwarp();
    ok = __all_sync(0xffffffffu, ok);
  }
  if (!ok) return mx_abort(abort, p.g.status);
  if (!rows) return;
  tc_fence_after();
  const uint32_t acc = tmem + me.lanes();
  const uint32_t place = static_cast<uint32_t>(me.q * 32 + me.lane) * 16;
  for (int i = 1; i < split; ++i) {
    const int o = (w.part + i) & (split - 1);  // (a CTA's first receiver is no other's)
    const uint32_t to = mapa_shared(stages, 2 * o + w.rank) + (w.part < o ? w.part : w.part - 1) * share + place;
    const uint32_t bar = mapa_shared(arrived, 2 * o + w.rank);
    for (int c = 32 * me.half; c < width; c += 64) {
      float v[32];
      tmem_ld32(acc + o * width + c, v);
#pragma unroll
      for (int j = 0; j < 32; j += 4) st_async4(to + static_cast<uint32_t>((c + j) >> 2) * (128 * 16), bar, v + j);
    }
  }
  ok = mbar_wait(arrived, 0, abort);
  __syncwarp();
  if (!__all_sync(0xffffffffu, ok)) return mx_abort(abort, p.g.status);
  for (; ch.i < ch.n; ch.i += 2) {
    float v[kCols];
    const int col = ch.column();
#pragma unroll
    for (int c = 0; c < kCols; c += 32) tmem_ld32(acc + w.part * width + col + c, v + c);
    const uint8_t* from = stages + (col >> 2) * (128 * 16) + place;
    for (int s = 1; s < split; ++s, from += share) {
#pragma unroll
      for (int j = 0; j < kCols; j += 4) {
        const float4 x = *reinterpret_cast<const float4*>(from + (j >> 2) * (128 * 16));
        v[j] = __fadd_rn(v[j], x.x);
        v[j + 1] = __fadd_rn(v[j + 1], x.y);
        v[j + 2] = __fadd_rn(v[j + 2], x.z);
        v[j + 3] = __fadd_rn(v[j + 3], x.w);
      }
    }
    if (!out.chunk(v, factor, ch.n0 + col, ch.row0)) return mx_abort(abort, p.g.status);
  }
  if (me.lane == 0) bulk_wait0();
}

template <bool F32, bool SHARED, int COLS>
__global__ void __launch_bounds__(kPrThreads, 1) mxf4_pair_kernel(const __grid_constant__ Mxf4PairParams p) {
  using C = PairCfg<COLS>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* stages = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(stages + C::kStages * C::kStageBytes);
  uint64_t* empty = full + C::kStages;
  uint64_t* done = empty + C::kStages;
  uint64_t* taken = done + 1;
  uint64_t* free_bar = taken + 1;
  uint64_t* arrived = free_bar + 1;
  uint64_t* ready = arrived + 1;   // [set of scales]
  uint64_t* loaded = ready + 4;    // [epilogue warp][2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(loaded + 2 * kPrOutWarps);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const PairPlace w = pair_place(p);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);  // uniform over the warp
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      mbar_init(&full[i], 2);  // the leader's producers
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < C::kSets; ++i) mbar_init(&ready[i], 1);
    mbar_init(done, 1);
    mbar_init(taken, 2 * kPrOutWarps);  // the epilogue warps of both CTAs
    for (int i = 0; i < 2 * kPrOutWarps; ++i) mbar_init(&loaded[i], 1);
    mbar_init(free_bar, 1u << p.log_split);
    mbar_init(arrived, 1);
    *abort = 0;
    fence_barrier_init();
    fence_proxy_async();
    if (SHARED) {
      // from every other pair, for each warp here that has rows, 32 of them of a share
      const int rows = p.g.M - pair_tile<COLS>(p, w.first).m0 - w.rank * 128, warps = max(0, min(4, (rows + 31) >> 5));
      const int others = (1 << p.log_split) - 1, width = COLS >> p.log_split;
      mbar_arrive_expect_tx(arrived, static_cast<uint32_t>(others * warps * 32 * width * 4));
    }
  } else if (threadIdx.x == 64) {
    prefetch_tmap(&p.a);
    prefetch_tmap(&p.b);
    prefetch_tmap(&p.a_scale);
    prefetch_tmap(&p.b_scale);
    if (p.tma) prefetch_tmap(&p.c);
    if (p.tma && p.g.residual) prefetch_tmap(&p.residual);
  }
  __syncwarp();
  cluster_arrive_relaxed();  // (the first warp behind its barriers' initialisation)
  if (warp == 1) {
    tmem_alloc_pair(tmem_slot, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();  // (the next kernel's CTAs take no tensor memory that this one still has to get)
  cluster_wait();  // the cluster's barriers exist before any load or arrive reaches them
  const uint32_t tmem = *tmem_slot;

  uint8_t* buffers = stages + C::kStages * C::kStageBytes + 1024;
  if (warp == 0) {
    if (elect_one()) mx_pair_producer<COLS, 0>(p, w, stages, full, empty, abort);
  } else if (warp == 10) {
    if (elect_one()) mx_pair_producer<COLS, 1>(p, w, stages, full, empty, abort);
  } else if (warp == 1) {
    if (w.rank == 0 && elect_one()) mx_pair_mma<COLS>(p, w, stages, full, ready, empty, done, taken, tmem, abort);
  } else if (warp == 11) {
    if (C::kApart && w.rank == 0 && elect_one()) mx_pair_scales<COLS>(p, w, stages, full, empty, ready, tmem, abort);
  } else if constexpr (SHARED) {
    mx_pair_shares<F32, COLS>(p, w, done, free_bar, arrived, loaded, tmem, stages, buffers, abort);
  } else {
    mx_pair_epilogue<F32, COLS>(p, w, done, taken, loaded, tmem, buffers, abort);
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
  // The peer is done with this CTA's barriers and tensor memory. (Nothing that was written is handed over here; with
  // release semantics the barrier waits 1,000 cycles for the stores of results.)
  cluster_arrive_relaxed();
  cluster_wait();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

using PairKernel = void (*)(Mxf4PairParams);
static PairKernel pair_kernel(bool shared, bool f32, int cols) {
  if (cols == 128) return f32 ? mxf4_pair_kernel<true, false, 128> : mxf4_pair_kernel<false, false, 128>;
  return shared ? (f32 ? mxf4_pair_kernel<true, true, 256> : mxf4_pair_kernel<false, true, 256>)
                : (f32 ? mxf4_pair_kernel<true, false, 256> : mxf4_pair_kernel<false, false, 256>);
}

// The answer is the device's (76, 36 and 15 clusters of 2, 4 and 8 CTAs on one
// with 152 SMs): asked once, of the kernel that has an SM to a CTA.
int mxf4_clusters(int ctas) {
  static std::atomic<int> known[16][3];  // (0: not known yet)
  const int log = ctas == 8 ? 2 : ctas == 4 ? 1 : 0;
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  std::atomic<int>* place = dev < 16 ? &known[dev][log] : nullptr;
  if (place && (n = place->load(std::memory_order_relaxed))) return n - 1;
  PairKernel kernel = pair_kernel(log > 0, true, 256);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2u << log);
  cfg.blockDim = dim3(kPrThreads);
  cfg.dynamicSmemBytes = PairCfg<256>::kSmem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2u << log;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PairCfg<256>::kSmem) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess)
    return 0;
  if (place) place->store(n + 1, std::memory_order_relaxed);
  return n;
}

cudaError_t launch_mxf4_pair(const Mxf4Gemm& g, cudaStream_t s) {
  Mxf4PairParams p;
  p.g = g;
  const int64_t m_tiles = (g.M - 1) / kPrRows + 1, wide = m_tiles * ((g.N - 1) / 256 + 1);
  const int64_t narrow = m_tiles * ((g.N - 1) / 128 + 1), pairs = std::max(1, mxf4_clusters(2));
  // Tiles of 128 rows of B where they take no more waves (4,096 rows of B, K 4,096, us for 256 and
  // 128: 300 rows of A 9.2, 7.7; 800 rows 9.9, 12.4). Of 256, a cluster's pairs share K where all of the tiles'
  // clusters run at once and K has the stages to make up for the sums' way. us for 128, and for 256 with 2 and 4 pairs:
  // 2,048 rows of B, K 4,096 (16 stages) 7.4, 8.8, 8.5; 4,608 and 11,008 (43 stages) 13.4, 14.0; 1,000 and 11,008 13.2,
  // 12.9, 10.4; 3,584 and 18,944 (74 stages), 150 rows of A 20.0, 17.8, 14.2, 500 rows 20.1, 18.4.
  int cols = (narrow - 1) / pairs <= (wide - 1) / pairs ? 128 : 256, log_split = 0;
  const int k_stages = (g.K - 1) / kPrK + 1;
  if (k_stages >= 24 && wide <= mxf4_clusters(8))
    log_split = 2;
  else if (k_stages >= 50 && wide <= mxf4_clusters(4))
    log_split = 1;
  if (log_split) cols = 256;
  const int64_t tiles = cols == 256 ? wide : narrow;
  if (narrow > INT32_MAX / 2) return cudaErrorInvalidValue;
  p.m_tiles = static_cast<int>(m_tiles);
  p.n_tiles = (g.N - 1) / cols + 1;
  p.tiles = static_cast<int>(tiles);
  p.log_split = log_split;
  const uint64_t bytes = static_cast<uint64_t>(mxf4_row_bytes(g.K));
  if (!make_byte_map(&p.a, g.a, g.M, bytes, g.ld_a, 128) ||
      !make_byte_map(&p.b, g.b, g.N, bytes, g.ld_b, static_cast<uint32_t>(cols / 2)) ||
      !make_scale_map(&p.a_scale, g.a_scale, g.M, g.K, 1) ||
      !make_scale_map(&p.b_scale, g.b_scale, g.N, g.K, static_cast<uint32_t>(cols / 128)))
    return cudaErrorInvalidValue;
  // Tensor stores want 16-byte rows, and end a row at a multiple of 16 bytes; anything else goes by plain ones.
  p.tma = (static_cast<int64_t>(g.N) * (g.f32 ? 4 : 2)) % 16 == 0 &&
          make_result_map(&p.c, g.c, g.f32, g.M, g.N, g.ld_c) &&
          (!g.residual || make_result_map(&p.residual, g.residual, g.f32, g.M, g.N, g.ld_residual));
  PairKernel kernel = pair_kernel(log_split > 0, g.f32, cols);
  const int smem = cols == 256 ? PairCfg<256>::kSmem : PairCfg<128>::kSmem, ctas = 2 << log_split;
  static std::atomic<uint64_t> devices[3][2];  // of each kernel
  cudaError_t e = mxf4_allow_smem(reinterpret_cast<const void*>(kernel), smem,
                                  &devices[cols == 128 ? 2 : log_split > 0][g.f32]);
  if (e != cudaSuccess) return e;
  const int64_t clusters = log_split ? tiles : std::min(tiles, pairs);
  return launch_pdl_cluster(kernel, dim3(static_cast<unsigned>(clusters * ctas)), kPrThreads, smem, ctas, s, p);
}

}  // namespace svl
