// Attention of the newest rows of each slot over its 4-bit KV cache:
//   o = sum_j softmax_j(scale * q . k_j) v_j
// over the positions j that the row at position pos sees: j <= pos, and with a
// window W > 0 only j > pos - W or j < sinks. A row with pos < 0 sees nothing
// and a row with pos >= max_len has no place in the cache: both give zeros.
//
// Bound by the cache's bytes (d_head * 9 / 8 per position and KV head) if a value
// costs no more than about three instructions' lanes on its way from memory, which
// is what decides the design:
//  - The products run on mma.m16n8 with float32 sums: S = K q with 16 positions as
//    rows and 8 columns, O^T = V^T P with 16 dimensions as rows. A column is a query
//    head of the KV head or one of its rows (drafted tokens); up to eight share one
//    pass over the cache. (tcgen05 would take 128 rows at a time, from shared or tensor
//    memory, to which every dequantised value would have to be written first, and leaves
//    its sums in tensor memory, from which they would come back for each 32 dimensions,
//    to be multiplied by their scales. Here codes and sums stay in registers.)
//  - K's codes become float16 operands by masking alone: n * 2^-24 and n * 2^-20
//    (subnormal numbers), both exact; q is scaled by a power of two to fill
//    float16's range (bf16 has fewer bits, so that it is exact but for elements
//    under 2^-31 of the head's largest), times 2^-4 where it meets the second kind,
//    the odd dimensions (exact but for elements under 2^-27 of the largest).
//    The -8 of s * (n - 8) costs nothing: the accumulators start at -8 * sum q of the
//    group. The scales multiply the 32-dimension partial sums in float32. (e4m3
//    operands would take fewer masks, but mma.sync converts them to float16 first.)
//  - V's codes become bf16 operands n - 8 (128 + n by masking, less 136; taken off
//    O at the end instead, the 8 would leave the rounding of sums of 8 s in
//    dimensions much smaller than their group). Its scales multiply the weights.
//    Weights and products are pairs of bf16 numbers, of 16 bits together and with
//    float32's range: float16 (one product instead of two, 15 % faster) would lose
//    weights under 2^-38 of the largest, which are all there is in a dimension where
//    the rows of larger weight hold zeros.
//
// Work is cut by tiles, not by heads or slots, so that ragged lengths and few slots
// fill the GPU alike: the tiles of all (slot, KV head, column tile) items in a row
// are divided evenly over the SMs and there over the warps. A warp walks its tiles
// with an online softmax, its next tiles on their way into a ring of its own in
// shared memory (cp.async). Items that end up in several warps are put together
// from their parts in order: in shared memory within a CTA, by a second launch
// across CTAs. Few and short items instead have a cluster of one to eight CTAs each,
// whose parts meet in its shared memory: one launch (attn_run has the rule).
//
// Measured, d_head 128 (times of the call in a graph, rates of the cache's bytes; a
// copy runs at 6.8 TB/s):
//  - 32 heads of their own, 8 slots of 4,000 to 16,000 positions: 55.0 us, 5.8 TB/s
//    (52.5 us without any arithmetic, some 6 of them launching and joining). Some 620
//    instructions a tile, of which 337 are the ALU's, keep it busy 62 % of the time.
//    16 slots of 250 to 450 positions: 12.3 us (8.6), two or three tiles a warp.
//  - 28 heads on 4 KV heads (seven columns), 8 slots of 20,000 to 40,000 positions:
//    37.6 us (26.7), 3.4 TB/s; four rows (28 columns, four passes) 113 us (45). Three warps
//    per scheduler are all that the registers allow, each a chain of products,
//    shuffles and exponentials: instructions issue in 47 and 58 % of the cycles, and
//    no single kind of arithmetic left out saves more than 8 %.
//  - one slot of 1,900 positions, 28 heads on 4 KV heads: 7.4 us of latencies (8.4 with
//    the second launch): launching 0.8, queries and first tile 1.3, a tile 1.1, its end
//    0.5, the warps' parts 1.0, the cluster's some 1.
#include <cuda_fp16.h>

#include "kv4.cuh"

namespace svl {

constexpr int kCols = 8;
constexpr int kMaxCtas = 256;
constexpr int kMergeThreads = 128;
constexpr int kClusterCtas = 8;  // most CTAs of a cluster

struct AttnParams {
  Kv4Attn a;
  int ncols;      // columns of an item: min(8, rows * heads per KV head)
  int col_tiles;  // items per KV head
  int run;        // CTAs of an item's cluster (0: tiles are dealt to all CTAs)
  int min_tiles;  // least tiles of a CTA that has any
  int grp;        // heads per KV head
  int columns;    // rows * grp
  float inv_grp;  // 1 / grp
  float* part;    // [CTAs][2][ncols * (d_head + 2)]: parts of items shared with other CTAs, the one from
                  // the CTA before and the one that the next goes on with
  int4* meta;     // [CTAs]: {slot (-1: none), item, KV head} of the latter, and the CTAs that it is in
};

// The tiles of a slot that any of its rows sees: `sink` tiles from 0 on, then those from `first`.
struct Span {
  int n, sink, first;
};
SVL_DEVINL Span slot_span(const Kv4Attn& a, int slot) {
  const int64_t start = a.start[slot];
  const int64_t last = start + a.rows < a.c.max_len ? start + a.rows : a.c.max_len;  // end of the last row's sight
  Span s{1, 1, 0};  // nothing visible: one tile, all masked, gives the zeros
  if (start >= a.c.max_len || last <= 0) return s;
  const int hi = static_cast<int>(last), lowest = static_cast<int>(start > 0 ? start : 0) + 1;
  const int lo = a.window > 0 && lowest > a.window ? lowest - a.window : 0;
  const int end = (hi - 1) / kKv4Tile + 1;
  s.first = lo / kKv4Tile;
  const int sinks = a.sinks < hi ? a.sinks : hi;
  const int st = sinks > 0 ? (sinks - 1) / kKv4Tile + 1 : 0;
  s.sink = st < s.first ? st : s.first;
  s.n = s.sink + end - s.first;
  return s;
}

// KV heads of a slot that run.
SVL_DEVINL int slot_heads(const Kv4Attn& a, int slot) {
  if (!a.gate.group_gate) return a.c.kv;
  int n = 0;
  for (int g = 0; g < a.gate.G; ++g) n += gate_on(a.gate, slot, g) ? a.c.kv / a.gate.G : 0;
  return n;
}
// The i-th of them.
SVL_DEVINL int slot_head(const Kv4Attn& a, int slot, int i) {
  if (!a.gate.group_gate) return i;
  const int per = a.c.kv / a.gate.G;
  for (int g = 0; g < a.gate.G; ++g) {
    if (!gate_on(a.gate, slot, g)) continue;
    if (i < per) return g * per + i;
    i -= per;
  }
  return 0;
}

// A walk over the row of all tiles: where the next tile is, how many the item has left, after how many it goes on
// behind the sinks.
struct Walk {
  const uint8_t* src;
  int p0, left, jump;
  int slot, item, items, head, start;
  Span span;
};
// `tile`: of the item
SVL_DEVINL void walk_item(const AttnParams& p, Walk& w, int tile) {
  w.head = slot_head(p.a, w.slot, p.col_tiles == 1 ? w.item : w.item / p.col_tiles);
  const int at = tile < w.span.sink ? tile : w.span.first + tile - w.span.sink;
  w.left = w.span.n - tile;
  w.jump = tile < w.span.sink ? w.span.sink - tile : 0;
  w.p0 = at * kKv4Tile;
  w.src = kv4_tile(p.a.c, w.slot, w.head, at);
}
SVL_DEVINL void walk_slot(const AttnParams& p, Walk& w) {
  w.items = slot_heads(p.a, w.slot) * p.col_tiles;
  w.span = slot_span(p.a, w.slot);
  w.start = p.a.start[w.slot];
}
// (only while there is a next tile)
template <int TB>
SVL_DEVINL void walk_next(const AttnParams& p, Walk& w) {
  if (--w.left > 0) {
    const int skip = --w.jump == 0 ? w.span.first - w.span.sink + 1 : 1;
    w.p0 += skip * kKv4Tile;
    w.src += static_cast<int64_t>(skip) * TB;
    return;
  }
  if (++w.item >= w.items) {
    w.item = 0;
    do {
      ++w.slot;
      walk_slot(p, w);
    } while (w.items == 0);
  }
  walk_item(p, w, 0);
}

SVL_DEVINL void cp16(uint32_t smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(gmem) : "memory");
}
SVL_DEVINL void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
SVL_DEVINL void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// D = A B + C, 16 x 8 x 16, float32 sums, float16 or bf16 operands.
SVL_DEVINL void mma16816_f16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1,
                             float c0, float c1, float c2, float c3) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
SVL_DEVINL void mma16816_bf16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit values, two neighbours of a row per lane, transposed.
SVL_DEVINL uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
SVL_DEVINL uint32_t pack_f16x2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
SVL_DEVINL float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
SVL_DEVINL float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
SVL_DEVINL __nv_bfloat162 as_bf16x2(uint32_t u) { return *reinterpret_cast<__nv_bfloat162*>(&u); }
SVL_DEVINL uint32_t bits_of(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }
constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;
// The lowest nibble of each half of a word, less 8, as bf16. `k128`: 128 in both halves, in a register (with a second
// constant, mask and sum would take an instruction each).
SVL_DEVINL uint32_t v_codes(uint32_t x, uint32_t k128) {
  uint32_t y;
  asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;" : "=r"(y) : "r"(x), "r"(k128));  // 128 + n
  return bits_of(__hadd2(as_bf16x2(y), as_bf16x2(0xc308c308u)));                // -136
}
SVL_DEVINL uint32_t bits_below(int n) { return n <= 0 ? 0u : (n >= 32 ? ~0u : (1u << n) - 1u); }
SVL_DEVINL float max_quads(float x) {  // over the eight lanes that share lane % 4
#pragma unroll
  for (int off = 4; off <= 16; off <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
  return x;
}

template <int J>
struct Words {
  uint32_t w[J];
};
template <int J>
SVL_DEVINL Words<J> lds_words(const uint8_t* p) {
  Words<J> r;
  if constexpr (J == 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    r.w[0] = u.x;
    r.w[1] = u.y;
    r.w[2] = u.z;
    r.w[3] = u.w;
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    r.w[0] = u.x;
    r.w[1] = u.y;
  }
  return r;
}

// The codes of two words (of pairs of rows 8 apart) as operands, nibble by nibble.
SVL_DEVINL void v_operands(uint32_t v0, uint32_t v1, uint32_t k128, uint32_t (*c)[2]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    c[k][0] = v_codes(v0 >> (4 * k), k128);
    c[k][1] = v_codes(v1 >> (4 * k), k128);
  }
}

// O^T += V^T P over 16 positions, up to eight columns: weights hi + lo of the positions 2 t, 2 t + 1 ([0]) and those
// + 8 ([1]) of the operand's column, V's words and scales of the same. MASK: `keep` is 0 at the positions that the
// column does not see, which do not count whatever their scales.
template <int J, bool MASK>
SVL_DEVINL void weighted_rows(float (*o)[2][4], const uint32_t* hi, const uint32_t* lo, const uint32_t* keep,
                              const Words<J>& u0, const Words<J>& u1, const Words<J>& v0, const Words<J>& v1,
                              uint32_t k128) {
#pragma unroll
  for (int j = 0; j < J; ++j) {
    // times the scales: the rounded product, and what it leaves
    uint32_t ph[2], pl[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const __nv_bfloat162 u = as_bf16x2(x ? u1.w[j] : u0.w[j]), w = as_bf16x2(hi[x]);
      const __nv_bfloat162 prod = __hmul2(w, u);
      ph[x] = bits_of(prod);
      pl[x] = bits_of(__hfma2(as_bf16x2(lo[x]), u, __hfma2(w, u, __hneg2(prod))));
      if (MASK) {
        ph[x] &= keep[x];
        pl[x] &= keep[x];
      }
    }
    uint32_t c[4][2];
    v_operands(v0.w[j], v1.w[j], k128, c);
#pragma unroll
    for (int k = 0; k < 2; ++k) mma16816_bf16(o[j][k], c[k][0], c[k + 2][0], c[k][1], c[k + 2][1], ph[0], ph[1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) mma16816_bf16(o[j][k], c[k][0], c[k + 2][0], c[k][1], c[k + 2][1], pl[0], pl[1]);
  }
}

// The row of a column, column / heads per KV head (exact: with half a column added the quotient is at least 2^-17 off
// an integer, and there are at most 16 rows and 2^16 heads).
SVL_DEVINL int column_row(const AttnParams& p, int col) {
  return static_cast<int>((static_cast<float>(col) + 0.5f) * p.inv_grp);
}

// Writes four neighbouring output dimensions of column `col` of an item.
SVL_DEVINL void store_out(const AttnParams& p, int slot, int head, int col, int d, float4 o) {
  const int r = column_row(p, col), h = head * p.grp + col - r * p.grp;
  __nv_bfloat16* out = p.a.out + (static_cast<int64_t>(slot) * p.a.rows + r) * p.a.ldo + h * p.a.c.dh + d;
  *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
}

// A part of an item holds, per column, the output of its positions alone (ncols *
// d_head floats), then the maximum (times log2 e) and the sum of their weights.
static int part_floats(int ncols, int dh) { return (ncols * (dh + 2) + 3) & ~3; }  // (whole float4s)

SVL_DEVINL void add_scaled(float4& o, float f, float4 x) {
  o.x = fmaf(f, x.x, o.x);
  o.y = fmaf(f, x.y, o.y);
  o.z = fmaf(f, x.z, o.z);
  o.w = fmaf(f, x.w, o.w);
}
// The weight 2^(m - M) l of a part beside the others' maximum M (0: it saw nothing).
SVL_DEVINL float part_weight(float m, float l, float M) { return l == 0.f ? 0.f : l * ex2(m - M); }

// NW: warps, NS: stages of a warp's ring. MODE: 0 for items of one column, 1 for up to four, 2 for up to eight.
// In modes 1 and 2 column c is column 2 (c % 4) + c / 4 of the operands, so that a lane's accumulators hold columns t
// (x = 0) and 4 + t (x = 1); in mode 1 the other operand column of a pair holds the lower halves of the scaled weights.
// In mode 0 the operands' columns 2 j and 2 j + 1 belong to group j of 32 dimensions: of q they hold that group alone,
// so that one chain of products gives lane t the sum of group t; of the weights the halves scaled for that group, so
// that one operand serves all dimensions, of whose sums lane t holds those of group t.
template <int DH, int NS, int NW, int MODE, bool CLUSTER>
__global__ void __launch_bounds__(NW * 32, 1) kv4_attn_kernel(AttnParams p, int slot_floats) {
  constexpr int J = DH / 32, TB = kv4_tile_bytes(DH), NT = MODE == 2 ? 2 : 1;
  constexpr int kAttnWarps = NW, kAttnThreads = NW * 32;
  static_assert(NW <= 16, "sums over the warps take 16 lanes");
  extern __shared__ __align__(128) uint8_t smem[];  // per warp: ring of NS tiles; then per warp a part
  __shared__ int warp_sum[kAttnWarps], prefix[kAttnThreads];
  __shared__ int4 tile_meta[kAttnWarps][NS];  // {first position, bit 0: first tile of its item, bit 1: last; slot,
                                              // item}
  __shared__ int4 tile_item[kAttnWarps][NS];  // {KV head, start of the slot, tiles of the item left after it, -}
  __shared__ int4 w_meta[kAttnWarps];   // {slot, item of the part in the ring (-1: none), state of the other part
                                        // (1: goes on, 2: ends), tiles of the ring's item left}
  __shared__ int4 w_first[kAttnWarps];  // slot, item and KV head of that other part; KV head of the ring's
  const Kv4Attn& a = p.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, t = lane & 3;
  uint8_t* ring = smem + warp * (NS * TB);
  float* first_part = reinterpret_cast<float*>(smem + kAttnWarps * (NS * TB)) + warp * slot_floats;
  float* last_part = reinterpret_cast<float*>(ring);
  pdl_begin(CLUSTER && a.late);

  // ---- this warp's share of all tiles; in a cluster, of those of its item
  int total, cta_tiles, index, sums = 0, per = 0;
  const int own = CLUSTER ? blockIdx.x / p.run : 0, own_slot = own / (a.c.kv * p.col_tiles);
  const int own_item = own % (a.c.kv * p.col_tiles);
  Walk req;
  if constexpr (CLUSTER) {
    req.slot = own_slot;
    req.item = own_item;
    walk_slot(p, req);
    if (req.item >= req.items) return;  // (the whole cluster)
    total = req.span.n;
    cta_tiles = max((total + p.run - 1) / p.run, 4);  // (10 tiles: 4 6.5 us, 6 6.7, 12 6.9)
    index = static_cast<int>(cluster_rank());
    if (lane == 0) w_meta[warp] = make_int4(-1, 0, 0, 0);
    __syncwarp();
  } else {
    per = (a.c.n_slots + kAttnThreads - 1) / kAttnThreads;
    {
      const int s0 = min(tid * per, a.c.n_slots), s1 = min(s0 + per, a.c.n_slots);
      int incl = 0;
      for (int s = s0; s < s1; ++s) incl += slot_heads(a, s) * p.col_tiles * slot_span(a, s).n;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += x;
      }
      prefix[tid] = incl;
      if (lane == 31) warp_sum[warp] = incl;
      if (tid < kAttnWarps) w_meta[tid] = make_int4(-1, 0, 0, 0);
    }
    __syncthreads();
    sums = lane < kAttnWarps ? warp_sum[lane] : 0;
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, sums, off);
      if (lane >= off) sums += x;
    }
    total = __shfl_sync(0xffffffffu, sums, kAttnWarps - 1);
    cta_tiles = max((total + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x), p.min_tiles);
    index = blockIdx.x;
  }
  const int cta0 = static_cast<int>(min(static_cast<int64_t>(total), static_cast<int64_t>(cta_tiles) * index));
  const int cta1 = total - cta0 < cta_tiles ? total : cta0 + cta_tiles;
  const int share = (cta1 - cta0) / kAttnWarps, more = (cta1 - cta0) % kAttnWarps;  // (the first `more`: one more)
  const int last = min(cta1 - cta0, kAttnWarps) - 1;                                // last warp with tiles
  auto warp_tile = [&](int w) { return cta0 + w * share + min(w, more); };
  const int w0 = warp_tile(warp), n = share + (warp < more ? 1 : 0);

  // ---- the tiles
  if (n > 0) {
    int asked = 0;
    if constexpr (CLUSTER) {
      walk_item(p, req, w0);
    } else {
      // the thread's share of the slots that holds tile w0, the slot, the item
      const int wi = __popc(__ballot_sync(0xffffffffu, lane < kAttnWarps && sums <= w0));
      const int base = wi > 0 ? __shfl_sync(0xffffffffu, sums, wi - 1) : 0;
      const int li = __popc(__ballot_sync(0xffffffffu, base + prefix[wi * 32 + lane] <= w0));
      int rest = w0 - base - (li > 0 ? prefix[wi * 32 + li - 1] : 0);
      req.slot = (wi * 32 + li) * per;
      for (walk_slot(p, req); rest >= req.items * req.span.n; walk_slot(p, req)) {
        rest -= req.items * req.span.n;
        ++req.slot;
      }
      req.item = rest / req.span.n;
      walk_item(p, req, rest - req.item * req.span.n);
    }
    const uint32_t ring_s = smem_u32(ring);
    int ask_stage = 0;
    auto request = [&]() {
#pragma unroll
      for (int i = 0; i < (TB / 16 + 31) / 32; ++i) {
        const int c = i * 32 + lane;
        if (TB / 16 % 32 == 0 || c < TB / 16) cp16(ring_s + ask_stage * TB + c * 16, req.src + c * 16);
      }
      if (lane == 0) {
        tile_meta[warp][ask_stage] =
            make_int4(req.p0, (req.left == req.span.n ? 1 : 0) | (req.left == 1 ? 2 : 0), req.slot, req.item);
        tile_item[warp][ask_stage] = make_int4(req.head, req.start, req.left - 1, 0);
      }
      ask_stage = ask_stage + 1 == NS ? 0 : ask_stage + 1;
      if (++asked < n) walk_next<TB>(p, req);
    };
#pragma unroll
    for (int k = 0; k < NS - 1; ++k) {
      if (asked < n) request();
      cp_commit();
    }
    __syncwarp();
    uint32_t q[J][4];
    float qsum[MODE == 0 ? 1 : J][NT], factor[NT], m[NT], l[NT], o[J][2][4];
    int end[NT], low[NT];
    int stage = 0, col0 = 0, whole_lo = 0, whole_hi = 0;
    uint32_t k128;
    asm volatile("mov.b32 %0, 0x43004300;" : "=r"(k128));
    bool started = false;
    for (int i = 0; i < n; ++i) {
      const int4 meta = tile_meta[warp][stage];
      if (i == 0 || (meta.y & 1)) {
        // a new item: its columns' queries as operands
        started = meta.y & 1;
        const int4 at = tile_item[warp][stage];
        col0 = p.col_tiles == 1 ? 0 : meta.w % p.col_tiles * kCols;
        const int cols = min(kCols, p.columns - col0);
        constexpr int C = MODE == 0 ? 1 : J;  // groups of q that a lane has
        // operand column g: the column's query, in mode 0 (even g) that of group g / 2
        const int col = MODE == 0 ? 0 : 4 * (g & 1) + (g >> 1);
        const bool has = MODE == 0 ? !(g & 1) && g < 2 * J : col < cols;
        uint4 raw[C];
#pragma unroll
        for (int j = 0; j < C; ++j) raw[j] = make_uint4(0, 0, 0, 0);
        if (has) {
          const int r = column_row(p, col0 + col), h = at.x * p.grp + col0 + col - r * p.grp;
          const uint4* src = reinterpret_cast<const uint4*>(
              a.q + (static_cast<int64_t>(meta.z) * a.rows + r) * a.ldq + h * DH + (MODE == 0 ? 16 * g : 0) + 8 * t);
#pragma unroll
          for (int j = 0; j < C; ++j) raw[j] = src[4 * j];
        }
        uint32_t big = 0;  // largest magnitude's bits
#pragma unroll
        for (int j = 0; j < C; ++j) {
          const uint32_t u[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) big = max(big, max(u[k] & 0x7fffu, u[k] >> 16 & 0x7fffu));
        }
        if (MODE == 0) {
          big = __reduce_max_sync(0xffffffffu, big);
        } else {
          big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
          big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
        }
        // times a power of two that takes it to [2^14, 2^15)
        const uint32_t eb = min(max(big >> 7, 14u), 254u);
        const float up = __uint_as_float((268 - eb) << 23), up4 = up * 0.0625f;
        float f = a.scale * 1.4426950408889634f * 1024.f * __uint_as_float(eb << 23);
        // Where that is past float32's range in any column, all have its root, of scale's sign, and scores are multiplied
        // by it twice (2^(eb - 127) as 2^odd times the square of a power of two; sqrt(log2 e) = 1.2011...).
        const bool wide = __any_sync(0xffffffffu, isinf(f) && big < 0x7f80u);
        if (wide) {
          const uint32_t odd = ~eb & 1u;
          f = sqrtf(fabsf(a.scale)) * (odd ? 1.6986436005760381f : 1.2011224087864498f) * 32.f *
              __uint_as_float((127 + eb - odd) / 2 << 23);
          f = copysignf(f, a.scale);
        }
        if (big >= 0x7f80u) f = NAN;  // a q that is not finite
#pragma unroll
        for (int j = 0; j < C; ++j) {
          const uint32_t u[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};  // dimensions 2 k, 2 k + 1 of the eight
          const uint32_t y[4] = {pack_f16x2(bf16_lo(u[0]) * up, bf16_lo(u[2]) * up),      // 0, 4
                                 pack_f16x2(bf16_lo(u[1]) * up, bf16_lo(u[3]) * up),      // 2, 6
                                 pack_f16x2(bf16_hi(u[0]) * up4, bf16_hi(u[2]) * up4),    // 1, 5
                                 pack_f16x2(bf16_hi(u[1]) * up4, bf16_hi(u[3]) * up4)};   // 3, 7
          float sum = 0.f;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&y[k]));
            sum += k < 2 ? z.x + z.y : 16.f * (z.x + z.y);
            if (MODE != 0) q[j][k] = y[k];
          }
          if (MODE == 0) {
#pragma unroll
            for (int i = 0; i < J; ++i)
#pragma unroll
              for (int k = 0; k < 4; ++k) q[i][k] = g == 2 * i ? y[k] : 0;
          }
          sum += __shfl_xor_sync(0xffffffffu, sum, 1);
          sum += __shfl_xor_sync(0xffffffffu, sum, 2);
          // (lane 8 t + 4 x holds operand column 2 t + x, whose accumulators are this lane's)
#pragma unroll
          for (int x = 0; x < NT; ++x) qsum[j][x] = __shfl_sync(0xffffffffu, sum * (-8.f / 16777216.f), 8 * t + 4 * x);
        }
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          factor[x] = MODE == 0 ? f : __shfl_sync(0xffffffffu, f, 8 * t + 4 * x);
          const int c = MODE == 0 ? 0 : 4 * x + t;
          const int64_t pos = static_cast<int64_t>(at.y) + column_row(p, col0 + c);
          // (-1: no such column)
          end[x] = c >= cols ? -1 : (pos >= 0 && pos < a.c.max_len ? static_cast<int>(pos) + 1 : 0);
          low[x] = a.window > 0 && end[x] > a.window ? end[x] - a.window : 0;
          m[x] = -INFINITY;
          l[x] = 0.f;
        }
        // what every column sees: [whole_lo, whole_hi), and below whole_hi the sinks
        {
          int lo = low[0], hi = end[0] < 0 ? 0x7fffffff : end[0];
          if (NT == 2) {
            lo = max(lo, low[NT - 1]);
            hi = min(hi, end[NT - 1] < 0 ? 0x7fffffff : end[NT - 1]);
          }
          whole_lo = MODE == 0 ? lo : __reduce_max_sync(0xffffffffu, lo);
          whole_hi = MODE == 0 ? hi : __reduce_min_sync(0xffffffffu, hi);
          // (an item whose factor is a root has no whole tiles: -1 says so, and costs the others no register)
          if (wide) whole_hi = -1;
        }
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int k = 0; k < 8; ++k) o[j][k >> 2][k & 3] = 0.f;
      }

      cp_wait<NS - 2>();
      __syncwarp();  // the tile is here for every lane, and the one before has been read by all
      if (asked < n) request();
      cp_commit();
      uint8_t* tile = ring + stage * TB;
      const int p0 = meta.x;
      const bool whole = p0 <= whole_hi - kKv4Tile && (p0 >= whole_lo || p0 <= a.sinks - kKv4Tile);

      // scores of the tile's 32 positions: rows g and g + 8 of both halves
      float s[2][2][NT];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Words<J> wa = lds_words<J>(tile + (64 * h + lane) * J * 4);
        const Words<J> wb = lds_words<J>(tile + (64 * h + 32 + lane) * J * 4);
        if constexpr (MODE == 0) {
          float d[4] = {qsum[0][0], 0.f, qsum[0][0], 0.f};
#pragma unroll
          for (int j = 0; j < J; ++j) {
            const uint32_t u = wa.w[j], v = wb.w[j], u8 = u >> 8, v8 = v >> 8;
            mma16816_f16(d, u & kLow, v & kLow, u8 & kLow, v8 & kLow, q[j][0], q[j][1], d[0], d[1], d[2], d[3]);
            mma16816_f16(d, u & kHigh, v & kHigh, u8 & kHigh, v8 & kHigh, q[j][2], q[j][3], d[0], d[1], d[2], d[3]);
          }
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float x = 0.f;
            if (t < J) {
              const int at = (16 * h + 8 * r + g) * J + t;
              const uint32_t u = reinterpret_cast<const uint16_t*>(tile + kv4_k_scales(DH))[at];
              x = bf16_lo(u) * d[2 * r];
            }
            x += __shfl_xor_sync(0xffffffffu, x, 1);
            s[h][r][0] = x + __shfl_xor_sync(0xffffffffu, x, 2);
          }
        } else {
          const uint8_t* sk = tile + kv4_k_scales(DH) + (16 * h + g) * J * 2;
          uint32_t ka[J / 2], kb[J / 2];
#pragma unroll
          for (int k = 0; k < J / 2; ++k) {
            ka[k] = reinterpret_cast<const uint32_t*>(sk)[k];
            kb[k] = reinterpret_cast<const uint32_t*>(sk + 8 * J * 2)[k];
          }
#pragma unroll
          for (int j = 0; j < J; ++j) {
            const uint32_t u = wa.w[j], v = wb.w[j], u8 = u >> 8, v8 = v >> 8;
            float d[4];
            constexpr int X = NT - 1;
            const float c1 = NT == 2 ? qsum[j][X] : 0.f;
            mma16816_f16(d, u & kLow, v & kLow, u8 & kLow, v8 & kLow, q[j][0], q[j][1], qsum[j][0], c1, qsum[j][0], c1);
            mma16816_f16(d, u & kHigh, v & kHigh, u8 & kHigh, v8 & kHigh, q[j][2], q[j][3], d[0], d[1], d[2], d[3]);
            const float fa = j & 1 ? bf16_hi(ka[j / 2]) : bf16_lo(ka[j / 2]);
            const float fb = j & 1 ? bf16_hi(kb[j / 2]) : bf16_lo(kb[j / 2]);
#pragma unroll
            for (int x = 0; x < NT; ++x) {
              s[h][0][x] = j ? fmaf(fa, d[x], s[h][0][x]) : fa * d[x];
              s[h][1][x] = j ? fmaf(fb, d[x + 2], s[h][1][x]) : fb * d[x + 2];
            }
          }
        }
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          s[h][0][x] *= factor[x];
          s[h][1][x] *= factor[x];
        }
      }
      uint32_t sight[NT];  // bit: the column sees the position of this lane's row 8 k + g, at 8 k
#pragma unroll
      for (int x = 0; x < NT; ++x) sight[x] = ~0u;
      if (!whole) {
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          const float again = whole_hi < 0 ? fabsf(factor[x]) : 1.f;
          sight[x] = (bits_below(end[x] - p0) & ~bits_below(low[x] - p0)) | bits_below(min(a.sinks, end[x]) - p0);
          sight[x] >>= g;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            s[k >> 1][k & 1][x] = sight[x] >> (8 * k) & 1u ? s[k >> 1][k & 1][x] * again : -INFINITY;
        }
      }
      // the running maximum moves when it is passed by more than a factor of two
      float top[NT];
      bool moves = false;
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        top[x] = max_quads(fmaxf(fmaxf(s[0][0][x], s[0][1][x]), fmaxf(s[1][0][x], s[1][1][x])));
        moves |= top[x] > m[x] + 1.f;
      }
      if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          const float mn = fmaxf(m[x], top[x]);
          const float f = mn == -INFINITY ? 1.f : ex2(m[x] - mn);
          m[x] = mn;
          l[x] *= f;
#pragma unroll
          for (int j = 0; j < J; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              o[j][k][x] *= f;
              o[j][k][x + 2] *= f;
              if (NT == 1) {
                o[j][k][1] *= f;
                o[j][k][3] *= f;
              }
            }
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Words<J> v0 = lds_words<J>(tile + kv4_v_codes(DH) + (64 * h + lane) * J * 4);
        const Words<J> v1 = lds_words<J>(tile + kv4_v_codes(DH) + (64 * h + 32 + lane) * J * 4);
        if constexpr (MODE == 0) {
          uint32_t b[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float w = ex2(s[h][r][0] - (m[0] == -INFINITY ? 0.f : m[0]));
            l[0] += w;
            float x = 0.f;
            if (t < J) {
              // the lane's row and group
              const int at = ((8 * h + 4 * r + (g >> 1)) * J + t) * 2 + (g & 1);
              const uint32_t u = reinterpret_cast<const uint16_t*>(tile + kv4_v_scales(DH))[at];
              x = w * bf16_lo(u);
            }
            if (!whole && !(sight[0] >> (16 * h + 8 * r) & 1u)) x = 0.f;  // not in sight: its scale does not matter
            const float hi = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
            b[r] = transpose8(pack_bf16x2(hi, x - hi));
          }
#pragma unroll
          for (int j = 0; j < J; ++j) {
            uint32_t c[4][2];
            v_operands(v0.w[j], v1.w[j], k128, c);
            mma16816_bf16(o[j][0], c[0][0], c[2][0], c[0][1], c[2][1], b[0], b[1]);
            mma16816_bf16(o[j][1], c[1][0], c[3][0], c[1][1], c[3][1], b[0], b[1]);
          }
        } else if constexpr (MODE == 1) {
          float w[2];
          Words<J> u[2];  // scales of this lane's rows and their neighbours
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            w[r] = ex2(s[h][r][0] - (m[0] == -INFINITY ? 0.f : m[0]));
            l[0] += w[r];
            u[r] = lds_words<J>(tile + kv4_v_scales(DH) + (8 * h + 4 * r + (g >> 1)) * J * 4);
            if (!whole && !(sight[0] >> (16 * h + 8 * r) & 1u)) {  // not in sight: as above
#pragma unroll
              for (int j = 0; j < J; ++j) u[r].w[j] = 0;
            }
          }
#pragma unroll
          for (int j = 0; j < J; ++j) {
            uint32_t b[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const float x = w[r] * __uint_as_float(__byte_perm(u[r].w[j], 0, g & 1 ? 0x3244 : 0x1044));
              const float hi = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
              b[r] = transpose8(pack_bf16x2(hi, x - hi));
            }
            uint32_t c[4][2];
            v_operands(v0.w[j], v1.w[j], k128, c);
            mma16816_bf16(o[j][0], c[0][0], c[2][0], c[0][1], c[2][1], b[0], b[1]);
            mma16816_bf16(o[j][1], c[1][0], c[3][0], c[1][1], c[3][1], b[0], b[1]);
          }
        } else {
          // weights as pairs of bf16 numbers, positions 2 t, 2 t + 1 and those + 8 of the operand's column
          uint32_t hi[2], lo[2], keep[2];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float w[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              w[x] = ex2(s[h][r][x % NT] - (m[x % NT] == -INFINITY ? 0.f : m[x % NT]));
              l[x % NT] += w[x];
            }
            const uint32_t u = pack_bf16x2(w[0], w[1]);
            hi[r] = transpose8(u);
            lo[r] = transpose8(pack_bf16x2(w[0] - bf16_lo(u), w[1] - bf16_hi(u)));
            if (!whole) {
              const int k = 16 * h + 8 * r;
              keep[r] = transpose8((sight[0] >> k & 1u ? 0xffffu : 0u) | (sight[NT - 1] >> k & 1u ? 0xffff0000u : 0u));
            }
          }
          const Words<J> u0 = lds_words<J>(tile + kv4_v_scales(DH) + (8 * h + t) * J * 4);
          const Words<J> u1 = lds_words<J>(tile + kv4_v_scales(DH) + (8 * h + 4 + t) * J * 4);
          if (whole) weighted_rows<J, false>(o, hi, lo, keep, u0, u1, v0, v1, k128);
          else weighted_rows<J, true>(o, hi, lo, keep, u0, u1, v0, v1, k128);
        }
      }

      stage = stage + 1 == NS ? 0 : stage + 1;
      const bool ended = meta.y & 2;
      if (ended || i + 1 == n) {
        // the item's end, or this warp's
        const int4 at = tile_item[warp][stage == 0 ? NS - 1 : stage - 1];
        float* part = started ? last_part : first_part;
        if (started && !ended) {
          cp_wait<0>();
          __syncwarp();  // the ring is free
        }
#pragma unroll
        for (int x = 0; x < NT; ++x) {
#pragma unroll
          for (int off = 4; off <= 16; off <<= 1) l[x] += __shfl_xor_sync(0xffffffffu, l[x], off);
          if (end[x] < 0) continue;
          const float inv = l[x] == 0.f ? 0.f : __fdividef(1.f, l[x]);
          const int col = MODE == 0 ? 0 : 4 * x + t;
          if (!(started && ended) && lane < (MODE == 0 ? 1 : 4)) {
            part[p.ncols * DH + 2 * col] = m[x];
            part[p.ncols * DH + 2 * col + 1] = l[x];
          }
          if constexpr (MODE == 0) {
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int j = 0; j < J; ++j)
              if (t == j)
                y = make_float4(o[j][0][0] + o[j][0][1], o[j][1][0] + o[j][1][1], o[j][0][2] + o[j][0][3],
                                o[j][1][2] + o[j][1][3]);
            if (t >= J) continue;
            y = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
            if (started && ended) store_out(p, meta.z, at.x, 0, 32 * t + 4 * g, y);
            else *reinterpret_cast<float4*>(part + 32 * t + 4 * g) = y;
          } else {
#pragma unroll
            for (int j = 0; j < J; ++j) {
              float4 y = make_float4(o[j][0][x], o[j][1][x], o[j][0][x + 2], o[j][1][x + 2]);
              if (MODE == 1) y = make_float4(y.x + o[j][0][1], y.y + o[j][1][1], y.z + o[j][0][3], y.w + o[j][1][3]);
              y = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
              if (started && ended) store_out(p, meta.z, at.x, col0 + col, 32 * j + 4 * g, y);
              else *reinterpret_cast<float4*>(part + col * DH + 32 * j + 4 * g) = y;
            }
          }
        }
        if (lane == 0 && !started) {
          w_meta[warp].z = ended ? 2 : 1;
          w_first[warp].x = meta.z;
          w_first[warp].y = meta.w;
          w_first[warp].z = at.x;
        }
        if (lane == 0 && started && !ended) {
          w_meta[warp].x = meta.z;
          w_meta[warp].y = meta.w;
          w_meta[warp].w = at.z;
          w_first[warp].w = at.x;
        }
      }
      __syncwarp();  // the next tile's meta
    }
    cp_wait<0>();
  }
  __syncthreads();

  // ---- items that several warps share are put together, (item, column) by (item, column)
  // (a cluster's CTAs have a part of one item, kept in shared memory for the others to read)
  float* out_part = CLUSTER ? reinterpret_cast<float*>(smem + kAttnWarps * (NS * TB + slot_floats * 4))
                            : p.part + static_cast<size_t>(blockIdx.x) * 2 * slot_floats;
  const int next_part = CLUSTER ? 0 : slot_floats;  // where the part that the next CTA goes on with is
  const int4 wm = lane <= last ? w_meta[lane] : make_int4(-1, 0, 0, 0);
  const uint32_t starts = __ballot_sync(0xffffffffu, wm.x >= 0);    // warps whose ring holds an item's start
  const uint32_t goes_on = __ballot_sync(0xffffffffu, wm.z == 1);   // warps within an item
  uint32_t ends = __ballot_sync(0xffffffffu, wm.z == 2);            // warps with an item's end
  if (!CLUSTER && tid == 0) {
    // the item that started here and goes on in the next CTA, and how many CTAs it is in
    int4 mt = make_int4(-1, 0, 0, 0);
    const int v = 31 - __clz(starts);
    if (starts && !(ends >> v >> 1)) {
      // (the rest of the start's part is in the warps after it)
      const int left = w_meta[v].w - (cta1 - warp_tile(v + 1));
      if (left > 0) mt = make_int4(w_meta[v].x, w_meta[v].y, w_first[v].w, 1 + (left + cta_tiles - 1) / cta_tiles);
    }
    p.meta[blockIdx.x] = mt;
  }
  if (last >= 0 && (goes_on >> last & 1u)) ends |= 1u << last;
  auto part_of = [&](int w, bool first) {
    return first ? reinterpret_cast<const float*>(smem + kAttnWarps * (NS * TB)) + w * slot_floats
                 : reinterpret_cast<const float*>(smem + w * (NS * TB));
  };
  int turn = 0;
  for (; ends; ends &= ends - 1) {
    const int to = __ffs(ends) - 1;  // the warp with the item's last part here; its first is the last start before that
    const uint32_t earlier = starts & ((1u << to) - 1u);
    const bool here = earlier != 0;
    const int from = here ? 31 - __clz(earlier) : 0;
    const bool done = here && !(goes_on >> to & 1u);
    const int4 it = w_first[to];
    const int c0 = p.col_tiles == 1 ? 0 : it.y % p.col_tiles * kCols, cols = min(kCols, p.columns - c0);
    for (int col = 0; col < cols; ++col) {
      const bool skip = turn != warp;
      turn = turn + 1 == kAttnWarps ? 0 : turn + 1;
      if (skip) continue;
      float m = -INFINITY, l = 0.f;
      if (lane <= to - from) {
        const float* x = part_of(from + lane, lane > 0 || !here) + p.ncols * DH + 2 * col;
        m = x[0];
        l = x[1];
      }
      float M = m;
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
      const float f = part_weight(m, l, M);
      float L = f;
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) L += __shfl_xor_sync(0xffffffffu, L, off);
      const float inv = L == 0.f ? 0.f : __fdividef(1.f, L);
      M = __shfl_sync(0xffffffffu, M, 0);
      L = __shfl_sync(0xffffffffu, L, 0);
      const float fi = f * __shfl_sync(0xffffffffu, inv, 0);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      const int d = 4 * lane;
      for (int w = from; w <= to; ++w) {
        const float x = __shfl_sync(0xffffffffu, fi, w - from);
        if (d < DH) add_scaled(o, x, *reinterpret_cast<const float4*>(part_of(w, w > from || !here) + col * DH + d));
      }
      if (done) {
        if (d < DH) store_out(p, it.x, it.z, c0 + col, d, o);
      } else {
        float* y = out_part + (here ? next_part : 0);
        if (d < DH) *reinterpret_cast<float4*>(y + col * DH + d) = o;
        if (lane == 0) {
          y[p.ncols * DH + 2 * col] = M;
          y[p.ncols * DH + 2 * col + 1] = L;
        }
      }
    }
  }
  if (last >= 0 && (starts >> last & 1u)) {
    const float* x = part_of(last, false);
    for (int i = tid; i < slot_floats; i += kAttnThreads) out_part[next_part + i] = x[i];
  }
  if constexpr (CLUSTER) {
    // ---- the item's parts: column c by warp c / run of CTA c % run
    const int parts = (total - 1) / cta_tiles + 1, c0 = own_item % p.col_tiles * kCols, col = index + p.run * warp;
    if (parts == 1) return;  // (the whole cluster: the item is done)
    cluster_sync();
    if (col < min(kCols, p.columns - c0)) {
      float m = -INFINITY, l = 0.f;
      if (lane < parts) {
        const float* x = out_part + p.ncols * DH + 2 * col;
        m = ld_cluster(mapa_shared(x, lane));
        l = ld_cluster(mapa_shared(x + 1, lane));
      }
      float M = m;
#pragma unroll
      for (int off = kClusterCtas / 2; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
      const float f = part_weight(m, l, M);
      float L = f;
#pragma unroll
      for (int off = kClusterCtas / 2; off > 0; off >>= 1) L += __shfl_xor_sync(0xffffffffu, L, off);
      const float inv = __shfl_sync(0xffffffffu, L == 0.f ? 0.f : __fdividef(1.f, L), 0);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      const int d = 4 * lane;
#pragma unroll
      for (int i = 0; i < kClusterCtas; ++i) {
        const float x = __shfl_sync(0xffffffffu, f, i) * inv;
        if (d < DH && i < parts) add_scaled(o, x, ld_cluster4(mapa_shared(out_part + col * DH + d, i)));
      }
      if (d < DH) store_out(p, own_slot, slot_head(a, own_slot, own_item / p.col_tiles), c0 + col, d, o);
    }
    cluster_sync();  // the others have read this CTA's part
  }
}

// Items shared by CTAs: block (c, column) puts together the one that starts in CTA c and goes on in others. The warps
// take its parts in turn, each with a running maximum, so that what has to be read is on its way at once. Bound by
// latency: 1.7 to 2.2 us of a call (the last CTA to arrive joining in the first launch took 6 us more).
template <int DH>
__global__ void __launch_bounds__(kMergeThreads) kv4_merge_kernel(AttnParams p, int slot_floats) {
  constexpr int kWarps = kMergeThreads / 32;
  __shared__ float warp_m[kWarps], warp_l[kWarps];
  __shared__ float4 sum[kWarps][32];
  const int c = blockIdx.x, col = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int d = 4 * lane;
  pdl_begin(p.a.late);
  // each warp's first part is read beside the meta that says whether it belongs to the item
  const float* first =
      p.part + (static_cast<size_t>(min(c + warp, static_cast<int>(gridDim.x) - 1)) * 2 + (warp == 0)) * slot_floats;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (d < DH) o = *reinterpret_cast<const float4*>(first + col * DH + d);
  float m = first[p.ncols * DH + 2 * col], l = first[p.ncols * DH + 2 * col + 1];
  const int4 it = p.meta[c];
  const int c0 = p.col_tiles == 1 ? 0 : it.y % p.col_tiles * kCols, n = it.w;
  if (it.x < 0 || c0 + col >= p.columns) return;
  // (o is kept with its weight l: sums of weighted outputs)
  o = make_float4(o.x * l, o.y * l, o.z * l, o.w * l);
  if (warp >= n) {
    m = -INFINITY;
    l = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll 4
  for (int i = warp + kWarps; i < n; i += kWarps) {
    const float* x = p.part + static_cast<size_t>(c + i) * 2 * slot_floats;
    const float xm = x[p.ncols * DH + 2 * col], xl = x[p.ncols * DH + 2 * col + 1];
    const float4 y = d < DH ? *reinterpret_cast<const float4*>(x + col * DH + d) : o;
    const float mn = fmaxf(m, xm), old = part_weight(m, l, mn), f = part_weight(xm, xl, mn);
    const float down = l == 0.f ? 0.f : ex2(m - mn);
    o = make_float4(o.x * down, o.y * down, o.z * down, o.w * down);
    add_scaled(o, f, y);
    l = old + f;
    m = mn;
  }
  sum[warp][lane] = o;
  if (lane == 0) {
    warp_m[warp] = m;
    warp_l[warp] = l;
  }
  __syncthreads();
  if (warp > 0 || d >= DH) return;
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) M = fmaxf(M, warp_m[w]);
  o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (warp_l[w] == 0.f) continue;
    const float f = ex2(warp_m[w] - M);
    L += warp_l[w] * f;
    add_scaled(o, f, sum[w][lane]);
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  store_out(p, it.x, it.z, c0 + col, d, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
}

static int attn_ncols(const Kv4Cache& c, int A, int rows) {
  const int cols = rows * (A / c.kv);
  return cols < kCols ? cols : kCols;
}

size_t kv4_attn_workspace(const Kv4Cache& c, int A, int rows) {
  const size_t floats = part_floats(attn_ncols(c, A, rows), c.dh);
  return kMaxCtas * (2 * floats * sizeof(float) + sizeof(int4));
}

// CTAs of an item's cluster (0: none, the tiles are dealt to all CTAs and a second launch joins them). Clusters need a
// single wave of CTAs: 14 clusters of eight fit the GPU and 16 do not (16 items of 60 tiles: 9.6 us dealt, 13.9 in
// clusters of eight, 9.4 of four), 32 of four and not 38, 76 of two. They save the second launch and lose where a CTA
// has many more tiles than its share of all, or where items differ much in length, which max_len alone bounds here: up
// to three tiles a warp and 14 tiles more. Dealt and in clusters, 28 heads on 4 KV heads: one slot of 1,100 positions
// 9.1 and 7.0 us, of 4,000 9.6 and 9.4; 8 heads on one, 6,000 positions 9.4 and 10.0; seven heads on each of 96 KV
// heads, 1,088 positions 12.1 and 10.9 (a CTA each), of 48, 4,000 positions 15.8 and 16.7 (two each).
static int attn_run(const Kv4Attn& a) {
  const int columns = a.rows * (a.A / a.c.kv), warps = columns == 1 ? 16 : 12;
  const int64_t items = static_cast<int64_t>(a.c.n_slots) * a.c.kv * ((columns + kCols - 1) / kCols);
  int64_t tiles = a.c.tiles;
  if (a.window > 0) {
    const int64_t near = (static_cast<int64_t>(a.window) + a.rows - 2) / kKv4Tile + 2;
    const int64_t seen = near + (a.sinks + static_cast<int64_t>(kKv4Tile) - 1) / kKv4Tile;
    tiles = seen < tiles ? seen : tiles;
  }
  const int run = items * 8 <= 96 ? 8 : items * 4 <= 128 ? 4 : items * 2 <= a.num_sms ? 2 : 1;
  if (items * run > a.num_sms || tiles > 3 * warps * run) return 0;
  return tiles / run <= items * tiles / a.num_sms + 14 ? run : 0;
}
int kv4_attn_launches(const Kv4Attn& a) { return attn_run(a) ? 1 : 2; }

template <int DH, int NS, int NW, int MODE>
static cudaError_t launch_attn(const AttnParams& p, int slot_floats, int grid, cudaStream_t s) {
  // The limit belongs to the kernel, not to the call: every call sets the one for the most columns of its mode, whatever
  // other threads launch meanwhile.
  const int most = part_floats(MODE == 0 ? 1 : MODE == 1 ? 4 : kCols, DH) * 4;
  constexpr int kRings = NW * NS * kv4_tile_bytes(DH);
  int smem = kRings + NW * slot_floats * 4;
  if (p.run) {
    smem += slot_floats * 4;
    const auto kernel = kv4_attn_kernel<DH, NS, NW, MODE, true>;
    const cudaError_t e =
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRings + (NW + 1) * most);
    if (e != cudaSuccess) return e;
    const unsigned items = static_cast<unsigned>(p.a.c.n_slots * p.a.c.kv * p.col_tiles);
    return launch_pdl_cluster(kernel, dim3(items * p.run), NW * 32, smem, p.run, s, p, slot_floats);
  }
  const auto kernel = kv4_attn_kernel<DH, NS, NW, MODE, false>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRings + NW * most);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(grid), NW * 32, smem, s, p, slot_floats);
  if (e != cudaSuccess) return e;
  return launch_pdl(kv4_merge_kernel<DH>, dim3(grid, p.ncols), kMergeThreads, 0, s, p, slot_floats);
}

cudaError_t launch_kv4_attention(const Kv4Attn& a, cudaStream_t s) {
  AttnParams p;
  p.a = a;
  p.ncols = attn_ncols(a.c, a.A, a.rows);
  p.col_tiles = (a.rows * (a.A / a.c.kv) + kCols - 1) / kCols;
  p.run = attn_run(a);
  p.min_tiles = 6;  // (1,900 rows of four KV heads: 2 10.5 us, 4 9.1, 6 9.0, 12 9.8)
  p.grp = a.A / a.c.kv;
  p.columns = a.rows * p.grp;
  p.inv_grp = 1.f / static_cast<float>(p.grp);
  const int slot_floats = part_floats(p.ncols, a.c.dh);
  const int grid = a.num_sms < kMaxCtas ? a.num_sms : kMaxCtas;
  p.meta = static_cast<int4*>(a.ws);
  p.part = reinterpret_cast<float*>(p.meta + kMaxCtas);
  // One column (a head per KV head and one row: the decode step of a model without grouped heads) as mode 0 and as
  // mode 1: 32 heads, 8 slots of 4,000 to 16,000 positions 55.9 and 66.9 us, 16 of 250 to 450 12.1 and 13.3. Four
  // columns as mode 1 and as mode 2: 32 heads on 8, 8 slots of 20,000 to 40,000 positions 55.8 and 61.0 us (d_head 64,
  // 16 heads on 4, 16 slots of 5,000 to 9,000: 15.1 and 17.0). Warps and stages: with 16 warps of 128 registers mode 2
  // takes 44.0 us for 28 heads on 4, 8 slots of 20,000 to 40,000 positions, instead of 37.5.
  if (a.c.dh == 64)
    return p.ncols == 1   ? launch_attn<64, 4, 16, 0>(p, slot_floats, grid, s)
           : p.ncols <= 4 ? launch_attn<64, 4, 12, 1>(p, slot_floats, grid, s)
                          : launch_attn<64, 4, 12, 2>(p, slot_floats, grid, s);
  return p.ncols == 1   ? launch_attn<128, 2, 16, 0>(p, slot_floats, grid, s)
         : p.ncols <= 4 ? launch_attn<128, 3, 12, 1>(p, slot_floats, grid, s)
                        : launch_attn<128, 3, 12, 2>(p, slot_floats, grid, s);
}

}  // namespace svl
