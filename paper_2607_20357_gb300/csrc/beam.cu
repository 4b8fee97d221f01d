// Beam search's selection. A beam w with running score c_w offers, for each id v,
// the candidate x_wv + (c_w - lse_w) with lse_w = log sum_v exp x_wv; a finished beam
// offers itself. The best K of a sample's candidates are taken: larger scores first,
// of equal ones the lower beam's, within a beam the larger logit's, then the lower
// id's. A beam's candidates thus come in the order of its logits: its best K are
// found in the one pass over the row that also sums the exponentials.
//
// Bound by the logits' bytes (4 per id). A row is cut into parts, a block each, so
// that few rows fill the GPU; every warp keeps the K best of what it has seen as a
// sorted list, one key per lane. Few logits ever reach a list: of the warps that a
// block has, each holds at least K / warps logits that are no less than its bar, so
// none under the lowest of these bars is among the K best; the bars start from the
// lanes' maxima of the first chunk. A chunk of 512 logits then costs a warp 16
// comparisons per lane and a vote. Sums of exponentials are kept per lane relative
// to the running maximum, in two float32 numbers. A second launch joins the parts,
// a warp per beam, and takes the sample's best.
//
// Measured: 32 samples of eight beams over 152,064 ids, 16 taken, a tenth of the beams
// finished: 35.2 us (139 MB; 20.5 us at the 6.8 TB/s of a copy), of which the second
// launch takes 4.3 and the upkeep of the lists some 6. One sample of four beams over
// 32,000 ids: 6.9 us, 3.0 of them the second launch.
#include "kv4.cuh"

namespace svl {

constexpr int kBeamWarps = 8, kBeamThreads = kBeamWarps * 32;
constexpr int kChunk = 512;         // logits of a warp's step: 16 per lane
constexpr int kBeamParts = 64;      // most parts of a row

// Orders floats as unsigned integers, -0 like 0.
SVL_DEVINL uint32_t order_bits(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
SVL_DEVINL float from_order_bits(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// Logit and id as one number, never 0: the larger is the better candidate.
SVL_DEVINL uint64_t beam_key(float x, int v) {
  return static_cast<uint64_t>(order_bits(x)) << 32 | (0xffffffffu - static_cast<uint32_t>(v));
}

// The keys that pass into a warp's list (lane i: the i-th best so far, 0 where there are fewer; lanes from K on
// hold keys that fell out).
SVL_DEVINL void list_insert(uint64_t& list, uint64_t key, bool pass, int K, int lane) {
  uint32_t left = __ballot_sync(0xffffffffu, pass);
  while (left) {
    const int src = __ffs(left) - 1;
    left &= left - 1;
    const uint64_t x = __shfl_sync(0xffffffffu, key, src);
    const int pos = __popc(__ballot_sync(0xffffffffu, list > x));
    const uint64_t up = __shfl_up_sync(0xffffffffu, list, 1);
    list = lane < pos ? list : (lane == pos ? x : up);
    // those that still pass
    const uint64_t last = __shfl_sync(0xffffffffu, list, K - 1);
    left &= __ballot_sync(0xffffffffu, key > last);
  }
}

// 32 numbers in descending order over the lanes (bitonic).
SVL_DEVINL uint32_t warp_sort(uint32_t x, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int step = size >> 1; step > 0; step >>= 1) {
      const uint32_t y = __shfl_xor_sync(0xffffffffu, x, step);
      x = ((lane & step) == 0) == ((lane & size) == 0) ? max(x, y) : min(x, y);
    }
  return x;
}

// The 32 largest of two lists (descending over the lanes), descending.
SVL_DEVINL uint64_t list_merge(uint64_t a, uint64_t b, int lane) {
  const uint64_t r = __shfl_xor_sync(0xffffffffu, b, 31);
  uint64_t x = a > r ? a : r;
#pragma unroll
  for (int step = 16; step > 0; step >>= 1) {
    const uint64_t y = __shfl_xor_sync(0xffffffffu, x, step);
    x = ((lane & step) == 0) == (x > y) ? x : y;
  }
  return x;
}

// s + t = a + b exactly
SVL_DEVINL void two_sum(float a, float b, float& s, float& t) {
  s = __fadd_rn(a, b);
  const float z = __fadd_rn(s, -a);
  t = __fadd_rn(__fadd_rn(a, -__fadd_rn(s, -z)), __fadd_rn(b, -z));
}

// exp(x - m); m = -inf: 0
SVL_DEVINL float exp_less(float x, float m) {
  return ex2((x - (m == -INFINITY ? 0.f : m)) * 1.4426950408889634f);
}

// The parts of a row: their K best keys [parts][K] and sums {m, sum exp(x - m)} (the sum NaN where a logit is NaN or
// inf).
struct BeamParts {
  uint64_t* keys;
  float2* sums;
  int parts, part;  // parts of a row, logits of a part (a multiple of kChunk)
};

// Block (row, part). VEC: rows are 16-byte aligned.
template <bool VEC>
__global__ void __launch_bounds__(kBeamThreads) beam_part_kernel(BeamArgs a, BeamParts p) {
  __shared__ uint64_t lists[kBeamWarps][kBeamMaxTake];
  __shared__ float wm[kBeamWarps], ws[kBeamWarps];
  __shared__ volatile uint32_t bars[kBeamWarps];  // of each warp, `each` of its logits are no less (as ordered bits)
  pdl_begin(false);
  const int row = blockIdx.x, part = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool fin = a.finished && a.finished[row];
  const float* x = a.logits + row * a.ld;
  const int v0 = part * p.part, v1 = min(a.V, v0 + p.part);
  float m = -INFINITY, s = 0.f, rest = 0.f;
  uint64_t list = 0, last = 0;  // last: the list's K-th key, in every lane
  const int active = min(kBeamWarps, (v1 - v0 + kChunk - 1) / kChunk), each = (a.K + active - 1) / active;
  uint32_t own = 0;  // K of this warp's logits are no less
  // lane l's k-th value of the chunk at c: id c + 128 (k / 4) + 4 l + k % 4, or c + 32 k + l where rows are not aligned
  auto load = [&](int c, float* y) {
#pragma unroll
    for (int k = 0; k < 16; k += 4) {
      if (VEC) {
        const int v = c + 32 * k + 4 * lane;
        if (v + 4 <= v1) {
          const float4 f = *reinterpret_cast<const float4*>(x + v);
          y[k] = f.x;
          y[k + 1] = f.y;
          y[k + 2] = f.z;
          y[k + 3] = f.w;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) y[k + i] = v + i < v1 ? x[v + i] : -INFINITY;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[k + i] = c + 32 * (k + i) + lane < v1 ? x[c + 32 * (k + i) + lane] : -INFINITY;
      }
    }
  };
  float y[16];
  int c = v0 + warp * kChunk;
  if (c < v1) load(c, y);  // (on its way before it is known whether the beam is finished)
  if (fin) return;
  if (c < v1) {
    float top = y[0];
#pragma unroll
    for (int k = 1; k < 16; ++k) top = fmaxf(top, y[k]);
    const uint32_t sorted = warp_sort(order_bits(top), lane);
    own = __shfl_sync(0xffffffffu, sorted, a.K - 1);
    const uint32_t bar = __shfl_sync(0xffffffffu, sorted, each - 1);
    if (lane == 0) bars[warp] = bar;
  }
  __syncthreads();
  for (; c < v1; c += kBeamWarps * kChunk) {
    float z[16];
    const int next = c + kBeamWarps * kChunk;
#pragma unroll
    for (int k = 0; k < 16; ++k) z[k] = y[k];
    if (next < v1) load(next, y);
    float top = z[0];
#pragma unroll
    for (int k = 1; k < 16; ++k) top = fmaxf(top, z[k]);
    if (top > m) {
      const float f = exp_less(m, top);
      s *= f;
      rest *= f;
      m = top;
    }
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += exp_less(z[k], m);
    float t;
    two_sum(s, sum, s, t);
    rest += t;
    const uint32_t low = max(own, __reduce_min_sync(0xffffffffu, lane < active ? bars[lane] : 0xffffffffu));
    if (!__any_sync(0xffffffffu, top >= from_order_bits(low))) continue;
    bool taken = false;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (!__any_sync(0xffffffffu, z[k] >= from_order_bits(low))) continue;
      const int v = VEC ? c + 128 * (k / 4) + 4 * lane + k % 4 : c + 32 * k + lane;
      const uint64_t key = beam_key(z[k], v);
      const bool pass = v < v1 && z[k] >= from_order_bits(low) && key > last;
      if (!__any_sync(0xffffffffu, pass)) continue;
      list_insert(list, key, pass, a.K, lane);
      last = __shfl_sync(0xffffffffu, list, a.K - 1);
      taken = true;
    }
    if (taken) {
      own = max(own, static_cast<uint32_t>(last >> 32));
      const uint32_t bar = static_cast<uint32_t>(__shfl_sync(0xffffffffu, list, each - 1) >> 32);
      if (lane == 0 && bar > bars[warp]) bars[warp] = bar;
    }
  }
  // ---- the warp's sums, then the block's
  s += rest;
  {
    float M = m;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    s = s * exp_less(m, M);  // (0 times 0 where the lane saw nothing)
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (lane == 0) {
      wm[warp] = M;
      ws[warp] = s;
    }
  }
  if (lane >= a.K) list = 0;  // (of what fell out, nothing is among the best)
#pragma unroll
  for (int n = kBeamWarps / 2; n > 0; n >>= 1) {
    if (warp >= n && warp < 2 * n) lists[warp][lane] = list;
    __syncthreads();
    if (warp < n) list = list_merge(list, lists[warp + n][lane], lane);
  }
  if (warp > 0) return;
  const int64_t at = static_cast<int64_t>(row) * p.parts + part;
  if (lane < a.K) p.keys[at * a.K + lane] = list;
  if (lane == 0) {
    float M = -INFINITY, S = 0.f;
#pragma unroll
    for (int w = 0; w < kBeamWarps; ++w) M = fmaxf(M, wm[w]);
#pragma unroll
    for (int w = 0; w < kBeamWarps; ++w) S += ws[w] * exp_less(wm[w], M);
    p.sums[at] = make_float2(M, S);
  }
}

// Block per sample, warp per beam: its parts joined, then the sample's best K taken one by one.
__global__ void __launch_bounds__(kKv4MaxBeams * 32) beam_join_kernel(BeamArgs a, BeamParts p) {
  __shared__ float cand[kKv4MaxBeams][kBeamMaxTake];
  __shared__ int token[kKv4MaxBeams][kBeamMaxTake];
  __shared__ uint8_t done[kKv4MaxBeams];
  pdl_begin(false);
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int row = blockIdx.x * a.W + w;
  // all that has to be read is on its way at once (a finished beam's parts hold whatever, and do not count)
  const float2* sums = p.sums + static_cast<int64_t>(row) * p.parts;
  const uint64_t* keys = p.keys + static_cast<int64_t>(row) * p.parts * a.K;
  constexpr int kEarly = 8;
  uint64_t early[kEarly];
#pragma unroll
  for (int i = 0; i < kEarly; ++i) early[i] = i < p.parts && lane < a.K ? keys[i * a.K + lane] : 0;
  const float score = a.scores[row];
  const bool fin = a.finished && a.finished[row];
  float M = -INFINITY;
  for (int i = lane; i < p.parts; i += 32) M = fmaxf(M, sums[i].x);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
  if (lane == 0) done[w] = fin;
  float c = -INFINITY;
  int id = lane;
  if (fin) {
    if (lane == 0) c = score;
    id = a.eos;
  } else {
    float S = 0.f;
    for (int i = lane; i < p.parts; i += 32) {
      const float2 x = sums[i];
      S += x.y * exp_less(x.x, M);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) S += __shfl_xor_sync(0xffffffffu, S, off);
    uint64_t list = early[0], last = __shfl_sync(0xffffffffu, list, a.K - 1);
    auto join = [&](uint64_t key) {
      if (!__any_sync(0xffffffffu, key > last)) return;
      list = list_merge(list, key, lane);
      last = __shfl_sync(0xffffffffu, list, a.K - 1);
    };
#pragma unroll
    for (int i = 1; i < kEarly; ++i) join(early[i]);
#pragma unroll 4
    for (int i = kEarly; i < p.parts; ++i) join(lane < a.K ? keys[static_cast<int64_t>(i) * a.K + lane] : 0);
    if (S > 0.f && M < INFINITY) {  // (a NaN sum is not)
      const float lse = M + logf(S);
      id = static_cast<int>(0xffffffffu - static_cast<uint32_t>(list));
      c = from_order_bits(static_cast<uint32_t>(list >> 32)) + (score - lse);
    }
  }
  if (isnan(c)) c = -INFINITY;
  if (lane < a.K) {
    cand[w][lane] = c;
    token[w][lane] = id;
  }
  __syncthreads();
  if (w > 0) return;
  // lane = beam, with the best candidate that is left of it
  int at = 0;
  const bool beam = lane < a.W;
  uint32_t mine = beam ? order_bits(cand[lane][0]) : 0;
  for (int k = 0; k < a.K; ++k) {
    const uint32_t best = __reduce_max_sync(0xffffffffu, mine);
    const int from = __ffs(__ballot_sync(0xffffffffu, beam && mine == best)) - 1;
    if (lane == from) {
      const int64_t o = static_cast<int64_t>(blockIdx.x) * a.K + k;
      const int t = token[lane][at];
      a.scores_out[o] = cand[lane][at];
      a.parent[o] = lane;
      a.token[o] = t;
      if (a.finished_out) a.finished_out[o] = done[lane] || t == a.eos;
      ++at;
      mine = at < a.K ? order_bits(cand[lane][at]) : 0;
    }
  }
}

// Parts of a row. 608 blocks (four on each SM) run at once, and a part costs a block as much as some 8,000 logits more:
// the fewest waves times that, with at most a part for every 4,096 logits or what is left of them (a chunk for each warp of
// a whole one; equal parts can be shorter, so that some of the warps have no chunk: 2,560 logits each of 4,097 to 5,120).
// All rows have as many parts: 256 rows of 152,064 have two each, 512 blocks in one wave.
static BeamParts beam_parts(int S, int W, int V) {
  BeamParts p{};
  const int64_t rows = static_cast<int64_t>(S) * W;
  const int most = (V + 4095) / 4096 < kBeamParts ? (V + 4095) / 4096 : kBeamParts;
  int64_t best = 0;
  for (int n = 1; n <= most; ++n) {
    const int64_t cost = (rows * n + 607) / 608 * ((V + n - 1) / n + 8000);
    if (n > 1 && cost >= best) continue;
    best = cost;
    p.part = ((V + n - 1) / n + kChunk - 1) / kChunk * kChunk;
  }
  p.parts = (V - 1) / p.part + 1;
  return p;
}

size_t beam_workspace(int S, int W, int V, int K) {
  const size_t n = static_cast<size_t>(S) * W * beam_parts(S, W, V).parts;
  return n * K * sizeof(uint64_t) + n * sizeof(float2);
}

cudaError_t launch_beam_select(const BeamArgs& a, cudaStream_t s) {
  BeamParts p = beam_parts(a.S, a.W, a.V);
  p.keys = static_cast<uint64_t*>(a.ws);
  p.sums = reinterpret_cast<float2*>(p.keys + static_cast<size_t>(a.S) * a.W * p.parts * a.K);
  const bool vec = (a.ld & 3) == 0 && (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0;
  const dim3 grid(a.S * a.W, p.parts);
  const cudaError_t e = vec ? launch_pdl(beam_part_kernel<true>, grid, kBeamThreads, 0, s, a, p)
                            : launch_pdl(beam_part_kernel<false>, grid, kBeamThreads, 0, s, a, p);
  if (e != cudaSuccess) return e;
  return launch_pdl(beam_join_kernel, dim3(a.S), a.W * 32, 0, s, a, p);
}

}  // namespace svl
