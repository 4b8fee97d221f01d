// Beam search's selection. A beam w with running score c_w offers, for each id v,
// the candidate x_wv + (c_w - lse_w) with lse_w = log sum_v exp x_wv; a finished beam
// offers itself. The best K of a sample's candidates are taken: larger scores first,
// of equal ones the lower beam's, within a beam the larger logit's, then the lower
// id's. (A beam's candidates thus come in the order of its logits, so that only its
// best K can be taken, and they are known before its lse is.)
#include "kv4.cuh"

namespace svl {

constexpr int kBeamThreads = 512;

// Orders floats as unsigned integers, -0 like 0 (NaN: see the callers).
SVL_DEVINL uint32_t order_bits(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
SVL_DEVINL float from_order_bits(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// Logit and id as one number: the larger is the better candidate.
SVL_DEVINL uint64_t beam_key(float x, int v) {
  return static_cast<uint64_t>(order_bits(x)) << 32 | (0xffffffffu - static_cast<uint32_t>(v));
}

SVL_DEVINL uint64_t block_max(uint64_t x, uint64_t* red) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    const uint64_t y = __shfl_xor_sync(0xffffffffu, x, off);
    x = y > x ? y : x;
  }
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = red[0];
  for (int i = 1; i < kBeamThreads / 32; ++i) x = red[i] > x ? red[i] : x;
  __syncthreads();
  return x;
}

// The K best candidates of each beam: keys [S * W][K] and the beam's offset c_w - lse_w.
__global__ void __launch_bounds__(kBeamThreads) beam_row_kernel(BeamArgs a, uint64_t* keys, float* offset) {
  __shared__ uint64_t red[kBeamThreads / 32];
  __shared__ double sums[kBeamThreads / 32];
  pdl_begin(false);
  const int row = blockIdx.x, tid = threadIdx.x;
  if (a.finished && a.finished[row]) return;
  const float* x = a.logits + row * a.ld;
  float m = -INFINITY;
  bool nan = false;
  for (int v = tid; v < a.V; v += kBeamThreads) {
    nan |= isnan(x[v]);
    m = fmaxf(m, x[v]);
  }
  nan = __syncthreads_or(nan);
  m = from_order_bits(static_cast<uint32_t>(block_max(static_cast<uint64_t>(order_bits(m)), red)));
  const bool alive = !nan && isfinite(m);
  if (alive) {
    double sum = 0;
    for (int v = tid; v < a.V; v += kBeamThreads) sum += expf(x[v] - m);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    if ((tid & 31) == 0) sums[tid >> 5] = sum;
    __syncthreads();
    if (tid == 0) {
      for (int i = 1; i < kBeamThreads / 32; ++i) sum += sums[i];
      offset[row] = a.scores[row] - static_cast<float>(m + log(sum));
    }
  } else if (tid == 0) {
    offset[row] = -INFINITY;
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < a.K; ++k) {
    uint64_t best = 0;
    for (int v = tid; v < a.V; v += kBeamThreads) {
      const uint64_t key = beam_key(alive ? x[v] : 0.f, v);
      if (key < last && key > best) best = key;
    }
    last = block_max(best, red);
    if (tid == 0) keys[static_cast<int64_t>(row) * a.K + k] = last;
  }
}

// Merges a sample's beams: one thread walks the heads of their lists.
__global__ void beam_merge_kernel(BeamArgs a, const uint64_t* keys, const float* offset) {
  pdl_begin(false);
  const int s = blockIdx.x * blockDim.x + threadIdx.x;
  if (s >= a.S) return;
  int at[kKv4MaxBeams];
  for (int w = 0; w < a.W; ++w) at[w] = 0;
  for (int k = 0; k < a.K; ++k) {
    float best = 0.f;
    int bw = -1, bt = 0;
    bool bf = false;
    for (int w = 0; w < a.W; ++w) {
      if (at[w] >= a.K) continue;
      const int row = s * a.W + w;
      const bool done = a.finished && a.finished[row];
      float c;
      int t = a.eos;
      if (done) {
        c = at[w] == 0 ? a.scores[row] : -INFINITY;
      } else {
        const uint64_t key = keys[static_cast<int64_t>(row) * a.K + at[w]];
        t = static_cast<int>(0xffffffffu - static_cast<uint32_t>(key));
        c = from_order_bits(static_cast<uint32_t>(key >> 32)) + offset[row];
      }
      if (isnan(c)) c = -INFINITY;
      if (bw < 0 || c > best) {
        best = c;
        bw = w;
        bt = t;
        bf = done;
      }
    }
    ++at[bw];
    const int64_t o = static_cast<int64_t>(s) * a.K + k;
    a.scores_out[o] = best;
    a.parent[o] = bw;
    a.token[o] = bt;
    if (a.finished_out) a.finished_out[o] = bf || bt == a.eos;
  }
}

size_t beam_workspace(int S, int W, int, int K) {
  const size_t rows = static_cast<size_t>(S) * W;
  return rows * K * sizeof(uint64_t) + rows * sizeof(float);
}

cudaError_t launch_beam_select(const BeamArgs& a, cudaStream_t s) {
  uint64_t* keys = static_cast<uint64_t*>(a.ws);
  float* offset = reinterpret_cast<float*>(keys + static_cast<size_t>(a.S) * a.W * a.K);
  const cudaError_t e = launch_pdl(beam_row_kernel, dim3(a.S * a.W), kBeamThreads, 0, s, a, keys, offset);
  if (e != cudaSuccess) return e;
  return launch_pdl(beam_merge_kernel, dim3((a.S + 31) / 32), 32, 0, s, a, keys, static_cast<const float*>(offset));
}

}  // namespace svl
