// Attention of the newest rows of each slot over its 4-bit KV cache:
//   o = sum_j softmax_j(scale * q . k_j) v_j
// over the positions j that the row at position pos sees: j <= pos, and with a
// window W > 0 only j > pos - W or j < sinks. A row with pos < 0 sees nothing
// and a row with pos >= max_len has no place in the cache: both give zeros.
#include "kv4.cuh"

namespace svl {

constexpr int kSimpleThreads = 32;

// A warp per (slot, row, head), a lane per d_head / 32 dimensions.
template <int DH>
__global__ void __launch_bounds__(kSimpleThreads) kv4_attn_kernel(Kv4Attn a) {
  constexpr int J = DH / 32;
  pdl_begin(a.late);
  const int b = blockIdx.z, r = blockIdx.y, h = blockIdx.x, lane = threadIdx.x;
  const int grp = a.A / a.c.kv, kvh = h / grp;
  if (!gate_on(a.gate, b, a.gate.G ? h / (a.A / a.gate.G) : 0)) return;
  const int64_t row = static_cast<int64_t>(b) * a.rows + r;
  const int64_t pos = static_cast<int64_t>(a.start[b]) + r;
  const int end = pos >= 0 && pos < a.c.max_len ? static_cast<int>(pos) + 1 : 0;
  const int lo = a.window > 0 && end > a.window ? end - a.window : 0;
  float q[J], o[J], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    q[j] = __bfloat162float(a.q[row * a.ldq + h * DH + 32 * j + lane]) * a.scale;
    o[j] = 0.f;
  }
  const int g = lane / 4;
  for (int p = 0; p < end; ++p) {
    if (p >= a.sinks && p < lo) p = lo;
    const uint8_t* tile = kv4_tile(a.c, b, kvh, p / kKv4Tile);
    const int i = p % kKv4Tile;
    float x = 0.f, v[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int nk = tile[((i * 4 + lane / 8) * J + j) * 4 + lane % 8 / 2] >> (4 * (lane & 1)) & 15;
      const int nv = tile[kv4_v_codes(DH) + ((((i / 8) * 8 + g) * 4 + i % 8 / 2) * J + j) * 4 + (i & 1) * 2 +
                          lane % 4 / 2] >> (4 * (lane & 1)) & 15;
      const float sk = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(tile + kv4_k_scales(DH))[i * J + j]);
      const float sv =
          __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(tile + kv4_v_scales(DH))[(i / 2 * J + j) * 2 + (i & 1)]);
      x = fmaf(q[j], sk * (nk - 8), x);
      v[j] = sv * (nv - 8);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    const float mn = fmaxf(m, x), corr = expf(m - mn), e = expf(x - mn);
    l = l * corr + e;
#pragma unroll
    for (int j = 0; j < J; ++j) o[j] = fmaf(e, v[j], o[j] * corr);
    m = mn;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int j = 0; j < J; ++j) a.out[row * a.ldo + h * DH + 32 * j + lane] = __float2bfloat16_rn(o[j] * inv);
}

size_t kv4_attn_workspace(const Kv4Cache&, int, int) { return 0; }

cudaError_t launch_kv4_attention(const Kv4Attn& a, cudaStream_t s) {
  const dim3 grid(a.A, a.rows, a.c.n_slots);
  return a.c.dh == 128 ? launch_pdl(kv4_attn_kernel<128>, grid, kSimpleThreads, 0, s, a)
                       : launch_pdl(kv4_attn_kernel<64>, grid, kSimpleThreads, 0, s, a);
}

}  // namespace svl
