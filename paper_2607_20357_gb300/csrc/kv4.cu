// Writing rows into the 4-bit KV cache, reading them back, and moving slots
// after a beam search's selection.
//
// A group of 32 values x is held as a scale s and 32 codes n of 4 bits. With e the
// value of largest magnitude (the positive one of two alike), s = e / -8 and
// n = clamp(rint(x / s) + 8, 0, 15) stand for s * (n - 8): e itself is met exactly
// (n = 0), and all sixteen codes are used. s is exact in bf16. A group with a value
// that is not finite gets the scale NaN and reads back as NaN; one whose |e| is
// under 2^-123 (a subnormal scale) is held as zeros: s = 0, n = 8.
#include "kv4.cuh"

namespace svl {

// Slot and position of packed row r; false where it is to be skipped.
struct RowPlace {
  int sample, slot, pos;
};
SVL_DEVINL bool row_place(const Kv4Rows& a, int64_t r, RowPlace& p) {
  int first;
  if (a.row_off) {
    if (r < a.row_off[0] || r >= a.row_off[a.n]) return false;
    p.sample = find_sample(a.row_off, a.n, static_cast<int>(r));
    first = a.row_off[p.sample];
  } else {
    p.sample = static_cast<int>(r);
    first = p.sample;
  }
  p.slot = p.sample * a.slot_step;
  const int64_t pos = (a.start ? a.start[p.sample] : 0) + (r - first);
  p.pos = static_cast<int>(pos < -1 ? -1 : (pos > a.c.max_len ? a.c.max_len : pos));
  return true;
}

// x / s rounded to the nearest integer, of two the even one, exactly. inv is 1 / s in
// float32, so t = x * inv is off by less than 2^-20 for |x / s| <= 8. x and s are bf16
// numbers: where x / s is not half an integer it is at least 2^-9 from one, so t
// rounded to a multiple of 2^-15 (by 384 = 1.5 * 2^8, whose last place that is) is
// half an integer exactly where x / s is.
SVL_DEVINL float kv4_code(float x, float inv) {
  const float t = __fadd_rn(__fadd_rn(__fmul_rn(x, inv), 384.f), -384.f);
  return fminf(rintf(t), 7.f) + 8.f;
}

// The scale (bf16 bits) of a group with largest value hi and smallest lo, all of them
// finite or not, and its reciprocal for kv4_code (0: every code is 8).
SVL_DEVINL uint16_t kv4_scale(float hi, float lo, bool finite, float& inv) {
  const float s = (hi >= -lo ? hi : lo) * -0.125f;
  inv = 0.f;
  if (!finite) return 0x7fc0;
  if (fabsf(s) < 1.17549435e-38f) return 0;
  inv = __frcp_rn(s);
  return __bfloat16_as_ushort(__float2bfloat16_rn(s));
}

constexpr int kRowThreads = 128;

// One thread per group of a row.
__global__ void __launch_bounds__(kRowThreads) kv4_write_kernel(Kv4Rows a) {
  pdl_begin(false);
  const int dh = a.c.dh, J = dh / 32, per_row = a.c.kv * J;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x;
  const int64_t r = i / per_row;
  if (r >= a.rows) return;
  const int hj = static_cast<int>(i - r * per_row), h = hj / J, j = hj - h * J;
  RowPlace at;
  if (!row_place(a, r, at) || at.pos < 0) return;
  if (at.pos >= a.c.max_len) {
    if (hj == 0) report(a.status, SVL_DEV_BAD_INDEX);
    return;
  }
  if (!gate_on(a.gate, at.sample, a.gate.G ? h / (a.c.kv / a.gate.G) : 0)) return;
  uint8_t* tile = kv4_tile(a.c, at.slot, h, at.pos / kKv4Tile);
  const int p = at.pos % kKv4Tile;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float x[32];
    float hi = -INFINITY, lo = INFINITY;
    bool fine = true;
#pragma unroll
    for (int d = 0; d < 32; ++d) {
      const int64_t c = static_cast<int64_t>(h) * dh + 32 * j + d;
      x[d] = __bfloat162float(which ? a.v[r * a.v_row + c * a.v_col] : a.k[r * a.k_row + c]);
      fine = fine && isfinite(x[d]);
      hi = fmaxf(hi, x[d]);
      lo = fminf(lo, x[d]);
    }
    float inv;
    const uint16_t s = kv4_scale(hi, lo, fine, inv);
    uint32_t w[4] = {0, 0, 0, 0};  // eight nibbles each
#pragma unroll
    for (int d = 0; d < 32; ++d)
      w[d / 8] |= static_cast<uint32_t>(inv == 0.f ? 8.f : kv4_code(x[d], inv)) << (4 * (d % 8));
    if (which == 0) {
#pragma unroll
      for (int t = 0; t < 4; ++t) reinterpret_cast<uint32_t*>(tile)[(p * 4 + t) * J + j] = w[t];
      reinterpret_cast<uint16_t*>(tile + kv4_k_scales(dh))[p * J + j] = s;
    } else {
      uint16_t* v = reinterpret_cast<uint16_t*>(tile + kv4_v_codes(dh));
#pragma unroll
      for (int g = 0; g < 8; ++g)
        v[((((p / 8) * 8 + g) * 4 + (p % 8) / 2) * J + j) * 2 + (p & 1)] =
            static_cast<uint16_t>(w[g / 2] >> (16 * (g & 1)));
      reinterpret_cast<uint16_t*>(tile + kv4_v_scales(dh))[((p / 2) * J + j) * 2 + (p & 1)] = s;
    }
  }
}

// One thread per group of a row; positions that the cache does not have read as 0.
__global__ void __launch_bounds__(kRowThreads) kv4_read_kernel(Kv4Rows a) {
  pdl_begin(false);
  const int dh = a.c.dh, J = dh / 32, per_row = a.c.kv * J;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kRowThreads + threadIdx.x;
  const int64_t r = i / per_row;
  if (r >= a.rows) return;
  const int hj = static_cast<int>(i - r * per_row), h = hj / J, j = hj - h * J;
  RowPlace at;
  if (!row_place(a, r, at)) return;
  const bool in = at.pos >= 0 && at.pos < a.c.max_len;
  const uint8_t* tile = in ? kv4_tile(a.c, at.slot, h, at.pos / kKv4Tile) : nullptr;
  const int p = at.pos % kKv4Tile;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    uint32_t w[4] = {0, 0, 0, 0};
    float s = 0.f;
    if (in && which == 0) {
#pragma unroll
      for (int t = 0; t < 4; ++t) w[t] = reinterpret_cast<const uint32_t*>(tile)[(p * 4 + t) * J + j];
      s = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(tile + kv4_k_scales(dh))[p * J + j]);
    } else if (in) {
      const uint16_t* v = reinterpret_cast<const uint16_t*>(tile + kv4_v_codes(dh));
#pragma unroll
      for (int g = 0; g < 8; ++g)
        w[g / 2] |= static_cast<uint32_t>(v[((((p / 8) * 8 + g) * 4 + (p % 8) / 2) * J + j) * 2 + (p & 1)])
                    << (16 * (g & 1));
      s = __bfloat162float(
          reinterpret_cast<const __nv_bfloat16*>(tile + kv4_v_scales(dh))[((p / 2) * J + j) * 2 + (p & 1)]);
    }
    __nv_bfloat16* out = which ? a.v_out + r * a.v_row : a.k_out + r * a.k_row;
#pragma unroll
    for (int d = 0; d < 32; ++d) {
      const int n = static_cast<int>(w[d / 8] >> (4 * (d % 8)) & 15u);
      out[static_cast<int64_t>(h) * dh + 32 * j + d] = __float2bfloat16_rn(s * static_cast<float>(n - 8));
    }
  }
}

static cudaError_t row_launch(void (*kernel)(Kv4Rows), const Kv4Rows& a, cudaStream_t s) {
  const int64_t threads = a.rows * a.c.kv * (a.c.dh / 32);
  const int64_t blocks = (threads + kRowThreads - 1) / kRowThreads;
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  if (blocks == 0) return cudaSuccess;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks)), kRowThreads, 0, s, a);
}

cudaError_t launch_kv4_write(const Kv4Rows& a, cudaStream_t s) { return row_launch(kv4_write_kernel, a, s); }
cudaError_t launch_kv4_read(const Kv4Rows& a, cudaStream_t s) { return row_launch(kv4_read_kernel, a, s); }

__global__ void kv4_lengths_kernel(const int* cu_seqlens, int n, int beams, int* len) {
  pdl_begin(false);
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) len[i] = cu_seqlens[i / beams + 1] - cu_seqlens[i / beams];
}
cudaError_t launch_kv4_lengths(const int* cu_seqlens, int B, int beams, int* len, cudaStream_t s) {
  return launch_pdl(kv4_lengths_kernel, dim3((B * beams + 127) / 128), 128, 0, s, cu_seqlens, B * beams, beams, len);
}

// One thread per 16 bytes of a tile, for all slots of a sample: each reads what the
// moved slots take over before it writes any of them, so the slots change in place
// whatever the parents are.
constexpr int kMoveThreads = 128;
__global__ void __launch_bounds__(kMoveThreads) kv4_reorder_kernel(Kv4Reorder a) {
  pdl_begin(false);
  const int sample = blockIdx.z % (a.c.n_slots / a.W), layer = blockIdx.z / (a.c.n_slots / a.W);
  const int head = blockIdx.y, tile = blockIdx.x;
  const int s0 = sample * a.W;
  int first = a.from ? a.from[sample] : 0;
  if (tile < (first > 0 ? first : 0) / kKv4Tile) return;
  const size_t layer_bytes = static_cast<size_t>(a.c.n_slots) * a.c.kv * a.c.tiles * kv4_tile_bytes(a.c.dh);
  Kv4Cache c = a.c;
  c.data += layer * layer_bytes;
  for (int i = threadIdx.x; i < kv4_tile_bytes(c.dh) / 16; i += kMoveThreads) {
    uint4 got[kKv4MaxBeams];
    uint32_t moved = 0;
    for (int w = 0; w < a.W; ++w) {
      const int p = a.parent[s0 + w];
      if (p < 0 || p >= a.W) {
        report(a.status, SVL_DEV_BAD_INDEX);
        continue;
      }
      if (p == w || tile * kKv4Tile >= a.len[s0 + p]) continue;
      moved |= 1u << w;
      got[w] = reinterpret_cast<const uint4*>(kv4_tile(c, s0 + p, head, tile))[i];
    }
    for (int w = 0; w < a.W; ++w)
      if (moved >> w & 1u) reinterpret_cast<uint4*>(kv4_tile(c, s0 + w, head, tile))[i] = got[w];
  }
}

cudaError_t launch_kv4_reorder(const Kv4Reorder& a, cudaStream_t s) {
  const dim3 grid(a.c.tiles, a.c.kv, a.c.n_slots / a.W * a.layers);
  return launch_pdl(kv4_reorder_kernel, grid, kMoveThreads, 0, s, a);
}

}  // namespace svl
