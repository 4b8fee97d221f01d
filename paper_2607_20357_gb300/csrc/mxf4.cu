// Rows of bf16 to MXFP4 and back. Every 32 consecutive values x of a row share
// a scale 2^e:
//
//   a = max |x|,  e = the smallest integer >= -127 with a <= 6 * 2^e,
//   code = e2m1(x * 2^-e), to nearest, ties to the even code.
//
// With a = 1.f * 2^E that is e = E - 2, or E - 1 where 1.f > 1.5: an integer
// addition and a comparison of a's bits. No value saturates (6 is the largest
// e2m1 value). e = E - 2 throughout would cut a block's largest values, those
// between 6 and 8 * 2^e, down to 6; the mean square error of normal values is the
// same (0.0134 of their square, 0.0132 with the cut), but it shrinks outliers by
// up to a quarter, always in one direction. Scaling by a power of two is exact, so the code is the one
// rounding. A block with a NaN or an infinity becomes the scale 255 (NaN) and
// codes of zero.
//
// All of it is bound by memory (2 bytes in, 17/32 out per value; SwiGLU 4 in),
// with about ten issue slots per value to spend at that rate.
#include <algorithm>

#include <cuda_fp16.h>

#include "mxf4.cuh"

namespace svl {

constexpr int kMxThreads = 256;
constexpr int kMxBatch = 4;  // units of 8 values a thread loads before it works on the first

// The scale byte of a block whose largest magnitude is `top` (>= 0).
SVL_DEVINL int scale_byte(float top) {
  const uint32_t u = __float_as_uint(top);
  const int b = static_cast<int>(u >> 23) - 2 + ((u & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return u >= 0x7F800000u ? 255 : max(b, 0);
}

// Eight values' codes, the first in the lowest nibble.
SVL_DEVINL uint32_t e2m1x8(const float* v) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}

SVL_DEVINL void floats8(const uint4& x, float* f) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[2 * q] = __uint_as_float(w[q] << 16);
    f[2 * q + 1] = __uint_as_float(w[q] & 0xFFFF0000u);
  }
}

// Largest magnitude of eight values, NaN if one is.
SVL_DEVINL float top8(const float* f) {
  float m = fabsf(f[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(f[i])));
  return m;
}

struct Unit {
  uint4 x, y;  // eight values; eight gains or ups
};

template <int SRC>
SVL_DEVINL Unit load_unit(const Mxf4Rows& a, int64_t row, int u) {
  Unit v;
  v.x = v.y = make_uint4(0, 0, 0, 0);
  if (row < a.rows && u * 8 < a.cols) {
    v.x = *reinterpret_cast<const uint4*>(a.src + row * a.ld_src + u * 8);
    if (SRC == MX_GAIN) v.y = *reinterpret_cast<const uint4*>(a.other + u * 8);
    if (SRC == MX_SWIGLU) v.y = *reinterpret_cast<const uint4*>(a.other + row * a.ld_other + u * 8);
  }
  return v;
}

// Quantises and stores one unit of 8 values of every lane; four consecutive lanes
// hold a block. Every lane of the warp takes part.
template <int SRC>
SVL_DEVINL void store_unit(const Mxf4Rows& a, int64_t row, int u, const Unit& v, float* squares) {
  float f[8], y[8];
  floats8(v.x, f);
  if (squares) {
#pragma unroll
    for (int i = 0; i < 8; ++i) *squares = fmaf(f[i], f[i], *squares);
  }
  if (SRC != MX_ROWS) floats8(v.y, y);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (SRC == MX_GAIN) f[i] = __fmul_rn(f[i], y[i]);
    if (SRC == MX_SWIGLU) f[i] = __fmul_rn(__fdiv_rn(f[i], __fadd_rn(1.f, expf(-f[i]))), y[i]);
  }
  float top = top8(f);
#pragma unroll
  for (int off = 1; off < 4; off <<= 1) {
    const float o = __shfl_xor_sync(0xffffffffu, top, off);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(top) : "f"(o));
  }
  const int b = scale_byte(top);
  // (times 0 where the block holds a NaN or an infinity: its codes are replaced)
  const float s = __uint_as_float(static_cast<uint32_t>(254 - min(b, 253)) << 23);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __fmul_rn(f[i], s);
  const uint32_t code = b == 255 ? 0u : e2m1x8(f);
  if (row >= a.rows) return;
  if (u < (a.cols + kMxBlock - 1) / kMxBlock * 4)
    *reinterpret_cast<uint32_t*>(a.codes + row * a.ld_codes + u * 4) = code;
  if ((u & 3) == 0) {
    const int64_t tile = (row >> 7) * mxf4_scale_tiles(a.cols) + (u >> 4);
    const int r = static_cast<int>(row & 127);
    a.scale[tile * kMxTileBytes + (r & 31) * 16 + (r >> 5) * 4 + ((u >> 2) & 3)] = static_cast<uint8_t>(b);
  }
}

// The rows as one sequence of units of 8 values, a row's rounded up to a scale
// tile's 16 (so that a block's lanes and a tile's bytes stay together); a warp
// takes 32 consecutive ones, kMxBatch times a grid's stride apart.
template <int SRC>
__global__ void __launch_bounds__(kMxThreads) mxf4_quantize_kernel(Mxf4Rows a) {
  pdl_begin(false);
  const int per_row = static_cast<int>(mxf4_scale_tiles(a.cols)) * 16;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kMxThreads;
  const int64_t d_row = stride / per_row;
  const int d_u = static_cast<int>(stride - d_row * per_row);
  int64_t first = static_cast<int64_t>(blockIdx.x) * kMxThreads + threadIdx.x;
  int64_t row = first / per_row;
  int u = static_cast<int>(first - row * per_row);
  // (the warp's first unit decides: all lanes of a warp stay together)
  while (__any_sync(0xffffffffu, row < a.rows)) {
    Unit v[kMxBatch];
    int64_t rows[kMxBatch];
    int us[kMxBatch];
#pragma unroll
    for (int i = 0; i < kMxBatch; ++i) {
      rows[i] = row;
      us[i] = u;
      v[i] = load_unit<SRC>(a, row, u);
      row += d_row;
      u += d_u;
      if (u >= per_row) {
        u -= per_row;
        ++row;
      }
    }
#pragma unroll
    for (int i = 0; i < kMxBatch; ++i) store_unit<SRC>(a, rows[i], us[i], v[i], nullptr);
  }
}

// The same with 1/rms of the rows: a CTA per row.
template <int SRC>
__global__ void __launch_bounds__(kMxThreads) mxf4_quantize_rms_kernel(Mxf4Rows a) {
  __shared__ float red[2][kMxThreads / 32];
  pdl_begin(false);
  const int per_row = static_cast<int>(mxf4_scale_tiles(a.cols)) * 16;
  const int steps = (per_row + kMxThreads - 1) / kMxThreads;
  int n = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, ++n) {
    float squares = 0.f;
    for (int i0 = 0; i0 < steps; i0 += kMxBatch) {
      Unit v[kMxBatch];
#pragma unroll
      for (int i = 0; i < kMxBatch; ++i) {
        const int u = (i0 + i) * kMxThreads + threadIdx.x;
        v[i] = load_unit<SRC>(a, u < per_row ? row : a.rows, u);
      }
#pragma unroll
      for (int i = 0; i < kMxBatch; ++i) {
        const int u = (i0 + i) * kMxThreads + threadIdx.x;
        if (i0 + i < steps) store_unit<SRC>(a, u < per_row ? row : a.rows, u, v[i], &squares);
      }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, off);
    float* rd = red[n & 1];  // (alternate, so that one barrier a row is enough)
    if ((threadIdx.x & 31) == 0) rd[threadIdx.x >> 5] = squares;
    __syncthreads();
    if (threadIdx.x == 0) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kMxThreads / 32; ++i) sum += rd[i];
      a.inv_rms[row] = __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fdiv_rn(sum, static_cast<float>(a.cols)), a.eps)));
    }
  }
}

__global__ void __launch_bounds__(kMxThreads) mxf4_dequantize_kernel(Mxf4Read a) {
  pdl_begin(false);
  const int per_row = (a.cols + 7) / 8;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * kMxThreads;
  const int64_t d_row = stride / per_row;
  const int d_u = static_cast<int>(stride - d_row * per_row);
  const int64_t first = static_cast<int64_t>(blockIdx.x) * kMxThreads + threadIdx.x;
  int64_t row = first / per_row;
  int u = static_cast<int>(first - row * per_row);
  while (row < a.rows) {
    uint32_t code[kMxBatch], b[kMxBatch];
    __nv_bfloat16* dst[kMxBatch];
#pragma unroll
    for (int i = 0; i < kMxBatch; ++i) {
      dst[i] = nullptr;
      if (row < a.rows) {
        dst[i] = a.dst + row * a.ld_dst + u * 8;
        code[i] = *reinterpret_cast<const uint32_t*>(a.codes + row * a.ld_codes + u * 4);
        const int64_t tile = (row >> 7) * mxf4_scale_tiles(a.cols) + (u >> 4);
        const int r = static_cast<int>(row & 127);
        b[i] = a.scale[tile * kMxTileBytes + (r & 31) * 16 + (r >> 5) * 4 + ((u >> 2) & 3)];
      }
      row += d_row;
      u += d_u;
      if (u >= per_row) {
        u -= per_row;
        ++row;
      }
    }
#pragma unroll
    for (int i = 0; i < kMxBatch; ++i) {
      if (!dst[i]) continue;
      // 2^(b - 127): b is the exponent field of a float, but 2^-127 is subnormal and 255 a NaN
      const float s = __uint_as_float(b[i] == 0 ? 0x400000u : b[i] == 255 ? 0x7FC00000u : b[i] << 23);
      uint32_t h[4], o[4];
      asm("{\n\t.reg .b8 a, b, c, d;\n\t"
          "mov.b32 {a, b, c, d}, %4;\n\t"
          "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
          "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
          : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
          : "r"(code[i]));
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 f = __half22float2(*reinterpret_cast<__half2*>(&h[q]));
        o[q] = pack_bf16x2(__fmul_rn(f.x, s), __fmul_rn(f.y, s));
      }
      *reinterpret_cast<uint4*>(dst[i]) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

// CTAs for n items of work of a thread each, kMxBatch of them at a time: at most
// eight per SM, which fill it.
static unsigned grid_for(int64_t n, int num_sms) {
  const int64_t want = (n + kMxThreads * kMxBatch - 1) / (kMxThreads * kMxBatch);
  return static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(want, 8 * static_cast<int64_t>(num_sms))));
}

cudaError_t launch_mxf4_quantize(Mxf4Source source, const Mxf4Rows& a, cudaStream_t s) {
  const unsigned grid = grid_for(a.rows * mxf4_scale_tiles(a.cols) * 16, a.num_sms);
  if (a.inv_rms) {
    const unsigned rows = static_cast<unsigned>(std::min<int64_t>(a.rows, 8 * static_cast<int64_t>(a.num_sms)));
    return source == MX_GAIN ? launch_pdl(mxf4_quantize_rms_kernel<MX_GAIN>, rows, kMxThreads, 0, s, a)
                             : launch_pdl(mxf4_quantize_rms_kernel<MX_ROWS>, rows, kMxThreads, 0, s, a);
  }
  switch (source) {
    case MX_ROWS: return launch_pdl(mxf4_quantize_kernel<MX_ROWS>, grid, kMxThreads, 0, s, a);
    case MX_GAIN: return launch_pdl(mxf4_quantize_kernel<MX_GAIN>, grid, kMxThreads, 0, s, a);
    default: return launch_pdl(mxf4_quantize_kernel<MX_SWIGLU>, grid, kMxThreads, 0, s, a);
  }
}

cudaError_t launch_mxf4_dequantize(const Mxf4Read& a, cudaStream_t s) {
  const unsigned grid = grid_for(a.rows * ((a.cols + 7) / 8), a.num_sms);
  return launch_pdl(mxf4_dequantize_kernel, grid, kMxThreads, 0, s, a);
}

}  // namespace svl
