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
// up to a quarter, always in one direction. Scaling by a power of two is exact,
// so the code is the one rounding. A block with a NaN or an infinity becomes the
// scale 255 (NaN) and codes of zero.
//
// All of it is bound by memory (2 bytes in, 17/32 out per value; SwiGLU 4 in), if
// a value costs no more than some ten issue slots: hence sixteen values a
// thread, whose block and row are found once, and operations on pairs.
// 18,944 x 3,584: rows 27.9 us (6.2 TB/s), with a gain 28.6, with 1/rms 30.5, with
// both 31.4, SwiGLU 48.2 (6.4 TB/s), reading back 32.3 (5.3 TB/s, four fifths of it writes).
#include <algorithm>

#include "mxf4.cuh"

namespace svl {

constexpr int kMxThreads = 256;

// The scale byte of a block whose largest magnitude has the bits u.
SVL_DEVINL int scale_byte(uint32_t u) {
  const int b = static_cast<int>(u >> 23) - 2 + ((u & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return u >= 0x7F800000u ? 255 : max(b, 0);
}

// Two float32 numbers in a register pair: one operation for both.
SVL_DEVINL uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
SVL_DEVINL uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
SVL_DEVINL uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
SVL_DEVINL float lo2(uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v)); }
SVL_DEVINL float hi2(uint64_t v) { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }
SVL_DEVINL uint64_t pair2(float lo, float hi) {
  return (static_cast<uint64_t>(__float_as_uint(hi)) << 32) | __float_as_uint(lo);
}
SVL_DEVINL uint64_t both2(float v) { return pair2(v, v); }

// Eight bf16 numbers as four pairs.
SVL_DEVINL void pairs8(const uint4& x, uint64_t* f) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) f[q] = (static_cast<uint64_t>(w[q] & 0xFFFF0000u) << 32) | (w[q] << 16);
}

// Eight values' codes, the first in the lowest nibble.
SVL_DEVINL uint32_t e2m1x8(const uint64_t* v) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(lo2(v[0])), "f"(hi2(v[0])), "f"(lo2(v[1])), "f"(hi2(v[1])), "f"(lo2(v[2])), "f"(hi2(v[2])),
        "f"(lo2(v[3])), "f"(hi2(v[3])));
  return r;
}

// Sixteen values of a row: half of a block.
struct Half {
  uint4 x[2], y[2];  // the values; ups
};

template <int SRC>
SVL_DEVINL void load_half(const Mxf4Rows& a, int64_t row, int u, Half& v) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = u * 16 + i * 8;
    v.x[i] = v.y[i] = make_uint4(0, 0, 0, 0);
    if (row < a.rows && c < a.cols) {
      v.x[i] = *reinterpret_cast<const uint4*>(a.src + row * a.ld_src + c);
      if (SRC == MX_SWIGLU) v.y[i] = *reinterpret_cast<const uint4*>(a.other + row * a.ld_other + c);
    }
  }
}

// The gains of sixteen columns.
SVL_DEVINL void load_gains(const Mxf4Rows& a, int u, uint4* gain) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int c = u * 16 + i * 8;
    gain[i] = c < a.cols ? *reinterpret_cast<const uint4*>(a.other + c) : make_uint4(0, 0, 0, 0);
  }
}

// gate / (1 + exp(-gate)) * up of two values, within 7 * 2^-23 of it (gates
// whose exponential passes 2^126 give 0). With log2(e) = H + L, H of 15 bits (a
// constant split as Cody and Waite do): exp(-g) = 2^(-gH) * exp(-g L ln 2). A bf16
// gate times H is exact, and the second factor is 1 - g L ln 2 within 2^-23 for
// every g that leaves exp(-g) to count. Seven operations a value where expf and a
// division took 80 us for 5,403 x 11,008 rows, twice what the memory takes.
SVL_DEVINL uint64_t swiglu2(uint64_t gate, uint64_t up) {
  const uint64_t t = mul2(gate, both2(-1.44268798828125f));
  const uint64_t rest = fma2(gate, both2(-4.888495152143634e-6f), both2(1.f));
  const uint64_t e = add2(mul2(pair2(ex2(lo2(t)), ex2(hi2(t))), rest), both2(1.f));
  float r0, r1;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(lo2(e)));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(hi2(e)));
  return mul2(mul2(gate, pair2(r0, r1)), up);
}

SVL_DEVINL uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// Quantises and stores the sixteen values of every lane; two neighbours hold a
// block. Every lane of the warp takes part.
template <int SRC, bool RMS>
SVL_DEVINL void store_half(const Mxf4Rows& a, int64_t row, int u, int n_units, int n_held, uint8_t* codes,
                           uint8_t* scale, const Half& v, const uint4* gain, uint64_t* squares) {
  uint64_t f[8];
  pairs8(v.x[0], f);
  pairs8(v.x[1], f + 4);
  if (RMS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) squares[i & 1] = fma2(f[i], f[i], squares[i & 1]);
  }
  // the largest magnitude's bits: ordered like the magnitudes, NaN above infinity
  uint32_t top;
  if (SRC == MX_ROWS) {
    const uint32_t w[8] = {v.x[0].x, v.x[0].y, v.x[0].z, v.x[0].w, v.x[1].x, v.x[1].y, v.x[1].z, v.x[1].w};
    uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
    for (int i = 1; i < 8; ++i) m = max_u16x2(m, w[i] & 0x7FFF7FFFu);
    top = max(m & 0xFFFF0000u, m << 16);
  } else {
    uint64_t y[8];
    pairs8(SRC == MX_GAIN ? gain[0] : v.y[0], y);
    pairs8(SRC == MX_GAIN ? gain[1] : v.y[1], y + 4);
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f[i] = SRC == MX_GAIN ? mul2(f[i], y[i]) : swiglu2(f[i], y[i]);
      asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(lo2(f[i])), "f"(hi2(f[i])));
    }
    top = __float_as_uint(m);
  }
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  const int b = scale_byte(top);
  // (times 2^-126 where the block holds a NaN or an infinity: its codes are replaced)
  const uint64_t s = both2(__uint_as_float(static_cast<uint32_t>(254 - min(b, 253)) << 23));
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = mul2(f[i], s);
  uint2 code = make_uint2(e2m1x8(f), e2m1x8(f + 4));
  if (b == 255) code = make_uint2(0, 0);
  if (row >= a.rows) return;
  if (u < n_held) *reinterpret_cast<uint2*>(codes + static_cast<int64_t>(u) * 8) = code;
  if ((u & 1) == 0 && u < n_units)
    scale[static_cast<int64_t>(u >> 3) * kMxTileBytes + ((u >> 1) & 3)] = static_cast<uint8_t>(b);
}

// A group of `group` threads (a power of two, 8 to kMxThreads) takes a row, or
// AT_ONCE rows that share the loads of their gains, sixteen values a thread and
// step: eight threads' values are a tile's 128 columns, so a block's lanes and a
// tile's bytes stay together.
template <int SRC, bool RMS, int AT_ONCE>
__global__ void __launch_bounds__(kMxThreads, 4) mxf4_quantize_kernel(Mxf4Rows a, int group) {
  constexpr int kBatch = AT_ONCE > 1 ? 1 : SRC == MX_ROWS ? 4 : 2;  // steps loaded before work on the first
  __shared__ float red[2][AT_ONCE][kMxThreads / 32];
  pdl_begin(false);
  const int j = threadIdx.x & (group - 1), per_cta = kMxThreads / group;
  const int64_t tiles = mxf4_scale_tiles(a.cols);
  const int n_units = static_cast<int>(tiles) * 8, n_held = (a.cols + kMxBlock - 1) / kMxBlock * 2;
  int n = 0;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * per_cta * AT_ONCE; r0 < a.rows;
       r0 += static_cast<int64_t>(gridDim.x) * per_cta * AT_ONCE, ++n) {
    int64_t row[AT_ONCE];
    uint8_t *codes[AT_ONCE], *scale[AT_ONCE];
    uint64_t squares[AT_ONCE][2];
#pragma unroll
    for (int q = 0; q < AT_ONCE; ++q) {
      row[q] = r0 + q * per_cta + threadIdx.x / group;
      codes[q] = a.codes + row[q] * a.ld_codes;
      scale[q] = a.scale + (row[q] >> 7) * tiles * kMxTileBytes + (row[q] & 31) * 16 + ((row[q] >> 5) & 3) * 4;
      squares[q][0] = squares[q][1] = 0;
    }
    for (int u0 = 0; u0 < n_units; u0 += kBatch * group) {
      Half v[kBatch][AT_ONCE];
      uint4 gain[kBatch][2];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (u0 + i * group < n_units) {
          if (SRC == MX_GAIN) load_gains(a, u0 + i * group + j, gain[i]);
#pragma unroll
          for (int q = 0; q < AT_ONCE; ++q) load_half<SRC>(a, row[q], u0 + i * group + j, v[i][q]);
        }
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (u0 + i * group < n_units) {
#pragma unroll
          for (int q = 0; q < AT_ONCE; ++q)
            store_half<SRC, RMS>(a, row[q], u0 + i * group + j, n_units, n_held, codes[q], scale[q], v[i][q], gain[i],
                                 squares[q]);
        }
      }
    }
    if (RMS) {
      float sum[AT_ONCE];
#pragma unroll
      for (int q = 0; q < AT_ONCE; ++q) {
        const uint64_t both = add2(squares[q][0], squares[q][1]);
        sum[q] = __fadd_rn(lo2(both), hi2(both));
      }
      for (int off = min(group, 32) >> 1; off > 0; off >>= 1) {
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], off);
      }
      if (group > 32) {
        // (alternate, so that one barrier each time is enough)
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
          for (int q = 0; q < AT_ONCE; ++q) red[n & 1][q][threadIdx.x >> 5] = sum[q];
        }
        __syncthreads();
      }
      if (j == 0) {
#pragma unroll
        for (int q = 0; q < AT_ONCE; ++q) {
          if (group > 32) {
            sum[q] = 0.f;
            for (int i = 0; i < group / 32; ++i) sum[q] += red[n & 1][q][(threadIdx.x >> 5) + i];
          }
          if (row[q] < a.rows)
            a.inv_rms[row[q]] =
                __fdiv_rn(1.f, __fsqrt_rn(__fadd_rn(__fdiv_rn(sum[q], static_cast<float>(a.cols)), a.eps)));
        }
      }
    }
  }
}

SVL_DEVINL uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// Eight codes as bf16 numbers. As float16 a code has its value in five bits of
// exponent and one of mantissa, which three places further right are the
// bf16 number 2^-112 times as large: `s` and, for the largest scales, `s2`
// make up for that. (b <= 142 has s = 2^(b - 127 + 112) and no s2.)
SVL_DEVINL uint4 bf16x8(uint32_t code, uint32_t s, uint32_t s2, bool far) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(code));
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    h[q] = mul_bf16x2(((h[q] >> 3) & 0x0FFF0FFFu) | (h[q] & 0x80008000u), s);
    if (far) h[q] = mul_bf16x2(h[q], s2);
  }
  return make_uint4(h[0], h[1], h[2], h[3]);
}

// Groups of threads take rows as in mxf4_quantize_kernel, eight values a thread
// and step, so that a warp stores 512 consecutive bytes (16 values a thread, two
// stores 32 bytes apart each: 42 us for 18,944 x 3,584, 32 with eight).
template <int STEPS, int AT_ONCE>
__global__ void __launch_bounds__(kMxThreads) mxf4_dequantize_kernel(Mxf4Read a, int group) {
  pdl_begin(false);
  const int j = threadIdx.x & (group - 1), per_cta = kMxThreads / group;
  const int64_t tiles = mxf4_scale_tiles(a.cols);
  const int n_units = a.cols / 8;
  for (int64_t r0 = static_cast<int64_t>(blockIdx.x) * per_cta * AT_ONCE + threadIdx.x / group; r0 < a.rows;
       r0 += static_cast<int64_t>(gridDim.x) * per_cta * AT_ONCE) {
    for (int u0 = j; u0 < n_units; u0 += STEPS * group) {
      uint32_t code[AT_ONCE][STEPS];
      int b[AT_ONCE][STEPS];
#pragma unroll
      for (int q = 0; q < AT_ONCE; ++q) {
        const int64_t row = r0 + q * per_cta;
        const uint8_t* codes = a.codes + row * a.ld_codes;
        const uint8_t* scale = a.scale + (row >> 7) * tiles * kMxTileBytes + (row & 31) * 16 + ((row >> 5) & 3) * 4;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const int u = u0 + i * group;
          if (u < n_units && row < a.rows) {
            code[q][i] = *reinterpret_cast<const uint32_t*>(codes + static_cast<int64_t>(u) * 4);
            b[q][i] = scale[static_cast<int64_t>(u >> 4) * kMxTileBytes + ((u >> 2) & 3)];
          }
        }
      }
#pragma unroll
      for (int q = 0; q < AT_ONCE; ++q) {
        const int64_t row = r0 + q * per_cta;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const int u = u0 + i * group;
          if (u >= n_units || row >= a.rows) break;
          const bool far = b[q][i] > 142;
          const uint32_t e = static_cast<uint32_t>(min(b[q][i], 142)) + 112;
          const uint32_t e2 = b[q][i] == 255 ? 0x7FC0u : static_cast<uint32_t>(max(b[q][i], 142) - 142 + 127) << 7;
          *reinterpret_cast<uint4*>(a.dst + row * a.ld_dst + static_cast<int64_t>(u) * 8) =
              bf16x8(code[q][i], (e << 7) * 0x10001u, e2 * 0x10001u, far);
        }
      }
    }
  }
}

// Threads per row: a warp, less for narrow rows (fewer lanes without values), more
// while the rows' groups have not `threads` in all, twice what the SMs hold when
// quantising, four times when reading back. us with half as many threads, as many, and
// two and four times as many: 5,403 x 11,008 quantised 30.7, 26.3, 27.5, 26.0, with
// 1/rms 31.9, 28.4, 31.6, 31.7, with a gain too 45.3, 32.1, 34.6, 36.5, read back 31.0,
// 28.8, 29.4, 29.5; 18,944 x 3,584 with 1/rms 30.5, 30.5, 35.4, 41.1; 2,000 x 18,944 with
// 1/rms 19.2, 20.2, 20.3, 20.2.
static int group_for(int64_t rows, int64_t units, int threads) {
  int group = 8;
  while (group < 32 && group < units) group *= 2;
  while (group < kMxThreads && group < units && rows * group < threads) group *= 2;
  return group;
}
static unsigned grid_for(int64_t rows, int group, int num_sms) {
  const int64_t ctas = (rows + kMxThreads / group - 1) / (kMxThreads / group);
  return static_cast<unsigned>(std::min<int64_t>(ctas, 8 * static_cast<int64_t>(num_sms)));
}

template <int SRC, int AT_ONCE>
static cudaError_t launch_quantize(const Mxf4Rows& a, int group, cudaStream_t s) {
  const unsigned grid = grid_for((a.rows + AT_ONCE - 1) / AT_ONCE, group, a.num_sms);
  return a.inv_rms ? launch_pdl(mxf4_quantize_kernel<SRC, true, AT_ONCE>, grid, kMxThreads, 0, s, a, group)
                   : launch_pdl(mxf4_quantize_kernel<SRC, false, AT_ONCE>, grid, kMxThreads, 0, s, a, group);
}

cudaError_t launch_mxf4_quantize(Mxf4Source source, const Mxf4Rows& a, cudaStream_t s) {
  const int64_t units = mxf4_scale_tiles(a.cols) * 8;
  const int group = group_for(a.rows, units, 2048 * a.num_sms);
  // Two rows at a time where a row is a single step, so that each thread has more than one on its way, and where rows
  // share the loads of their gains. Not where the SMs (four CTAs each) would then pass over more rows in all: 60,000 x
  // 256 7.9 us instead of 9.9, 18,944 x 3,584 with gains 28.6 instead of 31.7, but 5,403 x 11,008 33.3 instead of 30.4.
  // (Rows without gains are left at one: 18,944 x 3,584 27.6 and 27.9, but 5,403 x 11,008 31.9 and 26.3.)
  const int64_t wave = static_cast<int64_t>(kMxThreads / group) * 4 * a.num_sms;
  const int64_t ones = (a.rows + wave - 1) / wave, twos = (a.rows + 2 * wave - 1) / (2 * wave);
  const bool step = units <= group && ones > 2, fits = ones > 1 && 2 * twos <= ones;
  switch (source) {
    case MX_ROWS: return step ? launch_quantize<MX_ROWS, 2>(a, group, s) : launch_quantize<MX_ROWS, 1>(a, group, s);
    case MX_GAIN:
      return step || fits ? launch_quantize<MX_GAIN, 2>(a, group, s) : launch_quantize<MX_GAIN, 1>(a, group, s);
    default:
      return step ? launch_pdl(mxf4_quantize_kernel<MX_SWIGLU, false, 2>, grid_for((a.rows + 1) / 2, group, a.num_sms),
                               kMxThreads, 0, s, a, group)
                  : launch_pdl(mxf4_quantize_kernel<MX_SWIGLU, false, 1>, grid_for(a.rows, group, a.num_sms), kMxThreads,
                               0, s, a, group);
  }
}

cudaError_t launch_mxf4_dequantize(const Mxf4Read& a, cudaStream_t s) {
  const int group = group_for(a.rows, a.cols / 8, 4096 * a.num_sms);
  // four steps of a row, or four rows of one step (60,000 x 256 8.0 us instead of 10.1)
  if (a.cols / 8 <= group && a.rows > static_cast<int64_t>(kMxThreads / group) * 8 * a.num_sms)
    return launch_pdl(mxf4_dequantize_kernel<1, 4>, grid_for((a.rows + 3) / 4, group, a.num_sms), kMxThreads, 0, s, a,
                      group);
  return launch_pdl(mxf4_dequantize_kernel<4, 1>, grid_for(a.rows, group, a.num_sms), kMxThreads, 0, s, a, group);
}

}  // namespace svl
