// Writing rows into the 4-bit KV cache, reading them back, and moving slots
// after a beam search's selection.
//
// A group of 32 values x is held as a scale s and 32 codes n of 4 bits. With e the
// value of largest magnitude (the positive one of two alike), s = e / -8 and
// n = clamp(rint(x / s) + 8, 0, 15) stand for s * (n - 8): e itself is met exactly
// (n = 0), and all sixteen codes are used. s is exact in bf16. A group with a value
// that is not finite gets the scale NaN and reads back as NaN; one whose |e| is
// under 2^-123 (a subnormal scale) is held as zeros: s = 0, n = 8.
//
// Writing and reading move 5 1/8 bytes per value of K and V; both are bound by
// that. A warp takes the up to eight rows of one KV head that share an aligned
// group of eight positions (a "quad" of the cache's pairs of rows): its codes of K
// and of V are 4 * d_head contiguous bytes each, one 16-byte word per lane at
// d_head 128, and a lane's values are pieces of 16 bytes (K) and 8 bytes (V) of which
// the lanes of a group cover 64 contiguous ones.
//
// Measured (a copy runs at 6.8 TB/s, writing alone at 4.0): 7,156 rows of 32 KV heads
// of 128 written in 29.4 us (150 MB, 5.1 TB/s; the ALU is busy two thirds of the time
// with maxima, masks and codes, five operations a value), 16 rows in 3.3 us; the same
// 7,156 rows with V transposed, as the prefill leaves it, in 59 us (30 by rows under the
// same profiler: V comes in pieces of two bytes); 38,458
// rows of four KV heads read in 17.5 us (101 MB, 5.8 TB/s; four fifths of the bytes are
// written), 183 rows in 1.9 us. A thread per group instead took 491 and 257 us for the
// large calls: its loads and stores are strided.
#include "kv4.cuh"

namespace svl {

constexpr int kRowWarps = 4, kRowThreads = kRowWarps * 32;

// Units of work of a call: one per sample without row_off, else quads, of which
// sample b has room for row_off[b + 1] / 8 - row_off[b] / 8 + 2 from number
// row_off[b] / 8 + 2 b on: enough for its rows wherever they start, and known
// without a sum over the samples.
__host__ __device__ inline int64_t row_units(int64_t rows, int n, bool ragged) {
  return ragged ? rows / 8 + 2 * static_cast<int64_t>(n) : n;
}

// A unit's place: positions p + i of a slot, p a multiple of 8, for i0 <= i < i1, from packed rows row + i.
struct Unit {
  int sample, i0, i1;
  int64_t p, row;
};
SVL_DEVINL bool find_unit(const Kv4Rows& a, int64_t u, int lane, Unit& q) {
  int64_t first = u, count = 1;
  q.sample = static_cast<int>(u);
  if (a.row_off) {
    // the last sample whose units start at or before u: 32 places at a time
    int lo = 0, n = a.n;
    while (n > 1) {
      const int step = (n + 31) / 32, b = lo + min(lane * step, n - 1);
      const bool le = a.row_off[b] / 8 + 2 * static_cast<int64_t>(b) <= u;
      const int hit = 31 - __clz(__ballot_sync(0xffffffffu, le) | 1u);
      const int at = min(hit * step, n - 1);
      n = min(step, n - at);
      lo += at;
    }
    q.sample = lo;
    first = a.row_off[lo];
    count = a.row_off[lo + 1] - first;
    u -= first / 8 + 2 * static_cast<int64_t>(lo);
  } else {
    u = 0;
  }
  const int64_t start = a.start ? a.start[q.sample] : 0;
  q.p = ((start >> 3) + u) * 8;  // (rounds down)
  q.row = first + q.p - start;
  int64_t end = start + count - q.p;
  if (end > a.rows - q.row) end = a.rows - q.row;
  q.i0 = static_cast<int>(start > q.p ? start - q.p : 0);
  q.i1 = static_cast<int>(end < 8 ? end : 8);
  return first >= 0 && q.i1 > q.i0;
}

// The code of x, rint(x / s) + 8 (of two nearest the even one) and at most 15. inv is 1 / s to within
// 2^-23 of it, so x * inv is off by less than 2^-19 for |x / s| <= 8. x and s are bf16 numbers: where x / s is not
// half an integer it is at least 2^-9 from one. Rounded to a multiple of 2^-15 (the last place of 384 = 1.5 * 2^8),
// x * inv is thus half an integer exactly where x / s is, and on its side of it elsewhere; the second sum (1.5 * 2^23)
// rounds it to an integer.
SVL_DEVINL float kv4_code(float x, float inv) {  // less 8, as a float
  const float t = fminf(__fmaf_rn(x, inv, 384.f), 391.f);
  return __fadd_rn(__fadd_rn(t, 12582912.f - 384.f), -12582912.f);
}
// Four codes as 16 bits, lowest first. (The sums of products run beside the maxima, masks and shifts, of which there
// are enough: the kernel is bound by those.)
SVL_DEVINL uint32_t four_codes(float x0, float x1, float x2, float x3, float inv) {
  float n = kv4_code(x3, inv);
  n = __fmaf_rn(n, 16.f, kv4_code(x2, inv));
  n = __fmaf_rn(n, 16.f, kv4_code(x1, inv));
  n = __fmaf_rn(n, 16.f, kv4_code(x0, inv));
  // (8 * (1 + 16 + 256 + 4096) more, above 2^23: an integer's bits)
  return __float_as_uint(__fadd_rn(n, 8388608.f + 34952.f));
}

SVL_DEVINL __nv_bfloat162 b2(uint32_t u) { return *reinterpret_cast<__nv_bfloat162*>(&u); }
SVL_DEVINL uint32_t u2(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }
SVL_DEVINL bool finite2(uint32_t u) { return (u & 0x7f80u) != 0x7f80u && (u & 0x7f800000u) != 0x7f800000u; }
SVL_DEVINL float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Largest value and negative of the smallest (halves of a word; a NaN stays one) of a lane's N pairs of values.
template <int N>
SVL_DEVINL uint32_t pair_range(const uint32_t* u) {
  __nv_bfloat162 hi = b2(u[0]), lo = hi;
#pragma unroll
  for (int i = 1; i < N; ++i) {
    hi = __hmax2_nan(hi, b2(u[i]));
    lo = __hmin2_nan(lo, b2(u[i]));
  }
  const uint32_t h = u2(hi), l = u2(lo) ^ 0x80008000u;
  return u2(__hmax2_nan(b2(__byte_perm(h, l, 0x5410)), b2(__byte_perm(h, l, 0x7632))));
}
SVL_DEVINL uint32_t wider(uint32_t x, uint32_t y) { return u2(__hmax2_nan(b2(x), b2(y))); }

// The ranges of N groups (a power of two), of which each of the lanes that differ in the bits LOW .. HIGH of their
// number has a part: a lane ends up with the whole of one, that whose number the lowest of these bits are. The lanes
// hand each other the half of the groups that they do not keep.
template <int N, int LOW, int HIGH>
SVL_DEVINL uint32_t group_range(uint32_t* r, int lane) {
  int n = N;
#pragma unroll
  for (int off = HIGH; off >= LOW; off >>= 1) {
    if (N <= off / LOW) {
#pragma unroll
      for (int i = 0; i < N; ++i) r[i] = wider(r[i], __shfl_xor_sync(0xffffffffu, r[i], off));
      continue;
    }
    n /= 2;
    const bool upper = lane & off;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      if (i >= n) break;
      const uint32_t keep = upper ? r[i + n] : r[i], give = upper ? r[i] : r[i + n];
      r[i] = wider(keep, __shfl_xor_sync(0xffffffffu, give, off));
    }
  }
  return r[0];
}

// The scale (bf16 bits) of a group of that range, and its reciprocal for kv4_code (0: every code is 8).
SVL_DEVINL uint32_t group_scale(uint32_t range, float& inv) {
  const float2 f = unpack_bf16x2(range);
  const float s = f.x >= f.y ? f.x * -0.125f : f.y * 0.125f;
  const bool zero = !(fabsf(s) >= 1.17549435e-38f);
  inv = zero ? 0.f : rcp_approx(s);
  if (!finite2(range)) {
    inv = 0.f;
    return 0x7fc0;
  }
  return zero ? 0u : __float_as_uint(s) >> 16;
}

// Codes of four pairs of values.
SVL_DEVINL uint32_t word_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float inv_lo, float inv_hi) {
  const float2 x = unpack_bf16x2(a), y = unpack_bf16x2(b), z = unpack_bf16x2(c), w = unpack_bf16x2(d);
  return __byte_perm(four_codes(x.x, x.y, y.x, y.y, inv_lo), four_codes(z.x, z.y, w.x, w.y, inv_hi), 0x5410);
}

template <int J>
SVL_DEVINL void store_words(void* p, const uint32_t* w) {
  if constexpr (J == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}
template <int J>
SVL_DEVINL void load_words(const void* p, uint32_t* w) {
  if constexpr (J == 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    w[0] = u.x;
    w[1] = u.y;
    w[2] = u.z;
    w[3] = u.w;
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x;
    w[1] = u.y;
  }
}

// A warp per (unit, KV head): block (unit, heads). VT: V is given transposed (row r of dimension c at
// v[c * v_col + r]), as the QKV projection leaves it.
template <int DH, bool VT>
__global__ void __launch_bounds__(kRowThreads) kv4_write_kernel(Kv4Rows a) {
  constexpr int J = DH / 32;
  pdl_begin(false);
  const int lane = threadIdx.x & 31, h = blockIdx.y * (blockDim.x / 32) + (threadIdx.x >> 5);
  Unit q;
  if (h >= a.c.kv || !find_unit(a, blockIdx.x, lane, q) || q.p < 0) return;
  if (q.p + q.i1 > a.c.max_len) {
    if (h == 0 && lane == 0) report(a.status, SVL_DEV_BAD_INDEX);
    if (q.p + q.i0 >= a.c.max_len) return;
    q.i1 = static_cast<int>(a.c.max_len - q.p);
  }
  if (!gate_on(a.gate, q.sample, a.gate.G ? h / (a.c.kv / a.gate.G) : 0)) return;
  uint8_t* tile = kv4_tile(a.c, q.sample * a.slot_step, h, static_cast<int>(q.p / kKv4Tile));
  const int quad = static_cast<int>(q.p % kKv4Tile) / 8;
  // what the lane converts: of K row lane / 4, dimensions 32 j + 8 t + 0..7; of V rows 2 t and 2 t + 1,
  // 32 j + 4 g + 0..3
  const int g = lane >> 2, t = lane & 3;
  const bool row_in = g >= q.i0 && g < q.i1;
  const bool even = 2 * t >= q.i0 && 2 * t < q.i1, odd = 2 * t + 1 >= q.i0 && 2 * t + 1 < q.i1;
  uint4 k[J];
  uint2 v[2][J];
  const __nv_bfloat16* kp = a.k + (q.row + g) * a.k_row + h * DH + 8 * t;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    k[j] = make_uint4(0, 0, 0, 0);
    if (row_in) k[j] = *reinterpret_cast<const uint4*>(kp + 32 * j);
  }
  const __nv_bfloat16* vp = a.v + (q.row + 2 * t) * a.v_row + (h * DH + 4 * g) * a.v_col;
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int j = 0; j < J; ++j) {
      v[x][j] = make_uint2(0, 0);
      if (!(x ? odd : even)) continue;
      if (VT) {
        uint16_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = reinterpret_cast<const uint16_t*>(vp)[(32 * j + i) * a.v_col + x];
        v[x][j] = make_uint2(y[0] | static_cast<uint32_t>(y[1]) << 16, y[2] | static_cast<uint32_t>(y[3]) << 16);
      } else {
        v[x][j] = *reinterpret_cast<const uint2*>(vp + x * a.v_row + 32 * j);
      }
    }
  {
    // groups j of row g: lane t ends up with the scale of the group t % J
    uint32_t r[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint32_t u4[4] = {k[j].x, k[j].y, k[j].z, k[j].w};
      r[j] = pair_range<4>(u4);
    }
    float inv;
    const uint32_t s = group_scale(group_range<J, 1, 2>(r, lane), inv);
    uint32_t w4[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const float i = __shfl_sync(0xffffffffu, inv, (lane & ~3) | j);
      w4[j] = word_codes(k[j].x, k[j].y, k[j].z, k[j].w, i, i);
    }
    if (row_in) {
      store_words<J>(tile + (quad * 32 + lane) * J * 4, w4);
      uint16_t* scales = reinterpret_cast<uint16_t*>(tile + kv4_k_scales(DH));
      if (t < J) scales[(quad * 8 + g) * J + t] = static_cast<uint16_t>(s);
    }
  }
  // groups j of rows 2 t (number 2 j) and 2 t + 1 (2 j + 1): lane g ends up with the scale of number g % (2 J)
  uint32_t r[2 * J];
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint32_t u4[2] = {v[x][j].x, v[x][j].y};
      r[2 * j + x] = pair_range<2>(u4);
    }
  float inv;
  const uint32_t s = group_scale(group_range<2 * J, 4, 16>(r, lane), inv);
  uint32_t w4[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const float e = __shfl_sync(0xffffffffu, inv, 8 * j + t), o = __shfl_sync(0xffffffffu, inv, 8 * j + 4 + t);
    w4[j] = word_codes(v[0][j].x, v[0][j].y, v[1][j].x, v[1][j].y, e, o);
  }
  uint8_t* codes = tile + kv4_v_codes(DH) + (quad * 32 + lane) * J * 4;
  if (even && odd) {
    store_words<J>(codes, w4);
  } else if (even || odd) {  // the other row of the pair stays
#pragma unroll
    for (int j = 0; j < J; ++j)
      reinterpret_cast<uint16_t*>(codes)[2 * j + odd] = static_cast<uint16_t>(w4[j] >> (16 * odd));
  }
  if (g < 2 * J && (g & 1 ? odd : even))
    reinterpret_cast<uint16_t*>(tile + kv4_v_scales(DH))[(quad * 4 + t) * 2 * J + g] = static_cast<uint16_t>(s);
}

// One row per slot: a warp per (slot, KV head, K or V), four dimensions a lane. Bound by latency: 16 slots of 32 KV heads
// of 128 take 1.8 us, 3.3 with the warps of the kernel above, of whose eight positions one has a row (V transposed, in a
// decode step, the layer took 5 us less, with 64 slots 7).
template <int DH, bool VT>
__global__ void __launch_bounds__(kRowThreads) kv4_append_kernel(Kv4Rows a) {
  constexpr int J = DH / 32;
  pdl_begin(false);
  const int lane = threadIdx.x & 31, warp = blockIdx.y * (blockDim.x / 32) + (threadIdx.x >> 5), b = blockIdx.x;
  const int h = warp >> 1;
  const bool of_v = warp & 1, in = 4 * lane < DH;
  const int pos = a.start ? a.start[b] : 0;
  if (h >= a.c.kv || pos < 0) return;
  if (pos >= a.c.max_len) {
    if (warp == 0 && lane == 0) report(a.status, SVL_DEV_BAD_INDEX);
    return;
  }
  if (!gate_on(a.gate, b, a.gate.G ? h / (a.c.kv / a.gate.G) : 0)) return;
  const int d = h * DH + 4 * lane;
  uint2 x = make_uint2(0, 0);
  if (in) {
    if (VT && of_v) {
      const uint16_t* src = reinterpret_cast<const uint16_t*>(a.v) + b * a.v_row + d * a.v_col;
      uint16_t y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = src[i * a.v_col];
      x = make_uint2(y[0] | static_cast<uint32_t>(y[1]) << 16, y[2] | static_cast<uint32_t>(y[3]) << 16);
    } else {
      x = *reinterpret_cast<const uint2*>((of_v ? a.v + b * a.v_row : a.k + b * a.k_row) + d);
    }
  }
  // the eight lanes of a group
  const uint32_t u[2] = {x.x, x.y};
  uint32_t r = pair_range<2>(u);
#pragma unroll
  for (int off = 1; off < 8; off <<= 1) r = wider(r, __shfl_xor_sync(0xffffffffu, r, off));
  float inv;
  const uint32_t s = group_scale(r, inv);
  const float2 lo = unpack_bf16x2(x.x), hi = unpack_bf16x2(x.y);
  const uint16_t codes = static_cast<uint16_t>(four_codes(lo.x, lo.y, hi.x, hi.y, inv));
  if (!in) return;
  uint8_t* tile = kv4_tile(a.c, b * a.slot_step, h, pos / kKv4Tile);
  const int p = pos % kKv4Tile, j = lane >> 3, i = lane & 7;
  const int word = of_v ? p / 8 * 32 + i * 4 + p % 8 / 2 : p * 4 + i / 2, half = of_v ? p & 1 : i & 1;
  reinterpret_cast<uint16_t*>(tile + (of_v ? kv4_v_codes(DH) : 0))[(word * J + j) * 2 + half] = codes;
  if (i == 0)
    reinterpret_cast<uint16_t*>(tile + (of_v ? kv4_v_scales(DH) : kv4_k_scales(DH)))
        [of_v ? (p / 2 * J + j) * 2 + (p & 1) : p * J + j] = static_cast<uint16_t>(s);
}

// The lowest nibble of each half, less 8, times the halves of s, as bf16 (the product rounded once).
SVL_DEVINL uint32_t two_values(uint32_t x, uint32_t s, uint32_t k128) {
  uint32_t y;  // 128 + n (k128: 128 in both halves, in a register), less 136
  asm("lop3.b32 %0, %1, 0x000f000f, %2, 0xea;" : "=r"(y) : "r"(x), "r"(k128));
  return u2(__hmul2(__hadd2(b2(y), b2(0xc308c308u)), b2(s)));
}

// A warp per (unit, KV head), as for writing; positions that the cache does not have read as 0.
template <int DH>
__global__ void __launch_bounds__(kRowThreads) kv4_read_kernel(Kv4Rows a) {
  constexpr int J = DH / 32;
  pdl_begin(false);
  const int lane = threadIdx.x & 31, h = blockIdx.y * (blockDim.x / 32) + (threadIdx.x >> 5);
  Unit q;
  if (h >= a.c.kv || !find_unit(a, blockIdx.x, lane, q)) return;
  const int g = lane >> 2, t = lane & 3;
  const bool held = q.p >= 0 && q.p < a.c.max_len;
  uint32_t k128;
  asm volatile("mov.b32 %0, 0x43004300;" : "=r"(k128));
  uint32_t k[J], v[J], sk[J / 2], sv[J];
#pragma unroll
  for (int j = 0; j < J; ++j) k[j] = v[j] = sk[j / 2] = sv[j] = 0;
  if (held) {
    const uint8_t* tile = kv4_tile(a.c, q.sample * a.slot_step, h, static_cast<int>(q.p / kKv4Tile));
    const int quad = static_cast<int>(q.p % kKv4Tile) / 8;
    load_words<J>(tile + (quad * 32 + lane) * J * 4, k);
    load_words<J>(tile + kv4_v_codes(DH) + (quad * 32 + lane) * J * 4, v);
#pragma unroll
    for (int j = 0; j < J / 2; ++j)
      sk[j] = reinterpret_cast<const uint32_t*>(tile + kv4_k_scales(DH) + (quad * 8 + g) * J * 2)[j];
    load_words<J>(tile + kv4_v_scales(DH) + (quad * 4 + t) * J * 4, sv);
  }
  // rows that the cache does not have read as 0
  const int in = held ? static_cast<int>(q.p + 8 <= a.c.max_len ? 8 : a.c.max_len - q.p) : 0;
  if (in < 8) {
    const uint32_t keep = (2 * t < in ? 0xffffu : 0u) | (2 * t + 1 < in ? 0xffff0000u : 0u);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (g >= in) {
        k[j] = 0x88888888u;
        sk[j / 2] = 0;
      }
      v[j] = (v[j] & keep) | (0x88888888u & ~keep);
      sv[j] &= keep;
    }
  }
  if (g >= q.i0 && g < q.i1) {
    __nv_bfloat16* out = a.k_out + (q.row + g) * a.k_row + h * DH + 8 * t;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint32_t s = __byte_perm(sk[j / 2], 0, j & 1 ? 0x3232 : 0x1010);
      uint32_t y[4];  // dimensions i and i + 4
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = two_values(k[j] >> (4 * i), s, k128);
      *reinterpret_cast<uint4*>(out + 32 * j) =
          make_uint4(__byte_perm(y[0], y[1], 0x5410), __byte_perm(y[2], y[3], 0x5410), __byte_perm(y[0], y[1], 0x7632),
                     __byte_perm(y[2], y[3], 0x7632));
    }
  }
  const bool even = 2 * t >= q.i0 && 2 * t < q.i1, odd = 2 * t + 1 >= q.i0 && 2 * t + 1 < q.i1;
  __nv_bfloat16* out = a.v_out + (q.row + 2 * t) * a.v_row + h * DH + 4 * g;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    uint32_t y[4];  // dimension i of rows 2 t and 2 t + 1
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = two_values(v[j] >> (4 * i), sv[j], k128);
    if (even)
      *reinterpret_cast<uint2*>(out + 32 * j) =
          make_uint2(__byte_perm(y[0], y[1], 0x5410), __byte_perm(y[2], y[3], 0x5410));
    if (odd)
      *reinterpret_cast<uint2*>(out + a.v_row + 32 * j) =
          make_uint2(__byte_perm(y[0], y[1], 0x7632), __byte_perm(y[2], y[3], 0x7632));
  }
}

static cudaError_t row_launch(void (*kernel)(Kv4Rows), const Kv4Rows& a, cudaStream_t s) {
  const int64_t units = row_units(a.rows, a.n, a.row_off != nullptr);
  if (units > 0x7fffffff) return cudaErrorInvalidConfiguration;
  if (units == 0) return cudaSuccess;
  const int warps = a.c.kv < kRowWarps ? a.c.kv : kRowWarps;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(units), (a.c.kv + warps - 1) / warps), warps * 32, 0, s, a);
}

cudaError_t launch_kv4_write(const Kv4Rows& a, cudaStream_t s) {
  if (!a.row_off) {
    const auto kernel = a.c.dh == 128 ? (a.v_col == 1 ? kv4_append_kernel<128, false> : kv4_append_kernel<128, true>)
                                      : (a.v_col == 1 ? kv4_append_kernel<64, false> : kv4_append_kernel<64, true>);
    const int warps = 2 * a.c.kv < kRowWarps ? 2 * a.c.kv : kRowWarps;
    return launch_pdl(kernel, dim3(a.n, (2 * a.c.kv + warps - 1) / warps), warps * 32, 0, s, a);
  }
  if (a.c.dh == 128) return row_launch(a.v_col == 1 ? kv4_write_kernel<128, false> : kv4_write_kernel<128, true>, a, s);
  return row_launch(a.v_col == 1 ? kv4_write_kernel<64, false> : kv4_write_kernel<64, true>, a, s);
}
cudaError_t launch_kv4_read(const Kv4Rows& a, cudaStream_t s) {
  return row_launch(a.c.dh == 128 ? kv4_read_kernel<128> : kv4_read_kernel<64>, a, s);
}

__global__ void kv4_lengths_kernel(const int* cu_seqlens, int n, int beams, int* len) {
  pdl_begin(false);
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) len[i] = cu_seqlens[i / beams + 1] - cu_seqlens[i / beams];
}
cudaError_t launch_kv4_lengths(const int* cu_seqlens, int B, int beams, int* len, cudaStream_t s) {
  return launch_pdl(kv4_lengths_kernel, dim3((B * beams + 127) / 128), 128, 0, s, cu_seqlens, B * beams, beams, len);
}

// Reorder: block (part, KV head, layer and sample) moves its part of the bytes that the sample's slots hold of the head
// from position `from` on, 16 bytes a thread of all slots: each thread reads what the moved slots take over before it
// writes any of them, so the slots change in place whatever the parents are. Bound by the bytes read and written (the
// slots that stay are not touched); a slot's bytes of a head are contiguous. 32 whole slots of 300 to 640 positions, 32
// heads, four layers: 43.8 us (90 MB read, 166 MB written, 5.8 TB/s); the last 1 to 64 positions of 16 slots: 5.4 us.
constexpr int kMoveThreads = 256, kMoveUnits = 65535;
template <int W>
__global__ void __launch_bounds__(kMoveThreads) kv4_reorder_kernel(Kv4Reorder a) {
  pdl_begin(false);
  const uint32_t samples = a.c.n_slots / a.W, unit = a.unit0 + blockIdx.z;
  const int sample = unit % samples, layer = unit / samples;
  const int s0 = sample * a.W, TB = kv4_tile_bytes(a.c.dh);
  const int first = (a.from ? max(a.from[sample], 0) : 0) / kKv4Tile;
  // of each slot that moves: the parent, and the tiles that it holds
  int parent[W], end[W], last = first;
  bool bad = false;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    end[w] = 0;
    parent[w] = w < a.W ? a.parent[s0 + w] : w;
    if (parent[w] == w) continue;
    if (parent[w] < 0 || parent[w] >= a.W) {
      bad = true;
      continue;
    }
    const int len = min(a.len[s0 + parent[w]], a.c.max_len);
    end[w] = len > 0 ? (len - 1) / kKv4Tile + 1 : 0;
    last = max(last, end[w]);
  }
  if (bad && threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0) report(a.status, SVL_DEV_BAD_INDEX);
  const int64_t n = static_cast<int64_t>(last - first) * (TB / 16);
  const size_t slot = static_cast<size_t>(a.c.kv) * a.c.tiles * TB;
  uint4* base = reinterpret_cast<uint4*>(a.c.data + (static_cast<size_t>(layer) * a.c.n_slots + s0) * slot +
                                         (static_cast<size_t>(blockIdx.y) * a.c.tiles + first) * TB);
  for (int64_t i = blockIdx.x * kMoveThreads + threadIdx.x; i < n; i += gridDim.x * kMoveThreads) {
    const int tile = first + static_cast<int>(i / (TB / 16));
    uint4 got[W];
#pragma unroll
    for (int w = 0; w < W; ++w)
      if (tile < end[w]) got[w] = base[parent[w] * (slot / 16) + i];
#pragma unroll
    for (int w = 0; w < W; ++w)
      if (tile < end[w]) base[w * (slot / 16) + i] = got[w];
  }
}

// Parts of at least 4 KB (a step of a block), as many as give each SM eight blocks; a launch for every 65,535 layers and
// samples (along x, the only longer axis, they would be the fastest to change: the large call 43.8 -> 44.9 us).
int kv4_reorder_launches(const Kv4Reorder& a) { return (a.layers * (a.c.n_slots / a.W) - 1) / kMoveUnits + 1; }
cudaError_t launch_kv4_reorder(Kv4Reorder a, cudaStream_t s) {
  const int units = a.layers * (a.c.n_slots / a.W);
  const int64_t heads = static_cast<int64_t>(a.c.kv) * units;
  const int64_t words = static_cast<int64_t>(a.c.tiles) * kv4_tile_bytes(a.c.dh) / 16;
  const int64_t steps = (words + kMoveThreads - 1) / kMoveThreads;
  int64_t parts = (8 * 152 + heads - 1) / heads;
  parts = parts < steps ? parts : steps;
  const auto kernel = a.W <= 4 ? kv4_reorder_kernel<4> : a.W <= 8 ? kv4_reorder_kernel<8> : kv4_reorder_kernel<16>;
  for (a.unit0 = 0; a.unit0 < units; a.unit0 += kMoveUnits) {
    const int n = units - a.unit0 < kMoveUnits ? units - a.unit0 : kMoveUnits;
    const dim3 grid(static_cast<unsigned>(parts), a.c.kv, static_cast<unsigned>(n));
    const cudaError_t e = launch_pdl(kernel, grid, kMoveThreads, 0, s, a);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace svl
