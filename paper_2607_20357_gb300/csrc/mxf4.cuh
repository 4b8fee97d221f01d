// Matrices in 4-bit floating point with a power-of-two scale for every 32
// values of a row (MXFP4), as the tcgen05 block-scaled MMA (kind::mxf4) takes
// its operands.
//
//   codes   e2m1 (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5,
//           2, 3, 4, 6), two to a byte, the earlier value in the low nibble. A
//           row takes ceil(cols / 32) * 16 bytes; what its last block has
//           behind the row's end is zero.
//   scales  a byte b per block stands for 2^(b - 127), 255 for NaN. The bytes of
//           128 rows and four blocks (128 columns) are one tile of 512 bytes,
//           [row % 32][row % 128 / 32][block % 4]: sixteen consecutive bytes
//           hold four rows, 32 apart, of four blocks each, which is how tensor
//           memory wants them (a 32-bit column per 32 rows), so a tile goes
//           there by one tcgen05.cp as it lies. Tiles are
//           [ceil(rows / 128)][ceil(cols / 128)].
#pragma once

#include <atomic>

#include "common.cuh"

namespace svl {

constexpr int kMxBlock = 32;       // values that share a scale
constexpr int kMxTileBytes = 512;  // scales of 128 rows x 128 columns

__host__ __device__ constexpr int64_t mxf4_row_bytes(int64_t cols) { return (cols + kMxBlock - 1) / kMxBlock * 16; }
__host__ __device__ constexpr int64_t mxf4_scale_tiles(int64_t cols) { return (cols + 127) / 128; }
__host__ __device__ constexpr int64_t mxf4_scale_bytes(int64_t rows, int64_t cols) {
  return (rows + 127) / 128 * mxf4_scale_tiles(cols) * kMxTileBytes;
}

enum Mxf4Source : int { MX_ROWS = 0, MX_GAIN = 1, MX_SWIGLU = 2 };

struct Mxf4Rows {
  const __nv_bfloat16* src;    // the rows; MX_SWIGLU: the gate
  const __nv_bfloat16* other;  // MX_GAIN: the gain [cols]; MX_SWIGLU: up
  int64_t ld_src, ld_other;
  int64_t rows;
  int cols;
  uint8_t* codes;
  int64_t ld_codes;  // bytes
  uint8_t* scale;
  float eps;
  float* inv_rms;  // [rows] or nullptr
  int num_sms;
};
cudaError_t launch_mxf4_quantize(Mxf4Source source, const Mxf4Rows& a, cudaStream_t s);

struct Mxf4Read {
  const uint8_t* codes;
  int64_t ld_codes;
  const uint8_t* scale;
  int64_t rows;
  int cols;
  __nv_bfloat16* dst;
  int64_t ld_dst;
  int num_sms;
};
cudaError_t launch_mxf4_dequantize(const Mxf4Read& a, cudaStream_t s);

// C[m, n] = row_factor[m] * sum_k A[m, k] B[n, k] + residual[m, n]
struct Mxf4Gemm {
  const uint8_t* a;
  const uint8_t* b;
  int64_t ld_a, ld_b;  // bytes
  const uint8_t* a_scale;
  const uint8_t* b_scale;
  int M, N, K;
  const float* row_factor;  // [M] or nullptr
  const void* residual;     // C's type, or nullptr
  int64_t ld_residual;
  void* c;
  int64_t ld_c;
  bool f32;  // C is float32, else bf16
  uint32_t* status;
  int num_sms;
};
// cudaErrorInvalidValue: strides that no tensor map takes
cudaError_t launch_mxf4_gemm(const Mxf4Gemm& g, cudaStream_t s);
// Its kernel for more than 128 rows, on CTA pairs.
cudaError_t launch_mxf4_pair(const Mxf4Gemm& g, cudaStream_t s);
// How many clusters of 2, 4 or 8 CTAs the device runs at once, an SM to a CTA.
int mxf4_clusters(int ctas);

// Lets `kernel` have `bytes` of shared memory, the same in every call. Set once
// per device (0.3 us of a call's 3.6); `devices`: the kernel's own.
inline cudaError_t mxf4_allow_smem(const void* kernel, int bytes, std::atomic<uint64_t>* devices) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
  if (devices->load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) devices->fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// 2-D tensor map of `rows` rows of `bytes` bytes, `ld` bytes apart: boxes of
// 128 bytes x box_rows with 128-byte swizzle; what lies outside reads as zeros.
bool make_byte_map(CUtensorMap* m, const void* ptr, uint64_t rows, uint64_t bytes, uint64_t ld, uint32_t box_rows);
// The scales of `rows` rows of `cols` values: boxes of two tiles (256 columns) x box_tiles tiles of 128 rows.
bool make_scale_map(CUtensorMap* m, const void* ptr, int64_t rows, int64_t cols, uint32_t box_tiles);
// A result [rows, cols] of float32 or bf16, `ld` elements apart: boxes of 128 bytes x 32 rows with 128-byte swizzle.
bool make_result_map(CUtensorMap* m, const void* ptr, bool f32, uint64_t rows, uint64_t cols, uint64_t ld);

SVL_DEVINL void mx_abort(volatile int* abort, uint32_t* status) {
  *abort = 1;
  report(status, SVL_DEV_TIMEOUT);
}

}  // namespace svl
