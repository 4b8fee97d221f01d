// The 4-bit KV cache: layout, arguments and launchers of the kernels on it, and
// beam selection.
#pragma once

#include "kernels.cuh"

namespace svl {

// One layer's cache is [slots][KV heads][tiles] of tiles of 32 positions. A group
// is 32 consecutive dimensions of a row of K or V; J = d_head / 32 groups a row. A
// tile is 36 * d_head bytes:
//   codes of K   [32 rows][4 t][J j] words of eight nibbles, lowest first:
//                dimensions 32 j + 8 t + 0..7
//   codes of V   [2 strips][2 quads][8 g][4 t][J j] words: rows 16 strip + 8 quad
//                + 2 t in the low half and the next row in the high half,
//                dimensions 32 j + 4 g + 0..3, lowest nibble first
//   scales of K  [32 rows][J] bf16
//   scales of V  [16 row pairs][J][2] bf16
// so that what one lane of a 16 x 8 matrix instruction needs of K (rows by
// dimensions) and of V^T (dimensions by rows, two rows side by side) is contiguous
// and becomes operands by masking.
constexpr int kKv4Tile = 32;
__host__ __device__ constexpr int kv4_tile_bytes(int dh) { return 36 * dh; }
__host__ __device__ constexpr int kv4_v_codes(int dh) { return 16 * dh; }
__host__ __device__ constexpr int kv4_k_scales(int dh) { return 32 * dh; }
__host__ __device__ constexpr int kv4_v_scales(int dh) { return 34 * dh; }

struct Kv4Cache {
  uint8_t* data;
  int n_slots, kv, dh, max_len, tiles;
};

SVL_DEVINL uint8_t* kv4_tile(const Kv4Cache& c, int slot, int head, int tile) {
  return c.data + ((static_cast<size_t>(slot) * c.kv + head) * c.tiles + tile) * kv4_tile_bytes(c.dh);
}

// Whether a head group runs (group_gate == nullptr: all of them).
struct HeadGate {
  const uint8_t* layer_gate;
  const uint8_t* group_gate;
  int L, l, P, G;
};
SVL_DEVINL bool gate_on(const HeadGate& g, int b, int group) {
  return !g.group_gate || g.l < g.P ||
         (g.layer_gate[b * g.L + g.l] && g.group_gate[(static_cast<size_t>(b) * g.L + g.l) * g.G + group]);
}

// Rows to write: element (row r, column c) of K at k[r * k_row + c], of V at
// v[r * v_row + c * v_col]. Sample b's rows row_off[b] .. row_off[b + 1) - 1 (or row b,
// without row_off) go to slot b * slot_step, positions start[b] + 0, 1, ...
struct Kv4Rows {
  Kv4Cache c;
  int64_t rows;
  int n;  // samples
  int slot_step;
  const int* row_off;
  const int* start;  // nullptr: 0
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  int64_t k_row, v_row, v_col;
  __nv_bfloat16* k_out;  // read: rows out instead
  __nv_bfloat16* v_out;
  uint32_t* status;
  HeadGate gate;
};
cudaError_t launch_kv4_write(const Kv4Rows& a, cudaStream_t s);
cudaError_t launch_kv4_read(const Kv4Rows& a, cudaStream_t s);

// len[b * beams + w] = cu_seqlens[b + 1] - cu_seqlens[b]
cudaError_t launch_kv4_lengths(const int* cu_seqlens, int B, int beams, int* len, cudaStream_t s);

struct Kv4Attn {
  Kv4Cache c;
  int A, rows;
  const __nv_bfloat16* q;
  int64_t ldq;
  __nv_bfloat16* out;
  int64_t ldo;
  const int* start;
  int window, sinks;
  float scale;
  HeadGate gate;
  bool late;  // see QuantArgs
  void* ws;
  int num_sms;
};
size_t kv4_attn_workspace(const Kv4Cache& c, int A, int rows);
cudaError_t launch_kv4_attention(const Kv4Attn& a, cudaStream_t s);
int kv4_attn_launches(const Kv4Attn& a);
constexpr int kKv4MaxRows = 16;  // query rows per slot

struct Kv4Reorder {
  Kv4Cache c;
  int layers, W;
  int unit0;  // the launch's first (layer, sample)
  const int* parent;
  const int* from;
  const int* len;
  uint32_t* status;
};
constexpr int kKv4MaxBeams = 16;
cudaError_t launch_kv4_reorder(Kv4Reorder a, cudaStream_t s);
int kv4_reorder_launches(const Kv4Reorder& a);

struct BeamArgs {
  int S, W, V, K;
  const float* logits;
  int64_t ld;
  const float* scores;      // [S, W]
  const uint8_t* finished;  // [S, W] or nullptr
  int eos;
  float* scores_out;        // [S, K]
  int* parent;
  int* token;
  uint8_t* finished_out;    // or nullptr
  void* ws;
};
constexpr int kBeamMaxTake = 32;
size_t beam_workspace(int S, int W, int V, int K);
cudaError_t launch_beam_select(const BeamArgs& a, cudaStream_t s);

}  // namespace svl
