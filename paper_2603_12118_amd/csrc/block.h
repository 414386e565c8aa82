// Declarations of what an LLM layer does behind its attention: norms around a block, products with packed weights, a
// mixture-of-experts layer.
#pragma once
#include "common.h"

namespace cs {

struct NormResidualArgs {
  const void *x, *residual, *gate;          // gate: nullptr, one row (gate_row 0) or a row each
  void *r_out, *y;
  int64_t x_row, residual_row, gate_row, r_row, y_row;   // elements between rows
  const float *post_gain, *post_bias, *pre_gain, *pre_bias;
  int64_t n_rows;
  int32_t width;
  float eps, residual_scale, block_scale;
  float inv_width;                          // set by the launcher
};
cs_status launch_norm_residual(const NormResidualArgs& a, bool layer, int dtype, int residual_dtype, hipStream_t s);

// Packed weights: `matrices` of n rows of k values.  A matrix is tiles of 16 rows, the last one filled with zeros; a tile is blocks of
// 128 values along k, behind them (4 bits) their scales.  Lane l of a wave has row l % 16 and, in step s of a block, the eight values
// 32 s + 8 (l / 16) ..: the operand of a 16 x 16 x 32 product.
//   bf16:   step s of block b at 4096 b + 1024 s + 16 l (no more steps than k has)
//   4 bits: block b at 1024 b + 16 l + 4 s, eight codes, low bits first; behind the nb blocks 64 b + 4 (l % 16) + s the scale byte
struct PackedShape {
  int32_t format, n, k;
  int64_t matrices;
  int32_t tiles;            // of 16 rows
  int32_t blocks;           // of 128 values, the last one maybe of 32, 64 or 96
  int64_t tile_bytes;
};
inline PackedShape packed_shape(int32_t format, int64_t matrices, int32_t n, int32_t k) {
  const int32_t tiles = (int32_t)(((int64_t)n + 15) / 16), blocks = (int32_t)(((int64_t)k + 127) / 128);
  return PackedShape{format, n, k, matrices, tiles, blocks, format == CS_WEIGHTS_E2M1 ? (int64_t)blocks * 1088 : (int64_t)k * 32};
}
inline int64_t matrix_bytes(const PackedShape& p) { return p.tiles * p.tile_bytes; }

struct PackArgs {
  const void* w;            // [matrices, n, k] to pack, or (read) to fill
  int64_t w_row, w_matrix;  // elements
  unsigned char* packed;
  PackedShape shape;
  int32_t* err;
  int64_t first;            // set by the launcher: first tile of the launch
};
cs_status launch_weights_pack(const PackArgs& a, int dtype, hipStream_t s);
cs_status launch_weights_read(const PackArgs& a, int dtype, hipStream_t s);

struct LinearArgs {
  const unsigned char* packed;
  PackedShape shape;
  const bf16_t* x;
  int64_t x_row;
  const float* bias;
  void* out;
  int64_t out_row;
  int64_t n_rows;
  // set by the launcher
  int32_t splits, blocks_of_split, m_tiles;
  float* parts;             // [splits, n_rows / 16, tiles, 64 lanes, 4]
};
cs_status plan_linear_packed(const LinearArgs& a, size_t& bytes);
cs_status launch_linear_packed(const LinearArgs& a, int out_dtype, void* workspace, hipStream_t s);

constexpr int MAX_TOP = 32;
constexpr int MAX_EXPERTS = 1024;
constexpr int64_t MOE_ROWS = 4096;
constexpr int64_t MOE_WORKSPACE = (int64_t)1 << 31;      // bytes at most

struct MoeArgs {
  const bf16_t* x;
  int64_t x_row;
  const bf16_t* router;     // [experts, hidden]
  const float* choice_bias; // [experts] or nullptr
  const unsigned char* live;// [n_rows] or nullptr
  const unsigned char *up, *down;
  PackedShape up_shape, down_shape;
  bf16_t* y;
  int64_t y_row;
  int32_t* experts_out;     // [n_rows, top]
  float* weights_out;
  int64_t n_rows;
  int32_t hidden, inter, experts, shared, top, sigmoid, renormalise;
  float scale;
  // set by the launcher (workspace)
  int32_t slots;            // top + shared
  double* logits;           // [rows, experts]
  int32_t* counts;          // [experts + shared]
  int32_t* lists;           // [experts + shared, rows]: row * slots + slot
  bf16_t* h;                // [rows, slots, inter]
  float* parts;             // [rows, slots, hidden]
  int32_t list_row;
};
size_t moe_workspace(const MoeArgs& a);
cs_status launch_moe(const MoeArgs& a, void* workspace, hipStream_t s);

}  // namespace cs
