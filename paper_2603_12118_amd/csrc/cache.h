// Declarations of the LLM task's side: rotation of queries and keys, the 4-bit cache and attention over it.
#pragma once
#include "common.h"

namespace cs {

// n / d as a product with recip64(d), for n d < 2^64 (a slot times the tokens of a page: a pool of 2^44 slots would be a petabyte)
inline uint64_t recip64(uint64_t d) { return ~0ull / d + 1; }

// Workgroups of 256 threads that a launch may have: HIP refuses more than 2^32 - 1 threads along a dimension of the grid.
constexpr int64_t MAX_GROUPS = 0xffffffffll / 256;

struct QkArgs {
  const void *q, *k;
  void *q_out, *k_out;
  int64_t q_row, k_row, q_out_row, k_out_row;   // elements between rows
  int32_t norm;                                 // 0: gains are not looked at
  const float *q_gain, *k_gain;
  const float* cos_sin;                         // [n_positions, half, 2]
  const int32_t* positions;                     // [n_rows, axes]
  int64_t n_rows, n_positions;
  int32_t n_heads, n_kv_heads, head_dim, half, axes;
  // the axis pair j follows: 1 from end0 on or where j % 3 == 1 below lim1, 2 from end1 on or where j % 3 == 2 below lim2, else 0
  int32_t end0, end1;                           // contiguous sections (the number of pairs where they are interleaved)
  int32_t lim1, lim2;                           // interleaved ones (else 0)
  float eps;
  int32_t* err;
  int32_t parts;                                // set by the launcher: workgroup rows that share out a token's heads
};
cs_status launch_qk_norm_rope(const QkArgs& a, int dtype, hipStream_t s);

// A pool of pages (layout: cs_cache_config)
struct CacheShape {
  int32_t n_kv_heads, head_dim, page_tokens;
  int64_t n_pages;
  int64_t head_bytes;     // block of one page and head
  int64_t slots;          // n_pages * page_tokens
  uint64_t page_recip;    // recip64(page_tokens)
};
inline CacheShape cache_shape(const cs_cache_config& c) {
  const int64_t head_bytes = (int64_t)c.page_tokens * (c.head_dim + 2 * (c.head_dim / 32));
  return CacheShape{c.n_kv_heads, c.head_dim, c.page_tokens, c.n_pages, head_bytes, c.n_pages * c.page_tokens, recip64((uint64_t)c.page_tokens)};
}
struct CacheRows {
  unsigned char* pool;
  void *k, *v;
  int64_t k_row, v_row;   // elements
  const int64_t* slots;
  int64_t n_rows;
  CacheShape shape;
  int32_t* err;
};
cs_status launch_cache_write(const CacheRows& a, int dtype, hipStream_t s);
cs_status launch_cache_read(const CacheRows& a, int dtype, hipStream_t s);

struct CacheAttnArgs {
  const unsigned char* pool;
  const bf16_t* q;
  bf16_t* out;
  int64_t q_row, out_row;
  const int32_t *cu, *n_keys, *table;
  int64_t n_queries, max_keys;
  int32_t n_seqs, max_queries, table_width;
  int32_t n_heads, group; // group: heads that share a key/value head
  float scale_log2;       // |softmax scale| * log2(e), not zero
  uint32_t q_sign;        // 0x80008000 where the scale is negative: the queries turn their signs
  int32_t causal;
  CacheShape shape;
  int32_t* err;
  // set by the launcher
  int32_t more_than, at_most;   // rows of the sequences that a launch takes: the others are another's
  int32_t rows;           // rows (a row: a query and a head) a workgroup takes: 16 or 32 (their keys shared out to its waves) or 128
  int32_t row_blocks;     // blocks of so many rows that a sequence and key/value head have at most
  int32_t target;         // workgroups that fill the chip once
  int32_t least;          // tiles of 32 keys that a workgroup takes at least, if there are so many
  int32_t blocks;         // workgroups of the launch: those without work end at once (0: more than a grid may have, here or in the joining launch)
  int32_t join;           // 0: no sequence can be shared out; else the threads, in sixteens, that share a row's parts
  int32_t planned;        // the shares are worked out by a launch before
  int64_t units;          // ... units that the joining launch is laid out for
  int32_t join_groups;    // workgroups of the joining launch for a block of rows
  // parts, where a sequence's keys are shared out: [blocks, rows, head_dim] sums not yet normalised, and [blocks, rows, 2]
  // their maximum (log2 domain) and weight
  float *part_o, *part_ml;
  int32_t* share_of;      // [n_seqs, 4] first workgroup, shares, tiles of a share, first unit: left by the first launch, or by one before it, for the joining one
};
// Bytes of workspace the launches need, from the sizes alone; CS_ERR_UNSUPPORTED where one of them would be too large.
cs_status plan_cache_attention(const CacheAttnArgs& a, size_t& bytes);
cs_status launch_cache_attention(const CacheAttnArgs& a, void* workspace, hipStream_t s);

}  // namespace cs
