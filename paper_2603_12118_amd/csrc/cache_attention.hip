// Attention over the 4-bit cache.
//
// Rows: the queries of a sequence times the heads that share a key/value head, query by query.  A wave takes 16 rows and
// walks tiles of 32 keys.  S^T = K Q^T with v_mfma_f32_16x16x32_bf16, twice 16 keys: lane l then holds row l % 16 and keys
// 8p .. 8p+7 of the tile, p = l / 16 (key m of product u is token 8 (m / 4) + 4 u + m % 4 of the tile), which after the
// exponential is the B operand of O^T = V^T P^T as it stands.  A code times its power of two is exact in bf16, and the
// conversion instruction does it two codes at a time, so the cache is widened in registers between its load and the matrix
// instruction and what crosses the memory bus is 4.25 bits a value.
#include "cache.h"

#include <algorithm>
#include <type_traits>

namespace cs {

typedef __bf16 abf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 abf16x2 __attribute__((ext_vector_type(2)));
typedef float af32x2 __attribute__((ext_vector_type(2)));
typedef float af32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int au32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int au32x4 __attribute__((ext_vector_type(4)));
template <int N> struct Words;
template <> struct Words<2> { typedef au32x2 type; };
template <> struct Words<4> { typedef au32x4 type; };

__device__ __forceinline__ uint32_t pack2_k(float a, float b) {
  const af32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, abf16x2));
}
// codes 2 SEL, 2 SEL + 1 of a word, times 2^(byte - 127) where the byte is in bits 23..30 of `scale`: two bf16
template <int SEL>
__device__ __forceinline__ uint32_t widen2(uint32_t w, uint32_t scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, __uint_as_float(scale), SEL));
}
// byte B of w in bits 23..30
template <int B>
__device__ __forceinline__ uint32_t scale_of(uint32_t w) {
  return (B == 3 ? w >> 1 : w << (23 - 8 * B)) & 0x7f800000u;
}

// A wave's part of a 32-key tile as it lies in the cache
template <int NG>
struct KeyTile {
  typename Words<NG>::type k[2], v[2];   // K codes of the lane's key in either product; V codes of tokens 8p..8p+3, 8p+4..8p+7
  uint32_t k_scale[2];
  au32x2 v_scale;                        // of tokens 8p..8p+7, the group of the lane's V columns
};

// Sequence, key/value head and row tile of a workgroup, and the keys its rows see
struct RowTile {
  int b, h, q0, nq, keys, first, rows, tiles;
  bool cut;     // the GPU's lengths are larger than the host was told
};
__device__ __forceinline__ RowTile row_tile(const CacheAttnArgs& a, int unit) {
  RowTile t;
  const int rt = unit % a.row_tiles, bh = unit / a.row_tiles;
  t.h = bh % a.shape.n_kv_heads;
  t.b = bh / a.shape.n_kv_heads;
  const int64_t c0 = a.cu[t.b], c1 = a.cu[t.b + 1], n = a.n_keys[t.b];
  const int64_t q0 = c0 < 0 ? 0 : c0 > a.n_queries ? a.n_queries : c0;
  int64_t q1 = c1 < q0 ? q0 : c1 > a.n_queries ? a.n_queries : c1;
  t.cut = q0 != c0 || q1 != c1 || q1 - q0 > a.max_queries;
  if (q1 - q0 > a.max_queries) q1 = q0 + a.max_queries;
  const int64_t room = (int64_t)a.table_width * a.shape.page_tokens, most = a.max_keys < room ? a.max_keys : room;
  t.keys = (int)(n < 0 ? 0 : n > most ? most : n);
  t.cut |= t.keys != n;
  t.q0 = (int)q0;
  t.nq = (int)(q1 - q0);
  t.rows = t.nq * a.group;
  t.first = rt * 16;
  int seen = t.keys;
  if (a.causal) {
    const int last = (t.first + 15 < t.rows ? t.first + 15 : t.rows - 1) / a.group;
    seen = t.keys - t.nq + last + 1;
  }
  t.tiles = t.first < t.rows && seen > 0 ? (seen + 31) >> 5 : 0;
  return t;
}

template <int NG>
__global__ __launch_bounds__(256) void attend_rows_kernel(CacheAttnArgs a) {
  constexpr int D = 32 * NG, WAVES = 4, PITCH = D + 4;
  typedef typename Words<NG>::type words;
  __shared__ __align__(16) float state_o[WAVES][16][PITCH];
  __shared__ float state_m[WAVES][16], state_l[WAVES][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l15 = lane & 15, p = lane >> 4;
  const int split = blockIdx.x % a.splits;
  const RowTile t = row_tile(a, blockIdx.x / a.splits);
  if (t.cut && a.err && tid == 0) atomicOr(a.err, 1);
  if (t.first >= t.rows) return;                                    // (whole workgroups, before any barrier)
  if (split > 0 && split * a.chunk >= t.tiles) return;

  // ---- this wave's tiles
  int t0 = split * a.chunk, t1 = t0 + a.chunk < t.tiles ? t0 + a.chunk : t.tiles;
  {
    const int per = (t1 - t0 + WAVES - 1) / WAVES;
    t0 += wave * per;
    t1 = t0 + per < t1 ? t0 + per : t1;
  }
  // ---- the lane's row
  const int r = t.first + l15, rr = r < t.rows ? r : t.rows - 1, query = rr / a.group, sub = rr - query * a.group;
  const int64_t head = t.h * a.group + sub;
  int seen = a.causal ? t.keys - t.nq + query + 1 : t.keys;         // keys the row sees
  if (r >= t.rows || seen < 0) seen = 0;
  int seen_by_all = a.causal ? t.keys - t.nq + t.first / a.group + 1 : t.keys;   // ... and every row of the tile
  abf16x8 qf[NG];
  {
    const bf16_t* qp = a.q + (t.q0 + query) * a.q_row + head * D + 8 * p;
#pragma unroll
    for (int g = 0; g < NG; ++g) qf[g] = *reinterpret_cast<const abf16x8*>(qp + 32 * g);
  }
  af32x4 o[2 * NG];
#pragma unroll
  for (int i = 0; i < 2 * NG; ++i) o[i] = af32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, sum = 0.f;

  // ---- addresses.  Pages are found 64 at a time: lane i holds the number of page first_page + i.
  const int P = a.shape.page_tokens, page_tiles = P >> 5;
  const int key = 8 * (l15 >> 2) + (l15 & 3);
  const int k_off = key * (D / 2) + p * (4 * NG);
  const int v_off = P * (D / 2) + p * (4 * D) + l15 * (4 * NG);
  const int ks_off = P * D + key * NG, vs_off = P * (D + NG) + p * (8 * NG) + (l15 * NG >> 4) * 8;
  const int32_t* table = a.table + (int64_t)t.b * a.table_width;
  int page = t0 / page_tiles, in_page = t0 - page * page_tiles, first_page = page;
  const int last_page = t1 > t0 ? (t1 - 1) / page_tiles : page;
  auto load_pages = [&]() {
    const int x = first_page + lane;
    return x <= last_page ? table[x] : 0;
  };
  int pages = t1 > t0 ? load_pages() : 0;
  bool bad = false;
  KeyTile<NG> next;
  bool next_bad = false;
  auto load = [&]() {            // the tile at (page, in_page), and the step to the one behind it
    if (page - first_page >= 64) {
      first_page = page;
      pages = load_pages();
    }
    const int id = __builtin_amdgcn_readlane(pages, page - first_page);
    next_bad = id < 0 || id >= a.shape.n_pages;
    bad |= next_bad;
    const unsigned char* block = a.pool + ((int64_t)(next_bad ? 0 : id) * a.shape.n_kv_heads + t.h) * a.shape.head_bytes;
    const unsigned char* kp = block + in_page * (16 * D) + k_off;
    next.k[0] = *reinterpret_cast<const words*>(kp);
    next.k[1] = *reinterpret_cast<const words*>(kp + 2 * D);
    const unsigned char* vp = block + in_page * (16 * D) + v_off;
    next.v[0] = *reinterpret_cast<const words*>(vp);
    next.v[1] = *reinterpret_cast<const words*>(vp + 2 * D);
    const unsigned char* sp = block + in_page * (32 * NG) + ks_off;
    if constexpr (NG == 4) {
      next.k_scale[0] = *reinterpret_cast<const uint32_t*>(sp);
      next.k_scale[1] = *reinterpret_cast<const uint32_t*>(sp + 4 * NG);
    } else {
      next.k_scale[0] = *reinterpret_cast<const uint16_t*>(sp);
      next.k_scale[1] = *reinterpret_cast<const uint16_t*>(sp + 4 * NG);
    }
    next.v_scale = *reinterpret_cast<const au32x2*>(block + in_page * (32 * NG) + vs_off);
    if (++in_page == page_tiles) {
      in_page = 0;
      ++page;
    }
  };
  if (t0 < t1) load();
  for (int tile = t0; tile < t1; ++tile) {
    KeyTile<NG> c = next;
    const bool skip = next_bad;
    if (tile + 1 < t1) load();
    if (skip) continue;
    const int kv = tile * 32;
    af32x4 s[2] = {};
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      auto group = [&](auto G) {
        constexpr int g = decltype(G)::value;
        const uint32_t sc = scale_of<g>(c.k_scale[u]);
        au32x4 w;
        w[0] = widen2<0>(c.k[u][g], sc);
        w[1] = widen2<1>(c.k[u][g], sc);
        w[2] = widen2<2>(c.k[u][g], sc);
        w[3] = widen2<3>(c.k[u][g], sc);
        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(abf16x8, w), qf[g], s[u], 0, 0, 0);
      };
      group(std::integral_constant<int, 0>());
      group(std::integral_constant<int, 1>());
      if constexpr (NG == 4) {
        group(std::integral_constant<int, 2>());
        group(std::integral_constant<int, 3>());
      }
    }
    // ---- softmax in the log2 domain.  A score that the row does not see becomes -inf by selection: what lies behind
    // a sequence's end may be anything, NaN included, and so the V scales there become zero.
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s[i >> 2][i & 3] * a.scale_log2;
    if (kv + 32 > seen_by_all) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (kv + 8 * p + i >= seen) x[i] = -INFINITY;
      const int held = t.keys - (kv + 8 * p);       // tokens of the lane's eight that exist
      if (held < 8) {
        c.v_scale[0] = held >= 4 ? c.v_scale[0] : held > 0 ? c.v_scale[0] & ((1u << (8 * held)) - 1) : 0;
        c.v_scale[1] = held > 4 ? c.v_scale[1] & ((1u << (8 * (held - 4))) - 1) : 0;
      }
    }
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    constexpr float SLACK = 8.f;   // the running maximum moves only when a score exceeds it by more: probabilities stay below 2^8
    if (__any(top > m + SLACK || (m == -INFINITY && top > m))) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float moved = top > m + SLACK || m == -INFINITY ? fmaxf(top, m) : m;
      const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - moved);
      m = moved;
      sum *= alpha;
#pragma unroll
      for (int i = 0; i < 2 * NG; ++i) o[i] *= alpha;
    }
    const float shift = m == -INFINITY ? 0.f : m;
    au32x4 pw;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p0 = __builtin_amdgcn_exp2f(x[2 * i] - shift), p1 = __builtin_amdgcn_exp2f(x[2 * i + 1] - shift);
      sum += p0 + p1;
      pw[i] = pack2_k(p0, p1);
    }
    const abf16x8 pf = __builtin_bit_cast(abf16x8, pw);
    // ---- O^T += V^T P^T: columns 2b and 2b+1 of the lane's 2 NG, tokens 8p .. 8p+7
    uint32_t vs[8];
    vs[0] = scale_of<0>(c.v_scale[0]); vs[1] = scale_of<1>(c.v_scale[0]); vs[2] = scale_of<2>(c.v_scale[0]); vs[3] = scale_of<3>(c.v_scale[0]);
    vs[4] = scale_of<0>(c.v_scale[1]); vs[5] = scale_of<1>(c.v_scale[1]); vs[6] = scale_of<2>(c.v_scale[1]); vs[7] = scale_of<3>(c.v_scale[1]);
    auto column = [&](auto B) {
      constexpr int b = decltype(B)::value;
      au32x4 lo, hi;
#pragma unroll
      for (int i = 0; i < 4; ++i) {       // tokens 2i, 2i+1
        uint32_t e, f;
        if constexpr (NG == 4) {
          e = widen2<b>(c.v[i >> 1][(2 * i) & 3], vs[2 * i]);
          f = widen2<b>(c.v[i >> 1][(2 * i + 1) & 3], vs[2 * i + 1]);
        } else {
          e = widen2<b>(c.v[i >> 1][i & 1], vs[2 * i]);
          f = widen2<b + 2>(c.v[i >> 1][i & 1], vs[2 * i + 1]);
        }
        lo[i] = __builtin_amdgcn_perm(f, e, 0x05040100u);
        hi[i] = __builtin_amdgcn_perm(f, e, 0x07060302u);
      }
      o[2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(abf16x8, lo), pf, o[2 * b], 0, 0, 0);
      o[2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(abf16x8, hi), pf, o[2 * b + 1], 0, 0, 0);
    };
    column(std::integral_constant<int, 0>());
    column(std::integral_constant<int, 1>());
    if constexpr (NG == 4) {
      column(std::integral_constant<int, 2>());
      column(std::integral_constant<int, 3>());
    }
  }
  if (bad && a.err && lane == 0) atomicOr(a.err, 1);

  // ---- the waves' states, joined in their order.  o[i][e] is value (4p + e) 2 NG + i of the row
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < 2 * NG; i += 4)
      *reinterpret_cast<af32x4*>(&state_o[wave][l15][(4 * p + e) * 2 * NG + i]) = af32x4{o[i][e], o[i + 1][e], o[i + 2][e], o[i + 3][e]};
  if (p == 0) {
    state_m[wave][l15] = m;
    state_l[wave][l15] = sum;
  }
  __syncthreads();
  const int jr = tid >> 4, jc = (tid & 15) * (2 * NG);
  if (t.first + jr >= t.rows) return;
  float mm = state_m[0][jr];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) mm = fmaxf(mm, state_m[w][jr]);
  float ll = 0.f, acc[2 * NG] = {};
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const float mw = state_m[w][jr], f = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - mm);
    ll += f * state_l[w][jr];
#pragma unroll
    for (int i = 0; i < 2 * NG; ++i) acc[i] += f * state_o[w][jr][jc + i];
  }
  const int jq = (t.first + jr) / a.group;
  const int64_t token = t.q0 + jq, jh = t.h * a.group + (t.first + jr - jq * a.group);
  if (a.splits > 1) {
    const int64_t at = (split * a.n_queries + token) * a.n_heads + jh;
    af32x4* to = reinterpret_cast<af32x4*>(a.part_o + at * D + jc);
#pragma unroll
    for (int i = 0; i < 2 * NG; i += 4) to[i / 4] = af32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
    if ((tid & 15) == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(mm, ll);
  } else {
    const float inv = ll > 0.f ? 1.f / ll : 0.f;
    typename Words<NG>::type w;
#pragma unroll
    for (int i = 0; i < NG; ++i) w[i] = pack2_k(acc[2 * i] * inv, acc[2 * i + 1] * inv);
    *reinterpret_cast<typename Words<NG>::type*>(a.out + token * a.out_row + jh * D + jc) = w;
  }
}

// The splits of a row tile, joined in their order: 16 lanes a row, as the workgroups above end
template <int NG>
__global__ __launch_bounds__(256) void join_splits_kernel(CacheAttnArgs a) {
  constexpr int D = 32 * NG;
  const RowTile t = row_tile(a, blockIdx.x);
  const int jr = threadIdx.x >> 4, jc = (threadIdx.x & 15) * (2 * NG);
  if (t.first + jr >= t.rows) return;
  const int used = t.tiles > 0 ? (t.tiles + a.chunk - 1) / a.chunk : 1;
  const int jq = (t.first + jr) / a.group;
  const int64_t token = t.q0 + jq, jh = t.h * a.group + (t.first + jr - jq * a.group);
  const int64_t at = token * a.n_heads + jh, step = a.n_queries * a.n_heads;
  float mm = -INFINITY;
  for (int s = 0; s < used; ++s) mm = fmaxf(mm, a.part_ml[(at + s * step) * 2]);
  float ll = 0.f, acc[2 * NG] = {};
  for (int s = 0; s < used; ++s) {
    const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (at + s * step) * 2);
    const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - mm);
    ll += f * ml.y;
    const af32x4* from = reinterpret_cast<const af32x4*>(a.part_o + (at + s * step) * D + jc);
#pragma unroll
    for (int i = 0; i < 2 * NG; ++i) acc[i] += f * from[i / 4][i & 3];
  }
  const float inv = ll > 0.f ? 1.f / ll : 0.f;
  typename Words<NG>::type w;
#pragma unroll
  for (int i = 0; i < NG; ++i) w[i] = pack2_k(acc[2 * i] * inv, acc[2 * i + 1] * inv);
  *reinterpret_cast<typename Words<NG>::type*>(a.out + token * a.out_row + jh * D + jc) = w;
}

size_t plan_cache_attention(CacheAttnArgs& a) {
  const int64_t rows = (int64_t)a.max_queries * a.group;
  a.row_tiles = (int32_t)((rows + 15) / 16);
  const int64_t tiles = std::max<int64_t>(1, (a.max_keys + 31) / 32), base = std::max<int64_t>(1, (int64_t)a.n_seqs * a.shape.n_kv_heads * a.row_tiles);
  // four workgroups of four waves a compute unit, two tiles a wave at least
  const int64_t want = (1024 + base - 1) / base;
  a.chunk = (int32_t)std::max<int64_t>(8, (tiles + want - 1) / want);
  a.splits = (int32_t)((tiles + a.chunk - 1) / a.chunk);
  if (a.splits <= 1) return 0;
  const size_t parts = (size_t)a.splits * (size_t)a.n_queries * (size_t)a.n_heads;
  return parts * (size_t)(a.shape.head_dim + 2) * 4;
}

cs_status launch_cache_attention(const CacheAttnArgs& a, hipStream_t stream) {
  const int64_t units = (int64_t)a.n_seqs * a.shape.n_kv_heads * a.row_tiles, blocks = units * a.splits;
  if (blocks > 0x7fffffff) return fail(CS_ERR_UNSUPPORTED, "cs_attention_cache: too many rows");
  if (a.shape.head_dim == 128) hipLaunchKernelGGL((attend_rows_kernel<4>), dim3((unsigned)blocks), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((attend_rows_kernel<2>), dim3((unsigned)blocks), dim3(256), 0, stream, a);
  CS_HIP(hipGetLastError());
  if (a.splits > 1) {
    if (a.shape.head_dim == 128) hipLaunchKernelGGL((join_splits_kernel<4>), dim3((unsigned)units), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((join_splits_kernel<2>), dim3((unsigned)units), dim3(256), 0, stream, a);
    CS_HIP(hipGetLastError());
  }
  return CS_OK;
}

}  // namespace cs
