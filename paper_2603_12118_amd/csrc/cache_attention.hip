// Attention over the 4-bit cache.
//
// Rows: the queries of a sequence times the heads that share a key/value head, query by query.  A wave takes 16 rows and
// walks tiles of 32 keys.  S^T = K Q^T with v_mfma_f32_16x16x32_bf16, twice 16 keys: lane l then holds row l % 16 and keys
// 8p .. 8p+7 of the tile, p = l / 16 (key m of product u is token 8 (m / 4) + 4 u + m % 4 of the tile), which after the
// exponential is the B operand of O^T = V^T P^T as it stands.  A code times its power of two is exact in bf16, and the
// conversion instruction does it two codes at a time, so the cache is widened in registers between its load and the matrix
// instruction and what crosses the memory bus is 4.25 bits a value.
//
// Probabilities are rounded to bf16, the type the second product takes; their sum is that of the unrounded ones, in fp32 like scores,
// maxima, accumulators and parts.  The roundings are to nearest and independent, and cost 0.0018 .. 0.0023 of the result's norm where the
// rounding of the result alone costs 0.0016 .. 0.0017; probabilities in two bf16 parts would double the second product.
#include "cache.h"

#include <algorithm>
#include <type_traits>

namespace cs {

typedef __bf16 abf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 abf16x2 __attribute__((ext_vector_type(2)));
typedef float af32x2 __attribute__((ext_vector_type(2)));
typedef float af32x4 __attribute__((ext_vector_type(4)));
typedef float af32x16 __attribute__((ext_vector_type(16)));
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

// eight values of a query, their signs turned where `sign` has the sign bits of a pair
__device__ __forceinline__ abf16x8 load_q(const bf16_t* p, uint32_t sign) {
  au32x4 w = *reinterpret_cast<const au32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] ^= sign;
  return __builtin_bit_cast(abf16x8, w);
}

// A wave's part of a 32-key tile as it lies in the cache
template <int NG>
struct KeyTile {
  typename Words<NG>::type k[2], v[2];   // K codes of the lane's key in either product; V codes of tokens 8p..8p+3, 8p+4..8p+7
  uint32_t k_scale[2];
  au32x2 v_scale;                        // of tokens 8p..8p+7, the group of the lane's V columns
};

// ---- who does what.  The lengths are on the GPU only, so the workgroups share the work out themselves: up to 64 sequences, every wave
// reads all lengths, and from them come the tiles a workgroup takes (`chunk`: all work over `target` workgroups), the number of
// shares of each sequence's keys, and the sequence a workgroup belongs to.  A batch of long and short sequences then fills
// the chip as evenly as one of equal ones (64 sequences of 160 .. 16384 keys: 29 us, with shares by the longest 62).  More sequences are
// shared out by a launch of one workgroup before, which is 2 us slower than reading all lengths in every wave for 128 sequences of 2000 keys
// (35 us), and 512 ragged ones of up to 4000 take 67 us instead of 79.  Where no sequence can be shared out, a workgroup is a block of
// rows and reads the lengths of its own: 1024 sequences of 500 keys 58 us instead of 110, one 7.1 instead of 7.4.
struct Sequence {
  int q0, nq, keys, units, tiles;   // units: blocks of rows of all key/value heads
  bool cut;                         // a length on the GPU is not what the host was told
};
__device__ __forceinline__ Sequence sequence(const CacheAttnArgs& a, int b, int rows) {
  Sequence t = {};
  if (b >= a.n_seqs) return t;
  const int64_t c0 = a.cu[b], c1 = a.cu[b + 1], n = a.n_keys[b];
  const int64_t q0 = c0 < 0 ? 0 : c0 > a.n_queries ? a.n_queries : c0;
  int64_t q1 = c1 < q0 ? q0 : c1 > a.n_queries ? a.n_queries : c1;
  t.cut = q0 != c0 || q1 != c1 || q1 - q0 > a.max_queries;
  if (q1 - q0 > a.max_queries) q1 = q0 + a.max_queries;
  const int64_t room = (int64_t)a.table_width * a.shape.page_tokens, most = a.max_keys < room ? a.max_keys : room;
  t.keys = (int)(n < 0 ? 0 : n > most ? most : n);
  t.cut |= t.keys != n;
  t.q0 = (int)q0;
  t.nq = (int)(q1 - q0);
  const int64_t r = (int64_t)t.nq * a.group;
  t.units = r > a.more_than && r <= a.at_most ? (int)((r + rows - 1) / rows) * a.shape.n_kv_heads : 0;
  t.tiles = (t.keys + 31) >> 5;
  return t;
}
struct Share {
  Sequence seq;
  int b, chunk, shares, first;   // first: the sequence's first workgroup
};
// tiles a workgroup takes (more than work / target, so that the workgroups are fewer than target and one a unit)
__device__ __forceinline__ int chunk_of(const CacheAttnArgs& a, float work) {
  const float per = work / (float)a.target;
  const int chunk = per > 3e7f ? 1 << 25 : (int)per + 1;
  return chunk < a.least ? a.least : (chunk + 1) & ~1;
}
__device__ __forceinline__ int shares_of(const Sequence& t, int chunk) { return t.tiles > chunk ? (t.tiles + chunk - 1) / chunk : 1; }

// The last sequence whose entry of share_of (0: first workgroup, 3: first unit) is not behind `id`, by steps of 64
__device__ __forceinline__ int find_sequence(const CacheAttnArgs& a, int entry, int id) {
  int step = 1, b = 0;
  while ((int64_t)step * 64 < a.n_seqs) step *= 64;
  for (; step; step >>= 6) {
    const int64_t at = b + (int64_t)(threadIdx.x & 63) * step;
    const uint64_t upto = __ballot(at < a.n_seqs && a.share_of[4 * at + entry] <= id);
    b += (__builtin_popcountll(upto) - 1) * step;
  }
  return b;
}
// The share of workgroup `id`; false where there is none.  Whole waves.
__device__ __forceinline__ bool find_share(const CacheAttnArgs& a, int rows, int id, Share& s) {
  const int lane = threadIdx.x & 63, n = a.n_seqs;
  bool found;
  if (!a.join || a.planned) {
    if (!a.join) {
      const int per = a.shape.n_kv_heads * a.row_blocks;
      s.b = id / per;
      s.first = s.b * per;
      s.shares = 1;
      s.chunk = 1 << 25;
    } else {
      s.b = find_sequence(a, 0, id);
      const int4 share = *reinterpret_cast<const int4*>(a.share_of + 4 * (int64_t)s.b);
      s.first = share.x;
      s.shares = share.y;
      s.chunk = share.z;
    }
    s.seq = sequence(a, s.b, rows);
    found = id - s.first < s.seq.units * s.shares;
    if (!a.join && s.seq.cut && id == s.first && a.err && threadIdx.x == 0) atomicOr(a.err, 1);
  } else {
    const Sequence t = sequence(a, lane, rows);
    float work = (float)t.units * (float)t.tiles;
    const uint64_t cut = __ballot(t.cut);
    if (id == 0 && cut && a.err && threadIdx.x == 0) atomicOr(a.err, 1);
    for (int m = 1; m < n; m <<= 1) work += __shfl_xor(work, m);
    s.chunk = chunk_of(a, __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(work))));
    const int shares = shares_of(t, s.chunk), own = t.units * shares;
    int upto = own;
    for (int m = 1; m < n; m <<= 1) {
      const int x = __shfl_up(upto, m);
      upto += lane >= m ? x : 0;
    }
    const uint64_t hit = __ballot(lane < n && upto > id);
    found = hit != 0;
    s.b = found ? __builtin_ctzll(hit) : 0;
    s.shares = __builtin_amdgcn_readlane(shares, s.b);
    s.first = __builtin_amdgcn_readlane(upto - own, s.b);
    s.seq.q0 = __builtin_amdgcn_readlane(t.q0, s.b);
    s.seq.nq = __builtin_amdgcn_readlane(t.nq, s.b);
    s.seq.keys = __builtin_amdgcn_readlane(t.keys, s.b);
    s.seq.units = __builtin_amdgcn_readlane(t.units, s.b);
    s.seq.tiles = __builtin_amdgcn_readlane(t.tiles, s.b);
    if (found && id == s.first && threadIdx.x == 0) *reinterpret_cast<int4*>(a.share_of + 4 * s.b) = make_int4(s.first, s.shares, s.chunk, 0);
  }
  // (the same in every lane: into scalar registers)
  for (int* x : {&s.b, &s.first, &s.shares, &s.chunk, &s.seq.q0, &s.seq.nq, &s.seq.keys, &s.seq.units, &s.seq.tiles}) *x = __builtin_amdgcn_readfirstlane(*x);
  return __builtin_amdgcn_readfirstlane(found);
}

// The shares of more than 64 sequences, or of few that differ much, 1024 at a time, one workgroup.  Bound by latency (lengths, twice, and the sums between).
__global__ __launch_bounds__(1024) void share_out_kernel(CacheAttnArgs a) {
  __shared__ float work_of[16];
  __shared__ int upto_of[16], units_of[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  float work = 0.f;
  bool cut = false;
  for (int64_t b = tid; b < a.n_seqs; b += 1024) {
    const Sequence t = sequence(a, (int)b, a.rows);
    work += (float)t.units * (float)t.tiles;
    cut |= t.cut;
  }
  if (cut && a.err) atomicOr(a.err, 1);
  for (int m = 1; m < 64; m <<= 1) work += __shfl_xor(work, m);
  if (lane == 0) work_of[wave] = work;
  __syncthreads();
  work = 0.f;
  for (int w = 0; w < 16; ++w) work += work_of[w];
  const int chunk = chunk_of(a, work);
  int before = 0, units_before = 0;
  for (int64_t b0 = 0; b0 < a.n_seqs; b0 += 1024) {
    const int64_t b = b0 + tid;
    Sequence t = {};
    if (b < a.n_seqs) t = sequence(a, (int)b, a.rows);
    const int shares = shares_of(t, chunk), own = t.units * shares;
    int upto = own, units = t.units;
    for (int m = 1; m < 64; m <<= 1) {
      const int x = __shfl_up(upto, m), y = __shfl_up(units, m);
      upto += lane >= m ? x : 0;
      units += lane >= m ? y : 0;
    }
    if (lane == 63) {
      upto_of[wave] = upto;
      units_of[wave] = units;
    }
    __syncthreads();
    int all = 0, all_units = 0;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) {
        upto += upto_of[w];
        units += units_of[w];
      }
      all += upto_of[w];
      all_units += units_of[w];
    }
    if (b < a.n_seqs) *reinterpret_cast<int4*>(a.share_of + 4 * b) = make_int4(before + upto - own, shares, chunk, units_before + units - t.units);
    before += all;
    units_before += all_units;
    __syncthreads();
  }
}

// The block of rows that `unit` of a sequence is: the last rows, which see the most keys, first
struct RowBlock {
  int h, first, rows, seen;   // rows first .. of `rows`; keys its last row sees
};
__device__ __forceinline__ RowBlock row_block(const CacheAttnArgs& a, const Sequence& q, int unit, int rows) {
  RowBlock r;
  const int rb = unit / a.shape.n_kv_heads;
  r.h = unit - rb * a.shape.n_kv_heads;
  r.rows = q.nq * a.group;
  r.first = (q.units / a.shape.n_kv_heads - 1 - rb) * rows;
  const int last = (r.first + rows < r.rows ? r.first + rows : r.rows) - 1;
  r.seen = a.causal ? q.keys - q.nq + last / a.group + 1 : q.keys;
  r.seen = r.seen < 0 ? 0 : r.seen;
  return r;
}

// The running maximum moves only when a score exceeds it by more than SLACK, in the log2 domain: probabilities stay below 2^8, and the
// accumulators are rescaled on the first tile and on such a jump instead of on nearly every tile.
constexpr float SLACK = 8.f;

// values jc .. jc + 2 NG - 1 of row r, normalised
template <int NG>
__device__ __forceinline__ void store_row(const CacheAttnArgs& a, int q0, int h, int r, int jc, const float (&acc)[2 * NG], float weight) {
  const float inv = weight > 0.f ? 1.f / weight : weight == 0.f ? 0.f : weight;     // no key: zeros; NaN stays
  typename Words<NG>::type w;
#pragma unroll
  for (int i = 0; i < NG; ++i) w[i] = pack2_k(acc[2 * i] * inv, acc[2 * i + 1] * inv);
  const int query = r / a.group;
  const int64_t head = h * a.group + (r - query * a.group);
  *reinterpret_cast<typename Words<NG>::type*>(a.out + (q0 + query) * a.out_row + head * (32 * NG) + jc) = w;
}

// ---- few rows: 16 RT of them, a wave's keys its own.  The softmax keeps a running maximum and sum (fp32) a row and wave, joined at the end.
// Bound by the memory once there are enough keys: 64 sequences of 8192 (285 MB) 57 us with their join, 5.0 TB/s.  Fewer are bound by the way to
// a wave's first tile (arguments, lengths, page table, tile: four reads, one behind the other) and by the join: 64 of 160 .. 16384 keys
// (119 MB) 30 + 5.4 us, one of 131072 (71 MB) 18.2 + 7.3, one of 2048 5.5 + 5.0, six of up to 4097 with 5 queries 12.9 + 4.5.  While a wave
// works on a tile its next one is on its way: 17.8 MB over the chip, 2.8 us at 6.3 TB/s; two ahead do not fit the registers of four waves a
// SIMD.  The loop is some 200 vector and 16 matrix instructions a tile; an eighth fewer of the former changed nothing.
template <int NG, int RT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(RT == 1 ? 4 : 2))) void attend_rows_kernel(CacheAttnArgs a) {
  constexpr int D = 32 * NG, WAVES = 4, PITCH = D + 4, ROWS = 16 * RT;
  typedef typename Words<NG>::type words;
  __shared__ __align__(16) float state_o[WAVES][16][PITCH];
  __shared__ float state_m[WAVES][16], state_l[WAVES][16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l15 = lane & 15, p = lane >> 4;
  Share t;
  if (!find_share(a, ROWS, blockIdx.x, t)) return;           // (whole workgroups, before any barrier)
  const int rank = blockIdx.x - t.first, share = rank / t.seq.units, unit = rank - share * t.seq.units;
  const RowBlock rb = row_block(a, t.seq, unit, ROWS);

  // ---- this wave's tiles
  int t0 = share * t.chunk, t1 = (rb.seen + 31) >> 5;
  {
    if (share > 0 && t0 >= t1) return;
    t1 = t0 + t.chunk < t1 ? t0 + t.chunk : t1;
    const int per = (t1 - t0 + WAVES - 1) / WAVES;
    t0 += wave * per;
    t1 = t0 + per < t1 ? t0 + per : t1;
  }
  // ---- the lane's rows
  const int keys = t.seq.keys, nq = t.seq.nq;
  int seen[RT];                                                       // keys a row sees
  abf16x8 qf[RT][NG];
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    const int r = rb.first + 16 * x + l15, rr = r < rb.rows ? r : rb.rows - 1, query = rr / a.group;
    const int64_t head = rb.h * a.group + (rr - query * a.group);
    seen[x] = a.causal ? keys - nq + query + 1 : keys;
    if (r >= rb.rows) seen[x] = 0;
    const bf16_t* qp = a.q + (t.seq.q0 + query) * a.q_row + head * D + 8 * p;
#pragma unroll
    for (int g = 0; g < NG; ++g) qf[x][g] = load_q(qp + 32 * g, a.q_sign);
  }
  const int seen_by_all = a.causal ? keys - nq + rb.first / a.group + 1 : keys;
  af32x4 o[RT][2 * NG];
  float m[RT], shift[RT], sum[RT];       // the running maximum of the scores, the same times the scale, the weight
  const float slack = SLACK / a.scale_log2;
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    m[x] = -INFINITY;
    shift[x] = sum[x] = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * NG; ++i) o[x][i] = af32x4{0.f, 0.f, 0.f, 0.f};
  }

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
    const unsigned char* block = a.pool + ((int64_t)(next_bad ? 0 : id) * a.shape.n_kv_heads + rb.h) * a.shape.head_bytes;
    // (past the caches, right for codes that one workgroup reads: 64 sequences of 8192 keys 63.9 -> 57.4 us, ragged ones 38.6 -> 36.3.  Where several
    // blocks of rows read the same codes that costs nothing to 7 %: prompts of 500 and 1000 tokens 12.0 and 24.6 us either way, 8 x 8 drafts
    // 21.9 -> 23.5, 32 x 8 behind 8192 keys 65.7 -> 67.5; one token of 2048 keys 10.0 -> 10.4.)
    const unsigned char* kp = block + in_page * (16 * D) + k_off;
    next.k[0] = __builtin_nontemporal_load(reinterpret_cast<const words*>(kp));
    next.k[1] = __builtin_nontemporal_load(reinterpret_cast<const words*>(kp + 2 * D));
    const unsigned char* vp = block + in_page * (16 * D) + v_off;
    next.v[0] = __builtin_nontemporal_load(reinterpret_cast<const words*>(vp));
    next.v[1] = __builtin_nontemporal_load(reinterpret_cast<const words*>(vp + 2 * D));
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
    af32x4 s[RT][2] = {};
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
#pragma unroll
        for (int x = 0; x < RT; ++x) s[x][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(abf16x8, w), qf[x][g], s[x][u], 0, 0, 0);
      };
      group(std::integral_constant<int, 0>());
      group(std::integral_constant<int, 1>());
      if constexpr (NG == 4) {
        group(std::integral_constant<int, 2>());
        group(std::integral_constant<int, 3>());
      }
    }
    const bool masked = kv + 32 > seen_by_all;
    if (masked) {
      const int held = keys - (kv + 8 * p);           // tokens of the lane's eight that exist
      if (held < 8) {
        c.v_scale[0] = held >= 4 ? c.v_scale[0] : held > 0 ? c.v_scale[0] & ((1u << (8 * held)) - 1) : 0;
        c.v_scale[1] = held > 4 ? c.v_scale[1] & ((1u << (8 * (held - 4))) - 1) : 0;
      }
    }
    // ---- softmax, exp2 of scaled differences.  A score that the row does not see becomes -inf by selection: what lies behind
    // a sequence's end may be anything, NaN included, and so the V scales there are zero.
    abf16x8 pf[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = s[r][i >> 2][i & 3];
      if (masked) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (kv + 8 * p + i >= seen[r]) x[i] = -INFINITY;
      }
      float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      if (__any(top > m[r] + slack)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float moved = top > m[r] + slack || m[r] == -INFINITY ? fmaxf(top, m[r]) : m[r];
        const float alpha = m[r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(shift[r] - moved * a.scale_log2);
        m[r] = moved;
        shift[r] = m[r] == -INFINITY ? 0.f : m[r] * a.scale_log2;
        sum[r] *= alpha;
#pragma unroll
        for (int i = 0; i < 2 * NG; ++i) o[r][i] *= alpha;
      }
      au32x4 pw;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(x[2 * i], a.scale_log2, -shift[r]));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(x[2 * i + 1], a.scale_log2, -shift[r]));
        sum[r] += p0 + p1;
        pw[i] = pack2_k(p0, p1);
      }
      pf[r] = __builtin_bit_cast(abf16x8, pw);
    }
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
#pragma unroll
      for (int x = 0; x < RT; ++x) {
        o[x][2 * b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(abf16x8, lo), pf[x], o[x][2 * b], 0, 0, 0);
        o[x][2 * b + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(abf16x8, hi), pf[x], o[x][2 * b + 1], 0, 0, 0);
      }
    };
    column(std::integral_constant<int, 0>());
    column(std::integral_constant<int, 1>());
    if constexpr (NG == 4) {
      column(std::integral_constant<int, 2>());
      column(std::integral_constant<int, 3>());
    }
  }
  if (bad && a.err && lane == 0) atomicOr(a.err, 1);

  // ---- the waves' states, joined in their order, 16 rows at a time.  o[x][i][e] is value (4p + e) 2 NG + i of the row
  const int jr = tid >> 4, jc = (tid & 15) * (2 * NG);
#pragma unroll
  for (int x = 0; x < RT; ++x) {
    sum[x] += __shfl_xor(sum[x], 16);
    sum[x] += __shfl_xor(sum[x], 32);
    if (x > 0) __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < 2 * NG; i += 4)
        *reinterpret_cast<af32x4*>(&state_o[wave][l15][(4 * p + e) * 2 * NG + i]) = af32x4{o[x][i][e], o[x][i + 1][e], o[x][i + 2][e], o[x][i + 3][e]};
    if (p == 0) {
      state_m[wave][l15] = m[x] == -INFINITY ? m[x] : shift[x];
      state_l[wave][l15] = sum[x];
    }
    __syncthreads();
    const int r = rb.first + 16 * x + jr;
    if (r >= rb.rows) continue;
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
    if (t.shares > 1) {
      const int64_t at = (int64_t)blockIdx.x * ROWS + 16 * x + jr;
      af32x4* to = reinterpret_cast<af32x4*>(a.part_o + at * D + jc);
#pragma unroll
      for (int i = 0; i < 2 * NG; i += 4) to[i / 4] = af32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
      if ((tid & 15) == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(mm, ll);
    } else {
      store_row<NG>(a, t.seq.q0, rb.h, r, jc, acc, ll);
    }
  }
}

// ---- many rows: 128 of them, 32 a wave, the waves' keys the same.  Tiles of 64 keys are widened once, into LDS, by the whole
// workgroup (a thread: a quarter of a token of K, a word of four tokens of V): K as it is, V transposed, so that both products read
// 16 bytes a lane.  S^T = K Q^T and O^T = V^T P^T with
// v_mfma_f32_32x32x16_bf16: lane l has row l % 32 throughout, and what the exponential leaves is the second product's operand.
// Bound by the SIMDs, whose matrix and vector instructions share less than half of their time (two waves of 16 products and 128 FMAs: alternating
// 797 ns, interleaved 645, products alone 495, FMAs alone 473), and by the power: 2048 queries behind 14336 keys, 28 heads, 451 GFLOP,
// 473 .. 509 us on different cards, 890 .. 950 TFLOP/s (zeros for data: 450), matrix pipe busy 40 % of the cycles, vector unit 45 %.  Within
// 3 % of that: 256 rows a workgroup, K widened by every wave into registers without LDS, fragments asked for earlier, exponentials between
// the products, tiles two ahead.  Three waves a SIMD spill (569 us), 64 rows a wave move accumulators about (592).
// A column of V^T (value 2 NG j + d of a head, j = the word of a token that holds it) is row 16 d + j of the tile: the 16 lanes
// that write one d then write neighbouring rows, and a lane's results come out 2 NG values at a time.
template <int NG>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void attend_block_kernel(CacheAttnArgs a) {
  constexpr int D = 32 * NG, ROWS = 128, KS = D / 16;
  constexpr int KSTR = D * 2 + 16, VSTR = 64 * 2 + 16;      // bytes between rows of the tiles
  typedef typename Words<NG>::type words;
  __shared__ __align__(16) unsigned char k_lds[64 * KSTR];
  __shared__ __align__(16) unsigned char v_lds[D * VSTR];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l31 = lane & 31, lhi = lane >> 5;
  Share t;
  if (!find_share(a, ROWS, blockIdx.x, t)) return;          // (whole workgroups, before any barrier)
  const int rank = blockIdx.x - t.first, share = rank / t.seq.units, unit = rank - share * t.seq.units;
  const RowBlock rb = row_block(a, t.seq, unit, ROWS);
  const int t0 = share * t.chunk, seen_tiles = (rb.seen + 31) >> 5;       // (chunks are even)
  if (share > 0 && t0 >= seen_tiles) return;
  const int t1 = t0 + t.chunk < seen_tiles ? t0 + t.chunk : seen_tiles;

  // ---- the lane's row
  const int keys = t.seq.keys, nq = t.seq.nq, wave_first = rb.first + 32 * wave;
  const int r = wave_first + l31, rr = r < rb.rows ? r : rb.rows - 1, query = rr / a.group;
  const int64_t head = rb.h * a.group + (rr - query * a.group);
  const int seen = r < rb.rows ? (a.causal ? keys - nq + query + 1 : keys) : 0;
  // ... and of the wave: keys its first and its last row see
  const int wave_last = wave_first + 31 < rb.rows ? wave_first + 31 : rb.rows - 1;
  const int seen_first = a.causal ? keys - nq + wave_first / a.group + 1 : keys;
  const int seen_last = wave_first >= rb.rows ? 0 : a.causal ? keys - nq + wave_last / a.group + 1 : keys;
  abf16x8 qf[KS];
  {
    const bf16_t* qp = a.q + (t.seq.q0 + query) * a.q_row + head * D + 8 * lhi;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = load_q(qp + 16 * ks, a.q_sign);
  }
  af32x16 o[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
  float m = -INFINITY, shift = 0.f, sum = 0.f;
  const float slack = SLACK / a.scale_log2;

  // ---- staging: cache -> registers, a tile ahead -> LDS
  const int P = a.shape.page_tokens, page_tiles = P >> 5;
  const int32_t* table = a.table + (int64_t)t.b * a.table_width;
  int page = t0 / page_tiles, in_page = t0 - page * page_tiles, first_page = page, ahead = t0;
  const int last_page = t1 > t0 ? (t1 - 1) / page_tiles : page;
  auto load_pages = [&]() {
    const int x = first_page + lane;
    return x <= last_page ? table[x] : 0;
  };
  int pages = t1 > t0 ? load_pages() : 0;
  bool bad = false;
  words kw, vw;
  uint32_t ksc, vsc;
  // a thread's piece: token k_token of a half, part k_part of it; tokens 4 quad .., word j of each
  const int half = wave >> 1, k_token = (tid >> 2) & 31, k_part = tid & 3, quad = (tid >> 4) & 7, j = tid & 15;
  bool lost[2];                 // halves of the tile in registers that are in no page
  auto load_tile = [&]() {      // the tile of 64 keys at (page, in_page) = `ahead` tiles of 32, and the step to the next
    int page1 = page, in1 = in_page + 1;
    if (in1 == page_tiles) {
      in1 = 0;
      ++page1;
    }
    if (page1 - first_page >= 64) {
      first_page = page;
      pages = load_pages();
    }
    const int id0 = __builtin_amdgcn_readlane(pages, page - first_page), id1 = __builtin_amdgcn_readlane(pages, page1 - first_page);
    const bool there = ahead + 1 < t1;
    lost[0] = id0 < 0 || id0 >= a.shape.n_pages;
    lost[1] = there && (id1 < 0 || id1 >= a.shape.n_pages);
    bad |= lost[0] || lost[1];
    const unsigned char* block0 = a.pool + ((int64_t)(lost[0] ? 0 : id0) * a.shape.n_kv_heads + rb.h) * a.shape.head_bytes;
    const unsigned char* block1 = a.pool + ((int64_t)(lost[1] || !there ? 0 : id1) * a.shape.n_kv_heads + rb.h) * a.shape.head_bytes;
    const unsigned char* block = half ? block1 : block0;
    const int at = half ? in1 : in_page;
    kw = *reinterpret_cast<const words*>(block + at * (16 * D) + k_token * (D / 2) + k_part * (4 * NG));
    const unsigned char* sp = block + P * D + (at * 32 + k_token) * NG;
    if constexpr (NG == 4) ksc = *reinterpret_cast<const uint32_t*>(sp);
    else ksc = *reinterpret_cast<const uint16_t*>(sp);
    vw = *reinterpret_cast<const words*>(block + P * (D / 2) + at * (16 * D) + quad * (2 * D) + j * (4 * NG));
    vsc = *reinterpret_cast<const uint32_t*>(block + P * (D + NG) + at * (32 * NG) + (quad >> 1) * (8 * NG) + (j * NG >> 4) * 8 + (quad & 1) * 4);
    // tokens that do not exist have a scale of nothing: their codes may be anything, their product with zero must be zero
    const int held = (half ? lost[1] || !there : lost[0]) ? 0 : keys - (ahead * 32 + half * 32 + quad * 4);
    if (held < 4) vsc = held > 0 ? vsc & ((1u << (8 * held)) - 1) : 0;
    ahead += 2;
    in_page = in1 + 1;
    page = page1;
    if (in_page == page_tiles) {
      in_page = 0;
      ++page;
    }
  };
  // (quads 1 and 2 of every four change places: the eight tokens of a lane's operand are then 16 bytes side by side)
  const int place = 8 * half + ((quad & 4) | ((quad & 1) << 1) | ((quad >> 1) & 1));
  unsigned char* const k_to = k_lds + (tid >> 2) * KSTR + k_part * 16;
  unsigned char* const v_to = v_lds + j * VSTR + place * 8;
  auto store_tile = [&]() {
    auto group = [&](auto G) {
      constexpr int g = decltype(G)::value;
      const uint32_t sc = scale_of<g>(ksc);
      *reinterpret_cast<au32x4*>(k_to + g * 64) = au32x4{widen2<0>(kw[g], sc), widen2<1>(kw[g], sc), widen2<2>(kw[g], sc), widen2<3>(kw[g], sc)};
    };
    group(std::integral_constant<int, 0>());
    group(std::integral_constant<int, 1>());
    if constexpr (NG == 4) {
      group(std::integral_constant<int, 2>());
      group(std::integral_constant<int, 3>());
    }
    const uint32_t s0 = scale_of<0>(vsc), s1 = scale_of<1>(vsc), s2 = scale_of<2>(vsc), s3 = scale_of<3>(vsc);
    auto column = [&](auto B) {
      constexpr int b = decltype(B)::value;
      uint32_t x0, x1, x2, x3;          // values 2b, 2b + 1 of the four tokens
      if constexpr (NG == 4) {
        x0 = widen2<b>(vw[0], s0); x1 = widen2<b>(vw[1], s1); x2 = widen2<b>(vw[2], s2); x3 = widen2<b>(vw[3], s3);
      } else {
        x0 = widen2<b>(vw[0], s0); x1 = widen2<b + 2>(vw[0], s1); x2 = widen2<b>(vw[1], s2); x3 = widen2<b + 2>(vw[1], s3);
      }
      *reinterpret_cast<au32x2*>(v_to + 2 * b * 16 * VSTR) = au32x2{__builtin_amdgcn_perm(x1, x0, 0x05040100u), __builtin_amdgcn_perm(x3, x2, 0x05040100u)};
      *reinterpret_cast<au32x2*>(v_to + (2 * b + 1) * 16 * VSTR) = au32x2{__builtin_amdgcn_perm(x1, x0, 0x07060302u), __builtin_amdgcn_perm(x3, x2, 0x07060302u)};
    };
    column(std::integral_constant<int, 0>());
    column(std::integral_constant<int, 1>());
    if constexpr (NG == 4) {
      column(std::integral_constant<int, 2>());
      column(std::integral_constant<int, 3>());
    }
  };

  if (t0 < t1) load_tile();
  for (int tile = t0; tile < t1; tile += 2) {
    const int kv = tile * 32;
    __syncthreads();              // the tile before is consumed
    store_tile();
    const bool lost0 = lost[0], lost1 = lost[1];
    __syncthreads();
    if (tile + 2 < t1) load_tile();
    __builtin_amdgcn_sched_barrier(0);
    if (kv >= seen_last) continue;                  // (the whole wave) no row sees a key of the tile
    af32x16 s[2];
#pragma unroll
    for (int jt = 0; jt < 2; ++jt)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[jt][e] = 0.f;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int jt = 0; jt < 2; ++jt) {
        const abf16x8 kf = *reinterpret_cast<const abf16x8*>(k_lds + (jt * 32 + l31) * KSTR + ks * 32 + lhi * 16);
        s[jt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], s[jt], 0, 0, 0);
      }
    __builtin_amdgcn_s_setprio(0);
    // register e of a product holds key 8 (e / 4) + 4 lhi + e % 4
    if (kv + 64 > seen_first || lost0 || lost1) {
#pragma unroll
      for (int jt = 0; jt < 2; ++jt)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if ((jt ? lost1 : lost0) || kv + jt * 32 + 8 * (e >> 2) + 4 * lhi + (e & 3) >= seen) s[jt][e] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int jt = 0; jt < 2; ++jt)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[jt][e]);
    if (__any(top > m + slack)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float moved = top > m + slack || m == -INFINITY ? fmaxf(top, m) : m;
      const float alpha = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(shift - moved * a.scale_log2);
      m = moved;
      shift = m == -INFINITY ? 0.f : m * a.scale_log2;
      sum *= alpha;
#pragma unroll
      for (int i = 0; i < NG; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
    }
    abf16x8 pf[4];
#pragma unroll
    for (int jt = 0; jt < 2; ++jt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        au32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[jt][8 * u + 2 * e], a.scale_log2, -shift));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[jt][8 * u + 2 * e + 1], a.scale_log2, -shift));
          sum += p0 + p1;
          w[e] = pack2_k(p0, p1);
        }
        pf[jt * 2 + u] = __builtin_bit_cast(abf16x8, w);
      }
#pragma unroll
    for (int ku = 0; ku < 4; ++ku)
#pragma unroll
      for (int i = 0; i < NG; ++i) {
        const abf16x8 vf = *reinterpret_cast<const abf16x8*>(v_lds + (i * 32 + l31) * VSTR + ku * 32 + lhi * 16);
        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[ku], o[i], 0, 0, 0);
      }
  }
  if (bad && a.err && lane == 0) atomicOr(a.err, 1);

  // ---- register e of o[i] is row 16 (2 i + e / 8) + 8 (e / 4 % 2) + 4 lhi + e % 4 of the V^T tile
  sum += __shfl_xor(sum, 32);
  if (r >= rb.rows) return;
  const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
  const int64_t at = (int64_t)blockIdx.x * ROWS + 32 * wave + l31;
  if (t.shares > 1 && lhi == 0) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(m == -INFINITY ? m : shift, sum);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int word = 8 * (e >> 2) + 4 * lhi + (e & 3);
    float x[2 * NG];
#pragma unroll
    for (int d = 0; d < 2 * NG; ++d) x[d] = o[d >> 1][8 * (d & 1) + e];
    if (t.shares > 1) {
      af32x4* to = reinterpret_cast<af32x4*>(a.part_o + at * D + word * (2 * NG));
#pragma unroll
      for (int d = 0; d < 2 * NG; d += 4) to[d / 4] = af32x4{x[d], x[d + 1], x[d + 2], x[d + 3]};
    } else {
      words w;
#pragma unroll
      for (int d = 0; d < NG; ++d) w[d] = pack2_k(x[2 * d] * inv, x[2 * d + 1] * inv);
      *reinterpret_cast<words*>(a.out + (t.seq.q0 + query) * a.out_row + head * D + word * (2 * NG)) = w;
    }
  }
}

// ---- the shares of a row's keys, joined: 16 lanes a part, `join` parts of a row at a time, in an order that depends on
// the lengths alone.  Bound by latency (lengths, shares, parts, one behind the other): 4.4 .. 7.4 us, 13 where 57344 rows have two parts each.
// A launch of its own: a counter to tell the last workgroup of a row would have to be cleared by one.
template <int NG>
__global__ __launch_bounds__(256) void join_shares_kernel(CacheAttnArgs a) {
  constexpr int D = 32 * NG;
  __shared__ __align__(16) float state_o[16][D + 4];
  __shared__ float state_m[16], state_l[16];
  const int per = 16 / a.join;                               // rows of a workgroup
  const int block = blockIdx.x / a.join_groups, units = a.row_blocks * a.shape.n_kv_heads;
  const int b = a.planned ? find_sequence(a, 3, block) : block / units;
  const int4 share = *reinterpret_cast<const int4*>(a.share_of + 4 * (int64_t)b);
  const int unit = block - (a.planned ? share.w : b * units);
  const Sequence seq = sequence(a, b, a.rows);
  if (unit >= seq.units) return;                             // (whole workgroups, before any barrier)
  const int first = share.x, chunk = share.z;
  if (share.y == 1) return;
  // (lists of queries that overlap may have more parts than there is room for: theirs are not looked at)
  if (first < 0 || chunk < 1 || share.y != shares_of(seq, chunk) || first + (int64_t)seq.units * share.y > a.blocks) return;
  const RowBlock rb = row_block(a, seq, unit, a.rows);
  const int slot = threadIdx.x >> 4, jc = (threadIdx.x & 15) * (2 * NG);
  const int in_block = (blockIdx.x - block * a.join_groups) * per + slot / a.join;
  const int r = in_block < a.rows ? rb.first + in_block : rb.rows;
  const int seen_tiles = (rb.seen + 31) >> 5, used = seen_tiles > 0 ? (seen_tiles + chunk - 1) / chunk : 1;
  float mm = -INFINITY, ll = 0.f, acc[2 * NG] = {};
  if (r < rb.rows) {
    const int64_t at = ((int64_t)first + unit) * a.rows + in_block, step = (int64_t)seq.units * a.rows;
    constexpr int AHEAD = 4;                                 // parts asked for at a time
    for (int s0 = slot % a.join; s0 < used; s0 += AHEAD * a.join) {
      float2 ml[AHEAD];
      af32x4 v[AHEAD][NG / 2];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int s = s0 + u * a.join < used ? s0 + u * a.join : s0;
        ml[u] = *reinterpret_cast<const float2*>(a.part_ml + (at + s * step) * 2);
#pragma unroll
        for (int i = 0; i < NG / 2; ++i) v[u][i] = reinterpret_cast<const af32x4*>(a.part_o + (at + s * step) * D + jc)[i];
      }
      float top = mm;
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) top = fmaxf(top, ml[u].x);
      const float keep = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mm - top);
      mm = top;
      ll *= keep;
#pragma unroll
      for (int i = 0; i < 2 * NG; ++i) acc[i] *= keep;
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (s0 + u * a.join >= used) continue;
        const float f = ml[u].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[u].x - mm);    // (a NaN weight stays one)
        ll += f * ml[u].y;
#pragma unroll
        for (int i = 0; i < 2 * NG; ++i) acc[i] += f * v[u][i >> 2][i & 3];
      }
    }
  }
  if (a.join > 1) {
    state_m[slot] = mm;
    state_l[slot] = ll;
#pragma unroll
    for (int i = 0; i < 2 * NG; i += 4) *reinterpret_cast<af32x4*>(&state_o[slot][jc + i]) = af32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
    __syncthreads();
    if (slot % a.join) return;
    for (int u = 0; u < a.join; ++u) mm = fmaxf(mm, state_m[slot + u]);
    ll = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * NG; ++i) acc[i] = 0.f;
    for (int u = 0; u < a.join; ++u) {
      const float mu = state_m[slot + u], f = mu == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mu - mm);
      ll += f * state_l[slot + u];
#pragma unroll
      for (int i = 0; i < 2 * NG; ++i) acc[i] += f * state_o[slot + u][jc + i];
    }
  }
  if (r < rb.rows) store_row<NG>(a, seq.q0, rb.h, r, jc, acc, ll);
}

// The plan of the sequences with more than `more_than` rows and at most `at_most`
static size_t plan_rows(CacheAttnArgs& a) {
  const int64_t rows = std::min<int64_t>((int64_t)a.max_queries * a.group, a.at_most), all_rows = a.n_queries * a.group, tiles = (a.max_keys + 31) / 32;
  // Rows of a workgroup.  Widening the cache costs 32 rows as much as 16, and it is shared by 128: against that, blocks of 128 leave
  // most of the chip idle until there are about 1.2 10^8 products of a row and a key, and waste what a sequence's last block lacks.
  // 16 against 32, a token each: one sequence of 2048 keys 9.9 and 10.6 us, 64 of 160 .. 16384 36.4 and 49.4; 40 and 64 rows a unit
  // go either way by a tenth.  32 against 128: 64 rows a unit, 32 sequences of 8192 keys 69 and 92 us, 40 rows 42 and 48; prompts of
  // 500, 1000 and 2000 tokens, 28 heads (7 .. 112 million) 12.4 and 23, 26 and 37, 69 and 73; 512 tokens behind 8192 (125 million)
  // 113 and 93, four prompts of 1000 (128 million) 94 and 76, the largest chunk 599 and 489.
  const double work = (double)a.n_queries * (a.group * a.shape.n_kv_heads) * (double)a.max_keys;
  a.rows = rows <= 16 ? 16 : rows <= 64 || work < 1.2e8 ? 32 : 128;
  // Workgroups to share the work out to: as many as are on the chip at once (registers); of heads of 64 and 32 rows there would be 1024, but
  // 100 rows of each of 40 units take 19.1 us instead of 16.4 with 768.  (Heads of 64 as those of 128: 64 ragged sequences 20.5 us
  // instead of 19.8, chunks of 1024 behind 7168 212 instead of 187.)
  a.target = a.rows == 32 ? 512 : a.rows == 16 ? (a.shape.head_dim == 128 ? 1024 : 1280) : a.shape.head_dim == 128 ? 512 : 768;
  a.row_blocks = (int32_t)((rows + a.rows - 1) / a.rows);
  // units there may be: a sequence's last block of rows may be smaller than the others
  const int64_t seqs = std::min<int64_t>(a.n_seqs, all_rows / (a.more_than + 1)), each = (int64_t)a.n_seqs * a.row_blocks;
  const int64_t bound = std::min(seqs * a.row_blocks, seqs + all_rows / a.rows), row_units = bound * a.shape.n_kv_heads;
  a.blocks = 0;
  if (row_units > MAX_GROUPS) return 0;                      // (every launch has at least as many)
  // Tiles of a share, at least.  Up to 1024 keys one workgroup takes them all and there is nothing to join (32 sequences of 500 keys 13.9 ->
  // 9.7 us, one of 1000 the same); a few short rows are shared out finer (one token of 2048 keys 10.4 -> 9.8, of 4096 10.8 -> 10.4).
  a.least = a.rows == 128 ? 8 : tiles <= 32 ? 32 : row_units * ((tiles + 3) / 4) <= 256 ? 4 : 8;
  const int64_t most = std::max<int64_t>(1, (tiles + a.least - 1) / a.least);
  // (see find_share: a share is at least `least` tiles, and more than the work over `target`)
  const int64_t blocks = most > (1 << 20) ? row_units + a.target + 64 : std::min(row_units * most, row_units + a.target + 64);
  a.join = most == 1 ? 0 : 1;
  // (one launch: a workgroup for every block of rows that a sequence may have)
  const int64_t grid = a.join ? blocks : each > MAX_GROUPS ? each : each * a.shape.n_kv_heads;
  a.blocks = grid > MAX_GROUPS ? 0 : (int32_t)grid;
  if (!a.join || !a.blocks) return 0;
  a.planned = a.n_seqs > 64 || each > 2 * bound;
  a.units = a.planned ? row_units : each * a.shape.n_kv_heads;
  // a row's parts at a time: up to sixteen, while that is not more than 512 workgroups (64 ragged sequences 40.3 -> 38.3 us against
  // 2048, 128 rows of each of eight units 42.1 -> 40.2)
  const int64_t of_block = std::min<int64_t>(rows, a.rows);
  while (a.join < 16 && a.join < most && row_units * of_block * a.join * 2 <= 8192) a.join *= 2;
  a.join_groups = (int32_t)((of_block * a.join + 15) / 16);
  if (a.units * a.join_groups > MAX_GROUPS) {
    a.blocks = 0;
    return 0;
  }
  return (size_t)a.blocks * (size_t)a.rows * (size_t)(a.shape.head_dim + 2) * 4 + (size_t)a.n_seqs * 16;
}

// A batch of prompts and tokens: sequences of few rows and of many have launches of their own, with one workspace in turn.  (The host knows the
// number of queries and the most that a sequence has: half of n_seqs times that, or less, and the batch is taken for one.)  48 tokens behind 200
// .. 8000 keys and 512 queries behind 3584: 181 us as blocks of 128 rows, the two apart 101.
static int plan_parts(const CacheAttnArgs& a, CacheAttnArgs (&parts)[2]) {
  const int few = a.group <= 16 ? 16 : 32;
  parts[0] = a;
  parts[0].more_than = 0;
  parts[0].at_most = 0x7fffffff;
  if (a.group > 32 || (int64_t)a.max_queries * a.group <= 64 || a.n_queries * 2 > (int64_t)a.n_seqs * a.max_queries) return 1;
  parts[1] = parts[0];
  parts[0].more_than = parts[1].at_most = few;
  return 2;
}
cs_status plan_cache_attention(const CacheAttnArgs& a, size_t& bytes) {
  CacheAttnArgs parts[2];
  size_t need = 0;
  for (int n = a.n_seqs && a.n_queries && a.max_queries ? plan_parts(a, parts) : 0; n--;) {
    need = std::max(need, plan_rows(parts[n]));
    if (!parts[n].blocks) return fail(CS_ERR_UNSUPPORTED, "cs_attention_cache: more rows and sequences than a launch takes");
  }
  bytes = need;
  return CS_OK;
}

template <int NG>
static void launch_attend(const CacheAttnArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.blocks);
  if (a.rows == 16) hipLaunchKernelGGL((attend_rows_kernel<NG, 1>), grid, dim3(256), 0, stream, a);
  else if (a.rows == 32) hipLaunchKernelGGL((attend_rows_kernel<NG, 2>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((attend_block_kernel<NG>), grid, dim3(256), 0, stream, a);
}

static cs_status launch_rows(CacheAttnArgs& a, void* workspace, hipStream_t stream) {
  plan_rows(a);
  const int64_t joins = a.join ? a.units * a.join_groups : 0;
  a.part_o = static_cast<float*>(workspace);
  a.part_ml = a.part_o + (size_t)a.blocks * (size_t)a.rows * (size_t)a.shape.head_dim;
  a.share_of = reinterpret_cast<int32_t*>(a.part_ml + (size_t)a.blocks * (size_t)a.rows * 2);
  if (a.join && a.planned) {
    hipLaunchKernelGGL(share_out_kernel, dim3(1), dim3(1024), 0, stream, a);
    CS_HIP(hipGetLastError());
  }
  if (a.shape.head_dim == 128) launch_attend<4>(a, stream);
  else launch_attend<2>(a, stream);
  CS_HIP(hipGetLastError());
  if (joins) {
    if (a.shape.head_dim == 128) hipLaunchKernelGGL((join_shares_kernel<4>), dim3((unsigned)joins), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((join_shares_kernel<2>), dim3((unsigned)joins), dim3(256), 0, stream, a);
    CS_HIP(hipGetLastError());
  }
  return CS_OK;
}
cs_status launch_cache_attention(const CacheAttnArgs& a, void* workspace, hipStream_t stream) {
  CacheAttnArgs parts[2];
  const int n = plan_parts(a, parts);
  for (int i = 0; i < n; ++i)
    if (cs_status st = launch_rows(parts[i], workspace, stream)) return st;
  return CS_OK;
}

}  // namespace cs
