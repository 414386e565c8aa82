// Queries and keys normed and rotated in one pass; the 4-bit cache written and read.
//
// All three are bound by memory: a few operations a value.  Every access is 16 bytes a lane, and a lane keeps its values
// in registers from the load to the store.  Lanes of bf16 rows lie side by side; those of fp32 rows, and of values that pass
// the rotation, 32 bytes apart or 64, so that an instruction takes part of each line and the next one the rest.
// What is read once, or written and not read again here, goes past the caches (ONCE) where that measured faster.  Loops of calls on
// tensors that the caches do not hold, each as it was when the choice was made: rotation of 16384 x 32 heads of 128, bf16, loads
// 58.9 -> 50.9 us (stores too: 55.6); values out of the cache, 65536 rows of 4 heads of 128, stores 41.1 -> 25.7; rows into
// the cache, loads of 16384 rows of 8 heads 29.5 -> 32.0 with their reading back, so they are plain.
#include "cache.h"

#include <algorithm>
#include <type_traits>

namespace cs {

typedef unsigned int cu32x4 __attribute__((ext_vector_type(4)));
typedef float cf32x2 __attribute__((ext_vector_type(2)));
typedef float cf32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 cbf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack2_c(float a, float b) {
  const cf32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, cbf16x2));
}

template <bool ONCE, class T>
__device__ __forceinline__ T fetch(const T* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool ONCE, class T>
__device__ __forceinline__ void put(T v, T* p) {
  if constexpr (ONCE) __builtin_nontemporal_store(v, p);
  else *p = v;
}
// eight consecutive values of either type
template <bool BF16, bool ONCE>
__device__ __forceinline__ void load8(const void* base, int64_t at, float (&x)[8]) {
  if constexpr (BF16) {
    const cu32x4 u = fetch<ONCE>(reinterpret_cast<const cu32x4*>(static_cast<const bf16_t*>(base) + at));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
    const cf32x4* p = reinterpret_cast<const cf32x4*>(static_cast<const float*>(base) + at);
    const cf32x4 a = fetch<ONCE>(p), b = fetch<ONCE>(p + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
}
template <bool BF16, bool ONCE>
__device__ __forceinline__ void store8(void* base, int64_t at, const float (&x)[8]) {
  if constexpr (BF16) {
    cu32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = pack2_c(x[2 * i], x[2 * i + 1]);
    put<ONCE>(u, reinterpret_cast<cu32x4*>(static_cast<bf16_t*>(base) + at));
  } else {
    cf32x4* p = reinterpret_cast<cf32x4*>(static_cast<float*>(base) + at);
    put<ONCE>(cf32x4{x[0], x[1], x[2], x[3]}, p);
    put<ONCE>(cf32x4{x[4], x[5], x[6], x[7]}, p + 1);
  }
}

// ---- norm and rotation.  A lane holds sixteen values of a head: pairs 8l .. 8l+7, both members, so that the rotation
// needs no other lane; lanes behind the rotary part hold sixteen values that pass.  A head is LPH lanes (head_dim / 16 of
// them with values), a wave takes one token, 64 / LPH of its heads at a time: the angles are read once a token.
// 16384 rows of 32 heads of 128, bf16 (277 MB): 47.5 us, 5.8 TB/s; 1125 rows of 10 heads of 64, fp32: 4.7 us; one row: 3.2 us, a
// launch and three reads one behind the other (positions, angles, values).  What does not depend on one another is asked for at once: positions and
// angles one by one, and gains behind the sum, took 51.9, 5.5 and 4.3 us.
template <bool BF16, int LPH>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkArgs a) {
  constexpr int HEADS = 64 / LPH;               // heads of a wave at a time
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.n_rows) return;
  const int lane = threadIdx.x & 63, l = lane & (LPH - 1), slot = lane / LPH;
  int64_t pos[3];
#pragma unroll
  for (int x = 0; x < 3; ++x) pos[x] = a.positions[row * a.axes + (x < a.axes ? x : a.axes - 1)];      // (all at once, whatever the axes)
  bool bad = false;
#pragma unroll
  for (int x = 0; x < 3; ++x) bad |= pos[x] < 0 || pos[x] >= a.n_positions;
  if (bad) {
    if (a.err && lane == 0 && blockIdx.y == 0) atomicOr(a.err, 1);
    return;
  }
  const int rot_lanes = a.half >> 3;
  const bool turns = l < rot_lanes, has = l < (a.head_dim >> 4);
  const int d0 = turns ? 8 * l : 2 * a.half + 16 * (l - rot_lanes), d1 = turns ? a.half + 8 * l : d0 + 8;
  float c[8], s[8];
  const int first = turns ? 8 * l : 0;          // (every lane loads, so that nothing waits for a branch; those that do not turn drop it)
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int j = first + i, m = j % 3;
    const bool second = (j >= a.end0) | ((m == 1) & (j < a.lim1)), third = (j >= a.end1) | ((m == 2) & (j < a.lim2));
    const int64_t at = third ? pos[2] : second ? pos[1] : pos[0];
    const float2 cs = *reinterpret_cast<const float2*>(a.cos_sin + (at * a.half + j) * 2);
    c[i] = cs.x;
    s[i] = cs.y;
  }
  const int heads = a.n_heads + a.n_kv_heads, steps = (heads + HEADS - 1) / HEADS;
  for (int step = blockIdx.y; step < steps; step += a.parts) {
    const int h = step * HEADS + slot;
    const bool live = has && h < heads, is_q = h < a.n_heads;
    float x[8] = {}, y[8] = {};
    const void* src = is_q ? a.q : a.k;
    const int64_t at = is_q ? row * a.q_row + (int64_t)h * a.head_dim : row * a.k_row + (int64_t)(h - a.n_heads) * a.head_dim;
    float g0[8] = {}, g1[8] = {};
    if (live) {
      if (a.norm) {                     // (asked for with the values, not behind their sum)
        load8<false, false>(is_q ? a.q_gain : a.k_gain, d0, g0);
        load8<false, false>(is_q ? a.q_gain : a.k_gain, d1, g1);
      }
      load8<BF16, true>(src, at + d0, x);
      load8<BF16, true>(src, at + d1, y);
    }
    if (a.norm) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += x[i] * x[i] + y[i] * y[i];
#pragma unroll
      for (int m = 1; m < LPH; m <<= 1) sum += __shfl_xor(sum, m);
      const float r = rsqrtf(sum / (float)a.head_dim + a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= r * g0[i];
        y[i] *= r * g1[i];
      }
    }
    if (!live) continue;
    if (turns) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = x[i] * c[i] - y[i] * s[i];
        y[i] = y[i] * c[i] + x[i] * s[i];
        x[i] = u;
      }
    }
    const int64_t to = is_q ? row * a.q_out_row + (int64_t)h * a.head_dim : row * a.k_out_row + (int64_t)(h - a.n_heads) * a.head_dim;
    void* dst = is_q ? a.q_out : a.k_out;
    store8<BF16, false>(dst, to + d0, x);
    store8<BF16, false>(dst, to + d1, y);
  }
}

// p, `elements` of them further on
template <class T>
static T* moved(T* p, int64_t elements, int dtype) {
  typedef std::conditional_t<std::is_const<T>::value, const unsigned char, unsigned char> bytes;
  return p ? static_cast<bytes*>(p) + elements * (dtype == CS_BF16 ? 2 : 4) : nullptr;
}

// as many rows as a grid may have
static cs_status launch_qk_rows(QkArgs a, int dtype, hipStream_t stream) {
  const int lanes = a.head_dim <= 64 ? 4 : a.head_dim <= 128 ? 8 : 16;
  const int steps = (a.n_heads + a.n_kv_heads + 64 / lanes - 1) / (64 / lanes);
  const int64_t blocks = (a.n_rows + 3) / 4;
  // few tokens: their heads are shared out so that every wave has one step
  a.parts = (int)std::min<int64_t>(steps, std::max<int64_t>(1, 2048 / blocks));
  const dim3 grid((unsigned)blocks, (unsigned)a.parts);
  const bool b = dtype == CS_BF16;
  if (lanes == 4 && b) hipLaunchKernelGGL((qk_norm_rope_kernel<true, 4>), grid, dim3(256), 0, stream, a);
  else if (lanes == 4) hipLaunchKernelGGL((qk_norm_rope_kernel<false, 4>), grid, dim3(256), 0, stream, a);
  else if (lanes == 8 && b) hipLaunchKernelGGL((qk_norm_rope_kernel<true, 8>), grid, dim3(256), 0, stream, a);
  else if (lanes == 8) hipLaunchKernelGGL((qk_norm_rope_kernel<false, 8>), grid, dim3(256), 0, stream, a);
  else if (b) hipLaunchKernelGGL((qk_norm_rope_kernel<true, 16>), grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL((qk_norm_rope_kernel<false, 16>), grid, dim3(256), 0, stream, a);
  CS_HIP(hipGetLastError());
  return CS_OK;
}
cs_status launch_qk_norm_rope(const QkArgs& args, int dtype, hipStream_t stream) {
  for (int64_t first = 0; first < args.n_rows; first += MAX_GROUPS * 4) {
    QkArgs a = args;
    a.n_rows = std::min<int64_t>(args.n_rows - first, MAX_GROUPS * 4);
    a.q = moved(args.q, first * args.q_row, dtype);
    a.k = moved(args.k, first * args.k_row, dtype);
    a.q_out = moved(args.q_out, first * args.q_out_row, dtype);
    a.k_out = moved(args.k_out, first * args.k_out_row, dtype);
    a.positions = args.positions + first * args.axes;
    if (cs_status st = launch_qk_rows(a, dtype, stream)) return st;
  }
  return CS_OK;
}

// ---- the cache.  D / 8 lanes hold a row of one head, eight values each: a lane's K codes are one word, a group of 32
// values is four neighbouring lanes.  Rows go to slots in any order, so a row's codes are pieces of 4 bytes in two blocks; the rows of a
// workgroup, mostly neighbours, fill whole lines between them.  16384 rows of 8 heads of 128, bf16, in (67 MB + 18 MB): 13.9 us,
// 6.1 TB/s, and out again 14.0; 65536 rows of 4 heads out (36 + 134 MB): 25.7 us, 6.6 TB/s; 48 rows 3 us, the launch.
// Where the words of chunk c (values 8c .. 8c+7) of token `o` are in a block (see cs_cache_config).
template <int D>
struct Place {
  static constexpr int NG = D / 32;
  static __device__ __forceinline__ int k(int o, int c) { return o * (D / 2) + ((c & 3) * NG + (c >> 2)) * 4; }
  static __device__ __forceinline__ int64_t v(int64_t page, int o, int c) {   // D 128: a word; D 64: two half words 8 bytes apart
    return page * (D / 2) + (o >> 2) * (2 * D) + (D == 128 ? c * 16 + (o & 3) * 4 : c * 16 + (o & 3) * 2);
  }
  static __device__ __forceinline__ int64_t k_scale(int64_t page, int o, int g) { return page * D + o * NG + g; }
  static __device__ __forceinline__ int64_t v_scale(int64_t page, int o, int g) { return page * (D + NG) + (o >> 3) * (8 * NG) + g * 8 + (o & 7); }
};

// largest magnitude of the group's values as bits (NaN above infinity above every number)
__device__ __forceinline__ uint32_t group_max_bits(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  m = max(m, (uint32_t)__shfl_xor((int)m, 1));
  return max(m, (uint32_t)__shfl_xor((int)m, 2));
}

// Eight codes of a lane's values and the group's scale byte.  The byte: adding a quarter to the mantissa carries into the
// exponent from 1.75 on.  The conversion instruction divides by the scale exactly, rounds to nearest even and saturates.
__device__ __forceinline__ uint32_t quantise8(float (&x)[8], int& byte, bool& odd_values) {
  uint32_t m = group_max_bits(x);
  odd_values = m >= 0x7f800000u;
  if (odd_values) {               // (the four lanes of a group take this together)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] != x[i] ? 0.f : fminf(fmaxf(x[i], -3.4028234663852886e38f), 3.4028234663852886e38f);
    m = group_max_bits(x);
  }
  byte = (int)((m + 0x200000u) >> 23) - 2;
  byte = byte < 2 ? 2 : byte > 252 ? 252 : byte;
  const float scale = __uint_as_float((uint32_t)byte << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

template <bool BF16, int D>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheRows a) {
  constexpr int LANES = D / 8;
  const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (row >= a.n_rows) return;      // (whole groups of lanes)
  const int c = threadIdx.x % LANES, h = blockIdx.y;
  const int64_t slot = a.slots[row];
  float x[8], y[8];
  load8<BF16, false>(a.k, row * a.k_row + h * D + 8 * c, x);
  load8<BF16, false>(a.v, row * a.v_row + h * D + 8 * c, y);
  int kb, vb;
  bool ko, vo;
  const uint32_t kw = quantise8(x, kb, ko), vw = quantise8(y, vb, vo);        // (in front of the slot's branch: the rows come while the slot does)
  if (slot < 0 || slot >= a.shape.slots) {
    if (slot != -1 && a.err && c == 0 && h == 0) atomicOr(a.err, 1);
    return;
  }
  const int64_t page = (int64_t)__umul64hi((uint64_t)slot, a.shape.page_recip), P = a.shape.page_tokens;
  const int o = (int)(slot - page * P);
  unsigned char* block = a.pool + (page * a.shape.n_kv_heads + h) * a.shape.head_bytes;
  *reinterpret_cast<uint32_t*>(block + Place<D>::k(o, c)) = kw;
  unsigned char* vp = block + Place<D>::v(P, o, c);
  if constexpr (D == 128) {
    *reinterpret_cast<uint32_t*>(vp) = vw;
  } else {
    *reinterpret_cast<uint16_t*>(vp) = (uint16_t)vw;
    *reinterpret_cast<uint16_t*>(vp + 8) = (uint16_t)(vw >> 16);
  }
  if ((c & 3) == 0) {
    block[Place<D>::k_scale(P, o, c >> 2)] = (unsigned char)kb;
    block[Place<D>::v_scale(P, o, c >> 2)] = (unsigned char)vb;
    if ((ko || vo) && a.err) atomicOr(a.err, 2);
  }
}

__device__ __forceinline__ void values8(uint32_t w, int byte, float (&x)[8]) {
  const float scale = __uint_as_float((uint32_t)byte << 23);
  const cf32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const cf32x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  x[0] = p0.x; x[1] = p0.y; x[2] = p1.x; x[3] = p1.y; x[4] = p2.x; x[5] = p2.y; x[6] = p3.x; x[7] = p3.y;
}

template <bool BF16, int D>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheRows a) {
  constexpr int LANES = D / 8;
  const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (row >= a.n_rows) return;
  const int c = threadIdx.x % LANES, h = blockIdx.y;
  const int64_t slot = a.slots[row];
  float x[8] = {}, y[8] = {};
  if (slot >= 0 && slot < a.shape.slots) {
    const int64_t page = (int64_t)__umul64hi((uint64_t)slot, a.shape.page_recip), P = a.shape.page_tokens;
    const int o = (int)(slot - page * P);
    const unsigned char* block = a.pool + (page * a.shape.n_kv_heads + h) * a.shape.head_bytes;
    const unsigned char* vp = block + Place<D>::v(P, o, c);
    uint32_t vw;
    if constexpr (D == 128) vw = *reinterpret_cast<const uint32_t*>(vp);
    else vw = *reinterpret_cast<const uint16_t*>(vp) | (uint32_t)*reinterpret_cast<const uint16_t*>(vp + 8) << 16;
    values8(*reinterpret_cast<const uint32_t*>(block + Place<D>::k(o, c)), block[Place<D>::k_scale(P, o, c >> 2)], x);
    values8(vw, block[Place<D>::v_scale(P, o, c >> 2)], y);
  } else if (slot != -1 && a.err && c == 0 && h == 0) {
    atomicOr(a.err, 1);
  }
  store8<BF16, true>(a.k, row * a.k_row + h * D + 8 * c, x);
  store8<BF16, true>(a.v, row * a.v_row + h * D + 8 * c, y);
}

static int64_t blocks_of(const CacheRows& a) { return (a.n_rows + 2048 / a.shape.head_dim - 1) / (2048 / a.shape.head_dim); }
// as many rows at a time as a grid may have
template <class F>
static cs_status by_grids(const CacheRows& all, int dtype, F launch) {
  const int64_t most = MAX_GROUPS * (2048 / all.shape.head_dim);
  for (int64_t first = 0; first < all.n_rows; first += most) {
    CacheRows a = all;
    a.n_rows = std::min(all.n_rows - first, most);
    a.k = moved(all.k, first * all.k_row, dtype);
    a.v = moved(all.v, first * all.v_row, dtype);
    a.slots = all.slots + first;
    launch(a);
    CS_HIP(hipGetLastError());
  }
  return CS_OK;
}

cs_status launch_cache_write(const CacheRows& rows, int dtype, hipStream_t stream) {
  const int D = rows.shape.head_dim;
  return by_grids(rows, dtype, [&](const CacheRows& a) {
    const dim3 grid((unsigned)blocks_of(a), (unsigned)a.shape.n_kv_heads);
    const bool b = dtype == CS_BF16;
    if (D == 128 && b) hipLaunchKernelGGL((cache_write_kernel<true, 128>), grid, dim3(256), 0, stream, a);
    else if (D == 128) hipLaunchKernelGGL((cache_write_kernel<false, 128>), grid, dim3(256), 0, stream, a);
    else if (b) hipLaunchKernelGGL((cache_write_kernel<true, 64>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((cache_write_kernel<false, 64>), grid, dim3(256), 0, stream, a);
  });
}

cs_status launch_cache_read(const CacheRows& rows, int dtype, hipStream_t stream) {
  const int D = rows.shape.head_dim;
  return by_grids(rows, dtype, [&](const CacheRows& a) {
    const dim3 grid((unsigned)blocks_of(a), (unsigned)a.shape.n_kv_heads);
    const bool b = dtype == CS_BF16;
    if (D == 128 && b) hipLaunchKernelGGL((cache_read_kernel<true, 128>), grid, dim3(256), 0, stream, a);
    else if (D == 128) hipLaunchKernelGGL((cache_read_kernel<false, 128>), grid, dim3(256), 0, stream, a);
    else if (b) hipLaunchKernelGGL((cache_read_kernel<true, 64>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((cache_read_kernel<false, 64>), grid, dim3(256), 0, stream, a);
  });
}

}  // namespace cs
