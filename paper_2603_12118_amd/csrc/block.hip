// The norms around a block with its gate and residual scale; weights laid out for products.
#include "block.h"

#include <algorithm>
#include <type_traits>

#include "rows.h"

namespace cs {

// ---- norms around a block.  TPR lanes hold a row, P pieces of eight values each, from the loads to the stores: x and the residual are
// read once, r and y written once, and the two means (or means and variances, deviations from the mean, not differences of squares) are
// sums over the lanes in between.  Rows are independent, so r may lie on the residual and y on x.
// Bound by memory: 16384 rows of 3584, bf16 with an fp32 residual and a gate a row (822 MB), 149 us, 5.5 TB/s; by latency below some
// 1000 rows: one row 2.9 us, a launch, the reads and two sums one behind the other.  Asking for the gains with the rows instead of in front of
// each sum took 153 us to 149, storing past the caches 158 to 153 (1125 rows of 1280, fp32: 7.5 to 6.4), reading past them
// loses (159; 7.8).  Rows of 8192 in four pieces a lane and of 16384 in 1024 lanes: 4096 of them in bf16 60 and 118 us, 4.5 TB/s.  A wave a row, which needs no barrier, is slower from 1280 values on (1125 rows: 10.3 us).
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* shared, int& turn) {
  v = wave_sum(v);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    float* at = shared + (turn ^= W);                  // (two places in turn: one barrier a sum)
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += at[w];
  }
  return v;
}

template <bool XB, bool RB, bool LAYER, int TPR, int P, bool HOLD = P <= 2>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_residual_kernel(NormResidualArgs a) {
  constexpr int ROWS = TPR < 256 ? 256 / TPR : 1;
  __shared__ float shared[TPR > 64 ? 2 * TPR / 64 : 1];
  int turn = 0;
  const int64_t row = (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x / TPR : 0);
  if (ROWS > 1 && row >= a.n_rows) return;             // (a whole wave)
  const int l = threadIdx.x % TPR;
  int at[P];
  bool has[P];
  float pre[P][8], post[P][8];                         // gains
#pragma unroll
  for (int p = 0; p < P; ++p) {
    at[p] = 8 * (l + p * TPR);
    has[p] = at[p] < a.width;
    if (HOLD && has[p]) {                              // (for four pieces they would take the registers of two more waves)
      if (a.post_gain) load8<false, false>(a.post_gain, at[p], post[p]);
      load8<false, false>(a.pre_gain, at[p], pre[p]);
    }
  }

  // v = N(v) with a gain, and a bias where there is one
  auto normed = [&](float (&v)[P][8], float (&w)[P][8], const float* gain, const float* bias) {
    float mean = 0.f;
    if constexpr (LAYER) {
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int i = 0; i < 8; ++i) mean += has[p] ? v[p][i] : 0.f;
      mean = row_sum<TPR>(mean, shared, turn) * a.inv_width;
    }
    float sum = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (LAYER) v[p][i] -= mean;
        sum += has[p] ? v[p][i] * v[p][i] : 0.f;
      }
    if constexpr (!HOLD) {
#pragma unroll
      for (int p = 0; p < P; ++p)                      // (asked for before the sum is waited for)
        if (has[p]) load8<false, false>(gain, at[p], w[p]);
    }
    const float scale = 1.f / sqrtf(row_sum<TPR>(sum, shared, turn) * a.inv_width + a.eps);
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[p][i] *= scale * w[p][i];
    if (bias) {
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (has[p]) {
          float c[8];
          load8<false, false>(bias, at[p], c);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[p][i] += c[i];
        }
    }
  };

  float z[P][8], g[P][8], res[P][8];
#pragma unroll
  for (int p = 0; p < P; ++p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) z[p][i] = 0.f;
    if (has[p]) load8<XB, false>(a.x, row * a.x_row + at[p], z[p]);
  }
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (has[p]) load8<RB, false>(a.residual, row * a.residual_row + at[p], res[p]);
  if (a.gate) {
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (has[p]) load8<XB, false>(a.gate, row * a.gate_row + at[p], g[p]);
  }
  if (a.post_gain) normed(z, post, a.post_gain, a.post_bias);
  if (a.gate) {
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
      for (int i = 0; i < 8; ++i) z[p][i] *= g[p][i];
  }
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (has[p]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) z[p][i] = fmaf(a.block_scale, z[p][i], a.residual_scale * res[p][i]);
      store8<RB, true>(a.r_out, row * a.r_row + at[p], z[p]);
    }
  normed(z, pre, a.pre_gain, a.pre_bias);
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (has[p]) store8<XB, true>(a.y, row * a.y_row + at[p], z[p]);
}

// Workgroups that a launch may have (HIP refuses more than 2^32 - 1 threads along a dimension)
static int64_t max_groups(int threads) { return 0xffffffffll / threads; }

template <class T>
static T* further(T* p, int64_t elements, int dtype) {
  typedef std::conditional_t<std::is_const<T>::value, const unsigned char, unsigned char> bytes;
  return p ? static_cast<bytes*>(p) + elements * (dtype == CS_BF16 ? 2 : 4) : nullptr;
}

template <bool XB, bool RB, bool LAYER>
static void launch_norm_rows(const NormResidualArgs& a, hipStream_t s) {
  const unsigned rows = (unsigned)a.n_rows, quarter = (unsigned)((a.n_rows + 3) / 4);
  const int w = a.width;
  if (w <= 512) hipLaunchKernelGGL((norm_residual_kernel<XB, RB, LAYER, 64, 1>), dim3(quarter), dim3(256), 0, s, a);
  else if (w <= 1024) hipLaunchKernelGGL((norm_residual_kernel<XB, RB, LAYER, 64, 2>), dim3(quarter), dim3(256), 0, s, a);
  else if (w <= 2048) hipLaunchKernelGGL((norm_residual_kernel<XB, RB, LAYER, 256, 1>), dim3(rows), dim3(256), 0, s, a);
  else if (w <= 4096) hipLaunchKernelGGL((norm_residual_kernel<XB, RB, LAYER, 256, 2>), dim3(rows), dim3(256), 0, s, a);
  else if (w <= 8192) hipLaunchKernelGGL((norm_residual_kernel<XB, RB, LAYER, 256, 4>), dim3(rows), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((norm_residual_kernel<XB, RB, LAYER, 1024, 2>), dim3(rows), dim3(1024), 0, s, a);
}

cs_status launch_norm_residual(const NormResidualArgs& args, bool layer, int dtype, int residual_dtype, hipStream_t s) {
  const int64_t most = max_groups(1024);
  for (int64_t first = 0; first < args.n_rows; first += most) {
    NormResidualArgs a = args;
    a.n_rows = std::min(args.n_rows - first, most);
    a.x = further(args.x, first * args.x_row, dtype);
    a.gate = further(args.gate, first * args.gate_row, dtype);
    a.y = further(args.y, first * args.y_row, dtype);
    a.residual = further(args.residual, first * args.residual_row, residual_dtype);
    a.r_out = further(args.r_out, first * args.r_row, residual_dtype);
    a.inv_width = 1.f / (float)a.width;
    const bool xb = dtype == CS_BF16, rb = residual_dtype == CS_BF16;
    if (layer) {
      if (xb) rb ? launch_norm_rows<true, true, true>(a, s) : launch_norm_rows<true, false, true>(a, s);
      else rb ? launch_norm_rows<false, true, true>(a, s) : launch_norm_rows<false, false, true>(a, s);
    } else {
      if (xb) rb ? launch_norm_rows<true, true, false>(a, s) : launch_norm_rows<true, false, false>(a, s);
      else rb ? launch_norm_rows<false, true, false>(a, s) : launch_norm_rows<false, false, false>(a, s);
    }
    CS_HIP(hipGetLastError());
  }
  return CS_OK;
}

// ---- weights.  A wave takes a block: 16 rows of 128 values.  Lane l reads the eight values of each step that it will hold as an operand, so
// that what it writes lies at its own place: 16 bytes a lane of codes, or 16 bytes a step of bf16.  The four lanes of a row share its
// scales.  Rows of the last tile behind n become zeros.  128 matrices of 1536 x 2048 from bf16 (805 MB) into 4 bits:
// 265 - 305 us, 3.3 - 3.8 TB/s, into bf16 396, 4.1 TB/s, and read back 213 and 338; it is done once.
template <bool BF16, bool E2M1>
__global__ __launch_bounds__(256) void weights_pack_kernel(PackArgs a) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t tile = a.first + unit / a.shape.blocks;
  const int b = (int)(unit % a.shape.blocks);
  const int64_t m = tile / a.shape.tiles;
  if (m >= a.shape.matrices) return;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int64_t j = (tile % a.shape.tiles) * 16 + r;
  const int steps = min(4, (a.shape.k - 128 * b) / 32);
  const int64_t from = m * a.w_matrix + j * a.w_row + 128 * b + 8 * g;
  unsigned char* to = a.packed + tile * a.shape.tile_bytes;
  uint32_t codes[4], bytes = 0;
  bool odd = false;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    float x[8] = {};
    if (s < steps && j < a.shape.n) load8<BF16, true>(a.w, from + 32 * s, x);
    if constexpr (E2M1) {
      int byte;
      bool o;
      codes[s] = quantise8<16>(x, byte, o);
      bytes |= (uint32_t)byte << (8 * s);
      odd |= o;
    } else if (s < steps) {
      store8<true, false>(to, (int64_t)b * 2048 + s * 512 + lane * 8, x);
    }
  }
  if constexpr (E2M1) {
    *reinterpret_cast<cu32x4*>(to + (int64_t)b * 1024 + lane * 16) = cu32x4{codes[0], codes[1], codes[2], codes[3]};
    if (g == 0) *reinterpret_cast<uint32_t*>(to + (int64_t)a.shape.blocks * 1024 + b * 64 + r * 4) = bytes;
    if (odd && a.err) atomicOr(a.err, 2);
  }
}

template <bool BF16, bool E2M1>
__global__ __launch_bounds__(256) void weights_read_kernel(PackArgs a) {
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t tile = a.first + unit / a.shape.blocks;
  const int b = (int)(unit % a.shape.blocks);
  const int64_t m = tile / a.shape.tiles;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int64_t j = (tile % a.shape.tiles) * 16 + r;
  if (m >= a.shape.matrices || j >= a.shape.n) return;
  const int steps = min(4, (a.shape.k - 128 * b) / 32);
  const int64_t at = m * a.w_matrix + j * a.w_row + 128 * b + 8 * g;
  const unsigned char* from = a.packed + tile * a.shape.tile_bytes;
  cu32x4 codes = {};
  uint32_t bytes = 0;
  if constexpr (E2M1) {
    codes = *reinterpret_cast<const cu32x4*>(from + (int64_t)b * 1024 + lane * 16);
    bytes = *reinterpret_cast<const uint32_t*>(from + (int64_t)a.shape.blocks * 1024 + b * 64 + r * 4);
  }
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    if (s >= steps) break;
    float x[8];
    if constexpr (E2M1) values8(codes[s], (int)(bytes >> (8 * s) & 255), x);
    else load8<true, false>(from, (int64_t)b * 2048 + s * 512 + lane * 8, x);
    store8<BF16, true>(const_cast<void*>(a.w), at + 32 * s, x);
  }
}

template <class K>
static cs_status over_tiles(PackArgs a, hipStream_t s, K kernel) {
  const int64_t tiles = a.shape.matrices * a.shape.tiles, most = std::max<int64_t>(1, max_groups(256) * 4 / a.shape.blocks);
  for (a.first = 0; a.first < tiles; a.first += most) {
    // (a launch of fewer tiles than are left has whole workgroups' worth of units, or its last ones are another launch's too: the same bytes)
    const int64_t units = std::min(most, tiles - a.first) * a.shape.blocks;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, a);
    CS_HIP(hipGetLastError());
  }
  return CS_OK;
}
cs_status launch_weights_pack(const PackArgs& a, int dtype, hipStream_t s) {
  const bool e = a.shape.format == CS_WEIGHTS_E2M1;
  if (dtype == CS_BF16) return e ? over_tiles(a, s, weights_pack_kernel<true, true>) : over_tiles(a, s, weights_pack_kernel<true, false>);
  return e ? over_tiles(a, s, weights_pack_kernel<false, true>) : over_tiles(a, s, weights_pack_kernel<false, false>);
}
cs_status launch_weights_read(const PackArgs& a, int dtype, hipStream_t s) {
  const bool e = a.shape.format == CS_WEIGHTS_E2M1;
  if (dtype == CS_BF16) return e ? over_tiles(a, s, weights_read_kernel<true, true>) : over_tiles(a, s, weights_read_kernel<true, false>);
  return e ? over_tiles(a, s, weights_read_kernel<false, true>) : over_tiles(a, s, weights_read_kernel<false, false>);
}

}  // namespace cs
