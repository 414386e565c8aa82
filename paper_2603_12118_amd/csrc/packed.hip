// Products of rows with packed weights, and the experts of a mixture built on them.
//
// y^T = W x^T with v_mfma_f32_16x16x32_bf16: the weights are the first operand (a lane holds row l % 16, eight values along k), the rows
// the second (a lane holds row l % 16 of x, the same eight values of k), and a lane ends with four neighbouring columns of one row.
// Weights come from memory straight into the registers that hold the operand; 4-bit ones are widened there, exactly (a level times a power of two is a
// bf16 number), so no operand of theirs passes LDS.
#include "block.h"

#include <algorithm>

#include "rows.h"

namespace cs {

typedef __bf16 pbf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void plds_void;

template <int FMT>
struct Held;                          // a block of a tile (16 rows, 128 values along k), as a lane holds it
template <>
struct Held<CS_WEIGHTS_E2M1> {
  cu32x4 codes;
  uint32_t scales;
  __device__ __forceinline__ void load(const unsigned char* tile, int blocks, int b, int lane, int) {
    codes = __builtin_nontemporal_load(reinterpret_cast<const cu32x4*>(tile + (int64_t)b * 1024 + lane * 16));
    scales = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(tile + (int64_t)blocks * 1024 + b * 64 + (lane & 15) * 4));
  }
  template <int S>
  __device__ __forceinline__ pbf16x8 step() const {
    const uint32_t scale = scale_of<S>(scales), w = codes[S];
    return __builtin_bit_cast(pbf16x8, cu32x4{widen2<0>(w, scale), widen2<1>(w, scale), widen2<2>(w, scale), widen2<3>(w, scale)});
  }
};
template <>
struct Held<CS_WEIGHTS_BF16> {
  cu32x4 v[4];
  __device__ __forceinline__ void load(const unsigned char* tile, int, int b, int lane, int steps) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
      if (s < steps) v[s] = __builtin_nontemporal_load(reinterpret_cast<const cu32x4*>(tile + (int64_t)b * 4096 + s * 1024 + lane * 16));
  }
  template <int S>
  __device__ __forceinline__ pbf16x8 step() const { return __builtin_bit_cast(pbf16x8, v[S]); }
};

template <int S>
struct step_tag { static constexpr int value = S; };
// f(step_tag<0>) .. f(step_tag<3>), as many as a block has
template <class F>
__device__ __forceinline__ void each_step(int steps, F&& f) {
  f(step_tag<0>());
  if (steps > 1) f(step_tag<1>());
  if (steps > 2) f(step_tag<2>());
  if (steps > 3) f(step_tag<3>());
}
template <class F>
__device__ __forceinline__ void all_steps(F&& f) {
  f(step_tag<0>());
  f(step_tag<1>());
  f(step_tag<2>());
  f(step_tag<3>());
}

__device__ __forceinline__ cf32x4 mfma(pbf16x8 w, pbf16x8 x, cf32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0); }

// ---- up to 16 rows: no LDS on the way in.  acc[j] += blocks [b0, b1) of tile j times x.  xl: the lane's row of x, at 8 (lane / 16); lanes
// without a row (!live) keep zeros and load nothing.  U blocks are asked for together.
template <int FMT, int RT, int U>
__device__ __forceinline__ void direct_product(cf32x4 (&acc)[RT], const unsigned char* const (&tile)[RT], int blocks, int k, int b0, int b1,
                                               const bf16_t* xl, bool live, int lane) {
  int b = b0;
  const int full = min(b1, k / 128);
  for (; b + U <= full; b += U) {
    Held<FMT> w[U][RT];
    cu32x4 x[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < RT; ++j) w[u][j].load(tile[j], blocks, b + u, lane, 4);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        x[u][s] = cu32x4{0, 0, 0, 0};
        if (live) x[u][s] = *reinterpret_cast<const cu32x4*>(xl + (int64_t)(b + u) * 128 + s * 32);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      all_steps([&](auto t) {
        constexpr int S = decltype(t)::value;
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[j] = mfma(w[u][j].template step<S>(), __builtin_bit_cast(pbf16x8, x[u][S]), acc[j]);
      });
  }
  for (; b < b1; ++b) {
    const int steps = min(4, (k - 128 * b) / 32);
    Held<FMT> w[RT];
    cu32x4 x[4];
#pragma unroll
    for (int j = 0; j < RT; ++j) w[j].load(tile[j], blocks, b, lane, steps);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      x[s] = cu32x4{0, 0, 0, 0};
      if (live && s < steps) x[s] = *reinterpret_cast<const cu32x4*>(xl + (int64_t)b * 128 + s * 32);
    }
    each_step(steps, [&](auto t) {
      constexpr int S = decltype(t)::value;
#pragma unroll
      for (int j = 0; j < RT; ++j) acc[j] = mfma(w[j].template step<S>(), __builtin_bit_cast(pbf16x8, x[S]), acc[j]);
    });
  }
}

// four neighbouring columns of a row; `whole`: all of them are there and the place is aligned to them
template <bool BF16>
__device__ __forceinline__ void store4(void* out, int64_t at, cf32x4 v, int left, bool whole) {
  if constexpr (BF16) {
    bf16_t* p = static_cast<bf16_t*>(out) + at;
    const uint32_t a = pack2_c(v[0], v[1]), b = pack2_c(v[2], v[3]);
    if (whole) {
      *reinterpret_cast<uint2*>(p) = uint2{a, b};
    } else {
      const uint32_t h[4] = {a, a >> 16, b, b >> 16};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < left) p[i] = (bf16_t)h[i];
    }
  } else {
    float* p = static_cast<float*>(out) + at;
    if (whole) {
      *reinterpret_cast<cf32x4*>(p) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < left) p[i] = v[i];
    }
  }
}
__device__ __forceinline__ cf32x4 bias4(const float* bias, int n, int N) {
  cf32x4 b = {0.f, 0.f, 0.f, 0.f};
  if (bias) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < N) b[i] = bias[n + i];
  }
  return b;
}

// A workgroup takes RT tiles of the weights; its waves share out k and their sums are added in LDS, wave by wave.
template <int FMT, bool BF16, int RT>
__global__ __launch_bounds__(1024) void linear_direct_kernel(LinearArgs a, int whole_rows) {
  __shared__ cf32x4 part[16][RT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int t = lane & 15, g = lane >> 4;
  const bool live = t < (int)a.n_rows;
  const unsigned char* tile[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) tile[j] = a.packed + (int64_t)min((int)blockIdx.x * RT + j, a.shape.tiles - 1) * a.shape.tile_bytes;
  cf32x4 acc[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) acc[j] = cf32x4{0.f, 0.f, 0.f, 0.f};
  const int b0 = (int)((int64_t)a.shape.blocks * wave / waves), b1 = (int)((int64_t)a.shape.blocks * (wave + 1) / waves);
  direct_product<FMT, RT, FMT == CS_WEIGHTS_E2M1 ? 4 / RT : 2 / RT>(acc, tile, a.shape.blocks, a.shape.k, b0, b1, a.x + (live ? t : 0) * a.x_row + 8 * g, live, lane);
#pragma unroll
  for (int j = 0; j < RT; ++j) part[wave][j][lane] = acc[j];
  __syncthreads();
  if (wave >= RT) return;
  cf32x4 v = part[0][wave][lane];
  for (int w = 1; w < waves; ++w) v += part[w][wave][lane];
  const int n = (blockIdx.x * RT + wave) * 16 + 4 * g, left = a.shape.n - n;
  if (live && left > 0) store4<BF16>(a.out, t * a.out_row + n, v + bias4(a.bias, n, a.shape.n), left, whole_rows && left >= 4);
}

// ---- more rows: four waves share the rows' operands in LDS, chunks of NB blocks along k, each asked for while the one before is used,
// and each wave has RT tiles of the weights (and, WM > 1, every WM-th part of the rows).  A chunk's rows lie as the lanes take them: piece (tile of 16
// rows, step) is 1 KB in lane order, written and read without conflicts.
template <int FMT, int MT, int WM, int RT, int NB>
struct Staged {
  static constexpr int MTW = MT / WM;                  // tiles of rows of a wave
  static constexpr int UNITS = MT * NB * 4;            // pieces of a chunk
  static constexpr int PER_WAVE = (UNITS + 3) / 4;
  static constexpr int LDS = 2 * UNITS * 1024;

  // off: the lane's byte offset from x of (row, 8 (lane / 16)) in tile m of its turn; loads of chunk c
  template <class Off>
  static __device__ __forceinline__ void stage(const bf16_t* x, Off&& off, int c, int last_step, unsigned char* lds, int wave) {
#ifdef __HIP_DEVICE_COMPILE__   // (the builtin's resource type does not exist in the host pass)
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(x), 0, 0xFFFFFFFFu, 0x00020000);
#pragma unroll
    for (int i = 0; i < PER_WAVE; ++i) {
      const int u = i * 4 + wave;                      // step u / MT of the chunk, tile u % MT
      const int step = c * NB * 4 + u / MT;
      if (u < UNITS && step < last_step)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (plds_void*)(uintptr_t)(lds + u * 1024), 16, off(u % MT) + (uint32_t)step * 64, 0, 0, 0);
    }
#endif
  }

  // acc[j][m] += blocks [b0, b1) of tile[j] times tile m of the wave's rows.  All waves of the workgroup call it alike.
  template <class Off>
  static __device__ __forceinline__ void product(cf32x4 (&acc)[RT][MTW], const unsigned char* const (&tile)[RT], int blocks, int k, int b0, int b1,
                                                 const bf16_t* x, Off&& off, unsigned char* lds, int lane, int wave, int wm) {
    const int chunks = (b1 - b0 + NB - 1) / NB, last_step = min(4 * b1, k / 32);
    const int c_full = (last_step / 4 - b0) / NB;      // chunks that have all their steps
    Held<FMT> cur[RT][NB], next[RT][NB];
    auto weights = [&](Held<FMT> (&w)[RT][NB], int c) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int b = b0 + c * NB + i;
        if (b < b1) {
          const int steps = min(4, k / 32 - 4 * b);
#pragma unroll
          for (int j = 0; j < RT; ++j) w[j][i].load(tile[j], blocks, b, lane, steps);
        }
      }
    };
    // (pieces count steps from b0)
    const bf16_t* xs = x + (int64_t)b0 * 128;
    const int steps_here = last_step - 4 * b0;
    if (chunks > 0) {
      stage(xs, off, 0, steps_here, lds, wave);
      weights(cur, 0);
    }
    for (int c = 0; c < chunks; ++c) {
      const unsigned char* from = lds + (c & 1) * UNITS * 1024 + wm * MTW * 1024 + lane * 16;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's pieces of the chunk, and its weights
      __syncthreads();                                   // everyone's; and nobody reads the other half any more
      if (c + 1 < chunks) {
        stage(xs, off, c + 1, steps_here, lds + (~c & 1) * UNITS * 1024, wave);
        weights(next, c + 1);
      }
      auto use = [&](int i, auto t) {
        constexpr int S = decltype(t)::value;
        pbf16x8 f[MTW];
#pragma unroll
        for (int m = 0; m < MTW; ++m) f[m] = *reinterpret_cast<const pbf16x8*>(from + ((i * 4 + S) * MT + m) * 1024);
#pragma unroll
        for (int j = 0; j < RT; ++j) {
          const pbf16x8 w = cur[j][i].template step<S>();
#pragma unroll
          for (int m = 0; m < MTW; ++m) acc[j][m] = mfma(w, f[m], acc[j][m]);
        }
      };
      if (c < c_full) {
#pragma unroll
        for (int i = 0; i < NB; ++i) all_steps([&](auto t) { use(i, t); });
      } else {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const int steps = min(4, steps_here - (c * NB + i) * 4);
          if (steps > 0) each_step(steps, [&](auto t) { use(i, t); });
        }
      }
#pragma unroll
      for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int i = 0; i < NB; ++i) cur[j][i] = next[j][i];
    }
  }
};

template <int FMT, int OUT, int MT, int WM, int RT, int NB>      // OUT: 0 fp32, 1 bf16, 2 a part of the sums
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 8))) void linear_staged_kernel(LinearArgs a, int whole_rows) {
  typedef Staged<FMT, MT, WM, RT, NB> P;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave % WM, wn = wave / WM;
  const int t = lane & 15, g = lane >> 4;
  // workgroups that read the same weights are eight apart: on one XCD, one behind the other
  const int per = 8 * a.m_tiles, group = blockIdx.x / per, in = blockIdx.x % per;
  const int n_block = group * 8 + in % 8, split = blockIdx.y;
  const int64_t m0 = (int64_t)(in / 8) * (MT * 16);
  const int tile0 = (n_block * (4 / WM) + wn) * RT;
  if ((n_block * (4 / WM)) * RT >= a.shape.tiles) return;          // (the whole workgroup)
  const unsigned char* tile[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) tile[j] = a.packed + (int64_t)min(tile0 + j, a.shape.tiles - 1) * a.shape.tile_bytes;
  const bf16_t* x = a.x + m0 * a.x_row;
  const int rows = (int)min((int64_t)(MT * 16), a.n_rows - m0);
  auto off = [&](int m) { return (uint32_t)((int64_t)min(m * 16 + t, rows - 1) * a.x_row * 2) + 16 * g; };
  cf32x4 acc[RT][P::MTW];
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int m = 0; m < P::MTW; ++m) acc[j][m] = cf32x4{0.f, 0.f, 0.f, 0.f};
  const int b0 = split * a.blocks_of_split, b1 = min(a.shape.blocks, b0 + a.blocks_of_split);
  P::product(acc, tile, a.shape.blocks, a.shape.k, b0, b1, x, off, lds, lane, wave, wm);
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    const int n = (tile0 + j) * 16 + 4 * g, left = a.shape.n - n;
    const cf32x4 bias = bias4(OUT == 2 ? nullptr : a.bias, n, a.shape.n);
#pragma unroll
    for (int m = 0; m < P::MTW; ++m) {
      const int r = (wm * P::MTW + m) * 16 + t;
      if (r >= rows || left <= 0) continue;
      if constexpr (OUT == 2) store4<false>(a.parts, ((int64_t)split * a.n_rows + m0 + r) * a.shape.n + n, acc[j][m], left, a.shape.n % 4 == 0);
      else store4<OUT == 1>(a.out, (m0 + r) * a.out_row + n, acc[j][m] + bias, left, whole_rows && left >= 4);
    }
  }
}

// out = the sum of the parts, in their order, and the bias
template <bool BF16>
__global__ __launch_bounds__(256) void linear_join_kernel(LinearArgs a) {
  const int64_t total = a.n_rows * a.shape.n;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / a.shape.n, n = i - t * a.shape.n;
    float v = a.parts[i];
    for (int s = 1; s < a.splits; ++s) v += a.parts[s * total + i];
    if (a.bias) v += a.bias[n];
    if constexpr (BF16) static_cast<bf16_t*>(a.out)[t * a.out_row + n] = (bf16_t)pack2_c(v, v);
    else static_cast<float*>(a.out)[t * a.out_row + n] = v;
  }
}

namespace {

constexpr int DIRECT_ROWS = 16;

struct LinearPlan {
  int mt, m_tiles, n_cols, splits, blocks_of_split;
};
LinearPlan linear_plan(const LinearArgs& a) {
  LinearPlan p = {};
  p.mt = a.n_rows <= 32 ? 2 : a.n_rows <= 64 ? 4 : 8;
  p.m_tiles = (int)((a.n_rows + p.mt * 16 - 1) / (p.mt * 16));
  p.n_cols = p.mt == 8 && a.shape.format == CS_WEIGHTS_BF16 ? 64 : 128;
  const int64_t groups = (int64_t)p.m_tiles * ((a.shape.n + p.n_cols - 1) / p.n_cols);
  // workgroups that fill the chip twice, unless a part would have fewer than eight blocks
  const int64_t want = std::max<int64_t>(1, (512 + groups / 2) / groups);
  p.splits = (int)std::min<int64_t>({want, std::max(1, a.shape.blocks / 8), 32});
  p.blocks_of_split = (a.shape.blocks + p.splits - 1) / p.splits;
  p.splits = (a.shape.blocks + p.blocks_of_split - 1) / p.blocks_of_split;
  return p;
}

template <int FMT, int OUT, int MT, int WM, int RT, int NB>
cs_status run_staged(const LinearArgs& a, int whole_rows, hipStream_t s) {
  constexpr int LDS = Staged<FMT, MT, WM, RT, NB>::LDS;
  const auto kernel = linear_staged_kernel<FMT, OUT, MT, WM, RT, NB>;
  if (LDS > 65536) CS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
  const int cols = (4 / WM) * RT * 16;
  const int64_t n_blocks = (a.shape.n + cols - 1) / cols, grid = (n_blocks + 7) / 8 * 8 * a.m_tiles;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid, (unsigned)a.splits), dim3(256), LDS, s, a, whole_rows);
  CS_HIP(hipGetLastError());
  return CS_OK;
}
template <int FMT, int OUT>
cs_status run_rows(const LinearArgs& a, int mt, int whole_rows, hipStream_t s) {
  if (mt == 2) return run_staged<FMT, OUT, 2, 1, 2, FMT == CS_WEIGHTS_E2M1 ? 4 : 2>(a, whole_rows, s);
  if (mt == 4) return run_staged<FMT, OUT, 4, 1, 2, FMT == CS_WEIGHTS_E2M1 ? 2 : 1>(a, whole_rows, s);
  // (bf16 weights of four tiles, this chunk's and the next one's, do not fit the registers)
  return run_staged<FMT, OUT, 8, 2, FMT == CS_WEIGHTS_E2M1 ? 4 : 2, 1>(a, whole_rows, s);
}
template <int FMT>
cs_status run_linear(LinearArgs a, int out_dtype, void* workspace, hipStream_t s) {
  const bool bf16 = out_dtype == CS_BF16;
  const int size = bf16 ? 2 : 4;
  const int whole = ((reinterpret_cast<uintptr_t>(a.out) | (uint64_t)(a.out_row * size)) & (4 * size - 1)) == 0;
  if (a.n_rows <= DIRECT_ROWS) {
    // waves that fill the chip: of the tiles' blocks, so many a workgroup
    const int tiles = a.shape.tiles, waves = (int)std::min<int64_t>({16, a.shape.blocks, std::max<int64_t>(1, (4096 + tiles / 2) / tiles)});
    if (bf16) hipLaunchKernelGGL((linear_direct_kernel<FMT, true, 1>), dim3(tiles), dim3(64 * waves), 0, s, a, whole);
    else hipLaunchKernelGGL((linear_direct_kernel<FMT, false, 1>), dim3(tiles), dim3(64 * waves), 0, s, a, whole);
    CS_HIP(hipGetLastError());
    return CS_OK;
  }
  const LinearPlan p = linear_plan(a);
  a.m_tiles = p.m_tiles;
  a.splits = p.splits;
  a.blocks_of_split = p.blocks_of_split;
  a.parts = static_cast<float*>(workspace);
  if (p.splits == 1) return bf16 ? run_rows<FMT, 1>(a, p.mt, whole, s) : run_rows<FMT, 0>(a, p.mt, whole, s);
  if (cs_status st = run_rows<FMT, 2>(a, p.mt, whole, s)) return st;
  const unsigned groups = (unsigned)std::min<int64_t>((a.n_rows * a.shape.n + 255) / 256, 4096);
  if (bf16) hipLaunchKernelGGL((linear_join_kernel<true>), dim3(groups), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((linear_join_kernel<false>), dim3(groups), dim3(256), 0, s, a);
  CS_HIP(hipGetLastError());
  return CS_OK;
}

}  // namespace

cs_status plan_linear_packed(const LinearArgs& a, size_t& bytes) {
  bytes = 0;
  if (a.n_rows <= DIRECT_ROWS) return CS_OK;
  const LinearPlan p = linear_plan(a);
  if ((int64_t)p.m_tiles * ((a.shape.n + 63) / 64 + 8) > 0xffffffffll / 256) return fail(CS_ERR_UNSUPPORTED, "cs_linear_packed: more workgroups than a grid has");
  if (p.splits > 1) bytes = (size_t)p.splits * a.n_rows * a.shape.n * 4;
  return CS_OK;
}
cs_status launch_linear_packed(const LinearArgs& a, int out_dtype, void* workspace, hipStream_t s) {
  return a.shape.format == CS_WEIGHTS_E2M1 ? run_linear<CS_WEIGHTS_E2M1>(a, out_dtype, workspace, s) : run_linear<CS_WEIGHTS_BF16>(a, out_dtype, workspace, s);
}

// ---- the mixture of experts

// Scores of TT rows by EE experts a wave, in fp64: products of two bf16 numbers are exact there and their sum is off by less than any two
// experts' scores that are not equal are likely to lie apart, so that the choice is that of the definition.  The vector unit's fp64 rate is half its
// fp32 rate.  Also clears the experts' counts for the launch behind.
template <int TT, int EE>
__global__ __launch_bounds__(256) void moe_logits_kernel(MoeArgs a) {
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int e = threadIdx.x; e < a.experts + a.shared; e += 256) a.counts[e] = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int e0 = ((int)blockIdx.x * 4 + wave) * EE;
  const int64_t t0 = (int64_t)blockIdx.y * TT;
  if (e0 >= a.experts) return;
  const bf16_t *x[TT], *w[EE];
#pragma unroll
  for (int i = 0; i < TT; ++i) x[i] = a.x + min(t0 + i, a.n_rows - 1) * a.x_row;
#pragma unroll
  for (int i = 0; i < EE; ++i) w[i] = a.router + (int64_t)min(e0 + i, a.experts - 1) * a.hidden;
  double sum[TT][EE];
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = 0; j < EE; ++j) sum[i][j] = 0;
  for (int k = lane * 8; k < a.hidden; k += 512) {
    float xs[TT][8], ws[EE][8];
#pragma unroll
    for (int i = 0; i < TT; ++i) load8<true, false>(x[i], k, xs[i]);
#pragma unroll
    for (int i = 0; i < EE; ++i) load8<true, false>(w[i], k, ws[i]);
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      double wd[EE];
#pragma unroll
      for (int j = 0; j < EE; ++j) wd[j] = ws[j][v];
#pragma unroll
      for (int i = 0; i < TT; ++i) {
        const double xd = xs[i][v];
#pragma unroll
        for (int j = 0; j < EE; ++j) sum[i][j] = fma(xd, wd[j], sum[i][j]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TT; ++i)
#pragma unroll
    for (int j = 0; j < EE; ++j) {
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) sum[i][j] += __shfl_xor(sum[i][j], m);
      if (lane == 0 && t0 + i < a.n_rows && e0 + j < a.experts) a.logits[(t0 + i) * a.experts + e0 + j] = sum[i][j];
    }
}

// a double as a number that orders the same way; a NaN below every number
__device__ __forceinline__ uint64_t order_of(double v) {
  if (v != v) return 0;
  v += 0.0;                              // (-0 and 0 are equal)
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return u >> 63 ? ~u : u | 1ull << 63;
}

__device__ __forceinline__ double block_reduce(double v, bool largest, double* shared) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const double o = __shfl_xor(v, m);
    v = largest ? fmax(v, o) : v + o;
  }
  const int waves = blockDim.x >> 6;
  if (waves > 1) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = shared[0];
    for (int w = 1; w < waves; ++w) v = largest ? fmax(v, shared[w]) : v + shared[w];
  }
  return v;
}

// A workgroup takes a row: an expert's place is the number of experts that come before it, counted against all of them at once.  Rows are entered in
// the lists of their experts in whatever order the workgroups come: a row's results do not depend on its place in them.
__global__ __launch_bounds__(256) void moe_select_kernel(MoeArgs a) {
  __shared__ uint64_t key[MAX_EXPERTS];
  __shared__ double score_of[MAX_TOP], shared[4];
  __shared__ int chosen[MAX_TOP];
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, threads = blockDim.x, E = a.experts;
  const bool live = !a.live || a.live[t];
  if (!live) {
    if (tid < a.top) {
      a.experts_out[t * a.top + tid] = -1;
      a.weights_out[t * a.top + tid] = 0.f;
    }
    return;
  }
  const double* logits = a.logits + t * E;
  double top = -__builtin_inf(), sum = 0;
  if (!a.sigmoid) {                      // (fmax passes over a NaN; the sum keeps it)
    for (int e = tid; e < E; e += threads) top = fmax(top, logits[e]);
    top = block_reduce(top, true, shared);
    for (int e = tid; e < E; e += threads) sum += exp(logits[e] - top);
    sum = block_reduce(sum, false, shared);
  }
  auto score = [&](int e) { return a.sigmoid ? 1 / (1 + exp(-logits[e])) : exp(logits[e] - top) / sum; };
  for (int e = tid; e < E; e += threads) key[e] = order_of(a.choice_bias ? score(e) + (double)a.choice_bias[e] : logits[e]);
  __syncthreads();
  for (int e = tid; e < E; e += threads) {
    const uint64_t mine = key[e];
    int place = 0;
    for (int o = 0; o < E; ++o) place += (key[o] > mine) | ((key[o] == mine) & (o < e));
    if (place < a.top) {
      chosen[place] = e;
      score_of[place] = score(e);
    }
  }
  __syncthreads();
  if (tid >= a.slots) return;
  const int64_t cells = t * a.slots + tid;
  int e = a.experts + tid - a.top;       // a shared one
  if (tid < a.top) {
    double all = 0;
    for (int i = 0; i < a.top; ++i) all += score_of[i];
    const double w = a.renormalise ? score_of[tid] / all : score_of[tid];
    e = chosen[tid];
    a.experts_out[t * a.top + tid] = e;
    a.weights_out[t * a.top + tid] = (float)(w * (double)a.scale);
  }
  a.lists[(int64_t)e * a.list_row + atomicAdd(a.counts + e, 1)] = (int32_t)cells;
}

// The experts' products, rows by their lists, in blocks of up to 64.  UP: tiles come in pairs, gate and up, and h = silu(gate) * up is
// written; else the parts of y.
template <int FMT, bool UP, int MT>
__device__ __forceinline__ void expert_rows(const MoeArgs& a, int e, int n_block, const int32_t* list, int rows, unsigned char* lds) {
  constexpr int RT = 2, NB = FMT == CS_WEIGHTS_E2M1 ? (MT == 1 ? 4 : 2) : (MT == 1 ? 2 : 1);
  typedef Staged<FMT, MT, 1, RT, NB> P;
  const PackedShape& shape = UP ? a.up_shape : a.down_shape;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, g = lane >> 4;
  const unsigned char* matrix = (UP ? a.up : a.down) + (int64_t)e * shape.tiles * shape.tile_bytes;
  const int pairs = a.inter / 16;                      // UP: tiles of gate, and of up
  const int at = n_block * 4 + wave;
  int tiles[2] = {min(at, pairs - 1), min(at, pairs - 1) + pairs};
  if constexpr (!UP) {
    tiles[0] = min(2 * at, shape.tiles - 1);
    tiles[1] = min(2 * at + 1, shape.tiles - 1);
  }
  const unsigned char* tile[RT] = {matrix + tiles[0] * shape.tile_bytes, matrix + tiles[1] * shape.tile_bytes};
  uint32_t offs[MT];
  int cell[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    cell[m] = list[min(m * 16 + t, rows - 1)];
    offs[m] = (UP ? (uint32_t)(cell[m] / a.slots) * (uint32_t)a.x_row : (uint32_t)cell[m] * (uint32_t)a.inter) * 2 + 16 * g;
  }
  auto off = [&](int m) {
    uint32_t o = offs[0];
#pragma unroll
    for (int i = 1; i < MT; ++i) o = m == i ? offs[i] : o;
    return o;
  };
  cf32x4 acc[RT][MT];
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[j][m] = cf32x4{0.f, 0.f, 0.f, 0.f};
  P::product(acc, tile, shape.blocks, shape.k, 0, shape.blocks, UP ? a.x : a.h, off, lds, lane, wave, 0);
  if constexpr (UP) {
    if (at < pairs) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
        if (m * 16 + t < rows) {
          cf32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = acc[0][m][i] / (1.f + __expf(-acc[0][m][i])) * acc[1][m][i];
          store4<true>(a.h, (int64_t)cell[m] * a.inter + at * 16 + 4 * g, v, 4, true);
        }
    }
  } else {
#pragma unroll
    for (int j = 0; j < RT; ++j)
      if (2 * at + j < shape.tiles) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
          if (m * 16 + t < rows) store4<false>(a.parts, (int64_t)cell[m] * a.hidden + (2 * at + j) * 16 + 4 * g, acc[j][m], 4, true);
      }
  }
}

template <int FMT, bool UP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 8))) void moe_experts_kernel(MoeArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int e = blockIdx.y, n_block = blockIdx.x;
  const int count = a.counts[e];
  for (int r = blockIdx.z * 64; r < count; r += gridDim.z * 64) {
    if (r >= (int)gridDim.z * 64) __syncthreads();     // (the rows before are still being read)
    const int rows = min(64, count - r);
    const int32_t* list = a.lists + (int64_t)e * a.list_row + r;
    if (rows <= 16) expert_rows<FMT, UP, 1>(a, e, n_block, list, rows, lds);
    else if (rows <= 32) expert_rows<FMT, UP, 2>(a, e, n_block, list, rows, lds);
    else if (rows <= 48) expert_rows<FMT, UP, 3>(a, e, n_block, list, rows, lds);
    else expert_rows<FMT, UP, 4>(a, e, n_block, list, rows, lds);
  }
}

// y of a row: its parts by their weights, in the order of the slots, in fp32
__global__ __launch_bounds__(256) void moe_sum_kernel(MoeArgs a) {
  const int64_t t = blockIdx.x;
  const bool live = !a.live || a.live[t];
  const float* w = a.weights_out + t * a.top;
  for (int n = ((int)blockIdx.y * 256 + threadIdx.x) * 8; n < a.hidden; n += (int)gridDim.y * 2048) {
    float v[8] = {};
    if (live) {
      for (int i = 0; i < a.slots; ++i) {
        float p[8];
        load8<false, false>(a.parts, (t * a.slots + i) * a.hidden + n, p);
        const float weight = i < a.top ? w[i] : 1.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(weight, p[j], v[j]);
      }
    }
    store8<true, false>(a.y, t * a.y_row + n, v);
  }
}

namespace {

// Rows of a call that go through the launches together: they bound the workspace, and the rows of h lie within 32-bit offsets
int64_t group_rows(const MoeArgs& a) {
  const int64_t most = std::min<int64_t>(MOE_ROWS, 0xffffffffll / (2ll * (a.top + a.shared) * a.inter));
  return std::min(a.n_rows, most);
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

template <int FMT>
cs_status run_moe(const MoeArgs& a, hipStream_t s) {
  const int T = (int)a.n_rows, all = a.experts + a.shared;
  if (T < 4) hipLaunchKernelGGL((moe_logits_kernel<1, 1>), dim3((a.experts + 3) / 4, T), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((moe_logits_kernel<4, 4>), dim3((a.experts + 15) / 16, (T + 3) / 4), dim3(256), 0, s, a);
  CS_HIP(hipGetLastError());
  hipLaunchKernelGGL(moe_select_kernel, dim3(T), dim3(std::max(64, std::min(256, (a.experts + 63) / 64 * 64))), 0, s, a);
  CS_HIP(hipGetLastError());
  // workgroups for twice the rows that an expert has on average; those with more take them in turn
  const int z = (int)std::max<int64_t>(1, std::min<int64_t>((T + 63) / 64, (2ll * T * a.top / a.experts + 63) / 64));
  const int up_lds = 65536;
  hipLaunchKernelGGL((moe_experts_kernel<FMT, true>), dim3((a.inter / 16 + 3) / 4, all, z), dim3(256), up_lds, s, a);
  CS_HIP(hipGetLastError());
  hipLaunchKernelGGL((moe_experts_kernel<FMT, false>), dim3((a.hidden / 16 + 7) / 8, all, z), dim3(256), up_lds, s, a);
  CS_HIP(hipGetLastError());
  hipLaunchKernelGGL(moe_sum_kernel, dim3(T, T > 1024 ? 1 : (a.hidden + 2047) / 2048), dim3(256), 0, s, a);
  CS_HIP(hipGetLastError());
  return CS_OK;
}

// lays the workspace of one group of rows out; returns its bytes
size_t moe_layout(MoeArgs& a, void* workspace) {
  const int64_t rows = group_rows(a);
  unsigned char* base = static_cast<unsigned char*>(workspace);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    unsigned char* p = base + at;
    at += up16(bytes);
    return p;
  };
  a.slots = a.top + a.shared;
  a.list_row = (int32_t)rows;
  a.logits = reinterpret_cast<double*>(take((size_t)rows * a.experts * 8));
  a.counts = reinterpret_cast<int32_t*>(take((size_t)(a.experts + a.shared) * 4));
  a.lists = reinterpret_cast<int32_t*>(take((size_t)(a.experts + a.shared) * rows * 4));
  a.h = reinterpret_cast<bf16_t*>(take((size_t)rows * a.slots * a.inter * 2));
  a.parts = reinterpret_cast<float*>(take((size_t)rows * a.slots * a.hidden * 4));
  return at;
}

}  // namespace

size_t moe_workspace(const MoeArgs& args) {
  MoeArgs a = args;
  return moe_layout(a, nullptr);
}
cs_status launch_moe(const MoeArgs& args, void* workspace, hipStream_t s) {
  MoeArgs a = args;
  moe_layout(a, workspace);
  const int64_t most = group_rows(args);
  for (int64_t first = 0; first < args.n_rows; first += most) {
    a.n_rows = std::min(args.n_rows - first, most);
    a.x = args.x + first * args.x_row;
    a.y = args.y + first * args.y_row;
    a.live = args.live ? args.live + first : nullptr;
    a.experts_out = args.experts_out + first * args.top;
    a.weights_out = args.weights_out + first * args.top;
    if (cs_status st = a.up_shape.format == CS_WEIGHTS_E2M1 ? run_moe<CS_WEIGHTS_E2M1>(a, s) : run_moe<CS_WEIGHTS_BF16>(a, s)) return st;
  }
  return CS_OK;
}

}  // namespace cs
