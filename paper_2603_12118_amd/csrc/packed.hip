// Products of rows with packed weights, and the experts of a mixture built on them.
//
// y^T = W x^T with v_mfma_f32_16x16x32_bf16: the weights are the first operand (a lane holds row l % 16, eight values along k), the rows
// the second (a lane holds row l % 16 of x, the same eight values of k), and a lane ends with four neighbouring columns of one row.
// Weights come from memory straight into the registers that hold the operand; 4-bit ones are widened there, exactly (a level times a power of two is a
// bf16 number), so no operand of theirs passes LDS.  They are read with plain loads: past the caches the scales, 64 bytes a block, fetched
// their lines twice (one row of 28672 x 3584, 55 MB: 15.1 us past them, 11.7 through them).
//
// What bounds the products: memory up to some 32 rows, with few rows the time that the first load takes; from there on the instructions of the loop, of
// which from 128 rows the matrix pipe's and the widening beside them are most.  Figures: loops of calls on three sets of weights, 4 bits unless said otherwise.
#include "block.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "rows.h"

namespace cs {

typedef __bf16 pbf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void plds_void;

constexpr uint32_t PAST = 0x80000000u;                 // bytes a resource may address: offsets of rows and tiles are below
#ifdef __HIP_DEVICE_COMPILE__   // (the builtins' resource type does not exist in the host pass)
typedef __amdgpu_buffer_rsrc_t Resource;
__device__ __forceinline__ Resource resource(const void* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, PAST, 0x00020000); }
// `at` a lane's, `all` every lane's: PAST puts a load behind the bound
__device__ __forceinline__ cu32x4 fetch16(Resource r, uint32_t at, uint32_t all) { return __builtin_bit_cast(cu32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, __builtin_amdgcn_readfirstlane(all), 0)); }
__device__ __forceinline__ uint32_t fetch4(Resource r, uint32_t at, uint32_t all) { return __builtin_amdgcn_raw_buffer_load_b32(r, at, __builtin_amdgcn_readfirstlane(all), 0); }
__device__ __forceinline__ void fetch_lds16(Resource r, uint32_t at, uint32_t all, unsigned char* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (plds_void*)(uintptr_t)lds, 16, at, __builtin_amdgcn_readfirstlane(all), 0, 0);
}
#else
struct Resource {};
__device__ Resource resource(const void* p);
__device__ cu32x4 fetch16(Resource r, uint32_t at, uint32_t all);
__device__ uint32_t fetch4(Resource r, uint32_t at, uint32_t all);
__device__ void fetch_lds16(Resource r, uint32_t at, uint32_t all, unsigned char* lds);
#endif

template <int FMT>
struct Held;                          // a block of a tile (16 rows, 128 values along k), as a lane holds it
template <>
struct Held<CS_WEIGHTS_E2M1> {
  cu32x4 codes;
  uint32_t scales;
  __device__ __forceinline__ void load(const unsigned char* tile, int blocks, int b, int lane, int) {
    codes = *reinterpret_cast<const cu32x4*>(tile + (int64_t)b * 1024 + lane * 16);
    scales = *reinterpret_cast<const uint32_t*>(tile + (int64_t)blocks * 1024 + b * 64 + (lane & 15) * 4);
  }
  // the same through a resource, of the tile at byte `from` of it; nothing where there are no steps
  __device__ __forceinline__ void fetch(Resource r, int blocks, int b, int lane, int steps, uint32_t from = 0) {
    codes = fetch16(r, lane * 16, steps > 0 ? from + (uint32_t)b * 1024 : PAST);
    scales = fetch4(r, (lane & 15) * 4, steps > 0 ? from + (uint32_t)blocks * 1024 + (uint32_t)b * 64 : PAST);
  }
  __device__ __forceinline__ pbf16x8 at(int s) const {      // s: known when compiled
    return s == 0 ? step<0>() : s == 1 ? step<1>() : s == 2 ? step<2>() : step<3>();
  }
  __device__ __forceinline__ void cut(int) {}               // (codes are finite: times zeros they are zeros)
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
    for (int s = 0; s < 4; ++s)             // (a step that is not there: the one before, used with zeros)
      v[s] = *reinterpret_cast<const cu32x4*>(tile + (int64_t)b * 4096 + min(s, steps - 1) * 1024 + lane * 16);
  }
  __device__ __forceinline__ void fetch(Resource r, int, int b, int lane, int steps, uint32_t from = 0) {
#pragma unroll
    for (int s = 0; s < 4; ++s) v[s] = fetch16(r, lane * 16, s < steps ? from + (uint32_t)(b * 4096 + s * 1024) : PAST);
  }
  __device__ __forceinline__ pbf16x8 at(int s) const { return __builtin_bit_cast(pbf16x8, v[s]); }
  // as if the steps from `steps` on were zeros (an infinity among what stands in their place would make a NaN)
  __device__ __forceinline__ void cut(int steps) {
#pragma unroll
    for (int s = 0; s < 4; ++s)
      if (s >= steps) v[s] = cu32x4{0, 0, 0, 0};
  }
  template <int S>
  __device__ __forceinline__ pbf16x8 step() const { return __builtin_bit_cast(pbf16x8, v[S]); }
};

template <int S>
struct step_tag { static constexpr int value = S; };
template <class F>
__device__ __forceinline__ void all_steps(F&& f) {
  f(step_tag<0>());
  f(step_tag<1>());
  f(step_tag<2>());
  f(step_tag<3>());
}

__device__ __forceinline__ cf32x4 mfma(pbf16x8 w, pbf16x8 x, cf32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0); }

// ---- up to 16 rows: no LDS on the way in, no barrier.  acc[j] += blocks [b0, b1) of tile j times x.  xl: the lane's row of x, at 8 (lane / 16); lanes
// without a row (!live) keep zeros and load nothing: lanes of different rows take an address each, and that is what more rows cost.  U blocks are
// asked for together; the last ones, fewer or with fewer steps, with clamped places and zeros for operands, since a branch between the loads
// and their use would have them wait in scratch memory.
template <int FMT, int RT, int U>
__device__ __forceinline__ void direct_product(cf32x4 (&acc)[RT], const unsigned char* const (&tile)[RT], int blocks, int k, int b0, int b1,
                                               const bf16_t* xl, bool live, int lane) {
  const int last = min(4 * b1, k / 32);       // steps
  auto group = [&](int b, auto whole) {
    constexpr bool WHOLE = decltype(whole)::value;
    Held<FMT> w[U][RT];
    cu32x4 x[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int bb = WHOLE ? b + u : min(b + u, b1 - 1);
#pragma unroll
      for (int j = 0; j < RT; ++j) w[u][j].load(tile[j], blocks, bb, lane, WHOLE ? 4 : min(4, last - 4 * bb));
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        x[u][s] = cu32x4{0, 0, 0, 0};
        if (live && (WHOLE || 4 * (b + u) + s < last)) x[u][s] = *reinterpret_cast<const cu32x4*>(xl + (int64_t)(b + u) * 128 + s * 32);
      }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (!WHOLE) {
#pragma unroll
        for (int j = 0; j < RT; ++j) w[u][j].cut(last - 4 * (b + u));
      }
      all_steps([&](auto t) {
        constexpr int S = decltype(t)::value;
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[j] = mfma(w[u][j].template step<S>(), __builtin_bit_cast(pbf16x8, x[u][S]), acc[j]);
      });
    }
  };
  int b = b0;
  for (; 4 * (b + U) <= last; b += U) group(b, std::true_type());
  if (b < b1) group(b, std::false_type());
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

// A workgroup takes RT tiles of the weights; its waves share out k and their sums are added in LDS, wave by wave.  14336 x 3584: 2 rows 7.9 us,
// 8 rows 8.8 (3.1 TB/s); 3584 x 3584 in bf16, 8 rows: 7.0 us (3.7 TB/s).
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
  direct_product<FMT, RT, 2>(acc, tile, a.shape.blocks, a.shape.k, b0, b1, a.x + (live ? t : 0) * a.x_row + 8 * g, live, lane);
#pragma unroll
  for (int j = 0; j < RT; ++j) part[wave][j][lane] = acc[j];
  __syncthreads();
  for (int j = wave; j < RT; j += waves) {
    cf32x4 v = part[0][j][lane];
    for (int w = 1; w < waves; ++w) v += part[w][j][lane];
    const int n = (blockIdx.x * RT + j) * 16 + 4 * g, left = a.shape.n - n;
    if (live && left > 0) store4<BF16>(a.out, t * a.out_row + n, v + bias4(a.bias, n, a.shape.n), left, whole_rows && left >= 4);
  }
}

// One row: a wave's part of it waits in LDS as the lanes take it, 16 bytes for each quarter, the same for all 16 columns of the product (of which one
// is used): no lane is masked and no operand cleared.  A wave writes and reads its own part only.  28672 x 3584: 10.9 us, 5.0 TB/s (masked lanes,
// as above: 12.4); reading the weights alone takes 8.2.  4608 x 3584: 4.2 us, a launch and two reads one behind the other.
template <int FMT, bool BF16>
__global__ __launch_bounds__(1024) void linear_row_kernel(LinearArgs a, int whole_rows) {
  constexpr int U = FMT == CS_WEIGHTS_E2M1 ? 4 : 2;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ cf32x4 part[16][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, g = lane >> 4;
  const unsigned char* tile = a.packed + (int64_t)blockIdx.x * a.shape.tile_bytes;
  const int blocks = a.shape.blocks, b0 = (int)((int64_t)blocks * wave / waves), b1 = (int)((int64_t)blocks * (wave + 1) / waves);
  for (int c = 16 * b0 + lane; c < 16 * b1; c += 64) {       // (asked for ahead of the weights: loads come back in order)
    cu32x4 v = {0, 0, 0, 0};
    if (8 * c < a.shape.k) v = *reinterpret_cast<const cu32x4*>(a.x + 8 * c);
    *reinterpret_cast<cu32x4*>(lds + 16 * c) = v;
  }
  cf32x4 acc = {0.f, 0.f, 0.f, 0.f};
  const int last = a.shape.k / 32;
  for (int b = b0; b < b1; b += U) {
    Held<FMT> w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int bb = min(b + u, b1 - 1);
      w[u].load(tile, blocks, bb, lane, min(4, last - 4 * bb));
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (b + u < b1) {
        w[u].cut(last - 4 * (b + u));
        all_steps([&](auto t) {
          constexpr int S = decltype(t)::value;
          acc = mfma(w[u].template step<S>(), *reinterpret_cast<const pbf16x8*>(lds + (b + u) * 256 + S * 64 + g * 16), acc);
        });
      }
  }
  part[wave][lane] = acc;
  __syncthreads();
  if (wave) return;
  for (int w = 1; w < waves; ++w) acc += part[w][lane];
  const int n = blockIdx.x * 16 + 4 * g, left = a.shape.n - n;
  if ((lane & 15) == 0 && left > 0) store4<BF16>(a.out, n, acc + bias4(a.bias, n, a.shape.n), left, whole_rows && left >= 4);
}

// The order of a step's instructions: the first tile widened, then products with the next tile's widening between them (a product keeps the
// matrix pipe for 16 cycles and the issue for four: what stands between two of them is done meanwhile, behind them it would be waited for)
template <int FMT, int RT, int MT>
__device__ __forceinline__ void interleave() {
  if constexpr (FMT == CS_WEIGHTS_E2M1) {
    __builtin_amdgcn_sched_group_barrier(0x100, MT, 0);            // reads of LDS
    __builtin_amdgcn_sched_group_barrier(0x2, 6, 0);               // VALU
#pragma unroll
    for (int i = 0; i < RT * MT; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);             // MFMA
      __builtin_amdgcn_sched_group_barrier(0x2, (6 * (RT - 1) + RT * MT - 1) / (RT * MT), 0);
    }
  }
}

// ---- more rows: four waves share the rows' operands in LDS, and each wave has RT tiles of the weights.  The rows come in stages of SS steps, NS of them in turn: while one is used, NS - 1 are on their way; the weights, which come from
// farther, are asked for WD blocks ahead, into registers.  A piece (step, tile of 16 rows) is 1 KB, 64 bytes a row, and neighbouring lanes ask for
// neighbouring 16 bytes of a row (lanes that ask for different rows take an address each: 16 bytes a clock, not 64).  The four
// chunks of row t lie turned by t / 2, so that eight rows of a chunk are read from different banks.
// Both are buffer loads with a bound: what lies behind the last step is asked for behind the bound, and is zeros that cost no memory.  So
// the number of loads under way is always the same, the waits are constants, and no step of the loop is conditional.
// 256 rows, 28672 x 3584 (52.6 GFLOP): 46 - 48 us on different cards, 1.1 PFLOP/s, where a library product of 8192^3 in bf16 reaches 1.21.  Of that: rows by an address
// a lane 62 us to 48; chunks turned by t / 4, which leaves two rows on a bank, 48 to 46; an exit between the blocks of a turn, for which the
// accumulators were kept twice, 59 to 54 with four tiles a wave.  The matrix pipe is busy for two fifths of the cycles, LDS for one.  Four tiles a wave and
// one wave a SIMD: 53; the rows shared out to two pairs of waves, which widen twice: 48.  64 rows 18.6 us, 45 rows 15.9, 32 rows 13.1 (4.3 TB/s); there the
// loop's instructions take what its reads do: with reads that bring zeros, 45 rows of 3584 x 14336 take 12.2 us of 13.3.
template <int FMT, int MT, int RT, int SS, int NS, int WD>
struct Staged {
  static constexpr int UNITS = MT * SS;                // pieces of a stage
  static constexpr int XL = (UNITS + 3) / 4;           // loads of a wave for a stage (a wave without a piece fetches one again)
  static constexpr int WL = RT * (FMT == CS_WEIGHTS_E2M1 ? 2 : 4);
  static constexpr int PB = 4 / SS;                    // stages of a block
  static_assert((SS == 2 || SS == 4) && WD <= 3, "what the loop is written for");
  static constexpr int LDS = NS * UNITS * 1024;

  // acc[j][m] += blocks [b0, b1) of tile[j] times tile m of the rows.  All waves of the workgroup call it alike.
  // off(m): the byte offset from x of row lane / 4 of tile m.
  template <class Off>
  static __device__ __forceinline__ void product(cf32x4 (&acc)[RT][MT], const unsigned char* const (&tile)[RT], int blocks, int k, int b0, int b1,
                                                 const bf16_t* x, Off&& off, unsigned char* lds, int lane, int wave) {
    const int last = min(4 * b1, k / 32);              // steps
    const Resource rx = resource(x);
    Resource rw[RT];
#pragma unroll
    for (int j = 0; j < RT; ++j) rw[j] = resource(tile[j]);
    Held<FMT> w[WD + 1][RT];
    auto weights = [&](Held<FMT> (&h)[RT], int b) {
#pragma unroll
      for (int j = 0; j < RT; ++j) h[j].fetch(rw[j], blocks, b, lane, b < b1 ? last - 4 * b : 0);
    };
#pragma unroll
    for (int i = 0; i < WD; ++i) weights(w[i], b0 + i);
    uint32_t offs[XL];                                 // (behind the weights: off may read memory)
    int place[XL];
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      int u = i * 4 + wave;                            // step u / MT of the stage, tile u % MT
      u = u < UNITS ? u : UNITS - 1;
      offs[i] = off(u % MT) + (((lane & 3) ^ ((lane >> 3) & 3)) << 4);
      place[i] = u;
    }
    auto stage = [&](int first, int slot) {            // the stage from step `first` on, into the slot
#pragma unroll
      for (int i = 0; i < XL; ++i) {
        const int step = first + place[i] / MT;
        fetch_lds16(rx, offs[i], step < last ? (uint32_t)step * 64 : PAST, lds + (slot * UNITS + place[i]) * 1024);
      }
    };
#pragma unroll
    for (int i = 0; i < NS - 1; ++i) stage(4 * b0 + i * SS, i);
    __builtin_amdgcn_s_waitcnt(0x0f70);                // vmcnt(0): all of them, so that the first turns' waits, which count more loads behind, are enough
    int slot = 0, b = b0;
    const unsigned char* mine = lds + (lane & 15) * 64 + (((lane >> 4) ^ ((lane >> 1) & 3)) << 4);
    auto block = [&](auto turn) {
      constexpr int R = decltype(turn)::value;
#pragma unroll
      for (int i = 0; i < PB; ++i) {
        wait_for_stage(i);
        __builtin_amdgcn_s_barrier();                  // everyone's pieces are there, and nobody reads the slot before this one any more
        asm volatile("" ::: "memory");
        stage(4 * b + (i + NS - 1) * SS, slot == 0 ? NS - 1 : slot - 1);
        __builtin_amdgcn_sched_barrier(0);             // (the waits count the weights behind the rows)
        if (i == 0) weights(w[(R + WD) % (WD + 1)], b + WD);
        const unsigned char* from = mine + slot * (UNITS * 1024);
        pbf16x8 f[2][MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) f[0][m] = *reinterpret_cast<const pbf16x8*>(from + m * 1024);
#pragma unroll
        for (int t = 0; t < SS; ++t) {
          if (t + 1 < SS) {
#pragma unroll
            for (int m = 0; m < MT; ++m) f[(t + 1) & 1][m] = *reinterpret_cast<const pbf16x8*>(from + ((t + 1) * MT + m) * 1024);
          }
#pragma unroll
          for (int j = 0; j < RT; ++j) {
            const pbf16x8 v = w[R][j].at(i * SS + t);
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[j][m] = mfma(v, f[t & 1][m], acc[j][m]);
          }
          interleave<FMT, RT, MT>();
          __builtin_amdgcn_sched_barrier(0);           // (a step's operands are widened in it, not all at once ahead: registers)
        }
        slot = slot + 1 == NS ? 0 : slot + 1;
      }
      ++b;
    };
    while (b < b1) {                                    // (whole turns: a block behind the last one is zeros; an exit in between costs registers)
      block(step_tag<0>());
      if constexpr (WD >= 1) block(step_tag<1>());
      if constexpr (WD >= 2) block(step_tag<2>());
      if constexpr (WD >= 3) block(step_tag<3>());
    }
    // (the loads still under way write into LDS: they end before the workgroup's memory is another's, or is used again)
    __builtin_amdgcn_s_waitcnt(0x0f70);
  }

  // vmcnt and lgkmcnt(0): this wave's pieces of the stage have come, and what it read of the one before
  static __device__ __forceinline__ void wait_for_stage(int i) {
    // weights are asked for in a block's first stage, behind the rows of NS - 1 stages on
    constexpr auto behind = [](int at) {
      int n = (NS - 2) * XL;
      for (int s = 1; s < NS; ++s) n += ((at - s) % PB + PB) % PB == 0 ? WL : 0;
      return n < 63 ? n : 63;
    };
    constexpr auto code = [](int n) { return (n & 15) | (n >> 4) << 14 | 7 << 4; };
    if (PB == 1 || i == 0) __builtin_amdgcn_s_waitcnt(code(behind(0)));
    else __builtin_amdgcn_s_waitcnt(code(behind(1)));
  }
};

// The sums of 16 rows by a tile as a wave holds them, 1 KB: by their rows they would be written and read in pieces of 64 bytes (the call of 45 rows
// by 3584 x 14336, seven parts: 15.9 us to 14.4; 64 rows by 3584 x 3584, 13.3 to 11.1)
__device__ __forceinline__ cf32x4* part_of(const LinearArgs& a, int split, int m, int tile) {
  return reinterpret_cast<cf32x4*>(a.parts) + (((int64_t)split * ((a.n_rows + 15) / 16) + m) * a.shape.tiles + tile) * 64;
}

template <int FMT, int OUT, int MT, int RT, int SS, int NS, int WD>      // OUT: 0 fp32, 1 bf16, 2 a part of the sums
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 8))) void linear_staged_kernel(LinearArgs a, int whole_rows) {
  typedef Staged<FMT, MT, RT, SS, NS, WD> P;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = lane & 15, g = lane >> 4;
  // workgroups that read the same weights are eight apart: on one XCD, one behind the other
  const int per = 8 * a.m_tiles, group = blockIdx.x / per, in = blockIdx.x % per;
  const int n_block = group * 8 + in % 8, split = blockIdx.y;
  const int64_t m0 = (int64_t)(in / 8) * (MT * 16);
  const int tile0 = (n_block * 4 + wave) * RT;
  if (n_block * 4 * RT >= a.shape.tiles) return;          // (the whole workgroup)
  const unsigned char* tile[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) tile[j] = a.packed + (int64_t)min(tile0 + j, a.shape.tiles - 1) * a.shape.tile_bytes;
  const bf16_t* x = a.x + m0 * a.x_row;
  const int rows = (int)min((int64_t)(MT * 16), a.n_rows - m0);
  auto off = [&](int m) { return (uint32_t)((int64_t)min(m * 16 + (lane >> 2), rows - 1) * a.x_row * 2); };
  cf32x4 acc[RT][MT];
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[j][m] = cf32x4{0.f, 0.f, 0.f, 0.f};
  const int b0 = split * a.blocks_of_split, b1 = min(a.shape.blocks, b0 + a.blocks_of_split);
  P::product(acc, tile, a.shape.blocks, a.shape.k, b0, b1, x, off, lds, lane, wave);
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    const int n = (tile0 + j) * 16 + 4 * g, left = a.shape.n - n;
    const cf32x4 bias = bias4(OUT == 2 ? nullptr : a.bias, n, a.shape.n);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int r = m * 16 + t;
      if (r >= rows || left <= 0) continue;
      if constexpr (OUT == 2) part_of(a, split, (int)(m0 / 16) + m, tile0 + j)[lane] = acc[j][m];
      else store4<OUT == 1>(a.out, (m0 + r) * a.out_row + n, acc[j][m] + bias, left, whole_rows && left >= 4);
    }
  }
}

// out = the sum of the parts, in their order, and the bias: a wave takes 16 rows by a tile, up to eight parts asked for together.  45 rows of 3584, seven
// parts: 3.5 - 4.0 us behind 12.5 for the parts.
template <bool BF16>
__global__ __launch_bounds__(256) void linear_join_kernel(LinearArgs a, int whole_rows) {
  const int lane = threadIdx.x & 63, tile = (int)blockIdx.x * 4 + (threadIdx.x >> 6), m = blockIdx.y;
  const int64_t t = (int64_t)m * 16 + (lane & 15);
  const int n = tile * 16 + 4 * (lane >> 4), left = a.shape.n - n;
  if (left <= 0 || t >= a.n_rows) return;
  const cf32x4 bias = bias4(a.bias, n, a.shape.n);
  cf32x4 v = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.splits; s0 += 8) {
    cf32x4 p[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) p[s] = part_of(a, min(s0 + s, a.splits - 1), m, tile)[lane];
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s0 + s < a.splits) v += p[s];
  }
  store4<BF16>(a.out, t * a.out_row + n, v + bias, left, whole_rows && left >= 4);
}

namespace {

constexpr int DIRECT_ROWS = 16;        // at most

struct LinearPlan {
  int mt, m_tiles, splits, blocks_of_split;
};
LinearPlan linear_plan(const LinearArgs& a) {
  LinearPlan p = {};
  p.mt = a.n_rows <= 16 ? 1 : a.n_rows <= 32 ? 2 : a.n_rows <= 48 ? 3 : a.n_rows <= 64 ? 4 : 8;
  p.m_tiles = (int)((a.n_rows + p.mt * 16 - 1) / (p.mt * 16));
  const int64_t groups = (int64_t)p.m_tiles * ((a.shape.n + 127) / 128);
  // A workgroup for each CU, in whole turns of four blocks (45 rows, 3584 x 14336: 7 parts of 16 blocks 14.5 us, 6 of 20 15.5, 10 of 12 17.2, 14 of 8 16.4; a part more
  // costs its writing and reading, one less the time that a wave alone on its SIMD takes for a block)
  const int want = (int)std::max<int64_t>(1, 256 / groups), blocks = a.shape.blocks;
  p.blocks_of_split = std::min(blocks, ((blocks + want - 1) / want + 3) / 4 * 4);
  p.splits = (blocks + p.blocks_of_split - 1) / p.blocks_of_split;
  return p;
}

// Tiles that a workgroup of linear_direct_kernel takes: two (rows of x are then read once for both) where that leaves workgroups for half of the chip (16
// rows by one / two tiles, us: 4608 x 3584 9.2 / 6.4, 3584 x 14336 16 / 17).  bf16 weights, which are four times the bytes and need the registers: one
// (8 rows of 28672 x 3584: 39 / 41).
int direct_tiles(const PackedShape& shape) { return shape.format == CS_WEIGHTS_BF16 || shape.tiles < 256 ? 1 : 2; }
// Up to 16 rows go straight from memory where k would be split and a CU's workgroups read up to some 100 000 numbers of x between them: below that the joining
// launch costs more than these reads (straight and staged, us: 14336 x 3584, 8 rows 8.8 and 10.6, 16 rows 11.0 and 11.2; 3584 x 14336, 4 rows 10.2
// and 10.8, 16 rows 16.8 and 11.0; 1024 x 8192, 8 rows 7.6 and 8.7, 16 rows 10.2 and 8.8).  Where k is not split, staged is as fast from two rows on (28672 x
// 3584, 2 rows 11.5 and 10.6, 16 rows 14.6 and 10.9; 512 x 512 5.2 and 4.6).  bf16 weights the same, but that staged workgroups beyond one a CU
// read in too many places at once (100000 x 2048, 2 / 8 / 16 rows 69 / 73 / 90 and 87 / 89 / 90; 28672 x 3584, 16 rows 48.6 and 35.9).
bool is_direct(const LinearArgs& a, const LinearPlan& staged) {
  if (a.n_rows == 1 || a.n_rows > DIRECT_ROWS) return a.n_rows == 1;
  const int tiles = direct_tiles(a.shape);
  const double read = (double)a.n_rows * a.shape.k * std::max(1., (a.shape.tiles + tiles - 1) / tiles / 256.);
  if (a.shape.format == CS_WEIGHTS_BF16) return read <= 100e3 * std::max(1., a.shape.tiles / 1024.);
  return staged.splits > 1 && read <= 100e3;
}

template <int FMT, int OUT, int MT, int RT, int SS, int NS, int WD>
cs_status run_staged(const LinearArgs& a, int whole_rows, hipStream_t s) {
  constexpr int LDS = Staged<FMT, MT, RT, SS, NS, WD>::LDS;
  const auto kernel = linear_staged_kernel<FMT, OUT, MT, RT, SS, NS, WD>;
  static_assert(LDS <= 65536, "what a launch may have unasked");
  const int cols = 4 * RT * 16;
  const int64_t n_blocks = (a.shape.n + cols - 1) / cols, grid = (n_blocks + 7) / 8 * 8 * a.m_tiles;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid, (unsigned)a.splits), dim3(256), LDS, s, a, whole_rows);
  CS_HIP(hipGetLastError());
  return CS_OK;
}
template <int FMT, int OUT>
cs_status run_rows(const LinearArgs& a, int mt, int whole_rows, hipStream_t s) {
  constexpr int WD = FMT == CS_WEIGHTS_E2M1 ? 3 : 1;         // (bf16 weights are four times the registers)
  if (mt == 1) return run_staged<FMT, OUT, 1, 2, 4, 4, WD>(a, whole_rows, s);
  if (mt == 2) return run_staged<FMT, OUT, 2, 2, 4, 4, WD>(a, whole_rows, s);
  if (mt == 3) return run_staged<FMT, OUT, 3, 2, 4, 4, WD>(a, whole_rows, s);
  if (mt == 4) return run_staged<FMT, OUT, 4, 2, 4, 3, 1>(a, whole_rows, s);
  return run_staged<FMT, OUT, 8, 2, 2, 4, 1>(a, whole_rows, s);
}
// Waves of about four blocks each.
template <int FMT, bool BF16>
cs_status run_direct(const LinearArgs& a, int whole_rows, hipStream_t s) {
  const int tiles = a.shape.tiles, blocks = a.shape.blocks;
  const int waves = std::min({16, blocks, (blocks + 3) / 4});
  if (a.n_rows == 1 && blocks <= 160) {                      // (40 KB of LDS for the row, beside 16)
    hipLaunchKernelGGL((linear_row_kernel<FMT, BF16>), dim3(tiles), dim3(64 * waves), (size_t)blocks * 256, s, a, whole_rows);
  } else if (FMT == CS_WEIGHTS_E2M1 && direct_tiles(a.shape) == 2) {
    constexpr int TWO = FMT == CS_WEIGHTS_E2M1 ? 2 : 1;
    hipLaunchKernelGGL((linear_direct_kernel<FMT, BF16, TWO>), dim3((tiles + 1) / 2), dim3(64 * waves), 0, s, a, whole_rows);
  } else {
    hipLaunchKernelGGL((linear_direct_kernel<FMT, BF16, 1>), dim3(tiles), dim3(64 * waves), 0, s, a, whole_rows);
  }
  CS_HIP(hipGetLastError());
  return CS_OK;
}
template <int FMT>
cs_status run_linear(LinearArgs a, int out_dtype, void* workspace, hipStream_t s) {
  const bool bf16 = out_dtype == CS_BF16;
  const int size = bf16 ? 2 : 4;
  const int whole = ((reinterpret_cast<uintptr_t>(a.out) | (uint64_t)(a.out_row * size)) & (4 * size - 1)) == 0;
  const LinearPlan p = linear_plan(a);
  if (is_direct(a, p)) return bf16 ? run_direct<FMT, true>(a, whole, s) : run_direct<FMT, false>(a, whole, s);
  a.m_tiles = p.m_tiles;
  a.splits = p.splits;
  a.blocks_of_split = p.blocks_of_split;
  a.parts = static_cast<float*>(workspace);
  if (p.splits == 1) return bf16 ? run_rows<FMT, 1>(a, p.mt, whole, s) : run_rows<FMT, 0>(a, p.mt, whole, s);
  if (cs_status st = run_rows<FMT, 2>(a, p.mt, whole, s)) return st;
  const dim3 groups((unsigned)((a.shape.tiles + 3) / 4), (unsigned)((a.n_rows + 15) / 16));
  if (bf16) hipLaunchKernelGGL((linear_join_kernel<true>), groups, dim3(256), 0, s, a, whole);
  else hipLaunchKernelGGL((linear_join_kernel<false>), groups, dim3(256), 0, s, a, whole);
  CS_HIP(hipGetLastError());
  return CS_OK;
}

}  // namespace

cs_status plan_linear_packed(const LinearArgs& a, size_t& bytes) {
  bytes = 0;
  const LinearPlan p = linear_plan(a);
  if (is_direct(a, p)) return CS_OK;
  if ((int64_t)p.m_tiles * ((a.shape.n + 63) / 64 + 8) > 0xffffffffll / 256) return fail(CS_ERR_UNSUPPORTED, "cs_linear_packed: more workgroups than a grid has");
  if (p.splits > 1) bytes = (size_t)p.splits * ((a.n_rows + 15) / 16) * a.shape.tiles * 1024;
  return CS_OK;
}
cs_status launch_linear_packed(const LinearArgs& a, int out_dtype, void* workspace, hipStream_t s) {
  return a.shape.format == CS_WEIGHTS_E2M1 ? run_linear<CS_WEIGHTS_E2M1>(a, out_dtype, workspace, s) : run_linear<CS_WEIGHTS_BF16>(a, out_dtype, workspace, s);
}

// ---- the mixture of experts

// Numbers between the experts' counts: a line each, since the adds to one line go one behind the other
constexpr int COUNT_APART = 16;

// Scores in fp64: products of two bf16 numbers are exact there and their sum is off by less than any two experts' scores that are not equal
// are likely to lie apart, so that the choice is that of the definition; in fp32 two neighbours would change places in one row of some thousands.
// Also clears the experts' counts for the launch behind.
// A workgroup takes an expert and TT rows, its waves pieces of 512 values of k in turn.  One row by 128 experts of 2048: 2.7 us, a launch and a read; 48
// rows: 5.1 (a wave for four rows and four experts over all of k: 9.6).
template <int TT>
__global__ __launch_bounds__(256) void moe_logits_kernel(MoeArgs a) {
  __shared__ double part[4][TT];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x;
  const int64_t t0 = (int64_t)blockIdx.y * TT;
  if (e == 0 && blockIdx.y == 0)
    for (int i = threadIdx.x; i < a.experts + a.shared; i += 256) a.counts[i * COUNT_APART] = 0;
  const bf16_t *x[TT], *w = a.router + (int64_t)e * a.hidden;
#pragma unroll
  for (int i = 0; i < TT; ++i) x[i] = a.x + min(t0 + i, a.n_rows - 1) * a.x_row;
  double sum[TT] = {};
  for (int k = (wave * 64 + lane) * 8; k < a.hidden; k += 2048) {
    float xs[TT][8], ws[8];
    load8<true, false>(w, k, ws);
#pragma unroll
    for (int i = 0; i < TT; ++i) load8<true, false>(x[i], k, xs[i]);
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      const double wd = ws[v];
#pragma unroll
      for (int i = 0; i < TT; ++i) sum[i] = fma((double)xs[i][v], wd, sum[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < TT; ++i) {
    sum[i] = wave_sum(sum[i]);
    if (lane == 0) part[wave][i] = sum[i];
  }
  __syncthreads();
  const int i = threadIdx.x;
  if (i < TT && t0 + i < a.n_rows) a.logits[(t0 + i) * a.experts + e] = part[0][i] + part[1][i] + part[2][i] + part[3][i];
}

// The same for many rows, 16 of them by 16 experts a workgroup, its 16 waves sharing out k: v_mfma_f64_16x16x4_f64, whose operands a lane
// widens once for 16 products each.  512 rows by 128 experts of 2048: 9.5 us, 3.4 of them the matrix pipe's (64 cycles each); four waves, four reads one
// behind the other: 13; on the vector unit, where widening takes longer than the products, 16.
typedef double pf64x4 __attribute__((ext_vector_type(4)));
__global__ __launch_bounds__(1024) void moe_logits_tile_kernel(MoeArgs a) {
  __shared__ double part[16][4][64];
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int e = threadIdx.x; e < a.experts + a.shared; e += 1024) a.counts[e * COUNT_APART] = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int64_t t0 = (int64_t)blockIdx.y * 16;
  const int e0 = blockIdx.x * 16;
  const bf16_t* x = a.x + min(t0 + r, a.n_rows - 1) * a.x_row + 8 * g;
  const bf16_t* w = a.router + (int64_t)min(e0 + r, a.experts - 1) * a.hidden + 8 * g;
  const int steps = a.hidden / 32, s0 = steps * wave / 16, s1 = steps * (wave + 1) / 16;
  pf64x4 acc = {0, 0, 0, 0};
  constexpr int U = 4;
  for (int s = s0; s < s1; s += U) {
    float xs[U][8], ws[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      load8<true, false>(x, (int64_t)min(s + u, s1 - 1) * 32, xs[u]);
      load8<true, false>(w, (int64_t)min(s + u, s1 - 1) * 32, ws[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (s + u < s1) {
#pragma unroll
        for (int v = 0; v < 8; ++v) acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)xs[u][v], (double)ws[u][v], acc, 0, 0, 0);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) part[wave][i][lane] = acc[i];
  __syncthreads();
  if (wave >= 4) return;
  // wave i has rows 4 i + lane / 16: that is how the products lie
  double v = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) v += part[i][wave][lane];
  const int64_t t = t0 + 4 * wave + g;
  if (t < a.n_rows && e0 + r < a.experts) a.logits[t * a.experts + e0 + r] = v;
}

// a double as a number that orders the same way; a NaN below every number
__device__ __forceinline__ uint64_t order_of(double v) {
  if (v != v) return 0;
  v += 0.0;                              // (-0 and 0 are equal)
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  return u >> 63 ? ~u : u | 1ull << 63;
}

__device__ __forceinline__ double block_sum(double v, double* shared) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  return shared[0] + shared[1] + shared[2] + shared[3];
}
__device__ __forceinline__ double block_max(double v, double* shared) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) v = fmax(v, __shfl_xor(v, m));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmax(fmax(shared[0], shared[1]), fmax(shared[2], shared[3]));
}

// The experts of a row, found by a workgroup of 256: an expert's place is the number of experts that come before it, counted against all of
// them, the threads that an expert has to spare sharing them out.  The upper halves of the keys are compared, four at a time; the whole
// ones only where another's upper half is the same.  Where weights are asked for, thread i < top returns that of the i-th.
struct Choice {
  uint64_t key[MAX_EXPERTS];
  __attribute__((aligned(16))) uint32_t upper[MAX_EXPERTS + 32];
  double logit[MAX_EXPERTS];
  double shared[4];
  int expert[MAX_TOP];
};
__device__ __forceinline__ float choose(const MoeArgs& a, int64_t t, Choice& c, bool weights) {
  const int tid = threadIdx.x, E = a.experts;
  // a softmax needs its sum only where the scores themselves count
  const bool plain = a.renormalise && !a.choice_bias;
  double top = -__builtin_inf(), sum = 1;
  bool nan = false;
  for (int e = tid; e < E; e += 256) {
    const double l = a.logits[t * E + e];
    c.logit[e] = l;
    nan |= l != l;
    top = fmax(top, l);                  // (passes over a NaN; the sum keeps it)
  }
  if (!a.sigmoid && !plain) {
    top = block_max(top, c.shared);
    sum = 0;
    for (int e = tid; e < E; e += 256) sum += exp(c.logit[e] - top);
    sum = block_sum(sum, c.shared);
  }
  auto score = [&](double logit) { return a.sigmoid ? 1 / (1 + exp(-logit)) : exp(logit - top) / sum; };
  for (int e = tid; e < E; e += 256) {
    const double l = c.logit[e];
    const uint64_t k = order_of(a.choice_bias ? score(l) + (double)a.choice_bias[e] : l);
    c.key[e] = k;
    c.upper[e] = (uint32_t)(k >> 32);
  }
  if (tid < 32) c.upper[E + tid] = 0;    // (before none)
  nan = __syncthreads_or(nan);
  const int shares = E > 128 ? 1 : E > 64 ? 2 : E > 32 ? 4 : 8, each = (E / shares + 4) & ~3;        // (shares * each > E - 1, within upper)
  const int first = tid % shares * each;
  for (int e0 = 0; e0 < E; e0 += 256 / shares) {
    const int e = e0 + tid / shares, in = min(e, E - 1);
    const uint32_t mine = c.upper[in];
    int before = 0, not_behind = 0;
#pragma unroll 4
    for (int o = first; o < first + each; o += 4) {
      const cu32x4 v = *reinterpret_cast<const cu32x4*>(c.upper + o);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        before += v[i] > mine;
        not_behind += v[i] >= mine;
      }
    }
    if (not_behind - before > (in >= first && in < first + each)) {
      const uint64_t key = c.key[in];
      before = 0;
      for (int o = first; o < min(E, first + each); ++o) before += (c.key[o] > key) | ((c.key[o] == key) & (o < in));
    }
    for (int m = 1; m < shares; m <<= 1) before += __shfl_xor(before, m);
    if (e < E && before < a.top && tid % shares == 0) c.expert[before] = e;
  }
  __syncthreads();
  if (!weights || tid >= 64) return 0.f;
  double w = 0;
  if (tid < a.top) {
    if (!a.sigmoid && plain) top = c.logit[c.expert[0]];
    w = nan && !a.sigmoid ? __builtin_nan("") : score(c.logit[c.expert[tid]]);
  }
  if (a.renormalise) w /= wave_sum(w);
  return (float)(w * (double)a.scale);
}

// A workgroup takes a row.  Rows are entered in the lists of their experts in whatever order the workgroups come: a row's results do
// not depend on its place in them.  48 rows of 128 experts 5.4 us, 512 rows 7.0: a launch, the scores, three barriers and the add's way there
// and back, one behind the other.  (Instead of the lists, a map of experts and rows that the products' workgroups search: no faster here, and those lost 3 to 6 us.)
__global__ __launch_bounds__(256) void moe_select_kernel(MoeArgs a) {
  __shared__ Choice c;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  if (a.live && !a.live[t]) {
    if (tid < a.top) {
      a.experts_out[t * a.top + tid] = -1;
      a.weights_out[t * a.top + tid] = 0.f;
    }
    return;
  }
  const float w = choose(a, t, c, true);
  if (tid >= a.slots) return;
  int e = a.experts + tid - a.top;       // a shared one
  if (tid < a.top) {
    e = c.expert[tid];
    a.experts_out[t * a.top + tid] = e;
    a.weights_out[t * a.top + tid] = w;
  }
  a.lists[(int64_t)e * a.list_row + atomicAdd(a.counts + e * COUNT_APART, 1)] = (int32_t)(t * a.slots + tid);
}

// silu(gate) up, fp32.  It is written in bf16, the type of the second products' operand, half a step of 2^-8 each: y is then off by 0.0023 - 0.0024 of
// its norm (one row to 512), where fp32 or two bf16 parts of it leave 0.0016 - 0.0017, y's own rounding.  Two parts would be twice the second products' matrix
// instructions and twice the rows that they read.
__device__ __forceinline__ cf32x4 gated(cf32x4 gate, cf32x4 up) {
  cf32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = gate[i] / (1.f + __expf(-gate[i])) * up[i];
  return v;
}

// Which rows of which expert a workgroup takes, `size` at a time: of its expert's list every gridDim.z-th block; the shared experts, which every row
// has, are given a workgroup for each block instead (entries of blockIdx.y behind the others').
struct Share {
  int e, first, stride;
};
__device__ __forceinline__ Share share_of(const MoeArgs& a, int size) {
  const int y = blockIdx.y, z = blockIdx.z;
  if (y < a.experts) return {y, z * size, (int)gridDim.z * size};
  const int blocks = ((int)a.n_rows + size - 1) / size, i = y - a.experts;
  return {a.experts + i / blocks, z ? 0x7fffffff - 64 : i % blocks * size, blocks * size};
}
// Entry r + lane of an expert's list (whatever lies there, where it has no more rows)
__device__ __forceinline__ int listed_row(const MoeArgs& a, int e, int r) {
  return a.lists[(int64_t)e * a.list_row + min(r + (int)(threadIdx.x & 63), a.list_row - 1)];
}
int share_rows(const MoeArgs& a, int size) { return a.experts + a.shared * (((int)a.n_rows + size - 1) / size); }

// ---- few rows an expert: 16 at a time, straight from memory (direct_product), a workgroup's waves sharing out k.
// UP: a workgroup takes PAIRS pairs of tiles, gate and up.  ONE: the call has one row, and every workgroup chooses its experts for itself, which
// is less than a launch.  8 rows, 16 experts and a shared one of 3584 x 1280 in bf16 (211 MB): 41 us, 5.1 TB/s; one row, 8 of 128 experts of 2048 x
// 768 (13 MB): 9 us, of which choosing is about half.
template <int FMT, bool ONE, int PAIRS>
__global__ __launch_bounds__(256) void moe_few_up_kernel(MoeArgs a) {
  struct Nothing {};
  __shared__ union {
    std::conditional_t<ONE, Choice, Nothing> c;
    cf32x4 part[4][2 * PAIRS][64];
  } s;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, g = lane >> 4;
  const Share share = ONE ? Share{0, 0, 16} : share_of(a, 16);
  int e = share.e, count = 1, cell = blockIdx.y;
  if constexpr (ONE) {
    const bool live = !a.live || a.live[0], writes = blockIdx.x == 0 && blockIdx.y == 0;
    const int slot = blockIdx.y;
    if (!live) {
      if (writes && threadIdx.x < a.top) {
        a.experts_out[threadIdx.x] = -1;
        a.weights_out[threadIdx.x] = 0.f;
      }
      return;
    }
    e = a.experts + slot - a.top;
    if (slot < a.top) {
      const float w = choose(a, 0, s.c, writes);
      e = __builtin_amdgcn_readfirstlane(s.c.expert[slot]);
      if (writes && threadIdx.x < a.top) {
        a.experts_out[threadIdx.x] = s.c.expert[threadIdx.x];
        a.weights_out[threadIdx.x] = w;
      }
      __syncthreads();                   // (what follows lies in the same place)
    }
  } else {
    cell = a.lists[(int64_t)e * a.list_row + min(share.first + t, a.list_row - 1)];      // (asked for with the count, used where there is a row)
    count = a.counts[e * COUNT_APART];
  }
  const PackedShape& shape = a.up_shape;
  const int pairs = a.inter / 16;
  const unsigned char* matrix = a.up + (int64_t)e * shape.tiles * shape.tile_bytes;
  const unsigned char* tile[2 * PAIRS];
#pragma unroll
  for (int j = 0; j < PAIRS; ++j) {
    const int pair = min((int)blockIdx.x * PAIRS + j, pairs - 1);
    tile[2 * j] = matrix + (int64_t)pair * shape.tile_bytes;
    tile[2 * j + 1] = matrix + (int64_t)(pair + pairs) * shape.tile_bytes;
  }
  const int b0 = shape.blocks * wave / 4, b1 = shape.blocks * (wave + 1) / 4;
  for (int r = share.first; r < count; r += share.stride) {
    if (r != share.first) __syncthreads();
    const bool live = r + t < count;
    if (r != share.first) cell = a.lists[(int64_t)e * a.list_row + min(r + t, count - 1)];
    cf32x4 acc[2 * PAIRS];
#pragma unroll
    for (int j = 0; j < 2 * PAIRS; ++j) acc[j] = cf32x4{0.f, 0.f, 0.f, 0.f};
    const int64_t row = ONE || !live ? 0 : cell / a.slots;
    direct_product<FMT, 2 * PAIRS, FMT == CS_WEIGHTS_E2M1 ? 2 : 1>(acc, tile, shape.blocks, shape.k, b0, b1, a.x + row * a.x_row + 8 * g, live, lane);
#pragma unroll
    for (int j = 0; j < 2 * PAIRS; ++j) s.part[wave][j][lane] = acc[j];
    __syncthreads();
    const int pair = (int)blockIdx.x * PAIRS + wave;
    if (wave < PAIRS && pair < pairs && live) {
      cf32x4 v[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) v[i] = s.part[0][2 * wave + i][lane] + s.part[1][2 * wave + i][lane] + s.part[2][2 * wave + i][lane] + s.part[3][2 * wave + i][lane];
      store4<true>(a.h, (int64_t)cell * a.inter + pair * 16 + 4 * g, gated(v[0], v[1]), 4, true);
    }
  }
}

// DOWN, rows by their lists, into the parts of y: a workgroup takes 2 RT tiles, two waves to each RT of them.
template <int FMT, int RT>
__global__ __launch_bounds__(256) void moe_few_down_kernel(MoeArgs a) {
  __shared__ cf32x4 part[2][RT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, g = lane >> 4;
  const Share share = share_of(a, 16);
  const int e = share.e, at = (blockIdx.x * 2 + wave / 2) * RT, half = wave & 1;
  int cell = a.lists[(int64_t)e * a.list_row + min(share.first + t, a.list_row - 1)];    // (asked for with the count, used where there is a row)
  const int count = a.counts[e * COUNT_APART];
  const PackedShape& shape = a.down_shape;
  const unsigned char* matrix = a.down + (int64_t)e * shape.tiles * shape.tile_bytes;
  const unsigned char* tile[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) tile[j] = matrix + (int64_t)min(at + j, shape.tiles - 1) * shape.tile_bytes;
  const int b0 = half ? shape.blocks / 2 : 0, b1 = half ? shape.blocks : shape.blocks / 2;
  for (int r = share.first; r < count; r += share.stride) {
    if (r != share.first) __syncthreads();
    const bool live = r + t < count;
    if (r != share.first) cell = a.lists[(int64_t)e * a.list_row + min(r + t, count - 1)];
    cf32x4 acc[RT];
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[j] = cf32x4{0.f, 0.f, 0.f, 0.f};
    direct_product<FMT, RT, FMT == CS_WEIGHTS_E2M1 ? 3 : 1>(acc, tile, shape.blocks, shape.k, b0, b1, a.h + (int64_t)(live ? cell : 0) * a.inter + 8 * g, live, lane);
    if (half) {
#pragma unroll
      for (int j = 0; j < RT; ++j) part[wave / 2][j][lane] = acc[j];
    }
    __syncthreads();
    if (!half && live) {
#pragma unroll
      for (int j = 0; j < RT; ++j)
        if (at + j < shape.tiles)
          store4<false>(a.parts, (int64_t)cell * a.hidden + (at + j) * 16 + 4 * g, acc[j] + part[wave / 2][j][lane], 4, true);
    }
  }
}

// DOWN of one row, the whole sum: a workgroup takes a tile of y, its waves a part along k of a slot's expert each.  8 experts of 768 x 2048 (7 MB): 4.7 us, a
// launch, the experts' numbers, the weights, one behind the other.
template <int FMT>
__global__ __launch_bounds__(1024) void moe_row_sum_kernel(MoeArgs a, int shares) {
  __shared__ cf32x4 part[16][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, g = lane >> 4;
  const PackedShape& shape = a.down_shape;
  cf32x4 sum = {0.f, 0.f, 0.f, 0.f};
  if (!a.live || a.live[0])
    for (int unit = wave; unit < a.slots * shares; unit += 16) {
      const int slot = unit / shares, at = unit - slot * shares;
      const int e = __builtin_amdgcn_readfirstlane(slot < a.top ? a.experts_out[slot] : a.experts + slot - a.top);
      const float w = slot < a.top ? a.weights_out[slot] : 1.f;
      const unsigned char* tile[1] = {a.down + ((int64_t)e * shape.tiles + blockIdx.x) * shape.tile_bytes};
      cf32x4 acc[1] = {{0.f, 0.f, 0.f, 0.f}};
      direct_product<FMT, 1, FMT == CS_WEIGHTS_E2M1 ? 3 : 2>(acc, tile, shape.blocks, shape.k, shape.blocks * at / shares, shape.blocks * (at + 1) / shares,
                                                            a.h + (int64_t)slot * a.inter + 8 * g, t == 0, lane);
      sum += w * acc[0];
    }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave || t) return;
  for (int w = 1; w < 16; ++w) sum += part[w][lane];
  store4<true>(a.y, blockIdx.x * 16 + 4 * g, sum, 4, true);
}

// DOWN of up to 16 rows, the whole sum: a workgroup takes a tile of y and all experts, its waves an expert (or, where there are fewer, a part of one
// along k) at a time.  A row that the expert was not chosen for has zeros as its operand; its weight multiplies the expert's sum, and the
// waves' sums are added in LDS, so nothing is written but y.  (Which wave has an expert depends on the others that have rows: so does the order of a row's sum.)  8 rows, 1280 x 3584 in bf16 (105 MB): 19 - 23 us, 4.6 - 5.5 TB/s.
template <int FMT>
__global__ __launch_bounds__(1024) void moe_few_sum_kernel(MoeArgs a, int shares) {
  __shared__ cf32x4 part[16][64];
  __shared__ __attribute__((aligned(16))) signed char slot_of[MAX_EXPERTS][16];       // by expert and row: the row's slot, or none
  __shared__ float weight[16][MAX_TOP];
  __shared__ int used[MAX_EXPERTS], n_used;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, g = lane >> 4;
  const int rows = (int)a.n_rows, top = a.top, E = a.experts;
  const bool is = t < rows && (!a.live || a.live[t < rows ? t : 0]);
  for (int i = threadIdx.x; i < 4 * E; i += 1024) reinterpret_cast<uint32_t*>(slot_of)[i] = 0xffffffffu;
  __syncthreads();
  for (int i = threadIdx.x; i < rows * top; i += 1024) {
    const int e = a.experts_out[i], r = i / top;
    weight[r][i - r * top] = a.weights_out[i];
    if (e >= 0) slot_of[e][r] = (signed char)(i - r * top);
  }
  __syncthreads();
  if (wave == 0) {                                       // the experts that rows have, in their order
    int n = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
      bool any = false;
      if (e0 + lane < E) {
        const cu32x4 v = *reinterpret_cast<const cu32x4*>(slot_of[e0 + lane]);
        any = (v[0] & v[1] & v[2] & v[3]) != 0xffffffffu;
      }
      const uint64_t m = __ballot(any);
      if (any) used[n + __popcll(m & ((1ull << lane) - 1))] = e0 + lane;
      n += __popcll(m);
    }
    if (lane == 0) n_used = n;
  }
  __syncthreads();
  const PackedShape& shape = a.down_shape;
  cf32x4 sum = {0.f, 0.f, 0.f, 0.f};
  const int units = (n_used + a.shared) * shares;
  for (int unit = wave; unit < units; unit += 16) {
    const int i = unit / shares, at = unit - i * shares, mine = n_used;
    int e = E + i - mine, slot = is ? top + i - mine : -1;
    float w = 1.f;
    if (i < mine) {
      e = __builtin_amdgcn_readfirstlane(used[i]);
      slot = slot_of[e][t];
      w = slot >= 0 ? weight[t][slot] : 0.f;
    }
    const bool live = slot >= 0;
    const unsigned char* tile[1] = {a.down + ((int64_t)e * shape.tiles + blockIdx.x) * shape.tile_bytes};
    const int b0 = shape.blocks * at / shares, b1 = shape.blocks * (at + 1) / shares;
    cf32x4 acc[1] = {{0.f, 0.f, 0.f, 0.f}};
    direct_product<FMT, 1, FMT == CS_WEIGHTS_E2M1 ? 3 : 2>(acc, tile, shape.blocks, shape.k, b0, b1,
                                                          a.h + ((int64_t)(live ? t : 0) * a.slots + (live ? slot : 0)) * a.inter + 8 * g, live, lane);
    if (live) sum += w * acc[0];
  }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave || t >= rows) return;
  for (int w = 1; w < 16; ++w) sum += part[w][lane];
  store4<true>(a.y, (int64_t)t * a.y_row + blockIdx.x * 16 + 4 * g, sum, 4, true);
}

// The experts' products, rows by their lists, in blocks of up to 64.  UP: tiles come in pairs, gate and up, and h = silu(gate) * up is
// written; else the parts of y.  128 experts of 2048 x 768 (214 MB), 48 rows: 36 us, 5.9 TB/s; 512 rows: 44 us, where the matrix pipe (30 k cycles a
// SIMD), widening and what an expert of 48 rows takes longer than one of 32 add up.  Two tiles a wave 52 us, the weights of three blocks ahead 47.
constexpr int EXPERT_LDS = 36864;
// byte offset of a listed row, of x (UP) or h
template <bool UP>
__device__ __forceinline__ uint32_t row_offset(const MoeArgs& a, int cell) {
  return (UP ? (uint32_t)(cell / a.slots) * (uint32_t)a.x_row : (uint32_t)cell * (uint32_t)a.inter) * 2;
}
template <int FMT, bool UP, int MT, int RT, int WD>
__device__ __forceinline__ void expert_rows(const MoeArgs& a, int e, int n_block, int listed, int rows, unsigned char* lds) {
  constexpr int SS = MT == 4 ? 2 : 4, NS = MT == 4 ? 4 : 3;
  typedef Staged<FMT, MT, RT, SS, NS, WD> P;
  static_assert(P::LDS <= EXPERT_LDS, "what the launch gives");
  const PackedShape& shape = UP ? a.up_shape : a.down_shape;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, g = lane >> 4;
  const unsigned char* matrix = (UP ? a.up : a.down) + (int64_t)e * shape.tiles * shape.tile_bytes;
  const int pairs = a.inter / 16, at = (n_block * 4 + wave) * (UP ? RT / 2 : RT);        // UP: pairs of tiles, gate and up
  const unsigned char* tile[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) tile[j] = matrix + (int64_t)(UP ? min(at + j / 2, pairs - 1) + j % 2 * pairs : min(at + j, shape.tiles - 1)) * shape.tile_bytes;
  int cell[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) cell[m] = __shfl(listed, min(m * 16 + t, rows - 1));
  auto off = [&](int m) { return row_offset<UP>(a, __shfl(listed, min(m * 16 + (lane >> 2), rows - 1))); };
  cf32x4 acc[RT][MT];
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[j][m] = cf32x4{0.f, 0.f, 0.f, 0.f};
  P::product(acc, tile, shape.blocks, shape.k, 0, shape.blocks, UP ? a.x : a.h, off, lds, lane, wave);
#pragma unroll
  for (int j = 0; j < (UP ? RT / 2 : RT); ++j) {
    if (at + j >= (UP ? pairs : shape.tiles)) continue;
#pragma unroll
    for (int m = 0; m < MT; ++m)
      if (m * 16 + t < rows) {
        if constexpr (UP) store4<true>(a.h, (int64_t)cell[m] * a.inter + (at + j) * 16 + 4 * g, gated(acc[2 * j][m], acc[2 * j + 1][m]), 4, true);
        else store4<false>(a.parts, (int64_t)cell[m] * a.hidden + (at + j) * 16 + 4 * g, acc[j][m], 4, true);
      }
  }
}

template <int FMT, bool UP, int RT, int WD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 8))) void moe_experts_kernel(MoeArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const Share share = share_of(a, 64);
  const int e = share.e, n_block = blockIdx.x;
  int listed = listed_row(a, e, share.first);          // (asked for with the count)
  const int count = a.counts[e * COUNT_APART];
  for (int r = share.first; r < count; r += share.stride) {
    if (r != share.first) {
      __syncthreads();                                 // (the rows before are still being read)
      listed = listed_row(a, e, r);
    }
    const int rows = min(64, count - r);
    if (rows <= 16) expert_rows<FMT, UP, 1, RT, WD>(a, e, n_block, listed, rows, lds);
    else if (rows <= 32) expert_rows<FMT, UP, 2, RT, WD>(a, e, n_block, listed, rows, lds);
    else if (rows <= 48) expert_rows<FMT, UP, 3, RT, WD>(a, e, n_block, listed, rows, lds);
    else expert_rows<FMT, UP, 4, RT, WD>(a, e, n_block, listed, rows, lds);
  }
}

// DOWN where the rows of an expert fit LDS whole (inter up to 1152): eight waves read them from there, and each goes through its tiles, four
// at a time, without a barrier, the weights WD blocks ahead across the tiles' ends.  128 experts of 768 x 2048 (107 MB): 48 rows 22 us, 512 rows 33 (34 MB of
// parts among it); through stages 23 and 35.  One workgroup an expert 47, four 43: the first costs idle CUs, the other a second round of reading rows.
constexpr int RESIDENT_BLOCKS = 9;
template <int FMT, int MT>
__device__ __forceinline__ void resident_rows(const MoeArgs& a, int e, int listed, int rows, int tile0, int tile1, unsigned char* lds) {
  constexpr bool SMALL = FMT == CS_WEIGHTS_E2M1;
  constexpr int RT = SMALL ? 4 : 2, WD = SMALL ? 3 : 1;
  const PackedShape& shape = a.down_shape;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = lane & 15, g = lane >> 4;
  const int blocks = shape.blocks, steps = shape.k / 32;
  const Resource rw = resource(a.down + (int64_t)e * shape.tiles * shape.tile_bytes), rx = resource(a.h);
  const int total = (tile1 - tile0 + 8 * RT - 1) / (8 * RT) * blocks;          // blocks of all turns of the wave
  Held<FMT> w[WD + 1][RT];
  int ahead = 0, ahead_b = 0, ahead_tile = tile0 + wave * RT;
  auto weights = [&](Held<FMT> (&h)[RT]) {                                     // the next block
#pragma unroll
    for (int j = 0; j < RT; ++j)
      h[j].fetch(rw, blocks, ahead_b, lane, ahead < total && ahead_tile + j < tile1 ? steps - 4 * ahead_b : 0, (uint32_t)(ahead_tile + j) * (uint32_t)shape.tile_bytes);
    ++ahead;
    if (++ahead_b == blocks) {
      ahead_b = 0;
      ahead_tile += 8 * RT;
    }
  };
#pragma unroll
  for (int i = 0; i < WD; ++i) weights(w[i]);
  int cell[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) cell[m] = __shfl(listed, min(m * 16 + t, rows - 1));
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const uint32_t off = row_offset<false>(a, __shfl(listed, min(m * 16 + (lane >> 2), rows - 1))) + (((lane & 3) ^ ((lane >> 3) & 3)) << 4);
    for (int step = wave; step < 4 * blocks; step += 8) fetch_lds16(rx, off, step < steps ? (uint32_t)step * 64 : PAST, lds + (step * MT + m) * 1024);
  }
  __builtin_amdgcn_s_waitcnt(0x0f70);                  // vmcnt(0)
  __syncthreads();
  const unsigned char* mine = lds + (lane & 15) * 64 + (((lane >> 4) ^ ((lane >> 1) & 3)) << 4);
  cf32x4 acc[RT][MT];
  auto clear = [&]() {
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[j][m] = cf32x4{0.f, 0.f, 0.f, 0.f};
  };
  clear();
  int b = 0, tile = tile0 + wave * RT, done = 0;
  auto block = [&](auto turn) {
    constexpr int R = decltype(turn)::value;
    weights(w[(R + WD) % (WD + 1)]);
    const unsigned char* from = mine + b * 4 * MT * 1024;
    pbf16x8 f[2][MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) f[0][m] = *reinterpret_cast<const pbf16x8*>(from + m * 1024);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s < 3) {
#pragma unroll
        for (int m = 0; m < MT; ++m) f[(s + 1) & 1][m] = *reinterpret_cast<const pbf16x8*>(from + ((s + 1) * MT + m) * 1024);
      }
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        const pbf16x8 v = w[R][j].at(s);
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[j][m] = mfma(v, f[s & 1][m], acc[j][m]);
      }
      interleave<FMT, RT, MT>();
      __builtin_amdgcn_sched_barrier(0);
    }
    if (++b == blocks) {
      if (done < total) {
#pragma unroll
        for (int j = 0; j < RT; ++j)
          if (tile + j < tile1) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
              if (m * 16 + t < rows) store4<false>(a.parts, (int64_t)cell[m] * a.hidden + (tile + j) * 16 + 4 * g, acc[j][m], 4, true);
          }
      }
      clear();
      b = 0;
      tile += 8 * RT;
    }
    ++done;
  };
  while (done < total) {
    block(step_tag<0>());
    if constexpr (WD >= 1) block(step_tag<1>());
    if constexpr (WD >= 2) block(step_tag<2>());
    if constexpr (WD >= 3) block(step_tag<3>());
  }
}

template <int FMT>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void moe_resident_kernel(MoeArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const Share share = share_of(a, 64);
  const int e = share.e, tiles = a.down_shape.tiles;
  int listed = listed_row(a, e, share.first);          // (asked for with the count)
  const int count = a.counts[e * COUNT_APART];
  const int tile0 = (int)((int64_t)tiles * blockIdx.x / gridDim.x), tile1 = (int)((int64_t)tiles * (blockIdx.x + 1) / gridDim.x);
  for (int r = share.first; r < count; r += share.stride) {
    if (r != share.first) {
      __syncthreads();                                 // (the rows before are still being read)
      listed = listed_row(a, e, r);
    }
    const int rows = min(64, count - r);
    if (rows <= 16) resident_rows<FMT, 1>(a, e, listed, rows, tile0, tile1, lds);
    else if (rows <= 32) resident_rows<FMT, 2>(a, e, listed, rows, tile0, tile1, lds);
    else if (rows <= 48) resident_rows<FMT, 3>(a, e, listed, rows, tile0, tile1, lds);
    else resident_rows<FMT, 4>(a, e, listed, rows, tile0, tile1, lds);
  }
}

// y of a row: its parts by their weights, in the order of the slots, in fp32; eight parts asked for together.  512 rows of 8 parts of 2048 (34 MB): 7.0 us.
// (Parts in bf16 would be half of that and of the second products' writing, at an error of half a step each.)
__global__ __launch_bounds__(256) void moe_sum_kernel(MoeArgs a) {
  const int64_t t = blockIdx.x;
  const int n = ((int)blockIdx.y * 256 + threadIdx.x) * 4;
  if (n >= a.hidden) return;
  cf32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (!a.live || a.live[t]) {
    const float* from = a.parts + t * a.slots * a.hidden + n;
    for (int i0 = 0; i0 < a.slots; i0 += 8) {
      cf32x4 p[8];
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int slot = min(i0 + i, a.slots - 1);
        p[i] = *reinterpret_cast<const cf32x4*>(from + (int64_t)slot * a.hidden);
        w[i] = slot < a.top ? a.weights_out[t * a.top + slot] : 1.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i0 + i < a.slots) v += w[i] * p[i];
    }
  }
  store4<true>(a.y, t * a.y_row + n, v, 4, true);
}

namespace {

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

// Rows of a call that go through the launches together: as many as MOE_WORKSPACE holds (the counts and the widest row, 26 MB, fit in it), the
// rows of h within 32-bit offsets.  Each group reads its experts' weights again: 4096 rows of 256 experts of 7168 x 2048 and a shared one, top 8, take 4.48 ms
// and 1.14 GiB at once, 4.82 in two groups, 5.09 in three, so the bound is one that only wider layers meet.
int64_t group_rows(const MoeArgs& a) {
  const int64_t slots = a.top + a.shared, experts = a.experts + a.shared;
  const int64_t row = 8ll * a.experts + 4 * experts + slots * (2ll * a.inter + 4ll * a.hidden);      // what moe_layout takes for one
  const int64_t most = std::min<int64_t>({MOE_ROWS, 0x7fffffffll / (2 * slots * a.inter), (MOE_WORKSPACE - experts * COUNT_APART * 4 - 80) / row});
  return std::min(a.n_rows, most);
}

template <int FMT>
cs_status run_moe(const MoeArgs& a, hipStream_t s) {
  const int T = (int)a.n_rows;
  // Up to 16 rows: the second products and the sum in one launch, unless the experts that have rows are many for its hidden / 16 workgroups (128 experts
  // of 2048 x 768, 8 a row, in one and in two launches: 4 rows 33.0 and 32.1 us, 8 rows 50.1 and 43.7, 16 rows 69.3 and 57.1; 256 of 512 x 1024, 8 rows 47 and 36; 16
  // of 3584 x 1280, 8 rows 35.3 and 37.7; 24 of 1056 x 352, 16 rows 21.2 and 23.2)
  const double used = a.experts * (1 - std::pow(1 - (double)a.top / a.experts, T));
  const bool at_once = T == 1 || (T <= 16 && used * a.inter * (4096 - a.hidden) <= 50e6);
  if (T >= 64) hipLaunchKernelGGL(moe_logits_tile_kernel, dim3((a.experts + 15) / 16, (T + 15) / 16), dim3(1024), 0, s, a);
  else if ((int64_t)T * a.experts <= 1024) hipLaunchKernelGGL((moe_logits_kernel<1>), dim3(a.experts, T), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((moe_logits_kernel<4>), dim3(a.experts, (T + 3) / 4), dim3(256), 0, s, a);
  CS_HIP(hipGetLastError());
  if (T == 1) {
    hipLaunchKernelGGL((moe_few_up_kernel<FMT, true, 1>), dim3(a.inter / 16, a.slots), dim3(256), 0, s, a);
  } else {
    hipLaunchKernelGGL(moe_select_kernel, dim3(T), dim3(256), 0, s, a);
    CS_HIP(hipGetLastError());
    // Few rows an expert and little to read: 16 at a time, straight from memory (24 rows for 24 experts of 1056 x 352: 21 us, staged 27);
    // where the weights are what takes the time, staged is as fast or faster (us: 128 experts of 2048 x 768, 20 rows 61 and 61, 96 rows 85 and 79; 48 of
    // 2048 x 1024, 40 rows 50 and 47; but 16 of 3584 x 1280 and a shared one 48 and 54, in bf16 100 and 107).
    if (T <= 16 || ((int64_t)T * a.top <= 6 * a.experts && (int64_t)a.hidden * a.inter * a.experts <= 80 << 20)) {
      constexpr int PAIRS = FMT == CS_WEIGHTS_E2M1 ? 2 : 1;
      const int shares = share_rows(a, 16);
      hipLaunchKernelGGL((moe_few_up_kernel<FMT, false, PAIRS>), dim3(a.inter / 16 / PAIRS, shares), dim3(256), 0, s, a);
      if (!at_once) hipLaunchKernelGGL((moe_few_down_kernel<FMT, 2>), dim3((a.hidden / 16 + 3) / 4, shares), dim3(256), 0, s, a);
    } else {
      // workgroups for twice the rows that an expert has on average; those with more take them in turn
      const int z = (int)std::max<int64_t>(1, std::min<int64_t>((T + 63) / 64, (2ll * T * a.top / a.experts + 63) / 64)), shares = share_rows(a, 64);
      constexpr bool SMALL = FMT == CS_WEIGHTS_E2M1;           // (bf16 weights: half as many tiles a wave, for the registers)
      constexpr int RT = SMALL ? 4 : 2, DOWN_WD = SMALL ? 2 : 1;
      hipLaunchKernelGGL((moe_experts_kernel<FMT, true, RT, 1>), dim3((a.inter / 16 + 2 * RT - 1) / (2 * RT), shares, z), dim3(256), EXPERT_LDS, s, a);
      CS_HIP(hipGetLastError());
      if (a.down_shape.blocks <= RESIDENT_BLOCKS) {
        const int lds = a.down_shape.blocks * 16384;
        CS_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(moe_resident_kernel<FMT>), hipFuncAttributeMaxDynamicSharedMemorySize, RESIDENT_BLOCKS * 16384));
        const int parts = std::max(1, std::min((256 + shares * z - 1) / (shares * z), a.down_shape.tiles / (8 * RT)));
        hipLaunchKernelGGL((moe_resident_kernel<FMT>), dim3(parts, shares, z), dim3(512), lds, s, a);
      } else {
        hipLaunchKernelGGL((moe_experts_kernel<FMT, false, RT, DOWN_WD>), dim3((a.hidden / 16 + 4 * RT - 1) / (4 * RT), shares, z), dim3(256), EXPERT_LDS, s, a);
      }
    }
  }
  CS_HIP(hipGetLastError());
  if (at_once) {
    // parts of an expert, so that every wave has one where few experts have rows
    const int shares = std::max(1, std::min(a.down_shape.blocks, 16 / std::min(16, T * a.top + a.shared)));
    if (T == 1) hipLaunchKernelGGL((moe_row_sum_kernel<FMT>), dim3(a.hidden / 16), dim3(1024), 0, s, a, std::max(1, std::min(a.down_shape.blocks, 16 / std::min(16, a.slots))));
    else hipLaunchKernelGGL((moe_few_sum_kernel<FMT>), dim3(a.hidden / 16), dim3(1024), 0, s, a, shares);
  } else {
    hipLaunchKernelGGL(moe_sum_kernel, dim3(T, (a.hidden + 1023) / 1024), dim3(256), 0, s, a);
  }
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
  a.counts = reinterpret_cast<int32_t*>(take((size_t)(a.experts + a.shared) * COUNT_APART * 4));
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
