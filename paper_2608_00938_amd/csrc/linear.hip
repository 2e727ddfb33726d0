// Matrix product with its epilogue for gfx950:
//   out[r, n] = act(x_scale[r] * w_scale[n] * sum_k x[r, k] * w[n, k] + bias[n]) + residual[r, n]
// over fp32, bf16 or e4m3 inputs on the matrix core, accumulated in fp32.
//
// Orientation.  The weights are the matrix instruction's first operand and the
// activations its second, so that a lane's accumulators are consecutive outputs
// of one row.  Both operands lie in memory with k contiguous, and a lane of
// either reads 16-byte chunks of a row; which k of the chunk meet in which step
// is the same for both, which is all that a product needs.
#include <math.h>

#include "common.hpp"
#include "kernels.hpp"

namespace grace {

namespace {

// Input types.  The matrix core's 8-bit products are cut before they are added:
// of the eight of a group each loses what lies below 2^-13 of the largest one's
// power of two (probed), so a sum is up to 2^-10 of sum |x w| off, in the mean
// 1.4e-5 of the result.  That is a hundredth of the rounding to bf16, and E4M3
// outputs in bf16 take these instructions.  Outputs in fp32 take E4M3Wide: the
// values as bf16, which holds them exactly, whose products are summed in fp32.
struct E4M3 {
  using storage = uint8_t;
  static constexpr int kBytes = 1;
};
struct E4M3Wide : E4M3 {};
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
constexpr int kRowChunks = 8;     // 16-byte chunks of a tile's row: 128 bytes of k

// Place of chunk c of tile row `row`: consecutive rows put one chunk index on
// different banks.
__device__ __forceinline__ int slot(int row, int c) { return row * kRowChunks + (c ^ (row & 7)); }

// One step of a 32 x 32 tile: steps per tile row, chunks that a lane reads per
// step, what it makes of them, and the product.
template <class T> struct Step;
template <> struct Step<BF16> {
  static constexpr int kSteps = 4, kChunks = 1;
  using Frag = bf16x8;
  __device__ __forceinline__ static Frag make(const u32x4* c) { return __builtin_bit_cast(Frag, c[0]); }
  __device__ __forceinline__ static f32x16 run(Frag a, Frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Step<E4M3> {
  static constexpr int kSteps = 2, kChunks = 2;
  using Frag = i32x8;
  __device__ __forceinline__ static Frag make(const u32x4* c) {
    return Frag{(int)c[0].x, (int)c[0].y, (int)c[0].z, (int)c[0].w,
                (int)c[1].x, (int)c[1].y, (int)c[1].z, (int)c[1].w};
  }
  __device__ __forceinline__ static f32x16 run(Frag a, Frag b, f32x16 c) {
    // format 0 is e4m3; the block scales are 2^(127 - 127)
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0x7f7f7f7f, 0,
                                                           0x7f7f7f7f);
  }
};
template <> struct Step<E4M3Wide> {
  static constexpr int kSteps = 4, kChunks = 1;
  struct Frag { bf16x8 lo, hi; };
  __device__ __forceinline__ static bf16x8 widen(uint32_t u, uint32_t v) {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    const auto w = [](uint32_t x, bool high) {
      return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.f, true)
                                               : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, 1.f, false));
    };
    return __builtin_bit_cast(bf16x8, words{w(u, false), w(u, true), w(v, false), w(v, true)});
  }
  __device__ __forceinline__ static Frag make(const u32x4* c) {
    return {widen(c[0].x, c[0].y), widen(c[0].z, c[0].w)};
  }
  __device__ __forceinline__ static f32x16 run(const Frag& a, const Frag& b, f32x16 c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.lo, b.lo, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.hi, b.hi, c, 0, 0, 0);
  }
};
template <> struct Step<F32> {
  static constexpr int kSteps = 4, kChunks = 1;
  using Frag = f32x4;
  __device__ __forceinline__ static Frag make(const u32x4* c) { return __builtin_bit_cast(Frag, c[0]); }
  __device__ __forceinline__ static f32x16 run(Frag a, Frag b, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
  }
};

struct LinearArgs {
  const void *x, *w;
  const float *x_scale, *w_scale;
  const void *bias, *residual;
  void* out;
  int32_t R, N, K, act, out_dtype;
};

__device__ __forceinline__ float activate(float y, int act) {
  if (act == GRACE_ACT_RELU) return y < 0.f ? 0.f : y;      // a NaN stays
  if (act == GRACE_ACT_GELU) return 0.5f * y * erfcf(y * -0.70710678118654752f);   // 1 + erf without its cancellation
  if (act == GRACE_ACT_SILU) return y / (1.f + expf(-y));
  return y;
}

// N values, the choice made once.  Outputs in bf16 take the hardware's exp2 and
// reciprocal (a step each), and for the normal distribution's tail the form
// (c1 t + .. + c8 t^8) exp(-x^2), t = 1 / (1 + 0.46 x), of Hastings' approximations,
// its coefficients fitted for the least relative error: 7e-7 for every x >= 0, where
// half a step of bf16 is 2e-3.
template <class O, int N>
__device__ __forceinline__ void activate_all(float* y, int act) {
  if (act == GRACE_ACT_NONE) return;
  if (act == GRACE_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = y[e] < 0.f ? 0.f : y[e];
  } else if (act == GRACE_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (O::kBytes == 2) y[e] *= __builtin_amdgcn_rcpf(1.f + fast_exp2(-kLog2e * y[e]));
      else y[e] = activate(y[e], GRACE_ACT_SILU);
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (O::kBytes == 2) {
        const float x = fabsf(y[e]) * 0.70710678118654752f;
        const float t = __builtin_amdgcn_rcpf(fmaf(0.46f, x, 1.f));
        float q = fmaf(t, 0.0338674337f, -0.113352589f);
        q = fmaf(t, q, 0.0846516341f);
        q = fmaf(t, q, 0.0262629706f);
        q = fmaf(t, q, 0.0934410468f);
        q = fmaf(t, q, 0.115587346f);
        q = fmaf(t, q, 0.129778966f);
        q = fmaf(t, q, 0.129763514f);
        const float tail = t * q * fast_exp2(-kLog2e * x * x);
        y[e] *= y[e] < 0.f ? tail : 1.f - tail;
      } else {
        y[e] = activate(y[e], GRACE_ACT_GELU);
      }
    }
  }
}

__device__ __forceinline__ float load_out_type(const void* p, int64_t i, int dtype) {
  return dtype == GRACE_F32 ? ((const float*)p)[i] : bf16_bits_to_f32(((const uint16_t*)p)[i]);
}

// Outputs n .. n + 3 of row r.
__device__ __forceinline__ void finish4(const LinearArgs& a, int64_t r, int32_t n, const float* v) {
  const float xs = a.x_scale ? a.x_scale[r] : 1.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (n + e >= a.N) return;
    float y = v[e];
    if (a.x_scale) y *= xs;
    if (a.w_scale) y *= a.w_scale[n + e];
    if (a.bias) y += load_out_type(a.bias, n + e, a.out_dtype);
    y = activate(y, a.act);
    const int64_t at = r * a.N + n + e;
    if (a.residual) y += load_out_type(a.residual, at, a.out_dtype);
    if (a.out_dtype == GRACE_F32) ((float*)a.out)[at] = y;
    else ((uint16_t*)a.out)[at] = (uint16_t)pack_bf16x2(y, 0.f);
  }
}

// 16 bytes from any element on: the hardware takes them off their alignment.
template <class T>
__device__ __forceinline__ u32x4 load16(const typename T::storage* p) { return *(const u32x4_any*)p; }

// 16 bytes of a row of K elements from element k on, zeros past its end.
template <class T>
__device__ __forceinline__ u32x4 load_chunk(const typename T::storage* row, int32_t K, int32_t k) {
  constexpr int E = 16 / T::kBytes;
  if (k + E <= K) return load16<T>(row + k);
  if (k >= K) return u32x4{0, 0, 0, 0};
  if (K >= E) {                                            // the row's last 16 bytes, moved down
    const u32x4 c = load16<T>(row + (K - E));
    const int bits = (k + E - K) * T::kBytes * 8;          // 8 .. 120
    const uint64_t lo = (uint64_t)c.y << 32 | c.x, hi = (uint64_t)c.w << 32 | c.z;
    const uint64_t a = bits >= 64 ? hi >> (bits - 64) : lo >> bits | hi << (64 - bits), b = bits >= 64 ? 0 : hi >> bits;
    return u32x4{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
  }
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (k + e < K) {
      uint32_t bits;
      if constexpr (T::kBytes == 4) bits = __float_as_uint(row[k + e]);
      else bits = row[k + e];
      v[e * T::kBytes / 4] |= bits << (e * T::kBytes % 4 * 8);
    }
  }
  return v;
}

// ---------------------------------------------------------------------------
// Few rows, or few outputs of fp32: workgroups of 16 columns x 16 RT rows whose eight waves
// share out k and add up in LDS.
//
// Fragments come from memory in operand layout, without LDS: a lane reads 16 (e4m3:
// 32) bytes of a row, four lanes 64 or 128 consecutive ones, and several steps are
// under way at once; what bounds it is reading the weights.  Takes any size and
// alignment.
// ---------------------------------------------------------------------------
template <class T> struct Step16;
template <> struct Step16<BF16> {
  static constexpr int kChunks = 1;
  __device__ __forceinline__ static f32x4 run(const u32x4* a, const u32x4* b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[0]),
                                                   __builtin_bit_cast(bf16x8, b[0]), c, 0, 0, 0);
  }
};
template <> struct Step16<E4M3> {
  static constexpr int kChunks = 2;
  __device__ __forceinline__ static f32x4 run(const u32x4* a, const u32x4* b, f32x4 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(Step<E4M3>::make(a), Step<E4M3>::make(b), c, 0, 0,
                                                            0, 0x7f7f7f7f, 0, 0x7f7f7f7f);
  }
};
template <> struct Step16<E4M3Wide> {
  static constexpr int kChunks = 1;
  __device__ __forceinline__ static f32x4 run(const u32x4* a, const u32x4* b, f32x4 c) {
    const auto x = Step<E4M3Wide>::make(a), y = Step<E4M3Wide>::make(b);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.lo, y.lo, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.hi, y.hi, c, 0, 0, 0);
  }
};
template <> struct Step16<F32> {
  static constexpr int kChunks = 1;
  __device__ __forceinline__ static f32x4 run(const u32x4* a, const u32x4* b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[0][i]), __uint_as_float(b[0][i]), c, 0, 0, 0);
    return c;
  }
};

constexpr int kFewWaves = 8;

template <class T, int RT>
__global__ void __launch_bounds__(kFewWaves * 64) linear_few_kernel(LinearArgs a, uint32_t tiles_r, uint32_t first) {
  using S = Step16<T>;
  constexpr int kStepK = 64 * S::kChunks / T::kBytes;      // of a wave's step
  constexpr int kUnroll = RT == 1 ? 4 : 2;
  __shared__ f32x4 sums[kFewWaves][RT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t id = first + blockIdx.x;
  const int64_t r0 = (int64_t)(id % tiles_r) * (16 * RT);
  const int32_t n0 = (int32_t)(id / tiles_r) * 16;
  const int i16 = lane & 15, part = lane >> 4;
  const int32_t k_lane = part * (kStepK / 4);
  const typename T::storage* const w = (const typename T::storage*)a.w + min((int64_t)n0 + i16, (int64_t)a.N - 1) * a.K;
  const typename T::storage* x[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
    x[i] = (const typename T::storage*)a.x + min(r0 + i * 16 + i16, (int64_t)a.R - 1) * a.K;
  constexpr int E = 16 / T::kBytes;
  f32x4 acc[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) acc[i] = f32x4{0, 0, 0, 0};
  // whole steps, kUnroll of them at once, dealt out over the waves
  const int32_t whole = a.K / kStepK, groups = whole / kUnroll;
  for (int32_t g = wave; g < groups; g += kFewWaves) {
    const int32_t k = g * (kUnroll * kStepK) + k_lane;
    u32x4 fw[kUnroll][S::kChunks], fx[kUnroll][RT][S::kChunks];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) {
        fw[u][c] = load16<T>(w + k + u * kStepK + c * E);
#pragma unroll
        for (int i = 0; i < RT; ++i) fx[u][i][c] = load16<T>(x[i] + k + u * kStepK + c * E);
      }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int i = 0; i < RT; ++i) acc[i] = S::run(fw[u], fx[u][i], acc[i]);
  }
  // the steps that are left, the last one perhaps short: one a wave (there are at most kUnroll)
  const int32_t steps = (a.K + kStepK - 1) / kStepK, mine = groups * kUnroll + wave;
  if (mine < steps) {
    const int32_t k = mine * kStepK + k_lane;
    u32x4 fw[S::kChunks], fx[RT][S::kChunks];
#pragma unroll
    for (int c = 0; c < S::kChunks; ++c) {
      fw[c] = load_chunk<T>(w, a.K, k + c * E);
#pragma unroll
      for (int i = 0; i < RT; ++i) fx[i][c] = load_chunk<T>(x[i], a.K, k + c * E);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = S::run(fw, fx[i], acc[i]);
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) sums[wave][i][lane] = acc[i];
  __syncthreads();
  // lane l has row l % 16 and columns 4 (l / 16) .. + 3
  if (wave < RT) {
    f32x4 y = sums[0][wave][lane];
#pragma unroll
    for (int g = 1; g < kFewWaves; ++g) y += sums[g][wave][lane];
    const int64_t r = r0 + wave * 16 + i16;
    const float v[4] = {y[0], y[1], y[2], y[3]};
    if (r < a.R) finish4(a, r, n0 + part * 4, v);
  }
}

// ---------------------------------------------------------------------------
// Tile kernel: direct loads into a ring of LDS tiles.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// 16 bytes per lane from base + off to LDS at `to` + 16 * lane (base and `to`
// uniform over the wave).  As asm, so that the compiler does not wait for it where
// LDS is read: wait_loads does, ahead of the barrier that hands the tile on.
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, uint32_t to) {
  asm volatile("global_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "{m0}"(to) : "memory");
}
// Waits until at most N of the wave's loads are under way.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Which tile a workgroup takes.  Workgroup i runs on XCD i % 8: each XCD takes a
// contiguous eighth of the tiles, and these go through groups of 8 row tiles, one
// column of the group after the other, so that what an XCD runs at once is 8 row
// tiles and a few column tiles, read through its L2.
struct TileMap {
  uint32_t tiles_r, tiles_n, all, per;   // per: of an XCD
  __device__ bool take(uint32_t id, uint32_t& tr, uint32_t& tn) const {
    const uint32_t i = id % 8 * per + id / 8;
    if (id / 8 >= per || i >= all) return false;
    const uint32_t group = i / (8 * tiles_n), in = i - group * 8 * tiles_n;
    const uint32_t high = min(8u, tiles_r - group * 8);
    tn = in / high;
    tr = group * 8 + in - tn * high;
    return true;
  }
};

// Eight values from element i on, at any alignment, or the first `left` of them (EIGHTS:
// none or eight).
template <class O, bool EIGHTS>
__device__ __forceinline__ void load8(const void* p, int64_t i, int left, float* f) {
  const typename O::storage* at = (const typename O::storage*)p + i;
  if (EIGHTS ? left > 0 : left >= 8) {
#pragma unroll
    for (int c = 0; c < O::kBytes / 2; ++c) Chunk<O>::unpack(load16<O>(at + c * 4), f + c * 4);
  } else if (!EIGHTS) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) f[e] = load_out_type(at, e, O::kBytes == 4 ? GRACE_F32 : GRACE_BF16);
  }
}
template <class O, bool EIGHTS>
__device__ __forceinline__ void store8(void* p, int64_t i, int left, const float* f) {
  typename O::storage* at = (typename O::storage*)p + i;
  if (EIGHTS ? left > 0 : left >= 8) {
#pragma unroll
    for (int c = 0; c < O::kBytes / 2; ++c) *(u32x4_any*)(at + c * 4) = Chunk<O>::pack(f + c * 4);
  } else if (!EIGHTS) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) {
        if constexpr (O::kBytes == 4) at[e] = f[e];
        else at[e] = (uint16_t)pack_bf16x2(f[e], 0.f);
      }
  }
}

// WR x WN waves of RT x NT tiles of 32 x 32: BR rows of x against BN rows of w, in
// tiles of 128 bytes of k (whole cache lines: with 64 the L2 had twice the requests
// to serve and was the bound) that go round STAGES places in LDS.
//
// Order within a wave.  The products of a step go through the rows of the wave's
// tile; when a row is done its fragment of the next step is read into the same
// registers, the columns' fragments into a second set.  In a tile's last step the
// first row's products are followed by the hand-over: the next tile has landed and
// every wave has the rest of this one in registers (one barrier).  From there to the
// end of the next tile's first step the loads of the tile after next are issued into
// the stage just left, one or two after each row: all at once they fill the address
// path's queue and hold up the waves behind them (8192^3 bf16 973 us).
//
// DIRECT: 16-byte aligned rows of x and w (k a multiple of a chunk), loaded straight
// into LDS; others pass through registers on the way.  EIGHTS: N is a multiple of 8,
// which saves a branch at each store (262144 x 1024 -> 4096 e4m3 1500 -> 1475 us).
// Other outputs leave as whole lines as well, at any alignment: stored one by one from
// the accumulators 262144 x 512 -> 509 bf16 took 748 us instead of 188.
//
// What bounds it: of a long k the matrix core (8192^3 bf16 829 us = 1326 TFLOP/s, 76 %
// busy; e4m3 426 us = 2580), of a short one what is not under products.  Of 262144 x
// 1024 -> 4096 e4m3 with silu (1464 us, 495 of them writes at the copy rate) a 256 x 256
// tile spends some 5 thousand cycles on its first loads, 3 thousand on each of 8 tiles
// of k (2 thousand of products) and 10 to 15 thousand on its epilogue.
template <class T, class O, int WR, int WN, int RT, int NT, int STAGES, bool EIGHTS, bool DIRECT>
__global__ void __launch_bounds__(WR * WN * 64, 2) linear_tile_kernel(LinearArgs a, TileMap map, uint32_t first) {
  using S = Step<T>;
  constexpr int kTileWaves = WR * WN;
  constexpr int BR = WR * RT * 32, BN = WN * NT * 32, kRows = BR + BN;
  constexpr int kLoads = kRows / (kTileWaves * 8);         // of 8 rows
  constexpr int kStageBytes = kRows * 128;
  constexpr int kOutBytes = 32 * NT * 128;                 // 32 rows of a wave's sums
  static_assert(kTileWaves * kOutBytes <= STAGES * kStageBytes, "sums fit where the tiles were");
  // Tiles of k under way in registers: three where they are small (2000 x 1021 -> 509 bf16
  // 12.5 us with one, 10.8 with three; of e4m3, 2000 x 1001 -> 1000, 11.2 and 12.1).
  constexpr int kHeld = !DIRECT && RT * NT == 1 && T::kBytes > 1 ? 3 : 1;
  constexpr int kAhead = DIRECT ? STAGES : kHeld + 1;      // tile t + kAhead is loaded when t + 1 is handed over
  static_assert(DIRECT || STAGES == 2, "a tile read, a tile written");
  static_assert((STAGES & (STAGES - 1)) == 0, "tile t lies in stage t % STAGES");
  __shared__ __attribute__((aligned(256))) char lds[STAGES * kStageBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, col = lane & 31;

  // Loads: a wave's instruction covers 8 rows; lane l brings a chunk of row l / 8 to
  // place l % 8, where chunk c of row r lies at place c ^ (r / 2 % 8): 16 rows of one
  // chunk, as a fragment's lanes read them, are on different banks.
  const int64_t pitch = (int64_t)a.K * T::kBytes;
  const int chunk = (lane & 7) ^ ((wave * 4 + (lane >> 4)) & 7);
  const int32_t tiles = (int32_t)((pitch + 127) / 128);    // of k
  const int last_chunks = (int)((pitch - (int64_t)(tiles - 1) * 128) / 16);
  const bool beyond = chunk >= last_chunks;                // in the last tile: past k's end
  const uint32_t lds0 = lds_addr(lds);
  uint32_t tr, tn;
  if (!map.take(first + blockIdx.x, tr, tn)) return;
  const int64_t r0 = (int64_t)tr * BR;
  const int32_t n0 = (int32_t)(tn * BN);
  const char* const xb = (const char*)a.x + r0 * pitch;
  const char* const wb = (const char*)a.w + (int64_t)n0 * pitch;
  uint32_t off[kLoads];
  {
    const int rows = (int)min((int64_t)BR, (int64_t)a.R - r0) - 1, cols = min(BN, a.N - n0) - 1;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int row = (wave + j * kTileWaves) * 8 + (lane >> 3);
      off[j] = (uint32_t)((wave + j * kTileWaves) * 8 < BR ? min(row, rows) : min(row - BR, cols)) *
                   (uint32_t)pitch + chunk * 16;
    }
  }
  u32x4 held[kHeld][DIRECT ? 1 : kLoads];
  const auto load = [&](int32_t t, int h, int j) __attribute__((always_inline)) {
    const char* const from = ((wave + j * kTileWaves) * 8 < BR ? xb : wb) + (int64_t)t * 128;
    if constexpr (!DIRECT) {
      constexpr int E = 16 / T::kBytes;
      if (t < tiles - 1) held[h][j] = load16<T>((const typename T::storage*)(from + off[j]));
      else held[h][j] = load_chunk<T>((const typename T::storage*)(from + (off[j] - chunk * 16)),
                                   a.K - (tiles - 1) * (128 / T::kBytes), chunk * E);
      return;
    }
    // what lies past a row's end reads the row's first chunk of the tile, and is cleared later
    const uint32_t back = t == tiles - 1 && beyond ? chunk * 16 : 0;
    load_to_lds(from, off[j] - back, lds0 + (t & (STAGES - 1)) * kStageBytes + (wave + j * kTileWaves) * 1024);
  };
  constexpr int kPerRow = (kLoads + 2 * RT - 1) / (2 * RT); // loads after a row's products
  const auto load_part = [&](int32_t t, int h, int part) __attribute__((always_inline)) {
#pragma unroll
    for (int j = part * kPerRow; j < (part + 1) * kPerRow; ++j)
      if (j < kLoads) load(t, h, j);
  };
  // Tile t of k has landed, its end is clean, and every wave knows it.
  const auto hand_over = [&](int32_t t, int h, bool ahead) __attribute__((always_inline)) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        *(u32x4*)(lds + (t & (STAGES - 1)) * kStageBytes + (wave + j * kTileWaves) * 1024 + lane * 16) = held[h][j];
      lds_barrier();
      return;
    }
    if (STAGES > 2 && ahead) wait_loads<(STAGES - 2) * kLoads>();   // those of the tiles behind it
    else wait_loads<0>();
    if (t == tiles - 1 && beyond)
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        *(u32x4*)(lds + (t & (STAGES - 1)) * kStageBytes + (wave + j * kTileWaves) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
    lds_barrier();
  };

  f32x16 acc[RT][NT];
  const int wr = wave / WN * RT * 32, wn = wave % WN * NT * 32;
  const int swz = col >> 1 & 7;
  const char* const xrow = lds + (wr + col) * 128;
  const char* const wrow = lds + (BR + wn + col) * 128;
  typename S::Frag fr[RT == 1 ? 2 : RT], fn[2][NT];
  const auto frag = [&](const char* row, int stage, int s) {
    u32x4 c[S::kChunks];
#pragma unroll
    for (int i = 0; i < S::kChunks; ++i)
      c[i] = *(const u32x4*)(row + stage * kStageBytes + (((s * 2 + half) * S::kChunks + i) ^ swz) * 16);
    return S::make(c);
  };
  // tile t of k, whose registers are h of held; next: there is a tile behind it; half: tile
  // t + kAhead - 1 is there, whose loads are half issued, more: and one behind that
  const auto tile = [&](int32_t t, int h, auto next, auto half_left, auto more) __attribute__((always_inline)) {
    const int stage = t & (STAGES - 1), after = (t + 1) & (STAGES - 1);
#pragma unroll
    for (int s = 0; s < S::kSteps; ++s) {
      const bool last = s + 1 == S::kSteps;
      const int from = last ? after : stage, step = last ? 0 : s + 1;
      // no other row's products to read under: fragments a step ahead (2000 x 1021 -> 509 fp32
      // 32.8 -> 31.2 us; e4m3, two steps a tile, was slower)
      if constexpr (RT == 1 && S::kSteps == 4) {
        if (!last || next) {
          if (last) hand_over(t + 1, (h + 1) % kHeld, more);
#pragma unroll
          for (int j = 0; j < NT; ++j) fn[(s + 1) & 1][j] = frag(wrow + j * 32 * 128, from, step);
          fr[(s + 1) & 1] = frag(xrow, from, step);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[0][j] = S::run(fn[s & 1][j], fr[s & 1], acc[0][j]);
        __builtin_amdgcn_sched_barrier(0);
        if (last && more) load_part(t + kAhead, (h + 1) % kHeld, 0);
        if (s == 0 && half_left) load_part(t + kAhead - 1, h, 1);
        continue;
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = S::run(fn[s & 1][j], fr[i], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
        if (!last || next) {
          if (i == 0) {
            if (last) hand_over(t + 1, (h + 1) % kHeld, more);
#pragma unroll
            for (int j = 0; j < NT; ++j) fn[(s + 1) & 1][j] = frag(wrow + j * 32 * 128, from, step);
          }
          fr[i] = frag(xrow + i * 32 * 128, from, step);
        }
        if (last && more) load_part(t + kAhead, (h + 1) % kHeld, i);
        if (s == 0 && half_left) load_part(t + kAhead - 1, h, RT + i);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  struct Yes { constexpr operator bool() const { return true; } };
  struct No { constexpr operator bool() const { return false; } };

#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x16{0};
#pragma unroll
  for (int j = 0; j < kLoads; ++j) load(0, 0, j);
#pragma unroll
  for (int t = 1; t < kAhead - 1; ++t)
    if (t < tiles)
#pragma unroll
      for (int j = 0; j < kLoads; ++j) load(t, t % kHeld, j);
  constexpr int kHalf = kPerRow * RT < kLoads ? kPerRow * RT : kLoads;
  if (DIRECT && tiles >= STAGES) {
#pragma unroll
    for (int i = 0; i < RT; ++i) load_part(STAGES - 1, 0, i);
    wait_loads<(STAGES - 2) * kLoads + kHalf>();
    lds_barrier();
  } else {
    hand_over(0, 0, false);
    if (!DIRECT && tiles > kAhead - 1)
#pragma unroll
      for (int i = 0; i < RT; ++i) load_part(kAhead - 1, 0, i);
  }
  int32_t t = 0;
#pragma unroll
  for (int j = 0; j < NT; ++j) fn[0][j] = frag(wrow + j * 32 * 128, 0, 0);
#pragma unroll
  for (int i = 0; i < RT; ++i) fr[i] = frag(xrow + i * 32 * 128, 0, 0);
  if constexpr (kHeld > 1) {
    for (; t + kHeld - 1 + kAhead < tiles; t += kHeld)
#pragma unroll
      for (int h = 0; h < kHeld; ++h) tile(t + h, h, Yes{}, Yes{}, Yes{});
    for (; t < tiles; t += kHeld)
#pragma unroll
      for (int h = 0; h < kHeld; ++h)
        if (t + h < tiles) tile(t + h, h, t + h + 1 < tiles, t + h + kAhead - 1 < tiles, t + h + kAhead < tiles);
  } else {
    for (; t + STAGES < tiles; ++t) tile(t, 0, Yes{}, Yes{}, Yes{});
    if constexpr (STAGES == 2) {
      if (t + 1 < tiles) tile(t++, 0, Yes{}, Yes{}, No{});
    } else {
      for (; t + 1 < tiles; ++t) tile(t, 0, Yes{}, t + STAGES - 1 < tiles, No{});
    }
    tile(t, 0, No{}, No{}, No{});
  }
  // The products stay out of the epilogue's branches: there the compiler would set the
  // block scales for the lanes that store alone, and the matrix core reads all lanes'.
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) asm volatile("" : "+v"(acc[i][j]));
  lds_barrier();

  // Epilogue.  In the accumulators lane l has row l % 32 and, of every 8 columns, 4 (l /
  // 32) .. + 3; 32 rows at a time they go through LDS of the wave's own, so that a
  // lane has 8 columns, the same for all its rows, and rows leave as whole lines.
  constexpr int kRowChunk = NT * 8, kLanes = kRowChunk / 2, kPer = 32 * kLanes / 64;
  const auto at = [&](int row, int c) {                   // 16 rows of one chunk on different banks
    const int turn = kRowChunk == 16 ? row : row >> 1;
    return row * NT * 128 + (c ^ (turn & (kRowChunk - 1))) * 16;
  };
  char* const mine = lds + wave * kOutBytes;
  const int row_in = lane / kLanes, c = lane % kLanes * 2;
  const int32_t n = n0 + wn + c * 4;
  const int left = EIGHTS ? (n < a.N ? 8 : 0) : a.N - n;  // of the lane's columns
  float ws[8], bias[8], xs[RT][kPer];
#pragma unroll
  for (int e = 0; e < 8; ++e) ws[e] = 1.f, bias[e] = 0.f;
  if (a.w_scale) load8<F32, EIGHTS>(a.w_scale, n, left, ws);
  if (a.bias) load8<O, EIGHTS>(a.bias, n, left, bias);
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int q = 0; q < kPer; ++q)
      xs[i][q] = a.x_scale ? a.x_scale[min(r0 + wr + i * 32 + q * (64 / kLanes) + row_in, (int64_t)a.R - 1)] : 1.f;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(f32x4*)(mine + at(col, j * 8 + g * 2 + half)) =
            f32x4{acc[i][j][g * 4], acc[i][j][g * 4 + 1], acc[i][j][g * 4 + 2], acc[i][j][g * 4 + 3]};
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int row = q * (64 / kLanes) + row_in;
      const int64_t r = r0 + wr + i * 32 + row;
      float y[8], res[8];
      *(f32x4*)y = *(const f32x4*)(mine + at(row, c));
      *(f32x4*)(y + 4) = *(const f32x4*)(mine + at(row, c + 1));
      if (r >= a.R || left <= 0) continue;
      if (a.residual) load8<O, EIGHTS>(a.residual, r * a.N + n, left, res);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = fmaf(y[e] * xs[i][q], ws[e], bias[e]);   // (a product of scales may leave fp32)
      activate_all<O, 8>(y, a.act);
      if (a.residual)
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += res[e];
      store8<O, EIGHTS>(a.out, r * a.N + n, left, y);
    }
  }
}

template <class T, class O, int WR, int WN, int RT, int NT, int STAGES>
hipError_t run_tile(const LinearArgs& a, hipStream_t stream) {
  constexpr int BR = WR * RT * 32, BN = WN * NT * 32, kThreads = WR * WN * 64;
  const uint32_t tiles_r = (uint32_t)(((int64_t)a.R + BR - 1) / BR), tiles_n = (uint32_t)(((int64_t)a.N + BN - 1) / BN);
  const uint32_t all = tiles_r * tiles_n, per = (all + 7) / 8;
  const TileMap map{tiles_r, tiles_n, all, per};
  const uint32_t grid = 8 * per;
  // rows of x and w that start on 16 bytes
  const bool direct = (int64_t)a.K * T::kBytes % 16 == 0 && ((uintptr_t)a.x | (uintptr_t)a.w) % 16 == 0;
  const auto go = [&](auto kernel) {
    return launch_in_parts(grid, [&](uint32_t first, uint32_t count) {
      kernel<<<count, kThreads, 0, stream>>>(a, map, first);
    });
  };
  const bool eights = a.N % 8 == 0;
  if (direct && eights) return go(linear_tile_kernel<T, O, WR, WN, RT, NT, STAGES, true, true>);
  if (direct) return go(linear_tile_kernel<T, O, WR, WN, RT, NT, STAGES, false, true>);
  if constexpr (WR * WN == 4) {
    if (eights) return go(linear_tile_kernel<T, O, WR, WN, RT, NT, 2, true, false>);
    return go(linear_tile_kernel<T, O, WR, WN, RT, NT, 2, false, false>);
  }
  return run_tile<T, O, 2, 2, 2, 2, 2>(a, stream);         // the held tile's registers are not free there
}

template <class T, int RT>
hipError_t run_few(const LinearArgs& a, hipStream_t stream) {
  const uint32_t tiles_r = (uint32_t)(((int64_t)a.R + 16 * RT - 1) / (16 * RT)), tiles_n = ((uint32_t)a.N + 15) / 16;
  return launch_in_parts((int64_t)tiles_r * tiles_n, [&](uint32_t first, uint32_t count) {
    linear_few_kernel<T, RT><<<count, kFewWaves * 64, 0, stream>>>(a, tiles_r, first);
  });
}

template <class T, class O>
hipError_t run(const LinearArgs& a, hipStream_t stream) {
  const auto tiles = [&](int br, int bn) {
    return ((int64_t)a.R + br - 1) / br * (((int64_t)a.N + bn - 1) / bn);
  };
  // Few rows: the weights' reading counts, and the few-rows kernel reads them from every
  // CU (16 x 1024 -> 4096 bf16 4.5 us against 6.4 with 64 x 64 tiles, 32 x 4096 -> 4096
  // 14.4 against 18.8; 64 x 4096 -> 4096 21.6 against 18.8).  Few tiles of fp32 too, whose
  // products take eight times as long: eight waves share a tile there (512 x 1024 -> 512
  // 12.7 us against 22.0, 1000 x 1021 -> 509 22.6 against 26.6; in bf16 21.9 against 10.2).
  const int64_t pitch = (int64_t)a.K * T::kBytes;
  if (a.R <= 32 || (T::kBytes == 4 && tiles(64, 64) <= 128) || pitch >= (1 << 22)) {
    if (a.R <= 16) return run_few<T, 1>(a, stream);
    return a.R <= 32 ? run_few<T, 2>(a, stream) : run_few<T, 4>(a, stream);
  }
  // The tile by what it takes in rounds of workgroups over the 256 CUs (one of 256 x 256
  // or two smaller ones on each) and by its rate: per output 128 x 128 tiles take 1.2
  // times as long as 256 x 256 and 64 x 64 1.9 times (16384 x 2048 -> 2048 bf16 116, 137
  // and 215 us); one smaller workgroup on a CU has it to itself.
  const auto cost = [&](int64_t n, int area, int per_cu, float rate) {
    const int64_t rounds = n <= 256 ? 1 : (n + 256 * per_cu - 1) / (256 * per_cu) * per_cu;
    return (float)(rounds * area) * rate;
  };
  const float c256 = cost(tiles(256, 256), 256 * 256, 1, 1.f), c128 = cost(tiles(128, 128), 128 * 128, 2, 1.2f),
              c64 = cost(tiles(64, 64), 64 * 64, 2, 1.9f);
  if (c64 <= c128 && c64 <= c256) return run_tile<T, O, 2, 2, 1, 1, 4>(a, stream);
  return c128 <= c256 ? run_tile<T, O, 2, 2, 2, 2, 2>(a, stream) : run_tile<T, O, 2, 4, 4, 2, 2>(a, stream);
}

template <class T>
hipError_t run_out(const LinearArgs& a, hipStream_t stream) {
  return a.out_dtype == GRACE_F32 ? run<T, F32>(a, stream) : run<T, BF16>(a, stream);
}

}  // namespace

hipError_t launch_linear(const void* x, const float* x_scale, const void* w, const float* w_scale,
                         const void* bias, const void* residual, int32_t R, int32_t N, int32_t K,
                         int32_t act, int32_t dtype, int32_t out_dtype, void* out,
                         hipStream_t stream) {
  const LinearArgs a{x, w, x_scale, w_scale, bias, residual, out, R, N, K, act, out_dtype};
  if (dtype == GRACE_F32) return run_out<F32>(a, stream);
  if (dtype == GRACE_BF16) return run_out<BF16>(a, stream);
  return out_dtype == GRACE_BF16 ? run<E4M3, BF16>(a, stream) : run<E4M3Wide, F32>(a, stream);
}

}  // namespace grace
