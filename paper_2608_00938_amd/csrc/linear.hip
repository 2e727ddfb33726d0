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
// a chunk at any address: the hardware takes 16-byte loads off their alignment
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
  if (act == GRACE_ACT_GELU) return 0.5f * y * (1.f + erff(y * 0.70710678118654752f));
  if (act == GRACE_ACT_SILU) return y / (1.f + expf(-y));
  return y;
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

// Chunk c of row `row` (clamped into the matrix) at element k, zeros past K.
template <class T>
__device__ __forceinline__ u32x4 load_chunk(const void* base, int64_t row, int32_t K, int32_t k) {
  constexpr int E = 16 / T::kBytes;
  const typename T::storage* p = (const typename T::storage*)base + row * K + k;
  if (k + E <= K) return *(const u32x4_any*)p;
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (k + e < K) {
      uint32_t bits;
      if constexpr (T::kBytes == 4) bits = __float_as_uint(p[e]);
      else bits = p[e];
      v[e * T::kBytes / 4] |= bits << (e * T::kBytes % 4 * 8);
    }
  }
  return v;
}

// Four waves, WR x WN of them, of RT x NT tiles of 32 x 32 each; tiles of 128
// bytes of k pass through registers into LDS, the next one under the products
// of the current one.  Takes any size and alignment.
template <class T, int WR, int WN, int RT, int NT>
__global__ void __launch_bounds__(256) linear_kernel(LinearArgs a) {
  static_assert(WR * WN == 4, "four waves");
  constexpr int BR = WR * RT * 32, BN = WN * NT * 32, kPer = (BR + BN) * kRowChunks / 256;
  constexpr int kTileK = 128 / T::kBytes;
  using S = Step<T>;
  __shared__ u32x4 lds[(BR + BN) * kRowChunks];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int half = lane >> 5, col = lane & 31;
  const int64_t tiles_r = ((int64_t)a.R + BR - 1) / BR;
  const int64_t r0 = blockIdx.x % tiles_r * BR;
  const int32_t n0 = (int32_t)(blockIdx.x / tiles_r * BN);

  u32x4 next[kPer];
  auto fetch = [&](int32_t k0) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int chunk = tid + i * 256, row = chunk / kRowChunks;
      const int32_t k = k0 + chunk % kRowChunks * (16 / T::kBytes);
      if (row < BR) next[i] = load_chunk<T>(a.x, min(r0 + row, (int64_t)a.R - 1), a.K, k);
      else next[i] = load_chunk<T>(a.w, min((int64_t)n0 + row - BR, (int64_t)a.N - 1), a.K, k);
    }
  };
  f32x16 acc[RT][NT];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x16{0};
  fetch(0);
  const int wr = wave / WN * RT * 32, wn = BR + wave % WN * NT * 32;
  for (int64_t k0 = 0; k0 < a.K; k0 += kTileK) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int chunk = tid + i * 256;
      lds[slot(chunk / kRowChunks, chunk % kRowChunks)] = next[i];
    }
    __syncthreads();
    if (k0 + kTileK < a.K) fetch((int32_t)(k0 + kTileK));
#pragma unroll
    for (int s = 0; s < S::kSteps; ++s) {
      typename S::Frag fr[RT], fn[NT];
      const auto frag = [&](int row) {
        u32x4 c[S::kChunks];
#pragma unroll
        for (int i = 0; i < S::kChunks; ++i) c[i] = lds[slot(row, (s * 2 + half) * S::kChunks + i)];
        return S::make(c);
      };
#pragma unroll
      for (int i = 0; i < RT; ++i) fr[i] = frag(wr + i * 32 + col);
#pragma unroll
      for (int j = 0; j < NT; ++j) fn[j] = frag(wn + j * 32 + col);
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = S::run(fn[j], fr[i], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    const int64_t r = r0 + wr + i * 32 + col;
    if (r >= a.R) continue;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float v[4] = {acc[i][j][g * 4], acc[i][j][g * 4 + 1], acc[i][j][g * 4 + 2],
                            acc[i][j][g * 4 + 3]};
        finish4(a, r, n0 + (wn - BR) + j * 32 + g * 8 + half * 4, v);
      }
  }
}

template <class T>
hipError_t run(const LinearArgs& a, hipStream_t stream) {
  const int64_t tiles = (((int64_t)a.R + 63) / 64) * (((int64_t)a.N + 63) / 64);
  linear_kernel<T, 2, 2, 1, 1><<<(uint32_t)tiles, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(const void* x, const float* x_scale, const void* w, const float* w_scale,
                         const void* bias, const void* residual, int32_t R, int32_t N, int32_t K,
                         int32_t act, int32_t dtype, int32_t out_dtype, void* out,
                         hipStream_t stream) {
  const LinearArgs a{x, w, x_scale, w_scale, bias, residual, out, R, N, K, act, out_dtype};
  if (dtype == GRACE_F32) return run<F32>(a, stream);
  if (dtype == GRACE_BF16) return run<BF16>(a, stream);
  return out_dtype == GRACE_BF16 ? run<E4M3>(a, stream) : run<E4M3Wide>(a, stream);
}

}  // namespace grace
