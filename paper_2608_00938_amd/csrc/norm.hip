// Root-mean-square norm of the residual stream for gfx950: the residual's
// addition, the norm and the output's rounding (or its scaling into 8 bits) in
// one pass over the rows.
//
//   h = x + residual,  y = h / sqrt(mean(h^2) + eps) * weight
//
// A row stays in the registers of the NT lanes that own it (a wave up to 2048
// elements, a workgroup above), so every input is read once and every output
// written once: the bound is HBM (262144 x 1024 bf16 with residual and sum 372 us =
// 5.8 TB/s, 16384 x 2048 to e4m3 51 us; a wave per row needs no barrier, and rows too
// long for its registers take more waves).  Sums, the mean and the row's largest value
// are fp32; h is rounded to the stream's type only where it is stored, the norm
// takes the unrounded sum.
#include "common.hpp"
#include "kernels.hpp"

namespace grace {

namespace {

constexpr int kPerLane = 32;               // most row elements that a lane holds
constexpr float kE4m3Max = 448.f;
constexpr uint32_t kTinyBits = 0x0f800000u;  // 2^-96, the least maximum a scale is made from

// Sum or maximum over the NT lanes of a row; every lane gets it.  scratch: one
// word per wave and call, of the workgroup's own.
template <int NT>
__device__ __forceinline__ float row_sum(float x, float* scratch) {
  x = group_sum<32>(x);
  x += __shfl_xor(x, 32);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) x += scratch[w];
  }
  return x;
}
template <int NT>
__device__ __forceinline__ uint32_t row_max(uint32_t x, uint32_t* scratch) {
#pragma unroll
  for (int s = 1; s < 64; s *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, s));
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) x = max(x, scratch[w]);
  }
  return x;
}

// Loads and stores at any address: the hardware takes them off their alignment.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32_any __attribute__((aligned(1)));

// E (a 16-byte chunk) elements from element `at` of a row of D as fp32, those past
// its end 0.
template <class T>
__device__ __forceinline__ void load_elems(const typename T::storage* row, int32_t at, int32_t D, float* f) {
  constexpr int E = Chunk<T>::kElems;
  if (at + E <= D) {
    const u32x4 c = *(const u32x4_any*)(row + at);
    Chunk<T>::unpack(c, f);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      f[e] = 0.f;
      if (at + e < D) {
        if constexpr (T::kBytes == 4) f[e] = row[at + e];
        else f[e] = bf16_bits_to_f32(row[at + e]);
      }
    }
  }
}

// The same back, rounded to type TO.
template <int TO, int E>
__device__ __forceinline__ void store_elems(void* row, int32_t at, int32_t D, const float* f) {
  if (at + E <= D) {
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      if constexpr (TO == GRACE_F32)
        *(u32x4_any*)((float*)row + at + e) = u32x4{__float_as_uint(f[e]), __float_as_uint(f[e + 1]),
                                                    __float_as_uint(f[e + 2]), __float_as_uint(f[e + 3])};
      else if constexpr (TO == GRACE_E4M3 && E == 4)
        *(u32_any*)((uint8_t*)row + at) = pack_e4m3x4(f[0], f[1], f[2], f[3]);
      else if constexpr (TO == GRACE_BF16 && E == 4)
        *(u32x2_any*)((uint16_t*)row + at) = u32x2{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
    }
    if constexpr (TO == GRACE_BF16 && E == 8) *(u32x4_any*)((uint16_t*)row + at) = Chunk<BF16>::pack(f);
    if constexpr (TO == GRACE_E4M3 && E == 8)
      *(u32x2_any*)((uint8_t*)row + at) = u32x2{pack_e4m3x4(f[0], f[1], f[2], f[3]),
                                                pack_e4m3x4(f[4], f[5], f[6], f[7])};
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (at + e < D) {
        if constexpr (TO == GRACE_F32) ((float*)row)[at + e] = f[e];
        else if constexpr (TO == GRACE_BF16) ((uint16_t*)row)[at + e] = (uint16_t)pack_bf16x2(f[e], 0.f);
        else ((uint8_t*)row)[at + e] = (uint8_t)pack_e4m3x4(f[e], 0.f, 0.f, 0.f);
      }
  }
}

// NT lanes own a row; lane i takes the 16-byte groups of E elements at (i + j * NT) * E.
// Rows and tensors may start anywhere; a row's last group may be short.
template <class T, int NT, int NG, int OUT>
__global__ void __launch_bounds__(NT == 64 ? 256 : NT)
rms_norm_kernel(const typename T::storage* x, const typename T::storage* residual,
                const typename T::storage* weight, typename T::storage* sum, void* out,
                float* out_scale, int32_t R, int32_t D, float eps, uint32_t first) {
  __shared__ float scratch[2][NT / 64];
  constexpr int kRows = NT == 64 ? 4 : 1;      // rows of a workgroup
  const int lane = threadIdx.x % NT;
  const int64_t r = (int64_t)(first + blockIdx.x) * kRows + threadIdx.x / NT;
  if (r >= R) return;                          // whole waves of a one-wave row only
  constexpr int E = Chunk<T>::kElems;
  constexpr int kOutBytes = OUT == GRACE_F32 ? 4 : (OUT == GRACE_BF16 ? 2 : 1);
  const int64_t row = r * D;
  float h[NG][E], w[NG][E];
  // everything is read before the first write: sum may be x or residual itself
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int32_t at = (lane + j * NT) * E;
    if (at < D) load_elems<T>(x + row, at, D, h[j]);
    else
#pragma unroll
      for (int e = 0; e < E; ++e) h[j][e] = 0.f;
  }
  if (residual) {
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      const int32_t at = (lane + j * NT) * E;
      if (at < D) {
        float a[E];
        load_elems<T>(residual + row, at, D, a);
#pragma unroll
        for (int e = 0; e < E; ++e) h[j][e] += a[e];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int32_t at = (lane + j * NT) * E;
    if (at < D) load_elems<T>(weight, at, D, w[j]);
  }
  float ss = 0.f;
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int32_t at = (lane + j * NT) * E;
    if (sum && at < D) store_elems<T::kBytes == 4 ? GRACE_F32 : GRACE_BF16, E>(sum + row, at, D, h[j]);
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(h[j][e], h[j][e], ss);
  }
  const float inv = rsqrtf(row_sum<NT>(ss, scratch[0]) / (float)D + eps);
  uint32_t top = kTinyBits;                    // of |y| as bits, so that a NaN stays
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int32_t at = (lane + j * NT) * E;
    if (at < D) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        h[j][e] = h[j][e] * inv * w[j][e];
        if constexpr (OUT == GRACE_E4M3) top = max(top, __float_as_uint(h[j][e]) & 0x7fffffffu);
      }
    }
  }
  if constexpr (OUT == GRACE_E4M3) {
    const float amax = __uint_as_float(row_max<NT>(top, (uint32_t*)scratch[1]));
    const float up = kE4m3Max / amax;
    if (lane == 0) out_scale[r] = amax / kE4m3Max;
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int e = 0; e < E; ++e) h[j][e] *= up;
  }
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int32_t at = (lane + j * NT) * E;
    if (at < D) store_elems<OUT, E>((char*)out + row * kOutBytes, at, D, h[j]);
  }
}

struct NormArgs {
  const void *x, *residual, *weight;
  void *sum, *out;
  float* scale;
  int32_t R, D;
  float eps;
  hipStream_t stream;
};

template <class T, int NT, int NG, int OUT>
hipError_t run(const NormArgs& a) {
  using S = typename T::storage;
  const int64_t rows = NT == 64 ? 4 : 1;
  return launch_in_parts((a.R + rows - 1) / rows, [&](uint32_t first, uint32_t count) {
    rms_norm_kernel<T, NT, NG, OUT><<<count, NT == 64 ? 256 : NT, 0, a.stream>>>(
        (const S*)a.x, (const S*)a.residual, (const S*)a.weight, (S*)a.sum, a.out, a.scale, a.R, a.D,
        a.eps, first);
  });
}

// Groups per lane, the least power of two that holds the row.
template <class T, int NT, int OUT>
hipError_t pick_groups(const NormArgs& a) {
  constexpr int E = Chunk<T>::kElems, kMost = kPerLane / E;
  const int32_t need = (a.D + NT * E - 1) / (NT * E);
  if constexpr (kMost >= 8) {
    if (need > 4) return run<T, NT, 8, OUT>(a);
  }
  if (need > 2) return run<T, NT, 4, OUT>(a);
  return need > 1 ? run<T, NT, 2, OUT>(a) : run<T, NT, 1, OUT>(a);
}

template <class T, int OUT>
hipError_t pick_lanes(const NormArgs& a) {
  if (a.D <= 64 * kPerLane) return pick_groups<T, 64, OUT>(a);
  if (a.D <= 256 * kPerLane) return pick_groups<T, 256, OUT>(a);
  return pick_groups<T, 1024, OUT>(a);
}

template <class T>
hipError_t pick_out(const NormArgs& a, int32_t out_dtype) {
  if (out_dtype == GRACE_F32) return pick_lanes<T, GRACE_F32>(a);
  if (out_dtype == GRACE_BF16) return pick_lanes<T, GRACE_BF16>(a);
  return pick_lanes<T, GRACE_E4M3>(a);
}

}  // namespace

int32_t rms_norm_max_d() { return 1024 * kPerLane; }

hipError_t launch_rms_norm(const void* x, const void* residual, const void* weight, int32_t R,
                           int32_t D, float eps, int32_t dtype, int32_t out_dtype, void* sum,
                           void* out, float* out_scale, hipStream_t stream) {
  const NormArgs a{x, residual, weight, sum, out, out_scale, R, D, eps, stream};
  return dtype == GRACE_BF16 ? pick_out<BF16>(a, out_dtype) : pick_out<F32>(a, out_dtype);
}

}  // namespace grace
