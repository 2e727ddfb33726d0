// Sampling of a token per row with temperature, top-k, top-p and min-p, from
// given random numbers, for gfx950.
//
// A row's candidates are the tokens that the filter lets through with a logit
// above -inf, ordered by logit (descending), then by token (ascending).  With
// weights w = exp((z - z_best) / T), top-k keeps the first k of the order, top-p
// the shortest prefix of these whose mass reaches p of theirs, min-p those with
// w >= min_p.  The token is the first, in vocabulary order, whose running sum of
// kept weights exceeds u times their total.
//
// No sort: what each rule keeps is a prefix of the order, so it is a least key
// and how many tokens of that key are kept (the first in vocabulary order).  The
// keys are order-preserving bits of the logits, 0 for a token that is no
// candidate.
//
// Sums and weights are fp64, so that a draw next to a border falls as it does by
// the definition.
#include <math.h>

#include "common.hpp"
#include "kernels.hpp"

namespace grace {

namespace {

struct SampleArgs {
  const void* logits;
  const float *uniform, *prev;
  const uint32_t* mask;
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  int32_t *tokens;
  float* scores;
  int32_t R, M, V;
};

constexpr float kMostUniform = 1.f - 0x1p-24f;   // the largest fp32 below 1

// Order-preserving key of a logit above -inf; -0 as +0.
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k >> 31) ? k ^ 0x80000000u : ~k);
}

template <class T>
__device__ __forceinline__ float logit_at(const SampleArgs& a, int64_t r, int32_t v) {
  const typename T::storage* p = (const typename T::storage*)a.logits + r * a.V + v;
  if constexpr (T::kBytes == 4) return *p;
  else return bf16_bits_to_f32(*p);
}

// A request's rules, as every row of it applies them.
struct Rules {
  double T;            // 0: the best candidate
  uint32_t k;          // most tokens kept
  double p, least;     // p >= 1: no rule; least weight of a token, <= 1
  __device__ Rules(const SampleArgs& a, int32_t b) {
    const float t = a.temperature ? a.temperature[b] : 1.f;
    T = t > 0.f ? (double)t : 0.0;                         // a NaN too
    const int32_t n = a.top_k ? a.top_k[b] : 0;
    k = n > 0 ? (uint32_t)n : 0xffffffffu;
    const float q = a.top_p ? a.top_p[b] : 1.f;
    p = q > 0.f ? (double)q : 0.0;
    const float m = a.min_p ? a.min_p[b] : 0.f;
    least = m > 0.f ? fmin((double)m, 1.0) : 0.0;
  }
};

// The weight of a key; equal keys weigh the same, and the best key weighs 1.
__device__ __forceinline__ double weight_of(uint32_t key, uint32_t best, double T) {
  return key == best ? 1.0 : exp(((double)key_value(key) - (double)key_value(best)) / T);
}

constexpr int kThreads = 256, kWaves = kThreads / 64;

// Sum over the workgroup, for every thread.
template <class T>
__device__ T group_total(T x, T* scratch) {
  for (int s = 32; s > 0; s >>= 1) x += __shfl_xor(x, s);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = x;
  __syncthreads();
  x = scratch[0];
  for (int w = 1; w < kWaves; ++w) x += scratch[w];
  return x;
}
// Sum of the threads before this one, and of all.
template <class T>
__device__ T group_before(T x, T* scratch, T& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T s = x;
  for (int d = 1; d < 64; d <<= 1) {
    const T y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  __syncthreads();
  if (lane == 63) scratch[wave] = s;
  __syncthreads();
  T before = 0;
  all = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += scratch[w];
    all += scratch[w];
  }
  return before + s - x;
}

// One workgroup per row, the row read from memory at every step.  Any size.
template <class T>
__global__ void __launch_bounds__(kThreads) sample_kernel(SampleArgs a) {
  __shared__ double sums[kWaves];
  __shared__ uint32_t counts[kWaves];
  __shared__ int32_t found[2];
  const int tid = threadIdx.x;
  const int64_t r = blockIdx.x;
  const Rules rules(a, (int32_t)(r / a.M));
  const int64_t words = (a.V + 31) / 32;
  const auto key_at = [&](int32_t v) -> uint32_t {
    if (a.mask && !((a.mask[r * words + v / 32] >> (v % 32)) & 1)) return 0;
    const float z = logit_at<T>(a, r, v);
    return z > -INFINITY ? order_key(z) : 0u;              // a NaN is no candidate
  };

  // best candidate, and the whole row's log-sum-exp
  uint32_t best = 0;
  float top = -INFINITY;
  bool nan = false;
  for (int32_t v = tid; v < a.V; v += kThreads) {
    const float z = logit_at<T>(a, r, v);
    nan |= z != z;
    top = fmaxf(top, z);
    best = max(best, key_at(v));
  }
  uint32_t nans = nan;
  nans = group_total(nans, counts);
  for (int s = 32; s > 0; s >>= 1) {
    best = max(best, (uint32_t)__shfl_xor((int)best, s));
    top = fmaxf(top, __shfl_xor(top, s));
  }
  __syncthreads();
  if ((tid & 63) == 0) counts[tid >> 6] = best, sums[tid >> 6] = top;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) best = max(best, counts[w]), top = fmaxf(top, (float)sums[w]);
  __syncthreads();
  if (best == 0) {
    if (tid == 0) a.tokens[r] = -1, a.scores[r] = -INFINITY;
    return;
  }
  double e = 0;
  for (int32_t v = tid; v < a.V; v += kThreads) e += expf(logit_at<T>(a, r, v) - top);
  e = group_total(e, sums);

  const double T1 = rules.T > 0 ? rules.T : 1.0;
  const auto count_from = [&](uint32_t t) {                // candidates of key t and above
    uint32_t n = 0;
    for (int32_t v = tid; v < a.V; v += kThreads) n += key_at(v) >= t;
    return group_total(n, counts);
  };
  const auto mass_above = [&](uint32_t t) {                // of keys above t
    double m = 0;
    for (int32_t v = tid; v < a.V; v += kThreads) {
      const uint32_t k = key_at(v);
      if (k > t) m += weight_of(k, best, T1);
    }
    return group_total(m, sums);
  };

  // kept: keys above `cut`, and the first `ties` tokens of key `cut`
  uint32_t cut = 1, ties = 0xffffffffu;
  if (!(rules.T > 0)) {
    cut = best, ties = 1;
  } else if (rules.k < count_from(1)) {
    uint32_t lo = 1, hi = best;                            // count_from(lo) >= k always
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo + 1) / 2;
      if (count_from(mid) >= rules.k) lo = mid;
      else hi = mid - 1;
    }
    cut = lo;
    ties = rules.k - count_from(cut + 1);                  // keys end at that of +inf
  }
  if (rules.p < 1.0 && rules.T > 0) {
    // tokens of key cut that are kept (none where no rule has cut yet: key 1 is no logit's)
    const uint32_t at_cut = min(ties, count_from(cut) - count_from(cut + 1));
    const double end = at_cut ? at_cut * weight_of(cut, best, T1) : 0.0;
    const double target = rules.p * (mass_above(cut) + end);
    // the largest key whose mass, with all above, reaches the target
    uint32_t lo = cut, hi = best;
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo + 1) / 2;
      if (mass_above(mid - 1) >= target) lo = mid;
      else hi = mid - 1;
    }
    const double need = (target - mass_above(lo)) / weight_of(lo, best, T1);
    const uint32_t n = need > 1 ? (uint32_t)fmin(ceil(need), 4294967040.0) : 1;
    ties = lo == cut ? min(ties, n) : n;
    cut = lo;
  }

  // kept weights in vocabulary order: their total, then the draw
  uint32_t seen = 0;                                       // tokens of key cut so far
  const auto kept_weight = [&](int32_t base) {
    const int32_t v = base + tid;
    const uint32_t k = v < a.V ? key_at(v) : 0;
    uint32_t all;
    const uint32_t rank = seen + group_before((uint32_t)(k == cut), counts, all);
    seen += all;
    if (k < cut || k == 0 || (k == cut && rank >= ties)) return 0.0;
    const double w = weight_of(k, best, T1);
    return k == best || w >= rules.least ? w : 0.0;
  };
  double total = 0;
  for (int32_t base = 0; base < a.V; base += kThreads) total += group_total(kept_weight(base), sums);
  const float u = fminf(fmaxf(a.uniform[r], 0.f), kMostUniform);   // a NaN is 0
  const double goal = (double)u * total;
  if (tid == 0) found[0] = 0x7fffffff, found[1] = -1;
  __syncthreads();
  seen = 0;
  double before = 0;
  for (int32_t base = 0; base < a.V; base += kThreads) {
    const double w = kept_weight(base);
    double all;
    const double upto = before + group_before(w, sums, all) + w;
    if (w > 0) {
      if (upto > goal) atomicMin(&found[0], base + tid);
      atomicMax(&found[1], base + tid);
    }
    before += all;
    __syncthreads();
    if (found[0] != 0x7fffffff) break;
  }
  if (tid == 0) {
    const int32_t token = found[0] != 0x7fffffff ? found[0] : found[1];
    const float prev = a.prev ? a.prev[r] : 0.f;
    a.tokens[r] = token;
    a.scores[r] = nans ? NAN : prev + (float)((double)logit_at<T>(a, r, token) - (double)top - log(e));
  }
}

}  // namespace

int64_t sample_workspace_bytes(int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_sample(const void* logits, const float* uniform, const float* prev,
                         const uint32_t* mask, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, int32_t B, int32_t M, int32_t V,
                         bool bf16, void*, int32_t* tokens, float* scores, hipStream_t stream) {
  const SampleArgs a{logits, uniform, prev, mask, temperature, top_k, top_p, min_p, tokens, scores,
                     B * M, M, V};
  if (bf16) sample_kernel<BF16><<<a.R, kThreads, 0, stream>>>(a);
  else sample_kernel<F32><<<a.R, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace grace
