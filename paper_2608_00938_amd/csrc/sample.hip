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
// A draw next to a border has to fall as it does by the definition.  Rows in
// registers are decided with fp32 masses where these lie further from every border
// than they can be off, and else once more in fp64; the other rows are summed in
// fp64 throughout.
#include <float.h>
#include <math.h>

#include "common.hpp"
#include "kernels.hpp"
#include "wave.hpp"

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
  double T;            // 0: the best candidate; finite
  uint32_t k;          // most tokens kept
  double p, least;     // p >= 1: no rule; least weight of a token, <= 1
  __device__ Rules(const SampleArgs& a, int32_t b) {
    const float t = a.temperature ? a.temperature[b] : 1.f;
    T = t > 0.f ? (double)fminf(t, FLT_MAX) : 0.0;         // a NaN too
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

// ---------------------------------------------------------------------------
// One wave per row, the row in registers: rows of up to 512 * NCH tokens, lane l
// holding 8 consecutive tokens of every 512.
// ---------------------------------------------------------------------------
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));

__device__ __forceinline__ double wave_total(double x) {
  for (int s = 32; s > 0; s >>= 1) x += __shfl_xor(x, s);
  return x;
}
__device__ __forceinline__ float wave_total(float x) { return wave_sum(x); }
// Sum over the lanes up to this one.
template <class F>
__device__ __forceinline__ F wave_upto(F x) {
  const int lane = threadIdx.x & 63;
  for (int d = 1; d < 64; d <<= 1) {
    const F y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}
__device__ __forceinline__ float uniform(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
// Tokens of the wave for which each lane's bit is set.
__device__ __forceinline__ uint32_t lanes_with(bool b) {
  return (uint32_t)__builtin_popcountll(__ballot(b));
}

// How far fp32 masses are off, relative to the total: a weight's exponent a =
// (z - z_best) log2(e) / T is within 3 * 2^-24 |a| of its own (difference, factor and
// product rounded), which with the hardware's exp2 (one step) makes 2^-17.6 of a
// weight above 2^-40, and all smaller ones are below 2^-28 of the total; N + 8 additions
// of a sum add half a step each.
template <int N>
constexpr float mass_error() { return 0x1.6p-18f + (N + 8) * 0x1p-24f; }

// A row's tokens x (those that are no candidates -inf) under the rules; the token
// drawn.  F = double decides as the definition does.  F = float gives certain =
// false where a mass lies so near to a border that fp32 cannot tell its side.
template <class F, int N>
__device__ __forceinline__ int32_t draw(const float (&x)[N], float best, const Rules& rules, float u,
                                        bool& certain) {
  constexpr bool kExact = sizeof(F) == 8;
  const int lane = threadIdx.x & 63;
  const float c = (float)(1.4426950408889634 / rules.T);
  const auto weight = [&](float z) -> F {
    if constexpr (kExact) return z == best ? 1.0 : exp(((double)z - (double)best) / rules.T);
    else return z == best ? 1.f : fast_exp2((z - best) * c);
  };
  const auto count_from = [&](float t) {
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += lanes_with(x[i] >= t);
    return n;
  };
  const uint32_t best_key = uniform(order_key(best));
  // between two keys: halfway of the values and halfway of the keys in turn, so that
  // ordinary rows take few steps and any row at most 64
  const auto between = [&](uint32_t lo, uint32_t hi, int step) {
    uint32_t mid = lo + (hi - lo) / 2;
    if (step % 2 == 0) {
      const uint32_t k = order_key(0.5f * key_value(lo) + 0.5f * key_value(hi - 1));
      mid = uniform((uint32_t)min(max(k, lo + 1), hi - 1));
    }
    return mid;
  };

  // kept: values above `cut`, and the first `ties` tokens of value `cut`
  float cut = -INFINITY;
  uint32_t ties = 0xffffffffu, lo = 0x00800000u;            // key of the least finite fp32
  const uint32_t candidates = count_from(-FLT_MAX);
  uint32_t kept = candidates;
  if (rules.k < candidates) {
    uint32_t hi = best_key + 1, above = 0;                 // candidates from lo: more than k; from hi: `above` < k
    for (int step = 0;; ++step) {
      if (hi - lo == 1) {
        ties = rules.k - above;
        break;
      }
      const uint32_t mid = between(lo, hi, step), n = count_from(key_value(mid));
      if (n == rules.k) {
        lo = mid;
        break;
      }
      if (n > rules.k) lo = mid;
      else hi = mid, above = n;
    }
    cut = key_value(lo);
    kept = rules.k;
  }

  F w[N];
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = x[i] > -INFINITY ? weight(x[i]) : (F)0;
  const auto mass_from = [&](float t) {
    F m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m += x[i] >= t ? w[i] : (F)0;
    return wave_total(m);
  };
  constexpr F kOff = 2 * mass_error<N>();                  // of two masses' difference
  certain = true;
  if (rules.p < 1.0) {
    // all that top-k keeps: values above cut, and its ties
    const bool partial = ties != 0xffffffffu;
    F total = mass_from(key_value(lo + partial));
    if (partial) total += (F)ties * weight(cut);
    const F target = (F)rules.p * total, off = kOff * total;
    const uint32_t first = lo, first_ties = ties;
    uint32_t hi = best_key + 1;
    F mass_lo = total, mass_hi = 0;                        // from lo: at least the target; from hi: less
    uint32_t n_lo = kept, n_hi = 0;
    for (int step = 0; hi - lo > 1 && n_lo - n_hi > 1; ++step) {
      const uint32_t mid = between(lo, hi, step);
      const F m = mass_from(key_value(mid));
      const uint32_t n = count_from(key_value(mid));
      if (m >= target) lo = mid, mass_lo = m, n_lo = n;
      else hi = mid, mass_hi = m, n_hi = n;
    }
    // the best candidate is kept whatever the target
    const auto certain_of = [&](F past, F short_of, bool first_token) {
      return kExact || (past > off && (first_token || short_of > off));
    };
    if (n_lo - n_hi == 1) {
      // one token between: it reaches the target.  (Where it is one of top-k's cut
      // value, the ties stay top-k's.)
      certain = certain_of(mass_lo - target, target - mass_hi, n_hi == 0);
      if (lo != first) ties = 0xffffffffu;
    } else {
      // n_lo - n_hi tokens of one value
      const F each = weight(key_value(lo)), need = (target - mass_hi) / each, n = fmax(ceil(need), (F)1);
      certain = certain_of((n - need) * each, (need - n + 1) * each, n_hi == 0 && n == 1);
      ties = (uint32_t)n;
      if (lo == first) ties = min(ties, first_ties);
    }
    cut = key_value(lo);
  }

  // the kept weights in vocabulary order
  uint32_t seen = 0;                                       // tokens of value cut so far
  F sums[N / 8], all = 0;
#pragma unroll
  for (int ch = 0; ch < N / 8; ++ch) {
    F sum = 0;
    uint32_t rank = 0;
    if (ties != 0xffffffffu) {
      uint32_t mine = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) mine += x[ch * 8 + e] == cut;
      const uint32_t upto = wave_scan(mine);
      rank = seen + upto - mine;
      seen += __builtin_amdgcn_readlane(upto, 63);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = ch * 8 + e;
      bool in = x[i] >= cut && x[i] > -INFINITY;
      if (ties != 0xffffffffu && x[i] == cut) in = rank++ < ties;
      if (rules.least > 0) {
        const F least = (F)rules.least;
        if (!kExact && in && fabsf((float)(w[i] - least)) <= (float)(kOff * least)) certain = x[i] == best && certain;
        in = in && (w[i] >= least || x[i] == best);
      }
      w[i] = in ? w[i] : (F)0;
      sum += w[i];
    }
    sums[ch] = wave_upto(sum);
    all += __shfl(sums[ch], 63);
  }
  if (!kExact) certain = !__any(!certain);
  const F goal = (F)u * all;
  F before = 0;
  int32_t token = -1, start = -1;
#pragma unroll
  for (int ch = 0; ch < N / 8; ++ch) {
    const F end = before + __shfl(sums[ch], 63);
    const uint64_t past = __ballot(before + sums[ch] > goal);
    if (start < 0 && past) {
      const int l = __builtin_ctzll(past);
      start = (ch * 64 + l) * 8;
      // that lane's tokens, one after the other
      F run = before + (l ? __shfl(sums[ch], l ? l - 1 : 0) : (F)0);
      int32_t at = -1;
      bool clear = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const F next = run + w[ch * 8 + e];
        if (at < 0 && w[ch * 8 + e] > 0 && next > goal) {
          at = start + e;
          clear = goal - run > kOff * all && next - goal > kOff * all;
        }
        run = next;
      }
      token = __builtin_amdgcn_readlane(at, l);
      if (!kExact) certain = certain && __builtin_amdgcn_readlane((int)clear, l);
    }
    before = end;
  }
  if (token < 0) {
    // The sums' rounding alone: the first kept token from there on, or the last one.
    if (!kExact) certain = false;
    int32_t next = 0x7fffffff, last = -1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int32_t v = (i / 8 * 64 + lane) * 8 + i % 8;
      if (w[i] > 0) last = max(last, v);
      if (w[i] > 0 && start >= 0 && v >= start) next = min(next, v);
    }
    for (int s = 32; s > 0; s >>= 1) {
      next = min(next, __shfl_xor(next, s));
      last = max(last, __shfl_xor(last, s));
    }
    token = next != 0x7fffffff ? next : last;
  }
  return token;
}

template <class T, int NCH>
__global__ void __launch_bounds__(256) sample_wave_kernel(SampleArgs a) {
  constexpr int N = NCH * 8;
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (r >= a.R) return;                                    // whole waves
  const Rules rules(a, (int32_t)(r / a.M));
  float x[N];
  float top = -INFINITY;
  const typename T::storage* row = (const typename T::storage*)a.logits + r * a.V;
#pragma unroll
  for (int ch = 0; ch < NCH; ++ch) {
    const int32_t v = (ch * 64 + lane) * 8;
    if (v + 8 <= a.V) {
      u32x4 c = *(const u32x4_any*)(row + v);
      Chunk<T>::unpack(c, x + ch * 8);
      if constexpr (T::kBytes == 4) {
        c = *(const u32x4_any*)(row + v + 4);
        Chunk<T>::unpack(c, x + ch * 8 + 4);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[ch * 8 + e] = v + e < a.V ? logit_at<T>(a, r, v + e) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, x[ch * 8 + e]);
  }
  top = wave_max(top);
  float sum = 0;                                           // a NaN or +inf makes it NaN
#pragma unroll
  for (int i = 0; i < N; ++i) sum += fast_exp2((x[i] - top) * kLog2e);
  const float log_sum = logf(wave_sum(sum));
  float best = -INFINITY;
  const int64_t words = (a.V + 31) / 32;
#pragma unroll
  for (int ch = 0; ch < NCH; ++ch) {
    uint32_t bits = 0xff;
    if (a.mask) {
      const int32_t v = (ch * 64 + lane) * 8;
      bits = v < a.V ? ((const uint8_t*)(a.mask + r * words))[v / 8] : 0;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = ch * 8 + e;
      x[i] = fmaxf(keep_bit(x[i], bits, e), -INFINITY);    // a NaN is no candidate
      best = fmaxf(best, x[i]);
    }
  }
  best = uniform(wave_max(best));
  int32_t token = -1;
  if (best > -INFINITY) {
    if (rules.T > 0) {
      const float u = fminf(fmaxf(a.uniform[r], 0.f), kMostUniform);   // a NaN is 0
      bool certain;
      token = draw<float, N>(x, best, rules, u, certain);
      if (!certain) token = draw<double, N>(x, best, rules, u, certain);
    } else {
      token = 0x7fffffff;
#pragma unroll
      for (int i = N - 1; i >= 0; --i)
        if (x[i] == best) token = (i / 8 * 64 + lane) * 8 + i % 8;
      for (int s = 32; s > 0; s >>= 1) token = min(token, __shfl_xor(token, s));
    }
  }
  if (lane == 0) {
    const float prev = a.prev ? a.prev[r] : 0.f;
    a.tokens[r] = token;
    a.scores[r] = token < 0 ? -INFINITY : prev + (logit_at<T>(a, r, token) - top - log_sum);
  }
}

template <class T>
hipError_t run(const SampleArgs& a, hipStream_t stream) {
  const uint32_t waves = (uint32_t)(((int64_t)a.R + 3) / 4);
  if (a.V <= 512) sample_wave_kernel<T, 1><<<waves, 256, 0, stream>>>(a);
  else if (a.V <= 1024) sample_wave_kernel<T, 2><<<waves, 256, 0, stream>>>(a);
  else if (a.V <= 2048) sample_wave_kernel<T, 4><<<waves, 256, 0, stream>>>(a);
  else sample_kernel<T><<<a.R, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

int64_t sample_workspace_bytes(int32_t, int32_t, int32_t) { return 0; }

hipError_t launch_sample(const void* logits, const float* uniform, const float* prev,
                         const uint32_t* mask, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, int32_t B, int32_t M, int32_t V,
                         bool bf16, void*, int32_t* tokens, float* scores, hipStream_t stream) {
  const SampleArgs a{logits, uniform, prev, mask, temperature, top_k, top_p, min_p, tokens, scores,
                     B * M, M, V};
  return bf16 ? run<BF16>(a, stream) : run<F32>(a, stream);
}

}  // namespace grace
