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
// than they can be off, and else once more in fp64; longer rows are summed in fp64
// throughout.
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
  uint32_t first;              // of the launch's workgroups
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

__device__ __forceinline__ float uniform(float x) {
  return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x)));
}
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }

template <int CTRL, int ROWS>
__device__ __forceinline__ float shifted(float x) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xF, false));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double shifted(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xF, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Sum over the lanes up to this one, in the vector ALU.
template <class F>
__device__ __forceinline__ F wave_upto(F x) {
  x += shifted<0x111, 0xF>(x);   // row_shr:1
  x += shifted<0x112, 0xF>(x);   // row_shr:2
  x += shifted<0x114, 0xF>(x);   // row_shr:4
  x += shifted<0x118, 0xF>(x);   // row_shr:8
  x += shifted<0x142, 0xA>(x);   // row_bcast:15
  x += shifted<0x143, 0xC>(x);   // row_bcast:31
  return x;
}
__device__ __forceinline__ float lane_of(float x, int l) { return lane_value(x, l); }
__device__ __forceinline__ double lane_of(double x, int l) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, l);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), l);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_total(double x) { return lane_of(wave_upto(x), 63); }
__device__ __forceinline__ float wave_total(float x) { return uniform(wave_sum(x)); }

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

// ---------------------------------------------------------------------------
// One workgroup per row, for rows longer than a wave's registers hold.
//
// What each rule keeps is found in a histogram instead of a search over the row:
// one sweep counts the candidates by the upper half of their bits, which for bf16
// is their value, with each bin's mass; fp32 bins, and the one bin of the values
// next to zero, are cut again by their keys where a border falls into them.  A
// sweep then adds up the kept weights of each wave's piece of the vocabulary, the
// piece with the drawn token is dealt out again over the waves, and so on down to
// 512 tokens, which one wave goes through.  32 rows of 128000 bf16 take 74 us, bound by
// the vector ALU of the 32 CUs and the chain of steps; up to 8192 tokens 256 threads
// have the shorter chain, and two rows share a CU.
//
// All sums are fp64, whose exp2 costs a sweep some 90 cycles per wave of tokens; of
// bf16 only the bins need it.  fp32 bins are added by fp64 atomics in no fixed order,
// which moves a mass by less than 2^-40 of the row's.  Candidates whose weight is below
// 2^-63 are left out: all of a row's together are below 2^-39 of the total, a part that
// decides nothing but draws with u below 2^-30, which leave none out.
// ---------------------------------------------------------------------------
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(1)));

// 2^x for x <= 0, by the series of exp(f ln 2) on |f| <= 1/2 (to f^11: 6e-15).
__device__ __forceinline__ double exp2_f64(double x) {
  x = fmax(x, -1100.0);                                    // 0, for -inf too
  const double n = rint(x), y = (x - n) * 0.69314718055994530942;
  double s = 1.0 / 39916800;
  s = fma(s, y, 1.0 / 3628800);
  s = fma(s, y, 1.0 / 362880);
  s = fma(s, y, 1.0 / 40320);
  s = fma(s, y, 1.0 / 5040);
  s = fma(s, y, 1.0 / 720);
  s = fma(s, y, 1.0 / 120);
  s = fma(s, y, 1.0 / 24);
  s = fma(s, y, 1.0 / 6);
  s = fma(s, y, 0.5);
  s = fma(s, y, 1.0);
  s = fma(s, y, 1.0);
  return ldexp(s, (int)n);
}

// Bins by value, the largest first: kSide bins above zero, 128 to an octave, the last of
// 16 octaves above the row's largest magnitude; one bin for the smaller values of either
// sign; kSide below zero.  -inf, +inf and NaN fall into the outermost bins, which no
// other value of the row does.
struct Bins {
  static constexpr int kSide = 16 * 128, kCount = 2 * kSide + 1;
  int base;                                                // upper half of the bits below a side's first bin
  __device__ explicit Bins(float most) {
    const int e = (int)(__float_as_uint(most) >> 23 & 255) - 14;
    base = (max(e, 1) << 7) - 1;
  }
  __device__ __forceinline__ int of(float x) const {
    const uint32_t bits = __float_as_uint(x);
    const int out = min(max((int)(bits >> 16 & 0x7fff) - base, 0), kSide), sign = (int)bits >> 31;
    return kSide + ((out ^ ~sign) - ~sign);                // + out below zero, - out above
  }
  // Keys of a bin: [lo, hi).
  __device__ void keys(int bin, uint32_t& lo, uint32_t& hi) const {
    const int out = bin < kSide ? kSide - bin : bin - kSide;
    const uint32_t from = (uint32_t)(base + max(out, 1)) << 16, to = from + (1u << 16);   // magnitudes
    if (bin < kSide) {
      lo = 0x80000000u + from;
      hi = out == kSide ? 0xffffffffu : 0x80000000u + to;
    } else if (bin == kSide) {
      lo = 0x80000000u - from, hi = 0x80000000u + from;
    } else {
      lo = out == kSide ? 0u : 0x80000000u - to;
      hi = 0x80000000u - from;
    }
  }
};

template <class T, int NT>
struct RowSampler {
  static constexpr int kWaves = NT / 64, kParts = 1024;
  struct Shared {
    uint32_t count[Bins::kCount];
    double mass[Bins::kCount];                             // then, of bf16, a bin's weight
    uint32_t part_count[kParts];
    double part_mass[kParts];
    double sums[kWaves];
    uint32_t counts[kWaves];
    float tops[kWaves], bests[kWaves];
    int32_t found;
    uint32_t found_count;
    double found_mass;
  };
  const SampleArgs& a;
  Shared& s;
  const int64_t r;
  const int tid, lane, wave;
  const typename T::storage* row;
  const uint8_t* mask;                                     // the row's filter words, by bytes
  float best;
  double scale;                                            // log2(e) / T
  float least_x;                                           // candidates from here on count

  __device__ RowSampler(const SampleArgs& a_, Shared& s_)
      : a(a_), s(s_), r(a_.first + blockIdx.x), tid(threadIdx.x), lane(tid & 63),
        wave(__builtin_amdgcn_readfirstlane(tid >> 6)),
        row((const typename T::storage*)a_.logits + r * a_.V),
        mask(a_.mask ? (const uint8_t*)(a_.mask + r * ((a_.V + 31) / 32)) : nullptr) {}

  // Eight tokens from v on, a multiple of 8, as they lie in memory (-inf past the row's
  // end), and their filter bits.
  struct Raw {
    u32x4 c[T::kBytes / 2];
    uint32_t bits;
  };
  __device__ __forceinline__ Raw fetch(int32_t v) const {
    Raw x;
    if (v + 8 <= a.V) {
#pragma unroll
      for (int i = 0; i < T::kBytes / 2; ++i) x.c[i] = *(const u32x4_any*)(row + v + i * 4);
    } else {
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = v + e < a.V ? logit_at<T>(a, r, v + e) : -INFINITY;
#pragma unroll
      for (int i = 0; i < T::kBytes / 2; ++i) x.c[i] = Chunk<T>::pack(f + i * 4);
    }
    x.bits = mask && v < a.V ? mask[v / 8] : 0xff;
    return x;
  }
  __device__ __forceinline__ static void logits(const Raw& raw, float* x) {
#pragma unroll
    for (int i = 0; i < T::kBytes / 2; ++i) Chunk<T>::unpack(raw.c[i], x + i * 4);
  }
  // What is no candidate to -inf: filtered tokens, NaN.
  __device__ __forceinline__ static void filter(const Raw& raw, float* x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fmaxf(keep_bit(x[e], raw.bits, e), -INFINITY);
  }
  // f(raw) for the eights of this wave's piece of [lo, hi) (lo a multiple of 512); pieces
  // are multiples of 512.  The next two eights are under way while f has one: else the
  // wave waits for the L2 at each.
  __device__ static int32_t piece(int32_t lo, int32_t hi) {
    return ((hi - lo + kWaves - 1) / kWaves + 511) / 512 * 512;
  }
  template <class F>
  __device__ __forceinline__ void sweep_raw(int32_t lo, int32_t hi, F f) const {
    const int32_t n = piece(lo, hi), from = lo + wave * n, to = min(hi, from + n);
    if (from >= to) return;
    Raw x = fetch(from + lane * 8), y = x;
    if (from + 512 < to) y = fetch(from + 512 + lane * 8);
    for (int32_t v = from; v < to; v += 512) {
      Raw z = y;
      if (v + 1024 < to) z = fetch(v + 1024 + lane * 8);
      f(x);
      x = y, y = z;
    }
  }
  // f(x), the candidates' logits, -inf for others
  template <class F>
  __device__ __forceinline__ void sweep(int32_t lo, int32_t hi, F f) const {
    sweep_raw(lo, hi, [&](const Raw& raw) __attribute__((always_inline)) {
      float x[8];
      logits(raw, x);
      filter(raw, x);
      f(x);
    });
  }
  __device__ __forceinline__ double weight(float x) const {
    return x == best ? 1.0 : exp2_f64(((double)x - (double)best) * scale);
  }

  // Sum over the waves of what each wave has, for every thread.
  template <class V>
  __device__ V over_waves(V x, V* scratch) {
    __syncthreads();
    if (lane == 0) scratch[wave] = x;
    __syncthreads();
    V all = 0;
    for (int w = 0; w < kWaves; ++w) all += scratch[w];
    return all;
  }
  __device__ __forceinline__ static double lanes_upto(double x) { return wave_upto(x); }
  __device__ __forceinline__ static uint32_t lanes_upto(uint32_t x) { return wave_scan(x); }
  template <class V>
  __device__ __forceinline__ static V lanes_total(V x) {
    const V upto = lanes_upto(x);
    if constexpr (sizeof(V) == 8) return lane_of(upto, 63);
    else return (V)__builtin_amdgcn_readlane((int)upto, 63);
  }

  // In a histogram of n bins: the first bin with which the count reaches n_goal (by =
  // 0) or the mass m_goal (by = 1), and what lies before it; -1 if none does.
  __device__ int locate(const uint32_t* count, const double* mass, int n, int by, uint32_t n_goal,
                        double m_goal, uint32_t& n_before, double& m_before) {
    const int each = (n + NT - 1) / NT, lo = min(tid * each, n), hi = min(lo + each, n);
    uint32_t c = 0;
    double m = 0;
    for (int i = lo; i < hi; ++i) c += count[i], m += mass[i];
    const uint32_t cu = lanes_upto(c);
    const double mu = lanes_upto(m);
    __syncthreads();
    if (lane == 63) s.counts[wave] = cu, s.sums[wave] = mu;
    if (tid == 0) s.found = -1;
    __syncthreads();
    uint32_t cb = cu - c;
    double mb = 0;
    for (int w = 0; w < wave; ++w) cb += s.counts[w], mb += s.sums[w];
    // a lane's mass before is the sum that the lane below ends with, so that the lanes agree
    const double below = __shfl_up(mu, 1);
    const double end = mb + mu;
    mb += lane ? below : 0.0;
    const bool here = by ? mb < m_goal && end >= m_goal : cb < n_goal && cb + c >= n_goal;
    if (here) {                                            // rounding aside one of its bins; else its last
      for (int i = lo; i < hi; ++i) {
        if (!count[i]) continue;
        s.found = i, s.found_count = cb, s.found_mass = mb;
        cb += count[i], mb += mass[i];
        if (by ? mb >= m_goal : cb >= n_goal) break;
      }
    }
    __syncthreads();
    n_before = s.found_count, m_before = s.found_mass;
    const int found = s.found;
    __syncthreads();
    return found;
  }

  // Narrows the keys [lo, hi), which the border falls into, to one key or one token;
  // n_before, m_before: candidates and mass above hi.  n_at, m_at: those left in [lo, hi).
  __device__ void narrow(uint32_t& lo, uint32_t& hi, int by, uint32_t n_goal, double m_goal,
                         uint32_t& n_before, double& m_before, uint32_t& n_at, double& m_at) {
    while (hi - lo > 1 && n_at > 1) {
      const int shift = max(0, 22 - __builtin_clz(hi - lo - 1));   // (hi - lo - 1) >> shift < 1024
      for (int i = tid; i < kParts; i += NT) s.part_count[i] = 0, s.part_mass[i] = 0;
      __syncthreads();
      sweep(0, a.V, [&](const float* x) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t k = order_key(x[e]);
          if (x[e] >= least_x && k >= lo && k < hi) {
            const uint32_t i = (hi - 1 - k) >> shift;
            atomicAdd(&s.part_count[i], 1u);
            unsafeAtomicAdd(&s.part_mass[i], weight(x[e]));
          }
        }
      });
      __syncthreads();
      uint32_t nb;
      double mb;
      int i = locate(s.part_count, s.part_mass, kParts, by, n_goal - n_before, m_goal - m_before, nb, mb);
      if (i < 0) {                                         // rounding alone: the last of them
        for (i = kParts - 1; i > 0 && !s.part_count[i]; --i) {}
        nb = 0, mb = 0;
        for (int j = 0; j < i; ++j) nb += s.part_count[j], mb += s.part_mass[j];
      }
      n_before += nb, m_before += mb, n_at = s.part_count[i], m_at = s.part_mass[i];
      const uint32_t end = hi - ((uint32_t)i << shift), width = 1u << shift;
      lo = end - lo > width ? end - width : lo;
      hi = end;
      __syncthreads();
    }
  }

  __device__ void run() {
    const Rules rules(a, (int32_t)(r / a.M));
    // best candidate and largest logit
    float top = -INFINITY, most = -INFINITY;
    {
      sweep_raw(0, a.V, [&](const Raw& raw) __attribute__((always_inline)) {
        float x[8];
        logits(raw, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, x[e]);
        filter(raw, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmaxf(most, x[e]);
      });
      top = wave_max(top), most = wave_max(most);
      if (lane == 0) s.tops[wave] = top, s.bests[wave] = most;
      for (int i = tid; i < Bins::kCount; i += NT) s.count[i] = 0, s.mass[i] = 0;
      __syncthreads();
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, s.tops[w]), most = fmaxf(most, s.bests[w]);
      best = most;
    }
    if (!(best > -INFINITY)) {
      if (tid == 0) a.tokens[r] = -1, a.scores[r] = -INFINITY;
      return;
    }
    const float u = fminf(fmaxf(a.uniform[r], 0.f), kMostUniform);   // a NaN is 0
    const bool greedy = !(rules.T > 0);
    const double temp = greedy ? 1.0 : rules.T;
    scale = 1.4426950408889634 / temp;
    // (finite, so that it keeps -inf out too)
    least_x = greedy ? best : fmaxf((float)((double)best - (u < 0x1p-30f ? 1100 : 63) * 0.6931471805599453 * temp), -FLT_MAX);
    const Bins bins(fmaxf(fabsf(best), fabsf(least_x)));
    const bool cuts = !greedy && (rules.k < (uint32_t)a.V || rules.p < 1.0);

    // the row's sum of exp, and the histogram
    float e1 = 0;
    sweep_raw(0, a.V, [&](const Raw& raw) __attribute__((always_inline)) {
      float x[8];
      logits(raw, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) e1 += fast_exp2((x[e] - top) * kLog2e);   // a NaN or +inf makes it NaN
      if (!cuts) return;
      filter(raw, x);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (x[e] >= least_x) {
          const int b = bins.of(x[e]);
          atomicAdd(&s.count[b], 1u);
          if (kMasses || b == Bins::kSide) unsafeAtomicAdd(&s.mass[b], weight(x[e]));
        }
    });
    const float log_sum = logf((float)over_waves((double)wave_sum(e1), s.sums));

    // kept: values above cut, and the first `ties` tokens of value cut
    float cut = greedy ? best : -INFINITY;
    uint32_t ties = greedy ? 1u : 0xffffffffu;
    if (cuts) {
      if (!kMasses) {                                    // a bin of bf16 is one value
        for (int i = tid; i < Bins::kCount; i += NT)
          if (s.count[i] && i != Bins::kSide) {
            uint32_t lo, hi;
            bins.keys(i, lo, hi);
            s.mass[i] = s.count[i] * weight(bf16_of_keys(lo, hi));
          }
        __syncthreads();
      }
      uint32_t lo = 0, hi = 0, n_before, n_at;
      double m_before, m_at;
      const auto border = [&](int by, uint32_t n_goal, double m_goal) {
        const int bin = locate(s.count, s.mass, Bins::kCount, by, n_goal, m_goal, n_before, m_before);
        if (bin < 0) return false;
        n_at = s.count[bin], m_at = s.mass[bin];
        bins.keys(bin, lo, hi);
        if (kMasses || bin == Bins::kSide) narrow(lo, hi, by, n_goal, m_goal, n_before, m_before, n_at, m_at);
        else lo = order_key(bf16_of_keys(lo, hi));
        return true;
      };
      double total = -1;                                   // the mass that top-k keeps
      if (rules.k < (uint32_t)a.V && border(0, rules.k, 0)) {
        cut = key_value(lo);
        ties = rules.k - n_before;
        total = m_before + (n_at <= ties ? m_at : ties * weight(cut));
        if (n_at <= ties) ties = 0xffffffffu;              // all of them: no rank to keep
      }
      if (rules.p < 1.0) {
        if (total < 0) {
          double m = 0;
          for (int i = tid; i < Bins::kCount; i += NT) m += s.mass[i];
          total = over_waves(lanes_total(m), s.sums);
        }
        const double target = rules.p * total;
        if (!(target > 0)) {
          cut = best, ties = 1;
        } else if (border(1, 0, target)) {
          const float at = key_value(lo);
          if (n_at == 1 && hi - lo > 1) {
            // one token between the keys: it reaches the target
            if (at > cut) cut = at, ties = 0xffffffffu;
          } else {
            const double need = ceil((target - m_before) / weight(at));
            const uint32_t first = need > 1 ? (uint32_t)fmin(need, 4294967040.0) : 1u;
            ties = at == cut ? min(ties, first) : first;
            cut = at;
          }
        }
      }
    }

    // The draw: [lo, hi) of the vocabulary, `before` the kept mass below it, `seen` the
    // tokens of value cut below it.
    const double least = rules.least, w_cut = cut > -INFINITY ? weight(cut) : 0.0;
    const bool ranked = ties != 0xffffffffu;
    const double w_tie = w_cut >= least || cut == best ? w_cut : 0.0;
    const auto kept_weight = [&](float x) __attribute__((always_inline)) {                // of what is above the cut
      if (!(ranked ? x > cut : x >= cut) || !(x >= least_x)) return 0.0;
      const double w = weight(x);
      return w >= least || x == best ? w : 0.0;
    };
    // of bf16 a table by bins
    if constexpr (!kMasses) {
      __syncthreads();
      for (int i = tid; i < Bins::kCount; i += NT) {
        uint32_t lo, hi;
        bins.keys(i, lo, hi);
        const float x = bf16_of_keys(lo, hi);
        s.mass[i] = x <= best && i != Bins::kSide ? kept_weight(x) : 0.0;
      }
      __syncthreads();
    }
    const auto kept = [&](float x) __attribute__((always_inline)) {
      if constexpr (!kMasses) {
        const int b = bins.of(x);
        if (b != Bins::kSide) return s.mass[b];
      }
      return kept_weight(x);
    };
    // of eight tokens; those next to zero are few, and asked for once
    const float from = fmaxf(cut, least_x);
    const auto kept_sum = [&](const float* x) __attribute__((always_inline)) {
      double m = 0;
      if constexpr (kMasses) {
#pragma unroll
        for (int e = 0; e < 8; ++e) m += kept_weight(x[e]);
      } else {
        bool some = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (!(x[e] >= from)) continue;                   // most: LDS has fewer lanes to serve
          const int b = bins.of(x[e]);
          some |= b == Bins::kSide;
          m += s.mass[b];                                  // of that bin 0
        }
        if (some)
          for (int e = 0; e < 8; ++e)
            if (bins.of(x[e]) == Bins::kSide) m += kept_weight(x[e]);
      }
      return m;
    };
    int32_t lo = 0, hi = a.V;
    double before = 0, goal = -1;
    uint32_t seen = 0;
    while (hi - lo > 512 || goal < 0) {
      double m = 0;
      uint32_t n = 0;
      sweep(lo, hi, [&](const float* x) __attribute__((always_inline)) {
        m += kept_sum(x);
        if (ranked)
#pragma unroll
          for (int e = 0; e < 8; ++e) n += x[e] == cut;
      });
      m = lanes_total(m), n = lanes_total(n);
      __syncthreads();
      if (lane == 0) s.sums[wave] = m, s.counts[wave] = n;
      __syncthreads();
      const auto of_wave = [&](int w, uint32_t below) {
        const uint32_t left = ties > below ? ties - below : 0;
        return s.sums[w] + (ranked ? min(left, s.counts[w]) * w_tie : 0.0);
      };
      if (goal < 0) {
        double all = 0;
        uint32_t below = 0;
        for (int w = 0; w < kWaves; ++w) all += of_wave(w, below), below += s.counts[w];
        goal = (double)u * all;
      }
      // the first piece that the running sum passes the goal in; the sums' rounding
      // aside there is one, and else it is the last with anything in it
      const int32_t size = piece(lo, hi);
      int pick = -1;
      double pick_before = 0, run = before;
      uint32_t pick_seen = 0, run_seen = seen;
      for (int w = 0; w < kWaves; ++w) {
        const double mine = of_wave(w, run_seen);
        if (mine > 0) {
          pick = w, pick_before = run, pick_seen = run_seen;
          if (run + mine > goal) break;
        }
        run += mine, run_seen += s.counts[w];
      }
      lo += pick * size;
      hi = min(hi, lo + size);
      before = pick_before, seen = pick_seen;
      __syncthreads();
    }
    if (wave > 0) return;
    float x[8];
    const int32_t v0 = lo + lane * 8;
    {
      const Raw raw = fetch(v0);
      logits(raw, x);
      filter(raw, x);
    }
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) n += ranked && x[e] == cut;
    uint32_t rank = seen + lanes_upto(n) - n;
    double w[8], sum = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      w[e] = v0 + e < hi ? kept(x[e]) : 0.0;
      if (ranked && x[e] == cut && v0 + e < hi) w[e] = rank++ < ties ? w_tie : 0.0;
      sum += w[e];
    }
    const double upto = lanes_upto(sum);
    const double below = __shfl_up(upto, 1);               // by every lane: an idle one has no value
    double run = before + (lane ? below : 0.0);
    int32_t first = 0x7fffffff, last = -1;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      run += w[e];
      if (w[e] > 0) {
        last = v0 + e;
        if (run > goal && first == 0x7fffffff) first = v0 + e;
      }
    }
    for (int d = 32; d > 0; d >>= 1) first = min(first, __shfl_xor(first, d)), last = max(last, __shfl_xor(last, d));
    if (lane == 0) {
      const int32_t token = first != 0x7fffffff ? first : last;
      const float prev = a.prev ? a.prev[r] : 0.f;
      a.tokens[r] = token;
      a.scores[r] = prev + (logit_at<T>(a, r, token) - top - log_sum);
    }
  }
  // whether a bin holds different values, whose mass its tokens add up
  static constexpr bool kMasses = T::kBytes == 4;
  // the one bf16 value among the keys [lo, hi) of a bin
  __device__ static float bf16_of_keys(uint32_t lo, uint32_t hi) {
    return lo >> 31 ? key_value(lo) : key_value(hi - 1);
  }
};

template <class T, int NT>
__global__ void __launch_bounds__(NT) sample_row_kernel(SampleArgs a) {
  __shared__ typename RowSampler<T, NT>::Shared shared;
  RowSampler<T, NT>(a, shared).run();
}

// ---------------------------------------------------------------------------
// One wave per row, the row in registers: rows of up to 512 * NCH tokens, lane l
// holding 8 consecutive tokens of every 512.
//
// The vector ALU bounds it (90 % busy), so the cuts are found by few instructions:
// the wave adds its candidates into a histogram of its own in LDS, 256 bins of an
// eighth of a power of two of the weight, a scan over the lanes gives the bin that a
// border falls into, and that bin's few members are taken off from the top.  (A
// search for the border by halving took 1400 instructions a row instead of 800.)
//
// Masses are fp32 as long as they lie further from every border than they can be
// off; a row for which that fails (one in a thousand) is decided by fp64 masses.
// ---------------------------------------------------------------------------
constexpr uint32_t kAll = 0xffffffffu;
constexpr int kWaveBins = 256;
struct WaveBins {
  uint32_t count[kWaveBins];
  uint32_t mass[kWaveBins];    // in units that keep the whole row's below 2^31
};

// What the rules keep: values from `cut` on (ties = kAll), or the values above it and
// its first `ties` tokens in vocabulary order.
struct Cut {
  float value;
  uint32_t ties;
};

template <int N>
__device__ __forceinline__ uint32_t count_from(const float (&x)[N], float t) {
  uint32_t n = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) n += (uint32_t)__builtin_popcountll(__ballot(x[i] >= t));
  return n;
}

// The cuts by fp64 masses and a search over the keys: what the definition gives.
template <int N>
__device__ __forceinline__ Cut exact_cut(const float (&x)[N], float best, const Rules& rules) {
  const double scale = 1.4426950408889634 / rules.T;
  const auto weight = [&](float z) { return z == best ? 1.0 : exp2_f64(((double)z - (double)best) * scale); };
  const uint32_t best_key = uniform(order_key(best));
  Cut c{-FLT_MAX, kAll};
  uint32_t lo = 0x00800000u;                               // key of the least finite fp32
  uint32_t kept = count_from(x, -FLT_MAX);
  if (rules.k < kept) {
    uint32_t hi = best_key + 1, above = 0;                 // from lo: more than k; from hi: `above` < k
    while (hi - lo > 1) {
      const uint32_t mid = lo + (hi - lo) / 2, n = count_from(x, key_value(mid));
      if (n > rules.k) lo = mid;
      else hi = mid, above = n;
      if (n == rules.k) break;
    }
    if (above == rules.k) c = {key_value(hi), kAll}, lo = hi;
    else c = {key_value(lo), rules.k - above};
    kept = rules.k;
  }
  if (!(rules.p < 1.0)) return c;
  const auto mass_from = [&](float t) {
    double m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) m += x[i] >= t ? weight(x[i]) : 0.0;
    return wave_total(m);
  };
  const bool partial = c.ties != kAll;
  double total = mass_from(key_value(lo + partial));
  if (partial) total += c.ties * weight(c.value);
  const double target = rules.p * total;
  uint32_t hi = best_key + 1;
  double mass_hi = 0;
  const uint32_t first = lo;
  uint32_t n_lo = kept, n_hi = 0;
  while (hi - lo > 1 && n_lo - n_hi > 1) {                 // from lo: at least the target; from hi: less
    const uint32_t mid = lo + (hi - lo) / 2;
    const double m = mass_from(key_value(mid));
    const uint32_t n = count_from(x, key_value(mid));
    if (m >= target) lo = mid, n_lo = n;
    else hi = mid, mass_hi = m, n_hi = n;
  }
  if (n_lo - n_hi == 1) return {key_value(lo), lo == first ? c.ties : kAll};
  const double need = ceil((target - mass_hi) / weight(key_value(lo)));
  const uint32_t n = need > 1 ? (uint32_t)need : 1u;
  return {key_value(lo), lo == first ? min(c.ties, n) : n};
}

// The kept weights' draw; w: the weights of x.  F = float gives certain = false where a
// mass lies within `off` of a border, or a weight next to the least.
template <class F, int N>
__device__ __forceinline__ int32_t draw(const float (&x)[N], F (&w)[N], float best, Cut cut, F least, float u,
                                        F off, bool& certain) {
  constexpr bool kExact = sizeof(F) == 8;
  const int lane = threadIdx.x & 63;
  certain = true;
  uint32_t seen = 0;                                       // tokens of the cut's value so far
  F sums[N / 8], all = 0;
  bool clear = true;
#pragma unroll
  for (int ch = 0; ch < N / 8; ++ch) {
    F sum = 0;
    uint32_t rank = 0;
    if (cut.ties != kAll) {
      uint32_t mine = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) mine += x[ch * 8 + e] == cut.value;
      const uint32_t upto = wave_scan(mine);
      rank = seen + upto - mine;
      seen += __builtin_amdgcn_readlane(upto, 63);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = ch * 8 + e;
      bool in = x[i] >= cut.value;
      if (cut.ties != kAll && x[i] == cut.value) in = rank++ < cut.ties;
      if (least > 0) {
        // (a weight above 2^-40 is within 61 * 2^-23 of itself)
        if (!kExact && in && fabsf((float)(w[i] - least)) <= (float)least * 0x1p-17f) clear = clear && x[i] == best;
        in = in && (w[i] >= least || x[i] == best);
      }
      w[i] = in ? w[i] : (F)0;
      sum += w[i];
    }
    sums[ch] = wave_upto(sum);
    all += lane_of(sums[ch], 63);
  }
  if (!kExact) certain = !__any(!clear);
  const F goal = (F)u * all;
  F before = 0;
  int32_t token = -1, start = -1;
#pragma unroll
  for (int ch = 0; ch < N / 8; ++ch) {
    const F end = before + lane_of(sums[ch], 63);
    const uint64_t past = __ballot(before + sums[ch] > goal);
    if (start < 0 && past) {
      const int l = __builtin_ctzll(past);
      start = (ch * 64 + l) * 8;
      // that lane's tokens, one after the other
      F run = before + (l ? lane_of(sums[ch], l ? l - 1 : 0) : (F)0), from = run, to = run;
      int32_t at = -1;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const F next = run + w[ch * 8 + e];
        if (at < 0 && w[ch * 8 + e] > 0 && next > goal) at = start + e, from = run, to = next;
        run = next;
      }
      token = __builtin_amdgcn_readlane(at, l);
      if (!kExact)
        certain = certain && __builtin_amdgcn_readlane((int)(goal - from > off && to - goal > off), l);
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

template <int N>
__device__ __forceinline__ int32_t exact_draw(const float (&x)[N], float best, Cut cut, const Rules& rules, float u) {
  const double scale = 1.4426950408889634 / rules.T;
  double w[N];
#pragma unroll
  for (int i = 0; i < N; ++i)
    w[i] = x[i] == best ? 1.0 : (x[i] > -INFINITY ? exp2_f64(((double)x[i] - (double)best) * scale) : 0.0);
  bool certain;
  return draw<double, N>(x, w, best, cut, rules.least, u, 0.0, certain);
}

// The token of a row x (what is no candidate -inf) whose best candidate is `best`.
template <int N>
__device__ __forceinline__ int32_t sample_wave(const float (&x)[N], float best, const Rules& rules, float u,
                                               WaveBins& bins) {
  const int lane = threadIdx.x & 63;
  const float temp = (float)rules.T, c = kLog2e / temp, p = (float)rules.p;
  Cut cut{-FLT_MAX, kAll};
  // outside the range of fp32 arithmetic
  bool certain = best < INFINITY && temp >= FLT_MIN && c >= FLT_MIN;
  float w[N];
  if (certain) {
    // The exponent a = (z_best - z) c of a weight 2^-a is off by three roundings, 3 * 2^-24 of
    // itself, and exp2 by one step: the weight by a * 1.5 * 2^-23 + 2^-23 of itself.  A sum
    // adds N + 8 roundings of half a step.  off: how far two masses can be off together, of
    // sums of w and w a over the whole row (a from 32 on is cut off: those weights are
    // below 2^-32).  Bins are eighths of a; the last takes what is no candidate, too.
    float eighths[N], sum_w = 0, sum_wa = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      w[i] = fast_exp2((x[i] - best) * c);
      eighths[i] = fminf((best - x[i]) * (8.f * c), kWaveBins - 1);
      sum_w += w[i];
      sum_wa = fmaf(w[i], eighths[i], sum_wa);
    }
    sum_w = wave_total(sum_w);
    const float off = 2 * (wave_total(sum_wa) * 0x1.8p-26f + sum_w * (0x1p-23f + (N + 8) * 0x1p-24f));
    const uint32_t candidates = count_from(x, -FLT_MAX);
    const bool by_count = rules.k < candidates, by_mass = p < 1.f;
    if (by_count || by_mass) {
      uint32_t bin[N];
#pragma unroll
      for (int i = 0; i < N; ++i) bin[i] = (uint32_t)eighths[i];
      u32x4* const count4 = (u32x4*)bins.count;
      u32x4* const mass4 = (u32x4*)bins.mass;
      if (by_count) count4[lane] = u32x4{0, 0, 0, 0};
      if (by_mass) mass4[lane] = u32x4{0, 0, 0, 0};
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (by_count) {
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (x[i] > -INFINITY) atomicAdd(&bins.count[bin[i]], 1u);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      // the members of one bin, the best first: value and number
      float v[N];
      const auto open = [&](uint32_t b) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = bin[i] == b ? x[i] : -INFINITY;
      };
      const auto take = [&](float& value, uint32_t& number) {
        float m = v[0];
#pragma unroll
        for (int i = 1; i < N; ++i) m = fmaxf(m, v[i]);
        value = uniform(wave_max(m));
        number = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const bool same = v[i] == value;
          number += (uint32_t)__builtin_popcountll(__ballot(same));
          v[i] = same ? -INFINITY : v[i];
        }
      };
      // the bin with which the counts (or masses) of a scan over the bins reach the goal;
      // above: what lies before it
      const auto locate = [&](const u32x4& n4, uint32_t goal, uint32_t& above) {
        const uint32_t mine = n4.x + n4.y + n4.z + n4.w, upto = wave_scan(mine);
        const uint64_t past = __ballot(upto >= goal);
        const int l = past ? __builtin_ctzll(past) : 63;
        above = __builtin_amdgcn_readlane(upto - mine, l);
        uint32_t b = l * 4;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
          const uint32_t n = __builtin_amdgcn_readlane(n4[j], l);
          if (b == (uint32_t)l * 4 + j && above + n < goal) above += n, ++b;
        }
        return b;
      };
      if (by_count) {
        uint32_t above;
        const uint32_t b = locate(count4[lane], rules.k, above);
        open(b);
        for (;;) {
          float value;
          uint32_t n;
          take(value, n);
          cut.value = value;
          if (above + n >= rules.k) {
            if (above + n > rules.k) cut.ties = rules.k - above;
            break;
          }
          above += n;
        }
      }
      if (by_mass) {
        const bool partial = cut.ties != kAll;
        float total = sum_w;
        if (by_count) {
          float m = 0;
#pragma unroll
          for (int i = 0; i < N; ++i) m += (partial ? x[i] > cut.value : x[i] >= cut.value) ? w[i] : 0.f;
          total = wave_total(m);
          if (partial) total += cut.ties * fast_exp2((cut.value - best) * c);
        }
        const float target = p * total;
        // Added up as whole numbers, which LDS does at more than twice the speed of fp32
        // (65536 rows of 512 with top-p: 84 us for 186), and in no order that shows.
        constexpr float kUnit = 0x1p25f / N;
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (x[i] >= cut.value) atomicAdd(&bins.mass[bin[i]], (uint32_t)(w[i] * kUnit));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        uint32_t units;
        const uint32_t b = locate(mass4[lane], (uint32_t)(target * kUnit), units);
        float m = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) m += bin[i] < b ? w[i] : 0.f;
        float above = wave_total(m);
        open(b);
        for (;;) {
          float value;
          uint32_t n;
          take(value, n);
          if (!(value >= cut.value)) {                     // the masses' rounding
            certain = false;
            break;
          }
          const float each = fast_exp2((value - best) * c);
          if (above + n * each >= target) {
            // ties of the value that reach the target: the side of either border is certain
            const float need = (target - above) / each, first = fmaxf(ceilf(need), 1.f);
            certain = (first - need) * each > off && ((need - first + 1) * each > off || (above == 0 && first == 1));
            const uint32_t ties = (uint32_t)first;
            if (value == cut.value && partial) cut.ties = min(cut.ties, ties);
            else cut = {value, ties < n ? ties : kAll};
            break;
          }
          above += n * each;
        }
      }
    }
    if (!certain) cut = exact_cut<N>(x, best, rules);
    certain = true;
    const int32_t token = draw<float, N>(x, w, best, cut, (float)rules.least, u, off, certain);
    if (certain) return token;
  } else {
    cut = exact_cut<N>(x, best, rules);
  }
  return exact_draw<N>(x, best, cut, rules, u);
}

template <class T, int NCH>
__global__ void __launch_bounds__(256, NCH == 8 ? 1 : 2) sample_wave_kernel(SampleArgs a) {
  constexpr int N = NCH * 8;
  __shared__ WaveBins bins[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = (int64_t)(a.first + blockIdx.x) * 4 + wave;
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
  uint32_t bits[NCH];
  const int64_t words = (a.V + 31) / 32;
#pragma unroll
  for (int ch = 0; ch < NCH; ++ch) {
    const int32_t v = (ch * 64 + lane) * 8;
    bits[ch] = 0xff;
    if (a.mask) bits[ch] = v < a.V ? ((const uint8_t*)(a.mask + r * words))[v / 8] : 0;
  }
  top = wave_max(top);
  float sum = 0;                                           // a NaN or +inf makes it NaN
#pragma unroll
  for (int i = 0; i < N; ++i) sum += fast_exp2((x[i] - top) * kLog2e);
  const float log_sum = logf(wave_sum(sum));
  float best = -INFINITY;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = fmaxf(keep_bit(x[i], bits[i / 8], i % 8), -INFINITY);       // a NaN is no candidate
    best = fmaxf(best, x[i]);
  }
  best = uniform(wave_max(best));
  int32_t token = -1;
  if (best > -INFINITY) {
    if (rules.T > 0) {
      const float u = fminf(fmaxf(a.uniform[r], 0.f), kMostUniform);   // a NaN is 0
      token = sample_wave<N>(x, best, rules, u, bins[wave]);
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
hipError_t run(SampleArgs a, hipStream_t stream) {
  const int64_t workgroups = a.V <= 4096 ? ((int64_t)a.R + 3) / 4 : a.R;
  return launch_in_parts(workgroups, [&](uint32_t first, uint32_t count) {
    a.first = first;
    if (a.V <= 512) sample_wave_kernel<T, 1><<<count, 256, 0, stream>>>(a);
    else if (a.V <= 1024) sample_wave_kernel<T, 2><<<count, 256, 0, stream>>>(a);
    else if (a.V <= 2048) sample_wave_kernel<T, 4><<<count, 256, 0, stream>>>(a);
    else if (a.V <= 4096) sample_wave_kernel<T, 8><<<count, 256, 0, stream>>>(a);
    else if (a.V <= 8192) sample_row_kernel<T, 256><<<count, 256, 0, stream>>>(a);
    else sample_row_kernel<T, 1024><<<count, 1024, 0, stream>>>(a);
  });
}

}  // namespace

hipError_t launch_sample(const void* logits, const float* uniform, const float* prev,
                         const uint32_t* mask, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, int32_t B, int32_t M, int32_t V,
                         bool bf16, int32_t* tokens, float* scores, hipStream_t stream) {
  const SampleArgs a{logits, uniform, prev, mask, temperature, top_k, top_p, min_p, tokens, scores,
                     B * M, M, V, 0};
  return bf16 ? run<BF16>(a, stream) : run<F32>(a, stream);
}

}  // namespace grace
