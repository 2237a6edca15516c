// A token of each row of logits (hl_sample): temperature, top-k, top-p and min-p,
// and the token at which the kept weights' running sum passes u of their total.
//
// Weights are 2^((l - max) log2(e) / T), computed in float64 and held as whole
// numbers of 2^-43 of the greatest: sums of them are exact, so they do not depend
// on the order of additions, and equal logits have equal weights. Tokens below 2^-40
// of the greatest weigh nothing. The tokens that top-k and top-p keep are the first
// ones by (logit, lowest index); where they end is found from histograms, first of
// 2048 steps of the distance to the greatest logit, then, within one step, of the
// digits of the logits as ordered integers.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "gpu_host.h"

namespace hl {

constexpr uint32_t kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64, kSteps = 2048;
constexpr double kSpan = 40.0;  // powers of two below the greatest weight that a token may have
constexpr double kOne = 0x1p43;

struct SampleArgs {
  const void* logits;
  uint64_t stride;
  uint32_t vocab;
  const float* uniforms;
  const float *temperatures, *top_ps, *min_ps;  // null: the numbers below, for all rows
  const int32_t* top_ks;
  float temperature, top_p, min_p;
  int32_t top_k;
  int32_t* tokens;
  float* logprobs;
};

// A logit as an integer, the greater the logit the smaller; -0 is 0.
__device__ inline uint32_t rank_of(float l) {
  const uint32_t b = __builtin_bit_cast(uint32_t, l + 0.0f);
  return b & 0x80000000u ? b : b ^ 0x7FFFFFFFu;
}

template <class X>
__device__ inline X scan_wave(X v) {
#pragma unroll
  for (uint32_t d = 1; d < 64; d <<= 1) {
    const X o = __shfl_up(v, d);
    if (threadIdx.x % 64 >= d) v += o;
  }
  return v;
}

// The row's block. Every wave has a stretch of neighbouring logits, VEC of a lane
// next to each other. NV: logits a thread keeps in registers; 0: they are read
// again each time.
template <class T, int NV>
struct RowOf {
  static constexpr uint32_t VEC = 16 / sizeof(T), KEPT = NV ? NV : VEC;
  const T* row;
  uint32_t vocab, begin, end;  // this wave's stretch
  float v[KEPT];

  // VEC logits from `at` on; past the vocabulary and for NaN, -infinity
  __device__ static void read(const T* row, uint32_t vocab, uint32_t at, float* to) {
    typedef T Vec __attribute__((ext_vector_type(VEC)));
    struct __attribute__((packed, aligned(sizeof(T)))) Loose { Vec x; };  // a row may begin anywhere
    Vec x;
    if (at + VEC <= vocab) {
      x = reinterpret_cast<const Loose*>(row + at)->x;
    } else {
#pragma unroll
      for (uint32_t j = 0; j < VEC; ++j) x[j] = at + j < vocab ? row[at + j] : (T)-INFINITY;
    }
#pragma unroll
    for (uint32_t j = 0; j < VEC; ++j) to[j] = x[j] == x[j] ? (float)x[j] : -INFINITY;
  }

  __device__ void open(const T* r, uint32_t n) {
    row = r, vocab = n;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const uint32_t each = NV ? NV * 64 : (n + kSampleWaves * 64 * VEC - 1) / (kSampleWaves * 64 * VEC) * (64 * VEC);
    begin = wave * each < n ? wave * each : n, end = begin + each < n ? begin + each : n;
    if constexpr (NV) {
#pragma unroll
      for (uint32_t i = 0; i < NV / VEC; ++i) read(row, vocab, begin + (i * 64 + lane) * VEC, v + i * VEC);
    }
  }

  // f(logit, index) for this lane's logits, in the order of their indexes
  template <class F>
  __device__ __attribute__((always_inline)) void each(F f) {
    const uint32_t lane = threadIdx.x % 64;
    if constexpr (NV) {
#pragma unroll
      for (uint32_t i = 0; i < NV / VEC; ++i)
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) f(v[i * VEC + j], begin + (i * 64 + lane) * VEC + j);
    } else {
      for (uint32_t at = begin; at < end; at += 64 * VEC) {
        read(row, vocab, at + lane * VEC, v);
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) f(v[j], at + lane * VEC + j);
      }
    }
  }

  // The first index at which the running sum of weigh(logit, index) over the
  // wave's stretch is above `target`. Whole wave.
  template <class F>
  __device__ __attribute__((always_inline)) uint32_t pick(uint64_t target, F weigh) {
    const uint32_t lane = threadIdx.x % 64;
    uint64_t before = 0;
    uint32_t found = ~0u;
    const auto look = [&](const float* l, uint32_t at) __attribute__((always_inline)) {
      uint64_t w[VEC], sum = 0;
#pragma unroll
      for (uint32_t j = 0; j < VEC; ++j) w[j] = weigh(l[j], at + lane * VEC + j), sum += w[j];
      const uint64_t upto = before + scan_wave(sum);
      const uint64_t past = __ballot(upto > target);
      if (past) {
        uint64_t run = upto - sum;
        uint32_t mine = 0;
        bool there = false;
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) {
          run += w[j];
          if (!there && run > target) mine = at + lane * VEC + j, there = true;
        }
        found = __builtin_amdgcn_readlane(mine, __builtin_ctzll(past));
      }
      before = __shfl(upto, 63);
      return past != 0;
    };
    if constexpr (NV) {
#pragma unroll
      for (uint32_t i = 0; i < NV / VEC; ++i)
        if (found == ~0u) look(v + i * VEC, begin + i * 64 * VEC);
    } else {
      for (uint32_t at = begin; at < end; at += 64 * VEC) {
        read(row, vocab, at + lane * VEC, v);
        if (look(v, at)) break;
      }
    }
    return found;
  }
};

struct SampleLds {
  uint64_t mass[kSteps];
  uint32_t count[kSteps];
  double powers[64];  // 2^(i / 64)
  uint64_t wave[kSampleWaves];
  uint64_t before, in;
  uint32_t step, pick;
  float most;
};

// Sum over the block; s.wave has the waves'.
__device__ inline uint64_t add_block(SampleLds& s, uint64_t v) {
#pragma unroll
  for (uint32_t d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if (threadIdx.x % 64 == 0) s.wave[threadIdx.x / 64] = v;
  __syncthreads();
  uint64_t sum = 0;
  for (uint32_t w = 0; w < kSampleWaves; ++w) sum += s.wave[w];
  return sum;
}

// The first index at which the running sum of weigh over the row is above
// `target`, which is below its sum; s.wave has the waves' sums.
template <class R, class F>
__device__ inline uint32_t pick_block(SampleLds& s, R& r, uint64_t target, F weigh) {
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  uint64_t before = 0;
  for (uint32_t w = 0; w < wave; ++w) before += s.wave[w];
  if (threadIdx.x == 0) s.pick = 0;
  __syncthreads();
  if (before <= target && target < before + s.wave[wave]) {
    const uint32_t i = r.pick(target - before, weigh);
    if (threadIdx.x % 64 == 0) s.pick = i;
  }
  __syncthreads();
  const uint32_t i = s.pick;
  __syncthreads();
  return i;
}

// The step of a histogram at which its running sum reaches a goal; s.before is the
// sum before it, s.in what it has.
template <class H, class Reached>
__device__ inline uint32_t find_step(SampleLds& s, const H* hist, Reached reached) {
  const uint32_t at = 2 * threadIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint64_t x = hist[at], y = hist[at + 1], upto = scan_wave(x + y);
  if (threadIdx.x % 64 == 63) s.wave[wave] = upto;
  __syncthreads();
  uint64_t before = upto - x - y;
  for (uint32_t w = 0; w < wave; ++w) before += s.wave[w];
  if (!reached(before) && reached(before + x)) s.step = at, s.before = before, s.in = x;
  if (!reached(before + x) && reached(before + x + y)) s.step = at + 1, s.before = before + x, s.in = y;
  __syncthreads();
  return s.step;
}

template <class T, int NV>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(SampleArgs a) {
  __shared__ SampleLds s;
  const uint32_t row = blockIdx.x, tid = threadIdx.x;
  RowOf<T, NV> r;
  r.open(static_cast<const T*>(a.logits) + row * a.stride, a.vocab);
  if (tid < 64) s.powers[tid] = exp2((double)tid / 64.0);
  float top = -INFINITY;
  r.each([&](float l, uint32_t) { top = fmaxf(top, l); });
#pragma unroll
  for (uint32_t d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  __shared__ float s_top[kSampleWaves];
  if (tid % 64 == 0) s_top[tid / 64] = top;
  __syncthreads();
  float most = s_top[0];
  for (uint32_t w = 1; w < kSampleWaves; ++w) most = fmaxf(most, s_top[w]);
  if (most == -INFINITY) {  // nothing to draw
    if (tid == 0) a.tokens[row] = -1, a.logprobs[row] = -INFINITY;
    return;
  }
  const float temperature = a.temperatures ? a.temperatures[row] : a.temperature;
  const int32_t asked = a.top_ks ? a.top_ks[row] : a.top_k;
  const bool greedy = !(temperature > 0.0f);
  const uint32_t k = greedy ? 1 : asked <= 0 || (uint32_t)asked >= a.vocab ? 0 : (uint32_t)asked;  // 0: all
  if (k == 1) {
    const auto is_top = [&](float l, uint32_t) __attribute__((always_inline)) { return (uint64_t)(l == most); };
    uint64_t n = 0;
    r.each([&](float l, uint32_t i) { n += is_top(l, i); });
    add_block(s, n);
    const uint32_t i = pick_block(s, r, 0, is_top);
    if (tid == 0) a.tokens[row] = (int32_t)i, a.logprobs[row] = 0.0f;
    return;
  }
  const float top_p = a.top_ps ? a.top_ps[row] : a.top_p;
  const float least = a.min_ps ? a.min_ps[row] : a.min_p;
  const double rate = 1.4426950408889634 / (double)temperature;
  const double floor_w = least > 0.0f ? (double)fminf(least, 1.0f) : 0.0;
  const auto power = [&](float l) __attribute__((always_inline)) { return l == most ? 0.0 : ((double)l - (double)most) * rate; };
  const auto exact = [&](double y) __attribute__((always_inline)) {  // 2^y in units of kOne, y from -kSpan to 0
    const double z = floor(y * 64.0), x = (y * 64.0 - z) * (0.6931471805599453 / 64.0);
    const int n = (int)z;
    const double e = fma(x, fma(x, fma(x, fma(x, 1.0 / 120, 1.0 / 24), 1.0 / 6), 0.5), 1.0) * x;
    const double p = s.powers[n & 63];
    return ldexp(fma(p, e, p), n >> 6) * kOne;
  };
  const auto whole = [](double w) __attribute__((always_inline)) {  // to the nearest whole number
    return __builtin_bit_cast(uint64_t, w + 0x1p52) - 0x4330000000000000ull;
  };
  const float per = (float)((double)kSteps / kSpan * rate);
  const auto step_of = [&](float l) __attribute__((always_inline)) {  // the farther from the greatest, the later
    const float x = (most - l) * per;
    return l == most ? 0u : x < (float)(kSteps - 1) ? (uint32_t)x : kSteps - 1;
  };
  // Kept so far: the logits of rank below `last`, and those of it up to index `cut`.
  uint32_t last = ~0u, cut = ~0u;
  const auto in = [&](float l, uint32_t i) __attribute__((always_inline)) {
    const uint32_t x = rank_of(l);
    return power(l) >= -kSpan && (x < last || (x == last && i <= cut));
  };
  const auto zero = [&] {
    __syncthreads();
    for (uint32_t i = tid; i < kSteps; i += kSampleThreads) s.mass[i] = 0;
    for (uint32_t i = tid; i < kSteps; i += kSampleThreads) s.count[i] = 0;
    __syncthreads();
  };
  // Ends the kept ones where the running sum of weigh, in the order of the logits,
  // reaches a goal. reached(sum); weigh is the same for equal logits.
  const auto shorten = [&](auto* hist, auto weigh, auto reached) __attribute__((always_inline)) {
    typedef typename std::remove_reference<decltype(*hist)>::type H;
    zero();
    r.each([&](float l, uint32_t i) {
      if (in(l, i)) atomicAdd(&hist[step_of(l)], (H)weigh(l));
    });
    __syncthreads();
    const uint32_t step = find_step(s, hist, reached);
    uint64_t before = s.before;
    uint32_t prefix = 0, shift = 32;
    for (int pass = 0; pass < 3; ++pass) {
      const uint32_t width = pass < 2 ? 11 : 10;
      zero();
      r.each([&](float l, uint32_t i) {
        const uint32_t x = rank_of(l);
        if (in(l, i) && step_of(l) == step && (pass == 0 || x >> shift == prefix))
          atomicAdd(&hist[x >> (shift - width) & ((1u << width) - 1)], (H)weigh(l));
      });
      __syncthreads();
      const uint32_t digit = find_step(s, hist, [&](uint64_t sum) { return reached(before + sum); });
      prefix = prefix << width | digit;
      shift -= width;
      before += s.before;
    }
    // of the equal logits, as few of the lowest indexes as reach it
    const auto same = [&](float l, uint32_t i) __attribute__((always_inline)) { return (uint64_t)(rank_of(l) == prefix && in(l, i)); };
    uint64_t n = 0;
    r.each([&](float l, uint32_t i) { n += same(l, i); });
    const uint64_t all = add_block(s, n), each = s.in / all;
    uint64_t low = 1, high = all;
    while (low < high) {
      const uint64_t mid = (low + high) / 2;
      if (reached(before + mid * each)) high = mid;
      else low = mid + 1;
    }
    cut = pick_block(s, r, low - 1, same);
    last = prefix;
  };
  if (k) {
    uint64_t n = 0;
    r.each([&](float l, uint32_t i) { n += in(l, i); });
    if (add_block(s, n) > k)
      shorten(s.count, [](float) { return 1u; }, [&](uint64_t sum) { return sum >= k; });
  }
  const auto mass = [&](float l) __attribute__((always_inline)) { return whole(exact(power(l))); };
  if (top_p < 1.0f) {
    uint64_t n = 0;
    r.each([&](float l, uint32_t i) { n += in(l, i) ? mass(l) : 0; });
    const double goal = fmax((double)top_p * (double)add_block(s, n), 1.0);
    shorten(reinterpret_cast<unsigned long long*>(s.mass), [&](float l) { return (unsigned long long)mass(l); },
            [&](uint64_t sum) { return (double)sum >= goal; });
  }
  const auto weigh = [&](float l, uint32_t i) __attribute__((always_inline)) -> uint64_t {
    if (!in(l, i)) return 0;
    const double w = exact(power(l));
    return w >= floor_w * kOne || l == most ? whole(w) : 0;
  };
  uint64_t n = 0;
  r.each([&](float l, uint32_t i) { n += weigh(l, i); });
  const uint64_t total = add_block(s, n);
  const float u = a.uniforms[row];
  const double at = u > 0.0f ? floor((double)fminf(u, 1.0f) * (double)total) : 0.0;
  const uint64_t target = at < (double)(total - 1) ? (uint64_t)at : total - 1;
  const uint32_t token = pick_block(s, r, target, weigh);
  if (tid == 0) {
    const float l = (float)r.row[token];
    a.tokens[row] = (int32_t)token;
    a.logprobs[row] = (float)(power(l) * 0.6931471805599453 - log((double)total / kOne));
  }
}

template <class T, int NV>
static hl_status run_sample(const SampleArgs& a, uint32_t rows, hipStream_t s) {
  return enqueue(sample_kernel<T, NV>, dim3(rows), dim3(kSampleThreads), s, a);
}

template <class T>
static hl_status run_logits(const SampleArgs& a, uint32_t rows, hipStream_t s) {
  if (a.vocab <= 8 * kSampleThreads) return run_sample<T, 8>(a, rows, s);
  return run_sample<T, 0>(a, rows, s);
}

}  // namespace hl

using namespace hl;

extern "C" hl_status hl_sample(const hl_sampling* sampling, const void* logits_dev, hl_dtype dtype, uint64_t row_stride,
                               uint32_t rows, uint64_t vocab, const float* uniforms_dev, int32_t* tokens_dev,
                               float* logprobs_dev, void* stream) {
  if (!sampling || !logits_dev || !uniforms_dev || !tokens_dev || !logprobs_dev || rows == 0 || vocab == 0 ||
      (rows > 1 && row_stride < vocab))
    return HL_EINVAL;
  const uintptr_t size = dtype == HL_F32 ? 4 : 2;
  if ((dtype != HL_F32 && dtype != HL_BF16 && dtype != HL_F16) || !aligned(logits_dev, size)) return HL_EINVAL;
  for (const void* p : {(const void*)uniforms_dev, (const void*)tokens_dev, (const void*)logprobs_dev,
                        (const void*)sampling->temperature_dev, (const void*)sampling->top_k_dev,
                        (const void*)sampling->top_p_dev, (const void*)sampling->min_p_dev})
    if (!aligned(p, 4)) return HL_EINVAL;
  if (vocab >= (1u << 20) || row_stride >= (1ull << 40) || !grid_fits(rows, kSampleThreads)) return HL_EUNSUPPORTED;
  SampleArgs a = {};
  a.logits = logits_dev, a.stride = row_stride, a.vocab = (uint32_t)vocab, a.uniforms = uniforms_dev;
  a.temperatures = sampling->temperature_dev, a.top_ks = sampling->top_k_dev;
  a.top_ps = sampling->top_p_dev, a.min_ps = sampling->min_p_dev;
  a.temperature = sampling->temperature, a.top_k = sampling->top_k, a.top_p = sampling->top_p, a.min_p = sampling->min_p;
  a.tokens = tokens_dev, a.logprobs = logprobs_dev;
  const hipStream_t s = (hipStream_t)stream;
  return dtype == HL_F32    ? run_logits<float>(a, rows, s)
         : dtype == HL_BF16 ? run_logits<__bf16>(a, rows, s)
                            : run_logits<_Float16>(a, rows, s);
}
