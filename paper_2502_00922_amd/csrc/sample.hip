// A token of each row of logits (hl_sample): temperature, top-k, top-p and min-p,
// and the token at which the kept weights' running sum passes u of their total.
//
// Weights are 2^((l - max) log2(e) / T), computed in float64 and held as whole
// numbers of 2^-43 of the greatest: sums of them are exact, so they do not depend
// on the order of additions, and equal logits have equal weights. (A light weight has few
// bits of its own, three at 2^-40: sums over n tokens are off by n * 2^-43 at most.) Tokens
// below 2^-40 of the greatest weigh nothing. The tokens that top-k and top-p keep are the first
// ones by (logit, lowest index); where they end is found in two steps: a histogram
// of the distances to the greatest logit says in which of kSteps steps, and the few
// logits of that step, put on a list in the order of their indexes, say where in it.
//
// Rows are cut into slices, so that few rows use the whole GPU too. top_kernel finds
// each slice's greatest logit; step_kernel counts (or weighs) the steps, for the row
// and for its slice, and its last block of a row finds the border's step;
// list_kernel lists that step's logits; end_kernel, one block a row, has every slice's
// weight below the step and the list, and looks again only at the slice that the
// token is in. With top_k of kFew or less all that is kept is on the list, and nothing
// else is weighed. Where a list would be too long (more than kList logits in a step),
// the block takes the whole row's logits again for each digit of the border (slow_row):
// where many logits are equal near the border, or a million stand in the 1024 steps. That
// is slow: 0.94 ms for one row of 131072 bf16 logits around 20 (0.125 apart; top_p 0.9), 1.03
// for 64 (around 0: 0.068), 4.5 for one of 1000000 float32.
//
// The four kernels take 31 + 44 + 27 + 33 us for 256 rows of 131072 (134 MB, 26 us at a
// copy's rate) and 3.5 + 6.9 + 3.8 + 9.2 for one of 32000; with one block a row they took
// 386 and 104 us in all.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "gpu_host.h"

namespace hl {

constexpr uint32_t kSteps = 1024, kSlices = 64, kList = 2048, kFew = 1024;
constexpr uint32_t kMostSlice = 16384;  // logits of a slice: 64 for each lane of its waves
// Places of the list that a wave has of its own. One that lists more takes so many of the
// row's common ones, when it knows how many, and reads these logits again (with common
// places alone 64 rows of 131072 take 47.6 us, with these 42.8).
constexpr uint32_t kOwn = 64;
// Slices that a call's workspace has room for, at most (or one row's): more rows go through
// the kernels after each other. A compute unit has 16 blocks then, and the workspace is 174
// MB or less. us for 4096 rows of 32000 bf16 and 1024 of 131072, and MB: without an end 640
// and 463, 664 and 619; with 2048 slices 719 and 546, 54 and 29; with 4096 674 and 440, 108
// and 58.
constexpr uint32_t kAtOnce = 4096;
constexpr uint32_t kThreads = 256, kWaves = kThreads / 64;  // of a slice's blocks
constexpr uint32_t kEnd = 512, kEndWaves = kEnd / 64;       // of a row's last block
constexpr uint32_t kAhead = 4;    // loads of a lane in flight
constexpr uint32_t kPairs = 256;  // logits on a list, at most, that are compared each with each
constexpr double kSpan = 40.0;  // powers of two below the greatest weight that a token may have
constexpr double kLn2 = 0.6931471805599453;
constexpr double kOne = 0x1p43;

typedef unsigned long long u64;

// A row's part of the workspace; then its list, of a level's bits and its index above
// them, and its slices' weights of each step, one after the other.
struct RowWork {
  u64 mass[kSteps];
  uint32_t count[kSteps];
  u64 sum[kSlices];  // of the slice's weights that are kept whatever the list says
  float most[kSlices], lowest[kSlices];
  uint32_t first[kSlices];  // index of most
  uint32_t listed[kSlices * kWaves], at[kSlices * kWaves];  // by each of a slice's waves: how many, and from where on
  // The border. Steps below lo are kept as far as top_k and top_p go, above hi not;
  // those between, and step `other`, go on the list. by_count, by_mass: whether
  // top_k and top_p end there. From step `from` on, top_k's border is on the list.
  uint32_t lo, hi, other, from, by_count, by_mass;
  uint32_t arrived, used;              // used: of the list's common places
  u64 count_from, mass_from, mass_lo;  // of the steps below `from` and lo
  u64 unused;
};
static_assert(sizeof(RowWork) % 16 == 0, "rows and lists begin at 16 bytes");

struct SampleArgs {
  const void* logits;
  uint64_t stride;
  uint32_t vocab, slice, slices;  // slice: logits of one
  uint32_t common;                // of a row's list: kList, or all its logits
  const float* uniforms;
  const float *temperatures, *top_ps, *min_ps;  // null: the numbers below, for all rows
  const int32_t* top_ks;
  float temperature, top_p, min_p;
  int32_t top_k;
  int32_t* tokens;
  float* logprobs;
  uint8_t* work;

  __host__ __device__ uint32_t own() const { return slices * kWaves * kOwn; }  // places before the common ones
  __host__ __device__ uint64_t row_bytes() const {
    return sizeof(RowWork) + (own() + common + (uint64_t)slices * kSteps) * sizeof(u64);
  }
  __device__ RowWork& of_row(uint32_t row) const { return *reinterpret_cast<RowWork*>(work + row * row_bytes()); }
  __device__ u64* list_of(RowWork& w) const { return reinterpret_cast<u64*>(&w + 1); }
  __device__ u64* mass_of(RowWork& w, uint32_t i) const { return list_of(w) + own() + common + i * kSteps; }
};

// A logit as an integer, the greater the logit the smaller; -0 is 0.
__device__ inline uint32_t rank_of(float l) {
  const uint32_t b = __builtin_bit_cast(uint32_t, l + 0.0f);
  return b & 0x80000000u ? b : b ^ 0x7FFFFFFFu;
}

// v of another lane, by the row shifts and row broadcasts of scan_wave; `none` where
// there is no such lane.
template <int CTRL, int ROWS, class X>
__device__ inline X moved(X v, X none) {
  if constexpr (sizeof(X) == 8) {
    const u64 x = __builtin_bit_cast(u64, v), o = __builtin_bit_cast(u64, none);
    const uint32_t low = __builtin_amdgcn_update_dpp((uint32_t)o, (uint32_t)x, CTRL, ROWS, 0xF, false);
    const uint32_t high = __builtin_amdgcn_update_dpp((uint32_t)(o >> 32), (uint32_t)(x >> 32), CTRL, ROWS, 0xF, false);
    return __builtin_bit_cast(X, (u64)high << 32 | low);
  } else {
    const uint32_t x = __builtin_bit_cast(uint32_t, v), o = __builtin_bit_cast(uint32_t, none);
    return __builtin_bit_cast(X, (uint32_t)__builtin_amdgcn_update_dpp(o, x, CTRL, ROWS, 0xF, false));
  }
}

// f over the lanes up to this one. Whole wave; a few cycles a step, where a shuffle
// through LDS takes a hundred.
template <class X, class F>
__device__ inline X over_lanes(X v, X none, F f) {
  v = f(v, moved<0x111, 0xF>(v, none));  // lane - 1 of a row of 16
  v = f(v, moved<0x112, 0xF>(v, none));  // lane - 2
  v = f(v, moved<0x114, 0xF>(v, none));  // lane - 4
  v = f(v, moved<0x118, 0xF>(v, none));  // lane - 8
  v = f(v, moved<0x142, 0xA>(v, none));  // row 0's last to row 1, row 2's to row 3
  return f(v, moved<0x143, 0xC>(v, none));  // lane 31 to rows 2 and 3
}

template <class X>
__device__ inline X scan_wave(X v) {
  return over_lanes(v, (X)0, [](X x, X y) { return x + y; });
}

// v of a lane that is the same in the whole wave.
template <class X>
__device__ inline X lane_of(X v, uint32_t lane) {
  if constexpr (sizeof(X) == 8) {
    const u64 x = __builtin_bit_cast(u64, v);
    const uint32_t low = __builtin_amdgcn_readlane((uint32_t)x, lane), high = __builtin_amdgcn_readlane((uint32_t)(x >> 32), lane);
    return __builtin_bit_cast(X, (u64)high << 32 | low);
  } else {
    return __builtin_bit_cast(X, (uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(uint32_t, v), lane));
  }
}

template <class X>
__device__ inline X add_wave(X v) { return lane_of(scan_wave(v), 63); }

__device__ inline float most_wave(float v) {
  return lane_of(over_lanes(v, -INFINITY, [](float x, float y) { return fmaxf(x, y); }), 63);
}

// A value that other blocks of the kernel have added to: from the memory that all
// XCDs share.
template <class X>
__device__ inline X take(const X* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Logits at .. at+VEC-1 of a row as float32; past `end`, -infinity.
template <class T>
struct Logits {
  static constexpr uint32_t VEC = 16 / sizeof(T);
  __device__ static void read(const T* row, uint32_t end, uint32_t at, float (&to)[VEC]) {
    typedef T Vec __attribute__((ext_vector_type(VEC)));
    struct __attribute__((packed, aligned(sizeof(T)))) Loose { Vec x; };  // a row may begin anywhere
    Vec x;
    if (at + VEC <= end) {
      x = reinterpret_cast<const Loose*>(row + at)->x;
    } else {
#pragma unroll
      for (uint32_t j = 0; j < VEC; ++j) x[j] = at + j < end ? row[at + j] : (T)-INFINITY;
    }
#pragma unroll
    for (uint32_t j = 0; j < VEC; ++j) to[j] = (float)x[j];
  }
};

// f(logits, index of the first) for the vectors at begin + first, and again every
// STRIDE, kAhead loads at a time; ends where f is true, and then is. Whole wave.
template <class T, uint32_t STRIDE, class F>
__device__ __attribute__((always_inline)) inline bool for_vectors(const T* row, uint32_t begin, uint32_t end,
                                                                  uint32_t first, F f) {
  constexpr uint32_t VEC = Logits<T>::VEC;
  uint32_t at = begin;
  for (; at + kAhead * STRIDE <= end; at += kAhead * STRIDE) {
    float v[kAhead][VEC];
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) Logits<T>::read(row, ~0u, at + i * STRIDE + first, v[i]);
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i)
      if (f(v[i], at + i * STRIDE + first)) return true;
  }
  for (; at < end; at += STRIDE) {
    float v[VEC];
    Logits<T>::read(row, end, at + first, v);
    if (f(v, at + first)) return true;
  }
  return false;
}

// What a row's draw asks, and how its logits are weighed. `most`: the greatest.
struct Draw {
  float temperature, top_p, most, per;
  uint32_t k;                // 0: all
  double rate, rate64, top, floor_w;  // of a logit's distance: powers of two; floor_w: least weight kept, of 1
  bool greedy, few, border;  // few: all that is kept goes on the list; border: a step has to be found
  bool endless;              // the greatest logit is infinite

  __device__ Draw(const SampleArgs& a, uint32_t row, float m, float lowest) {
    temperature = a.temperatures ? a.temperatures[row] : a.temperature;
    top_p = a.top_ps ? a.top_ps[row] : a.top_p;
    const float p = a.min_ps ? a.min_ps[row] : a.min_p;
    const int32_t asked = a.top_ks ? a.top_ks[row] : a.top_k;
    k = asked <= 0 || (uint32_t)asked >= a.vocab ? 0 : (uint32_t)asked;
    greedy = !(temperature > 0.0f) || k == 1;
    most = m;
    rate = 1.0 / kLn2 / (double)temperature;
    floor_w = p > 0.0f ? (double)fminf(p, 1.0f) : 0.0;
    few = k && k <= kFew;
    border = k || top_p < 1.0f;
    endless = most == INFINITY;
    if (endless) most = 0.0f, lowest = 0.0f;
    const double far = fmin((double)most - (double)lowest, kSpan / rate);
    per = far > 0.0 ? (float)fmin((double)kSteps / far, 0x1p120) : 0.0f;
    top = (double)most, rate64 = rate * 64.0;
  }
  // A logit; where the greatest is infinite, 0 for those that are, and -infinity.
  __device__ float level(float l) const { return __builtin_expect(endless, 0) ? l == INFINITY ? 0.0f : -INFINITY : l; }
  template <uint32_t VEC>
  __device__ void levels(float (&v)[VEC]) const {
    if (__builtin_amdgcn_readfirstlane(endless))
#pragma unroll
      for (uint32_t j = 0; j < VEC; ++j) v[j] = level(v[j]);
  }
  // 64 log2 of the weight of a level; below -64 kSpan (or NaN) it is out
  __device__ double power(float x) const { return ((double)x - top) * rate64; }
  __device__ static bool weighs(double z) { return z >= -64.0 * kSpan; }
  // the farther from the greatest, the later
  __device__ uint32_t step(float x) const { return (uint32_t)fminf((most - x) * per, (float)(kSteps - 1)); }
  // 2^(z / 64) in whole numbers of 1 / kOne, for z from -64 kSpan to 0; powers: kOne *
  // 2^(i / 64), i = 0 .. 63
  __device__ static u64 whole(double z, const double* powers) {
    constexpr double c = kLn2 / 64.0;
    const double t = z + 0x1.8p52;  // its last bits are z rounded to a whole number
    const uint32_t n = (uint32_t)__builtin_bit_cast(u64, t);
    const double x = z - (t - 0x1.8p52);
    const double e = fma(x, fma(x, fma(x, fma(x, c * c * c * c / 24, c * c * c / 6), c * c / 2), c), 1.0);
    const u64 power = __builtin_bit_cast(u64, powers[n & 63]) + ((u64)((n & ~63u) << 14) << 32);  // times 2^(n >> 6)
    const double w = fma(__builtin_bit_cast(double, power), e, 0x1p52);
    return __builtin_bit_cast(u64, w) - 0x4330000000000000ull;
  }
  // whether min_p keeps a weight
  __device__ bool heavy(double z) const { return floor_w == 0.0 || z == 0.0 || exp2(z / 64.0) >= floor_w; }
};

// The table of whole(), by a block of 64 threads or more.
__device__ inline void fill_powers(double* powers) {
  if (threadIdx.x < 64) powers[threadIdx.x] = kOne * exp2((double)threadIdx.x / 64.0);
}

// The slice's greatest and least logits. Bound by HBM: this is the pass that brings
// the logits into the caches.
template <class T>
__global__ void __launch_bounds__(kThreads) top_kernel(SampleArgs a) {
  constexpr uint32_t VEC = Logits<T>::VEC, WAVES = kThreads / 64;
  __shared__ float s_most[WAVES], s_lowest[WAVES];
  __shared__ uint32_t s_first[WAVES];
  const uint32_t slice = blockIdx.x, row = blockIdx.y, tid = threadIdx.x;
  RowWork& w = a.of_row(row);
  if (slice == 0) {
    for (uint32_t i = tid; i < kSteps; i += kThreads) w.mass[i] = 0, w.count[i] = 0;
    if (tid == 0) w.arrived = 0, w.used = 0;
  }
  const T* logits = static_cast<const T*>(a.logits) + row * a.stride;
  const uint32_t begin = slice * a.slice, end = min(begin + a.slice, a.vocab);
  float most = -INFINITY, lowest = INFINITY;
  uint32_t first = begin;
  for_vectors<T, kThreads * VEC>(logits, begin, end, tid * VEC, [&](const float (&v)[VEC], uint32_t at) {
#pragma unroll
    for (uint32_t j = 0; j < VEC; ++j) {
      if (v[j] > most) most = v[j], first = at + j;
      lowest = fminf(lowest, v[j] > -INFINITY ? v[j] : INFINITY);  // NaN is neither
    }
    return false;
  });
#pragma unroll
  for (uint32_t d = 32; d; d >>= 1) {
    const float m = __shfl_xor(most, d);
    const uint32_t f = __shfl_xor(first, d);
    if (m > most || (m == most && f < first)) most = m, first = f;
    lowest = fminf(lowest, __shfl_xor(lowest, d));
  }
  if (tid % 64 == 0) s_most[tid / 64] = most, s_lowest[tid / 64] = lowest, s_first[tid / 64] = first;
  __syncthreads();
  if (tid != 0) return;
  for (uint32_t i = 1; i < WAVES; ++i) {
    if (s_most[i] > most || (s_most[i] == most && s_first[i] < first)) most = s_most[i], first = s_first[i];
    lowest = fminf(lowest, s_lowest[i]);
  }
  w.most[slice] = most, w.lowest[slice] = lowest, w.first[slice] = first;
}

// The row's greatest and least logits. Whole wave.
__device__ inline void ends_of(const SampleArgs& a, const RowWork& w, float& most, float& lowest) {
  const uint32_t lane = threadIdx.x % 64;
  most = most_wave(lane < a.slices ? w.most[lane] : -INFINITY);
  lowest = -most_wave(lane < a.slices ? -w.lowest[lane] : -INFINITY);
}

// Whether this is the last of a row's blocks to come here. The others' atomics have
// been performed by then.
__device__ inline bool last_of_row(const SampleArgs& a, uint32_t& arrived) {
  __shared__ uint32_t s_arrived;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0) s_arrived = __hip_atomic_fetch_add(&arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  asm volatile("" ::: "memory");
  return s_arrived == a.slices - 1;
}

// The sum of v over the block's threads before this one; `all`: over all of them.
template <uint32_t WAVES>
__device__ inline u64 scan_block(u64 v, u64& all) {
  __shared__ u64 s_wave[WAVES];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const u64 upto = scan_wave(v);
  if (threadIdx.x % 64 == 63) s_wave[wave] = upto;
  __syncthreads();
  u64 before = upto - v;
  all = 0;
#pragma unroll
  for (uint32_t i = 0; i < WAVES; ++i) {
    if (i < wave) before += s_wave[i];
    all += s_wave[i];
  }
  __syncthreads();
  return before;
}

template <uint32_t WAVES>
__device__ inline u64 add_block(u64 v) {
  u64 all;
  scan_block<WAVES>(v, all);
  return all;
}

// The first of N numbers a thread, one thread's after the other's, at which the
// running sum reaches a goal that the sum of all reaches; `before`: the sum before it.
template <uint32_t WAVES, uint32_t N, class Reached>
__device__ inline uint32_t find_first(const u64 (&v)[N], Reached reached, u64& before) {
  __shared__ u64 s_before;
  __shared__ uint32_t s_at;
  u64 sum = 0, all;
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) sum += v[i];
  u64 run = scan_block<WAVES>(sum, all);
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) {
    if (!reached(run) && reached(run + v[i])) s_at = N * threadIdx.x + i, s_before = run;
    run += v[i];
  }
  __syncthreads();
  before = s_before;
  const uint32_t at = s_at;
  __syncthreads();
  return at;
}

// The steps between which a row's border is, from its histogram. below: LDS for the
// sums of the steps before each, of weights and of logits.
__device__ inline void place_border(const Draw& d, RowWork& w, u64 (&below)[2][kSteps + 1]) {
  constexpr uint32_t N = kSteps / kThreads;
  __shared__ u64 s_wave[2][kWaves];
  __shared__ uint32_t s_at[3];
  const uint32_t tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  u64 v[2][N], sum[2] = {0, 0};
#pragma unroll
  for (uint32_t i = 0; i < N; ++i) {
    v[0][i] = d.few ? 0 : take(&w.mass[N * tid + i]), v[1][i] = d.k ? take(&w.count[N * tid + i]) : 0;
    sum[0] += v[0][i], sum[1] += v[1][i];
  }
#pragma unroll
  for (uint32_t x = 0; x < 2; ++x) {
    const u64 upto = scan_wave(sum[x]);
    if (tid % 64 == 63) s_wave[x][wave] = upto;
    sum[x] = upto - sum[x];
  }
  __syncthreads();
#pragma unroll
  for (uint32_t x = 0; x < 2; ++x) {
    for (uint32_t i = 0; i < wave; ++i) sum[x] += s_wave[x][i];
#pragma unroll
    for (uint32_t i = 0; i < N; ++i) below[x][N * tid + i] = sum[x], sum[x] += v[x][i];
    if (tid == kThreads - 1) below[x][kSteps] = sum[x];
  }
  __syncthreads();
  // the first step at which the running sum reaches a goal that the whole sum reaches
  const auto find = [&](uint32_t x, uint32_t to, auto reached) {
#pragma unroll
    for (uint32_t i = 0; i < N; ++i)
      if (!reached(below[x][N * tid + i]) && reached(below[x][N * tid + i + 1])) s_at[to] = N * tid + i;
  };
  bool by_count = d.k && below[1][kSteps] > d.k, by_mass = d.top_p < 1.0f;
  uint32_t at_k = kSteps, lo = kSteps, hi = kSteps;
  if (by_count) {
    find(1, 0, [&](u64 n) { return n >= d.k; });
    __syncthreads();
    lo = hi = at_k = s_at[0];
  }
  if (d.few) {
    lo = 0;
    if (!by_count) hi = kSteps - 1;
  } else {
    if (by_mass) {
      // what top_k keeps weighs this at least, and at most
      const u64 least = below[0][at_k], most = below[0][min(at_k + 1, kSteps)];
      const double first = fmax((double)d.top_p * (double)least, 1.0), second = fmax((double)d.top_p * (double)most, 1.0);
      find(0, 1, [&](u64 m) { return (double)m >= first; });
      find(0, 2, [&](u64 m) { return (double)m >= second; });
      __syncthreads();
      lo = s_at[1], hi = s_at[2];
    }
    if (d.floor_w > 0.0) {
      // the step of the least weight that min_p keeps, or either of two
      const double x = -log2(d.floor_w) / d.rate * (double)d.per;
      const uint32_t near = (uint32_t)fmin(fmax(x - 0.01, 0.0), kSteps - 1.0);
      const uint32_t far = (uint32_t)fmin(x + 0.01, kSteps - 1.0);
      if (far < lo) lo = near, hi = far, by_count = by_mass = false;
      else lo = min(lo, near);
    }
  }
  if (tid != 0) return;
  const bool apart = by_count && at_k > hi;  // top_k's step is not between lo and hi
  // (without a border of top_k's, all steps weigh what top_p goes by)
  const uint32_t from = apart ? at_k : by_count || d.few ? lo : kSteps;
  w.lo = lo, w.hi = hi, w.other = apart ? at_k : lo, w.from = from, w.by_count = by_count, w.by_mass = by_mass;
  w.count_from = below[1][from], w.mass_from = below[0][from], w.mass_lo = below[0][lo];
}

// The slice's histogram, added to the row's. Bound by the weights' arithmetic, some
// twenty instructions in float64 each, and by LDS atomics (256 x 131072: vector units 61 %
// of the time, 44 % of the waves' at waits, 3.1 TB/s).
template <class T>
__global__ void __launch_bounds__(kThreads) step_kernel(SampleArgs a) {
  constexpr uint32_t VEC = Logits<T>::VEC;
  __shared__ u64 s_below[2][kSteps + 1];
  __shared__ uint32_t s_count[kSteps];
  __shared__ double s_powers[64];
  u64* s_mass = s_below[0];
  const uint32_t slice = blockIdx.x, row = blockIdx.y, tid = threadIdx.x;
  RowWork& w = a.of_row(row);
  float most, lowest;
  ends_of(a, w, most, lowest);
  if (most == -INFINITY) return;
  const Draw d(a, row, most, lowest);
  if (d.greedy) return;
  fill_powers(s_powers);
  for (uint32_t i = tid; i < kSteps; i += kThreads) s_mass[i] = 0, s_count[i] = 0;
  __syncthreads();
  const T* logits = static_cast<const T*>(a.logits) + row * a.stride;
  const uint32_t begin = slice * a.slice, end = min(begin + a.slice, a.vocab);
  const auto each = [&](auto f) __attribute__((always_inline)) {
    for_vectors<T, kThreads * VEC>(logits, begin, end, tid * VEC,
                                   [&](float (&v)[VEC], uint32_t) __attribute__((always_inline)) {
      d.levels(v);
#pragma unroll
      for (uint32_t j = 0; j < VEC; ++j) {
        const double z = d.power(v[j]);
        if (Draw::weighs(z)) f(v[j], z);
      }
      return false;
    });
  };
  if (d.few) {
    each([&](float x, double) { atomicAdd(&s_count[d.step(x)], 1u); });
  } else if (d.border) {
    each([&](float x, double z) {
      const uint32_t i = d.step(x);
      atomicAdd(&s_mass[i], Draw::whole(z, s_powers));
      if (d.k) atomicAdd(&s_count[i], 1u);
    });
  } else {
    u64 sum = 0;
    each([&](float, double z) { sum += d.heavy(z) ? Draw::whole(z, s_powers) : 0; });
    sum = add_wave(sum);
    if (tid % 64 == 0) atomicAdd(&s_mass[0], sum);
    __syncthreads();
    if (tid == 0) w.sum[slice] = s_mass[0];
    return;
  }
  __syncthreads();
  for (uint32_t i = tid; i < kSteps; i += kThreads) {
    if (!d.few) {
      a.mass_of(w, slice)[i] = s_mass[i];
      if (s_mass[i]) atomicAdd(&w.mass[i], s_mass[i]);
    }
    if (s_count[i]) atomicAdd(&w.count[i], s_count[i]);
  }
  if (last_of_row(a, w.arrived)) place_border(d, w, s_below);
}

struct EndLds {
  u64 bin[kEnd], weight[kList];
  float logit[kList];
  uint32_t index[kList];
  double powers[64];
  u64 wave[kEndWaves], total[kSlices], limit;
  ulonglong2 pair[kPairs];  // a logit's place, and its weight if its step is not past hi
  uint32_t start[kSlices * kWaves], at[kSlices * kWaves], pick, members;
};

// A logit's place in the order: falling logits, of equal ones the lowest index first.
__device__ inline u64 place_of(float x, uint32_t i) { return (u64)rank_of(x) << 32 | i; }

// The place of the last logit at which the running sum of weights, in the order of the
// logits, does not reach a goal yet without it. `each` goes through logits whose ranks
// have all bits from `top` on equal, f(level, index, weight); `before` is the sum of
// those ahead of them. nth(rank, n): the index of the n-th logit of a rank.
template <class Each, class Reached, class Nth>
__device__ inline u64 find_border(EndLds& s, Each each, uint32_t top, uint32_t prefix, u64 before, Reached reached,
                                  Nth nth) {
  uint32_t shift = top;
  while (true) {
    // few enough of the prefix's logits are compared each with each
    if (threadIdx.x == 0) s.members = 0;
    __syncthreads();
    each([&](float x, uint32_t i, u64 weight) __attribute__((always_inline)) {
      if (shift < 32 && rank_of(x) >> shift != prefix) return;
      const uint32_t at = atomicAdd(&s.members, 1u);
      if (at < kPairs) s.pair[at] = {place_of(x, i), weight};
    });
    __syncthreads();
    const uint32_t members = s.members;
    if (members <= kPairs) {
      if (threadIdx.x < members) {
        const ulonglong2 mine = s.pair[threadIdx.x];
        u64 ahead = before;
        for (uint32_t i = 0; i < members; ++i) ahead += s.pair[i].x < mine.x ? s.pair[i].y : 0;
        if (!reached(ahead) && reached(ahead + mine.y)) s.limit = mine.x;
      }
      __syncthreads();
      return s.limit;
    }
    if (shift == 0) break;
    const uint32_t width = min(shift, 9u);
    static_assert(kEnd == 512, "a thread has a digit of 9 bits");
    s.bin[threadIdx.x] = 0;
    __syncthreads();
    each([&](float x, uint32_t, u64 weight) __attribute__((always_inline)) {
      const uint32_t r = rank_of(x);
      if (shift == 32 || r >> shift == prefix) atomicAdd(&s.bin[r >> (shift - width) & ((1u << width) - 1)], weight);
    });
    __syncthreads();
    const u64 bin[1] = {s.bin[threadIdx.x]};
    u64 ahead;
    const uint32_t digit = find_first<kEndWaves>(bin, [&](u64 sum) { return reached(before + sum); }, ahead);
    before += ahead, shift -= width;
    prefix = prefix << width | digit;
  }
  // of equal ones, which weigh the same, as few as reach it
  u64 sum = 0;
  each([&](float x, uint32_t, u64 weight) __attribute__((always_inline)) {
    if (rank_of(x) == prefix) sum += weight;
  });
  const u64 same = s.members, one = add_block<kEndWaves>(sum) / same;
  u64 low = 1, high = same;
  while (low < high) {
    const u64 mid = (low + high) / 2;
    if (reached(before + mid * one)) high = mid;
    else low = mid + 1;
  }
  return (u64)prefix << 32 | nth(prefix, low);
}

// A stretch of a row by the whole block; each wave has a part of neighbours.
template <class T>
struct Stretch {
  static constexpr uint32_t VEC = Logits<T>::VEC;
  const T* row;
  uint32_t begin, end;  // this wave's

  __device__ Stretch(const T* r, uint32_t from, uint32_t to) : row(r) {
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const uint32_t part = (to - from + kEnd * VEC - 1) / (kEnd * VEC) * (64 * VEC);
    begin = min(from + wave * part, to), end = min(begin + part, to);
  }
  // f(logit, index) for this lane's logits
  template <class F>
  __device__ __attribute__((always_inline)) void each(F f) const {
    for_vectors<T, 64 * VEC>(row, begin, end, threadIdx.x % 64 * VEC,
                             [&](const float (&v)[VEC], uint32_t at) __attribute__((always_inline)) {
#pragma unroll
      for (uint32_t j = 0; j < VEC; ++j) f(v[j], at + j);
      return false;
    });
  }
  // The first index at which the running sum of weigh(logit, index) over the stretch
  // is above `target`, which is below its sum.
  template <class F>
  __device__ __attribute__((always_inline)) uint32_t pick(EndLds& s, u64 target, F weigh) const {
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    u64 sum = 0;
    each([&](float l, uint32_t i) __attribute__((always_inline)) { sum += weigh(l, i); });
    sum = add_wave(sum);
    if (lane == 0) s.wave[wave] = sum;
    if (threadIdx.x == 0) s.pick = 0;
    __syncthreads();
    u64 before = 0;
    for (uint32_t i = 0; i < wave; ++i) before += s.wave[i];
    if (before <= target && target < before + sum) {
      for_vectors<T, 64 * VEC>(row, begin, end, lane * VEC,
                               [&](const float (&v)[VEC], uint32_t at) __attribute__((always_inline)) {
        u64 w[VEC], mine = 0;
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j) w[j] = weigh(v[j], at + j), mine += w[j];
        const u64 upto = before + scan_wave(mine), past = __ballot(upto > target);
        if (past) {
          u64 run = upto - mine;
          uint32_t found = 0;
          bool there = false;
#pragma unroll
          for (uint32_t j = 0; j < VEC; ++j) {
            run += w[j];
            if (!there && run > target) found = at + j, there = true;
          }
          if (lane == (uint32_t)__builtin_ctzll(past)) s.pick = found;
        }
        before = lane_of(upto, 63);
        return past != 0;
      });
    }
    __syncthreads();
    const uint32_t i = s.pick;
    __syncthreads();
    return i;
  }
};

// The whole number that a running sum must pass for the token of u.
__device__ inline u64 target_of(float u, u64 total) {
  const double at = u > 0.0f ? floor((double)fminf(u, 1.0f) * (double)total) : 0.0;
  return at < (double)(total - 1) ? (u64)at : total - 1;
}

template <class T>
__device__ inline void end_row(const SampleArgs& a, const Draw& d, uint32_t row, const T* logits, uint32_t token,
                               u64 total) {
  if (threadIdx.x != 0) return;
  const float l = (float)logits[token];
  a.tokens[row] = (int32_t)token;
  a.logprobs[row] = (float)(d.power(d.level(l)) * (kLn2 / 64.0) - log((double)total / kOne));
}

// A row by one block, from its logits alone.
template <class T>
__device__ inline void slow_row(const SampleArgs& a, const Draw& d, uint32_t row, const T* logits, EndLds& s) {
  const Stretch<T> all(logits, 0, a.vocab);
  u64 limit = ~0ull;  // the last place kept
  const auto mass = [&](float l, uint32_t i) __attribute__((always_inline)) -> u64 {
    const float x = d.level(l);
    const double z = d.power(x);
    return Draw::weighs(z) && place_of(x, i) <= limit ? Draw::whole(z, s.powers) : 0;
  };
  for (int stage = 0; stage < 2; ++stage) {  // top_k, top_p
    if (stage == 0 ? d.k == 0 : !(d.top_p < 1.0f)) continue;
    const auto each = [&](auto f) __attribute__((always_inline)) {
      all.each([&](float l, uint32_t i) __attribute__((always_inline)) {
        const u64 w = mass(l, i);
        if (w) f(d.level(l), i, stage == 0 ? 1 : w);
      });
    };
    u64 n = 0;
    each([&](float, uint32_t, u64 w) __attribute__((always_inline)) { n += w; });
    n = add_block<kEndWaves>(n);
    if (stage == 0 && n <= d.k) continue;
    const double goal = stage == 0 ? (double)d.k : fmax((double)d.top_p * (double)n, 1.0);
    limit = find_border(s, each, 32, 0, 0, [&](u64 sum) { return (double)sum >= goal; }, [&](uint32_t rank, u64 nth) {
      return all.pick(s, nth - 1, [&](float l, uint32_t i) __attribute__((always_inline)) {
        return (u64)(mass(l, i) && rank_of(d.level(l)) == rank);
      });
    });
  }
  const auto weigh = [&](float l, uint32_t i) __attribute__((always_inline)) -> u64 {
    const u64 w = mass(l, i);
    return w && d.heavy(d.power(d.level(l))) ? w : 0;
  };
  u64 n = 0;
  all.each([&](float l, uint32_t i) __attribute__((always_inline)) { n += weigh(l, i); });
  const u64 total = add_block<kEndWaves>(n);
  end_row(a, d, row, logits, all.pick(s, target_of(a.uniforms[row], total), weigh), total);
}

// Lists the logits of the border's steps, and adds up what the slice has below them. A
// lane keeps a bit for each of its logits, for a wave that lists more than it has places.
// Bound by reading the logits again (256 x 131072: 5.3 TB/s, a copy's rate).
template <class T>
__global__ void __launch_bounds__(kThreads) list_kernel(SampleArgs a) {
  constexpr uint32_t VEC = Logits<T>::VEC;
  const uint32_t slice = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid % 64;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid / 64);
  RowWork& w = a.of_row(row);
  float most, lowest;
  ends_of(a, w, most, lowest);
  if (most == -INFINITY) return;
  const Draw d(a, row, most, lowest);
  if (d.greedy || !d.border) return;
  const uint32_t lo = w.lo, hi = w.hi, other = w.other;
  if (!d.few) {
    const u64* mass = a.mass_of(w, slice);
    u64 base = 0;
    for (uint32_t i = tid; i < lo; i += kThreads) base += mass[i];
    base = add_block<kWaves>(base);
    if (tid == 0) w.sum[slice] = base;
  }
  // every wave has its part of the slice
  const T* logits = static_cast<const T*>(a.logits) + row * a.stride;
  const uint32_t part = a.slice / kWaves, begin = min(slice * a.slice + wave * part, a.vocab);
  static_assert(kMostSlice / kWaves == 64 * 64, "a lane has a bit for each of its logits");
  u64* list = a.list_of(w);
  const uint32_t own = (slice * kWaves + wave) * kOwn;
  u64 bits = 0;
  uint32_t shift = 0, listed = 0;
  // the next places of the lanes whose bits of a vector are `mine`
  const auto places = [&](uint32_t mine) {
    const uint32_t upto = scan_wave((uint32_t)__popc(mine)), place = listed + upto - __popc(mine);
    listed += lane_of(upto, 63);
    return place;
  };
  const auto entry = [](uint32_t at, float level) { return (u64)at << 32 | __builtin_bit_cast(uint32_t, level); };
  for_vectors<T, 64 * VEC>(logits, begin, min(begin + part, a.vocab), lane * VEC,
                           [&](float (&v)[VEC], uint32_t at) __attribute__((always_inline)) {
    uint32_t mine = 0;
    d.levels(v);
#pragma unroll
    for (uint32_t j = 0; j < VEC; ++j) {
      const uint32_t step = d.step(v[j]);
      mine |= (uint32_t)((step >= lo && step <= hi) || step == other) << j;
    }
    if (__any(mine != 0)) {
#pragma unroll
      for (uint32_t j = 0; j < VEC; ++j) mine &= ~((uint32_t)!Draw::weighs(d.power(v[j])) << j);
      bits |= (u64)mine << shift;
      uint32_t place = places(mine);
#pragma unroll
      for (uint32_t j = 0; j < VEC; ++j)
        if (mine >> j & 1) {
          if (place < kOwn) list[own + place] = entry(at + j, v[j]);
          ++place;
        }
    }
    shift += VEC;
    return false;
  });
  uint32_t to = own;
  if (listed > kOwn) {
    uint32_t used = 0;
    if (lane == 0) used = atomicAdd(&w.used, listed);
    used = __builtin_amdgcn_readfirstlane(used);
    to = a.own() + used;
    if (used + listed <= a.common) {  // else the row has more than kList, and no use for its list
      u64* common = list + to;
      listed = 0;
      for (uint32_t at = begin + lane * VEC; __any(bits != 0); at += 64 * VEC, bits >>= VEC) {
        const uint32_t mine = (uint32_t)bits & ((1u << VEC) - 1);
        if (!__any(mine != 0)) continue;
        uint32_t place = places(mine);
#pragma unroll
        for (uint32_t j = 0; j < VEC; ++j)
          if (mine >> j & 1) common[place++] = entry(at + j, d.level((float)logits[at + j]));
      }
    }
  }
  if (lane == 0) w.listed[slice * kWaves + wave] = listed, w.at[slice * kWaves + wave] = to;
}

// Ends a row from its list and the slices' sums. Bound by its barriers and waits, one
// after the other (62 to 67 % of the waves' time).
template <class T>
__global__ void __launch_bounds__(kEnd) end_kernel(SampleArgs a) {
  constexpr uint32_t EACH = kList / kEnd;
  __shared__ EndLds s;
  const uint32_t row = blockIdx.x, tid = threadIdx.x, lane = tid % 64;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid / 64);
  RowWork& w = a.of_row(row);
  const T* logits = static_cast<const T*>(a.logits) + row * a.stride;
  float most, lowest;
  ends_of(a, w, most, lowest);
  if (most == -INFINITY) {  // nothing to draw
    if (tid == 0) a.tokens[row] = -1, a.logprobs[row] = -INFINITY;
    return;
  }
  const Draw d(a, row, most, lowest);
  if (d.greedy) {
    const uint64_t at = __ballot(lane < a.slices && w.most[lane < a.slices ? lane : 0] == most);
    if (tid == 0) a.tokens[row] = (int32_t)w.first[__builtin_ctzll(at)], a.logprobs[row] = 0.0f;
    return;
  }
  const uint32_t lo = d.border ? w.lo : kSteps, hi = d.border ? w.hi : kSteps;
  fill_powers(s.powers);
  uint32_t n = 0;
  if (lo < kSteps) {
    static_assert(kSlices * kWaves <= kEnd, "a thread has a wave's list");
    const uint32_t mine = tid < a.slices * kWaves ? w.listed[tid] : 0;
    u64 all;
    const uint32_t start = (uint32_t)scan_block<kEndWaves>(mine, all);
    if (tid < kSlices * kWaves) s.start[tid] = start, s.at[tid] = tid < a.slices * kWaves ? w.at[tid] : 0;
    n = (uint32_t)all;
  }
  __syncthreads();
  if (n > kList) {
    slow_row<T>(a, d, row, logits, s);
    return;
  }
  // Logits each*tid .. of the list are this thread's: as few as take the whole list,
  // so that a short one is one logit a thread. `kept` has a bit for each.
  const uint32_t most_each = n <= kEnd ? 1 : EACH, first = most_each * tid;
  uint32_t kept = 0;
  for (uint32_t j = 0; j < most_each; ++j) {
    const uint32_t i = first + j;
    if (i >= n) break;
    uint32_t from = 0;  // the list that it is on
#pragma unroll
    for (uint32_t h = kSlices * kWaves / 2; h; h >>= 1)
      if (s.start[from + h] <= i) from += h;
    const u64 x = a.list_of(w)[s.at[from] + i - s.start[from]];
    const float l = __builtin_bit_cast(float, (uint32_t)x);
    s.logit[i] = l, s.index[i] = (uint32_t)(x >> 32);
    s.weight[i] = Draw::whole(d.power(l), s.powers);
    kept |= 1u << j;
  }
  if (tid == 0) s.limit = 0;
  __syncthreads();
  // f(place on the list) for this thread's that are kept still; those of which f is
  // false no longer are
  const auto each = [&](auto f) __attribute__((always_inline)) {
    for (uint32_t j = 0; j < most_each; ++j)
      if (kept >> j & 1) f(first + j);
  };
  const auto narrow = [&](auto f) __attribute__((always_inline)) {
    uint32_t still = 0;
    each([&](uint32_t i) {
      if (f(i)) still |= 1u << (i - first);
    });
    kept = still;
  };
  const auto weight_kept = [&] {
    u64 sum = 0;
    each([&](uint32_t i) { sum += s.weight[i]; });
    return sum;
  };
  const bool by_count = d.border && w.by_count, by_mass = d.border && w.by_mass;
  const uint32_t from = d.border ? w.from : kSteps;
  u64 limit = ~0ull;  // the last place kept, for the logits of listed steps
  if (n && n <= kPairs) {
    // each logit's predecessors
    const float l = tid < n ? s.logit[tid] : 0.0f;
    const u64 mine = tid < n ? place_of(l, s.index[tid]) : 0;
    const uint32_t step = tid < n ? d.step(l) : 0;
    if (tid < kPairs) s.pair[tid] = {tid < n ? mine : ~0ull, tid < n && step <= hi ? s.weight[tid] : 0};
    u64 count = by_count ? w.count_from - add_block<kEndWaves>(tid < n && step < from) : 0, mass = d.border ? w.mass_lo : 0;
    __syncthreads();
    if (by_count || by_mass) {
#pragma unroll 8
      for (uint32_t i = 0; i < (n + 7) / 8 * 8; ++i) {
        const ulonglong2 x = s.pair[i];
        const bool ahead = x.x < mine;
        count += ahead, mass += ahead ? x.y : 0;
      }
    }
    if (by_count) narrow([&](uint32_t) { return step < from || count < d.k; });
    if (by_mass) {
      u64 sum = 0;
      each([&](uint32_t i) { sum += step >= from ? s.weight[i] : 0; });
      const double goal = fmax((double)d.top_p * (double)(w.mass_from + add_block<kEndWaves>(sum)), 1.0);
      narrow([&](uint32_t) { return step <= hi && (double)mass < goal; });
    }
    each([&](uint32_t) { atomicMax(&s.limit, mine); });
    __syncthreads();
    limit = s.limit;
  } else if (n) {
    // bits in which the list's ranks differ
    uint32_t low = ~0u, high = 0;
    each([&](uint32_t i) { low = min(low, rank_of(s.logit[i])), high = max(high, rank_of(s.logit[i])); });
#pragma unroll
    for (uint32_t x = 32; x; x >>= 1) low = min(low, __shfl_xor(low, x)), high = max(high, __shfl_xor(high, x));
    if (lane == 0) s.wave[wave] = (u64)high << 32 | low;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kEndWaves; ++i)
      low = min(low, (uint32_t)s.wave[i]), high = max(high, (uint32_t)(s.wave[i] >> 32));
    const uint32_t top = low == high ? 0 : 32 - __builtin_clz(low ^ high);
    // Ends the listed logits of which `of` is true where the sum of `weigh` reaches `to`.
    const auto shorten = [&](auto of, auto weigh, u64 before, double to) __attribute__((always_inline)) {
      const auto some = [&](auto f) __attribute__((always_inline)) {
        each([&](uint32_t i) {
          if (of(i)) f(s.logit[i], s.index[i], weigh(i));
        });
      };
      const auto nth = [&](uint32_t rank, u64 which) {
        u64 same = 0, all;
        some([&](float x, uint32_t, u64) { same += rank_of(x) == rank; });
        u64 at = scan_block<kEndWaves>(same, all);
        some([&](float x, uint32_t i, u64) {
          if (rank_of(x) == rank && ++at == which) s.pick = i;
        });
        __syncthreads();
        return s.pick;
      };
      limit = find_border(s, some, top, top == 32 ? 0 : low >> top, before, [&](u64 sum) { return (double)sum >= to; }, nth);
      narrow([&](uint32_t i) { return place_of(s.logit[i], s.index[i]) <= limit; });
      __syncthreads();
    };
    if (by_count)
      shorten([&](uint32_t i) { return d.step(s.logit[i]) >= from; }, [](uint32_t) { return 1ull; }, w.count_from, (double)d.k);
    if (by_mass) {
      u64 sum = 0;
      each([&](uint32_t i) { sum += d.step(s.logit[i]) >= from ? s.weight[i] : 0; });
      const double goal = fmax((double)d.top_p * (double)(w.mass_from + add_block<kEndWaves>(sum)), 1.0);
      shorten([&](uint32_t i) { return d.step(s.logit[i]) <= hi; }, [&](uint32_t i) { return s.weight[i]; }, w.mass_lo, goal);
    }
  }
  if (d.floor_w > 0.0) narrow([&](uint32_t i) { return d.heavy(d.power(s.logit[i])); });
  const float u = a.uniforms[row];
  if (d.few) {  // the list is in the order of the indexes, and has all
    u64 total;
    u64 run = scan_block<kEndWaves>(weight_kept(), total);
    const u64 target = target_of(u, total);
    each([&](uint32_t i) {
      if (run <= target && run + s.weight[i] > target) s.pick = s.index[i];
      run += s.weight[i];
    });
    __syncthreads();
    end_row(a, d, row, logits, s.pick, total);
    return;
  }
  if (tid < kSlices) s.total[tid] = tid < a.slices ? w.sum[tid] : 0;
  __syncthreads();
  each([&](uint32_t i) { atomicAdd(&s.total[s.index[i] / a.slice], s.weight[i]); });
  __syncthreads();
  const u64 mine = s.total[lane], upto = scan_wave(mine), total = lane_of(upto, 63), target = target_of(u, total);
  const uint32_t in = (uint32_t)__builtin_ctzll(__ballot(upto > target));
  const u64 before = lane_of(upto - mine, in);
  const Stretch<T> there(logits, in * a.slice, min((in + 1) * a.slice, a.vocab));
  const uint32_t token = there.pick(s, target - before, [&](float l, uint32_t i) __attribute__((always_inline)) -> u64 {
    const float x = d.level(l);
    const double z = d.power(x);
    if (!Draw::weighs(z)) return 0;
    const uint32_t step = d.step(x);
    const bool is = step < lo || (step <= hi && place_of(x, i) <= limit);
    return is && d.heavy(z) ? Draw::whole(z, s.powers) : 0;
  });
  end_row(a, d, row, logits, token, total);
}

// Logits of a slice: as few as give every compute unit blocks, at least 2048, and
// no more slices than kSlices.
static uint32_t slice_of(uint64_t rows, uint64_t vocab) {
  const uint64_t blocks = 4 * (uint64_t)device_cus(), most = std::max<uint64_t>(1, blocks / rows);
  const uint64_t each = (vocab + most - 1) / most, least = std::max<uint64_t>(2048, (vocab + kSlices - 1) / kSlices);
  return (uint32_t)((std::min<uint64_t>(std::max(each, least), kMostSlice) + 2047) / 2048 * 2048);
}

// Fills in how rows are cut, and gives how many go through the kernels at once.
static uint32_t cut_rows(SampleArgs& a, uint32_t rows, uint64_t vocab) {
  a.vocab = (uint32_t)vocab, a.slice = slice_of(rows, vocab), a.slices = (a.vocab + a.slice - 1) / a.slice;
  a.common = std::min<uint32_t>(kList, (a.vocab + 1) / 2 * 2);
  return std::min(rows, std::max(1u, kAtOnce / a.slices));
}

template <class T>
static hl_status run_sample(SampleArgs a, uint32_t rows, uint32_t each, hipStream_t s) {
  for (uint32_t first = 0; first < rows; first += each) {
    const uint32_t n = std::min(each, rows - first);
    const dim3 grid(a.slices, n);
    hl_status st = enqueue(top_kernel<T>, grid, dim3(kThreads), s, a);
    if (st == HL_OK) st = enqueue(step_kernel<T>, grid, dim3(kThreads), s, a);
    if (st == HL_OK) st = enqueue(list_kernel<T>, grid, dim3(kThreads), s, a);
    if (st == HL_OK) st = enqueue(end_kernel<T>, dim3(n), dim3(kEnd), s, a);
    if (st != HL_OK) return st;
    a.logits = static_cast<const T*>(a.logits) + n * a.stride;
    a.uniforms += n, a.tokens += n, a.logprobs += n;
    if (a.temperatures) a.temperatures += n;
    if (a.top_ks) a.top_ks += n;
    if (a.top_ps) a.top_ps += n;
    if (a.min_ps) a.min_ps += n;
  }
  return HL_OK;
}

}  // namespace hl

using namespace hl;

extern "C" size_t hl_sample_workspace_bytes(uint32_t rows, uint64_t vocab) {
  if (rows == 0 || rows > 65535 || vocab == 0 || vocab >= (1u << 20)) return 0;
  SampleArgs a = {};
  const uint64_t at_once = cut_rows(a, rows, vocab);
  return at_once * a.row_bytes();
}

extern "C" hl_status hl_sample(const hl_sampling* sampling, const void* logits_dev, hl_dtype dtype, uint64_t row_stride,
                               uint32_t rows, uint64_t vocab, const float* uniforms_dev, int32_t* tokens_dev,
                               float* logprobs_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  if (!sampling || !logits_dev || !uniforms_dev || !tokens_dev || !logprobs_dev || !workspace_dev || rows == 0 ||
      vocab == 0 || (rows > 1 && row_stride < vocab))
    return HL_EINVAL;
  const uintptr_t size = dtype == HL_F32 ? 4 : 2;
  if ((dtype != HL_F32 && dtype != HL_BF16 && dtype != HL_F16) || !aligned(logits_dev, size) || !aligned(workspace_dev, 16))
    return HL_EINVAL;
  for (const void* p : {(const void*)uniforms_dev, (const void*)tokens_dev, (const void*)logprobs_dev,
                        (const void*)sampling->temperature_dev, (const void*)sampling->top_k_dev,
                        (const void*)sampling->top_p_dev, (const void*)sampling->min_p_dev})
    if (!aligned(p, 4)) return HL_EINVAL;
  if (vocab >= (1u << 20) || row_stride >= (1ull << 40) || rows > 65535) return HL_EUNSUPPORTED;
  SampleArgs a = {};
  const uint32_t at_once = cut_rows(a, rows, vocab);
  if (workspace_bytes < at_once * a.row_bytes()) return HL_EINVAL;
  a.logits = logits_dev, a.stride = row_stride, a.uniforms = uniforms_dev;
  a.temperatures = sampling->temperature_dev, a.top_ks = sampling->top_k_dev;
  a.top_ps = sampling->top_p_dev, a.min_ps = sampling->min_p_dev;
  a.temperature = sampling->temperature, a.top_k = sampling->top_k, a.top_p = sampling->top_p, a.min_p = sampling->min_p;
  a.tokens = tokens_dev, a.logprobs = logprobs_dev, a.work = static_cast<uint8_t*>(workspace_dev);
  const hipStream_t s = (hipStream_t)stream;
  return dtype == HL_F32    ? run_sample<float>(a, rows, at_once, s)
         : dtype == HL_BF16 ? run_sample<__bf16>(a, rows, at_once, s)
                            : run_sample<_Float16>(a, rows, at_once, s);
}
