// RMS norm with the residual's addition (hl_rms_norm): what stands between
// two compressed products of a decoder layer.
//
//   t = x + r,  y = t / sqrt(mean(t^2) + eps) * w
//
// y goes out in 32 or 16 bits, or in 8 (e4m3) with one float32 scale per group
// of columns: scale = max|y| / 448. t is held in float32 throughout: the norm
// is of the unrounded sum, and the sum is rounded once, to r's type.
//
// One row stays in the registers of its waves between the sum of squares and
// the scaling, so each input is read once and each output written once. Many
// rows are bound by HBM: 8192 rows of 8192 columns, bf16 to e4m3, take 90 us,
// 5.2 TB/s; 1021 rows of 4101 columns, float16, 9.2 us. Few rows are bound by
// the launch and two waits for memory: one of 4096, 3.3 us.
#include <algorithm>

#include "gpu_host.h"

namespace hl {

constexpr float kE4m3Max = 448.0f;
constexpr float kLeastNormal = 1.17549435e-38f;
constexpr uint32_t kMostHidden = HL_NORM_MAX_HIDDEN;

struct NormArgs {
  const void *x, *residual, *weight;
  void *sum, *out;
  float* scale;
  uint32_t tokens, hidden, group;  // group: columns per scale (0: the row)
  uint32_t waves;                  // of a row
  hl_dtype xt, rt, wt, ot;
  float eps;
};

constexpr int W = 8;  // columns of a load

// W consecutive elements as they lie in memory: W dwords hold them in any type.
struct Raw {
  uint32_t w[W];
};

// A row may start at any element: the copies become the widest loads and
// stores, which need no alignment (1021 rows of 4101 float16 take 9.2 us where
// loads of single elements took 21).
template <class E>
__device__ inline void load(Raw& r, const void* p, uint64_t at) {
  __builtin_memcpy(r.w, static_cast<const E*>(p) + at, W * sizeof(E));
}

// Loads all of a thread's vectors of one operand, with the choice of its type
// outside the loop so that they are in flight together.
template <int V>
__device__ inline void load_row(Raw (&r)[V], const void* p, hl_dtype t, uint64_t row, uint32_t end, uint32_t first,
                                uint32_t step) {
  if (t == HL_F32) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (first + v * step < end) load<uint32_t>(r[v], p, row + first + v * step);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (first + v * step < end) load<uint16_t>(r[v], p, row + first + v * step);
  }
}

__device__ inline float value_of(uint32_t bits, hl_dtype t) {
  if (t == HL_F32) return __builtin_bit_cast(float, bits);
  if (t == HL_BF16) return __builtin_bit_cast(float, bits << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// The type is looked at once for all W: a branch an element cost up to a
// quarter (4096 rows of 28672 bf16: 219 us, so 191).
__device__ inline void values(float (&f)[W], const Raw& r, hl_dtype t) {
  if (t == HL_F32) {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = __builtin_bit_cast(float, r.w[i]);
  } else if (t == HL_BF16) {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = __builtin_bit_cast(float, i % 2 ? r.w[i / 2] & 0xFFFF0000u : r.w[i / 2] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r.w[i / 2] >> (i % 2 * 16)));
  }
}

__device__ inline float one(const void* p, hl_dtype t, uint64_t at) {
  return value_of(t == HL_F32 ? static_cast<const uint32_t*>(p)[at] : static_cast<const uint16_t*>(p)[at], t);
}

__device__ inline void store(const float (&f)[W], void* p, hl_dtype t, uint64_t at) {
  if (t == HL_F32) {
    __builtin_memcpy(static_cast<float*>(p) + at, f, sizeof(f));
    return;
  }
  uint16_t h[W];
  if (t == HL_BF16) {
#pragma unroll
    for (int i = 0; i < W; ++i) h[i] = __builtin_bit_cast(uint16_t, (__bf16)f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < W; ++i) h[i] = __builtin_bit_cast(uint16_t, (_Float16)f[i]);
  }
  __builtin_memcpy(static_cast<uint16_t*>(p) + at, h, sizeof(h));
}

__device__ inline void store_one(float f, void* p, hl_dtype t, uint64_t at) {
  if (t == HL_F32)
    static_cast<float*>(p)[at] = f;
  else
    static_cast<uint16_t*>(p)[at] =
        t == HL_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)f) : __builtin_bit_cast(uint16_t, (_Float16)f);
}

// Two values to e4m3, in the low or the high half of `other` (to nearest, ties
// to even; the largest where the value's rounding would pass it).
template <bool HIGH>
__device__ inline uint32_t e4m3(float x, float y, uint32_t other) {
  x = x != x ? x : fminf(fmaxf(x, -kE4m3Max), kE4m3Max);
  y = y != y ? y : fminf(fmaxf(y, -kE4m3Max), kE4m3Max);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, (int)other, HIGH);
}

// f / scale. Divided: the product with a rounded 1 / scale comes out a step of
// e4m3 off for some quotients next to the middle of two. 8192 rows
// of 8192 columns take 90 us, and 84 with the product; 4096 of 28672 229 and 197.
__device__ inline void store_e4m3(const float (&f)[W], float scale, void* p, uint64_t at) {
  uint32_t d[W / 4];
#pragma unroll
  for (int i = 0; i < W / 4; ++i) {
    d[i] = e4m3<false>(f[4 * i] / scale, f[4 * i + 1] / scale, 0);
    d[i] = e4m3<true>(f[4 * i + 2] / scale, f[4 * i + 3] / scale, d[i]);
  }
  __builtin_memcpy(static_cast<uint8_t*>(p) + at, d, sizeof(d));
}

// Sum (or maximum) over the waves of a row, the same in all of them. `slot`:
// a row of LDS that no other reduction of this launch uses.
template <bool MAX>
__device__ inline float over_row(float v, uint32_t waves, float* slot) {
  for (int d = 32; d; d >>= 1) {
    const float o = __shfl_xor(v, d);
    v = MAX ? fmaxf(v, o) : v + o;
  }
  if (waves == 1) return v;
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  if (lane == 0) slot[wave] = v;
  __syncthreads();
  v = lane < waves ? slot[lane] : 0.0f;
  for (int d = 8; d; d >>= 1) {
    const float o = __shfl_xor(v, d);
    v = MAX ? fmaxf(v, o) : v + o;
  }
  return __shfl(v, 0);
}

// V loads a thread and operand. A block is one row of `waves` waves, or
// (waves == 1) blockDim/64 rows. Lane l of a row holds columns
// (v*threads + l)*W .., so loads are contiguous over the lanes and a group of
// 32, 64 or 128 columns is 4, 8 or 16 neighbouring lanes. Up to 7 columns at
// the row's end that make no whole load are one lane's each.
template <int V>
__global__ void __launch_bounds__(1024) norm_kernel(NormArgs a) {
  __shared__ float s_sum[16], s_max[16];
  const uint32_t rows = a.waves == 1 ? blockDim.x / 64 : 1;
  const uint32_t token = blockIdx.x * rows + (a.waves == 1 ? threadIdx.x / 64 : 0);
  if (token >= a.tokens) return;  // a whole wave, and only where a wave is a row
  const uint32_t tid = a.waves == 1 ? threadIdx.x % 64 : threadIdx.x;
  const uint32_t first = tid * W, step = a.waves * 64 * W, end = a.hidden / W * W;
  const uint64_t row = (uint64_t)token * a.hidden;
  Raw x[V], r[V], g[V];
  load_row<V>(x, a.x, a.xt, row, end, first, step);
  if (a.residual) load_row<V>(r, a.residual, a.rt, row, end, first, step);
  load_row<V>(g, a.weight, a.wt, 0, end, first, step);
  const bool odd = tid < a.hidden - end;
  const uint64_t last = row + end + tid;
  float t1 = 0.0f, g1 = 0.0f;
  if (odd) {
    t1 = one(a.x, a.xt, last), g1 = one(a.weight, a.wt, end + tid);
    if (a.residual) store_one(t1 += one(a.residual, a.rt, last), a.sum, a.rt, last);
  }
  float t[V][W], sq = t1 * t1;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const bool in = first + v * step < end;
    if (in) {
      values(t[v], x[v], a.xt);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) t[v][i] = 0.0f;
    }
    if (a.residual && in) {
      float f[W];
      values(f, r[v], a.rt);
#pragma unroll
      for (int i = 0; i < W; ++i) t[v][i] += f[i];
      store(t[v], a.sum, a.rt, row + first + v * step);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) sq = fmaf(t[v][i], t[v][i], sq);
  }
  const float inv = 1.0f / sqrtf(over_row<false>(sq, a.waves, s_sum) / (float)a.hidden + a.eps);
  t1 = t1 * inv * g1;  // in this order: inv * weight may leave the range where out does not
  float most = odd ? fabsf(t1) : 0.0f;
  if (odd && a.ot != HL_E4M3) store_one(t1, a.out, a.ot, last);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t at = first + v * step;
    if (at < end) {
      float f[W];
      values(f, g[v], a.wt);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        t[v][i] = t[v][i] * inv * f[i];
        most = fmaxf(most, fabsf(t[v][i]));
      }
      if (a.ot != HL_E4M3) store(t[v], a.out, a.ot, row + at);
    }
  }
  if (a.ot != HL_E4M3) return;
  auto scale_of = [](float top) {
    const float s = top / kE4m3Max;
    return s >= kLeastNormal ? s : 1.0f;
  };
  if (a.group == 0) {
    const float s = scale_of(over_row<true>(most, a.waves, s_max));
    if (tid == 0) a.scale[token] = s;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (first + v * step < end) store_e4m3(t[v], s, a.out, row + first + v * step);
    if (odd) static_cast<uint8_t*>(a.out)[last] = (uint8_t)e4m3<false>(t1 / s, 0.0f, 0);
    return;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t at = first + v * step;
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) top = fmaxf(top, fabsf(t[v][i]));  // zeros past the row's end
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    const float wider = fmaxf(top, __shfl_xor(top, 4));
    top = a.group > 32 ? wider : top;
    const float widest = fmaxf(top, __shfl_xor(top, 8));
    top = a.group > 64 ? widest : top;
    if (at < end) {
      const float s = scale_of(top);
      if (at % a.group == 0) a.scale[(uint64_t)token * (a.hidden / a.group) + at / a.group] = s;
      store_e4m3(t[v], s, a.out, row + at);
    }
  }
}

template <int V>
static hl_status launch_norm(const NormArgs& a, hipStream_t s) {
  const uint32_t rows = a.waves == 1 ? 4 : 1, threads = a.waves == 1 ? 256 : a.waves * 64;
  const uint64_t blocks = ((uint64_t)a.tokens + rows - 1) / rows;
  if (!grid_fits(blocks, threads)) return HL_EUNSUPPORTED;
  return enqueue(norm_kernel<V>, dim3((uint32_t)blocks), dim3(threads), s, a);
}

static uint32_t dtype_bytes(hl_dtype t) { return t == HL_F32 ? 4 : t == HL_E4M3 ? 1 : 2; }

}  // namespace hl

using namespace hl;

extern "C" hl_status hl_rms_norm(const void* x_dev, hl_dtype x_dtype, const void* residual_dev, hl_dtype r_dtype,
                                 const void* weight_dev, hl_dtype w_dtype, uint64_t tokens, uint64_t hidden, float eps,
                                 void* sum_dev, void* out_dev, hl_dtype out_dtype, uint32_t group, float* scale_dev,
                                 void* stream) {
  auto value = [](hl_dtype t) { return t == HL_F32 || t == HL_BF16 || t == HL_F16; };
  if (!x_dev || !weight_dev || !out_dev || tokens == 0 || hidden == 0 || !(eps >= 0.0f)) return HL_EINVAL;
  if (!value(x_dtype) || !value(w_dtype) || (!value(out_dtype) && out_dtype != HL_E4M3)) return HL_EINVAL;
  if (residual_dev && (!value(r_dtype) || !sum_dev)) return HL_EINVAL;
  const bool e4m3 = out_dtype == HL_E4M3;
  if (e4m3 ? !scale_dev || !aligned(scale_dev, 4) : group != 0) return HL_EINVAL;
  if (group && ((group != 32 && group != 64 && group != 128) || hidden % group)) return HL_EINVAL;
  // every pointer at its element's size (the loads take any address), and with a
  // group at 16 bytes, as the header has it
  bool wide = aligned(x_dev, 16) && aligned(weight_dev, 16) && aligned(out_dev, 16);
  bool fits = aligned(x_dev, dtype_bytes(x_dtype)) && aligned(weight_dev, dtype_bytes(w_dtype)) &&
              aligned(out_dev, dtype_bytes(out_dtype));
  if (residual_dev) {
    wide = wide && aligned(residual_dev, 16) && aligned(sum_dev, 16);
    fits = fits && aligned(residual_dev, dtype_bytes(r_dtype)) && aligned(sum_dev, dtype_bytes(r_dtype));
  }
  if (!fits || (group && !wide)) return HL_EINVAL;
  if (hidden > kMostHidden || tokens >= (1ull << 31)) return HL_EUNSUPPORTED;

  NormArgs a = {};
  a.x = x_dev, a.residual = residual_dev, a.weight = weight_dev, a.sum = sum_dev, a.out = out_dev;
  a.scale = scale_dev;
  a.tokens = (uint32_t)tokens, a.hidden = (uint32_t)hidden, a.group = group;
  a.xt = x_dtype, a.rt = r_dtype, a.wt = w_dtype, a.ot = out_dtype, a.eps = eps;
  const hipStream_t s = (hipStream_t)stream;
  // The fewest loads a thread that 8 waves a row allow (16, where 4 loads do not
  // do): with more waves, fewer rows are on a compute unit at a time. 2048 rows
  // of 16384 to e4m3 take 51 us with 8 waves and 65 with 16, one row of 8192
  // takes 3.8 us with either.
  const uint32_t vectors = std::max(a.hidden / W, 1u), each = vectors <= 512 ? 1 : vectors <= 1024 ? 2 : 4;
  a.waves = (vectors + each * 64 - 1) / (each * 64);
  if (each == 1) return launch_norm<1>(a, s);
  if (each == 2) return launch_norm<2>(a, s);
  return launch_norm<4>(a, s);
}
