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
// the scaling, so each input is read once and each output written once: the
// kernel is bound by HBM on many rows, and by launch and two load latencies on
// few.
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

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// W consecutive elements as they lie in memory: W dwords hold them in any type.
template <int W>
struct Raw {
  uint32_t __attribute__((ext_vector_type(W))) w;
};

template <int W>
__device__ inline void load_32(Raw<W>& r, const void* p, uint64_t at) {
  const uint32_t* q = reinterpret_cast<const uint32_t*>(p) + at;
  if constexpr (W >= 4) {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(q + i);
      for (int j = 0; j < 4; ++j) r.w[i + j] = v[j];
    }
  } else {
    for (int i = 0; i < W; ++i) r.w[i] = q[i];
  }
}

template <int W>
__device__ inline void load_16(Raw<W>& r, const void* p, uint64_t at) {
  const uint16_t* q = reinterpret_cast<const uint16_t*>(p) + at;
  if constexpr (W == 8) {
    const u32x4 v = *reinterpret_cast<const u32x4*>(q);
    for (int j = 0; j < 4; ++j) r.w[j] = v[j];
  } else if constexpr (W == 4) {
    const u32x2 v = *reinterpret_cast<const u32x2*>(q);
    r.w[0] = v[0], r.w[1] = v[1];
  } else {
    r.w[0] = q[0];
  }
}

// Loads all of a thread's vectors of one operand, with the choice of its type
// outside the loop so that they are in flight together.
template <int W, int V>
__device__ inline void load_row(Raw<W> (&r)[V], const void* p, hl_dtype t, uint64_t row, uint32_t hidden,
                                uint32_t first, uint32_t step) {
  if (t == HL_F32) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (first + v * step < hidden) load_32(r[v], p, row + first + v * step);
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (first + v * step < hidden) load_16(r[v], p, row + first + v * step);
  }
}

template <int W>
__device__ inline float element(const Raw<W>& r, hl_dtype t, int i) {
  const uint32_t whole = r.w[i];
  if (t == HL_F32) return __builtin_bit_cast(float, whole);
  const uint32_t h = W == 1 ? r.w[0] : (r.w[i / 2] >> (i % 2 * 16)) & 0xFFFF;
  if (t == HL_BF16) return __builtin_bit_cast(float, h << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
}

__device__ inline uint32_t half_bits(float f, hl_dtype t) {
  return t == HL_BF16 ? (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f)
                      : (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)f);
}

template <int W>
__device__ inline void store(const float (&f)[W], void* p, hl_dtype t, uint64_t at) {
  if (t == HL_F32) {
    float* q = reinterpret_cast<float*>(p) + at;
    if constexpr (W >= 4) {
      for (int i = 0; i < W; i += 4) *reinterpret_cast<float4*>(q + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
    } else {
      for (int i = 0; i < W; ++i) q[i] = f[i];
    }
    return;
  }
  uint16_t* q = reinterpret_cast<uint16_t*>(p) + at;
  if constexpr (W == 1) {
    q[0] = (uint16_t)half_bits(f[0], t);
  } else {
    uint32_t d[W / 2];
#pragma unroll
    for (int i = 0; i < W / 2; ++i) d[i] = half_bits(f[2 * i], t) | (half_bits(f[2 * i + 1], t) << 16);
    if constexpr (W == 8)
      *reinterpret_cast<u32x4*>(q) = u32x4{d[0], d[1], d[2], d[3]};
    else
      *reinterpret_cast<u32x2*>(q) = u32x2{d[0], d[1]};
  }
}

// Rounds W values to e4m3 (to nearest, ties to even; the largest where the
// scaled value's rounding would pass it).
template <int W>
__device__ inline void store_e4m3(const float (&f)[W], float inv, void* p, uint64_t at) {
  uint8_t* q = reinterpret_cast<uint8_t*>(p) + at;
  float s[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const float y = f[i] * inv;
    s[i] = y != y ? y : fminf(fmaxf(y, -kE4m3Max), kE4m3Max);
  }
  if constexpr (W == 1) {
    q[0] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(s[0], s[0], 0, false);
  } else {
    uint32_t d[W / 4];
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      int b = __builtin_amdgcn_cvt_pk_fp8_f32(s[4 * i], s[4 * i + 1], 0, false);
      d[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(s[4 * i + 2], s[4 * i + 3], b, true);
    }
    if constexpr (W == 8)
      *reinterpret_cast<u32x2*>(q) = u32x2{d[0], d[1]};
    else
      *reinterpret_cast<uint32_t*>(q) = d[0];
  }
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

// W elements a load, V loads a thread. A block is one row of `waves` waves, or
// (waves == 1) blockDim/64 rows. Lane l of a row holds columns
// (v*threads + l)*W .., so loads are contiguous over the lanes and a group of
// 32, 64 or 128 columns is 4, 8 or 16 neighbouring lanes.
template <int W, int V>
__global__ void __launch_bounds__(1024) norm_kernel(NormArgs a) {
  __shared__ float s_sum[16], s_max[16];
  const uint32_t rows = a.waves == 1 ? blockDim.x / 64 : 1;
  const uint32_t token = blockIdx.x * rows + (a.waves == 1 ? threadIdx.x / 64 : 0);
  if (token >= a.tokens) return;  // a whole wave, and only where a wave is a row
  const uint32_t tid = a.waves == 1 ? threadIdx.x % 64 : threadIdx.x;
  const uint32_t first = tid * W, step = a.waves * 64 * W;
  const uint64_t row = (uint64_t)token * a.hidden;
  Raw<W> x[V], r[V], g[V];
  load_row<W, V>(x, a.x, a.xt, row, a.hidden, first, step);
  if (a.residual) load_row<W, V>(r, a.residual, a.rt, row, a.hidden, first, step);
  load_row<W, V>(g, a.weight, a.wt, 0, a.hidden, first, step);
  float t[V][W], sq = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const bool in = first + v * step < a.hidden;
#pragma unroll
    for (int i = 0; i < W; ++i) t[v][i] = in ? element(x[v], a.xt, i) : 0.0f;
    if (a.residual && in) {
#pragma unroll
      for (int i = 0; i < W; ++i) t[v][i] += element(r[v], a.rt, i);
      store(t[v], a.sum, a.rt, row + first + v * step);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) sq = fmaf(t[v][i], t[v][i], sq);
  }
  const float inv = 1.0f / sqrtf(over_row<false>(sq, a.waves, s_sum) / (float)a.hidden + a.eps);
  float most = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const uint32_t at = first + v * step;
    if (at < a.hidden) {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        t[v][i] *= inv * element(g[v], a.wt, i);
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
      if (first + v * step < a.hidden) store_e4m3(t[v], 1.0f / s, a.out, row + first + v * step);
    return;
  }
  if constexpr (W == 8) {  // a group's rows start at 16 bytes, so its loads are of 8
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
      if (at < a.hidden) {
        const float s = scale_of(top);
        if (at % a.group == 0) a.scale[(uint64_t)token * (a.hidden / a.group) + at / a.group] = s;
        store_e4m3(t[v], 1.0f / s, a.out, row + at);
      }
    }
  }
}

template <int W, int V>
static hl_status launch_norm(const NormArgs& a, hipStream_t s) {
  const uint32_t rows = a.waves == 1 ? 4 : 1;
  return enqueue(norm_kernel<W, V>, dim3((a.tokens + rows - 1) / rows), dim3(a.waves == 1 ? 256 : a.waves * 64), s, a);
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
  // every pointer at its element's size; 16 bytes allow the widest loads
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
  // The widest load that every row's start allows; the fewest loads a thread
  // that 16 waves a row allow.
  const uint32_t width = !wide ? 1 : hidden % 8 == 0 ? 8 : hidden % 4 == 0 ? 4 : 1;
  const uint32_t vectors = (uint32_t)((hidden + width - 1) / width);
  uint32_t each = width == 1 ? 4 : 1;
  while (each * 1024 < vectors) each *= 2;
  a.waves = (vectors + each * 64 - 1) / (each * 64);
  if (width == 8) {
    if (each == 1) return launch_norm<8, 1>(a, s);
    if (each == 2) return launch_norm<8, 2>(a, s);
    return launch_norm<8, 4>(a, s);
  }
  if (width == 4) {
    if (each == 1) return launch_norm<4, 1>(a, s);
    if (each == 2) return launch_norm<4, 2>(a, s);
    if (each == 4) return launch_norm<4, 4>(a, s);
    return launch_norm<4, 8>(a, s);
  }
  if (each == 4) return launch_norm<1, 4>(a, s);
  if (each == 8) return launch_norm<1, 8>(a, s);
  if (each == 16) return launch_norm<1, 16>(a, s);
  return launch_norm<1, 32>(a, s);
}
