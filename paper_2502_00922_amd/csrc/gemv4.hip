// Products with a matrix of 4-bit codes (hl_gemv4):
//   y[b][r] = sum_k x[b][k] * (base + scale * (code[r][k] - 8)),
// a scale (and a base, or none) for each GROUP = 32, 64 or 128 columns of a row.
//
// The matrix instruction's left operand is 16 + code, exact in bf16 and f16 and one
// and-or of a nibble in place; per group the products with x and with ones give
//   scale * (sum x (16 + code) - 24 sum x) + base * sum x.
// A wave has RT 16-row tiles and every W-th stretch of 128 * AHEAD columns, a block
// the W waves of the same rows, which are added in LDS in their order. A lane loads
// 16 bytes of a row, four lanes 64; two rounds of lane swaps turn the four words of
// four lanes, so that each instruction's 32 columns are neighbours and of one group.
#include <algorithm>
#include <type_traits>

#include "gpu_host.h"

namespace hl {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct Gemv4Args {
  const uint8_t* codes;
  const uint16_t *scales, *bases, *x;
  float* y;
  uint32_t rows, cols, batch, groups;  // groups: of a row
};

template <class T>
__device__ inline f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (std::is_same<T, __bf16>::value)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
}

// Ends a row of matrix instructions: the instructions after it may write the
// operands of those before. On gfx950 a product has come out wrong now and then
// when the instruction right after it wrote one of its operand registers; the
// compiler places no wait states there, and five are enough.
__device__ inline void row_end() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 4");
  __builtin_amdgcn_sched_barrier(0);
}

// x of lane N of each 16.
template <int N>
__device__ inline float lane_of(float x) {
  const int i = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, 0x150 + N, 0xF, 0xF, true));
}

// Keeps what is made of v behind the instructions before.
__device__ inline uint32_t after(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}

template <class T>
__device__ inline float number(uint32_t bits) {
  if constexpr (std::is_same<T, __bf16>::value) return __builtin_bit_cast(float, bits << 16);
  return (float)__builtin_bit_cast(T, (uint16_t)bits);
}

template <int N, class F>
__device__ inline void every(F f) {
  if constexpr (N > 0) {
    every<N - 1>(f);
    f(std::integral_constant<int, N - 1>());
  }
}

// Words 0 .. 3 of four lanes, 16 apart, turned: word j of lane group c becomes word
// c of lane group j.
__device__ inline void turn4(u32x4& w) {
  const auto swap32 = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane32_swap(a, b, false, false); };
  const auto swap16 = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane16_swap(a, b, false, false); };
  const u32x2 x = __builtin_bit_cast(u32x2, swap32(w[0], w[2])), y = __builtin_bit_cast(u32x2, swap32(w[1], w[3]));
  const u32x2 u = __builtin_bit_cast(u32x2, swap16(x[0], y[0])), v = __builtin_bit_cast(u32x2, swap16(x[1], y[1]));
  w = u32x4{u[0], u[1], v[0], v[1]};
}

// Columns 0 4 1 5 2 6 3 7 of the 8 whose codes a word has, plus 16, in pairs.
template <class T>
__device__ inline u32x4 operand4(uint32_t w) {
  if constexpr (std::is_same<T, __bf16>::value) {
    constexpr uint32_t m = 0x00780078u, one = 0x41804180u;
    return u32x4{((w << 3) & m) | one, ((w >> 1) & m) | one, ((w >> 5) & m) | one, ((w >> 9) & m) | one};
  }
  constexpr uint32_t m = 0x03C003C0u, one = 0x4C004C00u;
  return u32x4{((w << 6) & m) | one, ((w << 2) & m) | one, ((w >> 2) & m) | one, ((w >> 6) & m) | one};
}

// A stretch's codes and its groups' scales and bases: lane n of each 16 has the
// scale of the stretch's group n, of rows 4c .. 4c+3.
template <int GROUP, bool BASES, int RT, int AHEAD>
struct Stretch {
  u32x4 codes[RT][AHEAD];
  uint32_t scale[RT][4], base[RT][BASES ? 4 : 1];
};

template <int GROUP, bool BASES, int RT, int AHEAD>
__device__ inline void load_stretch(Stretch<GROUP, BASES, RT, AHEAD>& s, const Gemv4Args& a, uint32_t row0,
                                    uint32_t col) {
  const uint32_t lane = threadIdx.x % 64, n = lane % 16, c = lane / 16;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const uint32_t row = min(row0 + 16 * rt + n, a.rows - 1);
    const uint8_t* p = a.codes + (uint64_t)row * (a.cols / 2);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)  // past the columns, the last ones again: x is 0 there
      s.codes[rt][i] = *reinterpret_cast<const u32x4*>(p + min(col + 128 * i + 32 * c, a.cols - 32) / 2);
    const uint32_t g = min(col / GROUP + n, a.groups - 1);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint64_t at = (uint64_t)min(row0 + 16 * rt + 4 * c + r, a.rows - 1) * a.groups + g;
      s.scale[rt][r] = a.scales[at];
      if constexpr (BASES) s.base[rt][r] = a.bases[at];
    }
  }
}

// W waves a block; T, S: types of x and of the scales.
template <class T, class S, int GROUP, bool BASES, int RT, int AHEAD, int W>
__global__ void __launch_bounds__(64 * W) gemv4_kernel(Gemv4Args a) {
  constexpr uint32_t COLS = 128 * AHEAD, RB = BASES ? 4 : 1;
  __shared__ float s_y[W][RT * 16][17];
  const uint32_t lane = threadIdx.x % 64, n = lane % 16, c = lane / 16;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t row0 = blockIdx.x * 16 * RT;
  const uint16_t* xp = a.x + (uint64_t)min(n, a.batch - 1) * a.cols + 8 * c;
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  constexpr uint32_t unit = std::is_same<T, __bf16>::value ? 0x3F803F80u : 0x3C003C00u;
  u32x4 ones = {unit, unit, unit, unit};
  asm volatile("" : "+v"(ones));
  f32x4 y[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) y[rt] = zero;
  Stretch<GROUP, BASES, RT, AHEAD> s;
  uint32_t col = wave * COLS;
  if (col < a.cols) load_stretch(s, a, row0, col);
  while (col < a.cols) {
    Stretch<GROUP, BASES, RT, AHEAD> next;
    if (col + W * COLS < a.cols) load_stretch(next, a, row0, col + W * COLS);
    every<AHEAD>([&](auto nth) {
      constexpr int i = decltype(nth)::value;
      constexpr int PARTS = 128 / GROUP, EACH = 4 / PARTS;  // groups of 128 columns, instructions of a group
      u32x4 xs[4], codes[RT * 4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const uint32_t at = col + 128 * i + 32 * t;
        u32x4 v = {0, 0, 0, 0};
        if (at < a.cols) v = *reinterpret_cast<const u32x4*>(xp + at);
        xs[t] = u32x4{__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                      __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
        asm volatile("" : "+v"(xs[t]));
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        u32x4 w = s.codes[rt][i];
        turn4(w);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          codes[rt * 4 + t] = operand4<T>(w[t]);
          asm volatile("" : "+v"(codes[rt * 4 + t]));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      f32x4 sum[PARTS], part[RT][PARTS];
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        sum[p] = zero;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) part[rt][p] = zero;
#pragma unroll
        for (int t = p * EACH; t < (p + 1) * EACH; ++t) {
          sum[p] = product<T>(ones, xs[t], sum[p]);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) part[rt][p] = product<T>(codes[rt * 4 + t], xs[t], part[rt][p]);
        }
      }
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        asm volatile("" : "+v"(sum[p]));
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) asm volatile("" : "+v"(part[rt][p]));
      }
      row_end();
#pragma unroll
      for (int t = 0; t < 4; ++t) asm volatile("" ::"v"(xs[t]));
#pragma unroll
      for (int t = 0; t < 4 * RT; ++t) asm volatile("" ::"v"(codes[t]));
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float scale = number<S>(after(s.scale[rt][r])), base = BASES ? number<S>(after(s.base[rt][r % RB])) : 0.0f;
          every<PARTS>([&](auto mth) {
            constexpr int p = decltype(mth)::value, g = i * PARTS + p;
            const float v = fmaf(-24.0f, sum[p][r], part[rt][p][r]);
            y[rt][r] = fmaf(lane_of<g>(scale), v, y[rt][r]);
            if constexpr (BASES) y[rt][r] = fmaf(lane_of<g>(base), sum[p][r], y[rt][r]);
          });
        }
    });
    asm volatile("" ::"v"(ones));
    s = next;
    col += W * COLS;
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int r = 0; r < 4; ++r) s_y[wave][16 * rt + 4 * c + r][n] = y[rt][r];
  __syncthreads();
  for (uint32_t x = threadIdx.x; x < a.batch * 16 * RT; x += 64 * W) {
    const uint32_t b = x / (16 * RT), r = x % (16 * RT);
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += s_y[w][r][b];
    if (row0 + r < a.rows) a.y[(uint64_t)b * a.rows + row0 + r] = v;
  }
}

template <class T, class S, int GROUP, bool BASES>
static hl_status run_gemv4(const Gemv4Args& a, hipStream_t s) {
  return enqueue(gemv4_kernel<T, S, GROUP, BASES, 1, 2, 8>, dim3((a.rows + 15) / 16), dim3(512), s, a);
}

template <class T, class S, int GROUP>
static hl_status run_bases(const Gemv4Args& a, hipStream_t s) {
  return a.bases ? run_gemv4<T, S, GROUP, true>(a, s) : run_gemv4<T, S, GROUP, false>(a, s);
}

template <class T, class S>
static hl_status run_group(const Gemv4Args& a, uint32_t group, hipStream_t s) {
  return group == 32 ? run_bases<T, S, 32>(a, s) : group == 64 ? run_bases<T, S, 64>(a, s) : run_bases<T, S, 128>(a, s);
}

}  // namespace hl

using namespace hl;

extern "C" hl_status hl_gemv4(const uint8_t* codes_dev, const void* scales_dev, const void* bases_dev,
                              hl_dtype scale_dtype, uint64_t rows, uint64_t cols, uint32_t group, const void* x_dev,
                              hl_dtype x_dtype, uint32_t batch, float* y_dev, void* stream) {
  if (!codes_dev || !scales_dev || !x_dev || !y_dev || rows == 0 || cols == 0 || batch == 0 || batch > HL_MAX_BATCH)
    return HL_EINVAL;
  if ((group != 32 && group != 64 && group != 128) || cols % group) return HL_EINVAL;
  if ((x_dtype != HL_BF16 && x_dtype != HL_F16) || (scale_dtype != HL_BF16 && scale_dtype != HL_F16)) return HL_EINVAL;
  if (!aligned(codes_dev, 16) || !aligned(x_dev, 16) || !aligned(scales_dev, 2) || !aligned(bases_dev, 2) ||
      !aligned(y_dev, 4))
    return HL_EINVAL;
  if (cols >= (1ull << 31) || rows >= (1ull << 31) || !grid_fits((rows + 15) / 16, 1024)) return HL_EUNSUPPORTED;
  Gemv4Args a = {};
  a.codes = codes_dev, a.scales = static_cast<const uint16_t*>(scales_dev);
  a.bases = static_cast<const uint16_t*>(bases_dev), a.x = static_cast<const uint16_t*>(x_dev), a.y = y_dev;
  a.rows = (uint32_t)rows, a.cols = (uint32_t)cols, a.batch = batch, a.groups = (uint32_t)(cols / group);
  const hipStream_t s = (hipStream_t)stream;
  if (x_dtype == HL_BF16)
    return scale_dtype == HL_BF16 ? run_group<__bf16, __bf16>(a, group, s) : run_group<__bf16, _Float16>(a, group, s);
  return scale_dtype == HL_BF16 ? run_group<_Float16, __bf16>(a, group, s) : run_group<_Float16, _Float16>(a, group, s);
}
