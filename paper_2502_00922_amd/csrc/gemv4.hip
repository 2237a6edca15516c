// Products with a matrix of 4-bit codes (hl_gemv4):
//   y[b][r] = sum_k x[b][k] * (base + scale * (code[r][k] - 8)),
// a scale (and a base, or none) for each GROUP = 32, 64 or 128 columns of a row.
//
// The matrix instruction's right operand is 16 + code, exact in bf16 and f16 and a shift
// and an and-or of a nibble; what is too much of it is where the sums begin: a product of
// x with a constant operand that all rows share. (128 or 64 + code, where a nibble is in
// place for it, save a shift in four and lose three bits of the sums and of their range.)
// x is the left one: a lane's four sums are then of one row of the matrix, whose scale
// the lane has loaded itself.
// A wave has RT 16-row tiles and every W-th stretch of 512 columns, a block the W waves
// of the same rows, which are added in LDS in their order. A lane loads 16 bytes of a
// row, four lanes 64; two rounds of lane swaps turn the four words of four lanes, so
// that each instruction's 32 columns are neighbours and of one group.
// Bound by the loads' way to the compute units where there are few rows (4096 x 4096
// for one row of x 5.2 us, 1.7 TB/s, the waves at waits 56 % of their time). Of 28672 x
// 8192 for 16 with bases (60 us, 2.2 TB/s) neither memory nor the vector (28 %) nor the
// matrix units (10 %) are the bound by themselves: the 1.4 waves that a SIMD has in the mean
// wait for their instructions' turn 53 % of their time and for loads 22 %. Sixteen
// waves a block instead of eight for matrices of at most 2048 rows gain nothing (1024 x
// 8192 for one 6.8 and 7.7 us).
#include <algorithm>
#include <type_traits>

#include "gpu_host.h"
#include "matrix.h"

namespace hl {

struct Gemv4Args {
  const uint8_t* codes;
  const uint16_t *scales, *bases, *x;
  float* y;
  uint32_t rows, cols, batch, groups;  // groups: of a row
};

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

// Words 0 .. 3 of four lanes, 16 apart, turned: word j of lane group c becomes word
// c of lane group j.
__device__ inline void turn4(u32x4& w) {
  const auto swap32 = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane32_swap(a, b, false, false); };
  const auto swap16 = [](uint32_t a, uint32_t b) { return __builtin_amdgcn_permlane16_swap(a, b, false, false); };
  const u32x2 x = __builtin_bit_cast(u32x2, swap32(w[0], w[2])), y = __builtin_bit_cast(u32x2, swap32(w[1], w[3]));
  const u32x2 u = __builtin_bit_cast(u32x2, swap16(x[0], y[0])), v = __builtin_bit_cast(u32x2, swap16(x[1], y[1]));
  w = u32x4{u[0], u[1], v[0], v[1]};
}

// The right operand of 8 columns' codes, columns 0 4 1 5 2 6 3 7 in pairs.
template <class T>
__device__ inline u32x4 operand(const Codes<T>& form, uint32_t w) {
  return u32x4{form.template pair<0>(w), form.template pair<4>(w), form.template pair<8>(w), form.template pair<12>(w)};
}

// Rows from which on a wave has two row tiles, and a block four waves: x is loaded
// for both, and there are blocks enough. us, one tile and eight waves against this:
// 28672 x 8192 for 16 rows 82 and 59, for one 40 and 36, 8192 x 28672 for 16 rows 76
// and 51, 8192 x 8192 for four 15.5 and 12.9; 4096 x 4096 for one 5.5 and 7.1, 1024 x
// 8192 for 16 13.3 and 15.7.
constexpr uint32_t kTwoTiles = 8192;
constexpr int kChunks = 4;  // of 128 columns: a stretch, whose groups' scales are loaded together
constexpr uint32_t kStretch = 128 * kChunks;

// The scales (or bases) of a stretch's groups, of the lane's rows, in pairs.
template <int GROUP, int RT>
struct Scales {
  static constexpr int N = kStretch / GROUP;
  uint32_t v[RT][N / 2];
};

// row: the lane's rows' first, counted in elements from the block's first row; total:
// elements from there to the tensor's end. A row's pairs may begin in the middle of a
// word (loads of other alignments take twice the time), and the last ones begin early
// enough to end in the tensor. Past a row's end are the next one's: no group has them.
template <int GROUP, int RT>
__device__ inline void load_scales(Scales<GROUP, RT>& s, const Gemv4Args& a, const uint16_t* from, uint32_t first, uint64_t total,
                                   const uint32_t (&row)[RT]) {
  constexpr uint32_t N = Scales<GROUP, RT>::N, WORDS = N / 2 + 1;
  if (total < N + 2) {  // a few scales in all
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (uint32_t g = 0; g < N; g += 2) {
        const uint32_t low = from[min(row[rt] + first + g, (uint32_t)total - 1)];
        s.v[rt][g / 2] = low | (uint32_t)from[min(row[rt] + first + g + 1, (uint32_t)total - 1)] << 16;
      }
    return;
  }
  // An odd number of groups puts every second row's first in the middle of a word, for
  // which the load has one word more.
  const bool odd = a.groups % 2;
  const uint32_t last = ((uint32_t)min(total, (uint64_t)0xFFFFFFF0u) - N - 2 * odd) & ~1u;
  uint32_t w[RT][WORDS], early[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const uint32_t at = row[rt] + first, to = min(at & ~1u, last);
    early[rt] = at - to;
    __builtin_memcpy(w[rt], __builtin_assume_aligned(from + to, 4), 2 * N);  // 16 rows begin at a word
  }
  if (odd) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      w[rt][N / 2] = *reinterpret_cast<const uint32_t*>(from + (row[rt] + first - early[rt] + N));
#pragma unroll
      for (uint32_t g = 0; g < N / 2; ++g) s.v[rt][g] = __builtin_amdgcn_alignbit(w[rt][g + 1], w[rt][g], early[rt] % 2 * 16);
    }
  } else {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (uint32_t g = 0; g < N / 2; ++g) s.v[rt][g] = w[rt][g];
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (!__any(early[rt] > 1)) continue;
#pragma unroll 1
    for (uint32_t i = 2; i < N + 2; i += 2)
#pragma unroll
      for (uint32_t g = 0; g < N / 2; ++g) {
        const uint32_t next = g + 1 < N / 2 ? s.v[rt][g + 1 < N / 2 ? g + 1 : 0]
                                            : i == 2 && odd ? w[rt][N / 2] >> (early[rt] % 2 * 16) : 0;
        s.v[rt][g] = i <= early[rt] ? next : s.v[rt][g];
      }
    if (total % 2) {  // the tensor's last scale is half a word
      const uint32_t end = from[total - 1], at = (uint32_t)total - 1 - row[rt] - first;
#pragma unroll
      for (uint32_t g = 0; g < N / 2; ++g)
        s.v[rt][g] = at == 2 * g ? end : at == 2 * g + 1 ? (s.v[rt][g] & 0xFFFFu) | end << 16 : s.v[rt][g];
    }
  }
}

// 128 columns' codes and x.
template <int RT>
struct Chunk {
  u32x4 codes[RT], x[4];
};

// codes, x: at the block's first row and the batch's; row, b: the lane's offsets from
// there. Past the columns, the last ones again: x is taken as 0 there.
template <int RT>
__device__ inline void load_chunk(Chunk<RT>& k, const Gemv4Args& a, const uint8_t* codes, const uint32_t (&row)[RT],
                                  uint32_t b, uint32_t col) {
  const uint8_t* x = reinterpret_cast<const uint8_t*>(a.x);
  col = min(col, a.cols - 32);
  const uint32_t at = min(threadIdx.x % 64 / 16 * 32, a.cols - 32 - col) / 2;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) k.codes[rt] = *reinterpret_cast<const u32x4*>(codes + col / 2 + (row[rt] + at));
#pragma unroll
  for (int t = 0; t < 4; ++t) k.x[t] = *reinterpret_cast<const u32x4*>(x + 2 * min(col + 32 * t, a.cols - 32) + b);
}

// The product's loop reads a chunk ahead of the one it multiplies: everything
// that a chunk takes is on its way before, x as well, for loads come back in order and
// a wait for x would be one for the codes behind it.
// W waves a block; T, S: types of x and of the scales.
template <class T, class S, int GROUP, bool BASES, int RT, int W>
__global__ void __launch_bounds__(64 * W, 2) gemv4_kernel(Gemv4Args a) {
  constexpr int PARTS = 128 / GROUP, EACH = 4 / PARTS;  // groups of a chunk, instructions of a group
  constexpr int SET = RT < 2 ? RT : 2;                  // row tiles whose products follow each other
  __shared__ float s_y[W][RT * 16][17];
  const uint32_t lane = threadIdx.x % 64, n = lane % 16, c = lane / 16;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t row0 = blockIdx.x * 16 * RT, b = (min(n, a.batch - 1) * a.cols + 8 * c) * 2;
  const uint8_t* first = a.codes + (uint64_t)row0 * (a.cols / 2);
  const uint16_t* first_scale = a.scales + (uint64_t)row0 * a.groups;
  const uint16_t* first_base = BASES ? a.bases + (uint64_t)row0 * a.groups : nullptr;
  uint32_t row[RT], scale_row[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const uint32_t r = min(row0 + 16 * rt + n, a.rows - 1) - row0;
    row[rt] = r * (a.cols / 2), scale_row[rt] = r * a.groups;
  }
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  const Codes<T> form;
  constexpr uint32_t unit = std::is_same<T, __bf16>::value ? 0x3F803F80u : 0x3C003C00u;
  u32x4 ones = {unit, unit, unit, unit}, offset = {Codes<T>::LESS, Codes<T>::LESS, Codes<T>::LESS, Codes<T>::LESS};
  asm volatile("" : "+v"(ones), "+v"(offset));
  f32x4 y[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) y[rt] = zero;
  Scales<GROUP, RT> scale, next_scale, base, next_base;
  const uint64_t total = (uint64_t)(a.rows - row0) * a.groups;
  const auto scales_at = [&](uint32_t col) {
    load_scales<GROUP, RT>(next_scale, a, first_scale, col / GROUP, total, scale_row);
    if constexpr (BASES) load_scales<GROUP, RT>(next_base, a, first_base, col / GROUP, total, scale_row);
  };
  Chunk<RT> ring[2];
  // Blocks begin at different columns: rows are often a power of two apart, and all
  // blocks at one column would keep few of the memory's channels busy.
  const uint32_t stretches = (a.cols + kStretch - 1) / kStretch, turn = blockIdx.x % stretches;
  const auto column = [&](uint32_t i) { return (i + turn < stretches ? i + turn : i + turn - stretches) * kStretch; };
  uint32_t nth = wave, col = nth < stretches ? column(nth) : a.cols;
  if (nth < stretches) {
    scales_at(col);
    load_chunk<RT>(ring[0], a, first, row, b, col);
  }
  while (nth < stretches) {
    scale = next_scale;
    if constexpr (BASES) base = next_base;
    nth += W;
    const uint32_t then = nth < stretches ? column(nth) : col;
    scales_at(then);
    each<kChunks>([&](auto chunk) {
      constexpr int i = decltype(chunk)::value;
      const uint32_t at = col + 128 * i, next = i + 1 < kChunks ? at + 128 : then;
      load_chunk<RT>(ring[(i + 1) % 2], a, first, row, b, next);
      if (at >= a.cols) return;
      Chunk<RT>& k = ring[i % 2];
      if (at + 128 > a.cols) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (at + 32 * t >= a.cols) k.x[t] = u32x4{0, 0, 0, 0};
      }
      u32x4 xs[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const u32x4 v = k.x[t];
        xs[t] = u32x4{__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                      __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
        asm volatile("" : "+v"(xs[t]));
      }
      f32x4 sum[PARTS], less[PARTS];  // of x; of x times the offsets
#pragma unroll
      for (int r0 = 0; r0 < RT; r0 += SET) {
        u32x4 codes[SET * 4];
#pragma unroll
        for (int rt = 0; rt < SET; ++rt) {
          u32x4 w = k.codes[r0 + rt];
          turn4(w);
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            codes[rt * 4 + t] = operand(form, w[t]);
            asm volatile("" : "+v"(codes[rt * 4 + t]));
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x4 part[SET][PARTS];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          if (r0 == 0) {
#pragma unroll
            for (int t = p * EACH; t < (p + 1) * EACH; ++t) {
              less[p] = mfma<T>(xs[t], offset, t == p * EACH ? zero : less[p]);
              if constexpr (BASES) sum[p] = mfma<T>(xs[t], ones, t == p * EACH ? zero : sum[p]);
            }
          }
        }
#pragma unroll
        for (int t = 0; t < EACH; ++t)
#pragma unroll
          for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int rt = 0; rt < SET; ++rt)
              part[rt][p] = mfma<T>(xs[p * EACH + t], codes[rt * 4 + p * EACH + t], t == 0 ? less[p] : part[rt][p]);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          if constexpr (BASES) asm volatile("" : "+v"(sum[p]));
          asm volatile("" : "+v"(less[p]));
#pragma unroll
          for (int rt = 0; rt < SET; ++rt) asm volatile("" : "+v"(part[rt][p]));
        }
        products_end();
#pragma unroll
        for (int t = 0; t < 4; ++t) asm volatile("" ::"v"(xs[t]));
#pragma unroll
        for (int t = 0; t < 4 * SET; ++t) asm volatile("" ::"v"(codes[t]));
        asm volatile("" ::"v"(ones), "v"(offset));
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          if (at + GROUP * p >= a.cols) break;  // what is there is not this row's
          constexpr auto pick = [](uint32_t pair, int g) { return g % 2 ? pair >> 16 : pair & 0xFFFFu; };
#pragma unroll
          for (int rt = 0; rt < SET; ++rt) {
            const int g = i * PARTS + p;
            const float sc = number<S>(pick(after(scale.v[r0 + rt][g / 2]), g));
            const float bs = BASES ? number<S>(pick(after(base.v[r0 + rt][g / 2]), g)) : 0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              y[r0 + rt][r] = fmaf(sc, part[rt][p][r], y[r0 + rt][r]);
              if constexpr (BASES) y[r0 + rt][r] = fmaf(bs, sum[p][r], y[r0 + rt][r]);
            }
          }
        }
      }
    });
    col = then;
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int r = 0; r < 4; ++r) s_y[wave][16 * rt + n][4 * c + r] = y[rt][r];
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
  if (a.rows >= kTwoTiles)
    return enqueue(gemv4_kernel<T, S, GROUP, BASES, 2, 4>, dim3((a.rows + 31) / 32), dim3(256), s, a);
  return enqueue(gemv4_kernel<T, S, GROUP, BASES, 1, 8>, dim3((a.rows + 15) / 16), dim3(512), s, a);
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
  if (!aligned(codes_dev, 16) || !aligned(x_dev, 16) || !aligned(scales_dev, 4) || !aligned(bases_dev, 4) ||
      !aligned(y_dev, 4))
    return HL_EINVAL;
  if (cols >= (1ull << 24) || rows >= (1ull << 31) || !grid_fits((rows + 15) / 16, 1024)) return HL_EUNSUPPORTED;
  Gemv4Args a = {};
  a.codes = codes_dev, a.scales = static_cast<const uint16_t*>(scales_dev);
  a.bases = static_cast<const uint16_t*>(bases_dev), a.x = static_cast<const uint16_t*>(x_dev), a.y = y_dev;
  a.rows = (uint32_t)rows, a.cols = (uint32_t)cols, a.batch = batch, a.groups = (uint32_t)(cols / group);
  const hipStream_t s = (hipStream_t)stream;
  if (x_dtype == HL_BF16)
    return scale_dtype == HL_BF16 ? run_group<__bf16, __bf16>(a, group, s) : run_group<__bf16, _Float16>(a, group, s);
  return scale_dtype == HL_BF16 ? run_group<_Float16, __bf16>(a, group, s) : run_group<_Float16, _Float16>(a, group, s);
}
