// Rows of a cache in 4 bits: written from new tokens' keys and values
// (hl_cache_write4) and read back (hl_cache_read4).
//
// 32 columns from lo to hi get base = (7 lo + 8 hi) / 15 and scale = the larger of
// (hi - base) / 7 and (base - lo) / 8, each rounded to bf16, and a column the code
// of the whole number in -8 .. 7 nearest to (x - base) / scale, ties to even. Which
// is nearest is found in float32, and again in float64 within 2^-10 of a tie, where
// the 2^-18 that float32 may be off could decide.
#include <algorithm>
#include <type_traits>

#include "cache4.h"
#include "gpu_host.h"

namespace hl {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kRowThreads = 256;
constexpr uint64_t kMostRows = 0xFFFFFF00u;  // of a call: a block's count in 32 bits

// Whole quotients of 32-bit numbers by d, by a product and two shifts (Granlund and
// Montgomery 1994, figure 4.1).
struct Divider {
  uint32_t d, factor, shift0, shift1;
  static Divider by(uint32_t d) {
    uint32_t bits = 0;
    while ((1ull << bits) < d) ++bits;
    return {d, (uint32_t)((((1ull << bits) - d) << 32) / d + 1), std::min(bits, 1u), bits ? bits - 1 : 0};
  }
  __device__ uint32_t operator()(uint32_t n) const {
    const uint32_t t = __umulhi(factor, n);
    return (t + ((n - t) >> shift0)) >> shift1;
  }
};

// Sequence, token of it and key head of a row.
struct RowPlace {
  uint32_t b, t, head;
  __device__ RowPlace(uint32_t row, Divider heads, Divider tokens) {
    const uint32_t token = heads(row);
    head = row - token * heads.d, b = tokens(token), t = token - b * tokens.d;
  }
};

struct WriteArgs {
  const uint16_t* from[2];  // keys, values
  uint8_t* to[2];
  uint64_t from_seq[2], from_token[2], from_head[2];  // in 16-bit elements
  uint64_t to_seq[2], to_token[2], to_head[2];        // in bytes
  const int32_t* lens;
  Divider tokens, heads;
  uint32_t capacity, rows;
};

// The greater (lesser) of x over the four lanes of a quad.
template <class F>
__device__ inline float over_quad(float x, F f) {
  const auto other = [](float v, auto ctrl) {
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, decltype(ctrl)::value, 0xF, 0xF, true));
  };
  x = f(x, other(x, std::integral_constant<int, 0xB1>()));  // lanes 1 0 3 2
  return f(x, other(x, std::integral_constant<int, 0x4E>()));  // lanes 2 3 0 1
}

// inverse: 1 / scale. (x - base) * inverse is off by 2^-18 where it is in range; where
// a tiny scale makes it infinite or NaN, its distance to a tie is a NaN.
__device__ inline uint32_t code4(float x, float base, float scale, float inverse) {
  const float q = (x - base) * inverse, r = rintf(q);
  float n = r;
  if (!(fabsf(fabsf(q - r) - 0.5f) > 0x1p-10f)) n = (float)rint(((double)x - (double)base) / (double)scale);
  return (uint32_t)(fminf(fmaxf(n, -8.0f), 7.0f) + 8.0f);
}

// Four lanes a group of 32 columns, 8 columns each; the rows are put together in
// LDS and stored in 16-byte pieces. 16384 tokens of 8 key heads of 128 columns, keys
// and values, 88 MB: 30 us, 0.57 of a copy's rate, bound by the vector instructions
// (some 40 a column pair; 43 us with a division each column and 64-bit quotients for
// the places).
template <class T, uint32_t G>
__global__ void __launch_bounds__(kRowThreads) write4_kernel(WriteArgs a) {
  constexpr uint32_t LANES = 4 * G, ROWS = kRowThreads / LANES, BYTES = row4_bytes(G);
  __shared__ __attribute__((aligned(16))) uint8_t s_row[ROWS * BYTES];
  const uint32_t set = blockIdx.y, lane = threadIdx.x % LANES, nth = threadIdx.x / LANES;
  const uint32_t first = blockIdx.x * ROWS;
  if (nth < ROWS) {
    const RowPlace r(min(first + nth, a.rows - 1), a.heads, a.tokens);
    const uint32_t g = lane / 4, c = lane % 4;
    const uint16_t* p = a.from[set] + r.b * a.from_seq[set] + r.t * a.from_token[set] + r.head * a.from_head[set] + 8 * lane;
    typedef T T8 __attribute__((ext_vector_type(8)));
    const T8 x = *reinterpret_cast<const T8*>(p);
    float lo = (float)x[0], hi = lo, odd = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) lo = fminf(lo, (float)x[i]), hi = fmaxf(hi, (float)x[i]), odd += (float)x[i] * 0.0f;
    lo = over_quad(lo, [](float u, float v) { return fminf(u, v); });
    hi = over_quad(hi, [](float u, float v) { return fmaxf(u, v); });
    odd = over_quad(odd, [](float u, float v) { return u + v; });
    const float base = (float)(__bf16)((7.0f * lo + 8.0f * hi) / 15.0f);
    const float scale = (float)(__bf16)fmaxf((hi - base) / 7.0f, (base - lo) / 8.0f);
    const bool good = odd == 0.0f && base - base == 0.0f && scale - scale == 0.0f;
    const float inverse = 1.0f / scale;
    uint8_t* to = s_row + nth * BYTES;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      uint32_t low = 8, high = 8;
      if (good && scale > 0.0f) {
        low = code4((float)x[2 * j], base, scale, inverse);
        high = code4((float)x[2 * j + 1], base, scale, inverse);
      }
      to[(4 * c + j) * G + g] = (uint8_t)(low | high << 4);
    }
    if (c == 0) {
      const uint32_t s = __builtin_bit_cast(uint32_t, scale) >> 16, z = __builtin_bit_cast(uint32_t, base) & 0xFFFF0000u;
      reinterpret_cast<uint32_t*>(to + 16 * G)[g] = good ? s | z : 0x7FC07FC0u;
    }
    for (uint32_t i = 20 * G + lane; i < BYTES; i += LANES) to[i] = 0;
  }
  __syncthreads();
  for (uint32_t x = threadIdx.x; x < ROWS * (BYTES / 16); x += kRowThreads) {
    const uint32_t row = first + x / (BYTES / 16);
    if (row >= a.rows) continue;
    const RowPlace r(row, a.heads, a.tokens);
    const int64_t slot = a.lens ? (int64_t)a.lens[r.b] - (int64_t)a.tokens.d + (int64_t)r.t : (int64_t)r.t;
    if (slot < 0 || slot >= (int64_t)a.capacity) continue;
    uint8_t* to = a.to[set] + r.b * a.to_seq[set] + (uint64_t)slot * a.to_token[set] + r.head * a.to_head[set];
    *reinterpret_cast<u32x4*>(to + x % (BYTES / 16) * 16) = *reinterpret_cast<const u32x4*>(s_row + x * 16);
  }
}

struct ReadArgs {
  const uint8_t* from;
  void* out;
  uint64_t seq, token, head;  // of the rows, in bytes
  Divider tokens, heads;
  uint32_t rows;
};

// Four lanes a group, 8 columns each. Bound by HBM: 16384 tokens of 8 key heads of 128 columns, 44 MB, 9 us.
template <class T, uint32_t G>
__global__ void __launch_bounds__(kRowThreads) read4_kernel(ReadArgs a) {
  constexpr uint32_t LANES = 4 * G, ROWS = kRowThreads / LANES;
  const uint32_t lane = threadIdx.x % LANES, nth = threadIdx.x / LANES;
  const uint32_t row = blockIdx.x * ROWS + nth;
  if (nth >= ROWS || row >= a.rows) return;
  const RowPlace r(row, a.heads, a.tokens);
  const uint8_t* p = a.from + r.b * a.seq + r.t * a.token + r.head * a.head;
  const uint32_t g = lane / 4, c = lane % 4;
  const uint32_t pair = reinterpret_cast<const uint32_t*>(p + 16 * G)[g];
  const float scale = __builtin_bit_cast(float, pair << 16), base = __builtin_bit_cast(float, pair & 0xFFFF0000u);
  typedef T T8 __attribute__((ext_vector_type(8)));
  T8 x;
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    const uint32_t codes = p[(4 * c + j) * G + g];
    x[2 * j] = (T)fmaf(scale, (float)(int)(codes & 15) - 8.0f, base);
    x[2 * j + 1] = (T)fmaf(scale, (float)(int)(codes >> 4) - 8.0f, base);
  }
  *reinterpret_cast<T8*>(static_cast<T*>(a.out) + (uint64_t)row * (32 * G) + 8 * lane) = x;
}

template <class F>
static hl_status with_groups(uint32_t groups, F f) {
  switch (groups) {
    case 1: return f(std::integral_constant<uint32_t, 1>());
    case 2: return f(std::integral_constant<uint32_t, 2>());
    case 3: return f(std::integral_constant<uint32_t, 3>());
    case 4: return f(std::integral_constant<uint32_t, 4>());
    case 5: return f(std::integral_constant<uint32_t, 5>());
    case 6: return f(std::integral_constant<uint32_t, 6>());
    case 7: return f(std::integral_constant<uint32_t, 7>());
    default: return f(std::integral_constant<uint32_t, 8>());
  }
}

}  // namespace hl

using namespace hl;

static hl_status check_rows(uint64_t batch, uint64_t tokens, uint64_t heads, uint32_t dim) {
  if (batch == 0 || tokens == 0 || heads == 0 || dim == 0 || dim % 32) return HL_EINVAL;
  if (dim > HL_ATTENTION_MAX_DIM || batch > 65535 || heads > 65535 || tokens >= (1ull << 30)) return HL_EUNSUPPORTED;
  const uint64_t rows = kRowThreads / (dim / 8);  // of a block
  if (batch * tokens * heads > kMostRows) return HL_EUNSUPPORTED;
  return grid_fits((batch * tokens * heads + rows - 1) / rows, kRowThreads) ? HL_OK : HL_EUNSUPPORTED;
}

static hl_status check_strides(const hl_kv* s) {
  if (!s || s->tokens == 0 || !s->k_dev || !s->v_dev || !aligned(s->k_dev, 16) || !aligned(s->v_dev, 16))
    return HL_EINVAL;
  for (uint64_t x : {s->k_token, s->v_token, s->k_head, s->v_head, s->k_seq, s->v_seq}) {
    if (x % 8) return HL_EINVAL;
    if (x >= (1ull << 40)) return HL_EUNSUPPORTED;
  }
  return HL_OK;
}

extern "C" size_t hl_cache4_row_bytes(uint32_t dim) {
  return dim && dim % 32 == 0 && dim <= HL_ATTENTION_MAX_DIM ? row4_bytes(dim / 32) : 0;
}

extern "C" hl_status hl_cache_write4(const hl_kv* from, hl_dtype dtype, const hl_kv* cache, uint32_t batch,
                                     uint32_t kv_heads, uint32_t dim, const int32_t* lens_dev, void* stream) {
  hl_status st = check_strides(from);
  if (st == HL_OK) st = check_strides(cache);
  if (st == HL_OK) st = check_rows(batch, from->tokens, kv_heads, dim);
  if (st != HL_OK) return st;
  if ((dtype != HL_BF16 && dtype != HL_F16) || !aligned(lens_dev, 4)) return HL_EINVAL;
  if (cache->tokens >= (1ull << 30)) return HL_EUNSUPPORTED;
  WriteArgs a = {};
  a.from[0] = static_cast<const uint16_t*>(from->k_dev), a.from[1] = static_cast<const uint16_t*>(from->v_dev);
  a.to[0] = static_cast<uint8_t*>(const_cast<void*>(cache->k_dev));
  a.to[1] = static_cast<uint8_t*>(const_cast<void*>(cache->v_dev));
  a.from_seq[0] = from->k_seq, a.from_token[0] = from->k_token, a.from_head[0] = from->k_head;
  a.from_seq[1] = from->v_seq, a.from_token[1] = from->v_token, a.from_head[1] = from->v_head;
  a.to_seq[0] = 2 * cache->k_seq, a.to_token[0] = 2 * cache->k_token, a.to_head[0] = 2 * cache->k_head;
  a.to_seq[1] = 2 * cache->v_seq, a.to_token[1] = 2 * cache->v_token, a.to_head[1] = 2 * cache->v_head;
  a.lens = lens_dev, a.tokens = Divider::by((uint32_t)from->tokens), a.heads = Divider::by(kv_heads);
  a.capacity = (uint32_t)cache->tokens, a.rows = (uint32_t)(batch * from->tokens * kv_heads);
  return with_groups(dim / 32, [&](auto g) {
    constexpr uint32_t G = decltype(g)::value, rows = kRowThreads / (4 * G);
    const dim3 grid((uint32_t)(((uint64_t)a.rows + rows - 1) / rows), 2), block(kRowThreads);
    return dtype == HL_BF16 ? enqueue(write4_kernel<__bf16, G>, grid, block, (hipStream_t)stream, a)
                            : enqueue(write4_kernel<_Float16, G>, grid, block, (hipStream_t)stream, a);
  });
}

extern "C" hl_status hl_cache_read4(const void* rows_dev, uint64_t seq_stride, uint64_t token_stride,
                                    uint64_t head_stride, uint32_t batch, uint64_t tokens, uint32_t heads,
                                    uint32_t dim, void* out_dev, hl_dtype dtype, void* stream) {
  if (!rows_dev || !out_dev || !aligned(rows_dev, 16) || !aligned(out_dev, 16)) return HL_EINVAL;
  if (dtype != HL_F32 && dtype != HL_BF16 && dtype != HL_F16) return HL_EINVAL;
  for (uint64_t x : {seq_stride, token_stride, head_stride}) {
    if (x % 16) return HL_EINVAL;
    if (x >= (1ull << 41)) return HL_EUNSUPPORTED;
  }
  const hl_status st = check_rows(batch, tokens, heads, dim);
  if (st != HL_OK) return st;
  ReadArgs a = {};
  a.from = static_cast<const uint8_t*>(rows_dev), a.out = out_dev;
  a.seq = seq_stride, a.token = token_stride, a.head = head_stride;
  a.tokens = Divider::by((uint32_t)tokens), a.heads = Divider::by(heads), a.rows = (uint32_t)(batch * tokens * heads);
  return with_groups(dim / 32, [&](auto g) {
    constexpr uint32_t G = decltype(g)::value, rows = kRowThreads / (4 * G);
    const dim3 grid((uint32_t)(((uint64_t)a.rows + rows - 1) / rows)), block(kRowThreads);
    return dtype == HL_F32    ? enqueue(read4_kernel<float, G>, grid, block, (hipStream_t)stream, a)
           : dtype == HL_BF16 ? enqueue(read4_kernel<__bf16, G>, grid, block, (hipStream_t)stream, a)
                              : enqueue(read4_kernel<_Float16, G>, grid, block, (hipStream_t)stream, a);
  });
}
