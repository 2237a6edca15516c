// Attention of a batch over one prefix that all its sequences share and over
// each sequence's own cache (hl_prefix_attention).
//
//   o = sum_j p_j v_j,  p_j = exp(s_j - m) / sum_j exp(s_j - m),  s_j = scale q.k_j
//
// Work. A "row" is one query vector (sequence, new token, head). The rows of
// one key head that see the same keys form an item: over the prefix, the rows
// of the whole batch (so the prefix is read once for all of them), over an own
// cache, the rows of its sequence; up to 128 rows an item, more items beyond.
// Every item's keys are cut into units of 128, all units stand in one line
// (the prefix's items, then the sequences'), and each block takes an equal
// stretch of the line, whatever the lengths are. It walks an item's keys with
// the running maximum and sum of the softmax and leaves (maximum, sum,
// unnormalised output) of its part in the workspace; the join kernel adds the
// parts of each row. Lengths are read on the device; nothing depends on the
// order in which blocks run, and there are no atomics.
//
// Inside a block a wave works alone: it loads 32 keys and their values from
// memory to registers, one step ahead, and no LDS or barrier stands in its
// loop. The matrix instruction takes K as its left operand and Q as its right,
// so a lane ends up with scores of one query (lane % 16), which is also what
// the second product needs of P as its right operand: the keys are only
// numbered differently in the two products, and P never leaves its lane. The
// values are loaded as rows (lane % 16 owns 8 neighbouring columns of 8 keys)
// and turned in registers, one byte permutation for two elements; the columns
// of one lane go to 8 different instructions, so that turning needs no other
// lane's data.
#include <algorithm>
#include <type_traits>

#include "gpu_host.h"

namespace hl {

constexpr uint32_t kUnit = 128;        // keys of a unit
constexpr uint32_t kWaves = 4;         // of a block
constexpr uint32_t kStep = 32;         // keys of a wave's step
constexpr float kSlack = 8.0f;         // powers of two that a score may pass the maximum kept for it by
constexpr float kLog2e = 1.44269504088896341f;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// One set of keys and values: strides in elements.
struct Kv {
  const uint16_t *k, *v;
  uint64_t k_seq, k_head, v_seq, v_head;
  uint32_t k_token, v_token;
  uint32_t tokens;  // the prefix's length, or an own cache's capacity
};

// Rows of an item: `tile` = 16 * R * across, R 16-row tiles a wave, `across`
// waves side by side (the other kWaves / across take other keys).
struct Tiling {
  uint32_t r, across, tiles;  // tiles: items of one head (and sequence)
  __host__ __device__ uint32_t rows() const { return 16 * r * across; }
};

struct AttentionArgs {
  Kv prefix, own;
  const uint16_t* q;
  const int32_t* lens;
  uint16_t* out;
  float* lse;
  const float* weight_in;
  float* weight_out;
  float *part_o, *part_ml, *row_ml, *scores;  // workspace
  uint32_t batch, queries, heads, kv_heads, dim, share;  // share: query heads of a key head
  uint32_t blocks, part_rows, score_stride;
  Tiling tp, to;
  float scale2;  // scale * log2(e): scores are kept in powers of two
};

__device__ inline uint32_t own_length(const AttentionArgs& a, uint32_t b) {
  const int32_t n = a.lens[b];
  return n <= 0 ? 0 : min((uint32_t)n, a.own.tokens);
}

__host__ __device__ inline uint32_t units_of(uint32_t keys) { return (keys + kUnit - 1) / kUnit; }

// Where sequence b's units begin in the line, counted from the own caches'
// first, and how many units one of its items has.
struct OwnPlace {
  uint32_t b, begin, each;
};

// Sum of all sequences' units before b (b = batch: of all). Whole wave.
__device__ inline uint32_t own_units_before(const AttentionArgs& a, uint32_t b) {
  uint32_t sum = 0;
  const uint32_t items = a.kv_heads * a.to.tiles;
  for (uint32_t i = threadIdx.x % 64; i < b; i += 64) sum += items * units_of(own_length(a, i));
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  return __builtin_amdgcn_readfirstlane(sum);
}

// The sequence that unit u (counted as above) belongs to. Whole wave.
__device__ inline OwnPlace own_place(const AttentionArgs& a, uint32_t u) {
  const uint32_t lane = threadIdx.x % 64, items = a.kv_heads * a.to.tiles;
  uint32_t base = 0;
  for (uint32_t b0 = 0; b0 < a.batch; b0 += 64) {
    const uint32_t each = b0 + lane < a.batch ? units_of(own_length(a, b0 + lane)) : 0;
    uint32_t end = items * each;
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(end, d);
      if (lane >= (uint32_t)d) end += o;
    }
    const uint64_t past = __ballot(base + end > u);
    if (past) {
      const int l = __builtin_ctzll(past);
      const uint32_t e = __builtin_amdgcn_readlane(each, l), f = __builtin_amdgcn_readlane(end, l);
      return {b0 + (uint32_t)l, base + f - items * e, e};
    }
    base += __builtin_amdgcn_readlane(end, 63);
  }
  return {a.batch, base, 1};  // past the line's end: no caller asks
}

// The block that unit u of `total` is in when `blocks` share them, at most one
// block a unit: block k has floor(k*total/blocks) up to
// floor((k+1)*total/blocks), never none.
__device__ inline uint32_t block_of(uint32_t u, uint32_t total, uint32_t blocks) {
  return (uint32_t)((((uint64_t)u + 1) * blocks - 1) / total);
}

template <class T>
__device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (std::is_same<T, __bf16>::value)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
}

// Ends a row of matrix instructions: nothing is moved across it, and the
// instructions after it may write the operands of those before. On gfx950 a
// product has come out wrong now and then when the instruction right after it
// wrote one of its operand registers; the compiler places no wait states
// there, and five are enough.
__device__ inline void products_end() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 4");
  __builtin_amdgcn_sched_barrier(0);
}

// Two float32 to two 16-bit values, each rounded to nearest.
template <class T>
__device__ inline uint32_t pack(float lo, float hi) {
  typedef T pair __attribute__((ext_vector_type(2)));
  const pair p = {(T)lo, (T)hi};
  return __builtin_bit_cast(uint32_t, p);
}

template <class T>
__device__ inline float widen(uint32_t h) {
  if constexpr (std::is_same<T, __bf16>::value)
    return __builtin_bit_cast(float, h << 16);
  else
    return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
}

// Whether a 16-bit value is an infinity or NaN.
template <class T>
__device__ inline bool beyond(uint32_t h) {
  constexpr uint32_t e = std::is_same<T, __bf16>::value ? 0x7F80 : 0x7C00;
  return (h & e) == e;
}

// What one wave needs of an item.
struct Item {
  const uint16_t *k, *v, *q;    // at the sequence and key head; q at the item's first token and head
  float* scores;                // of the item's rows, or null
  uint32_t k_token, v_token;
  uint32_t keys;                // of the set
  uint32_t back;                // keys that the first token does not see (0: no order among the keys)
  bool ordered;                 // token i sees keys - back + i keys
  uint32_t row0, rows;          // first row of the item's tile, rows of the whole head (and sequence)
};

// D: columns held (64, 128 or 256); the head's own count may be less (FULL: it
// is D). VE: neighbouring value columns of a lane, in HALVES groups of 16*VE.
template <int D>
struct Shape {
  static constexpr int VE = D == 64 ? 4 : 8;
  static constexpr int HALVES = D == 256 ? 2 : 1;
  static constexpr int KS = D / 32;         // steps of the first product
  static constexpr int TILES = D / 16;      // of the second product's output
};

template <int D>
struct Tile {
  u32x4 k[2][Shape<D>::KS];
  uint32_t v[8][Shape<D>::HALVES][Shape<D>::VE / 2];
};

// Key of value row e in lane group c, counted from the step's first: the order
// in which the first product leaves its scores in a lane.
__device__ inline uint32_t key_of(uint32_t c, int e) { return (e < 4 ? 0 : 12) + 4 * c + e; }

// Loads keys key .. key+31 of `it`; past its end, its last key again.
template <int D, bool FULL>
__device__ inline void load_tile(Tile<D>& t, const Item& it, uint32_t dim, uint32_t key) {
  using S = Shape<D>;
  const uint32_t lane = threadIdx.x % 64, n = lane % 16, c = lane / 16;
  const uint16_t* kp = it.k + (uint64_t)key * it.k_token;
  const uint16_t* vp = it.v + (uint64_t)key * it.v_token;
  uint32_t ko[2], vo[8], left = it.keys - 1 - key;
  if (left >= kStep - 1) {
    ko[0] = n * it.k_token, ko[1] = ko[0] + 16 * it.k_token;
    vo[0] = 4 * c * it.v_token;
#pragma unroll
    for (int e = 1; e < 8; ++e) vo[e] = vo[0] + (key_of(0, e)) * it.v_token;
  } else {
    ko[0] = min(n, left) * it.k_token, ko[1] = min(16 + n, left) * it.k_token;
#pragma unroll
    for (int e = 0; e < 8; ++e) vo[e] = min(key_of(c, e), left) * it.v_token;
  }
#pragma unroll
  for (int s = 0; s < S::KS; ++s) {
    const uint32_t d = c * 8 + s * 32;
    const bool in = FULL || d < dim;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(kp + (ko[h] + (in ? d : 0)));
      t.k[h][s] = in ? w : u32x4{0, 0, 0, 0};
    }
  }
#pragma unroll
  for (int h = 0; h < S::HALVES; ++h) {
    uint32_t d = n * S::VE + h * 128;
    if (!FULL && d >= dim) d = 0;  // columns that no output is stored from
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (S::VE == 8) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(vp + (vo[e] + d));
        for (int j = 0; j < 4; ++j) t.v[e][h][j] = w[j];
      } else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(vp + (vo[e] + d));
        for (int j = 0; j < 2; ++j) t.v[e][h][j] = w[j];
      }
    }
  }
}

// Running state of R 16-row tiles of a wave: lane's query is lane % 16 of each.
template <int D, int R>
struct State {
  u32x4 q[R][Shape<D>::KS];
  f32x4 o[R][Shape<D>::TILES];
  float m[R], l[R];    // maximum (0 while there is none), this lane's part of the sum
  bool some[R];        // whether m is a score's
  uint32_t seen[R];    // keys that the query sees
};

// Contributions of values that are infinite or NaN, which the matrix product
// has taken as 0: a query that does not see their key must not meet them.
template <class T, int D, int R>
__device__ inline void add_beyond(State<D, R>& st, const float (&p)[R][2][4], const Item& it,
                                                     uint32_t dim, uint32_t key) {
  using S = Shape<D>;
  const uint32_t lane = threadIdx.x % 64, n = lane % 16, c = lane / 16;
  for (uint32_t j = 0; j < kStep && key + j < it.keys; ++j) {
    const uint16_t* row = it.v + (uint64_t)(key + j) * it.v_token;
#pragma unroll
    for (int rt = 0; rt < R; ++rt) {
      float w = 0.0f;
#pragma unroll
      for (uint32_t h = 0; h < 2; ++h)
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) w = h == j / 16 && r == j % 4 ? p[rt][h][r] : w;
      w = __shfl(w, (j % 16 / 4) * 16 + n);
      if (key + j >= st.seen[rt]) continue;
#pragma unroll
      for (int t = 0; t < S::TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint32_t d = t / S::VE * 128 + (4 * c + r) * S::VE + t % S::VE;
          if (d >= dim) continue;
          const uint32_t b = row[d];
          if (beyond<T>(b)) st.o[rt][t][r] += w * widen<T>(b);
        }
    }
  }
}

// One step: scores of 32 keys, their weights, and the weighted values.
// `all`: keys that every query of the wave sees; `most`: that some query sees.
template <class T, int D, int R>
__device__ inline void step(State<D, R>& st, Tile<D>& t, const AttentionArgs& a, const Item& it, uint32_t key,
                            uint32_t all, uint32_t most, uint32_t wave_row) {
  using S = Shape<D>;
  const uint32_t lane = threadIdx.x % 64, n = lane % 16, c = lane / 16;
  const bool edge = key + kStep > all;
  f32x4 s[R][2];
  float p[R][2][4];
  u32x4 w[R];
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int rt = 0; rt < R; ++rt)
#pragma unroll
    for (int h = 0; h < 2; ++h) s[rt][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < S::KS; ++i)
#pragma unroll
    for (int rt = 0; rt < R; ++rt)
#pragma unroll
      for (int h = 0; h < 2; ++h) s[rt][h] = mfma<T>(t.k[h][i], st.q[rt][i], s[rt][h]);
  products_end();
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    float top = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) p[rt][h][r] = s[rt][h][r] * a.scale2;
    if (edge) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (key + 16 * h + 4 * c + r >= st.seen[rt]) p[rt][h][r] = -INFINITY;
    }
    if (it.scores) {
      const uint32_t row = wave_row + 16 * rt + n;
      if (row < it.rows) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<float4*>(it.scores + (uint64_t)row * a.score_stride + key + 16 * h + 4 * c) =
              make_float4(p[rt][h][0], p[rt][h][1], p[rt][h][2], p[rt][h][3]);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, p[rt][h][r]);
    // The maximum need not be the true one, only near it: the output is
    // scaled again when a score passes it by more than 2^8, so the weights
    // stay in the 16-bit types' range and most steps scale nothing.
    if (__any(top > (st.some[rt] ? st.m[rt] + kSlack : -INFINITY))) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const bool had = st.some[rt];
      const float was = st.m[rt];
      const float now = had ? fmaxf(was, top) : top;
      if (now != -INFINITY) {
        const float f = had ? __builtin_amdgcn_exp2f(was - now) : 0.0f;
        st.m[rt] = now, st.some[rt] = true;
        st.l[rt] *= f;
#pragma unroll
        for (int i = 0; i < S::TILES; ++i) st.o[rt][i] *= f;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[rt][h][r] = __builtin_amdgcn_exp2f(p[rt][h][r] - st.m[rt]);
        st.l[rt] += p[rt][h][r];
      }
    w[rt] = u32x4{pack<T>(p[rt][0][0], p[rt][0][1]), pack<T>(p[rt][0][2], p[rt][0][3]),
                  pack<T>(p[rt][1][0], p[rt][1][1]), pack<T>(p[rt][1][2], p[rt][1][3])};
  }
  if (edge) {
    // values that no query sees count 0, whatever they are; those that only
    // some see must be finite in the product
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool in = key + key_of(c, e) < most;
#pragma unroll
      for (int h = 0; h < S::HALVES; ++h)
#pragma unroll
        for (int j = 0; j < S::VE / 2; ++j) {
          uint32_t& d = t.v[e][h][j];
          if (!in) d = 0;
          if (it.ordered) {
            if (beyond<T>(d)) d &= 0xFFFF0000u, odd = true;
            if (beyond<T>(d >> 16)) d &= 0xFFFFu, odd = true;
          }
        }
    }
    if (it.ordered && __any(odd)) add_beyond<T, D, R>(st, p, it, a.dim, key);
  }
#pragma unroll
  for (int h = 0; h < S::HALVES; ++h) {
    u32x4 vt[S::VE];
#pragma unroll
    for (int i = 0; i < S::VE; ++i) {
      const uint32_t sel = i % 2 ? 0x07060302u : 0x05040100u;
#pragma unroll
      for (int e = 0; e < 4; ++e) vt[i][e] = __builtin_amdgcn_perm(t.v[2 * e + 1][h][i / 2], t.v[2 * e][h][i / 2], sel);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < S::VE; ++i)
#pragma unroll
      for (int rt = 0; rt < R; ++rt) st.o[rt][h * S::VE + i] = mfma<T>(vt[i], w[rt], st.o[rt][h * S::VE + i]);
    products_end();
  }
}

// A block's LDS: each wave's output rows, padded by 4 so that rows start in
// different banks, and their (maximum, sum).
template <int D, int R>
constexpr uint32_t lds_floats() {
  return kWaves * 16 * R * (D + 4) + kWaves * 16 * R * 2;
}

// Keys [k0, k1) of an item by one block; writes the part at `slot`.
template <class T, int D, bool FULL, int R>
__device__ inline void part(const AttentionArgs& a, const Item& it, const Tiling& tl, uint32_t k0, uint32_t k1,
                            uint32_t slot, float* lds) {
  using S = Shape<D>;
  const uint32_t lane = threadIdx.x % 64, n = lane % 16, c = lane / 16;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t across = tl.across, along = kWaves / across;
  const uint32_t wr = wave % across, kw = wave / across;
  const uint32_t wave_row = it.row0 + wr * 16 * R;
  State<D, R> st;
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    st.m[rt] = 0.0f, st.l[rt] = 0.0f, st.some[rt] = false;
#pragma unroll
    for (int i = 0; i < S::TILES; ++i) st.o[rt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t row = min(wave_row + 16 * rt + n, it.rows - 1), tok = row / a.share;
    st.seen[rt] = it.ordered ? (it.keys + tok > it.back ? it.keys + tok - it.back : 0) : it.keys;
    const uint16_t* q = it.q + ((uint64_t)tok * a.heads + row % a.share) * a.dim;
#pragma unroll
    for (int s = 0; s < S::KS; ++s) {
      const uint32_t d = c * 8 + s * 32;
      const bool in = FULL || d < a.dim;
      const u32x4 w = *reinterpret_cast<const u32x4*>(q + (in ? d : 0));
      st.q[rt][s] = in ? w : u32x4{0, 0, 0, 0};
    }
  }
  // keys seen by the wave's first and last row
  uint32_t all = it.keys, most = it.keys;
  if (it.ordered) {
    const uint32_t first = min(wave_row, it.rows - 1) / a.share, last = min(wave_row + 16 * R, it.rows) - 1;
    all = it.keys + first > it.back ? it.keys + first - it.back : 0;
    most = it.keys + last / a.share > it.back ? it.keys + last / a.share - it.back : 0;
  }
  const uint32_t end = wave_row < it.rows ? min(k1, most) : 0;
  uint32_t key = k0 + kStep * kw;
  const uint32_t stride = kStep * along;
  if (key < end) {
    Tile<D> t0, t1;
    load_tile<D, FULL>(t0, it, a.dim, key);
    while (true) {
      if constexpr (D == 256) {  // two steps' keys do not fit the registers
        step<T, D, R>(st, t0, a, it, key, all, most, wave_row);
        if ((key += stride) >= end) break;
        load_tile<D, FULL>(t0, it, a.dim, key);
        continue;
      }
      uint32_t next = key + stride;
      if (next < end) load_tile<D, FULL>(t1, it, a.dim, next);
      step<T, D, R>(st, t0, a, it, key, all, most, wave_row);
      if (next >= end) break;
      key = next, next += stride;
      if (next < end) load_tile<D, FULL>(t0, it, a.dim, next);
      step<T, D, R>(st, t1, a, it, key, all, most, wave_row);
      if (next >= end) break;
      key = next;
    }
  }
  // join the waves that had other keys of the same rows
  float* lds_ml = lds + kWaves * 16 * R * (D + 4);
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    float l = st.l[rt];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    const uint32_t row = wave * 16 * R + 16 * rt + n;
    if (c == 0) lds_ml[2 * row] = st.some[rt] || l != l ? st.m[rt] : -INFINITY, lds_ml[2 * row + 1] = l;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int h = 0; h < S::HALVES; ++h)
#pragma unroll
        for (int q = 0; q < S::VE; q += 4) {
          const int i = h * S::VE + q;
          *reinterpret_cast<float4*>(lds + (uint64_t)row * (D + 4) + h * 128 + (4 * c + r) * S::VE + q) =
              make_float4(st.o[rt][i][r], st.o[rt][i + 1][r], st.o[rt][i + 2][r], st.o[rt][i + 3][r]);
        }
  }
  __syncthreads();
  const uint32_t rows = min(tl.rows(), it.rows - it.row0);
  float* po = a.part_o + (uint64_t)slot * a.part_rows * D;
  float* pml = a.part_ml + (uint64_t)slot * a.part_rows * 2;
  for (uint32_t x = threadIdx.x; x < rows * (D / 4); x += kWaves * 64) {
    const uint32_t row = x / (D / 4), d = x % (D / 4) * 4;
    const uint32_t at = row / (16 * R) * 16 * R + row % (16 * R);  // of key wave 0
    float m = -INFINITY, l = 0.0f;
    for (uint32_t k = 0; k < along; ++k) m = fmaxf(m, lds_ml[2 * (at + k * across * 16 * R)]);
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t k = 0; k < along; ++k) {
      const uint32_t from = at + k * across * 16 * R;
      const float mk = lds_ml[2 * from];
      const float f = mk == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mk - m);
      const float4 v = *reinterpret_cast<const float4*>(lds + (uint64_t)from * (D + 4) + d);
      o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
      l += f * lds_ml[2 * from + 1];
    }
    *reinterpret_cast<float4*>(po + (uint64_t)row * D + d) = o;
    if (d == 0) pml[2 * row] = m, pml[2 * row + 1] = l;
  }
  __syncthreads();
}

// Blocks that stand next to each other in the line go to the same XCD, where
// the row tiles of one head find its keys in the L2 (blocks are dealt to the 8
// XCDs in turn).
__device__ inline uint32_t line_block(uint32_t blocks) {
  return blocks % 8 ? blockIdx.x : blockIdx.x % 8 * (blocks / 8) + blockIdx.x / 8;
}

template <class T, int D, bool FULL, int RMAX>
__global__ void __launch_bounds__(256, 1) parts_kernel(AttentionArgs a) {
  __shared__ __attribute__((aligned(16))) float lds[lds_floats<D, RMAX>()];
  const uint32_t up = units_of(a.prefix.tokens), prefix_units = a.kv_heads * a.tp.tiles * up;
  const uint32_t total = prefix_units + own_units_before(a, a.own.tokens ? a.batch : 0);
  const uint32_t blk = line_block(a.blocks), blocks = min(a.blocks, total);
  if (blk >= blocks) return;
  uint32_t u = (uint32_t)((uint64_t)blk * total / blocks);
  const uint32_t end = (uint32_t)(((uint64_t)blk + 1) * total / blocks);
  while (u < end) {
    Item it;
    uint32_t item, in, each, head;
    const bool shared = u < prefix_units;
    if (shared) {
      item = u / up, in = u % up, each = up, head = item / a.tp.tiles;
      it.k = a.prefix.k + head * a.prefix.k_head, it.v = a.prefix.v + head * a.prefix.v_head;
      it.k_token = a.prefix.k_token, it.v_token = a.prefix.v_token;
      it.q = a.q + (uint64_t)head * a.share * a.dim;
      it.keys = a.prefix.tokens, it.back = 0, it.ordered = false;
      it.row0 = item % a.tp.tiles * a.tp.rows(), it.rows = a.batch * a.queries * a.share;
      it.scores = nullptr;
    } else {
      const OwnPlace pl = own_place(a, u - prefix_units);
      const uint32_t x = u - prefix_units - pl.begin, y = x / pl.each;
      in = x % pl.each, each = pl.each, head = y / a.to.tiles;
      item = a.kv_heads * a.tp.tiles + pl.b * a.kv_heads * a.to.tiles + y;
      it.k = a.own.k + pl.b * a.own.k_seq + head * a.own.k_head;
      it.v = a.own.v + pl.b * a.own.v_seq + head * a.own.v_head;
      it.k_token = a.own.k_token, it.v_token = a.own.v_token;
      it.q = a.q + ((uint64_t)pl.b * a.queries * a.heads + (uint64_t)head * a.share) * a.dim;
      it.keys = own_length(a, pl.b), it.back = a.queries - 1, it.ordered = a.queries > 1;
      it.row0 = y % a.to.tiles * a.to.rows(), it.rows = a.queries * a.share;
      it.scores = a.scores
                      ? a.scores + ((uint64_t)pl.b * a.kv_heads + head) * it.rows * a.score_stride
                      : nullptr;
    }
    const uint32_t take = min(each - in, end - u);
    const Tiling& tl = shared ? a.tp : a.to;
    if (RMAX == 1 || tl.r == 1)
      part<T, D, FULL, 1>(a, it, tl, in * kUnit, (in + take) * kUnit, blk + item, lds);
    else
      part<T, D, FULL, RMAX>(a, it, tl, in * kUnit, (in + take) * kUnit, blk + item, lds);
    u += take;
  }
}

// Adds a row's parts, one wave a row: lane's columns are lane*D/64 ..
template <class T, int D>
__global__ void __launch_bounds__(256) join_kernel(AttentionArgs a) {
  constexpr int E = D / 64;
  const uint32_t lane = threadIdx.x % 64;
  const uint32_t row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64);
  if (row >= a.batch * a.queries * a.heads) return;
  const uint32_t tok = row / a.heads, hq = row % a.heads, b = tok / a.queries, head = hq / a.share, g = hq % a.share;
  const uint32_t up = units_of(a.prefix.tokens), prefix_units = a.kv_heads * a.tp.tiles * up;
  uint32_t own_each = 0, own_begin = 0, total = prefix_units;
  if (a.own.tokens) {
    own_each = units_of(own_length(a, b));
    own_begin = prefix_units + own_units_before(a, b);
    total += own_units_before(a, a.batch);
  }
  const uint32_t blocks = min(a.blocks, total);
  // the row's parts: over the prefix, then over its own keys
  uint32_t slot[2] = {0, 0}, at[2], count[2] = {0, 0};
  const uint32_t rp = tok * a.share + g, ro = tok % a.queries * a.share + g;
  at[0] = rp % a.tp.rows(), at[1] = ro % a.to.rows();
  if (up) {
    const uint32_t item = head * a.tp.tiles + rp / a.tp.rows(), u = item * up;
    const uint32_t first = block_of(u, total, blocks);
    slot[0] = first + item, count[0] = block_of(u + up - 1, total, blocks) - first + 1;
  }
  if (own_each) {
    const uint32_t y = head * a.to.tiles + ro / a.to.rows(), u = own_begin + y * own_each;
    const uint32_t first = block_of(u, total, blocks);
    slot[1] = first + a.kv_heads * a.tp.tiles + b * a.kv_heads * a.to.tiles + y;
    count[1] = block_of(u + own_each - 1, total, blocks) - first + 1;
  }
  const uint32_t parts = count[0] + count[1];
  auto place = [&](uint32_t i) {
    return i < count[0] ? (uint64_t)(slot[0] + i) * a.part_rows + at[0]
                        : (uint64_t)(slot[1] + i - count[0]) * a.part_rows + at[1];
  };
  float m = -INFINITY, l = 0.0f, o[E];
  for (int e = 0; e < E; ++e) o[e] = 0.0f;
  for (uint32_t i0 = 0; i0 < parts; i0 += 64) {
    const uint32_t some = min(64u, parts - i0);
    float mi = -INFINITY, li = 0.0f;
    if (lane < some) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + 2 * place(i0 + lane));
      mi = ml.x, li = ml.y;
    }
    float top = mi;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float now = fmaxf(m, top);
    const float f0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - now);
    const float fi = mi == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mi - now);
    float sum = fi * li;
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    l = l * f0 + sum, m = now;
    for (int e = 0; e < E; ++e) o[e] *= f0;
#pragma unroll 8
    for (uint32_t i = 0; i < some; ++i) {
      const float f = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(uint32_t, fi), i));
      const float* p = a.part_o + place(i0 + i) * D + lane * E;
      for (int e = 0; e < E; ++e) o[e] += f * p[e];
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (lane * E < a.dim) {
    uint16_t* q = a.out + (uint64_t)row * a.dim + lane * E;
    if constexpr (E == 1) {
      q[0] = (uint16_t)pack<T>(o[0] * inv, 0.0f);
    } else {
      for (int e = 0; e < E; e += 2) *reinterpret_cast<uint32_t*>(q + e) = pack<T>(o[e] * inv, o[e + 1] * inv);
    }
  }
  if (lane == 0) {
    if (a.lse) a.lse[row] = l == 0.0f ? -INFINITY : m / kLog2e + logf(l);
    if (a.row_ml) a.row_ml[2 * row] = l == 0.0f ? 0.0f : m, a.row_ml[2 * row + 1] = inv;
  }
}

// weight_out = weight_in + the weight that the call's rows gave each own key;
// a thread adds its key's rows in their order.
__global__ void __launch_bounds__(256) weights_kernel(AttentionArgs a) {
  const uint32_t head = blockIdx.y, b = blockIdx.z, key = blockIdx.x * 256 + threadIdx.x;
  if (key >= a.own.tokens) return;
  const uint64_t at = ((uint64_t)b * a.kv_heads + head) * a.own.tokens + key;
  float w = 0.0f;
  if (key < own_length(a, b)) {
    const uint32_t rows = a.queries * a.share;
    const float* s = a.scores + ((uint64_t)b * a.kv_heads + head) * rows * a.score_stride + key;
    const float* ml = a.row_ml + 2 * ((uint64_t)b * a.queries * a.heads + (uint64_t)head * a.share);
    // the scores that the mask hides (of the earlier of several tokens) are not there
    const uint32_t newer = own_length(a, b) - 1 - key;
    for (uint32_t i = newer < a.queries ? a.queries - 1 - newer : 0; i < a.queries; ++i)
      for (uint32_t g = 0; g < a.share; ++g) {
        const float* r = ml + 2 * ((uint64_t)i * a.heads + g);
        w += __builtin_amdgcn_exp2f(s[(uint64_t)(i * a.share + g) * a.score_stride] - r[0]) * r[1];
      }
  }
  a.weight_out[at] = a.weight_in ? a.weight_in[at] + w : w;
}

// ------------------------------------------------------------------- host

// Rows a wave and waves side by side for items of `rows` rows.
static Tiling tiling(uint64_t rows, uint32_t dim) {
  Tiling t;
  t.r = rows > 16 && dim <= 128 ? 2 : 1;
  t.across = rows <= 16 * t.r ? 1 : rows <= 32 * t.r ? 2 : 4;
  t.tiles = (uint32_t)((rows + t.rows() - 1) / t.rows());
  return t;
}

struct AttentionPlan {
  AttentionArgs a;
  uint64_t bytes, part_o, part_ml, row_ml, scores;  // of the workspace: its size and its parts' places
};

static hl_status check_kv(const hl_kv& s, uint64_t tokens, uint32_t dim, bool sequences) {
  if (tokens == 0) return HL_OK;
  if (!s.k_dev || !s.v_dev || !aligned(s.k_dev, 16) || !aligned(s.v_dev, 16)) return HL_EINVAL;
  const uint64_t strides[6] = {s.k_token, s.v_token, s.k_head, s.v_head, sequences ? s.k_seq : 0, sequences ? s.v_seq : 0};
  for (uint64_t x : strides) {
    if (x % 8) return HL_EINVAL;
    if (x >= (1ull << 40)) return HL_EUNSUPPORTED;
  }
  // a step's offsets (32 tokens and a row) stay within 32 bits
  if (s.k_token >= (1ull << 26) || s.v_token >= (1ull << 26)) return HL_EUNSUPPORTED;
  (void)dim;
  return HL_OK;
}

static Kv kv_of(const hl_kv& s) {
  Kv k = {};
  k.tokens = (uint32_t)s.tokens;
  if (s.tokens == 0) return k;
  k.k = static_cast<const uint16_t*>(s.k_dev), k.v = static_cast<const uint16_t*>(s.v_dev);
  k.k_seq = s.k_seq, k.k_head = s.k_head, k.v_seq = s.v_seq, k.v_head = s.v_head;
  k.k_token = (uint32_t)s.k_token, k.v_token = (uint32_t)s.v_token;
  return k;
}

static hl_status attention_plan(const hl_attention* h, bool weights, AttentionPlan* pl) {
  if (!h || h->batch == 0 || h->queries == 0 || h->heads == 0 || h->kv_heads == 0 || h->heads % h->kv_heads ||
      h->dim == 0 || h->dim % 8 || !(h->scale == h->scale) || (h->dtype != HL_BF16 && h->dtype != HL_F16))
    return HL_EINVAL;
  if (weights && h->own.tokens == 0) return HL_EINVAL;
  hl_status st = check_kv(h->prefix, h->prefix.tokens, h->dim, false);
  if (st == HL_OK) st = check_kv(h->own, h->own.tokens, h->dim, true);
  if (st != HL_OK) return st;
  const uint64_t rows = (uint64_t)h->batch * h->queries * h->heads;
  if (h->dim > HL_ATTENTION_MAX_DIM || h->prefix.tokens >= (1ull << 30) || h->own.tokens >= (1ull << 30) ||
      h->queries >= (1u << 24) || h->batch > 65535 || h->kv_heads > 65535 || rows >= (1ull << 28))
    return HL_EUNSUPPORTED;
  AttentionArgs& a = pl->a;
  a = {};
  a.prefix = kv_of(h->prefix), a.own = kv_of(h->own);
  a.batch = h->batch, a.queries = h->queries, a.heads = h->heads, a.kv_heads = h->kv_heads, a.dim = h->dim;
  a.share = h->heads / h->kv_heads;
  a.scale2 = h->scale * kLog2e;
  a.tp = tiling((uint64_t)h->batch * h->queries * a.share, h->dim);
  a.to = tiling((uint64_t)h->queries * a.share, h->dim);
  const uint64_t items = (uint64_t)h->kv_heads * (a.tp.tiles + (uint64_t)h->batch * a.to.tiles);
  const uint64_t units = (uint64_t)h->kv_heads * ((uint64_t)a.tp.tiles * units_of(a.prefix.tokens) +
                                                  (uint64_t)h->batch * a.to.tiles * units_of(a.own.tokens));
  if (units >= (1ull << 31)) return HL_EUNSUPPORTED;
  a.blocks = (uint32_t)std::max<uint64_t>(1, std::min<uint64_t>((uint64_t)device_cus(), units));
  a.part_rows = std::max(a.tp.rows(), a.to.rows());
  const uint32_t held = h->dim <= 64 ? 64 : h->dim <= 128 ? 128 : 256;
  const uint64_t slots = a.blocks + items;
  uint64_t n = 0;
  auto take = [&](uint64_t floats) {
    const uint64_t at = n;
    n += (floats * 4 + 255) / 256 * 256;
    return at;
  };
  pl->part_o = take(slots * a.part_rows * held);
  pl->part_ml = take(slots * a.part_rows * 2);
  a.score_stride = (a.own.tokens + kStep - 1) / kStep * kStep;
  pl->row_ml = weights ? take(rows * 2) : 0;
  pl->scores = weights ? take((uint64_t)h->batch * h->heads * h->queries * a.score_stride) : 0;
  pl->bytes = n;
  return HL_OK;
}

template <class T, int D, bool FULL, int RMAX>
static hl_status run(const AttentionArgs& a, hipStream_t s) {
  hl_status st = enqueue(parts_kernel<T, D, FULL, RMAX>, dim3(a.blocks), dim3(kWaves * 64), s, a);
  if (st != HL_OK) return st;
  const uint32_t rows = a.batch * a.queries * a.heads;
  st = enqueue(join_kernel<T, D>, dim3((rows + 3) / 4), dim3(256), s, a);
  if (st != HL_OK || !a.scores) return st;
  return enqueue(weights_kernel, dim3((a.own.tokens + 255) / 256, a.kv_heads, a.batch), dim3(256), s, a);
}

template <class T, int D, bool FULL>
static hl_status run_rows(const AttentionArgs& a, hipStream_t s) {
  if constexpr (D <= 128) {
    if (a.tp.r > 1 || a.to.r > 1) return run<T, D, FULL, 2>(a, s);
  }
  return run<T, D, FULL, 1>(a, s);
}

template <class T>
static hl_status run_type(const AttentionArgs& a, hipStream_t s) {
  if (a.dim == 64) return run_rows<T, 64, true>(a, s);
  if (a.dim < 64) return run_rows<T, 64, false>(a, s);
  if (a.dim == 128) return run_rows<T, 128, true>(a, s);
  if (a.dim < 128) return run_rows<T, 128, false>(a, s);
  if (a.dim == 256) return run_rows<T, 256, true>(a, s);
  return run_rows<T, 256, false>(a, s);
}

}  // namespace hl

using namespace hl;

extern "C" size_t hl_attention_workspace_bytes(const hl_attention* attention, int with_weights) {
  AttentionPlan pl;
  return attention_plan(attention, with_weights != 0, &pl) == HL_OK ? pl.bytes : 0;
}

extern "C" hl_status hl_prefix_attention(const hl_attention* attention, const void* q_dev, const int32_t* lens_dev,
                                         void* out_dev, float* lse_dev, const float* weight_in_dev,
                                         float* weight_out_dev, void* workspace_dev, size_t workspace_bytes,
                                         void* stream) {
  if (!attention || !q_dev || !out_dev || !workspace_dev || (weight_in_dev && !weight_out_dev)) return HL_EINVAL;
  if (attention->own.tokens && !lens_dev) return HL_EINVAL;
  if (!aligned(q_dev, 16) || !aligned(out_dev, 16) || !aligned(workspace_dev, 16) || !aligned(lens_dev, 4) ||
      !aligned(lse_dev, 4) || !aligned(weight_in_dev, 4) || !aligned(weight_out_dev, 4))
    return HL_EINVAL;
  AttentionPlan pl;
  const hl_status st = attention_plan(attention, weight_out_dev != nullptr, &pl);
  if (st != HL_OK) return st;
  if (workspace_bytes < pl.bytes) return HL_EINVAL;
  AttentionArgs& a = pl.a;
  uint8_t* ws = static_cast<uint8_t*>(workspace_dev);
  a.q = static_cast<const uint16_t*>(q_dev), a.out = static_cast<uint16_t*>(out_dev);
  a.lens = lens_dev, a.lse = lse_dev, a.weight_in = weight_in_dev, a.weight_out = weight_out_dev;
  a.part_o = reinterpret_cast<float*>(ws + pl.part_o), a.part_ml = reinterpret_cast<float*>(ws + pl.part_ml);
  if (weight_out_dev) {
    a.row_ml = reinterpret_cast<float*>(ws + pl.row_ml);
    a.scores = reinterpret_cast<float*>(ws + pl.scores);
  }
  return attention->dtype == HL_BF16 ? run_type<__bf16>(a, (hipStream_t)stream)
                                     : run_type<_Float16>(a, (hipStream_t)stream);
}
