// Attention of a batch over one prefix that all its sequences share and over
// each sequence's own cache (hl_prefix_attention).
//
//   o = sum_j p_j v_j,  p_j = exp(s_j - m) / sum_j exp(s_j - m),  s_j = scale q.k_j
//
// Work. A "row" is one query vector (sequence, new token, head). The rows of
// one key head that see the same keys form an item: over the prefix, the rows
// of the whole batch (so the prefix is read once for all of them), over an own
// cache, the rows of its sequence; up to 128 rows an item, more items beyond.
// Every item's keys are cut into units of 128, and each block takes an equal
// stretch of units, whatever the lengths are. It walks an item's keys with the
// running maximum and sum of the softmax and leaves (maximum, sum, unnormalised
// output) of its part in the workspace; the join kernel adds the parts of each
// row. Lengths are read on the device; nothing depends on the order in which
// blocks run, and there are no atomics.
//
// Items of up to 16 rows (a decode step's own caches) are "narrow": the four
// waves of a block take different keys, 32 at a time, straight from memory to
// registers and one step ahead; nothing in their loop waits for another wave,
// and their four results are added in LDS at the end. Larger items are "wide":
// the four waves have different rows and the same keys, which the block loads
// from memory to LDS without registers between, up to 64 at a time while those
// before them are computed, so that memory is read once for up to 128 rows. The narrow
// items' units stand in one line and the wide items' in another, and the blocks
// are divided between the two by their units.
//
// The matrix instruction takes K as its left operand and Q as its right, so a
// lane ends up with scores of one query (lane % 16), which is also what the
// second product needs of P as its right operand: the keys are only numbered
// differently in the two products, and P never leaves its lane. The values'
// operand has 8 keys of one column in a lane. Narrow items read rows (lane % 16
// owns 8 neighbouring columns of 8 keys) and turn them in registers, one byte
// permutation for two elements; the columns of one lane go to 8 different
// instructions, so that turning needs no other lane's data. Wide items let the
// transposing LDS read do it, whose 16 lanes exchange 4 keys of 16 columns.
//
// Bounds and times (16 bits, 128 columns, 8 key heads, both kernels). Memory
// bounds a decode step: 16 sequences of 32 heads on 4096 own keys each take 58
// us (268 MB, 4.6 TB/s), on 131072 shared keys 111 us (537 MB, 4.8 TB/s), of 64
// heads 122. Many new tokens are bound by the order within a step (scores, then
// softmax, then values): 4 x 256 of them on 4096 shared and 512 own keys take 119
// us (75 GFLOP, 630 TFLOP/s), and the matrix units are busy 38 % of the first
// kernel's time, the vector units 45 %. Short calls are
// bound by their launches and by a few waits for memory in a row: 16 sequences
// on 8192 shared keys take 18 us, three times what reading the keys takes.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "gpu_host.h"

namespace hl {

constexpr uint32_t kUnit = 128;        // keys of a unit
constexpr uint32_t kStep = 32;         // keys of a wave's step
constexpr uint32_t kWaves = 4;         // of a block
constexpr uint32_t kThreads = 64 * kWaves;
// Units of a wide stretch, at least, where there are so many: a stretch leaves a
// part of 64 rows or more, as many bytes as a unit has. 16 sequences on 8192
// shared keys take 18.3 us so, with one unit 20.4.
constexpr uint32_t kLeastWide = 2;
// Units of 128 rows that a block has, at least, where items have so many: two
// tiles a wave halve the reads of LDS for a product, and double what a part
// writes and the join reads. 128 rows a key head on 8192 shared keys (one unit a
// block): 27.2 us with two tiles, 23.3 with one; on 32768 (four) 49.3 and 41.8; on
// 65536 (eight) 72.3 and 73.8; on 131072 123 and 129; 4 x 128 new tokens on 4096
// (eight) 72 and 83.
constexpr uint64_t kManyUnits = 8;
constexpr float kSlack = 8.0f;         // powers of two that a score may pass the maximum kept for it by
constexpr float kLog2e = 1.44269504088896341f;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// One set of keys and values: strides in elements.
struct Kv {
  const uint16_t *k, *v;
  uint64_t k_seq, k_head, v_seq, v_head;
  uint32_t k_token, v_token;
  uint32_t tokens;  // the prefix's length, or an own cache's capacity
};

// Rows of an item: 16 (narrow), or r 16-row tiles for each wave (wide).
struct Tiling {
  uint32_t r, tiles;  // r: 0 narrow; tiles: items of one head (and sequence)
  __host__ __device__ uint32_t rows() const { return r ? 16 * r * kWaves : 16; }
};

struct AttentionArgs {
  Kv prefix, own;
  const uint16_t* q;
  const int32_t* lens;
  uint16_t* out;
  float* lse;
  const float* weight_in;
  float* weight_out;
  float *wide_o, *wide_ml, *narrow_o, *narrow_ml, *row_ml, *scores;  // workspace
  uint32_t batch, queries, heads, kv_heads, dim, share;  // share: query heads of a key head
  uint32_t blocks, wide_rows, narrow_rows, score_stride;  // rows: of a part's place in the workspace
  Tiling tp, to;
  float scale2;  // |scale| * log2(e), or 1: scores are kept in powers of two
  uint32_t q_and, q_xor;  // on pairs of q: its sign is the scale's, and it is 0 where the scale is
};

__device__ inline uint32_t own_length(const AttentionArgs& a, uint32_t b) {
  const int32_t n = a.lens[b];
  return n <= 0 ? 0 : min((uint32_t)n, a.own.tokens);
}

__host__ __device__ inline uint32_t units_of(uint32_t keys) { return (keys + kUnit - 1) / kUnit; }

// Sum over the lanes up to this one. Whole wave; by row shifts and row
// broadcasts, which take a few cycles where a shuffle through LDS takes a
// hundred.
__device__ inline uint32_t scan_lanes(uint32_t v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // lane - 1 of a row of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);  // lane - 2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);  // lane - 4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);  // lane - 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row 0's last to row 1, row 2's to row 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // lane 31 to rows 2 and 3
  return v;
}

// The own caches' part of their line: sequence after sequence, 64 at a time a
// lane each. `each`: units of one of a sequence's items, `end`: where its units
// end, from where the 64 sequences' begin.
struct OwnLine {
  uint32_t each, end, first;  // first: sequence of lane 0
};

__device__ inline OwnLine own_line(const AttentionArgs& a, uint32_t first) {
  const uint32_t b = first + threadIdx.x % 64;
  OwnLine o;
  o.first = first;
  o.each = b < a.batch ? units_of(own_length(a, b)) : 0;
  o.end = scan_lanes(a.kv_heads * a.to.tiles * o.each);
  return o;
}

// Units of sequences 0 .. b-1 (b = batch: of all). Whole wave.
__device__ inline uint32_t own_units_before(const AttentionArgs& a, const OwnLine& o, uint32_t b) {
  if (a.own.tokens == 0 || b == 0) return 0;
  uint32_t sum = 0, b0 = 0;
  for (; b0 + 64 < b; b0 += 64) sum += __builtin_amdgcn_readlane(own_line(a, b0).end, 63);
  return sum + __builtin_amdgcn_readlane(b0 == o.first ? o.end : own_line(a, b0).end, b - 1 - b0);
}

// Where sequence b's units begin in the line, counted from the own caches'
// first, and how many units one of its items has.
struct OwnPlace {
  uint32_t b, begin, each;
};

// The sequence that unit u (counted as above) belongs to. Whole wave.
__device__ inline OwnPlace own_place(const AttentionArgs& a, const OwnLine& o, uint32_t u) {
  const uint32_t items = a.kv_heads * a.to.tiles;
  uint32_t base = 0;
  for (uint32_t b0 = 0; b0 < a.batch; b0 += 64) {
    const OwnLine l = b0 == o.first ? o : own_line(a, b0);
    const uint64_t past = __ballot(base + l.end > u);
    if (past) {
      const int i = __builtin_ctzll(past);
      const uint32_t each = __builtin_amdgcn_readlane(l.each, i), end = __builtin_amdgcn_readlane(l.end, i);
      return {b0 + (uint32_t)i, base + end - items * each, each};
    }
    base += __builtin_amdgcn_readlane(l.end, 63);
  }
  return {a.batch - 1, base, 1};  // past the line's end: no caller asks
}

// A line of units and those that share it, `takers` at most one a unit: taker k
// has units floor(k*total/takers) up to floor((k+1)*total/takers), never none.
struct Line {
  uint32_t total, takers;
  __device__ uint32_t first(uint32_t k) const { return (uint32_t)((uint64_t)k * total / takers); }
  // takers, about, of `units` units that follow each other
  uint32_t parts(uint32_t units) const { return total ? (uint32_t)((uint64_t)units * takers / total) + 1 : 0; }
  __device__ uint32_t taker(uint32_t u) const { return (uint32_t)((((uint64_t)u + 1) * takers - 1) / total); }
};

// Both lines; `wide_blocks` of the blocks, a multiple of 8, take the wide one.
struct Lines {
  Line wide, narrow;
  uint32_t prefix_units, wide_blocks;
};

__host__ __device__ inline Lines lines_of(const AttentionArgs& a, uint32_t own_units) {
  Lines l;
  l.prefix_units = a.kv_heads * a.tp.tiles * units_of(a.prefix.tokens);
  l.wide.total = (a.tp.r ? l.prefix_units : 0) + (a.to.r ? own_units : 0);
  l.narrow.total = l.prefix_units + own_units - l.wide.total;
  uint32_t w = 0;
  if (l.wide.total) {
    w = a.blocks;
    if (l.narrow.total) w = (uint32_t)((uint64_t)a.blocks * l.wide.total / (l.wide.total + l.narrow.total));
    w = std::min(w, (l.wide.total + kLeastWide - 1) / kLeastWide);
    w = std::min((w + 7) / 8 * 8, a.blocks - (l.narrow.total ? 8 : 0));
    w = std::max(w, 8u);
  }
  l.wide_blocks = w;
  l.wide.takers = std::min(w, l.wide.total);
  l.narrow.takers = std::min(a.blocks - w, l.narrow.total);
  return l;
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

// Ends a row of matrix instructions: the instructions after it may write the
// operands of those before. On gfx950 a product has come out wrong now and then
// when the instruction right after it wrote one of its operand registers; the
// compiler places no wait states there, and five are enough.
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

// All bits of each half that is an infinity or NaN (whose exponent is all
// ones, so that one more carries into the sign's place).
template <class T>
__device__ inline uint32_t beyond(uint32_t pair) {
  constexpr uint32_t e = std::is_same<T, __bf16>::value ? 0x7F807F80u : 0x7C007C00u;
  const uint32_t m = ((pair & e) + (std::is_same<T, __bf16>::value ? 0x00800080u : 0x04000400u)) & 0x80008000u;
  return (m - (m >> 15)) | m;
}

// Keeps sums with v from being formed before the loop that needs them, where
// they would take a register each.
__device__ inline uint32_t here(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}

__device__ inline uint32_t lane_id() { return here(threadIdx.x % 64); }

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

// A narrow step's keys and values, as rows.
template <int D>
struct Tile {
  static constexpr bool TURNED = false;
  u32x4 k[2][Shape<D>::KS];
  uint32_t v[8][Shape<D>::HALVES][Shape<D>::VE / 2];
};

// A wide step's: the values as the second product's left operands, output tile
// i having columns 16*i ...
template <int D>
struct TurnedTile {
  static constexpr bool TURNED = true;
  u32x4 k[2][Shape<D>::KS];
  u32x4 v[Shape<D>::TILES];
};

// Key of value row e in lane group c, counted from the step's first: the order
// in which the first product leaves its scores in a lane.
__device__ inline uint32_t key_of(uint32_t c, int e) { return (e < 4 ? 0 : 12) + 4 * c + e; }

// Loads keys (values) key .. key+31 of `it`; where they may pass its end
// (LAST), its last one again.
template <int D, bool FULL, bool LAST>
__device__ inline void load_k(Tile<D>& t, const Item& it, uint32_t dim, uint32_t key) {
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16;
  const uint8_t* kp = reinterpret_cast<const uint8_t*>(it.k + (uint64_t)key * it.k_token);
  const uint32_t left = it.keys - 1 - key, bytes = 2 * it.k_token, first = here(n * bytes);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t at = LAST ? min(16 * h + n, left) * bytes : first + 16 * h * bytes;
#pragma unroll
    for (int s = 0; s < Shape<D>::KS; ++s) {
      const uint32_t d = c * 8 + s * 32;
      const bool in = FULL || d < dim;
      const u32x4 w = *reinterpret_cast<const u32x4*>(kp + (at + (in ? 2 * d : 0)));
      t.k[h][s] = in ? w : u32x4{0, 0, 0, 0};
    }
  }
}

template <int D, bool FULL, bool LAST>
__device__ inline void load_v(Tile<D>& t, const Item& it, uint32_t dim, uint32_t key) {
  using S = Shape<D>;
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16;
  const uint8_t* vp = reinterpret_cast<const uint8_t*>(it.v + (uint64_t)key * it.v_token);
  const uint32_t left = it.keys - 1 - key, bytes = 2 * it.v_token;
#pragma unroll
  for (int h = 0; h < S::HALVES; ++h) {
    uint32_t d = n * S::VE + h * 128;
    if (!FULL && d >= dim) d = 0;  // columns that no output is stored from
    const uint32_t first = here(4 * c * bytes + 2 * d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t at = LAST ? min(key_of(c, e), left) * bytes + 2 * d : first + key_of(0, e) * bytes;
      if constexpr (S::VE == 8) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(vp + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) t.v[e][h][j] = w[j];
      } else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(vp + at);
        t.v[e][h][0] = w[0], t.v[e][h][1] = w[1];
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
  float limit[R];      // m + kSlack; -infinity while m is no score
  uint32_t seen[R];    // keys that the query sees
  uint32_t odd;        // whether a value of this lane was taken out of the product
};

// Output tiles whose values are turned at a time: an operand takes 4 registers.
constexpr int set_of(int d) { return d == 256 ? 2 : 4; }

// The left operands of output tiles i0 .. i0+SET-1: values of 8 keys, for the
// columns that the tiles give this lane. All are turned before a product may
// follow.
template <int D, int SET>
__device__ inline void turn(u32x4 (&vt)[SET], const Tile<D>& t, int i0) {
  using S = Shape<D>;
#pragma unroll
  for (int i = i0; i < i0 + SET; ++i) {
    const uint32_t sel = i % 2 ? 0x07060302u : 0x05040100u;
    const int h = i / S::VE, j = i % S::VE / 2;
#pragma unroll
    for (int e = 0; e < 4; ++e) vt[i - i0][e] = __builtin_amdgcn_perm(t.v[2 * e + 1][h][j], t.v[2 * e][h][j], sel);
  }
#pragma unroll
  for (int i = 0; i < SET; ++i) asm volatile("" : "+v"(vt[i]));
  __builtin_amdgcn_sched_barrier(0);
}

// Ends the products of these operands, which keep their registers until then.
template <int SET>
__device__ inline void turned_end(const u32x4 (&vt)[SET]) {
  products_end();
#pragma unroll
  for (int i = 0; i < SET; ++i) asm volatile("" ::"v"(vt[i]));
}

// The left operands of a wide item's output tiles i0 .. i0+SET-1, two bytes at
// a time from memory: for the few steps that add_beyond looks at again.
template <int SET>
__device__ inline void gather_v(u32x4 (&vt)[SET], const Item& it, uint32_t dim, uint32_t key, int i0) {
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16, left = it.keys - 1 - key;
#pragma unroll
  for (int i = 0; i < SET; ++i) {
    const uint16_t* column = it.v + min((i0 + i) * 16 + n, dim - 1);  // past the head's, its last one
    const auto value = [&](int e) {
      return (uint32_t)column[(uint64_t)(key + min(key_of(c, e), left)) * it.v_token];
    };
#pragma unroll
    for (int e = 0; e < 8; e += 2) vt[i][e / 2] = value(e) | value(e + 1) << 16;
  }
}

// A pair of values to powers of two that say what each is: 1 for +infinity, 64
// for -infinity, 4096 for a NaN, and 0 for the rest. Sums over a step's 32 keys
// still tell them apart.
template <class T>
__device__ inline uint32_t kinds(uint32_t pair) {
  constexpr bool bf = std::is_same<T, __bf16>::value;
  constexpr uint32_t one = bf ? 0x3F803F80u : 0x3C003C00u, sixtyfour = bf ? 0x42804280u : 0x54005400u,
                     big = bf ? 0x45804580u : 0x6C006C00u, mantissa = bf ? 0x007F007Fu : 0x03FF03FFu;
  const uint32_t sign = pair & 0x80008000u, minus = (sign - (sign >> 15)) | sign;
  const uint32_t some = (((pair & mantissa) + mantissa) << (bf ? 8 : 5)) & 0x80008000u, nan = (some - (some >> 15)) | some;
  return beyond<T>(pair) & ((nan & big) | (~nan & ((minus & sixtyfour) | (~minus & one))));
}

// Adds to the outputs what the infinite and NaN values of keys key .. end
// make of them, for the queries that see their keys alone: in the product with
// the weights, where a hidden key has weight 0, they would make NaN of the
// others too. A wave's steps are `stride` keys apart.
template <class T, int D, bool FULL, int R, bool TURNED>
__device__ inline void add_beyond(State<D, R>& st, const Item& it, uint32_t dim, uint32_t key, uint32_t end,
                                  uint32_t stride) {
  const uint32_t c = lane_id() / 16;
  constexpr uint32_t one = std::is_same<T, __bf16>::value ? 0x3F80u : 0x3C00u;
#pragma unroll 1
  for (; key < end; key += stride) {
    Tile<D> t;
    if constexpr (!TURNED) load_v<D, FULL, true>(t, it, dim, key);
    u32x4 sees[R];
#pragma unroll
    for (int rt = 0; rt < R; ++rt)
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        sees[rt][e / 2] =
            (key + key_of(c, e) < st.seen[rt] ? one : 0) | (key + key_of(c, e + 1) < st.seen[rt] ? one << 16 : 0);
#pragma unroll
    for (int i0 = 0; i0 < Shape<D>::TILES; i0 += set_of(D)) {
      u32x4 vt[set_of(D)];
      if constexpr (TURNED)
        gather_v<set_of(D)>(vt, it, dim, key, i0);
      else
        turn<D, set_of(D)>(vt, t, i0);
#pragma unroll
      for (int i = 0; i < set_of(D); ++i) {
        u32x4 kind;
#pragma unroll
        for (int e = 0; e < 4; ++e) kind[e] = kinds<T>(vt[i][e]);
#pragma unroll
        for (int rt = 0; rt < R; ++rt) {
          const f32x4 sum = mfma<T>(kind, sees[rt], f32x4{0.0f, 0.0f, 0.0f, 0.0f});
          products_end();
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int n = (int)sum[r];
            const float up = n & 63 ? INFINITY : 0.0f, down = n & 4032 ? -INFINITY : 0.0f;
            st.o[rt][i0 + i][r] += n >= 4096 ? __builtin_nanf("") : up + down;
          }
        }
      }
    }
  }
}

// One step: scores of 32 keys, their weights, and the weighted values. EDGE:
// some query may not see some of the keys; `most`: keys that some query sees.
// get_k and get_v bring the step's keys and values into the tile.
template <class T, int D, int R, bool EDGE, class Keys, class GetK, class GetV>
__device__ inline void step(State<D, R>& st, Keys& t, const AttentionArgs& a, const Item& it, uint32_t key,
                            uint32_t most, uint32_t wave_row, GetK get_k, GetV get_v) {
  using S = Shape<D>;
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16;
  f32x4 s[R][2];
  u32x4 w[R];
  get_k(t, it, a.dim, key);
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
  if constexpr (!EDGE) get_v(t, it, a.dim, key);  // on its way during the softmax
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    if constexpr (EDGE) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (key + 16 * h + 4 * c + r >= st.seen[rt]) s[rt][h][r] = -INFINITY;
    }
    if (it.scores) {
      const uint32_t row = here(wave_row + 16 * rt + n);  // nothing of this is formed in a call without weights
      if (row < it.rows) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *reinterpret_cast<f32x4*>(it.scores + (uint64_t)row * a.score_stride + key + 16 * h + 4 * c) =
              s[rt][h] * a.scale2;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) top = fmaxf(top, s[rt][h][r]);
    top *= a.scale2;
    // The maximum need not be the true one, only near it: the output is
    // scaled again when a score passes it by more than 2^8, so the weights
    // stay in the 16-bit types' range and most steps scale nothing.
    if (__any(top > st.limit[rt])) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const bool had = st.limit[rt] != -INFINITY;
      const float was = st.m[rt];
      const float now = had ? fmaxf(was, top) : top;
      if (now != -INFINITY) {
        const float f = had ? __builtin_amdgcn_exp2f(was - now) : 0.0f;
        st.m[rt] = now, st.limit[rt] = now + kSlack;
        st.l[rt] *= f;
#pragma unroll
        for (int i = 0; i < S::TILES; ++i) st.o[rt][i] *= f;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float p[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[r] = __builtin_amdgcn_exp2f(fmaf(s[rt][h][r], a.scale2, -st.m[rt]));
        st.l[rt] += p[r];
      }
      w[rt][2 * h] = pack<T>(p[0], p[1]), w[rt][2 * h + 1] = pack<T>(p[2], p[3]);
    }
  }
  if constexpr (EDGE) {
    get_v(t, it, a.dim, key);
    // values that no query sees count 0, whatever they are; those that only
    // some see must be finite in the product (add_beyond has the others)
    const uint32_t some = it.ordered ? ~0u : 0u;
    const auto clean = [&](uint32_t v, uint32_t in) {
      const uint32_t d = v & in, off = beyond<T>(d) & some;
      st.odd |= off;
      return d & ~off;
    };
    uint32_t in[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) in[e] = key + key_of(c, e) < most ? ~0u : 0u;
    if constexpr (Keys::TURNED) {
#pragma unroll
      for (int i = 0; i < S::TILES; ++i)
#pragma unroll
        for (int e = 0; e < 8; e += 2)
          t.v[i][e / 2] = clean(t.v[i][e / 2], (in[e] & 0xFFFFu) | (in[e + 1] & 0xFFFF0000u));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int h = 0; h < S::HALVES; ++h)
#pragma unroll
          for (int j = 0; j < S::VE / 2; ++j) t.v[e][h][j] = clean(t.v[e][h][j], in[e]);
    }
  }
  if constexpr (Keys::TURNED) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < S::TILES; ++i)
#pragma unroll
      for (int rt = 0; rt < R; ++rt) st.o[rt][i] = mfma<T>(t.v[i], w[rt], st.o[rt][i]);
    products_end();
  } else {
#pragma unroll
    for (int i0 = 0; i0 < S::TILES; i0 += set_of(D)) {
      u32x4 vt[set_of(D)];
      turn<D, set_of(D)>(vt, t, i0);
#pragma unroll
      for (int i = 0; i < set_of(D); ++i)
#pragma unroll
        for (int rt = 0; rt < R; ++rt) st.o[rt][i0 + i] = mfma<T>(vt[i], w[rt], st.o[rt][i0 + i]);
      turned_end<set_of(D)>(vt);
    }
  }
}

// LDS buffers of a wide item, a step's keys and values each. Half of them are
// computed while the other half is loaded, and the waves meet once a half: 4 x
// 256 new tokens on 4096 shared keys take 118.7 us so, and 122.9 with a meeting
// and a load each step.
constexpr uint32_t buffers(int d) { return d == 256 ? 2 : 4; }
constexpr uint32_t buffer_bytes(int d) { return kStep * d * 4; }

// A block's LDS in floats: a narrow item's result of every wave (rows padded
// by 4, so that they start in different banks) and their (maximum, sum), or a
// wide item's buffers.
template <int D, int RW>
constexpr uint32_t lds_floats() {
  constexpr uint32_t narrow = kWaves * 16 * (D + 4) + kWaves * 16 * 2;
  constexpr uint32_t wide = RW ? buffers(D) * buffer_bytes(D) / 4 : 0;
  return narrow > wide ? narrow : wide;
}

// Starts a wave's state: its queries, from row `wave_row` of the item's head.
template <int D, bool FULL, int R>
__device__ inline void begin(State<D, R>& st, const AttentionArgs& a, const Item& it, uint32_t wave_row) {
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16;
  st.odd = 0;
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    st.m[rt] = 0.0f, st.l[rt] = 0.0f, st.limit[rt] = -INFINITY;
#pragma unroll
    for (int i = 0; i < Shape<D>::TILES; ++i) st.o[rt][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t row = min(wave_row + 16 * rt + n, it.rows - 1), tok = row / a.share;
    st.seen[rt] = it.ordered ? (it.keys + tok > it.back ? it.keys + tok - it.back : 0) : it.keys;
    const uint16_t* q = it.q + ((uint64_t)tok * a.heads + row % a.share) * a.dim;
#pragma unroll
    for (int s = 0; s < Shape<D>::KS; ++s) {
      const uint32_t d = c * 8 + s * 32;
      const bool in = FULL || d < a.dim;
      const u32x4 w = *reinterpret_cast<const u32x4*>(q + (in ? d : 0));
      st.q[rt][s] = in ? (w & a.q_and) ^ a.q_xor : u32x4{0, 0, 0, 0};
    }
  }
}

// Keys that the token of a head's row sees.
__device__ inline uint32_t seen_by(const AttentionArgs& a, const Item& it, uint32_t row) {
  const uint32_t n = it.keys + min(row, it.rows - 1) / a.share;
  return !it.ordered ? it.keys : n > it.back ? n - it.back : 0;
}

// The sum of a query's weights, of which each of its four lanes has a part.
__device__ inline float over_lanes(float l) {
  l += __shfl_xor(l, 16);
  return l + __shfl_xor(l, 32);
}

// A wave's share of a narrow item's keys [.., k1): 32 from `key` on, and again
// every `stride`.
template <class T, int D, bool FULL>
__device__ inline void narrow_keys(State<D, 1>& st, const AttentionArgs& a, const Item& it, uint32_t key, uint32_t k1,
                                   uint32_t stride) {
  const uint32_t all = seen_by(a, it, it.row0), most = seen_by(a, it, it.row0 + 15), end = min(k1, most);
  const uint32_t whole = min(end, all);  // steps that end here or before hide no key
  if constexpr (D == 256) {  // two steps' keys do not fit the registers
    for (; key + kStep <= whole; key += stride) {
      Tile<D> t;
      step<T, D, 1, false>(st, t, a, it, key, most, it.row0, load_k<D, FULL, false>, load_v<D, FULL, false>);
    }
  } else if (key + kStep <= whole) {
    const auto load = [&](Tile<D>& t, uint32_t at) {
      load_k<D, FULL, false>(t, it, a.dim, at);
      load_v<D, FULL, false>(t, it, a.dim, at);
    };
    const auto there = [](Tile<D>&, const Item&, uint32_t, uint32_t) {};
    Tile<D> t0, t1;
    load(t0, key);
    while (true) {
      bool more = key + stride + kStep <= whole;
      if (more) load(t1, key + stride);
      step<T, D, 1, false>(st, t0, a, it, key, most, it.row0, there, there);
      key += stride;
      if (!more) break;
      more = key + stride + kStep <= whole;
      if (more) load(t0, key + stride);
      step<T, D, 1, false>(st, t1, a, it, key, most, it.row0, there, there);
      key += stride;
      if (!more) break;
    }
  }
  const uint32_t edge = key;
#pragma unroll 1
  for (; key < end; key += stride) {
    Tile<D> t;
    step<T, D, 1, true>(st, t, a, it, key, most, it.row0, load_k<D, FULL, true>, load_v<D, FULL, true>);
  }
  if (__any(st.odd != 0)) add_beyond<T, D, FULL, 1, false>(st, it, a.dim, edge, end, stride);
  st.odd = 0;
}

// Adds the results that WAVES waves have of the same 16 rows and calls
// out(row, d, o, m, l) for four columns from d on of each of the first `rows`.
template <int D, int WAVES, class Out>
__device__ inline void add_waves(const State<D, 1>& st, uint32_t rows, float* lds, Out out) {
  using S = Shape<D>;
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  float* lds_ml = lds + WAVES * 16 * (D + 4);
  const float sum = over_lanes(st.l[0]);
  const uint32_t at = here(wave * 16 + n);  // formed here: no register holds it through the loops
  if (c == 0) lds_ml[2 * at] = st.limit[0] != -INFINITY || sum != sum ? st.m[0] : -INFINITY, lds_ml[2 * at + 1] = sum;
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int h = 0; h < S::HALVES; ++h)
#pragma unroll
      for (int q = 0; q < S::VE; q += 4) {
        const int i = h * S::VE + q;
        *reinterpret_cast<float4*>(lds + (uint64_t)at * (D + 4) + h * 128 + (4 * c + r) * S::VE + q) =
            make_float4(st.o[0][i][r], st.o[0][i + 1][r], st.o[0][i + 2][r], st.o[0][i + 3][r]);
      }
  __syncthreads();
  for (uint32_t x = here(threadIdx.x); x < rows * (D / 4); x += WAVES * 64) {
    const uint32_t row = x / (D / 4), d = x % (D / 4) * 4;
    float m = -INFINITY, l = 0.0f;
    for (uint32_t k = 0; k < WAVES; ++k) m = fmaxf(m, lds_ml[2 * (row + 16 * k)]);
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t k = 0; k < WAVES; ++k) {
      const uint32_t from = row + 16 * k;
      const float mk = lds_ml[2 * from];
      const float f = mk == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mk - m);
      const float4 v = *reinterpret_cast<const float4*>(lds + (uint64_t)from * (D + 4) + d);
      o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
      l += f * lds_ml[2 * from + 1];
    }
    out(row, d, o, m, l);
  }
}

// Keys [k0, k1) of a narrow item by one block; writes the part at `slot`.
template <class T, int D, bool FULL>
__device__ inline void narrow_part(const AttentionArgs& a, const Item& it, uint32_t k0, uint32_t k1, uint32_t slot,
                                   float* lds) {
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  State<D, 1> st;
  begin<D, FULL, 1>(st, a, it, 0);
  narrow_keys<T, D, FULL>(st, a, it, k0 + kStep * wave, k1, kUnit);
  float* po = a.narrow_o + (uint64_t)slot * a.narrow_rows * D;
  float* pml = a.narrow_ml + (uint64_t)slot * a.narrow_rows * 2;
  add_waves<D, kWaves>(st, it.rows, lds,
                       [&](uint32_t row, uint32_t d, float4 o, float m, float l) {
                         *reinterpret_cast<float4*>(po + (uint64_t)row * D + d) = o;
                         if (d == 0) pml[2 * row] = m, pml[2 * row + 1] = l;
                       });
  __syncthreads();
}

// Which place of its row in an LDS buffer 16-byte piece j has, and which piece
// has place j: pairs of pieces change places with the row's number. The 8 lanes
// that read one piece of 8 rows in one cycle, and the 16 that read a pair of
// pieces of 4 rows, then use different banks.
template <int D>
__device__ inline uint32_t place(uint32_t row, uint32_t j) {
  return j ^ 2 * (D == 64 ? row / 2 % 4 : row % 8);
}

// 64 lanes' 16 bytes at base + offset (each lane's own) to LDS, one lane's after
// the other's from `lds` on. Counted by vmcnt alone: the compiler, which would
// wait for all such loads before any read of LDS, does not see it. (M0 holds the
// LDS address; nothing else here uses it.)
__device__ inline void load_to_lds(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 1\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(offset), "s"(base)
               : "memory");
}

// Loads of one wave for a buffer, of keys and of values.
template <int D>
constexpr uint32_t loads_each() {
  return kStep * D * 2 / 1024 / kWaves;
}

// This lane's pieces' places in memory, in bytes from a step's first key and
// value, where the step's keys are all there.
template <int D>
struct Offsets {
  uint32_t k[loads_each<D>()], v[loads_each<D>()];
};

template <int D, bool FULL>
__device__ inline Offsets<D> offsets(const Item& it, uint32_t dim) {
  constexpr uint32_t pieces = D / 8, rows = 64 / pieces;
  const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  Offsets<D> o;
#pragma unroll
  for (uint32_t i = 0; i < loads_each<D>(); ++i) {
    const uint32_t row = (wave * loads_each<D>() + i) * rows + lane / pieces;
    uint32_t d = place<D>(row, lane % pieces) * 16;
    if (!FULL && d >= 2 * dim) d = 0;
    o.k[i] = row * 2 * it.k_token + d, o.v[i] = row * 2 * it.v_token + d;
  }
  return o;
}

// This wave's quarter of keys key .. key+31 of `it` to the buffer at `lds`;
// past its end, its last key again, and past the head's columns, its first
// columns again.
template <int D, bool FULL>
__device__ inline void load_buffer(const Item& it, uint32_t dim, uint32_t key, uint32_t lds, const Offsets<D>& o) {
  constexpr uint32_t pieces = D / 8, rows = 64 / pieces;  // rows of a load
  const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint8_t* kp = reinterpret_cast<const uint8_t*>(it.k + (uint64_t)key * it.k_token);
  const uint8_t* vp = reinterpret_cast<const uint8_t*>(it.v + (uint64_t)key * it.v_token);
  const uint32_t left = it.keys - 1 - key;
  if (left >= kStep - 1) {
#pragma unroll
    for (uint32_t i = 0; i < loads_each<D>(); ++i) {
      const uint32_t x = wave * loads_each<D>() + i;
      load_to_lds(kp, o.k[i], lds + x * 1024);
      load_to_lds(vp, o.v[i], lds + buffer_bytes(D) / 2 + x * 1024);
    }
    return;
  }
#pragma unroll
  for (uint32_t i = 0; i < loads_each<D>(); ++i) {
    const uint32_t x = wave * loads_each<D>() + i, row = x * rows + lane / pieces, from = min(row, left);
    uint32_t d = place<D>(row, lane % pieces) * 16;
    if (!FULL && d >= 2 * dim) d = 0;
    load_to_lds(kp, from * 2 * it.k_token + d, lds + x * 1024);
    load_to_lds(vp, from * 2 * it.v_token + d, lds + buffer_bytes(D) / 2 + x * 1024);
  }
}

// Waits until this wave's loads are done, and for the other waves.
__device__ inline void buffers_ready() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Keys [k0, k1) of a wide item by one block; each wave writes its rows of the
// part at `slot`.
template <class T, int D, bool FULL, int R>
__device__ inline void wide_part(const AttentionArgs& a, const Item& it, uint32_t k0, uint32_t k1, uint32_t slot,
                                 float* lds) {
  using S = Shape<D>;
  constexpr uint32_t bytes = buffer_bytes(D), ring = buffers(D), half = ring / 2;
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const uint32_t wave_row = it.row0 + wave * 16 * R;
  const uint32_t most = seen_by(a, it, wave_row + 16 * R - 1), all = seen_by(a, it, it.row0);
  const uint32_t end = min(k1, seen_by(a, it, it.row0 + 16 * R * kWaves - 1));
  const uint32_t mine = wave_row < it.rows ? min(end, most) : 0;
  const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  const uint32_t steps = k0 < end ? (end - k0 + kStep - 1) / kStep : 0;
  const Offsets<D> places = offsets<D, FULL>(it, a.dim);
#pragma unroll
  for (uint32_t i = 0; i < half; ++i)
    if (i < steps) load_buffer<D, FULL>(it, a.dim, k0 + i * kStep, at + i * bytes, places);
  State<D, R> st;
  begin<D, FULL, R>(st, a, it, wave_row);
  // Steps begin at multiples of 8 rows, so which banks a lane's pieces are in
  // does not depend on the step.
  constexpr int KD = S::KS < 4 ? S::KS : 4;  // of 256 columns, the second half is 16 pieces on
  uint32_t kofs[KD];
#pragma unroll
  for (int s = 0; s < KD; ++s) kofs[s] = n * D * 2 + place<D>(n, c + 4 * s) * 16;
  // Columns 16*i .. of keys 4*c .. 4*c+3: of each key 4 lanes read 4 columns.
  // Tile i's pieces are tile 0's with 2*i changed in their number.
  const uint32_t vrow = 4 * c + n / 4;
  const uint32_t vofs = bytes / 2 + vrow * D * 2 + place<D>(vrow, n % 4 / 2) * 16 + n % 2 * 8;
  uint32_t from;  // the step's buffer
  const auto get_k = [&](TurnedTile<D>& t, const Item&, uint32_t dim, uint32_t) {
#pragma unroll
    for (int s = 0; s < S::KS; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(lds) + from + kofs[s % KD] +
                                                        s / KD * 256 + h * 16 * D * 2);
        t.k[h][s] = FULL || c * 8 + s * 32 < dim ? w : u32x4{0, 0, 0, 0};
      }
  };
  const auto get_v = [&](TurnedTile<D>& t, const Item&, uint32_t, uint32_t) {
#pragma unroll
    for (int i = 0; i < S::TILES; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t v = at + ((from + vofs) ^ (i % 8 * 32)) + i / 8 * 256 + h * 16 * D * 2;
        const s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)v);
        const u32x2 d = __builtin_bit_cast(u32x2, w);
        t.v[i][2 * h] = d[0], t.v[i][2 * h + 1] = d[1];
      }
  };
  const auto ready = [&](uint32_t i) {
    if (i % half == 0) {
      // Half of the buffers are loaded, and all waves have left the others.
      buffers_ready();
#pragma unroll
      for (uint32_t j = i + half; j < i + ring; ++j)
        if (j < steps) load_buffer<D, FULL>(it, a.dim, k0 + j * kStep, at + j % ring * bytes, places);
    }
    from = i % ring * bytes;
  };
  // the steps that hide no key of any wave, then the rest
  const uint32_t whole = k0 < min(end, all) ? (min(end, all) - k0) / kStep : 0;
  uint32_t i = 0;
#pragma unroll 1
  for (; i < whole; ++i) {
    ready(i);
    if (mine == 0) continue;
    TurnedTile<D> t;
    step<T, D, R, false>(st, t, a, it, k0 + i * kStep, most, wave_row, get_k, get_v);
  }
#pragma unroll 1
  for (; i < steps; ++i) {
    ready(i);
    if (k0 + i * kStep >= mine) continue;
    TurnedTile<D> t;
    step<T, D, R, true>(st, t, a, it, k0 + i * kStep, most, wave_row, get_k, get_v);
  }
  if (__any(st.odd != 0)) add_beyond<T, D, FULL, R, true>(st, it, a.dim, k0 + whole * kStep, mine, kStep);
  __syncthreads();  // the buffers are free
  float* po = a.wide_o + (uint64_t)slot * a.wide_rows * D;
  float* pml = a.wide_ml + (uint64_t)slot * a.wide_rows * 2;
#pragma unroll
  for (int rt = 0; rt < R; ++rt) {
    const float sum = over_lanes(st.l[rt]);
    const uint32_t row = here(wave * 16 * R + 16 * rt + n);
    if (it.row0 + row >= it.rows) continue;
    if (c == 0) pml[2 * row] = st.limit[rt] != -INFINITY || sum != sum ? st.m[rt] : -INFINITY, pml[2 * row + 1] = sum;
#pragma unroll
    for (int i = 0; i < S::TILES; ++i)
      *reinterpret_cast<f32x4*>(po + (uint64_t)row * D + 16 * i + 4 * c) = st.o[rt][i];
  }
}

// A head's rows of the whole batch over the prefix, from row0 on.
__device__ inline Item prefix_item(const AttentionArgs& a, uint32_t head, uint32_t row0) {
  Item it;
  it.k = a.prefix.k + head * a.prefix.k_head, it.v = a.prefix.v + head * a.prefix.v_head;
  it.k_token = a.prefix.k_token, it.v_token = a.prefix.v_token;
  it.q = a.q + (uint64_t)head * a.share * a.dim;
  it.keys = a.prefix.tokens, it.back = 0, it.ordered = false;
  it.row0 = row0, it.rows = a.batch * a.queries * a.share;
  it.scores = nullptr;
  return it;
}

// A head's rows of sequence b over its own cache, from row0 on.
__device__ inline Item own_item(const AttentionArgs& a, uint32_t b, uint32_t head, uint32_t row0) {
  Item it;
  it.k = a.own.k + b * a.own.k_seq + head * a.own.k_head, it.v = a.own.v + b * a.own.v_seq + head * a.own.v_head;
  it.k_token = a.own.k_token, it.v_token = a.own.v_token;
  it.q = a.q + ((uint64_t)b * a.queries * a.heads + (uint64_t)head * a.share) * a.dim;
  it.keys = own_length(a, b), it.back = a.queries - 1, it.ordered = a.queries > 1;
  it.row0 = row0, it.rows = a.queries * a.share;
  it.scores = a.scores ? a.scores + ((uint64_t)b * a.kv_heads + head) * it.rows * a.score_stride : nullptr;
  return it;
}

// Unit u of a line: its item, the unit's number in it, and the item's units.
struct Place {
  Item it;
  uint32_t item, in, each;
};

// WIDE: of the wide line. Its items are numbered the prefix's first, then the
// sequences'. Whole wave.
template <bool WIDE>
__device__ inline Place place_of(const AttentionArgs& a, const OwnLine& line, const Lines& l, uint32_t u) {
  Place p;
  const bool has_prefix = WIDE == (a.tp.r != 0);
  const uint32_t before = has_prefix ? l.prefix_units : 0;
  if (u < before) {
    p.each = units_of(a.prefix.tokens), p.item = u / p.each, p.in = u % p.each;
    p.it = prefix_item(a, p.item / a.tp.tiles, p.item % a.tp.tiles * a.tp.rows());
  } else {
    const OwnPlace own = own_place(a, line, u - before);
    const uint32_t x = u - before - own.begin, y = x / own.each;
    p.each = own.each, p.in = x % own.each;
    p.item = (has_prefix ? a.kv_heads * a.tp.tiles : 0) + own.b * a.kv_heads * a.to.tiles + y;
    p.it = own_item(a, own.b, y / a.to.tiles, y % a.to.tiles * a.to.rows());
  }
  return p;
}

// RW: 16-row tiles of a wave in wide items (0: the call has none).
template <class T, int D, bool FULL, int RW>
__global__ void __launch_bounds__(kThreads, 2) parts_kernel(AttentionArgs a) {
  __shared__ __attribute__((aligned(16))) float lds[lds_floats<D, RW>()];
  const OwnLine line = a.own.tokens ? own_line(a, 0) : OwnLine{0, 0, 0};
  const Lines l = lines_of(a, own_units_before(a, line, a.batch));
  // Blocks are dealt to the 8 XCDs in turn. Each XCD has its share of both
  // lines, and takers that stand next to each other, so that the row tiles of a
  // head find its keys in the L2.
  const uint32_t xcd = blockIdx.x % 8, nth = blockIdx.x / 8, wide = l.wide_blocks / 8;
  if (RW && nth < wide) {
    const uint32_t taker = xcd * wide + nth;
    if (taker >= l.wide.takers) return;
    const uint32_t end = l.wide.first(taker + 1);
    for (uint32_t u = l.wide.first(taker); u < end;) {
      const Place p = place_of<true>(a, line, l, u);
      const uint32_t take = min(p.each - p.in, end - u);
      wide_part<T, D, FULL, RW ? RW : 1>(a, p.it, p.in * kUnit, (p.in + take) * kUnit, taker + p.item, lds);
      u += take;
    }
    return;
  }
  const uint32_t taker = xcd * (a.blocks / 8 - wide) + nth - wide;
  if (taker >= l.narrow.takers) return;
  const uint32_t end = l.narrow.first(taker + 1);
  for (uint32_t u = l.narrow.first(taker); u < end;) {
    const Place p = place_of<false>(a, line, l, u);
    const uint32_t take = min(p.each - p.in, end - u);
    narrow_part<T, D, FULL>(a, p.it, p.in * kUnit, (p.in + take) * kUnit, taker + p.item, lds);
    u += take;
  }
}

// What weight a key gets from a sequence's rows of one key head: the sum of
// exp2(score - m) * inv, with (m, inv) of row r at ml[2 * (r / share * step +
// r % share)]. Scores that the mask hides (of the earlier of several tokens)
// are not there.
__device__ inline float key_weight(const AttentionArgs& a, const float* scores, const float* ml, uint32_t step,
                                   uint32_t key, uint32_t keys) {
  const uint32_t newer = keys - 1 - key;
  float w = 0.0f;
  for (uint32_t i = newer < a.queries ? a.queries - 1 - newer : 0; i < a.queries; ++i)
    for (uint32_t g = 0; g < a.share; ++g) {
      const float* r = ml + 2 * ((uint64_t)i * step + g);
      w += __builtin_amdgcn_exp2f(scores[(uint64_t)(i * a.share + g) * a.score_stride + key] - r[0]) * r[1];
    }
  return w;
}

constexpr uint32_t kSoloWaves = 8;

// A whole sequence and key head by one block, over the prefix and its own keys:
// no parts, no second kernel. Rows of a head: at most 16. Bound by the waits for
// memory, one for every 256 keys: 16 sequences on 512 own keys of 8 key heads
// take 11 us (33 MB, 3 TB/s).
template <class T, int D, bool FULL>
__global__ void __launch_bounds__(kSoloWaves * 64, 2) solo_kernel(AttentionArgs a) {
  __shared__ __attribute__((aligned(16))) float lds[kSoloWaves * 16 * (D + 4) + kSoloWaves * 16 * 2];
  __shared__ float s_ml[32];
  const uint32_t head = blockIdx.x, b = blockIdx.y, rows = a.queries * a.share;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  constexpr uint32_t stride = kSoloWaves * kStep;
  Item own = {};
  if (a.own.tokens) own = own_item(a, b, head, 0);
  Item pre = prefix_item(a, head, 0);
  pre.q += (uint64_t)b * a.queries * a.heads * a.dim, pre.rows = rows;
  State<D, 1> st;
  begin<D, FULL, 1>(st, a, pre, 0);  // every row sees the whole prefix
  if (pre.keys) narrow_keys<T, D, FULL>(st, a, pre, kStep * wave, pre.keys, stride);
  if (a.own.tokens) {
    const uint32_t n = lane_id() % 16;
    st.seen[0] = seen_by(a, own, n);
    // the waves that had a step of the prefix less than the others begin
    narrow_keys<T, D, FULL>(st, a, own, kStep * ((wave - (pre.keys + kStep - 1) / kStep) % kSoloWaves), own.keys, stride);
  }
  const uint64_t first = (uint64_t)b * a.queries * a.heads + (uint64_t)head * a.share;
  add_waves<D, kSoloWaves>(st, rows, lds, [&](uint32_t row, uint32_t d, float4 o, float m, float l) {
    const uint64_t at = first + (uint64_t)(row / a.share) * a.heads + row % a.share;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (d < a.dim)
      *reinterpret_cast<u32x2*>(a.out + at * a.dim + d) =
          u32x2{pack<T>(o.x * inv, o.y * inv), pack<T>(o.z * inv, o.w * inv)};
    if (d == 0) {
      if (a.lse) a.lse[at] = l == 0.0f ? -INFINITY : m / kLog2e + logf(l);
      s_ml[2 * row] = l == 0.0f ? 0.0f : m, s_ml[2 * row + 1] = inv;
    }
  });
  if (!a.weight_out) return;
  __syncthreads();  // the block's scores are written
  const uint64_t at = ((uint64_t)b * a.kv_heads + head) * a.own.tokens;
  for (uint32_t key = threadIdx.x; key < a.own.tokens; key += kSoloWaves * 64) {
    const float w = key < own.keys ? key_weight(a, own.scores, s_ml, a.share, key, own.keys) : 0.0f;
    a.weight_out[at + key] = a.weight_in ? a.weight_in[at + key] + w : w;
  }
}

// Parts of a row from which on a block joins it, about: fewer do not hide what
// adding its groups' results in LDS takes. 4 sequences on 8192 shared keys (64
// parts) take 15.8 us so and 22.2 with D/4 lanes a row, 16 sequences (32 parts)
// 19.4 and 20.6; 16 on 4096 own keys (5 parts) 65.3 and 62.4, 8 x 8 new tokens on
// 2000 shared and 777 own (up to 9) 37 and 22.
constexpr uint32_t kManyParts = 16;
constexpr uint32_t kAhead = 8;  // parts whose loads a joining thread has in flight

// Where a row's parts are: over the prefix, then over its own keys.
struct RowParts {
  const float2* ml[2];
  const float* o[2];
  uint32_t step[2], count[2];  // step: rows from one part to the next
};

// Whole wave; the row may be another in each lane.
template <int D>
__device__ inline RowParts parts_of(const AttentionArgs& a, uint32_t row) {
  const uint32_t tok = row / a.heads, hq = row % a.heads, b = tok / a.queries, head = hq / a.share, g = hq % a.share;
  const uint32_t up = units_of(a.prefix.tokens);
  uint32_t own_each = 0, own_begin = 0, own_units = 0;
  if (a.own.tokens) {
    own_each = units_of(own_length(a, b));
    for (uint32_t b0 = 0; b0 < a.batch; b0 += 64) {
      const OwnLine line = own_line(a, b0);
      const uint32_t at = b - b0 - 1, end = __shfl(line.end, at % 64);
      if (b == b0) own_begin = own_units;
      if (at < 63) own_begin = own_units + end;
      own_units += __builtin_amdgcn_readlane(line.end, 63);
    }
  }
  const Lines lines = lines_of(a, own_units);
  RowParts p = {};
  const auto find = [&](int x, const Tiling& tl, uint32_t r, uint32_t item, uint32_t u, uint32_t each) {
    const Line line = tl.r ? lines.wide : lines.narrow;
    const uint32_t first = line.taker(u), rows = tl.r ? a.wide_rows : a.narrow_rows;
    const uint64_t at = (uint64_t)(first + item) * rows + r % tl.rows();
    p.count[x] = line.taker(u + each - 1) - first + 1, p.step[x] = rows;
    p.ml[x] = reinterpret_cast<const float2*>(tl.r ? a.wide_ml : a.narrow_ml) + at;
    p.o[x] = (tl.r ? a.wide_o : a.narrow_o) + at * D;
  };
  const bool both = (a.tp.r != 0) == (a.to.r != 0);  // one line has both
  if (up) {
    const uint32_t r = tok * a.share + g, item = head * a.tp.tiles + r / a.tp.rows();
    find(0, a.tp, r, item, item * up, up);
  }
  if (own_each) {
    const uint32_t r = tok % a.queries * a.share + g, y = head * a.to.tiles + r / a.to.rows();
    find(1, a.to, r, (both ? a.kv_heads * a.tp.tiles : 0) + b * a.kv_heads * a.to.tiles + y,
         (both ? lines.prefix_units : 0) + own_begin + y * own_each, own_each);
  }
  return p;
}

__device__ inline float2 part_ml(const RowParts& p, uint32_t i) {
  return i < p.count[0] ? p.ml[0][(uint64_t)i * p.step[0]] : p.ml[1][(uint64_t)(i - p.count[0]) * p.step[1]];
}

// Adds a row's parts, each a maximum, a sum and D columns in float32: bound by
// two waits for memory, one for the maxima (and as many columns as the registers
// hold) and one for the rest, 6 us for 512 rows of up to 20 parts; many rows are
// bound by its bandwidth, 18 us for 32768 rows. D/4 lanes have four columns of a row each; they are all
// that a row has, or (SPLIT, for few rows) a block has one row, whose parts its
// 1024/D groups of lanes take in turn.
template <class T, int D, bool SPLIT>
__global__ void __launch_bounds__(256) join_kernel(AttentionArgs a) {
  constexpr uint32_t L = D / 4, GROUPS = 256 / L, STREAMS = SPLIT ? GROUPS : 1;
  const uint32_t rows = a.batch * a.queries * a.heads;
  const uint32_t ln = threadIdx.x % L, group = threadIdx.x / L, stream = SPLIT ? group : 0;
  const uint32_t own_row = SPLIT ? blockIdx.x : blockIdx.x * GROUPS + group;
  const uint32_t row = min(own_row, rows - 1);  // lanes past the last row repeat it and store nothing
  const RowParts rp = parts_of<D>(a, row);
  const uint32_t parts = (rp.count[0] + rp.count[1] + STREAMS - 1 - stream) / STREAMS;  // of this group
  // Also where f is 0: a part without a key that the row sees has zeros, and an
  // infinite or NaN value that the row does see must not get lost, however small
  // its weight (nothing else in the call drops it).
  const auto add = [](float4& o, float f, float4 p) { o.x += f * p.x, o.y += f * p.y, o.z += f * p.z, o.w += f * p.w; };
  // outputs of parts x .. x+kAhead-1, their loads in flight together; past the last part, it again
  float4 p[kAhead];
  const auto load = [&](uint32_t x) {
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j) {
      const uint32_t i = min(x + j, parts - 1) * STREAMS + stream;
      p[j] = *reinterpret_cast<const float4*>(i < rp.count[0]
                                                  ? rp.o[0] + (uint64_t)i * rp.step[0] * D + ln * 4
                                                  : rp.o[1] + (uint64_t)(i - rp.count[0]) * rp.step[1] * D + ln * 4);
    }
  };
  float m = -INFINITY, l = 0.0f;
  float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (uint32_t i0 = 0; i0 < parts; i0 += L) {
    const uint32_t some = min(L, parts - i0);
    float mi = -INFINITY, li = 0.0f;
    if (ln < some) {
      const float2 ml = part_ml(rp, (i0 + ln) * STREAMS + stream);
      mi = ml.x, li = ml.y;
    }
    load(i0);
    float top = mi;
    for (uint32_t d = L / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float now = fmaxf(m, top);
    const float f0 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - now);
    const float fi = mi == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mi - now);
    float sum = fi * li;
    for (uint32_t d = L / 2; d; d >>= 1) sum += __shfl_xor(sum, d);
    l = l * f0 + sum, m = now;
    o.x *= f0, o.y *= f0, o.z *= f0, o.w *= f0;
    for (uint32_t i = 0; i < some; i += kAhead) {
      if (i) load(i0 + i);
#pragma unroll
      for (uint32_t j = 0; j < kAhead; ++j) {
        const float f = __shfl(fi, (i + j) % L, L);
        if (i + j < some) add(o, f, p[j]);
      }
    }
  }
  if constexpr (SPLIT) {
    __shared__ float s_m[GROUPS], s_l[GROUPS];
    __shared__ float4 s_o[GROUPS][L];
    if (ln == 0) s_m[group] = m, s_l[group] = l;
    s_o[group][ln] = o;
    __syncthreads();
    if (group != 0) return;
    m = -INFINITY, l = 0.0f;
    for (uint32_t w = 0; w < GROUPS; ++w) m = fmaxf(m, s_m[w]);
    o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t w = 0; w < GROUPS; ++w) {
      const float f = s_m[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(s_m[w] - m);
      l += f * s_l[w];
      add(o, f, s_o[w][ln]);
    }
  }
  if (own_row >= rows) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (ln * 4 < a.dim)
    *reinterpret_cast<u32x2*>(a.out + (uint64_t)row * a.dim + ln * 4) =
        u32x2{pack<T>(o.x * inv, o.y * inv), pack<T>(o.z * inv, o.w * inv)};
  if (ln == 0) {
    if (a.lse) a.lse[row] = l == 0.0f ? -INFINITY : m / kLog2e + logf(l);
    if (a.row_ml) a.row_ml[2 * row] = l == 0.0f ? 0.0f : m, a.row_ml[2 * row + 1] = inv;
  }
}

// weight_out = weight_in + the weight that the call's rows gave each own key;
// a thread adds its key's rows in their order, so that the sum is the same in
// every run. The scores come from the parts kernel through the workspace: 8
// sequences of 64 heads and 4096 keys, 8 MB, 5.4 us, most of it launch and wait.
__global__ void __launch_bounds__(256) weights_kernel(AttentionArgs a) {
  const uint32_t head = blockIdx.y, b = blockIdx.z, key = blockIdx.x * 256 + threadIdx.x;
  if (key >= a.own.tokens) return;
  const uint64_t item = (uint64_t)b * a.kv_heads + head, at = item * a.own.tokens + key;
  const uint32_t keys = own_length(a, b);
  float w = 0.0f;
  if (key < keys)
    w = key_weight(a, a.scores + item * a.queries * a.share * a.score_stride,
                   a.row_ml + 2 * ((uint64_t)b * a.queries * a.heads + (uint64_t)head * a.share), a.heads, key, keys);
  a.weight_out[at] = a.weight_in ? a.weight_in[at] + w : w;
}


// ------------------------------------------------------------------- host

// Items of `rows` rows: narrow up to 16; wide ones take r 16-row tiles a wave.
// Of 16 rows or fewer, all but one of a wide item's waves would have none: one
// sequence (4 rows a key head) on 2048 own keys takes 11.6 us, wide 14.8; on 8192
// shared keys 14.8 and 15.5.
static Tiling tiling(uint64_t rows, uint32_t r) {
  Tiling t;
  t.r = rows <= 16 ? 0 : r;
  t.tiles = (uint32_t)((rows + t.rows() - 1) / t.rows());
  return t;
}

// Keys up to which a block takes a sequence and key head alone, and the same
// where there is a block for every second compute unit. One sequence on 256 own
// keys takes 5.6 us so and 9.0 in parts, on 512 8.0 and 9.4, on 768 9.8 and 9.5
// (but one launch for two), on 1024 13.2 and 10.1; 16 sequences on 768 17.6 and
// 19.9, on 1024 22 and 23, on 1536 30 and 28.
constexpr uint64_t kSoloKeys = 768, kSoloKeysMany = 1024;

// A workspace's size, at least: 0 says that the arguments are bad, and
// allocations of 0 bytes have no address.
constexpr uint64_t kLeastWorkspace = 512;

struct AttentionPlan {
  AttentionArgs a;
  uint64_t bytes, wide_o, wide_ml, narrow_o, narrow_ml, row_ml, scores;  // of the workspace: its size and its parts' places
  bool solo, wide, split;  // wide: whether the call has wide items; split: whether a block joins a row
  uint64_t join_blocks;
};

static hl_status check_kv(const hl_kv& s, uint64_t tokens, uint32_t dim, bool sequences) {
  if (tokens == 0) return HL_OK;
  if (!s.k_dev || !s.v_dev || !aligned(s.k_dev, 16) || !aligned(s.v_dev, 16)) return HL_EINVAL;
  const uint64_t strides[6] = {s.k_token, s.v_token, s.k_head, s.v_head, sequences ? s.k_seq : 0, sequences ? s.v_seq : 0};
  for (uint64_t x : strides) {
    if (x % 8) return HL_EINVAL;
    if (x >= (1ull << 40)) return HL_EUNSUPPORTED;
  }
  // the offsets in bytes within 64 tokens stay within 32 bits
  if (s.k_token >= (1ull << 25) || s.v_token >= (1ull << 25)) return HL_EUNSUPPORTED;
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
  a.scale2 = h->scale == 0.0f ? 1.0f : fabsf(h->scale) * kLog2e;
  a.q_and = h->scale == 0.0f ? 0 : ~0u, a.q_xor = h->scale < 0.0f ? 0x80008000u : 0;
  const uint64_t shared_rows = (uint64_t)h->batch * h->queries * a.share, own_rows = (uint64_t)h->queries * a.share;
  // two blocks a compute unit: what their registers allow, and they hide each
  // other's waits; a multiple of 8, for the XCDs
  const uint64_t cus = (uint64_t)device_cus(), most = std::max<uint64_t>(16, cus * 2 / 8 * 8);
  // most that the lengths can come to, of each line
  uint64_t prefix_items, own_items, prefix_units, own_units, wide_units;
  uint32_t r = std::max(shared_rows, own_rows) > 64 && h->dim <= 128 ? 2 : 1;
  for (;; r = 1) {
    a.tp = tiling(shared_rows, r), a.to = tiling(own_rows, r);
    // A set without keys has no items: those of a line are numbered on from the
    // prefix's, and each has a part.
    if (a.prefix.tokens == 0) a.tp.tiles = 0;
    if (a.own.tokens == 0) a.to.tiles = 0;
    prefix_items = (uint64_t)h->kv_heads * a.tp.tiles, own_items = (uint64_t)h->batch * h->kv_heads * a.to.tiles;
    prefix_units = prefix_items * units_of(a.prefix.tokens), own_units = own_items * units_of(a.own.tokens);
    wide_units = (a.tp.r ? prefix_units : 0) + (a.to.r ? own_units : 0);
    if (r == 1 || wide_units >= kManyUnits * most) break;
  }
  const uint64_t narrow_units = prefix_units + own_units - wide_units;
  if (prefix_units + own_units >= (1ull << 31)) return HL_EUNSUPPORTED;
  const uint64_t asked = wide_units / kLeastWide + narrow_units + 15;
  a.blocks = (uint32_t)std::min<uint64_t>(most, std::max<uint64_t>(16, asked / 8 * 8));
  a.wide_rows = std::max(a.tp.r ? a.tp.rows() : 0, a.to.r ? a.to.rows() : 0);
  a.narrow_rows = (uint32_t)std::min<uint64_t>(16, std::max(a.tp.r ? 0 : shared_rows, a.to.r ? 0 : own_rows));
  const uint32_t held = h->dim <= 64 ? 64 : h->dim <= 128 ? 128 : 256;
  // A line's parts: a block (its taker) has one of each item that it takes units
  // of, at taker + item, and both only grow along the line.
  const uint64_t wide_slots = wide_units ? a.blocks + (a.tp.r ? prefix_items : 0) + (a.to.r ? own_items : 0) : 0;
  const uint64_t narrow_slots = narrow_units ? a.blocks + (a.tp.r ? 0 : prefix_items) + (a.to.r ? 0 : own_items) : 0;
  uint64_t n = 0;
  auto take = [&](uint64_t floats) {
    const uint64_t at = n;
    n += (floats * 4 + 255) / 256 * 256;
    return at;
  };
  // A block a sequence and key head where that is short: it reads the prefix
  // again for each sequence (from the L2s, as far as it is the same), and saves
  // the second kernel.
  pl->solo = own_rows <= 16 && a.prefix.tokens + a.own.tokens <=
                                   ((uint64_t)h->batch * h->kv_heads * 2 >= cus ? kSoloKeysMany : kSoloKeys);
  pl->wide = wide_units != 0;
  const Lines lines = lines_of(a, (uint32_t)own_units);
  pl->split = (a.tp.r ? lines.wide : lines.narrow).parts(units_of(a.prefix.tokens)) +
                  (a.to.r ? lines.wide : lines.narrow).parts(units_of(a.own.tokens)) > kManyParts;
  const uint64_t each = pl->split ? 1 : 1024 / held;  // rows of a joining block
  pl->join_blocks = (rows + each - 1) / each;
  if (!pl->solo && !grid_fits(pl->join_blocks, 256)) return HL_EUNSUPPORTED;
  const uint64_t wide = pl->solo ? 0 : wide_slots * a.wide_rows, narrow = pl->solo ? 0 : narrow_slots * a.narrow_rows;
  pl->wide_o = take(wide * held), pl->wide_ml = take(wide * 2);
  pl->narrow_o = take(narrow * held), pl->narrow_ml = take(narrow * 2);
  a.score_stride = (a.own.tokens + kStep - 1) / kStep * kStep;
  pl->row_ml = weights && !pl->solo ? take(rows * 2) : 0;
  pl->scores = weights ? take((uint64_t)h->batch * h->heads * h->queries * a.score_stride) : 0;
  pl->bytes = std::max(n, kLeastWorkspace);
  return HL_OK;
}

template <class T, int D, bool FULL, int RW>
static hl_status run(const AttentionPlan& pl, hipStream_t s) {
  const AttentionArgs& a = pl.a;
  hl_status st = enqueue(parts_kernel<T, D, FULL, RW>, dim3(a.blocks), dim3(kThreads), s, a);
  if (st != HL_OK) return st;
  // A block a row where it has many parts, each of which is a trip to memory.
  const dim3 blocks((uint32_t)pl.join_blocks);
  st = pl.split ? enqueue(join_kernel<T, D, true>, blocks, dim3(256), s, a)
                : enqueue(join_kernel<T, D, false>, blocks, dim3(256), s, a);
  if (st != HL_OK || !a.scores) return st;
  return enqueue(weights_kernel, dim3((a.own.tokens + 255) / 256, a.kv_heads, a.batch), dim3(256), s, a);
}

template <class T, int D, bool FULL>
static hl_status run_rows(const AttentionPlan& pl, hipStream_t s) {
  const AttentionArgs& a = pl.a;
  if (pl.solo) return enqueue(solo_kernel<T, D, FULL>, dim3(a.kv_heads, a.batch), dim3(kSoloWaves * 64), s, a);
  const uint32_t r = std::max(a.tp.r, a.to.r);
  if (!pl.wide) return run<T, D, FULL, 0>(pl, s);
  if constexpr (D <= 128) {
    if (r == 2) return run<T, D, FULL, 2>(pl, s);
  }
  return run<T, D, FULL, 1>(pl, s);
}

template <class T>
static hl_status run_type(const AttentionPlan& pl, hipStream_t s) {
  const AttentionArgs& a = pl.a;
  if (a.dim == 64) return run_rows<T, 64, true>(pl, s);
  if (a.dim < 64) return run_rows<T, 64, false>(pl, s);
  if (a.dim == 128) return run_rows<T, 128, true>(pl, s);
  if (a.dim < 128) return run_rows<T, 128, false>(pl, s);
  if (a.dim == 256) return run_rows<T, 256, true>(pl, s);
  return run_rows<T, 256, false>(pl, s);
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
  a.wide_o = reinterpret_cast<float*>(ws + pl.wide_o), a.wide_ml = reinterpret_cast<float*>(ws + pl.wide_ml);
  a.narrow_o = reinterpret_cast<float*>(ws + pl.narrow_o), a.narrow_ml = reinterpret_cast<float*>(ws + pl.narrow_ml);
  if (weight_out_dev) {
    a.row_ml = reinterpret_cast<float*>(ws + pl.row_ml);
    a.scores = reinterpret_cast<float*>(ws + pl.scores);
  }
  return attention->dtype == HL_BF16 ? run_type<__bf16>(pl, (hipStream_t)stream)
                                     : run_type<_Float16>(pl, (hipStream_t)stream);
}
