// What the attention kernels over 16-bit and over 4-bit keys and values share:
// their arguments, how the work is cut and found, and the host's plan of a call.
#pragma once
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "gpu_host.h"
#include "matrix.h"

namespace hl {

constexpr uint32_t kUnit = 128;        // keys of a unit
constexpr uint32_t kStep = 32;         // keys of a wave's step
constexpr uint32_t kWaves = 4;         // of a block
constexpr uint32_t kThreads = 64 * kWaves;
// Units of a wide stretch, at least, where there are so many: a stretch leaves a
// part of 64 rows or more, as many bytes as a unit has. 16 sequences on 8192
// shared keys take 18.3 us so, with one unit 20.4. In 4 bits (two units, one): 23.0 and
// 23.5, on 2048 18.4 and 15.7, 64 new tokens of one on 2048 shared and 512 own 29.1 and
// 36.5.
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

typedef short s16x4 __attribute__((ext_vector_type(4)));

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
  uint32_t wide_cost, item_cost;  // of a wide unit and, beyond its units, of a narrow item, in narrow units
  uint32_t narrow_items;          // most of them
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
    const uint64_t cost = (uint64_t)l.wide.total * a.wide_cost;
    const uint64_t rest = (uint64_t)l.narrow.total + a.item_cost * (uint64_t)std::min(a.narrow_items, l.narrow.total);
    if (l.narrow.total) w = (uint32_t)(a.blocks * cost / (cost + rest));
    w = std::min(w, (l.wide.total + kLeastWide - 1) / kLeastWide);
    w = std::min((w + 7) / 8 * 8, a.blocks - (l.narrow.total ? 8 : 0));
    w = std::max(w, 8u);
  }
  l.wide_blocks = w;
  l.wide.takers = std::min(w, l.wide.total);
  l.narrow.takers = std::min(a.blocks - w, l.narrow.total);
  return l;
}

// Two float32 to two 16-bit values, each rounded to nearest.
template <class T>
__device__ inline uint32_t pack(float lo, float hi) {
  typedef T pair __attribute__((ext_vector_type(2)));
  const pair p = {(T)lo, (T)hi};
  return __builtin_bit_cast(uint32_t, p);
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

// Key of value row e in lane group c, counted from the step's first: the order
// in which the first product leaves its scores in a lane.
__device__ inline uint32_t key_of(uint32_t c, int e) { return (e < 4 ? 0 : 12) + 4 * c + e; }

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

struct AttentionPlan {
  AttentionArgs a;
  uint64_t bytes, wide_o, wide_ml, narrow_o, narrow_ml, row_ml, scores;  // of the workspace: its size and its parts' places
  bool solo, wide, split;  // wide: whether the call has wide items; split: whether a block joins a row
  uint64_t join_blocks;
};

// Checks a call's shape and plans it, for keys and values in 16 or in 4 bits (whose
// wide items have one 16-row tile a wave).
hl_status attention_plan(const hl_attention* attention, bool weights, bool four_bits, AttentionPlan* plan);

// Checks a call's arguments and plans it; fills the plan's arguments with the
// buffers and the workspace's parts.
hl_status attention_setup(const hl_attention* attention, const void* q_dev, const int32_t* lens_dev, void* out_dev,
                          float* lse_dev, const float* weight_in_dev, float* weight_out_dev, void* workspace_dev,
                          size_t workspace_bytes, bool four_bits, AttentionPlan* plan);

// Adds the parts that a call's blocks have left, and then the keys' weights.
hl_status attention_join(const AttentionPlan& plan, hl_dtype dtype, hipStream_t s);

}  // namespace hl
