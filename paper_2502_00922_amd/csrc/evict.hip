// Eviction from a cache by accumulated attention weight (hl_cache_evict): of
// each sequence and key head the newest tokens and the heaviest of the others
// are kept and moved, in their order, to a smaller cache.
//
// select_kernel, one block a (sequence, key head), finds the weight of the last
// token kept by its digits (11, 11 and 10 bits of the weight as an ordered
// integer: a histogram in LDS each), then numbers the kept tokens with one prefix
// sum over the block; ties go to the lowest slot. It reads the weights, a
// hundredth of the cache, once, and holds them in registers. The atomics of the
// histograms, the barriers between its passes and the scattered stores of the
// slots bound it: 32 caches of 65536 tokens take 42 us, 128 of 4096 8.4 us.
// move_kernel copies the kept rows in 16-byte pieces and is bound by HBM: 16384
// of 65536 rows of 32 caches, 128 columns of K and of V, 537 MB read and written,
// 107 us (5.0 TB/s). A selecting block with few rows to move moves them itself:
// 256 of 1024 tokens of 8 key heads, 9.0 us for both.
#include <algorithm>

#include "gpu_host.h"

namespace hl {

constexpr uint32_t kThreads = 1024, kWaves = kThreads / 64;
constexpr uint32_t kRow = 4 * kThreads;  // weights of a row: four a thread, next to each other
constexpr uint32_t kBins = 2048;
constexpr uint64_t kFewMoved = 65536;    // columns of K (and of V) that a selecting block moves itself, at most (below)
constexpr uint32_t kCopies = 4;          // of the histogram: lanes of a wave often count in one bin
constexpr uint32_t kCopy = kBins + 16;   // their distance: a bin's copies are in different banks

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct EvictArgs {
  const float* weight;
  const int32_t* lens;
  float* weight_out;
  int32_t *slots, *lens_out;
  const uint16_t *k, *v;
  uint16_t *k_out, *v_out;
  uint64_t k_seq, k_token, k_head, v_seq, v_token, v_head;                          // of the cache
  uint64_t ko_seq, ko_token, ko_head, vo_seq, vo_token, vo_head;                    // of the smaller one
  uint32_t batch, kv_heads, dim, tokens, keep, recent;
};

// A weight as an integer of the same order; -0 equals 0, NaN is below all.
__device__ inline uint32_t ordered(float w) {
  if (w != w) return 0;
  const uint32_t b = __builtin_bit_cast(uint32_t, w + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The weight that an ordered integer stands for; w[i] itself where two weights
// have one integer.
__device__ inline float weight_of(uint32_t key, const float* w, uint32_t i) {
  if (key == 0 || key == 0x80000000u) return w[i];
  return __builtin_bit_cast(float, key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

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

// A thread's rows of weights as ordered integers: weight x of row r is token
// base + r*kRow + 4*thread + x. Places from `old` on get 0, the least of all, and
// stand after every token: as fewer than `old` tokens are to be found, none of
// these is, and nothing below tells them from tokens.
template <uint32_t ROWS>
__device__ inline void load_keys(uint32_t (&key)[ROWS][4], const float* w, uint32_t base, uint32_t old) {
  const bool wide = (reinterpret_cast<uintptr_t>(w) & 15) == 0;
  float f[ROWS][4];  // all loads first, so that they are in flight together
#pragma unroll
  for (uint32_t r = 0; r < ROWS; ++r) {
    const uint32_t at = base + r * kRow + 4 * threadIdx.x;
    if (wide && base + (r + 1) * kRow <= old) {
      const float4 v = *reinterpret_cast<const float4*>(w + at);
      f[r][0] = v.x, f[r][1] = v.y, f[r][2] = v.z, f[r][3] = v.w;
    } else {
#pragma unroll
      for (uint32_t x = 0; x < 4; ++x) f[r][x] = at + x < old ? w[at + x] : __builtin_nanf("");
    }
  }
#pragma unroll
  for (uint32_t r = 0; r < ROWS; ++r)
#pragma unroll
    for (uint32_t x = 0; x < 4; ++x) key[r][x] = ordered(f[r][x]);
}

constexpr uint32_t kMoves = 4;  // 16-byte pieces of K, and of V, a thread has in flight

// Moves pieces x0, x0 + step, .. (kMoves of them) of a sequence's kept rows:
// piece(x) = (row, key head, first column), none from `count` on. Slots that
// hold no token give zeros.
template <class Piece>
__device__ inline void move(const EvictArgs& a, uint32_t b, uint64_t x0, uint32_t step, uint64_t count, Piece piece) {
  u32x4 k[kMoves], v[kMoves];
  int32_t slot[kMoves];
  uint32_t row[kMoves], head[kMoves], d[kMoves];
#pragma unroll
  for (uint32_t m = 0; m < kMoves; ++m) {
    if (x0 + m * step >= count) continue;
    piece(x0 + m * step, row[m], head[m], d[m]);
    slot[m] = a.slots[((uint64_t)b * a.kv_heads + head[m]) * a.keep + row[m]];
  }
#pragma unroll
  for (uint32_t m = 0; m < kMoves; ++m) {
    if (x0 + m * step >= count) continue;
    k[m] = v[m] = u32x4{0, 0, 0, 0};
    if (slot[m] < 0) continue;
    const uint64_t s = (uint32_t)slot[m];
    k[m] = *reinterpret_cast<const u32x4*>(a.k + b * a.k_seq + s * a.k_token + head[m] * a.k_head + d[m]);
    v[m] = *reinterpret_cast<const u32x4*>(a.v + b * a.v_seq + s * a.v_token + head[m] * a.v_head + d[m]);
  }
#pragma unroll
  for (uint32_t m = 0; m < kMoves; ++m) {
    if (x0 + m * step >= count) continue;
    *reinterpret_cast<u32x4*>(a.k_out + b * a.ko_seq + row[m] * a.ko_token + head[m] * a.ko_head + d[m]) = k[m];
    *reinterpret_cast<u32x4*>(a.v_out + b * a.vo_seq + row[m] * a.vo_token + head[m] * a.vo_head + d[m]) = v[m];
  }
}

// ROWS: rows of weights that stay in registers. Longer caches are read again
// for each digit, ROWS rows at a time.
template <uint32_t ROWS>
__device__ inline void select(const EvictArgs& a) {
  __shared__ uint32_t s_bin[kCopies][kCopy];
  __shared__ uint32_t s_wave[kWaves], s_digit, s_above, s_in;
  __shared__ uint32_t s_more[ROWS * kWaves], s_same[ROWS * kWaves];
  const uint32_t head = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid % 64;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const uint64_t item = (uint64_t)b * a.kv_heads + head;
  const float* w = a.weight + item * a.tokens;
  float* w_out = a.weight_out + item * a.keep;
  int32_t* slots = a.slots + item * a.keep;
  const int32_t len = a.lens[b];
  const uint32_t n = len <= 0 ? 0 : min((uint32_t)len, a.tokens);
  if (head == 0 && tid == 0) a.lens_out[b] = (int32_t)min(n, a.keep);
  if (n <= a.keep) {
    for (uint32_t i = tid; i < a.keep; i += kThreads) {
      slots[i] = i < n ? (int32_t)i : -1;
      w_out[i] = i < n ? w[i] : 0.0f;
    }
    return;
  }
  const uint32_t old = n - a.recent, need = a.keep - a.recent;  // need < old
  uint32_t key[ROWS][4];
  const bool held = old <= ROWS * kRow;
  if (need) load_keys<ROWS>(key, w, 0, old);
  for (uint32_t i = tid; i < a.recent; i += kThreads) {
    slots[need + i] = (int32_t)(old + i);
    w_out[need + i] = w[old + i];
  }
  if (need == 0) return;
  // The digits, from the highest, of the last weight kept: `prefix` has those
  // found, `left` counts the tokens still to take among the weights that begin
  // with it, `shift` is what of a weight is not compared yet.
  uint32_t prefix = 0, left = need, shift = 32;
  for (int pass = 0; pass < 3; ++pass) {
    const uint32_t width = pass < 2 ? 11 : 10, bins = 1u << width;
    for (uint32_t i = tid; i < kCopies * kCopy; i += kThreads) (&s_bin[0][0])[i] = 0;
    __syncthreads();
    for (uint32_t base = 0; base < old; base += ROWS * kRow) {
      if (!held) load_keys<ROWS>(key, w, base, old);
#pragma unroll
      for (uint32_t r = 0; r < ROWS; ++r) {
        if (base + r * kRow >= old) break;
#pragma unroll
        for (uint32_t x = 0; x < 4; ++x)
          if (pass == 0 || key[r][x] >> shift == prefix)
            atomicAdd(&s_bin[tid % kCopies][(key[r][x] >> (shift - width)) & (bins - 1)], 1u);
      }
    }
    __syncthreads();
    // thread t has bins 2t and 2t+1 counted from the highest; the counts above
    // them say which bin the last token kept is in
    uint32_t high = 0, low = 0;
    const uint32_t at = bins - 2 - 2 * tid;
    if (2 * tid < bins)
      for (uint32_t c = 0; c < kCopies; ++c) high += s_bin[c][at + 1], low += s_bin[c][at];
    const uint32_t sum = scan_lanes(high + low);
    if (lane == 63) s_wave[wave] = sum;
    __syncthreads();
    const uint32_t waves = scan_lanes(lane < kWaves ? s_wave[lane] : 0);
    const uint32_t above = sum - high - low + (wave ? __builtin_amdgcn_readlane(waves, wave - 1) : 0);
    if (above < left && left <= above + high) s_digit = at + 1, s_above = above, s_in = high;
    if (above + high < left && left <= above + high + low) s_digit = at, s_above = above + high, s_in = low;
    __syncthreads();
    prefix = prefix << width | s_digit;
    left -= s_above;
    shift -= width;
    if (s_in == left) break;  // all that begin so are kept: lower digits do not matter
  }
  // Kept: the first digits above `prefix`, and the first `left` tokens equal to
  // it. Each token's place is the number of kept ones before it.
  uint32_t more0 = 0, same0 = 0;  // of earlier rows
  for (uint32_t base = 0; base < old; base += ROWS * kRow) {
    if (!held) load_keys<ROWS>(key, w, base, old);
    uint32_t ahead[ROWS];  // above and equal (high half) in this row and wave before this thread
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < ROWS; ++r) {
      uint32_t mine = 0;
#pragma unroll
      for (uint32_t x = 0; x < 4; ++x) {
        const uint32_t d = key[r][x] >> shift;
        mine += d > prefix ? 1u : d == prefix ? 1u << 16 : 0u;
      }
      const uint32_t sum = scan_lanes(mine);
      ahead[r] = sum - mine;
      if (lane == 63) s_more[r * kWaves + wave] = sum & 0xFFFF, s_same[r * kWaves + wave] = sum >> 16;
    }
    __syncthreads();
    if (wave == 0) {
      uint32_t more = more0, same = same0;
      for (uint32_t i = 0; i < ROWS * kWaves; i += 64) {
        const bool in = i + lane < ROWS * kWaves;
        const uint32_t m = in ? s_more[i + lane] : 0, e = in ? s_same[i + lane] : 0;
        const uint32_t ms = scan_lanes(m), es = scan_lanes(e);
        if (in) s_more[i + lane] = more + ms - m, s_same[i + lane] = same + es - e;
        more += __builtin_amdgcn_readlane(ms, 63), same += __builtin_amdgcn_readlane(es, 63);
      }
      if (lane == 0) s_above = more, s_in = same;
    }
    __syncthreads();
    more0 = s_above, same0 = s_in;
#pragma unroll
    for (uint32_t r = 0; r < ROWS; ++r) {
      uint32_t more = s_more[r * kWaves + wave] + (ahead[r] & 0xFFFF), same = s_same[r * kWaves + wave] + (ahead[r] >> 16);
#pragma unroll
      for (uint32_t x = 0; x < 4; ++x) {
        const uint32_t i = base + r * kRow + 4 * tid + x, d = key[r][x] >> shift;
        if (d > prefix || (d == prefix && same < left)) {
          const uint32_t to = more + min(same, left);
          slots[to] = (int32_t)i;
          w_out[to] = weight_of(key[r][x], w, i);
        }
        more += d > prefix, same += d == prefix;
      }
    }
  }
}

// MOVE: each block moves the rows that it has found, too.
template <uint32_t ROWS, bool MOVE>
__global__ void __launch_bounds__(1024) select_kernel(EvictArgs a) {
  select<ROWS>(a);
  if constexpr (MOVE) {
    __syncthreads();  // the block's slots are written
    const uint32_t pieces = a.dim / 8, count = a.keep * pieces, own = blockIdx.x;
    for (uint32_t x0 = threadIdx.x; x0 < count; x0 += kThreads * kMoves)
      move(a, blockIdx.y, x0, kThreads, count, [&](uint64_t x, uint32_t& row, uint32_t& head, uint32_t& d) {
        row = (uint32_t)x / pieces, head = own, d = (uint32_t)x % pieces * 8;
      });
  }
}

// A sequence's kept rows by many blocks, all key heads of a row together.
__global__ void __launch_bounds__(256) move_kernel(EvictArgs a) {
  const uint32_t pieces = a.dim / 8;
  move(a, blockIdx.y, (uint64_t)blockIdx.x * 256 * kMoves + threadIdx.x, 256, (uint64_t)a.keep * a.kv_heads * pieces,
       [&](uint64_t x, uint32_t& row, uint32_t& head, uint32_t& d) {
         const uint32_t y = (uint32_t)(x / pieces);
         row = y / a.kv_heads, head = y % a.kv_heads, d = (uint32_t)(x % pieces) * 8;
       });
}

}  // namespace hl

using namespace hl;

static hl_status check_cache(const hl_kv* c) {
  if (!c || c->tokens == 0 || !c->k_dev || !c->v_dev || !aligned(c->k_dev, 16) || !aligned(c->v_dev, 16))
    return HL_EINVAL;
  for (uint64_t x : {c->k_token, c->v_token, c->k_head, c->v_head, c->k_seq, c->v_seq}) {
    if (x % 8) return HL_EINVAL;
    if (x >= (1ull << 40)) return HL_EUNSUPPORTED;
  }
  return HL_OK;
}

extern "C" hl_status hl_cache_evict(const hl_kv* from, const hl_kv* to, uint32_t batch, uint32_t kv_heads,
                                    uint32_t dim, const float* weight_dev, const int32_t* lens_dev, uint64_t keep,
                                    uint64_t recent, float* weight_out_dev, int32_t* slots_dev, int32_t* lens_out_dev,
                                    void* stream) {
  hl_status st = check_cache(from);
  if (st == HL_OK) st = check_cache(to);
  if (st != HL_OK) return st;
  if (!weight_dev || !lens_dev || !weight_out_dev || !slots_dev || !lens_out_dev || batch == 0 || kv_heads == 0 ||
      dim == 0 || dim % 8 || keep == 0 || recent > keep || to->tokens < keep)
    return HL_EINVAL;
  if (!aligned(weight_dev, 4) || !aligned(lens_dev, 4) || !aligned(weight_out_dev, 4) || !aligned(slots_dev, 4) ||
      !aligned(lens_out_dev, 4))
    return HL_EINVAL;
  if (from->tokens >= (1ull << 30) || keep >= (1ull << 30) || batch > 65535 || kv_heads > 65535 || dim > 65536)
    return HL_EUNSUPPORTED;
  const uint64_t blocks = (keep * kv_heads * (dim / 8) + 256 * kMoves - 1) / (256 * kMoves);
  if (keep * kv_heads >= (1ull << 32) || !grid_fits(blocks, 256)) return HL_EUNSUPPORTED;
  EvictArgs a = {};
  a.weight = weight_dev, a.lens = lens_dev, a.weight_out = weight_out_dev, a.slots = slots_dev;
  a.lens_out = lens_out_dev;
  a.k = static_cast<const uint16_t*>(from->k_dev), a.v = static_cast<const uint16_t*>(from->v_dev);
  a.k_out = static_cast<uint16_t*>(const_cast<void*>(to->k_dev));
  a.v_out = static_cast<uint16_t*>(const_cast<void*>(to->v_dev));
  a.k_seq = from->k_seq, a.k_token = from->k_token, a.k_head = from->k_head;
  a.v_seq = from->v_seq, a.v_token = from->v_token, a.v_head = from->v_head;
  a.ko_seq = to->k_seq, a.ko_token = to->k_token, a.ko_head = to->k_head;
  a.vo_seq = to->v_seq, a.vo_token = to->v_token, a.vo_head = to->v_head;
  a.batch = batch, a.kv_heads = kv_heads, a.dim = dim, a.tokens = (uint32_t)from->tokens;
  a.keep = (uint32_t)keep, a.recent = (uint32_t)recent;
  const hipStream_t s = (hipStream_t)stream;
  const dim3 items(kv_heads, batch), threads(kThreads);
  // A block that finds few rows moves them itself, which saves a kernel: 256 rows
  // of 128 columns of 8 caches take 9.0 us so and 10.1 with a kernel more, 512
  // 11.6 and 10.4 (but the host has one launch for two, which a captured graph
  // does not gain), 1024 16.9 and 11.5.
  if (from->tokens <= kRow && keep * dim <= kFewMoved) return enqueue(select_kernel<1, true>, items, threads, s, a);
  // As few rows of weights a thread as hold a cache: selecting with 16 takes 13 us
  // longer for 16 x 8 caches of 1024 tokens and of 4096.
  st = from->tokens <= kRow ? enqueue(select_kernel<1, false>, items, threads, s, a)
       : from->tokens <= 4 * kRow ? enqueue(select_kernel<4, false>, items, threads, s, a)
                                  : enqueue(select_kernel<16, false>, items, threads, s, a);
  if (st != HL_OK) return st;
  return enqueue(move_kernel, dim3((uint32_t)blocks, batch), dim3(256), s, a);
}
