// Attention over a shared prefix and own caches held in 4 bits
// (hl_prefix_attention4): the work is cut as for 16 bits, and each step
// multiplies the codes themselves.
//
// A value is base + scale * (code - 8), with a pair (scale, base) for each 32
// columns of a row. The matrix instruction's operand is 16 + code, which is exact in
// bf16 and in f16 and takes a shift and an and-or of a nibble; what is too much of it, 8
// as well, is taken off by products with constants. (128 or 64 + code, where a nibble is
// in place for it, save a shift in four and 4 % of the time of 192 rows on 65536 keys,
// and lose three bits of the sums and of their range.)
//   q.k = sum_g scale_g * (q.(16 + code) - 24 Q_g) + base_g * Q_g,  Q_g the sum of q's group
//   o_d = sum_j w_j (16 + code_jd) - 24 w_j + p_j base_jg,          w_j = p_j * scale_jg
// with w rounded to 16 bits once and the same w in both products, so that its error
// meets a centred code alone. For q.k the rows' pairs are a left operand as they lie in
// memory: times (-24 Q_g, Q_g), split into three bf16 pieces that hold every bit of the
// float32, they give the last two terms, and times a one they put each key's scale
// where the products leave its scores. For o, lane n of 16 has element n of a key's
// pairs: an instruction takes the scale that it needs from that lane, and the eight
// keys of a lane are a left operand whose rows are the elements, for the last term.
//
// Long own caches are bound by the lines of memory that their rows lie in, not by their
// bytes: 16 sequences' tokens of 32 heads on 8 on 16384 own keys (335 MB) take 106 us
// where the 80-byte rows of a token's heads are neighbours, 76 (4.4 TB/s) where a head's
// tokens are. (With 2048 shared ones and lengths up to 16384, 64 heads, the kernel reads
// 388 MB, at 4.7 TB/s, for 189 MB of rows.) Fewer vector instructions a step changed
// neither. Many rows are bound by instructions: each of a block's waves makes operands of
// all codes and pairs for 16 rows of its own (4 x 256 tokens of 32 heads on 4096 shared and
// 512 own keys 265 us, the vector units 61 % and the matrix units 23 % of the time; 192 rows
// on 65536 keys 178). Short calls are bound by a part's start and end.
#include "attention_core.h"
#include "cache4.h"

namespace hl {

template <int G>
constexpr int held4() { return G <= 2 ? 64 : G <= 4 ? 128 : 256; }  // columns of a part's row in the workspace

// A step's keys and values: lane n = lane % 16 of group c = lane / 16 has the
// codes of 8 columns of each group of keys n and 16 + n and their pairs (of 8
// groups, half of them), and of 8 values (key_of) element n of the pairs and the codes
// of 2 columns of each group.
template <int G>
struct Tile4 {
  static constexpr int VW = (G + 3) / 4;
  uint32_t k[2][G];
  u32x4 kr[2];
  uint32_t v[8][VW];
  uint32_t ve[8];
};

template <int G>
struct State4 {
  static constexpr int E = G > 4 ? 2 : 1;
  u32x4 q[G], e[E];  // e: pieces of (minus what is too much of q's sums, Q_g)
  f32x4 o[2 * G];    // o[2g + i][r] is column 32g + 8c + 2r + i
  f32x4 base;        // sums of p times the pairs' element 4c + r
  float mean[G];     // this lane's part of the sum of p * base, of steps with hidden keys
  float m, l, limit;
  uint32_t seen;
};

// Bytes i and j (counted from the first word's) of words w as the low bytes of
// two halves.
template <int N>
__device__ inline uint32_t bytes(const uint32_t (&w)[N], int i, int j) {
  return __builtin_amdgcn_perm(w[j / 4], w[i / 4], 0x0C000C00u | (uint32_t)(4 + j % 4) << 16 | (uint32_t)(i % 4));
}

// N bytes at p, which is aligned to A.
template <int N, int A>
__device__ inline void fetch(void* to, const uint8_t* p) {
  __builtin_memcpy(to, __builtin_assume_aligned(p, A), N);
}

// Keys and values key .. key+31 of `it`; where they may pass its end (LAST), its
// last one again. A row's last loads end within its zeros.
template <int G, bool LAST>
__device__ inline void load4(Tile4<G>& t, const Item& it, uint32_t key) {
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16, left = it.keys - 1 - key;
  const uint8_t* kp = reinterpret_cast<const uint8_t*>(it.k + (uint64_t)key * it.k_token);
  const uint8_t* vp = reinterpret_cast<const uint8_t*>(it.v + (uint64_t)key * it.v_token);
  const uint32_t kb = 2 * it.k_token, vb = 2 * it.v_token;
  // the lanes' offsets are the same for all keys of theirs where none is past the end:
  // what differs is in the scalar part of the address
  const auto k_at = [&](int h, uint32_t byte) {
    return LAST ? kp + (min(16 * h + n, left) * kb + byte) : kp + (uint64_t)(16 * h) * kb + (n * kb + byte);
  };
  const auto v_at = [&](int e, uint32_t byte) {
    return LAST ? vp + (min(key_of(c, e), left) * vb + byte) : vp + (uint64_t)key_of(0, e) * vb + (key_of(c, 0) * vb + byte);
  };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    fetch<4 * G, G % 4 == 0 ? 16 : G % 2 == 0 ? 8 : 4>(t.k[h], k_at(h, 4 * G * c));
    fetch<16, 16>(&t.kr[h], k_at(h, 16 * G + (G > 4 ? c % 2 * 16 : 0)));
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      if constexpr (G < 4) t.kr[h][d] = d < G ? t.kr[h][d] : 0;
      if constexpr (G > 4 && G < 8) t.kr[h][d] = 4 + d < G || c % 2 == 0 ? t.kr[h][d] : 0;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    fetch<4 * Tile4<G>::VW, G % 8 == 0 ? 8 : G % 4 == 0 ? 4 : G % 2 == 0 ? 2 : 1>(t.v[e], v_at(e, G * n));
    t.ve[e] = *reinterpret_cast<const uint16_t*>(v_at(e, 16 * G + min(n, 2u * G - 1) * 2));
  }
}

__device__ inline float low_of(uint32_t pair) { return __builtin_bit_cast(float, pair << 16); }
__device__ inline float high_of(uint32_t pair) { return __builtin_bit_cast(float, pair & 0xFFFF0000u); }

// x of lane N of each 16.
template <int N>
__device__ inline float from_lane(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), 0x150 + N, 0xF, 0xF, true));
}

// p[e] times s[e] of lane N of each 16, in one instruction each: two wait states after
// s and p have been written are what reading another lane takes.
template <int N>
__device__ inline void times_lane(float (&x)[8], const float (&s)[8], const float (&p)[8]) {
#define HL_TIMES(o, i, j) "v_mul_f32_dpp %" o ", %" i ", %" j " row_newbcast:%24 row_mask:0xf bank_mask:0xf\n\t"
  asm("s_nop 1\n\t" HL_TIMES("0", "8", "16") HL_TIMES("1", "9", "17") HL_TIMES("2", "10", "18") HL_TIMES("3", "11", "19")
          HL_TIMES("4", "12", "20") HL_TIMES("5", "13", "21") HL_TIMES("6", "14", "22") HL_TIMES("7", "15", "23")
      : "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3]), "=&v"(x[4]), "=&v"(x[5]), "=&v"(x[6]), "=&v"(x[7])
      : "v"(s[0]), "v"(s[1]), "v"(s[2]), "v"(s[3]), "v"(s[4]), "v"(s[5]), "v"(s[6]), "v"(s[7]), "v"(p[0]), "v"(p[1]),
        "v"(p[2]), "v"(p[3]), "v"(p[4]), "v"(p[5]), "v"(p[6]), "v"(p[7]), "n"(N));
#undef HL_TIMES
}

// Keeps operands in their registers up to here, past products_end.
template <int N>
__device__ inline void keep(const u32x4 (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" ::"v"(v[i]));
}

// One step: scores of 32 keys, their weights, and the weighted values. EDGE:
// some query may not see some of the keys, whatever their rows hold.
template <class T, int G, bool EDGE>
__device__ inline void step4(State4<G>& st, const Tile4<G>& t, const Codes<T>& kf, const Codes<__bf16>& vf,
                             const AttentionArgs& a, const Item& it, uint32_t key, uint32_t wave_row) {
  using S = State4<G>;
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16;
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  f32x4 s[2];
  constexpr int KSET = G > 4 ? 2 : G;  // groups whose products follow each other
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u32x4 pairs[1] = {t.kr[h]};
#pragma unroll
    for (int g0 = 0; g0 < G; g0 += KSET) {
      u32x4 codes[KSET], one[KSET];
#pragma unroll
      for (int i = 0; i < KSET; ++i) {
        const int g = g0 + i < G ? g0 + i : G - 1;
        const uint32_t p01 = bytes(t.k[h], g, G + g), p23 = bytes(t.k[h], 2 * G + g, 3 * G + g);
        codes[i] = u32x4{kf.template pair<0>(p01), kf.template pair<4>(p01), kf.template pair<0>(p23), kf.template pair<4>(p23)};
        one[i] = u32x4{0, 0, 0, 0};
        one[i][g % 4] = c == (uint32_t)(g / 4) ? 0x3F80u : 0;
        asm volatile("" : "+v"(codes[i]));
      }
      __builtin_amdgcn_sched_barrier(0);
      f32x4 part[KSET], scale[KSET];
#pragma unroll
      for (int i = 0; i < KSET; ++i) {
        scale[i] = mfma<__bf16>(pairs[0], one[i], zero);
        part[i] = mfma<T>(codes[i], st.q[g0 + i < G ? g0 + i : G - 1], zero);
      }
      if (g0 == 0) {
        s[h] = mfma<__bf16>(pairs[0], st.e[0], zero);
        if constexpr (S::E == 2) s[h] = mfma<__bf16>(pairs[0], st.e[1], s[h]);
      }
      products_end();
      keep(codes), keep(one), keep(pairs);
#pragma unroll
      for (int i = 0; i < KSET; ++i)
        if (g0 + i < G) {
#pragma unroll
          for (int r = 0; r < 4; ++r) s[h][r] = fmaf(scale[i][r], part[i][r], s[h][r]);
        }
    }
  }
  float p[8];
  if constexpr (EDGE) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (key + key_of(c, e) >= st.seen) s[e / 4][e % 4] = -INFINITY;
  }
  if (it.scores) {
    const uint32_t row = here(wave_row + n);  // nothing of this is formed in a call without weights
    if (row < it.rows) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<f32x4*>(it.scores + (uint64_t)row * a.score_stride + key + 16 * h + 4 * c) = s[h] * a.scale2;
    }
  }
  float top = -INFINITY;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = fmaxf(top, s[e / 4][e % 4]);
  top *= a.scale2;
  // The maximum need only be near the true one, as for 16 bits.
  if (__any(top > st.limit)) {
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const bool had = st.limit != -INFINITY;
    const float was = st.m;
    const float now = had ? fmaxf(was, top) : top;
    if (now != -INFINITY) {
      const float f = had ? __builtin_amdgcn_exp2f(was - now) : 0.0f;
      st.m = now, st.limit = now + kSlack;
      st.l *= f;
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) st.o[i] *= f;
      st.base *= f;
#pragma unroll
      for (int g = 0; g < G; ++g) st.mean[g] *= f;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = __builtin_amdgcn_exp2f(fmaf(s[e / 4][e % 4], a.scale2, -st.m));
    st.l += p[e];
  }
  // w is rounded to bf16, whose range holds any scale. Where the output has 11
  // bits, what the rounding leaves is a second operand.
  constexpr int PIECES = std::is_same<T, __bf16>::value ? 1 : 2;
  constexpr int SET = G % 2 || G > 3 ? 1 : 2;  // groups whose products follow each other
  float scales[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) scales[e] = low_of(t.ve[e]);
  // rounds eight numbers to operands
  const auto round = [](u32x4* to, const float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      to[0][j] = pack<__bf16>(x[2 * j], x[2 * j + 1]);
      if constexpr (PIECES == 2) to[1][j] = pack<__bf16>(x[2 * j] - low_of(to[0][j]), x[2 * j + 1] - high_of(to[0][j]));
    }
#pragma unroll
    for (int y = 0; y < PIECES; ++y) asm volatile("" : "+v"(to[y]));
  };
  constexpr uint32_t minus = Codes<__bf16>::LESS;
  u32x4 less[1] = {u32x4{minus, minus, minus, minus}};
  asm volatile("" : "+v"(less[0]));
  // rows whose keys all queries see: p times the pairs' elements, for the bases
  constexpr int BASES = EDGE ? 0 : 1;
  u32x4 pairs[1], pw[PIECES];
  if constexpr (!EDGE) {
#pragma unroll
    for (int j = 0; j < 4; ++j) pairs[0][j] = t.ve[2 * j] | t.ve[2 * j + 1] << 16;
    asm volatile("" : "+v"(pairs[0]));
    round(&pw[0], p);
  }
  each<G / SET>([&](auto nth) {
    constexpr int g0 = decltype(nth)::value * SET;
    u32x4 codes[2 * SET], w[SET * PIECES];
    each<SET>([&](auto mth) {
      constexpr int i = decltype(mth)::value, g = g0 + i;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t both = __builtin_amdgcn_perm(t.v[2 * j + 1][g / 4], t.v[2 * j][g / 4],
                                                    0x0C000C00u | (uint32_t)(4 + g % 4) << 16 | (uint32_t)(g % 4));
        codes[2 * i][j] = vf.pair<0>(both), codes[2 * i + 1][j] = vf.pair<4>(both);
      }
      asm volatile("" : "+v"(codes[2 * i]), "+v"(codes[2 * i + 1]));
      float x[8];
      times_lane<2 * g>(x, scales, p);
      if constexpr (EDGE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // a row that the query does not see may hold anything
          const bool sees = key + key_of(c, e) < st.seen;
          const float b = fmaf(p[e], from_lane<2 * g + 1>(scales[e]), st.mean[g]);
          x[e] = sees ? x[e] : 0.0f;
          st.mean[g] = sees ? b : st.mean[g];
        }
      }
      round(&w[i * PIECES], x);
    });
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < SET; ++i)
#pragma unroll
      for (int y = 0; y < PIECES; ++y) {
        const u32x4 x = w[i * PIECES + y];
        f32x4 &even = st.o[2 * (g0 + i)], &odd = st.o[2 * (g0 + i) + 1];
        even = mfma<__bf16>(codes[2 * i], x, even), odd = mfma<__bf16>(codes[2 * i + 1], x, odd);
        even = mfma<__bf16>(less[0], x, even), odd = mfma<__bf16>(less[0], x, odd);
      }
    if constexpr (g0 == 0 && BASES) {
#pragma unroll
      for (int y = 0; y < PIECES; ++y) st.base = mfma<__bf16>(pairs[0], pw[y], st.base);
    }
    products_end();
    keep(codes), keep(w), keep(less);
    if constexpr (g0 == 0 && BASES) keep(pairs), keep(pw);
  });
}

// Starts a wave's state: its queries, from row `wave_row` of the item's head.
template <class T, int G>
__device__ inline void begin4(State4<G>& st, const AttentionArgs& a, const Item& it, uint32_t wave_row) {
  using S = State4<G>;
  typedef T pair __attribute__((ext_vector_type(2)));
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16;
  st.m = 0.0f, st.l = 0.0f, st.limit = -INFINITY;
  const uint32_t row = min(wave_row + n, it.rows - 1), tok = row / a.share;
  st.seen = seen_by(a, it, row);
  const uint16_t* q = it.q + ((uint64_t)tok * a.heads + row % a.share) * (32 * G);
  float sum[G], less[G];
  st.base = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int g = 0; g < G; ++g) {
    st.o[2 * g] = st.o[2 * g + 1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    st.mean[g] = 0.0f;
    const u32x4 x = (*reinterpret_cast<const u32x4*>(q + 32 * g + 8 * c) & a.q_and) ^ a.q_xor;
    float all = 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t two = x[j];  // an element itself is not what a bit cast takes
      const pair y = __builtin_bit_cast(pair, two);
      all += (float)y[0] + (float)y[1];
    }
    sum[g] = over_lanes(all), less[g] = -24.0f * sum[g];
    // the order in which a pair of bytes gives its codes
#pragma unroll
    for (int j = 0; j < 4; ++j)
      st.q[g][j] = __builtin_amdgcn_perm(x[j / 2 * 2 + 1], x[j / 2 * 2], j % 2 ? 0x07060302u : 0x05040100u);
  }
  // pieces 0, 1 and 2 of a float32, of 8 bits each
  const auto piece = [](float x, uint32_t i) {
    const float p0 = (float)(__bf16)x, p1 = (float)(__bf16)(x - p0), p2 = x - p0 - p1;
    return i == 0 ? p0 : i == 1 ? p1 : i == 2 ? p2 : 0.0f;
  };
#pragma unroll
  for (int e = 0; e < S::E; ++e)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t part = S::E == 1 ? c : 2 * e + c / 2;
      const auto of = [&](const float (&v)[G]) {
        float x = j < G ? v[j < G ? j : 0] : 0.0f;
        if constexpr (S::E == 2) {
          float y = 4 + j < G ? v[4 + j < G ? 4 + j : 0] : 0.0f;
          asm volatile("" : "+v"(x), "+v"(y));  // two registers, no array in memory
          x = c % 2 ? y : x;
        }
        return piece(x, part);
      };
      st.e[e][j] = pack<__bf16>(of(less), of(sum));
    }
}

// A wave's share of an item's keys [.., k1) for its rows: 32 from `key` on, and
// again every `stride`. Loads are a step ahead, and there are always as many of them
// (at the end, of the last step again): waits count them.
template <class T, int G>
__device__ inline void keys4(State4<G>& st, const AttentionArgs& a, const Item& it, uint32_t wave_row, uint32_t key,
                             uint32_t k1, uint32_t stride) {
  const Codes<T> kf;
  const Codes<__bf16> vf;
  const uint32_t all = seen_by(a, it, wave_row), most = seen_by(a, it, wave_row + 15), end = min(k1, most);
  const uint32_t whole = min(end, all);  // steps that end here or before hide no key
  const auto run = [&](const Tile4<G>& t) __attribute__((always_inline)) {
    step4<T, G, false>(st, t, kf, vf, a, it, key, wave_row);
    key += stride;
  };
  if (key + kStep <= whole) {
    const uint32_t last = key + (whole - kStep - key) / stride * stride;
    if constexpr (G > 4) {  // several steps' rows do not fit the registers
#pragma unroll 1
      while (key <= last) {
        Tile4<G> t;
        load4<G, false>(t, it, key);
        run(t);
      }
    } else {
      Tile4<G> t0, t1;
      load4<G, false>(t0, it, key);
      while (true) {
        load4<G, false>(t1, it, min(key + stride, last));
        run(t0);
        if (key > last) break;
        load4<G, false>(t0, it, min(key + stride, last));
        run(t1);
        if (key > last) break;
      }
    }
  }
#pragma unroll 1
  for (; key < end; key += stride) {
    Tile4<G> t;
    load4<G, true>(t, it, key);
    step4<T, G, true>(st, t, kf, vf, a, it, key, wave_row);
  }
}

// Columns 32g + 8c .. of a wave's query n, eight for each group: out(first column, four of them).
template <int G, class Out>
__device__ inline void columns4(const State4<G>& st, Out out) {
  const uint32_t n = lane_id() % 16, c = lane_id() / 16;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    const float shift = over_lanes(st.mean[g]) + __shfl(st.base[(2 * g + 1) % 4], (2 * g + 1) / 4 * 16 + n);
    const f32x4 x = st.o[2 * g], y = st.o[2 * g + 1];
    out(32 * g + 8 * c, f32x4{x[0] + shift, y[0] + shift, x[1] + shift, y[1] + shift});
    out(32 * g + 8 * c + 4, f32x4{x[2] + shift, y[2] + shift, x[3] + shift, y[3] + shift});
  }
}

// Adds the results that WAVES waves have of the same 16 rows and calls
// out(row, d, o, m, l) for four columns from d on of each of the first `rows`.
template <int G, int WAVES, class Out>
__device__ inline void add_waves4(const State4<G>& st, uint32_t rows, float* lds, Out out) {
  constexpr uint32_t D = 32 * G;
  const uint32_t lane = lane_id(), n = lane % 16, c = lane / 16;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  float* lds_ml = lds + WAVES * 16 * (D + 4);
  const float sum = over_lanes(st.l);
  const uint32_t at = here(wave * 16 + n);  // formed here: no register holds it through the loops
  if (c == 0) lds_ml[2 * at] = st.limit != -INFINITY || sum != sum ? st.m : -INFINITY, lds_ml[2 * at + 1] = sum;
  columns4<G>(st, [&](uint32_t d, f32x4 o) { *reinterpret_cast<f32x4*>(lds + (uint64_t)at * (D + 4) + d) = o; });
  __syncthreads();
  for (uint32_t x = here(threadIdx.x); x < rows * (D / 4); x += WAVES * 64) {
    const uint32_t row = x / (D / 4), d = x % (D / 4) * 4;
    float m = -INFINITY, l = 0.0f;
    for (uint32_t k = 0; k < WAVES; ++k) m = fmaxf(m, lds_ml[2 * (row + 16 * k)]);
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t k = 0; k < WAVES; ++k) {
      const uint32_t from = row + 16 * k;
      const float mk = lds_ml[2 * from];
      const float f = mk == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mk - m);
      o += f * *reinterpret_cast<const f32x4*>(lds + (uint64_t)from * (D + 4) + d);
      l += f * lds_ml[2 * from + 1];
    }
    out(row, d, o, m, l);
  }
}

// Keys [k0, k1) of a narrow item by one block, whose waves take different keys;
// writes the part at `slot`.
template <class T, int G>
__device__ inline void narrow_part4(const AttentionArgs& a, const Item& it, uint32_t k0, uint32_t k1, uint32_t slot,
                                    float* lds) {
  constexpr uint32_t H = held4<G>();
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  State4<G> st;
  begin4<T, G>(st, a, it, 0);
  keys4<T, G>(st, a, it, 0, k0 + kStep * wave, k1, kUnit);
  float* po = a.narrow_o + (uint64_t)slot * a.narrow_rows * H;
  float* pml = a.narrow_ml + (uint64_t)slot * a.narrow_rows * 2;
  add_waves4<G, kWaves>(st, it.rows, lds, [&](uint32_t row, uint32_t d, f32x4 o, float m, float l) {
    *reinterpret_cast<f32x4*>(po + (uint64_t)row * H + d) = o;
    if (d == 0) pml[2 * row] = m, pml[2 * row + 1] = l;
  });
  __syncthreads();
}

// Keys [k0, k1) of a wide item by one block, whose waves take different rows;
// each writes its rows of the part at `slot`.
template <class T, int G>
__device__ inline void wide_part4(const AttentionArgs& a, const Item& it, uint32_t k0, uint32_t k1, uint32_t slot) {
  constexpr uint32_t H = held4<G>();
  const uint32_t n = lane_id() % 16, c = lane_id() / 16;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wave_row = it.row0 + wave * 16;
  if (wave_row >= it.rows) return;
  State4<G> st;
  begin4<T, G>(st, a, it, wave_row);
  keys4<T, G>(st, a, it, wave_row, k0, k1, kStep);
  float* po = a.wide_o + (uint64_t)slot * a.wide_rows * H;
  float* pml = a.wide_ml + (uint64_t)slot * a.wide_rows * 2;
  const float sum = over_lanes(st.l);
  const uint32_t row = here(wave * 16 + n);
  const bool in = it.row0 + row < it.rows;
  if (in && c == 0)
    pml[2 * row] = st.limit != -INFINITY || sum != sum ? st.m : -INFINITY, pml[2 * row + 1] = sum;
  columns4<G>(st, [&](uint32_t d, f32x4 o) {
    if (in) *reinterpret_cast<f32x4*>(po + (uint64_t)row * H + d) = o;
  });
}

// WIDE: whether the call has wide items. A wave has 16 rows of them: two such tiles (128
// columns) would not fit its registers.
template <class T, int G, bool WIDE>
__global__ void __launch_bounds__(kThreads, 2) parts4_kernel(AttentionArgs a) {
  __shared__ __attribute__((aligned(16))) float lds[kWaves * 16 * (32 * G + 4) + kWaves * 16 * 2];
  const OwnLine line = a.own.tokens ? own_line(a, 0) : OwnLine{0, 0, 0};
  const Lines l = lines_of(a, own_units_before(a, line, a.batch));
  const uint32_t xcd = blockIdx.x % 8, nth = blockIdx.x / 8, wide = l.wide_blocks / 8;
  if (WIDE && nth < wide) {
    const uint32_t taker = xcd * wide + nth;
    if (taker >= l.wide.takers) return;
    const uint32_t end = l.wide.first(taker + 1);
    for (uint32_t u = l.wide.first(taker); u < end;) {
      const Place p = place_of<true>(a, line, l, u);
      const uint32_t take = min(p.each - p.in, end - u);
      wide_part4<T, G>(a, p.it, p.in * kUnit, (p.in + take) * kUnit, taker + p.item);
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
    narrow_part4<T, G>(a, p.it, p.in * kUnit, (p.in + take) * kUnit, taker + p.item, lds);
    u += take;
  }
}

// A whole sequence and key head by one block, over the prefix and its own keys.
// Rows of a head: at most 16.
template <class T, int G>
__global__ void __launch_bounds__(kSoloWaves * 64, 2) solo4_kernel(AttentionArgs a) {
  __shared__ __attribute__((aligned(16))) float lds[kSoloWaves * 16 * (32 * G + 4) + kSoloWaves * 16 * 2];
  __shared__ float s_ml[32];
  const uint32_t head = blockIdx.x, b = blockIdx.y, rows = a.queries * a.share;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  constexpr uint32_t stride = kSoloWaves * kStep;
  Item own = {};
  if (a.own.tokens) own = own_item(a, b, head, 0);
  Item pre = prefix_item(a, head, 0);
  pre.q += (uint64_t)b * a.queries * a.heads * a.dim, pre.rows = rows;
  State4<G> st;
  begin4<T, G>(st, a, pre, 0);  // every row sees the whole prefix
  if (pre.keys) keys4<T, G>(st, a, pre, 0, kStep * wave, pre.keys, stride);
  if (a.own.tokens) {
    st.seen = seen_by(a, own, lane_id() % 16);
    // the waves that had a step of the prefix less than the others begin
    keys4<T, G>(st, a, own, 0, kStep * ((wave - (pre.keys + kStep - 1) / kStep) % kSoloWaves), own.keys, stride);
  }
  const uint64_t first = (uint64_t)b * a.queries * a.heads + (uint64_t)head * a.share;
  add_waves4<G, kSoloWaves>(st, rows, lds, [&](uint32_t row, uint32_t d, f32x4 o, float m, float l) {
    const uint64_t at = first + (uint64_t)(row / a.share) * a.heads + row % a.share;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    *reinterpret_cast<u32x2*>(a.out + at * (32 * G) + d) =
        u32x2{pack<T>(o[0] * inv, o[1] * inv), pack<T>(o[2] * inv, o[3] * inv)};
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

// ------------------------------------------------------------------- host

template <class T, int G>
static hl_status run4(const AttentionPlan& pl, hl_dtype dtype, hipStream_t s) {
  const AttentionArgs& a = pl.a;
  if (pl.solo) return enqueue(solo4_kernel<T, G>, dim3(a.kv_heads, a.batch), dim3(kSoloWaves * 64), s, a);
  const dim3 blocks(a.blocks), threads(kThreads);
  const hl_status st = pl.wide ? enqueue(parts4_kernel<T, G, true>, blocks, threads, s, a)
                               : enqueue(parts4_kernel<T, G, false>, blocks, threads, s, a);
  return st != HL_OK ? st : attention_join(pl, dtype, s);
}

template <class T>
static hl_status run_groups4(const AttentionPlan& pl, hl_dtype dtype, hipStream_t s) {
  switch (pl.a.dim / 32) {
    case 1: return run4<T, 1>(pl, dtype, s);
    case 2: return run4<T, 2>(pl, dtype, s);
    case 3: return run4<T, 3>(pl, dtype, s);
    case 4: return run4<T, 4>(pl, dtype, s);
    case 5: return run4<T, 5>(pl, dtype, s);
    case 6: return run4<T, 6>(pl, dtype, s);
    case 7: return run4<T, 7>(pl, dtype, s);
    default: return run4<T, 8>(pl, dtype, s);
  }
}

}  // namespace hl

using namespace hl;

extern "C" size_t hl_attention4_workspace_bytes(const hl_attention* attention, int with_weights) {
  AttentionPlan pl;
  if (!attention || attention->dim % 32) return 0;
  return attention_plan(attention, with_weights != 0, true, &pl) == HL_OK ? pl.bytes : 0;
}

extern "C" hl_status hl_prefix_attention4(const hl_attention* attention, const void* q_dev, const int32_t* lens_dev,
                                          void* out_dev, float* lse_dev, const float* weight_in_dev,
                                          float* weight_out_dev, void* workspace_dev, size_t workspace_bytes,
                                          void* stream) {
  if (!attention || attention->dim % 32) return HL_EINVAL;
  AttentionPlan pl;
  const hl_status st = attention_setup(attention, q_dev, lens_dev, out_dev, lse_dev, weight_in_dev, weight_out_dev,
                                       workspace_dev, workspace_bytes, true, &pl);
  if (st != HL_OK) return st;
  return attention->dtype == HL_BF16 ? run_groups4<__bf16>(pl, HL_BF16, (hipStream_t)stream)
                                     : run_groups4<_Float16>(pl, HL_F16, (hipStream_t)stream);
}
