// Attention over a cache held in 4 bits (gfx950), and the selection of the blocks that it reads.
//
//   out = sum_s p_s v_s,  p = softmax_s(q . k_s / sqrt(hd)),  over all slots that a token sees or those of its listed blocks
//
// The query heads of a KV head and the sequence's new tokens are the rows of two products on the matrix cores.  Queries and results of this
// library are fp32, and a cache read in 4 bits should lose nothing beyond its rounding: both products take the cache's values as they are and
// the fp32 operand as a sum of short terms that hold all 24 bits.
//   S = K Q^T: on the product of scaled 4-bit and 6-bit numbers, which takes K's codes and scale bytes unchanged and a slot's 128 channels at once.  A tile
//     of 16 slots is the A operand, lane l holding channels hd / 4 (l / 16) .. of slot l % 16: a quarter of a slot's codes, under one scale; a
//     query is five terms of 6 bits (16 x 16 x 128 products in the 16 cycles of 16 x 16 x 32 bf16 ones).  A lane then holds the scores of slots
//     4 (l / 16) + i of row l % 16,
//   O^T = V^T P^T: which is where the B operand of the second product wants them: elements 4 t + i of lane group g are slot 4 g + i of
//     tile t.  Here the sum runs over slots, each with a scale of its own, so that V is made bf16 (exactly; one conversion gives two numbers, the
//     scale included) and the weights are three bf16 terms.  The A operand needs eight slots of a channel side by side: lane l takes channels
//     hd / 16 (l % 16) .. of those slots, pairs of slots meeting in a register by one permutation.
// The running maximum, sum and result of a row stay in the lanes of its column; nothing passes through LDS until a wave's share of
// the context is done.
// Bound: a single token by the chain of one step a wave (2048 slots of 8 KV heads 6.9 us and 3.7 of the join; 0.3 us of bytes), long contexts with many
// rows by the instructions of a step on two waves a SIMD: 48 products of 16 cycles, 20 of the other kind and some 240 vector instructions for 32 slots of 32 rows.
// Four sequences of 6 tokens at 4096 .. 32768 slots of 8 KV heads 30.6 us in a graph (34 with K as bf16 too, in three terms), sixteen of 16 tokens at 512 .. 1067 on 4
// heads, 112 rows each, 18.9 (20.3); a large bf16 product's rate would allow 13 and 6.  Over lists every token has workgroups of its own, which read and convert a
// block again that several tokens list: 32 blocks for each of those four sequences' tokens 24.3 us, 24 for each of sixteen sequences' 16 tokens, seven heads to a KV
// head, 69.
#include "launch_common.hpp"
#include "lane_ops.hpp"

#include <string.h>

namespace es {

constexpr float kLowest = -3.4028235e38f;
constexpr int kStep = 32;        // slots of a wave's step

__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float unit, std::integral_constant<int, 0>) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0)); }
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float unit, std::integral_constant<int, 1>) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1)); }
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float unit, std::integral_constant<int, 2>) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2)); }
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float unit, std::integral_constant<int, 3>) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3)); }
template <int I>
__device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float unit) {
  return bf16_pair(codes, unit, std::integral_constant<int, I>{});
}
__device__ __forceinline__ float unit_of(uint32_t scale) { return __uint_as_float(scale << 23); }  // 255: infinity, of which the conversion makes NaN

// One workgroup's place.  Without lists: a chunk of an entry's steps and RT tiles of its rows; with them, a token and a chunk of its list.
template <bool LIST, int RT>
struct KvqPlace {
  int e, h, l, c, row0, rows, len, old;  // entry, KV head, layer, chunk; first row and how many; slots that any row sees; that all do but for
                                         // their own and those after
  int n_tok;                             // token of the first row
  __device__ __forceinline__ explicit KvqPlace(const KvqArgs& a) {
    e = 0;
#pragma unroll
    for (int i = 1; i < kMaxCols; ++i) e += (int)blockIdx.x >= a.first_wg[i];
    const KvqEntry& en = a.entry[e];
    const int w = blockIdx.x - a.first_wg[e];
    h = blockIdx.y;
    l = blockIdx.z;
    if (LIST) {
      n_tok = w / en.chunks;
      c = w % en.chunks;
      row0 = n_tok * a.group;
      rows = a.group;
      old = en.len - en.n + n_tok;
      len = old + 1;
    } else {
      const int tile = w % en.tiles;
      c = w / en.tiles;
      row0 = tile * 16 * RT;
      rows = min(16 * RT, en.n * a.group - row0);
      n_tok = token_of(a, row0);
      old = en.len - en.n + n_tok;
      len = en.len - en.n + token_of(a, row0 + rows - 1) + 1;
    }
  }
  static __device__ __forceinline__ int token_of(const KvqArgs& a, int row) { return (int)(((float)row + 0.5f) * a.inv_group); }  // row < 128: off by far less than half a step
  __device__ __forceinline__ size_t cache_row(const KvqArgs& a) const {
    return (((size_t)l * a.n_seqs + a.entry[e].seq) * a.heads + h) * (size_t)a.max_slots;
  }
};

// The (layer, sequence, KV head)'s arrays.
struct KvqRow {
  const uint8_t *kc, *vc, *ks, *vs;
};

// Codes and scales of a step of 32 slots from s on, as the lane needs them.  Slots past the last fetch the last one.
template <int HD>
struct KvqStep {
  static constexpr int KW = HD / 32;  // words of K codes of a lane and tile: 8 channels each; scales of a slot
  typedef uint32_t kword __attribute__((ext_vector_type(KW)));
  uint32_t k[2][KW], ks[2], v[2][4];
  kword vs[2];  // the scales of the lane's four slots of a tile side by side
  template <class T>
  static __device__ __forceinline__ T fetch(const uint8_t* p) {  // scales may lie anywhere
    T x;
    __builtin_memcpy(&x, p, sizeof(T));
    return x;
  }
  __device__ __forceinline__ void set_k(int t, kword w) {
#pragma unroll
    for (int i = 0; i < KW; ++i) k[t][i] = w[i];
  }
  __device__ __forceinline__ void load_k(const KvqRow& row, int s, int len) {
    const uint32_t lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15, own = g * (HD / 8), own_scale = HD == 128 ? g : g >> 1;
    if (s + kStep <= len) {
      const uint8_t *kc = row.kc + (size_t)s * (HD / 2), *sc = row.ks + (size_t)s * KW;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        set_k(t, *reinterpret_cast<const kword*>(kc + (c * (HD / 2) + own) + t * 16 * (HD / 2)));
        ks[t] = (sc + (c * KW + own_scale))[t * 16 * KW];
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t slot = min((uint32_t)s + 16 * t + c, (uint32_t)len - 1);
        set_k(t, *reinterpret_cast<const kword*>(row.kc + (slot * (HD / 2) + own)));
        ks[t] = row.ks[slot * KW + own_scale];
      }
    }
  }
  __device__ __forceinline__ void load_v(const KvqRow& row, int s, int len) {
    typedef typename std::conditional<HD == 128, uint32_t, uint16_t>::type part;  // a lane's channels; a slot's scales
    const uint32_t lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    if (s + kStep <= len) {
      const uint8_t *vc = row.vc + (size_t)s * (HD / 2), *sc = row.vs + (size_t)s * KW;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint8_t* vp = vc + (4 * g * (HD / 2) + c * sizeof(part)) + t * 16 * (HD / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[t][i] = *reinterpret_cast<const part*>(vp + i * (HD / 2));
        vs[t] = fetch<kword>(sc + 4 * g * KW + t * 16 * KW);
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        part sc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t slot = min((uint32_t)s + 16 * t + 4 * g + i, (uint32_t)len - 1);
          v[t][i] = *reinterpret_cast<const part*>(row.vc + (slot * (HD / 2) + c * (uint32_t)sizeof(part)));
          sc[i] = fetch<part>(row.vs + slot * KW);
        }
        vs[t] = __builtin_bit_cast(kword, sc);
      }
    }
  }
  // The scale of the lane's channels of V in slot i of tile t.
  __device__ __forceinline__ uint32_t v_scale(int t, int i) const {
    const int c = threadIdx.x & 15;
    if constexpr (HD == 128) return __builtin_amdgcn_ubfe(vs[t][i], 8 * (c >> 2), 8);
    else return __builtin_amdgcn_ubfe(vs[t][i / 2], 16 * (i % 2) + 8 * (c >> 3), 8);
  }
};

// A row's query in the lane's quarter of the channels, scaled, as kTerms times 32 E2M3 numbers (head_dim 64: sixteen, and zeros), the scale of a
// term 2^-5 of that of the one before.  The first one's makes the largest magnitude of the 32 2 .. 4, where a place is worth a quarter: what a
// term leaves is an eighth at most, and 4 to the next one; what the last leaves, 2^-24 of the largest magnitude.  units: the scales' bytes (255,
// NaN, where a channel is not finite).
constexpr int kTerms = 5;
typedef uint32_t u32x6 __attribute__((ext_vector_type(6)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x6 __attribute__((ext_vector_type(6)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
template <int HD, bool LIST, int RT>
__device__ __forceinline__ void query_terms(const KvqArgs& a, const KvqPlace<LIST, RT>& p, int row, u32x6 (&code)[kTerms], uint32_t (&unit)[kTerms]) {
  const int g = (threadIdx.x & 63) >> 4, r = p.row0 + row, tok = p.token_of(a, r);
  const f32x4* src = reinterpret_cast<const f32x4*>(a.q + p.l * ((size_t)a.n_tokens * a.Hq * HD) + ((size_t)(a.entry[p.e].q_first + tok) * a.Hq + p.h * a.group + (r - tok * a.group)) * HD + g * (HD / 4));
  f32x16 even = {}, odd = {};  // as the conversion takes them
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < HD / 16; ++i) {
    const f32x4 v = src[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x = v[j] * a.scale;
      top = max(top, __float_as_uint(x) & 0x7FFFFFFFu);
      if (j % 2) odd[2 * i + j / 2] = x;
      else even[2 * i + j / 2] = x;
    }
  }
  const uint32_t first = max(top >> 23, 22u) - 1;  // the largest magnitude becomes 2 .. 4; the last scale is a normal number
#pragma unroll
  for (int t = 0; t < kTerms; ++t) {
    const float u = __uint_as_float((first - 5 * t) << 23);
    code[t] = __builtin_amdgcn_cvt_scalef32_2xpk16_fp6_f32(even, odd, u);
    unit[t] = top >= 0x7F800000u ? 255u : first - 5 * t;
    if (t + 1 == kTerms) break;
    const auto taken = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(code[t], u);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      even[i] -= taken[2 * i];
      odd[i] -= taken[2 * i + 1];
    }
  }
}

// The queries of RT tiles of 16 rows as B operands: split by one wave, held by all; rows past the last are the last one's.  FOLD (four rows at most):
// column 4 t + r of the first operand is term t of row r, column r of the second the last term, its other columns are zero.
template <int HD, bool FOLD, int RT>
struct KvqQueries {
  static constexpr int N = FOLD ? 2 : kTerms;
  u32x6 q[RT][N];
  uint32_t unit[RT][2];  // four to a word (FOLD: one)
  struct Stage {
    u32x6 q[RT][FOLD ? 1 : kTerms][FOLD ? 1 : 64];
    uint32_t unit[RT][2][FOLD ? 1 : 64];
  };
  template <int NW, bool LIST>
  __device__ __forceinline__ void load(const KvqArgs& a, const KvqPlace<LIST, RT>& p, Stage& stage) {
    const int lane = threadIdx.x & 63, n = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    u32x6 c[kTerms];
    uint32_t u[kTerms];
    if constexpr (FOLD) {
      query_terms<HD>(a, p, min(n & 3, p.rows - 1), c, u);
      const int t = n >> 2;
      q[0][0] = t == 0 ? c[0] : t == 1 ? c[1] : t == 2 ? c[2] : c[3];
      unit[0][0] = t == 0 ? u[0] : t == 1 ? u[1] : t == 2 ? u[2] : u[3];
      q[0][1] = t == 0 ? c[4] : u32x6{};
      unit[0][1] = u[4];
    } else {
      if (wave < RT) {
        query_terms<HD>(a, p, min(wave * 16 + n, p.rows - 1), c, u);
#pragma unroll
        for (int t = 0; t < kTerms; ++t) stage.q[wave][t][lane] = c[t];
        stage.unit[wave][0][lane] = u[0] | u[1] << 8 | u[2] << 16 | u[3] << 24;
        stage.unit[wave][1][lane] = u[4];
      }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < RT; ++r) {
#pragma unroll
        for (int t = 0; t < kTerms; ++t) q[r][t] = stage.q[r][t][lane];
        unit[r][0] = stage.unit[r][0][lane];
        unit[r][1] = stage.unit[r][1][lane];
      }
    }
  }
  // += K Q^T of 16 slots: a lane's 32 codes of a slot, and their scale
  template <int I, int U, int BYTE>
  __device__ __forceinline__ void add(f32x4& x, int r, i32x8 k, uint32_t k_unit) const {
    const i32x6 b = __builtin_bit_cast(i32x6, q[r][I]);
    const i32x8 wide = __builtin_shufflevector(b, b, 0, 1, 2, 3, 4, 5, -1, -1);
    x = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k, wide, x, 4, 2, 0, (int)k_unit, BYTE, (int)unit[r][U]);
  }
  __device__ __forceinline__ void scores(f32x4 (&x)[RT][2], const i32x8 (&k)[2], const uint32_t (&k_unit)[2]) const {
    const auto term = [&](auto i, auto u, auto byte) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < 2; ++t) add<decltype(i)::value, decltype(u)::value, decltype(byte)::value>(x[r][t], r, k[t], k_unit[t]);
    };
    // the smallest term first; products on one accumulator 2 RT apart
    if constexpr (FOLD) {
      term(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{}, std::integral_constant<int, 0>{});
      term(std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{});
    } else {
      term(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{}, std::integral_constant<int, 0>{});
      term(std::integral_constant<int, 3>{}, std::integral_constant<int, 0>{}, std::integral_constant<int, 3>{});
      term(std::integral_constant<int, 2>{}, std::integral_constant<int, 0>{}, std::integral_constant<int, 2>{});
      term(std::integral_constant<int, 1>{}, std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{});
      term(std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{});
    }
  }
};

__device__ __forceinline__ float fold_terms(float x) {  // over columns n, n + 4, n + 8, n + 12: the same bits in all of them
  x += dpp<0x128>(x);  // row_ror:8
  return x + dpp<0x124>(x);  // row_ror:4
}
__device__ __forceinline__ float over_groups_max(float x) {
  const auto f = [](float u, float v) { return fmaxf(u, v); };
  return across<true>(across<false>(x, f), f);
}
__device__ __forceinline__ float over_groups_sum(float x) {
  const auto f = [](float u, float v) { return u + v; };
  return across<true>(across<false>(x, f), f);
}

// The running softmax of a wave's share of a row tile: row l % 16 (FOLD: l % 4) in lane l.  Weights are taken relative to a reference m, a score that
// was the highest once: it moves only when one lies more than kHeadroom above it, since every move multiplies the results, and 2^kHeadroom times too
// large a weight is as exact.  What is added up of V is that much larger too: it stays finite while slots times the largest V are below 2^119.  (A reference
// that starts kHeadroom above the score would lose weights below 2^-118 of the highest instead of those below 2^-126.)
constexpr float kHeadroom = 8.f;
template <int HD, bool FOLD>
struct KvqRows {
  static constexpr int CPV = HD / 16;  // channels of V that a lane takes
  float m = kLowest, shift = 0.f;      // shift: -m, 0 while there is none
  float l = 0.f;                       // sum of the lane's own slots' weights
  f32x4 o[CPV];                        // o[j][i]: channel (4 (l / 16) + i) CPV + j (FOLD: term l % 16 / 4 of it)

  __device__ __forceinline__ KvqRows() {
#pragma unroll
    for (int j = 0; j < CPV; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // Scores -> weights, as the fragments of the second product.  edge: some row does not see all of the step's slots; seen: how many the
  // lane's does.  The shift is added to whole scores: an accumulator that started from it would round them to the last place of a reference that may lie
  // far below, of a step of slots that hardly count.  (Four sequences of 6 tokens at 4096 .. 32768 slots 30.4 us, 30.0 that way; others within 1%.)
  __device__ __forceinline__ void weigh(f32x4 (&x)[2], bool edge, int s, int seen, u32x4 (&pf)[FOLD ? 1 : 3]) {
    const int lane = threadIdx.x & 63, g = lane >> 4;
    if (edge) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[t][i] = s + 16 * t + 4 * g + i < seen ? x[t][i] : -INFINITY;
    }
    float top = fmaxf(fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[0][2], x[0][3])), fmaxf(fmaxf(x[1][0], x[1][1]), fmaxf(x[1][2], x[1][3])));
    if (__any(top + shift > kHeadroom || m == kLowest)) {
      // by the row's own scores: a row that others' moves moved would have bits that go by slots it does not see
      const float highest = over_groups_max(top), to = highest + shift > kHeadroom || m == kLowest ? fmaxf(m, highest) : m, f = pow2(m - to);
      l *= f;
#pragma unroll
      for (int j = 0; j < CPV; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[j][i] *= f;
      m = to;
      shift = to == kLowest ? 0.f : -to;
    }
    float p[8];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[4 * t + i] = pow2(x[t][i] + shift);
        l += p[4 * t + i];
      }
    // in three terms (FOLD: the lane's column takes its own)
    const int term = (lane & 15) >> 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a = p[2 * i], b = p[2 * i + 1];
      uint32_t w = pack_bf16x2(a, b);
      if (!FOLD) pf[0][i] = w;
#pragma unroll
      for (int t = 1; t < 3; ++t) {
        const bool next = !FOLD || term >= t;
        a -= next ? __uint_as_float(w << 16) : 0.f;
        b -= next ? __uint_as_float(w & 0xFFFF0000u) : 0.f;
        w = pack_bf16x2(a, b);
        if (!FOLD) pf[t % (FOLD ? 1 : 3)][i] = w;
      }
      if (FOLD) pf[0][i] = term < 3 ? w : 0u;
    }
  }
};

// A step added to a wave's RT row tiles.  The next one's codes (next < 0: there is none) are requested as soon as this one's have been made bf16.
template <int HD, bool FOLD, int RT>
__device__ __forceinline__ void add_step(KvqRows<HD, FOLD> (&R)[RT], KvqStep<HD>& st, const KvqQueries<HD, FOLD, RT>& Q, const KvqRow& row, bool edge, int s,
                                         int next, const int (&seen)[RT], int len) {
  constexpr int CPV = HD / 16, TERMS = FOLD ? 1 : 3;
  const int g = (threadIdx.x & 63) >> 4;
  f32x4 x[RT][2];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < 2; ++t) x[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  i32x8 k[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if constexpr (HD == 128) k[t] = i32x8{(int)st.k[t][0], (int)st.k[t][1], (int)st.k[t][2], (int)st.k[t][3]};
    else k[t] = i32x8{(int)st.k[t][0], (int)st.k[t][1]};
  }
  Q.scores(x, k, st.ks);
  if (next >= 0) st.load_k(row, next, len);
  if constexpr (FOLD) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[0][t][i] = fold_terms(x[0][t][i]);
  }
  // V.  A step at an edge may hold NaN where some row does not see it, whose weight of 0 would not hide it
  float unit[8];
  bool poisoned[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) poisoned[r] = false;
  uint32_t scale[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) scale[e] = st.v_scale(e / 4, e % 4);
  if (edge) {
    bool nan = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) nan = nan || scale[e] == 255;
    if (__any(nan)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) scale[e] = scale[e] == 255 ? 0 : scale[e];
      const int block = HD == 128 ? g : g >> 1;  // of the lane's channels in o
      for (int i = s; i < min(s + kStep, len); ++i) {
        const bool here = row.vs[(uint32_t)i * (HD / 32) + block] == 255;
#pragma unroll
        for (int r = 0; r < RT; ++r) poisoned[r] = poisoned[r] || (here && i < seen[r]);
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) unit[e] = unit_of(scale[e]);
  u32x4 f[CPV];  // eight slots of a channel
  const auto channels = [&](auto pair) {
    constexpr int P = decltype(pair)::value;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = bf16_pair<P>(st.v[i / 2][2 * (i % 2)], unit[2 * i]), b = bf16_pair<P>(st.v[i / 2][2 * (i % 2) + 1], unit[2 * i + 1]);
      f[2 * P][i] = __builtin_amdgcn_perm(b, a, 0x05040100u);
      f[2 * P + 1][i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    }
  };
  channels(std::integral_constant<int, 0>{});
  channels(std::integral_constant<int, 1>{});
  if constexpr (HD == 128) {
    channels(std::integral_constant<int, 2>{});
    channels(std::integral_constant<int, 3>{});
  }
  if (next >= 0) st.load_v(row, next, len);
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    u32x4 pf[TERMS];
    R[r].weigh(x[r], edge, s, seen[r], pf);
#pragma unroll
    for (int t = 0; t < TERMS; ++t)
#pragma unroll
      for (int j = 0; j < CPV; ++j) mma<bf16_t>(R[r].o[j], f[j], pf[t]);
    if (edge && poisoned[r]) {
#pragma unroll
      for (int j = 0; j < CPV; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) R[r].o[j][i] = NAN;
    }
  }
}

// grid (chunks and groups of row tiles of all entries, KV heads, layers).  The workgroup's waves take its steps in turn; their results meet in LDS.
// (Two waves to a SIMD at least: otherwise the compiler keeps results in the other half of the registers and moves them to and fro.)
template <int HD, bool FOLD, bool LIST, int RT, int NW>
__global__ __launch_bounds__(NW * 64, 2) void kvq_attn_kernel(KvqArgs a) {
  constexpr int ROWS = FOLD ? 4 : 16, CPV = HD / 16;
  __shared__ float s_m[RT][NW][ROWS], s_l[RT][NW][ROWS];
  __shared__ union Space {
    f32x4 o[RT][NW][ROWS][HD / 4 + 1];  // all tiles at once (one after the other: 31.3 us for 30.6); a row's results four banks behind the last's: sixteen lanes store the same channels of sixteen rows
    typename KvqQueries<HD, FOLD, RT>::Stage q;
    __device__ Space() {}
  } space;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const KvqPlace<LIST, RT> p(a);
  const KvqEntry& en = a.entry[p.e];
  const size_t at_row = p.cache_row(a);
  const KvqRow row = {a.c.kc + at_row * (HD / 2), a.c.vc + at_row * (HD / 2), a.c.ks + at_row * (HD / 32), a.c.vs + at_row * (HD / 32)};
  KvqRows<HD, FOLD> R[RT];
  KvqQueries<HD, FOLD, RT> Q;
  KvqStep<HD> st;
  int seen[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int my_row = FOLD ? n & 3 : 16 * r + n;
    seen[r] = my_row < p.rows ? en.len - en.n + p.token_of(a, p.row0 + my_row) + 1 : 0;
  }
  if constexpr (LIST) {
    // the chunk's entries, one to a lane, and which of them count
    const int32_t* list = a.blocks + (((size_t)p.l * a.n_tokens + en.q_first + p.n_tok) * a.heads + p.h) * a.n_blocks;
    const int at = p.c * a.chunk + lane;
    const bool there = lane < a.chunk && at < a.n_blocks;
    const int b = there ? list[at] : -1, before = there && at > 0 ? list[at - 1] : -1;
    unsigned long long left = __ballot(there && b > before && b >= 0 && b < (p.len + kKvqBlock - 1) / kKvqBlock);
    int slot = -1, half = 2;  // of the next step: a block is two
    int turn = 0;
    const auto next = [&]() -> int {  // the first slot of the wave's next step, or -1
      for (;;) {
        if (half == 2) {
          if (!left) return -1;
          slot = __builtin_amdgcn_readlane(b, __builtin_ctzll(left)) * kKvqBlock;
          left &= left - 1;
          half = 0;
        }
        const int s = slot + kStep * half++;
        if (s >= p.len) continue;
        if (turn++ % NW == wave) return s;
      }
    };
    int s = next();
    if (s >= 0) {
      st.load_k(row, s, p.len);
      st.load_v(row, s, p.len);
    }
    Q.template load<NW>(a, p, space.q);
    while (s >= 0) {
      const int after = next();
      add_step(R, st, Q, row, s + kStep > p.old + 1, s, after, seen, p.len);
      s = after;
    }
  } else {
    const int steps = (p.len + kStep - 1) / kStep, end = min(steps, (p.c + 1) * a.chunk);
    int i = p.c * a.chunk + wave;
    if (i < end) {
      st.load_k(row, i * kStep, p.len);
      st.load_v(row, i * kStep, p.len);
    }
    Q.template load<NW>(a, p, space.q);
    for (; i < end; i += NW) add_step(R, st, Q, row, (i + 1) * kStep > p.old + 1, i * kStep, i + NW < end ? (i + NW) * kStep : -1, seen, p.len);
  }
  // the waves' shares
  const size_t part = ((size_t)p.l * a.heads + p.h) * a.part_pitch + en.first_part;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const float l = over_groups_sum(R[r].l);
    if (lane < ROWS) {
      s_m[r][wave][lane] = R[r].m;
      s_l[r][wave][lane] = l;
    }
  }
  __syncthreads();  // and queries have been read
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int my_row = n % ROWS;
    float top = kLowest;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, s_m[r][w][my_row]);
    const float f = pow2(R[r].m - top);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[CPV];
#pragma unroll
      for (int j = 0; j < CPV; ++j) x[j] = (FOLD ? fold_terms(R[r].o[j][i]) : R[r].o[j][i]) * f;
      if (!FOLD || n < 4)
#pragma unroll
        for (int j = 0; j < CPV; j += 4) space.o[r][wave][my_row][((4 * g + i) * CPV + j) / 4] = f32x4{x[j], x[j + 1], x[j + 2], x[j + 3]};
    }
  }
  __syncthreads();
  for (int u = threadIdx.x; u < p.rows * (HD / 4); u += NW * 64) {
    const int row = u / (HD / 4), r = row / 16, k = row % 16, c = u % (HD / 4), ra = p.row0 + row;
    f32x4 sum = space.o[r][0][k][c];
    float m = s_m[r][0][k];
#pragma unroll
    for (int w = 1; w < NW; ++w) {
      sum += space.o[r][w][k][c];
      m = fmaxf(m, s_m[r][w][k]);
    }
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) all += s_l[r][w][k] * pow2(s_m[r][w][k] - m);
    if (en.chunks == 1) {
      const int tok = p.token_of(a, ra);
      f32x4* out = reinterpret_cast<f32x4*>(a.out + p.l * ((size_t)a.n_tokens * a.Hq * HD) + ((size_t)(en.q_first + tok) * a.Hq + p.h * a.group + (ra - tok * a.group)) * HD);
      const float inv = all == 0.f ? 0.f : 1.f / all;
      out[c] = sum * inv;
    } else {
      const size_t at = part + (size_t)ra * en.chunks + p.c;
      reinterpret_cast<f32x4*>(a.part)[at * (HD / 4) + c] = sum;
      if (c == 0) a.part_ml[at] = make_float2(m, all);
    }
  }
}

// The pieces of a row joined: a workgroup to every (token, query head, layer), of which HD / 4 threads stand side by side over the channels
// and the groups of them take pieces in turn.  Sums have a fixed order.  3.7 us, most of it the
// launch and a round through memory: pieces are requested before their maximum is known (4.0 otherwise).
template <int HD>
__global__ __launch_bounds__(256) void kvq_join_kernel(KvqArgs a) {
  constexpr int C4 = HD / 4, PARTS = 256 / C4, AHEAD = 4;  // threads side by side over the channels; pieces at a time; rounds of them requested first
  __shared__ float s_m[4], s_l[4];
  __shared__ f32x4 s_sum[PARTS][C4];
  const int t = blockIdx.x, j = blockIdx.y, l = blockIdx.z, tid = threadIdx.x, wave = tid >> 6;
  int e = 0;
#pragma unroll
  for (int i = 1; i < kMaxCols; ++i) e += i < a.n_entries && t >= a.entry[i].q_first;
  const KvqEntry& en = a.entry[e];
  if (en.chunks == 1) return;
  const int h = j / a.group, row = (t - en.q_first) * a.group + j % a.group;
  const size_t at = ((size_t)l * a.heads + h) * a.part_pitch + en.first_part + (size_t)row * en.chunks;
  const int c4 = tid % C4, c0 = tid / C4;
  f32x4 x[AHEAD];
  float xm[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int c = min(c0 + i * PARTS, en.chunks - 1);
    x[i] = reinterpret_cast<const f32x4*>(a.part)[(at + c) * C4 + c4];
    xm[i] = a.part_ml[at + c].x;
  }
  float m = kLowest;
  for (int c = tid; c < en.chunks; c += 256) m = fmaxf(m, a.part_ml[at + c].x);
  m = lanes_max(m, 64);
  if ((tid & 63) == 0) s_m[wave] = m;
  __syncthreads();
  m = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  float sum = 0.f;
  for (int c = tid; c < en.chunks; c += 256) {
    const float2 x = a.part_ml[at + c];
    sum += x.y * pow2(x.x - m);
  }
  sum = lanes_sum(sum, 64);
  if ((tid & 63) == 0) s_l[wave] = sum;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (c0 + i * PARTS < en.chunks) o += x[i] * pow2(xm[i] - m);
  for (int c = c0 + AHEAD * PARTS; c < en.chunks; c += PARTS) o += reinterpret_cast<const f32x4*>(a.part)[(at + c) * C4 + c4] * pow2(a.part_ml[at + c].x - m);
  s_sum[c0][c4] = o;
  __syncthreads();
  if (tid >= C4) return;
  const float all = (s_l[0] + s_l[1]) + (s_l[2] + s_l[3]);
#pragma unroll
  for (int i = 1; i < PARTS; ++i) o += s_sum[i][c4];
  const float inv = all == 0.f ? 0.f : 1.f / all;
  reinterpret_cast<f32x4*>(a.out + ((size_t)l * a.n_tokens * a.Hq + (size_t)t * a.Hq + j) * HD)[c4] = o * inv;
}

// How a call is cut: into no more workgroups than CUs.  What one does before its first step and after its last (queries, results of its waves joined,
// 5 us) costs as much as three to five steps of a wave, and a second round of workgroups adds it again.  us a call in a graph, with at most 256 : 512
// workgroups: one token at 32768 and 65536 slots of 8 KV heads 16.0 : 21.6 and 21.0 : 26.4, sixteen at 8192 35.6 : 41.1, six at 16384 16.9 : 24.1,
// sixteen of 16 tokens at 512 .. 1067 on 4 heads 18.6 : 36.7; at 16384 slots of 4 heads 11.2 : 14.1.
//   Row tiles to a wave: one, or two where there are more than sixteen rows: V of a step is then made bf16 once for both.
//   Waves: eight, but four where a wave of eight would have two steps or less.  four : eight, one token: 2048 slots of 8 heads (512 steps) 9.2 : 10.5,
//   16384 of 4 (2048) 11.2 : 11.7, sixteen lists of 24 blocks on 4 heads (3072) 24.7 : 25.4, 32768 of 8 (8192) 16.0 : 16.0, 65536 22.6 : 20.9, sixteen at
//   8192 41.0 : 36.0.
//   Contexts of two steps a wave are not cut: no second launch.  cut : whole, 8 KV heads: one token at 256, 512, 768, 1024 slots 8.9 : 7.2,
//   8.9 : 8.3, 9.0 : 9.4, 9.0 : 10.6, six at 512 and 1024 12.0 : 10.8, 12.1 : 14.7.
constexpr int kKvqCus = 256, kKvqFewSteps = 4096, kKvqWhole = 16;
struct KvqCut {
  int rows, tiles, waves;  // rows of a sequence's (a token's) queries on a KV head; row tiles to a wave; waves of a workgroup
  bool whole;              // no context is cut
};
static KvqCut kvq_cut(const KvqArgs& a, int n_layers) {
  KvqCut c = {0, 1, 4, false};
  long steps = 0;
  for (int i = 0; i < a.n_entries; ++i) {
    c.rows = std::max(c.rows, a.n_blocks ? a.group : a.entry[i].n * a.group);
    steps += a.n_blocks ? 2l * a.entry[i].n * a.n_blocks : (a.entry[i].len + kStep - 1) / kStep;
  }
  int longest = 0;
  for (int i = 0; i < a.n_entries; ++i) longest = std::max(longest, a.n_blocks ? 2 * a.n_blocks : (a.entry[i].len + kStep - 1) / kStep);
  c.whole = longest <= kKvqWhole;
  if (c.whole && longest > 4) c.waves = 8;
  if (c.rows > 16) c.tiles = 2;
  if (c.tiles == 2 || steps * a.heads * n_layers > kKvqFewSteps) c.waves = 8;
  return c;
}
void kvq_plan(KvqArgs& a, int n_layers) {
  a.inv_group = 1.f / (float)a.group;
  const KvqCut cut = kvq_cut(a, n_layers);
  const auto pieces = [&](const KvqEntry& e) { return a.n_blocks ? a.n_blocks : (e.len + kStep - 1) / kStep; };
  for (int i = 0; i < a.n_entries; ++i) a.entry[i].tiles = a.n_blocks ? 1 : (a.entry[i].n * a.group + 16 * cut.tiles - 1) / (16 * cut.tiles);
  const auto count = [&](int chunk) {  // workgroups; of chunks of one, their work
    long wgs = 0;
    for (int i = 0; i < a.n_entries; ++i) wgs += (long)((pieces(a.entry[i]) + chunk - 1) / chunk) * (a.n_blocks ? a.entry[i].n : a.entry[i].tiles);
    return wgs * a.heads * n_layers;
  };
  // a step at least for every wave (a block of a list is two); with lists an entry to a lane at most; no more than twice what a CU has to do on
  // average, so that one long context beside many short ones is not one workgroup's
  const int least = a.n_blocks ? cut.waves / 2 : cut.waves;
  const long most = std::min<long>(a.n_blocks ? 64 : 65536 / kStep, std::max<long>(least, (2 * count(1) / kKvqCus + least - 1) / least * least));
  int lo = 1, hi = (int)(most / least);  // the shortest chunk, in these units, that leaves no more workgroups than CUs, or the longest
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (count(mid * least) <= kKvqCus) hi = mid;
    else lo = mid + 1;
  }
  a.chunk = lo * least;
  if (cut.whole) a.chunk = a.n_blocks ? a.n_blocks : 65536 / kStep;
  int wg = 0;
  size_t part = 0;
  for (int i = 0; i < kMaxCols; ++i) {
    a.first_wg[i] = INT32_MAX;
    if (i >= a.n_entries) continue;
    KvqEntry& e = a.entry[i];
    e.chunks = (pieces(e) + a.chunk - 1) / a.chunk;
    e.first_part = part;
    a.first_wg[i] = wg;
    wg += e.chunks * (a.n_blocks ? e.n : e.tiles);
    part += (size_t)e.n * a.group * e.chunks;
  }
  a.n_wgs = wg;
  a.part_pitch = part;
}
static bool kvq_joined(const KvqArgs& a) {
  for (int i = 0; i < a.n_entries; ++i)
    if (a.entry[i].chunks > 1) return true;
  return false;
}
static size_t kvq_part_bytes(int hd) { return hd * sizeof(float) + sizeof(float2); }
size_t kvq_bytes_used(const KvqArgs& a, int n_layers, int hd) { return kvq_joined(a) ? a.part_pitch * a.heads * n_layers * kvq_part_bytes(hd) : 0; }

// Workgroups that a call may have beyond one chunk of everything.  A chunk either leaves no more workgroups than CUs, or it is twice what a CU has to
// do on average, with which all pieces are kKvqCus / 2 chunks and a part of one more to each; rounded to `least` pieces, four or more (lists: two),
// it may come out short by a part in least + 1.
static long kvq_more_wgs(long once, bool lists) { return std::max<long>(kKvqCus - once, kKvqCus / 2 * (lists ? 3 : 5) / (lists ? 2 : 4)); }

// What holds this call and every one like it whose contexts, or lists, are shorter: of those it is often a shorter one that has most pieces.
size_t kvq_workspace_bytes(const KvqArgs& a, int n_layers, int hd) {
  const KvqCut cut = kvq_cut(a, n_layers);
  if (cut.whole) return 0;
  const long hl = (long)a.heads * n_layers;
  long wgs = 0, rows = 0;  // of a (layer, KV head), one chunk of everything
  for (int i = 0; i < a.n_entries; ++i) {
    wgs += a.n_blocks ? a.entry[i].n : a.entry[i].tiles;
    rows += a.entry[i].n * a.group;
  }
  const long more = kvq_more_wgs(wgs * hl, a.n_blocks) / hl;
  long parts = 0;
  bool joined = false;
  for (int i = 0; i < a.n_entries; ++i) {
    const KvqEntry& e = a.entry[i];
    // lists are all cut alike, into chunks of 64 entries at most
    const long chunks = a.n_blocks ? std::min<long>(a.n_blocks, std::max<long>(1 + more / wgs, (a.n_blocks + 63) / 64))
                                   : std::min<long>((e.len + kStep - 1) / kStep, 1 + more / e.tiles);
    joined = joined || chunks > 1;
    parts += e.n * a.group * chunks;
  }
  if (!a.n_blocks) parts = std::min(parts, rows + more * std::min(16 * cut.tiles, cut.rows));
  return joined ? (size_t)(parts * hl) * kvq_part_bytes(hd) : 0;
}

// ... and every call of up to max_tokens new tokens of a sequence and lists of up to max_blocks.
size_t kvq_workspace_limit(int n_seqs, int heads, int group, int n_layers, int hd, int max_tokens, int max_slots, int max_blocks) {
  const long hl = (long)heads * n_layers, rows = (long)n_seqs * max_tokens * group * hl, tokens = (long)n_seqs * max_tokens * hl;
  const long steps = (max_slots + kStep - 1) / kStep;
  long parts = 0;
  if (steps > kKvqWhole) parts = std::min(rows * steps, rows + kKvqCus * std::min(32, max_tokens * group));
  if (2 * max_blocks > kKvqWhole)
    parts = std::max(parts, std::min(rows * max_blocks, group * std::max({(long)kKvqCus, tokens + kvq_more_wgs(tokens, true), tokens * ((max_blocks + 63) / 64)})));
  return (size_t)parts * kvq_part_bytes(hd);
}

void launch_kvq_attention(const KvqArgs& args, int n_layers, int hd, hipStream_t st) {
  KvqArgs a = args;
  if (a.n_entries == 0) return;
  a.part_ml = reinterpret_cast<float2*>(a.part + a.part_pitch * a.heads * n_layers * hd);
  const KvqCut cut = kvq_cut(a, n_layers);
  const bool fold = cut.rows <= 4;
  auto go = [&](auto kernel, auto join) {
    hipLaunchKernelGGL(kernel, dim3(a.n_wgs, a.heads, n_layers), dim3(cut.waves * 64), 0, st, a);
    if (kvq_joined(a)) hipLaunchKernelGGL(join, dim3(a.n_tokens, a.Hq, n_layers), dim3(256), 0, st, a);
  };
  auto pick = [&](auto hd_, auto join) {
    constexpr int HD = decltype(hd_)::value;
    const auto by_waves = [&](auto waves) {
      constexpr int NW = decltype(waves)::value;
      if (a.blocks) fold ? go(kvq_attn_kernel<HD, true, true, 1, NW>, join) : go(kvq_attn_kernel<HD, false, true, 1, NW>, join);
      else fold ? go(kvq_attn_kernel<HD, true, false, 1, NW>, join) : go(kvq_attn_kernel<HD, false, false, 1, NW>, join);
    };
    if (cut.tiles == 2) go(kvq_attn_kernel<HD, false, false, 2, 8>, join);
    else cut.waves == 8 ? by_waves(std::integral_constant<int, 8>{}) : by_waves(std::integral_constant<int, 4>{});
  };
  if (hd == 128) pick(std::integral_constant<int, 128>{}, kvq_join_kernel<128>);
  else pick(std::integral_constant<int, 64>{}, kvq_join_kernel<64>);
}

// ------------------------------------------------------------------------------------------
// Selection: (1) the blocks' scores, a workgroup to some blocks of a sequence, which reads their bounds once for all its new tokens;
// (2) a workgroup to every (layer, token, KV head) finds a score that as many blocks reach as shall stay, bit by bit, and writes the list.
// ------------------------------------------------------------------------------------------
// grid (groups of blocks of all entries, KV heads, layers).  G: query heads of a KV head, or one more: their queries are requested together.
// Products and sums are fp64, whose operands are exact: blocks are compared with each other, and a
// rounding that went one way for one and the other way for its neighbour would show as another list.  The bound that a channel takes goes by q's sign: where a
// block has no number (plus, minus infinity), the larger of both products would be plus infinity, and NaN be read first.  Bound: the chain of two loads, and eight products a lane
// and query; 512 blocks of 8 KV heads, one token 3.6 us (0.3 of bytes), sixteen sequences of 63 .. 250 blocks with seven heads to a KV head 5.9;
// several tokens one after the other: four sequences of 6 tokens at 64 .. 512 blocks 9.3, sixteen of 16 at 63 .. 180 on 4 heads 33.7.
template <int HD, int G>
__global__ __launch_bounds__(256) void kvq_score_kernel(KvqSelectArgs a) {
  constexpr int LANES = HD / 8, BLOCKS = 256 / LANES;  // lanes to a block: eight channels each
  int e = 0;
#pragma unroll
  for (int i = 1; i < kMaxCols; ++i) e += (int)blockIdx.x >= a.first_wg[i];
  const KvqEntry& en = a.entry[e];
  const int h = blockIdx.y, l = blockIdx.z, lane = threadIdx.x % LANES;
  const int block = (blockIdx.x - a.first_wg[e]) * BLOCKS + threadIdx.x / LANES;
  const int held = (en.len + kKvqBlock - 1) / kKvqBlock;
  const u32x4* src = reinterpret_cast<const u32x4*>(a.bounds + ((((size_t)l * a.n_seqs + en.seq) * a.heads + h) * a.max_blocks + min(block, held - 1)) * 2 * HD) + lane;
  const u32x4 lo_bits = src[0], hi_bits = src[HD / 8];
  for (int t = 0; t < en.n; ++t) {
    const f32x4* q = reinterpret_cast<const f32x4*>(a.q + (((size_t)l * a.n_tokens + en.q_first + t) * a.Hq + h * a.group) * HD + lane * 8);
    f32x4 x[G][2];
#pragma unroll
    for (int j = 0; j < G; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) x[j][i] = q[min(j, a.group - 1) * (HD / 4) + i];
    float lo[8], hi[8];
    unpack<bf16_t>(lo_bits, lo);
    unpack<bf16_t>(hi_bits, hi);
    double best = NAN;
#pragma unroll
    for (int j = 0; j < G; ++j) {
      double s = 0.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = x[j][i / 4][i % 4];
        s = fma((double)v, (double)(v > 0.f ? hi[i] : lo[i]), s);
      }
      best = fmax(best, lanes_sum(s, LANES));  // passes over NaN; a head twice is the head
    }
    if (lane == 0 && block < held) a.scores[(((size_t)l * a.n_tokens + en.q_first + t) * a.heads + h) * a.most + block] = best;
  }
}

// The order of scores as unsigned numbers: NaN below everything, the two zeros alike.
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return 1ull << 32;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// A workgroup to every list; thread i holds blocks kSelectThreads j + i.  Bound: a chain of counts and barriers, two bits of the scores' upper
// halves a round, from the first bit that differs until as many blocks reach the bound as shall stay: 32 of 512 blocks 6.9 us.  (One bit a
// round, and queries requested one after the other: selection and attention of those sixteen sequences 27.1 us in a graph instead of 25.6.  A
// wave with all blocks in its registers: 10 us, much of which its instructions took to arrive, three thousand, each executed a few times.)
constexpr int kSelectThreads = 256, kSelectWaves = kSelectThreads / 64, kSelectRegs = kMaxKvqSelect / kSelectThreads;
struct SelectShared {
  int count[2][3][kSelectWaves];
  uint32_t any[kSelectWaves], all[kSelectWaves];
};
// How many of the workgroup's keys reach each of three numbers; turn: 0 and 1 in turn, so that a call's counts are read before the next but one writes there.
struct Three {
  int n[3];
};
__device__ __forceinline__ Three count_from(const uint32_t (&key)[kSelectRegs], uint32_t a, uint32_t b, uint32_t c, SelectShared& sh, int& turn) {
  Three r = {{0, 0, 0}};
#pragma unroll
  for (int j = 0; j < kSelectRegs; ++j) {
    r.n[0] += __popcll(__ballot(key[j] >= a));
    r.n[1] += __popcll(__ballot(key[j] >= b));
    r.n[2] += __popcll(__ballot(key[j] >= c));
  }
  if ((threadIdx.x & 63) < 3) {
    const int i = threadIdx.x & 63;
    sh.count[turn][i][threadIdx.x >> 6] = i == 0 ? r.n[0] : i == 1 ? r.n[1] : r.n[2];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    r.n[i] = 0;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) r.n[i] += sh.count[turn][i][w];
  }
  turn ^= 1;
  return r;
}
// A bound that `want` of the numbers reach, or, where equal ones prevent that, the want-th highest.  Two bits at a time from `bit` (odd) down, the bits
// above being those of `bound`, until as many reach it as are wanted.  A 0 counts for nothing.
__device__ __forceinline__ uint32_t bound_of(const uint32_t (&key)[kSelectRegs], int want, uint32_t bound, int bit, SelectShared& sh, int& turn) {
  for (bit -= 1; bit >= 0; bit -= 2) {
    const uint32_t step = 1u << bit;
    const Three r = count_from(key, bound + step, bound + 2 * step, bound + 3 * step, sh, turn);
    const int digit = r.n[2] >= want ? 3 : r.n[1] >= want ? 2 : r.n[0] >= want ? 1 : 0;
    bound += digit * step;
    if (r.n[2] == want || r.n[1] == want || r.n[0] == want) break;  // the highest number that as many reach is one that exactly they reach
  }
  return bound;
}

__global__ __launch_bounds__(kSelectThreads) void kvq_select_kernel(KvqSelectArgs a) {
  __shared__ SelectShared sh;
  const int t = blockIdx.x, h = blockIdx.y, l = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int e = 0;
#pragma unroll
  for (int i = 1; i < kMaxCols; ++i) e += i < a.n_entries && t >= a.entry[i].q_first;
  const KvqEntry& en = a.entry[e];
  const int seen = en.len - en.n + (t - en.q_first) + 1, held = (seen + kKvqBlock - 1) / kKvqBlock;
  const size_t list = ((size_t)l * a.n_tokens + t) * a.heads + h;
  const double* scores = a.scores + list * a.most;
  int32_t* out = a.out + list * a.n_select;
  const int want = min(a.n_select, held), last0 = max(0, held - a.last), n_forced = min(held, a.first) + held - max(last0, min(held, a.first));
  // the halves of the keys; 0, 0: no block.  A key's upper half is never 0; 0, ~0: a block that stays anyway
  uint32_t hi[kSelectRegs], lo[kSelectRegs], any = 0, all = ~0u;
#pragma unroll
  for (int j = 0; j < kSelectRegs; ++j) {
    const int b = kSelectThreads * j + tid;
    const bool there = b < held, forced = there && (b < a.first || b >= last0);
    uint64_t key = 0;
    if (there) key = score_key(scores[b]);
    hi[j] = forced ? 0 : (uint32_t)(key >> 32);
    lo[j] = forced ? ~0u : (uint32_t)key;
    any |= hi[j];
    all &= hi[j] ? hi[j] : ~0u;
  }
  // those that stay: over (bound_hi, bound_lo), and of those at it the lowest blocks; the forced ones first of all
  const bool only_forced = n_forced >= want;
  uint32_t bound_hi = ~0u, bound_lo = ~0u;
  int turn = 0;
  if (!only_forced) {
    const int more = want - n_forced;
    any = wave_or(any);
    all = ~wave_or(~all);
    if (lane == 0) sh.any[wave] = any, sh.all[wave] = all;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) any |= sh.any[w], all &= sh.all[w];
    const int top = (31 - __builtin_clz((any ^ all) | 1u)) | 1;  // the highest bit that they differ in, or the one above
    bound_hi = bound_of(hi, more, all >> top >> 1 << top << 1, top, sh, turn);
    const Three r = count_from(hi, bound_hi, bound_hi + 1, ~0u, sh, turn);  // no upper half is all ones
    bound_lo = 0;
    if (r.n[0] > more) {  // scores alike in the upper half
      uint32_t same[kSelectRegs];
#pragma unroll
      for (int j = 0; j < kSelectRegs; ++j) same[j] = hi[j] == bound_hi ? lo[j] : 0;
      bound_lo = bound_of(same, more - r.n[1], 0, 31, sh, turn);
    }
  }
  int group[kSelectRegs];  // 2: stays, 1: stays as one of the lowest, 0: does not
  uint32_t grade[kSelectRegs];
#pragma unroll
  for (int j = 0; j < kSelectRegs; ++j) {
    const bool forced = hi[j] == 0 && lo[j] != 0;
    group[j] = only_forced ? forced : forced || hi[j] > bound_hi || (hi[j] == bound_hi && lo[j] > bound_lo) ? 2 : hi[j] == bound_hi && lo[j] == bound_lo;
    grade[j] = (uint32_t)group[j];
  }
  int ties = want - count_from(grade, 2, 3, 3, sh, turn).n[0], at = 0;
  const unsigned long long below = (1ull << lane) - 1;
  // in the order of the blocks: runs of kSelectThreads, in them the waves.  tied and stay: of the waves in front, then of all
#pragma unroll
  for (int j = 0; j < kSelectRegs; ++j) {
    if (kSelectThreads * j < held) {
      const unsigned long long tied = __ballot(group[j] == 1), sure = __ballot(group[j] == 2);
      __syncthreads();
      if (lane == 0) sh.count[0][0][wave] = __popcll(tied), sh.count[0][1][wave] = __popcll(sure);
      __syncthreads();
      int tied_before = 0, tied_all = 0, sure_before = 0, sure_all = 0;
#pragma unroll
      for (int w = 0; w < kSelectWaves; ++w) {
        tied_before += w < wave ? sh.count[0][0][w] : 0;
        sure_before += w < wave ? sh.count[0][1][w] : 0;
        tied_all += sh.count[0][0][w];
        sure_all += sh.count[0][1][w];
      }
      const int tied_in_front = tied_before + __popcll(tied & below);
      if (group[j] == 2 || (group[j] == 1 && tied_in_front < ties))
        out[at + sure_before + __popcll(sure & below) + min(tied_in_front, ties)] = kSelectThreads * j + tid;
      at += sure_all + min(tied_all, ties);
      ties -= min(tied_all, ties);
    }
  }
  for (int i = at + tid; i < a.n_select; i += kSelectThreads) out[i] = -1;
}

size_t kvq_select_workspace_bytes(const KvqSelectArgs& a, int n_layers) { return (size_t)n_layers * a.n_tokens * a.heads * a.most * sizeof(double); }

void launch_kvq_select(const KvqSelectArgs& args, int n_layers, int hd, hipStream_t st) {
  KvqSelectArgs a = args;
  if (a.n_entries == 0) return;
  const int per = 256 / (hd / 8);
  int wg = 0;
  for (int i = 0; i < kMaxCols; ++i) {
    a.first_wg[i] = INT32_MAX;
    if (i >= a.n_entries) continue;
    a.first_wg[i] = wg;
    wg += ((a.entry[i].len + kKvqBlock - 1) / kKvqBlock + per - 1) / per;
  }
  auto score = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(wg, a.heads, n_layers), dim3(256), 0, st, a); };
  auto pick = [&](auto hd_) {
    constexpr int HD = decltype(hd_)::value;
    if (a.group > 4) score(kvq_score_kernel<HD, 8>);
    else if (a.group > 2) score(kvq_score_kernel<HD, 4>);
    else score(kvq_score_kernel<HD, 2>);
  };
  if (hd == 128) pick(std::integral_constant<int, 128>{});
  else pick(std::integral_constant<int, 64>{});
  hipLaunchKernelGGL(kvq_select_kernel, dim3(a.n_tokens, a.heads, n_layers), dim3(kSelectThreads), 0, st, a);
}

}  // namespace es
