// The attention weight that cached slots receive (gfx950): for every KV head and slot, the probabilities that the queries of the
// new tokens give it, added up over the tokens and over the query heads that share the KV head.
//
//   w'[s] = w[s] + sum over rows r of softmax_s(q_r . k_s / sqrt(hd)),   a row: one query head of one new token
//
// The queries of a KV head are the rows of a matrix product with its keys, on the matrix cores: a tile of 16 slots is the A
// operand, 16 rows are the B operand, so a lane holds four slots' scores of one row.  bf16 keys meet the queries as three bf16
// terms, which hold all 24 bits of them, fp32 keys as they are: weights are added up over a whole generation and compared with
// each other, so they are kept to fp32.  Two launches, since a row's sum is known only at the end of its context:
//   (1) weigh_stats_kernel   per chunk of the context: every row's maximum and sum of exp(score - maximum);
//   (2) weigh_add_kernel     the scores once more, their probabilities, the sums over the rows.
// (Keeping the scores between the two would take four bytes a row and slot: 16 beside the 256 or 512 of a key for four rows, 512 for
// 128.  Neither built nor measured.)  Contexts of a few hundred slots are one launch, weigh_short_kernel.
// Long contexts read the keys twice: 61 440 slots of 8 KV heads, 126 MB, 23.8 and 25.8 us (5.1 TB/s), where a kernel that only reads
// takes 17.5 us if the last-level cache holds them and 19.9 if not.  Many rows are bound by what a wave does with a tile of scores: 16
// sequences of 16 tokens and 800 slots, 112 rows a KV head, 12.3 and 13.0 us, of which the keys alone would be 1.8 and the products,
// three terms of each, 3.7.
#include "launch_common.hpp"
#include "lane_ops.hpp"

#include <string.h>

namespace es {

constexpr int kWeighMaxTiles = 8;    // of 16 rows: 16 tokens, 8 query heads per KV head
constexpr int kWeighSums = 4096;     // sums over rows that a workgroup gathers: slots of its chunk times the groups of its waves
constexpr float kLowest = -3.4028235e38f;

template <typename T>
struct WeighTerms {
  static constexpr int N = 1;
};
template <>
struct WeighTerms<bf16_t> {
  static constexpr int N = 3;
};
template <typename T, int HD>
struct WeighGeom {
  static constexpr int EPL = Tr<T>::EPL, KT = Tr<T>::KT, NKT = HD / KT, TERMS = WeighTerms<T>::N;
};

// One workgroup: a chunk of one sequence's context, one KV head, one layer.  A wave takes one row tile; waves share out the tiles
// in groups (a power of two of them) and the chunk's slot tiles inside a group.
template <int NW>
struct WeighPlace {
  int e, h, l, c;      // entry, KV head, layer, chunk
  int rows, old, len;  // query rows; slots that were there before; slots
  int s0, s1;          // the chunk
  int tiles, groups, splits, group, split;
  __device__ __forceinline__ WeighPlace(const WeighArgs& a) {
    e = 0;
#pragma unroll
    for (int i = 1; i < kMaxCols; ++i) e += (int)blockIdx.x >= a.first_wg[i];
    const WeighEntry& en = a.entry[e];
    c = blockIdx.x - a.first_wg[e];
    h = blockIdx.y;
    l = blockIdx.z;
    rows = en.n * a.group;
    len = en.len;
    old = en.len - en.n;
    s0 = c * a.chunk;
    s1 = min(len, s0 + a.chunk);
    tiles = (rows + 15) / 16;
    const int log2_groups = tiles <= 1 ? 0 : tiles <= 2 ? 1 : tiles <= 4 ? 2 : 3;
    groups = 1 << log2_groups;
    splits = NW >> log2_groups;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    group = wave & (groups - 1);
    split = wave >> log2_groups;
  }
  __device__ __forceinline__ size_t cache_row(const WeighArgs& a) const {  // the first slot of the (layer, sequence, KV head)
    return (((size_t)l * a.n_seqs + a.entry[e].seq) * a.heads + h) * (size_t)a.max_slots;
  }
  __device__ __forceinline__ int token_of(const WeighArgs& a, int row) const { return (int)(((float)row + 0.5f) * a.inv_group); }  // row < 128: off by far less than half a step
  __device__ __forceinline__ int seen_by(const WeighArgs& a, int row) const { return old + token_of(a, row) + 1; }  // slots that a row attends to
};

// K fragments of the 16 slots from s on: lane l holds slot s + l % 16.  Slots past the last fetch the last one.
template <typename T, int HD>
struct WeighKeys {
  u32x4 k[HD / Tr<T>::KT];
  __device__ __forceinline__ void load(const T* k_row, int s, int len) {
    const int lane = threadIdx.x & 63;
    const T* src = k_row + (uint32_t)min(s + (lane & 15), len - 1) * HD + (lane >> 4) * Tr<T>::EPL;
#pragma unroll
    for (int kt = 0; kt < HD / Tr<T>::KT; ++kt) k[kt] = *reinterpret_cast<const u32x4*>(src + kt * Tr<T>::KT);
  }
};

// The queries of the wave's row tile, scaled, as B fragments: lane l holds row l % 16, elements (l / 16) EPL .. of every k tile.
// Rows past the last take the last one's queries; their scores are not used.
template <typename T, int HD, int NW>
struct WeighQueries {
  typedef WeighGeom<T, HD> Geo;
  u32x4 q[Geo::NKT][Geo::TERMS];
  static __device__ __forceinline__ void fragment(const float* src, float scale, u32x4 (&out)[Geo::TERMS]) {
    float x[Geo::EPL];
#pragma unroll
    for (int i = 0; i < Geo::EPL / 4; ++i) {
      const f32x4 v = reinterpret_cast<const f32x4*>(src)[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * i + j] = v[j] * scale;
    }
    if constexpr (Geo::TERMS == 3) {
      bf16x8 hi, lo;
      split_bf16x8(x, hi, lo);
      out[0] = __builtin_bit_cast(u32x4, hi);
      out[1] = __builtin_bit_cast(u32x4, lo);
      out[2] = __builtin_bit_cast(u32x4, third_bf16x8(x, hi, lo));
    } else {
      out[0] = u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
  }
  // stage: LDS for up to NW / 2 tiles.  Where several waves need a tile its terms are made once and handed round there.
  __device__ __forceinline__ void load(const WeighArgs& a, const WeighPlace<NW>& p, u32x4* stage) {
    const int lane = threadIdx.x & 63;
    const float* base = a.q + p.l * a.q_layer_pitch + ((size_t)a.entry[p.e].q_first * a.Hq + p.h * a.group) * HD + (lane >> 4) * Geo::EPL;
    auto row_at = [&](int tile) {
      const int r = min(tile * 16 + (lane & 15), p.rows - 1), tok = p.token_of(a, r);
      return base + (uint32_t)(tok * a.Hq + (r - tok * a.group)) * HD;
    };
    if (p.splits > 1) {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      for (int i = wave; i < p.tiles * Geo::NKT; i += NW) {
        u32x4 f[Geo::TERMS];
        fragment(row_at(i / Geo::NKT) + i % Geo::NKT * Geo::KT, a.scale, f);
#pragma unroll
        for (int t = 0; t < Geo::TERMS; ++t) stage[(i * Geo::TERMS + t) * 64 + lane] = f[t];
      }
      __syncthreads();
      const int tile = min(p.group, p.tiles - 1);
#pragma unroll
      for (int kt = 0; kt < Geo::NKT; ++kt)
#pragma unroll
        for (int t = 0; t < Geo::TERMS; ++t) q[kt][t] = stage[((tile * Geo::NKT + kt) * Geo::TERMS + t) * 64 + lane];
    } else {
      const float* src = row_at(min(p.group, p.tiles - 1));
#pragma unroll
      for (int kt = 0; kt < Geo::NKT; ++kt) fragment(src + kt * Geo::KT, a.scale, q[kt]);
    }
  }
};

// Scores of a slot tile and a row tile.  SLOTS_IN_LANES: element i of lane l is row 4 (l / 16) + i, slot s + l % 16; otherwise slot
// s + 4 (l / 16) + i, row l % 16.
template <typename T, int HD, int NW, bool SLOTS_IN_LANES>
__device__ __forceinline__ f32x4 scores_of(const WeighKeys<T, HD>& kf, const WeighQueries<T, HD, NW>& Q) {
  typedef WeighGeom<T, HD> Geo;
  f32x4 x[Geo::TERMS];
#pragma unroll
  for (int t = 0; t < Geo::TERMS; ++t) x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int kt = 0; kt < Geo::NKT; ++kt)
#pragma unroll
    for (int t = 0; t < Geo::TERMS; ++t) {
      if (SLOTS_IN_LANES) mma<T>(x[t], Q.q[kt][t], kf.k[kt]);
      else mma<T>(x[t], kf.k[kt], Q.q[kt][t]);
    }
  if constexpr (Geo::TERMS == 3) x[0] += x[1] + x[2];
  return x[0];
}

// The wave's slot tiles; `first` holds the keys of the tile that the wave loads first, requested already.
// Four waves (one row tile): every wave loads its own tiles, the next one's keys requested before the present one's are used.
// Eight: the waves need the same keys.  Each loads one tile of a round of eight, they meet in LDS in the order of the operand, and
// the next round's are on their way while the scores are worked out.  (Every wave loading all the keys that it needs has few
// different ones under way: sixteen sequences of 16 tokens, 112 rows, 35 us a call, and 24 so.
// Keys of two rounds ahead in registers: 144 of them, one workgroup to a CU, and 52.7 us for these 126 MB instead of 49.8.)
template <typename T, int HD, int NW>
constexpr int weigh_keys() {
  return NW == 4 ? 0 : NW * WeighGeom<T, HD>::NKT * 64;
}
// body(n, s, kf): n slot tiles (1 or 2), from slots s[0], s[1] on.
template <typename T, int HD, int NW, class Body>
__device__ __forceinline__ void each_tile(const T* k_row, const WeighPlace<NW>& p, WeighKeys<T, HD>& first, u32x4* space, const Body& body) {
  typedef std::integral_constant<int, 1> One;
  typedef std::integral_constant<int, 2> Two;
  if constexpr (NW == 4) {
    const int step = 16 * NW;
    WeighKeys<T, HD> next;
    for (int s = p.s0 + 16 * p.split; s < p.s1; s += 2 * step) {
      if (s + step < p.s1) next.load(k_row, s + step, p.len);
      body(One{}, &s, &first);
      if (s + step >= p.s1) return;
      if (s + 2 * step < p.s1) first.load(k_row, s + 2 * step, p.len);
      const int after = s + step;
      body(One{}, &after, &next);
    }
  } else {
    constexpr int NKT = WeighGeom<T, HD>::NKT;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int base = p.s0; base < p.s1; base += 16 * NW) {
      __syncthreads();  // the last round's keys (before the first: the queries' terms) have been read
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) space[(wave * NKT + kt) * 64 + lane] = first.k[kt];
      __syncthreads();
      if (base + 16 * NW < p.s1) first.load(k_row, base + 16 * (NW + wave), p.len);
      if (p.group >= p.tiles) continue;
      const int n = min(NW, (p.s1 - base + 15) / 16);  // tiles of this round
      for (int t = p.split; t < n; t += 2 * p.splits) {  // two at a time: their chains of dependent steps run side by side
        WeighKeys<T, HD> kf[2];
        const int t1 = min(t + p.splits, n - 1), s[2] = {base + 16 * t, base + 16 * t1};
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
          kf[0].k[kt] = space[(t * NKT + kt) * 64 + lane];
          kf[1].k[kt] = space[(t1 * NKT + kt) * 64 + lane];
        }
        if (t + p.splits < n) body(Two{}, s, kf);
        else body(One{}, s, kf);
      }
    }
  }
}

// LDS of a workgroup: the terms of the queries of up to NW / 2 row tiles, then the keys.
template <typename T, int HD, int NW>
constexpr int weigh_space() {
  constexpr int terms = NW / 2 * WeighGeom<T, HD>::NKT * WeighGeom<T, HD>::TERMS * 64;
  return terms > weigh_keys<T, HD, NW>() ? terms : weigh_keys<T, HD, NW>();
}

// Scores are carried in units of log 2 (the scale holds log2(e) / sqrt(hd)).
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
// two partial (maximum, sum) of a row; nothing is (kLowest, 0)
__device__ __forceinline__ void join(float& m, float& l, float om, float ol) {
  const float top = fmaxf(m, om);
  l = l * pow2(m - top) + ol * pow2(om - top);
  m = top;
}

// Every row's maximum and sum over the workgroup's chunk: thread r returns those of row r.
template <typename T, int HD, int NW>
__device__ __forceinline__ float2 chunk_stats(const WeighArgs& a, const WeighPlace<NW>& p, const T* k_row, const WeighQueries<T, HD, NW>& Q,
                                              WeighKeys<T, HD>& first, u32x4* s_space, float (&s_m)[NW][16], float (&s_l)[NW][16]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = p.group * 16 + (lane & 15), seen = row < p.rows ? p.seen_by(a, row) : 0;
  float m = kLowest, l = 0.f;
  each_tile<T, HD, NW>(k_row, p, first, s_space, [&](auto n, const int* s, const WeighKeys<T, HD>* kf) {
    constexpr int N = decltype(n)::value;
    f32x4 x[N];
    float top = m;
#pragma unroll
    for (int t = 0; t < N; ++t) {
      x[t] = scores_of<T, HD, NW, false>(kf[t], Q);
      if (s[t] + 16 > p.old + 1) {  // only the last tiles hold slots that some row does not see
#pragma unroll
        for (int i = 0; i < 4; ++i) x[t][i] = s[t] + 4 * (lane >> 4) + i < seen ? x[t][i] : -INFINITY;
      }
      top = fmaxf(fmaxf(fmaxf(top, x[t][0]), fmaxf(x[t][1], x[t][2])), x[t][3]);
    }
    l *= pow2(m - top);
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) l += pow2(x[t][i] - top);
    m = top;
  });
  // the four lanes of a row, then the waves that share its tile
  for (int off = 16; off < 64; off <<= 1) join(m, l, __shfl_xor(m, off, 64), __shfl_xor(l, off, 64));
  if (lane < 16) {
    s_m[wave][lane] = m;
    s_l[wave][lane] = l;
  }
  __syncthreads();
  const int r = min((int)threadIdx.x, p.rows - 1);  // there are at least as many threads as rows
  float top = s_m[r / 16][r % 16], sum = s_l[r / 16][r % 16];
  for (int w = 1; w < p.splits; ++w) join(top, sum, s_m[w * p.groups + r / 16][r % 16], s_l[w * p.groups + r / 16][r % 16]);
  return make_float2(top, sum);
}

// The chunk's probabilities, added up over the rows and to the weights.  s_row: every row's maximum and 1 / sum over its context.
template <typename T, int HD, int NW>
__device__ __forceinline__ void chunk_add(const WeighArgs& a, const WeighPlace<NW>& p, const T* k_row, size_t row_at, const WeighQueries<T, HD, NW>& Q,
                                          WeighKeys<T, HD>& first, u32x4* s_space, const float2* s_row, float* sums) {
  const int lane = threadIdx.x & 63;
  float* s_sum = sums + p.group * a.chunk;
  // the lane's four rows; those past the last give nothing
  float m[4], inv[4];
  int seen[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = p.group * 16 + 4 * (lane >> 4) + i;
    const float2 x = s_row[min(row, p.rows - 1)];
    m[i] = x.x;
    inv[i] = x.y;
    seen[i] = row < p.rows ? p.seen_by(a, row) : 0;
  }
  const bool full = p.group * 16 + 16 <= p.rows;
  each_tile<T, HD, NW>(k_row, p, first, s_space, [&](auto n, const int* s, const WeighKeys<T, HD>* kf) {
    constexpr int N = decltype(n)::value;
#pragma unroll
    for (int t = 0; t < N; ++t) {
      const f32x4 x = scores_of<T, HD, NW, true>(kf[t], Q);
      const bool all = full && s[t] + 16 <= p.old + 1;  // every row is one and sees every slot
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float prob = pow2(x[i] - m[i]) * inv[i];
        sum += all || s[t] + (lane & 15) < seen[i] ? prob : 0.f;
      }
      sum = across<false>(sum, [](float u, float v) { return u + v; });
      sum = across<true>(sum, [](float u, float v) { return u + v; });
      if (lane < 16) s_sum[s[t] - p.s0 + lane] = sum;
    }
  });
  __syncthreads();
  for (int i = threadIdx.x; i < p.s1 - p.s0; i += NW * 64) {
    float sum = sums[i];
    for (int g = 1; g < p.tiles; ++g) sum += sums[g * a.chunk + i];
    const int s = p.s0 + i;
    const float before = a.w_in && s < p.old ? a.w_in[row_at + s] : 0.f;  // the new tokens' slots start from nothing
    a.w_out[row_at + s] = before + sum;
  }
}

// grid (chunks of all entries, KV heads, layers), as the others'
template <typename T, int HD, int NW>
__global__ __launch_bounds__(NW * 64) void weigh_stats_kernel(WeighArgs a) {
  __shared__ u32x4 s_space[weigh_space<T, HD, NW>()];
  __shared__ float s_m[NW][16], s_l[NW][16];
  const WeighPlace<NW> p(a);
  const WeighEntry& e = a.entry[p.e];
  const T* k_row = reinterpret_cast<const T*>(a.k) + p.cache_row(a) * HD;
  WeighKeys<T, HD> first;
  first.load(k_row, p.s0 + 16 * (threadIdx.x >> 6), p.len);
  WeighQueries<T, HD, NW> Q;
  Q.load(a, p, s_space);
  const float2 mine = chunk_stats<T, HD, NW>(a, p, k_row, Q, first, s_space, s_m, s_l);
  const int r = threadIdx.x;
  if (r < p.rows) a.stats[((size_t)p.l * a.heads + p.h) * a.stats_pitch + e.first_stat + (size_t)r * e.chunks + p.c] = mine;
}

template <typename T, int HD, int NW>
__global__ __launch_bounds__(NW * 64) void weigh_add_kernel(WeighArgs a) {
  constexpr int NT = NW * 64;
  __shared__ u32x4 s_space[weigh_space<T, HD, NW>()];
  __shared__ f32x4 s_sums[kWeighSums / 4];
  __shared__ float2 s_row[kWeighMaxTiles * 16];
  const WeighPlace<NW> p(a);
  const WeighEntry& e = a.entry[p.e];
  const size_t row_at = p.cache_row(a);
  const T* k_row = reinterpret_cast<const T*>(a.k) + row_at * HD;
  WeighKeys<T, HD> first;
  first.load(k_row, p.s0 + 16 * (threadIdx.x >> 6), p.len);
  // the rows' maxima and sums over all chunks: as many lanes to a row as there are threads for each, one to four rows' worth
  const float2* st0 = a.stats + ((size_t)p.l * a.heads + p.h) * a.stats_pitch + e.first_stat;
  const int log2_per_row = p.rows <= NT / 64 ? 6 : p.rows <= NT / 32 ? 5 : p.rows <= NT / 16 ? 4 : p.rows <= NT / 8 ? 3 : 2;  // rows <= NT / 4
  const int r = threadIdx.x >> log2_per_row, c0 = threadIdx.x & ((1 << log2_per_row) - 1);
  const float2* st = st0 + (size_t)min(r, p.rows - 1) * e.chunks;
  constexpr int kAhead = 4;  // requested in front of the queries
  float2 ahead[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) ahead[i] = st[min(c0 + (i << log2_per_row), e.chunks - 1)];
  WeighQueries<T, HD, NW> Q;
  Q.load(a, p, s_space);
  float rm = kLowest, rl = 0.f;
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (c0 + (i << log2_per_row) < e.chunks) join(rm, rl, ahead[i].x, ahead[i].y);
  for (int c = c0 + (kAhead << log2_per_row); c < e.chunks; c += 1 << log2_per_row) join(rm, rl, st[c].x, st[c].y);
  for (int off = 1; off < 1 << log2_per_row; off <<= 1) join(rm, rl, __shfl_xor(rm, off, 64), __shfl_xor(rl, off, 64));
  if (r < p.rows && c0 == 0) s_row[r] = make_float2(rm, 1.f / rl);
  __syncthreads();
  chunk_add<T, HD, NW>(a, p, k_row, row_at, Q, first, s_space, s_row, reinterpret_cast<float*>(s_sums));
}

// Contexts of one chunk each: both in one launch.
template <typename T, int HD, int NW>
__global__ __launch_bounds__(NW * 64) void weigh_short_kernel(WeighArgs a) {
  __shared__ u32x4 s_space[weigh_space<T, HD, NW>()];
  __shared__ float s_m[NW][16], s_l[NW][16];
  __shared__ f32x4 s_sums[kWeighSums / 4];
  __shared__ float2 s_row[kWeighMaxTiles * 16];
  const WeighPlace<NW> p(a);
  const size_t row_at = p.cache_row(a);
  const T* k_row = reinterpret_cast<const T*>(a.k) + row_at * HD;
  WeighKeys<T, HD> first;
  first.load(k_row, p.s0 + 16 * (threadIdx.x >> 6), p.len);
  WeighQueries<T, HD, NW> Q;
  Q.load(a, p, s_space);
  const float2 mine = chunk_stats<T, HD, NW>(a, p, k_row, Q, first, s_space, s_m, s_l);
  first.load(k_row, p.s0 + 16 * (threadIdx.x >> 6), p.len);
  if ((int)threadIdx.x < p.rows) s_row[threadIdx.x] = make_float2(mine.x, 1.f / mine.y);
  __syncthreads();
  chunk_add<T, HD, NW>(a, p, k_row, row_at, Q, first, s_space, s_row, reinterpret_cast<float*>(s_sums));
}

// How the contexts are cut: workgroups of four waves where no entry has more than one row tile, else of eight; chunks of a multiple
// of 64 slots, so long that there is a workgroup to a CU at most.  What a workgroup does before its first scores (the queries'
// terms, the sums of all chunks) is then done once for its share of the keys.  us a call, 32 query heads on 8 KV heads but for (*),
// 28 on 4, with at most 256 / 512 / 1024 / 2048 workgroups: one token each at 4096 .. 32768 slots 45 / 50 / 52 / 48, 16 at 8192
// 18 / 21 / 38 / 38, 12 each at four times 2048 16.5 / 18.2 / 33 / 33, (*) 16 at 32768 40 / 43 / 69 / 165, 6 each in fp32 at twice
// 8192 40 / 45 / 59 / 104.  Two row tiles of bf16 are the exception where their chunks are long: the keys that a round brings serve two
// waves each only, and two workgroups to a CU have more of them under way; but twice the chunks are twice the statistics that every
// workgroup joins, so only where a workgroup still has more than two rounds.  us a call in a graph, keys from memory, with at most
// 256 / 512 workgroups, by the slots of a chunk that 512 leave (query heads on KV heads, tokens of each sequence, slots):
//    64  8 on 1, 4 at 32768 16.5 / 24.1; 16 on 8, 12 at 4096 12.5 / 15.5
//   128  32 on 8, 6 at 8192 15.4 / 16.4; 28 on 4, 4 at 16384 15.5 / 17.6; 8 on 1, 4 at 65536 19.3 / 25.0
//   192  32 on 8, 6 at 12288 17.8 / 19.2; 28 on 4, 4 at 24576 17.8 / 20.4; 16 on 8, 12 at 12288 17.8 / 19.3
//   256  32 on 8, 6 at 16384 21.1 / 20.3, at sixteen times 1024 21.7 / 22.2; 28 on 4, 4 at 32768 21.3 / 21.2; 8 on 1, 4 at twice 65536
//        22.3 / 23.8; heads of 64: 32 on 8, 6 at 16384 15.6 / 14.9, 14 on 2, 3 at 65536 16.6 / 18.5
//   320  32 on 8, 6 at 20480 26.1 / 26.1
//   384  32 on 8, 6 at 24576 29.3 / 27.0
//   512  32 on 8, 6 at 32768 35.3 / 33.0, 5 at sixteen times 2048 35.4 / 33.1; 28 on 4, 3 at 65536 35.2 / 34.3; heads of 64: 32 on 8,
//        6 at 32768 23.6 / 20.1
//  1024  32 on 8, 6 at 4096 .. 32768 61.8 / 52.2 (with at most 1024 workgroups 56.8), at 65536 58.3 / 55.5
constexpr int kWeighCus = 256;
static int most_rows(const WeighArgs& a) {
  int rows = 1;
  for (int i = 0; i < a.n_entries; ++i) rows = std::max(rows, a.entry[i].n * a.group);
  return rows;
}
// Contexts that a workgroup goes through twice sooner than a second launch has done its part.  us a call in a graph, 32 query heads on
// 8 KV heads, two launches and one: one token at 128, 256, 512 slots 7.9, 8.0, 8.1 and 6.0, 7.7, 11.2, six 10.3, 10.5, 10.7 and
// 7.1, 9.4, 13.4, sixteen sequences of six 10.9, 14.6, 15.7 and 7.4, 9.8, 14.0; but one in fp32 9.3, 9.4 and 8.7, 12.3, sixteen with
// 28 heads on 4 14.0, 14.2 and 11.6, 17.3.
static int weigh_short(int rows, int dtype) { return rows <= 32 && dtype == 1 ? 256 : 128; }
constexpr int kWeighTwoRounds = 2 * 8 * 16;  // slots of two rounds of eight tiles
static int weigh_chunk(const WeighArgs& a, int n_layers, int dtype) {
  const int rows = most_rows(a), groups = rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 ? 4 : 8;
  int longest = 0;
  for (int i = 0; i < a.n_entries; ++i) longest = std::max(longest, a.entry[i].len);
  if (longest <= weigh_short(rows, dtype)) return (longest + 63) / 64 * 64;
  auto cut = [&](long wgs_most) {
    int chunk = 64;
    for (; chunk < kWeighSums / groups; chunk += 64) {
      long wgs = 0;
      for (int i = 0; i < a.n_entries; ++i) wgs += (a.entry[i].len + chunk - 1) / chunk;
      if (wgs * a.heads * n_layers <= wgs_most) break;
    }
    return chunk;
  };
  if (groups == 2 && dtype == 1) {
    const int chunk = cut(2 * kWeighCus);
    if (chunk > kWeighTwoRounds) return chunk;
  }
  return cut(kWeighCus);
}

// Fills in how the entries (seq, n, len, q_first are set) are cut.
void weigh_plan(WeighArgs& a, int n_layers, int dtype) {
  a.chunk = weigh_chunk(a, n_layers, dtype);
  a.inv_group = 1.f / (float)a.group;
  int wg = 0;
  size_t stat = 0;
  for (int i = 0; i < kMaxCols; ++i) {
    a.first_wg[i] = INT32_MAX;
    if (i >= a.n_entries) continue;
    WeighEntry& e = a.entry[i];
    e.chunks = (e.len + a.chunk - 1) / a.chunk;
    e.first_stat = stat;
    a.first_wg[i] = wg;
    wg += e.chunks;
    stat += (size_t)e.n * a.group * e.chunks;
  }
  a.n_wgs = wg;
  a.stats_pitch = stat;
}
size_t weigh_workspace_bytes(const WeighArgs& a, int n_layers) { return a.stats_pitch * a.heads * n_layers * sizeof(float2); }

size_t weigh_workspace_limit(int B, int heads, int group, int max_tokens, int max_slots) {
  const size_t least = kWeighSums / kWeighMaxTiles;  // contexts too long for that many workgroups are cut into chunks of at least this
  const size_t wgs = std::max((size_t)2 * kWeighCus, (size_t)B * heads * ((max_slots + least - 1) / least));
  return wgs * max_tokens * group * sizeof(float2);
}

void launch_weigh(const WeighArgs& a, int n_layers, int dtype, int hd, hipStream_t st) {
  if (a.n_entries == 0) return;
  const dim3 grid(a.n_wgs, a.heads, n_layers);
  bool one_chunk = true;
  for (int i = 0; i < a.n_entries; ++i) one_chunk = one_chunk && a.entry[i].chunks == 1;
  auto go = [&](auto waves, auto stats, auto add, auto both) {
    const dim3 block(decltype(waves)::value * 64);
    if (one_chunk) {
      ES_LAUNCH(both, grid, block, 0, st, a);
      return;
    }
    ES_LAUNCH(stats, grid, block, 0, st, a);
    ES_LAUNCH(add, grid, block, 0, st, a);
  };
  typedef std::integral_constant<int, 4> Four;
  typedef std::integral_constant<int, 8> Eight;
  const bool narrow = most_rows(a) <= 16;
  DISPATCH_T(dtype, {
    if (hd == 128 && narrow) go(Four{}, weigh_stats_kernel<T, 128, 4>, weigh_add_kernel<T, 128, 4>, weigh_short_kernel<T, 128, 4>);
    else if (hd == 128) go(Eight{}, weigh_stats_kernel<T, 128, 8>, weigh_add_kernel<T, 128, 8>, weigh_short_kernel<T, 128, 8>);
    else if (narrow) go(Four{}, weigh_stats_kernel<T, 64, 4>, weigh_add_kernel<T, 64, 4>, weigh_short_kernel<T, 64, 4>);
    else go(Eight{}, weigh_stats_kernel<T, 64, 8>, weigh_add_kernel<T, 64, 8>, weigh_short_kernel<T, 64, 8>);
  });
}

}  // namespace es
