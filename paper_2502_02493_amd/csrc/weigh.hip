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
#include "launch_common.hpp"

#include <string.h>

namespace es {

constexpr int kWeighThreads = 256, kWeighWaves = kWeighThreads / 64;
constexpr int kWeighTileRows = 2;  // row tiles a wave holds the queries of

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

// One workgroup: a chunk of one sequence's context, one KV head, one layer.
struct WeighPlace {
  int e, h, l, c;         // entry, KV head, layer, chunk
  int rows, old, len;     // query rows; slots that were there before; slots
  int s0, s1;             // the chunk
  int tiles, groups, splits, group, split;  // row tiles; waves share them out in groups, and the slots inside a group
};
__device__ __forceinline__ WeighPlace weigh_place(const WeighArgs& a) {
  WeighPlace p;
  p.e = 0;
#pragma unroll
  for (int i = 1; i < kMaxCols; ++i) p.e += (int)blockIdx.x >= a.entry[i].first_wg;
  const WeighEntry& e = a.entry[p.e];
  p.c = blockIdx.x - e.first_wg;
  p.h = blockIdx.y;
  p.l = blockIdx.z;
  p.rows = e.n * a.group;
  p.len = e.len;
  p.old = e.len - e.n;
  p.s0 = p.c * a.chunk;
  p.s1 = min(p.len, p.s0 + a.chunk);
  p.tiles = (p.rows + 15) / 16;
  p.groups = p.tiles <= kWeighTileRows ? 1 : p.tiles <= 2 * kWeighTileRows ? 2 : 4;
  p.splits = kWeighWaves / p.groups;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  p.group = wave % p.groups;
  p.split = wave / p.groups;
  return p;
}

// The queries of the wave's row tiles as B fragments: lane l holds row l % 16, elements (l / 16) EPL .. of every k tile.  Rows past
// the last take the last one's queries; their scores are not used.
template <typename T, int HD>
struct WeighQueries {
  typedef WeighGeom<T, HD> Geo;
  u32x4 q[kWeighTileRows][Geo::NKT][Geo::TERMS];
  int seen[kWeighTileRows];  // slots that the lane's row attends to; 0: no row

  __device__ __forceinline__ void load(const WeighArgs& a, const WeighPlace& p) {
    const int lane = threadIdx.x & 63;
    const WeighEntry& e = a.entry[p.e];
#pragma unroll
    for (int t = 0; t < kWeighTileRows; ++t) {
      const int row = (p.group + t * p.groups) * 16 + (lane & 15);
      const bool there = row < p.rows;
      const int r = min(row, p.rows - 1), tok = r / a.group, g = r - tok * a.group;
      seen[t] = there ? p.old + tok + 1 : 0;
      const float* src = a.q + p.l * a.q_layer_pitch + ((size_t)(e.q_first + tok) * a.Hq + p.h * a.group + g) * HD + (lane >> 4) * Geo::EPL;
#pragma unroll
      for (int kt = 0; kt < Geo::NKT; ++kt) {
        if constexpr (Geo::TERMS == 3) {
          float x[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = src[kt * Geo::KT + j];
          bf16x8 hi, lo;
          split_bf16x8(x, hi, lo);
          q[t][kt][0] = __builtin_bit_cast(u32x4, hi);
          q[t][kt][1] = __builtin_bit_cast(u32x4, lo);
          q[t][kt][2] = __builtin_bit_cast(u32x4, third_bf16x8(x, hi, lo));
        } else {
          q[t][kt][0] = *reinterpret_cast<const u32x4*>(src + kt * Geo::KT);
        }
      }
    }
  }
};

// K fragments of the 16 slots from s on: lane l holds slot s + l % 16.  Slots past the last fetch the last one.
template <typename T, int HD>
__device__ __forceinline__ void load_keys(const T* k_row, int s, int len, u32x4 (&kf)[HD / Tr<T>::KT]) {
  const int lane = threadIdx.x & 63;
  const T* src = k_row + (size_t)min(s + (lane & 15), len - 1) * HD + (lane >> 4) * Tr<T>::EPL;
#pragma unroll
  for (int kt = 0; kt < HD / Tr<T>::KT; ++kt) kf[kt] = *reinterpret_cast<const u32x4*>(src + kt * Tr<T>::KT);
}

// element i of the lane: score of slot s + 4 (l / 16) + i in the lane's row
template <typename T, int HD>
__device__ __forceinline__ f32x4 scores_of(const u32x4 (&kf)[HD / Tr<T>::KT], const u32x4 (&q)[WeighGeom<T, HD>::NKT][WeighGeom<T, HD>::TERMS]) {
  typedef WeighGeom<T, HD> Geo;
  f32x4 s = {0.f, 0.f, 0.f, 0.f}, s1 = s, s2 = s;
#pragma unroll
  for (int kt = 0; kt < Geo::NKT; ++kt) {
    mma<T>(s, kf[kt], q[kt][0]);
    if constexpr (Geo::TERMS == 3) {
      mma<T>(s1, kf[kt], q[kt][1]);
      mma<T>(s2, kf[kt], q[kt][2]);
    }
  }
  if constexpr (Geo::TERMS == 3) s += s1 + s2;
  return s;
}

__device__ __forceinline__ float ref_of(float m) { return m == -INFINITY ? 0.f : m; }  // nothing yet: exp(-inf - 0) = 0

// grid (chunks of all entries, KV heads, layers)
template <typename T, int HD>
__global__ __launch_bounds__(kWeighThreads) void weigh_stats_kernel(WeighArgs a) {
  __shared__ float s_m[kWeighWaves][kWeighTileRows][16], s_l[kWeighWaves][kWeighTileRows][16];
  const WeighPlace p = weigh_place(a);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T* k_row = reinterpret_cast<const T*>(a.k) + (((size_t)p.l * a.n_seqs + a.entry[p.e].seq) * a.heads + p.h) * (size_t)a.max_slots * HD;
  WeighQueries<T, HD> Q;
  Q.load(a, p);
  float m[kWeighTileRows], l[kWeighTileRows];
#pragma unroll
  for (int t = 0; t < kWeighTileRows; ++t) m[t] = -INFINITY, l[t] = 0.f;
  for (int s = p.s0 + 16 * p.split; s < p.s1; s += 16 * p.splits) {
    u32x4 kf[HD / Tr<T>::KT];
    load_keys<T, HD>(k_row, s, p.len, kf);
#pragma unroll
    for (int t = 0; t < kWeighTileRows; ++t) {
      if (p.group + t * p.groups >= p.tiles) break;
      f32x4 x = scores_of<T, HD>(kf, Q.q[t]);
      float top = m[t];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = s + 4 * (lane >> 4) + i < Q.seen[t] ? x[i] * a.scale : -INFINITY;
        top = fmaxf(top, x[i]);
      }
      const float ref = ref_of(top);
      float sum = l[t] * __expf(m[t] - ref);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += __expf(x[i] - ref);
      m[t] = top;
      l[t] = sum;
    }
  }
  // the four lanes of a row, then the waves that share its tile
#pragma unroll
  for (int t = 0; t < kWeighTileRows; ++t) {
    for (int off = 16; off < 64; off <<= 1) {
      const float om = __shfl_xor(m[t], off, 64), ol = __shfl_xor(l[t], off, 64);
      const float top = fmaxf(m[t], om), ref = ref_of(top);
      l[t] = l[t] * __expf(m[t] - ref) + ol * __expf(om - ref);
      m[t] = top;
    }
    if (lane < 16) {
      s_m[wave][t][lane] = m[t];
      s_l[wave][t][lane] = l[t];
    }
  }
  __syncthreads();
  for (int r = threadIdx.x; r < p.rows; r += kWeighThreads) {
    const int tile = r / 16, grp = tile % p.groups, t = tile / p.groups;
    float top = -INFINITY;
    for (int w = 0; w < p.splits; ++w) top = fmaxf(top, s_m[w * p.groups + grp][t][r % 16]);
    const float ref = ref_of(top);
    float sum = 0.f;
    for (int w = 0; w < p.splits; ++w) sum += s_l[w * p.groups + grp][t][r % 16] * __expf(s_m[w * p.groups + grp][t][r % 16] - ref);
    const WeighEntry& e = a.entry[p.e];
    float2* out = a.stats + ((size_t)p.l * a.heads + p.h) * a.stats_pitch + e.first_stat + (size_t)r * e.chunks + p.c;
    *out = make_float2(top, sum);
  }
}

// grid as above
template <typename T, int HD>
__global__ __launch_bounds__(kWeighThreads) void weigh_add_kernel(WeighArgs a) {
  constexpr int kMaxRows = kWeighWaves * kWeighTileRows * 16;
  __shared__ float s_m[kMaxRows], s_inv[kMaxRows];
  __shared__ float s_sum[kWeighWaves][kWeighMaxChunk];
  const WeighPlace p = weigh_place(a);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const WeighEntry& e = a.entry[p.e];
  const size_t row_at = (((size_t)p.l * a.n_seqs + e.seq) * a.heads + p.h) * (size_t)a.max_slots;
  const T* k_row = reinterpret_cast<const T*>(a.k) + row_at * HD;
  WeighQueries<T, HD> Q;
  Q.load(a, p);
  for (int r = wave; r < p.rows; r += kWeighWaves) {
    const float2* st = a.stats + ((size_t)p.l * a.heads + p.h) * a.stats_pitch + e.first_stat + (size_t)r * e.chunks;
    float m = -INFINITY, l = 0.f;
    for (int c = lane; c < e.chunks; c += 64) {
      const float2 x = st[c];
      const float top = fmaxf(m, x.x), ref = ref_of(top);
      l = l * __expf(m - ref) + x.y * __expf(x.x - ref);
      m = top;
    }
    for (int off = 1; off < 64; off <<= 1) {
      const float om = __shfl_xor(m, off, 64), ol = __shfl_xor(l, off, 64);
      const float top = fmaxf(m, om), ref = ref_of(top);
      l = l * __expf(m - ref) + ol * __expf(om - ref);
      m = top;
    }
    if (lane == 0) {
      s_m[r] = m;
      s_inv[r] = 1.f / l;
    }
  }
  __syncthreads();
  float m[kWeighTileRows], inv[kWeighTileRows];
#pragma unroll
  for (int t = 0; t < kWeighTileRows; ++t) {
    const int r = min((p.group + t * p.groups) * 16 + (lane & 15), p.rows - 1);
    m[t] = s_m[r];
    inv[t] = s_inv[r];
  }
  for (int s = p.s0 + 16 * p.split; s < p.s1; s += 16 * p.splits) {
    u32x4 kf[HD / Tr<T>::KT];
    load_keys<T, HD>(k_row, s, p.len, kf);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < kWeighTileRows; ++t) {
      if (p.group + t * p.groups >= p.tiles) break;
      const f32x4 x = scores_of<T, HD>(kf, Q.q[t]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float prob = __expf(x[i] * a.scale - m[t]) * inv[t];
        sum[i] += s + 4 * (lane >> 4) + i < Q.seen[t] ? prob : 0.f;
      }
    }
    for (int off = 1; off < 16; off <<= 1)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], off, 64);
    if ((lane & 15) == 0) *reinterpret_cast<f32x4*>(&s_sum[p.group][s - p.s0 + 4 * (lane >> 4)]) = sum;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.s1 - p.s0; i += kWeighThreads) {
    float sum = 0.f;
    for (int g = 0; g < p.groups; ++g) sum += s_sum[g][i];
    const int s = p.s0 + i;
    const float before = a.w_in && s < p.old ? a.w_in[row_at + s] : 0.f;  // the new tokens' slots start from nothing
    a.w_out[row_at + s] = before + sum;
  }
}

constexpr long kWeighMostWgs = 2048;

// Chunks: short enough that the workgroups fill the chip several times over, from one tile per wave up.
static int weigh_chunk(const WeighArgs& a, int n_layers) {
  int chunk = 64;
  for (; chunk < kWeighMaxChunk; chunk *= 2) {
    long wgs = 0;
    for (int i = 0; i < a.n_entries; ++i) wgs += (a.entry[i].len + chunk - 1) / chunk;
    if (wgs * a.heads * n_layers <= kWeighMostWgs) break;
  }
  return chunk;
}

// Fills in how the entries (seq, n, len, q_first are set) are cut.
void weigh_plan(WeighArgs& a, int n_layers) {
  a.chunk = weigh_chunk(a, n_layers);
  int wg = 0;
  size_t stat = 0;
  for (int i = 0; i < kMaxCols; ++i) {
    WeighEntry& e = a.entry[i];
    if (i >= a.n_entries) {
      memset(&e, 0, sizeof e);
      e.first_wg = INT32_MAX;
      continue;
    }
    e.chunks = (e.len + a.chunk - 1) / a.chunk;
    e.first_wg = wg;
    e.first_stat = stat;
    wg += e.chunks;
    stat += (size_t)e.n * a.group * e.chunks;
  }
  a.n_wgs = wg;
  a.stats_pitch = stat;
}
size_t weigh_workspace_bytes(const WeighArgs& a, int n_layers) { return a.stats_pitch * a.heads * n_layers * sizeof(float2); }

size_t weigh_workspace_limit(int max_tokens, int B, int heads, int group, int max_slots) {
  const size_t wgs = std::max((size_t)kWeighMostWgs, (size_t)B * heads * ((max_slots + kWeighMaxChunk - 1) / kWeighMaxChunk));
  return wgs * max_tokens * group * sizeof(float2);
}

void launch_weigh(const WeighArgs& a, int n_layers, int dtype, int hd, hipStream_t st) {
  if (a.n_entries == 0) return;
  DISPATCH_T(dtype, {
    const dim3 grid(a.n_wgs, a.heads, n_layers);
    if (hd == 128) {
      hipLaunchKernelGGL((weigh_stats_kernel<T, 128>), grid, dim3(kWeighThreads), 0, st, a);
      hipLaunchKernelGGL((weigh_add_kernel<T, 128>), grid, dim3(kWeighThreads), 0, st, a);
    } else {
      hipLaunchKernelGGL((weigh_stats_kernel<T, 64>), grid, dim3(kWeighThreads), 0, st, a);
      hipLaunchKernelGGL((weigh_add_kernel<T, 64>), grid, dim3(kWeighThreads), 0, st, a);
    }
  });
}

}  // namespace es
