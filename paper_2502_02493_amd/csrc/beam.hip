// Selection over beams and vocabulary (gfx950): the n_select best continuations of every group of beams.
//
//   score(w, v) = c_w + l_w[v] / T - log sum_u exp(l_w[u] / T),  descending; of equal scores the lowest beam, of one beam's the
//   highest logit, of equal logits the lowest token.
//
// Which candidate comes first is decided by comparing scores of different beams, so they are formed in double precision; inside
// a beam the order is that of the fp32 logits themselves.  Two launches:
//   (1) beam_slice_kernel  per beam and vocabulary slice: slice maximum and sum of exp((l - max) / T), and the slice's n_select
//                          highest logits in order.  A thread holds its logits in registers: the slice is read once.
//   (2) beam_pick_kernel   per group: the beams' sums from their slices', then the best of the slices' lists.
#include "kernels.h"
#include "lane_ops.hpp"

namespace es {

constexpr int kSliceThreads = 512, kSliceRegs = 8, kSliceMax = kSliceThreads * kSliceRegs;
constexpr int kListMax = 1024;  // candidates ranked in LDS
constexpr int kPickThreads = 1024;

// A candidate of (1): logit and token as one number whose order is that of the candidates of a beam.  0: none.
typedef unsigned long long cand_t;
__device__ __forceinline__ uint32_t ordered_bits(float f) {  // order-preserving; not 0 for anything but a NaN of all ones
  const uint32_t u = __float_as_uint(f + 0.f);               // -0 and 0 are one logit
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ unsigned long long ordered_bits(double f) {
  const unsigned long long u = __builtin_bit_cast(unsigned long long, f + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ cand_t make_cand(float logit, int token) {
  if (!(logit > -INFINITY)) return 0;  // minus infinity and NaN are no candidates
  return (cand_t)ordered_bits(logit) << 32 | (uint32_t)~token;
}
__device__ __forceinline__ int cand_token(cand_t c) { return (int)~(uint32_t)c; }
__device__ __forceinline__ float cand_logit(cand_t c) {
  const uint32_t k = (uint32_t)(c >> 32);
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// Slices of a row: as many as it takes for a thread to hold kSliceRegs logits, more while the workgroups are fewer than the CUs.
static int beam_slices(long rows, int V) {
  int slices = (V + kSliceMax - 1) / kSliceMax;
  while (rows * slices < 256 && V >= 2 * slices * kSliceThreads) slices *= 2;
  return slices;
}

// Workspace: [rows][slices][2] doubles (maximum, sum), then [rows][slices][n_select] candidates.
size_t beam_select_workspace_bytes(int groups, int beams, int V, int n_select) {
  const long rows = (long)groups * beams;
  return (size_t)rows * beam_slices(rows, V) * (2 * sizeof(double) + n_select * sizeof(cand_t));
}

struct BeamArgs {
  const float* logits;
  const float* scores;
  const int32_t* ended;
  int beams, V, n_select, slices, end_token;
  double inv_T;
  double* stats;
  cand_t* cands;
  int32_t* tokens_out;
  int32_t* parents_out;
  float* scores_out;
};

// grid (slices, rows)
__global__ __launch_bounds__(kSliceThreads) void beam_slice_kernel(BeamArgs a) {
  constexpr int NW = kSliceThreads / 64;
  __shared__ double sh_d[NW];
  __shared__ float sh_f[NW];
  __shared__ cand_t s_list[kListMax];
  __shared__ int s_n, s_wave[NW];
  const int slice = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (!(a.scores[row] > -INFINITY) || (a.ended && a.ended[row])) return;  // (2) looks at neither
  const float* l_row = a.logits + (size_t)row * a.V;
  const int per = (a.V + a.slices - 1) / a.slices, v0 = min(a.V, slice * per), v1 = min(a.V, v0 + per);
  float l[kSliceRegs];
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i) {
    const int v = v0 + i * kSliceThreads + tid;
    l[i] = v < v1 ? l_row[v] : -INFINITY;
    l[i] = l[i] == l[i] ? l[i] : -INFINITY;
  }
  float mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i) mx = fmaxf(mx, l[i]);
  mx = block_max<NW>(mx, sh_f);
  const double ref = mx == -INFINITY ? 0.0 : (double)mx;
  double z = 0.0;
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i)
    if (v0 + i * kSliceThreads < v1) z += exp(((double)l[i] - ref) * a.inv_T);  // uniform; slots past the end add 0
  z = block_sum<NW>(z, sh_d);
  const size_t at = (size_t)row * a.slices + slice;
  if (tid == 0) {
    a.stats[2 * at] = (double)mx;
    a.stats[2 * at + 1] = z;
  }
  // The n_select highest.  A bound from below: of at least n_select groups of threads the lowest maximum, which as many logits
  // reach.  Few more do: with 16 groups of 256 logits some 50 of 4096.
  const int lanes = a.n_select <= NW ? 64 : a.n_select <= 2 * NW ? 32 : a.n_select <= 4 * NW ? 16 : 8;
  float own = l[0];
#pragma unroll
  for (int i = 1; i < kSliceRegs; ++i) own = fmaxf(own, l[i]);
  own = lanes_max(own, lanes);
  for (int off = lanes; off < 64; off <<= 1) own = fminf(own, __shfl_xor(own, off, 64));
  if (lane == 0) sh_f[wave] = own;
  if (tid == 0) s_n = 0;
  __syncthreads();
  float bound = sh_f[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) bound = fminf(bound, sh_f[w]);
  auto cand = [&](int i) { return make_cand(l[i], v0 + i * kSliceThreads + tid); };  // none past the slice: minus infinity
  auto collect = [&](auto&& reaches) {
#pragma unroll
    for (int i = 0; i < kSliceRegs; ++i)
      if (reaches(i)) {
        const int at_n = atomicAdd(&s_n, 1);
        if (at_n < kListMax) s_list[at_n] = cand(i);
      }
    __syncthreads();
  };
  collect([&](int i) { return l[i] >= bound && l[i] > -INFINITY; });
  if (s_n > kListMax) {
    // Many equal logits, or groups that a mask empties: the n_select-th candidate itself, bit by bit
    cand_t least = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const cand_t t = least | (cand_t)1 << bit;
      int n = 0;
#pragma unroll
      for (int i = 0; i < kSliceRegs; ++i) n += __popcll(__ballot(cand(i) >= t));
      __syncthreads();
      if (lane == 0) s_wave[wave] = n;
      __syncthreads();
      n = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) n += s_wave[w];
      if (n >= a.n_select) least = t;
    }
    __syncthreads();
    if (tid == 0) s_n = 0;
    __syncthreads();
    collect([&](int i) { return cand(i) >= least && cand(i) != 0; });
  }
  // in order: a candidate's place is the number of those above it
  const int n = s_n;
  cand_t* list = a.cands + at * a.n_select;
  for (int i = tid; i < n; i += kSliceThreads) {
    const cand_t c = s_list[i];
    int above = 0;
    for (int j = 0; j < n; ++j) above += s_list[j] > c;
    if (above < a.n_select) list[above] = c;
  }
  if (tid >= n && tid < a.n_select) list[tid] = 0;
}

// A candidate of (2).  Order: score, then beam, then what (1) goes by.
struct Pick {
  double score;
  cand_t cand;
  int beam;
};
__device__ __forceinline__ bool before(const Pick& a, const Pick& b) {
  return a.score != b.score ? a.score > b.score : a.beam != b.beam ? a.beam < b.beam : a.cand > b.cand;
}

// grid (groups)
__global__ __launch_bounds__(kPickThreads) void beam_pick_kernel(BeamArgs a) {
  constexpr int NW = kPickThreads / 64;
  __shared__ double s_top[kMaxBeams], s_log[kMaxBeams], s_cum[kMaxBeams];
  __shared__ Pick s_list[kListMax];
  __shared__ unsigned long long s_bound[kMaxSelect];
  __shared__ int s_n;
  __shared__ int s_kind[kMaxBeams];  // 0 no candidates, 1 its lists, 2 the end token alone
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, S = a.slices, K = a.n_select;
  for (int w = wave; w < a.beams; w += NW) {
    const int row = g * a.beams + w;
    const float cum = a.scores[row];
    const int kind = !(cum > -INFINITY) ? 0 : a.ended && a.ended[row] ? 2 : 1;
    double top = -INFINITY, sum = 0.0;
    if (kind == 1) {
      const double* st = a.stats + (size_t)row * S * 2;
      float m = -INFINITY;
      for (int s = lane; s < S; s += 64) m = fmaxf(m, (float)st[2 * s]);
      top = (double)lanes_max(m, 64);
      for (int s = lane; s < S; s += 64)
        if (st[2 * s] > -INFINITY) sum += st[2 * s + 1] * exp((st[2 * s] - top) * a.inv_T);
      sum = lanes_sum(sum, 64);
    }
    if (lane == 0) {
      s_kind[w] = kind;
      s_top[w] = top;
      s_log[w] = kind == 1 ? log(sum) : 0.0;
      s_cum[w] = (double)cum;
    }
  }
  if (tid < kMaxSelect) s_bound[tid] = 0;
  if (tid == 0) s_n = 0;
  __syncthreads();
  // a list: (beam, slice); an ended beam is one of a single candidate
  const int lists = a.beams * S;
  const cand_t* cands = a.cands + (size_t)g * lists * K;
  auto entry = [&](int i, int j, Pick& p) {  // the j-th candidate of list i; false: there is none
    const int w = i / S, s = i - w * S;
    p.beam = w;
    if (s_kind[w] == 1) {
      p.cand = j < K ? cands[(size_t)i * K + j] : 0;
      p.score = s_cum[w] + (((double)cand_logit(p.cand) - s_top[w]) * a.inv_T - s_log[w]);
      return p.cand != 0 && p.score > -INFINITY;  // a beam without a distribution offers nothing
    }
    p.cand = (cand_t)1 << 63 | (uint32_t)~a.end_token;
    p.score = s_cum[w];
    return s_kind[w] == 2 && s == 0 && j == 0;
  };
  // As in (1): the lists' first candidates dealt to at least n_select groups, and the lowest of the groups' maxima.
  const int groups = K <= 16 ? 16 : K <= 32 ? 32 : 64;
  const int depth = min(K, (2 * groups + lists - 1) / lists);
  for (int i = tid; i < lists; i += kPickThreads)
    for (int j = 0; j < depth; ++j) {
      Pick p;
      if (!entry(i, j, p)) break;
      atomicMax(&s_bound[(i * depth + j) & (groups - 1)], ordered_bits(p.score));
    }
  __syncthreads();
  unsigned long long bound = ~0ull;
  for (int i = 0; i < groups; ++i) bound = min(bound, s_bound[i]);
  for (int i = tid; i < lists; i += kPickThreads)
    for (int j = 0; j < K; ++j) {
      Pick p;
      if (!entry(i, j, p) || ordered_bits(p.score) < bound) break;
      const int at = atomicAdd(&s_n, 1);
      if (at < kListMax) s_list[at] = p;
    }
  __syncthreads();
  const int n = s_n;
  auto write = [&](int k, const Pick& p) {
    a.tokens_out[(size_t)g * K + k] = cand_token(p.cand);
    a.parents_out[(size_t)g * K + k] = p.beam;
    a.scores_out[(size_t)g * K + k] = (float)p.score;
  };
  if (n <= kListMax) {
    for (int i = tid; i < n; i += kPickThreads) {
      const Pick p = s_list[i];
      int above = 0;
      for (int j = 0; j < n; ++j) above += before(s_list[j], p);
      if (above < K) write(above, p);
    }
    if (tid >= n && tid < K) {
      a.tokens_out[(size_t)g * K + tid] = a.parents_out[(size_t)g * K + tid] = -1;
      a.scores_out[(size_t)g * K + tid] = -INFINITY;
    }
    return;
  }
  // Many equal scores: the best head of the lists, K times (there are more than K candidates)
  Pick taken = {INFINITY, 0, -1};  // everything that comes before it has been handed out
  for (int k = 0; k < K; ++k) {
    Pick best = {-INFINITY, 0, kMaxBeams};
    for (int i = tid; i < lists; i += kPickThreads)
      for (int j = 0; j < K; ++j) {
        Pick p;
        if (!entry(i, j, p)) break;
        if (!before(taken, p)) continue;
        if (before(p, best)) best = p;
        break;
      }
    for (int off = 32; off > 0; off >>= 1) {
      const Pick o = {__shfl_xor(best.score, off, 64), (cand_t)__shfl_xor((unsigned long long)best.cand, off, 64), __shfl_xor(best.beam, off, 64)};
      if (before(o, best)) best = o;
    }
    __syncthreads();
    if (lane == 0) s_list[wave] = best;
    __syncthreads();
    for (int w = 0; w < NW; ++w)
      if (before(s_list[w], best)) best = s_list[w];
    if (tid == 0) write(k, best);
    taken = best;
  }
}

void launch_beam_select(const float* logits, const float* scores, const int32_t* ended, int groups, int beams, int V, int n_select,
                        double T, int end_token, int32_t* tokens_out, int32_t* parents_out, float* scores_out, void* ws, hipStream_t st) {
  BeamArgs a;
  const long rows = (long)groups * beams;
  a.logits = logits; a.scores = scores; a.ended = ended; a.beams = beams; a.V = V; a.n_select = n_select; a.end_token = end_token;
  a.slices = beam_slices(rows, V);
  a.inv_T = 1.0 / T;
  a.stats = (double*)ws;
  a.cands = (cand_t*)(a.stats + (size_t)rows * a.slices * 2);
  a.tokens_out = tokens_out; a.parents_out = parents_out; a.scores_out = scores_out;
  hipLaunchKernelGGL(beam_slice_kernel, dim3(a.slices, (unsigned)rows), dim3(kSliceThreads), 0, st, a);
  hipLaunchKernelGGL(beam_pick_kernel, dim3(groups), dim3(kPickThreads), 0, st, a);
}

}  // namespace es
