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
constexpr int kPickThreads = 1024;

// A candidate of (1): logit and token as one number whose order is that of the candidates of a beam.  0: none.
typedef unsigned long long cand_t;
__device__ __forceinline__ uint32_t ordered_bits(float f) {  // order-preserving; not 0 for anything but a NaN of all ones
  const uint32_t u = __float_as_uint(f + 0.f);               // -0 and 0 are one logit
  return u & 0x80000000u ? ~u : u | 0x80000000u;
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
  __shared__ cand_t sh_c[NW];
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
  // the n_select highest, one after the other
  cand_t c[kSliceRegs];
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i) c[i] = v0 + i * kSliceThreads + tid < v1 ? make_cand(l[i], v0 + i * kSliceThreads + tid) : 0;
  for (int k = 0; k < a.n_select; ++k) {
    cand_t best = 0;
#pragma unroll
    for (int i = 0; i < kSliceRegs; ++i) best = max(best, c[i]);
    for (int off = 32; off > 0; off >>= 1) best = max(best, (cand_t)__shfl_xor((unsigned long long)best, off, 64));
    __syncthreads();
    if (lane == 0) sh_c[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) best = max(best, sh_c[w]);
    if (tid == 0) a.cands[at * a.n_select + k] = best;
#pragma unroll
    for (int i = 0; i < kSliceRegs; ++i) c[i] = c[i] == best ? 0 : c[i];
  }
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

// grid (groups): the slices' lists merged, the best head at a time.
__global__ __launch_bounds__(kPickThreads) void beam_pick_kernel(BeamArgs a) {
  constexpr int NW = kPickThreads / 64;
  __shared__ double s_top[kMaxBeams], s_log[kMaxBeams], s_cum[kMaxBeams];
  __shared__ Pick s_best[NW];
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
  __syncthreads();
  const Pick none = {-INFINITY, 0, kMaxBeams};
  // a list: (beam, slice); an ended beam is a list of one.  The thread's lists: tid, tid + kPickThreads, ...
  const int lists = a.beams * S;
  Pick taken = {INFINITY, 0, -1};  // everything that comes before it has been handed out
  for (int k = 0; k < K; ++k) {
    Pick best = none;
    for (int i = tid; i < lists; i += kPickThreads) {
      const int w = i / S, s = i - w * S;
      if (s_kind[w] == 0 || (s_kind[w] == 2 && s > 0)) continue;
      if (s_kind[w] == 2) {
        const Pick p = {s_cum[w], (cand_t)1 << 63 | (uint32_t)~a.end_token, w};
        if (before(taken, p) && before(p, best)) best = p;
        continue;
      }
      const cand_t* list = a.cands + ((size_t)(g * a.beams + w) * S + s) * K;
      for (int j = 0; j < K; ++j) {
        const cand_t c = list[j];
        if (!c) break;
        const Pick p = {s_cum[w] + (((double)cand_logit(c) - s_top[w]) * a.inv_T - s_log[w]), c, w};
        if (!(p.score > -INFINITY)) break;  // a beam without a distribution
        if (!before(taken, p)) continue;
        if (before(p, best)) best = p;
        break;
      }
    }
    for (int off = 32; off > 0; off >>= 1) {
      const Pick o = {__shfl_xor(best.score, off, 64), (cand_t)__shfl_xor((unsigned long long)best.cand, off, 64), __shfl_xor(best.beam, off, 64)};
      if (before(o, best)) best = o;
    }
    __syncthreads();
    if (lane == 0) s_best[wave] = best;
    __syncthreads();
    for (int w = 0; w < NW; ++w)
      if (before(s_best[w], best)) best = s_best[w];
    if (tid == 0) {
      const bool any = best.beam < kMaxBeams;
      a.tokens_out[(size_t)g * K + k] = any ? cand_token(best.cand) : -1;
      a.parents_out[(size_t)g * K + k] = any ? best.beam : -1;
      a.scores_out[(size_t)g * K + k] = any ? (float)best.score : -INFINITY;
    }
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
