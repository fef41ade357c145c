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
// Neither sorts: a bound from below that at least n_select candidates reach (the lowest maximum of as many disjoint groups) leaves
// some n_select ln(n_select) of them, whose places are counted.  Taking the best n_select times over, one workgroup-wide maximum
// after the other, was 78 us a call (128 256 words, sixteen beams, the sixteen best), this is 15.1; 64 beams in sixteen groups of
// 152 064 words 66 and 19.4.
// Bound by the chain of dependent steps.  Of the 9.9 us of (1) the loads take 1.3, the exponentials 1.0, bound and candidates 1.1, their
// places 1.2, of the 6.0 of (2) statistics and logarithm 2.4, bound 0.8, selection and places 1.9.  The other five of (1) are not
// accounted for: four rows of 1000 words take 5.1 as well, and the compiler spills 45 scalar registers there.  29 MB of logits (48 rows
// that count) take (1) 14.8; a kernel that only reads is through with as much in 7.
// More than 32: a bound that some 250 candidates reach, ranked all against all: sixteen beams, the 64 best, 42 .. 45 us.
#include "launch_common.hpp"
#include "lane_ops.hpp"

namespace es {

constexpr int kSliceThreads = 256, kSliceRegs = 16, kSliceMax = kSliceThreads * kSliceRegs;
constexpr int kListMax = 1024;  // candidates ranked in LDS

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

// Slices of a row: as many as it takes for a thread to hold kSliceRegs logits, more while the workgroups are fewer than the CUs and a
// thread keeps more than one.
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
  double inv_T, log2e_T;
  double* stats;
  cand_t* cands;
  int32_t* tokens_out;
  int32_t* parents_out;
  float* scores_out;
};

// A slice's sum on top of another maximum: sum exp((m - top) / T), top >= m.  Nothing where nothing is finite.
__device__ __forceinline__ double rescaled(double sum, double m, double top, double log2e_T) {
  const double u = (m - top) * log2e_T;
  return u > -1000.0 ? sum * exp2_below(u) : 0.0;
}

// grid (slices, rows)
__global__ __launch_bounds__(kSliceThreads) __attribute__((amdgpu_waves_per_eu(8))) void beam_slice_kernel(BeamArgs a) {
  constexpr int NW = kSliceThreads / 64, kWaveList = kListMax / NW;
  __shared__ u32x2 s_list[NW][kWaveList];  // (token, logit); later the candidates of all waves
  __shared__ int s_above[NW][64];
  __shared__ double s_sum[NW];
  __shared__ float s_max[NW], s_bound[NW];
  __shared__ int s_count[NW];
  const int slice = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (!(a.scores[row] > -INFINITY) || (a.ended && a.ended[row])) return;  // (2) looks at neither
  const float* l_row = a.logits + (size_t)row * a.V;
  const int per = (a.V + a.slices - 1) / a.slices, v0 = min(a.V, slice * per), v1 = min(a.V, v0 + per);
  float l[kSliceRegs];
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i) l[i] = l_row[min(v0 + i * kSliceThreads + tid, a.V - 1)];
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i) l[i] = v0 + i * kSliceThreads + tid < v1 ? l[i] : -INFINITY;
  float own = -INFINITY;  // a maximum passes over NaNs
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i) own = fmaxf(own, l[i]);
  // A bound of the n_select highest from below: of at least n_select groups of neighbouring threads the lowest maximum, which as many
  // logits reach.  Few more do: with 16 groups of 256 logits some 50 of 4096.  A group has its share of every register's logits, so only
  // a slice of fewer logits than threads, or masks, leave one empty; then every logit is a candidate.
  // (For more than 32 the groups were eight threads' halves of the slice, of which the second is empty below 2048 logits: two beams of
  // 128 256 words, 64 of them, 74.9 us a call in a graph, 32.0 with groups of four threads; slices of 4008 words 42 .. 45 both ways.)
  const int lanes = a.n_select <= NW ? 64 : a.n_select <= 2 * NW ? 32 : a.n_select <= 4 * NW ? 16 : a.n_select <= 8 * NW ? 8 : 4;
  const float top = lanes_max(own, 64), least_max = groups_min(lanes == 4 ? quad_max(own) : lanes_max(own, lanes), lanes);
  // Every wave's sum on top of its own maximum: no wait for the others'.  What lies 1000 powers of two below, minus infinities and
  // NaNs among it, counts as 2^-1000.
  const double ref = top == -INFINITY ? 0.0 : (double)top;
  double z = 0.0;
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i) z += exp2_below(fmax(((double)l[i] - ref) * a.log2e_T, -1000.0));
  z = lanes_sum(z, 64);
  if (lane == 0) {
    s_max[wave] = top;
    s_bound[wave] = least_max;
    s_sum[wave] = z;
  }
  __syncthreads();
  const size_t at = (size_t)row * a.slices + slice;
  float bound = s_bound[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) bound = fminf(bound, s_bound[w]);
  bound = fmaxf(bound, -3.4028235e38f);  // minus infinity is no candidate
  auto cand = [&](int i) { return make_cand(l[i], v0 + i * kSliceThreads + tid); };
  // every wave lists its own: no counter, and as a rule a comparison is all there is to do
  int mine = 0;
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i) {
    const unsigned long long who = __ballot(l[i] >= bound);
    if (who) {
      const int place = mine + __popcll(who & ((1ull << lane) - 1));
      if ((who >> lane & 1) && place < kWaveList) s_list[wave][place] = u32x2{(uint32_t)(v0 + i * kSliceThreads + tid), __float_as_uint(l[i])};
      mine += __popcll(who);
    }
  }
  if (lane == 0) s_count[wave] = mine;
  __syncthreads();
  int count[NW], n = 0;
  bool fits = true;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    count[w] = s_count[w];
    fits = fits && count[w] <= kWaveList;
    n += count[w];
  }
  cand_t* list = a.cands + at * a.n_select;
  if (wave == NW - 1) {  // the slice's maximum and sum
    float all = s_max[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) all = fmaxf(all, s_max[w]);
    double sum = 0.0;
    for (int w = 0; w < NW; ++w) sum += rescaled(s_sum[w], s_max[w], all, a.log2e_T);
    if (lane == 0) {
      a.stats[2 * at] = (double)all;
      a.stats[2 * at + 1] = all == INFINITY ? __builtin_nan("") : all == -INFINITY ? 0.0 : sum;
    }
  }
  auto entry = [&](int i) {  // of the waves' lists, one after the other
    int w = 0;
#pragma unroll
    for (int k = 0; k < NW - 1; ++k) {
      const bool next = w == k && i >= count[k];
      i -= next ? count[k] : 0;
      w += next;
    }
    const u32x2 c = s_list[w][max(i, 0)];
    return make_cand(__uint_as_float(c[1]), (int)c[0]);
  };
  // in order: a candidate's place is the number of those above it
  if (n <= 64) {  // as a rule: a lane's candidate each, the others handed round by a quarter of them to a wave
    const cand_t own_c = entry(min(lane, n - 1)), c = lane < n ? own_c : 0;
    int above = 0;
    for (int i = 4 * wave; i < n; i += 4 * NW)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const cand_t o = (cand_t)(uint32_t)__builtin_amdgcn_readlane((int)(c >> 32), i + k) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)c, i + k);
        above += o > c;
      }
    s_above[wave][lane] = above;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < NW; ++w) above += s_above[w][lane];
    if (lane < n && above < a.n_select) list[above] = c;
    if (lane >= n && lane < a.n_select) list[lane] = 0;
    return;
  }
  cand_t* s_flat = reinterpret_cast<cand_t*>(&s_list[0][0]);
  if (fits) {
    cand_t all[kListMax / kSliceThreads];
#pragma unroll
    for (int k = 0; k < kListMax / kSliceThreads; ++k) all[k] = entry(min(tid + k * kSliceThreads, n - 1));
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kListMax / kSliceThreads; ++k)
      if (tid + k * kSliceThreads < n) s_flat[tid + k * kSliceThreads] = all[k];
    __syncthreads();
    for (int i = tid; i < n; i += kSliceThreads) {
      const cand_t c = s_flat[i];
      int above = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) above += s_flat[j] > c;
      if (above < a.n_select) list[above] = c;
    }
    return;
  }
  // Many equal logits, or groups that a mask empties: the n_select-th candidate itself, bit by bit, then those from it on (all logits
  // of sixteen beams of 128 256 words alike: 114 us a call for the sixteen best, with the selection from lists of ties in (2))
  cand_t last = 0;
  for (int bit = 63; bit >= 0; --bit) {
    const cand_t t = last | (cand_t)1 << bit;
    int reach = 0;
#pragma unroll
    for (int i = 0; i < kSliceRegs; ++i) reach += __popcll(__ballot(cand(i) >= t));
    __syncthreads();
    if (lane == 0) s_count[wave] = reach;
    __syncthreads();
    reach = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) reach += s_count[w];
    if (reach >= a.n_select) last = t;
  }
  __syncthreads();
  if (tid == 0) s_count[0] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSliceRegs; ++i)
    if (cand(i) >= last && cand(i) != 0) s_flat[atomicAdd(&s_count[0], 1)] = cand(i);  // n_select of them: candidates are all different
  __syncthreads();
  n = s_count[0];
  if (tid < n) {
    int above = 0;
    for (int j = 0; j < n; ++j) above += s_flat[j] > s_flat[tid];
    list[above] = s_flat[tid];
  }
}

// A candidate of (2) as two numbers whose order is that of the candidates: its score, then beam (the lowest first), logit and token.
static_assert(kMaxBeams <= 64 && kMaxBeamVocab <= 1 << 20, "beam, logit and token share 64 bits");
struct alignas(16) Pick {
  uint64_t score, tie;
};
__device__ __forceinline__ Pick make_pick(double score, int beam, uint32_t logit_bits, int token) {
  return Pick{ordered_bits(score), (uint64_t)(63 - beam) << 52 | (uint64_t)logit_bits << 20 | (uint32_t)(0xFFFFF - token)};
}
__device__ __forceinline__ bool before(const Pick& a, const Pick& b) {
  return (int)(a.score > b.score) | ((int)(a.score == b.score) & (int)(a.tie > b.tie));
}

// grid (groups).  A thread takes a list: (beam, slice); the lists are sorted, and few reach far.
constexpr int kHead = 4;  // candidates of a list that are looked at side by side
template <int NT>
__global__ __launch_bounds__(NT) void beam_pick_kernel(BeamArgs a) {
  constexpr int NW = NT / 64;
  __shared__ double s_top[kMaxBeams], s_log[kMaxBeams], s_cum[kMaxBeams];
  __shared__ int s_kind[kMaxBeams];  // 0 no candidates, 1 its lists, 2 the end token alone
  __shared__ Pick s_list[kListMax];
  __shared__ unsigned long long s_bound[kMaxSelect];
  __shared__ int s_n, s_rank[kListMax];
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), S = a.slices, K = a.n_select;
  const int lists = a.beams * S;
  const cand_t* cands = a.cands + (size_t)g * lists * K;
  cand_t c[kHead];
  auto load_head = [&](int i) {
#pragma unroll
    for (int j = 0; j < kHead; ++j) c[j] = cands[(size_t)min(i, lists - 1) * K + min(j, K - 1)];
  };
  // A wave takes a beam's sums at a time; the first one's are requested in front of the lists, which are needed behind them.
  double m0, z0;
  float cum;
  int ended;
  auto load_beam = [&](int w) {
    const int row = g * a.beams + min(w, a.beams - 1), s0 = min(lane, S - 1);
    m0 = a.stats[((size_t)row * S + s0) * 2];  // of a beam without candidates: whatever is there
    z0 = a.stats[((size_t)row * S + s0) * 2 + 1];
    cum = a.scores[row];
    ended = a.ended ? a.ended[row] : 0;
  };
  load_beam(wave);
  asm volatile("" ::: "memory");
  load_head(tid);
  for (int w = wave; w < a.beams; w += NW) {
    const double* st = a.stats + (size_t)(g * a.beams + w) * S * 2;
    if (w != wave) load_beam(w);
    float m = (float)m0;
    double top = (double)lanes_max(m, 64), sum = lane < S ? rescaled(z0, m0, top, a.log2e_T) : 0.0;
    if (S > 64) {
      for (int s = lane + 64; s < S; s += 64) m = fmaxf(m, (float)st[2 * s]);
      top = (double)lanes_max(m, 64);
      sum = rescaled(z0, m0, top, a.log2e_T);
      for (int s = lane + 64; s < S; s += 64) sum += rescaled(st[2 * s + 1], st[2 * s], top, a.log2e_T);
    }
    sum = lanes_sum(sum, 64);
    if (lane == 0) {
      s_kind[w] = !(cum > -INFINITY) ? 0 : ended ? 2 : 1;
      s_top[w] = top;
      s_log[w] = log(sum);
      s_cum[w] = (double)cum;
    }
  }
  for (int i = tid; i < kListMax; i += NT) s_rank[i] = 0;
  if (tid < kMaxSelect) s_bound[tid] = 0;
  if (tid == 0) s_n = 0;
  __syncthreads();
  auto entry = [&](int w, int s, int j, cand_t cand, Pick& p) {  // the j-th candidate of list (w, s); false: there is none
    if (s_kind[w] == 1) {
      const double score = s_cum[w] + (((double)cand_logit(cand) - s_top[w]) * a.inv_T - s_log[w]);
      p = make_pick(score, w, (uint32_t)(cand >> 32), cand_token(cand));
      return (int)(j < K) & (int)(cand != 0) & (int)(score > -INFINITY);  // a beam without a distribution offers nothing
    }
    p = make_pick(s_cum[w], w, 0, a.end_token);
    return (int)(s_kind[w] == 2) & (int)(s == 0) & (int)(j == 0);
  };
  // As in (1): the heads of the live beams' lists dealt to at least n_select groups, and the lowest of the groups' maxima.  Where
  // these lists are few, the first candidates of each.  A group that stays empty bounds nothing: then there are few lists (all
  // their candidates fit), or lists that masks have emptied.
  const int groups = K <= 8 ? 8 : K <= 16 ? 16 : K <= 32 ? 32 : 64;
  const unsigned long long live = __ballot(lane < a.beams && s_kind[min(lane, a.beams - 1)] == 1);
  const bool heads_do = __popcll(live) * S >= 4 * groups;
  // a thread's (last) list: its beam and the scores of its first candidates, as many as there are
  int list_w = 0;
  Pick head[kHead];
  int there = 0;
  auto look_at = [&](int i) {
    list_w = i / S;
    there = 0;
    bool in = true;
#pragma unroll
    for (int j = 0; j < kHead; ++j) {
      in = (int)in & (int)entry(list_w, i - list_w * S, j, c[j], head[j]);
      there += in;
    }
  };
  for (int i = tid; i < lists; i += NT) {
    if (i >= NT) load_head(i);
    look_at(i);
    const int number = __popcll(live & ((1ull << list_w) - 1)) * S + i - list_w * S;
#pragma unroll
    for (int j = 0; j < kHead; ++j) {
      if (j < there) atomicMax(&s_bound[(heads_do ? number : number * kHead + j) & (groups - 1)], (unsigned long long)head[j].score);
      if (heads_do) break;
    }
  }
  __syncthreads();
  const uint64_t bound = lanes_fold((uint64_t)s_bound[lane & (groups - 1)], groups, [](uint64_t x, uint64_t y) { return x < y ? x : y; });
  for (int i = tid; i < lists; i += NT) {
    if (lists > NT) {
      load_head(i);
      look_at(i);
    }
    int reach = 0;
#pragma unroll
    for (int j = 0; j < kHead; ++j) reach += j < there && head[j].score >= bound;  // sorted: the first ones
    if (reach) {
      int at = atomicAdd(&s_n, reach);
#pragma unroll
      for (int j = 0; j < kHead; ++j, ++at)
        if (j < reach && at < kListMax) s_list[at] = head[j];
    }
    bool in = reach == kHead;
    for (int j = kHead; j < K && in; ++j) {
      Pick q;
      in = (int)entry(list_w, 0, j, cands[(size_t)i * K + j], q) & (int)(q.score >= bound);
      if (in) {
        const int at = atomicAdd(&s_n, 1);
        if (at < kListMax) s_list[at] = q;
      }
    }
  }
  __syncthreads();
  const int n = s_n;
  auto write = [&](int k, const Pick& p) {
    const uint64_t u = p.score >> 63 ? p.score & ~(1ull << 63) : ~p.score;
    a.tokens_out[(size_t)g * K + k] = 0xFFFFF - (int)(p.tie & 0xFFFFF);
    a.parents_out[(size_t)g * K + k] = 63 - (int)(p.tie >> 52);
    a.scores_out[(size_t)g * K + k] = (float)__builtin_bit_cast(double, u);
  };
  if (n <= kListMax) {
    // A candidate's place is the number of those before it: a lane takes one and the waves share out the others.
    for (int j0 = 0; j0 < n; j0 += 64) {
      const Pick own = s_list[min(j0 + lane, n - 1)];
      int above = 0;
#pragma unroll 4
      for (int i = wave; i < n; i += NW) above += before(s_list[i], own);
      if (j0 + lane < n && above) atomicAdd(&s_rank[j0 + lane], above);
    }
    __syncthreads();
    for (int i = tid; i < n; i += NT) {
      const int above = s_rank[i];
      if (above < K) write(above, s_list[i]);
    }
    if (tid >= n && tid < K) {
      a.tokens_out[(size_t)g * K + tid] = a.parents_out[(size_t)g * K + tid] = -1;
      a.scores_out[(size_t)g * K + tid] = -INFINITY;
    }
    return;
  }
  // Many equal scores: the best of the lists, K times (there are more than K candidates).  Every time a thread goes through its lists
  // up to the first candidate that is left: K times K steps for a list that holds all of the best.  All logits alike, the 64 best of
  // sixteen beams of 128 256 words 657 us a call, of 64 beams of 152 064 886.
  Pick taken = {~0ull, ~0ull};  // everything that comes before it has been handed out
  for (int k = 0; k < K; ++k) {
    Pick best = {0, 0};
    for (int i = tid; i < lists; i += NT)
      for (int j = 0; j < K; ++j) {
        Pick p;
        if (!entry(i / S, i % S, j, cands[(size_t)i * K + j], p)) break;
        if (!before(taken, p)) continue;
        if (before(p, best)) best = p;
        break;
      }
    for (int off = 32; off > 0; off >>= 1) {
      const Pick o = {(uint64_t)__shfl_xor((unsigned long long)best.score, off, 64), (uint64_t)__shfl_xor((unsigned long long)best.tie, off, 64)};
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
  a.log2e_T = 1.4426950408889634 / T;
  a.stats = (double*)ws;
  a.cands = (cand_t*)(a.stats + (size_t)rows * a.slices * 2);
  a.tokens_out = tokens_out; a.parents_out = parents_out; a.scores_out = scores_out;
  hipLaunchKernelGGL(beam_slice_kernel, dim3(a.slices, (unsigned)rows), dim3(kSliceThreads), 0, st, a);
  if ((long)beams * a.slices <= 256) hipLaunchKernelGGL(beam_pick_kernel<256>, dim3(groups), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(beam_pick_kernel<1024>, dim3(groups), dim3(1024), 0, st, a);
}

}  // namespace es
