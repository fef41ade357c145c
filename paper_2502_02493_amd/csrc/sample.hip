// Sampling under top-k, top-p and min-p from given random numbers (gfx950).
//
// Words stand in the order of their logits, the highest first, of equal ones the lowest token; each has the weight
// exp((x - max) / T).  What stays is a run from the front of that order (top-k, top-p and min-p each keep one, the shortest counts), and
// the token drawn is the first whose running weight passes u times that of the run.  So all of it comes down to one question, asked up to
// three times: which word of the order is the first to bring the running count or weight to a given number?
// Weights are whole multiples of 2^-s: sums of them are exact, so neither the order of atomic additions nor how a row is cut up
// shows in a result.
//
// Rows of more than 4096 words are not sorted.  A histogram of weights (and counts, for top_k) over y = (max - x) log2(e) / T tells
// for each question the bin that its word lies in, or, where it depends on the word that answers another one, a few of them.  The words
// of these bins, some hundred, are sorted and answer it exactly; of all others their bin says whether they stay.  Rows whose bins hold too many
// (thousands of nearly equal logits; or a top_k of thousands at a low temperature, whose word lies past y = 48, where four bins hold a doubling of y) go digit
// by digit through their words' place numbers instead: with top_k = 4000 of 152 064 normal logits at T = 0.05 a call of one row takes 80 .. 700 us, 22 at T >= 0.3.
// Three passes over a row, the last one writing: 96 rows of 152 064 words, whose kept logits are written, 71 us in a graph; 117 MB read and written
// once would be 23 at the rate of a copy, and the rows read twice more 17 at that of a kernel that only reads.
#include "launch_common.hpp"
#include "lane_ops.hpp"

#include <string.h>

namespace es {

typedef unsigned long long u64;
constexpr int kTokenBits = 20;
static_assert(kMaxSampleVocab == 1 << kTokenBits, "a place number holds a token");
// Bins: evenly over y up to 48, where weights end, or to the lowest logit's; then four to a doubling.  Every workgroup that lists words sums all of
// them up, so that twice as many cost more than their shorter lists save.
constexpr int kBins = 1024, kFineBins = 896;
constexpr int kNear = 4096;  // words that are sorted
constexpr int kDigitBins = 2048;
constexpr int kShortRow = 4096;   // words of a row that are sorted, all of them
constexpr int kRowWords = 8192;   // words of a row that stays with one workgroup
constexpr double kFar = 48.0;

// A word's place number: the higher, the earlier in the order; 0 is no word (minus infinity, NaN).
__device__ __forceinline__ u64 place_of(float x, int v) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(x + 0.f);  // the two zeros alike
  const uint32_t key = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
  return (u64)key << kTokenBits | (u64)(kMaxSampleVocab - 1 - v);
}
__device__ __forceinline__ int token_at(u64 place) { return kMaxSampleVocab - 1 - (int)(place & (kMaxSampleVocab - 1)); }
__device__ __forceinline__ float logit_at(u64 place) {
  const uint32_t key = (uint32_t)(place >> kTokenBits);
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

struct SampleArgs {
  const float* logits;
  const float* u;
  int V, top_k;           // top_k 0: all
  double log2e_T, top_p;  // log2(e) / T
  double min_z;           // T log(min_p), what a logit may lie below the highest; minus infinity: all
  double unit;            // 2^s
  int32_t* tokens;
  float* out;
  // a row's slices, and its cuts: more of them, where a workgroup has less to do
  int slices, per, cuts, per_cut;
  float2* slice_ends;  // [row][slices]  highest and lowest logit
  u64* weight;         // [row][kBins]
  uint32_t* count;     // [row][kBins + 1], the last one counting near words
  u64* near;           // [row][kNear]
  struct NearBins* bins;  // [row]
};

// What a word's logit says, given the row's highest and lowest.
struct Weigher {
  double top, log2e_T, unit, far, per_y;  // fine bins reach to y = far, per_y of them to 1
  __device__ __forceinline__ Weigher(const SampleArgs& a, float highest, float lowest)
      : top((double)highest), log2e_T(a.log2e_T), unit(a.unit) {
    far = fmin(kFar, fmax(below(lowest), 1e-6));
    per_y = (double)kFineBins / far;
  }
  __device__ __forceinline__ double below(float x) const { return (top - (double)x) * log2e_T; }
  __device__ __forceinline__ u64 weight(double y) const {
    const double w = exp2_below(-fmin(y, kFar)) * unit + 4503599627370496.0;  // 2^52: the sum's last bit is worth 1
    return y < kFar ? __builtin_bit_cast(u64, w) & 0xFFFFFFFFFFFFFull : 0;
  }
  __device__ __forceinline__ int bin(double y) const {  // never falls as y rises
    if (y < far) return min((int)(y * per_y), kFineBins - 1);
    const uint32_t b = __float_as_uint((float)(y * (1.0 / far)));
    return kFineBins + min(max((int)(b >> 21) - (127 << 2), 0), kBins - kFineBins - 1);
  }
  // A logit that all words of bin b are below (times < 1) or above (times > 1): y at the bin's start, rounded outwards.
  __device__ __forceinline__ float logit_at_bin(int b, double times) const {
    if (b >= kBins) return times > 1.0 ? -INFINITY : INFINITY;
    const double y = b <= kFineBins ? (double)b / per_y : far * (double)__uint_as_float((uint32_t)(b - kFineBins + (127 << 2)) << 21);
    const double x = top - y * times / log2e_T, room = 1e-6 * (fabs(top) + fabs(x)) + 1e-37;
    return (float)(times > 1.0 ? x - room : x + room);
  }
  __device__ __forceinline__ bool over(float x, double min_z) const { return (double)x - top >= min_z; }
};

// Words of row[v0, v1): body(x, v), eight loads of a thread under way.
template <int NT, class Body>
__device__ __forceinline__ void each_word(const float* row, int v0, int v1, const Body& body) {
  constexpr int N = 8;
  for (int base = v0; base < v1; base += N * NT) {
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int v = base + i * NT + (int)threadIdx.x;
      x[i] = v < v1 ? row[v] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (x[i] > -INFINITY) body(x[i], base + i * NT + (int)threadIdx.x);
  }
}

// Running sum over the wave's lanes, the own one included.
__device__ __forceinline__ u64 running_sum(u64 v) {
  const auto moved = [](u64 x, auto ctrl, auto rows) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
    return (u64)hi << 32 | lo;
  };
  typedef std::integral_constant<int, 0xF> All;
  v += moved(v, std::integral_constant<int, 0x111>{}, All{});  // row_shr by 1, 2, 4, 8: zeros come in
  v += moved(v, std::integral_constant<int, 0x112>{}, All{});
  v += moved(v, std::integral_constant<int, 0x114>{}, All{});
  v += moved(v, std::integral_constant<int, 0x118>{}, All{});
  v += moved(v, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});  // row_bcast15
  v += moved(v, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});  // row_bcast31
  return v;
}
// Running sums of two numbers over the threads of a workgroup, in front of the thread; all: the whole sums.  sh: NT / 64 pairs, which nobody
// reads any more.
struct Sums {
  u64 weight, count;
};
template <int NT>
__device__ __forceinline__ Sums sums_before(Sums v, Sums* sh, Sums& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Sums run = {running_sum(v.weight), running_sum(v.count)};
  if (lane == 63) sh[wave] = run;
  __syncthreads();
  Sums before = {run.weight - v.weight, run.count - v.count};
  all = Sums{0, 0};
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const Sums o = sh[w];
    before.weight += w < wave ? o.weight : 0;
    before.count += w < wave ? o.count : 0;
    all.weight += o.weight;
    all.count += o.count;
  }
  return before;
}
template <int NT>
__device__ __forceinline__ u64 sum_all(u64 v, Sums* sh) {
  Sums all;
  __syncthreads();
  sums_before<NT>(Sums{v, 0}, sh, all);
  return all.weight;
}

// A row's bins in LDS: first their counts and weights, then, at(b), those in front of each, a place left out after every 32, for steps
// of several bins.
template <int NT>
struct Bins {
  static constexpr int kPlaces = kBins + kBins / 32 + 1;
  u64 weight[kPlaces];
  uint32_t count[kPlaces];
  Sums scan[NT / 64];
  static __device__ __forceinline__ int at(int b) { return b + (b >> 5); }
  __device__ __forceinline__ u64 weight_before(int b) const { return weight[at(b)]; }
  __device__ __forceinline__ uint32_t count_before(int b) const { return count[at(b)]; }
};

// The bins that matter, as up to four runs in ascending order, apart from each other: what is in front of a word is what its list has in
// front of it and what lies between the runs.
struct NearBins {
  int lo[4], hi[4], k_on, p_on, m_on, k_bin, p_bin, m_bin, draw_bin;  // ..._bin: the first that may hold the answer
  int keep;                                                            // words of bins before it stay; of the others only such as are in the runs may
  u64 weight[4], count[4];  // not on the list, in front of the run
  u64 all, m_front;         // the row's weight; what is in front of the border's bin of min_p
  float x0, x1;             // logits outside are in none of the runs
  float stays;              // logits over it stay
  __device__ __forceinline__ bool has(int bin) const {
    bool in = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) in = in || (bin >= lo[i] && bin <= hi[i]);
    return in;
  }
  __device__ __forceinline__ bool lists(const Weigher& w, float x) const { return x >= x0 && x <= x1 && has(w.bin(w.below(x))); }
  // What is not on the list in front of a word of a listed bin.
  __device__ __forceinline__ u64 unlisted(const u64 (&of)[4], int bin) const {
    u64 n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += bin >= lo[i] && bin <= hi[i] ? of[i] : 0;
    return n;
  }
};
__device__ __forceinline__ u64 top_p_target(double top_p, u64 all) { return max((u64)1, min(all, (u64)ceil(top_p * (double)all))); }
__device__ __forceinline__ u64 draw_target(double u, u64 all) { return u < 1.0 ? max((u64)1, min(all, (u64)(fmax(u, 0.0) * (double)all) + 1)) : max((u64)1, all); }

// counts and weights of the thread's bins, from tid * kBins / NT on -> those in front of every bin
template <int NT>
__device__ __forceinline__ void scan_bins(Bins<NT>& b, u64 (&w)[kBins / NT], uint32_t (&c)[kBins / NT]) {
  constexpr int N = kBins / NT;
  const int tid = threadIdx.x;
  Sums own = {0, 0}, all;
#pragma unroll
  for (int i = 0; i < N; ++i) own.weight += w[i], own.count += c[i];
  Sums before = sums_before<NT>(own, b.scan, all);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    b.weight[b.at(tid * N + i)] = before.weight;
    b.count[b.at(tid * N + i)] = (uint32_t)before.count;
    before.weight += w[i];
    before.count += c[i];
  }
  if (tid == 0) b.weight[b.at(kBins)] = all.weight, b.count[b.at(kBins)] = (uint32_t)all.count;
  __syncthreads();
}

// The bin that holds the word at which the running weight (count) reaches a target, 1 or more and no more than there is: a wave's work, every
// sixteenth sum first, then the sixteen between.
template <int NT, class A>
__device__ __forceinline__ int bin_that_reaches(const Bins<NT>& b, const A* run, u64 target) {
  static_assert(kBins == 16 * 64, "sixteen bins to a lane");
  const int lane = threadIdx.x & 63;
  const int group = __popcll(__ballot(run[b.at(16 * lane + 16)] < target));
  return 16 * group + __popcll(__ballot(lane < 16 && run[b.at(16 * group + (lane & 15) + 1)] < target));
}

// Which bins matter.  b: sums in front of the bins.  The weight of the first top_k words, and of all that stay, is known here up to the
// words of one bin: whatever depends on it gets the bins between what either end asks for.  One wave's work, with few instructions: executed once,
// they take longer to arrive than to run (by all waves, with barriers at each search: 22.4 us a call for one row of 128 256, 32.7 for sixteen).
template <int NT>
__device__ __forceinline__ void near_bins(const SampleArgs& a, const Weigher& w, double u, Bins<NT>& b, NearBins& n) {
  if (threadIdx.x < 64) {
    int lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) lo[i] = kBins, hi[i] = -1;
    const u64 all = b.weight_before(kBins);
    u64 z0 = all, z1 = all;
    int cut0 = kBins, cut1 = kBins;
    const bool k_on = a.top_k > 0 && (uint32_t)a.top_k < b.count_before(kBins), p_on = a.top_p < 1.0, m_on = a.min_z > -INFINITY;
    if (k_on) {
      lo[0] = hi[0] = cut0 = cut1 = bin_that_reaches(b, b.count, (u64)a.top_k);
      z0 = b.weight_before(cut0);
      z1 = b.weight_before(cut0 + 1);
    }
    if (p_on) {
      lo[1] = bin_that_reaches(b, b.weight, top_p_target(a.top_p, z0));
      hi[1] = bin_that_reaches(b, b.weight, top_p_target(a.top_p, z1));
      cut0 = min(cut0, lo[1]);
      cut1 = min(cut1, hi[1]);
    }
    u64 m_front = 0;
    if (m_on) {
      lo[2] = hi[2] = w.bin(-a.min_z * w.log2e_T);
      cut0 = min(cut0, lo[2]);
      cut1 = min(cut1, hi[2]);
      m_front = b.weight_before(lo[2]);
    }
    if (a.tokens) {
      lo[3] = bin_that_reaches(b, b.weight, draw_target(u, cut0 < kBins ? b.weight_before(cut0) : all));
      hi[3] = bin_that_reaches(b, b.weight, draw_target(u, cut1 < kBins ? b.weight_before(cut1 + 1) : all));
    }
    if (threadIdx.x == 0) {
      n.k_on = k_on; n.p_on = p_on; n.m_on = m_on;
      n.k_bin = lo[0];
      n.p_bin = lo[1];
      n.m_bin = m_on ? lo[2] : -1;
      n.draw_bin = lo[3];
      n.keep = cut0;
      n.all = all;
      n.m_front = m_front;
    }
    // in ascending order, those that meet made one (the later of them empty)
    const auto order = [&](int i, int j) {
      const bool swap = lo[j] < lo[i];
      const int l = lo[i], h = hi[i];
      lo[i] = swap ? lo[j] : l;
      hi[i] = swap ? hi[j] : h;
      lo[j] = swap ? l : lo[j];
      hi[j] = swap ? h : hi[j];
    };
    order(0, 1); order(2, 3); order(0, 2); order(1, 3); order(1, 2);
    int end = -1, first = kBins;  // of the runs so far
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      hi[i] = lo[i] < kBins ? hi[i] : -1;
      lo[i] = max(lo[i], end + 1);
      const bool any = lo[i] <= hi[i];
      end = any ? hi[i] : end;
      first = any ? min(first, lo[i]) : first;
    }
    // a run to a lane: what lies in front of it, less what the runs before it list; then a border to a lane
    const int lane = threadIdx.x, at = lane & 3;
    const int my_lo = at == 0 ? lo[0] : at == 1 ? lo[1] : at == 2 ? lo[2] : lo[3], my_hi = at == 0 ? hi[0] : at == 1 ? hi[1] : at == 2 ? hi[2] : hi[3];
    const bool any = lane < 4 && my_lo <= my_hi;
    const u64 w0 = any ? b.weight_before(my_lo) : 0, w1 = any ? b.weight_before(my_hi + 1) - w0 : 0;
    const u64 c0 = any ? b.count_before(my_lo) : 0, c1 = any ? b.count_before(my_hi + 1) - c0 : 0;
    const u64 w_listed = running_sum(w1) - w1, c_listed = running_sum(c1) - c1;
    if (lane < 4) {
      n.lo[lane] = my_lo;
      n.hi[lane] = my_hi;
      n.weight[lane] = any ? w0 - w_listed : 0;
      n.count[lane] = any ? c0 - c_listed : 0;
    }
    const float x = w.logit_at_bin(lane == 0 ? end + 1 : lane == 1 ? first : cut0, lane == 0 ? 1.0 + 1e-5 : 1.0 - 1e-5);
    if (lane == 0) n.x0 = x;
    if (lane == 1) n.x1 = x;
    if (lane == 2) n.stays = cut0 < kBins ? x : -INFINITY;
  }
  __syncthreads();
}
// The words that stay: those up to a place, and over the highest logit plus min_z.
struct Cut {
  u64 from;
  int token;
};

// A workgroup's words in descending order, word E tid + e in the thread's e: by buckets that follow the order, or, where one of them
// would hold too many (equal logits, one far away from the others), by exchanges.
constexpr int kBuckets = 2048, kMaxBucket = 32;  // 512 equal words to a bucket, ranked among themselves, take longer than the exchanges
template <int NT>
struct SortSpace {
  uint32_t start[kBuckets + 1];
  uint32_t waves[NT / 64], too_many;
};

// Exchanges inside a thread, inside a wave, and between waves through LDS.
__device__ __forceinline__ u64 exchanged(u64 own, u64 other, bool larger) { return (own > other) == larger ? own : other; }
template <int NT, int E>
__device__ __forceinline__ void sort_by_exchanges(u64 (&x)[E], u64* lds) {
  const int tid = threadIdx.x;
#pragma unroll 1
  for (int k = 2; k <= NT * E; k *= 2) {
#pragma unroll 1
    for (int j = k / 2; j > 0; j /= 2) {
      const int m = j / E;
      const bool larger = ((tid & m) == 0) == (((tid * E) & k) == 0);  // from E on: what the thread keeps of its pairs
      if (j >= 64 * E) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) lds[e * NT + tid] = x[e];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = exchanged(x[e], lds[e * NT + (tid ^ m)], larger);
      } else if (j < E) {
#pragma unroll
        for (int step = 1; step < E; step *= 2) {
          if (step != j) continue;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            if (e & step) continue;
            const bool swap = (x[e] < x[e + step]) == (((tid * E + e) & k) == 0);
            const u64 a = x[e];
            x[e] = swap ? x[e + step] : a;
            x[e + step] = swap ? a : x[e + step];
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = exchanged(x[e], __shfl_xor(x[e], m), larger);
      }
    }
  }
}

// x: n words altogether (0: none), each in bucket[e] (-1: none), which do not fall along the order; lds: NT * E words, nobody reads or
// writes any.  One pass counts the buckets, their starts are summed up, the words go there, and each looks for its place among the few of its own.
template <int NT, int E>
__device__ __forceinline__ void sort_words(u64 (&x)[E], const int (&bucket)[E], int n, u64* lds, SortSpace<NT>& sp) {
  constexpr int N = kBuckets / NT;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) sp.start[i * NT + tid] = 0;
  if (tid == 0) sp.too_many = 0;
  __syncthreads();
  uint32_t at[E];
#pragma unroll
  for (int e = 0; e < E; ++e) at[e] = bucket[e] >= 0 ? atomicAdd(&sp.start[bucket[e]], 1u) : 0;
  __syncthreads();
  uint32_t own[N], sum = 0;
  bool many = false;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    own[i] = sp.start[tid * N + i];
    sum += own[i];
    many = many || own[i] > kMaxBucket;
  }
  const uint32_t run = (uint32_t)running_sum(sum);
  if (lane == 63) sp.waves[wave] = run;
  if (__ballot(many) && lane == 0) sp.too_many = 1;
  __syncthreads();
  if (sp.too_many) {
    sort_by_exchanges<NT, E>(x, lds);
    return;
  }
  uint32_t before = run - sum;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) before += w < wave ? sp.waves[w] : 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sp.start[tid * N + i] = before;
    before += own[i];
  }
  if (tid == NT - 1) sp.start[kBuckets] = before;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (bucket[e] >= 0) lds[sp.start[bucket[e]] + at[e]] = x[e];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (bucket[e] < 0) continue;
    const uint32_t first = sp.start[bucket[e]], end = sp.start[bucket[e] + 1];
    at[e] = first;
    for (uint32_t i = first; i < end; ++i) at[e] += lds[i] > x[e];
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (bucket[e] >= 0) lds[at[e]] = x[e];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = tid * E + e < n ? lds[tid * E + e] : 0;
}

struct Answer {
  u64 place, weight;
};
template <int NT>
struct ResolveSpace {
  Sums scan[NT / 64];
  Answer answer[3];
};

// Sorted words, E of them in a thread (0: none), answer all questions: those of the near bins, or (ALL) every one of a row.  Near words
// stand in out (if any) already: those that go are put out.
template <int NT, int E, bool ALL>
__device__ __forceinline__ Cut resolve(const SampleArgs& a, const Weigher& w, double u, const NearBins& near, const u64 (&x)[E], float* out, ResolveSpace<NT>& sp) {
  const int tid = threadIdx.x;
  // weights and counts up to and with every word
  u64 own[E], weight[E], count[E];
  Sums sum = {0, 0}, all;
  u64 in_bin = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float v = logit_at(x[e]);
    const double y = w.below(v);
    const bool word = x[e] != 0;
    own[e] = word ? w.weight(y) : 0;
    sum.weight += own[e];
    weight[e] = sum.weight;
    count[e] = tid * E + e + 1;
    bool in_m_bin = true;
    if constexpr (!ALL) {
      const int bin = w.bin(y);
      if (word) {
        weight[e] += near.unlisted(near.weight, bin);
        count[e] += near.unlisted(near.count, bin);
      }
      in_m_bin = bin == near.m_bin;
    }
    if (word && in_m_bin && w.over(v, a.min_z)) in_bin += own[e];
  }
  sum.count = in_bin;
  const Sums before = sums_before<NT>(sum, sp.scan, all);
  in_bin = all.count;
#pragma unroll
  for (int e = 0; e < E; ++e) weight[e] += before.weight;
  const auto find = [&](int question, bool by_count, u64 target) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const u64 now = by_count ? count[e] : weight[e], front = now - (by_count ? 1 : own[e]);
      if (x[e] && front < target && target <= now) sp.answer[question] = Answer{x[e], weight[e]};
    }
    __syncthreads();
    return sp.answer[question];
  };
  Cut cut = {1, -1};
  u64 stay = ALL ? all.weight : near.all;
  if (near.k_on) {
    const Answer k = find(0, true, (u64)a.top_k);
    cut.from = k.place;
    stay = k.weight;
  }
  if (near.p_on) {
    const Answer p = find(1, false, top_p_target(a.top_p, stay));
    cut.from = max(cut.from, p.place);
    stay = p.weight;
  }
  if (a.tokens) {
    // over the border of min_p: the bins in front of the border's, and its own words that are
    if (near.m_on) stay = min(stay, (ALL ? 0 : near.m_front) + in_bin);
    cut.token = token_at(find(2, false, draw_target(u, stay)).place);
  }
  if constexpr (!ALL)
    if (out)
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (x[e] && !(x[e] >= cut.from && w.over(logit_at(x[e]), a.min_z))) out[token_at(x[e])] = -INFINITY;
  return cut;
}
template <int NT, int E>
__device__ __forceinline__ Cut resolve_list(const SampleArgs& a, const Weigher& w, double u, const NearBins& near, const u64* words, int n, float* out, u64* lds,
                                            ResolveSpace<NT>& sp, SortSpace<NT>& sort) {
  u64 x[E];
  int bucket[E];
  int bins = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) bins += max(0, near.hi[i] - near.lo[i] + 1);
  const int parts = kBuckets / max(1, bins);  // buckets of a near bin
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = e * NT + threadIdx.x;
    x[e] = i < n ? words[i] : 0;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const double y = w.below(logit_at(x[e]));
    const int bin = w.bin(y);
    int index = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) index += min(bin, near.hi[i] + 1) > near.lo[i] ? min(bin, near.hi[i] + 1) - near.lo[i] : 0;
    const int part = bin < kFineBins ? min((int)((y * w.per_y - (double)bin) * (double)parts), parts - 1) : 0;
    bucket[e] = x[e] ? index * parts + part : -1;
  }
  __syncthreads();  // words may stand where they are sorted
  sort_words<NT, E>(x, bucket, n, lds, sort);
  return resolve<NT, E, false>(a, w, u, near, x, out, sp);
}
template <int NT>
__device__ __forceinline__ Cut resolve_any(const SampleArgs& a, const Weigher& w, double u, const NearBins& near, const u64* words, int n, float* out, u64* lds,
                                           ResolveSpace<NT>& sp, SortSpace<NT>& sort) {
  if (n <= 2 * NT) return resolve_list<NT, 2>(a, w, u, near, words, n, out, lds, sp, sort);
  return resolve_list<NT, kNear / NT>(a, w, u, near, words, n, out, lds, sp, sort);
}

// ------------------------------------------------------------------------------------------
// Digit by digit: for rows whose bins hold more words than are sorted: five passes over the row for an answer (152 064 equal logits 1.3 ms).
// ------------------------------------------------------------------------------------------
struct Digits {
  u64 weight[kDigitBins];
  uint32_t count[kDigitBins];
};

// The place of the first near word at which the count (or weight) of the near words so far reaches `target`, 1 or more and no more than all do.
template <int NT, bool BY_WEIGHT>
__device__ __forceinline__ u64 first_to_reach(const float* row, int V, const Weigher& w, const NearBins& near, u64 target, Digits& d, Sums* scan, u64& s_bin) {
  const int tid = threadIdx.x;
  constexpr int N = kDigitBins / NT;
  u64 prefix = 0;
  int shift = 32 + kTokenBits;
  for (int digit = 0; digit < 5; ++digit) {
    const int bits = digit < 2 ? 11 : 10, above = shift;
    shift -= bits;
    for (int i = tid; i < kDigitBins; i += NT) d.weight[i] = 0, d.count[i] = 0;
    __syncthreads();
    each_word<NT>(row, 0, V, [&](float x, int v) {
      const u64 p = place_of(x, v);
      if (p >> above != prefix || !near.lists(w, x)) return;
      const int bin = kDigitBins - 1 - ((int)(p >> shift) & ((1 << bits) - 1));  // the highest first
      if (BY_WEIGHT) atomicAdd(&d.weight[bin], w.weight(w.below(x)));
      else atomicAdd(&d.count[bin], 1u);
    });
    __syncthreads();
    u64 n[N], sum = 0;
    Sums all;
#pragma unroll
    for (int i = 0; i < N; ++i) sum += n[i] = BY_WEIGHT ? d.weight[tid * N + i] : d.count[tid * N + i];
    u64 before = sums_before<NT>(Sums{sum, 0}, scan, all).weight;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (before < target && target <= before + n[i]) {
        s_bin = kDigitBins - 1 - (tid * N + i);
        d.weight[0] = before;  // read as a bin already
      }
      before += n[i];
    }
    __syncthreads();
    prefix = prefix << bits | s_bin;
    target -= d.weight[0];
    __syncthreads();
  }
  return prefix;
}

// row: where the near words stand, which is out if there is one (what is neither near nor stays is gone from it).
template <int NT>
__device__ __forceinline__ Cut resolve_by_digits(const SampleArgs& a, const Weigher& w, double u, const NearBins& near, const float* row, float* out, Digits& d, Sums* scan) {
  __shared__ u64 s_bin;
  const auto weight_from = [&](u64 place, auto which) {
    u64 s = 0;
    each_word<NT>(row, 0, a.V, [&](float x, int v) {
      if (place_of(x, v) >= place && near.lists(w, x) && which(x)) s += w.weight(w.below(x));
    });
    return sum_all<NT>(s, scan);
  };
  const auto any = [](float) { return true; };
  Cut cut = {1, -1};
  u64 stay = near.all;
  if (near.k_on) {
    cut.from = first_to_reach<NT, false>(row, a.V, w, near, (u64)a.top_k - near.unlisted(near.count, near.k_bin), d, scan, s_bin);
    stay = near.unlisted(near.weight, near.k_bin) + weight_from(cut.from, any);
  }
  if (near.p_on) {
    const u64 p = first_to_reach<NT, true>(row, a.V, w, near, top_p_target(a.top_p, stay) - near.unlisted(near.weight, near.p_bin), d, scan, s_bin);
    cut.from = max(cut.from, p);
    stay = near.unlisted(near.weight, near.p_bin) + weight_from(p, any);
  }
  if (a.tokens) {
    if (near.m_on) stay = min(stay, near.m_front + weight_from(1, [&](float x) { return w.bin(w.below(x)) == near.m_bin && w.over(x, a.min_z); }));
    cut.token = token_at(first_to_reach<NT, true>(row, a.V, w, near, draw_target(u, stay) - near.unlisted(near.weight, near.draw_bin), d, scan, s_bin));
  }
  if (out)
    each_word<NT>(row, 0, a.V, [&](float x, int v) {
      if (near.lists(w, x) && !(place_of(x, v) >= cut.from && w.over(x, a.min_z))) out[v] = -INFINITY;
    });
  return cut;
}

// ------------------------------------------------------------------------------------------
// A row to a workgroup.
// ------------------------------------------------------------------------------------------
template <int NT>
union SampleSpace {
  struct {
    Bins<NT> bins;
    u64 words[kNear];
  };
  Digits digits;
};
__device__ __forceinline__ bool no_word(float top) { return !(top > -INFINITY && top < INFINITY); }

// Highest and lowest logit of the words of a workgroup's part of a row.
template <int NT>
__device__ __forceinline__ float2 ends_of(const float* row, int v0, int v1, float* sh) {
  float hi = -INFINITY, lo = INFINITY;
  each_word<NT>(row, v0, v1, [&](float x, int) {
    hi = fmaxf(hi, x);
    lo = fminf(lo, x);
  });
  hi = block_max<NT / 64>(hi, sh);
  lo = -block_max<NT / 64>(-lo, sh + NT / 64);
  return make_float2(hi, lo);
}
// counts: only top_k asks for them.
template <int NT>
__device__ __forceinline__ void add_to_bins(const Weigher& w, const float* row, int v0, int v1, u64* weight, uint32_t* count, bool counts) {
  const auto all = [&](auto with_counts) {
    each_word<NT>(row, v0, v1, [&](float x, int) {
      const double y = w.below(x);
      const int b = w.bin(y);
      if (decltype(with_counts)::value) atomicAdd(&count[b], 1u);
      if (y < kFar) atomicAdd(&weight[b], w.weight(y));
    });
  };
  if (counts) all(std::true_type{});
  else all(std::false_type{});
}
// The near words of a part of a row, listed in any order: a wave asks for places once for every eight words of its lanes.  *n counts
// them all, those past kNear, which are not listed, too.  out (if any): the words that stay, and near ones.
template <int NT>
__device__ __forceinline__ void list_near(const Weigher& w, const NearBins& near, const float* row, float* out, int v0, int v1, u64* words, uint32_t* n) {
  constexpr int kAhead = 8;
  const float x0 = near.x0, x1 = near.x1, stays = near.stays;
  const int lane = threadIdx.x & 63;
  for (int base = v0; base < v1; base += kAhead * NT) {
    float x[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int v = base + i * NT + (int)threadIdx.x;
      x[i] = v < v1 ? row[v] : -INFINITY;
    }
    unsigned long long in[kAhead];
    int found = 0;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      bool is = x[i] > -INFINITY && x[i] >= x0 && x[i] <= x1, keep = x[i] > stays;
      if (is) {
        const int bin = w.bin(w.below(x[i]));
        is = near.has(bin);
        keep = keep || is || bin < near.keep;
      }
      const int v = base + i * NT + (int)threadIdx.x;
      if (out && v < v1) out[v] = keep ? x[i] : -INFINITY;
      in[i] = __ballot(is);
      found += __popcll(in[i]);
    }
    if (found == 0) continue;
    uint32_t at = 0;
    if (lane == 0) at = atomicAdd(n, (uint32_t)found);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint32_t mine = at + __popcll(in[i] & ((1ull << lane) - 1));
      if ((in[i] >> lane & 1) && mine < kNear) words[mine] = place_of(x[i], base + i * NT + (int)threadIdx.x);
      at += __popcll(in[i]);
    }
  }
}

template <int NT>
__global__ __launch_bounds__(NT) void sample_row_kernel(SampleArgs a) {
  __shared__ SampleSpace<NT> sp;
  __shared__ ResolveSpace<NT> rs;
  __shared__ SortSpace<NT> sort;
  __shared__ float s_ends[2 * NT / 64];
  __shared__ NearBins near;
  __shared__ uint32_t s_near;
  const int tid = threadIdx.x;
  const size_t r = blockIdx.x;
  const float* row = a.logits + r * a.V;
  float* out = a.out ? a.out + r * a.V : nullptr;
  for (int i = tid; i < kBins; i += NT) sp.bins.weight[i] = 0, sp.bins.count[i] = 0;
  if (tid == 0) s_near = 0;
  const float2 ends = ends_of<NT>(row, 0, a.V, s_ends);
  if (no_word(ends.x)) {
    if (a.tokens && tid == 0) a.tokens[r] = -1;
    if (out)
      for (int v = tid; v < a.V; v += NT) out[v] = -INFINITY;
    return;
  }
  const Weigher w(a, ends.x, ends.y);
  const double u = a.tokens ? (double)a.u[r] : 0.0;
  add_to_bins<NT>(w, row, 0, a.V, sp.bins.weight, sp.bins.count, a.top_k > 0);
  __syncthreads();
  constexpr int N = kBins / NT;
  u64 bw[N];
  uint32_t bc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) bw[i] = sp.bins.weight[tid * N + i], bc[i] = sp.bins.count[tid * N + i];
  scan_bins(sp.bins, bw, bc);
  near_bins(a, w, u, sp.bins, near);
  Cut cut;
  list_near<NT>(w, near, row, out, 0, a.V, sp.words, &s_near);
  __syncthreads();
  const int n = (int)s_near;
  if (n <= kNear) cut = resolve_any<NT>(a, w, u, near, sp.words, n, out, sp.words, rs, sort);
  else cut = resolve_by_digits<NT>(a, w, u, near, out ? out : row, out, sp.digits, rs.scan);
  if (a.tokens && tid == 0) a.tokens[r] = cut.token;
}

// A short row: all of its words are sorted.  As wide as pays (us in a graph, 1 row : 600 rows, threads x words): 250 words 256 x 1
// 4.6 : 6.6, 256 x 2 5.0 : 7.1; 500 words 256 x 2 5.5 : 7.8, 512 x 1 5.4 : 8.9; 1000 words 512 x 2 6.5 : 10.8, 256 x 4 7.2 : 10.4,
// 1024 x 1 7.8 : 21.3; 2000 words 512 x 4 8.9 : 18.6, 256 x 8 11.5 : 16.5, 1024 x 2 9.2 : 25.8; 4000 words 1024 x 4 12.8 : 39.0,
// 512 x 8 14.9 : 33.5, the way of longer rows 16.5 : 48.9; 8000 words 1024 x 8 27.8 : 88.8, the way of longer rows 18.7 : 57.3.
template <int NT, int E>
__global__ __launch_bounds__(NT) void sample_short_kernel(SampleArgs a) {
  __shared__ u64 s_words[NT * E];
  __shared__ ResolveSpace<NT> rs;
  __shared__ SortSpace<NT> sort;
  __shared__ float s_ends[2 * NT / 64];
  const int tid = threadIdx.x;
  const size_t r = blockIdx.x;
  const float* row = a.logits + r * a.V;
  float* out = a.out ? a.out + r * a.V : nullptr;
  const double u = a.tokens ? (double)a.u[r] : 0.0;
  float v[E];  // which words a thread brings is all the same to the sort: those that lie side by side in memory
  u64 x[E];
  float hi = -INFINITY, lo = INFINITY;
  int words = 0;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = e * NT + tid;
    v[e] = i < a.V ? row[i] : -INFINITY;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    x[e] = place_of(v[e], e * NT + tid);
    words += x[e] != 0;
    hi = fmaxf(hi, v[e]);
    if (x[e]) lo = fminf(lo, v[e]);
  }
  const float top = block_max<NT / 64>(hi, s_ends), low = -block_max<NT / 64>(-lo, s_ends + NT / 64);
  if (no_word(top)) {
    if (a.tokens && tid == 0) a.tokens[r] = -1;
    if (out)
      for (int i = tid; i < a.V; i += NT) out[i] = -INFINITY;
    return;
  }
  const Weigher w(a, top, low);
  const int n = (int)sum_all<NT>((u64)words, rs.scan);
  NearBins near;
  near.k_on = a.top_k > 0 && a.top_k < n;
  near.p_on = a.top_p < 1.0;
  near.m_on = a.min_z > -INFINITY;
  const double per_y = (double)(kBuckets - 1) / fmax(w.below(low), 1e-6);
  int bucket[E];
#pragma unroll
  for (int e = 0; e < E; ++e) bucket[e] = x[e] ? min((int)(w.below(v[e]) * per_y), kBuckets - 1) : -1;
  sort_words<NT, E>(x, bucket, n, s_words, sort);
  __syncthreads();
  const Cut cut = resolve<NT, E, true>(a, w, u, near, x, nullptr, rs);
  if (a.tokens && tid == 0) a.tokens[r] = cut.token;
  if (out)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = e * NT + tid;
      if (i < a.V) out[i] = place_of(v[e], i) >= cut.from && w.over(v[e], a.min_z) ? v[e] : -INFINITY;
    }
}

// ------------------------------------------------------------------------------------------
// A row to several workgroups, in four launches: (1) the slices' highest and lowest logits; (2) their bins, added up; (3) the words of the
// near bins, in one list, and what stays without them; (4) one workgroup sorts the list, draws, and puts out the near words that go.
// ------------------------------------------------------------------------------------------
constexpr int kSliceNT = 1024, kMaxSlices = 64, kSliceWgs = 512, kMaxSlicedRows = 1024;
constexpr int kCutNT = 256, kMaxCuts = 64, kCutWgs = 2048;
constexpr int kFinishNT = 512;

__device__ __forceinline__ float2 row_ends(const SampleArgs& a, float2* s_ends) {
  if (threadIdx.x < 64) {
    const float2 e = (int)threadIdx.x < a.slices ? a.slice_ends[(size_t)blockIdx.y * kMaxSlices + threadIdx.x] : make_float2(-INFINITY, INFINITY);
    const float hi = lanes_max(e.x, 64), lo = -lanes_max(-e.y, 64);
    if (threadIdx.x == 0) *s_ends = make_float2(hi, lo);
  }
  __syncthreads();
  return *s_ends;
}

// grid (slices, rows).  A pass of reading: 96 rows of 152 064 11.3 us (5.2 TB/s).
__global__ __launch_bounds__(kSliceNT) void sample_ends_kernel(SampleArgs a) {
  __shared__ float s_ends[2 * kSliceNT / 64];
  const size_t r = blockIdx.y;
  const int v0 = min(a.V, (int)blockIdx.x * a.per), v1 = min(a.V, v0 + a.per);
  for (int i = blockIdx.x * kSliceNT + threadIdx.x; i <= kBins; i += a.slices * kSliceNT) {
    if (i < kBins) a.weight[r * kBins + i] = 0;
    a.count[r * (kBins + 1) + i] = 0;
  }
  const float2 ends = ends_of<kSliceNT>(a.logits + r * a.V, v0, v1, s_ends);
  if (threadIdx.x == 0) a.slice_ends[r * kMaxSlices + blockIdx.x] = ends;
}

// The same pass, and an exponential in double precision and an atomic addition in LDS for every word: 22.5 us.  Of a CU's 43 000 busy cycles the vector units
// work for 32 000 (36 instructions a word), LDS for 11 400, 7 400 of them bank conflicts: arithmetic before atomics.  (With counts of all bins, which only
// top_k asks for, 25.  The bins that matter worked out here, by the last of a row's workgroups, instead of by all of the next launch: 34.6, and 24.3
// there instead of 27.9: the wait for the atomic additions.)
__global__ __launch_bounds__(kSliceNT) void sample_bins_kernel(SampleArgs a) {
  __shared__ u64 s_weight[kBins];
  __shared__ uint32_t s_count[kBins];
  __shared__ float2 s_ends;
  const int tid = threadIdx.x;
  const size_t r = blockIdx.y;
  const int v0 = min(a.V, (int)blockIdx.x * a.per), v1 = min(a.V, v0 + a.per);
  for (int i = tid; i < kBins; i += kSliceNT) s_weight[i] = 0, s_count[i] = 0;
  const float2 ends = row_ends(a, &s_ends);
  if (no_word(ends.x)) return;
  const Weigher w(a, ends.x, ends.y);
  add_to_bins<kSliceNT>(w, a.logits + r * a.V, v0, v1, s_weight, s_count, a.top_k > 0);
  __syncthreads();
  for (int i = tid; i < kBins; i += kSliceNT) {
    if (s_count[i]) atomicAdd(&a.count[r * (kBins + 1) + i], s_count[i]);
    if (s_weight[i]) atomicAdd(&a.weight[r * kBins + i], s_weight[i]);
  }
}

// grid (cuts, rows).  Reads and writes the row: 27.2 us (4.3 TB/s); of a single row of 128 256 9.1, of which 2 to 3 are the bins, which every
// workgroup sums up for itself.  Workgroups of 256 threads, 2048 of them at most: 1024 threads make the 71 us of all four launches 81, 1024
// workgroups of 512 threads change nothing.
__global__ __launch_bounds__(kCutNT) void sample_near_kernel(SampleArgs a) {
  __shared__ Bins<kCutNT> bins;
  __shared__ NearBins near;
  __shared__ float2 s_ends;
  constexpr int N = kBins / kCutNT;
  const int tid = threadIdx.x;
  const size_t r = blockIdx.y;
  const int v0 = min(a.V, (int)blockIdx.x * a.per_cut), v1 = min(a.V, v0 + a.per_cut);
  u64 bw[N];
  uint32_t bc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) bw[i] = a.weight[r * kBins + tid * N + i], bc[i] = a.count[r * (kBins + 1) + tid * N + i];
  const double u = a.tokens ? (double)a.u[r] : 0.0;
  float* out = a.out ? a.out + r * a.V : nullptr;
  const float2 ends = row_ends(a, &s_ends);
  if (no_word(ends.x)) {
    if (out)
      for (int v = v0 + tid; v < v1; v += kCutNT) out[v] = -INFINITY;
    return;
  }
  const Weigher w(a, ends.x, ends.y);
  scan_bins(bins, bw, bc);
  near_bins(a, w, u, bins, near);
  if (blockIdx.x == 0 && tid == 0) a.bins[r] = near;
  list_near<kCutNT>(w, near, a.logits + r * a.V, out, v0, v1, a.near + r * kNear, &a.count[r * (kBins + 1) + kBins]);
}

// grid (1, rows).  A chain of some ten barriers: 5.8 .. 6.9 us.
__global__ __launch_bounds__(kFinishNT) void sample_finish_kernel(SampleArgs a) {
  __shared__ union {
    u64 words[kNear];
    Digits digits;
  } sp;
  __shared__ ResolveSpace<kFinishNT> rs;
  __shared__ SortSpace<kFinishNT> sort;
  __shared__ float2 s_ends;
  const size_t r = blockIdx.y;
  const float* row = a.logits + r * a.V;
  float* out = a.out ? a.out + r * a.V : nullptr;
  const float2 ends = row_ends(a, &s_ends);
  if (no_word(ends.x)) {
    if (a.tokens && threadIdx.x == 0) a.tokens[r] = -1;
    return;
  }
  const Weigher w(a, ends.x, ends.y);
  const double u = a.tokens ? (double)a.u[r] : 0.0;
  const NearBins near = a.bins[r];
  const uint32_t n = a.count[r * (kBins + 1) + kBins];
  Cut cut;
  if (n <= kNear) cut = resolve_any<kFinishNT>(a, w, u, near, a.near + r * kNear, (int)n, out, sp.words, rs, sort);
  else cut = resolve_by_digits<kFinishNT>(a, w, u, near, out ? out : row, out, sp.digits, rs.scan);
  if (a.tokens && threadIdx.x == 0) a.tokens[r] = cut.token;
}

// One launch or four.  A row kept to one workgroup costs one launch, and a time that grows with the row; cut up it pays from some
// 8 thousand words on (us in a graph, one launch : four): 1 row of 6000 17.7 : 19.6, of 12 000 23.5 : 20.1 and of 152 064 142 : 24;
// 96 rows of 6000 18.5 : 23.7, of 12 000 24.7 : 28.4, of 24 000 34.7 : 32.0, of 152 064 156 : 77; 600 rows of 12 000 71 : 60, of
// 152 064 502 : 403.  Rows that fill the chip by themselves gain little: 1200 of 152 064 849 : 792, with top_k 676 : 715.
static bool whole_rows(int rows, int V) { return V <= kRowWords || rows > kMaxSlicedRows; }
static size_t sample_row_bytes() { return kMaxSlices * sizeof(float2) + kBins * sizeof(u64) + (kBins + 1) * sizeof(uint32_t) + kNear * sizeof(u64) + sizeof(NearBins); }
size_t sample_bytes_used(int rows, int V) { return whole_rows(rows, V) ? 16 : rows * sample_row_bytes(); }
// ... and by any call of fewer rows or words: more than kMaxSlicedRows rows need none, but a call of some of them may follow.
size_t sample_workspace_bytes(int rows, int V) { return sample_bytes_used(std::min(rows, kMaxSlicedRows), V); }

void launch_sample(const float* logits, const float* u, int rows, int V, double T, int top_k, double top_p, double min_p, int32_t* tokens_out,
                   float* logits_out, void* ws, hipStream_t st) {
  SampleArgs a;
  memset(&a, 0, sizeof a);
  a.logits = logits; a.u = u; a.V = V; a.top_k = top_k; a.top_p = top_p;
  a.log2e_T = 1.4426950408889634 / T;
  a.min_z = min_p > 0.0 ? T * log(min_p) : -INFINITY;
  int bits = 0;
  while ((1 << bits) < V) ++bits;
  a.unit = ldexp(1.0, std::min(51, 62 - bits));
  a.tokens = tokens_out; a.out = logits_out;
  if (whole_rows(rows, V)) {
    const auto short_row = [&](auto nt, auto e) {
      constexpr int NT = decltype(nt)::value, E = decltype(e)::value;
      hipLaunchKernelGGL((sample_short_kernel<NT, E>), dim3(rows), dim3(NT), 0, st, a);
    };
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, 2> Two;
    typedef std::integral_constant<int, 4> Four;
    if (V <= 256) short_row(std::integral_constant<int, 256>{}, One{});
    else if (V <= 512) short_row(std::integral_constant<int, 256>{}, Two{});
    else if (V <= 1024) short_row(std::integral_constant<int, 512>{}, Two{});
    else if (V <= 2048) short_row(std::integral_constant<int, 512>{}, Four{});
    else if (V <= kShortRow) short_row(std::integral_constant<int, 1024>{}, Four{});
    else hipLaunchKernelGGL(sample_row_kernel<1024>, dim3(rows), dim3(1024), 0, st, a);
    return;
  }
  a.slices = std::max(1, std::min({kMaxSlices, (V + 4095) / 4096, kSliceWgs / rows}));
  a.per = (V + a.slices - 1) / a.slices;
  a.cuts = std::max(1, std::min({kMaxCuts, (V + 2047) / 2048, kCutWgs / rows}));
  a.per_cut = (V + a.cuts - 1) / a.cuts;
  a.weight = (u64*)ws;
  a.near = a.weight + (size_t)rows * kBins;
  a.bins = (NearBins*)(a.near + (size_t)rows * kNear);
  a.slice_ends = (float2*)(a.bins + rows);
  a.count = (uint32_t*)(a.slice_ends + (size_t)rows * kMaxSlices);
  const dim3 grid(a.slices, rows), block(kSliceNT);
  hipLaunchKernelGGL(sample_ends_kernel, grid, block, 0, st, a);
  hipLaunchKernelGGL(sample_bins_kernel, grid, block, 0, st, a);
  hipLaunchKernelGGL(sample_near_kernel, dim3(a.cuts, rows), dim3(kCutNT), 0, st, a);
  hipLaunchKernelGGL(sample_finish_kernel, dim3(1, rows), dim3(kFinishNT), 0, st, a);
}

}  // namespace es
