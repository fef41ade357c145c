// Sampling under top-k, top-p and min-p from given random numbers (gfx950).
//
// Words stand in the order of their logits, the highest first, of equal ones the lowest token; each has the weight
// exp((x - max) / T).  What stays is a run from the front of that order (top-k, top-p and min-p each keep one, the shortest counts), and
// the token drawn is the first whose running weight passes u times that of the run.  So all of it comes down to one question, asked up to
// three times: which word of the order is the first to bring the running count or weight to a given number?
// Weights are whole multiples of 2^-s: sums of them are exact, so neither the order of atomic additions nor how a row is cut up
// shows in a result.
//
// No row is sorted.  A histogram of counts and weights over y = (max - x) log2(e) / T, sixteen bins to a factor of two in weight, tells
// for each question the bin that its word lies in, or, where it depends on the word that answers another one, a few of them.  The words
// of these bins, some hundred, are sorted and answer it exactly.  Rows whose bins hold too many (thousands of nearly equal
// logits) go digit by digit through their words' place numbers instead.
#include "launch_common.hpp"
#include "lane_ops.hpp"

#include <string.h>

namespace es {

typedef unsigned long long u64;
constexpr int kTokenBits = 20;
static_assert(kMaxSampleVocab == 1 << kTokenBits, "a place number holds a token");
constexpr int kBins = 1024, kFineBins = 768;  // kFineBins up to y = 48, where weights end; then eight to a doubling of y
constexpr int kNear = 4096;                   // words that are sorted
constexpr int kDigitBins = 2048;
constexpr int kShortRow = 2048;  // words of a row that one small workgroup takes

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
  // rows cut into slices
  int slices, per;
  float* slice_max;  // [row][slices]
  u64* weight;       // [row][kBins]
  uint32_t* count;   // [row][kBins + 1], the last one counting near words
  u64* near;         // [row][kNear]
};

// What a word's logit says, given the row's highest.
struct Weigher {
  double top, log2e_T, unit;
  __device__ __forceinline__ double below(float x) const { return (top - (double)x) * log2e_T; }
  __device__ __forceinline__ u64 weight(double y) const {  // exact below 2^52: the sum's last bit is worth 1
    const double w = exp2_below(fmax(-y, -1000.0)) * unit + 4503599627370496.0;
    return __builtin_bit_cast(u64, w) & 0xFFFFFFFFFFFFFull;
  }
  __device__ __forceinline__ int bin(double y) const {  // never falls as y rises
    if (y < 48.0) return (int)(y * 16.0);
    const uint32_t b = __float_as_uint((float)(y * (1.0 / 48.0)));
    return kFineBins + min((int)(b >> 20) - (127 << 3), kBins - kFineBins - 1);
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

// Running sums over the threads of a workgroup, in front of the thread; all: the whole.  sh: NT / 64 numbers, which nobody reads any more.
template <int NT>
__device__ __forceinline__ u64 sum_before(u64 v, u64* sh, u64& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 run = v;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const u64 o = __shfl_up(run, off, 64);
    if (lane >= off) run += o;
  }
  if (lane == 63) sh[wave] = run;
  __syncthreads();
  u64 before = run - v;
  all = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const u64 o = sh[w];
    before += w < wave ? o : 0;
    all += o;
  }
  return before;
}
template <int NT>
__device__ __forceinline__ u64 sum_all(u64 v, u64* sh) {
  u64 all;
  __syncthreads();
  sum_before<NT>(v, sh, all);
  return all;
}

// A row's bins in LDS: counts and weights in front of each.
template <int NT>
struct Bins {
  u64 weight[kBins + 1], near_weight[kBins];  // in front of the bin; of those words that are near
  uint32_t count[kBins + 1], near_count[kBins];
  u64 scan[4][NT / 64];
  int found[2];
};
struct Near {  // bins whose words are sorted: four ranges, and where the cutoff is sought
  int lo[4], hi[4];
  bool k_on, p_on, m_on;
  __device__ __forceinline__ bool has(int bin) const {
    bool in = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) in = in || (bin >= lo[i] && bin <= hi[i]);
    return in;
  }
};
__device__ __forceinline__ u64 top_p_target(double top_p, u64 all) { return max((u64)1, min(all, (u64)ceil(top_p * (double)all))); }
__device__ __forceinline__ u64 draw_target(double u, u64 all) { return u < 1.0 ? max((u64)1, min(all, (u64)(fmax(u, 0.0) * (double)all) + 1)) : max((u64)1, all); }

// counts and weights of the bins -> those in front of each (in place)
template <int NT>
__device__ __forceinline__ void scan_bins(Bins<NT>& b) {
  constexpr int N = kBins / NT;
  const int tid = threadIdx.x;
  u64 w[N], sw = 0;
  uint32_t c[N];
  u64 sc = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sw += w[i] = b.weight[tid * N + i];
    sc += c[i] = b.count[tid * N + i];
  }
  u64 all_w, all_c;
  u64 before_w = sum_before<NT>(sw, b.scan[0], all_w), before_c = sum_before<NT>(sc, b.scan[1], all_c);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    b.weight[tid * N + i] = before_w;
    b.count[tid * N + i] = (uint32_t)before_c;
    before_w += w[i];
    before_c += c[i];
  }
  if (tid == 0) b.weight[kBins] = all_w, b.count[kBins] = (uint32_t)all_c;
  __syncthreads();
}

// The bins that hold the words at which the running weight (count) reaches two targets, 1 or more and no more than there is.
template <int NT, class A>
__device__ __forceinline__ void bins_that_reach(Bins<NT>& b, const A* run, u64 t0, u64 t1, int& b0, int& b1) {
  for (int i = threadIdx.x; i < kBins; i += NT) {
    const u64 before = run[i], after = run[i + 1];
    if (before < t0 && t0 <= after) b.found[0] = i;
    if (before < t1 && t1 <= after) b.found[1] = i;
  }
  __syncthreads();
  b0 = b.found[0];
  b1 = b.found[1];
  __syncthreads();
}

// Which bins matter.  b: sums in front of the bins.  The weight of the first top_k words, and of all that stay, is known here up to the
// words of one bin: whatever depends on it gets the bins between what either end asks for.
template <int NT>
__device__ __forceinline__ Near near_bins(const SampleArgs& a, const Weigher& w, double u, Bins<NT>& b) {
  Near n;
#pragma unroll
  for (int i = 0; i < 4; ++i) n.lo[i] = 1, n.hi[i] = 0;
  const u64 all = b.weight[kBins];
  u64 z0 = all, z1 = all;
  int cut0 = kBins, cut1 = kBins;
  n.k_on = a.top_k > 0 && (uint32_t)a.top_k < b.count[kBins];
  n.p_on = a.top_p < 1.0;
  n.m_on = a.min_z > -INFINITY;
  if (n.k_on) {
    bins_that_reach(b, b.count, (u64)a.top_k, (u64)a.top_k, cut0, cut1);
    n.lo[0] = n.hi[0] = cut0;
    z0 = b.weight[cut0];
    z1 = b.weight[cut0 + 1];
  }
  if (n.p_on) {
    bins_that_reach(b, b.weight, top_p_target(a.top_p, z0), top_p_target(a.top_p, z1), n.lo[1], n.hi[1]);
    cut0 = min(cut0, n.lo[1]);
    cut1 = min(cut1, n.hi[1]);
  }
  if (n.m_on) {
    n.lo[2] = n.hi[2] = w.bin(-a.min_z * w.log2e_T);
    cut0 = min(cut0, n.lo[2]);
    cut1 = min(cut1, n.hi[2]);
  }
  if (a.tokens) {
    const u64 t0 = cut0 < kBins ? b.weight[cut0] : all, t1 = cut1 < kBins ? b.weight[cut1 + 1] : all;
    bins_that_reach(b, b.weight, draw_target(u, t0), draw_target(u, t1), n.lo[3], n.hi[3]);
  }
  return n;
}

// The words that stay: those up to a place, and over the highest logit plus min_z.
struct Cut {
  u64 from;
  int token;
};

// n words of the near bins, sorted here, answer all questions.  b: sums in front of the bins.
template <int NT>
__device__ __forceinline__ Cut resolve(const SampleArgs& a, const Weigher& w, double u, Bins<NT>& b, const Near& near, u64* words, int n) {
  const int tid = threadIdx.x;
  int size = 2;
  while (size < n) size *= 2;
  for (int i = n + tid; i < size; i += NT) words[i] = 0;
  {  // what of the sums in front of a bin is of near words
    constexpr int N = kBins / NT;
    u64 sw = 0, sc = 0, nw[N], nc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = tid * N + i;
      const bool in = near.has(at);
      sw += nw[i] = in ? b.weight[at + 1] - b.weight[at] : 0;
      sc += nc[i] = in ? b.count[at + 1] - b.count[at] : 0;
    }
    u64 all;
    u64 before_w = sum_before<NT>(sw, b.scan[2], all), before_c = sum_before<NT>(sc, b.scan[3], all);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      b.near_weight[tid * N + i] = before_w;
      b.near_count[tid * N + i] = (uint32_t)before_c;
      before_w += nw[i];
      before_c += nc[i];
    }
  }
  __syncthreads();
  for (int k = 2; k <= size; k *= 2)
    for (int j = k / 2; j > 0; j /= 2) {
      for (int i = tid; i < size / 2; i += NT) {
        const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
        const u64 x = words[lo], y = words[hi];
        if ((x < y) == ((lo & k) == 0)) words[lo] = y, words[hi] = x;
      }
      __syncthreads();
    }
  // running weights, a thread's words side by side
  const int per = (size + NT - 1) / NT, i0 = min(n, tid * per), i1 = min(n, i0 + per);
  u64 own = 0, all;
  for (int i = i0; i < i1; ++i) own += w.weight(w.below(logit_at(words[i])));
  const u64 before = sum_before<NT>(own, b.scan[0], all);
  const auto first_of_mine = [&](auto reaches) {  // reaches(count, weight, place) with the words up to this one
    u64 run = before;
    for (int i = i0; i < i1; ++i) {
      const double y = w.below(logit_at(words[i]));
      const int bin = w.bin(y);
      run += w.weight(y);
      if (reaches((u64)(i + 1) + b.count[bin] - b.near_count[bin], run + b.weight[bin] - b.near_weight[bin], words[i])) return;
    }
  };
  __shared__ u64 s_place, s_weight;
  // where the running count (weight) first reaches a number, inside a thread's words: the word in front of it has not
  const auto find = [&](bool by_count, u64 target, u64& place, u64& weight) {
    __syncthreads();
    first_of_mine([&](u64 c, u64 wt, u64 p) {
      const u64 self = w.weight(w.below(logit_at(p)));
      const u64 now = by_count ? c : wt, front = by_count ? c - 1 : wt - self;
      if (front < target && target <= now) s_place = p, s_weight = wt;
      return now >= target;
    });
    __syncthreads();
    place = s_place;
    weight = s_weight;
  };
  Cut cut = {1, -1};
  u64 stay = b.weight[kBins], place, weight;
  if (near.k_on) {
    find(true, (u64)a.top_k, place, weight);
    cut.from = place;
    stay = weight;
  }
  if (near.p_on) {
    find(false, top_p_target(a.top_p, stay), place, weight);
    cut.from = max(cut.from, place);
    stay = weight;
  }
  if (a.tokens) {
    if (near.m_on) {
      // the weight of the words over the border: of the bins in front of the border's, and of its own words that are
      u64 in_bin = 0;
      for (int i = i0; i < i1; ++i) {
        const float x = logit_at(words[i]);
        const double y = w.below(x);
        if (w.bin(y) == near.lo[2] && w.over(x, a.min_z)) in_bin += w.weight(y);
      }
      stay = min(stay, b.weight[near.lo[2]] + sum_all<NT>(in_bin, b.scan[1]));
    }
    find(false, draw_target(u, stay), place, weight);
    cut.token = token_at(place);
  }
  return cut;
}

// ------------------------------------------------------------------------------------------
// Digit by digit: for rows whose bins hold more words than are sorted.
// ------------------------------------------------------------------------------------------
struct Digits {
  u64 weight[kDigitBins];
  uint32_t count[kDigitBins];
};

// The place of the first word at which the count (or weight) of the words so far reaches `target`, 1 or more, which all words from `limit`
// on together do.
template <int NT, bool BY_WEIGHT>
__device__ u64 first_to_reach(const float* row, int V, const Weigher& w, u64 target, u64 limit, Digits& d, u64 (&scan)[NT / 64], u64& s_bin) {
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
      if (p < limit || p >> above != prefix) return;
      const int bin = kDigitBins - 1 - ((int)(p >> shift) & ((1 << bits) - 1));  // the highest first
      if (BY_WEIGHT) atomicAdd(&d.weight[bin], w.weight(w.below(x)));
      else atomicAdd(&d.count[bin], 1u);
    });
    __syncthreads();
    u64 n[N], sum = 0, all;
#pragma unroll
    for (int i = 0; i < N; ++i) sum += n[i] = BY_WEIGHT ? d.weight[tid * N + i] : d.count[tid * N + i];
    u64 before = sum_before<NT>(sum, scan, all);
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

template <int NT>
__device__ Cut resolve_by_digits(const SampleArgs& a, const Weigher& w, double u, const float* row, Digits& d, u64 (&scan)[NT / 64]) {
  __shared__ u64 s_bin;
  const auto sum_from = [&](u64 limit, auto of) {
    u64 s = 0;
    each_word<NT>(row, 0, a.V, [&](float x, int v) {
      if (place_of(x, v) >= limit) s += of(x);
    });
    return sum_all<NT>(s, scan);
  };
  const auto weight = [&](float x) { return w.weight(w.below(x)); };
  Cut cut = {1, -1};
  if (a.top_k > 0 && sum_from(1, [](float) { return (u64)1; }) > (u64)a.top_k) cut.from = first_to_reach<NT, false>(row, a.V, w, a.top_k, 1, d, scan, s_bin);
  if (a.top_p < 1.0) cut.from = first_to_reach<NT, true>(row, a.V, w, top_p_target(a.top_p, sum_from(cut.from, weight)), cut.from, d, scan, s_bin);
  if (a.tokens) {
    const u64 stay = sum_from(cut.from, [&](float x) { return w.over(x, a.min_z) ? weight(x) : 0; });
    cut.token = token_at(first_to_reach<NT, true>(row, a.V, w, draw_target(u, stay), cut.from, d, scan, s_bin));
  }
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

template <int NT>
__device__ __forceinline__ void write_row(const SampleArgs& a, const Weigher& w, const Cut& cut, const float* row, float* out, int v0, int v1) {
  constexpr int N = 8;
  for (int base = v0; base < v1; base += N * NT) {
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int v = base + i * NT + (int)threadIdx.x;
      x[i] = v < v1 ? row[v] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int v = base + i * NT + (int)threadIdx.x;
      const u64 p = place_of(x[i], v);
      if (v < v1) out[v] = p >= cut.from && w.over(x[i], a.min_z) ? x[i] : -INFINITY;
    }
  }
}

template <int NT>
__global__ __launch_bounds__(NT) void sample_row_kernel(SampleArgs a) {
  __shared__ SampleSpace<NT> sp;
  __shared__ float s_max[NT / 64];
  __shared__ int s_near;
  __shared__ u64 s_scan[NT / 64];
  const int tid = threadIdx.x;
  const size_t r = blockIdx.x;
  const float* row = a.logits + r * a.V;
  float* out = a.out ? a.out + r * a.V : nullptr;
  for (int i = tid; i < kBins; i += NT) sp.bins.weight[i] = 0, sp.bins.count[i] = 0;
  if (tid == 0) s_near = 0;
  float top = -INFINITY;
  each_word<NT>(row, 0, a.V, [&](float x, int) { top = fmaxf(top, x); });
  top = block_max<NT / 64>(top, s_max);
  if (!(top > -INFINITY && top < INFINITY)) {
    if (a.tokens && tid == 0) a.tokens[r] = -1;
    if (out)
      for (int v = tid; v < a.V; v += NT) out[v] = -INFINITY;
    return;
  }
  const Weigher w = {(double)top, a.log2e_T, a.unit};
  const double u = a.tokens ? (double)a.u[r] : 0.0;
  each_word<NT>(row, 0, a.V, [&](float x, int) {
    const double y = w.below(x);
    const int b = w.bin(y);
    atomicAdd(&sp.bins.count[b], 1u);
    atomicAdd(&sp.bins.weight[b], w.weight(y));
  });
  __syncthreads();
  scan_bins(sp.bins);
  const Near near = near_bins(a, w, u, sp.bins);
  each_word<NT>(row, 0, a.V, [&](float x, int v) {
    if (!near.has(w.bin(w.below(x)))) return;
    const int at = atomicAdd(&s_near, 1);
    if (at < kNear) sp.words[at] = place_of(x, v);
  });
  __syncthreads();
  const int n = s_near;
  Cut cut;
  if (n <= kNear) {
    cut = resolve(a, w, u, sp.bins, near, sp.words, n);
  } else {
    __syncthreads();
    cut = resolve_by_digits<NT>(a, w, u, row, sp.digits, s_scan);
  }
  if (a.tokens && tid == 0) a.tokens[r] = cut.token;
  if (out) write_row<NT>(a, w, cut, row, out, 0, a.V);
}

// ------------------------------------------------------------------------------------------
// A row to several workgroups, in four launches: (1) the slices' highest logits; (2) their bins, added up; (3) the words of the near
// bins, in one list; (4) which sorts it, every slice's workgroup for itself where kept logits are written.
// ------------------------------------------------------------------------------------------
constexpr int kSliceNT = 512, kMaxSlices = 64;

__device__ __forceinline__ float top_of(const SampleArgs& a, float* s_top) {
  if (threadIdx.x < 64) {
    const float* m = a.slice_max + (size_t)blockIdx.y * kMaxSlices;
    const float top = lanes_max((int)threadIdx.x < a.slices ? m[threadIdx.x] : -INFINITY, 64);
    if (threadIdx.x == 0) *s_top = top;
  }
  __syncthreads();
  return *s_top;
}
__device__ __forceinline__ bool no_word(float top) { return !(top > -INFINITY && top < INFINITY); }

// grid (slices, rows), all of them
__global__ __launch_bounds__(kSliceNT) void sample_max_kernel(SampleArgs a) {
  __shared__ float s_max[kSliceNT / 64];
  const size_t r = blockIdx.y;
  const int v0 = min(a.V, (int)blockIdx.x * a.per), v1 = min(a.V, v0 + a.per);
  for (int i = blockIdx.x * kSliceNT + threadIdx.x; i <= kBins; i += a.slices * kSliceNT) {
    if (i < kBins) a.weight[r * kBins + i] = 0;
    a.count[r * (kBins + 1) + i] = 0;
  }
  float top = -INFINITY;
  each_word<kSliceNT>(a.logits + r * a.V, v0, v1, [&](float x, int) { top = fmaxf(top, x); });
  top = block_max<kSliceNT / 64>(top, s_max);
  if (threadIdx.x == 0) a.slice_max[r * kMaxSlices + blockIdx.x] = top;
}

__global__ __launch_bounds__(kSliceNT) void sample_bins_kernel(SampleArgs a) {
  __shared__ u64 s_weight[kBins];
  __shared__ uint32_t s_count[kBins];
  __shared__ float s_top;
  const int tid = threadIdx.x;
  const size_t r = blockIdx.y;
  const int v0 = min(a.V, (int)blockIdx.x * a.per), v1 = min(a.V, v0 + a.per);
  for (int i = tid; i < kBins; i += kSliceNT) s_weight[i] = 0, s_count[i] = 0;
  const float top = top_of(a, &s_top);
  if (no_word(top)) return;
  const Weigher w = {(double)top, a.log2e_T, a.unit};
  each_word<kSliceNT>(a.logits + r * a.V, v0, v1, [&](float x, int) {
    const double y = w.below(x);
    const int b = w.bin(y);
    atomicAdd(&s_count[b], 1u);
    atomicAdd(&s_weight[b], w.weight(y));
  });
  __syncthreads();
  for (int i = tid; i < kBins; i += kSliceNT)
    if (s_count[i]) {
      atomicAdd(&a.count[r * (kBins + 1) + i], s_count[i]);
      if (s_weight[i]) atomicAdd(&a.weight[r * kBins + i], s_weight[i]);
    }
}

template <int NT>
__device__ __forceinline__ void load_bins(const SampleArgs& a, size_t r, Bins<NT>& b) {
  for (int i = threadIdx.x; i < kBins; i += NT) {
    b.weight[i] = a.weight[r * kBins + i];
    b.count[i] = a.count[r * (kBins + 1) + i];
  }
  __syncthreads();
  scan_bins(b);
}

__global__ __launch_bounds__(kSliceNT) void sample_near_kernel(SampleArgs a) {
  __shared__ Bins<kSliceNT> bins;
  __shared__ float s_top;
  const size_t r = blockIdx.y;
  const int v0 = min(a.V, (int)blockIdx.x * a.per), v1 = min(a.V, v0 + a.per);
  const float top = top_of(a, &s_top);
  if (no_word(top)) return;
  const Weigher w = {(double)top, a.log2e_T, a.unit};
  load_bins(a, r, bins);
  const Near near = near_bins(a, w, a.tokens ? (double)a.u[r] : 0.0, bins);
  each_word<kSliceNT>(a.logits + r * a.V, v0, v1, [&](float x, int v) {
    if (!near.has(w.bin(w.below(x)))) return;
    const uint32_t at = atomicAdd(&a.count[r * (kBins + 1) + kBins], 1u);
    if (at < kNear) a.near[r * kNear + at] = place_of(x, v);
  });
}

// grid (slices or 1, rows)
__global__ __launch_bounds__(kSliceNT) void sample_finish_kernel(SampleArgs a) {
  __shared__ SampleSpace<kSliceNT> sp;
  __shared__ float s_top;
  __shared__ u64 s_scan[kSliceNT / 64];
  const int tid = threadIdx.x;
  const size_t r = blockIdx.y;
  const float* row = a.logits + r * a.V;
  float* out = a.out ? a.out + r * a.V : nullptr;
  int v0 = min(a.V, (int)blockIdx.x * a.per), v1 = min(a.V, v0 + a.per);
  const float top = top_of(a, &s_top);
  if (no_word(top)) {
    if (a.tokens && blockIdx.x == 0 && tid == 0) a.tokens[r] = -1;
    if (out)
      for (int v = v0 + tid; v < v1; v += kSliceNT) out[v] = -INFINITY;
    return;
  }
  const Weigher w = {(double)top, a.log2e_T, a.unit};
  const double u = a.tokens ? (double)a.u[r] : 0.0;
  const uint32_t n = a.count[r * (kBins + 1) + kBins];
  Cut cut;
  if (n <= kNear) {
    load_bins(a, r, sp.bins);
    const Near near = near_bins(a, w, u, sp.bins);
    for (int i = tid; i < (int)n; i += kSliceNT) sp.words[i] = a.near[r * kNear + i];
    cut = resolve(a, w, u, sp.bins, near, sp.words, (int)n);
  } else {
    // one workgroup reads the whole row, which may be where the results go
    if (blockIdx.x > 0) return;
    v0 = 0;
    v1 = a.V;
    cut = resolve_by_digits<kSliceNT>(a, w, u, row, sp.digits, s_scan);
  }
  if (a.tokens && blockIdx.x == 0 && tid == 0) a.tokens[r] = cut.token;
  if (out) write_row<kSliceNT>(a, w, cut, row, out, v0, v1);
}

static int sample_slices(int rows, int V) {
  if (V <= kShortRow) return 1;
  return std::max(1, std::min({kMaxSlices, (V + 2047) / 2048, 512 / rows}));
}
static size_t sample_row_bytes() { return kMaxSlices * sizeof(float) + kBins * sizeof(u64) + (kBins + 4) * sizeof(uint32_t) + kNear * sizeof(u64); }
size_t sample_workspace_bytes(int rows, int V) { return sample_slices(rows, V) > 1 ? rows * sample_row_bytes() : 16; }

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
  a.slices = sample_slices(rows, V);
  if (a.slices == 1) {
    if (V <= kShortRow) hipLaunchKernelGGL(sample_row_kernel<256>, dim3(rows), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(sample_row_kernel<1024>, dim3(rows), dim3(1024), 0, st, a);
    return;
  }
  a.per = (V + a.slices - 1) / a.slices;
  a.weight = (u64*)ws;
  a.near = a.weight + (size_t)rows * kBins;
  a.count = (uint32_t*)(a.near + (size_t)rows * kNear);
  a.slice_max = (float*)(a.count + (size_t)rows * (kBins + 1));
  const dim3 grid(a.slices, rows), block(kSliceNT);
  hipLaunchKernelGGL(sample_max_kernel, grid, block, 0, st, a);
  hipLaunchKernelGGL(sample_bins_kernel, grid, block, 0, st, a);
  hipLaunchKernelGGL(sample_near_kernel, grid, block, 0, st, a);
  hipLaunchKernelGGL(sample_finish_kernel, dim3(a.out ? a.slices : 1, rows), block, 0, st, a);
}

}  // namespace es
