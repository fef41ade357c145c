// Sampling under top-k, top-p and min-p from given random numbers (gfx950).
//
// Words stand in the order of their logits, the highest first, of equal ones the lowest token; each has the weight
// exp((x - max) / T).  What stays is a run from the front of that order (top-k, top-p and min-p each keep one, the shortest counts), and
// the token drawn is the first whose running weight passes u times that of the run.  So all of it comes down to one question: which word
// of the order is the first to bring a running count or weight to a given number?  It is answered digit by digit of the words' place
// numbers (the logit's 32 bits in the order of floats, then the token), by a histogram of counts and weights for each.
// Weights are whole multiples of 2^-s: sums of them are exact, so neither the order of atomic additions nor how a row is cut up
// shows in a result.
#include "launch_common.hpp"
#include "lane_ops.hpp"

namespace es {

typedef unsigned long long u64;
constexpr int kTokenBits = 20;
static_assert(kMaxSampleVocab == 1 << kTokenBits, "a place number holds a token");
constexpr int kSampleThreads = 1024;
constexpr int kSampleBins = 2048;

// A word's place number: the higher, the earlier in the order; 0 is no word (minus infinity, NaN).
__device__ __forceinline__ u64 place_of(float x, int v) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(x + 0.f);  // the two zeros alike
  const uint32_t key = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
  return (u64)key << kTokenBits | (u64)(kMaxSampleVocab - 1 - v);
}

struct SampleArgs {
  const float* logits;
  const float* u;
  int V, top_k;  // top_k 0: all
  double T, inv_T, top_p, min_z;  // min_z: T log(min_p), what a logit may lie below the highest; minus infinity: all
  double unit;                    // 2^s
  int32_t* tokens;
  float* out;
};

struct RowOf {
  const float* x;
  double top, inv_T, unit;
  int V;
  __device__ __forceinline__ u64 weight(float v) const { return (u64)__double2ull_rn(exp(((double)v - top) * inv_T) * unit); }
};

struct SampleShared {
  u64 weight[kSampleBins];
  uint32_t count[kSampleBins];
  u64 wave_weight[kSampleThreads / 64];
  uint32_t wave_count[kSampleThreads / 64];
  int bin;
  u64 over_weight;
  uint32_t over_count;
  float wave_max[kSampleThreads / 64];
};

__device__ __forceinline__ u64 block_sum_u64(u64 v, SampleShared& sh) {
  for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.wave_weight[threadIdx.x >> 6] = v;
  __syncthreads();
  u64 s = 0;
  for (int w = 0; w < kSampleThreads / 64; ++w) s += sh.wave_weight[w];
  return s;
}

// The place of the first word at which the count (or weight) of the words so far reaches `target`, 1 or more, which all words from `limit`
// on together do.
template <bool BY_WEIGHT>
__device__ u64 first_to_reach(const RowOf& r, u64 target, u64 limit, SampleShared& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  u64 prefix = 0;
  int shift = 32 + kTokenBits;
  for (int digit = 0; digit < 5; ++digit) {
    const int bits = digit < 2 ? 11 : 10, above = shift;
    shift -= bits;
    for (int i = tid; i < kSampleBins; i += kSampleThreads) sh.weight[i] = 0, sh.count[i] = 0;
    __syncthreads();
    for (int v = tid; v < r.V; v += kSampleThreads) {
      const float x = r.x[v];
      const u64 p = place_of(x, v);
      if (p == 0 || p < limit || p >> above != prefix) continue;
      const int bin = (int)(p >> shift) & ((1 << bits) - 1);
      atomicAdd(&sh.count[bin], 1u);
      if (BY_WEIGHT) {
        const u64 w = r.weight(x);
        if (w) atomicAdd(&sh.weight[bin], w);
      }
    }
    __syncthreads();
    // running sums from the highest bin down, two bins a thread
    const int b1 = kSampleBins - 1 - 2 * tid, b0 = b1 - 1;
    const u64 n1 = BY_WEIGHT ? sh.weight[b1] : sh.count[b1], n0 = BY_WEIGHT ? sh.weight[b0] : sh.count[b0];
    u64 run = n1 + n0;
    for (int off = 1; off < 64; off <<= 1) {
      const u64 o = __shfl_up(run, off, 64);
      if (lane >= off) run += o;
    }
    if (lane == 63) sh.wave_weight[wave] = run;
    __syncthreads();
    u64 before = run - (n1 + n0);
    for (int w = 0; w < wave; ++w) before += sh.wave_weight[w];
    if (before < target && target <= before + n1) sh.bin = b1, sh.over_weight = before;
    else if (before + n1 < target && target <= before + n1 + n0) sh.bin = b0, sh.over_weight = before + n1;
    __syncthreads();
    prefix = prefix << bits | (u64)sh.bin;
    target -= sh.over_weight;
  }
  return prefix;
}

__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(SampleArgs a) {
  __shared__ SampleShared sh;
  const int tid = threadIdx.x;
  const float* row = a.logits + (size_t)blockIdx.x * a.V;
  float top = -INFINITY;
  for (int v = tid; v < a.V; v += kSampleThreads) {
    const float x = row[v];
    if (x > top) top = x;
  }
  top = block_max<kSampleThreads / 64>(top, sh.wave_max);
  const bool none = !(top > -INFINITY && top < INFINITY);
  float* out = a.out ? a.out + (size_t)blockIdx.x * a.V : nullptr;
  if (none) {
    if (a.tokens && tid == 0) a.tokens[blockIdx.x] = -1;
    if (out)
      for (int v = tid; v < a.V; v += kSampleThreads) out[v] = -INFINITY;
    return;
  }
  const RowOf r = {row, (double)top, a.inv_T, a.unit, a.V};
  u64 from = 1;  // the last place that stays
  if (a.top_k > 0) {
    u64 words = 0;
    for (int v = tid; v < a.V; v += kSampleThreads) words += row[v] > -INFINITY;
    if (block_sum_u64(words, sh) > (u64)a.top_k) from = first_to_reach<false>(r, a.top_k, from, sh);
  }
  const auto weight_from = [&](u64 limit) {
    u64 w = 0;
    for (int v = tid; v < a.V; v += kSampleThreads) {
      const u64 p = place_of(row[v], v);
      if (p && p >= limit) w += r.weight(row[v]);
    }
    return block_sum_u64(w, sh);
  };
  if (a.top_p < 1.0) {
    const u64 all = weight_from(from);
    from = first_to_reach<true>(r, min(all, max((u64)1, (u64)ceil(a.top_p * (double)all))), from, sh);
  }
  if (a.min_z > -INFINITY) {
    u64 least = ~0ull;
    for (int v = tid; v < a.V; v += kSampleThreads) {
      const float x = row[v];
      if ((double)x - r.top >= a.min_z) least = min(least, place_of(x, v));
    }
    for (int off = 32; off; off >>= 1) least = min(least, __shfl_xor(least, off, 64));
    __syncthreads();
    if ((tid & 63) == 0) sh.wave_weight[tid >> 6] = least;
    __syncthreads();
    for (int w = 0; w < kSampleThreads / 64; ++w) least = min(least, sh.wave_weight[w]);
    from = max(from, least);
  }
  if (a.tokens) {
    const u64 all = weight_from(from);
    const double u = (double)a.u[blockIdx.x];
    const u64 target = u < 1.0 ? min(all, (u64)(max(u, 0.0) * (double)all) + 1) : all;
    const u64 at = first_to_reach<true>(r, target, from, sh);
    if (tid == 0) a.tokens[blockIdx.x] = kMaxSampleVocab - 1 - (int)(at & (kMaxSampleVocab - 1));
  }
  if (out)
    for (int v = tid; v < a.V; v += kSampleThreads) {
      const float x = row[v];
      const u64 p = place_of(x, v);
      out[v] = p && p >= from ? x : -INFINITY;
    }
}

size_t sample_workspace_bytes(int rows, int V) { return 16; }

void launch_sample(const float* logits, const float* u, int rows, int V, double T, int top_k, double top_p, double min_p, int32_t* tokens_out,
                   float* logits_out, void* ws, hipStream_t st) {
  SampleArgs a;
  a.logits = logits; a.u = u; a.V = V; a.top_k = top_k; a.T = T; a.inv_T = 1.0 / T; a.top_p = top_p;
  a.min_z = min_p > 0.0 ? T * log(min_p) : -INFINITY;
  int bits = 0;
  while ((1 << bits) < V) ++bits;
  a.unit = ldexp(1.0, std::min(52, 62 - bits));
  a.tokens = tokens_out; a.out = logits_out;
  hipLaunchKernelGGL(sample_row_kernel, dim3(rows), dim3(kSampleThreads), 0, st, a);
}

}  // namespace es
