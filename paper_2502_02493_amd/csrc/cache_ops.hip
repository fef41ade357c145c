// Operators on KV caches [layer][sequence][KV head][slot][head_dim] (gfx950): the beams' slots put in the order of their parents,
// and the lightest slots dropped.  Bytes are moved, nothing is computed but which.
#include "launch_common.hpp"

namespace es {

// ------------------------------------------------------------------------------------------
// Reorder: sequence first + i takes the slots [from, to) of its parent.  A thread owns one piece of a slot of one (layer, KV head)
// for all sequences: it loads every sequence's new piece before it stores any, so the caches may be reordered in place, whatever
// the parents are.
// ------------------------------------------------------------------------------------------
constexpr int kReorderThreads = 256;

template <int NS, typename P>
__global__ __launch_bounds__(kReorderThreads) void reorder_kernel(const P* ks, const P* vs, P* kd, P* vd, ReorderArgs a) {
  const size_t i = (size_t)blockIdx.x * kReorderThreads + threadIdx.x;
  if (i >= a.run) return;
  const int l = blockIdx.y / a.heads, h = blockIdx.y % a.heads;
  const size_t base = l * a.layer_pitch + h * a.head_pitch + a.offset + i;
  const P* src = (blockIdx.z ? vs : ks) + base;
  P* dst = (blockIdx.z ? vd : kd) + base;
  P v[NS];
  int from[NS];  // uniform
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const int i_seq = min(j, a.n - 1), self = a.first + i_seq;
    from[j] = a.parents ? self : a.source;
    if (a.parents) {
      const int p = __builtin_amdgcn_readfirstlane(a.parents[i_seq]);
      if (p >= 0 && p < a.beams) from[j] = a.first + i_seq / a.beams * a.beams + p;
    }
    v[j] = src[from[j] * a.seq_pitch];
  }
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const int self = a.first + j;
    if (j < a.n && (from[j] != self || !a.in_place)) dst[self * a.seq_pitch] = v[j];
  }
}

template <typename P>
static void launch_reorder_as(const void* k, const void* v, void* k_out, void* v_out, const ReorderArgs& all, int n_layers, hipStream_t st) {
  // the grid's second extent is limited: whole layers at a time
  const int at_once = std::max(1, 65535 / all.heads);
  const unsigned nx = (unsigned)((all.run + kReorderThreads - 1) / kReorderThreads), nz = v ? 2 : 1;
  for (int l0 = 0; l0 < n_layers; l0 += at_once) {
    const int nl = std::min(at_once, n_layers - l0);
    ReorderArgs a = all;
    a.offset += l0 * a.layer_pitch;
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(nx, nl * a.heads, nz), dim3(kReorderThreads), 0, st, (const P*)k, (const P*)v, (P*)k_out, (P*)v_out, a);
    };
    if (a.n <= 4) go(reorder_kernel<4, P>);
    else if (a.n <= 8) go(reorder_kernel<8, P>);
    else go(reorder_kernel<16, P>);
  }
}

void launch_kv_reorder(const void* k, const void* v, void* k_out, void* v_out, const KvLayout& g, int slot_bytes, const int32_t* parents, int source,
                       int first, int n, int beams, int from, int to, hipStream_t st) {
  if (to <= from || n < 1) return;
  const int piece = slot_bytes % 16 == 0 ? 16 : 4, ppr = slot_bytes / piece;
  ReorderArgs a;
  a.parents = parents; a.source = source; a.first = first; a.n = n; a.beams = beams; a.heads = g.n_heads;
  a.in_place = k == k_out;
  a.run = (size_t)(to - from) * ppr;
  a.offset = (size_t)from * ppr;
  a.head_pitch = (size_t)g.max_slots * ppr;
  a.seq_pitch = a.head_pitch * g.n_heads;
  a.layer_pitch = a.seq_pitch * g.n_seqs;
  if (piece == 16) launch_reorder_as<u32x4>(k, v, k_out, v_out, a, g.n_layers, st);
  else launch_reorder_as<uint32_t>(k, v, k_out, v_out, a, g.n_layers, st);
}

// ------------------------------------------------------------------------------------------
// Evict: of every (layer, sequence, KV head) the last `recent` slots and the heaviest of the others stay, in slot order.
//   (1) evict_select_kernel  a workgroup per (layer, sequence, KV head) holds its weights in registers, finds the weight of the
//                            last heavy slot bit by bit, and writes the list of kept slots and their weights;
//   (2) evict_move_kernel    the kept rows of K and V, elsewhere; or evict_shift_kernel, down inside the same cache.
// ------------------------------------------------------------------------------------------
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;

// The order of weights as unsigned numbers: NaN below everything, the two zeros alike.  0 is no weight.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w == w ? (u & 0x80000000u ? ~u : u | 0x80000000u) : 1u;
}

// grid (layers x sequences x KV heads); NR: weights a thread holds.  weights_out may be weights.
template <int NR>
__global__ __launch_bounds__(kSelThreads) void evict_select_kernel(const float* weights, float* weights_out, int32_t* slots_out, EvictArgs a) {
  __shared__ int s_count[2][kSelWaves];
  __shared__ int s_gt[NR * kSelWaves], s_eq[NR * kSelWaves];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = row / a.heads % a.n_seqs;
  const int n = a.len[b], keep = min(a.keep[b], n), recent = min(a.recent, keep), m = n - recent, need = keep - recent;
  if (keep <= 0) return;
  const float* w_row = weights + (size_t)row * a.max_slots;
  float w[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int s = r * kSelThreads + tid;
    w[r] = s < n ? w_row[s] : 0.f;
  }
  auto key = [&](int r) { return r * kSelThreads + tid < m ? weight_key(w[r]) : 0u; };
  int phase = 0;
  auto count = [&](uint32_t least) {  // keys >= least, over the workgroup
    int c = 0;
#pragma unroll
    for (int r = 0; r < NR; ++r) c += __popcll(__ballot(key(r) >= least));
    if (lane == 0) s_count[phase][wave] = c;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int i = 0; i < kSelWaves; ++i) all += s_count[phase][i];
    phase ^= 1;
    return all;
  };
  // The need-th largest key, from the highest bit down.  above: keys over it that all stay; equal ones stay up to `need`.
  uint32_t t = 0, above;
  int ties;
  bool whole = need == 0;  // keys > above are exactly the ones that stay
  if (!whole) {
    for (int bit = 31; bit >= 0 && !whole; --bit) {
      const uint32_t c = t | 1u << bit;
      const int k = count(c);
      if (k >= need) t = c;
      whole = k == need;
    }
  }
  if (need == 0) {
    above = 0xFFFFFFFFu;
    ties = 0;
  } else if (whole) {
    above = t - 1;
    ties = 0;
  } else {
    above = t;
    ties = need - (t == 0xFFFFFFFFu ? 0 : count(t + 1));
  }
  auto stays = [&](int r) {
    const int s = r * kSelThreads + tid;
    return s < m ? key(r) > above : s < n;
  };
  auto tied = [&](int r) { return ties > 0 && r * kSelThreads + tid < m && key(r) == above; };
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int gt = __popcll(__ballot(stays(r))), eq = __popcll(__ballot(tied(r)));
    if (lane == 0) {
      s_gt[r * kSelWaves + wave] = gt;
      s_eq[r * kSelWaves + wave] = eq;
    }
  }
  __syncthreads();
  // running sums over (r, wave), the order of the slots
  if (wave == 0) {
    int base_gt = 0, base_eq = 0;
    for (int i0 = 0; i0 < NR * kSelWaves; i0 += 64) {
      const int i = i0 + lane;
      const int gt = s_gt[i], eq = s_eq[i];
      int sg = gt, se = eq;
      for (int off = 1; off < 64; off <<= 1) {
        const int og = __shfl_up(sg, off, 64), oe = __shfl_up(se, off, 64);
        if (lane >= off) sg += og, se += oe;
      }
      s_gt[i] = base_gt + sg - gt;
      s_eq[i] = base_eq + se - eq;
      base_gt += __shfl(sg, 63, 64);
      base_eq += __shfl(se, 63, 64);
    }
  }
  __syncthreads();
  const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const bool st = stays(r), eq = tied(r);
    const int gt_before = s_gt[r * kSelWaves + wave] + __popcll(__ballot(st) & below);
    const int eq_before = s_eq[r * kSelWaves + wave] + __popcll(__ballot(eq) & below);
    if (st || (eq && eq_before < ties)) {
      const size_t at = (size_t)row * a.out_slots + gt_before + min(eq_before, ties);
      slots_out[at] = r * kSelThreads + tid;
      weights_out[at] = w[r];
    }
  }
}

// grid (pieces of the longest sequence's kept rows, layers x sequences x KV heads, K / V)
constexpr int kMoveThreads = 256, kMovePieces = 4;
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(const u32x4* k, const u32x4* v, u32x4* k_out, u32x4* v_out,
                                                                  const int32_t* __restrict__ slots, EvictArgs a) {
  const int row = a.row0 + blockIdx.y, b = row / a.heads % a.n_seqs;
  const int kept = min(a.keep[b], a.len[b]), log2_ppr = a.log2_ppr;
  const u32x4* src = (blockIdx.z ? v : k) + ((size_t)row * a.max_slots << log2_ppr);
  u32x4* dst = (blockIdx.z ? v_out : k_out) + ((size_t)row * a.out_slots << log2_ppr);
  const int32_t* list = slots + (size_t)row * a.out_slots;
  const int i0 = blockIdx.x * (kMoveThreads * kMovePieces) + threadIdx.x, n = kept << log2_ppr;
  u32x4 x[kMovePieces];
#pragma unroll
  for (int j = 0; j < kMovePieces; ++j) {
    const int i = i0 + j * kMoveThreads;
    if (i < n) x[j] = src[((size_t)list[i >> log2_ppr] << log2_ppr) + (i & ((1 << log2_ppr) - 1))];
  }
#pragma unroll
  for (int j = 0; j < kMovePieces; ++j) {
    const int i = i0 + j * kMoveThreads;
    if (i < n) dst[i] = x[j];
  }
}

// The same inside one cache: a workgroup per (layer, sequence, KV head) and K or V walks the list upwards.  A kept row moves to a
// lower slot or stays, so the rows of later rounds lie above everything that this round writes; inside a round every load is done
// before the first store.
constexpr int kShiftThreads = 512, kShiftPieces = 4;
__global__ __launch_bounds__(kShiftThreads) void evict_shift_kernel(u32x4* k, u32x4* v, const int32_t* __restrict__ slots, EvictArgs a) {
  const int row = blockIdx.x, b = row / a.heads % a.n_seqs;
  const int kept = min(a.keep[b], a.len[b]), log2_ppr = a.log2_ppr;
  if (kept == a.len[b]) return;
  u32x4* rows = (blockIdx.y ? v : k) + ((size_t)row * a.max_slots << log2_ppr);
  const int32_t* list = slots + (size_t)row * a.out_slots;
  const int n = kept << log2_ppr;
  for (int base = 0; base < n; base += kShiftThreads * kShiftPieces) {
    u32x4 x[kShiftPieces];
#pragma unroll
    for (int j = 0; j < kShiftPieces; ++j) {
      const int i = base + j * kShiftThreads + threadIdx.x;
      if (i < n) x[j] = rows[((size_t)list[i >> log2_ppr] << log2_ppr) + (i & ((1 << log2_ppr) - 1))];
    }
    // the loads are done when their values are here: the barrier alone does not wait for them
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kShiftPieces; ++j) {
      const int i = base + j * kShiftThreads + threadIdx.x;
      if (i < n) rows[i] = x[j];
    }
  }
}

void launch_kv_evict(const void* k, const void* v, const float* weights, void* k_out, void* v_out, float* weights_out, int32_t* slots_out,
                     const KvLayout& g, int slot_bytes, const EvictArgs& plan, hipStream_t st) {
  EvictArgs a = plan;
  a.heads = g.n_heads; a.n_seqs = g.n_seqs; a.max_slots = g.max_slots; a.row0 = 0;
  a.log2_ppr = __builtin_ctz(slot_bytes / 16);
  int longest = 0, most = 0;
  for (int b = 0; b < g.n_seqs; ++b)
    if (a.keep[b] > 0) longest = std::max(longest, a.len[b]), most = std::max(most, std::min(a.keep[b], a.len[b]));
  if (most == 0) return;
  const int rows = g.n_layers * g.n_seqs * g.n_heads;
  auto select = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(rows), dim3(kSelThreads), 0, st, weights, weights_out, slots_out, a); };
  if (longest <= 4 * kSelThreads) select(evict_select_kernel<4>);
  else if (longest <= 16 * kSelThreads) select(evict_select_kernel<16>);
  else if (longest <= 32 * kSelThreads) select(evict_select_kernel<32>);
  else select(evict_select_kernel<64>);
  if (k == k_out) {
    hipLaunchKernelGGL(evict_shift_kernel, dim3(rows, 2), dim3(kShiftThreads), 0, st, (u32x4*)k_out, (u32x4*)v_out, slots_out, a);
    return;
  }
  const unsigned nx = (unsigned)((((size_t)most << a.log2_ppr) + kMoveThreads * kMovePieces - 1) / (kMoveThreads * kMovePieces));
  for (; a.row0 < rows; a.row0 += 65535)
    hipLaunchKernelGGL(evict_move_kernel, dim3(nx, std::min(65535, rows - a.row0), 2), dim3(kMoveThreads), 0, st, (const u32x4*)k,
                       (const u32x4*)v, (u32x4*)k_out, (u32x4*)v_out, slots_out, a);
}

}  // namespace es
