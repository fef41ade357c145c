// Operators on KV caches [layer][sequence][KV head][slot][head_dim] (gfx950): the beams' slots put in the order of their parents,
// and the lightest slots dropped.  Bytes are moved, nothing is computed but which.
#include "launch_common.hpp"
#include "lane_ops.hpp"

namespace es {

// ------------------------------------------------------------------------------------------
// Reorder: sequence first + i takes the slots [from, to) of its parent.  A thread owns one piece of a slot of one (layer, KV head)
// for all sequences: it loads every sequence's new piece before it stores any, so the caches may be reordered in place, whatever
// the parents are.  Bound by memory: all 2048 slots of four sequences of 32 layers and 8 KV heads, three of them read, 1.88 GB, in
// 320 us (5.8 TB/s); five drafted slots of eight sequences, 7.9 MB, in 5 us, of which a launch is the larger part.  In place a sequence
// that keeps its own slots is read all the same: the whole caches of four, of which none, two or four take another's, 172, 303, 344 us.
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
//   (1) evict_select_kernel  a workgroup per (layer, sequence, KV head) finds the weight of the last heavy slot by counting, and
//                            writes the list of kept slots and their weights;
//   (2) evict_move_kernel    the kept rows of K and V, elsewhere; or evict_shift_kernel, down inside the same cache.
// Where few rows stay, (1) moves them itself: a launch less, while the list is short enough for one workgroup.  us a call, a launch
// apart and in one: 8 lists of 64, 128, 256 and 512 rows of 128 bytes 11.5, 12.3, 12.2, 12.0 and 9.1, 9.5, 9.9, 12.8; 256 lists
// of 64, 128, 256, 512 and 1024 rows of 256 bytes 12.1, 15.0, 20.4, 29.3, 58.5 and 9.5, 12.8, 18.6, 28.4, 63.5; in place the same to
// 1 us but for the last, 52 and 48.
// (2) is bound by memory: 268 MB (1024 rows of 256 lists) in 49 us, 5.5 TB/s.  (1) is bound by its chain of steps for short rows, 256 of
// 2048 weights 9.2 us, and by instructions for long ones, 256 of up to 32768 34 us.
// In place a list is one workgroup's, a barrier to every 32 KB, so few lists are slow: both launches, apart and in place, 256 lists of 2048
// slots of which 1024 stay 59 and 45 us (from memory 79), 112 of 32768 -> 16384 391 and 444, eight of 32768 -> 16384 52 and 205, eight of
// 65536 -> 32768 111 and 401.  Lists of sequences that are left alone have workgroups too, which end at once: with one of four or of
// eight sequences thinned 128 us instead of 79, with one of five 90: those that work lie a power of two apart in the grid and, by that
// pattern, meet on few CUs (not traced).
// The weight is found digit by digit: a histogram of the highest eleven bits of all weights, then of the next eleven of those that
// share these, then of the last ten.  (Bit by bit, every step counting all weights again, 256 rows of up to 32768 took 88 us.)
// ------------------------------------------------------------------------------------------
constexpr int kBins = 2048;
constexpr int kFewKept = 256;          // rows that (1) moves itself: at most so many ...
constexpr int kFewBytes = 32 * 1024;   // ... and so many bytes of K

// The order of weights as unsigned numbers: NaN below everything, the two zeros alike.  0 is no weight.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f), key = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
  return w == w ? key : 1u;
}
// The number of a key of at least minus infinity's.  Between the zeros there is none: the one below them for -0.
constexpr uint32_t kLowestKey = 0x007FFFFFu;
__device__ __forceinline__ float weight_of(uint32_t key) {
  key -= key == 0x7FFFFFFFu;
  return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}

// Running sums of two numbers over the threads of a workgroup of NW waves, in front of the thread; all: the whole sums.  sh: 2 NW
// numbers, which nobody reads any more.
struct Pair {
  int x, y;
};
template <int NW>
__device__ __forceinline__ Pair sum_before(Pair v, Pair* sh, Pair& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Pair s = {(int)lanes_running_sum(v.x), (int)lanes_running_sum(v.y)};
  if (lane == 63) sh[wave] = s;
  __syncthreads();
  Pair before = {s.x - v.x, s.y - v.y};
  all = Pair{0, 0};
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const Pair o = sh[w];
    before.x += w < wave ? o.x : 0;
    before.y += w < wave ? o.y : 0;
    all.x += o.x;
    all.y += o.y;
  }
  return before;
}

// The rows of a list of n slots, moved by a workgroup of NT threads to the front of dst, which may be src: the list ascends, so the
// rows of later rounds lie above everything that a round writes, and inside a round every load is done before the first store.
template <int NT, class Slot>
__device__ __forceinline__ void move_rows(const u32x4* src, u32x4* dst, int n, int log2_ppr, const Slot& slot_of) {
  constexpr int kPieces = 4;
  const int pieces = n << log2_ppr, mask = (1 << log2_ppr) - 1;
  for (int base = 0; base < pieces; base += NT * kPieces) {
    u32x4 x[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = min(base + j * NT + (int)threadIdx.x, pieces - 1);
      x[j] = src[((size_t)slot_of(i >> log2_ppr) << log2_ppr) + (i & mask)];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the loads are done when their values are here: the barrier alone does not wait for them
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = base + j * NT + threadIdx.x;
      if (i < pieces) dst[i] = x[j];
    }
  }
}

// grid (layers x sequences x KV heads).  A thread takes NR neighbouring slots of every run of NT * NR; weights are read again for every
// digit (a row of 65536 is 256 KB, which the L2 holds).  weights_out may be weights.
template <int NT, bool MOVE>
__global__ __launch_bounds__(NT) void evict_select_kernel(const float* weights, float* weights_out, int32_t* slots_out, EvictArgs a, const u32x4* k,
                                                          const u32x4* v, u32x4* k_out, u32x4* v_out) {
  constexpr int NW = NT / 64, NR = 8, kRun = NT * NR;
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  __shared__ i32x4 s_hist[kBins / 4];  // the highest bin first
  __shared__ Pair s_scan[2][NW];
  __shared__ int s_bin, s_over, s_in;
  __shared__ int s_kept[MOVE ? kFewKept : 1];
  __shared__ int s_slot[kRun];      // what stays of a run, on its way out: scattered stores of single words took longer than
  __shared__ float s_weight[kRun];  // everything else there
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int b = row / a.heads % a.n_seqs;
  const int n = a.len[b], keep = min(a.keep[b], n), recent = min(a.recent, keep), m = n - recent, need = keep - recent;
  if (keep <= 0) return;
  const float* w_row = weights + (size_t)row * a.max_slots;
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));  // rows need not lie on 16 bytes
  float w[NR], next[NR];
  auto load = [&](float (&to)[NR], int first) {
#pragma unroll
    for (int r = 0; r < NR; r += 4) {
      if (first + r + 3 < n) {
        const f32x4_any x = *reinterpret_cast<const f32x4_any*>(w_row + first + r);
#pragma unroll
        for (int j = 0; j < 4; ++j) to[r + j] = x[j];
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) to[r + j] = first + r + j < n ? w_row[first + r + j] : 0.f;
      }
    }
  };
  // A row of one run stays in registers; of a longer one the next run (after the last, the first) is on its way while one is used.
  load(w, tid * NR);
  auto request = [&](int run) {
    if (n > kRun) load(next, (run + kRun < n ? run + kRun : 0) + tid * NR);
  };
  auto advance = [&] {
    if (n > kRun)
#pragma unroll
      for (int r = 0; r < NR; ++r) w[r] = next[r];
  };
  // Keys over `above` stay, and of those equal to `tie` the first `ties`.
  uint32_t above = 0xFFFFFFFFu, tie = 0;
  int ties = 0;
  if (need > 0) {
    uint32_t prefix = 0;
    int left = need;
    for (int digit = 0; digit < 3; ++digit) {
      const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
      for (int i = tid; i < kBins / 4; i += NT) s_hist[i] = i32x4{0, 0, 0, 0};
      __syncthreads();
      int* hist = reinterpret_cast<int*>(s_hist);
      for (int run = 0; run < n; run += kRun) {
        const int first = run + tid * NR;
        request(run);
        auto count = [&](auto whole_run) {
#pragma unroll
          for (int r = 0; r < NR; ++r) {
            const uint32_t key = weight_key(w[r]);
            const bool counts = (int)(decltype(whole_run)::value || first + r < m) & (int)(digit == 0 || key >> (shift + bits) == prefix);
            if (!decltype(whole_run)::value || digit > 0) {
              if (!__ballot(counts)) continue;
            }
            const int bin = kBins - 1 - (int)((key >> shift) & ((1u << bits) - 1));
            // many equal weights are common (slots that nothing has attended to have none): those of the first lane's bin at once
            const int lead_bin = __builtin_amdgcn_readfirstlane(bin);
            const unsigned long long same = __ballot(counts && bin == lead_bin);
            if (counts && bin != lead_bin) atomicAdd(&hist[bin], 1);
            if (lane == 0) atomicAdd(&hist[lead_bin], __popcll(same));
          }
        };
        if (run + kRun <= m) count(std::true_type{});
        else count(std::false_type{});
        advance();
      }
      __syncthreads();
      // the bin that the left-th highest lies in
      constexpr int kPer = kBins / NT;
      int in[kPer], own = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) own += in[i] = hist[tid * kPer + i];
      Pair all;
      int over = sum_before<NW>(Pair{own, 0}, s_scan[digit & 1], all).x;
      if (over < left && left <= over + own) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if (over < left && left <= over + in[i]) {
            s_bin = kBins - 1 - (tid * kPer + i);
            s_over = over;
            s_in = in[i];
          }
          over += in[i];
        }
      }
      __syncthreads();
      prefix = prefix << bits | (uint32_t)s_bin;
      left -= s_over;
      const bool whole = s_in == left;  // everything with this prefix stays
      if (whole || digit == 2) {
        tie = prefix << shift;
        above = whole ? (tie ? tie - 1 : 0) : tie;
        ties = whole ? 0 : left;
        break;
      }
    }
  }
  // Slots that stay: their places are running sums over the threads, in the order of the slots.  A place lies below its slot, in
  // runs that have been read.
  int32_t* list = slots_out + (size_t)row * a.out_slots;
  float* w_list = weights_out + (size_t)row * a.out_slots;
  Pair so_far = {0, 0};  // sure to stay, and equal to `tie`
  const bool numbers = ties == 0 && above >= kLowestKey;
  const float over = weight_of(above);  // 0xFFFFFFFF: a NaN, which nothing is over
  __syncthreads();
  int turn = 0;
  for (int run = 0; run < n; run += kRun, turn ^= 1) {
    const int first = run + tid * NR;
    request(run);
    int base = 0, end = 0;
    // plain: a slot stays if its weight is over a number, which as a rule is all there is to it
    auto emit = [&](auto plain, auto whole_run) {
      constexpr bool P = decltype(plain)::value, W = decltype(whole_run)::value;
      auto stays = [&](int r) { return W || first + r < m ? (P ? w[r] > over : weight_key(w[r]) > above) : first + r < n; };
      auto tied = [&](int r) { return !P && ties > 0 && first + r < m && weight_key(w[r]) == tie; };
      Pair own = {0, 0}, all;
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        own.x += stays(r);
        if (!P) own.y += tied(r);
      }
      Pair before = sum_before<NW>(own, s_scan[turn], all);
      base = so_far.x + min(so_far.y, ties);
      before.x += so_far.x - base;
      before.y += so_far.y;
      so_far.x += all.x;
      so_far.y += all.y;
      end = so_far.x + min(so_far.y, ties);
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const bool s = stays(r), t = tied(r);
        if (s || (!P && t && before.y < ties)) {
          const int at = before.x + (P ? 0 : min(before.y, ties));
          s_slot[at] = first + r;
          s_weight[at] = w[r];
        }
        before.x += s;
        if (!P) before.y += t;
      }
    };
    if (!numbers) emit(std::false_type{}, std::false_type{});
    else if (run + kRun <= m) emit(std::true_type{}, std::true_type{});
    else emit(std::true_type{}, std::false_type{});
    __syncthreads();
    for (int i = tid; i < end - base; i += NT) {
      list[base + i] = s_slot[i];
      w_list[base + i] = s_weight[i];
      if (MOVE) s_kept[base + i] = s_slot[i];
    }
    advance();
  }
  if (MOVE) {
    if (k == k_out && keep == n) return;
    __syncthreads();
    const size_t in = (size_t)row * a.max_slots << a.log2_ppr, out = (size_t)row * a.out_slots << a.log2_ppr;
    const auto slot = [&](int j) { return s_kept[j]; };
    move_rows<NT>(k + in, k_out + out, keep, a.log2_ppr, slot);
    move_rows<NT>(v + in, v_out + out, keep, a.log2_ppr, slot);
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

// The same inside one cache: a workgroup per (layer, sequence, KV head) and K or V.
constexpr int kShiftThreads = 512;
__global__ __launch_bounds__(kShiftThreads) void evict_shift_kernel(u32x4* k, u32x4* v, const int32_t* __restrict__ slots, EvictArgs a) {
  const int row = blockIdx.x, b = row / a.heads % a.n_seqs;
  const int kept = min(a.keep[b], a.len[b]);
  if (kept == a.len[b]) return;
  u32x4* rows = (blockIdx.y ? v : k) + ((size_t)row * a.max_slots << a.log2_ppr);
  const int32_t* list = slots + (size_t)row * a.out_slots;
  move_rows<kShiftThreads>(rows, rows, kept, a.log2_ppr, [&](int j) { return list[j]; });
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
  const bool move = most <= kFewKept && most * slot_bytes <= kFewBytes;
  auto select = [&](int threads, auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(rows), dim3(threads), 0, st, weights, weights_out, slots_out, a, (const u32x4*)k, (const u32x4*)v,
                       (u32x4*)k_out, (u32x4*)v_out);
  };
  if (longest <= 2048 && move) select(256, evict_select_kernel<256, true>);
  else if (longest <= 2048) select(256, evict_select_kernel<256, false>);
  else if (move) select(1024, evict_select_kernel<1024, true>);
  else select(1024, evict_select_kernel<1024, false>);
  if (move) return;
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
