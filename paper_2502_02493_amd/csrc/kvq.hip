// Caches held in 4 bits (gfx950): slots brought in and read back.  32 neighbouring channels of a slot share a power of two
// 2^E, E = max(floor(log2(max)) - 2, -120); a code is the nearest E2M1 number to x 2^-E, which the conversion instructions round
// to (ties to the even code, 6 above) and give back without rounding.  A scale byte of 255 stands for NaN.
#include "launch_common.hpp"
#include "lane_ops.hpp"

namespace es {

template <typename T>
struct Oct {  // eight neighbouring values
  u32x4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Oct<T> fetch_oct(const T* p) {
  Oct<T> o;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(T) / 2); ++i) o.w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + i);
  return o;
}
__device__ __forceinline__ void unpack_oct(const Oct<bf16_t>& o, float (&x)[8]) { unpack<bf16_t>(o.w[0], x); }
__device__ __forceinline__ void unpack_oct(const Oct<float>& o, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(o.w[i / 4][i % 4]);
}

// Eight codes of a lane, the scale shared with the three lanes beside it (groups of four).
struct Coded {
  uint32_t codes, scale;
};
__device__ __forceinline__ Coded encode(const float (&x)[8]) {
  uint32_t top = 0;  // magnitudes in the order of their bits: infinities and NaN above all numbers
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));  // quad_perm [1,0,3,2]
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));  // quad_perm [2,3,0,1]
  if (top >= 0x7F800000u) return Coded{0u, 255u};
  const int byte = max((int)(top >> 23) - 2, 7);  // E + 127; below the normal numbers the exponent field is 0
  const float unit = __uint_as_float((uint32_t)byte << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], unit, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], unit, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], unit, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], unit, 3);
  return Coded{c, (uint32_t)byte};
}
// ... and as eight bf16
__device__ __forceinline__ u32x4 decode(uint32_t codes, uint32_t scale) {
  const float unit = __uint_as_float(scale << 23);  // 255: infinity, which the conversion makes NaN of
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3))};
}

__device__ __forceinline__ int entry_of(const KvqMoveArgs& a) {
  int e = 0;
#pragma unroll
  for (int i = 1; i < kMaxCols; ++i) e += (int)blockIdx.x >= a.first_wg[i];
  return e;
}

// A workgroup: the slots of one block of kKvqBlock that a sequence stores, in one layer and KV head, of K (z = 0) or V.  A lane
// takes eight channels of a slot, the scale is the maximum over four lanes.  K's bounds are taken from the values as they are held, from all slots of
// the block: those that were there are read back, which a block's workgroup alone writes.
// Bound: memory.  2048 slots of bf16 in 32 layers of 8 KV heads of 128, 268 MB read and 73 written: 72 us (4.7 TB/s; a copy that moves as many bytes
// 65), the bounds 8 of them.  What is read once goes past the caches (91 us otherwise), what is written, which the next attention reads, does not
// (codes written past them too: 4 us more).  Of fp32, 537 MB read and 73 written, 114 us (5.3 TB/s).  One slot of each of sixteen sequences: 4.6 us, a launch and three rounds through memory.
template <typename T, int HD>
__global__ __launch_bounds__(256) void kvq_store_kernel(KvqMoveArgs a) {
  constexpr int kOcts = HD / 8, kUnits = kKvqBlock * kOcts, kTurns = kUnits / 256;
  __shared__ u32x4 s_held[kUnits];  // [slot][HD] bf16
  __shared__ float s_lo[4][HD], s_hi[4][HD];
  const int ei = entry_of(a), tid = threadIdx.x;
  const KvqMoveEntry& e = a.entry[ei];
  const int lh = a.lh0 + blockIdx.y, l = lh / a.heads, h = lh % a.heads;
  const size_t row = ((size_t)l * a.n_seqs + e.seq) * a.heads + h;
  const int block = e.at4 / kKvqBlock + blockIdx.x - a.first_wg[ei], slot0 = block * kKvqBlock;
  const T* src = reinterpret_cast<const T*>(blockIdx.z ? a.v : a.k) + row * a.slots * HD;
  uint32_t* codes = reinterpret_cast<uint32_t*>(blockIdx.z ? a.c.vc : a.c.kc) + row * a.max_slots * kOcts;
  uint8_t* scales = (blockIdx.z ? a.c.vs : a.c.ks) + row * a.max_slots * (HD / 32);
  const bool bounds = blockIdx.z == 0 && a.c.bounds;
  Oct<T> x[kTurns];
#pragma unroll
  for (int j = 0; j < kTurns; ++j) {
    const int u = j * 256 + tid, slot = slot0 + u / kOcts, i = slot - e.at4;
    if (i >= 0 && i < e.n) x[j] = fetch_oct(src + (size_t)(e.at + i) * HD + u % kOcts * 8);
  }
#pragma unroll
  for (int j = 0; j < kTurns; ++j) {
    const int u = j * 256 + tid, slot = slot0 + u / kOcts, i = slot - e.at4;  // the four lanes of a scale: of one slot
    Coded c = {0u, 255u};
    if (i >= 0 && i < e.n) {
      float v[8];
      unpack_oct(x[j], v);
      c = encode(v);
      codes[(size_t)slot * kOcts + u % kOcts] = c.codes;
      if (u % 4 == 0) scales[(size_t)slot * (HD / 32) + u % kOcts / 4] = (uint8_t)c.scale;
    } else if (bounds && slot < e.len) {
      c.codes = codes[(size_t)slot * kOcts + u % kOcts];
      c.scale = scales[(size_t)slot * (HD / 32) + u % kOcts / 4];
    }
    if (bounds) s_held[u] = decode(c.codes, c.scale);  // slots past the last: NaN, which the bounds pass over
  }
  if (!bounds) return;
  __syncthreads();
  constexpr int kPairs = HD / 2, kParts = 256 / kPairs, kSlots = kKvqBlock / kParts;
  const uint32_t* held = reinterpret_cast<const uint32_t*>(s_held);
  const int pair = tid % kPairs, part = tid / kPairs;
  float lo[2] = {INFINITY, INFINITY}, hi[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    const uint32_t w = held[(part * kSlots + s) * kPairs + pair];
    const float x0 = __uint_as_float(w << 16), x1 = __uint_as_float(w & 0xFFFF0000u);
    lo[0] = fminf(lo[0], x0); hi[0] = fmaxf(hi[0], x0);
    lo[1] = fminf(lo[1], x1); hi[1] = fmaxf(hi[1], x1);
  }
  // HD 64 has eight parts: two to each of the four places, joined inside the wave
  if constexpr (kParts == 8) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      lo[i] = across<true>(lo[i], [](float u, float v) { return fminf(u, v); });
      hi[i] = across<true>(hi[i], [](float u, float v) { return fmaxf(u, v); });
    }
  }
  const int wave = tid >> 6;
  s_lo[wave][2 * pair] = lo[0]; s_lo[wave][2 * pair + 1] = lo[1];
  s_hi[wave][2 * pair] = hi[0]; s_hi[wave][2 * pair + 1] = hi[1];
  __syncthreads();
  if (tid >= HD) return;
  const int n_blocks = (a.max_slots + kKvqBlock - 1) / kKvqBlock;
  uint16_t* out = a.c.bounds + (row * n_blocks + block) * 2 * HD + tid;
  const float l4 = fminf(fminf(s_lo[0][tid], s_lo[1][tid]), fminf(s_lo[2][tid], s_lo[3][tid]));
  const float h4 = fmaxf(fmaxf(s_hi[0][tid], s_hi[1][tid]), fmaxf(s_hi[2][tid], s_hi[3][tid]));
  out[0] = (uint16_t)(__float_as_uint(l4) >> 16);  // bf16 numbers: nothing is cut off
  out[HD] = (uint16_t)(__float_as_uint(h4) >> 16);
}

// The way back: a lane takes eight channels of a slot.  Bound: memory, by what it writes, past the caches: the same 2048 slots 49 us (6.9 TB/s
// of reads and writes), 57 through them.  Both launches with one octet under way in a lane 141 us, two 116, four 118, eight 119.
// Into fp32, 73 MB read and 537 written, 249 us (2.4 TB/s): a lane writes two pieces of 16 bytes, so that a store of the wave leaves every other piece out;
// how much of the time that is has not been measured apart.
constexpr int kLoadTurns = 2;
template <typename T, int HD>
__global__ __launch_bounds__(256) void kvq_load_kernel(KvqMoveArgs a) {
  constexpr int kOcts = HD / 8;
  const int ei = entry_of(a);
  const KvqMoveEntry& e = a.entry[ei];
  const int lh = a.lh0 + blockIdx.y, l = lh / a.heads, h = lh % a.heads;
  const size_t row = ((size_t)l * a.n_seqs + e.seq) * a.heads + h;
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(blockIdx.z ? a.c.vc : a.c.kc) + (row * a.max_slots + e.at4) * kOcts;
  const uint8_t* scales = (blockIdx.z ? a.c.vs : a.c.ks) + (row * a.max_slots + e.at4) * (HD / 32);
  T* out = reinterpret_cast<T*>(const_cast<void*>(blockIdx.z ? a.v : a.k)) + (row * a.slots + e.at) * HD;
  const int n = e.n * kOcts, u0 = (blockIdx.x - a.first_wg[ei]) * (256 * kLoadTurns) + threadIdx.x;
  uint32_t c[kLoadTurns], s[kLoadTurns];
#pragma unroll
  for (int j = 0; j < kLoadTurns; ++j) {
    const int u = u0 + j * 256;
    if (u < n) c[j] = codes[u], s[j] = scales[u / 4];
  }
#pragma unroll
  for (int j = 0; j < kLoadTurns; ++j) {
    const int u = u0 + j * 256;
    if (u >= n) continue;
    const u32x4 b = decode(c[j], s[j]);
    u32x4* to = reinterpret_cast<u32x4*>(out + (size_t)u * 8);
    if constexpr (sizeof(T) == 2) {
      __builtin_nontemporal_store(b, to);
    } else {
      __builtin_nontemporal_store(u32x4{b[0] << 16, b[0] & 0xFFFF0000u, b[1] << 16, b[1] & 0xFFFF0000u}, to);
      __builtin_nontemporal_store(u32x4{b[2] << 16, b[2] & 0xFFFF0000u, b[3] << 16, b[3] & 0xFFFF0000u}, to + 1);
    }
  }
}

// wgs(entry): workgroups of an entry, per (layer, KV head) and of K or V
template <class Wgs, class Kernel>
static void launch_moves(KvqMoveArgs a, int n_layers, const Wgs& wgs, Kernel kernel, hipStream_t st) {
  int n = 0;
  for (int i = 0; i < kMaxCols; ++i) {
    a.first_wg[i] = INT32_MAX;
    if (i >= a.n_entries) continue;
    a.first_wg[i] = n;
    n += wgs(a.entry[i]);
  }
  if (n == 0) return;
  const int all = n_layers * a.heads;
  for (a.lh0 = 0; a.lh0 < all; a.lh0 += 65535)
    hipLaunchKernelGGL(kernel, dim3(n, std::min(65535, all - a.lh0), 2), dim3(256), 0, st, a);
}

void launch_kvq_store(const KvqMoveArgs& a, int n_layers, int dtype, int hd, hipStream_t st) {
  const auto wgs = [](const KvqMoveEntry& e) { return (e.at4 + e.n - 1) / kKvqBlock - e.at4 / kKvqBlock + 1; };
  DISPATCH_T(dtype, {
    if (hd == 128) launch_moves(a, n_layers, wgs, kvq_store_kernel<T, 128>, st);
    else launch_moves(a, n_layers, wgs, kvq_store_kernel<T, 64>, st);
  });
}

void launch_kvq_load(const KvqMoveArgs& a, int n_layers, int dtype, int hd, hipStream_t st) {
  const auto wgs = [hd](const KvqMoveEntry& e) { return (e.n * (hd / 8) + 256 * kLoadTurns - 1) / (256 * kLoadTurns); };
  DISPATCH_T(dtype, {
    if (hd == 128) launch_moves(a, n_layers, wgs, kvq_load_kernel<T, 128>, st);
    else launch_moves(a, n_layers, wgs, kvq_load_kernel<T, 64>, st);
  });
}

}  // namespace es
