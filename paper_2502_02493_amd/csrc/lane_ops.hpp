// Reductions across the lanes of a wavefront and across the waves of a workgroup, for the kernels whose chain of dependent
// steps is what they cost (acceptance, selection over beams).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace es {

// Reductions over 8, 16, 32 or 64 neighbouring lanes (n, uniform) by operand swizzles, every lane receiving the result; a shuffle
// through LDS per step would stand in the chain that these kernels are.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ uint64_t dpp(uint64_t u) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, true);
  return (uint64_t)lo | ((uint64_t)hi << 32);
}
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  return __builtin_bit_cast(double, dpp<CTRL>(__builtin_bit_cast(uint64_t, v)));
}
// f of the values of lanes l and l ^ 16 (l ^ 32)
template <bool HALF, class F>
__device__ __forceinline__ float across(float v, const F& f) {
  const uint32_t a = __builtin_bit_cast(uint32_t, v);
  const auto s = HALF ? __builtin_amdgcn_permlane32_swap(a, a, false, false) : __builtin_amdgcn_permlane16_swap(a, a, false, false);
  return f(__builtin_bit_cast(float, (uint32_t)s[0]), __builtin_bit_cast(float, (uint32_t)s[1]));
}
template <bool HALF, class F>
__device__ __forceinline__ uint64_t across(uint64_t u, const F& f) {
  const uint32_t lo = (uint32_t)u, hi = (uint32_t)(u >> 32);
  const auto l = HALF ? __builtin_amdgcn_permlane32_swap(lo, lo, false, false) : __builtin_amdgcn_permlane16_swap(lo, lo, false, false);
  const auto h = HALF ? __builtin_amdgcn_permlane32_swap(hi, hi, false, false) : __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
  return f((uint64_t)l[0] | ((uint64_t)h[0] << 32), (uint64_t)l[1] | ((uint64_t)h[1] << 32));
}
template <bool HALF, class F>
__device__ __forceinline__ double across(double v, const F& f) {
  const auto g = [&](uint64_t a, uint64_t b) { return __builtin_bit_cast(uint64_t, f(__builtin_bit_cast(double, a), __builtin_bit_cast(double, b))); };
  return __builtin_bit_cast(double, across<HALF>(__builtin_bit_cast(uint64_t, v), g));
}
template <typename V, class F>
__device__ __forceinline__ V lanes_fold(V v, int n, const F& f) {
  v = f(v, dpp<0xB1>(v));   // quad_perm [1,0,3,2]
  v = f(v, dpp<0x4E>(v));   // quad_perm [2,3,0,1]
  v = f(v, dpp<0x141>(v));  // row_half_mirror
  if (n >= 16) v = f(v, dpp<0x140>(v));  // row_mirror
  if (n >= 32) v = across<false>(v, f);
  if (n >= 64) v = across<true>(v, f);
  return v;
}
template <typename V>
__device__ __forceinline__ V lanes_sum(V v, int n) {
  return lanes_fold(v, n, [](V a, V b) { return a + b; });
}
__device__ __forceinline__ float lanes_max(float v, int n) {
  return lanes_fold(v, n, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float quad_max(float v) {  // of four neighbouring lanes
  v = fmaxf(v, dpp<0xB1>(v));
  return fmaxf(v, dpp<0x4E>(v));
}

// Running sum over the wave's lanes, the own one included.
__device__ __forceinline__ uint32_t lanes_running_sum(uint32_t v) {
  const auto moved = [](uint32_t x, auto ctrl, auto rows) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, decltype(rows)::value, 0xF, false); };
  typedef std::integral_constant<int, 0xF> All;
  v += moved(v, std::integral_constant<int, 0x111>{}, All{});  // row_shr by 1, 2, 4, 8: zeros come in
  v += moved(v, std::integral_constant<int, 0x112>{}, All{});
  v += moved(v, std::integral_constant<int, 0x114>{}, All{});
  v += moved(v, std::integral_constant<int, 0x118>{}, All{});
  v += moved(v, std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xA>{});  // row_bcast15: the rows' ends to the second and fourth
  v += moved(v, std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xC>{});  // row_bcast31: the second's to the upper two
  return v;
}

// The lowest of the wave's values, which are the same in every lane of each group of n (4, 8, 16, 32 or 64) neighbours.
__device__ __forceinline__ float groups_min(float v, int n) {
  const auto f = [](float a, float b) { return fminf(a, b); };
  if (n <= 4) v = f(v, dpp<0x141>(v));  // row_half_mirror
  if (n <= 8) v = f(v, dpp<0x140>(v));  // row_mirror
  if (n <= 16) v = across<false>(v, f);
  if (n <= 32) v = across<true>(v, f);
  return v;
}

// Over the workgroup of NW waves: the waves' results in order, the same bits in every thread.
template <int NW>
__device__ __forceinline__ double block_sum(double v, double* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = lanes_sum(v, 64);
  __syncthreads();  // sh may still be read from the previous call
  if (lane == 0) sh[wave] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < NW; ++w) t += sh[w];
  return t;
}
template <int NW>
__device__ __forceinline__ float block_max(float v, float* sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = lanes_max(v, 64);
  if (lane == 0) sh[wave] = v;
  __syncthreads();
  float t = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) t = fmaxf(t, sh[w]);
  return t;
}

// the value of one lane, for every lane
__device__ __forceinline__ double lane_value(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)lo | ((uint64_t)hi << 32));
}

}  // namespace es
