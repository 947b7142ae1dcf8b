// lanes.h -- a wave's lanes together, by exchanges that need no LDS.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace grid {

// f of the values of all lanes that share `lane / N` (N: 1 .. 64, a power of two, the same for the whole wave), in each
// of them.  f is associative and commutative.
template <typename F>
__device__ inline uint32_t across(uint32_t x, F f, int N = 64) {
  if (N > 1) x = f(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));   // lane ^ 1
  if (N > 2) x = f(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));   // lane ^ 2
  if (N > 4) x = f(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xF, 0xF, true));  // 7 - lane, of 8
  if (N > 8) x = f(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x140, 0xF, 0xF, true));  // 15 - lane, of 16
  if (N > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = f(r[0], r[1]);
  }
  if (N > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = f(r[0], r[1]);
  }
  return x;
}
__device__ inline float max_across(float x, int N = 64) {
  return __uint_as_float(across(
      __float_as_uint(x),
      [](uint32_t p, uint32_t q) { return __float_as_uint(fmaxf(__uint_as_float(p), __uint_as_float(q))); }, N));
}
__device__ inline float sum_across(float x, int N = 64) {
  return __uint_as_float(across(
      __float_as_uint(x), [](uint32_t p, uint32_t q) { return __float_as_uint(__uint_as_float(p) + __uint_as_float(q)); },
      N));
}
__device__ inline int min_across(int x, int N = 64) {
  return (int)across((uint32_t)x, [](uint32_t p, uint32_t q) { return (uint32_t)min((int)p, (int)q); }, N);
}

}  // namespace grid
