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


// The same for 64 bits, over all lanes of a wave.
template <typename F>
__device__ inline uint64_t across64(uint64_t x, F f) {
  const auto both = [](uint32_t hi, uint32_t lo) { return (uint64_t)hi << 32 | lo; };
  uint32_t lo, hi;
#define GRID_STEP(ctrl)                                                                           \
  lo = (uint32_t)x, hi = (uint32_t)(x >> 32);                                                     \
  x = f(x, both((uint32_t)__builtin_amdgcn_mov_dpp((int)hi, ctrl, 0xF, 0xF, true),                \
                (uint32_t)__builtin_amdgcn_mov_dpp((int)lo, ctrl, 0xF, 0xF, true)));
  GRID_STEP(0xB1)
  GRID_STEP(0x4E)
  GRID_STEP(0x141)
  GRID_STEP(0x140)
#undef GRID_STEP
  lo = (uint32_t)x, hi = (uint32_t)(x >> 32);
  auto l = __builtin_amdgcn_permlane16_swap(lo, lo, false, false), h = __builtin_amdgcn_permlane16_swap(hi, hi, false, false);
  x = f(both(h[0], l[0]), both(h[1], l[1]));
  lo = (uint32_t)x, hi = (uint32_t)(x >> 32);
  l = __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
  h = __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
  return f(both(h[0], l[0]), both(h[1], l[1]));
}
__device__ inline uint64_t max_across(uint64_t x) {
  return across64(x, [](uint64_t p, uint64_t q) { return p > q ? p : q; });
}
__device__ inline uint64_t min_across(uint64_t x) {
  return across64(x, [](uint64_t p, uint64_t q) { return p < q ? p : q; });
}
__device__ inline uint64_t sum_across(uint64_t x) {
  return across64(x, [](uint64_t p, uint64_t q) { return p + q; });
}

// The sum over the lanes up to and with this one.
__device__ inline uint32_t sum_upto(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);  // from 1, 2, 4, 8 lanes down, in rows of 16
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);  // a row's last to the next, in rows 1 and 3
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);  // lane 31 to rows 2 and 3
  return x;
}
__device__ inline uint64_t sum_upto(uint64_t x) {
#define GRID_STEP(ctrl, rows)                                                                     \
  x += (uint64_t)(uint32_t)__builtin_amdgcn_update_dpp(0, (int)(x >> 32), ctrl, rows, 0xF, false) << 32 | \
       (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xF, false);
  GRID_STEP(0x111, 0xF)
  GRID_STEP(0x112, 0xF)
  GRID_STEP(0x114, 0xF)
  GRID_STEP(0x118, 0xF)
  GRID_STEP(0x142, 0xA)
  GRID_STEP(0x143, 0xC)
#undef GRID_STEP
  return x;
}

// A value of lane i, the same i in all lanes.
__device__ inline uint64_t lane_of(uint64_t x, int i) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, i);
}

}  // namespace grid
