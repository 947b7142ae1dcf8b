// sample.hip -- grid_sample: one token of every row from its masked and filtered distribution (gfx950).
//
// A workgroup takes a row.  It goes over it for the maximum, then, where a filter cuts, finds the last kept token in the
// order of the logits by digits of their keys, from the highest on: a histogram of the digit over what is left, and the bin
// in which the count reaches top_k, or the mass top_p.  Of equal logits at the cut the lower indexes are kept, found the same
// way by digits of the index.  The last pass races w / noise over what is kept.
//
// Masses are whole numbers, w times a power of two: their sums do not depend on the order of the atomics.
#include <algorithm>
#include <string>
#include <type_traits>

#include "lanes.h"
#include "paged.h"

using namespace grid;

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kNone = 0x7FFFFFFF;

struct SampleArgs {
  const void* logits;
  const uint32_t* mask;
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *noise;
  int64_t ls, ms, ns;
  int32_t* tokens;
  float* logprobs;
  int32_t V, shift;  // shift: a mass is w * 2^shift, so that V of them fit 63 bits
};

// Logits in their order, as whole numbers; -0 is 0.
__device__ inline uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float value_of(uint32_t key) {
  return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xFFFFFFFFu));
}

__device__ inline uint64_t best_across(uint64_t k) {
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t x = __shfl_xor((unsigned long long)k, o);
    k = x > k ? x : k;
  }
  return k;
}

struct Shared {
  uint64_t mass[256];
  uint32_t count[256];
  float f[2][kWaves];
  uint64_t best[kWaves];
  uint64_t above_mass;
  uint32_t above, bin;
};

// What of a row is kept: keys above `key`, and of equal ones the indexes up to `index`.
struct Cut {
  uint32_t key;
  int index;
  uint64_t mass;  // of what is kept
};

template <typename T>
struct Rows {
  const SampleArgs& a;
  Shared& sh;
  const T* row;
  const uint8_t* mask;
  float m, c;

  // f(logit, token) of every allowed token
  template <typename F>
  __device__ void each(F f) const {
    for (int t = (int)threadIdx.x * 8; t < a.V; t += kThreads * 8) {
      uint32_t bits = mask ? mask[t >> 3] : 0xFFu;
      if (a.V - t < 8) bits &= (1u << (a.V - t)) - 1u;
      for (int i = 0; i < 8; ++i)
        if (bits >> i & 1) f((float)row[t + i], t + i);
    }
  }
  __device__ float weight(float l) const { return __builtin_amdgcn_exp2f((l - m) * c); }
  __device__ uint64_t mass(float l) const { return (uint64_t)__builtin_ldexpf(weight(l), a.shift); }

  // The bin in which the counts (or masses) from the highest bin on (the lowest: !down) reach the target; it is taken out of
  // the target what the bins before hold.
  __device__ uint32_t reached(uint64_t& target, bool by_mass, bool down) {
    __syncthreads();
    if (threadIdx.x < 64) {
      const int lane = (int)threadIdx.x;
      uint64_t v[4], mine = 0;
      for (int i = 0; i < 4; ++i) {
        const int at = down ? 255 - (lane * 4 + i) : lane * 4 + i;
        v[i] = by_mass ? sh.mass[at] : sh.count[at];
        mine += v[i];
      }
      uint64_t upto = mine;
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t x = __shfl_up((unsigned long long)upto, o);
        if (lane >= o) upto += x;
      }
      const uint64_t hit = __ballot(upto >= target);
      if (hit == 0 ? lane == 63 : lane == __builtin_ctzll(hit)) {
        uint64_t before = upto - mine;
        int i = 0;
        while (i < 3 && before + v[i] < target) before += v[i++];
        sh.bin = (uint32_t)(down ? 255 - (lane * 4 + i) : lane * 4 + i);
        sh.above_mass = before;
      }
    }
    __syncthreads();
    const uint32_t bin = sh.bin;
    target -= sh.above_mass;
    __syncthreads();
    return bin;
  }
  __device__ void clear() {
    __syncthreads();
    for (int i = (int)threadIdx.x; i < 256; i += kThreads) sh.mass[i] = 0, sh.count[i] = 0;
    __syncthreads();
  }

  // The cut at which the count (or the mass) of the tokens in order reaches `target`, 1 or more and no more than there is.
  __device__ Cut cut(uint64_t target, bool by_mass, const Cut& within) {
    uint32_t key = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      clear();
      each([&](float l, int t) {
        const uint32_t k = key_of(l);
        if (k < within.key || (k == within.key && t > within.index)) return;
        if (shift < 24 && k >> (shift + 8) != key >> (shift + 8)) return;
        if (by_mass)
          atomicAdd((unsigned long long*)&sh.mass[k >> shift & 255], (unsigned long long)mass(l));
        else
          atomicAdd(&sh.count[k >> shift & 255], 1u);
      });
      key |= reached(target, by_mass, true) << shift;
    }
    // of the equal ones as many as reach it, the lower indexes first
    const uint64_t unit = by_mass ? max((uint64_t)1, mass(value_of(key))) : 1;
    uint64_t ties = (target + unit - 1) / unit;
    uint32_t index = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (shift > 0 && a.V >> shift == 0) continue;
      clear();
      each([&](float l, int t) {
        if (key_of(l) != key || (key == within.key && t > within.index)) return;
        if (shift < 24 && (uint32_t)t >> (shift + 8) != index >> (shift + 8)) return;
        atomicAdd(&sh.count[t >> shift & 255], 1u);
      });
      index |= reached(ties, false, false) << shift;
    }
    return {key, (int)index, 0};
  }
};

__device__ inline float block_max(Shared& sh, float x) {
  x = max_across(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.f[0][threadIdx.x >> 6] = x;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) x = fmaxf(x, sh.f[0][w]);
  return x;
}
__device__ inline float block_sum(Shared& sh, float x) {
  x = sum_across(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.f[1][threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.f;
  for (int w = 0; w < kWaves; ++w) x += sh.f[1][w];
  return x;
}
__device__ inline uint64_t block_best(Shared& sh, uint64_t x) {
  x = best_across(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = x;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) x = max(x, sh.best[w]);
  return x;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int64_t b = blockIdx.x;
  const float t = a.temperature ? a.temperature[b] : 1.f;
  const bool greedy = !a.noise || !(t > 0.f);
  Rows<T> r = {a, sh, (const T*)a.logits + b * a.ls, a.mask ? (const uint8_t*)(a.mask + b * a.ms) : nullptr, 0.f,
               greedy ? kLog2e : fminf(fmaxf(kLog2e / t, 1e-30f), 1e38f)};
  float m = -INFINITY;
  bool broken = false;
  r.each([&](float l, int) {
    m = fmaxf(m, l);
    broken |= !(l < INFINITY);
  });
  m = block_max(sh, m);
  if (__syncthreads_or(broken) || !(m > -INFINITY)) {
    if (threadIdx.x == 0) a.tokens[b] = -1, a.logprobs[b] = 0.f;
    return;
  }
  r.m = m;
  Cut kept = {0, kNone, 0};
  float low = 0.f;  // the smallest weight that is kept
  if (!greedy) {
    const int k = a.top_k ? a.top_k[b] : 0;
    const float p = a.top_p ? a.top_p[b] : 1.f, q = a.min_p ? a.min_p[b] : 0.f;
    low = q > 0.f ? fminf(q, 1.f) : 0.f;
    if (k > 0 && k < a.V) kept = r.cut((uint64_t)k, false, kept);
    if (p < 1.f) {
      r.clear();
      uint64_t mine = 0;
      r.each([&](float l, int t) {
        const uint32_t key = key_of(l);
        if (key > kept.key || (key == kept.key && t <= kept.index)) mine += r.mass(l);
      });
      if (mine) atomicAdd((unsigned long long*)&sh.mass[0], (unsigned long long)mine);
      __syncthreads();
      const uint64_t all = sh.mass[0];
      const double want = __builtin_ceil((double)fmaxf(p, 0.f) * (double)all);
      kept = r.cut(min(max((uint64_t)want, (uint64_t)1), all), true, kept);
    }
  }
  float z = 0.f;
  uint64_t best = 0;
  const float* noise = a.noise ? a.noise + b * a.ns : nullptr;
  r.each([&](float l, int t) {
    const uint32_t key = key_of(l);
    const float w = r.weight(l);
    if (key < kept.key || (key == kept.key && t > kept.index) || w < low) return;
    z += w;
    const float score = greedy ? (l == m ? 1.f : 0.f) : w * __builtin_amdgcn_rcpf(noise[t]);
    if (score > 0.f) best = max(best, (uint64_t)__float_as_uint(score) << 32 | (uint32_t)~t);
  });
  z = block_sum(sh, z);
  best = block_best(sh, best);
  if (threadIdx.x == 0) {
    const int token = best ? (int)~(uint32_t)best : -1;
    a.tokens[b] = token;
    a.logprobs[b] = token < 0 ? 0.f : ((float)r.row[token] - m) * (r.c / kLog2e) - logf(z);
  }
}

}  // namespace

extern "C" int grid_sample(const grid_sample_args* args, void* stream) {
  clear_error();
  auto bad = [](const char* what) { return fail(GRID_E_ARG, std::string("grid_sample: ") + what); };
  if (!args) return bad("null argument");
  const grid_sample_args& g = *args;
  if (g.B < 1 || g.B > 1 << 20 || g.V < 1 || g.V > (1 << 30) - 2048) return bad("sizes");
  if (g.dtype != GRID_DTYPE_F32 && g.dtype != GRID_DTYPE_BF16 && g.dtype != GRID_DTYPE_F16) return bad("dtype");
  if (!g.logits || !g.tokens || !g.logprobs) return bad("null pointer");
  if (g.logits_stride < 0 || g.mask_stride < 0 || g.noise_stride < 0) return bad("negative stride");
  SampleArgs a;
  a.logits = g.logits;
  a.mask = g.mask;
  a.temperature = g.temperature;
  a.top_k = g.top_k;
  a.top_p = g.top_p;
  a.min_p = g.min_p;
  a.noise = g.noise;
  a.ls = g.logits_stride;
  a.ms = g.mask_stride;
  a.ns = g.noise_stride;
  a.tokens = g.tokens;
  a.logprobs = g.logprobs;
  a.V = g.V;
  a.shift = 40;
  while (a.shift > 0 && (uint64_t)g.V > (uint64_t)1 << (62 - a.shift)) --a.shift;
  const auto go = [&](auto type) {
    using T = decltype(type);
    hipLaunchKernelGGL(sample_kernel<T>, dim3((unsigned)g.B), dim3(kThreads), 0, (hipStream_t)stream, a);
  };
  if (g.dtype == GRID_DTYPE_F32)
    go(float());
  else if (g.dtype == GRID_DTYPE_BF16)
    go(bf16_t());
  else
    go(f16_t());
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_sample launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
