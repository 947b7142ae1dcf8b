// verify.hip -- grid_verify: drafted tokens against the target's masked distribution (gfx950).
//
// Two launches.  The first reads every row once, in slices, and leaves per slice the largest allowed logit m and
// z = sum exp((l - m) / T), taken online.  The second joins a sequence's rows, finds the first refused draft and races
// that one row's weights over the given noise: the argmax of w / noise needs no normaliser and no order, so the row is
// split over workgroups whose best meet in an integer maximum (score bits, then the complement of the index: the
// lowest index on ties, whatever the order).  The last workgroup of a sequence writes its outputs.
#include <algorithm>
#include <string>

#include "paged.h"

using namespace grid;

namespace {

constexpr int kThreads = 256;
constexpr int kStep = kThreads * 8;  // tokens a workgroup takes a step: 8 a thread, one byte of mask
constexpr int kMaxSlices = 64;       // of a row: a wave joins them
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLow = -3.402823466e38f;

struct VerifyArgs {
  const void* logits;
  const uint32_t* mask;
  const int32_t *draft, *draft_len;
  const float *probs, *uniform, *noise, *temperature;
  int64_t ls[2], ms[2], ps[2], ns;
  int32_t *tokens, *accepted;
  float* logprobs;
  float4* part;   // [rows][slices]: m, z, index of m
  uint64_t* best; // [B][2]: the residual's race, p's own
  uint32_t* done; // [B]: workgroups that have raced
  int32_t B, K, V, slices, slice, races, race;
};

// Sequence b's factor of the exponent (log2 e / T) and whether it is greedy.  The factor stays finite and above 0, so
// that 0 * factor is 0 and -inf * factor is -inf.
__device__ inline float factor_of(const VerifyArgs& a, int b, bool& greedy) {
  const float t = a.temperature ? a.temperature[b] : 1.f;
  greedy = !a.noise || !(t > 0.f);
  return greedy ? kLog2e : fminf(fmaxf(kLog2e / t, 1e-30f), 1e38f);
}

__device__ inline int drafted(const VerifyArgs& a, int b) {
  return a.draft_len ? min(max(a.draft_len[b], 0), a.K) : a.K;
}

template <typename T>
struct Raw {
  T x[8];
};

// Rows of odd vocabularies start anywhere: 16-byte loads from any address that fits the type.
template <typename T>
__device__ inline void load8(const T* p, float (&x)[8]) {
  Raw<T> r;
  __builtin_memcpy(&r, p, sizeof(r));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)r.x[i];
}

// 8 entries from token t on; those at or after V read as `other`.
template <typename T>
__device__ inline void load8_end(const T* row, int t, int V, float other, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = t + i < V ? (float)row[t + i] : other;
}

// mask bits of tokens t .. t + 7 (t a multiple of 8, t < V); bits at or after V are not trusted
__device__ inline uint32_t bits8(const uint32_t* mask, int t, int V) {
  uint32_t m = mask ? ((const uint8_t*)mask)[t >> 3] : 0xFFu;
  if (t + 8 > V) m &= (1u << (V - t)) - 1u;
  return m;
}

struct Online {
  float m, z;
  int idx;
  __device__ static Online empty() { return {kLow, 0.f, 0x7FFFFFFF}; }
  __device__ void take(const float (&x)[8], uint32_t bits, int t, float c, bool greedy) {
    float v[8], top = kLow;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = bits >> i & 1 ? x[i] : -INFINITY;
      top = fmaxf(top, v[i]);
    }
    if (top > m || (idx == 0x7FFFFFFF && greedy)) {
      if (greedy) {
#pragma unroll
        for (int i = 7; i >= 0; --i)
          if (v[i] == top) idx = t + i;
      }
      z *= __builtin_amdgcn_exp2f((m - top) * c);
      m = top;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) z += __builtin_amdgcn_exp2f((v[i] - m) * c);
  }
  __device__ void join(float om, float oz, int oi, float c) {
    const float top = fmaxf(m, om);
    z = z * __builtin_amdgcn_exp2f((m - top) * c) + oz * __builtin_amdgcn_exp2f((om - top) * c);
    idx = om > m ? oi : om == m ? min(idx, oi) : idx;
    m = top;
  }
  __device__ void across(float c) {
    for (int o = 32; o > 0; o >>= 1) {
      const float om = __shfl_xor(m, o), oz = __shfl_xor(z, o);
      const int oi = __shfl_xor(idx, o);
      join(om, oz, oi, c);
    }
  }
};

template <typename T>
__global__ __launch_bounds__(kThreads) void stats_kernel(VerifyArgs a) {
  const int tid = (int)threadIdx.x, slice = (int)blockIdx.x % a.slices, r = (int)blockIdx.x / a.slices;
  const int b = r / (a.K + 1), j = r - b * (a.K + 1);
  if (j == 0 && slice == 0 && tid == 0) {
    a.best[2 * b] = a.best[2 * b + 1] = 0;
    a.done[b] = 0;
  }
  if (j > drafted(a, b)) return;
  bool greedy;
  const float c = factor_of(a, b, greedy);
  const T* row = (const T*)a.logits + b * a.ls[0] + j * a.ls[1];
  const uint32_t* mask = a.mask ? a.mask + b * a.ms[0] + j * a.ms[1] : nullptr;
  const int end = min(a.V, (slice + 1) * a.slice);
  Online o = Online::empty();
  for (int t = slice * a.slice + tid * 8; t < end; t += kStep) {
    float x[8];
    if (t + 8 <= a.V)
      load8(row + t, x);
    else
      load8_end(row, t, a.V, -INFINITY, x);
    o.take(x, bits8(mask, t, a.V), t, c, greedy);
  }
  o.across(c);
  __shared__ Online wave[kThreads / 64];
  if ((tid & 63) == 0) wave[tid >> 6] = o;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kThreads / 64; ++w) o.join(wave[w].m, wave[w].z, wave[w].idx, c);
    a.part[(int64_t)r * a.slices + slice] = make_float4(o.m, o.z, __int_as_float(o.idx), 0.f);
  }
}

__device__ inline uint64_t race_key(float score, int t) {
  return score > 0.f ? (uint64_t)__float_as_uint(score) << 32 | (uint32_t)~t : 0;
}

__device__ inline uint64_t max_across(uint64_t k) {
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t x = __shfl_xor((unsigned long long)k, o);
    k = x > k ? x : k;
  }
  return k;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void pick_kernel(VerifyArgs a) {
  const int tid = (int)threadIdx.x, lane = tid & 63, part = (int)blockIdx.x % a.races, b = (int)blockIdx.x / a.races;
  bool greedy;
  const float c = factor_of(a, b, greedy);
  if (greedy && part > 0) return;
  const int n = drafted(a, b);
  const T* rows = (const T*)a.logits + b * a.ls[0];
  const uint32_t* masks = a.mask ? a.mask + b * a.ms[0] : nullptr;
  __shared__ Online row[64];
  __shared__ int first;
  __shared__ uint64_t wave_best[2][kThreads / 64];
  for (int j = tid >> 6; j <= n; j += kThreads / 64) {
    Online o = Online::empty();
    if (lane < a.slices) {
      const float4 p = a.part[((int64_t)b * (a.K + 1) + j) * a.slices + lane];
      o.m = p.x;
      o.z = p.y;
      o.idx = __float_as_int(p.z);
    }
    o.across(c);
    if (lane == 0) row[j] = o;
  }
  __syncthreads();
  // weight of token t in row j, 0 where it is not allowed
  auto weight = [&](int j, int t) {
    if ((uint32_t)t >= (uint32_t)a.V || (masks && !(masks[j * a.ms[1] + (t >> 5)] >> (t & 31) & 1))) return 0.f;
    return __builtin_amdgcn_exp2f(((float)rows[j * a.ls[1] + t] - row[j].m) * c);
  };
  if (tid < 64) {
    bool ok = false;
    if (tid < n) {
      const int x = a.draft[(int64_t)b * a.K + tid];
      const float z = row[tid].z;
      if (z > 0.f && (uint32_t)x < (uint32_t)a.V) {
        if (greedy) {
          ok = x == row[tid].idx;
        } else {
          const float q = a.probs ? a.probs[b * a.ps[0] + tid * a.ps[1] + x] : 1.f;
          ok = a.uniform[(int64_t)b * a.K + tid] * q < weight(tid, x) / z;
        }
      }
    }
    const uint64_t refused = __ballot(!ok);  // lane n refuses (n <= 63)
    if (tid == 0) first = __builtin_ctzll(refused);
  }
  __syncthreads();
  const int at = first;
  const Online o = row[at];
  const bool alive = o.z > 0.f;  // not for NaN
  int token = -1;
  if (greedy) {
    if (alive) token = o.idx;
  } else {
    // the race over this workgroup's part of row `at`
    const int x = at < n ? a.draft[(int64_t)b * a.K + at] : -1;
    const float* q = at < n && a.probs ? a.probs + b * a.ps[0] + at * a.ps[1] : nullptr;
    const T* lrow = rows + at * a.ls[1];
    const uint32_t* mask = masks ? masks + at * a.ms[1] : nullptr;
    const float* noise = a.noise + b * a.ns;
    const float over = 1.f / o.z;
    uint64_t left = 0, whole = 0;
    const int end = alive ? min(a.V, (part + 1) * a.race) : 0;
    for (int t = part * a.race + tid * 8; t < end; t += kStep) {
      float l[8], e[8], d[8];
      if (t + 8 <= a.V) {
        load8(lrow + t, l);
        load8(noise + t, e);
        if (q) load8(q + t, d);
      } else {
        load8_end(lrow, t, a.V, -INFINITY, l);
        load8_end(noise, t, a.V, 1.f, e);
        if (q) load8_end(q, t, a.V, 0.f, d);
      }
      const uint32_t bits = bits8(mask, t, a.V);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = bits >> i & 1 ? __builtin_amdgcn_exp2f((l[i] - o.m) * c) * over : 0.f;
        const float rate = __builtin_amdgcn_rcpf(e[i]);
        const float rest = q ? fmaxf(p - d[i], 0.f) : t + i == x ? 0.f : p;
        left = max(left, race_key(rest * rate, t + i));
        whole = max(whole, race_key(p * rate, t + i));
      }
    }
    left = max_across(left);
    whole = max_across(whole);
    if (lane == 0) {
      wave_best[0][tid >> 6] = left;
      wave_best[1][tid >> 6] = whole;
    }
    __syncthreads();
    __shared__ bool last;
    if (tid == 0) {
      for (int w = 1; w < kThreads / 64; ++w) {
        left = max(left, wave_best[0][w]);
        whole = max(whole, wave_best[1][w]);
      }
      unsigned long long* best = (unsigned long long*)(a.best + 2 * b);
      __hip_atomic_fetch_max(best, left, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_fetch_max(best + 1, whole, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      last = __hip_atomic_fetch_add(a.done + b, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.races - 1;
      if (last) {
        left = __hip_atomic_load(best, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        whole = __hip_atomic_load(best + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        wave_best[0][0] = left ? left : whole;
      }
    }
    __syncthreads();
    if (!last) return;
    const uint64_t key = wave_best[0][0];
    if (key) token = (int)~(uint32_t)key;
  }
  if (tid <= a.K) {
    const int mine = tid < at ? a.draft[(int64_t)b * a.K + tid] : tid == at ? token : -1;
    float lp = 0.f;
    if (mine >= 0) lp = ((float)rows[tid * a.ls[1] + mine] - row[tid].m) * (c / kLog2e) - logf(row[tid].z);
    a.tokens[(int64_t)b * (a.K + 1) + tid] = mine;
    a.logprobs[(int64_t)b * (a.K + 1) + tid] = lp;
  }
  if (tid == 0) a.accepted[b] = at;
}

// How many pieces `units` rows of V tokens are cut into, and their tokens: about 2048 workgroups in all, none of less
// than two steps, so that short batches fill the chip and long ones are not cut at all.
void pieces(int64_t units, int V, int most, int32_t& n, int32_t& len) {
  const int64_t want = std::max<int64_t>(1, (2048 + units - 1) / units);
  const int fit = std::max(1, (V + 2 * kStep - 1) / (2 * kStep));
  n = (int32_t)std::min<int64_t>({want, fit, most});
  len = (int32_t)((((int64_t)V + n - 1) / n + kStep - 1) / kStep * kStep);
  n = (int32_t)(((int64_t)V + len - 1) / len);
}

bool sizes_ok(int32_t B, int32_t K, int32_t V) {
  return B >= 1 && B <= 65535 && K >= 0 && K <= 63 && V >= 1 && V <= INT32_MAX - 2 * kStep;
}

size_t head_bytes(int32_t B) { return ((size_t)B * 20 + 255) / 256 * 256; }

}  // namespace

extern "C" size_t grid_verify_workspace_bytes(int32_t B, int32_t K, int32_t V) {
  if (!sizes_ok(B, K, V)) return 0;
  int32_t n, len;
  pieces((int64_t)B * (K + 1), V, kMaxSlices, n, len);
  return head_bytes(B) + (size_t)B * (size_t)(K + 1) * (size_t)n * sizeof(float4);
}

extern "C" int grid_verify(const grid_verify_args* args, void* stream) {
  clear_error();
  auto bad = [](const char* what) { return fail(GRID_E_ARG, std::string("grid_verify: ") + what); };
  if (!args) return bad("null argument");
  const grid_verify_args& g = *args;
  if (!sizes_ok(g.B, g.K, g.V)) return bad("sizes");
  if (g.dtype != GRID_DTYPE_F32 && g.dtype != GRID_DTYPE_BF16 && g.dtype != GRID_DTYPE_F16) return bad("dtype");
  if (!g.logits || !g.tokens || !g.accepted || !g.logprobs || !g.workspace) return bad("null pointer");
  if (g.K > 0 && !g.draft) return bad("no drafts");
  if (!g.noise != !g.uniform && (g.K > 0 || g.uniform)) return bad("uniform and noise come together");
  if (g.draft_probs && !g.noise) return bad("draft_probs without random numbers");
  if (g.logits_stride[0] < 0 || g.logits_stride[1] < 0 || g.mask_stride[0] < 0 || g.mask_stride[1] < 0 ||
      g.probs_stride[0] < 0 || g.probs_stride[1] < 0 || g.noise_stride < 0)
    return bad("negative stride");
  const size_t need = grid_verify_workspace_bytes(g.B, g.K, g.V);
  if ((uintptr_t)g.workspace % 16 != 0 || g.workspace_bytes < need) return bad("workspace too small or not aligned");
  VerifyArgs a;
  a.logits = g.logits;
  a.mask = g.mask;
  a.draft = g.draft;
  a.draft_len = g.draft_len;
  a.probs = g.draft_probs;
  a.uniform = g.uniform;
  a.noise = g.noise;
  a.temperature = g.temperature;
  for (int i = 0; i < 2; ++i) {
    a.ls[i] = g.logits_stride[i];
    a.ms[i] = g.mask_stride[i];
    a.ps[i] = g.probs_stride[i];
  }
  a.ns = g.noise_stride;
  a.tokens = g.tokens;
  a.accepted = g.accepted;
  a.logprobs = g.logprobs;
  a.best = (uint64_t*)g.workspace;
  a.done = (uint32_t*)(a.best + 2 * (size_t)g.B);
  a.part = (float4*)((uint8_t*)g.workspace + head_bytes(g.B));
  a.B = g.B;
  a.K = g.K;
  a.V = g.V;
  const int64_t rows = (int64_t)g.B * (g.K + 1);
  pieces(rows, g.V, kMaxSlices, a.slices, a.slice);
  pieces(g.B, g.V, 1 << 20, a.races, a.race);
  if (!g.noise) a.races = 1;
  hipStream_t s = (hipStream_t)stream;
  const dim3 one((unsigned)(rows * a.slices)), two((unsigned)((int64_t)g.B * a.races));
  auto launch = [&](auto type) {
    using T = decltype(type);
    hipLaunchKernelGGL(stats_kernel<T>, one, dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(pick_kernel<T>, two, dim3(kThreads), 0, s, a);
  };
  if (g.dtype == GRID_DTYPE_F32)
    launch(float());
  else if (g.dtype == GRID_DTYPE_BF16)
    launch(__bf16());
  else
    launch(_Float16());
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_verify launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
