// verify.hip -- grid_verify: drafted tokens against the target's masked distribution (gfx950).
//
// Two launches.  The first goes over the rows once: a workgroup takes a piece (some thousand tokens) of a row and leaves the
// largest allowed logit m, z = sum exp((l - m) / T), and the best of the race exp((l - m) / T) / noise: an argmax that needs
// no normaliser and no order.  Large batches have workgroups that take the piece of several rows of a sequence, one after
// the other, with the noise of these tokens in registers.  Logits are read only where the mask allows one of a thread's 8
// tokens.  The second joins a sequence's rows and finds the first refused draft.  Where
// drafts come without probabilities, what is left of p after a refusal is p without the draft, so the first pass has
// raced it already.  Otherwise max(p - q, 0) of that one row is raced by several workgroups, whose best meet in an integer
// maximum (score bits, then the complement of the index: the lowest index on ties, whatever the order); the last of them
// writes the sequence's outputs.
//
// Bound by latency more than by bytes: 32 sequences of up to 4 drafts, 151936 tokens in bf16, take 19.5 us (the first
// launch 16.3, the second 4.5) for 52 MB of rows, masks and noise, of which the masked part is not read; 64 of up to 7, 50257
// in float32, with the drafter's probabilities, 26.4 us (16.8 and 10.4, the race's atomics in turn among the latter).  The
// former have one row a workgroup, the latter one or two: every chain of lengths, mask, logits and join begins anew.
#include <algorithm>
#include <string>
#include <type_traits>

#include "lanes.h"
#include "paged.h"

using namespace grid;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
template <typename T>                    // steps of 512 tokens, 8 a lane, that a wave takes of a row: 16-bit rows have
constexpr int kSteps = 8 / sizeof(T);    // the longer ones, for the same registers
constexpr int kPiece = kWaves * 512;     // tokens of a workgroup's piece, for each step
constexpr int kStep = kThreads * 8;      // tokens that a workgroup of the residual's race takes a step
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLow = -3.402823466e38f;
constexpr int kNone = 0x7FFFFFFF;

struct VerifyArgs {
  const void* logits;
  const uint32_t* mask;
  const int32_t *draft, *draft_len;
  const float *probs, *uniform, *noise, *temperature;
  int64_t ls[2], ms[2], ps[2], ns;
  int32_t *tokens, *accepted;
  float* logprobs;
  float4* part;   // [B][K + 1][pieces]: m, z, best score (relative to m), its index (greedy: of m)
  uint64_t* best; // [B]: the residual's race
  uint32_t* done; // [B]: workgroups that have raced
  int32_t B, K, V, pieces, groups, races, race;
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

// 8 entries as they are in memory, in whole registers.
template <typename T>
struct Raw {
  static constexpr int N = sizeof(T) * 2;
  uint32_t w[N];
  __device__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    if constexpr (std::is_same<T, bf16_t>::value) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    return (float)__builtin_bit_cast(f16_t, (uint16_t)(w[i / 2] >> (i & 1) * 16));
  }
  // the first 8 entries, of which `have` exist (the others read as the last)
  __device__ void load_short(const T* row, int have) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      constexpr int E = 4 / sizeof(T);
      T e[E];
#pragma unroll
      for (int k = 0; k < E; ++k) e[k] = row[min(i * E + k, have - 1)];
      __builtin_memcpy(&w[i], e, 4);
    }
  }
};

// Rows of odd vocabularies start anywhere: 16-byte loads from any address that fits the type.
template <typename T>
__device__ inline void load8(const T* p, float (&x)[8]) {
  Raw<T> r;
  __builtin_memcpy(&r, p, sizeof(r));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = r.at(i);
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

// What is known of some of a row's tokens.  score: the largest w / noise, relative to m as w is; idx: its lowest index,
// or of a greedy row the lowest index of m.
struct Row {
  float m, z, score;
  int idx;
};

// The lanes' parts of a row as one, in every lane.
__device__ inline Row join_lanes(Row r, float c, bool greedy) {
  const float m = max_across(r.m), f = __builtin_amdgcn_exp2f((r.m - m) * c);
  const float s = r.score * f, best = max_across(s);
  const int idx = min_across((greedy ? r.m == m : s == best) ? r.idx : kNone);
  return {m, sum_across(r.z * f), best, idx};
}

// A workgroup takes a piece of the rows of one sequence that are in one group (one row, or several).
enum class Rows { kAll, kMasked, kShort };  // all tokens allowed, mask rows, fewer than 8 tokens (masked or not)

template <typename T, bool GREEDY, Rows ROWS>
__device__ __forceinline__ void scan(const VerifyArgs& a, Row (&wave_row)[2][kWaves], int b, int piece, int from, int to,
                                     int n, float c) {
  constexpr int S = kSteps<T>;
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const T* rows = (const T*)a.logits + b * a.ls[0];
  const uint32_t* masks = a.mask ? a.mask + b * a.ms[0] : nullptr;
  // (scalar loads, which do not wait for those of the rows)
  const auto* drafts = (const __attribute__((address_space(4))) int32_t*)(a.draft + (int64_t)b * a.K);
  const int t0 = (piece * kWaves + wave) * S * 512 + lane * 8;
  // A step's 8 tokens start at a multiple of 8, t0 + 512 s.  At the end of a row the 8 last ones are read instead, with
  // the bits of those before t0 + 512 s cleared; a vocabulary of less than 8 has one such step only.
  const auto base = [&](int s) { return max(min(t0 + s * 512, a.V - 8), 0); };

  float rate[S][8];  // 1 / noise
  if constexpr (!GREEDY) {
    const float* e = a.noise + b * a.ns;
    if constexpr (ROWS != Rows::kShort) {
#pragma unroll
      for (int s = 0; s < S; ++s) load8(e + base(s), rate[s]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) rate[0][i] = e[min(i, a.V - 1)];
    }
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int i = 0; i < 8; ++i) rate[s][i] = __builtin_amdgcn_rcpf(rate[s][i]);
  }

  // The mask two rows ahead, the logits one, without branches: what is on its way stays countable.  Where none of its 8
  // tokens is allowed a lane reads the row's first ones, as all such lanes do.
  uint32_t bits[2][S];
  Raw<T> raw[2][S];
  const auto get_bits = [&](int j, uint32_t (&x)[S]) {
#pragma unroll
    for (int s = 0; s < S; ++s) {
      const int t = t0 + s * 512, last = min(t, a.V - 1);
      uint32_t m = 0xFFu;
      if (ROWS == Rows::kMasked || (ROWS == Rows::kShort && masks)) m = ((const uint8_t*)(masks + j * a.ms[1]))[last >> 3];
      m &= (1u << min(max(a.V - t, 0), 8)) - 1u;
      x[s] = m << (t - base(s) & 7);
    }
  };
  const auto get_logits = [&](int j, const uint32_t (&x)[S], Raw<T> (&y)[S]) {
    const T* row = rows + j * a.ls[1];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if constexpr (ROWS != Rows::kShort)
        __builtin_memcpy(y[s].w, row + (x[s] ? base(s) : 0), sizeof(y[s].w));
      else if (s == 0)
        y[s].load_short(row, a.V);
    }
  };
  const auto judge = [&](int j, const uint32_t (&x)[S], const Raw<T> (&y)[S]) {
    Row r = {kLow, 0.f, 0.f, kNone};
    // a lane's tokens by number, s * 8 + i: the best one's, and that of a certain draft, which takes no part in its row's race
    int code = -1, leave = -1;
    if (!GREEDY && !a.probs && j < n) {
      const int d = drafts[j], s = (d - t0) >> 9;
      if (d >= t0 && s < S && d - t0 - s * 512 < 8 && d < a.V) leave = s * 8 + d - base(s);
    }
    const bool here = __any(leave >= 0);
    uint32_t any = 0;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      any |= x[s];
      if (!__any(x[s] != 0)) continue;
      float v[8], top = r.m;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = x[s] >> i & 1 ? y[s].at(i) : -INFINITY;
        top = fmaxf(top, v[i]);
      }
      if constexpr (GREEDY)
        if (top > r.m || code < 0)
#pragma unroll
          for (int i = 7; i >= 0; --i) code = v[i] == top ? s * 8 + i : code;
      const float f = __builtin_amdgcn_exp2f((r.m - top) * c);
      r.m = top;
      r.z *= f;
      r.score *= f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float w = __builtin_amdgcn_exp2f((v[i] - top) * c);
        r.z += w;
        if constexpr (!GREEDY) v[i] = w * rate[s][i];
      }
      if constexpr (!GREEDY) {
        if (here)
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = s * 8 + i == leave ? 0.f : v[i];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          code = v[i] > r.score ? s * 8 + i : code;
          r.score = fmaxf(r.score, v[i]);
        }
      }
    }
    r.idx = code < 0 ? kNone : base(code / 8) + code % 8;
    if (__any(any != 0)) r = join_lanes(r, c, GREEDY);
    // the waves' parts meet; two rows' slots in turn, so one barrier a row is enough
    if (lane == 0) wave_row[j & 1][wave] = r;
    __syncthreads();
    if (wave == 0) {
      r = lane < kWaves ? wave_row[j & 1][lane] : Row{kLow, 0.f, 0.f, kNone};
      r = join_lanes(r, c, GREEDY);
      if (lane == 0)
        a.part[((int64_t)b * (a.K + 1) + j) * a.pieces + piece] = make_float4(r.m, r.z, r.score, __int_as_float(r.idx));
    }
  };

  get_bits(from, bits[0]);
  get_logits(from, bits[0], raw[0]);
  if (from + 1 < to) get_bits(from + 1, bits[1]);
  for (int j = from; j < to; j += 2) {
    // rows j and j + 1, whose buffers are 0 and 1
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (j + k >= to) break;
      uint32_t now[S];
#pragma unroll
      for (int s = 0; s < S; ++s) now[s] = bits[k][s];
      if (j + k + 1 < to) get_logits(j + k + 1, bits[k ^ 1], raw[k ^ 1]);
      if (j + k + 2 < to) get_bits(j + k + 2, bits[k]);
      judge(j + k, now, raw[k]);
    }
  }
}

template <typename T, Rows ROWS>
__global__ __launch_bounds__(kThreads, 3) void scan_kernel(VerifyArgs a) {
  // The groups of one piece of a sequence are 8 workgroups apart: on one die, whose cache then holds their noise.
  const uint32_t units = (uint32_t)a.B * (uint32_t)a.pieces, eight = blockIdx.x / (8u * (uint32_t)a.groups);
  const uint32_t in = blockIdx.x - eight * 8u * (uint32_t)a.groups, unit = eight * 8 + in % 8;
  if (unit >= units) return;
  const int group = (int)(in / 8), piece = (int)(unit % (uint32_t)a.pieces), b = (int)(unit / (uint32_t)a.pieces);
  if (piece == 0 && group == 0 && threadIdx.x == 0) {
    a.best[b] = 0;
    a.done[b] = 0;
  }
  const int n = drafted(a, b), from = group * (a.K + 1) / a.groups, to = min((group + 1) * (a.K + 1) / a.groups, n + 1);
  if (from >= to) return;
  __shared__ Row wave_row[2][kWaves];
  bool greedy;
  const float c = factor_of(a, b, greedy);
  if (greedy)
    scan<T, true, ROWS>(a, wave_row, b, piece, from, to, n, c);
  else
    scan<T, false, ROWS>(a, wave_row, b, piece, from, to, n, c);
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
  __shared__ Row row[64];
  __shared__ int first;
  // the lane's draft, and what is known of it without its row's sums
  int x = -1;
  bool allowed = false;
  float l = 0.f, uq = 0.f;
  if (tid < n) {
    x = a.draft[(int64_t)b * a.K + tid];
    if ((uint32_t)x < (uint32_t)a.V) {
      l = (float)rows[tid * a.ls[1] + x];
      allowed = !masks || (masks[tid * a.ms[1] + (x >> 5)] >> (x & 31) & 1);
      if (!greedy) uq = a.uniform[(int64_t)b * a.K + tid] * (a.probs ? a.probs[b * a.ps[0] + tid * a.ps[1] + x] : 1.f);
    }
  }
  for (int j = tid >> 6; j <= n; j += kThreads / 64) {
    Row r = {kLow, 0.f, 0.f, kNone};
    for (int p = lane; p < a.pieces; p += 64) {
      const float4 y = a.part[((int64_t)b * (a.K + 1) + j) * a.pieces + p];
      const float m = fmaxf(r.m, y.x), f = __builtin_amdgcn_exp2f((r.m - m) * c), g = __builtin_amdgcn_exp2f((y.x - m) * c);
      const int idx = __float_as_int(y.w);
      if (greedy ? y.x > r.m || r.idx == kNone : y.z * g > r.score * f) r.idx = idx;  // pieces in order: the lowest
      r.score = fmaxf(r.score * f, y.z * g);
      r.z = r.z * f + y.y * g;
      r.m = m;
    }
    r = join_lanes(r, c, greedy);
    if (lane == 0) row[j] = r;
  }
  __syncthreads();
  if (tid < 64) {
    bool ok = false;
    if (tid < n && allowed && row[tid].z > 0.f)
      ok = greedy ? x == row[tid].idx : uq < __builtin_amdgcn_exp2f((l - row[tid].m) * c) / row[tid].z;
    const uint64_t refused = __ballot(!ok);  // lane n refuses (n <= 63)
    if (tid == 0) first = __builtin_ctzll(refused);
  }
  __syncthreads();
  const int at = first;
  const Row o = row[at];
  int token = o.z > 0.f && o.idx != kNone ? o.idx : -1;  // o.z is not above 0 where it is NaN
  if (!greedy && o.z > 0.f && at < n) {
    const int refused = a.draft[(int64_t)b * a.K + at];
    if (!a.probs) {
      // the draft was all that is allowed (noise that is not finite leaves no token too, whatever the draft is)
      const bool is_allowed = (uint32_t)refused < (uint32_t)a.V &&
                              (!masks || (masks[at * a.ms[1] + (refused >> 5)] >> (refused & 31) & 1));
      if (token < 0 && is_allowed) token = refused;
    } else {
      // the race over this workgroup's part of what is left of row `at`
      const float* q = a.probs + b * a.ps[0] + at * a.ps[1];
      const T* lrow = rows + at * a.ls[1];
      const uint32_t* mask = masks ? masks + at * a.ms[1] : nullptr;
      const float* noise = a.noise + b * a.ns;
      const float over = 1.f / o.z;
      uint64_t left = 0;
      const int end = min(a.V, (part + 1) * a.race);
      for (int t = part * a.race + tid * 8; t < end; t += kStep) {
        const uint32_t bits = bits8(mask, t, a.V);
        if (!bits) continue;
        float y[8], e[8], d[8];
        if (t + 8 <= a.V) {
          load8(lrow + t, y);
          load8(noise + t, e);
          load8(q + t, d);
        } else {
          load8_end(lrow, t, a.V, -INFINITY, y);
          load8_end(noise, t, a.V, 1.f, e);
          load8_end(q, t, a.V, 0.f, d);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float p = bits >> i & 1 ? __builtin_amdgcn_exp2f((y[i] - o.m) * c) * over : 0.f;
          left = max(left, race_key(fmaxf(p - d[i], 0.f) * __builtin_amdgcn_rcpf(e[i]), t + i));
        }
      }
      left = max_across(left);
      __shared__ uint64_t wave_best[kThreads / 64];
      __shared__ bool last;
      if (lane == 0) wave_best[tid >> 6] = left;
      __syncthreads();
      if (tid == 0) {
        for (int w = 1; w < kThreads / 64; ++w) left = max(left, wave_best[w]);
        unsigned long long* best = (unsigned long long*)a.best + b;
        // Both are atomics at the device's point of coherence, and the first is done before the second begins: no fence
        // over other memory is needed, for nothing else passes between the workgroups.
        __hip_atomic_fetch_max(best, left, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        last = __hip_atomic_fetch_add(a.done + b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.races - 1;
        if (last) wave_best[0] = __hip_atomic_fetch_max(best, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      if (!last) return;
      if (const uint64_t key = wave_best[0]) token = (int)~(uint32_t)key;  // otherwise p itself
    }
  }
  if (part > 0 && !(a.probs && !greedy && o.z > 0.f && at < n)) return;
  if (tid <= a.K) {
    const int mine = tid < at ? a.draft[(int64_t)b * a.K + tid] : tid == at ? token : -1;
    float lp = 0.f;
    if (mine >= 0) lp = ((float)rows[tid * a.ls[1] + mine] - row[tid].m) * (c / kLog2e) - logf(row[tid].z);
    a.tokens[(int64_t)b * (a.K + 1) + tid] = mine;
    a.logprobs[(int64_t)b * (a.K + 1) + tid] = lp;
  }
  if (tid == 0) a.accepted[b] = at;
}

// The launch.  A sequence's rows are dealt to so many groups that there are about 4096 workgroups, or one for each row
// (4096 was the best of 600 to 8192 for the batches above: fewer read the noise less often, and leave too few to run).  The
// residual's race is cut into about 1024 workgroups, none of less than a step (the best of 512 to 4096).
void plan(VerifyArgs& a, int steps) {
  a.pieces = (int32_t)(((int64_t)a.V + steps * kPiece - 1) / (steps * kPiece));
  const int64_t all = (int64_t)a.B * a.pieces;
  a.groups = (int32_t)std::min<int64_t>(a.K + 1, (4096 + all - 1) / all);
  const int64_t want = std::max<int64_t>(1, 1024 / a.B), fit = ((int64_t)a.V + kStep - 1) / kStep;
  const int64_t n = std::min(want, fit);
  a.race = (int32_t)((((int64_t)a.V + n - 1) / n + kStep - 1) / kStep * kStep);
  a.races = (int32_t)(((int64_t)a.V + a.race - 1) / a.race);
}

// (tokens are counted in 32 bits past a row's end: to the end of the last piece, and of the races' last part, which begins
// before V and is no longer than V and a step)
bool sizes_ok(int32_t B, int32_t K, int32_t V) {
  return B >= 1 && B <= 65535 && K >= 0 && K <= 63 && V >= 1 && V <= (1 << 30) - kStep;
}

size_t head_bytes(int32_t B) { return ((size_t)B * 12 + 255) / 256 * 256; }

}  // namespace

extern "C" size_t grid_verify_workspace_bytes(int32_t B, int32_t K, int32_t V) {
  if (!sizes_ok(B, K, V)) return 0;
  const size_t pieces = ((size_t)V + kSteps<float> * kPiece - 1) / (kSteps<float> * kPiece);  // 16-bit rows have fewer
  return head_bytes(B) + (size_t)B * (size_t)(K + 1) * pieces * sizeof(float4);
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
  a.done = (uint32_t*)(a.best + (size_t)g.B);
  a.part = (float4*)((uint8_t*)g.workspace + head_bytes(g.B));
  a.B = g.B;
  a.K = g.K;
  a.V = g.V;
  plan(a, g.dtype == GRID_DTYPE_F32 ? kSteps<float> : kSteps<bf16_t>);
  if (!g.noise || !g.draft_probs) a.races = 1;
  const int64_t one = ((int64_t)g.B * a.pieces + 7) / 8 * 8 * a.groups, two = (int64_t)g.B * a.races;
  if (one > 1 << 23 || two > 1 << 23) return fail(GRID_E_CAPACITY, "grid_verify: too many rows for one launch");
  hipStream_t s = (hipStream_t)stream;
  auto launch = [&](auto type) {
    using T = decltype(type);
    const dim3 blocks((unsigned)one), threads(kThreads);
    if (g.V < 8)
      hipLaunchKernelGGL((scan_kernel<T, Rows::kShort>), blocks, threads, 0, s, a);
    else if (g.mask)
      hipLaunchKernelGGL((scan_kernel<T, Rows::kMasked>), blocks, threads, 0, s, a);
    else
      hipLaunchKernelGGL((scan_kernel<T, Rows::kAll>), blocks, threads, 0, s, a);
    hipLaunchKernelGGL(pick_kernel<T>, dim3((unsigned)two), dim3(kThreads), 0, s, a);
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
