// sample.hip -- grid_sample: one token of every row from its masked and filtered distribution (gfx950).
//
// Two launches.  The first takes pieces of the rows into registers.  Without top_k and top_p it races w / noise over them,
// relative to the piece's largest logit, as an argmax that needs no normaliser.  Otherwise it leaves a histogram of the
// piece: counts and masses by sixteenths of an octave of the weight, 64 octaves from the piece's largest downwards.  Bins are
// cut from log2 of the weight itself, so pieces need not know each other's largest logits.
//
// In the second every workgroup of a row adds up its pieces' histograms and finds the bins in which the count reaches top_k
// and the mass top_p.  Tokens of the bins before are kept: it races those of its piece; those of the bins at a cut go to
// a list.  The last of the row's workgroups orders the list by digits of the keys (of equal logits the lower indexes are
// kept), races what is kept of it, and joins all.  Masses are whole numbers, whose sums do not depend on the order of the
// atomics; partial sums of floats have a place each.
//
// A row whose list is too long (nearly all logits alike), or whose exponents are out of all bounds, is taken by one
// workgroup, digit by digit over the row itself.
//
// Bounds.  256 rows of 50257 in float32 have 51 MB to read, 10 us; the launches take 20 and 38 us, of which the rows alone
// are 14, a workgroup's vector units being busy half of the time; then noise and what a flat nucleus lists, ordered by
// digits.  32 rows of 151936 in bf16 take 11 and 18 us, one 6 and 12: some ten dependent reads in two launches, and the
// pieces' histograms, which every workgroup of a row adds up for itself (a launch that did it once would cost what it
// saves; it grows with the square of V: a row of 4 million 58 us, 16 million 388, 64 million 4.6 ms).  A workgroup remembers
// each wave's largest logit of a step, so waves whose tokens are all below the cuts do not read them again: of the 256 rows
// 54 us for 65.
#include <algorithm>
#include <string>
#include <type_traits>

#include "lanes.h"
#include "paged.h"

using namespace grid;

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kStep = kThreads * 8;  // tokens that a workgroup takes at a time
constexpr int kHeld = 4;               // steps of a piece, at most: what registers hold where two workgroups share a compute unit
constexpr int kBins = 1024, kPerOctave = 16;
constexpr int kList = 4096;  // tokens of a piece's bins at the cuts, at most
constexpr int kTops = kHeld * kWaves;
constexpr int kDigit = 9;    // bits, a thread for each value
static_assert(1 << kDigit == kThreads && kBins == 2 * kThreads, "");
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kNone = 0x7FFFFFFF;

struct Piece {
  float m, z;     // largest logit (NaN: one that is not a number); sum of the weights relative to it
  uint64_t best;  // of the race: the score relative to m, and the complement of the token (greedy: of m); or the mass of all
                  // bins, a weight of 1 at the upper edge of the highest having 2^shift
  float l;        // the best's logit
  int halves;     // of the bins, that hold something
};
// What a workgroup of the second launch leaves: the best that it kept, its logit and the kept weights' sum; tokens listed.
struct Left {
  uint64_t best, l_z, listed;
};

struct SampleArgs {
  const void* logits;
  const uint32_t* mask;
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *noise;
  int64_t ls, ms, ns;
  int32_t* tokens;
  float* logprobs;
  int32_t V, pieces, steps, room;  // room: of a piece's list
  int32_t count_bits, mass_shift;  // an entry of a histogram: mass << count_bits | count
  int32_t shift;                   // of whole rows: a mass is w * 2^shift
  Piece* piece;    // [B][pieces]
  Left* left;      // [B][pieces]
  uint32_t* done;  // [B]
  uint64_t* list;  // [B][pieces][room]: key << 32 | complement of the token
  uint64_t* hist;  // [B][pieces][kBins]
  float* tops;     // [B][pieces][kTops]: the largest logit of a wave's part of a step
};

// Logits in their order, as whole numbers; -0 is 0.
__device__ inline uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float value_of(uint32_t key) {
  return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xFFFFFFFFu));
}
// What decides a race: the score, then the lower token; 0 where nothing is raced.
__device__ inline uint64_t race_key(float score, int t) {
  return score > 0.f ? (uint64_t)__float_as_uint(score) << 32 | (uint32_t)~t : 0;
}
__device__ inline float maximum_across(float x) {  // NaN if one is
  return __uint_as_float(across(__float_as_uint(x), [](uint32_t p, uint32_t q) {
    return __float_as_uint(__builtin_elementwise_maximum(__uint_as_float(p), __uint_as_float(q)));
  }));
}

struct Shared {
  uint64_t mass[256];
  uint32_t count[256];
  float f[kWaves];
  uint64_t best[kWaves], low[kWaves];
  uint64_t before;
  uint32_t bin;
};

__device__ inline float block_maximum(Shared& sh, float x) {
  x = maximum_across(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.f[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) x = __builtin_elementwise_maximum(x, sh.f[w]);
  return x;
}
__device__ inline float block_sum(Shared& sh, float x) {
  x = sum_across(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.f[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) x += sh.f[w];
  return x;
}
__device__ inline uint64_t block_sum(Shared& sh, uint64_t x) {
  x = sum_across(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) x += sh.best[w];
  return x;
}
__device__ inline uint64_t block_best(Shared& sh, uint64_t x) {
  x = max_across(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWaves; ++w) x = max(x, sh.best[w]);
  return x;
}

// What a row asks for.
struct Row {
  const void* logits;
  const uint8_t* mask;
  const float* noise;
  float c;      // log2 e / temperature
  float top_p, low;
  int top_k;    // 0: all
  bool greedy, cuts;  // cuts: top_k or top_p are in force
  __device__ bool filtered() const { return cuts || low > 0.f; }
};
template <typename T>
__device__ inline Row row_of(const SampleArgs& a, int64_t b) {
  Row r;
  const float t = a.temperature ? a.temperature[b] : 1.f, p = a.top_p ? a.top_p[b] : 1.f, q = a.min_p ? a.min_p[b] : 0.f;
  const int k = a.top_k ? a.top_k[b] : 0;
  r.logits = (const T*)a.logits + b * a.ls;
  r.mask = a.mask ? (const uint8_t*)(a.mask + b * a.ms) : nullptr;
  r.noise = a.noise ? a.noise + b * a.ns : nullptr;
  r.greedy = !a.noise || !(t > 0.f);
  r.c = r.greedy ? kLog2e : fminf(fmaxf(kLog2e / t, 1e-30f), 1e30f);
  r.top_k = !r.greedy && k > 0 && k < a.V ? k : 0;
  r.top_p = !r.greedy && p < 1.f ? fmaxf(p, 0.f) : 1.f;
  r.low = !r.greedy && q > 0.f ? fminf(q, 1.f) : 0.f;
  r.cuts = r.top_k > 0 || r.top_p < 1.f;
  return r;
}

// The weight's place in octaves of a sixteenth; whole parts of it are bins.  (c times a power of two: exact.)
__device__ inline float place(float l, float c) { return l * (c * kPerOctave); }

// 8 logits as they are in memory.
template <typename T>
struct Raw {
  static constexpr int N = sizeof(T) * 2;
  uint32_t w[N];
  __device__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    if constexpr (std::is_same<T, bf16_t>::value) return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
    return (float)__builtin_bit_cast(f16_t, (uint16_t)(w[i / 2] >> (i & 1) * 16));
  }
  // x where bit i of `bits` is set, otherwise -inf
  __device__ float at(int i, uint32_t bits) const {
    const uint32_t on = (uint32_t)((int32_t)(bits << (31 - i)) >> 31);
    return __uint_as_float((on & __float_as_uint(at(i))) | (~on & 0xFF800000u));
  }
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

// The 8 tokens of a lane's step: from which one they are read (the row's last 8 at its end), and which count.
struct Eight {
  int from;
  uint32_t bits;
};
__device__ inline Eight eight_of(const SampleArgs& a, const Row& r, int t) {
  uint32_t bits = r.mask && t < a.V ? r.mask[t >> 3] : 0xFFu;
  bits &= (1u << min(max(a.V - t, 0), 8)) - 1u;
  const int from = max(min(t, a.V - 8), 0);
  return {from, bits << (t - from & 7)};
}
template <typename T>
__device__ inline void load_eight(const SampleArgs& a, const Row& r, const Eight& e, Raw<T>& x) {
  const T* row = (const T*)r.logits;
  if (a.V >= 8)
    __builtin_memcpy(x.w, row + (e.bits ? e.from : 0), sizeof(x.w));  // (none counts: the row's first, which are at hand)
  else
    x.load_short(row, a.V);
}
__device__ inline void load_noise(const SampleArgs& a, const Row& r, const Eight& e, float (&x)[8]) {
  if (a.V >= 8)
    __builtin_memcpy(x, r.noise + e.from, 32);
  else
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = r.noise[min(i, a.V - 1)];
}

// The mass of a bin, `j` below that to whose upper edge it is relative, from a histogram's.
__device__ inline uint64_t mass_of(const SampleArgs& a, uint64_t mass, int j) {
  const float part = __builtin_amdgcn_exp2f(-(float)(j % kPerOctave) * (1.f / kPerOctave));
  return (uint64_t)((double)mass * __builtin_ldexp((double)part, a.shift - a.mass_shift - j / kPerOctave));
}

// ------------------------------------------------------------------------------------------- keys, digit by digit
// What is kept: keys above `key`, and of equal ones the tokens up to `index`.
struct Cut {
  uint32_t key;
  int index;
  __device__ bool has(uint32_t k, int t) const { return k > key || (k == key && t <= index); }
};

__device__ inline void clear(Shared& sh) {
  __syncthreads();
  if (threadIdx.x < 256) sh.mass[threadIdx.x] = 0, sh.count[threadIdx.x] = 0;
  __syncthreads();
}

// The bin in which the counts (or masses) from the highest bin on (the lowest: !down) reach the target; what the bins before
// hold is taken out of the target.
__device__ inline uint32_t reached(Shared& sh, uint64_t& target, bool by_mass, bool down) {
  __syncthreads();
  if (threadIdx.x < 64) {
    const int lane = (int)threadIdx.x;
    uint64_t v[4], mine = 0;
    for (int i = 0; i < 4; ++i) {
      const int at = down ? 255 - (lane * 4 + i) : lane * 4 + i;
      v[i] = by_mass ? sh.mass[at] : sh.count[at];
      mine += v[i];
    }
    const uint64_t upto = sum_upto(mine);
    const uint64_t hit = __ballot(upto >= target);
    if (hit == 0 ? lane == 63 : lane == __builtin_ctzll(hit)) {
      uint64_t before = upto - mine;
      int i = 0;
      while (i < 3 && before + v[i] < target) before += v[i++];
      sh.bin = (uint32_t)(down ? 255 - (lane * 4 + i) : lane * 4 + i);
      sh.before = before;
    }
  }
  __syncthreads();
  const uint32_t bin = sh.bin;
  target -= sh.before;
  __syncthreads();
  return bin;
}

// The cut at which, in order, the count (or the mass) of the tokens that each() goes over reaches `target`, which is 1 or
// more; all of them where it is more than there is.  mass(l) is the same for equal logits.
template <typename Each, typename Mass>
__device__ Cut find_cut(Shared& sh, int V, uint64_t target, bool by_mass, Each each, Mass mass) {
  uint32_t key = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    clear(sh);
    each([&](float l, int) {
      const uint32_t k = key_of(l);
      if (shift < 24 && k >> (shift + 8) != key >> (shift + 8)) return;
      if (by_mass)
        atomicAdd((unsigned long long*)&sh.mass[k >> shift & 255], (unsigned long long)mass(l));
      else
        atomicAdd(&sh.count[k >> shift & 255], 1u);
    });
    key |= reached(sh, target, by_mass, true) << shift;
  }
  // of the equal ones as many as reach it, the lower indexes first
  const uint64_t unit = by_mass ? max((uint64_t)1, mass(value_of(key))) : 1;
  uint64_t ties = (target + unit - 1) / unit;
  uint32_t index = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (shift > 0 && V >> shift == 0) continue;
    clear(sh);
    each([&](float l, int t) {
      if (key_of(l) != key) return;
      if (shift < 24 && (uint32_t)t >> (shift + 8) != index >> (shift + 8)) return;
      atomicAdd(&sh.count[t >> shift & 255], 1u);
    });
    index |= reached(sh, ties, false, false) << shift;
  }
  return {key, (int)index};
}

__device__ inline void write_token(const SampleArgs& a, const Row& r, int64_t b, uint64_t best, float l, float m, float z) {
  a.tokens[b] = best ? (int)~(uint32_t)best : -1;
  a.logprobs[b] = best ? (l - m) * (r.c / kLog2e) - logf(z) : 0.f;
}

// A whole row by itself: for rows that the histograms do not serve.
template <typename T>
__device__ __forceinline__ void whole_row(const SampleArgs& a, const Row& r, Shared& sh, int64_t b, float m) {
  const T* row = (const T*)r.logits;
  const auto each = [&](auto f) {
    for (int t = (int)threadIdx.x * 8; t < a.V; t += kStep) {
      const Eight e = eight_of(a, r, t);
      if (!e.bits) continue;
      Raw<T> x;
      load_eight(a, r, e, x);
#pragma unroll 1
      for (int i = 0; i < 8; ++i)
        if (e.bits >> i & 1) f((float)row[e.from + i], e.from + i);
    }
  };
  const auto weight = [&](float l) { return __builtin_amdgcn_exp2f((l - m) * r.c); };
  const auto mass = [&](float l) { return (uint64_t)__builtin_ldexpf(weight(l), a.shift); };
  Cut kept = {0, kNone};
  if (r.top_k > 0) kept = find_cut(sh, a.V, (uint64_t)r.top_k, false, each, mass);
  if (r.top_p < 1.f) {
    const Cut within = kept;
    const auto among = [&](auto f) {
      each([&](float l, int t) {
        if (within.has(key_of(l), t)) f(l, t);
      });
    };
    clear(sh);
    uint64_t mine = 0;
    among([&](float l, int) { mine += mass(l); });
    if (mine) atomicAdd((unsigned long long*)&sh.mass[0], (unsigned long long)mine);
    __syncthreads();
    const double want = __builtin_ceil((double)r.top_p * (double)sh.mass[0]);
    kept = find_cut(sh, a.V, max((uint64_t)want, (uint64_t)1), true, among, mass);
  }
  float z = 0.f;
  uint64_t best = 0;
  each([&](float l, int t) {
    const float w = weight(l);
    if (!kept.has(key_of(l), t) || w < r.low) return;
    z += w;
    best = max(best, race_key(r.greedy ? (l == m ? 1.f : 0.f) : w * __builtin_amdgcn_rcpf(r.noise[t]), t));
  });
  z = block_sum(sh, z);
  best = block_best(sh, best);
  if (threadIdx.x == 0) write_token(a, r, b, best, best ? (float)row[(int)~(uint32_t)best] : 0.f, m, z);
}

// A thread's part of a race: its tokens come in order, so of equal scores the first is kept.
struct Race {
  float z, score, l;  // the weights' sum; the best score and its logit
  int t;
  // logit l, log2 of the weight, noise; weights below `low` are left out
  __device__ void take(float logit, float log_w, float noise, float low, int token) {
    const float w = __builtin_amdgcn_exp2f(log_w);
    if (w < low) return;
    z += w;
    const float now = w * __builtin_amdgcn_rcpf(noise);
    const bool more = now > score;
    score = more ? now : score;
    l = more ? logit : l;
    t = more ? token : t;
  }
  __device__ uint64_t key() const { return race_key(score, t); }
};

// ------------------------------------------------------------------------------------------------------ first launch
// Bins from this one on hold no cut: what lies so far below the largest weight, V of them at most, is together less than the
// mass that top_p leaves out.
__device__ inline int deepest(const SampleArgs& a, const Row& r) {
  if (r.top_k > 0) return kBins;
  const float octaves = __builtin_amdgcn_logf((float)a.V) - __builtin_amdgcn_logf(1.f - r.top_p) + 1.f;
  return (int)fminf(octaves * kPerOctave, (float)(kBins - 1)) + 1;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void pieces_kernel(SampleArgs a) {
  constexpr int H = kHeld;
  __shared__ Shared sh;
  __shared__ uint64_t hist[kBins];
  const int tid = (int)threadIdx.x, piece = (int)(blockIdx.x % (uint32_t)a.pieces);
  const int64_t b = blockIdx.x / (uint32_t)a.pieces;
  const Row r = row_of<T>(a, b);
  Eight e[H];
  Raw<T> x[H];
#pragma unroll
  for (int s = 0; s < H; ++s) {
    if (s >= a.steps) continue;
    e[s] = eight_of(a, r, (piece * a.steps + s) * kStep + tid * 8);
  }
#pragma unroll
  for (int s = 0; s < H; ++s) {
    if (s >= a.steps) continue;
    load_eight(a, r, e[s], x[s]);
  }
  if (r.cuts)
    for (int i = tid; i < kBins; i += kThreads) hist[i] = 0;
  if (piece == 0 && tid == 0) a.done[b] = 0;
  float m = -INFINITY, tops[H];
#pragma unroll
  for (int s = 0; s < H; ++s) {
    if (s >= a.steps) continue;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; i += 2)
      top = __builtin_elementwise_maximum(top, __builtin_elementwise_maximum(x[s].at(i, e[s].bits), x[s].at(i + 1, e[s].bits)));
    tops[s] = top;
    m = __builtin_elementwise_maximum(m, top);
  }
  m = block_maximum(sh, m);
  float z = 0.f, l_best = 0.f;
  uint64_t mine = 0, best = 0;
  int halves = 1;
  const bool alive = m > -INFINITY && m < INFINITY;
  if (alive && r.cuts) {
    const float top = __builtin_floorf(place(m, r.c)), end = (float)deepest(a, r), edge = (top + 1.f) * (1.f / kPerOctave);
    const float unit = __builtin_ldexpf(1.f, a.mass_shift);
    float rest = 0.f;
#pragma unroll
    for (int s = 0; s < H; ++s) {
      if (s >= a.steps) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float l = x[s].at(i, e[s].bits), at = __builtin_floorf(place(l, r.c)), down = top - at;
        if (down < end) {
          // the weight relative to the bin's upper edge, below or about 1
          uint32_t mass = 0;
          if (r.top_p < 1.f)
            mass = (uint32_t)(__builtin_amdgcn_exp2f(__builtin_fmaf(l, r.c, (at + 1.f) * (-1.f / kPerOctave))) * unit);
          atomicAdd((unsigned long long*)&hist[(int)down], (unsigned long long)((uint64_t)mass << a.count_bits | 1u));
        } else {
          rest += __builtin_amdgcn_exp2f(__builtin_fmaf(l, r.c, -edge));
        }
      }
    }
    __syncthreads();
    uint64_t* to = a.hist + (b * a.pieces + piece) * kBins;
    const uint64_t x[2] = {hist[tid], hist[kThreads + tid]};
    for (int h = 0; h < 2; ++h) best += mass_of(a, x[h] >> a.count_bits, h * kThreads + tid);
    to[tid] = x[0];
    if (__syncthreads_or(x[1] != 0)) {
      to[kThreads + tid] = x[1];
      halves = 2;
    }
    best = block_sum(sh, best + (uint64_t)__builtin_ldexpf(rest, a.shift));
    mine = tid == 0 ? best : 0;
  } else if (alive && !r.filtered()) {
    Race race = {0.f, 0.f, 0.f, 0};
#pragma unroll
    for (int s = 0; s < H; ++s) {
      if (s >= a.steps) continue;
      float n[8];
      if (!r.greedy) load_noise(a, r, e[s], n);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float l = x[s].at(i, e[s].bits);
        if (r.greedy) {
          race.z += __builtin_amdgcn_exp2f((l - m) * r.c);
          const bool more = l == m && race.score == 0.f;
          race.t = more ? e[s].from + i : race.t;
          race.score = more ? 1.f : race.score;
        } else if (e[s].bits >> i & 1) {
          race.take(l, (l - m) * r.c, n[i], 0.f, e[s].from + i);
        }
      }
    }
    mine = race.key();
    l_best = r.greedy ? m : race.l;
    z = race.z;
    z = block_sum(sh, z);
    best = block_best(sh, mine);
  }
  if (r.cuts)
#pragma unroll
    for (int s = 0; s < H; ++s) {
      if (s >= a.steps) continue;
      const float top = maximum_across(tops[s]);
      if ((tid & 63) == 0) a.tops[(b * a.pieces + piece) * kTops + s * kWaves + (tid >> 6)] = top;
    }
  // (no two threads have the same token)
  if (best ? mine == best : tid == 0) a.piece[b * a.pieces + piece] = {m, z, best, l_best, halves};
}

// ----------------------------------------------------------------------------------------------------- second launch
// Where a row is cut, in bins below its highest.  Masses are whole: a weight of 1 at the upper edge of bin 0 has 2^shift.
struct Bins {
  int sure;                          // bins before this one are kept whole
  int p_from, p_to;                  // the bins in which top_p may cut (p_from > p_to: none)
  int k;                             // the bin in which top_k cuts (kBins: none)
  uint32_t k_left, k_count;          // tokens that are kept of it, of so many
  uint64_t k_mass, k_before;         // its mass, and that of the bins before it
  uint64_t p_before, all;            // of the bins before p_from, of all
};
__device__ inline Bins no_cuts() { return {kBins, kBins, -1, kBins, 0, 0, 0, 0, 0, 0}; }

// The row's bins, from its pieces'; all threads.  A lane has piece `lane` (of more than 64: read again).  The lower half of the
// bins is looked at only where a cut lies there.
__device__ inline Bins bins_of(const SampleArgs& a, const Row& r, int64_t b, float top, Piece own_piece, Shared& sh, Bins& found) {
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint64_t* hist = a.hist + b * a.pieces * kBins;
  if (tid == 0) found = no_cuts();
  uint64_t all = 0, below = 0, mass[2] = {0, 0}, upto[2] = {0, 0};
  uint32_t count = 0;
  double want = 0.0;
  for (int h = 0; h < 2; ++h) {
    uint32_t n = 0;
    uint64_t sum = 0;
    for (int p0 = 0; p0 < a.pieces; p0 += 64) {
      Piece x = own_piece;
      if (p0 > 0) {
        x.m = -INFINITY;
        if (p0 + lane < a.pieces) x = a.piece[b * a.pieces + p0 + lane];
      }
      // the piece's bin 0 among the row's; one of no tokens is far below
      const float down = top - __builtin_floorf(place(x.m, r.c));
      const int off = (int)fminf(down, (float)kBins), end = down < (float)kBins ? x.halves * kThreads : 0;
      if (h == 0 && end > 0) {
        const float part = __builtin_amdgcn_exp2f(-(float)(off % kPerOctave) * (1.f / kPerOctave));
        all += (uint64_t)((double)x.best * __builtin_ldexp((double)part, -(off / kPerOctave)));
      }
      // Pieces that are asked for together.  It matters little: of 32000 to 262144 tokens, 1 to 256 rows, top_k 50 or a nucleus
      // of 0.9, passes take with 4, 8 and 16 between 3 % less and 3 % more than with 10, with 20 up to 6 % more.
      constexpr int kAhead = 10;
      for (int p = 0; p < min(64, a.pieces - p0); p += kAhead) {
        uint64_t y[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int q = min(p + i, 63), from = h * kThreads + tid - __builtin_amdgcn_readlane(off, q);
          const bool in = p + i < 64 && from >= 0 && from < __builtin_amdgcn_readlane(end, q);  // (end: 0 past the last piece)
          y[i] = hist[in ? (int64_t)(p0 + q) * kBins + from : 0];
          y[i] = in ? y[i] : 0;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          n += (uint32_t)y[i] & ((1u << a.count_bits) - 1);
          sum += y[i] >> a.count_bits;
        }
      }
    }
    if (h == 0) {
      all = sum_across(all);
      want = (double)r.top_p * (double)all;
    }
    mass[h] = mass_of(a, sum, h * kThreads + tid);
    // counts and masses up to and with each bin
    uint32_t c = sum_upto(n);
    uint64_t w = sum_upto(mass[h]), total = below;
    if (h > 0) __syncthreads();
    if (lane == 63) sh.count[wave] = c, sh.best[wave] = w;
    __syncthreads();
    uint32_t counted = count;
    c += count;
    w += below;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const uint64_t x = sh.best[i];
      const uint32_t y = sh.count[i];
      c += i < wave ? y : 0;
      w += i < wave ? x : 0;
      total += x;
      counted += y;
    }
    count = counted;
    below = total;
    upto[h] = w;
    if (r.top_k > 0 && c >= (uint32_t)r.top_k && c - n < (uint32_t)r.top_k) {
      found.k = h * kThreads + tid;
      found.k_left = (uint32_t)r.top_k - (c - n);
      found.k_count = n;
      found.k_mass = mass[h];
      found.k_before = w - mass[h];
    }
    if (r.top_k > 0 ? count >= (uint32_t)r.top_k : (double)below >= want * (1.0 + 1e-9)) break;
  }
  if (tid == 0) found.all = all;
  __syncthreads();
  if (r.top_p < 1.f) {
    double lo = (double)all, hi = (double)all;
    if (found.k < kBins) {
      // (the largest ones of the bin are kept, whose weights differ by a factor of 2^(1 / 16) at most)
      const double before = (double)found.k_before, mine = (double)found.k_mass;
      const double share = mine * ((double)found.k_left / (double)found.k_count);
      lo = before + share;
      hi = before + fmin(mine, share * 1.05);
    }
    const uint64_t from = max((uint64_t)(lo * (double)r.top_p * (1.0 - 1e-9)), (uint64_t)1);
    const uint64_t to = max((uint64_t)(hi * (double)r.top_p * (1.0 + 1e-9)), from);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint64_t w = upto[h], before = w - mass[h];
      if (w >= from && before < from) found.p_from = h * kThreads + tid, found.p_before = before;
      if (w >= to && before < to) found.p_to = h * kThreads + tid;
    }
    // (a target that rounding puts past all there is: the last bin)
    if (tid == 0 && to > below) found.p_to = kBins - 1;
    if (tid == 0 && from > below) found.p_from = kBins - 1, found.p_before = below;
    __syncthreads();
  }
  Bins f = found;
  f.sure = min(f.k, f.p_from);
  return f;
}

// The tokens of a row's bins at the cuts, as one workgroup orders them.  An entry is key << 32 | complement of the token:
// larger ones come first, and a cut is the smallest entry that is kept.
struct Listed {
  const SampleArgs& a;
  const Row& r;
  Shared& sh;
  uint64_t* digits;  // [kThreads]
  uint64_t* held;    // [kHeldList]: the entries, where they are no more
  const Bins& f;
  int64_t b;
  float m, top;
  uint32_t n;
  // Masses are w * 2^shift, relative to the upper edge of the highest bin on the list, so a weight is 1 and a rounding at
  // most: the sum of n is below 2^63 and a few roundings.
  int shift;
  static constexpr int kHeldList = kList;
  static __device__ int shift_of(uint32_t n) { return min(46, 31 + __builtin_clz(n | 1u)); }

  __device__ int highest() const { return min(f.k, f.p_from); }
  __device__ float edge() const { return (top - (float)highest() + 1.f) * (1.f / kPerOctave); }
  static __device__ float logit(uint64_t x) { return value_of((uint32_t)(x >> 32)); }
  __device__ int bin(uint64_t x) const { return (int)fminf(top - __builtin_floorf(place(logit(x), r.c)), (float)kBins); }
  __device__ uint64_t mass(uint64_t x) const {
    return (uint64_t)__builtin_ldexpf(__builtin_amdgcn_exp2f(__builtin_fmaf(logit(x), r.c, -edge())), shift);
  }
  // The mass of the listed tokens that top_p keeps, where top_k keeps so much of its bin.
  __device__ uint64_t target(uint64_t k_mass) const {
    // the list's masses relative to the row's
    const double unit = __builtin_ldexp((double)__builtin_amdgcn_exp2f(-(float)(highest() % kPerOctave) * (1.f / kPerOctave)),
                                        a.shift - highest() / kPerOctave - shift);
    const double all = f.k < kBins ? (double)f.k_before + (double)k_mass * unit : (double)f.all;
    const double want = __builtin_ceil(((double)r.top_p * all - (double)f.p_before) / unit);
    return want > 1.0 ? (uint64_t)fmin(want, 0x1.8p63) : 1;  // (more than all there is: all)
  }
  __device__ float score(uint64_t x) const {
    const float w = __builtin_amdgcn_exp2f((logit(x) - m) * r.c);
    return w < r.low ? -1.f : w * __builtin_amdgcn_rcpf(r.noise[(int)~(uint32_t)x]);  // -1: min_p leaves it out
  }
  static __device__ uint64_t key(uint64_t x, float score) {
    return score > 0.f ? (uint64_t)__float_as_uint(score) << 32 | (uint32_t)x : 0;
  }
  // f(entry) of all of them
  template <typename F>
  __device__ void each(F g) const {
    if (n <= kHeldList) {
      for (uint32_t i = threadIdx.x; i < n; i += kThreads) g(held[i]);
      return;
    }
    // (a wave a piece: 151936 tokens, std 0.6, a nucleus of 0.9 62 us for 89, the pieces one after the other)
    for (int p = (int)threadIdx.x >> 6; p < a.pieces; p += kWaves) {
      const int64_t at = b * a.pieces + p;
      const uint32_t have = (uint32_t)__hip_atomic_load(&a.left[at].listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll 4
      for (uint32_t i = threadIdx.x & 63; i < have; i += 64)
        g(__hip_atomic_load(a.list + at * a.room + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    }
  }

  // Up to 64 E, E a lane of the first wave: a token's place and the mass before it are counted, by all waves where there are
  // more than a few.  best: of the kept ones' race, its logit in l; returns their mass.  (Of other waves nothing is returned.)
  static constexpr uint32_t kAlone = 24;  // up to so many a wave counts by itself
  template <int E>
  __device__ uint64_t by_count(uint32_t* before, uint64_t& best, float& l) const {
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint64_t x[E], own[E], mass_before[E];
    uint32_t places[E];
    float mine[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t i = (uint32_t)(e * 64 + lane);
      x[e] = i < n ? held[i] : 0;
      mine[e] = x[e] && wave == 0 ? score(x[e]) : -1.f;
      own[e] = x[e] ? mass(x[e]) : 0;
      mass_before[e] = 0;
      places[e] = 0;
    }
    if (n > kAlone) {
      // before[i] and digits[i] gather what the waves count, a part of the entries each
      if (tid < 64 * E) before[tid] = 0, digits[tid] = 0;
      __syncthreads();
    }
    const uint32_t waves = n > kAlone ? kWaves : 1, part = (n + waves - 1) / waves;
    const uint32_t from = min((uint32_t)wave * part, n), to = n > kAlone || wave == 0 ? min(from + part, n) : from;
    for (uint32_t i = from; i < to; ++i) {
      const uint64_t y = held[i], w = mass(y);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const bool first = y > x[e];
        places[e] += first;
        mass_before[e] += first ? w : 0;
      }
    }
    if (n > kAlone) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (places[e]) {
          atomicAdd(&before[e * 64 + lane], places[e]);
          atomicAdd((unsigned long long*)&digits[e * 64 + lane], (unsigned long long)mass_before[e]);
        }
      __syncthreads();
    }
    if (wave > 0) return 0;
    if (n > kAlone)
#pragma unroll
      for (int e = 0; e < E; ++e) places[e] = before[e * 64 + lane], mass_before[e] = digits[e * 64 + lane];
    bool kept[E];
    int at[E];
    uint32_t whole = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      at[e] = x[e] ? bin(x[e]) : kBins;
      whole += (uint32_t)__builtin_popcountll(__ballot(at[e] < f.k && x[e]));
    }
    uint64_t k_mass = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      kept[e] = x[e] && (at[e] < f.k || places[e] - whole < f.k_left);
      if (kept[e] && at[e] == f.k) k_mass += own[e];
    }
    if (r.top_p < 1.f) {
      if (f.k < kBins) k_mass = sum_across(k_mass);
      const uint64_t want = target(k_mass);
#pragma unroll
      for (int e = 0; e < E; ++e) kept[e] = kept[e] && at[e] <= f.p_to && mass_before[e] < want;
    }
    uint64_t first = 0, entry = 0, sum = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (!kept[e] || !(mine[e] >= 0.f)) continue;
      sum += own[e];
      entry = key(x[e], mine[e]) > first ? x[e] : entry;
      first = max(first, key(x[e], mine[e]));
    }
    best = max_across(first);
    const uint64_t winner = __ballot(best && first == best);
    l = logit(lane_of(entry, winner ? __builtin_ctzll(winner) : 0));
    return sum_across(sum);
  }

  // The smallest entry of those that `among` takes that is kept when, in order, their count (or mass) has to reach `target`,
  // which is no more than there is: 9 bits at a time, from the highest in which they differ.
  template <typename Among>
  __device__ uint64_t cut(uint64_t target, bool by_mass, Among among) const {
    constexpr uint64_t kLast = kThreads - 1;
    uint64_t lo = 1, hi = ~0ull;
    for (;;) {
      uint64_t most = 0, least = ~0ull;
      each([&](uint64_t x) {
        if (x >= lo && x <= hi && among(x)) most = max(most, x), least = min(least, x);
      });
      most = max_across(most);
      least = min_across(least);
      __syncthreads();
      if ((threadIdx.x & 63) == 0) sh.best[threadIdx.x >> 6] = most, sh.low[threadIdx.x >> 6] = least;
      digits[threadIdx.x] = 0;
      __syncthreads();
      for (int w = 0; w < kWaves; ++w) most = max(most, sh.best[w]), least = min(least, sh.low[w]);
      if (most <= least) return least;  // one is left (none: all are kept)
      const int shift = max(64 - kDigit - __builtin_clzll(most ^ least), 0);
      each([&](uint64_t x) {
        if (x >= lo && x <= hi && among(x))
          atomicAdd((unsigned long long*)&digits[kLast - (x >> shift & kLast)], (unsigned long long)(by_mass ? mass(x) : 1));
      });
      __syncthreads();
      // the digit at which the target is reached
      const int j = (int)threadIdx.x, lane = j & 63;
      const uint64_t own = digits[j];
      uint64_t upto = sum_upto(own);
      if (lane == 63) sh.best[j >> 6] = upto;
      if (j == 0) sh.bin = kLast - (uint32_t)(least >> shift & kLast), sh.before = 0;  // (where rounding leaves the target out of reach)
      __syncthreads();
      for (int w = 0; w < j >> 6; ++w) upto += sh.best[w];
      if (upto >= target && upto - own < target) sh.bin = (uint32_t)j, sh.before = upto - own;
      __syncthreads();
      target -= sh.before;
      const uint64_t prefix = shift + kDigit < 64 ? most >> (shift + kDigit) << kDigit : 0;
      lo = (prefix | (kLast - sh.bin)) << shift;
      hi = lo | ((1ull << shift) - 1);
    }
  }
  // Any number, by the workgroup.
  __device__ uint64_t by_digits(uint64_t& best, float& l) const {
    uint64_t by_k = 0, kept = 0;
    if (f.k < kBins) by_k = cut(f.k_left, false, [&](uint64_t x) { return bin(x) == f.k; });
    const auto in_k = [&](uint64_t x) { return bin(x) < f.k || x >= by_k; };
    if (r.top_p < 1.f) {
      uint64_t k_mass = 0;
      if (f.k < kBins) {
        each([&](uint64_t x) {
          if (bin(x) == f.k && x >= by_k) k_mass += mass(x);
        });
        k_mass = block_sum(sh, k_mass);
      }
      kept = cut(target(k_mass), true, [&](uint64_t x) { return bin(x) <= f.p_to && in_k(x); });
    }
    uint64_t sum = 0, mine = 0, entry = 0;
    each([&](uint64_t x) {
      if (x < kept || !in_k(x)) return;
      const float s = score(x);
      if (s < 0.f) return;
      sum += mass(x);
      entry = key(x, s) > mine ? x : entry;
      mine = max(mine, key(x, s));
    });
    best = block_best(sh, mine);
    if (best && mine == best) sh.f[0] = logit(entry);
    sum = block_sum(sh, sum);
    l = sh.f[0];
    return sum;
  }
};

template <typename T>
__global__ __launch_bounds__(kThreads, 6) void draw_kernel(SampleArgs a) {
  __shared__ Shared sh;
  __shared__ uint64_t digits[kThreads], held[Listed::kHeldList];
  __shared__ Bins found;
  __shared__ uint32_t told, listed;
  const int tid = (int)threadIdx.x, lane = tid & 63, piece = (int)(blockIdx.x % (uint32_t)a.pieces);
  const int64_t b = blockIdx.x / (uint32_t)a.pieces;
  const Row r = row_of<T>(a, b);
  Piece own = {-INFINITY, 0.f, 0, 0.f, 0};
  if (lane < a.pieces) own = a.piece[b * a.pieces + lane];
  const float top_lane = r.cuts && lane < kTops ? a.tops[(b * a.pieces + piece) * kTops + lane] : 0.f;
  float m = own.m;
  for (int p = 64 + lane; p < a.pieces; p += 64) m = __builtin_elementwise_maximum(m, a.piece[b * a.pieces + p].m);
  m = maximum_across(m);
  const bool alive = m > -INFINITY && m < INFINITY;
  if (piece > 0 && !(alive && r.filtered())) return;
  if (!alive) {
    if (tid == 0) a.tokens[b] = -1, a.logprobs[b] = 0.f;
    return;
  }
  if (!r.filtered()) {
    // the pieces' races, joined
    if (tid >= 64) return;
    uint64_t best = 0;
    float z = 0.f, l = 0.f;
    for (int p = lane; p < a.pieces; p += 64) {
      const Piece y = a.piece[b * a.pieces + p];
      const float f = y.m > -INFINITY ? __builtin_amdgcn_exp2f((y.m - m) * r.c) : 0.f;
      z += y.z * f;
      // A piece's best runs again relative to the row's largest logit: equals of different pieces stay equal, which scores of
      // the pieces times their factors would not be in the last bit.
      const int t = (int)~(uint32_t)y.best;
      float score = y.m == m ? 1.f : 0.f;
      if (!r.greedy && y.best) score = __builtin_amdgcn_exp2f((y.l - m) * r.c) * __builtin_amdgcn_rcpf(r.noise[t]);
      const uint64_t key = y.best ? race_key(score, t) : 0;
      l = key > best ? y.l : l;
      best = max(best, key);
    }
    const uint64_t all = max_across(best);
    z = sum_across(z);
    if (all ? best == all : lane == 0) write_token(a, r, b, all, l, m, z);
    return;
  }
  const float top = __builtin_floorf(place(m, r.c));
  Bins f = no_cuts();
  bool whole = false;
  if (r.cuts) {
    // bins are whole numbers that a float tells apart
    whole = !(__builtin_fabsf(top) < 4194304.f);
    if (whole && piece > 0) return;
  }
  if (!whole) {
    if (tid == 0) listed = 0;
    if (r.cuts)
      f = bins_of(a, r, b, top, own, sh, found);
    else
      __syncthreads();
    // The piece's tokens: kept, on the list, or neither; a wave's steps that lie below the cuts are not
    // read.  Bins are told by the places of their edges.
    const int lowest = max(f.sure - 1, max(f.k < kBins ? f.k : -1, f.p_to));
    const float sure = top - (float)f.sure + 1.f, end = top - (float)lowest;  // kept from the one on, listed from the other on
    const float p_end = top - (float)f.p_to, k_begin = top - (float)f.k + 1.f;  // but between the cuts nothing is
    Race race = {0.f, 0.f, 0.f, 0};
    constexpr int kAhead = 2;  // steps that are asked for together
    uint32_t ask = (1u << a.steps) - 1;
    if (r.cuts)
      for (int s = 0; s < kHeld; ++s) {
        const float highest = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(top_lane), s * kWaves + (tid >> 6)));
        if (!(place(highest, r.c) >= end)) ask &= ~(1u << s);
      }
    while (ask) {
      int step[kAhead];
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        step[s] = ask ? __builtin_ctz(ask) : -1;
        ask &= ask - 1;
      }
      Eight e[kAhead];
      Raw<T> x[kAhead];
      uint32_t kept[kAhead], open[kAhead];
      float n[kAhead][8];
#pragma unroll
      for (int s = 0; s < kAhead; ++s)
        e[s] = step[s] >= 0 ? eight_of(a, r, (piece * a.steps + step[s]) * kStep + tid * 8) : Eight{0, 0};
#pragma unroll
      for (int s = 0; s < kAhead; ++s)
        if (step[s] >= 0) load_eight(a, r, e[s], x[s]);
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        kept[s] = e[s].bits;
        open[s] = 0;
        if (!r.cuts) continue;
        uint32_t first = 0, some = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float at = place(x[s].at(i), r.c);
          first |= (uint32_t)(at >= sure) << i;
          some |= (uint32_t)(at >= end && (at >= p_end || at < k_begin)) << i;
        }
        kept[s] = first & e[s].bits;
        open[s] = some & ~first & e[s].bits;
      }
#pragma unroll
      for (int s = 0; s < kAhead; ++s)
        if (kept[s]) load_noise(a, r, e[s], n[s]);
#pragma unroll
      for (int s = 0; s < kAhead; ++s)
        for (uint32_t left = open[s]; left; left &= left - 1) {
          const int i = __builtin_ctz(left);
          const uint32_t at = atomicAdd(&listed, 1u);
          float l = 0.f;
#pragma unroll
          for (int k = 0; k < 8; ++k) l = k == i ? x[s].at(k) : l;
          if (at < (uint32_t)a.room) held[at] = (uint64_t)key_of(l) << 32 | (uint32_t)~(e[s].from + i);
        }
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        if (!__any(kept[s] != 0)) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (kept[s] >> i & 1) race.take(x[s].at(i), (x[s].at(i) - m) * r.c, n[s][i], r.low, e[s].from + i);
      }
    }
    const uint64_t mine = race.key();
    const float l_best = race.l;
    float z = race.z;
    z = block_sum(sh, z);
    const uint64_t best = block_best(sh, mine);
    const int64_t at = b * a.pieces + piece;
    if (best ? mine == best : tid == 0) {
      __hip_atomic_store(&a.left[at].best, best, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&a.left[at].l_z, (uint64_t)__float_as_uint(l_best) << 32 | __float_as_uint(z), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&a.left[at].listed, (uint64_t)listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    for (uint32_t i = (uint32_t)tid; i < min(listed, (uint32_t)a.room); i += kThreads)
      __hip_atomic_store(a.list + at * a.room + i, held[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // All that passes between the workgroups goes by atomics at the device's point of coherence, and is done before the count.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) told = __hip_atomic_fetch_add(a.done + b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (told != (uint32_t)a.pieces - 1) return;
    // The last of the row's workgroups: what all of them left, in every wave.
    uint64_t others = 0, n = 0, over = 0;
    float l = 0.f;
    z = 0.f;
    for (int p0 = 0; p0 < a.pieces; p0 += 64) {
      Left y = {0, 0, 0};
      if (p0 + lane < a.pieces) {
        const Left* from = a.left + b * a.pieces + p0 + lane;
        y.best = __hip_atomic_load(&from->best, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        y.l_z = __hip_atomic_load(&from->l_z, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        y.listed = __hip_atomic_load(&from->listed, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      l = y.best > others ? __uint_as_float((uint32_t)(y.l_z >> 32)) : l;
      others = max(others, y.best);
      z += __uint_as_float((uint32_t)y.l_z);
      over |= y.listed > (uint64_t)a.room;
      // the entries, one piece's after the other's
      const uint64_t upto = sum_upto(y.listed), here = lane_of(upto, 63);
      if (!__any(over != 0) && n + here <= Listed::kHeldList)
        for (int p = tid >> 6; p < min(64, a.pieces - p0); p += kWaves) {
          const uint32_t have = (uint32_t)lane_of(y.listed, p), to = (uint32_t)(n + lane_of(upto, p)) - have;
          for (uint32_t i = (uint32_t)lane; i < have; i += 64)
            held[to + i] = __hip_atomic_load(a.list + (b * a.pieces + p0 + p) * a.room + i, __ATOMIC_RELAXED,
                                             __HIP_MEMORY_SCOPE_AGENT);
        }
      n += here;
    }
    if (!__any(over != 0)) {
      const uint64_t first = max_across(others);
      const uint64_t owner = __ballot(others == first);
      l = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(l), __builtin_ctzll(owner)));
      z = sum_across(z);
      __syncthreads();
      const Listed x = {a, r, sh, digits, held, f, b, m, top, (uint32_t)n, Listed::shift_of((uint32_t)n)};
      uint64_t best = 0, mass = 0;
      float l_listed = 0.f;
      if (n <= Listed::kAlone && tid >= 64) return;
      if (n <= 64)
        mass = x.by_count<1>(sh.count, best, l_listed);
      else if (n <= 128)
        mass = x.by_count<2>(sh.count, best, l_listed);
      else
        mass = x.by_digits(best, l_listed);
      if (tid > 0) return;
      // (where nothing is listed the edge may be out of all bounds)
      if (mass)
        z += (float)((double)mass * __builtin_ldexp(1.0, -x.shift)) * __builtin_amdgcn_exp2f(__builtin_fmaf(-m, r.c, x.edge()));
      if (best > first)
        write_token(a, r, b, best, l_listed, m, z);
      else
        write_token(a, r, b, first, l, m, z);
      return;
    }
  }
  whole_row<T>(a, r, sh, b, m);
}

// The launches.  Rows are cut into pieces so that there are about 320 workgroups, none of less than two steps unless the row is
// shorter, and none of more than registers hold (512, 640 and 1024 workgroups, what runs at once and more, were within 2 us:
// each piece more is a histogram more).  So many rows share a pair of launches that the workspace stays below 256 MiB, or
// is one row's.
struct Plan {
  int pieces, steps, room, rows;
  size_t row_bytes;
};
Plan plan(int32_t B, int32_t V) {
  Plan p;
  const int64_t all = ((int64_t)V + kStep - 1) / kStep, fill = (320 + B - 1) / B;
  const int64_t pieces = std::max((all + kHeld - 1) / kHeld, std::min(fill, (all + 1) / 2));
  p.steps = (int)((all + pieces - 1) / pieces);
  p.pieces = (int)((all + p.steps - 1) / p.steps);
  p.room = std::min(V, kList);
  p.row_bytes = (size_t)p.pieces * (kBins * 8 + (size_t)p.room * 8 + sizeof(Left) + sizeof(Piece) + kTops * 4) + 8;
  p.rows = (int)std::max<size_t>(1, std::min<size_t>((size_t)B, ((size_t)1 << 28) / p.row_bytes));
  return p;
}
size_t bytes_of(const Plan& p) { return (size_t)p.rows * p.row_bytes + 16; }
bool sizes_ok(int32_t B, int32_t V) { return B >= 1 && B <= 1 << 20 && V >= 1 && V <= (1 << 30) - 2048; }

}  // namespace

extern "C" size_t grid_sample_workspace_bytes(int32_t B, int32_t V) {
  if (!sizes_ok(B, V)) return 0;
  return bytes_of(plan(B, V));
}

extern "C" int grid_sample(const grid_sample_args* args, void* stream) {
  clear_error();
  auto bad = [](const char* what) { return fail(GRID_E_ARG, std::string("grid_sample: ") + what); };
  if (!args) return bad("null argument");
  const grid_sample_args& g = *args;
  if (!sizes_ok(g.B, g.V)) return bad("sizes");
  if (g.dtype != GRID_DTYPE_F32 && g.dtype != GRID_DTYPE_BF16 && g.dtype != GRID_DTYPE_F16) return bad("dtype");
  if (!g.logits || !g.tokens || !g.logprobs) return bad("null pointer");
  if (g.logits_stride < 0 || g.mask_stride < 0 || g.noise_stride < 0) return bad("negative stride");
  const Plan p = plan(g.B, g.V);
  if (!g.workspace || (uintptr_t)g.workspace % 16 != 0 || g.workspace_bytes < bytes_of(p))
    return bad("workspace too small or not aligned");
  SampleArgs a;
  a.ls = g.logits_stride;
  a.ms = g.mask_stride;
  a.ns = g.noise_stride;
  a.V = g.V;
  a.pieces = p.pieces;
  a.steps = p.steps;
  a.room = p.room;
  a.count_bits = 1;
  while ((int64_t)1 << a.count_bits <= (int64_t)p.steps * kStep) ++a.count_bits;
  a.mass_shift = std::min(30, 62 - 2 * a.count_bits);
  a.shift = 46;
  while ((uint64_t)g.V > (uint64_t)1 << (62 - a.shift)) --a.shift;
  const size_t all = (size_t)p.rows * (size_t)p.pieces;
  a.hist = (uint64_t*)g.workspace;
  a.list = a.hist + all * kBins;
  a.left = (Left*)(a.list + all * (size_t)p.room);
  a.piece = (Piece*)(a.left + all);
  a.tops = (float*)(a.piece + all);
  a.done = (uint32_t*)(a.tops + all * kTops);
  const hipStream_t s = (hipStream_t)stream;
  for (int32_t b = 0; b < g.B; b += p.rows) {
    const int32_t rows = std::min(p.rows, g.B - b);
    const auto go = [&](auto type) {
      using T = decltype(type);
      a.logits = (const T*)g.logits + b * g.logits_stride;
      a.mask = g.mask ? g.mask + b * g.mask_stride : nullptr;
      a.noise = g.noise ? g.noise + b * g.noise_stride : nullptr;
      a.temperature = g.temperature ? g.temperature + b : nullptr;
      a.top_k = g.top_k ? g.top_k + b : nullptr;
      a.top_p = g.top_p ? g.top_p + b : nullptr;
      a.min_p = g.min_p ? g.min_p + b : nullptr;
      a.tokens = g.tokens + b;
      a.logprobs = g.logprobs + b;
      const dim3 blocks((unsigned)rows * (unsigned)p.pieces);
      hipLaunchKernelGGL(pieces_kernel<T>, blocks, dim3(kThreads), 0, s, a);
      hipLaunchKernelGGL(draw_kernel<T>, blocks, dim3(kThreads), 0, s, a);
    };
    if (g.dtype == GRID_DTYPE_F32)
      go(float());
    else if (g.dtype == GRID_DTYPE_BF16)
      go(bf16_t());
    else
      go(f16_t());
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_sample launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
