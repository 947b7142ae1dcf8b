// attend.hip -- grid_attend: attention of a chunk of new tokens over a paged cache (gfx950).
//
// The query heads that share a key head, at all tokens of a chunk, are rows of one matrix (row = token * group + head
// in the group), so a key or value is read once for all of them, whether a chunk is one token or a prompt.  A
// workgroup takes a tile of rows and a range of keys; it streams stages of keys and values from their pages into LDS,
// directly and two deep, and goes over them once with the running maximum and sum of the softmax.
//
// Matrix instructions (32 x 32 x 16) compute S^T = K Q^T: a lane then holds one query row's scores for 16 of 32 keys,
// its row's maximum and sum are the lane's own but for one exchange between the wave's halves, and its weights, rounded
// and packed, are in place as the second operand of O^T += V^T P^T: that product adds over keys in any order, so V's
// rows are read, transposed on the way from LDS, in the order the scores lie in.
//
// Bounds (bf16, heads of 128; a copy reaches 5.09 TB/s here, a product of 8192^3 1392 TFLOP/s).  Few rows read the cache
// once: 64 sequences of up to 8192 keys, 8 key heads, one token each, take 183 us, 4.9 TB/s of it; 32 of up to 4096, 4 key
// heads, up to 5 tokens, 44 us, 3.1 TB/s (35 the shares, 8 stages each, 5 the joining); one of 1500 keys 11 us, two launches
// of dependent reads.  Prompts are bound by the vector and matrix units together, which hardly overlap here (43 % and 42 %
// busy): 2 chunks of 2048 tokens after 4096, 28 heads on 4, take 318 us, 945 TFLOP/s, batches of 16 of them 1026; 4 of
// heads of 64, 16 on 16, 222 us, 774 (vector units 52 %, matrix units 34 %); 4 of heads of 256, 8 on 1, 395 us, 870.  So the
// weights' exponentials, sums and roundings are nearly all that is left of the vector instructions in a stage, and
// scores a stage ahead of the sums, their instructions woven into the weights', are slower for the registers they need.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "lanes.h"
#include "paged.h"

using namespace grid;

namespace {

typedef float float16_v __attribute__((ext_vector_type(16)));
typedef short short4_v __attribute__((ext_vector_type(4)));

template <typename T>
struct Vec;
template <>
struct Vec<bf16_t> {
  typedef __bf16 two __attribute__((ext_vector_type(2)));
  typedef __bf16 eight __attribute__((ext_vector_type(8)));
  static constexpr uint32_t kExp = 0x7F807F80u, kOne = 0x00800080u;  // exponents of a pair; their lowest bits
  static __device__ float16_v mfma(eight a, eight b, float16_v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Vec<f16_t> {
  typedef _Float16 two __attribute__((ext_vector_type(2)));
  typedef _Float16 eight __attribute__((ext_vector_type(8)));
  static constexpr uint32_t kExp = 0x7C007C00u, kOne = 0x04000400u;
  static __device__ float16_v mfma(eight a, eight b, float16_v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};

struct AttendArgs {
  const uint16_t* q;
  uint16_t* out;
  uint32_t qs[2], os[2];  // token, head
  float* lse;
  float2* part_ml;  // [slots][rows of a tile]: maximum (in base 2 units of the scaled score), sum
  float* part_o;    // [slots][rows of a tile][D], not divided by the sum
  int2* runs;       // [sequences][key heads]: first and last workgroup of the unit (few rows)
  Divisor group;
  int32_t hq, max_q, max_kv, window;
  // many rows: workgroups; tiles a sequence and key head, ranges of len keys (whole stages); units side by side (kPacked)
  int32_t blocks, tiles, splits, len, bundle;
  float c;                     // |scale| * log2 e, above 0
  bool negate;                 // scale < 0: the queries are negated

  static __device__ uint64_t at(const uint32_t* stride, int t, int h) {
    return (uint64_t)t * stride[0] + (uint64_t)h * stride[1];
  }
};

constexpr int kPacked = -1;

constexpr float kLn2 = 0.693147180559945309417f, kLog2e = 1.44269504088896340736f;

// First key that a sequence's rows are given: the window of its first new token, down to a whole stage of 128.
__device__ inline int first_key(const AttendArgs& a, const Chunk& c) {
  return a.window ? max(0, c.kv - c.n - a.window + 1) & ~127 : 0;
}

__device__ inline bool is_bad(const AttendArgs& a, const Chunk& c) { return !c.ok || c.n > a.max_q || c.kv > a.max_kv; }

__device__ inline float other_half(float x) {  // the value of lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return (threadIdx.x & 32) ? __uint_as_float(r[0]) : __uint_as_float(r[1]);
}

// 16 bytes a lane from global memory (uniform base + the lane's offset in bytes) to LDS at `to` + 16 * lane (to:
// uniform, bytes from the start of LDS).  Written as assembly because the compiler waits for all such loads before any
// LDS read; they are counted by vmcnt.  LDS reads issued before are waited for first: they may be of what is overwritten.
// The compiler counts no wait states in here: a load into LDS needs one after the write of M0.
// (M0 is among the registers that the compiler allots to nothing, which it remarks on.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void to_lds(const void* base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(to)
               : "memory", "m0");
}
__device__ inline void to_lds(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N>  // until at most the last N are under way
__device__ inline void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ inline void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

#define GRID_LDS __attribute__((address_space(3)))

// The swizzle: 16-byte piece c of a row of keys or values lies at piece c ^ swz(row), so that the 32 rows of one piece
// (K's operand) and 4 rows of 64 bytes (V's, transposed) lie in different banks.
template <int D>
__device__ constexpr int swz(int row) {
  return D == 64 ? ((row >> 1 & 1) << 2 | (row >> 2 & 3)) : ((row & 3) << 2 | (row >> 2 & 3));
}

// What a workgroup notes in LDS on its way: the keys whose values were cleaned (first, and after the last), whether a page
// was not in the cache, and whether the sequence is bad for a chunk before it.
__device__ inline void no_fix(int* fix) {
  if (threadIdx.x == 0) {
    fix[0] = INT32_MAX;
    fix[1] = 0;
    fix[2] = 0;
    fix[3] = 0;
  }
}
struct Nothing {
  __device__ void operator()() const {}
};

// RW x KW waves: RW * 32 rows, stages of KW * KT keys of which a wave takes KT.
//  - RW == 1: a wave loads its own keys and waits for nobody.  One stage is held; the next keys are fetched when the
//    scores have been computed, the next values when the sums have, so loads are in flight all the time.
//  - RW > 1: the waves share the stages; two are held, the next one is fetched while one is worked on.
// UNI: pages hold whole runs of 16 rows, so the address of a load is a scalar and an offset of the lane.
template <typename T, int D_, int RW_, int KW_, int KT_, int WGS_, bool UNI_>
struct Tile {
  static constexpr int D = D_, RW = RW_, KW = KW_, KT = KT_, WGS = WGS_;
  static constexpr bool UNI = UNI_, PRIV = RW == 1;
  static constexpr int W = RW * KW, NT = 64 * W, TM = 32 * RW, SK = KW * KT;
  static constexpr int PR = D / 8;            // 16-byte pieces of a row
  static constexpr int RPI = 64 / PR;         // rows that one load instruction brings
  static constexpr int WR = SK / W;           // rows that a wave brings: of the keys, as many of the values
  static constexpr int LOADS = WR / RPI;      // load instructions for them
  static constexpr int RUN = WR < 16 ? WR : 16, RUNS = WR / RUN;  // rows that share a page lookup
  static constexpr int KB = KT / 32, DB = D / 32, QS = D / 16;
  static constexpr uint32_t kHalf = SK * D * 2;  // bytes of a stage's keys
  static constexpr uint32_t kStages = (PRIV ? 1 : 2) * 2 * kHalf;
  static constexpr uint32_t kMerge = KW == 1 ? 0 : KW * TM * (2 + D / 2 + 4) * 4;  // what waves of other keys meet in
  static constexpr uint32_t kLds = kStages > kMerge ? kStages : kMerge;
  typedef typename Vec<T>::eight Eight;
  static_assert(WR % RPI == 0 && 128 % SK == 0 && KT % 32 == 0, "");

  // One sequence's key head, one tile of rows, the keys s_lo .. s_hi - 1 (s_lo a multiple of the stage).  whole: these
  // are all the keys the rows see, the result is written; otherwise the sums go to slot `slot`.  fix: in LDS, no_fix()
  // for all to see; so is it for the next call after a barrier and no_fix().  meanwhile: what all threads do while the
  // first pages are looked up; they may find that the sequence is bad (fix[3]), and nothing is written.
  template <typename F>
  static __device__ __forceinline__ void run(const Paged& P, const AttendArgs& a, uint8_t* lds, int* fix, const Chunk& ch,
                                             int b, int g, int tile, int s_lo, int s_hi, bool whole, int64_t slot,
                                             F meanwhile);
};

template <typename T, int D_, int RW_, int KW_, int KT_, int WGS_, bool UNI_>
template <typename F>
__device__ __forceinline__ void Tile<T, D_, RW_, KW_, KT_, WGS_, UNI_>::run(const Paged& P, const AttendArgs& a,
                                                                            uint8_t* lds, int* fix, const Chunk& ch,
                                                                            int b, int g, int tile, int s_lo, int s_hi,
                                                                            bool whole, int64_t slot, F meanwhile) {
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW, half = lane >> 5, col = lane & 31;
  const int G = (int)a.group.d, rows = ch.n * G, first_pos = ch.kv - ch.n;

  // this wave's rows: lane's query, its position, the wave's range of positions
  const int r0 = tile * TM + rw * 32, r = min(r0 + col, rows - 1);
  const bool alive = r0 < rows;
  const int qi = (int)a.group.quot((uint32_t)r), qh = g * G + r - qi * G, qt = ch.first + qi, pos = first_pos + qi;
  const int pos_min = first_pos + (int)a.group.quot((uint32_t)min(r0, rows - 1));
  const int pos_max = first_pos + (int)a.group.quot((uint32_t)min(r0 + 31, rows - 1));

  // Loads.  Load i of a wave brings RPI rows from row WR * wave + i * RPI of the stage on, a lane piece `lane % PR` of
  // row `lane / PR`.  At and after s_hi come rows that the same page holds, or the last ones again, and before s_seen, the
  // first key that a row of the tile sees, page 0 where the table has no page: nothing is made of them, whatever they hold.
  const uint32_t base = (uint32_t)(uintptr_t)(GRID_LDS uint8_t*)lds;
  const uint16_t *kg = P.k + (uint64_t)g * P.ks[2], *vg = P.v + (uint64_t)g * P.vs[2];
  const auto* table = (const __attribute__((address_space(4))) int32_t*)(P.table + (int64_t)b * P.table_stride);
  const int lrow = lane / PR;
  constexpr int FIND = UNI ? RUNS : LOADS;
  int32_t page[FIND];
  uint32_t row[FIND];
  bool missing = false;
  const int s_seen = a.window ? first_pos + (int)a.group.quot((uint32_t)(tile * TM)) - a.window + 1 : 0;
  const auto find = [&](int s0) {
    const auto key = [&](int i) {
      const int s = s0 + wave * WR + (UNI ? i * RUN : i * RPI + lrow);
      return UNI ? min(s, (s_hi - 1) & ~(RUN - 1)) : min(s, s_hi - 1);
    };
#pragma unroll
    for (int i = 0; i < FIND; ++i) {
      const uint32_t at = (uint32_t)key(i), c = P.page.quot(at);
      row[i] = at - c * P.page.d;
      page[i] = table[c];
    }
#pragma unroll
    for (int i = 0; i < FIND; ++i) {
      const bool in = P.in_cache(page[i]);
      missing |= !in && key(i) + (UNI ? RUN : 1) > s_seen;
      page[i] = in ? page[i] : 0;
    }
  };
  const auto fetch = [&](const uint16_t* x, const uint32_t* st, uint32_t to) {
    to += (uint32_t)(wave * WR * D * 2);
    const uint32_t step = lrow * st[1];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int piece = lane % PR ^ swz<D>(wave * WR + i * RPI + lrow);
      if constexpr (UNI) {
        constexpr int PER = RUN / RPI;
        // (scalars, whatever registers they were kept in)
        const int pg = __builtin_amdgcn_readfirstlane(page[i / PER]);
        const uint32_t r = (uint32_t)__builtin_amdgcn_readfirstlane((int)row[i / PER]);
        to_lds(x + P.at(st, pg, r + (uint32_t)(i % PER * RPI)), (step + piece * 8) * 2, to + i * 1024);
      } else {
        to_lds(x + P.at(st, page[i], row[i]) + piece * 8, to + i * 1024);
      }
    }
  };

  Eight q[QS];
  const auto load_q = [&] {
    const uint16_t* src = a.q + a.at(a.qs, qt, qh) + half * 8;
    const uint32_t flip = a.negate ? 0x80008000u : 0u;
#pragma unroll
    for (int k = 0; k < QS; ++k) {
      uint4 x = *(const uint4*)(src + k * 16);
      x.x ^= flip, x.y ^= flip, x.z ^= flip, x.w ^= flip;
      q[k] = __builtin_bit_cast(Eight, x);
    }
  };

  float16_v o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -INFINITY, l = 0.f;

  // S^T of the wave's keys
  float16_v s[KB];
  const auto scores = [&](const uint8_t* ks) {
    // Piece 2 k + half of the row, at its place: the bits of k by exclusive or, which is one instruction with the sum.
    int at = col * D * 2 + (half ^ swz<D>(col)) * 16;
    asm volatile("" : "+v"(at));  // anew every time: registers are short
    constexpr int N = QS * KB, AHEAD = 6;
    Eight kk[N];
    const auto read = [&](int j) { kk[j] = *(const Eight*)(ks + (at ^ j / KB * 32) + j % KB * 32 * D * 2); };
#pragma unroll
    for (int j = 0; j < AHEAD && j < N; ++j) read(j);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (j + AHEAD < N) read(j + AHEAD);
      s[j % KB] = Vec<T>::mfma(kk[j], q[j / KB], s[j % KB]);
      if constexpr (!PRIV) __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto mask = [&](int k0) {
    // the lane's keys are k0 + 4 * half and constants more
    const int from = k0 + 4 * half, hi = min(pos, s_hi - 1) - from, lo = (a.window ? pos - a.window : -1) - from;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = kb * 32 + 8 * (i / 4) + i % 4;
        s[kb][i] = key <= hi && key > lo ? s[kb][i] : -INFINITY;
      }
  };
  // Values that are not finite must not meet a weight of 0 in a product.  In stages where some row does not see some
  // key they are taken out, by the wave that loaded them, and added at the end to the rows that see them (settle).
  const auto clean = [&](uint32_t at, int s0) {
    uint4* mine = (uint4*)(lds + (at - base) + wave * WR * D * 2 + lane * 16);
    uint32_t found = 0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const uint4 x = mine[i * 64];
      found |= (x.x & Vec<T>::kExp) + Vec<T>::kOne;
      found |= (x.y & Vec<T>::kExp) + Vec<T>::kOne;
      found |= (x.z & Vec<T>::kExp) + Vec<T>::kOne;
      found |= (x.w & Vec<T>::kExp) + Vec<T>::kOne;
    }
    if (__any((found & 0x80008000u) != 0)) {
      for (int i = 0; i < LOADS * 4; ++i) {
        uint32_t* x = (uint32_t*)(mine + i / 4 * 64) + i % 4;
        const uint32_t e = (*x & Vec<T>::kExp) + Vec<T>::kOne;
        *x &= (e & 0x8000u ? 0u : 0xFFFFu) | (e & 0x80000000u ? 0u : 0xFFFF0000u);
      }
      if (lane == 0) {
        atomicMin(&fix[0], s0 + wave * WR);
        atomicMax(&fix[1], s0 + (wave + 1) * WR);
      }
    }
  };
  const auto masked = [&](int k0) {
    return k0 + KT - 1 > pos_min || k0 + KT > s_hi || (a.window && k0 <= pos_max - a.window);
  };
  const auto softmax = [&] {
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
    top = fmaxf(top, other_half(top));
    // The reference of the exponents follows the maximum only when it grows by more than 8 in base 2: weights stay
    // below 2^8, and most stages need no rescaling.
    if (__any(top > m && !((top - m) * a.c <= 8.f))) {
      const float now = fmaxf(m, top), ref = now == -INFINITY ? 0.f : now;
      const float keep = __builtin_amdgcn_exp2f((m - ref) * a.c);
      l *= keep;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= keep;
      m = now;
    }
    const float mc = (m == -INFINITY ? 0.f : m) * a.c;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][i], a.c, -mc));
        l += s[kb][i];
      }
  };
  const auto sums = [&](const uint8_t* vs) {
    // V's operand: entry d * 32 + col of 8 keys, in the order the scores lie in.  A lane reads of rows
    // 16 t + 8 j + rr the pieces 4 d + piece, at their places.
    const int l16 = lane & 15, rr = 4 * half + (l16 >> 2), piece = (lane >> 4 & 1) * 2 + (l16 >> 1 & 1);
    int at = rr * D * 2 + (piece ^ swz<D>(rr)) * 16 + (l16 & 1) * 8;
    asm volatile("" : "+v"(at));
#pragma unroll
    for (int t = 0; t < KT / 16; ++t) {
      Eight p;
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = (T)s[t / 2][t % 2 * 8 + i];
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        union {
          short4_v four[2];
          Eight all;
        } v;
#pragma unroll
        for (int j = 0; j < 2; ++j)  // (the swizzle of a row 8 on differs by 2)
          v.four[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (GRID_LDS short4_v*)(vs + (at ^ (d * 4 ^ j * 2) * 16) + (16 * t + 8 * j) * D * 2));
        o[d] = Vec<T>::mfma(v.all, p, o[d]);
      }
    }
  };

  if constexpr (PRIV) {
    const uint8_t *ks = lds + kw * KT * D * 2, *vs = ks + kHalf;
    const bool any = s_lo + kw * KT < s_hi;
    if (any) find(s_lo);
    meanwhile();
    if (any) {
      fetch(kg, P.ks, base);
      fetch(vg, P.vs, base + kHalf);
      load_q();
    }
    for (int s0 = s_lo; s0 + kw * KT < s_hi; s0 += SK) {
      const int k0 = s0 + kw * KT;
      const bool more = k0 + SK < s_hi;
      if (more) find(s0 + SK);
      wait_loads<LOADS>();
      scores(ks);
      wait_reads();
      if (more) {
        fetch(kg, P.ks, base);
        wait_loads<LOADS>();
      } else {
        wait_loads<0>();
      }
      if (masked(k0)) {
        mask(k0);
        clean(base + kHalf, s0);
      }
      softmax();
      sums(vs);
      wait_reads();
      if (more) fetch(vg, P.vs, base + kHalf);
    }
  } else {
    find(s_lo);
    meanwhile();
    fetch(kg, P.ks, base);
    fetch(vg, P.vs, base + kHalf);
    load_q();
    if (s_lo + SK < s_hi) find(s_lo + SK);
    // stages that some row of the tile does not see all of
    const int tile_min = first_pos + (int)a.group.quot((uint32_t)(tile * TM));
    const int tile_max = first_pos + (int)a.group.quot((uint32_t)min(tile * TM + TM, rows) - 1u);
    const auto torn = [&](int s0) {
      return s0 + SK - 1 > tile_min || s0 + SK > s_hi || (a.window && s0 <= tile_max - a.window);
    };
    wait_loads<0>();
    if (torn(s_lo)) clean(base + kHalf, s_lo);
    __syncthreads();
    uint32_t buf = 0;
    for (int s0 = s_lo; s0 < s_hi; s0 += SK) {
      if (s0 + SK < s_hi) {
        fetch(kg, P.ks, base + (buf ^ 2 * kHalf));
        fetch(vg, P.vs, base + (buf ^ 2 * kHalf) + kHalf);
        if (s0 + 2 * SK < s_hi) find(s0 + 2 * SK);
      }
      const int k0 = s0 + kw * KT;
      if (alive && k0 < s_hi && k0 <= pos_max && (!a.window || k0 + KT > pos_min - a.window + 1)) {
        const uint8_t *ks = lds + buf + kw * KT * D * 2, *vs = ks + kHalf;
        scores(ks);
        if (masked(k0)) mask(k0);
        softmax();
        sums(vs);
      }
      buf ^= 2 * kHalf;
      wait_reads();
      wait_loads<0>();
      if (s0 + SK < s_hi && torn(s0 + SK)) clean(base + buf + kHalf, s0 + SK);
      __syncthreads();
    }
  }
  l += other_half(l);
  if (missing) fix[2] = 1;
  __syncthreads();
  if constexpr (!std::is_same<F, Nothing>::value)
    if (fix[3]) return;
  if (fix[2]) l = NAN;
  float mc = m * a.c;  // -inf where the row saw nothing

  // adds to four sums of the row at position p the values that were taken out and that it sees
  const int fix_lo = fix[0], fix_hi = min(fix[1], s_hi);
  const auto settle = [&](float4& x, int p, int e) {
    if (fix_lo >= fix_hi) return;
    for (int s = max(fix_lo, a.window ? p - a.window + 1 : 0); s < min(fix_hi, p + 1); ++s) {
      uint32_t rr;
      const int id = P.page_of(b, (uint32_t)s, rr);
      if (!P.in_cache(id)) continue;
      T y[4];
      __builtin_memcpy(y, vg + P.at(P.vs, id, rr) + e, 8);
      const float f[4] = {(float)y[0], (float)y[1], (float)y[2], (float)y[3]};
      x.x += __builtin_isfinite(f[0]) ? 0.f : f[0];
      x.y += __builtin_isfinite(f[1]) ? 0.f : f[1];
      x.z += __builtin_isfinite(f[2]) ? 0.f : f[2];
      x.w += __builtin_isfinite(f[3]) ? 0.f : f[3];
    }
  };

  // waves that took other keys of the same rows: their sums meet in LDS
  if constexpr (KW > 1) {
    constexpr int DH = D / 2;                     // in two halves of the entries, for room
    float2* ml = (float2*)lds;                    // [KW][TM]
    float* os = (float*)(lds + KW * 2 * TM * 4);  // [KW][TM][DH + 4]
    if (half == 0) ml[kw * TM + rw * 32 + col] = make_float2(mc, l);
    float* mine = os + (kw * TM + rw * 32 + col) * (DH + 4);
    constexpr int PART = 32 * DH / 4 / 64 / KW;  // float4s a lane
#pragma unroll
    for (int hd = 0; hd < 2; ++hd) {
      if (hd > 0) __syncthreads();
#pragma unroll
      for (int d = 0; d < DB / 2; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float16_v& x = o[hd * (DB / 2) + d];
          *(float4*)(mine + d * 32 + 2 * i + 4 * half) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        }
      __syncthreads();
      // a wave adds up a part of its rows' entries
#pragma unroll
      for (int j = 0; j < PART; ++j) {
        const int at = (j * KW + kw) * 64 + lane, rr = rw * 32 + at / (DH / 4), e = at % (DH / 4) * 4;
        if (tile * TM + rr >= rows) continue;
        float rm = -INFINITY, rl = 0.f;
#pragma unroll
        for (int w = 0; w < KW; ++w) rm = fmaxf(rm, ml[w * TM + rr].x);
        const float ref = rm == -INFINITY ? 0.f : rm;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          const float2 p = ml[w * TM + rr];
          const float f = __builtin_amdgcn_exp2f(p.x - ref);
          const float4 y = *(const float4*)(os + (w * TM + rr) * (DH + 4) + e);
          rl += p.y * f;
          x.x += y.x * f, x.y += y.y * f, x.z += y.z * f, x.w += y.w * f;
        }
        const int i = (int)a.group.quot((uint32_t)(tile * TM + rr)), h = g * G + tile * TM + rr - i * G, t = ch.first + i;
        settle(x, first_pos + i, hd * DH + e);
        if (whole) {
          const float over = rl == 0.f ? 0.f : 1.f / rl;
          T y[4] = {(T)(x.x * over), (T)(x.y * over), (T)(x.z * over), (T)(x.w * over)};
          *(uint2*)(a.out + a.at(a.os, t, h) + hd * DH + e) = *(uint2*)y;
          if (a.lse && e == 0 && hd == 0) a.lse[(int64_t)t * a.hq + h] = (rm + __builtin_amdgcn_logf(rl)) * kLn2;
        } else {
          *(float4*)(a.part_o + (slot * TM + rr) * D + hd * DH + e) = x;
          if (e == 0 && hd == 0) a.part_ml[slot * TM + rr] = make_float2(rm, rl);
        }
      }
    }
  } else {
    if (r0 + col >= rows) return;
    if (whole) {
      const float over = l == 0.f ? 0.f : 1.f / l;
      uint16_t* dst = a.out + a.at(a.os, qt, qh) + 4 * half;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          float4 x = make_float4(o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]);
          settle(x, pos, d * 32 + 2 * i + 4 * half);
          T y[4] = {(T)(x.x * over), (T)(x.y * over), (T)(x.z * over), (T)(x.w * over)};
          *(uint2*)(dst + d * 32 + 2 * i) = *(uint2*)y;
        }
      if (a.lse && half == 0) a.lse[(int64_t)qt * a.hq + qh] = (mc + __builtin_amdgcn_logf(l)) * kLn2;
    } else {
      const int64_t at = slot * TM + rw * 32 + col;
      float* dst = a.part_o + at * D + 4 * half;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          {
          float4 x = make_float4(o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]);
          settle(x, pos, d * 32 + 2 * i + 4 * half);
          *(float4*)(dst + d * 32 + 2 * i) = x;
          }
      if (half == 0) a.part_ml[at] = make_float2(mc, l);
    }
  }
}

// The rows of a bad sequence, of the first whose chunk is not in order all that follow: those after it are bad too.
template <typename T, int D>
__device__ void fill_nan(const Paged& P, const AttendArgs& a, const Chunk& ch, int b, int nt) {
  const int32_t end = P.cu_q[b + 1];
  const int from = min(max(ch.first, 0), P.T), to = in_order(P, ch.first, end) ? end : P.T;
  for (int64_t i = threadIdx.x; i < (int64_t)(to - from) * a.hq * D; i += nt) {
    const int t = from + (int)(i / (a.hq * D)), e = (int)(i % (a.hq * D));
    ((T*)a.out)[a.at(a.os, t, e / D) + e % D] = (T)NAN;
    if (a.lse && e % D == 0) a.lse[(int64_t)t * a.hq + e / D] = NAN;
  }
}

// Many rows: a workgroup a tile of rows of one sequence and key head and one of `splits` ranges of keys.
template <typename T, typename X>
__global__ __launch_bounds__(X::NT, X::W * X::WGS / 4) void tiles_kernel(Paged P, AttendArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[X::kLds];
  __shared__ int fix[4];
  no_fix(fix);
  __syncthreads();
  // Workgroups are dealt to the 8 dies in turn; a die is to read the same keys for the tiles that it runs together.  A unit
  // is a sequence and key head.
  const uint32_t per = (uint32_t)(a.tiles * a.splits);
  uint32_t id = 0, rank = 0;
  int split = 0, tile, g, b;
  if (a.bundle == kPacked) {
    // Many sequences of which few have many rows: workgroups are numbered by the rows there are.  The tiles of sequence b are
    // numbers cu_q[b] * group / TM + b (rounded down) and on; for a chunk of n tokens the next sequence's begin n * group / TM,
    // rounded down, and 1 later at least, so after its last.  The sequence is the last whose numbers begin at or before this one.
    if (blockIdx.x >= (uint32_t)a.blocks) return;
    const int lane = (int)threadIdx.x & 63, G = (int)a.group.d, u = (int)(blockIdx.x / (uint32_t)P.hkv);
    g = (int)(blockIdx.x % (uint32_t)P.hkv);
    uint64_t stop = 0;
    for (b = 0; b < P.B && !stop; b += 64) {
      const int x = min(b + lane, P.B - 1);
      const int32_t first = P.cu_q[x], end = P.cu_q[x + 1];
      stop = __ballot(b + lane < P.B && (!in_order(P, first, end) || end * G / X::TM + x + 1 > u));
    }
    if (!stop) return;
    b += __builtin_ctzll(stop) - 64;
    tile = u - min(max(P.cu_q[b], 0), P.T) * G / X::TM - b;
    if (tile < 0) return;  // before the first sequence
  } else if (a.bundle == 0) {
    // Many units that all run at once: runs of 16 that follow one another go to one die, so that the keys are shared and
    // chunks of many tiles spread over the dies; every other round of the dies is reversed, for a unit's tiles come the
    // longest first (7 chunks of up to 77 tokens, a window of 300, 5 key heads: 8.2 us; with a unit a die 9.2, with an
    // eighth of them all a die 9.9).  Against bundles as below it gains where tiles differ and hardly matters for one a unit
    // (that case 9.4 us and 9.9, 64 single tokens 12.0 and 11.9, 12 ragged chunks of 40 17.8 and 17.7); 20 chunks of 30, all
    // alike, it costs 32.7 us for 28.9.
    constexpr uint32_t kRun = 16;
    const uint32_t round = blockIdx.x / (8 * kRun), die = blockIdx.x % 8;
    const uint32_t at = (round * 8 + (round & 1 ? 7 - die : die)) * kRun + blockIdx.x / 8 % kRun;
    if (at >= (uint32_t)a.blocks) return;
    id = at / per;
    rank = at - id * per;
  } else {
    // `bundle` units side by side, the longest tiles of all first, so that the last to run are short (of ranges of keys the
    // last ones, that early rows see little of).  A die has its own units of a bundle of a multiple of 8, or of 4 or 2
    // shares them with few others.  (A chunk of 2048 tokens after 4096, 4 units of 112 tiles: 175 us, in runs of 16 213.)
    const uint32_t begun = blockIdx.x / ((uint32_t)a.bundle * per), in = blockIdx.x - begun * (uint32_t)a.bundle * per;
    if (blockIdx.x >= (uint32_t)a.blocks) return;
    const uint32_t first = begun * (uint32_t)a.bundle, side = min((uint32_t)a.bundle, (uint32_t)a.blocks / per - first);
    rank = in / side;
    id = first + in - rank * side;
  }
  if (a.bundle != kPacked) {
    split = (int)(rank / (uint32_t)a.tiles);
    tile = a.tiles - 1 - (int)(rank % (uint32_t)a.tiles);
    g = (int)(id % (uint32_t)P.hkv);
    b = (int)(id / (uint32_t)P.hkv);
  }
  const Chunk ch = chunk_of(P, b);
  // Whether the chunks before are in order is asked now and told when the pages have been looked up: up to 1000 sequences
  // that costs nothing that shows (chunks of 9 tokens after 300, 16 heads on 2 of 64: 60 sequences 9.6 us, 1000 64.0, and 62.9
  // without), 4000 take 223 us and 216 without, 16000 846 and 735.
  const bool searched = a.bundle == kPacked;  // they were looked at above
  const OrderBefore before(P, b, (int)threadIdx.x);
  if (is_bad(a, ch)) {
    if (split > 0 || tile > 0 || g > 0) return;
    if (!searched && !before.ok(P, b, (int)threadIdx.x, X::NT)) fix[3] = 1;
    __syncthreads();
    if (!fix[3]) fill_nan<T, X::D>(P, a, ch, b, X::NT);
    return;
  }
  if (tile * X::TM >= ch.n * (int)a.group.d) return;
  // the keys that the tile's rows see, within the range
  const int start = first_key(a, ch), first_pos = ch.kv - ch.n;
  const int first_i = (int)a.group.quot((uint32_t)(tile * X::TM));
  const int last_i = min((int)a.group.quot((uint32_t)(tile * X::TM + X::TM - 1)), ch.n - 1);
  const int seen = a.window ? max(0, first_pos + first_i - a.window + 1) : 0;
  const int s_lo = max(start + split * a.len, seen) / X::SK * X::SK;
  const int s_hi = (int)min((int64_t)start + (int64_t)(split + 1) * a.len, (int64_t)first_pos + last_i + 1);
  if (s_lo >= s_hi) return;
  X::run(P, a, lds, fix, ch, b, g, tile, s_lo, s_hi, ch.kv - start <= a.len,
         (((int64_t)b * P.hkv + g) * a.tiles + tile) * a.splits + split, [&] {
           if (!searched && !before.ok(P, b, (int)threadIdx.x, X::NT)) fix[3] = 1;
         });
}

__device__ inline uint64_t uniform(uint64_t x) {  // the same in all lanes: known to be
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// floor(i * total / n) and floor(i * n / total), i <= total, n <= 2^9: in 32 bits where they fit, as they do but for caches
// of a thousand million positions.
__device__ inline uint64_t scaled(uint64_t i, uint64_t by, uint64_t over, uint64_t total) {
  if (total < 1u << 22) return (uint32_t)(i * by) / (uint32_t)over;
  return i * by / over;
}

// Few rows: every sequence's rows are one tile, and the work is the stages of all sequences and key heads in a row,
// cut into equal shares: workgroup i takes stages i * total / n .. (i + 1) * total / n - 1, whatever units they belong
// to.  So all finish together, however ragged the lengths.  Of a unit that workgroups share, the sums of the one that
// begins it go to its slot 2 i + 1, those of the others to 2 i; runs tells the joining kernel which they are.
template <typename T, typename X>
__global__ __launch_bounds__(X::NT, X::W * X::WGS / 4) void shares_kernel(Paged P, AttendArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[X::kLds];
  __shared__ uint64_t waves[X::W], found[2], kept[4];
  __shared__ int broken_of[X::W];
  __shared__ int fix[4];
  no_fix(fix);
  const int tid = (int)threadIdx.x, lane = tid & 63;
  const uint64_t me = blockIdx.x, heads = (uint64_t)P.hkv;
  const auto stages = [&](const Chunk& c) {
    return is_bad(a, c) || c.n == 0 ? 0u : (uint32_t)((c.kv - first_key(a, c) + X::SK - 1) / X::SK);
  };
  const bool few = P.B <= 64;  // sequences: a lane each, in every wave; otherwise a run of them each thread
  const int per = few ? 1 : (P.B + X::NT - 1) / X::NT, b0 = min((few ? lane : tid) * per, P.B), b1 = min(b0 + per, P.B);
  Chunk own = {0, 0, 0, false};
  uint64_t mine = 0;
  int broken = P.B;  // the first sequence whose chunk is not in order: it and all after it have no stages
  for (int b = b0; b < b1; ++b) {
    own = chunk_of(P, b);
    if (!in_order(P, own.first, P.cu_q[b + 1])) {
      broken = b;
      break;
    }
    mine += stages(own);
  }
  if (few) {
    const uint64_t all = __ballot(broken < P.B);
    broken = all ? __builtin_ctzll(all) : P.B;
  } else {
    broken = min_across(broken);
    if (lane == 0) broken_of[tid >> 6] = broken;
    __syncthreads();
    for (int w = 0; w < X::W; ++w) broken = min(broken, broken_of[w]);
  }
  if (b0 > broken) mine = 0;
  uint64_t upto = mine;  // with the stages of the sequences before
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t x = __shfl_up((unsigned long long)upto, o);
    if (lane >= o) upto += x;
  }
  uint64_t total;
  if (few) {
    total = __shfl((unsigned long long)upto, 63);
  } else {
    if (lane == 63) waves[tid >> 6] = upto;
    __syncthreads();
    total = 0;
    for (int w = 0; w < X::W; ++w) {
      if (w < tid >> 6) upto += waves[w];
      total += waves[w];
    }
  }
  total = uniform(total * heads);
  if (few ? __any(b0 < b1 && is_bad(a, own)) : true)
    for (int b = (int)me; b < min(P.B, broken + 1); b += (int)gridDim.x) {
      const Chunk c = chunk_of(P, b);
      if (is_bad(a, c)) fill_nan<T, X::D>(P, a, c, b, X::NT);
    }
  uint64_t n = min((uint64_t)gridDim.x, total);  // no share is empty
  if (me >= n) return;
  uint64_t x = uniform(scaled(total, me, n, total));
  uint64_t end = uniform(scaled(total, me + 1, n, total));
  const bool here = x >= (upto - mine) * heads && x < upto * heads;
  int b;
  uint64_t first;  // stages before sequence b
  Chunk ch;
  if (few) {
    b = __builtin_ctzll(__ballot(here));
    first = uniform(__shfl((unsigned long long)(upto - mine), b)) * heads;
    ch.first = __builtin_amdgcn_readlane(own.first, b);
    ch.n = __builtin_amdgcn_readlane(own.n, b);
    ch.kv = __builtin_amdgcn_readlane(own.kv, b);
    ch.ok = true;
    __syncthreads();  // no_fix
  } else {
    if (here) {
      uint64_t before = upto - mine;
      int i = b0;
      for (; i < b1 - 1; ++i) {
        const uint32_t s = stages(chunk_of(P, i));
        if (x < (before + s) * heads) break;
        before += s;
      }
      found[0] = (uint64_t)i;
      found[1] = before;
    }
    __syncthreads();
    b = __builtin_amdgcn_readfirstlane((int)found[0]);
    first = uniform(found[1]) * heads;
    ch = chunk_of(P, b);
  }
  for (;;) {
    const uint64_t s = stages(ch);
    if (x >= first + s * heads) {  // the next sequence (b < P.B: x < end <= total)
      first += s * heads;
      ch = chunk_of(P, ++b);
      continue;
    }
    const int g = __builtin_amdgcn_readfirstlane((int)((uint32_t)(x - first) / (uint32_t)s));
    const uint64_t unit = first + (uint64_t)g * s, stop = min(end, unit + s);
    const bool whole = x == unit && stop == unit + s;
    if (x == unit && tid == 0)
      a.runs[(int64_t)b * P.hkv + g] =
          make_int2((int)me, whole ? (int)me : (int)(((unit + s) * n - 1) / total));
    const int start = first_key(a, ch);
    const int s_lo = __builtin_amdgcn_readfirstlane(start + (int)(x - unit) * X::SK);
    const int s_hi = __builtin_amdgcn_readfirstlane(min(ch.kv, start + (int)(stop - unit) * X::SK));
    // what the loop goes on with waits in LDS: the stages need the scalar registers
    if (tid == 0) {
      kept[0] = stop;
      kept[1] = end;
      kept[2] = first;
      kept[3] = total;
    }
    X::run(P, a, lds, fix, ch, b, g, 0, s_lo, s_hi, whole, (int64_t)me * 2 + (x == unit), Nothing());
    x = uniform(kept[0]);
    end = uniform(kept[1]);
    if (x >= end) return;
    first = uniform(kept[2]);
    total = uniform(kept[3]);
    n = min((uint64_t)gridDim.x, total);
    __syncthreads();
    no_fix(fix);
    __syncthreads();
  }
}

// The parts of a row (a token and head) joined by WAVES waves: D / 4 lanes a part, several parts side by side.
template <typename T, int D, int TM, bool SHARES, int WAVES>
__global__ __launch_bounds__(256) void join_kernel(Paged P, AttendArgs a) {
  constexpr int L = D / 4, N = 64 * WAVES / L, R = 4 / WAVES;  // lanes a part, parts side by side, rows a workgroup
  const int tid = (int)threadIdx.x, lane = tid & 63, in = tid % (64 * WAVES), e = in % L * 4, side = in / L;
  const uint32_t u = blockIdx.x * R + (uint32_t)tid / (64 * WAVES);
  const int t = (int)(u / (uint32_t)a.hq), h = (int)(u % (uint32_t)a.hq);
  bool live = t < P.T;
  int b;
  const Chunk ch = chunk_of_token(P, t, b);
  live = live && !is_bad(a, ch) && t >= ch.first && t < ch.first + ch.n;
  const int G = (int)a.group.d, g = (int)a.group.quot((uint32_t)h), r = (t - ch.first) * G + h - g * G;
  int from = 0, to = -1;
  int64_t slots = 0;
  if (live) {
    if constexpr (SHARES) {
      const int2 run = a.runs[(int64_t)b * P.hkv + g];
      from = run.x;
      to = run.y;
      live = from != to;
    } else {
      const int start = first_key(a, ch), pos = ch.kv - ch.n + t - ch.first;
      live = ch.kv - start > a.len;
      from = (max(a.window ? pos - a.window + 1 : 0, start) - start) / a.len;
      to = (pos - start) / a.len;
      slots = (((int64_t)b * P.hkv + g) * a.tiles + r / TM) * a.splits;
    }
  }
  if (!live) {
    if constexpr (WAVES > 1) return;  // the whole workgroup
    to = from - 1;
  }
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto take = [&](float om, float ol, float4 x) {
    const float now = fmaxf(m, om), ref = now == -INFINITY ? 0.f : now;
    const float keep = __builtin_amdgcn_exp2f(m - ref), add = __builtin_amdgcn_exp2f(om - ref);
    l = l * keep + ol * add;
    o.x = o.x * keep + x.x * add, o.y = o.y * keep + x.y * add;
    o.z = o.z * keep + x.z * add, o.w = o.w * keep + x.w * add;
    m = now;
  };
#pragma unroll 4
  for (int s = from + side; s <= to; s += N) {
    const int64_t at = (SHARES ? (int64_t)s * 2 + (s == from) : slots + s) * TM + r % TM;
    const float2 p = a.part_ml[at];
    take(p.x, p.y, *(const float4*)(a.part_o + at * D + e));
  }
  // the sides of a wave, then the waves
#pragma unroll
  for (int d = L; d < 64; d <<= 1) {
    const float om = __shfl_xor(m, d), ol = __shfl_xor(l, d);
    take(om, ol, make_float4(__shfl_xor(o.x, d), __shfl_xor(o.y, d), __shfl_xor(o.z, d), __shfl_xor(o.w, d)));
  }
  if constexpr (WAVES > 1) {
    __shared__ float2 ml[WAVES];
    __shared__ float4 os[WAVES][L];
    if (lane == 0) ml[tid >> 6] = make_float2(m, l);
    if (lane < L) os[tid >> 6][lane] = o;
    __syncthreads();
    if (tid >= L) return;
#pragma unroll
    for (int i = 1; i < WAVES; ++i) take(ml[i].x, ml[i].y, os[i][tid]);
  }
  if (!live || side > 0) return;
  const float over = l == 0.f ? 0.f : 1.f / l;
  T y[4] = {(T)(o.x * over), (T)(o.y * over), (T)(o.z * over), (T)(o.w * over)};
  *(uint2*)(a.out + a.at(a.os, t, h) + e) = *(uint2*)y;
  if (a.lse && e == 0) a.lse[(int64_t)t * a.hq + h] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Keys that a sequence's rows are given, at most: with a window those of its chunk too, from a multiple of 128 on.
int64_t span_of(const grid_paged_cache* c, const grid_chunks* x, const grid_attend_args* g) {
  const int64_t span = std::min<int64_t>(g->max_kv, (int64_t)x->table_cols * c->page_size);
  return g->window ? std::min<int64_t>(span, (int64_t)g->window + g->max_q + 127) : span;
}
constexpr int64_t kStage = 64;  // the shortest stage of the shares

int check(const grid_paged_cache* cache, const grid_chunks* chunks, const grid_attend_args* g, bool pointers) {
  const int rc = check_paged("grid_attend", cache, chunks, pointers);
  if (rc != GRID_OK) return rc;
  auto bad = [](const char* what) { return fail(GRID_E_ARG, std::string("grid_attend: ") + what); };
  if (!g) return bad("null argument");
  const int D = cache->head_dim;
  if (D != 64 && D != 128 && D != 256) return bad("head_dim is 64, 128 or 256");
  if (g->n_heads < 1 || g->n_heads > 1024 || g->n_heads % cache->n_kv_heads != 0)
    return bad("n_heads is a multiple of the key heads, at most 1024");
  if (g->max_q < 1 || g->max_kv < 1 || g->window < 0) return bad("max_q, max_kv or window");
  if (!std::isfinite(g->scale)) return bad("scale");
  if ((int64_t)std::min(g->max_q, chunks->n_tokens) * (g->n_heads / cache->n_kv_heads) >= 1 << 30)
    return fail(GRID_E_CAPACITY, "grid_attend: 2^30 rows of a sequence and key head or more");
  // (the shares count the stages of a sequence, all key heads together, in 32 bits)
  if ((span_of(cache, chunks, g) + kStage - 1) / kStage * cache->n_kv_heads >= (int64_t)1 << 32)
    return fail(GRID_E_CAPACITY, "grid_attend: 2^38 keys of a sequence in all key heads or more");
  if (!pointers || chunks->n_tokens == 0) return GRID_OK;
  if (!g->q || !g->out) return bad("null pointer");
  if (!rows_fit(g->q, g->q_stride, 2) || !rows_fit(g->out, g->out_stride, 2))
    return bad("rows are 16-byte aligned, their strides multiples of 8");
  return GRID_OK;
}


// The launch.
//  - Up to 64 rows a sequence and key head: one tile of 32 or 64, and equal shares of the stages, two workgroups a compute
//    unit, or fewer where there are fewer stages.
//  - More rows: tiles of 128; where they are fewer than 3/4 of the workgroups that run at once the keys are split, into
//    ranges of 512 or more, made alike, so of 384 at least (a chunk after a cache, 6144 keys together, 28 heads on 4 of
//    128: of 1280 tokens 148 us split and 160 whole, of 2048, 7/8 of the workgroups, 202 and 175).  Where sequences times
//    the tiles of the longest chunk exceed a launch, workgroups are numbered by the rows there are (5000 chunks of up to 7
//    tokens and one of 700, 16 heads on 1 of 64: 209 us).
//  - Few keys, where tiles of 32 run all at once: those, a workgroup each for all its keys.  Four waves share a tile's
//    keys, and nothing needs joining.  Up to 64 rows that saves the joining launch and costs the keys in turn: a token of 28
//    heads on 4 of 128 after 256 keys takes 7.0 us so and 10.2 shared, after 512 9.4 and 10.6, after 1024 14.6 and 10.4;
//    where the tiles fill the chip shares only add parts (64 tokens, 32 heads on 8, 1 to 2048 keys: 48 us and 59; 32
//    chunks of 8: 30 and 42).  Where they fill half of it or more: 40 tokens of 28 heads on 4, 512 keys 13.1 us and 21.7,
//    1024 19.7 and 25.9, 1536 27.3 and 30.9; of 60, 1024 24.3 and 31.4.  Heads of 256 have one workgroup a compute unit and
//    are slower so sooner: a token of 8 heads on 1, 256 keys 10.9 us and 12.3, 384 12.9 and 13.0, 512 15.5 and 13.0; 40 of
//    them, 384 15.1 and 14.7 (200 of them 20.9 and 43.6, and still faster so at 640).  Of more rows, against tiles of 128: 7
//    chunks of up to 77 tokens, 5 key heads of 64, under a window of 300 9.3 us and 15.6, of 900 13.8 and 18.9; after 1024
//    keys, all seen, 15.7 and 20.4, 2048 25.8 and 24.1; 4 chunks of 100, 28 heads on 4, 1024 22.6 and 28.9, 2048 36.5 and
//    34.4; 2 of 128 with heads of 256, 1024 28.8 and 33.3, 2048 47.6 and 36.3.
constexpr int kComputeUnits = 256;
constexpr int64_t kMostBlocks = (int64_t)1 << 23;  // of a launch: below 2^32 threads
struct Shape {
  int tm, splits, len;
  int64_t tiles, blocks;
  bool shares, join, packed;
  int64_t at_once;  // workgroups that run side by side (many rows)
  int64_t parts;  // of a row, on average over the units (a long sequence among short ones has more)
  size_t slots;   // of parts
};
Shape shape_of(const grid_paged_cache* c, const grid_chunks* x, const grid_attend_args* g) {
  Shape s;
  const int group = g->n_heads / c->n_kv_heads;
  const int64_t rows = (int64_t)std::min(g->max_q, std::max(1, x->n_tokens)) * group;
  const int64_t span = span_of(c, x, g);
  const int64_t heads = (int64_t)c->n_kv_heads * x->n_seqs;
  const int64_t small = heads * ((rows + 31) / 32);  // tiles of 32
  const int few_keys = rows > 64                   ? 1024
                       : c->head_dim == 256        ? 384
                       : small >= kComputeUnits     ? 2048
                       : small >= kComputeUnits / 2 ? 1024
                                                    : 640;
  const bool narrow = small <= 2 * kComputeUnits && span <= few_keys;
  s.shares = rows <= 64 && !narrow;
  s.packed = false;
  s.tm = rows <= 32 || narrow ? 32
         : rows <= 64                                                                                  ? 64
                                                                                                       : 128;
  s.tiles = (rows + s.tm - 1) / s.tm;
  s.splits = 1;
  s.len = INT32_MAX;
  s.at_once = (c->head_dim == 256 ? 1 : 2) * kComputeUnits;
  if (s.shares) {
    const int64_t stages = (span + kStage - 1) / kStage;
    s.blocks = std::min<int64_t>(heads * stages, 2 * kComputeUnits);
    s.join = stages > 1;
    s.parts = s.blocks / heads;
    s.slots = (size_t)s.blocks * 2;
    return s;
  }
  s.blocks = heads * s.tiles;
  // a joining workgroup a row has to fit a launch
  if (s.tm == 128 && 4 * s.blocks < 3 * s.at_once && (int64_t)x->n_tokens * g->n_heads <= 1 << 22) {
    const int64_t len = (std::max<int64_t>(512, span * s.blocks / (4 * kComputeUnits)) + 127) / 128 * 128;
    if (len < span) {  // ranges alike
      s.splits = (int)((span + len - 1) / len);
      s.len = (int)(((span + s.splits - 1) / s.splits + 127) / 128 * 128);
      s.blocks *= s.splits;
    }
  }
  if (s.blocks > kMostBlocks) {
    s.packed = true;
    s.blocks = c->n_kv_heads * ((int64_t)x->n_tokens * group / s.tm + x->n_seqs);
  }
  s.join = s.splits > 1;
  s.parts = s.splits;
  s.slots = s.join ? (size_t)s.blocks : 0;
  return s;
}

size_t runs_bytes(const grid_paged_cache* c, const grid_chunks* x) {
  return ((size_t)x->n_seqs * (size_t)c->n_kv_heads * sizeof(int2) + 15) / 16 * 16;
}
size_t workspace_of(const grid_paged_cache* c, const grid_chunks* x, const Shape& s) {
  return runs_bytes(c, x) + s.slots * (size_t)s.tm * (size_t)(c->head_dim + 2) * 4;
}

template <typename T, int D, int RW, int KW, int KT, int WGS, bool SHARES>
void launch(const Paged& P, const AttendArgs& a, const Shape& s, hipStream_t stream) {
  const auto go = [&](auto tile) {
    using X = decltype(tile);
    if constexpr (SHARES)
      hipLaunchKernelGGL((shares_kernel<T, X>), dim3((unsigned)s.blocks), dim3(X::NT), 0, stream, P, a);
    else
      hipLaunchKernelGGL((tiles_kernel<T, X>), dim3((unsigned)((s.blocks + 127) / 128 * 128)), dim3(X::NT), 0, stream, P, a);
  };
  if (P.page.d % 16 == 0)
    go(Tile<T, D, RW, KW, KT, WGS, true>());
  else
    go(Tile<T, D, RW, KW, KT, WGS, false>());
  if (!s.join) return;
  const unsigned rows = (unsigned)P.T * (unsigned)a.hq;
  if (s.parts <= 16)  // a row's: a wave takes them in a few steps
    hipLaunchKernelGGL((join_kernel<T, D, RW * 32, SHARES, 1>), dim3((rows + 3) / 4), dim3(256), 0, stream, P, a);
  else
    hipLaunchKernelGGL((join_kernel<T, D, RW * 32, SHARES, 4>), dim3(rows), dim3(256), 0, stream, P, a);
}

// Waves of rows and of keys, keys a wave and workgroups a compute unit, by what fits in LDS and registers.
// Tiles of 128 take the longest stages that fit two workgroups a compute unit, of heads of 256 one: there a stage of 64
// keys for one of 32 took 4 chunks of 2048 tokens after 4096, 8 heads on 1, from 495 us to 400.
template <typename T>
void choose(const Paged& P, const AttendArgs& a, const Shape& s, hipStream_t stream) {
  const auto with = [&](auto few, auto some, auto many, auto narrow) {
    if (s.tm == 128)
      many();
    else if (!s.shares)
      narrow();
    else if (s.tm == 32)
      few();
    else
      some();
  };
  if (P.D == 64)
    with([&] { launch<T, 64, 1, 4, 32, 2, true>(P, a, s, stream); }, [&] { launch<T, 64, 2, 2, 32, 2, true>(P, a, s, stream); },
         [&] { launch<T, 64, 4, 1, 128, 2, false>(P, a, s, stream); },
         [&] { launch<T, 64, 1, 4, 32, 2, false>(P, a, s, stream); });
  else if (P.D == 128)
    with([&] { launch<T, 128, 1, 4, 32, 2, true>(P, a, s, stream); },
         [&] { launch<T, 128, 2, 2, 32, 2, true>(P, a, s, stream); },
         [&] { launch<T, 128, 4, 1, 64, 2, false>(P, a, s, stream); },
         [&] { launch<T, 128, 1, 4, 32, 2, false>(P, a, s, stream); });
  else
    with([&] { launch<T, 256, 1, 4, 32, 1, true>(P, a, s, stream); },
         [&] { launch<T, 256, 2, 2, 32, 1, true>(P, a, s, stream); },
         [&] { launch<T, 256, 4, 1, 64, 1, false>(P, a, s, stream); },
         [&] { launch<T, 256, 1, 4, 32, 1, false>(P, a, s, stream); });
}

}  // namespace

extern "C" size_t grid_attend_workspace_bytes(const grid_paged_cache* cache, const grid_chunks* chunks,
                                              const grid_attend_args* args) {
  if (check(cache, chunks, args, false) != GRID_OK) return 0;
  return workspace_of(cache, chunks, shape_of(cache, chunks, args));
}

extern "C" int grid_attend(const grid_paged_cache* cache, const grid_chunks* chunks, const grid_attend_args* args,
                           void* stream) {
  clear_error();
  const int rc = check(cache, chunks, args, true);
  if (rc != GRID_OK) return rc;
  if (chunks->n_tokens == 0) return GRID_OK;
  const Shape s = shape_of(cache, chunks, args);
  if (!args->workspace || (uintptr_t)args->workspace % 16 != 0 ||
      args->workspace_bytes < workspace_of(cache, chunks, s))
    return fail(GRID_E_ARG, "grid_attend: workspace too small or not aligned");
  if (s.blocks > kMostBlocks || (s.join && (int64_t)chunks->n_tokens * args->n_heads > kMostBlocks))
    return fail(GRID_E_CAPACITY, "grid_attend: too many rows for one launch");
  AttendArgs a;
  a.q = (const uint16_t*)args->q;
  a.out = (uint16_t*)args->out;
  for (int i = 0; i < 2; ++i) {
    a.qs[i] = (uint32_t)args->q_stride[i];
    a.os[i] = (uint32_t)args->out_stride[i];
  }
  a.lse = args->lse;
  a.runs = (int2*)args->workspace;
  a.part_o = (float*)((uint8_t*)args->workspace + runs_bytes(cache, chunks));
  a.part_ml = (float2*)(a.part_o + s.slots * (size_t)s.tm * (size_t)cache->head_dim);
  a.group = Divisor((uint32_t)(args->n_heads / cache->n_kv_heads));
  a.hq = args->n_heads;
  a.max_q = args->max_q;
  a.max_kv = args->max_kv;
  // A window that no position exceeds is none, so positions less it and a few stages stay in 32 bits.
  const int64_t most = std::min<int64_t>(args->max_kv, (int64_t)chunks->table_cols * cache->page_size);
  a.window = args->window >= most ? 0 : args->window;
  a.blocks = (int32_t)s.blocks;
  a.tiles = (int32_t)s.tiles;
  a.splits = s.splits;
  a.len = s.len;
  // as many units side by side as fill the chip
  const int64_t per = s.tiles * s.splits, units = s.blocks / per, fill = (s.at_once + per - 1) / per;
  if (s.packed)
    a.bundle = kPacked;
  else
    a.bundle = s.blocks <= s.at_once && units > 8 ? 0 : (int32_t)std::min<int64_t>(units, (fill + 7) / 8 * 8);
  a.negate = args->scale < 0.f;
  a.c = std::fmin(std::fmax(std::fabs(args->scale) * kLog2e, 1e-30f), 1e30f);
  const Paged P = make_paged(cache, chunks);
  if (cache->dtype == GRID_DTYPE_BF16)
    choose<bf16_t>(P, a, s, (hipStream_t)stream);
  else
    choose<f16_t>(P, a, s, (hipStream_t)stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_attend launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
