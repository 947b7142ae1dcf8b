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
#include <algorithm>
#include <cmath>
#include <type_traits>

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
  int64_t qs[2], os[2];
  float* lse;
  float2* part_ml;  // [splits][tokens][heads]: maximum (in base 2 units of the scaled score), sum
  float* part_o;    // [splits][tokens][heads][D], not divided by the sum
  Divisor group;
  int32_t hq, max_q, max_kv, window, tiles, splits, len;  // len: keys of a split, a multiple of the stage
  float c;          // |scale| * log2 e, above 0
  bool negate;      // scale < 0: the queries are negated
};

constexpr float kLn2 = 0.693147180559945309417f, kLog2e = 1.44269504088896340736f;

// First key of the splits of a sequence: the window of its first new token, down to a whole stage of 128.
__device__ inline int split_start(const AttendArgs& a, const Chunk& c) {
  return a.window ? max(0, c.kv - c.n - a.window + 1) & ~127 : 0;
}

__device__ inline float other_half(float x) {  // the value of lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return (threadIdx.x & 32) ? __uint_as_float(r[0]) : __uint_as_float(r[1]);
}

// 16 bytes a lane from global memory (uniform base + the lane's offset in bytes) to LDS at `to` + 16 * lane (to:
// uniform, bytes from the start of LDS).  Written as assembly because the compiler waits for all such loads before any
// LDS read; they are counted by vmcnt.  LDS reads issued before are waited for first: they may be of what is overwritten.
__device__ inline void to_lds(const void* base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(to) : "memory");
}
__device__ inline void to_lds(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory");
}
__device__ inline void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ inline void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

#define GRID_LDS __attribute__((address_space(3)))

// The swizzle: 16-byte piece c of a row of keys or values lies at piece c ^ swz(row), so that the 32 rows of one piece
// (K's operand) and 4 rows of 64 bytes (V's, transposed) lie in different banks.
template <int D>
__device__ constexpr int swz(int row) {
  return D == 64 ? ((row >> 1 & 1) << 2 | (row >> 2 & 3)) : ((row & 3) << 2 | (row >> 2 & 3));
}

// RW x KW waves: RW * 32 rows, stages of KW * KT keys of which a wave takes KT.  With one wave of rows a wave loads its
// own keys and waits for nobody; otherwise the stage is shared.  DEPTH stages are held.  UNI: the rows that one load
// instruction brings (64 / PR) lie in one page, so their address is a scalar and an offset that does not change.
template <typename T, int D, int RW, int KW, int KT, int DEPTH, int WGS, bool UNI>
__global__ __launch_bounds__(64 * RW * KW, RW * KW * WGS / 4) void tile_kernel(Paged P, AttendArgs a) {
  typedef typename Vec<T>::eight Eight;
  constexpr int W = RW * KW, NT = 64 * W, TM = 32 * RW, SK = KW * KT;
  constexpr int PR = D / 8;               // 16-byte pieces of a row
  constexpr int RPI = 64 / PR;            // rows that one load instruction brings
  constexpr int LOADS = SK * PR / NT;     // of the keys, as many of the values, a thread
  constexpr int KB = KT / 32, DB = D / 32, QS = D / 16;
  constexpr bool PRIV = RW == 1;
  constexpr uint32_t kHalf = SK * D * 2;  // bytes of a stage's keys
  constexpr uint32_t kMerge = KW == 1 ? 0 : KW * TM * (2 + D / 2 + 4) * 4;  // what waves of other keys meet in
  constexpr uint32_t kLds = DEPTH * 2 * kHalf > kMerge ? DEPTH * 2 * kHalf : kMerge;
  static_assert(SK * PR % NT == 0 && 128 % SK == 0 && KT % RPI == 0, "");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kLds];

  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW, half = lane >> 5, col = lane & 31;
  // block -> (sequence, key head, tile, split)
  uint32_t id = blockIdx.x;
  const int split = (int)(id % (uint32_t)a.splits);
  id /= (uint32_t)a.splits;
  const int tile = a.tiles - 1 - (int)(id % (uint32_t)a.tiles);  // the longest first
  id /= (uint32_t)a.tiles;
  const int g = (int)(id % (uint32_t)P.hkv), b = (int)(id / (uint32_t)P.hkv);

  const Chunk ch = chunk_of(P, b);
  const int G = (int)a.group.d;
  if (!ch.ok || ch.n > a.max_q || ch.kv > a.max_kv) {
    // a bad sequence's rows: NaN, by its first block
    if (split == 0 && tile == 0 && g == 0) {
      const int from = min(max(ch.first, 0), P.T), to = min(max(P.cu_q[b + 1], from), P.T);
      for (int64_t i = tid; i < (int64_t)(to - from) * a.hq * D; i += NT) {
        const int t = from + (int)(i / (a.hq * D)), e = (int)(i % (a.hq * D));
        ((T*)a.out)[t * a.os[0] + (e / D) * a.os[1] + e % D] = (T)NAN;
        if (a.lse && e % D == 0) a.lse[(int64_t)t * a.hq + e / D] = NAN;
      }
    }
    return;
  }
  const int rows = ch.n * G, first_pos = ch.kv - ch.n;
  if (tile * TM >= rows) return;
  // the keys of this block: those its rows see, within the split
  const int start = split_start(a, ch);
  const int last_i = min((int)a.group.quot((uint32_t)(tile * TM + TM - 1)), ch.n - 1);
  const int first_i = (int)a.group.quot((uint32_t)(tile * TM));
  const int lo_tile = a.window ? max(0, first_pos + first_i - a.window + 1) : 0;
  const int s_lo = max(start + split * a.len, lo_tile) / SK * SK;
  const int s_hi = (int)min((int64_t)start + (int64_t)(split + 1) * a.len, (int64_t)first_pos + last_i + 1);
  if (s_lo >= s_hi) return;
  const bool whole = ch.kv - start <= a.len;  // one split: the result, not a part of it

  // this wave's rows: lane's query, its position, the wave's range of positions
  const int r0 = tile * TM + rw * 32, r = min(r0 + col, rows - 1);
  const bool alive = r0 < rows;
  const int qi = (int)a.group.quot((uint32_t)r), qh = g * G + r - qi * G, qt = ch.first + qi, pos = first_pos + qi;
  const int pos_min = first_pos + (int)a.group.quot((uint32_t)min(r0, rows - 1));
  const int pos_max = first_pos + (int)a.group.quot((uint32_t)min(r0 + 31, rows - 1));

  Eight q[QS];
  {
    const uint16_t* src = a.q + qt * a.qs[0] + qh * a.qs[1] + half * 8;
    const uint32_t flip = a.negate ? 0x80008000u : 0u;
#pragma unroll
    for (int k = 0; k < QS; ++k) {
      uint4 x = *(const uint4*)(src + k * 16);
      x.x ^= flip, x.y ^= flip, x.z ^= flip, x.w ^= flip;
      q[k] = __builtin_bit_cast(Eight, x);
    }
  }

  // Stage rows: load i of a wave brings RPI rows from row_of(i) on, a lane piece `lane % PR` of row `lane / PR`.
  const auto row_of = [&](int i) { return PRIV ? kw * KT + i * RPI : (i * W + wave) * RPI; };
  const uint32_t base = (uint32_t)(uintptr_t)(GRID_LDS uint8_t*)lds;
  const int lrow = lane / PR;
  int32_t page[LOADS];
  uint32_t row[LOADS];
  bool missing = false;
  const auto find = [&](int s0) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      if constexpr (UNI) {
        const uint32_t s = (uint32_t)min(s0 + row_of(i), (s_hi - 1) / RPI * RPI);
        const uint32_t c = P.page.quot(s);
        row[i] = s - c * P.page.d;
        page[i] = ((const __attribute__((address_space(4))) int32_t*)(P.table + (int64_t)b * P.table_stride))[c];
      } else {
        page[i] = P.page_of(b, (uint32_t)min(s0 + row_of(i) + lrow, s_hi - 1), row[i]);
      }
    }
  };
  const auto fetch = [&](int s0, int buf) {
    if constexpr (PRIV) wait_reads();
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int rr = row_of(i) + lrow, piece = lane % PR ^ swz<D>(rr);
      const bool in = P.in_cache(page[i]);
      missing |= !in;
      const uint32_t pg = in ? (uint32_t)page[i] : 0u;
      const uint32_t to = base + (uint32_t)buf * 2 * kHalf + (uint32_t)row_of(i) * D * 2;
      const uint16_t* k = P.k + (uint64_t)pg * (uint32_t)P.ks[0] + (uint64_t)row[i] * (uint32_t)P.ks[1] + g * P.ks[2];
      const uint16_t* v = P.v + (uint64_t)pg * (uint32_t)P.vs[0] + (uint64_t)row[i] * (uint32_t)P.vs[1] + g * P.vs[2];
      if constexpr (UNI) {
        // rows at and after s_hi: the last row again
        const uint32_t r = (uint32_t)min(lrow, s_hi - 1 - min(s0 + row_of(i), (s_hi - 1) / RPI * RPI));
        to_lds(k, (r * (uint32_t)P.ks[1] + piece * 8) * 2, to);
        to_lds(v, (r * (uint32_t)P.vs[1] + piece * 8) * 2, to + kHalf);
      } else {
        to_lds(k + piece * 8, to);
        to_lds(v + piece * 8, to + kHalf);
      }
    }
  };
  const auto arrived = [&] {
    wait_loads();
    if constexpr (!PRIV) __syncthreads();
  };

  float16_v o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -INFINITY, l = 0.f;

  find(s_lo);
  if constexpr (DEPTH > 1) {
    fetch(s_lo, 0);
    if (s_lo + SK < s_hi) find(s_lo + SK);
    arrived();
  }
  int buf = 0;
  for (int s0 = s_lo; s0 < s_hi; s0 += SK, buf ^= DEPTH - 1) {
    if constexpr (DEPTH > 1) {
      if (s0 + SK < s_hi) {
        fetch(s0 + SK, buf ^ 1);
        if (s0 + 2 * SK < s_hi) find(s0 + 2 * SK);
      }
    } else {
      fetch(s0, 0);
      if (s0 + SK < s_hi) find(s0 + SK);
      arrived();
    }
    const int k0 = s0 + kw * KT;  // this wave's keys
    const bool work = alive && k0 <= pos_max && k0 < s_hi && (!a.window || k0 + KT > pos_min - a.window + 1);
    if (work) {
      const uint8_t* ks = lds + buf * 2 * kHalf + kw * KT * D * 2;
      const uint8_t* vs = ks + kHalf;
      float16_v s[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
        for (int k = 0; k < QS; ++k) {
          const int piece = (2 * k + half) ^ swz<D>(col);
          const Eight kk = *(const Eight*)(ks + (kb * 32 + col) * D * 2 + piece * 16);
          s[kb] = Vec<T>::mfma(kk, q[k], s[kb]);
        }
      }
      const bool masked = k0 + KT - 1 > pos_min || k0 + KT > s_hi || (a.window && k0 <= pos_max - a.window);
      bool poison = false;
      if (masked) {
        const int hi = min(pos, s_hi - 1), lo = a.window ? pos - a.window : -1;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = k0 + kb * 32 + 8 * (i / 4) + 4 * half + i % 4;
            s[kb][i] = key <= hi && key > lo ? s[kb][i] : -INFINITY;
          }
        // values that are not finite must not meet a weight of 0 in a product
        uint32_t found = 0;
#pragma unroll
        for (int i = 0; i < KT * D * 2 / 1024; ++i) {
          const uint4 x = *(const uint4*)(vs + i * 1024 + lane * 16);
          found |= (x.x & Vec<T>::kExp) + Vec<T>::kOne;
          found |= (x.y & Vec<T>::kExp) + Vec<T>::kOne;
          found |= (x.z & Vec<T>::kExp) + Vec<T>::kOne;
          found |= (x.w & Vec<T>::kExp) + Vec<T>::kOne;
        }
        poison = __any((found & 0x80008000u) != 0);
      }
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
      auto product = [&](auto clean) {
#pragma unroll
        for (int t = 0; t < KT / 16; ++t) {
          Eight p;
#pragma unroll
          for (int i = 0; i < 8; ++i) p[i] = (T)s[t / 2][t % 2 * 8 + i];
#pragma unroll
          for (int d = 0; d < DB; ++d) {
            union {
              short4_v four[2];
              uint32_t pair[4];
              Eight all;
            } v;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const int l16 = lane & 15, rr = 16 * t + 8 * j + 4 * half + (l16 >> 2);
              const int piece = (d * 4 + (lane >> 4 & 1) * 2 + (l16 >> 1 & 1)) ^ swz<D>(rr);
              v.four[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (GRID_LDS short4_v*)(vs + rr * D * 2 + piece * 16 + (l16 & 1) * 8));
            }
            if constexpr (clean())
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t e = (v.pair[j] & Vec<T>::kExp) + Vec<T>::kOne;
                v.pair[j] &= (e & 0x8000u ? 0u : 0xFFFFu) | (e & 0x80000000u ? 0u : 0xFFFF0000u);
              }
            o[d] = Vec<T>::mfma(v.all, p, o[d]);
          }
        }
      };
      if (!poison) {
        product(std::false_type());
      } else {
        // the finite values as ever; then the others, one by one, where their weight is above 0
        product(std::true_type());
        for (int kk = 0; kk < KT; ++kk) {
          const int reg = kk / 32 * 16 + (kk >> 3 & 3) * 4 + (kk & 3);
          float p = 0.f;
#pragma unroll
          for (int i = 0; i < KB * 16; ++i) p = i == reg ? s[i / 16][i % 16] : p;
          p = (float)(T)__shfl(p, col + (kk & 4) * 8);
          const uint16_t* vr = (const uint16_t*)(vs + kk * D * 2);
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int e = d * 32 + 8 * (i / 4) + 4 * half + i % 4;
              const uint16_t v = vr[(e / 8 ^ swz<D>(kk)) * 8 + e % 8];
              if ((v & Vec<T>::kExp) + Vec<T>::kOne & 0x8000u && p > 0.f) o[d][i] += p * (float)__builtin_bit_cast(T, v);
            }
        }
      }
    }
    if constexpr (DEPTH > 1)
      arrived();
    else if constexpr (!PRIV)
      __syncthreads();
  }
  l += other_half(l);
  missing = __syncthreads_or(missing);
  if (missing) l = NAN;
  float mc = m * a.c;  // -inf where the row saw nothing

  // waves that took other keys of the same rows: their sums meet in LDS
  if constexpr (KW > 1) {
    constexpr int DH = D / 2;                     // in two halves of the entries, for room
    float* ml = (float*)lds;                      // [KW][2][TM]
    float* os = (float*)(lds + KW * 2 * TM * 4);  // [KW][TM][DH + 4]
    if (half == 0) {
      ml[(kw * 2 + 0) * TM + rw * 32 + col] = mc;
      ml[(kw * 2 + 1) * TM + rw * 32 + col] = l;
    }
    __syncthreads();
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) top = fmaxf(top, ml[w * 2 * TM + rw * 32 + col]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < KW; ++w)
      sum += ml[(w * 2 + 1) * TM + rw * 32 + col] * __builtin_amdgcn_exp2f(ml[w * 2 * TM + rw * 32 + col] - ref);
    const float keep = __builtin_amdgcn_exp2f(mc - ref);
    mc = top;
    l = sum;
    __syncthreads();
    if (kw == 0 && half == 0) {
      ml[rw * 32 + col] = mc;
      ml[TM + rw * 32 + col] = l;
    }
    float* mine = os + (kw * TM + rw * 32 + col) * (DH + 4);
    constexpr int PART = 32 * DH / 4 / 64 / KW;  // float4s a lane
#pragma unroll
    for (int hd = 0; hd < 2; ++hd) {
#pragma unroll
      for (int d = 0; d < DB / 2; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float16_v& x = o[hd * (DB / 2) + d];
          *(float4*)(mine + d * 32 + 2 * i + 4 * half) =
              make_float4(x[i] * keep, x[i + 1] * keep, x[i + 2] * keep, x[i + 3] * keep);
        }
      __syncthreads();
      // a wave adds up a part of its rows' entries
#pragma unroll
      for (int j = 0; j < PART; ++j) {
        const int at = (j * KW + kw) * 64 + lane, rr = rw * 32 + at / (DH / 4), e = at % (DH / 4) * 4;
        if (tile * TM + rr >= rows) continue;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          const float4 y = *(const float4*)(os + (w * TM + rr) * (DH + 4) + e);
          x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
        }
        const int i = (int)a.group.quot((uint32_t)(tile * TM + rr)), h = g * G + tile * TM + rr - i * G, t = ch.first + i;
        const float rm = ml[rr], rl = ml[TM + rr];
        if (whole) {
          const float over = rl == 0.f ? 0.f : 1.f / rl;
          T y[4] = {(T)(x.x * over), (T)(x.y * over), (T)(x.z * over), (T)(x.w * over)};
          *(uint2*)(a.out + t * a.os[0] + h * a.os[1] + hd * DH + e) = *(uint2*)y;
          if (a.lse && e == 0 && hd == 0) a.lse[(int64_t)t * a.hq + h] = (rm + __builtin_amdgcn_logf(rl)) * kLn2;
        } else {
          const int64_t slot = ((int64_t)split * P.T + t) * a.hq + h;
          *(float4*)(a.part_o + slot * D + hd * DH + e) = x;
          if (e == 0 && hd == 0) a.part_ml[slot] = make_float2(rm, rl);
        }
      }
      if (hd == 0) __syncthreads();
    }
  } else {
    if (r0 + col >= rows) return;
    if (whole) {
      const float over = l == 0.f ? 0.f : 1.f / l;
      uint16_t* dst = a.out + qt * a.os[0] + qh * a.os[1] + 4 * half;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          T y[4] = {(T)(o[d][i] * over), (T)(o[d][i + 1] * over), (T)(o[d][i + 2] * over), (T)(o[d][i + 3] * over)};
          *(uint2*)(dst + d * 32 + 2 * i) = *(uint2*)y;
        }
      if (a.lse && half == 0) a.lse[(int64_t)qt * a.hq + qh] = (mc + __builtin_amdgcn_logf(l)) * kLn2;
    } else {
      const int64_t slot = ((int64_t)split * P.T + qt) * a.hq + qh;
      float* dst = a.part_o + slot * D + 4 * half;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *(float4*)(dst + d * 32 + 2 * i) = make_float4(o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]);
      if (half == 0) a.part_ml[slot] = make_float2(mc, l);
    }
  }
}

// The splits of a row joined: a workgroup a token and head, D / 4 lanes a split, several splits side by side.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_kernel(Paged P, AttendArgs a) {
  constexpr int L = D / 4, N = 256 / L;
  const int tid = (int)threadIdx.x, lane = tid & 63, e = tid % L * 4, side = tid / L;
  const int t = (int)(blockIdx.x / (uint32_t)a.hq), h = (int)(blockIdx.x % (uint32_t)a.hq);
  int b = 0;
  for (int s = 0; s < P.B; s += 64) b += __popcll(__ballot(s + lane < P.B && P.cu_q[s + lane + 1] <= t));
  if (b >= P.B) return;
  const Chunk ch = chunk_of(P, b);
  if (!ch.ok || ch.n > a.max_q || ch.kv > a.max_kv || t < ch.first || t >= ch.first + ch.n) return;
  const int start = split_start(a, ch);
  if (ch.kv - start <= a.len) return;
  const int pos = ch.kv - ch.n + t - ch.first;
  const int from = (max(a.window ? pos - a.window + 1 : 0, start) - start) / a.len, to = (pos - start) / a.len;
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
    const int64_t slot = ((int64_t)s * P.T + t) * a.hq + h;
    const float2 p = a.part_ml[slot];
    take(p.x, p.y, *(const float4*)(a.part_o + slot * D + e));
  }
  __shared__ float2 ml[N];
  __shared__ float4 os[N][L];
  if (e == 0) ml[side] = make_float2(m, l);
  os[side][tid % L] = o;
  __syncthreads();
  if (side > 0) return;
#pragma unroll
  for (int n = 1; n < N; ++n) take(ml[n].x, ml[n].y, os[n][tid]);
  const float over = l == 0.f ? 0.f : 1.f / l;
  T y[4] = {(T)(o.x * over), (T)(o.y * over), (T)(o.z * over), (T)(o.w * over)};
  *(uint2*)(a.out + t * a.os[0] + h * a.os[1] + e) = *(uint2*)y;
  if (a.lse && tid == 0) a.lse[(int64_t)t * a.hq + h] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

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
  if (!pointers || chunks->n_tokens == 0) return GRID_OK;
  if (!g->q || !g->out) return bad("null pointer");
  if (!rows_fit(g->q, g->q_stride, 2) || !rows_fit(g->out, g->out_stride, 2))
    return bad("rows are 16-byte aligned, their strides multiples of 8");
  return GRID_OK;
}


// Rows of a tile, and the ranges of keys: with few tiles the keys are split until there are about 4096 workgroups,
// none with fewer than 256 keys.
struct Shape {
  int tm, splits, len;
  int64_t tiles, blocks;
};
Shape shape_of(const grid_paged_cache* c, const grid_chunks* x, const grid_attend_args* g) {
  Shape s;
  const int group = g->n_heads / c->n_kv_heads;
  const int64_t rows = (int64_t)std::min(g->max_q, std::max(1, x->n_tokens)) * group;
  s.tm = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  s.tiles = (rows + s.tm - 1) / s.tm;
  const int64_t units = s.tiles * c->n_kv_heads * x->n_seqs;
  int64_t span = std::min<int64_t>(g->max_kv, (int64_t)x->table_cols * c->page_size);
  if (g->window) span = std::min<int64_t>(span, (int64_t)g->window + g->max_q + 127);
  s.len = (int)std::min<int64_t>(std::max<int64_t>(256, (span * units / 1024 + 127) / 128 * 128), 32 * s.tm);
  s.splits = (int)((span + s.len - 1) / s.len);
  s.blocks = units * s.splits;
  return s;
}

size_t workspace_of(const grid_paged_cache* c, const grid_chunks* x, const grid_attend_args* g, const Shape& s) {
  if (s.splits <= 1) return 16;
  return (size_t)s.splits * (size_t)x->n_tokens * (size_t)g->n_heads * (size_t)(c->head_dim + 2) * 4;
}

template <typename T, int D, int RW, int KW, int KT, int DEPTH, int WGS>
void launch(const Paged& P, const AttendArgs& a, const Shape& s, hipStream_t stream) {
  const dim3 blocks((unsigned)s.blocks), threads(64 * RW * KW);
  if (P.page.d % (512 / D) == 0)
    hipLaunchKernelGGL((tile_kernel<T, D, RW, KW, KT, DEPTH, WGS, true>), blocks, threads, 0, stream, P, a);
  else
    hipLaunchKernelGGL((tile_kernel<T, D, RW, KW, KT, DEPTH, WGS, false>), blocks, threads, 0, stream, P, a);
  if (s.splits > 1) {
    const dim3 rows((unsigned)P.T * (unsigned)a.hq);
    hipLaunchKernelGGL((join_kernel<T, D>), rows, dim3(256), 0, stream, P, a);
  }
}

template <typename T>
void choose(const Paged& P, const AttendArgs& a, const Shape& s, hipStream_t stream) {
  if (P.D == 64)
    s.tm == 32   ? launch<T, 64, 1, 4, 32, 1, 2>(P, a, s, stream)
    : s.tm == 64 ? launch<T, 64, 2, 2, 32, 1, 2>(P, a, s, stream)
                 : launch<T, 64, 4, 1, 64, 2, 2>(P, a, s, stream);
  else if (P.D == 128)
    s.tm == 32   ? launch<T, 128, 1, 4, 32, 1, 2>(P, a, s, stream)
    : s.tm == 64 ? launch<T, 128, 2, 2, 32, 1, 2>(P, a, s, stream)
                 : launch<T, 128, 4, 1, 64, 2, 2>(P, a, s, stream);
  else
    s.tm == 32   ? launch<T, 256, 1, 4, 32, 1, 1>(P, a, s, stream)
    : s.tm == 64 ? launch<T, 256, 2, 2, 32, 1, 1>(P, a, s, stream)
                 : launch<T, 256, 4, 1, 32, 2, 1>(P, a, s, stream);
}

}  // namespace

extern "C" size_t grid_attend_workspace_bytes(const grid_paged_cache* cache, const grid_chunks* chunks,
                                              const grid_attend_args* args) {
  if (check(cache, chunks, args, false) != GRID_OK) return 0;
  return workspace_of(cache, chunks, args, shape_of(cache, chunks, args));
}

extern "C" int grid_attend(const grid_paged_cache* cache, const grid_chunks* chunks, const grid_attend_args* args,
                           void* stream) {
  clear_error();
  const int rc = check(cache, chunks, args, true);
  if (rc != GRID_OK) return rc;
  if (chunks->n_tokens == 0) return GRID_OK;
  const Shape s = shape_of(cache, chunks, args);
  if (!args->workspace || (uintptr_t)args->workspace % 16 != 0 ||
      args->workspace_bytes < workspace_of(cache, chunks, args, s))
    return fail(GRID_E_ARG, "grid_attend: workspace too small or not aligned");
  if (s.blocks > (int64_t)1 << 23) return fail(GRID_E_CAPACITY, "grid_attend: too many tiles for one launch");
  AttendArgs a;
  a.q = (const uint16_t*)args->q;
  a.out = (uint16_t*)args->out;
  for (int i = 0; i < 2; ++i) {
    a.qs[i] = args->q_stride[i];
    a.os[i] = args->out_stride[i];
  }
  a.lse = args->lse;
  a.part_o = (float*)args->workspace;
  a.part_ml = (float2*)(a.part_o + (size_t)s.splits * chunks->n_tokens * args->n_heads * cache->head_dim);
  a.group = Divisor((uint32_t)(args->n_heads / cache->n_kv_heads));
  a.hq = args->n_heads;
  a.max_q = args->max_q;
  a.max_kv = args->max_kv;
  a.window = args->window;
  a.tiles = (int32_t)s.tiles;
  a.splits = s.splits;
  a.len = s.len;
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
