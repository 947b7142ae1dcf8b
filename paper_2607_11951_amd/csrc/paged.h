// paged.h -- the paged cache and the chunks of a batch as the kernels see them.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "host.h"

namespace grid {

int fail(int code, const std::string& msg);
void clear_error();

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// n / d for n < 2^31 as (n * mul) >> shift: with l = ceil(log2 d), mul = floor(2^(31 + l) / d) + 1 exceeds
// 2^(31 + l) / d by at most 1 = 2^l / 2^l, an error of n / 2^(31 + l) * 2^l / d < 1 / d in the quotient.
struct Divisor {
  uint32_t d, mul, shift;
  explicit Divisor(uint32_t div = 1) : d(div) {
    uint32_t l = 0;
    while ((1u << l) < div) ++l;
    mul = (uint32_t)(((uint64_t)1 << (31 + l)) / div + 1);
    shift = 31 + l;
  }
  __host__ __device__ uint32_t quot(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> shift); }
};

struct Paged {
  uint16_t *k, *v;  // both dtypes have 16 bits
  uint32_t ks[3], vs[3];  // page, row, head
  const int32_t* table;
  int64_t table_stride;
  const int32_t* kv_len;
  const int32_t* cu_q;
  Divisor page;
  int32_t n_pages, cols, hkv, D, B, T;
  int64_t reach;  // positions the table has room for

  // where a row of a page lies, in elements from its head's first
  static __device__ uint64_t at(const uint32_t* stride, int page, uint32_t row) {
    return (uint64_t)(uint32_t)page * stride[0] + (uint64_t)row * stride[1];
  }
  // page id of position s (0 <= s < reach) of sequence b: may be out of range, see in_cache
  __device__ int page_of(int b, uint32_t s, uint32_t& row) const {
    const uint32_t c = page.quot(s);
    row = s - c * page.d;
    return table[(int64_t)b * table_stride + c];
  }
  __device__ bool in_cache(int id) const { return (uint32_t)id < (uint32_t)n_pages; }
};

// Checks a cache and chunks; the message names the call.
int check_paged(const char* call, const grid_paged_cache* c, const grid_chunks* x, bool pointers);
Paged make_paged(const grid_paged_cache* c, const grid_chunks* x);
// Whether rows at these strides (elements of 16 bits, below 2^31) can be read 16 bytes at a time.
bool rows_fit(const void* p, const int64_t* strides, int n);

struct Chunk {
  int32_t first, n, kv;  // first token, new tokens, cached tokens with them
  bool ok;
};
// Whether a chunk's first token and end are in the packed arrays, in this order.  From the first chunk on that is not in
// order all are bad: so chunks that are good follow one another, and no token belongs to two.
__device__ inline bool in_order(const Paged& P, int32_t first, int32_t end) {
  return first >= 0 && end >= first && end <= P.T;
}
__device__ inline Chunk chunk_of(const Paged& P, int32_t first, int32_t end, int32_t kv) {
  Chunk c;
  c.first = first;
  c.kv = kv;
  c.ok = in_order(P, first, end);
  c.n = c.ok ? end - first : 0;
  c.ok = c.ok && kv >= c.n && kv <= P.reach;
  return c;
}
// (by itself: the chunks before are not looked at)
__device__ inline Chunk chunk_of(const Paged& P, int b) { return chunk_of(P, P.cu_q[b], P.cu_q[b + 1], P.kv_len[b]); }

// Whether the chunks of the sequences before b are in order, as `all` threads find together of whom this is the one
// `tid`: the first entries are asked for at once, and what is found is told later.  (Entries that do not decrease are in
// order but for the first and the last; where that is past the rows b's own chunk is out of order too, and has no rows.)
struct OrderBefore {
  int32_t zeroth, x, next;
  __device__ OrderBefore(const Paged& P, int b, int tid)
      : zeroth(P.cu_q[0]), x(P.cu_q[min(tid, b)]), next(P.cu_q[min(tid + 1, b)]) {}
  __device__ bool ok(const Paged& P, int b, int tid, int all) const {
    bool down = x > next || (b > 0 && zeroth < 0);
#pragma unroll 4
    for (int s = all + 4 * tid; s < b; s += 4 * all) {
      const int32_t* at = P.cu_q + min(s, b - 4);
      int32_t y[4];
      __builtin_memcpy(y, at, 16);
      const int32_t last = at[4];
      down |= (y[0] > y[1]) | (y[1] > y[2]) | (y[2] > y[3]) | (y[3] > last);
    }
    return !down;
  }
};

// The sequence of token t, and its chunk: not ok if t belongs to none (t may also lie before the chunk).  A whole
// wave asks for one token: the lanes hold the chunks of 64 sequences, and of the first that is not in order or ends after
// t the lane hands its own out.
__device__ inline Chunk chunk_of_token(const Paged& P, int t, int& b) {
  const int lane = (int)threadIdx.x & 63;
  for (b = 0; b < P.B; b += 64) {
    const int x = min(b + lane, P.B - 1);
    const int32_t first = P.cu_q[x], end = P.cu_q[x + 1], kv = P.kv_len[x];
    const uint64_t stop = __ballot(b + lane < P.B && (end > t || !in_order(P, first, end)));
    if (stop) {
      const int i = __builtin_ctzll(stop);
      b += i;
      return chunk_of(P, __builtin_amdgcn_readlane(first, i), __builtin_amdgcn_readlane(end, i),
                      __builtin_amdgcn_readlane(kv, i));
    }
  }
  return {0, 0, 0, false};
}

}  // namespace grid
