// pages.hip -- grid_kv_copy and grid_kv_fork: the pages of a cache, copied, forked, freed and given out (gfx950).
//
// Copies take 16 bytes a lane, 8 in flight, in the order of the page's rows (or heads, where these lie further apart).  They are
// bound by bytes: 500 pages of 16 rows, 8 heads of 128, in 32 layers take 412 us, 5.1 TB/s, which is what a plain copy
// reaches; with accesses that are kept in the caches, 592.  A workgroup moves 32 KiB, of small pages several pairs: 1000 pages of
// one row, 4 heads of 128, in 48 layers take 39 us, a workgroup a pair 124.
//
// A fork of few rows in a small pool is one workgroup's, with the reference counts in LDS.  Otherwise it is four launches.
// The first writes the kept part of the new rows' tables and the reference counts as they were; the second counts: pages that
// a row's parent keeps for itself, which are nearly all, are neither taken out nor put in.  The third says for every row
// whether its last page has to be copied and how many pages it needs, and which pages are free, 64 a word; the fourth gives
// the rows theirs: a row's first is as many free pages on as the rows before it need.  Forks are bound by reads that wait for
// others and the borders between launches: 512 rows of up to 8192 tokens, pages of 16, take 19.2 us (4.1, 5.1, 3.4 and 7.2 a launch).
// Every row adds up the needs of those before it, and one that shares its last page looks at all rows' last pages: 4096 rows
// that grow take 31 us and forked in pairs 46, 16384 109 and 228, 65535 732 and 1960.
#include <algorithm>
#include <string>

#include "lanes.h"
#include "paged.h"

using namespace grid;

namespace {

constexpr int kThreads = 256;

// -------------------------------------------------------------------------------------------------------------- copy
struct CopyArgs {
  uint16_t *k, *v;
  const int32_t *src, *dst, *rows;
  int64_t page_stride[2], row_stride[2], head_stride[2], layer_stride[2];  // keys', values'
  Divisor parts, inner, pieces;  // workgroups a page and layer; heads (or rows) of a row (or head); pieces of a vector
  Divisor whole;                 // pieces of a page and layer
  int64_t units;                 // in all: groups of pairs, layers, keys and values, parts
  int32_t page_size, hkv, n_pages, layers, n, group;  // group: pairs that a workgroup takes together (small pages)
  bool rows_inside;
};

typedef uint32_t Piece __attribute__((ext_vector_type(4)));
constexpr int kAhead = 8;

// GROUPS: pages of so few pieces that a workgroup takes several pairs.
template <bool GROUPS>
__global__ __launch_bounds__(kThreads) void copy_kernel(CopyArgs a) {
  const int tid = (int)threadIdx.x;
  for (int64_t u = blockIdx.x; u < a.units; u += gridDim.x) {
    const int64_t upper = u / a.parts.d;
    const int part = (int)(u - upper * a.parts.d), kv = (int)(upper & 1);
    const int first = (int)((upper >> 1) / a.layers), layer = (int)((upper >> 1) - (int64_t)first * a.layers);
    uint16_t* base = (kv ? a.v : a.k) + layer * a.layer_stride[kv];
    Piece x[kAhead];
    Piece* to[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      uint32_t e = (uint32_t)part * (kThreads * kAhead) + (uint32_t)(j * kThreads + tid);
      int i = first;
      bool in = true;
      if constexpr (GROUPS) {
        const uint32_t sub = a.whole.quot(e);
        e -= sub * a.whole.d;
        i = first * a.group + (int)sub;
        in = (int)sub < a.group && i < a.n;
        i = min(i, a.n - 1);
      }
      const int src = a.src[i], dst = a.dst[i], rows = a.rows ? min(max(a.rows[i], 0), a.page_size) : a.page_size;
      in = in && (uint32_t)src < (uint32_t)a.n_pages && (uint32_t)dst < (uint32_t)a.n_pages && src != dst && e < a.whole.d;
      const uint32_t vec = a.pieces.quot(e), piece = e - vec * a.pieces.d, out = a.inner.quot(vec), at = vec - out * a.inner.d;
      const uint32_t r = a.rows_inside ? at : out, h = a.rows_inside ? out : at;
      in = in && r < (uint32_t)rows;
      const int64_t offset = r * a.row_stride[kv] + h * a.head_stride[kv] + piece * 8;
      to[j] = in ? (Piece*)(base + dst * a.page_stride[kv] + offset) : nullptr;
      if (in) x[j] = __builtin_nontemporal_load((const Piece*)(base + src * a.page_stride[kv] + offset));
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (to[j]) __builtin_nontemporal_store(x[j], to[j]);
  }
}

// -------------------------------------------------------------------------------------------------------------- fork
struct RowPlan {
  int32_t kept, grow;
  int32_t last;  // the page that the row would write into, or -1
  int32_t copy;
  int32_t bad;
};

struct ForkArgs {
  const int32_t *table, *held, *parent, *keep, *room, *refs;
  int32_t *table_out, *held_out, *refs_out, *copies, *status;
  int64_t ts, os;
  uint64_t* free;       // a bit a page
  int32_t* free_count;  // [chunks]
  int32_t* last;        // [n_rows]: of the plans
  int32_t* need;        // [n_rows]: pages, with the copy of `last`
  RowPlan* plan;        // [n_rows]
  Divisor page;
  int32_t n_in, n_rows, cols, n_pages, chunks, chunk;  // chunk: pages that a workgroup looks through
};

__device__ inline int held_of(const ForkArgs& a, int r) { return min(max(a.held[r], 0), a.cols); }
__device__ inline int pages_for(const ForkArgs& a, int tokens) {
  const uint32_t q = a.page.quot((uint32_t)tokens);
  return (int)(q + (q * a.page.d < (uint32_t)tokens));
}
__device__ inline bool is_page(const ForkArgs& a, int p) { return (uint32_t)p < (uint32_t)a.n_pages; }

// What row b asks for, but for its kept entries, which may be no pages.
__device__ inline RowPlan plan_of(const ForkArgs& a, int b, int& from, int& keep) {
  from = a.parent[b];
  keep = from < 0 ? 0 : a.keep[b];
  RowPlan p = {0, 0, -1, 0, 0};
  p.bad = from < -1 || from >= a.n_in || keep < 0;
  if (!p.bad) {
    p.kept = pages_for(a, keep);
    p.grow = pages_for(a, max(a.room[b], keep)) - p.kept;
    p.bad = (from >= 0 && p.kept > held_of(a, from)) || p.kept + p.grow > a.cols;
  }
  return p;
}
// Whether a row that keeps so much writes into the last of its kept pages.
__device__ inline bool writes_on(const ForkArgs& a, const RowPlan& p, int b, int keep) {
  return p.kept > 0 && a.room[b] > keep && (uint32_t)p.kept * a.page.d != (uint32_t)keep;
}
__device__ inline int rows_in_last(const ForkArgs& a, int keep) {
  return (int)((uint32_t)keep - a.page.quot((uint32_t)keep) * a.page.d);
}

// The new rows' kept pages, and the counts as they were.
__global__ __launch_bounds__(kThreads) void keep_kernel(ForkArgs a) {
  const int tid = (int)threadIdx.x;
  if ((int)blockIdx.x >= a.n_rows) {
    const int64_t first = (int64_t)((int)blockIdx.x - a.n_rows) * a.chunk;
#pragma unroll 4
    for (int i = tid; i < a.chunk; i += kThreads)
      if (first + i < a.n_pages) a.refs_out[first + i] = a.refs[first + i];
    return;
  }
  const int b = (int)blockIdx.x;
  int from, keep;
  RowPlan p = plan_of(a, b, from, keep);
  bool bad = p.bad;
  const int32_t* old = a.table + (int64_t)(bad ? 0 : max(from, 0)) * a.ts;
  int32_t* out = a.table_out + b * a.os;
  if (!bad)
    for (int c = tid; c < p.kept; c += kThreads) bad |= !is_page(a, old[c]);
  if (__syncthreads_or(bad)) p = {0, 0, -1, 0, 1};
  for (int c = tid; c < a.cols; c += kThreads) out[c] = c < p.kept ? old[c] : -1;
  if (tid == 0) {
    if (writes_on(a, p, b, keep)) p.last = old[p.kept - 1];
    a.plan[b] = p;
    a.last[b] = p.last;
  }
}

// What the old rows give up and what the new ones take from others.
__global__ __launch_bounds__(kThreads) void count_kernel(ForkArgs a) {
  const int tid = (int)threadIdx.x, r = (int)blockIdx.x;
  const int kept = r < a.n_rows ? a.plan[r].kept : 0, from = r < a.n_rows ? a.parent[r] : -1;
  if (r < a.n_in) {
    const int32_t* old = a.table + r * a.ts;
    for (int c = (from == r ? kept : 0) + tid; c < held_of(a, r); c += kThreads)
      if (is_page(a, old[c])) atomicAdd(a.refs_out + old[c], -1);
  }
  if (r < a.n_rows && from != r) {
    const int32_t* mine = a.table_out + r * a.os;
    for (int c = tid; c < kept; c += kThreads) atomicAdd(a.refs_out + mine[c], 1);
  }
}

// Whether row b, that would write into page `last` which `refs` hold, has to copy it: others than rows that write hold it,
// or one of these comes before.  Asked by N threads together, of whom this is the one `tid`; add: their sum.
template <int N, typename Add>
__device__ inline bool copies_last(const int32_t* lasts, int n_rows, int b, int last, int refs, int tid, Add add) {
  uint32_t x = 0;  // rows that write into it, and those of them before b
  uint32_t y = 0;
  for (int r = tid; r < n_rows; r += N)
    if (lasts[r] == last) {
      ++x;
      y += r < b;
    }
  x = add(x);
  y = add(y);
  return x != (uint32_t)refs || y > 0;
}

__global__ __launch_bounds__(kThreads) void need_kernel(ForkArgs a) {
  __shared__ uint32_t sums[kThreads / 64];
  const int tid = (int)threadIdx.x, lane = tid & 63;
  const auto add = [&](uint32_t x) {  // over the workgroup
    x = across(x, [](uint32_t p, uint32_t q) { return p + q; });
    __syncthreads();
    if (lane == 0) sums[tid >> 6] = x;
    __syncthreads();
    x = 0;
    for (int w = 0; w < kThreads / 64; ++w) x += sums[w];
    return x;
  };
  if ((int)blockIdx.x >= a.n_rows) {
    const int chunk = (int)blockIdx.x - a.n_rows;
    uint32_t mine = 0;
#pragma unroll 4
    for (int w = tid >> 6; w < a.chunk / 64; w += kThreads / 64) {
      const int64_t p = (int64_t)chunk * a.chunk + w * 64 + lane;
      const uint64_t x = __ballot(p < a.n_pages && a.refs_out[min(p, (int64_t)a.n_pages - 1)] == 0);
      if (lane == 0) a.free[(int64_t)chunk * (a.chunk / 64) + w] = x;
      if (lane == 0) mine += (uint32_t)__builtin_popcountll(x);
    }
    mine = add(mine);
    if (tid == 0) a.free_count[chunk] = (int)mine;
    return;
  }
  const int b = (int)blockIdx.x, last = a.last[b];
  int copy = 0;
  if (last >= 0) {
    const int refs = a.refs_out[last];
    if (refs > 1) copy = copies_last<kThreads>(a.last, a.n_rows, b, last, refs, tid, add);
  }
  if (tid == 0) {
    a.plan[b].copy = copy;
    a.need[b] = a.plan[b].grow + copy;
  }
}

// Row b's n-th new page (of its need, a copy first).
__device__ inline void give(const ForkArgs& a, const RowPlan& p, int b, int n, int page) {
  int32_t* out = a.table_out + b * a.os;
  if (p.copy && n == 0) {
    out[p.kept - 1] = page;
    a.copies[b] = p.last;
    a.copies[a.n_rows + b] = page;
    a.copies[2 * (int64_t)a.n_rows + b] = rows_in_last(a, a.keep[b]);
  } else {
    out[p.kept + n - p.copy] = page;
  }
}
__device__ inline void say(const ForkArgs& a, const RowPlan& p, int b, bool ok) {
  a.status[b] = p.bad ? GRID_ROW_BAD_CONFIG : ok ? GRID_ROW_OK : GRID_ROW_OVERFLOW;
  a.held_out[b] = p.kept + (ok ? p.grow : 0);
  if (!(ok && p.copy)) {
    a.copies[b] = a.copies[a.n_rows + b] = -1;
    a.copies[2 * (int64_t)a.n_rows + b] = 0;
  }
}

__global__ __launch_bounds__(kThreads) void give_kernel(ForkArgs a) {
  __shared__ uint64_t waves[kThreads / 64], start[kThreads];
  __shared__ int hits[kThreads], n_hits;
  const int tid = (int)threadIdx.x, lane = tid & 63, b = (int)blockIdx.x;
  // the sum over the threads up to and with this one; all: over all
  const auto upto = [&](uint64_t x, uint64_t& all) {
    uint64_t sum = sum_upto(x);
    __syncthreads();
    if (lane == 63) waves[tid >> 6] = sum;
    __syncthreads();
    all = 0;
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < tid >> 6) sum += waves[w];
      all += waves[w];
    }
    return sum;
  };
  // the first pages' counts and the needs of the rows before are asked for together
  uint64_t before = 0, free = 0, first, total;
  const uint64_t count = tid < a.chunks ? (uint64_t)a.free_count[tid] : 0;
  for (int r = tid; r < b; r += kThreads) before += (uint64_t)a.need[r];
  for (int c = kThreads + tid; c < a.chunks; c += kThreads) free += (uint64_t)a.free_count[c];
  const RowPlan p = a.plan[b];
  const uint64_t need = (uint64_t)(p.grow + p.copy);
  upto(before, first);
  upto(count + free, total);
  const bool ok = need == 0 || first + need <= total;
  if (tid == 0) say(a, p, b, ok);
  if (!ok || need == 0) return;
  uint64_t seen = 0;
  for (int c0 = 0; c0 < a.chunks && seen < first + need; c0 += kThreads) {
    uint64_t here;
    const uint64_t own = c0 == 0 ? count : c0 + tid < a.chunks ? (uint64_t)a.free_count[c0 + tid] : 0;
    const uint64_t begin = seen + upto(own, here) - own;
    if (tid == 0) n_hits = 0;
    __syncthreads();
    if (own > 0 && begin + own > first && begin < first + need) {  // (in any order)
      const int at = atomicAdd(&n_hits, 1);
      hits[at] = c0 + tid;
      start[at] = begin;
    }
    __syncthreads();
    for (int i = tid >> 6; i < n_hits; i += kThreads / 64) {
      const int chunk = hits[i];
      uint64_t at = start[i];
      for (int w = 0; w < a.chunk / 64 && at < first + need; w += 64) {
        const uint64_t word = w + lane < a.chunk / 64 ? a.free[(int64_t)chunk * (a.chunk / 64) + w + lane] : 0;
        const uint32_t own = (uint32_t)__builtin_popcountll(word), rank = sum_upto(own);
        int64_t n = (int64_t)(at + rank - own) - (int64_t)first;  // the lane's first free page is the row's n-th
        for (uint64_t x = word; x && n < (int64_t)need; x &= x - 1, ++n) {
          if (n < 0) continue;
          const int page = chunk * a.chunk + (w + lane) * 64 + __builtin_ctzll(x);
          if (p.copy && n == 0) atomicAdd(a.refs_out + p.last, -1);
          give(a, p, b, (int)n, page);
          a.refs_out[page] = 1;
        }
        at += (uint32_t)__builtin_amdgcn_readlane((int)rank, 63);
      }
    }
    seen += here;
    __syncthreads();
  }
}

// Few rows in a small pool: one workgroup.
constexpr int kFewThreads = 1024, kFewRows = 32, kFewPages = 16384, kFewEntries = 16384;
__global__ __launch_bounds__(kFewThreads) void few_kernel(ForkArgs a) {
  __shared__ int32_t refs[kFewPages];
  __shared__ uint64_t free[kFewPages / 64];
  __shared__ uint32_t upto[kFewPages / 64 + 1], waves[kFewThreads / 64];  // free pages before a word
  __shared__ RowPlan plans[kFewRows];
  __shared__ int32_t lasts[kFewRows];
  __shared__ uint32_t first[kFewRows + 1];  // pages that the rows before need
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
  constexpr int W = kFewThreads / 64;
  for (int p = tid; p < a.n_pages; p += kFewThreads) refs[p] = a.refs[p];
  for (int b = wave; b < a.n_rows; b += W) {
    int from, keep;
    RowPlan p = plan_of(a, b, from, keep);
    bool bad = p.bad;
    const int32_t* old = a.table + (int64_t)(bad ? 0 : max(from, 0)) * a.ts;
    if (!bad)
      for (int c = lane; c < p.kept; c += 64) bad |= !is_page(a, old[c]);
    if (__any(bad)) p = {0, 0, -1, 0, 1};
    for (int c = lane; c < a.cols; c += 64) a.table_out[b * a.os + c] = c < p.kept ? old[c] : -1;
    if (lane == 0) {
      if (writes_on(a, p, b, keep)) p.last = old[p.kept - 1];
      plans[b] = p;
      lasts[b] = p.last;
    }
  }
  __syncthreads();
  for (int r = wave; r < max(a.n_in, a.n_rows); r += W) {
    const int kept = r < a.n_rows ? plans[r].kept : 0, from = r < a.n_rows ? a.parent[r] : -1;
    if (r < a.n_in)
      for (int c = (from == r ? kept : 0) + lane; c < held_of(a, r); c += 64) {
        const int p = a.table[r * a.ts + c];
        if (is_page(a, p)) atomicAdd(refs + p, -1);
      }
    if (r < a.n_rows && from != r)
      for (int c = lane; c < kept; c += 64) atomicAdd(refs + a.table[from * a.ts + c], 1);
  }
  __syncthreads();
  const auto scan = [&](uint32_t x, uint32_t& all) {  // before this thread
    uint32_t sum = sum_upto(x);
    __syncthreads();
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    all = 0;
    for (int w = 0; w < W; ++w) {
      if (w < wave) sum += waves[w];
      all += waves[w];
    }
    return sum - x;
  };
  const int words = (a.n_pages + 63) / 64;
  for (int w = wave; w < words; w += W) {
    const int p = w * 64 + lane;
    const uint64_t x = __ballot(p < a.n_pages && refs[min(p, a.n_pages - 1)] == 0);
    if (lane == 0) free[w] = x;
  }
  for (int b = wave; b < a.n_rows; b += W) {
    const int last = lasts[b], held = last >= 0 ? refs[last] : 0;
    int copy = 0;
    if (held > 1)
      copy = copies_last<64>(lasts, a.n_rows, b, last, held, lane,
                             [](uint32_t x) { return across(x, [](uint32_t p, uint32_t q) { return p + q; }); });
    if (lane == 0) plans[b].copy = copy;
  }
  __syncthreads();
  uint32_t total, all;
  const uint32_t before = scan(tid < words ? (uint32_t)__builtin_popcountll(free[tid]) : 0, total);
  if (tid < words) upto[tid] = before;
  const uint32_t needs = scan(tid < a.n_rows ? (uint32_t)(plans[tid].grow + plans[tid].copy) : 0, all);
  if (tid < a.n_rows) first[tid] = needs;
  __syncthreads();
  for (int b = wave; b < a.n_rows; b += W) {
    const RowPlan p = plans[b];
    const uint32_t need = (uint32_t)(p.grow + p.copy);
    const bool ok = need == 0 || first[b] + need <= total;
    if (lane == 0) say(a, p, b, ok);
    if (!ok) continue;
    for (uint32_t n = (uint32_t)lane; n < need; n += 64) {
      // the word that has the free page of this rank, and the page
      uint32_t rank = first[b] + n;
      int lo = 0, hi = words;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (upto[mid] <= rank ? lo : hi) = mid;
      }
      uint64_t x = free[lo];
      for (rank -= upto[lo]; rank > 0; --rank) x &= x - 1;
      const int page = lo * 64 + __builtin_ctzll(x);
      if (p.copy && n == 0) atomicAdd(refs + p.last, -1);
      give(a, p, b, (int)n, page);
      refs[page] = 1;
    }
  }
  __syncthreads();
  for (int p = tid; p < a.n_pages; p += kFewThreads) a.refs_out[p] = refs[p];
}

bool fork_sizes(int32_t n_rows, int32_t n_pages) {
  return n_rows >= 1 && n_rows <= 65535 && n_pages >= 1 && n_pages <= 1 << 26;
}
// 1024 pages a chunk, or as many more as give 1024 chunks at most.
int chunk_of_pages(int32_t n_pages) {
  int chunk = 1024;
  while ((int64_t)chunk * 1024 < n_pages) chunk *= 2;
  return chunk;
}

}  // namespace

extern "C" int grid_kv_copy(const grid_paged_cache* cache, const grid_copy_args* args, void* stream) {
  clear_error();
  auto bad = [](const char* what) { return fail(GRID_E_ARG, std::string("grid_kv_copy: ") + what); };
  const int rc = check_cache("grid_kv_copy", cache, true);
  if (rc != GRID_OK) return rc;
  if (!args) return bad("null argument");
  const grid_copy_args& g = *args;
  if (g.n < 0 || g.n > 1 << 20) return bad("0 to 2^20 pairs");
  if (g.n_layers < 1 || g.n_layers > 1024) return bad("1 to 1024 layers");
  if (!layers_fit(g.n_layers, g.k_layer_stride, g.v_layer_stride)) return bad("layer strides");
  if (g.n == 0) return GRID_OK;
  if (!g.src || !g.dst) return bad("null pointer");
  CopyArgs a;
  a.k = (uint16_t*)cache->k_pages;
  a.v = (uint16_t*)cache->v_pages;
  a.src = g.src;
  a.dst = g.dst;
  a.rows = g.rows;
  for (int i = 0; i < 2; ++i) {
    const int64_t* s = i ? cache->v_stride : cache->k_stride;
    a.page_stride[i] = s[0];
    a.row_stride[i] = s[1];
    a.head_stride[i] = s[2];
    a.layer_stride[i] = i ? g.v_layer_stride : g.k_layer_stride;
  }
  a.rows_inside = a.head_stride[0] > a.row_stride[0];
  a.pieces = Divisor((uint32_t)cache->head_dim / 8);
  a.inner = Divisor((uint32_t)(a.rows_inside ? cache->page_size : cache->n_kv_heads));
  const int64_t all = (int64_t)cache->page_size * cache->n_kv_heads * (cache->head_dim / 8);
  if (all >= (int64_t)1 << 30) return fail(GRID_E_CAPACITY, "grid_kv_copy: a page has 2^30 pieces of 16 bytes or more");
  a.parts = Divisor((uint32_t)((all + kThreads * kAhead - 1) / (kThreads * kAhead)));
  a.whole = Divisor((uint32_t)all);
  a.group = (int32_t)std::max<int64_t>(1, kThreads * kAhead / all);
  a.units = (int64_t)((g.n + a.group - 1) / a.group) * g.n_layers * 2 * a.parts.d;
  a.page_size = cache->page_size;
  a.hkv = cache->n_kv_heads;
  a.n_pages = cache->n_pages;
  a.layers = g.n_layers;
  a.n = g.n;
  const dim3 blocks((unsigned)std::min<int64_t>(a.units, 1 << 20));
  if (a.group > 1)
    hipLaunchKernelGGL(copy_kernel<true>, blocks, dim3(kThreads), 0, (hipStream_t)stream, a);
  else
    hipLaunchKernelGGL(copy_kernel<false>, blocks, dim3(kThreads), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_kv_copy launch: ") + hipGetErrorString(e));
  return GRID_OK;
}

extern "C" size_t grid_kv_fork_workspace_bytes(int32_t n_rows, int32_t n_pages) {
  if (!fork_sizes(n_rows, n_pages)) return 0;
  const size_t chunk = (size_t)chunk_of_pages(n_pages), chunks = ((size_t)n_pages + chunk - 1) / chunk;
  return chunks * (chunk / 8 + 4) + (size_t)n_rows * (sizeof(RowPlan) + 8);
}

extern "C" int grid_kv_fork(const grid_fork_args* args, void* stream) {
  clear_error();
  auto bad = [](const char* what) { return fail(GRID_E_ARG, std::string("grid_kv_fork: ") + what); };
  if (!args) return bad("null argument");
  const grid_fork_args& g = *args;
  if (!fork_sizes(g.n_rows, g.n_pages) || g.n_in < 1 || g.n_in > 65535) return bad("rows or pages");
  if (g.page_size < 1 || g.page_size > 65536) return bad("page_size");
  if (g.table_cols < 1 || (int64_t)g.table_cols * g.page_size > INT32_MAX) return bad("the block table has 2^31 positions or more");
  if (g.table_stride < g.table_cols || g.table_out_stride < g.table_cols) return bad("table strides");
  if (!g.table || !g.held || !g.parent || !g.keep || !g.room || !g.refs || !g.table_out || !g.held_out || !g.refs_out ||
      !g.copies || !g.status)
    return bad("null pointer");
  if (g.table == g.table_out || g.held == g.held_out) return bad("the new table and numbers are arrays of their own");
  if (!g.workspace || (uintptr_t)g.workspace % 16 != 0 ||
      g.workspace_bytes < grid_kv_fork_workspace_bytes(g.n_rows, g.n_pages))
    return bad("workspace too small or not aligned");
  ForkArgs a;
  a.table = g.table;
  a.held = g.held;
  a.parent = g.parent;
  a.keep = g.keep;
  a.room = g.room;
  a.refs = g.refs;
  a.table_out = g.table_out;
  a.held_out = g.held_out;
  a.refs_out = g.refs_out;
  a.copies = g.copies;
  a.status = g.status;
  a.ts = g.table_stride;
  a.os = g.table_out_stride;
  a.page = Divisor((uint32_t)g.page_size);
  a.n_in = g.n_in;
  a.n_rows = g.n_rows;
  a.cols = g.table_cols;
  a.n_pages = g.n_pages;
  a.chunk = chunk_of_pages(g.n_pages);
  a.chunks = (g.n_pages + a.chunk - 1) / a.chunk;
  a.free = (uint64_t*)g.workspace;
  a.free_count = (int32_t*)(a.free + (size_t)a.chunks * (size_t)(a.chunk / 64));
  a.last = a.free_count + a.chunks;
  a.need = a.last + g.n_rows;
  a.plan = (RowPlan*)(a.need + g.n_rows);
  const hipStream_t s = (hipStream_t)stream;
  const unsigned rows = (unsigned)g.n_rows, both = (unsigned)std::max(g.n_rows, g.n_in), chunks = (unsigned)a.chunks;
  // One workgroup takes 7.4 us for 8 rows of 700 tokens and 14.1 for 32 of 1500 (pages of 16), four launches 15.1 and 16.0; for
  // 64 rows of 1500 it would take 25.9, for 16 of 8192 14.5, they 17.9 and 16.5.
  if (std::max(g.n_rows, g.n_in) <= kFewRows && g.n_pages <= kFewPages &&
      (int64_t)(g.n_rows + g.n_in) * g.table_cols <= kFewEntries) {
    hipLaunchKernelGGL(few_kernel, dim3(1), dim3(kFewThreads), 0, s, a);
  } else {
    hipLaunchKernelGGL(keep_kernel, dim3(rows + (g.refs == g.refs_out ? 0 : chunks)), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(count_kernel, dim3(both), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(need_kernel, dim3(rows + chunks), dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL(give_kernel, dim3(rows), dim3(kThreads), 0, s, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_kv_fork launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
