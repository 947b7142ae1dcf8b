// pages.hip -- grid_kv_copy and grid_kv_fork: the pages of a cache, copied, forked, freed and given out (gfx950).
//
// Copies take 16 bytes a lane, 8 in flight, in the order of the page's rows (or heads, where these lie further apart).  They are
// bound by bytes: 500 pages of 16 rows, 8 heads of 128, in 32 layers take 412 us, 5.1 TB/s, which is what a plain copy
// reaches; with accesses that are kept in the caches, 592.
//
// A fork is four launches.  The first writes the kept part of the new rows' tables and the reference counts as they were;
// the second counts: pages that a row's parent keeps for itself, which are nearly all, are neither taken out nor put in.  The
// third says for every row whether its last page has to be copied and how many pages it needs, and which pages are free, 64 a
// word; the fourth gives the rows theirs: a row's first is as many free pages on as the rows before it need.
#include <algorithm>
#include <string>

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
  int64_t units;                 // in all: pairs, layers, keys and values, parts
  int32_t page_size, hkv, n_pages, layers, n;
  bool rows_inside;
};

typedef uint32_t Piece __attribute__((ext_vector_type(4)));
constexpr int kAhead = 8;

__global__ __launch_bounds__(kThreads) void copy_kernel(CopyArgs a) {
  const int tid = (int)threadIdx.x;
  for (int64_t u = blockIdx.x; u < a.units; u += gridDim.x) {
    const int64_t whole = u / a.parts.d;
    const int part = (int)(u - whole * a.parts.d), kv = (int)(whole & 1);
    const int i = (int)((whole >> 1) / a.layers), layer = (int)((whole >> 1) - (int64_t)i * a.layers);
    const int src = a.src[i], dst = a.dst[i], rows = a.rows ? min(max(a.rows[i], 0), a.page_size) : a.page_size;
    if ((uint32_t)src >= (uint32_t)a.n_pages || (uint32_t)dst >= (uint32_t)a.n_pages || src == dst) continue;
    uint16_t* base = (kv ? a.v : a.k) + layer * a.layer_stride[kv];
    const uint16_t* from = base + src * a.page_stride[kv];
    uint16_t* to = base + dst * a.page_stride[kv];
    const uint32_t all = (uint32_t)a.page_size * (uint32_t)a.hkv * a.pieces.d;
    Piece x[kAhead];
    int64_t at[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const uint32_t e = (uint32_t)part * (kThreads * kAhead) + (uint32_t)(j * kThreads + tid);
      const uint32_t vec = a.pieces.quot(e), piece = e - vec * a.pieces.d, out = a.inner.quot(vec), in = vec - out * a.inner.d;
      const uint32_t r = a.rows_inside ? in : out, h = a.rows_inside ? out : in;
      at[j] = e < all && r < (uint32_t)rows ? r * a.row_stride[kv] + h * a.head_stride[kv] + piece * 8 : -1;
      if (at[j] >= 0) x[j] = __builtin_nontemporal_load((const Piece*)(from + at[j]));
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (at[j] >= 0) __builtin_nontemporal_store(x[j], (Piece*)(to + at[j]));
  }
}

// -------------------------------------------------------------------------------------------------------------- fork
constexpr int kChunk = 4096;  // pages that a workgroup looks through

struct RowPlan {
  int32_t kept, grow;
  int32_t last;  // the page that the row would write into, or -1
  int32_t need;  // pages, with the copy of `last`
  int32_t copy;
  int32_t bad;
};

struct ForkArgs {
  const int32_t *table, *held, *parent, *keep, *room, *refs;
  int32_t *table_out, *held_out, *refs_out, *copies, *status;
  int64_t ts, os;
  RowPlan* plan;       // [n_rows]
  int32_t* last;       // [n_rows]: of the plans
  uint64_t* free;      // [chunks][kChunk / 64]
  int32_t* free_count; // [chunks]
  Divisor page;
  int32_t n_in, n_rows, cols, n_pages, chunks;
};

__device__ inline int held_of(const ForkArgs& a, int r) { return min(max(a.held[r], 0), a.cols); }
__device__ inline int pages_for(const ForkArgs& a, int tokens) {
  const uint32_t q = a.page.quot((uint32_t)tokens);
  return (int)(q + (q * a.page.d < (uint32_t)tokens));
}
__device__ inline bool is_page(const ForkArgs& a, int p) { return (uint32_t)p < (uint32_t)a.n_pages; }

// The new rows' kept pages, and the counts as they were.
__global__ __launch_bounds__(kThreads) void keep_kernel(ForkArgs a) {
  const int tid = (int)threadIdx.x;
  if ((int)blockIdx.x >= a.n_rows) {
    const int64_t first = (int64_t)((int)blockIdx.x - a.n_rows) * kChunk;
    for (int i = tid; i < kChunk && first + i < a.n_pages; i += kThreads) a.refs_out[first + i] = a.refs[first + i];
    return;
  }
  const int b = (int)blockIdx.x, from = a.parent[b], keep = from < 0 ? 0 : a.keep[b], room = a.room[b];
  bool bad = from < -1 || from >= a.n_in || keep < 0;
  RowPlan p = {0, 0, -1, 0, 0, 0};
  if (!bad) {
    p.kept = pages_for(a, keep);
    p.grow = pages_for(a, max(room, keep)) - p.kept;
    bad = (from >= 0 && p.kept > held_of(a, from)) || p.kept + p.grow > a.cols;
  }
  const int32_t* old = a.table + (int64_t)max(from, 0) * a.ts;
  int32_t* out = a.table_out + b * a.os;
  if (!bad)
    for (int c = tid; c < p.kept; c += kThreads) bad |= !is_page(a, old[c]);
  if (__syncthreads_or(bad)) p = {0, 0, -1, 0, 0, 1};
  for (int c = tid; c < a.cols; c += kThreads) out[c] = c < p.kept ? old[c] : -1;
  if (tid == 0) {
    if (p.kept > 0 && room > keep && (uint32_t)p.kept * a.page.d != (uint32_t)keep) p.last = old[p.kept - 1];
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

__global__ __launch_bounds__(kThreads) void need_kernel(ForkArgs a) {
  const int tid = (int)threadIdx.x, lane = tid & 63;
  if ((int)blockIdx.x >= a.n_rows) {
    __shared__ int32_t counts[kThreads / 64];
    const int chunk = (int)blockIdx.x - a.n_rows;
    int mine = 0;
    for (int w = tid >> 6; w < kChunk / 64; w += kThreads / 64) {
      const int64_t p = (int64_t)chunk * kChunk + w * 64 + lane;
      const uint64_t x = __ballot(p < a.n_pages && a.refs_out[min(p, (int64_t)a.n_pages - 1)] == 0);
      if (lane == 0) a.free[(int64_t)chunk * (kChunk / 64) + w] = x;
      mine += __builtin_popcountll(x);
    }
    if (lane == 0) counts[tid >> 6] = mine;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kThreads / 64; ++w) mine += counts[w];
      a.free_count[chunk] = mine;
    }
    return;
  }
  const int b = (int)blockIdx.x;
  const int last = a.plan[b].last;
  int copy = 0;
  if (last >= 0) {
    const int refs = a.refs_out[last];
    if (refs > 1) {  // others hold it: only rows that write into it, and none before this one?
      __shared__ int32_t writers, before;
      if (tid == 0) writers = before = 0;
      __syncthreads();
      int w = 0, lower = 0;
      for (int r = tid; r < a.n_rows; r += kThreads)
        if (a.last[r] == last) {
          ++w;
          lower += r < b;
        }
      if (w) atomicAdd(&writers, w);
      if (lower) atomicAdd(&before, lower);
      __syncthreads();
      copy = writers != refs || before > 0;
    }
  }
  if (tid == 0) {
    a.plan[b].copy = copy;
    a.plan[b].need = a.plan[b].grow + copy;
  }
}

// The sum of x over the workgroup's threads before this one; `all`: over all of them.
__device__ inline int64_t before_in_block(int64_t x, int64_t* waves, int64_t& all) {
  const int tid = (int)threadIdx.x, lane = tid & 63;
  int64_t upto = x;
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up((long long)upto, o);
    if (lane >= o) upto += y;
  }
  __syncthreads();
  if (lane == 63) waves[tid >> 6] = upto;
  __syncthreads();
  all = 0;
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < tid >> 6) upto += waves[w];
    all += waves[w];
  }
  return upto - x;
}

__global__ __launch_bounds__(kThreads) void give_kernel(ForkArgs a) {
  __shared__ int64_t waves[kThreads / 64], start[kThreads];
  const int tid = (int)threadIdx.x, lane = tid & 63, b = (int)blockIdx.x;
  const RowPlan p = a.plan[b];
  int64_t sum = 0, first, total;
  for (int r = tid; r < b; r += kThreads) sum += a.plan[r].need;
  before_in_block(sum, waves, first);  // pages that the rows before need
  sum = 0;
  for (int c = tid; c < a.chunks; c += kThreads) sum += a.free_count[c];
  before_in_block(sum, waves, total);
  const bool ok = p.need == 0 || first + p.need <= total;
  int32_t* out = a.table_out + b * a.os;
  if (tid == 0) {
    a.status[b] = p.bad ? GRID_ROW_BAD_CONFIG : ok ? GRID_ROW_OK : GRID_ROW_OVERFLOW;
    a.held_out[b] = p.kept + (ok ? p.grow : 0);
    if (!(ok && p.copy)) {
      a.copies[b] = a.copies[a.n_rows + b] = -1;
      a.copies[2 * (int64_t)a.n_rows + b] = 0;
    }
  }
  if (!ok || p.need == 0) return;
  int64_t before = 0;
  for (int c0 = 0; c0 < a.chunks && before < first + p.need; c0 += kThreads) {
    int64_t here;
    const int64_t mine = before_in_block(c0 + tid < a.chunks ? a.free_count[c0 + tid] : 0, waves, here);
    start[tid] = before + mine;
    __syncthreads();
    for (int i = tid >> 6; i < kThreads && c0 + i < a.chunks; i += kThreads / 64) {
      const int64_t at = start[i], end = i + 1 < kThreads ? start[i + 1] : before + here;
      if (end <= first || at >= first + p.need) continue;
      const uint64_t word = a.free[(int64_t)(c0 + i) * (kChunk / 64) + lane];
      int rank = __builtin_popcountll(word);
      const int own = rank;
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(rank, o);
        if (lane >= o) rank += y;
      }
      int64_t n = at + rank - own - first;  // the lane's first free page is the row's n-th
      for (uint64_t x = word; x && n < p.need; x &= x - 1, ++n) {
        if (n < 0) continue;
        const int page = (c0 + i) * kChunk + lane * 64 + __builtin_ctzll(x);
        if (p.copy && n == 0) {
          out[p.kept - 1] = page;
          a.copies[b] = p.last;
          a.copies[a.n_rows + b] = page;
          const uint32_t keep = (uint32_t)a.keep[b];
          a.copies[2 * (int64_t)a.n_rows + b] = (int32_t)(keep - a.page.quot(keep) * a.page.d);
          atomicAdd(a.refs_out + p.last, -1);
        } else {
          out[p.kept + (int)n - p.copy] = page;
        }
        a.refs_out[page] = 1;
      }
    }
    before += here;
    __syncthreads();
  }
}

bool fork_sizes(int32_t n_rows, int32_t n_pages) {
  return n_rows >= 1 && n_rows <= 65535 && n_pages >= 1 && n_pages <= 1 << 26;
}
size_t chunks_of(int32_t n_pages) { return ((size_t)n_pages + kChunk - 1) / kChunk; }

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
  a.units = (int64_t)g.n * g.n_layers * 2 * a.parts.d;
  a.page_size = cache->page_size;
  a.hkv = cache->n_kv_heads;
  a.n_pages = cache->n_pages;
  a.layers = g.n_layers;
  a.n = g.n;
  hipLaunchKernelGGL(copy_kernel, dim3((unsigned)std::min<int64_t>(a.units, 1 << 20)), dim3(kThreads), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_kv_copy launch: ") + hipGetErrorString(e));
  return GRID_OK;
}

extern "C" size_t grid_kv_fork_workspace_bytes(int32_t n_rows, int32_t n_pages) {
  if (!fork_sizes(n_rows, n_pages)) return 0;
  const size_t chunks = chunks_of(n_pages);
  return chunks * (kChunk / 8) + (size_t)n_rows * (sizeof(RowPlan) + 4) + chunks * 4;
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
  a.chunks = (int32_t)chunks_of(g.n_pages);
  a.free = (uint64_t*)g.workspace;
  a.plan = (RowPlan*)(a.free + (size_t)a.chunks * (kChunk / 64));
  a.last = (int32_t*)(a.plan + g.n_rows);
  a.free_count = a.last + g.n_rows;
  const hipStream_t s = (hipStream_t)stream;
  const unsigned rows = (unsigned)g.n_rows, both = (unsigned)std::max(g.n_rows, g.n_in), chunks = (unsigned)a.chunks;
  hipLaunchKernelGGL(keep_kernel, dim3(rows + (g.refs == g.refs_out ? 0 : chunks)), dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(count_kernel, dim3(both), dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(need_kernel, dim3(rows + chunks), dim3(kThreads), 0, s, a);
  hipLaunchKernelGGL(give_kernel, dim3(rows), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_kv_fork launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
