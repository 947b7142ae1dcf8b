// tree.hip -- grid_tree_masks and grid_commit_tree: what a step with a tree of drafts needs before and after the model (gfx950).
//
// A node comes after its parent, so a chain of parents is one of falling places.  A wave takes 64 places and finds the
// ancestors among these of each, twice as many a step, and the first ancestor before them; a node's words are then those of
// at most one place in every 64.  For the branch that the target's tokens follow each node tells its parent if it is such a
// child, the lowest place counts, and the path is followed; every workgroup of a sequence does so for itself, and moves
// its columns of the rows: a thread has the same 16 bytes of all rows, so those it writes are those it has read before.
//
// The masks are bound by a handful of dependent reads (32 trees of 64 nodes 3.4 us, one of 1024, a chain, 22; followed place by
// place 134), and so is the commit of few sequences (a chain of 64 nodes, all kept, 7 us; with a search of the chunk a node 20).
// 64 trees of up to 64 nodes, 8 heads of 128 in 32 layers, take 14 us: 5 until the branches are known, then their bytes (with
// rows that the caches keep, which nobody reads soon, 5 more).
#include <algorithm>
#include <string>

#include "paged.h"

using namespace grid;

namespace {

constexpr int kThreads = 256;
constexpr int kMost = 1024;  // nodes of a tree
constexpr int kNone = 0x7FFFFFFF;
typedef uint32_t Piece __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------------------------------- masks
struct MaskArgs {
  const int32_t* parent;
  uint32_t* masks;
  int32_t* depth;
  int64_t stride;
  int32_t max_q, words, window;  // window: bits of a node, the nearest ancestors', at most
};

__global__ __launch_bounds__(kThreads) void masks_kernel(Paged P, MaskArgs a) {
  __shared__ uint64_t bits[kMost];  // a place and its ancestors among its 64
  __shared__ int32_t out[kMost];    // the first ancestor before these, -1: none
  const int b = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63;
  const int32_t first = P.cu_q[b], end = P.cu_q[b + 1];
  const OrderBefore before(P, b, tid);
  if (__syncthreads_or(!before.ok(P, b, tid, kThreads))) return;  // the first that is not in order has these rows
  const bool ordered = in_order(P, first, end), tree = ordered && end - first <= a.max_q;
  const int from = min(max(first, 0), P.T), n = (ordered ? end : P.T) - from;
  if (tree) {
    for (int base = tid & ~63; base < n; base += kThreads) {
      const int i = base + lane;
      int p = i < n ? a.parent[from + i] : -1;
      if (p < 0 || p >= i) p = -1;
      // x: the places from i up to q, the next ancestor's lane (-1: all of them); p: then the first before
      uint64_t x = 1ull << lane;
      int q = p >= base ? p - base : -1;
      while (__any(q >= 0)) {
        const int next = q >= 0 ? q : lane;
        const uint64_t y = (uint64_t)__shfl((unsigned long long)x, next);
        const int out_of = __shfl(p, next), after = __shfl(q, next);
        if (q >= 0) x |= y, p = out_of, q = after;
      }
      if (i < n) bits[i] = x, out[i] = p;
    }
    __syncthreads();
  }
  for (int i = tid; i < n; i += kThreads) {
    uint32_t* words = a.masks + (int64_t)(from + i) * a.stride;
    int at = tree ? i : -1, deep = -1;
    for (int w = (a.words - 1) / 2; w >= 0; --w) {
      uint64_t x = 0;
      if (at >= w * 64) {
        x = bits[at];
        at = out[at];
        deep += __builtin_popcountll(x);
        // the lowest places are the furthest ancestors: what lies past the window goes
        for (int past = min(deep + 1 - a.window, __builtin_popcountll(x)); past > 0; --past) x &= x - 1;
      }
      words[2 * w] = (uint32_t)x;
      if (2 * w + 1 < a.words) words[2 * w + 1] = (uint32_t)(x >> 32);
    }
    a.depth[from + i] = max(deep, 0);
  }
}

// ------------------------------------------------------------------------------------------------------------ commit
struct CommitArgs {
  const int32_t *tokens, *parent, *sampled, *start;
  int32_t *path, *length, *next;
  int64_t path_stride, k_layer, v_layer;
  Divisor pieces;  // 16-byte pieces of a head's vector
  int32_t max_q, layers, parts;
};

// A workgroup a sequence, a layer and a part of the columns (16-byte pieces of a row of keys and values).
__global__ __launch_bounds__(kThreads) void commit_kernel(Paged P, CommitArgs a) {
  __shared__ int32_t up[kMost], said[kMost], child[kMost], path[kMost], page[kMost];  // child: that the branch takes, or kNone
  __shared__ int found;
  const int tid = (int)threadIdx.x, lane = tid & 63;
  const int part = (int)(blockIdx.x % (uint32_t)a.parts), b = (int)(blockIdx.x / (uint32_t)a.parts), layer = (int)blockIdx.y;
  const int32_t first = P.cu_q[b], end = P.cu_q[b + 1];
  const OrderBefore before(P, b, tid);
  const bool ordered = !__syncthreads_or(!before.ok(P, b, tid, kThreads));
  Chunk c = {first, end - first, 0, ordered && in_order(P, first, end)};
  if (c.ok && a.layers > 0) c = chunk_of(P, first, end, P.kv_len[b]);
  const int from = a.start ? a.start[b] : 0;
  const int n = c.ok && c.n <= a.max_q && from >= 0 && from < c.n ? c.n : 0;
  constexpr int kEach = kMost / kThreads;
  int32_t token[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = tid + k * kThreads;
    token[k] = -1;
    if (i >= n) continue;
    const int32_t p = a.parent[first + i];
    token[k] = a.tokens[first + i];
    up[i] = p >= 0 && p < i ? p : -1;
    said[i] = a.sampled[first + i];
    child[i] = kNone;
    if (a.layers > 0) {
      uint32_t row;
      page[i] = P.page_of(b, (uint32_t)(c.kv - c.n + i), row);
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = tid + k * kThreads;
    if (token[k] >= 0 && up[i] >= 0 && said[up[i]] == token[k]) atomicMin(&child[up[i]], i);
  }
  __syncthreads();
  if (tid < 64) {
    int length = 0, at = -1;
    if (n > 0) {
      for (int i = from; i >= 0; i = up[i]) ++length;
      int j = length;
      for (int i = from; i >= 0; i = up[i]) {
        --j;
        if (lane == 0) path[j] = i;
      }
      at = from;
      if (n <= 64) {
        const int mine = lane < n ? child[lane] : kNone;
        for (int c; (c = __builtin_amdgcn_readlane(mine, at)) != kNone; at = c, ++length)
          if (lane == 0) path[length] = c;
      } else {
        for (int c; (c = child[at]) != kNone; at = c, ++length)
          if (lane == 0) path[length] = c;
      }
    }
    if (lane == 0) {
      found = length;
      if (part == 0 && layer == 0) {
        a.length[b] = length;
        a.next[b] = length > 0 ? said[at] : -1;
      }
    }
  }
  __syncthreads();
  const int length = found;
  if (part == 0 && layer == 0)
    for (int i = tid; i < a.max_q; i += kThreads) a.path[(int64_t)b * a.path_stride + i] = i < length ? path[i] : -1;
  if (a.layers == 0) return;
  const int columns = P.hkv * (int)a.pieces.d, u = part * kThreads + tid;
  if (u >= 2 * columns) return;
  const bool key = u < columns;
  const uint32_t column = (uint32_t)(key ? u : u - columns), head = a.pieces.quot(column), piece = column - head * a.pieces.d;
  uint16_t* base = (key ? P.k + layer * a.k_layer : P.v + layer * a.v_layer) + piece * 8;
  const uint32_t stride[3] = {key ? P.ks[0] : P.vs[0], key ? P.ks[1] : P.vs[1], key ? P.ks[2] : P.vs[2]};
  const uint64_t from_head = (uint64_t)head * stride[2];
  const int text = c.kv - c.n;  // cached tokens before the chunk
  constexpr int AHEAD = 8;
  for (int i = 0; i < length; i += AHEAD) {
    Piece x[AHEAD];
    Piece* to[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      to[j] = nullptr;
      if (i + j >= length || path[i + j] == i + j) continue;
      const int p = page[path[i + j]], q = page[i + j];
      if (!P.in_cache(p) || !P.in_cache(q)) continue;
      const uint32_t s = (uint32_t)(text + path[i + j]), t = (uint32_t)(text + i + j);
      x[j] = __builtin_nontemporal_load((const Piece*)(base + P.at(stride, p, s - P.page.quot(s) * P.page.d) + from_head));
      to[j] = (Piece*)(base + P.at(stride, q, t - P.page.quot(t) * P.page.d) + from_head);
    }
    // (a row's place is before those that the later ones come from)
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (to[j]) __builtin_nontemporal_store(x[j], to[j]);
  }
}

}  // namespace

// Chunks by themselves.
static Paged no_cache(const int32_t* cu_q, int32_t n_seqs, int32_t n_tokens) {
  Paged p;
  p.k = p.v = nullptr;
  for (int i = 0; i < 3; ++i) p.ks[i] = p.vs[i] = 0;
  p.table = p.kv_len = nullptr;
  p.table_stride = p.reach = 0;
  p.n_pages = p.cols = p.hkv = p.D = 0;
  p.cu_q = cu_q;
  p.B = n_seqs;
  p.T = n_tokens;
  return p;
}

static int tree_masks(const std::string& call, const grid_tree_args* args, int32_t window, void* stream) {
  auto bad = [&](const char* what) { return fail(GRID_E_ARG, call + ": " + what); };
  if (!args) return bad("null argument");
  if (window < 0) return bad("window");
  const grid_tree_args& g = *args;
  if (g.n_seqs < 1 || g.n_seqs > 65535) return bad("1 to 65535 sequences");
  if (g.n_tokens < 0 || g.n_tokens > 1 << 24) return bad("n_tokens");
  if (g.max_q < 1 || g.max_q > kMost) return bad("max_q is 1 to 1024");
  if (g.stride_words < (g.max_q + 31) / 32) return bad("fewer words than max_q bits");
  if (!g.cu_q) return bad("null pointer");
  if (g.n_tokens == 0) return GRID_OK;
  if (!g.parent || !g.masks || !g.depth) return bad("null pointer");
  const Paged P = no_cache(g.cu_q, g.n_seqs, g.n_tokens);
  MaskArgs a;
  a.parent = g.parent;
  a.masks = g.masks;
  a.depth = g.depth;
  a.stride = g.stride_words;
  a.max_q = g.max_q;
  a.words = (g.max_q + 31) / 32;
  a.window = window ? window : kMost;
  hipLaunchKernelGGL(masks_kernel, dim3((unsigned)g.n_seqs), dim3(kThreads), 0, (hipStream_t)stream, P, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, call + " launch: " + hipGetErrorString(e));
  return GRID_OK;
}

extern "C" int grid_tree_masks(const grid_tree_args* args, void* stream) {
  clear_error();
  return tree_masks("grid_tree_masks", args, 0, stream);
}

extern "C" int grid_tree_masks_window(const grid_tree_args* args, int32_t window, void* stream) {
  clear_error();
  return tree_masks("grid_tree_masks_window", args, window, stream);
}

extern "C" int grid_commit_tree(const grid_paged_cache* cache, const grid_chunks* chunks, const grid_commit_args* args,
                                void* stream) {
  clear_error();
  auto bad = [](const char* what) { return fail(GRID_E_ARG, std::string("grid_commit_tree: ") + what); };
  if (!args) return bad("null argument");
  const grid_commit_args& g = *args;
  if (g.n_layers < 0 || g.n_layers > 1024) return bad("0 to 1024 layers");
  if (g.max_q < 1 || g.max_q > kMost) return bad("max_q is 1 to 1024");
  if (g.path_stride < g.max_q) return bad("path_stride");
  if (!g.path || !g.length || !g.next) return bad("null pointer");
  Paged P;
  if (g.n_layers > 0) {
    const int rc = check_paged("grid_commit_tree", cache, chunks, true);
    if (rc != GRID_OK) return rc;
    if (!layers_fit(g.n_layers, g.k_layer_stride, g.v_layer_stride)) return bad("layer strides");
    P = make_paged(cache, chunks);
  } else {
    if (!chunks || !chunks->cu_q) return bad("null argument");
    if (chunks->n_seqs < 1 || chunks->n_seqs > 65535) return bad("1 to 65535 sequences");
    if (chunks->n_tokens < 0 || chunks->n_tokens > 1 << 24) return bad("n_tokens");
    P = no_cache(chunks->cu_q, chunks->n_seqs, chunks->n_tokens);
  }
  if (P.T > 0 && (!g.tokens || !g.parent || !g.sampled)) return bad("null pointer");
  CommitArgs a;
  a.tokens = g.tokens;
  a.parent = g.parent;
  a.sampled = g.sampled;
  a.start = g.start;
  a.path = g.path;
  a.length = g.length;
  a.next = g.next;
  a.path_stride = g.path_stride;
  a.k_layer = g.k_layer_stride;
  a.v_layer = g.v_layer_stride;
  a.max_q = g.max_q;
  a.layers = g.n_layers;
  a.pieces = Divisor((uint32_t)std::max(1, P.D / 8));
  a.parts = g.n_layers > 0 ? (2 * P.hkv * (P.D / 8) + kThreads - 1) / kThreads : 1;
  // (65535 sequences of 256 parts at most, below 2^24 workgroups; a launch has less than 2^32 threads in all)
  const dim3 all((unsigned)P.B * (unsigned)a.parts, (unsigned)std::max(1, g.n_layers));
  if ((uint64_t)all.x * all.y > 1u << 23) return fail(GRID_E_CAPACITY, "grid_commit_tree: too many rows for one launch");
  hipLaunchKernelGGL(commit_kernel, all, dim3(kThreads), 0, (hipStream_t)stream, P, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_commit_tree launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
