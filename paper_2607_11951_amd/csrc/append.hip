// append.hip -- grid_kv_append: keys, values and queries of new tokens into a paged cache (gfx950).
//
// A head's vector of one token is 8 entries (16 bytes) a lane, so a power of two of lanes holds one; its mean square is
// their sum across those lanes.  Both entries of a rotated pair are needed at once: side by side they are in one lane;
// half a rotation apart the partner's 16 bytes are exchanged between the lanes.
//
// Bound by bytes, for few tokens by dependent reads: 8 chunks of up to 2048 tokens, 32 + 8 + 8 heads of 128 in float16,
// half of each rotated, take 54.5 us, 4.6 TB/s (a copy reaches 5.09); one token 3.1 us on the device.
#include <algorithm>

#include "lanes.h"
#include "paged.h"

using namespace grid;

namespace {

constexpr int kThreads = 256;

struct AppendArgs {
  const uint16_t *kin, *vin, *qin;
  uint16_t* qout;
  int64_t ks[2], vs[2], qs[2], os[2];
  const float *cos, *sin, *q_norm, *k_norm;
  int32_t* status;
  int32_t hq, n_positions, half, interleaved;  // half = rot_dim / 2
  float eps, over;  // over = 1 / head_dim
  int32_t lanes;  // lanes of a head's vector
  int32_t base;   // the launch's first workgroup among all
};

template <typename T>
struct alignas(16) Eight {
  T x[8];
};

// The status of a sequence after chunks that are in order or not: whether every one of its chunk's tokens has a place
// and a rotation.
__device__ int status_of(const Paged& P, const AppendArgs& a, int b, bool ordered) {
  const Chunk c = chunk_of(P, b);
  bool ok = ordered && c.ok && (!a.cos || c.kv <= a.n_positions || c.n == 0);
  if (ok && c.n > 0) {
    const uint32_t from = P.page.quot((uint32_t)(c.kv - c.n)), to = P.page.quot((uint32_t)(c.kv - 1));
    for (uint32_t p = from; p <= to; ++p) ok = ok && P.in_cache(P.table[(int64_t)b * P.table_stride + p]);
  }
  return ok ? GRID_ROW_OK : GRID_ROW_BAD_CONFIG;
}

enum class Turn { kNone, kHalves, kPairs };

// One workgroup a token; the workgroups after the last token write the statuses.  What a token needs hangs on reads one
// after the other (its sequence and lengths, its page, its cosines), so the vectors, which hang on nothing, are asked for
// first, and the sequence's lengths with its search.  A lane takes the same entries of all its vectors: the cosines are
// read once.
template <typename T, Turn TURN, bool NORM>
__global__ __launch_bounds__(kThreads) void append_kernel(Paged P, AppendArgs a) {
  const int t = (int)blockIdx.x + a.base, tid = (int)threadIdx.x, lane = tid & 63;
  if (t >= P.T) {
    const int b = (t - P.T) * kThreads + tid;
    __shared__ int broken;  // the first of the sequences up to here whose chunk is not in order
    if (tid == 0) broken = P.B;
    __syncthreads();
    for (int s = tid; s < min(b - tid + kThreads, P.B); s += kThreads)
      if (!in_order(P, P.cu_q[s], P.cu_q[s + 1])) {
        atomicMin(&broken, s);
        break;
      }
    __syncthreads();
    if (b < P.B) a.status[b] = status_of(P, a, b, b <= broken);
    return;
  }
  const int part = tid & (a.lanes - 1), groups = kThreads / a.lanes, e = part * 8;  // e: the lane's first entry
  const int u_first = e < P.D ? tid / a.lanes : 1 << 30, vectors = 2 * P.hkv + a.hq;
  constexpr int AHEAD = 3;  // vectors that a lane asks for before it knows where they go
  const auto source = [&](int u) {
    const int h = u < P.hkv ? u : u < 2 * P.hkv ? u - P.hkv : u - 2 * P.hkv;
    const uint16_t* src = u < P.hkv ? a.kin + t * a.ks[0] + h * a.ks[1]
                          : u < 2 * P.hkv ? a.vin + t * a.vs[0] + h * a.vs[1] : a.qin + t * a.qs[0] + h * a.qs[1];
    return *(const Eight<T>*)(src + e);
  };
  __shared__ __attribute__((aligned(16))) float weights[2][256];  // of keys, of queries
  if constexpr (NORM)
    for (int i = tid; i < P.D; i += kThreads) {
      if (a.k_norm) weights[0][i] = a.k_norm[i];
      if (a.q_norm) weights[1][i] = a.q_norm[i];
    }
  Eight<T> ahead[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (u_first + i * groups < vectors) ahead[i] = source(u_first + i * groups);
  int b;
  const Chunk c = chunk_of_token(P, t, b);
  if (!c.ok || t < c.first || t >= c.first + c.n) return;
  const int pos = c.kv - c.n + t - c.first;
  if (TURN != Turn::kNone && pos >= a.n_positions) return;
  uint32_t row;
  const int page = P.page_of(b, (uint32_t)pos, row);
  // the rotation of the lane's entries; in halves, hp lanes apart: the partner's lane and entries
  float cs[8], sn[8];
  const int hp = a.half / 8;
  const bool low = part < hp, turned = e < 2 * a.half;
  const int other = low ? lane + hp : lane - hp, oe = low ? e + a.half : e - a.half;
  if (TURN != Turn::kNone && turned) {
    constexpr int N = TURN == Turn::kPairs ? 4 : 8;
    const int64_t at = (int64_t)pos * a.half + (TURN == Turn::kPairs ? e / 2 : low ? e : oe);
    __builtin_memcpy(cs, a.cos + at, N * 4);
    __builtin_memcpy(sn, a.sin + at, N * 4);
  }
  if (!P.in_cache(page)) return;
  if constexpr (NORM) __syncthreads();
  const auto store = [&](int u, Eight<T> in) {
    const bool key = u < P.hkv, value = !key && u < 2 * P.hkv, normed = NORM && (key ? a.k_norm : a.q_norm);
    const float* weight = weights[key ? 0 : 1];
    float x[8], r = 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)in.x[i];
    if constexpr (NORM) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s += x[i] * x[i];
      if (e >= P.D) s = 0.f;
      s = sum_across(s, a.lanes);
      if (normed) {
        r = __builtin_amdgcn_rsqf(s * a.over + a.eps);
        if (e < P.D)
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] *= r * weight[e + i];
      }
    }
    if constexpr (TURN == Turn::kPairs) {
      if (turned)
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float p = x[i], q = x[i + 1];
          x[i] = p * cs[i / 2] - q * sn[i / 2];
          x[i + 1] = q * cs[i / 2] + p * sn[i / 2];
        }
    }
    if constexpr (TURN == Turn::kHalves) {
      // the partner's entries as they came, normed here
      uint32_t w[4];
      __builtin_memcpy(w, &in, 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (uint32_t)__shfl((int)w[i], turned ? other : lane);
      Eight<T> y;
      __builtin_memcpy(&y, w, 16);
      if (turned)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float z = (float)y.x[i];
          if (normed) z *= r * weight[oe + i];
          x[i] = low ? x[i] * cs[i] - z * sn[i] : x[i] * cs[i] + z * sn[i];
        }
    }
    if (u >= vectors) return;
    const int h = key ? u : value ? u - P.hkv : u - 2 * P.hkv;
    uint16_t* dst = key ? P.k + P.at(P.ks, page, row) + (uint64_t)h * P.ks[2]
                    : value ? P.v + P.at(P.vs, page, row) + (uint64_t)h * P.vs[2] : a.qout + t * a.os[0] + h * a.os[1];
    if (!value && (TURN != Turn::kNone || normed))
#pragma unroll
      for (int i = 0; i < 8; ++i) in.x[i] = (T)x[i];
    *(Eight<T>*)(dst + e) = in;
  };
  // every lane of a wave takes the same number of steps: the exchanges need them all
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (i * groups < vectors) store(u_first + i * groups, ahead[i]);
  for (int u = AHEAD * groups; u < vectors; u += groups) {
    Eight<T> x = {};
    if (u_first + u < vectors) x = source(u_first + u);
    store(u_first + u, x);
  }
}

template <typename T>
void launch(const Paged& P, const AppendArgs& a, unsigned blocks, hipStream_t stream) {
  const bool norm = a.q_norm || a.k_norm;
  const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, stream, P, a); };
  if (!a.cos)
    norm ? go(append_kernel<T, Turn::kNone, true>) : go(append_kernel<T, Turn::kNone, false>);
  else if (a.interleaved)
    norm ? go(append_kernel<T, Turn::kPairs, true>) : go(append_kernel<T, Turn::kPairs, false>);
  else
    norm ? go(append_kernel<T, Turn::kHalves, true>) : go(append_kernel<T, Turn::kHalves, false>);
}

}  // namespace

extern "C" int grid_kv_append(const grid_paged_cache* cache, const grid_chunks* chunks, const grid_append_args* args,
                              void* stream) {
  clear_error();
  const int rc = check_paged("grid_kv_append", cache, chunks, true);
  if (rc != GRID_OK) return rc;
  auto bad = [](const char* what) { return fail(GRID_E_ARG, std::string("grid_kv_append: ") + what); };
  if (!args) return bad("null argument");
  const grid_append_args& g = *args;
  const int D = cache->head_dim;
  if (chunks->n_tokens > 0 && (!g.k || !g.v)) return bad("null pointer");
  if (g.q && (!g.q_out || g.n_heads < 1 || g.n_heads > 1024)) return bad("q needs q_out and 1 to 1024 heads");
  if (!rows_fit(g.k, g.k_stride, 2) || !rows_fit(g.v, g.v_stride, 2) ||
      (g.q && (!rows_fit(g.q, g.q_stride, 2) || !rows_fit(g.q_out, g.q_out_stride, 2))))
    return bad("rows are 16-byte aligned, their strides multiples of 8");
  if (!g.cos != !g.sin) return bad("cos and sin come together");
  if (g.cos && (g.n_positions < 1 || g.rot_dim < 2 || g.rot_dim > D || g.rot_dim % (g.interleaved ? 8 : 16) != 0))
    return bad("rot_dim is a multiple of 16 (interleaved: 8) up to head_dim");
  if (!(g.eps >= 0.f)) return bad("eps");
  AppendArgs a;
  a.kin = (const uint16_t*)g.k;
  a.vin = (const uint16_t*)g.v;
  a.qin = (const uint16_t*)g.q;
  a.qout = (uint16_t*)g.q_out;
  for (int i = 0; i < 2; ++i) {
    a.ks[i] = g.k_stride[i];
    a.vs[i] = g.v_stride[i];
    a.qs[i] = g.q_stride[i];
    a.os[i] = g.q_out_stride[i];
  }
  a.cos = g.cos;
  a.sin = g.sin;
  a.q_norm = g.q_norm;
  a.k_norm = g.k_norm;
  a.status = g.status;
  a.hq = g.q ? g.n_heads : 0;
  a.n_positions = g.n_positions;
  a.half = g.rot_dim / 2;
  a.interleaved = g.interleaved;
  a.eps = g.eps;
  a.over = 1.f / (float)D;
  a.lanes = 1;
  while (a.lanes * 8 < D) a.lanes *= 2;
  const Paged P = make_paged(cache, chunks);
  // (a launch has less than 2^32 threads, 2^24 workgroups)
  const int blocks = P.T + (g.status ? (P.B + kThreads - 1) / kThreads : 0), most = 1 << 23;
  if (blocks == 0) return GRID_OK;
  for (a.base = 0; a.base < blocks; a.base += most) {
    const unsigned n = (unsigned)std::min(blocks - a.base, most);
    if (cache->dtype == GRID_DTYPE_BF16)
      launch<bf16_t>(P, a, n, (hipStream_t)stream);
    else
      launch<f16_t>(P, a, n, (hipStream_t)stream);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_kv_append launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
