// append.hip -- grid_kv_append: keys, values and queries of new tokens into a paged cache (gfx950).
//
// A head's vector of one token is 8 entries (16 bytes) a lane, so a power of two of lanes holds one; its mean square is
// a butterfly over those lanes.  Both entries of a rotated pair are needed at once: side by side they are in one lane;
// half a rotation apart the partner's 16 bytes are exchanged between the lanes.
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
  float eps;
  int32_t lanes;  // lanes of a head's vector
};

template <typename T>
struct alignas(16) Eight {
  T x[8];
};

// A sequence's status: whether every one of its chunk's tokens has a place and a rotation.
__device__ int status_of(const Paged& P, const AppendArgs& a, int b) {
  const Chunk c = chunk_of(P, b);
  bool ok = c.ok && (!a.cos || c.kv <= a.n_positions || c.n == 0);
  if (ok && c.n > 0) {
    const uint32_t from = P.page.quot((uint32_t)(c.kv - c.n)), to = P.page.quot((uint32_t)(c.kv - 1));
    for (uint32_t p = from; p <= to; ++p) ok = ok && P.in_cache(P.table[(int64_t)b * P.table_stride + p]);
  }
  return ok ? GRID_ROW_OK : GRID_ROW_BAD_CONFIG;
}

template <typename T>
__device__ void turn(float (&x)[8], const AppendArgs& a, const float* weight, int D, int part, int pos) {
  const int e = part * 8;  // the lane's first entry
  if (weight) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[i] * x[i];
    if (e >= D) s = 0.f;
    for (int o = a.lanes >> 1; o > 0; o >>= 1) s += __shfl_xor(s, o);
    const float r = 1.0f / sqrtf(s / (float)D + a.eps);
    if (e < D)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= r * weight[e + i];
  }
  if (!a.cos) return;
  const float* cs = a.cos + (int64_t)pos * a.half;
  const float* sn = a.sin + (int64_t)pos * a.half;
  if (a.interleaved) {
    if (e < 2 * a.half)
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float c = cs[(e + i) / 2], s = sn[(e + i) / 2], u = x[i], v = x[i + 1];
        x[i] = u * c - v * s;
        x[i + 1] = v * c + u * s;
      }
    return;
  }
  const int hp = a.half / 8;  // the partner's distance in lanes
  const bool low = part < hp, in = part < 2 * hp;
  const int lane = (int)threadIdx.x & 63, from = in ? (low ? lane + hp : lane - hp) : lane;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = __shfl(x[i], from);
    if (in) {
      const int j = (low ? e : e - a.half) + i;
      x[i] = low ? x[i] * cs[j] - y * sn[j] : x[i] * cs[j] + y * sn[j];
    }
  }
}

// One workgroup a token; the workgroups after the last token write the statuses.
template <typename T>
__global__ __launch_bounds__(kThreads) void append_kernel(Paged P, AppendArgs a) {
  const int t = (int)blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63;
  if (t >= P.T) {
    const int b = (t - P.T) * kThreads + tid;
    if (b < P.B) a.status[b] = status_of(P, a, b);
    return;
  }
  // the token's sequence: as many as end at or before it
  int b = 0;
  for (int s = 0; s < P.B; s += 64)
    b += __popcll(__ballot(s + lane < P.B && P.cu_q[s + lane + 1] <= t));
  if (b >= P.B) return;
  const Chunk c = chunk_of(P, b);
  if (!c.ok || t < c.first || t >= c.first + c.n) return;
  const int pos = c.kv - c.n + t - c.first;
  if (a.cos && pos >= a.n_positions) return;
  uint32_t row;
  const int page = P.page_of(b, (uint32_t)pos, row);
  if (!P.in_cache(page)) return;
  const int part = tid & (a.lanes - 1), group = tid / a.lanes, groups = kThreads / a.lanes;
  const bool real = part * 8 < P.D;
  const int vectors = 2 * P.hkv + a.hq;
  // every lane of a wave takes the same number of steps: the exchanges need them all
  for (int u0 = 0; u0 < vectors; u0 += groups) {
    const int u = u0 + group;
    const bool mine = real && u < vectors;
    const int kind = u < P.hkv ? 0 : u < 2 * P.hkv ? 1 : 2;
    const int h = kind == 0 ? u : kind == 1 ? u - P.hkv : u - 2 * P.hkv;
    Eight<T> in = {};
    if (mine) {
      const uint16_t* src = kind == 0 ? a.kin + t * a.ks[0] + h * a.ks[1]
                            : kind == 1 ? a.vin + t * a.vs[0] + h * a.vs[1] : a.qin + t * a.qs[0] + h * a.qs[1];
      in = *(const Eight<T>*)(src + part * 8);
    }
    const float* weight = kind == 2 ? a.q_norm : a.k_norm;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)in.x[i];
    turn<T>(x, a, weight, P.D, part, pos);
    if (!mine) continue;
    uint16_t* dst = kind == 0 ? P.k + page * P.ks[0] + row * P.ks[1] + h * P.ks[2]
                    : kind == 1 ? P.v + page * P.vs[0] + row * P.vs[1] + h * P.vs[2] : a.qout + t * a.os[0] + h * a.os[1];
    Eight<T> out = in;
    if (kind != 1 && (weight || a.cos))
#pragma unroll
      for (int i = 0; i < 8; ++i) out.x[i] = (T)x[i];
    *(Eight<T>*)(dst + part * 8) = out;
  }
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
  a.lanes = 1;
  while (a.lanes * 8 < D) a.lanes *= 2;
  const Paged P = make_paged(cache, chunks);
  const int blocks = P.T + (g.status ? (P.B + kThreads - 1) / kThreads : 0);
  if (blocks == 0) return GRID_OK;
  if (cache->dtype == GRID_DTYPE_BF16)
    hipLaunchKernelGGL(append_kernel<bf16_t>, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, P, a);
  else
    hipLaunchKernelGGL(append_kernel<f16_t>, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, P, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_kv_append launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
