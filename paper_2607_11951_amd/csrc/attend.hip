// attend.hip -- grid_attend: attention of a chunk of new tokens over a paged cache (gfx950).
#include <cmath>

#include "paged.h"

using namespace grid;

namespace {

struct AttendArgs {
  const uint16_t* q;
  uint16_t* out;
  int64_t qs[2], os[2];
  float* lse;
  int32_t hq, group, max_q, max_kv, window;
  float scale;
};

// One wave a token and query head: 64 keys a step, a lane a key for the scores, a lane some of the entries for the sum.
template <typename T, int D>
__global__ __launch_bounds__(64) void attend_kernel(Paged P, AttendArgs a) {
  const int t = (int)blockIdx.x, h = (int)blockIdx.y, lane = (int)threadIdx.x;
  int b = 0;
  for (int s = 0; s < P.B; s += 64) b += __popcll(__ballot(s + lane < P.B && P.cu_q[s + lane + 1] <= t));
  if (b >= P.B) return;
  const Chunk c = chunk_of(P, b);
  if (t < P.cu_q[b]) return;
  const int g = h / a.group;
  __shared__ float q[D];
  __shared__ float w[64];
  __shared__ int64_t vat[64];
  for (int i = lane; i < D; i += 64) q[i] = (float)((const T*)a.q)[t * a.qs[0] + h * a.qs[1] + i];
  __syncthreads();
  bool bad = !c.ok || c.n > a.max_q || c.kv > a.max_kv;
  const int pos = c.kv - c.n + t - c.first;
  const int low = a.window ? max(0, pos - a.window + 1) : 0;
  float m = -INFINITY, z = 0.f, o[D / 64] = {};
  for (int s0 = low; !bad && s0 <= pos; s0 += 64) {
    const int s = s0 + lane;
    float x = -INFINITY;
    bool missing = false;
    if (s <= pos) {
      uint32_t row;
      const int page = P.page_of(b, (uint32_t)s, row);
      missing = !P.in_cache(page);
      if (!missing) {
        const T* k = (const T*)P.k + page * P.ks[0] + row * P.ks[1] + g * P.ks[2];
        vat[lane] = page * P.vs[0] + row * P.vs[1] + g * P.vs[2];
        x = 0.f;
        for (int i = 0; i < D; ++i) x += q[i] * (float)k[i];
        x *= a.scale;
      }
    }
    bad = __any(missing);
    if (bad) break;
    float top = x;
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float now = fmaxf(m, top);
    const float keep = now == -INFINITY ? 1.f : __expf(m - now);
    const float p = s <= pos && now != -INFINITY ? __expf(x - now) : 0.f;
    float sum = p;
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    z = z * keep + sum;
    m = now;
    w[lane] = (float)(T)p;
    __syncthreads();
    for (int i = 0; i < D / 64; ++i) o[i] *= keep;
    const int n = min(64, pos - s0 + 1);
    for (int j = 0; j < n; ++j)
      for (int i = 0; i < D / 64; ++i) o[i] += w[j] * (float)((const T*)P.v)[vat[j] + lane + 64 * i];
    __syncthreads();
  }
  const float over = z > 0.f ? 1.f / z : z == 0.f ? 0.f : z;
  for (int i = 0; i < D / 64; ++i)
    ((T*)a.out)[t * a.os[0] + h * a.os[1] + lane + 64 * i] = (T)(bad ? NAN : o[i] * over);
  if (a.lse && lane == 0) a.lse[(int64_t)t * a.hq + h] = bad ? NAN : m + logf(z);
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

}  // namespace

extern "C" size_t grid_attend_workspace_bytes(const grid_paged_cache* cache, const grid_chunks* chunks,
                                              const grid_attend_args* args) {
  if (check(cache, chunks, args, false) != GRID_OK) return 0;
  return 16;
}

extern "C" int grid_attend(const grid_paged_cache* cache, const grid_chunks* chunks, const grid_attend_args* args,
                           void* stream) {
  clear_error();
  const int rc = check(cache, chunks, args, true);
  if (rc != GRID_OK) return rc;
  if (chunks->n_tokens == 0) return GRID_OK;
  if (!args->workspace || (uintptr_t)args->workspace % 16 != 0 ||
      args->workspace_bytes < grid_attend_workspace_bytes(cache, chunks, args))
    return fail(GRID_E_ARG, "grid_attend: workspace too small or not aligned");
  AttendArgs a;
  a.q = (const uint16_t*)args->q;
  a.out = (uint16_t*)args->out;
  for (int i = 0; i < 2; ++i) {
    a.qs[i] = args->q_stride[i];
    a.os[i] = args->out_stride[i];
  }
  a.lse = args->lse;
  a.hq = args->n_heads;
  a.group = args->n_heads / cache->n_kv_heads;
  a.max_q = args->max_q;
  a.max_kv = args->max_kv;
  a.window = args->window;
  a.scale = args->scale;
  const Paged P = make_paged(cache, chunks);
  const dim3 blocks((unsigned)P.T, (unsigned)a.hq);
  auto launch = [&](auto type) {
    using T = decltype(type);
    if (P.D == 64)
      hipLaunchKernelGGL((attend_kernel<T, 64>), blocks, dim3(64), 0, (hipStream_t)stream, P, a);
    else if (P.D == 128)
      hipLaunchKernelGGL((attend_kernel<T, 128>), blocks, dim3(64), 0, (hipStream_t)stream, P, a);
    else
      hipLaunchKernelGGL((attend_kernel<T, 256>), blocks, dim3(64), 0, (hipStream_t)stream, P, a);
  };
  if (cache->dtype == GRID_DTYPE_BF16)
    launch(bf16_t());
  else
    launch(f16_t());
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(GRID_E_HIP, std::string("grid_attend launch: ") + hipGetErrorString(e));
  return GRID_OK;
}
