// paged.hip -- host checks of the paged cache, its chunks, and the sizes of both.
#include "paged.h"

namespace grid {

bool rows_fit(const void* p, const int64_t* strides, int n) {
  if ((uintptr_t)p % 16 != 0) return false;
  for (int i = 0; i < n; ++i)
    if (strides[i] < 0 || strides[i] >= (int64_t)1 << 31 || strides[i] % 8 != 0) return false;
  return true;
}

bool layers_fit(int layers, int64_t k_stride, int64_t v_stride) {
  for (int64_t s : {k_stride, v_stride})
    if (s < 0 || s % 8 != 0 || s >= (int64_t)1 << 48 || (layers > 1 && s == 0)) return false;
  return true;
}

int check_cache(const char* call, const grid_paged_cache* c, bool pointers) {
  auto bad = [&](const char* what) { return fail(GRID_E_ARG, std::string(call) + ": " + what); };
  if (!c) return bad("null argument");
  if (c->dtype != GRID_DTYPE_BF16 && c->dtype != GRID_DTYPE_F16) return bad("the cache's dtype is bf16 or f16");
  if (c->n_pages < 1 || c->page_size < 1 || c->page_size > 65536) return bad("pages");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return bad("key heads");
  if (c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 != 0) return bad("head_dim is a multiple of 8 up to 256");
  if (!pointers) return GRID_OK;
  if (!c->k_pages || !c->v_pages) return bad("null pointer");
  if (!rows_fit(c->k_pages, c->k_stride, 3) || !rows_fit(c->v_pages, c->v_stride, 3))
    return bad("pages are 16-byte aligned, their strides multiples of 8");
  for (const int64_t* s : {c->k_stride, c->v_stride})
    if (s[1] >= 1 << 27 || s[2] >= 1 << 27) return bad("strides");
  return GRID_OK;
}

int check_paged(const char* call, const grid_paged_cache* c, const grid_chunks* x, bool pointers) {
  auto bad = [&](const char* what) { return fail(GRID_E_ARG, std::string(call) + ": " + what); };
  if (!x) return bad("null argument");
  const int rc = check_cache(call, c, false);
  if (rc != GRID_OK) return rc;
  if (x->n_seqs < 1 || x->n_seqs > 65535) return bad("1 to 65535 sequences");
  if (x->n_tokens < 0 || x->n_tokens > 1 << 24) return bad("n_tokens");
  if (x->table_cols < 1 || x->table_stride < x->table_cols) return bad("block table");
  // (positions are counted in 32 bits, a few stages past the end)
  if ((int64_t)x->table_cols * c->page_size > INT32_MAX - 4096) return bad("the block table has 2^31 - 4096 positions or more");
  if (!pointers) return GRID_OK;
  if (!x->block_table || !x->kv_len || !x->cu_q) return bad("null pointer");
  return check_cache(call, c, true);
}

Paged make_paged(const grid_paged_cache* c, const grid_chunks* x) {
  Paged p;
  p.k = (uint16_t*)c->k_pages;
  p.v = (uint16_t*)c->v_pages;
  for (int i = 0; i < 3; ++i) {
    p.ks[i] = (uint32_t)c->k_stride[i];
    p.vs[i] = (uint32_t)c->v_stride[i];
  }
  p.table = x->block_table;
  p.table_stride = x->table_stride;
  p.kv_len = x->kv_len;
  p.cu_q = x->cu_q;
  p.page = Divisor((uint32_t)c->page_size);
  p.n_pages = c->n_pages;
  p.cols = x->table_cols;
  p.hkv = c->n_kv_heads;
  p.D = c->head_dim;
  p.B = x->n_seqs;
  p.T = x->n_tokens;
  p.reach = (int64_t)x->table_cols * c->page_size;
  return p;
}

}  // namespace grid
