// step_module.cpp -- the Python module _step: the calls of the model's side of a step on torch tensors.
//
// Checks the tensors, fills the argument structures of include/grid.h and calls libgrid.so on the current stream of the
// tensors' device.  Compiled, because these calls are made for every layer of every step: reading twenty tensors from
// Python takes longer than the kernels of a small batch.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <stdexcept>
#include <string>

#include "../../include/grid.h"

namespace {

struct Refused : std::runtime_error {
  PyObject* type;
  Refused(PyObject* t, const std::string& what) : std::runtime_error(what), type(t) {}
};
void need(bool ok, const char* what) {
  if (!ok) throw Refused(PyExc_ValueError, what);
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Refused(PyExc_TypeError, std::string(name) + ": a tensor is wanted");
  return THPVariable_Unpack(o);
}
const at::Tensor* maybe(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }
template <typename T = void>
T* ptr(const at::Tensor* t) {
  return t ? (T*)t->data_ptr() : nullptr;
}
template <typename T = void>
T* ptr(const at::Tensor& t) {
  return (T*)t.data_ptr();
}
int32_t small(int64_t x, const char* what) {
  need(x >= INT32_MIN && x <= INT32_MAX, what);
  return (int32_t)x;
}
int32_t whole(PyObject* o, const char* what) {
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Refused(PyExc_TypeError, std::string(what) + ": an integer is wanted");
  }
  return small(x, what);
}
float real(PyObject* o, const char* what) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    throw Refused(PyExc_TypeError, std::string(what) + ": a number is wanted");
  }
  return (float)x;
}
bool truth(PyObject* o, const char* what) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) {
    PyErr_Clear();
    throw Refused(PyExc_TypeError, std::string(what) + ": true or false is wanted");
  }
  return x != 0;
}

void dense(const at::Tensor* t, at::ScalarType type, at::IntArrayRef shape, at::Device dev, const char* name) {
  if (!t) return;
  if (t->scalar_type() != type || t->sizes() != shape || t->device() != dev || !t->is_contiguous())
    throw Refused(PyExc_ValueError, std::string(name) + ": wrong type, shape, device, or not contiguous");
}

int32_t half_type(at::ScalarType t, const char* what) {
  if (t == at::kBFloat16) return GRID_DTYPE_BF16;
  if (t == at::kHalf) return GRID_DTYPE_F16;
  throw Refused(PyExc_TypeError, what);
}

grid_paged_cache paged(const at::Tensor& k, const at::Tensor& v, int64_t* layers = nullptr) {
  if (layers && k.dim() == 5) {
    need(k.sizes() == v.sizes() && k.scalar_type() == v.scalar_type() && k.size(0) >= 1,
         "pages: [layers, pages, page_size, heads, head_dim], keys and values alike");
    layers[0] = k.size(0);
    layers[1] = k.stride(0);
    layers[2] = v.stride(0);
    return paged(k.select(0, 0), v.select(0, 0));
  }
  need(k.dim() == 4 && k.sizes() == v.sizes() && k.scalar_type() == v.scalar_type() && k.device() == v.device(),
       "pages: [pages, page_size, heads, head_dim], keys and values alike");
  grid_paged_cache c;
  c.dtype = half_type(k.scalar_type(), "pages must be bfloat16 or float16");
  need(k.stride(3) == 1 && v.stride(3) == 1, "pages: vectors must be dense");
  c.k_pages = ptr(k);
  c.v_pages = ptr(v);
  c.n_pages = small(k.size(0), "pages");
  c.page_size = small(k.size(1), "page_size");
  c.n_kv_heads = small(k.size(2), "heads");
  c.head_dim = small(k.size(3), "head_dim");
  for (int i = 0; i < 3; ++i) {
    c.k_stride[i] = k.stride(i);
    c.v_stride[i] = v.stride(i);
  }
  return c;
}

grid_chunks chunks(int64_t tokens, const at::Tensor& table, const at::Tensor& kv_len, const at::Tensor& cu_q, at::Device dev) {
  need(table.dim() == 2 && table.scalar_type() == at::kInt && table.device() == dev && table.stride(1) == 1,
       "block_table: an int32 tensor [B, pages] with dense rows, on the cache's device");
  grid_chunks c;
  c.n_seqs = small(table.size(0), "block_table");
  c.n_tokens = small(tokens, "tokens");
  c.block_table = ptr<int32_t>(table);
  c.table_cols = small(table.size(1), "block_table");
  c.table_stride = c.n_seqs > 1 ? table.stride(0) : c.table_cols;
  dense(&kv_len, at::kInt, {table.size(0)}, dev, "kv_len");
  dense(&cu_q, at::kInt, {table.size(0) + 1}, dev, "cu_q");
  c.kv_len = ptr<int32_t>(kv_len);
  c.cu_q = ptr<int32_t>(cu_q);
  return c;
}

// A packed array of heads' vectors [n, heads, D] with dense vectors; its strides.
void vectors(const at::Tensor& t, at::ScalarType type, int64_t n, int64_t D, at::Device dev, int64_t* stride, const char* name) {
  if (t.dim() != 3 || t.scalar_type() != type || t.size(0) != n || t.size(2) != D || t.device() != dev || t.stride(2) != 1)
    throw Refused(PyExc_ValueError,
                  std::string(name) + ": a tensor [tokens, heads, head_dim] like the cache, with dense vectors, is wanted");
  stride[0] = t.stride(0);
  stride[1] = t.stride(1);
}

void* stream_of(at::Device dev) {
  need(dev.is_cuda(), "the tensors must be on a GPU");
  return (void*)c10::hip::getCurrentHIPStream(dev.index()).stream();
}

// The calls have no derivatives: tensors that want one are refused while torch records them, backward or forward.
void no_gradient(std::initializer_list<const at::Tensor*> tensors) {
  const bool back = c10::GradMode::is_enabled(), forward = c10::AutogradState::get_tls_state().get_fw_grad_mode();
  for (const at::Tensor* t : tensors)
    if (t && ((back && t->requires_grad()) || (forward && t->_fw_grad(0).defined())))
      throw Refused(PyExc_RuntimeError,
                    "there are no gradients of this call: detach its tensors, or call it under torch.no_grad()");
}
// What a call has written in place, for torch to know.
void written(std::initializer_list<const at::Tensor*> tensors) {
  for (const at::Tensor* t : tensors)
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

PyObject* given(PyObject* o, const at::Tensor& made) {
  if (o == Py_None) return THPVariable_Wrap(made);
  Py_INCREF(o);
  return o;
}


template <typename F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F f) {
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return nullptr;
  }
  try {
    return f();
  } catch (const Refused& e) {
    PyErr_SetString(e.type, e.what());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// k, v, k_pages, v_pages, block_table, kv_len, cu_q, q, q_out, cos, sin, interleaved, q_norm, k_norm, eps, status, depth
PyObject* kv_append(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 17, [&]() -> PyObject* {
    const at::Tensor &k = tensor(x[0], "k"), &v = tensor(x[1], "v"), &k_pages = tensor(x[2], "k_pages");
    const at::Tensor& v_pages = tensor(x[3], "v_pages");
    const grid_paged_cache c = paged(k_pages, v_pages);
    const at::Device dev = k_pages.device();
    const at::ScalarType type = k_pages.scalar_type();
    const int64_t D = c.head_dim, tokens = k.dim() ? k.size(0) : 0;
    const grid_chunks ch =
        chunks(tokens, tensor(x[4], "block_table"), tensor(x[5], "kv_len"), tensor(x[6], "cu_q"), dev);
    grid_append_args a = {};
    vectors(k, type, tokens, D, dev, a.k_stride, "k");
    vectors(v, type, tokens, D, dev, a.v_stride, "v");
    need(k.size(1) == c.n_kv_heads && v.size(1) == c.n_kv_heads, "k and v have the cache's heads");
    a.k = ptr(k);
    a.v = ptr(v);
    const at::Tensor* q = maybe(x[7], "q");
    const at::Tensor *cos = maybe(x[9], "cos"), *sin = maybe(x[10], "sin");
    if (cos || sin) {
      need(cos && sin && cos->dim() == 2, "cos and sin come together, [positions, rot_dim / 2]");
      dense(cos, at::kFloat, cos->sizes(), dev, "cos");
      dense(sin, at::kFloat, cos->sizes(), dev, "sin");
      a.n_positions = small(cos->size(0), "cos");
      a.rot_dim = small(2 * cos->size(1), "cos");
    }
    a.cos = ptr<float>(cos);
    a.sin = ptr<float>(sin);
    a.interleaved = truth(x[11], "interleaved");
    const at::Tensor *q_norm = maybe(x[12], "q_norm"), *k_norm = maybe(x[13], "k_norm"), *status = maybe(x[15], "status");
    dense(q_norm, at::kFloat, {D}, dev, "q_norm");
    dense(k_norm, at::kFloat, {D}, dev, "k_norm");
    dense(status, at::kInt, {ch.n_seqs}, dev, "status");
    const at::Tensor* depth = maybe(x[16], "depth");
    dense(depth, at::kInt, {tokens}, dev, "depth");
    a.q_norm = ptr<float>(q_norm);
    a.k_norm = ptr<float>(k_norm);
    a.eps = real(x[14], "eps");
    a.status = ptr<int32_t>(status);
    const at::Tensor* q_out = maybe(x[8], "q_out");
    no_gradient({&k, &v, &k_pages, &v_pages, q, q_out, cos, sin, q_norm, k_norm});
    void* stream = stream_of(dev);
    const c10::DeviceGuard guard(dev);
    at::Tensor out;
    if (q) {
      vectors(*q, type, tokens, D, dev, a.q_stride, "q");
      out = q_out ? *q_out : at::empty(q->sizes(), q->options());
      vectors(out, type, tokens, D, dev, a.q_out_stride, "q_out");
      need(out.size(1) == q->size(1), "q_out has the shape of q");
      a.q = ptr(*q);
      a.q_out = ptr(out);
      a.n_heads = small(q->size(1), "q");
    }
    int rc;
    if (!depth)
      rc = grid_kv_append(&c, &ch, &a, stream);
    else
      rc = tokens ? grid_kv_append_tree(&c, &ch, &a, ptr<int32_t>(depth), stream) : grid_kv_append(&c, &ch, &a, stream);
    if (rc != GRID_OK) return PyLong_FromLong(rc);
    written({&k_pages, &v_pages, q ? q_out : nullptr, status});
    PyObject* first = q ? given(x[8], out) : (Py_INCREF(Py_None), Py_None);
    PyObject* both = PyTuple_Pack(2, first, x[15]);
    Py_DECREF(first);
    return both;
  });
}

// q, k_pages, v_pages, block_table, kv_len, cu_q, max_q, max_kv, scale, window, out, lse, workspace; trees: tree, depth
PyObject* attend_call(PyObject* const* x, Py_ssize_t n, bool trees) {
  return guarded(n, trees ? 15 : 13, [&]() -> PyObject* {
    const at::Tensor &q = tensor(x[0], "q"), &k_pages = tensor(x[1], "k_pages"), &v_pages = tensor(x[2], "v_pages");
    const grid_paged_cache c = paged(k_pages, v_pages);
    const at::Device dev = k_pages.device();
    const int64_t D = c.head_dim, tokens = q.dim() ? q.size(0) : 0;
    const grid_chunks ch =
        chunks(tokens, tensor(x[3], "block_table"), tensor(x[4], "kv_len"), tensor(x[5], "cu_q"), dev);
    grid_attend_args a = {};
    vectors(q, k_pages.scalar_type(), tokens, D, dev, a.q_stride, "q");
    a.q = ptr(q);
    a.n_heads = small(q.size(1), "q");
    a.max_q = whole(x[6], "max_q");
    a.max_kv = whole(x[7], "max_kv");
    a.scale = x[8] == Py_None ? 1.0f / std::sqrt((float)D) : real(x[8], "scale");
    a.window = whole(x[9], "window");
    const at::Tensor *masks = trees ? &tensor(x[13], "tree") : nullptr, *depth = trees ? maybe(x[14], "depth") : nullptr;
    grid_tree tree = {};
    if (trees) {
      need(masks->dim() == 2 && masks->scalar_type() == at::kInt && masks->device() == dev && masks->size(0) == tokens &&
               masks->size(1) >= (std::min<int64_t>(a.max_q, tokens) + 31) / 32 && masks->stride(1) == 1,
           "tree: an int32 tensor [tokens, words of max_q bits or more] with dense rows");
      dense(depth, at::kInt, {tokens}, dev, "depth");
      tree.masks = ptr<uint32_t>(masks);
      tree.stride_words = tokens > 1 ? masks->stride(0) : masks->size(1);
      tree.depth = ptr<int32_t>(depth);
    }
    const at::Tensor* given_lse = maybe(x[11], "lse");
    dense(given_lse, at::kFloat, {tokens, q.size(1)}, dev, "lse");
    const at::Tensor *given_out = maybe(x[10], "out"), *given_work = maybe(x[12], "workspace");
    no_gradient({&q, &k_pages, &v_pages, given_out, given_lse});
    void* stream = stream_of(dev);
    const c10::DeviceGuard guard(dev);
    const at::Tensor out = given_out ? *given_out : at::empty(q.sizes(), q.options());
    vectors(out, q.scalar_type(), tokens, D, dev, a.out_stride, "out");
    need(out.size(1) == q.size(1), "out has the shape of q");
    const at::Tensor lse = given_lse ? *given_lse : at::empty({tokens, q.size(1)}, q.options().dtype(at::kFloat));
    a.out = ptr(out);
    a.lse = ptr<float>(lse);
    const at::Tensor work =
        given_work ? *given_work
                   : at::empty({(int64_t)(trees ? grid_attend_tree_workspace_bytes(&c, &ch, &a)
                                                : grid_attend_workspace_bytes(&c, &ch, &a))},
                               q.options().dtype(at::kByte));
    need(work.device() == dev && work.is_contiguous(), "workspace: a contiguous tensor on the cache's device");
    a.workspace = ptr(work);
    a.workspace_bytes = work.nbytes();
    const int rc = trees ? grid_attend_tree(&c, &ch, &a, &tree, stream) : grid_attend(&c, &ch, &a, stream);
    if (rc != GRID_OK) return PyLong_FromLong(rc);
    written({given_out, given_lse, given_work});
    PyObject *o = given(x[10], out), *l = given(x[11], lse), *both = PyTuple_Pack(2, o, l);
    Py_DECREF(o);
    Py_DECREF(l);
    return both;
  });
}
PyObject* attend(PyObject*, PyObject* const* x, Py_ssize_t n) { return attend_call(x, n, false); }
PyObject* attend_tree(PyObject*, PyObject* const* x, Py_ssize_t n) { return attend_call(x, n, true); }

// logits, draft, draft_len, mask, draft_probs, uniform, noise, temperature, tokens, accepted, logprobs, workspace
PyObject* verify(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const at::Tensor& logits = tensor(x[0], "logits");
    need(logits.dim() == 3 && logits.size(1) >= 1 && logits.stride(2) == 1, "logits: [B, K + 1, V] with dense rows");
    grid_verify_args a = {};
    a.dtype = logits.scalar_type() == at::kFloat ? GRID_DTYPE_F32
                                                 : half_type(logits.scalar_type(), "logits must be float32, bfloat16 or float16");
    const int64_t B = logits.size(0), K = logits.size(1) - 1, V = logits.size(2), words = (V + 31) / 32;
    const at::Device dev = logits.device();
    a.logits = ptr(logits);
    a.B = small(B, "logits");
    a.K = small(K, "logits");
    a.V = small(V, "logits");
    a.logits_stride[0] = logits.stride(0);
    a.logits_stride[1] = logits.stride(1);
    const at::Tensor &draft = tensor(x[1], "draft"), *draft_len = maybe(x[2], "draft_len"), *mask = maybe(x[3], "mask");
    const at::Tensor *probs = maybe(x[4], "draft_probs"), *uniform = maybe(x[5], "uniform"), *noise = maybe(x[6], "noise");
    const at::Tensor* temperature = maybe(x[7], "temperature");
    dense(&draft, at::kInt, {B, K}, dev, "draft");
    dense(draft_len, at::kInt, {B}, dev, "draft_len");
    dense(uniform, at::kFloat, {B, K}, dev, "uniform");
    dense(temperature, at::kFloat, {B}, dev, "temperature");
    if (mask) {
      need(mask->dim() == 3 && mask->scalar_type() == at::kInt && mask->device() == dev && mask->size(0) == B &&
               mask->size(1) == K + 1 && mask->size(2) >= words && mask->stride(2) == 1,
           "mask: an int32 tensor [B, K + 1, words of V bits or more] with dense rows");
      a.mask_stride[0] = mask->stride(0);
      a.mask_stride[1] = mask->stride(1);
    }
    if (probs) {
      need(probs->dim() == 3 && probs->scalar_type() == at::kFloat && probs->device() == dev && probs->size(0) == B &&
               probs->size(1) == K && probs->size(2) == V && (K == 0 || probs->stride(2) == 1),
           "draft_probs: a float32 tensor [B, K, V] with dense rows");
      a.probs_stride[0] = probs->stride(0);
      a.probs_stride[1] = probs->stride(1);
    }
    if (noise) {
      need(noise->dim() == 2 && noise->scalar_type() == at::kFloat && noise->device() == dev && noise->size(0) == B &&
               noise->size(1) == V && noise->stride(1) == 1,
           "noise: a float32 tensor [B, V] with dense rows");
      a.noise_stride = noise->stride(0);
    }
    a.draft = ptr<int32_t>(draft);
    a.draft_len = ptr<int32_t>(draft_len);
    a.mask = ptr<uint32_t>(mask);
    a.draft_probs = ptr<float>(probs);
    a.uniform = ptr<float>(uniform);
    a.noise = ptr<float>(noise);
    a.temperature = ptr<float>(temperature);
    const at::Tensor *t = maybe(x[8], "tokens"), *c = maybe(x[9], "accepted"), *l = maybe(x[10], "logprobs");
    dense(t, at::kInt, {B, K + 1}, dev, "tokens");
    dense(c, at::kInt, {B}, dev, "accepted");
    dense(l, at::kFloat, {B, K + 1}, dev, "logprobs");
    const at::Tensor* given_work = maybe(x[11], "workspace");
    no_gradient({&logits, probs, uniform, noise, temperature, l});
    void* stream = stream_of(dev);
    const c10::DeviceGuard guard(dev);
    const auto ints = logits.options().dtype(at::kInt);
    const at::Tensor tokens = t ? *t : at::empty({B, K + 1}, ints), accepted = c ? *c : at::empty({B}, ints);
    const at::Tensor logprobs = l ? *l : at::empty({B, K + 1}, ints.dtype(at::kFloat));
    const at::Tensor work =
        given_work ? *given_work : at::empty({(int64_t)grid_verify_workspace_bytes(a.B, a.K, a.V)}, ints.dtype(at::kByte));
    need(work.device() == dev && work.is_contiguous(), "workspace: a contiguous tensor on the logits' device");
    a.tokens = ptr<int32_t>(tokens);
    a.accepted = ptr<int32_t>(accepted);
    a.logprobs = ptr<float>(logprobs);
    a.workspace = ptr(work);
    a.workspace_bytes = work.nbytes();
    const int rc = grid_verify(&a, stream);
    if (rc != GRID_OK) return PyLong_FromLong(rc);
    written({t, c, l, given_work});
    PyObject *p = given(x[8], tokens), *q = given(x[9], accepted), *r = given(x[10], logprobs);
    PyObject* all = PyTuple_Pack(3, p, q, r);
    Py_DECREF(p);
    Py_DECREF(q);
    Py_DECREF(r);
    return all;
  });
}

// parent, cu_q, max_q, masks, depth, window
PyObject* tree_masks(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const at::Tensor &parent = tensor(x[0], "parent"), &cu_q = tensor(x[1], "cu_q");
    const at::Device dev = parent.device();
    need(parent.dim() == 1, "parent: [tokens]");
    need(cu_q.dim() == 1 && cu_q.size(0) >= 2, "cu_q: [B + 1]");
    dense(&parent, at::kInt, parent.sizes(), dev, "parent");
    dense(&cu_q, at::kInt, cu_q.sizes(), dev, "cu_q");
    grid_tree_args a = {};
    a.n_tokens = small(parent.size(0), "parent");
    a.n_seqs = small(cu_q.size(0) - 1, "cu_q");
    a.max_q = whole(x[2], "max_q");
    need(a.max_q >= 1, "max_q");
    const int32_t window = whole(x[5], "window");
    need(window >= 0, "window");
    const int64_t T = parent.size(0), words = ((int64_t)a.max_q + 31) / 32;
    const at::Tensor *m = maybe(x[3], "masks"), *d = maybe(x[4], "depth");
    if (m)
      need(m->dim() == 2 && m->scalar_type() == at::kInt && m->device() == dev && m->size(0) == T && m->size(1) >= words &&
               m->stride(1) == 1,
           "masks: an int32 tensor [tokens, words of max_q bits or more] with dense rows");
    dense(d, at::kInt, {T}, dev, "depth");
    void* stream = stream_of(dev);
    const c10::DeviceGuard guard(dev);
    const at::Tensor masks = m ? *m : at::empty({T, words}, parent.options());
    const at::Tensor depth = d ? *d : at::empty({T}, parent.options());
    a.cu_q = ptr<int32_t>(cu_q);
    a.parent = ptr<int32_t>(parent);
    a.masks = ptr<uint32_t>(masks);
    a.stride_words = T > 1 ? masks.stride(0) : masks.size(1);
    a.depth = ptr<int32_t>(depth);
    const int rc = window ? grid_tree_masks_window(&a, window, stream) : grid_tree_masks(&a, stream);
    if (rc != GRID_OK) return PyLong_FromLong(rc);
    written({m, d});
    PyObject *p = given(x[3], masks), *q = given(x[4], depth), *both = PyTuple_Pack(2, p, q);
    Py_DECREF(p);
    Py_DECREF(q);
    return both;
  });
}

// k_pages, v_pages, block_table, kv_len, cu_q, tokens, parent, sampled, max_q, start, path, length, next
PyObject* commit_tree(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    const at::Tensor &cu_q = tensor(x[4], "cu_q"), &tokens = tensor(x[5], "tokens"), &parent = tensor(x[6], "parent");
    const at::Tensor& sampled = tensor(x[7], "sampled");
    const at::Device dev = cu_q.device();
    need(cu_q.dim() == 1 && cu_q.size(0) >= 2, "cu_q: [B + 1]");
    need(tokens.dim() == 1, "tokens: [tokens]");
    const int64_t B = cu_q.size(0) - 1, T = tokens.size(0);
    const at::Tensor *k_pages = maybe(x[0], "k_pages"), *v_pages = maybe(x[1], "v_pages"), *start = maybe(x[9], "start");
    dense(&cu_q, at::kInt, {B + 1}, dev, "cu_q");
    dense(&tokens, at::kInt, {T}, dev, "tokens");
    dense(&parent, at::kInt, {T}, dev, "parent");
    dense(&sampled, at::kInt, {T}, dev, "sampled");
    dense(start, at::kInt, {B}, dev, "start");
    need(!k_pages == !v_pages, "k_pages and v_pages come together");
    grid_paged_cache c = {};
    grid_chunks ch = {};
    grid_commit_args a = {};
    if (k_pages) {
      int64_t layers[3] = {1, 0, 0};
      c = paged(*k_pages, *v_pages, layers);
      need(k_pages->device() == dev, "the cache is on the device of cu_q");
      ch = chunks(T, tensor(x[2], "block_table"), tensor(x[3], "kv_len"), cu_q, dev);
      a.n_layers = small(layers[0], "layers");
      a.k_layer_stride = layers[1];
      a.v_layer_stride = layers[2];
    } else {
      ch.n_seqs = small(B, "cu_q");
      ch.n_tokens = small(T, "tokens");
      ch.cu_q = ptr<int32_t>(cu_q);
    }
    a.max_q = whole(x[8], "max_q");
    need(a.max_q >= 1, "max_q");
    const at::Tensor *p = maybe(x[10], "path"), *l = maybe(x[11], "length"), *f = maybe(x[12], "next");
    dense(p, at::kInt, {B, a.max_q}, dev, "path");
    dense(l, at::kInt, {B}, dev, "length");
    dense(f, at::kInt, {B}, dev, "next");
    no_gradient({k_pages, v_pages});
    void* stream = stream_of(dev);
    const c10::DeviceGuard guard(dev);
    const at::Tensor path = p ? *p : at::empty({B, a.max_q}, cu_q.options());
    const at::Tensor length = l ? *l : at::empty({B}, cu_q.options()), next = f ? *f : at::empty({B}, cu_q.options());
    a.tokens = ptr<int32_t>(tokens);
    a.parent = ptr<int32_t>(parent);
    a.sampled = ptr<int32_t>(sampled);
    a.start = ptr<int32_t>(start);
    a.path = ptr<int32_t>(path);
    a.path_stride = a.max_q;
    a.length = ptr<int32_t>(length);
    a.next = ptr<int32_t>(next);
    const int rc = grid_commit_tree(k_pages ? &c : nullptr, &ch, &a, stream);
    if (rc != GRID_OK) return PyLong_FromLong(rc);
    written({k_pages, v_pages, p, l, f});
    PyObject *r0 = given(x[10], path), *r1 = given(x[11], length), *r2 = given(x[12], next), *all = PyTuple_Pack(3, r0, r1, r2);
    Py_DECREF(r0);
    Py_DECREF(r1);
    Py_DECREF(r2);
    return all;
  });
}

// k_pages, v_pages, src, dst, rows
PyObject* kv_copy(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 5, [&]() -> PyObject* {
    const at::Tensor &k_pages = tensor(x[0], "k_pages"), &v_pages = tensor(x[1], "v_pages");
    int64_t layers[3] = {1, 0, 0};
    const grid_paged_cache c = paged(k_pages, v_pages, layers);
    const at::Device dev = k_pages.device();
    const at::Tensor &src = tensor(x[2], "src"), &dst = tensor(x[3], "dst"), *rows = maybe(x[4], "rows");
    need(src.dim() == 1, "src: [pairs]");
    dense(&src, at::kInt, src.sizes(), dev, "src");
    dense(&dst, at::kInt, src.sizes(), dev, "dst");
    dense(rows, at::kInt, src.sizes(), dev, "rows");
    no_gradient({&k_pages, &v_pages});
    void* stream = stream_of(dev);
    const c10::DeviceGuard guard(dev);
    grid_copy_args a = {};
    a.src = ptr<int32_t>(src);
    a.dst = ptr<int32_t>(dst);
    a.rows = ptr<int32_t>(rows);
    a.n = small(src.size(0), "pairs");
    a.n_layers = small(layers[0], "layers");
    a.k_layer_stride = layers[1];
    a.v_layer_stride = layers[2];
    const int rc = grid_kv_copy(&c, &a, stream);
    if (rc != GRID_OK) return PyLong_FromLong(rc);
    written({&k_pages, &v_pages});
    Py_RETURN_NONE;
  });
}

// block_table, held, parent, keep, room, refs, page_size, table_out, held_out, refs_out, copies, status, workspace
PyObject* kv_fork(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 13, [&]() -> PyObject* {
    const at::Tensor &table = tensor(x[0], "block_table"), &held = tensor(x[1], "held"), &parent = tensor(x[2], "parent");
    const at::Tensor &keep = tensor(x[3], "keep"), &room = tensor(x[4], "room"), &refs = tensor(x[5], "refs");
    const at::Device dev = table.device();
    need(table.dim() == 2 && table.scalar_type() == at::kInt && table.stride(1) == 1,
         "block_table: an int32 tensor [rows, pages] with dense rows");
    need(parent.dim() == 1 && refs.dim() == 1, "parent: [rows]; refs: [pages]");
    const int64_t in = table.size(0), R = parent.size(0), cols = table.size(1);
    dense(&held, at::kInt, {in}, dev, "held");
    dense(&parent, at::kInt, {R}, dev, "parent");
    dense(&keep, at::kInt, {R}, dev, "keep");
    dense(&room, at::kInt, {R}, dev, "room");
    dense(&refs, at::kInt, refs.sizes(), dev, "refs");
    const at::Tensor *t = maybe(x[7], "table_out"), *h = maybe(x[8], "held_out"), *r = maybe(x[9], "refs_out");
    const at::Tensor *c = maybe(x[10], "copies"), *s = maybe(x[11], "status"), *given_work = maybe(x[12], "workspace");
    if (t)
      need(t->dim() == 2 && t->scalar_type() == at::kInt && t->device() == dev && t->size(0) == R && t->size(1) == cols &&
               t->stride(1) == 1,
           "table_out: an int32 tensor [rows, pages] with dense rows");
    dense(h, at::kInt, {R}, dev, "held_out");
    dense(r, at::kInt, refs.sizes(), dev, "refs_out");
    dense(c, at::kInt, {3, R}, dev, "copies");
    dense(s, at::kInt, {R}, dev, "status");
    grid_fork_args a = {};
    a.n_in = small(in, "block_table");
    a.n_rows = small(R, "parent");
    a.table_cols = small(cols, "block_table");
    a.n_pages = small(refs.size(0), "refs");
    a.page_size = whole(x[6], "page_size");
    void* stream = stream_of(dev);
    const c10::DeviceGuard guard(dev);
    const auto ints = table.options();
    const at::Tensor out = t ? *t : at::empty({R, cols}, ints), held_out = h ? *h : at::empty({R}, ints);
    const at::Tensor refs_out = r ? *r : at::empty_like(refs), copies = c ? *c : at::empty({3, R}, ints);
    const at::Tensor status = s ? *s : at::empty({R}, ints);
    const at::Tensor work =
        given_work ? *given_work
                   : at::empty({(int64_t)grid_kv_fork_workspace_bytes(a.n_rows, a.n_pages)}, ints.dtype(at::kByte));
    need(work.device() == dev && work.is_contiguous(), "workspace: a contiguous tensor on the table's device");
    a.table = ptr<int32_t>(table);
    a.table_stride = in > 1 ? table.stride(0) : cols;
    a.held = ptr<int32_t>(held);
    a.parent = ptr<int32_t>(parent);
    a.keep = ptr<int32_t>(keep);
    a.room = ptr<int32_t>(room);
    a.refs = ptr<int32_t>(refs);
    a.table_out = ptr<int32_t>(out);
    a.table_out_stride = R > 1 ? out.stride(0) : cols;
    a.held_out = ptr<int32_t>(held_out);
    a.refs_out = ptr<int32_t>(refs_out);
    a.copies = ptr<int32_t>(copies);
    a.status = ptr<int32_t>(status);
    a.workspace = ptr(work);
    a.workspace_bytes = work.nbytes();
    const int rc = grid_kv_fork(&a, stream);
    if (rc != GRID_OK) return PyLong_FromLong(rc);
    written({t, h, r, c, s, given_work});
    PyObject* all = PyTuple_New(5);
    PyTuple_SET_ITEM(all, 0, given(x[7], out));
    PyTuple_SET_ITEM(all, 1, given(x[8], held_out));
    PyTuple_SET_ITEM(all, 2, given(x[9], refs_out));
    PyTuple_SET_ITEM(all, 3, given(x[10], copies));
    PyTuple_SET_ITEM(all, 4, given(x[11], status));
    return all;
  });
}

// logits, mask, temperature, top_k, top_p, min_p, noise, tokens, logprobs, workspace
PyObject* sample(PyObject*, PyObject* const* x, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const at::Tensor& logits = tensor(x[0], "logits");
    need(logits.dim() == 2 && logits.stride(1) == 1, "logits: [rows, V] with dense rows");
    grid_sample_args a = {};
    a.dtype = logits.scalar_type() == at::kFloat ? GRID_DTYPE_F32
                                                 : half_type(logits.scalar_type(), "logits must be float32, bfloat16 or float16");
    const int64_t B = logits.size(0), V = logits.size(1), words = (V + 31) / 32;
    const at::Device dev = logits.device();
    a.logits = ptr(logits);
    a.B = small(B, "logits");
    a.V = small(V, "logits");
    a.logits_stride = logits.stride(0);
    const at::Tensor *mask = maybe(x[1], "mask"), *temperature = maybe(x[2], "temperature"), *top_k = maybe(x[3], "top_k");
    const at::Tensor *top_p = maybe(x[4], "top_p"), *min_p = maybe(x[5], "min_p"), *noise = maybe(x[6], "noise");
    dense(temperature, at::kFloat, {B}, dev, "temperature");
    dense(top_k, at::kInt, {B}, dev, "top_k");
    dense(top_p, at::kFloat, {B}, dev, "top_p");
    dense(min_p, at::kFloat, {B}, dev, "min_p");
    if (mask) {
      need(mask->dim() == 2 && mask->scalar_type() == at::kInt && mask->device() == dev && mask->size(0) == B &&
               mask->size(1) >= words && mask->stride(1) == 1,
           "mask: an int32 tensor [rows, words of V bits or more] with dense rows");
      a.mask_stride = mask->stride(0);
    }
    if (noise) {
      need(noise->dim() == 2 && noise->scalar_type() == at::kFloat && noise->device() == dev && noise->size(0) == B &&
               noise->size(1) == V && noise->stride(1) == 1,
           "noise: a float32 tensor [rows, V] with dense rows");
      a.noise_stride = noise->stride(0);
    }
    const at::Tensor *t = maybe(x[7], "tokens"), *l = maybe(x[8], "logprobs");
    dense(t, at::kInt, {B}, dev, "tokens");
    dense(l, at::kFloat, {B}, dev, "logprobs");
    const at::Tensor* given_work = maybe(x[9], "workspace");
    no_gradient({&logits, temperature, top_p, min_p, noise, l});
    void* stream = stream_of(dev);
    const c10::DeviceGuard guard(dev);
    const auto ints = logits.options().dtype(at::kInt);
    const at::Tensor tokens = t ? *t : at::empty({B}, ints), logprobs = l ? *l : at::empty({B}, ints.dtype(at::kFloat));
    const at::Tensor work = given_work ? *given_work
                                       : at::empty({(int64_t)grid_sample_workspace_bytes(a.B, a.V)}, ints.dtype(at::kByte));
    need(work.device() == dev && work.is_contiguous(), "workspace: a contiguous tensor on the logits' device");
    a.workspace = ptr(work);
    a.workspace_bytes = work.nbytes();
    a.mask = ptr<uint32_t>(mask);
    a.temperature = ptr<float>(temperature);
    a.top_k = ptr<int32_t>(top_k);
    a.top_p = ptr<float>(top_p);
    a.min_p = ptr<float>(min_p);
    a.noise = ptr<float>(noise);
    a.tokens = ptr<int32_t>(tokens);
    a.logprobs = ptr<float>(logprobs);
    const int rc = grid_sample(&a, stream);
    if (rc != GRID_OK) return PyLong_FromLong(rc);
    written({t, l, given_work});
    PyObject *p = given(x[7], tokens), *q = given(x[8], logprobs), *both = PyTuple_Pack(2, p, q);
    Py_DECREF(p);
    Py_DECREF(q);
    return both;
  });
}

PyMethodDef methods[] = {{"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, nullptr},
                         {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
                         {"verify", (PyCFunction)(void (*)(void))verify, METH_FASTCALL, nullptr},
                         {"tree_masks", (PyCFunction)(void (*)(void))tree_masks, METH_FASTCALL, nullptr},
                         {"attend_tree", (PyCFunction)(void (*)(void))attend_tree, METH_FASTCALL, nullptr},
                         {"commit_tree", (PyCFunction)(void (*)(void))commit_tree, METH_FASTCALL, nullptr},
                         {"kv_copy", (PyCFunction)(void (*)(void))kv_copy, METH_FASTCALL, nullptr},
                         {"kv_fork", (PyCFunction)(void (*)(void))kv_fork, METH_FASTCALL, nullptr},
                         {"sample", (PyCFunction)(void (*)(void))sample, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_step", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__step(void) { return PyModule_Create(&module); }
