// Marshalling of the calls of block-sparse attention and of the many-tensor optimiser (part of ha_binding.cpp, by the same rule: what is not plain and
// right gives None, and the Python code takes the call).  These calls allocate what the Python code would: outputs and workspaces that were not given.
// A refusal of the library gives None too, for the Python code's message: it has enqueued nothing.  A device error may follow launches that are on their way,
// so that the call must not be made twice, and is raised here.
//
// Host time per call in Python / here, us: key_means 13.1 / 5.6, select_blocks 17.0 / 7.0, sparse_forward 22.9 / 6.7, sparse_grad (eight launches) 56 / 41,
// grad_norm (two launches) 15.9 / 12.6.
#pragma once

namespace {

typedef ha_status (*means_fn)(const ha_sparse_problem *, const ha_view *, int32_t, float *, void *);
typedef size_t (*sparse_bytes_fn)(const ha_sparse_problem *);
typedef ha_status (*select_fn)(const ha_sparse_problem *, const ha_view *, const float *, int32_t *, void *, size_t, void *);
typedef ha_status (*sparse_forward_fn)(const ha_sparse_problem *, const ha_view *, const ha_view *, const ha_view *, const int32_t *, const ha_view *, float *,
                                       void *, size_t, void *);
typedef ha_status (*sparse_grad_fn)(const ha_sparse_problem *, const ha_view *, const ha_view *, const ha_view *, const int32_t *, const ha_view *, const float *,
                                    const ha_view *, const ha_view *, const ha_view *, const ha_view *, void *, size_t, void *);
typedef ha_status (*norm_fn)(int32_t, const ha_tensor *, float, float *, void *, size_t, void *);
typedef ha_status (*clip_fn)(int32_t, const ha_tensor *, const ha_tensor *, const float *, void *);
typedef ha_status (*many_fn)(const ha_optimizer *, int32_t, const ha_param *, const float *, void *);

struct Calls {
  means_fn means;
  sparse_bytes_fn select_bytes;
  select_fn select;
  sparse_bytes_fn forward_bytes;
  sparse_forward_fn forward;
  sparse_bytes_fn grad_bytes;
  sparse_grad_fn grad;
  norm_fn norm;
  clip_fn clip;
  many_fn many;
};
Calls g_calls = {};
PyObject *g_get_device = nullptr, *g_native = nullptr, *g_tensors = nullptr, *g_error = nullptr;      // the current device's index; "native", "tensors"; HybridAttnError(status, where)

// What a call gives whose status is not HA_OK.
PyObject *failed(ha_status st, const char *where) {
  if (st != HA_ERR_DEVICE) Py_RETURN_NONE;
  if (!g_error) return PyErr_Format(PyExc_RuntimeError, "%s: device error", where);
  const Ref e(PyObject_CallFunction(g_error, "is", static_cast<int>(st), where));
  if (e.p) PyErr_SetObject(g_error, e.p);
  return nullptr;
}

// The tensor's device is the current one, and the call goes to its current stream.
bool here(PyObject *stream, const at::Tensor &t, void **out) {
  if (stream != Py_None || !t.is_cuda()) return false;
  const Ref d(PyObject_CallNoArgs(g_get_device));
  if (!d.p || PyLong_AsLong(d.p) != t.get_device()) {
    PyErr_Clear();
    return false;
  }
  return stream_of(stream, t, out);
}

bool view_of(const at::Tensor *t, const at::Tensor &like, ha_view *v) {
  if (!t || t->dim() != 4 || t->scalar_type() != like.scalar_type() || t->device() != like.device() || (t->stride(3) != 1 && t->size(3) > 1)) return false;
  *v = ha_view{t->data_ptr(), t->stride(0), t->stride(1), t->stride(2)};
  return true;
}

bool same_sizes(const at::Tensor &a, const at::Tensor &b) { return a.sizes() == b.sizes(); }

bool per_entry(PyObject *o, int64_t B, const at::Tensor &like, const int32_t **out) {
  *out = nullptr;
  if (o == Py_None) return true;
  const at::Tensor *t = tensor(o);
  if (!t || t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != B || !t->is_contiguous() || t->device() != like.device()) return false;
  *out = static_cast<const int32_t *>(t->data_ptr());
  return true;
}

bool plain(const at::Tensor *t, at::ScalarType type, at::IntArrayRef sizes, const at::Tensor &like) {
  return t && t->scalar_type() == type && t->sizes() == sizes && t->is_contiguous() && t->device() == like.device();
}

at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor &like) { return at::empty(sizes, at::TensorOptions().dtype(type).device(like.device())); }

// A new tensor in the order of t's dimensions in memory, without its gaps and broadcast dimensions.
at::Tensor dense_like(const at::Tensor &t) {
  int order[3] = {0, 1, 2};
  for (int i = 1; i < 3; ++i)
    for (int j = i; j > 0 && t.stride(order[j - 1]) < t.stride(order[j]); --j) std::swap(order[j - 1], order[j]);
  int64_t strides[4] = {0, 0, 0, 1}, at = std::max<int64_t>(t.size(3), 1);
  for (int i = 2; i >= 0; --i) {
    strides[order[i]] = at;
    at *= std::max<int64_t>(t.size(order[i]), 1);
  }
  return at::empty_strided(t.sizes(), at::IntArrayRef(strides, 4), t.options());
}

// Workspace of `need` bytes: the one given, or a new one that `keep` holds.
bool workspace_of(PyObject *o, size_t need, const at::Tensor &like, at::Tensor *keep, void **ptr, size_t *bytes) {
  if (o == Py_None) {
    *bytes = need;
    *ptr = nullptr;
    if (need == 0) return true;
    *keep = fresh({static_cast<int64_t>(need)}, at::kByte, like);
    *ptr = keep->data_ptr();
    return true;
  }
  const at::Tensor *t = tensor(o);
  if (!t || t->device() != like.device() || !t->is_contiguous()) return false;
  *ptr = t->data_ptr();
  *bytes = static_cast<size_t>(t->numel()) * t->element_size();
  return true;
}

// Sizes of a problem with q [B, H, N_q, d] and keys [B, H_kv, N_k, d]; the rest is the caller's.
bool sizes_of(ha_sparse_problem *p, const at::Tensor &like, int64_t H, int64_t Nq, int64_t Hkv, int64_t Nk) {
  const int64_t most = std::numeric_limits<int32_t>::max();
  if (like.dim() != 4 || H > most || Nq > most || Hkv > most || Nk > most || Nk < 0 || like.size(0) > most || like.size(3) > most) return false;
  if (like.scalar_type() != at::kBFloat16 && like.scalar_type() != at::kFloat) return false;
  *p = ha_sparse_problem{};
  p->B = static_cast<int32_t>(like.size(0));
  p->H = static_cast<int32_t>(H);
  p->H_kv = static_cast<int32_t>(Hkv);
  p->N_q = static_cast<int32_t>(Nq);
  p->N_k = static_cast<int32_t>(Nk);
  p->d_head = static_cast<int32_t>(like.size(3));
  p->dtype = like.scalar_type() == at::kBFloat16 ? HA_BF16 : HA_F32;
  p->q_block = 128;
  p->k_block = 64;
  p->n_select = 1;
  p->near_tokens = -1;
  p->softmax_scale = static_cast<float>(std::pow(static_cast<double>(std::max<int64_t>(like.size(3), 1)), -0.5));
  return true;
}
bool block_sizes(PyObject *qb, PyObject *kb, ha_sparse_problem *p) {
  return (!qb || small_int(qb, &p->q_block)) && small_int(kb, &p->k_block) && (p->q_block == 64 || p->q_block == 128) && (p->k_block == 64 || p->k_block == 128);
}
bool flag(PyObject *o, int32_t *out) {
  if (!PyBool_Check(o)) return false;
  *out = o == Py_True;
  return true;
}
int64_t blocks_of(int64_t n, int32_t block) { return (n + block - 1) / block; }

#define HA_CALL(ST, EXPR)      \
  Py_BEGIN_ALLOW_THREADS       \
  ST = EXPR;                   \
  Py_END_ALLOW_THREADS

// key_means(k, k_block, key_len, only_last, out, stream) -> means
PyObject *key_means(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 6 || !g_calls.means) Py_RETURN_NONE;
  try {
    const at::Tensor *k = tensor(args[0]), *out = args[4] == Py_None ? nullptr : tensor(args[4]);
    ha_sparse_problem p;
    ha_view kv;
    int32_t last;
    void *stream;
    if (!k || !view_of(k, *k, &kv) || !sizes_of(&p, *k, k->size(1), 0, k->size(1), k->size(2)) || !block_sizes(nullptr, args[1], &p) ||
        !per_entry(args[2], k->size(0), *k, &p.key_len) || !small_int(args[3], &last) || (last != 0 && !out) || !here(args[5], *k, &stream))
      Py_RETURN_NONE;
    const int64_t sizes[] = {k->size(0), k->size(1), blocks_of(k->size(2), p.k_block), k->size(3)};
    if (args[4] != Py_None && !plain(out, at::kFloat, sizes, *k)) Py_RETURN_NONE;
    const at::Tensor means = out ? *out : fresh(sizes, at::kFloat, *k);
    ha_status st;
    HA_CALL(st, g_calls.means(&p, &kv, last, static_cast<float *>(means.data_ptr()), stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_key_means");
    return THPVariable_Wrap(means);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// select_blocks(q, means, n_keys, n_select, q_block, k_block, causal, q_start, key_len, keep_first, near, out, workspace, stream) -> blocks
PyObject *select_blocks(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 14 || !g_calls.select) Py_RETURN_NONE;
  try {
    const at::Tensor *q = tensor(args[0]), *means = tensor(args[1]), *out = args[11] == Py_None ? nullptr : tensor(args[11]);
    ha_sparse_problem p;
    ha_view qv;
    int32_t n_keys;
    void *stream;
    if (!q || !means || means->dim() != 4 || !view_of(q, *q, &qv) || !small_int(args[2], &n_keys) || !sizes_of(&p, *q, q->size(1), q->size(2), means->size(1), n_keys) ||
        !small_int(args[3], &p.n_select) || p.n_select < 1 || !block_sizes(args[4], args[5], &p) || !flag(args[6], &p.causal) || !per_entry(args[7], q->size(0), *q, &p.q_start) ||
        !per_entry(args[8], q->size(0), *q, &p.key_len) || !small_int(args[9], &p.keep_first) || !small_int(args[10], &p.near_tokens) || !here(args[13], *q, &stream))
      Py_RETURN_NONE;
    const int64_t means_sizes[] = {q->size(0), means->size(1), blocks_of(n_keys, p.k_block), q->size(3)};
    const int64_t sizes[] = {q->size(0), means->size(1), blocks_of(q->size(2), p.q_block), p.n_select};
    if (!plain(means, at::kFloat, means_sizes, *q) || (args[11] != Py_None && !plain(out, at::kInt, sizes, *q))) Py_RETURN_NONE;
    at::Tensor keep;
    void *ws;
    size_t bytes;
    if (!workspace_of(args[12], g_calls.select_bytes(&p), *q, &keep, &ws, &bytes)) Py_RETURN_NONE;
    const at::Tensor blocks = out ? *out : fresh(sizes, at::kInt, *q);
    ha_status st;
    HA_CALL(st, g_calls.select(&p, &qv, static_cast<const float *>(means->data_ptr()), static_cast<int32_t *>(blocks.data_ptr()), ws, bytes, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_select_blocks");
    return THPVariable_Wrap(blocks);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// q, k, v, blocks, and args[at ..] = q_block, k_block, causal, q_start, key_len, softmax_scale
bool attention_problem(PyObject *const *args, int at, ha_sparse_problem *p, ha_view *qv, ha_view *kv, ha_view *vv, const int32_t **lists) {
  const at::Tensor *q = tensor(args[0]), *k = tensor(args[1]), *v = tensor(args[2]), *blocks = tensor(args[3]);
  if (!q || !k || !v || !blocks || blocks->dim() != 4 || !view_of(q, *q, qv) || !view_of(k, *q, kv) || !view_of(v, *q, vv) || !same_sizes(*k, *v) || k->size(0) != q->size(0) ||
      k->size(3) != q->size(3) || blocks->size(3) > (1 << 20) || !sizes_of(p, *q, q->size(1), q->size(2), k->size(1), k->size(2)) || !block_sizes(args[at], args[at + 1], p) ||
      !flag(args[at + 2], &p->causal) || !per_entry(args[at + 3], q->size(0), *q, &p->q_start) || !per_entry(args[at + 4], q->size(0), *q, &p->key_len) ||
      (args[at + 5] != Py_None && !number(args[at + 5], &p->softmax_scale)))
    return false;
  p->n_select = static_cast<int32_t>(blocks->size(3));
  const int64_t sizes[] = {q->size(0), k->size(1), blocks_of(q->size(2), p->q_block), blocks->size(3)};
  if (!plain(blocks, at::kInt, sizes, *q)) return false;
  *lists = static_cast<const int32_t *>(blocks->data_ptr());
  return true;
}

// sparse_forward(q, k, v, blocks, q_block, k_block, causal, q_start, key_len, softmax_scale, with_lse, out, lse, workspace, stream) -> (out, lse)
PyObject *sparse_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 15 || !g_calls.forward) Py_RETURN_NONE;
  try {
    ha_sparse_problem p;
    ha_view qv, kv, vv, ov;
    const int32_t *lists;
    void *stream, *ws;
    size_t bytes;
    int32_t with_lse;
    if (!attention_problem(args, 4, &p, &qv, &kv, &vv, &lists) || !flag(args[10], &with_lse)) Py_RETURN_NONE;
    const at::Tensor &q = *tensor(args[0]);
    const at::Tensor *out = args[11] == Py_None ? nullptr : tensor(args[11]), *lse = args[12] == Py_None ? nullptr : tensor(args[12]);
    const int64_t rows[] = {q.size(0), q.size(1), q.size(2)};
    if (!here(args[14], q, &stream) || (args[11] != Py_None && (!out || !same_sizes(*out, q))) || (args[12] != Py_None && !plain(lse, at::kFloat, rows, q))) Py_RETURN_NONE;
    at::Tensor keep, new_lse;
    const at::Tensor o = out ? *out : dense_like(q);
    if (!view_of(&o, q, &ov)) Py_RETURN_NONE;
    if (lse) new_lse = *lse;
    else if (with_lse) new_lse = fresh(rows, at::kFloat, q);
    if (!workspace_of(args[13], g_calls.forward_bytes(&p), q, &keep, &ws, &bytes)) Py_RETURN_NONE;
    float *lse_at = new_lse.defined() ? static_cast<float *>(new_lse.data_ptr()) : nullptr;
    ha_status st;
    HA_CALL(st, g_calls.forward(&p, &qv, &kv, &vv, lists, &ov, lse_at, ws, bytes, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_sparse_forward");
    const Ref o_py(THPVariable_Wrap(o));
    if (!new_lse.defined()) return PyTuple_Pack(2, o_py.p, Py_None);
    const Ref l_py(THPVariable_Wrap(new_lse));
    return PyTuple_Pack(2, o_py.p, l_py.p);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// sparse_grad(q, k, v, blocks, out, lse, grad_out, q_block, k_block, causal, q_start, key_len, softmax_scale, grad_q, grad_k, grad_v, workspace, stream) -> three gradients
PyObject *sparse_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 18 || !g_calls.grad) Py_RETURN_NONE;
  try {
    ha_sparse_problem p;
    ha_view qv, kv, vv, ov, dv, gv[3];
    const int32_t *lists;
    void *stream, *ws;
    size_t bytes;
    if (!attention_problem(args, 7, &p, &qv, &kv, &vv, &lists)) Py_RETURN_NONE;
    const at::Tensor &q = *tensor(args[0]), &k = *tensor(args[1]);
    const at::Tensor *out = tensor(args[4]), *lse = tensor(args[5]), *dout = tensor(args[6]);
    const int64_t rows[] = {q.size(0), q.size(1), q.size(2)};
    if (!here(args[17], q, &stream) || !view_of(out, q, &ov) || !view_of(dout, q, &dv) || !same_sizes(*out, q) || !same_sizes(*dout, q) || !plain(lse, at::kFloat, rows, q)) Py_RETURN_NONE;
    at::Tensor keep, grads[3];
    for (int i = 0; i < 3; ++i) {
      const at::Tensor &like = i == 0 ? q : k;
      const at::Tensor *given = args[13 + i] == Py_None ? nullptr : tensor(args[13 + i]);
      if (args[13 + i] != Py_None && (!given || !same_sizes(*given, like))) Py_RETURN_NONE;
      grads[i] = given ? *given : dense_like(i == 2 ? *tensor(args[2]) : like);
      if (!view_of(&grads[i], q, &gv[i])) Py_RETURN_NONE;
    }
    if (!workspace_of(args[16], std::max<size_t>(256, g_calls.grad_bytes(&p)), q, &keep, &ws, &bytes)) Py_RETURN_NONE;
    const float *lse_at = static_cast<const float *>(lse->data_ptr());
    ha_status st;
    HA_CALL(st, g_calls.grad(&p, &qv, &kv, &vv, lists, &ov, lse_at, &dv, &gv[0], &gv[1], &gv[2], ws, bytes, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_sparse_grad");
    const Ref a(THPVariable_Wrap(grads[0])), b(THPVariable_Wrap(grads[1])), c(THPVariable_Wrap(grads[2]));
    return PyTuple_Pack(3, a.p, b.p, c.p);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// One tensor of a list: contiguous, on the GPU that *device names (-1: none yet), of a type that the library has.
bool listed(PyObject *o, int64_t *device, const at::Tensor **t, int32_t *type) {
  *t = tensor(o);
  if (!*t || !(*t)->is_cuda() || !(*t)->is_contiguous() || (*device >= 0 && (*t)->get_device() != *device)) return false;
  if ((*t)->scalar_type() != at::kFloat && (*t)->scalar_type() != at::kBFloat16) return false;
  *device = (*t)->get_device();
  *type = (*t)->scalar_type() == at::kFloat ? HA_F32 : HA_BF16;
  return true;
}

// One entry of a ParamList's five lists: master, gradient, moments, copy (the last three may be None).
bool described(PyObject *const *list, Py_ssize_t i, int64_t *device, ha_param *out) {
  void *at[5];
  int32_t type[5] = {HA_F32, HA_F32, HA_F32, HA_F32, HA_BF16};
  int64_t size = 0;
  for (int f = 0; f < 5; ++f) {
    PyObject *o = PyList_GET_ITEM(list[f], i);
    at[f] = nullptr;
    if (f >= 2 && o == Py_None) continue;
    const at::Tensor *t;
    if (!listed(o, device, &t, &type[f]) || (f != 1 && f != 4 && type[f] != HA_F32) || (f > 0 && t->numel() != size)) return false;
    size = t->numel();
    at[f] = t->data_ptr();
  }
  *out = ha_param{static_cast<float *>(at[0]), at[1], static_cast<float *>(at[2]), static_cast<float *>(at[3]), at[4], static_cast<uint64_t>(size), type[1], type[4]};
  return true;
}
// The five lists of a ParamList, of one length.
bool five_lists(PyObject *o, PyObject **list) {
  if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 5) return false;
  for (int f = 0; f < 5; ++f) {
    list[f] = PyTuple_GET_ITEM(o, f);
    if (!PyList_CheckExact(list[f]) || PyList_GET_SIZE(list[f]) != PyList_GET_SIZE(list[0])) return false;
  }
  return true;
}

// Whether the descriptors are those of the tensors as they are now.
bool still(PyObject *tensors, const ha_tensor *d, Py_ssize_t n, int64_t device) {
  if (!PyList_CheckExact(tensors) || PyList_GET_SIZE(tensors) != n) return false;
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor *t;
    int32_t type;
    if (!listed(PyList_GET_ITEM(tensors, i), &device, &t, &type) || d[i].data != t->data_ptr() || d[i].n != static_cast<uint64_t>(t->numel()) || d[i].dtype != type) return false;
  }
  return true;
}
bool still(PyObject *tensors, const ha_param *d, Py_ssize_t n, int64_t device) {
  PyObject *list[5];
  if (!five_lists(tensors, list) || PyList_GET_SIZE(list[0]) != n) return false;
  for (Py_ssize_t i = 0; i < n; ++i) {
    ha_param p;
    if (!described(list, i, &device, &p) || p.master != d[i].master || p.grad != d[i].grad || p.m != d[i].m || p.v != d[i].v || p.param_io != d[i].param_io || p.n != d[i].n ||
        p.grad_dtype != d[i].grad_dtype || p.io_dtype != d[i].io_dtype)
      return false;
  }
  return true;
}

// The `native` tuple of a TensorList or a ParamList: address of the descriptors, how many, workspace bytes of the norm, device index.  A list whose tensors have other
// memory than is described is left to the Python code, which describes it anew.
struct List {
  void *at;
  int32_t n;
  size_t bytes;
  int64_t device;
};
template <typename Descriptor>
bool list_of(PyObject *o, List *out) {
  const Ref t(PyObject_GetAttr(o, g_native));
  if (!t.p || !PyTuple_CheckExact(t.p) || PyTuple_GET_SIZE(t.p) != 4) {
    PyErr_Clear();
    return false;
  }
  out->at = PyLong_AsVoidPtr(PyTuple_GET_ITEM(t.p, 0));
  out->n = static_cast<int32_t>(PyLong_AsLong(PyTuple_GET_ITEM(t.p, 1)));
  out->bytes = PyLong_AsSize_t(PyTuple_GET_ITEM(t.p, 2));
  out->device = PyLong_AsLong(PyTuple_GET_ITEM(t.p, 3));
  const Ref tensors(PyErr_Occurred() ? nullptr : PyObject_GetAttr(o, g_tensors));
  if (!tensors.p) {
    PyErr_Clear();
    return false;
  }
  return out->device >= 0 && still(tensors.p, static_cast<const Descriptor *>(out->at), out->n, out->device);
}
bool result_of(PyObject *o, int64_t device, const at::Tensor **out) {
  const at::Tensor *t = tensor(o);
  if (!t || !t->is_cuda() || t->get_device() != device || t->scalar_type() != at::kFloat || t->dim() != 1 || t->size(0) != 2 || !t->is_contiguous()) return false;
  *out = t;
  return true;
}

// grad_norm(list, max_norm, result, workspace, stream) -> result
PyObject *grad_norm(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 5 || !g_calls.norm) Py_RETURN_NONE;
  try {
    List list;
    float max_norm;
    const at::Tensor *given = nullptr;
    if (!list_of<ha_tensor>(args[0], &list) || !number(args[1], &max_norm) || (args[2] != Py_None && !result_of(args[2], list.device, &given))) Py_RETURN_NONE;
    const at::Tensor result = given ? *given : at::empty({2}, at::TensorOptions().dtype(at::kFloat).device(at::kCUDA, static_cast<c10::DeviceIndex>(list.device)));
    at::Tensor keep;
    void *stream, *ws;
    size_t bytes;
    if (!here(args[4], result, &stream) || !workspace_of(args[3], list.bytes, result, &keep, &ws, &bytes)) Py_RETURN_NONE;
    float *to = static_cast<float *>(result.data_ptr());
    ha_status st;
    HA_CALL(st, g_calls.norm(list.n, static_cast<const ha_tensor *>(list.at), max_norm, to, ws, bytes, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_grad_norm");
    return THPVariable_Wrap(result);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// grad_clip(list, result, out list, stream) -> status, or None (the Python code has compared the lists' sizes)
PyObject *grad_clip(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 4 || !g_calls.clip) Py_RETURN_NONE;
  try {
    List list, out;
    const at::Tensor *result;
    void *stream;
    if (!list_of<ha_tensor>(args[0], &list) || !list_of<ha_tensor>(args[2], &out) || list.n != out.n || list.device != out.device || !result_of(args[1], list.device, &result) ||
        !here(args[3], *result, &stream))
      Py_RETURN_NONE;
    const float *from = static_cast<const float *>(result->data_ptr());
    ha_status st;
    HA_CALL(st, g_calls.clip(list.n, static_cast<const ha_tensor *>(list.at), static_cast<const ha_tensor *>(out.at), from, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_grad_clip");
    return PyLong_FromLong(st);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// update_many(list, lr, kind, step, grad_scale, beta1, beta2, eps, weight_decay, result, stream) -> status, or None
PyObject *update_many(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 11 || !g_calls.many) Py_RETURN_NONE;
  try {
    List list;
    ha_optimizer o = {};
    const at::Tensor *result = nullptr;
    void *stream;
    if (!list_of<ha_param>(args[0], &list) || !number(args[1], &o.lr) || !small_int(args[2], &o.kind) || !small_int(args[3], &o.step) || !number(args[4], &o.grad_scale) ||
        !number(args[5], &o.beta1) || !number(args[6], &o.beta2) || !number(args[7], &o.eps) || !number(args[8], &o.weight_decay) ||
        !result_of(args[9], list.device, &result) || !here(args[10], *result, &stream))
      Py_RETURN_NONE;
    const float *from = static_cast<const float *>(result->data_ptr());
    ha_status st;
    HA_CALL(st, g_calls.many(&o, list.n, static_cast<const ha_param *>(list.at), from, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_param_update_many");
    return PyLong_FromLong(st);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// describe_tensors(list, address of as many ha_tensor) -> (device index, sizes), or None
PyObject *describe_tensors(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 2 || !PyList_CheckExact(args[0])) Py_RETURN_NONE;
  try {
    ha_tensor *to = static_cast<ha_tensor *>(PyLong_AsVoidPtr(args[1]));
    const Py_ssize_t count = PyList_GET_SIZE(args[0]);
    const Ref sizes(PyList_New(count));
    if (!to || !sizes.p) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    int64_t device = -1;
    for (Py_ssize_t i = 0; i < count; ++i) {
      const at::Tensor *t;
      int32_t type;
      if (!listed(PyList_GET_ITEM(args[0], i), &device, &t, &type)) Py_RETURN_NONE;
      to[i] = ha_tensor{t->data_ptr(), static_cast<uint64_t>(t->numel()), type, 0};
      PyObject *size = PyLong_FromLongLong(t->numel());
      if (!size) return nullptr;
      PyList_SET_ITEM(sizes.p, i, size);
    }
    return Py_BuildValue("(LO)", static_cast<long long>(device), sizes.p);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// describe_params((masters, grads, m, v, copies), address of as many ha_param) -> device index, or None
PyObject *describe_params(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 2) Py_RETURN_NONE;
  try {
    ha_param *to = static_cast<ha_param *>(PyLong_AsVoidPtr(args[1]));
    PyObject *list[5];
    if (!to || !five_lists(args[0], list)) {
      PyErr_Clear();
      Py_RETURN_NONE;
    }
    int64_t device = -1;
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list[0]); ++i)
      if (!described(list, i, &device, &to[i])) Py_RETURN_NONE;
    return PyLong_FromLongLong(device);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// bind_calls(addresses of the ten functions in the order of Calls, current-device function, class of errors)
PyObject *bind_calls(PyObject *, PyObject *args) {
  PyObject *list, *get_device, *error = nullptr;
  if (!PyArg_ParseTuple(args, "O!O|O", &PyTuple_Type, &list, &get_device, &error)) return nullptr;
  void *at[sizeof(Calls) / sizeof(void *)];
  constexpr Py_ssize_t N = sizeof(at) / sizeof(at[0]);
  if (PyTuple_GET_SIZE(list) != N) {
    PyErr_SetString(PyExc_ValueError, "another number of functions is wanted");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < N; ++i) at[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(list, i));
  if (PyErr_Occurred()) return nullptr;
  Py_INCREF(get_device);
  Py_XSETREF(g_get_device, get_device);
  Py_XINCREF(error);
  Py_XSETREF(g_error, error);
  if (!g_native && !(g_native = PyUnicode_InternFromString("native"))) return nullptr;
  if (!g_tensors && !(g_tensors = PyUnicode_InternFromString("tensors"))) return nullptr;
  static_assert(sizeof(g_calls) == sizeof(at), "function pointers only");
  std::memcpy(&g_calls, at, sizeof(g_calls));
  Py_RETURN_NONE;
}

}  // namespace
