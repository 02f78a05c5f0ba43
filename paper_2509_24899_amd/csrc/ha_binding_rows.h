// Marshalling of the calls of rotary positions and of paged caches (part of ha_binding.cpp, by the rules of ha_binding_calls.h: what is not plain and right gives None, and the
// Python code takes the call).
//
// Host time per call in Python / here, us: rotate 17 / 5, norm_rotate 25 / 6, its gradient 37 / 11, paged_append 23 / 5, paged_forward 19 / 5, paged_weights 17 / 4, paged_evict 27 / 10.
#pragma once

namespace {

struct RowCalls {
  ha_status (*rotate)(const ha_rows_problem *, const ha_rotary *, const ha_view *, const ha_view *, int32_t, void *);
  ha_status (*norm)(const ha_rows_problem *, const ha_rotary *, const ha_view *, const ha_view *, const float *, const float *, const ha_view *, const ha_view *, void *);
  size_t (*grad_bytes)(const ha_rows_problem *);
  ha_status (*grad)(const ha_rows_problem *, const ha_rotary *, const ha_view *, const ha_view *, const ha_view *, const ha_view *, const float *, const float *, const ha_view *,
                    const ha_view *, float *, float *, void *, size_t, void *);
  ha_status (*append)(const ha_paged_problem *, const ha_rotary *, int32_t, float, const ha_view *, const ha_view *, const ha_view *, const float *, const float *, const ha_view *,
                      const ha_view *, const ha_view *, void *);
  size_t (*forward_bytes)(const ha_paged_problem *);
  ha_status (*forward)(const ha_paged_problem *, const ha_view *, const ha_view *, const ha_view *, const ha_view *, float *, void *, size_t, void *);
  size_t (*weights_bytes)(const ha_paged_problem *);
  ha_status (*weights)(const ha_paged_problem *, const ha_view *, const ha_view *, const float *, const float *, float *, void *, size_t, void *);
  size_t (*evict_bytes)(const ha_paged_problem *, int32_t);
  ha_status (*evict)(const ha_paged_problem *, int32_t, int32_t, int32_t, const float *, const int32_t *, int32_t, const ha_view *, const ha_view *, int32_t *, float *, int32_t *,
                     void *, size_t, void *);
};
RowCalls g_rows = {};

bool fits(int64_t n) { return n >= 0 && n <= std::numeric_limits<int32_t>::max(); }
bool float_type(const at::Tensor &t, int32_t *out) {
  *out = t.scalar_type() == at::kBFloat16 ? HA_BF16 : HA_F32;
  return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat;
}
// An argument that may be None: *t is null then.
bool maybe(PyObject *o, const at::Tensor **t) {
  *t = nullptr;
  if (o == Py_None) return true;
  return (*t = tensor(o)) != nullptr;
}
// A contiguous fp32 (or int32) tensor of these sizes, or None.
template <typename T>
bool maybe_plain(PyObject *o, at::ScalarType type, at::IntArrayRef sizes, const at::Tensor &like, T **out) {
  const at::Tensor *t;
  *out = nullptr;
  if (!maybe(o, &t) || (t && !plain(t, type, sizes, like))) return false;
  if (t) *out = static_cast<T *>(t->data_ptr());
  return true;
}

// rotary: None or a tuple (freq, axis, interleaved, magnitude); positions [tokens, axes] or, with B > 0, [B, tokens, axes].
bool rotary_of(PyObject *o, PyObject *positions, int64_t tokens, int64_t B, const at::Tensor &like, ha_rotary *r) {
  *r = ha_rotary{};
  r->interleaved = r->n_axes = 1;
  r->magnitude = 1.f;
  if (o == Py_None) return true;
  if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) return false;
  const at::Tensor *freq = tensor(PyTuple_GET_ITEM(o, 0)), *axis, *at_ = tensor(positions);
  if (!freq || !at_ || !maybe(PyTuple_GET_ITEM(o, 1), &axis) || freq->dim() != 1 || !fits(2 * freq->size(0)) || !plain(freq, at::kDouble, freq->sizes(), like) ||
      (axis && !plain(axis, at::kInt, freq->sizes(), like)) || !flag(PyTuple_GET_ITEM(o, 2), &r->interleaved) || !number(PyTuple_GET_ITEM(o, 3), &r->magnitude))
    return false;
  const int64_t dim = at_->dim();
  if ((dim != 2 && dim != 3) || !plain(at_, at::kInt, at_->sizes(), like) || at_->size(dim - 2) != tokens || !fits(at_->size(dim - 1)) || (dim == 3 && at_->size(0) != B)) return false;
  r->freq = static_cast<const double *>(freq->data_ptr());
  r->axis = axis ? static_cast<const int32_t *>(axis->data_ptr()) : nullptr;
  r->positions = static_cast<const int32_t *>(at_->data_ptr());
  r->positions_stride_b = dim == 3 && B > 1 ? tokens * at_->size(2) : 0;
  r->rot_dim = static_cast<int32_t>(2 * freq->size(0));
  r->n_axes = static_cast<int32_t>(at_->size(dim - 1));
  return true;
}

bool rows_of(const at::Tensor &q, const at::Tensor *k, ha_rows_problem *p) {
  if (q.dim() != 4 || !fits(q.size(0)) || !fits(q.size(1)) || !fits(q.size(2)) || !fits(q.size(3))) return false;
  if (k && (k->dim() != 4 || k->size(0) != q.size(0) || k->size(2) != q.size(2) || k->size(3) != q.size(3) || !fits(k->size(1)))) return false;
  *p = ha_rows_problem{static_cast<int32_t>(q.size(0)), static_cast<int32_t>(q.size(1)), k ? static_cast<int32_t>(k->size(1)) : 0, static_cast<int32_t>(q.size(2)),
                       static_cast<int32_t>(q.size(3)), 0, 0.f};
  return float_type(q, &p->dtype);
}

// An output of like's shape: the one given, or a new one; its view.
bool output_of(PyObject *o, const at::Tensor &like, at::Tensor *out, ha_view *v) {
  const at::Tensor *t;
  if (!maybe(o, &t) || (t && !same_sizes(*t, like))) return false;
  *out = t ? *t : dense_like(like);
  return view_of(out, like, v);
}

// rotate(x, rotary, positions, transposed, out, stream) -> out
PyObject *rotate(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 6 || !g_rows.rotate) Py_RETURN_NONE;
  try {
    const at::Tensor *x = tensor(args[0]);
    ha_rows_problem p;
    ha_rotary r;
    ha_view xv, ov;
    int32_t transposed;
    void *stream;
    at::Tensor out;
    if (!x || args[1] == Py_None || !rows_of(*x, nullptr, &p) || !view_of(x, *x, &xv) || !rotary_of(args[1], args[2], x->size(2), x->size(0), *x, &r) || !flag(args[3], &transposed) ||
        !here(args[5], *x, &stream) || !output_of(args[4], *x, &out, &ov))
      Py_RETURN_NONE;
    ha_status st;
    HA_CALL(st, g_rows.rotate(&p, &r, &xv, &ov, transposed, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_rotate");
    return THPVariable_Wrap(out);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (a, b) with None in the place of a null tensor
PyObject *tuple_of(std::initializer_list<const at::Tensor *> list) {
  PyObject *t = PyTuple_New(static_cast<Py_ssize_t>(list.size()));
  Py_ssize_t i = 0;
  if (t)
    for (const at::Tensor *x : list) {
      PyObject *o = x && x->defined() ? THPVariable_Wrap(*x) : Py_None;
      if (o == Py_None) Py_INCREF(o);
      PyTuple_SET_ITEM(t, i++, o);
    }
  return t;
}

// norm_rotate(q, k, w_q, w_k, rotary, positions, eps, q_out, k_out, stream) -> (q_out, k_out)
PyObject *norm_rotate(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 10 || !g_rows.norm) Py_RETURN_NONE;
  try {
    const at::Tensor *q = tensor(args[0]), *k;
    ha_rows_problem p;
    ha_rotary r;
    ha_view qv, kv, qo, ko;
    const float *w[2];
    void *stream;
    at::Tensor q_out, k_out;
    if (!q || !maybe(args[1], &k) || !rows_of(*q, k, &p) || !view_of(q, *q, &qv) || (k && !view_of(k, *q, &kv)) || (!k && args[8] != Py_None) || !number(args[6], &p.eps)) Py_RETURN_NONE;
    const int64_t d[] = {q->size(3)};
    if (!maybe_plain(args[2], at::kFloat, d, *q, &w[0]) || !maybe_plain(args[3], at::kFloat, d, *q, &w[1]) || !rotary_of(args[4], args[5], q->size(2), q->size(0), *q, &r) ||
        !here(args[9], *q, &stream) || !output_of(args[7], *q, &q_out, &qo) || (k && !output_of(args[8], *k, &k_out, &ko)))
      Py_RETURN_NONE;
    ha_status st;
    HA_CALL(st, g_rows.norm(&p, &r, &qv, k ? &kv : nullptr, w[0], w[1], &qo, k ? &ko : nullptr, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_norm_rotate");
    return tuple_of({&q_out, &k_out});
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// norm_rotate_grad(grad_q, grad_k, q, k, w_q, w_k, rotary, positions, eps, grad_in_q, grad_in_k, grad_w_q, grad_w_k, workspace, stream) -> four gradients
PyObject *norm_rotate_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 15 || !g_rows.grad) Py_RETURN_NONE;
  try {
    const at::Tensor *x[2] = {tensor(args[2]), nullptr}, *g[2] = {tensor(args[0]), nullptr};
    if (!x[0] || !g[0] || !maybe(args[3], &x[1]) || !maybe(args[1], &g[1]) || !x[1] != !g[1] || (!x[1] && (args[10] != Py_None || args[12] != Py_None))) Py_RETURN_NONE;
    const at::Tensor &q = *x[0];
    ha_rows_problem p;
    ha_rotary r;
    ha_view xv[2], gv[2], ov[2];
    const float *w[2];
    at::Tensor out[2], dw[2], keep;
    void *stream, *ws;
    size_t bytes;
    if (!rows_of(q, x[1], &p) || !number(args[8], &p.eps) || !rotary_of(args[6], args[7], q.size(2), q.size(0), q, &r) || !here(args[14], q, &stream)) Py_RETURN_NONE;
    const int64_t d[] = {q.size(3)};
    const int count = x[1] ? 2 : 1;
    for (int i = 0; i < 2; ++i) {
      float *sum;
      if (!maybe_plain(args[4 + i], at::kFloat, d, q, &w[i]) || !maybe_plain(args[11 + i], at::kFloat, d, q, &sum) || (sum && !w[i])) Py_RETURN_NONE;
      if (i < count && (!same_sizes(*g[i], *x[i]) || !view_of(x[i], q, &xv[i]) || !view_of(g[i], q, &gv[i]) || !output_of(args[9 + i], *x[i], &out[i], &ov[i]))) Py_RETURN_NONE;
      if (i < count && w[i]) dw[i] = sum ? *tensor(args[11 + i]) : fresh(d, at::kFloat, q);
    }
    const bool sums = dw[0].defined() || dw[1].defined();
    if (!workspace_of(args[13], sums ? g_rows.grad_bytes(&p) : 0, q, &keep, &ws, &bytes)) Py_RETURN_NONE;
    float *sum_at[2];
    for (int i = 0; i < 2; ++i) sum_at[i] = dw[i].defined() ? static_cast<float *>(dw[i].data_ptr()) : nullptr;
    ha_status st;
    HA_CALL(st, g_rows.grad(&p, &r, &gv[0], count == 2 ? &gv[1] : nullptr, &xv[0], count == 2 ? &xv[1] : nullptr, w[0], w[1], &ov[0], count == 2 ? &ov[1] : nullptr, sum_at[0], sum_at[1],
                            ws, bytes, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_norm_rotate_grad");
    return tuple_of({&out[0], &out[1], &dw[0], &dw[1]});
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

bool packed_view(const at::Tensor *t, const at::Tensor &like, ha_view *v) {
  if (!t || t->dim() != 3 || t->scalar_type() != like.scalar_type() || t->device() != like.device() || (t->stride(2) != 1 && t->size(2) > 1)) return false;
  *v = ha_view{t->data_ptr(), 0, t->stride(1), t->stride(0)};
  return true;
}
// A new tensor of [T, heads, d] in the order of t's dimensions in memory, without its gaps and broadcast dimensions.
at::Tensor packed_like(const at::Tensor &t) {
  const int64_t T = t.size(0), H = t.size(1), d = t.size(2);
  const bool rows = t.stride(0) >= t.stride(1);
  const int64_t strides[] = {rows ? H * d : d, rows ? d : T * d, 1};
  return at::empty_strided(t.sizes(), strides, t.options());
}
bool packed_output(PyObject *o, const at::Tensor &like, at::Tensor *out, ha_view *v) {
  const at::Tensor *t;
  if (!maybe(o, &t) || (t && !same_sizes(*t, like))) return false;
  *out = t ? *t : packed_like(like);
  return packed_view(out, like, v);
}

// rows [T, heads, d], pools, and args[0 ..] = page_table, key_len
bool paged_of(const at::Tensor &like, int64_t T, int64_t H, const at::Tensor *k, const at::Tensor *v, PyObject *const *args, ha_paged_problem *p, ha_view *kv, ha_view *vv) {
  const at::Tensor *table = tensor(args[0]);
  if (!k || !view_of(k, like, kv) || (v && (!view_of(v, like, vv) || !same_sizes(*k, *v))) || !table || table->dim() != 2 || !plain(table, at::kInt, table->sizes(), like)) return false;
  *p = ha_paged_problem{};
  const int32_t *length;
  if (args[1] == Py_None || !per_entry(args[1], table->size(0), like, &length) || !float_type(like, &p->dtype)) return false;
  for (int64_t n : {table->size(0), table->size(1), T, H, k->size(0), k->size(1), k->size(2), k->size(3)})
    if (!fits(n)) return false;
  p->B = static_cast<int32_t>(table->size(0));
  p->H = static_cast<int32_t>(H);
  p->H_kv = static_cast<int32_t>(k->size(1));
  p->T = static_cast<int32_t>(T);
  p->d_head = static_cast<int32_t>(k->size(3));
  p->n_pages = static_cast<int32_t>(k->size(0));
  p->page = static_cast<int32_t>(k->size(2));
  p->max_pages = static_cast<int32_t>(table->size(1));
  p->softmax_scale = static_cast<float>(std::pow(static_cast<double>(std::max<int64_t>(k->size(3), 1)), -0.5));
  p->page_table = static_cast<const int32_t *>(table->data_ptr());
  p->key_len = length;
  return true;
}
// args[0 ..] = q_offset, max_new
bool new_tokens(PyObject *const *args, const at::Tensor &like, ha_paged_problem *p) {
  if (!per_entry(args[0], static_cast<int64_t>(p->B) + 1, like, &p->q_offset)) return false;
  if (args[1] != Py_None) return small_int(args[1], &p->max_new);
  if (!p->q_offset && (p->B == 0 || p->T % p->B)) return false;
  p->max_new = p->q_offset ? p->T : p->T / p->B;
  return true;
}

// paged_append(q, k, v, k_pages, v_pages, page_table, key_len, q_offset, max_new, w_q, w_k, rotary, positions, eps, q_out, stream) -> (q_out,)
PyObject *paged_append(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 16 || !g_rows.append) Py_RETURN_NONE;
  try {
    const at::Tensor *q, *k = tensor(args[1]), *v = tensor(args[2]);
    ha_paged_problem p;
    ha_rotary r;
    ha_view qv, kv, vv, kp, vp, ov;
    const float *w[2];
    float eps = 0.f;
    void *stream;
    at::Tensor out;
    if (!k || !maybe(args[0], &q) || !packed_view(k, *k, &kv) || !packed_view(v, *k, &vv) || !same_sizes(*k, *v) || (q && (!packed_view(q, *k, &qv) || q->size(0) != k->size(0) || q->size(2) != k->size(2))) ||
        (!q && args[14] != Py_None) || !paged_of(*k, k->size(0), (q ? q : k)->size(1), tensor(args[3]), tensor(args[4]), args + 5, &p, &kp, &vp) || !tensor(args[4]) ||
        k->size(1) != p.H_kv || k->size(2) != p.d_head || !new_tokens(args + 7, *k, &p))
      Py_RETURN_NONE;
    const int64_t d[] = {k->size(2)};
    const bool norm = args[13] != Py_None;
    if (!maybe_plain(args[9], at::kFloat, d, *k, &w[0]) || !maybe_plain(args[10], at::kFloat, d, *k, &w[1]) || (norm ? !number(args[13], &eps) : w[0] || w[1]) ||
        !rotary_of(args[11], args[12], k->size(0), 0, *k, &r) || !here(args[15], *k, &stream) || (q && !packed_output(args[14], *q, &out, &ov)))
      Py_RETURN_NONE;
    ha_status st;
    HA_CALL(st, g_rows.append(&p, &r, norm, eps, q ? &qv : nullptr, &kv, &vv, w[0], w[1], &kp, &vp, q ? &ov : nullptr, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_paged_append");
    return tuple_of({&out});
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// paged_forward(q, k_pages, v_pages, page_table, key_len, q_offset, max_new, causal, softmax_scale, with_lse, out, lse, workspace, stream) -> (out, lse)
PyObject *paged_forward(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 14 || !g_rows.forward) Py_RETURN_NONE;
  try {
    const at::Tensor *q = tensor(args[0]);
    ha_paged_problem p;
    ha_view qv, kp, vp, ov;
    int32_t with_lse;
    float *lse;
    void *stream, *ws;
    size_t bytes;
    at::Tensor out, new_lse, keep;
    if (!q || !packed_view(q, *q, &qv) || !tensor(args[2]) || !paged_of(*q, q->size(0), q->size(1), tensor(args[1]), tensor(args[2]), args + 3, &p, &kp, &vp) || q->size(2) != p.d_head ||
        !new_tokens(args + 5, *q, &p) || !flag(args[7], &p.causal) || (args[8] != Py_None && !number(args[8], &p.softmax_scale)) || !flag(args[9], &with_lse) || !here(args[13], *q, &stream))
      Py_RETURN_NONE;
    const int64_t rows[] = {q->size(0), q->size(1)};
    if (!maybe_plain(args[11], at::kFloat, rows, *q, &lse) || !packed_output(args[10], *q, &out, &ov) || !workspace_of(args[12], g_rows.forward_bytes(&p), *q, &keep, &ws, &bytes)) Py_RETURN_NONE;
    if (lse) {
      new_lse = *tensor(args[11]);
    } else if (with_lse) {
      new_lse = fresh(rows, at::kFloat, *q);
      lse = static_cast<float *>(new_lse.data_ptr());
    }
    ha_status st;
    HA_CALL(st, g_rows.forward(&p, &qv, &kp, &vp, &ov, lse, ws, bytes, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_paged_forward");
    return tuple_of({&out, &new_lse});
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// paged_weights(q, k_pages, lse, weights, page_table, key_len, q_offset, max_new, causal, softmax_scale, out, workspace, stream) -> out
PyObject *paged_weights(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 13 || !g_rows.weights) Py_RETURN_NONE;
  try {
    const at::Tensor *q = tensor(args[0]);
    ha_paged_problem p;
    ha_view qv, kp;
    float *lse, *weights, *given;
    void *stream, *ws;
    size_t bytes;
    at::Tensor out, keep;
    if (!q || !packed_view(q, *q, &qv) || !paged_of(*q, q->size(0), q->size(1), tensor(args[1]), nullptr, args + 4, &p, &kp, nullptr) || q->size(2) != p.d_head ||
        !new_tokens(args + 6, *q, &p) || !flag(args[8], &p.causal) || (args[9] != Py_None && !number(args[9], &p.softmax_scale)) || !here(args[12], *q, &stream))
      Py_RETURN_NONE;
    const int64_t rows[] = {q->size(0), q->size(1)}, slots[] = {p.B, p.H_kv, static_cast<int64_t>(p.max_pages) * p.page};
    if (args[2] == Py_None || !maybe_plain(args[2], at::kFloat, rows, *q, &lse) || !maybe_plain(args[3], at::kFloat, slots, *q, &weights) || !maybe_plain(args[10], at::kFloat, slots, *q, &given))
      Py_RETURN_NONE;
    out = given ? *tensor(args[10]) : weights ? *tensor(args[3]) : fresh(slots, at::kFloat, *q);
    if (!workspace_of(args[11], g_rows.weights_bytes(&p), *q, &keep, &ws, &bytes)) Py_RETURN_NONE;
    float *to = static_cast<float *>(out.data_ptr());
    ha_status st;
    HA_CALL(st, g_rows.weights(&p, &qv, &kp, lse, weights, to, ws, bytes, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_paged_weights");
    return THPVariable_Wrap(out);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// paged_evict(k_pages, v_pages, weights, page_table, key_len, keep, out_table, keep_first, keep_last, len_out, weights_out, kept, workspace, stream) -> (len_out, weights_out, kept)
PyObject *paged_evict(PyObject *, PyObject *const *args, Py_ssize_t n) {
  if (n != 14 || !g_rows.evict) Py_RETURN_NONE;
  try {
    const at::Tensor *k = tensor(args[0]), *v = tensor(args[1]), *to = tensor(args[6]);
    ha_paged_problem p;
    ha_view kp, vp;
    int32_t keep, first, last, *lengths, *kept;
    float *weights, *weights_out;
    void *stream, *ws;
    size_t bytes;
    at::Tensor held;
    if (!k || !v || k->dim() != 4 || !paged_of(*k, 0, k->size(1), k, v, args + 3, &p, &kp, &vp) || !small_int(args[5], &keep) || keep < 1 || !small_int(args[7], &first) ||
        !small_int(args[8], &last) || !here(args[13], *k, &stream) || !to || to->dim() != 2 || !fits(to->size(1)))
      Py_RETURN_NONE;
    p.causal = 1;
    const int64_t slots[] = {p.B, p.H_kv, static_cast<int64_t>(p.max_pages) * p.page}, stay[] = {p.B, p.H_kv, keep}, entries[] = {p.B}, tables[] = {p.B, to->size(1)};
    // (no new tokens: a list of none)
    p.max_new = 0;
    if (args[2] == Py_None || !maybe_plain(args[2], at::kFloat, slots, *k, &weights) || !plain(to, at::kInt, tables, *k) || !maybe_plain(args[9], at::kInt, entries, *k, &lengths) ||
        !maybe_plain(args[10], at::kFloat, slots, *k, &weights_out) || !maybe_plain(args[11], at::kInt, stay, *k, &kept) ||
        !workspace_of(args[12], g_rows.evict_bytes(&p, keep), *k, &held, &ws, &bytes))
      Py_RETURN_NONE;
    const at::Tensor a = lengths ? *tensor(args[9]) : fresh(entries, at::kInt, *k), b = weights_out ? *tensor(args[10]) : fresh(slots, at::kFloat, *k),
                     c = kept ? *tensor(args[11]) : fresh(stay, at::kInt, *k);
    const int32_t *table = static_cast<const int32_t *>(to->data_ptr());
    const int32_t pages = static_cast<int32_t>(to->size(1));
    lengths = static_cast<int32_t *>(a.data_ptr());
    weights_out = static_cast<float *>(b.data_ptr());
    kept = static_cast<int32_t *>(c.data_ptr());
    ha_status st;
    HA_CALL(st, g_rows.evict(&p, keep, first, last, weights, table, pages, &kp, &vp, lengths, weights_out, kept, ws, bytes, stream));
    if (st != HA_OK) return failed(st, "hybrid_attn_paged_evict");
    return tuple_of({&a, &b, &c});
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// bind_rows(addresses of the eleven functions in the order of RowCalls); behind bind_calls
PyObject *bind_rows(PyObject *, PyObject *args) {
  PyObject *list;
  if (!PyArg_ParseTuple(args, "O!", &PyTuple_Type, &list)) return nullptr;
  void *at[sizeof(RowCalls) / sizeof(void *)];
  constexpr Py_ssize_t N = sizeof(at) / sizeof(at[0]);
  if (PyTuple_GET_SIZE(list) != N) {
    PyErr_SetString(PyExc_ValueError, "another number of functions is wanted");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < N; ++i) at[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(list, i));
  if (PyErr_Occurred()) return nullptr;
  static_assert(sizeof(g_rows) == sizeof(at), "function pointers only");
  std::memcpy(static_cast<void *>(&g_rows), at, sizeof(g_rows));
  Py_RETURN_NONE;
}

}  // namespace
#undef HA_CALL
