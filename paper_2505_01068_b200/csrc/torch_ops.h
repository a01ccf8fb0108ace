// Marshalling of the calls of gsit_ops.h; a part of torch_ext.cpp, whose helpers it uses.  Arguments in the order of the Python
// functions in binding.py.

// Row stride (elements) of a [B, L, H, hd] view whose heads are contiguous and whose rows are evenly spaced over all samples.
int64_t head_rows(const at::Tensor& t, const char* what) {
  require(t.is_cuda() && t.dim() == 4, what);
  const int64_t B = t.size(0), L = t.size(1), H = t.size(2), hd = t.size(3);
  require((hd == 1 || t.stride(3) == 1) && (H == 1 || t.stride(2) == hd), what);
  if (L == 1) return B > 1 ? t.stride(0) : H * hd;
  require(B == 1 || t.stride(0) == L * t.stride(1), what);
  return t.stride(1);
}
// ... of a [B, L, d] view.
int64_t feature_rows(const at::Tensor& t, const char* what) {
  require(t.is_cuda() && t.dim() == 3 && (t.size(2) == 1 || t.stride(2) == 1), what);
  if (t.size(1) == 1) return t.size(0) > 1 ? t.stride(0) : t.size(2);
  require(t.size(0) == 1 || t.stride(0) == t.size(1) * t.stride(1), what);
  return t.stride(1);
}
const float* float_vector(const at::Tensor* t, int64_t n, const char* what) {
  require(t == nullptr || (t->is_cuda() && t->scalar_type() == at::kFloat && t->is_contiguous() && t->numel() == n), what);
  return static_cast<const float*>(ptr(t));
}
// A workspace that the caller gives.
const at::Tensor* scratch(PyObject* o) {
  const at::Tensor* t = opt_tensor(o);
  require(t == nullptr || (t->is_cuda() && t->is_contiguous()), "workspace: contiguous, on the device");
  return t;
}
PyObject* pack(std::initializer_list<at::Tensor> ts) {
  PyObject* tuple = PyTuple_New((Py_ssize_t)ts.size());
  if (tuple == nullptr) throw PyFail{};
  Py_ssize_t i = 0;
  for (const at::Tensor& t : ts) {
    PyObject* o = THPVariable_Wrap(t);
    if (o == nullptr) {
      Py_DECREF(tuple);
      throw PyFail{};
    }
    PyTuple_SET_ITEM(tuple, i++, o);
  }
  return tuple;
}
void require_length(const gsit_shape& s, int64_t L) {
  require((int64_t)s.seg_len[0] + s.seg_len[1] + s.seg_len[2] == L, "seg_len adds up to the length of the rows");
}

// Positions (may be null where none are read) and how many pairs belong to each axis.
gsit_rotary read_rotary(const at::Tensor* pos, PyObject* of_axis, int64_t B, int64_t L, int64_t hd, int64_t HK) {
  gsit_rotary r = {};
  PyObject* sections = PySequence_Fast(of_axis, "sections must be a sequence of one to three numbers of pairs");
  if (sections == nullptr) throw PyFail{};
  const Py_ssize_t axes = PySequence_Fast_GET_SIZE(sections);
  bool read = axes >= 1 && axes <= 3;
  for (Py_ssize_t i = 0; read && i < axes; ++i) {
    const long v = PyLong_AsLong(PySequence_Fast_GET_ITEM(sections, i));
    if (v == -1 && PyErr_Occurred()) {
      Py_DECREF(sections);
      throw PyFail{};
    }
    read = v >= 0 && v <= hd;
    r.sections[i] = (int32_t)v;
  }
  Py_DECREF(sections);
  require(read, "sections: one to three numbers of pairs, none negative or above head_dim");
  r.kv_heads = (int32_t)HK;
  if (pos == nullptr) return r;
  require(pos->is_cuda() && pos->scalar_type() == at::kInt && (pos->dim() == 2 || pos->dim() == 3) && pos->size(0) == axes && pos->size(-1) == L &&
              (L == 1 || pos->stride(-1) == 1), "positions: int32 [axes, B, L] or [axes, L] on the device");
  require(pos->dim() == 2 || pos->size(1) == B || pos->size(1) == 1, "positions: one row per sample, or one for all");
  r.positions = static_cast<const int32_t*>(pos->data_ptr());
  r.axis_stride = axes > 1 ? pos->stride(0) : 0;
  r.batch_stride = pos->dim() == 3 && pos->size(1) > 1 ? pos->stride(1) : 0;
  return r;
}

// q, k (or None), positions, sections, seg_len, valid_len, base, interleaved, out_q, out_k, backward
PyObject* rotary(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0]), &pos = tensor(a[2]);
  const at::Tensor *k = opt_tensor(a[1]), *valid = opt_tensor(a[5]), *out_q = opt_tensor(a[8]), *out_k = opt_tensor(a[9]);
  const int64_t ldq = head_rows(q, "q: [B, L, H, hd] on the device, heads contiguous, rows evenly spaced");
  const int64_t B = q.size(0), L = q.size(1), H = q.size(2), hd = q.size(3);
  int64_t ldk = 0, HK = 0;
  if (k != nullptr) {
    ldk = head_rows(*k, "k: [B, L, H, hd] on the device, heads contiguous, rows evenly spaced");
    HK = k->size(2);
    require(k->size(0) == B && k->size(1) == L && k->size(3) == hd && k->scalar_type() == q.scalar_type(), "q and k share batch, length, head width and dtype");
  }
  const gsit_shape s = make_shape(B, a[4], H * hd, H, valid, dtype_code(q), GSIT_PHASE_INTRA, 0, 0.0);
  require_length(s, L);
  gsit_rotary r = read_rotary(&pos, a[3], B, L, hd, HK);
  r.base = as_float(a[6]);
  r.interleaved = as_bool(a[7]);
  at::Tensor mq, mk;
  auto result = [&](const at::Tensor* given, const at::Tensor& like, at::Tensor& made) {
    if (given == nullptr) made = empty(like.sizes(), like.scalar_type(), like.device());
    else {
      require(given->sizes() == like.sizes() && given->scalar_type() == like.scalar_type(), "results: shape and dtype of the inputs");
      made = *given;
    }
    return head_rows(made, "results: [B, L, H, hd] on the device, heads contiguous, rows evenly spaced");
  };
  const int64_t ldqo = result(out_q, q, mq), ldko = k == nullptr ? 0 : result(out_k, *k, mk);
  const auto call = as_bool(a[10]) ? gsit_rotary_bwd : gsit_rotary_fwd;
  gsit_status st;
  {
    NoGil n;
    st = call(&s, &r, q.data_ptr(), ldq, ptr(k), ldk, mq.data_ptr(), ldqo, k == nullptr ? nullptr : mk.data_ptr(), ldko, stream());
  }
  check(st, "gsit_rotary");
  if (k == nullptr) return THPVariable_Wrap(std::move(mq));
  return pack({mq, mk});
}

// Everything lies on the current device: kernels run there, and their pointers are not looked at.
void here(std::initializer_list<const at::Tensor*> ts) {
  const int dev = c10::cuda::current_device();
  for (const at::Tensor* t : ts) require(t == nullptr || (t->is_cuda() && t->device().index() == dev), "tensors on the current device");
}
const float* gamma_of(const at::Tensor* t, int64_t hd) { return float_vector(t, hd, "gamma: contiguous float32 [head_dim] on the device"); }

const char* const HEAD_ROWS = "[B, L, H, hd] on the device, heads contiguous, rows evenly spaced";

// q, k (or None), q_gamma, k_gamma, positions, sections, seg_len, valid_len, base, interleaved, eps, out_q, out_k
// and backward: dq, dk in front, want_params, workspace behind
template <bool BWD> PyObject* head_norm(PyObject* const* args) {
  PyObject* const* a = args + (BWD ? 2 : 0);
  const at::Tensor& q = tensor(a[0]);
  const at::Tensor *k = opt_tensor(a[1]), *q_gamma = opt_tensor(a[2]), *k_gamma = opt_tensor(a[3]), *pos = opt_tensor(a[4]), *valid = opt_tensor(a[7]);
  const at::Tensor *out_q = opt_tensor(a[11]), *out_k = opt_tensor(a[12]);
  const at::Tensor *dq = BWD ? &tensor(args[0]) : nullptr, *dk = BWD ? opt_tensor(args[1]) : nullptr, *ws = BWD ? scratch(a[14]) : nullptr;
  here({&q, k, q_gamma, k_gamma, pos, valid, out_q, out_k, dq, dk, ws});
  const int64_t ldq = head_rows(q, HEAD_ROWS), ldk = k == nullptr ? 0 : head_rows(*k, HEAD_ROWS);
  const int64_t B = q.size(0), L = q.size(1), H = q.size(2), hd = q.size(3), HK = k == nullptr ? 0 : k->size(2);
  require(k == nullptr || (k->size(0) == B && k->size(1) == L && k->size(3) == hd && k->scalar_type() == q.scalar_type()),
          "q and k share batch, length, head width and dtype");
  require(k != nullptr || (out_k == nullptr && k_gamma == nullptr && dk == nullptr), "without k there is nothing for it");
  const gsit_shape s = make_shape(B, a[6], H * hd, H, valid, dtype_code(q), GSIT_PHASE_INTRA, 0, 0.0);
  require_length(s, L);
  gsit_rotary r = {};
  r.kv_heads = (int32_t)HK;
  if (a[5] != Py_None) {
    r = read_rotary(pos, a[5], B, L, hd, HK);
    require(pos != nullptr || r.sections[0] + r.sections[1] + r.sections[2] == 0, "positions: int32 [axes, B, L] or [axes, L] on the device");
  } else {
    require(pos == nullptr, "positions are read with sections only");
  }
  r.base = as_float(a[8]);
  r.interleaved = as_bool(a[9]);
  const float eps = (float)as_float(a[10]);
  const float *gq = gamma_of(q_gamma, hd), *gk = gamma_of(k_gamma, hd);
  int64_t lddq = 0, lddk = 0;
  if constexpr (BWD) {
    require(dq->sizes() == q.sizes() && dq->scalar_type() == q.scalar_type() && (dk == nullptr) == (k == nullptr) &&
                (k == nullptr || (dk->sizes() == k->sizes() && dk->scalar_type() == q.scalar_type())), "gradients: shape and dtype of q and k");
    lddq = head_rows(*dq, HEAD_ROWS);
    lddk = dk == nullptr ? 0 : head_rows(*dk, HEAD_ROWS);
  }
  at::Tensor mq, mk, gam_q, gam_k, made_ws;
  auto result = [&](const at::Tensor* given, const at::Tensor& like, at::Tensor& made) {
    if (given == nullptr) made = empty(like.sizes(), like.scalar_type(), like.device());
    else {
      require(given->sizes() == like.sizes() && given->scalar_type() == like.scalar_type(), "results: shape and dtype of the inputs");
      made = *given;
    }
    return head_rows(made, HEAD_ROWS);
  };
  const int64_t ldqo = result(out_q, q, mq), ldko = k == nullptr ? 0 : result(out_k, *k, mk);
  void* ko = k == nullptr ? nullptr : mk.data_ptr();
  const bool params = BWD && as_bool(a[13]);
  if (params) {
    gam_q = empty({hd}, at::kFloat, q.device());
    if (k != nullptr) gam_k = empty({hd}, at::kFloat, q.device());
    if (ws == nullptr) {
      const size_t need = gsit_head_norm_rotary_bwd_workspace(&s);
      if (need == (size_t)-1) check(GSIT_ERR_UNSUPPORTED, "gsit_head_norm_rotary_bwd_workspace");
      made_ws = empty({(int64_t)need}, at::kByte, q.device());
      ws = &made_ws;
    }
  }
  gsit_status st;
  {
    NoGil n;
    if constexpr (!BWD)
      st = gsit_head_norm_rotary_fwd(&s, &r, eps, q.data_ptr(), ldq, gq, ptr(k), ldk, gk, mq.data_ptr(), ldqo, ko, ldko, stream());
    else
      st = gsit_head_norm_rotary_bwd(&s, &r, eps, q.data_ptr(), ldq, gq, ptr(k), ldk, gk, dq->data_ptr(), lddq, ptr(dk), lddk, mq.data_ptr(), ldqo, ko, ldko,
                                     params ? static_cast<float*>(gam_q.data_ptr()) : nullptr, params && k != nullptr ? static_cast<float*>(gam_k.data_ptr()) : nullptr,
                                     ptr(ws), ws == nullptr ? 0 : (size_t)ws->nbytes(), stream());
  }
  check(st, BWD ? "gsit_head_norm_rotary_bwd" : "gsit_head_norm_rotary_fwd");
  if (params && k == nullptr) return pack({mq, gam_q});
  if (params) return pack({mq, mk, gam_q, gam_k});
  if (k == nullptr) return THPVariable_Wrap(std::move(mq));
  return pack({mq, mk});
}

// Shape of a call on rows [B, L, d] (seg_len None: one segment) with a geometry that reads no heads.
gsit_shape row_shape(const at::Tensor& x, PyObject* seg, const at::Tensor* valid) {
  gsit_shape s;
  if (seg == Py_None) {
    PyObject* one = Py_BuildValue("(Lii)", (long long)x.size(1), 0, 0);
    if (one == nullptr) throw PyFail{};
    try {
      s = make_shape(x.size(0), one, x.size(2), 1, valid, GSIT_F32, GSIT_PHASE_INTRA, 0, 0.0);
    } catch (...) {
      Py_DECREF(one);
      throw;
    }
    Py_DECREF(one);
  } else {
    s = make_shape(x.size(0), seg, x.size(2), 1, valid, GSIT_F32, GSIT_PHASE_INTRA, 0, 0.0);
  }
  require_length(s, x.size(1));
  return s;
}

// x, gamma, beta, seg_len, valid_len, eps, out dtype as a code (-1: of x), want_stats, out
PyObject* layer_norm_fwd(PyObject* const* a) {
  const at::Tensor& x = tensor(a[0]);
  const at::Tensor *gamma = opt_tensor(a[1]), *beta = opt_tensor(a[2]), *valid = opt_tensor(a[4]), *out = opt_tensor(a[8]);
  const int64_t ldx = feature_rows(x, "x: [B, L, d] on the device, features contiguous, rows evenly spaced");
  const gsit_shape s = row_shape(x, a[3], valid);
  const int64_t d = x.size(2), code = as_int(a[6]);
  const float* ga = float_vector(gamma, d, "gamma: contiguous float32 [d]");
  const float* be = float_vector(beta, d, "beta: contiguous float32 [d]");
  at::Tensor y, mean, rstd;
  if (out != nullptr) {
    require(out->sizes() == x.sizes(), "out: shape of x");
    y = *out;
  } else {
    y = empty(x.sizes(), code < 0 ? x.scalar_type() : code == GSIT_BF16 ? at::kBFloat16 : at::kFloat, x.device());
  }
  const int64_t ldy = feature_rows(y, "out: [B, L, d] on the device, features contiguous, rows evenly spaced");
  const bool stats = as_bool(a[7]);
  if (stats) {
    mean = empty({x.size(0), x.size(1)}, at::kFloat, x.device());
    rstd = empty({x.size(0), x.size(1)}, at::kFloat, x.device());
  }
  const int32_t tx = dtype_code(x), ty = dtype_code(y);
  const float eps = (float)as_float(a[5]);
  gsit_status st;
  {
    NoGil n;
    st = gsit_layer_norm_fwd(&s, tx, x.data_ptr(), ldx, ga, be, eps, ty, y.data_ptr(), ldy,
                             stats ? static_cast<float*>(mean.data_ptr()) : nullptr, stats ? static_cast<float*>(rstd.data_ptr()) : nullptr, stream());
  }
  check(st, "gsit_layer_norm_fwd");
  if (!stats) return THPVariable_Wrap(std::move(y));
  return pack({y, mean, rstd});
}

// dy, x, mean, rstd, gamma, seg_len, valid_len, residual, want_params, out, workspace
PyObject* layer_norm_bwd(PyObject* const* a) {
  const at::Tensor &dy = tensor(a[0]), &x = tensor(a[1]), &mean = tensor(a[2]), &rstd = tensor(a[3]);
  const at::Tensor *gamma = opt_tensor(a[4]), *valid = opt_tensor(a[6]), *residual = opt_tensor(a[7]), *out = opt_tensor(a[9]), *ws = scratch(a[10]);
  const int64_t ldx = feature_rows(x, "x: [B, L, d] on the device, features contiguous, rows evenly spaced");
  const int64_t lddy = feature_rows(dy, "dy: [B, L, d] on the device, features contiguous, rows evenly spaced");
  require(dy.sizes() == x.sizes(), "dy and x share their shape");
  const gsit_shape s = row_shape(x, a[5], valid);
  const int64_t d = x.size(2), rows = x.size(0) * x.size(1);
  const float* ga = float_vector(gamma, d, "gamma: contiguous float32 [d]");
  const float* mu = float_vector(&mean, rows, "mean: contiguous float32 [B, L]");
  const float* rs = float_vector(&rstd, rows, "rstd: contiguous float32 [B, L]");
  int64_t ldres = 0;
  if (residual != nullptr) {
    require(residual->sizes() == x.sizes() && residual->scalar_type() == x.scalar_type(), "residual: shape and dtype of x");
    ldres = feature_rows(*residual, "residual: [B, L, d] on the device, features contiguous, rows evenly spaced");
  }
  at::Tensor dx, dgamma, dbeta, made_ws;
  if (out != nullptr) {
    require(out->sizes() == x.sizes() && out->scalar_type() == x.scalar_type(), "out: shape and dtype of x");
    dx = *out;
  } else {
    dx = empty(x.sizes(), x.scalar_type(), x.device());
  }
  const int64_t lddx = feature_rows(dx, "out: [B, L, d] on the device, features contiguous, rows evenly spaced");
  const bool params = as_bool(a[8]);
  if (params) {
    dgamma = empty({d}, at::kFloat, x.device());
    dbeta = empty({d}, at::kFloat, x.device());
    if (ws == nullptr) {
      const size_t need = gsit_layer_norm_bwd_workspace(&s);
      if (need == (size_t)-1) check(GSIT_ERR_UNSUPPORTED, "gsit_layer_norm_bwd_workspace");
      made_ws = empty({(int64_t)need}, at::kByte, x.device());
      ws = &made_ws;
    }
  }
  const int32_t tx = dtype_code(x), ty = dtype_code(dy);
  gsit_status st;
  {
    NoGil n;
    st = gsit_layer_norm_bwd(&s, ty, dy.data_ptr(), lddy, tx, x.data_ptr(), ldx, mu, rs, ga, ptr(residual), ldres, dx.data_ptr(), lddx,
                             params ? static_cast<float*>(dgamma.data_ptr()) : nullptr, params ? static_cast<float*>(dbeta.data_ptr()) : nullptr,
                             ptr(ws), ws == nullptr ? 0 : (size_t)ws->nbytes(), stream());
  }
  check(st, "gsit_layer_norm_bwd");
  if (!params) return THPVariable_Wrap(std::move(dx));
  return pack({dx, dgamma, dbeta});
}

// The rule of an attention call: softcap, slopes, times, documents, causal, prefix at a[0] .. a[5].
gsit_score_rule score_rule(PyObject* const* a, int64_t B, int64_t L, int64_t H, int64_t HK) {
  gsit_score_rule r = {};
  r.softcap = (float)as_float(a[0]);
  r.slopes = float_vector(opt_tensor(a[1]), H, "slopes: contiguous float32 [heads] on the device");
  r.times = float_vector(opt_tensor(a[2]), B * L, "times: contiguous float32 [B, L] on the device");
  const at::Tensor* docs = opt_tensor(a[3]);
  require(docs == nullptr || (docs->is_cuda() && docs->scalar_type() == at::kInt && docs->is_contiguous() && docs->numel() == B * L),
          "documents: contiguous int32 [B, L] on the device");
  r.documents = static_cast<const int32_t*>(ptr(docs));
  r.causal = as_bool(a[4]);
  r.prefix = float_vector(opt_tensor(a[5]), B, "prefix: contiguous float32 [B] on the device");
  r.kv_heads = (int32_t)HK;
  return r;
}

const char* const QKV_VIEWS = "q, k, v: [B, L, H, hd] on the device, heads contiguous, rows evenly spaced";

// q, k, v, seg_len, valid_len, phase, custom_mask, scale, softcap, slopes, times, documents, causal, prefix, q_len, want_lse, out
PyObject* scored_fwd(PyObject* const* a) {
  const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]);
  const at::Tensor *valid = opt_tensor(a[4]), *out = opt_tensor(a[16]);
  const int64_t ldq = head_rows(q, QKV_VIEWS), ldk = head_rows(k, QKV_VIEWS), ldv = head_rows(v, QKV_VIEWS);
  const int64_t B = q.size(0), Lq = q.size(1), H = q.size(2), hd = q.size(3), L = k.size(1), HK = k.size(2);
  require(k.sizes() == v.sizes() && k.size(0) == B && k.size(3) == hd && k.scalar_type() == q.scalar_type() && v.scalar_type() == q.scalar_type(),
          "q, k and v share batch, head width and dtype, k and v their shape");
  const gsit_shape s = make_shape(B, a[3], H * hd, H, valid, dtype_code(q), as_int(a[5]), as_int(a[6]), as_float(a[7]));
  require_length(s, L);
  gsit_score_rule r = score_rule(a + 8, B, L, H, HK);
  if (a[14] != Py_None) {
    r.tail = 1;
    read_segments(a[14], r.q_len);
    require((int64_t)r.q_len[0] + r.q_len[1] + r.q_len[2] == Lq, "q_len adds up to the rows of q");
  } else {
    require(Lq == L, "q, k and v share their length (or q_len says how many of the newest positions q holds)");
  }
  const bool want_lse = as_bool(a[15]);
  at::Tensor made, lse;
  if (out == nullptr) made = empty({B, Lq, H * hd}, q.scalar_type(), q.device());
  else require(out->is_cuda() && out->is_contiguous() && out->scalar_type() == q.scalar_type() && out->numel() == B * Lq * H * hd, "out: contiguous [B, L, d] of q's dtype");
  if (want_lse) lse = empty({B, H, Lq}, at::kFloat, q.device());
  void* dst = out != nullptr ? out->data_ptr() : made.data_ptr();
  float* lse_p = want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr;
  gsit_status st;
  {
    NoGil n;
    st = gsit_im_scored_attention_fwd(&s, &r, q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, dst, lse_p, nullptr, 0, stream());
  }
  check(st, "gsit_im_scored_attention_fwd");
  if (!want_lse) return out != nullptr ? Py_NewRef(a[16]) : THPVariable_Wrap(std::move(made));
  return pack({out != nullptr ? *out : made, lse});
}

// dout, q, k, v, out, lse, seg_len, valid_len, phase, custom_mask, scale, softcap, slopes, times, documents, causal, prefix, grads, workspace
PyObject* scored_bwd(PyObject* const* a) {
  const at::Tensor &dout = tensor(a[0]), &q = tensor(a[1]), &k = tensor(a[2]), &v = tensor(a[3]), &out = tensor(a[4]), &lse = tensor(a[5]);
  const at::Tensor *valid = opt_tensor(a[7]), *ws = scratch(a[18]);
  const int64_t ldq = head_rows(q, QKV_VIEWS), ldk = head_rows(k, QKV_VIEWS), ldv = head_rows(v, QKV_VIEWS);
  const int64_t B = q.size(0), L = q.size(1), H = q.size(2), hd = q.size(3), HK = k.size(2);
  require(k.sizes() == v.sizes() && k.size(0) == B && k.size(1) == L && k.size(3) == hd && k.scalar_type() == q.scalar_type() &&
              v.scalar_type() == q.scalar_type(), "q, k and v share batch, length, head width and dtype, k and v their shape");
  for (const at::Tensor* t : {&out, &dout})
    require(t->scalar_type() == q.scalar_type() && t->dim() == 3 && t->size(0) == B && t->size(1) == L && t->size(2) == H * hd, "out, dout: [B, L, d] of q's dtype");
  const int64_t ldo = feature_rows(out, "out: [B, L, d] on the device, features contiguous, rows evenly spaced");
  const int64_t lddo = feature_rows(dout, "dout: [B, L, d] on the device, features contiguous, rows evenly spaced");
  const float* lse_p = float_vector(&lse, B * H * L, "lse: contiguous float32 [B, H, L] on the device");
  const gsit_shape s = make_shape(B, a[6], H * hd, H, valid, dtype_code(q), as_int(a[8]), as_int(a[9]), as_float(a[10]));
  require_length(s, L);
  const gsit_score_rule r = score_rule(a + 11, B, L, H, HK);
  at::Tensor grad[3], made_ws;
  int64_t ld[3];
  const at::Tensor* like[3] = {&q, &k, &v};
  PyObject* given = a[17] == Py_None ? nullptr : PySequence_Fast(a[17], "grads must be a sequence of three tensors");
  if (a[17] != Py_None && given == nullptr) throw PyFail{};
  struct Release {
    PyObject* o;
    ~Release() { Py_XDECREF(o); }
  } release{given};
  require(given == nullptr || PySequence_Fast_GET_SIZE(given) == 3, "grads must be a sequence of three tensors");
  for (int i = 0; i < 3; ++i) {
    if (given != nullptr) {
      grad[i] = tensor(PySequence_Fast_GET_ITEM(given, i));
      require(grad[i].sizes() == like[i]->sizes() && grad[i].scalar_type() == q.scalar_type(), "grads: shape and dtype of q, k and v");
    } else {
      grad[i] = empty(like[i]->sizes(), q.scalar_type(), q.device());
    }
    ld[i] = head_rows(grad[i], "grads: [B, L, H, hd] on the device, heads contiguous, rows evenly spaced");
  }
  const size_t need = gsit_scored_attention_bwd_workspace(&s, &r);
  if (ws == nullptr && need != (size_t)-1) {
    made_ws = empty({(int64_t)need}, at::kByte, q.device());
    ws = &made_ws;
  }
  gsit_status st;
  {
    NoGil n;
    st = gsit_im_scored_attention_bwd(&s, &r, q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, out.data_ptr(), ldo, lse_p, dout.data_ptr(), lddo,
                                      grad[0].data_ptr(), ld[0], grad[1].data_ptr(), ld[1], grad[2].data_ptr(), ld[2], ptr(ws),
                                      ws == nullptr ? 0 : (size_t)ws->nbytes(), stream());
  }
  check(st, "gsit_im_scored_attention_bwd");
  return pack({grad[0], grad[1], grad[2]});
}
