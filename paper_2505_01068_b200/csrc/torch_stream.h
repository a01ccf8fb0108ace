// Marshalling of the calls of gsit_stream.h; a part of torch_ext.cpp, whose helpers it uses.  A cache comes as its tensors, in the order of
// streaming.StreamCache: tables, lengths, free, n_free, times, keys, values, key_scale, value_scale, open_keys, open_values.

const at::Tensor& whole(PyObject* o, at::ScalarType t, const char* what) {
  const at::Tensor& x = tensor(o);
  require(x.scalar_type() == t && x.is_contiguous(), what);
  return x;
}
// The first four: tables and the list of pages.
gsit_cache tables_of(PyObject* const* a) {
  const at::Tensor& tables = whole(a[0], at::kInt, "tables: contiguous int32 [B, 3, blocks]");
  const at::Tensor& lengths = whole(a[1], at::kInt, "lengths: contiguous int32 [B, 3]");
  const at::Tensor& list = whole(a[2], at::kInt, "free: contiguous int32 [pages]");
  const at::Tensor& n_free = whole(a[3], at::kInt, "n_free: contiguous int32 [1]");
  here({&tables, &lengths, &list, &n_free});
  require(tables.dim() == 3 && tables.size(1) == 3 && lengths.dim() == 2 && lengths.size(0) == tables.size(0) && lengths.size(1) == 3,
          "tables: [B, 3, blocks], lengths: [B, 3]");
  require(list.dim() == 1 && list.numel() <= 0x7fffffff && tables.size(2) <= 0x7fffffff && n_free.numel() == 1, "free: [pages], n_free: [1]");
  gsit_cache c = {};
  c.batch = (int32_t)tables.size(0);
  c.blocks = (int32_t)tables.size(2);
  c.pages = (int32_t)list.numel();
  c.tables = static_cast<int32_t*>(tables.data_ptr());
  c.lengths = static_cast<int32_t*>(lengths.data_ptr());
  c.free_list = static_cast<int32_t*>(list.data_ptr());
  c.n_free = static_cast<int32_t*>(n_free.data_ptr());
  return c;
}
gsit_cache cache_of(PyObject* const* a) {
  gsit_cache c = tables_of(a);
  const at::Tensor* times = opt_tensor(a[4]);
  const at::Tensor &keys = tensor(a[5]), &values = tensor(a[6]), &ok = tensor(a[9]), &ov = tensor(a[10]);
  const at::Tensor& ks = whole(a[7], at::kFloat, "scales: contiguous float32 [pages, kv_heads]");
  const at::Tensor& vs = whole(a[8], at::kFloat, "scales: contiguous float32 [pages, kv_heads]");
  here({times, &keys, &values, &ks, &vs, &ok, &ov});
  require(ok.dim() == 6 && ok.size(0) == c.batch && ok.size(1) == 3 && ok.size(2) == 2 && ok.size(4) == GSIT_CACHE_BLOCK && ok.sizes() == ov.sizes() &&
              ok.scalar_type() == ov.scalar_type() && ok.is_contiguous() && ov.is_contiguous(), "open rows: contiguous [B, 3, 2, kv_heads, 32, hd]");
  const int64_t hk = ok.size(3), hd = ok.size(5);
  require(keys.scalar_type() == at::kChar || keys.scalar_type() == at::kFloat8_e4m3fn, "keys: int8 or float8_e4m3fn");
  require(keys.scalar_type() == values.scalar_type() && keys.is_contiguous() && values.is_contiguous() && keys.sizes() == values.sizes() && keys.dim() == 3 &&
              keys.size(0) == c.pages && keys.size(1) == hk && keys.size(2) == GSIT_CACHE_BLOCK * hd, "keys, values: contiguous [pages, kv_heads, 32 * hd]");
  require(ks.dim() == 2 && ks.size(0) == c.pages && ks.size(1) == hk && ks.sizes() == vs.sizes(), "scales: contiguous float32 [pages, kv_heads]");
  require(times == nullptr || (times->scalar_type() == at::kFloat && times->is_contiguous() && times->dim() == 2 && times->size(0) == c.pages &&
                               times->size(1) == GSIT_CACHE_BLOCK), "times: contiguous float32 [pages, 32]");
  c.kind = keys.scalar_type() == at::kChar ? GSIT_CACHE_INT8 : GSIT_CACHE_E4M3;
  c.dtype = dtype_code(ok);
  c.kv_heads = (int32_t)hk;
  c.head_dim = (int32_t)hd;
  c.keys = keys.data_ptr();
  c.values = values.data_ptr();
  c.key_scale = static_cast<float*>(ks.data_ptr());
  c.value_scale = static_cast<float*>(vs.data_ptr());
  c.times = times == nullptr ? nullptr : static_cast<float*>(times->data_ptr());
  c.open_keys = ok.data_ptr();
  c.open_values = ov.data_ptr();
  return c;
}
const int32_t* int_vector(const at::Tensor* t, int64_t n, const char* what) {
  require(t == nullptr || (t->scalar_type() == at::kInt && t->is_contiguous() && t->numel() == n), what);
  return static_cast<const int32_t*>(ptr(t));
}
// Moments [B, L] of a step's rows, any strides.
struct RowMoments {
  const float* p;
  int64_t batch, row;
};
RowMoments moments(const at::Tensor* t, int64_t B, int64_t L) {
  if (t == nullptr) return {nullptr, 0, 0};
  require(t->scalar_type() == at::kFloat && t->dim() == 2 && t->size(0) == B && t->size(1) == L, "times: float32 [B, L] on the device");
  return {static_cast<const float*>(t->data_ptr()), t->stride(0), t->stride(1)};
}
// Shape of a step's rows.
gsit_shape step_shape(const gsit_cache& c, PyObject* seg, const at::Tensor* valid) {
  return make_shape(c.batch, seg, 1, 1, valid, GSIT_F32, GSIT_PHASE_INTRA, 0, 0.0);
}
int64_t rows_of(const gsit_shape& s) { return (int64_t)s.seg_len[0] + s.seg_len[1] + s.seg_len[2]; }

at::Tensor slots_for(const at::Tensor* given, const gsit_cache& c, int64_t L, const at::Device& dev) {
  if (given == nullptr) return empty({c.batch, L}, at::kInt, dev);
  require(given->scalar_type() == at::kInt && given->is_contiguous() && given->dim() == 2 && given->size(0) == c.batch && given->size(1) == L, "slots: contiguous int32 [B, L]");
  return *given;
}
const int32_t* ended_of(const at::Tensor* t, const gsit_cache& c) { return int_vector(t, c.batch, "ended: contiguous int32 [B]"); }
const int32_t* held_of(const at::Tensor* t, const gsit_cache& c) { return int_vector(t, 3 * (int64_t)c.batch, "held: contiguous int32 [B, 3]"); }

// tables, lengths, free, n_free, seg_len, valid_len, ended, held, slots
PyObject* cache_plan(PyObject* const* a) {
  const gsit_cache c = tables_of(a);
  const at::Tensor *valid = opt_tensor(a[5]), *ended = opt_tensor(a[6]), *held = opt_tensor(a[7]), *slots = opt_tensor(a[8]);
  here({valid, ended, held, slots});
  const gsit_shape s = step_shape(c, a[4], valid);
  for (int n : s.seg_len) require(n >= 0, "seg_len: no length is negative");
  const int32_t *e = ended_of(ended, c), *h = held_of(held, c);
  at::Tensor made = slots_for(slots, c, rows_of(s), tensor(a[0]).device());
  gsit_status st;
  {
    NoGil n;
    st = gsit_cache_plan(&s, &c, h, e, static_cast<int32_t*>(made.data_ptr()), stream());
  }
  check(st, "gsit_cache_plan");
  return THPVariable_Wrap(std::move(made));
}

// Row strides of a step's keys and values.
struct NewRows {
  int64_t ldk, ldv;
};
NewRows new_rows(const at::Tensor& k, const at::Tensor& v, const gsit_cache& c, int64_t L) {
  require(k.dim() == 4 && k.sizes() == v.sizes() && k.size(0) == c.batch && k.size(1) == L && k.size(2) == c.kv_heads && k.size(3) == c.head_dim &&
              dtype_code(k) == c.dtype && v.scalar_type() == k.scalar_type(), "k, v: [B, L, kv_heads, hd] of the cache's type");
  return {head_rows(k, HEAD_ROWS), head_rows(v, HEAD_ROWS)};
}

// the cache (11), k, v, slots, seg_len, times
PyObject* cache_append(PyObject* const* a) {
  const gsit_cache c = cache_of(a);
  const at::Tensor &k = tensor(a[11]), &v = tensor(a[12]), &slots = tensor(a[13]);
  const at::Tensor *times = opt_tensor(a[15]);
  here({&k, &v, &slots, times});
  const gsit_shape s = step_shape(c, a[14], nullptr);
  const int64_t L = rows_of(s);
  const NewRows ld = new_rows(k, v, c, L);
  const int32_t* sl = int_vector(&slots, c.batch * L, "slots: contiguous int32 [B, L]");
  const RowMoments tm = moments(times, c.batch, L);
  gsit_status st;
  {
    NoGil n;
    st = gsit_cache_append(&s, &c, k.data_ptr(), ld.ldk, v.data_ptr(), ld.ldv, sl, tm.p, tm.batch, tm.row, stream());
  }
  check(st, "gsit_cache_append");
  Py_RETURN_NONE;
}

// the cache (11), seg_len, out_k, out_v
PyObject* cache_read(PyObject* const* a) {
  const gsit_cache c = cache_of(a);
  const at::Tensor *out_k = opt_tensor(a[12]), *out_v = opt_tensor(a[13]);
  here({out_k, out_v});
  const gsit_shape s = step_shape(c, a[11], nullptr);
  for (int n : s.seg_len) require(n >= 0, "seg_len: no length is negative");
  const int64_t L = rows_of(s);
  const at::Tensor& like = tensor(a[9]);
  at::Tensor mk, mv;
  auto result = [&](const at::Tensor* given, at::Tensor& made) {
    if (given == nullptr) made = empty({c.batch, L, c.kv_heads, c.head_dim}, like.scalar_type(), like.device());
    else made = *given;
    require(made.dim() == 4 && made.size(0) == c.batch && made.size(1) == L && made.size(2) == c.kv_heads && made.size(3) == c.head_dim &&
                made.scalar_type() == like.scalar_type(), "results: [B, L, kv_heads, hd] of the cache's type");
    return head_rows(made, HEAD_ROWS);
  };
  const int64_t ldk = result(out_k, mk), ldv = result(out_v, mv);
  gsit_status st;
  {
    NoGil n;
    st = gsit_cache_read(&s, &c, mk.data_ptr(), ldk, mv.data_ptr(), ldv, stream());
  }
  check(st, "gsit_cache_read");
  return pack({mk, mv});
}

// Queries, rule, result and workspace of an attention call.
struct AttentionCall {
  gsit_shape s;
  gsit_score_rule r;
  RowMoments times;
  int64_t ldq;
  at::Tensor out, made_ws;
  void* ws;
  size_t ws_bytes;
};
AttentionCall attention_call(const gsit_cache& c, const at::Tensor& q, PyObject* seg, const at::Tensor* valid, PyObject* phase, PyObject* mask, PyObject* scale, PyObject* softcap,
                             const at::Tensor* slopes, const at::Tensor* times, PyObject* causal, const at::Tensor* out, const at::Tensor* ws) {
  AttentionCall x = {};
  x.ldq = head_rows(q, HEAD_ROWS);
  const int64_t B = q.size(0), L = q.size(1), H = q.size(2), hd = q.size(3);
  require(B == c.batch && hd == c.head_dim && dtype_code(q) == c.dtype, "q: [B, L, H, hd] of the cache's batch, head width and type");
  x.s = make_shape(B, seg, H * hd, H, valid, c.dtype, as_int(phase), as_int(mask), as_float(scale));
  require_length(x.s, L);
  x.r.softcap = (float)as_float(softcap);
  x.r.slopes = float_vector(slopes, H, "slopes: contiguous float32 [heads] on the device");
  x.times = moments(times, B, L);
  x.r.causal = as_bool(causal);
  if (out == nullptr) x.out = empty({B, L, H * hd}, q.scalar_type(), q.device());
  else x.out = *out;
  require(x.out.is_contiguous() && x.out.scalar_type() == q.scalar_type() && x.out.numel() == B * L * H * hd, "out: contiguous [B, L, d] of q's dtype");
  if (ws == nullptr) {
    const size_t need = gsit_cached_attention_workspace(&x.s, &x.r, &c);
    if (need != (size_t)-1 && need > 0) {
      x.made_ws = empty({(int64_t)need}, at::kByte, q.device());
      ws = &x.made_ws;
    }
  }
  x.ws = ptr(ws);
  x.ws_bytes = ws == nullptr ? 0 : (size_t)ws->nbytes();
  return x;
}

// the cache (11), q, seg_len, valid_len, phase, custom_mask, scale, softcap, slopes, times, causal, want_lse, out, workspace
PyObject* cached_attention(PyObject* const* a) {
  const gsit_cache c = cache_of(a);
  const at::Tensor& q = tensor(a[11]);
  const at::Tensor *valid = opt_tensor(a[13]), *slopes = opt_tensor(a[18]), *times = opt_tensor(a[19]), *out = opt_tensor(a[22]), *ws = scratch(a[23]);
  here({&q, valid, slopes, times, out, ws});
  AttentionCall x = attention_call(c, q, a[12], valid, a[14], a[15], a[16], a[17], slopes, times, a[20], out, ws);
  const bool want_lse = as_bool(a[21]);
  at::Tensor lse;
  if (want_lse) lse = empty({q.size(0), q.size(2), q.size(1)}, at::kFloat, q.device());
  gsit_status st;
  {
    NoGil n;
    st = gsit_im_cached_attention_fwd(&x.s, &x.r, &c, q.data_ptr(), x.ldq, x.times.p, x.times.batch, x.times.row, x.out.data_ptr(),
                                      want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr, x.ws, x.ws_bytes, stream());
  }
  check(st, "gsit_im_cached_attention_fwd");
  if (!want_lse) return THPVariable_Wrap(std::move(x.out));
  return pack({x.out, lse});
}

// the cache (11), q, k, v, seg_len, valid_len, ended, held, phase, custom_mask, scale, softcap, slopes, times, causal, slots, out, workspace
PyObject* cache_step(PyObject* const* a) {
  const gsit_cache c = cache_of(a);
  const at::Tensor &q = tensor(a[11]), &k = tensor(a[12]), &v = tensor(a[13]);
  const at::Tensor *valid = opt_tensor(a[15]), *ended = opt_tensor(a[16]), *held = opt_tensor(a[17]), *slopes = opt_tensor(a[22]), *times = opt_tensor(a[23]),
                   *slots = opt_tensor(a[25]), *out = opt_tensor(a[26]), *ws = scratch(a[27]);
  here({&q, &k, &v, valid, ended, held, slopes, times, slots, out, ws});
  AttentionCall x = attention_call(c, q, a[14], valid, a[18], a[19], a[20], a[21], slopes, times, a[24], out, ws);
  const NewRows ld = new_rows(k, v, c, q.size(1));
  const int32_t *e = ended_of(ended, c), *h = held_of(held, c);
  at::Tensor made = slots_for(slots, c, q.size(1), q.device());
  gsit_status st;
  {
    NoGil n;
    st = gsit_cache_step(&x.s, &x.r, &c, h, e, static_cast<int32_t*>(made.data_ptr()), q.data_ptr(), x.ldq, k.data_ptr(), ld.ldk, v.data_ptr(), ld.ldv, x.times.p, x.times.batch,
                         x.times.row, x.out.data_ptr(), nullptr, x.ws, x.ws_bytes, stream());
  }
  check(st, "gsit_cache_step");
  return pack({x.out, made});
}
