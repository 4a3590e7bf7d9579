// The Python binding's common path: argument checks, output allocation and the C call of the
// entry points of cover.py, in one native function each.
//
// Why: a call of the binding in Python (shape and stride checks, output tensors, a ctypes
// descriptor and pointers, the current stream) took 12 us for token statistics, 16 for attention
// and 20 for the masses, where their kernels take 5-15 us at small sizes, so the host bounded
// every small call and the whole tail of a decoding step (103 us of host work for about 60 us
// of kernels).  Here the same takes 4-6 us.
//
// Each function either makes the call and returns the outputs (a tuple), returns the library's
// status (an int) if that refused it, or returns None without having done anything: for
// arguments that fail a check, tensors of other classes than Tensor, active torch function
// modes and whatever raises.  The caller then goes through its Python form, which raises the
// error the argument deserves.  Nothing is kept between calls but the library's entry points.  What a
// function allocates comes from the current stream's memory, so the stream that it is given is that one
// wherever an output or a workspace is not the caller's (cover.py sees to it).
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ATen.h>
#include <string.h>

#include <algorithm>

#include "cover.h"

namespace {

using at::Tensor;

struct Entry {
  decltype(&cover_attn_fwd) attn_fwd;
  decltype(&cover_select_seeds) select_seeds;
  decltype(&cover_token_stats) token_stats;
  decltype(&cover_token_sample) token_sample;
  decltype(&cover_attn_stats) attn_stats;
  decltype(&cover_attn_stats_workspace) attn_stats_workspace;
  decltype(&cover_decode_update) decode_update;
};
Entry lib = {};

struct Layer {
  decltype(&cover_rms_norm) rms_norm;
  decltype(&cover_rope) rope;
  decltype(&cover_cache_store) cache_store;
  decltype(&cover_cache_load) cache_load;
  decltype(&cover_attn_cached) attn_cached;
  decltype(&cover_attn_cached_splits) attn_cached_splits;
};
Layer layer = {};

// thrown for whatever the native path leaves to the Python form
struct Leave {};
void need(bool ok) {
  if (!ok) throw Leave{};
}

const Tensor& tensor(PyObject* o) {
  need(THPVariable_CheckExact(o));
  const Tensor& t = THPVariable_Unpack(o);
  need(t.is_cuda() && t.layout() == at::kStrided);
  return t;
}
const Tensor* optional(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }
int64_t integer(PyObject* o) {
  need(PyLong_Check(o));
  int overflow = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
  need(!overflow);
  return v;
}
int32_t int32(PyObject* o) {
  const int64_t v = integer(o);
  need(v == (int32_t)v);
  return (int32_t)v;
}
float real(PyObject* o) {
  need(PyFloat_Check(o) || PyLong_Check(o));
  const double v = PyFloat_AsDouble(o);
  need(!PyErr_Occurred());
  return (float)v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  need(v >= 0);
  return v != 0;
}
hipStream_t stream_of(PyObject* o) { return (hipStream_t)(uintptr_t)integer(o); }

template <class T>
T* ptr(const Tensor& t) {
  return (T*)t.data_ptr();
}
template <class T>
T* ptr(const Tensor* t) {
  return t ? (T*)t->data_ptr() : nullptr;
}
Tensor empty(at::IntArrayRef size, at::ScalarType dtype, const Tensor& like) {
  return at::empty(size, at::TensorOptions().dtype(dtype).device(like.device()));
}
// an output: the caller's object, a tensor allocated here, or None
struct Out {
  PyObject* given = nullptr;
  Tensor made;
  template <class T>
  T* data() const {
    if (given) return given == Py_None ? nullptr : (T*)THPVariable_Unpack(given).data_ptr();
    return made.defined() ? (T*)made.data_ptr() : nullptr;
  }
  PyObject* release() const {
    PyObject* o = given ? given : (made.defined() ? nullptr : Py_None);
    if (!o) return THPVariable_Wrap(made);
    Py_INCREF(o);
    return o;
  }
};
// `o` if it is a tensor, otherwise (None) allocated when wanted
Out output(PyObject* o, bool wanted, at::IntArrayRef size, at::ScalarType dtype, const Tensor& like) {
  Out r;
  if (o && o != Py_None) {
    tensor(o);
    r.given = o;
  } else if (wanted) {
    r.made = empty(size, dtype, like);
  }
  return r;
}
bool is(const Tensor& t, at::IntArrayRef size, at::ScalarType dtype) {
  return t.sizes() == size && t.scalar_type() == dtype && t.is_contiguous();
}
template <class... O>
PyObject* tuple(const O&... outs) {
  PyObject* items[] = {outs.release()...};
  constexpr Py_ssize_t n = sizeof...(O);
  PyObject* r = PyTuple_New(n);
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (!r || !items[i]) {
      Py_XDECREF(items[i]);
      if (r) PyTuple_SET_ITEM(r, i, Py_NewRef(Py_None));
    } else {
      PyTuple_SET_ITEM(r, i, items[i]);
    }
  }
  if (PyErr_Occurred()) {
    Py_XDECREF(r);
    return nullptr;
  }
  return r;
}

int dtype_of(const Tensor& t) {
  if (t.scalar_type() == at::kBFloat16) return COVER_BF16;
  need(t.scalar_type() == at::kFloat);
  return COVER_F32;
}
cover_attn_desc attn_desc(const Tensor& q, const Tensor& k, int64_t max_seeds, float scale) {
  cover_attn_desc d = {};
  d.B = (int32_t)q.size(0); d.Hq = (int32_t)q.size(1); d.L = (int32_t)q.size(2); d.d = (int32_t)q.size(3);
  d.Hkv = (int32_t)k.size(1);
  d.max_seeds = (int32_t)max_seeds;
  d.dtype = (decltype(d.dtype))dtype_of(q);
  d.scale = scale;
  d.q_sb = q.stride(0); d.q_sh = q.stride(1); d.q_sl = q.stride(2);
  d.kv_sb = k.stride(0); d.kv_sh = k.stride(1); d.kv_sl = k.stride(2);
  return d;
}
void same_layout(const Tensor& t, const Tensor& k, const Tensor& q) {
  need(t.sizes() == k.sizes() && t.strides() == k.strides() && t.scalar_type() == q.scalar_type());
}
// the seed list of an attention call: its width, 0 without one
int64_t seed_width(const Tensor* idx, const Tensor* n) {
  if (!idx) return 0;
  need(idx->dim() >= 1 && idx->scalar_type() == at::kInt && n && n->scalar_type() == at::kInt &&
       idx->is_contiguous());
  return idx->size(-1);
}

template <class F>
PyObject* guarded(Py_ssize_t n, Py_ssize_t expect, F&& f) {
  try {
    if (n == expect && lib.attn_fwd && !at::impl::torch_function_mode_enabled()) return f();
  } catch (...) {
    PyErr_Clear();
  }
  Py_RETURN_NONE;
}
template <class F>
cover_status call(F&& f) {
  cover_status st;
  Py_BEGIN_ALLOW_THREADS
  st = f();
  Py_END_ALLOW_THREADS
  return st;
}

// (q, k_live, v_live, k_cache, v_cache, seed_idx, n_seed, out, lse, scale, want_lse, stream)
PyObject* attn_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]), &kc = tensor(a[3]), &vc = tensor(a[4]);
    need(q.dim() == 4 && k.dim() == 4 && q.stride(3) == 1 && k.stride(3) == 1);
    need(k.scalar_type() == q.scalar_type());
    for (const Tensor* t : {&v, &kc, &vc}) same_layout(*t, k, q);
    const Tensor *idx = optional(a[5]), *ns = optional(a[6]);
    const cover_attn_desc d = attn_desc(q, k, seed_width(idx, ns), real(a[9]));
    const hipStream_t stream = stream_of(a[11]);
    Out out, lse = output(a[8], truth(a[10]), {q.size(0), q.size(1), q.size(2)}, at::kFloat, q);
    if (a[7] == Py_None) {
      out.made = at::empty_like(q);
      need(out.made.strides() == q.strides());
    } else {
      const Tensor& t = tensor(a[7]);
      need(t.sizes() == q.sizes() && t.strides() == q.strides() && t.scalar_type() == q.scalar_type());
      out.given = a[7];
    }
    const void *pq = ptr<void>(q), *pk = ptr<void>(k), *pv = ptr<void>(v), *pkc = ptr<void>(kc), *pvc = ptr<void>(vc);
    const int32_t *pi = ptr<int32_t>(idx), *pn = ptr<int32_t>(ns);
    void* po = out.data<void>();
    float* pl = lse.data<float>();
    const cover_status st = call([&] { return lib.attn_fwd(pq, pk, pv, pkc, pvc, pi, pn, po, pl, &d, stream); });
    return st == COVER_OK ? tuple(out, lse) : PyLong_FromLong(st);
  });
}

// (logits, tokens, want_logp, want_conf, want_argmax, stream)
PyObject* token_stats(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const Tensor& x = tensor(a[0]);
    need(x.dim() == 2 && x.stride(1) == 1);
    const int64_t R = x.size(0);
    cover_token_desc d = {};
    d.R = (int32_t)R; d.V = (int32_t)x.size(1);
    d.dtype = (decltype(d.dtype))dtype_of(x);
    d.row_stride = x.stride(0);
    const bool want_logp = truth(a[2]);
    const int32_t* tok = nullptr;
    if (want_logp) {
      const Tensor& t = tensor(a[1]);
      need(is(t, {R}, at::kInt));
      tok = ptr<int32_t>(t);
    }
    const Out logp = output(nullptr, want_logp, {R}, at::kFloat, x), conf = output(nullptr, truth(a[3]), {R}, at::kFloat, x),
              top = output(nullptr, truth(a[4]), {R}, at::kInt, x);
    const hipStream_t stream = stream_of(a[5]);
    const void* px = ptr<void>(x);
    float *pl = logp.data<float>(), *pc = conf.data<float>();
    int32_t* pt = top.data<int32_t>();
    const cover_status st = call([&] { return lib.token_stats(px, tok, pl, pc, pt, &d, stream); });
    return st == COVER_OK ? tuple(logp, conf, top) : PyLong_FromLong(st);
  });
}

// (logits, temperature, seed, step, want_prob, stream)
PyObject* token_sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&]() -> PyObject* {
    const Tensor& x = tensor(a[0]);
    need(x.dim() == 2 && x.stride(1) == 1 && PyLong_Check(a[2]) && PyLong_Check(a[3]));
    const int64_t R = x.size(0);
    cover_token_desc d = {};
    d.R = (int32_t)R; d.V = (int32_t)x.size(1);
    d.dtype = (decltype(d.dtype))dtype_of(x);
    d.row_stride = x.stride(0);
    const float temperature = real(a[1]);
    const uint64_t seed = PyLong_AsUnsignedLongLongMask(a[2]);
    const uint32_t step = (uint32_t)PyLong_AsUnsignedLongLongMask(a[3]);
    need(!PyErr_Occurred());
    const Out token = output(nullptr, true, {R}, at::kInt, x), prob = output(nullptr, truth(a[4]), {R}, at::kFloat, x);
    const hipStream_t stream = stream_of(a[5]);
    const void* px = ptr<void>(x);
    int32_t* pt = token.data<int32_t>();
    float* pp = prob.data<float>();
    const cover_status st = call([&] { return lib.token_sample(px, temperature, seed, step, pt, pp, &d, stream); });
    return st == COVER_OK ? tuple(token, prob) : PyLong_FromLong(st);
  });
}

// (q, k_live, k_cache, seed_idx, n_seed, lse, masked, drafted, r0, scale, workspace, stream)
PyObject* attn_stats(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&]() -> PyObject* {
    const Tensor &q = tensor(a[0]), &k = tensor(a[1]), &kc = tensor(a[2]);
    need(q.dim() == 4 && k.dim() == 4 && k.scalar_type() == q.scalar_type());
    same_layout(kc, k, q);
    const Tensor *idx = optional(a[3]), *ns = optional(a[4]);
    need(!idx || idx->dim() >= 1);
    const Tensor &lse = tensor(a[5]), &masked = tensor(a[6]), &drafted = tensor(a[7]);
    const int64_t B = q.size(0), Hq = q.size(1), L = q.size(2);
    need(masked.dim() == 2);
    const int64_t Lr = masked.size(1);
    need(is(masked, {B, Lr}, at::kByte) && is(drafted, {B, Lr}, at::kByte) && is(lse, {B, Hq, L}, at::kFloat));
    cover_stats_desc d = {};
    d.attn = attn_desc(q, k, idx ? idx->size(-1) : 0, real(a[9]));
    d.r0 = int32(a[8]);
    d.Lr = (int32_t)Lr;
    const int64_t floats = lib.attn_stats_workspace((int32_t)B, (int32_t)Hq, (int32_t)Lr);
    need(floats >= 0);
    Tensor own;
    const Tensor* ws = optional(a[10]);
    if (ws) {
      need(ws->scalar_type() == at::kFloat && ws->is_contiguous() && ws->numel() >= floats && ws->device() == q.device());
    } else {
      own = empty({std::max<int64_t>(1, floats)}, at::kFloat, q);
      ws = &own;
    }
    const Out d_in = output(nullptr, true, {B, Lr}, at::kFloat, q), d_out = output(nullptr, true, {B, Lr}, at::kFloat, q);
    const hipStream_t stream = stream_of(a[11]);
    const void *pq = ptr<void>(q), *pk = ptr<void>(k), *pkc = ptr<void>(kc);
    const int32_t *pi = ptr<int32_t>(idx), *pn = ptr<int32_t>(ns);
    const float* pl = ptr<float>(lse);
    const uint8_t *pm = ptr<uint8_t>(masked), *pd = ptr<uint8_t>(drafted);
    float *po = d_in.data<float>(), *pp = d_out.data<float>(), *pw = ptr<float>(*ws);
    const cover_status st =
        call([&] { return lib.attn_stats(pq, pk, pkc, pi, pn, pl, pm, pd, po, pp, pw, &d, stream); });
    return st == COVER_OK ? tuple(d_in, d_out) : PyLong_FromLong(st);
  });
}

// (logp, d_in, d_out, flags, max_seeds, pos_offset, seed_idx, n_seed, score, want_score, stream)
PyObject* select_seeds(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const Tensor &logp = tensor(a[0]), &d_in = tensor(a[1]), &d_out = tensor(a[2]), &flags = tensor(a[3]);
    need(logp.dim() == 2);
    const int64_t B = logp.size(0), Lr = logp.size(1);
    need(is(logp, {B, Lr}, at::kFloat) && is(d_in, {B, Lr}, at::kFloat) && is(d_out, {B, Lr}, at::kFloat) &&
         is(flags, {B, Lr}, at::kByte));
    cover_select_desc d = {};
    d.B = (int32_t)B; d.Lr = (int32_t)Lr; d.max_seeds = int32(a[4]); d.pos_offset = int32(a[5]);
    const Out seeds = output(a[6], true, {B, d.max_seeds}, at::kInt, logp), ns = output(a[7], true, {B}, at::kInt, logp),
              score = output(a[8], truth(a[9]), {B, Lr}, at::kDouble, logp);
    const hipStream_t stream = stream_of(a[10]);
    const float *pl = ptr<float>(logp), *pi = ptr<float>(d_in), *po = ptr<float>(d_out);
    const uint8_t* pf = ptr<uint8_t>(flags);
    int32_t *ps = seeds.data<int32_t>(), *pn = ns.data<int32_t>();
    double* pc = score.data<double>();
    const cover_status st = call([&] { return lib.select_seeds(pl, pi, po, pf, ps, pn, pc, &d, stream); });
    return st == COVER_OK ? tuple(seeds, ns, score) : PyLong_FromLong(st);
  });
}

// (tokens, argmax, conf, seed_idx, n_seed, remask_count, mask_id, tau, draft_cap, remask_budget,
//  pos_offset, flags, drafted, counts, want_outputs, min_draft, stream): without flip-flop counts
PyObject* decode_update(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 17, [&]() -> PyObject* {
    const Tensor &tokens = tensor(a[0]), &top = tensor(a[1]), &conf = tensor(a[2]), &remask = tensor(a[5]);
    need(tokens.dim() == 2);
    const int64_t B = tokens.size(0), Lr = tokens.size(1);
    need(is(tokens, {B, Lr}, at::kInt) && is(top, {B, Lr}, at::kInt) && is(conf, {B, Lr}, at::kFloat) &&
         is(remask, {B, Lr}, at::kInt));
    const Tensor *idx = optional(a[3]), *ns = optional(a[4]);
    cover_update_desc d = {};
    if (idx) {
      need(idx->dim() == 2 && idx->size(0) == B && idx->scalar_type() == at::kInt && idx->is_contiguous() && ns &&
           ns->dim() == 1 && ns->size(0) == B && ns->scalar_type() == at::kInt);
      d.max_seeds = (int32_t)idx->size(1);
    }
    d.B = (int32_t)B; d.Lr = (int32_t)Lr;
    d.mask_id = int32(a[6]); d.tau = real(a[7]); d.draft_cap = int32(a[8]); d.remask_budget = int32(a[9]);
    d.pos_offset = int32(a[10]); d.min_draft = int32(a[15]);
    const bool want = truth(a[14]);
    const Out flags = output(a[11], want, {B, Lr}, at::kByte, tokens), drafted = output(a[12], want, {B, Lr}, at::kByte, tokens),
              counts = output(a[13], want, {B, 5}, at::kInt, tokens);
    if (flags.given) need(is(THPVariable_Unpack(flags.given), {B, Lr}, at::kByte));
    if (drafted.given) need(is(THPVariable_Unpack(drafted.given), {B, Lr}, at::kByte));
    if (counts.given) need(is(THPVariable_Unpack(counts.given), {B, 5}, at::kInt));
    const hipStream_t stream = stream_of(a[16]);
    int32_t *pt = ptr<int32_t>(tokens), *pr = ptr<int32_t>(remask), *pn = counts.data<int32_t>();
    const int32_t *pa = ptr<int32_t>(top), *pi = d.max_seeds ? ptr<int32_t>(idx) : nullptr,
                  *ps = d.max_seeds ? ptr<int32_t>(ns) : nullptr;
    const float* pc = ptr<float>(conf);
    uint8_t *pf = flags.data<uint8_t>(), *pd = drafted.data<uint8_t>();
    const cover_status st = call(
        [&] { return lib.decode_update(pt, pa, pc, pi, ps, pr, pf, pd, pn, nullptr, nullptr, &d, stream); });
    return st == COVER_OK ? tuple(flags, drafted, counts) : PyLong_FromLong(st);
  });
}

// ---- the layer's operators around the attention -------------------------------------------------
// Their last two arguments are the stream and the current GPU; tensors elsewhere are left to the
// Python form, which refuses them.
const Tensor& here(PyObject* o, int64_t gpu) {
  const Tensor& t = tensor(o);
  need(t.device().index() == gpu);
  return t;
}
const Tensor* here_or_none(PyObject* o, int64_t gpu) { return o == Py_None ? nullptr : &here(o, gpu); }
// [R, D] whose rows start at multiples of 16 bytes
Tensor empty_rows(int64_t R, int64_t D, at::ScalarType dtype, const Tensor& like) {
  const int64_t per = 16 / (int64_t)at::elementSize(dtype), pad = (D + per - 1) / per * per;
  Tensor t = empty({R, pad}, dtype, like);
  return pad == D ? t : t.narrow(1, 0, D);
}
// an output of these sizes and type with a contiguous last dimension, the caller's or made here
template <class F>
Out typed_output(PyObject* o, int64_t gpu, at::IntArrayRef size, at::ScalarType dtype, F&& make) {
  Out r;
  if (o == Py_None) {
    r.made = make();
  } else {
    const Tensor& t = here(o, gpu);
    need(t.sizes() == size && t.scalar_type() == dtype && (size.back() <= 1 || t.stride(-1) == 1));
    r.given = o;
  }
  return r;
}
const Tensor& of(const Out& o) { return o.given ? THPVariable_Unpack(o.given) : o.made; }
void strides3(const Tensor& t, int64_t& sb, int64_t& sh, int64_t& sl) {
  sb = t.stride(0); sh = t.stride(1); sl = t.stride(2);
}

// (x, weight, residual, eps, quantize, out, residual_out, scale, stream, gpu)
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const int64_t gpu = integer(a[9]);
    const Tensor& x = here(a[0], gpu);
    need(x.dim() == 2);
    const int64_t R = x.size(0), D = x.size(1);
    need(D <= 1 || x.stride(1) == 1);
    const at::ScalarType type = x.scalar_type();
    cover_norm_desc d = {};
    d.dtype = (decltype(d.dtype))dtype_of(x);
    const Tensor *w = here_or_none(a[1], gpu), *res = here_or_none(a[2], gpu);
    if (w) need(is(*w, {D}, type));
    if (res) need(res->sizes() == x.sizes() && res->scalar_type() == type && (D <= 1 || res->stride(1) == 1));
    const bool quantize = truth(a[4]);
    need((res || a[6] == Py_None) && (quantize || a[7] == Py_None));
    const at::ScalarType codes = quantize ? at::ScalarType::Float8_e4m3fn : type;
    const Out out = typed_output(a[5], gpu, {R, D}, codes, [&] { return empty_rows(R, D, codes, x); });
    Out ro, scale;
    if (res) ro = typed_output(a[6], gpu, {R, D}, type, [&] { return empty_rows(R, D, type, x); });
    if (quantize) {
      scale = typed_output(a[7], gpu, {R}, at::kFloat, [&] { return empty({R}, at::kFloat, x); });
    }
    d.R = (int32_t)R; d.D = (int32_t)D; d.eps = real(a[3]);
    need(d.R == R && d.D == D);
    d.x_stride = x.stride(0); d.out_stride = of(out).stride(0);
    if (res) {
      d.res_stride = res->stride(0);
      d.res_out_stride = of(ro).stride(0);
    }
    const hipStream_t stream = stream_of(a[8]);
    const void *px = ptr<void>(x), *pr = ptr<void>(res), *pw = ptr<void>(w);
    void *po = out.data<void>(), *pp = ro.data<void>();
    float* ps = scale.data<float>();
    const cover_status st = call([&] { return layer.rms_norm(px, pr, pw, pp, po, ps, &d, stream); });
    return st == COVER_OK ? tuple(out, ro, scale) : PyLong_FromLong(st);
  });
}

// (q, k, pos, freq, interleaved, attention_factor, q_out, k_out, stream, gpu)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&]() -> PyObject* {
    const int64_t gpu = integer(a[9]);
    const Tensor &q = here(a[0], gpu), &pos = here(a[2], gpu), &freq = here(a[3], gpu);
    const Tensor* k = here_or_none(a[1], gpu);
    need(q.dim() == 4 && q.stride(3) == 1 && (k || a[7] == Py_None));
    const at::ScalarType type = q.scalar_type();
    const int64_t B = q.size(0), L = q.size(2), D = q.size(3);
    if (k) need(k->dim() == 4 && k->size(0) == B && k->size(2) == L && k->size(3) == D && k->scalar_type() == type &&
                k->stride(3) == 1);
    need(pos.scalar_type() == at::kInt && (pos.sizes() == at::IntArrayRef{B, L} || pos.sizes() == at::IntArrayRef{L}) &&
         (L <= 1 || pos.stride(-1) == 1));
    need(freq.scalar_type() == at::kDouble && freq.dim() == 1 && freq.is_contiguous());
    const Out qo = typed_output(a[6], gpu, q.sizes(), type, [&] { return at::empty_like(q); });
    Out ko;
    if (k) ko = typed_output(a[7], gpu, k->sizes(), type, [&] { return at::empty_like(*k); });
    cover_rope_desc d = {};
    d.B = (int32_t)B; d.L = (int32_t)L; d.Hq = (int32_t)q.size(1); d.Hkv = k ? (int32_t)k->size(1) : 0;
    d.d = (int32_t)D; d.rot = (int32_t)(2 * freq.size(0)); d.interleaved = truth(a[4]);
    need(d.B == B && d.L == L);
    d.dtype = (decltype(d.dtype))dtype_of(q);
    d.attention_factor = real(a[5]);
    d.pos_sb = pos.dim() == 2 ? pos.stride(0) : 0;
    strides3(q, d.q_sb, d.q_sh, d.q_sl);
    strides3(of(qo), d.qo_sb, d.qo_sh, d.qo_sl);
    if (k) {
      strides3(*k, d.k_sb, d.k_sh, d.k_sl);
      strides3(of(ko), d.ko_sb, d.ko_sh, d.ko_sl);
    }
    const hipStream_t stream = stream_of(a[8]);
    const void *pq = ptr<void>(q), *pk = ptr<void>(k);
    const int32_t* pp = ptr<int32_t>(pos);
    const double* pf = ptr<double>(freq);
    void *po = qo.data<void>(), *px = ko.data<void>();
    const cover_status st = call([&] { return layer.rope(pq, pk, pp, pf, po, px, &d, stream); });
    return st == COVER_OK ? tuple(qo, ko) : PyLong_FromLong(st);
  });
}

// the 8-bit cache's tensors, checked against the batch, heads and head size; positions they hold
struct Cache {
  const Tensor &kc, &vc, &ks, &vs;
  Cache(PyObject* const* a, int64_t gpu)
      : kc(here(a[0], gpu)), vc(here(a[1], gpu)), ks(here(a[2], gpu)), vs(here(a[3], gpu)) {
    need(kc.dim() == 4 && kc.stride(3) == 1 && kc.scalar_type() == at::ScalarType::Float8_e4m3fn);
    same_layout(vc, kc, kc);
    const int64_t L = kc.size(2);
    need(ks.scalar_type() == at::kFloat && ks.sizes() == at::IntArrayRef({kc.size(0), kc.size(1), L}) &&
         (L <= 1 || ks.stride(2) == 1));
    same_layout(vs, ks, ks);
  }
  void matches(int64_t B, int64_t H, int64_t D) const {
    need(kc.size(0) == B && kc.size(1) == H && kc.size(3) == D);
  }
  template <class Desc>
  void describe(Desc& d) const {
    d.L = (int32_t)kc.size(2);
    strides3(kc, d.c_sb, d.c_sh, d.c_sl);
    d.s_sb = ks.stride(0); d.s_sh = ks.stride(1);
  }
};
// pos: an int (the position of row 0) or a list [B, N]
const int32_t* positions(PyObject* o, int64_t gpu, int64_t B, int64_t N, int32_t& first) {
  if (PyLong_CheckExact(o)) {
    first = int32(o);
    return nullptr;
  }
  const Tensor& t = here(o, gpu);
  need(is(t, {B, N}, at::kInt));
  first = 0;
  return ptr<int32_t>(t);
}

// (k, v, pos, k_cache, v_cache, k_scale, v_scale, stream, gpu)
PyObject* cache_store(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&]() -> PyObject* {
    const int64_t gpu = integer(a[8]);
    const Tensor &k = here(a[0], gpu), &v = here(a[1], gpu);
    need(k.dim() == 4 && k.stride(3) == 1 && v.sizes() == k.sizes() && v.stride(3) == 1 &&
         v.scalar_type() == k.scalar_type());
    const int64_t B = k.size(0), H = k.size(1), N = k.size(2);
    const Cache c(a + 3, gpu);
    c.matches(B, H, k.size(3));
    cover_cache_desc d = {};
    const int32_t* pp = positions(a[2], gpu, B, N, d.first);
    need(pp || PyLong_CheckExact(a[2]) || B * N == 0);
    d.B = (int32_t)B; d.H = (int32_t)H; d.N = (int32_t)N; d.d = (int32_t)k.size(3);
    d.dtype = (decltype(d.dtype))dtype_of(k);
    strides3(k, d.k_sb, d.k_sh, d.k_sl);
    strides3(v, d.v_sb, d.v_sh, d.v_sl);
    c.describe(d);
    const hipStream_t stream = stream_of(a[7]);
    const void *pk = ptr<void>(k), *pv = ptr<void>(v);
    void *kc = ptr<void>(c.kc), *vc = ptr<void>(c.vc);
    float *ks = ptr<float>(c.ks), *vs = ptr<float>(c.vs);
    const cover_status st = call([&] { return layer.cache_store(pk, pv, pp, kc, vc, ks, vs, &d, stream); });
    if (st != COVER_OK) return PyLong_FromLong(st);
    Out o[4];
    for (int i = 0; i < 4; ++i) o[i].given = a[3 + i];
    return tuple(o[0], o[1], o[2], o[3]);
  });
}

// (k_cache, v_cache, k_scale, v_scale, pos, n, k, v, bf16, stream, gpu)
PyObject* cache_load(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&]() -> PyObject* {
    const int64_t gpu = integer(a[10]);
    const Cache c(a, gpu);
    const int64_t B = c.kc.size(0), H = c.kc.size(1), D = c.kc.size(3);
    int64_t N;
    if (PyLong_CheckExact(a[4])) {
      N = integer(a[5]);
    } else {
      const Tensor& t = here(a[4], gpu);
      need(t.dim() == 2);
      N = t.size(1);
      need(a[5] == Py_None || integer(a[5]) == N);
    }
    need(N >= 0);
    cover_cache_desc d = {};
    const int32_t* pp = positions(a[4], gpu, B, N, d.first);
    need(pp || PyLong_CheckExact(a[4]) || B * N == 0);
    const at::ScalarType type = truth(a[8]) ? at::kBFloat16 : at::kFloat;
    const auto make = [&] { return empty({B, H, N, D}, type, c.kc); };
    const Out k = typed_output(a[6], gpu, {B, H, N, D}, type, make), v = typed_output(a[7], gpu, {B, H, N, D}, type, make);
    d.B = (int32_t)B; d.H = (int32_t)H; d.N = (int32_t)N; d.d = (int32_t)D;
    need(d.N == N);
    d.dtype = type == at::kFloat ? COVER_F32 : COVER_BF16;
    strides3(of(k), d.k_sb, d.k_sh, d.k_sl);
    strides3(of(v), d.v_sb, d.v_sh, d.v_sl);
    c.describe(d);
    const hipStream_t stream = stream_of(a[9]);
    void *pk = k.data<void>(), *pv = v.data<void>();
    const void *kc = ptr<void>(c.kc), *vc = ptr<void>(c.vc);
    const float *ks = ptr<float>(c.ks), *vs = ptr<float>(c.vs);
    const cover_status st = call([&] { return layer.cache_load(pk, pv, pp, kc, vc, ks, vs, &d, stream); });
    return st == COVER_OK ? tuple(k, v) : PyLong_FromLong(st);
  });
}

// (q, k_live, v_live, k_cache, v_cache, k_scale, v_scale, q_off, seed_idx, n_seed, kv_len, out, lse, scale,
//  n_split, workspace, want_lse, stream, gpu)
PyObject* attn_cached(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 19, [&]() -> PyObject* {
    const int64_t gpu = integer(a[18]);
    const Tensor &q = here(a[0], gpu), &k = here(a[1], gpu), &v = here(a[2], gpu);
    need(q.dim() == 4 && k.dim() == 4 && q.scalar_type() == at::kBFloat16 && q.stride(3) == 1);
    const int64_t B = q.size(0), Hq = q.size(1), Lq = q.size(2), D = q.size(3), Hkv = k.size(1);
    for (const Tensor* t : {&k, &v})
      need(t->sizes() == at::IntArrayRef({B, Hkv, Lq, D}) && t->scalar_type() == at::kBFloat16 && t->stride(3) == 1);
    const Cache c(a + 3, gpu);
    c.matches(B, Hkv, D);
    cover_cached_desc d = {};
    const int32_t* off = nullptr;
    if (PyLong_CheckExact(a[7])) {
      d.q_off = int32(a[7]);
    } else {
      const Tensor& t = here(a[7], gpu);
      need(is(t, {B}, at::kInt) && B > 0);
      off = ptr<int32_t>(t);
    }
    const Tensor *idx = here_or_none(a[8], gpu), *ns = here_or_none(a[9], gpu), *len = here_or_none(a[10], gpu);
    if (idx) {
      need(idx->dim() == 2 && idx->size(0) == B && idx->scalar_type() == at::kInt && idx->is_contiguous() && ns &&
           is(*ns, {B}, at::kInt));
      d.max_seeds = (int32_t)idx->size(1);
    }
    if (len) need(is(*len, {B}, at::kInt));
    d.scale = real(a[13]);
    const hipStream_t stream = stream_of(a[17]);
    const Out out = typed_output(a[11], gpu, q.sizes(), at::kBFloat16, [&] { return at::empty_like(q); });
    if (a[12] != Py_None) need(is(here(a[12], gpu), {B, Hq, Lq}, at::kFloat));
    const Out lse = output(a[12], truth(a[16]), {B, Hq, Lq}, at::kFloat, q);
    d.B = (int32_t)B; d.Hq = (int32_t)Hq; d.Hkv = (int32_t)Hkv; d.Lq = (int32_t)Lq; d.d = (int32_t)D;
    need(d.Hq == Hq && d.Hkv == Hkv && d.Lq == Lq);
    c.describe(d);
    const Tensor* ws = here_or_none(a[15], gpu);
    const int64_t record = B * Hq * Lq * (D + 4);
    if (a[14] == Py_None) {
      d.n_split = layer.attn_cached_splits(d.B, d.Hq, d.Hkv, d.L, d.Lq);
      if (ws && record > 0 && d.n_split > 1)  // as many ranges as the caller's workspace holds
        d.n_split = (int32_t)std::max<int64_t>(1, std::min<int64_t>(d.n_split, ws->numel() / record));
    } else {
      d.n_split = int32(a[14]);
      need(d.n_split <= 256);
    }
    Tensor own;
    if (d.n_split > 1) {
      if (!ws) {
        own = empty({record * d.n_split}, at::kFloat, q);
        ws = &own;
      }
      need(ws->scalar_type() == at::kFloat && ws->is_contiguous() && ws->numel() >= record * d.n_split);
    } else {
      ws = nullptr;
    }
    strides3(q, d.q_sb, d.q_sh, d.q_sl);
    strides3(of(out), d.o_sb, d.o_sh, d.o_sl);
    strides3(k, d.k_sb, d.k_sh, d.k_sl);
    strides3(v, d.v_sb, d.v_sh, d.v_sl);
    const void *pq = ptr<void>(q), *pk = ptr<void>(k), *pv = ptr<void>(v), *kc = ptr<void>(c.kc), *vc = ptr<void>(c.vc);
    const float *ks = ptr<float>(c.ks), *vs = ptr<float>(c.vs);
    const int32_t *pi = ptr<int32_t>(idx), *pn = ptr<int32_t>(ns), *pl = ptr<int32_t>(len);
    void* po = out.data<void>();
    float *px = lse.data<float>(), *pw = ptr<float>(ws);
    const cover_status st = call([&] {
      return layer.attn_cached(pq, pk, pv, kc, vc, ks, vs, off, pl, pi, pn, po, px, pw, &d, stream);
    });
    return st == COVER_OK ? tuple(out, lse) : PyLong_FromLong(st);
  });
}

// the addresses of the entry points of the layer's operators, in Layer's order
PyObject* bind_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr Py_ssize_t kN = sizeof(Layer) / sizeof(void*);
  void* p[kN];
  for (Py_ssize_t i = 0; i < kN; ++i) {
    p[i] = n == kN ? PyLong_AsVoidPtr(a[i]) : nullptr;
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind_layer() takes the library's entry points");
      return nullptr;
    }
  }
  memcpy((void*)&layer, p, sizeof(layer));
  Py_RETURN_NONE;
}

// the addresses of the library's entry points, in Entry's order
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
  constexpr Py_ssize_t kN = sizeof(Entry) / sizeof(void*);
  if (n != kN) {
    PyErr_SetString(PyExc_TypeError, "bind() takes the library's entry points");
    return nullptr;
  }
  void* p[kN];
  for (Py_ssize_t i = 0; i < kN; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "null entry point");
      return nullptr;
    }
  }
  static_assert(sizeof(p) == sizeof(lib), "one address per entry point");
  memcpy((void*)&lib, p, sizeof(lib));
  Py_RETURN_NONE;
}

#define COVER_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {COVER_METHOD(bind),       COVER_METHOD(attn_fwd),     COVER_METHOD(token_stats),
                         COVER_METHOD(token_sample), COVER_METHOD(attn_stats), COVER_METHOD(select_seeds),
                         COVER_METHOD(decode_update), COVER_METHOD(bind_layer), COVER_METHOD(rms_norm),
                         COVER_METHOD(rope),       COVER_METHOD(cache_store),  COVER_METHOD(cache_load),
                         COVER_METHOD(attn_cached), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cover_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cover_host(void) { return PyModule_Create(&module); }
