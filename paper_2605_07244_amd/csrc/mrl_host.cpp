// Host side of the calls that take a few microseconds on the GPU, as a CPython extension: checks the tensors, allocates the
// outputs, calls the C ABI.  What Python needs for that is most of such a call: advantages of 128 x 8 rollouts 11.4 us
// a call through ctypes and torch.empty, now 6.6 (the kernel takes 5.7); alignment of short rows 13.3 and 9.3.
//
// A function here returns None for anything it does not take as it is (no plain torch.Tensor, another dtype, not
// contiguous, not on a GPU, any exception): the caller then goes through the Python path, whose checks and errors are
// the ones that count.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/mrl.h"

namespace {

// A tensor argument: pointer of a plain contiguous GPU tensor of the dtype; None -> nullptr if allowed.
bool tensor_arg(PyObject* o, at::ScalarType type, bool optional, void** ptr) {
  if (o == Py_None) { *ptr = nullptr; return optional; }
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous()) return false;
  *ptr = const_cast<void*>(t.const_data_ptr());
  return true;
}

bool int_arg(PyObject* o, int64_t* v) {
  if (!PyLong_CheckExact(o)) return false;
  *v = PyLong_AsLongLong(o);
  if (*v == -1 && PyErr_Occurred()) { PyErr_Clear(); return false; }
  return true;
}
bool int32_arg(PyObject* o, int32_t* v) {
  int64_t w;
  if (!int_arg(o, &w) || w < INT32_MIN || w > INT32_MAX) return false;
  *v = (int32_t)w;
  return true;
}
bool float_arg(PyObject* o, float* v) {
  if (!PyFloat_CheckExact(o)) return false;
  *v = (float)PyFloat_AS_DOUBLE(o);
  return true;
}

at::Tensor new_like(const at::Tensor& t, at::IntArrayRef sizes, at::ScalarType type) {
  return at::empty(sizes, t.options().dtype(type).requires_grad(false));
}

// (rewards, group_id, G, in_stats, scored, is_own, mode, eps_norm, ddof, mix_alpha, neg_thresh, pos_thresh, baseline_shift, stream)
// -> (status, adv, mean, std, flags) or None
PyObject* advantages(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    void *rewards, *group, *in_stats, *scored, *own, *shift;
    int32_t G, mode, ddof;
    float eps, mix, neg, pos;
    int64_t stream;
    if (n != 14 || !tensor_arg(a[0], at::kFloat, false, &rewards) || !tensor_arg(a[1], at::kInt, false, &group) || !int32_arg(a[2], &G) ||
        !tensor_arg(a[3], at::kByte, true, &in_stats) || !tensor_arg(a[4], at::kByte, true, &scored) ||
        !tensor_arg(a[5], at::kByte, true, &own) || !int32_arg(a[6], &mode) || !float_arg(a[7], &eps) || !int32_arg(a[8], &ddof) ||
        !float_arg(a[9], &mix) || !float_arg(a[10], &neg) || !float_arg(a[11], &pos) || !tensor_arg(a[12], at::kFloat, true, &shift) ||
        !int_arg(a[13], &stream) || G <= 0 || (shift != nullptr && THPVariable_Unpack(a[12]).numel() != G))
      Py_RETURN_NONE;
    const at::Tensor& r = THPVariable_Unpack(a[0]);
    const int64_t B = r.numel();
    if (B == 0) Py_RETURN_NONE;
    at::Tensor adv = new_like(r, {B}, at::kFloat), mean = new_like(r, {G}, at::kFloat), std = new_like(r, {G}, at::kFloat);
    at::Tensor flags = new_like(r, {G}, at::kByte);
    // (whatever may throw stands before the GIL is given up: the handler below needs it)
    float *const adv_ptr = static_cast<float*>(adv.mutable_data_ptr()), *const mean_ptr = static_cast<float*>(mean.mutable_data_ptr());
    float* const std_ptr = static_cast<float*>(std.mutable_data_ptr());
    uint8_t* const flags_ptr = static_cast<uint8_t*>(flags.mutable_data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_group_advantages(static_cast<float*>(rewards), static_cast<int32_t*>(group), static_cast<uint8_t*>(in_stats),
                              static_cast<uint8_t*>(scored), static_cast<uint8_t*>(own), static_cast<float*>(shift), B, G, mode, eps, ddof,
                              mix, neg, pos, adv_ptr, mean_ptr, std_ptr, flags_ptr, reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(iNNNN)", rc, THPVariable_Wrap(std::move(adv)), THPVariable_Wrap(std::move(mean)),
                         THPVariable_Wrap(std::move(std)), THPVariable_Wrap(std::move(flags)));
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (src_logp, src_mask, src_word_map, src_map_len, tgt_mask, tgt_word_map, tgt_map_len, max_words, ignore_value, want_bad_count, stream)
// -> (status, out, bad or None) or None
PyObject* align(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    void* p[7];
    static const at::ScalarType types[7] = {at::kFloat, at::kByte, at::kInt, at::kInt, at::kByte, at::kInt, at::kInt};
    int32_t words;
    float ignore;
    int64_t stream;
    if (n != 11) Py_RETURN_NONE;
    for (int i = 0; i < 7; ++i)
      if (!tensor_arg(a[i], types[i], false, &p[i])) Py_RETURN_NONE;
    if (!int32_arg(a[7], &words) || !float_arg(a[8], &ignore) || (a[9] != Py_True && a[9] != Py_False) || !int_arg(a[10], &stream))
      Py_RETURN_NONE;
    const at::Tensor &src = THPVariable_Unpack(a[0]), &tgt = THPVariable_Unpack(a[4]);
    if (src.dim() != 2 || tgt.dim() < 2 || src.size(1) > INT32_MAX || tgt.size(1) > INT32_MAX || src.numel() == 0 || tgt.numel() == 0)
      Py_RETURN_NONE;
    const int64_t B = src.size(0), S_src = src.size(1), S_tgt = tgt.size(1);
    at::Tensor out = new_like(src, {B, S_tgt}, at::kFloat), bad;
    if (a[9] == Py_True) bad = new_like(src, {1}, at::kLong);
    float* const out_ptr = static_cast<float*>(out.mutable_data_ptr());
    int64_t* const bad_ptr = bad.defined() ? static_cast<int64_t*>(bad.mutable_data_ptr()) : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_thl_word_align(static_cast<float*>(p[0]), static_cast<uint8_t*>(p[1]), static_cast<int32_t*>(p[2]), static_cast<int32_t*>(p[3]),
                            static_cast<uint8_t*>(p[4]), static_cast<int32_t*>(p[5]), static_cast<int32_t*>(p[6]), B, (int32_t)S_src,
                            (int32_t)S_tgt, words, ignore, out_ptr, bad_ptr, reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    Py_INCREF(Py_None);
    PyObject* second = Py_None;
    if (bad.defined()) { Py_DECREF(Py_None); second = THPVariable_Wrap(std::move(bad)); }
    return Py_BuildValue("(iNN)", rc, THPVariable_Wrap(std::move(out)), second);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// A tensor argument of one of the types that calls (5) and (6) take, on the given device; its shape is checked by the caller.
bool typed_arg(PyObject* o, int64_t device, const at::Tensor** t, int32_t* type) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& x = THPVariable_Unpack(o);
  if (!x.is_cuda() || !x.is_contiguous() || x.get_device() != device) return false;
  if (x.scalar_type() == at::kBFloat16) *type = MRL_BF16;
  else if (x.scalar_type() == at::kFloat) *type = MRL_F32;
  else return false;
  *t = &x;
  return true;
}
bool same_rows(const at::Tensor& a, const at::Tensor& b) { return a.dim() == 2 && a.size(0) == b.size(0) && a.size(1) == b.size(1); }
bool mask_arg(PyObject* o, int64_t device, int64_t N, const uint8_t** mask) {
  void* p;
  if (!tensor_arg(o, at::kByte, true, &p)) return false;
  if (o != Py_None && (THPVariable_Unpack(o).numel() != N || THPVariable_Unpack(o).get_device() != device)) return false;
  *mask = static_cast<const uint8_t*>(p);
  return true;
}

// (x, weight, eps, residual, token_mask, out_dtype, scale_block, device, stream) -> (status, y, h or None, scale or None) or None
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    const at::Tensor *x, *w, *res = nullptr;
    int32_t xt, wt, rt = MRL_F32, yt, block;
    int64_t device, stream;
    float eps;
    const uint8_t* mask;
    if (n != 9 || !int_arg(a[7], &device) || !int_arg(a[8], &stream) || !typed_arg(a[0], device, &x, &xt) || !typed_arg(a[1], device, &w, &wt) ||
        !float_arg(a[2], &eps) || (a[3] != Py_None && !typed_arg(a[3], device, &res, &rt)) || x->dim() != 2 || x->numel() == 0 ||
        !mask_arg(a[4], device, x->size(0), &mask) || !THPDtype_Check(a[5]) || !int32_arg(a[6], &block) || x->size(1) > INT32_MAX ||
        w->dim() != 1 || w->size(0) != x->size(1) || (res != nullptr && !same_rows(*res, *x)) || (block != 0 && block != 128))
      Py_RETURN_NONE;
    const at::ScalarType out = reinterpret_cast<THPDtype*>(a[5])->scalar_type;
    if (out == at::kFloat) yt = MRL_F32;
    else if (out == at::kBFloat16) yt = MRL_BF16;
    else if (out == at::kFloat8_e4m3fn) yt = MRL_E4M3;
    else Py_RETURN_NONE;
    const int64_t N = x->size(0), d = x->size(1);
    at::Tensor y = new_like(*x, {N, d}, out), h, scale;
    if (res != nullptr) h = new_like(*x, {N, d}, res->scalar_type());
    if (yt == MRL_E4M3) scale = block != 0 ? new_like(*x, {N, (d + block - 1) / block}, at::kFloat) : new_like(*x, {N}, at::kFloat);
    const void *xp = x->const_data_ptr(), *wp = w->const_data_ptr(), *rp = res != nullptr ? res->const_data_ptr() : nullptr;
    void *yp = y.mutable_data_ptr(), *hp = h.defined() ? h.mutable_data_ptr() : nullptr;
    float* const sp = scale.defined() ? static_cast<float*>(scale.mutable_data_ptr()) : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_rms_norm(xp, rp, wp, mask, N, (int32_t)d, eps, xt, rt, wt, yt, block, hp, yp, sp, reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(iNNN)", rc, THPVariable_Wrap(std::move(y)), THPVariable_Wrap(std::move(h)), THPVariable_Wrap(std::move(scale)));
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (dy, h, weight, eps, d_residual, token_mask, dx_dtype, out_dweight, accumulate, want_dweight, workspace, device, stream)
// -> (status, dx, dweight or None) or None
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    const at::Tensor *dy, *h, *w, *res = nullptr, *given = nullptr;
    int32_t dyt, ht, wt, rt, gt, dxt;
    int64_t device, stream;
    float eps;
    const uint8_t* mask;
    if (n != 13 || !int_arg(a[11], &device) || !int_arg(a[12], &stream) || !typed_arg(a[0], device, &dy, &dyt) || !typed_arg(a[1], device, &h, &ht) ||
        !typed_arg(a[2], device, &w, &wt) || !float_arg(a[3], &eps) || (a[4] != Py_None && !typed_arg(a[4], device, &res, &rt)) || h->dim() != 2 ||
        h->numel() == 0 || !mask_arg(a[5], device, h->size(0), &mask) || !THPDtype_Check(a[6]) ||
        (a[7] != Py_None && !typed_arg(a[7], device, &given, &gt)) || (a[8] != Py_True && a[8] != Py_False) || (a[9] != Py_True && a[9] != Py_False) ||
        a[10] != Py_None || h->size(1) > INT32_MAX || !same_rows(*dy, *h) || w->dim() != 1 || w->size(0) != h->size(1) ||
        (res != nullptr && (rt != ht || !same_rows(*res, *h))) ||
        (given != nullptr && (gt != MRL_F32 || given->dim() != 1 || given->size(0) != h->size(1))) || (a[8] == Py_True && given == nullptr))
      Py_RETURN_NONE;
    const at::ScalarType out = reinterpret_cast<THPDtype*>(a[6])->scalar_type;
    if (out == at::kFloat) dxt = MRL_F32;
    else if (out == at::kBFloat16) dxt = MRL_BF16;
    else Py_RETURN_NONE;
    const int64_t N = h->size(0), d = h->size(1);
    at::Tensor dx = new_like(*h, {N, d}, out), dw, ws;
    if (given != nullptr) dw = *given;
    else if (a[9] == Py_True) dw = new_like(*h, {d}, at::kFloat);
    size_t bytes = 0;
    if (dw.defined()) {
      bytes = mrl_rms_norm_backward_workspace(N, (int32_t)d);
      if (bytes == 0) Py_RETURN_NONE;
      ws = new_like(*h, {(int64_t)bytes}, at::kByte);
    }
    const void *dyp = dy->const_data_ptr(), *hp = h->const_data_ptr(), *wp = w->const_data_ptr(), *rp = res != nullptr ? res->const_data_ptr() : nullptr;
    void *dxp = dx.mutable_data_ptr(), *wsp = ws.defined() ? ws.mutable_data_ptr() : nullptr;
    float* const dwp = dw.defined() ? static_cast<float*>(dw.mutable_data_ptr()) : nullptr;
    const int accumulate = a[8] == Py_True;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_rms_norm_backward(dyp, hp, wp, rp, mask, N, (int32_t)d, eps, dyt, ht, wt, dxt, accumulate, dxp, dwp, wsp, bytes,
                               reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    PyObject* second = a[7];
    if (given != nullptr) Py_INCREF(second); else second = THPVariable_Wrap(std::move(dw));
    return Py_BuildValue("(iNN)", rc, THPVariable_Wrap(std::move(dx)), second);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (address of a plan's table, tensors, max_norm, workspace, device, stream) -> (status, [norm, coefficient]) or None
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    int64_t table, device, stream;
    int32_t count;
    void* ws;
    if (n != 6 || !int_arg(a[0], &table) || !int32_arg(a[1], &count) || !PyFloat_CheckExact(a[2]) || !tensor_arg(a[3], at::kByte, false, &ws) ||
        !int_arg(a[4], &device) || !int_arg(a[5], &stream))
      Py_RETURN_NONE;
    const at::Tensor& w = THPVariable_Unpack(a[3]);
    if (w.get_device() != device) Py_RETURN_NONE;
    const double max_norm = PyFloat_AS_DOUBLE(a[2]);
    const size_t bytes = (size_t)w.numel();
    at::Tensor out = new_like(w, {2}, at::kFloat);
    float* const out_ptr = static_cast<float*>(out.mutable_data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_grad_norm(reinterpret_cast<const mrl_param_tensor*>(table), count, max_norm, out_ptr, ws, bytes, reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(iN)", rc, THPVariable_Wrap(std::move(out)));
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (address of a plan's table, tensors, workspace (which says where the plan is), lr, step, beta1, beta2, eps, norm_coef or None, seed, skip_nonfinite,
// state_dtype, device, stream) -> (status,) or None
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    int64_t table, device, stream, step, seed;
    int32_t count, state;
    void *ws, *coef;
    if (n != 14 || !int_arg(a[0], &table) || !int32_arg(a[1], &count) || !tensor_arg(a[2], at::kByte, false, &ws) || !PyFloat_CheckExact(a[3]) ||
        !int_arg(a[4], &step) || !PyFloat_CheckExact(a[5]) || !PyFloat_CheckExact(a[6]) || !PyFloat_CheckExact(a[7]) ||
        !tensor_arg(a[8], at::kFloat, true, &coef) || !int_arg(a[9], &seed) || (a[10] != Py_True && a[10] != Py_False) || !int32_arg(a[11], &state) ||
        !int_arg(a[12], &device) || !int_arg(a[13], &stream) || THPVariable_Unpack(a[2]).get_device() != device || seed < 0)
      Py_RETURN_NONE;
    if (coef != nullptr && (THPVariable_Unpack(a[8]).numel() != 2 || THPVariable_Unpack(a[8]).get_device() != device)) Py_RETURN_NONE;
    const mrl_adamw_config c = {PyFloat_AS_DOUBLE(a[3]), PyFloat_AS_DOUBLE(a[5]), PyFloat_AS_DOUBLE(a[6]), PyFloat_AS_DOUBLE(a[7]), step, (uint64_t)seed,
                                state, a[10] == Py_True, nullptr, nullptr};
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_adamw(reinterpret_cast<const mrl_param_tensor*>(table), count, &c, coef != nullptr ? static_cast<const float*>(coef) + 1 : nullptr,
                   reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(i)", rc);
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// Tensors of one int32 or float for each of N rows, or None.
bool rows_arg(PyObject* o, at::ScalarType type, int64_t device, int64_t N, bool optional, void** p) {
  if (!tensor_arg(o, type, optional, p)) return false;
  return o == Py_None || (THPVariable_Unpack(o).numel() == N && THPVariable_Unpack(o).get_device() == device);
}
bool flag_arg(PyObject* o, bool* v) {
  *v = o == Py_True;
  return o == Py_True || o == Py_False;
}
bool float_dtype(PyObject* o, at::ScalarType* type, int32_t* code) {
  if (!THPDtype_Check(o)) return false;
  *type = reinterpret_cast<THPDtype*>(o)->scalar_type;
  *code = *type == at::kBFloat16 ? MRL_BF16 : MRL_F32;
  return *type == at::kFloat || *type == at::kBFloat16;
}
template <class T> T* data_or_null(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.mutable_data_ptr()) : nullptr; }

// (logits, k, target_ids, token_mask, temperature, want_lse, want_entropy, device, stream) -> (status, ids, top_logp, logp, lse, entropy) or None
PyObject* top_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    int64_t device, stream;
    int32_t k, type;
    float temperature;
    bool want_lse, want_entropy;
    if (n != 9 || !int_arg(a[7], &device) || !int_arg(a[8], &stream) || !THPVariable_CheckExact(a[0]) || !int32_arg(a[1], &k) || !float_arg(a[4], &temperature) ||
        !flag_arg(a[5], &want_lse) || !flag_arg(a[6], &want_entropy))
      Py_RETURN_NONE;
    const at::Tensor& z = THPVariable_Unpack(a[0]);
    if (!z.is_cuda() || z.get_device() != device || z.dim() != 2 || z.numel() == 0 || z.size(1) > INT32_MAX) Py_RETURN_NONE;
    if (z.scalar_type() == at::kBFloat16) type = MRL_BF16;
    else if (z.scalar_type() == at::kFloat) type = MRL_F32;
    else Py_RETURN_NONE;
    const int64_t N = z.size(0), V = z.size(1);
    void *targets, *mask;
    if ((V > 1 && z.stride(1) != 1) || (N > 1 && z.stride(0) < V) || k < 0 || k > V || !rows_arg(a[2], at::kInt, device, N, true, &targets) ||
        !rows_arg(a[3], at::kByte, device, N, true, &mask))
      Py_RETURN_NONE;
    const size_t bytes = mrl_top_logprobs_workspace(N, (int32_t)V, k);
    if (bytes == 0) Py_RETURN_NONE;
    at::Tensor ids, top, logp, lse, entropy, ws;
    if (k > 0) { ids = new_like(z, {N, k}, at::kInt); top = new_like(z, {N, k}, at::kFloat); }
    if (targets != nullptr) logp = new_like(z, {N}, at::kFloat);
    if (want_lse) lse = new_like(z, {N}, at::kFloat);
    if (want_entropy) entropy = new_like(z, {N}, at::kFloat);
    if (bytes > 256) ws = new_like(z, {(int64_t)bytes}, at::kByte);
    const void* zp = z.const_data_ptr();
    int32_t* const ids_ptr = data_or_null<int32_t>(ids);
    float *const top_ptr = data_or_null<float>(top), *const logp_ptr = data_or_null<float>(logp), *const lse_ptr = data_or_null<float>(lse);
    float* const entropy_ptr = data_or_null<float>(entropy);
    void* const ws_ptr = data_or_null<void>(ws);
    const int64_t stride = N > 1 ? z.stride(0) : V;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_top_logprobs(zp, stride, static_cast<int32_t*>(targets), static_cast<uint8_t*>(mask), N, (int32_t)V, k, type, temperature, ids_ptr, top_ptr, logp_ptr,
                          lse_ptr, entropy_ptr, ws_ptr, ws_ptr != nullptr ? bytes : 0, reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(iNNNNN)", rc, THPVariable_Wrap(std::move(ids)), THPVariable_Wrap(std::move(top)), THPVariable_Wrap(std::move(logp)),
                         THPVariable_Wrap(std::move(lse)), THPVariable_Wrap(std::move(entropy)));
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (table, ids, scale, token_mask, out_dtype, device, stream) -> (status, y) or None
PyObject* embedding(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    const at::Tensor* table;
    int64_t device, stream;
    int32_t tt, yt;
    float scale;
    void *ids, *mask;
    at::ScalarType out;
    if (n != 7 || !int_arg(a[5], &device) || !int_arg(a[6], &stream) || !typed_arg(a[0], device, &table, &tt) || !float_arg(a[2], &scale) ||
        !float_dtype(a[4], &out, &yt) || table->dim() != 2 || table->numel() == 0 || table->size(0) > INT32_MAX || table->size(1) > INT32_MAX ||
        !THPVariable_CheckExact(a[1]))
      Py_RETURN_NONE;
    const at::Tensor& which = THPVariable_Unpack(a[1]);
    const int64_t N = which.numel(), V = table->size(0), d = table->size(1);
    if (N == 0 || which.dim() != 1 || !rows_arg(a[1], at::kInt, device, N, false, &ids) || !rows_arg(a[3], at::kByte, device, N, true, &mask)) Py_RETURN_NONE;
    at::Tensor y = new_like(*table, {N, d}, out);
    const void* tp = table->const_data_ptr();
    void* const yp = y.mutable_data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_embedding(tp, static_cast<int32_t*>(ids), static_cast<uint8_t*>(mask), N, (int32_t)d, (int32_t)V, scale, tt, yt, yp, reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(iN)", rc, THPVariable_Wrap(std::move(y)));
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (dy, ids, V, scale, token_mask, out_dtype, device, stream) -> (status, gradient) or None
PyObject* embedding_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    const at::Tensor* dy;
    int64_t device, stream;
    int32_t yt, ot, V;
    float scale;
    void *ids, *mask;
    at::ScalarType out;
    if (n != 8 || !int_arg(a[6], &device) || !int_arg(a[7], &stream) || !typed_arg(a[0], device, &dy, &yt) || !int32_arg(a[2], &V) || !float_arg(a[3], &scale) ||
        !float_dtype(a[5], &out, &ot) || dy->dim() != 2 || dy->numel() == 0 || dy->size(1) > INT32_MAX || V <= 0 || !THPVariable_CheckExact(a[1]))
      Py_RETURN_NONE;
    const int64_t N = dy->size(0), d = dy->size(1);
    if (THPVariable_Unpack(a[1]).dim() != 1 || !rows_arg(a[1], at::kInt, device, N, false, &ids) || !rows_arg(a[4], at::kByte, device, N, true, &mask)) Py_RETURN_NONE;
    const size_t bytes = mrl_embedding_backward_workspace(N, (int32_t)d, V);
    if (bytes == 0) Py_RETURN_NONE;
    at::Tensor table = new_like(*dy, {V, d}, out), ws = new_like(*dy, {(int64_t)bytes}, at::kByte);
    const void* dyp = dy->const_data_ptr();
    void *const tp = table.mutable_data_ptr(), *const wsp = ws.mutable_data_ptr();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_embedding_backward(dyp, static_cast<int32_t*>(ids), static_cast<uint8_t*>(mask), N, (int32_t)d, V, scale, yt, ot, 0, tp, wsp, bytes,
                                reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(iN)", rc, THPVariable_Wrap(std::move(table)));
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

// (hidden, lm_head_w, teacher_ids, teacher_logp, token_mask, row_weight, temperature, renormalize, dh_dtype, dw_dtype, chunk_rows, want_dH, want_dW, device, stream)
// -> (status, kl, dH, dW, stats) or None
PyObject* distill(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    const at::Tensor *h, *w;
    int64_t device, stream;
    int32_t ht, wt;
    mrl_distill_config c = {};
    void *mask, *weight, *ids, *logp;
    bool want_dH, want_dW;
    if (n != 15 || !int_arg(a[13], &device) || !int_arg(a[14], &stream) || !typed_arg(a[0], device, &h, &ht) || !typed_arg(a[1], device, &w, &wt) || ht != wt ||
        !float_arg(a[6], &c.temperature) || !int32_arg(a[7], &c.renormalize) || !int32_arg(a[8], &c.dh_dtype) || !int32_arg(a[9], &c.dw_dtype) ||
        !int32_arg(a[10], &c.chunk_rows) || !flag_arg(a[11], &want_dH) || !flag_arg(a[12], &want_dW) || h->dim() != 2 || w->dim() != 2 || h->numel() == 0 ||
        w->numel() == 0 || h->size(1) != w->size(1) || h->size(1) > INT32_MAX || w->size(0) > INT32_MAX || !tensor_arg(a[2], at::kInt, false, &ids) ||
        !tensor_arg(a[3], at::kFloat, false, &logp))
      Py_RETURN_NONE;
    const at::Tensor &ti = THPVariable_Unpack(a[2]), &tl = THPVariable_Unpack(a[3]);
    const int64_t N = h->size(0), d = h->size(1), V = w->size(0);
    if (ti.dim() != 2 || ti.size(0) != N || ti.size(1) > INT32_MAX || !same_rows(ti, tl) || ti.get_device() != device || tl.get_device() != device ||
        !rows_arg(a[4], at::kByte, device, N, true, &mask) || !rows_arg(a[5], at::kFloat, device, N, true, &weight) ||
        (c.dh_dtype != MRL_F32 && c.dh_dtype != MRL_BF16) || (c.dw_dtype != MRL_F32 && c.dw_dtype != MRL_BF16))
      Py_RETURN_NONE;
    const int32_t k = (int32_t)ti.size(1);
    const size_t bytes = mrl_distill_loss_workspace(N, (int32_t)d, (int32_t)V, k, ht, &c);
    if (bytes == 0) Py_RETURN_NONE;
    at::Tensor kl = new_like(*h, {N}, at::kFloat), dH, dW, stats = new_like(*h, {(int64_t)sizeof(mrl_distill_stats)}, at::kByte);
    if (want_dH) dH = new_like(*h, {N, d}, c.dh_dtype == MRL_BF16 ? at::kBFloat16 : at::kFloat);
    if (want_dW) dW = new_like(*h, {V, d}, c.dw_dtype == MRL_BF16 ? at::kBFloat16 : at::kFloat);
    at::Tensor ws = new_like(*h, {(int64_t)bytes}, at::kByte);
    const void *hp = h->const_data_ptr(), *wp = w->const_data_ptr();
    float* const klp = static_cast<float*>(kl.mutable_data_ptr());
    void *const dHp = data_or_null<void>(dH), *const dWp = data_or_null<void>(dW), *const wsp = ws.mutable_data_ptr();
    mrl_distill_stats* const sp = static_cast<mrl_distill_stats*>(stats.mutable_data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mrl_distill_loss_fwd_bwd(hp, wp, static_cast<int32_t*>(ids), static_cast<float*>(logp), static_cast<uint8_t*>(mask), static_cast<float*>(weight), N,
                                  (int32_t)d, (int32_t)V, k, ht, &c, klp, dHp, dWp, sp, wsp, bytes, reinterpret_cast<void*>(stream));
    Py_END_ALLOW_THREADS
    return Py_BuildValue("(iNNNN)", rc, THPVariable_Wrap(std::move(kl)), THPVariable_Wrap(std::move(dH)), THPVariable_Wrap(std::move(dW)),
                         THPVariable_Wrap(std::move(stats)));
  } catch (...) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
}

PyMethodDef methods[] = {
    {"advantages", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(advantages)), METH_FASTCALL, nullptr},
    {"align", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(align)), METH_FASTCALL, nullptr},
    {"rms_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rms_norm)), METH_FASTCALL, nullptr},
    {"rms_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rms_norm_backward)), METH_FASTCALL, nullptr},
    {"grad_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(grad_norm)), METH_FASTCALL, nullptr},
    {"adamw", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(adamw)), METH_FASTCALL, nullptr},
    {"top_logprobs", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(top_logprobs)), METH_FASTCALL, nullptr},
    {"embedding", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(embedding)), METH_FASTCALL, nullptr},
    {"embedding_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(embedding_backward)), METH_FASTCALL, nullptr},
    {"distill", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(distill)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "mrl_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_mrl_host() {
  PyObject* m = PyModule_Create(&module);
  // (the torch whose C++ interface this was compiled against: the caller compares before the first use)
  if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", MRL_TORCH_VERSION) != 0) Py_CLEAR(m);
  return m;
}
