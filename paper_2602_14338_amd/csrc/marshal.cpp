// The binding's native part.
//
//   group_advantage(...), logprob_fwd(...), ...: a whole call whose arguments are all plain - tensors of the expected dtype,
//   on the GPU and contiguous, ints that fit, floats - straight to the entry point whose address bind() was given.
//   Anything else, also whatever the call would refuse, gives NotImplemented with nothing done, and the binding goes
//   its general way, which converts or raises.  (ctypes and the parameter structure were 2 of the 5.7 us of a call that
//   launches one small kernel.)
//
// Checks and device pointers of a call's tensors in one step: the part of the binding that costs most of a small
// call when it runs in Python (fifteen tensors at 0.5 us each against 3 us for a launch).
//
//   pointers(t0, dtype0, name0, t1, dtype1, name1, ...) -> (address or None, ...)
//
// Per tensor, in this order: None stays None; it must live on the GPU, have the dtype (None: any) and be
// contiguous.  Anything but a plain tensor or parameter goes to the Python function given to setup(), which
// performs the same checks.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include "../../include/aero.h"

namespace {

PyObject* g_error = nullptr;      // exception class of the binding
PyObject* g_general = nullptr;    // pointer of any other kind of tensor: f(t, dtype, name)

PyObject* setup(PyObject*, PyObject* args) {
  PyObject *error, *general;
  if (!PyArg_ParseTuple(args, "OO", &error, &general)) return nullptr;
  Py_INCREF(error);
  Py_INCREF(general);
  Py_XSETREF(g_error, error);
  Py_XSETREF(g_general, general);
  Py_RETURN_NONE;
}

PyObject* pointers(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
  HANDLE_TH_ERRORS
  if (!g_error || n_args % 3 != 0) {
    PyErr_SetString(PyExc_TypeError, "pointers: expected (tensor, dtype, name) triples after setup()");
    return nullptr;
  }
  THPObjectPtr out(PyTuple_New(n_args / 3));
  if (!out) return nullptr;
  for (Py_ssize_t i = 0; i < n_args; i += 3) {
    PyObject *t = args[i], *dtype = args[i + 1], *name = args[i + 2], *value;
    if (t == Py_None) {
      value = Py_NewRef(Py_None);
    } else if (!THPVariable_CheckExact(t)) {
      value = PyObject_CallFunctionObjArgs(g_general, t, dtype, name, nullptr);
    } else {
      const at::Tensor& x = THPVariable_Unpack(t);
      if (!x.is_cuda()) {
        PyErr_Format(g_error, "%U: expected a GPU tensor", name);
        return nullptr;
      }
      if (dtype != Py_None && x.scalar_type() != reinterpret_cast<THPDtype*>(dtype)->scalar_type) {
        THPObjectPtr got(PyObject_GetAttrString(t, "dtype"));
        if (got) PyErr_Format(g_error, "%U: expected dtype %S, got %S", name, dtype, got.get());
        return nullptr;
      }
      if (!x.is_contiguous()) {
        PyErr_Format(g_error, "%U: expected a contiguous tensor", name);
        return nullptr;
      }
      value = PyLong_FromVoidPtr(x.data_ptr());
    }
    if (!value) return nullptr;
    PyTuple_SET_ITEM(out.get(), i / 3, value);
  }
  return out.release();
  END_HANDLE_TH_ERRORS
}

// ---- whole calls ----
PyObject* g_stream = nullptr;     // torch's current raw stream of a device index
PyObject* g_params = nullptr;     // class of group_advantage's parameters
PyObject* g_pair_params = nullptr;    // of the preference losses'
PyObject* g_adamw_params = nullptr;   // of the AdamW step's
decltype(&aero_group_advantage) g_group_advantage = nullptr;
decltype(&aero_logprob_fwd) g_logprob_fwd = nullptr;
decltype(&aero_grpo_loss_bwd) g_loss_bwd = nullptr;
decltype(&aero_grpo_loss_bwd_noalloc) g_loss_bwd_noalloc = nullptr;
decltype(&aero_lmhead_logprob_fused) g_fused = nullptr;
decltype(&aero_topk_logprob) g_topk = nullptr;
decltype(&aero_distill_loss_bwd) g_distill = nullptr;
decltype(&aero_verify_draft) g_verify = nullptr;
decltype(&aero_embedding_fwd) g_embed_fwd = nullptr;
decltype(&aero_embedding_bwd) g_embed_bwd = nullptr;
decltype(&aero_preference_loss) g_pair = nullptr;
decltype(&aero_preference_loss_bwd) g_pair_bwd = nullptr;
decltype(&aero_grad_norm) g_norm = nullptr;
decltype(&aero_adamw_step) g_adamw = nullptr;

PyObject* bind(PyObject*, PyObject* args) {
  PyObject *stream, *params, *pair_params, *adamw_params;
  unsigned long long f[14];
  if (!PyArg_ParseTuple(args, "OOOOKKKKKKKKKKKKKK", &stream, &params, &pair_params, &adamw_params, &f[0], &f[1], &f[2], &f[3], &f[4], &f[5],
                        &f[6], &f[7], &f[8], &f[9], &f[10], &f[11], &f[12], &f[13]))
    return nullptr;
  Py_INCREF(stream);
  Py_INCREF(params);
  Py_INCREF(pair_params);
  Py_INCREF(adamw_params);
  Py_XSETREF(g_stream, stream);
  Py_XSETREF(g_params, params);
  Py_XSETREF(g_pair_params, pair_params);
  Py_XSETREF(g_adamw_params, adamw_params);
  g_group_advantage = reinterpret_cast<decltype(g_group_advantage)>(f[0]);
  g_logprob_fwd = reinterpret_cast<decltype(g_logprob_fwd)>(f[1]);
  g_loss_bwd = reinterpret_cast<decltype(g_loss_bwd)>(f[2]);
  g_loss_bwd_noalloc = reinterpret_cast<decltype(g_loss_bwd_noalloc)>(f[3]);
  g_fused = reinterpret_cast<decltype(g_fused)>(f[4]);
  g_topk = reinterpret_cast<decltype(g_topk)>(f[5]);
  g_distill = reinterpret_cast<decltype(g_distill)>(f[6]);
  g_verify = reinterpret_cast<decltype(g_verify)>(f[7]);
  g_embed_fwd = reinterpret_cast<decltype(g_embed_fwd)>(f[8]);
  g_embed_bwd = reinterpret_cast<decltype(g_embed_bwd)>(f[9]);
  g_pair = reinterpret_cast<decltype(g_pair)>(f[10]);
  g_pair_bwd = reinterpret_cast<decltype(g_pair_bwd)>(f[11]);
  g_norm = reinterpret_cast<decltype(g_norm)>(f[12]);
  g_adamw = reinterpret_cast<decltype(g_adamw)>(f[13]);
  Py_RETURN_NONE;
}

// The arguments of a call, taken in order; ok turns false at the first one that is not plain.
struct Plain {
  PyObject* const* next;
  bool ok = true;

  const at::Tensor* tensor() {   // nullptr: None, or not plain
    PyObject* o = *next++;
    if (o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) {
      ok = false;
      return nullptr;
    }
    const at::Tensor& x = THPVariable_Unpack(o);
    if (!x.is_cuda() || !x.is_contiguous()) ok = false;
    return &x;
  }
  void* any() {
    const at::Tensor* x = tensor();
    return x && ok ? x->data_ptr() : nullptr;
  }
  template <class T> T* of(at::ScalarType type) {
    const at::Tensor* x = tensor();
    if (x && x->scalar_type() != type) ok = false;
    return x && ok ? static_cast<T*>(x->data_ptr()) : nullptr;
  }
  float* f32() { return of<float>(at::kFloat); }
  int32_t* i32() { return of<int32_t>(at::kInt); }
  uint8_t* u8() { return of<uint8_t>(at::kByte); }
  int64_t integer(int64_t lo, int64_t hi) { return integer_of(*next++, lo, hi); }
  int64_t integer_of(PyObject* o, int64_t lo, int64_t hi) {
    int overflow = 1;
    const int64_t v = PyLong_CheckExact(o) ? PyLong_AsLongLongAndOverflow(o, &overflow) : 0;
    if (overflow || v < lo || v > hi) ok = false;
    return v;
  }
  int32_t int32() { return int32_t(integer(INT32_MIN, INT32_MAX)); }
  int64_t int64() { return integer(INT64_MIN, INT64_MAX); }
  float real() { return real_of(*next++); }
  float real_of(PyObject* o) {
    if (PyFloat_CheckExact(o)) return float(PyFloat_AS_DOUBLE(o));
    return float(integer_of(o, -(1 << 24), 1 << 24));
  }
};

// Storage code of logits (-1: none).
int32_t dtype_code(const at::Tensor& x) {
  switch (x.scalar_type()) {
    case at::kFloat: return AERO_F32;
    case at::kBFloat16: return AERO_BF16;
    case at::kHalf: return AERO_F16;
    case at::kFloat8_e4m3fn: return AERO_F8E4M3;
    default: return -1;
  }
}

// torch's current stream on the tensor's device.
bool stream_of(const at::Tensor& x, void** stream) {
  THPObjectPtr device(PyLong_FromLong(x.get_device()));
  if (!device) return false;
  THPObjectPtr handle(PyObject_CallOneArg(g_stream, device));
  if (!handle) return false;
  *stream = PyLong_AsVoidPtr(handle);
  return !PyErr_Occurred();
}

// A call whose arguments are plain: the entry point without the interpreter lock, its status as an int.
template <class Call> PyObject* finish(const Plain& p, const at::Tensor* on, Call call) {
  if (!p.ok || !on) Py_RETURN_NOTIMPLEMENTED;
  void* stream = nullptr;
  if (!stream_of(*on, &stream)) return nullptr;
  aero_status status;
  Py_BEGIN_ALLOW_THREADS
  status = call(stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

const at::Tensor* peek(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

PyObject* group_advantage(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 15 || !g_group_advantage) Py_RETURN_NOTIMPLEMENTED;
  static PyObject* names[9];
  if (!names[8]) {
    const char* const text[9] = {"k_ratio", "s_rescue", "tau_num", "tau_den", "zero_keep", "reject_enable", "posterior_mode", "alpha0", "beta0"};
    for (int k = 0; k < 9; ++k)
      if (!(names[k] = PyUnicode_InternFromString(text[k]))) return nullptr;
  }
  Plain p{args};
  const float* rewards = p.f32();
  const int32_t* lengths = p.i32();
  const at::Tensor* on = peek(*p.next);
  const int32_t* offsets = p.i32();
  const uint32_t* keys = static_cast<uint32_t*>(p.any());
  const int32_t Q = p.int32(), R = p.int32();
  PyObject* params = *p.next++;
  if (reinterpret_cast<PyObject*>(Py_TYPE(params)) != g_params) Py_RETURN_NOTIMPLEMENTED;
  int32_t whole[7];
  float prior[2];
  for (int k = 0; k < 9; ++k) {
    THPObjectPtr v(PyObject_GetAttr(params, names[k]));
    if (!v) {   // no such attribute: the general way raises
      PyErr_Clear();
      Py_RETURN_NOTIMPLEMENTED;
    }
    if (k < 7) whole[k] = int32_t(p.integer_of(v, INT32_MIN, INT32_MAX));
    else prior[k - 7] = p.real_of(v);
  }
  const aero_adv_params c{whole[0], whole[1], whole[2], whole[3], whole[4], whole[5], whole[6], prior[0], prior[1]};
  float *adv = p.f32(), *weight = p.f32();
  uint8_t* mask = p.u8();
  int32_t *index = p.i32(), *kept = p.i32();
  uint8_t *zero_var = p.u8(), *category = p.u8();
  int32_t* err = p.i32();
  return finish(p, on, [&](void* s) {
    return g_group_advantage(rewards, lengths, offsets, keys, Q, R, &c, adv, weight, mask, index, kept, zero_var, category, err, s);
  });
  END_HANDLE_TH_ERRORS
}

PyObject* logprob_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 10 || !g_logprob_fwd) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const at::Tensor* on = peek(*p.next);
  const void* logits = p.any();
  const int32_t dtype = on ? dtype_code(*on) : -1;
  if (dtype < 0) p.ok = false;
  const int64_t T = p.int64();
  const int32_t V = p.int32();
  const int64_t ld = p.int64();
  const int32_t* targets = p.i32();
  const uint8_t* active = p.u8();
  float *logprob = p.f32(), *entropy = p.f32(), *lse = p.f32();
  int32_t* err = p.i32();
  return finish(p, on, [&](void* s) { return g_logprob_fwd(logits, dtype, T, V, ld, targets, active, logprob, entropy, lse, err, s); });
  END_HANDLE_TH_ERRORS
}

// loss_bwd(logits, T, V, ld, targets, lse, entropy, old_logprob, token_rollout, adv, weight, R, eps_lo, eps_hi, grad_scale,
//          entropy_coef, kl_coef, ref_logprob, loss, clip_frac, logprob_out, entropy_out, lse_out, dlogits, err_flag
//          [, workspace]): with the workspace aero_grpo_loss_bwd, without it aero_grpo_loss_bwd_noalloc
PyObject* loss_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if ((n != 25 && n != 26) || !g_loss_bwd) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const at::Tensor* on = peek(*p.next);
  const void* logits = p.any();
  const int32_t dtype = on ? dtype_code(*on) : -1;
  if (dtype < 0) p.ok = false;
  const int64_t T = p.int64();
  const int32_t V = p.int32();
  const int64_t ld = p.int64();
  const int32_t* targets = p.i32();
  const float *lse = p.f32(), *entropy = p.f32(), *old = p.f32();
  const int32_t* owner = p.i32();
  const float *adv = p.f32(), *weight = p.f32();
  const int32_t R = p.int32();
  const float eps_lo = p.real(), eps_hi = p.real(), scale = p.real(), ent_coef = p.real(), kl_coef = p.real();
  const float* ref = p.f32();
  float *loss = p.f32(), *clip = p.f32(), *lp_out = p.f32(), *ent_out = p.f32(), *lse_out = p.f32();
  const at::Tensor* d = peek(*p.next);
  void* dlogits = p.any();
  if (d && on && d->scalar_type() != on->scalar_type()) p.ok = false;
  int32_t* err = p.i32();
  if (n == 25)
    return finish(p, on, [&](void* s) {
      return g_loss_bwd_noalloc(logits, dtype, T, V, ld, targets, lse, entropy, old, owner, adv, weight, R, eps_lo, eps_hi, scale,
                                ent_coef, kl_coef, ref, loss, clip, lp_out, ent_out, lse_out, dlogits, err, s);
    });
  const at::Tensor* w = peek(*p.next);
  void* ws = p.any();
  const size_t bytes = w ? w->nbytes() : 0;
  return finish(p, on, [&](void* s) {
    return g_loss_bwd(logits, dtype, T, V, ld, targets, lse, entropy, old, owner, adv, weight, R, eps_lo, eps_hi, scale, ent_coef,
                      kl_coef, ref, loss, clip, lp_out, ent_out, lse_out, dlogits, err, ws, bytes, s);
  });
  END_HANDLE_TH_ERRORS
}

// fused(hidden, weight, T, H, V, targets, logprob, entropy, lse, old_logprob, token_rollout, adv, weight_rollout, R, eps_lo,
//       eps_hi, grad_scale, entropy_coef, kl_coef, ref_logprob, loss, clip_frac, dhidden, dweight, dweight_accumulate, err_flag,
//       workspace)
PyObject* fused(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 27 || !g_fused) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const at::Tensor* on = peek(*p.next);
  const void *hidden = p.of<void>(at::kBFloat16), *weight = p.of<void>(at::kBFloat16);
  const int64_t T = p.int64();
  const int32_t H = p.int32(), V = p.int32();
  const int32_t* targets = p.i32();
  float *logprob = p.f32(), *entropy = p.f32(), *lse = p.f32();
  const float* old = p.f32();
  const int32_t* owner = p.i32();
  const float *adv = p.f32(), *weight_rollout = p.f32();
  const int32_t R = p.int32();
  const float eps_lo = p.real(), eps_hi = p.real(), scale = p.real(), ent_coef = p.real(), kl_coef = p.real();
  const float* ref = p.f32();
  float *loss = p.f32(), *clip = p.f32();
  void* dhidden = p.of<void>(at::kBFloat16);
  const at::Tensor* dw = peek(*p.next);
  void* dweight = p.any();
  int32_t dw_dtype = dw ? dtype_code(*dw) : AERO_F32;
  if (dw_dtype < 0) p.ok = false;
  PyObject* accumulate = *p.next++;
  if (accumulate == Py_True) dw_dtype |= AERO_DW_ACCUMULATE;
  else if (accumulate != Py_False) p.ok = false;
  int32_t* err = p.i32();
  const at::Tensor* w = peek(*p.next);
  void* ws = p.any();
  const size_t bytes = w ? w->nbytes() : 0;
  return finish(p, on, [&](void* s) {
    return g_fused(hidden, weight, T, H, V, targets, logprob, entropy, lse, old, owner, adv, weight_rollout, R, eps_lo, eps_hi, scale,
                   ent_coef, kl_coef, ref, loss, clip, dhidden, dweight, dw_dtype, err, ws, bytes, s);
  });
  END_HANDLE_TH_ERRORS
}

// topk(logits, T, V, ld, row_active, K, index, logprob, lse, workspace)
PyObject* topk(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 10 || !g_topk) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const at::Tensor* on = peek(*p.next);
  const void* logits = p.any();
  const int32_t dtype = on ? dtype_code(*on) : -1;
  if (dtype < 0) p.ok = false;
  const int64_t T = p.int64();
  const int32_t V = p.int32();
  const int64_t ld = p.int64();
  const uint8_t* active = p.u8();
  const int32_t K = p.int32();
  int32_t* index = p.i32();
  float *logprob = p.f32(), *lse = p.f32();
  const at::Tensor* w = peek(*p.next);
  void* ws = p.any();
  const size_t bytes = w ? w->nbytes() : 0;
  return finish(p, on, [&](void* s) { return g_topk(logits, dtype, T, V, ld, active, K, index, logprob, lse, ws, bytes, s); });
  END_HANDLE_TH_ERRORS
}

// distill(logits, T, V, ld, teacher_index, teacher_logprob, K, token_weight, tail, grad_scale, loss, row_loss, dlogits, err_flag, workspace)
PyObject* distill(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 15 || !g_distill) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const at::Tensor* on = peek(*p.next);
  const void* logits = p.any();
  const int32_t dtype = on ? dtype_code(*on) : -1;
  if (dtype < 0) p.ok = false;
  const int64_t T = p.int64();
  const int32_t V = p.int32();
  const int64_t ld = p.int64();
  const int32_t* index = p.i32();
  const float* logprob = p.f32();
  const int32_t K = p.int32();
  const float* weight = p.f32();
  const int32_t tail = p.int32();
  const float scale = p.real();
  float *loss = p.f32(), *row_loss = p.f32();
  const at::Tensor* d = peek(*p.next);
  void* dlogits = p.any();
  if (d && on && d->scalar_type() != on->scalar_type()) p.ok = false;
  int32_t* err = p.i32();
  const at::Tensor* w = peek(*p.next);
  void* ws = p.any();
  const size_t bytes = w ? w->nbytes() : 0;
  return finish(p, on, [&](void* s) {
    return g_distill(logits, dtype, T, V, ld, index, logprob, K, weight, tail, scale, loss, row_loss, dlogits, err, ws, bytes, s);
  });
  END_HANDLE_TH_ERRORS
}

// verify(target_logits, draft_logits, B, G, V, ld, draft_tokens, draft_count, uniform, noise, accepted, tokens, logprob, err_flag, workspace)
PyObject* verify(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 15 || !g_verify) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const at::Tensor* on = peek(*p.next);
  const void* target = p.any();
  const int32_t dtype = on ? dtype_code(*on) : -1;
  if (dtype < 0) p.ok = false;
  const at::Tensor* d = peek(*p.next);
  const void* draft = p.any();
  if (d && on && d->scalar_type() != on->scalar_type()) p.ok = false;
  const int32_t B = p.int32(), G = p.int32(), V = p.int32();
  const int64_t ld = p.int64();
  const int32_t *drafted = p.i32(), *count = p.i32();
  const float *uniform = p.f32(), *noise = p.f32();
  int32_t *accepted = p.i32(), *tokens = p.i32();
  float* logprob = p.f32();
  int32_t* err = p.i32();
  const at::Tensor* w = peek(*p.next);
  void* ws = p.any();
  const size_t bytes = w ? w->nbytes() : 0;
  return finish(p, on, [&](void* s) {
    return g_verify(target, draft, dtype, B, G, V, ld, drafted, count, uniform, noise, accepted, tokens, logprob, err, ws, bytes, s);
  });
  END_HANDLE_TH_ERRORS
}

// embed_fwd(table, V, H, ids, T, scale, out, ld_out, err_flag)
PyObject* embed_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 9 || !g_embed_fwd) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const at::Tensor* on = peek(*p.next);
  const void* table = p.any();
  const int32_t dtype = on ? dtype_code(*on) : -1;
  if (dtype < 0) p.ok = false;
  const int32_t V = p.int32(), H = p.int32();
  const int32_t* ids = p.i32();
  const int64_t T = p.int64();
  const float scale = p.real();
  const at::Tensor* o = peek(*p.next);
  void* out = p.any();
  if (o && on && o->scalar_type() != on->scalar_type()) p.ok = false;
  const int64_t ld = p.int64();
  int32_t* err = p.i32();
  return finish(p, on, [&](void* s) { return g_embed_fwd(table, dtype, V, H, ids, T, scale, out, ld, err, s); });
  END_HANDLE_TH_ERRORS
}

// embed_bwd(dout, T, H, ld_dout, ids, V, scale, dtable, accumulate, err_flag, workspace)
PyObject* embed_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 11 || !g_embed_bwd) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const at::Tensor* on = peek(*p.next);
  const void* dout = p.any();
  const int32_t dtype = on ? dtype_code(*on) : -1;
  if (dtype < 0) p.ok = false;
  const int64_t T = p.int64();
  const int32_t H = p.int32();
  const int64_t ld = p.int64();
  const int32_t* ids = p.i32();
  const int32_t V = p.int32();
  const float scale = p.real();
  const at::Tensor* t = peek(*p.next);
  void* table = p.any();
  int32_t out_dtype = t ? dtype_code(*t) : -1;
  if (out_dtype < 0) p.ok = false;
  PyObject* accumulate = *p.next++;
  if (accumulate == Py_True) out_dtype |= AERO_DW_ACCUMULATE;
  else if (accumulate != Py_False) p.ok = false;
  int32_t* err = p.i32();
  const at::Tensor* w = peek(*p.next);
  void* ws = p.any();
  const size_t bytes = w ? w->nbytes() : 0;
  return finish(p, on, [&](void* s) {
    return g_embed_bwd(dout, dtype, T, H, ld, ids, V, scale, table, out_dtype, err, ws, bytes, s);
  });
  END_HANDLE_TH_ERRORS
}

// The next argument, an object of exactly the given class: its attributes, each handed to take(index, value).
template <int N, class Take> void attributes(Plain& p, PyObject* cls, PyObject* (&names)[N], const char* const (&text)[N], Take take) {
  PyObject* params = *p.next++;
  if (reinterpret_cast<PyObject*>(Py_TYPE(params)) != cls) {
    p.ok = false;
    return;
  }
  for (int k = 0; k < N; ++k) {
    if (!names[k] && !(names[k] = PyUnicode_InternFromString(text[k]))) throw python_error();
    THPObjectPtr v(PyObject_GetAttr(params, names[k]));
    if (!v) {   // no such attribute: the general way raises
      PyErr_Clear();
      p.ok = false;
      return;
    }
    take(k, v.get());
  }
}

aero_preference_params pair_params(Plain& p) {
  static PyObject* names[5];
  static const char* const text[5] = {"kind", "average", "beta", "smoothing", "margin"};
  int32_t whole[2] = {};
  float real[3] = {};
  attributes(p, g_pair_params, names, text, [&](int k, PyObject* v) {
    if (k < 2) whole[k] = int32_t(p.integer_of(v, INT32_MIN, INT32_MAX));
    else real[k - 2] = p.real_of(v);
  });
  return aero_preference_params{whole[0], whole[1], real[0], real[1], real[2]};
}

// pair(logprob, T, ref_logprob, token_rollout, R, chosen, rejected, weight, P, params, loss, margin, ratio, drollout, err_flag, workspace)
PyObject* pair(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 16 || !g_pair) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const float* logprob = p.f32();
  const int64_t T = p.int64();
  const float* ref = p.f32();
  const int32_t* owner = p.i32();
  const int32_t R = p.int32();
  const int32_t *chosen = p.i32(), *rejected = p.i32();
  const float* weight = p.f32();
  const int32_t P = p.int32();
  const aero_preference_params c = pair_params(p);
  const at::Tensor* on = peek(*p.next);
  float *loss = p.f32(), *margin = p.f32(), *ratio = p.f32(), *slope = p.f32();
  int32_t* err = p.i32();
  const at::Tensor* w = peek(*p.next);
  void* ws = p.any();
  const size_t bytes = w ? w->nbytes() : 0;
  return finish(p, on, [&](void* s) {
    return g_pair(logprob, T, ref, owner, R, chosen, rejected, weight, P, &c, loss, margin, ratio, slope, err, ws, bytes, s);
  });
  END_HANDLE_TH_ERRORS
}

// pair_bwd(logits, T, V, ld, targets, ref_logprob, token_rollout, R, chosen, rejected, weight, P, params, grad_scale, loss, margin, ratio,
//          logprob, dlogits, err_flag, workspace)
PyObject* pair_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 21 || !g_pair_bwd) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const at::Tensor* on = peek(*p.next);
  const void* logits = p.any();
  const int32_t dtype = on ? dtype_code(*on) : -1;
  if (dtype < 0) p.ok = false;
  const int64_t T = p.int64();
  const int32_t V = p.int32();
  const int64_t ld = p.int64();
  const int32_t* targets = p.i32();
  const float* ref = p.f32();
  const int32_t* owner = p.i32();
  const int32_t R = p.int32();
  const int32_t *chosen = p.i32(), *rejected = p.i32();
  const float* weight = p.f32();
  const int32_t P = p.int32();
  const aero_preference_params c = pair_params(p);
  const float scale = p.real();
  float *loss = p.f32(), *margin = p.f32(), *ratio = p.f32(), *lp_out = p.f32();
  const at::Tensor* d = peek(*p.next);
  void* dlogits = p.any();
  if (d && on && d->scalar_type() != on->scalar_type()) p.ok = false;
  int32_t* err = p.i32();
  const at::Tensor* w = peek(*p.next);
  void* ws = p.any();
  const size_t bytes = w ? w->nbytes() : 0;
  return finish(p, on, [&](void* s) {
    return g_pair_bwd(logits, dtype, T, V, ld, targets, ref, owner, R, chosen, rejected, weight, P, &c, scale, loss, margin, ratio, lp_out,
                      dlogits, err, ws, bytes, s);
  });
  END_HANDLE_TH_ERRORS
}

// norm(image address, table, grad_scale, max_norm, norm, factor, workspace)
PyObject* norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 7 || !g_norm) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const void* image = reinterpret_cast<const void*>(p.int64());
  const at::Tensor* on = peek(*p.next);
  void* table = p.any();
  const float scale = p.real(), most = p.real();
  float *out = p.f32(), *factor = p.f32();
  const at::Tensor* w = peek(*p.next);
  void* ws = p.any();
  const size_t bytes = w ? w->nbytes() : 0;
  return finish(p, on, [&](void* s) { return g_norm(image, table, scale, most, out, factor, ws, bytes, s); });
  END_HANDLE_TH_ERRORS
}

// adamw(image address, table, params, step, factor, lr_factor)
PyObject* adamw(PyObject*, PyObject* const* args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != 6 || !g_adamw) Py_RETURN_NOTIMPLEMENTED;
  Plain p{args};
  const void* image = reinterpret_cast<const void*>(p.int64());
  const at::Tensor* on = peek(*p.next);
  void* table = p.any();
  static PyObject* names[7];
  static const char* const text[7] = {"lr", "beta1", "beta2", "eps", "weight_decay", "seed", "stochastic"};
  aero_adamw_params c{};
  double* const real[5] = {&c.lr, &c.beta1, &c.beta2, &c.eps, &c.weight_decay};
  attributes(p, g_adamw_params, names, text, [&](int k, PyObject* v) {
    if (k < 5 && PyFloat_CheckExact(v)) *real[k] = PyFloat_AS_DOUBLE(v);
    else if (k < 5) *real[k] = double(p.integer_of(v, -(1 << 24), 1 << 24));
    else if (k == 5) c.seed = uint64_t(p.integer_of(v, 0, INT64_MAX));
    else if (v == Py_True || v == Py_False) c.stochastic = v == Py_True;
    else p.ok = false;
  });
  int32_t* step = p.i32();
  const float *factor = p.f32(), *lr_factor = p.f32();
  return finish(p, on, [&](void* s) { return g_adamw(image, table, &c, step, factor, lr_factor, s); });
  END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)> constexpr PyCFunction fast() {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F));
}

PyMethodDef methods[] = {
    {"setup", setup, METH_VARARGS, "setup(error class, pointer function for other kinds of tensors)"},
    {"bind", bind, METH_VARARGS, "bind(raw stream function, three parameter classes, fourteen entry points' addresses)"},
    {"pointers", fast<pointers>(), METH_FASTCALL, "pointers(t0, dtype0, name0, ...) -> tuple of addresses"},
    {"group_advantage", fast<group_advantage>(), METH_FASTCALL, "status, or NotImplemented"},
    {"logprob_fwd", fast<logprob_fwd>(), METH_FASTCALL, "status, or NotImplemented"},
    {"loss_bwd", fast<loss_bwd>(), METH_FASTCALL, "status, or NotImplemented"},
    {"fused", fast<fused>(), METH_FASTCALL, "status, or NotImplemented"},
    {"topk", fast<topk>(), METH_FASTCALL, "status, or NotImplemented"},
    {"distill", fast<distill>(), METH_FASTCALL, "status, or NotImplemented"},
    {"verify", fast<verify>(), METH_FASTCALL, "status, or NotImplemented"},
    {"embed_fwd", fast<embed_fwd>(), METH_FASTCALL, "status, or NotImplemented"},
    {"embed_bwd", fast<embed_bwd>(), METH_FASTCALL, "status, or NotImplemented"},
    {"pair", fast<pair>(), METH_FASTCALL, "status, or NotImplemented"},
    {"pair_bwd", fast<pair_bwd>(), METH_FASTCALL, "status, or NotImplemented"},
    {"norm", fast<norm>(), METH_FASTCALL, "status, or NotImplemented"},
    {"adamw", fast<adamw>(), METH_FASTCALL, "status, or NotImplemented"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
