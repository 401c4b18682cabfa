// The calls a training loop makes every step, for CPython: argument marshalling in C++ instead of
// ctypes.  The functions of libnoloco.so are handed over by address when the binding loads, so this
// module links against nothing.  A step of a small arena is bound by the host: through ctypes
// plan_groups took 6.2 us and outer_step 12.5 us, of which the C ABI itself takes 4.5.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#define NPY_NO_DEPRECATED_API NPY_1_7_API_VERSION
#include <numpy/arrayobject.h>

#include <cstdint>
#include <cstring>

#include "noloco.h"

namespace {

decltype(&noloco_plan_groups) plan_groups_fn = nullptr;
decltype(&noloco_outer_step) outer_step_fn = nullptr;
decltype(&noloco_replica_spread) spread_fn = nullptr;
decltype(&noloco_replica_spread_noalloc) spread_noalloc_fn = nullptr;
PyObject* to_int32 = nullptr;      // callable: anything array-like -> contiguous int32 numpy array
PyObject* data_ptr_name = nullptr;

// Address of a device buffer: None, an integer, or an object with data_ptr().
bool address_of(PyObject* x, void** out) {
  if (x == Py_None) { *out = nullptr; return true; }
  PyObject* value = nullptr;
  if (PyLong_CheckExact(x)) {
    value = Py_NewRef(x);
  } else {
    PyObject* method = PyObject_GetAttr(x, data_ptr_name);
    if (method != nullptr) {
      value = PyObject_CallNoArgs(method);
      Py_DECREF(method);
      if (value != nullptr && !PyLong_CheckExact(value)) {      // whatever int() takes
        PyObject* made = PyNumber_Long(value);
        Py_DECREF(value);
        value = made;
      }
    } else if (PyErr_ExceptionMatches(PyExc_AttributeError)) {
      PyErr_Clear();
      value = PyNumber_Long(x);
    }
  }
  if (value == nullptr) return false;
  *out = reinterpret_cast<void*>(static_cast<uintptr_t>(PyLong_AsUnsignedLongLongMask(value)));
  Py_DECREF(value);
  return !PyErr_Occurred();
}

// `values` as a contiguous int32 array, converted if it is anything else.  (numpy's own view: its buffer
// protocol builds a format string, 1 us each time.)
struct Int32Array {
  PyArrayObject* array = nullptr;
  ~Int32Array() { Py_XDECREF(array); }
  static bool fits(PyObject* x) {
    return PyArray_Check(x) && PyArray_TYPE(reinterpret_cast<PyArrayObject*>(x)) == NPY_INT32 &&
           PyArray_NDIM(reinterpret_cast<PyArrayObject*>(x)) > 0 && PyArray_ISCARRAY_RO(reinterpret_cast<PyArrayObject*>(x));
  }
  bool open(PyObject* values) {
    if (fits(values)) {
      array = reinterpret_cast<PyArrayObject*>(Py_NewRef(values));
      return true;
    }
    PyObject* made = PyObject_CallOneArg(to_int32, values);
    if (made == nullptr) return false;
    if (fits(made)) {
      array = reinterpret_cast<PyArrayObject*>(made);
      return true;
    }
    // ascontiguousarray() keeps an array that is contiguous at an odd address: it is copied to an aligned one
    array = reinterpret_cast<PyArrayObject*>(PyArray_FROMANY(made, NPY_INT32, 1, 0, NPY_ARRAY_IN_ARRAY));
    Py_DECREF(made);
    return array != nullptr;
  }
  int32_t* data() const { return static_cast<int32_t*>(PyArray_DATA(array)); }
  int32_t rows() const { return static_cast<int32_t>(PyArray_DIM(array, 0)); }
};

bool float_at(PyObject* seq, Py_ssize_t i, float* out) {
  PyObject* item = nullptr;
  if (PyTuple_CheckExact(seq) && i < PyTuple_GET_SIZE(seq)) {
    item = Py_NewRef(PyTuple_GET_ITEM(seq, i));
  } else if (PyObject* key = PyLong_FromSsize_t(i)) {
    item = PyObject_GetItem(seq, key);
    Py_DECREF(key);
  }
  if (item == nullptr) return false;
  PyObject* value = PyNumber_Float(item);
  Py_DECREF(item);
  if (value == nullptr) return false;
  *out = static_cast<float>(PyFloat_AS_DOUBLE(value));
  Py_DECREF(value);
  return true;
}

bool counted(Py_ssize_t got, Py_ssize_t want) {
  if (got == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, got);
  return false;
}

// plan_groups(seed, step, W, n, members, offsets): the last two are int32 arrays to fill
PyObject* plan_groups(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 6)) return nullptr;
  const uint64_t seed = PyLong_AsUnsignedLongLongMask(args[0]), step = PyLong_AsUnsignedLongLongMask(args[1]);
  const int32_t W = static_cast<int32_t>(PyLong_AsUnsignedLongLongMask(args[2]));
  const int32_t n = static_cast<int32_t>(PyLong_AsUnsignedLongLongMask(args[3]));
  if (PyErr_Occurred()) return nullptr;
  Int32Array members, offsets;
  if (!members.open(args[4]) || !offsets.open(args[5])) return nullptr;
  noloco_status status;
  Py_BEGIN_ALLOW_THREADS
  status = plan_groups_fn(seed, step, W, n, members.data(), offsets.data());
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// outer_step((plan, worker_stride, W, theta_dtype), phi, delta, theta, hparams, members, offsets, stream)
PyObject* outer_step(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 8)) return nullptr;
  PyObject* layout = args[0];
  void *plan, *phi, *delta, *theta, *stream;
  if (!address_of(PyTuple_GET_ITEM(layout, 0), &plan) || !address_of(args[1], &phi) || !address_of(args[2], &delta) ||
      !address_of(args[3], &theta) || !address_of(args[7], &stream))
    return nullptr;
  noloco_arena arena;
  std::memset(&arena, 0, sizeof(arena));       // the step does not read the segments
  arena.phi = static_cast<float*>(phi);
  arena.delta = static_cast<float*>(delta);
  arena.theta = theta;
  arena.worker_stride = PyLong_AsLongLong(PyTuple_GET_ITEM(layout, 1));
  arena.W = static_cast<int32_t>(PyLong_AsLongLong(PyTuple_GET_ITEM(layout, 2)));
  arena.theta_dtype = static_cast<int32_t>(PyLong_AsLongLong(PyTuple_GET_ITEM(layout, 3)));
  noloco_hparams hp;
  if (PyErr_Occurred() || !float_at(args[4], 0, &hp.alpha) || !float_at(args[4], 1, &hp.beta) ||
      !float_at(args[4], 2, &hp.gamma))
    return nullptr;
  Int32Array members, offsets;
  if (!members.open(args[5]) || !offsets.open(args[6])) return nullptr;
  const int32_t groups = offsets.rows() - 1;
  noloco_status status;
  Py_BEGIN_ALLOW_THREADS
  status = outer_step_fn(static_cast<noloco_launch_plan*>(plan), &arena, &hp, members.data(), offsets.data(), groups, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

PyObject* spread(decltype(spread_fn) fn, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 5)) return nullptr;
  void *plan, *x, *out, *stream;
  if (!address_of(PyTuple_GET_ITEM(args[0], 0), &plan) || !address_of(args[1], &x) || !address_of(args[3], &out) ||
      !address_of(args[4], &stream))
    return nullptr;
  const int32_t x_dtype = static_cast<int32_t>(PyLong_AsUnsignedLongLongMask(args[2]));
  if (PyErr_Occurred()) return nullptr;
  noloco_status status;
  Py_BEGIN_ALLOW_THREADS
  status = fn(static_cast<noloco_launch_plan*>(plan), x, x_dtype, static_cast<double*>(out), stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// replica_spread((plan, ...), x, x_dtype, out_std, stream)
PyObject* replica_spread(PyObject*, PyObject* const* args, Py_ssize_t count) { return spread(spread_fn, args, count); }
PyObject* replica_spread_noalloc(PyObject*, PyObject* const* args, Py_ssize_t count) {
  return spread(spread_noalloc_fn, args, count);
}

// bind(addresses of noloco_plan_groups, _outer_step, _replica_spread, _replica_spread_noalloc, to_int32)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 5)) return nullptr;
  void* fn[4];
  for (int i = 0; i < 4; ++i)
    if (!address_of(args[i], &fn[i])) return nullptr;
  plan_groups_fn = reinterpret_cast<decltype(plan_groups_fn)>(fn[0]);
  outer_step_fn = reinterpret_cast<decltype(outer_step_fn)>(fn[1]);
  spread_fn = reinterpret_cast<decltype(spread_fn)>(fn[2]);
  spread_noalloc_fn = reinterpret_cast<decltype(spread_noalloc_fn)>(fn[3]);
  Py_XDECREF(to_int32);
  to_int32 = Py_NewRef(args[4]);
  Py_RETURN_NONE;
}

decltype(&noloco_orthogonalize) orthogonalize_fn = nullptr;
decltype(&noloco_muon_step) muon_step_fn = nullptr;
decltype(&noloco_embed_lookup) lookup_fn = nullptr;
decltype(&noloco_embed_gradient) gradient_fn = nullptr;

bool int32_of(PyObject* x, int32_t* out) {
  *out = static_cast<int32_t>(PyLong_AsUnsignedLongLongMask(x));
  return !PyErr_Occurred();
}

bool float_of(PyObject* x, float* out) {
  PyObject* value = PyNumber_Float(x);
  if (value == nullptr) return false;
  *out = static_cast<float>(PyFloat_AS_DOUBLE(value));
  Py_DECREF(value);
  return true;
}

// Newton-Schulz coefficients, a sequence of (a, b, c) for every step, with eps and products.  More steps than the library
// takes are counted but not kept: it refuses them by their number.
struct Method {
  float k[3 * NOLOCO_MAX_NEWTON_SCHULZ_STEPS];
  noloco_newton_schulz method;
  bool open(PyObject* coefficients, PyObject* eps, PyObject* products) {
    const Py_ssize_t steps = PySequence_Size(coefficients);
    if (steps < 0) return false;
    for (Py_ssize_t s = 0; s < steps; ++s) {
      PyObject* step = PySequence_GetItem(coefficients, s);
      if (step == nullptr) return false;
      const Py_ssize_t count = PySequence_Size(step);
      if (count != 3) {
        Py_DECREF(step);
        if (count >= 0) PyErr_SetString(PyExc_ValueError, "coefficients: three numbers for every step");
        return false;
      }
      for (Py_ssize_t i = 0; i < 3; ++i) {
        float value;
        if (!float_at(step, i, &value)) {
          Py_DECREF(step);
          return false;
        }
        if (s < NOLOCO_MAX_NEWTON_SCHULZ_STEPS) k[3 * s + i] = value;
      }
      Py_DECREF(step);
    }
    method.steps = steps > INT32_MAX ? INT32_MAX : static_cast<int32_t>(steps);
    method.coefficients = k;
    return float_of(eps, &method.eps) && int32_of(products, &method.products);
  }
};

// orthogonalize(plan, x, x_dtype, out, out_dtype, coefficients, eps, products, stream)
PyObject* orthogonalize(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 9)) return nullptr;
  void *plan, *x, *out, *stream;
  int32_t x_dtype, out_dtype;
  Method method;
  if (!address_of(args[0], &plan) || !address_of(args[1], &x) || !int32_of(args[2], &x_dtype) || !address_of(args[3], &out) ||
      !int32_of(args[4], &out_dtype) || !method.open(args[5], args[6], args[7]) || !address_of(args[8], &stream))
    return nullptr;
  noloco_status status;
  Py_BEGIN_ALLOW_THREADS
  status = orthogonalize_fn(static_cast<noloco_muon_plan*>(plan), x, x_dtype, out, out_dtype, &method.method, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// muon_step(plan, theta, theta_dtype, grad, grad_dtype, momentum, (lr, mu, weight_decay), nesterov, coefficients, eps, products, stream)
PyObject* muon_step(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 12)) return nullptr;
  void *plan, *theta, *grad, *momentum, *stream;
  int32_t theta_dtype, grad_dtype;
  noloco_muon_hparams hp;
  Method method;
  if (!address_of(args[0], &plan) || !address_of(args[1], &theta) || !int32_of(args[2], &theta_dtype) || !address_of(args[3], &grad) ||
      !int32_of(args[4], &grad_dtype) || !address_of(args[5], &momentum) || !float_at(args[6], 0, &hp.lr) || !float_at(args[6], 1, &hp.mu) ||
      !float_at(args[6], 2, &hp.weight_decay) || !int32_of(args[7], &hp.nesterov) || !method.open(args[8], args[9], args[10]) ||
      !address_of(args[11], &stream))
    return nullptr;
  noloco_status status;
  Py_BEGIN_ALLOW_THREADS
  status = muon_step_fn(static_cast<noloco_muon_plan*>(plan), theta, theta_dtype, grad, grad_dtype, static_cast<float*>(momentum), &hp,
                        &method.method, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// What lookup and gradient share: (plan, first, first_dtype, tokens, token_type, num_tokens, scale, second, second_dtype ...)
struct Embedding {
  void *plan, *first, *tokens, *second;
  int32_t first_dtype, token_type, second_dtype;
  int64_t num_tokens;
  float scale;
  bool open(PyObject* const* args) {
    if (!address_of(args[0], &plan) || !address_of(args[1], &first) || !int32_of(args[2], &first_dtype) || !address_of(args[3], &tokens) ||
        !int32_of(args[4], &token_type))
      return false;
    num_tokens = PyLong_AsLongLong(args[5]);
    return !PyErr_Occurred() && float_of(args[6], &scale) && address_of(args[7], &second) && int32_of(args[8], &second_dtype);
  }
};

// embed_lookup(plan, table, table_dtype, tokens, token_type, num_tokens, scale, out, out_dtype, stream)
PyObject* embed_lookup(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 10)) return nullptr;
  Embedding e;
  void* stream;
  if (!e.open(args) || !address_of(args[9], &stream)) return nullptr;
  noloco_status status;
  Py_BEGIN_ALLOW_THREADS
  status = lookup_fn(static_cast<noloco_embedding_plan*>(e.plan), e.first, e.first_dtype, e.tokens, e.token_type, e.num_tokens, e.scale,
                     e.second, e.second_dtype, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// embed_gradient(plan, dout, dout_dtype, tokens, token_type, num_tokens, scale, grad, grad_dtype, accumulate, stream)
PyObject* embed_gradient(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 11)) return nullptr;
  Embedding e;
  int32_t accumulate;
  void* stream;
  if (!e.open(args) || !int32_of(args[9], &accumulate) || !address_of(args[10], &stream)) return nullptr;
  noloco_status status;
  Py_BEGIN_ALLOW_THREADS
  status = gradient_fn(static_cast<noloco_embedding_plan*>(e.plan), e.first, e.first_dtype, e.tokens, e.token_type, e.num_tokens, e.scale,
                       e.second, e.second_dtype, accumulate, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// bind_inner(addresses of noloco_orthogonalize, _muon_step, _embed_lookup, _embed_gradient)
PyObject* bind_inner(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 4)) return nullptr;
  void* fn[4];
  for (int i = 0; i < 4; ++i)
    if (!address_of(args[i], &fn[i])) return nullptr;
  orthogonalize_fn = reinterpret_cast<decltype(orthogonalize_fn)>(fn[0]);
  muon_step_fn = reinterpret_cast<decltype(muon_step_fn)>(fn[1]);
  lookup_fn = reinterpret_cast<decltype(lookup_fn)>(fn[2]);
  gradient_fn = reinterpret_cast<decltype(gradient_fn)>(fn[3]);
  Py_RETURN_NONE;
}

decltype(&noloco_layer_norm) layer_norm_fn = nullptr;
decltype(&noloco_layer_norm_gradient) layer_norm_gradient_fn = nullptr;
decltype(&noloco_linear) linear_fn = nullptr;
decltype(&noloco_linear_gradient) linear_gradient_fn = nullptr;
decltype(&noloco_token_log_probs) log_probs_fn = nullptr;
decltype(&noloco_token_log_probs_gradient) log_probs_gradient_fn = nullptr;

// The arguments of a call, one after the other, as the types they are taken as.
struct Arguments {
  PyObject* const* args;
  bool take(void** out) { return address_of(*args++, out); }
  bool take(float** out) { return take(reinterpret_cast<void**>(out)); }
  bool take(int32_t** out) { return take(reinterpret_cast<void**>(out)); }
  bool take(int32_t* out) { return int32_of(*args++, out); }
  bool take(float* out) { return float_of(*args++, out); }
  bool take(int64_t* out) {
    *out = PyLong_AsLongLong(*args++);
    return !PyErr_Occurred();
  }
  template <typename... T> bool all(T*... out) { return (take(out) && ...); }
};

template <typename Call> PyObject* status_of(const Call& call) {
  noloco_status status;
  Py_BEGIN_ALLOW_THREADS
  status = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// layer_norm(plan, norm, x, x_dtype, theta, theta_dtype, num_tokens, eps, out, out_dtype, stats, stream)
PyObject* layer_norm(PyObject*, PyObject* const* args, Py_ssize_t count) {
  void *plan, *x, *theta, *out, *stream;
  float *stats, eps;
  int32_t norm, x_dtype, theta_dtype, out_dtype;
  int64_t tokens;
  if (!counted(count, 12) || !Arguments{args}.all(&plan, &norm, &x, &x_dtype, &theta, &theta_dtype, &tokens, &eps, &out, &out_dtype, &stats, &stream))
    return nullptr;
  return status_of([&] {
    return layer_norm_fn(static_cast<noloco_layer_norm_plan*>(plan), norm, x, x_dtype, theta, theta_dtype, tokens, eps, out, out_dtype, stats, stream);
  });
}

// layer_norm_gradient(plan, norm, dout, dout_dtype, x, x_dtype, theta, theta_dtype, stats, num_tokens, add, dx, dx_dtype, grad, grad_dtype,
//                     accumulate, stream)
PyObject* layer_norm_gradient(PyObject*, PyObject* const* args, Py_ssize_t count) {
  void *plan, *dout, *x, *theta, *add, *dx, *grad, *stream;
  float* stats;
  int32_t norm, dout_dtype, x_dtype, theta_dtype, dx_dtype, grad_dtype, accumulate;
  int64_t tokens;
  if (!counted(count, 17) || !Arguments{args}.all(&plan, &norm, &dout, &dout_dtype, &x, &x_dtype, &theta, &theta_dtype, &stats, &tokens, &add, &dx,
                                                  &dx_dtype, &grad, &grad_dtype, &accumulate, &stream))
    return nullptr;
  return status_of([&] {
    return layer_norm_gradient_fn(static_cast<noloco_layer_norm_plan*>(plan), norm, dout, dout_dtype, x, x_dtype, theta, theta_dtype, stats, tokens,
                                  add, dx, dx_dtype, grad, grad_dtype, accumulate, stream);
  });
}

// linear(plan, layer, x, x_dtype, theta, theta_dtype, num_tokens, activation, residual, before, out, out_dtype, stream)
PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t count) {
  void *plan, *x, *theta, *residual, *before, *out, *stream;
  int32_t layer, x_dtype, theta_dtype, activation, out_dtype;
  int64_t tokens;
  if (!counted(count, 13) || !Arguments{args}.all(&plan, &layer, &x, &x_dtype, &theta, &theta_dtype, &tokens, &activation, &residual, &before, &out,
                                                  &out_dtype, &stream))
    return nullptr;
  return status_of([&] {
    return linear_fn(static_cast<noloco_linear_plan*>(plan), layer, x, x_dtype, theta, theta_dtype, tokens, activation, residual, before, out,
                     out_dtype, stream);
  });
}

// linear_gradient(plan, layer, dout, dout_dtype, x, x_dtype, theta, theta_dtype, num_tokens, activation, before, add, dx, dx_dtype, grad,
//                 grad_dtype, accumulate, stream)
PyObject* linear_gradient(PyObject*, PyObject* const* args, Py_ssize_t count) {
  void *plan, *dout, *x, *theta, *before, *add, *dx, *grad, *stream;
  int32_t layer, dout_dtype, x_dtype, theta_dtype, activation, dx_dtype, grad_dtype, accumulate;
  int64_t tokens;
  if (!counted(count, 18) || !Arguments{args}.all(&plan, &layer, &dout, &dout_dtype, &x, &x_dtype, &theta, &theta_dtype, &tokens, &activation, &before,
                                                  &add, &dx, &dx_dtype, &grad, &grad_dtype, &accumulate, &stream))
    return nullptr;
  return status_of([&] {
    return linear_gradient_fn(static_cast<noloco_linear_plan*>(plan), layer, dout, dout_dtype, x, x_dtype, theta, theta_dtype, tokens, activation,
                              before, add, dx, dx_dtype, grad, grad_dtype, accumulate, stream);
  });
}

// token_log_probs(plan, logits, logits_dtype, tokens, token_type, num_tokens, log_probs, entropy, norms, top, top_tokens, top_log_probs, stream)
PyObject* token_log_probs(PyObject*, PyObject* const* args, Py_ssize_t count) {
  void *plan, *logits, *tokens, *stream;
  float *log_probs, *entropy, *norms, *top_log_probs;
  int32_t logits_dtype, token_type, top, *top_tokens;
  int64_t num_tokens;
  if (!counted(count, 13) || !Arguments{args}.all(&plan, &logits, &logits_dtype, &tokens, &token_type, &num_tokens, &log_probs, &entropy, &norms, &top,
                                                  &top_tokens, &top_log_probs, &stream))
    return nullptr;
  return status_of([&] {
    return log_probs_fn(static_cast<noloco_log_prob_plan*>(plan), logits, logits_dtype, tokens, token_type, num_tokens, log_probs, entropy, norms, top,
                        top_tokens, top_log_probs, stream);
  });
}

// token_log_probs_gradient(plan, logits, logits_dtype, tokens, token_type, num_tokens, norms, dlog_probs, dentropy, entropy, dlogits,
//                          dlogits_dtype, stream)
PyObject* token_log_probs_gradient(PyObject*, PyObject* const* args, Py_ssize_t count) {
  void *plan, *logits, *tokens, *dlogits, *stream;
  float *norms, *dlog_probs, *dentropy, *entropy;
  int32_t logits_dtype, token_type, dlogits_dtype;
  int64_t num_tokens;
  if (!counted(count, 13) || !Arguments{args}.all(&plan, &logits, &logits_dtype, &tokens, &token_type, &num_tokens, &norms, &dlog_probs, &dentropy,
                                                  &entropy, &dlogits, &dlogits_dtype, &stream))
    return nullptr;
  return status_of([&] {
    return log_probs_gradient_fn(static_cast<noloco_log_prob_plan*>(plan), logits, logits_dtype, tokens, token_type, num_tokens, norms, dlog_probs,
                                 dentropy, entropy, dlogits, dlogits_dtype, stream);
  });
}

// bind_model(addresses of noloco_layer_norm, _layer_norm_gradient, _linear, _linear_gradient, _token_log_probs, _token_log_probs_gradient)
PyObject* bind_model(PyObject*, PyObject* const* args, Py_ssize_t count) {
  if (!counted(count, 6)) return nullptr;
  void* fn[6];
  for (int i = 0; i < 6; ++i)
    if (!address_of(args[i], &fn[i])) return nullptr;
  layer_norm_fn = reinterpret_cast<decltype(layer_norm_fn)>(fn[0]);
  layer_norm_gradient_fn = reinterpret_cast<decltype(layer_norm_gradient_fn)>(fn[1]);
  linear_fn = reinterpret_cast<decltype(linear_fn)>(fn[2]);
  linear_gradient_fn = reinterpret_cast<decltype(linear_gradient_fn)>(fn[3]);
  log_probs_fn = reinterpret_cast<decltype(log_probs_fn)>(fn[4]);
  log_probs_gradient_fn = reinterpret_cast<decltype(log_probs_gradient_fn)>(fn[5]);
  Py_RETURN_NONE;
}

template <typename F> PyCFunction fast(F f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {
    {"bind", fast(bind), METH_FASTCALL, nullptr},
    {"plan_groups", fast(plan_groups), METH_FASTCALL, nullptr},
    {"outer_step", fast(outer_step), METH_FASTCALL, nullptr},
    {"replica_spread", fast(replica_spread), METH_FASTCALL, nullptr},
    {"replica_spread_noalloc", fast(replica_spread_noalloc), METH_FASTCALL, nullptr},
    {"bind_inner", fast(bind_inner), METH_FASTCALL, nullptr},
    {"orthogonalize", fast(orthogonalize), METH_FASTCALL, nullptr},
    {"muon_step", fast(muon_step), METH_FASTCALL, nullptr},
    {"embed_lookup", fast(embed_lookup), METH_FASTCALL, nullptr},
    {"embed_gradient", fast(embed_gradient), METH_FASTCALL, nullptr},
    {"bind_model", fast(bind_model), METH_FASTCALL, nullptr},
    {"layer_norm", fast(layer_norm), METH_FASTCALL, nullptr},
    {"layer_norm_gradient", fast(layer_norm_gradient), METH_FASTCALL, nullptr},
    {"linear", fast(linear), METH_FASTCALL, nullptr},
    {"linear_gradient", fast(linear_gradient), METH_FASTCALL, nullptr},
    {"token_log_probs", fast(token_log_probs), METH_FASTCALL, nullptr},
    {"token_log_probs_gradient", fast(token_log_probs_gradient), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) {
  import_array();
  data_ptr_name = PyUnicode_InternFromString("data_ptr");
  return data_ptr_name == nullptr ? nullptr : PyModule_Create(&module);
}
