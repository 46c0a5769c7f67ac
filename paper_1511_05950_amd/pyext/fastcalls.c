/* CPython entry points of the calls a training loop makes per gradient and per update.  Same calls and errors as through
 * ctypes; what they save is the argument conversion (a ctypes call with out-parameters costs about a microsecond, these about
 * a tenth), which bounds small networks: at 30-softsync an update of the CIFAR-shaped net takes about 10 us of GPU time and
 * six calls.  Linked against libsasgd.so, which lies next to this module. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <float.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#ifdef SASGD_TORCH_TENSORS
#include <ATen/dlpack.h>               /* torch's tensors through their C interface */
#endif

#include "../../include/sasgd.h"

static PyObject* error_class;     /* binding.SasgdError(code, message) */
static PyObject* s_data_ptr;      /* "data_ptr" */
static PyObject* s_ctypes;        /* "ctypes" */
static PyObject* s_data;          /* "data" */
static PyObject* s_dtype;         /* "dtype" */
static PyObject* s_shape;         /* "shape" */
static PyObject* s_stride;        /* "stride" */
static PyObject* s_element_size;  /* "element_size" */
static PyObject* s_get_device;    /* "get_device" */

static PyObject* raise_code(int code, const char* msg) {
  PyObject* exc = PyObject_CallFunction(error_class, "is", code, msg);
  if (exc) {
    PyErr_SetObject(error_class, exc);
    Py_DECREF(exc);
  }
  return NULL;
}
static PyObject* raise_ctx(sasgd_ctx* ctx, int code) { return raise_code(code, sasgd_last_error(ctx)); }

/* Address of None, an integer, a torch tensor or a numpy array; -1 on error (exception set). */
static int address(PyObject* o, void** out) {
  PyObject* v;
  if (o == Py_None) {
    *out = NULL;
    return 0;
  }
  if (PyLong_Check(o)) {
    *out = PyLong_AsVoidPtr(o);
    return PyErr_Occurred() ? -1 : 0;
  }
  v = PyObject_CallMethodNoArgs(o, s_data_ptr);
  if (!v) {
    PyObject* c;
    if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return -1;
    PyErr_Clear();
    c = PyObject_GetAttr(o, s_ctypes);
    v = c ? PyObject_GetAttr(c, s_data) : NULL;
    Py_XDECREF(c);
    if (!v) {
      PyErr_SetObject(PyExc_TypeError, (PyObject*)Py_TYPE(o));
      return -1;
    }
  }
  *out = PyLong_AsVoidPtr(v);
  Py_DECREF(v);
  return PyErr_Occurred() ? -1 : 0;
}

/* Python and numpy integers; a float is refused, as ctypes refuses it. */
static int integer(PyObject* o, long long* out) {
  PyObject* v;
  if (PyLong_Check(o)) {
    *out = PyLong_AsLongLong(o);
    return *out == -1 && PyErr_Occurred() ? -1 : 0;
  }
  v = PyNumber_Index(o);
  if (!v) return -1;
  *out = PyLong_AsLongLong(v);
  Py_DECREF(v);
  return *out == -1 && PyErr_Occurred() ? -1 : 0;
}
static int integer32(PyObject* o, int32_t* out) {
  long long v;
  if (integer(o, &v)) return -1;
  if (v < INT32_MIN || v > INT32_MAX) {
    PyErr_SetString(PyExc_OverflowError, "value does not fit 32 bits");
    return -1;
  }
  *out = (int32_t)v;
  return 0;
}

/* The same with int() applied first: staleness values of any numeric type. */
static int as_integer32(PyObject* o, int32_t* out) {
  PyObject* v;
  int bad;
  if (PyLong_Check(o)) return integer32(o, out);
  v = PyNumber_Long(o);
  if (!v) return -1;
  bad = integer32(v, out);
  Py_DECREF(v);
  return bad;
}

#define NARGS(n) \
  if (nargs != (n)) return PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", (n), nargs)
#define CTX(o)                      \
  void* h;                          \
  sasgd_ctx* ctx;                   \
  if (address((o), &h)) return NULL; \
  ctx = (sasgd_ctx*)h

static PyObject* get_minibatch(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  int32_t learner;
  void *x, *y;
  int rc;
  NARGS(4);
  CTX(a[0]);
  if (integer32(a[1], &learner) || address(a[2], &x) || address(a[3], &y)) return NULL;
  rc = sasgd_getMinibatch(ctx, learner, (const float*)x, (const int32_t*)y);
  if (rc) return raise_ctx(ctx, rc);
  Py_RETURN_NONE;
}

static PyObject* pull_weights(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  int32_t learner, stale;
  int64_t ts = 0;
  int rc;
  NARGS(3);
  CTX(a[0]);
  if (integer32(a[1], &learner) || integer32(a[2], &stale)) return NULL;
  rc = sasgd_pullWeights(ctx, learner, stale, &ts);
  if (rc) return raise_ctx(ctx, rc);
  return PyLong_FromLongLong(ts);
}

static PyObject* push_gradient(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  int32_t learner, tau = 0;
  int rc;
  NARGS(2);
  CTX(a[0]);
  if (integer32(a[1], &learner)) return NULL;
  rc = sasgd_pushGradient(ctx, learner, &tau);
  if (rc) return raise_ctx(ctx, rc);
  return PyLong_FromLong(tau);
}

static PyObject* push_gradient_external(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  void* g;
  long long ts;
  int32_t tau = 0;
  int rc;
  NARGS(3);
  CTX(a[0]);
  if (address(a[1], &g) || integer(a[2], &ts)) return NULL;
  rc = sasgd_pushGradientExternal(ctx, (const float*)g, ts, &tau);
  if (rc) return raise_ctx(ctx, rc);
  return PyLong_FromLong(tau);
}

static PyObject* sum_gradients(PyObject* self, PyObject* h0) {
  int32_t pending = 0;
  int rc;
  CTX(h0);
  rc = sasgd_sumGradients(ctx, &pending);
  if (rc) return raise_ctx(ctx, rc);
  return PyLong_FromLong(pending);
}

static PyObject* apply_update(PyObject* self, PyObject* h0) {
  int64_t ts = 0;
  int rc;
  CTX(h0);
  Py_BEGIN_ALLOW_THREADS            /* calls that may launch kernels leave the interpreter to other threads, as ctypes does */
  rc = sasgd_applyUpdate(ctx, &ts);
  Py_END_ALLOW_THREADS
  if (rc) return raise_ctx(ctx, rc);
  return PyLong_FromLongLong(ts);
}

static PyObject* timestamp(PyObject* self, PyObject* h0) {
  int64_t ts = 0;
  int rc;
  CTX(h0);
  rc = sasgd_timestamp(ctx, &ts);
  if (rc) return raise_ctx(ctx, rc);
  return PyLong_FromLongLong(ts);
}

/* A learner list: at most as many entries as a context can have learners (more is refused by the library's own check of the
 * count, which needs no entry beyond the first). */
#define MOST 64
static PyObject* calc_gradient(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  int32_t ids[MOST];
  Py_ssize_t n, k;
  void* loss;
  PyObject* seq;
  int rc;
  NARGS(3);
  CTX(a[0]);
  if (address(a[2], &loss)) return NULL;
  seq = PySequence_Fast(a[1], "learners must be a sequence");
  if (!seq) return NULL;
  n = PySequence_Fast_GET_SIZE(seq);
  for (k = 0; k < n && k < MOST; k++)
    if (integer32(PySequence_Fast_GET_ITEM(seq, k), &ids[k])) {
      Py_DECREF(seq);
      return NULL;
    }
  Py_DECREF(seq);
  Py_BEGIN_ALLOW_THREADS
  rc = sasgd_calcGradient(ctx, ids, n > MOST ? MOST + 1 : (int32_t)n, (float*)loss);
  Py_END_ALLOW_THREADS
  if (rc) return raise_ctx(ctx, rc);
  Py_RETURN_NONE;
}

/* apply_update_no_alloc(theta_in, theta_out, v, shadow, num_params, grads, staleness, lr_mode, alpha0, momentum, weight_decay,
 * stream) */
static PyObject* apply_update_no_alloc(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  void *tin, *tout, *v, *shadow, *stream;
  long long P;
  int32_t mode, stale[SASGD_NOALLOC_MAX_GRADIENTS];
  const float* grads[SASGD_NOALLOC_MAX_GRADIENTS];
  double alpha0, momentum, decay;
  Py_ssize_t c, k, nst;
  PyObject *gs, *ss;
  char err[256] = "";
  int rc, bad = 0;
  NARGS(12);
  if (address(a[0], &tin) || address(a[1], &tout) || address(a[2], &v) || address(a[3], &shadow) || integer(a[4], &P) ||
      integer32(a[7], &mode) || address(a[11], &stream))
    return NULL;
  alpha0 = PyFloat_AsDouble(a[8]);
  momentum = PyFloat_AsDouble(a[9]);
  decay = PyFloat_AsDouble(a[10]);
  if (PyErr_Occurred()) return NULL;
  gs = PySequence_Fast(a[5], "grads_dev must be a sequence");
  if (!gs) return NULL;
  ss = PySequence_Fast(a[6], "staleness must be a sequence");
  if (!ss) {
    Py_DECREF(gs);
    return NULL;
  }
  c = PySequence_Fast_GET_SIZE(gs);
  nst = PySequence_Fast_GET_SIZE(ss);
  if (nst > (c ? c : 1)) {                  /* one staleness per gradient; missing ones read as 0, as an array of c zeros does */
    PyErr_SetString(PyExc_IndexError, "more staleness values than gradients");
    bad = 1;
  }
  for (k = 0; !bad && k < c && k < SASGD_NOALLOC_MAX_GRADIENTS; k++) {
    void* g;
    stale[k] = 0;
    bad = address(PySequence_Fast_GET_ITEM(gs, k), &g) || (k < nst && as_integer32(PySequence_Fast_GET_ITEM(ss, k), &stale[k]));
    grads[k] = (const float*)g;
  }
  Py_DECREF(ss);
  if (bad) {
    Py_DECREF(gs);
    return NULL;
  }
  Py_BEGIN_ALLOW_THREADS            /* (gs may be all that holds the gradients: a generator's) */
  rc = sasgd_applyUpdateNoAlloc((const float*)tin, (float*)tout, (float*)v, (uint16_t*)shadow, P,
                                c > SASGD_NOALLOC_MAX_GRADIENTS ? SASGD_NOALLOC_MAX_GRADIENTS + 1 : (int32_t)c, grads, stale, mode, (float)alpha0,
                                (float)momentum, (float)decay, stream, err, sizeof(err));
  Py_END_ALLOW_THREADS
  Py_DECREF(gs);
  if (rc) return raise_code(rc, err);
  return PyLong_FromLong(rc);
}

/* A tensor as the calls below need it. */
#define MOST_DIMS 8
enum { KIND_OTHER = -1 };             /* else SASGD_FP32, SASGD_BF16 */
typedef struct {
  void* data;
  int device, kind, dims, itemsize;
  const int64_t *shape, *stride;       /* elements */
  int64_t own[2 * MOST_DIMS];
} view;

static PyObject *tensor_class, *fp32_type, *bf16_type;      /* torch.Tensor, torch.float32, torch.bfloat16: set_tensor_class */
#ifdef SASGD_TORCH_TENSORS
static const DLPackExchangeAPI* exchange;                   /* torch's C interface to its tensors, where it has one: 20 ns a tensor instead of 200 */
#endif

static int bad(PyObject* kind, const char* what, const char* why) {
  PyErr_Format(kind, "%s %s", what, why);
  return -1;
}

static int tuple_of(PyObject* o, PyObject* name, int call, int64_t* out, int* dims) {
  PyObject* t = call ? PyObject_CallMethodNoArgs(o, name) : PyObject_GetAttr(o, name);
  Py_ssize_t k, n;
  if (!t) return -1;
  n = PyTuple_Check(t) ? PyTuple_GET_SIZE(t) : MOST_DIMS + 1;
  if (n > MOST_DIMS) {
    Py_DECREF(t);
    return bad(PyExc_ValueError, "a tensor", "has too many dimensions");
  }
  for (k = 0; k < n; k++) out[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, k));
  Py_DECREF(t);
  *dims = (int)n;
  return PyErr_Occurred() ? -1 : 0;
}

static int view_of(PyObject* o, view* v) {
  PyObject* a;
#ifdef SASGD_TORCH_TENSORS
  if (exchange && (PyObject*)Py_TYPE(o) == tensor_class) {
    DLTensor t;
    if (exchange->dltensor_from_py_object_no_sync(o, &t) == 0 && t.ndim <= MOST_DIMS) {
      int k;
      int64_t n = 1;
      v->data = (char*)t.data + t.byte_offset;
      v->device = t.device.device_type == kDLCUDA || t.device.device_type == kDLROCM ? t.device.device_id : -1;
      v->kind = t.dtype.lanes != 1 ? KIND_OTHER : t.dtype.code == kDLFloat && t.dtype.bits == 32 ? SASGD_FP32
                : t.dtype.code == kDLBfloat && t.dtype.bits == 16 ? SASGD_BF16 : KIND_OTHER;
      v->itemsize = (t.dtype.bits + 7) / 8;
      v->dims = t.ndim;
      v->shape = t.shape;
      v->stride = t.strides;
      if (!t.strides) {
        for (k = t.ndim - 1; k >= 0; k--) {
          v->own[k] = n;
          n *= t.shape[k];
        }
        v->stride = v->own;
      }
      return 0;
    }
    PyErr_Clear();                     /* a kind of tensor that it does not show */
  }
#endif
  if (address(o, &v->data)) return -1;
  a = PyObject_CallMethodNoArgs(o, s_get_device);
  if (!a) return -1;
  v->device = (int)PyLong_AsLong(a);
  Py_DECREF(a);
  a = PyObject_GetAttr(o, s_dtype);
  if (!a) return -1;
  v->kind = a == fp32_type ? SASGD_FP32 : a == bf16_type ? SASGD_BF16 : KIND_OTHER;
  Py_DECREF(a);
  a = PyObject_CallMethodNoArgs(o, s_element_size);
  if (!a) return -1;
  v->itemsize = (int)PyLong_AsLong(a);
  Py_DECREF(a);
  v->shape = v->own;
  v->stride = v->own + MOST_DIMS;
  return tuple_of(o, s_shape, 0, v->own, &v->dims) || tuple_of(o, s_stride, 1, v->own + MOST_DIMS, &v->dims) ? -1 : 0;
}

static int64_t elements(const view* v) {
  int64_t n = 1;
  int k;
  for (k = 0; k < v->dims; k++) n *= v->shape[k];
  return n;
}
static int contiguous(const view* v) {
  int64_t n = 1;
  int k;
  for (k = v->dims - 1; k >= 0; k--) {
    if (v->shape[k] != 1 && v->stride[k] != n && elements(v) > 0) return 0;
    n *= v->shape[k];
  }
  return 1;
}

/* A contiguous tensor on the device, of `kind` where that is not KIND_OTHER, of at least `least` elements. */
static int want(PyObject* o, const char* name, int device, int kind, int64_t least, view* v) {
  if (view_of(o, v)) return -1;
  if (v->device != device) return bad(PyExc_ValueError, name, "is not on the current device");
  if (kind != KIND_OTHER && v->kind != kind) return bad(PyExc_TypeError, name, kind == SASGD_FP32 ? "must be float32" : "must be bfloat16");
  if (!contiguous(v)) return bad(PyExc_ValueError, name, "must be contiguous");
  if (elements(v) < least) return bad(PyExc_ValueError, name, "has too few elements");
  return 0;
}

/* Bytes and address of a workspace (None: none). */
static int workspace_of(PyObject* o, int device, void** data, size_t* bytes) {
  view v;
  *data = NULL;
  *bytes = 0;
  if (o == Py_None) return 0;
  if (want(o, "workspace", device, KIND_OTHER, 0, &v)) return -1;
  *data = v.data;
  *bytes = (size_t)elements(&v) * (size_t)v.itemsize;
  return 0;
}

/* The tensors of a list: contiguous, on the device, all of the first one's kind (*kind; SASGD_FP32 of an empty list).  numel: their lengths,
 * written, or where `known` compared with. */
static int list_of(PyObject* seq, Py_ssize_t n, int device, int* kind, const void** data, size_t apart, int64_t* numel, size_t numel_apart, int known) {
  Py_ssize_t k;
  for (k = 0; k < n; k++) {
    view v;
    int64_t count, *at = (int64_t*)((char*)numel + (size_t)k * numel_apart);
    if (view_of(PySequence_Fast_GET_ITEM(seq, k), &v)) return -1;
    if (v.device != device) return bad(PyExc_ValueError, "a gradient", "is not on the current device");
    if (v.kind == KIND_OTHER) return bad(PyExc_TypeError, "a gradient", "must be float32 or bfloat16");
    if (*kind == KIND_OTHER) *kind = v.kind;
    if (v.kind != *kind) return bad(PyExc_TypeError, "a gradient", "has another type than the first one");
    if (v.dims == 1) {
      count = v.shape[0];
      if (count > 1 && v.stride[0] != 1) return bad(PyExc_ValueError, "a gradient", "must be contiguous");
    } else {
      count = elements(&v);
      if (!contiguous(&v)) return bad(PyExc_ValueError, "a gradient", "must be contiguous");
    }
    if (known && count != *at) return bad(PyExc_ValueError, "a gradient", "has not its tensor's length");
    if (!known) *at = count;
    data[(size_t)k * apart] = v.data;
  }
  return 0;
}

/* gradient_norm(grads, max_norm, out, workspace, device, stream) */
static PyObject* gradient_norm(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  int32_t device;
  int kind = KIND_OTHER;
  double max_norm;
  void *work, *stream;
  size_t bytes;
  Py_ssize_t n;
  PyObject* seq;
  const void** grads;
  int64_t* numel;
  view out;
  char err[256] = "";
  int rc = 0, failed;
  NARGS(6);
  max_norm = PyFloat_AsDouble(a[1]);
  if (PyErr_Occurred()) return NULL;
  if (integer32(a[4], &device) || address(a[5], &stream) || want(a[2], "out", device, SASGD_FP32, 2, &out) || workspace_of(a[3], device, &work, &bytes)) return NULL;
  if (bytes < SASGD_NORM_WORKSPACE) {
    PyErr_Format(PyExc_ValueError, "gradientNorm needs a workspace of %d bytes", SASGD_NORM_WORKSPACE);
    return NULL;
  }
  seq = PySequence_Fast(a[0], "grads must be a sequence");
  if (!seq) return NULL;
  n = PySequence_Fast_GET_SIZE(seq);
  grads = (const void**)PyMem_Malloc(sizeof(void*) * (size_t)(n ? n : 1));
  numel = (int64_t*)PyMem_Malloc(sizeof(int64_t) * (size_t)(n ? n : 1));
  failed = !grads || !numel || n > INT32_MAX;
  if (failed) PyErr_NoMemory();
  else failed = list_of(seq, n, device, &kind, grads, 1, numel, sizeof(int64_t), 0);
  if (!failed) {
    /* (0 would stand for no bound) */
    const float bound = max_norm > 0 && (float)max_norm == 0.f ? FLT_TRUE_MIN : (float)max_norm;
    Py_BEGIN_ALLOW_THREADS
    rc = sasgd_gradientNorm(grads, numel, (int32_t)n, kind == KIND_OTHER ? SASGD_FP32 : kind, bound, (float*)out.data, work, stream, err, sizeof(err));
    Py_END_ALLOW_THREADS
  }
  Py_DECREF(seq);                     /* (it may be all that holds the gradients: a generator's) */
  PyMem_Free(grads);
  PyMem_Free(numel);
  if (failed) return NULL;
  if (rc) return raise_code(rc, err);
  Py_RETURN_NONE;
}

/* adamw_tensors(weights, outs, copies, device, tensors): fills the array of sasgd_tensor at `tensors` from lists of one length (an entry of copies may be
 * None); returns how many elements their moments have. */
static PyObject* adamw_tensors(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  int32_t device;
  void* to;
  int64_t elements_ = 0;
  Py_ssize_t n, k;
  NARGS(5);
  if (integer32(a[3], &device) || address(a[4], &to)) return NULL;
  if (!PyList_Check(a[0]) || !PyList_Check(a[1]) || !PyList_Check(a[2])) return PyErr_Format(PyExc_TypeError, "lists are needed");
  n = PyList_GET_SIZE(a[0]);
  if (PyList_GET_SIZE(a[1]) != n || PyList_GET_SIZE(a[2]) != n) return PyErr_Format(PyExc_ValueError, "outs and copies need an entry per tensor");
  for (k = 0; k < n; k++) {
    sasgd_tensor* t = (sasgd_tensor*)to + k;
    view w, o, c;
    if (want(PyList_GET_ITEM(a[0], k), "a weight", device, SASGD_FP32, 0, &w)) return NULL;
    t->numel = elements(&w);
    t->theta_in = (const float*)w.data;
    t->theta_out = (float*)w.data;
    t->shadow_out = NULL;
    if (PyList_GET_ITEM(a[1], k) != PyList_GET_ITEM(a[0], k)) {
      if (want(PyList_GET_ITEM(a[1], k), "an out", device, SASGD_FP32, t->numel, &o)) return NULL;
      t->theta_out = (float*)o.data;
    }
    if (PyList_GET_ITEM(a[2], k) != Py_None) {
      if (want(PyList_GET_ITEM(a[2], k), "a copy", device, SASGD_BF16, t->numel, &c)) return NULL;
      t->shadow_out = (uint16_t*)c.data;
    }
    elements_ += (t->numel + 255) / 256 * 256;
  }
  return PyLong_FromLongLong(elements_);
}

/* apply_adamw(rule, tensors, count, moments, grads, staleness, step, step_dev, factor, device, stream): rule, tensors and moments are addresses of the
 * C structures, grads a sequence of c sequences of `count` tensors; the rule's grad_type becomes theirs. */
static PyObject* apply_adamw(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  void *rule, *tensors, *moments, *step_dev, *stream;
  int32_t count, device, stale[SASGD_NOALLOC_MAX_GRADIENTS];
  int kind = KIND_OTHER, rc = 0, failed = 0;
  long long step;
  Py_ssize_t c, l, held = 0;
  PyObject *lists, *st, *one[SASGD_NOALLOC_MAX_GRADIENTS];      /* one[0 .. held): they may be all that holds the gradients */
  const void** grads;
  view factor;
  char err[256] = "";
  NARGS(11);
  if (address(a[0], &rule) || address(a[1], &tensors) || integer32(a[2], &count) || address(a[3], &moments) || integer(a[6], &step) ||
      address(a[7], &step_dev) || integer32(a[9], &device) || address(a[10], &stream))
    return NULL;
  factor.data = NULL;
  if (a[8] != Py_None && want(a[8], "scale", device, SASGD_FP32, 1, &factor)) return NULL;
  lists = PySequence_Fast(a[4], "grads must be a sequence of sequences");
  if (!lists) return NULL;
  st = PySequence_Fast(a[5], "staleness must be a sequence");
  if (!st) {
    Py_DECREF(lists);
    return NULL;
  }
  c = PySequence_Fast_GET_SIZE(lists);
  if (c < 1 || c > SASGD_NOALLOC_MAX_GRADIENTS || PySequence_Fast_GET_SIZE(st) != c) {
    Py_DECREF(lists);
    Py_DECREF(st);
    return raise_code(SASGD_EINVAL, "applyAdamW: 1..64 gradients and as many staleness values are needed");
  }
  for (l = 0; !failed && l < c; l++) failed = as_integer32(PySequence_Fast_GET_ITEM(st, l), &stale[l]);
  Py_DECREF(st);
  grads = failed ? NULL : (const void**)PyMem_Malloc(sizeof(void*) * (size_t)(count > 0 ? count : 1) * (size_t)c);
  if (!failed && !grads) {
    PyErr_NoMemory();
    failed = 1;
  }
  for (l = 0; !failed && l < c; l++) {
    one[l] = PySequence_Fast(PySequence_Fast_GET_ITEM(lists, l), "grads must be a sequence of sequences");
    if (!one[l]) {
      failed = 1;
      break;
    }
    held = l + 1;
    if (PySequence_Fast_GET_SIZE(one[l]) != count) {
      PyErr_SetString(PyExc_ValueError, "a gradient has another number of tensors than the weights");
      failed = 1;
    } else {
      failed = list_of(one[l], count, device, &kind, grads + l, (size_t)c, &((sasgd_tensor*)tensors)->numel, sizeof(sasgd_tensor), 1);
    }
  }
  if (!failed) {
    if (kind != KIND_OTHER) ((sasgd_adamw*)rule)->grad_type = kind;
    Py_BEGIN_ALLOW_THREADS
    rc = sasgd_applyAdamW((const sasgd_adamw*)rule, (const sasgd_tensor*)tensors, count, grads, (int32_t)c, stale, (const sasgd_moments*)moments, step,
                          (const int64_t*)step_dev, (const float*)factor.data, stream, err, sizeof(err));
    Py_END_ALLOW_THREADS
  }
  while (held > 0) {
    held--;
    Py_DECREF(one[held]);
  }
  Py_DECREF(lists);
  PyMem_Free(grads);
  if (failed) return NULL;
  if (rc) return raise_code(rc, err);
  Py_RETURN_NONE;
}

/* A tensor [images, ..., channels] as images of evenly spaced pixels with their channels side by side. */
static int pixels(const char* name, const view* v, int64_t* positions, int64_t* image, int64_t* pixel) {
  int k;
  const int last = v->dims - 1;
  *positions = 1;
  if (v->dims < 2) return bad(PyExc_ValueError, name, "must be [images, ..., channels]");
  *pixel = v->shape[last];
  if (v->shape[last] > 1 && v->stride[last] != 1) return bad(PyExc_ValueError, name, "must have its channels last, side by side");
  for (k = last - 1; k >= 1; k--) {
    if (v->shape[k] == 1) continue;
    if (*positions == 1) *pixel = v->stride[k];
    else if (v->stride[k] != *pixel * *positions) return bad(PyExc_ValueError, name, "must have its positions evenly apart");
    *positions *= v->shape[k];
  }
  *image = v->shape[0] > 1 ? v->stride[0] : *pixel * *positions;
  /* (a stride of 0 would stand for a dense tensor) */
  if ((*positions > 1 && *pixel < v->shape[last]) || (v->shape[0] > 1 && *image == 0)) return bad(PyExc_ValueError, name, "must not have its values in one place");
  return 0;
}
static int same_shape(const view* a, const view* b) {
  return a->dims == b->dims && a->kind == b->kind && memcmp(a->shape, b->shape, sizeof(int64_t) * (size_t)a->dims) == 0;
}

/* x, y (or dy; may be None), scale and shift (None: none) of a group normalisation, checked, and its shape. */
static int norm_shape(PyObject* ox, PyObject* oy, PyObject* oscale, PyObject* oshift, int32_t groups, int32_t activation, double eps, int device, view* x, view* y,
                      void** scale, void** shift, sasgd_norm_shape* s) {
  int64_t p;
  view v;
  int k, type = KIND_OTHER;
  PyObject* params[2] = {oscale, oshift};
  void** data[2] = {scale, shift};
  memset(s, 0, sizeof(*s));
  if (view_of(ox, x)) return -1;
  if (x->kind == KIND_OTHER) return bad(PyExc_TypeError, "x", "must be float32 or bfloat16");
  if (device >= 0 && x->device != device) return bad(PyExc_ValueError, "x", "is not on the current device");
  if (pixels("x", x, &s->positions, &s->x_image, &s->x_pixel)) return -1;
  if (oy != Py_None) {
    if (view_of(oy, y)) return -1;
    if (!same_shape(x, y)) return bad(PyExc_ValueError, "y", "must have the shape and the type of x");
    if (y->device != device) return bad(PyExc_ValueError, "y", "is not on the current device");
    if (pixels("y", y, &p, &s->y_image, &s->y_pixel)) return -1;
  }
  s->images = x->shape[0];
  s->channels = x->shape[x->dims - 1] > INT32_MAX ? INT32_MAX : (int32_t)x->shape[x->dims - 1];
  for (k = 0; k < 2; k++) {
    *data[k] = NULL;
    if (params[k] == Py_None) continue;
    if (want(params[k], "a parameter", device, KIND_OTHER, 0, &v)) return -1;
    if (elements(&v) != s->channels) return bad(PyExc_ValueError, "a parameter", "must have one value per channel");
    if (v.kind == KIND_OTHER || (type != KIND_OTHER && v.kind != type)) return bad(PyExc_TypeError, "scale and shift", "must both be float32 or both bfloat16");
    type = v.kind;
    *data[k] = v.data;
  }
  s->groups = groups;
  s->type = x->kind;
  s->param_type = type == KIND_OTHER ? SASGD_FP32 : type;
  s->activation = activation;
  s->eps = (float)eps;
  return 0;
}

/* group_norm_workspace(x, groups, gradient) */
static PyObject* group_norm_workspace(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  sasgd_norm_shape s;
  int32_t groups, gradient;
  void *scale, *shift;
  size_t bytes;
  view x, y;
  NARGS(3);
  if (integer32(a[1], &groups) || integer32(a[2], &gradient) || norm_shape(a[0], Py_None, Py_None, Py_None, groups, 0, 1.0, -1, &x, &y, &scale, &shift, &s)) return NULL;
  if (sasgd_groupNormWorkspace(&s, gradient, &bytes)) return raise_code(SASGD_EINVAL, "groupNormWorkspace: bad shape");
  return PyLong_FromSize_t(bytes);
}

/* group_norm(x, scale, shift, groups, y, stats, activation, eps, workspace, device, stream) */
static PyObject* group_norm(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  sasgd_norm_shape s;
  int32_t groups, activation, device;
  void *scale, *shift, *work, *stream;
  size_t bytes;
  double eps;
  view x, y, stats;
  char err[256] = "";
  int rc;
  NARGS(11);
  eps = PyFloat_AsDouble(a[7]);
  if (PyErr_Occurred()) return NULL;
  if (integer32(a[3], &groups) || integer32(a[6], &activation) || integer32(a[9], &device) || address(a[10], &stream)) return NULL;
  if (a[4] == Py_None) {
    PyErr_SetString(PyExc_TypeError, "y must be a tensor");
    return NULL;
  }
  if (norm_shape(a[0], a[4], a[1], a[2], groups, activation, eps, device, &x, &y, &scale, &shift, &s) || workspace_of(a[8], device, &work, &bytes)) return NULL;
  stats.data = NULL;
  if (a[5] != Py_None && want(a[5], "stats", device, SASGD_FP32, 2 * s.images * groups, &stats)) return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = sasgd_groupNorm(&s, x.data, scale, shift, y.data, (float*)stats.data, work, bytes, stream, err, sizeof(err));
  Py_END_ALLOW_THREADS
  if (rc) return raise_code(rc, err);
  Py_RETURN_NONE;
}

/* group_norm_gradient(x, scale, shift, groups, stats, dy, dx, dscale, dshift, activation, workspace, device, stream) */
static PyObject* group_norm_gradient(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  sasgd_norm_shape s;
  int32_t groups, activation, device;
  int64_t p, image, pixel;
  void *scale, *shift, *work, *stream;
  size_t bytes;
  view x, dy, stats, dx, dscale, dshift;
  char err[256] = "";
  int rc;
  NARGS(13);
  if (integer32(a[3], &groups) || integer32(a[9], &activation) || integer32(a[11], &device) || address(a[12], &stream)) return NULL;
  if (a[5] == Py_None) {
    PyErr_SetString(PyExc_TypeError, "dy must be a tensor");
    return NULL;
  }
  if (norm_shape(a[0], a[5], a[1], a[2], groups, activation, 1.0, device, &x, &dy, &scale, &shift, &s) || workspace_of(a[10], device, &work, &bytes) ||
      want(a[4], "stats", device, SASGD_FP32, 2 * s.images * groups, &stats))
    return NULL;
  dx.data = dscale.data = dshift.data = NULL;
  if (a[6] != Py_None) {
    if (view_of(a[6], &dx) || pixels("dx", &dx, &p, &image, &pixel)) return NULL;
    if (dx.device != device || !same_shape(&x, &dx) || image != s.y_image || pixel != s.y_pixel) {
      PyErr_SetString(PyExc_ValueError, "dx must have the shape, type and device of x and the strides of dy");
      return NULL;
    }
  }
  if ((a[7] != Py_None && want(a[7], "dscale", device, SASGD_FP32, s.channels, &dscale)) || (a[8] != Py_None && want(a[8], "dshift", device, SASGD_FP32, s.channels, &dshift)))
    return NULL;
  Py_BEGIN_ALLOW_THREADS
  rc = sasgd_groupNormGradient(&s, x.data, scale, shift, (const float*)stats.data, dy.data, dx.data, (float*)dscale.data, (float*)dshift.data, work, bytes, stream, err,
                               sizeof(err));
  Py_END_ALLOW_THREADS
  if (rc) return raise_code(rc, err);
  Py_RETURN_NONE;
}

/* set_tensor_class(torch.Tensor, torch.float32, torch.bfloat16) */
static PyObject* set_tensor_class(PyObject* self, PyObject* const* a, Py_ssize_t nargs) {
  NARGS(3);
  Py_INCREF(a[0]);
  Py_INCREF(a[1]);
  Py_INCREF(a[2]);
  tensor_class = a[0];
  fp32_type = a[1];
  bf16_type = a[2];
#ifdef SASGD_TORCH_TENSORS
  PyObject* capsule = PyObject_GetAttrString(a[0], "__dlpack_c_exchange_api__");
  if (capsule) {
    const DLPackExchangeAPI* api = (const DLPackExchangeAPI*)PyCapsule_GetPointer(capsule, "dlpack_exchange_api");
    if (api && api->header.version.major == DLPACK_MAJOR_VERSION && api->dltensor_from_py_object_no_sync) exchange = api;
    Py_DECREF(capsule);
  }
  PyErr_Clear();
#endif
  Py_RETURN_NONE;
}

static PyObject* set_error_class(PyObject* self, PyObject* cls) {
  Py_INCREF(cls);
  Py_XDECREF(error_class);
  error_class = cls;
  Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {FAST(get_minibatch),
                                FAST(pull_weights),
                                FAST(push_gradient),
                                FAST(push_gradient_external),
                                FAST(calc_gradient),
                                FAST(apply_update_no_alloc),
                                FAST(gradient_norm),
                                FAST(adamw_tensors),
                                FAST(apply_adamw),
                                FAST(group_norm_workspace),
                                FAST(group_norm),
                                FAST(group_norm_gradient),
                                FAST(set_tensor_class),
                                {"sum_gradients", sum_gradients, METH_O, NULL},
                                {"apply_update", apply_update, METH_O, NULL},
                                {"timestamp", timestamp, METH_O, NULL},
                                {"set_error_class", set_error_class, METH_O, NULL},
                                {NULL, NULL, 0, NULL}};

static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcalls", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fastcalls(void) {
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  s_ctypes = PyUnicode_InternFromString("ctypes");
  s_data = PyUnicode_InternFromString("data");
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_element_size = PyUnicode_InternFromString("element_size");
  s_get_device = PyUnicode_InternFromString("get_device");
  if (!s_data_ptr || !s_ctypes || !s_data || !s_dtype || !s_shape || !s_stride || !s_element_size || !s_get_device) return NULL;
  Py_INCREF(PyExc_RuntimeError);
  error_class = PyExc_RuntimeError;
  return PyModule_Create(&module);
}
