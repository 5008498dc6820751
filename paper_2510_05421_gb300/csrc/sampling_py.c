/* CPython side of the page plans and of sampling (include/dvi.h): checks a
 * call's tensors, makes its outputs and the library call.  Like the paged cache's
 * (paged_py.c), and for the same reason: these calls take a few microseconds on the
 * GPU.  (Of verify_drafts' enqueueing, 9.7 us with Python around these checks: three
 * outputs 2.4, a launch 1.8, a look at a tensor 0.3.) */
#include "tensor_py.h"

typedef dvi_status (*probs_fn)(int, const void*, int64_t, int, int, const dvi_sampling*, float*, int64_t, int32_t*,
                               dvi_stream);
typedef dvi_status (*verify_fn)(const dvi_draft_batch*, const float*, int64_t, const float*, int64_t, int32_t*,
                                int32_t*, int32_t*, dvi_stream);
typedef dvi_status (*plan_fn)(const dvi_page_pool*, const int32_t*, const int32_t*, int, int, int32_t*, int64_t*,
                              int32_t*, dvi_stream);

static probs_fn g_probs;
static verify_fn g_verify;
static plan_fn g_plan;
static PyObject *g_i64, *g_empty, *g_error;

#define MAX_VOCAB (1 << 18)

/* f32 rows [n, vocab] that may lie apart: elements from row to row. */
static int are_rows(const char* what, const Tensor* t, int64_t n, int64_t vocab, int64_t device, int64_t* ld) {
  if (t->dtype != g_f32 || t->dims != 2 || t->size[0] != n || t->size[1] != vocab) {
    PyErr_Format(PyExc_ValueError, "%s must be float32 [%lld, %lld]", what, (long long)n, (long long)vocab);
    return 0;
  }
  if (t->device != device) return refuse(what, "not on the call's device");
  *ld = n <= 1 ? vocab : t->step[0];
  if (n && ((vocab > 1 && t->step[1] != 1) || *ld < vocab)) return refuse(what, "each row must be contiguous");
  return 1;
}
static int rows_of(const char* what, PyObject* o, int64_t n, int64_t vocab, int64_t device, uintptr_t* ptr,
                   int64_t* ld) {
  Tensor t;
  if (!look(o, what, &t) || !are_rows(what, &t, n, vocab, device, ld)) return 0;
  *ptr = t.ptr;
  return 1;
}

/* A contiguous array [n] of `dtype`. */
static int is_array(const char* what, const Tensor* t, PyObject* dtype, int64_t n, int64_t device) {
  if (t->dtype != dtype || t->dims != 1 || t->size[0] != n || !contiguous(t)) {
    PyErr_Format(PyExc_ValueError, "%s must be contiguous %s [%lld]", what, dtype == g_f32 ? "float32" : "int32",
                 (long long)n);
    return 0;
  }
  return t->device == device || refuse(what, "not on the call's device");
}
static int array_of(const char* what, PyObject* o, PyObject* dtype, int64_t n, int64_t device, uintptr_t* ptr) {
  Tensor t;
  if (!look(o, what, &t) || !is_array(what, &t, dtype, n, device)) return 0;
  *ptr = t.ptr;
  return 1;
}

/* A new contiguous tensor on the current device, [n] or (width >= 0) [n, width], and its address. */
static PyObject* new_tensor(int64_t n, int64_t width, PyObject* dtype, uintptr_t* ptr) {
  PyObject *size = width < 0 ? Py_BuildValue("(L)", (long long)n) : Py_BuildValue("(LL)", (long long)n, (long long)width);
  PyObject *step = width < 0 ? Py_BuildValue("(i)", 1) : Py_BuildValue("(Li)", (long long)width, 1);
  PyObject* t = NULL;
  int64_t p;
  if (size && step) {
    PyObject* args[3] = {size, step, dtype};
    t = PyObject_Vectorcall(g_empty, args, 3, NULL);
  }
  Py_XDECREF(size);
  Py_XDECREF(step);
  if (t && !call_int(t, s_data_ptr, &p)) Py_CLEAR(t);
  if (t) *ptr = (uintptr_t)p;
  return t;
}

/* `out` where the library took the call, else its error. */
static PyObject* result(const char* what, dvi_status rc, PyObject* out) {
  static const char* const names[] = {"DVI_OK", "DVI_ERR_INVALID_ARG", "DVI_ERR_CAPACITY", "DVI_ERR_NONFINITE",
                                      "DVI_ERR_CUDA", "DVI_ERR_UNIMPLEMENTED", "DVI_ERR_TIMEOUT"};
  if (rc == DVI_OK) return out;
  Py_XDECREF(out);
  if (rc < 0 && rc >= -6)
    PyErr_Format(g_error, "%s: %s", what, names[-rc]);
  else
    PyErr_Format(g_error, "%s: %d", what, (int)rc);
  return NULL;
}

/* A number, and a whole one (past 64 bits: the nearest), of any type that says it is one: numpy's scalars are not
 * Python's numbers. */
static int not_a_number(const char* what) {
  if (PyErr_ExceptionMatches(PyExc_TypeError) || PyErr_ExceptionMatches(PyExc_ValueError) ||
      PyErr_ExceptionMatches(PyExc_OverflowError)) {
    PyErr_Clear();
    refuse(what, "not a number that it may be");
  }
  return 0;
}
static int number_of(const char* what, PyObject* o, double* v) {
  *v = PyFloat_AsDouble(o);
  return !(*v == -1.0 && PyErr_Occurred()) || not_a_number(what);
}
static int whole_of(const char* what, PyObject* o, int64_t* v) {
  PyObject* i = PyNumber_Index(o);
  if (!i) return not_a_number(what);
  int past;
  *v = PyLong_AsLongLongAndOverflow(i, &past);
  Py_DECREF(i);
  if (past) *v = past > 0 ? INT64_MAX : INT64_MIN;
  return 1;
}
/* Whether a setting is a number (1) or a contiguous array [n] of `dtype`, one for each row (2); 0: refused.  Python's
 * own numbers first, then tensors: the others are found by not being one. */
static int setting_of(const char* what, PyObject* o, PyObject* dtype, int64_t n, int64_t device, uintptr_t* ptr) {
  if (dtype == g_f32 ? PyFloat_Check(o) || PyLong_Check(o) : PyLong_Check(o)) return 1;
  Tensor t;
  if (look(o, what, &t)) {
    *ptr = t.ptr;
    return is_array(what, &t, dtype, n, device) ? 2 : 0;
  }
  if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return 0;
  PyErr_Clear();
  const PyNumberMethods* m = Py_TYPE(o)->tp_as_number;
  if (m && (m->nb_index || (dtype == g_f32 && m->nb_float))) return 1;
  return refuse(what, dtype == g_f32 ? "must be a number or a tensor" : "must be a whole number or a tensor");
}

/* A device status word, or None. */
static int status_of(const char* what, PyObject* o, int64_t device, int32_t** out) {
  uintptr_t p = 0;
  if (o != Py_None && !array_of(what, o, g_i32, 1, device, &p)) return 0;
  *out = (int32_t*)p;
  return 1;
}

/* probs(logits, temperature, top_k, top_p, out or None, status, stream) -> out */
static PyObject* py_probs(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  if (!count(n_args, 7)) return NULL;
  Tensor t;
  if (!look(a[0], "token_probs: logits", &t)) return NULL;
  if ((t.dtype != g_f32 && t.dtype != g_bf16) || t.dims != 2 || t.size[1] < 1 || t.size[1] > MAX_VOCAB ||
      t.size[0] > (1 << 30)) {
    refuse("token_probs: logits", "must be float32 or bfloat16 [n, vocab], vocab 1 to 262144");
    return NULL;
  }
  if (t.device < 0) {
    refuse("token_probs: logits", "not on a CUDA device");
    return NULL;
  }
  const int64_t n = t.size[0], vocab = t.size[1], ld = n <= 1 ? vocab : t.step[0];
  if (n && ((vocab > 1 && t.step[1] != 1) || ld < vocab)) {
    refuse("token_probs: logits", "each row must be contiguous");
    return NULL;
  }
  uintptr_t out, p = 0;
  int64_t ld_out;
  dvi_sampling s = {NULL, NULL, NULL, 0.f, 0, 0.f};
  double v;
  int64_t k;
  int kind = setting_of("token_probs: temperature", a[1], g_f32, n, t.device, &p);
  if (!kind || (kind == 1 && !number_of("token_probs: temperature", a[1], &v))) return NULL;
  if (kind == 1) {
    if (!(v >= 0.0)) {
      refuse("token_probs", "temperature must be at least 0");
      return NULL;
    }
    /* (a temperature above 0 stays above it in f32) */
    s.temperature_all = v > 0.0 && v < 1e-37 ? 1e-37f : (float)v;
  }
  s.temperature = (const float*)p;
  p = 0;
  kind = setting_of("token_probs: top_k", a[2], g_i32, n, t.device, &p);
  if (!kind || (kind == 1 && !whole_of("token_probs: top_k", a[2], &k))) return NULL;
  if (kind == 1) {
    if (k < 0) {
      refuse("token_probs", "top_k must not be negative");
      return NULL;
    }
    s.top_k_all = k > MAX_VOCAB ? MAX_VOCAB : (int)k;
  }
  s.top_k = (const int32_t*)p;
  p = 0;
  kind = setting_of("token_probs: top_p", a[3], g_f32, n, t.device, &p);
  if (!kind || (kind == 1 && !number_of("token_probs: top_p", a[3], &v))) return NULL;
  if (kind == 1) {
    if (!(v >= 0.0)) {
      refuse("token_probs", "top_p must be at least 0");
      return NULL;
    }
    s.top_p_all = (float)v;
  }
  s.top_p = (const float*)p;
  int32_t* status;
  if (!status_of("token_probs: status", a[5], t.device, &status)) return NULL;
  dvi_stream stream = (dvi_stream)PyLong_AsVoidPtr(a[6]);
  if (PyErr_Occurred()) return NULL;
  PyObject* to;
  if (a[4] == Py_None) {
    to = new_tensor(n, vocab, g_f32, &out);
    if (!to) return NULL;
    ld_out = vocab;
  } else {
    if (!rows_of("token_probs: out", a[4], n, vocab, t.device, &out, &ld_out)) return NULL;
    to = Py_NewRef(a[4]);
  }
  const int type = t.dtype == g_f32 ? DVI_F32 : DVI_BF16;
  dvi_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_probs(type, (const void*)t.ptr, ld, (int)n, (int)vocab, &s, (float*)out, ld_out, status, stream);
  Py_END_ALLOW_THREADS
  return result("token_probs", rc, to);
}

/* verify(target, draft_ids, u_accept, u_token, draft, draft_start, max_drafts, bonus, status, stream)
 *   -> (ids, n_committed, n_accepted) */
static PyObject* py_verify(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  if (!count(n_args, 10)) return NULL;
  Tensor t, u, d;
  if (!look(a[0], "verify_drafts: target", &t) || !look(a[3], "verify_drafts: u_token", &u) ||
      !look(a[1], "verify_drafts: draft_ids", &d))
    return NULL;
  if (t.dtype != g_f32 || t.dims != 2 || t.size[1] < 1 || t.size[1] > MAX_VOCAB) {
    refuse("verify_drafts: target", "must be float32 [rows, vocab], vocab 1 to 262144");
    return NULL;
  }
  if (t.device < 0) {
    refuse("verify_drafts: target", "not on a CUDA device");
    return NULL;
  }
  if (u.dtype != g_f32 || u.dims != 1 || u.size[0] > (1 << 16)) {
    refuse("verify_drafts: u_token", "must be float32 [n_seqs], at most 65536 of them");
    return NULL;
  }
  if (d.dtype != g_i32 || d.dims != 1 || d.size[0] > (1 << 30)) {
    refuse("verify_drafts: draft_ids", "must be int32 [n_drafts]");
    return NULL;
  }
  const int64_t B = u.size[0], n = d.size[0], vocab = t.size[1];
  const int bonus = PyObject_IsTrue(a[7]);
  if (bonus < 0) return NULL;
  if (B == 0 && n) {
    refuse("verify_drafts", "drafts without a sequence");
    return NULL;
  }
  int64_t most = n;
  uintptr_t start = 0, ua, q = 0;
  int64_t ld_p, ld_q = 0;
  if (a[5] == Py_None) {
    if (B && n % B) {
      PyErr_Format(PyExc_ValueError, "verify_drafts: %lld drafts do not divide into %lld sequences (give draft_start)",
                   (long long)n, (long long)B);
      return NULL;
    }
    most = B ? n / B : 0;
  } else if (!array_of("verify_drafts: draft_start", a[5], g_i32, B + 1, t.device, &start)) {
    return NULL;
  }
  if (a[6] != Py_None) {
    int64_t m;
    if (!whole_of("verify_drafts: max_drafts", a[6], &m)) return NULL;
    if (m < 0 || (a[5] == Py_None && m < most)) {
      refuse("verify_drafts", "max_drafts must not be negative, nor below the drafts of each sequence");
      return NULL;
    }
    most = m;
  }
  if (most > (1 << 20)) {
    refuse("verify_drafts", "at most 2^20 drafts of a sequence (give max_drafts)");
    return NULL;
  }
  if (!are_rows("verify_drafts: target", &t, n + (bonus ? B : 0), vocab, t.device, &ld_p) ||
      !is_array("verify_drafts: draft_ids", &d, g_i32, n, t.device) ||
      !array_of("verify_drafts: u_accept", a[2], g_f32, n, t.device, &ua) ||
      !is_array("verify_drafts: u_token", &u, g_f32, B, t.device) ||
      (a[4] != Py_None && !rows_of("verify_drafts: draft", a[4], n, vocab, t.device, &q, &ld_q)))
    return NULL;
  int32_t* status;
  if (!status_of("verify_drafts: status", a[8], t.device, &status)) return NULL;
  dvi_stream stream = (dvi_stream)PyLong_AsVoidPtr(a[9]);
  if (PyErr_Occurred()) return NULL;
  PyObject* got = PyTuple_New(3);
  if (!got) return NULL;
  uintptr_t at[3];
  for (int i = 0; i < 3; ++i) {
    PyObject* o = new_tensor(B, i ? -1 : most + (bonus ? 1 : 0), g_i32, &at[i]);
    if (!o) {
      Py_DECREF(got);
      return NULL;
    }
    PyTuple_SET_ITEM(got, i, o);
  }
  const dvi_draft_batch b = {(int)B, (int)vocab, (int)n, (int)most, bonus ? 1 : 0, (const int32_t*)start,
                             (const int32_t*)d.ptr, (const float*)ua, (const float*)u.ptr, status};
  dvi_status rc;
  Py_BEGIN_ALLOW_THREADS
  /* (an empty tensor's rows need no memory, a drafter without rows is still one) */
  rc = g_verify(&b, (const float*)t.ptr, ld_p, n ? (const float*)q : NULL, ld_q, (int32_t*)at[0], (int32_t*)at[1],
                (int32_t*)at[2], stream);
  Py_END_ALLOW_THREADS
  return result("verify_drafts", rc, got);
}

/* plan(pool, device, lens, rows, n_rows or None, whether row starts are wanted, stream)
 *   -> (row_start, slots, positions), None for what is not wanted */
static PyObject* py_plan(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  if (!count(n_args, 7)) return NULL;
  const dvi_page_pool* pool = (const dvi_page_pool*)PyLong_AsVoidPtr(a[0]);
  const int64_t device = PyLong_AsLongLong(a[1]);
  if (PyErr_Occurred()) return NULL;
  const int64_t B = pool->n_seqs;
  int64_t each = 0, n_rows = 0;
  uintptr_t lens, rows = 0, at[3] = {0, 0, 0};
  if (!array_of("plan: lens", a[2], g_i32, B, device, &lens)) return NULL;
  const int kind = setting_of("plan: rows", a[3], g_i32, B, device, &rows);
  if (!kind || (kind == 1 && !whole_of("plan: rows", a[3], &each))) return NULL;
  if (kind == 1) {
    if (each < 0 || each > (1 << 30)) {
      refuse("plan", "rows must be 0 to 2^30");
      return NULL;
    }
  }
  if (a[4] != Py_None) {
    if (!whole_of("plan: n_rows", a[4], &n_rows)) return NULL;
    if (n_rows < 0 || n_rows > (1 << 30)) {
      refuse("plan", "n_rows must be 0 to 2^30");
      return NULL;
    }
  }
  const int starts = PyObject_IsTrue(a[5]);
  dvi_stream stream = (dvi_stream)PyLong_AsVoidPtr(a[6]);
  if (starts < 0 || PyErr_Occurred()) return NULL;
  PyObject* got = PyTuple_New(3);
  if (!got) return NULL;
  for (int i = 0; i < 3; ++i) {
    PyObject* o = Py_None;
    if (i == 0 ? starts : a[4] != Py_None) {
      o = new_tensor(i ? n_rows : B + 1, -1, i == 1 ? g_i64 : g_i32, &at[i]);
      if (!o) {
        Py_DECREF(got);
        return NULL;
      }
    } else {
      Py_INCREF(o);
    }
    PyTuple_SET_ITEM(got, i, o);
  }
  dvi_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_plan(pool, (const int32_t*)lens, (const int32_t*)rows, (int)each, (int)n_rows, (int32_t*)at[0],
              (int64_t*)at[1], (int32_t*)at[2], stream);
  Py_END_ALLOW_THREADS
  return result("plan", rc, got);
}

/* init(probs, verify, plan addresses, int32, int64, float32, bfloat16, a function (size, stride, dtype) that makes a
 *      tensor on the current device, the class of the library's errors) */
static PyObject* py_init(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  if (!count(n_args, 9)) return NULL;
  g_probs = (probs_fn)PyLong_AsVoidPtr(a[0]);
  g_verify = (verify_fn)PyLong_AsVoidPtr(a[1]);
  g_plan = (plan_fn)PyLong_AsVoidPtr(a[2]);
  if (PyErr_Occurred()) return NULL;
  g_i32 = Py_NewRef(a[3]);
  g_i64 = Py_NewRef(a[4]);
  g_f32 = Py_NewRef(a[5]);
  g_bf16 = Py_NewRef(a[6]);
  g_empty = Py_NewRef(a[7]);
  g_error = Py_NewRef(a[8]);
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"init", (PyCFunction)(void (*)(void))py_init, METH_FASTCALL, NULL},
                                {"plan", (PyCFunction)(void (*)(void))py_plan, METH_FASTCALL, NULL},
                                {"probs", (PyCFunction)(void (*)(void))py_probs, METH_FASTCALL, NULL},
                                {"verify", (PyCFunction)(void (*)(void))py_verify, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sampling", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__sampling(void) {
  if (!intern_names()) return NULL;
  return PyModule_Create(&module);
}
