/* CPython side of the paged cache's binding: checks a call's tensors and makes
 * the library call.  It does what ctypes and Python checks would do, in about
 * a third of their time: a decode step's calls are so short that the checks
 * bound them (one greedy token's attend: 9 us on the GPU, 11.5 us to enqueue
 * through ctypes).
 *
 * It does not link the library: init() gets the addresses of the entry points.
 * Every refusal is a ValueError, raised before the library is called.  Other
 * threads run while the library has a call: a launch waits where the GPU's queue
 * is full, perhaps for a host function in Python. */
#include "tensor_py.h"

typedef dvi_status (*append_fn)(const dvi_paged_cache*, const dvi_paged_batch*, int, const void*, int64_t,
                                const void*, int64_t, const float*, int, int, const void*, int64_t, void*, int64_t,
                                int, dvi_stream);
typedef dvi_status (*attend_fn)(const dvi_paged_cache*, const dvi_paged_batch*, const dvi_paged_options*, int,
                                const void*, int64_t, void*, int64_t, void*, size_t, dvi_stream);
typedef dvi_status (*read_fn)(const dvi_paged_cache*, const dvi_paged_batch*, int, void*, void*, dvi_stream);

typedef uint64_t (*capture_fn)(dvi_stream);

static append_fn g_append;
static attend_fn g_attend;
static read_fn g_read;
static capture_fn g_capture;

/* The cache a call is on. */
typedef struct {
  const dvi_paged_cache* c;
  int64_t device;
  int32_t* status;
} Cache;

static int cache_of(PyObject* address, PyObject* device, PyObject* status, Cache* c) {
  c->c = (const dvi_paged_cache*)PyLong_AsVoidPtr(address);
  c->device = PyLong_AsLongLong(device);
  c->status = (int32_t*)PyLong_AsVoidPtr(status);
  return !PyErr_Occurred();
}

static int batch_of(const Cache* c, const char* what, PyObject* table, PyObject* lens, int64_t n_rows,
                    PyObject* row_start, PyObject* max_rows, dvi_paged_batch* b) {
  Tensor t, l;
  if (!look(table, what, &t) || !look(lens, what, &l)) return 0;
  if (t.dtype != g_i32 || l.dtype != g_i32 || t.dims != 2 || l.dims != 1)
    return refuse(what, "table must be int32 [B, max_pages] and lens int32 [B]");
  const int64_t B = t.size[0], width = t.size[1];
  if (l.size[0] != B || !contiguous(&t) || !contiguous(&l))
    return refuse(what, "table and lens must be contiguous, with one row and one length a sequence");
  if (t.device != c->device || l.device != c->device) return refuse(what, "table and lens must be on the cache's device");
  if (B < 1 || B > 1024 || width < 1 || width > (1 << 30) / c->c->page_tokens)
    return refuse(what, "1 to 1024 sequences, tables of at most 2^30 positions");
  if (n_rows < 0 || n_rows > (1 << 30)) return refuse(what, "0 to 2^30 rows");
  int64_t most;
  uintptr_t start = 0;
  if (row_start == Py_None) {
    if (n_rows % B) {
      PyErr_Format(PyExc_ValueError, "%s: %lld rows do not divide into %lld sequences (give row_start)", what,
                   (long long)n_rows, (long long)B);
      return 0;
    }
    most = n_rows / B;
  } else {
    Tensor r;
    if (!look(row_start, what, &r)) return 0;
    if (r.dtype != g_i32 || r.dims != 1 || r.size[0] != B + 1 || !contiguous(&r) || r.device != c->device)
      return refuse(what, "row_start must be contiguous int32 [B + 1] on the cache's device");
    start = r.ptr;
    most = n_rows;
    if (max_rows != Py_None) {
      const int64_t m = PyLong_AsLongLong(max_rows);
      if (m == -1 && PyErr_Occurred()) return 0;
      if (m < 0) return refuse(what, "max_rows must not be negative");
      if (m < most) most = m;
    }
  }
  b->n_seqs = (int)B;
  b->max_pages = (int)width;
  b->n_rows = (int)n_rows;
  b->max_rows = (int)most;
  b->table = (const int32_t*)t.ptr;
  b->lens = (const int32_t*)l.ptr;
  b->row_start = (const int32_t*)start;
  b->status = c->status;
  return 1;
}

/* Rows [n_rows, heads, head_dim] of `dtype` whose rows may lie apart: elements from row to row. */
static int rows_of(const Cache* c, const char* what, PyObject* o, PyObject* dtype, int64_t n_rows, int64_t heads,
                   uintptr_t* ptr, int64_t* ld) {
  Tensor t;
  if (!look(o, what, &t)) return 0;
  const int64_t D = c->c->head_dim, esz = dtype == g_f32 ? 4 : 2;
  if (t.dtype != dtype || t.dims != 3 || t.size[0] != n_rows || t.size[1] != heads || t.size[2] != D) {
    PyErr_Format(PyExc_ValueError, "%s must be %s [%lld, %lld, %lld]", what, dtype == g_f32 ? "float32" : "bfloat16",
                 (long long)n_rows, (long long)heads, (long long)D);
    return 0;
  }
  *ld = n_rows <= 1 ? heads * D : t.step[0];
  if (t.step[2] != 1 || (heads > 1 && t.step[1] != D) || *ld < heads * D)
    return refuse(what, "each row's heads must be contiguous");
  if (t.device != c->device) return refuse(what, "not on the cache's device");
  if (t.ptr % 16 || *ld * esz % 16) return refuse(what, "rows must start on 16-byte boundaries");
  *ptr = t.ptr;
  return 1;
}

/* dtype, rows and heads of a call's first tensor. */
static int lead_of(const char* what, PyObject* o, PyObject** dtype, int64_t* n, int64_t* heads) {
  PyObject* r = PyObject_GetAttr(o, s_dtype);
  if (!r) return 0;
  *dtype = r;
  Py_DECREF(r);
  int64_t size[4];
  r = PyObject_GetAttr(o, s_shape);
  if (!r) return 0;
  const int dims = ints_of(r, size, -1);
  Py_DECREF(r);
  if ((*dtype != g_bf16 && *dtype != g_f32) || dims != 3) {
    PyErr_Clear();
    return refuse(what, "must be bfloat16 or float32 [n, heads, head_dim]");
  }
  *n = size[0];
  *heads = size[1];
  return 1;
}

/* append(cache, device, status, table, lens, k, v, q, rotary, row_start, max_rows, q_out, stream) -> status */
static PyObject* py_append(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  Cache c;
  dvi_paged_batch b;
  PyObject* dtype;
  int64_t n, H, heads = 0, ld_k, ld_v, ld_q = 0, ld_o = 0, rot_dim = 0, n_pos = 0;
  uintptr_t k, v, q = 0, o = 0, rot = 0;
  if (!count(n_args, 13) || !cache_of(a[0], a[1], a[2], &c) || !lead_of("append: k", a[5], &dtype, &n, &H) ||
      !batch_of(&c, "append", a[3], a[4], n, a[9], a[10], &b) ||
      !rows_of(&c, "append: k", a[5], dtype, n, c.c->n_kv_heads, &k, &ld_k) ||
      !rows_of(&c, "append: v", a[6], dtype, n, c.c->n_kv_heads, &v, &ld_v))
    return NULL;
  if (a[8] != Py_None) {
    Tensor t;
    if (!look(a[8], "append: rotary", &t)) return NULL;
    if (t.dtype != g_f32 || t.dims != 3 || t.size[2] != 2 || !contiguous(&t) || t.device != c.device || t.ptr % 16 ||
        t.size[0] < 1 || t.size[0] > (1 << 30)) {
      refuse("append: rotary", "must be contiguous float32 [n_pos, rot_dim / 2, 2] on the cache's device");
      return NULL;
    }
    n_pos = t.size[0];
    rot_dim = 2 * t.size[1];
    if (rot_dim % 16 || rot_dim < 16 || rot_dim > c.c->head_dim) {
      refuse("append: rotary", "rot_dim must be a multiple of 16 up to head_dim");
      return NULL;
    }
    rot = t.ptr;
  }
  if (a[7] != Py_None) {
    PyObject* qt;
    int64_t qn;
    if (!lead_of("append: q", a[7], &qt, &qn, &heads)) return NULL;
    if (heads < 1 || a[11] == Py_None) {
      refuse("append: q", "no heads, or no q_out");
      return NULL;
    }
    if (!rows_of(&c, "append: q", a[7], dtype, n, heads, &q, &ld_q) ||
        !rows_of(&c, "append: q_out", a[11], dtype, n, heads, &o, &ld_o))
      return NULL;
  } else if (a[11] != Py_None) {
    refuse("append", "q_out without q");
    return NULL;
  }
  dvi_stream stream = (dvi_stream)PyLong_AsVoidPtr(a[12]);
  if (PyErr_Occurred()) return NULL;
  const int type = dtype == g_f32 ? DVI_F32 : DVI_BF16;
  dvi_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_append(c.c, &b, type, (const void*)k, ld_k, (const void*)v, ld_v, (const float*)rot, (int)rot_dim, (int)n_pos,
                (const void*)q, ld_q, (void*)o, ld_o, (int)heads, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* attend(cache, device, status, table, lens, q, out, scale, softcap, window, slopes, row_start, max_rows, workspace,
 *        bytes, stream) -> status */
static PyObject* py_attend(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  Cache c;
  dvi_paged_batch b;
  dvi_paged_options op;
  PyObject* dtype;
  int64_t n, heads, ld_q, ld_o;
  uintptr_t q, o;
  if (!count(n_args, 16) || !cache_of(a[0], a[1], a[2], &c) || !lead_of("attend: q", a[5], &dtype, &n, &heads))
    return NULL;
  if (heads < 1 || heads % c.c->n_kv_heads || heads > (1 << 16)) {
    refuse("attend", "the query heads do not divide over the KV heads");
    return NULL;
  }
  if (!batch_of(&c, "attend", a[3], a[4], n, a[11], a[12], &b) ||
      !rows_of(&c, "attend: q", a[5], dtype, n, heads, &q, &ld_q) ||
      !rows_of(&c, "attend: out", a[6], dtype, n, heads, &o, &ld_o))
    return NULL;
  const double scale = PyFloat_AsDouble(a[7]), softcap = PyFloat_AsDouble(a[8]);
  const int64_t window = PyLong_AsLongLong(a[9]);
  if (PyErr_Occurred()) return NULL;
  if (!((float)scale > 0.f && scale < 1e30) || !(softcap >= 0.0 && softcap < 1e30) || window < 0 || window > 0x7fffffff) {
    refuse("attend", "needs scale > 0, softcap >= 0 and window >= 0");
    return NULL;
  }
  if (softcap > 0.0 && !(scale / softcap < 1e30)) {
    refuse("attend", "softcap must be 0 or more than 1e-30 of scale");
    return NULL;
  }
  op.n_heads = (int)heads;
  op.scale = (float)scale;
  op.softcap = (float)softcap;
  op.window = (int)window;
  op.slopes = NULL;
  if (a[10] != Py_None) {
    Tensor t;
    if (!look(a[10], "attend: slopes", &t)) return NULL;
    if (t.dtype != g_f32 || t.dims != 1 || t.size[0] != heads || !contiguous(&t) || t.device != c.device) {
      refuse("attend: slopes", "must be contiguous float32 [H_q] on the cache's device");
      return NULL;
    }
    op.slopes = (const float*)t.ptr;
  }
  void* ws = PyLong_AsVoidPtr(a[13]);
  const size_t bytes = PyLong_AsSize_t(a[14]);
  dvi_stream stream = (dvi_stream)PyLong_AsVoidPtr(a[15]);
  if (PyErr_Occurred()) return NULL;
  const int type = dtype == g_f32 ? DVI_F32 : DVI_BF16;
  dvi_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_attend(c.c, &b, &op, type, (const void*)q, ld_q, (void*)o, ld_o, ws, bytes, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* read(cache, device, status, table, lens, k_out, v_out, row_start, max_rows, stream) -> status */
static PyObject* py_read(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  Cache c;
  dvi_paged_batch b;
  PyObject* dtype;
  int64_t n, H, ld;
  uintptr_t k, v;
  if (!count(n_args, 10) || !cache_of(a[0], a[1], a[2], &c) || !lead_of("read: k", a[5], &dtype, &n, &H) ||
      !batch_of(&c, "read", a[3], a[4], n, a[7], a[8], &b) ||
      !rows_of(&c, "read: k", a[5], dtype, n, c.c->n_kv_heads, &k, &ld) ||
      !rows_of(&c, "read: v", a[6], dtype, n, c.c->n_kv_heads, &v, &ld))
    return NULL;
  dvi_stream stream = (dvi_stream)PyLong_AsVoidPtr(a[9]);
  if (PyErr_Occurred()) return NULL;
  const int type = dtype == g_f32 ? DVI_F32 : DVI_BF16;
  dvi_status rc;
  Py_BEGIN_ALLOW_THREADS
  rc = g_read(c.c, &b, type, (void*)k, (void*)v, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(rc);
}

/* capture(stream) -> the id of the capture it is in, 0 if it is in none */
static PyObject* py_capture(PyObject* self, PyObject* stream) {
  (void)self;
  dvi_stream s = (dvi_stream)PyLong_AsVoidPtr(stream);
  if (PyErr_Occurred()) return NULL;
  return PyLong_FromUnsignedLongLong(g_capture ? g_capture(s) : 0);
}

/* init(append, attend, read addresses, int32, float32, bfloat16[, capture address]) */
static PyObject* py_init(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
  (void)self;
  if (n_args != 7 && !count(n_args, 6)) return NULL;
  g_append = (append_fn)PyLong_AsVoidPtr(a[0]);
  g_attend = (attend_fn)PyLong_AsVoidPtr(a[1]);
  g_read = (read_fn)PyLong_AsVoidPtr(a[2]);
  g_capture = n_args == 7 ? (capture_fn)PyLong_AsVoidPtr(a[6]) : NULL;
  if (PyErr_Occurred()) return NULL;
  g_i32 = Py_NewRef(a[3]);
  g_f32 = Py_NewRef(a[4]);
  g_bf16 = Py_NewRef(a[5]);
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"init", (PyCFunction)(void (*)(void))py_init, METH_FASTCALL, NULL},
                                {"append", (PyCFunction)(void (*)(void))py_append, METH_FASTCALL, NULL},
                                {"attend", (PyCFunction)(void (*)(void))py_attend, METH_FASTCALL, NULL},
                                {"capture", py_capture, METH_O, NULL},
                                {"read", (PyCFunction)(void (*)(void))py_read, METH_FASTCALL, NULL},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__paged(void) {
  if (!intern_names()) return NULL;
  return PyModule_Create(&module);
}
