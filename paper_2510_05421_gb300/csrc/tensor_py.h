/* What the CPython modules of the bindings share: a look at a torch tensor
 * through its Python attributes (so that they know nothing of torch's C++
 * layout), and refusals as ValueErrors. */
#ifndef DVI_TENSOR_PY_H_
#define DVI_TENSOR_PY_H_

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/dvi.h"

static PyObject *g_i32, *g_f32, *g_bf16;                                  /* torch dtypes */
static PyObject *s_dtype, *s_shape, *s_stride, *s_get_device, *s_data_ptr; /* interned names */

typedef struct {
  PyObject* dtype;      /* borrowed: a torch dtype lives as long as torch */
  int dims;
  int64_t size[4], step[4];
  int64_t device;
  uintptr_t ptr;
} Tensor;

static int intern_names(void) {
  s_dtype = PyUnicode_InternFromString("dtype");
  s_shape = PyUnicode_InternFromString("shape");
  s_stride = PyUnicode_InternFromString("stride");
  s_get_device = PyUnicode_InternFromString("get_device");
  s_data_ptr = PyUnicode_InternFromString("data_ptr");
  if (!s_dtype || !s_shape || !s_stride || !s_get_device || !s_data_ptr) return 0;
  return 1;
}

static int ints_of(PyObject* tuple, int64_t* out, int want) {
  if (!PyTuple_Check(tuple) || (want >= 0 && PyTuple_GET_SIZE(tuple) != want) || PyTuple_GET_SIZE(tuple) > 4) return -1;
  const int n = (int)PyTuple_GET_SIZE(tuple);
  for (int i = 0; i < n; ++i) {
    out[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(tuple, i));
    if (out[i] == -1 && PyErr_Occurred()) return -1;
  }
  return n;
}

static int call_int(PyObject* o, PyObject* name, int64_t* out) {
  PyObject* r = PyObject_CallMethodNoArgs(o, name);
  if (!r) return 0;
  *out = (int64_t)PyLong_AsUnsignedLongLongMask(r);
  Py_DECREF(r);
  return !PyErr_Occurred();
}

/* What a tensor is; an AttributeError or the like passes through as it is. */
static int look(PyObject* o, const char* what, Tensor* t) {
  PyObject* r = PyObject_GetAttr(o, s_dtype);
  if (!r) return 0;
  t->dtype = r;
  Py_DECREF(r);
  r = PyObject_GetAttr(o, s_shape);
  if (!r) return 0;
  t->dims = ints_of(r, t->size, -1);
  Py_DECREF(r);
  if (t->dims >= 0) {
    r = PyObject_CallMethodNoArgs(o, s_stride);
    if (!r) return 0;
    if (ints_of(r, t->step, t->dims) < 0) t->dims = -1;
    Py_DECREF(r);
  }
  if (t->dims < 0) {
    if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "%s: too many dimensions", what);
    return 0;
  }
  int64_t p;
  if (!call_int(o, s_get_device, &t->device) || !call_int(o, s_data_ptr, &p)) return 0;
  t->ptr = (uintptr_t)p;
  return 1;
}

static int contiguous(const Tensor* t) {
  int64_t step = 1;
  for (int i = t->dims - 1; i >= 0; --i) {
    if (t->size[i] == 0) return 1;
    if (t->size[i] != 1 && t->step[i] != step) return 0;
    step *= t->size[i];
  }
  return 1;
}

static int refuse(const char* what, const char* why) {
  PyErr_Format(PyExc_ValueError, "%s: %s", what, why);
  return 0;
}

static int count(Py_ssize_t got, Py_ssize_t want) {
  if (got == want) return 1;
  PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, got);
  return 0;
}

#endif /* DVI_TENSOR_PY_H_ */
