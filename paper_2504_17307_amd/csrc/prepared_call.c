/* One marshalled call of the C ABI as a Python object: calling it makes that call again (uccl_prepare).  A call of
 * few small messages is bound by the host, and ctypes spends a seventh of it on taking C arguments out of their objects
 * and putting them into a frame each time.  Here they lie ready (loops of prepared calls, us each, by ctypes / here /
 * the same loop in C: a reset 3.02 / 2.76 / 2.68, 14 records of 4 KiB 3.73 / 3.45 / 3.34, or in a process in which HIP
 * launches faster 2.49 / 2.26 / 2.18 and 2.81 / 2.36 / 2.28; a call of no records 0.10). */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stddef.h>
#include <stdint.h>
#include <structmember.h>

enum { MOST = 13 };

typedef struct {
  PyObject_HEAD
  vectorcallfunc call;
  void* fn;
  int n;
  uint64_t a[MOST];
  PyObject *failed, *keeps;   /* called with a code other than 0; what the caller gave */
  PyObject *holds, *name;     /* what else the arguments point into; of the function (either may be NULL) */
  PyObject *dict, *weak;
} Prepared;

/* Every argument of the ABI's functions is a pointer or a whole number of at most 64 bits: each takes one integer
 * register or one 8-byte stack slot of the x86-64 System V convention, of which the callee reads as much as its
 * type has. */
#if !defined(__x86_64__) || defined(_WIN32)
#error "prepared calls rely on the x86-64 System V calling convention"
#endif
typedef uint64_t W;
static int invoke(const Prepared* p) {
  const W* a = p->a;
  void* f = p->fn;
  switch (p->n) {
    case 0: return ((int (*)(void))f)();
    case 1: return ((int (*)(W))f)(a[0]);
    case 2: return ((int (*)(W, W))f)(a[0], a[1]);
    case 3: return ((int (*)(W, W, W))f)(a[0], a[1], a[2]);
    case 4: return ((int (*)(W, W, W, W))f)(a[0], a[1], a[2], a[3]);
    case 5: return ((int (*)(W, W, W, W, W))f)(a[0], a[1], a[2], a[3], a[4]);
    case 6: return ((int (*)(W, W, W, W, W, W))f)(a[0], a[1], a[2], a[3], a[4], a[5]);
    case 7: return ((int (*)(W, W, W, W, W, W, W))f)(a[0], a[1], a[2], a[3], a[4], a[5], a[6]);
    case 8: return ((int (*)(W, W, W, W, W, W, W, W))f)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]);
    case 9: return ((int (*)(W, W, W, W, W, W, W, W, W))f)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8]);
    case 10: return ((int (*)(W, W, W, W, W, W, W, W, W, W))f)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9]);
    case 11: return ((int (*)(W, W, W, W, W, W, W, W, W, W, W))f)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10]);
    case 12: return ((int (*)(W, W, W, W, W, W, W, W, W, W, W, W))f)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11]);
    default: return ((int (*)(W, W, W, W, W, W, W, W, W, W, W, W, W))f)(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11], a[12]);
  }
}

static PyObject* prepared_vectorcall(PyObject* self, PyObject* const* args, size_t nargsf, PyObject* names) {
  (void)args;
  if (PyVectorcall_NARGS(nargsf) != 0 || (names != NULL && PyTuple_GET_SIZE(names) != 0)) {
    PyErr_SetString(PyExc_TypeError, "a prepared call takes no arguments");
    return NULL;
  }
  const Prepared* const p = (const Prepared*)self;
  int code;
  Py_BEGIN_ALLOW_THREADS   /* a launch may wait for room in its stream's queue */
  code = invoke(p);
  Py_END_ALLOW_THREADS
  if (code != 0) {
    PyObject* const r = PyObject_CallFunction(p->failed, "i", code);
    Py_XDECREF(r);
    if (r == NULL) return NULL;
  }
  Py_RETURN_NONE;
}

static PyObject* prepared_new(PyTypeObject* type, PyObject* args, PyObject* kw) {
  unsigned long long fn;
  PyObject *values, *failed, *keeps, *holds = NULL, *name = NULL;
  if (kw != NULL && PyDict_GET_SIZE(kw) != 0) {
    PyErr_SetString(PyExc_TypeError, "no keyword arguments");
    return NULL;
  }
  if (!PyArg_ParseTuple(args, "KO!OO|OO", &fn, &PyTuple_Type, &values, &failed, &keeps, &holds, &name)) return NULL;
  const Py_ssize_t n = PyTuple_GET_SIZE(values);
  if (fn == 0 || n > MOST || !PyCallable_Check(failed)) {
    PyErr_SetString(PyExc_ValueError, "a function's address, at most 13 whole numbers, a callable and what to keep");
    return NULL;
  }
  Prepared* const p = (Prepared*)type->tp_alloc(type, 0);
  if (p == NULL) return NULL;
  p->call = prepared_vectorcall;
  p->fn = (void*)(uintptr_t)fn;
  p->n = (int)n;
  Py_INCREF(failed);
  p->failed = failed;
  Py_INCREF(keeps);
  p->keeps = keeps;
  Py_XINCREF(holds);
  p->holds = holds;
  Py_XINCREF(name);
  p->name = name;
  for (Py_ssize_t i = 0; i < n; ++i) {
    p->a[i] = PyLong_AsUnsignedLongLongMask(PyTuple_GET_ITEM(values, i));
    if (PyErr_Occurred()) {
      Py_DECREF(p);
      return NULL;
    }
  }
  return (PyObject*)p;
}

static int prepared_traverse(PyObject* self, visitproc visit, void* arg) {
  Py_VISIT(((Prepared*)self)->failed);
  Py_VISIT(((Prepared*)self)->keeps);
  Py_VISIT(((Prepared*)self)->holds);
  Py_VISIT(((Prepared*)self)->name);
  Py_VISIT(((Prepared*)self)->dict);
  return 0;
}
static int prepared_clear(PyObject* self) {
  Py_CLEAR(((Prepared*)self)->failed);
  Py_CLEAR(((Prepared*)self)->keeps);
  Py_CLEAR(((Prepared*)self)->holds);
  Py_CLEAR(((Prepared*)self)->name);
  Py_CLEAR(((Prepared*)self)->dict);
  return 0;
}
static void prepared_dealloc(PyObject* self) {
  PyObject_GC_UnTrack(self);
  if (((Prepared*)self)->weak != NULL) PyObject_ClearWeakRefs(self);
  prepared_clear(self);
  Py_TYPE(self)->tp_free(self);
}

static PyMemberDef members[] = {{"keeps", T_OBJECT_EX, offsetof(Prepared, keeps), READONLY, NULL},
                                {"__name__", T_OBJECT_EX, offsetof(Prepared, name), 0, NULL},
                                {NULL, 0, 0, 0, NULL}};
static PyGetSetDef getset[] = {{"__dict__", PyObject_GenericGetDict, PyObject_GenericSetDict, NULL, NULL}, {NULL, NULL, NULL, NULL, NULL}};
static PyTypeObject prepared_type = {
    PyVarObject_HEAD_INIT(NULL, 0).tp_name = "paper_2504_17307_amd._prepared.Prepared",
    .tp_basicsize = sizeof(Prepared),
    .tp_dealloc = prepared_dealloc,
    .tp_vectorcall_offset = offsetof(Prepared, call),
    .tp_call = PyVectorcall_Call,
    .tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_GC | Py_TPFLAGS_HAVE_VECTORCALL,
    .tp_traverse = prepared_traverse,
    .tp_clear = prepared_clear,
    .tp_members = members,
    .tp_getset = getset,
    .tp_dictoffset = offsetof(Prepared, dict),
    .tp_weaklistoffset = offsetof(Prepared, weak),
    .tp_new = prepared_new,
};
/* Tensors as arguments of the row operators: asking one for its address, sizes and type through the interpreter takes 0.1 us each, and a call has
 * several, or a list of hundreds (uccl_gradient_norm, uccl_gradient_clip).  The DLPack standard's table of C functions (its version 1, which tensor types offer as
 * __dlpack_c_exchange_api__) has one that fills in a struct for a tensor.  300 tensors: 18 us so, 1400 in Python. */
typedef struct { int32_t type, id; } DlDevice;
typedef struct { uint8_t code, bits; uint16_t lanes; } DlType;
typedef struct {
  void* data;
  DlDevice device;
  int32_t ndim;
  DlType dtype;
  int64_t *shape, *strides;
  uint64_t byte_offset;
} DlTensor;
typedef struct {
  uint32_t major, minor;
  void* previous;
  void *allocate, *managed_from_object, *managed_to_object;   /* not used here */
  int (*tensor_from_object)(void* object, DlTensor* out);     /* what it points to is the object's */
} DlFunctions;
typedef struct { uint64_t data, stride, scales, scale_stride; uint32_t rows, cols, dtype, reserved; } RowsStruct;   /* uccl_rows */

static int contiguous(const DlTensor* t, int64_t* n) {
  int64_t all = 1;
  int dense = 1;
  for (int32_t i = t->ndim - 1; i >= 0; --i) {
    if (t->shape[i] != 1 && t->strides != NULL && t->strides[i] != all) dense = 0;
    if (t->shape[i] != 0 && all > INT64_MAX / t->shape[i]) return 0;
    all *= t->shape[i];
  }
  *n = all;
  return dense || all == 0;
}

static const DlFunctions* functions;
static PyTypeObject* tensor_types[2];   /* torch.Tensor and torch.nn.Parameter: what another object would be taken for is not known */

/* read_tensors(functions, torch.Tensor, torch.nn.Parameter): whether tensors can be read by the functions below. */
static PyObject* read_tensors(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
  (void)self;
  functions = NULL;
  if (n_args != 3 || !PyCapsule_CheckExact(args[0]) || !PyType_Check(args[1]) || !PyType_Check(args[2])) Py_RETURN_FALSE;
  const DlFunctions* const f = (const DlFunctions*)PyCapsule_GetPointer(args[0], PyCapsule_GetName(args[0]));
  if (f == NULL) return NULL;
  if (f->major != 1 || f->tensor_from_object == NULL) Py_RETURN_FALSE;
  for (int i = 0; i < 2; ++i) {
    Py_INCREF(args[i + 1]);
    Py_XDECREF(tensor_types[i]);
    tensor_types[i] = (PyTypeObject*)args[i + 1];
  }
  Py_INCREF(args[0]);   /* for the process's life */
  functions = f;
  Py_RETURN_TRUE;
}

static int read_tensor(PyObject* object, DlTensor* t) {
  if (functions == NULL || (Py_TYPE(object) != tensor_types[0] && Py_TYPE(object) != tensor_types[1])) return 0;
  if (functions->tensor_from_object(object, t) == 0) return 1;
  PyErr_Clear();
  return 0;
}

static int rows_of_contiguous(const DlTensor* t, int64_t most, RowsStruct* out) {
  int64_t elements;
  const int f32 = t->dtype.code == 2 && t->dtype.bits == 32, f16 = t->dtype.code == 2 && t->dtype.bits == 16, bf16 = t->dtype.code == 4 && t->dtype.bits == 16;
  if (!(f32 || f16 || bf16) || t->dtype.lanes != 1 || !contiguous(t, &elements) || elements > most) return 0;
  *out = (RowsStruct){(uint64_t)(uintptr_t)t->data + t->byte_offset, (uint64_t)(elements == 0 ? 1 : elements) * (t->dtype.bits / 8), 0, 0, 1, (uint32_t)elements, f32 ? 0u : bf16 ? 1u : 2u, 0};
  return 1;
}

/* contiguous_rows(tensors, like, most): the bytes of one uccl_rows for every tensor of the first list, and for those of the second (the same list: the same bytes), or None: one
 * of them is not contiguous, of a type without rows, of more than `most` elements, or not of the shape and type of the one beside it. */
static PyObject* contiguous_rows(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
  (void)self;
  if (n_args != 3 || !PyList_CheckExact(args[0]) || !PyList_CheckExact(args[1])) Py_RETURN_NONE;
  const long long most = PyLong_AsLongLong(args[2]);
  if (PyErr_Occurred()) return NULL;
  const Py_ssize_t n = PyList_GET_SIZE(args[0]);
  const int same = args[0] == args[1];
  if (PyList_GET_SIZE(args[1]) != n) Py_RETURN_NONE;
  PyObject* const first = PyBytes_FromStringAndSize(NULL, n * (Py_ssize_t)sizeof(RowsStruct));
  PyObject* const second = same ? first : PyBytes_FromStringAndSize(NULL, n * (Py_ssize_t)sizeof(RowsStruct));
  if (same) Py_XINCREF(second);
  int fits = first != NULL && second != NULL;
  for (Py_ssize_t i = 0; fits && i < n; ++i) {
    DlTensor t, u;
    fits = read_tensor(PyList_GET_ITEM(args[0], i), &t) && rows_of_contiguous(&t, most, (RowsStruct*)PyBytes_AS_STRING(first) + i);
    if (fits && !same) {
      fits = read_tensor(PyList_GET_ITEM(args[1], i), &u) && rows_of_contiguous(&u, most, (RowsStruct*)PyBytes_AS_STRING(second) + i) && u.ndim == t.ndim && u.dtype.code == t.dtype.code &&
             u.dtype.bits == t.dtype.bits;
      for (int32_t d = 0; fits && d < t.ndim; ++d) fits = u.shape[d] == t.shape[d];
    }
  }
  PyObject* const both = fits ? PyTuple_Pack(2, first, second) : NULL;
  const int failed = first == NULL || second == NULL || (fits && both == NULL);
  Py_XDECREF(first);
  Py_XDECREF(second);
  if (failed) return NULL;
  if (both != NULL) return both;
  Py_RETURN_NONE;
}

/* vector_address(tensor, whether it is float32 and not int32, elements): where it is, or None: it is not contiguous, of another type or length. */
static PyObject* vector_address(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
  (void)self;
  DlTensor t;
  int64_t elements;
  if (n_args != 3 || !read_tensor(args[0], &t) || t.dtype.bits != 32 || t.dtype.lanes != 1 || t.dtype.code != (args[1] == Py_True ? 2 : 0) || !contiguous(&t, &elements) ||
      elements != PyLong_AsLongLong(args[2])) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  return PyLong_FromUnsignedLongLong((uint64_t)(uintptr_t)t.data + t.byte_offset);
}

/* matrix_rows(tensor): the bytes of its uccl_rows, or None: it is of a type with scales, or not a matrix by rows of fewer than 2^32 rows and columns. */
static PyObject* matrix_rows(PyObject* self, PyObject* const* args, Py_ssize_t n_args) {
  (void)self;
  DlTensor t;
  if (n_args == 1 && read_tensor(args[0], &t) && t.strides != NULL && t.dtype.lanes == 1 && (t.ndim == 2 || t.ndim == 3)) {
    const int f32 = t.dtype.code == 2 && t.dtype.bits == 32, f16 = t.dtype.code == 2 && t.dtype.bits == 16, bf16 = t.dtype.code == 4 && t.dtype.bits == 16;
    const int64_t groups = t.ndim == 3 ? t.shape[0] : 1, each = t.shape[t.ndim - 2], cols = t.shape[t.ndim - 1], last = t.strides[t.ndim - 1];
    int64_t step = t.strides[t.ndim - 2];
    const int small = groups <= 0xFFFFFFFF && each <= 0xFFFFFFFF && cols <= 0xFFFFFFFF && (each == 0 || groups <= 0xFFFFFFFF / each);
    int fits = small && (f32 || f16 || bf16) && (last == 1 || cols <= 1);
    if (fits && t.ndim == 3) {
      if (each == 1) step = t.strides[0];
      else if (groups > 1 && each != 0 && cols != 0 && t.strides[0] != each * step) fits = 0;
    }
    if (fits && step >= 0) {
      const RowsStruct r = {(uint64_t)(uintptr_t)t.data + t.byte_offset, (uint64_t)step * (t.dtype.bits / 8), 0, 0, (uint32_t)(groups * each), (uint32_t)cols, f32 ? 0u : bf16 ? 1u : 2u, 0};
      return PyBytes_FromStringAndSize((const char*)&r, sizeof r);
    }
  }
  Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"read_tensors", (PyCFunction)(void (*)(void))read_tensors, METH_FASTCALL, NULL},
                                {"vector_address", (PyCFunction)(void (*)(void))vector_address, METH_FASTCALL, NULL},
                                {"matrix_rows", (PyCFunction)(void (*)(void))matrix_rows, METH_FASTCALL, NULL},
                                {"contiguous_rows", (PyCFunction)(void (*)(void))contiguous_rows, METH_FASTCALL, NULL}, {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_prepared", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__prepared(void) {
  if (PyType_Ready(&prepared_type) < 0) return NULL;
  PyObject* const m = PyModule_Create(&module);
  if (m == NULL) return NULL;
  Py_INCREF(&prepared_type);
  if (PyModule_AddObject(m, "Prepared", (PyObject*)&prepared_type) < 0) {
    Py_DECREF(&prepared_type);
    Py_DECREF(m);
    return NULL;
  }
  return m;
}
