/* The check of one tensor argument, for binding.py, six or so of which a call makes: 0.6 us each in Python, 0.22 here.  A
 * client-server cycle (19 calls, 25 launches), which the host bounds: 151 -> 146 us enqueued and in all, of which the GPU needs
 * 96 when it never waits.  The stable CPython API; whatever the tensor's
 * attributes say, they say here as they would there. */
#define PY_SSIZE_T_CLEAN
#define Py_LIMITED_API 0x030a0000      /* CPython 3.10 and later load the same file */
#include <Python.h>

static PyObject *tensor_type, *s_is_cuda, *s_is_contiguous, *s_dtype, *s_numel, *s_data_ptr;
static PyObject *s_get_device, *s_element_size, *s_shape, *s_stride;
static PyObject *is_contiguous, *numel, *data_ptr, *get_device, *element_size, *stride_of;     /* torch.Tensor's own, for what is no subclass of it */

static PyObject *call(PyObject *t, int plain, PyObject *method, PyObject *name)
{
    return plain ? PyObject_CallFunctionObjArgs(method, t, NULL) : PyObject_CallMethodObjArgs(t, name, NULL);
}

/* 1, 0, or -1 with an exception */
static int truth(PyObject *o)
{
    if (!o) return -1;
    const int r = PyObject_IsTrue(o);
    Py_DECREF(o);
    return r;
}

/* dev(tensor or None, dtype, numel, name) -> address or None: a contiguous CUDA tensor of that type with at least that many elements */
static PyObject *dev(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 4) return PyErr_Format(PyExc_TypeError, "dev: 4 arguments expected, not %zd", n);
    PyObject *t = args[0], *name = args[3];
    if (t == Py_None) Py_RETURN_NONE;
    const int plain = (PyObject *)Py_TYPE(t) == tensor_type;
    if (!plain) {
        const int is = PyObject_IsInstance(t, tensor_type);
        if (is < 0) return NULL;
        if (!is) return PyErr_Format(PyExc_TypeError, "%S: expected a torch tensor", name);
    }
    int ok = truth(PyObject_GetAttr(t, s_is_cuda));
    if (ok > 0) ok = truth(call(t, plain, is_contiguous, s_is_contiguous));
    if (ok < 0) return NULL;
    if (!ok) return PyErr_Format(PyExc_ValueError, "%S: must be a contiguous CUDA tensor", name);
    PyObject *dtype = PyObject_GetAttr(t, s_dtype);
    if (!dtype) return NULL;
    if (dtype != args[1]) {
        const int differ = PyObject_RichCompareBool(dtype, args[1], Py_NE);
        if (differ > 0) PyErr_Format(PyExc_ValueError, "%S: dtype %S, expected %S", name, dtype, args[1]);
        if (differ) {
            Py_DECREF(dtype);
            return NULL;
        }
    }
    Py_DECREF(dtype);
    PyObject *have = call(t, plain, numel, s_numel);
    if (!have) return NULL;
    const int less = PyObject_RichCompareBool(have, args[2], Py_LT);
    if (less > 0) PyErr_Format(PyExc_ValueError, "%S: %S elements, the call touches %S", name, have, args[2]);
    Py_DECREF(have);
    if (less) return NULL;
    return call(t, plain, data_ptr, s_data_ptr);
}

/* whether the tensor is on that device; 1, 0 or -1 with an exception */
static int is_on(PyObject *t, PyObject *index)
{
    PyObject *at = call(t, (PyObject *)Py_TYPE(t) == tensor_type, get_device, s_get_device);
    if (!at) return -1;
    const int same = PyObject_RichCompareBool(at, index, Py_EQ);
    Py_DECREF(at);
    return same;
}

/* dev_on(tensor or None, dtype, numel, name, device index): dev, of a tensor on that device */
static PyObject *dev_on(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    if (n != 5) return PyErr_Format(PyExc_TypeError, "dev_on: 5 arguments expected, not %zd", n);
    PyObject *at = dev(self, args, 4);
    if (!at || args[0] == Py_None) return at;
    const int same = is_on(args[0], args[4]);
    if (same > 0) return at;
    Py_DECREF(at);
    return same ? NULL : PyErr_Format(PyExc_ValueError, "%S: must be on the cache's device", args[3]);
}

/* room_on(tensor or None, name, device index) -> (address, bytes) or (None, 0): a contiguous CUDA tensor on that device */
static PyObject *room_on(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 3) return PyErr_Format(PyExc_TypeError, "room_on: 3 arguments expected, not %zd", n);
    PyObject *t = args[0];
    if (t == Py_None) return Py_BuildValue("(Oi)", Py_None, 0);
    const int plain = (PyObject *)Py_TYPE(t) == tensor_type;
    if (!plain) {
        const int is = PyObject_IsInstance(t, tensor_type);
        if (is < 0) return NULL;
        if (!is) return PyErr_Format(PyExc_TypeError, "%S: expected a torch tensor", args[1]);
    }
    int ok = truth(PyObject_GetAttr(t, s_is_cuda));
    if (ok > 0) ok = truth(call(t, plain, is_contiguous, s_is_contiguous));
    if (ok < 0) return NULL;
    if (!ok) return PyErr_Format(PyExc_ValueError, "%S: must be a contiguous CUDA tensor", args[1]);
    ok = is_on(t, args[2]);
    if (ok < 0) return NULL;
    if (!ok) return PyErr_Format(PyExc_ValueError, "%S: must be on the cache's device", args[1]);
    PyObject *count = call(t, plain, numel, s_numel), *size = count ? call(t, plain, element_size, s_element_size) : NULL;
    PyObject *bytes = size ? PyNumber_Multiply(count, size) : NULL, *at = bytes ? call(t, plain, data_ptr, s_data_ptr) : NULL;
    PyObject *both = at ? PyTuple_Pack(2, at, bytes) : NULL;
    Py_XDECREF(count);
    Py_XDECREF(size);
    Py_XDECREF(bytes);
    Py_XDECREF(at);
    return both;
}

/* the k-th number of a tuple, or -1 with an exception */
static long long item_of(PyObject *tuple, Py_ssize_t k)
{
    PyObject *o = PySequence_GetItem(tuple, k);
    if (!o) return -1;
    const long long v = PyLong_AsLongLong(o);
    Py_DECREF(o);
    return v;
}

/* rows_on(tensor, dtype, heads, dh, name, device index) -> (address, elements from row to row): a CUDA tensor [T, heads, dh] on that device whose
 * heads lie behind each other, its rows anywhere further on (a part of a projection's output).  1.7 us in Python, 0.6 here. */
static PyObject *rows_on(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    (void)self;
    if (n != 6) return PyErr_Format(PyExc_TypeError, "rows_on: 6 arguments expected, not %zd", n);
    PyObject *t = args[0], *name = args[4];
    const int plain = (PyObject *)Py_TYPE(t) == tensor_type;
    if (!plain) {
        const int is = PyObject_IsInstance(t, tensor_type);
        if (is < 0) return NULL;
        if (!is) return PyErr_Format(PyExc_TypeError, "%S: expected a torch tensor", name);
    }
    const long long heads = PyLong_AsLongLong(args[2]), dh = PyLong_AsLongLong(args[3]);
    if (PyErr_Occurred()) return NULL;
    PyObject *shape = PyObject_GetAttr(t, s_shape);
    if (!shape) return NULL;
    const Py_ssize_t dims = PySequence_Size(shape);
    const long long T = dims == 3 ? item_of(shape, 0) : 0, h = dims == 3 ? item_of(shape, 1) : -1, d = dims == 3 ? item_of(shape, 2) : -1;
    Py_DECREF(shape);
    if (PyErr_Occurred()) return NULL;
    if (h != heads || d != dh) return PyErr_Format(PyExc_ValueError, "%S: must be [T, %lld, %lld]", name, heads, dh);
    PyObject *dtype = PyObject_GetAttr(t, s_dtype);
    if (!dtype) return NULL;
    const int differ = dtype == args[1] ? 0 : PyObject_RichCompareBool(dtype, args[1], Py_NE);
    if (differ > 0) PyErr_Format(PyExc_ValueError, "%S: dtype %S, expected %S", name, dtype, args[1]);
    Py_DECREF(dtype);
    if (differ) return NULL;
    PyObject *stride = call(t, plain, stride_of, s_stride);
    if (!stride) return NULL;
    const long long row = item_of(stride, 0), head = item_of(stride, 1), elem = item_of(stride, 2);
    Py_DECREF(stride);
    if (PyErr_Occurred()) return NULL;
    const int few = T <= 1;                            /* a stride that is never taken may be any number */
    const int cuda = truth(PyObject_GetAttr(t, s_is_cuda));
    if (cuda < 0) return NULL;
    if (!cuda || (elem != 1 && dh > 1) || (head != dh && heads > 1) || (row < heads * dh && !few))
        return PyErr_Format(PyExc_ValueError, "%S: must be a CUDA tensor whose heads lie behind each other", name);
    const int same = is_on(t, args[5]);
    if (same < 0) return NULL;
    if (!same) return PyErr_Format(PyExc_ValueError, "%S: must be on the same device as the others", name);
    PyObject *at = call(t, plain, data_ptr, s_data_ptr);
    return at ? Py_BuildValue("(NL)", at, few ? heads * dh : row) : NULL;
}

static PyMethodDef methods[] = {
    {"dev", (PyCFunction)(void (*)(void))dev, METH_FASTCALL,
     "Device pointer (a number: the argument types make the pointer) of a tensor after checking it can hold what the call touches."},
    {"dev_on", (PyCFunction)(void (*)(void))dev_on, METH_FASTCALL, "dev, of a tensor on the device given."},
    {"room_on", (PyCFunction)(void (*)(void))room_on, METH_FASTCALL, "Address and bytes of a workspace on the device given."},
    {"rows_on", (PyCFunction)(void (*)(void))rows_on, METH_FASTCALL, "Address and row stride of a tensor [T, heads, dh] on the device given, whose rows may lie apart."},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_argcheck", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__argcheck(void)
{
    PyObject *torch = PyImport_ImportModule("torch");
    if (!torch) return NULL;
    tensor_type = PyObject_GetAttrString(torch, "Tensor");
    Py_DECREF(torch);
    if (!tensor_type) return NULL;
    is_contiguous = PyObject_GetAttrString(tensor_type, "is_contiguous");
    numel = PyObject_GetAttrString(tensor_type, "numel");
    data_ptr = PyObject_GetAttrString(tensor_type, "data_ptr");
    get_device = PyObject_GetAttrString(tensor_type, "get_device");
    element_size = PyObject_GetAttrString(tensor_type, "element_size");
    stride_of = PyObject_GetAttrString(tensor_type, "stride");
    if (!is_contiguous || !numel || !data_ptr || !get_device || !element_size || !stride_of) return NULL;
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_numel = PyUnicode_InternFromString("numel");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_element_size = PyUnicode_InternFromString("element_size");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    if (!s_is_cuda || !s_is_contiguous || !s_dtype || !s_numel || !s_data_ptr || !s_get_device || !s_element_size || !s_shape || !s_stride) return NULL;
    return PyModule_Create(&module);
}
