/* What the binding looks at in a call's tensors, in one call instead of forty: a Python call for each attribute of a dozen
 * tensors takes longer than the library's own work.  Knows nothing of a tensor but its Python attributes. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

static PyObject *s_dtype, *s_shape, *s_get_device, *s_is_contiguous, *s_stride, *s_data_ptr;

/* 1: t is as `want` = (type, shape, strides or None for packed) says, on `device`, and *address is its address; 0: it is
 * not, or it has not these attributes. */
static int fits(PyObject *t, PyObject *want, long device, PyObject **address) {
    PyObject *x;
    int ok;
    *address = NULL;
    if (want == Py_None || t == Py_None) {
        if (want != t) return 0;
        *address = Py_NewRef(Py_None);
        return 1;
    }
    if (!(x = PyObject_GetAttr(t, s_dtype))) return 0;
    ok = x == PyTuple_GET_ITEM(want, 0);
    Py_DECREF(x);
    if (!ok || !(x = PyObject_CallMethodNoArgs(t, s_get_device))) return 0;
    ok = PyLong_Check(x) && PyLong_AsLong(x) == device;
    Py_DECREF(x);
    if (!ok || !(x = PyObject_GetAttr(t, s_shape))) return 0;
    ok = PyObject_RichCompareBool(x, PyTuple_GET_ITEM(want, 1), Py_EQ) == 1;
    Py_DECREF(x);
    if (!ok) return 0;
    if (PyTuple_GET_ITEM(want, 2) == Py_None) {
        if (!(x = PyObject_CallMethodNoArgs(t, s_is_contiguous))) return 0;
        ok = x == Py_True;
    } else {
        if (!(x = PyObject_CallMethodNoArgs(t, s_stride))) return 0;
        ok = PyObject_RichCompareBool(x, PyTuple_GET_ITEM(want, 2), Py_EQ) == 1;
    }
    Py_DECREF(x);
    if (!ok) return 0;
    return (*address = PyObject_CallMethodNoArgs(t, s_data_ptr)) != NULL;
}

/* find(calls, tensors, device, rest) -> (call, addresses) or None: the first of the list `calls`, tuples that start with
 * (looks, rest), whose `rest` equals the given one and whose looks the tensors have. */
static PyObject *find(PyObject *self, PyObject *const *args, Py_ssize_t n_args) {
    (void)self;
    if (n_args != 4 || !PyList_Check(args[0]) || !PyTuple_Check(args[1])) {
        PyErr_SetString(PyExc_TypeError, "find(list, tuple, int, rest)");
        return NULL;
    }
    PyObject *calls = args[0], *tensors = args[1];
    const long device = PyLong_AsLong(args[2]);
    if (device == -1 && PyErr_Occurred()) return NULL;
    const Py_ssize_t n = PyTuple_GET_SIZE(tensors);
    for (Py_ssize_t c = 0; c < PyList_GET_SIZE(calls); ++c) {
        PyObject *call = Py_NewRef(PyList_GET_ITEM(calls, c)); /* attributes are code: the list may change meanwhile */
        PyObject *looks = PyTuple_GET_ITEM(call, 0), *addresses = NULL;
        int ok = PyTuple_GET_SIZE(looks) == n && PyObject_RichCompareBool(PyTuple_GET_ITEM(call, 1), args[3], Py_EQ) == 1;
        if (ok && !(addresses = PyTuple_New(n))) {
            Py_DECREF(call);
            return NULL;
        }
        for (Py_ssize_t i = 0; ok && i < n; ++i) {
            PyObject *address;
            ok = fits(PyTuple_GET_ITEM(tensors, i), PyTuple_GET_ITEM(looks, i), device, &address);
            if (ok) PyTuple_SET_ITEM(addresses, i, address);
        }
        if (PyErr_Occurred()) PyErr_Clear(); /* what is wrong is said where the call is made anew */
        if (ok) {
            PyObject *found = PyTuple_Pack(2, call, addresses);
            Py_DECREF(call);
            Py_DECREF(addresses);
            return found;
        }
        Py_XDECREF(addresses);
        Py_DECREF(call);
    }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"find", (PyCFunction)(void (*)(void))find, METH_FASTCALL, "The call that these tensors fit."},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_match", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__match(void) {
    static const char *const names[] = {"dtype", "shape", "get_device", "is_contiguous", "stride", "data_ptr"};
    PyObject **const strings[] = {&s_dtype, &s_shape, &s_get_device, &s_is_contiguous, &s_stride, &s_data_ptr};
    for (int i = 0; i < 6; ++i)
        if (!(*strings[i] = PyUnicode_InternFromString(names[i]))) return NULL;
    return PyModule_Create(&module);
}
