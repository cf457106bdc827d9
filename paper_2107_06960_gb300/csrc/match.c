/* Calls that are like one made before: looks at their tensors and makes them, in one call instead of forty.  (A Python call
 * for each attribute of a dozen tensors, and ctypes' conversions, take longer than the library's own work.)  Knows
 * nothing of a tensor but its Python attributes. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include "../../include/mafat.h"

static PyObject *s_dtype, *s_shape, *s_get_device, *s_is_contiguous, *s_stride, *s_data_ptr;

/* 1: t is as `want` = (type, shape, strides or None for packed) says, on `device`, and *address is its address; 0: it is
 * not, or it has not these attributes. */
static int fits(PyObject *t, PyObject *want, long device, void **address) {
    PyObject *x;
    int ok;
    *address = NULL;
    if (want == Py_None || t == Py_None) return want == t;
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
    if (!(x = PyObject_CallMethodNoArgs(t, s_data_ptr))) return 0;
    *address = PyLong_Check(x) ? PyLong_AsVoidPtr(x) : NULL;
    ok = PyLong_Check(x) && !PyErr_Occurred();
    Py_DECREF(x);
    return ok;
}

/* The library's entries, as they are loaded (set by bind). */
static __typeof__(&mafat_block_norm) block_norm;
static __typeof__(&mafat_rotary_run) rotary_run;
static __typeof__(&mafat_tree_run) tree_run;
static __typeof__(&mafat_adjust_logits) adjust_logits;
enum { kNorm, kRotary, kTree, kLogits, kEntries };
static const Py_ssize_t kTensors[kEntries] = {8, 8, 12, 14};
enum { kMostTensors = 14 };

/* bind(address of each entry): before the first run. */
static PyObject *bind(PyObject *self, PyObject *args) {
    unsigned long long p[kEntries];
    (void)self;
    if (!PyArg_ParseTuple(args, "KKKK", &p[0], &p[1], &p[2], &p[3])) return NULL;
    block_norm = (__typeof__(block_norm))(uintptr_t)p[kNorm];
    rotary_run = (__typeof__(rotary_run))(uintptr_t)p[kRotary];
    tree_run = (__typeof__(tree_run))(uintptr_t)p[kTree];
    adjust_logits = (__typeof__(adjust_logits))(uintptr_t)p[kLogits];
    Py_RETURN_NONE;
}

static mafat_status make(int entry, const void *plan, uintptr_t what, void *const *t, void *stream) {
    switch (entry) {
    case kNorm: return block_norm((const mafat_block_norm_desc *)what, t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7], stream);
    case kRotary:
        return rotary_run(plan, (const mafat_rotary_call *)what, t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7], stream);
    case kTree:
        return tree_run(plan, t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7], t[8], t[9], (int32_t)what, t[10], t[11], stream);
    default:
        return adjust_logits((const mafat_logits_desc *)what, t[0], t[1], t[2], t[3], t[4], t[5], t[6], t[7], t[8], t[9], t[10], t[11],
                             t[12], t[13], stream);
    }
}

/* run(entry, calls, tensors, device, rest, plan, stream) -> status or None: makes the first of the list `calls`, tuples of
 * (looks, rest, what, ...), whose `rest` equals the given one and whose looks the tensors have.  `what` is the address of
 * its descriptor, of a tree whether it is shared.  None: there is none. */
static PyObject *run(PyObject *self, PyObject *const *args, Py_ssize_t n_args) {
    (void)self;
    if (n_args != 7 || !PyList_Check(args[1]) || !PyTuple_Check(args[2])) {
        PyErr_SetString(PyExc_TypeError, "run(entry, list, tuple, device, rest, plan, stream)");
        return NULL;
    }
    const long entry = PyLong_AsLong(args[0]), device = PyLong_AsLong(args[3]);
    if (PyErr_Occurred()) return NULL;
    PyObject *calls = args[1], *tensors = args[2];
    const Py_ssize_t n = PyTuple_GET_SIZE(tensors);
    if (entry < 0 || entry >= kEntries || n != kTensors[entry] || !block_norm) {
        PyErr_SetString(PyExc_ValueError, "no such entry, or not of so many tensors");
        return NULL;
    }
    void *plan = args[5] == Py_None ? NULL : PyLong_AsVoidPtr(args[5]), *stream = args[6] == Py_None ? NULL : PyLong_AsVoidPtr(args[6]);
    if (PyErr_Occurred()) return NULL;
    for (Py_ssize_t c = 0; c < PyList_GET_SIZE(calls); ++c) {
        PyObject *call = Py_NewRef(PyList_GET_ITEM(calls, c)); /* attributes are code: the list may change meanwhile */
        PyObject *looks = PyTuple_GET_ITEM(call, 0);
        void *t[kMostTensors];
        int ok = PyTuple_GET_SIZE(looks) == n && PyObject_RichCompareBool(PyTuple_GET_ITEM(call, 1), args[4], Py_EQ) == 1;
        for (Py_ssize_t i = 0; ok && i < n; ++i) ok = fits(PyTuple_GET_ITEM(tensors, i), PyTuple_GET_ITEM(looks, i), device, &t[i]);
        if (PyErr_Occurred()) PyErr_Clear(); /* what is wrong is said where the call is made anew */
        if (ok) {
            const uintptr_t what = (uintptr_t)PyLong_AsVoidPtr(PyTuple_GET_ITEM(call, 2));
            mafat_status status = MAFAT_OK;
            if (!PyErr_Occurred()) {
                Py_BEGIN_ALLOW_THREADS
                status = make((int)entry, plan, what, t, stream);
                Py_END_ALLOW_THREADS
            }
            Py_DECREF(call); /* and with it the descriptor, where it has been dropped from the list */
            return PyErr_Occurred() ? NULL : PyLong_FromLong((long)status);
        }
        Py_DECREF(call);
    }
    Py_RETURN_NONE;
}

static PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, "The library's entries."},
                                {"run", (PyCFunction)(void (*)(void))run, METH_FASTCALL, "A call that is like one made before."},
                                {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_match", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__match(void) {
    static const char *const names[] = {"dtype", "shape", "get_device", "is_contiguous", "stride", "data_ptr"};
    PyObject **const strings[] = {&s_dtype, &s_shape, &s_get_device, &s_is_contiguous, &s_stride, &s_data_ptr};
    for (int i = 0; i < 6; ++i)
        if (!(*strings[i] = PyUnicode_InternFromString(names[i]))) return NULL;
    return PyModule_Create(&module);
}
