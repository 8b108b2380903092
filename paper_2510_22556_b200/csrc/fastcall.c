/* Calls of the C ABI from Python without ctypes' per-argument objects: bind(address) returns a builtin
 * that takes integers (device or host addresses, sizes, handles), None (a null pointer) and tuples
 * or lists of numbers (passed as int arrays that live for the call), and returns the status code.  What counts as an
 * integer is what the ctypes declarations take.
 * Marshalling only, like the ctypes declarations in binding.py, which are used where this module has not
 * been built; a decode call's share of host time goes from 1.0 to 0.3 us.
 *
 * Every parameter of the entry points is an integer or a pointer, so one prototype with as many
 * 64-bit integers as the longest of them serves them all (x86-64 and AArch64 calling conventions: the
 * first ones in registers, the rest in eight-byte stack slots; what a callee does not take it ignores).
 * The interpreter lock is released during the call (the host-buffer pass waits for the device). */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

enum { kMaxArgs = 26, kMaxInts = 256 };
typedef uint64_t u;
typedef int (*entry)(u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u);

/* What ctypes makes of an int argument: anything with an index (numpy and torch integers too), its low bits. */
static int take_scalar(PyObject* x, u* out)
{
    if (PyLong_Check(x)) {
        *out = PyLong_AsUnsignedLongLongMask(x);
    } else {
        PyObject* v = PyNumber_Index(x);
        if (!v) return -1;
        *out = PyLong_AsUnsignedLongLongMask(v);
        Py_DECREF(v);
    }
    return PyErr_Occurred() ? -1 : 0;
}

/* What c_int makes of int(x). */
static int take_element(PyObject* x, int* out)
{
    PyObject* v = PyLong_Check(x) ? Py_NewRef(x) : PyNumber_Long(x);
    if (!v) return -1;
    *out = (int)(unsigned)PyLong_AsUnsignedLongMask(v);
    Py_DECREF(v);
    return PyErr_Occurred() ? -1 : 0;
}

static PyObject* invoke(PyObject* self, PyObject* const* args, Py_ssize_t n)
{
    u a[kMaxArgs] = {0};
    int stack[kMaxInts], *ints = stack;
    PyObject* seq[kMaxArgs] = {0};                     /* sequence arguments as tuples of this call's own */
    PyObject* result = NULL;
    Py_ssize_t used = 0;
    if (n > kMaxArgs) return PyErr_Format(PyExc_TypeError, "%zd arguments, at most %d", n, kMaxArgs);
    for (Py_ssize_t i = 0; i < n; ++i)
        if (PyTuple_Check(args[i]) || PyList_Check(args[i])) {
            seq[i] = PySequence_Tuple(args[i]);
            if (!seq[i]) goto done;
            used += PyTuple_GET_SIZE(seq[i]);
        }
    if (used > kMaxInts && !(ints = PyMem_Malloc(used * sizeof(int)))) {
        PyErr_NoMemory();
        goto done;
    }
    used = 0;
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (seq[i]) {
            a[i] = (u)(uintptr_t)(ints + used);
            for (Py_ssize_t k = 0; k < PyTuple_GET_SIZE(seq[i]); ++k)
                if (take_element(PyTuple_GET_ITEM(seq[i], k), ints + used++) < 0) goto done;
        } else if (args[i] != Py_None && take_scalar(args[i], &a[i]) < 0) {
            goto done;
        }
    }
    const entry f = (entry)(uintptr_t)PyLong_AsUnsignedLongLong(self);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11], a[12], a[13], a[14], a[15], a[16], a[17],
           a[18], a[19], a[20], a[21], a[22], a[23], a[24], a[25]);
    Py_END_ALLOW_THREADS
    result = PyLong_FromLong(rc);
done:
    for (Py_ssize_t i = 0; i < n; ++i) Py_XDECREF(seq[i]);
    if (ints != stack) PyMem_Free(ints);
    return result;
}

static PyMethodDef invoke_def = {"entry", (PyCFunction)(void (*)(void))invoke, METH_FASTCALL, "calls one entry point of the C ABI"};

static PyObject* bind(PyObject* module, PyObject* address)
{
    (void)module;
    if (!PyLong_Check(address)) return PyErr_Format(PyExc_TypeError, "an address");
    return PyCFunction_New(&invoke_def, address);
}

/* A decoding step is one short call per layer, and most of its host time is Python's: bind_decode(address) returns a builtin
 * that takes the tensors themselves, (params, q, k_cache, v_cache, n_valid, out, lse, ws, stream), and asks them for what
 * sablock_decode_attention wants to know. */
static PyObject *s_data_ptr, *s_shape, *s_numel;

static int take_method(PyObject* t, PyObject* name, u* out)
{
    if (t == Py_None) return 0;                        /* a null pointer */
    PyObject* v = PyObject_CallMethodNoArgs(t, name);
    if (!v) return -1;
    const int rc = take_scalar(v, out);
    Py_DECREF(v);
    return rc;
}

/* Extent `dim` of a tensor; it has `rank` dimensions (0: any number). */
static int take_extent(PyObject* t, Py_ssize_t rank, Py_ssize_t dim, u* out)
{
    PyObject* shape = PyObject_GetAttr(t, s_shape);
    if (!shape) return -1;
    int rc = -1;
    if (!PyTuple_Check(shape)) PyErr_SetString(PyExc_TypeError, "a tensor");
    else if (rank && PyTuple_GET_SIZE(shape) != rank) PyErr_Format(PyExc_ValueError, "%zd dimensions, not %zd", PyTuple_GET_SIZE(shape), rank);
    else if (dim >= PyTuple_GET_SIZE(shape)) PyErr_SetString(PyExc_IndexError, "too few dimensions");
    else rc = take_scalar(PyTuple_GET_ITEM(shape, dim), out);
    Py_DECREF(shape);
    return rc;
}

static PyObject* invoke_decode(PyObject* self, PyObject* const* args, Py_ssize_t n)
{
    typedef int (*decode)(u, u, u, u, u, u, u, u, u, u, u, u);
    u p = 0, q = 0, k = 0, v = 0, valid = 0, out = 0, lse = 0, ws = 0, ws_bytes = 0, stream = 0, n_prob = 0, n_rows = 0;
    if (n != 9) return PyErr_Format(PyExc_TypeError, "%zd arguments, not 9", n);
    if (take_scalar(args[0], &p) < 0 || take_extent(args[1], 3, 0, &n_prob) < 0 || take_extent(args[2], 0, 1, &n_rows) < 0 ||
        take_method(args[1], s_data_ptr, &q) < 0 || take_method(args[2], s_data_ptr, &k) < 0 || take_method(args[3], s_data_ptr, &v) < 0 ||
        take_method(args[4], s_data_ptr, &valid) < 0 || take_method(args[5], s_data_ptr, &out) < 0 || take_method(args[6], s_data_ptr, &lse) < 0 ||
        take_method(args[7], s_data_ptr, &ws) < 0 || take_method(args[7], s_numel, &ws_bytes) < 0 || take_scalar(args[8], &stream) < 0)
        return NULL;
    const decode f = (decode)(uintptr_t)PyLong_AsUnsignedLongLong(self);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(p, n_prob, q, k, v, n_rows, valid, out, lse, ws, ws_bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

static PyMethodDef invoke_decode_def = {"decode", (PyCFunction)(void (*)(void))invoke_decode, METH_FASTCALL, "calls sablock_decode_attention"};

static PyObject* bind_decode(PyObject* module, PyObject* address)
{
    (void)module;
    if (!PyLong_Check(address)) return PyErr_Format(PyExc_TypeError, "an address");
    return PyCFunction_New(&invoke_decode_def, address);
}

/* What the calls over a paged cache check of a tensor, a few attributes each, in a third of the time that the same takes in
 * Python.  fits(tensor, dtype, device, shape): whether it is that and contiguous; token_stride(tensor, dtype, device, n, heads, channels):
 * elements from token to token of a tensor [n, heads, channels] whose heads are contiguous (0 where n < 2), -1 where it is none (nor is one
 * token repeated: a stride of 0 says contiguous). */
static PyObject *s_dtype, *s_device, *s_contiguous, *s_stride;

/* 1: attribute `name` of t equals v; 0: it does not; -1: an error. */
static int attr_equals(PyObject* t, PyObject* name, PyObject* v)
{
    PyObject* x = PyObject_GetAttr(t, name);
    if (!x) return -1;
    const int rc = x == v ? 1 : PyObject_RichCompareBool(x, v, Py_EQ);
    Py_DECREF(x);
    return rc;
}

static PyObject* fits(PyObject* module, PyObject* const* args, Py_ssize_t n)
{
    (void)module;
    if (n != 4) return PyErr_Format(PyExc_TypeError, "%zd arguments, not 4", n);
    int rc = attr_equals(args[0], s_dtype, args[1]);
    if (rc == 1) rc = attr_equals(args[0], s_device, args[2]);
    if (rc == 1) rc = attr_equals(args[0], s_shape, args[3]);
    if (rc == 1) {
        PyObject* x = PyObject_CallMethodNoArgs(args[0], s_contiguous);
        if (!x) return NULL;
        rc = x == Py_True;
        Py_DECREF(x);
    }
    return rc < 0 ? NULL : PyBool_FromLong(rc);
}

/* Integers of a tuple of three. */
static int take_three(PyObject* t, long long (*x)[3])
{
    if (!PyTuple_Check(t) || PyTuple_GET_SIZE(t) != 3) return 0;
    for (int i = 0; i < 3; ++i) {
        (*x)[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
        if ((*x)[i] == -1 && PyErr_Occurred()) return -1;
    }
    return 1;
}

/* 1: t is a contiguous tensor of that type, device and n elements in one dimension; 0: it is not; -1: an error. */
static int fits_vector(PyObject* t, PyObject* dtype, PyObject* device, long long n)
{
    int rc = attr_equals(t, s_dtype, dtype);
    if (rc == 1) rc = attr_equals(t, s_device, device);
    if (rc != 1) return rc;
    PyObject* x = PyObject_GetAttr(t, s_shape);
    if (!x) return -1;
    rc = PyTuple_Check(x) && PyTuple_GET_SIZE(x) == 1 && (n < 0 || PyLong_AsLongLong(PyTuple_GET_ITEM(x, 0)) == n);
    Py_DECREF(x);
    if (rc != 1) return rc;
    x = PyObject_CallMethodNoArgs(t, s_contiguous);
    if (!x) return -1;
    rc = x == Py_True;
    Py_DECREF(x);
    return rc;
}

/* What token_stride says, for a type, a device and sizes that are at hand; -2: an error. */
static long long stride_of(PyObject* t, PyObject* dtype, PyObject* device, long long n, long long heads, long long d)
{
    long long size[3], stride[3];
    int rc = attr_equals(t, s_dtype, dtype);
    if (rc == 1) rc = attr_equals(t, s_device, device);
    if (rc == 1) {
        PyObject* x = PyObject_GetAttr(t, s_shape);
        if (!x) return -2;
        rc = take_three(x, &size);
        Py_DECREF(x);
    }
    if (rc == 1) rc = size[0] == n && size[1] == heads && size[2] == d;
    if (rc == 1) {
        PyObject* x = PyObject_CallMethodNoArgs(t, s_stride);
        if (!x) return -2;
        rc = take_three(x, &stride);
        Py_DECREF(x);
    }
    if (rc < 0) return -2;
    if (rc == 1 && n > 0) rc = (d < 2 || stride[2] == 1) && (heads < 2 || stride[1] == d) && (n < 2 || stride[0] > 0);
    return rc != 1 ? -1 : n > 1 ? stride[0] : 0;
}

static PyObject* token_stride(PyObject* module, PyObject* const* args, Py_ssize_t n)
{
    (void)module;
    long long want[3];
    if (n != 6) return PyErr_Format(PyExc_TypeError, "%zd arguments, not 6", n);
    for (int i = 0; i < 3; ++i) {
        want[i] = PyLong_AsLongLong(args[3 + i]);
        if (want[i] == -1 && PyErr_Occurred()) return NULL;
    }
    const long long s = stride_of(args[0], args[1], args[2], want[0], want[1], want[2]);
    return s == -2 ? NULL : PyLong_FromLongLong(s);
}

/* Appending is one short call per layer and token: bind_append(address) returns a builtin that takes the tensors themselves,
 * (params, pages, (dtype, device, n_seqs, n_kv_heads, n_q_heads, head_dim, int32, float32, empty_like), k, v, q, q_out, positions,
 * inv_freq, interleaved, cu_new, stream), checks them and calls sablock_paged_append.  It returns the rotated queries (None without
 * queries), a status code that is not 0, or NotImplemented where an argument does not fit: the caller says then which. */
static PyObject* invoke_append(PyObject* self, PyObject* const* args, Py_ssize_t n_args)
{
    typedef int (*append)(u, u, u, u, u, u, u, u, u, u, u, u, u, u, u, u);
    u p = 0, pages = 0, k = 0, v = 0, q = 0, out = 0, pos = 0, freq = 0, cu = 0, stream = 0, n = 0, rotary = 0;
    long long want[4], ks, vs, qs = 0;
    if (n_args != 12) return PyErr_Format(PyExc_TypeError, "%zd arguments, not 12", n_args);
    PyObject* spec = args[2];
    if (!PyTuple_Check(spec) || PyTuple_GET_SIZE(spec) != 9) return PyErr_Format(PyExc_TypeError, "a description of nine parts");
    PyObject *dtype = PyTuple_GET_ITEM(spec, 0), *device = PyTuple_GET_ITEM(spec, 1), *i32 = PyTuple_GET_ITEM(spec, 6), *f32 = PyTuple_GET_ITEM(spec, 7);
    for (int i = 0; i < 4; ++i) {
        want[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(spec, 2 + i));
        if (want[i] == -1 && PyErr_Occurred()) return NULL;
    }
    const long long seqs = want[0], hkv = want[1], heads = want[2], d = want[3];
    if (take_scalar(args[0], &p) < 0 || take_scalar(args[1], &pages) < 0 || take_scalar(args[11], &stream) < 0 || take_extent(args[3], 3, 0, &n) < 0) {
        if (PyErr_ExceptionMatches(PyExc_ValueError) || PyErr_ExceptionMatches(PyExc_AttributeError)) {      /* no tensor of three dimensions */
            PyErr_Clear();
            Py_RETURN_NOTIMPLEMENTED;
        }
        return NULL;
    }
    const int turned = PyObject_IsTrue(args[9]);
    if (turned < 0) return NULL;
    const int has_q = args[5] != Py_None, made = has_q && args[6] == Py_None;
    int rc = (ks = stride_of(args[3], dtype, device, (long long)n, hkv, d)) >= 0 && (vs = stride_of(args[4], dtype, device, (long long)n, hkv, d)) >= 0;
    if (rc && has_q) rc = (qs = stride_of(args[5], dtype, device, (long long)n, heads, d)) >= 0;
    if (rc && !made) rc = args[6] == Py_None;        /* (a caller's own buffer takes the other way) */
    if (rc && made) rc = qs == 0 || qs >= heads * d; /* (so do tokens that overlap: what looks like them would not be contiguous) */
    if (rc && args[7] != Py_None) rc = fits_vector(args[7], i32, device, (long long)n) == 1;
    if (rc && args[8] != Py_None) {
        rc = fits_vector(args[8], f32, device, -1) == 1 && take_extent(args[8], 1, 0, &rotary) == 0;
        rotary *= 2;
    }
    if (rc && args[10] != Py_None) rc = fits_vector(args[10], i32, device, seqs + 1) == 1;
    if (!rc) {
        PyErr_Clear();
        Py_RETURN_NOTIMPLEMENTED;
    }
    PyObject* result = Py_NewRef(Py_None);
    if (made) {
        Py_DECREF(result);
        result = PyObject_CallOneArg(PyTuple_GET_ITEM(spec, 8), args[5]);      /* (contiguous: tokens apart are not kept apart) */
        if (!result) return NULL;
    }
    if (take_method(args[3], s_data_ptr, &k) < 0 || take_method(args[4], s_data_ptr, &v) < 0 || take_method(args[5], s_data_ptr, &q) < 0 ||
        take_method(result, s_data_ptr, &out) < 0 || take_method(args[7], s_data_ptr, &pos) < 0 || take_method(args[8], s_data_ptr, &freq) < 0 ||
        take_method(args[10], s_data_ptr, &cu) < 0) {
        Py_DECREF(result);
        return NULL;
    }
    const append f = (append)(uintptr_t)PyLong_AsUnsignedLongLong(self);
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = f(p, pages, n, cu, k, (u)ks, v, (u)vs, q, (u)qs, out, pos, freq, rotary, (u)turned, stream);
    Py_END_ALLOW_THREADS
    if (code == 0) return result;
    Py_DECREF(result);
    return PyLong_FromLong(code);
}

static PyMethodDef invoke_append_def = {"append", (PyCFunction)(void (*)(void))invoke_append, METH_FASTCALL, "calls sablock_paged_append"};

static PyObject* bind_append(PyObject* module, PyObject* address)
{
    (void)module;
    if (!PyLong_Check(address)) return PyErr_Format(PyExc_TypeError, "an address");
    return PyCFunction_New(&invoke_append_def, address);
}

static PyMethodDef methods[] = {{"bind_append", bind_append, METH_O, "bind_append(address): sablock_paged_append for tensors"},
                                {"fits", (PyCFunction)(void (*)(void))fits, METH_FASTCALL, "fits(tensor, dtype, device, shape)"},
                                {"token_stride", (PyCFunction)(void (*)(void))token_stride, METH_FASTCALL,
                                 "token_stride(tensor, dtype, device, n, heads, channels)"},
                                {"bind_decode", bind_decode, METH_O, "bind_decode(address): sablock_decode_attention for tensors"},
                                {"bind", bind, METH_O, "bind(address): a callable for the entry point at that address"}, {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", NULL, -1, methods, NULL, NULL, NULL, NULL};
PyMODINIT_FUNC PyInit__fastcall(void)
{
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_shape = PyUnicode_InternFromString("shape");
    s_numel = PyUnicode_InternFromString("numel");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_device = PyUnicode_InternFromString("device");
    s_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_stride = PyUnicode_InternFromString("stride");
    return s_data_ptr && s_shape && s_numel && s_dtype && s_device && s_contiguous && s_stride ? PyModule_Create(&module) : NULL;
}
