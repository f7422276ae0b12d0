// Argument marshalling of the calls a serving loop makes for every layer (CPython extension module ppd_call): the same
// conversions that the ctypes binding does, for a fifth of its time.  Each function takes the address of a libppd entry
// point first, so this module links to nothing; the GIL is released around the call.
// A small step is bound by the host: ctypes cost 1.1 us of the 4.0 us of an append call and 2.2 of the 5.6 of an
// attention call whose plan is on the device.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

static PyObject *s_data_ptr, *s_value, *s_shape, *s_element_size, *s_is_floating_point, *s_is_contiguous;
static PyObject *t_void_p, *f_cast;  // ctypes.c_void_p and ctypes.cast

// What a ctypes parameter of type c_void_p takes: None, an int and a c_void_p (a context's handle) here, anything else --
// objects with _as_parameter_ (torch.cuda.Stream is one), pointers, arrays -- by ctypes itself, which also refuses the rest
static int to_handle(PyObject* o, void** out) {
    *out = NULL;
    if (o == Py_None) return 1;
    if (PyLong_Check(o)) {
        *out = (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(o);
        return !PyErr_Occurred();
    }
    PyObject* p = (PyObject*)Py_TYPE(o) == t_void_p ? Py_NewRef(o) : PyObject_CallFunctionObjArgs(f_cast, o, t_void_p, NULL);
    if (!p) return 0;
    PyObject* v = PyObject_GetAttr(p, s_value);
    Py_DECREF(p);
    if (!v) return 0;
    if (v != Py_None) *out = (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}
// a tensor's data_ptr(), or None or an int that already is an address
static int to_address(PyObject* o, void** out) {
    if (o == Py_None || PyLong_Check(o)) return to_handle(o, out);
    PyObject* v = PyObject_CallMethodNoArgs(o, s_data_ptr);
    if (!v) return 0;
    const int ok = to_handle(v, out);
    Py_DECREF(v);
    return ok;
}
static int to_int(PyObject* o, int64_t* out) {
    PyObject* v = PyNumber_Long(o);
    if (!v) return 0;
    *out = (int64_t)PyLong_AsUnsignedLongLongMask(v);
    Py_DECREF(v);
    return !PyErr_Occurred();
}
// `o` as an int, or x.shape[dim] if it is None
static int to_int_or_shape(PyObject* o, PyObject* x, Py_ssize_t dim, int64_t* out) {
    if (o != Py_None) return to_int(o, out);
    PyObject* shape = PyObject_GetAttr(x, s_shape);
    if (!shape) return 0;
    PyObject* v = PySequence_GetItem(shape, dim);
    Py_DECREF(shape);
    if (!v) return 0;
    const int ok = to_int(v, out);
    Py_DECREF(v);
    return ok;
}
// `o` as an int of 32 bits, or x.shape[dim] if it is None and x is given.  0 with *why set (and no error) if it does not fit: the call is refused
// with that message.
static int to_int32(PyObject* o, PyObject* x, Py_ssize_t dim, const char* name, int32_t* out, PyObject** why) {
    if (o == Py_None && x) {
        int64_t wide;
        if (!to_int_or_shape(o, x, dim, &wide)) return 0;
        *out = (int32_t)wide;
        return 1;
    }
    PyObject* v = PyNumber_Long(o);
    if (!v) return 0;
    int over;
    const long long wide = PyLong_AsLongLongAndOverflow(v, &over);
    Py_DECREF(v);
    if (wide == -1 && PyErr_Occurred()) return 0;
    if (over || wide != (int32_t)wide) {
        *why = PyUnicode_FromFormat("%s does not fit 32 bits", name);
        return 0;
    }
    *out = (int32_t)wide;
    return 1;
}
// Whether a tensor's elements are what the call takes (an address or None is taken on trust): 0 with *why set if not.
static int call_int(PyObject* o, PyObject* method, int64_t* out) {
    PyObject* v = PyObject_CallMethodNoArgs(o, method);
    if (!v) return 0;
    const int ok = to_int(v, out);
    Py_DECREF(v);
    return ok;
}
static int has_elements(PyObject* o, const char* name, int64_t bytes, int floating, const char* type, PyObject** why) {
    int64_t size, is_floating;
    if (o == Py_None || PyLong_Check(o)) return 1;
    if (!call_int(o, s_element_size, &size) || !call_int(o, s_is_floating_point, &is_floating)) return 0;
    if (size == bytes && (is_floating != 0) == floating) return 1;
    *why = PyUnicode_FromFormat("%s has to be of %s", name, type);
    return 0;
}
// Whether a tensor whose strides are taken from its shape (`stride` is None) has these strides.
static int is_dense(PyObject* o, PyObject* stride, const char* name, PyObject** why) {
    int64_t dense;
    if (stride != Py_None || o == Py_None || PyLong_Check(o)) return 1;
    if (!call_int(o, s_is_contiguous, &dense)) return 0;
    if (dense) return 1;
    *why = PyUnicode_FromFormat("%s has to be contiguous, or its stride given", name);
    return 0;
}
static int expect(Py_ssize_t have, Py_ssize_t want) {
    if (have == want) return 1;
    PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
    return 0;
}

typedef int32_t (*append_fn)(void*, const void*, const void*, void*, const int64_t*, int64_t, void*);
typedef int32_t (*land_fn)(void*, const void*, const void*, void*, int64_t, int32_t, const int64_t*, int64_t, void*);
typedef int32_t (*mixed_fn)(void*, const void*, const void*, const int32_t*, int32_t, const int32_t*, const int32_t*, int32_t, float, void*, void*);

// kv_append(fn, ctx, k, v, kv_pages, slot_mapping, T, stream) -> status
static PyObject* call_append(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *k, *v, *pages, *slots, *stream;
    int64_t T;
    (void)self;
    if (!expect(n, 8) || !to_handle(a[0], &fn) || !to_handle(a[1], &ctx) || !to_int_or_shape(a[6], a[5], 0, &T) ||
        !to_address(a[2], &k) || !to_address(a[3], &v) || !to_address(a[4], &pages) ||
        !to_address(a[5], &slots) || !to_handle(a[7], &stream))
        return NULL;
    int32_t status;
    Py_BEGIN_ALLOW_THREADS
    status = ((append_fn)fn)(ctx, k, v, pages, (const int64_t*)slots, T, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// kv_land(fn, ctx, k, v, kv_pages, layer_stride_elems, num_layers, slot_mapping, T, stream) -> status
static PyObject* call_land(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *k, *v, *pages, *slots, *stream;
    int64_t stride, layers, T;
    (void)self;
    if (!expect(n, 10) || !to_handle(a[0], &fn) || !to_handle(a[1], &ctx) || !to_int_or_shape(a[8], a[7], 0, &T) ||
        !to_address(a[2], &k) || !to_address(a[3], &v) || !to_address(a[4], &pages) ||
        !to_int(a[5], &stride) || !to_int(a[6], &layers) || !to_address(a[7], &slots) || !to_handle(a[9], &stream))
        return NULL;
    int32_t status;
    Py_BEGIN_ALLOW_THREADS
    status = ((land_fn)fn)(ctx, k, v, pages, stride, (int32_t)layers, (const int64_t*)slots, T, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// A one-dimensional contiguous array of native 32-bit integers: 1 and a filled buffer; anything else: 0, no error
static int int32_array(PyObject* o, Py_buffer* b) {
    if (!PyObject_CheckBuffer(o)) return 0;
    if (PyObject_GetBuffer(o, b, PyBUF_C_CONTIGUOUS | PyBUF_FORMAT) != 0) {
        PyErr_Clear();
        return 0;
    }
    if (b->ndim == 1 && b->itemsize == 4 && b->format && b->format[0] == 'i' && b->format[1] == 0) return 1;
    PyBuffer_Release(b);
    return 0;
}

// mixed_attention(fn, ctx, q, kv_pages, page_tables, max_pages, L, n, scale, out, stream) -> status, or None if L and n are not
// plain int32 arrays yet
static PyObject* call_mixed(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *q, *pages, *tables, *out, *stream;
    int64_t max_pages;
    Py_buffer L, nn;
    (void)self;
    if (!expect(n, 11)) return NULL;
    if (!int32_array(a[6], &L)) Py_RETURN_NONE;
    if (!int32_array(a[7], &nn)) {
        PyBuffer_Release(&L);
        Py_RETURN_NONE;
    }
    PyObject* result = NULL;
    PyObject* scale = NULL;
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && to_int_or_shape(a[5], a[4], 1, &max_pages) &&
        to_address(a[2], &q) && to_address(a[3], &pages) && to_address(a[4], &tables) &&
        (scale = PyNumber_Float(a[8])) && to_address(a[9], &out) && to_handle(a[10], &stream)) {
        const float s = (float)PyFloat_AS_DOUBLE(scale);
        int32_t status;
        Py_BEGIN_ALLOW_THREADS
        status = ((mixed_fn)fn)(ctx, q, pages, (const int32_t*)tables, (int32_t)max_pages, (const int32_t*)L.buf, (const int32_t*)nn.buf,
                                (int32_t)L.shape[0], s, out, stream);
        Py_END_ALLOW_THREADS
        result = PyLong_FromLong(status);
    }
    Py_XDECREF(scale);
    PyBuffer_Release(&nn);
    PyBuffer_Release(&L);
    return result;
}

// Two int32 arrays of one length: 1 and both buffers filled, else 0 and none is
static int int32_arrays(PyObject* x, PyObject* y, Py_buffer* a, Py_buffer* b) {
    if (!int32_array(x, a)) return 0;
    if (!int32_array(y, b)) {
        PyBuffer_Release(a);
        return 0;
    }
    if (a->shape[0] == b->shape[0]) return 1;
    PyBuffer_Release(b);
    PyBuffer_Release(a);
    return 0;
}

typedef int32_t (*tree_fn)(void*, const void*, const void*, const int32_t*, int32_t, const uint64_t*, int32_t, const int32_t*, const int32_t*, int32_t, float, void*, void*);
typedef int32_t (*weighted_fn)(void*, const void*, const void*, const int32_t*, int32_t, const int32_t*, const int32_t*, int32_t, float, void*, float*, int64_t, void*);
typedef int32_t (*select_fn)(void*, const float*, int64_t, const int32_t*, int32_t, int32_t, int32_t, int32_t, int32_t*, int64_t, void*);
typedef int32_t (*compact_fn)(void*, void*, int64_t, int32_t, const int32_t*, int32_t, const int32_t*, int64_t, int64_t, int64_t, const int32_t*, const int32_t*, int32_t,
                              float*, int64_t, void*);

// tree_attention(fn, ctx, q, kv_pages, page_tables, max_pages, tree_mask, mask_words, L, n, scale, out, stream) -> status, or None if L and n are
// not plain int32 arrays of one length yet, or, for arguments that cannot be passed on, a message
static PyObject* call_tree(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *q, *pages, *tables, *mask, *out, *stream;
    int32_t max_pages, words;
    PyObject* why = NULL;
    Py_buffer L, nn;
    (void)self;
    if (!expect(n, 13)) return NULL;
    if (!int32_arrays(a[8], a[9], &L, &nn)) Py_RETURN_NONE;
    PyObject* result = NULL;
    PyObject* scale = NULL;
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && to_int32(a[5], a[4], 1, "max_pages", &max_pages, &why) && to_int32(a[7], a[6], 1, "mask_words", &words, &why) &&
        to_address(a[2], &q) && to_address(a[3], &pages) && has_elements(a[4], "page_tables", 4, 0, "int32", &why) &&
        is_dense(a[4], a[5], "page_tables", &why) && to_address(a[4], &tables) &&
        has_elements(a[6], "tree_mask", 8, 0, "int64 or uint64", &why) && is_dense(a[6], a[7], "tree_mask", &why) && to_address(a[6], &mask) &&
        (scale = PyNumber_Float(a[10])) && to_address(a[11], &out) && to_handle(a[12], &stream)) {
        const float s = (float)PyFloat_AS_DOUBLE(scale);
        int32_t status;
        Py_BEGIN_ALLOW_THREADS
        status = ((tree_fn)fn)(ctx, q, pages, (const int32_t*)tables, max_pages, (const uint64_t*)mask, words, (const int32_t*)L.buf,
                               (const int32_t*)nn.buf, (int32_t)L.shape[0], s, out, stream);
        Py_END_ALLOW_THREADS
        result = PyLong_FromLong(status);
    }
    Py_XDECREF(scale);
    PyBuffer_Release(&nn);
    PyBuffer_Release(&L);
    return why ? why : result;
}

// weighted_attention(fn, ctx, q, kv_pages, page_tables, max_pages, L, n, scale, out, weights, weight_stride, stream) -> the same
static PyObject* call_weighted(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *q, *pages, *tables, *out, *weights, *stream;
    int32_t max_pages;
    int64_t stride;
    PyObject* why = NULL;
    Py_buffer L, nn;
    (void)self;
    if (!expect(n, 13)) return NULL;
    if (!int32_arrays(a[6], a[7], &L, &nn)) Py_RETURN_NONE;
    PyObject* result = NULL;
    PyObject* scale = NULL;
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && to_int32(a[5], a[4], 1, "max_pages", &max_pages, &why) && to_int_or_shape(a[11], a[10], -1, &stride) &&
        to_address(a[2], &q) && to_address(a[3], &pages) && has_elements(a[4], "page_tables", 4, 0, "int32", &why) &&
        is_dense(a[4], a[5], "page_tables", &why) && to_address(a[4], &tables) &&
        (scale = PyNumber_Float(a[8])) &&
        to_address(a[9], &out) && has_elements(a[10], "weights", 4, 1, "float32", &why) &&
        is_dense(a[10], a[11], "weights", &why) && to_address(a[10], &weights) && to_handle(a[12], &stream)) {
        const float s = (float)PyFloat_AS_DOUBLE(scale);
        int32_t status;
        Py_BEGIN_ALLOW_THREADS
        status = ((weighted_fn)fn)(ctx, q, pages, (const int32_t*)tables, max_pages, (const int32_t*)L.buf, (const int32_t*)nn.buf,
                                   (int32_t)L.shape[0], s, out, (float*)weights, stride, stream);
        Py_END_ALLOW_THREADS
        result = PyLong_FromLong(status);
    }
    Py_XDECREF(scale);
    PyBuffer_Release(&nn);
    PyBuffer_Release(&L);
    return why ? why : result;
}

// kv_select(fn, ctx, weights, weight_stride, length, budget, sinks, recent, keep, keep_stride, stream) -> status, or None if length is not a plain
// int32 array yet
static PyObject* call_select(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *weights, *keep, *stream;
    int64_t stride, keep_stride;
    int32_t budget, sinks, recent;
    PyObject* why = NULL;
    Py_buffer len;
    (void)self;
    if (!expect(n, 11)) return NULL;
    if (!int32_array(a[4], &len)) Py_RETURN_NONE;
    PyObject* result = NULL;
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && to_int_or_shape(a[3], a[2], -1, &stride) && to_int_or_shape(a[9], a[8], -1, &keep_stride) &&
        has_elements(a[2], "weights", 4, 1, "float32", &why) && is_dense(a[2], a[3], "weights", &why) &&
        has_elements(a[8], "keep", 4, 0, "int32", &why) && is_dense(a[8], a[9], "keep", &why) &&
        to_address(a[2], &weights) && to_int32(a[5], NULL, 0, "budget", &budget, &why) && to_int32(a[6], NULL, 0, "sinks", &sinks, &why) &&
        to_int32(a[7], NULL, 0, "recent", &recent, &why) && to_address(a[8], &keep) && to_handle(a[10], &stream)) {
        int32_t status;
        Py_BEGIN_ALLOW_THREADS
        status = ((select_fn)fn)(ctx, (const float*)weights, stride, (const int32_t*)len.buf, (int32_t)len.shape[0], budget, sinks, recent,
                                 (int32_t*)keep, keep_stride, stream);
        Py_END_ALLOW_THREADS
        result = PyLong_FromLong(status);
    }
    PyBuffer_Release(&len);
    return why ? why : result;
}

// kv_compact(fn, ctx, kv_pages, layer_stride_elems, num_layers, page_tables, max_pages, keep, keep_layer, keep_seq, keep_head, first, count, weights,
// weight_stride, stream) -> status, or None if first and count are not plain int32 arrays of one length yet
static PyObject* call_compact(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *pages, *tables, *keep, *weights, *stream;
    int64_t layer_stride, kl, ks, kh, stride = 0;
    int32_t layers, max_pages;
    PyObject* why = NULL;
    Py_buffer first, count;
    (void)self;
    if (!expect(n, 16)) return NULL;
    if (!int32_arrays(a[11], a[12], &first, &count)) Py_RETURN_NONE;
    PyObject* result = NULL;
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && to_address(a[2], &pages) && to_int(a[3], &layer_stride) &&
        to_int32(a[4], NULL, 0, "num_layers", &layers, &why) && to_int32(a[6], a[5], 1, "max_pages", &max_pages, &why) && has_elements(a[5], "page_tables", 4, 0, "int32", &why) &&
        is_dense(a[5], a[6], "page_tables", &why) && to_address(a[5], &tables) && has_elements(a[7], "keep", 4, 0, "int32", &why) &&
        has_elements(a[13], "weights", 4, 1, "float32", &why) && is_dense(a[13], a[14], "weights", &why) && to_address(a[7], &keep) && to_int(a[8], &kl) && to_int(a[9], &ks) &&
        to_int(a[10], &kh) && (a[13] == Py_None || to_int_or_shape(a[14], a[13], -1, &stride)) && to_address(a[13], &weights) && to_handle(a[15], &stream)) {
        int32_t status;
        Py_BEGIN_ALLOW_THREADS
        status = ((compact_fn)fn)(ctx, pages, layer_stride, layers, (const int32_t*)tables, max_pages, (const int32_t*)keep, kl, ks, kh,
                                  (const int32_t*)first.buf, (const int32_t*)count.buf, (int32_t)first.shape[0], (float*)weights, stride, stream);
        Py_END_ALLOW_THREADS
        result = PyLong_FromLong(status);
    }
    PyBuffer_Release(&count);
    PyBuffer_Release(&first);
    return why ? why : result;
}

static PyMethodDef kMethods[] = {
    {"kv_append", (PyCFunction)(void (*)(void))call_append, METH_FASTCALL, NULL},
    {"kv_land", (PyCFunction)(void (*)(void))call_land, METH_FASTCALL, NULL},
    {"mixed_attention", (PyCFunction)(void (*)(void))call_mixed, METH_FASTCALL, NULL},
    {"tree_attention", (PyCFunction)(void (*)(void))call_tree, METH_FASTCALL, NULL},
    {"weighted_attention", (PyCFunction)(void (*)(void))call_weighted, METH_FASTCALL, NULL},
    {"kv_select", (PyCFunction)(void (*)(void))call_select, METH_FASTCALL, NULL},
    {"kv_compact", (PyCFunction)(void (*)(void))call_compact, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "ppd_call", "Calls of libppd's per-layer entry points.", -1, kMethods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit_ppd_call(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_value = PyUnicode_InternFromString("value");
    s_shape = PyUnicode_InternFromString("shape");
    s_element_size = PyUnicode_InternFromString("element_size");
    s_is_floating_point = PyUnicode_InternFromString("is_floating_point");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    PyObject* ctypes = PyImport_ImportModule("ctypes");
    if (!ctypes) return NULL;
    t_void_p = PyObject_GetAttrString(ctypes, "c_void_p");
    f_cast = PyObject_GetAttrString(ctypes, "cast");
    Py_DECREF(ctypes);
    if (!s_data_ptr || !s_value || !s_shape || !s_element_size || !s_is_floating_point || !s_is_contiguous || !t_void_p || !f_cast) return NULL;
    return PyModule_Create(&kModule);
}
