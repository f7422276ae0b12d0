// Argument marshalling of the calls a serving loop makes for every layer (CPython extension module ppd_call): the same
// conversions that the ctypes binding does, for a fifth of its time.  Each function takes the address of a libppd entry
// point first, so this module links to nothing; the GIL is released around the call.
// A small step is bound by the host: ctypes cost 1.1 us of the 4.0 us of an append call and 2.2 of the 5.6 of an
// attention call whose plan is on the device.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

static PyObject *s_data_ptr, *s_value, *s_shape, *s_stride, *s_dtype, *s_torch, *s_is_contiguous, *s_is_cuda, *s_is_pinned, *s_num_q_heads, *s_num_kv_heads, *s_head_dim;
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
// `o` as an int of 32 bits.  0 with *why set (and no error) if it does not fit: the call is refused with that message.
static int to_int32(PyObject* o, const char* name, int32_t* out, PyObject** why) {
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
// The same of 64 bits.
static int to_int64(PyObject* o, const char* name, int64_t* out, PyObject** why) {
    PyObject* v = PyNumber_Long(o);
    if (!v) return 0;
    int over;
    *out = PyLong_AsLongLongAndOverflow(v, &over);
    Py_DECREF(v);
    if (over) *why = PyUnicode_FromFormat("%s does not fit 64 bits", name);
    return !over && !PyErr_Occurred();
}
// Whether a tensor's elements are of one of two of torch's types (an address or None is taken on trust): 0 with *why set if not.  `types` holds the
// type objects once torch has been found.
typedef struct { const char* names[2]; PyObject* types[2]; } elem_types;
static elem_types t_float32 = {{"float32", "float32"}, {NULL, NULL}}, t_int32 = {{"int32", "int32"}, {NULL, NULL}}, t_mask = {{"int64", "uint64"}, {NULL, NULL}};
static elem_types t_bf16 = {{"bfloat16", "int16"}, {NULL, NULL}}, t_int64 = {{"int64", "int64"}, {NULL, NULL}};
static int has_elements(PyObject* o, const char* name, elem_types* t, PyObject** why) {
    if (o == Py_None || PyLong_Check(o)) return 1;
    if (!t->types[1]) {
        PyObject* torch = PyImport_GetModule(s_torch);
        if (!torch) return !PyErr_Occurred();  // then it is not one of its tensors
        for (int i = 0; i < 2; ++i)
            if (!t->types[i] && !(t->types[i] = PyObject_GetAttrString(torch, t->names[i]))) {
                Py_DECREF(torch);
                return 0;
            }
        Py_DECREF(torch);
    }
    PyObject* type = PyObject_GetAttr(o, s_dtype);
    if (!type) return 0;
    const int ok = type == t->types[0] || type == t->types[1];
    Py_DECREF(type);
    if (!ok) *why = PyUnicode_FromFormat("%s has to be of type %s", name, t->names[0]);
    return ok;
}
// What a handle that ppd_create of the binding has made says of its context's shape; 0 for another one
static int64_t shape_of(PyObject* ctx, PyObject* name) {
    int64_t value = 0;
    PyObject* v = PyObject_GetAttr(ctx, name);
    if (!v || !to_int(v, &value)) {
        PyErr_Clear();
        value = 0;
    }
    Py_XDECREF(v);
    return value;
}
static int64_t heads_of(PyObject* ctx) { return shape_of(ctx, s_num_kv_heads); }
// The stride of a tensor's rows: as given, or the last axis of a contiguous tensor of `outer` rows (at least; exactly, where further ones are
// addressed behind these) for each of `heads` KV heads (0: not known).
static int row_stride(PyObject* o, PyObject* stride, const char* name, int64_t outer, int64_t heads, int exact, int64_t* out, PyObject** why) {
    if (stride != Py_None || o == Py_None || PyLong_Check(o)) return to_int_or_shape(stride, o, -1, out);
    PyObject* v = PyObject_CallMethodNoArgs(o, s_is_contiguous);
    const int dense = v ? PyObject_IsTrue(v) : -1;
    Py_XDECREF(v);
    if (dense == 0) *why = PyUnicode_FromFormat("%s has to be contiguous, or its stride given", name);
    if (dense <= 0) return 0;
    PyObject* shape = PyObject_GetAttr(o, s_shape);
    if (!shape) return 0;
    if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) < 1) {
        Py_DECREF(shape);
        *why = PyUnicode_FromFormat("%s needs an axis of rows", name);
        return 0;
    }
    const Py_ssize_t axes = PyTuple_GET_SIZE(shape);
    int64_t rows = 1, axis = heads;
    for (Py_ssize_t i = 0; i < axes; ++i) {
        const int64_t len = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
        if (i == axes - 1) *out = len;
        else rows *= len;
        if (axes > 2 && i == axes - 2) axis = len;
    }
    Py_DECREF(shape);
    if (PyErr_Occurred()) return 0;
    const int64_t want = outer * (heads > 0 ? heads : 1);
    if ((heads <= 0 || axis == heads) && (!exact ? rows >= want : heads > 0 ? rows == want : want > 0 && rows % want == 0)) return 1;
    *why = heads > 0 ? PyUnicode_FromFormat("%s has %lld rows, the call needs %lld for each of %lld KV heads", name, (long long)rows, (long long)outer, (long long)heads)
                     : PyUnicode_FromFormat("%s has %lld rows, the call needs %lld for each KV head", name, (long long)rows, (long long)outer);
    return 0;
}
// The same in 32 bits, of a tensor of `outer` rows
static int row_stride32(PyObject* o, PyObject* stride, const char* name, const char* stride_name, int64_t outer, int32_t* out, PyObject** why) {
    int64_t wide;
    if (stride != Py_None) return to_int32(stride, stride_name, out, why);
    if (!row_stride(o, stride, name, outer, 0, 0, &wide, why)) return 0;
    *out = wide <= INT32_MAX ? (int32_t)wide : INT32_MAX;
    return 1;
}
// A tensor [rows][heads][dim] whose heads lie side by side: its row stride (as given, or the tensor's), and its heads.  It has to have `rows` rows at
// least, and *heads heads of `dim` elements where these are known (not 0).  *width, where asked for: elements of a row.  An address needs its
// stride given.
static int head_rows(PyObject* o, PyObject* given, const char* name, int64_t rows, int64_t dim, int64_t* heads, int64_t* stride, int64_t* width, PyObject** why) {
    if (o == Py_None || PyLong_Check(o)) {
        *stride = 0;
        if (given != Py_None) return to_int64(given, "a stride", stride, why);
        if (o == Py_None || rows <= 1) return 1;
        *why = PyUnicode_FromFormat("%s is an address: its stride has to be given", name);
        return 0;
    }
    if (!has_elements(o, name, &t_bf16, why)) return 0;
    int64_t shape[3], strides[3];
    PyObject* s = PyObject_GetAttr(o, s_shape);
    PyObject* t = s ? PyObject_CallMethodNoArgs(o, s_stride) : NULL;
    int ok = s && t;
    if (ok && (!PyTuple_Check(s) || !PyTuple_Check(t) || PyTuple_GET_SIZE(s) != 3 || PyTuple_GET_SIZE(t) != 3)) {
        *why = PyUnicode_FromFormat("%s has to have three axes: rows, heads, elements", name);
        ok = 0;
    }
    for (int i = 0; ok && i < 3; ++i) {
        shape[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, i));
        strides[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(t, i));
        ok = !PyErr_Occurred();
    }
    Py_XDECREF(t);
    Py_XDECREF(s);
    if (!ok) return 0;
    if (shape[0] < rows || (*heads > 0 && shape[1] != *heads) || (dim > 0 && shape[2] != dim)) {
        *why = PyUnicode_FromFormat("%s is [%lld][%lld][%lld], the call needs %lld rows of %lld heads of %lld (0: any)", name, (long long)shape[0],
                                    (long long)shape[1], (long long)shape[2], (long long)rows, (long long)*heads, (long long)dim);
        return 0;
    }
    if (strides[2] != 1 || (shape[1] > 1 && strides[1] != shape[2]) || (rows > 1 && given != Py_None)) {
        *why = strides[2] != 1 || (shape[1] > 1 && strides[1] != shape[2]) ? PyUnicode_FromFormat("the heads of a row of %s have to be contiguous", name)
                                                                          : PyUnicode_FromFormat("%s is a tensor: its stride is its own", name);
        return 0;
    }
    *heads = shape[1];
    *stride = strides[0];
    if (width) *width = shape[1] * shape[2];
    return 1;
}
// The same of rows without gaps, or an address
static int dense_rows(PyObject* o, const char* name, int64_t rows, int64_t dim, int64_t* heads, PyObject** why) {
    int64_t stride, width;
    if (o == Py_None || PyLong_Check(o)) return 1;
    if (!head_rows(o, Py_None, name, rows, dim, heads, &stride, &width, why)) return 0;
    if (rows <= 1 || stride == width) return 1;
    *why = PyUnicode_FromFormat("%s has to be contiguous", name);
    return 0;
}
// A contiguous int64 tensor of `rows` elements at least (`counted`: these are as many as it says itself), or an address
static int int64_vector(PyObject* o, const char* name, int64_t rows, int counted, PyObject** why) {
    int64_t have = rows;
    if (o == Py_None || PyLong_Check(o)) return 1;
    if (!has_elements(o, name, &t_int64, why) || (!counted && !to_int_or_shape(Py_None, o, 0, &have))) return 0;
    if (have >= rows && rows <= 1) return 1;
    PyObject* v = PyObject_CallMethodNoArgs(o, s_is_contiguous);
    const int dense = v ? PyObject_IsTrue(v) : -1;
    Py_XDECREF(v);
    if (dense < 0) return 0;
    if (dense && have >= rows) return 1;
    *why = dense ? PyUnicode_FromFormat("%s has %lld elements, the call needs %lld", name, (long long)have, (long long)rows) : PyUnicode_FromFormat("%s has to be contiguous", name);
    return 0;
}
// `o` as an int, or the length of a tensor's first axis if it is None; an address needs it given
static int row_count(PyObject* o, PyObject* x, const char* name, int64_t* out, PyObject** why) {
    if (o == Py_None && (x == Py_None || PyLong_Check(x))) {
        *why = PyUnicode_FromFormat("%s is an address: T has to be given", name);
        return 0;
    }
    return o != Py_None ? to_int64(o, "T", out, why) : to_int_or_shape(o, x, 0, out);
}
// Whether the GPU reaches a tensor's memory: kernels that were given other host memory's addresses would fault.  An address or None is taken on
// trust; so is everything where there is no context, which the library refuses.
static int on_gpu(void* ctx, PyObject* o, const char* name, PyObject** why) {
    if (!ctx || o == Py_None || PyLong_Check(o)) return 1;
    PyObject* v = PyObject_GetAttr(o, s_is_cuda);
    if (!v) {
        PyErr_Clear();  // not one of torch's tensors
        return 1;
    }
    int ok = v == Py_True;
    Py_DECREF(v);
    if (ok) return 1;
    v = PyObject_CallMethodNoArgs(o, s_is_pinned);
    ok = v ? PyObject_IsTrue(v) : -1;
    Py_XDECREF(v);
    if (ok == 0) *why = PyUnicode_FromFormat("%s has to be on the GPU", name);
    return ok > 0;
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
    int64_t rows = 0;
    for (Py_ssize_t i = 0; i < nn.shape[0]; ++i) rows += ((const int32_t*)nn.buf)[i];
    PyObject* result = NULL;
    PyObject* scale = NULL;
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && row_stride32(a[4], a[5], "page_tables", "max_pages", L.shape[0], &max_pages, &why) &&
        row_stride32(a[6], a[7], "tree_mask", "mask_words", rows, &words, &why) &&
        to_address(a[2], &q) && to_address(a[3], &pages) && has_elements(a[4], "page_tables", &t_int32, &why) && to_address(a[4], &tables) &&
        has_elements(a[6], "tree_mask", &t_mask, &why) && to_address(a[6], &mask) &&
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
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && row_stride32(a[4], a[5], "page_tables", "max_pages", L.shape[0], &max_pages, &why) &&
        row_stride(a[10], a[11], "weights", L.shape[0], heads_of(a[1]), 0, &stride, &why) &&
        to_address(a[2], &q) && to_address(a[3], &pages) && has_elements(a[4], "page_tables", &t_int32, &why) && to_address(a[4], &tables) &&
        (scale = PyNumber_Float(a[8])) && to_address(a[9], &out) && has_elements(a[10], "weights", &t_float32, &why) && to_address(a[10], &weights) && to_handle(a[12], &stream)) {
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
    const int64_t heads = heads_of(a[1]);
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && row_stride(a[2], a[3], "weights", len.shape[0], heads, 0, &stride, &why) &&
        row_stride(a[8], a[9], "keep", len.shape[0], heads, 0, &keep_stride, &why) &&
        has_elements(a[2], "weights", &t_float32, &why) && has_elements(a[8], "keep", &t_int32, &why) &&
        to_address(a[2], &weights) && to_int32(a[5], "budget", &budget, &why) && to_int32(a[6], "sinks", &sinks, &why) &&
        to_int32(a[7], "recent", &recent, &why) && to_address(a[8], &keep) && to_handle(a[10], &stream)) {
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
        to_int32(a[4], "num_layers", &layers, &why) && row_stride32(a[5], a[6], "page_tables", "max_pages", first.shape[0], &max_pages, &why) &&
        has_elements(a[5], "page_tables", &t_int32, &why) && to_address(a[5], &tables) && has_elements(a[7], "keep", &t_int32, &why) &&
        has_elements(a[13], "weights", &t_float32, &why) &&
        (a[13] == Py_None || row_stride(a[13], a[14], "weights", layers * (int64_t)first.shape[0], heads_of(a[1]), layers > 1 && first.shape[0] > 0, &stride, &why)) &&
        to_address(a[7], &keep) && to_int(a[8], &kl) && to_int(a[9], &ks) && to_int(a[10], &kh) && to_address(a[13], &weights) && to_handle(a[15], &stream)) {
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

typedef int32_t (*rope_fn)(void*, const void*, int64_t, int32_t, const int64_t*, int64_t, int32_t, void*, int64_t, void*);
typedef int32_t (*append_rotated_fn)(void*, const void*, int64_t, const void*, int64_t, const void*, int64_t, const int64_t*, void*, const int64_t*, int64_t, void*, void*);

// rope(fn, ctx, x, x_stride, heads, positions, T, transpose, out, out_stride, stream) -> status, or, for arguments that cannot be passed on, a message
static PyObject* call_rope(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *x, *positions, *out, *stream;
    int64_t T, heads = 0, x_stride, out_stride;
    int32_t heads32;
    PyObject* why = NULL;
    (void)self;
    if (!expect(n, 11)) return NULL;
    const int64_t dim = shape_of(a[1], s_head_dim);
    if (a[4] != Py_None) {
        if (!to_int32(a[4], "heads", &heads32, &why)) return why;
        heads = heads32;
    }
    const int transpose = PyObject_IsTrue(a[7]);
    if (transpose >= 0 && to_handle(a[0], &fn) && to_handle(a[1], &ctx) && row_count(a[6], a[5], "positions", &T, &why) && int64_vector(a[5], "positions", T, a[6] == Py_None, &why) &&
        head_rows(a[2], a[3], "x", T, dim, &heads, &x_stride, NULL, &why) && head_rows(a[8], a[9], "out", T, dim, &heads, &out_stride, NULL, &why) &&
        on_gpu(ctx, a[2], "x", &why) && on_gpu(ctx, a[5], "positions", &why) && on_gpu(ctx, a[8], "out", &why) &&
        to_address(a[2], &x) && to_address(a[5], &positions) && to_address(a[8], &out) && to_handle(a[10], &stream)) {
        int32_t status;
        Py_BEGIN_ALLOW_THREADS
        status = ((rope_fn)fn)(ctx, x, x_stride, (int32_t)(heads <= INT32_MAX ? heads : INT32_MAX), (const int64_t*)positions, T, transpose, out, out_stride, stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    }
    return why;
}

// kv_append_rotated(fn, ctx, q, q_stride, k, k_stride, v, v_stride, positions, kv_pages, slot_mapping, T, q_out, stream) -> the same
static PyObject* call_append_rotated(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *q, *k, *v, *positions, *pages, *slots, *q_out, *stream;
    int64_t T, q_stride, k_stride, v_stride;
    PyObject* why = NULL;
    (void)self;
    if (!expect(n, 14)) return NULL;
    const int64_t dim = shape_of(a[1], s_head_dim);
    int64_t hq = shape_of(a[1], s_num_q_heads), hkv = shape_of(a[1], s_num_kv_heads);
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && row_count(a[11], a[10], "slot_mapping", &T, &why) && int64_vector(a[10], "slot_mapping", T, a[11] == Py_None, &why) &&
        int64_vector(a[8], "positions", T, 0, &why) && head_rows(a[2], a[3], "q", T, dim, &hq, &q_stride, NULL, &why) &&
        dense_rows(a[12], "q_out", T, dim, &hq, &why) &&
        head_rows(a[4], a[5], "k", T, dim, &hkv, &k_stride, NULL, &why) && head_rows(a[6], a[7], "v", T, dim, &hkv, &v_stride, NULL, &why) &&
        on_gpu(ctx, a[2], "q", &why) && on_gpu(ctx, a[4], "k", &why) && on_gpu(ctx, a[6], "v", &why) && on_gpu(ctx, a[8], "positions", &why) &&
        on_gpu(ctx, a[10], "slot_mapping", &why) && on_gpu(ctx, a[12], "q_out", &why) &&
        to_address(a[2], &q) && to_address(a[4], &k) && to_address(a[6], &v) && to_address(a[8], &positions) && to_address(a[9], &pages) &&
        to_address(a[10], &slots) && to_address(a[12], &q_out) && to_handle(a[13], &stream)) {
        int32_t status;
        Py_BEGIN_ALLOW_THREADS
        status = ((append_rotated_fn)fn)(ctx, q, q_stride, k, k_stride, v, v_stride, (const int64_t*)positions, pages, (const int64_t*)slots, T, q_out, stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(status);
    }
    return why;
}

typedef int32_t (*prefix_fn)(void*, const void*, const void*, const int32_t*, int32_t, const int32_t*, const int32_t*, const int32_t*, int32_t, float, void*, void*);

// prefix_attention(fn, ctx, q, kv_pages, page_tables, max_pages, shared, L, n, scale, out, stream) -> status, or None if shared, L and n are not plain
// int32 arrays of one length yet, or, for arguments that cannot be passed on, a message
static PyObject* call_prefix(PyObject* self, PyObject* const* a, Py_ssize_t n) {
    void *fn, *ctx, *q, *pages, *tables, *out, *stream;
    int32_t max_pages;
    PyObject* why = NULL;
    Py_buffer shared, L, nn;
    (void)self;
    if (!expect(n, 12)) return NULL;
    if (!int32_arrays(a[7], a[8], &L, &nn)) Py_RETURN_NONE;
    const int plain = int32_array(a[6], &shared);
    if (!plain || shared.shape[0] != L.shape[0]) {
        if (plain) PyBuffer_Release(&shared);
        PyBuffer_Release(&nn);
        PyBuffer_Release(&L);
        Py_RETURN_NONE;
    }
    PyObject* result = NULL;
    PyObject* scale = NULL;
    const int64_t dim = shape_of(a[1], s_head_dim);
    int64_t rows = 0, hq = shape_of(a[1], s_num_q_heads);
    for (Py_ssize_t i = 0; i < nn.shape[0]; ++i) rows += ((const int32_t*)nn.buf)[i];
    if (to_handle(a[0], &fn) && to_handle(a[1], &ctx) && row_stride32(a[4], a[5], "page_tables", "max_pages", L.shape[0], &max_pages, &why) &&
        has_elements(a[4], "page_tables", &t_int32, &why) && dense_rows(a[2], "q", rows, dim, &hq, &why) && dense_rows(a[10], "out", rows, dim, &hq, &why) &&
        on_gpu(ctx, a[2], "q", &why) && on_gpu(ctx, a[4], "page_tables", &why) && on_gpu(ctx, a[10], "out", &why) &&
        to_address(a[2], &q) && to_address(a[3], &pages) && to_address(a[4], &tables) && (scale = PyNumber_Float(a[9])) && to_address(a[10], &out) &&
        to_handle(a[11], &stream)) {
        const float s = (float)PyFloat_AS_DOUBLE(scale);
        int32_t status;
        Py_BEGIN_ALLOW_THREADS
        status = ((prefix_fn)fn)(ctx, q, pages, (const int32_t*)tables, max_pages, (const int32_t*)shared.buf, (const int32_t*)L.buf, (const int32_t*)nn.buf,
                                 (int32_t)L.shape[0], s, out, stream);
        Py_END_ALLOW_THREADS
        result = PyLong_FromLong(status);
    }
    Py_XDECREF(scale);
    PyBuffer_Release(&shared);
    PyBuffer_Release(&nn);
    PyBuffer_Release(&L);
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
    {"rope", (PyCFunction)(void (*)(void))call_rope, METH_FASTCALL, NULL},
    {"prefix_attention", (PyCFunction)(void (*)(void))call_prefix, METH_FASTCALL, NULL},
    {"kv_append_rotated", (PyCFunction)(void (*)(void))call_append_rotated, METH_FASTCALL, NULL},
    {NULL, NULL, 0, NULL},
};
static struct PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "ppd_call", "Calls of libppd's per-layer entry points.", -1, kMethods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit_ppd_call(void) {
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_value = PyUnicode_InternFromString("value");
    s_shape = PyUnicode_InternFromString("shape");
    s_dtype = PyUnicode_InternFromString("dtype");
    s_torch = PyUnicode_InternFromString("torch");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_is_cuda = PyUnicode_InternFromString("is_cuda");
    s_is_pinned = PyUnicode_InternFromString("is_pinned");
    s_num_kv_heads = PyUnicode_InternFromString("num_kv_heads");
    s_num_q_heads = PyUnicode_InternFromString("num_q_heads");
    s_head_dim = PyUnicode_InternFromString("head_dim");
    s_stride = PyUnicode_InternFromString("stride");
    PyObject* ctypes = PyImport_ImportModule("ctypes");
    if (!ctypes) return NULL;
    t_void_p = PyObject_GetAttrString(ctypes, "c_void_p");
    f_cast = PyObject_GetAttrString(ctypes, "cast");
    Py_DECREF(ctypes);
    if (!s_data_ptr || !s_value || !s_shape || !s_dtype || !s_torch || !s_is_contiguous || !s_is_cuda || !s_is_pinned || !s_num_kv_heads || !s_num_q_heads || !s_head_dim || !s_stride || !t_void_p || !f_cast) return NULL;
    return PyModule_Create(&kModule);
}
