/* cg_calls.c -- the calls of the draft trees and the block matrices from Python, for small sizes, where the host's time
 * is most of a call's: the checks of the binding's Python functions (tree.py, block8.py) on torch tensors and the call
 * of the library, without the interpreter between them. MEASURED: one commit with its 10 tensors 7.0 us of host time
 * (11.1 by Python and ctypes), a plan 4.7 (6.7), an attention call 11.7 (16.3), an encoding 4.5 (6.7), a product 5.0
 * (7.9).
 *
 * Each function returns the library's status, or None without having called it if anything is not as it should be;
 * the Python function then looks for itself and says what. Tensors are of the type torch.Tensor itself; what is asked
 * of them goes through their Python attributes, so that nothing here depends on torch's headers. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <float.h>

#include "../../include/codecgauge_block8.h"
#include "../../include/codecgauge_tree.h"

/* The entry points' own types: a call that does not fit its declaration does not compile. */
static struct {
    __typeof__(&cg_tree_plan) plan;
    __typeof__(&cg_tree_attention) attention;
    __typeof__(&cg_tree_commit) commit;
    __typeof__(&cg_block8_encode) encode;
    __typeof__(&cg_block8_matmul) matmul;
} lib;
static PyObject *tensor_type, *t_int32, *t_float32, *t_bf16, *t_fp16, *t_e4m3;
static PyObject *s_dtype, *s_get_device, *s_numel, *s_is_contiguous, *s_data_ptr, *s_shape, *s_stride, *s_nbytes;

/* A method without arguments that returns a whole number; -1 and an error set where it does not. */
static long long number(PyObject* t, PyObject* name) {
    PyObject* r = PyObject_CallMethodNoArgs(t, name);
    if (!r) return -1;
    const long long v = PyLong_AsLongLong(r);
    Py_DECREF(r);
    return v;
}
static int is_true(PyObject* t, PyObject* name) {
    PyObject* r = PyObject_CallMethodNoArgs(t, name);
    const int yes = r == Py_True;
    Py_XDECREF(r);
    return yes;
}
/* Of which element type the tensor is (0: none) and whether it lies on the device. */
static PyObject* type_on(PyObject* t, long long dev) {
    if ((PyObject*)Py_TYPE(t) != tensor_type || number(t, s_get_device) != dev) return NULL;
    PyObject* d = PyObject_GetAttr(t, s_dtype);
    Py_XDECREF(d);   /* (the module holds the types that it compares with) */
    return d;
}
/* Where its data begins. */
static void* address(PyObject* t) {
    PyObject* r = PyObject_CallMethodNoArgs(t, s_data_ptr);
    if (!r) return NULL;
    void* p = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return p;
}
/* Shape (up to n dimensions) into dims; their number, or -1. */
static int shape_of(PyObject* t, long long* dims, int n, PyObject* name, int call) {
    PyObject* s = call ? PyObject_CallMethodNoArgs(t, name) : PyObject_GetAttr(t, name);
    if (!s || !PyTuple_Check(s) || PyTuple_GET_SIZE(s) > n) {
        Py_XDECREF(s);
        return -1;
    }
    const int k = (int)PyTuple_GET_SIZE(s);
    for (int i = 0; i < k; i++) dims[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s, i));
    Py_DECREF(s);
    return k;
}

/* A contiguous array of at least n 32-bit integers. */
static int ints(PyObject* t, long long n, long long dev, void** p) {
    if (type_on(t, dev) != t_int32 || number(t, s_numel) < n || !is_true(t, s_is_contiguous)) return 0;
    *p = address(t);
    return 1;
}
static int elem(PyObject* type) { return type == t_bf16 ? CG_BF16 : type == t_fp16 ? CG_FP16 : -1; }

static int int32_of(PyObject* v, int32_t* out) {
    const long long x = PyLong_AsLongLong(v);
    if (x != (int32_t)x || (x == -1 && PyErr_Occurred())) return 0;
    *out = (int32_t)x;
    return 1;
}
/* The members of the binding's Pages. */
static int pages_of(PyObject* v, cg_pages* p) {
    if (!PyTuple_Check(v) || PyTuple_GET_SIZE(v) != 6) return 0;
    int32_t* to[6] = {&p->n_pages, &p->page, &p->H, &p->d, &p->n_req, &p->max_pages};
    for (int i = 0; i < 6; i++)
        if (!int32_of(PyTuple_GET_ITEM(v, i), to[i])) return 0;
    return 1;
}
/* A matrix [R][K] whose rows are contiguous, and its row stride (0 for at most one row). */
static int matrix(PyObject* t, long long R, long long K, void** p, int64_t* stride) {
    long long d[2], s[2];
    if (shape_of(t, d, 2, s_shape, 0) != 2 || d[0] != R || d[1] != K || shape_of(t, s, 2, s_stride, 1) != 2 || (s[1] != 1 && K > 1)) return 0;
    *stride = R > 1 ? s[0] : 0;
    *p = address(t);
    return 1;
}
static int scales(PyObject* t, long long R, long long K, long long rows, long long dev, void** p) {
    long long d[2];
    if (type_on(t, dev) != t_float32 || shape_of(t, d, 2, s_shape, 0) != 2 || d[0] != (R + rows - 1) / rows || d[1] != (K + CG_BLOCK8 - 1) / CG_BLOCK8 ||
        !is_true(t, s_is_contiguous))
        return 0;
    *p = address(t);
    return 1;
}
/* [n][heads][d] with its two strides (0 where there is but one element). */
static int heads(PyObject* t, PyObject* type, long long n, long long h, long long d, long long dev, void** p, int64_t* tok, int64_t* head) {
    long long x[3], s[3];
    if (type_on(t, dev) != type || shape_of(t, x, 3, s_shape, 0) != 3 || x[0] != n || x[1] != h || x[2] != d || shape_of(t, s, 3, s_stride, 1) != 3 || s[2] != 1)
        return 0;
    *tok = n > 1 ? s[0] : 0;
    *head = h > 1 ? s[1] : 0;
    *p = address(t);
    return 1;
}
static int mask_rows(PyObject* t, long long n, long long dev, void** p, int32_t* words) {
    long long d[2];
    if (type_on(t, dev) != t_int32 || shape_of(t, d, 2, s_shape, 0) != 2 || d[0] != n || d[1] != (int32_t)d[1] || !is_true(t, s_is_contiguous)) return 0;
    *words = (int32_t)d[1];
    *p = address(t);
    return 1;
}

static PyObject* look(void) {
    PyErr_Clear();
    Py_RETURN_NONE;
}
#define CALL(expr)                               \
    do {                                         \
        int rc_;                                 \
        if (PyErr_Occurred()) return look();     \
        Py_BEGIN_ALLOW_THREADS rc_ = (expr);     \
        Py_END_ALLOW_THREADS                     \
        return PyLong_FromLong(rc_);             \
    } while (0)

/* max_new, window, sinks, parents, seq_lens, cu_new, positions, masks, device, stream */
static PyObject* tree_plan(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
    int32_t max_new, window, sinks, words;
    void *parents, *lens, *cu, *positions, *masks;
    if (n_args != 10 || !int32_of(a[0], &max_new) || !int32_of(a[1], &window) || !int32_of(a[2], &sinks)) return look();
    const long long dev = PyLong_AsLongLong(a[8]);
    void* stream = PyLong_AsVoidPtr(a[9]);
    if ((PyObject*)Py_TYPE(a[4]) != tensor_type || (PyObject*)Py_TYPE(a[6]) != tensor_type) return look();
    const long long r = number(a[4], s_numel), n = number(a[6], s_numel);
    if (r != (int32_t)r || n != (int32_t)n || !ints(a[3], n, dev, &parents) || !ints(a[4], r, dev, &lens) || !ints(a[5], r + 1, dev, &cu) ||
        !ints(a[6], n, dev, &positions) || !mask_rows(a[7], n, dev, &masks, &words))
        return look();
    CALL(lib.plan((int32_t)r, (int32_t)n, max_new, window, sinks, parents, lens, cu, positions, masks, words, stream));
}

/* pages, how, q, pool, block_table, seq_lens, cu_new, positions, masks, out, lse, workspace, device, stream */
static PyObject* tree_attention(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
    cg_pages p;
    cg_paged_attn h;
    int32_t words;
    long long x[5];
    void *q, *pool, *table, *lens, *cu, *positions = NULL, *masks, *out, *lse = NULL;
    if (n_args != 14 || !pages_of(a[0], &p) || !PyTuple_Check(a[1]) || PyTuple_GET_SIZE(a[1]) != 5) return look();
    const long long dev = PyLong_AsLongLong(a[12]);
    void* stream = PyLong_AsVoidPtr(a[13]);
    if (!int32_of(PyTuple_GET_ITEM(a[1], 0), &h.n_rep) || !int32_of(PyTuple_GET_ITEM(a[1], 1), &h.max_new) ||
        !int32_of(PyTuple_GET_ITEM(a[1], 3), &h.window) || !int32_of(PyTuple_GET_ITEM(a[1], 4), &h.sinks))
        return look();
    const double scale = PyFloat_AsDouble(PyTuple_GET_ITEM(a[1], 2));
    if (!(scale >= -FLT_MAX && scale <= FLT_MAX)) return look();
    h.scale = (float)scale;
    PyObject* type = type_on(a[3], dev);
    if (!type || (p.dtype = elem(type)) < 0 || shape_of(a[3], x, 5, s_shape, 0) != 5 || x[0] != 2 || x[1] != p.n_pages || x[2] != p.H ||
        x[3] != p.page || x[4] != p.d || !is_true(a[3], s_is_contiguous) || (PyObject*)Py_TYPE(a[2]) != tensor_type)
        return look();
    pool = address(a[3]);
    if (shape_of(a[2], x, 3, s_shape, 0) != 3 || x[0] != (int32_t)x[0]) return look();
    const long long n = x[0], hq = (long long)p.H * h.n_rep, r = p.n_req;
    h.n_tok = (int32_t)n;
    if (!heads(a[2], type, n, hq, p.d, dev, &q, &h.q_tok, &h.q_head) || !heads(a[9], type, n, hq, p.d, dev, &out, &h.o_tok, &h.o_head) ||
        !ints(a[4], r * p.max_pages, dev, &table) || !ints(a[5], r, dev, &lens) || !ints(a[6], r + 1, dev, &cu) ||
        (a[7] == Py_None ? h.window != 0 : !ints(a[7], n, dev, &positions)) || !mask_rows(a[8], n, dev, &masks, &words))
        return look();
    if (a[10] != Py_None) {
        if (type_on(a[10], dev) != t_float32 || number(a[10], s_numel) < n * hq || !is_true(a[10], s_is_contiguous)) return look();
        lse = address(a[10]);
    }
    if (!type_on(a[11], dev) || !is_true(a[11], s_is_contiguous)) return look();
    void* workspace = address(a[11]);
    PyObject* bytes = PyObject_GetAttr(a[11], s_nbytes);
    if (!bytes) return look();
    const size_t room = PyLong_AsSize_t(bytes);
    Py_DECREF(bytes);
    CALL(lib.attention(&p, &h, words, q, pool, table, lens, cu, positions, masks, out, lse, workspace, room, stream));
}

/* pages, max_new, parents, leaves, seq_lens, cu_new, block_table, pool, lens_left, free_pages, free_count, free_left, device, stream */
static PyObject* tree_commit(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
    cg_pages p;
    int32_t max_new, layers = 0;
    void *parents, *leaves, *lens, *cu, *table, *pool = NULL, *left = NULL, *free = NULL, *count = NULL, *free_left = NULL;
    if (n_args != 14 || !pages_of(a[0], &p) || !int32_of(a[1], &max_new)) return look();
    const long long dev = PyLong_AsLongLong(a[12]), r = p.n_req;
    void* stream = PyLong_AsVoidPtr(a[13]);
    p.dtype = CG_BF16;
    if (a[7] != Py_None) {
        long long x[6];
        PyObject* type = type_on(a[7], dev);
        const int k = type ? shape_of(a[7], x, 6, s_shape, 0) : -1;
        if (k < 5 || (p.dtype = elem(type)) < 0 || (k == 6 && (x[0] < 1 || x[0] != (int32_t)x[0])) || x[k - 5] != 2 || x[k - 4] != p.n_pages ||
            x[k - 3] != p.H || x[k - 2] != p.page || x[k - 1] != p.d || !is_true(a[7], s_is_contiguous))
            return look();
        layers = k == 6 ? (int32_t)x[0] : 1;
        pool = address(a[7]);
    }
    if ((PyObject*)Py_TYPE(a[2]) != tensor_type) return look();
    const long long n = number(a[2], s_numel);
    if (n != (int32_t)n || !ints(a[2], n, dev, &parents) || !ints(a[3], r, dev, &leaves) || !ints(a[4], r, dev, &lens) || !ints(a[5], r + 1, dev, &cu) ||
        !ints(a[6], r * p.max_pages, dev, &table))
        return look();
    if (a[8] != Py_None) {
        if (!ints(a[8], r, dev, &left) || !ints(a[9], p.n_pages, dev, &free) || !ints(a[10], 1, dev, &count) || !ints(a[11], 1, dev, &free_left)) return look();
    } else if (a[9] != Py_None || a[10] != Py_None || a[11] != Py_None) {
        return look();
    }
    CALL(lib.commit(&p, (int32_t)n, max_new, layers, parents, leaves, lens, cu, table, pool, left, free, count, free_left, stream));
}

/* x, codes, scales, rows, device, stream */
static PyObject* block8_encode(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
    int32_t rows;
    long long d[2];
    void *x, *codes, *sc;
    int64_t xs, cs;
    if (n_args != 6 || !int32_of(a[3], &rows) || (rows != 1 && rows != CG_BLOCK8)) return look();
    const long long dev = PyLong_AsLongLong(a[4]);
    void* stream = PyLong_AsVoidPtr(a[5]);
    PyObject* type = type_on(a[0], dev);
    const int e = type ? elem(type) : -1;
    if (e < 0 || shape_of(a[0], d, 2, s_shape, 0) != 2 || !matrix(a[0], d[0], d[1], &x, &xs) || type_on(a[1], dev) != t_e4m3 ||
        !matrix(a[1], d[0], d[1], &codes, &cs) || !scales(a[2], d[0], d[1], rows, dev, &sc))
        return look();
    CALL(lib.encode(e, d[0], d[1], rows, x, xs, codes, cs, sc, stream));
}

/* x, x_scales, w, w_scales, out, device, stream */
static PyObject* block8_matmul(PyObject* self, PyObject* const* a, Py_ssize_t n_args) {
    long long d[2], wd[2];
    void *x, *xsc, *w, *wsc, *out;
    int64_t xs, ws, os;
    if (n_args != 7) return look();
    const long long dev = PyLong_AsLongLong(a[5]);
    void* stream = PyLong_AsVoidPtr(a[6]);
    PyObject* type = type_on(a[4], dev);
    const int e = type ? elem(type) : -1;
    if (e < 0 || type_on(a[0], dev) != t_e4m3 || type_on(a[2], dev) != t_e4m3 || shape_of(a[0], d, 2, s_shape, 0) != 2 ||
        shape_of(a[2], wd, 2, s_shape, 0) != 2 || !matrix(a[0], d[0], d[1], &x, &xs) || !matrix(a[2], wd[0], d[1], &w, &ws) ||
        !matrix(a[4], d[0], wd[0], &out, &os) || !scales(a[1], d[0], d[1], 1, dev, &xsc) || !scales(a[3], wd[0], d[1], CG_BLOCK8, dev, &wsc))
        return look();
    CALL(lib.matmul(e, d[0], wd[0], d[1], x, xs, xsc, w, ws, wsc, out, os, stream));
}

/* The type torch.Tensor, the element types int32, float32, bfloat16, float16, float8_e4m3fn, and the addresses of the
 * five entry points. */
static PyObject* setup(PyObject* self, PyObject* args) {
    Py_ssize_t f[5];
    PyObject* t[6];
    if (!PyArg_ParseTuple(args, "OOOOOOnnnnn", &t[0], &t[1], &t[2], &t[3], &t[4], &t[5], &f[0], &f[1], &f[2], &f[3], &f[4])) return NULL;
    PyObject** to[6] = {&tensor_type, &t_int32, &t_float32, &t_bf16, &t_fp16, &t_e4m3};
    for (int i = 0; i < 6; i++) Py_XSETREF(*to[i], Py_NewRef(t[i]));
    lib.plan = (__typeof__(lib.plan))f[0];
    lib.attention = (__typeof__(lib.attention))f[1];
    lib.commit = (__typeof__(lib.commit))f[2];
    lib.encode = (__typeof__(lib.encode))f[3];
    lib.matmul = (__typeof__(lib.matmul))f[4];
    Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, NULL}
static PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, NULL}, FAST(tree_plan), FAST(tree_attention), FAST(tree_commit),
                                FAST(block8_encode), FAST(block8_matmul), {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Calls of libcodecgauge without the interpreter between checks and call.", -1, methods,
                                    NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__calls(void) {
    s_dtype = PyUnicode_InternFromString("dtype");
    s_get_device = PyUnicode_InternFromString("get_device");
    s_numel = PyUnicode_InternFromString("numel");
    s_is_contiguous = PyUnicode_InternFromString("is_contiguous");
    s_data_ptr = PyUnicode_InternFromString("data_ptr");
    s_shape = PyUnicode_InternFromString("shape");
    s_stride = PyUnicode_InternFromString("stride");
    s_nbytes = PyUnicode_InternFromString("nbytes");
    return PyModule_Create(&module);
}
