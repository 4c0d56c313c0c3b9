// cg_calls.cpp -- the calls of the draft trees and the block matrices from Python, for small sizes, where the host's time
// is most of a call's: the checks of the binding's Python functions (tree.py, block8.py) on torch tensors and the call
// of the library, without the interpreter between them. One commit with its 10 tensors 4.4 us of
// host time (10.9 by Python and ctypes; 7.0 by way of the tensors' Python attributes), a plan 3.0 (6.4; 4.7), an attention call
// 7.9 (15.3; 11.7), an encoding 3.0 (6.4; 4.5), a product 3.0 (7.7; 5.0).
//
// Each function returns the library's status, or None without having called it if anything is not as it should be;
// the Python function then looks for itself and says what. Tensors are of the type torch.Tensor itself or torch.nn.Parameter
// (which most weights are; sent the longer way from here they cost 3 us more than without this module); other subclasses take the
// longer way.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

#include <cfloat>

#include "../../include/codecgauge_block8.h"
#include "../../include/codecgauge_tree.h"

namespace {

// The entry points' own types: a call that does not fit its declaration does not compile.
struct {
    decltype(&cg_tree_plan) plan;
    decltype(&cg_tree_attention) attention;
    decltype(&cg_tree_commit) commit;
    decltype(&cg_block8_encode) encode;
    decltype(&cg_block8_matmul) matmul;
} lib;
PyObject* tensor_type;

struct Refused {};   // thrown by what follows
void need(bool ok) {
    if (!ok) throw Refused{};
}

int64_t number(PyObject* v) {
    const long long x = PyLong_AsLongLong(v);
    need(x != -1 || !PyErr_Occurred());
    return x;
}
int32_t int32_of(PyObject* v) {
    const int64_t x = number(v);
    need(x == (int32_t)x);
    return (int32_t)x;
}
void* address_of(PyObject* v) {
    void* p = PyLong_AsVoidPtr(v);
    need(p || !PyErr_Occurred());
    return p;
}

const at::Tensor& tensor(PyObject* o) {
    need((PyObject*)Py_TYPE(o) == tensor_type || THPVariable_CheckExact(o));
    return THPVariable_Unpack(o);
}
const at::Tensor& tensor(PyObject* o, at::ScalarType type, int64_t dev) {
    const at::Tensor& t = tensor(o);
    need(t.scalar_type() == type && t.get_device() == dev);
    return t;
}
template <class T = void>
T* data(const at::Tensor& t) {
    return static_cast<T*>(t.data_ptr());
}
// A contiguous array of at least n numbers.
int32_t* ints(PyObject* o, int64_t n, int64_t dev) {
    const at::Tensor& t = tensor(o, at::kInt, dev);
    need(t.numel() >= n && t.is_contiguous());
    return data<int32_t>(t);
}
int32_t elem(const at::Tensor& t) {
    need(t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf);
    return t.scalar_type() == at::kHalf ? CG_FP16 : CG_BF16;
}

// The members of the binding's Pages.
cg_pages pages_of(PyObject* v) {
    need(PyTuple_Check(v) && PyTuple_GET_SIZE(v) == 6);
    cg_pages p{};
    int32_t* to[6] = {&p.n_pages, &p.page, &p.H, &p.d, &p.n_req, &p.max_pages};
    for (int i = 0; i < 6; i++) *to[i] = int32_of(PyTuple_GET_ITEM(v, i));
    return p;
}
// A matrix whose rows are contiguous; its row stride is 0 for at most one row.
struct Matrix {
    void* p;
    int64_t rows, cols, stride;
    Matrix(PyObject* o, at::ScalarType type, int64_t dev) {
        const at::Tensor& t = tensor(o, type, dev);
        need(t.dim() == 2);
        rows = t.size(0);
        cols = t.size(1);
        need(t.stride(1) == 1 || cols <= 1);
        stride = rows > 1 ? t.stride(0) : 0;
        p = data(t);
    }
    Matrix(PyObject* o, at::ScalarType type, int64_t dev, int64_t R, int64_t K) : Matrix(o, type, dev) { need(rows == R && cols == K); }
};
float* scales(PyObject* o, int64_t R, int64_t K, int64_t rows, int64_t dev) {
    const at::Tensor& t = tensor(o, at::kFloat, dev);
    need(t.dim() == 2 && t.size(0) == (R + rows - 1) / rows && t.size(1) == (K + CG_BLOCK8 - 1) / CG_BLOCK8 && t.is_contiguous());
    return data<float>(t);
}
// [n][heads][d] with its two strides (0 where there is but one element).
void* heads(PyObject* o, at::ScalarType type, int64_t n, int64_t h, int64_t d, int64_t dev, int64_t* tok, int64_t* head) {
    const at::Tensor& t = tensor(o, type, dev);
    need(t.dim() == 3 && t.size(0) == n && t.size(1) == h && t.size(2) == d && t.stride(2) == 1);
    *tok = n > 1 ? t.stride(0) : 0;
    *head = h > 1 ? t.stride(1) : 0;
    return data(t);
}
uint32_t* mask_rows(PyObject* o, int64_t n, int64_t dev, int32_t* words) {
    const at::Tensor& t = tensor(o, at::kInt, dev);
    need(t.dim() == 2 && t.size(0) == n && t.size(1) == (int32_t)t.size(1) && t.is_contiguous());
    *words = (int32_t)t.size(1);
    return data<uint32_t>(t);
}
bool is_pool(const at::Tensor& t, const cg_pages& p, int64_t dev) {
    const int64_t k = t.dim() - 5;
    return k >= 0 && t.get_device() == dev && t.size(k) == 2 && t.size(k + 1) == p.n_pages && t.size(k + 2) == p.H && t.size(k + 3) == p.page &&
           t.size(k + 4) == p.d && t.is_contiguous();
}

template <class Fn, class... Args>
int call(Fn fn, Args... args) {
    int rc;
    Py_BEGIN_ALLOW_THREADS rc = fn(args...);
    Py_END_ALLOW_THREADS
    return rc;
}

// max_new, window, sinks, parents, seq_lens, cu_new, positions, masks, device, stream
int tree_plan(PyObject* const* a) {
    const int64_t dev = number(a[8]), r = tensor(a[4]).numel(), n = tensor(a[6]).numel();
    need(r == (int32_t)r && n == (int32_t)n);
    int32_t words;
    uint32_t* masks = mask_rows(a[7], n, dev, &words);
    return call(lib.plan, (int32_t)r, (int32_t)n, int32_of(a[0]), int32_of(a[1]), int32_of(a[2]), ints(a[3], n, dev), ints(a[4], r, dev),
                ints(a[5], r + 1, dev), ints(a[6], n, dev), masks, words, address_of(a[9]));
}

// pages, how, q, pool, block_table, seq_lens, cu_new, positions, masks, out, lse, workspace, device, stream
int tree_attention(PyObject* const* a) {
    cg_pages p = pages_of(a[0]);
    cg_paged_attn h{};
    need(PyTuple_Check(a[1]) && PyTuple_GET_SIZE(a[1]) == 5);
    h.n_rep = int32_of(PyTuple_GET_ITEM(a[1], 0));
    h.max_new = int32_of(PyTuple_GET_ITEM(a[1], 1));
    const double scale = PyFloat_AsDouble(PyTuple_GET_ITEM(a[1], 2));
    need((scale != -1.0 || !PyErr_Occurred()) && scale >= -FLT_MAX && scale <= FLT_MAX);
    h.scale = (float)scale;
    h.window = int32_of(PyTuple_GET_ITEM(a[1], 3));
    h.sinks = int32_of(PyTuple_GET_ITEM(a[1], 4));
    const int64_t dev = number(a[12]);
    const at::Tensor &pool = tensor(a[3]), &q = tensor(a[2]);
    p.dtype = elem(pool);
    need(pool.dim() == 5 && is_pool(pool, p, dev) && q.dim() == 3 && q.size(0) == (int32_t)q.size(0));
    const int64_t n = q.size(0), hq = (int64_t)p.H * h.n_rep, r = p.n_req;
    h.n_tok = (int32_t)n;
    const void* qp = heads(a[2], pool.scalar_type(), n, hq, p.d, dev, &h.q_tok, &h.q_head);
    void* op = heads(a[9], pool.scalar_type(), n, hq, p.d, dev, &h.o_tok, &h.o_head);
    int32_t words;
    const uint32_t* masks = mask_rows(a[8], n, dev, &words);
    const int32_t* positions = nullptr;
    if (a[7] == Py_None) need(h.window == 0);
    else positions = ints(a[7], n, dev);
    float* lse = nullptr;
    if (a[10] != Py_None) {
        const at::Tensor& t = tensor(a[10], at::kFloat, dev);
        need(t.numel() >= n * hq && t.is_contiguous());
        lse = data<float>(t);
    }
    const at::Tensor& workspace = tensor(a[11]);
    need(workspace.get_device() == dev && workspace.is_contiguous());
    return call(lib.attention, &p, &h, words, qp, data(pool), ints(a[4], r * p.max_pages, dev), ints(a[5], r, dev), ints(a[6], r + 1, dev), positions,
                masks, op, lse, data(workspace), workspace.nbytes(), address_of(a[13]));
}

// pages, max_new, parents, leaves, seq_lens, cu_new, block_table, pool, lens_left, free_pages, free_count, free_left, device, stream
int tree_commit(PyObject* const* a) {
    cg_pages p = pages_of(a[0]);
    const int64_t dev = number(a[12]), r = p.n_req, n = tensor(a[2]).numel();
    need(n == (int32_t)n);
    p.dtype = CG_BF16;
    int32_t layers = 0;
    void* pool = nullptr;
    if (a[7] != Py_None) {
        const at::Tensor& t = tensor(a[7]);
        p.dtype = elem(t);
        need((t.dim() == 5 || (t.dim() == 6 && t.size(0) >= 1 && t.size(0) == (int32_t)t.size(0))) && is_pool(t, p, dev));
        layers = t.dim() == 6 ? (int32_t)t.size(0) : 1;
        pool = data(t);
    }
    int32_t *left = nullptr, *free = nullptr, *count = nullptr, *free_left = nullptr;
    if (a[8] != Py_None) {
        left = ints(a[8], r, dev);
        free = ints(a[9], p.n_pages, dev);
        count = ints(a[10], 1, dev);
        free_left = ints(a[11], 1, dev);
    } else {
        need(a[9] == Py_None && a[10] == Py_None && a[11] == Py_None);
    }
    return call(lib.commit, &p, (int32_t)n, int32_of(a[1]), layers, ints(a[2], n, dev), ints(a[3], r, dev), ints(a[4], r, dev), ints(a[5], r + 1, dev),
                ints(a[6], r * p.max_pages, dev), pool, left, free, count, free_left, address_of(a[13]));
}

// x, codes, scales, rows, device, stream
int block8_encode(PyObject* const* a) {
    const int32_t rows = int32_of(a[3]);
    need(rows == 1 || rows == CG_BLOCK8);
    const int64_t dev = number(a[4]);
    const at::Tensor& t = tensor(a[0]);
    const int32_t type = elem(t);
    const Matrix x(a[0], t.scalar_type(), dev), codes(a[1], at::kFloat8_e4m3fn, dev, x.rows, x.cols);
    return call(lib.encode, type, x.rows, x.cols, rows, x.p, x.stride, codes.p, codes.stride, scales(a[2], x.rows, x.cols, rows, dev), address_of(a[5]));
}

// x, x_scales, w, w_scales, out, device, stream
int block8_matmul(PyObject* const* a) {
    const int64_t dev = number(a[5]);
    const at::Tensor& t = tensor(a[4]);
    const int32_t type = elem(t);
    const Matrix x(a[0], at::kFloat8_e4m3fn, dev), w(a[2], at::kFloat8_e4m3fn, dev);
    need(w.cols == x.cols);
    const Matrix out(a[4], t.scalar_type(), dev, x.rows, w.rows);
    return call(lib.matmul, type, x.rows, w.rows, x.cols, x.p, x.stride, scales(a[1], x.rows, x.cols, 1, dev), w.p, w.stride,
                scales(a[3], w.rows, w.cols, CG_BLOCK8, dev), out.p, out.stride, address_of(a[6]));
}

template <int (*CALL)(PyObject* const*), Py_ssize_t N>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        if (n == N) return PyLong_FromLong(CALL(args));
    } catch (...) {   // (Refused, and torch's own: a tensor without memory, for one)
    }
    PyErr_Clear();
    Py_RETURN_NONE;
}

// The type torch.Tensor, and the addresses of the five entry points.
PyObject* setup(PyObject*, PyObject* args) {
    Py_ssize_t f[5];
    PyObject* t;
    if (!PyArg_ParseTuple(args, "Onnnnn", &t, &f[0], &f[1], &f[2], &f[3], &f[4])) return nullptr;
    Py_INCREF(t);
    tensor_type = t;
    lib.plan = reinterpret_cast<decltype(lib.plan)>(f[0]);
    lib.attention = reinterpret_cast<decltype(lib.attention)>(f[1]);
    lib.commit = reinterpret_cast<decltype(lib.commit)>(f[2]);
    lib.encode = reinterpret_cast<decltype(lib.encode)>(f[3]);
    lib.matmul = reinterpret_cast<decltype(lib.matmul)>(f[4]);
    Py_RETURN_NONE;
}

template <int (*CALL)(PyObject* const*), Py_ssize_t N>
PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<CALL, N>)), METH_FASTCALL, nullptr};
}
PyMethodDef methods[] = {{"setup", setup, METH_VARARGS, nullptr}, method<tree_plan, 10>("tree_plan"), method<tree_attention, 14>("tree_attention"),
                         method<tree_commit, 14>("tree_commit"), method<block8_encode, 6>("block8_encode"),
                         method<block8_matmul, 7>("block8_matmul"), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", "Calls of libcodecgauge without the interpreter between checks and call.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", CG_TORCH_VERSION) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
