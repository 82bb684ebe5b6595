// Takes torch tensors apart for the calls whose kernels run only a few microseconds (patch_qk_norm_rope, its gradient,
// patch_kv_append, patch_prefix_attention): a CPython module that checks types, shapes and strides and calls the C ABI by address.
// Nothing else happens here -- no allocation, no kernels; the checks of sizes, alignment and device are the library's own.
// Why not ctypes: a call with four tensors of heads and twenty arguments spent 4 us in Python attribute look-ups and argument
// conversion, as much again as the launch (8.8 us against 4.6 us for a decode step's 64 tokens appended, whose kernel takes 3.4).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>
#include "../../include/patch.h"

namespace {

constexpr const char* kHeads = "heads are bf16 CUDA tensors [tokens, heads, D] whose rows hold the heads side by side";

struct Bad { const char* what; };

const at::Tensor* tensor(PyObject* o, const char* what) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw Bad{what};
    return &THPVariable_Unpack(o);
}
// rows of heads [M, H, D], any pitch; None: no heads
struct Rows { void* p = nullptr; int64_t ld = 0, M = -1, D = -1; int H = 0; };
Rows rows(PyObject* o) {
    Rows r;
    const at::Tensor* t = tensor(o, kHeads);
    if (!t) return r;
    if (!t->is_cuda() || t->scalar_type() != at::kBFloat16 || t->dim() != 3) throw Bad{kHeads};
    const auto size = t->sizes(), stride = t->strides();
    if (stride[2] != 1 || (stride[1] != size[2] && size[1] != 1) || size[1] > (1 << 20)) throw Bad{kHeads};
    r.p = t->data_ptr();
    r.M = size[0];
    r.H = int(size[1]);
    r.D = size[2];
    r.ld = r.M > 1 ? stride[0] : r.H * r.D;
    return r;
}
void same(const Rows& a, int64_t M, int64_t D, const char* what) {
    if (a.p && (a.M != M || a.D != D)) throw Bad{what};
}
// n contiguous values of a type; None: null
void* values(PyObject* o, at::ScalarType type, int64_t n, const char* what) {
    const at::Tensor* t = tensor(o, what);
    if (!t) return nullptr;
    if (!t->is_cuda() || t->scalar_type() != type || t->numel() < n || (n >= 0 && t->numel() != n) || !t->is_contiguous()) throw Bad{what};
    return t->data_ptr();
}
void* status_word(PyObject* o) {
    const at::Tensor* t = tensor(o, "status is an int32 CUDA tensor");
    if (!t) return nullptr;
    if (!t->is_cuda() || t->scalar_type() != at::kInt || t->numel() < 1) throw Bad{"status is an int32 CUDA tensor"};
    return t->data_ptr();
}
void* workspace_of(PyObject* o, size_t& bytes) {
    bytes = 0;
    const at::Tensor* t = tensor(o, "workspace is a contiguous CUDA tensor");
    if (!t) return nullptr;
    if (!t->is_cuda() || !t->is_contiguous()) throw Bad{"workspace is a contiguous CUDA tensor"};
    bytes = t->nbytes();
    return t->data_ptr();
}
template <class F> F function(PyObject* o) { return reinterpret_cast<F>(PyLong_AsVoidPtr(o)); }
void* address(PyObject* o) { return o == Py_None ? nullptr : PyLong_AsVoidPtr(o); }

// Runs `f` (-> status) and turns refusals into AssertionError.
template <class F> PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F&& f) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        return nullptr;
    }
    try {
        const int rc = f();
        return PyErr_Occurred() ? nullptr : PyLong_FromLong(rc);
    } catch (const Bad& b) {
        PyErr_SetString(PyExc_AssertionError, b.what);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
template <class F> int unlocked(F&& f) {          // the launch itself, without the interpreter's lock
    if (PyErr_Occurred()) return -1;              // a number was none: nothing is launched
    PyThreadState* s = PyEval_SaveThread();
    const int rc = f();
    PyEval_RestoreThread(s);
    return rc;
}

// (function, Q, K, wq, wk, eps, rope, positions, Q_out, K_out, status, stream)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 12, [&] {
        const Rows q = rows(a[1]), k = rows(a[2]), qo = rows(a[8]), ko = rows(a[9]);
        const int64_t M = q.p || q.M >= 0 ? q.M : k.M, D = q.M >= 0 ? q.D : k.D;
        if (M < 0 || qo.H != q.H || ko.H != k.H || (q.M >= 0 && (qo.M != M || qo.D != D)) ||
            (k.M >= 0 && (k.M != M || k.D != D || ko.M != M || ko.D != D)))
            throw Bad{"queries, keys and their results have the same tokens and D, results their inputs' heads"};
        const void* wq = values(a[3], at::kBFloat16, D, "wq: D contiguous bf16 values on the GPU");
        const void* wk = values(a[4], at::kBFloat16, D, "wk: D contiguous bf16 values on the GPU");
        const float eps = float(PyFloat_AsDouble(a[5]));
        const auto* rope = static_cast<const patch_rope_t*>(address(a[6]));
        const auto* pos = static_cast<const int32_t*>(values(a[7], at::kInt, M, "positions: an int32 value on the GPU for every token"));
        int* status = static_cast<int*>(status_word(a[10]));
        void* stream = address(a[11]);
        auto f = function<decltype(&patch_qk_norm_rope)>(a[0]);
        return unlocked([&] { return f(q.p, q.ld, q.H, k.p, k.ld, k.H, M, int(D), wq, wk, eps, rope, pos, qo.p, qo.ld, ko.p, ko.ld, status, stream); });
    });
}

// (function, gQ_out, gK_out, Q, K, wq, wk, eps, rope, positions, gQ, gK, gwq, gwk, workspace, status, stream)
PyObject* qk_norm_rope_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 17, [&] {
        const Rows gqo = rows(a[1]), gko = rows(a[2]), q = rows(a[3]), k = rows(a[4]), gq = rows(a[10]), gk = rows(a[11]);
        const int64_t M = gqo.M >= 0 ? gqo.M : gko.M, D = gqo.M >= 0 ? gqo.D : gko.D;
        const char* what = "gradients, inputs and results have the same tokens, heads and D";
        if (M < 0 || gq.H != gqo.H || gk.H != gko.H || (q.p && q.H != gqo.H) || (k.p && k.H != gko.H)) throw Bad{what};
        for (const Rows* r : {&gqo, &gko, &q, &k, &gq, &gk}) same(*r, M, D, what);
        const void* wq = values(a[5], at::kBFloat16, D, "wq: D contiguous bf16 values on the GPU");
        const void* wk = values(a[6], at::kBFloat16, D, "wk: D contiguous bf16 values on the GPU");
        const float eps = float(PyFloat_AsDouble(a[7]));
        const auto* rope = static_cast<const patch_rope_t*>(address(a[8]));
        const auto* pos = static_cast<const int32_t*>(values(a[9], at::kInt, M, "positions: an int32 value on the GPU for every token"));
        auto* gwq = static_cast<float*>(values(a[12], at::kFloat, D, "gwq: D contiguous float32 values on the GPU"));
        auto* gwk = static_cast<float*>(values(a[13], at::kFloat, D, "gwk: D contiguous float32 values on the GPU"));
        size_t bytes;
        void* ws = workspace_of(a[14], bytes);
        int* status = static_cast<int*>(status_word(a[15]));
        void* stream = address(a[16]);
        auto f = function<decltype(&patch_qk_norm_rope_backward)>(a[0]);
        return unlocked([&] {
            return f(gqo.p, gqo.ld, gko.p, gko.ld, q.p, q.ld, gqo.H, k.p, k.ld, gko.H, M, int(D), wq, wk, eps, rope, pos, gq.p, gq.ld, gk.p,
                     gk.ld, gwq, gwk, ws, bytes, status, stream);
        });
    });
}

// (function, cache, K, V, slots, wk, eps, rope, positions, Q, wq, Q_out, status, stream)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 14, [&] {
        const auto* cache = static_cast<const patch_kv_cache_t*>(address(a[1]));
        const Rows k = rows(a[2]), v = rows(a[3]), q = rows(a[9]), qo = rows(a[11]);
        const int64_t M = k.M, D = cache->D;
        const char* what = "keys and values have the cache's heads and D, all operands the same tokens";
        if (k.M < 0 || v.M != M || k.H != cache->Hkv || v.H != cache->Hkv || k.D != D || v.D != D || qo.H != q.H) throw Bad{what};
        same(q, M, D, what);
        same(qo, M, D, what);
        const auto* slots = static_cast<const int64_t*>(values(a[4], at::kLong, M, "slots: an int64 value on the GPU for every token"));
        const void* wk = values(a[5], at::kBFloat16, D, "wk: D contiguous bf16 values on the GPU");
        const float eps = float(PyFloat_AsDouble(a[6]));
        const auto* rope = static_cast<const patch_rope_t*>(address(a[7]));
        const auto* pos = static_cast<const int32_t*>(values(a[8], at::kInt, M, "positions: an int32 value on the GPU for every token"));
        const void* wq = values(a[10], at::kBFloat16, D, "wq: D contiguous bf16 values on the GPU");
        int* status = static_cast<int*>(status_word(a[12]));
        void* stream = address(a[13]);
        auto f = function<decltype(&patch_kv_append)>(a[0]);
        return unlocked([&] { return f(cache, k.p, k.ld, v.p, v.ld, slots, M, wk, eps, rope, pos, q.p, q.ld, q.H, wq, qo.p, qo.ld, status, stream); });
    });
}

// (function, cache, Q, prefix_pages, prefix_len, page_table, suffix_lens, scale, O, lse, workspace, status, stream)
PyObject* prefix_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        const auto* cache = static_cast<const patch_kv_cache_t*>(address(a[1]));
        const Rows q = rows(a[2]), o = rows(a[8]);
        const int64_t prefix_len = PyLong_AsLongLong(a[4]);
        const at::Tensor* table = tensor(a[5], "page_table is a contiguous int32 CUDA tensor [B, pages]");
        if (!table || !table->is_cuda() || table->scalar_type() != at::kInt || table->dim() != 2 || !table->is_contiguous())
            throw Bad{"page_table is a contiguous int32 CUDA tensor [B, pages]"};
        const int64_t B = table->size(0), ld = table->size(1), T = B ? q.M / B : 1;
        if (q.M < 0 || o.M != q.M || o.H != q.H || q.D != cache->D || o.D != q.D || q.M != B * T || T > (1 << 24))
            throw Bad{"Q and O are [B T, Hq, D] with the cache's D"};
        const int64_t need = prefix_len > 0 ? (prefix_len + cache->page_size - 1) / cache->page_size : 0;
        const at::Tensor* pages = tensor(a[3], "prefix_pages is a contiguous int32 CUDA tensor that covers prefix_len");
        if (need && (!pages || !pages->is_cuda() || pages->scalar_type() != at::kInt || !pages->is_contiguous() || pages->numel() < need))
            throw Bad{"prefix_pages is a contiguous int32 CUDA tensor that covers prefix_len"};
        const auto* lens = static_cast<const int32_t*>(values(a[6], at::kInt, B, "suffix_lens: an int32 value on the GPU for every sequence"));
        const float scale = a[7] == Py_None ? 1.0f / std::sqrt(float(cache->D)) : float(PyFloat_AsDouble(a[7]));
        auto* lse = static_cast<float*>(values(a[9], at::kFloat, q.M * q.H, "lse: contiguous float32 [B T, Hq] on the GPU"));
        size_t bytes;
        void* ws = workspace_of(a[10], bytes);
        int* status = static_cast<int*>(status_word(a[11]));
        void* stream = address(a[12]);
        const auto* list = need ? static_cast<const int32_t*>(pages->data_ptr()) : nullptr;
        const auto* tab = static_cast<const int32_t*>(table->data_ptr());
        auto f = function<decltype(&patch_prefix_attention)>(a[0]);
        return unlocked([&] { return f(cache, q.p, q.ld, B, int(T), q.H, list, prefix_len, tab, ld, lens, scale, o.p, o.ld, lse, ws, bytes, status, stream); });
    });
}

PyMethodDef methods[] = {
    {"qk_norm_rope", reinterpret_cast<PyCFunction>(qk_norm_rope), METH_FASTCALL, nullptr},
    {"qk_norm_rope_backward", reinterpret_cast<PyCFunction>(qk_norm_rope_backward), METH_FASTCALL, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(kv_append), METH_FASTCALL, nullptr},
    {"prefix_attention", reinterpret_cast<PyCFunction>(prefix_attention), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// PATCH_BUILT: which torch this was compiled against (build.py), looked at before anything is called
PyMODINIT_FUNC PyInit__marshal() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built", PATCH_BUILT) < 0) Py_CLEAR(m);
    return m;
}
