// CPython entry to the product calls: the arguments of gemm_f32 and its siblings, handed to the library without ctypes.
//
// A small product takes the GPU 3 us, and its call took the host 4.2 us from Python, of which the library's own
// share is 1.5: the rest was a Python function, three attribute look-ups and thirteen ctypes conversions.  Here
// whole-number arguments are converted directly.  Whatever is not plain (keywords, a missing argument, anything but whole
// numbers in range, errors to be raised) goes to the ctypes function of the same name, which alone defines what is
// accepted and what is raised.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

#include <utility>

#include "gemm_routed.h"

typedef int (*product_fn)(int64_t, int64_t, int64_t, const void *, int, int64_t, const void *, int, int64_t, void *, int, int64_t,
                          void *);

static const int kProducts = 5;
static product_fn g_product[kProducts];   // null until the library is loaded
static PyObject *g_general[kProducts];    // the ctypes functions
static PyObject *g_check;                 // raises for a status
static PyObject *g_data_ptr;              // the string "data_ptr"

// a plain Python whole number that fits; false (no error set) otherwise
static inline bool whole(PyObject *x, int64_t *out)
{
    if (!PyLong_CheckExact(x)) return false;
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(x, &overflow);
    if (overflow) return false;
    *out = v;
    return true;
}

// a device address: None, a whole number, or what an object's data_ptr() returns; 0 no, 1 yes, -1 error set
static inline int address(PyObject *x, void **out)
{
    int64_t v;
    if (x == Py_None) {
        *out = nullptr;
        return 1;
    }
    if (PyLong_CheckExact(x)) {
        if (!whole(x, &v)) return 0;
        *out = (void *)(uintptr_t)v;
        return 1;
    }
    PyObject *p = PyObject_CallMethodNoArgs(x, g_data_ptr);
    if (p == nullptr) {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return -1;
        PyErr_Clear();
        return 0;
    }
    const bool ok = whole(p, &v);
    Py_DECREF(p);
    *out = (void *)(uintptr_t)v;
    return ok ? 1 : 0;
}

static PyObject *call(int which, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    int64_t n[12];
    void *ptr[4] = {nullptr, nullptr, nullptr, nullptr};  // A, B, C, stream
    bool plain = g_product[which] != nullptr && kwnames == nullptr && nargs >= 12 && nargs <= 14;
    for (int i = 0; plain && i < 12; ++i) {
        if (i == 3 || i == 6 || i == 9) {
            const int ok = address(args[i], &ptr[i / 3 - 1]);
            if (ok < 0) return nullptr;
            plain = ok != 0;
        } else {
            plain = whole(args[i], &n[i]) && (i % 3 != 1 || i < 4 || (n[i] >= INT32_MIN && n[i] <= INT32_MAX));
        }
    }
    if (plain && nargs > 12) {
        int64_t v = 0;
        plain = args[12] == Py_None || whole(args[12], &v);
        ptr[3] = (void *)(uintptr_t)v;
    }
    const bool check = nargs < 14 || args[13] == Py_True;
    if (plain && !check) plain = args[13] == Py_False;
    if (plain) {
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_product[which](n[0], n[1], n[2], ptr[0], (int)n[4], n[5], ptr[1], (int)n[7], n[8], ptr[2], (int)n[10], n[11], ptr[3]);
        Py_END_ALLOW_THREADS
        PyObject *const status = PyLong_FromLong(rc);
        if (rc == 0 || !check || status == nullptr) return status;
        PyObject *const r = PyObject_CallOneArg(g_check, status);
        Py_DECREF(status);
        return r;
    }
    return PyObject_Vectorcall(g_general[which], args, (size_t)nargs, kwnames);
}

#define PRODUCT(I, NAME, DOC)                                                                                             \
    static PyObject *py_##NAME(PyObject *, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)                     \
    {                                                                                                                      \
        return call(I, args, nargs, kwnames);                                                                              \
    }                                                                                                                      \
    PyDoc_STRVAR(doc_##NAME, #NAME "(M, N, K, A, layoutA, lda, B, layoutB, ldb, C, layoutC, ldc, stream=None, check=True)\n--\n\n" DOC);
PRODUCT(0, gemm_f32, "C = A*B, binary32. A, B, C: device addresses or tensors; stream: hipStream_t as int.")
PRODUCT(1, gemm_f16f32, "C = A*B, binary16 operands, binary32 accumulation and result.")
PRODUCT(2, gemm_f16f16, "C = A*B, binary16 operands, binary32 accumulation, C rounded to binary16 (16-bit patterns).")
PRODUCT(3, gemm_bf16f32, "C = A*B, bfloat16 operands (16-bit patterns), binary32 accumulation and result.")
PRODUCT(4, gemm_f16f32_noalloc, "gemm_f16f32 that never allocates: K-slice partials go to the library's fixed per-GPU array.")

// general(index, function): the ctypes function calls fall back to
static PyObject *py_general(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    int64_t i;
    if (nargs != 2 || !whole(args[0], &i) || i < 0 || i >= kProducts) {
        PyErr_SetString(PyExc_TypeError, "general(index, function)");
        return nullptr;
    }
    Py_INCREF(args[1]);
    Py_XSETREF(g_general[i], args[1]);
    Py_RETURN_NONE;
}

// bind(check, address, ...): what raises for a status, and the loaded library's functions in the order above
static PyObject *py_bind(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    int64_t v[kProducts];
    for (int i = 0; i < kProducts; ++i) {
        if (nargs != kProducts + 1 || !whole(args[i + 1], &v[i])) {
            PyErr_SetString(PyExc_TypeError, "bind: a function and five addresses");
            return nullptr;
        }
    }
    Py_INCREF(args[0]);
    Py_XSETREF(g_check, args[0]);
    for (int i = 0; i < kProducts; ++i) g_product[i] = (product_fn)(uintptr_t)v[i];
    Py_RETURN_NONE;
}

// ---------------------------------------------------------------------------
// The calls of gemm_routed.h, in the same way: an argument's kind follows from its type in the header.  The last one, the stream, may
// be missing; then comes `check`.
// ---------------------------------------------------------------------------
union Value { int64_t l; void *p; double f; };
enum Kind { INT, INT64, ADDRESS, FLOAT };
template <typename T> struct Argument {  // an address
    static const Kind kind = ADDRESS;
    static T of(const Value &v) { return (T)v.p; }
};
template <> struct Argument<int> {
    static const Kind kind = INT;
    static int of(const Value &v) { return (int)v.l; }
};
template <> struct Argument<int64_t> {
    static const Kind kind = INT64;
    static int64_t of(const Value &v) { return v.l; }
};
template <> struct Argument<float> {
    static const Kind kind = FLOAT;
    static float of(const Value &v) { return (float)v.f; }
};
template <typename F> struct Call;
template <typename... A> struct Call<int (*)(A...)> {
    static constexpr Kind kinds[] = {Argument<A>::kind...};
    static constexpr int count = sizeof...(A);
    template <size_t... I> static int with(void *fn, const Value *v, std::index_sequence<I...>) { return ((int (*)(A...))fn)(Argument<A>::of(v[I])...); }
    static int call(void *fn, const Value *v) { return with(fn, v, std::index_sequence_for<A...>()); }
};
struct Routed { const Kind *kinds; int count; int (*call)(void *, const Value *); };
#define CALL(NAME) {Call<decltype(&NAME)>::kinds, Call<decltype(&NAME)>::count, Call<decltype(&NAME)>::call}
static const Routed kRouted[] = {CALL(gemm_route), CALL(gemm_route_backward), CALL(gemm_route_plan), CALL(gemm_grouped),
                                 CALL(gemm_grouped_wgrad), CALL(gemm_combine), CALL(gemm_combine_backward), CALL(gemm_adapters)};
static const int kRoutedCalls = sizeof(kRouted) / sizeof(kRouted[0]), kMostArguments = 24;
static void *g_routed[kRoutedCalls];             // null until the library is loaded
static PyObject *g_routed_general[kRoutedCalls];  // the ctypes functions

static PyObject *call_routed(int which, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    const Routed &r = kRouted[which];
    const Py_ssize_t most = r.count;  // with the stream
    Value v[kMostArguments];
    bool plain = g_routed[which] != nullptr && kwnames == nullptr && nargs >= most - 1 && nargs <= most + 1;
    for (Py_ssize_t i = 0; plain && i < most - 1; ++i) {
        switch (r.kinds[i]) {
        case ADDRESS: {
            const int ok = address(args[i], &v[i].p);
            if (ok < 0) return nullptr;
            plain = ok != 0;
            break;
        }
        case FLOAT:
            plain = PyFloat_CheckExact(args[i]);
            if (plain) v[i].f = PyFloat_AS_DOUBLE(args[i]);
            break;
        default: plain = whole(args[i], &v[i].l) && (r.kinds[i] == INT64 || (v[i].l >= INT32_MIN && v[i].l <= INT32_MAX));
        }
    }
    v[most - 1].p = nullptr;
    if (plain && nargs >= most) {
        int64_t stream = 0;
        plain = args[most - 1] == Py_None || whole(args[most - 1], &stream);
        v[most - 1].p = (void *)(uintptr_t)stream;
    }
    const bool check = nargs <= most || args[most] == Py_True;
    if (plain && !check) plain = args[most] == Py_False;
    if (!plain) return PyObject_Vectorcall(g_routed_general[which], args, (size_t)nargs, kwnames);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = r.call(g_routed[which], v);
    Py_END_ALLOW_THREADS
    PyObject *const status = PyLong_FromLong(rc);
    if (rc == 0 || !check || status == nullptr) return status;
    PyObject *const raised = PyObject_CallOneArg(g_check, status);
    Py_DECREF(status);
    return raised;
}

#define ROUTED(I, NAME, SIGNATURE, DOC)                                                                                    \
    static PyObject *py_##NAME(PyObject *, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)                     \
    {                                                                                                                      \
        return call_routed(I, args, nargs, kwnames);                                                                       \
    }                                                                                                                      \
    PyDoc_STRVAR(doc_##NAME, #NAME "(" SIGNATURE ", stream=None, check=True)\n--\n\n" DOC);
ROUTED(0, gemm_route,
       "elem, tokens, experts, logits, ld, bias, score, groups, top_groups, group_top, top_k, renormalise, scale, weights, indices",
       "Scores of a router, the top_k experts of every token and their weights.")
ROUTED(1, gemm_route_backward,
       "elem, tokens, experts, logits, ld, score, top_k, renormalise, scale, indices, d_weights, d_logits, ld_d",
       "Gradient of gemm_route's weights for the logits.")
ROUTED(2, gemm_route_plan,
       "tokens, top_k, experts, indices, offsets, token_of, slot_of",
       "The tokens' entries sorted by expert: offsets of the experts' slots, a slot's token, an entry's slot.")
ROUTED(3, gemm_grouped,
       "kind, groups, offsets, rows, N, K, A, a_rows, lda, row_map, B, layoutB, ldb, strideB, C, ldc",
       "C(i,:) = A(row_map[i],:) * B_e for the rows i of every group e.")
ROUTED(4, gemm_grouped_wgrad,
       "kind, groups, offsets, rows, M, N, A, a_rows, lda, row_map, D, ldd, C, layoutC, ldc, strideC",
       "C_e = sum over the rows i of group e of A(row_map[i],:)^T * D(i,:).")
ROUTED(5, gemm_combine,
       "kind, tokens, top_k, N, Y, y_rows, ldy, slot_of, weights, out, ldo",
       "out(t,:) = sum over j of weights[t][j] * Y(slot_of[t][j],:).")
ROUTED(6, gemm_combine_backward,
       "elem, tokens, top_k, N, d_out, ldo, Y, y_rows, ldy, slot_of, weights, dY, lddy, d_weights",
       "Gradients of gemm_combine for Y and the weights.")
ROUTED(7, gemm_adapters,
       "kind, rows, N, K, A, lda, B, layoutB, ldb, adapters, rank, adapter_of, scales, down, layout_down, ld_down, stride_down, up, layout_up, ld_up, stride_up, C, ldc",
       "C(i,:) = A(i,:) * B + scales[a] * (A(i,:) * down_a) * up_a with a = adapter_of[i].")

// routed_general(index, function), routed_bind(address, ...): as general() and bind(), which says what raises for a status
static PyObject *py_routed_general(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    int64_t i;
    if (nargs != 2 || !whole(args[0], &i) || i < 0 || i >= kRoutedCalls) {
        PyErr_SetString(PyExc_TypeError, "routed_general(index, function)");
        return nullptr;
    }
    Py_INCREF(args[1]);
    Py_XSETREF(g_routed_general[i], args[1]);
    Py_RETURN_NONE;
}
static PyObject *py_routed_bind(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    int64_t v[kRoutedCalls];
    for (int i = 0; i < kRoutedCalls; ++i) {
        if (nargs != kRoutedCalls || !whole(args[i], &v[i])) {
            PyErr_SetString(PyExc_TypeError, "routed_bind: eight addresses");
            return nullptr;
        }
    }
    for (int i = 0; i < kRoutedCalls; ++i) g_routed[i] = (void *)(uintptr_t)v[i];
    Py_RETURN_NONE;
}

#define ENTRY(NAME) {#NAME, (PyCFunction)(void (*)(void))py_##NAME, METH_FASTCALL | METH_KEYWORDS, doc_##NAME}
static PyMethodDef methods[] = {ENTRY(gemm_f32), ENTRY(gemm_f16f32), ENTRY(gemm_f16f16), ENTRY(gemm_bf16f32), ENTRY(gemm_f16f32_noalloc),
                                {"general", (PyCFunction)(void (*)(void))py_general, METH_FASTCALL, nullptr},
                                {"bind", (PyCFunction)(void (*)(void))py_bind, METH_FASTCALL, nullptr},
                                ENTRY(gemm_route), ENTRY(gemm_route_backward), ENTRY(gemm_route_plan), ENTRY(gemm_grouped),
                                ENTRY(gemm_grouped_wgrad), ENTRY(gemm_combine), ENTRY(gemm_combine_backward), ENTRY(gemm_adapters),
                                {"routed_general", (PyCFunction)(void (*)(void))py_routed_general, METH_FASTCALL, nullptr},
                                {"routed_bind", (PyCFunction)(void (*)(void))py_routed_bind, METH_FASTCALL, nullptr},
                                {nullptr, nullptr, 0, nullptr}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

PyMODINIT_FUNC PyInit__binding(void)
{
    g_data_ptr = PyUnicode_InternFromString("data_ptr");
    return g_data_ptr == nullptr ? nullptr : PyModule_Create(&module);
}
