// What binding.py does for the operators over a paged key-value cache, where it takes time: looking at a dozen tensors (type, size, device, strides) and
// handing their addresses to the library.  A decoding step makes these calls once per layer, and in Python the look alone took as long as
// the launch (attn_kv_pages 3.7 of 7.8 us, attn_qkv_prepare 4.4 of 8.5); here, with the launch, a call takes 4 us.
//
// A Python module of three functions that take everything by position and return the library's code; a tensor that does not fit is a ValueError.  The
// library's functions are handed in (bind), so that there is one copy of it in the process, whoever loaded it.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

#include "sawattn.h"

namespace {

decltype(&attn_kv_pages) g_kv_pages;
decltype(&attn_qkv_prepare) g_qkv_prepare;
decltype(&attn_decode) g_decode;
int (*g_get_device)(int*);      // hipGetDevice, hipSetDevice
int (*g_set_device)(int);

struct Refused {};      // an error is set

[[noreturn]] void refuse(const char* name, const char* what) {
    PyErr_Format(PyExc_ValueError, "%s must be %s", name, what);
    throw Refused{};
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) refuse(name, "a tensor");
    return THPVariable_Unpack(o);
}

int device_of(const at::Tensor& t) { return t.is_cuda() ? (int)t.get_device() : -1; }

// Address of a contiguous tensor of n elements of this type on this device, whatever its shape; NULL for None where that is allowed.
template <typename T>
T* flat(PyObject* o, const char* name, at::ScalarType type, int64_t n, int device, bool optional = false) {
    if (optional && o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != type || t.numel() != n || device_of(t) != device || !t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous tensor of %lld elements of type %s on the other tensors' device", name,
                     (long long)n, at::toString(type));
        throw Refused{};
    }
    return static_cast<T*>(t.data_ptr());
}

struct PageTable {
    int32_t* at;
    int64_t stride;
    int wide;
    PageTable(PyObject* o, int64_t R, int device) {
        const at::Tensor& t = tensor(o, "the page table");
        if (t.scalar_type() != at::kInt || device_of(t) != device || t.dim() != 2 || t.size(0) != R || (t.size(1) > 1 && t.stride(1) != 1) ||
            t.size(1) > INT32_MAX)
            refuse("the page table", "an int32 [requests, pages] device tensor with contiguous rows");
        wide = (int)t.size(1);
        stride = R == 1 ? std::max<int64_t>(t.stride(0), wide) : t.stride(0);
        at = static_cast<int32_t*>(t.data_ptr());
    }
};

int input_type(const at::Tensor& t) { return t.scalar_type() == at::kHalf ? SAWATTN_F16 : t.scalar_type() == at::kBFloat16 ? SAWATTN_BF16 : -1; }

long long whole(PyObject* o) {
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) throw Refused{};
    return x;
}

int small(PyObject* o, const char* name) {
    const long long x = whole(o);
    if (x < INT32_MIN || x > INT32_MAX) refuse(name, "a 32-bit number");
    return (int)x;
}

float real(PyObject* o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Refused{};
    return (float)x;
}

void* pointer(PyObject* o) { return o == Py_None ? nullptr : reinterpret_cast<void*>(whole(o)); }

// The library's call with `device` current, without the interpreter's lock: a launch can wait for room in the queue.
template <typename F, typename... A>
int launch(int device, F* call, A... args) {
    PyThreadState* const state = PyEval_SaveThread();
    int before = -1, rc = SAWATTN_ERR_RUNTIME;
    const bool there = g_get_device(&before) == 0 && (before == device || g_set_device(device) == 0);
    if (there) rc = call(args...);
    if (before != device && before >= 0) (void)g_set_device(before);
    PyEval_RestoreThread(state);
    if (!there) {
        PyErr_Format(PyExc_RuntimeError, "device %d cannot be made current", device);
        throw Refused{};
    }
    return rc;
}

// Runs `f`, a binding's body: nothing leaves it but a code or a Python error.
template <typename F>
PyObject* guarded(Py_ssize_t given, Py_ssize_t wanted, F&& f) {
    try {
        if (given != wanted) {
            PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", wanted, given);
            return nullptr;
        }
        if (!g_decode) {
            PyErr_SetString(PyExc_RuntimeError, "bind has not been called");
            return nullptr;
        }
        return PyLong_FromLong(f());
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// bind(addresses of attn_kv_pages, attn_qkv_prepare, attn_decode, hipGetDevice, hipSetDevice)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "five addresses expected");
        return nullptr;
    }
    void* p[5];
    for (int i = 0; i < 5; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a null address");
            return nullptr;
        }
    }
    g_kv_pages = reinterpret_cast<decltype(g_kv_pages)>(p[0]);
    g_qkv_prepare = reinterpret_cast<decltype(g_qkv_prepare)>(p[1]);
    g_decode = reinterpret_cast<decltype(g_decode)>(p[2]);
    g_get_device = reinterpret_cast<decltype(g_get_device)>(p[3]);
    g_set_device = reinterpret_cast<decltype(g_set_device)>(p[4]);
    Py_RETURN_NONE;
}

// kv_pages(lengths, new_tokens, table, free_pages, free_state, lengths_out, granted, token_offsets, free_state_out, slots, positions, page_size,
//          stream)
PyObject* kv_pages(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&] {
        const at::Tensor& lengths = tensor(a[0], "lengths");
        const int device = device_of(lengths);
        if (device < 0) refuse("lengths", "a device tensor");
        const int64_t R = lengths.numel(), ring = tensor(a[3], "free_pages").numel(), tokens = tensor(a[9], "slots").numel();
        if (R > INT32_MAX || ring > INT32_MAX || tokens > INT32_MAX) refuse("lengths, free_pages and slots", "of fewer than 2^31 elements");
        const PageTable table(a[2], R, device);
        const auto i32 = [&](int i, const char* name, int64_t size) { return flat<int32_t>(a[i], name, at::kInt, size, device); };
        return launch(device, g_kv_pages, i32(0, "lengths", R), i32(1, "new_tokens", R), (int)R, table.at, table.stride, table.wide, small(a[11], "page_size"),
                          i32(3, "free_pages", ring), (int)ring, i32(4, "free_state", 2), i32(5, "lengths_out", R), i32(6, "granted", R),
                          i32(7, "token_offsets", R + 1), i32(8, "free_state_out", 2), flat<int64_t>(a[9], "slots", at::kLong, tokens, device),
                          i32(10, "positions", tokens), (int)tokens, pointer(a[12]));
    });
}

// qkv_prepare(q, k, v, q_out, k_out, v_out, cache address, cache device, slots, positions, q_weight, k_weight, eps, frequencies, interleaved, stream)
PyObject* qkv_prepare(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 16, [&] {
        const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k");
        const int device = device_of(q), type = input_type(q);
        const int64_t dims = q.dim();
        if (device < 0 || type < 0 || (dims != 3 && dims != 4)) refuse("q", "a [B, N, H, d] or [N, H, d] device tensor, float16 or bfloat16");
        for (int64_t i = 0; i < dims; ++i)
            if (k.dim() != dims || (i != dims - 2 && k.size(i) != q.size(i))) refuse("k", "shaped like q in all dimensions but the heads");
        for (int64_t i = 0; i < dims; ++i)
            if (q.size(i) > INT32_MAX || k.size(i) > INT32_MAX) refuse("q and k", "of fewer than 2^31 rows in each dimension");
        const int64_t B = dims == 4 ? q.size(0) : 1, N = q.size(dims - 3), H = q.size(dims - 2), KH = k.size(dims - 2), d = q.size(dims - 1);
        const auto rows = [&](int i, const char* name, const at::Tensor& like) {
            if (a[i] == Py_None) return sawattn_rows{nullptr, 0, 0, 0};
            const at::Tensor& t = tensor(a[i], name);
            if (t.sizes() != like.sizes() || t.scalar_type() != q.scalar_type() || device_of(t) != device || t.stride(dims - 1) != 1)
                refuse(name, "of q's type, on its device, shaped like q or k and contiguous in its last dimension");
            return sawattn_rows{t.data_ptr(), dims == 4 ? t.stride(0) : 0, t.stride(dims - 3), t.stride(dims - 2)};
        };
        const sawattn_qkv all = {rows(0, "q", q), rows(1, "k", k), rows(2, "v", k), rows(3, "q_out", q), rows(4, "k_out", k), rows(5, "v_out", k)};
        const auto* cache = static_cast<const sawattn_kv_cache*>(pointer(a[6]));
        if (cache && small(a[7], "cache device") != device) refuse("the cache", "on the other tensors' device");
        const int64_t half = a[13] == Py_None ? 0 : tensor(a[13], "frequencies").numel();
        if (half > INT32_MAX / 2) refuse("frequencies", "of at most d / 2 elements");
        const auto* frequencies = flat<double>(a[13], "frequencies", at::kDouble, half, device, true);
        const int interleaved = PyObject_IsTrue(a[14]);
        if (interleaved < 0) throw Refused{};
        return launch(device, g_qkv_prepare, &all, cache, flat<int64_t>(a[8], "slots", at::kLong, B * N, device, true),
                             flat<int32_t>(a[9], "positions", at::kInt, B * N, device), flat<float>(a[10], "q_weight", at::kFloat, d, device, true),
                             flat<float>(a[11], "k_weight", at::kFloat, d, device, true), real(a[12]), half ? frequencies : nullptr, (int)(2 * half),
                             interleaved, (int)B, (int)N, (int)H, (int)KH, (int)d, type, pointer(a[15]));
    });
}

// decode(Q, O, cache address, cache device, table, lengths, scale, window, workspace, stream)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&] {
        const at::Tensor &Q = tensor(a[0], "Q"), &O = tensor(a[1], "O"), &workspace = tensor(a[8], "workspace");
        const auto* cache = static_cast<const sawattn_kv_cache*>(pointer(a[2]));
        if (!cache) refuse("cache", "given");
        const int device = small(a[3], "cache device");
        if (Q.dim() != 3 || device < 0 || device_of(Q) != device || input_type(Q) != cache->dtype || Q.stride(2) != 1 || Q.size(2) != cache->d ||
            Q.size(0) > INT32_MAX || Q.size(1) > INT32_MAX)
            refuse("Q", "a [R, H, d] tensor of the cache's device, dtype and d, contiguous in its last dimension");
        const int out = O.scalar_type() == at::kFloat ? (int)SAWATTN_F32 : input_type(O);
        if (out < 0 || O.sizes() != Q.sizes() || device_of(O) != device || O.stride(2) != 1)
            refuse("O", "shaped like Q, on its device, contiguous in its last dimension (f16, bf16 or f32)");
        if (device_of(workspace) != device || !workspace.is_contiguous()) refuse("workspace", "a contiguous tensor on the other tensors' device");
        const int64_t R = Q.size(0);
        const PageTable table(a[4], R, device);
        return launch(device, g_decode, static_cast<const void*>(Q.data_ptr()), Q.stride(0), Q.stride(1), O.data_ptr(), O.stride(0), O.stride(1), out, cache, table.at, table.stride, table.wide,
                        flat<int32_t>(a[5], "lengths", at::kInt, R, device), (int)R, (int)Q.size(1), real(a[6]), small(a[7], "window"), workspace.data_ptr(),
                        workspace.nbytes(), pointer(a[9]));
    });
}

PyMethodDef g_functions[] = {{"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, nullptr},
                             {"kv_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_pages)), METH_FASTCALL, nullptr},
                             {"qkv_prepare", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(qkv_prepare)), METH_FASTCALL, nullptr},
                             {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(decode)), METH_FASTCALL, nullptr},
                             {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_paged", nullptr, -1, g_functions, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged() { return PyModule_Create(&g_module); }
