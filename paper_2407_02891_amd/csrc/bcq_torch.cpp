// The serving operators' objects (serving.py) in native code: what a call checks, allocates and passes on, over torch tensors.
//
// A call of a few tokens is over on the GPU in 3 to 10 us; its checks and its two allocations took 9 to 14 us in Python and take about 2 here.  Nothing here
// computes: the entry points of include/bcq.h do, through the library that bind() is given.  Errors are raised as the package's BcqError.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <dlfcn.h>

#include <string>

#include "../../include/bcq.h"

namespace {

PyObject *g_error = nullptr;  // BcqError
struct {
    decltype(&bcq_rotate) rotate;
    decltype(&bcq_attend) attend;
    decltype(&bcq_attend_workspace_bytes) attend_workspace_bytes;
    decltype(&bcq_lora) lora;
    decltype(&bcq_lora_workspace_bytes) lora_workspace_bytes;
} g_bcq;

// A refusal or a failed call, on its way to Python.
struct Refused {
    int status;
    std::string where;
};

[[noreturn]] void refuse(const char *where, const std::string &what) { throw Refused{BCQ_ERR_INVALID_ARG, std::string(where) + " (" + what + ")"}; }

const at::Tensor &tensor(PyObject *o, const char *where, const char *name)
{
    if (!THPVariable_Check(o)) refuse(where, std::string(name) + ": a tensor");
    return THPVariable_Unpack(o);
}

// What the tensors of a call have in common with those that the object holds.
struct Place {
    at::ScalarType type;
    c10::Device device;
    const char *where;

    int64_t rows(const at::Tensor &t, const char *name, int64_t rows, int64_t cols) const  // the row stride of a matrix whose rows are contiguous
    {
        if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols || t.scalar_type() != type || t.device() != device || (t.stride(1) != 1 && cols > 1))
            refuse(where, std::string(name) + ": [" + std::to_string(rows) + "][" + std::to_string(cols) + "] of " + c10::toString(type) + " on " +
                              device.str() + ", rows contiguous");
        return rows > 1 ? t.stride(0) : cols;  // (the stride of a lone row means nothing)
    }
    const int32_t *ints(PyObject *o, const char *name, int64_t n) const
    {
        const at::Tensor &t = tensor(o, where, name);
        if (t.scalar_type() != at::kInt || t.dim() != 1 || t.size(0) != n || t.device() != device || !t.is_contiguous())
            refuse(where, std::string(name) + ": contiguous int32 of " + std::to_string(n) + " on " + device.str());
        return static_cast<const int32_t *>(t.data_ptr());
    }
    const void *weight(PyObject *o, const char *name, int64_t n) const
    {
        if (o == Py_None) return nullptr;
        const at::Tensor &t = tensor(o, where, name);
        if (t.scalar_type() != type || t.dim() != 1 || t.size(0) != n || t.device() != device || !t.is_contiguous())
            refuse(where, std::string(name) + ": contiguous [" + std::to_string(n) + "] of " + c10::toString(type) + " on " + device.str());
        return t.data_ptr();
    }
    at::Tensor fresh(int64_t rows, int64_t cols) const { return at::empty({rows, cols}, at::TensorOptions().dtype(type).device(device)); }
    at::Tensor scratch(size_t bytes) const { return at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(device)); }
};

int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{-1, ""};
    return v;
}
// An int32 argument of the C interface.
int32_t int32(PyObject *o, const char *where, const char *name)
{
    const int64_t v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) refuse(where, std::string(name) + ": beyond 32 bits");
    return (int32_t)v;
}
double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{-1, ""};
    return v;
}
bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused{-1, ""};
    return v;
}

void succeeded(bcq_status status, const char *where)
{
    if (status != BCQ_OK) throw Refused{status, where};
}

// One of the functions below, with its argument count checked and what it throws turned into Python's errors.
template <int COUNT, at::Tensor (*CALL)(PyObject *const *)>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != COUNT) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected", COUNT);
        return nullptr;
    }
    try {
        return THPVariable_Wrap(CALL(args));
    } catch (const Refused &r) {
        if (!PyErr_Occurred()) {
            PyObject *what = Py_BuildValue("(is)", r.status, r.where.c_str());
            if (what) PyErr_SetObject(g_error, what);
            Py_XDECREF(what);
        }
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

template <class T>
T *address(PyObject *o)
{
    return reinterpret_cast<T *>(integer(o));
}

// What rows are divided by (the entry points check the rest of the cache).
int64_t head_dim(const bcq_cache &c, const char *where)
{
    if (c.head_dim < 1) refuse(where, "cache: heads without elements");
    return c.head_dim;
}

// rotate(desc, k, v, qkv, positions, cos_sin, slots, q_weight, k_weight, eps, interleaved, out, stream)
at::Tensor rotate(PyObject *const *a)
{
    const char *const where = "PagedCache.rotate";
    const bcq_cache *const c = address<const bcq_cache>(a[0]);
    const at::Tensor &k = tensor(a[1], where, "k"), &v = tensor(a[2], where, "v"), &qkv = tensor(a[3], where, "qkv");
    const Place place{k.scalar_type(), k.device(), where};
    const c10::DeviceGuard there(place.device);  // (launches go to the current device)
    const int64_t D = head_dim(*c, where);
    if (qkv.dim() != 2 || qkv.size(1) % D || qkv.size(1) / D <= 2 * (int64_t)c->kv_heads)
        refuse(where, "qkv: [tokens][heads * head_dim], at least one q head before the k and v heads");
    const int64_t T = qkv.size(0), q_heads = qkv.size(1) / D - 2 * c->kv_heads;
    if (T > INT32_MAX || q_heads > INT32_MAX) refuse(where, "qkv: too large");
    const int64_t ld = place.rows(qkv, "qkv", T, qkv.size(1));
    const int32_t *const positions = place.ints(a[4], "positions", T), *const slots = place.ints(a[6], "slots", T);
    const float *table = nullptr;
    int64_t most = 1, rot = 0;
    if (a[5] != Py_None) {
        const at::Tensor &t = tensor(a[5], where, "cos_sin");
        if (t.dim() != 2 || t.scalar_type() != at::kFloat || t.device() != place.device || !t.is_contiguous() || t.size(0) > INT32_MAX || t.size(1) > INT32_MAX)
            refuse(where, "cos_sin: contiguous float32 [positions][rot_dim]");
        most = t.size(0), rot = t.size(1), table = static_cast<const float *>(t.data_ptr());
    }
    const void *const q_weight = place.weight(a[7], "q_weight", D), *const k_weight = place.weight(a[8], "k_weight", D);
    const at::Tensor out = a[11] == Py_None ? place.fresh(T, q_heads * D) : tensor(a[11], where, "out");
    const int64_t ld_q = place.rows(out, "out", T, q_heads * D);
    succeeded(g_bcq.rotate(c, (int32_t)T, (int32_t)q_heads, qkv.data_ptr(), ld, positions, table, (int32_t)most, (int32_t)rot, truth(a[10]), q_weight,
                           k_weight, (float)number(a[9]), out.data_ptr(), ld_q, slots, k.data_ptr(), v.data_ptr(), address<void>(a[12])),
              where);
    return out;
}

// attend(desc, k, v, q, q_start, kv_len, pages, max_new, scale, causal, window, out, stream)
at::Tensor attend(PyObject *const *a)
{
    const char *const where = "PagedCache.attend";
    const bcq_cache *const c = address<const bcq_cache>(a[0]);
    const at::Tensor &k = tensor(a[1], where, "k"), &v = tensor(a[2], where, "v"), &q = tensor(a[3], where, "q"), &pages = tensor(a[6], where, "pages");
    const Place place{k.scalar_type(), k.device(), where};
    const c10::DeviceGuard there(place.device);  // (launches go to the current device)
    const int64_t D = head_dim(*c, where);
    if (q.dim() != 2 || q.size(1) % D) refuse(where, "q: [tokens][q_heads * head_dim]");
    if (pages.dim() != 2 || pages.scalar_type() != at::kInt || pages.device() != place.device || !pages.is_contiguous())
        refuse(where, "pages: contiguous int32 [requests][max_pages]");
    const int64_t T = q.size(0), R = pages.size(0), max_pages = pages.size(1), q_heads = q.size(1) / D;
    if (T > INT32_MAX || R > INT32_MAX - 1 || max_pages > INT32_MAX || q_heads > INT32_MAX) refuse(where, "q or pages: too large");
    const int64_t ld = place.rows(q, "q", T, q.size(1));
    const int32_t *const q_start = place.ints(a[4], "q_start", R + 1), *const kv_len = place.ints(a[5], "kv_len", R);
    const int32_t max_new = int32(a[7], where, "max_new"), window = int32(a[10], where, "window");
    const at::Tensor out = a[11] == Py_None ? place.fresh(T, q.size(1)) : tensor(a[11], where, "out");
    const int64_t ld_out = place.rows(out, "out", T, q.size(1));
    const size_t bytes = g_bcq.attend_workspace_bytes(c, (int32_t)T, (int32_t)R, (int32_t)q_heads, (int32_t)max_pages, max_new);
    const at::Tensor workspace = bytes ? place.scratch(bytes) : at::Tensor();
    succeeded(g_bcq.attend(c, k.data_ptr(), v.data_ptr(), (int32_t)T, (int32_t)R, (int32_t)q_heads, q.data_ptr(), ld, q_start, kv_len,
                           static_cast<const int32_t *>(pages.data_ptr()), (int32_t)max_pages, max_new, (float)number(a[8]), truth(a[9]), window,
                           out.data_ptr(), ld_out, bytes ? workspace.data_ptr() : nullptr, address<void>(a[12])),
              where);
    return out;
}

// add(desc, A, B, rank, scale, X, adapter, base, out, stream); rank and scale are addresses or None
at::Tensor add(PyObject *const *a)
{
    const char *const where = "Adapters.add";
    const bcq_adapters *const d = address<const bcq_adapters>(a[0]);
    const at::Tensor &A = tensor(a[1], where, "A"), &B = tensor(a[2], where, "B"), &X = tensor(a[5], where, "X"), &base = tensor(a[7], where, "base");
    const Place place{A.scalar_type(), A.device(), where};
    const c10::DeviceGuard there(place.device);
    if (X.dim() != 2 || X.size(0) > INT32_MAX) refuse(where, "X: [tokens][N]");
    const int64_t T = X.size(0), ldx = place.rows(X, "X", T, d->N), ld_base = place.rows(base, "base", T, d->M);
    const int32_t *const adapter = place.ints(a[6], "adapter", T);
    const at::Tensor out = a[8] == Py_None ? place.fresh(T, d->M) : tensor(a[8], where, "out");
    const int64_t ldy = place.rows(out, "out", T, d->M);
    const size_t bytes = g_bcq.lora_workspace_bytes(d, (int32_t)T);
    const at::Tensor workspace = bytes ? place.scratch(bytes) : at::Tensor();
    succeeded(g_bcq.lora(d, A.data_ptr(), B.data_ptr(), a[3] == Py_None ? nullptr : address<const int32_t>(a[3]),
                         a[4] == Py_None ? nullptr : address<const float>(a[4]), (int32_t)T, adapter, X.data_ptr(), ldx, base.data_ptr(), ld_base, out.data_ptr(),
                         ldy, bytes ? workspace.data_ptr() : nullptr, address<void>(a[9])),
              where);
    return out;
}

// bind(handle of libbcq, BcqError)
PyObject *bind(PyObject *, PyObject *args)
{
    unsigned long long handle;
    PyObject *error;
    if (!PyArg_ParseTuple(args, "KO", &handle, &error)) return nullptr;
    void *const lib = reinterpret_cast<void *>(handle);
    const auto find = [&](auto &to, const char *name) {
        to = reinterpret_cast<std::remove_reference_t<decltype(to)>>(dlsym(lib, name));
        if (!to) PyErr_Format(PyExc_RuntimeError, "libbcq has no %s", name);
        return to != nullptr;
    };
    if (!find(g_bcq.rotate, "bcq_rotate") || !find(g_bcq.attend, "bcq_attend") || !find(g_bcq.attend_workspace_bytes, "bcq_attend_workspace_bytes") ||
        !find(g_bcq.lora, "bcq_lora") || !find(g_bcq.lora_workspace_bytes, "bcq_lora_workspace_bytes"))
        return nullptr;
    Py_INCREF(error);
    Py_XSETREF(g_error, error);
    Py_RETURN_NONE;
}

template <int COUNT, at::Tensor (*CALL)(PyObject *const *)>
PyCFunction fast()
{
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&guarded<COUNT, CALL>));
}

PyMethodDef g_methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                           {"rotate", fast<13, rotate>(), METH_FASTCALL, nullptr},
                           {"attend", fast<13, attend>(), METH_FASTCALL, nullptr},
                           {"add", fast<10, add>(), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_serving", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving() { return PyModule_Create(&g_module); }
