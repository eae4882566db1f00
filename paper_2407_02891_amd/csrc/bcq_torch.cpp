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
    decltype(&bcq_attend_shared) attend_shared;
    decltype(&bcq_attend_shared_workspace_bytes) attend_shared_workspace_bytes;
    decltype(&bcq_plan) plan;
    decltype(&bcq_sample) sample;
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
    template <class T>
    T *vector(PyObject *o, const char *name, int64_t n, at::ScalarType of) const  // null for None
    {
        if (o == Py_None) return nullptr;
        const at::Tensor &t = tensor(o, where, name);
        if (t.scalar_type() != of || t.dim() != 1 || t.size(0) != n || t.device() != device || !t.is_contiguous())
            refuse(where, std::string(name) + ": contiguous " + c10::toString(of) + " [" + std::to_string(n) + "] on " + device.str());
        return static_cast<T *>(t.data_ptr());
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
PyObject *wrapped(const at::Tensor &t) { return THPVariable_Wrap(t); }
PyObject *wrapped(PyObject *o) { return o; }

template <int COUNT, auto CALL>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != COUNT) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected", COUNT);
        return nullptr;
    }
    try {
        return wrapped(CALL(args));
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

at::ScalarType of(int32_t dtype) { return dtype == BCQ_BF16 ? at::kBFloat16 : at::kHalf; }

// k and v lie as the descriptor says that they do (a program may have put others in their place).
void check_cache(const bcq_cache &c, const at::Tensor &k, const at::Tensor &v, const char *where)
{
    const int64_t sizes[4] = {c.num_pages, c.kv_heads, c.page_size, c.head_dim}, strides[4] = {c.page_stride, c.head_stride, c.slot_stride, 1};
    bool same = k.device() == v.device();
    for (const at::Tensor *t : {&k, &v}) {
        same = same && t->dim() == 4 && t->scalar_type() == of(c.dtype);
        for (int i = 0; same && i < 4; ++i) same = t->size(i) == sizes[i] && (t->stride(i) == strides[i] || sizes[i] <= 1);
    }
    if (!same) refuse(where, "k, v: shape, strides and type that the cache was made with");
}

// rotate(desc, k, v, qkv, positions, cos_sin, slots, q_weight, k_weight, eps, interleaved, out, stream)
at::Tensor rotate(PyObject *const *a)
{
    const char *const where = "PagedCache.rotate";
    const bcq_cache *const c = address<const bcq_cache>(a[0]);
    const at::Tensor &k = tensor(a[1], where, "k"), &v = tensor(a[2], where, "v"), &qkv = tensor(a[3], where, "qkv");
    const Place place{k.scalar_type(), k.device(), where};
    const c10::DeviceGuard there(place.device);  // (launches go to the current device)
    check_cache(*c, k, v, where);
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

// What both attentions are given: desc, k, v, q, q_start, kv_len, pages, max_new first.
struct Attended {
    const bcq_cache *cache;
    Place place;
    const at::Tensor &k, &v, &q, &pages;
    int64_t T, R, max_pages, q_heads, ld;
    const int32_t *q_start, *kv_len;
    int32_t max_new;

    Attended(PyObject *const *a, const char *where)
        : cache(address<const bcq_cache>(a[0])), place{tensor(a[1], where, "k").scalar_type(), tensor(a[1], where, "k").device(), where}, k(tensor(a[1], where, "k")),
          v(tensor(a[2], where, "v")), q(tensor(a[3], where, "q")), pages(tensor(a[6], where, "pages"))
    {
        check_cache(*cache, k, v, where);
        const int64_t D = head_dim(*cache, where);
        if (q.dim() != 2 || q.size(1) % D) refuse(where, "q: [tokens][q_heads * head_dim]");
        if (pages.dim() != 2 || pages.scalar_type() != at::kInt || pages.device() != place.device || !pages.is_contiguous())
            refuse(where, "pages: contiguous int32 [requests][max_pages]");
        T = q.size(0), R = pages.size(0), max_pages = pages.size(1), q_heads = q.size(1) / D;
        if (T > INT32_MAX || R > INT32_MAX - 1 || max_pages > INT32_MAX || q_heads > INT32_MAX) refuse(where, "q or pages: too large");
        ld = place.rows(q, "q", T, q.size(1));
        q_start = place.ints(a[4], "q_start", R + 1), kv_len = place.ints(a[5], "kv_len", R);
        max_new = int32(a[7], where, "max_new");
    }
    at::Tensor result(PyObject *out) const { return out == Py_None ? place.fresh(T, q.size(1)) : tensor(out, place.where, "out"); }
};

// attend(desc, k, v, q, q_start, kv_len, pages, max_new, scale, causal, window, out, stream)
at::Tensor attend(PyObject *const *a)
{
    const char *const where = "PagedCache.attend";
    const Attended x(a, where);
    const c10::DeviceGuard there(x.place.device);  // (launches go to the current device)
    const int32_t window = int32(a[10], where, "window");
    const at::Tensor out = x.result(a[11]);
    const int64_t ld_out = x.place.rows(out, "out", x.T, x.q.size(1));
    const size_t bytes = g_bcq.attend_workspace_bytes(x.cache, (int32_t)x.T, (int32_t)x.R, (int32_t)x.q_heads, (int32_t)x.max_pages, x.max_new);
    const at::Tensor workspace = bytes ? x.place.scratch(bytes) : at::Tensor();
    succeeded(g_bcq.attend(x.cache, x.k.data_ptr(), x.v.data_ptr(), (int32_t)x.T, (int32_t)x.R, (int32_t)x.q_heads, x.q.data_ptr(), x.ld, x.q_start, x.kv_len,
                           static_cast<const int32_t *>(x.pages.data_ptr()), (int32_t)x.max_pages, x.max_new, (float)number(a[8]), truth(a[9]), window,
                           out.data_ptr(), ld_out, bytes ? workspace.data_ptr() : nullptr, address<void>(a[12])),
              where);
    return out;
}

// attend_shared(desc, k, v, q, q_start, kv_len, pages, max_new, group_start, shared_len, max_shared, scale, causal, window, out, stream)
at::Tensor attend_shared(PyObject *const *a)
{
    const char *const where = "PagedCache.attend_shared";
    const Attended x(a, where);
    const c10::DeviceGuard there(x.place.device);
    const at::Tensor &lengths = tensor(a[9], where, "shared_len");
    if (lengths.dim() != 1 || lengths.size(0) > INT32_MAX - 1) refuse(where, "shared_len: int32 [groups]");
    const int64_t groups = lengths.size(0);
    const int32_t *const shared_len = x.place.ints(a[9], "shared_len", groups), *const group_start = x.place.ints(a[8], "group_start", groups + 1);
    const int32_t max_shared = int32(a[10], where, "max_shared"), window = int32(a[13], where, "window");
    const at::Tensor out = x.result(a[14]);
    const int64_t ld_out = x.place.rows(out, "out", x.T, x.q.size(1));
    const size_t bytes =
        g_bcq.attend_shared_workspace_bytes(x.cache, (int32_t)x.T, (int32_t)x.R, (int32_t)groups, (int32_t)x.q_heads, (int32_t)x.max_pages, x.max_new);
    const at::Tensor workspace = bytes ? x.place.scratch(bytes) : at::Tensor();
    succeeded(g_bcq.attend_shared(x.cache, x.k.data_ptr(), x.v.data_ptr(), (int32_t)x.T, (int32_t)x.R, (int32_t)groups, (int32_t)x.q_heads, x.q.data_ptr(), x.ld,
                                  x.q_start, x.kv_len, static_cast<const int32_t *>(x.pages.data_ptr()), (int32_t)x.max_pages, x.max_new, group_start, shared_len,
                                  max_shared, (float)number(a[11]), truth(a[12]), window, out.data_ptr(), ld_out, bytes ? workspace.data_ptr() : nullptr,
                                  address<void>(a[15])),
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
    if (A.dim() != 3 || A.size(0) != d->count || A.size(1) != d->max_rank || A.size(2) != d->N || B.dim() != 3 || B.size(0) != d->count || B.size(1) != d->M ||
        B.size(2) != d->max_rank || A.scalar_type() != of(d->dtype) || B.scalar_type() != A.scalar_type() || !A.is_contiguous() || !B.is_contiguous() ||
        B.device() != A.device())
        refuse(where, "A, B: shape and type that the adapters were made with, contiguous");
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

// Elements [from, from + n) of a contiguous tensor, as narrow gives them but without the dispatcher (six of them took 3 us of a step's 9).
at::Tensor stretch(const at::Tensor &all, int64_t from, int64_t n)
{
    auto part = c10::make_intrusive<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), all.dtype());
    part->set_sizes_contiguous({n});
    part->set_storage_offset(from);
    return at::Tensor(std::move(part));
}

// step(desc, pages, held, fixed, free_pages, free_count, cached, fresh, tokens, trial, out, names, stream): a dict of the tensors that `names` names, in the order
// of the entry point's arguments; those of `out`, or new ones.
PyObject *step(PyObject *const *a)
{
    const char *const where = "PageTable.step";
    const bcq_page_table *const d = address<const bcq_page_table>(a[0]);
    const at::Tensor &pages = tensor(a[1], where, "pages");
    const Place place{at::kInt, pages.device(), where};
    const c10::DeviceGuard there(place.device);
    const int64_t R = d->requests, T = int32(a[8], where, "tokens");
    if (pages.dim() != 2 || pages.size(0) != R || pages.size(1) != d->max_pages || pages.scalar_type() != at::kInt || !pages.is_contiguous())
        refuse(where, "pages: contiguous int32 [" + std::to_string(R) + "][" + std::to_string(d->max_pages) + "], as the table was made with");
    if (T < 0) refuse(where, "tokens: negative");
    int32_t *const held = place.vector<int32_t>(a[2], "held", R, at::kInt), *const fixed = place.vector<int32_t>(a[3], "fixed", R, at::kInt);
    int32_t *const free_pages = place.vector<int32_t>(a[4], "free", d->num_pages, at::kInt), *const free_count = place.vector<int32_t>(a[5], "free_count", 1, at::kInt);
    const int32_t *const cached = place.ints(a[6], "cached", R), *const fresh = place.ints(a[7], "fresh", R);
    const bool trial = truth(a[9]);
    // q_start, kv_len, lack, held, free_count, positions, slots, owner
    constexpr int kOut = 8;
    const int64_t sizes[kOut] = {R + 1, R, R, R, 1, T, T, T};
    PyObject *const names = a[11];
    if (!PyTuple_Check(names) || PyTuple_GET_SIZE(names) != kOut) refuse(where, "names: of eight tensors");
    int32_t *to[kOut];
    PyObject *out = a[10];
    const auto mine = [&](int i) { return !trial && (i == 3 || i == 4); };  // the table's own counts
    if (out != Py_None) {
        if (!PyDict_Check(out)) refuse(where, "out: a dict as an earlier step returned it");
        for (int i = 0; i < kOut; ++i) {
            PyObject *const t = PyDict_GetItem(out, PyTuple_GET_ITEM(names, i));
            const char *const name = PyUnicode_AsUTF8(PyTuple_GET_ITEM(names, i));
            if (!t || t == Py_None) refuse(where, std::string("out: without ") + (name ? name : "a tensor"));
            to[i] = place.vector<int32_t>(t, name ? name : "out", sizes[i], at::kInt);
        }
        if (mine(3) ? to[3] != held || to[4] != free_count : to[3] == held || to[4] == free_count)
            refuse(where, mine(3) ? "out: held and free_count of a trial" : "out: the table's own held and free_count, which a trial leaves");
        Py_INCREF(out);
    } else {
        int64_t total = 0;
        for (int i = 0; i < kOut; ++i) total += mine(i) ? 0 : (sizes[i] + 3) & ~int64_t(3);  // (each at 16 bytes)
        const at::Tensor all = at::empty({total}, at::TensorOptions().dtype(at::kInt).device(place.device));
        out = PyDict_New();
        if (!out) throw Refused{-1, ""};
        int64_t from = 0;
        for (int i = 0; i < kOut; ++i) {
            PyObject *t;
            if (mine(i)) {
                t = a[i == 3 ? 2 : 5];
                Py_INCREF(t);
                to[i] = i == 3 ? held : free_count;
            } else {
                const at::Tensor part = stretch(all, from, sizes[i]);
                from += (sizes[i] + 3) & ~int64_t(3);
                to[i] = static_cast<int32_t *>(part.data_ptr());
                t = THPVariable_Wrap(part);
            }
            const bool put = t && PyDict_SetItem(out, PyTuple_GET_ITEM(names, i), t) == 0;
            Py_XDECREF(t);
            if (!put) {  // (Python's own error stands)
                Py_DECREF(out);
                throw Refused{-1, ""};
            }
        }
    }
    const bcq_status status = g_bcq.plan(d, static_cast<int32_t *>(pages.data_ptr()), held, fixed, free_pages, free_count, cached, fresh, (int32_t)T, to[0], to[1],
                                         to[2], to[3], to[4], to[5], to[6], to[7], address<void>(a[12]));
    if (status != BCQ_OK) {
        Py_DECREF(out);
        throw Refused{status, where};
    }
    return out;
}

// draw(temperature, top_k, top_p, min_p, logits, uniform, out, stream): (tokens, probabilities)
PyObject *draw(PyObject *const *a)
{
    const char *const where = "Sampler.draw";
    const at::Tensor &temperature = tensor(a[0], where, "temperature"), &logits = tensor(a[4], where, "logits");
    if (logits.scalar_type() != at::kHalf && logits.scalar_type() != at::kBFloat16) refuse(where, "logits: float16 or bfloat16");
    const Place place{logits.scalar_type(), temperature.device(), where};
    const c10::DeviceGuard there(place.device);
    const int64_t R = temperature.size(0);
    if (logits.dim() != 2 || logits.size(1) > INT32_MAX || logits.size(1) < 1) refuse(where, "logits: [rows][vocabulary]");
    const int64_t V = logits.size(1), ld = place.rows(logits, "logits", R, V);
    const float *const top_p = place.vector<float>(a[2], "top_p", R, at::kFloat), *const min_p = place.vector<float>(a[3], "min_p", R, at::kFloat);
    const int32_t *const top_k = place.vector<int32_t>(a[1], "top_k", R, at::kInt);
    const float *const uniform = place.vector<float>(tensor(a[5], where, "uniform").defined() ? a[5] : Py_None, "uniform", R, at::kFloat);
    at::Tensor token, probability;
    if (a[6] == Py_None) {
        token = at::empty({R}, at::TensorOptions().dtype(at::kInt).device(place.device));
        probability = at::empty({R}, at::TensorOptions().dtype(at::kFloat).device(place.device));
    } else {
        if (!PyTuple_Check(a[6]) || PyTuple_GET_SIZE(a[6]) != 2) refuse(where, "out: (tokens, probabilities)");
        place.ints(PyTuple_GET_ITEM(a[6], 0), "out[0]", R);
        token = tensor(PyTuple_GET_ITEM(a[6], 0), where, "out[0]"), probability = tensor(PyTuple_GET_ITEM(a[6], 1), where, "out[1]");
        place.vector<float>(PyTuple_GET_ITEM(a[6], 1), "out[1]", R, at::kFloat);
    }
    succeeded(g_bcq.sample(place.type == at::kBFloat16 ? BCQ_BF16 : BCQ_F16, (int32_t)R, (int32_t)V, logits.data_ptr(), ld,
                           place.vector<float>(a[0], "temperature", R, at::kFloat), top_k, top_p, min_p, uniform, static_cast<int32_t *>(token.data_ptr()),
                           static_cast<float *>(probability.data_ptr()), address<void>(a[7])),
              where);
    PyObject *const t = THPVariable_Wrap(token), *const p = THPVariable_Wrap(probability);
    PyObject *const both = t && p ? PyTuple_Pack(2, t, p) : nullptr;
    Py_XDECREF(t);
    Py_XDECREF(p);
    return both;
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
        !find(g_bcq.lora, "bcq_lora") || !find(g_bcq.lora_workspace_bytes, "bcq_lora_workspace_bytes") ||
        !find(g_bcq.attend_shared, "bcq_attend_shared") || !find(g_bcq.attend_shared_workspace_bytes, "bcq_attend_shared_workspace_bytes") ||
        !find(g_bcq.plan, "bcq_plan") || !find(g_bcq.sample, "bcq_sample"))
        return nullptr;
    Py_INCREF(error);
    Py_XSETREF(g_error, error);
    Py_RETURN_NONE;
}

template <int COUNT, auto CALL>
PyCFunction fast()
{
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(&guarded<COUNT, CALL>));
}

PyMethodDef g_methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                           {"rotate", fast<13, rotate>(), METH_FASTCALL, nullptr},
                           {"attend", fast<13, attend>(), METH_FASTCALL, nullptr},
                           {"attend_shared", fast<16, attend_shared>(), METH_FASTCALL, nullptr},
                           {"add", fast<10, add>(), METH_FASTCALL, nullptr},
                           {"step", fast<13, step>(), METH_FASTCALL, nullptr},
                           {"draw", fast<8, draw>(), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_serving", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__serving() { return PyModule_Create(&g_module); }
