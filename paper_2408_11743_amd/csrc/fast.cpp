// The common case of the cache operators' Python calls (kv.py, cache.py): tensors as they
// nearly always are are checked, the output is allocated and the C entry point
// called without a step in Python, since a decode step waits for the host
// between these small launches.  Whatever is not so, or a call that the library's
// own checks refuse, returns None with nothing done, and the Python side, which names
// faults and copies views, takes it from there.  A HIP error raises: part of the
// call may have reached the GPU, and it must not be made again.
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <ATen/TracerMode.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>

#include <cmath>
#include <cstring>

#include "marlin.h"

namespace {

decltype(&marlin_kv_append) g_append;
decltype(&marlin_paged_attention) g_attend;
decltype(&marlin_select_pages) g_select;
decltype(&marlin_kv_append8) g_append8;
decltype(&marlin_cache_attention) g_cache_attention;
decltype(&marlin_assign_pages) g_assign;
PyObject *g_raw_stream, *g_workspaces, *g_buf;  // current stream of a device; (device, stream) -> workspace; "buf"
PyObject *g_error;                              // MarlinError(function, status)

// A strided tensor of exactly PyTorch's type with memory of its own on a GPU, not lazily negated, without a gradient or
// tangent to carry on; else NULL.
const at::Tensor *plain(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && !t.is_neg() &&
                   !(t.requires_grad() && c10::GradMode::is_enabled()) && !t._fw_grad(0).defined()
               ? &t
               : nullptr;
}

// A dispatch mode, a trace or a transform is to see the call: it is the registered operator's.
bool watched()
{
    return c10::impl::TorchDispatchModeTLS::any_modes_set() || at::tracer::impl::is_dispatch_enabled() ||
           c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
}

struct Place {
    at::ScalarType dtype;
    int device;
    bool same(const at::Tensor *t) const { return t && t->scalar_type() == dtype && t->get_device() == device; }
    bool ints(const at::Tensor *t, int64_t dims) const
    {
        return t && t->scalar_type() == at::kInt && t->get_device() == device && t->dim() == dims &&
               (t->size(-1) <= 1 || t->stride(-1) == 1);
    }
};

bool dtype_of(at::ScalarType s, int64_t &d)
{
    d = s == at::kBFloat16 ? MARLIN_BF16 : MARLIN_F16;
    return s == at::kBFloat16 || s == at::kHalf;
}

bool aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// [rows, heads, head dim] that the kernels can read as it lies.
bool rows_ok(const at::Tensor &t, int64_t D)
{
    return t.dim() == 3 && t.size(2) == D && t.stride(2) == 1 && ((t.stride(0) | t.stride(1)) & 7) == 0 && aligned(t.const_data_ptr());
}

bool caches_ok(const at::Tensor &k, const at::Tensor &v)
{
    return k.dim() == 4 && k.sizes() == v.sizes() && k.is_contiguous() && v.is_contiguous();
}

at::Tensor dense(const at::Tensor &like, at::IntArrayRef sizes, at::ScalarType dtype)
{
    return at::Tensor(at::detail::empty_cuda(sizes, dtype, like.device(), std::nullopt));
}

bool out_ok(PyObject *o, const at::Tensor &q, const Place &at, at::Tensor &out)
{
    if (o == Py_None) {
        out = dense(q, q.sizes(), at.dtype);
        return true;
    }
    const at::Tensor *t = plain(o);
    if (!at.same(t) || t->sizes() != q.sizes() || !t->is_contiguous()) return false;
    out = *t;
    return true;
}

bool stream_of(int device, PyObject *&object, hipStream_t &stream)
{
    PyObject *d = PyLong_FromLong(device);
    object = d ? PyObject_CallOneArg(g_raw_stream, d) : nullptr;
    Py_XDECREF(d);
    if (!object) return false;
    stream = reinterpret_cast<hipStream_t>(PyLong_AsVoidPtr(object));
    return !PyErr_Occurred();
}

// The buffer of the caller's workspace, or of this device and stream (ops.py's), if there is one.
bool workspace_of(PyObject *given, int device, PyObject *stream, void *&data, uint64_t &bytes)
{
    PyObject *w = given;
    if (w == Py_None) {
        PyObject *key = Py_BuildValue("(iO)", device, stream);
        w = key ? PyDict_GetItemWithError(g_workspaces, key) : nullptr;
        Py_XDECREF(key);
        if (!w) return false;
    }
    PyObject *buf = PyObject_GetAttr(w, g_buf);
    const at::Tensor *t = buf ? plain(buf) : nullptr;
    const bool ok = t && t->get_device() == device && t->is_contiguous();
    if (ok) {
        data = t->data_ptr();
        bytes = t->nbytes();
    }
    Py_XDECREF(buf);
    return ok;
}

PyObject *not_here()
{
    if (PyErr_Occurred()) PyErr_Clear();  // the Python side will meet it again
    Py_RETURN_NONE;
}

PyObject *refused(const char *function, marlin_status_t status)
{
    if (status != MARLIN_ERR_HIP) return not_here();
    PyObject *e = PyObject_CallFunction(g_error, "si", function, (int)status);
    if (e) PyErr_SetObject(g_error, e);
    Py_XDECREF(e);
    return nullptr;
}

// q, k, v, k_cache, v_cache, table, lengths, cos_sin, starts, interleaved, bounds, out
PyObject *kv_append(PyObject *, PyObject *const *o, Py_ssize_t n)
try {
    if (n != 12 || !g_append || watched()) return not_here();
    const at::Tensor *q = plain(o[0]), *k = plain(o[1]), *v = plain(o[2]), *kc = plain(o[3]), *vc = plain(o[4]);
    const at::Tensor *table = plain(o[5]), *lengths = plain(o[6]);
    if (!kc) return not_here();
    const Place at{kc->scalar_type(), kc->get_device()};
    marlin_kv_append_args a;
    if (!dtype_of(at.dtype, a.dtype) || !at.same(vc) || !at.same(q) || !at.same(k) || !at.same(v) || !at.ints(table, 2) ||
        !at.ints(lengths, 1) || !caches_ok(*kc, *vc))
        return not_here();
    const int64_t D = kc->size(3);
    if (!rows_ok(*q, D) || !rows_ok(*k, D) || !rows_ok(*v, D) || k->sizes() != v->sizes() || k->size(0) != q->size(0) ||
        k->size(1) != kc->size(1) || lengths->size(0) != table->size(0))
        return not_here();
    a.cos_sin = nullptr;
    a.positions = a.rot = 0;
    if (o[7] != Py_None) {
        const at::Tensor *c = plain(o[7]);
        if (!c || c->scalar_type() != at::kFloat || c->get_device() != at.device || c->dim() != 2 || !c->is_contiguous())
            return not_here();
        a.positions = c->size(0);
        a.rot = c->size(1);
        a.cos_sin = a.rot ? c->const_data_ptr<float>() : nullptr;
    }
    a.starts = nullptr;
    if (o[8] != Py_None) {
        const at::Tensor *s = plain(o[8]);
        if (!at.ints(s, 1) || s->size(0) != table->size(0) + 1) return not_here();
        a.starts = s->const_data_ptr<int32_t>();
    } else if (q->size(0) != table->size(0)) {
        return not_here();
    }
    const int interleaved = PyObject_IsTrue(o[9]);
    if (interleaved < 0) return not_here();
    a.bounds = nullptr;
    if (o[10] != Py_None) {
        const at::Tensor *b = plain(o[10]);
        if (!at.same(b) || b->dim() != 4 || b->size(0) != kc->size(0) || b->size(1) != kc->size(1) || b->size(2) != 2 ||
            b->size(3) != D || !b->is_contiguous())
            return not_here();
        a.bounds = b->data_ptr();
    }
    at::Tensor out;
    if (!out_ok(o[11], *q, at, out)) return not_here();
    a.q = q->const_data_ptr();
    a.k = k->const_data_ptr();
    a.v = v->const_data_ptr();
    a.q_row = q->stride(0);
    a.q_head = q->stride(1);
    a.k_row = k->stride(0);
    a.k_head = k->stride(1);
    a.v_row = v->stride(0);
    a.v_head = v->stride(1);
    a.q_out = out.data_ptr();
    a.k_cache = kc->data_ptr();
    a.v_cache = vc->data_ptr();
    a.interleaved = interleaved;
    a.table = table->const_data_ptr<int32_t>();
    a.table_row = table->stride(0);
    a.lengths = lengths->const_data_ptr<int32_t>();
    a.tokens = q->size(0);
    a.B = table->size(0);
    a.heads = q->size(1);
    a.kv_heads = kc->size(1);
    a.head_dim = D;
    a.pages = kc->size(0);
    a.page_size = kc->size(2);
    a.width = table->size(1);
    PyObject *stream;
    hipStream_t s;
    if (!stream_of(at.device, stream, s)) return not_here();
    const c10::DeviceGuard guard(kc->device());
    const marlin_status_t status = g_append(&a, s);
    Py_DECREF(stream);
    if (status != MARLIN_OK) return refused("marlin_kv_append", status);
    if (o[11] != Py_None) {
        Py_INCREF(o[11]);
        return o[11];
    }
    return THPVariable_Wrap(std::move(out));
} catch (const std::exception &) {
    return not_here();
}

// q, k_cache, v_cache, table, lengths, scale, return_lse, out, workspace
PyObject *paged_attention(PyObject *, PyObject *const *o, Py_ssize_t n)
try {
    if (n != 9 || !g_attend || watched()) return not_here();
    const at::Tensor *q = plain(o[0]), *kc = plain(o[1]), *vc = plain(o[2]), *table = plain(o[3]), *lengths = plain(o[4]);
    if (!kc || !table) return not_here();
    const Place at{kc->scalar_type(), kc->get_device()};
    const bool per_head = table->dim() == 3;
    marlin_paged_attention_args a;
    if (!dtype_of(at.dtype, a.dtype) || !at.same(vc) || !at.same(q) || !at.ints(table, per_head ? 3 : 2) || !at.ints(lengths, 1) ||
        !caches_ok(*kc, *vc))
        return not_here();
    const int64_t D = kc->size(3);
    if (!rows_ok(*q, D) || q->size(0) != table->size(0) || lengths->size(0) != table->size(0) ||
        (per_head && table->size(1) != kc->size(1)))
        return not_here();
    a.scale = 1.0 / std::sqrt((double)D);
    if (o[5] != Py_None) {
        a.scale = PyFloat_AsDouble(o[5]);
        if (PyErr_Occurred()) return not_here();
    }
    const int with_lse = PyObject_IsTrue(o[6]);
    at::Tensor out, lse;
    if (with_lse < 0 || !out_ok(o[7], *q, at, out)) return not_here();
    if (with_lse) lse = dense(*q, {q->size(0), q->size(1)}, at::kFloat);
    a.q = q->const_data_ptr();
    a.q_row = q->stride(0);
    a.q_head = q->stride(1);
    a.k_cache = kc->const_data_ptr();
    a.v_cache = vc->const_data_ptr();
    a.table = table->const_data_ptr<int32_t>();
    a.table_row = table->stride(0);
    a.table_head = per_head ? table->stride(1) : 0;
    a.lengths = lengths->const_data_ptr<int32_t>();
    a.out = out.data_ptr();
    a.lse = with_lse ? lse.data_ptr<float>() : nullptr;
    a.B = q->size(0);
    a.heads = q->size(1);
    a.kv_heads = kc->size(1);
    a.head_dim = D;
    a.pages = kc->size(0);
    a.page_size = kc->size(2);
    a.width = table->size(-1);
    PyObject *stream;
    hipStream_t s;
    if (!stream_of(at.device, stream, s)) return not_here();
    const c10::DeviceGuard guard(kc->device());
    const bool ready = workspace_of(o[8], at.device, stream, a.workspace, a.workspace_bytes);
    Py_DECREF(stream);
    if (!ready) return not_here();
    const marlin_status_t status = g_attend(&a, s);
    if (status != MARLIN_OK) return refused("marlin_paged_attention", status);
    PyObject *first = o[7];
    if (first != Py_None)
        Py_INCREF(first);
    else
        first = THPVariable_Wrap(std::move(out));
    if (!with_lse || !first) return first;
    return Py_BuildValue("(NN)", first, THPVariable_Wrap(std::move(lse)));
} catch (const std::exception &) {
    return not_here();
}

// q, bounds, table, lengths, page_size, select, workspace
PyObject *select_pages(PyObject *, PyObject *const *o, Py_ssize_t n)
try {
    if (n != 7 || !g_select || watched()) return not_here();
    const at::Tensor *q = plain(o[0]), *bounds = plain(o[1]), *table = plain(o[2]), *lengths = plain(o[3]);
    if (!bounds) return not_here();
    const Place at{bounds->scalar_type(), bounds->get_device()};
    marlin_select_pages_args a;
    if (!dtype_of(at.dtype, a.dtype) || !at.same(q) || !at.ints(table, 2) || !at.ints(lengths, 1) || bounds->dim() != 4 ||
        bounds->size(2) != 2 || !bounds->is_contiguous() || !rows_ok(*q, bounds->size(3)) || q->size(0) != table->size(0) ||
        lengths->size(0) != table->size(0))
        return not_here();
    a.page_size = PyLong_AsLongLong(o[4]);
    a.select = PyLong_AsLongLong(o[5]);
    if (PyErr_Occurred() || a.select < 1 || a.select > (1 << 20)) return not_here();
    at::Tensor chosen = dense(*q, {q->size(0), bounds->size(1), a.select}, at::kInt);
    at::Tensor tokens = dense(*q, {q->size(0)}, at::kInt);
    a.q = q->const_data_ptr();
    a.q_row = q->stride(0);
    a.q_head = q->stride(1);
    a.bounds = bounds->const_data_ptr();
    a.table = table->const_data_ptr<int32_t>();
    a.table_row = table->stride(0);
    a.lengths = lengths->const_data_ptr<int32_t>();
    a.chosen = chosen.data_ptr<int32_t>();
    a.chosen_lengths = tokens.data_ptr<int32_t>();
    a.B = q->size(0);
    a.heads = q->size(1);
    a.kv_heads = bounds->size(1);
    a.head_dim = bounds->size(3);
    a.pages = bounds->size(0);
    a.width = table->size(1);
    PyObject *stream;
    hipStream_t s;
    if (!stream_of(at.device, stream, s)) return not_here();
    const c10::DeviceGuard guard(bounds->device());
    const bool ready = workspace_of(o[6], at.device, stream, a.workspace, a.workspace_bytes);
    Py_DECREF(stream);
    if (!ready) return not_here();
    const marlin_status_t status = g_select(&a, s);
    if (status != MARLIN_OK) return refused("marlin_select_pages", status);
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(chosen)), THPVariable_Wrap(std::move(tokens)));
} catch (const std::exception &) {
    return not_here();
}

// Scales [pages, kv heads, 2, page size / 16] of an 8-bit cache, dense.
bool scales_ok(const at::Tensor *s, const at::Tensor &k, int device)
{
    return s && s->scalar_type() == at::kFloat && s->get_device() == device && s->dim() == 4 && s->size(0) == k.size(0) &&
           s->size(1) == k.size(1) && s->size(2) == 2 && s->size(3) == k.size(2) / 16 && s->is_contiguous();
}

// q, k, v, k_cache, v_cache, scales, table, lengths, cos_sin, starts, interleaved, out
PyObject *kv_append8(PyObject *, PyObject *const *o, Py_ssize_t n)
try {
    if (n != 12 || !g_append8 || watched()) return not_here();
    const at::Tensor *q = plain(o[0]), *k = plain(o[1]), *v = plain(o[2]), *kc = plain(o[3]), *vc = plain(o[4]);
    const at::Tensor *scales = plain(o[5]), *table = plain(o[6]), *lengths = plain(o[7]);
    if (!kc || !q) return not_here();
    const Place at{q->scalar_type(), kc->get_device()}, codes{at::kFloat8_e4m3fn, at.device};
    marlin_kv_append8_args a;
    if (!dtype_of(at.dtype, a.dtype) || !codes.same(kc) || !codes.same(vc) || !at.same(q) || !at.same(k) || !at.same(v) ||
        !at.ints(table, 2) || !at.ints(lengths, 1) || !caches_ok(*kc, *vc) || !scales_ok(scales, *kc, at.device))
        return not_here();
    const int64_t D = kc->size(3);
    if (!rows_ok(*q, D) || !rows_ok(*k, D) || !rows_ok(*v, D) || k->sizes() != v->sizes() || k->size(0) != q->size(0) ||
        k->size(1) != kc->size(1) || lengths->size(0) != table->size(0))
        return not_here();
    a.cos_sin = nullptr;
    a.positions = a.rot = 0;
    if (o[8] != Py_None) {
        const at::Tensor *c = plain(o[8]);
        if (!c || c->scalar_type() != at::kFloat || c->get_device() != at.device || c->dim() != 2 || !c->is_contiguous())
            return not_here();
        a.positions = c->size(0);
        a.rot = c->size(1);
        a.cos_sin = a.rot ? c->const_data_ptr<float>() : nullptr;
    }
    a.starts = nullptr;
    if (o[9] != Py_None) {
        const at::Tensor *s = plain(o[9]);
        if (!at.ints(s, 1) || s->size(0) != table->size(0) + 1) return not_here();
        a.starts = s->const_data_ptr<int32_t>();
    } else if (q->size(0) != table->size(0)) {
        return not_here();
    }
    const int interleaved = PyObject_IsTrue(o[10]);
    if (interleaved < 0) return not_here();
    at::Tensor out;
    if (!out_ok(o[11], *q, at, out)) return not_here();
    a.q = q->const_data_ptr();
    a.k = k->const_data_ptr();
    a.v = v->const_data_ptr();
    a.q_row = q->stride(0);
    a.q_head = q->stride(1);
    a.k_row = k->stride(0);
    a.k_head = k->stride(1);
    a.v_row = v->stride(0);
    a.v_head = v->stride(1);
    a.q_out = out.data_ptr();
    a.k_cache = kc->data_ptr();
    a.v_cache = vc->data_ptr();
    a.scales = scales->data_ptr<float>();
    a.interleaved = interleaved;
    a.table = table->const_data_ptr<int32_t>();
    a.table_row = table->stride(0);
    a.lengths = lengths->const_data_ptr<int32_t>();
    a.tokens = q->size(0);
    a.B = table->size(0);
    a.heads = q->size(1);
    a.kv_heads = kc->size(1);
    a.head_dim = D;
    a.pages = kc->size(0);
    a.page_size = kc->size(2);
    a.width = table->size(1);
    PyObject *stream;
    hipStream_t s;
    if (!stream_of(at.device, stream, s)) return not_here();
    const c10::DeviceGuard guard(kc->device());
    const marlin_status_t status = g_append8(&a, s);
    Py_DECREF(stream);
    if (status != MARLIN_OK) return refused("marlin_kv_append8", status);
    if (o[11] != Py_None) {
        Py_INCREF(o[11]);
        return o[11];
    }
    return THPVariable_Wrap(std::move(out));
} catch (const std::exception &) {
    return not_here();
}

// None (0) or a number from 1 on, and a number from 0 on.
bool visible_of(PyObject *window, PyObject *sinks, int64_t &w, int64_t &s)
{
    w = window == Py_None ? 0 : PyLong_AsLongLong(window);
    s = PyLong_AsLongLong(sinks);
    return !PyErr_Occurred() && (window == Py_None || w >= 1) && s >= 0;
}

// q, k_cache, v_cache, table, lengths, scales, starts, window, sinks, scale, return_lse, out, workspace
PyObject *cache_attention(PyObject *, PyObject *const *o, Py_ssize_t n)
try {
    if (n != 13 || !g_cache_attention || watched()) return not_here();
    const at::Tensor *q = plain(o[0]), *kc = plain(o[1]), *vc = plain(o[2]), *table = plain(o[3]), *lengths = plain(o[4]);
    if (!q || !kc || !table) return not_here();
    const Place at{q->scalar_type(), kc->get_device()};
    const bool eight = o[5] != Py_None, several = o[6] != Py_None, per_head = !several && table->dim() == 3;
    const Place cache{eight ? at::kFloat8_e4m3fn : at.dtype, at.device};
    marlin_cache_attention_args a;
    if (!dtype_of(at.dtype, a.dtype) || !at.same(q) || !cache.same(kc) || !cache.same(vc) || !at.ints(table, per_head ? 3 : 2) ||
        !at.ints(lengths, 1) || !caches_ok(*kc, *vc))
        return not_here();
    const int64_t D = kc->size(3);
    if (!rows_ok(*q, D) || lengths->size(0) != table->size(0) || (!several && q->size(0) != table->size(0)) ||
        (per_head && table->size(1) != kc->size(1)))
        return not_here();
    a.scales = nullptr;
    if (eight) {
        const at::Tensor *s = plain(o[5]);
        if (!scales_ok(s, *kc, at.device)) return not_here();
        a.scales = s->const_data_ptr<float>();
    }
    a.starts = nullptr;
    if (several) {
        const at::Tensor *s = plain(o[6]);
        if (!at.ints(s, 1) || s->size(0) != table->size(0) + 1) return not_here();
        a.starts = s->const_data_ptr<int32_t>();
    }
    if (!visible_of(o[7], o[8], a.window, a.sinks)) return not_here();
    a.scale = 1.0 / std::sqrt((double)D);
    if (o[9] != Py_None) {
        a.scale = PyFloat_AsDouble(o[9]);
        if (PyErr_Occurred()) return not_here();
    }
    const int with_lse = PyObject_IsTrue(o[10]);
    at::Tensor out, lse;
    if (with_lse < 0 || !out_ok(o[11], *q, at, out)) return not_here();
    if (with_lse) lse = dense(*q, {q->size(0), q->size(1)}, at::kFloat);
    a.q = q->const_data_ptr();
    a.q_row = q->stride(0);
    a.q_head = q->stride(1);
    a.k_cache = kc->const_data_ptr();
    a.v_cache = vc->const_data_ptr();
    a.table = table->const_data_ptr<int32_t>();
    a.table_row = table->stride(0);
    a.table_head = per_head ? table->stride(1) : 0;
    a.lengths = lengths->const_data_ptr<int32_t>();
    a.tokens = q->size(0);
    a.out = out.data_ptr();
    a.lse = with_lse ? lse.data_ptr<float>() : nullptr;
    a.B = table->size(0);
    a.heads = q->size(1);
    a.kv_heads = kc->size(1);
    a.head_dim = D;
    a.pages = kc->size(0);
    a.page_size = kc->size(2);
    a.width = table->size(-1);
    PyObject *stream;
    hipStream_t s;
    if (!stream_of(at.device, stream, s)) return not_here();
    const c10::DeviceGuard guard(kc->device());
    const bool ready = workspace_of(o[12], at.device, stream, a.workspace, a.workspace_bytes);
    Py_DECREF(stream);
    if (!ready) return not_here();
    const marlin_status_t status = g_cache_attention(&a, s);
    if (status != MARLIN_OK) return refused("marlin_cache_attention", status);
    PyObject *first = o[11];
    if (first != Py_None)
        Py_INCREF(first);
    else
        first = THPVariable_Wrap(std::move(out));
    if (!with_lse || !first) return first;
    return Py_BuildValue("(NN)", first, THPVariable_Wrap(std::move(lse)));
} catch (const std::exception &) {
    return not_here();
}

// table, lengths, new, free, free_count, page_size, tokens, window, sinks, workspace, back
PyObject *assign_pages(PyObject *, PyObject *const *o, Py_ssize_t n)
try {
    if (n != 11 || !g_assign || watched()) return not_here();
    const at::Tensor *table = plain(o[0]), *lengths = plain(o[1]), *fresh = plain(o[2]), *free = plain(o[3]), *count = plain(o[4]);
    if (!table) return not_here();
    const Place at{at::kInt, table->get_device()};
    marlin_assign_pages_args a;
    if (!at.ints(table, 2) || !at.ints(lengths, 1) || !at.ints(fresh, 1) || !at.ints(free, 1) || !at.ints(count, 1) ||
        lengths->size(0) != table->size(0) || fresh->size(0) != table->size(0) || count->size(0) != 1 ||
        (table->size(0) > 1 && table->stride(0) < table->size(1)))
        return not_here();
    a.back = nullptr;
    if (o[10] != Py_None) {
        const at::Tensor *t = plain(o[10]);
        if (!at.ints(t, 1) || t->size(0) != table->size(0)) return not_here();
        a.back = t->const_data_ptr<int32_t>();
    }
    a.page_size = PyLong_AsLongLong(o[5]);
    a.tokens = PyLong_AsLongLong(o[6]);
    if (PyErr_Occurred() || a.tokens < 0 || a.tokens > (1 << 24) || !visible_of(o[7], o[8], a.window, a.sinks)) return not_here();
    at::Tensor starts = dense(*table, {table->size(0) + 1}, at::kInt), slots = dense(*table, {a.tokens}, at::kLong);
    a.table = table->data_ptr<int32_t>();
    a.table_row = table->stride(0);
    a.lengths = lengths->data_ptr<int32_t>();
    a.new_tokens = fresh->const_data_ptr<int32_t>();
    a.free_pages = free->data_ptr<int32_t>();
    a.free_count = count->data_ptr<int32_t>();
    a.starts = starts.data_ptr<int32_t>();
    a.slots = slots.data_ptr<int64_t>();
    a.B = table->size(0);
    a.width = table->size(1);
    a.pages = free->size(0);
    PyObject *stream;
    hipStream_t s;
    if (!stream_of(at.device, stream, s)) return not_here();
    const c10::DeviceGuard guard(table->device());
    const bool ready = workspace_of(o[9], at.device, stream, a.workspace, a.workspace_bytes);
    Py_DECREF(stream);
    if (!ready) return not_here();
    const marlin_status_t status = g_assign(&a, s);
    if (status != MARLIN_OK) return refused("marlin_assign_pages", status);
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(starts)), THPVariable_Wrap(std::move(slots)));
} catch (const std::exception &) {
    return not_here();
}

// addresses of marlin_kv_append8, marlin_cache_attention, marlin_assign_pages; connect comes first
PyObject *connect_cache(PyObject *, PyObject *args)
{
    unsigned long long append8, attention, assign;
    if (!PyArg_ParseTuple(args, "KKK", &append8, &attention, &assign)) return nullptr;
    g_append8 = reinterpret_cast<decltype(g_append8)>(append8);
    g_cache_attention = reinterpret_cast<decltype(g_cache_attention)>(attention);
    g_assign = reinterpret_cast<decltype(g_assign)>(assign);
    Py_RETURN_NONE;
}

// addresses of marlin_kv_append, marlin_paged_attention, marlin_select_pages; raw stream function; workspaces; MarlinError
PyObject *connect(PyObject *, PyObject *args)
{
    unsigned long long append, attend, select;
    PyObject *stream, *workspaces, *error;
    if (!PyArg_ParseTuple(args, "KKKOO!O", &append, &attend, &select, &stream, &PyDict_Type, &workspaces, &error)) return nullptr;
    g_append = reinterpret_cast<decltype(g_append)>(append);
    g_attend = reinterpret_cast<decltype(g_attend)>(attend);
    g_select = reinterpret_cast<decltype(g_select)>(select);
    Py_INCREF(stream);
    Py_XSETREF(g_raw_stream, stream);
    Py_INCREF(workspaces);
    Py_XSETREF(g_workspaces, workspaces);
    Py_INCREF(error);
    Py_XSETREF(g_error, error);
    if (!g_buf && !(g_buf = PyUnicode_InternFromString("buf"))) return nullptr;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"connect", connect, METH_VARARGS, nullptr},
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(kv_append)), METH_FASTCALL, nullptr},
    {"paged_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(paged_attention)), METH_FASTCALL, nullptr},
    {"select_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(select_pages)), METH_FASTCALL, nullptr},
    {"connect_cache", connect_cache, METH_VARARGS, nullptr},
    {"kv_append8", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(kv_append8)), METH_FASTCALL, nullptr},
    {"cache_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cache_attention)), METH_FASTCALL, nullptr},
    {"assign_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(assign_pages)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fast(void) { return PyModule_Create(&module); }
