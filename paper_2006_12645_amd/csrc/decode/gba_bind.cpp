// gba_bind.cpp -- the per-call half of paper_2006_12645_amd/decode.py: checks
// the tensors of one call, makes its outputs and enters the C ABI.
//
// The calls of a decoding step are bound by the host: a launch takes 3.4 us
// here, and the checks and allocations of one call in Python 3 to 7 more.
// Arguments come as decode.py passes them (no keywords).  Handles are the
// addresses of their C structs, which the Python handle keeps alive together
// with the tensors that they point to.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <string>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "gba.h"

namespace {

PyObject *gba_error = nullptr;  // gba.GbaError

template <class... A>
[[noreturn]] void refuse(PyObject *kind, const char *format, A... a)
{
    PyErr_Format(kind, format, a...);
    throw python_error();
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, "%s must be a tensor", name);
    return THPVariable_Unpack(o);
}

int64_t number(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}

template <class T>
T *handle(PyObject *o)
{
    return static_cast<T *>(PyLong_AsVoidPtr(o));
}

gba_stream_t stream_of(PyObject *o) { return static_cast<gba_stream_t>(PyLong_AsVoidPtr(o)); }

at::ScalarType type_of(gba_dtype d) { return d == GBA_F16 ? at::kHalf : at::kBFloat16; }

void on_gpu(const at::Tensor &t, const char *name, at::ScalarType type, int64_t device)
{
    if (t.scalar_type() != type || !t.is_cuda())
        refuse(PyExc_TypeError, "%s must be a CUDA tensor of %s", name, type == at::kHalf ? "float16" : type == at::kBFloat16 ? "bfloat16" : type == at::kInt ? "int32" : "int64");
    if (t.get_device() != device) refuse(PyExc_ValueError, "%s is on another device than what it is used with", name);
}

// A contiguous tensor of this type and shape (columns < 0: one dimension).
void whole(const at::Tensor &t, const char *name, at::ScalarType type, int64_t device, int64_t rows, int64_t columns = -1)
{
    on_gpu(t, name, type, device);
    const bool fits = columns < 0 ? t.dim() == 1 && t.size(0) == rows : t.dim() == 2 && t.size(0) == rows && t.size(1) == columns;
    if (!fits || !t.is_contiguous())
        refuse(PyExc_ValueError, "%s must be a contiguous tensor of %lld%s elements", name, (long long)rows,
                                columns < 0 ? "" : (" x " + std::to_string(columns)).c_str());
}

void check(gba_status s, const char *what)
{
    if (s == GBA_OK) return;
    PyObject *e = PyObject_CallFunction(gba_error, "is", (int)s, what);
    if (e != nullptr) {
        PyErr_SetObject(reinterpret_cast<PyObject *>(Py_TYPE(e)), e);
        Py_DECREF(e);
    }
    throw python_error();
}

void count_is(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) refuse(PyExc_TypeError, "%lld arguments, not %lld", (long long)want, (long long)n);
}

// The row stride of a row-major matrix.
int64_t row_stride(const at::Tensor &t, const char *name)
{
    const int64_t rows = t.size(0), columns = t.size(1), ld = rows > 1 ? t.stride(0) : columns > 0 ? columns : 1;
    if ((columns > 1 && t.stride(1) != 1) || ld < columns) refuse(PyExc_ValueError, "%s must be a row-major matrix", name);
    return ld;
}

// (weight, device, x, bias, out, act, stream)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_is(n, 7);
    const gba_q4_weight *w = handle<gba_q4_weight>(a[0]);
    const int64_t device = number(a[1]);
    const at::ScalarType type = type_of(w->dtype);
    const at::Tensor &x = tensor(a[2], "x");
    on_gpu(x, "x", type, device);
    if (x.dim() != 2 || x.size(1) != w->K) refuse(PyExc_ValueError, "x must be (M, %lld), as the weight has that many rows", (long long)w->K);
    const int64_t lda = row_stride(x, "x"), M = x.size(0);
    const void *bias = nullptr;
    if (a[3] != Py_None) {
        const at::Tensor &b = tensor(a[3], "bias");
        on_gpu(b, "bias", type, device);
        if (b.dim() != 1 || b.size(0) != w->N || (w->N > 1 && b.stride(0) != 1)) refuse(PyExc_ValueError, "bias must be a contiguous (N,) vector");
        bias = b.const_data_ptr();
    }
    at::Tensor out;
    if (a[4] == Py_None) {
        out = at::empty({M, w->N}, x.options());
    } else {
        out = tensor(a[4], "out");
        on_gpu(out, "out", type, device);
        if (out.dim() != 2 || out.size(0) != M || out.size(1) != w->N) refuse(PyExc_ValueError, "out must be an (M, N) matrix");
    }
    check(gba_q4_linear(w, M, x.const_data_ptr(), lda, bias, (gba_act)number(a[5]), out.mutable_data_ptr(), row_stride(out, "out"),
                        stream_of(a[6])),
          "gba_q4_linear");
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// (tables, device, lens, new, parents, tokens, tree, out, stream): the five
// maps, the last one None where there is no tree
PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_is(n, 9);
    const gba_block_tables *b = handle<gba_block_tables>(a[0]);
    const int64_t device = number(a[1]), tokens = number(a[5]), R = b->requests;
    const bool tree = a[6] == Py_True;
    const at::Tensor &lens = tensor(a[2], "lens"), &fresh = tensor(a[3], "new");
    whole(lens, "lens", at::kInt, device, R);
    whole(fresh, "new", at::kInt, device, R);
    if (tree == (a[4] == Py_None)) refuse(PyExc_ValueError, tree ? "a tree's steps need parents" : "parents come with tree=True");
    const int32_t *parents = nullptr;
    if (tree) {
        const at::Tensor &t = tensor(a[4], "parents");
        whole(t, "parents", at::kInt, device, tokens);
        parents = t.const_data_ptr<int32_t>();
    }
    static const char *const names[5] = {"out.offsets", "out.slots", "out.positions", "out.status", "out.mask"};
    const int64_t sizes[5] = {R + 1, tokens, tokens, R, tokens};
    at::Tensor out[5];
    const int count = tree ? 5 : 4;
    if (a[7] == Py_None) {
        for (int i = 0; i < count; ++i)
            out[i] = i < 4 ? at::empty({sizes[i]}, lens.options()) : at::empty({tokens, 1}, lens.options().dtype(at::kLong));
    } else {
        if (!PyTuple_Check(a[7]) || PyTuple_GET_SIZE(a[7]) != 5) refuse(PyExc_TypeError, "out must be a StepMaps");
        for (int i = 0; i < count; ++i) {
            out[i] = tensor(PyTuple_GET_ITEM(a[7], i), names[i]);
            if (i < 4) whole(out[i], names[i], at::kInt, device, sizes[i]);
            else whole(out[i], names[i], at::kLong, device, tokens, 1);
        }
    }
    check(gba_tables_step(b, lens.const_data_ptr<int32_t>(), fresh.const_data_ptr<int32_t>(), parents, tokens,
                          out[0].mutable_data_ptr<int32_t>(), out[1].mutable_data_ptr<int32_t>(), out[2].mutable_data_ptr<int32_t>(),
                          out[3].mutable_data_ptr<int32_t>(),
                          tree ? reinterpret_cast<uint64_t *>(out[4].mutable_data_ptr<int64_t>()) : nullptr, stream_of(a[8])),
          "gba_tables_step");
    PyObject *maps = PyTuple_New(5);
    if (maps == nullptr) throw python_error();
    for (int i = 0; i < 5; ++i) {
        PyObject *o = Py_None;
        if (i < count) o = THPVariable_Wrap(std::move(out[i]));
        else Py_INCREF(o);
        PyTuple_SET_ITEM(maps, i, o);
    }
    return maps;
    END_HANDLE_TH_ERRORS
}

// (cache, device, k, v, slots, stream)
PyObject *store(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_is(n, 6);
    const gba_paged_cache *c = handle<gba_paged_cache>(a[0]);
    const int64_t device = number(a[1]);
    const at::Tensor &slots = tensor(a[4], "slots");
    on_gpu(slots, "slots", at::kInt, device);
    if (slots.dim() != 1 || !slots.is_contiguous()) refuse(PyExc_ValueError, "slots must be a contiguous vector");
    const int64_t tokens = slots.size(0);
    const at::Tensor *kv[2] = {&tensor(a[2], "k"), &tensor(a[3], "v")};
    for (int i = 0; i < 2; ++i) {
        const at::Tensor &t = *kv[i];
        on_gpu(t, i ? "v" : "k", type_of(c->dtype), device);
        if (t.dim() != 3 || t.size(0) != tokens || t.size(1) != c->heads || t.size(2) != c->dim)
            refuse(PyExc_ValueError, "%s must be (%lld, %lld, %lld)", i ? "v" : "k", (long long)tokens, (long long)c->heads, (long long)c->dim);
        if (c->dim > 1 && t.stride(2) != 1) refuse(PyExc_ValueError, "dim must be contiguous in %s", i ? "v" : "k");
    }
    check(gba_cache_store(c, tokens, kv[0]->const_data_ptr(), kv[0]->stride(0), kv[0]->stride(1), kv[1]->const_data_ptr(), kv[1]->stride(0),
                          kv[1]->stride(1), slots.const_data_ptr<int32_t>(), stream_of(a[5])),
          "gba_cache_store");
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// What a call of attention is given, into a gba_attention or gba_q4_attention
// whose cache is set: false where the workspace is too small, and `need` says
// what it needs.  The arguments are those of attend().
template <class D, class Need>
bool describe(D &d, PyObject *const *a, at::Tensor &out, const char *what, Need workspace_size, size_t &need)
{
    const int64_t device = number(a[1]);
    const at::ScalarType type = type_of(d.cache.dtype);
    const at::Tensor &q = tensor(a[2], "q"), &table = tensor(a[3], "table"), &lens = tensor(a[4], "lens"), &offsets = tensor(a[5], "offsets");
    on_gpu(q, "q", type, device);
    if (q.dim() != 3 || q.size(2) != d.cache.dim || d.cache.heads == 0 || q.size(1) % d.cache.heads != 0)
        refuse(PyExc_ValueError, "q must be (tokens, a multiple of %lld, %lld)", (long long)d.cache.heads, (long long)d.cache.dim);
    if (table.dim() != 2) refuse(PyExc_ValueError, "table must be (requests, width)");
    d.requests = table.size(0);
    d.width = table.size(1);
    d.tokens = q.size(0);
    d.q_heads = q.size(1);
    d.max_new = number(a[6]);
    whole(table, "table", at::kInt, device, d.requests, d.width);
    whole(lens, "lens", at::kInt, device, d.requests);
    whole(offsets, "offsets", at::kInt, device, d.requests + 1);
    d.mask = nullptr;
    if (a[7] != Py_None) {
        const at::Tensor &m = tensor(a[7], "mask");
        on_gpu(m, "mask", at::kLong, device);
        if (m.numel() != d.tokens || !m.is_contiguous()) refuse(PyExc_ValueError, "mask must be one contiguous word for each token");
        d.mask = reinterpret_cast<const uint64_t *>(m.const_data_ptr<int64_t>());
    }
    const double scale = PyFloat_AsDouble(a[8]);
    if (scale == -1.0 && PyErr_Occurred()) throw python_error();
    d.scale = (float)scale;
    d.workspace = nullptr;
    d.workspace_bytes = 0;
    if (a[9] != Py_None) {
        out = tensor(a[9], "out");
        on_gpu(out, "out", type, device);
        if (!out.sizes().equals(q.sizes())) refuse(PyExc_ValueError, "out must have the shape of q");
    }
    if (d.cache.dim > 1 && (q.stride(2) != 1 || (out.defined() && out.stride(2) != 1))) refuse(PyExc_ValueError, "dim must be contiguous in q and out");
    d.q = q.const_data_ptr();
    d.q_token = q.stride(0);
    d.q_head = q.stride(1);
    d.table = table.const_data_ptr<int32_t>();
    d.lens = lens.const_data_ptr<int32_t>();
    d.offsets = offsets.const_data_ptr<int32_t>();
    if (!out.defined()) out = at::empty(q.sizes(), q.options());
    d.out = out.mutable_data_ptr();
    d.out_token = out.stride(0);
    d.out_head = out.stride(1);
    if (a[10] != Py_None) {
        const at::Tensor &w = tensor(a[10], "workspace");
        if (w.scalar_type() != at::kByte || !w.is_cuda() || w.get_device() != device || !w.is_contiguous())
            refuse(PyExc_TypeError, "workspace must be a contiguous uint8 CUDA tensor");
        d.workspace = w.mutable_data_ptr();
        d.workspace_bytes = (size_t)w.numel();
    }
    if (a[11] != Py_True) return true;
    need = 0;
    check(workspace_size(need), what);
    return need <= d.workspace_bytes;
}

// (cache, device, q, table, lens, offsets, max_new, mask, scale, out,
// workspace, wants_workspace, stream, and where there is a window it and the
// sinks): the output, or the bytes of a workspace that is to be passed
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 13) count_is(n, 15);
    const bool bounded = n == 15;
    const int64_t window = bounded ? number(a[13]) : 0, sinks = bounded ? number(a[14]) : 0;
    const char *what = bounded ? "gba_window_attention" : "gba_tree_attention";
    gba_attention d;
    d.cache = *handle<gba_paged_cache>(a[0]);
    at::Tensor out;
    size_t need;
    const auto size = [&](size_t &bytes) {
        return bounded ? gba_window_attention_workspace_size(&d, window, sinks, &bytes) : gba_tree_attention_workspace_size(&d, &bytes);
    };
    if (!describe(d, a, out, what, size, need)) return PyLong_FromSize_t(need);
    check(bounded ? gba_window_attention(&d, window, sinks, stream_of(a[12])) : gba_tree_attention(&d, stream_of(a[12])), what);
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// The same over a cache in 4 bits.
PyObject *attend_q4(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 13) count_is(n, 15);
    gba_q4_attention d;
    d.cache = *handle<gba_q4_cache>(a[0]);
    d.window = d.sinks = 0;
    if (n == 15) {
        d.window = number(a[13]);
        d.sinks = number(a[14]);
        if (d.window < 1) check(GBA_EINVAL, "gba_q4_attend");  // (0 is none in C)
    }
    at::Tensor out;
    size_t need;
    if (!describe(d, a, out, "gba_q4_attend", [&](size_t &bytes) { return gba_q4_attend_workspace_size(&d, &bytes); }, need))
        return PyLong_FromSize_t(need);
    check(gba_q4_attend(&d, stream_of(a[12])), "gba_q4_attend");
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// A (tokens, heads, dim) tensor of a cache's rows.
template <class C>
void token_rows(const at::Tensor &t, const char *name, const C *c, int64_t device, int64_t tokens)
{
    on_gpu(t, name, type_of(c->dtype), device);
    if (t.dim() != 3 || t.size(0) != tokens || t.size(1) != c->heads || t.size(2) != c->dim)
        refuse(PyExc_ValueError, "%s must be (%lld, %lld, %lld)", name, (long long)tokens, (long long)c->heads, (long long)c->dim);
    if (c->dim > 1 && t.stride(2) != 1) refuse(PyExc_ValueError, "dim must be contiguous in %s", name);
}

int64_t slot_count(const at::Tensor &slots, int64_t device)
{
    on_gpu(slots, "slots", at::kInt, device);
    if (slots.dim() != 1 || !slots.is_contiguous()) refuse(PyExc_ValueError, "slots must be a contiguous vector");
    return slots.size(0);
}

// (cache, device, k, v, slots, stream), of a cache in 4 bits
PyObject *store_q4(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_is(n, 6);
    const gba_q4_cache *c = handle<gba_q4_cache>(a[0]);
    const int64_t device = number(a[1]);
    const at::Tensor &k = tensor(a[2], "k"), &v = tensor(a[3], "v"), &slots = tensor(a[4], "slots");
    const int64_t tokens = slot_count(slots, device);
    token_rows(k, "k", c, device, tokens);
    token_rows(v, "v", c, device, tokens);
    check(gba_q4_cache_store(c, tokens, k.const_data_ptr(), k.stride(0), k.stride(1), v.const_data_ptr(), v.stride(0), v.stride(1),
                             slots.const_data_ptr<int32_t>(), stream_of(a[5])),
          "gba_q4_cache_store");
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}

// (cache, device, slots, k or None, v or None, stream): k and v
PyObject *load_q4(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count_is(n, 6);
    const gba_q4_cache *c = handle<gba_q4_cache>(a[0]);
    const int64_t device = number(a[1]);
    const at::Tensor &slots = tensor(a[2], "slots");
    const int64_t tokens = slot_count(slots, device);
    at::Tensor out[2];
    for (int i = 0; i < 2; ++i) {
        if (a[3 + i] == Py_None) {
            out[i] = at::empty({tokens, c->heads, c->dim}, slots.options().dtype(type_of(c->dtype)));
        } else {
            out[i] = tensor(a[3 + i], i ? "v" : "k");
            token_rows(out[i], i ? "v" : "k", c, device, tokens);
        }
    }
    check(gba_q4_cache_load(c, tokens, slots.const_data_ptr<int32_t>(), out[0].mutable_data_ptr(), out[0].stride(0), out[0].stride(1),
                            out[1].mutable_data_ptr(), out[1].stride(0), out[1].stride(1), stream_of(a[5])),
          "gba_q4_cache_load");
    PyObject *both = PyTuple_New(2);
    if (both == nullptr) throw python_error();
    for (int i = 0; i < 2; ++i) PyTuple_SET_ITEM(both, i, THPVariable_Wrap(std::move(out[i])));
    return both;
    END_HANDLE_TH_ERRORS
}

PyObject *set_error(PyObject *, PyObject *e)
{
    Py_INCREF(e);
    Py_XSETREF(gba_error, e);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"linear", reinterpret_cast<PyCFunction>(linear), METH_FASTCALL, nullptr},
                         {"step", reinterpret_cast<PyCFunction>(step), METH_FASTCALL, nullptr},
                         {"store", reinterpret_cast<PyCFunction>(store), METH_FASTCALL, nullptr},
                         {"attend", reinterpret_cast<PyCFunction>(attend), METH_FASTCALL, nullptr},
                         {"store_q4", reinterpret_cast<PyCFunction>(store_q4), METH_FASTCALL, nullptr},
                         {"load_q4", reinterpret_cast<PyCFunction>(load_q4), METH_FASTCALL, nullptr},
                         {"attend_q4", reinterpret_cast<PyCFunction>(attend_q4), METH_FASTCALL, nullptr},
                         {"set_error", set_error, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_gba_decode", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__gba_decode(void) { return PyModule_Create(&module); }
