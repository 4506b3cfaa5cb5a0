// The operators of include/rh_seq.h for Python: checks of the tensors, outputs, the call.  They are called once per layer and frame
// with a few rows each, where what lies ahead of the launch is most of the time: from C++ a call costs 4 to 6 us of the host's, as
// much as one of torch's own, through ctypes and torch's Python functions 7 to 11.  The library's functions come in by
// address (init), so that this module and the ctypes binding call the same one.  A call returns its outputs, or the status (an int) where the
// library refuses; what the library cannot see of a tensor is an AssertionError.
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "rh_seq.h"

static decltype(&rh_cache_plan) f_plan;
static decltype(&rh_cache_write) f_write;
static decltype(&rh_cache_attend) f_attend;
static decltype(&rh_norm_residual) f_norm;
static decltype(&rh_matvec_packed) f_matvec;

struct refused { const char* why; };
static void need(bool ok, const char* why) { if (!ok) throw refused{why}; }

#define BEGIN HANDLE_TH_ERRORS try {
#define END } catch (const refused& e) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_AssertionError, e.why); return nullptr; } END_HANDLE_TH_ERRORS

static const at::Tensor& on_gpu(PyObject* o, const char* why)
{
    need(THPVariable_CheckExact(o) || THPVariable_Check(o), why);
    const at::Tensor& t = THPVariable_Unpack(o);
    need(t.is_cuda(), why);
    return t;
}
static long integer(PyObject* o, const char* why)
{
    const long v = PyLong_AsLong(o);
    need(v != -1 || !PyErr_Occurred(), why);
    return v;
}
static int32_t word(PyObject* o, const char* why)           // what does not fit becomes what the library refuses
{
    const long v = integer(o, why);
    return v > INT32_MAX ? INT32_MAX : v < INT32_MIN ? INT32_MIN : (int32_t)v;
}
static bool truth(PyObject* o, const char* why)
{
    const int v = PyObject_IsTrue(o);
    need(v >= 0, why);                                       // what it raised stays
    return v != 0;
}
static int32_t fits(int64_t v, const char* why) { need(v >= 0 && v <= INT32_MAX, why); return (int32_t)v; }
// a call's context, and the tensors that it takes, which lie on its device
struct context {
    rh_ctx* handle;
    long device;
    explicit context(PyObject* o)                            // (handle, index of the device)
    {
        need(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 2, "a context's handle and device");
        handle = (rh_ctx*)integer(PyTuple_GET_ITEM(o, 0), "a context's handle");
        device = integer(PyTuple_GET_ITEM(o, 1), "a context's device");
    }
    const at::Tensor& tensor(PyObject* o, const char* why) const
    {
        const at::Tensor& t = on_gpu(o, why);
        need(t.get_device() == device, "a tensor of another device than the context's");
        return t;
    }
    const at::Tensor& dense(PyObject* o, at::ScalarType type, const char* why) const
    {
        const at::Tensor& t = tensor(o, why);
        need(t.scalar_type() == type && t.is_contiguous(), why);
        return t;
    }
    rh_kv_cache cache(PyObject* o) const;
};
static int32_t type_of(const at::Tensor& t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return RH_T_F32;
    case at::kBFloat16: return RH_T_BF16;
    case at::kFloat8_e4m3fn: return RH_T_E4M3;
    default: throw refused{"float32, bfloat16 or float8_e4m3fn"};
    }
}
static at::Tensor fresh(at::IntArrayRef shape, const at::Tensor& like, at::ScalarType type) { return at::empty(shape, like.options().dtype(type)); }
static at::Tensor part(const at::Tensor& t, int64_t first, int64_t n)
{
    at::AutoDispatchBelowADInplaceOrView plain;              // whole numbers: nothing of them is differentiated
    return t.narrow(0, first, n);
}
static PyObject* given(PyObject* o) { return o == Py_None ? nullptr : o; }
static PyObject* status(rh_status st) { return PyLong_FromLong(st); }
static PyObject* wrap(const at::Tensor& t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}
static PyObject* tuple_of(std::initializer_list<PyObject*> items)
{
    PyObject* r = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject* o : items) {
        if (!o || !r) { Py_XDECREF(o); Py_CLEAR(r); continue; }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}

// kv_desc(k, v, k_scale, v_scale) -> bytes of a placed_cache
struct placed_cache { rh_kv_cache cache; int64_t device; };
static PyObject* kv_desc(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    BEGIN
    need(n == 4, "k, v, k_scale, v_scale");
    const at::Tensor &k = on_gpu(a[0], "k on the GPU"), &v = on_gpu(a[1], "v on the GPU");
    need(k.get_device() == v.get_device(), "k and v on one device");
    need(k.scalar_type() == v.scalar_type() && k.dim() == 4 && v.sizes() == k.sizes(), "k and v alike, [n_pages, page, heads, dim]");
    need(k.stride(3) == 1 && v.stride(3) == 1, "the elements of a head lie side by side");
    placed_cache placed;
    memset(&placed, 0, sizeof placed);
    rh_kv_cache& c = placed.cache;
    placed.device = k.get_device();
    c.k = k.data_ptr(); c.v = v.data_ptr();
    c.type = type_of(k);
    c.n_pages = fits(k.size(0), "n_pages"); c.page = fits(k.size(1), "page"); c.heads = fits(k.size(2), "heads"); c.dim = fits(k.size(3), "dim");
    for (int i = 0; i < 3; ++i) { c.k_stride[i] = k.stride(i); c.v_stride[i] = v.stride(i); }
    for (int i = 0; i < 2; ++i) {
        if (!given(a[2 + i])) continue;
        const at::Tensor& s = on_gpu(a[2 + i], "scales on the GPU");
        need(s.get_device() == k.get_device() && s.scalar_type() == at::kFloat && s.is_contiguous(), "scales float32, dense, on the device of k and v");
        need(s.dim() == 3 && s.size(0) == c.n_pages && s.size(1) == c.heads && s.size(2) == c.page, "scales [n_pages, heads, page]");
        (i ? c.v_scale : c.k_scale) = (float*)s.data_ptr();
    }
    return PyBytes_FromStringAndSize((const char*)&placed, sizeof placed);
    END
}
rh_kv_cache context::cache(PyObject* o) const
{
    placed_cache c;
    need(PyBytes_Check(o) && PyBytes_GET_SIZE(o) == sizeof c, "a cache's descriptor");
    memcpy(&c, PyBytes_AS_STRING(o), sizeof c);
    need(c.device == device, "a cache on another device than the context's");
    return c.cache;
}

// A call's ctx is (handle, index of its device).
// cache_plan(ctx, n_new, lengths, block_table, free_pages, free_count, page, n_slots, new_lengths, new_count)
static PyObject* cache_plan(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    BEGIN
    need(nargs == 10, "ten arguments");
    const context on(a[0]);
    const at::Tensor &n_new = on.dense(a[1], at::kInt, "n_new int32, dense"), &lengths = on.dense(a[2], at::kInt, "lengths int32, dense");
    const at::Tensor &table = on.dense(a[3], at::kInt, "block_table int32, dense"), &pages = on.dense(a[4], at::kInt, "free_pages int32, dense");
    const at::Tensor& count = on.dense(a[5], at::kInt, "free_count int32, dense");
    const int32_t n = fits(n_new.numel(), "n_new"), page = word(a[6], "page"), n_slots = word(a[7], "n_slots");
    need(lengths.numel() == n && table.dim() == 2 && table.size(0) == n && count.numel() == 1, "a length and a row of the table for every stream");
    // one allocation for all outputs that are not given
    const int64_t room = n_slots > 0 ? n_slots : 0, more = given(a[8]) ? 0 : n;
    const at::Tensor made = fresh({room + n + 1 + more + (given(a[9]) ? 0 : 1)}, n_new, at::kInt);
    const at::Tensor slots = part(made, 0, room), off = part(made, room, n + 1);
    const at::Tensor after = given(a[8]) ? on.dense(a[8], at::kInt, "new_lengths int32, dense") : part(made, room + n + 1, n);
    const at::Tensor left = given(a[9]) ? on.dense(a[9], at::kInt, "new_count int32, dense") : part(made, room + n + 1 + more, 1);
    need(after.numel() == n && left.numel() == 1, "new_lengths and new_count as long as lengths and free_count");
    const rh_status st = f_plan(on.handle, (const int32_t*)n_new.data_ptr(), (const int32_t*)lengths.data_ptr(), n, page, fits(pages.numel(), "free_pages"),
                                fits(table.size(1), "block_table"), (int32_t*)table.data_ptr(), (int32_t*)pages.data_ptr(), (const int32_t*)count.data_ptr(),
                                (int32_t*)slots.data_ptr(), n_slots, (int32_t*)off.data_ptr(), (int32_t*)after.data_ptr(), (int32_t*)left.data_ptr());
    if (st != RH_OK) return status(st);
    return tuple_of({wrap(slots), wrap(off), wrap(after), wrap(left)});
    END
}

// cache_write(ctx, cache, k, v, slots)
static PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    BEGIN
    need(nargs == 5, "five arguments");
    const context on(a[0]);
    const rh_kv_cache c = on.cache(a[1]);
    const at::Tensor &k = on.tensor(a[2], "k on the GPU"), &v = on.tensor(a[3], "v on the GPU"), &slots = on.dense(a[4], at::kInt, "slots int32, dense");
    const int32_t n = fits(slots.numel(), "slots");
    need(k.scalar_type() == v.scalar_type() && k.dim() == 3 && k.size(0) == n && k.size(1) == c.heads && k.size(2) == c.dim && v.sizes() == k.sizes(),
         "k and v alike, [n, heads, dim] of the cache");
    need(k.stride(2) == 1 && v.stride(2) == 1, "the elements of a head lie side by side");
    const int64_t ks[2] = {k.stride(0), k.stride(1)}, vs[2] = {v.stride(0), v.stride(1)};
    return status(f_write(on.handle, &c, k.data_ptr(), ks, v.data_ptr(), vs, type_of(k), (const int32_t*)slots.data_ptr(), n));
    END
}

// cache_attend(ctx, cache, q, block_table, lengths, scale, window, out, want_lse) -> (out, lse or None)
static PyObject* cache_attend(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    BEGIN
    need(nargs == 9, "nine arguments");
    const context on(a[0]);
    const rh_kv_cache c = on.cache(a[1]);
    const at::Tensor &q = on.tensor(a[2], "q on the GPU"), &table = on.dense(a[3], at::kInt, "block_table int32, dense"), &lengths = on.dense(a[4], at::kInt, "lengths int32, dense");
    need(q.dim() == 3 && q.size(2) == c.dim && q.stride(2) == 1, "q [n_streams, q_heads, dim] of the cache, elements side by side");
    const int32_t n = fits(q.size(0), "q"), heads = fits(q.size(1), "q");
    need(table.dim() == 2 && table.size(0) == n && lengths.numel() == n, "a length and a row of the table for every stream");
    const double scale = given(a[5]) ? PyFloat_AsDouble(a[5]) : 1.0 / std::sqrt((double)c.dim);
    need(!PyErr_Occurred(), "scale");
    const int32_t window = word(a[6], "window");
    const at::Tensor out = given(a[7]) ? on.tensor(a[7], "out on the GPU") : fresh(q.sizes(), q, q.scalar_type());
    need(out.scalar_type() == q.scalar_type() && out.is_contiguous() && out.sizes() == q.sizes(), "out as q, dense");
    at::Tensor lse;
    if (truth(a[8], "want_lse")) lse = fresh({n, heads}, q, at::kFloat);
    const int64_t qs[2] = {q.stride(0), q.stride(1)};
    const rh_status st = f_attend(on.handle, &c, q.data_ptr(), qs, type_of(q), heads, (const int32_t*)table.data_ptr(), fits(table.size(1), "block_table"),
                                  (const int32_t*)lengths.data_ptr(), n, (float)scale, window, out.data_ptr(), lse.defined() ? (float*)lse.data_ptr() : nullptr);
    if (st != RH_OK) return status(st);
    return tuple_of({wrap(out), wrap(lse)});
    END
}

// norm_residual(ctx, x, weight, residual, eps, outputs, sum_out) -> (sum, y, y8, y8_scale), None where not asked for
static PyObject* norm_residual(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    BEGIN
    need(nargs == 7, "seven arguments");
    const context on(a[0]);
    const at::Tensor &x = on.tensor(a[1], "x on the GPU"), &weight = on.dense(a[2], at::kFloat, "weight float32, dense");
    need(x.dim() == 2 && x.stride(1) == 1 && weight.numel() == x.size(1), "x [rows, cols], elements side by side, and a weight for every column");
    const int32_t rows = fits(x.size(0), "x"), cols = fits(x.size(1), "x");
    const double eps = PyFloat_AsDouble(a[4]);
    need(!PyErr_Occurred(), "eps");
    const bool same = PyUnicode_Check(a[5]) && !PyUnicode_CompareWithASCIIString(a[5], "same"), both = PyUnicode_Check(a[5]) && !PyUnicode_CompareWithASCIIString(a[5], "both");
    need(same || both || (PyUnicode_Check(a[5]) && !PyUnicode_CompareWithASCIIString(a[5], "e4m3")), "outputs \"same\", \"e4m3\" or \"both\"");
    at::Tensor residual, sum, y, y8, scale;
    if (given(a[3])) {
        residual = on.tensor(a[3], "residual on the GPU");
        need(residual.scalar_type() == x.scalar_type() && residual.sizes() == x.sizes() && residual.stride(1) == 1, "residual as x");
        sum = given(a[6]) ? on.tensor(a[6], "sum_out on the GPU") : fresh(x.sizes(), x, x.scalar_type());
        need(sum.scalar_type() == x.scalar_type() && sum.sizes() == x.sizes() && sum.stride(1) == 1, "sum_out as x");
    }
    if (same || both) y = fresh(x.sizes(), x, x.scalar_type());
    if (!same) { y8 = fresh(x.sizes(), x, at::kFloat8_e4m3fn); scale = fresh({rows}, x, at::kFloat); }
    auto row = [&](const at::Tensor& t) { return t.defined() && rows > 1 ? t.stride(0) : (int64_t)cols; };
    auto at_ = [](const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; };
    const rh_status st = f_norm(on.handle, x.data_ptr(), row(x), at_(residual), row(residual), (const float*)weight.data_ptr(), type_of(x), rows, cols,
                                (float)eps, at_(sum), row(sum), at_(y), (uint8_t*)at_(y8), (float*)at_(scale));
    if (st != RH_OK) return status(st);
    return tuple_of({wrap(sum), wrap(y), wrap(y8), wrap(scale)});
    END
}

// matvec_packed(ctx, x, w, w_scale, x_scale, relu, out_dtype, out) -> out
static PyObject* matvec_packed(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    BEGIN
    need(nargs == 8, "eight arguments");
    const context on(a[0]);
    const at::Tensor &x = on.tensor(a[1], "x on the GPU"), &w = on.dense(a[2], at::kByte, "w uint8, dense"), &ws = on.dense(a[3], at::kByte, "w_scale uint8, dense");
    need(x.dim() == 2 && x.stride(1) == 1 && ws.dim() == 2 && w.dim() == 2, "x [rows, n_in], elements side by side, w and w_scale of two dimensions");
    const int32_t rows = fits(x.size(0), "x"), n_in = fits(x.size(1), "x"), n_out = fits(ws.size(0), "w_scale");
    const int64_t blocks = ws.size(1);
    need(blocks == ((int64_t)n_in + 31) / 32 && w.size(0) == n_out && w.size(1) == 16 * blocks, "w [n_out, 16 * ceil(n_in / 32)], w_scale [n_out, ceil(n_in / 32)]");
    const float* xs = nullptr;
    if (given(a[4])) {
        const at::Tensor& s = on.dense(a[4], at::kFloat, "x_scale float32, dense");
        need(s.numel() == rows, "x_scale [rows]");
        xs = (const float*)s.data_ptr();
    }
    need(!given(a[6]) || THPDtype_Check(a[6]), "out_dtype a torch.dtype");
    const at::ScalarType kind = given(a[6]) ? ((THPDtype*)a[6])->scalar_type : x.scalar_type() == at::kFloat ? at::kFloat : at::kBFloat16;
    const at::Tensor out = given(a[7]) ? on.tensor(a[7], "out on the GPU") : fresh({rows, n_out}, x, kind);
    need(out.dim() == 2 && out.size(0) == rows && out.size(1) == n_out && out.stride(1) == 1 && (!given(a[6]) || out.scalar_type() == kind), "out [rows, n_out]");
    const bool relu = truth(a[5], "relu");
    const rh_status st = f_matvec(on.handle, x.data_ptr(), type_of(x), rows > 1 ? x.stride(0) : n_in, xs, (const uint8_t*)w.data_ptr(), (const uint8_t*)ws.data_ptr(),
                                  rows, n_out, n_in, relu, out.data_ptr(), type_of(out), rows > 1 ? out.stride(0) : n_out);
    if (st != RH_OK) return status(st);
    return wrap(out);
    END
}

// init(plan, write, attend, norm, matvec): addresses of the library's functions
static PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    BEGIN
    need(n == 5, "five addresses");
    f_plan = (decltype(f_plan))integer(a[0], "an address"); f_write = (decltype(f_write))integer(a[1], "an address");
    f_attend = (decltype(f_attend))integer(a[2], "an address"); f_norm = (decltype(f_norm))integer(a[3], "an address");
    f_matvec = (decltype(f_matvec))integer(a[4], "an address");
    Py_RETURN_NONE;
    END
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
static PyMethodDef methods[] = {METHOD(kv_desc), METHOD(cache_plan), METHOD(cache_write), METHOD(cache_attend), METHOD(norm_residual), METHOD(matvec_packed), METHOD(init),
                                {nullptr, nullptr, 0, nullptr}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_seq", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
PyMODINIT_FUNC PyInit__seq() { return PyModule_Create(&module); }
