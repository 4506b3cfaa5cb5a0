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
static decltype(&rh_state_conv) f_conv;
static decltype(&rh_state_scan) f_scan;
static decltype(&rh_norm_gated) f_gated;

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

// which outputs of a norm are asked for
struct kinds {
    bool plain, quantised;
    explicit kinds(PyObject* o)
    {
        auto is = [&](const char* name) { return PyUnicode_Check(o) && !PyUnicode_CompareWithASCIIString(o, name); };
        const bool both = is("both");
        plain = is("same") || both; quantised = is("e4m3") || both;
        need(plain || quantised, "outputs \"same\", \"e4m3\" or \"both\"");
    }
};

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
    const kinds out(a[5]);
    at::Tensor residual, sum, y, y8, scale;
    if (given(a[3])) {
        residual = on.tensor(a[3], "residual on the GPU");
        need(residual.scalar_type() == x.scalar_type() && residual.sizes() == x.sizes() && residual.stride(1) == 1, "residual as x");
        sum = given(a[6]) ? on.tensor(a[6], "sum_out on the GPU") : fresh(x.sizes(), x, x.scalar_type());
        need(sum.scalar_type() == x.scalar_type() && sum.sizes() == x.sizes() && sum.stride(1) == 1, "sum_out as x");
    }
    if (out.plain) y = fresh(x.sizes(), x, x.scalar_type());
    if (out.quantised) { y8 = fresh(x.sizes(), x, at::kFloat8_e4m3fn); scale = fresh({rows}, x, at::kFloat); }
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

// The rows and states of a call: offsets, slots, past and into, the state's first dimension being the pool.
static rh_state_rows rows_of(const context& on, PyObject* offsets, PyObject* slots, PyObject* past, PyObject* into, int64_t n_rows, int64_t n_slots)
{
    rh_state_rows r = {};
    const at::Tensor& s = on.dense(slots, at::kInt, "slots int32, dense");
    r.slots = (const int32_t*)s.data_ptr();
    r.n_streams = fits(s.numel(), "slots"); r.n_rows = fits(n_rows, "rows"); r.n_slots = fits(n_slots, "state");
    if (given(offsets)) {
        const at::Tensor& t = on.dense(offsets, at::kInt, "offsets int32, dense");
        need(t.numel() == s.numel() + 1, "offsets [n_streams + 1]");
        r.offsets = (const int32_t*)t.data_ptr();
    } else need(n_rows == s.numel(), "a row for every stream, or offsets");
    for (int i = 0; i < 2; ++i) {
        PyObject* o = i ? into : past;
        if (!given(o)) continue;
        const at::Tensor& t = on.dense(o, at::kInt, i ? "into int32, dense" : "past int32, dense");
        need(t.numel() == s.numel(), "past and into as long as slots");
        (i ? r.into : r.past) = (const int32_t*)t.data_ptr();
    }
    return r;
}
// a matrix whose rows' elements lie side by side, of `like`'s type and shape
static const at::Tensor& as(const context& on, PyObject* o, const at::Tensor& like, const char* why)
{
    const at::Tensor& t = on.tensor(o, why);
    need(t.scalar_type() == like.scalar_type() && t.sizes() == like.sizes() && t.stride(1) == 1, why);
    return t;
}
static int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
// no element of one matrix (its rows' elements side by side) lies in the other: all of it ahead or behind, or columns side by side in rows of one length
struct matrix {
    int64_t at, rows, stride, bytes;                         // bytes: of a row's elements
    explicit matrix(const at::Tensor& t)
    {
        const int64_t size = (int64_t)t.element_size();
        at = (int64_t)t.data_ptr(); rows = t.size(0);
        bytes = rows ? t.numel() / rows * size : 0;
        stride = rows > 1 ? t.stride(0) * size : bytes;
    }
};
static bool apart(const matrix& a, const matrix& b)
{
    if (!a.bytes || !b.bytes || a.at + (a.rows - 1) * a.stride + a.bytes <= b.at || b.at + (b.rows - 1) * b.stride + b.bytes <= a.at) return true;
    if (a.rows < 2 || b.rows < 2 || a.stride != b.stride || a.stride <= 0) return false;
    const int64_t at = ((b.at - a.at) % a.stride + a.stride) % a.stride;     // b's columns in a's rows
    return at >= a.bytes && at + b.bytes <= a.stride;
}

// state_conv(ctx, x, weight, state, slots, bias, offsets, past, into, silu, out) -> out
static PyObject* state_conv(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    BEGIN
    need(nargs == 11, "eleven arguments");
    const context on(a[0]);
    const at::Tensor &x = on.tensor(a[1], "x on the GPU"), &weight = on.dense(a[2], at::kFloat, "weight float32, dense"), &state = on.tensor(a[3], "state on the GPU");
    need(x.dim() == 2 && x.stride(1) == 1, "x [rows, channels], elements side by side");
    need(weight.dim() == 2 && weight.size(1) == x.size(1), "weight [width, channels]");
    const int32_t channels = fits(x.size(1), "channels"), width = fits(weight.size(0), "width");
    need(state.scalar_type() == x.scalar_type() && state.is_contiguous() && state.dim() == 3 && state.size(1) == width - 1 && state.size(2) == channels,
         "state as x, dense, [n_slots, width - 1, channels]");
    const float* bias = nullptr;
    if (given(a[5])) {
        const at::Tensor& t = on.dense(a[5], at::kFloat, "bias float32, dense");
        need(t.numel() == channels, "bias [channels]");
        bias = (const float*)t.data_ptr();
    }
    const rh_state_rows rows = rows_of(on, a[6], a[4], a[7], a[8], x.size(0), state.size(0));
    const bool silu = truth(a[9], "silu");
    const at::Tensor out = given(a[10]) ? as(on, a[10], x, "out as x") : fresh(x.sizes(), x, x.scalar_type());
    need(!given(a[10]) || (apart(matrix(out), matrix(x)) && apart(matrix(out), matrix(state))), "out apart from x and state");
    const rh_status st = f_conv(on.handle, &rows, x.data_ptr(), row_stride(x), (const float*)weight.data_ptr(), bias, type_of(x), channels, width, silu, state.data_ptr(),
                                out.data_ptr(), row_stride(out));
    if (st != RH_OK) return status(st);
    return wrap(out);
    END
}

// state_scan(ctx, x, dt, a, b, c, state, slots, skip, gate, dt_bias, softplus, offsets, past, into, out) -> out
static PyObject* state_scan(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    BEGIN
    need(nargs == 16, "sixteen arguments");
    const context on(a[0]);
    const at::Tensor& x = on.tensor(a[1], "x on the GPU");
    need(x.dim() == 2 && x.stride(1) == 1, "x [rows, channels], elements side by side");
    const at::Tensor &dt = as(on, a[2], x, "dt as x"), &fade = on.dense(a[3], at::kFloat, "a float32, dense"), &state = on.dense(a[6], at::kFloat, "state float32, dense");
    rh_scan_inputs in = {};
    in.type = type_of(x); in.channels = fits(x.size(1), "channels");
    need(fade.dim() == 2 && fade.size(0) == in.channels, "a [channels, n]");
    in.n = fits(fade.size(1), "n");
    need(state.dim() == 3 && state.size(1) == in.channels && state.size(2) == in.n, "state [n_slots, channels, n]");
    const at::Tensor &b = on.tensor(a[4], "b on the GPU"), &c = on.tensor(a[5], "c on the GPU");
    need(b.dim() == 3 && b.size(0) == x.size(0) && b.size(2) == in.n && c.sizes() == b.sizes() && b.scalar_type() == x.scalar_type() && c.scalar_type() == x.scalar_type(),
         "b and c alike, [rows, groups, n] of x's type");
    in.groups = fits(b.size(1), "groups");
    auto side_by_side = [&](const at::Tensor& t) { return (t.size(2) < 2 || t.stride(2) == 1) && (t.size(1) < 2 || t.stride(1) == t.size(2)); };
    need(side_by_side(b) && side_by_side(c), "the elements of a row of b and of c side by side");
    auto wide = [&](const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : (int64_t)in.groups * in.n; };
    auto per_channel = [&](PyObject* o, const char* why) -> const float* {
        if (!given(o)) return nullptr;
        const at::Tensor& t = on.dense(o, at::kFloat, why);
        need(t.numel() == in.channels, why);
        return (const float*)t.data_ptr();
    };
    in.x = x.data_ptr(); in.dt = dt.data_ptr(); in.b = b.data_ptr(); in.c = c.data_ptr(); in.a = (const float*)fade.data_ptr();
    in.x_stride = row_stride(x); in.dt_stride = row_stride(dt); in.b_stride = wide(b); in.c_stride = wide(c);
    in.skip = per_channel(a[8], "skip float32 [channels], dense"); in.dt_bias = per_channel(a[10], "dt_bias float32 [channels], dense");
    const at::Tensor* gate = given(a[9]) ? &as(on, a[9], x, "gate as x") : nullptr;
    if (gate) { in.gate = gate->data_ptr(); in.gate_stride = row_stride(*gate); }
    in.softplus = truth(a[11], "softplus");
    const rh_state_rows rows = rows_of(on, a[12], a[7], a[13], a[14], x.size(0), state.size(0));
    const at::Tensor out = given(a[15]) ? as(on, a[15], x, "out as x") : fresh(x.sizes(), x, x.scalar_type());
    if (given(a[15])) {
        const matrix y(out);
        need(apart(y, matrix(x)) && apart(y, matrix(dt)) && (!gate || apart(y, matrix(*gate))) && apart(y, matrix(b)) && apart(y, matrix(c)) && apart(y, matrix(state)),
             "out apart from the inputs and the state");
    }
    const rh_status st = f_scan(on.handle, &rows, &in, (float*)state.data_ptr(), out.data_ptr(), row_stride(out));
    if (st != RH_OK) return status(st);
    return wrap(out);
    END
}

// norm_gated(ctx, x, gate, weight, groups, eps, outputs) -> (y, y8, y8_scale), None where not asked for
static PyObject* norm_gated(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    BEGIN
    need(nargs == 7, "seven arguments");
    const context on(a[0]);
    const at::Tensor &x = on.tensor(a[1], "x on the GPU"), &weight = on.dense(a[3], at::kFloat, "weight float32, dense");
    need(x.dim() == 2 && x.stride(1) == 1 && weight.numel() == x.size(1), "x [rows, cols], elements side by side, and a weight for every column");
    const at::Tensor& gate = as(on, a[2], x, "gate as x");
    const int32_t rows = fits(x.size(0), "x"), cols = fits(x.size(1), "x"), groups = word(a[4], "groups");
    const double eps = PyFloat_AsDouble(a[5]);
    need(!PyErr_Occurred(), "eps");
    const kinds out(a[6]);
    at::Tensor y, y8, scale;
    if (out.plain) y = fresh(x.sizes(), x, x.scalar_type());
    if (out.quantised) { y8 = fresh(x.sizes(), x, at::kFloat8_e4m3fn); scale = fresh({rows}, x, at::kFloat); }
    auto at_ = [](const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; };
    const rh_status st = f_gated(on.handle, x.data_ptr(), row_stride(x), gate.data_ptr(), row_stride(gate), (const float*)weight.data_ptr(), type_of(x), rows, cols, groups,
                                 (float)eps, at_(y), (uint8_t*)at_(y8), (float*)at_(scale));
    if (st != RH_OK) return status(st);
    return tuple_of({wrap(y), wrap(y8), wrap(scale)});
    END
}

// init(plan, write, attend, norm, matvec, conv, scan, gated): addresses of the library's functions
static PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    BEGIN
    need(n == 8, "eight addresses");
    f_plan = (decltype(f_plan))integer(a[0], "an address"); f_write = (decltype(f_write))integer(a[1], "an address");
    f_attend = (decltype(f_attend))integer(a[2], "an address"); f_norm = (decltype(f_norm))integer(a[3], "an address");
    f_matvec = (decltype(f_matvec))integer(a[4], "an address"); f_conv = (decltype(f_conv))integer(a[5], "an address");
    f_scan = (decltype(f_scan))integer(a[6], "an address"); f_gated = (decltype(f_gated))integer(a[7], "an address");
    Py_RETURN_NONE;
    END
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
static PyMethodDef methods[] = {METHOD(kv_desc), METHOD(cache_plan), METHOD(cache_write), METHOD(cache_attend), METHOD(norm_residual), METHOD(matvec_packed),
                                METHOD(state_conv), METHOD(state_scan), METHOD(norm_gated), METHOD(init), {nullptr, nullptr, 0, nullptr}};
static PyModuleDef module = {PyModuleDef_HEAD_INIT, "_seq", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};
PyMODINIT_FUNC PyInit__seq() { return PyModule_Create(&module); }
