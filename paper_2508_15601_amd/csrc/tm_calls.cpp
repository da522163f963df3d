// The online entry points of the Python binding as native calls: the argument checks of binding.py's functions and the
// call into the C ABI, without an interpreted step in between.
//
// Why native: a decode call's kernel lasts 3-10 us, and the interpreted checks plus ctypes marshalling took 8-10 us of
// host time per call, so a stream of small calls was bound by the host (K = N = 4096, M = 1: 8.5 us per call against
// 3.5 us of kernel).  Here a tensor argument costs a type check and a few field reads.
//
// Tensors are checked as the binding promises: device tensor and data type (TypeError), contiguous and of the shape the
// handle asks for (ValueError), errors of the library as TmError.  The interpreter lock is released during the library
// call.
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/autograd/python_variable.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <initializer_list>

#include "tm_attn.h"
#include "tm_paged.h"
#include "tm_w4.h"

namespace {

PyObject* g_tm_error = nullptr;                          // binding.TmError
PyObject *s_h, *s_K, *s_N, *s_experts, *s_batch, *s_kv_heads, *s_stream, *s_table, *s_offsets, *s_positions,
    *s_max_count, *s_max_len, *s_weight, *s_eps, *s_offset, *s_centred, *s_pages, *s_count;    // attribute names, interned

struct Failed {};                                        // a Python exception is set

[[noreturn]] void raise(PyObject* type, const char* text)
{
    PyErr_SetString(type, text);
    throw Failed{};
}

// int(o) and float(o): everything the two builtins take.
long long as_int(PyObject* o)
{
    PyObject* n = PyLong_CheckExact(o) ? (Py_INCREF(o), o) : PyNumber_Long(o);
    if (!n) throw Failed{};
    const long long v = PyLong_AsLongLong(n);
    Py_DECREF(n);
    if (v == -1 && PyErr_Occurred()) throw Failed{};
    return v;
}

double as_double(PyObject* o)
{
    PyObject* f = PyFloat_CheckExact(o) ? (Py_INCREF(o), o) : PyNumber_Float(o);
    if (!f) throw Failed{};
    const double v = PyFloat_AS_DOUBLE(f);
    Py_DECREF(f);
    return v;
}

PyObject* attr(PyObject* o, PyObject* name)              // new reference
{
    PyObject* v = PyObject_GetAttr(o, name);
    if (!v) throw Failed{};
    return v;
}

long long int_attr(PyObject* o, PyObject* name)
{
    PyObject* v = attr(o, name);
    const long long x = PyLong_AsLongLong(v);
    Py_DECREF(v);
    if (x == -1 && PyErr_Occurred()) throw Failed{};
    return x;
}

void* handle_of(PyObject* owner, const char* freed)
{
    const long long h = int_attr(owner, s_h);
    if (!h) raise(PyExc_ValueError, freed);
    return (void*)h;
}

const at::Tensor& tensor(PyObject* o, const char* what)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s must be a device tensor", what);
        throw Failed{};
    }
    return THPVariable_Unpack(o);
}

void* device_ptr(const at::Tensor& t, at::ScalarType type, const char* what)
{
    if (!t.is_cuda()) {
        PyErr_Format(PyExc_TypeError, "%s must be a device tensor", what);
        throw Failed{};
    }
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s must have dtype torch.%s, got %S", what,
                     type == at::kHalf ? "float16" : type == at::kInt ? "int32" : type == at::kLong ? "int64" : "uint8",
                     (PyObject*)torch::getTHPDtype(t.scalar_type()));
        throw Failed{};
    }
    if (!t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be contiguous", what);
        throw Failed{};
    }
    return t.data_ptr();
}

uint16_t* half_ptr(const at::Tensor& t, const char* what) { return (uint16_t*)device_ptr(t, at::kHalf, what); }

bool shape_is(const at::Tensor& t, std::initializer_list<int64_t> want)
{
    const auto have = t.sizes();
    if (have.size() != want.size()) return false;
    size_t i = 0;
    for (int64_t w : want)
        if (have[i++] != w) return false;
    return true;
}

tm_stream stream_of(PyObject* stream)
{
    if (stream == Py_None) return (tm_stream)c10::hip::getCurrentHIPStream().stream();
    return (tm_stream)int_attr(stream, s_stream);
}

template <class F>
void call(F&& f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    if (rc == TM_OK) return;
    PyObject* args = Py_BuildValue("(is)", rc, tm_last_error());
    if (args) {
        PyErr_SetObject(g_tm_error, args);
        Py_DECREF(args);
    }
    throw Failed{};
}

thread_local int t_device = -1;                          // the current device, asked for once a call

// Shared frame of the entry points: argument count, exceptions, and the object handed back (the output tensor or None).
template <class F>
PyObject* entry(Py_ssize_t have, Py_ssize_t want, PyObject* result, F&& f)
{
    if (have != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, have);
        return nullptr;
    }
    t_device = -1;
    try {
        f();
    } catch (const Failed&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
    Py_INCREF(result);
    return result;
}

constexpr const char* kPackedFreed = "packed handle already freed";
constexpr const char* kGroupFreed = "expert group already freed";
constexpr const char* kCacheFreed = "cache already freed";
constexpr const char* kGemmShapes = "X/Y shapes do not match the packed weight";

// The product's own arguments, checked: X [M][K], Y [M][n_out].
struct GemmArgs {
    const at::Tensor &X, &Y;
    const int64_t M, N;
    GemmArgs(PyObject* x, PyObject* packed, PyObject* y, bool halved, const char* shapes)
        : X(tensor(x, "X")), Y(tensor(y, "Y")), M(X.dim() > 0 ? X.size(0) : 0), N(int_attr(packed, s_N))
    {
        if (X.dim() != 2 || X.size(1) != int_attr(packed, s_K) || !shape_is(Y, {M, halved ? N / 2 : N})) raise(PyExc_ValueError, shapes);
    }
};

PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n)          // X, packed, Y, stream
{
    return entry(n, 4, n > 2 ? a[2] : Py_None, [&] {
        GemmArgs g(a[0], a[1], a[2], false, kGemmShapes);
        if (g.M == 0) return;
        const uint16_t* x = half_ptr(g.X, "X");
        const auto* h = (const tm_packed_w4*)handle_of(a[1], kPackedFreed);
        uint16_t* y = half_ptr(g.Y, "Y");
        const tm_stream st = stream_of(a[3]);
        call([&] { return tm_gemm_w4a16(x, h, y, (int)g.M, st); });
    });
}

PyObject* gemm_static(PyObject*, PyObject* const* a, Py_ssize_t n)   // X, packed, Y, stream
{
    return entry(n, 4, n > 2 ? a[2] : Py_None, [&] {
        GemmArgs g(a[0], a[1], a[2], false, kGemmShapes);
        if (g.M == 0) return;
        const uint16_t* x = half_ptr(g.X, "X");
        const auto* h = (const tm_packed_w4*)handle_of(a[1], kPackedFreed);
        uint16_t* y = half_ptr(g.Y, "Y");
        const tm_stream st = stream_of(a[3]);
        call([&] { return tm_gemm_w4a16_static(x, h, y, (int)g.M, st); });
    });
}

PyObject* gemm_ws(PyObject*, PyObject* const* a, Py_ssize_t n)       // X, packed, Y, workspace, stream
{
    return entry(n, 5, n > 2 ? a[2] : Py_None, [&] {
        GemmArgs g(a[0], a[1], a[2], false, kGemmShapes);
        if (g.M == 0) return;
        const uint16_t* x = half_ptr(g.X, "X");
        const auto* h = (const tm_packed_w4*)handle_of(a[1], kPackedFreed);
        uint16_t* y = half_ptr(g.Y, "Y");
        const at::Tensor& w = tensor(a[3], "workspace");
        void* ws = device_ptr(w, at::kByte, "workspace");
        const size_t bytes = (size_t)w.numel();
        const tm_stream st = stream_of(a[4]);
        call([&] { return tm_gemm_w4a16_ws(x, h, y, (int)g.M, ws, bytes, st); });
    });
}

PyObject* gemm_ex(PyObject*, PyObject* const* a, Py_ssize_t n)       // X, packed, Y, bias, residual, act, stream
{
    return entry(n, 7, n > 2 ? a[2] : Py_None, [&] {
        constexpr const char* shapes = "X / Y / bias / residual shapes do not match the packed weight";
        const int act = (int)as_int(a[5]);
        GemmArgs g(a[0], a[1], a[2], act == TM_ACT_SILU_MUL, shapes);
        const at::Tensor* bias = a[3] == Py_None ? nullptr : &tensor(a[3], "bias");
        const at::Tensor* residual = a[4] == Py_None ? nullptr : &tensor(a[4], "residual");
        if ((bias && !shape_is(*bias, {g.N})) || (residual && residual->sizes() != g.Y.sizes())) raise(PyExc_ValueError, shapes);
        if (g.M == 0) return;
        tm_epilogue epi{};
        if (bias) epi.bias = half_ptr(*bias, "bias");
        if (residual) epi.residual = half_ptr(*residual, "residual");
        epi.act = act;
        const uint16_t* x = half_ptr(g.X, "X");
        const auto* h = (const tm_packed_w4*)handle_of(a[1], kPackedFreed);
        uint16_t* y = half_ptr(g.Y, "Y");
        const tm_stream st = stream_of(a[6]);
        call([&] { return tm_gemm_w4a16_ex(x, h, y, (int)g.M, &epi, st); });
    });
}

PyObject* gemm_grouped(PyObject*, PyObject* const* a, Py_ssize_t n)  // X, group, offsets, Y, act, stream
{
    return entry(n, 6, n > 3 ? a[3] : Py_None, [&] {
        constexpr const char* shapes = "X/Y/offsets shapes do not match the expert group";
        const int act = (int)as_int(a[4]);
        GemmArgs g(a[0], a[1], a[3], act == TM_ACT_SILU_MUL, shapes);
        const at::Tensor& off = tensor(a[2], "offsets");
        PyObject* experts = attr(a[1], s_experts);
        const Py_ssize_t count = PyObject_Size(experts);
        Py_DECREF(experts);
        if (count < 0) throw Failed{};
        if (off.numel() != count + 1) raise(PyExc_ValueError, shapes);
        if (g.M == 0) return;
        const uint16_t* x = half_ptr(g.X, "X");
        const auto* h = (const tm_expert_group*)handle_of(a[1], kGroupFreed);
        const auto* o = (const int32_t*)device_ptr(off, at::kInt, "offsets");
        uint16_t* y = half_ptr(g.Y, "Y");
        const tm_stream st = stream_of(a[5]);
        call([&] { return tm_gemm_w4a16_grouped_act(x, h, o, y, (int)g.M, act, st); });
    });
}

PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n)     // cache, K_new, V_new, positions, stream
{
    return entry(n, 5, Py_None, [&] {
        const at::Tensor &K = tensor(a[1], "K_new"), &V = tensor(a[2], "V_new"), &pos = tensor(a[3], "positions");
        const int64_t batch = int_attr(a[0], s_batch);
        if (K.dim() != 4 || K.sizes() != V.sizes() || K.size(0) != batch || K.size(2) != int_attr(a[0], s_kv_heads) ||
            K.size(3) != 128 || pos.numel() != batch)
            raise(PyExc_ValueError, "K_new / V_new / positions shapes do not match the cache");
        auto* h = (tm_kv_cache*)handle_of(a[0], kCacheFreed);
        const uint16_t *k = half_ptr(K, "K_new"), *v = half_ptr(V, "V_new");
        const auto* p = (const int32_t*)device_ptr(pos, at::kInt, "positions");
        const tm_stream st = stream_of(a[4]);
        call([&] { return tm_kv_append(h, k, v, p, (int)K.size(1), st); });
    });
}

PyObject* attn_decode(PyObject*, PyObject* const* a, Py_ssize_t n)   // Q, cache, lens, O, scale, max_len, stream
{
    return entry(n, 7, n > 3 ? a[3] : Py_None, [&] {
        const at::Tensor &Q = tensor(a[0], "Q"), &lens = tensor(a[2], "lens"), &O = tensor(a[3], "O");
        const int64_t batch = int_attr(a[1], s_batch);
        if (Q.dim() != 3 || Q.size(0) != batch || Q.size(2) != 128 || O.sizes() != Q.sizes() || lens.numel() != batch)
            raise(PyExc_ValueError, "Q / O / lens shapes do not match the cache");
        const uint16_t* q = half_ptr(Q, "Q");
        const auto* h = (const tm_kv_cache*)handle_of(a[1], kCacheFreed);
        const auto* l = (const int32_t*)device_ptr(lens, at::kInt, "lens");
        uint16_t* o = half_ptr(O, "O");
        const float scale = (float)as_double(a[4]);
        const int max_len = (int)as_int(a[5]);
        const tm_stream st = stream_of(a[6]);
        call([&] { return tm_attn_decode(q, h, l, o, (int)Q.size(1), scale, max_len, st); });
    });
}

PyObject* attn_prefill(PyObject*, PyObject* const* a, Py_ssize_t n)  // Q, cache, positions, O, scale, counts, stream
{
    return entry(n, 7, n > 3 ? a[3] : Py_None, [&] {
        const at::Tensor &Q = tensor(a[0], "Q"), &O = tensor(a[3], "O"), &pos = tensor(a[2], "positions");
        const at::Tensor* counts = a[5] == Py_None ? nullptr : &tensor(a[5], "counts");
        if (Q.dim() != 4 || Q.size(3) != 128 || O.sizes() != Q.sizes())
            raise(PyExc_ValueError, "Q and O must be [batch][count][q_heads][128]");
        // The launch covers every sequence of the cache, and the C ABI cannot see how long an array is: a shorter one would be
        // read, and O written, out of range.  (A longer one is fine: its first `batch` entries count.)
        const int64_t batch = int_attr(a[1], s_batch);
        if (Q.size(0) < batch || pos.numel() < batch || (counts && counts->numel() < batch))
            raise(PyExc_ValueError, "Q / O / positions / counts have fewer sequences than the cache");
        const auto* c = counts ? (const int32_t*)device_ptr(*counts, at::kInt, "counts") : nullptr;
        const uint16_t* q = half_ptr(Q, "Q");
        const auto* h = (const tm_kv_cache*)handle_of(a[1], kCacheFreed);
        const auto* p = (const int32_t*)device_ptr(pos, at::kInt, "positions");
        uint16_t* o = half_ptr(O, "O");
        const double scale_d = PyFloat_AsDouble(a[4]);                     // a number: no text here, unlike float()
        if (scale_d == -1.0 && PyErr_Occurred()) throw Failed{};
        const float scale = (float)scale_d;
        const tm_stream st = stream_of(a[6]);
        call([&] { return tm_attn_prefill(q, h, p, c, (int)Q.size(1), o, (int)Q.size(2), scale, st); });
    });
}

// ---- paged cache and rotary positions.  Tensors have to lie on the current device; rows of token arrays may lie apart (a part of a fused
// projection's output is taken as it lies), heads and dimensions may not.

constexpr const char* kRopeFreed = "rope already freed";
constexpr const char* kPagedFreed = "paged cache already freed";

void on_current_device(const at::Tensor& t, const char* what)
{
    if (t_device < 0) t_device = (int)c10::hip::current_device();
    if (t.get_device() != t_device) {
        PyErr_Format(PyExc_ValueError, "%s is on device %d, the current device is %d", what, (int)t.get_device(), t_device);
        throw Failed{};
    }
}

const int32_t* int_ptr(const at::Tensor& t, const char* what)
{
    const auto* p = (const int32_t*)device_ptr(t, at::kInt, what);
    on_current_device(t, what);
    return p;
}

// fp16 [tokens][heads][dim]
struct TokenRows {
    uint16_t* p;
    int64_t stride;
    TokenRows(const at::Tensor& t, const char* what)
    {
        if (!t.is_cuda() || t.scalar_type() != at::kHalf) device_ptr(t, at::kHalf, what);          // raises what it raises for the other entry points
        on_current_device(t, what);
        const int64_t heads = t.size(1), dim = t.size(2);
        if ((dim > 1 && t.stride(2) != 1) || (heads > 1 && t.stride(1) != dim) || (t.size(0) > 1 && t.stride(0) < heads * dim)) {
            PyErr_Format(PyExc_ValueError, "%s must have contiguous heads and rows that do not overlap", what);
            throw Failed{};
        }
        p = (uint16_t*)t.data_ptr();
        stride = t.size(0) > 1 ? t.stride(0) : heads * dim;
    }
};

// The sequences of a call: a binding.PagedBatch.  It keeps the tensors; their addresses are read here.
struct Sequences {
    tm_paged_batch b{};
    Sequences(PyObject* batch, int64_t tokens)
    {
        PyObject* held[3] = {nullptr, nullptr, nullptr};
        try {
            held[0] = attr(batch, s_table), held[1] = attr(batch, s_offsets), held[2] = attr(batch, s_positions);
            const at::Tensor &table = tensor(held[0], "table"), &offsets = tensor(held[1], "offsets"), &positions = tensor(held[2], "positions");
            if (table.dim() != 2 || offsets.numel() != table.size(0) + 1 || positions.numel() != table.size(0))
                raise(PyExc_ValueError, "need table [batch][max_pages], offsets [batch + 1], positions [batch]");
            b.table = int_ptr(table, "table");
            b.offsets = int_ptr(offsets, "offsets");
            b.positions = int_ptr(positions, "positions");
            b.batch = whole(table.size(0), "batch");
            b.max_pages = whole(table.size(1), "max_pages");
            b.tokens = whole(tokens, "tokens");
            b.max_count = whole(int_attr(batch, s_max_count), "max_count");
            b.max_len = whole(int_attr(batch, s_max_len), "max_len");
        } catch (...) {
            for (PyObject* o : held) Py_XDECREF(o);
            throw;
        }
        for (PyObject* o : held) Py_DECREF(o);
    }
    static int whole(int64_t v, const char* what)
    {
        if (v < 0 || v > 0x7fffffff) {
            PyErr_Format(PyExc_ValueError, "%s = %lld out of range", what, (long long)v);
            throw Failed{};
        }
        return (int)v;
    }
};

// int32 [tokens], or [tokens][axes] where a rope has several.
bool positions_fit(const at::Tensor& pos, int64_t tokens)
{
    return (pos.dim() == 1 || (pos.dim() == 2 && pos.size(1) > 1)) && pos.size(0) == tokens;
}
void check_axes(const at::Tensor& pos, const tm_rope* rope)
{
    const int axes = tm_rope_axes(rope);
    if ((pos.dim() == 1 ? 1 : pos.size(1)) != axes) {
        PyErr_Format(PyExc_ValueError, "the rope has %d axes, positions must be [tokens]%s", axes, axes == 1 ? "" : "[axes]");
        throw Failed{};
    }
}

PyObject* rope_apply(PyObject*, PyObject* const* a, Py_ssize_t n)    // X, positions, rope, Y, stream
{
    return entry(n, 5, n > 3 ? a[3] : Py_None, [&] {
        const at::Tensor &X = tensor(a[0], "X"), &pos = tensor(a[1], "positions"), &Y = tensor(a[3], "Y");
        if (X.dim() != 3 || Y.sizes() != X.sizes() || !positions_fit(pos, X.size(0))) raise(PyExc_ValueError, "need X and Y [tokens][heads][dim], positions [tokens] or [tokens][axes]");
        const TokenRows x(X, "X"), y(Y, "Y");
        const int32_t* p = int_ptr(pos, "positions");
        const auto* h = (const tm_rope*)handle_of(a[2], kRopeFreed);
        check_axes(pos, h);
        const int tokens = Sequences::whole(X.size(0), "tokens"), heads = Sequences::whole(X.size(1), "heads"), dim = Sequences::whole(X.size(2), "dim");
        const tm_stream st = stream_of(a[4]);
        call([&] { return tm_rope_apply(x.p, x.stride, p, h, y.p, y.stride, tokens, heads, dim, st); });
    });
}

// A binding.HeadNorm, or None.  `held` keeps its weight.
struct Norm {
    PyObject* held = nullptr;
    tm_head_norm n{};
    bool on = false;
    Norm() = default;
    Norm(const Norm&) = delete;
    ~Norm() { Py_XDECREF(held); }
    void read(PyObject* o, int64_t heads, int64_t dim, const char* what)
    {
        if (o == Py_None) return;
        held = attr(o, s_weight);
        if (held != Py_None) {
            const at::Tensor& w = tensor(held, what);
            n.weight = half_ptr(w, what);
            on_current_device(w, what);
            if (!shape_is(w, {dim}) && !shape_is(w, {heads, dim})) {
                PyErr_Format(PyExc_ValueError, "%s must be [%lld] or [%lld][%lld]", what, (long long)dim, (long long)heads, (long long)dim);
                throw Failed{};
            }
            n.weight_stride = w.dim() == 2 ? dim : 0;
        }
        PyObject* values[3] = {nullptr, nullptr, nullptr};
        try {
            values[0] = attr(o, s_eps), values[1] = attr(o, s_offset), values[2] = attr(o, s_centred);
            n.eps = as_double(values[0]);
            n.offset = as_double(values[1]);
            const int centred = PyObject_IsTrue(values[2]);
            if (centred < 0) throw Failed{};
            n.centred = centred;
        } catch (...) {
            for (PyObject* v : values) Py_XDECREF(v);
            throw;
        }
        for (PyObject* v : values) Py_DECREF(v);
        on = true;
    }
    const tm_head_norm* get() const { return on ? &n : nullptr; }
};

PyObject* heads_apply(PyObject*, PyObject* const* a, Py_ssize_t n)   // rope, positions, Q, Q_out, q_norm, K, K_out, k_norm, stream
{
    return entry(n, 9, Py_None, [&] {
        const at::Tensor* given[2][2] = {};
        int64_t tokens = -1, dim = 0;
        static const char* const names[2][3] = {{"Q", "Q_out", "q_norm's weight"}, {"K", "K_out", "k_norm's weight"}};
        for (int i = 0; i < 2; ++i) {
            PyObject *x = a[2 + 3 * i], *y = a[3 + 3 * i];
            if ((x == Py_None) != (y == Py_None)) raise(PyExc_ValueError, i ? "K and K_out go together" : "Q and Q_out go together");
            if (x == Py_None) {
                if (a[4 + 3 * i] != Py_None) raise(PyExc_ValueError, i ? "k_norm without K" : "q_norm without Q");
                continue;
            }
            given[i][0] = &tensor(x, names[i][0]), given[i][1] = &tensor(y, names[i][1]);
            const at::Tensor& t = *given[i][0];
            if (t.dim() != 3 || given[i][1]->sizes() != t.sizes() || (tokens >= 0 && (t.size(0) != tokens || t.size(2) != dim)))
                raise(PyExc_ValueError, "need Q, Q_out [tokens][q_heads][dim] and K, K_out [tokens][k_heads][dim]");
            tokens = t.size(0), dim = t.size(2);
        }
        if (tokens < 0) raise(PyExc_ValueError, "neither Q nor K");
        if ((a[0] == Py_None) != (a[1] == Py_None)) raise(PyExc_ValueError, "a rope and positions go together");
        const int32_t* p = nullptr;
        const tm_rope* rope = nullptr;
        if (a[0] != Py_None) {
            const at::Tensor& pos = tensor(a[1], "positions");
            if (!positions_fit(pos, tokens)) raise(PyExc_ValueError, "need positions [tokens] or [tokens][axes]");
            p = int_ptr(pos, "positions");
            rope = (const tm_rope*)handle_of(a[0], kRopeFreed);
            check_axes(pos, rope);
        }
        Norm norms[2];
        tm_head_rows rows[2] = {};
        for (int i = 0; i < 2; ++i) {
            if (!given[i][0]) continue;
            const TokenRows x(*given[i][0], names[i][0]), y(*given[i][1], names[i][1]);
            norms[i].read(a[4 + 3 * i], given[i][0]->size(1), dim, names[i][2]);
            rows[i] = tm_head_rows{x.p, x.stride, y.p, y.stride, Sequences::whole(given[i][0]->size(1), "heads"), norms[i].get()};
        }
        const int count = Sequences::whole(tokens, "tokens"), width = Sequences::whole(dim, "dim");
        const tm_stream st = stream_of(a[8]);
        call([&] { return tm_heads_apply(given[0][0] ? &rows[0] : nullptr, given[1][0] ? &rows[1] : nullptr, p, rope, count, width, st); });
    });
}

// A binding.PageList, and where the count goes: `left`, or its own count.
struct Pages {
    PyObject* held[2] = {nullptr, nullptr};
    tm_page_list l{};
    Pages(const Pages&) = delete;
    Pages(PyObject* list, PyObject* left)
    {
        try {
            held[0] = attr(list, s_pages), held[1] = attr(list, s_count);
            const at::Tensor &pages = tensor(held[0], "pages"), &count = tensor(held[1], "count"), &out = left == Py_None ? count : tensor(left, "left");
            if (pages.dim() != 1 || count.numel() != 1 || out.numel() != 1) raise(PyExc_ValueError, "need pages [capacity], count [1], left [1]");
            l.pages = (int32_t*)int_ptr(pages, "pages");
            l.count = int_ptr(count, "count");
            l.left = (int32_t*)int_ptr(out, "left");
            l.capacity = Sequences::whole(pages.size(0), "capacity");
        } catch (...) {
            drop();
            throw;
        }
    }
    ~Pages() { drop(); }
    void drop()
    {
        for (PyObject*& o : held) Py_CLEAR(o);
    }
};

const int32_t* row_ints(PyObject* o, int64_t rows, const char* what)
{
    const at::Tensor& t = tensor(o, what);
    if (!shape_is(t, {rows})) {
        PyErr_Format(PyExc_ValueError, "%s must be [%lld]", what, (long long)rows);
        throw Failed{};
    }
    return int_ptr(t, what);
}

PyObject* paged_assign(PyObject*, PyObject* const* a, Py_ssize_t n)  // cache, list, batch, lens, counts, slots, short, lens_out, left, tokens, stream
{
    return entry(n, 11, Py_None, [&] {
        int64_t tokens = a[9] == Py_None ? -1 : as_int(a[9]);
        int64_t* slots = nullptr;
        if (a[5] != Py_None) {
            const at::Tensor& t = tensor(a[5], "slots");
            if (t.dim() != 1 || t.numel() < tokens) raise(PyExc_ValueError, "slots must be [tokens]");
            slots = (int64_t*)device_ptr(t, at::kLong, "slots");
            on_current_device(t, "slots");
            if (tokens < 0) tokens = t.numel();
        }
        if (tokens < 0) raise(PyExc_ValueError, "need slots or tokens");
        const Sequences seqs(a[2], tokens);
        const Pages list(a[1], a[8]);
        tm_paged_step s{};
        s.lens = row_ints(a[3], seqs.b.batch, "lens");
        s.counts = row_ints(a[4], seqs.b.batch, "counts");
        s.lens_out = (int32_t*)(a[7] == Py_None ? s.lens : row_ints(a[7], seqs.b.batch, "lens_out"));
        s.lacking = a[6] == Py_None ? nullptr : (int32_t*)row_ints(a[6], seqs.b.batch, "short");
        s.table = (int32_t*)seqs.b.table;
        s.offsets = (int32_t*)seqs.b.offsets;
        s.positions = (int32_t*)seqs.b.positions;
        s.slots = slots;
        s.batch = seqs.b.batch, s.max_pages = seqs.b.max_pages, s.tokens = seqs.b.tokens;
        auto* h = (tm_paged_cache*)handle_of(a[0], kPagedFreed);
        const tm_stream st = stream_of(a[10]);
        call([&] { return tm_paged_assign(h, &list.l, &s, st); });
    });
}

PyObject* paged_release(PyObject*, PyObject* const* a, Py_ssize_t n) // cache, list, table, from, to, left, stream
{
    return entry(n, 7, Py_None, [&] {
        const at::Tensor& table = tensor(a[2], "table");
        if (table.dim() != 2) raise(PyExc_ValueError, "need table [batch][max_pages]");
        auto* entries = (int32_t*)int_ptr(table, "table");
        const int batch = Sequences::whole(table.size(0), "batch"), max_pages = Sequences::whole(table.size(1), "max_pages");
        const int32_t* from = a[3] == Py_None ? nullptr : row_ints(a[3], batch, "first");
        const int32_t* to = a[4] == Py_None ? nullptr : row_ints(a[4], batch, "last");
        const Pages list(a[1], a[5]);
        auto* h = (tm_paged_cache*)handle_of(a[0], kPagedFreed);
        const tm_stream st = stream_of(a[6]);
        call([&] { return tm_paged_release(h, &list.l, entries, batch, max_pages, from, to, st); });
    });
}

void check_tokens(const at::Tensor& t, int64_t tokens, int64_t heads, const char* what)
{
    if (!shape_is(t, {tokens, heads, 128})) {
        PyErr_Format(PyExc_ValueError, "%s must be [%lld][%lld][128]", what, (long long)tokens, (long long)heads);
        throw Failed{};
    }
}

PyObject* paged_append(PyObject*, PyObject* const* a, Py_ssize_t n)  // cache, batch, K, V, rope, Q, Q_out, stream, q_norm, k_norm, positions
{
    return entry(n, 11, n > 6 ? a[6] : Py_None, [&] {
        const at::Tensor &K = tensor(a[2], "K"), &V = tensor(a[3], "V");
        const int64_t tokens = K.dim() ? K.size(0) : 0, heads = int_attr(a[0], s_kv_heads);
        check_tokens(K, tokens, heads, "K");
        check_tokens(V, tokens, heads, "V");
        const Sequences seqs(a[1], tokens);
        const TokenRows k(K, "K"), v(V, "V");
        auto* h = (tm_paged_cache*)handle_of(a[0], kPagedFreed);
        const auto* rope = a[4] == Py_None ? nullptr : (const tm_rope*)handle_of(a[4], kRopeFreed);
        const uint16_t* q = nullptr;
        uint16_t* q_out = nullptr;
        int64_t q_stride = 0, q_out_stride = 0;
        int q_heads = 0;
        if ((a[5] == Py_None) != (a[6] == Py_None)) raise(PyExc_ValueError, "Q and Q_out go together");
        if (a[5] != Py_None) {
            const at::Tensor &Q = tensor(a[5], "Q"), &Q_out = tensor(a[6], "Q_out");
            if (Q.dim() != 3) raise(PyExc_ValueError, "Q must be [tokens][q_heads][128]");
            check_tokens(Q, tokens, Q.size(1), "Q");
            check_tokens(Q_out, tokens, Q.size(1), "Q_out");
            const TokenRows in(Q, "Q"), out(Q_out, "Q_out");
            q = in.p, q_stride = in.stride, q_out = out.p, q_out_stride = out.stride;
            q_heads = Sequences::whole(Q.size(1), "q_heads");
        }
        Norm q_norm, k_norm;
        if (a[8] != Py_None && !q) raise(PyExc_ValueError, "q_norm without Q");
        q_norm.read(a[8], q_heads, 128, "q_norm's weight");
        k_norm.read(a[9], heads, 128, "k_norm's weight");
        tm_append_heads of{rope, nullptr, q_norm.get(), k_norm.get()};
        if (a[10] != Py_None) {
            const at::Tensor& pos = tensor(a[10], "positions");
            if (!rope) raise(PyExc_ValueError, "positions without a rope");
            if (!positions_fit(pos, tokens)) raise(PyExc_ValueError, "need positions [tokens] or [tokens][axes]");
            of.positions = int_ptr(pos, "positions");
            check_axes(pos, rope);
        }
        const tm_stream st = stream_of(a[7]);
        call([&] { return tm_paged_append_heads(h, &seqs.b, k.p, k.stride, v.p, v.stride, &of, q, q_stride, q_out, q_out_stride, q_heads, st); });
    });
}

PyObject* paged_read(PyObject*, PyObject* const* a, Py_ssize_t n)    // cache, batch, K, V, stream
{
    return entry(n, 5, Py_None, [&] {
        const at::Tensor &K = tensor(a[2], "K"), &V = tensor(a[3], "V");
        const int64_t tokens = K.dim() ? K.size(0) : 0, heads = int_attr(a[0], s_kv_heads);
        check_tokens(K, tokens, heads, "K");
        check_tokens(V, tokens, heads, "V");
        const Sequences seqs(a[1], tokens);
        uint16_t *k = half_ptr(K, "K"), *v = half_ptr(V, "V");
        on_current_device(K, "K");
        on_current_device(V, "V");
        const auto* h = (const tm_paged_cache*)handle_of(a[0], kPagedFreed);
        const tm_stream st = stream_of(a[4]);
        call([&] { return tm_paged_read(h, &seqs.b, k, v, st); });
    });
}

// window (None: none) and sinks of a call.
struct Window {
    int window = 0x7fffffff, sinks;
    Window(PyObject* of, PyObject* first) : sinks(whole(first, "sinks"))
    {
        if (of != Py_None) window = whole(of, "window");
        else if (sinks) raise(PyExc_ValueError, "sinks without a window");
    }
    static int whole(PyObject* v, const char* what)
    {
        const long long x = as_int(v);
        if (x < -0x7fffffffLL || x > 0x7fffffffLL) {
            PyErr_Format(PyExc_ValueError, "%s = %lld out of range", what, x);
            throw Failed{};
        }
        return (int)x;
    }
};

PyObject* paged_attn(PyObject*, PyObject* const* a, Py_ssize_t n)    // Q, cache, batch, O, scale, stream, window (None: none), sinks
{
    return entry(n, 8, n > 3 ? a[3] : Py_None, [&] {
        const at::Tensor &Q = tensor(a[0], "Q"), &O = tensor(a[3], "O");
        if (Q.dim() != 3 || Q.size(2) != 128 || O.sizes() != Q.sizes()) raise(PyExc_ValueError, "Q and O must be [tokens][q_heads][128]");
        const Sequences seqs(a[2], Q.size(0));
        const TokenRows q(Q, "Q");
        uint16_t* o = half_ptr(O, "O");
        on_current_device(O, "O");
        const auto* h = (const tm_paged_cache*)handle_of(a[1], kPagedFreed);
        const int q_heads = Sequences::whole(Q.size(1), "q_heads");
        const float scale = (float)as_double(a[4]);
        const tm_stream st = stream_of(a[5]);
        const Window w(a[6], a[7]);
        call([&] { return tm_paged_attn_window(q.p, q.stride, h, &seqs.b, o, q_heads, scale, w.window, w.sinks, st); });
    });
}

PyObject* paged_plan(PyObject*, PyObject* const* a, Py_ssize_t n)    // cache, batch, tokens, q_heads, window, sinks -> (columns, column_rows, rows, pieces)
{
    int v[4] = {0, 0, 0, 0};
    PyObject* none = entry(n, 6, Py_None, [&] {
        const Sequences seqs(a[1], as_int(a[2]));
        const auto* h = (const tm_paged_cache*)handle_of(a[0], kPagedFreed);
        const int q_heads = Sequences::whole(as_int(a[3]), "q_heads");
        const Window w(a[4], a[5]);
        call([&] { return tm_get_paged_window_plan(h, &seqs.b, q_heads, w.window, w.sinks, &v[0], &v[1], &v[2], &v[3]); });
    });
    if (!none) return nullptr;
    Py_DECREF(none);
    return Py_BuildValue("(iiii)", v[0], v[1], v[2], v[3]);
}

PyObject* paged_form(PyObject*, PyObject* const* a, Py_ssize_t n)    // cache, batch, tokens, q_heads, window, sinks -> (launches, column_ctas, alone)
{
    int v[3] = {0, 0, 0};
    PyObject* none = entry(n, 6, Py_None, [&] {
        const Sequences seqs(a[1], as_int(a[2]));
        const auto* h = (const tm_paged_cache*)handle_of(a[0], kPagedFreed);
        const int q_heads = Sequences::whole(as_int(a[3]), "q_heads");
        const Window w(a[4], a[5]);
        call([&] { return tm_get_paged_window_form(h, &seqs.b, q_heads, w.window, w.sinks, &v[0], &v[1], &v[2]); });
    });
    if (!none) return nullptr;
    Py_DECREF(none);
    return Py_BuildValue("(iiN)", v[0], v[1], PyBool_FromLong(v[2]));
}

PyObject* set_error(PyObject*, PyObject* type)
{
    Py_INCREF(type);
    Py_XDECREF(g_tm_error);
    g_tm_error = type;
    Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
constexpr PyMethodDef fast(const char* name)
{
    return {name, (PyCFunction)(void (*)(void))F, METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {fast<gemm>("gemm"),
                           fast<gemm_static>("gemm_static"),
                           fast<gemm_ws>("gemm_ws"),
                           fast<gemm_ex>("gemm_ex"),
                           fast<gemm_grouped>("gemm_grouped"),
                           fast<kv_append>("kv_append"),
                           fast<attn_decode>("attn_decode"),
                           fast<attn_prefill>("attn_prefill"),
                           fast<rope_apply>("rope_apply"),
                           fast<heads_apply>("heads_apply"),
                           fast<paged_assign>("paged_assign"),
                           fast<paged_release>("paged_release"),
                           fast<paged_append>("paged_append"),
                           fast<paged_read>("paged_read"),
                           fast<paged_attn>("paged_attn"),
                           fast<paged_plan>("paged_plan"),
                           fast<paged_form>("paged_form"),
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "tm_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit_tm_calls()
{
    PyObject** names[] = {&s_h, &s_K, &s_N, &s_experts, &s_batch, &s_kv_heads, &s_stream, &s_table, &s_offsets, &s_positions, &s_max_count, &s_max_len,
                           &s_weight, &s_eps, &s_offset, &s_centred, &s_pages, &s_count};
    const char* texts[] = {"_h", "K", "N", "experts", "batch", "kv_heads", "cuda_stream", "table", "offsets", "positions", "max_count", "max_len", "weight", "eps", "offset", "centred", "pages", "count"};
    for (int i = 0; i < 18; ++i)
        if (!(*names[i] = PyUnicode_InternFromString(texts[i]))) return nullptr;
    return PyModule_Create(&g_module);
}
