// The hot calls of sar.py: tensors checked and handed over to the C entry points.
//
// A short step is bound by the host: written in Python over ctypes, a call cost 2.5 to 3 us beside the entry point's own
// (HIP launches, 3 us each), and an all-blocks call another 1 to 2 us for every block, whose tensors were looked at attribute
// by attribute.  The functions here take the arguments of sar.py's functions of the same names, in their order, and check
// what those state; they keep nothing between calls.
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include <limits>
#include <string>
#include <vector>

#include "../../include/sar_mi355x.h"

namespace {

// A Python error is set.
struct Raised {};

// What the library, or a check here, refuses: sar.SarError with this code and text.
struct Refused {
    int code;
    std::string text;
};

[[noreturn]] void raise_sar(int code, const std::string& text) { throw Refused{code, text}; }

// SarError is that of the package this module was imported as a part of, whatever its name.
void set_error(PyObject* self, const Refused& r)
{
    const char* own = PyModule_GetName(self);
    if (!own) return;
    std::string name(own);
    name.erase(name.rfind('.') + 1);
    PyObject* m = PyImport_ImportModule((name + "sar").c_str());
    PyObject* type = m ? PyObject_GetAttrString(m, "SarError") : nullptr;
    PyObject* e = type ? PyObject_CallFunction(type, "is", r.code, r.text.c_str()) : nullptr;
    if (e) PyErr_SetObject(type, e);
    Py_XDECREF(e);
    Py_XDECREF(type);
    Py_XDECREF(m);
}

[[noreturn]] void refuse(const char* fmt, ...) __attribute__((format(printf, 1, 2)));
void refuse(const char* fmt, ...)
{
    char text[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof text, fmt, ap);
    va_end(ap);
    raise_sar(SAR_ERR_INVALID_ARG, text);
}

void check(int rc)
{
    if (rc != SAR_OK) raise_sar(rc, sar_last_error());
}

// ---- arguments

const at::Tensor& tensor(PyObject* o)
{
    if (!THPVariable_Check(o)) {
        // (None has none of a tensor's attributes, and says so)
        PyErr_Format(o == Py_None ? PyExc_AttributeError : PyExc_TypeError, "expected a tensor, got %s", Py_TYPE(o)->tp_name);
        throw Raised{};
    }
    return THPVariable_Unpack(o);
}

template <typename T = void>
T* ptr_of(const at::Tensor& t)
{
    if (!t.is_contiguous()) {
        PyErr_SetString(PyExc_AssertionError, "tensors passed to the library must be contiguous");
        throw Raised{};
    }
    return static_cast<T*>(t.data_ptr());
}

// the address of a tensor, or null for None
template <typename T = void>
T* ptr(PyObject* o)
{
    return o == Py_None ? nullptr : ptr_of<T>(tensor(o));
}

// an address given as a number, or null for None
template <typename T>
T* address(PyObject* o)
{
    if (o == Py_None) return nullptr;
    PyObject* n = PyLong_Check(o) ? (Py_INCREF(o), o) : PyObject_GetAttrString(o, "value");   // (ctypes.c_void_p)
    if (!n) throw Raised{};
    void* p = n == Py_None ? nullptr : PyLong_AsVoidPtr(n);
    Py_DECREF(n);
    if (PyErr_Occurred()) throw Raised{};
    return static_cast<T*>(p);
}

int64_t integer(PyObject* o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}

float real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised{};
    return (float)v;
}

int truth(PyObject* o)
{
    PyObject* n = PyNumber_Long(o);
    if (!n) throw Raised{};
    const long long v = PyLong_AsLongLong(n);
    Py_DECREF(n);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v != 0;
}

std::string type_name(at::ScalarType t)
{
    return std::string("torch.") + c10::getDtypeNames(t).first;
}

int dtype_code(at::ScalarType t)
{
    if (t == at::kFloat) return SAR_F32;
    if (t == at::kBFloat16) return SAR_BF16;
    raise_sar(SAR_ERR_UNSUPPORTED, "dtype " + type_name(t));
}

size_t bytes_of(PyObject* o) { return tensor(o).numel() * tensor(o).element_size(); }

// ... of scratch that a call may do without
size_t bytes_if(PyObject* o) { return o == Py_None ? 0 : bytes_of(o); }

std::string shape_text(const at::Tensor& t)
{
    std::string s = "(";
    for (int64_t d = 0; d < t.dim(); ++d) s += (d ? ", " : "") + std::to_string(t.size(d));
    return s + (t.dim() == 1 ? ",)" : ")");
}

// The C side takes one size for both.
void same_shape(const at::Tensor& a, PyObject* o)
{
    if (o == Py_None) return;
    const at::Tensor& b = tensor(o);
    if (a.sizes() != b.sizes() || a.scalar_type() != b.scalar_type())
        raise_sar(SAR_ERR_INVALID_ARG, "tensors of shape " + shape_text(a) + " " + type_name(a.scalar_type()) + " and " +
                                           shape_text(b) + " " + type_name(b.scalar_type()) + " must match");
}

// The sizes of a tensor of `N` dimensions.
template <int N>
void unpack_sizes(const at::Tensor& t, int64_t (&out)[N])
{
    if (t.dim() != N) {
        PyErr_Format(PyExc_ValueError, "expected a tensor of %d dimensions, got %lld", N, (long long)t.dim());
        throw Raised{};
    }
    for (int d = 0; d < N; ++d) out[d] = t.size(d);
}

// torch.cuda.<what>()
PyObject* cuda(const char* what)
{
    PyObject* m = PyImport_ImportModule("torch.cuda");
    PyObject* r = m ? PyObject_CallMethod(m, what, nullptr) : nullptr;
    Py_XDECREF(m);
    if (!r) throw Raised{};
    Py_DECREF(r);                    // (True, False, or an object that is not looked at)
    return r;
}

// The stream work is sent to: torch's current one, which sets up the device where nothing has; null where there is none.
void* stream()
{
    static bool ready = false;       // torch.cuda.is_initialized() does not go back
    if (!ready) {
        if (cuda("is_initialized") != Py_True) {
            if (cuda("is_available") != Py_True) return nullptr;
            cuda("current_stream");
        }
        ready = true;
    }
    return c10::hip::getCurrentHIPStream().stream();
}

// A sar.Blocks object.
struct Blocks {
    const sar_blocks_t* h;
    int P = 0;
    int64_t n_dst = 0;
    bool compact;
    explicit Blocks(PyObject* b)
    {
        static PyObject *const addr = PyUnicode_InternFromString("_addr"), *const flags = PyUnicode_InternFromString("flags");
        PyObject* a = PyObject_GetAttr(b, addr);
        if (!a) throw Raised{};
        if (a == Py_None) {
            Py_DECREF(a);
            raise_sar(SAR_ERR_STATE, "blocks handle already freed");
        }
        h = static_cast<const sar_blocks_t*>(PyLong_AsVoidPtr(a));
        Py_DECREF(a);
        if (PyErr_Occurred()) throw Raised{};
        PyObject* f = PyObject_GetAttr(b, flags);
        if (!f) throw Raised{};
        compact = (PyLong_AsLong(f) & SAR_BUILD_COMPACT) != 0;
        Py_DECREF(f);
        if (PyErr_Occurred()) throw Raised{};
        check(sar_blocks_info(h, &P, &n_dst));
    }
    sar_block_view view(int64_t q) const
    {
        sar_block_view v;
        check(sar_blocks_get(h, (int)q, &v));
        return v;
    }
    void rows(int64_t q, PyObject* o) const
    {
        if (o == Py_None) return;
        const int64_t n = view(q).n_src, has = tensor(o).size(0);
        if (has != n) refuse("block %lld has %lld sources, tensor has %lld rows", (long long)q, (long long)n, (long long)has);
    }
    void err_rows(int64_t q, PyObject* o) const
    {
        if (o == Py_None) return;
        const sar_block_view v = view(q);
        const int64_t n = compact ? v.n_t_rows : v.n_src, has = tensor(o).size(0);
        if (has != n) refuse("block %lld's error has %lld rows, tensor has %lld", (long long)q, (long long)n, (long long)has);
    }
    void dst(PyObject* o) const
    {
        if (o == Py_None) return;
        const int64_t has = tensor(o).size(0);
        if (has != n_dst) refuse("handle has %lld destinations, tensor has %lld rows", (long long)n_dst, (long long)has);
    }
};

// One tensor per block (or None): their addresses, for the calls that reinterpret the memory.
struct List {
    PyObject* items = nullptr;
    std::vector<void*> p;
    List() = default;
    List(const List&) = delete;
    ~List() { Py_XDECREF(items); }
    void open(PyObject* seq)
    {
        // by position: a set has no order, and an iterator is at its end after one look
        if (!PySequence_Check(seq) && !THPVariable_Check(seq)) {
            PyErr_Format(PyExc_TypeError, "expected one tensor per block, got %s", Py_TYPE(seq)->tp_name);
            throw Raised{};
        }
        items = PySequence_Fast(seq, "expected one tensor per block");
        if (!items) throw Raised{};
    }
    PyObject* at(int64_t q) const
    {
        if (q >= PySequence_Fast_GET_SIZE(items)) {
            PyErr_SetString(PyExc_IndexError, "list index out of range");
            throw Raised{};
        }
        return PySequence_Fast_GET_ITEM(items, q);
    }
    void take(const char* what, at::ScalarType dtype, int64_t row_values)
    {
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(items);
        p.assign(n, nullptr);
        for (Py_ssize_t k = 0; k < n; ++k) {
            PyObject* o = PySequence_Fast_GET_ITEM(items, k);
            if (o == Py_None) continue;
            const at::Tensor& t = tensor(o);
            if (!t.is_cuda() || !t.is_contiguous()) refuse("%s[%d] must be a contiguous device tensor", what, (int)k);
            if (t.scalar_type() != dtype)
                refuse("%s[%d] is %s, the call needs %s", what, (int)k, type_name(t.scalar_type()).c_str(),
                       type_name(dtype).c_str());
            if (t.numel() != t.size(0) * row_values)
                refuse("%s[%d] has %lld values per row, the call needs %lld", what, (int)k,
                       (long long)(t.numel() / std::max<int64_t>(t.size(0), 1)), (long long)row_values);
            p[k] = t.data_ptr();
        }
    }
    template <typename T>
    T* const* as() const
    {
        return items ? reinterpret_cast<T* const*>(p.data()) : nullptr;
    }
};

// ---- calls

// The entry point, without Python's lock, as ctypes makes a call.
template <typename F>
void call(F&& f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    check(rc);
}

template <int N, typename F>
PyObject* entry(PyObject* self, PyObject* const* a, Py_ssize_t n, F&& f)
{
    HANDLE_TH_ERRORS
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        f(a);
    } catch (const Raised&) {
        return nullptr;
    } catch (const Refused& r) {
        set_error(self, r);
        return nullptr;
    }
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}
#define SAR_CALL(name, n_args) \
    PyObject* name(PyObject* self, PyObject* const* args, Py_ssize_t n) { return entry<n_args>(self, args, n, [](PyObject* const* a) {
#define SAR_CALL_END }); }

// b, Zq, mean, out, residual, act
SAR_CALL(spmm_all, 6)
    const Blocks b(a[0]);
    List Z;
    Z.open(a[1]);
    for (int q = 0; q < b.P; ++q) b.rows(q, Z.at(q));
    b.dst(a[3]);
    const at::Tensor& out = tensor(a[3]);
    same_shape(out, a[4]);
    const int64_t F = out.size(-1);
    Z.take("Zq", out.scalar_type(), F);
    const int dt = dtype_code(out.scalar_type()), mean = truth(a[2]), act = (int)integer(a[5]);
    void *const r = ptr(a[4]), *const o = ptr_of(out), *const st = stream();
    call([&] { return sar_spmm_all(b.h, Z.as<const void>(), dt, (int)F, mean, r, act, o, st); });
SAR_CALL_END

// h, dH, act, G
SAR_CALL(act_bwd, 4)
    const at::Tensor& h = tensor(a[0]);
    same_shape(h, a[1]);
    same_shape(h, a[3]);
    void *const p = ptr_of(h), *const d = ptr(a[1]), *const g = ptr(a[3]), *const st = stream();
    const int dt = dtype_code(h.scalar_type()), act = (int)integer(a[2]);
    const int64_t count = h.numel();
    call([&] { return sar_act_bwd(p, d, act, g, dt, count, st); });
SAR_CALL_END

// b, G, mean, dZq
SAR_CALL(spmm_bwd_all, 4)
    const Blocks b(a[0]);
    List dZ;
    dZ.open(a[3]);
    for (int q = 0; q < b.P; ++q) b.err_rows(q, dZ.at(q));
    b.dst(a[1]);
    const at::Tensor& G = tensor(a[1]);
    const int64_t F = G.size(-1);
    dZ.take("dZq", G.scalar_type(), F);
    const int dt = dtype_code(G.scalar_type()), mean = truth(a[2]);
    void *const g = ptr_of(G), *const st = stream();
    call([&] { return sar_spmm_bwd_all(b.h, g, mean, dt, (int)F, dZ.as<void>(), st); });
SAR_CALL_END

// Eq, t_rank, accumulate, Ep
SAR_CALL(error_add, 4)
    const at::Tensor& Ep = tensor(a[3]);
    const int64_t rows = Ep.size(0), F = Ep.numel() / std::max<int64_t>(rows, 1);
    if (a[0] != Py_None) {
        const at::Tensor& Eq = tensor(a[0]);
        if (Eq.scalar_type() != Ep.scalar_type() || Eq.numel() != Eq.size(0) * F)
            refuse("Eq and Ep must have the same row width and type");
    }
    void *const e = ptr(a[0]), *const p = ptr_of(Ep), *const st = stream();
    const int32_t* const rank = address<const int32_t>(a[1]);
    const int acc = truth(a[2]), dt = dtype_code(Ep.scalar_type());
    call([&] { return sar_error_add(e, rank, acc, p, dt, rows, (int)F, st); });
SAR_CALL_END

// Z, a, score
SAR_CALL(gat_scores, 3)
    const at::Tensor& Z = tensor(a[0]);
    int64_t hd[2];
    unpack_sizes(tensor(a[1]), hd);
    void *const z = ptr_of(Z), *const st = stream();
    float *const v = ptr<float>(a[1]), *const s = ptr<float>(a[2]);
    const int dt = dtype_code(Z.scalar_type());
    const int64_t rows = Z.size(0);
    call([&] { return sar_gat_scores(z, dt, rows, (int)hd[0], (int)hd[1], v, s, st); });
SAR_CALL_END

// m, l, acc
SAR_CALL(gat_fwd_begin, 3)
    int64_t nhd[3];
    unpack_sizes(tensor(a[2]), nhd);
    float *const m = ptr<float>(a[0]), *const l = ptr<float>(a[1]), *const acc = ptr<float>(a[2]);
    void* const st = stream();
    call([&] { return sar_gat_fwd_begin(m, l, acc, nhd[0], (int)nhd[1], (int)nhd[2], st); });
SAR_CALL_END

// b, q, Zq, s, tq, a_l, slope, m, l, acc
SAR_CALL(gat_fwd_block, 10)
    const Blocks b(a[0]);
    const int64_t q = integer(a[1]);
    int64_t nhd[3];
    unpack_sizes(tensor(a[9]), nhd);
    b.rows(q, a[2]);
    b.rows(q, a[4]);
    for (int k : {3, 7, 8, 9}) b.dst(a[k]);
    void *const z = ptr(a[2]), *const st = stream();
    float *const s = ptr<float>(a[3]), *const t = ptr<float>(a[4]), *const al = ptr<float>(a[5]);
    float *const m = ptr<float>(a[7]), *const l = ptr<float>(a[8]), *const acc = ptr<float>(a[9]);
    const int dt = dtype_code(tensor(a[2]).scalar_type());
    const float slope = real(a[6]);
    call([&] { return sar_gat_fwd_block(b.h, (int)q, z, s, t, al, dt, (int)nhd[1], (int)nhd[2], slope, m, l, acc, st); });
SAR_CALL_END

// m, l, acc, out, L, act
SAR_CALL(gat_fwd_end, 6)
    int64_t nhd[3];
    unpack_sizes(tensor(a[2]), nhd);
    float *const m = ptr<float>(a[0]), *const l = ptr<float>(a[1]), *const acc = ptr<float>(a[2]), *const L = ptr<float>(a[4]);
    void *const out = ptr(a[3]), *const st = stream();
    const int act = (int)integer(a[5]), dt = dtype_code(tensor(a[3]).scalar_type());
    call([&] { return sar_gat_fwd_end(m, l, acc, act, out, L, dt, nhd[0], (int)nhd[1], (int)nhd[2], st); });
SAR_CALL_END

// b, Zq, s, tq, a_l, slope, out, L, act
SAR_CALL(gat_fwd_all, 9)
    const Blocks b(a[0]);
    const at::Tensor& out = tensor(a[6]);
    int64_t nhd[3];
    unpack_sizes(out, nhd);
    List Z, t;
    Z.open(a[1]);
    if (a[3] != Py_None) t.open(a[3]);
    for (int q = 0; q < b.P; ++q) {
        b.rows(q, Z.at(q));
        if (t.items) b.rows(q, t.at(q));
    }
    for (int k : {2, 6, 7}) b.dst(a[k]);
    Z.take("Zq", out.scalar_type(), nhd[1] * nhd[2]);
    if (t.items) t.take("tq", at::kFloat, nhd[1]);
    float *const s = ptr<float>(a[2]), *const al = ptr<float>(a[4]), *const L = ptr<float>(a[7]);
    void *const o = ptr_of(out), *const st = stream();
    const int dt = dtype_code(out.scalar_type()), act = (int)integer(a[8]);
    const float slope = real(a[5]);
    call([&] {
        return sar_gat_fwd_all(b.h, Z.as<const void>(), s, t.as<const float>(), al, dt, (int)nhd[1], (int)nhd[2], slope, act, o,
                               L, st);
    });
SAR_CALL_END

// G, out, s, L, rec, ds, act, Gact
SAR_CALL(gat_bwd_begin, 8)
    const at::Tensor& G = tensor(a[0]);
    int64_t nhd[3];
    unpack_sizes(G, nhd);
    same_shape(G, a[1]);
    same_shape(G, a[7]);
    void *const g = ptr_of(G), *const o = ptr(a[1]), *const ga = ptr(a[7]), *const st = stream();
    float *const s = ptr<float>(a[2]), *const L = ptr<float>(a[3]), *const rec = ptr<float>(a[4]), *const ds = ptr<float>(a[5]);
    const int act = (int)integer(a[6]), dt = dtype_code(G.scalar_type());
    call([&] { return sar_gat_bwd_begin(g, o, s, L, act, ga, dt, rec, ds, nhd[0], (int)nhd[1], (int)nhd[2], st); });
SAR_CALL_END

// b, q, Zq, G, tq, rec, a_l, slope, dZq, dtq, ds, da_l, work
SAR_CALL(gat_bwd_block, 13)
    const Blocks b(a[0]);
    const int64_t q = integer(a[1]);
    int64_t hd[2];
    unpack_sizes(tensor(a[6]), hd);
    b.rows(q, a[2]);
    b.rows(q, a[4]);
    b.err_rows(q, a[8]);
    b.err_rows(q, a[9]);
    for (int k : {3, 5, 10}) b.dst(a[k]);
    void *const z = ptr(a[2]), *const g = ptr(a[3]), *const dz = ptr(a[8]), *const work = ptr(a[12]), *const st = stream();
    float *const t = ptr<float>(a[4]), *const rec = ptr<float>(a[5]), *const al = ptr<float>(a[6]), *const dt_q = ptr<float>(a[9]);
    float *const ds = ptr<float>(a[10]), *const da = ptr<float>(a[11]);
    const int dt = dtype_code(tensor(a[3]).scalar_type());
    const float slope = real(a[7]);
    const size_t wb = bytes_of(a[12]);
    call([&] {
        return sar_gat_bwd_block(b.h, (int)q, z, g, t, rec, al, dt, (int)hd[0], (int)hd[1], slope, dz, dt_q, ds, da, work, wb, st);
    });
SAR_CALL_END

// b, Zq, G, tq, rec, a_l, slope, dZq, dtq, ds, da_l, work
SAR_CALL(gat_bwd_all, 12)
    const Blocks b(a[0]);
    int64_t hd[2];
    unpack_sizes(tensor(a[5]), hd);
    List Z, t, dZ, dt_q;
    Z.open(a[1]);
    if (a[3] != Py_None) t.open(a[3]);
    dZ.open(a[7]);
    if (a[8] != Py_None) dt_q.open(a[8]);
    for (int q = 0; q < b.P; ++q) {
        b.rows(q, Z.at(q));
        if (t.items) b.rows(q, t.at(q));
        b.err_rows(q, dZ.at(q));
        if (dt_q.items) b.err_rows(q, dt_q.at(q));
    }
    for (int k : {2, 4, 9}) b.dst(a[k]);
    const at::Tensor& G = tensor(a[2]);
    Z.take("Zq", G.scalar_type(), hd[0] * hd[1]);
    if (t.items) t.take("tq", at::kFloat, hd[0]);
    dZ.take("dZq", G.scalar_type(), hd[0] * hd[1]);
    if (dt_q.items) dt_q.take("dtq", at::kFloat, hd[0]);
    void *const g = ptr_of(G), *const work = ptr(a[11]), *const st = stream();
    float *const rec = ptr<float>(a[4]), *const al = ptr<float>(a[5]), *const ds = ptr<float>(a[9]), *const da = ptr<float>(a[10]);
    const int dt = dtype_code(G.scalar_type());
    const float slope = real(a[6]);
    const size_t wb = bytes_of(a[11]);
    call([&] {
        return sar_gat_bwd_all(b.h, Z.as<const void>(), g, t.as<const float>(), rec, al, dt, (int)hd[0], (int)hd[1], slope,
                               dZ.as<void>(), dt_q.as<float>(), ds, da, work, wb, st);
    });
SAR_CALL_END

// Zdst, ds, a_r, dZadd, dZdst, da_r, work, dZadd_rank
SAR_CALL(gat_bwd_end, 8)
    const at::Tensor& Z = tensor(a[0]);
    int64_t hd[2];
    unpack_sizes(tensor(a[2]), hd);
    void *const z = ptr_of(Z), *const add = ptr(a[3]), *const out = ptr(a[4]), *const work = ptr(a[6]), *const st = stream();
    float *const ds = ptr<float>(a[1]), *const ar = ptr<float>(a[2]), *const da = ptr<float>(a[5]);
    const int32_t* const rank = address<const int32_t>(a[7]);
    const int dt = dtype_code(Z.scalar_type());
    const int64_t rows = Z.size(0);
    const size_t wb = bytes_of(a[6]);
    call([&] {
        return sar_gat_bwd_end(z, ds, ar, add, rank, out, da, dt, rows, (int)hd[0], (int)hd[1], work, wb, st);
    });
SAR_CALL_END

// X, W, Z, a_score, score, a_score2, score2
SAR_CALL(linear_fwd, 7)
    const at::Tensor &X = tensor(a[0]), &W = tensor(a[1]);
    int64_t nk[2], hd[2] = {0, 0};
    unpack_sizes(X, nk);
    const int64_t F = W.size(1);
    if (a[3] != Py_None) unpack_sizes(tensor(a[3]), hd);
    void *const x = ptr_of(X), *const z = ptr(a[2]), *const st = stream();
    float* const w = ptr_of<float>(W);
    float *const a1 = ptr<float>(a[3]), *const s1 = ptr<float>(a[4]), *const a2 = ptr<float>(a[5]), *const s2 = ptr<float>(a[6]);
    const int dt = dtype_code(X.scalar_type());
    call([&] {
        return sar_linear_fwd(x, w, z, dt, nk[0], (int)nk[1], (int)F, (int)hd[0], (int)hd[1], a1, s1, a2, s2, st);
    });
SAR_CALL_END

int64_t inner(PyObject* X, PyObject* W) { return X != Py_None ? tensor(X).size(1) : tensor(W).size(0); }

// X, dZ, W, dW, dX, work
SAR_CALL(linear_bwd, 6)
    const at::Tensor& dZ = tensor(a[1]);
    const int64_t rows = dZ.size(0), F = dZ.numel() / std::max<int64_t>(rows, 1), K = inner(a[0], a[2]);
    void *const x = ptr(a[0]), *const dz = ptr_of(dZ), *const dx = ptr(a[4]), *const work = ptr(a[5]), *const st = stream();
    float *const w = ptr<float>(a[2]), *const dw = ptr<float>(a[3]);
    const int dt = dtype_code(dZ.scalar_type());
    const size_t wb = bytes_if(a[5]);
    call([&] { return sar_linear_bwd(x, dz, w, dw, dx, dt, rows, (int)K, (int)F, work, wb, st); });
SAR_CALL_END

// X, E, E_rank, ds, a_r, H, D, W, dW, dX, n, dtype code, work, rows
SAR_CALL(linear_bwd_rows, 14)
    const int64_t K = inner(a[0], a[7]), n_E = a[1] == Py_None ? 0 : tensor(a[1]).size(0), n_rows = integer(a[10]);
    void *const x = ptr(a[0]), *const e = ptr(a[1]), *const dx = ptr(a[9]), *const rows = ptr(a[13]), *const work = ptr(a[12]);
    const int32_t* const rank = address<const int32_t>(a[2]);
    float *const ds = ptr<float>(a[3]), *const ar = ptr<float>(a[4]), *const w = ptr<float>(a[7]), *const dw = ptr<float>(a[8]);
    const int H = (int)integer(a[5]), D = (int)integer(a[6]), dt = (int)integer(a[11]);
    void* const st = stream();
    const size_t wb = bytes_if(a[12]);
    call([&] {
        return sar_linear_bwd_rows(x, e, rank, n_E, ds, ar, H, D, w, dw, dx, dt, n_rows, (int)K, rows, work, wb, st);
    });
SAR_CALL_END

// ---- the node-wise operators.  Every tensor has the shape and type that the call states, and lies on the current device, whose
// stream the work is sent to.

const at::Tensor& given(PyObject* o, const char* what, at::ScalarType dtype, std::initializer_list<int64_t> shape)
{
    const at::Tensor& t = tensor(o);
    if (t.scalar_type() != dtype) refuse("%s is %s, the call needs %s", what, type_name(t.scalar_type()).c_str(), type_name(dtype).c_str());
    if (t.sizes() != at::IntArrayRef(shape)) {
        std::string s;
        for (int64_t d : shape) s += (s.empty() ? "" : ", ") + std::to_string(d);
        refuse("%s has shape %s, the call needs (%s)", what, shape_text(t).c_str(), s.c_str());
    }
    if (!t.is_contiguous()) refuse("%s must be contiguous", what);
    return t;
}

template <typename T = void>
T* at_of(PyObject* o, const char* what, at::ScalarType dtype, std::initializer_list<int64_t> shape)
{
    return static_cast<T*>(given(o, what, dtype, shape).data_ptr());
}

template <typename T = void>
T* at_if(PyObject* o, const char* what, at::ScalarType dtype, std::initializer_list<int64_t> shape)
{
    return o == Py_None ? nullptr : at_of<T>(o, what, dtype, shape);
}

// (the library takes widths and numbers of types as int)
int64_t within_int(int64_t v)
{
    if (v > std::numeric_limits<int>::max())
        raise_sar(SAR_ERR_UNSUPPORTED, ("a size of " + std::to_string(v) + " is more than the call takes").c_str());
    return v;
}

// The first of a call's tensors, which says how many rows and columns there are, and of which type.
struct Rows {
    at::ScalarType dtype;
    int code;
    int64_t n, width;
    void* p;
};
Rows rows_of(PyObject* o, const char* what)
{
    const at::Tensor& t = tensor(o);
    const int code = dtype_code(t.scalar_type());
    int64_t s[2];
    unpack_sizes(t, s);
    return {t.scalar_type(), code, s[0], within_int(s[1]), at_of(o, what, t.scalar_type(), {s[0], s[1]})};
}

// Rows in 8 bits: a pair (q, e), or None.
struct Packed {
    int8_t* q = nullptr;
    uint8_t* e = nullptr;
};
bool is_pair(PyObject* o) { return PyTuple_Check(o) || PyList_Check(o); }
Packed packed(PyObject* o, const char* what, int64_t n, int64_t K)
{
    if (o == Py_None) return {};
    if (!is_pair(o) || PySequence_Fast_GET_SIZE(o) != 2) refuse("%s: packed rows are a pair (q, e)", what);
    PyObject* const* const items = PySequence_Fast_ITEMS(o);
    return {at_of<int8_t>(items[0], what, at::kChar, {n, (K + 15) / 16 * 16}), at_of<uint8_t>(items[1], what, at::kByte, {n, (K + 31) / 32})};
}

// Scratch: any type, any shape, or None.
void* scratch(PyObject* o)
{
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o);
    if (!t.is_contiguous()) refuse("work must be contiguous");
    return t.data_ptr();
}

// The last check: whatever tensors a call's arguments are or hold lie on the current device.
void all_here(PyObject* const* a, int n)
{
    for (int k = 0; k < n; ++k) {
        if (is_pair(a[k])) {
            all_here(PySequence_Fast_ITEMS(a[k]), (int)PySequence_Fast_GET_SIZE(a[k]));
        } else if (THPVariable_Check(a[k])) {
            const at::Tensor& t = THPVariable_Unpack(a[k]);
            if (!t.is_cuda()) refuse("the call takes device tensors, and one of shape %s is in host memory", shape_text(t).c_str());
            if (t.get_device() != c10::hip::current_device())
                refuse("a tensor of shape %s is on device %d, the current one is %d", shape_text(t).c_str(), (int)t.get_device(),
                       (int)c10::hip::current_device());
        }
    }
}

// X, (q, e)
SAR_CALL(pack, 2)
    const Rows X = rows_of(a[0], "X");
    if (a[1] == Py_None) refuse("packed rows are a pair (q, e)");
    const Packed p = packed(a[1], "packed rows", X.n, X.width);
    void* const st = stream();
    all_here(a, 2);
    call([&] { return sar_pack(X.p, X.code, X.n, (int)X.width, p.q, p.e, st); });
SAR_CALL_END

// (q, e), X
SAR_CALL(unpack, 2)
    const Rows X = rows_of(a[1], "X");
    if (a[0] == Py_None) refuse("packed rows are a pair (q, e)");
    const Packed p = packed(a[0], "packed rows", X.n, X.width);
    void* const st = stream();
    all_here(a, 2);
    call([&] { return sar_unpack(p.q, p.e, X.code, X.n, (int)X.width, X.p, st); });
SAR_CALL_END

// X, gamma, beta, eps, Y, stats, X's (q, e), Y's (q, e)
SAR_CALL(layernorm_fwd, 8)
    const Rows X = rows_of(a[0], "X");
    const int64_t D = X.width;
    float *const gamma = at_if<float>(a[1], "gamma", at::kFloat, {D}), *const beta = at_if<float>(a[2], "beta", at::kFloat, {D});
    const float eps = real(a[3]);
    void* const Y = at_of(a[4], "Y", X.dtype, {X.n, D});
    float* const stats = at_if<float>(a[5], "stats", at::kFloat, {X.n, 2});
    const Packed xp = packed(a[6], "Xp", X.n, D), yp = packed(a[7], "Yp", X.n, D);
    void* const st = stream();
    all_here(a, 8);
    call([&] { return sar_layernorm_fwd(X.p, gamma, beta, eps, Y, stats, X.code, X.n, (int)D, xp.q, xp.e, yp.q, yp.e, st); });
SAR_CALL_END

// dY, X or its (q, e), stats, gamma, accumulate, dX, dgamma, dbeta, work
SAR_CALL(layernorm_bwd, 9)
    const Rows dY = rows_of(a[0], "dY");
    const int64_t n = dY.n, D = dY.width;
    const bool p = is_pair(a[1]);
    void* const X = p ? nullptr : at_of(a[1], "X", dY.dtype, {n, D});
    const Packed xp = p ? packed(a[1], "X", n, D) : Packed{};
    float *const stats = at_of<float>(a[2], "stats", at::kFloat, {n, 2}), *const gamma = at_if<float>(a[3], "gamma", at::kFloat, {D});
    const int acc = truth(a[4]);
    void *const dX = at_if(a[5], "dX", dY.dtype, {n, D}), *const work = scratch(a[8]), *const st = stream();
    float *const dg = at_if<float>(a[6], "dgamma", at::kFloat, {D}), *const db = at_if<float>(a[7], "dbeta", at::kFloat, {D});
    const size_t wb = bytes_if(a[8]);
    all_here(a, 9);
    call([&] { return sar_layernorm_bwd(dY.p, X, xp.q, xp.e, stats, gamma, acc, dX, dg, db, dY.code, n, (int)D, work, wb, st); });
SAR_CALL_END

// The weights of T types, and where each type's rows begin.
struct TypedW {
    int64_t T, K, F;
    float* W;
    int32_t* ptr;
};
TypedW typed_w(PyObject* W, PyObject* ptr, int64_t K, int64_t F)
{
    int64_t s[3];
    unpack_sizes(tensor(W), s);
    if (K < 0) K = s[1];
    if (F < 0) F = s[2];
    return {within_int(s[0]), within_int(K), within_int(F), at_of<float>(W, "W", at::kFloat, {s[0], K, F}), at_of<int32_t>(ptr, "type_ptr", at::kInt, {s[0] + 1})};
}

// X, W, type_ptr, Z, work
SAR_CALL(linear_typed_fwd, 5)
    const Rows X = rows_of(a[0], "X");
    const TypedW w = typed_w(a[1], a[2], X.width, -1);
    void *const Z = at_of(a[3], "Z", X.dtype, {X.n, w.F}), *const work = scratch(a[4]), *const st = stream();
    const size_t wb = bytes_if(a[4]);
    all_here(a, 5);
    call([&] { return sar_linear_typed_fwd(X.p, w.W, w.ptr, (int)w.T, Z, X.code, X.n, (int)w.K, (int)w.F, work, wb, st); });
SAR_CALL_END

// X or its (q, e) or None, dZ, W, type_ptr, accumulate, dW, dX, work
SAR_CALL(linear_typed_bwd, 8)
    const Rows dZ = rows_of(a[1], "dZ");
    const TypedW w = typed_w(a[2], a[3], -1, dZ.width);
    const bool p = is_pair(a[0]);
    void* const X = p ? nullptr : at_if(a[0], "X", dZ.dtype, {dZ.n, w.K});
    const Packed xp = p ? packed(a[0], "X", dZ.n, w.K) : Packed{};
    const int acc = truth(a[4]);
    float* const dW = at_if<float>(a[5], "dW", at::kFloat, {w.T, w.K, w.F});
    void *const dX = at_if(a[6], "dX", dZ.dtype, {dZ.n, w.K}), *const work = scratch(a[7]), *const st = stream();
    const size_t wb = bytes_if(a[7]);
    all_here(a, 8);
    call([&] {
        return sar_linear_typed_bwd(X, xp.q, xp.e, dZ.p, w.W, w.ptr, (int)w.T, acc, dW, dX, dZ.code, dZ.n, (int)w.K, (int)w.F, work, wb, st);
    });
SAR_CALL_END

// (q, e) or None, dZ, W, accumulate, dW, dX, work
SAR_CALL(linear_bwd_packed, 7)
    const Rows dZ = rows_of(a[1], "dZ");
    int64_t kf[2];
    unpack_sizes(tensor(a[2]), kf);
    const int64_t K = within_int(kf[0]), F = dZ.width;
    float* const W = at_of<float>(a[2], "W", at::kFloat, {K, F});
    const Packed xp = packed(a[0], "X", dZ.n, K);
    const int acc = truth(a[3]);
    float* const dW = at_if<float>(a[4], "dW", at::kFloat, {K, F});
    void *const dX = at_if(a[5], "dX", dZ.dtype, {dZ.n, K}), *const work = scratch(a[6]), *const st = stream();
    const size_t wb = bytes_if(a[6]);
    all_here(a, 7);
    call([&] { return sar_linear_bwd_packed(xp.q, xp.e, dZ.p, W, acc, dW, dX, dZ.code, dZ.n, (int)K, (int)F, work, wb, st); });
SAR_CALL_END

// W [K, F]; what is not known of it otherwise (-1) it says itself.
struct PlainW {
    int64_t K, F;
    float* W;
};
PlainW plain_w(PyObject* W, int64_t K, int64_t F)
{
    int64_t s[2];
    unpack_sizes(tensor(W), s);
    if (K < 0) K = s[0];
    if (F < 0) F = s[1];
    return {within_int(K), within_int(F), at_of<float>(W, "W", at::kFloat, {K, F})};
}

// (an enumeration's number)
int whole(PyObject* o)
{
    const int64_t v = integer(o);
    if (v < std::numeric_limits<int>::min() || v > std::numeric_limits<int>::max())
        raise_sar(SAR_ERR_UNSUPPORTED, ("a number of " + std::to_string(v) + " is more than the call takes").c_str());
    return (int)v;
}

// X, W, bias, res, act, res_after, Y, A, work
SAR_CALL(linear_act_fwd, 9)
    const Rows X = rows_of(a[0], "X");
    const PlainW w = plain_w(a[1], X.width, -1);
    float* const bias = at_if<float>(a[2], "bias", at::kFloat, {w.F});
    void* const res = at_if(a[3], "res", X.dtype, {X.n, w.F});
    const int act = whole(a[4]), after = truth(a[5]);
    void *const Y = at_of(a[6], "Y", X.dtype, {X.n, w.F}), *const A = at_if(a[7], "A", X.dtype, {X.n, w.F});
    void *const work = scratch(a[8]), *const st = stream();
    const size_t wb = bytes_if(a[8]);
    all_here(a, 9);
    call([&] { return sar_linear_act_fwd(X.p, w.W, bias, res, act, after, Y, A, X.code, X.n, (int)w.K, (int)w.F, work, wb, st); });
SAR_CALL_END

// dY, A, X or None, W, act, accumulate, dW, db, dX, dA, work
SAR_CALL(linear_act_bwd, 11)
    const Rows dY = rows_of(a[0], "dY");
    const PlainW w = plain_w(a[3], -1, dY.width);
    void *const A = at_if(a[1], "A", dY.dtype, {dY.n, w.F}), *const X = at_if(a[2], "X", dY.dtype, {dY.n, w.K});
    const int act = whole(a[4]), acc = truth(a[5]);
    float *const dW = at_if<float>(a[6], "dW", at::kFloat, {w.K, w.F}), *const db = at_if<float>(a[7], "db", at::kFloat, {w.F});
    void *const dX = at_if(a[8], "dX", dY.dtype, {dY.n, w.K}), *const dA = at_if(a[9], "dA", dY.dtype, {dY.n, w.F});
    void *const work = scratch(a[10]), *const st = stream();
    const size_t wb = bytes_if(a[10]);
    all_here(a, 11);
    call([&] { return sar_linear_act_bwd(dY.p, A, X, w.W, act, acc, dW, db, dX, dA, dY.code, dY.n, (int)w.K, (int)w.F, work, wb, st); });
SAR_CALL_END

// Top classes: a pair (values [n, k], classes [n, k]), or None.
struct Top {
    int k = 0;
    float* value = nullptr;
    int32_t* index = nullptr;
};
Top top_of(PyObject* o, int64_t n)
{
    if (o == Py_None) return {};
    if (!is_pair(o) || PySequence_Fast_GET_SIZE(o) != 2) refuse("top classes are a pair (values, classes)");
    PyObject* const* const items = PySequence_Fast_ITEMS(o);
    int64_t s[2];
    unpack_sizes(tensor(items[0]), s);
    return {(int)within_int(s[1]), at_of<float>(items[0], "top values", at::kFloat, {n, s[1]}), at_of<int32_t>(items[1], "top classes", at::kInt, {n, s[1]})};
}

// X, label, logp, lse, entropy, (values, classes), work
SAR_CALL(logprob_fwd, 7)
    const Rows X = rows_of(a[0], "X");
    int32_t* const label = at_if<int32_t>(a[1], "label", at::kInt, {X.n});
    float *const logp = at_if<float>(a[2], "logp", at::kFloat, {X.n}), *const lse = at_if<float>(a[3], "lse", at::kFloat, {X.n});
    float* const entropy = at_if<float>(a[4], "entropy", at::kFloat, {X.n});
    const Top top = top_of(a[5], X.n);
    void *const work = scratch(a[6]), *const st = stream();
    const size_t wb = bytes_if(a[6]);
    all_here(a, 7);
    call([&] { return sar_logprob_fwd(X.p, label, logp, lse, entropy, top.k, top.value, top.index, X.code, X.n, (int)X.width, work, wb, st); });
SAR_CALL_END

// X, label, lse, entropy, dlogp, dentropy, dX
SAR_CALL(logprob_bwd, 7)
    const Rows X = rows_of(a[0], "X");
    int32_t* const label = at_if<int32_t>(a[1], "label", at::kInt, {X.n});
    float *const lse = at_of<float>(a[2], "lse", at::kFloat, {X.n}), *const entropy = at_if<float>(a[3], "entropy", at::kFloat, {X.n});
    float *const dlogp = at_if<float>(a[4], "dlogp", at::kFloat, {X.n}), *const dentropy = at_if<float>(a[5], "dentropy", at::kFloat, {X.n});
    void *const dX = at_of(a[6], "dX", X.dtype, {X.n, X.width}), *const st = stream();
    all_here(a, 7);
    call([&] { return sar_logprob_bwd(X.p, label, lse, entropy, dlogp, dentropy, dX, X.code, X.n, (int)X.width, st); });
SAR_CALL_END

// X, (values, classes), temperature, loss, lse, work
SAR_CALL(distill_fwd, 6)
    const Rows X = rows_of(a[0], "X");
    if (a[1] == Py_None) refuse("top classes are a pair (values, classes)");
    const Top top = top_of(a[1], X.n);
    const float temperature = real(a[2]);
    float *const loss = at_if<float>(a[3], "loss", at::kFloat, {X.n}), *const lse = at_if<float>(a[4], "lse", at::kFloat, {X.n});
    void *const work = scratch(a[5]), *const st = stream();
    const size_t wb = bytes_if(a[5]);
    all_here(a, 6);
    call([&] { return sar_distill_fwd(X.p, top.k, top.value, top.index, temperature, loss, lse, X.code, X.n, (int)X.width, work, wb, st); });
SAR_CALL_END

// X, (values, classes), temperature, lse, dloss, dX
SAR_CALL(distill_bwd, 6)
    const Rows X = rows_of(a[0], "X");
    if (a[1] == Py_None) refuse("top classes are a pair (values, classes)");
    const Top top = top_of(a[1], X.n);
    const float temperature = real(a[2]);
    float *const lse = at_of<float>(a[3], "lse", at::kFloat, {X.n}), *const dloss = at_of<float>(a[4], "dloss", at::kFloat, {X.n});
    void *const dX = at_of(a[5], "dX", X.dtype, {X.n, X.width}), *const st = stream();
    all_here(a, 6);
    call([&] { return sar_distill_bwd(X.p, top.k, top.value, top.index, temperature, lse, dloss, dX, X.code, X.n, (int)X.width, st); });
SAR_CALL_END

#define SAR_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    SAR_METHOD(spmm_all), SAR_METHOD(act_bwd), SAR_METHOD(spmm_bwd_all), SAR_METHOD(error_add), SAR_METHOD(gat_scores),
    SAR_METHOD(gat_fwd_begin), SAR_METHOD(gat_fwd_block), SAR_METHOD(gat_fwd_end), SAR_METHOD(gat_fwd_all),
    SAR_METHOD(gat_bwd_begin), SAR_METHOD(gat_bwd_block), SAR_METHOD(gat_bwd_all), SAR_METHOD(gat_bwd_end),
    SAR_METHOD(linear_fwd), SAR_METHOD(linear_bwd), SAR_METHOD(linear_bwd_rows), SAR_METHOD(pack), SAR_METHOD(unpack),
    SAR_METHOD(layernorm_fwd), SAR_METHOD(layernorm_bwd), SAR_METHOD(linear_typed_fwd), SAR_METHOD(linear_typed_bwd),
    SAR_METHOD(linear_bwd_packed), SAR_METHOD(linear_act_fwd), SAR_METHOD(linear_act_bwd), SAR_METHOD(logprob_fwd), SAR_METHOD(logprob_bwd),
    SAR_METHOD(distill_fwd), SAR_METHOD(distill_bwd), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding()
{
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", SAR_BUILT_FOR) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
