// Argument marshalling of the token-step calls (tc_step_tables, tc_rope_append, tc_digest_blocks, tc_select_blocks,
// tc_block_attn): tensors are checked - type, device, shape, contiguity, for the device arrays' lengths are taken from one
// another - and handed over as addresses.  Through ctypes and the tensors' Python attributes this took 7 to 13 us per call, as much
// as the kernels; here it takes under 1 us.  Nothing is kept from one call for the next.
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <string>
#include <tuple>

namespace {

PyObject *g_error;                      // callable: (status, text) -> exception
PyObject *s_cuda_stream;

constexpr int kInvalid = -1;

// An argument that is not what the call takes.
struct Refused { std::string text; };
// A Python error is set.
struct Raised {};

long long integer(PyObject *x)
{
    const long long v = PyLong_AsLongLong(x);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}

double real(PyObject *x)
{
    const double v = PyFloat_AsDouble(x);
    if (v == -1.0 && PyErr_Occurred()) throw Raised{};
    return v;
}

void *address(PyObject *x)
{
    if (x == Py_None) return nullptr;
    void *p = PyLong_AsVoidPtr(x);
    if (!p && PyErr_Occurred()) throw Raised{};
    return p;
}

void *stream_of(PyObject *s)
{
    if (s == Py_None || PyLong_Check(s)) return address(s);
    PyObject *a = PyObject_GetAttr(s, s_cuda_stream);
    if (!a) throw Raised{};
    void *p = PyLong_AsVoidPtr(a);
    Py_DECREF(a);
    if (!p && PyErr_Occurred()) throw Raised{};
    return p;
}

const at::Tensor &tensor(PyObject *x, const char *name)
{
    if (!THPVariable_Check(x)) throw Refused{std::string(name) + " is no tensor"};
    return THPVariable_Unpack(x);
}

// The length of a dimension of a tensor with so many of them (what else it has to be is checked where it is handed over).
int64_t length(PyObject *x, const char *name, int64_t dims, int64_t dim)
{
    const at::Tensor &t = tensor(x, name);
    if (t.dim() != dims) throw Refused{std::string(name) + ": expected " + std::to_string(dims) + " dimensions, got " + std::to_string(t.dim())};
    return t.size(dim);
}

int32_t narrow(int64_t n, const char *name)
{
    if (n < INT32_MIN || n > INT32_MAX) throw Refused{std::string(name) + " is out of range"};
    return (int32_t)n;
}

// What a context is made of: (address, Hq, Hkv, D, bf16, digest bytes, device), and the arguments of its calls.
struct Ctx {
    void *address;
    int64_t hq, hkv, d;
    at::ScalarType type;
    int64_t digest_bytes, device;
    explicit Ctx(PyObject *t)
    {
        if (!PyTuple_Check(t) || PyTuple_GET_SIZE(t) != 7) throw Refused{"bad context"};
        address = ::address(PyTuple_GET_ITEM(t, 0));
        hq = integer(PyTuple_GET_ITEM(t, 1));
        hkv = integer(PyTuple_GET_ITEM(t, 2));
        d = integer(PyTuple_GET_ITEM(t, 3));
        type = integer(PyTuple_GET_ITEM(t, 4)) ? at::kBFloat16 : at::kFloat;
        digest_bytes = integer(PyTuple_GET_ITEM(t, 5));
        device = integer(PyTuple_GET_ITEM(t, 6));
    }

    [[noreturn]] void refuse(const at::Tensor &t, const char *name, at::ScalarType type, at::IntArrayRef shape) const
    {
        std::string s = std::string(name) + ": expected a contiguous tensor " + c10::toString(type) + " [";
        for (const int64_t n : shape) s += " " + std::to_string(n);
        s += " ] on device " + std::to_string(device) + ", got " + std::string(c10::toString(t.scalar_type())) + " [";
        for (const int64_t n : t.sizes()) s += " " + std::to_string(n);
        throw Refused{s + (t.is_cuda() ? " ] on device " + std::to_string((int)t.get_device()) : " ] in host memory")};
    }

    bool holds(const at::Tensor &t, at::ScalarType type) const { return t.scalar_type() == type && t.is_cuda() && t.get_device() == device; }

    // A contiguous tensor of this type and shape on the context's device.
    void *array(PyObject *x, const char *name, at::ScalarType type, at::IntArrayRef shape) const
    {
        const at::Tensor &t = tensor(x, name);
        if (!holds(t, type) || t.sizes() != shape || !t.is_contiguous()) refuse(t, name, type, shape);
        return t.data_ptr();
    }

    // One of any shape.
    void *any_shape(PyObject *x, const char *name, at::ScalarType type, int64_t &numel) const
    {
        const at::Tensor &t = tensor(x, name);
        if (!holds(t, type) || !t.is_contiguous()) refuse(t, name, type, t.sizes());
        numel = t.numel();
        return t.data_ptr();
    }

    // Rows [n][heads][D] that may stand apart.
    void *rows(PyObject *x, const char *name, int64_t n, int64_t heads, int64_t &stride) const
    {
        const at::Tensor &t = tensor(x, name);
        const int64_t shape[3] = {n, heads, d};
        if (!holds(t, type) || t.sizes() != at::IntArrayRef(shape, 3) ||
            (t.numel() > 0 && ((d > 1 && t.stride(2) != 1) || (heads > 1 && t.stride(1) != d))))
            refuse(t, name, type, at::IntArrayRef(shape, 3));
        stride = n > 1 ? t.stride(0) : heads * d;
        return t.data_ptr();
    }
};

constexpr at::ScalarType kI32 = at::kInt, kI64 = at::kLong;

// The call itself, other Python threads running meanwhile (a launch waits where the queue is full).
template <typename R, typename... P, typename... A>
R call(R (*fn)(P...), const std::tuple<A...> &args)
{
    struct Unlocked {
        PyThreadState *state = PyEval_SaveThread();
        ~Unlocked() { PyEval_RestoreThread(state); }
    } unlocked;
    return std::apply(fn, args);
}

template <typename F, F kBody, int kArgs>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != kArgs) { PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", kArgs, n); return nullptr; }
    try {
        return PyLong_FromLong(kBody(args));
    } catch (const Raised &) {
    } catch (const Refused &r) {
        PyObject *e = g_error ? PyObject_CallFunction(g_error, "is", kInvalid, r.text.c_str()) : nullptr;
        if (e) { PyErr_SetObject((PyObject *)Py_TYPE(e), e); Py_DECREF(e); }
        else if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, r.text.c_str());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// fn, ctx, seq_len, new_len, block_table, spare, spare_used, spare_next, end_len, cu_new, slot_map, token_pos, token_seq,
// full_block, status, stream
int32_t step_tables(PyObject *const *a)
{
    typedef int32_t (*fn_t)(void *, const void *, const void *, int32_t, void *, int32_t, const void *, int32_t, const void *, void *, void *, void *,
                            void *, void *, void *, void *, int32_t, void *, void *);
    const Ctx c(a[1]);
    const int64_t B = length(a[4], "block_table", 2, 0), mb = length(a[4], "block_table", 2, 1), ns = length(a[5], "spare", 1, 0),
                  n = length(a[10], "slot_map", 1, 0);
    return call((fn_t)address(a[0]), std::make_tuple(
        c.address, c.array(a[2], "seq_len", kI32, {B}), c.array(a[3], "new_len", kI32, {B}), narrow(B, "B"), c.array(a[4], "block_table", kI32, {B, mb}),
        narrow(mb, "max_blocks"), c.array(a[5], "spare", kI32, {ns}), narrow(ns, "spare"), c.array(a[6], "spare_used", kI32, {1}),
        c.array(a[7], "spare_next", kI32, {1}), c.array(a[8], "end_len", kI32, {B}), c.array(a[9], "cu_new", kI32, {B + 1}),
        c.array(a[10], "slot_map", kI64, {n}), c.array(a[11], "token_pos", kI32, {n}), c.array(a[12], "token_seq", kI32, {n}),
        c.array(a[13], "full_block", kI32, {n}), narrow(n, "n_tokens"), c.array(a[14], "status", kI32, {2}), stream_of(a[15])));
}

// fn, ctx, layer, q, k, v, pos, sections (address or None), number of sections, rope_theta, slot_map, q_out, stream
int32_t rope_append(PyObject *const *a)
{
    typedef int32_t (*fn_t)(void *, int32_t, const void *, int64_t, const void *, int64_t, const void *, int64_t, const void *, int32_t, const void *,
                            double, const void *, int32_t, void *, void *);
    const Ctx c(a[1]);
    const int64_t n = length(a[10], "slot_map", 1, 0);
    const bool one = tensor(a[6], "pos").dim() == 1;
    const int64_t axes = one ? 1 : length(a[6], "pos", 2, 0);
    void *sections = address(a[7]);
    if (sections && integer(a[8]) != axes) throw Refused{"sections for another number of axes"};
    int64_t qs, ks, vs;
    void *q = c.rows(a[3], "q", n, c.hq, qs), *k = c.rows(a[4], "k", n, c.hkv, ks), *v = c.rows(a[5], "v", n, c.hkv, vs);
    void *pos = one ? c.array(a[6], "pos", kI32, {n}) : c.array(a[6], "pos", kI32, {axes, n});
    return call((fn_t)address(a[0]), std::make_tuple(c.address, narrow(integer(a[2]), "layer"), q, qs, k, ks, v, vs, pos, narrow(axes, "axes"), sections, real(a[9]),
                                 c.array(a[10], "slot_map", kI64, {n}), narrow(n, "n_tokens"), c.array(a[11], "q_out", c.type, {n, c.hq, c.d}), stream_of(a[12])));
}

// fn, ctx, l0, l1, entries, digests, stream
int32_t digest_blocks(PyObject *const *a)
{
    typedef int32_t (*fn_t)(void *, int32_t, int32_t, const void *, int32_t, void *, void *);
    const Ctx c(a[1]);
    int64_t n;
    void *entries = c.any_shape(a[4], "entries", kI32, n);
    return call((fn_t)address(a[0]), std::make_tuple(c.address, narrow(integer(a[2]), "l0"), narrow(integer(a[3]), "l1"), entries, narrow(n, "entries"),
                                 c.array(a[5], "digests", at::kChar, {c.digest_bytes}), stream_of(a[6])));
}

// fn, ctx, layer, q, token_seq, token_pos, block_table, digests, n_sink, n_top, n_local, lists, workspace, stream
int32_t select_blocks(PyObject *const *a)
{
    typedef int32_t (*fn_t)(void *, int32_t, const void *, const void *, const void *, int32_t, const void *, int32_t, int32_t, const void *, int32_t,
                            int32_t, int32_t, void *, void *, size_t, void *);
    const Ctx c(a[1]);
    const int64_t n = length(a[4], "token_seq", 1, 0), B = length(a[6], "block_table", 2, 0), mb = length(a[6], "block_table", 2, 1);
    const int32_t sink = narrow(integer(a[8]), "n_sink"), top = narrow(integer(a[9]), "n_top"), local = narrow(integer(a[10]), "n_local");
    int64_t bytes;
    void *ws = c.any_shape(a[12], "workspace", at::kByte, bytes);
    return call((fn_t)address(a[0]), std::make_tuple(
        c.address, narrow(integer(a[2]), "layer"), c.array(a[3], "q", c.type, {n, c.hq, c.d}), c.array(a[4], "token_seq", kI32, {n}),
        c.array(a[5], "token_pos", kI32, {n}), narrow(n, "n_tokens"), c.array(a[6], "block_table", kI32, {B, mb}), narrow(B, "B"), narrow(mb, "max_blocks"),
        c.array(a[7], "digests", at::kChar, {c.digest_bytes}), sink, top, local,
        c.array(a[11], "lists", kI32, {n, c.hkv, (int64_t)sink + top + local}), ws, (size_t)bytes, stream_of(a[13])));
}

// fn, ctx, layer, q, token_seq, token_pos, block_table, lists, out, sm_scale, workspace, stream
int32_t block_attn(PyObject *const *a)
{
    typedef int32_t (*fn_t)(void *, int32_t, const void *, const void *, const void *, int32_t, const void *, int32_t, int32_t, const void *, int32_t,
                            void *, float, void *, size_t, void *);
    const Ctx c(a[1]);
    const int64_t n = length(a[4], "token_seq", 1, 0), B = length(a[6], "block_table", 2, 0), mb = length(a[6], "block_table", 2, 1),
                  nl = length(a[7], "lists", 3, 2);
    int64_t bytes;
    void *ws = c.any_shape(a[10], "workspace", at::kByte, bytes);
    return call((fn_t)address(a[0]), std::make_tuple(
        c.address, narrow(integer(a[2]), "layer"), c.array(a[3], "q", c.type, {n, c.hq, c.d}), c.array(a[4], "token_seq", kI32, {n}),
        c.array(a[5], "token_pos", kI32, {n}), narrow(n, "n_tokens"), c.array(a[6], "block_table", kI32, {B, mb}), narrow(B, "B"), narrow(mb, "max_blocks"),
        c.array(a[7], "lists", kI32, {n, c.hkv, nl}), narrow(nl, "lists"), c.array(a[8], "out", c.type, {n, c.hq, c.d}), (float)real(a[9]), ws,
        (size_t)bytes, stream_of(a[11])));
}

PyObject *set_error(PyObject *, PyObject *f)
{
    Py_INCREF(f);
    Py_XSETREF(g_error, f);
    Py_RETURN_NONE;
}

#define METHOD(name, args) {#name, (PyCFunction)(void (*)(void))guarded<decltype(&name), &name, args>, METH_FASTCALL, "marshal one tc_" #name " call"}

PyMethodDef methods[] = {METHOD(step_tables, 16), METHOD(rope_append, 13), METHOD(digest_blocks, 7), METHOD(select_blocks, 14), METHOD(block_attn, 12),
                         {"set_error", set_error, METH_O, "callable that makes the exception of a refused argument from (status, text)"},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_py_step", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__py_step(void)
{
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    return PyModule_Create(&module);
}
