// torch_args.cpp -- checks the tensors of the language model operators and
// writes their addresses, sizes and strides into the structs of libscan.h.
//
// A single token's step takes its kernel a few microseconds, and checking a
// dozen tensors in Python took longer than that (15 us a call of
// selective_scan_step with one row, of which the kernel has 4).  Host code
// only: what is computed is computed by libscan.so, which is called by the
// binding with what is returned here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <sstream>

#include "../../include/libscan.h"

namespace {

struct Raised {};  // a Python error is set

template <class... A>
[[noreturn]] void raise(PyObject* type, const A&... parts) {
    std::ostringstream s;
    (s << ... << parts);
    PyErr_SetString(type, s.str().c_str());
    throw Raised();
}

std::string text(at::IntArrayRef shape) {
    std::ostringstream s;
    s << "(";
    for (size_t i = 0; i < shape.size(); ++i) s << (i ? ", " : "") << shape[i];
    s << (shape.size() == 1 ? ",)" : ")");
    return s.str();
}

const char* text(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return "torch.float32";
        case at::kHalf: return "torch.float16";
        case at::kBFloat16: return "torch.bfloat16";
        case at::kInt: return "torch.int32";
        default: return c10::toString(t);
    }
}

const at::Tensor& tensor(PyObject* o, const char* name, int64_t dims, const char* shape) {
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, name, ": expected a torch.Tensor", shape);
    const at::Tensor& t = THPVariable_Unpack(o);
    if (dims >= 0 && t.dim() != dims)
        raise(PyExc_TypeError, name, ": expected ", dims, " dims", shape, ", got ", t.dim());
    return t;
}

int64_t code(const at::Tensor& t, const char* name) {
    switch (t.scalar_type()) {
        case at::kFloat: return LIBSCAN_F32;
        case at::kHalf: return LIBSCAN_F16;
        case at::kBFloat16: return LIBSCAN_BF16;
        default:
            raise(PyExc_TypeError, name, ": expected float32, float16 or bfloat16, got ",
                  text(t.scalar_type()));
    }
}

// The operand that sets the others' sizes and GPU.
const at::Tensor& first(PyObject* o, const char* name, int64_t dims, int64_t& type) {
    const at::Tensor& t = tensor(o, name, -1, "");
    type = code(t, name);
    if (!t.is_cuda()) raise(PyExc_ValueError, name, ": expected a GPU tensor, got ", t.device());
    if (t.dim() != dims)
        raise(PyExc_ValueError, name, ": expected ", dims, " dims, got ", t.dim());
    return t;
}

// Checks an operand's type, shape and place, and that its last dimension has
// unit stride (dense: all of it is contiguous).
const at::Tensor& operand(PyObject* o, const char* name, at::ScalarType type,
                          at::IntArrayRef shape, const at::Tensor& on, bool dense) {
    const at::Tensor& t = tensor(o, name, -1, "");
    if (t.scalar_type() != type)
        raise(PyExc_TypeError, name, ": expected ", text(type), ", got ", text(t.scalar_type()));
    if (t.sizes() != shape)
        raise(PyExc_ValueError, name, ": expected shape ", text(shape), ", got ", text(t.sizes()));
    if (t.device() != on.device())
        raise(PyExc_ValueError, name, ": expected a tensor on the GPU of the first operand, got ",
              t.device());
    if (dense) {
        if (!t.is_contiguous()) raise(PyExc_ValueError, name, ": must be contiguous");
    } else if (t.dim() > 0 && t.size(-1) > 1 && t.stride(-1) != 1 && t.numel() > 0) {
        raise(PyExc_ValueError, name, ": the last dimension must have unit stride");
    }
    return t;
}

template <class T = void>
T* address(PyObject* o, const char* name, at::ScalarType type, at::IntArrayRef shape,
           const at::Tensor& on, bool dense) {
    return o == Py_None ? nullptr : (T*)operand(o, name, type, shape, on, dense).data_ptr();
}

// Says that the call records no graph, if one of its first n arguments (tensors or
// None by now) would have it recorded.
void no_graph(PyObject* const* a, int n, const char* instead) {
    if (!c10::GradMode::is_enabled()) return;
    for (int i = 0; i < n; ++i) {
        if (a[i] == Py_None || !THPVariable_Unpack(a[i]).requires_grad()) continue;
        const std::string s = std::string("an argument requires gradients, but no autograd graph "
                                          "is recorded here: ") + instead;
        // (the caller of the binding's function)
        if (PyErr_WarnEx(PyExc_UserWarning, s.c_str(), 2) < 0) throw Raised();
        return;
    }
}

bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised();
    return v != 0;
}

template <class S>
PyObject* packed(const S& s) {
    static_assert(sizeof(S) % 8 == 0, "fields are 8 bytes wide");
    return PyBytes_FromStringAndSize((const char*)&s, sizeof(S));
}

// (x, weight, bias, state, lengths, silu, step): a libscan_conv
PyObject* conv(PyObject* const* a) {
    libscan_conv p{};
    const bool step = truth(a[6]);
    const at::Tensor& x = first(a[0], "x", step ? 2 : 3, p.type);
    const at::ScalarType kind = x.scalar_type();
    p.batch = x.size(0);
    p.steps = step ? 1 : x.size(1);
    p.dim = x.size(-1);
    const at::Tensor& w = tensor(a[1], "weight", 2, " (dim x width)");
    if (w.scalar_type() != kind && w.scalar_type() != at::kFloat)
        raise(PyExc_TypeError, "weight: expected ", text(kind), " or torch.float32, got ",
              text(w.scalar_type()));
    p.weight_type = code(w, "weight");
    p.width = w.size(1);
    p.silu = truth(a[5]);
    p.x = operand(a[0], "x", kind, x.sizes(), x, false).data_ptr();
    p.x_batch = x.stride(0);
    p.x_step = step ? 0 : x.stride(1);
    p.weight = operand(a[1], "weight", w.scalar_type(), {p.dim, p.width}, x, true).data_ptr();
    p.bias = address(a[2], "bias", w.scalar_type(), {p.dim}, x, true);
    p.state = address(a[3], "state", kind, {p.batch, p.width - 1, p.dim}, x, true);
    p.lengths = address<int32_t>(a[4], "lengths", at::kInt, {p.batch}, x, true);
    no_graph(a, 5, step ? "a step has no gradients" : "causal_conv_backward forms the gradients");
    return packed(p);
}

// (x, dt, A, B, C, D, z, dt_bias, state, lengths, softplus, step): a libscan_ssm
PyObject* ssm(PyObject* const* a) {
    libscan_ssm p{};
    const bool step = truth(a[11]);
    const at::Tensor& x = first(a[0], "x", step ? 2 : 3, p.type);
    const at::ScalarType kind = x.scalar_type();
    p.batch = x.size(0);
    p.steps = step ? 1 : x.size(1);
    p.dim = x.size(-1);
    const at::Tensor& A = tensor(a[2], "A", 2, " (dim x n)");
    const at::Tensor& B = tensor(a[3], "B", step ? 3 : 4,
                                 step ? " (batch x groups x n)" : " (batch x steps x groups x n)");
    p.n = A.size(1);
    p.groups = B.size(-2);
    p.softplus = truth(a[10]);
    const int64_t b4[] = {p.batch, p.steps, p.groups, p.n}, b3[] = {p.batch, p.groups, p.n};
    const at::IntArrayRef bc = step ? at::IntArrayRef(b3) : at::IntArrayRef(b4);
    p.x = operand(a[0], "x", kind, x.sizes(), x, false).data_ptr();
    p.x_batch = x.stride(0);
    p.x_step = step ? 0 : x.stride(1);
    const at::Tensor& dt = operand(a[1], "dt", kind, x.sizes(), x, false);
    p.dt = dt.data_ptr();
    p.dt_batch = dt.stride(0);
    p.dt_step = step ? 0 : dt.stride(1);
    if (a[6] != Py_None) {
        const at::Tensor& z = operand(a[6], "z", kind, x.sizes(), x, false);
        p.z = z.data_ptr();
        p.z_batch = z.stride(0);
        p.z_step = step ? 0 : z.stride(1);
    }
    p.B = operand(a[3], "B", kind, bc, x, false).data_ptr();
    p.B_batch = B.stride(0);
    p.B_step = step ? 0 : B.stride(1);
    p.B_group = B.stride(-2);
    const at::Tensor& C = operand(a[4], "C", kind, bc, x, false);
    p.C = C.data_ptr();
    p.C_batch = C.stride(0);
    p.C_step = step ? 0 : C.stride(1);
    p.C_group = C.stride(-2);
    p.A = (const float*)operand(a[2], "A", at::kFloat, {p.dim, p.n}, x, true).data_ptr();
    p.D = address<float>(a[5], "D", at::kFloat, {p.dim}, x, true);
    p.dt_bias = address<float>(a[7], "dt_bias", at::kFloat, {p.dim}, x, true);
    p.state = address<float>(a[8], "state", at::kFloat, {p.batch, p.dim, p.n}, x, true);
    p.lengths = address<int32_t>(a[9], "lengths", at::kInt, {p.batch}, x, true);
    no_graph(a, 10, step ? "a step has no gradients"
                         : "selective_scan_backward forms the gradients");
    return packed(p);
}

double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Raised();
    return v;
}

// (q, k, v, log_decay, state, lengths, scale, step): a libscan_attend
PyObject* attend(PyObject* const* a) {
    libscan_attend p{};
    const bool step = truth(a[7]);
    const at::Tensor& q = first(a[0], "q", step ? 3 : 4, p.type);
    const at::ScalarType kind = q.scalar_type();
    const at::Tensor& v = tensor(a[2], "v", step ? 3 : 4,
                                 step ? " (batch x heads x dv)" : " (batch x steps x heads x dv)");
    p.batch = q.size(0);
    p.steps = step ? 1 : q.size(1);
    p.groups = q.size(-2);
    p.dk = q.size(-1);
    p.heads = v.size(-2);
    p.dv = v.size(-1);
    if (p.groups < 1 || p.heads % p.groups)
        raise(PyExc_ValueError, "v: expected heads in equal groups over the ", p.groups,
              " of q and k, got ", p.heads);
    const int64_t v4[] = {p.batch, p.steps, p.heads, p.dv}, v3[] = {p.batch, p.heads, p.dv};
    const int64_t each[] = {p.batch, p.steps, p.heads};
    const at::Tensor& k = operand(a[1], "k", kind, q.sizes(), q, false);
    p.q = operand(a[0], "q", kind, q.sizes(), q, false).data_ptr();
    p.q_batch = q.stride(0);
    p.q_step = step ? 0 : q.stride(1);
    p.q_head = q.stride(-2);
    p.k = k.data_ptr();
    p.k_batch = k.stride(0);
    p.k_step = step ? 0 : k.stride(1);
    p.k_head = k.stride(-2);
    p.v = operand(a[2], "v", kind, step ? at::IntArrayRef(v3) : at::IntArrayRef(v4), q, false)
              .data_ptr();
    p.v_batch = v.stride(0);
    p.v_step = step ? 0 : v.stride(1);
    p.v_head = v.stride(-2);
    const at::Tensor& g = tensor(a[3], "log_decay", -1, "");
    p.fixed = g.dim() == 1;
    if (p.fixed) {
        p.log_decay = address<float>(a[3], "log_decay", at::kFloat, {p.heads}, q, true);
    } else {
        const int64_t rows[] = {p.batch, p.heads};
        p.log_decay = address<float>(a[3], "log_decay", at::kFloat,
                                     step ? at::IntArrayRef(rows) : at::IntArrayRef(each), q,
                                     false);
        p.decay_batch = g.stride(0);
        p.decay_step = step ? 0 : g.stride(1);
    }
    p.state = address<float>(a[4], "state", at::kFloat, {p.batch, p.heads, p.dk, p.dv}, q, true);
    p.lengths = address<int32_t>(a[5], "lengths", at::kInt, {p.batch}, q, true);
    p.scale = a[6] == Py_None ? 1.0 / std::sqrt((double)p.dk) : real(a[6]);
    no_graph(a, 6, step ? "a step has no gradients"
                        : "linear_attention_backward forms the gradients");
    return packed(p);
}

// (x, weight, bias, residual, groups, eps): a libscan_norm
PyObject* norm(PyObject* const* a) {
    libscan_norm p{};
    const at::Tensor& any = tensor(a[0], "x", -1, "");
    const at::Tensor& x = first(a[0], "x", any.dim() == 2 ? 2 : 3, p.type);
    const at::ScalarType kind = x.scalar_type();
    const bool rows = x.dim() == 2;
    p.batch = rows ? 1 : x.size(0);
    p.steps = x.size(-2);
    p.dim = x.size(-1);
    p.groups = PyLong_AsLongLong(a[4]);
    if (PyErr_Occurred()) throw Raised();
    if (p.groups < 1 || p.dim % p.groups)
        raise(PyExc_ValueError, "groups: expected a divisor of ", p.dim, " channels, got ",
              p.groups);
    p.eps = real(a[5]);
    p.x = operand(a[0], "x", kind, x.sizes(), x, false).data_ptr();
    p.x_batch = rows ? 0 : x.stride(0);
    p.x_step = x.stride(-2);
    if (a[3] != Py_None) {
        const at::Tensor& r = operand(a[3], "residual", kind, x.sizes(), x, false);
        p.residual = r.data_ptr();
        p.residual_batch = rows ? 0 : r.stride(0);
        p.residual_step = r.stride(-2);
    }
    at::ScalarType weights = kind;
    for (int i = 1; i < 3; ++i) {
        if (a[i] == Py_None) continue;
        const char* name = i == 1 ? "weight" : "bias";
        const at::Tensor& w = tensor(a[i], name, 1, "");
        if (i == 1 || a[1] == Py_None) weights = w.scalar_type();
        if (weights != kind && weights != at::kFloat)
            raise(PyExc_TypeError, name, ": expected ", text(kind), " or torch.float32, got ",
                  text(weights));
        (i == 1 ? p.weight : p.bias) = operand(a[i], name, weights, {p.dim}, x, true).data_ptr();
    }
    p.weight_type = weights == kind ? p.type : LIBSCAN_F32;
    no_graph(a, 4, "layer_norm_backward forms the gradients");
    return packed(p);
}

// (logits, history, history_len, prompt_len, repetition, presence, frequency,
// bias_ids, bias_values, allowed, temperature): a libscan_logits
PyObject* logits(PyObject* const* a) {
    libscan_logits p{};
    const at::Tensor& x = first(a[0], "logits", 2, p.type);
    p.rows = x.size(0);
    p.vocab = x.size(1);
    p.logits = operand(a[0], "logits", x.scalar_type(), x.sizes(), x, false).data_ptr();
    p.logits_row = x.stride(0);
    if (a[1] != Py_None) {
        const at::Tensor& h = tensor(a[1], "history", 2, " (rows x tokens)");
        p.history_cols = h.size(1);
        p.history = (const int32_t*)operand(a[1], "history", at::kInt, {p.rows, p.history_cols}, x,
                                            false).data_ptr();
        p.history_row = h.stride(0);
    } else {
        for (int i = 2; i < 7; ++i)
            if (a[i] != Py_None) raise(PyExc_ValueError, "penalties need a history");
    }
    p.history_len = address<int32_t>(a[2], "history_len", at::kInt, {p.rows}, x, true);
    p.prompt_len = address<int32_t>(a[3], "prompt_len", at::kInt, {p.rows}, x, true);
    p.repetition = address<float>(a[4], "repetition", at::kFloat, {p.rows}, x, true);
    p.presence = address<float>(a[5], "presence", at::kFloat, {p.rows}, x, true);
    p.frequency = address<float>(a[6], "frequency", at::kFloat, {p.rows}, x, true);
    if ((a[7] == Py_None) != (a[8] == Py_None))
        raise(PyExc_ValueError, "bias_ids and bias_values go together");
    if (a[7] != Py_None) {
        p.biases = tensor(a[7], "bias_ids", 2, " (rows x entries)").size(1);
        p.bias_ids = address<int32_t>(a[7], "bias_ids", at::kInt, {p.rows, p.biases}, x, true);
        p.bias_values = address<float>(a[8], "bias_values", at::kFloat, {p.rows, p.biases}, x, true);
    }
    if (a[9] != Py_None) {
        const at::Tensor& al =
            operand(a[9], "allowed", at::kInt, {p.rows, (p.vocab + 31) / 32}, x, false);
        p.allowed = (const int32_t*)al.data_ptr();
        p.allowed_row = al.stride(0);
    }
    p.temperature = address<float>(a[10], "temperature", at::kFloat, {p.rows}, x, true);
    no_graph(a, 11, "processed logits have no gradients");
    return packed(p);
}

// (t, name, like, shape, fp32): checks a further operand of `like`'s type (or
// fp32) and GPU, dense, and returns its address (None: for None)
PyObject* dense(PyObject* const* a) {
    if (a[0] == Py_None) Py_RETURN_NONE;
    const char* name = PyUnicode_AsUTF8(a[1]);
    if (!name) throw Raised();
    const at::Tensor& like = THPVariable_Unpack(a[2]);
    int64_t shape[8];
    const Py_ssize_t n = PyTuple_Check(a[3]) ? PyTuple_GET_SIZE(a[3]) : -1;
    if (n < 0 || n > 8) raise(PyExc_TypeError, name, ": a shape of at most 8 dims");
    for (Py_ssize_t i = 0; i < n; ++i) {
        shape[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(a[3], i));
        if (PyErr_Occurred()) throw Raised();
    }
    const at::ScalarType type = truth(a[4]) ? at::kFloat : like.scalar_type();
    void* p = operand(a[0], name, type, {shape, (size_t)n}, like, true).data_ptr();
    if (!p) Py_RETURN_NONE;
    return PyLong_FromVoidPtr(p);
}

// (like, fp32): a new dense tensor of like's shape, GPU and type (or fp32)
PyObject* empty(PyObject* const* a) {
    const at::Tensor& like = THPVariable_Unpack(a[0]);
    const at::ScalarType type = truth(a[1]) ? at::kFloat : like.scalar_type();
    return THPVariable_Wrap(at::empty(like.sizes(), like.options().dtype(type)));
}

// (count, like): a new fp32 vector on like's GPU
PyObject* floats(PyObject* const* a) {
    const int64_t n = PyLong_AsLongLong(a[0]);
    if (PyErr_Occurred()) throw Raised();
    return THPVariable_Wrap(
        at::empty({n}, THPVariable_Unpack(a[1]).options().dtype(at::kFloat)));
}

// (address of a size query of libscan.h, struct bytes, sizes): its status, then
// the sizes
PyObject* sizes(PyObject* const* a) {
    void* fn = PyLong_AsVoidPtr(a[0]);
    const char* p = PyBytes_AsString(a[1]);
    const long n = PyLong_AsLong(a[2]);
    if (PyErr_Occurred()) throw Raised();
    size_t v[3] = {0, 0, 0};
    int status;
    if (n == 1)
        status = ((int (*)(const void*, size_t*))fn)(p, v);
    else if (n == 2)
        status = ((int (*)(const void*, size_t*, size_t*))fn)(p, v, v + 1);
    else
        status = ((int (*)(const void*, size_t*, size_t*, size_t*))fn)(p, v, v + 1, v + 2);
    PyObject* out = PyTuple_New(1 + n);
    if (!out) throw Raised();
    PyTuple_SET_ITEM(out, 0, PyLong_FromLong(status));
    for (long i = 0; i < n; ++i) PyTuple_SET_ITEM(out, 1 + i, PyLong_FromSize_t(v[i]));
    return out;
}

// (bytes, like): uninitialised memory on like's GPU
PyObject* memory(PyObject* const* a) {
    const int64_t n = PyLong_AsLongLong(a[0]);
    if (PyErr_Occurred()) throw Raised();
    return THPVariable_Wrap(
        at::empty({n}, THPVariable_Unpack(a[1]).options().dtype(at::kByte)));
}

template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Raised&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define ENTRY(f, n) {#f, (PyCFunction)(void (*)(void))entry<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(conv, 7),  ENTRY(ssm, 12),  ENTRY(logits, 11),
                         ENTRY(attend, 8), ENTRY(norm, 6),
                         ENTRY(dense, 5), ENTRY(empty, 2), ENTRY(sizes, 3),
                         ENTRY(memory, 2), ENTRY(floats, 2), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_args", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_args(void) { return PyModule_Create(&module); }
