// The calls of the operators around the recurrence as a Python extension module: a tensor's type, shape, layout and device are
// checked here and its address handed to the C ABI.  (In Python the checks of a call's six to thirteen tensors took 6 to 12 us,
// longer than a decode step's kernel; here a call takes about 1 us.)
//
// Every function takes the address of its C function first, then the layer (context, device, B, H, K, V, type of io), the tensors
// (None where one is optional), the numbers, and the stream's handle; it returns the C function's status.
#include <torch/csrc/autograd/python_variable.h>

#include <Python.h>

#include <initializer_list>
#include <stdexcept>
#include <string>

#include "sketchssm.h"

namespace {

struct Bad : std::runtime_error {
    using std::runtime_error::runtime_error;
};

struct Layer {
    sketchssm_ctx* ctx;
    int device, B, H, K, V;
    at::ScalarType io;
};

std::string text_of(const at::Tensor& t) {
    std::string s = std::string(c10::toString(t.scalar_type())) + " (";
    for (int64_t n : t.sizes()) s += std::to_string(n) + ", ";
    return s + ") on " + t.device().str();
}

[[noreturn]] void refuse(const char* name, const char* layout, at::ScalarType type, const int64_t* size, size_t dim, int device, const at::Tensor& t) {
    std::string s = std::string(name) + " is a " + layout + c10::toString(type) + " tensor (";
    for (size_t i = 0; i < dim; ++i) s += std::to_string(size[i]) + ", ";
    throw Bad(s + ") on cuda:" + std::to_string(device) + ": got " + text_of(t));
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) throw Bad(std::string(name) + " is a tensor");
    return THPVariable_Unpack(o);
}

bool same(const at::Tensor& t, at::ScalarType type, std::initializer_list<int64_t> size, int device) {
    return t.scalar_type() == type && t.is_cuda() && t.get_device() == device && t.sizes().equals(at::IntArrayRef(size.begin(), size.size()));
}

// A tensor's address; where it has no elements some address that is not null, as the C ABI takes a null pointer for an absent tensor
// (and reads or writes none of it).
void* place(const at::Tensor& t) {
    alignas(16) static char nothing[16];
    return t.numel() > 0 ? t.data_ptr() : nothing;
}

// A dense tensor's address (None: a null pointer).
void* dense(PyObject* o, const char* name, const Layer& l, at::ScalarType type, std::initializer_list<int64_t> size) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o, name);
    if (!same(t, type, size, l.device) || !t.is_contiguous()) refuse(name, "dense ", type, size.begin(), size.size(), l.device, t);
    return place(t);
}

struct Rows {
    void* p;
    int64_t stride;
};

// A tensor whose rows (first axis) may be strided: its address and the distance of two rows in elements.
Rows rows(PyObject* o, const char* name, const Layer& l, at::ScalarType type, std::initializer_list<int64_t> size) {
    const at::Tensor& t = tensor(o, name);
    if (!same(t, type, size, l.device)) refuse(name, "", type, size.begin(), size.size(), l.device, t);
    int64_t row = 1;
    for (int64_t d = (int64_t)size.size() - 1; d > 0; --d) {
        if (t.size(d) != 1 && t.stride(d) != row) throw Bad(std::string(name) + ": the elements of a row are dense");
        row *= t.size(d);
    }
    return {place(t), t.size(0) > 1 ? t.stride(0) : row};
}

long long number(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Bad("an argument is no integer");
    }
    return v;
}
void* address(PyObject* o) { return reinterpret_cast<void*>(static_cast<uintptr_t>(number(o))); }

constexpr at::ScalarType kF32 = at::kFloat, kBF16 = at::kBFloat16, kE4M3 = at::kFloat8_e4m3fn;

at::ScalarType f32_or_bf16(const at::Tensor& t, const char* name) {
    if (t.scalar_type() != kF32 && t.scalar_type() != kBF16) throw Bad(std::string(name) + " is f32 or bf16");
    return t.scalar_type();
}
int code(at::ScalarType t) { return t == kBF16 ? SKETCHSSM_BF16 : SKETCHSSM_F32; }

// An axis' size, which the C ABI takes as an int.
int64_t size_of(const at::Tensor& t, int64_t dim, int64_t axes, const char* name) {
    if (t.dim() != axes) throw Bad(std::string(name) + " has " + std::to_string(axes) + " axes");
    if (t.size(dim) > 0x7fffffff) throw Bad(std::string(name) + ": an axis is longer than 2^31 - 1");
    return t.size(dim);
}
int small(PyObject* o, const char* name) {
    const long long v = number(o);
    if (v < -0x7fffffffll || v > 0x7fffffffll) throw Bad(std::string(name) + " is out of range");
    return (int)v;
}

struct Work {
    void* p;
    size_t bytes;
};
// Scratch (None: none).
Work scratch(PyObject* o, const Layer& l) {
    if (o == Py_None) return {nullptr, 0};
    const at::Tensor& w = tensor(o, "work");
    if (!w.is_cuda() || w.get_device() != l.device || !w.is_contiguous()) throw Bad("work is a dense tensor on the layer's device");
    return {w.data_ptr(), w.nbytes()};
}

// (function, context, device, B, H, K, V, io): the first eight arguments of every call
constexpr int kHead = 8;
Layer layer(PyObject* const* a) {
    return {static_cast<sketchssm_ctx*>(address(a[1])), (int)number(a[2]), (int)number(a[3]), (int)number(a[4]), (int)number(a[5]), (int)number(a[6]),
            number(a[7]) == SKETCHSSM_BF16 ? kBF16 : kF32};
}

template <typename F>
PyObject* call(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, F&& f) {
    if (n != kHead + want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        const Layer l = layer(a);
        return PyLong_FromLong(f(l, a + kHead));
    } catch (const Bad& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// prompts (address), T, x, weight, bias, state, out, flags, stream
PyObject* causal_conv(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 9, [fn = n ? a[0] : nullptr](const Layer& l, PyObject* const* v) {
        const int64_t T = number(v[1]), C = size_of(tensor(v[3], "weight"), 0, 2, "weight"), W = size_of(tensor(v[3], "weight"), 1, 2, "weight");
        const Rows x = rows(v[2], "x", l, l.io, {T, C}), out = rows(v[6], "out", l, l.io, {T, C});
        return reinterpret_cast<decltype(&sketchssm_causal_conv)>(address(fn))(
            l.ctx, static_cast<const sketchssm_prompts*>(address(v[0])), (int)C, (int)W, dense(v[3], "weight", l, kF32, {C, W}),
            dense(v[4], "bias", l, kF32, {C}), dense(v[5], "state", l, l.io, {l.B, W - 1, C}), x.p, x.stride, out.p, out.stride,
            (uint32_t)number(v[7]), address(v[8]));
    });
}

// x, dt, weight, bias, state, a, dt_bias, q, k, v, beta, decay, groups, stream
PyObject* conv_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 14, [fn = n ? a[0] : nullptr](const Layer& l, PyObject* const* v) {
        const int64_t G = small(v[12], "groups"), C = (int64_t)l.H * l.V + 2 * G * l.K, W = size_of(tensor(v[2], "weight"), 1, 2, "weight");
        const Rows x = rows(v[0], "x", l, l.io, {l.B, C}), dt = rows(v[1], "dt", l, l.io, {l.B, l.H});
        return reinterpret_cast<decltype(&sketchssm_conv_step)>(address(fn))(
            l.ctx, (int)G, (int)W, dense(v[2], "weight", l, kF32, {C, W}), dense(v[3], "bias", l, kF32, {C}),
            dense(v[4], "state", l, l.io, {l.B, W - 1, C}), x.p, x.stride, dt.p, dt.stride, dense(v[5], "a", l, kF32, {l.H}),
            dense(v[6], "dt_bias", l, kF32, {l.H}), dense(v[7], "q", l, l.io, {l.B, l.H, l.K}), dense(v[8], "k", l, l.io, {l.B, l.H, l.K}),
            dense(v[9], "v", l, l.io, {l.B, l.H, l.V}), dense(v[10], "beta", l, kF32, {l.B, l.H}), dense(v[11], "decay", l, kF32, {l.B, l.H}),
            address(v[13]));
    });
}

// prompts (address), T, q, k, v, dt, a, out, dt_bias, skip, work, stream
PyObject* prompt_scan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 12, [fn = n ? a[0] : nullptr](const Layer& l, PyObject* const* v) {
        const int64_t T = number(v[1]), G = size_of(tensor(v[2], "q"), 1, 3, "q");
        const at::ScalarType od = f32_or_bf16(tensor(v[7], "out"), "out");
        const Rows q = rows(v[2], "q", l, l.io, {T, G, l.K}), k = rows(v[3], "k", l, l.io, {T, G, l.K}), x = rows(v[4], "v", l, l.io, {T, l.H, l.V}),
                   dt = rows(v[5], "dt", l, l.io, {T, l.H}), out = rows(v[7], "out", l, od, {T, l.H, l.V});
        const Work work = scratch(v[10], l);
        return reinterpret_cast<decltype(&sketchssm_prompt_scan)>(address(fn))(
            l.ctx, static_cast<const sketchssm_prompts*>(address(v[0])), (int)G, q.p, q.stride, k.p, k.stride, x.p, x.stride, dt.p, dt.stride,
            dense(v[6], "a", l, kF32, {l.H}), dense(v[8], "dt_bias", l, kF32, {l.H}), dense(v[9], "skip", l, kF32, {l.H}), out.p, out.stride,
            code(od), work.p, work.bytes, address(v[11]));
    });
}

// x, weight, out, out8, scale, residual, residual_out, gate, skip, skip_weight, eps, group, stream
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 13, [fn = n ? a[0] : nullptr](const Layer& l, PyObject* const* v) {
        const at::Tensor& xt = tensor(v[0], "x");
        const int64_t T = size_of(xt, 0, 2, "x"), D = size_of(xt, 1, 2, "x");
        const at::ScalarType xd = f32_or_bf16(xt, "x");
        const Rows x = rows(v[0], "x", l, xd, {T, D}), none = {nullptr, 0};
        const Rows gate = v[7] == Py_None ? none : rows(v[7], "gate", l, l.io, {T, D}), skip = v[8] == Py_None ? none : rows(v[8], "skip", l, l.io, {T, D});
        const int64_t heads = v[9] == Py_None ? 0 : size_of(tensor(v[9], "skip_weight"), 0, 1, "skip_weight");
        const double eps = PyFloat_AsDouble(v[10]);
        if (eps == -1.0 && PyErr_Occurred()) {
            PyErr_Clear();
            throw Bad("eps is no number");
        }
        return reinterpret_cast<decltype(&sketchssm_rms_norm)>(address(fn))(
            l.ctx, (int)T, (int)D, small(v[11], "group"), (float)eps, x.p, x.stride, code(xd), dense(v[1], "weight", l, kF32, {D}),
            dense(v[5], "residual", l, l.io, {T, D}), dense(v[6], "residual_out", l, l.io, {T, D}), gate.p, gate.stride, skip.p, skip.stride,
            dense(v[9], "skip_weight", l, kF32, {heads}), (int)heads, dense(v[2], "out", l, l.io, {T, D}), dense(v[3], "out8", l, kE4M3, {T, D}),
            dense(v[4], "scale", l, kF32, {T, (D + 127) / 128}), address(v[12]));
    });
}

// a, a_scale, w, w_scale, out, stream
PyObject* scaled_matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 6, [fn = n ? a[0] : nullptr](const Layer& l, PyObject* const* v) {
        const int64_t M = size_of(tensor(v[0], "a"), 0, 2, "a"), K = size_of(tensor(v[0], "a"), 1, 2, "a"), N = size_of(tensor(v[2], "w"), 0, 2, "w"), kb = (K + 127) / 128;
        const at::ScalarType od = f32_or_bf16(tensor(v[4], "out"), "out");
        const Rows out = rows(v[4], "out", l, od, {M, N});
        return reinterpret_cast<decltype(&sketchssm_scaled_matmul)>(address(fn))(
            l.ctx, (int)M, (int)N, (int)K, dense(v[0], "a", l, kE4M3, {M, K}), dense(v[1], "a_scale", l, kF32, {M, kb}), dense(v[2], "w", l, kE4M3, {N, K}),
            dense(v[3], "w_scale", l, kF32, {(N + 127) / 128, kb}), out.p, out.stride, code(od), address(v[5]));
    });
}

bool kda(PyObject* o) { return number(o) == SKETCHSSM_KDA; }
float real(PyObject* o, const char* name) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Bad(std::string(name) + " is no number");
    }
    return (float)x;
}
// The arguments of the decays of n rows: a number a head, or one for every channel of its keys (dense within a row).
Rows decays(PyObject* o, const Layer& l, bool per_channel, int64_t n) {
    if (!per_channel) return rows(o, "dt", l, l.io, {n, l.H});
    const at::Tensor& t = tensor(o, "dt");
    return t.dim() == 3 ? rows(o, "dt", l, l.io, {n, l.H, l.K}) : rows(o, "dt", l, l.io, {n, (int64_t)l.H * l.K});
}
void* biases(PyObject* o, const Layer& l, bool per_channel) {
    return per_channel ? dense(o, "dt_bias", l, kF32, {l.H, l.K}) : dense(o, "dt_bias", l, kF32, {l.H});
}

// kind, x, b, dt, weight, bias, state, a, dt_bias, q, k, v, beta, decay, groups, eps, q_scale, stream
PyObject* delta_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 18, [fn = n ? a[0] : nullptr](const Layer& l, PyObject* const* v) {
        const bool ch = kda(v[0]);
        const int64_t G = small(v[14], "groups"), C = (int64_t)l.H * l.V + 2 * G * l.K, W = size_of(tensor(v[4], "weight"), 1, 2, "weight");
        const Rows x = rows(v[1], "x", l, l.io, {l.B, C}), b = rows(v[2], "b", l, l.io, {l.B, l.H}), dt = decays(v[3], l, ch, l.B);
        return reinterpret_cast<decltype(&sketchssm_delta_step)>(address(fn))(
            l.ctx, (int)G, (int)W, real(v[15], "eps"), real(v[16], "q_scale"), dense(v[4], "weight", l, kF32, {C, W}), dense(v[5], "bias", l, kF32, {C}),
            dense(v[6], "state", l, l.io, {l.B, W - 1, C}), x.p, x.stride, b.p, b.stride, dt.p, dt.stride, dense(v[7], "a", l, kF32, {l.H}),
            biases(v[8], l, ch), dense(v[9], "q", l, l.io, {l.B, l.H, l.K}), dense(v[10], "k", l, l.io, {l.B, l.H, l.K}),
            dense(v[11], "v", l, l.io, {l.B, l.H, l.V}), dense(v[12], "beta", l, kF32, {l.B, l.H}),
            ch ? dense(v[13], "decay", l, l.io, {l.B, l.H, l.K}) : dense(v[13], "decay", l, kF32, {l.B, l.H}), address(v[17]));
    });
}

// kind, prompts (address), T, q, k, v, b, dt, a, out, dt_bias, work, eps, q_scale, stream
PyObject* delta_scan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 15, [fn = n ? a[0] : nullptr](const Layer& l, PyObject* const* v) {
        const bool ch = kda(v[0]);
        const int64_t T = number(v[2]), G = size_of(tensor(v[3], "q"), 1, 3, "q");
        const at::ScalarType od = f32_or_bf16(tensor(v[9], "out"), "out");
        const Rows q = rows(v[3], "q", l, l.io, {T, G, l.K}), k = rows(v[4], "k", l, l.io, {T, G, l.K}), x = rows(v[5], "v", l, l.io, {T, l.H, l.V}),
                   b = rows(v[6], "b", l, l.io, {T, l.H}), dt = decays(v[7], l, ch, T), out = rows(v[9], "out", l, od, {T, l.H, l.V});
        const Work w = scratch(v[11], l);
        return reinterpret_cast<decltype(&sketchssm_delta_scan)>(address(fn))(
            l.ctx, static_cast<const sketchssm_prompts*>(address(v[1])), (int)G, real(v[12], "eps"), real(v[13], "q_scale"), q.p, q.stride, k.p, k.stride,
            x.p, x.stride, b.p, b.stride, dt.p, dt.stride, dense(v[8], "a", l, kF32, {l.H}), biases(v[10], l, ch), out.p, out.stride, code(od), w.p,
            w.bytes, address(v[14]));
    });
}

// x, weight, out8, scale, out, residual, residual_out, gate, flags, eps, stream
PyObject* integer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 11, [fn = n ? a[0] : nullptr](const Layer& l, PyObject* const* v) {
        const at::Tensor& xt = tensor(v[0], "x");
        const int64_t T = size_of(xt, 0, 2, "x"), D = size_of(xt, 1, 2, "x"), group = size_of(tensor(v[1], "weight"), 0, 1, "weight");
        const at::ScalarType xd = f32_or_bf16(xt, "x");
        const Rows x = rows(v[0], "x", l, xd, {T, D}), none = {nullptr, 0}, gate = v[7] == Py_None ? none : rows(v[7], "gate", l, l.io, {T, D});
        return reinterpret_cast<decltype(&sketchssm_integer_norm)>(address(fn))(
            l.ctx, (int)T, (int)D, (int)group, real(v[9], "eps"), x.p, x.stride, code(xd), dense(v[1], "weight", l, kF32, {group}),
            dense(v[5], "residual", l, l.io, {T, D}), dense(v[6], "residual_out", l, l.io, {T, D}), gate.p, gate.stride, (uint32_t)number(v[8]),
            dense(v[4], "out", l, l.io, {T, D}), dense(v[2], "out8", l, at::kChar, {T, D}), dense(v[3], "scale", l, kF32, {T}), address(v[10]));
    });
}

// a, a_scale, w, w_scale, out, stream
PyObject* integer_matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(a, n, 6, [fn = n ? a[0] : nullptr](const Layer& l, PyObject* const* v) {
        const int64_t M = size_of(tensor(v[0], "a"), 0, 2, "a"), K = size_of(tensor(v[0], "a"), 1, 2, "a"), N = size_of(tensor(v[2], "w"), 0, 2, "w");
        const at::ScalarType od = f32_or_bf16(tensor(v[4], "out"), "out");
        const Rows out = rows(v[4], "out", l, od, {M, N});
        return reinterpret_cast<decltype(&sketchssm_integer_matmul)>(address(fn))(
            l.ctx, (int)M, (int)N, (int)K, dense(v[0], "a", l, at::kChar, {M, K}), dense(v[1], "a_scale", l, kF32, {M}), dense(v[2], "w", l, at::kChar, {N, K}),
            dense(v[3], "w_scale", l, kF32, {N}), out.p, out.stride, code(od), address(v[5]));
    });
}

#define SKETCHSSM_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {SKETCHSSM_METHOD(causal_conv), SKETCHSSM_METHOD(conv_step),    SKETCHSSM_METHOD(prompt_scan),
                          SKETCHSSM_METHOD(rms_norm),    SKETCHSSM_METHOD(scaled_matmul), SKETCHSSM_METHOD(delta_step), SKETCHSSM_METHOD(delta_scan),
                          SKETCHSSM_METHOD(integer_norm),   SKETCHSSM_METHOD(integer_matmul), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_layer_calls", "Calls of the operators around the recurrence.", -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layer_calls(void) { return PyModule_Create(&kModule); }
