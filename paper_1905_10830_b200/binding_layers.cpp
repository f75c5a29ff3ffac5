// The Python side of the layer calls (tc_quantize_blocks, tc_matmul_blocks, tc_residual_norms and its backward), as a module of
// CPython functions: a single token's call takes the GPU 2 to 7 us, and reading, checking and making its tensors took
// Python and ctypes 6 to 19 us.  It checks tensors, makes those that are returned and calls the C ABI, whose entry points it is
// given as addresses; nothing is computed here.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "tc.h"

namespace {

decltype(&tc_quantize_blocks) call_quantize = nullptr;
decltype(&tc_matmul_blocks) call_matmul = nullptr;
decltype(&tc_residual_norms) call_norms = nullptr;
decltype(&tc_residual_norms_backward) call_backward = nullptr;
PyObject *error_type = nullptr, *blocks_type = nullptr;              // TcError(code, where); Blocks(codes, scales, cols, square)
PyObject *name_codes = nullptr, *name_scales = nullptr, *name_cols = nullptr, *name_square = nullptr;

struct Bad { std::string what; };                                    // a ValueError
struct Raised {};                                                    // a Python error that is set already

// An owned reference.
struct Ref {
    PyObject *p = nullptr;
    Ref() = default;
    explicit Ref(PyObject *o) : p(o) { if (!o) throw Raised{}; }
    Ref(Ref &&o) noexcept : p(o.p) { o.p = nullptr; }
    Ref &operator=(Ref &&o) noexcept { std::swap(p, o.p); return *this; }
    ~Ref() { Py_XDECREF(p); }
    PyObject *give() { PyObject *o = p; p = nullptr; return o; }
};
PyObject *none()
{
    Py_INCREF(Py_None);
    return Py_None;
}

struct Call {
    tc_ctx *ctx;
    int device;
    void *stream;
    Call(PyObject *const *args)
    {
        ctx = args[0] == Py_None ? nullptr : (tc_ctx *)PyLong_AsVoidPtr(args[0]);   // (a closed context has no address: the call refuses it)
        device = (int)PyLong_AsLong(args[1]);
        stream = PyLong_AsVoidPtr(args[2]);
        if (PyErr_Occurred()) throw Raised{};
    }
    void check(tc_status status, const char *where) const
    {
        if (status == TC_OK) return;
        Ref e(PyObject_CallFunction(error_type, "is", (int)status, where));
        PyErr_SetObject(error_type, e.p);
        throw Raised{};
    }
};

const at::Tensor &tensor_of(PyObject *o)
{
    if (!THPVariable_Check(o)) throw Bad{"expected a torch tensor"};
    return THPVariable_Unpack(o);
}
bool on_device(const at::Tensor &t, int device) { return t.is_cuda() && t.get_device() == device && t.is_contiguous(); }

tc_tensor map_of(const at::Tensor &x, int device)
{
    if (!x.is_cuda() || !x.is_contiguous() || x.dim() != 4) throw Bad{"expected a contiguous 4-d CUDA tensor (NCHW)"};
    if (x.get_device() != device) throw Bad{"expected tensors on the context's device"};
    const auto type = x.scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) throw Bad{"dtype must be float32 or bfloat16"};
    for (int i = 0; i < 4; ++i)
        if (x.size(i) > INT32_MAX) throw Bad{"tensor sides must fit 32 bits"};
    return tc_tensor{x.data_ptr(), (int32_t)x.size(0), (int32_t)x.size(1), (int32_t)x.size(2), (int32_t)x.size(3), type == at::kFloat ? TC_F32 : TC_BF16};
}
int64_t pixels_of(const tc_tensor &t) { return (int64_t)t.n * t.h * t.w; }

// A tensor of the shape and type of `h`; a tensor without values has no address, but it is there.
void *like(PyObject *o, const at::Tensor &h, int device, const char *name)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor_of(o);
    if (!on_device(t, device) || t.scalar_type() != h.scalar_type() || t.sizes() != h.sizes())
        throw Bad{std::string(name) + ": expected a contiguous tensor of the shape and type of the first, on the context's device"};
    return t.numel() ? t.data_ptr() : (void *)16;
}
float *vector(PyObject *o, int64_t n, int device, const char *name)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor_of(o);
    if (!on_device(t, device) || t.scalar_type() != at::kFloat || t.numel() != n)
        throw Bad{std::string(name) + ": expected " + std::to_string(n) + " contiguous float32 values on the context's device"};
    return (float *)t.data_ptr();
}
at::Tensor make(at::IntArrayRef sizes, at::ScalarType type, int device)
{
    return at::detail::empty_cuda(sizes, type, at::Device(at::kCUDA, (c10::DeviceIndex)device), c10::nullopt);
}
at::Tensor make_like(const at::Tensor &t) { return make(t.sizes(), t.scalar_type(), t.get_device()); }
Ref wrap(const at::Tensor &t) { return Ref(THPVariable_Wrap(t)); }

// Blocks: the C structure, of a new one together with the Python object.
struct BlocksRef {
    Ref object;
    tc_blocks blocks{};
};
void shape_of_scales(int64_t rows, int64_t cols, bool square, int64_t (&shape)[2])
{
    const int64_t tall = (rows + 127) / 128;
    shape[0] = (cols + 127) / 128;
    shape[1] = square ? tall : tall * 128;
}
BlocksRef new_blocks(int64_t rows, int64_t cols, bool square, int device)
{
    BlocksRef b;
    int64_t shape[2];
    if (rows > INT32_MAX || cols > INT32_MAX) throw Bad{"block matrix: rows and cols must fit 32 bits"};
    shape_of_scales(rows, cols, square, shape);
    const int64_t ld = (cols + 15) / 16 * 16;
    const at::Tensor codes = make({rows, ld}, at::kFloat8_e4m3fn, device), scales = make(shape, at::kFloat, device);
    Ref c = wrap(codes), s = wrap(scales), n(PyLong_FromLongLong(cols));
    PyObject *const args[4] = {c.p, s.p, n.p, square ? Py_True : Py_False};
    b.object = Ref(PyObject_Vectorcall(blocks_type, args, 4, nullptr));
    b.blocks = tc_blocks{codes.data_ptr(), (float *)scales.data_ptr(), ld, (int32_t)rows, (int32_t)cols, square};
    return b;
}
tc_blocks given_blocks(PyObject *o, int device)
{
    Ref c(PyObject_GetAttr(o, name_codes)), s(PyObject_GetAttr(o, name_scales)), n(PyObject_GetAttr(o, name_cols)), q(PyObject_GetAttr(o, name_square));
    const at::Tensor &codes = tensor_of(c.p), &scales = tensor_of(s.p);
    const int64_t cols = PyLong_AsLongLong(n.p);
    const int square = PyObject_IsTrue(q.p);
    if (PyErr_Occurred()) throw Raised{};
    if (!on_device(codes, device) || !on_device(scales, device) || codes.dim() != 2 || scales.dim() != 2 || codes.scalar_type() != at::kFloat8_e4m3fn ||
        scales.scalar_type() != at::kFloat)
        throw Bad{"block matrices have contiguous float8_e4m3fn codes [rows, ld] and float32 scales on the context's device"};
    int64_t shape[2];
    shape_of_scales(codes.size(0), cols, square, shape);
    if (cols < 0 || cols > codes.size(1) || scales.size(0) != shape[0] || scales.size(1) != shape[1] || codes.size(0) > INT32_MAX || codes.size(1) > INT32_MAX)
        throw Bad{"block matrix: codes, scales and cols do not belong together"};
    return tc_blocks{codes.data_ptr(), (float *)scales.data_ptr(), codes.size(1), (int32_t)codes.size(0), (int32_t)cols, square};
}

template <typename F>
PyObject *guarded(PyObject *const *args, Py_ssize_t given, Py_ssize_t wanted, F body)
{
    HANDLE_TH_ERRORS
    try {
        if (given != wanted) throw Bad{"wrong number of arguments"};
        return body(Call(args), args + 3);
    } catch (const Bad &b) {
        PyErr_SetString(PyExc_ValueError, b.what.c_str());
    } catch (const Raised &) {
    }
    return nullptr;
    END_HANDLE_TH_ERRORS
}
// The C call, without the interpreter's lock (it may wait for memory).
template <typename F>
tc_status unlocked(F call)
{
    PyThreadState *const state = PyEval_SaveThread();
    const tc_status status = call();
    PyEval_RestoreThread(state);
    return status;
}

// x, rows, square, out
PyObject *quantize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 7, [](const Call &c, PyObject *const *a) -> PyObject * {
        const tc_tensor x = map_of(tensor_of(a[0]), c.device);
        const char *rows = PyUnicode_Check(a[1]) ? PyUnicode_AsUTF8(a[1]) : "";
        if (!rows) throw Raised{};
        const bool both = !strcmp(rows, "both"), pixels = both || !strcmp(rows, "pixels"), channels = both || !strcmp(rows, "channels");
        if (!pixels && !channels) throw Bad{"rows: \"pixels\", \"channels\" or \"both\""};
        const int square = PyObject_IsTrue(a[2]);
        if (square < 0) throw Raised{};
        PyObject *outs[2] = {a[3], a[3]};
        Ref pair;
        if (a[3] != Py_None && both) {
            pair = Ref(PySequence_Tuple(a[3]));
            if (PyTuple_GET_SIZE(pair.p) != 2) throw Bad{"out: Blocks as this call returns them"};
            outs[0] = PyTuple_GET_ITEM(pair.p, 0);
            outs[1] = PyTuple_GET_ITEM(pair.p, 1);
        }
        BlocksRef b[2];
        const int64_t p = pixels_of(x);
        for (int i = 0; i < 2; ++i) {
            if (!(i ? channels : pixels)) continue;
            if (a[3] == Py_None) b[i] = new_blocks(i ? x.c : p, i ? p : x.c, square, c.device);
            else {
                b[i].blocks = given_blocks(outs[i], c.device);
                if (!b[i].blocks.square != !square) throw Bad{"out: Blocks as this call returns them"};
                Py_INCREF(outs[i]);
                b[i].object = Ref(outs[i]);
            }
        }
        c.check(unlocked([&] { return call_quantize(c.ctx, &x, pixels ? &b[0].blocks : nullptr, channels ? &b[1].blocks : nullptr, c.stream); }), "tc_quantize_blocks");
        if (both) return PyTuple_Pack(2, b[0].object.p, b[1].object.p);
        return b[pixels ? 0 : 1].object.give();
    });
}

// a, b, shape, dtype, bias, relu, out
PyObject *matmul(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 10, [](const Call &c, PyObject *const *a) -> PyObject * {
        const tc_blocks ma = given_blocks(a[0], c.device), mb = given_blocks(a[1], c.device);
        const int relu = PyObject_IsTrue(a[5]);
        if (relu < 0) throw Raised{};
        Ref made;
        PyObject *out = a[6];
        if (out == Py_None) {
            int64_t shape[3] = {ma.rows, 1, 1};
            if (a[2] != Py_None) {
                Ref s(PySequence_Tuple(a[2]));
                if (PyTuple_GET_SIZE(s.p) != 3) throw Bad{"shape: expected (N, H, W)"};
                for (int i = 0; i < 3; ++i) shape[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s.p, i));
                if (PyErr_Occurred()) throw Raised{};
            }
            const at::ScalarType type = THPDtype_Check(a[3]) ? ((THPDtype *)a[3])->scalar_type : at::kInt;
            if (type != at::kFloat && type != at::kBFloat16) throw Bad{"dtype must be float32 or bfloat16"};
            for (const int64_t v : shape)
                if (v < 0 || v > INT32_MAX) throw Bad{"shape: expected (N, H, W)"};
            made = wrap(make({shape[0], mb.rows, shape[1], shape[2]}, type, c.device));
            out = made.p;
        }
        const tc_tensor t = map_of(tensor_of(out), c.device);
        const float *bias = vector(a[4], mb.rows, c.device, "bias");
        c.check(unlocked([&] { return call_matmul(c.ctx, &ma, &mb, bias, relu, &t, c.stream); }), "tc_matmul_blocks");
        Py_INCREF(out);
        return out;
    });
}

// y, after, gate, scale, before, eps
tc_norm_params norm_params(PyObject *const *a, const at::Tensor &h, int device)
{
    const bool map = a[2] != Py_None && tensor_of(a[2]).dim() == 4;
    const double eps = PyFloat_AsDouble(a[5]);
    if (PyErr_Occurred()) throw Raised{};
    const int64_t c = h.size(1);
    return tc_norm_params{like(a[0], h, device, "y"), vector(a[1], c, device, "after"), map ? nullptr : vector(a[2], c, device, "gate"),
                          map ? like(a[2], h, device, "gate") : nullptr, vector(a[3], 1, device, "scale"), vector(a[4], c, device, "before"), (float)eps};
}

// h, then norm_params', blocks, sum_out, out
PyObject *norms(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 13, [](const Call &c, PyObject *const *a) -> PyObject * {
        const at::Tensor &h = tensor_of(a[0]);
        const tc_tensor t = map_of(h, c.device);
        const tc_norm_params p = norm_params(a + 1, h, c.device);
        const bool both = PyUnicode_Check(a[7]) && PyUnicode_CompareWithASCIIString(a[7], "both") == 0;
        const int blocks = both || PyObject_IsTrue(a[7]);
        if (PyErr_Occurred()) throw Raised{};
        Ref sum, x, pair;
        void *at_sum = nullptr, *at_x = nullptr;
        BlocksRef codes;
        const bool has_y = a[1] != Py_None, has_x = a[5] != Py_None;
        PyObject *out_x = a[9], *out_codes = a[9];
        if (both && has_x && a[9] != Py_None) {
            pair = Ref(PySequence_Tuple(a[9]));
            if (PyTuple_GET_SIZE(pair.p) != 2) throw Bad{"out: a tensor and Blocks as this call returns them"};
            out_x = PyTuple_GET_ITEM(pair.p, 0);
            out_codes = PyTuple_GET_ITEM(pair.p, 1);
        }
        if (has_y) {
            if (a[8] == Py_None) sum = wrap(make_like(h));
            else { Py_INCREF(a[8]); sum = Ref(a[8]); }
            at_sum = like(sum.p, h, c.device, "sum_out");
        } else { Py_INCREF(a[0]); sum = Ref(a[0]); }
        if (has_x && (both || !blocks)) {
            if (out_x == Py_None) x = wrap(make_like(h));
            else { Py_INCREF(out_x); x = Ref(out_x); }
            at_x = like(x.p, h, c.device, "out");
        }
        if (has_x && blocks) {
            if (out_codes == Py_None) codes = new_blocks(pixels_of(t), t.c, false, c.device);
            else {
                codes.blocks = given_blocks(out_codes, c.device);
                Py_INCREF(out_codes);
                codes.object = Ref(out_codes);
            }
            x = both ? Ref(PyTuple_Pack(2, x.p, codes.object.p)) : std::move(codes.object);
        } else if (!has_x) x = Ref(none());
        c.check(unlocked([&] { return call_norms(c.ctx, &t, &p, at_sum, at_x, has_x && blocks ? &codes.blocks : nullptr, c.stream); }), "tc_residual_norms");
        return PyTuple_Pack(2, sum.p, x.p);
    });
}

// s, dx, ds, then norm_params': (h, y, after, gate, scale, before)
PyObject *backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 12, [](const Call &c, PyObject *const *a) -> PyObject * {
        const at::Tensor &s = tensor_of(a[0]);
        const tc_tensor t = map_of(s, c.device);
        const tc_norm_params p = norm_params(a + 3, s, c.device);
        const void *dx = like(a[1], s, c.device, "dx"), *ds = like(a[2], s, c.device, "ds");
        PyObject *const of[6] = {a[0], a[3], a[4], a[5], a[6], a[7]};                // s, y, after, gate, scale, before
        Ref grads[6];
        void *at[6];
        for (int i = 0; i < 6; ++i) {
            if (of[i] == Py_None) {
                grads[i] = Ref(none());
                at[i] = nullptr;
            } else {
                const at::Tensor g = make_like(tensor_of(of[i]));
                at[i] = g.data_ptr();
                grads[i] = wrap(g);
            }
        }
        const tc_norm_grads out{at[0], at[1], p.gate_map ? at[3] : nullptr, (float *)at[2], p.gate_map ? nullptr : (float *)at[3], (float *)at[4], (float *)at[5]};
        c.check(unlocked([&] { return call_backward(c.ctx, &t, &p, dx, ds, &out, c.stream); }), "tc_residual_norms_backward");
        return PyTuple_Pack(6, grads[0].p, grads[1].p, grads[2].p, grads[3].p, grads[4].p, grads[5].p);
    });
}

// addresses of the four entry points, TcError, Blocks
PyObject *init(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) { PyErr_SetString(PyExc_ValueError, "wrong number of arguments"); return nullptr; }
    call_quantize = (decltype(call_quantize))PyLong_AsVoidPtr(args[0]);
    call_matmul = (decltype(call_matmul))PyLong_AsVoidPtr(args[1]);
    call_norms = (decltype(call_norms))PyLong_AsVoidPtr(args[2]);
    call_backward = (decltype(call_backward))PyLong_AsVoidPtr(args[3]);
    Py_INCREF(args[4]);
    Py_INCREF(args[5]);
    error_type = args[4];
    blocks_type = args[5];
    name_codes = PyUnicode_InternFromString("codes");
    name_scales = PyUnicode_InternFromString("scales");
    name_cols = PyUnicode_InternFromString("cols");
    name_square = PyUnicode_InternFromString("square");
    if (PyErr_Occurred()) return nullptr;
    return none();
}

PyMethodDef methods[] = {{"init", (PyCFunction)(void *)init, METH_FASTCALL, nullptr},
                         {"quantize", (PyCFunction)(void *)quantize, METH_FASTCALL, nullptr},
                         {"matmul", (PyCFunction)(void *)matmul, METH_FASTCALL, nullptr},
                         {"norms", (PyCFunction)(void *)norms, METH_FASTCALL, nullptr},
                         {"backward", (PyCFunction)(void *)backward, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layers", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layers(void) { return PyModule_Create(&module); }
