// The Python side of the layer calls (codes, their products, norms and their gradients), as a module of
// CPython functions: a single token's call takes the GPU 2 to 7 us, and reading, checking and making its tensors took
// Python and ctypes 6 to 19 us.  It checks tensors, makes those that are returned and calls the C ABI, whose entry points it is
// given as addresses; nothing is computed here.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <vector>

#include "tc.h"

namespace {

decltype(&tc_quantize_blocks) call_quantize = nullptr;
decltype(&tc_matmul_blocks) call_matmul = nullptr;
decltype(&tc_residual_norms) call_norms = nullptr;
decltype(&tc_residual_norms_backward) call_backward = nullptr;
decltype(&tc_quantize_rows) call_quantize_rows = nullptr;
decltype(&tc_matmul_rows) call_matmul_rows = nullptr;
decltype(&tc_group_norm) call_group_norm = nullptr;
decltype(&tc_group_norm_backward) call_group_backward = nullptr;
decltype(&tc_gradient_norm) call_gradient_norm = nullptr;
decltype(&tc_clip_gradients) call_clip_gradients = nullptr;
struct EntryPoint { const char *name; void *at; };                   // of the C ABI, and the pointer that keeps it
const EntryPoint entry_points[] = {{"tc_quantize_blocks", &call_quantize}, {"tc_matmul_blocks", &call_matmul}, {"tc_residual_norms", &call_norms},
                                   {"tc_residual_norms_backward", &call_backward}, {"tc_quantize_rows", &call_quantize_rows}, {"tc_matmul_rows", &call_matmul_rows},
                                   {"tc_group_norm", &call_group_norm}, {"tc_group_norm_backward", &call_group_backward},
                                   {"tc_gradient_norm", &call_gradient_norm}, {"tc_clip_gradients", &call_clip_gradients}};
PyObject *error_type = nullptr, *blocks_type = nullptr;              // TcError(code, where); Blocks(codes, scales, cols, square)
PyObject *rows_type = nullptr;                                       // Rows(codes, scales, cols)
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

// Checks of type, device and sides that all 4-d tensors have in common.
tc_tensor sides_of(const at::Tensor &x, int device)
{
    if (x.get_device() != device) throw Bad{"expected tensors on the context's device"};
    const auto type = x.scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) throw Bad{"dtype must be float32 or bfloat16"};
    for (int i = 0; i < 4; ++i)
        if (x.size(i) > INT32_MAX) throw Bad{"tensor sides must fit 32 bits"};
    return tc_tensor{x.data_ptr(), (int32_t)x.size(0), (int32_t)x.size(1), (int32_t)x.size(2), (int32_t)x.size(3), type == at::kFloat ? TC_F32 : TC_BF16};
}
tc_tensor map_of(const at::Tensor &x, int device)
{
    if (!x.is_cuda() || !x.is_contiguous() || x.dim() != 4) throw Bad{"expected a contiguous 4-d CUDA tensor (NCHW)"};
    return sides_of(x, device);
}
bool channels_last(const at::Tensor &x) { return x.dim() == 4 && x.is_contiguous(at::MemoryFormat::ChannelsLast); }
// The same of a tensor whose channels may be neighbours in memory: pixels of 1 x 1 then.
tc_tensor map_of_either(const at::Tensor &x, int device)
{
    if (x.is_cuda() && !x.is_contiguous() && channels_last(x)) {
        const tc_tensor t = sides_of(x, device);
        if ((int64_t)t.h * t.w > INT32_MAX || (int64_t)t.n * (t.h * t.w) > INT32_MAX) throw Bad{"a channels_last tensor's pixels must fit 32 bits"};
        return tc_tensor{t.data, t.n * t.h * t.w, t.c, 1, 1, t.dtype};
    }
    return map_of(x, device);
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
at::Tensor make(at::IntArrayRef sizes, at::ScalarType type, int device, bool last = false)
{
    return at::detail::empty_cuda(sizes, type, at::Device(at::kCUDA, (c10::DeviceIndex)device), last ? c10::optional<at::MemoryFormat>(at::MemoryFormat::ChannelsLast) : c10::nullopt);
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

// Rows: the same.
struct RowsRef {
    Ref object;
    tc_rows rows{};
};
RowsRef new_rows(int64_t rows, int64_t cols, int device)
{
    RowsRef r;
    if (rows > INT32_MAX || cols > INT32_MAX) throw Bad{"matrix of integers: rows and cols must fit 32 bits"};
    const int64_t ld = (cols + 15) / 16 * 16;
    const at::Tensor codes = make({rows, ld}, at::kChar, device), scales = make({rows}, at::kFloat, device);
    Ref c = wrap(codes), s = wrap(scales), n(PyLong_FromLongLong(cols));
    PyObject *const args[3] = {c.p, s.p, n.p};
    r.object = Ref(PyObject_Vectorcall(rows_type, args, 3, nullptr));
    r.rows = tc_rows{codes.data_ptr(), (float *)scales.data_ptr(), ld, (int32_t)rows, (int32_t)cols};
    return r;
}
tc_rows given_rows(PyObject *o, int device)
{
    Ref c(PyObject_GetAttr(o, name_codes)), s(PyObject_GetAttr(o, name_scales)), n(PyObject_GetAttr(o, name_cols));
    const at::Tensor &codes = tensor_of(c.p), &scales = tensor_of(s.p);
    const int64_t cols = PyLong_AsLongLong(n.p);
    if (PyErr_Occurred()) throw Raised{};
    if (!on_device(codes, device) || !on_device(scales, device) || codes.dim() != 2 || scales.dim() != 1 || codes.scalar_type() != at::kChar ||
        scales.scalar_type() != at::kFloat)
        throw Bad{"matrices of integers have contiguous int8 codes [rows, ld] and float32 scales [rows] on the context's device"};
    if (cols < 0 || cols > codes.size(1) || scales.size(0) != codes.size(0) || codes.size(0) > INT32_MAX || codes.size(1) > INT32_MAX)
        throw Bad{"matrix of integers: codes, scales and cols do not belong together"};
    return tc_rows{codes.data_ptr(), (float *)scales.data_ptr(), codes.size(1), (int32_t)codes.size(0), (int32_t)cols};
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

// A new tensor (N, O, H, W) for rows of the given number, by the caller's shape (N, H, W) or None and dtype.
at::Tensor make_output(PyObject *shape_arg, PyObject *dtype, int64_t rows, int64_t channels, bool last, int device)
{
    int64_t shape[3] = {rows, 1, 1};
    if (shape_arg != Py_None) {
        Ref s(PySequence_Tuple(shape_arg));
        if (PyTuple_GET_SIZE(s.p) != 3) throw Bad{"shape: expected (N, H, W)"};
        for (int i = 0; i < 3; ++i) shape[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(s.p, i));
        if (PyErr_Occurred()) throw Raised{};
    }
    const at::ScalarType type = THPDtype_Check(dtype) ? ((THPDtype *)dtype)->scalar_type : at::kInt;
    if (type != at::kFloat && type != at::kBFloat16) throw Bad{"dtype must be float32 or bfloat16"};
    for (const int64_t v : shape)
        if (v < 0 || v > INT32_MAX) throw Bad{"shape: expected (N, H, W)"};
    return make({shape[0], channels, shape[1], shape[2]}, type, device, last);
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
            made = wrap(make_output(a[2], a[3], ma.rows, mb.rows, false, c.device));
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

// x, rows, out
PyObject *quantize_rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 6, [](const Call &c, PyObject *const *a) -> PyObject * {
        const tc_tensor x = map_of_either(tensor_of(a[0]), c.device);
        const char *kind = PyUnicode_Check(a[1]) ? PyUnicode_AsUTF8(a[1]) : "";
        if (!kind) throw Raised{};
        const bool both = !strcmp(kind, "both"), pixels = both || !strcmp(kind, "pixels"), channels = both || !strcmp(kind, "channels");
        if (!pixels && !channels) throw Bad{"rows: \"pixels\", \"channels\" or \"both\""};
        PyObject *outs[2] = {a[2], a[2]};
        Ref pair;
        if (a[2] != Py_None && both) {
            pair = Ref(PySequence_Tuple(a[2]));
            if (PyTuple_GET_SIZE(pair.p) != 2) throw Bad{"out: Rows as this call returns them"};
            outs[0] = PyTuple_GET_ITEM(pair.p, 0);
            outs[1] = PyTuple_GET_ITEM(pair.p, 1);
        }
        RowsRef r[2];
        const int64_t p = pixels_of(x);
        for (int i = 0; i < 2; ++i) {
            if (!(i ? channels : pixels)) continue;
            if (a[2] == Py_None) r[i] = new_rows(i ? x.c : p, i ? p : x.c, c.device);
            else {
                r[i].rows = given_rows(outs[i], c.device);
                Py_INCREF(outs[i]);
                r[i].object = Ref(outs[i]);
            }
        }
        c.check(unlocked([&] { return call_quantize_rows(c.ctx, &x, pixels ? &r[0].rows : nullptr, channels ? &r[1].rows : nullptr, c.stream); }), "tc_quantize_rows");
        if (both) return PyTuple_Pack(2, r[0].object.p, r[1].object.p);
        return r[pixels ? 0 : 1].object.give();
    });
}

// a, b, shape, dtype, bias, relu, channels_last, out
PyObject *matmul_rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 11, [](const Call &c, PyObject *const *a) -> PyObject * {
        const tc_rows ma = given_rows(a[0], c.device), mb = given_rows(a[1], c.device);
        const int relu = PyObject_IsTrue(a[5]), last = PyObject_IsTrue(a[6]);
        if (relu < 0 || last < 0) throw Raised{};
        Ref made;
        PyObject *out = a[7];
        if (out == Py_None) {
            made = wrap(make_output(a[2], a[3], ma.rows, mb.rows, last, c.device));
            out = made.p;
        }
        const at::Tensor &to = tensor_of(out);
        const tc_tensor t = map_of_either(to, c.device);
        if (out != made.p && to.size(1) != mb.rows) throw Bad{"out: expected a tensor whose channels are b's rows"};
        const float *bias = vector(a[4], mb.rows, c.device, "bias");
        c.check(unlocked([&] { return call_matmul_rows(c.ctx, &ma, &mb, bias, relu, &t, c.stream); }), "tc_matmul_rows");
        Py_INCREF(out);
        return out;
    });
}

// A channels_last tensor, as the C structure names its sides.
tc_tensor last_map_of(const at::Tensor &x, int device)
{
    if (!x.is_cuda() || !channels_last(x)) throw Bad{"expected a 4-d CUDA tensor in channels_last order"};
    return sides_of(x, device);
}
// A channels_last tensor of the shape and type of `x`.
void *last_like(PyObject *o, const at::Tensor &x, int device, const char *name)
{
    const at::Tensor &t = tensor_of(o);
    if (!t.is_cuda() || t.get_device() != device || t.scalar_type() != x.scalar_type() || t.sizes() != x.sizes() || !channels_last(t))
        throw Bad{std::string(name) + ": expected a channels_last tensor of the shape and type of the first, on the context's device"};
    return t.numel() ? t.data_ptr() : (void *)16;
}
at::Tensor make_last(const at::Tensor &x) { return make(x.sizes(), x.scalar_type(), x.get_device(), true); }
float *stats_of(PyObject *o, int64_t n, int64_t groups, int device)
{
    const at::Tensor &t = tensor_of(o);
    if (!on_device(t, device) || t.scalar_type() != at::kFloat || t.dim() != 3 || t.size(0) != n || (groups >= 0 && t.size(1) != groups) || t.size(2) != 2 || t.size(1) > INT32_MAX)
        throw Bad{"stats: expected contiguous float32 values [N, groups, 2] on the context's device"};
    return t.numel() ? (float *)t.data_ptr() : (float *)16;
}
int activation_of(PyObject *o)
{
    if (o == Py_None) return TC_ACT_NONE;
    if (PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, "relu") == 0) return TC_ACT_RELU;
    if (PyUnicode_Check(o) && PyUnicode_CompareWithASCIIString(o, "silu") == 0) return TC_ACT_SILU;
    throw Bad{"activation: None, \"relu\" or \"silu\""};
}

// x, groups, weight, bias, eps, activation, codes, out, stats_out
PyObject *group_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 12, [](const Call &c, PyObject *const *a) -> PyObject * {
        const at::Tensor &x = tensor_of(a[0]);
        const tc_tensor t = last_map_of(x, c.device);
        const int64_t groups = PyLong_AsLongLong(a[1]);
        const double eps = PyFloat_AsDouble(a[4]);
        if (PyErr_Occurred()) throw Raised{};
        if (groups < 1 || t.c % groups) throw Bad{"groups: expected a divisor of the number of channels"};
        const tc_group_params p{(int32_t)groups, activation_of(a[5]), vector(a[2], t.c, c.device, "weight"), vector(a[3], t.c, c.device, "bias"), (float)eps};
        const bool both = PyUnicode_Check(a[6]) && PyUnicode_CompareWithASCIIString(a[6], "both") == 0;
        if (PyUnicode_Check(a[6]) && !both) throw Bad{"codes: False, True or \"both\""};
        const int codes = both || PyObject_IsTrue(a[6]);
        if (PyErr_Occurred()) throw Raised{};
        PyObject *out_y = a[7], *out_codes = a[7];
        Ref pair, y, result, stats;
        if (both && a[7] != Py_None) {
            pair = Ref(PySequence_Tuple(a[7]));
            if (PyTuple_GET_SIZE(pair.p) != 2) throw Bad{"out: a tensor and Rows as this call returns them"};
            out_y = PyTuple_GET_ITEM(pair.p, 0);
            out_codes = PyTuple_GET_ITEM(pair.p, 1);
        }
        void *at_y = nullptr;
        if (both || !codes) {
            if (out_y == Py_None) y = wrap(make_last(x));
            else { Py_INCREF(out_y); y = Ref(out_y); }
            at_y = last_like(y.p, x, c.device, "out");
        }
        RowsRef r;
        if (codes) {
            if (out_codes == Py_None) r = new_rows(pixels_of(t), t.c, c.device);
            else {
                r.rows = given_rows(out_codes, c.device);
                Py_INCREF(out_codes);
                r.object = Ref(out_codes);
            }
            result = both ? Ref(PyTuple_Pack(2, y.p, r.object.p)) : std::move(r.object);
        } else
            result = std::move(y);
        if (a[8] == Py_None) stats = wrap(make({t.n, groups, 2}, at::kFloat, c.device));
        else { Py_INCREF(a[8]); stats = Ref(a[8]); }
        float *const at_stats = stats_of(stats.p, t.n, groups, c.device);
        c.check(unlocked([&] { return call_group_norm(c.ctx, &t, &p, at_y, codes ? &r.rows : nullptr, at_stats, c.stream); }), "tc_group_norm");
        return PyTuple_Pack(2, result.p, stats.p);
    });
}

// x, dy, stats, weight, bias, activation: (x, weight, bias)
PyObject *group_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 9, [](const Call &c, PyObject *const *a) -> PyObject * {
        const at::Tensor &x = tensor_of(a[0]);
        const tc_tensor t = last_map_of(x, c.device);
        const void *const dy = last_like(a[1], x, c.device, "dy");
        const float *const stats = stats_of(a[2], t.n, -1, c.device);
        const int64_t groups = tensor_of(a[2]).size(1);
        if (groups < 1 || t.c % groups) throw Bad{"stats: as tc_group_norm returned them for these maps"};
        const tc_group_params p{(int32_t)groups, activation_of(a[5]), vector(a[3], t.c, c.device, "weight"), vector(a[4], t.c, c.device, "bias"), 0.f};
        Ref dx = wrap(make_last(x)), vectors[2];
        float *at[2] = {};
        for (int i = 0; i < 2; ++i) {
            if (a[3 + i] == Py_None) { vectors[i] = Ref(none()); continue; }
            const at::Tensor g = make({t.c}, at::kFloat, c.device);
            at[i] = (float *)g.data_ptr();
            vectors[i] = wrap(g);
        }
        void *const to = THPVariable_Unpack(dx.p).numel() ? THPVariable_Unpack(dx.p).data_ptr() : nullptr;
        c.check(unlocked([&] { return call_group_backward(c.ctx, &t, &p, stats, dy, to, at[0], at[1], c.stream); }), "tc_group_norm_backward");
        return PyTuple_Pack(3, dx.p, vectors[0].p, vectors[1].p);
    });
}

// tensors, max_norm or None (the norm alone), out, norm_out
PyObject *gradients(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded(args, n, 7, [](const Call &c, PyObject *const *a) -> PyObject * {
        const bool clip = a[1] != Py_None;
        const double max_norm = clip ? PyFloat_AsDouble(a[1]) : 0.0;
        Ref tensors(PySequence_Fast(a[0], "expected a list of tensors")), outs;
        if (a[2] != Py_None) outs = Ref(PySequence_Fast(a[2], "out: expected a list of tensors"));
        if (PyErr_Occurred()) throw Raised{};
        const Py_ssize_t count = PySequence_Fast_GET_SIZE(tensors.p);
        if (count > INT32_MAX || (outs.p && PySequence_Fast_GET_SIZE(outs.p) != count)) throw Bad{"out: expected as many tensors"};
        std::vector<tc_gradient> list((size_t)count);
        for (Py_ssize_t i = 0; i < count; ++i) {
            const at::Tensor &t = tensor_of(PySequence_Fast_GET_ITEM(tensors.p, i));
            if (!t.is_cuda() || t.get_device() != c.device) throw Bad{"expected tensors on the context's device"};
            if (t.scalar_type() != at::kFloat && t.scalar_type() != at::kBFloat16) throw Bad{"dtype must be float32 or bfloat16"};
            if (!t.is_non_overlapping_and_dense()) throw Bad{"expected tensors whose values lie one behind the other"};
            void *out = t.data_ptr();
            if (outs.p) {
                const at::Tensor &o = tensor_of(PySequence_Fast_GET_ITEM(outs.p, i));
                if (!o.is_cuda() || o.get_device() != c.device || o.scalar_type() != t.scalar_type() || o.sizes() != t.sizes() || o.strides() != t.strides())
                    throw Bad{"out: expected tensors of the shapes, strides and types of the first, on the context's device"};
                out = o.data_ptr();
            }
            list[i] = tc_gradient{t.data_ptr(), out, t.numel(), t.scalar_type() == at::kFloat ? TC_F32 : TC_BF16};
        }
        Ref norm;
        if (a[3] == Py_None) norm = wrap(make({1}, at::kFloat, c.device));
        else { Py_INCREF(a[3]); norm = Ref(a[3]); }
        float *const at = vector(norm.p, 1, c.device, "norm_out");
        c.check(unlocked([&] {
                    return clip ? call_clip_gradients(c.ctx, list.data(), (int32_t)count, (float)max_norm, at, c.stream) : call_gradient_norm(c.ctx, list.data(), (int32_t)count, at, c.stream);
                }),
                clip ? "tc_clip_gradients" : "tc_gradient_norm");
        return norm.give();
    });
}

// addresses of the entry points by name, TcError, Blocks, Rows
PyObject *init(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 4 || !PyDict_Check(args[0])) { PyErr_SetString(PyExc_ValueError, "wrong arguments"); return nullptr; }
    for (const EntryPoint &e : entry_points) {
        PyObject *const at = PyDict_GetItemString(args[0], e.name);
        if (!at) { PyErr_SetString(PyExc_ValueError, e.name); return nullptr; }
        *(void **)e.at = PyLong_AsVoidPtr(at);
    }
    for (int i = 1; i < 4; ++i) Py_INCREF(args[i]);
    error_type = args[1];
    blocks_type = args[2];
    rows_type = args[3];
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
                         {"quantize_rows", (PyCFunction)(void *)quantize_rows, METH_FASTCALL, nullptr},
                         {"matmul_rows", (PyCFunction)(void *)matmul_rows, METH_FASTCALL, nullptr},
                         {"group_norm", (PyCFunction)(void *)group_norm, METH_FASTCALL, nullptr},
                         {"gradients", (PyCFunction)(void *)gradients, METH_FASTCALL, nullptr},
                         {"group_backward", (PyCFunction)(void *)group_backward, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layers", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layers(void)
{
    PyObject *const m = PyModule_Create(&module), *const names = PyTuple_New(sizeof entry_points / sizeof *entry_points);
    for (size_t i = 0; names && i < sizeof entry_points / sizeof *entry_points; ++i) PyTuple_SET_ITEM(names, i, PyUnicode_FromString(entry_points[i].name));
    if (!m || !names || PyErr_Occurred() || PyModule_AddObject(m, "entry_points", names) < 0) { Py_XDECREF(names); Py_XDECREF(m); return nullptr; }
    return m;
}
