// The argument marshalling of binding.py's calls in native code: a CPython module whose Calls objects hold the
// entry points of one loaded libquest.so and call them with the pointers, sizes and strides of torch tensors.
//
// A call from Python through ctypes spends 2.5 to 3 us of its 5 on reading tensors' attributes one by one and converting
// the arguments, more than the launch itself; here both take 0.3 us.  Only the ordinary call is taken: exact tensors
// (no subclass, no active torch-function mode), plain Python numbers in the range of their C type,
// sizes of the expected rank.  For anything else a method returns None, nothing having been called, and binding.py goes the
// general way, which also is the one that raises for what is wrong.
#include <Python.h>

#include <string.h>

#include <initializer_list>
#include <limits>

#include <ATen/PythonTorchFunctionTLS.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/quest.h"

namespace {

struct Entries {
    decltype(&quest_hadamard_quantize) quantize;
    decltype(&quest_hadamard_quantize_pair) quantize_pair;
    decltype(&quest_hadamard_quantize_fp4) quantize_fp4;
    decltype(&quest_hadamard_quantize_fp4_pair) quantize_fp4_pair;
    decltype(&quest_lowbit_gemm) lowbit_gemm;
    decltype(&quest_lowbit_gemm_fp4) lowbit_gemm_fp4;
    decltype(&quest_trust_backward) trust_backward;
    decltype(&quest_trust_backward_pair) trust_backward_pair;
    decltype(&quest_grad_gemm) grad_gemm;
    decltype(&quest_grad_gemm_fp4) grad_gemm_fp4;
    decltype(&quest_weight_only_gemm) weight_only_gemm;
};
constexpr Py_ssize_t kEntries = sizeof(Entries) / sizeof(void *);

struct Calls {
    PyObject_HEAD
    Entries entry;
};

// Reads the arguments one after another; `plain` stays true while each is what the quick way takes.
class Reader {
public:
    Reader(PyObject *const *args, Py_ssize_t count, Py_ssize_t expected) : args_(args), plain(count == expected) {}

    int64_t integer(int64_t low, int64_t high)
    {
        PyObject *o = next();
        if (!plain || !PyLong_CheckExact(o))
            return refuse();
        int overflow = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
        return overflow || v < low || v > high ? refuse() : v;
    }
    int32_t i32() { return (int32_t)integer(std::numeric_limits<int32_t>::min(), std::numeric_limits<int32_t>::max()); }
    int64_t i64() { return integer(std::numeric_limits<int64_t>::min(), std::numeric_limits<int64_t>::max()); }
    float f32()
    {
        PyObject *o = next();
        if (!plain || !PyFloat_CheckExact(o)) {
            refuse();
            return 0.0f;
        }
        return (float)PyFloat_AS_DOUBLE(o);
    }
    const at::Tensor *tensor()
    {
        PyObject *o = next();
        if (!plain || !THPVariable_CheckExact(o) || at::impl::torch_function_mode_enabled()) {
            refuse();
            return nullptr;
        }
        return &THPVariable_Unpack(o);
    }
    // a tensor of two dimensions, the second one contiguous or not (the entry points take row pitches only)
    const at::Tensor *matrix()
    {
        const at::Tensor *t = tensor();
        if (t && t->dim() != 2) {
            refuse();
            return nullptr;
        }
        return t;
    }
    const at::Tensor *tensor_or_none()
    {
        if (plain && args_[at_] == Py_None) {
            ++at_;
            return nullptr;
        }
        return tensor();
    }
    quest_dtype dtype(const at::Tensor *t)
    {
        if (t && t->scalar_type() == at::kBFloat16)
            return QUEST_BF16;
        if (!t || t->scalar_type() != at::kFloat)
            refuse();
        return QUEST_F32;
    }
    int64_t size(const at::Tensor *t, int64_t dim) { return t && dim < t->dim() ? t->size(dim) : refuse(); }
    int64_t stride(const at::Tensor *t, int64_t dim) { return t && dim < t->dim() ? t->stride(dim) : refuse(); }
    PyObject *object() { return next(); }
    void require(bool condition)
    {
        if (!condition)
            refuse();
    }

private:
    PyObject *next() { return plain ? args_[at_++] : nullptr; }
    int64_t refuse()
    {
        plain = false;
        return 0;
    }

    PyObject *const *args_;
    Py_ssize_t at_ = 0;

public:
    bool plain;
};

template <typename T = uint8_t>
T *pointer(const at::Tensor *t)
{
    return t ? static_cast<T *>(t->data_ptr()) : nullptr;
}

int64_t bytes(const at::Tensor *t)
{
    return t ? t->numel() * t->element_size() : 0;
}

// The call itself on the stream that `ask_stream` returns the handle of, without the interpreter lock; its status as a number
template <typename Call>
PyObject *enqueue(PyObject *ask_stream, Call &&call)
{
    PyObject *handle = PyObject_CallNoArgs(ask_stream);
    if (!handle)
        return nullptr;
    void *stream = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (!stream && PyErr_Occurred())
        return nullptr;
    quest_status status;
    Py_BEGIN_ALLOW_THREADS
    status = call(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

#define QUEST_ENTRY()                                              \
    const Entries &entry = reinterpret_cast<Calls *>(self)->entry; \
    HANDLE_TH_ERRORS
#define QUEST_PLAIN_OR_NONE(READER) \
    if (!(READER).plain)            \
        Py_RETURN_NONE;

// Arguments of the methods in brackets; `stream`: a callable that returns the stream's handle
// (x, had_block, bits, alpha, outer_trust, codes, scales, mask, xh_out, stream)
PyObject *hadamard_quantize(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_ENTRY()
    Reader r(args, count, 10);
    const at::Tensor *x = r.matrix();
    const int32_t block = r.i32(), bits = r.i32();
    const float alpha = r.f32(), outer = r.f32();
    const at::Tensor *codes = r.tensor(), *scales = r.tensor(), *mask = r.tensor_or_none(), *xh = r.tensor_or_none();
    PyObject *ask_stream = r.object();
    const quest_dtype dtype = r.dtype(x);
    QUEST_PLAIN_OR_NONE(r)
    void *px = pointer(x);
    uint8_t *pc = pointer(codes), *pm = pointer(mask);
    float *ps = pointer<float>(scales), *ph = pointer<float>(xh);
    const int64_t rows = x->size(0), cols = x->size(1), ld = x->stride(0);
    return enqueue(ask_stream, [&](void *stream) { return entry.quantize(px, dtype, rows, cols, ld, block, bits, alpha, outer, pc, ps, pm, ph, stream); });
    END_HANDLE_TH_ERRORS
}

// (x, had_block, alpha, codes, scales, mask, xh_out, stream)
PyObject *hadamard_quantize_fp4(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_ENTRY()
    Reader r(args, count, 8);
    const at::Tensor *x = r.matrix();
    const int32_t block = r.i32();
    const float alpha = r.f32();
    const at::Tensor *codes = r.tensor(), *scales = r.tensor(), *mask = r.tensor_or_none(), *xh = r.tensor_or_none();
    PyObject *ask_stream = r.object();
    const quest_dtype dtype = r.dtype(x);
    QUEST_PLAIN_OR_NONE(r)
    void *px = pointer(x);
    uint8_t *pc = pointer(codes), *pm = pointer(mask);
    float *ps = pointer<float>(scales), *ph = pointer<float>(xh);
    const int64_t rows = x->size(0), cols = x->size(1), ld = x->stride(0);
    return enqueue(ask_stream, [&](void *stream) { return entry.quantize_fp4(px, dtype, rows, cols, ld, block, alpha, pc, ps, pm, ph, stream); });
    END_HANDLE_TH_ERRORS
}

// (x, w, had_block, bits, alpha, outer_trust, x_codes, x_scales, x_mask, w_codes, w_scales, w_mask, stream); with E2M1 without
// bits and outer_trust
template <bool FP4>
PyObject *hadamard_quantize_pair(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_ENTRY()
    Reader r(args, count, FP4 ? 11 : 13);
    const at::Tensor *x = r.matrix(), *w = r.matrix();
    const int32_t block = r.i32(), bits = FP4 ? 4 : r.i32();
    const float alpha = r.f32(), outer = FP4 ? -1.0f : r.f32();
    const at::Tensor *x_codes = r.tensor(), *x_scales = r.tensor(), *x_mask = r.tensor_or_none();
    const at::Tensor *w_codes = r.tensor(), *w_scales = r.tensor(), *w_mask = r.tensor_or_none();
    PyObject *ask_stream = r.object();
    const quest_dtype dtype = r.dtype(x);
    r.require(r.plain && x->size(1) == w->size(1) && x->scalar_type() == w->scalar_type());
    QUEST_PLAIN_OR_NONE(r)
    void *px = pointer(x), *pw = pointer(w);
    uint8_t *xc = pointer(x_codes), *xm = pointer(x_mask), *wc = pointer(w_codes), *wm = pointer(w_mask);
    float *xs = pointer<float>(x_scales), *ws = pointer<float>(w_scales);
    const int64_t cols = x->size(1), rows_x = x->size(0), rows_w = w->size(0), ld_x = x->stride(0), ld_w = w->stride(0);
    return enqueue(ask_stream, [&](void *stream) {
        return FP4 ? entry.quantize_fp4_pair(px, rows_x, ld_x, xc, xs, xm, pw, rows_w, ld_w, wc, ws, wm, dtype, cols, block,
                                             alpha, stream)
                   : entry.quantize_pair(px, rows_x, ld_x, xc, xs, xm, pw, rows_w, ld_w, wc, ws, wm, dtype, cols, block, bits,
                                         alpha, outer, stream);
    });
    END_HANDLE_TH_ERRORS
}

// (a_codes, a_scales, b_codes, b_scales, K, bits, y, acc_out, workspace, stream)
PyObject *lowbit_gemm(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_ENTRY()
    Reader r(args, count, 10);
    const at::Tensor *a = r.tensor(), *a_scales = r.tensor(), *b = r.tensor(), *b_scales = r.tensor();
    const int64_t K = r.i64();
    const int32_t bits = r.i32();
    const at::Tensor *y = r.tensor_or_none(), *acc = r.tensor_or_none(), *workspace = r.tensor_or_none();
    PyObject *ask_stream = r.object();
    const int64_t M = r.size(a, 0), N = r.size(b, 0), ld_y = y ? r.stride(y, 0) : N;
    QUEST_PLAIN_OR_NONE(r)
    uint8_t *pa = pointer(a), *pb = pointer(b);
    float *sa = pointer<float>(a_scales), *sb = pointer<float>(b_scales);
    void *py = pointer(y), *pws = pointer(workspace);
    int32_t *pacc = pointer<int32_t>(acc);
    const int64_t scratch = bytes(workspace);
    return enqueue(ask_stream, [&](void *stream) { return entry.lowbit_gemm(pa, sa, M, pb, sb, N, K, bits, py, ld_y, pacc, pws, scratch, stream); });
    END_HANDLE_TH_ERRORS
}

// (a_codes, a_scales, b_codes, b_scales, K, y, acc_out, stream)
PyObject *lowbit_gemm_fp4(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_ENTRY()
    Reader r(args, count, 8);
    const at::Tensor *a = r.tensor(), *a_scales = r.tensor(), *b = r.tensor(), *b_scales = r.tensor();
    const int64_t K = r.i64();
    const at::Tensor *y = r.tensor_or_none(), *acc = r.tensor_or_none();
    PyObject *ask_stream = r.object();
    const int64_t M = r.size(a, 0), N = r.size(b, 0), ld_y = y ? r.stride(y, 0) : N;
    QUEST_PLAIN_OR_NONE(r)
    uint8_t *pa = pointer(a), *pb = pointer(b);
    float *sa = pointer<float>(a_scales), *sb = pointer<float>(b_scales), *pacc = pointer<float>(acc);
    void *py = pointer(y);
    return enqueue(ask_stream, [&](void *stream) { return entry.lowbit_gemm_fp4(pa, sa, M, pb, sb, N, K, py, ld_y, pacc, stream); });
    END_HANDLE_TH_ERRORS
}

// (g, mask, had_block, out, stream)
PyObject *trust_backward(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_ENTRY()
    Reader r(args, count, 5);
    const at::Tensor *g = r.matrix(), *mask = r.tensor_or_none();
    const int32_t block = r.i32();
    const at::Tensor *out = r.tensor();
    PyObject *ask_stream = r.object();
    const quest_dtype g_dtype = r.dtype(g), out_dtype = r.dtype(out);
    QUEST_PLAIN_OR_NONE(r)
    void *pg = pointer(g), *po = pointer(out);
    uint8_t *pm = pointer(mask);
    const int64_t rows = g->size(0), cols = g->size(1);
    return enqueue(ask_stream, [&](void *stream) { return entry.trust_backward(pg, g_dtype, pm, rows, cols, block, po, out_dtype, stream); });
    END_HANDLE_TH_ERRORS
}

// (g_x, mask_x, g_w, mask_w, had_block, out_x, out_w, stream)
PyObject *trust_backward_pair(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_ENTRY()
    Reader r(args, count, 8);
    const at::Tensor *gx = r.matrix(), *mask_x = r.tensor_or_none(), *gw = r.matrix(), *mask_w = r.tensor_or_none();
    const int32_t block = r.i32();
    const at::Tensor *out_x = r.tensor(), *out_w = r.tensor();
    PyObject *ask_stream = r.object();
    const quest_dtype g_dtype = r.dtype(gx), out_dtype = r.dtype(out_x);
    r.require(r.plain && gx->size(1) == gw->size(1) && gx->scalar_type() == gw->scalar_type() &&
              out_x->scalar_type() == out_w->scalar_type());
    QUEST_PLAIN_OR_NONE(r)
    void *px = pointer(gx), *pw = pointer(gw), *ox = pointer(out_x), *ow = pointer(out_w);
    uint8_t *mx = pointer(mask_x), *mw = pointer(mask_w);
    const int64_t rows_x = gx->size(0), rows_w = gw->size(0), cols = gx->size(1);
    return enqueue(ask_stream, [&](void *stream) {
        return entry.trust_backward_pair(px, mx, rows_x, ox, pw, mw, rows_w, ow, g_dtype, cols, block, out_dtype, stream);
    });
    END_HANDLE_TH_ERRORS
}

// (which, dy, q_codes, q_scales, bits, M, N, K, out, workspace, stream); with E2M1 without bits
template <bool FP4>
PyObject *grad_gemm(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_ENTRY()
    Reader r(args, count, FP4 ? 10 : 11);
    const int32_t which = r.i32();
    const at::Tensor *dy = r.tensor(), *codes = r.tensor(), *scales = r.tensor();
    const int32_t bits = FP4 ? 4 : r.i32();
    const int64_t M = r.i64(), N = r.i64(), K = r.i64();
    const at::Tensor *out = r.tensor(), *workspace = r.tensor_or_none();
    PyObject *ask_stream = r.object();
    QUEST_PLAIN_OR_NONE(r)
    void *pdy = pointer(dy), *po = pointer(out), *pws = pointer(workspace);
    uint8_t *pc = pointer(codes);
    float *ps = pointer<float>(scales);
    const int64_t scratch = bytes(workspace);
    return enqueue(ask_stream, [&](void *stream) {
        return FP4 ? entry.grad_gemm_fp4(which, pdy, pc, ps, M, N, K, po, pws, scratch, stream)
                   : entry.grad_gemm(which, pdy, pc, ps, bits, M, N, K, po, pws, scratch, stream);
    });
    END_HANDLE_TH_ERRORS
}

// (x, w_codes, w_scales, bits, y, workspace, stream)
PyObject *weight_only_gemm(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_ENTRY()
    Reader r(args, count, 7);
    const at::Tensor *x = r.matrix(), *codes = r.tensor(), *scales = r.tensor();
    const int32_t bits = r.i32();
    const at::Tensor *y = r.tensor(), *workspace = r.tensor_or_none();
    PyObject *ask_stream = r.object();
    const int64_t N = r.size(codes, 0);
    QUEST_PLAIN_OR_NONE(r)
    void *px = pointer(x), *py = pointer(y), *pws = pointer(workspace);
    uint8_t *pc = pointer(codes);
    float *ps = pointer<float>(scales);
    const int64_t M = x->size(0), K = x->size(1), scratch = bytes(workspace);
    return enqueue(ask_stream, [&](void *stream) { return entry.weight_only_gemm(px, pc, ps, bits, M, N, K, py, pws, scratch, stream); });
    END_HANDLE_TH_ERRORS
}

// ---- the calls on microscaled operands and of the norm.  binding.py checks shapes, types, strides and places of all tensors of
// these; here a call is plain if it passes the same checks.

struct MxEntries {
    decltype(&quest_hadamard_quantize_mx) quantize;
    decltype(&quest_dequantize_mx) dequantize;
    decltype(&quest_lowbit_gemm_mx) gemm;
    decltype(&quest_grad_gemm_mx) grad_gemm;
    decltype(&quest_rms_norm_mx) rms_norm;
    decltype(&quest_rms_norm_backward) rms_norm_backward;
};
constexpr Py_ssize_t kMxEntries = sizeof(MxEntries) / sizeof(void *);

struct MxCalls {
    PyObject_HEAD
    MxEntries entry;
};

// Reader with those checks; `device` of the methods' arguments: a callable that returns the current device's number
class MxReader : public Reader {
public:
    MxReader(PyObject *const *args, Py_ssize_t count, Py_ssize_t expected) : Reader(args, count, expected) {}

    quest_mx_format format()
    {
        const int32_t f = i32();
        require(f == QUEST_MX_E2M1 || f == QUEST_MX_E4M3);
        return (quest_mx_format)f;
    }
    // a matrix whose rows are contiguous; its row stride
    int64_t rows_of(const at::Tensor *t, int64_t rows, int64_t cols)
    {
        require(plain && t && t->dim() == 2 && t->size(0) == rows && t->size(1) == cols && (cols == 1 || t->stride(1) == 1));
        return !plain ? 0 : rows > 1 ? t->stride(0) : cols;
    }
    void packed(const at::Tensor *t, at::ScalarType type, int64_t rows, int64_t cols)
    {
        require(plain && (!t || (t->dim() == 2 && t->scalar_type() == type && t->size(0) == rows && t->size(1) == cols && t->is_contiguous())));
    }
    void packed(const at::Tensor *t, at::ScalarType type, int64_t count)
    {
        require(plain && (!t || (t->dim() == 1 && t->scalar_type() == type && t->size(0) == count && t->is_contiguous())));
    }
    void operand(const at::Tensor *codes, const at::Tensor *scales, const at::Tensor *mask, quest_mx_format format, int64_t rows,
                 int64_t cols)
    {
        packed(codes, at::kByte, rows, format == QUEST_MX_E4M3 ? cols : cols / 2);
        packed(scales, at::kByte, rows, cols / QUEST_MX_GROUP);
        packed(mask, at::kByte, rows, cols / 8);
    }
    // its size is taken to be its memory's
    void scratch(const at::Tensor *t) { require(plain && (!t || t->is_contiguous())); }
    // Whether all tensors are on the device whose number `ask_device` returns (tensors in host memory have the number -1)
    void on_device(PyObject *ask_device, std::initializer_list<const at::Tensor *> tensors)
    {
        if (!plain)
            return;
        PyObject *number = PyObject_CallNoArgs(ask_device);
        const long device = number ? PyLong_AsLong(number) : -1;
        Py_XDECREF(number);
        if (PyErr_Occurred()) {
            PyErr_Clear();   // binding.py asks again, and raises
            require(false);
        }
        for (const at::Tensor *t : tensors)
            require(!t || t->get_device() == device);
    }
};

#define QUEST_MX_ENTRY()                                               \
    const MxEntries &entry = reinterpret_cast<MxCalls *>(self)->entry; \
    HANDLE_TH_ERRORS

// (x, had_block, format, codes, scales, mask, stream, device)
PyObject *mx_quantize(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_MX_ENTRY()
    MxReader r(args, count, 8);
    const at::Tensor *x = r.matrix();
    const int32_t block = r.i32();
    const quest_mx_format format = r.format();
    const at::Tensor *codes = r.tensor(), *scales = r.tensor(), *mask = r.tensor_or_none();
    PyObject *ask_stream = r.object(), *ask_device = r.object();
    const quest_dtype dtype = r.dtype(x);
    const int64_t rows = r.size(x, 0), cols = r.size(x, 1), ld = r.rows_of(x, rows, cols);
    r.operand(codes, scales, mask, format, rows, cols);
    r.on_device(ask_device, {x, codes, scales, mask});
    QUEST_PLAIN_OR_NONE(r)
    void *px = pointer(x);
    uint8_t *pc = pointer(codes), *ps = pointer(scales), *pm = pointer(mask);
    return enqueue(ask_stream, [&](void *stream) { return entry.quantize(px, dtype, rows, cols, ld, block, format, pc, ps, pm, stream); });
    END_HANDLE_TH_ERRORS
}

// (codes, scales, format, out, stream, device)
PyObject *mx_dequantize(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_MX_ENTRY()
    MxReader r(args, count, 6);
    const at::Tensor *codes = r.tensor(), *scales = r.tensor();
    const quest_mx_format format = r.format();
    const at::Tensor *out = r.matrix();
    PyObject *ask_stream = r.object(), *ask_device = r.object();
    const quest_dtype dtype = r.dtype(out);
    const int64_t rows = r.size(out, 0), cols = r.size(out, 1), ld = r.rows_of(out, rows, cols);
    r.operand(codes, scales, nullptr, format, rows, cols);
    r.on_device(ask_device, {codes, scales, out});
    QUEST_PLAIN_OR_NONE(r)
    uint8_t *pc = pointer(codes), *ps = pointer(scales);
    void *po = pointer(out);
    return enqueue(ask_stream, [&](void *stream) { return entry.dequantize(pc, ps, format, rows, cols, po, dtype, ld, stream); });
    END_HANDLE_TH_ERRORS
}

// (a_codes, a_scales, a_format, b_codes, b_scales, K, y, acc_out, stream, device)
PyObject *mx_gemm(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_MX_ENTRY()
    MxReader r(args, count, 10);
    const at::Tensor *a = r.tensor(), *a_scales = r.tensor();
    const quest_mx_format format = r.format();
    const at::Tensor *b = r.tensor(), *b_scales = r.tensor();
    const int64_t K = r.i64();
    const at::Tensor *y = r.tensor_or_none(), *acc = r.tensor_or_none();
    PyObject *ask_stream = r.object(), *ask_device = r.object();
    const int64_t M = r.size(a, 0), N = r.size(b, 0);
    r.operand(a, a_scales, nullptr, format, M, K);
    r.operand(b, b_scales, nullptr, QUEST_MX_E2M1, N, K);
    r.require(!y || y->scalar_type() == at::kBFloat16);
    const int64_t ld_y = y ? r.rows_of(y, M, N) : N;
    r.packed(acc, at::kFloat, M, N);
    r.on_device(ask_device, {a, a_scales, b, b_scales, y, acc});
    QUEST_PLAIN_OR_NONE(r)
    uint8_t *pa = pointer(a), *sa = pointer(a_scales), *pb = pointer(b), *sb = pointer(b_scales);
    void *py = pointer(y);
    float *pacc = pointer<float>(acc);
    return enqueue(ask_stream, [&](void *stream) { return entry.gemm(pa, sa, format, M, pb, sb, N, K, py, ld_y, pacc, stream); });
    END_HANDLE_TH_ERRORS
}

// (which, dy, q_codes, q_scales, format, M, N, K, out, workspace, stream, device)
PyObject *mx_grad_gemm(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_MX_ENTRY()
    MxReader r(args, count, 12);
    const int32_t which = r.i32();
    const at::Tensor *dy = r.tensor(), *codes = r.tensor(), *scales = r.tensor();
    const quest_mx_format format = r.format();
    const int64_t M = r.i64(), N = r.i64(), K = r.i64();
    const at::Tensor *out = r.tensor(), *workspace = r.tensor_or_none();
    PyObject *ask_stream = r.object(), *ask_device = r.object();
    r.packed(dy, at::kBFloat16, M, N);
    r.operand(codes, scales, nullptr, format, which == 1 ? M : N, K);
    r.packed(out, at::kBFloat16, which == 1 ? N : M, K);
    r.scratch(workspace);
    r.on_device(ask_device, {dy, codes, scales, out, workspace});
    QUEST_PLAIN_OR_NONE(r)
    void *pdy = pointer(dy), *po = pointer(out), *pws = pointer(workspace);
    uint8_t *pc = pointer(codes), *ps = pointer(scales);
    const int64_t scratch = bytes(workspace);
    return enqueue(ask_stream, [&](void *stream) { return entry.grad_gemm(which, pdy, pc, ps, format, M, N, K, po, pws, scratch, stream); });
    END_HANDLE_TH_ERRORS
}

// (x, weight, eps, had_block, format, codes, scales, mask, residual, h_out, y_out, rstd, stream, device)
PyObject *mx_rms_norm(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_MX_ENTRY()
    MxReader r(args, count, 14);
    const at::Tensor *x = r.matrix(), *weight = r.tensor();
    const float eps = r.f32();
    const int32_t block = r.i32(), asked = r.i32();   // (both are looked at where there are codes)
    const at::Tensor *codes = r.tensor_or_none(), *scales = r.tensor_or_none(), *mask = r.tensor_or_none();
    const at::Tensor *residual = r.tensor_or_none(), *h = r.tensor_or_none(), *y = r.tensor_or_none(), *rstd = r.tensor_or_none();
    PyObject *ask_stream = r.object(), *ask_device = r.object();
    const quest_dtype dtype = r.dtype(x), weight_dtype = r.dtype(weight);
    const int64_t rows = r.size(x, 0), cols = r.size(x, 1), ld_x = r.rows_of(x, rows, cols);
    r.require(r.plain && (!residual || residual->scalar_type() == x->scalar_type()));
    const int64_t ld_residual = residual ? r.rows_of(residual, rows, cols) : 0;
    r.require(!codes || asked == QUEST_MX_E2M1 || asked == QUEST_MX_E4M3);
    const quest_mx_format format = (quest_mx_format)asked;
    r.operand(codes, scales, mask, format, rows, cols);
    if (r.plain) {
        r.packed(weight, weight->scalar_type(), cols);
        r.packed(h, x->scalar_type(), rows, cols);
        r.packed(y, x->scalar_type(), rows, cols);
        r.packed(rstd, at::kFloat, rows);
    }
    r.on_device(ask_device, {x, weight, codes, scales, mask, residual, h, y, rstd});
    QUEST_PLAIN_OR_NONE(r)
    void *px = pointer(x), *pr = pointer(residual), *pw = pointer(weight), *ph = pointer(h), *py = pointer(y);
    uint8_t *pc = pointer(codes), *ps = pointer(scales), *pm = pointer(mask);
    float *pt = pointer<float>(rstd);
    return enqueue(ask_stream, [&](void *stream) {
        return entry.rms_norm(px, ld_x, pr, ld_residual, dtype, pw, weight_dtype, rows, cols, eps, ph, py, block, format, pc, ps, pm, pt,
                              stream);
    });
    END_HANDLE_TH_ERRORS
}

// (dy, h, weight, rstd, dh, dx, dweight, workspace, stream, device)
PyObject *mx_rms_norm_backward(PyObject *self, PyObject *const *args, Py_ssize_t count)
{
    QUEST_MX_ENTRY()
    MxReader r(args, count, 10);
    const at::Tensor *dy = r.matrix(), *h = r.matrix(), *weight = r.tensor(), *rstd = r.tensor(), *dh = r.tensor_or_none();
    const at::Tensor *dx = r.tensor(), *dweight = r.tensor_or_none(), *workspace = r.tensor_or_none();
    PyObject *ask_stream = r.object(), *ask_device = r.object();
    const quest_dtype dtype = r.dtype(h), weight_dtype = r.dtype(weight);
    const int64_t rows = r.size(h, 0), cols = r.size(h, 1);
    if (r.plain) {
        for (const at::Tensor *t : {h, dy, dh, dx})
            r.packed(t, h->scalar_type(), rows, cols);
        r.packed(weight, weight->scalar_type(), cols);
        r.packed(rstd, at::kFloat, rows);
        r.packed(dweight, at::kFloat, cols);
    }
    r.scratch(workspace);
    r.on_device(ask_device, {dy, h, weight, rstd, dh, dx, dweight, workspace});
    QUEST_PLAIN_OR_NONE(r)
    void *pdy = pointer(dy), *ph = pointer(h), *pw = pointer(weight), *pdh = pointer(dh), *pdx = pointer(dx), *pws = pointer(workspace);
    float *pt = pointer<float>(rstd), *pdw = pointer<float>(dweight);
    const int64_t scratch = bytes(workspace);
    return enqueue(ask_stream, [&](void *stream) {
        return entry.rms_norm_backward(pdy, ph, dtype, pw, weight_dtype, pt, pdh, rows, cols, pdx, pdw, pws, scratch, stream);
    });
    END_HANDLE_TH_ERRORS
}

#undef QUEST_ENTRY
#undef QUEST_MX_ENTRY
#undef QUEST_PLAIN_OR_NONE

// Object(addresses of the entry points in the order of Table)
template <typename Object, typename Table, Py_ssize_t COUNT>
PyObject *new_calls(PyTypeObject *type, PyObject *args, PyObject *)
{
    if (PyTuple_GET_SIZE(args) != COUNT) {
        PyErr_SetString(PyExc_TypeError, "one address for each entry point");
        return nullptr;
    }
    auto *self = reinterpret_cast<Object *>(type->tp_alloc(type, 0));
    if (!self)
        return nullptr;
    void *address[COUNT];
    for (Py_ssize_t i = 0; i < COUNT; ++i) {
        address[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args, i));
        if (!address[i]) {
            if (!PyErr_Occurred())
                PyErr_SetString(PyExc_ValueError, "null entry point");
            Py_DECREF(self);
            return nullptr;
        }
    }
    memcpy(&self->entry, address, sizeof(Table));
    return reinterpret_cast<PyObject *>(self);
}

#define QUEST_METHOD(NAME, FUNCTION) {NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(FUNCTION)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {QUEST_METHOD("hadamard_quantize", hadamard_quantize),
                         QUEST_METHOD("hadamard_quantize_pair", hadamard_quantize_pair<false>),
                         QUEST_METHOD("hadamard_quantize_fp4", hadamard_quantize_fp4),
                         QUEST_METHOD("hadamard_quantize_fp4_pair", hadamard_quantize_pair<true>),
                         QUEST_METHOD("lowbit_gemm", lowbit_gemm),
                         QUEST_METHOD("lowbit_gemm_fp4", lowbit_gemm_fp4),
                         QUEST_METHOD("trust_backward", trust_backward),
                         QUEST_METHOD("trust_backward_pair", trust_backward_pair),
                         QUEST_METHOD("grad_gemm", grad_gemm<false>),
                         QUEST_METHOD("grad_gemm_fp4", grad_gemm<true>),
                         QUEST_METHOD("weight_only_gemm", weight_only_gemm),
                         {nullptr, nullptr, 0, nullptr}};
PyMethodDef mx_methods[] = {QUEST_METHOD("hadamard_quantize_mx", mx_quantize),
                            QUEST_METHOD("dequantize_mx", mx_dequantize),
                            QUEST_METHOD("lowbit_gemm_mx", mx_gemm),
                            QUEST_METHOD("grad_gemm_mx", mx_grad_gemm),
                            QUEST_METHOD("rms_norm_mx", mx_rms_norm),
                            QUEST_METHOD("rms_norm_backward", mx_rms_norm_backward),
                            {nullptr, nullptr, 0, nullptr}};
#undef QUEST_METHOD

PyTypeObject calls_type = {PyVarObject_HEAD_INIT(nullptr, 0) "quest_python.Calls", sizeof(Calls)};
PyTypeObject mx_calls_type = {PyVarObject_HEAD_INIT(nullptr, 0) "quest_python.MxCalls", sizeof(MxCalls)};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "quest_python", nullptr, -1, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_quest_python(void)
{
    calls_type.tp_flags = mx_calls_type.tp_flags = Py_TPFLAGS_DEFAULT;
    calls_type.tp_methods = methods;
    calls_type.tp_new = new_calls<Calls, Entries, kEntries>;
    mx_calls_type.tp_methods = mx_methods;
    mx_calls_type.tp_new = new_calls<MxCalls, MxEntries, kMxEntries>;
    if (PyType_Ready(&calls_type) < 0 || PyType_Ready(&mx_calls_type) < 0)
        return nullptr;
    PyObject *m = PyModule_Create(&module);
    if (!m)
        return nullptr;
    if (PyModule_AddStringConstant(m, "TORCH_BUILD", QUEST_TORCH_BUILD) < 0) {   // binding.py compares it
        Py_DECREF(m);
        return nullptr;
    }
    const struct {
        const char *name;
        PyTypeObject *type;
    } types[] = {{"Calls", &calls_type}, {"MxCalls", &mx_calls_type}};
    for (const auto &t : types) {
        Py_INCREF(t.type);
        if (PyModule_AddObject(m, t.name, reinterpret_cast<PyObject *>(t.type)) < 0) {
            Py_DECREF(t.type);
            Py_DECREF(m);
            return nullptr;
        }
    }
    return m;
}
