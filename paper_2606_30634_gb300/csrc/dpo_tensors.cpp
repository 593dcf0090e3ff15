// dpo_tensors.cpp -- the feed-forward calls of include/dpo.h on PyTorch tensors: the
// part of ffn.py between its signatures and the C ABI (checks, pitches, outputs and
// workspaces from PyTorch's allocator, the current stream), as a Python module.
//
// A small call is as long as its host side: the norm of one row takes 4 us on the GPU, and
// the same checks, three allocations and a ctypes call took 17 us in Python.
//
// The C ABI's functions come as addresses (bind), so the library that dpo.load() chose
// is the one that is called. Nothing here throws past its entry points.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/util/DimVector.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>

#include "dpo.h"

namespace {

using at::Tensor;

// ---- the library ----

struct Library {
    decltype(&dpo_pack8) pack8 = nullptr;
    decltype(&dpo_unpack8) unpack8 = nullptr;
    decltype(&dpo_rmsnorm) rmsnorm = nullptr;
    decltype(&dpo_rmsnorm_backward) rmsnorm_backward = nullptr;
    decltype(&dpo_rmsnorm_workspace) rmsnorm_workspace = nullptr;
    decltype(&dpo_ffn_forward) ffn_forward = nullptr;
    decltype(&dpo_ffn_backward) ffn_backward = nullptr;
    decltype(&dpo_ffn_workspace) ffn_workspace = nullptr;
    decltype(&dpo_last_error) last_error = nullptr;
    PyObject *error = nullptr;   // DpoError
};
Library g_lib;

// ---- errors ----

struct Bad {   // a tensor that does not fit
    PyObject *type;
    std::string what;
};
[[noreturn]] void value_error(const std::string &s) { throw Bad{PyExc_ValueError, s}; }
[[noreturn]] void type_error(const std::string &s) { throw Bad{PyExc_TypeError, s}; }
struct Refused {   // by the library
    int code;
};
void check(int rc)
{
    if (rc != DPO_OK)
        throw Refused{rc};
}

template <class F> PyObject *guarded(F &&f)
{
    HANDLE_TH_ERRORS
    try {
        if (g_lib.error == nullptr) {
            PyErr_SetString(PyExc_RuntimeError, "dpo_tensors is not bound to a library");
            return nullptr;
        }
        return f();
    } catch (const Bad &e) {
        PyErr_SetString(e.type, e.what.c_str());
    } catch (const Refused &e) {
        PyObject *v = PyObject_CallFunction(g_lib.error, "is", e.code, g_lib.last_error(nullptr));
        if (v != nullptr) {
            PyErr_SetObject(g_lib.error, v);
            Py_DECREF(v);
        }
    }
    return nullptr;
    END_HANDLE_TH_ERRORS
}

// ---- tensors ----

std::string shape(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i)
        r += (i ? ", " : "") + std::to_string(s[i]);
    return r + ")";
}

const Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o))
        type_error(std::string(name) + ": a tensor is needed");
    return THPVariable_Unpack(o);
}

int dtype_of(const Tensor &t, const char *name)
{
    if (t.scalar_type() == at::kBFloat16)
        return DPO_BF16;
    if (t.scalar_type() != at::kFloat)
        type_error(std::string(name) + ": " + toString(t.scalar_type()) + " (float32 or bfloat16)");
    return DPO_F32;
}

void on_device(const Tensor &t, at::Device device, const char *name)
{
    if (t.device() != device)
        value_error(std::string(name) + " is on " + t.device().str() + ", not " + device.str());
}

// A matrix of contiguous rows: the leading dimensions flattened without a copy.
struct Mat {
    void *p;
    int64_t rows, cols, ld;
};
Mat rows_of(const Tensor &t, const char *name)
{
    if (!t.is_cuda())
        value_error(std::string(name) + " is not a CUDA tensor");
    const auto size = t.sizes(), stride = t.strides();
    const int n = (int)size.size();
    if (n == 0)
        value_error(std::string(name) + " has no dimensions");
    Mat m = {t.data_ptr(), 1, size[n - 1], 0};
    if (m.cols > 1 && stride[n - 1] != 1)
        value_error(std::string(name) + ": the last dimension is not contiguous");
    int64_t next = -1;   // the stride that the next dimension out has to have
    for (int i = n - 2; i >= 0; --i) {
        m.rows *= size[i];
        if (size[i] == 1)
            continue;
        if (next < 0)
            m.ld = stride[i];
        else if (stride[i] != next && t.numel() != 0)
            value_error(std::string(name) + ": leading dimensions do not flatten to rows");
        next = stride[i] * size[i];
    }
    if (m.rows <= 1) {   // a single row may report any stride; a pitch that can be one is kept
        const int64_t s = n > 1 ? stride[n - 2] : 0;
        m.ld = s >= m.cols && s % 16 == 0 ? s : m.cols;
    }
    return m;
}

void fits(const Tensor &t, at::ScalarType type, at::IntArrayRef size, at::Device device,
          const char *name)
{
    if (t.scalar_type() != type)
        type_error(std::string(name) + ": " + toString(t.scalar_type()) + ", expected " + toString(type));
    if (t.sizes() != size)
        value_error(std::string(name) + ": shape " + shape(t.sizes()) + ", expected " + shape(size));
    on_device(t, device, name);
}

void *vector_of(const Tensor &t, int64_t n, at::Device device, const char *name)
{
    if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1))
        value_error(std::string(name) + ": expected " + std::to_string(n) + " contiguous elements");
    on_device(t, device, name);
    return t.data_ptr();
}

void *matrix_of(const Tensor &t, int64_t rows, int64_t cols, at::ScalarType type, at::Device device,
                const char *name)
{
    if (t.scalar_type() != type)
        type_error(std::string(name) + ": " + toString(t.scalar_type()) + ", expected " + toString(type));
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols || !t.is_contiguous())
        value_error(std::string(name) + ": expected a contiguous matrix of shape " + shape({rows, cols}) +
                    ", got " + shape(t.sizes()));
    on_device(t, device, name);
    return t.data_ptr();
}

// A weight of the block, whose products take bf16.
void *weight_of(const Tensor &t, int64_t rows, int64_t cols, at::Device device, const char *name)
{
    if (t.scalar_type() == at::kFloat)
        type_error(std::string(name) + ": Float, expected BFloat16 (an optimizer's stale weights are "
                   "with stash_dtype=DPO_BF16)");
    return matrix_of(t, rows, cols, at::kBFloat16, device, name);
}

constexpr int64_t groups(int64_t cols) { return (cols + DPO_PACK8_GROUP - 1) / DPO_PACK8_GROUP; }

dpo_packed8 packed_of(PyObject *codes, PyObject *scales, int64_t rows, int64_t cols,
                      at::Device device, const char *name)
{
    const Tensor &q = tensor(codes, name), &s = tensor(scales, name);
    Mat m[2];
    for (int i = 0; i < 2; ++i) {
        const Tensor &t = i ? s : q;
        const int64_t n = i ? groups(cols) : cols;
        if (t.scalar_type() != at::kByte)
            type_error(std::string(name) + ": " + toString(t.scalar_type()) + ", expected uint8");
        m[i] = rows_of(t, name);
        if (m[i].rows != rows || m[i].cols != n)
            value_error(std::string(name) + ": shape " + shape(t.sizes()) + ", expected " +
                        shape({rows, n}));
        on_device(t, device, name);
    }
    return {(uint8_t *)m[0].p, (uint8_t *)m[1].p, m[0].ld, m[1].ld};
}

Tensor make(at::IntArrayRef size, at::ScalarType type, at::Device device)
{
    return at::empty(size, at::TensorOptions().dtype(type).device(device));
}

struct Packed {
    Tensor codes, scales;
    dpo_packed8 p;
};
// What stands for a tensor of this shape: codes of the same shape, and scales that differ
// in the last dimension.
Packed make_packed(at::IntArrayRef size, at::Device device)
{
    Packed q;
    c10::DimVector groups_of(size.begin(), size.end());
    const int64_t cols = size.back(), ng = groups(cols);
    groups_of.back() = ng;
    q.codes = make(size, at::kByte, device);
    q.scales = make(groups_of, at::kByte, device);
    q.p = {(uint8_t *)q.codes.data_ptr(), (uint8_t *)q.scales.data_ptr(), cols, ng};
    return q;
}
// A matrix whose codes have a pitch of whole 32 bytes.
Packed make_kept(int64_t rows, int64_t cols, at::Device device)
{
    const int64_t ld = (cols + 31) / 32 * 32;
    if (ld == cols)
        return make_packed({rows, cols}, device);
    Packed q;
    q.codes = at::empty_strided({rows, cols}, {ld, 1},
                                at::TensorOptions().dtype(at::kByte).device(device));
    q.scales = make({rows, groups(cols)}, at::kByte, device);
    q.p = {(uint8_t *)q.codes.data_ptr(), (uint8_t *)q.scales.data_ptr(), ld, groups(cols)};
    return q;
}

// The current stream of the tensors' device, which has to be the current one.
void *stream_of(const Tensor &t, const char *name)
{
    const auto current = c10::cuda::current_device();
    if (t.device().index() != current)
        value_error(std::string(name) + " is on " + t.device().str() + "; the current device is cuda:" +
                    std::to_string((int)current));
    return c10::cuda::getCurrentCUDAStream(current).stream();
}

PyObject *wrap(const Tensor &t)
{
    if (!t.defined())
        Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
template <class... T> PyObject *tuple(const T &...t)
{
    PyObject *r = PyTuple_New(sizeof...(T));
    if (r == nullptr)
        return nullptr;
    Py_ssize_t i = 0;
    bool ok = true;
    auto put = [&](const Tensor &x) {
        PyObject *o = wrap(x);
        ok = ok && o != nullptr;
        PyTuple_SET_ITEM(r, i++, o);
    };
    (put(t), ...);
    if (!ok) {
        Py_DECREF(r);
        return nullptr;
    }
    return r;
}

int integer(PyObject *o)
{
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        type_error("an integer is needed");
    }
    return (int)v;
}

bool expect(Py_ssize_t n, Py_ssize_t want)
{
    if (n == want)
        return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", n, want);
    return false;
}

// ---- calls ----

// pack8(x) -> codes, scales
PyObject *pack8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 1))
        return nullptr;
    return guarded([&] {
        const Tensor &x = tensor(a[0], "x");
        const Mat m = rows_of(x, "x");
        const int dt = dtype_of(x, "x");
        void *const s = stream_of(x, "x");
        const Packed q = make_packed(x.sizes(), x.device());
        check(g_lib.pack8(m.p, (dpo_dtype)dt, m.rows, m.cols, m.ld, &q.p, s));
        return tuple(q.codes, q.scales);
    });
}

// unpack8(codes, scales, out or None, bf16) -> out
PyObject *unpack8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 4))
        return nullptr;
    return guarded([&] {
        const Tensor &q = tensor(a[0], "p");
        const Mat m = rows_of(q, "p");
        const dpo_packed8 p = packed_of(a[0], a[1], m.rows, m.cols, q.device(), "p");
        void *const s = stream_of(q, "p");
        Tensor out;
        if (a[2] == Py_None) {
            out = make(q.sizes(), integer(a[3]) ? at::kBFloat16 : at::kFloat, q.device());
        } else {
            out = tensor(a[2], "out");
            fits(out, out.scalar_type(), q.sizes(), q.device(), "out");
        }
        const Mat o = rows_of(out, "out");
        check(g_lib.unpack8(&p, m.rows, m.cols, o.p, (dpo_dtype)dtype_of(out, "out"), o.ld, s));
        return wrap(out);
    });
}

// add_rms_norm(x, weight, residual or None, eps, save8) -> y, h, rstd, codes, scales
PyObject *add_rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 5))
        return nullptr;
    const double eps = PyFloat_AsDouble(a[3]);
    if (eps == -1.0 && PyErr_Occurred())
        return nullptr;
    return guarded([&] {
        const Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight");
        const Mat m = rows_of(x, "x");
        const at::Device device = x.device();
        void *const s = stream_of(x, "x");
        dpo_rmsnorm_args k{};
        k.dtype = dtype_of(x, "x");
        k.weight_dtype = dtype_of(w, "weight");
        k.weight = vector_of(w, m.cols, device, "weight");
        Tensor h = x;
        if (a[2] != Py_None) {
            const Tensor &r = tensor(a[2], "residual");
            fits(r, x.scalar_type(), x.sizes(), device, "residual");
            const Mat rm = rows_of(r, "residual");
            k.residual = rm.p;
            k.ld_residual = rm.ld;
            h = make(x.sizes(), x.scalar_type(), device);
            k.h = h.data_ptr();
        }
        const Tensor y = make(x.sizes(), x.scalar_type(), device);
        const Tensor rstd = make({m.rows}, at::kFloat, device);
        Packed q;
        if (integer(a[4])) {
            q = make_packed(x.sizes(), device);
            k.x8 = q.p;
        }
        k.x = m.p;
        k.y = y.data_ptr();
        k.rstd = static_cast<float *>(rstd.data_ptr());
        k.rows = m.rows;
        k.cols = k.ld_h = k.ld_y = m.cols;
        k.ld_x = m.ld;
        k.eps = (float)eps;
        check(g_lib.rmsnorm(&k, s));
        return tuple(y, h, rstd, q.codes, q.scales);
    });
}

// add_rms_norm_backward(dy, weight, rstd, h or None, codes or None, scales, dh or None,
//                       dweight or None, accumulate) -> dx, dweight
PyObject *add_rms_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 9))
        return nullptr;
    return guarded([&] {
        const Tensor &dy = tensor(a[0], "dy"), &w = tensor(a[1], "weight"),
                     &rstd = tensor(a[2], "rstd");
        const Mat m = rows_of(dy, "dy");
        const at::Device device = dy.device();
        void *const s = stream_of(dy, "dy");
        dpo_rmsnorm_backward_args k{};
        k.dtype = dtype_of(dy, "dy");
        k.weight_dtype = dtype_of(w, "weight");
        k.weight = vector_of(w, m.cols, device, "weight");
        if (rstd.scalar_type() != at::kFloat)
            type_error(std::string("rstd: ") + toString(rstd.scalar_type()) + ", expected Float");
        k.rstd = static_cast<const float *>(vector_of(rstd, m.rows, device, "rstd"));
        if (a[3] != Py_None) {
            const Tensor &h = tensor(a[3], "h");
            fits(h, dy.scalar_type(), dy.sizes(), device, "h");
            const Mat hm = rows_of(h, "h");
            k.h = hm.p;
            k.ld_h = hm.ld;
        } else {
            k.x8 = packed_of(a[4], a[5], m.rows, m.cols, device, "x8");
        }
        if (a[6] != Py_None) {
            const Tensor &dh = tensor(a[6], "dh");
            fits(dh, dy.scalar_type(), dy.sizes(), device, "dh");
            const Mat dm = rows_of(dh, "dh");
            k.dh = dm.p;
            k.ld_dh = dm.ld;
        }
        const Tensor dw =
            a[7] == Py_None ? make({m.cols}, at::kFloat, device) : tensor(a[7], "dweight");
        k.dweight = vector_of(dw, m.cols, device, "dweight");
        k.dweight_dtype = dtype_of(dw, "dweight");
        k.accumulate = integer(a[8]);
        const Tensor dx = make(dy.sizes(), dy.scalar_type(), device);
        check(g_lib.rmsnorm_workspace(m.rows, m.cols, &k.workspace_bytes));
        const Tensor ws = make({k.workspace_bytes}, at::kByte, device);
        k.workspace = ws.data_ptr();
        k.dy = m.p;
        k.dx = dx.data_ptr();
        k.rows = m.rows;
        k.cols = k.ld_dx = m.cols;
        k.ld_dy = m.ld;
        check(g_lib.rmsnorm_backward(&k, s));
        return tuple(dx, dw);
    });
}

// gated_ffn(x, w_gate, w_up, w_down, act, keep, out or None)
//     -> out, gate (codes or bf16), gate scales, up, up scales
PyObject *gated_ffn(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 7))
        return nullptr;
    return guarded([&] {
        const Tensor &x = tensor(a[0], "x"), &wg = tensor(a[1], "w_gate");
        const Mat m = rows_of(x, "x");
        if (x.scalar_type() != at::kBFloat16)
            type_error(std::string("x: ") + toString(x.scalar_type()) + " (bfloat16)");
        const at::Device device = x.device();
        void *const s = stream_of(x, "x");
        if (wg.dim() != 2)
            value_error("w_gate: expected a matrix");
        dpo_ffn_args k{};
        k.tokens = m.rows;
        k.dim = m.cols;
        k.hidden = wg.size(0);
        k.w_gate = weight_of(wg, k.hidden, k.dim, device, "w_gate");
        k.w_up = weight_of(tensor(a[2], "w_up"), k.hidden, k.dim, device, "w_up");
        k.w_down = weight_of(tensor(a[3], "w_down"), k.dim, k.hidden, device, "w_down");
        check(g_lib.ffn_workspace(k.tokens, k.dim, k.hidden, 0, &k.workspace_bytes, nullptr));
        Tensor out;
        if (a[6] == Py_None) {
            out = make(x.sizes(), at::kBFloat16, device);
        } else {
            out = tensor(a[6], "out");
            fits(out, at::kBFloat16, x.sizes(), device, "out");
        }
        const Mat o = rows_of(out, "out");
        k.act = integer(a[4]);
        k.keep = integer(a[5]);
        Packed g, u;
        Tensor g16, u16;
        if (k.keep == DPO_KEEP_8BIT) {
            g = make_kept(k.tokens, k.hidden, device);
            u = make_kept(k.tokens, k.hidden, device);
            k.gate8 = g.p;
            k.up8 = u.p;
        } else if (k.keep == DPO_KEEP_BF16) {
            g16 = make({k.tokens, k.hidden}, at::kBFloat16, device);
            u16 = make({k.tokens, k.hidden}, at::kBFloat16, device);
            k.gate = g16.data_ptr();
            k.up = u16.data_ptr();
        }
        const Tensor ws = make({k.workspace_bytes}, at::kByte, device);
        k.workspace = ws.data_ptr();
        k.x = m.p;
        k.ld_x = m.ld;
        k.out = o.p;
        k.ld_out = o.ld;
        check(g_lib.ffn_forward(&k, s));
        return k.keep == DPO_KEEP_BF16 ? tuple(out, g16, Tensor(), u16, Tensor())
                                       : tuple(out, g.codes, g.scales, u.codes, u.scales);
    });
}

// gated_ffn_backward(dout, act, keep, gate, gate scales, up, up scales, w_gate, w_up, w_down,
//                    dw_gate, dw_up, dw_down, x or None, codes or None, scales, gain or None,
//                    accumulate, dx or None) -> dx
PyObject *gated_ffn_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 19))
        return nullptr;
    return guarded([&] {
        const Tensor &dout = tensor(a[0], "dout"), &wg = tensor(a[7], "w_gate");
        const Mat m = rows_of(dout, "dout");
        if (dout.scalar_type() != at::kBFloat16)
            type_error(std::string("dout: ") + toString(dout.scalar_type()) + " (bfloat16)");
        const at::Device device = dout.device();
        void *const s = stream_of(dout, "dout");
        if (wg.dim() != 2)
            value_error("w_gate: expected a matrix");
        dpo_ffn_backward_args k{};
        k.tokens = m.rows;
        k.dim = m.cols;
        k.hidden = wg.size(0);
        k.w_gate = weight_of(wg, k.hidden, k.dim, device, "w_gate");
        k.w_up = weight_of(tensor(a[8], "w_up"), k.hidden, k.dim, device, "w_up");
        k.w_down = weight_of(tensor(a[9], "w_down"), k.dim, k.hidden, device, "w_down");
        const Tensor &dwg = tensor(a[10], "dw_gate");
        const at::ScalarType gt = dwg.scalar_type();
        k.grad_dtype = dtype_of(dwg, "dw_gate");
        k.dw_gate = matrix_of(dwg, k.hidden, k.dim, gt, device, "dw_gate");
        k.dw_up = matrix_of(tensor(a[11], "dw_up"), k.hidden, k.dim, gt, device, "dw_up");
        k.dw_down = matrix_of(tensor(a[12], "dw_down"), k.dim, k.hidden, gt, device, "dw_down");
        if (a[13] != Py_None) {
            const Tensor &x = tensor(a[13], "x");
            fits(x, at::kBFloat16, dout.sizes(), device, "x");
            const Mat xm = rows_of(x, "x");
            k.x = xm.p;
            k.ld_x = xm.ld;
        } else {
            k.x8 = packed_of(a[14], a[15], m.rows, m.cols, device, "x8");
            if (a[16] != Py_None) {
                const Tensor &gain = tensor(a[16], "gain");
                k.gain = vector_of(gain, m.cols, device, "gain");
                k.gain_dtype = dtype_of(gain, "gain");
            }
        }
        k.act = integer(a[1]);
        k.keep = integer(a[2]);
        if (k.keep == DPO_KEEP_8BIT) {
            k.gate8 = packed_of(a[3], a[4], k.tokens, k.hidden, device, "kept");
            k.up8 = packed_of(a[5], a[6], k.tokens, k.hidden, device, "kept");
        } else {
            k.gate = matrix_of(tensor(a[3], "kept"), k.tokens, k.hidden, at::kBFloat16, device, "kept");
            k.up = matrix_of(tensor(a[5], "kept"), k.tokens, k.hidden, at::kBFloat16, device, "kept");
        }
        k.accumulate = integer(a[17]);
        check(g_lib.ffn_workspace(k.tokens, k.dim, k.hidden, a[13] == Py_None, nullptr,
                                  &k.workspace_bytes));
        Tensor dx;
        if (a[18] == Py_None) {
            dx = make(dout.sizes(), at::kBFloat16, device);
        } else {
            dx = tensor(a[18], "dx");
            fits(dx, at::kBFloat16, dout.sizes(), device, "dx");
        }
        const Mat xo = rows_of(dx, "dx");
        const Tensor ws = make({k.workspace_bytes}, at::kByte, device);
        k.workspace = ws.data_ptr();
        k.dout = m.p;
        k.ld_dout = m.ld;
        k.dx = xo.p;
        k.ld_dx = xo.ld;
        check(g_lib.ffn_backward(&k, s));
        return wrap(dx);
    });
}

// bind(DpoError, addresses in the order of Library)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (!expect(n, 10))
        return nullptr;
    void *p[9];
    for (int i = 0; i < 9; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i + 1]);
        if (p[i] == nullptr) {
            if (!PyErr_Occurred())
                PyErr_SetString(PyExc_ValueError, "an address is 0");
            return nullptr;
        }
    }
    Library l;
    l.pack8 = (decltype(l.pack8))p[0];
    l.unpack8 = (decltype(l.unpack8))p[1];
    l.rmsnorm = (decltype(l.rmsnorm))p[2];
    l.rmsnorm_backward = (decltype(l.rmsnorm_backward))p[3];
    l.rmsnorm_workspace = (decltype(l.rmsnorm_workspace))p[4];
    l.ffn_forward = (decltype(l.ffn_forward))p[5];
    l.ffn_backward = (decltype(l.ffn_backward))p[6];
    l.ffn_workspace = (decltype(l.ffn_workspace))p[7];
    l.last_error = (decltype(l.last_error))p[8];
    Py_INCREF(a[0]);
    Py_XDECREF(g_lib.error);
    l.error = a[0];
    g_lib = l;
    Py_RETURN_NONE;
}

#define FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {FAST(bind),        FAST(pack8),     FAST(unpack8),
                           FAST(add_rms_norm), FAST(add_rms_norm_backward),
                           FAST(gated_ffn),   FAST(gated_ffn_backward),
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "dpo_tensors", nullptr, -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_dpo_tensors(void) { return PyModule_Create(&g_module); }
