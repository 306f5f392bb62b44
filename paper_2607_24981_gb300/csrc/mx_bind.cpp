// mx_bind.cpp -- the Python side of the microscaled 4-bit and mixture-of-experts entry points (mx.py) as a CPython extension.
//
// It does what the rest of the binding does in Python: reads tensors' addresses, sizes and strides, makes room for
// results, and calls the C-ABI on the current stream; nothing is computed here.  These calls are a few microseconds on
// the device, and reading some ten properties of five tensors in Python took 9 of the 16 us of a call.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdarg>
#include <cstdint>
#include <string>

#include "ilwdetr.h"

namespace {

// The entry points, as the library that the package has loaded holds them, and the package's exception.
struct Library {
    decltype(&ilwdetr_last_error) last_error;
    decltype(&ilwdetr_mx_quantize) quantize;
    decltype(&ilwdetr_mx_dequantize) dequantize;
    decltype(&ilwdetr_mx_gemm) gemm;
    decltype(&ilwdetr_moe_route_workspace_bytes) route_bytes;
    decltype(&ilwdetr_moe_route) route;
    decltype(&ilwdetr_moe_combine) combine;
} lib = {};
PyObject *g_error = nullptr;

struct Failed {};  // a Python exception is set

[[noreturn]] void fail(const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    PyErr_SetString(g_error ? g_error : PyExc_RuntimeError, buf);
    throw Failed();
}
void check(int rc, const char *what) {
    if (rc != 0) fail("%s failed (%d): %s", what, rc, lib.last_error());
}

const at::Tensor &tensor(PyObject *o, const char *what) {
    if (!THPVariable_Check(o)) fail("%s: a tensor is wanted, not %s", what, Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}
bool given(PyObject *o) { return o && o != Py_None; }

int form_of(at::ScalarType t, bool int8, const char *what) {
    switch (t) {
        case at::kFloat: return ILW_FP32;
        case at::kHalf: return ILW_FP16;
        case at::kBFloat16: return ILW_BF16;
        case at::kChar:
            if (int8) return 8;
            [[fallthrough]];
        default: fail("%s: %s is none of float32, float16, bfloat16%s", what, c10::toString(t), int8 ? ", int8" : "");
    }
}

// All tensors of a call are on the GPU of its first one.
void same_gpu(const at::Tensor &t, const at::Tensor &first, const char *what) {
    if (t.device() != first.device()) fail("%s: tensors on more than one device, %s and %s", what, first.device().str().c_str(), t.device().str().c_str());
}

// A float matrix on the GPU with contiguous rows.  No or a single row may carry any stride: then at least what holds a row.
struct Matrix {
    int form;
    int64_t rows, cols, ld;
    void *data;
};
Matrix matrix(const at::Tensor &t, const at::Tensor &first, const char *what, bool int8 = false) {
    Matrix m;
    m.form = form_of(t.scalar_type(), int8, what);
    if (t.dim() != 2) fail("%s: a tensor of %d dimensions, not 2", what, (int)t.dim());
    m.rows = t.size(0), m.cols = t.size(1), m.ld = t.stride(0);
    if (!t.is_cuda() || (t.stride(1) != 1 && m.cols > 1 && m.rows > 0)) fail("%s: a tensor is not on the GPU, or its rows are not contiguous", what);
    same_gpu(t, first, what);
    if (m.rows <= 1 || m.cols == 0) m.ld = std::max(m.ld, m.cols);
    m.data = t.data_ptr();
    return m;
}
const int32_t *indices(const at::Tensor &t, const at::Tensor &first, const char *what) {
    if (t.scalar_type() != at::kInt || !t.is_cuda() || !t.is_contiguous()) fail("%s: indices, slots and offsets are contiguous int32 CUDA tensors", what);
    same_gpu(t, first, what);
    return (const int32_t *)t.data_ptr();
}
// `rows` rows of `cols` float32 values, or the same values in one dimension.
const float *weights(const at::Tensor &t, const at::Tensor &first, int64_t rows, int64_t cols, const char *what, const char *name) {
    if (t.scalar_type() != at::kFloat || !t.is_cuda() || !t.is_contiguous() || t.numel() != rows * cols || (t.dim() > 1 && t.size(t.dim() - 1) != cols))
        fail("%s: %s is a contiguous float32 CUDA tensor (%lld, %lld)", what, name, (long long)rows, (long long)cols);
    same_gpu(t, first, what);
    return (const float *)t.data_ptr();
}

// An MXFP4 tensor: the tuple (codes, scales, k).
struct Mx {
    int64_t lead, rows, k, scale_cols;   // (lead: 1 without a leading dimension; scale_cols: bytes of a row of scales)
    const uint8_t *codes, *scales;
    int64_t ldc, lds, between_c, between_s;
    const at::Tensor *t;                 // codes
};
Mx mx(PyObject *o, int dims, const at::Tensor *first, const char *what) {
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3) fail("%s: an MxTensor is wanted, not %s", what, Py_TYPE(o)->tp_name);
    const at::Tensor &c = tensor(PyTuple_GET_ITEM(o, 0), what), &s = tensor(PyTuple_GET_ITEM(o, 1), what);
    Mx m;
    m.k = PyLong_AsLongLong(PyTuple_GET_ITEM(o, 2));
    if (m.k == -1 && PyErr_Occurred()) throw Failed();
    if (m.k < 1 || m.k > INT32_MAX) fail("%s: an MXFP4 tensor of k=%lld", what, (long long)m.k);
    const int64_t nb = (m.k + 31) / 32;
    bool fits = c.scalar_type() == at::kByte && s.scalar_type() == at::kByte && c.dim() == dims && s.dim() == dims && c.size(dims - 1) >= 16 * nb && s.size(dims - 1) >= nb;
    for (int i = 0; fits && i + 1 < dims; ++i) fits = c.size(i) == s.size(i);
    if (!fits)
        fail("%s: an MXFP4 tensor of k=%lld has uint8 codes [..., %lld] and scales [..., >= %lld] of %d dimensions", what, (long long)m.k,
             (long long)(16 * nb), (long long)nb, dims);
    if (!c.is_cuda() || !s.is_cuda() || ((c.stride(dims - 1) != 1 || s.stride(dims - 1) != 1) && c.numel()))
        fail("%s: codes or scales are not on the GPU, or their rows are not contiguous", what);
    same_gpu(s, c, what);
    if (first) same_gpu(c, *first, what);
    m.lead = dims == 3 ? c.size(0) : 1;
    m.rows = c.size(dims - 2), m.scale_cols = s.size(dims - 1);
    m.ldc = c.stride(dims - 2), m.lds = s.stride(dims - 2);
    if (m.rows <= 1 || c.size(dims - 1) == 0) {  // (no or a single row may carry any stride)
        m.ldc = std::max(m.ldc, (c.size(dims - 1) + 15) / 16 * 16);
        m.lds = std::max(m.lds, (s.size(dims - 1) + 15) / 16 * 16);
    }
    m.between_c = dims == 3 ? c.stride(0) : 0, m.between_s = dims == 3 ? s.stride(0) : 0;
    m.codes = (const uint8_t *)c.data_ptr(), m.scales = (const uint8_t *)s.data_ptr();
    m.t = &c;
    return m;
}

// A call launches on its tensors' GPU, on that GPU's current stream.
struct Launch {
    c10::cuda::CUDAGuard device;
    ilw_stream_t stream;
    explicit Launch(const at::Tensor &t) : device(t.device()), stream(c10::cuda::getCurrentCUDAStream(t.get_device()).stream()) {}
};
at::Tensor room(at::IntArrayRef size, at::ScalarType type, const at::Tensor &like) { return at::empty(size, at::TensorOptions().dtype(type).device(like.device())); }
// Several results in one allocation (an allocation is a good part of a short call): the tensor of `size` and `type` that begins
// `bytes` into `whole`, `bytes` a multiple of its element size.
at::Tensor part_of(const at::Tensor &whole, int64_t bytes, at::IntArrayRef size, at::ScalarType type) {
    const caffe2::TypeMeta meta = c10::scalarTypeToTypeMeta(type);
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(whole.storage()), whole.key_set(), meta);
    t.unsafeGetTensorImpl()->set_storage_offset(bytes / (int64_t)meta.itemsize());
    t.unsafeGetTensorImpl()->set_sizes_contiguous(size);
    return t;
}
PyObject *wrap(const at::Tensor &t) { return THPVariable_Wrap(t); }
// The dtype argument, or what it stands for when it is None.
at::ScalarType dtype_or(PyObject *o, at::ScalarType otherwise, const char *what) {
    if (!given(o)) return otherwise;
    if (!THPDtype_Check(o)) fail("%s: a torch.dtype is wanted, not %s", what, Py_TYPE(o)->tp_name);
    return ((THPDtype *)o)->scalar_type;
}
int64_t whole(PyObject *o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Failed();
    return v;
}

// quantize(X, gather, out) -> (codes, scales, k)
PyObject *quantize(PyObject *const *a) {
    const char *what = "mx_quantize";
    const at::Tensor &X = tensor(a[0], what);
    const Matrix x = matrix(X, X, what, true);
    int64_t rows = x.rows;
    const int32_t *at = nullptr;
    if (given(a[1])) {
        const at::Tensor &g = tensor(a[1], what);
        at = indices(g, X, what);
        rows = g.numel();
    }
    const int64_t nb = (x.cols + 31) / 32, pad = (nb + 15) / 16 * 16;
    if (given(a[2])) {
        const Mx m = mx(a[2], 2, &X, what);
        if (m.k != x.cols || m.rows != rows)
            fail("%s: out holds %lld rows of %lld, not %lld of %lld", what, (long long)m.rows, (long long)m.k, (long long)rows, (long long)x.cols);
        // (each row of scales is filled up to a multiple of 16 bytes; more than the tensor holds are not its own)
        if (m.scale_cols < pad) fail("%s: scales of out have rows of %lld bytes: at least %lld, a multiple of 16", what, (long long)m.scale_cols, (long long)pad);
        const Launch on(X);
        check(lib.quantize(x.data, x.form, x.ld, x.rows, at, rows, (int32_t)std::min<int64_t>(x.cols, INT32_MAX), (uint8_t *)m.codes, m.ldc,
                           (uint8_t *)m.scales, m.lds, on.stream),
              what);
        return Py_NewRef(a[2]);
    }
    const at::Tensor both = room({rows * (16 * nb + pad)}, at::kByte, X), codes = part_of(both, 0, {rows, 16 * nb}, at::kByte),
                     scales = part_of(both, rows * 16 * nb, {rows, pad}, at::kByte);
    const Launch on(X);
    check(lib.quantize(x.data, x.form, x.ld, x.rows, at, rows, (int32_t)std::min<int64_t>(x.cols, INT32_MAX), (uint8_t *)codes.data_ptr(), 16 * nb,
                       (uint8_t *)scales.data_ptr(), pad, on.stream),
          what);
    return Py_BuildValue("(NNL)", wrap(codes), wrap(scales), (long long)x.cols);
}

// dequantize(m, dtype, out)
PyObject *dequantize(PyObject *const *a) {
    const char *what = "mx_dequantize";
    const Mx m = mx(a[0], 2, nullptr, what);
    const at::Tensor out = given(a[2]) ? tensor(a[2], what) : room({m.rows, m.k}, dtype_or(a[1], at::kFloat, what), *m.t);
    const Matrix y = matrix(out, *m.t, what);
    if (y.rows != m.rows || y.cols != m.k)
        fail("%s: out is (%lld, %lld), not (%lld, %lld)", what, (long long)y.rows, (long long)y.cols, (long long)m.rows, (long long)m.k);
    const Launch on(*m.t);
    check(lib.dequantize(m.codes, m.ldc, m.scales, m.lds, m.rows, (int32_t)m.k, y.data, y.form, y.ld, on.stream), what);
    return wrap(out);
}

// gemm(A, W, offsets, bias, act, dtype, out)
PyObject *gemm(PyObject *const *a) {
    const bool grouped = given(a[2]);
    const char *what = grouped ? "mx_grouped_linear" : "mx_linear";
    const Mx A = mx(a[0], 2, nullptr, what), W = mx(a[1], grouped ? 3 : 2, A.t, what);
    const int64_t act = whole(a[4]), N = W.rows, wide = act == ILW_ACT_SILU_GATE ? N / 2 : N;
    if (A.k != W.k) fail("%s: A has k=%lld, W k=%lld", what, (long long)A.k, (long long)W.k);
    if (N > INT32_MAX || W.lead > INT32_MAX) fail("%s: rows or experts past 2^31", what);
    ilw_mx_gemm_t p = {};
    p.struct_size = sizeof(p);
    p.a_codes = A.codes, p.a_ldc = A.ldc, p.a_scales = A.scales, p.a_lds = A.lds;
    p.w_codes = W.codes, p.w_ldc = W.ldc, p.w_codes_stride = W.between_c;
    p.w_scales = W.scales, p.w_lds = W.lds, p.w_scales_stride = W.between_s;
    if (grouped) {
        const at::Tensor &off = tensor(a[2], what);
        p.offsets = indices(off, *A.t, what);
        if (off.numel() != W.lead + 1) fail("%s: %lld experts need %lld offsets, not %lld", what, (long long)W.lead, (long long)W.lead + 1, (long long)off.numel());
    }
    if (given(a[3])) p.bias = weights(tensor(a[3], what), *A.t, W.lead, N, what, "bias");
    const at::Tensor out = given(a[6]) ? tensor(a[6], what) : room({A.rows, wide}, dtype_or(a[5], at::kBFloat16, what), *A.t);
    const Matrix y = matrix(out, *A.t, what);
    if (y.rows != A.rows || y.cols != wide)
        fail("%s: out is (%lld, %lld), not (%lld, %lld)", what, (long long)y.rows, (long long)y.cols, (long long)A.rows, (long long)wide);
    p.M = A.rows, p.N = (int32_t)N, p.K = (int32_t)A.k, p.experts = (int32_t)W.lead, p.act = (int32_t)act, p.y_form = y.form;
    p.Y = y.data, p.ldy = y.ld;
    const Launch on(*A.t);
    check(lib.gemm(&p, on.stream), what);
    return wrap(out);
}

// route(logits, k, renormalize) -> (expert, weight, offsets, source, slot)
PyObject *route(PyObject *const *a) {
    const char *what = "moe_route";
    const at::Tensor &x = tensor(a[0], what);
    const Matrix m = matrix(x, x, what);
    const int64_t k = whole(a[1]), kk = k >= 1 && k <= ILW_MOE_MAX_TOP ? k : 0;  // (any other k is refused below: nothing is made for it)
    const int renormalize = PyObject_IsTrue(a[2]);
    if (renormalize < 0) throw Failed();
    if (m.rows > INT32_MAX || m.cols > INT32_MAX || k > INT32_MAX || k < INT32_MIN) fail("%s: more than 2^31 tokens or experts", what);
    const int32_t T = (int32_t)m.rows, E = (int32_t)m.cols;
    const size_t bytes = lib.route_bytes(T, E);
    const int64_t n = T * kk, words = 4 * n + E + 1;  // expert, weight, source, slot, offsets, then the workspace
    const at::Tensor all = room({4 * words + (int64_t)bytes}, at::kByte, x);
    const at::Tensor expert = part_of(all, 0, {T, kk}, at::kInt), weight = part_of(all, 4 * n, {T, kk}, at::kFloat),
                     source = part_of(all, 8 * n, {n}, at::kInt), slot = part_of(all, 12 * n, {T, kk}, at::kInt),
                     offsets = part_of(all, 16 * n, {(int64_t)E + 1}, at::kInt);
    const Launch on(x);
    check(lib.route(m.data, m.form, m.ld, T, E, (int32_t)k, renormalize, (int32_t *)expert.data_ptr(), (float *)weight.data_ptr(),
                    (int32_t *)offsets.data_ptr(), (int32_t *)source.data_ptr(), (int32_t *)slot.data_ptr(), bytes ? (char *)all.data_ptr() + 4 * words : nullptr, bytes,
                    on.stream),
          what);
    return Py_BuildValue("(NNNNN)", wrap(expert), wrap(weight), wrap(offsets), wrap(source), wrap(slot));
}

// combine(Y, slot, weight, residual, out)
PyObject *combine(PyObject *const *a) {
    const char *what = "moe_combine";
    const at::Tensor &Y = tensor(a[0], what), &slot = tensor(a[1], what);
    const Matrix y = matrix(Y, Y, what);
    const int32_t *at = indices(slot, Y, what);
    if (slot.dim() != 2) fail("%s: slot has %d dimensions, not 2", what, (int)slot.dim());
    const int64_t T = slot.size(0), k = slot.size(1);
    const float *w = weights(tensor(a[2], what), Y, T, k, what, "weight");
    if (T > INT32_MAX || k > INT32_MAX || y.cols > INT32_MAX) fail("%s: more than 2^31 tokens or columns", what);
    auto same = [&](const Matrix &m, const char *name) {
        if (m.form != y.form || m.rows != T || m.cols != y.cols)
            fail("%s: %s is (%lld, %lld), not (%lld, %lld), or of another type than Y", what, name, (long long)m.rows, (long long)m.cols, (long long)T, (long long)y.cols);
    };
    Matrix res = {};
    if (given(a[3])) same(res = matrix(tensor(a[3], what), Y, what), "residual");
    const at::Tensor out = given(a[4]) ? tensor(a[4], what) : room({T, y.cols}, Y.scalar_type(), Y);
    const Matrix o = matrix(out, Y, what);
    same(o, "out");
    const Launch on(Y);
    check(lib.combine(y.data, y.form, y.ld, y.rows, at, w, (int32_t)T, (int32_t)k, (int32_t)y.cols, res.data, res.ld, o.data, o.ld, on.stream), what);
    return wrap(out);
}

// bind(exception, addresses of the entry points in the order of Library)
PyObject *bind(PyObject *const *a) {
    Py_XSETREF(g_error, Py_NewRef(a[0]));
    void **to = (void **)&lib;
    for (size_t i = 0; i < sizeof(lib) / sizeof(void *); ++i) to[i] = (void *)(uintptr_t)whole(a[i + 1]);
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%d arguments are wanted, not %d", N, (int)n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Failed &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
#define ILW_METHOD(f, n) {#f, (PyCFunction)(void (*)(void))call<f, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ILW_METHOD(bind, 8), ILW_METHOD(quantize, 3), ILW_METHOD(dequantize, 3), ILW_METHOD(gemm, 7), ILW_METHOD(route, 3),
                         ILW_METHOD(combine, 5), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_mxbind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mxbind(void) { return PyModule_Create(&module_def); }
