// Tensor arguments of the calls of a decoding step (4-bit weights, rows in 8 bits, norms, routing) -> the C ABI (include/qnn.h):
// checks, the result's allocation on the current stream, and the call, in one step from Python.  A step of decoding makes these
// calls for every layer with microseconds of work each; through ctypes the marshalling alone took longer than the small ones run
// (a call with a new result 10.7 us, of which 2.9 the launch, and 4.5 here; with a result given 8.9 and 3.4).
// Argument marshalling only: every step of the work runs inside libqnn's kernels.
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_strided.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/core/AutogradState.h>
#include <c10/core/GradMode.h>
#include <c10/core/TensorImpl.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "qnn.h"

namespace {

struct Refused : std::exception {                       // becomes a ValueError
    const char *what_;
    explicit Refused(const char *w) : what_(w) {}
    const char *what() const noexcept override { return what_; }
};

const at::Tensor &tensor_of(PyObject *o, const char *what) {
    if (!THPVariable_Check(o)) throw Refused(what);
    return THPVariable_Unpack(o);
}
bool given(PyObject *o) { return o != Py_None; }

int type_of(const at::Tensor &t) {
    switch (t.scalar_type()) {
        case at::kFloat: return QNN_F32;
        case at::kBFloat16: return QNN_BF16;
        case at::kHalf: return QNN_F16;
        default: throw Refused("rows must be float32, bfloat16 or float16");
    }
}

// These calls record no gradients: an operand that requires one, while they are recorded, would lose it without a word, and so would one that
// carries a forward-mode tangent.
void check_no_graph(const at::Tensor &t) {
    if (t.requires_grad() && c10::GradMode::is_enabled())
        throw Refused("these calls record no gradients: detach tensors that require grad, or call under torch.no_grad()");
    if (t._fw_grad(0).defined() && c10::AutogradState::get_tls_state().get_fw_grad_mode())
        throw Refused("these calls carry no forward-mode tangents: pass the primal alone");
}

struct Rows {
    int type;
    int64_t rows, ld;
};
// [rows, width] whose rows may lie apart but not overlap; width < 0: any.
Rows rows_of(const at::Tensor &t, int64_t width) {
    Rows r;
    check_no_graph(t);
    r.type = type_of(t);
    if (t.dim() != 2 || (width >= 0 && t.size(1) != width)) throw Refused("rows must be [rows, width] with the width of the weights");
    r.rows = t.size(0);
    const int64_t cols = t.size(1);
    r.ld = r.rows > 1 ? t.stride(0) : std::max(t.stride(0), cols);
    if ((cols > 1 && r.rows > 0 && t.stride(1) != 1) || r.ld < cols) throw Refused("rows must be contiguous and must not overlap");
    return r;
}

struct Weights {
    const at::Tensor &codes, &scales, &alpha;
    int64_t n, k, group, experts;
};
// args: codes, scales, alpha, n, k, group
Weights weights_of(PyObject *const *a) {
    Weights w{tensor_of(a[0], "codes must be a tensor"), tensor_of(a[1], "scales must be a tensor"), tensor_of(a[2], "alpha must be a tensor"),
              PyLong_AsLongLong(a[3]), PyLong_AsLongLong(a[4]), PyLong_AsLongLong(a[5]), 0};
    if (PyErr_Occurred()) throw python_error();
    if (w.group != 32 && w.group != 64 && w.group != 128) throw Refused("group must be 32, 64 or 128");
    if (w.codes.scalar_type() != at::kInt || w.scales.scalar_type() != at::kByte || w.alpha.scalar_type() != at::kFloat ||
        !w.codes.is_contiguous() || !w.scales.is_contiguous() || !w.alpha.is_contiguous())
        throw Refused("codes, scales and alpha must be contiguous int32, uint8 and float32");
    check_no_graph(w.alpha);
    const int64_t tn = (w.n + 127) / 128, tk = (w.k + 127) / 128;
    const auto c = w.codes.sizes(), s = w.scales.sizes();
    if (w.n < 1 || w.k < 1 || c.size() != 6 || c[1] != tn || c[2] != tk || c[3] != 4 || c[4] != 128 || c[5] != 4)
        throw Refused("codes do not have the shape of an n x k matrix");
    w.experts = c[0];
    if (s.size() != 5 || s[0] != w.experts || s[1] != tn || s[2] != tk || s[3] != 128 / w.group || s[4] != 128 || w.alpha.dim() != 1 ||
        w.alpha.size(0) != w.experts)
        throw Refused("scales or alpha do not have the shape that goes with the codes");
    return w;
}

int64_t experts_of(const at::Tensor &offsets) {
    if (offsets.scalar_type() != at::kInt || offsets.dim() != 1 || !offsets.is_contiguous() || offsets.size(0) < 2)
        throw Refused("offsets must be contiguous int32 [experts + 1]");
    return offsets.size(0) - 1;
}

// Everything on one CUDA device, which is the current one; its stream.
void *stream_for(const at::Tensor &first, std::initializer_list<const at::Tensor *> others) {
    if (!first.is_cuda()) throw Refused("rows must be on the current CUDA device");
    const auto device = first.get_device();
    if (device != c10::cuda::current_device()) throw Refused("rows must be on the current CUDA device");
    for (const at::Tensor *t : others)
        if (!t->is_cuda() || t->get_device() != device) throw Refused("all tensors must be on the device of the rows");
    return c10::cuda::getCurrentCUDAStream(device).stream();
}

at::Tensor result_for(PyObject *out, const at::Tensor &like, int64_t rows, int64_t width, int64_t *ld) {
    if (!given(out)) {
        *ld = width;
        return at::empty({rows, width}, like.options());
    }
    const at::Tensor &t = tensor_of(out, "out must be a tensor");
    const Rows r = rows_of(t, width);
    if (t.scalar_type() != like.scalar_type() || r.rows != rows || !t.is_cuda() || t.get_device() != like.get_device())
        throw Refused("out must be [rows, width] of the type and on the device of the rows");
    *ld = r.ld;
    return t;
}

// New memory on a device, from torch's allocator without its dispatcher (0.3 us less).
at::Tensor new_array(const at::Tensor &like, at::ScalarType type, at::IntArrayRef sizes) {
    return at::Tensor(at::detail::empty_cuda(sizes, type, like.device(), std::nullopt));
}

at::Tensor workspace_for(PyObject *workspace, size_t need, const at::Tensor &like) {
    if (given(workspace)) {
        const at::Tensor &t = tensor_of(workspace, "workspace must be a tensor");
        if (!t.is_cuda() || t.get_device() != like.get_device() || !t.is_contiguous()) throw Refused("workspace must be contiguous on the device of the rows");
        return t;
    }
    return need ? new_array(like, at::kByte, {(int64_t)need}) : at::Tensor();
}

PyObject *answer(int status, at::Tensor &&result) { return status == QNN_OK ? THPVariable_Wrap(std::move(result)) : PyLong_FromLong(status); }

// g4_matvec(x, codes, scales, alpha, n, k, group, out, workspace)
PyObject *g4_matvec(PyObject *const *a) {
    const at::Tensor &x = tensor_of(a[0], "x must be a tensor");
    const Weights w = weights_of(a + 1);
    const Rows r = rows_of(x, w.k);
    if (w.experts != 1) throw Refused("g4_matvec takes one matrix");
    void *stream = stream_for(x, {&w.codes, &w.scales, &w.alpha});
    int64_t ldo;
    at::Tensor out = result_for(a[7], x, r.rows, w.n, &ldo);
    const at::Tensor ws = workspace_for(a[8], qnn_g4_matvec_workspace(x.data_ptr(), r.type, r.rows, r.ld, (int)w.n, (int)w.k), x);
    const int status = qnn_g4_matvec(x.data_ptr(), r.type, r.rows, r.ld, (const uint32_t *)w.codes.data_ptr(), (const uint8_t *)w.scales.data_ptr(),
                                     (const float *)w.alpha.data_ptr(), (int)w.n, (int)w.k, (int)w.group, out.data_ptr(), ldo,
                                     ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.nbytes() : 0, stream);
    return answer(status, std::move(out));
}

// g4_expert_gemm / _backward_data(rows, codes, scales, alpha, n, k, group, offsets, out, workspace)
template <bool BACKWARD>
PyObject *g4_expert(PyObject *const *a) {
    const at::Tensor &x = tensor_of(a[0], "x must be a tensor");
    const Weights w = weights_of(a + 1);
    const Rows r = rows_of(x, BACKWARD ? w.n : w.k);
    const at::Tensor &offsets = tensor_of(a[7], "offsets must be a tensor");
    if (experts_of(offsets) != w.experts) throw Refused("offsets must have experts + 1 entries");
    void *stream = stream_for(x, {&w.codes, &w.scales, &w.alpha, &offsets});
    int64_t ldo;
    at::Tensor out = result_for(a[8], x, r.rows, BACKWARD ? w.k : w.n, &ldo);
    const size_t need = (BACKWARD ? qnn_g4_expert_backward_data_workspace : qnn_g4_expert_gemm_workspace)(x.data_ptr(), r.type, r.rows, r.ld,
                                                                                                      (int)w.experts, (int)w.n, (int)w.k);
    const at::Tensor ws = workspace_for(a[9], need, x);
    const int status = (BACKWARD ? qnn_g4_expert_backward_data : qnn_g4_expert_gemm)(
        x.data_ptr(), r.type, r.rows, r.ld, (const int32_t *)offsets.data_ptr(), (int)w.experts, (const uint32_t *)w.codes.data_ptr(),
        (const uint8_t *)w.scales.data_ptr(), (const float *)w.alpha.data_ptr(), (int)w.n, (int)w.k, (int)w.group, out.data_ptr(), ldo,
        ws.defined() ? ws.data_ptr() : nullptr, ws.defined() ? ws.nbytes() : 0, stream);
    return answer(status, std::move(out));
}

// expert_gemm_backward_weights(dy, x, offsets, gw, workspace)
PyObject *expert_weights(PyObject *const *a) {
    const at::Tensor &dy = tensor_of(a[0], "dy must be a tensor"), &x = tensor_of(a[1], "x must be a tensor");
    const Rows d = rows_of(dy, -1), r = rows_of(x, -1);
    if (d.type != r.type || d.rows != r.rows) throw Refused("dy and x must have the same type and number of rows");
    const at::Tensor &offsets = tensor_of(a[2], "offsets must be a tensor");
    const int64_t experts = experts_of(offsets), n = dy.size(1), k = x.size(1);
    void *stream = stream_for(x, {&dy, &offsets});
    at::Tensor gw;
    if (given(a[3])) {
        gw = tensor_of(a[3], "gw must be a tensor");
        check_no_graph(gw);
        if (gw.scalar_type() != at::kFloat || !gw.is_contiguous() || !gw.is_cuda() || gw.get_device() != x.get_device() || gw.dim() != 3 ||
            gw.size(0) != experts || gw.size(1) != n || gw.size(2) != k)
            throw Refused("gw must be contiguous float32 [experts, n, k] on the device of the rows");
    } else {
        gw = at::empty({experts, n, k}, x.options().dtype(at::kFloat));
    }
    const bool sizes = experts <= INT32_MAX && n <= INT32_MAX && k <= INT32_MAX;
    const size_t need = sizes ? qnn_expert_backward_weights_workspace(dy.data_ptr(), x.data_ptr(), d.type, d.rows, d.ld, r.ld, (int)experts, (int)n, (int)k) : 0;
    const at::Tensor ws = workspace_for(a[4], need, x);
    const int status = !sizes ? (int)QNN_E_RANGE
                              : qnn_expert_backward_weights(dy.data_ptr(), x.data_ptr(), d.type, d.rows, d.ld, r.ld, (const int32_t *)offsets.data_ptr(),
                                                            (int)experts, (int)n, (int)k, (float *)gw.data_ptr(), ws.defined() ? ws.data_ptr() : nullptr,
                                                            ws.defined() ? ws.nbytes() : 0, stream);
    return answer(status, std::move(gw));
}

// ------------------------------------------------------------------------------------------------ rows in 8 bits, norms, routing

int64_t whole_units(int64_t k) { return (k + 15) / 16 * 16; }
void check_int(int64_t v) {
    if (v > INT32_MAX) throw Refused("a size does not fit 32 bits");
}
int64_t int_of(PyObject *o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
float float_of(PyObject *o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return (float)v;
}
void *pointer(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

// The results of one call.  Small ones lie in one allocation, each on 16 bytes: an allocation takes half a microsecond, and a decoding
// step's results are small.  One that is kept then keeps the others' memory too, 256 KB at most, and one that is saved is saved with
// all of it (both: clone it).  Larger ones have allocations of their own.
class Results {
  public:
    Results(const at::Tensor &like) : like_(like) {}
    // an array of rows x width elements, rows `ld` apart; 0 rows of anything is an empty array
    void add(at::Tensor &t, at::ScalarType type, int64_t rows, int64_t width, int64_t ld) { parts_[count_++] = {&t, type, rows, width, ld, false}; }
    void add(at::Tensor &t, at::ScalarType type, int64_t size) { parts_[count_++] = {&t, type, size, 1, 1, true}; }
    void make() {
        int64_t total = 0;
        for (int i = 0; i < count_; ++i) total += bytes(parts_[i]);
        if (total > TOGETHER || count_ == 1) {
            for (int i = 0; i < count_; ++i) {
                const Part &p = parts_[i];
                *p.t = p.flat ? new_array(like_, p.type, {p.rows}) : p.ld == p.width ? new_array(like_, p.type, {p.rows, p.width})
                                                                                     : at::empty_strided({p.rows, p.width}, {p.ld, 1}, like_.options().dtype(p.type));
            }
            return;
        }
        const at::Tensor all = new_array(like_, at::kByte, {total});
        int64_t at_byte = 0;
        for (int i = 0; i < count_; ++i) {
            const Part &p = parts_[i];
            *p.t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(p.type));
            c10::TensorImpl *impl = p.t->unsafeGetTensorImpl();
            const int64_t size = (int64_t)c10::elementSize(p.type);
            const std::array<int64_t, 2> sizes{p.rows, p.width}, strides{p.flat ? 1 : p.ld, 1};
            const size_t dims = p.flat ? 1 : 2;
            impl->set_sizes_and_strides(at::IntArrayRef(sizes.data(), dims), at::IntArrayRef(strides.data(), dims), at_byte / size);
            at_byte += bytes(p);
        }
    }

  private:
    static constexpr int64_t TOGETHER = 256 * 1024;
    struct Part {
        at::Tensor *t;
        at::ScalarType type;
        int64_t rows, width, ld;
        bool flat;
    };
    static int64_t bytes(const Part &p) { return whole_units(p.rows * p.ld * (int64_t)c10::elementSize(p.type)); }
    const at::Tensor &like_;
    Part parts_[6];
    int count_ = 0;
};

// A tuple of results, or the status.
PyObject *answers(int status, std::initializer_list<at::Tensor *> results) {
    if (status != QNN_OK) return PyLong_FromLong(status);
    PyObject *tuple = PyTuple_New((Py_ssize_t)results.size());
    if (!tuple) throw python_error();
    Py_ssize_t i = 0;
    for (at::Tensor *t : results) PyTuple_SET_ITEM(tuple, i++, THPVariable_Wrap(std::move(*t)));
    return tuple;
}

// An optional tensor of `size` contiguous elements of a type.
at::Tensor vector_of(PyObject *o, at::ScalarType type, int64_t size, const char *what) {
    if (!given(o)) return at::Tensor();
    const at::Tensor &t = tensor_of(o, what);
    check_no_graph(t);
    if (t.scalar_type() != type || t.numel() != size || !t.is_contiguous()) throw Refused(what);
    return t;
}

struct Codes {
    const at::Tensor &codes, &scales;
    int64_t rows, k, ld;
};
// args: codes int8 [rows, k], scales fp32 [rows]
Codes codes_of(PyObject *const *a) {
    Codes c{tensor_of(a[0], "codes must be a tensor"), tensor_of(a[1], "scales must be a tensor"), 0, 0, 0};
    check_no_graph(c.scales);
    if (c.codes.scalar_type() != at::kChar || c.codes.dim() != 2 || c.scales.scalar_type() != at::kFloat || c.scales.dim() != 1 || !c.scales.is_contiguous())
        throw Refused("rows in 8 bits are codes int8 [rows, k] and contiguous scales float32 [rows]");
    c.rows = c.codes.size(0);
    c.k = c.codes.size(1);
    c.ld = c.rows > 1 ? c.codes.stride(0) : std::max(c.codes.stride(0), whole_units(c.k));
    if (c.rows <= 1 && c.ld % 16 != 0) c.ld = whole_units(c.ld);
    if (c.scales.size(0) != c.rows) throw Refused("codes and scales must have the same number of rows");
    if ((c.k > 1 && c.rows > 0 && c.codes.stride(1) != 1) || c.ld < c.k) throw Refused("rows of codes must be contiguous and must not overlap");
    check_int(c.k);
    return c;
}
void check_like(const at::Tensor &t, const Rows &r, const at::Tensor &like, const Rows &l) {
    if (r.type != l.type || r.rows != l.rows || t.size(1) != like.size(1)) throw Refused("all rows must have the same type and shape");
}

// i8_quantize(x)
PyObject *i8_quantize(PyObject *const *a) {
    const at::Tensor &x = tensor_of(a[0], "x must be a tensor");
    const Rows r = rows_of(x, -1);
    const int64_t k = x.size(1);
    check_int(k);
    void *stream = stream_for(x, {});
    at::Tensor codes, scales;
    Results results(x);
    results.add(codes, at::kChar, r.rows, k, whole_units(k));
    results.add(scales, at::kFloat, r.rows);
    results.make();
    const int status = qnn_i8_quantize(x.data_ptr(), r.type, r.rows, (int)k, r.ld, (int8_t *)codes.data_ptr(), whole_units(k), (float *)scales.data_ptr(), stream);
    return answers(status, {&codes, &scales});
}

at::ScalarType real_type_of(PyObject *o) {
    if (!THPDtype_Check(o)) throw Refused("dtype must be a torch.dtype");
    const at::ScalarType t = reinterpret_cast<THPDtype *>(o)->scalar_type;
    if (t != at::kFloat && t != at::kBFloat16 && t != at::kHalf) throw Refused("dtype must be float32, bfloat16 or float16");
    return t;
}
int code_of(at::ScalarType t) { return t == at::kFloat ? QNN_F32 : t == at::kBFloat16 ? QNN_BF16 : QNN_F16; }
// Rows of a result: as given, checked, or new.
at::Tensor rows_for(PyObject *out, const at::Tensor &like, at::ScalarType type, int64_t rows, int64_t width, int64_t *ld) {
    if (!given(out)) {
        *ld = width;
        return new_array(like, type, {rows, width});
    }
    const at::Tensor &t = tensor_of(out, "out must be a tensor");
    const Rows r = rows_of(t, width);
    if (t.scalar_type() != type || r.rows != rows || !t.is_cuda() || t.get_device() != like.get_device())
        throw Refused("out must be [rows, width] of the result's type and on the device of the rows");
    *ld = r.ld;
    return t;
}

// i8_decode(codes, scales, dtype, out)
PyObject *i8_decode(PyObject *const *a) {
    const Codes c = codes_of(a);
    const at::ScalarType type = real_type_of(a[2]);
    void *stream = stream_for(c.codes, {&c.scales});
    int64_t ld;
    at::Tensor out = rows_for(a[3], c.codes, type, c.rows, c.k, &ld);
    const int status = qnn_i8_decode((const int8_t *)c.codes.data_ptr(), (const float *)c.scales.data_ptr(), c.rows, (int)c.k, c.ld, code_of(type),
                                     out.data_ptr(), ld, stream);
    return answer(status, std::move(out));
}

// i8_gemm(x codes, x scales, w codes, w scales, dtype, bias, out)
PyObject *i8_gemm(PyObject *const *a) {
    const Codes x = codes_of(a), w = codes_of(a + 2);
    if (x.k != w.k) throw Refused("rows and weights must have the same length");
    check_int(w.rows);
    const at::ScalarType type = real_type_of(a[4]);
    const at::Tensor bias = vector_of(a[5], at::kFloat, w.rows, "bias must be contiguous float32 [features]");
    void *stream = bias.defined() ? stream_for(x.codes, {&x.scales, &w.codes, &w.scales, &bias}) : stream_for(x.codes, {&x.scales, &w.codes, &w.scales});
    int64_t ld;
    at::Tensor out = rows_for(a[6], x.codes, type, x.rows, w.rows, &ld);
    const int status = qnn_i8_gemm((const int8_t *)x.codes.data_ptr(), (const float *)x.scales.data_ptr(), x.rows, x.ld, (const int8_t *)w.codes.data_ptr(),
                                   (const float *)w.scales.data_ptr(), (int)w.rows, (int)w.k, w.ld, (const float *)pointer(bias), code_of(type),
                                   out.data_ptr(), ld, stream);
    return answer(status, std::move(out));
}

// The gain of a norm: [width] of the rows' type or float32.
const at::Tensor &gain_of(PyObject *o, const Rows &r, int64_t width, int *type) {
    const at::Tensor &g = tensor_of(o, "gain must be a tensor");
    check_no_graph(g);
    *type = type_of(g);
    if (g.dim() != 1 || g.size(0) != width || !g.is_contiguous() || (*type != r.type && *type != QNN_F32))
        throw Refused("gain must be contiguous [width] of the rows' type or float32");
    return g;
}

// rms_norm(x, gain, eps, residual, real, eight): (y, codes, scales, h, rstd), None for what is not asked for; h is x without a residual
PyObject *rms_norm(PyObject *const *a) {
    const at::Tensor &x = tensor_of(a[0], "x must be a tensor");
    const Rows r = rows_of(x, -1);
    const int64_t k = x.size(1);
    check_int(k);
    int gain_type;
    const at::Tensor &gain = gain_of(a[1], r, k, &gain_type);
    const float eps = float_of(a[2]);
    const bool real = PyObject_IsTrue(a[4]) == 1, eight = PyObject_IsTrue(a[5]) == 1;
    at::Tensor residual, h, y, codes, scales, rstd;
    Results results(x);
    int64_t ldr = 0;
    void *stream;
    if (given(a[3])) {
        residual = tensor_of(a[3], "residual must be a tensor");
        const Rows q = rows_of(residual, k);
        check_like(residual, q, x, r);
        ldr = q.ld;
        stream = stream_for(x, {&gain, &residual});
        results.add(h, x.scalar_type(), r.rows, k, k);
    } else {
        stream = stream_for(x, {&gain});
    }
    if (real) results.add(y, x.scalar_type(), r.rows, k, k);
    if (eight) {
        results.add(codes, at::kChar, r.rows, k, whole_units(k));
        results.add(scales, at::kFloat, r.rows);
    }
    results.add(rstd, at::kFloat, r.rows);
    results.make();
    const int status = qnn_rms_norm(x.data_ptr(), r.type, r.rows, (int)k, r.ld, pointer(residual), ldr, gain.data_ptr(), gain_type, eps, pointer(h), k,
                                    pointer(y), k, (int8_t *)pointer(codes), whole_units(k), (float *)pointer(scales), (float *)rstd.data_ptr(), stream);
    if (!h.defined()) h = x;
    return answers(status, {&y, &codes, &scales, &h, &rstd});
}

// rms_norm_backward(dy, h, gain, rstd, dh, workspace): (dx, dgain)
PyObject *rms_norm_backward(PyObject *const *a) {
    const at::Tensor &dy = tensor_of(a[0], "dy must be a tensor"), &h = tensor_of(a[1], "h must be a tensor");
    const Rows r = rows_of(dy, -1), q = rows_of(h, -1);
    check_like(h, q, dy, r);
    const int64_t k = dy.size(1);
    check_int(k);
    int gain_type;
    const at::Tensor &gain = gain_of(a[2], r, k, &gain_type);
    if (!given(a[3])) throw Refused("rstd must be contiguous float32 [rows]");
    const at::Tensor rstd = vector_of(a[3], at::kFloat, r.rows, "rstd must be contiguous float32 [rows]");
    at::Tensor dh;
    int64_t lddh = 0;
    void *stream;
    if (given(a[4])) {
        dh = tensor_of(a[4], "dh must be a tensor");
        const Rows d = rows_of(dh, k);
        check_like(dh, d, dy, r);
        lddh = d.ld;
        stream = stream_for(dy, {&h, &gain, &rstd, &dh});
    } else {
        stream = stream_for(dy, {&h, &gain, &rstd});
    }
    at::Tensor dx, dgain;
    Results results(dy);
    results.add(dx, dy.scalar_type(), r.rows, k, k);
    results.add(dgain, at::kFloat, k);
    results.make();
    const at::Tensor ws = workspace_for(a[5], qnn_rms_norm_backward_workspace(r.rows, (int)k), dy);
    const int status = qnn_rms_norm_backward(dy.data_ptr(), r.type, r.rows, (int)k, r.ld, h.data_ptr(), q.ld, gain.data_ptr(), gain_type,
                                             (const float *)rstd.data_ptr(), pointer(dh), lddh, dx.data_ptr(), k, (float *)dgain.data_ptr(), pointer(ws),
                                             ws.defined() ? ws.nbytes() : 0, stream);
    return answers(status, {&dx, &dgain});
}

// route(logits, top, flags, bias, groups, top_groups, factor, mask, workspace): (experts, weights, order, place, offsets)
PyObject *route(PyObject *const *a) {
    const at::Tensor &logits = tensor_of(a[0], "logits must be a tensor");
    const Rows r = rows_of(logits, -1);
    const int64_t experts = logits.size(1), top = int_of(a[1]), groups = int_of(a[4]), top_groups = int_of(a[5]);
    if (experts > 1024 || top < 1 || top > 32 || groups < 1 || groups > 32 || top_groups < 1 || top_groups > 32) return PyLong_FromLong(QNN_E_ARG);
    const at::Tensor bias = vector_of(a[3], at::kFloat, experts, "bias must be contiguous float32 [experts]");
    at::Tensor mask;
    if (given(a[7])) {
        mask = tensor_of(a[7], "mask must be a tensor");
        if ((mask.scalar_type() != at::kBool && mask.scalar_type() != at::kByte) || mask.numel() != r.rows || !mask.is_contiguous())
            throw Refused("mask must be contiguous bool or uint8 [tokens]");
    }
    void *stream = stream_for(logits, {});
    for (const at::Tensor *t : std::initializer_list<const at::Tensor *>{&bias, &mask})
        if (t->defined()) stream_for(*t, {&logits});
    at::Tensor chosen, weights, order, place, offsets;
    Results results(logits);
    results.add(chosen, at::kInt, r.rows, top, top);
    results.add(weights, at::kFloat, r.rows, top, top);
    results.add(order, at::kInt, r.rows * top);
    results.add(place, at::kInt, r.rows, top, top);
    results.add(offsets, at::kInt, experts + 1);
    results.make();
    const at::Tensor ws = workspace_for(a[8], qnn_route_workspace(r.rows, (int)experts, (int)top), logits);
    const int status = qnn_route(logits.data_ptr(), r.type, r.rows, (int)experts, r.ld, (int)top, (unsigned)int_of(a[2]), (const float *)pointer(bias),
                                 (int)groups, (int)top_groups, float_of(a[6]), (const uint8_t *)pointer(mask), (int32_t *)chosen.data_ptr(),
                                 (float *)weights.data_ptr(), (int32_t *)order.data_ptr(), (int32_t *)place.data_ptr(), (int32_t *)offsets.data_ptr(),
                                 pointer(ws), ws.defined() ? ws.nbytes() : 0, stream);
    return answers(status, {&chosen, &weights, &order, &place, &offsets});
}

// route_backward(dweights, logits, experts, flags, factor, out)
PyObject *route_backward(PyObject *const *a) {
    const at::Tensor &dweights = tensor_of(a[0], "dweights must be a tensor"), &logits = tensor_of(a[1], "logits must be a tensor"),
                     &chosen = tensor_of(a[2], "experts must be a tensor");
    const Rows r = rows_of(logits, -1);
    check_no_graph(dweights);
    if (dweights.scalar_type() != at::kFloat || chosen.scalar_type() != at::kInt || dweights.dim() != 2 || chosen.dim() != 2 ||
        dweights.sizes() != chosen.sizes() || dweights.size(0) != r.rows || !dweights.is_contiguous() || !chosen.is_contiguous())
        throw Refused("dweights and experts must be contiguous float32 and int32 [tokens, top]");
    const int64_t experts = logits.size(1), top = chosen.size(1);
    if (experts > 1024 || top > 32) return PyLong_FromLong(QNN_E_ARG);
    void *stream = stream_for(logits, {&dweights, &chosen});
    int64_t ld;
    at::Tensor out = result_for(a[5], logits, r.rows, experts, &ld);
    const int status = qnn_route_backward((const float *)dweights.data_ptr(), logits.data_ptr(), r.type, r.rows, (int)experts, r.ld, (int)top,
                                          (unsigned)int_of(a[3]), (const int32_t *)chosen.data_ptr(), float_of(a[4]), out.data_ptr(), ld, stream);
    return answer(status, std::move(out));
}

template <PyObject *(*F)(PyObject *const *), int ARGS>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    if (count != ARGS) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Refused &e) {
        PyErr_SetString(PyExc_ValueError, e.what());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"g4_matvec", (PyCFunction)(void (*)(void))entry<g4_matvec, 9>, METH_FASTCALL, nullptr},
    {"g4_expert_gemm", (PyCFunction)(void (*)(void))entry<g4_expert<false>, 10>, METH_FASTCALL, nullptr},
    {"g4_expert_gemm_backward_data", (PyCFunction)(void (*)(void))entry<g4_expert<true>, 10>, METH_FASTCALL, nullptr},
    {"expert_gemm_backward_weights", (PyCFunction)(void (*)(void))entry<expert_weights, 5>, METH_FASTCALL, nullptr},
    {"i8_quantize", (PyCFunction)(void (*)(void))entry<i8_quantize, 1>, METH_FASTCALL, nullptr},
    {"i8_decode", (PyCFunction)(void (*)(void))entry<i8_decode, 4>, METH_FASTCALL, nullptr},
    {"i8_gemm", (PyCFunction)(void (*)(void))entry<i8_gemm, 7>, METH_FASTCALL, nullptr},
    {"rms_norm", (PyCFunction)(void (*)(void))entry<rms_norm, 6>, METH_FASTCALL, nullptr},
    {"rms_norm_backward", (PyCFunction)(void (*)(void))entry<rms_norm_backward, 6>, METH_FASTCALL, nullptr},
    {"route", (PyCFunction)(void (*)(void))entry<route, 9>, METH_FASTCALL, nullptr},
    {"route_backward", (PyCFunction)(void (*)(void))entry<route_backward, 6>, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "tensor arguments of the calls of a decoding step", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
