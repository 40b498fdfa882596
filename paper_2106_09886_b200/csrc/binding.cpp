// Tensor arguments of the 4-bit-weight calls -> the C ABI (include/qnn.h): checks, the result's allocation on the current
// stream, and the call, in one step from Python.  A step of decoding makes these calls for every layer with microseconds of
// work each; through ctypes the marshalling alone took longer than the small ones run (a call with a new result 10.7 us, of which
// 2.9 the launch, and 4.5 here; with a result given 8.9 and 3.4).
// Argument marshalling only: every step of the work runs inside libqnn's kernels.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/core/GradMode.h>
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

// These calls record no gradients: an operand that requires one, while they are recorded, would lose it without a word.
void check_no_graph(const at::Tensor &t) {
    if (t.requires_grad() && c10::GradMode::is_enabled())
        throw Refused("these calls record no gradients: detach tensors that require grad, or call under torch.no_grad()");
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

at::Tensor workspace_for(PyObject *workspace, size_t need, const at::Tensor &like) {
    if (given(workspace)) {
        const at::Tensor &t = tensor_of(workspace, "workspace must be a tensor");
        if (!t.is_cuda() || t.get_device() != like.get_device() || !t.is_contiguous()) throw Refused("workspace must be contiguous on the device of the rows");
        return t;
    }
    return need ? at::empty({(int64_t)need}, like.options().dtype(at::kByte)) : at::Tensor();
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
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", "tensor arguments of the 4-bit-weight calls", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
