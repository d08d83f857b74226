// The usual calls of the operators of lm_train_api.cu, from torch tensors to the C ABI without the interpreter in between: a call on small tensors is as long as
// its host side takes (with ctypes 10 to 13 us, 5 of them the launch). "Usual" means plain CUDA tensors on the current device, torch's current stream, results
// allocated here. Whatever is not usual, or not right, gives None, and operators.py does it, or says what is wrong with it.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <algorithm>
#include <exception>
#include <vector>

#include "a2cid2.h"

namespace {

PyObject* g_error = nullptr;  // binding.A2Error

// An argument that is not as usual.
struct Unusual {};

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) throw Unusual();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.requires_grad() && at::GradMode::is_enabled()) throw Unusual();
    return t;
}
int64_t whole(PyObject* o) {
    if (!PyLong_CheckExact(o)) throw Unusual();
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Unusual();
    }
    return v;
}
double number(PyObject* o) {
    if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
    return (double)whole(o);
}
int32_t code_of(at::ScalarType t) {
    if (t == at::kFloat) return A2_F32;
    if (t == at::kBFloat16) return A2_BF16;
    throw Unusual();
}
void need(bool ok) {
    if (!ok) throw Unusual();
}

struct Matrix {
    const at::Tensor& t;
    int64_t rows, cols, pitch;
    explicit Matrix(const at::Tensor& m) : t(m) {
        need(m.dim() == 2);
        rows = m.size(0), cols = m.size(1);
        need(cols == 1 || m.stride(1) == 1);
        pitch = rows > 1 ? m.stride(0) : std::max<int64_t>(cols, 1);
    }
};

// The matrix that says device and type of a call: on the current device.
struct First : Matrix {
    int32_t type;
    explicit First(PyObject* o) : Matrix(tensor(o)) {
        need(t.is_cuda() && t.device().index() == c10::cuda::current_device());
        type = code_of(t.scalar_type());
    }
    Matrix like(PyObject* o) const {  // another one of its shape
        const at::Tensor& m = tensor(o);
        need(m.scalar_type() == t.scalar_type() && m.device() == t.device());
        Matrix r(m);
        need(r.rows == rows && r.cols == cols);
        return r;
    }
    const void* vector(PyObject* o, int64_t n, at::ScalarType type) const {  // or NULL for None
        if (o == Py_None) return nullptr;
        const at::Tensor& v = tensor(o);
        need(v.scalar_type() == type && v.device() == t.device() && v.dim() == 1 && v.size(0) == n && v.is_contiguous());
        return v.const_data_ptr();
    }
    at::Tensor make(at::IntArrayRef sizes) const { return at::empty(sizes, t.options()); }
    at::Tensor make(at::IntArrayRef sizes, at::ScalarType type) const { return at::empty(sizes, t.options().dtype(type)); }
    void* stream() const { return c10::cuda::getCurrentCUDAStream(t.device().index()).stream(); }
};

// Workspace of the size that the library asks for.
struct Workspace {
    at::Tensor t;
    Workspace(const First& like, int64_t bytes) {
        if (bytes) t = like.make({bytes}, at::kByte);
    }
    void* address() const { return t.defined() ? t.data_ptr() : nullptr; }
    int64_t bytes() const { return t.defined() ? t.size(0) : 0; }
};

struct Failed {};  // a Python error is set

void check(int code) {
    if (code == A2_OK) return;
    PyObject* e = g_error ? PyObject_CallFunction(g_error, "is", code, a2cid2_last_error(nullptr)) : nullptr;
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
        PyErr_SetString(PyExc_RuntimeError, a2cid2_last_error(nullptr));
    }
    throw Failed();
}

PyObject* wrap(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    PyObject* o = THPVariable_Wrap(t);
    if (!o) throw Failed();
    return o;
}
PyObject* tuple(std::initializer_list<at::Tensor> all) {
    PyObject* r = PyTuple_New((Py_ssize_t)all.size());
    if (!r) throw Failed();
    Py_ssize_t i = 0;
    for (const at::Tensor& t : all) {
        PyObject* o = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
        if (!o) {
            Py_DECREF(r);
            throw Failed();
        }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}

// No C++ exception leaves a function of the module.
template <PyObject* (*F)(PyObject* const*)>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n, Py_ssize_t wanted) {
    if (n != wanted) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Unusual&) {
        Py_RETURN_NONE;
    } catch (const Failed&) {
        return nullptr;
    } catch (const std::exception& e) {  // out of memory and the like: torch's own error comes from the other way
        Py_RETURN_NONE;
    }
}

// x, weight, residual, eps
PyObject* rms_norm(PyObject* const* a) {
    const First x(a[0]);
    const void* weight = x.vector(a[1], x.cols, x.t.scalar_type());
    const double eps = number(a[3]);
    const bool with = a[2] != Py_None;
    const void* residual = nullptr;
    int64_t pitch = 0;
    if (with) {
        const Matrix r = x.like(a[2]);
        residual = r.t.const_data_ptr(), pitch = r.pitch;
    }
    at::Tensor out = x.make({x.rows, x.cols}), sum;
    if (with) sum = x.make({x.rows, x.cols});
    check(a2cid2_rms_norm(x.t.const_data_ptr(), x.pitch, residual, pitch, weight, x.rows, x.cols, eps, with ? sum.data_ptr() : nullptr, x.cols, out.data_ptr(), x.cols,
                          x.type, x.stream()));
    return with ? tuple({out, sum}) : wrap(out);
}

// x, weight, residual, eps, block
PyObject* rms_norm_quantized(PyObject* const* a) {
    const First x(a[0]);
    const void* weight = x.vector(a[1], x.cols, x.t.scalar_type());
    const double eps = number(a[3]);
    const int64_t block = whole(a[4]);
    need(block == 0 || block == 32 || block == 64 || block == 128);
    const bool with = a[2] != Py_None;
    const void* residual = nullptr;
    int64_t pitch = 0;
    if (with) {
        const Matrix r = x.like(a[2]);
        residual = r.t.const_data_ptr(), pitch = r.pitch;
    }
    at::Tensor values = x.make({x.rows, x.cols}, at::kFloat8_e4m3fn), scales = x.make({x.rows, block ? (x.cols + block - 1) / block : 1}, at::kFloat), sum;
    if (with) sum = x.make({x.rows, x.cols});
    check(a2cid2_rms_norm_e4m3(x.t.const_data_ptr(), x.pitch, residual, pitch, weight, x.rows, x.cols, eps, with ? sum.data_ptr() : nullptr, x.cols, block, values.data_ptr(),
                               x.cols, scales.data_ptr<float>(), x.type, x.stream()));
    return with ? tuple({values, scales, sum}) : tuple({values, scales});
}

// grad_out, x, weight, eps, grad_sum, whether grad_x and grad_weight are wanted
PyObject* rms_norm_grad(PyObject* const* a) {
    const First g(a[0]);
    const Matrix x = g.like(a[1]);
    const void* weight = g.vector(a[2], g.cols, g.t.scalar_type());
    const double eps = number(a[3]);
    const void* sum = nullptr;
    int64_t pitch = 0;
    if (a[4] != Py_None) {
        const Matrix s = g.like(a[4]);
        sum = s.t.const_data_ptr(), pitch = s.pitch;
    }
    const bool want_x = a[5] == Py_True, want_weight = a[6] == Py_True && weight;
    int64_t bytes = 0;
    check(a2cid2_rms_norm_grad_workspace(g.rows, g.cols, want_weight, g.type, &bytes));
    at::Tensor gx, gw;
    if (want_x) gx = g.make({g.rows, g.cols});
    if (want_weight) gw = g.make({g.cols});
    const Workspace ws(g, bytes);
    check(a2cid2_rms_norm_grad(g.t.const_data_ptr(), g.pitch, x.t.const_data_ptr(), x.pitch, weight, sum, pitch, g.rows, g.cols, eps, want_x ? gx.data_ptr() : nullptr, g.cols,
                               want_weight ? gw.data_ptr() : nullptr, g.type, ws.address(), ws.bytes(), g.stream()));
    return tuple({gx, gw});
}

// logits, k, score, bias, groups, top_groups, group_score, renormalize, scale
PyObject* route(PyObject* const* a) {
    const First z(a[0]);
    const int64_t k = whole(a[1]), score = whole(a[2]), groups = whole(a[4]), top_groups = whole(a[5]), group_score = whole(a[6]);
    need(k >= 1 && k <= z.cols);
    const void* bias = z.vector(a[3], z.cols, at::kFloat);
    const double scale = number(a[8]);
    at::Tensor ids = z.make({z.rows, k}, at::kInt), weights = z.make({z.rows, k}, at::kFloat), counts = z.make({z.cols}, at::kInt);
    check(a2cid2_route(z.t.const_data_ptr(), z.pitch, z.rows, z.cols, k, (int32_t)score, static_cast<const float*>(bias), groups, top_groups, (int32_t)group_score,
                       a[7] == Py_True, scale, ids.data_ptr<int32_t>(), weights.data_ptr<float>(), counts.data_ptr<int32_t>(), z.type, z.stream()));
    return tuple({ids, weights, counts});
}

// logits, ids, grad_weights, score, renormalize, scale
PyObject* route_grad(PyObject* const* a) {
    const First z(a[0]);
    const at::Tensor &ids = tensor(a[1]), &g = tensor(a[2]);
    need(ids.scalar_type() == at::kInt && g.scalar_type() == at::kFloat && ids.device() == z.t.device() && g.device() == z.t.device());
    need(ids.dim() == 2 && g.dim() == 2 && ids.size(0) == z.rows && g.size(0) == z.rows && ids.size(1) == g.size(1) && ids.is_contiguous() && g.is_contiguous());
    const int64_t score = whole(a[3]);
    const double scale = number(a[5]);
    at::Tensor out = z.make({z.rows, z.cols});
    check(a2cid2_route_grad(z.t.const_data_ptr(), z.pitch, ids.const_data_ptr<int32_t>(), g.const_data_ptr<float>(), z.rows, z.cols, ids.size(1), (int32_t)score,
                            a[4] == Py_True, scale, out.data_ptr(), z.cols, z.type, z.stream()));
    return wrap(out);
}

// The tensors of a list, or of a tuple, on the current device, with what the library wants to know of each.
void describe(const at::Tensor& t, const at::Tensor& o, bool per_worker, bool written, a2cid2_gradient_t& g) {
    void* const out = written ? o.mutable_data_ptr() : nullptr;
    g = {t.const_data_ptr(), out, 0, 0, 1, t.numel(), 0, 0, code_of(t.scalar_type())};
    if (per_worker) {
        // a worker's part of a tensor is one piece of memory
        g.cols = 1;
        for (int64_t d = t.dim() - 1; d >= 1; --d) {
            need(t.size(d) == 1 || (t.stride(d) == g.cols && o.stride(d) == g.cols));
            g.cols *= t.size(d);
        }
        if (t.size(0) > 1) g.worker_stride = t.stride(0), g.out_worker_stride = o.stride(0);
    } else {
        need(t.is_contiguous() && o.is_contiguous());
    }
    g.pitch = g.out_pitch = g.cols;
}

// tensors, out (or None: in place), per_worker, max_norm (or None: the norms alone), zero_nonfinite
PyObject* clip(PyObject* const* a) {
    need((PyList_CheckExact(a[0]) || PyTuple_CheckExact(a[0])) && (a[1] == Py_None || PyList_CheckExact(a[1]) || PyTuple_CheckExact(a[1])));
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
    need(n > 0 && (a[1] == Py_None || PySequence_Fast_GET_SIZE(a[1]) == n));
    const bool per_worker = a[2] == Py_True, norms_alone = a[3] == Py_None;
    const double max_norm = norms_alone ? 0.0 : number(a[3]);
    std::vector<a2cid2_gradient_t> all((size_t)n);
    const int device = c10::cuda::current_device();
    int64_t workers = 1;
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* const one = PySequence_Fast_GET_ITEM(a[0], i);
        const at::Tensor& t = tensor(one);
        const at::Tensor& o = a[1] == Py_None ? t : tensor(PySequence_Fast_GET_ITEM(a[1], i));
        need(t.is_cuda() && t.device().index() == device && o.device() == t.device() && o.scalar_type() == t.scalar_type() && o.sizes() == t.sizes());
        if (per_worker) {
            need(t.dim() >= 1 && (i == 0 || t.size(0) == workers) && t.numel() > 0);
            workers = t.size(0);
        }
        describe(t, o, per_worker, !norms_alone, all[(size_t)i]);
    }
    int64_t bytes = 0;
    check(a2cid2_clip_gradients_workspace(n, workers, &bytes));
    const at::Tensor& any = THPVariable_Unpack(PySequence_Fast_GET_ITEM(a[0], 0));
    const auto options = any.options();
    at::Tensor norms = per_worker ? at::empty({workers}, options.dtype(at::kFloat)) : at::empty({}, options.dtype(at::kFloat));
    const at::Tensor ws = at::empty({bytes}, options.dtype(at::kByte));
    void* const stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    check(norms_alone ? a2cid2_gradient_norms(all.data(), n, workers, norms.data_ptr<float>(), ws.data_ptr(), bytes, stream)
                      : a2cid2_clip_gradients(all.data(), n, workers, max_norm, a[4] == Py_True, norms.data_ptr<float>(), ws.data_ptr(), bytes, stream));
    return wrap(norms);
}

// values, scales, dtype: 0 float32, 1 bfloat16
PyObject* dequantize(PyObject* const* a) {
    const Matrix v(tensor(a[0]));
    const at::Tensor& scales = tensor(a[1]);
    need(v.t.is_cuda() && v.t.device().index() == c10::cuda::current_device() && v.t.scalar_type() == at::kFloat8_e4m3fn);
    need(scales.scalar_type() == at::kFloat && scales.device() == v.t.device() && scales.dim() == 2 && scales.size(0) == v.rows && scales.is_contiguous());
    const int64_t blocks = scales.size(1), type = whole(a[2]);
    int64_t block = 0;
    if (blocks != 1)
        for (const int64_t b : {128, 64, 32})
            if ((v.cols + b - 1) / b == blocks) block = b;
    need(blocks == 1 || block != 0);
    at::Tensor out = at::empty({v.rows, v.cols}, v.t.options().dtype(type == A2_BF16 ? at::kBFloat16 : at::kFloat));
    check(a2cid2_dequantize_e4m3(v.t.const_data_ptr(), v.pitch, scales.const_data_ptr<float>(), v.rows, v.cols, block, out.data_ptr(), v.cols, (int32_t)type,
                                 c10::cuda::getCurrentCUDAStream(v.t.device().index()).stream()));
    return wrap(out);
}

PyObject* set_error(PyObject* const* a) {
    Py_XSETREF(g_error, Py_NewRef(a[0]));
    Py_RETURN_NONE;
}

#define A2_CALL(name, count) \
    {#name, reinterpret_cast<PyCFunction>(static_cast<PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t)>( \
         [](PyObject* self, PyObject* const* args, Py_ssize_t n) { return guarded<name>(self, args, n, count); })), METH_FASTCALL, nullptr}

PyMethodDef g_methods[] = {A2_CALL(rms_norm, 4), A2_CALL(rms_norm_quantized, 5), A2_CALL(rms_norm_grad, 7), A2_CALL(route, 9), A2_CALL(route_grad, 6),
                           A2_CALL(clip, 5), A2_CALL(dequantize, 3), A2_CALL(set_error, 1), {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&g_module); }
