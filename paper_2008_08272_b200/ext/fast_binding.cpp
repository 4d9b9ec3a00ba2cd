// The binding's call path in native code: argument checks on torch tensors, allocation of outputs the caller
// did not supply, the current stream, and the C-ABI call, in one C function per operator.  An operator of a
// few microseconds costs more on the host than on the GPU, so this path is what small calls are made of:
// written in Python over ctypes the same steps took 8 to 17 us per call, here 1 to 2 us.
//
// A call that is not entirely ordinary (an argument that is no contiguous fp32 CUDA tensor, a status other
// than OK, a shape that does not fit) returns None without having launched anything, and the Python caller
// repeats it through its checked path, which raises the precise error.
#include <Python.h>
#include <dlfcn.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "onnx_b200.h"

namespace {

struct Abi {
    decltype(&onnx_conv2d_run) conv_run;
    decltype(&onnx_conv2d_add_run) conv_add_run;
    decltype(&onnx_conv2d_run_packed) conv_run_packed;
    decltype(&onnx_conv2d_run_packed_sampled) conv_run_packed_sampled;
    decltype(&onnx_conv2d_run_packed_rounded) conv_run_packed_rounded;
    decltype(&onnx_gemm_workspace_bytes) gemm_workspace_bytes;
    decltype(&onnx_gemm_run) gemm_run;
    decltype(&onnx_maxpool2d_shape) maxpool2d_shape;
    decltype(&onnx_maxpool2d_run) maxpool2d_run;
    decltype(&onnx_global_average_pool_run) global_average_pool_run;
    decltype(&onnxb_dispatch_state) dispatch_state;
    decltype(&onnx_quantize_rows_run) quantize_rows_run;
    decltype(&onnx_gemm_int8_workspace_bytes) gemm_int8_workspace_bytes;
    decltype(&onnx_gemm_int8_run) gemm_int8_run;
    decltype(&onnx_gated_workspace_bytes) gated_workspace_bytes;
    decltype(&onnx_gated_run) gated_run;
    decltype(&onnx_gated_int8_run) gated_int8_run;
    decltype(&onnx_gated_backward_workspace_bytes) gated_backward_workspace_bytes;
    decltype(&onnx_gated_backward_run) gated_backward_run;
} abi;

struct Plan {                    // what a convolution descriptor resolved to
    onnxb_conv2d_desc_t desc;
    int64_t y[4];
    size_t workspace;            // bytes onnx_conv2d_run needs
    size_t packed;               // bytes of the copy of W (0: none)
    bool packed_needs_ws;        // onnx_conv2d_run_packed needs the workspace too
};

// An argument as the library takes it: nullptr for None; `fine` cleared when it is anything but a contiguous
// fp32 CUDA tensor.
inline const float *in_ptr(PyObject *o, bool &fine, const at::Tensor **t = nullptr) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) { fine = false; return nullptr; }
    const at::Tensor &x = THPVariable_Unpack(o);
    if (!x.is_cuda() || x.scalar_type() != at::kFloat || !x.is_contiguous()) { fine = false; return nullptr; }
    if (t) *t = &x;
    return static_cast<const float *>(x.data_ptr());
}

// A workspace tensor of any type, or None.
inline void *ws_ptr(PyObject *o, size_t &bytes, bool &fine) {
    bytes = 0;
    if (o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) { fine = false; return nullptr; }
    const at::Tensor &x = THPVariable_Unpack(o);
    bytes = x.nbytes();
    return x.data_ptr();
}

// (only asked for once the tensors are known to be CUDA tensors: without a device it throws)
inline void *stream_ptr(PyObject *o, bool &fine) {
    if (!fine) return nullptr;
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject *a = PyObject_GetAttrString(o, "cuda_stream");
    if (!a) { PyErr_Clear(); fine = false; return nullptr; }
    void *p = PyLong_AsVoidPtr(a);
    Py_DECREF(a);
    if (PyErr_Occurred()) { PyErr_Clear(); fine = false; }
    return p;
}

// Memory for a call on `st`; `given` is the stream argument it came from.  The allocator hands a block out and takes it back in
// the order of the stream it was made on: made on another than the call's, the block's last user may not have finished when the
// call's kernels begin, nor they when its next one does.  A result goes on to be used from the current stream, too.
inline at::Tensor new_tensor(at::IntArrayRef size, at::ScalarType type, const at::Device &dev, PyObject *given, void *st, bool is_result) {
    if (given != Py_None) {
        const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(dev.index());
        if (current.stream() != st) {
            const c10::cuda::CUDAStreamGuard on(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(st), dev.index()));
            at::Tensor t(at::detail::empty_cuda(size, type, dev, c10::nullopt));
            if (is_result) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), current);
            return t;
        }
    }
    return at::Tensor(at::detail::empty_cuda(size, type, dev, c10::nullopt));
}

// The result: the caller's own Y object, or the tensor made here.
inline PyObject *result(PyObject *given, at::Tensor &made) {
    if (given == Py_None) return THPVariable_Wrap(std::move(made));
    Py_INCREF(given);
    return given;
}

inline PyObject *slow_path() { Py_RETURN_NONE; }

inline Plan *plan_of(PyObject *o) { return static_cast<Plan *>(PyCapsule_GetPointer(o, "onnxb.plan")); }

void plan_free(PyObject *o) { delete plan_of(o); }

// bind(path): resolve the C ABI in the library the ctypes binding has loaded
PyObject *py_bind(PyObject *, PyObject *arg) {
    const char *path = PyUnicode_AsUTF8(arg);
    if (!path) return nullptr;
    void *h = dlopen(path, RTLD_NOW | RTLD_NOLOAD);
    if (!h) { PyErr_SetString(PyExc_OSError, "the library is not loaded"); return nullptr; }
    bool ok = true;
    auto get = [&](auto &fn, const char *name) {
        fn = reinterpret_cast<std::decay_t<decltype(fn)>>(dlsym(h, name));
        ok = ok && fn;
    };
    get(abi.conv_run, "onnx_conv2d_run");
    get(abi.conv_add_run, "onnx_conv2d_add_run");
    get(abi.conv_run_packed, "onnx_conv2d_run_packed");
    get(abi.conv_run_packed_sampled, "onnx_conv2d_run_packed_sampled");
    get(abi.conv_run_packed_rounded, "onnx_conv2d_run_packed_rounded");
    get(abi.gemm_workspace_bytes, "onnx_gemm_workspace_bytes");
    get(abi.gemm_run, "onnx_gemm_run");
    get(abi.maxpool2d_shape, "onnx_maxpool2d_shape");
    get(abi.maxpool2d_run, "onnx_maxpool2d_run");
    get(abi.global_average_pool_run, "onnx_global_average_pool_run");
    get(abi.dispatch_state, "onnxb_dispatch_state");
    get(abi.quantize_rows_run, "onnx_quantize_rows_run");
    get(abi.gemm_int8_workspace_bytes, "onnx_gemm_int8_workspace_bytes");
    get(abi.gemm_int8_run, "onnx_gemm_int8_run");
    get(abi.gated_workspace_bytes, "onnx_gated_workspace_bytes");
    get(abi.gated_run, "onnx_gated_run");
    get(abi.gated_int8_run, "onnx_gated_int8_run");
    get(abi.gated_backward_workspace_bytes, "onnx_gated_backward_workspace_bytes");
    get(abi.gated_backward_run, "onnx_gated_backward_run");
    if (!ok) { PyErr_SetString(PyExc_OSError, "a symbol of the C ABI is missing"); return nullptr; }
    Py_RETURN_NONE;
}

// plan(desc address, (n, m, p, q), workspace bytes, packed bytes, whether a run from the copy needs workspace) -> capsule
PyObject *py_plan(PyObject *, PyObject *args) {
    unsigned long long desc, ws, packed;
    long long y[4];
    int needs;
    if (!PyArg_ParseTuple(args, "K(LLLL)KKp", &desc, &y[0], &y[1], &y[2], &y[3], &ws, &packed, &needs)) return nullptr;
    Plan *p = new Plan{reinterpret_cast<onnxb_conv2d_desc_t>(desc), {y[0], y[1], y[2], y[3]}, (size_t)ws, (size_t)packed, needs != 0};
    return PyCapsule_New(p, "onnxb.plan", plan_free);
}

// n integers of a tuple or list; None leaves the defaults
inline bool ints(PyObject *o, int64_t *out, Py_ssize_t n) {
    if (o == Py_None) return true;
    PyObject *const *items;
    if (PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == n) items = &PyTuple_GET_ITEM(o, 0);
    else if (PyList_CheckExact(o) && PyList_GET_SIZE(o) == n) items = &PyList_GET_ITEM(o, 0);
    else return false;
    for (Py_ssize_t i = 0; i < n; ++i) {
        if (!PyLong_CheckExact(items[i])) return false;
        out[i] = PyLong_AsLongLong(items[i]);
    }
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

// conv(plan, X, W, packed, B, R, Y, workspace, stream): run (packed and R None), run_add (R given) or
// run_packed (packed given); with three more arguments (dims, strides, Y_rounded)
// packed is given, R, of those rows and columns, is read at every such row and column, and Y_rounded, if any, gets Y rounded;
// dims and strides None: R, if any, is read as it lies
PyObject *py_conv(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9 && n != 12) return slow_path();
    Plan *p = plan_of(a[0]);
    if (!p) { PyErr_Clear(); return slow_path(); }
    bool fine = true;
    const at::Tensor *xt = nullptr;
    size_t packed_bytes, ws_bytes;
    const float *x = in_ptr(a[1], fine, &xt), *w = in_ptr(a[2], fine);
    const void *packed = ws_ptr(a[3], packed_bytes, fine);
    const float *b = in_ptr(a[4], fine), *r = in_ptr(a[5], fine);
    float *y = const_cast<float *>(in_ptr(a[6], fine));
    void *ws = ws_ptr(a[7], ws_bytes, fine), *st = stream_ptr(a[8], fine);
    if (!fine || !x || !w) return slow_path();
    const bool pre = a[3] != Py_None;
    int64_t dims[2], every[2];
    float *y_rounded = n == 12 ? const_cast<float *>(in_ptr(a[11], fine)) : nullptr;
    const bool sampled = n == 12 && a[9] != Py_None;
    if (!fine || (n == 12 && !pre) || (sampled && (!r || a[10] == Py_None || !ints(a[9], dims, 2) || !ints(a[10], every, 2)))) return slow_path();
    at::Tensor ym, wm;
    if (!y) {
        ym = new_tensor(p->y, at::kFloat, xt->device(), a[8], st, true);
        y = static_cast<float *>(ym.data_ptr());
    }
    if (!ws && p->workspace && (!pre || p->packed_needs_ws || packed_bytes < p->packed)) {
        wm = new_tensor({(int64_t)p->workspace}, at::kByte, xt->device(), a[8], st, false);
        ws = wm.data_ptr();
        ws_bytes = p->workspace;
    }
    const onnxb_status s = sampled   ? abi.conv_run_packed_sampled(p->desc, x, w, packed, packed_bytes, b, r, dims, every, y, y_rounded, ws, ws_bytes, st)
                           : n == 12 ? abi.conv_run_packed_rounded(p->desc, x, w, packed, packed_bytes, b, r, y, y_rounded, ws, ws_bytes, st)
                           : pre ? abi.conv_run_packed(p->desc, x, w, packed, packed_bytes, b, r, y, ws, ws_bytes, st)
                           : r ? abi.conv_add_run(p->desc, x, w, b, r, y, ws, ws_bytes, st)
                               : abi.conv_run(p->desc, x, w, b, y, ws, ws_bytes, st);
    return s == ONNXB_OK ? result(a[6], ym) : slow_path();
}

// gemm(A, B, C, alpha, beta, transA, transB, relu, Y, workspace, stream)
PyObject *py_gemm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 11) return slow_path();
    bool fine = true;
    const at::Tensor *at_ = nullptr, *bt = nullptr, *ct = nullptr;
    const float *A = in_ptr(a[0], fine, &at_), *B = in_ptr(a[1], fine, &bt), *C = in_ptr(a[2], fine, &ct);
    const double alpha = PyFloat_AsDouble(a[3]), beta = PyFloat_AsDouble(a[4]);
    const int ta = PyObject_IsTrue(a[5]), tb = PyObject_IsTrue(a[6]), relu = PyObject_IsTrue(a[7]);
    if (PyErr_Occurred()) { PyErr_Clear(); return slow_path(); }
    float *y = const_cast<float *>(in_ptr(a[8], fine));
    size_t ws_bytes;
    void *ws = ws_ptr(a[9], ws_bytes, fine), *st = stream_ptr(a[10], fine);
    if (!fine || !A || !B || at_->dim() != 2 || bt->dim() != 2) return slow_path();
    const int64_t M = at_->size(ta ? 1 : 0), K = at_->size(ta ? 0 : 1), N = bt->size(tb ? 0 : 1);
    if (bt->size(tb ? 1 : 0) != K || (ct && ct->dim() > 2)) return slow_path();
    int64_t c_dims[2] = {1, 1};
    const int c_rank = ct ? (int)ct->dim() : 0;
    for (int i = 0; i < c_rank; ++i) c_dims[i] = ct->size(i);
    at::Tensor ym, wm;
    if (!y) {
        ym = new_tensor({M, N}, at::kFloat, at_->device(), a[10], st, true);
        y = static_cast<float *>(ym.data_ptr());
    }
    if (!ws) {
        const size_t need = abi.gemm_workspace_bytes(ta, tb, M, N, K);
        if (need) {
            wm = new_tensor({(int64_t)need}, at::kByte, at_->device(), a[10], st, false);
            ws = wm.data_ptr();
            ws_bytes = need;
        }
    }
    const onnxb_status s = abi.gemm_run(ta, tb, (float)alpha, (float)beta, M, N, K, A, B, C, c_rank, C ? c_dims : nullptr,
                                        relu, y, ws, ws_bytes, st);
    return s == ONNXB_OK ? result(a[8], ym) : slow_path();
}

// maxpool(X, kernel_shape, pads, strides, Y, stream)
PyObject *py_maxpool(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 6) return slow_path();
    bool fine = true;
    const at::Tensor *xt = nullptr;
    const float *x = in_ptr(a[0], fine, &xt);
    int64_t ks[2], pads[4] = {0, 0, 0, 0}, st[2] = {0, 0}, yd[4];
    if (a[1] == Py_None || !ints(a[1], ks, 2) || !ints(a[2], pads, 4) || !ints(a[3], st, 2)) return slow_path();
    float *y = const_cast<float *>(in_ptr(a[4], fine));
    void *stream = stream_ptr(a[5], fine);
    if (!fine || !x || xt->dim() != 4) return slow_path();
    const int64_t *xd = xt->sizes().data();
    if (abi.maxpool2d_shape(xd, ks, pads, st, yd) != ONNXB_OK) return slow_path();
    at::Tensor ym;
    if (!y) {
        ym = new_tensor(yd, at::kFloat, xt->device(), a[5], stream, true);
        y = static_cast<float *>(ym.data_ptr());
    }
    return abi.maxpool2d_run(xd, ks, pads, st, x, y, stream) == ONNXB_OK ? result(a[4], ym) : slow_path();
}

// gap(X, Y, stream)
PyObject *py_gap(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 3) return slow_path();
    bool fine = true;
    const at::Tensor *xt = nullptr;
    const float *x = in_ptr(a[0], fine, &xt);
    float *y = const_cast<float *>(in_ptr(a[1], fine));
    void *stream = stream_ptr(a[2], fine);
    if (!fine || !x || xt->dim() != 4) return slow_path();
    at::Tensor ym;
    if (!y) {
        ym = new_tensor({xt->size(0), xt->size(1), 1, 1}, at::kFloat, xt->device(), a[2], stream, true);
        y = static_cast<float *>(ym.data_ptr());
    }
    return abi.global_average_pool_run(xt->sizes().data(), x, y, stream) == ONNXB_OK ? result(a[1], ym) : slow_path();
}

// --------------------------------------------------------------------- dense layers of 8- and 16-bit operands
// One call's tensors: CUDA tensors of the current device, two-dimensional with the elements of a row one right after the other (`matrix`),
// or contiguous fp32 of a given length (`vector`).  Anything else clears `fine`.
struct Views {
    bool fine = true;
    c10::DeviceIndex device = -1;
    PyObject *given_stream;
    void *stream = nullptr;

    explicit Views(PyObject *given) : given_stream(given) {}

    const at::Tensor *on_device(PyObject *o) {
        if (!THPVariable_CheckExact(o)) { fine = false; return nullptr; }
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda()) { fine = false; return nullptr; }
        if (device < 0) {
            device = t.device().index();
            if (device != c10::cuda::current_device()) fine = false;
            stream = stream_ptr(given_stream, fine);
            if (fine && given_stream != Py_None) {              // (a stream of another device: the checked path says so)
                PyObject *a = PyObject_GetAttrString(given_stream, "device_index");
                if (!a) PyErr_Clear();
                else {
                    fine = PyLong_AsLong(a) == device;
                    Py_DECREF(a);
                    if (PyErr_Occurred()) { PyErr_Clear(); fine = false; }
                }
            }
        }
        if (t.device().index() != device) fine = false;
        return &t;
    }
    void take(const at::Tensor &t, onnxb_matrix &m) {
        const at::ScalarType type = t.scalar_type();
        m.type = type == at::kFloat ? ONNXB_FLOAT : type == at::kChar ? ONNXB_INT8 : type == at::kHalf ? ONNXB_FLOAT16 : type == at::kBFloat16 ? ONNXB_BFLOAT16 : 0;
        if (!m.type || t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) { fine = false; return; }
        m.data = t.data_ptr();
        m.rows = t.size(0);
        m.cols = t.size(1);
        m.ld = m.rows > 1 ? t.stride(0) : m.cols;
        m.reserved = 0;
    }
    // the view, or nullptr for None
    onnxb_matrix *matrix(PyObject *o, onnxb_matrix &m) {
        if (o == Py_None) return nullptr;
        const at::Tensor *t = on_device(o);
        if (t) take(*t, m);
        return &m;
    }
    float *vector(PyObject *o, int64_t size) {
        if (o == Py_None) return nullptr;
        const at::Tensor *t = on_device(o);
        if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->numel() != size) { fine = false; return nullptr; }
        return static_cast<float *>(t->data_ptr());
    }
    at::Tensor made(at::IntArrayRef size, at::ScalarType type, bool is_result = true) {
        return new_tensor(size, type, at::Device(at::kCUDA, device), given_stream, stream, is_result);
    }
    // Whether the results and the workspace that the caller gives can be taken; asked before anything is made for the call
    bool takes(std::initializer_list<PyObject *> results, PyObject *workspace) {
        onnxb_matrix m{};
        for (PyObject *o : results) matrix(o, m);
        if (workspace != Py_None) {
            const at::Tensor *t = on_device(workspace);
            if (t && !t->is_contiguous()) fine = false;
        }
        return fine;
    }
    // a result: the caller's, or one made here
    onnxb_matrix *result(PyObject *given, int64_t rows, int64_t cols, int32_t type, at::Tensor &t, onnxb_matrix &m) {
        if (given != Py_None) return matrix(given, m);
        t = made({rows, cols}, type == ONNXB_FLOAT ? at::kFloat : type == ONNXB_FLOAT16 ? at::kHalf : at::kBFloat16);
        m = onnxb_matrix{t.data_ptr(), rows, cols, cols, type, 0};
        return &m;
    }
    // the caller's workspace, or one of `need` bytes
    void *workspace(PyObject *given, size_t need, at::Tensor &t, size_t &bytes) {
        bytes = 0;
        if (given != Py_None) {
            const at::Tensor *g = on_device(given);
            if (!g) return nullptr;
            bytes = g->nbytes();
            return g->data_ptr();
        }
        if (!need) return nullptr;
        t = made({(int64_t)need}, at::kByte, false);
        bytes = need;
        return t.data_ptr();
    }
};

// The code of an activation's name; -1 for none
inline int activation_of(PyObject *o) {
    static const char *const names[] = {"silu", "gelu", "gelu_tanh", "relu"};
    if (PyUnicode_Check(o))
        for (int i = 0; i < 4; ++i)
            if (PyUnicode_CompareWithASCIIString(o, names[i]) == 0) return i;
    return -1;
}
// The code of a type of floats, by torch's object or by name; 0 for anything else
inline int32_t float_type_of(PyObject *o) {
    if (THPDtype_Check(o)) {
        const at::ScalarType t = reinterpret_cast<THPDtype *>(o)->scalar_type;
        return t == at::kFloat ? ONNXB_FLOAT : t == at::kHalf ? ONNXB_FLOAT16 : t == at::kBFloat16 ? ONNXB_BFLOAT16 : 0;
    }
    if (!PyUnicode_Check(o)) return 0;
    return PyUnicode_CompareWithASCIIString(o, "float32") == 0 ? ONNXB_FLOAT : PyUnicode_CompareWithASCIIString(o, "float16") == 0 ? ONNXB_FLOAT16
           : PyUnicode_CompareWithASCIIString(o, "bfloat16") == 0 ? ONNXB_BFLOAT16 : 0;
}

// quantize_rows(X, Q, scale, stream) -> (Q, scale)
PyObject *py_quantize_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 4) return slow_path();
    Views v(a[3]);
    onnxb_matrix x{}, q{};
    if (!v.matrix(a[0], x) || !v.fine || x.rows < 1) return slow_path();
    at::Tensor qt, st;
    float *scale = v.vector(a[2], x.rows);
    v.matrix(a[1], q);
    if (!v.fine) return slow_path();
    if (a[1] == Py_None) {
        const int64_t pitch = (x.cols + 15) / 16 * 16;
        qt = v.made({x.rows, pitch}, at::kChar);
        if (pitch != x.cols) qt = qt.narrow(1, 0, x.cols);
        v.take(qt, q);
    }
    if (!scale) {
        st = v.made({x.rows}, at::kFloat);
        scale = static_cast<float *>(st.data_ptr());
    }
    if (abi.quantize_rows_run(&x, &q, scale, v.stream) != ONNXB_OK) return slow_path();
    return Py_BuildValue("(NN)", result(a[1], qt), result(a[2], st));
}

// gemm_int8(A, a_scale, B, b_scale, C, relu, dtype, Y, workspace, stream)
PyObject *py_gemm_int8(PyObject *, PyObject *const *o, Py_ssize_t n) {
    if (n != 10) return slow_path();
    Views v(o[9]);
    onnxb_matrix a{}, b{}, y{};
    if (!v.matrix(o[0], a) || !v.matrix(o[2], b) || !v.fine) return slow_path();
    const float *sa = v.vector(o[1], a.rows), *sb = v.vector(o[3], b.rows), *c = v.vector(o[4], b.rows);
    const int relu = PyObject_IsTrue(o[5]);
    const int32_t type = o[7] == Py_None ? float_type_of(o[6]) : ONNXB_FLOAT;
    if (PyErr_Occurred()) { PyErr_Clear(); return slow_path(); }
    if (!type || !v.takes({o[7]}, o[8])) return slow_path();
    at::Tensor yt, wt;
    size_t ws_bytes;
    v.result(o[7], a.rows, b.rows, type, yt, y);
    void *ws = v.workspace(o[8], abi.gemm_int8_workspace_bytes(&a, &b), wt, ws_bytes);
    if (abi.gemm_int8_run(&a, sa, &b, sb, c, relu, &y, ws, ws_bytes, v.stream) != ONNXB_OK) return slow_path();
    return result(o[7], yt);
}

// gated(X, Wg, Wu, activation, save, H, G, U, workspace, stream) -> H, or (H, G, U)
PyObject *py_gated(PyObject *, PyObject *const *o, Py_ssize_t n) {
    if (n != 10) return slow_path();
    Views v(o[9]);
    onnxb_matrix x{}, wg{}, wu{}, h{}, g{}, u{};
    if (!v.matrix(o[0], x) || !v.matrix(o[1], wg) || !v.matrix(o[2], wu) || !v.fine) return slow_path();
    const int activation = activation_of(o[3]), asked = PyObject_IsTrue(o[4]);
    if (PyErr_Occurred()) { PyErr_Clear(); return slow_path(); }
    if (activation < 0 || (x.type != ONNXB_FLOAT16 && x.type != ONNXB_BFLOAT16) || !v.takes({o[5], o[6], o[7]}, o[8])) return slow_path();
    const bool save = asked || o[6] != Py_None || o[7] != Py_None;
    at::Tensor ht, gt, ut, wt;
    size_t ws_bytes;
    v.result(o[5], x.rows, wg.rows, x.type, ht, h);
    if (save) {
        v.result(o[6], x.rows, wg.rows, x.type, gt, g);
        v.result(o[7], x.rows, wg.rows, x.type, ut, u);
    }
    void *ws = v.workspace(o[8], abi.gated_workspace_bytes(&x, &wg, &wu), wt, ws_bytes);
    if (abi.gated_run(&x, &wg, &wu, activation, &h, save ? &g : nullptr, save ? &u : nullptr, ws, ws_bytes, v.stream) != ONNXB_OK)
        return slow_path();
    if (!save) return result(o[5], ht);
    return Py_BuildValue("(NNN)", result(o[5], ht), result(o[6], gt), result(o[7], ut));
}

// gated_int8(A, a_scale, Wg, g_scale, Wu, u_scale, activation, dtype, H, workspace, stream)
PyObject *py_gated_int8(PyObject *, PyObject *const *o, Py_ssize_t n) {
    if (n != 11) return slow_path();
    Views v(o[10]);
    onnxb_matrix a{}, wg{}, wu{}, h{};
    if (!v.matrix(o[0], a) || !v.matrix(o[2], wg) || !v.matrix(o[4], wu) || !v.fine) return slow_path();
    const float *sa = v.vector(o[1], a.rows), *sg = v.vector(o[3], wg.rows), *su = v.vector(o[5], wu.rows);
    const int activation = activation_of(o[6]);
    const int32_t type = o[8] == Py_None ? float_type_of(o[7]) : ONNXB_FLOAT;
    if (activation < 0 || !type || !v.takes({o[8]}, o[9])) return slow_path();
    at::Tensor ht, wt;
    size_t ws_bytes;
    v.result(o[8], a.rows, wg.rows, type, ht, h);
    void *ws = v.workspace(o[9], abi.gated_workspace_bytes(&a, &wg, &wu), wt, ws_bytes);
    if (abi.gated_int8_run(&a, sa, &wg, sg, &wu, su, activation, &h, ws, ws_bytes, v.stream) != ONNXB_OK) return slow_path();
    return result(o[8], ht);
}

// gated_backward(dH, X, Wg, Wu, G, U, activation, dX wanted, dWg wanted, dWu wanted, dX, dWg, dWu, workspace, stream) -> (dX, dWg, dWu)
PyObject *py_gated_backward(PyObject *, PyObject *const *o, Py_ssize_t n) {
    if (n != 15) return slow_path();
    Views v(o[14]);
    onnxb_matrix in[6] = {}, out[3] = {};
    onnxb_matrix *ins[6], *outs[3] = {nullptr, nullptr, nullptr};
    const int activation = activation_of(o[6]);
    bool want[3];
    for (int i = 0; i < 3; ++i) want[i] = o[10 + i] != Py_None || PyObject_IsTrue(o[7 + i]) == 1;
    if (PyErr_Occurred()) { PyErr_Clear(); return slow_path(); }
    for (int i = 0; i < 6; ++i) {
        const bool used = i == 1 ? want[1] || want[2] : i == 2 || i == 3 ? want[0] : true;
        ins[i] = used ? v.matrix(o[i], in[i]) : nullptr;
        if (used && !ins[i]) return slow_path();
    }
    if (!v.fine || activation < 0 || !(want[0] || want[1] || want[2]) || (in[0].type != ONNXB_FLOAT16 && in[0].type != ONNXB_BFLOAT16)) return slow_path();
    if (!v.takes({o[10], o[11], o[12]}, o[13])) return slow_path();
    const int64_t width = ins[1] ? in[1].cols : in[2].cols;
    at::Tensor ts[3], wt;
    for (int i = 0; i < 3; ++i)
        if (want[i]) outs[i] = v.result(o[10 + i], i == 0 ? in[0].rows : in[0].cols, width, in[0].type, ts[i], out[i]);
    size_t ws_bytes;
    void *ws = v.workspace(o[13], abi.gated_backward_workspace_bytes(ins[0], ins[1], ins[2], ins[3], outs[0], outs[1], outs[2]), wt, ws_bytes);
    if (abi.gated_backward_run(ins[0], ins[1], ins[2], ins[3], ins[4], ins[5], activation, outs[0], outs[1], outs[2], ws, ws_bytes,
                                          v.stream) != ONNXB_OK)
        return slow_path();
    PyObject *got[3];
    for (int i = 0; i < 3; ++i) {
        got[i] = want[i] ? result(o[10 + i], ts[i]) : Py_None;
        if (!want[i]) Py_INCREF(Py_None);
    }
    return Py_BuildValue("(NNN)", got[0], got[1], got[2]);
}

// Address, type, sizes and strides of a tensor, or of those in a tuple or a dict (whose entry "input" is left out); false for anything else
bool add_state(PyObject *o, std::vector<int64_t> &out) {
    if (THPVariable_CheckExact(o)) {
        const at::Tensor &x = THPVariable_Unpack(o);
        out.push_back((int64_t)reinterpret_cast<uintptr_t>(x.data_ptr()));
        out.push_back((int64_t)x.scalar_type() << 32 | x.dim());
        out.insert(out.end(), x.sizes().begin(), x.sizes().end());
        out.insert(out.end(), x.strides().begin(), x.strides().end());
        return true;
    }
    if (PyTuple_CheckExact(o)) {
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(o); ++i)
            if (!add_state(PyTuple_GET_ITEM(o, i), out)) return false;
        return true;
    }
    if (!PyDict_CheckExact(o)) return false;
    PyObject *key, *value;
    for (Py_ssize_t i = 0; PyDict_Next(o, &i, &key, &value);) {
        if (!PyUnicode_Check(key)) return false;
        if (PyUnicode_CompareWithASCIIString(key, "input") != 0 && !add_state(value, out)) return false;
    }
    return true;
}

// state(tensors, tuples, dicts...): that of all of them and the library's dispatch state, as bytes
PyObject *py_state(PyObject *, PyObject *const *a, Py_ssize_t n) {
    std::vector<int64_t> out;
    out.reserve(4096);
    out.push_back((int64_t)abi.dispatch_state());
    for (Py_ssize_t i = 0; i < n; ++i)
        if (!add_state(a[i], out)) return slow_path();
    return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(out.data()), (Py_ssize_t)(out.size() * sizeof(int64_t)));
}

// a C++ exception (out of memory, no device) also leads to the checked path, which raises its own
template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *self, PyObject *const *a, Py_ssize_t n) {
    try {
        return F(self, a, n);
    } catch (...) {
        return slow_path();
    }
}

PyMethodDef methods[] = {
    {"bind", py_bind, METH_O, nullptr},
    {"plan", py_plan, METH_VARARGS, nullptr},
    {"conv", reinterpret_cast<PyCFunction>(&guarded<py_conv>), METH_FASTCALL, nullptr},
    {"gemm", reinterpret_cast<PyCFunction>(&guarded<py_gemm>), METH_FASTCALL, nullptr},
    {"maxpool", reinterpret_cast<PyCFunction>(&guarded<py_maxpool>), METH_FASTCALL, nullptr},
    {"gap", reinterpret_cast<PyCFunction>(&guarded<py_gap>), METH_FASTCALL, nullptr},
    {"quantize_rows", reinterpret_cast<PyCFunction>(&guarded<py_quantize_rows>), METH_FASTCALL, nullptr},
    {"gemm_int8", reinterpret_cast<PyCFunction>(&guarded<py_gemm_int8>), METH_FASTCALL, nullptr},
    {"gated", reinterpret_cast<PyCFunction>(&guarded<py_gated>), METH_FASTCALL, nullptr},
    {"gated_int8", reinterpret_cast<PyCFunction>(&guarded<py_gated_int8>), METH_FASTCALL, nullptr},
    {"gated_backward", reinterpret_cast<PyCFunction>(&guarded<py_gated_backward>), METH_FASTCALL, nullptr},
    {"state", reinterpret_cast<PyCFunction>(&guarded<py_state>), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_onnxb_fast", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__onnxb_fast(void) { return PyModule_Create(&module); }
