// Host path of the Python package in native code: argument checks, allocation of outputs and
// workspace, the call into librmm.so and the autograd node, without a Python frame or a ctypes
// conversion per argument (a forward + backward through RMMLinear took 92 us of host time in Python,
// more than the kernels of a RoBERTa-base attention projection).
//
// Every function takes its arguments by position and returns
//   - its result,
//   - a negative int: the rmm_status_t of the library call, or
//   - NotImplemented: something about the arguments is unusual (wrong type, device, shape, layout);
//     the caller then goes through the checks in binding.py, which say what.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_cpp_function.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>

#include "../../include/rmm.h"

namespace {

using at::Tensor;
using torch::autograd::Node;
using torch::autograd::SavedVariable;
using torch::autograd::variable_list;
using namespace torch::autograd;  // (for the property and method tables of Python nodes)

int dtype_code(const Tensor &t) {
    return t.scalar_type() == at::kBFloat16 ? RMM_DTYPE_BF16 : t.scalar_type() == at::kFloat ? RMM_DTYPE_F32 : -1;
}

void *current_stream(const Tensor &t) {
    return c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(t.device().index()).stream();
}

// A dense GPU tensor of the given matrix shape (cols < 0: a vector of `rows`), dtype and device.
bool is_matrix(const Tensor &t, int64_t rows, int64_t cols, const Tensor &like) {
    return t.is_cuda() && t.scalar_type() == like.scalar_type() && t.device() == like.device() && t.is_contiguous() &&
           (cols < 0 ? t.dim() == 1 && t.size(0) == rows : t.dim() == 2 && t.size(0) == rows && t.size(1) == cols);
}

Tensor new_matrix(const Tensor &like, int64_t rows, int64_t cols) { return at::empty({rows, cols}, like.options().requires_grad(false)); }

Tensor scratch(const Tensor &like, size_t need) {
    return at::empty({(int64_t)(need > 16 ? need : 16)}, like.options().dtype(at::kByte).requires_grad(false));
}

const void *ptr(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }
void *mut(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

struct NoGil {
    PyThreadState *state;
    NoGil() : state(PyGILState_Check() ? PyEval_SaveThread() : nullptr) {}
    ~NoGil() {
        if (state != nullptr) PyEval_RestoreThread(state);
    }
};

// ---- the library calls on checked tensors; undefined tensors = absent / to be allocated

int run_forward(const Tensor &X, const Tensor &W, const Tensor &bias, int64_t k, int kind, rmm_rng_state_t st, Tensor &Y,
                Tensor &X_proj, Tensor ws, bool need_xproj) {
    const int64_t n = X.size(0), d_in = X.size(1), d_out = W.size(0);
    const rmm_layer_desc_t desc = {n, d_in, d_out, k, dtype_code(X), kind};
    if (!Y.defined()) Y = new_matrix(X, n, d_out);
    if (!X_proj.defined() && need_xproj) X_proj = new_matrix(X, k, d_in);
    if (!ws.defined() && need_xproj) {
        const size_t need = rmm_workspace_bytes(&desc, RMM_OP_FORWARD);
        if (need > 0) ws = scratch(X, need);
    }
    void *stream = current_stream(X);
    const size_t ws_bytes = ws.defined() ? ws.nbytes() : 0;
    NoGil free_;
    return rmm_forward(&desc, st, ptr(X), ptr(W), ptr(bias), mut(Y), mut(X_proj), mut(ws), ws_bytes, stream);
}

int run_backward(const Tensor &dY, const Tensor &W, const Tensor &X_proj, int kind, rmm_rng_state_t st, bool need_dX,
                 bool need_db, Tensor &dX, Tensor &dW, Tensor &db, Tensor ws, bool accumulate) {
    const int64_t n = dY.size(0), d_out = dY.size(1), k = X_proj.size(0), d_in = X_proj.size(1);
    const rmm_layer_desc_t desc = {n, d_in, d_out, k, dtype_code(dY), kind};
    if (need_dX && !dX.defined()) dX = new_matrix(dY, n, d_in);
    if (!dW.defined()) dW = new_matrix(dY, d_out, d_in);
    if (need_db && !db.defined()) db = at::empty({d_out}, dY.options().requires_grad(false));
    if (!ws.defined()) ws = scratch(dY, rmm_workspace_bytes(&desc, RMM_OP_BACKWARD));
    void *stream = current_stream(dY);
    const size_t ws_bytes = ws.nbytes();
    NoGil free_;
    return (accumulate ? rmm_backward_accumulate : rmm_backward)(&desc, st, ptr(dY), ptr(W), ptr(X_proj), mut(dX), mut(dW),
                                                                mut(db), mut(ws), ws_bytes, stream);
}

// ---- autograd

struct LinearBackward : public Node {
    SavedVariable W_, X_proj_;  // X itself is not kept
    int kind = 0;
    rmm_rng_state_t st{};
    std::vector<int64_t> x_sizes;
    bool has_bias = false;

    std::mutex &mutex_for_python() { return mutex_; }

    std::string name() const override { return "RMMLinearFunctionBackward"; }

    void release_variables() override {
        std::lock_guard<std::mutex> lock(mutex_);
        W_.reset_data();
        X_proj_.reset_data();
    }

    variable_list apply(variable_list &&grads) override {
        std::lock_guard<std::mutex> lock(mutex_);
        variable_list out(has_bias ? 3 : 2);
        if (!grads[0].defined()) return out;
        const Tensor W = W_.unpack(), X_proj = X_proj_.unpack();
        at::NoGradGuard no_grad;
        const Tensor dY = grads[0].reshape({-1, W.size(0)}).contiguous();
        TORCH_CHECK(dY.scalar_type() == W.scalar_type() && dY.is_cuda(), "RMMLinear: the gradient must be a GPU tensor of dtype ",
                    W.scalar_type());
        Tensor dX, dW, db;
        if (task_should_compute_output(0)) dX = at::empty(x_sizes, dY.options());
        const int rc = run_backward(dY, W, X_proj, kind, st, dX.defined(),
                                    has_bias && task_should_compute_output(2), dX, dW, db, Tensor(), false);
        TORCH_CHECK(rc == RMM_OK, "rmm_backward: ", rmm_status_string(rc), " (status ", rc, ")");
        out[0] = dX;
        out[1] = dW;
        if (has_bias) out[2] = db;
        return out;
    }
};

PyObject *saved_tensors(PyObject *self, void *) {
    HANDLE_TH_ERRORS
    auto *node = static_cast<LinearBackward *>(reinterpret_cast<torch::autograd::THPCppFunction *>(self)->cdata.get());
    Tensor W, X_proj;
    {
        std::lock_guard<std::mutex> lock(node->mutex_for_python());
        W = node->W_.unpack(), X_proj = node->X_proj_.unpack();
    }
    PyObject *out = PyTuple_New(2);
    if (out == nullptr) return nullptr;
    PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(W));
    PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(X_proj));
    return out;
    END_HANDLE_TH_ERRORS
}

// ---- Python arguments

struct Unusual {};  // -> NotImplemented

Tensor arg_tensor(PyObject *o, bool optional = false) {
    if (o == Py_None && optional) return Tensor();
    if (!THPVariable_Check(o)) throw Unusual();
    return THPVariable_Unpack(o);
}
int64_t arg_int(PyObject *o) {
    if (!PyLong_CheckExact(o)) throw Unusual();
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred() != nullptr) {
        PyErr_Clear();
        throw Unusual();
    }
    return v;
}
uint64_t arg_u64(PyObject *o) {  // modulo 2^64, as ctypes does it
    if (!PyLong_CheckExact(o)) throw Unusual();
    return PyLong_AsUnsignedLongLongMask(o);
}
int arg_kind(PyObject *o) {
    const int64_t v = arg_int(o);
    if (v < INT32_MIN || v > INT32_MAX) throw Unusual();
    return (int)v;
}
bool arg_bool(PyObject *o) {
    if (o == Py_True) return true;
    if (o == Py_False || o == Py_None) return false;
    throw Unusual();
}
void need(bool ok) {
    if (!ok) throw Unusual();
}
void need_scratch(const Tensor &ws, const Tensor &like) { need(!ws.defined() || (ws.is_cuda() && ws.is_contiguous() && ws.device() == like.device())); }
PyObject *wrap(const Tensor &t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject *unusual() {
    Py_INCREF(Py_NotImplemented);
    return Py_NotImplemented;
}

#define RMM_BEGIN(COUNT)                                                      \
    HANDLE_TH_ERRORS                                                          \
    if (nargs != COUNT) {                                                     \
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");       \
        return nullptr;                                                       \
    }                                                                         \
    try {
#define RMM_END                                                               \
    }                                                                         \
    catch (const Unusual &) {                                                 \
        return unusual();                                                     \
    }                                                                         \
    END_HANDLE_TH_ERRORS

// forward(X, W, bias, k, kind, seed, offset, Y, X_proj, ws, need_xproj) -> (Y, X_proj)
PyObject *py_forward(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(11)
    const Tensor X = arg_tensor(a[0]), W = arg_tensor(a[1]), bias = arg_tensor(a[2], true), ws = arg_tensor(a[9], true);
    Tensor Y = arg_tensor(a[7], true), X_proj = arg_tensor(a[8], true);
    const int64_t k = arg_int(a[3]);
    const int kind = arg_kind(a[4]);
    const rmm_rng_state_t st = {arg_u64(a[5]), arg_u64(a[6])};
    const bool need_xproj = arg_bool(a[10]);
    need(X.is_cuda() && X.dim() == 2 && X.is_contiguous() && dtype_code(X) >= 0 && k >= 1 && W.dim() == 2);
    const int64_t n = X.size(0), d_in = X.size(1), d_out = W.size(0);
    need(is_matrix(W, d_out, d_in, X) && (!bias.defined() || is_matrix(bias, d_out, -1, X)) &&
         (!Y.defined() || is_matrix(Y, n, d_out, X)) && (!X_proj.defined() || is_matrix(X_proj, k, d_in, X)));
    need_scratch(ws, X);
    const int rc = run_forward(X, W, bias, k, kind, st, Y, X_proj, ws, need_xproj);
    if (rc != RMM_OK) return PyLong_FromLong(rc);
    PyObject *out = PyTuple_New(2);
    if (out == nullptr) return nullptr;
    PyTuple_SET_ITEM(out, 0, wrap(Y));
    PyTuple_SET_ITEM(out, 1, wrap(X_proj));
    return out;
    RMM_END
}

// backward(dY, W, X_proj, kind, seed, offset, need_dX, need_dbias, dX, dW, dbias, ws, accumulate) -> (dX, dW, dbias)
PyObject *py_backward(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(13)
    const Tensor dY = arg_tensor(a[0]), W = arg_tensor(a[1]), X_proj = arg_tensor(a[2]), ws = arg_tensor(a[11], true);
    Tensor dX = arg_tensor(a[8], true), dW = arg_tensor(a[9], true), db = arg_tensor(a[10], true);
    const int kind = arg_kind(a[3]);
    const rmm_rng_state_t st = {arg_u64(a[4]), arg_u64(a[5])};
    const bool need_dX = arg_bool(a[6]), need_db = arg_bool(a[7]), accumulate = arg_bool(a[12]);
    need(dY.is_cuda() && dY.dim() == 2 && dY.is_contiguous() && dtype_code(dY) >= 0 && X_proj.dim() == 2);
    const int64_t n = dY.size(0), d_out = dY.size(1), k = X_proj.size(0), d_in = X_proj.size(1);
    need(is_matrix(W, d_out, d_in, dY) && is_matrix(X_proj, k, d_in, dY) && (!dX.defined() || is_matrix(dX, n, d_in, dY)) &&
         (!dW.defined() || is_matrix(dW, d_out, d_in, dY)) && (!db.defined() || is_matrix(db, d_out, -1, dY)));
    need(!accumulate || (dW.defined() && (db.defined() || !need_db)));
    need_scratch(ws, dY);
    const int rc = run_backward(dY, W, X_proj, kind, st, need_dX, need_db, dX, dW, db, ws, accumulate);
    if (rc != RMM_OK) return PyLong_FromLong(rc);
    PyObject *out = PyTuple_New(3);
    if (out == nullptr) return nullptr;
    PyTuple_SET_ITEM(out, 0, wrap(dX));
    PyTuple_SET_ITEM(out, 1, wrap(dW));
    PyTuple_SET_ITEM(out, 2, wrap(db));
    return out;
    RMM_END
}

// sketch(A, k, kind, seed, offset, out, ws) -> out
PyObject *py_sketch(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(7)
    const Tensor A = arg_tensor(a[0]);
    Tensor out = arg_tensor(a[5], true), ws = arg_tensor(a[6], true);
    const int64_t k = arg_int(a[1]);
    const int kind = arg_kind(a[2]);
    const rmm_rng_state_t st = {arg_u64(a[3]), arg_u64(a[4])};
    need(A.is_cuda() && A.dim() == 2 && A.is_contiguous() && dtype_code(A) >= 0 && k >= 1);
    const int64_t n = A.size(0), d = A.size(1);
    need(!out.defined() || is_matrix(out, k, d, A));
    need_scratch(ws, A);
    if (!out.defined()) out = new_matrix(A, k, d);
    if (!ws.defined()) {
        const rmm_layer_desc_t desc = {n, d, d, k, dtype_code(A), kind};
        ws = scratch(A, rmm_workspace_bytes(&desc, RMM_OP_SKETCH));
    }
    void *stream = current_stream(A);
    int rc;
    {
        NoGil free_;
        rc = rmm_sketch(n, d, k, dtype_code(A), kind, st, ptr(A), mut(out), mut(ws), ws.nbytes(), stream);
    }
    return rc != RMM_OK ? PyLong_FromLong(rc) : wrap(out);
    RMM_END
}

// variance_stats(X, dY, k, kind, out, ws) -> out
PyObject *py_variance_stats(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(6)
    const Tensor X = arg_tensor(a[0]), dY = arg_tensor(a[1]);
    Tensor out = arg_tensor(a[4], true), ws = arg_tensor(a[5], true);
    const int64_t k = arg_int(a[2]);
    const int kind = arg_kind(a[3]);
    need(X.is_cuda() && X.dim() == 2 && X.is_contiguous() && dtype_code(X) >= 0 && dY.dim() == 2 && k >= 1);
    const int64_t n = X.size(0), d_in = X.size(1), d_out = dY.size(1);
    need(is_matrix(dY, n, d_out, X));
    need(!out.defined() || (out.is_cuda() && out.device() == X.device() && out.scalar_type() == at::kDouble && out.is_contiguous() &&
                            out.dim() == 1 && out.size(0) == 8));
    need_scratch(ws, X);
    const rmm_layer_desc_t desc = {n, d_in, d_out, k, dtype_code(X), kind};
    if (!out.defined()) out = at::empty({8}, X.options().dtype(at::kDouble).requires_grad(false));
    if (!ws.defined()) ws = scratch(X, rmm_workspace_bytes(&desc, RMM_OP_VARIANCE));
    void *stream = current_stream(X);
    int rc;
    {
        NoGil free_;
        rc = rmm_variance_stats(&desc, ptr(X), ptr(dY), (double *)mut(out), mut(ws), ws.nbytes(), stream);
    }
    return rc != RMM_OK ? PyLong_FromLong(rc) : wrap(out);
    RMM_END
}

// The layer calls below make their output without torch operators and hang their own node on it, so whatever
// watches operators or Python autograd functions would see nothing of them: a trace would hold an allocation that
// nobody fills, a forward-mode derivative would be dropped without a word, and a transform's wrapper has no memory.
// Such calls take the Python function, which torch records or refuses as any other.
bool watched(const Tensor &t) {
    return t.defined() && (t._fw_grad(/*level=*/0).defined() || !t.has_storage());
}
bool all_watched() {
    return torch::jit::tracer::isTracing() || c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
}
void need_unwatched(const Tensor &X, const Tensor &W, const Tensor &bias) {
    need(!all_watched() && !watched(X) && !watched(W) && !watched(bias));
}

// watched(tensors or None ..) -> bool
PyObject *py_watched(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    bool yes = all_watched();
    for (Py_ssize_t i = 0; i < nargs && !yes; ++i) yes = THPVariable_Check(a[i]) && watched(THPVariable_Unpack(a[i]));
    return PyBool_FromLong(yes);
    END_HANDLE_TH_ERRORS
}

// X as a dense n x d_in matrix
Tensor rows_of(const Tensor &X, const Tensor &W) {
    need(X.is_cuda() && X.dim() >= 1 && dtype_code(X) >= 0 && X.numel() > 0 && W.dim() == 2 && X.size(-1) == W.size(1));
    return X.dim() == 2 && X.is_contiguous() ? X : X.reshape({-1, X.size(-1)}).contiguous();
}
// An uninitialised tensor of X's leading dimensions and `last` columns (only its address goes to the library).
Tensor like_rows(const Tensor &X, int64_t last) {
    c10::SmallVector<int64_t, 4> s(X.sizes().begin(), X.sizes().end());
    s.back() = last;
    return at::empty(s, X.options().requires_grad(false));
}

// linear(X, W, bias, k, kind, seed, offset) -> Y with the autograd history of RMMLinearFunction
PyObject *py_linear(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(7)
    const Tensor X = arg_tensor(a[0]), W = arg_tensor(a[1]), bias = arg_tensor(a[2], true);
    const int64_t k = arg_int(a[3]);
    const int kind = arg_kind(a[4]);
    const rmm_rng_state_t st = {arg_u64(a[5]), arg_u64(a[6])};
    need(k >= 1);
    need_unwatched(X, W, bias);
    Tensor Y, X_proj, Wc;
    {
        at::NoGradGuard no_grad;
        const Tensor X2 = rows_of(X, W);
        Wc = W.contiguous();
        need(is_matrix(Wc, W.size(0), W.size(1), X2) && (!bias.defined() || is_matrix(bias, W.size(0), -1, X2)));
        Y = like_rows(X, W.size(0));
        const int rc = run_forward(X2, Wc, bias, k, kind, st, Y, X_proj, Tensor(), true);
        if (rc != RMM_OK) return PyLong_FromLong(rc);
    }
    if (torch::autograd::compute_requires_grad(X, W, bias)) {
        std::shared_ptr<LinearBackward> node(new LinearBackward(), torch::autograd::deleteNode);
        node->set_next_edges(bias.defined() ? torch::autograd::collect_next_edges(X, W, bias)
                                            : torch::autograd::collect_next_edges(X, W));
        node->W_ = SavedVariable(Wc, false);
        node->X_proj_ = SavedVariable(X_proj, false);
        node->kind = kind, node->st = st, node->has_bias = bias.defined();
        node->x_sizes.assign(X.sizes().begin(), X.sizes().end());
        torch::autograd::set_history(Y, node);
    }
    return wrap(Y);
    RMM_END
}

// infer(X, W, bias, kind) -> Y; nothing is kept, no sketch is made
PyObject *py_infer(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(4)
    const Tensor X = arg_tensor(a[0]), W = arg_tensor(a[1]), bias = arg_tensor(a[2], true);
    const int kind = arg_kind(a[3]);
    need_unwatched(X, W, bias);
    at::NoGradGuard no_grad;
    const Tensor X2 = rows_of(X, W), Wc = W.contiguous();
    need(is_matrix(Wc, W.size(0), W.size(1), X2) && (!bias.defined() || is_matrix(bias, W.size(0), -1, X2)));
    Tensor Y = like_rows(X, W.size(0)), X_proj;
    const int rc = run_forward(X2, Wc, bias, 1, kind, rmm_rng_state_t{0, 0}, Y, X_proj, Tensor(), false);
    if (rc != RMM_OK) return PyLong_FromLong(rc);
    return wrap(Y);
    RMM_END
}

// ---- 8-bit operands, and the norm in front of them

int f8_code(at::ScalarType t) { return t == at::kFloat8_e4m3fn ? RMM_F8_E4M3 : t == at::kFloat8_e5m2 ? RMM_F8_E5M2 : -1; }
int scale_code(at::ScalarType t) { return t == at::kFloat ? RMM_SCALE_F32 : t == at::kFloat8_e8m0fnu ? RMM_SCALE_E8M0 : -1; }
at::ScalarType arg_dtype(PyObject *o) {
    if (!THPDtype_Check(o)) throw Unusual();
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}
int64_t blocks8(int64_t d) { return (d + 127) / 128; }
int64_t pitch16(int64_t d) { return (d + 15) / 16 * 16; }

// New memory beside `like`, straight from the allocator: a call of these has up to five outputs, and the way through the dispatcher
// is half a microsecond for each (a norm of one token 7.1 -> 6.0 us of host time, the launch among them).
Tensor fresh(const Tensor &like, at::IntArrayRef sizes, at::ScalarType dtype) {
    return Tensor(at::detail::empty_cuda(sizes, dtype, like.device(), c10::nullopt));
}
// rows x cols of a new buffer with rows of `pitch`.
Tensor new_pitched(const Tensor &like, int64_t rows, int64_t cols, int64_t pitch, at::ScalarType dtype) {
    Tensor t = fresh(like, {rows, pitch}, dtype);
    if (pitch != cols) t.unsafeGetTensorImpl()->set_sizes_and_strides(at::IntArrayRef{rows, cols}, at::IntArrayRef{pitch, 1});
    return t;
}
// An 8-bit matrix: its two tensors and the descriptor.
struct Pair8 {
    Tensor data, scales;
    rmm_mat8_t m;
};
Pair8 new_mat8(const Tensor &like, int64_t rows, int64_t cols, bool weights, at::ScalarType f8, at::ScalarType scale) {
    Pair8 p;
    const int64_t ld = pitch16(cols), lds = weights ? blocks8(cols) : pitch16(rows);
    p.data = new_pitched(like, rows, cols, ld, f8);
    p.scales = weights ? new_pitched(like, blocks8(rows), lds, lds, scale) : new_pitched(like, blocks8(cols), rows, lds, scale);
    p.m = {p.data.data_ptr(), ld, p.scales.data_ptr(), lds, f8_code(f8), scale_code(scale)};
    return p;
}
// The descriptor of given tensors (anything unusual about them is left to binding.py).
rmm_mat8_t old_mat8(const Tensor &data, const Tensor &scales, bool weights, const Tensor &like) {
    need(data.is_cuda() && scales.is_cuda() && data.device() == like.device() && scales.device() == like.device());
    need(data.dim() == 2 && scales.dim() == 2 && f8_code(data.scalar_type()) >= 0 && scale_code(scales.scalar_type()) >= 0);
    const int64_t rows = data.size(0), cols = data.size(1), high = weights ? blocks8(rows) : blocks8(cols), wide = weights ? blocks8(cols) : rows;
    need(scales.size(0) == high && scales.size(1) == wide);
    const int64_t ld = rows > 1 ? data.stride(0) : pitch16(std::max(data.stride(0), cols));
    const int64_t lds = high > 1 ? scales.stride(0) : weights ? std::max(scales.stride(0), wide) : pitch16(std::max(scales.stride(0), wide));
    need((cols == 1 || data.stride(1) == 1) && ld % 16 == 0 && ld >= cols);
    need((wide == 1 || scales.stride(1) == 1) && lds >= wide && (weights || lds % 16 == 0));
    return {data.data_ptr(), ld, scales.data_ptr(), lds, f8_code(data.scalar_type()), scale_code(scales.scalar_type())};
}
PyObject *tuple_of(std::initializer_list<Tensor> ts) {
    PyObject *out = PyTuple_New((Py_ssize_t)ts.size());
    if (out == nullptr) return nullptr;
    Py_ssize_t i = 0;
    for (const Tensor &t : ts) PyTuple_SET_ITEM(out, i++, wrap(t));
    return out;
}
bool is_input(const Tensor &t, int64_t dims) { return t.is_cuda() && t.dim() == dims && t.is_contiguous() && dtype_code(t) >= 0 && t.numel() > 0; }

// quantize8(A, f8, scale_dtype) -> (data, scales)
PyObject *py_quantize8(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(3)
    const Tensor A = arg_tensor(a[0]);
    const at::ScalarType f8 = arg_dtype(a[1]), scale = arg_dtype(a[2]);
    need(is_input(A, 2) && f8_code(f8) >= 0 && scale_code(scale) >= 0);
    const c10::DeviceGuard guard(A.device());
    const Pair8 out = new_mat8(A, A.size(0), A.size(1), false, f8, scale);
    void *stream = current_stream(A);
    int rc;
    {
        NoGil free_;
        rc = rmm_quantize8(A.size(0), A.size(1), dtype_code(A), ptr(A), &out.m, stream);
    }
    return rc != RMM_OK ? PyLong_FromLong(rc) : tuple_of({out.data, out.scales});
    RMM_END
}

// quantize8_weight(W, f8, scale_dtype, transposed) -> (data, scales[, data_t, scales_t])
PyObject *py_quantize8_weight(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(4)
    const Tensor W = arg_tensor(a[0]);
    const at::ScalarType f8 = arg_dtype(a[1]), scale = arg_dtype(a[2]);
    const bool transposed = arg_bool(a[3]);
    need(is_input(W, 2) && f8_code(f8) >= 0 && scale_code(scale) >= 0);
    const c10::DeviceGuard guard(W.device());
    const Pair8 out = new_mat8(W, W.size(0), W.size(1), true, f8, scale);
    Pair8 t;
    if (transposed) t = new_mat8(W, W.size(1), W.size(0), true, f8, scale);
    void *stream = current_stream(W);
    int rc;
    {
        NoGil free_;
        rc = rmm_quantize8_weight(W.size(0), W.size(1), dtype_code(W), ptr(W), &out.m, transposed ? &t.m : nullptr, stream);
    }
    if (rc != RMM_OK) return PyLong_FromLong(rc);
    return transposed ? tuple_of({out.data, out.scales, t.data, t.scales}) : tuple_of({out.data, out.scales});
    RMM_END
}

// linear8(X8, x_scales, W8, w_scales, bias, dtype, Y) -> Y
PyObject *py_linear8(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(7)
    const Tensor X = arg_tensor(a[0]), xs = arg_tensor(a[1]), W = arg_tensor(a[2]), ws = arg_tensor(a[3]), bias = arg_tensor(a[4], true);
    const at::ScalarType dtype = arg_dtype(a[5]);
    Tensor Y = arg_tensor(a[6], true);
    need((dtype == at::kBFloat16 || dtype == at::kFloat) && X.dim() == 2 && W.dim() == 2 && X.size(1) == W.size(1) && X.numel() > 0 && W.numel() > 0);
    const rmm_mat8_t x = old_mat8(X, xs, false, X), w = old_mat8(W, ws, true, X);
    need(w.f8 == RMM_F8_E4M3 && w.scale == x.scale);
    const int64_t n = X.size(0), d_in = X.size(1), d_out = W.size(0);
    const c10::DeviceGuard guard(X.device());
    if (!Y.defined()) Y = fresh(X, {n, d_out}, dtype);
    need(Y.scalar_type() == dtype && Y.device() == X.device() && is_matrix(Y, n, d_out, Y));
    need(!bias.defined() || is_matrix(bias, d_out, -1, Y));
    void *stream = current_stream(X);
    int rc;
    {
        NoGil free_;
        rc = rmm_linear8(n, d_in, d_out, dtype == at::kBFloat16 ? RMM_DTYPE_BF16 : RMM_DTYPE_F32, &x, &w, ptr(bias), mut(Y), stream);
    }
    return rc != RMM_OK ? PyLong_FromLong(rc) : wrap(Y);
    RMM_END
}

// rms_norm(X, weight, residual, eps, need_Y, f8, scale_dtype) -> (Y, H, rstd, Y8, scales)
PyObject *py_rms_norm(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(7)
    const Tensor X = arg_tensor(a[0]), weight = arg_tensor(a[1]), residual = arg_tensor(a[2], true);
    need(PyFloat_CheckExact(a[3]));
    const float eps = (float)PyFloat_AS_DOUBLE(a[3]);
    const bool need_Y = arg_bool(a[4]), eight = a[5] != Py_None;
    need(is_input(X, 2));
    const int64_t n = X.size(0), d = X.size(1);
    need(is_matrix(weight, d, -1, X) && (!residual.defined() || is_matrix(residual, n, d, X)));
    const c10::DeviceGuard guard(X.device());
    Pair8 y8;
    if (eight) {
        const at::ScalarType f8 = arg_dtype(a[5]), scale = arg_dtype(a[6]);
        need(f8_code(f8) >= 0 && scale_code(scale) >= 0);
        y8 = new_mat8(X, n, d, false, f8, scale);
    }
    const Tensor H = residual.defined() ? fresh(X, {n, d}, X.scalar_type()) : X, rstd = fresh(X, {n}, at::kFloat);
    const Tensor Y = need_Y ? fresh(X, {n, d}, X.scalar_type()) : Tensor();
    void *stream = current_stream(X);
    int rc;
    {
        NoGil free_;
        rc = rmm_rms_norm(n, d, dtype_code(X), eps, ptr(X), ptr(residual), ptr(weight), residual.defined() ? mut(H) : nullptr, mut(Y),
                                eight ? &y8.m : nullptr, (float *)mut(rstd), stream);
    }
    return rc != RMM_OK ? PyLong_FromLong(rc) : tuple_of({Y, H, rstd, y8.data, y8.scales});
    RMM_END
}

// rms_norm_backward(dY, H, weight, rstd, dH, need_dX, need_dweight) -> (dX, dweight)
PyObject *py_rms_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t nargs) {
    RMM_BEGIN(7)
    const Tensor dY = arg_tensor(a[0]), H = arg_tensor(a[1]), weight = arg_tensor(a[2]), rstd = arg_tensor(a[3]), dH = arg_tensor(a[4], true);
    const bool need_dX = arg_bool(a[5]), need_dw = arg_bool(a[6]);
    need(is_input(dY, 2));
    const int64_t n = dY.size(0), d = dY.size(1);
    need(is_matrix(H, n, d, dY) && is_matrix(weight, d, -1, dY) && (!dH.defined() || is_matrix(dH, n, d, dY)));
    need(rstd.is_cuda() && rstd.device() == dY.device() && rstd.scalar_type() == at::kFloat && rstd.is_contiguous() && rstd.dim() == 1 &&
         rstd.size(0) == n);
    const c10::DeviceGuard guard(dY.device());
    const Tensor dX = need_dX ? fresh(dY, {n, d}, dY.scalar_type()) : Tensor(), dw = need_dw ? fresh(dY, {d}, dY.scalar_type()) : Tensor();
    const Tensor ws = need_dw ? fresh(dY, {(int64_t)rmm_rms_norm_workspace_bytes(n, d, dtype_code(dY))}, at::kByte) : Tensor();
    void *stream = current_stream(dY);
    int rc;
    {
        NoGil free_;
        rc = rmm_rms_norm_backward(n, d, dtype_code(dY), ptr(dY), ptr(dH), ptr(H), ptr(weight), (const float *)ptr(rstd), mut(dX), mut(dw),
                                         mut(ws), need_dw ? ws.nbytes() : 0, stream);
    }
    return rc != RMM_OK ? PyLong_FromLong(rc) : tuple_of({dX, dw});
    RMM_END
}

#define RMM_METHOD(NAME) {#NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_##NAME)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {RMM_METHOD(forward), RMM_METHOD(backward), RMM_METHOD(sketch), RMM_METHOD(variance_stats),
                         RMM_METHOD(linear),  RMM_METHOD(infer),    RMM_METHOD(quantize8), RMM_METHOD(quantize8_weight),
                         RMM_METHOD(linear8), RMM_METHOD(rms_norm), RMM_METHOD(rms_norm_backward), RMM_METHOD(watched),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rmm_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

PyTypeObject node_type;
// (torch's own table of these, THP_FUNCTION_DEFAULT_METHODS, names a function that its headers do not declare)
PyMethodDef node_methods[] = {{"_register_hook_dict", THPCppFunction_register_hook_dict, METH_O, nullptr},
                              {"register_hook", THPCppFunction_register_hook, METH_O, nullptr},
                              {"register_prehook", THPCppFunction_register_prehook, METH_O, nullptr},
                              {"name", THPCppFunction_name, METH_NOARGS, nullptr},
                              {"_sequence_nr", THPCppFunction_sequence_nr, METH_NOARGS, nullptr},
                              {nullptr, nullptr, 0, nullptr}};
PyGetSetDef node_properties[] = {THP_FUNCTION_DEFAULT_PROPERTIES,
                                 {(char *)"saved_tensors", saved_tensors, nullptr, nullptr, nullptr},
                                 {nullptr, nullptr, nullptr, nullptr, nullptr}};

}  // namespace

PyMODINIT_FUNC PyInit__rmm_host(void) {
    PyObject *m = PyModule_Create(&module);
    if (m == nullptr) return nullptr;
    torch::autograd::_initFunctionPyTypeObject(node_type, "RMMLinearFunctionBackward", node_properties, node_methods);
    torch::autograd::registerCppFunction(typeid(LinearBackward), &node_type);
    return m;
}
