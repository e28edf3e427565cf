// The plain case of the binding's per-tensor calls as native code (module _mxq_host): arguments that are ordinary
// contiguous CUDA tensors, on the current stream.  One call checks them, allocates the outputs that were not
// given and calls the C ABI; through Python attribute calls and ctypes the same took 2 - 3 times the launch itself.
//
// Every function returns None -- having enqueued nothing -- for anything else: other types and devices, tensor
// subclasses, tensors without storage (vmap, grad and functionalization wrappers), active torch modes, a stream
// argument, a status other than MXQ_OK (a failed launch of slice_scale_multi, which may follow others, is raised at
// once).  The caller in binding.py then takes its general path, which handles the case or raises the error it
// always raised.
#include <Python.h>

#include <cmath>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include "../../include/mxq.h"

namespace {

// ---- the C ABI of the loaded library (addresses from the binding, see bind) -----------------------------

struct Api {
    decltype(&mxq_quantize) quantize;
    decltype(&mxq_slice_scale) slice_scale;
    decltype(&mxq_slice_scale_multi) slice_scale_multi;
    decltype(&mxq_dequantize) dequantize;
    decltype(&mxq_tiled_scales_bytes) tiled_scales_bytes;
    decltype(&mxq_quantize_tiled) quantize_tiled;
    decltype(&mxq_slice_scale_tiled) slice_scale_tiled;
    decltype(&mxq_fake_quant) fake_quant;
    decltype(&mxq_fake_quant_bwd) fake_quant_bwd;
    decltype(&mxq_codes_bytes) codes_bytes;
    decltype(&mxq_matmul) matmul;
    decltype(&mxq_quantize_matrix) quantize_matrix;
    decltype(&mxq_matrix_codes_bytes) matrix_codes_bytes;
    decltype(&mxq_matrix_scales_bytes) matrix_scales_bytes;
    decltype(&mxq_moe) moe;
    decltype(&mxq_moe_workspace_bytes) moe_workspace_bytes;
    decltype(&mxq_cache_write) cache_write;
    decltype(&mxq_cache_read) cache_read;
    decltype(&mxq_cache_attention) cache_attention;
    decltype(&mxq_cache_attention_workspace_bytes) cache_attention_workspace_bytes;
} api;

PyObject* formats = nullptr;          // the binding's name -> id dict
PyTypeObject* parameter = nullptr;    // torch.nn.Parameter
PyObject* mxq_error = nullptr;        // the binding's MxqError(status, what)

// ---- arguments ------------------------------------------------------------------------------------------

bool modes_active()
{
    return c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::torch_function_mode_enabled();
}

// An ordinary contiguous CUDA tensor with storage, or null.
const at::Tensor* plain(PyObject* o)
{
    if (!THPVariable_CheckExact(o) && Py_TYPE(o) != parameter) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.unsafeGetTensorImpl()->is_python_dispatch() || !t.has_storage() ||
        t.layout() != at::kStrided || !t.is_contiguous())
        return nullptr;
    return &t;
}

bool dtype_id(at::ScalarType t, int* id)
{
    if (t == at::kFloat) *id = MXQ_F32;
    else if (t == at::kBFloat16) *id = MXQ_BF16;
    else return false;
    return true;
}

bool dtype_id(const at::Tensor& t, int* id) { return dtype_id(t.scalar_type(), id); }

bool as_int(PyObject* o, int* v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long x = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || x != (int)x) return false;
    *v = (int)x;
    return true;
}

bool as_count(PyObject* o, int64_t* v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return !overflow && *v >= 0;
}

bool format_id(PyObject* o, int* v)
{
    if (!PyUnicode_CheckExact(o)) return false;
    PyObject* id = PyDict_GetItemWithError(formats, o);      // borrowed
    if (!id) {
        PyErr_Clear();
        return false;
    }
    return as_int(id, v);
}

mxq_stream current_stream() { return static_cast<mxq_stream>(c10::cuda::getCurrentCUDAStream().stream()); }

// The interpreter's lock is released while a call allocates and enqueues: a launch waits when the queue is full, an
// allocation may wait for the device, and other Python threads (or a host callback that the queue itself waits for)
// have to run meanwhile.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked&) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// What `fn` returns, run without the lock.
template <class FN>
int unlocked(FN&& fn)
{
    Unlocked u;
    return fn();
}

// An output argument: the given tensor, or a new one when it is None.
struct Output {
    const at::Tensor* tensor = nullptr;
    at::Tensor made;

    bool take(PyObject* o) { return o == Py_None || (tensor = plain(o)); }
    void make(at::IntArrayRef sizes, at::ScalarType type, const at::Tensor& like)
    {
        if (!tensor) tensor = &(made = at::empty(sizes, at::TensorOptions().dtype(type).device(like.device())));
    }
    void make_like(const at::Tensor& like)
    {
        if (!tensor) tensor = &(made = at::empty_like(like));
    }
    void* data() const { return tensor->data_ptr(); }
    uint8_t* bytes() const { return static_cast<uint8_t*>(tensor->data_ptr()); }
    PyObject* result(PyObject* given) const
    {
        if (given == Py_None) return THPVariable_Wrap(made);
        Py_INCREF(given);
        return given;
    }
};

PyObject* pair(PyObject* a, PyObject* b)
{
    PyObject* t = a && b ? PyTuple_New(2) : nullptr;
    if (!t) {
        Py_XDECREF(a);
        Py_XDECREF(b);
        return nullptr;
    }
    PyTuple_SET_ITEM(t, 0, a);
    PyTuple_SET_ITEM(t, 1, b);
    return t;
}

uint8_t* bytes(const at::Tensor& t) { return static_cast<uint8_t*>(t.data_ptr()); }

// Sets MxqError(rc, what) as the Python error.
PyObject* raise_mxq_error(int rc, const char* what)
{
    if (PyObject* e = PyObject_CallFunction(mxq_error, "is", rc, what)) {
        PyErr_SetObject(mxq_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

#define GENERAL_UNLESS(cond) \
    if (!(cond)) Py_RETURN_NONE

// ---- the calls ------------------------------------------------------------------------------------------

// quantize(src, fmt, block, codes, scales, stream)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, dt;
    GENERAL_UNLESS(nargs == 6 && a[5] == Py_None && format_id(a[1], &fmt) && as_int(a[2], &block) && block > 0 && !modes_active());
    const at::Tensor* src = plain(a[0]);
    Output codes, scales;
    GENERAL_UNLESS(src && dtype_id(*src, &dt) && codes.take(a[3]) && scales.take(a[4]));
    const int rc = unlocked([&] {
        const int64_t n = src->numel();
        codes.make({(int64_t)api.codes_bytes((size_t)n, fmt)}, at::kByte, *src);
        scales.make({n / block}, at::kByte, *src);
        return api.quantize(src->data_ptr(), dt, (size_t)n, fmt, block, codes.data(), scales.bytes(), current_stream());
    });
    GENERAL_UNLESS(rc == MXQ_OK);
    return pair(codes.result(a[3]), scales.result(a[4]));
    END_HANDLE_TH_ERRORS
}

// slice_scale(codes, scales, n, src_fmt, dst_fmt, block, out_codes, out_scales, stream)
PyObject* slice_scale(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int src_fmt, dst_fmt, block;
    int64_t n;
    GENERAL_UNLESS(nargs == 9 && a[8] == Py_None && as_count(a[2], &n) && format_id(a[3], &src_fmt) && format_id(a[4], &dst_fmt) &&
                   as_int(a[5], &block) && block > 0 && !modes_active());
    const at::Tensor *codes = plain(a[0]), *scales = plain(a[1]);
    Output oc, os;
    GENERAL_UNLESS(codes && scales && oc.take(a[6]) && os.take(a[7]));
    const int rc = unlocked([&] {
        oc.make({(int64_t)api.codes_bytes((size_t)n, dst_fmt)}, at::kByte, *codes);
        os.make({n / block}, at::kByte, *codes);
        return api.slice_scale(codes->data_ptr(), bytes(*scales), (size_t)n, block, src_fmt, dst_fmt, oc.data(), os.bytes(),
                               current_stream());
    });
    GENERAL_UNLESS(rc == MXQ_OK);
    return pair(oc.result(a[6]), os.result(a[7]));
    END_HANDLE_TH_ERRORS
}

// slice_scale_multi(codes, scales, n, src_fmt, dst_fmts, block, outs, stream), outs None
PyObject* slice_scale_multi(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int src_fmt, block;
    int64_t n;
    GENERAL_UNLESS(nargs == 8 && a[6] == Py_None && a[7] == Py_None && as_count(a[2], &n) && format_id(a[3], &src_fmt) &&
                   as_int(a[5], &block) && block > 0 && !modes_active());
    GENERAL_UNLESS(PyList_CheckExact(a[4]) || PyTuple_CheckExact(a[4]));
    const Py_ssize_t k = PySequence_Fast_GET_SIZE(a[4]);
    GENERAL_UNLESS(k <= MXQ_MULTI_TARGETS_MAX);
    const at::Tensor *codes = plain(a[0]), *scales = plain(a[1]);
    GENERAL_UNLESS(codes && scales);
    int fmts[MXQ_MULTI_TARGETS_MAX];
    for (Py_ssize_t t = 0; t < k; ++t) GENERAL_UNLESS(format_id(PySequence_Fast_GET_ITEM(a[4], t), &fmts[t]));
    Output oc[MXQ_MULTI_TARGETS_MAX], os[MXQ_MULTI_TARGETS_MAX];
    const int rc = unlocked([&] {
        void* pc[MXQ_MULTI_TARGETS_MAX];
        uint8_t* ps[MXQ_MULTI_TARGETS_MAX];
        for (Py_ssize_t t = 0; t < k; ++t) {
            oc[t].make({(int64_t)api.codes_bytes((size_t)n, fmts[t])}, at::kByte, *codes);
            os[t].make({n / block}, at::kByte, *codes);
            pc[t] = oc[t].data();
            ps[t] = os[t].bytes();
        }
        return api.slice_scale_multi(codes->data_ptr(), bytes(*scales), (size_t)n, block, src_fmt, (int)k, fmts, pc, ps,
                                     current_stream());
    });
    // (other launches of the call may precede the one that failed: the general path would enqueue them again)
    if (rc == MXQ_ERR_CUDA) return raise_mxq_error(rc, "mxq_slice_scale_multi");
    GENERAL_UNLESS(rc == MXQ_OK);
    PyObject* list = PyList_New(k);
    if (!list) return nullptr;
    for (Py_ssize_t t = 0; t < k; ++t) {
        PyObject* p = pair(oc[t].result(Py_None), os[t].result(Py_None));
        if (!p) {
            Py_DECREF(list);
            return nullptr;
        }
        PyList_SET_ITEM(list, t, p);
    }
    return list;
    END_HANDLE_TH_ERRORS
}

// dequantize(codes, scales, n, fmt, block, dtype, dst, stream)
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, dt;
    int64_t n;
    GENERAL_UNLESS(nargs == 8 && a[7] == Py_None && as_count(a[2], &n) && format_id(a[3], &fmt) && as_int(a[4], &block) &&
                   !modes_active());
    const at::Tensor *codes = plain(a[0]), *scales = plain(a[1]);
    Output dst;
    GENERAL_UNLESS(codes && scales && dst.take(a[6]));
    at::ScalarType type = at::kFloat;
    if (dst.tensor) {
        GENERAL_UNLESS(dtype_id(*dst.tensor, &dt));
    } else {
        GENERAL_UNLESS(THPDtype_Check(a[5]));
        type = reinterpret_cast<THPDtype*>(a[5])->scalar_type;
        GENERAL_UNLESS(dtype_id(type, &dt));
    }
    const int rc = unlocked([&] {
        dst.make({n}, type, *codes);
        return api.dequantize(codes->data_ptr(), bytes(*scales), (size_t)n, fmt, block, dst.data(), dt, current_stream());
    });
    GENERAL_UNLESS(rc == MXQ_OK);
    return dst.result(a[6]);
    END_HANDLE_TH_ERRORS
}

// quantize_tiled(src, fmt, block, codes, tiled_scales, stream)
PyObject* quantize_tiled(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, dt;
    GENERAL_UNLESS(nargs == 6 && a[5] == Py_None && format_id(a[1], &fmt) && as_int(a[2], &block) && !modes_active());
    const at::Tensor* src = plain(a[0]);
    Output codes, scales;
    GENERAL_UNLESS(src && dtype_id(*src, &dt) && src->dim() == 2 && codes.take(a[3]) && scales.take(a[4]));
    const int rc = unlocked([&] {
        const int64_t rows = src->size(0), cols = src->size(1);
        codes.make({(int64_t)api.codes_bytes((size_t)(rows * cols), fmt)}, at::kByte, *src);
        scales.make({(int64_t)api.tiled_scales_bytes((size_t)rows, (size_t)(cols / 32))}, at::kByte, *src);
        return api.quantize_tiled(src->data_ptr(), dt, (size_t)rows, (size_t)cols, fmt, block, codes.data(), scales.bytes(),
                                  current_stream());
    });
    GENERAL_UNLESS(rc == MXQ_OK);
    return pair(codes.result(a[3]), scales.result(a[4]));
    END_HANDLE_TH_ERRORS
}

// slice_scale_tiled(codes, scales, rows, cols, src_fmt, dst_fmt, block, out_codes, out_tiled_scales, stream)
PyObject* slice_scale_tiled(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int src_fmt, dst_fmt, block;
    int64_t rows, cols;
    GENERAL_UNLESS(nargs == 10 && a[9] == Py_None && as_count(a[2], &rows) && as_count(a[3], &cols) && rows < (1ll << 31) &&
                   cols < (1ll << 31) && format_id(a[4], &src_fmt) && format_id(a[5], &dst_fmt) && as_int(a[6], &block) &&
                   !modes_active());
    const at::Tensor *codes = plain(a[0]), *scales = plain(a[1]);
    Output oc, os;
    GENERAL_UNLESS(codes && scales && oc.take(a[7]) && os.take(a[8]));
    const int rc = unlocked([&] {
        oc.make({(int64_t)api.codes_bytes((size_t)(rows * cols), dst_fmt)}, at::kByte, *codes);
        os.make({(int64_t)api.tiled_scales_bytes((size_t)rows, (size_t)(cols / 32))}, at::kByte, *codes);
        return api.slice_scale_tiled(codes->data_ptr(), bytes(*scales), (size_t)rows, (size_t)cols, block, src_fmt, dst_fmt, oc.data(),
                                     os.bytes(), current_stream());
    });
    GENERAL_UNLESS(rc == MXQ_OK);
    return pair(oc.result(a[7]), os.result(a[8]));
    END_HANDLE_TH_ERRORS
}

// fake_quant(src, fmt, block, mode, dst, stream)
PyObject* fake_quant(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, mode, dt;
    GENERAL_UNLESS(nargs == 6 && a[5] == Py_None && format_id(a[1], &fmt) && as_int(a[2], &block) && as_int(a[3], &mode) &&
                   !modes_active());
    const at::Tensor* src = plain(a[0]);
    Output dst;
    GENERAL_UNLESS(src && dtype_id(*src, &dt) && dst.take(a[4]));
    const int rc = unlocked([&] {
        dst.make_like(*src);
        return api.fake_quant(src->data_ptr(), dt, (size_t)src->numel(), fmt, block, mode, dst.data(), current_stream());
    });
    GENERAL_UNLESS(rc == MXQ_OK);
    return dst.result(a[4]);
    END_HANDLE_TH_ERRORS
}

// fake_quant_bwd(grad_out, grad_in, stream)
PyObject* fake_quant_bwd(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int dt;
    GENERAL_UNLESS(nargs == 3 && a[2] == Py_None && !modes_active());
    const at::Tensor* g = plain(a[0]);
    Output dst;
    GENERAL_UNLESS(g && dtype_id(*g, &dt) && dst.take(a[1]));
    const int rc = unlocked([&] {
        dst.make_like(*g);
        return api.fake_quant_bwd(g->data_ptr(), dt, (size_t)g->numel(), dst.data(), current_stream());
    });
    GENERAL_UNLESS(rc == MXQ_OK);
    return dst.result(a[1]);
    END_HANDLE_TH_ERRORS
}

// ---- calls with all arguments marshalled beforehand --------------------------------------------------------

// run_prepared(kind, arguments as a bytes object of int64s): the status.  (PreparedCall in binding.py; kinds in its
// _PREPARED.)
PyObject* run_prepared(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    if (nargs != 2 || !PyLong_CheckExact(a[0]) || !PyBytes_CheckExact(a[1]) || PyBytes_GET_SIZE(a[1]) < 9 * (Py_ssize_t)sizeof(int64_t)) {
        PyErr_SetString(PyExc_TypeError, "run_prepared(kind, arguments)");
        return nullptr;
    }
    int64_t v[9];
    memcpy(v, PyBytes_AS_STRING(a[1]), sizeof(v));
    auto ptr = [&](int i) { return reinterpret_cast<void*>(v[i]); };
    auto u8 = [&](int i) { return reinterpret_cast<uint8_t*>(v[i]); };
    auto num = [&](int i) { return (int)v[i]; };
    const long kind = PyLong_AsLong(a[0]);
    const int rc = unlocked([&] {
        const mxq_stream s = current_stream();
        switch (kind) {
        case 0: return api.quantize(ptr(0), num(1), (size_t)v[2], num(3), num(4), ptr(5), u8(6), s);
        case 1: return api.slice_scale(ptr(0), u8(1), (size_t)v[2], num(3), num(4), num(5), ptr(6), u8(7), s);
        case 2: return api.dequantize(ptr(0), u8(1), (size_t)v[2], num(3), num(4), ptr(5), num(6), s);
        case 3: return api.fake_quant(ptr(0), num(1), (size_t)v[2], num(3), num(4), num(5), ptr(6), s);
        case 4: return api.fake_quant_bwd(ptr(0), num(1), (size_t)v[2], ptr(3), s);
        default: return (int)MXQ_ERR_FORMAT;
        }
    });
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// ---- the straight-through estimator as an autograd node -----------------------------------------------------

struct NotPlain {};                    // the launch was refused: the general path raises the error

// MxqError(rc, what) out of a backward pass, which runs without the interpreter's lock and on a thread of its own.
[[noreturn]] void throw_mxq_error(int rc, const char* what)
{
    pybind11::gil_scoped_acquire lock;
    raise_mxq_error(rc, what);
    python_error raised;
    raised.persist();
    throw python_error(std::move(raised));
}

struct FakeQuantSTE : torch::autograd::Function<FakeQuantSTE> {
    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, int64_t fmt, int64_t block, int64_t mode,
                              bool copy_grad)
    {
        ctx->saved_data["copy_grad"] = copy_grad;
        int dt = 0;
        dtype_id(x, &dt);
        at::Tensor y = at::empty_like(x);
        if (api.fake_quant(x.data_ptr(), dt, (size_t)x.numel(), (int)fmt, (int)block, (int)mode, y.data_ptr(), current_stream()) != MXQ_OK)
            throw NotPlain{};
        return y;
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        at::Tensor g = grads[0];       // identity: the incoming gradient itself, or a copy of it
        if (ctx->saved_data["copy_grad"].toBool()) {
            const at::Tensor src = g.contiguous();
            int dt = 0;
            TORCH_CHECK_TYPE(dtype_id(src, &dt), "mxq tensors are float32 or bfloat16, got ", src.scalar_type());
            TORCH_CHECK_VALUE(src.is_cuda(), "grad_out must be a CUDA tensor (libmxq has no CPU path)");
            at::NoGradGuard no_grad;
            at::Tensor copy = at::empty_like(src);
            const int rc = api.fake_quant_bwd(src.data_ptr(), dt, (size_t)src.numel(), copy.data_ptr(), current_stream());
            if (rc != MXQ_OK) throw_mxq_error(rc, "mxq_fake_quant_bwd");
            g = copy;
        }
        return {g, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
    }
};

// fake_quant_ste(x, fmt, block, mode, copy_grad)
PyObject* fake_quant_ste(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, mode, dt;
    GENERAL_UNLESS(nargs == 5 && format_id(a[1], &fmt) && as_int(a[2], &block) && as_int(a[3], &mode) && PyBool_Check(a[4]) &&
                   !modes_active() && !torch::jit::tracer::isTracing());
    const at::Tensor* x = plain(a[0]);
    // (forward-mode AD and functorch transforms: the Python function says what it supports)
    const bool transforms = c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
    GENERAL_UNLESS(x && dtype_id(*x, &dt) && !x->_fw_grad(0).defined() && !transforms);
    at::Tensor y;
    try {
        Unlocked u;
        y = FakeQuantSTE::apply(*x, (int64_t)fmt, (int64_t)block, (int64_t)mode, a[4] == Py_True);
    } catch (const NotPlain&) {
        Py_RETURN_NONE;
    }
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// ---- products that read the codes -------------------------------------------------------------------------

// Is the tensor on `device`, and is that the current one?
bool here(const at::Tensor& t, c10::Device device) { return t.device() == device && device.index() == c10::cuda::current_device(); }

// Codes or scales: at least `n` bytes on the current device.
bool operand(const at::Tensor* t, int64_t n, c10::Device device) { return t && t->scalar_type() == at::kByte && t->numel() >= n && here(*t, device); }

// matmul(a_codes, a_scales, b_codes, b_scales, m, n, k, fmt, block, dtype, out, stream)
PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, dt;
    int64_t m, n, k;
    GENERAL_UNLESS(nargs == 12 && a[11] == Py_None && as_count(a[4], &m) && as_count(a[5], &n) && as_count(a[6], &k) && format_id(a[7], &fmt) &&
                   as_int(a[8], &block) && block > 0 && m < (1ll << 31) && n < (1ll << 31) && k < (1ll << 31) && !modes_active());
    const at::Tensor *ac = plain(a[0]), *as = plain(a[1]), *bc = plain(a[2]), *bs = plain(a[3]);
    Output out;
    GENERAL_UNLESS(ac && out.take(a[10]));
    const c10::Device dev = ac->device();
    GENERAL_UNLESS(operand(ac, m * k, dev) && operand(as, m * k / block, dev) && operand(bc, n * k, dev) && operand(bs, n * k / block, dev));
    at::ScalarType type = at::kFloat;
    if (out.tensor) {
        GENERAL_UNLESS(dtype_id(*out.tensor, &dt) && out.tensor->numel() == m * n && here(*out.tensor, dev));
    } else {
        GENERAL_UNLESS(THPDtype_Check(a[9]));
        type = reinterpret_cast<THPDtype*>(a[9])->scalar_type;
        GENERAL_UNLESS(dtype_id(type, &dt));
    }
    const int rc = unlocked([&] {
        out.make({m, n}, type, *ac);
        return api.matmul(ac->data_ptr(), bytes(*as), bc->data_ptr(), bytes(*bs), (size_t)m, (size_t)n, (size_t)k, fmt, block, out.data(), dt,
                          current_stream());
    });
    GENERAL_UNLESS(rc == MXQ_OK);
    return out.result(a[10]);
    END_HANDLE_TH_ERRORS
}

// The quantization of a matrix along its rows (codes, scales) and of its transpose (codes_t, scales_t); undefined where not wanted.
struct MatrixCodes {
    at::Tensor codes, scales, codes_t, scales_t;
    int make(const at::Tensor& x, int dt, int64_t rows, int64_t cols, int fmt, int block, bool by_rows, bool by_cols)
    {
        const auto u8 = at::TensorOptions().dtype(at::kByte).device(x.device());
        if (by_rows) {
            codes = at::empty({(int64_t)api.matrix_codes_bytes((size_t)rows, (size_t)cols, block)}, u8);
            scales = at::empty({(int64_t)api.matrix_scales_bytes((size_t)rows, (size_t)cols, block)}, u8);
        }
        if (by_cols) {
            codes_t = at::empty({(int64_t)api.matrix_codes_bytes((size_t)cols, (size_t)rows, block)}, u8);
            scales_t = at::empty({(int64_t)api.matrix_scales_bytes((size_t)cols, (size_t)rows, block)}, u8);
        }
        auto ptr = [](const at::Tensor& t) { return t.defined() ? static_cast<uint8_t*>(t.data_ptr()) : nullptr; };
        return api.quantize_matrix(x.data_ptr(), dt, (size_t)rows, (size_t)cols, fmt, block, ptr(codes), ptr(scales), ptr(codes_t), ptr(scales_t),
                                   current_stream());
    }
};

// quantize_matrix(src, fmt, block, rows, cols, stream)
PyObject* quantize_matrix(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, dt;
    GENERAL_UNLESS(nargs == 6 && a[5] == Py_None && format_id(a[1], &fmt) && as_int(a[2], &block) && block > 0 && PyBool_Check(a[3]) &&
                   PyBool_Check(a[4]) && !modes_active());
    const at::Tensor* src = plain(a[0]);
    GENERAL_UNLESS(src && dtype_id(*src, &dt) && src->dim() == 2 && here(*src, src->device()));
    MatrixCodes q;
    const int rc = unlocked([&] { return q.make(*src, dt, src->size(0), src->size(1), fmt, block, a[3] == Py_True, a[4] == Py_True); });
    GENERAL_UNLESS(rc == MXQ_OK);
    PyObject* t = PyTuple_New(4);
    if (!t) return nullptr;
    const at::Tensor* got[4] = {&q.codes, &q.scales, &q.codes_t, &q.scales_t};
    for (int i = 0; i < 4; ++i) {
        PyObject* o = got[i]->defined() ? THPVariable_Wrap(*got[i]) : Py_NewRef(Py_None);
        if (!o) {
            Py_DECREF(t);
            return nullptr;
        }
        PyTuple_SET_ITEM(t, i, o);
    }
    return t;
    END_HANDLE_TH_ERRORS
}

// moe(x, logits, up_codes, up_scales, down_codes, down_scales, inner, top_k, fmt, block, renormalize, out, workspace, stream)
PyObject* moe(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, dt, top_k;
    int64_t inner;
    GENERAL_UNLESS(nargs == 14 && a[13] == Py_None && as_count(a[6], &inner) && inner > 0 && inner < (1ll << 31) && as_int(a[7], &top_k) && top_k > 0 &&
                   format_id(a[8], &fmt) && as_int(a[9], &block) && block > 0 && PyBool_Check(a[10]) && !modes_active());
    const at::Tensor *x = plain(a[0]), *logits = plain(a[1]), *uc = plain(a[2]), *us = plain(a[3]), *dc = plain(a[4]), *ds = plain(a[5]);
    Output out, ws;
    GENERAL_UNLESS(x && logits && dtype_id(*x, &dt) && x->dim() == 2 && logits->dim() == 2 && logits->scalar_type() == at::kFloat &&
                   logits->size(0) == x->size(0) && out.take(a[11]) && ws.take(a[12]));
    const c10::Device dev = x->device();
    const int64_t tokens = x->size(0), hidden = x->size(1), experts = logits->size(1);
    GENERAL_UNLESS(hidden > 0 && hidden < (1ll << 31) && experts > 0 && experts < (1 << 16) && inner * hidden < (1ll << 42));
    const int64_t weights = experts * hidden * inner;
    GENERAL_UNLESS(here(*x, dev) && here(*logits, dev) && operand(uc, (int64_t)api.codes_bytes((size_t)(2 * weights), fmt), dev) &&
                   operand(us, 2 * weights / block, dev) && operand(dc, (int64_t)api.codes_bytes((size_t)weights, fmt), dev) &&
                   operand(ds, weights / block, dev));
    GENERAL_UNLESS(!out.tensor || (out.tensor->sizes() == x->sizes() && out.tensor->scalar_type() == x->scalar_type() && here(*out.tensor, dev)));
    GENERAL_UNLESS(!ws.tensor || operand(ws.tensor, 0, dev));
    const int rc = unlocked([&] {
        out.make_like(*x);
        ws.make({(int64_t)api.moe_workspace_bytes((size_t)tokens, top_k, (size_t)inner, dt)}, at::kByte, *x);
        const mxq_moe_layer layer{uc->data_ptr(), bytes(*us), dc->data_ptr(), bytes(*ds), (size_t)hidden, (size_t)inner, (int)experts, fmt, block};
        return api.moe(&layer, x->data_ptr(), dt, static_cast<const float*>(logits->data_ptr()), (size_t)tokens, top_k, a[10] == Py_True, out.data(),
                       ws.data(), (size_t)ws.tensor->numel(), current_stream());
    });
    // (the first of the call's two launches may precede the one that failed)
    if (rc == MXQ_ERR_CUDA) return raise_mxq_error(rc, "mxq_moe");
    GENERAL_UNLESS(rc == MXQ_OK);
    return out.result(a[11]);
    END_HANDLE_TH_ERRORS
}

// A contiguous tensor at an address that the kernels take, a multiple of 32: itself, or a copy where it is a view that begins elsewhere (a
// slice, a parameter in a flat buffer, the gradient of an output that went through cat).
at::Tensor placed(const at::Tensor& t)
{
    return reinterpret_cast<uintptr_t>(t.data_ptr()) % 32 ? t.clone(at::MemoryFormat::Contiguous) : t;
}

// y = Q(x) Q(w)^T with dx = Q(dy) Q(w^T)^T and dw = Q(dy^T) Q(x^T)^T: what _LinearSTE of binding.py does, for x [..., k] and w [n, k].
struct LinearSTE : torch::autograd::Function<LinearSTE> {
    static int64_t up(int64_t v, int64_t block) { return (v + block - 1) / block * block; }
    static int product(const at::Tensor& a, const at::Tensor& as, const at::Tensor& b, const at::Tensor& bs, int64_t m, int64_t n, int64_t k, int64_t block,
                       const at::Tensor& out)
    {
        int dt = 0;
        dtype_id(out, &dt);
        return api.matmul(a.data_ptr(), bytes(as), b.data_ptr(), bytes(bs), (size_t)m, (size_t)n, (size_t)k, MXQ_FP8_E4M3, (int)block, out.data_ptr(), dt,
                          current_stream());
    }

    static at::Tensor forward(torch::autograd::AutogradContext* ctx, const at::Tensor& x, const at::Tensor& w, int64_t block, bool need_x, bool need_w)
    {
        const int64_t k = w.size(1), n = w.size(0), m = x.numel() / k;
        int xt = 0, wt = 0;
        dtype_id(x, &xt);
        dtype_id(w, &wt);
        MatrixCodes qx, qw;
        if (qx.make(placed(x), xt, m, k, MXQ_FP8_E4M3, (int)block, true, need_w) != MXQ_OK) throw NotPlain{};
        if (qw.make(placed(w), wt, n, k, MXQ_FP8_E4M3, (int)block, true, need_x) != MXQ_OK) throw NotPlain{};
        std::vector<int64_t> sizes = x.sizes().vec();
        sizes.back() = n;
        at::Tensor y = at::empty(sizes, x.options());
        if (product(qx.codes, qx.scales, qw.codes, qw.scales, m, n, up(k, block), block, y) != MXQ_OK) throw NotPlain{};
        ctx->save_for_backward({qx.codes_t, qx.scales_t, qw.codes_t, qw.scales_t});
        ctx->saved_data["block"] = block;
        ctx->saved_data["sizes"] = x.sizes().vec();
        ctx->saved_data["n"] = n;
        ctx->saved_data["x_type"] = x.scalar_type();
        ctx->saved_data["w_type"] = w.scalar_type();
        return y;
    }

    static torch::autograd::variable_list backward(torch::autograd::AutogradContext* ctx, torch::autograd::variable_list grads)
    {
        const auto saved = ctx->get_saved_variables();
        const std::vector<int64_t> sizes = ctx->saved_data["sizes"].toIntVector();
        const int64_t block = ctx->saved_data["block"].toInt(), n = ctx->saved_data["n"].toInt(), k = sizes.back();
        int64_t m = 1;
        for (size_t i = 0; i + 1 < sizes.size(); ++i) m *= sizes[i];
        const bool need_x = saved[2].defined() && ctx->needs_input_grad(0), need_w = saved[0].defined() && ctx->needs_input_grad(1);
        torch::autograd::variable_list out(5);
        if (!grads[0].defined() || !(need_x || need_w)) return out;
        {
            at::NoGradGuard no_grad;
            int dt = 0;
            TORCH_CHECK_TYPE(dtype_id(grads[0], &dt), "mxq tensors are float32 or bfloat16, got ", grads[0].scalar_type());
            TORCH_CHECK_VALUE(grads[0].is_cuda(), "the gradient must be a CUDA tensor (libmxq has no CPU path)");
            const at::Tensor dy = placed(grads[0].contiguous());
            MatrixCodes q;
            int rc = q.make(dy, dt, m, n, MXQ_FP8_E4M3, (int)block, need_x, need_w);
            if (rc != MXQ_OK) throw_mxq_error(rc, "mxq_quantize_matrix");
            if (need_x) {
                out[0] = at::empty(sizes, dy.options().dtype(ctx->saved_data["x_type"].toScalarType()));
                rc = product(q.codes, q.scales, saved[2], saved[3], m, k, up(n, block), block, out[0]);
                if (rc != MXQ_OK) throw_mxq_error(rc, "mxq_matmul");
            }
            if (need_w) {
                out[1] = at::empty({n, k}, dy.options().dtype(ctx->saved_data["w_type"].toScalarType()));
                rc = product(q.codes_t, q.scales_t, saved[0], saved[1], n, k, up(m, block), block, out[1]);
                if (rc != MXQ_OK) throw_mxq_error(rc, "mxq_matmul");
            }
        }
        // The quantizers have no second derivative, and dx depends on w, dw on x, even for a constant dy: what a pass with a graph
        // of its own (create_graph) returns says so where it is differentiated.
        if (at::GradMode::is_enabled()) {
            for (const at::Tensor& t : out)
                if (t.defined()) t.set_requires_grad(true);
            const auto refuse = std::make_shared<torch::autograd::DelayedError>("linear_ste can be differentiated once only", 5);
            return (*refuse)(std::move(out));
        }
        return out;
    }
};

// linear_ste(x, w, block)
PyObject* linear_ste(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int block, dt;
    GENERAL_UNLESS(nargs == 3 && as_int(a[2], &block) && (block == 32 || block == 64 || block == 128) && !modes_active() &&
                   !torch::jit::tracer::isTracing());
    const at::Tensor *x = plain(a[0]), *w = plain(a[1]);
    const bool transforms = c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
    GENERAL_UNLESS(x && w && dtype_id(*x, &dt) && dtype_id(*w, &dt) && x->dim() >= 1 && w->dim() == 2 && x->size(-1) == w->size(1) && x->numel() > 0 &&
                   w->numel() > 0 && here(*x, x->device()) && here(*w, x->device()) && !x->_fw_grad(0).defined() && !w->_fw_grad(0).defined() &&
                   !transforms);
    const bool grad = at::GradMode::is_enabled();
    at::Tensor y;
    try {
        Unlocked u;
        y = LinearSTE::apply(*x, *w, (int64_t)block, grad && x->requires_grad(), grad && w->requires_grad());
    } catch (const NotPlain&) {
        Py_RETURN_NONE;
    }
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// ---- a paged cache of keys and values held as codes ---------------------------------------------------------

// The four buffers of a cache, whose shapes agree, on the current device.
bool cache_of(PyObject* const* a, int fmt, int block, mxq_cache* c, c10::Device* dev)
{
    const at::Tensor* t[4];
    for (int i = 0; i < 4; ++i)
        if (!(t[i] = plain(a[i])) || t[i]->scalar_type() != at::kByte || t[i]->dim() != 4) return false;
    *dev = t[0]->device();
    const int64_t bits = fmt == MXQ_FP8_E4M3 || fmt == MXQ_INT8 ? 8 : fmt == MXQ_FP4_E2M1 || fmt == MXQ_INT4 ? 4 : 0;
    if (!bits || block <= 0) return false;
    const int64_t pages = t[0]->size(0), heads = t[0]->size(1), page = t[0]->size(2), dim = t[0]->size(3) * 8 / bits;
    if (heads > MXQ_CACHE_HEADS_MAX || page > 4096 || dim > 4096) return false;
    for (int i = 0; i < 4; ++i)
        if (!here(*t[i], *dev) || t[i]->size(0) != pages || t[i]->size(1) != heads || t[i]->size(2) != page ||
            t[i]->size(3) != (i % 2 ? dim / block : t[0]->size(3)))
            return false;
    *c = mxq_cache{t[0]->data_ptr(), bytes(*t[1]), t[2]->data_ptr(), bytes(*t[3]), (size_t)pages, (int)page, (int)heads, (int)dim, fmt, block};
    return true;
}

bool ints(PyObject* o, int64_t n, c10::Device dev, const int32_t** to)
{
    const at::Tensor* t = plain(o);
    if (!t || t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != n || !here(*t, dev)) return false;
    *to = static_cast<const int32_t*>(t->data_ptr());
    return true;
}

bool batch_of(PyObject* table, PyObject* lengths, PyObject* starts, c10::Device dev, mxq_batch* b)
{
    const at::Tensor* t = plain(table);
    if (!t || t->scalar_type() != at::kInt || t->dim() != 2 || !here(*t, dev)) return false;
    *b = mxq_batch{static_cast<const int32_t*>(t->data_ptr()), nullptr, nullptr, (size_t)t->size(0), (size_t)t->size(1)};
    return (!lengths || ints(lengths, t->size(0), dev, &b->lengths)) && (starts == Py_None || ints(starts, t->size(0) + 1, dev, &b->starts));
}

// A [tokens, heads, head_dim] tensor that the kernels take as it lies.
const at::Tensor* rows_of(PyObject* o, c10::Device dev, mxq_rows* r)
{
    if (!THPVariable_CheckExact(o) && Py_TYPE(o) != parameter) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    int dt;
    if (!t.defined() || !t.is_cuda() || t.unsafeGetTensorImpl()->is_python_dispatch() || !t.has_storage() || t.layout() != at::kStrided || t.dim() != 3 ||
        !dtype_id(t, &dt) || !here(t, dev))
        return nullptr;
    const int64_t size = t.element_size();
    if (t.stride(2) != 1 || t.stride(0) < 0 || t.stride(1) < 0 || t.stride(0) * size % 32 || t.stride(1) * size % 32) return nullptr;
    *r = mxq_rows{t.data_ptr(), (size_t)t.stride(0), (size_t)t.stride(1)};
    return &t;
}

// cache_write(k, v, k_codes, k_scales, v_codes, v_scales, table, lengths, fmt, block, starts, stream)
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, dt;
    mxq_cache c;
    mxq_batch b;
    mxq_rows kr, vr;
    c10::Device dev(c10::kCUDA, 0);
    GENERAL_UNLESS(nargs == 12 && a[11] == Py_None && format_id(a[8], &fmt) && as_int(a[9], &block) && !modes_active());
    GENERAL_UNLESS(cache_of(a + 2, fmt, block, &c, &dev) && batch_of(a[6], a[7], a[10], dev, &b));
    const at::Tensor *k = rows_of(a[0], dev, &kr), *v = rows_of(a[1], dev, &vr);
    GENERAL_UNLESS(k && v && dtype_id(*k, &dt) && v->scalar_type() == k->scalar_type() && k->sizes() == v->sizes() && k->size(1) == c.heads &&
                   k->size(2) == c.head_dim);
    const int rc = unlocked([&] { return api.cache_write(&c, &b, &kr, &vr, dt, (size_t)k->size(0), current_stream()); });
    GENERAL_UNLESS(rc == MXQ_OK);
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// cache_read(k_codes, k_scales, v_codes, v_scales, table, starts, total, fmt, block, dtype, out, stream), out None
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, dt;
    int64_t total;
    mxq_cache c;
    mxq_batch b;
    c10::Device dev(c10::kCUDA, 0);
    GENERAL_UNLESS(nargs == 12 && a[10] == Py_None && a[11] == Py_None && as_count(a[6], &total) && format_id(a[7], &fmt) && as_int(a[8], &block) &&
                   THPDtype_Check(a[9]) && !modes_active());
    const at::ScalarType type = reinterpret_cast<THPDtype*>(a[9])->scalar_type;
    GENERAL_UNLESS(dtype_id(type, &dt) && cache_of(a, fmt, block, &c, &dev) && a[5] != Py_None && batch_of(a[4], nullptr, a[5], dev, &b));
    at::Tensor k, v;
    const int rc = unlocked([&] {
        const auto options = at::TensorOptions().dtype(type).device(dev);
        k = at::empty({total, c.heads, c.head_dim}, options);
        v = at::empty({total, c.heads, c.head_dim}, options);
        return api.cache_read(&c, &b, (size_t)total, k.data_ptr(), v.data_ptr(), dt, current_stream());
    });
    GENERAL_UNLESS(rc == MXQ_OK);
    return pair(THPVariable_Wrap(k), THPVariable_Wrap(v));
    END_HANDLE_TH_ERRORS
}

// cache_attention(q, k_codes, k_scales, v_codes, v_scales, table, lengths, fmt, block, starts, scale, causal, window, out, lse, workspace, stream)
PyObject* cache_attention(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    int fmt, block, dt;
    int64_t window;
    mxq_cache c;
    mxq_batch b;
    mxq_rows qr;
    c10::Device dev(c10::kCUDA, 0);
    GENERAL_UNLESS(nargs == 17 && a[16] == Py_None && format_id(a[7], &fmt) && as_int(a[8], &block) && (a[10] == Py_None || PyFloat_CheckExact(a[10])) &&
                   PyBool_Check(a[11]) && as_count(a[12], &window) && !modes_active());
    GENERAL_UNLESS(cache_of(a + 1, fmt, block, &c, &dev) && batch_of(a[5], a[6], a[9], dev, &b));
    const at::Tensor* q = rows_of(a[0], dev, &qr);
    Output out, ws;
    GENERAL_UNLESS(q && dtype_id(*q, &dt) && q->size(2) == c.head_dim && q->size(1) <= (1 << 16) && out.take(a[13]) && ws.take(a[15]));
    GENERAL_UNLESS(!out.tensor || (out.tensor->sizes() == q->sizes() && out.tensor->scalar_type() == q->scalar_type() && here(*out.tensor, dev)));
    GENERAL_UNLESS(!ws.tensor || operand(ws.tensor, 0, dev));
    float* lse = nullptr;
    if (a[14] != Py_None) {
        const at::Tensor* t = plain(a[14]);
        GENERAL_UNLESS(t && t->scalar_type() == at::kFloat && t->dim() == 2 && t->size(0) == q->size(0) && t->size(1) == q->size(1) && here(*t, dev));
        lse = static_cast<float*>(t->data_ptr());
    }
    const int q_heads = (int)q->size(1);
    const size_t tokens = (size_t)q->size(0);
    const double scale = a[10] == Py_None ? 1 / std::sqrt((double)c.head_dim) : PyFloat_AS_DOUBLE(a[10]);
    const int rc = unlocked([&] {
        out.make(q->sizes(), q->scalar_type(), *q);
        ws.make({(int64_t)api.cache_attention_workspace_bytes(&c, &b, q_heads, dt, tokens)}, at::kByte, *q);
        return api.cache_attention(&c, &b, &qr, q_heads, dt, tokens, (float)scale, a[11] == Py_True, (size_t)window, out.data(), lse, ws.data(),
                                   (size_t)ws.tensor->numel(), current_stream());
    });
    // (the first of the call's two launches may precede the one that failed)
    if (rc == MXQ_ERR_CUDA) return raise_mxq_error(rc, "mxq_cache_attention");
    GENERAL_UNLESS(rc == MXQ_OK);
    return out.result(a[13]);
    END_HANDLE_TH_ERRORS
}

// bind(addresses by name, formats, torch.nn.Parameter, MxqError)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t nargs)
{
    if (nargs != 4 || !PyDict_Check(a[0]) || !PyDict_Check(a[1]) || !PyType_Check(a[2]) || !PyType_Check(a[3])) {
        PyErr_SetString(PyExc_TypeError, "bind(addresses, formats, parameter type, error type)");
        return nullptr;
    }
    bool ok = true;
    auto take = [&](const char* name, auto& fn) {
        PyObject* v = PyDict_GetItemString(a[0], name);
        void* p = v ? PyLong_AsVoidPtr(v) : nullptr;
        if (!p) ok = false;
        fn = reinterpret_cast<std::decay_t<decltype(fn)>>(p);
    };
    Api n{};
    take("mxq_quantize", n.quantize);
    take("mxq_slice_scale", n.slice_scale);
    take("mxq_slice_scale_multi", n.slice_scale_multi);
    take("mxq_dequantize", n.dequantize);
    take("mxq_tiled_scales_bytes", n.tiled_scales_bytes);
    take("mxq_quantize_tiled", n.quantize_tiled);
    take("mxq_slice_scale_tiled", n.slice_scale_tiled);
    take("mxq_fake_quant", n.fake_quant);
    take("mxq_fake_quant_bwd", n.fake_quant_bwd);
    take("mxq_codes_bytes", n.codes_bytes);
    take("mxq_matmul", n.matmul);
    take("mxq_quantize_matrix", n.quantize_matrix);
    take("mxq_matrix_codes_bytes", n.matrix_codes_bytes);
    take("mxq_matrix_scales_bytes", n.matrix_scales_bytes);
    take("mxq_moe", n.moe);
    take("mxq_moe_workspace_bytes", n.moe_workspace_bytes);
    take("mxq_cache_write", n.cache_write);
    take("mxq_cache_read", n.cache_read);
    take("mxq_cache_attention", n.cache_attention);
    take("mxq_cache_attention_workspace_bytes", n.cache_attention_workspace_bytes);
    if (!ok) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, "an entry point has no address");
        return nullptr;
    }
    api = n;
    Py_INCREF(a[1]);
    Py_INCREF(a[2]);
    Py_INCREF(a[3]);
    Py_XSETREF(mxq_error, a[3]);
    Py_XSETREF(formats, a[1]);
    Py_XSETREF(parameter, reinterpret_cast<PyTypeObject*>(a[2]));
    Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(bind),           FAST(quantize),          FAST(slice_scale), FAST(slice_scale_multi),
                         FAST(dequantize),     FAST(quantize_tiled),    FAST(slice_scale_tiled), FAST(fake_quant),
                         FAST(fake_quant_bwd), FAST(run_prepared),      FAST(fake_quant_ste),
                         FAST(matmul),         FAST(quantize_matrix),   FAST(moe),         FAST(linear_ste),
                         FAST(cache_write),    FAST(cache_read),        FAST(cache_attention), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mxq_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mxq_host() { return PyModule_Create(&module); }
