// train_ops.cpp -- the Python module _train_ops: checks tensors, allocates results and calls the C ABI for the operators of
// the training step (include/ssgd.h).  train_ops.py documents the functions and holds their signatures; what is here is what
// a ctypes call would do, in a tenth of its time: the smallest of these operators take the GPU two microseconds.
//
// Every function takes its arguments by position, None for what is left out.  Errors of the C ABI are raised as the class
// given to set_error_class.
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <string>
#include <vector>

#include "../../include/ssgd.h"

namespace {

PyObject* g_error_class = nullptr;

// An exception that is already set in Python
struct Raised {};

[[noreturn]] void raise(PyObject* type, const std::string& what) {
    PyErr_SetString(type, what.c_str());
    throw Raised{};
}
void check(int code, const char* what) {
    if (code == SSGD_OK) return;
    if (g_error_class) {
        PyObject* e = PyObject_CallFunction(g_error_class, "is", code, what);
        if (e) {
            PyErr_SetObject(g_error_class, e);
            Py_DECREF(e);
        }
    } else {
        PyErr_Format(PyExc_RuntimeError, "%s: %s", what, ssgd_strerror(code));
    }
    throw Raised{};
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, std::string(name) + ": need a tensor");
    return THPVariable_Unpack(o);
}
const at::Tensor* optional_tensor(PyObject* o, const char* name) { return o == Py_None ? nullptr : &tensor(o, name); }

// The device of a call's first tensor, which has to be the current one
int device_of(const at::Tensor& t, const char* name) {
    if (!t.is_cuda()) raise(PyExc_TypeError, std::string(name) + ": need a CUDA tensor");
    const int dev = (int)t.get_device(), current = (int)c10::cuda::current_device();
    if (dev != current)
        raise(PyExc_ValueError, std::string(name) + ": on device " + std::to_string(dev) + ", but the current device is " + std::to_string(current));
    return dev;
}

struct Rows { int64_t rows, n, ld; };
// A tensor read as rows of its last dimension
Rows rows_of(const at::Tensor& t, const char* name, int dev) {
    if (!t.is_cuda() || t.get_device() != dev) raise(PyExc_TypeError, std::string(name) + ": need a tensor on CUDA device " + std::to_string(dev));
    if (t.dim() == 2) {
        Rows r{t.size(0), t.size(1), t.stride(0)};
        if (r.n > 1 && t.stride(1) != 1) raise(PyExc_TypeError, std::string(name) + ": the elements of a row must be adjacent");
        if (r.rows <= 1) r.ld = r.n;
        else if (r.ld < r.n) raise(PyExc_TypeError, std::string(name) + ": rows overlap");
        return r;
    }
    if (t.dim() > 0 && t.is_contiguous()) {
        const int64_t n = t.size(-1);
        return Rows{n ? t.numel() / n : 0, n, n};
    }
    raise(PyExc_TypeError, std::string(name) + ": need a 2-dimensional tensor with adjacent row elements, or a contiguous one");
}

int32_t format_of(const at::Tensor& t, const char* name) {
    switch (t.scalar_type()) {
        case at::kFloat: return SSGD_FMT_F32;
        case at::kHalf: return SSGD_FMT_F16;
        case at::kBFloat16: return SSGD_FMT_BF16;
        default: raise(PyExc_TypeError, std::string(name) + ": need float32, float16 or bfloat16");
    }
}

// Address of a contiguous tensor of n elements of a type; NULL for one that is left out
void* flat(const at::Tensor* t, at::ScalarType type, int64_t n, const char* name, int dev) {
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->numel() != n || !t->is_contiguous() || !t->is_cuda() || t->get_device() != dev)
        raise(PyExc_TypeError, std::string(name) + ": need a contiguous tensor of " + std::to_string(n) + " elements of " +
                                   std::string(at::toString(type)) + " on CUDA device " + std::to_string(dev));
    return t->data_ptr();
}
float* flat_f32(const at::Tensor* t, int64_t n, const char* name, int dev) {
    return static_cast<float*>(flat(t, at::kFloat, n, name, dev));
}

// A new tensor, without the detour over the dispatcher
at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type, int dev) {
    return at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, (c10::DeviceIndex)dev), std::nullopt);
}

// The tensor that a result goes to: the caller's, which has to be like `like`, or a new contiguous one
at::Tensor result_like(const at::Tensor* out, const at::Tensor& like, const char* name, int dev, int64_t* ld, const char* of) {
    if (!out) {
        *ld = like.dim() ? like.size(-1) : 1;
        return fresh(like.sizes(), like.scalar_type(), dev);
    }
    if (out->sizes() != like.sizes() || out->scalar_type() != like.scalar_type())
        raise(PyExc_TypeError, std::string(name) + ": need " + of + " shape and type");
    *ld = rows_of(*out, name, dev).ld;
    return *out;
}
// A tensor of the caller's that has been written to (NULL: none): autograd has to know.  Behind the launch, so that a call that
// is refused leaves it as it was.
void written(const at::Tensor* t) {
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}
at::Tensor new_f32(at::IntArrayRef shape, int dev) { return fresh(shape, at::kFloat, dev); }

void* stream_of(int dev) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream(); }

int64_t integer(PyObject* o, const char* name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        raise(PyExc_TypeError, std::string(name) + ": need an integer");
    }
    return v;
}
double number(PyObject* o, const char* name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        raise(PyExc_TypeError, std::string(name) + ": need a number");
    }
    return v;
}
PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* wrap_or_none(const at::Tensor& t) {
    if (t.defined()) return wrap(t);
    Py_RETURN_NONE;
}

// (x, weight, bias, eps, out) -> (y, stats)
PyObject* layer_norm(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const int dev = device_of(x, "x");
    const Rows r = rows_of(x, "x", dev);
    const int32_t fmt = format_of(x, "x");
    const at::Tensor *w = optional_tensor(a[1], "weight"), *b = optional_tensor(a[2], "bias");
    const at::Tensor* param = w ? w : b;
    const int32_t fmt_w = param ? format_of(*param, "weight") : fmt;
    const at::ScalarType type_w = param ? param->scalar_type() : x.scalar_type();
    const void *wp = flat(w, type_w, r.n, "weight", dev), *bp = flat(b, type_w, r.n, "bias", dev);
    int64_t ld_y = 0;
    const at::Tensor* out = optional_tensor(a[4], "out");
    at::Tensor y = result_like(out, x, "out", dev, &ld_y, "x's");
    at::Tensor stats = new_f32({2, r.rows}, dev);
    check(ssgd_layer_norm(x.data_ptr(), r.ld, fmt, wp, bp, fmt_w, r.rows, r.n, (float)number(a[3], "eps"), y.data_ptr(), ld_y,
                          stats.data_ptr<float>(), stream_of(dev)), "ssgd_layer_norm");
    written(out);
    return Py_BuildValue("(NN)", wrap(y), wrap(stats));
}

// (dy, x, weight, stats, dx, dw, db, accumulate, need_params) -> (dx, dw, db)
PyObject* layer_norm_backward(PyObject* const* a) {
    const at::Tensor& x = tensor(a[1], "x");
    const int dev = device_of(x, "x");
    const Rows r = rows_of(x, "x", dev);
    const int32_t fmt = format_of(x, "x");
    const at::Tensor& dy = tensor(a[0], "dy");
    if (dy.sizes() != x.sizes() || dy.scalar_type() != x.scalar_type()) raise(PyExc_TypeError, "dy: need x's shape and type");
    const Rows rd = rows_of(dy, "dy", dev);
    const at::Tensor* w = optional_tensor(a[2], "weight");
    const int32_t fmt_w = w ? format_of(*w, "weight") : fmt;
    const void* wp = w ? flat(w, w->scalar_type(), r.n, "weight", dev) : nullptr;
    const float* stats = flat_f32(&tensor(a[3], "stats"), 2 * r.rows, "stats", dev);
    int64_t ld_dx = 0;
    const at::Tensor* dx_in = optional_tensor(a[4], "dx");
    at::Tensor dx = result_like(dx_in, x, "dx", dev, &ld_dx, "x's");
    const at::Tensor *dw_in = optional_tensor(a[5], "dw"), *db_in = optional_tensor(a[6], "db");
    const bool accumulate = PyObject_IsTrue(a[7]), need = PyObject_IsTrue(a[8]);
    at::Tensor dw, db;
    if (need) {
        if (accumulate && (!dw_in || !db_in)) raise(PyExc_ValueError, "accumulate: needs dw and db");
        dw = dw_in ? *dw_in : new_f32({r.n}, dev);
        db = db_in ? *db_in : new_f32({r.n}, dev);
    }
    float *dwp = need ? flat_f32(&dw, r.n, "dw", dev) : nullptr, *dbp = need ? flat_f32(&db, r.n, "db", dev) : nullptr;
    size_t bytes = 0;
    check(ssgd_layer_norm_backward_workspace(r.rows, r.n, &bytes), "ssgd_layer_norm_backward_workspace");
    // of the current stream: what is enqueued below runs before anything that gets this memory next
    const c10::DataPtr ws = c10::cuda::CUDACachingAllocator::get()->allocate(bytes);
    check(ssgd_layer_norm_backward(dy.data_ptr(), rd.ld, x.data_ptr(), r.ld, fmt, wp, fmt_w, stats, r.rows, r.n, dx.data_ptr(), ld_dx, dwp,
                                   dbp, accumulate ? 1 : 0, ws.get(), bytes, stream_of(dev)), "ssgd_layer_norm_backward");
    written(dx_in);
    if (need) { written(dw_in); written(db_in); }
    return Py_BuildValue("(NNN)", wrap(dx), wrap_or_none(dw), wrap_or_none(db));
}

struct Ids { const void* p; int32_t bytes; };
Ids ids_of(const at::Tensor& ids, int64_t rows, int dev) {
    const at::ScalarType type = ids.scalar_type();
    if (type != at::kLong && type != at::kInt) raise(PyExc_TypeError, "ids: need int64 or int32");
    return Ids{flat(&ids, type, rows, "ids", dev), type == at::kLong ? 8 : 4};
}
Rows logits_of(const at::Tensor& z, int dev) {
    if (z.dim() != 2) raise(PyExc_TypeError, "logits: need [rows][vocab]");
    return rows_of(z, "logits", dev);
}

// (logits, ids, top, scale) -> (stats, top_idx, top_logp)
PyObject* token_logprobs(PyObject* const* a) {
    const at::Tensor& z = tensor(a[0], "logits");
    const int dev = device_of(z, "logits");
    const Rows r = logits_of(z, dev);
    const int32_t fmt = format_of(z, "logits");
    const Ids ids = ids_of(tensor(a[1], "ids"), r.rows, dev);
    const int64_t top = integer(a[2], "top");
    if (top < 0 || top > INT32_MAX) check(SSGD_EINVAL, "ssgd_token_logprobs");
    at::Tensor stats = new_f32({3, r.rows}, dev), idx, logp;
    if (top > SSGD_MAX_TOP) check(SSGD_ETOOBIG, "ssgd_token_logprobs");
    if (top) {
        idx = fresh({r.rows, top}, at::kInt, dev);
        logp = new_f32({r.rows, top}, dev);
    }
    check(ssgd_token_logprobs(z.data_ptr(), r.ld, fmt, ids.p, ids.bytes, r.rows, r.n, (float)number(a[3], "scale"), (int32_t)top,
                              stats.data_ptr<float>(), top ? idx.data_ptr<int32_t>() : nullptr, top ? logp.data_ptr<float>() : nullptr,
                              stream_of(dev)), "ssgd_token_logprobs");
    return Py_BuildValue("(NNN)", wrap(stats), wrap_or_none(idx), wrap_or_none(logp));
}

// (logits, ids, lse, d_logp, entropy, d_entropy, top_idx, d_top, scale, out) -> dlogits
PyObject* token_logprobs_backward(PyObject* const* a) {
    const at::Tensor& z = tensor(a[0], "logits");
    const int dev = device_of(z, "logits");
    const Rows r = logits_of(z, dev);
    const int32_t fmt = format_of(z, "logits");
    const Ids ids = ids_of(tensor(a[1], "ids"), r.rows, dev);
    const float* lse = flat_f32(&tensor(a[2], "lse"), r.rows, "lse", dev);
    const float* d_logp = flat_f32(optional_tensor(a[3], "d_logp"), r.rows, "d_logp", dev);
    const float* entropy = flat_f32(optional_tensor(a[4], "entropy"), r.rows, "entropy", dev);
    const float* d_entropy = flat_f32(optional_tensor(a[5], "d_entropy"), r.rows, "d_entropy", dev);
    const at::Tensor *idx = optional_tensor(a[6], "top_idx"), *d_top = optional_tensor(a[7], "d_top");
    if (!idx != !d_top) raise(PyExc_ValueError, "top_idx and d_top: give both or neither");
    if (d_entropy && !entropy) raise(PyExc_ValueError, "d_entropy: needs the forward pass's entropy");
    int64_t top = 0;
    if (idx) {
        if (idx->dim() != 2 || idx->size(0) != r.rows) raise(PyExc_TypeError, "top_idx: need [rows][top]");
        top = idx->size(1);
        if (top > SSGD_MAX_TOP) check(SSGD_ETOOBIG, "ssgd_token_logprobs_backward");
    }
    const int32_t* idx_p = static_cast<int32_t*>(flat(idx, at::kInt, r.rows * top, "top_idx", dev));
    const float* d_top_p = flat_f32(d_top, r.rows * top, "d_top", dev);
    int64_t ld_out = 0;
    const at::Tensor* out_in = optional_tensor(a[9], "out");
    at::Tensor out = result_like(out_in, z, "out", dev, &ld_out, "the logits'");
    check(ssgd_token_logprobs_backward(z.data_ptr(), r.ld, fmt, ids.p, ids.bytes, r.rows, r.n, (float)number(a[8], "scale"), lse, entropy,
                                       d_logp, d_entropy, (int32_t)top, idx_p, d_top_p, out.data_ptr(), ld_out, stream_of(dev)),
          "ssgd_token_logprobs_backward");
    written(out_in);
    return wrap(out);
}

// One member of all descriptors from a list of tensors.  They are looked at in every step: a parameter may have been given
// other storage in the meantime.
template <typename F>
void column(PyObject* list, Py_ssize_t count, const char* name, at::ScalarType type, int dev, const int64_t* sizes, int64_t per, F set) {
    if (!PyList_Check(list) || PyList_GET_SIZE(list) != count) raise(PyExc_ValueError, std::string(name) + ": need one tensor per parameter");
    for (Py_ssize_t i = 0; i < count; ++i) {
        const at::Tensor& t = tensor(PyList_GET_ITEM(list, i), name);
        const int64_t n = (sizes[i] + per - 1) / per;
        if (t.scalar_type() != type || t.numel() != n || !t.is_contiguous() || !t.is_cuda() || t.get_device() != dev)
            raise(PyExc_TypeError, std::string(name) + "[" + std::to_string(i) + "]: need a contiguous tensor of " + std::to_string(n) +
                                       " elements of " + std::string(at::toString(type)) + " on CUDA device " + std::to_string(dev));
        set(i, t);
    }
}

// An object's memory, held for the duration of a call
struct Memory {
    Py_buffer view{};
    explicit Memory(PyObject* o) {
        if (PyObject_GetBuffer(o, &view, PyBUF_CONTIG) != 0) throw Raised{};
    }
    ~Memory() { PyBuffer_Release(&view); }
    Memory(const Memory&) = delete;
    Memory& operator=(const Memory&) = delete;
};

// (buffer, params, m, v, m_scale, v_scale, copies, grads, device, lr, b1, b2, eps, decay, step, grad_scale, seed): the buffer (int64: room
// for an ssgd_adamw_tensor per parameter and, behind them all, a size per parameter); the lists; None for what there is not
PyObject* adamw_step(PyObject* const* a) {
    const Memory memory(a[0]);
    auto* desc = static_cast<ssgd_adamw_tensor*>(memory.view.buf);
    const int dev = (int)integer(a[8], "device");
    if (dev != (int)c10::cuda::current_device())
        raise(PyExc_ValueError, "grads: the parameters are on device " + std::to_string(dev) + ", which is not the current one");
    const Py_ssize_t count = memory.view.len / (Py_ssize_t)(sizeof(ssgd_adamw_tensor) + 8);
    if (count < 1 || !PyList_Check(a[1]) || PyList_GET_SIZE(a[1]) != count) raise(PyExc_ValueError, "params: not as many as there were");
    const auto* sizes = reinterpret_cast<const int64_t*>(desc + count);
    const at::ScalarType type_p = tensor(PyList_GET_ITEM(a[1], 0), "params").scalar_type();
    if (type_p != at::kFloat && type_p != at::kBFloat16) raise(PyExc_TypeError, "params: need float32 or bfloat16");
    const bool small = a[4] != Py_None, copied = a[6] != Py_None;
    const at::ScalarType type_s = small ? at::kFloat8_e4m3fn : at::kFloat;
    PyObject* grads = a[7];
    if ((!PyList_Check(grads) && !PyTuple_Check(grads)) || PySequence_Fast_GET_SIZE(grads) != count)
        raise(PyExc_ValueError, "grads: need one tensor per parameter");
    PyObject** items = PySequence_Fast_ITEMS(grads);
    at::ScalarType type = at::kFloat;
    bool known = false;
    for (Py_ssize_t i = 0; i < count; ++i) {
        desc[i] = ssgd_adamw_tensor{};
        if (items[i] == Py_None) continue;                 // left alone: no elements
        const at::Tensor& g = tensor(items[i], "grads");
        if (!known) type = g.scalar_type();
        known = true;
        if (g.scalar_type() != type || g.numel() != sizes[i] || !g.is_contiguous() || !g.is_cuda() || g.get_device() != dev)
            raise(PyExc_TypeError, "grads[" + std::to_string(i) + "]: need a contiguous tensor of " + std::to_string(sizes[i]) + " elements of " +
                                       std::string(at::toString(type)) + " on CUDA device " + std::to_string(dev));
        desc[i].g = g.data_ptr();
        desc[i].n = sizes[i];
    }
    int32_t fmt_g = SSGD_FMT_F32, fmt_copy = SSGD_FMT_BF16;
    if (type == at::kBFloat16) fmt_g = SSGD_FMT_BF16;
    else if (type == at::kHalf) fmt_g = SSGD_FMT_F16;
    else if (type != at::kFloat) raise(PyExc_TypeError, "grads: need float32, bfloat16 or float16");
    column(a[1], count, "params", type_p, dev, sizes, 1, [&](Py_ssize_t i, const at::Tensor& t) { desc[i].p = t.data_ptr(); });
    column(a[2], count, "m", type_s, dev, sizes, 1, [&](Py_ssize_t i, const at::Tensor& t) { desc[i].m = t.data_ptr(); });
    column(a[3], count, "v", type_s, dev, sizes, 1, [&](Py_ssize_t i, const at::Tensor& t) { desc[i].v = t.data_ptr(); });
    if (small) {
        column(a[4], count, "m_scale", at::kFloat, dev, sizes, SSGD_ADAMW_BLOCK,
               [&](Py_ssize_t i, const at::Tensor& t) { desc[i].m_scale = static_cast<float*>(t.data_ptr()); });
        column(a[5], count, "v_scale", at::kFloat, dev, sizes, SSGD_ADAMW_BLOCK,
               [&](Py_ssize_t i, const at::Tensor& t) { desc[i].v_scale = static_cast<float*>(t.data_ptr()); });
    }
    if (copied) {
        if (!PyList_Check(a[6]) || PyList_GET_SIZE(a[6]) != count) raise(PyExc_ValueError, "copies: need one tensor per parameter");
        const at::ScalarType type_c = tensor(PyList_GET_ITEM(a[6], 0), "copies").scalar_type();
        if (type_c != at::kHalf && type_c != at::kBFloat16) raise(PyExc_TypeError, "copies: need bfloat16 or float16");
        fmt_copy = type_c == at::kHalf ? SSGD_FMT_F16 : SSGD_FMT_BF16;
        column(a[6], count, "copies", type_c, dev, sizes, 1, [&](Py_ssize_t i, const at::Tensor& t) { desc[i].copy = t.data_ptr(); });
    }
    const float* grad_scale = flat_f32(optional_tensor(a[15], "grad_scale"), 1, "grad_scale", dev);
    const bool stochastic = a[16] != Py_None;
    const uint64_t seed = stochastic ? PyLong_AsUnsignedLongLongMask(a[16]) : 0;
    if (PyErr_Occurred()) throw Raised{};
    check(ssgd_adamw_step(desc, (int32_t)count, type_p == at::kBFloat16 ? SSGD_FMT_BF16 : SSGD_FMT_F32, fmt_g,
                          small ? SSGD_FMT_E4M3 : SSGD_FMT_F32, fmt_copy, number(a[9], "lr"), number(a[10], "beta1"), number(a[11], "beta2"),
                          number(a[12], "eps"), number(a[13], "weight_decay"), integer(a[14], "step"), grad_scale, stochastic, seed,
                          stream_of(dev)), "ssgd_adamw_step");
    for (Py_ssize_t i = 0; i < count; ++i) {
        if (!desc[i].n) continue;
        written(&tensor(PyList_GET_ITEM(a[1], i), "params"));
        if (copied) written(&tensor(PyList_GET_ITEM(a[6], i), "copies"));
    }
    Py_RETURN_NONE;
}

// Memory of the current stream: what is enqueued behind runs before anything that gets it next
c10::DataPtr scratch(size_t bytes) { return c10::cuda::CUDACachingAllocator::get()->allocate(bytes); }

// (logits, ids, old_logp, advantages, ref_logp, weights, low, high, kl, entropy, scale, need_grad, out) -> (stats, dlogits)
PyObject* policy_loss(PyObject* const* a) {
    const at::Tensor& z = tensor(a[0], "logits");
    const int dev = device_of(z, "logits");
    const Rows r = logits_of(z, dev);
    const int32_t fmt = format_of(z, "logits");
    const Ids ids = ids_of(tensor(a[1], "ids"), r.rows, dev);
    const float *old_logp = flat_f32(&tensor(a[2], "old_logp"), r.rows, "old_logp", dev),
                *advantages = flat_f32(&tensor(a[3], "advantages"), r.rows, "advantages", dev),
                *ref_logp = flat_f32(optional_tensor(a[4], "ref_logp"), r.rows, "ref_logp", dev),
                *weights = flat_f32(optional_tensor(a[5], "weights"), r.rows, "weights", dev);
    const float low = (float)number(a[6], "clip"), high = (float)number(a[7], "clip"), kl = (float)number(a[8], "kl"),
                entropy = (float)number(a[9], "entropy"), scale = (float)number(a[10], "scale");
    if (kl != 0.f && !ref_logp) raise(PyExc_ValueError, "kl: needs ref_logp");
    const at::Tensor* out_in = optional_tensor(a[12], "out");
    const bool need = PyObject_IsTrue(a[11]);
    if (out_in && !need) raise(PyExc_ValueError, "out: only with need_grad");
    int64_t ld_out = 0;
    at::Tensor stats = new_f32({5, r.rows}, dev), out;
    if (need) out = result_like(out_in, z, "out", dev, &ld_out, "the logits'");
    check(ssgd_policy_loss(z.data_ptr(), r.ld, fmt, ids.p, ids.bytes, r.rows, r.n, scale, old_logp, advantages, ref_logp, weights, low, high, kl,
                           entropy, stats.data_ptr<float>(), need ? out.data_ptr() : nullptr, ld_out, stream_of(dev)), "ssgd_policy_loss");
    written(out_in);
    return Py_BuildValue("(NN)", wrap(stats), wrap_or_none(out));
}

// (logp, ref_logp, starts, weights, kind, beta, smoothing, average, need_grad, out) -> (loss, rewards, d_logp)
PyObject* preference_loss(PyObject* const* a) {
    const at::Tensor& logp = tensor(a[0], "logp");
    const int dev = device_of(logp, "logp");
    const int64_t tokens = logp.numel();
    const float *lp = flat_f32(&logp, tokens, "logp", dev), *ref = flat_f32(optional_tensor(a[1], "ref_logp"), tokens, "ref_logp", dev);
    const at::Tensor& starts = tensor(a[2], "starts");
    const at::ScalarType type = starts.scalar_type();
    if (type != at::kLong && type != at::kInt) raise(PyExc_TypeError, "starts: need int64 or int32");
    const int64_t n = starts.numel();
    if (n % 2 != 1) raise(PyExc_ValueError, "starts: need two per pair and the end");
    const void* sp = flat(&starts, type, n, "starts", dev);
    const int64_t pairs = n / 2;
    const float* weights = flat_f32(optional_tensor(a[3], "weights"), pairs, "weights", dev);
    const at::Tensor* out_in = optional_tensor(a[9], "out");
    const bool need = PyObject_IsTrue(a[8]);
    if (out_in && !need) raise(PyExc_ValueError, "out: only with need_grad");
    at::Tensor loss = new_f32({pairs}, dev), rewards = new_f32({2, pairs}, dev), d;
    if (need) d = out_in ? *out_in : new_f32(logp.sizes(), dev);
    float* dp = need ? flat_f32(&d, tokens, "out", dev) : nullptr;
    size_t bytes = 0;
    check(ssgd_preference_loss_workspace(tokens, pairs, &bytes), "ssgd_preference_loss_workspace");
    const c10::DataPtr ws = scratch(bytes);
    check(ssgd_preference_loss(lp, ref, tokens, sp, type == at::kLong ? 8 : 4, pairs, weights, (int32_t)integer(a[4], "kind"),
                               (float)number(a[5], "beta"), (float)number(a[6], "label_smoothing"), PyObject_IsTrue(a[7]),
                               loss.data_ptr<float>(), rewards.data_ptr<float>(), dp, ws.get(), bytes, stream_of(dev)), "ssgd_preference_loss");
    written(out_in);
    return Py_BuildValue("(NNN)", wrap(loss), wrap(rewards), wrap_or_none(d));
}

// (x, steps, a, b, c, eps, products, out) -> the orthogonalised x
PyObject* orthogonalize(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const int dev = device_of(x, "x");
    if (x.dim() < 2) raise(PyExc_TypeError, "x: need a matrix, or a batch of them");
    const int32_t fmt = format_of(x, "x");
    const Rows r = rows_of(x, "x", dev);
    int64_t ld_out = 0;
    const at::Tensor* out_in = optional_tensor(a[7], "out");
    at::Tensor out = result_like(out_in, x, "out", dev, &ld_out, "x's");
    const int64_t rows = x.size(-2), cols = x.size(-1), count = rows * cols ? x.numel() / (rows * cols) : 0;
    if (count > INT32_MAX) check(SSGD_ETOOBIG, "ssgd_orthogonalize");
    std::vector<ssgd_matrix> list((size_t)count);
    const int64_t bytes_each = x.element_size();
    for (int64_t i = 0; i < count; ++i)
        list[i] = ssgd_matrix{static_cast<char*>(out.data_ptr()) + i * rows * ld_out * bytes_each,
                              static_cast<const char*>(x.data_ptr()) + i * rows * r.ld * bytes_each, nullptr, ld_out, r.ld, rows, cols, 0.0};
    const int32_t products = (int32_t)integer(a[6], "products");
    size_t bytes = 0;
    check(ssgd_orthogonalize_workspace(list.data(), (int32_t)count, fmt, products, &bytes), "ssgd_orthogonalize_workspace");
    const c10::DataPtr ws = scratch(bytes);
    check(ssgd_orthogonalize(list.data(), (int32_t)count, fmt, products, (int32_t)integer(a[1], "steps"), number(a[2], "coefficients"),
                             number(a[3], "coefficients"), number(a[4], "coefficients"), number(a[5], "eps"), ws.get(), bytes, stream_of(dev)),
          "ssgd_orthogonalize");
    written(out_in);
    return wrap(out);
}

// (params, m, scales, grads, device, lr, momentum, nesterov, decay, steps, a, b, c, eps, products, grad_scale): lists of as many members
PyObject* muon_step(PyObject* const* a) {
    const int dev = (int)integer(a[4], "device");
    if (dev != (int)c10::cuda::current_device())
        raise(PyExc_ValueError, "grads: the parameters are on device " + std::to_string(dev) + ", which is not the current one");
    for (int i = 0; i < 3; ++i)
        if (!PyList_Check(a[i]) || PyList_GET_SIZE(a[i]) != PyList_GET_SIZE(a[0])) raise(PyExc_ValueError, "params: not as many as there were");
    const Py_ssize_t count = PyList_GET_SIZE(a[0]);
    PyObject* grads = a[3];
    if ((!PyList_Check(grads) && !PyTuple_Check(grads)) || PySequence_Fast_GET_SIZE(grads) != count)
        raise(PyExc_ValueError, "grads: need one tensor per parameter");
    PyObject** items = PySequence_Fast_ITEMS(grads);
    std::vector<ssgd_matrix> list;
    at::ScalarType type_p = at::kFloat, type_g = at::kFloat;
    bool known = false;
    for (Py_ssize_t i = 0; i < count; ++i) {
        if (items[i] == Py_None) continue;                 // left alone
        const at::Tensor &p = tensor(PyList_GET_ITEM(a[0], i), "params"), &m = tensor(PyList_GET_ITEM(a[1], i), "m"), &g = tensor(items[i], "grads");
        if (!known) {
            type_p = p.scalar_type();
            type_g = g.scalar_type();
        }
        known = true;
        const std::string at = "[" + std::to_string(i) + "]";
        auto whole = [&](const at::Tensor& t, at::ScalarType type, const char* name) {
            if (t.scalar_type() != type || t.sizes() != p.sizes() || !t.is_contiguous() || !t.is_cuda() || t.get_device() != dev)
                raise(PyExc_TypeError, name + at + ": need a contiguous tensor of the parameter's shape of " + std::string(at::toString(type)) +
                                           " on CUDA device " + std::to_string(dev));
        };
        if (p.dim() < 2) raise(PyExc_TypeError, "params" + at + ": need a matrix, or a batch of them");
        whole(p, type_p, "params");
        whole(m, at::kFloat, "m");
        whole(g, type_g, "grads");
        const double scale = number(PyList_GET_ITEM(a[2], i), "scale");
        const int64_t rows = p.size(-2), cols = p.size(-1), each = rows * cols, n = each ? p.numel() / each : 0;
        for (int64_t j = 0; j < n; ++j)
            list.push_back(ssgd_matrix{static_cast<char*>(p.data_ptr()) + j * each * (int64_t)p.element_size(),
                                       static_cast<const char*>(g.data_ptr()) + j * each * (int64_t)g.element_size(),
                                       static_cast<float*>(m.data_ptr()) + j * each, cols, cols, rows, cols, scale});
    }
    if (list.empty()) Py_RETURN_NONE;
    if (list.size() > INT32_MAX) check(SSGD_ETOOBIG, "ssgd_muon_step");
    if (type_p != at::kFloat && type_p != at::kBFloat16) raise(PyExc_TypeError, "params: need float32 or bfloat16");
    int32_t fmt_g = SSGD_FMT_F32;
    const int32_t fmt_p = type_p == at::kBFloat16 ? SSGD_FMT_BF16 : SSGD_FMT_F32;
    if (type_g == at::kBFloat16) fmt_g = SSGD_FMT_BF16;
    else if (type_g == at::kHalf) fmt_g = SSGD_FMT_F16;
    else if (type_g != at::kFloat) raise(PyExc_TypeError, "grads: need float32, bfloat16 or float16");
    const float* grad_scale = flat_f32(optional_tensor(a[15], "grad_scale"), 1, "grad_scale", dev);
    const int32_t products = (int32_t)integer(a[14], "products");
    size_t bytes = 0;
    check(ssgd_orthogonalize_workspace(list.data(), (int32_t)list.size(), fmt_p, products, &bytes), "ssgd_orthogonalize_workspace");
    const c10::DataPtr ws = scratch(bytes);
    check(ssgd_muon_step(list.data(), (int32_t)list.size(), fmt_p, fmt_g, products, number(a[5], "lr"), number(a[6], "momentum"),
                         PyObject_IsTrue(a[7]), number(a[8], "weight_decay"), (int32_t)integer(a[9], "steps"), number(a[10], "coefficients"),
                         number(a[11], "coefficients"), number(a[12], "coefficients"), number(a[13], "eps"), grad_scale, ws.get(), bytes,
                         stream_of(dev)), "ssgd_muon_step");
    for (Py_ssize_t i = 0; i < count; ++i) {
        if (items[i] == Py_None) continue;
        written(&tensor(PyList_GET_ITEM(a[0], i), "params"));
        written(&tensor(PyList_GET_ITEM(a[1], i), "m"));
    }
    Py_RETURN_NONE;
}

PyObject* status(PyObject* const*) {
    check(ssgd_train_ops_status(stream_of((int)c10::cuda::current_device())), "ssgd_train_ops_status");
    Py_RETURN_NONE;
}

PyObject* set_error_class(PyObject* const* a) {
    Py_INCREF(a[0]);
    Py_XDECREF(g_error_class);
    g_error_class = a[0];
    Py_RETURN_NONE;
}

// No C++ exception leaves the module
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "need %d arguments", N);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const Raised&) {
        return nullptr;
    } catch (const std::exception& e) {        // torch's allocator, out of memory
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define ENTRY(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<name, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(layer_norm, 5), ENTRY(layer_norm_backward, 9), ENTRY(token_logprobs, 4), ENTRY(token_logprobs_backward, 10),
                         ENTRY(adamw_step, 17), ENTRY(policy_loss, 13), ENTRY(preference_loss, 10), ENTRY(orthogonalize, 8),
                         ENTRY(muon_step, 16), ENTRY(status, 0),
                         ENTRY(set_error_class, 1), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train_ops", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train_ops() { return PyModule_Create(&module); }
