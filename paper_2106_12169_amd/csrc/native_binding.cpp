// Python module `_native`: the per-call half of binding.py and network.py in native code.
//
// A call on a small layer takes the GPU about 4 us, so what the host spends per call is what such a layer costs.
// Through ctypes (argument conversion, a tensor check and a stream look-up in Python per call) that was 6 - 8 us, of
// which the launch itself is about 2; a network pass of 19 launches was bound by it (181 us of host work against
// 131 us on the GPU).  Here the tensors are unpacked through torch's own C++ interface and the entry point of
// include/apnn.h is called directly; a Chain holds the descriptors and tensors of a whole network and enqueues it
// with one call.  Nothing is computed here, and nothing depends on values: marshalling only.
//
// As with ctypes, the interpreter lock is released while the library runs (a launch can wait for queue space).
#include <Python.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <c10/util/SmallVector.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstring>
#include <exception>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "../../include/apnn.h"

namespace {

PyObject *g_error = nullptr;                              // binding.ApnnError

void *current_stream() { return static_cast<void *>(c10::hip::getCurrentHIPStream().stream()); }

// Status of a library call -> None, or ApnnError(status, text).
PyObject *finish(int status)
{
    if (status == APNN_OK) Py_RETURN_NONE;
    PyObject *args = Py_BuildValue("(is)", status, apnn_last_error());
    PyObject *e = args && g_error ? PyObject_CallObject(g_error, args) : nullptr;
    Py_XDECREF(args);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
        PyErr_SetString(PyExc_RuntimeError, apnn_last_error());
    }
    return nullptr;
}

// A Python object that is held (made, moved and dropped with the interpreter lock).
class Held {
public:
    explicit Held(PyObject *o) : o_(o) { Py_INCREF(o_); }
    Held(Held &&other) noexcept : o_(std::exchange(other.o_, nullptr)) {}
    Held &operator=(Held &&) = delete;
    ~Held() { Py_XDECREF(o_); }
    PyObject *get() const { return o_; }

private:
    PyObject *o_;
};

// A tensor whose device pointer stands `offset` bytes into a recorded step.  The Python object is held, as by any other
// owner: what it stands for can be exchanged (torch.utils.swap_tensors), which a reference to its tensor would forbid.
struct Ref {
    size_t offset;
    Held tensor;
};

// What a kernel is given of a tensor: its device pointer.  False (Python error set) if it has none that can be used.
bool device_pointer(const at::Tensor &t, void *&p)
{
    if (t.is_cuda() && t.is_contiguous()) {
        p = t.data_ptr();
        return true;
    }
    PyErr_SetString(PyExc_AssertionError, "device, contiguous tensors only");
    return false;
}

// Reads positional arguments in order; after the first failure (Python error set) everything reads as zero.
class Args {
public:
    Args(PyObject *const *a, Py_ssize_t n, Py_ssize_t want) : a_(a)
    {
        if (n != want) { ok_ = false; PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", want, n); }
    }
    bool ok() const { return ok_; }
    PyObject *object() { return ok_ ? a_[i_++] : nullptr; }
    long long integer() { return integer(object()); }
    int small() { return static_cast<int>(integer()); }
    float real() { return real(object()); }
    void *tensor() { return tensor(object()); }

    // Pointers read by `tensor_into` are also noted in `refs`, by their place in the record that starts at `base`.
    void note(const void *base, std::vector<Ref> *refs) { base_ = static_cast<const char *>(base); refs_ = refs; }
    template <class T> void tensor_into(T *&field)
    {
        PyObject *o = object();
        field = static_cast<T *>(tensor(o));
        if (refs_ && ok_ && o != Py_None) refs_->push_back({static_cast<size_t>(reinterpret_cast<const char *>(&field) - base_), Held(o)});
    }

    long long integer(PyObject *o)
    {
        if (!ok_) return 0;
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) {                // (numpy integers and the like)
            PyErr_Clear();
            PyObject *n = PyNumber_Index(o);
            const long long w = n ? PyLong_AsLongLong(n) : 0;
            Py_XDECREF(n);
            if (PyErr_Occurred()) ok_ = false;
            return w;
        }
        return v;
    }
    // what int(o) gives
    int flag()
    {
        PyObject *o = object();
        if (!ok_ || PyLong_Check(o)) return static_cast<int>(integer(o));
        PyObject *n = PyNumber_Long(o);
        if (!n) ok_ = false;
        const int v = static_cast<int>(integer(n));
        Py_XDECREF(n);
        return v;
    }
    float real(PyObject *o)
    {
        if (!ok_) return 0.0f;
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) ok_ = false;
        return static_cast<float>(v);
    }
    // device pointer of a tensor, null for None
    void *tensor(PyObject *o)
    {
        if (!ok_ || o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) {
            ok_ = false;
            PyErr_SetString(PyExc_TypeError, "a torch tensor is expected");
            return nullptr;
        }
        void *p = nullptr;
        ok_ = device_pointer(THPVariable_Unpack(o), p);
        return p;
    }
    // sizes of a tensor of `n` dimensions
    void sizes(PyObject *o, int n, int64_t *out)
    {
        for (int i = 0; i < n; ++i) out[i] = 0;
        if (!ok_) return;
        if (!THPVariable_Check(o)) {
            ok_ = false;
            PyErr_SetString(PyExc_TypeError, "a torch tensor is expected");
            return;
        }
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.dim() != n) {
            ok_ = false;
            PyErr_Format(PyExc_ValueError, "a tensor of %d dimensions is expected, got %lld", n, static_cast<long long>(t.dim()));
            return;
        }
        for (int i = 0; i < n; ++i) out[i] = t.size(i);
    }
    // a binding.Conv (plain attributes)
    apnn_conv_desc conv()
    {
        static const char *const names[13] = {"N", "H", "W", "Cin", "Cout", "R", "S", "stride", "pad", "p", "q", "encW", "encX"};
        static PyObject *keys[13];
        if (!keys[0])
            for (int i = 0; i < 13; ++i) keys[i] = PyUnicode_InternFromString(names[i]);
        PyObject *d = object();
        int64_t v[13] = {};
        for (int i = 0; i < 13 && ok_; ++i) {
            PyObject *o = PyObject_GetAttr(d, keys[i]);
            if (!o) { ok_ = false; break; }
            v[i] = integer(o);
            Py_DECREF(o);
        }
        apnn_conv_desc c;
        c.N = v[0]; c.H = v[1]; c.W = v[2]; c.Cin = v[3]; c.Cout = v[4];
        c.R = static_cast<int>(v[5]); c.S = static_cast<int>(v[6]);
        c.stride = static_cast<int>(v[7]); c.pad = static_cast<int>(v[8]);
        c.p = static_cast<int>(v[9]); c.q = static_cast<int>(v[10]);
        c.encW = static_cast<apnn_encoding>(v[11]); c.encX = static_cast<apnn_encoding>(v[12]);
        return c;
    }

private:
    PyObject *const *a_;
    Py_ssize_t i_ = 0;
    bool ok_ = true;
    const char *base_ = nullptr;
    std::vector<Ref> *refs_ = nullptr;
};

template <class F> PyObject *call(F &&f)
{
    void *stream = current_stream();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(stream);
    Py_END_ALLOW_THREADS
    return finish(rc);
}

// One layer as apnn_layer takes it: descriptor, weights, features, packed output.
struct Layer {
    apnn_layer_desc L;
    const uint32_t *W, *X;
    uint32_t *out;
};

// (d, W, X, is_gemm, q_out, scale, bias, residual, q_res, res_scale, acc_out, float_out, out, pool)
constexpr Py_ssize_t kLayerArgs = 14;
void read_layer(Args &a, Layer &y)
{
    y.L.conv = a.conv();
    a.tensor_into(y.W);
    a.tensor_into(y.X);
    y.L.is_gemm = a.flag();
    y.L.q_out = a.small();
    a.tensor_into(y.L.scale_dev);
    a.tensor_into(y.L.bias_dev);
    a.tensor_into(y.L.residual_dev);
    y.L.q_res = a.small();
    y.L.res_scale = a.real();
    a.tensor_into(y.L.acc_out_dev);
    a.tensor_into(y.L.float_out_dev);
    if (y.L.q_out > 0) a.tensor_into(y.out);
    else a.object();                                      // (there is no packed output: whatever is given is not looked at)
    y.L.pool = a.small();
}

PyObject *py_set_error(PyObject *, PyObject *cls)
{
    Py_INCREF(cls);
    Py_XDECREF(g_error);
    g_error = cls;
    Py_RETURN_NONE;
}

PyObject *py_pack(PyObject *, PyObject *const *args, Py_ssize_t n)      // (src, bits, enc, out)
{
    Args a(args, n, 4);
    int64_t s[2];
    PyObject *src = a.object();
    a.sizes(src, 2, s);
    const void *p = a.tensor(src);
    const int bits = a.small(), enc = a.small();
    auto *out = static_cast<uint32_t *>(a.tensor());
    if (!a.ok()) return nullptr;
    return call([&](void *st) { return apnn_pack(p, s[0], s[1], bits, static_cast<apnn_encoding>(enc), out, st); });
}

PyObject *py_pack_fmap(PyObject *, PyObject *const *args, Py_ssize_t n) // (src, layout, bits, enc, out)
{
    Args a(args, n, 5);
    int64_t s[4];
    PyObject *src = a.object();
    a.sizes(src, 4, s);
    const void *p = a.tensor(src);
    const int layout = a.small(), bits = a.small(), enc = a.small();
    auto *out = static_cast<uint32_t *>(a.tensor());
    if (!a.ok()) return nullptr;
    const bool nhwc = layout == APNN_LAYOUT_NHWC;
    return call([&](void *st) {
        return apnn_pack_fmap(p, static_cast<apnn_layout>(layout), s[0], nhwc ? s[1] : s[2], nhwc ? s[2] : s[3], nhwc ? s[3] : s[1],
                              bits, static_cast<apnn_encoding>(enc), out, st);
    });
}

PyObject *py_quantize(PyObject *, PyObject *const *args, Py_ssize_t n)  // (src, zero, step, bits, out)
{
    Args a(args, n, 5);
    int64_t s[2];
    PyObject *src = a.object();
    a.sizes(src, 2, s);
    const auto *p = static_cast<const float *>(a.tensor(src));
    const float zero = a.real(), step = a.real();
    const int bits = a.small();
    auto *out = static_cast<uint32_t *>(a.tensor());
    if (!a.ok()) return nullptr;
    return call([&](void *st) { return apnn_quantize(p, s[0], s[1], zero, step, bits, out, st); });
}

PyObject *py_gemm(PyObject *, PyObject *const *args, Py_ssize_t n)      // (W, X, M, N, K, p, q, encW, encX, out)
{
    Args a(args, n, 10);
    const auto *W = static_cast<const uint32_t *>(a.tensor());
    const auto *X = static_cast<const uint32_t *>(a.tensor());
    const int64_t M = a.integer(), N = a.integer(), K = a.integer();
    const int p = a.small(), q = a.small(), encW = a.small(), encX = a.small();
    PyObject *result = a.object();                        // (one without elements is not written, wherever it is)
    const bool empty = result && THPVariable_Check(result) && THPVariable_Unpack(result).numel() == 0;
    auto *out = empty ? nullptr : static_cast<int32_t *>(a.tensor(result));
    if (!a.ok()) return nullptr;
    return call([&](void *st) {
        return apnn_gemm(W, X, out, M, N, K, p, q, static_cast<apnn_encoding>(encW), static_cast<apnn_encoding>(encX), st);
    });
}

PyObject *py_conv2d(PyObject *, PyObject *const *args, Py_ssize_t n)    // (d, W, X, out)
{
    Args a(args, n, 4);
    const apnn_conv_desc d = a.conv();
    const auto *W = static_cast<const uint32_t *>(a.tensor());
    const auto *X = static_cast<const uint32_t *>(a.tensor());
    auto *out = static_cast<int32_t *>(a.tensor());
    if (!a.ok()) return nullptr;
    return call([&](void *st) { return apnn_conv2d(&d, W, X, out, st); });
}

PyObject *py_layer(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a(args, n, kLayerArgs);
    Layer y{};
    read_layer(a, y);
    if (!a.ok()) return nullptr;
    return call([&](void *st) { return apnn_layer(&y.L, y.W, y.X, y.out, st); });
}

PyObject *py_layer_pair(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a(args, n, 2 * kLayerArgs);
    Layer x{}, y{};
    read_layer(a, x);
    read_layer(a, y);
    if (!a.ok()) return nullptr;
    return call([&](void *st) { return apnn_layer_pair(&x.L, x.W, x.X, x.out, &y.L, y.W, y.X, y.out, st); });
}

PyObject *py_input_layer(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Args a(args, n, kLayerArgs);
    Layer y{};
    read_layer(a, y);
    if (!a.ok()) return nullptr;
    return call([&](void *st) { return apnn_input_layer(&y.L, y.W, reinterpret_cast<const uint8_t *>(y.X), y.out, st); });
}

PyObject *py_maxpool(PyObject *, PyObject *const *args, Py_ssize_t n)   // (X, N, H, W, C, bits, k, stride, pad, out)
{
    Args a(args, n, 10);
    const auto *X = static_cast<const uint32_t *>(a.tensor());
    const int64_t N = a.integer(), H = a.integer(), W = a.integer(), C = a.integer();
    const int bits = a.small(), k = a.small(), stride = a.small(), pad = a.small();
    auto *out = static_cast<uint32_t *>(a.tensor());
    if (!a.ok()) return nullptr;
    return call([&](void *st) { return apnn_maxpool(X, N, H, W, C, bits, k, stride, pad, out, st); });
}

PyObject *py_sumpool(PyObject *, PyObject *const *args, Py_ssize_t n)   // (X, N, H, W, C, bits, out_bits, out)
{
    Args a(args, n, 8);
    const auto *X = static_cast<const uint32_t *>(a.tensor());
    const int64_t N = a.integer(), H = a.integer(), W = a.integer(), C = a.integer();
    const int bits = a.small(), out_bits = a.small();
    auto *out = static_cast<uint32_t *>(a.tensor());
    if (!a.ok()) return nullptr;
    return call([&](void *st) { return apnn_sumpool(X, N, H, W, C, bits, out_bits, out, st); });
}

PyObject *py_sumpool_fc(PyObject *, PyObject *const *args, Py_ssize_t n)    // (X, N, H, W, C, bits, Wt, Cout, p, encW, out)
{
    Args a(args, n, 11);
    const auto *X = static_cast<const uint32_t *>(a.tensor());
    const int64_t N = a.integer(), H = a.integer(), W = a.integer(), C = a.integer();
    const int bits = a.small();
    const auto *Wt = static_cast<const uint32_t *>(a.tensor());
    const int64_t Cout = a.integer();
    const int p = a.small(), encW = a.small();
    auto *out = static_cast<int32_t *>(a.tensor());
    if (!a.ok()) return nullptr;
    return call([&](void *st) { return apnn_sumpool_fc(X, N, H, W, C, bits, Wt, Cout, p, static_cast<apnn_encoding>(encW), out, st); });
}

// ---- operators on typed tensors (8-bit products with scales, the 4-bit cache): their sizes, types and strides are the tensors'
// own, so they are checked here; what the library checks itself is left to it.  All tensors of a call lie on one device, whose
// current stream is used whichever device is current.  There is no backward pass: what autograd would have to follow is refused, and what
// a call writes into counts as changed, so that a backward pass that needs its old values fails.

class Tensors {
public:
    Tensors(PyObject *const *a, Py_ssize_t n, Py_ssize_t want) : a_(a)
    {
        if (n != want) fail(PyExc_TypeError, "%zd arguments expected, got %zd", want, n);
    }
    bool ok() const { return ok_; }
    PyObject *object() { return a_[i_++]; }

    // The next argument as a device tensor of `dim` dimensions (any number: -1) whose last one is contiguous; null for None where that may be.
    const at::Tensor *strided(const char *name, int dim, bool optional = false)
    {
        if (!ok_) return nullptr;
        PyObject *o = object();
        if (optional && o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) return fail(PyExc_TypeError, "%s: a torch tensor is expected", name);
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda()) return fail(PyExc_AssertionError, "%s: a device tensor is expected", name);
        if (t.requires_grad() && at::GradMode::is_enabled())
            return fail(PyExc_RuntimeError, "%s: requires a gradient, and there is no backward pass (detach it, or call under torch.no_grad())", name);
        if (dim >= 0 && t.dim() != dim) return fail(PyExc_ValueError, "%s: %d dimensions are expected, got %lld", name, dim, static_cast<long long>(t.dim()));
        if (t.dim() && t.size(-1) > 1 && t.stride(-1) != 1) return fail(PyExc_AssertionError, "%s: the last dimension has to be contiguous", name);
        for (int64_t s : t.strides())
            if (s < 0) return fail(PyExc_ValueError, "%s: negative stride", name);
        if (!have_device_) { device_ = t.device(); have_device_ = true; }
        if (t.device() != device_) return fail(PyExc_ValueError, "%s: on another device than the call's other tensors", name);
        return &t;
    }
    // The same, contiguous as a whole and of type `type`.
    const at::Tensor *dense(const char *name, int dim, at::ScalarType type, bool optional = false)
    {
        const at::Tensor *t = strided(name, dim, optional);
        if (!t) return nullptr;
        if (t->scalar_type() != type) return fail(PyExc_TypeError, "%s: type %s is expected, got %s", name, c10::toString(type), c10::toString(t->scalar_type()));
        if (!t->is_contiguous()) return fail(PyExc_AssertionError, "%s: a contiguous tensor is expected", name);
        return t;
    }
    // fp32, fp16 or bf16
    apnn_dtype type(const char *name, const at::Tensor *t)
    {
        if (!ok_ || !t) return APNN_F32;
        switch (t->scalar_type()) {
            case at::kFloat: return APNN_F32;
            case at::kHalf: return APNN_F16;
            case at::kBFloat16: return APNN_BF16;
            default: fail(PyExc_TypeError, "%s: float32, float16 or bfloat16 is expected, got %s", name, c10::toString(t->scalar_type())); return APNN_F32;
        }
    }
    void same_type(const char *name, const at::Tensor *t, const at::Tensor *as)
    {
        if (ok_ && t && as && t->scalar_type() != as->scalar_type())
            fail(PyExc_TypeError, "%s: type %s is expected, got %s", name, c10::toString(as->scalar_type()), c10::toString(t->scalar_type()));
    }
    void sizes(const char *name, const at::Tensor *t, at::IntArrayRef want)
    {
        if (!ok_ || !t) return;
        if (t->sizes() == want) return;
        char is[64], be[64];
        text(is, sizeof is, t->sizes());
        text(be, sizeof be, want);
        fail(PyExc_ValueError, "%s: size (%s) is expected, got (%s)", name, be, is);
    }
    long long integer()
    {
        if (!ok_) return 0;
        PyObject *n = PyNumber_Index(object());
        const long long v = n ? PyLong_AsLongLong(n) : 0;
        Py_XDECREF(n);
        if (PyErr_Occurred()) ok_ = false;
        return v;
    }
    float real()
    {
        if (!ok_) return 0.0f;
        const double v = PyFloat_AsDouble(object());
        if (v == -1.0 && PyErr_Occurred()) ok_ = false;
        return static_cast<float>(v);
    }
    template <class... A> std::nullptr_t fail(PyObject *error, const char *format, A... a)
    {
        if (ok_) PyErr_Format(error, format, a...);
        ok_ = false;
        return nullptr;
    }
    at::Device device() const { return device_; }

    // A result: the next argument, or where it is None a new tensor, contiguous, of these sizes and type.
    at::Tensor result(const char *name, at::IntArrayRef want, at::ScalarType type, bool dense)
    {
        if (!ok_) return {};
        if (a_[i_] == Py_None) {
            ++i_;
            return at::empty(want, at::TensorOptions().dtype(type).device(device_));
        }
        const at::Tensor *t = strided(name, static_cast<int>(want.size()));
        if (!t) return {};
        if (t->scalar_type() != type) fail(PyExc_TypeError, "%s: type %s is expected, got %s", name, c10::toString(type), c10::toString(t->scalar_type()));
        if (ok_ && dense && !t->is_contiguous()) fail(PyExc_AssertionError, "%s: a contiguous tensor is expected", name);
        sizes(name, t, want);
        if (ok_) writes(t);
        return *t;
    }
    // The call writes into this tensor of the caller's.
    void writes(const at::Tensor *t)
    {
        if (!t->is_inference()) written_.push_back(t->unsafeGetTensorImpl());
    }
    // Whether the next argument is None; it is passed over if so.
    bool none()
    {
        if (!ok_ || a_[i_] != Py_None) return false;
        ++i_;
        return true;
    }

    // Calls the library on the tensors' device: f(stream).
    template <class F> PyObject *call(F &&f)
    {
        const c10::DeviceGuard guard(device_);
        void *stream = static_cast<void *>(c10::hip::getCurrentHIPStream(device_.index()).stream());
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = f(stream);
        Py_END_ALLOW_THREADS
        if (rc == APNN_OK)
            for (c10::TensorImpl *t : written_) t->bump_version();
        return finish(rc);
    }

private:
    static void text(char *to, size_t room, at::IntArrayRef v)
    {
        size_t at = 0;
        to[0] = 0;
        for (size_t i = 0; i < v.size() && at < room; ++i) at += static_cast<size_t>(snprintf(to + at, room - at, i ? ", %lld" : "%lld", static_cast<long long>(v[i])));
    }

    PyObject *const *a_;
    Py_ssize_t i_ = 0;
    bool ok_ = true, have_device_ = false;
    at::Device device_ = at::Device(at::kCUDA, 0);
    c10::SmallVector<c10::TensorImpl *, 4> written_;
};

template <class T> T *data(const at::Tensor *t) { return t ? static_cast<T *>(t->data_ptr()) : nullptr; }

// None, or what a call that succeeded returns.
PyObject *returned(PyObject *none, const at::Tensor &t)
{
    if (!none) return nullptr;
    Py_DECREF(none);
    return THPVariable_Wrap(t);
}
PyObject *returned(PyObject *none, const at::Tensor &t, const at::Tensor &u)
{
    if (!none) return nullptr;
    Py_DECREF(none);
    PyObject *pair = PyTuple_New(2), *x = THPVariable_Wrap(t), *y = THPVariable_Wrap(u);
    if (!pair || !x || !y) {
        Py_XDECREF(pair);
        Py_XDECREF(x);
        Py_XDECREF(y);
        return nullptr;
    }
    PyTuple_SET_ITEM(pair, 0, x);
    PyTuple_SET_ITEM(pair, 1, y);
    return pair;
}

PyObject *py_quantize_tokens(PyObject *, PyObject *const *args, Py_ssize_t n)   // (src, codes or None, scale or None) -> (codes, scale)
{
    Tensors a(args, n, 3);
    const at::Tensor *src = a.strided("src", 2);
    const apnn_dtype type = a.type("src", src);
    if (!a.ok()) return nullptr;
    const int64_t rows = src->size(0), K = src->size(1), ld = rows > 1 ? src->stride(0) : K;
    const at::Tensor codes = a.result("codes", {rows, apnn_token_pitch(K)}, at::kChar, true), scale = a.result("scale", {rows}, at::kFloat, true);
    if (!a.ok()) return nullptr;
    return returned(a.call([&](void *st) { return apnn_quantize_tokens(data<void>(src), type, rows, K, ld, data<int8_t>(&codes), data<float>(&scale), st); }), codes, scale);
}

// (X, x_scale, W, w_scale, K, bias, out or None, dtype of a new result) -> out
PyObject *py_gemm_scaled(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Tensors a(args, n, 8);
    const at::Tensor *X = a.dense("X", 2, at::kChar), *xs = a.dense("x_scale", 1, at::kFloat), *W = a.dense("W", 2, at::kChar), *ws = a.dense("w_scale", 1, at::kFloat);
    const int64_t K = a.integer();
    const at::Tensor *bias = a.dense("bias", 1, at::kFloat, true);
    if (!a.ok()) return nullptr;
    const int64_t M = X->size(0), N = W->size(0), pitch = apnn_token_pitch(K);
    a.sizes("X", X, {M, pitch});
    a.sizes("W", W, {N, pitch});
    a.sizes("x_scale", xs, {M});
    a.sizes("w_scale", ws, {N});
    a.sizes("bias", bias, {N});
    if (!a.ok()) return nullptr;
    at::Tensor out;
    if (a.none()) {
        PyObject *type = a.object();
        if (!THPDtype_Check(type)) a.fail(PyExc_TypeError, "dtype: a torch.dtype is expected");
        else out = at::empty({M, N}, at::TensorOptions().dtype(reinterpret_cast<THPDtype *>(type)->scalar_type).device(a.device()));
    } else if (const at::Tensor *given = a.strided("out", 2)) {
        out = *given;
        a.sizes("out", given, {M, N});
        a.writes(given);
    }
    const apnn_dtype type = a.type("out", &out);
    if (!a.ok()) return nullptr;
    const int64_t ldy = M > 1 ? out.stride(0) : N;
    return returned(a.call([&](void *st) {
        return apnn_gemm_scaled(data<int8_t>(X), data<float>(xs), data<int8_t>(W), data<float>(ws), data<float>(bias), data<void>(&out), type, M, N, K, ldy, st);
    }), out);
}

// A size that the library takes as 32 bits; what does not fit is one that it refuses.
int narrow(int64_t v) { return static_cast<int>(std::clamp<int64_t>(v, INT32_MIN, INT32_MAX)); }

// the four arrays of a binding.KVCache, which the call may write into
apnn_kv_cache read_cache(Tensors &a, bool written = false)
{
    apnn_kv_cache c = {};
    const at::Tensor *kc = a.dense("k_codes", 4, at::kByte), *ks = a.dense("k_scale", 4, at::kByte), *vc = a.dense("v_codes", 4, at::kByte), *vs = a.dense("v_scale", 4, at::kByte);
    if (!a.ok()) return c;
    const int64_t pages = kc->size(0), heads = kc->size(1), page = kc->size(2), D = 2 * kc->size(3);
    a.sizes("k_scale", ks, {pages, heads, page, D / 32});
    a.sizes("v_codes", vc, {pages, heads, page, D / 2});
    a.sizes("v_scale", vs, {pages, heads, page, D / 32});
    if (!a.ok()) return c;
    if (written)
        for (const at::Tensor *t : {kc, ks, vc, vs}) a.writes(t);
    c.k_codes_dev = data<uint8_t>(kc);
    c.k_scale_dev = data<uint8_t>(ks);
    c.v_codes_dev = data<uint8_t>(vc);
    c.v_scale_dev = data<uint8_t>(vs);
    c.pages = pages;
    c.heads = narrow(heads);
    c.page_size = narrow(page);
    c.D = narrow(D);
    return c;
}

// (k_codes, k_scale, v_codes, v_scale, k, v, slots, positions, table, interleaved, q or None, q_out or None) -> q_out, None without q
PyObject *py_kv_append(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Tensors a(args, n, 12);
    const apnn_kv_cache c = read_cache(a, true);
    const at::Tensor *k = a.strided("k", 3), *v = a.strided("v", 3), *slots = a.dense("slots", 1, at::kLong);
    const at::Tensor *positions = a.dense("positions", 1, at::kInt, true), *table = a.dense("table", 2, at::kFloat, true);
    const long long interleaved = a.integer();
    const at::Tensor *q = a.strided("q", 3, true);
    apnn_kv_tokens t = {};
    t.type = a.type("k", k);
    a.same_type("v", v, k);
    a.same_type("q", q, k);
    if (!a.ok()) return nullptr;
    t.tokens = k->size(0);
    a.sizes("k", k, {t.tokens, c.heads, c.D});
    a.sizes("v", v, {t.tokens, c.heads, c.D});
    a.sizes("slots", slots, {t.tokens});
    a.sizes("positions", positions, {t.tokens});
    if (!table != !positions) a.fail(PyExc_ValueError, "positions go with a table, and a table with positions");
    at::Tensor q_out;
    if (q) {
        a.sizes("q", q, {t.tokens, q->size(1), c.D});
        q_out = a.result("q_out", {t.tokens, q->size(1), c.D}, q->scalar_type(), false);
    } else if (!a.none()) {
        a.fail(PyExc_ValueError, "q_out goes with q");
    }
    if (!a.ok()) return nullptr;
    t.k_dev = data<void>(k);
    t.v_dev = data<void>(v);
    t.k_token_stride = k->stride(0); t.k_head_stride = k->stride(1);
    t.v_token_stride = v->stride(0); t.v_head_stride = v->stride(1);
    t.slot_dev = data<int64_t>(slots);
    if (table) {
        t.rot = narrow(table->size(1));
        t.interleaved = interleaved != 0;
        t.table_dev = data<float>(table);
        t.table_rows = table->size(0);
        t.position_dev = data<int32_t>(positions);
    }
    if (q && q->size(1)) {
        t.q_heads = narrow(q->size(1));
        t.q_dev = data<void>(q);
        t.q_out_dev = data<void>(&q_out);
        t.q_token_stride = q->stride(0); t.q_head_stride = q->stride(1);
        t.q_out_token_stride = q_out.stride(0); t.q_out_head_stride = q_out.stride(1);
    }
    PyObject *none = a.call([&](void *st) { return apnn_kv_append(&c, &t, st); });
    return q ? returned(none, q_out) : none;
}

PyObject *py_kv_read(PyObject *, PyObject *const *args, Py_ssize_t n)           // (k_codes, k_scale, v_codes, v_scale, slots, dtype) -> (k, v)
{
    Tensors a(args, n, 6);
    const apnn_kv_cache c = read_cache(a);
    const at::Tensor *slots = a.dense("slots", 1, at::kLong);
    if (!a.ok()) return nullptr;
    PyObject *type = a.object();
    if (!THPDtype_Check(type)) a.fail(PyExc_TypeError, "dtype: a torch.dtype is expected");
    if (!a.ok()) return nullptr;
    const auto options = at::TensorOptions().dtype(reinterpret_cast<THPDtype *>(type)->scalar_type).device(a.device());
    const int64_t count = slots->size(0);
    const at::Tensor k = at::empty({count, c.heads, c.D}, options), v = at::empty({count, c.heads, c.D}, options);
    const apnn_dtype as = a.type("dtype", &k);
    if (!a.ok()) return nullptr;
    return returned(a.call([&](void *st) { return apnn_kv_read(&c, data<int64_t>(slots), count, data<void>(&k), data<void>(&v), as, st); }), k, v);
}

// (k_codes, k_scale, v_codes, v_scale, q, lens, pages, scale, q_start or None, max_q or None, out or None, workspace or None) -> out
PyObject *py_kv_attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Tensors a(args, n, 12);
    const apnn_kv_cache c = read_cache(a);
    const at::Tensor *q = a.strided("q", 3), *lens = a.dense("lens", 1, at::kInt), *pages = a.dense("pages", 2, at::kInt);
    apnn_kv_attention_desc d = {};
    d.scale = a.real();
    const at::Tensor *q_start = a.dense("q_start", 1, at::kInt, true);
    if (!a.ok()) return nullptr;
    d.tokens = q->size(0);
    d.seqs = lens->size(0);
    d.max_pages = pages->size(1);
    d.max_q = a.none() ? (q_start ? d.tokens : 1) : a.integer();
    d.type = a.type("q", q);
    a.sizes("q", q, {d.tokens, q->size(1), c.D});
    a.sizes("pages", pages, {d.seqs, d.max_pages});
    a.sizes("q_start", q_start, {d.seqs + 1});
    const at::Tensor out = a.result("out", {d.tokens, q->size(1), c.D}, q->scalar_type(), false), *workspace = a.dense("workspace", 1, at::kByte, true);
    if (!a.ok()) return nullptr;
    d.q_heads = narrow(q->size(1));
    d.q_dev = data<void>(q);
    d.out_dev = data<void>(&out);
    d.q_token_stride = q->stride(0); d.q_head_stride = q->stride(1);
    d.out_token_stride = out.stride(0); d.out_head_stride = out.stride(1);
    d.q_start_dev = data<int32_t>(q_start);
    d.len_dev = data<int32_t>(lens);
    d.page_dev = data<int32_t>(pages);
    at::Tensor own;                                       // of this call: freed on return, in the stream's order
    void *scratch = data<void>(workspace);
    size_t bytes = workspace ? static_cast<size_t>(workspace->numel()) : 0;
    if (!workspace) {
        bytes = apnn_kv_attention_workspace_bytes(&d, &c);
        if (bytes) {
            own = at::empty({static_cast<int64_t>(bytes)}, at::TensorOptions().dtype(at::kByte).device(a.device()));
            scratch = own.data_ptr();
        }
    }
    return returned(a.call([&](void *st) { return apnn_kv_attention(&d, &c, scratch, bytes, st); }), out);
}

PyObject *py_kv_attention_workspace(PyObject *, PyObject *const *args, Py_ssize_t n)    // (heads, page_size, D, tokens, q_heads, seqs, max_pages, ragged, max_q)
{
    Tensors a(args, n, 9);
    apnn_kv_cache c = {};
    apnn_kv_attention_desc d = {};
    c.heads = narrow(a.integer());
    c.page_size = narrow(a.integer());
    c.D = narrow(a.integer());
    d.tokens = a.integer();
    d.q_heads = narrow(a.integer());
    d.seqs = a.integer();
    d.max_pages = a.integer();
    static const int32_t some = 0;
    d.q_start_dev = a.integer() ? &some : nullptr;        // (whether there is one is all that counts)
    d.max_q = a.integer();
    d.type = APNN_F16;
    if (!a.ok()) return nullptr;
    const size_t bytes = apnn_kv_attention_workspace_bytes(&d, &c);
    if (!bytes && apnn_last_error()[0]) return finish(APNN_ERR_INVALID_ARG);
    return PyLong_FromSize_t(bytes);
}

// ---- Chain: the library calls of a network in order, recorded once (descriptors and the tensors they were given) and
// enqueued by one call.  The tensors are held, and their device pointers are checked and taken anew by every pass, so that
// one whose storage is exchanged is read where it is now, and refused if it now lies on the host or is strided.
struct Step {
    enum Kind { INPUT, LAYER, PAIR, MAXPOOL, SUMPOOL, SUMPOOL_FC } kind;
    Layer a, b;                                           // INPUT, LAYER: a; PAIR: a and b
    // pooling
    const uint32_t *X, *Wt;
    int64_t N, H, W, C, Cout;
    int bits, k, stride, pad, out_bits, p, encW;
    void *out;
};
static_assert(std::is_trivially_copyable<Step>::value, "pointers are written into copies by offset");

struct Record {
    Step step{};
    std::vector<Ref> refs;

    // The step with the pointers of now; false (Python error set) if a tensor has none that can be used.
    bool resolve(Step &s) const
    {
        s = step;
        for (const Ref &r : refs) {
            void *p = nullptr;
            if (!device_pointer(THPVariable_Unpack(r.tensor.get()), p)) return false;
            std::memcpy(reinterpret_cast<char *>(&s) + r.offset, &p, sizeof p);
        }
        return true;
    }
};

struct ChainObject {
    PyObject_HEAD
    std::vector<Record> *records;
};

PyObject *chain_new(PyTypeObject *type, PyObject *, PyObject *)
{
    auto *self = reinterpret_cast<ChainObject *>(type->tp_alloc(type, 0));
    if (self && !(self->records = new (std::nothrow) std::vector<Record>())) {
        Py_DECREF(self);
        return PyErr_NoMemory();
    }
    return reinterpret_cast<PyObject *>(self);
}

void chain_dealloc(PyObject *self)
{
    delete reinterpret_cast<ChainObject *>(self)->records;
    PyTypeObject *type = Py_TYPE(self);
    type->tp_free(self);
    Py_DECREF(type);
}

// Reads one call's arguments with `read` into a new record.
template <class F> PyObject *append(PyObject *self, Args a, Step::Kind kind, F &&read)
{
    Record r;
    r.step.kind = kind;
    a.note(&r.step, &r.refs);
    read(a, r.step);
    if (!a.ok()) return nullptr;
    reinterpret_cast<ChainObject *>(self)->records->push_back(std::move(r));
    Py_RETURN_NONE;
}

PyObject *chain_input_layer(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    return append(self, Args(args, n, kLayerArgs), Step::INPUT, [](Args &a, Step &s) { read_layer(a, s.a); });
}

PyObject *chain_layer(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    return append(self, Args(args, n, kLayerArgs), Step::LAYER, [](Args &a, Step &s) { read_layer(a, s.a); });
}

PyObject *chain_layer_pair(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    return append(self, Args(args, n, 2 * kLayerArgs), Step::PAIR, [](Args &a, Step &s) {
        read_layer(a, s.a);
        read_layer(a, s.b);
    });
}

void read_frame(Args &a, Step &s)
{
    a.tensor_into(s.X);
    s.N = a.integer(); s.H = a.integer(); s.W = a.integer(); s.C = a.integer();
    s.bits = a.small();
}

PyObject *chain_maxpool(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    return append(self, Args(args, n, 10), Step::MAXPOOL, [](Args &a, Step &s) {
        read_frame(a, s);
        s.k = a.small(); s.stride = a.small(); s.pad = a.small();
        a.tensor_into(s.out);
    });
}

PyObject *chain_sumpool(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    return append(self, Args(args, n, 8), Step::SUMPOOL, [](Args &a, Step &s) {
        read_frame(a, s);
        s.out_bits = a.small();
        a.tensor_into(s.out);
    });
}

PyObject *chain_sumpool_fc(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    return append(self, Args(args, n, 11), Step::SUMPOOL_FC, [](Args &a, Step &s) {
        read_frame(a, s);
        a.tensor_into(s.Wt);
        s.Cout = a.integer(); s.p = a.small(); s.encW = a.small();
        a.tensor_into(s.out);
    });
}

int run_step(const Step &s, const void *image, void *stream)
{
    switch (s.kind) {
        case Step::INPUT: return apnn_input_layer(&s.a.L, s.a.W, static_cast<const uint8_t *>(image), s.a.out, stream);
        case Step::LAYER: return apnn_layer(&s.a.L, s.a.W, s.a.X, s.a.out, stream);
        case Step::PAIR: return apnn_layer_pair(&s.a.L, s.a.W, s.a.X, s.a.out, &s.b.L, s.b.W, s.b.X, s.b.out, stream);
        case Step::MAXPOOL:
            return apnn_maxpool(s.X, s.N, s.H, s.W, s.C, s.bits, s.k, s.stride, s.pad, static_cast<uint32_t *>(s.out), stream);
        case Step::SUMPOOL: return apnn_sumpool(s.X, s.N, s.H, s.W, s.C, s.bits, s.out_bits, static_cast<uint32_t *>(s.out), stream);
        case Step::SUMPOOL_FC:
            return apnn_sumpool_fc(s.X, s.N, s.H, s.W, s.C, s.bits, s.Wt, s.Cout, s.p, static_cast<apnn_encoding>(s.encW),
                                   static_cast<int32_t *>(s.out), stream);
    }
    return APNN_ERR_INVALID_ARG;
}

PyObject *chain_run(PyObject *self, PyObject *const *args, Py_ssize_t n)    // (image)
{
    Args a(args, n, 1);
    const void *image = a.tensor();
    if (!a.ok()) return nullptr;
    const auto &records = *reinterpret_cast<ChainObject *>(self)->records;
    std::vector<Step> steps(records.size());              // this pass's own, made while the interpreter lock is held
    for (size_t i = 0; i < records.size(); ++i)
        if (!records[i].resolve(steps[i])) return nullptr;
    return call([&](void *st) {
        for (const Step &s : steps)
            if (const int rc = run_step(s, image, st)) return rc;
        return static_cast<int>(APNN_OK);
    });
}

// What a network is made of, as bytes that stay equal for as long as no entry of any of it is set, exchanged or removed:
// (class of its layers, list of layers, dict of layers, dicts ...).  The interpreter gives a dict a number that no dict has
// had before whenever it is made or modified; a layer counts by the dict of its attributes.  None if it cannot be told:
// containers or layers of another class (what they answer can come from methods), or an interpreter that counts otherwise.
#if PY_VERSION_HEX < 0x030B0000
bool add_version(std::vector<uint64_t> &out, PyObject *dict)
{
    if (!dict || !PyDict_CheckExact(dict)) return false;
    out.push_back(reinterpret_cast<PyDictObject *>(dict)->ma_version_tag);
    return true;
}

bool add_layer_version(std::vector<uint64_t> &out, PyObject *layer, PyObject *cls)
{
    if (reinterpret_cast<PyObject *>(Py_TYPE(layer)) != cls) return false;
    PyObject **dict = _PyObject_GetDictPtr(layer);
    return dict && add_version(out, *dict);
}
#endif

PyObject *py_versions(PyObject *, PyObject *const *args, Py_ssize_t n)
{
#if PY_VERSION_HEX < 0x030B0000
    if (n < 3) { PyErr_SetString(PyExc_TypeError, "a class, a list and at least one dict are expected"); return nullptr; }
    std::vector<uint64_t> tags;
    if (!PyList_CheckExact(args[1]) && !PyTuple_CheckExact(args[1])) Py_RETURN_NONE;
    for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(args[1]); ++i)
        if (!add_layer_version(tags, PySequence_Fast_GET_ITEM(args[1], i), args[0])) Py_RETURN_NONE;
    for (Py_ssize_t i = 2; i < n; ++i)
        if (!add_version(tags, args[i])) Py_RETURN_NONE;
    PyObject *key, *layer;
    for (Py_ssize_t at = 0; PyDict_Next(args[2], &at, &key, &layer);)
        if (!add_layer_version(tags, layer, args[0])) Py_RETURN_NONE;
    return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(tags.data()), static_cast<Py_ssize_t>(tags.size() * sizeof(uint64_t)));
#else
    Py_RETURN_NONE;
#endif
}

Py_ssize_t chain_length(PyObject *self) { return static_cast<Py_ssize_t>(reinterpret_cast<ChainObject *>(self)->records->size()); }

// What torch or the standard library throws (a tensor without storage or sizes, no device, no memory) becomes a Python
// error: no exception leaves a function that the interpreter calls.
using Function = PyObject *(PyObject *, PyObject *const *, Py_ssize_t);
template <Function F> PyObject *guarded(PyObject *self, PyObject *const *args, Py_ssize_t n)
{
    try {
        return F(self, args, n);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define FAST(name, f) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(guarded<f>)), METH_FASTCALL, nullptr}

PyMethodDef chain_methods[] = {
    FAST("input_layer", chain_input_layer), FAST("layer", chain_layer), FAST("layer_pair", chain_layer_pair),
    FAST("maxpool", chain_maxpool), FAST("sumpool", chain_sumpool), FAST("sumpool_fc", chain_sumpool_fc),
    FAST("run", chain_run), {nullptr, nullptr, 0, nullptr}};

PyType_Slot chain_slots[] = {{Py_tp_new, reinterpret_cast<void *>(chain_new)}, {Py_tp_dealloc, reinterpret_cast<void *>(chain_dealloc)},
                             {Py_tp_methods, chain_methods}, {Py_sq_length, reinterpret_cast<void *>(chain_length)}, {0, nullptr}};
PyType_Spec chain_spec = {"paper_2106_12169_amd._native.Chain", sizeof(ChainObject), 0, Py_TPFLAGS_DEFAULT, chain_slots};

PyMethodDef methods[] = {
    {"set_error_class", py_set_error, METH_O, nullptr},
    FAST("pack", py_pack), FAST("pack_fmap", py_pack_fmap), FAST("quantize", py_quantize), FAST("gemm", py_gemm),
    FAST("conv2d", py_conv2d), FAST("layer", py_layer), FAST("layer_pair", py_layer_pair), FAST("input_layer", py_input_layer),
    FAST("maxpool", py_maxpool), FAST("sumpool", py_sumpool), FAST("sumpool_fc", py_sumpool_fc), FAST("versions", py_versions),
    FAST("quantize_tokens", py_quantize_tokens), FAST("gemm_scaled", py_gemm_scaled), FAST("kv_append", py_kv_append), FAST("kv_read", py_kv_read),
    FAST("kv_attention", py_kv_attention), FAST("kv_attention_workspace", py_kv_attention_workspace),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void)
{
    PyObject *m = PyModule_Create(&module_def);
    if (!m) return nullptr;
    PyObject *chain = PyType_FromSpec(&chain_spec);
    if (!chain || PyModule_AddObject(m, "Chain", chain) < 0) {
        Py_XDECREF(chain);
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
