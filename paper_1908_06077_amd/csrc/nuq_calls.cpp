// The library's launching calls from Python without ctypes: tensors are looked at and their addresses gathered in C++, then
// the C entry point of include/nuq.h is called on the current stream.  A step on some ten thousand coordinates is bound by
// this work: 17 to 25 tensors per call, half a microsecond each in Python.  Step on 4 x 65 537 coordinates 38.7 -> 18.9 us,
// decode of as many 15.8 -> 8.0, encode of 8 x 65 537 28.9 -> 11.5.
//
// Every function returns the entry point's code, or None for anything but the plain case: another type of object, a tensor
// of another type, size or placement, a number out of range.  The caller (binding.py) then goes through its own checks,
// which raise what they always raised or accept what they always accepted.  Nothing is launched before that is decided.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/TensorSubclassLikeUtils.h>
#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <vector>

#include "../../include/nuq.h"

namespace {

constexpr uint64_t kMax = 32;       // workers per call (NUQ_MAX_WORKERS)

PyObject *g_get_device, *g_raw_stream;                              // torch._C._cuda_getDevice, _cuda_getCurrentRawStream
PyObject *g_norms, *g_bit_off, *g_words, *g_sync;                   // attribute names

// libnuq.so's entry points, in the order of `bind`'s argument.
#define NUQ_CALLS(X)                                                                                                  \
    X(nuq_num_buckets) X(nuq_num_sync) X(nuq_huffman_num_sync) X(nuq_fixed_words) X(nuq_quantize_encode_batch)       \
    X(nuq_decode_accumulate) X(nuq_decode_momentum_step) X(nuq_quantize_encode_table_batch)                          \
    X(nuq_decode_accumulate_table) X(nuq_quantize_pack_fixed_batch) X(nuq_unpack_accumulate_fixed)                   \
    X(nuq_quantize_pack_fixed_table_batch) X(nuq_unpack_accumulate_fixed_table)                                      \
    X(nuq_quantize_encode_huffman_batch) X(nuq_decode_accumulate_huffman) X(nuq_moments_accumulate)                  \
    X(nuq_gradient_norm) X(nuq_adamw_step) X(nuq_adamw_step_coded) X(nuq_state_blocks) X(nuq_layer_norm_forward)     \
    X(nuq_layer_norm_backward) X(nuq_adamw_state_values)
#define NUQ_POINTER(name) decltype(&::name) p_##name = nullptr;
NUQ_CALLS(NUQ_POINTER)

struct NotPlain {};       // thrown by what follows; becomes None

void need(bool ok)
{
    if (!ok)
        throw NotPlain{};
}

uint64_t whole(PyObject *o, uint64_t top)
{
    need(PyLong_CheckExact(o));
    const unsigned long long x = PyLong_AsUnsignedLongLong(o);
    need(!PyErr_Occurred() && x <= top);
    return x;
}
uint32_t u32(PyObject *o) { return (uint32_t)whole(o, UINT32_MAX); }

double real(PyObject *o)
{
    need(PyFloat_CheckExact(o) || PyLong_CheckExact(o));
    const double x = PyFloat_AsDouble(o);
    need(!PyErr_Occurred());
    return x;
}

int truth(PyObject *o)
{
    need(PyBool_Check(o));
    return o == Py_True ? 1 : 0;
}

// A list or tuple of at most kMax things (its items are borrowed).
struct Items {
    PyObject *seq;
    uint64_t n;
    explicit Items(PyObject *o, uint64_t least = 1, uint64_t most = kMax) : seq(o)
    {
        need(PyList_CheckExact(o) || PyTuple_CheckExact(o));
        n = (uint64_t)PySequence_Fast_GET_SIZE(o);
        need(n >= least && n <= most);
    }
    PyObject *operator[](uint64_t i) const { return PySequence_Fast_GET_ITEM(seq, (Py_ssize_t)i); }
};

const at::Tensor &device_tensor(PyObject *o)
{
    need(THPVariable_CheckExact(o));
    const at::Tensor &t = THPVariable_Unpack(o);
    need(t.is_cuda() && t.layout() == at::kStrided && t.is_contiguous() && t.has_storage() && !at::isTensorSubclassLike(t));
    return t;
}

template <class T>
T *address(PyObject *o, at::ScalarType type, uint64_t least = 0, uint64_t *numel = nullptr)
{
    const at::Tensor &t = device_tensor(o);
    need(t.scalar_type() == type && (uint64_t)t.numel() >= least);
    if (numel)
        *numel = (uint64_t)t.numel();
    return static_cast<T *>(t.data_ptr());
}
template <class T>
T *exactly(PyObject *o, at::ScalarType type, uint64_t n)
{
    uint64_t have;
    T *p = address<T>(o, type, 0, &have);
    need(have == n);
    return p;
}

struct Bytes {
    void *p;
    uint64_t n;
    explicit Bytes(PyObject *o)
    {
        const at::Tensor &t = device_tensor(o);
        p = t.data_ptr();
        n = (uint64_t)t.numel() * t.element_size();
    }
};

template <class T>
using Array = std::array<T, kMax>;

// K gradients of one length.
struct Gradients {
    Array<const float *> v;
    uint64_t K, d;
    explicit Gradients(PyObject *o)
    {
        const Items items(o);
        K = items.n;
        for (uint64_t k = 0; k < K; ++k) {
            uint64_t n;
            v[k] = address<const float>(items[k], at::kFloat, 0, &n);
            need(k == 0 || n == d);
            d = n;
        }
    }
};

struct Seeds {
    Array<uint64_t> x;
    Seeds(PyObject *o, uint64_t K)
    {
        const Items items(o);
        need(items.n == K);
        for (uint64_t k = 0; k < K; ++k) {
            need(PyLong_CheckExact(items[k]));
            x[k] = PyLong_AsUnsignedLongLongMask(items[k]);       // modulo 2^64
        }
    }
};

template <class T>
struct Tensors {
    Array<T *> p;
    Tensors(PyObject *o, uint64_t K, at::ScalarType type, uint64_t least)
    {
        const Items items(o);
        need(items.n == K);
        for (uint64_t k = 0; k < K; ++k)
            p[k] = address<T>(items[k], type, least);
    }
};

// K messages.  sized: every array is looked at for the size that d, bucket and the stride imply.
struct Messages {
    Array<float *> norms;
    Array<uint64_t *> bit_off;
    Array<uint32_t *> words, sync;
    Array<uint64_t> len;
    uint64_t K;
    Messages(PyObject *o, uint64_t d, uint32_t bucket, uint32_t stride, bool huffman = false, bool sized = true)
    {
        const Items items(o);
        K = items.n;
        need(bucket > 0);
        const uint64_t B = p_nuq_num_buckets(d, bucket);
        const uint64_t nsync = B * (huffman ? p_nuq_huffman_num_sync : p_nuq_num_sync)(bucket, stride);
        for (uint64_t k = 0; k < K; ++k) {
            norms[k] = field<float>(items[k], g_norms, at::kFloat, sized ? B : 0, nullptr);
            bit_off[k] = field<uint64_t>(items[k], g_bit_off, at::kLong, sized ? B + 1 : 0, nullptr);
            words[k] = field<uint32_t>(items[k], g_words, at::kInt, 0, &len[k]);
            sync[k] = field<uint32_t>(items[k], g_sync, at::kInt, sized ? nsync : 0, nullptr);
        }
    }
    template <class T>
    static T *field(PyObject *m, PyObject *name, at::ScalarType type, uint64_t least, uint64_t *numel)
    {
        PyObject *o = PyObject_GetAttr(m, name);
        need(o != nullptr);
        struct Release {
            PyObject *o;
            ~Release() { Py_DECREF(o); }               // (the message holds the tensor)
        } release{o};
        if (o == Py_None && !least && !numel)
            return nullptr;
        return address<T>(o, type, least, numel);
    }
};

struct Levels {
    std::array<float, 16> x;
    uint32_t s;
    explicit Levels(PyObject *o)
    {
        const Items items(o, 3, 16);
        s = (uint32_t)items.n - 2u;
        for (uint64_t j = 0; j < items.n; ++j)
            x[j] = (float)real(items[j]);
    }
};

struct Lengths {
    std::array<uint8_t, 16> x;
    Lengths(PyObject *o, uint32_t s)
    {
        const Items items(o, 3, 16);
        need(items.n == (uint64_t)s + 2u);
        for (uint64_t j = 0; j < items.n; ++j)
            x[j] = (uint8_t)whole(items[j], 255);
    }
};

// The current stream of the current device, as torch.cuda.current_stream().
nuq_stream_t stream()
{
    PyObject *dev = PyObject_CallNoArgs(g_get_device);
    need(dev != nullptr);
    PyObject *raw = PyObject_CallOneArg(g_raw_stream, dev);
    Py_DECREF(dev);
    need(raw != nullptr);
    void *p = PyLong_AsVoidPtr(raw);
    Py_DECREF(raw);
    need(!PyErr_Occurred());
    return p;
}

template <class F, class... A>
PyObject *launch(F f, A... args)
{
    const nuq_stream_t st = stream();
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = f(args..., st);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(code);
}

// A METH_FASTCALL function of n arguments from a body that takes them.
template <Py_ssize_t n, PyObject *(*body)(PyObject *const *)>
PyObject *entry(PyObject *, PyObject *const *a, Py_ssize_t got)
{
    try {
        need(got == n);
        return body(a);
    } catch (...) {                     // NotPlain, or what a tensor's method throws
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject *quantize_encode_batch(PyObject *const *a)      // vs, bucket, s, seeds, stride, messages, workspace
{
    const Gradients g(a[0]);
    const uint32_t bucket = u32(a[1]), s = u32(a[2]), stride = u32(a[4]);
    const Seeds seeds(a[3], g.K);
    const Messages m(a[5], g.d, bucket, stride);
    need(m.K == g.K);
    const Bytes ws(a[6]);
    return launch(p_nuq_quantize_encode_batch, (uint32_t)g.K, g.v.data(), seeds.x.data(), g.d, bucket, s, stride, m.norms.data(),
                  m.bit_off.data(), m.words.data(), m.len.data(), m.sync.data(), ws.p, ws.n);
}

PyObject *decode_accumulate(PyObject *const *a)          // messages, d, bucket, s, stride, scale, accumulate, out
{
    const uint64_t d = whole(a[1], UINT64_MAX);
    const uint32_t bucket = u32(a[2]), s = u32(a[3]), stride = u32(a[4]);
    const Messages m(a[0], d, bucket, stride);
    float *out = exactly<float>(a[7], at::kFloat, d);
    return launch(p_nuq_decode_accumulate, (uint32_t)m.K, m.norms.data(), m.bit_off.data(), m.words.data(), m.len.data(),
                  m.sync.data(), d, bucket, s, stride, (float)real(a[5]), truth(a[6]), out);
}

PyObject *decode_momentum_step(PyObject *const *a)       // messages, d, bucket, s, stride, scale, alpha, mu, l, w, yl
{
    const uint64_t d = whole(a[1], UINT64_MAX);
    const uint32_t bucket = u32(a[2]), s = u32(a[3]), stride = u32(a[4]);
    const Messages m(a[0], d, bucket, stride);
    float *w = exactly<float>(a[9], at::kFloat, d), *yl = exactly<float>(a[10], at::kFloat, d);
    return launch(p_nuq_decode_momentum_step, (uint32_t)m.K, m.norms.data(), m.bit_off.data(), m.words.data(), m.len.data(),
                  m.sync.data(), d, bucket, s, stride, (float)real(a[5]), (float)real(a[6]), (float)real(a[7]),
                  (float)real(a[8]), w, yl);
}

PyObject *quantize_encode_table_batch(PyObject *const *a)    // vs, bucket, levels, norm_kind, seeds, stride, messages, workspace
{
    const Gradients g(a[0]);
    const uint32_t bucket = u32(a[1]), kind = u32(a[3]), stride = u32(a[5]);
    const Levels lev(a[2]);
    const Seeds seeds(a[4], g.K);
    const Messages m(a[6], g.d, bucket, stride);
    need(m.K == g.K);
    const Bytes ws(a[7]);
    return launch(p_nuq_quantize_encode_table_batch, (uint32_t)g.K, g.v.data(), seeds.x.data(), g.d, bucket, lev.s, lev.x.data(),
                  kind, stride, m.norms.data(), m.bit_off.data(), m.words.data(), m.len.data(), m.sync.data(), ws.p, ws.n);
}

PyObject *decode_accumulate_table(PyObject *const *a)    // messages, d, bucket, levels, stride, scale, accumulate, out
{
    const uint64_t d = whole(a[1], UINT64_MAX);
    const uint32_t bucket = u32(a[2]), stride = u32(a[4]);
    const Levels lev(a[3]);
    const Messages m(a[0], d, bucket, stride);
    float *out = exactly<float>(a[7], at::kFloat, d);
    return launch(p_nuq_decode_accumulate_table, (uint32_t)m.K, m.norms.data(), m.bit_off.data(), m.words.data(), m.len.data(),
                  m.sync.data(), d, bucket, lev.s, stride, lev.x.data(), (float)real(a[5]), truth(a[6]), out);
}

PyObject *quantize_pack_fixed_batch(PyObject *const *a)  // vs, bucket, s, b, seeds, norms, packed
{
    const Gradients g(a[0]);
    const uint32_t bucket = u32(a[1]), s = u32(a[2]), b = u32(a[3]);
    const Seeds seeds(a[4], g.K);
    const Tensors<float> norms(a[5], g.K, at::kFloat, 0);
    const Tensors<uint32_t> packed(a[6], g.K, at::kInt, 0);
    return launch(p_nuq_quantize_pack_fixed_batch, (uint32_t)g.K, g.v.data(), seeds.x.data(), g.d, bucket, s, b, norms.p.data(),
                  packed.p.data());
}

PyObject *unpack_accumulate_fixed(PyObject *const *a)    // norms, packed, d, bucket, s, b, scale, accumulate, out
{
    const uint64_t K = Items(a[0]).n, d = whole(a[2], UINT64_MAX);
    const Tensors<const float> norms(a[0], K, at::kFloat, 0);
    const Tensors<const uint32_t> packed(a[1], K, at::kInt, 0);
    float *out = exactly<float>(a[8], at::kFloat, d);
    return launch(p_nuq_unpack_accumulate_fixed, (uint32_t)K, norms.p.data(), packed.p.data(), d, u32(a[3]), u32(a[4]), u32(a[5]),
                  (float)real(a[6]), truth(a[7]), out);
}

PyObject *quantize_pack_fixed_table_batch(PyObject *const *a)    // vs, bucket, levels, norm_kind, b, seeds, norms, packed
{
    const Gradients g(a[0]);
    const uint32_t bucket = u32(a[1]), kind = u32(a[3]), b = u32(a[4]);
    const Levels lev(a[2]);
    const Seeds seeds(a[5], g.K);
    need(bucket > 0);
    const Tensors<float> norms(a[6], g.K, at::kFloat, p_nuq_num_buckets(g.d, bucket));
    const Tensors<uint32_t> packed(a[7], g.K, at::kInt, p_nuq_fixed_words(g.d, bucket, b));
    return launch(p_nuq_quantize_pack_fixed_table_batch, (uint32_t)g.K, g.v.data(), seeds.x.data(), g.d, bucket, lev.s,
                  lev.x.data(), kind, b, norms.p.data(), packed.p.data());
}

PyObject *unpack_accumulate_fixed_table(PyObject *const *a)      // norms, packed, d, bucket, levels, b, scale, accumulate, out
{
    const uint64_t K = Items(a[0]).n, d = whole(a[2], UINT64_MAX);
    const uint32_t bucket = u32(a[3]), b = u32(a[5]);
    const Levels lev(a[4]);
    need(bucket > 0);
    const Tensors<const float> norms(a[0], K, at::kFloat, p_nuq_num_buckets(d, bucket));
    const Tensors<const uint32_t> packed(a[1], K, at::kInt, p_nuq_fixed_words(d, bucket, b));
    float *out = exactly<float>(a[8], at::kFloat, d);
    return launch(p_nuq_unpack_accumulate_fixed_table, (uint32_t)K, norms.p.data(), packed.p.data(), d, bucket, lev.s,
                  lev.x.data(), b, (float)real(a[6]), truth(a[7]), out);
}

PyObject *quantize_encode_huffman_batch(PyObject *const *a)      // vs, bucket, s, seeds, stride, lengths, messages, workspace
{
    const Gradients g(a[0]);
    const uint32_t bucket = u32(a[1]), s = u32(a[2]), stride = u32(a[4]);
    const Seeds seeds(a[3], g.K);
    const Lengths len(a[5], s);
    const Messages m(a[6], g.d, bucket, stride, true, false);
    need(m.K == g.K);
    const Bytes ws(a[7]);
    return launch(p_nuq_quantize_encode_huffman_batch, (uint32_t)g.K, g.v.data(), seeds.x.data(), g.d, bucket, s, stride,
                  len.x.data(), m.norms.data(), m.bit_off.data(), m.words.data(), m.len.data(), m.sync.data(), ws.p, ws.n);
}

PyObject *decode_accumulate_huffman(PyObject *const *a)  // messages, d, bucket, s, stride, lengths, scale, accumulate, out
{
    const uint64_t d = whole(a[1], UINT64_MAX);
    const uint32_t bucket = u32(a[2]), s = u32(a[3]), stride = u32(a[4]);
    const Lengths len(a[5], s);
    const Messages m(a[0], d, bucket, stride, true);
    float *out = exactly<float>(a[8], at::kFloat, d);
    return launch(p_nuq_decode_accumulate_huffman, (uint32_t)m.K, m.norms.data(), m.bit_off.data(), m.words.data(), m.len.data(),
                  m.sync.data(), d, bucket, s, stride, len.x.data(), (float)real(a[6]), truth(a[7]), out);
}

PyObject *moments_accumulate(PyObject *const *a)         // g, total, total_sq
{
    uint64_t d;
    const float *g = address<const float>(a[0], at::kFloat, 0, &d);
    double *total = exactly<double>(a[1], at::kDouble, d), *total_sq = exactly<double>(a[2], at::kDouble, d);
    return launch(p_nuq_moments_accumulate, g, total, total_sq, d);
}

// ---- the optimizer and the layer norm ----

uint32_t type_of(at::ScalarType t)
{
    need(t == at::kFloat || t == at::kBFloat16 || t == at::kHalf);
    return t == at::kFloat ? NUQ_F32 : t == at::kBFloat16 ? NUQ_BF16 : NUQ_F16;
}

// Device tensors of one type, each as long as `like` says (where it says anything).
struct Many {
    std::vector<void *> p;
    std::vector<uint64_t> n;
    at::ScalarType type = at::kFloat;
    explicit Many(PyObject *o, const std::vector<uint64_t> *like = nullptr)
    {
        const Items items(o, like ? like->size() : 0, like ? like->size() : UINT32_MAX);
        p.resize(items.n);
        n.resize(items.n);
        for (uint64_t i = 0; i < items.n; ++i) {
            const at::Tensor &t = device_tensor(items[i]);
            p[i] = t.data_ptr();
            n[i] = (uint64_t)t.numel();
            need(i == 0 || t.scalar_type() == type);
            type = t.scalar_type();
            need(!like || n[i] == (*like)[i]);
        }
    }
    Many(PyObject *o, const std::vector<uint64_t> *like, at::ScalarType wanted) : Many(o, like) { need(n.empty() || type == wanted); }
    template <class T>
    T *const *as() const
    {
        return reinterpret_cast<T *const *>(p.data());
    }
};

PyObject *gradient_norm(PyObject *const *a)              // grads, max_norm, workspace, out
{
    const Many g(a[0]);
    const Bytes ws(a[2]);
    return launch(p_nuq_gradient_norm, (uint32_t)g.n.size(), g.as<const void>(), g.n.data(), type_of(g.type), (float)real(a[1]), ws.p,
                  ws.n, address<float>(a[3], at::kFloat, 2));
}

// The arguments that both steps share: ws, grads; decays, alpha, beta1, beta2, eps, t, coefficient, copies from `at` on.
struct StepArguments {
    Many w, g;
    std::vector<float> decay;
    std::vector<void *> copy;
    uint32_t g_type, copy_type = NUQ_BF16;
    double alpha, beta1, beta2, eps;
    uint64_t t;
    const float *c = nullptr;
    StepArguments(PyObject *const *a, int at) : w(a[0], nullptr, at::kFloat), g(a[1], &w.n), g_type(type_of(g.type))
    {
        if (a[at] != Py_None) {
            const Items items(a[at], w.n.size(), w.n.size());
            decay.resize(items.n);
            for (uint64_t i = 0; i < items.n; ++i)
                decay[i] = (float)real(items[i]);
        }
        alpha = real(a[at + 1]);
        beta1 = real(a[at + 2]);
        beta2 = real(a[at + 3]);
        eps = real(a[at + 4]);
        t = whole(a[at + 5], UINT64_MAX);
        if (a[at + 6] != Py_None)
            c = address<const float>(a[at + 6], at::kFloat, 1);
        if (a[at + 7] != Py_None && !w.n.empty()) {
            Many m(a[at + 7], &w.n);
            copy_type = type_of(m.type);
            copy.swap(m.p);
        }
    }
    const float *decays() const { return decay.empty() ? nullptr : decay.data(); }
    void *const *copies() const { return copy.empty() ? nullptr : copy.data(); }
};

PyObject *adamw_step(PyObject *const *a)                 // ws, grads, ms, vs, decays, alpha, beta1, beta2, eps, t, coefficient, copies
{
    const StepArguments S(a, 4);
    const Many m(a[2], &S.w.n, at::kFloat), v(a[3], &S.w.n, at::kFloat);
    return launch(p_nuq_adamw_step, (uint32_t)S.w.n.size(), S.w.as<float>(), S.g.as<const void>(), m.as<float>(), v.as<float>(),
                  S.copies(), S.w.n.data(), S.decays(), S.g_type, S.copy_type, S.alpha, S.beta1, S.beta2, S.eps, S.t, S.c);
}

PyObject *adamw_step_coded(PyObject *const *a)           // ws, grads, ms, vs, scales, decays, ... as above
{
    const StepArguments S(a, 5);
    const Many m(a[2], &S.w.n, at::kFloat8_e4m3fn), v(a[3], &S.w.n, at::kByte);
    std::vector<uint64_t> two(S.w.n.size());
    for (size_t i = 0; i < two.size(); ++i)
        two[i] = 2u * p_nuq_state_blocks(S.w.n[i]);
    const Many scales(a[4], &two, at::kFloat);
    return launch(p_nuq_adamw_step_coded, (uint32_t)S.w.n.size(), S.w.as<float>(), S.g.as<const void>(), m.as<uint8_t>(),
                  v.as<uint8_t>(), scales.as<float>(), S.copies(), S.w.n.data(), S.decays(), S.g_type, S.copy_type, S.alpha, S.beta1,
                  S.beta2, S.eps, S.t, S.c);
}

PyObject *adamw_state_values(PyObject *const *a)         // m_codes, v_codes, scales, m, v
{
    uint64_t n;
    const uint8_t *m = address<const uint8_t>(a[0], at::kFloat8_e4m3fn, 0, &n), *v = exactly<const uint8_t>(a[1], at::kByte, n);
    const float *scales = address<const float>(a[2], at::kFloat, 2u * p_nuq_state_blocks(n));
    return launch(p_nuq_adamw_state_values, m, v, scales, n, exactly<float>(a[3], at::kFloat, n), exactly<float>(a[4], at::kFloat, n));
}

// `rows` rows of `hidden` elements of one type, or none (0 rows asked: as many as there are).
struct Rows {
    void *p = nullptr;
    uint64_t ld = 0, rows = 0;
    uint32_t hidden = 0;
    at::ScalarType type = at::kFloat;
    Rows(PyObject *o, const Rows *like)
    {
        if (o == Py_None)
            return;
        need(THPVariable_CheckExact(o));
        const at::Tensor &t = THPVariable_Unpack(o);
        need(t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && !at::isTensorSubclassLike(t) && t.dim() >= 1);
        const int64_t last = t.size(-1);
        need(last >= 1 && last <= INT32_MAX);
        hidden = (uint32_t)last;
        rows = (uint64_t)t.numel() / hidden;
        type = t.scalar_type();
        if (t.dim() == 2) {
            need(hidden == 1 || t.stride(1) == 1);
            ld = (uint64_t)t.stride(0);
        } else {
            need(t.is_contiguous());
            ld = hidden;
        }
        p = t.data_ptr();
        need(!like || (like->rows == rows && like->hidden == hidden && like->type == type));
    }
};

// A contiguous vector of n elements, or none.
struct Vector {
    void *p = nullptr;
    at::ScalarType type = at::kFloat;
    bool there = false;
    Vector(PyObject *o, uint64_t n)
    {
        if (o == Py_None)
            return;
        const at::Tensor &t = device_tensor(o);
        need((uint64_t)t.numel() == n);
        p = t.data_ptr();
        type = t.scalar_type();
        there = true;
    }
    float *floats() const
    {
        need(type == at::kFloat);
        return static_cast<float *>(p);
    }
};

uint32_t weight_type(at::ScalarType rows, std::initializer_list<const Vector *> vectors)
{
    at::ScalarType type = at::kFloat;
    bool any = false;
    for (const Vector *v : vectors)
        if (v->there) {
            need(!any || v->type == type);
            type = v->type;
            any = true;
        }
    need(type == at::kFloat || type == rows);
    return type_of(type);
}

PyObject *layer_norm_forward(PyObject *const *a)         // x, residual, weight, bias, eps, total, y, mean, rstd
{
    const Rows x(a[0], nullptr), residual(a[1], &x), total(a[5], &x), y(a[6], &x);
    need(x.hidden > 0 && y.hidden > 0 && (residual.hidden > 0) == (total.hidden > 0));
    const Vector weight(a[2], x.hidden), bias(a[3], x.hidden), mean(a[7], x.rows), rstd(a[8], x.rows);
    return launch(p_nuq_layer_norm_forward, x.p, x.ld, residual.p, residual.ld, weight.p, bias.p, x.rows, x.hidden,
                  (float)real(a[4]), type_of(x.type), weight_type(x.type, {&weight, &bias}), total.p, total.ld, y.p, y.ld,
                  mean.floats(), rstd.floats());
}

PyObject *layer_norm_backward(PyObject *const *a)        // dy, x, weight, mean, rstd, add, dx, dweight, dbias, workspace
{
    const Rows x(a[1], nullptr), dy(a[0], &x), add(a[5], &x), dx(a[6], &x);
    need(x.hidden > 0 && dy.hidden > 0 && dx.hidden > 0);
    const Vector weight(a[2], x.hidden), mean(a[3], x.rows), rstd(a[4], x.rows), dweight(a[7], x.hidden), dbias(a[8], x.hidden);
    need(mean.there && rstd.there);
    void *ws = nullptr;
    uint64_t bytes = 0;
    if (a[9] != Py_None) {
        const Bytes b(a[9]);
        ws = b.p;
        bytes = b.n;
    }
    return launch(p_nuq_layer_norm_backward, dy.p, dy.ld, x.p, x.ld, weight.p, mean.floats(), rstd.floats(), add.p, add.ld, x.rows,
                  x.hidden, type_of(x.type), weight_type(x.type, {&weight, &dweight, &dbias}), dx.p, dx.ld, dweight.p, dbias.p, ws,
                  bytes);
}

// bind(addresses of the entry points in NUQ_CALLS' order, torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream)
PyObject *bind(PyObject *, PyObject *args)
{
    PyObject *addresses, *get_device, *raw_stream;
    if (!PyArg_ParseTuple(args, "O!OO", &PyTuple_Type, &addresses, &get_device, &raw_stream))
        return nullptr;
    Py_ssize_t i = 0;
#define NUQ_BIND(name)                                                                                                \
    if (i >= PyTuple_GET_SIZE(addresses)) {                                                                           \
        PyErr_SetString(PyExc_ValueError, "an address per entry point");                                              \
        return nullptr;                                                                                               \
    }                                                                                                                 \
    p_##name = reinterpret_cast<decltype(p_##name)>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i++)));              \
    if (PyErr_Occurred())                                                                                             \
        return nullptr;
    NUQ_CALLS(NUQ_BIND)
    Py_INCREF(get_device);
    Py_INCREF(raw_stream);
    g_get_device = get_device;
    g_raw_stream = raw_stream;
    Py_RETURN_NONE;
}

PyObject *names(PyObject *, PyObject *)
{
#define NUQ_NAME(name) "s"
    return Py_BuildValue("(" NUQ_CALLS(NUQ_NAME) ")"
#undef NUQ_NAME
#define NUQ_NAME(name) , #name
                         NUQ_CALLS(NUQ_NAME));
}

#define NUQ_METHOD(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&entry<n, name>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"names", names, METH_NOARGS, nullptr},
    NUQ_METHOD(quantize_encode_batch, 7),
    NUQ_METHOD(decode_accumulate, 8),
    NUQ_METHOD(decode_momentum_step, 11),
    NUQ_METHOD(quantize_encode_table_batch, 8),
    NUQ_METHOD(decode_accumulate_table, 8),
    NUQ_METHOD(quantize_pack_fixed_batch, 7),
    NUQ_METHOD(unpack_accumulate_fixed, 9),
    NUQ_METHOD(quantize_pack_fixed_table_batch, 8),
    NUQ_METHOD(unpack_accumulate_fixed_table, 9),
    NUQ_METHOD(quantize_encode_huffman_batch, 8),
    NUQ_METHOD(decode_accumulate_huffman, 9),
    NUQ_METHOD(moments_accumulate, 3),
    NUQ_METHOD(gradient_norm, 4),
    NUQ_METHOD(adamw_step, 12),
    NUQ_METHOD(adamw_step_coded, 13),
    NUQ_METHOD(adamw_state_values, 5),
    NUQ_METHOD(layer_norm_forward, 9),
    NUQ_METHOD(layer_norm_backward, 10),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_nuq_calls", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__nuq_calls()
{
    g_norms = PyUnicode_InternFromString("norms");
    g_bit_off = PyUnicode_InternFromString("bit_off");
    g_words = PyUnicode_InternFromString("words");
    g_sync = PyUnicode_InternFromString("sync");
    if (!g_norms || !g_bit_off || !g_words || !g_sync)
        return nullptr;
    PyObject *m = PyModule_Create(&g_module);
    if (m && (PyModule_AddObject(m, "header_key", PyLong_FromUnsignedLongLong(NUQ_HEADER_KEY)) ||      // see build.py
              PyModule_AddStringConstant(m, "torch_version", NUQ_TORCH_VERSION)))
        Py_CLEAR(m);
    return m;
}
