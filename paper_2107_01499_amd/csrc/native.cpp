// The host path of an ordinary call: torch tensors in, one C entry point of libbagua_hip.so out, without a Python
// object or a ctypes conversion per argument.
//
// Every function takes exactly the arguments of the function of its name in binding.py, checks what that one checks (device,
// contiguity, dtype, size of every tensor) and launches.  It answers True when it has made the call, raises BaguaError when the
// entry point refused it, and answers False, having done nothing, whenever anything about an argument is out of the ordinary:
// binding.py's general path then decides, and words the error.  A round of short launches is bound by this path: a call
// took 5.2 .. 6.4 us of host time (20 with the forty tensors of a ring of eight, 32 with a ring of sixteen), of which the launch itself
// needs 2.5.
#include <Python.h>

#include <stddef.h>
#include <stdint.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>

#include "bagua_hip.h"

namespace {

#define BAGUA_NATIVE(X)                                                                                                          \
    X(bagua_bucket_flatten_run) X(bagua_bucket_unflatten_run) X(bagua_compress_minmax_u8) X(bagua_sign_compress_ef)             \
    X(bagua_momentum_sign_compress_ef) X(bagua_flatten_compress_minmax_u8) X(bagua_flatten_sign_compress_ef)                    \
    X(bagua_decompress_unflatten) X(bagua_decompress_reduce_recompress) X(bagua_decompress) X(bagua_decentralized_avg)          \
    X(bagua_decentralized_avg_peers) X(bagua_decentralized_avg_peers_lp) X(bagua_lp_encode) X(bagua_lp_apply_mix)               \
    X(bagua_reduce_compress_minmax_u8) X(bagua_reduce_compress_sign_ef) X(bagua_centralized_avg_fp) X(bagua_decompress_sgd_step) \
    X(bagua_decompress_adam_step) X(bagua_compress_topk_ef) X(bagua_decompress_reduce_recompress_topk) X(bagua_decompress_topk) \
    X(bagua_decompress_sgd_step_topk) X(bagua_decompress_adam_step_topk)

// Those of the calls on a plan and of rows of logits; their functions here go by the second part of the name.
#define BAGUA_NATIVE_STEPS(X) X(grad_norm) X(adamw_step) X(balance_stats) X(balance_grad) X(route) X(route_grad) X(distill_loss) X(distill_grad)

// The entry points, as binding.py's library has them: the address of each, so that both paths call one and the same library.
#define X(name) decltype(&name) f_##name = nullptr;
BAGUA_NATIVE(X)
#undef X
#define X(name) decltype(&bagua_##name) f_bagua_##name = nullptr;
BAGUA_NATIVE_STEPS(X)
#undef X
PyObject* g_error = nullptr;        // binding.BaguaError
PyObject* g_raw_stream = nullptr;   // device index -> raw handle of its current stream
PyObject* g_device = nullptr;       // -> index of the current device

enum Kind { kAny, kF32, kU8, kI32, kI16 };
constexpr size_t kLargest = static_cast<size_t>(1) << 48;   // sizes beyond it go the general way; products of them cannot overflow

size_t chunks_of(size_t n, size_t chunk) { return chunk ? (n + chunk - 1) / chunk : 0; }

// Address of a tensor that the call reads or writes `bytes` of; nullptr for None.  False: not an ordinary one.
bool tensor_ptr(PyObject* o, Kind kind, size_t bytes, void** p)
{
    *p = nullptr;
    if (o == Py_None) return true;
    if (!THPVariable_CheckTypeExact(Py_TYPE(o))) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || !t.is_contiguous()) return false;
    const at::ScalarType type = t.scalar_type();
    if (kind != kAny && type != (kind == kF32 ? at::kFloat : kind == kU8 ? at::kByte : kind == kI32 ? at::kInt : at::kShort)) return false;
    if (t.nbytes() < bytes) return false;
    *p = t.data_ptr();
    return true;
}

// The arguments of one call.  ok turns false at the first one that the general path has to look at.
struct Args {
    PyObject* const* a;
    bool ok;
    Args(PyObject* const* args, Py_ssize_t given, Py_ssize_t expected)
        : a(args), ok(given == expected && at::impl::PythonTorchFunctionTLS::stack_len() == 0 && !torch::jit::tracer::isTracing())
    {
    }
    void* ptr(int i, Kind kind, size_t bytes)
    {
        void* p = nullptr;
        ok = ok && tensor_ptr(a[i], kind, bytes, &p);
        return p;
    }
    bool given(int i) const { return a[i] != Py_None; }
    float* f32(int i, size_t elements) { return static_cast<float*>(ptr(i, kF32, elements * sizeof(float))); }
    size_t numel_of(PyObject* o)
    {
        ok = ok && THPVariable_CheckTypeExact(Py_TYPE(o));
        return ok ? static_cast<size_t>(THPVariable_Unpack(o).numel()) : 0;
    }
    size_t numel(int i) { return ok ? numel_of(a[i]) : 0; }
    size_t size(int i)
    {
        if (!ok || !PyLong_CheckExact(a[i])) { ok = false; return 0; }
        const size_t v = PyLong_AsSize_t(a[i]);
        if (PyErr_Occurred()) PyErr_Clear(), ok = false;
        else if (v > kLargest) ok = false;
        return v;
    }
    int small(int i)   // a codec or a mode
    {
        const size_t v = size(i);
        ok = ok && v < 256;
        return static_cast<int>(v);
    }
    double number(int i)
    {
        if (!ok || !(PyFloat_CheckExact(a[i]) || PyLong_CheckExact(a[i]))) { ok = false; return 0.0; }
        const double v = PyFloat_AsDouble(a[i]);
        if (PyErr_Occurred()) PyErr_Clear(), ok = false;
        return v;
    }
    float real(int i) { return static_cast<float>(number(i)); }
    bool flag(int i)
    {
        ok = ok && PyBool_Check(a[i]);
        return a[i] == Py_True;
    }
    // A list of workers' tensors into p; k = how many there have to be, or -1.  The value: how many there are.
    template <typename T>
    int list(int i, Kind kind, size_t bytes, T** p, int k = -1)
    {
        if (!ok || !(PyList_CheckExact(a[i]) || PyTuple_CheckExact(a[i]))) { ok = false; return 0; }
        const Py_ssize_t count = PySequence_Fast_GET_SIZE(a[i]);
        if (count < 1 || count > BAGUA_MAX_WORKERS || (k >= 0 && count != k)) { ok = false; return 0; }
        PyObject** items = PySequence_Fast_ITEMS(a[i]);
        for (Py_ssize_t j = 0; j < count && ok; ++j) {
            void* q = nullptr;
            ok = tensor_ptr(items[j], kind, bytes, &q);
            p[j] = static_cast<T*>(q);
        }
        return static_cast<int>(count);
    }
    size_t numel_of_first(int i)
    {
        if (!ok || !(PyList_CheckExact(a[i]) || PyTuple_CheckExact(a[i])) || PySequence_Fast_GET_SIZE(a[i]) < 1) { ok = false; return 0; }
        return numel_of(PySequence_Fast_GET_ITEM(a[i], 0));
    }
    void indexes(int i, int* p, int k)
    {
        if (!ok || !(PyList_CheckExact(a[i]) || PyTuple_CheckExact(a[i])) || PySequence_Fast_GET_SIZE(a[i]) != k) { ok = false; return; }
        for (int j = 0; j < k && ok; ++j) {
            PyObject* o = PySequence_Fast_GET_ITEM(a[i], j);
            const long v = PyLong_CheckExact(o) ? PyLong_AsLong(o) : -1;
            if (PyErr_Occurred()) PyErr_Clear();
            ok = v >= 0 && v < BAGUA_MAX_WORKERS;
            p[j] = static_cast<int>(v);
        }
    }
    // A list of workers' matrices (2-D, the elements of a row next to each other, all rows equally far apart) of one type: addresses and
    // numbers of rows into p and rows, where those are given what they have to be (known: of the rows).  columns: -1 = of the first one.
    struct Matrices {
        int count = 0;
        at::ScalarType type = at::kFloat;
        int64_t columns = -1, ld = -1;
        size_t stride() const { return static_cast<size_t>(ld < 0 ? columns : ld); }
    };
    Matrices matrices(int i, const void** p, size_t* rows, bool known, int64_t columns, int expected)
    {
        Matrices m;
        m.columns = columns;
        if (!ok || !(PyList_CheckExact(a[i]) || PyTuple_CheckExact(a[i]))) { ok = false; return m; }
        const Py_ssize_t count = PySequence_Fast_GET_SIZE(a[i]);
        if (count < 1 || count > BAGUA_MAX_WORKERS || (expected >= 0 && count != expected)) { ok = false; return m; }
        m.count = static_cast<int>(count);
        PyObject** items = PySequence_Fast_ITEMS(a[i]);
        for (Py_ssize_t j = 0; j < count; ++j) {
            if (!THPVariable_CheckTypeExact(Py_TYPE(items[j]))) { ok = false; return m; }
            const at::Tensor& t = THPVariable_Unpack(items[j]);
            if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() != 2) { ok = false; return m; }
            const int64_t r = t.size(0), c = t.size(1);
            if (j == 0) m.type = t.scalar_type(), m.columns = m.columns < 0 ? c : m.columns;
            if (t.scalar_type() != m.type || c != m.columns || (known && static_cast<size_t>(r) != rows[j]) || (r > 0 && c > 1 && t.stride(1) != 1)) { ok = false; return m; }
            if (r > 1) {
                if (t.stride(0) < c || (m.ld >= 0 && t.stride(0) != m.ld)) { ok = false; return m; }
                m.ld = t.stride(0);
            }
            rows[j] = static_cast<size_t>(r);
            p[j] = r ? t.data_ptr() : nullptr;
        }
        return m;
    }
    // The workers' masks, or nullptr for None.
    const uint8_t* const* masks(int i, const uint8_t** p, const size_t* rows, int count)
    {
        if (!ok || !given(i)) return nullptr;
        if (!(PyList_CheckExact(a[i]) || PyTuple_CheckExact(a[i])) || PySequence_Fast_GET_SIZE(a[i]) != count) { ok = false; return nullptr; }
        PyObject** items = PySequence_Fast_ITEMS(a[i]);
        for (int j = 0; j < count && ok; ++j) {
            void* q = nullptr;
            ok = items[j] != Py_None && tensor_ptr(items[j], kAny, rows[j], &q);
            const at::ScalarType type = ok ? THPVariable_Unpack(items[j]).scalar_type() : at::kByte;
            ok = ok && (type == at::kByte || type == at::kBool);
            p[j] = rows[j] ? static_cast<const uint8_t*>(q) : nullptr;
        }
        return p;
    }
    // A list of workers' contiguous tensors of one type with `per` elements for every row: their type.
    at::ScalarType row_vectors(int i, const void** p, const size_t* rows, int count, size_t per)
    {
        at::ScalarType type = at::kByte;
        if (!ok || !(PyList_CheckExact(a[i]) || PyTuple_CheckExact(a[i])) || PySequence_Fast_GET_SIZE(a[i]) != count) { ok = false; return type; }
        PyObject** items = PySequence_Fast_ITEMS(a[i]);
        for (int j = 0; j < count && ok; ++j) {
            void* q = nullptr;
            ok = items[j] != Py_None && tensor_ptr(items[j], kAny, 0, &q);
            if (!ok) break;
            const at::Tensor& t = THPVariable_Unpack(items[j]);
            if (j == 0) type = t.scalar_type();
            ok = t.scalar_type() == type && static_cast<size_t>(t.numel()) / per >= rows[j];
            p[j] = rows[j] ? q : nullptr;
        }
        return type;
    }
    size_t slots(size_t keep, size_t n, size_t chunk)
    {
        ok = ok && keep <= chunk;   // (or the entry point refuses it)
        return ok ? chunks_of(n, chunk) * keep : 0;
    }
    // Per-codec sizes: bytes of the code stream, and of the per-chunk metadata.
    static size_t code_bytes(int codec, size_t n) { return codec == BAGUA_CODEC_MINMAX_U8 ? n : (n + 31) / 32 * 4; }
    static size_t meta_floats(int codec, size_t n, size_t chunk) { return chunks_of(n, chunk) * (codec == BAGUA_CODEC_MINMAX_U8 ? 2 : 1); }
};

// The raw handle of the stream argument; None is the current stream of the current device.  False: a Python error is set.
bool stream_handle(PyObject* o, void** s)
{
    PyObject* v = nullptr;
    if (o == Py_None) {
        PyObject* device = PyObject_CallNoArgs(g_device);
        if (!device) return false;
        v = PyObject_CallOneArg(g_raw_stream, device);
        Py_DECREF(device);
    } else {
        v = PyObject_GetAttrString(o, "cuda_stream");
    }
    if (!v) return false;
    const unsigned long long h = PyLong_AsUnsignedLongLongMask(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) return false;
    *s = reinterpret_cast<void*>(static_cast<uintptr_t>(h));
    return true;
}

// Marshals with `prepare`, which leaves Args::ok and answers a callable that makes the call on a stream.  Other threads run
// meanwhile, as they do in a call through ctypes.
template <typename F>
PyObject* call(const char* name, PyObject* const* a, Py_ssize_t given, Py_ssize_t expected, const F& prepare)
{
    int status = 0;
    try {
        Args args(a, given, expected);
        if (!args.ok) Py_RETURN_FALSE;
        const auto launch = prepare(args);
        if (!args.ok) Py_RETURN_FALSE;
        void* s = nullptr;
        if (!stream_handle(a[expected - 1], &s)) {
            PyErr_Clear();
            Py_RETURN_FALSE;
        }
        Py_BEGIN_ALLOW_THREADS
        status = launch(s);
        Py_END_ALLOW_THREADS
    } catch (...) {   // a tensor without memory of its own, and the like (nothing has been launched: the entry points do not throw)
        if (PyErr_Occurred()) PyErr_Clear();
        Py_RETURN_FALSE;
    }
    if (status == BAGUA_OK) Py_RETURN_TRUE;
    PyObject* e = PyObject_CallFunction(g_error, "si", name, status);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

template <typename T>
struct Ptrs {
    T* p[BAGUA_MAX_WORKERS];
};
struct Indexes {
    int i[BAGUA_MAX_WORKERS];
};

#define PY(name, expected)                                                              \
    PyObject* py_##name(PyObject*, PyObject* const* a, Py_ssize_t given)                \
    {                                                                                   \
        return call(#name, a, given, expected, [](Args& v) {
#define PY_END \
        });    \
    }

// ------------------------------------------------------------------------------------------ (arguments as in binding.py)
PY(bagua_bucket_flatten_run, 4)   // workspace, T, bucket, stream
    const void* ws = v.ptr(0, kAny, 0);
    const size_t T = v.size(1), n = v.numel(2);
    float* bucket = v.f32(2, 0);
    return [=](void* s) { return f_bagua_bucket_flatten_run(ws, T, bucket, n, s); };
PY_END

PY(bagua_bucket_unflatten_run, 4)   // workspace, T, bucket, stream
    const void* ws = v.ptr(0, kAny, 0);
    const size_t T = v.size(1), n = v.numel(2);
    const float* bucket = v.f32(2, 0);
    return [=](void* s) { return f_bagua_bucket_unflatten_run(ws, T, bucket, n, s); };
PY_END

PY(bagua_compress_minmax_u8, 6)   // x, residual, chunk, codes, minmax, stream
    const size_t n = v.numel(0), chunk = v.size(2);
    const float* x = v.f32(0, 0);
    float* res = v.f32(1, n);
    uint8_t* codes = static_cast<uint8_t*>(v.ptr(3, kU8, n));
    float* mm = v.f32(4, 2 * chunks_of(n, chunk));
    return [=](void* s) { return f_bagua_compress_minmax_u8(x, res, n, chunk, codes, mm, s); };
PY_END

PY(bagua_sign_compress_ef, 6)   // x, residual, chunk, bits, scale, stream
    const size_t n = v.numel(0), chunk = v.size(2);
    const float* x = v.f32(0, 0);
    float* res = v.f32(1, n);
    uint32_t* bits = static_cast<uint32_t*>(v.ptr(3, kI32, v.code_bytes(BAGUA_CODEC_SIGN1, n)));
    float* scale = v.f32(4, chunks_of(n, chunk));
    return [=](void* s) { return f_bagua_sign_compress_ef(x, res, n, chunk, bits, scale, s); };
PY_END

PY(bagua_momentum_sign_compress_ef, 8)   // g, m, beta1, residual, chunk, bits, scale, stream
    const size_t n = v.numel(0), chunk = v.size(4);
    const float* g = v.f32(0, 0);
    const float* m = v.f32(1, n);
    const float beta1 = v.real(2);
    float* res = v.f32(3, n);
    uint32_t* bits = static_cast<uint32_t*>(v.ptr(5, kI32, v.code_bytes(BAGUA_CODEC_SIGN1, n)));
    float* scale = v.f32(6, chunks_of(n, chunk));
    return [=](void* s) { return f_bagua_momentum_sign_compress_ef(g, m, beta1, res, n, chunk, bits, scale, s); };
PY_END

PY(bagua_flatten_compress_minmax_u8, 9)   // workspace, T, residual, n, chunk, codes, minmax, bucket_out, stream
    const void* ws = v.ptr(0, kAny, 0);
    const size_t T = v.size(1), n = v.size(3), chunk = v.size(4);
    float* res = v.f32(2, n);
    uint8_t* codes = static_cast<uint8_t*>(v.ptr(5, kU8, n));
    float* mm = v.f32(6, 2 * chunks_of(n, chunk));
    float* out = v.f32(7, n);
    return [=](void* s) { return f_bagua_flatten_compress_minmax_u8(ws, T, res, n, chunk, codes, mm, out, s); };
PY_END

PY(bagua_flatten_sign_compress_ef, 9)   // workspace, T, residual, n, chunk, bits, scale, bucket_out, stream
    const void* ws = v.ptr(0, kAny, 0);
    const size_t T = v.size(1), n = v.size(3), chunk = v.size(4);
    float* res = v.f32(2, n);
    uint32_t* bits = static_cast<uint32_t*>(v.ptr(5, kI32, v.code_bytes(BAGUA_CODEC_SIGN1, n)));
    float* scale = v.f32(6, chunks_of(n, chunk));
    float* out = v.f32(7, n);
    return [=](void* s) { return f_bagua_flatten_sign_compress_ef(ws, T, res, n, chunk, bits, scale, out, s); };
PY_END

PY(bagua_decompress_unflatten, 8)   // codec, codes, meta, n, chunk, workspace, T, stream
    const int codec = v.small(0);
    const size_t n = v.size(3), chunk = v.size(4), T = v.size(6);
    const void* codes = v.ptr(1, kAny, v.code_bytes(codec, n));
    const float* meta = v.f32(2, v.meta_floats(codec, n, chunk));
    const void* ws = v.ptr(5, kAny, 0);
    return [=](void* s) { return f_bagua_decompress_unflatten(codec, codes, meta, n, chunk, ws, T, s); };
PY_END

PY(bagua_decompress_reduce_recompress, 10)   // codec, codes_in, meta_in, server_residual, n, chunk, codes_out, meta_out, out_fp32, stream
    const int codec = v.small(0);
    const size_t n = v.size(4), chunk = v.size(5);
    const size_t cb = v.code_bytes(codec, n), mf = v.meta_floats(codec, n, chunk);
    Ptrs<const void> ci;
    Ptrs<const float> mi;
    const int k = v.list(1, kAny, cb, ci.p);
    v.list(2, kF32, mf * sizeof(float), mi.p, k);
    float* eps = v.f32(3, n);
    void* co = v.ptr(6, kAny, cb);
    float* mo = v.f32(7, mf);
    float* out = v.f32(8, n);
    return [=](void* s) { return f_bagua_decompress_reduce_recompress(codec, ci.p, mi.p, k, eps, n, chunk, co, mo, out, s); };
PY_END

PY(bagua_decompress, 7)   // codec, codes, meta, n, chunk, out, stream
    const int codec = v.small(0);
    const size_t n = v.size(3), chunk = v.size(4);
    const void* codes = v.ptr(1, kAny, v.code_bytes(codec, n));
    const float* meta = v.f32(2, v.meta_floats(codec, n, chunk));
    float* out = v.f32(5, n);
    return [=](void* s) { return f_bagua_decompress(codec, codes, meta, n, chunk, out, s); };
PY_END

PY(bagua_decentralized_avg, 8)   // mode, x_in, x_out, xhat, codes, minmax, chunk, stream
    const int mode = v.small(0);
    const size_t n = v.numel_of_first(1), chunk = v.size(6), bytes = n * sizeof(float);
    Ptrs<const float> in;
    Ptrs<float> out, hat, mm;
    Ptrs<uint8_t> cd;
    const int k = v.list(1, kF32, bytes, in.p);
    v.list(2, kF32, bytes, out.p, k);
    const bool has_hat = v.given(3), has_codes = v.given(4), has_mm = v.given(5);
    if (has_hat) v.list(3, kF32, bytes, hat.p, k);
    if (has_codes) v.list(4, kU8, n, cd.p, k);
    if (has_mm) v.list(5, kF32, 2 * chunks_of(n, chunk) * sizeof(float), mm.p, k);
    return [=](void* s) {
        return f_bagua_decentralized_avg(mode, in.p, out.p, has_hat ? hat.p : nullptr, has_codes ? cd.p : nullptr, has_mm ? mm.p : nullptr, k, n,
                                         chunk, s);
    };
PY_END

PY(bagua_decentralized_avg_peers, 4)   // x_in, x_out, peer, stream
    const size_t n = v.numel_of_first(0), bytes = n * sizeof(float);
    Ptrs<const float> in;
    Ptrs<float> out;
    Indexes peer{};
    const int k = v.list(0, kF32, bytes, in.p);
    v.list(1, kF32, bytes, out.p, k);
    v.indexes(2, peer.i, k);
    return [=](void* s) { return f_bagua_decentralized_avg_peers(in.p, out.p, peer.i, k, n, s); };
PY_END

PY(bagua_decentralized_avg_peers_lp, 8)   // x_in, x_out, xhat, codes, minmax, peer, chunk, stream
    const size_t n = v.numel_of_first(0), chunk = v.size(6), bytes = n * sizeof(float);
    Ptrs<const float> in;
    Ptrs<float> out, hat, mm;
    Ptrs<uint8_t> cd;
    Indexes peer{};
    const int k = v.list(0, kF32, bytes, in.p);
    v.list(1, kF32, bytes, out.p, k);
    v.list(2, kF32, bytes, hat.p, k);
    v.list(3, kU8, n, cd.p, k);
    v.list(4, kF32, 2 * chunks_of(n, chunk) * sizeof(float), mm.p, k);
    v.indexes(5, peer.i, k);
    return [=](void* s) { return f_bagua_decentralized_avg_peers_lp(in.p, out.p, hat.p, cd.p, mm.p, peer.i, k, n, chunk, s); };
PY_END

PY(bagua_lp_encode, 6)   // x, xhat, chunk, codes, minmax, stream
    const size_t n = v.numel(0), chunk = v.size(2);
    const float* x = v.f32(0, 0);
    float* hat = v.f32(1, n);
    uint8_t* codes = static_cast<uint8_t*>(v.ptr(3, kU8, n));
    float* mm = v.f32(4, 2 * chunks_of(n, chunk));
    return [=](void* s) { return f_bagua_lp_encode(x, hat, n, chunk, codes, mm, s); };
PY_END

PY(bagua_lp_apply_mix, 11)   // x, xhat_own, xhat_left, xhat_right, codes_left, minmax_left, codes_right, minmax_right, chunk, x_out, stream
    const size_t n = v.numel(0), chunk = v.size(8), nm = 2 * chunks_of(n, chunk);
    const float *x = v.f32(0, 0), *own = v.f32(1, n);
    float *left = v.f32(2, n), *right = v.f32(3, n);
    const uint8_t* cl = static_cast<const uint8_t*>(v.ptr(4, kU8, n));
    const float* ml = v.f32(5, nm);
    const uint8_t* cr = static_cast<const uint8_t*>(v.ptr(6, kU8, n));
    const float* mr = v.f32(7, nm);
    float* out = v.f32(9, n);
    return [=](void* s) { return f_bagua_lp_apply_mix(x, own, left, right, cl, ml, cr, mr, n, chunk, out, s); };
PY_END

PY(bagua_reduce_compress_minmax_u8, 6)   // xs, residual, chunk, codes, minmax, stream
    const size_t n = v.numel_of_first(0), chunk = v.size(2);
    Ptrs<const float> xs;
    const int k = v.list(0, kF32, n * sizeof(float), xs.p);
    float* res = v.f32(1, n);
    uint8_t* codes = static_cast<uint8_t*>(v.ptr(3, kU8, n));
    float* mm = v.f32(4, 2 * chunks_of(n, chunk));
    return [=](void* s) { return f_bagua_reduce_compress_minmax_u8(xs.p, k, res, n, chunk, codes, mm, s); };
PY_END

PY(bagua_reduce_compress_sign_ef, 6)   // xs, residual, chunk, bits, scale, stream
    const size_t n = v.numel_of_first(0), chunk = v.size(2);
    Ptrs<const float> xs;
    const int k = v.list(0, kF32, n * sizeof(float), xs.p);
    float* res = v.f32(1, n);
    uint32_t* bits = static_cast<uint32_t*>(v.ptr(3, kI32, v.code_bytes(BAGUA_CODEC_SIGN1, n)));
    float* scale = v.f32(4, chunks_of(n, chunk));
    return [=](void* s) { return f_bagua_reduce_compress_sign_ef(xs.p, k, res, n, chunk, bits, scale, s); };
PY_END

PY(bagua_centralized_avg_fp, 3)   // xs, out, stream
    const size_t n = v.numel_of_first(0);
    Ptrs<const float> xs;
    const int k = v.list(0, kF32, n * sizeof(float), xs.p);
    float* out = v.f32(1, n);
    return [=](void* s) { return f_bagua_centralized_avg_fp(xs.p, k, n, out, s); };
PY_END

PY(bagua_decompress_sgd_step, 11)   // codec, codes, meta, n, chunk, param, momentum_buf, lr, momentum, weight_decay, stream
    const int codec = v.small(0);
    const size_t n = v.size(3), chunk = v.size(4);
    const void* codes = v.ptr(1, kAny, v.code_bytes(codec, n));
    const float* meta = v.f32(2, v.meta_floats(codec, n, chunk));
    float *param = v.f32(5, n), *mom = v.f32(6, n);
    const float lr = v.real(7), mu = v.real(8), wd = v.real(9);
    return [=](void* s) { return f_bagua_decompress_sgd_step(codec, codes, meta, n, chunk, param, mom, lr, mu, wd, s); };
PY_END

// codec, codes, meta, n, chunk, param, m, v, lr, beta1, beta2, eps, weight_decay, variance_frozen, stream
PY(bagua_decompress_adam_step, 15)
    const int codec = v.small(0);
    const size_t n = v.size(3), chunk = v.size(4);
    const void* codes = v.ptr(1, kAny, v.code_bytes(codec, n));
    const float* meta = v.f32(2, v.meta_floats(codec, n, chunk));
    float *param = v.f32(5, n), *m1 = v.f32(6, n), *m2 = v.f32(7, n);
    const float lr = v.real(8), b1 = v.real(9), b2 = v.real(10), eps = v.real(11), wd = v.real(12);
    const bool frozen = v.flag(13);
    return [=](void* s) { return f_bagua_decompress_adam_step(codec, codes, meta, n, chunk, param, m1, m2, lr, b1, b2, eps, wd, frozen, s); };
PY_END

PY(bagua_compress_topk_ef, 7)   // x, residual, chunk, keep, idx, val, stream
    const size_t n = v.numel(0), chunk = v.size(2), keep = v.size(3);
    const size_t slots = v.slots(keep, n, chunk);
    const float* x = v.f32(0, 0);
    float* res = v.f32(1, n);
    uint16_t* idx = static_cast<uint16_t*>(v.ptr(4, kI16, slots * sizeof(uint16_t)));
    float* val = v.f32(5, slots);
    return [=](void* s) { return f_bagua_compress_topk_ef(x, res, n, chunk, keep, idx, val, s); };
PY_END

PY(bagua_decompress_reduce_recompress_topk, 10)   // idx_in, val_in, keep, server_residual, n, chunk, idx_out, val_out, out_fp32, stream
    const size_t keep = v.size(2), n = v.size(4), chunk = v.size(5);
    const size_t slots = v.slots(keep, n, chunk);
    Ptrs<const uint16_t> ii;
    Ptrs<const float> vi;
    const int k = v.list(0, kI16, slots * sizeof(uint16_t), ii.p);
    v.list(1, kF32, slots * sizeof(float), vi.p, k);
    float* eps = v.f32(3, n);
    uint16_t* io = static_cast<uint16_t*>(v.ptr(6, kI16, slots * sizeof(uint16_t)));
    float *vo = v.f32(7, slots), *out = v.f32(8, n);
    return [=](void* s) { return f_bagua_decompress_reduce_recompress_topk(ii.p, vi.p, k, keep, eps, n, chunk, io, vo, out, s); };
PY_END

PY(bagua_decompress_topk, 7)   // idx, val, n, chunk, keep, out, stream
    const size_t n = v.size(2), chunk = v.size(3), keep = v.size(4);
    const size_t slots = v.slots(keep, n, chunk);
    const uint16_t* idx = static_cast<const uint16_t*>(v.ptr(0, kI16, slots * sizeof(uint16_t)));
    const float* val = v.f32(1, slots);
    float* out = v.f32(5, n);
    return [=](void* s) { return f_bagua_decompress_topk(idx, val, n, chunk, keep, out, s); };
PY_END

PY(bagua_decompress_sgd_step_topk, 11)   // idx, val, n, chunk, keep, param, momentum_buf, lr, momentum, weight_decay, stream
    const size_t n = v.size(2), chunk = v.size(3), keep = v.size(4);
    const size_t slots = v.slots(keep, n, chunk);
    const uint16_t* idx = static_cast<const uint16_t*>(v.ptr(0, kI16, slots * sizeof(uint16_t)));
    const float* val = v.f32(1, slots);
    float *param = v.f32(5, n), *mom = v.f32(6, n);
    const float lr = v.real(7), mu = v.real(8), wd = v.real(9);
    return [=](void* s) { return f_bagua_decompress_sgd_step_topk(idx, val, n, chunk, keep, param, mom, lr, mu, wd, s); };
PY_END

// idx, val, n, chunk, keep, param, m, v, lr, beta1, beta2, eps, weight_decay, variance_frozen, stream
PY(bagua_decompress_adam_step_topk, 15)
    const size_t n = v.size(2), chunk = v.size(3), keep = v.size(4);
    const size_t slots = v.slots(keep, n, chunk);
    const uint16_t* idx = static_cast<const uint16_t*>(v.ptr(0, kI16, slots * sizeof(uint16_t)));
    const float* val = v.f32(1, slots);
    float *param = v.f32(5, n), *m1 = v.f32(6, n), *m2 = v.f32(7, n);
    const float lr = v.real(8), b1 = v.real(9), b2 = v.real(10), eps = v.real(11), wd = v.real(12);
    const bool frozen = v.flag(13);
    return [=](void* s) { return f_bagua_decompress_adam_step_topk(idx, val, n, chunk, keep, param, m1, m2, lr, b1, b2, eps, wd, frozen, s); };
PY_END

#undef PY
#define PY(name, expected)                                                              \
    PyObject* py_##name(PyObject*, PyObject* const* a, Py_ssize_t given)                \
    {                                                                                   \
        return call("bagua_" #name, a, given, expected, [](Args& v) {

// The address of a plan that its object holds.
const bagua_tensor_plan_t* plan_at(size_t v) { return reinterpret_cast<const bagua_tensor_plan_t*>(v); }
int type_of(at::ScalarType t) { return t == at::kFloat ? BAGUA_F32 : t == at::kBFloat16 ? BAGUA_BF16 : t == at::kHalf ? BAGUA_F16 : -1; }

PY(grad_norm, 5)   // address of the plan, out, max_norm, grad_scale, stream
    const size_t plan = v.size(0);
    float* out = v.f32(1, 2);
    const double most = v.number(2), scale = v.number(3);
    v.ok = v.ok && out;
    return [=](void* s) { return f_bagua_grad_norm(plan_at(plan), scale, most, out, s); };
PY_END

PY(adamw_step, 10)   // address of the plan, step, lr, beta1, beta2, eps, weight_decay, clip, seed, stream
    const size_t plan = v.size(0), step = v.size(1), seed = v.size(8);
    const double lr = v.number(2), b1 = v.number(3), b2 = v.number(4), eps = v.number(5), wd = v.number(6);
    const float* clip = v.f32(7, 2);
    v.ok = v.ok && seed <= 0xffffffffu;
    return [=](void* s) { return f_bagua_adamw_step(plan_at(plan), step, lr, b1, b2, eps, wd, clip, static_cast<uint32_t>(seed), s); };
PY_END

PY(balance_stats, 10)   // logits, ids, mask, counts, prob, workspace, alpha, loss, weight, stream
    struct {
        const void *x[BAGUA_MAX_WORKERS], *i[BAGUA_MAX_WORKERS];
        const uint8_t* m[BAGUA_MAX_WORKERS];
        size_t rows[BAGUA_MAX_WORKERS];
    } p;
    const auto x = v.matrices(0, p.x, p.rows, false, -1, -1);
    const auto i = v.matrices(1, p.i, p.rows, true, -1, x.count);
    const bool masked = v.masks(2, p.m, p.rows, x.count) != nullptr;
    v.ok = v.ok && type_of(x.type) >= 0 && (i.type == at::kInt || i.type == at::kLong) && x.columns <= BAGUA_MAX_EXPERTS && i.columns <= x.columns;
    const size_t e = v.ok ? static_cast<size_t>(x.columns) : 0;
    int32_t* counts = static_cast<int32_t*>(v.ptr(3, kI32, (e + 1) * sizeof(int32_t)));
    float *prob = v.f32(4, e), *loss = v.f32(7, 1), *weight = v.f32(8, e);
    void* ws = v.ptr(5, kAny, 0);
    const size_t bytes = v.ok && v.given(5) ? THPVariable_Unpack(v.a[5]).nbytes() : 0;
    const double alpha = v.number(6);
    return [=](void* s) {
        return f_bagua_balance_stats(type_of(x.type), p.x, x.stride(), p.rows, x.count, static_cast<int>(e), p.i, i.type == at::kInt ? 4 : 8, i.stride(),
                                     static_cast<int>(i.columns), masked ? p.m : nullptr, counts, prob, alpha, loss, weight, ws, bytes, s);
    };
PY_END

PY(balance_grad, 6)   // logits, mask, weight, upstream, dlogits, stream
    struct {
        const void *x[BAGUA_MAX_WORKERS], *o[BAGUA_MAX_WORKERS];
        const uint8_t* m[BAGUA_MAX_WORKERS];
        size_t rows[BAGUA_MAX_WORKERS];
    } p;
    const auto x = v.matrices(0, p.x, p.rows, false, -1, -1);
    const bool masked = v.masks(1, p.m, p.rows, x.count) != nullptr;
    const auto o = v.matrices(4, p.o, p.rows, true, x.columns, x.count);
    v.ok = v.ok && type_of(x.type) >= 0 && o.type == x.type && x.columns <= BAGUA_MAX_EXPERTS;
    const size_t e = v.ok ? static_cast<size_t>(x.columns) : 0;
    const float *weight = v.f32(2, e), *up = v.f32(3, 1);
    return [=](void* s) {
        return f_bagua_balance_grad(type_of(x.type), p.x, x.stride(), p.rows, x.count, static_cast<int>(e), masked ? p.m : nullptr, weight, up,
                                    const_cast<void* const*>(p.o), o.stride(), s);
    };
PY_END

PY(route, 12)   // logits, mask, ids, weights, bias, score, groups, top_groups, group_best, renormalise, scale, stream
    struct {
        const void *x[BAGUA_MAX_WORKERS], *i[BAGUA_MAX_WORKERS], *w[BAGUA_MAX_WORKERS];
        const uint8_t* m[BAGUA_MAX_WORKERS];
        size_t rows[BAGUA_MAX_WORKERS];
    } p;
    const auto x = v.matrices(0, p.x, p.rows, false, -1, -1);
    const bool masked = v.masks(1, p.m, p.rows, x.count) != nullptr;
    const auto i = v.matrices(2, p.i, p.rows, true, -1, x.count);
    const auto w = v.matrices(3, p.w, p.rows, true, i.columns, x.count);
    v.ok = v.ok && type_of(x.type) >= 0 && (i.type == at::kInt || i.type == at::kLong) && w.type == at::kFloat && x.columns <= BAGUA_MAX_EXPERTS && i.columns <= x.columns;
    const size_t e = v.ok ? static_cast<size_t>(x.columns) : 0;
    const float* bias = v.f32(4, e);
    const int score = v.small(5), groups = v.small(6), top_groups = v.small(7), best = v.small(8);
    const bool renormalise = v.flag(9);
    const double scale = v.number(10);
    return [=](void* s) {
        return f_bagua_route(type_of(x.type), p.x, x.stride(), p.rows, x.count, static_cast<int>(e), masked ? p.m : nullptr, bias, score, groups, top_groups, best,
                             static_cast<int>(i.columns), renormalise, scale, const_cast<void* const*>(p.i), i.type == at::kInt ? 4 : 8, i.stride(),
                             reinterpret_cast<float* const*>(const_cast<void* const*>(p.w)), w.stride(), s);
    };
PY_END

PY(route_grad, 9)   // logits, ids, weights, dweights, dlogits, score, renormalise, scale, stream
    struct {
        const void *x[BAGUA_MAX_WORKERS], *i[BAGUA_MAX_WORKERS], *u[BAGUA_MAX_WORKERS], *o[BAGUA_MAX_WORKERS];
        size_t rows[BAGUA_MAX_WORKERS];
    } p;
    const int score = v.small(5);
    const bool renormalise = v.flag(6), of_weights = renormalise && score == BAGUA_SCORE_SOFTMAX;
    const double scale = v.number(7);
    const auto o = v.matrices(4, p.o, p.rows, false, -1, -1);
    const auto i = v.matrices(1, p.i, p.rows, true, -1, o.count);
    const auto u = v.matrices(3, p.u, p.rows, true, i.columns, o.count);
    const auto x = v.matrices(of_weights ? 2 : 0, p.x, p.rows, true, of_weights ? i.columns : o.columns, o.count);
    v.ok = v.ok && type_of(o.type) >= 0 && (i.type == at::kInt || i.type == at::kLong) && u.type == at::kFloat && x.type == (of_weights ? at::kFloat : o.type) &&
           o.columns <= BAGUA_MAX_EXPERTS && i.columns <= o.columns;
    // (whether the list that is not read fits the others is the general path's to say)
    const int other = of_weights ? 0 : 2;
    v.ok = v.ok && (!v.given(other) || ((PyList_CheckExact(v.a[other]) || PyTuple_CheckExact(v.a[other])) && PySequence_Fast_GET_SIZE(v.a[other]) == o.count));
    return [=](void* s) {
        return f_bagua_route_grad(type_of(o.type), of_weights ? nullptr : p.x, of_weights ? 0 : x.stride(), p.rows, o.count, static_cast<int>(o.columns), p.i,
                                  i.type == at::kInt ? 4 : 8, i.stride(), static_cast<int>(i.columns), of_weights ? reinterpret_cast<const float* const*>(p.x) : nullptr,
                                  of_weights ? x.stride() : 0, reinterpret_cast<const float* const*>(p.u), u.stride(), score, renormalise, scale,
                                  const_cast<void* const*>(p.o), o.stride(), s);
    };
PY_END

// What both passes of a distillation begin with: logits, ids, teacher, labels, mask.
struct Distilled {
    const void *x[BAGUA_MAX_WORKERS], *i[BAGUA_MAX_WORKERS], *t[BAGUA_MAX_WORKERS], *b[BAGUA_MAX_WORKERS];
    const uint8_t* m[BAGUA_MAX_WORKERS];
    size_t rows[BAGUA_MAX_WORKERS];
    size_t ld, ids_ld, teacher_ld, vocab;
    at::ScalarType dtype;
    int type, teacher, k, top, id_bytes, label_bytes;
    bool masked;
    explicit Distilled(Args& v)
    {
        const auto mx = v.matrices(0, x, rows, false, -1, -1);
        const auto mi = v.matrices(1, i, rows, true, -1, mx.count);
        const auto mt = v.matrices(2, t, rows, true, mi.columns, mx.count);
        const bool labelled = v.given(3);
        const at::ScalarType label = labelled ? v.row_vectors(3, b, rows, mx.count, 1) : at::kLong;
        masked = v.masks(4, m, rows, mx.count) != nullptr;
        type = type_of(dtype = mx.type), teacher = type_of(mt.type), k = mx.count;
        ld = mx.stride(), ids_ld = mi.stride(), teacher_ld = mt.stride(), vocab = static_cast<size_t>(mx.columns);
        v.ok = v.ok && type >= 0 && teacher >= 0 && (mi.type == at::kInt || mi.type == at::kLong) && (label == at::kInt || label == at::kLong) &&
               mx.columns <= BAGUA_MAX_VOCABULARY && mi.columns <= BAGUA_MAX_TEACHER_ENTRIES;
        top = v.ok ? static_cast<int>(mi.columns) : 0, id_bytes = mi.type == at::kInt ? 4 : 8, label_bytes = !labelled ? 0 : label == at::kInt ? 4 : 8;
    }
};

PY(distill_loss, 12)   // logits, ids, teacher, labels, mask, loss, stats, workspace, temperature, teacher_weight, label_weight, stream
    const Distilled d(v);
    struct {
        const void *l[BAGUA_MAX_WORKERS], *s[BAGUA_MAX_WORKERS];
    } p;
    const bool fp32 = v.row_vectors(5, p.l, d.rows, d.k, 1) == at::kFloat && v.row_vectors(6, p.s, d.rows, d.k, 3) == at::kFloat;
    v.ok = v.ok && fp32;
    void* ws = v.ptr(7, kAny, 0);
    const size_t bytes = v.ok && v.given(7) ? THPVariable_Unpack(v.a[7]).nbytes() : 0;
    const double temperature = v.number(8), teach = v.number(9), tell = v.number(10);
    return [=](void* s) {
        return f_bagua_distill_loss(d.type, d.x, d.ld, d.rows, d.k, d.vocab, d.i, d.id_bytes, d.ids_ld, d.top, d.teacher, d.t, d.teacher_ld, d.label_bytes ? d.b : nullptr,
                                    d.label_bytes, d.masked ? d.m : nullptr, temperature, teach, tell, reinterpret_cast<float* const*>(const_cast<void* const*>(p.l)),
                                    reinterpret_cast<float* const*>(const_cast<void* const*>(p.s)), ws, bytes, s);
    };
PY_END

PY(distill_grad, 12)   // logits, ids, teacher, labels, mask, stats, upstream, dlogits, temperature, teacher_weight, label_weight, stream
    const Distilled d(v);
    struct {
        const void *s[BAGUA_MAX_WORKERS], *u[BAGUA_MAX_WORKERS], *o[BAGUA_MAX_WORKERS];
        size_t rows[BAGUA_MAX_WORKERS];
    } p;
    for (int w = 0; w < d.k; ++w) p.rows[w] = d.rows[w];
    bool fp32 = v.row_vectors(5, p.s, d.rows, d.k, 3) == at::kFloat;
    const bool per_row = PyList_CheckExact(v.a[6]) || PyTuple_CheckExact(v.a[6]), up = v.given(6);
    if (per_row) {
        fp32 = v.row_vectors(6, p.u, d.rows, d.k, 1) == at::kFloat && fp32;
    } else {
        const float* one = v.f32(6, 1);
        for (int w = 0; w < d.k; ++w) p.u[w] = one;
    }
    const auto o = v.matrices(7, p.o, p.rows, true, static_cast<int64_t>(d.vocab), d.k);
    v.ok = v.ok && fp32 && o.type == d.dtype;
    const double temperature = v.number(8), teach = v.number(9), tell = v.number(10);
    return [=](void* s) {
        return f_bagua_distill_grad(d.type, d.x, d.ld, d.rows, d.k, d.vocab, d.i, d.id_bytes, d.ids_ld, d.top, d.teacher, d.t, d.teacher_ld, d.label_bytes ? d.b : nullptr,
                                    d.label_bytes, d.masked ? d.m : nullptr, temperature, teach, tell, reinterpret_cast<const float* const*>(p.s),
                                    up ? reinterpret_cast<const float* const*>(p.u) : nullptr, per_row, const_cast<void* const*>(p.o), o.stride(), s);
    };
PY_END

#undef PY
#undef PY_END

// The marshalling of a plan, which has thousands of tensors: numbers of elements, and addresses, as the words of a bytes object that the
// entry point reads in place of an array.  False where anything is out of the ordinary, as above.
//
// tensor_sizes(tensors)
PyObject* tensor_sizes(PyObject*, PyObject* const* a, Py_ssize_t given)
{
    if (given != 1 || !PyList_CheckExact(a[0])) Py_RETURN_FALSE;
    const Py_ssize_t count = PyList_GET_SIZE(a[0]);
    PyObject* out = PyBytes_FromStringAndSize(nullptr, count * static_cast<Py_ssize_t>(sizeof(size_t)));
    if (!out) return nullptr;
    size_t* n = reinterpret_cast<size_t*>(PyBytes_AS_STRING(out));
    for (Py_ssize_t i = 0; i < count; ++i) {
        PyObject* o = PyList_GET_ITEM(a[0], i);
        if (!THPVariable_CheckTypeExact(Py_TYPE(o))) {
            Py_DECREF(out);
            Py_RETURN_FALSE;
        }
        n[i] = static_cast<size_t>(THPVariable_Unpack(o).numel());
    }
    return out;
}

// tensor_addresses(tensors, one tensor of their type, sizes, per, exact): of contiguous tensors on the GPU with an element for `per` of
// each size, rounded up, or exactly as many
PyObject* tensor_addresses(PyObject*, PyObject* const* a, Py_ssize_t given)
{
    if (given != 5 || !PyList_CheckExact(a[0]) || !THPVariable_CheckTypeExact(Py_TYPE(a[1])) || !PyBytes_CheckExact(a[2])) Py_RETURN_FALSE;
    const Py_ssize_t count = PyList_GET_SIZE(a[0]);
    const size_t per = PyLong_AsSize_t(a[3]);
    if (PyErr_Occurred()) return nullptr;
    if (per == 0 || PyBytes_GET_SIZE(a[2]) != count * static_cast<Py_ssize_t>(sizeof(size_t))) Py_RETURN_FALSE;
    const at::ScalarType type = THPVariable_Unpack(a[1]).scalar_type();
    const size_t* n = reinterpret_cast<const size_t*>(PyBytes_AS_STRING(a[2]));
    PyObject* out = PyBytes_FromStringAndSize(nullptr, count * static_cast<Py_ssize_t>(sizeof(void*)));
    if (!out) return nullptr;
    void** p = reinterpret_cast<void**>(PyBytes_AS_STRING(out));
    bool ok = true;
    try {
        for (Py_ssize_t i = 0; i < count && ok; ++i) {
            PyObject* o = PyList_GET_ITEM(a[0], i);
            ok = THPVariable_CheckTypeExact(Py_TYPE(o));
            if (!ok) break;
            const at::Tensor& t = THPVariable_Unpack(o);
            const size_t need = n[i] / per + (n[i] % per != 0), has = static_cast<size_t>(t.numel());
            ok = t.is_cuda() && t.layout() == at::kStrided && t.is_contiguous() && t.scalar_type() == type && (a[4] == Py_True ? has == need : has >= need);
            if (ok) p[i] = need ? t.data_ptr() : nullptr;
        }
    } catch (...) {
        if (PyErr_Occurred()) PyErr_Clear();
        ok = false;
    }
    if (ok) return out;
    Py_DECREF(out);
    Py_RETURN_FALSE;
}

// bind(library, error, raw_stream, device): library = {name of an entry point: its address}
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t given)
{
    if (given != 4 || !PyDict_Check(a[0])) {
        PyErr_SetString(PyExc_TypeError, "bind(library, error, raw_stream, device)");
        return nullptr;
    }
#define X(name)                                                            \
    {                                                                      \
        PyObject* at = PyDict_GetItemString(a[0], #name);                  \
        void* p = at ? PyLong_AsVoidPtr(at) : nullptr;                     \
        if (!p) {                                                          \
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, #name); \
            return nullptr;                                                \
        }                                                                  \
        f_##name = reinterpret_cast<decltype(&name)>(p);                   \
    }
    BAGUA_NATIVE(X)
#undef X
#define X(name)                                                                     \
    {                                                                               \
        PyObject* at = PyDict_GetItemString(a[0], "bagua_" #name);                  \
        void* p = at ? PyLong_AsVoidPtr(at) : nullptr;                              \
        if (!p) {                                                                   \
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, "bagua_" #name); \
            return nullptr;                                                         \
        }                                                                           \
        f_bagua_##name = reinterpret_cast<decltype(&bagua_##name)>(p);              \
    }
    BAGUA_NATIVE_STEPS(X)
#undef X
    PyObject** keep[3] = {&g_error, &g_raw_stream, &g_device};
    for (int i = 0; i < 3; ++i) {
        Py_INCREF(a[1 + i]);
        Py_XSETREF(*keep[i], a[1 + i]);
    }
    Py_RETURN_NONE;
}

#define X(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr},
PyMethodDef g_methods[] = {BAGUA_NATIVE(X) BAGUA_NATIVE_STEPS(X){"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bind)), METH_FASTCALL, nullptr},
                           {"tensor_sizes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(tensor_sizes)), METH_FASTCALL, nullptr},
                           {"tensor_addresses", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(tensor_addresses)), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
#undef X
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() { return PyModule_Create(&g_module); }
