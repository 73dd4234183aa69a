// The host side of a forward, decode or cache call from Python, natively: reads the tensors, allocates result and scratch with torch's allocator and
// calls the C ABI.  A call of one head x 128 rows is 8 us on the GPU and took the host 11.5 in Python (ctypes alone 2.3, strides, sizes and
// two allocations the rest); from here such calls follow each other at the GPU's pace, 8.1 us, and a single call ends 5 to 7 us earlier.
//
// It serves the ordinary forms only: plain torch tensors of the right types and shapes on the GPU.  For everything else -- and for every mistake --
// it returns NotImplemented without having done anything, and binding.py's own code takes the call, which words the errors.  A status of the C ABI
// other than 0 comes back as an integer.
#include <Python.h>

#include <ATen/Functions.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "llla.h"

namespace {

using ForwardFn = decltype(&llla_forward_ex);
using DecodeFn = decltype(&llla_decode_path);
using SizeFn = size_t (*)(int, int, int, int, llla_dtype);

constexpr int64_t MAX_DIM = 2147483647;

bool is_tensor(PyObject *o) { return THPVariable_CheckExact(o); }

bool dtype_of(at::ScalarType s, llla_dtype &t)
{
    if (s == at::kFloat) t = LLLA_F32;
    else if (s == at::kBFloat16) t = LLLA_BF16;
    else return false;
    return true;
}

// a [B, H, n, d] tensor on the GPU with unit stride along d
bool rows4(const at::Tensor &t, llla_strides &s)
{
    if (t.dim() != 4 || t.stride(3) != 1) return false;
    s = llla_strides{t.stride(0), t.stride(1), t.stride(2)};
    return true;
}

bool number(PyObject *o, double &v)
{
    if (!PyFloat_CheckExact(o)) return false;
    v = PyFloat_AS_DOUBLE(o);
    return true;
}

bool flag(PyObject *o, int &v)
{
    if (!PyBool_Check(o)) return false;
    v = o == Py_True;
    return true;
}

// dtype of a new result: None is float32
bool result_type(PyObject *o, at::ScalarType &t)
{
    llla_dtype unused;
    if (o == Py_None) t = at::kFloat;
    else if (THPDtype_Check(o)) t = reinterpret_cast<THPDtype *>(o)->scalar_type;
    else return false;
    return dtype_of(t, unused);
}

struct Scratch {
    at::Tensor own;
    void *ptr;
    size_t bytes;
};

// the caller's scratch, or without any `need` bytes from torch's allocator
Scratch scratch(const at::Tensor *given, size_t need, const at::Device &device)
{
    Scratch s;
    if (given == nullptr) {
        s.own = at::empty({(int64_t)(need < 256 ? 256 : need)}, at::TensorOptions().dtype(at::kByte).device(device));
        given = &s.own;
    }
    s.ptr = given->data_ptr();
    s.bytes = (size_t)given->numel() * given->element_size();
    return s;
}

PyObject *not_implemented() { Py_RETURN_NOTIMPLEMENTED; }

// The stream of a call: a handle, or what to call for the current stream's (asked only now that the tensors are known to be on the GPU)
void *stream_of(PyObject *o)
{
    if (PyLong_Check(o)) return PyLong_AsVoidPtr(o);
    PyObject *r = PyObject_CallNoArgs(o);
    if (r == nullptr) return nullptr;
    void *s = PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    return s;
}

// Other threads go on while torch allocates (which can wait for the GPU, or free what it holds and try again) and while the C ABI is called (a launch
// can wait for room in the queue), as they do where Python makes these calls.  Taken back on the way out, exceptions included.
struct WithoutGil {
    PyThreadState *state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

// forward(llla_forward_ex, llla_forward_workspace_bytes, Q, K, V, lam, scale, causal, out_dtype, path, workspace, out, return_stats, stream)
PyObject *forward(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    if (n_args != 14) return not_implemented();
    for (int i = 2; i < 5; ++i)
        if (!is_tensor(a[i])) return not_implemented();
    const at::Tensor &Q = THPVariable_Unpack(a[2]), &K = THPVariable_Unpack(a[3]), &V = THPVariable_Unpack(a[4]);
    llla_dtype in, out = LLLA_F32;
    llla_strides sq, sk, sv, so;
    at::ScalarType out_type;
    double lambda = 0., scale;
    int causal, stats;
    if (!Q.is_cuda() || !K.is_cuda() || !V.is_cuda() || K.scalar_type() != Q.scalar_type() || V.scalar_type() != Q.scalar_type() ||
        !dtype_of(Q.scalar_type(), in) || !rows4(Q, sq) || !rows4(K, sk) || !rows4(V, sv) || K.sizes() != Q.sizes() || V.sizes() != Q.sizes() ||
        !number(a[6], scale) || !flag(a[7], causal) || !result_type(a[8], out_type) || !flag(a[12], stats))
        return not_implemented();
    const int64_t B = Q.size(0), H = Q.size(1), n = Q.size(2), d = Q.size(3);
    if (B > MAX_DIM || H > MAX_DIM || n > MAX_DIM || d > MAX_DIM) return not_implemented();
    const float *lam_rows = nullptr;
    if (is_tensor(a[5])) {
        const at::Tensor &l = THPVariable_Unpack(a[5]);
        if (!l.is_cuda() || l.scalar_type() != at::kFloat || l.dim() != 3 || l.size(0) != B || l.size(1) != H || l.size(2) != n || !l.is_contiguous())
            return not_implemented();
        lam_rows = static_cast<const float *>(l.data_ptr());
    } else if (!number(a[5], lambda)) {
        return not_implemented();
    }
    if (a[11] != Py_None && (!is_tensor(a[11]) || !dtype_of(THPVariable_Unpack(a[11]).scalar_type(), out) || !rows4(THPVariable_Unpack(a[11]), so)))
        return not_implemented();
    const long path = PyLong_AsLong(a[9]);
    if (path < 0) return not_implemented();
    if (a[10] != Py_None && !is_tensor(a[10])) return not_implemented();

    void *stream = stream_of(a[13]);
    if (PyErr_Occurred()) return nullptr;
    const ForwardFn call = reinterpret_cast<ForwardFn>(PyLong_AsVoidPtr(a[0]));
    const SizeFn size = reinterpret_cast<SizeFn>(PyLong_AsVoidPtr(a[1]));
    const at::Tensor *given = a[10] == Py_None ? nullptr : &THPVariable_Unpack(a[10]);
    at::Tensor O, rho, delta;
    if (a[11] != Py_None) O = THPVariable_Unpack(a[11]);
    llla_status st;
    {
        WithoutGil released;
        const at::TensorOptions options = at::TensorOptions().device(Q.device()).dtype(at::kFloat);
        if (!O.defined()) {
            O = at::empty({B, H, n, d}, options.dtype(out_type));
            dtype_of(out_type, out);
            so = llla_strides{O.stride(0), O.stride(1), O.stride(2)};
        }
        if (stats) {
            rho = at::empty({B, H, n, d}, options);
            delta = at::empty({B, H, n}, options);
        }
        const Scratch ws = scratch(given, given ? 0 : size((int)B, (int)H, (int)n, (int)d, in), Q.device());
        st = call(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), sq, sk, sv, so, (int)B, (int)H, (int)n, (int)d, in, out, causal, (float)lambda,
                  lam_rows, (float)scale, stats ? static_cast<float *>(rho.data_ptr()) : nullptr,
                  stats ? static_cast<float *>(delta.data_ptr()) : nullptr, (llla_path)path, ws.ptr, ws.bytes, stream);
    }
    if (st != LLLA_OK) return PyLong_FromLong(st);
    PyObject *result;
    if (a[11] != Py_None) {
        Py_INCREF(a[11]);
        result = a[11];
    } else {
        result = THPVariable_Wrap(O);
    }
    if (!stats || result == nullptr) return result;
    PyObject *t = PyTuple_New(3);
    PyTuple_SET_ITEM(t, 0, result);
    PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(rho));
    PyTuple_SET_ITEM(t, 2, THPVariable_Wrap(delta));
    return t;
    END_HANDLE_TH_ERRORS
}

// decode(llla_decode_path, llla_decode_workspace_bytes, q, Kc, Vc, lam, scale, seqlens, out_dtype, path, workspace, out, stream)
PyObject *decode(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    if (n_args != 13) return not_implemented();
    for (int i = 2; i < 5; ++i)
        if (!is_tensor(a[i])) return not_implemented();
    const at::Tensor &q = THPVariable_Unpack(a[2]), &K = THPVariable_Unpack(a[3]), &V = THPVariable_Unpack(a[4]);
    llla_dtype in, out = LLLA_F32;
    llla_strides sk, sv;
    at::ScalarType out_type;
    double lambda, scale;
    if (!q.is_cuda() || !K.is_cuda() || !V.is_cuda() || K.scalar_type() != q.scalar_type() || V.scalar_type() != q.scalar_type() ||
        !dtype_of(q.scalar_type(), in) || !rows4(K, sk) || !rows4(V, sv) || V.sizes() != K.sizes() || !number(a[5], lambda) || !number(a[6], scale) ||
        !result_type(a[8], out_type))
        return not_implemented();
    const int64_t B = K.size(0), H = K.size(1), n = K.size(2), d = K.size(3);
    if (B > MAX_DIM || H > MAX_DIM || n > MAX_DIM || d > MAX_DIM) return not_implemented();
    if (q.dim() != 3 || q.size(0) != B || q.size(1) != H || q.size(2) != d || !q.is_contiguous()) return not_implemented();
    const int32_t *lens = nullptr;
    if (a[7] != Py_None) {
        if (!is_tensor(a[7])) return not_implemented();
        const at::Tensor &l = THPVariable_Unpack(a[7]);
        if (l.scalar_type() != at::kInt || !l.is_cuda() || l.numel() != B) return not_implemented();
        lens = static_cast<const int32_t *>(l.data_ptr());
    }
    if (a[11] != Py_None && (!is_tensor(a[11]) || !dtype_of(THPVariable_Unpack(a[11]).scalar_type(), out))) return not_implemented();
    const long path = PyLong_AsLong(a[9]);
    if (path < 0) return not_implemented();
    if (a[10] != Py_None && !is_tensor(a[10])) return not_implemented();

    void *stream = stream_of(a[12]);
    if (PyErr_Occurred()) return nullptr;
    const DecodeFn call = reinterpret_cast<DecodeFn>(PyLong_AsVoidPtr(a[0]));
    const SizeFn size = reinterpret_cast<SizeFn>(PyLong_AsVoidPtr(a[1]));
    const at::Tensor *given = a[10] == Py_None ? nullptr : &THPVariable_Unpack(a[10]);
    at::Tensor o;
    if (a[11] != Py_None) o = THPVariable_Unpack(a[11]);
    llla_status st;
    {
        WithoutGil released;
        if (!o.defined()) {
            o = at::empty({B, H, d}, at::TensorOptions().device(q.device()).dtype(out_type));
            dtype_of(out_type, out);
        }
        const Scratch ws = scratch(given, given ? 0 : size((int)B, (int)H, (int)n, (int)d, in), q.device());
        st = call(q.data_ptr(), K.data_ptr(), V.data_ptr(), o.data_ptr(), sk, sv, lens, (int)B, (int)H, (int)n, (int)d, in, out, (float)lambda, (float)scale,
                  (llla_path)path, ws.ptr, ws.bytes, stream);
    }
    if (st != LLLA_OK) return PyLong_FromLong(st);
    if (a[11] != Py_None) {
        Py_INCREF(a[11]);
        return a[11];
    }
    return THPVariable_Wrap(o);
    END_HANDLE_TH_ERRORS
}

// An optional contiguous array of `type` on `device`; its sizes are `want`
bool array(PyObject *o, at::ScalarType type, at::IntArrayRef want, const at::Device &device, void *&p)
{
    p = nullptr;
    if (o == Py_None) return true;
    if (!is_tensor(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.scalar_type() != type || t.device() != device || t.sizes() != want || !t.is_contiguous()) return false;
    p = t.data_ptr();
    return true;
}

// A Cache (a tuple of K, V, k_exp, v_exp, scores, pos) on the current GPU
bool cache_of(PyObject *o, llla_cache &c, at::Tensor &K)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 6 || !is_tensor(PyTuple_GET_ITEM(o, 0)) || !is_tensor(PyTuple_GET_ITEM(o, 1))) return false;
    K = THPVariable_Unpack(PyTuple_GET_ITEM(o, 0));
    const at::Tensor &V = THPVariable_Unpack(PyTuple_GET_ITEM(o, 1));
    if (!K.is_cuda() || V.device() != K.device() || V.scalar_type() != K.scalar_type() || !rows4(K, c.sk) || !rows4(V, c.sv) || V.sizes() != K.sizes()) return false;
    if (c10::impl::VirtualGuardImpl(K.device().type()).getDevice() != K.device()) return false;
    const bool codes = K.scalar_type() == at::kChar || K.scalar_type() == at::kFloat8_e4m3fn;
    if (codes) c.type = K.scalar_type() == at::kChar ? LLLA_I8 : LLLA_E4M3;
    else if (!dtype_of(K.scalar_type(), c.type)) return false;
    const int64_t B = K.size(0), H = K.size(1), n = K.size(2), d = K.size(3);
    if (B > MAX_DIM || H > MAX_DIM || n > MAX_DIM - 63 || d > MAX_DIM) return false;
    c.B = (int)B; c.H = (int)H; c.L_max = (int)n; c.d = (int)d;
    c.K = K.data_ptr();
    c.V = V.data_ptr();
    void *ke = nullptr, *ve = nullptr, *scores, *pos;
    if (codes && (!array(PyTuple_GET_ITEM(o, 2), at::kChar, {B, H, (n + 63) / 64}, K.device(), ke) ||
                  !array(PyTuple_GET_ITEM(o, 3), at::kChar, {B, H, (n + 63) / 64}, K.device(), ve) || ke == nullptr || ve == nullptr))
        return false;
    if (!array(PyTuple_GET_ITEM(o, 4), at::kFloat, {B, H, n}, K.device(), scores) || !array(PyTuple_GET_ITEM(o, 5), at::kInt, {B, H, n}, K.device(), pos)) return false;
    c.k_exp = static_cast<int8_t *>(ke);
    c.v_exp = static_cast<int8_t *>(ve);
    c.scores = static_cast<float *>(scores);
    c.pos = static_cast<int32_t *>(pos);
    return true;
}

// cache_append(llla_cache_append, cache, k, v, seqlens, new_lens, first_pos, stream)
PyObject *cache_append(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    llla_cache c{};
    at::Tensor K;
    if (n_args != 8 || !cache_of(a[1], c, K) || !is_tensor(a[2]) || !is_tensor(a[3])) return not_implemented();
    const at::Tensor &k = THPVariable_Unpack(a[2]), &v = THPVariable_Unpack(a[3]);
    llla_strides sk, sv;
    llla_dtype in;
    if (k.device() != K.device() || v.device() != K.device() || k.scalar_type() != v.scalar_type() || !dtype_of(k.scalar_type(), in) || !rows4(k, sk) || !rows4(v, sv) ||
        k.sizes() != v.sizes() || k.size(0) != c.B || k.size(1) != c.H || k.size(3) != c.d || k.size(2) > MAX_DIM)
        return not_implemented();
    void *lens[3];
    for (int i = 0; i < 3; ++i)
        if (!array(a[4 + i], at::kInt, {c.B}, K.device(), lens[i])) return not_implemented();
    void *stream = stream_of(a[7]);
    if (PyErr_Occurred()) return nullptr;
    const auto call = reinterpret_cast<decltype(&llla_cache_append)>(PyLong_AsVoidPtr(a[0]));
    llla_status st;
    {
        WithoutGil released;
        st = call(&c, k.data_ptr(), v.data_ptr(), sk, sv, (int)k.size(2), in, static_cast<int32_t *>(lens[0]), static_cast<int32_t *>(lens[1]),
                  static_cast<int32_t *>(lens[2]), stream);
    }
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// The caller's scratch of a cache call: None, or a contiguous tensor on the cache's device
bool given_scratch(PyObject *o, const at::Device &device, const at::Tensor *&t)
{
    t = nullptr;
    if (o == Py_None) return true;
    if (!is_tensor(o)) return false;
    t = &THPVariable_Unpack(o);
    return t->device() == device && t->is_contiguous();
}

// decode_q8(llla_decode_q8, llla_decode_q8_workspace_bytes, q, cache, lam, scale, seqlens, out_dtype, workspace, out, stream)
PyObject *decode_q8(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    llla_cache c{};
    at::Tensor K;
    if (n_args != 11 || !is_tensor(a[2]) || !cache_of(a[3], c, K)) return not_implemented();
    const at::Tensor &q = THPVariable_Unpack(a[2]);
    llla_dtype in, out = LLLA_F32;
    double lambda, scale;
    at::ScalarType out_type;
    void *lens;
    const at::Tensor *given;
    if ((c.type != LLLA_I8 && c.type != LLLA_E4M3) || q.device() != K.device() || !dtype_of(q.scalar_type(), in) || q.dim() != 3 || !q.is_contiguous() || q.size(0) != c.B ||
        q.size(2) != c.d || q.size(1) > MAX_DIM || !number(a[4], lambda) || !number(a[5], scale) || !array(a[6], at::kInt, {c.B}, K.device(), lens) ||
        !result_type(a[7], out_type) || !given_scratch(a[8], K.device(), given))
        return not_implemented();
    at::Tensor o;
    if (a[9] != Py_None) {
        if (!is_tensor(a[9])) return not_implemented();
        o = THPVariable_Unpack(a[9]);
        if (!dtype_of(o.scalar_type(), out) || o.sizes() != q.sizes() || !o.is_contiguous() || o.device() != K.device()) return not_implemented();
    }
    void *stream = stream_of(a[10]);
    if (PyErr_Occurred()) return nullptr;
    const auto call = reinterpret_cast<decltype(&llla_decode_q8)>(PyLong_AsVoidPtr(a[0]));
    const auto size = reinterpret_cast<decltype(&llla_decode_q8_workspace_bytes)>(PyLong_AsVoidPtr(a[1]));
    const int H = (int)q.size(1);
    llla_status st;
    {
        WithoutGil released;
        if (!o.defined()) {
            o = at::empty(q.sizes(), at::TensorOptions().device(q.device()).dtype(out_type));
            dtype_of(out_type, out);
        }
        const Scratch ws = scratch(given, given ? 0 : size(&c, H), K.device());
        st = call(q.data_ptr(), &c, o.data_ptr(), static_cast<int32_t *>(lens), H, in, out, (float)lambda, (float)scale, ws.ptr, ws.bytes, stream);
    }
    if (st != LLLA_OK) return PyLong_FromLong(st);
    if (a[9] != Py_None) {
        Py_INCREF(a[9]);
        return a[9];
    }
    return THPVariable_Wrap(o);
    END_HANDLE_TH_ERRORS
}

// cache_scores(llla_cache_scores, llla_cache_scores_workspace_bytes, Q, cache, scale, seqlens, workspace, stream)
PyObject *cache_scores(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    HANDLE_TH_ERRORS
    llla_cache c{};
    at::Tensor K;
    if (n_args != 8 || !is_tensor(a[2]) || !cache_of(a[3], c, K) || c.scores == nullptr) return not_implemented();
    const at::Tensor &Q = THPVariable_Unpack(a[2]);
    llla_dtype in;
    double scale;
    void *lens;
    const at::Tensor *given;
    const int64_t dims = Q.dim();
    if ((dims != 3 && dims != 4) || Q.device() != K.device() || !dtype_of(Q.scalar_type(), in) || Q.stride(dims - 1) != 1 || Q.size(0) != c.B || Q.size(dims - 1) != c.d ||
        Q.size(1) > MAX_DIM || (dims == 4 && Q.size(2) > MAX_DIM) || (c.type != LLLA_I8 && c.type != LLLA_E4M3 && c.type != in) || !number(a[4], scale) ||
        !array(a[5], at::kInt, {c.B}, K.device(), lens) || !given_scratch(a[6], K.device(), given))
        return not_implemented();
    const int H = (int)Q.size(1), nq = dims == 3 ? 1 : (int)Q.size(2);
    const llla_strides sq{Q.stride(0), Q.stride(1), dims == 3 ? c.d : Q.stride(2)};
    void *stream = stream_of(a[7]);
    if (PyErr_Occurred()) return nullptr;
    const auto call = reinterpret_cast<decltype(&llla_cache_scores)>(PyLong_AsVoidPtr(a[0]));
    const auto size = reinterpret_cast<decltype(&llla_cache_scores_workspace_bytes)>(PyLong_AsVoidPtr(a[1]));
    llla_status st;
    {
        WithoutGil released;
        const Scratch ws = scratch(given, given ? 0 : size(&c, H, nq, in), K.device());
        st = call(Q.data_ptr(), &c, sq, static_cast<int32_t *>(lens), H, nq, in, (float)scale, ws.ptr, ws.bytes, stream);
    }
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"forward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(forward)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(decode)), METH_FASTCALL, nullptr},
    {"cache_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(cache_append)), METH_FASTCALL, nullptr},
    {"decode_q8", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(decode_q8)), METH_FASTCALL, nullptr},
    {"cache_scores", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(cache_scores)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "llla_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_llla_host() { return PyModule_Create(&module); }
