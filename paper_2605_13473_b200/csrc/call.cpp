// Argument marshalling of the hot calls (python module _osdn_call): torch tensors -> device pointers, the
// current stream of the current device, one call into libosdn.so.
//
// A decode step of one sequence is 2.7 us of GPU work, so the host side is what its caller waits for.  Built
// from Python objects (ctypes conversions, one method call per tensor property) that side took 10.9 us, with
// plain integers through ctypes 6.7 us; here the conversions take a few nanoseconds per tensor.
#include <Python.h>

#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <iterator>

#include "../../include/osdn.h"

namespace {

enum Call { FWD, BWD, KDA_FWD, KDA_BWD, PRECOND, RATIO, DECODE, FWD_STATIC,
            SCAN_FWD, SCAN_BWD, SCAN_STEP, CONV_FWD, CONV_BWD, CONV_STEP, NORM_FWD, NORM_BWD, CALLS };
// tensor arguments of each call, the workspace (an own pair of pointer and size in the ABI) included
constexpr int kTensors[CALLS] = {12, 20, 12, 20, 6, 7, 9, 11, 6, 9, 4, 6, 11, 5, 8, 13};
enum Params { LAYER, SCAN, CONV, NORM, PARAMS };
constexpr size_t kParamsBytes[PARAMS] = {sizeof(osdn_params), sizeof(osdn_scan_params), sizeof(osdn_conv_params),
                                         sizeof(osdn_qk_norm_params)};
Params params_of(long which)
{
    return which < SCAN_FWD ? LAYER : which < CONV_FWD ? SCAN : which < NORM_FWD ? CONV : NORM;
}

// ---- the operators on rows of channels: what each tensor has to be -------------------------------------------
enum Type { IO, F32, F64, I32, BYTES };
struct Expect {
    const char* name;
    Type type;
    int64_t numel;        // -1: any
    int64_t row = 0;      // elements from one token to the next where that is not the packed width
    int64_t width = 0;    // elements of a token's row (row != 0)
    int64_t head = 0;     //   and of its heads
    int64_t tokens = 0;
};

struct Shape {   // tokens and sequences of a batch
    int64_t tokens, seqs;
};
template <typename P> Shape shape_of(const P& p)
{
    return {p.nseq > 0 ? (int64_t)p.T : (int64_t)p.B * p.T, p.nseq > 0 ? (int64_t)p.nseq : (int64_t)p.B};
}

// Fills `e` with what the tensors of call `which` are under these (valid) params; entries the library does not require may be None.
void expect(long which, const void* params, Expect* e)
{
    if (which < CONV_FWD) {
        const auto& p = *static_cast<const osdn_scan_params*>(params);
        const Shape sh = shape_of(p);
        const int64_t n = sh.tokens * p.C, st = sh.seqs * p.C;
        if (which == SCAN_FWD) {
            const Expect x[] = {{"x", IO, n}, {"gate", F32, n}, {"init_state", F32, st}, {"out", IO, n},
                                {"final_state", F32, st}, {"workspace", BYTES, -1}};
            std::copy(std::begin(x), std::end(x), e);
        } else if (which == SCAN_BWD) {
            const Expect x[] = {{"x", IO, n}, {"gate", F32, n}, {"init_state", F32, st}, {"dout", IO, n},
                                {"dfinal_state", F32, st}, {"dx", IO, n}, {"dgate", F32, n}, {"dinit_state", F32, st},
                                {"workspace", BYTES, -1}};
            std::copy(std::begin(x), std::end(x), e);
        } else {
            const Expect x[] = {{"x", IO, n}, {"gate", F32, n}, {"state", F32, st}, {"out", IO, n}};
            std::copy(std::begin(x), std::end(x), e);
        }
    } else if (which < NORM_FWD) {
        const auto& p = *static_cast<const osdn_conv_params*>(params);
        const Shape sh = shape_of(p);
        const int64_t n = sh.tokens * p.C, st = sh.seqs * (p.W - 1) * p.C, w = (int64_t)p.C * p.W;
        if (which == CONV_FWD) {
            const Expect x[] = {{"x", IO, n}, {"weight", F32, w}, {"bias", F32, p.C}, {"init_state", IO, st}, {"out", IO, n},
                                {"final_state", IO, st}};
            std::copy(std::begin(x), std::end(x), e);
        } else if (which == CONV_BWD) {
            const Expect x[] = {{"x", IO, n}, {"weight", F32, w}, {"bias", F32, p.C}, {"init_state", IO, st}, {"dout", IO, n},
                                {"dfinal_state", IO, st}, {"dx", IO, n}, {"dweight", F32, w}, {"dbias", F32, p.C},
                                {"dinit_state", IO, st}, {"workspace", BYTES, -1}};
            std::copy(std::begin(x), std::end(x), e);
        } else {
            const Expect x[] = {{"x", IO, n}, {"weight", F32, w}, {"bias", F32, p.C}, {"state", IO, st}, {"out", IO, n}};
            std::copy(std::begin(x), std::end(x), e);
        }
    } else {
        const auto& p = *static_cast<const osdn_qk_norm_params*>(params);
        const int64_t tok = shape_of(p).tokens, wq = (int64_t)p.Hq * p.D, wk = (int64_t)p.Hk * p.D;
        const Expect in[] = {{"q", IO, tok * wq, p.q_row, wq, p.D, tok}, {"k", IO, tok * wk, p.k_row, wk, p.D, tok},
                             {"q_weight", F32, p.D}, {"k_weight", F32, p.D}, {"inv_freq", F64, p.rot_dim / 2},
                             {"positions", I32, tok}};
        e = std::copy(std::begin(in), std::end(in), e);
        if (which == NORM_FWD) {
            const Expect x[] = {{"q_out", IO, tok * wq}, {"k_out", IO, tok * wk}};
            std::copy(std::begin(x), std::end(x), e);
        } else {
            const Expect x[] = {{"dq_out", IO, tok * wq}, {"dk_out", IO, tok * wk}, {"dq", IO, tok * wq, p.dq_row, wq, p.D, tok},
                                {"dk", IO, tok * wk, p.dk_row, wk, p.D, tok}, {"dq_weight", F32, p.D}, {"dk_weight", F32, p.D},
                                {"workspace", BYTES, -1}};
            std::copy(std::begin(x), std::end(x), e);
        }
    }
}

// Whether a tensor steps through memory as the params say: contiguous, or a [tokens, heads, D] or [tokens, width] view of wider
// rows.  The kernels take `tokens` steps of `row`, so that a view of as many elements in fewer or other rows ends too early.
bool rows_match(const at::Tensor& t, const Expect& e)
{
    if (e.row == 0 || e.row == e.width) return t.is_contiguous();
    if (t.dim() < 2 || t.size(0) != e.tokens || (e.tokens > 1 && t.stride(0) != e.row)) return false;
    if (t.dim() == 2) return t.size(1) == e.width && t.stride(1) == 1;
    return t.dim() == 3 && t.size(2) == e.head && t.size(1) * e.head == e.width && t.stride(2) == 1 &&
           (t.size(1) == 1 || t.stride(1) == e.head);
}

// Type, size and layout; the device is asked for once all of them are what they have to be.
bool checked_layout(PyObject* o, const Expect& e, bool bf16)
{
    if (o == Py_None) return true;
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: the OSDN library takes torch tensors (or None)", e.name);
        return false;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    const at::ScalarType want = e.type == IO ? (bf16 ? at::kBFloat16 : at::kFloat)
                                : e.type == F32 ? at::kFloat : e.type == F64 ? at::kDouble : at::kInt;
    if (e.type != BYTES && t.scalar_type() != want) {
        PyErr_Format(PyExc_ValueError, "%s: wrong dtype", e.name);
        return false;
    }
    if (e.numel >= 0 && t.numel() != e.numel) {
        PyErr_Format(PyExc_ValueError, "%s: %lld elements, %lld expected", e.name, (long long)t.numel(), (long long)e.numel);
        return false;
    }
    if (!rows_match(t, e)) {
        PyErr_Format(PyExc_ValueError, e.row ? "%s: rows are not laid out as the params say" : "%s: must be contiguous", e.name);
        return false;
    }
    return true;
}

bool checked_pointer(PyObject* o, const Expect& e, int device, void** out, size_t* bytes)
{
    if (o == Py_None) {
        *out = nullptr;
        if (e.type == BYTES) *bytes = 0;
        return true;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != device) {
        PyErr_Format(PyExc_ValueError, "%s: not on the current CUDA device", e.name);
        return false;
    }
    *out = t.data_ptr();
    if (e.type == BYTES) *bytes = t.nbytes();
    return true;
}

bool pointer_of(PyObject* o, void** out, size_t* bytes)
{
    if (o == Py_None) {
        *out = nullptr;
        return true;
    }
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "the OSDN library takes torch tensors (or None)");
        return false;
    }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "tensors passed to the OSDN library must be contiguous");
        return false;
    }
    *out = t.data_ptr();
    if (bytes) *bytes = t.nbytes();
    return true;
}

template <typename F> int with_workspace(F fn, const osdn_params* p, void** x, size_t bytes, void* st);
using Fwd = decltype(&osdn_fwd);
using Bwd = decltype(&osdn_bwd);
template <> int with_workspace<Fwd>(Fwd fn, const osdn_params* p, void** x, size_t bytes, void* st)
{
    auto f = [&](int i) { return static_cast<float*>(x[i]); };
    return fn(p, x[0], x[1], x[2], f(3), f(4), f(5), f(6), f(7), x[8], f(9), f(10), x[11], bytes, st);
}
template <> int with_workspace<Bwd>(Bwd fn, const osdn_params* p, void** x, size_t bytes, void* st)
{
    auto f = [&](int i) { return static_cast<float*>(x[i]); };
    return fn(p, x[0], x[1], x[2], f(3), f(4), f(5), f(6), f(7), x[8], f(9), f(10), x[11], x[12], x[13], f(14), f(15),
              f(16), f(17), f(18), x[19], bytes, st);
}

struct GilReleased {   // taken back on every way out
    PyThreadState* state = PyEval_SaveThread();
    ~GilReleased() { PyEval_RestoreThread(state); }
};

PyObject* g_params_type[PARAMS] = {};   // binding.OsdnParams, ScanParams, ConvParams, QkNormParams

// register(*types): the classes of call's params
PyObject* register_params(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != PARAMS) {
        PyErr_SetString(PyExc_TypeError, "register(*types): one class for each kind of params");
        return nullptr;
    }
    for (int i = 0; i < PARAMS; ++i) {
        Py_INCREF(args[i]);
        Py_XSETREF(g_params_type[i], args[i]);
    }
    Py_RETURN_NONE;
}

int run_rows(long which, const void* params, void** x, size_t bytes, void* st)
{
    auto f = [&](int i) { return static_cast<float*>(x[i]); };
    const auto* s = static_cast<const osdn_scan_params*>(params);
    const auto* c = static_cast<const osdn_conv_params*>(params);
    const auto* n = static_cast<const osdn_qk_norm_params*>(params);
    switch (which) {
        case SCAN_FWD: return osdn_scan_fwd(s, x[0], f(1), f(2), x[3], f(4), x[5], bytes, st);
        case SCAN_BWD: return osdn_scan_bwd(s, x[0], f(1), f(2), x[3], f(4), x[5], f(6), f(7), x[8], bytes, st);
        case SCAN_STEP: return osdn_scan_step(s, x[0], f(1), f(2), x[3], st);
        case CONV_FWD: return osdn_short_conv_fwd(c, x[0], f(1), f(2), x[3], x[4], x[5], st);
        case CONV_BWD:
            return osdn_short_conv_bwd(c, x[0], f(1), f(2), x[3], x[4], x[5], x[6], f(7), f(8), x[9], x[10], bytes, st);
        case CONV_STEP: return osdn_short_conv_step(c, x[0], f(1), f(2), x[3], x[4], st);
        case NORM_FWD:
            return osdn_qk_norm_fwd(n, x[0], x[1], f(2), f(3), static_cast<double*>(x[4]), static_cast<int32_t*>(x[5]), x[6], x[7], st);
        default:
            return osdn_qk_norm_bwd(n, x[0], x[1], f(2), f(3), static_cast<double*>(x[4]), static_cast<int32_t*>(x[5]), x[6], x[7],
                                    x[8], x[9], f(10), f(11), x[12], bytes, st);
    }
}

bool valid_rows(long which, const void* params)
{
    switch (params_of(which)) {
        case SCAN: return osdn_scan_workspace_bytes(static_cast<const osdn_scan_params*>(params)) != 0;
        case CONV: return osdn_short_conv_workspace_bytes(static_cast<const osdn_conv_params*>(params)) != 0;
        default: return osdn_qk_norm_workspace_bytes(static_cast<const osdn_qk_norm_params*>(params)) != 0;
    }
}

bool is_bf16(long which, const void* params)
{
    switch (params_of(which)) {
        case SCAN: return static_cast<const osdn_scan_params*>(params)->io_dtype == OSDN_BF16;
        case CONV: return static_cast<const osdn_conv_params*>(params)->io_dtype == OSDN_BF16;
        default: return static_cast<const osdn_qk_norm_params*>(params)->io_dtype == OSDN_BF16;
    }
}

// Packed batches: the tensor that the params' cu_seqlens points into is on the device as well.  (Params whose pointer the caller has
// set by hand have none, and nothing is known of it.)
bool checked_boundaries(long which, const void* params, PyObject* object, int device)
{
    const Params kind = params_of(which);
    const int32_t nseq = kind == SCAN   ? static_cast<const osdn_scan_params*>(params)->nseq
                         : kind == CONV ? static_cast<const osdn_conv_params*>(params)->nseq
                                        : static_cast<const osdn_qk_norm_params*>(params)->nseq;
    if (nseq == 0) return true;
    PyObject* const o = PyObject_GetAttrString(object, "_cu_seqlens");
    if (!o) {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return false;
        PyErr_Clear();
        return true;
    }
    bool ok = true;
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        ok = t.is_cuda() && t.get_device() == device;
    }
    Py_DECREF(o);
    if (!ok) PyErr_SetString(PyExc_ValueError, "cu_seqlens: not on the current CUDA device");
    return ok;
}

// call(which, params, *tensors) -> status code of the library
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n < 2) {
        PyErr_SetString(PyExc_TypeError, "call(which, params, *tensors)");
        return nullptr;
    }
    const long which = PyLong_AsLong(args[0]);
    if (which == -1 && PyErr_Occurred()) return nullptr;
    if (which < FWD || which >= CALLS || n - 2 != kTensors[which]) {
        PyErr_SetString(PyExc_TypeError, "unknown call, or a wrong number of tensors");
        return nullptr;
    }
    const Params kind = params_of(which);
    const int known = g_params_type[kind] ? PyObject_IsInstance(args[1], g_params_type[kind]) : 0;
    if (known < 0) return nullptr;
    if (!known) {
        PyErr_SetString(PyExc_TypeError, kind == LAYER ? "params: not an OsdnParams" : "params: not this call's params");
        return nullptr;
    }
    Py_buffer view;   // the ctypes structure's own memory
    if (PyObject_GetBuffer(args[1], &view, PyBUF_SIMPLE) != 0) return nullptr;
    PyObject* result = nullptr;
    void* x[20];
    size_t bytes = 0;
    bool ok = view.len >= (Py_ssize_t)kParamsBytes[kind];
    if (!ok) PyErr_SetString(PyExc_TypeError, "params: not an OsdnParams");
    // torch throws where a tensor has no memory of its own (under vmap or grad) or there is no device: nothing may leave
    // through the C entry, it would end the process
    try {
        if (ok && kind != LAYER) {
            Expect e[13];
            const bool valid = valid_rows(which, view.buf);   // if not, the library says why
            const bool bf16 = is_bf16(which, view.buf);
            if (valid) expect(which, view.buf, e);
            for (Py_ssize_t i = 0; ok && valid && i < n - 2; ++i) ok = checked_layout(args[2 + i], e[i], bf16);
            const int device = ok && valid ? c10::cuda::current_device() : -1;
            for (Py_ssize_t i = 0; ok && valid && i < n - 2; ++i) ok = checked_pointer(args[2 + i], e[i], device, &x[i], &bytes);
            if (ok && valid) ok = checked_boundaries(which, view.buf, args[1], device);
            if (!valid) std::fill(std::begin(x), std::end(x), nullptr);
            if (ok) {
                void* st = valid ? c10::cuda::getCurrentCUDAStream().stream() : nullptr;
                int rc = 0;
                {
                    const GilReleased released;
                    rc = run_rows(which, view.buf, x, bytes, st);
                }
                result = PyLong_FromLong(rc);
            }
            ok = false;   // done
        }
        for (Py_ssize_t i = 0; ok && i < n - 2; ++i) ok = pointer_of(args[2 + i], &x[i], &bytes);   // the workspace is the last
        if (ok) {
            void* st = c10::cuda::getCurrentCUDAStream().stream();
            const osdn_params* p = static_cast<const osdn_params*>(view.buf);
            auto f = [&](int i) { return static_cast<float*>(x[i]); };
            int rc = 0;
            {
                const GilReleased released;   // a launch may wait for room in the stream
                switch (which) {
                    case FWD: rc = with_workspace<Fwd>(&osdn_fwd, p, x, bytes, st); break;
                    case KDA_FWD: rc = with_workspace<Fwd>(&osdn_kda_fwd, p, x, bytes, st); break;
                    case BWD: rc = with_workspace<Bwd>(&osdn_bwd, p, x, bytes, st); break;
                    case KDA_BWD: rc = with_workspace<Bwd>(&osdn_kda_bwd, p, x, bytes, st); break;
                    case PRECOND: rc = osdn_precond_update(p, x[0], f(1), f(2), f(3), x[4], f(5), st); break;
                    case RATIO: rc = osdn_residual_ratio(p, x[0], f(1), f(2), f(3), f(4), f(5), f(6), st); break;
                    case DECODE: rc = osdn_decode_step(p, x[0], x[1], x[2], f(3), f(4), f(5), f(6), f(7), x[8], st); break;
                    case FWD_STATIC:
                        rc = osdn_fwd_static(p, x[0], x[1], x[2], f(3), f(4), f(5), f(6), f(7), x[8], f(9), f(10), st);
                        break;
                }
            }
            result = PyLong_FromLong(rc);
        }
    } catch (const c10::Error& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    PyBuffer_Release(&view);
    return result;
}

PyMethodDef methods[] = {{"call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call)), METH_FASTCALL,
                          "call(which, params, *tensors) -> status code"},
                         {"register", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(register_params)), METH_FASTCALL,
                          "register(*types): the classes of call's params"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_osdn_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__osdn_call() { return PyModule_Create(&module); }
