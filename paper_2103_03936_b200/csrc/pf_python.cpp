// The Python side of the library: argument marshalling from torch tensors to the C ABI of include/pf.h,
// as one CPython extension module (_pf_native) linked against libpf.so.
//
// It exists because the calls it serves are short: a layer forward at a small batch runs a few
// microseconds on the GPU, and marshalling it through ctypes cost 15-20 us of host time per call
// (attribute look-ups on the tensors, one conversion per argument, torch.empty through the dispatcher).
// Here a call checks its tensors, takes its outputs and its workspace from torch's caching allocator
// and enters the C function without leaving native code.
//
// Every function takes the keyword arguments of its wrapper in binding.py by position.  `prepare` calls
// return (Prepared, outputs): an object that issues the C call with these arguments when it is called.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <functional>
#include <string>
#include <vector>

#include "pf.h"

namespace {

PyObject* g_pf_error = nullptr;      // binding.PfError, set once by binding.py

struct PyError {                     // becomes a Python exception of this type
    PyObject* type;
    std::string what;
};
[[noreturn]] void value_error(const std::string& s) { throw PyError{PyExc_ValueError, s}; }

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) throw PyError{PyExc_TypeError, std::string(name) + ": need a torch tensor"};
    return THPVariable_Unpack(o);
}
// An optional tensor argument: None gives an undefined tensor.
at::Tensor optional(PyObject* o, const char* name) {
    return o == Py_None ? at::Tensor() : at::Tensor(tensor(o, name));
}

int dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == at::kBFloat16) return PF_BF16;
    if (t.scalar_type() == at::kFloat) return PF_F32;
    throw PyError{PyExc_TypeError, std::string("unsupported dtype ") + c10::toString(t.scalar_type())};
}
void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// Row pitch of a 2-D CUDA matrix with unit column stride (0 for an absent one).
int64_t pitch(const at::Tensor& t, const char* name) {
    if (!t.defined()) return 0;
    if (!t.is_cuda() || t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1))
        value_error(std::string(name) + ": need a 2-D CUDA tensor with unit column stride");
    return t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(t.stride(0), t.size(1));
}

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like) {
    if (!like.is_cuda()) value_error("need CUDA tensors");
    return at::detail::empty_cuda(shape, type, like.device(), std::nullopt);
}

struct Stream {
    cudaStream_t s;
    bool current;        // the stream that torch's allocator orders its blocks by
};
Stream stream_of(PyObject* o) {
    const cudaStream_t cur = c10::cuda::getCurrentCUDAStream().stream();
    if (o == Py_None) return {cur, true};
    PyObject* v = PyObject_GetAttrString(o, "cuda_stream");
    if (!v) throw python_error();
    void* p = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) throw python_error();
    return {static_cast<cudaStream_t>(p), static_cast<cudaStream_t>(p) == cur};
}

// An output that the caller has not given, for a call with the argument `stream`.  On a stream other than torch's current one it is
// recorded, as a workspace is: a caller who drops it at once must not have its memory handed out again while the call still has to write it.
at::Tensor output(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& like, PyObject* stream) {
    at::Tensor t = empty(shape, type, like);
    if (stream == Py_None) return t;
    const Stream st = stream_of(stream);
    if (!st.current) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), c10::cuda::getStreamFromExternal(st.s, like.device().index()));
    return t;
}

// The caller's workspace, or a block of torch's caching allocator.  Such a block goes back to the
// allocator when the wrapper returns, while kernels that use it may still be queued: that is safe on
// torch's current stream (blocks are reused in stream order) and is made safe on any other stream by
// recording that stream on the block.
struct Workspace {
    at::Tensor given;
    c10::DataPtr own;
    void* p = nullptr;
    size_t bytes = 0;
};
Workspace workspace(PyObject* o, size_t need, const at::Tensor& like, const Stream& st) {
    Workspace w;
    if (o != Py_None) {
        w.given = tensor(o, "workspace");
        // (of a strided or expanded one the kernels would use memory that is not its)
        if (!w.given.is_cuda() || w.given.device() != like.device() || !w.given.is_contiguous())
            value_error("workspace: need a contiguous CUDA tensor on the device of the other tensors");
        w.p = w.given.data_ptr();
        w.bytes = static_cast<size_t>(w.given.numel());
        return w;
    }
    w.bytes = std::max<size_t>(need, 256);
    const c10::Device cur(c10::kCUDA, c10::cuda::current_device());
    if (like.device() != cur) {              // tensors of another device: a block of that device
        w.given = empty({static_cast<int64_t>(w.bytes)}, at::kByte, like);
        w.p = w.given.data_ptr();
        if (!st.current)
            c10::cuda::CUDACachingAllocator::recordStream(w.given.storage().data_ptr(),
                                                          c10::cuda::getStreamFromExternal(st.s, like.device().index()));
        return w;
    }
    w.own = c10::cuda::CUDACachingAllocator::get()->allocate(w.bytes);
    w.p = w.own.get();
    if (!st.current) c10::cuda::CUDACachingAllocator::recordStream(w.own, c10::cuda::getStreamFromExternal(st.s, cur.index()));
    return w;
}

void check(int status, const char* where) {
    if (status == PF_OK) return;
    PyObject* e = PyObject_CallFunction(g_pf_error, "is", status, where);
    if (e) {
        PyErr_SetObject(g_pf_error, e);
        Py_DECREF(e);
    }
    throw python_error();
}

// ---------------------------------------------------------------------------- prepared calls
struct PreparedState {
    std::function<int()> call;
    const char* where;
    std::vector<at::Tensor> keep;
    Workspace ws;
};
struct Prepared {
    PyObject_HEAD
    PreparedState* st;
};
PyObject* prepared_call(PyObject* self, PyObject*, PyObject*) {
    HANDLE_TH_ERRORS
    PreparedState* st = reinterpret_cast<Prepared*>(self)->st;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = st->call();
    Py_END_ALLOW_THREADS
    check(status, st->where);
    Py_RETURN_NONE;
    END_HANDLE_TH_ERRORS
}
void prepared_free(PyObject* self) {
    PyTypeObject* type = Py_TYPE(self);
    delete reinterpret_cast<Prepared*>(self)->st;
    PyObject_Free(self);
    Py_DECREF(type);
}
PyType_Slot g_prepared_slots[] = {{Py_tp_call, reinterpret_cast<void*>(prepared_call)},
                                  {Py_tp_dealloc, reinterpret_cast<void*>(prepared_free)},
                                  {Py_tp_doc, const_cast<char*>("A C call with its arguments marshalled once; keeps its tensors alive.")},
                                  {0, nullptr}};
PyType_Spec g_prepared_spec = {"_pf_native.Prepared", sizeof(Prepared), 0, Py_TPFLAGS_DEFAULT | Py_TPFLAGS_DISALLOW_INSTANTIATION, g_prepared_slots};
PyTypeObject* g_prepared_type = nullptr;

// Issues the call now (returns `out`), or wraps it (returns (Prepared, out)); steals `out`.
template <typename F>
PyObject* issue(bool prepare, F&& f, const char* where, Workspace&& ws, std::vector<at::Tensor> keep, PyObject* out) {
    if (!out) throw python_error();
    if (!prepare) {
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = f();
        Py_END_ALLOW_THREADS
        if (st != PF_OK) {
            Py_DECREF(out);
            check(st, where);
        }
        return out;
    }
    Prepared* p = PyObject_New(Prepared, g_prepared_type);
    if (!p) {
        Py_DECREF(out);
        throw python_error();
    }
    p->st = new PreparedState{std::function<int()>(std::forward<F>(f)), where, std::move(keep), std::move(ws)};
    return Py_BuildValue("(NN)", reinterpret_cast<PyObject*>(p), out);
}

PyObject* wrap(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject* tuple(std::initializer_list<at::Tensor> ts) {
    PyObject* out = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) PyTuple_SET_ITEM(out, i++, wrap(t));
    return out;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v == 1;
}
int64_t integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}

template <PyObject* (*body)(PyObject* const*)>
PyObject* entry_impl(PyObject* const* a) {
    HANDLE_TH_ERRORS
    try {
        return body(a);
    } catch (const PyError& e) {
        PyErr_SetString(e.type, e.what.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}
template <PyObject* (*body)(PyObject* const*), int kArgs>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != kArgs) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", kArgs, n);
        return nullptr;
    }
    return entry_impl<body>(a);
}

void rows_cols(const at::Tensor& t, const char* name, int64_t* rows, int64_t* cols) {
    if (t.dim() != 2) value_error(std::string(name) + ": need a 2-D CUDA tensor with unit column stride");
    *rows = t.size(0);
    *cols = t.size(1);
}

// ---------------------------------------------------------------------------- linear
// 0 x, 1 U, 2 V, 3 bias, 4 act, 5 y, 6 T_stash, 7 want_stash, 8 workspace, 9 stream, 10 prepare, 11 with_act
PyObject* linear_fwd(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor& U = tensor(a[1], "U");
    const at::Tensor& V = tensor(a[2], "V");
    const int dt = dtype_code(x);
    int64_t m, k, n, r;
    rows_cols(x, "x", &m, &k);
    rows_cols(V, "V", &n, &r);
    if (U.dim() != 2 || U.size(0) != k || U.size(1) != r) value_error("U must be [k, r] and V [n, r]");
    const at::Tensor bias = optional(a[3], "bias");
    if (bias.defined() && (bias.dim() != 1 || bias.size(0) != n || bias.scalar_type() != x.scalar_type() || !bias.is_contiguous()))
        value_error("bias must be a contiguous [n] tensor of x's dtype");
    const int act = static_cast<int>(integer(a[4]));
    at::Tensor y = optional(a[5], "y"), T = optional(a[6], "T_stash");
    if (!y.defined()) y = output({m, n}, x.scalar_type(), x, a[9]);
    if (!T.defined() && truth(a[7])) T = output({m, r}, x.scalar_type(), x, a[9]);
    const Stream st = stream_of(a[9]);
    Workspace ws = workspace(a[8], a[8] == Py_None ? pf_lowrank_linear_workspace(m, k, n, r, dt, 0) : 0, x, st);
    auto f = [=, px = ptr(x), pu = ptr(U), pv = ptr(V), pb = ptr(bias), py = ptr(y), pt = ptr(T), ldx = pitch(x, "x"),
              ldu = pitch(U, "U"), ldv = pitch(V, "V"), ldy = pitch(y, "y"), ldt = pitch(T, "T_stash"), wp = ws.p, wb = ws.bytes, s = st.s] {
        return pf_lowrank_linear_fwd_act(px, ldx, pu, ldu, pv, ldv, pb, act, py, ldy, pt, ldt, m, k, n, r, dt, wp, wb, s);
    };
    const bool prepare = truth(a[10]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {x, U, V, bias, y, T};
    return issue(prepare, f, truth(a[11]) ? "pf_lowrank_linear_fwd_act" : "pf_lowrank_linear_fwd", std::move(ws), std::move(keep),
                 T.defined() ? tuple({y, T}) : wrap(y));
}

// 0 x, 1 U, 2 V, 3 y, 4 T_stash, 5 stream
PyObject* linear_fwd_static(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor& U = tensor(a[1], "U");
    const at::Tensor& V = tensor(a[2], "V");
    const at::Tensor& y = tensor(a[3], "y");
    const at::Tensor T = optional(a[4], "T_stash");
    const int dt = dtype_code(x);
    int64_t m, k, n, r;
    rows_cols(x, "x", &m, &k);
    rows_cols(V, "V", &n, &r);
    if (U.dim() != 2 || U.size(0) != k || U.size(1) != r) value_error("U must be [k, r] and V [n, r]");
    const Stream st = stream_of(a[5]);
    const int64_t ldx = pitch(x, "x"), ldu = pitch(U, "U"), ldv = pitch(V, "V"), ldy = pitch(y, "y"), ldt = pitch(T, "T_stash");
    auto f = [=, px = ptr(x), pu = ptr(U), pv = ptr(V), py = ptr(y), pt = ptr(T), s = st.s] {
        return pf_lowrank_linear_fwd_static(px, ldx, pu, ldu, pv, ldv, py, ldy, pt, ldt, m, k, n, r, dt, s);
    };
    return issue(false, f, "pf_lowrank_linear_fwd_static", Workspace(), {}, T.defined() ? tuple({y, T}) : wrap(y));
}

unsigned grad_flags(PyObject* accumulate, PyObject* f32) {
    return (truth(accumulate) ? PF_GRAD_ACCUMULATE : 0u) | (truth(f32) ? PF_GRAD_F32 : 0u);
}

// 0 x, 1 U, 2 V, 3 dY, 4 T_stash, 5 need_dX, 6 dX, 7 dU, 8 dV, 9 accumulate, 10 grads_f32, 11 workspace, 12 stream, 13 prepare
PyObject* linear_bwd(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor& U = tensor(a[1], "U");
    const at::Tensor& V = tensor(a[2], "V");
    const at::Tensor& dY = tensor(a[3], "dY");
    const at::Tensor T = optional(a[4], "T_stash");
    const int dt = dtype_code(x);
    int64_t m, k, n, r;
    rows_cols(x, "x", &m, &k);
    rows_cols(V, "V", &n, &r);
    const unsigned flags = grad_flags(a[9], a[10]);
    const at::ScalarType gdt = (flags & PF_GRAD_F32) ? at::kFloat : x.scalar_type();
    at::Tensor dX = optional(a[6], "dX"), dU = optional(a[7], "dU"), dV = optional(a[8], "dV");
    if ((flags & PF_GRAD_ACCUMULATE) && (!dU.defined() || !dV.defined())) value_error("accumulate=True needs the dU and dV to add to");
    if (!dX.defined() && truth(a[5])) dX = output({m, k}, x.scalar_type(), x, a[12]);
    if (!dU.defined()) dU = output({k, r}, gdt, x, a[12]);
    if (!dV.defined()) dV = output({n, r}, gdt, x, a[12]);
    if (dU.scalar_type() != gdt || dV.scalar_type() != gdt)
        value_error("dU and dV must be float32 with grads_f32=True and of x's dtype otherwise");
    const Stream st = stream_of(a[12]);
    Workspace ws = workspace(a[11], a[11] == Py_None ? pf_lowrank_linear_workspace(m, k, n, r, dt, 1) : 0, x, st);
    auto f = [=, px = ptr(x), pu = ptr(U), pv = ptr(V), pdy = ptr(dY), pt = ptr(T), pdx = ptr(dX), pdu = ptr(dU), pdv = ptr(dV),
              ldx = pitch(x, "x"), ldu = pitch(U, "U"), ldv = pitch(V, "V"), lddy = pitch(dY, "dY"), ldt = pitch(T, "T_stash"),
              lddx = pitch(dX, "dX"), lddu = pitch(dU, "dU"), lddv = pitch(dV, "dV"), wp = ws.p, wb = ws.bytes, s = st.s] {
        return pf_lowrank_linear_bwd_ex(px, ldx, pu, ldu, pv, ldv, pdy, lddy, pt, ldt, pdx, lddx, pdu, lddu, pdv, lddv, m, k, n, r, dt,
                                        flags, wp, wb, s);
    };
    const bool prepare = truth(a[13]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {x, U, V, dY, T, dX, dU, dV};
    return issue(prepare, f, flags ? "pf_lowrank_linear_bwd_ex" : "pf_lowrank_linear_bwd", std::move(ws), std::move(keep),
                 tuple({dX, dU, dV}));
}

// 0 y, 1 dY, 2 act, 3 want_dbias, 4 dbias, 5 workspace, 6 stream
PyObject* bias_act_bwd(PyObject* const* a) {
    const at::Tensor y = optional(a[0], "y");
    const at::Tensor& dY = tensor(a[1], "dY");
    const int dt = dtype_code(dY);
    const int act = static_cast<int>(integer(a[2]));
    int64_t m, n;
    rows_cols(dY, "dY", &m, &n);
    at::Tensor db = optional(a[4], "dbias");
    if (!db.defined() && truth(a[3])) db = output({n}, dY.scalar_type(), dY, a[6]);
    const Stream st = stream_of(a[6]);
    Workspace ws = workspace(a[5], db.defined() && a[5] == Py_None ? pf_bias_act_bwd_workspace(m, n) : 0, dY, st);
    auto f = [=, py = ptr(y), pdy = ptr(dY), pdb = ptr(db), ldy = pitch(y, "y"), lddy = pitch(dY, "dY"), wp = ws.p, wb = ws.bytes, s = st.s] {
        return pf_bias_act_bwd(py, ldy, pdy, lddy, pdb, m, n, act, dt, wp, wb, s);
    };
    return issue(false, f, "pf_bias_act_bwd", std::move(ws), {}, wrap(db));
}

// ---------------------------------------------------------------------------- grouped linear
struct Group {
    void* p;
    int64_t ld, gs;
};
// (pointer, row pitch, group stride) of a [groups, rows, cols] tensor (unit column stride), or of a 2-D
// [rows, cols] tensor shared by all groups (stride 0) where that is allowed.
Group group(const at::Tensor& t, const char* name, int64_t groups, bool may_share = false) {
    if (!t.defined()) return {nullptr, 0, 0};
    if (t.dim() == 2 && may_share) return {t.data_ptr(), pitch(t, name), 0};
    if (!t.is_cuda() || t.dim() != 3 || t.size(0) != groups || (t.size(2) > 1 && t.stride(2) != 1))
        value_error(std::string(name) + ": need a CUDA tensor [groups, rows, cols] with unit column stride");
    return {t.data_ptr(), t.size(1) > 1 ? t.stride(1) : std::max<int64_t>(t.stride(1), t.size(2)), t.stride(0)};
}

// 0 x, 1 U, 2 V, 3 y, 4 T_stash, 5 want_stash, 6 workspace, 7 stream, 8 prepare
PyObject* grouped_fwd(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor& U = tensor(a[1], "U");
    const at::Tensor& V = tensor(a[2], "V");
    const int dt = dtype_code(U);
    if (U.dim() != 3 || V.dim() != 3 || x.dim() < 2) value_error("U must be [G, k, r], V [G, n, r], x [G, m, k] or [m, k]");
    const int64_t G = U.size(0), k = U.size(1), r = U.size(2), n = V.size(1), m = x.size(-2);
    if (V.size(0) != G || V.size(2) != r || x.size(-1) != k) value_error("U must be [G, k, r], V [G, n, r], x [G, m, k] or [m, k]");
    at::Tensor y = optional(a[3], "y"), T = optional(a[4], "T_stash");
    if (!y.defined()) y = output({G, m, n}, U.scalar_type(), U, a[7]);
    if (!T.defined() && truth(a[5])) T = output({G, m, r}, U.scalar_type(), U, a[7]);
    const Stream st = stream_of(a[7]);
    const int g = static_cast<int>(G);
    Workspace ws = workspace(a[6], a[6] == Py_None ? pf_lowrank_linear_grouped_workspace(g, m, k, n, r, dt, 0) : 0, U, st);
    auto f = [=, gx = group(x, "x", G, true), gu = group(U, "U", G), gv = group(V, "V", G), gy = group(y, "y", G), gt = group(T, "T_stash", G),
              wp = ws.p, wb = ws.bytes, s = st.s] {
        return pf_lowrank_linear_grouped_fwd(g, gx.p, gx.ld, gx.gs, gu.p, gu.ld, gu.gs, gv.p, gv.ld, gv.gs, gy.p, gy.ld, gy.gs, gt.p, gt.ld,
                                             gt.gs, m, k, n, r, dt, wp, wb, s);
    };
    const bool prepare = truth(a[8]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {x, U, V, y, T};
    return issue(prepare, f, "pf_lowrank_linear_grouped_fwd", std::move(ws), std::move(keep), T.defined() ? tuple({y, T}) : wrap(y));
}

// 0 x, 1 U, 2 V, 3 dY, 4 T_stash, 5 need_dX, 6 dX, 7 dU, 8 dV, 9 workspace, 10 stream, 11 prepare
PyObject* grouped_bwd(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor& U = tensor(a[1], "U");
    const at::Tensor& V = tensor(a[2], "V");
    const at::Tensor& dY = tensor(a[3], "dY");
    const at::Tensor T = optional(a[4], "T_stash");
    const int dt = dtype_code(U);
    if (U.dim() != 3 || V.dim() != 3 || x.dim() < 2) value_error("U must be [G, k, r], V [G, n, r], x [G, m, k] or [m, k]");
    const int64_t G = U.size(0), k = U.size(1), r = U.size(2), n = V.size(1), m = x.size(-2);
    at::Tensor dX = optional(a[6], "dX"), dU = optional(a[7], "dU"), dV = optional(a[8], "dV");
    if (!dX.defined() && truth(a[5])) dX = x.dim() == 2 ? output({m, k}, U.scalar_type(), U, a[10]) : output({G, m, k}, U.scalar_type(), U, a[10]);
    if (!dU.defined()) dU = output({G, k, r}, U.scalar_type(), U, a[10]);
    if (!dV.defined()) dV = output({G, n, r}, U.scalar_type(), U, a[10]);
    const Stream st = stream_of(a[10]);
    const int g = static_cast<int>(G);
    Workspace ws = workspace(a[9], a[9] == Py_None ? pf_lowrank_linear_grouped_workspace(g, m, k, n, r, dt, 1) : 0, U, st);
    auto f = [=, gx = group(x, "x", G, true), gu = group(U, "U", G), gv = group(V, "V", G), gdy = group(dY, "dY", G), gt = group(T, "T_stash", G),
              gdx = group(dX, "dX", G, true), gdu = group(dU, "dU", G), gdv = group(dV, "dV", G), wp = ws.p, wb = ws.bytes, s = st.s] {
        return pf_lowrank_linear_grouped_bwd(g, gx.p, gx.ld, gx.gs, gu.p, gu.ld, gu.gs, gv.p, gv.ld, gv.gs, gdy.p, gdy.ld, gdy.gs, gt.p, gt.ld,
                                             gt.gs, gdx.p, gdx.ld, gdx.gs, gdu.p, gdu.ld, gdu.gs, gdv.p, gdv.ld, gdv.gs, m, k, n, r, dt, wp,
                                             wb, s);
    };
    const bool prepare = truth(a[11]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {x, U, V, dY, T, dX, dU, dV};
    return issue(prepare, f, "pf_lowrank_linear_grouped_bwd", std::move(ws), std::move(keep), tuple({dX, dU, dV}));
}

// ---------------------------------------------------------------------------- convolution
struct Conv {
    int N, H, W, C, R, O, kh, kw, Ho, Wo, stride, pad;
};
Conv conv_dims(const at::Tensor& x, const at::Tensor& U, const at::Tensor& V, PyObject* stride, PyObject* pad) {
    const struct { const at::Tensor* t; const char* name; int dims; } all[3] = {{&x, "x", 4}, {&U, "U", 4}, {&V, "V", 2}};
    for (const auto& e : all) {
        if (!e.t->is_cuda() || !e.t->is_contiguous()) value_error(std::string(e.name) + ": need a contiguous CUDA tensor");
        if (e.t->dim() != e.dims) value_error("x must be [N, H, W, C], U [kh, kw, C, R] and V [O, R]");
    }
    Conv c;
    c.N = static_cast<int>(x.size(0)); c.H = static_cast<int>(x.size(1)); c.W = static_cast<int>(x.size(2)); c.C = static_cast<int>(x.size(3));
    c.kh = static_cast<int>(U.size(0)); c.kw = static_cast<int>(U.size(1)); c.R = static_cast<int>(U.size(3));
    c.O = static_cast<int>(V.size(0));
    if (U.size(2) != c.C || V.size(1) != c.R) value_error("U must be [kh, kw, C, R] and V [O, R]");
    c.stride = static_cast<int>(integer(stride)); c.pad = static_cast<int>(integer(pad));
    if (c.stride == 0) throw PyError{PyExc_ZeroDivisionError, "integer division or modulo by zero"};
    auto out = [&](int size, int k) {        // floor division
        const int num = size + 2 * c.pad - k;
        int q = num / c.stride;
        if (num % c.stride != 0 && ((num < 0) != (c.stride < 0))) --q;
        return q + 1;
    };
    c.Ho = out(c.H, c.kh); c.Wo = out(c.W, c.kw);
    return c;
}
size_t conv_workspace(const Conv& c, int dt, int bwd) {
    return pf_lowrank_conv_workspace(c.N, c.H, c.W, c.C, c.R, c.O, c.kh, c.kw, c.stride, c.pad, dt, bwd);
}

// 0 x, 1 U, 2 V, 3 stride, 4 pad, 5 y, 6 T_stash, 7 want_stash, 8 workspace, 9 stream, 10 prepare
PyObject* conv_fwd(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor& U = tensor(a[1], "U");
    const at::Tensor& V = tensor(a[2], "V");
    const int dt = dtype_code(x);
    const Conv c = conv_dims(x, U, V, a[3], a[4]);
    at::Tensor y = optional(a[5], "y"), T = optional(a[6], "T_stash");
    if (!y.defined()) y = output({c.N, c.Ho, c.Wo, c.O}, x.scalar_type(), x, a[9]);
    if (!T.defined() && truth(a[7])) T = output({c.N, c.Ho, c.Wo, c.R}, x.scalar_type(), x, a[9]);
    const Stream st = stream_of(a[9]);
    Workspace ws = workspace(a[8], a[8] == Py_None ? conv_workspace(c, dt, 0) : 0, x, st);
    auto f = [=, px = ptr(x), pu = ptr(U), pv = ptr(V), py = ptr(y), pt = ptr(T), wp = ws.p, wb = ws.bytes, s = st.s] {
        return pf_lowrank_conv_fwd(px, pu, pv, py, pt, c.N, c.H, c.W, c.C, c.R, c.O, c.kh, c.kw, c.stride, c.pad, dt, wp, wb, s);
    };
    const bool prepare = truth(a[10]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {x, U, V, y, T};
    return issue(prepare, f, "pf_lowrank_conv_fwd", std::move(ws), std::move(keep), T.defined() ? tuple({y, T}) : wrap(y));
}

// 0 x, 1 U, 2 V, 3 dY, 4 stride, 5 pad, 6 T_stash, 7 need_dX, 8 dX, 9 dU, 10 dV, 11 accumulate, 12 grads_f32, 13 workspace,
// 14 stream, 15 prepare
PyObject* conv_bwd(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor& U = tensor(a[1], "U");
    const at::Tensor& V = tensor(a[2], "V");
    const at::Tensor& dY = tensor(a[3], "dY");
    const int dt = dtype_code(x);
    const Conv c = conv_dims(x, U, V, a[4], a[5]);
    if (!dY.is_contiguous() || dY.dim() != 4 || dY.size(0) != c.N || dY.size(1) != c.Ho || dY.size(2) != c.Wo || dY.size(3) != c.O)
        value_error("dY must be contiguous [N, Ho, Wo, O]");
    const at::Tensor T = optional(a[6], "T_stash");
    at::Tensor dX = optional(a[8], "dX"), dU = optional(a[9], "dU"), dV = optional(a[10], "dV");
    if (!dX.defined() && truth(a[7])) dX = output(x.sizes(), x.scalar_type(), x, a[14]);
    const unsigned flags = grad_flags(a[11], a[12]);
    const at::ScalarType gdt = (flags & PF_GRAD_F32) ? at::kFloat : x.scalar_type();
    if ((flags & PF_GRAD_ACCUMULATE) && (!dU.defined() || !dV.defined())) value_error("accumulate=True needs the dU and dV to add to");
    if (!dU.defined()) dU = output(U.sizes(), gdt, x, a[14]);
    if (!dV.defined()) dV = output(V.sizes(), gdt, x, a[14]);
    if (dU.scalar_type() != gdt || dV.scalar_type() != gdt || !dU.is_contiguous() || !dV.is_contiguous())
        value_error("dU and dV must be contiguous, float32 with grads_f32=True and of x's dtype otherwise");
    const Stream st = stream_of(a[14]);
    Workspace ws = workspace(a[13], a[13] == Py_None ? conv_workspace(c, dt, 1) : 0, x, st);
    auto f = [=, px = ptr(x), pu = ptr(U), pv = ptr(V), pdy = ptr(dY), pt = ptr(T), pdx = ptr(dX), pdu = ptr(dU), pdv = ptr(dV), wp = ws.p,
              wb = ws.bytes, s = st.s] {
        return pf_lowrank_conv_bwd_ex(px, pu, pv, pdy, pt, pdx, pdu, pdv, c.N, c.H, c.W, c.C, c.R, c.O, c.kh, c.kw, c.stride, c.pad, dt, flags,
                                      wp, wb, s);
    };
    const bool prepare = truth(a[15]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {x, U, V, dY, T, dX, dU, dV};
    return issue(prepare, f, flags ? "pf_lowrank_conv_bwd_ex" : "pf_lowrank_conv_bwd", std::move(ws), std::move(keep), tuple({dX, dU, dV}));
}

// ---------------------------------------------------------------------------- flat gradient buffer
struct TensorList {
    std::vector<void*> ptrs;
    std::vector<int64_t> numels, offsets;     // offsets: prefix sums of numels, one more entry
    std::vector<at::Tensor> keep;
    at::Tensor first;
};
// The tensors of a list; `like` (or else the first one) sets the dtype that all of them must have.
TensorList tensor_list(PyObject* seq, const at::Tensor& like, const char* whose, bool keep) {
    TensorList l;
    PyObject* fast = PySequence_Fast(seq, "grads: need a sequence of tensors");
    if (!fast) throw python_error();
    struct Drop { PyObject* o; ~Drop() { Py_DECREF(o); } } drop{fast};
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
    l.ptrs.resize(n); l.numels.resize(n); l.offsets.resize(n + 1);
    at::ScalarType type = at::kFloat;
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor& t = tensor(PySequence_Fast_GET_ITEM(fast, i), "grads");
        if (i == 0) {
            l.first = t;
            const at::Tensor& ref = like.defined() ? like : t;
            dtype_code(ref);
            type = ref.scalar_type();
        }
        if (!t.is_cuda() || !t.is_contiguous() || t.scalar_type() != type)
            value_error(std::string("grads: contiguous CUDA tensors of ") + whose + " dtype");
        l.ptrs[i] = t.data_ptr();
        l.numels[i] = t.numel();
        l.offsets[i + 1] = l.offsets[i] + l.numels[i];
        if (keep) l.keep.push_back(t);
    }
    return l;
}
PyObject* offset_list(const std::vector<int64_t>& offs) {
    PyObject* out = PyList_New(static_cast<Py_ssize_t>(offs.size()));
    for (size_t i = 0; out && i < offs.size(); ++i) PyList_SET_ITEM(out, static_cast<Py_ssize_t>(i), PyLong_FromLongLong(offs[i]));
    return out;
}

// 0 grads (not empty), 1 flat, 2 stream, 3 prepare
PyObject* pack(PyObject* const* a) {
    at::Tensor flat = optional(a[1], "flat");
    const bool prepare = truth(a[3]);
    TensorList l = tensor_list(a[0], at::Tensor(), "one", prepare);
    const int dt = dtype_code(l.first), count = static_cast<int>(l.ptrs.size());
    if (!flat.defined()) flat = output({l.offsets[count]}, l.first.scalar_type(), l.first, a[2]);
    const Stream st = stream_of(a[2]);
    PyObject* out = Py_BuildValue("(NN)", wrap(flat), offset_list(l.offsets));
    std::vector<at::Tensor> keep = std::move(l.keep);
    if (prepare) keep.push_back(flat);
    l.first = at::Tensor();
    auto f = [l = std::move(l), dt, p = ptr(flat), n = flat.numel(), s = st.s, count]() mutable {
        return pf_pack_factor_grads(l.ptrs.data(), l.numels.data(), count, dt, p, n, l.offsets.data(), nullptr, 0, s);
    };
    return issue(prepare, std::move(f), "pf_pack_factor_grads", Workspace(), std::move(keep), out);
}

// 0 flat, 1 grads (not empty), 2 stream
PyObject* unpack(PyObject* const* a) {
    const at::Tensor& flat = tensor(a[0], "flat");
    TensorList l = tensor_list(a[1], flat, "flat's", false);
    const int dt = dtype_code(flat);
    const Stream st = stream_of(a[2]);
    void* p = ptr(flat);
    const int64_t n = flat.numel();
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = pf_unpack_factor_grads(p, n, l.ptrs.data(), l.numels.data(), static_cast<int>(l.ptrs.size()), dt, l.offsets.data(), nullptr, 0, st.s);
    Py_END_ALLOW_THREADS
    check(status, "pf_unpack_factor_grads");
    return offset_list(l.offsets);
}

// ---------------------------------------------------------------------------- operators around the layers
// The device of a call's tensors: all of them have to be on one, which is made current for the call.
struct OnDevice {
    c10::Device device;
    c10::cuda::OptionalCUDAGuard guard;
    explicit OnDevice(const at::Tensor& t, const char* name) : device(t.device()) {
        if (!t.is_cuda()) value_error(std::string(name) + ": need a CUDA tensor");
        guard.set_device(device);
    }
    // An argument of a dtype and number of dimensions (undefined ones pass).
    void check(const at::Tensor& t, const char* name, at::ScalarType type, int64_t dims, bool contiguous) const {
        if (!t.defined()) return;
        if (t.device() != device || t.scalar_type() != type || t.dim() != dims || (contiguous && !t.is_contiguous()))
            value_error(std::string(name) + ": need a " + (contiguous ? "contiguous " : "") + c10::toString(type) + " tensor of " + std::to_string(dims) +
                        " dimensions on " + device.str());
    }
};
// Issues a C call (or prepares it) with the tensors' device current.
template <typename F>
PyObject* issue_on(const OnDevice& on, bool prepare, F&& f, const char* where, Workspace&& ws, std::vector<at::Tensor> keep, PyObject* out) {
    if (!prepare) return issue(false, std::forward<F>(f), where, std::move(ws), {}, out);
    return issue(true, [f = std::forward<F>(f), index = on.device.index()]() mutable {
        const c10::cuda::CUDAGuard guard(index);
        return f();
    }, where, std::move(ws), std::move(keep), out);
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw python_error();
    return v;
}
int int_of(PyObject* o, const char* name) {
    const int64_t v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) value_error(std::string(name) + ": out of range");
    return static_cast<int>(v);
}

// Rows [tokens, heads, dim] with contiguous elements.
struct Heads {
    void* p;
    int64_t ld, s;
};
Heads heads_of(const OnDevice& on, const at::Tensor& t, const char* name, const at::Tensor& like) {
    if (!t.defined()) return {nullptr, 0, 0};
    if (!like.defined()) value_error(std::string(name) + ": given without the rows that it goes with");
    on.check(t, name, like.scalar_type(), 3, false);
    if (t.sizes() != like.sizes() || (t.size(2) > 1 && t.stride(2) != 1))
        value_error(std::string(name) + ": need [tokens, heads, dim] with contiguous elements, as q or k");
    return {t.data_ptr(), t.stride(0), t.stride(1)};
}
// What both directions have in common.
struct Rope {
    at::Tensor q, k, wq, wk, inv_freq, positions;
    int64_t tokens;
    int q_heads, k_heads, dim, rot, dt;
};
Rope rope_args(const OnDevice& on, PyObject* const* a) {
    Rope r{optional(a[0], "q"), optional(a[1], "k"), optional(a[2], "wq"), optional(a[3], "wk"), tensor(a[4], "inv_freq"), optional(a[5], "positions")};
    const at::Tensor& any = r.q.defined() ? r.q : r.k;
    r.dt = dtype_code(any);
    if (any.dim() != 3) value_error("q and k must be [tokens, heads, dim]");
    if (r.k.defined() && r.q.defined()) {
        on.check(r.k, "k", r.q.scalar_type(), 3, false);
        if (r.k.size(0) != r.q.size(0) || r.k.size(2) != r.q.size(2)) value_error("q and k must have the same tokens and dim");
    }
    r.tokens = any.size(0);
    const int64_t dim = any.size(2), q_heads = r.q.defined() ? r.q.size(1) : 0, k_heads = r.k.defined() ? r.k.size(1) : 0;
    on.check(r.wq, "wq", any.scalar_type(), 1, true);
    on.check(r.wk, "wk", any.scalar_type(), 1, true);
    on.check(r.inv_freq, "inv_freq", at::kFloat, 1, true);
    on.check(r.positions, "positions", at::kLong, 1, true);
    if ((r.wq.defined() && r.wq.size(0) != dim) || (r.wk.defined() && r.wk.size(0) != dim)) value_error("wq and wk must be [dim]");
    if (r.positions.defined() && r.positions.size(0) != r.tokens) value_error("positions must be [tokens]");
    if (dim > INT32_MAX || q_heads > INT32_MAX || k_heads > INT32_MAX || r.inv_freq.size(0) > INT32_MAX / 2) value_error("q, k or inv_freq: too large");
    r.dim = static_cast<int>(dim);
    r.q_heads = static_cast<int>(q_heads);
    r.k_heads = static_cast<int>(k_heads);
    r.rot = static_cast<int>(2 * r.inv_freq.size(0));
    return r;
}
const at::Tensor& first_of(PyObject* a, PyObject* b) { return a == Py_None ? tensor(b, "q or k") : tensor(a, "q"); }

// 0 q, 1 k, 2 wq, 3 wk, 4 inv_freq, 5 positions, 6 style, 7 eps, 8 q_out, 9 k_out, 10 stream, 11 prepare
PyObject* qk_fwd(PyObject* const* a) {
    const OnDevice on(first_of(a[0], a[1]), "q");
    const Rope r = rope_args(on, a);
    const int style = int_of(a[6], "style");
    const double eps = real(a[7]);
    at::Tensor qo = optional(a[8], "q_out"), ko = optional(a[9], "k_out");
    if (!qo.defined() && r.q.defined()) qo = output(r.q.sizes(), r.q.scalar_type(), r.q, a[10]);
    if (!ko.defined() && r.k.defined()) ko = output(r.k.sizes(), r.k.scalar_type(), r.k, a[10]);
    const Stream st = stream_of(a[10]);
    auto f = [=, q = heads_of(on, r.q, "q", r.q), k = heads_of(on, r.k, "k", r.k), xq = heads_of(on, qo, "q_out", r.q), xk = heads_of(on, ko, "k_out", r.k),
              wq = ptr(r.wq), wk = ptr(r.wk), pos = static_cast<const int64_t*>(ptr(r.positions)), fr = static_cast<const float*>(ptr(r.inv_freq)),
              tokens = r.tokens, hq = r.q_heads, hk = r.k_heads, dim = r.dim, rot = r.rot, dt = r.dt, s = st.s] {
        return pf_qk_norm_rope_fwd(q.p, q.ld, q.s, k.p, k.ld, k.s, wq, wk, pos, fr, xq.p, xq.ld, xq.s, xk.p, xk.ld, xk.s, tokens, hq, hk, dim, rot, style,
                                   eps, dt, s);
    };
    const bool prepare = truth(a[11]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {r.q, r.k, r.wq, r.wk, r.inv_freq, r.positions, qo, ko};
    return issue_on(on, prepare, f, "pf_qk_norm_rope_fwd", Workspace(), std::move(keep), tuple({qo, ko}));
}

// 0 q, 1 k, 2 wq, 3 wk, 4 inv_freq, 5 positions, 6 style, 7 eps, 8 dq_out, 9 dk_out, 10 dq, 11 dk, 12 need_dw, 13 dwq, 14 dwk, 15 accumulate,
// 16 grads_f32, 17 workspace, 18 stream, 19 prepare
PyObject* qk_bwd(PyObject* const* a) {
    const OnDevice on(first_of(a[0], a[1]), "q");
    const Rope r = rope_args(on, a);
    const at::Tensor& any = r.q.defined() ? r.q : r.k;
    const int style = int_of(a[6], "style");
    const double eps = real(a[7]);
    const at::Tensor gq = optional(a[8], "dq_out"), gk = optional(a[9], "dk_out");
    if (gq.defined() != r.q.defined() || gk.defined() != r.k.defined()) value_error("dq_out goes with q, dk_out with k");
    at::Tensor dq = optional(a[10], "dq"), dk = optional(a[11], "dk"), dwq = optional(a[13], "dwq"), dwk = optional(a[14], "dwk");
    if (!dq.defined() && r.q.defined()) dq = output(r.q.sizes(), any.scalar_type(), any, a[18]);
    if (!dk.defined() && r.k.defined()) dk = output(r.k.sizes(), any.scalar_type(), any, a[18]);
    const unsigned flags = grad_flags(a[15], a[16]);
    const at::ScalarType wdt = (flags & PF_GRAD_F32) ? at::kFloat : any.scalar_type();
    if (truth(a[12])) {
        if ((flags & PF_GRAD_ACCUMULATE) && ((r.q_heads > 0 && r.wq.defined() && !dwq.defined()) || (r.k_heads > 0 && r.wk.defined() && !dwk.defined())))
            value_error("accumulate=True needs the dwq and dwk to add to");
        if (!dwq.defined() && r.q_heads > 0 && r.wq.defined()) dwq = output({r.dim}, wdt, any, a[18]);
        if (!dwk.defined() && r.k_heads > 0 && r.wk.defined()) dwk = output({r.dim}, wdt, any, a[18]);
    }
    on.check(dwq, "dwq", wdt, 1, true);
    on.check(dwk, "dwk", wdt, 1, true);
    if ((dwq.defined() && dwq.size(0) != r.dim) || (dwk.defined() && dwk.size(0) != r.dim)) value_error("dwq and dwk must be [dim]");
    const Stream st = stream_of(a[18]);
    Workspace ws;
    if (a[17] != Py_None || dwq.defined() || dwk.defined())
        ws = workspace(a[17], a[17] == Py_None ? pf_qk_norm_rope_bwd_workspace(r.tokens, r.q_heads, r.k_heads, r.dim) : 0, any, st);
    auto f = [=, q = heads_of(on, r.q, "q", r.q), k = heads_of(on, r.k, "k", r.k), yq = heads_of(on, gq, "dq_out", r.q), yk = heads_of(on, gk, "dk_out", r.k),
              xq = heads_of(on, dq, "dq", r.q), xk = heads_of(on, dk, "dk", r.k), wq = ptr(r.wq), wk = ptr(r.wk),
              pos = static_cast<const int64_t*>(ptr(r.positions)), fr = static_cast<const float*>(ptr(r.inv_freq)), pwq = ptr(dwq), pwk = ptr(dwk),
              tokens = r.tokens, hq = r.q_heads, hk = r.k_heads, dim = r.dim, rot = r.rot, dt = r.dt, wp = ws.p, wb = ws.bytes, s = st.s] {
        return pf_qk_norm_rope_bwd(q.p, q.ld, q.s, k.p, k.ld, k.s, wq, wk, pos, fr, yq.p, yq.ld, yq.s, yk.p, yk.ld, yk.s, xq.p, xq.ld, xq.s, xk.p, xk.ld,
                                   xk.s, pwq, pwk, tokens, hq, hk, dim, rot, style, eps, dt, flags, wp, wb, s);
    };
    const bool prepare = truth(a[19]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {r.q, r.k, r.wq, r.wk, r.inv_freq, r.positions, gq, gk, dq, dk, dwq, dwk};
    return issue_on(on, prepare, f, "pf_qk_norm_rope_bwd", std::move(ws), std::move(keep), tuple({dq, dk, dwq, dwk}));
}

int32_t* ints(const at::Tensor& t) { return static_cast<int32_t*>(ptr(t)); }
float* floats(const at::Tensor& t) { return static_cast<float*>(ptr(t)); }
void expect(bool ok, const char* what) {
    if (!ok) value_error(what);
}
// A matrix argument [rows, cols] (rows and cols -1: any) of the call's dtype, at any pitch.
int64_t matrix(const OnDevice& on, const at::Tensor& t, const char* name, at::ScalarType type, int64_t rows, int64_t cols) {
    if (!t.defined()) return 0;
    on.check(t, name, type, 2, false);
    if ((rows >= 0 && t.size(0) != rows) || (cols >= 0 && t.size(1) != cols)) value_error(std::string(name) + ": does not fit the other matrices");
    return pitch(t, name);
}

// 0 ids, 1 experts, 2 capacity, 3 slots, 4 sources, 5 counts, 6 offsets, 7 workspace, 8 stream, 9 prepare
PyObject* expert_sort(PyObject* const* a) {
    const at::Tensor& ids = tensor(a[0], "ids");
    const OnDevice on(ids, "ids");
    on.check(ids, "ids", at::kInt, 2, true);
    const int experts = int_of(a[1], "experts");
    const int64_t capacity = integer(a[2]), tokens = ids.size(0);
    expect(ids.size(1) <= INT32_MAX, "ids: too large");
    const int k = static_cast<int>(ids.size(1));
    expect(experts >= 1 && experts < INT32_MAX && capacity >= 0 && capacity <= INT32_MAX && k >= 1,
           "need at least one expert and one choice, and a capacity from 0 on");
    if (pf_expert_rows(1, 1, experts, 0) == 0) check(PF_ERR_UNSUPPORTED, "pf_expert_sort");      // (before lists for so many are taken)
    const int64_t rows = pf_expert_rows(tokens, k, experts, capacity);
    at::Tensor slots = optional(a[3], "slots"), sources = optional(a[4], "sources"), counts = optional(a[5], "counts"), offsets = optional(a[6], "offsets");
    if (!slots.defined()) slots = output({tokens, k}, at::kInt, ids, a[8]);
    if (!sources.defined()) sources = output({rows}, at::kInt, ids, a[8]);
    if (!counts.defined()) counts = output({experts}, at::kInt, ids, a[8]);
    if (!offsets.defined()) offsets = output({experts + 1}, at::kInt, ids, a[8]);
    on.check(slots, "slots", at::kInt, 2, true);
    on.check(sources, "sources", at::kInt, 1, true);
    on.check(counts, "counts", at::kInt, 1, true);
    on.check(offsets, "offsets", at::kInt, 1, true);
    expect(slots.sizes() == ids.sizes() && sources.size(0) == rows && counts.size(0) == experts && offsets.size(0) == experts + 1,
           "slots must be as ids, sources [rows], counts [experts], offsets [experts + 1]");
    const Stream st = stream_of(a[8]);
    const size_t need = a[7] == Py_None ? pf_expert_sort_workspace(tokens, k, experts) : 0;
    Workspace ws;
    if (need > 0 || a[7] != Py_None) ws = workspace(a[7], need, ids, st);
    auto f = [=, pi = ints(ids), ps = ints(slots), pr = ints(sources), pc = ints(counts), po = ints(offsets), wp = ws.p, wb = ws.bytes, s = st.s] {
        return pf_expert_sort(pi, tokens, k, experts, capacity, ps, pr, pc, po, wp, wb, s);
    };
    const bool prepare = truth(a[9]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {ids, slots, sources, counts, offsets};
    return issue_on(on, prepare, f, "pf_expert_sort", std::move(ws), std::move(keep), tuple({slots, sources, counts, offsets}));
}

struct Choice {
    int64_t tokens;
    int k;
};
Choice choice(const OnDevice& on, const at::Tensor& slots, const at::Tensor& sources, int64_t rows) {
    on.check(slots, "slots", at::kInt, 2, true);
    on.check(sources, "sources", at::kInt, 1, true);
    expect(slots.size(1) <= INT32_MAX, "slots: too large");
    expect(!sources.defined() || sources.size(0) == rows, "sources: one for each row is needed");
    return {slots.size(0), static_cast<int>(slots.size(1))};
}

// 0 x, 1 slots, 2 sources, 3 xs, 4 stream, 5 prepare
PyObject* expert_dispatch_fwd(PyObject* const* a) {
    const at::Tensor& x = tensor(a[0], "x");
    const at::Tensor& slots = tensor(a[1], "slots");
    const at::Tensor& sources = tensor(a[2], "sources");
    const OnDevice on(x, "x");
    const int dt = dtype_code(x);
    expect(sources.dim() == 1, "sources: need [rows]");
    const int64_t rows = sources.size(0);
    const Choice c = choice(on, slots, sources, rows);
    const int64_t ldx = matrix(on, x, "x", x.scalar_type(), c.tokens, -1), width = x.size(1);
    at::Tensor xs = optional(a[3], "xs");
    if (!xs.defined()) xs = output({rows, width}, x.scalar_type(), x, a[4]);
    const int64_t ldxs = matrix(on, xs, "xs", x.scalar_type(), rows, width);
    const Stream st = stream_of(a[4]);
    auto f = [=, px = ptr(x), ps = ints(slots), pr = ints(sources), py = ptr(xs), s = st.s] {
        return pf_expert_dispatch_fwd(px, ldx, ps, pr, py, ldxs, c.tokens, c.k, rows, width, dt, s);
    };
    const bool prepare = truth(a[5]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {x, slots, sources, xs};
    return issue_on(on, prepare, f, "pf_expert_dispatch_fwd", Workspace(), std::move(keep), wrap(xs));
}

// 0 ys (dxs), 1 slots, 2 weights (None: ones), 3 y (dx), 4 stream, 5 prepare, 6 backward of dispatch
PyObject* expert_combine_fwd(PyObject* const* a) {
    const bool backward = truth(a[6]);
    const at::Tensor& ys = tensor(a[0], backward ? "dxs" : "ys");
    const at::Tensor& slots = tensor(a[1], "slots");
    const at::Tensor weights = optional(a[2], "weights");
    const OnDevice on(ys, backward ? "dxs" : "ys");
    const int dt = dtype_code(ys);
    const int64_t ldys = matrix(on, ys, backward ? "dxs" : "ys", ys.scalar_type(), -1, -1), rows = ys.size(0), width = ys.size(1);
    const Choice c = choice(on, slots, at::Tensor(), rows);
    on.check(weights, "weights", at::kFloat, 2, true);
    expect(!weights.defined() || weights.sizes() == slots.sizes(), "weights must be as slots");
    at::Tensor y = optional(a[3], backward ? "dx" : "y");
    if (!y.defined()) y = output({c.tokens, width}, ys.scalar_type(), ys, a[4]);
    const int64_t ldy = matrix(on, y, backward ? "dx" : "y", ys.scalar_type(), c.tokens, width);
    const Stream st = stream_of(a[4]);
    auto f = [=, py = ptr(ys), ps = ints(slots), pw = floats(weights), po = ptr(y), s = st.s] {
        return backward ? pf_expert_dispatch_bwd(py, ldys, ps, po, ldy, c.tokens, c.k, rows, width, dt, s)
                        : pf_expert_combine_fwd(py, ldys, ps, pw, po, ldy, c.tokens, c.k, rows, width, dt, s);
    };
    const bool prepare = truth(a[5]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {ys, slots, weights, y};
    return issue_on(on, prepare, f, backward ? "pf_expert_dispatch_bwd" : "pf_expert_combine_fwd", Workspace(), std::move(keep), wrap(y));
}

// 0 ys, 1 slots, 2 sources, 3 weights, 4 dy, 5 need_dys, 6 dys, 7 need_dweights, 8 dweights, 9 stream, 10 prepare
PyObject* expert_combine_bwd(PyObject* const* a) {
    const at::Tensor& ys = tensor(a[0], "ys");
    const at::Tensor& slots = tensor(a[1], "slots");
    const at::Tensor& sources = tensor(a[2], "sources");
    const at::Tensor& weights = tensor(a[3], "weights");
    const at::Tensor& dy = tensor(a[4], "dy");
    const OnDevice on(ys, "ys");
    const int dt = dtype_code(ys);
    const int64_t ldys = matrix(on, ys, "ys", ys.scalar_type(), -1, -1), rows = ys.size(0), width = ys.size(1);
    const Choice c = choice(on, slots, sources, rows);
    on.check(weights, "weights", at::kFloat, 2, true);
    expect(weights.sizes() == slots.sizes(), "weights must be as slots");
    const int64_t lddy = matrix(on, dy, "dy", ys.scalar_type(), c.tokens, width);
    at::Tensor dys = optional(a[6], "dys"), dw = optional(a[8], "dweights");
    if (!dys.defined() && truth(a[5])) dys = output({rows, width}, ys.scalar_type(), ys, a[9]);
    if (!dw.defined() && truth(a[7])) dw = output(slots.sizes(), at::kFloat, ys, a[9]);
    const int64_t lddys = matrix(on, dys, "dys", ys.scalar_type(), rows, width);
    on.check(dw, "dweights", at::kFloat, 2, true);
    expect(!dw.defined() || dw.sizes() == slots.sizes(), "dweights must be as slots");
    const Stream st = stream_of(a[9]);
    auto f = [=, py = ptr(ys), ps = ints(slots), pr = ints(sources), pw = floats(weights), pg = ptr(dy), pd = ptr(dys), pdw = floats(dw), s = st.s] {
        return pf_expert_combine_bwd(py, ldys, ps, pr, pw, pg, lddy, pd, lddys, pdw, c.tokens, c.k, rows, width, dt, s);
    };
    const bool prepare = truth(a[10]);
    std::vector<at::Tensor> keep;
    if (prepare) keep = {ys, slots, sources, weights, dy, dys, dw};
    return issue_on(on, prepare, f, "pf_expert_combine_bwd", Workspace(), std::move(keep), tuple({dys, dw}));
}

// The contiguous tensors of a list that goes with the parameters: numels[i] elements each, or one for each 256 of them.
template <typename P>
std::vector<P> array_list(PyObject* seq, const char* name, const OnDevice& on, at::ScalarType type, const std::vector<int64_t>& numels, bool scales,
                          std::vector<at::Tensor>* keep) {
    std::vector<P> out;
    if (seq == Py_None) return out;
    PyObject* fast = PySequence_Fast(seq, "need sequences of tensors");
    if (!fast) throw python_error();
    struct Drop { PyObject* o; ~Drop() { Py_DECREF(o); } } drop{fast};
    const size_t n = static_cast<size_t>(PySequence_Fast_GET_SIZE(fast));
    if (n != numels.size()) value_error(std::string(name) + ": need one tensor for each parameter");
    out.resize(n);
    for (size_t i = 0; i < n; ++i) {
        const at::Tensor& t = tensor(PySequence_Fast_GET_ITEM(fast, static_cast<Py_ssize_t>(i)), name);
        if (t.device() != on.device || t.scalar_type() != type || !t.is_contiguous() || t.numel() != (scales ? (numels[i] + 255) / 256 : numels[i]))
            value_error(std::string(name) + ": need contiguous " + c10::toString(type) + " tensors on " + on.device.str() +
                        (scales ? " of one element for each 256 of the parameter" : " of as many elements as the parameter"));
        out[i] = static_cast<P>(t.data_ptr());
        if (keep) keep->push_back(t);
    }
    return out;
}

// 0 params (not empty), 1 grads, 2 m, 3 v, 4 masters, 5 m_scales, 6 v_scales, 7 lr, 8 beta1, 9 beta2, 10 eps, 11 weight_decay, 12 step, 13 grad_scale,
// 14 seed, 15 scalars, 16 stream, 17 prepare
PyObject* adamw_step(PyObject* const* a) {
    PyObject* fast = PySequence_Fast(a[0], "params: need a sequence of tensors");
    if (!fast) throw python_error();
    struct Drop { PyObject* o; ~Drop() { Py_DECREF(o); } } drop{fast};
    const Py_ssize_t count = PySequence_Fast_GET_SIZE(fast);
    const at::Tensor& first = tensor(PySequence_Fast_GET_ITEM(fast, 0), "params");
    const OnDevice on(first, "params");
    const int pdt = dtype_code(first);
    std::vector<int64_t> n(static_cast<size_t>(count));
    for (Py_ssize_t i = 0; i < count; ++i) n[i] = tensor(PySequence_Fast_GET_ITEM(fast, i), "params").numel();
    auto first_type = [&](PyObject* seq, const char* name) {
        PyObject* o = PySequence_GetItem(seq, 0);
        if (!o) throw python_error();
        struct Hold { PyObject* o; ~Hold() { Py_DECREF(o); } } hold{o};
        return tensor(o, name).scalar_type();
    };
    const at::ScalarType gt = first_type(a[1], "grads"), mt = first_type(a[2], "m");
    if (gt != at::kFloat && gt != at::kBFloat16) throw PyError{PyExc_TypeError, std::string("grads: unsupported dtype ") + c10::toString(gt)};
    const bool state8 = mt == at::kFloat8_e4m3fn;
    if (!state8 && mt != at::kFloat) throw PyError{PyExc_TypeError, std::string("m: unsupported dtype ") + c10::toString(mt)};
    if (state8 != (a[5] != Py_None) || state8 != (a[6] != Py_None)) value_error("m_scales and v_scales go with states in 8 bits (m float8_e4m3fn, v float8_e5m2)");
    if (a[4] != Py_None && pdt != PF_BF16) value_error("masters go with bfloat16 parameters");
    const bool prepare = truth(a[17]);
    std::vector<at::Tensor> keep;
    std::vector<at::Tensor>* const k = prepare ? &keep : nullptr;
    auto params = array_list<void*>(fast, "params", on, first.scalar_type(), n, false, k);
    auto grads = array_list<const void*>(a[1], "grads", on, gt, n, false, k);
    auto m = array_list<void*>(a[2], "m", on, mt, n, false, k);
    auto v = array_list<void*>(a[3], "v", on, state8 ? at::kFloat8_e5m2 : at::kFloat, n, false, k);
    auto masters = array_list<float*>(a[4], "masters", on, at::kFloat, n, false, k);
    auto ms = array_list<float*>(a[5], "m_scales", on, at::kFloat, n, true, k);
    auto vs = array_list<float*>(a[6], "v_scales", on, at::kFloat, n, true, k);
    if (v.empty()) value_error("v: need one tensor for each parameter");
    pf_adamw h;
    h.lr = real(a[7]); h.beta1 = real(a[8]); h.beta2 = real(a[9]); h.eps = real(a[10]); h.weight_decay = real(a[11]);
    h.step = integer(a[12]);
    h.grad_scale = static_cast<float>(real(a[13]));
    const int64_t seed = integer(a[14]);
    if (seed < 0 || seed > 0xffffffffLL) value_error("seed: need 0 .. 2^32 - 1");
    h.seed = static_cast<uint32_t>(seed);
    const at::Tensor scalars = optional(a[15], "scalars");
    on.check(scalars, "scalars", at::kFloat, 1, true);
    if (scalars.defined() && scalars.size(0) != 5) value_error("scalars: need the five of pf_adamw_scalars");
    if (prepare && scalars.defined()) keep.push_back(scalars);
    const Stream st = stream_of(a[16]);
    const int gdt = gt == at::kBFloat16 ? PF_BF16 : PF_F32, state = state8 ? PF_STATE_8BIT : PF_STATE_F32, c = static_cast<int>(count);
    auto f = [=, params = std::move(params), grads = std::move(grads), m = std::move(m), v = std::move(v), masters = std::move(masters), ms = std::move(ms),
              vs = std::move(vs), n = std::move(n), sc = static_cast<const pf_adamw_scalars*>(ptr(scalars)), s = st.s] {
        return pf_adamw_step(params.data(), masters.empty() ? nullptr : masters.data(), grads.data(), m.data(), v.data(), ms.empty() ? nullptr : ms.data(),
                             vs.empty() ? nullptr : vs.data(), n.data(), c, pdt, gdt, state, &h, sc, s);
    };
    Py_INCREF(Py_None);
    return issue_on(on, prepare, std::move(f), "pf_adamw_step", Workspace(), std::move(keep), Py_None);
}

PyObject* set_error(PyObject*, PyObject* cls) {
    Py_INCREF(cls);
    Py_XSETREF(g_pf_error, cls);
    Py_RETURN_NONE;
}

#define PF_ENTRY(name, args) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<name, args>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {PF_ENTRY(linear_fwd, 12), PF_ENTRY(linear_fwd_static, 6), PF_ENTRY(linear_bwd, 14), PF_ENTRY(bias_act_bwd, 7),
                           PF_ENTRY(grouped_fwd, 9), PF_ENTRY(grouped_bwd, 12), PF_ENTRY(conv_fwd, 11), PF_ENTRY(conv_bwd, 16),
                           PF_ENTRY(pack, 4), PF_ENTRY(unpack, 3), PF_ENTRY(qk_fwd, 12), PF_ENTRY(qk_bwd, 20),
                           PF_ENTRY(expert_sort, 10), PF_ENTRY(expert_dispatch_fwd, 6), PF_ENTRY(expert_combine_fwd, 7), PF_ENTRY(expert_combine_bwd, 11),
                           PF_ENTRY(adamw_step, 18), {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_pf_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pf_native(void) {
    g_prepared_type = reinterpret_cast<PyTypeObject*>(PyType_FromSpec(&g_prepared_spec));
    if (!g_prepared_type) return nullptr;
    return PyModule_Create(&g_module);
}
