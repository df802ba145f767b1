// Native half of the Python binding: argument checks, output allocation and the call into the C ABI, without the interpreter.
//
// A decode step of one sequence runs for about 3 us on the device; marshalled in Python (descriptor fields through ctypes,
// device and stream context managers, a dozen attribute reads) the call took 16 us of host time, which was then also what a
// batch of 64 sequences took (8.6 us on the device).  Semantics are those of binding.py's docstrings: CUDA, contiguous tensors
// (ValueError), dtypes (TypeError), KlaError for a non-zero status, the current stream of q's device, outputs allocated from
// torch's caching allocator.  No arithmetic happens here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <c10/cuda/CUDAException.h>
#include <c10/cuda/CUDAGraphsC10Utils.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <initializer_list>
#include <utility>
#include <vector>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "kla.h"

namespace {

PyObject *g_kla_error = nullptr;   // binding.KlaError
PyObject *g_status_for = nullptr;  // binding._status_for: the binding's own status word of a device

struct Failed {};   // a Python exception has been set

[[noreturn]] void fail(PyObject *type, const char *msg, const char *name = nullptr)
{
    if (name) PyErr_Format(type, "%s %s", name, msg);
    else PyErr_SetString(type, msg);
    throw Failed();
}

const at::Tensor *opt_tensor(PyObject *o, const char *name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) fail(PyExc_ValueError, "must be a contiguous CUDA tensor", name);
    return &THPVariable_Unpack(o);
}
const at::Tensor &tensor(PyObject *o, const char *name)
{
    const at::Tensor *t = opt_tensor(o, name);
    if (!t) fail(PyExc_ValueError, "must be a tensor", name);
    return *t;
}
// device address of a contiguous CUDA tensor (null for none), as binding._dev
void *addr(const at::Tensor *t, const char *name)
{
    if (!t) return nullptr;
    if (!t->is_cuda() || !t->is_contiguous()) fail(PyExc_ValueError, "must be a contiguous CUDA tensor", name);
    return t->data_ptr();
}
float *addr_f32(const at::Tensor *t, const char *name)
{
    void *p = addr(t, name);
    if (t && t->scalar_type() != at::kFloat) fail(PyExc_TypeError, "must be torch.float32", name);
    return static_cast<float *>(p);
}
int32_t kla_dtype_of(const at::Tensor &t)
{
    if (t.scalar_type() == at::kFloat) return KLA_F32;
    if (t.scalar_type() == at::kBFloat16) return KLA_BF16;
    fail(PyExc_TypeError, "q, k, v, out must be float32 or bfloat16");
}
at::ScalarType dtype_arg(PyObject *o, const at::Tensor &like)
{
    if (o == Py_None) return like.scalar_type();
    if (!THPDtype_Check(o)) fail(PyExc_TypeError, "out_dtype must be a torch.dtype");
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}
double number(PyObject *o)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Failed();
    return x;
}
long integer(PyObject *o)
{
    const long x = PyLong_AsLong(o);
    if (x == -1 && PyErr_Occurred()) throw Failed();
    return x;
}
// Larger buffers than a call needs are the caller's business; smaller ones would be read or written past their end.
void holds(const at::Tensor *t, int64_t n, const char *name)
{
    if (t && t->numel() < n) fail(PyExc_ValueError, "holds fewer elements than the call takes", name);
}
void one_dtype(const at::Tensor &q, const at::Tensor &k, const at::Tensor &v)
{
    if (k.scalar_type() != q.scalar_type() || v.scalar_type() != q.scalar_type()) fail(PyExc_TypeError, "q, k, v must share one dtype");
}
// Packed input: the host copy of the offsets, contiguous, and the number of sequences.
at::Tensor offsets(const at::Tensor &cu, PyObject *host_seqlens, int64_t *n_seq)
{
    if (cu.scalar_type() != at::kInt) fail(PyExc_TypeError, "cu_seqlens must be int32");
    const at::Tensor &host = tensor(host_seqlens, "host_seqlens");
    if (host.is_cuda() || host.scalar_type() != at::kInt) fail(PyExc_TypeError, "host_seqlens must be a CPU int32 tensor");
    *n_seq = cu.numel() - 1;
    holds(&host, *n_seq + 1, "host_seqlens");
    return host.contiguous();
}
bool has_shape(const at::Tensor &t, at::IntArrayRef shape) { return t.sizes() == shape; }

// The status word of a call: the caller's, else the binding's own of the device (kept alive by the binding).
int32_t *status_word(PyObject *given, c10::Device device)
{
    PyObject *o = given;   // borrowed
    if (o == Py_None) {
        PyObject *dev = PyLong_FromLong(device.index());
        o = dev ? PyObject_CallOneArg(g_status_for, dev) : nullptr;
        Py_XDECREF(dev);
        if (!o) throw Failed();
        Py_DECREF(o);
    }
    const at::Tensor &t = tensor(o, "status_word");
    void *p = addr(&t, "status_word");
    if (t.scalar_type() != at::kInt) fail(PyExc_TypeError, "must be torch.int32", "status_word");
    return static_cast<int32_t *>(p);
}

void check(kla_status st)
{
    if (st == KLA_OK) return;
    PyObject *e = PyObject_CallFunction(g_kla_error, "is", (int)st, kla_status_str(st));
    if (e) {
        PyErr_SetObject(g_kla_error, e);
        Py_DECREF(e);
    }
    throw Failed();
}

// kla_decode_step / kla_decode_steps / kla_dg_decode_step:
// (q, k, v, log_alpha, eta, eps, state_inout, out, out_dtype, flags, kind)   kind 0: one step, 1: steps, 2: diagonal gates
PyObject *decode(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 11) {
        PyErr_SetString(PyExc_TypeError, "decode: 11 arguments");
        return nullptr;
    }
    try {
        const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
        const at::Tensor &la = tensor(a[3], "log_alpha"), &eta = tensor(a[4], "eta"), &state = tensor(a[6], "state_inout");
        const float eps = (float)number(a[5]);
        const long kind = integer(a[10]);
        const int lead = kind == 1 ? 1 : 0;
        if (q.dim() != 3 + lead || v.dim() < 1) fail(PyExc_ValueError, lead ? "q must be [n, B, H, d_k]" : "q must be [B, H, d_k]");
        const int64_t steps = lead ? q.size(0) : 1, B = q.size(lead), H = q.size(lead + 1), d_k = q.size(-1), d_v = v.size(-1);
        const at::Tensor *given = opt_tensor(a[7], "out");
        one_dtype(q, k, v);
        const int64_t units = steps * B * H;
        holds(&k, units * d_k, "k");
        holds(&v, units * d_v, "v");
        holds(&la, kind == 2 ? units * d_k : units, "log_alpha");
        holds(&eta, units, "eta");
        holds(&state, B * H * d_k * d_v, "state_inout");
        holds(given, units * d_v, "out");
        void *qa = addr(&q, "q");
        const c10::cuda::OptionalCUDAGuard guard(q.device());
        at::Tensor out;
        if (given) out = *given;
        else if (lead) out = at::empty({steps, B, H, d_v}, q.options().dtype(dtype_arg(a[8], q)));
        else out = at::empty({B, H, d_v}, q.options().dtype(dtype_arg(a[8], q)));
        kla_desc d = {};
        d.B = d.n_seq = (int32_t)B;
        d.T = 1;
        d.H = (int32_t)H;
        d.d_k = (int32_t)d_k;
        d.d_v = (int32_t)d_v;
        d.io_dtype = kla_dtype_of(q);
        d.out_dtype = kla_dtype_of(out);
        d.flags = (int32_t)integer(a[9]);
        d.stream = c10::cuda::getCurrentCUDAStream(q.device().index()).stream();
        void *ka = addr(&k, "k"), *va = addr(&v, "v"), *oa = addr(&out, "out");
        float *laa = addr_f32(&la, "log_alpha"), *ea = addr_f32(&eta, "eta"), *sa = addr_f32(&state, "state_inout");
        kla_status st;
        Py_BEGIN_ALLOW_THREADS
        st = kind == 2 ? kla_dg_decode_step(&d, qa, ka, va, laa, ea, eps, sa, oa) : kla_decode_steps(&d, (int32_t)steps, qa, ka, va, laa, ea, eps, sa, oa);
        Py_END_ALLOW_THREADS
        check(st);
        if (given) {
            Py_INCREF(a[7]);
            return a[7];
        }
        return THPVariable_Wrap(std::move(out));
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// kla_chunk_fwd (dg = 0) and kla_dg_fwd (dg = 1), without the measurement aids of binding.kla_chunk_fwd:
// (q, k, v, log_alpha, eta, eps, chunk, init_state, out, final_state, cu_seqlens, host_seqlens, out_dtype, flags,
//  want_final_state, status_word, dg) -> (out, final_state)
PyObject *forward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 17) {
        PyErr_SetString(PyExc_TypeError, "forward: 17 arguments");
        return nullptr;
    }
    try {
        const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
        const at::Tensor &la = tensor(a[3], "log_alpha"), &eta = tensor(a[4], "eta");
        const float eps = (float)number(a[5]);
        const int32_t chunk = (int32_t)integer(a[6]);
        const bool dg = integer(a[16]) != 0;
        if (q.dim() != 4 || v.dim() < 1) fail(PyExc_ValueError, "q must be [B, T, H, d_k]");
        const int64_t B = q.size(0), T = q.size(1), H = q.size(2), d_k = q.size(3), d_v = v.size(-1);
        if (!has_shape(k, q.sizes()) || !has_shape(v, {B, T, H, d_v})) fail(PyExc_ValueError, "q, k, v shapes disagree");
        if (!has_shape(eta, {B, T, H}) || !(dg ? has_shape(la, {B, T, H, d_k}) : has_shape(la, {B, T, H})))
            fail(PyExc_ValueError, dg ? "log_alpha must be [B, T, H, d_k] and eta [B, T, H]" : "log_alpha, eta must be [B, T, H]");
        one_dtype(q, k, v);
        int64_t n_seq = B;
        const at::Tensor *cu = opt_tensor(a[10], "cu_seqlens");
        at::Tensor host;
        if (cu) host = offsets(*cu, a[11], &n_seq);
        const at::Tensor *out_given = opt_tensor(a[8], "out"), *fin_given = opt_tensor(a[9], "final_state"), *init = opt_tensor(a[7], "init_state");
        holds(out_given, B * T * H * d_v, "out");
        holds(fin_given, n_seq * H * d_k * d_v, "final_state");
        void *qa = addr(&q, "q");
        const c10::cuda::OptionalCUDAGuard guard(q.device());
        at::Tensor out, fin, ws;
        if (out_given) out = *out_given;
        else out = at::empty({B, T, H, d_v}, q.options().dtype(dtype_arg(a[12], q)));
        if (fin_given) fin = *fin_given;
        else if (integer(a[14])) fin = at::empty({n_seq, H, d_k, d_v}, q.options().dtype(at::kFloat));
        if (init && !has_shape(*init, {n_seq, H, d_k, d_v})) fail(PyExc_ValueError, "init_state must be [n_seq, H, d_k, d_v]");
        kla_desc d = {};
        d.B = (int32_t)B;
        d.T = (int32_t)T;
        d.H = (int32_t)H;
        d.d_k = (int32_t)d_k;
        d.d_v = (int32_t)d_v;
        d.n_seq = (int32_t)n_seq;
        d.cu_seqlens = static_cast<const int32_t *>(addr(cu, "cu_seqlens"));
        d.host_seqlens = cu ? static_cast<const int32_t *>(host.data_ptr()) : nullptr;
        d.io_dtype = kla_dtype_of(q);
        d.out_dtype = kla_dtype_of(out);
        d.flags = (int32_t)integer(a[13]);
        d.stream = c10::cuda::getCurrentCUDAStream(q.device().index()).stream();
        if (!dg) d.status_word = status_word(a[15], q.device());   // (kernels of diagonal gates wait for nothing)
        if (!dg) {
            if (const size_t need = kla_chunk_fwd_workspace_bytes(&d, chunk)) {
                ws = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
                d.workspace = ws.data_ptr();
                d.workspace_bytes = need;
            }
        }
        void *ka = addr(&k, "k"), *va = addr(&v, "v"), *oa = addr(&out, "out");
        float *laa = addr_f32(&la, "log_alpha"), *ea = addr_f32(&eta, "eta"), *ia = addr_f32(init, "init_state");
        float *fa = fin.defined() ? addr_f32(&fin, "final_state") : nullptr;
        kla_status st;
        Py_BEGIN_ALLOW_THREADS
        st = dg ? kla_dg_fwd(&d, qa, ka, va, laa, ea, eps, ia, oa, fa) : kla_chunk_fwd(&d, qa, ka, va, laa, ea, eps, chunk, ia, oa, fa);
        Py_END_ALLOW_THREADS
        check(st);
        PyObject *po, *pf;
        if (out_given) Py_INCREF(po = a[8]);
        else po = THPVariable_Wrap(std::move(out));
        if (fin_given || !fin.defined()) Py_INCREF(pf = a[9]);   // (None when no final state is wanted)
        else pf = THPVariable_Wrap(std::move(fin));
        if (!po || !pf) {
            Py_XDECREF(po);
            Py_XDECREF(pf);
            return nullptr;
        }
        PyObject *r = PyTuple_New(2);
        PyTuple_SET_ITEM(r, 0, po);
        PyTuple_SET_ITEM(r, 1, pf);
        return r;
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// kla_bwd: (q, k, v, log_alpha, eta, eps, d_out, init_state, d_final_state, cu_seqlens, host_seqlens, flags, want_dinit_state,
// workspace, status_word) -> dict
PyObject *backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 15) {
        PyErr_SetString(PyExc_TypeError, "backward: 15 arguments");
        return nullptr;
    }
    try {
        const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
        const at::Tensor &la = tensor(a[3], "log_alpha"), &eta = tensor(a[4], "eta"), &d_out = tensor(a[6], "d_out");
        const float eps = (float)number(a[5]);
        if (q.dim() != 4 || v.dim() < 1) fail(PyExc_ValueError, "q must be [B, T, H, d_k]");
        const int64_t B = q.size(0), T = q.size(1), H = q.size(2), d_k = q.size(3), d_v = v.size(-1);
        if (!has_shape(d_out, {B, T, H, d_v}) || d_out.scalar_type() != q.scalar_type())
            fail(PyExc_ValueError, "d_out must be [B, T, H, d_v] with the dtype of q");
        one_dtype(q, k, v);
        int64_t n_seq = B;
        const at::Tensor *cu = opt_tensor(a[9], "cu_seqlens"), *init = opt_tensor(a[7], "init_state"), *dfin = opt_tensor(a[8], "d_final_state");
        const at::Tensor *given = opt_tensor(a[13], "workspace");
        at::Tensor host;
        if (cu) host = offsets(*cu, a[10], &n_seq);
        holds(&k, q.numel(), "k");
        holds(&v, B * T * H * d_v, "v");
        holds(&la, B * T * H, "log_alpha");
        holds(&eta, B * T * H, "eta");
        holds(init, n_seq * H * d_k * d_v, "init_state");
        holds(dfin, n_seq * H * d_k * d_v, "d_final_state");
        void *qa = addr(&q, "q");
        const c10::cuda::OptionalCUDAGuard guard(q.device());
        kla_desc d = {};
        d.B = (int32_t)B;
        d.T = (int32_t)T;
        d.H = (int32_t)H;
        d.d_k = (int32_t)d_k;
        d.d_v = (int32_t)d_v;
        d.n_seq = (int32_t)n_seq;
        d.cu_seqlens = static_cast<const int32_t *>(addr(cu, "cu_seqlens"));
        d.host_seqlens = cu ? static_cast<const int32_t *>(host.data_ptr()) : nullptr;
        d.io_dtype = kla_dtype_of(q);
        d.out_dtype = KLA_F32;
        d.flags = (int32_t)integer(a[11]);
        d.stream = c10::cuda::getCurrentCUDAStream(q.device().index()).stream();
        d.status_word = status_word(a[14], q.device());
        const auto f32 = q.options().dtype(at::kFloat);
        const bool want = PyObject_IsTrue(a[12]) == 1;
        at::Tensor g[6] = {at::empty({B, T, H, d_k}, f32), at::empty({B, T, H, d_k}, f32), at::empty({B, T, H, d_v}, f32),
                           at::empty({B, T, H}, f32), at::empty({B, T, H}, f32), want ? at::empty({n_seq, H, d_k, d_v}, f32) : at::Tensor()};
        at::Tensor ws;
        if (given) ws = *given;
        else if (const size_t need = kla_bwd_workspace_bytes(&d)) ws = at::empty({(int64_t)need}, q.options().dtype(at::kByte));
        if (ws.defined()) {
            d.workspace = addr(&ws, "workspace");
            d.workspace_bytes = (size_t)ws.numel() * ws.element_size();
        }
        void *ka = addr(&k, "k"), *va = addr(&v, "v"), *da = addr(&d_out, "d_out");
        float *laa = addr_f32(&la, "log_alpha"), *ea = addr_f32(&eta, "eta"), *ia = addr_f32(init, "init_state"), *fa = addr_f32(dfin, "d_final_state");
        float *ga[6];
        for (int i = 0; i < 6; ++i) ga[i] = g[i].defined() ? static_cast<float *>(g[i].data_ptr()) : nullptr;
        kla_status st;
        Py_BEGIN_ALLOW_THREADS
        st = kla_bwd(&d, qa, ka, va, laa, ea, eps, ia, da, fa, ga[0], ga[1], ga[2], ga[3], ga[4], ga[5]);
        Py_END_ALLOW_THREADS
        check(st);
        static const char *const names[6] = {"dq", "dk", "dv", "dlog_alpha", "deta", "dinit_state"};
        PyObject *r = PyDict_New();
        for (int i = 0; r && i < 6; ++i) {
            PyObject *o = g[i].defined() ? THPVariable_Wrap(std::move(g[i])) : (Py_INCREF(Py_None), Py_None);
            if (!o || PyDict_SetItemString(r, names[i], o) != 0) Py_CLEAR(r);
            Py_XDECREF(o);
        }
        return r;
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// ---- operators around a mixer ------------------------------------------------------------------------------------------------------

// Rows of a tensor whose last `inner` dimensions are dense and whose leading ones step uniformly: the address of the first row and
// the elements from one to the next.
void *row_addr(const at::Tensor &t, int inner, const char *name, int64_t *stride)
{
    if (!t.is_cuda()) fail(PyExc_ValueError, "must be a CUDA tensor", name);
    const int lead = (int)t.dim() - inner;
    int64_t dense = 1;
    for (int i = (int)t.dim() - 1; i >= lead; --i) {
        if (t.size(i) != 1 && t.stride(i) != dense) fail(PyExc_ValueError, "must have dense rows", name);
        dense *= t.size(i);
    }
    int64_t step = dense, rows = 1;
    bool first = true;
    for (int i = lead - 1; i >= 0; --i) {
        if (t.size(i) == 1) continue;
        if (first) step = t.stride(i);
        else if (t.stride(i) != step * rows) fail(PyExc_ValueError, "must have rows at one distance from each other", name);
        first = false;
        rows *= t.size(i);
    }
    *stride = step;
    return t.data_ptr();
}
void same_device(const at::Tensor &t, const at::Tensor &as, const char *name)
{
    if (t.device() != as.device()) fail(PyExc_ValueError, "must be on the device of the other tensors", name);
}
// An optional fp32 parameter vector.
float *param(const at::Tensor *t, const at::Tensor &x, at::IntArrayRef shape, const char *name)
{
    if (!t) return nullptr;
    if (!has_shape(*t, shape)) fail(PyExc_ValueError, "has another shape than the call takes", name);
    float *p = addr_f32(t, name);
    same_device(*t, x, name);
    return p;
}
// An optional dense array of the given shape and dtype.
void *array(const at::Tensor *t, const at::Tensor &x, at::IntArrayRef shape, at::ScalarType dtype, const char *name)
{
    if (!t) return nullptr;
    if (!has_shape(*t, shape)) fail(PyExc_ValueError, "has another shape than the call takes", name);
    if (t->scalar_type() != dtype) fail(PyExc_TypeError, "has another dtype than the call takes", name);
    void *p = addr(t, name);
    same_device(*t, x, name);
    return p;
}
at::ScalarType io_of(const at::Tensor &x, const char *name)
{
    if (x.scalar_type() != at::kFloat && x.scalar_type() != at::kBFloat16) fail(PyExc_TypeError, "must be float32 or bfloat16", name);
    return x.scalar_type();
}
int32_t dtype_code(at::ScalarType t) { return t == at::kFloat ? KLA_F32 : KLA_BF16; }
int32_t small(int64_t x)
{
    if (x < 0 || x > INT32_MAX) fail(PyExc_ValueError, "a size does not fit 32 bits");
    return (int32_t)x;
}

// Sequences of a call into its descriptor; `host` keeps the host offsets alive.
void sequences(kla_desc *d, const at::Tensor &x, PyObject *cu_seqlens, PyObject *host_seqlens, at::Tensor *host)
{
    int64_t n_seq = x.size(0);
    const at::Tensor *cu = opt_tensor(cu_seqlens, "cu_seqlens");
    if (cu) {
        *host = offsets(*cu, host_seqlens, &n_seq);
        d->cu_seqlens = static_cast<const int32_t *>(addr(cu, "cu_seqlens"));
        same_device(*cu, x, "cu_seqlens");
        d->host_seqlens = static_cast<const int32_t *>(host->data_ptr());
    }
    d->B = small(x.size(0));
    d->T = small(x.size(1));
    d->n_seq = small(n_seq);
}
kla_desc desc_of(const at::Tensor &x, at::ScalarType io, PyObject *flags)
{
    kla_desc d = {};
    d.io_dtype = d.out_dtype = dtype_code(io);
    d.flags = (int32_t)integer(flags);
    d.stream = c10::cuda::getCurrentCUDAStream(x.device().index()).stream();
    return d;
}
at::Tensor scratch(kla_desc *d, const at::Tensor &x, size_t need)
{
    at::Tensor ws;
    if (need) {
        ws = at::empty({(int64_t)need}, x.options().dtype(at::kByte));
        d->workspace = ws.data_ptr();
        d->workspace_bytes = need;
    }
    return ws;
}
PyObject *wrap(at::Tensor t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(t));
}
PyObject *pair(at::Tensor a, at::Tensor b)
{
    PyObject *x = wrap(std::move(a)), *y = x ? wrap(std::move(b)) : nullptr, *r = y ? PyTuple_New(2) : nullptr;
    if (!r) {
        Py_XDECREF(x);
        Py_XDECREF(y);
        return nullptr;
    }
    PyTuple_SET_ITEM(r, 0, x);
    PyTuple_SET_ITEM(r, 1, y);
    return r;
}
PyObject *dict(std::initializer_list<std::pair<const char *, at::Tensor>> items)
{
    PyObject *r = PyDict_New();
    for (const auto &it : items) {
        PyObject *o = r ? wrap(it.second) : nullptr;
        if (!o || PyDict_SetItemString(r, it.first, o) != 0) Py_CLEAR(r);
        Py_XDECREF(o);
    }
    return r;
}
// Runs `call` without the interpreter's lock, so that it must not raise, and raises for a status other than KLA_OK.
template <typename F>
void run(F call)
{
    kla_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    check(st);
}
template <typename F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, const char *name, F body)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "%s: %zd arguments", name, want);
        return nullptr;
    }
    try {
        return body();
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// What the three calls of the convolution share.
struct Conv {
    const at::Tensor &x, &weight;
    const at::Tensor *bias;
    at::ScalarType io;
    int64_t C, W, stride = 0;
    void *xa;
    float *wa, *ba;
    int32_t channels, taps;
    Conv(PyObject *x_, PyObject *w_, PyObject *b_, int dims) : x(tensor(x_, "x")), weight(tensor(w_, "weight")), bias(opt_tensor(b_, "bias"))
    {
        io = io_of(x, "x");
        if (x.dim() != dims) fail(PyExc_ValueError, dims == 2 ? "x must be [B, C]" : "x must be [B, T, C]");
        if (weight.dim() != 2 || weight.size(0) != x.size(-1)) fail(PyExc_ValueError, "weight must be [C, taps]");
        C = x.size(-1);
        W = weight.size(1);
        xa = row_addr(x, 1, "x", &stride);
        wa = param(&weight, x, {C, W}, "weight");
        ba = param(bias, x, {C}, "bias");
        channels = small(C);
        taps = small(W);
    }
};

// kla_conv_fwd: (x, weight, bias, init_state, out, final_state, cu_seqlens, host_seqlens, flags, want_final_state) -> (out, final_state)
PyObject *conv_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, "conv_fwd", [&]() -> PyObject * {
        const Conv c(a[0], a[1], a[2], 3);
        const c10::cuda::OptionalCUDAGuard guard(c.x.device());
        kla_desc d = desc_of(c.x, c.io, a[8]);
        at::Tensor host, out, fin;
        sequences(&d, c.x, a[6], a[7], &host);
        const std::vector<int64_t> state = {d.n_seq, c.W - 1, c.C};
        const at::Tensor *init = opt_tensor(a[3], "init_state"), *og = opt_tensor(a[4], "out"), *fg = opt_tensor(a[5], "final_state");
        void *ia = array(init, c.x, state, c.io, "init_state");
        if (og) out = *og;
        else out = at::empty(c.x.sizes(), c.x.options());
        if (fg) fin = *fg;
        else if (integer(a[9]) && c.W > 0) fin = at::empty(state, c.x.options());
        void *oa = array(&out, c.x, c.x.sizes(), c.io, "out"), *fa = fin.defined() ? array(&fin, c.x, state, c.io, "final_state") : nullptr;
        if (oa == c.xa && d.B > 0 && d.T > 0) fail(PyExc_ValueError, "must not be the input", "out");
        run([&] { return kla_conv_fwd(&d, c.channels, c.taps, c.xa, c.stride, c.wa, c.ba, ia, oa, fa); });
        return pair(out, fin);
    });
}

// kla_conv_step: (x, weight, state_inout, bias, out, flags) -> out
PyObject *conv_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 6, "conv_step", [&]() -> PyObject * {
        const Conv c(a[0], a[1], a[3], 2);
        const c10::cuda::OptionalCUDAGuard guard(c.x.device());
        kla_desc d = desc_of(c.x, c.io, a[5]);
        d.B = d.n_seq = small(c.x.size(0));
        d.T = 1;
        const at::Tensor &state = tensor(a[2], "state_inout"), *og = opt_tensor(a[4], "out");
        void *sa = array(&state, c.x, {c.x.size(0), c.W - 1, c.C}, c.io, "state_inout");
        at::Tensor out;
        if (og) out = *og;
        else out = at::empty(c.x.sizes(), c.x.options());
        void *oa = array(&out, c.x, c.x.sizes(), c.io, "out");
        run([&] { return kla_conv_step(&d, c.channels, c.taps, c.xa, c.stride, c.wa, c.ba, sa, oa); });
        return wrap(out);
    });
}

// kla_conv_bwd: (x, weight, d_out, bias, init_state, d_final_state, cu_seqlens, host_seqlens, flags, want_dinit_state) -> dict
PyObject *conv_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, "conv_bwd", [&]() -> PyObject * {
        const Conv c(a[0], a[1], a[3], 3);
        const c10::cuda::OptionalCUDAGuard guard(c.x.device());
        kla_desc d = desc_of(c.x, c.io, a[8]);
        at::Tensor host;
        sequences(&d, c.x, a[6], a[7], &host);
        const std::vector<int64_t> state = {d.n_seq, c.W - 1, c.C};
        const at::Tensor &dout = tensor(a[2], "d_out");
        void *ga = array(&dout, c.x, c.x.sizes(), c.io, "d_out");
        void *ia = array(opt_tensor(a[4], "init_state"), c.x, state, c.io, "init_state");
        void *fa = array(opt_tensor(a[5], "d_final_state"), c.x, state, c.io, "d_final_state");
        at::Tensor dx = at::empty(c.x.sizes(), c.x.options()), dw = at::empty({c.C, c.W}, c.weight.options()), db, di;
        if (c.ba) db = at::empty({c.C}, c.weight.options());
        if (integer(a[9]) && c.W > 0) di = at::empty(state, c.x.options());
        at::Tensor ws = scratch(&d, c.x, kla_conv_bwd_workspace_bytes(&d, c.channels, c.taps));
        run([&] {
            return kla_conv_bwd(&d, c.channels, c.taps, c.xa, c.stride, c.wa, c.ba, ia, ga, fa, dx.data_ptr(), dw.data_ptr<float>(),
                                db.defined() ? db.data_ptr<float>() : nullptr, di.defined() ? di.data_ptr() : nullptr);
        });
        return dict({{"dx", dx}, {"dweight", dw}, {"dbias", db}, {"dinit_state", di}});
    });
}

// What the three calls of the scan share: q, k, v, dt, a and d_skip.
struct Ssm {
    const at::Tensor &q, &k, &v, &dt, &a;
    const at::Tensor *skip;
    at::ScalarType io;
    int64_t H, G, N, P, qs = 0, ks = 0, vs = 0;
    void *qa, *ka, *va;
    float *dta, *aa, *sa;
    int32_t groups;
    std::vector<int64_t> state;   // shape, but for its first entry
    Ssm(PyObject *const *x, PyObject *skip_, int lead)
        : q(tensor(x[0], "q")), k(tensor(x[1], "k")), v(tensor(x[2], "v")), dt(tensor(x[3], "dt")), a(tensor(x[4], "a")), skip(opt_tensor(skip_, "d_skip"))
    {
        io = io_of(v, "v");
        if (v.dim() != lead + 2 || q.dim() != lead + 2) fail(PyExc_ValueError, lead == 1 ? "q must be [B, G, d_k] and v [B, H, d_v]" : "q must be [B, T, G, d_k] and v [B, T, H, d_v]");
        H = v.size(-2);
        P = v.size(-1);
        G = q.size(-2);
        N = q.size(-1);
        for (int i = 0; i < lead; ++i)
            if (q.size(i) != v.size(i)) fail(PyExc_ValueError, "q, k, v shapes disagree");
        if (!has_shape(k, q.sizes())) fail(PyExc_ValueError, "q, k, v shapes disagree");
        one_dtype(q, k, v);
        qa = row_addr(q, 2, "q", &qs);
        ka = row_addr(k, 2, "k", &ks);
        va = row_addr(v, 2, "v", &vs);
        same_device(q, v, "q");
        same_device(k, v, "k");
        dta = param(&dt, v, v.sizes().slice(0, lead + 1), "dt");
        aa = param(&a, v, {H}, "a");
        sa = param(skip, v, {H}, "d_skip");
        state = {0, H, N, P};
        groups = small(G);
    }
    void into(kla_desc *d)
    {
        d->H = small(H);
        d->d_k = small(N);
        d->d_v = small(P);
        state[0] = d->n_seq;
    }
};

// kla_ssm_fwd: (q, k, v, dt, a, d_skip, init_state, out, final_state, cu_seqlens, host_seqlens, out_dtype, flags, want_final_state,
// status_word) -> (out, final_state)
PyObject *ssm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 15, "ssm_fwd", [&]() -> PyObject * {
        Ssm s(a, a[5], 2);
        const c10::cuda::OptionalCUDAGuard guard(s.v.device());
        kla_desc d = desc_of(s.v, s.io, a[12]);
        at::Tensor host, out, fin;
        sequences(&d, s.v, a[9], a[10], &host);
        s.into(&d);
        void *ia = array(opt_tensor(a[6], "init_state"), s.v, s.state, at::kFloat, "init_state");
        const at::Tensor *og = opt_tensor(a[7], "out"), *fg = opt_tensor(a[8], "final_state");
        if (og) out = *og;
        else out = at::empty(s.v.sizes(), s.v.options().dtype(dtype_arg(a[11], s.v)));
        if (fg) fin = *fg;
        else if (integer(a[13])) fin = at::empty(s.state, s.v.options().dtype(at::kFloat));
        void *oa = array(&out, s.v, s.v.sizes(), io_of(out, "out"), "out"), *fa = fin.defined() ? array(&fin, s.v, s.state, at::kFloat, "final_state") : nullptr;
        d.out_dtype = dtype_code(out.scalar_type());
        d.status_word = status_word(a[14], s.v.device());
        at::Tensor ws = scratch(&d, s.v, kla_ssm_fwd_workspace_bytes(&d, s.groups));
        run([&] { return kla_ssm_fwd(&d, s.groups, s.qa, s.qs, s.ka, s.ks, s.va, s.vs, s.dta, s.aa, s.sa, static_cast<float *>(ia), oa, static_cast<float *>(fa)); });
        return pair(out, fin);
    });
}

// kla_ssm_step: (q, k, v, dt, a, state_inout, d_skip, out, out_dtype, flags) -> out
PyObject *ssm_step(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, "ssm_step", [&]() -> PyObject * {
        Ssm s(a, a[6], 1);
        const c10::cuda::OptionalCUDAGuard guard(s.v.device());
        kla_desc d = desc_of(s.v, s.io, a[9]);
        d.B = d.n_seq = small(s.v.size(0));
        d.T = 1;
        s.into(&d);
        const at::Tensor &state = tensor(a[5], "state_inout"), *og = opt_tensor(a[7], "out");
        void *sa = array(&state, s.v, s.state, at::kFloat, "state_inout");
        at::Tensor out;
        if (og) out = *og;
        else out = at::empty(s.v.sizes(), s.v.options().dtype(dtype_arg(a[8], s.v)));
        void *oa = array(&out, s.v, s.v.sizes(), io_of(out, "out"), "out");
        d.out_dtype = dtype_code(out.scalar_type());
        run([&] { return kla_ssm_step(&d, s.groups, s.qa, s.qs, s.ka, s.ks, s.va, s.vs, s.dta, s.aa, s.sa, static_cast<float *>(sa), oa); });
        return wrap(out);
    });
}

// kla_ssm_bwd: (q, k, v, dt, a, d_out, d_skip, init_state, d_final_state, cu_seqlens, host_seqlens, flags, want_dinit_state, status_word) -> dict
PyObject *ssm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 14, "ssm_bwd", [&]() -> PyObject * {
        Ssm s(a, a[6], 2);
        const c10::cuda::OptionalCUDAGuard guard(s.v.device());
        kla_desc d = desc_of(s.v, s.io, a[11]);
        at::Tensor host;
        sequences(&d, s.v, a[9], a[10], &host);
        s.into(&d);
        const at::Tensor &dout = tensor(a[5], "d_out");
        void *ga = array(&dout, s.v, s.v.sizes(), s.io, "d_out");
        void *ia = array(opt_tensor(a[7], "init_state"), s.v, s.state, at::kFloat, "init_state");
        void *fa = array(opt_tensor(a[8], "d_final_state"), s.v, s.state, at::kFloat, "d_final_state");
        d.status_word = status_word(a[13], s.v.device());
        const auto f32 = s.v.options().dtype(at::kFloat);
        at::Tensor dq = at::empty(s.q.sizes(), s.v.options()), dk = at::empty(s.q.sizes(), s.v.options()), dv = at::empty(s.v.sizes(), s.v.options());
        at::Tensor ddt = at::empty(s.dt.sizes(), f32), da = at::empty({s.H}, f32), dd, di;
        if (s.sa) dd = at::empty({s.H}, f32);
        if (integer(a[12])) di = at::empty(s.state, f32);
        at::Tensor ws = scratch(&d, s.v, kla_ssm_bwd_workspace_bytes(&d, s.groups));
        run([&] {
            return kla_ssm_bwd(&d, s.groups, s.qa, s.qs, s.ka, s.ks, s.va, s.vs, s.dta, s.aa, s.sa, static_cast<float *>(ia), ga, static_cast<float *>(fa),
                               dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ddt.data_ptr<float>(), da.data_ptr<float>(),
                               dd.defined() ? dd.data_ptr<float>() : nullptr, di.defined() ? di.data_ptr<float>() : nullptr);
        });
        return dict({{"dq", dq}, {"dk", dk}, {"dv", dv}, {"ddt", ddt}, {"da", da}, {"dd", dd}, {"dinit_state", di}});
    });
}

// What both calls of the norms share.
struct Norm {
    const at::Tensor &x, &weight;
    const at::Tensor *residual, *scale, *gate;
    at::ScalarType io, res;
    int64_t D, group, xs = 0, zs = 0;
    void *xa, *ra, *za = nullptr;
    float *wa, *sa, eps;
    int32_t width, per;   // channels of a row, of a group
    Norm(PyObject *x_, PyObject *w_, PyObject *eps_, PyObject *r_, PyObject *s_, PyObject *z_, PyObject *group_)
        : x(tensor(x_, "x")), weight(tensor(w_, "weight")), residual(opt_tensor(r_, "residual")), scale(opt_tensor(s_, "scale")), gate(opt_tensor(z_, "gate"))
    {
        io = res = io_of(x, "x");
        if (x.dim() < 1) fail(PyExc_ValueError, "x must be [..., width]");
        D = x.size(-1);
        group = group_ == Py_None ? D : integer(group_);
        eps = (float)number(eps_);
        xa = row_addr(x, 1, "x", &xs);
        wa = param(&weight, x, {D}, "weight");
        sa = param(scale, x, {D}, "scale");
        if (residual) res = io_of(*residual, "residual");
        ra = array(residual, x, x.sizes(), res, "residual");
        if (gate) {
            if (!has_shape(*gate, x.sizes())) fail(PyExc_ValueError, "has another shape than the call takes", "gate");
            if (gate->scalar_type() != io) fail(PyExc_TypeError, "has another dtype than the call takes", "gate");
            za = row_addr(*gate, 1, "gate", &zs);
            same_device(*gate, x, "gate");
        }
        width = small(D);
        per = small(group);
    }
    kla_desc desc(PyObject *flags) const
    {
        kla_desc d = desc_of(x, io, flags);
        d.B = d.n_seq = 1;
        d.T = small(D ? x.numel() / D : 0);
        return d;
    }
};

// kla_norm_fwd: (x, weight, eps, residual, scale, gate, group, out, residual_out, flags) -> (out, residual_out)
PyObject *norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, "norm_fwd", [&]() -> PyObject * {
        const Norm m(a[0], a[1], a[2], a[3], a[4], a[5], a[6]);
        const c10::cuda::OptionalCUDAGuard guard(m.x.device());
        kla_desc d = m.desc(a[9]);
        const at::Tensor *og = opt_tensor(a[7], "out"), *rg = opt_tensor(a[8], "residual_out");
        at::Tensor out, res;
        if (og) out = *og;
        else out = at::empty(m.x.sizes(), m.x.options());
        if (rg) res = *rg;
        else if (m.residual) res = at::empty(m.x.sizes(), m.residual->options());
        if (rg && !m.residual) fail(PyExc_ValueError, "needs a residual", "residual_out");
        void *oa = array(&out, m.x, m.x.sizes(), m.io, "out"), *ra = res.defined() ? array(&res, m.x, m.x.sizes(), m.res, "residual_out") : nullptr;
        run([&] { return kla_norm_fwd(&d, m.width, m.per, m.xa, m.xs, m.ra, dtype_code(m.res), m.sa, m.za, m.zs, m.wa, m.eps, oa, ra); });
        return pair(out, res);
    });
}

// kla_norm_bwd: (x, weight, eps, d_out, residual, scale, gate, group, d_residual_out, flags) -> dict
PyObject *norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 10, "norm_bwd", [&]() -> PyObject * {
        const Norm m(a[0], a[1], a[2], a[4], a[5], a[6], a[7]);
        const c10::cuda::OptionalCUDAGuard guard(m.x.device());
        kla_desc d = m.desc(a[9]);
        const at::Tensor &dout = tensor(a[3], "d_out"), *dres = opt_tensor(a[8], "d_residual_out");
        if (dres && !m.residual) fail(PyExc_ValueError, "needs a residual", "d_residual_out");
        void *ga = array(&dout, m.x, m.x.sizes(), m.io, "d_out"), *da = array(dres, m.x, m.x.sizes(), m.res, "d_residual_out");
        at::Tensor dx = at::empty(m.x.sizes(), m.x.options()), dw = at::empty({m.D}, m.weight.options()), dr, ds, dz;
        if (m.residual) dr = at::empty(m.x.sizes(), m.residual->options());
        if (m.scale) ds = at::empty({m.D}, m.weight.options());
        if (m.gate) dz = at::empty(m.x.sizes(), m.x.options());
        at::Tensor ws = scratch(&d, m.x, kla_norm_bwd_workspace_bytes(&d, m.width, m.per));
        run([&] {
            return kla_norm_bwd(&d, m.width, m.per, m.xa, m.xs, m.ra, dtype_code(m.res), m.sa, m.za, m.zs, m.wa, m.eps, ga, da, dx.data_ptr(),
                                dr.defined() ? dr.data_ptr() : nullptr, ds.defined() ? ds.data_ptr<float>() : nullptr,
                                dz.defined() ? dz.data_ptr() : nullptr, dw.data_ptr<float>());
        });
        return dict({{"dx", dx}, {"dweight", dw}, {"dresidual", dr}, {"dscale", ds}, {"dgate", dz}});
    });
}

// new_status_word(device index) -> int32[1], zero.  Made on a stream of its own and complete on return: on the current stream, if that is
// being captured, the word would belong to the graph, whose every replay would clear it.
PyObject *new_status_word(PyObject *, PyObject *index)
{
    try {
        const c10::Device device(c10::kCUDA, (c10::DeviceIndex)integer(index));
        const c10::cuda::CUDAGuard guard(device);
        const c10::cuda::CUDAStreamCaptureModeGuard relaxed(cudaStreamCaptureModeRelaxed);   // (of this thread, for a moment)
        cudaStream_t own;
        C10_CUDA_CHECK(cudaStreamCreateWithFlags(&own, cudaStreamNonBlocking));
        at::Tensor word;
        {
            const c10::cuda::CUDAStreamGuard on(c10::cuda::getStreamFromExternal(own, device.index()));
            word = at::zeros({1}, at::TensorOptions().device(device).dtype(at::kInt));
        }
        C10_CUDA_CHECK(cudaStreamSynchronize(own));
        C10_CUDA_CHECK(cudaStreamDestroy(own));
        return THPVariable_Wrap(std::move(word));
    } catch (const Failed &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyObject *init(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "init: 2 arguments");
        return nullptr;
    }
    Py_INCREF(g_kla_error = a[0]);
    Py_INCREF(g_status_for = a[1]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"init", (PyCFunction)(void (*)())init, METH_FASTCALL, nullptr},
                         {"decode", (PyCFunction)(void (*)())decode, METH_FASTCALL, nullptr},
                         {"forward", (PyCFunction)(void (*)())forward, METH_FASTCALL, nullptr},
                         {"new_status_word", new_status_word, METH_O, nullptr},
                         {"conv_fwd", (PyCFunction)(void (*)())conv_fwd, METH_FASTCALL, nullptr},
                         {"conv_step", (PyCFunction)(void (*)())conv_step, METH_FASTCALL, nullptr},
                         {"conv_bwd", (PyCFunction)(void (*)())conv_bwd, METH_FASTCALL, nullptr},
                         {"ssm_fwd", (PyCFunction)(void (*)())ssm_fwd, METH_FASTCALL, nullptr},
                         {"ssm_step", (PyCFunction)(void (*)())ssm_step, METH_FASTCALL, nullptr},
                         {"ssm_bwd", (PyCFunction)(void (*)())ssm_bwd, METH_FASTCALL, nullptr},
                         {"norm_fwd", (PyCFunction)(void (*)())norm_fwd, METH_FASTCALL, nullptr},
                         {"norm_bwd", (PyCFunction)(void (*)())norm_bwd, METH_FASTCALL, nullptr},
                         {"backward", (PyCFunction)(void (*)())backward, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host(void) { return PyModule_Create(&module); }
