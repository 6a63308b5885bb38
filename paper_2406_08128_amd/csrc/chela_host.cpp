// The host path of the decode step and of whole sequences without the interpreter: checks, the outputs' allocation, the current
// stream and the call into libchela.so for plain device tensors.  A step is over in 4.5 us on the GPU; through the binding's own lines, a dozen attribute
// look-ups, torch.empty() and ctypes, the host needed 8.9 us for it, of which the launch is 3.4.
//
// step(function, q, k, v, g or None, S, eps, y or None, stream or None) -> y, a status of the library (int, not 0), or None:
// "not the plain case", and nothing has been done.  The binding then takes its own path, which says what is wrong or serves the
// case (other devices, subclasses, modes).  function: address of chela_linattn_step (g is None) or chela_linattn_step_gated.
//
// Likewise, with the functions' addresses first and the stream last:
//   forward(f, f32, Q, K, V, S_in, S_out, chunk, stream) -> O; with f32 = None (chela_linattn_fwd_state: bf16 only) -> (O, S_out)
//   backward(f, f32, Q, K, V, dO, chunk, stream) -> (dQ, dK, dV); f32 = None: chela_linattn_noncausal_bwd, bf16 only, chunk not looked at
//   gated(f, saved_bytes, Q or Z, K or affine, V, G, eps, want_O, want_saved, stream) -> (Y, O or None, saved or None);
//       saved_bytes = None: chela_linattn_noncausal_fwd_gated
//   gate_norm_bwd(f, O, G, dY, eps, stream) -> (dO, dG)
//   zbwd_saved(f, Z, affine, V, dO, saved, stream) -> (dZ, d_affine, dV)
//   spectrum(f, bytes, k_long, stream) -> spectrum
//   conv_fwd(f, f32, X, w_short, spectrum, stream) -> Z;  conv_bwd(f, f32, X, w_short, spectrum, dZ, stream) -> (dX, d_w_short, d_k_long)
//   short_conv_fwd(f, f32, X, w, bias, silu, cu, S_in, S_out, slots, Y, stream) -> Y
//   short_conv_step(f, f32, x, w, S, bias, silu, slots, y, stream) -> y
//   selscan_fwd(f, f32, saved_bytes, U, delta, A, Bm, Cm, D, Z, delta_bias, softplus, cu, S_in, S_out, slots, want_saved, Y, stream) -> (Y, saved)
//   selscan_step(f, f32, u, delta, A, Bm, Cm, S, D, z, delta_bias, softplus, slots, y, stream) -> y
//   block_norm_fwd(f, f32, Y, X, gate, w_post, w_pre, scale, eps, stream) -> (X_out, Nrm)
//   short_conv_bwd(f, f32, X, w, dY, bias, silu, cu, S_in, dS_out, want_dS_in, stream) -> (dX, dw, dbias, dS_in)
//   selscan_bwd(f, f32, saved_bytes, U, delta, A, Bm, Cm, dY, D, Z, delta_bias, softplus, cu, S_in, dS_out, want_dS_in, saved, stream)
//       -> (dU, ddelta, dA, dB, dC, dD, dZ, ddelta_bias, dS_in)
//   block_norm_bwd(f, f32, Y, X_out, dX_out, dN, gate, w_post, w_pre, scale, eps, in_place, stream) -> (dY, dgate, dX, dw_post, dw_pre)
//   gated_delta_fwd(f, f32, saved_bytes, Q, K, V, g, beta, scale, cu, S_in, S_out, slots, want_saved, O, stream) -> (O, saved)
//   gated_delta_bwd(f, f32, saved_bytes, Q, K, V, g, beta, dO, scale, cu, S_in, dS_out, want_dS_in, saved, stream)
//       -> (dQ, dK, dV, dg, dbeta, dS_in)
//   gated_delta_step(f, f32, q, k, v, g, beta, S, scale, slots, o, stream) -> o
//   layer_norm_fwd(f, f32, X, w, b, Y, eps, stream) -> (X_out, Nrm)
//   layer_norm_bwd(f, f32, X_out, dN, w, want_db, dX_out, eps, in_place, stream) -> (dX, dw, db)
// Host side of a call, us, the binding's own lines and these: forward, one launch, 8.5 and 4.4, two launches 9.7 and 6.2; with the
// state 9.9 and 4.8, 12.1 and 7.2; backward, two launches, 11.4 and 7.5; the three calls of a gated layer's step, six launches, 39.6 and 23;
// spectrum, forward and gradient of a convolution, 22.5 and 15; both directions on 64 rows of 512 channels: short convolution, four launches, 39 and
// 21, selective scan, nine launches, 90 and 42, block norms 27 and 14.
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

typedef int (*step_fn)(const void*, const void*, const void*, float*, void*, int, int, int, int, void*);
typedef int (*step_gated_fn)(const void*, const void*, const void*, const void*, float*, void*, float, int, int, int, int, void*);

// a dense device tensor of exactly the class torch.Tensor
bool plain(PyObject* o, at::ScalarType type, c10::DeviceIndex dev)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && t.scalar_type() == type &&
           t.get_device() == dev && t.is_contiguous() && !t.key_set().has_any(c10::DispatchKeySet({c10::DispatchKey::FuncTorchBatched,
               c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize, c10::DispatchKey::Python}));
}

// (before there is a current device to ask for: a machine may have none)
bool on_gpu(PyObject* o) { return THPVariable_CheckExact(o) && THPVariable_Unpack(o).defined() && THPVariable_Unpack(o).is_cuda(); }

// something that wants to see, or to change, what is done with tensors
bool modes() { return at::impl::PythonTorchFunctionTLS::stack_len() > 0 || c10::impl::TorchDispatchModeTLS::any_modes_set(); }

struct without_interpreter_lock {
    PyThreadState* const state = PyEval_SaveThread();
    ~without_interpreter_lock() { PyEval_RestoreThread(state); }
};

PyObject* step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 9) { PyErr_SetString(PyExc_TypeError, "step takes nine arguments"); return nullptr; }
    if (modes()) Py_RETURN_NONE;
    PyObject *oq = a[1], *ok = a[2], *ov = a[3], *og = a[4], *oS = a[5], *oy = a[7], *ostream = a[8];
    if (!THPVariable_CheckExact(oq) || (ostream != Py_None) || !PyFloat_CheckExact(a[6])) Py_RETURN_NONE;
    const at::Tensor& q = THPVariable_Unpack(oq);
    if (!q.defined() || !q.is_cuda()) Py_RETURN_NONE;
    const c10::DeviceIndex dev = c10::hip::current_device();
    if (!plain(oq, at::kBFloat16, dev) || !plain(ok, at::kBFloat16, dev) || !plain(ov, at::kBFloat16, dev) ||
        !plain(oS, at::kFloat, dev) || (og != Py_None && !plain(og, at::kBFloat16, dev)) ||
        (oy != Py_None && !plain(oy, at::kBFloat16, dev)))
        Py_RETURN_NONE;
    const at::Tensor &k = THPVariable_Unpack(ok), &v = THPVariable_Unpack(ov), &S = THPVariable_Unpack(oS);
    if (q.dim() != 3 || k.sizes() != q.sizes() || v.dim() != 3) Py_RETURN_NONE;
    const int64_t B = q.size(0), H = q.size(1), dk = q.size(2), dv = v.size(2);
    const int64_t lim = 0x7fffffff;
    if (v.size(0) != B || v.size(1) != H || B > lim || H > lim || dk > lim || dv > lim) Py_RETURN_NONE;
    if (S.dim() != 4 || S.size(0) != B || S.size(1) != H || S.size(2) != dk || S.size(3) != dv) Py_RETURN_NONE;
    if (og != Py_None && THPVariable_Unpack(og).sizes() != v.sizes()) Py_RETURN_NONE;
    if (oy != Py_None && THPVariable_Unpack(oy).sizes() != v.sizes()) Py_RETURN_NONE;
    const unsigned long long fn = PyLong_AsUnsignedLongLong(a[0]);
    if (PyErr_Occurred()) return nullptr;
    const void *pq = q.data_ptr(), *pk = k.data_ptr(), *pv = v.data_ptr();
    const void* pg = og != Py_None ? THPVariable_Unpack(og).data_ptr() : nullptr;
    float *pS = (float*)S.data_ptr(), eps = (float)PyFloat_AS_DOUBLE(a[6]);
    const at::TensorOptions like = q.options().requires_grad(false);
    at::Tensor y;
    if (oy != Py_None) y = THPVariable_Unpack(oy);
    int rc;
    {
        // (both may wait for the GPU, the launch for room in a queue: other threads go on, as they do through ctypes)
        const without_interpreter_lock free;
        if (oy == Py_None) y = at::empty({B, H, dv}, like);
        void *py = y.data_ptr(), *st = (void*)c10::hip::getCurrentHIPStream(dev).stream();
        rc = og == Py_None
                 ? reinterpret_cast<step_fn>(fn)(pq, pk, pv, pS, py, (int)B, (int)H, (int)dk, (int)dv, st)
                 : reinterpret_cast<step_gated_fn>(fn)(pq, pk, pv, pg, pS, py, eps, (int)B, (int)H, (int)dk, (int)dv, st);
    }
    if (rc != 0) return PyLong_FromLong(rc);
    if (oy != Py_None) { Py_INCREF(oy); return oy; }
    return THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

typedef int (*fwd_fn)(const void*, const void*, const void*, void*, int, int, int, int, int, int, void*);
typedef int (*fwd_state_fn)(const void*, const void*, const void*, const float*, void*, float*, int, int, int, int, int, int, void*);
typedef int (*bwd_fn)(const void*, const void*, const void*, const void*, void*, void*, void*, int, int, int, int, int, int, void*);
typedef int (*noncausal_bwd_fn)(const void*, const void*, const void*, const void*, void*, void*, void*, int, int, int, int, int, void*);
typedef int (*gated_fn)(const void*, const void*, const void*, const void*, void*, void*, void*, float, int, int, int, int, int, int, void*);
typedef int (*noncausal_gated_fn)(const void*, const void*, const void*, const void*, void*, void*, float, int, int, int, int, int, void*);
typedef size_t (*saved_bytes_fn)(int, int, int, int, int, int);
typedef int (*gate_norm_bwd_fn)(const void*, const void*, const void*, void*, void*, float, long long, int, void*);
typedef int (*zbwd_saved_fn)(const void*, const float*, const void*, const void*, const void*, void*, float*, void*, int, int, int, int, int,
                             int, void*);
typedef size_t (*spectrum_bytes_fn)(int, int);
typedef int (*spectrum_fn)(const float*, void*, int, int, void*);
typedef int (*conv_fwd_fn)(const void*, const float*, int, const void*, void*, int, int, int, void*);
typedef int (*conv_bwd_fn)(const void*, const float*, int, const void*, const void*, void*, float*, float*, int, int, int, void*);

// Q, K [B,H,N,dk] and V [B,H,N,dv], plain and of one type that there is a function for.
struct Sequences {
    int B, H, N, dk, dv, chunk;
    c10::DeviceIndex dev;
    at::ScalarType type;
    bool read(PyObject* const* qkv, bool f32_too, PyObject* ochunk, PyObject* ostream)
    {
        if (modes() || ostream != Py_None || !on_gpu(qkv[0])) return false;
        const int64_t lim = 0x7fffffff;
        int overflow = 0;
        long c = 64;
        if (ochunk != nullptr) {
            if (!PyLong_CheckExact(ochunk)) return false;
            c = PyLong_AsLongAndOverflow(ochunk, &overflow);
            if (overflow || c < 0 || c > lim) return false;
        }
        const at::Tensor& q = THPVariable_Unpack(qkv[0]);
        type = q.scalar_type();
        dev = c10::hip::current_device();
        if (type != at::kBFloat16 && !(f32_too && type == at::kFloat)) return false;
        for (int i = 0; i < 3; ++i) if (!plain(qkv[i], type, dev)) return false;
        const at::Tensor &k = THPVariable_Unpack(qkv[1]), &v = THPVariable_Unpack(qkv[2]);
        if (q.dim() != 4 || k.sizes() != q.sizes() || v.dim() != 4) return false;
        for (int i = 0; i < 4; ++i) if (q.size(i) > lim || v.size(i) > lim || (i < 3 && v.size(i) != q.size(i))) return false;
        B = (int)q.size(0); H = (int)q.size(1); N = (int)q.size(2); dk = (int)q.size(3); dv = (int)v.size(3);
        chunk = (int)c;
        return true;
    }
    bool is_affine(PyObject* o) const
    {
        if (!plain(o, at::kFloat, dev)) return false;
        const at::Tensor& t = THPVariable_Unpack(o);
        return t.dim() == 3 && t.size(0) == 4 && t.size(1) == H && t.size(2) == dk;
    }
    bool is_state(PyObject* o) const
    {
        if (!plain(o, at::kFloat, dev)) return false;
        const at::Tensor& t = THPVariable_Unpack(o);
        return t.dim() == 4 && t.size(0) == B && t.size(1) == H && t.size(2) == dk && t.size(3) == dv;
    }
};

PyObject* none() { Py_INCREF(Py_None); return Py_None; }

// The tensors as a tuple, None for those that are not there.
template <size_t N>
PyObject* wrap(at::Tensor (&t)[N])
{
    PyObject* all = PyTuple_New(N);
    for (size_t i = 0; all != nullptr && i < N; ++i) {
        PyObject* o = t[i].defined() ? THPVariable_Wrap(std::move(t[i])) : none();
        if (o == nullptr) { Py_DECREF(all); return nullptr; }
        PyTuple_SET_ITEM(all, i, o);
    }
    return all;
}

template <typename F>
F address(PyObject* o) { return reinterpret_cast<F>(PyLong_AsUnsignedLongLong(o)); }
void* stream_of(c10::DeviceIndex dev) { return (void*)c10::hip::getCurrentHIPStream(dev).stream(); }
at::TensorOptions like(const at::Tensor& t) { return t.options().requires_grad(false); }

PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 9) { PyErr_SetString(PyExc_TypeError, "forward takes nine arguments"); return nullptr; }
    const bool with_state = a[1] == Py_None;
    Sequences x;
    if (!x.read(a + 2, !with_state, a[7], a[8])) Py_RETURN_NONE;
    PyObject *oin = a[5], *oout = a[6];
    if ((oin != Py_None && !(with_state && x.is_state(oin))) || (oout != Py_None && !(with_state && x.is_state(oout)))) Py_RETURN_NONE;
    PyObject* const of = a[x.type == at::kFloat ? 1 : 0];
    const auto f = address<fwd_fn>(of);
    const auto f_state = address<fwd_state_fn>(of);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor& q = THPVariable_Unpack(a[2]);
    const void *pq = q.data_ptr(), *pk = THPVariable_Unpack(a[3]).data_ptr(), *pv = THPVariable_Unpack(a[4]).data_ptr();
    const float* pin = oin != Py_None ? (const float*)THPVariable_Unpack(oin).data_ptr() : nullptr;
    at::Tensor out[2];
    if (oout != Py_None) out[1] = THPVariable_Unpack(oout);
    int rc;
    {
        const without_interpreter_lock free;
        out[0] = at::empty({x.B, x.H, x.N, x.dv}, like(q));
        if (with_state && oout == Py_None) out[1] = at::empty({x.B, x.H, x.dk, x.dv}, like(q).dtype(at::kFloat));
        void *po = out[0].data_ptr(), *st = stream_of(x.dev);
        rc = with_state ? f_state(pq, pk, pv, pin, po, (float*)out[1].data_ptr(), x.B, x.H, x.N, x.dk, x.dv, x.chunk, st)
                        : f(pq, pk, pv, po, x.B, x.H, x.N, x.dk, x.dv, x.chunk, st);
    }
    if (rc != 0) return PyLong_FromLong(rc);
    return with_state ? wrap(out) : THPVariable_Wrap(std::move(out[0]));       // (S_out as it came: a tensor has one Python object)
    END_HANDLE_TH_ERRORS
}

PyObject* backward(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 8) { PyErr_SetString(PyExc_TypeError, "backward takes eight arguments"); return nullptr; }
    const bool causal = a[1] != Py_None;
    Sequences x;
    if (!x.read(a + 2, causal, causal ? a[6] : nullptr, a[7]) || !plain(a[5], x.type, x.dev)) Py_RETURN_NONE;
    const at::Tensor &q = THPVariable_Unpack(a[2]), &v = THPVariable_Unpack(a[4]), &d = THPVariable_Unpack(a[5]);
    if (d.sizes() != v.sizes()) Py_RETURN_NONE;
    PyObject* const of = a[x.type == at::kFloat ? 1 : 0];
    const auto f = address<bwd_fn>(of);
    const auto f_noncausal = address<noncausal_bwd_fn>(of);
    if (PyErr_Occurred()) return nullptr;
    const void *pq = q.data_ptr(), *pk = THPVariable_Unpack(a[3]).data_ptr(), *pv = v.data_ptr(), *pd = d.data_ptr();
    at::Tensor g[3];
    int rc;
    {
        const without_interpreter_lock free;
        for (int i = 0; i < 3; ++i) g[i] = at::empty({x.B, x.H, x.N, i < 2 ? x.dk : x.dv}, like(q));
        void *p0 = g[0].data_ptr(), *p1 = g[1].data_ptr(), *p2 = g[2].data_ptr(), *st = stream_of(x.dev);
        rc = causal ? f(pq, pk, pv, pd, p0, p1, p2, x.B, x.H, x.N, x.dk, x.dv, x.chunk, st)
                    : f_noncausal(pq, pk, pv, pd, p0, p1, p2, x.B, x.H, x.N, x.dk, x.dv, st);
    }
    return rc != 0 ? PyLong_FromLong(rc) : wrap(g);
    END_HANDLE_TH_ERRORS
}

PyObject* gated(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "gated takes ten arguments"); return nullptr; }
    const bool causal = a[1] != Py_None;
    Sequences x;
    // (the second operand: keys of the first one's shape, or the affine parameters [4,H,dk])
    PyObject* const first[3] = {a[2], a[2], a[4]};
    if (!x.read(first, false, nullptr, a[9]) || !PyFloat_CheckExact(a[6])) Py_RETURN_NONE;
    const at::Tensor &q = THPVariable_Unpack(a[2]), &v = THPVariable_Unpack(a[4]);
    if (plain(a[3], at::kBFloat16, x.dev) ? THPVariable_Unpack(a[3]).sizes() != q.sizes() : !(causal && x.is_affine(a[3]))) Py_RETURN_NONE;
    if (!plain(a[5], at::kBFloat16, x.dev) || THPVariable_Unpack(a[5]).sizes() != v.sizes()) Py_RETURN_NONE;
    const int want_O = PyObject_IsTrue(a[7]), want_saved = PyObject_IsTrue(a[8]);
    if (want_O < 0 || want_saved < 0) return nullptr;
    const auto f = address<gated_fn>(a[0]);
    const auto f_noncausal = address<noncausal_gated_fn>(a[0]);
    const auto bytes = causal ? address<saved_bytes_fn>(a[1]) : nullptr;
    if (PyErr_Occurred()) return nullptr;
    const void *pq = q.data_ptr(), *pk = THPVariable_Unpack(a[3]).data_ptr(), *pv = v.data_ptr(), *pg = THPVariable_Unpack(a[5]).data_ptr();
    const float eps = (float)PyFloat_AS_DOUBLE(a[6]);
    at::Tensor out[3];      // Y, O, saved
    int rc;
    {
        const without_interpreter_lock free;
        for (int i = 0; i < (want_O ? 2 : 1); ++i) out[i] = at::empty({x.B, x.H, x.N, x.dv}, like(q));
        if (causal && want_saved) {
            const size_t need = bytes(x.B, x.H, x.N, x.dk, x.dv, 64);
            out[2] = at::empty({(int64_t)(need < 16 ? 16 : need) / 4}, like(q).dtype(at::kFloat));
        }
        void *pY = out[0].data_ptr(), *pO = want_O ? out[1].data_ptr() : nullptr, *ps = out[2].defined() ? out[2].data_ptr() : nullptr;
        rc = causal ? f(pq, pk, pv, pg, pO, pY, ps, eps, x.B, x.H, x.N, x.dk, x.dv, 64, stream_of(x.dev))
                    : f_noncausal(pq, pk, pv, pg, pO, pY, eps, x.B, x.H, x.N, x.dk, x.dv, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : wrap(out);
    END_HANDLE_TH_ERRORS
}

PyObject* gate_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "gate_norm_bwd takes six arguments"); return nullptr; }
    if (modes() || a[5] != Py_None || !PyFloat_CheckExact(a[4]) || !on_gpu(a[1])) Py_RETURN_NONE;
    const c10::DeviceIndex dev = c10::hip::current_device();
    for (int i = 1; i < 4; ++i) if (!plain(a[i], at::kBFloat16, dev)) Py_RETURN_NONE;
    const at::Tensor &o = THPVariable_Unpack(a[1]), &g = THPVariable_Unpack(a[2]), &d = THPVariable_Unpack(a[3]);
    if (o.dim() < 1 || g.sizes() != o.sizes() || d.sizes() != o.sizes() || o.size(-1) < 1 || o.size(-1) > 0x7fffffff) Py_RETURN_NONE;
    const auto f = address<gate_norm_bwd_fn>(a[0]);
    if (PyErr_Occurred()) return nullptr;
    const void *po = o.data_ptr(), *pg = g.data_ptr(), *pd = d.data_ptr();
    const float eps = (float)PyFloat_AS_DOUBLE(a[4]);
    at::Tensor out[2];
    int rc;
    {
        const without_interpreter_lock free;
        for (at::Tensor& t : out) t = at::empty(o.sizes(), like(o));
        rc = f(po, pg, pd, out[0].data_ptr(), out[1].data_ptr(), eps, (long long)(o.numel() / o.size(-1)), (int)o.size(-1), stream_of(dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : wrap(out);
    END_HANDLE_TH_ERRORS
}

PyObject* zbwd_saved(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "zbwd_saved takes seven arguments"); return nullptr; }
    Sequences x;
    PyObject* const zv[3] = {a[1], a[1], a[3]};
    if (!x.read(zv, false, nullptr, a[6]) || !x.is_affine(a[2]) || !plain(a[4], at::kBFloat16, x.dev) || !plain(a[5], at::kFloat, x.dev))
        Py_RETURN_NONE;
    const at::Tensor &z = THPVariable_Unpack(a[1]), &v = THPVariable_Unpack(a[3]), &d = THPVariable_Unpack(a[4]);
    if (d.sizes() != v.sizes()) Py_RETURN_NONE;
    const auto f = address<zbwd_saved_fn>(a[0]);
    if (PyErr_Occurred()) return nullptr;
    const void *pz = z.data_ptr(), *pv = v.data_ptr(), *pd = d.data_ptr(), *ps = THPVariable_Unpack(a[5]).data_ptr();
    const float* pa = (const float*)THPVariable_Unpack(a[2]).data_ptr();
    at::Tensor g[3];
    int rc;
    {
        const without_interpreter_lock free;
        g[0] = at::empty({x.B, x.H, x.N, x.dk}, like(z));
        g[1] = at::empty({4, x.H, x.dk}, like(z).dtype(at::kFloat));
        g[2] = at::empty({x.B, x.H, x.N, x.dv}, like(z));
        rc = f(pz, pa, pv, pd, ps, g[0].data_ptr(), (float*)g[1].data_ptr(), g[2].data_ptr(), x.B, x.H, x.N, x.dk, x.dv, 64, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : wrap(g);
    END_HANDLE_TH_ERRORS
}

// A plain tensor of the type with as many dimensions, none beyond an int.
bool plain_sizes(PyObject* o, at::ScalarType type, c10::DeviceIndex dev, int64_t dims)
{
    if (!plain(o, type, dev)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.dim() != dims) return false;
    for (int64_t i = 0; i < dims; ++i) if (t.size(i) > 0x7fffffff) return false;
    return true;
}

PyObject* spectrum(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 4) { PyErr_SetString(PyExc_TypeError, "spectrum takes four arguments"); return nullptr; }
    if (modes() || a[3] != Py_None || !on_gpu(a[2])) Py_RETURN_NONE;
    const c10::DeviceIndex dev = c10::hip::current_device();
    if (!plain_sizes(a[2], at::kFloat, dev, 2)) Py_RETURN_NONE;
    const at::Tensor& k = THPVariable_Unpack(a[2]);
    const int d = (int)k.size(0), L = (int)k.size(1);
    const auto f = address<spectrum_fn>(a[0]);
    const auto bytes = address<spectrum_bytes_fn>(a[1]);
    if (PyErr_Occurred()) return nullptr;
    const size_t need = bytes(d, L);
    if (need == 0) Py_RETURN_NONE;
    const float* pk = (const float*)k.data_ptr();
    at::Tensor s;
    int rc;
    {
        const without_interpreter_lock free;
        s = at::empty({(int64_t)(need < 16 ? 16 : need) / 4}, like(k));
        rc = f(pk, s.data_ptr(), d, L, stream_of(dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : THPVariable_Wrap(std::move(s));
    END_HANDLE_TH_ERRORS
}

// X [B,d,L], w_short [d,m] or None, the spectrum (whatever its size: that is the caller's business, as in the binding).
struct Conv {
    int B, d, L, m;
    c10::DeviceIndex dev;
    at::ScalarType type;
    const float* w;
    bool read(PyObject* ox, PyObject* ow, PyObject* os, PyObject* ostream)
    {
        if (modes() || ostream != Py_None || !on_gpu(ox)) return false;
        const at::Tensor& x = THPVariable_Unpack(ox);
        type = x.scalar_type();
        dev = c10::hip::current_device();
        if ((type != at::kBFloat16 && type != at::kFloat) || !plain_sizes(ox, type, dev, 3) || !plain(os, at::kFloat, dev)) return false;
        B = (int)x.size(0); d = (int)x.size(1); L = (int)x.size(2); m = 0; w = nullptr;
        if (ow == Py_None) return true;
        if (!plain_sizes(ow, at::kFloat, dev, 2) || THPVariable_Unpack(ow).size(0) != d) return false;
        m = (int)THPVariable_Unpack(ow).size(1);
        w = (const float*)THPVariable_Unpack(ow).data_ptr();
        return true;
    }
};

PyObject* conv_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "conv_fwd takes six arguments"); return nullptr; }
    Conv c;
    if (!c.read(a[2], a[3], a[4], a[5])) Py_RETURN_NONE;
    const auto f = address<conv_fwd_fn>(a[c.type == at::kFloat ? 1 : 0]);
    if (PyErr_Occurred()) return nullptr;
    const at::Tensor& x = THPVariable_Unpack(a[2]);
    const void *px = x.data_ptr(), *ps = THPVariable_Unpack(a[4]).data_ptr();
    at::Tensor z;
    int rc;
    {
        const without_interpreter_lock free;
        z = at::empty({c.B, c.d, c.L}, like(x));
        rc = f(px, c.w, c.m, ps, z.data_ptr(), c.B, c.d, c.L, stream_of(c.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : THPVariable_Wrap(std::move(z));
    END_HANDLE_TH_ERRORS
}

PyObject* conv_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "conv_bwd takes seven arguments"); return nullptr; }
    Conv c;
    if (!c.read(a[2], a[3], a[4], a[6]) || !plain(a[5], c.type, c.dev)) Py_RETURN_NONE;
    const at::Tensor &x = THPVariable_Unpack(a[2]), &dz = THPVariable_Unpack(a[5]);
    if (dz.sizes() != x.sizes()) Py_RETURN_NONE;
    const auto f = address<conv_bwd_fn>(a[c.type == at::kFloat ? 1 : 0]);
    if (PyErr_Occurred()) return nullptr;
    const void *px = x.data_ptr(), *ps = THPVariable_Unpack(a[4]).data_ptr(), *pd = dz.data_ptr();
    at::Tensor g[3];        // dX, d_w_short, d_k_long
    int rc;
    {
        const without_interpreter_lock free;
        g[0] = at::empty({c.B, c.d, c.L}, like(x));
        if (c.w != nullptr || a[3] != Py_None) g[1] = at::empty({c.d, c.m}, like(x).dtype(at::kFloat));
        g[2] = at::empty({c.d, c.L}, like(x).dtype(at::kFloat));
        rc = f(px, c.w, c.m, ps, pd, g[0].data_ptr(), g[1].defined() ? (float*)g[1].data_ptr() : nullptr, (float*)g[2].data_ptr(), c.B, c.d,
               c.L, stream_of(c.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : wrap(g);
    END_HANDLE_TH_ERRORS
}

// ---- operators on rows: tensors whose rows may be slices of wider ones
typedef int (*short_conv_fwd_fn)(const void*, long long, const float*, int, const float*, int, const int*, int, int, int, const void*, void*,
                                 const int*, int, void*, void*);
typedef int (*short_conv_step_fn)(const void*, long long, const float*, int, const float*, int, void*, const int*, int, int, int, void*, void*);
typedef int (*selscan_fwd_fn)(const void*, long long, const void*, long long, const float*, const void*, long long, const void*, long long,
                              const float*, const void*, long long, const float*, int, const int*, int, int, int, int, int, const float*,
                              float*, const int*, int, void*, void*, void*);
typedef int (*selscan_step_fn)(const void*, long long, const void*, long long, const float*, const void*, long long, const void*, long long,
                               const float*, const void*, long long, const float*, int, float*, const int*, int, int, int, int, int, void*, void*);
typedef size_t (*selscan_saved_fn)(int, int, int);
typedef int (*block_norm_fwd_fn)(const void*, const void*, const void*, const float*, const float*, void*, void*, float, float, long long, int,
                                 int, void*);
typedef int (*short_conv_bwd_fn)(const void*, long long, const float*, int, const float*, int, const int*, int, int, int, const void*, const void*,
                                 long long, const void*, void*, float*, float*, void*, void*);
typedef int (*selscan_bwd_fn)(const void*, long long, const void*, long long, const float*, const void*, long long, const void*, long long,
                              const float*, const void*, long long, const float*, int, const int*, int, int, int, int, int, const float*,
                              const void*, long long, const float*, const void*, void*, void*, float*, void*, void*, float*, void*, float*, float*,
                              void*);
typedef int (*block_norm_bwd_fn)(const void*, const void*, const void*, const float*, const float*, const void*, const void*, void*, void*, void*,
                                 float*, float*, float, float, long long, int, int, void*);

#define CHELA_DELTA_IN                                                                                                \
    const void*, long long, const void*, long long, const void*, long long, const void*, long long, const void*, long long, float
typedef int (*delta_fwd_fn)(CHELA_DELTA_IN, const int*, int, int, int, int, int, int, const float*, float*, const int*, int, void*, void*, void*);
typedef int (*delta_bwd_fn)(CHELA_DELTA_IN, const int*, int, int, int, int, int, int, const float*, const void*, long long, const float*,
                            const void*, void*, void*, void*, void*, void*, float*, void*);
typedef int (*delta_step_fn)(CHELA_DELTA_IN, float*, const int*, int, int, int, int, int, int, void*, void*);
typedef size_t (*delta_saved_fn)(int, int, int, int, int, int, int);
typedef int (*layer_norm_fwd_fn)(const void*, const void*, const float*, const float*, void*, void*, float, long long, int, int, void*);
typedef int (*layer_norm_bwd_fn)(const void*, const float*, const void*, const void*, void*, float*, float*, float, long long, int, int, void*);

struct Rows {
    c10::DeviceIndex dev;
    at::ScalarType type;
    int64_t lead[2], T, D;          // leading sizes (one or two), their product, the row's width
    int dims;
    int n_seq, n_slots;
    const int *cu, *slots;

    // a tensor of that type there, contiguous or not
    bool there(PyObject* o, at::ScalarType t) const
    {
        if (!THPVariable_CheckExact(o)) return false;
        const at::Tensor& x = THPVariable_Unpack(o);
        return x.defined() && x.is_cuda() && x.layout() == at::kStrided && x.has_storage() && x.scalar_type() == t && x.get_device() == dev &&
               !x.key_set().has_any(c10::DispatchKeySet({c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                                         c10::DispatchKey::Functionalize, c10::DispatchKey::Python}));
    }
    // The first tensor, [B, L, D] or [T, D], and its sequences.
    bool first(PyObject* o, PyObject* ocu, PyObject* ostream)
    {
        if (modes() || ostream != Py_None || !on_gpu(o)) return false;
        const at::Tensor& x = THPVariable_Unpack(o);
        type = x.scalar_type();
        dev = c10::hip::current_device();
        if ((type != at::kBFloat16 && type != at::kFloat) || !there(o, type)) return false;
        dims = (int)x.dim() - 1;
        if (dims < 1 || dims > 2) return false;
        T = 1;
        for (int i = 0; i < dims; ++i) {
            lead[i] = x.size(i);
            if (lead[i] > 0x7fffffff) return false;
            T *= lead[i];
        }
        D = x.size(dims);
        if (T > 0x7fffffff || D > 0x7fffffff) return false;
        cu = slots = nullptr;
        n_seq = dims == 2 ? (int)lead[0] : 1;
        if (ocu != Py_None) {
            if (dims != 1 || !plain(ocu, at::kInt, dev)) return false;
            const at::Tensor& c = THPVariable_Unpack(ocu);
            if (c.dim() != 1 || c.size(0) < 1 || c.size(0) > 0x7fffffff) return false;
            n_seq = (int)c.size(0) - 1;
            cu = (const int*)c.data_ptr();
        }
        n_slots = n_seq;
        return true;
    }
    // A tensor with the first one's rows and `width` elements in each: address and stride of the rows.
    bool rows(PyObject* o, int64_t width, const void** p, long long* ld) const
    {
        if (!there(o, type)) return false;
        const at::Tensor& x = THPVariable_Unpack(o);
        if (x.dim() < dims + 1) return false;
        for (int i = 0; i < dims; ++i) if (x.size(i) != lead[i]) return false;
        int64_t w = 1;
        for (int k = (int)x.dim() - 1; k >= dims; --k) {
            if (x.size(k) > 1 && x.stride(k) != w) return false;
            w *= x.size(k);
        }
        if (w != width) return false;
        int64_t step = -1, n = 1;
        for (int k = dims - 1; k >= 0; --k) {
            if (x.size(k) <= 1) continue;
            if (step < 0) step = x.stride(k);
            else if (x.stride(k) != step * n) return false;
            n *= x.size(k);
        }
        *p = x.data_ptr();
        *ld = step < 0 ? (width > 1 ? width : 1) : step;
        return true;
    }
    template <typename T_>
    bool dense(PyObject* o, at::ScalarType t, at::IntArrayRef sizes, bool optional, T_** p) const
    {
        *p = nullptr;
        if (optional && o == Py_None) return true;
        if (!plain(o, t, dev) || THPVariable_Unpack(o).sizes() != sizes) return false;
        *p = (T_*)THPVariable_Unpack(o).data_ptr();
        return true;
    }
    bool slot_map(PyObject* o, PyObject* states)
    {
        if (o == Py_None) return true;
        if (states == Py_None || !THPVariable_CheckExact(states) || THPVariable_Unpack(states).dim() < 1) return false;
        const int64_t n = THPVariable_Unpack(states).size(0);
        if (n > 0x7fffffff || !dense(o, at::kInt, {n_seq}, false, &slots)) return false;
        n_slots = (int)n;
        return true;
    }
    PyObject* function(PyObject* const* a) const { return a[type == at::kFloat ? 1 : 0]; }
};

// True or False, or something else: -1
int flag(PyObject* o) { return o == Py_True ? 1 : o == Py_False ? 0 : -1; }

PyObject* given_or(PyObject* o, at::Tensor& made)
{
    if (o == Py_None) return THPVariable_Wrap(std::move(made));
    Py_INCREF(o);
    return o;
}

PyObject* short_conv_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 12) { PyErr_SetString(PyExc_TypeError, "short_conv_fwd takes twelve arguments"); return nullptr; }
    Rows x;
    const void *px, *pin;
    long long ldx;
    const float *pw, *pb;
    void *pout, *py;
    const int silu = flag(a[5]);
    if (silu < 0 || !x.first(a[2], a[6], a[11]) || !x.rows(a[2], x.D, &px, &ldx) || !plain_sizes(a[3], at::kFloat, x.dev, 2)) Py_RETURN_NONE;
    const int64_t m = THPVariable_Unpack(a[3]).size(1);
    if (m < 1 || !x.dense(a[3], at::kFloat, {x.D, m}, false, &pw) || !x.dense(a[4], at::kFloat, {x.D}, true, &pb) ||
        !x.slot_map(a[9], a[7] != Py_None ? a[7] : a[8]) || !x.dense(a[7], x.type, {x.n_slots, m - 1, x.D}, true, &pin) ||
        !x.dense(a[8], x.type, {x.n_slots, m - 1, x.D}, true, &pout))
        Py_RETURN_NONE;
    const at::Tensor& X = THPVariable_Unpack(a[2]);
    if (!x.dense(a[10], x.type, X.sizes(), true, &py)) Py_RETURN_NONE;
    const auto f = address<short_conv_fwd_fn>(x.function(a));
    if (PyErr_Occurred()) return nullptr;
    at::Tensor y;
    int rc;
    {
        const without_interpreter_lock free;
        if (a[10] == Py_None) { y = at::empty(X.sizes(), like(X).memory_format(at::MemoryFormat::Contiguous)); py = y.data_ptr(); }
        rc = f(px, ldx, pw, (int)m, pb, silu, x.cu, x.n_seq, (int)x.T, (int)x.D, pin, pout, x.slots, x.n_slots, py, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : given_or(a[10], y);
    END_HANDLE_TH_ERRORS
}

PyObject* short_conv_step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "short_conv_step takes ten arguments"); return nullptr; }
    Rows x;
    const void* px;
    long long ldx;
    const float *pw, *pb;
    void *ps, *py;
    const int silu = flag(a[6]);
    if (silu < 0 || !x.first(a[2], Py_None, a[9]) || x.dims != 1 || !x.rows(a[2], x.D, &px, &ldx) || !plain_sizes(a[3], at::kFloat, x.dev, 2))
        Py_RETURN_NONE;
    x.n_seq = x.n_slots = (int)x.T;
    const int64_t m = THPVariable_Unpack(a[3]).size(1);
    if (m < 1 || !x.dense(a[3], at::kFloat, {x.D, m}, false, &pw) || !x.dense(a[5], at::kFloat, {x.D}, true, &pb) || !x.slot_map(a[7], a[4]) ||
        !x.dense(a[4], x.type, {x.n_slots, m - 1, x.D}, false, &ps) || !x.dense(a[8], x.type, {x.T, x.D}, true, &py))
        Py_RETURN_NONE;
    const at::Tensor& X = THPVariable_Unpack(a[2]);
    const auto f = address<short_conv_step_fn>(x.function(a));
    if (PyErr_Occurred()) return nullptr;
    at::Tensor y;
    int rc;
    {
        const without_interpreter_lock free;
        if (a[8] == Py_None) { y = at::empty({x.T, x.D}, like(X)); py = y.data_ptr(); }
        rc = f(px, ldx, pw, (int)m, pb, silu, ps, x.slots, x.n_slots, (int)x.T, (int)x.D, py, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : given_or(a[8], y);
    END_HANDLE_TH_ERRORS
}

// What the scan's calls have in common: U, delta, A, Bm, Cm and D, Z, delta_bias.
struct Scan {
    const void *U, *delta, *Bm, *Cm, *Z = nullptr;
    long long ldu, ldd, ldb, ldc, ldz = 0;
    const float *A, *D, *bias;
    int64_t N, G;
    bool read(const Rows& x, PyObject* const* five, PyObject* const* three)
    {
        if (!x.rows(five[0], x.D, &U, &ldu) || !x.rows(five[1], x.D, &delta, &ldd) || !THPVariable_CheckExact(five[3]) ||
            !THPVariable_CheckExact(five[4]))
            return false;
        const at::Tensor &b = THPVariable_Unpack(five[3]), &c = THPVariable_Unpack(five[4]);
        if (!b.defined() || !c.defined() || THPVariable_Unpack(five[1]).dim() != x.dims + 1 || b.dim() < x.dims + 1 || b.dim() > x.dims + 2 ||
            b.sizes() != c.sizes())
            return false;
        N = b.size(-1);
        G = b.dim() == x.dims + 2 ? b.size(-2) : 1;
        if (N > 0x7fffffff || G > 0x7fffffff) return false;
        if (three[1] != Py_None && (!x.rows(three[1], x.D, &Z, &ldz) || THPVariable_Unpack(three[1]).dim() != x.dims + 1)) return false;
        return x.rows(five[3], N * G, &Bm, &ldb) && x.rows(five[4], N * G, &Cm, &ldc) && x.dense(five[2], at::kFloat, {N, x.D}, false, &A) &&
               x.dense(three[0], at::kFloat, {x.D}, true, &D) && x.dense(three[2], at::kFloat, {x.D}, true, &bias);
    }
};

PyObject* selscan_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 19) { PyErr_SetString(PyExc_TypeError, "selscan_fwd takes nineteen arguments"); return nullptr; }
    Rows x;
    Scan s;
    const float* pin;
    float* pout;
    void* py;
    const int softplus = flag(a[11]), want_saved = flag(a[16]);
    if (softplus < 0 || want_saved < 0 || !x.first(a[3], a[12], a[18]) || !s.read(x, a + 3, a + 8) ||
        !x.slot_map(a[15], a[13] != Py_None ? a[13] : a[14]) || !x.dense(a[13], at::kFloat, {x.n_slots, s.N, x.D}, true, &pin) ||
        !x.dense(a[14], at::kFloat, {x.n_slots, s.N, x.D}, true, &pout))
        Py_RETURN_NONE;
    const at::Tensor& U = THPVariable_Unpack(a[3]);
    if (!x.dense(a[17], x.type, U.sizes(), true, &py)) Py_RETURN_NONE;
    const auto f = address<selscan_fwd_fn>(x.function(a));
    const auto bytes = address<selscan_saved_fn>(a[2]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor y, saved;
    int rc;
    {
        const without_interpreter_lock free;
        if (a[17] == Py_None) { y = at::empty(U.sizes(), like(U).memory_format(at::MemoryFormat::Contiguous)); py = y.data_ptr(); }
        if (want_saved) {
            const size_t need = bytes((int)x.T, (int)x.D, (int)s.N);
            saved = at::empty({(int64_t)(need < 16 ? 16 : need) / 4}, like(U).dtype(at::kFloat));
        }
        rc = f(s.U, s.ldu, s.delta, s.ldd, s.A, s.Bm, s.ldb, s.Cm, s.ldc, s.D, s.Z, s.ldz, s.bias, softplus, x.cu, x.n_seq, (int)x.T, (int)x.D,
               (int)s.N, (int)s.G, pin, pout, x.slots, x.n_slots, py, want_saved ? saved.data_ptr() : nullptr, stream_of(x.dev));
    }
    if (rc != 0) return PyLong_FromLong(rc);
    PyObject* both = PyTuple_New(2);
    if (both == nullptr) return nullptr;
    PyObject *first = given_or(a[17], y), *second = want_saved ? THPVariable_Wrap(std::move(saved)) : none();
    if (first == nullptr || second == nullptr) { Py_XDECREF(first); Py_XDECREF(second); Py_DECREF(both); return nullptr; }
    PyTuple_SET_ITEM(both, 0, first);
    PyTuple_SET_ITEM(both, 1, second);
    return both;
    END_HANDLE_TH_ERRORS
}

PyObject* selscan_step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 15) { PyErr_SetString(PyExc_TypeError, "selscan_step takes fifteen arguments"); return nullptr; }
    Rows x;
    Scan s;
    float* ps;
    void* py;
    const int softplus = flag(a[11]);
    if (softplus < 0 || !x.first(a[2], Py_None, a[14]) || x.dims != 1 || !s.read(x, a + 2, a + 8)) Py_RETURN_NONE;
    x.n_seq = x.n_slots = (int)x.T;
    if (!x.slot_map(a[12], a[7]) || !x.dense(a[7], at::kFloat, {x.n_slots, s.N, x.D}, false, &ps) || !x.dense(a[13], x.type, {x.T, x.D}, true, &py))
        Py_RETURN_NONE;
    const at::Tensor& U = THPVariable_Unpack(a[2]);
    const auto f = address<selscan_step_fn>(x.function(a));
    if (PyErr_Occurred()) return nullptr;
    at::Tensor y;
    int rc;
    {
        const without_interpreter_lock free;
        if (a[13] == Py_None) { y = at::empty({x.T, x.D}, like(U)); py = y.data_ptr(); }
        rc = f(s.U, s.ldu, s.delta, s.ldd, s.A, s.Bm, s.ldb, s.Cm, s.ldc, s.D, s.Z, s.ldz, s.bias, softplus, ps, x.slots, x.n_slots, (int)x.T,
               (int)x.D, (int)s.N, (int)s.G, py, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : given_or(a[13], y);
    END_HANDLE_TH_ERRORS
}

// (with Y: in front of the first block the binding's own lines)
PyObject* block_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "block_norm_fwd takes ten arguments"); return nullptr; }
    if (modes() || a[9] != Py_None || !PyFloat_CheckExact(a[7]) || !PyFloat_CheckExact(a[8]) || !on_gpu(a[2]) || !on_gpu(a[3])) Py_RETURN_NONE;
    Rows x;
    x.dev = c10::hip::current_device();
    x.type = THPVariable_Unpack(a[2]).scalar_type();
    const at::Tensor& X = THPVariable_Unpack(a[3]);
    const at::ScalarType xt = X.scalar_type();
    if ((x.type != at::kBFloat16 && x.type != at::kFloat) || (xt != x.type && xt != at::kFloat) || X.dim() < 1) Py_RETURN_NONE;
    const int64_t D = X.size(-1);
    if (D < 1 || D > 0x7fffffff) Py_RETURN_NONE;
    const void *pY, *pX, *pg;
    const float *pp, *pn;
    if (!x.dense(a[2], x.type, X.sizes(), false, &pY) || !x.dense(a[3], xt, X.sizes(), false, &pX) || !x.dense(a[4], x.type, X.sizes(), true, &pg) ||
        !x.dense(a[5], at::kFloat, {D}, true, &pp) || !x.dense(a[6], at::kFloat, {D}, true, &pn))
        Py_RETURN_NONE;
    const auto f = address<block_norm_fwd_fn>(a[x.type == at::kFloat ? 1 : 0]);
    if (PyErr_Occurred()) return nullptr;
    const float scale = (float)PyFloat_AS_DOUBLE(a[7]), eps = (float)PyFloat_AS_DOUBLE(a[8]);
    at::Tensor out[2];
    int rc;
    {
        const without_interpreter_lock free;
        out[0] = at::empty(X.sizes(), like(X));
        if (pn != nullptr || a[6] != Py_None) out[1] = at::empty(X.sizes(), like(X).dtype(x.type));
        rc = f(pY, pg, pX, pp, pn, out[0].data_ptr(), out[1].defined() ? out[1].data_ptr() : nullptr, scale, eps, (long long)(X.numel() / D), (int)D,
               xt != x.type, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : wrap(out);
    END_HANDLE_TH_ERRORS
}

// A new contiguous tensor's address, where there is to be one.
template <typename T_ = void>
T_* make(at::Tensor& t, bool wanted, at::IntArrayRef sizes, const at::TensorOptions& o)
{
    if (!wanted) return nullptr;
    t = at::empty(sizes, o);
    return (T_*)t.data_ptr();
}

PyObject* short_conv_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 12) { PyErr_SetString(PyExc_TypeError, "short_conv_bwd takes twelve arguments"); return nullptr; }
    Rows x;
    const void *px, *pdy, *pin, *pds;
    long long ldx, lddy;
    const float *pw, *pb;
    const int silu = flag(a[6]), want = flag(a[10]);
    if (silu < 0 || want < 0 || !x.first(a[2], a[7], a[11]) || !x.rows(a[2], x.D, &px, &ldx) || !x.rows(a[4], x.D, &pdy, &lddy) ||
        THPVariable_Unpack(a[4]).dim() != x.dims + 1 || !plain_sizes(a[3], at::kFloat, x.dev, 2))
        Py_RETURN_NONE;
    const int64_t m = THPVariable_Unpack(a[3]).size(1);
    if (m < 1 || !x.dense(a[3], at::kFloat, {x.D, m}, false, &pw) || !x.dense(a[5], at::kFloat, {x.D}, true, &pb) ||
        !x.dense(a[8], x.type, {x.n_seq, m - 1, x.D}, true, &pin) || !x.dense(a[9], x.type, {x.n_seq, m - 1, x.D}, true, &pds))
        Py_RETURN_NONE;
    const at::Tensor& X = THPVariable_Unpack(a[2]);
    const auto f = address<short_conv_bwd_fn>(x.function(a));
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out[4];
    int rc;
    {
        const without_interpreter_lock free;
        const at::TensorOptions io = like(X).memory_format(at::MemoryFormat::Contiguous), f32 = io.dtype(at::kFloat);
        void* dx = make(out[0], true, X.sizes(), io);
        float *dw = make<float>(out[1], true, {x.D, m}, f32), *db = make<float>(out[2], a[5] != Py_None, {x.D}, f32);
        void* ds = make(out[3], want != 0, {x.n_seq, m - 1, x.D}, io);
        rc = f(px, ldx, pw, (int)m, pb, silu, x.cu, x.n_seq, (int)x.T, (int)x.D, pin, pdy, lddy, pds, dx, dw, db, ds, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : wrap(out);
    END_HANDLE_TH_ERRORS
}

PyObject* selscan_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 19) { PyErr_SetString(PyExc_TypeError, "selscan_bwd takes nineteen arguments"); return nullptr; }
    Rows x;
    Scan s;
    const void *pdy, *psaved = nullptr;
    long long lddy;
    const float *pin, *pds;
    const int softplus = flag(a[12]), want = flag(a[16]);
    if (softplus < 0 || want < 0 || !x.first(a[3], a[13], a[18]) || !s.read(x, a + 3, a + 9) || !x.rows(a[8], x.D, &pdy, &lddy) ||
        THPVariable_Unpack(a[8]).dim() != x.dims + 1 || !x.dense(a[14], at::kFloat, {x.n_seq, s.N, x.D}, true, &pin) ||
        !x.dense(a[15], at::kFloat, {x.n_seq, s.N, x.D}, true, &pds))
        Py_RETURN_NONE;
    const auto f = address<selscan_bwd_fn>(x.function(a));
    const auto bytes = address<selscan_saved_fn>(a[2]);
    if (PyErr_Occurred()) return nullptr;
    if (a[17] != Py_None) {
        if (!plain(a[17], at::kFloat, x.dev)) Py_RETURN_NONE;
        const at::Tensor& saved = THPVariable_Unpack(a[17]);
        if ((size_t)saved.numel() * 4 < bytes((int)x.T, (int)x.D, (int)s.N)) Py_RETURN_NONE;
        psaved = saved.data_ptr();
    }
    const at::Tensor &U = THPVariable_Unpack(a[3]), &B = THPVariable_Unpack(a[6]);
    at::Tensor out[9];
    int rc;
    {
        const without_interpreter_lock free;
        const at::TensorOptions io = like(U).memory_format(at::MemoryFormat::Contiguous), f32 = io.dtype(at::kFloat);
        void *du = make(out[0], true, U.sizes(), io), *dd = make(out[1], true, U.sizes(), io);
        float* dA = make<float>(out[2], true, {s.N, x.D}, f32);
        void *dB = make(out[3], true, B.sizes(), io), *dC = make(out[4], true, B.sizes(), io);
        float* dD = make<float>(out[5], a[9] != Py_None, {x.D}, f32);
        void* dZ = make(out[6], a[10] != Py_None, U.sizes(), io);
        float *db = make<float>(out[7], a[11] != Py_None, {x.D}, f32), *ds = make<float>(out[8], want != 0, {x.n_seq, s.N, x.D}, f32);
        rc = f(s.U, s.ldu, s.delta, s.ldd, s.A, s.Bm, s.ldb, s.Cm, s.ldc, s.D, s.Z, s.ldz, s.bias, softplus, x.cu, x.n_seq, (int)x.T, (int)x.D,
               (int)s.N, (int)s.G, pin, pdy, lddy, pds, psaved, du, dd, dA, dB, dC, dD, dZ, db, ds, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : wrap(out);
    END_HANDLE_TH_ERRORS
}

PyObject* block_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 13) { PyErr_SetString(PyExc_TypeError, "block_norm_bwd takes thirteen arguments"); return nullptr; }
    const int in_place = flag(a[11]);
    if (modes() || a[12] != Py_None || in_place < 0 || !PyFloat_CheckExact(a[9]) || !PyFloat_CheckExact(a[10]) || !on_gpu(a[2]) || !on_gpu(a[3]))
        Py_RETURN_NONE;
    Rows x;
    x.dev = c10::hip::current_device();
    x.type = THPVariable_Unpack(a[2]).scalar_type();
    const at::Tensor& X = THPVariable_Unpack(a[3]);
    const at::ScalarType xt = X.scalar_type();
    if ((x.type != at::kBFloat16 && x.type != at::kFloat) || (xt != x.type && xt != at::kFloat) || X.dim() < 1) Py_RETURN_NONE;
    const int64_t D = X.size(-1);
    if (D < 1 || D > 0x7fffffff || (a[5] == Py_None) != (a[8] == Py_None) || (in_place && a[4] == Py_None)) Py_RETURN_NONE;
    const void *pY, *pX, *pg, *pdn;
    void* pdx;
    const float *pp, *pn;
    if (!x.dense(a[2], x.type, X.sizes(), false, &pY) || !x.dense(a[3], xt, X.sizes(), false, &pX) || !x.dense(a[4], xt, X.sizes(), true, &pdx) ||
        !x.dense(a[5], x.type, X.sizes(), true, &pdn) || !x.dense(a[6], x.type, X.sizes(), true, &pg) ||
        !x.dense(a[7], at::kFloat, {D}, true, &pp) || !x.dense(a[8], at::kFloat, {D}, true, &pn))
        Py_RETURN_NONE;
    const auto f = address<block_norm_bwd_fn>(a[x.type == at::kFloat ? 1 : 0]);
    if (PyErr_Occurred()) return nullptr;
    const float scale = (float)PyFloat_AS_DOUBLE(a[9]), eps = (float)PyFloat_AS_DOUBLE(a[10]);
    at::Tensor out[5];
    int rc;
    {
        const without_interpreter_lock free;
        const at::TensorOptions io = like(X).dtype(x.type), f32 = like(X).dtype(at::kFloat);
        void *dY = make(out[0], true, X.sizes(), io), *dg = make(out[1], a[6] != Py_None, X.sizes(), io);
        void* dX = in_place ? pdx : make(out[2], true, X.sizes(), like(X));
        float *dp = make<float>(out[3], a[7] != Py_None, {D}, f32), *dn = make<float>(out[4], a[8] != Py_None, {D}, f32);
        rc = f(pY, pg, pX, pp, pn, pdx, pdn, dY, dg, dX, dp, dn, scale, eps, (long long)(X.numel() / D), (int)D, xt != x.type, stream_of(x.dev));
    }
    if (rc != 0) return PyLong_FromLong(rc);
    PyObject* all = wrap(out);
    if (all != nullptr && in_place) {
        PyObject* was = PyTuple_GET_ITEM(all, 2);
        Py_INCREF(a[4]);
        PyTuple_SET_ITEM(all, 2, a[4]);
        Py_DECREF(was);
    }
    return all;
    END_HANDLE_TH_ERRORS
}

// What the gated delta rule's calls have in common: Q, K, V, g, beta, scale.
struct Delta {
    const void *Q, *K, *V, *g = nullptr, *beta;
    long long ldq, ldk, ldv, ldg = 0, ldb;
    int64_t H, Hk, dk, dv;
    float scale;
    bool read(Rows& x, PyObject* const* five, PyObject* oscale, PyObject* ocu, PyObject* ostream)
    {
        if (!PyFloat_CheckExact(oscale) || !x.first(five[4], ocu, ostream) || !x.there(five[0], x.type) || !x.there(five[1], x.type) ||
            !x.there(five[2], x.type))
            return false;
        const at::Tensor &q = THPVariable_Unpack(five[0]), &k = THPVariable_Unpack(five[1]), &v = THPVariable_Unpack(five[2]);
        if (q.dim() != x.dims + 2 || v.dim() != x.dims + 2 || k.sizes() != q.sizes()) return false;
        H = x.D;
        Hk = q.size(-2);
        dk = q.size(-1);
        dv = v.size(-1);
        scale = (float)PyFloat_AS_DOUBLE(oscale);
        if (v.size(-2) != H || Hk < 1 || H % Hk != 0 || Hk > 0x7fffffff || dk > 0x7fffffff || dv > 0x7fffffff) return false;
        if (five[3] != Py_None && (!x.rows(five[3], H, &g, &ldg) || THPVariable_Unpack(five[3]).dim() != x.dims + 1)) return false;
        return x.rows(five[0], Hk * dk, &Q, &ldq) && x.rows(five[1], Hk * dk, &K, &ldk) && x.rows(five[2], H * dv, &V, &ldv) &&
               x.rows(five[4], H, &beta, &ldb);
    }
};

PyObject* gated_delta_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 16) { PyErr_SetString(PyExc_TypeError, "gated_delta_fwd takes sixteen arguments"); return nullptr; }
    Rows x;
    Delta s;
    const float* pin;
    float* pout;
    void* po;
    const int want_saved = flag(a[13]);
    if (want_saved < 0 || !s.read(x, a + 3, a[8], a[9], a[15]) || !x.slot_map(a[12], a[10] != Py_None ? a[10] : a[11]) ||
        !x.dense(a[10], at::kFloat, {x.n_slots, s.H, s.dk, s.dv}, true, &pin) ||
        !x.dense(a[11], at::kFloat, {x.n_slots, s.H, s.dk, s.dv}, true, &pout))
        Py_RETURN_NONE;
    const at::Tensor& V = THPVariable_Unpack(a[5]);
    if (!x.dense(a[14], x.type, V.sizes(), true, &po)) Py_RETURN_NONE;
    const auto f = address<delta_fwd_fn>(x.function(a));
    const auto bytes = address<delta_saved_fn>(a[2]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor o, saved;
    int rc;
    {
        const without_interpreter_lock free;
        if (a[14] == Py_None) { o = at::empty(V.sizes(), like(V).memory_format(at::MemoryFormat::Contiguous)); po = o.data_ptr(); }
        if (want_saved) {
            const size_t need = bytes((int)x.T, x.n_seq, x.cu != nullptr, (int)s.H, (int)s.dk, (int)s.dv, x.type == at::kFloat);
            saved = at::empty({(int64_t)(need < 16 ? 16 : need) / 4}, like(V).dtype(at::kFloat));
        }
        rc = f(s.Q, s.ldq, s.K, s.ldk, s.V, s.ldv, s.g, s.ldg, s.beta, s.ldb, s.scale, x.cu, x.n_seq, (int)x.T, (int)s.H, (int)s.Hk, (int)s.dk,
               (int)s.dv, pin, pout, x.slots, x.n_slots, po, want_saved ? saved.data_ptr() : nullptr, stream_of(x.dev));
    }
    if (rc != 0) return PyLong_FromLong(rc);
    PyObject* both = PyTuple_New(2);
    if (both == nullptr) return nullptr;
    PyObject *first = given_or(a[14], o), *second = want_saved ? THPVariable_Wrap(std::move(saved)) : none();
    if (first == nullptr || second == nullptr) { Py_XDECREF(first); Py_XDECREF(second); Py_DECREF(both); return nullptr; }
    PyTuple_SET_ITEM(both, 0, first);
    PyTuple_SET_ITEM(both, 1, second);
    return both;
    END_HANDLE_TH_ERRORS
}

PyObject* gated_delta_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 16) { PyErr_SetString(PyExc_TypeError, "gated_delta_bwd takes sixteen arguments"); return nullptr; }
    Rows x;
    Delta s;
    const void *pdo, *psaved = nullptr;
    long long lddo;
    const float *pin, *pds;
    const int want = flag(a[13]);
    if (want < 0 || !s.read(x, a + 3, a[9], a[10], a[15]) || !x.rows(a[8], s.H * s.dv, &pdo, &lddo) ||
        THPVariable_Unpack(a[8]).sizes() != THPVariable_Unpack(a[5]).sizes() ||
        !x.dense(a[11], at::kFloat, {x.n_seq, s.H, s.dk, s.dv}, true, &pin) || !x.dense(a[12], at::kFloat, {x.n_seq, s.H, s.dk, s.dv}, true, &pds))
        Py_RETURN_NONE;
    const auto f = address<delta_bwd_fn>(x.function(a));
    const auto bytes = address<delta_saved_fn>(a[2]);
    if (PyErr_Occurred()) return nullptr;
    if (a[14] != Py_None) {
        if (!plain(a[14], at::kFloat, x.dev)) Py_RETURN_NONE;
        const at::Tensor& saved = THPVariable_Unpack(a[14]);
        if ((size_t)saved.numel() * 4 < bytes((int)x.T, x.n_seq, x.cu != nullptr, (int)s.H, (int)s.dk, (int)s.dv, x.type == at::kFloat)) Py_RETURN_NONE;
        psaved = saved.data_ptr();
    }
    const at::Tensor &Q = THPVariable_Unpack(a[3]), &V = THPVariable_Unpack(a[5]), &beta = THPVariable_Unpack(a[7]);
    at::Tensor out[6];
    int rc;
    {
        const without_interpreter_lock free;
        const at::TensorOptions io = like(V).memory_format(at::MemoryFormat::Contiguous);
        void *dQ = make(out[0], true, Q.sizes(), io), *dK = make(out[1], true, Q.sizes(), io), *dV = make(out[2], true, V.sizes(), io);
        void *dg = make(out[3], a[6] != Py_None, beta.sizes(), io), *db = make(out[4], true, beta.sizes(), io);
        float* ds = make<float>(out[5], want != 0, {x.n_seq, s.H, s.dk, s.dv}, io.dtype(at::kFloat));
        rc = f(s.Q, s.ldq, s.K, s.ldk, s.V, s.ldv, s.g, s.ldg, s.beta, s.ldb, s.scale, x.cu, x.n_seq, (int)x.T, (int)s.H, (int)s.Hk, (int)s.dk,
               (int)s.dv, pin, pdo, lddo, pds, psaved, dQ, dK, dV, dg, db, ds, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : wrap(out);
    END_HANDLE_TH_ERRORS
}

PyObject* gated_delta_step(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 12) { PyErr_SetString(PyExc_TypeError, "gated_delta_step takes twelve arguments"); return nullptr; }
    Rows x;
    Delta s;
    float* ps;
    void* po;
    if (!s.read(x, a + 2, a[8], Py_None, a[11]) || x.dims != 1) Py_RETURN_NONE;
    x.n_seq = x.n_slots = (int)x.T;
    if (!x.slot_map(a[9], a[7]) || !x.dense(a[7], at::kFloat, {x.n_slots, s.H, s.dk, s.dv}, false, &ps) ||
        !x.dense(a[10], x.type, {x.T, s.H, s.dv}, true, &po))
        Py_RETURN_NONE;
    const auto f = address<delta_step_fn>(x.function(a));
    if (PyErr_Occurred()) return nullptr;
    at::Tensor o;
    int rc;
    {
        const without_interpreter_lock free;
        if (a[10] == Py_None) { o = at::empty({x.T, s.H, s.dv}, like(THPVariable_Unpack(a[4]))); po = o.data_ptr(); }
        rc = f(s.Q, s.ldq, s.K, s.ldk, s.V, s.ldv, s.g, s.ldg, s.beta, s.ldb, s.scale, ps, x.slots, x.n_slots, (int)x.T, (int)s.H, (int)s.Hk,
               (int)s.dk, (int)s.dv, po, stream_of(x.dev));
    }
    return rc != 0 ? PyLong_FromLong(rc) : given_or(a[10], o);
    END_HANDLE_TH_ERRORS
}

// The stream X, and beside it a tensor of the I/O type (or X's own).
struct Stream {
    Rows x;
    at::ScalarType type;             // X's
    int64_t D;
    const void* pX;
    bool read(PyObject* oX, PyObject* beside, PyObject* oeps, PyObject* ostream)
    {
        if (modes() || ostream != Py_None || !PyFloat_CheckExact(oeps) || !on_gpu(oX) || (beside != Py_None && !on_gpu(beside))) return false;
        x.dev = c10::hip::current_device();
        const at::Tensor& X = THPVariable_Unpack(oX);
        type = X.scalar_type();
        x.type = beside != Py_None ? THPVariable_Unpack(beside).scalar_type() : type;
        if ((x.type != at::kBFloat16 && x.type != at::kFloat) || (type != x.type && type != at::kFloat) || X.dim() < 1) return false;
        D = X.size(-1);
        return D >= 1 && D <= 0x7fffffff && x.dense(oX, type, X.sizes(), false, &pX);
    }
};

PyObject* layer_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 8) { PyErr_SetString(PyExc_TypeError, "layer_norm_fwd takes eight arguments"); return nullptr; }
    Stream s;
    const void* pY;
    const float *pw, *pb;
    if (!s.read(a[2], a[5], a[6], a[7])) Py_RETURN_NONE;
    const at::Tensor& X = THPVariable_Unpack(a[2]);
    if (!s.x.dense(a[5], s.x.type, X.sizes(), true, &pY) || !s.x.dense(a[3], at::kFloat, {s.D}, true, &pw) ||
        !s.x.dense(a[4], at::kFloat, {s.D}, true, &pb))
        Py_RETURN_NONE;
    const auto f = address<layer_norm_fwd_fn>(s.x.function(a));
    if (PyErr_Occurred()) return nullptr;
    const float eps = (float)PyFloat_AS_DOUBLE(a[6]);
    at::Tensor out[2];
    int rc;
    {
        const without_interpreter_lock free;
        void* px = make(out[0], a[5] != Py_None, X.sizes(), like(X));
        void* pn = make(out[1], true, X.sizes(), like(X).dtype(s.x.type));
        rc = f(s.pX, pY, pw, pb, px, pn, eps, (long long)(X.numel() / s.D), (int)s.D, s.type != s.x.type, stream_of(s.x.dev));
    }
    if (rc != 0) return PyLong_FromLong(rc);
    PyObject* both = wrap(out);
    if (both != nullptr && a[5] == Py_None) {
        PyObject* was = PyTuple_GET_ITEM(both, 0);
        Py_INCREF(a[2]);
        PyTuple_SET_ITEM(both, 0, a[2]);
        Py_DECREF(was);
    }
    return both;
    END_HANDLE_TH_ERRORS
}

PyObject* layer_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "layer_norm_bwd takes ten arguments"); return nullptr; }
    const int want_db = flag(a[5]), in_place = flag(a[8]);
    Stream s;
    const void* pdn;
    void* pdx;
    const float* pw;
    if (want_db < 0 || in_place < 0 || (in_place && a[6] == Py_None) || !s.read(a[2], a[3], a[7], a[9]) || a[3] == Py_None) Py_RETURN_NONE;
    const at::Tensor& X = THPVariable_Unpack(a[2]);
    if (!s.x.dense(a[3], s.x.type, X.sizes(), false, &pdn) || !s.x.dense(a[6], s.type, X.sizes(), true, &pdx) ||
        !s.x.dense(a[4], at::kFloat, {s.D}, true, &pw))
        Py_RETURN_NONE;
    const auto f = address<layer_norm_bwd_fn>(s.x.function(a));
    if (PyErr_Occurred()) return nullptr;
    const float eps = (float)PyFloat_AS_DOUBLE(a[7]);
    at::Tensor out[3];
    int rc;
    {
        const without_interpreter_lock free;
        const at::TensorOptions f32 = like(X).dtype(at::kFloat);
        void* dX = in_place ? pdx : make(out[0], true, X.sizes(), like(X));
        float *dw = make<float>(out[1], a[4] != Py_None, {s.D}, f32), *db = make<float>(out[2], want_db != 0, {s.D}, f32);
        rc = f(s.pX, pw, pdx, pdn, dX, dw, db, eps, (long long)(X.numel() / s.D), (int)s.D, s.type != s.x.type, stream_of(s.x.dev));
    }
    if (rc != 0) return PyLong_FromLong(rc);
    PyObject* all = wrap(out);
    if (all != nullptr && in_place) {
        PyObject* was = PyTuple_GET_ITEM(all, 0);
        Py_INCREF(a[6]);
        PyTuple_SET_ITEM(all, 0, a[6]);
        Py_DECREF(was);
    }
    return all;
    END_HANDLE_TH_ERRORS
}

#define CHELA_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CHELA_METHOD(step), CHELA_METHOD(forward), CHELA_METHOD(backward), CHELA_METHOD(gated),
                         CHELA_METHOD(gate_norm_bwd), CHELA_METHOD(zbwd_saved), CHELA_METHOD(spectrum), CHELA_METHOD(conv_fwd),
                         CHELA_METHOD(conv_bwd), CHELA_METHOD(short_conv_fwd), CHELA_METHOD(short_conv_step), CHELA_METHOD(selscan_fwd),
                         CHELA_METHOD(selscan_step), CHELA_METHOD(block_norm_fwd), CHELA_METHOD(short_conv_bwd), CHELA_METHOD(selscan_bwd),
                         CHELA_METHOD(block_norm_bwd), CHELA_METHOD(gated_delta_fwd), CHELA_METHOD(gated_delta_bwd),
                         CHELA_METHOD(gated_delta_step), CHELA_METHOD(layer_norm_fwd), CHELA_METHOD(layer_norm_bwd), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_chela_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__chela_host() { return PyModule_Create(&module); }
