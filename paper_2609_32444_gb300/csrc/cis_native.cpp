// cis_native.cpp -- the binding's calls in native code: argument checks, output
// tensors and the library call of binding.py's functions, without Python's cost
// per tensor.
//
// Bound: the host.  A fused pass of T=256, V=1024 keeps the GPU busy for 13 us,
// and its call took 45 us of Python (checks of five tensors, seven outputs,
// twenty-six converted arguments); from here it takes 17 us, 7.5 of them the
// library's (three launches).
//
// Every function takes its Python counterpart's arguments by position, and
// answers with that function's result; with an int, the library's error; or with
// None where an argument is not what the plain case expects (a tensor of another
// kind, type, shape or device): then nothing was done, and the counterpart goes
// on in Python, where the checks raise.
//
// Data pointers are taken before the GIL is released: a tensor without storage (a
// functorch wrapper, which passes for a plain tensor) raises there.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>
#include <string.h>

#include <algorithm>
#include <initializer_list>
#include <utility>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "cis.h"

namespace {

using at::Tensor;

struct Library {
    decltype(&cis_loss_workspace_size) loss_ws = nullptr;
    decltype(&cis_loss_fwd_bwd) loss = nullptr;
    decltype(&cis_token_logprobs) logprobs = nullptr;
    decltype(&cis_weights) weights = nullptr;
    decltype(&cis_binned_sums_workspace_size) bins_ws = nullptr;
    decltype(&cis_binned_sums) bins = nullptr;
    decltype(&cis_mismatch_diagnostics) diagnostics = nullptr;
    decltype(&cis_sample_tokens) sample = nullptr;
    decltype(&cis_topk_logprobs) topk = nullptr;
    decltype(&cis_distill_workspace_size) distill_ws = nullptr;
    decltype(&cis_distill_fwd_bwd) distill = nullptr;
    decltype(&cis_rmsnorm_fwd) norm = nullptr;
    decltype(&cis_rmsnorm_bwd_workspace_size) norm_bwd_ws = nullptr;
    decltype(&cis_rmsnorm_bwd) norm_bwd = nullptr;
    decltype(&cis_lmhead_logits) head = nullptr;
    decltype(&cis_verify_workspace_size) verify_ws = nullptr;
    decltype(&cis_verify_tokens) verify = nullptr;
} lib;

// A tensor argument: None, or a plain tensor (no subclass) with strides.
bool take(PyObject *o, const Tensor *&t)
{
    t = nullptr;
    if (o == Py_None)
        return true;
    if (!THPVariable_CheckExact(o))
        return false;
    t = &THPVariable_Unpack(o);
    return t->defined() && t->layout() == at::kStrided;
}
bool on_gpu(const Tensor *t) { return t == nullptr || t->is_cuda(); }
// None, or a contiguous vector of T elements on the GPU.
bool vec(const Tensor *t, at::ScalarType dt, int64_t T)
{
    return t == nullptr || (t->is_cuda() && t->scalar_type() == dt && t->dim() == 1 &&
                            t->size(0) == T && t->is_contiguous());
}
// Rows with unit column stride: their number and stride.
bool rows(const Tensor &x, int64_t &T, int64_t &ld)
{
    if (x.dim() != 2 || (x.size(1) > 1 && x.stride(1) != 1))
        return false;
    T = x.size(0);
    ld = T > 1 ? x.stride(0) : x.size(1);
    return true;
}
bool dtype_code(at::ScalarType t, int32_t &code)
{
    if (t != at::kBFloat16 && t != at::kFloat)
        return false;
    code = t == at::kBFloat16 ? CIS_BF16 : CIS_F32;
    return true;
}
bool integer(PyObject *o, int64_t &v)
{
    if (!PyLong_CheckExact(o))
        return false;
    int over = 0;
    v = PyLong_AsLongLongAndOverflow(o, &over);
    return over == 0;
}
bool flag(PyObject *o, bool &v)
{
    v = o == Py_True;
    return PyBool_Check(o);
}
// The parameter struct behind a ctypes object of the binding's own type, copied.
PyObject *params_type = nullptr, *distill_type = nullptr;
template <typename P> bool params_of(PyObject *o, const PyObject *type, P &p)
{
    Py_buffer b;
    if (reinterpret_cast<PyObject *>(Py_TYPE(o)) != type || !PyObject_CheckBuffer(o) ||
        PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) {
        PyErr_Clear();
        return false;
    }
    const bool ok = b.len == (Py_ssize_t)sizeof(p);
    if (ok)
        memcpy(&p, b.buf, sizeof(p));
    PyBuffer_Release(&b);
    return ok;
}
// None, or a status word.
bool status(const Tensor *t)
{
    return t == nullptr || (t->scalar_type() == at::kInt && t->numel() >= 1);
}
bool params(PyObject *o, cis_params_t &p) { return params_of(o, params_type, p); }
// Every given tensor is on the device of x, and that is the current one.
bool together(const Tensor &x, std::initializer_list<const Tensor *> ts)
{
    for (const Tensor *t : ts)
        if (t && t->device() != x.device())
            return false;
    return x.is_cuda() && x.device().index() == c10::cuda::current_device();
}
// None: the rows' length; else at most that.
bool vocabulary(PyObject *o, const Tensor &z, int64_t &V)
{
    if (o == Py_None) {
        V = z.size(1);
        return true;
    }
    return integer(o, V) && V <= z.size(1);
}

template <typename T = void> T *ptr(const Tensor *t)
{
    return t ? static_cast<T *>(t->data_ptr()) : nullptr;
}
template <typename T = void> T *ptr(const Tensor &t)
{
    return t.defined() ? ptr<T>(&t) : nullptr;
}
Tensor fresh(at::IntArrayRef shape, at::ScalarType dt, const at::Device &dev)
{
    return at::empty(shape, at::TensorOptions().dtype(dt).device(dev));
}
Tensor fresh_if(bool want, int64_t n, at::ScalarType dt, const at::Device &dev)
{
    return want ? fresh({n}, dt, dev) : Tensor();
}
void *stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

PyObject *none() { Py_RETURN_NONE; }
PyObject *wrap(const Tensor &t) { return t.defined() ? THPVariable_Wrap(t) : none(); }
PyObject *dict(std::initializer_list<std::pair<const char *, Tensor>> items)
{
    PyObject *d = PyDict_New();
    for (const auto &it : items) {
        PyObject *v = d ? wrap(it.second) : nullptr;
        if (v == nullptr || PyDict_SetItemString(d, it.first, v) != 0) {
            Py_XDECREF(v);
            Py_XDECREF(d);
            return nullptr;
        }
        Py_DECREF(v);
    }
    return d;
}

// (logits, ids, lp_infer, adv, params, lp_old, mask, cu_seqlens, dlogits,
//  dlogits_dtype, V, want_lp, want_w, want_trunc, workspace, want_entropy)
PyObject *loss_fwd_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *z, *ids, *lpi, *adv, *old, *mask, *cu, *dz_in, *ws_in;
    cis_params_t P;
    bool want[3], want_ent;
    if (n != 16 || !take(a[0], z) || !take(a[1], ids) || !take(a[2], lpi) || !take(a[3], adv) ||
        !params(a[4], P) || !take(a[5], old) || !take(a[6], mask) || !take(a[7], cu) ||
        !take(a[8], dz_in) || !flag(a[11], want[0]) || !flag(a[12], want[1]) ||
        !flag(a[13], want[2]) || !take(a[14], ws_in) || !flag(a[15], want_ent))
        return none();
    int64_t T, ld, V, To, ldo;
    int32_t code, code_out;
    if (!z || !ids || !lpi || !adv || !z->is_cuda() || !rows(*z, T, ld) ||
        !dtype_code(z->scalar_type(), code) || !vec(ids, at::kInt, T) ||
        !vec(lpi, at::kFloat, T) || !vec(adv, at::kFloat, T) || !vec(old, at::kFloat, T) ||
        !vec(mask, at::kByte, T) || !on_gpu(cu) || !on_gpu(dz_in))
        return none();
    if (cu && (cu->scalar_type() != at::kInt || cu->dim() != 1))
        return none();
    if (a[10] == Py_None)
        V = z->size(1);
    else if (!integer(a[10], V))
        return none();
    at::ScalarType dt = z->scalar_type();
    if (a[9] != Py_None) {
        if (!THPDtype_Check(a[9]))
            return none();
        dt = reinterpret_cast<THPDtype *>(a[9])->scalar_type;
    }
    if (dz_in)
        dt = dz_in->scalar_type();
    if (!dtype_code(dt, code_out) || V < 0)
        return none();
    if (dz_in && (!rows(*dz_in, To, ldo) || To != T || dz_in->size(1) < V))
        return none();
    size_t need = 0;
    if (lib.loss_ws(T, V, &need) != CIS_OK)
        return none();
    const at::Device dev = z->device();
    const Tensor dz = dz_in ? *dz_in : fresh({T, V}, dt, dev);
    rows(dz, To, ldo);
    const Tensor lp = fresh_if(want[0], T, at::kFloat, dev), w = fresh_if(want[1], T, at::kFloat, dev);
    const Tensor tr = fresh_if(want[2], T, at::kByte, dev);
    const Tensor ent = fresh_if(want_ent, T, at::kFloat, dev);
    const Tensor stats = fresh({(int64_t)sizeof(cis_stats_t)}, at::kByte, dev);
    const Tensor loss = fresh({1}, at::kDouble, dev);
    const Tensor ws = ws_in && ws_in->numel() >= (int64_t)need ? *ws_in
                                                               : fresh({(int64_t)need}, at::kByte, dev);
    const void *pz = ptr(z);
    const int32_t *pids = ptr<int32_t>(ids), *pcu = ptr<int32_t>(cu);
    const float *plpi = ptr<float>(lpi), *pold = ptr<float>(old), *padv = ptr<float>(adv);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    const int64_t nseq = cu ? cu->size(0) - 1 : 0;
    void *pdz = ptr(dz), *pws = ptr(ws);
    float *plp = ptr<float>(lp), *pw = ptr<float>(w), *pent = ptr<float>(ent);
    uint8_t *ptrunc = ptr<uint8_t>(tr);
    cis_stats_t *pstats = ptr<cis_stats_t>(stats);
    double *ploss = ptr<double>(loss);
    const size_t nws = (size_t)ws.numel();
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.loss(pz, code, T, V, ld, pids, plpi, pold, padv, pmask, pcu, nseq, &P, pdz, code_out,
                  ldo, plp, pw, ptrunc, pent, pstats, ploss, pws, nws, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return dict({{"dlogits", dz}, {"lp", lp}, {"w", w}, {"trunc", tr}, {"entropy", ent},
                 {"loss", loss}, {"stats", stats}, {"workspace", ws}});
    END_HANDLE_TH_ERRORS
}

// (logits, ids, mask, V, want_lse, dev_status, want_entropy)
PyObject *token_logprobs(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *z, *ids, *mask, *st;
    bool want_lse, want_ent;
    if (n != 7 || !take(a[0], z) || !take(a[1], ids) || !take(a[2], mask) ||
        !flag(a[4], want_lse) || !take(a[5], st) || !flag(a[6], want_ent))
        return none();
    int64_t T, ld, V;
    int32_t code;
    if (!z || !ids || !z->is_cuda() || !rows(*z, T, ld) || !dtype_code(z->scalar_type(), code) ||
        !vec(ids, at::kInt, T) || !vec(mask, at::kByte, T))
        return none();
    if (a[3] == Py_None)
        V = z->size(1);
    else if (!integer(a[3], V))
        return none();
    const at::Device dev = z->device();
    const Tensor lp = fresh({T}, at::kFloat, dev), lse = fresh_if(want_lse, T, at::kFloat, dev);
    const Tensor ent = fresh_if(want_ent, T, at::kFloat, dev);
    const void *pz = ptr(z);
    const int32_t *pids = ptr<int32_t>(ids);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    float *plp = ptr<float>(lp), *plse = ptr<float>(lse), *pent = ptr<float>(ent);
    int32_t *pst = ptr<int32_t>(st);
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.logprobs(pz, code, T, V, ld, pids, pmask, plp, plse, pent, pst, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    if (want_ent)
        return Py_BuildValue("NNN", wrap(lp), wrap(lse), wrap(ent));
    return want_lse ? Py_BuildValue("NN", wrap(lp), wrap(lse)) : wrap(lp);
    END_HANDLE_TH_ERRORS
}

// (lp_train, lp_infer, params, mask, want_trunc, want_eps, cu_seqlens)
PyObject *weights(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *lt, *li, *mask, *cu;
    cis_params_t P;
    bool want_tr, want_eps;
    if (n != 7 || !take(a[0], lt) || !take(a[1], li) || !params(a[2], P) || !take(a[3], mask) ||
        !flag(a[4], want_tr) || !flag(a[5], want_eps) || !take(a[6], cu))
        return none();
    if (!lt || !li || lt->dim() != 1)
        return none();
    const int64_t T = lt->size(0);
    if (!vec(lt, at::kFloat, T) || !vec(li, at::kFloat, T) || !vec(mask, at::kByte, T))
        return none();
    if (cu && (!cu->is_cuda() || cu->scalar_type() != at::kInt || cu->dim() != 1 ||
               !cu->is_contiguous()))
        return none();
    const at::Device dev = lt->device();
    const Tensor w = fresh({T}, at::kFloat, dev), tr = fresh_if(want_tr, T, at::kByte, dev);
    const Tensor eps = fresh_if(want_eps, T, at::kFloat, dev);
    const float *plt = ptr<float>(lt), *pli = ptr<float>(li);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    const int32_t *pcu = ptr<int32_t>(cu);
    const int64_t nseq = cu ? cu->size(0) - 1 : 0;
    float *pw = ptr<float>(w), *peps = ptr<float>(eps);
    uint8_t *ptrunc = ptr<uint8_t>(tr);
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.weights(plt, pli, pmask, T, pcu, nseq, &P, pw, ptrunc, peps, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return Py_BuildValue("NNN", wrap(w), wrap(tr), wrap(eps));
    END_HANDLE_TH_ERRORS
}

// (key, edges, values, mask): edges a list or tuple of floats or ints, values
// one of tensors
PyObject *binned_sums(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *key, *mask, *v;
    if (n != 4 || !take(a[0], key) || !take(a[3], mask) || !key || key->dim() != 1 ||
        !(PyList_CheckExact(a[1]) || PyTuple_CheckExact(a[1])) ||
        !(PyList_CheckExact(a[2]) || PyTuple_CheckExact(a[2])))
        return none();
    const int64_t T = key->size(0);
    const Py_ssize_t ne = PySequence_Fast_GET_SIZE(a[1]), nv = PySequence_Fast_GET_SIZE(a[2]);
    if (!vec(key, at::kFloat, T) || !vec(mask, at::kByte, T) || ne < 2 || ne > CIS_MAX_BINS + 1 ||
        nv > CIS_MAX_BIN_VALUES)
        return none();
    double edges[CIS_MAX_BINS + 1];
    for (Py_ssize_t i = 0; i < ne; ++i) {
        PyObject *e = PySequence_Fast_GET_ITEM(a[1], i);
        if (!PyFloat_CheckExact(e))
            return none();
        edges[i] = PyFloat_AS_DOUBLE(e);
    }
    const float *vals[CIS_MAX_BIN_VALUES] = {};
    for (Py_ssize_t i = 0; i < nv; ++i) {
        if (!take(PySequence_Fast_GET_ITEM(a[2], i), v) || !v || !vec(v, at::kFloat, T))
            return none();
        vals[i] = ptr<float>(v);
    }
    const int32_t nb = (int32_t)ne - 1;
    size_t need = 0;
    if (lib.bins_ws(T, nb, (int32_t)nv, &need) != CIS_OK)
        return none();
    const at::Device dev = key->device();
    const Tensor ws = fresh({(int64_t)need + 256}, at::kByte, dev);
    const Tensor counts = fresh({(int64_t)nb}, at::kLong, dev);
    const Tensor sums = fresh({(int64_t)nv, (int64_t)nb}, at::kDouble, dev);
    uint8_t *w = ptr<uint8_t>(ws);
    w += (256 - (reinterpret_cast<uintptr_t>(w) & 255)) & 255;
    const float *pkey = ptr<float>(key);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    int64_t *pcounts = ptr<int64_t>(counts);
    double *psums = nv ? ptr<double>(sums) : nullptr;
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.bins(pkey, pmask, T, edges, nb, nv ? vals : nullptr, (int32_t)nv, pcounts, psums, w,
                  need, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return Py_BuildValue("NN", wrap(counts), wrap(sums));
    END_HANDLE_TH_ERRORS
}

// (logits_train, logits_infer, ids, params, mask, V, dev_status)
PyObject *mismatch_diagnostics(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *zt, *zi, *ids, *mask, *st;
    cis_params_t P;
    if (n != 7 || !take(a[0], zt) || !take(a[1], zi) || !take(a[2], ids) || !params(a[3], P) ||
        !take(a[4], mask) || !take(a[6], st))
        return none();
    int64_t T, Ti, ldt, ldi, V;
    int32_t code;
    if (!zt || !zi || !ids || !zt->is_cuda() || !zi->is_cuda() ||
        zt->scalar_type() != zi->scalar_type() || !rows(*zt, T, ldt) || !rows(*zi, Ti, ldi) ||
        Ti != T || !dtype_code(zt->scalar_type(), code) || !vec(ids, at::kInt, T) ||
        !vec(mask, at::kByte, T))
        return none();
    if (a[5] == Py_None)
        V = std::min(zt->size(1), zi->size(1));
    else if (!integer(a[5], V))
        return none();
    const at::Device dev = zt->device();
    Tensor o[5];
    for (Tensor &t : o)
        t = fresh({T}, at::kFloat, dev);
    const void *pzt = ptr(zt), *pzi = ptr(zi);
    const int32_t *pids = ptr<int32_t>(ids);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    float *po[5];
    for (int i = 0; i < 5; ++i)
        po[i] = ptr<float>(o[i]);
    int32_t *pst = ptr<int32_t>(st);
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.diagnostics(pzt, pzi, code, T, V, ldt, ldi, pids, pmask, &P, po[0], po[1], po[2],
                         po[3], po[4], pst, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return dict({{"eps", o[0]}, {"logk", o[1]}, {"p", o[2]}, {"bias2", o[3]}, {"dvar", o[4]}});
    END_HANDLE_TH_ERRORS
}

// (logits, u, temperature, top_k, top_p, min_p, mask, V, want_lp, want_lp_sampled, dev_status)
PyObject *sample_tokens(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *z, *u, *tau, *k, *p, *m, *mask, *st;
    bool want_lp, want_lps;
    if (n != 11 || !take(a[0], z) || !take(a[1], u) || !take(a[2], tau) || !take(a[3], k) ||
        !take(a[4], p) || !take(a[5], m) || !take(a[6], mask) || !flag(a[8], want_lp) ||
        !flag(a[9], want_lps) || !take(a[10], st))
        return none();
    int64_t T, ld, V;
    int32_t code;
    if (!z || !u || !together(*z, {u, tau, k, p, m, mask, st}) || !rows(*z, T, ld) ||
        !dtype_code(z->scalar_type(), code) || !vocabulary(a[7], *z, V) ||
        !vec(u, at::kFloat, T) || !vec(tau, at::kFloat, T) || !vec(k, at::kInt, T) ||
        !vec(p, at::kFloat, T) || !vec(m, at::kFloat, T) || !vec(mask, at::kByte, T) ||
        !status(st))
        return none();
    const at::Device dev = z->device();
    const Tensor ids = fresh({T}, at::kInt, dev), lp = fresh_if(want_lp, T, at::kFloat, dev);
    const Tensor lps = fresh_if(want_lps, T, at::kFloat, dev);
    const void *pz = ptr(z);
    const float *pu = ptr<float>(u), *ptau = ptr<float>(tau), *pp = ptr<float>(p);
    const float *pm = ptr<float>(m);
    const int32_t *pk = ptr<int32_t>(k);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    int32_t *pids = ptr<int32_t>(ids), *pst = ptr<int32_t>(st);
    float *plp = ptr<float>(lp), *plps = ptr<float>(lps);
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.sample(pz, code, T, V, ld, pu, ptau, pk, pp, pm, pmask, pids, plp, plps, pst, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return Py_BuildValue("NNN", wrap(ids), wrap(lp), wrap(lps));
    END_HANDLE_TH_ERRORS
}

// (logits, K, temperature, mask, V, want_lse, dev_status)
PyObject *topk_logprobs(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *z, *mask, *st;
    bool want_lse;
    int64_t T, ld, V, K;
    int32_t code;
    if (n != 7 || !take(a[0], z) || !integer(a[1], K) || !PyFloat_CheckExact(a[2]) ||
        !take(a[3], mask) || !flag(a[5], want_lse) || !take(a[6], st))
        return none();
    if (!z || !together(*z, {mask, st}) || !rows(*z, T, ld) ||
        !dtype_code(z->scalar_type(), code) || !vocabulary(a[4], *z, V) ||
        !vec(mask, at::kByte, T) || !status(st) || K < 1 || K > CIS_MAX_TOPK)
        return none();
    const double tau = PyFloat_AS_DOUBLE(a[2]);
    const at::Device dev = z->device();
    const Tensor ids = fresh({T, K}, at::kInt, dev), lp = fresh({T, K}, at::kFloat, dev);
    const Tensor lse = fresh_if(want_lse, T, at::kFloat, dev);
    const void *pz = ptr(z);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    int32_t *pids = ptr<int32_t>(ids), *pst = ptr<int32_t>(st);
    float *plp = ptr<float>(lp), *plse = ptr<float>(lse);
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.topk(pz, code, T, V, ld, (int32_t)K, tau, pmask, pids, plp, plse, pst, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return Py_BuildValue("NNN", wrap(ids), wrap(lp), wrap(lse));
    END_HANDLE_TH_ERRORS
}

// (logits, top_ids, top_lp, params, token_weight, mask, cu_seqlens, dlogits, dlogits_dtype, V,
//  want_grad, workspace)
PyObject *distill_fwd_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *z, *ids, *lp, *w, *mask, *cu, *dz_in, *ws_in;
    cis_distill_params_t P;
    bool grad;
    if (n != 12 || !take(a[0], z) || !take(a[1], ids) || !take(a[2], lp) ||
        !params_of(a[3], distill_type, P) || !take(a[4], w) || !take(a[5], mask) ||
        !take(a[6], cu) || !take(a[7], dz_in) || !flag(a[10], grad) || !take(a[11], ws_in))
        return none();
    int64_t T, ld, V, To, ldo, Tl, ldl, Tp, ldp;
    int32_t code, code_out;
    if (!z || !ids || !lp || !together(*z, {ids, lp, w, mask, cu, dz_in, ws_in}) ||
        !rows(*z, T, ld) || !dtype_code(z->scalar_type(), code) || !vocabulary(a[9], *z, V) ||
        V < 0 || !rows(*ids, Tl, ldl) || !rows(*lp, Tp, ldp) || Tl != T || Tp != T ||
        ldl != ldp || ids->size(1) != lp->size(1) || ids->scalar_type() != at::kInt ||
        lp->scalar_type() != at::kFloat || !vec(w, at::kFloat, T) || !vec(mask, at::kByte, T))
        return none();
    if ((cu && (cu->scalar_type() != at::kInt || cu->dim() != 1 || !cu->is_contiguous())) ||
        (ws_in && !ws_in->is_contiguous()))
        return none();
    at::ScalarType dt = z->scalar_type();
    if (a[8] != Py_None) {
        if (!THPDtype_Check(a[8]))
            return none();
        dt = reinterpret_cast<THPDtype *>(a[8])->scalar_type;
    }
    if (dz_in)
        dt = dz_in->scalar_type();
    if (!dtype_code(dt, code_out) || ids->size(1) > CIS_MAX_TOPK ||
        (dz_in && (!rows(*dz_in, To, ldo) || To != T || dz_in->size(1) < V)))
        return none();
    size_t need = 0;
    if (lib.distill_ws(T, &need) != CIS_OK)
        return none();
    const at::Device dev = z->device();
    Tensor dz;
    ldo = V;
    if (dz_in)
        dz = *dz_in;
    else if (grad)
        dz = fresh({T, V}, dt, dev);
    if (dz.defined())
        rows(dz, To, ldo);
    const Tensor kl = fresh({T}, at::kFloat, dev), loss = fresh({1}, at::kDouble, dev);
    const Tensor ws = ws_in && ws_in->numel() >= (int64_t)need ? *ws_in
                                                               : fresh({(int64_t)need}, at::kByte, dev);
    const void *pz = ptr(z);
    const int32_t *pids = ptr<int32_t>(ids), *pcu = ptr<int32_t>(cu);
    const float *plp = ptr<float>(lp), *pw = ptr<float>(w);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    const int32_t K = (int32_t)ids->size(1);
    const int64_t nseq = cu ? cu->size(0) - 1 : 0;
    void *pdz = ptr(dz), *pws = ptr(ws);
    float *pkl = ptr<float>(kl);
    double *ploss = ptr<double>(loss);
    const size_t nws = (size_t)ws.numel();
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.distill(pz, code, T, V, ld, pids, plp, K, ldl, pw, pmask, pcu, nseq, &P, pdz,
                     code_out, ldo, pkl, ploss, pws, nws, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return dict({{"dlogits", dz}, {"kl", kl}, {"loss", loss}, {"workspace", ws}});
    END_HANDLE_TH_ERRORS
}

// None, or [T, H] rows of `dt` with unit column stride.
bool like(const Tensor *t, int64_t T, int64_t H, at::ScalarType dt, int64_t &ld)
{
    int64_t n;
    ld = H;
    return t == nullptr ||
           (t->scalar_type() == dt && rows(*t, n, ld) && n == T && t->size(1) == H);
}
bool norm_weight(const Tensor *w, int64_t H, int32_t &code)
{
    return w && w->dim() == 1 && w->size(0) == H && w->is_contiguous() &&
           dtype_code(w->scalar_type(), code);
}

// (x, weight, residual, eps, mask, want_y, want_q)
PyObject *rmsnorm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *x, *w, *r, *mask;
    bool want_y, want_q;
    int64_t T, ld, ldr;
    int32_t code, wcode;
    if (n != 7 || !take(a[0], x) || !take(a[1], w) || !take(a[2], r) ||
        !PyFloat_CheckExact(a[3]) || !take(a[4], mask) || !flag(a[5], want_y) ||
        !flag(a[6], want_q))
        return none();
    if (!x || !w || !together(*x, {w, r, mask}) || !rows(*x, T, ld) ||
        !dtype_code(x->scalar_type(), code))
        return none();
    const int64_t H = x->size(1);
    const at::ScalarType dt = x->scalar_type();
    if (!like(r, T, H, dt, ldr) || !norm_weight(w, H, wcode) || !vec(mask, at::kByte, T) ||
        !(want_y || want_q || r))
        return none();
    const double eps = PyFloat_AS_DOUBLE(a[3]);
    const at::Device dev = x->device();
    const Tensor h = r ? fresh({T, H}, dt, dev) : Tensor();
    const Tensor y = want_y ? fresh({T, H}, dt, dev) : Tensor();
    const Tensor q = want_q ? fresh({T, H}, at::kFloat8_e4m3fn, dev) : Tensor();
    const Tensor sc = fresh_if(want_q, T, at::kFloat, dev);
    const void *px = ptr(x), *pw = ptr(w), *pr = ptr(r);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    void *ph = ptr(h), *py = ptr(y), *pq = ptr(q);
    float *psc = ptr<float>(sc);
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.norm(px, code, T, H, ld, pr, ldr, pw, wcode, eps, pmask, ph, py, pq, psc, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return dict({{"h", h}, {"y", y}, {"q", q}, {"scale", sc}});
    END_HANDLE_TH_ERRORS
}

// (dy, h, weight, dh, eps, mask, workspace)
PyObject *rmsnorm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *dy, *h, *w, *dh, *mask, *ws_in;
    int64_t T, ldh, ldy, lddh;
    int32_t code, wcode;
    if (n != 7 || !take(a[0], dy) || !take(a[1], h) || !take(a[2], w) || !take(a[3], dh) ||
        !PyFloat_CheckExact(a[4]) || !take(a[5], mask) || !take(a[6], ws_in))
        return none();
    if (!dy || !h || !w || !together(*h, {dy, w, dh, mask, ws_in}) || !rows(*h, T, ldh) ||
        !dtype_code(h->scalar_type(), code))
        return none();
    const int64_t H = h->size(1);
    const at::ScalarType dt = h->scalar_type();
    size_t need = 0;
    if (!like(dy, T, H, dt, ldy) || !like(dh, T, H, dt, lddh) || !norm_weight(w, H, wcode) ||
        !vec(mask, at::kByte, T) || (ws_in && !ws_in->is_contiguous()) ||
        lib.norm_bwd_ws(T, H, &need) != CIS_OK)
        return none();
    const double eps = PyFloat_AS_DOUBLE(a[4]);
    const at::Device dev = h->device();
    const Tensor dx = fresh({T, H}, dt, dev), dw = fresh({H}, at::kFloat, dev);
    const Tensor ws = ws_in && ws_in->nbytes() >= need ? *ws_in
                                                       : fresh({(int64_t)need}, at::kByte, dev);
    const void *pdy = ptr(dy), *ph = ptr(h), *pw = ptr(w), *pdh = ptr(dh);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    void *pdx = ptr(dx), *pws = ptr(ws);
    float *pdw = ptr<float>(dw);
    const size_t nws = ws.nbytes();
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.norm_bwd(pdy, ph, code, T, H, ldy, ldh, pw, wcode, pdh, lddh, eps, pmask, pdx, pdw,
                      pws, nws, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return dict({{"dx", dx}, {"dweight", dw}});
    END_HANDLE_TH_ERRORS
}

// A contiguous matrix of 8-bit numbers, and a scale a row.
bool e4m3_rows(const Tensor *x, const Tensor *scale)
{
    return x && scale && x->dim() == 2 && x->scalar_type() == at::kFloat8_e4m3fn &&
           x->is_contiguous() && vec(scale, at::kFloat, x->size(0));
}

// (hidden, hidden_scale, weight, weight_scale, logits_dtype, logits, dev_status)
PyObject *lmhead_logits(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *x, *xs, *w, *ws, *z_in, *st;
    if (n != 7 || !take(a[0], x) || !take(a[1], xs) || !take(a[2], w) || !take(a[3], ws) ||
        !THPDtype_Check(a[4]) || !take(a[5], z_in) || !take(a[6], st))
        return none();
    if (!e4m3_rows(x, xs) || !e4m3_rows(w, ws) || !together(*x, {xs, w, ws, z_in, st}) ||
        x->size(1) != w->size(1) || !status(st))
        return none();
    const int64_t T = x->size(0), H = x->size(1), V = w->size(0);
    at::ScalarType dt = reinterpret_cast<THPDtype *>(a[4])->scalar_type;
    int64_t To, ld = V;
    int32_t code;
    if (z_in && (!rows(*z_in, To, ld) || To != T || z_in->size(1) < V))
        return none();
    if (z_in)
        dt = z_in->scalar_type();
    if (!dtype_code(dt, code))
        return none();
    const Tensor z = z_in ? *z_in : fresh({T, V}, dt, x->device());
    const void *px = ptr(x), *pw = ptr(w);
    const float *pxs = ptr<float>(xs), *pws = ptr<float>(ws);
    void *pz = ptr(z);
    int32_t *pst = ptr<int32_t>(st);
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.head(px, pxs, pw, pws, T, H, V, pz, code, ld, pst, s);
    Py_END_ALLOW_THREADS
    return rc != CIS_OK ? PyLong_FromLong(rc) : wrap(z);
    END_HANDLE_TH_ERRORS
}

// (logits, draft_ids, cu_drafts, u, u_last, max_drafts, draft_logits, temperature,
//  draft_temperature, mask, V, want_lp, want_lp_sampled, dev_status, workspace)
PyObject *verify_tokens(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    const Tensor *z, *ids, *cu, *u, *ul, *zd, *tau, *taud, *mask, *st, *ws_in;
    bool want_lp, want_lps;
    int64_t D, T, ld, V, Td, ldd;
    int32_t code;
    if (n != 15 || !take(a[0], z) || !take(a[1], ids) || !take(a[2], cu) || !take(a[3], u) ||
        !take(a[4], ul) || !integer(a[5], D) || !take(a[6], zd) || !take(a[7], tau) ||
        !take(a[8], taud) || !take(a[9], mask) || !flag(a[11], want_lp) ||
        !flag(a[12], want_lps) || !take(a[13], st) || !take(a[14], ws_in))
        return none();
    if (!z || !ids || !cu || !u || !ul ||
        !together(*z, {ids, cu, u, ul, zd, tau, taud, mask, st, ws_in}) || !rows(*z, T, ld) ||
        !dtype_code(z->scalar_type(), code) || !vocabulary(a[10], *z, V) || D < 0 ||
        D > CIS_MAX_DRAFTS || cu->dim() != 1 || cu->size(0) < 1)
        return none();
    const int64_t B = cu->size(0) - 1, N = ids->numel();
    size_t need = 0;
    if (T != N + B || N > B * D || !vec(cu, at::kInt, B + 1) || !vec(ids, at::kInt, N) ||
        !vec(u, at::kFloat, N) || !vec(ul, at::kFloat, B) || !vec(tau, at::kFloat, B) ||
        !vec(taud, at::kFloat, B) || !vec(mask, at::kByte, B) || !status(st) ||
        (ws_in && !ws_in->is_contiguous()) ||
        lib.verify_ws(B, V, (int32_t)D, &need) != CIS_OK)
        return none();
    ldd = V;
    if (zd && (zd->scalar_type() != z->scalar_type() || !rows(*zd, Td, ldd) || Td != N ||
               zd->size(1) < V))
        return none();
    const at::Device dev = z->device();
    const Tensor tok = fresh({B, D + 1}, at::kInt, dev), kept = fresh({B}, at::kInt, dev);
    const Tensor lp = want_lp ? fresh({B, D + 1}, at::kFloat, dev) : Tensor();
    const Tensor lps = want_lps ? fresh({B, D + 1}, at::kFloat, dev) : Tensor();
    const Tensor ws = ws_in && ws_in->nbytes() >= need ? *ws_in
                                                       : fresh({(int64_t)need}, at::kByte, dev);
    const void *pz = ptr(z), *pzd = ptr(zd);
    const int32_t *pids = ptr<int32_t>(ids), *pcu = ptr<int32_t>(cu);
    const float *pu = ptr<float>(u), *pul = ptr<float>(ul), *ptau = ptr<float>(tau);
    const float *ptaud = ptr<float>(taud);
    const uint8_t *pmask = ptr<uint8_t>(mask);
    int32_t *ptok = ptr<int32_t>(tok), *pkept = ptr<int32_t>(kept), *pst = ptr<int32_t>(st);
    float *plp = ptr<float>(lp), *plps = ptr<float>(lps);
    void *pws = ptr(ws);
    const size_t nws = ws.nbytes();
    int rc;
    void *s = stream();
    Py_BEGIN_ALLOW_THREADS
    rc = lib.verify(pz, code, B, N, V, ld, pids, pcu, (int32_t)D, pzd, ldd, pu, pul, ptau, ptaud,
                    pmask, ptok, pkept, plp, plps, pst, pws, nws, s);
    Py_END_ALLOW_THREADS
    if (rc != CIS_OK)
        return PyLong_FromLong(rc);
    return Py_BuildValue("NNNN", wrap(tok), wrap(kept), wrap(lp), wrap(lps));
    END_HANDLE_TH_ERRORS
}

// init(path, params type, distillation's params type): the library's entry points, and the
// types of `params`.
PyObject *init(PyObject *, PyObject *args)
{
    const char *path;
    PyObject *type, *distill;
    if (!PyArg_ParseTuple(args, "sOO", &path, &type, &distill))
        return nullptr;
    void *h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (h == nullptr)
        return PyErr_Format(PyExc_ImportError, "%s", dlerror());
    bool ok = true;
    auto get = [&](auto &f, const char *name) {
        f = reinterpret_cast<std::decay_t<decltype(f)>>(dlsym(h, name));
        ok = ok && f != nullptr;
    };
    get(lib.loss_ws, "cis_loss_workspace_size");
    get(lib.loss, "cis_loss_fwd_bwd");
    get(lib.logprobs, "cis_token_logprobs");
    get(lib.weights, "cis_weights");
    get(lib.bins_ws, "cis_binned_sums_workspace_size");
    get(lib.bins, "cis_binned_sums");
    get(lib.diagnostics, "cis_mismatch_diagnostics");
    get(lib.sample, "cis_sample_tokens");
    get(lib.topk, "cis_topk_logprobs");
    get(lib.distill_ws, "cis_distill_workspace_size");
    get(lib.distill, "cis_distill_fwd_bwd");
    get(lib.norm, "cis_rmsnorm_fwd");
    get(lib.norm_bwd_ws, "cis_rmsnorm_bwd_workspace_size");
    get(lib.norm_bwd, "cis_rmsnorm_bwd");
    get(lib.head, "cis_lmhead_logits");
    get(lib.verify_ws, "cis_verify_workspace_size");
    get(lib.verify, "cis_verify_tokens");
    if (!ok)
        return PyErr_Format(PyExc_ImportError, "%s lacks an entry point", path);
    Py_INCREF(type);
    Py_XSETREF(params_type, type);
    Py_INCREF(distill);
    Py_XSETREF(distill_type, distill);
    return none();
}

template <typename F> PyCFunction fast(F f)
{
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef methods[] = {
    {"init", init, METH_VARARGS, nullptr},
    {"loss_fwd_bwd", fast(loss_fwd_bwd), METH_FASTCALL, nullptr},
    {"token_logprobs", fast(token_logprobs), METH_FASTCALL, nullptr},
    {"weights", fast(weights), METH_FASTCALL, nullptr},
    {"binned_sums", fast(binned_sums), METH_FASTCALL, nullptr},
    {"mismatch_diagnostics", fast(mismatch_diagnostics), METH_FASTCALL, nullptr},
    {"sample_tokens", fast(sample_tokens), METH_FASTCALL, nullptr},
    {"topk_logprobs", fast(topk_logprobs), METH_FASTCALL, nullptr},
    {"rmsnorm_fwd", fast(rmsnorm_fwd), METH_FASTCALL, nullptr},
    {"rmsnorm_bwd", fast(rmsnorm_bwd), METH_FASTCALL, nullptr},
    {"lmhead_logits", fast(lmhead_logits), METH_FASTCALL, nullptr},
    {"verify_tokens", fast(verify_tokens), METH_FASTCALL, nullptr},
    {"distill_fwd_bwd", fast(distill_fwd_bwd), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_cis_native", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__cis_native() { return PyModule_Create(&module); }
