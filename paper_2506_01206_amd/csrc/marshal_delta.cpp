// Argument marshalling of the gated-delta layer core and of the constrained choice of children (binding.py), as marshal.cpp does
// it for the other entry points; its functions stand in the module of their own `_marshal._delta`, compiled into the same library.
// Here every tensor has to live on the GPU that is current, the one whose stream the call goes to.
#include "marshal.h"

#include <cmath>

namespace {

struct Api {
    decltype(&::mamba_gated_delta_workspace_bytes) gated_delta_workspace_bytes;
    decltype(&::mamba_gated_delta_fwd) gated_delta_fwd;
    decltype(&::mamba_gated_delta_step) gated_delta_step;
    decltype(&::mamba_token_counts) token_counts;
    decltype(&::mamba_logits_constrain_fwd) logits_constrain_fwd;
    decltype(&::mamba_topk_constrained_workspace_bytes) topk_constrained_workspace_bytes;
    decltype(&::mamba_topk_constrained_fwd) topk_constrained_fwd;
} api;

float number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyFailed();
    return (float)v;
}

// scale: N^-1/2 for None
float scale_of(PyObject *o, int64_t N) { return o == Py_None ? (float)(1.0 / std::sqrt((double)(N > 0 ? N : 1))) : number(o); }

PyObject *gated_delta_fwd(Args a)
{
    PyObject *q = a[0], *v = a[2];
    Out out(a[10]), h_final(a[11]);
    const at::Tensor &vt = tensor(v, "v");
    const auto s = sizes(v, "v", 4), qs = sizes(q, "q", 4);
    const int64_t B = s[0], L = s[1], H = s[2], P = s[3], Hk = qs[2], N = qs[3];
    const auto type = vt.scalar_type();
    const int io = io_code(vt);
    placed(vt, "v");
    out.unless_given(vt, s, type);
    if (flag(a[13])) h_final.unless_given(vt, {B, H, P, N}, at::kFloat);
    const Workspace ws(a[12], io == MAMBA_BF16 ? api.gated_delta_workspace_bytes(B, L, H, Hk, P, N) : 0, vt);
    const void *qp = ptr(q, type, {B, L, Hk, N}, "q"), *kp = ptr(a[1], type, {B, L, Hk, N}, "k"), *dtp = ptr(a[3], type, {B, L, H}, "dt");
    const float *A = fptr(a[4], {H}, "A");
    const void *bp = ptr(a[5], type, {B, L, H}, "beta"), *zp = ptr(a[6], type, {B, L, H, P}, "z");
    const float *nw = fptr(a[7], {P}, "norm_w"), *db = fptr(a[8], {H}, "dt_bias"), *h0 = fptr(a[9], {B, H, P, N}, "h0");
    void *op = ptr(out.object, type, {B, L, H, P}, "out");
    float *hf = fptr(h_final.object, {B, H, P, N}, "h_final");
    on_current_device({q, a[1], v, a[3], a[4], a[5], a[6], a[7], a[8], a[9], out.object, h_final.object, a[12]});
    Call{"mamba_gated_delta_fwd", api.gated_delta_fwd, qp, kp, static_cast<const void *>(pointer(vt)), dtp, A, bp, zp, nw, db, h0, op, hf,
         ws.data, ws.bytes, B, L, H, Hk, P, N, scale_of(a[14], N), number(a[15]), flag(a[16]), flag(a[17]), flag(a[18]), io, stream_of(a[19])};
    return result({out.object, h_final.object});
}

PyObject *gated_delta_step(Args a)
{
    PyObject *h_in = a[0], *q = a[1], *v = a[3], *parent = a[10];
    Out h_out(a[11]), out(a[12]);
    const at::Tensor &vt = tensor(v, "v");
    const auto s = sizes(v, "v", 3), qs = sizes(q, "q", 3);
    const int64_t n_in = sizes(h_in, "h_in", 4)[0], n_out = s[0], H = s[1], P = s[2], Hk = qs[1], N = qs[2];
    const auto type = vt.scalar_type();
    const int io = io_code(vt);
    placed(vt, "v");
    h_out.unless_given(vt, {n_out, H, P, N}, at::kFloat);
    out.unless_given(vt, s, type);
    float *ho = fptr(h_out.object, {n_out, H, P, N}, "h_out");
    const float *hi = fptr(h_in, {n_in, H, P, N}, "h_in");
    const int32_t *pp = static_cast<const int32_t *>(ptr(parent, at::kInt, {n_out}, "parent_idx"));
    const void *qp = ptr(q, type, {n_out, Hk, N}, "q"), *kp = ptr(a[2], type, {n_out, Hk, N}, "k"), *dtp = ptr(a[4], type, {n_out, H}, "dt");
    const float *A = fptr(a[5], {H}, "A");
    const void *bp = ptr(a[6], type, {n_out, H}, "beta"), *zp = ptr(a[7], type, {n_out, H, P}, "z");
    const float *nw = fptr(a[8], {P}, "norm_w"), *db = fptr(a[9], {H}, "dt_bias");
    void *op = ptr(out.object, type, {n_out, H, P}, "out");
    on_current_device({h_in, q, a[2], v, a[4], a[5], a[6], a[7], a[8], a[9], parent, h_out.object, out.object});
    Call{"mamba_gated_delta_step", api.gated_delta_step, ho, hi, pp, qp, kp, static_cast<const void *>(pointer(vt)), dtp, A, bp, zp, nw, db,
         op, n_out, n_in, H, Hk, P, N, scale_of(a[13], N), number(a[14]), flag(a[15]), flag(a[16]), flag(a[17]), io, stream_of(a[18])};
    return result({h_out.object, out.object});
}

PyObject *token_counts(Args a)
{
    PyObject *tokens = a[0];
    Out counts(a[2]);
    const at::Tensor &tt = tensor(tokens, "tokens");
    const auto s = sizes(tokens, "tokens", 2);
    const int64_t S = s[0], L = s[1], V = integer(a[1]);
    placed(tt, "tokens");
    const bool given = counts.object != Py_None;
    counts.unless_given(tt, {S, V}, at::kInt);
    const int32_t *tp = static_cast<const int32_t *>(ptr(tokens, at::kInt, {S, L}, "tokens"));
    int32_t *cp = static_cast<int32_t *>(ptr(counts.object, at::kInt, {S, V}, "counts"));
    on_current_device({tokens, counts.object});
    Call{"mamba_token_counts", api.token_counts, tp, cp, S, L, V, given ? 1 : 0, flag(a[3]), stream_of(a[4])};
    Py_INCREF(counts.object);
    return counts.object;
}

// the rules of a call on logits (M, V): a[0 .. 6] are counts, penalties, seq_idx, path, bias, mask, mask_idx
mamba_constraints_t constraints(Args a, int64_t M, int64_t V)
{
    mamba_constraints_t c = {};
    if (a[0] != Py_None) c.n_seq = sizes(a[0], "counts", 2)[0];
    if (a[1] != Py_None) c.n_seq = sizes(a[1], "penalties", 2)[0];
    if (a[3] != Py_None) c.path_len = sizes(a[3], "path", 2)[1];
    if (a[5] != Py_None) c.n_masks = sizes(a[5], "mask", 2)[0];
    // (a tensor of no rows has no address, and would pass for a rule that is left out)
    if (M > 0 && a[5] != Py_None && c.n_masks == 0) fail(PyExc_ValueError, "%s must have a row", "mask");
    if (M > 0 && (a[0] != Py_None || a[1] != Py_None) && c.n_seq == 0) fail(PyExc_ValueError, "%s must have a row", a[0] != Py_None ? "counts" : "penalties");
    c.counts = static_cast<const int32_t *>(ptr(a[0], at::kInt, {c.n_seq, V}, "counts"));
    c.penalties = fptr(a[1], {c.n_seq, 3}, "penalties");
    c.seq_idx = static_cast<const int32_t *>(ptr(a[2], at::kInt, {M}, "seq_idx"));
    c.path = static_cast<const int32_t *>(ptr(a[3], at::kInt, {M, c.path_len}, "path"));
    c.bias = fptr(a[4], {V}, "bias");
    c.mask = static_cast<const int32_t *>(ptr(a[5], at::kInt, {c.n_masks, (V + 31) / 32}, "mask"));
    c.mask_idx = static_cast<const int32_t *>(ptr(a[6], at::kInt, {M}, "mask_idx"));
    on_current_device({a[0], a[1], a[2], a[3], a[4], a[5], a[6]});
    return c;
}

PyObject *logits_constrain_fwd(Args a)
{
    PyObject *logits = a[0];
    Out out(a[8]);
    const at::Tensor &lt = tensor(logits, "logits");
    const auto s = sizes(logits, "logits", 2);
    const int64_t M = s[0], V = s[1];
    const auto type = lt.scalar_type();
    const int io = io_code(lt);
    placed(lt, "logits");
    out.unless_given(lt, s, type);
    const mamba_constraints_t c = constraints(a + 1, M, V);
    void *op = ptr(out.object, type, {M, V}, "out");
    on_current_device({logits, out.object});
    Call{"mamba_logits_constrain_fwd", api.logits_constrain_fwd, static_cast<const void *>(pointer(lt)), &c, op, M, V, io, stream_of(a[9])};
    Py_INCREF(out.object);
    return out.object;
}

PyObject *topk_constrained_fwd(Args a)
{
    PyObject *logits = a[0];
    Out idx(a[9]), val(a[10]), path_out(a[11]);
    const at::Tensor &lt = tensor(logits, "logits");
    const auto s = sizes(logits, "logits", 2);
    const int64_t M = s[0], V = s[1], k = integer(a[1]);
    const int io = io_code(lt);
    placed(lt, "logits");
    if (k < 1 || k > 8) {
        PyErr_SetString(PyExc_ValueError, "k must be from 1 to 8");
        throw PyFailed();
    }
    const mamba_constraints_t c = constraints(a + 2, M, V);
    idx.unless_given(lt, {M, k}, at::kInt);
    val.unless_given(lt, {M, k}, at::kFloat);
    if (flag(a[12])) path_out.unless_given(lt, {M * k, c.path_len + 1}, at::kInt);
    const Workspace ws(a[13], api.topk_constrained_workspace_bytes(M, V, (int)k), lt);
    int32_t *ip = static_cast<int32_t *>(ptr(idx.object, at::kInt, {M, k}, "idx"));
    float *vp = fptr(val.object, {M, k}, "val");
    int32_t *pp = static_cast<int32_t *>(ptr(path_out.object, at::kInt, {M * k, c.path_len + 1}, "path_out"));
    on_current_device({logits, idx.object, val.object, path_out.object, a[13]});
    Call{"mamba_topk_constrained_fwd", api.topk_constrained_fwd, static_cast<const void *>(pointer(lt)), &c, ip, vp, pp, ws.data, ws.bytes, M, V,
         (int)k, io, stream_of(a[14])};
    return result({idx.object, val.object, path_out.object});
}

PyObject *bind(PyObject *, Args args, Py_ssize_t n) { return bind_to<Api, &api>(args, n); }

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&bind)), METH_FASTCALL, nullptr},
    MAMBA_ENTRY(gated_delta_fwd, 20), MAMBA_ENTRY(gated_delta_step, 19), MAMBA_ENTRY(token_counts, 5),
    MAMBA_ENTRY(logits_constrain_fwd, 10), MAMBA_ENTRY(topk_constrained_fwd, 15), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal._delta", "argument marshalling of the gated-delta entry points", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyObject *marshal_delta_module() { return PyModule_Create(&module); }
