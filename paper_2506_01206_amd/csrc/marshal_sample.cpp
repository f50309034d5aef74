// Argument marshalling of drawn children, the verification of trees and adapted projections (binding.py), as marshal.cpp does it for the
// other entry points; its functions stand in the module of their own `_marshal._sample`, compiled into the same library.  Here every
// tensor has to live on the GPU that is current, the one whose stream the call goes to.
#include "marshal.h"

namespace {

struct Api {
    decltype(&::mamba_sample_workspace_bytes) sample_workspace_bytes;
    decltype(&::mamba_sample_fwd) sample_fwd;
    decltype(&::mamba_tree_verify_workspace_bytes) tree_verify_workspace_bytes;
    decltype(&::mamba_tree_verify_fwd) tree_verify_fwd;
    decltype(&::mamba_linear_adapted_workspace_bytes) linear_adapted_workspace_bytes;
    decltype(&::mamba_linear_adapted_fwd) linear_adapted_fwd;
} api;

const int32_t *ints(PyObject *o, Shape shape, const char *name) { return static_cast<const int32_t *>(ptr(o, at::kInt, shape, name)); }

PyObject *sample_fwd(Args a)
{
    PyObject *logits = a[0], *u = a[1], *params = a[2], *top_k = a[3], *seq_idx = a[4], *path = a[5];
    Out idx(a[6]), prob(a[7]), dist(a[8]), path_out(a[9]);
    const at::Tensor &lt = tensor(logits, "logits");
    const auto s = sizes(logits, "logits", 2);
    const int64_t M = s[0], V = s[1], k = sizes(u, "u", 2)[1];
    const int io = io_code(lt);
    placed(lt, "logits");
    if (k < 1 || k > 8) {
        PyErr_SetString(PyExc_ValueError, "u must have from 1 to 8 columns");
        throw PyFailed();
    }
    mamba_sampling_t r = {};
    r.n_seq = sizes(params, "params", 2)[0];
    if (path != Py_None) r.path_len = sizes(path, "path", 2)[1];
    r.params = fptr(params, {r.n_seq, 3}, "params");
    r.top_k = ints(top_k, {r.n_seq}, "top_k");
    r.seq_idx = ints(seq_idx, {M}, "seq_idx");
    r.path = ints(path, {M, r.path_len}, "path");
    idx.unless_given(lt, {M, k}, at::kInt);
    prob.unless_given(lt, {M, k}, at::kFloat);
    if (flag(a[10])) dist.unless_given(lt, {M, V}, at::kFloat);
    if (flag(a[11])) path_out.unless_given(lt, {M * k, r.path_len + 1}, at::kInt);
    const Workspace ws(a[12], api.sample_workspace_bytes(M, V, (int)k), lt);
    const float *up = fptr(u, {M, k}, "u");
    int32_t *ip = const_cast<int32_t *>(ints(idx.object, {M, k}, "idx"));
    float *pp = fptr(prob.object, {M, k}, "prob"), *dp = fptr(dist.object, {M, V}, "dist");
    int32_t *op = const_cast<int32_t *>(ints(path_out.object, {M * k, r.path_len + 1}, "path_out"));
    on_current_device({logits, u, params, top_k, seq_idx, path, idx.object, prob.object, dist.object, path_out.object, a[12]});
    Call{"mamba_sample_fwd", api.sample_fwd, static_cast<const void *>(pointer(lt)), &r, up, ip, pp, dp, op, ws.data, ws.bytes, M, V, (int)k, io,
         stream_of(a[13])};
    return result({idx.object, prob.object, dist.object, path_out.object});
}

PyObject *tree_verify_fwd(Args a)
{
    PyObject *p = a[0], *q = a[1], *tokens = a[2], *u_accept = a[3], *u_sample = a[4], *tree = a[5];
    Out out(a[6]), count(a[7]), node(a[8]);
    const at::Tensor &pt = tensor(p, "p");
    const auto s = sizes(p, "p", 3);
    const int64_t S = s[0], V = s[2], gamma = PyTuple_Check(tree) ? (int64_t)PyTuple_GET_SIZE(tree) : -1;
    placed(pt, "p");
    if (gamma < 1 || gamma > MAMBA_MAX_DEPTH) {
        PyErr_Format(PyExc_ValueError, "tree must be a tuple of 1 to %d numbers", MAMBA_MAX_DEPTH);
        throw PyFailed();
    }
    int32_t fan[MAMBA_MAX_DEPTH];
    int64_t rows = 1, nodes = 1, inner = 0;
    for (int64_t i = 0; i < gamma; ++i) {
        const int64_t n = integer(PyTuple_GET_ITEM(tree, i));
        if (n < 1 || n > 8 || nodes > 65535) {
            PyErr_SetString(PyExc_ValueError, "tree must have numbers from 1 to 8, and no more than 65535 nodes");
            throw PyFailed();
        }
        fan[i] = (int32_t)n, inner = nodes, rows *= n, nodes += rows;
    }
    out.unless_given(pt, {S, gamma + 1}, at::kInt);
    count.unless_given(pt, {S}, at::kInt);
    node.unless_given(pt, {S, gamma}, at::kInt);
    const float *pp = fptr(p, {S, nodes, V}, "p"), *qp = fptr(q, {S, inner, V}, "q");
    const int32_t *tp = ints(tokens, {S, nodes - 1}, "tokens");
    const float *ua = fptr(u_accept, {S, nodes - 1}, "u_accept"), *us = fptr(u_sample, {S}, "u_sample");
    int32_t *op = const_cast<int32_t *>(ints(out.object, {S, gamma + 1}, "out")), *cp = const_cast<int32_t *>(ints(count.object, {S}, "count")),
            *np = const_cast<int32_t *>(ints(node.object, {S, gamma}, "node"));
    const Workspace ws(a[9], api.tree_verify_workspace_bytes(S), pt);
    on_current_device({p, q, tokens, u_accept, u_sample, out.object, count.object, node.object, a[9]});
    Call{"mamba_tree_verify_fwd", api.tree_verify_fwd, pp, qp, tp, ua, us, op, cp, np, ws.data, ws.bytes, static_cast<const int32_t *>(fan), (int)gamma, S, V,
         stream_of(a[10])};
    return result({out.object, count.object, node.object});
}

// widths of up to three outputs that share the columns: a[9], a[11], a[13]; the outputs a[8], a[10], a[12]; how many are to be returned: a[14]
PyObject *linear_adapted_fwd(Args a)
{
    PyObject *x = a[0], *w = a[1], *lora_a = a[2], *lora_b = a[3], *idx = a[4], *scale = a[5], *bias = a[6], *residual = a[7];
    Out out[3] = {Out(a[8]), Out(a[10]), Out(a[12])};
    const int64_t width[3] = {integer(a[9]), integer(a[11]), integer(a[13])}, used = integer(a[14]);
    const at::Tensor &xt = tensor(x, "x");
    const auto s = sizes(x, "x", 2), as = sizes(lora_a, "lora_a", 3);
    const int64_t M = s[0], K = s[1], N = sizes(w, "w", 2)[0], n = as[0], rank = as[1];
    placed(xt, "x");
    if (xt.scalar_type() != at::kBFloat16) typed(xt, at::kBFloat16, "x");
    const at::ScalarType bf = at::kBFloat16;
    for (int i = 0; i < 3; ++i)
        if (i < used) out[i].unless_given(xt, {M, width[i]}, bf);
    const Workspace ws(a[15], api.linear_adapted_workspace_bytes(M, rank), xt);
    const void *wp = ptr(w, bf, {N, K}, "w"), *ap = ptr(lora_a, bf, {n, rank, K}, "lora_a"), *bp = ptr(lora_b, bf, {n, N, rank}, "lora_b");
    const int32_t *ip = ints(idx, {M}, "adapter_idx");
    const float *sp = fptr(scale, {n}, "scale"), *bias_p = fptr(bias, {N}, "bias");
    const void *rp = ptr(residual, bf, {M, N}, "residual");
    void *op[3];
    const char *const names[3] = {"outs[0]", "outs[1]", "outs[2]"};
    for (int i = 0; i < 3; ++i) op[i] = ptr(out[i].object, bf, {M, width[i]}, names[i]);
    on_current_device({x, w, lora_a, lora_b, idx, scale, bias, residual, out[0].object, out[1].object, out[2].object, a[15]});
    Call{"mamba_linear_adapted_fwd", api.linear_adapted_fwd, static_cast<const void *>(pointer(xt)), wp, bias_p, rp, ap, bp, sp, ip, op[0], width[0], op[1],
         width[1], op[2], width[2], ws.data, ws.bytes, M, K, rank, n, (int)MAMBA_BF16, stream_of(a[16])};
    PyObject *const all[3] = {out[0].object, out[1].object, out[2].object};
    return result(all, all + used);
}

PyObject *bind(PyObject *, Args args, Py_ssize_t n) { return bind_to<Api, &api>(args, n); }

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&bind)), METH_FASTCALL, nullptr},
    MAMBA_ENTRY(sample_fwd, 14), MAMBA_ENTRY(tree_verify_fwd, 11), MAMBA_ENTRY(linear_adapted_fwd, 17), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal._sample", "argument marshalling of drawn children, verification and adapted projections", -1,
                      methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyObject *marshal_sample_module() { return PyModule_Create(&module); }
