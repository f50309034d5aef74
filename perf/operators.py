"""The operators of a gated-delta drafter that this library has kernels for, as cases that can be timed and compared.

A case is a dict of plain values.  ``listed()`` gives the fixed ones, ``draw(rng)`` another one of the same ranges;
``prepare(case, seed)`` makes what a program has in hand before the call, ``run(state)`` makes one pass: with ``own`` false in
elementary torch operations, with ``own`` true through the library's entry points.  Kinds of case:

  prefill    gated delta rule of one layer over a context: chunks, states in and out
  step       one token of the gated delta rule for all live branches of a draft tree, each from its parent's state
  constrain  logits of some rows with penalties for repeated tokens, biases and grammar masks, as a verifier samples from them
  children   the same on the way into the choice of every branch's children, with the token counts of the prefix formed first

Per head h, with q and k divided by their length (qk_norm), delta = softplus(dt + dt_bias), a = exp(A delta), b = sigmoid(beta):
  S_t = a_t S_{t-1} (I - b_t k_t k_t^T) + b_t v_t k_t^T,  o_t = scale S_t q_t,  out = rmsnorm(o) norm_w silu(z)
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
VOCAB = 50280
EPS = 1e-6
CHUNK = 64                             # steps of the plain form that are taken together
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LARGEST = 32768 * 32 * 128 * 128       # tokens x heads x state elements of the largest context
LARGEST_STEP = 128 * 32 * 128 * 128    # branches x heads x state elements of the widest draft position
LARGEST_ROWS = 128 * 131072            # logits of the largest call


def listed():
    return [
        # a short prompt in a small layer: less than one chunk, launches and latency count
        dict(name="prefill_37_small", kind="prefill", batch=1, L=37, H=6, Hk=6, N=64, P=64, z=True, norm=True, h0=False),
        # an ordinary chat prompt on a layer of the 130M shape (24 heads of 64 channels)
        dict(name="prefill_2k", kind="prefill", batch=1, L=2048, H=24, Hk=24, N=128, P=64, z=True, norm=True, h0=False),
        # a batch of contexts of no particular length, continued from states, two value heads to a key head
        dict(name="prefill_4x1000", kind="prefill", batch=4, L=1000, H=16, Hk=8, N=128, P=128, z=False, norm=False, h0=True),
        # a long document on a narrow layer
        dict(name="prefill_8191_narrow", kind="prefill", batch=1, L=8191, H=12, Hk=4, N=64, P=128, z=True, norm=False, h0=True),
        # long-context encoding on a wide layer: the largest call
        dict(name="prefill_32k_wide", kind="prefill", batch=1, L=32768, H=32, Hk=16, N=128, P=128, z=True, norm=True, h0=False),
        # sequential drafting: one branch, one token
        dict(name="step_1", kind="step", io="bf16", n_out=1, n_in=1, H=24, Hk=24, N=128, P=64, z=True, norm=True),
        # the widest position of the tree (3,3,2): children continue from their parents' states; float32 activations
        dict(name="step_18_tree", kind="step", io="f32", n_out=18, n_in=9, H=12, Hk=4, N=64, P=128, z=True, norm=False),
        # many branches of a wide layer: bytes of states
        dict(name="step_128_wide", kind="step", io="bf16", n_out=128, n_in=64, H=32, Hk=16, N=128, P=128, z=True, norm=True),
        # the root of a tree: one row, its prefix of an ordinary length
        dict(name="children_1", kind="children", io="bf16", M=1, S=1, V=VOCAB, L=333, T=0, k=3, bias=True, mask="none", path=False),
        # a position in the depth of a tree under a grammar, branches of 8 requests with long prefixes
        dict(name="children_96_tree", kind="children", io="bf16", M=96, S=8, V=VOCAB, L=8000, T=4, k=2, bias=True, mask="mixed", path=True),
        # all nodes of a tree for the verifier
        dict(name="constrain_19", kind="constrain", io="bf16", M=19, S=1, V=VOCAB, L=2000, T=4, bias=True, mask="mixed"),
        # many requests, a large vocabulary, float32 logits: the largest call
        dict(name="constrain_128_131071", kind="constrain", io="f32", M=128, S=128, V=131071, L=2000, T=3, bias=False, mask="mixed"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("prefill", "prefill", "prefill", "step", "step", "children", "children", "constrain"))
    flip = lambda p=0.5: rng.random() < p
    if kind in ("prefill", "step"):
        N, P = rng.choice((64, 128)), rng.choice((64, 128))
        group = rng.choice((1, 1, 2, 3, 4))
        Hk = _log_int(rng, 1, 32 // group)
        H = Hk * group
        c = dict(kind=kind, H=H, Hk=Hk, N=N, P=P, z=flip(0.7), norm=flip())
        if kind == "prefill":
            batch = _log_int(rng, 1, 8)
            c.update(batch=batch, L=_log_int(rng, 1, min(32768, LARGEST // (batch * H * N * P))), h0=flip())
        else:
            n_out = _log_int(rng, 1, min(256, LARGEST_STEP // (H * N * P)))
            c.update(io=rng.choice(("bf16", "bf16", "f32")), n_out=n_out, n_in=_log_int(rng, 1, n_out))
        return c
    V = rng.choice((VOCAB, _log_int(rng, 1000, 131072)))
    M = _log_int(rng, 1, min(128, LARGEST_ROWS // V))
    c = dict(kind=kind, io=rng.choice(("bf16", "bf16", "f32")), M=M, S=rng.choice((1, _log_int(rng, 1, M))), V=V, L=_log_int(rng, 1, 16384),
             T=rng.randint(0, 8), bias=flip(), mask=rng.choice(("none", "mixed", "mixed", "few")))
    if kind == "children":
        c.update(k=rng.randint(1, 8), path=flip(0.7))
    return c


# ----------------------------------------------------------------------------------------------------------- inputs
class _Draws:
    def __init__(self, seed):
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(int(seed))

    def normal(self, *shape, std=1.0):
        return torch.empty(shape, device=DEV).normal_(0.0, std, generator=self.gen)

    def uniform(self, lo, hi, *shape):
        return torch.empty(shape, device=DEV).uniform_(lo, hi, generator=self.gen)

    def ints(self, hi, *shape):
        return torch.randint(0, hi, shape, device=DEV, generator=self.gen, dtype=torch.int32)


def _delta_inputs(case, d, rows, t):
    """Activations of `rows` (leading sizes) and the layer's parameters.  q, k, v come out of a conv with SiLU, so that keys lean to one
    side; time steps are spread over 0.001 .. 0.1 as a layer's initialisation spreads them, decay rates over 1 .. 16."""
    H, Hk, N, P = (case[n] for n in ("H", "Hk", "N", "P"))

    def silu(*shape):
        x = d.normal(*shape)
        return (x * torch.sigmoid(x)).to(t)
    dt0 = torch.exp(d.uniform(math.log(1e-3), math.log(0.1), H))
    return dict(q=silu(*rows, Hk, N), k=silu(*rows, Hk, N), v=silu(*rows, H, P), dt=d.normal(*rows, H).to(t), beta=d.normal(*rows, H).to(t),
                A=-d.uniform(1.0, 16.0, H), dt_bias=dt0 + torch.log(-torch.expm1(-dt0)),
                z=d.normal(*rows, H, P).to(t) if case["z"] else None, norm_w=1.0 + d.normal(P, std=0.1) if case["norm"] else None)


def prepare(case, seed):
    d, kind = _Draws(seed), case["kind"]
    s = dict(kind=kind)
    if kind == "prefill":
        B, L, H, P, N = (case[n] for n in ("batch", "L", "H", "P", "N"))
        s["args"] = _delta_inputs(case, d, (B, L), torch.bfloat16)
        s["h0"] = d.normal(B, H, P, N, std=0.3) if case["h0"] else None
        s["out"] = torch.empty(B, L, H, P, dtype=torch.bfloat16, device=DEV)
        s["h_final"] = torch.empty(B, H, P, N, device=DEV)
        if own:
            m = _binding()
            s["workspace"] = torch.empty(max(16, m.mamba_gated_delta_workspace_bytes(B, L, H, case["Hk"], P, N)), dtype=torch.uint8, device=DEV)
    elif kind == "step":
        n_out, n_in, H, P, N = (case[n] for n in ("n_out", "n_in", "H", "P", "N"))
        t = TYPES[case["io"]]
        s["args"] = _delta_inputs(case, d, (n_out,), t)
        s["h_in"] = d.normal(n_in, H, P, N, std=0.3)
        s["parent"] = d.ints(n_in, n_out)
        s["h_out"] = torch.empty(n_out, H, P, N, device=DEV)
        s["out"] = torch.empty(n_out, H, P, dtype=t, device=DEV)
    else:
        M, S, V, T = (case[n] for n in ("M", "S", "V", "T"))
        t = TYPES[case["io"]]
        # tokens of a text: few of them make up most of it
        tokens = lambda *shape: (V * d.uniform(0.0, 1.0, *shape) ** 3).to(torch.int32).clamp_(max=V - 1)
        s["logits"] = d.normal(M, V, std=2.5).to(t)
        s["tokens"] = tokens(S, case["L"])
        s["penalties"] = torch.stack([d.uniform(1.0, 1.4, S), d.uniform(0.0, 1.0, S), d.uniform(0.0, 0.5, S)], 1).contiguous()
        s["seq"] = d.ints(S, M)
        s["path"] = tokens(M, T) if T else None
        s["bias"] = d.normal(V) * (d.uniform(0.0, 1.0, V) < 0.01) if case["bias"] else None
        s["mask"] = s["mask_idx"] = None
        if case["mask"] != "none":
            # rows of a grammar's masks: nearly everything, about half, a handful, nothing; a row of logits is under one of them or none
            share = (0.97, 0.5, 6.0 / V, 0.0) if case["mask"] == "mixed" else (1.5 / V, 0.0, 6.0 / V, 40.0 / V)
            W = (V + 31) // 32
            allowed = d.uniform(0.0, 1.0, 4, W * 32) < torch.tensor(share, device=DEV)[:, None]
            bit = torch.tensor([1 << i for i in range(31)] + [-(1 << 31)], dtype=torch.int32, device=DEV)
            s["mask"] = (allowed.view(4, W, 32) * bit).sum(-1, dtype=torch.int32)
            s["mask_idx"] = d.ints(5, M) - 1
        if kind == "constrain":
            s["counts"] = _counts(s["tokens"], V)
            s["out"] = torch.empty(M, V, dtype=t, device=DEV)
        else:
            s["k"], s["V"] = case["k"], V
            s["idx"] = torch.empty(M, case["k"], dtype=torch.int32, device=DEV)
            s["val"] = torch.empty(M, case["k"], device=DEV)
            s["path_out"] = torch.empty(M * case["k"], T + 1, dtype=torch.int32, device=DEV) if case["path"] else None
    return s


# ----------------------------------------------------------------------------------------------------------- one pass
def _binding():
    from paper_2506_01206_amd import binding
    return binding


def run(s):
    return _OWN[s["kind"]](s) if own else _PLAIN[s["kind"]](s)


def _own_prefill(s):
    return _binding().mamba_gated_delta_fwd(**s["args"], h0=s["h0"], out=s["out"], h_final=s["h_final"], workspace=s["workspace"], eps=EPS)


def _own_step(s):
    return _binding().mamba_gated_delta_step(s["h_in"], **s["args"], parent_idx=s["parent"], h_out=s["h_out"], out=s["out"], eps=EPS)


def _own_constrain(s):
    return _binding().mamba_logits_constrain_fwd(s["logits"], counts=s["counts"], penalties=s["penalties"], seq_idx=s["seq"], path=s["path"],
                                                 bias=s["bias"], mask=s["mask"], mask_idx=s["mask_idx"], out=s["out"])


def _own_children(s):
    m = _binding()
    counts = m.mamba_token_counts(s["tokens"], s["V"])
    idx, val, path_out = m.mamba_topk_constrained_fwd(
        s["logits"], s["k"], counts=counts, penalties=s["penalties"], seq_idx=s["seq"], path=s["path"], bias=s["bias"], mask=s["mask"],
        mask_idx=s["mask_idx"], idx=s["idx"], val=s["val"], path_out=s["path_out"])
    return (counts, idx, val) if path_out is None else (counts, idx, val, path_out)


def _delta_factors(a, heads):
    """q, k (one for each of the heads), v, log decay and write strength in float32."""
    q, k, v = a["q"].float(), a["k"].float(), a["v"].float()
    q = q / torch.sqrt((q * q).sum(-1, keepdim=True) + EPS) * q.shape[-1] ** -0.5
    k = k / torch.sqrt((k * k).sum(-1, keepdim=True) + EPS)
    group = heads // q.shape[-2]
    q, k = q.repeat_interleave(group, -2), k.repeat_interleave(group, -2)
    u = a["dt"].float() + a["dt_bias"]
    delta = torch.clamp(u, min=0) + torch.log1p(torch.exp(-torch.abs(u)))
    return q, k, v, a["A"] * delta, torch.sigmoid(a["beta"].float())


def _gated(o, a):
    if a["norm_w"] is not None:
        o = o / torch.sqrt((o * o).mean(-1, keepdim=True) + EPS) * a["norm_w"]
    if a["z"] is not None:
        z = a["z"].float()
        o = o * (z * torch.sigmoid(z))
    return o


def _plain_prefill(s):
    """In chunks: inside one, the tokens' writes u solve a triangular system; from one to the next only the state goes on."""
    a = s["args"]
    B, L, H, P = a["v"].shape
    N = a["q"].shape[-1]
    q, k, v, g, b = _delta_factors(a, H)
    n = (L + CHUNK - 1) // CHUNK
    pad = n * CHUNK - L

    def chunks(x):                                               # (B, L, H, ...) -> (B, H, n, CHUNK, ...), zeros behind the end
        x = torch.cat([x, x.new_zeros(B, pad, *x.shape[2:])], 1) if pad else x
        x = x.view(B, n, CHUNK, *x.shape[2:])
        return x.permute(0, 3, 1, 2, *range(4, x.dim())).contiguous()
    q, k, v, g, b = chunks(q), chunks(k), chunks(v), chunks(g), chunks(b)
    G = g.cumsum(-1)
    t = torch.arange(CHUNK, device=q.device)
    low, diag = t[:, None] > t[None, :], t[:, None] >= t[None, :]
    decay = torch.exp(torch.where(diag, G[..., :, None] - G[..., None, :], G.new_tensor(-math.inf)))
    kt = k.transpose(-1, -2).contiguous()
    system = (k @ kt) * decay * b[..., :, None] * low
    inverse = torch.eye(CHUNK, device=q.device).expand(B, H, n, CHUNK, CHUNK).contiguous()
    for i in range(1, CHUNK):
        inverse[..., i, :] -= (system[..., i, :i, None] * inverse[..., :i, :]).sum(-2)
    inner = (q @ kt) * decay
    eG, tail = torch.exp(G), torch.exp(G[..., -1:] - G)
    S = torch.zeros(B, H, P, N, device=q.device) if s["h0"] is None else s["h0"]
    out = []
    for c in range(n):
        St = S.transpose(-1, -2).contiguous()
        u = inverse[:, :, c] @ (b[:, :, c, :, None] * (v[:, :, c] - eG[:, :, c, :, None] * (k[:, :, c] @ St)))
        out.append(eG[:, :, c, :, None] * (q[:, :, c] @ St) + inner[:, :, c] @ u)
        S = eG[:, :, c, -1, None, None] * S + (u * tail[:, :, c, :, None]).transpose(-1, -2).contiguous() @ k[:, :, c]
    o = torch.stack(out, 1).permute(0, 1, 3, 2, 4).reshape(B, n * CHUNK, H, P)[:, :L]
    return _gated(o, a).to(torch.bfloat16), S


def _plain_step(s):
    a = s["args"]
    q, k, v, g, b = _delta_factors(a, a["v"].shape[-2])
    S = s["h_in"][s["parent"].long()] * torch.exp(g)[..., None, None]
    u = b[..., None] * (v - (S * k[..., None, :]).sum(-1))
    S = S + u[..., None] * k[..., None, :]
    return S, _gated((S * q[..., None, :]).sum(-1), a).to(a["v"].dtype)


def _counts(tokens, V):
    counts = torch.zeros(tokens.shape[0], V, dtype=torch.int32, device=tokens.device)
    return counts.scatter_add_(1, tokens.long(), torch.ones_like(tokens))


def _adjusted(s, counts):
    """Adjusted logits in float32, and which tokens a row may take."""
    x = s["logits"].float()
    M, V = x.shape
    c = counts[s["seq"].long()]
    if s["path"] is not None:
        c = c.scatter_add(1, s["path"].long(), torch.ones_like(s["path"]))
    rep, presence, frequency = (p[:, None] for p in s["penalties"][s["seq"].long()].unbind(1))
    seen = c > 0
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = torch.where(seen, (x - frequency * c.float()) - presence, x)
    if s["bias"] is not None:
        x = x + s["bias"]
    if s["mask"] is None:
        return x, torch.ones_like(seen)
    v = torch.arange(V, device=x.device)
    allowed = (s["mask"][:, (v // 32).long()] >> (v % 32).to(torch.int32)) & 1
    allowed = torch.cat([allowed != 0, torch.ones(1, V, dtype=torch.bool, device=x.device)])
    return x, allowed[s["mask_idx"].long()]                      # (row -1: no mask)


def _plain_constrain(s):
    x, allowed = _adjusted(s, s["counts"])
    return torch.where(allowed, x, x.new_tensor(-math.inf)).to(s["logits"].dtype)


def _plain_children(s):
    counts = _counts(s["tokens"], s["V"])
    x, left = _adjusted(s, counts)
    M, V = x.shape
    v = torch.arange(V, device=x.device)
    idx, val = [], []
    for _ in range(s["k"]):
        best = torch.where(left, x, x.new_tensor(-math.inf)).amax(1, keepdim=True)
        i = torch.where(left & (x == best), v, V).amin(1)        # the first of the largest
        idx.append(torch.where(i < V, i, -1))
        val.append(best[:, 0])
        left = left & (v != i[:, None])
    idx, val = torch.stack(idx, 1).to(torch.int32), torch.stack(val, 1)
    if s["path_out"] is None:
        return counts, idx, val
    path = idx.view(-1, 1)
    if s["path"] is not None:
        path = torch.cat([s["path"].repeat_interleave(s["k"], 0), path], 1)
    return counts, idx, val, path


_OWN = dict(prefill=_own_prefill, step=_own_step, constrain=_own_constrain, children=_own_children)
_PLAIN = dict(prefill=_plain_prefill, step=_plain_step, constrain=_plain_constrain, children=_plain_children)


# ----------------------------------------------------------------------------------------------------------- definition in 64 bits
def _recurrence(S, q, k, v, g, b, scale):
    """One token: S (..., H, P, N); the definition written out."""
    S = S * torch.exp(g)[..., None, None]
    S = S + (b[..., None] * (v - torch.einsum("...pn,...n->...p", S, k)))[..., None] * k[..., None, :]
    return S, torch.einsum("...pn,...n->...p", S, q) * scale


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("prefill", "step"):
        a = {n: None if x is None else x.double() for n, x in s["args"].items()}
        group = case["H"] // case["Hk"]
        unit = lambda x: (x * (x.square().sum(-1, keepdim=True) + EPS).rsqrt()).repeat_interleave(group, -2)
        q, k = unit(a["q"]), unit(a["k"])
        g = a["A"] * torch.nn.functional.softplus(a["dt"] + a["dt_bias"], threshold=1000.0)
        b, scale = torch.sigmoid(a["beta"]), case["N"] ** -0.5
        if case["kind"] == "step":
            S, o = _recurrence(s["h_in"][s["parent"].long()].double(), q, k, a["v"], g, b, scale)
        else:
            S = s["h0"].double() if case["h0"] else torch.zeros(case["batch"], case["H"], case["P"], case["N"], dtype=torch.float64, device=DEV)
            o = torch.empty_like(a["v"])
            for t in range(case["L"]):
                S, o[:, t] = _recurrence(S, q[:, t], k[:, t], a["v"][:, t], g[:, t], b[:, t], scale)
        if case["norm"]:
            o = o * (o.square().mean(-1, keepdim=True) + EPS).rsqrt() * a["norm_w"]
        if case["z"]:
            o = o * a["z"] / (1.0 + torch.exp(-a["z"]))
        return (S, o) if case["kind"] == "step" else (o, S)
    wide = ("logits", "penalties", "bias")
    host = {n: None if s[n] is None else (s[n].double() if n in wide else s[n]).cpu().numpy()
            for n in wide + ("tokens", "seq", "path", "mask", "mask_idx")}
    M, V = host["logits"].shape
    x = host["logits"].copy()
    allowed = np.ones((M, V), dtype=bool)
    for r in range(M):
        q = host["seq"][r]
        times = np.bincount(host["tokens"][q], minlength=V)
        if host["path"] is not None:
            times = times + np.bincount(host["path"][r], minlength=V)
        rep, presence, frequency = host["penalties"][q]
        was = times > 0
        y = x[r, was]
        x[r, was] = np.where(y > 0, y / rep, y * rep) - frequency * times[was] - presence
        if host["bias"] is not None:
            x[r] += host["bias"]
        if host["mask"] is not None and host["mask_idx"][r] >= 0:
            words = np.ascontiguousarray(host["mask"][host["mask_idx"][r]]).view(np.uint8)
            allowed[r] = np.unpackbits(words, bitorder="little")[:V] != 0
    x[~allowed] = -np.inf
    if case["kind"] == "constrain":
        return torch.from_numpy(x)
    # the tokens have no value in 64 bits (which of two nearly equal ones is first is a matter of the rounding); their logits have
    best = -np.sort(-x, axis=1)[:, :case["k"]]
    val = np.full((M, case["k"]), -np.inf)
    val[:, :best.shape[1]] = best
    val = torch.from_numpy(val)
    return (None, None, val, None) if case["path"] else (None, None, val)


def work(case):
    """Bytes: inputs read and outputs written once.  Flops: prefill, the products of the chunked form (chunks of 64, triangles counted
    whole); step, the recurrence; logits, a handful of operations on each."""
    kind = case["kind"]
    if kind in ("prefill", "step"):
        H, Hk, N, P = (case[n] for n in ("H", "Hk", "N", "P"))
        e = 2 if kind == "prefill" else TYPES[case["io"]].itemsize
        rows = case["batch"] * case["L"] if kind == "prefill" else case["n_out"]
        act = rows * e * (2 * Hk * N + H * P * (3 if case["z"] else 2) + 2 * H) + 4 * (2 * H + (P if case["norm"] else 0))
        if kind == "prefill":
            states = case["batch"] * H * P * N * 4 * (2 if case["h0"] else 1)
            return {"bytes": act + states, "flops": rows * 2 * (2 * Hk * CHUNK * N + H * (2 * CHUNK * P + 3 * N * P))}
        states = (min(case["n_in"], case["n_out"]) + case["n_out"]) * H * P * N * 4
        return {"bytes": act + states + 4 * rows, "flops": rows * H * P * N * 7}
    M, V = case["M"], case["V"]
    e = TYPES[case["io"]].itemsize
    seqs = min(case["S"], M)
    side = seqs * V * 4 + seqs * 12 + M * 4 * (1 + case["T"]) + (V * 4 if case["bias"] else 0)
    if case["mask"] != "none":
        side += min(M, 4) * ((V + 31) // 32) * 4 + M * 4
    if kind == "constrain":
        return {"bytes": side + 2 * M * V * e, "flops": M * V * 4}
    outputs = M * case["k"] * (8 + (4 * (case["T"] + 1) if case["path"] else 0))
    return {"bytes": side + case["S"] * case["L"] * 4 + case["S"] * V * 4 + M * V * e + outputs, "flops": M * V * 5}
