"""The operators of drafting for a verifier that samples, for many requests at once, as cases that can be timed and compared.

A case is a dict of plain values.  ``listed()`` gives the fixed ones, ``draw(rng)`` another one of the same ranges;
``prepare(case, seed)`` makes what a program has in hand before the call, ``run(state)`` makes one pass: with ``own`` false in
elementary torch operations, with ``own`` true through the library's entry points.  Kinds of case:

  adapted  a projection that all rows share with the low-rank adapter of each row's request beside it
             out = x W^T + bias + residual + scale_a (x A_a^T) B_a^T
  sample   the children of draft branches, or the next tokens of requests, drawn without replacement from their logits under temperature,
           top-k, top-p and min-p, with given random numbers; with it, where it is wanted, the distribution that they are drawn from
             w = exp((x - max x) / T), kept: those with w >= min_p, of those the top_k largest, of those the fewest that make up top_p
  verify   which path of a tree of such children a target accepts, and the token behind it
             accepted: u < min(1, p / q); rejected: p = (p - q)_+ / its sum, q = q without the child / its sum; none: drawn from p
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
VOCAB = 50280
LARGEST_PRODUCT = 16384 * 4096 * 2048  # rows x outputs x inputs of the largest projection
LARGEST_ROWS = 128 * 131072            # logits of the largest call
LARGEST_TREES = 32 * 11 * 131072       # probabilities of the largest verification
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one branch of one request through an output projection of the 130M shape: launches and latency count
        dict(name="adapted_1", kind="adapted", M=1, K=1536, N=768, R=8, n=1, rows="one", splits=1, bias=False, residual=True),
        # a draft position of 8 requests with 3 branches each at the LM head, every request with its own adapter
        dict(name="adapted_24_head", kind="adapted", M=24, K=768, N=VOCAB, R=16, n=8, rows="mixed", splits=1, bias=False, residual=False),
        # a prompt under one adapter, of no particular length
        dict(name="adapted_333", kind="adapted", M=333, K=768, N=1536, R=16, n=4, rows="one", splits=2, bias=False, residual=False),
        # many contexts one after the other, some without an adapter; higher rank, several outputs
        dict(name="adapted_4097_contexts", kind="adapted", M=4097, K=1024, N=2048, R=64, n=16, rows="contexts", splits=2, bias=True, residual=False),
        # contexts of a wide layer: the largest call
        dict(name="adapted_16k_wide", kind="adapted", M=16384, K=2048, N=4096, R=32, n=32, rows="contexts", splits=1, bias=False, residual=True),
        # the next token of one request
        dict(name="sample_1", kind="sample", io="bf16", M=1, S=1, V=VOCAB, k=1, filters="top_p", dist=False, path=False),
        # a position in the depth of a tree: 2 children of each of 9 branches, with the distribution that verification needs
        dict(name="sample_9_children", kind="sample", io="bf16", M=9, S=1, V=VOCAB, k=2, filters="all", dist=True, path=True),
        # branches of 8 requests, each with settings of its own
        dict(name="sample_96_requests", kind="sample", io="bf16", M=96, S=8, V=VOCAB, k=3, filters="mixed", dist=False, path=True),
        # many requests, a large vocabulary, float32 logits, distributions: the largest call
        dict(name="sample_128_131071", kind="sample", io="f32", M=128, S=128, V=131071, k=1, filters="mixed", dist=True, path=False),
        # one request's tree
        dict(name="verify_1_tree", kind="verify", S=1, V=VOCAB, tree="3,2,2,1,1", noise=1.0, filters="top_p"),
        # trees of 8 requests, target and drafter far apart: most of it is rejected
        dict(name="verify_8_far", kind="verify", S=8, V=VOCAB, tree="3,2,2", noise=3.0, filters="none"),
        # chains of 32 requests over a large vocabulary
        dict(name="verify_32_chains", kind="verify", S=32, V=131071, tree="1,1,1,1,1", noise=0.7, filters="none"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("adapted", "adapted", "sample", "sample", "verify"))
    flip = lambda p=0.5: rng.random() < p
    if kind == "adapted":
        head = flip(0.2)
        K = 8 * _log_int(rng, 8, 512)
        N = _log_int(rng, 8192, 131072) if head else 8 * _log_int(rng, 1, 512)
        M = _log_int(rng, 1, 64 if head else max(1, min(16384, LARGEST_PRODUCT // (K * N))))
        R = 8 * _log_int(rng, 1, 16)
        splits = 1 if head else rng.choice((1, 1, 2, 3)) if N >= 24 else 1
        return dict(kind=kind, M=M, K=K, N=N, R=R, n=_log_int(rng, 1, min(64, 1024 // R)), rows=rng.choice(("one", "mixed", "contexts")), splits=splits,
                    bias=flip(0.3), residual=splits == 1 and not head and flip())
    V = rng.choice((VOCAB, _log_int(rng, 1000, 131072)))
    if kind == "sample":
        M = _log_int(rng, 1, min(128, LARGEST_ROWS // V))
        return dict(kind=kind, io=rng.choice(("bf16", "bf16", "f32")), M=M, S=rng.choice((1, _log_int(rng, 1, M))), V=V, k=rng.randint(1, 8),
                    filters=rng.choice(("none", "top_k", "top_p", "min_p", "all", "mixed", "mixed")), dist=flip(), path=flip())
    tree = [rng.choice((1, 1, 2, 3)) for _ in range(rng.randint(1, 5))]
    while _nodes(tree)[0] + _nodes(tree)[1] > 80:
        tree.pop()
    S = _log_int(rng, 1, max(1, min(32, LARGEST_TREES // (V * (_nodes(tree)[0] + _nodes(tree)[1])))))
    return dict(kind=kind, S=S, V=V, tree=",".join(map(str, tree)), noise=round(rng.uniform(0.2, 3.0), 2), filters=rng.choice(("none", "top_k", "top_p", "all")))


def _nodes(tree):
    """Nodes of a tree, the root among them, and those of them that have children."""
    rows = [1]
    for n in tree:
        rows.append(rows[-1] * n)
    return sum(rows), sum(rows[:-1])


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


def _settings(case, d, S):
    """temperature, top_p, min_p (S, 3) and top_k (S), as users choose them; "mixed": every sequence others, some of them greedy."""
    T, k = d.uniform(0.6, 1.2, S), 20 + d.ints(81, S)
    p, m = d.uniform(0.8, 0.99, S), d.uniform(0.02, 0.1, S)
    which = {"none": 0, "top_k": 1, "top_p": 2, "min_p": 4, "all": 7}.get(case["filters"])
    on = d.ints(8, S) if which is None else torch.full((S,), which, dtype=torch.int32, device=DEV)
    if which is None:
        T = torch.where(d.uniform(0.0, 1.0, S) < 0.1, torch.zeros_like(T), T)
    k = torch.where((on & 1) != 0, k, torch.zeros_like(k))
    p = torch.where((on & 2) != 0, p, torch.ones_like(p))
    m = torch.where((on & 4) != 0, m, torch.zeros_like(m))
    return torch.stack([T, p, m], 1).contiguous(), k


def _segments(case, d):
    """The adapter of every row (-1: none)."""
    M, n = case["M"], case["n"]
    if case["rows"] == "one":
        return torch.full((M,), n - 1, dtype=torch.int32, device=DEV)
    if case["rows"] == "mixed":
        return d.ints(n + 1, M) - 1
    ends = d.ints(M, 2 * n).sort().values                        # contexts of no particular lengths, each with one of the adapters or none
    which = d.ints(n + 1, 2 * n + 1) - 1
    return which[torch.searchsorted(ends, torch.arange(M, device=DEV, dtype=torch.int32), right=True)].contiguous()


def prepare(case, seed):
    d, kind = _Draws(seed), case["kind"]
    s = dict(kind=kind)
    if kind == "adapted":
        M, K, N, R, n = (case[x] for x in ("M", "K", "N", "R", "n"))
        bf = torch.bfloat16
        s["x"], s["w"] = d.normal(M, K).to(bf), d.normal(N, K, std=K ** -0.5).to(bf)
        s["a"], s["b"] = d.normal(n, R, K, std=K ** -0.5).to(bf), d.normal(n, N, R, std=0.3 * R ** -0.5).to(bf)
        s["scale"], s["idx"] = d.uniform(0.5, 2.0, n), _segments(case, d)
        s["bias"] = d.normal(N, std=0.1) if case["bias"] else None
        s["residual"] = d.normal(M, N).to(bf) if case["residual"] else None
        widths = [N // 8 // case["splits"] * 8] * (case["splits"] - 1)
        s["widths"] = widths + [N - sum(widths)]
        s["outs"] = [torch.empty(M, c, dtype=bf, device=DEV) for c in s["widths"]]
        if own:
            s["workspace"] = torch.empty(max(16, _binding().mamba_linear_adapted_workspace_bytes(M, R)), dtype=torch.uint8, device=DEV)
    elif kind == "sample":
        M, S, V, k = (case[x] for x in ("M", "S", "V", "k"))
        # rows of a language model: some nearly certain, some wide open
        s["logits"] = (d.normal(M, V) * d.uniform(1.5, 4.0, M, 1)).to(TYPES[case["io"]])
        s["u"] = d.uniform(0.0, 1.0, M, k)
        s["params"], s["top_k"] = _settings(case, d, S)
        s["seq"] = d.ints(S, M)
        s["path"] = d.ints(V, M, 4) if case["path"] else None
        s["idx"], s["prob"] = torch.empty(M, k, dtype=torch.int32, device=DEV), torch.empty(M, k, device=DEV)
        s["dist"] = torch.empty(M, V, device=DEV) if case["dist"] else None
        s["path_out"] = torch.empty(M * k, 5, dtype=torch.int32, device=DEV) if case["path"] else None
        if own:
            s["workspace"] = torch.empty(max(16, _binding().mamba_sample_workspace_bytes(M, V, k)), dtype=torch.uint8, device=DEV)
    else:
        S, V = case["S"], case["V"]
        tree = [int(n) for n in case["tree"].split(",")]
        total, inner = _nodes(tree)
        params, top_k = _settings(case, d, S)
        q, p, tokens, rows, first = [], [], [], 1, 0
        for n in [*tree, 0]:                                     # position by position, so that little more than the outputs is held
            logits = d.normal(S, rows, V, std=2.5)
            p.append(_soft(logits + d.normal(S, rows, V, std=case["noise"]), params, top_k))
            if n:
                q.append(_soft(logits, params, top_k))
                race = q[-1] / -torch.log(d.uniform(1e-7, 1.0 - 1e-7, S, rows, V))   # drawn without replacement: the n first to arrive
                got = race.topk(n, dim=-1)
                tokens.append(torch.where(got.values > 0, got.indices, -1).to(torch.int32).reshape(S, rows * n))
                rows *= n
        s["p"], s["q"], s["tokens"], s["tree"] = torch.cat(p, 1), torch.cat(q, 1), torch.cat(tokens, 1), tree
        del p, q
        s["u_accept"], s["u_sample"] = d.uniform(0.0, 1.0, S, total - 1), d.uniform(0.0, 1.0, S)
        s["out"] = torch.empty(S, len(tree) + 1, dtype=torch.int32, device=DEV)
        s["count"] = torch.empty(S, dtype=torch.int32, device=DEV)
        s["node"] = torch.empty(S, len(tree), dtype=torch.int32, device=DEV)
    return s


def _soft(logits, params, top_k):
    """Filtered probabilities (S, rows, V) float32, for inputs (neither side's)."""
    S, rows, V = logits.shape
    x = logits / params[:, 0].clamp(min=0.05)[:, None, None]
    if int((top_k > 0).sum()):
        kth = x.topk(100, dim=-1).values.gather(-1, (top_k.long() - 1).clamp(min=0)[:, None, None].expand(S, rows, 1))
        x = torch.where((top_k[:, None, None] <= 0) | (x >= kth), x, x.new_tensor(-math.inf))
    w = torch.softmax(x, -1)
    if float(params[:, 1].min()) < 1.0:
        for i in range(S):
            v, order = w[i].sort(-1, descending=True)
            v = torch.where(v.cumsum(-1) - v < params[i, 1], v, v.new_zeros(()))
            w[i].scatter_(-1, order, v)
    w = torch.where(w >= params[:, 2, None, None] * w.amax(-1, keepdim=True), w, w.new_zeros(()))
    return w / w.sum(-1, keepdim=True)


# ----------------------------------------------------------------------------------------------------------- one pass
def _binding():
    from paper_2506_01206_amd import binding
    return binding


def run(s):
    return _OWN[s["kind"]](s) if own else _PLAIN[s["kind"]](s)


def _own_adapted(s):
    return _binding().mamba_linear_adapted_fwd(s["x"], s["w"], s["a"], s["b"], s["idx"], scale=s["scale"], bias=s["bias"], residual=s["residual"],
                                               splits=s["widths"], outs=s["outs"], workspace=s["workspace"])


def _own_sample(s):
    got = _binding().mamba_sample_fwd(s["logits"], s["u"], s["params"], top_k=s["top_k"], seq_idx=s["seq"], path=s["path"], idx=s["idx"],
                                      prob=s["prob"], dist=s["dist"], path_out=s["path_out"], workspace=s["workspace"])
    return tuple(t for t in got if t is not None)


def _own_verify(s):
    return _binding().mamba_tree_verify_fwd(s["p"], s["q"], s["tokens"], s["u_accept"], s["u_sample"], s["tree"], out=s["out"], count=s["count"],
                                            node=s["node"])


def _plain_adapted(s):
    x, n = s["x"].float(), s["a"].shape[0]
    R = s["a"].shape[1]
    y = x @ s["w"].float().t()
    # all adapters side by side, then of every row only its own
    t = (x @ s["a"].float().view(n * R, -1).t()).view(-1, n, R) * s["scale"][:, None]
    t = t * (s["idx"][:, None] == torch.arange(n, device=x.device))[:, :, None]
    y = y + t.view(-1, n * R) @ s["b"].float().permute(0, 2, 1).reshape(n * R, -1)
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return tuple(c.to(torch.bfloat16).contiguous() for c in y.split(s["widths"], 1))


def _first(cumulative, bound, V):
    """Index of the first element above the bound in every row (V where there is none)."""
    v = torch.arange(V, device=cumulative.device)
    return torch.where(cumulative > bound, v, V).amin(1)


def _plain_sample(s):
    x = s["logits"].double()
    M, V = x.shape
    par, top_k = s["params"].double()[s["seq"].long()], s["top_k"][s["seq"].long()].long()[:, None]
    T, top_p, min_p = (c[:, None] for c in par.unbind(1))
    x, order = x.sort(dim=1, descending=True, stable=True)       # equal ones stay in the order of their indices
    at = torch.arange(V, device=x.device)
    w = torch.where(T > 0, torch.exp((x - x[:, :1]) / torch.where(T > 0, T, torch.ones_like(T))), (at == 0).double())
    w = torch.where((w >= torch.clamp(min_p, max=1.0)) & ((top_k <= 0) | (at < top_k)), w, torch.zeros_like(w))
    c = w.cumsum(1)
    w = torch.where((at == 0) | (top_p >= 1) | (c - w < top_p * c[:, -1:]), w, torch.zeros_like(w))
    w = torch.zeros_like(w).scatter(1, order, w)
    total = w.sum(1, keepdim=True)
    dist = w / total
    idx, prob = [], []
    for j in range(s["u"].shape[1]):
        c = w.cumsum(1)
        i = _first(c, s["u"][:, j:j + 1].double() * c[:, -1:], V)
        some = (c[:, -1] > 0) & (i < V)
        i = torch.where(some, i, 0)
        idx.append(torch.where(some, i, -1))
        prob.append(torch.where(some, dist.gather(1, i[:, None])[:, 0], torch.zeros_like(total[:, 0])))
        w = torch.where(some[:, None] & (at == i[:, None]), torch.zeros_like(w), w)
    idx, prob = torch.stack(idx, 1).to(torch.int32), torch.stack(prob, 1).float()
    out = (idx, prob) + ((dist.float(),) if s["dist"] is not None else ())
    if s["path"] is not None:
        out += (torch.cat([s["path"].repeat_interleave(idx.shape[1], 0), idx.view(-1, 1)], 1),)
    return out


def _plain_verify(s):
    tree, S, V = s["tree"], s["p"].shape[0], s["p"].shape[2]
    dev = s["p"].device
    each, at = torch.arange(S, device=dev), torch.arange(V, device=dev)
    row = torch.zeros(S, dtype=torch.long, device=dev)           # the node within its position
    node_first, drawn_first = 0, 0                               # of the position's nodes, and of its children's tokens
    alive = torch.ones(S, dtype=torch.bool, device=dev)
    count = torch.zeros(S, dtype=torch.long, device=dev)
    out = torch.full((S, len(tree) + 1), -1, dtype=torch.long, device=dev)
    node = torch.full((S, len(tree)), -1, dtype=torch.long, device=dev)
    final = torch.zeros(S, V, dtype=torch.float64, device=dev)
    rows = 1
    for i, n in enumerate(tree):
        P, q0 = s["p"][each, node_first + row].double(), s["q"][each, node_first + row].double()
        Q, left = q0, torch.ones(S, V, dtype=torch.bool, device=dev)
        taken = torch.full((S,), -1, dtype=torch.long, device=dev)
        for j in range(n):
            child = row * n + j
            c, u = s["tokens"][each, drawn_first + child].long(), s["u_accept"][each, drawn_first + child].double()
            known, c = (c >= 0) & (c < V), c.clamp(0, V - 1)
            a, b = P.gather(1, c[:, None])[:, 0], Q.gather(1, c[:, None])[:, 0]
            ratio = torch.where(b > 0, a / torch.where(b > 0, b, torch.ones_like(b)), (a > 0).double())
            open_ = known & (taken < 0)
            yes = open_ & (u < torch.clamp(ratio, max=1.0))
            taken = torch.where(yes, child, taken)
            no = (open_ & ~yes)[:, None]
            left = left & ~(no & (at == c[:, None]))
            r = torch.clamp(P - Q, min=0.0)
            mass = r.sum(1, keepdim=True)
            P = torch.where(no & (mass > 0), r / torch.where(mass > 0, mass, torch.ones_like(mass)), P)
            rest = torch.where(left, q0, torch.zeros_like(q0))
            mass = rest.sum(1, keepdim=True)
            Q = torch.where(no, torch.where(mass > 0, rest / torch.where(mass > 0, mass, torch.ones_like(mass)), torch.zeros_like(rest)), Q)
        yes = alive & (taken >= 0)
        final = torch.where((alive & ~yes)[:, None], P, final)
        token = s["tokens"][each, drawn_first + taken.clamp(min=0)].long()
        out[:, i] = torch.where(yes, token, out[:, i])
        node[:, i] = torch.where(yes, taken, node[:, i])
        count += yes
        alive = yes
        row = torch.where(yes, taken, row * n)
        node_first += rows
        drawn_first += rows * n
        rows *= n
    final = torch.where(alive[:, None], s["p"][each, node_first + row].double(), final)
    c = final.cumsum(1)
    i = _first(c, s["u_sample"][:, None].double() * c[:, -1:], V)
    out.scatter_(1, count[:, None], torch.where((c[:, -1] > 0) & (i < V), i, -1)[:, None])
    return out.to(torch.int32), (count + 1).to(torch.int32), node.to(torch.int32)


_OWN = dict(adapted=_own_adapted, sample=_own_sample, verify=_own_verify)
_PLAIN = dict(adapted=_plain_adapted, sample=_plain_sample, verify=_plain_verify)


# ----------------------------------------------------------------------------------------------------------- definition in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adapted":
        x = s["x"].double()
        y = x @ s["w"].double().t()
        for a in range(case["n"]):
            mine = torch.nonzero(s["idx"] == a)[:, 0]
            if mine.numel():
                y[mine] += s["scale"][a].double() * (x[mine] @ s["a"][a].double().t()) @ s["b"][a].double().t()
        if case["bias"]:
            y += s["bias"].double()
        if case["residual"]:
            y += s["residual"].double()
        return tuple(c.contiguous() for c in y.split(s["widths"], 1))
    host = {n: t.cpu().numpy() if torch.is_tensor(t) else t for n, t in s.items() if n != "logits"}
    if case["kind"] == "sample":
        return _exact_sample(case, host, s["logits"].double().cpu().numpy())
    return _exact_verify(host)


def _inverse(weights, u):
    """First index whose cumulative weight exceeds u times the sum, None where nothing has weight."""
    c = np.cumsum(weights)
    if not c[-1] > 0:
        return None
    return min(int(np.searchsorted(c, u * c[-1], side="right")), int(np.flatnonzero(weights)[-1]))


def _exact_sample(case, host, logits):
    M, V = logits.shape
    k = case["k"]
    idx, prob, dist = np.full((M, k), -1, np.int32), np.zeros((M, k)), np.zeros((M, V))
    for m in range(M):
        q, x = host["seq"][m], logits[m]
        T, top_p, min_p = (float(f) for f in host["params"][q])
        order = np.argsort(-x, kind="stable")
        if T == 0.0:
            order = order[:1]
        if host["top_k"][q] > 0:
            order = order[:host["top_k"][q]]
        w = np.exp((x[order] - x[order[0]]) / (T if T > 0 else 1.0))
        w = w[w >= min(min_p, 1.0)]
        keep = len(w)
        if top_p < 1.0:
            keep = min(keep, int(np.searchsorted(np.cumsum(w), top_p * w.sum(), side="left")) + 1)
        dist[m, order[:keep]] = w[:keep] / w[:keep].sum()
        left = dist[m].copy()
        for j in range(k):
            v = _inverse(left, float(host["u"][m, j]))
            if v is None:
                break
            idx[m, j], prob[m, j], left[v] = v, dist[m, v], 0.0
    out = [torch.from_numpy(idx), torch.from_numpy(prob)] + ([torch.from_numpy(dist)] if case["dist"] else [])
    if case["path"]:
        out.append(torch.from_numpy(np.concatenate([np.repeat(host["path"], k, 0), idx.reshape(-1, 1)], 1)))
    return tuple(out)


def _exact_verify(host):
    tree, (S, _, V) = host["tree"], host["p"].shape
    out, node = np.full((S, len(tree) + 1), -1, np.int32), np.full((S, len(tree)), -1, np.int32)
    count = np.zeros(S, np.int32)
    for b in range(S):
        row, rows, nodes, drawn, done = 0, 1, 0, 0, None
        for i, n in enumerate(tree):
            P = host["p"][b, nodes + row].astype(np.float64)
            q = host["q"][b, nodes + row].astype(np.float64)
            Q, taken = q.copy(), None
            for j in range(n):
                at = drawn + row * n + j
                c = int(host["tokens"][b, at])
                if not 0 <= c < V:
                    continue
                ratio = P[c] / Q[c] if Q[c] > 0 else float(P[c] > 0)
                if float(host["u_accept"][b, at]) < min(1.0, ratio):
                    taken = row * n + j
                    out[b, i], node[b, i] = c, taken
                    break
                gap = np.maximum(P - Q, 0.0)
                if gap.sum() > 0:
                    P = gap / gap.sum()
                q[c] = 0.0
                Q = q / q.sum() if q.sum() > 0 else np.zeros(V)
            if taken is None:
                done = P
                break
            row, nodes, drawn, rows = taken, nodes + rows, drawn + rows * n, rows * n
            count[b] = i + 1
        v = _inverse(host["p"][b, nodes + row].astype(np.float64) if done is None else done, float(host["u_sample"][b]))
        out[b, count[b]] = -1 if v is None else v
        count[b] += 1
    return torch.from_numpy(out), torch.from_numpy(count), torch.from_numpy(node)


def work(case):
    """Bytes: inputs read and outputs written once (adapters: those that rows can have; verification: p and q of the node where a path ends,
    the fewest that decide it).  Flops: products; a 64-bit exponential of some 20 operations for a logit; a handful for a probability."""
    if case["kind"] == "adapted":
        M, K, N, R = (case[x] for x in ("M", "K", "N", "R"))
        used = 1 if case["rows"] == "one" else min(case["n"], M)
        size = 2 * (M * K + N * K + M * N * (2 if case["residual"] else 1) + used * R * (K + N)) + 4 * (M + used + (N if case["bias"] else 0))
        return {"bytes": size, "flops": 2 * M * (K * N + R * (K + N))}
    V = case["V"]
    if case["kind"] == "sample":
        M, k = case["M"], case["k"]
        small = min(case["S"], M) * 16 + M * 4 + M * k * 12 + (M * 16 + M * k * 20 if case["path"] else 0)
        return {"bytes": M * V * (TYPES[case["io"]].itemsize + (4 if case["dist"] else 0)) + small, "flops": M * V * 24}
    return {"bytes": case["S"] * (2 * V * 4 + 64), "flops": case["S"] * V * 8}
