"""Verification of drafted trees on the device (mamba_tree_verify_fwd): pins of the oracle, refusals (no GPU needed), and the kernel against the
oracle and the host's verification of chains."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import sampling as oracle


def some_trees(rng, S, V, tree, noise, sharp=2.0, filtered=False):
    rows = oracle.tree_rows(tree)
    nodes, inner = sum(rows), sum(rows[:-1])
    logits = rng.standard_normal((S, nodes, V)) * sharp

    def soft(x):
        w = np.exp(x - x.max(-1, keepdims=True))
        if filtered:
            w[w < 0.05] = 0.0
        return (w / w.sum(-1, keepdims=True)).astype(np.float32)
    p, q = soft(logits + noise * rng.standard_normal(logits.shape)), soft(logits[:, :inner])
    tokens = np.empty((S, nodes - 1), np.int32)
    for s in range(S):
        child = node = 0
        for r, n in zip(rows, tree):
            for _ in range(r):
                left = q[s, node].astype(np.float64)
                for _ in range(n):
                    v = oracle.draw(left, rng.uniform())
                    tokens[s, child] = v
                    if v >= 0:
                        left[v] = 0.0
                    child += 1
                node += 1
    return dict(p=p, q=q, tokens=tokens, u_accept=rng.uniform(size=(S, nodes - 1)).astype(np.float32), u_sample=rng.uniform(size=S).astype(np.float32), tree=tree)


# ----------------------------------------------------------------------------------------------------------- the oracle
def test_oracle_emits_tokens_as_the_target_does():
    """Exactness: children drawn from q without replacement, the first emitted token is distributed as p, whatever q is."""
    rng = np.random.default_rng(1)
    V, tree, S = 5, (3,), 40000
    p, q = rng.dirichlet(np.ones(V)), rng.dirichlet(np.ones(V))
    p, q = np.broadcast_to(p.astype(np.float32), (S, 4, V)), np.broadcast_to(q.astype(np.float32), (S, 1, V))
    order = q[:, 0] / rng.exponential(size=(S, V))               # the first to arrive: drawn without replacement
    tokens = np.argsort(-order, axis=1)[:, :3].astype(np.int32)
    out, _, _ = oracle.verify(p, q, tokens, rng.uniform(size=(S, 3)), rng.uniform(size=S), tree)
    share = np.bincount(out[:, 0], minlength=V) / S
    assert np.abs(share - p[0, 0]).max() < 5 * 0.5 / np.sqrt(S)  # five standard deviations at most


def test_oracle_on_chains_is_the_host_verification():
    from oracle import tree_search
    rng = np.random.default_rng(2)
    c = some_trees(rng, 30, 11, (1, 1, 1), 1.0)
    out, count, _ = oracle.verify(**c)
    for s in range(30):
        ref = tree_search.verify(c["p"][s], c["q"][s], c["tokens"][s], c["u_accept"][s], c["u_sample"][s], False)
        assert out[s, :count[s]].tolist() == ref


# ----------------------------------------------------------------------------------------------------------- refusals, without a GPU
def P(i):
    return (i + 1) << 40


@pytest.fixture(scope="module")
def m():
    from paper_2506_01206_amd import binding
    return binding


def call(m, p=P(0), q=P(1), tokens=P(2), ua=P(3), us=P(4), out=P(5), count=P(6), node=P(7), ws=P(8), ws_bytes=1 << 39, tree=(3, 2), gamma=None, S=4, V=100):
    arr = None if tree is None else (ctypes.c_int32 * max(len(tree), 1))(*tree)
    return m.lib.mamba_tree_verify_fwd(p, q, tokens, ua, us, out, count, node, ws, ws_bytes, arr, (len(tree) if tree else 1) if gamma is None else gamma, S, V, None)


def test_refusals(m):
    S = m.STATUS
    for name in ("p", "q", "tokens", "ua", "us", "out", "count", "node"):
        assert call(m, **{name: None}) == S["NULL_POINTER"], name
        assert call(m, **{name: P(9) + 2}) == S["MISALIGNED"], name
    assert call(m, tree=None) == S["NULL_POINTER"]
    assert call(m, ws=P(9) + 8) == S["MISALIGNED"] and call(m, ws=None) == S["WORKSPACE"]
    assert call(m, ws_bytes=m.mamba_tree_verify_workspace_bytes(4) - 1) == S["WORKSPACE"]
    assert m.mamba_tree_verify_workspace_bytes(0) == 0 and m.mamba_tree_verify_workspace_bytes(-1) == 0 and m.mamba_tree_verify_workspace_bytes(1 << 40) == 0
    for bad in (dict(gamma=0), dict(tree=(1,) * 17), dict(tree=(3, 0)), dict(tree=(-1,)), dict(S=-1), dict(V=-1), dict(V=0), dict(S=1 << 21, V=1 << 40)):
        assert call(m, **bad) == S["BAD_SHAPE"], bad
    for bad in (dict(tree=(9,)), dict(tree=(8,) * 6), dict(S=1 << 24), dict(S=1 << 20, V=50000), dict(V=(1 << 25) + 1)):
        assert call(m, **bad) == S["UNSUPPORTED"], bad
    assert call(m, S=0) == S["OK"]
    for a, b in (("out", 2), ("count", 0), ("node", 4), ("count", 5), ("node", 6), ("ws", 0), ("ws", 5), ("node", 8)):
        assert call(m, **{a: P(b)}) == S["ALIAS"], (a, b)


def test_binding_refuses_trees_that_are_none(m):
    p = torch.zeros(1, 3, 10)
    with pytest.raises(ValueError, match="GPU"):
        m.mamba_tree_verify_fwd(p, p[:, :2], p, p, p, (1, 1))


# ----------------------------------------------------------------------------------------------------------- the kernel
gpu = pytest.mark.gpu
DEV = "cuda:0"


def on_device(c):
    return {n: torch.from_numpy(np.ascontiguousarray(v)).to(DEV) if isinstance(v, np.ndarray) else v for n, v in c.items()}


def check(m, c):
    got = m.mamba_tree_verify_fwd(**on_device(c))
    ref = oracle.verify(**c)
    for g, r, what in zip(got, ref, ("out", "count", "node")):
        assert np.array_equal(g.cpu().numpy(), r), (what, g.cpu().numpy()[:3], r[:3])
    return ref


@gpu
@pytest.mark.parametrize("tree", [(1,), (3,), (8,), (1, 1, 1, 1, 1), (3, 2, 2, 1, 1), (2, 3, 1), (1,) * 16], ids=str)
@pytest.mark.parametrize("V", [1, 2, 3, 5, 1001, 4096, 4097, 9000])
def test_against_oracle(m, tree, V):
    rng = np.random.default_rng(V + 31 * len(tree))
    S = 3 if V > 4000 and sum(oracle.tree_rows(tree)) > 30 else 12
    seen = set()
    for noise, filtered in ((0.0, False), (0.5, False), (1.5, True), (4.0, False), (0.0, True)):
        _, count, _ = check(m, some_trees(rng, S, V, tree, noise, filtered=filtered))
        seen |= set(count.tolist())
    assert len(seen) > 1 or V <= max(tree)                       # (where a node's children are the whole vocabulary, one of them is accepted)


@gpu
def test_large_vocabularies(m):
    rng = np.random.default_rng(9)
    check(m, some_trees(rng, 2, 50280, (3, 2), 2.0))
    check(m, some_trees(rng, 3, 131071, (1, 1), 0.7))
    check(m, some_trees(rng, 1, 700001, (2,), 1.0))              # pieces of more than one trip


@gpu
def test_long_offsets(m):
    """Sequences whose offsets pass 32 bits: as each by itself."""
    S, V, tree = 1100, (1 << 20) + 3, (1, 1)
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    gen = torch.Generator(device=DEV)
    gen.manual_seed(2)
    p, q = torch.rand(S, 3, V, device=DEV, generator=gen), torch.rand(S, 2, V, device=DEV, generator=gen)
    tokens = torch.randint(0, V, (S, 2), device=DEV, generator=gen, dtype=torch.int32)
    ua, us = torch.rand(S, 2, device=DEV, generator=gen), torch.rand(S, device=DEV, generator=gen)
    got = m.mamba_tree_verify_fwd(p, q, tokens, ua, us, tree)
    for b in (0, 682, 1023, S - 1):
        at = slice(b, b + 1)
        one = m.mamba_tree_verify_fwd(p[at].clone(), q[at].clone(), tokens[at].clone(), ua[at].clone(), us[at].clone(), tree)
        assert all(torch.equal(x[at], y) for x, y in zip(got, one)), b
    assert bool(((got[0] >= 0).sum(1) == got[1]).all()) and len(got[1].unique()) > 1


@gpu
def test_more_rejections_than_rounds(m):
    """Children that the target does not want, fifteen of them on one way."""
    rng = np.random.default_rng(15)
    for tree in ((8, 8, 2), (5, 5, 5)):
        c = some_trees(rng, 4, 400, tree, 0.5)
        rows = oracle.tree_rows(tree)
        u = np.ones(c["u_accept"].shape, np.float32) - np.float32(2.0 ** -24)
        first = 0
        for r, n in zip(rows, tree):                             # the last child of every node is taken, where its ratio is above zero
            u[:, first + n - 1:first + r * n:n] = 0.0
            first += r * n
        check(m, {**c, "u_accept": u})
        check(m, {**c, "u_accept": np.full_like(u, 1 - 2.0 ** -24)})


@gpu
def test_a_target_of_one_token_and_rows_of_nothing(m):
    rng = np.random.default_rng(10)
    c = some_trees(rng, 8, 300, (2, 2), 1.0)
    greedy = np.zeros_like(c["p"])
    np.put_along_axis(greedy, c["p"].argmax(-1)[..., None], 1.0, -1)
    check(m, {**c, "p": greedy})
    check(m, {**c, "p": np.zeros_like(c["p"])})                  # nothing to draw: -1
    check(m, {**c, "q": np.zeros_like(c["q"])})                  # children that the drafter gave nothing
    check(m, {**c, "tokens": np.full_like(c["tokens"], -1)})     # no children at all
    check(m, {**c, "tokens": np.where(rng.uniform(size=c["tokens"].shape) < 0.4, [300], c["tokens"]).astype(np.int32)})
    same = c["tokens"].copy()
    same[:, 1::2] = same[:, 0::2]                                # the same child twice
    check(m, {**c, "tokens": same})
    for u in (0.0, 1 - 2.0 ** -24):
        check(m, {**c, "u_sample": np.full_like(c["u_sample"], u)})
        check(m, {**c, "u_accept": np.full_like(c["u_accept"], u)})


@gpu
def test_no_number_ends_the_walk_in_bounds(m):
    """NaN and infinities among the probabilities: what comes out are tokens of the vocabulary or -1, and counts in range."""
    rng = np.random.default_rng(11)
    c = some_trees(rng, 6, 500, (3, 2), 1.0)
    for name in ("p", "q", "u_accept", "u_sample"):
        for bad in (np.nan, np.inf, -np.inf):
            v = c[name].copy()
            v[rng.uniform(size=v.shape) < 0.2] = bad
            out, count, node = (t.cpu().numpy() for t in m.mamba_tree_verify_fwd(**on_device({**c, name: v})))
            assert ((out >= -1) & (out < 500)).all() and ((count >= 1) & (count <= 3)).all() and ((node >= -1) & (node < 6)).all()


@gpu
def test_chains_as_the_host_verifies_them(m):
    from paper_2506_01206_amd import tree_search
    rng = np.random.default_rng(12)
    c = some_trees(rng, 20, 700, (1, 1, 1, 1), 1.0)
    out, count, node = (t.cpu().numpy() for t in m.mamba_tree_verify_fwd(**on_device(c)))
    for s in range(20):
        ref = list(tree_search.sd_verify(c["p"][s], c["q"][s], c["tokens"][s], c["u_accept"][s], float(c["u_sample"][s]), greedy=False))
        assert out[s, :count[s]].tolist() == ref
        assert node[s].tolist() == [0] * (count[s] - 1) + [-1] * (5 - count[s])


@gpu
def test_streams_graphs_and_given_outputs(m):
    rng = np.random.default_rng(13)
    c = on_device(some_trees(rng, 7, 5001, (3, 2), 1.0))
    ref = m.mamba_tree_verify_fwd(**c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = m.mamba_tree_verify_fwd(**c, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    outs = [torch.full((t.shape[0] + 1,) + t.shape[1:], -9, dtype=torch.int32, device=DEV) for t in ref]
    ws = torch.empty(m.mamba_tree_verify_workspace_bytes(7), dtype=torch.uint8, device=DEV)
    one = lambda: m.mamba_tree_verify_fwd(**c, out=outs[0][:7], count=outs[1][:7], node=outs[2][:7], workspace=ws)
    one()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        one()
    for _ in range(3):
        for t in outs:
            t.fill_(-9)
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        for a, b, o in zip(ref, got, outs):
            assert torch.equal(a, b) and torch.equal(a, o[:7]) and bool((o[7:] == -9).all())
        c["u_accept"].copy_(torch.rand_like(c["u_accept"]))
        ref = got = m.mamba_tree_verify_fwd(**c)


@gpu
def test_refusals_of_the_binding(m):
    c = on_device(some_trees(np.random.default_rng(14), 2, 50, (2, 2), 1.0))
    for bad in (dict(tree=(2, 3)), dict(tree=()), dict(tree=(2, 9)), dict(p=c["p"][:, :-1].contiguous()), dict(q=c["q"].double()), dict(tokens=c["tokens"].long()),
                dict(u_sample=c["u_sample"][:1]), dict(p=c["p"].transpose(0, 1)), dict(u_accept=c["u_accept"].cpu())):
        with pytest.raises((ValueError, TypeError)):
            m.mamba_tree_verify_fwd(**{**c, **bad})
