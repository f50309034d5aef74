"""Rounds of a drafter that draws its children, under adapters and a verifier's rules, with the verification of its trees: the operators
together, eager and captured, every position against the oracle."""
import os
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import constrain as oc
from oracle import sampling as oracle

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


# ----------------------------------------------------------------------------------------------------------- without a GPU
@pytest.fixture
def host_drafter():
    if not os.path.exists(os.path.join(ROOT, "paper_2506_01206_amd", "libmamba_hip.so")):
        from paper_2506_01206_amd import build
        build.build()
    from paper_2506_01206_amd.drafter import MambaDrafter
    block = SimpleNamespace(d_inner=128, d_state=16, d_conv=4)
    return MambaDrafter(torch.zeros(1000, 64, dtype=BF16), [block], torch.ones(64))


def test_settings_as_they_are_set_and_refused(host_drafter):
    d = host_drafter
    for bad in (dict(temperature=-1.0), dict(temperature=float("nan")), dict(top_p=float("nan")), dict(min_p=float("nan"))):
        with pytest.raises(ValueError):
            d.sample(**bad)
        assert d._sampling is None
    d.sample(0.5, 7, 0.75, 0.25)
    s = d._sampling
    assert s["params"].tolist() == [[0.5, 0.75, 0.25]] and s["top_k"].tolist() == [7]
    with pytest.raises(ValueError):
        d.sample(-2.0)
    d.sample()
    assert d._sampling is s and s["params"].tolist() == [[1.0, 1.0, 0.0]] and s["top_k"].tolist() == [0]
    d.sample(None)
    assert d._sampling is None
    with pytest.raises(RuntimeError, match="sample"):
        d.verify((1, 1), torch.zeros(3, 1000))


def test_adapters_as_they_are_set_and_refused(host_drafter):
    d = host_drafter
    a, b = torch.zeros(3, 16, 64, dtype=BF16), torch.zeros(3, 1000, 16, dtype=BF16)
    with pytest.raises(RuntimeError, match="adapt"):
        d.use_adapter(0)
    for bad in (dict(lora_a=a[:, :, :8]), dict(lora_b=b[:2]), dict(lora_b=None), dict(scale=torch.ones(2)), dict(which=3), dict(which=-1), dict(lora_a=a.float()),
                dict(lora_a=a[:, :12], lora_b=b[..., :12]), dict(lora_a=a[0])):
        with pytest.raises(ValueError):
            d.adapt(**{**dict(lora_a=a, lora_b=b), **bad})
        assert d._adapters is None
    d.adapt(a, b, which=2)
    assert d._adapters["which"].tolist() == [2]
    for bad in (-2, 3):
        with pytest.raises(ValueError):
            d.use_adapter(bad)
    d.use_adapter(-1)
    assert d._adapters["which"].tolist() == [-1]
    d.adapt(None)
    assert d._adapters is None


# ----------------------------------------------------------------------------------------------------------- rounds
def small_drafter(layers=2, V=1003, seed=0):
    """A drafter of the widths that the library's kernels take, random weights; a vocabulary whose rows start anywhere."""
    from paper_2506_01206_amd import binding as b
    from paper_2506_01206_amd.drafter import MambaDrafter
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s, std=0.05, dtype=BF16: (torch.randn(*s, generator=gen) * std).to(dtype).to(DEV)
    dm, d, N, r = 64, 128, 16, 8
    blocks = [b.Block(dict(norm_w=1 + n(dm, dtype=F32), in_proj_w=n(2 * d, dm, std=0.2), conv_w=n(d, 4, std=0.4, dtype=F32), conv_b=n(d, dtype=F32),
                           x_proj_w=n(r + 2 * N, d, std=0.2), dt_proj_w=n(d, r, std=0.2), dt_bias=n(d, dtype=F32) - 3, Dskip=1 + n(d, dtype=F32),
                           A=-torch.arange(1, N + 1, dtype=F32, device=DEV).repeat(d, 1).contiguous(), out_proj_w=n(dm, d, std=0.2))) for _ in range(layers)]
    return MambaDrafter(n(V, dm, std=0.4), blocks, 1 + n(dm, dtype=F32))


@pytest.mark.gpu
@pytest.mark.parametrize("use_graph", [False, True])
def test_rounds(use_graph):
    d = small_drafter()
    V, tree, gamma = d.V, (3, 2, 1, 2), 4
    rows = oracle.tree_rows(tree)
    rng = np.random.default_rng(8)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    rand = lambda *s: torch.rand(*s, device=DEV, generator=gen)
    prefix = torch.from_numpy(rng.integers(0, V, 40).astype(np.int32)).to(DEV)
    d.prefill(prefix)
    plain_root = d.root_logits.clone()
    greedy = [t.clone() for t in d.draft(tree, use_graph)[0]]
    bf = lambda *s, std: torch.from_numpy((rng.standard_normal(s) * std).astype(np.float32)).to(DEV, BF16)
    a, b = bf(3, 8, 64, std=0.125), bf(3, V, 8, std=0.5)
    settings = [(1.0, 0, 1.0, 0.0), (0.7, 50, 0.95, 0.0), (1.4, 0, 0.9, 0.01), (0.0, 0, 1.0, 0.0)]
    seen = []
    for which, rules in ((None, False), (0, False), (2, True), (-1, True), (None, True)):
        if which is None:
            d.adapt(None)
        elif d._adapters is None:
            d.adapt(a, b, which=which)
        else:
            d.use_adapter(which)
        d.constrain(1.3, 0.2, 0.1) if rules else d.constrain(None)
        d.prefill(prefix)
        assert torch.equal(d.root_logits, plain_root) == (which in (None, -1))
        counts = oc.token_counts(prefix.cpu().numpy()[None], V, prompt=True)
        for T, top_k, top_p, min_p in settings:
            d.sample(T, top_k, top_p, min_p)
            u = rand(sum(rows[1:]))
            tokens, _ = d.draft(tree, use_graph, u=u)
            bufs = d._buffers(tree)
            path, at, q = None, 0, []
            for i, n in enumerate(tree, 1):
                logits = (d.root_logits if i == 1 else bufs["pos"][i - 1]["logits"]).float().cpu().numpy()
                if rules:
                    x, ok = oc.constrain(logits, counts, np.array([[1.3, 0.2, 0.1]], np.float32), path=path)
                    logits = torch.from_numpy(np.where(ok, x, -np.inf)).to(BF16).float().numpy()
                ui = u[at:at + rows[i]].view(-1, n).cpu().numpy()
                at += rows[i]
                idx, prob, dist = oracle.sample(logits, ui, np.array([[T, top_p, min_p]], np.float32), [top_k])
                assert np.array_equal(tokens[i - 1].cpu().numpy(), idx.reshape(-1)), (which, rules, i)
                q.append(dist)
                path = idx.reshape(-1, 1) if path is None else np.concatenate([np.repeat(path, n, 0), idx.reshape(-1, 1)], 1)
                assert np.array_equal(bufs["pos"][i]["path"].cpu().numpy(), path)
            q = np.concatenate(q)
            got_q = bufs["drawn"]["q"][0].cpu().numpy()
            assert np.abs(got_q - q).max() <= 2.0 ** -24
            # a target that is near the drafter, one that is far
            inner = sum(rows[:-1])
            for noise in (0.3, 2.0):
                w = np.concatenate([q, rng.dirichlet(np.ones(V), rows[-1])]) * np.exp(noise * rng.standard_normal((sum(rows), V))) + 1e-9
                p = torch.from_numpy((w / w.sum(1, keepdims=True)).astype(np.float32)).to(DEV)
                ua, us = rand(sum(rows) - 1), rand(1)
                out, count, node = d.verify(tree, p, ua, us)
                ro, rc, rn = oracle.verify(p.cpu().numpy()[None], got_q[None, :inner], np.concatenate([t.cpu().numpy() for t in tokens])[None], ua.cpu().numpy()[None],
                                           us.cpu().numpy(), tree)
                assert np.array_equal(out.cpu().numpy(), ro[0]) and int(count[0]) == rc[0] and np.array_equal(node.cpu().numpy(), rn[0])
                seen.append(int(count[0]))
    assert len(set(seen)) > 2
    out, count, node = d.verify(tree, p)                        # torch's random numbers
    assert 1 <= int(count[0]) <= gamma + 1 and out.shape == (gamma + 1,) and node.shape == (gamma,)
    d.draft(tree, use_graph)
    with pytest.raises(ValueError, match="random numbers"):
        d.draft(tree, use_graph, u=rand(5))
    d.sample(None), d.constrain(None), d.adapt(None)
    d.prefill(prefix)
    assert all(torch.equal(x, y) for x, y in zip(greedy, d.draft(tree, use_graph)[0]))


@pytest.mark.gpu
def test_rounds_of_several_requests_with_the_operators_themselves():
    """Hidden rows of many requests through an adapted LM head, rules, draws and verification, one launch after the other and from a graph."""
    from paper_2506_01206_amd import binding as m
    gen = torch.Generator(device=DEV)
    gen.manual_seed(9)
    S, n, V, dm, R = 6, 3, 5003, 64, 8
    randn = lambda *s, std=1.0: torch.empty(s, device=DEV).normal_(0, std, generator=gen)
    rand = lambda *s: torch.rand(*s, device=DEV, generator=gen)
    head, a, b = randn(V, dm, std=0.3).to(BF16), randn(4, R, dm, std=0.125).to(BF16), randn(4, V, R, std=0.5).to(BF16)
    hidden = randn(S, dm).to(BF16)
    adapter = torch.tensor([0, 3, -1, 1, 0, 2], dtype=torch.int32, device=DEV)
    par = torch.tensor([[0.8, 0.95, 0.0], [1.0, 1.0, 0.02], [0.7, 1.0, 0.0]] * 2, device=DEV)
    top_k = torch.tensor([0, 0, 40] * 2, dtype=torch.int32, device=DEV)
    counts = m.mamba_token_counts(torch.randint(0, V, (S, 30), device=DEV, generator=gen, dtype=torch.int32), V)
    pen = torch.tensor([[1.2, 0.1, 0.1]] * S, device=DEV)
    u, ua, us = rand(S, n), rand(S, n), rand(S)
    target = torch.softmax(randn(S, 1 + n, V, std=2.0), -1)
    logits, q = torch.empty(S, V, dtype=BF16, device=DEV), torch.empty(S, 1, V, device=DEV)
    idx, prob = torch.empty(S, n, dtype=torch.int32, device=DEV), torch.empty(S, n, device=DEV)
    ws1 = torch.empty(m.mamba_linear_adapted_workspace_bytes(S, R), dtype=torch.uint8, device=DEV)
    ws2 = torch.empty(m.mamba_sample_workspace_bytes(S, V, n), dtype=torch.uint8, device=DEV)
    ws3 = torch.empty(m.mamba_tree_verify_workspace_bytes(S), dtype=torch.uint8, device=DEV)
    outs = [torch.empty(S, 2, dtype=torch.int32, device=DEV), torch.empty(S, dtype=torch.int32, device=DEV), torch.empty(S, 1, dtype=torch.int32, device=DEV)]

    def chain():
        m.mamba_linear_adapted_fwd(hidden, head, a, b, adapter, outs=[logits], workspace=ws1)
        m.mamba_logits_constrain_fwd(logits, counts=counts, penalties=pen, out=logits)
        m.mamba_sample_fwd(logits, u, par, top_k=top_k, idx=idx, prob=prob, dist=q.view(S, V), workspace=ws2)
        m.mamba_tree_verify_fwd(target, q, idx, ua, us, (n,), out=outs[0], count=outs[1], node=outs[2], workspace=ws3)
    chain()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        chain()
    for _ in range(4):
        for t in (u, ua, us):
            t.copy_(torch.rand_like(t))
        hidden.copy_(torch.randn_like(hidden))
        chain()
        ref = [t.clone() for t in (logits, idx, prob, q, *outs)]
        for t in (logits, idx, prob, q, *outs):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(ref, (logits, idx, prob, q, *outs)))
        ri, _, _ = oracle.sample(logits.double().cpu().numpy(), u.cpu().numpy(), par.cpu().numpy(), top_k.cpu().numpy())
        assert np.array_equal(idx.cpu().numpy(), ri)
        ro, rc, rn = oracle.verify(target.cpu().numpy(), q.cpu().numpy(), idx.cpu().numpy(), ua.cpu().numpy(), us.cpu().numpy(), (n,))
        assert all(np.array_equal(t.cpu().numpy(), r) for t, r in zip(outs, (ro, rc, rn)))


@pytest.mark.gpu
def test_a_tree_that_was_not_drawn_is_not_verified():
    """What an earlier round drew is not what a greedy round's children came from."""
    d, tree = small_drafter(layers=1), (2, 1)
    d.prefill(torch.arange(20, dtype=torch.int32, device=DEV))
    p = torch.full((5, d.V), 1.0 / d.V, device=DEV)
    for use_graph in (False, True):
        d.sample(0.8)
        d.draft(tree, use_graph)
        d.verify(tree, p)
        d.sample(None)
        d.draft(tree, use_graph)
        with pytest.raises(RuntimeError, match="drawn"):
            d.verify(tree, p)
        with pytest.raises(RuntimeError, match="drawn"):
            d.verify((3,), p)
