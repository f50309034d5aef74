"""A draft round of a gated-delta layer under a verifier's rules: context, children, their states and the next position's children, as a
drafter runs them; every stage against its oracle on what the stage before it left, and the round captured and replayed.

Tolerances: those of the layer core (tests/test_gated_delta.py), from the device's own inputs at every stage; children exactly."""
import os

import numpy as np
import pytest
import torch

from gpu_util import DEV, assert_close, to_host, values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
V, H, HK, N, P, TREE = 1003, 8, 2, 64, 64, (3, 2, 2)
DM, OUT = 256, H * P


@pytest.fixture(scope="module")
def m():
    if not os.path.exists(os.path.join(ROOT, "paper_2506_01206_amd", "libmamba_hip.so")):
        from paper_2506_01206_amd import build
        build.build()
    from paper_2506_01206_amd import binding
    return binding


class Layer:
    def __init__(self, m, seed):
        self.m = m
        gen = torch.Generator().manual_seed(seed)
        n = lambda *s, std: (torch.randn(*s, generator=gen) * std).to(BF16).to(DEV)
        self.table, self.head = n(V, DM, std=1.0), n(V, OUT, std=0.05)
        self.w_qk, self.w_vz, self.w_db = n(2 * HK * N, DM, std=0.06), n(2 * OUT, DM, std=0.06), n(2 * H, DM, std=0.06)
        self.fixed = dict(A=-torch.linspace(0.5, 8, H, device=DEV), dt_bias=torch.linspace(-4, -1, H, device=DEV), norm_w=torch.ones(P, device=DEV))

    def inputs(self, tokens, shape):
        """The layer's tensors of some tokens; shape: their leading dimensions."""
        x = self.m.mamba_embedding_fwd(tokens, self.table)
        q, k = self.m.mamba_linear_fwd(x, self.w_qk, splits=(HK * N, HK * N))
        v, z = self.m.mamba_linear_fwd(x, self.w_vz, splits=(OUT, OUT))
        dt, beta = self.m.mamba_linear_fwd(x, self.w_db, splits=(H, H))
        return dict(q=q.view(*shape, HK, N), k=k.view(*shape, HK, N), v=v.view(*shape, H, P), z=z.view(*shape, H, P), dt=dt.view(*shape, H),
                    beta=beta.view(*shape, H), **self.fixed)

    def logits(self, out):
        return self.m.mamba_linear_fwd(out.reshape(-1, OUT), self.head)[0]

    def context(self, tokens):
        c = self.inputs(tokens, (1, tokens.numel()))
        out, state = self.m.mamba_gated_delta_fwd(**c)
        return c, out, state, self.logits(out[0, -1:])

    def round(self, state, logits, rules, h=None):
        """Position by position: (children, their values, their paths, inputs, states, outputs, logits)."""
        path, kept = None, []
        for i, n in enumerate(TREE):
            idx, val, path = self.m.mamba_topk_constrained_fwd(logits, n, **rules, path=path, want_path=True)
            c = self.inputs(idx.view(-1), (idx.numel(),))
            parent = torch.arange(idx.numel(), device=DEV, dtype=I32) // n
            state, out = self.m.mamba_gated_delta_step(state, **c, parent_idx=parent)
            logits = self.logits(out)
            kept.append((idx, val, path, c, state, out, logits))
        return kept


def host(c):
    return {n: values(to_host(x)) for n, x in c.items()}


@pytest.mark.gpu
@pytest.mark.parametrize("L", [5, 200, 2500])
def test_a_draft_round(m, L):
    from oracle import constrain as oc, delta
    print("\n[gpu-case] draft round of a gated-delta layer, context %d" % L, flush=True)
    rng = np.random.default_rng(L)
    layer = Layer(m, 1)
    text = torch.from_numpy(rng.integers(0, V, L).astype(np.int32)).to(DEV)
    counts = m.mamba_token_counts(text[None], V)
    allowed = rng.random((1, V)) < 0.6
    words = np.zeros((1, (V + 31) // 32 * 4), np.uint8)
    words[:, :(V + 7) // 8] = np.packbits(allowed, axis=1, bitorder="little")
    rules = dict(counts=counts, penalties=torch.tensor([[1.2, 0.3, 0.05]], device=DEV), mask=torch.from_numpy(words.view(np.int32)).to(DEV),
                 bias=torch.from_numpy((0.1 * rng.standard_normal(V)).astype(np.float32)).to(DEV))
    c, out, root, logits = layer.context(text)
    ro, rs = delta.delta_scan(**host(c))
    assert_close(values(to_host(out)), ro, 2.0 ** -8 + 2e-4, "context")
    assert_close(to_host(root), rs, 1e-4, "context's state")
    kept = layer.round(root, logits, rules)
    n_counts, path, state = oc.token_counts(text.cpu().numpy()[None], V), None, to_host(root)
    for i, (idx, val, p, c, s, o, lg) in enumerate(kept):
        x, ok = oc.constrain(logits.float().cpu().numpy(), n_counts, rules["penalties"].cpu().numpy(), path=path, bias=rules["bias"].cpu().numpy(),
                             mask=words.view(np.int32))
        ri, rv, path = oc.children(x, ok, TREE[i], path)
        assert np.array_equal(idx.cpu().numpy(), ri) and np.array_equal(val.cpu().numpy(), rv) and np.array_equal(p.cpu().numpy(), path)
        parent = np.arange(idx.numel()) // TREE[i]
        rs, ro = delta.delta_step(state, parent=parent, **host(c))
        assert_close(to_host(s), rs, 1e-5, "states of position %d" % i)
        assert_close(values(to_host(o)), ro, 2.0 ** -8 + 2e-4, "outputs of position %d" % i)
        state, logits = to_host(s), lg


@pytest.mark.gpu
def test_a_captured_round_of_one_context_after_another(m):
    print("\n[gpu-case] captured draft round of a gated-delta layer", flush=True)
    rng = np.random.default_rng(3)
    layer = Layer(m, 2)
    root, first = torch.empty(1, H, P, N, device=DEV), torch.empty(1, V, dtype=BF16, device=DEV)
    counts = torch.zeros(1, V, dtype=I32, device=DEV)
    rules = dict(counts=counts, penalties=torch.tensor([[1.1, 0.2, 0.1]], device=DEV))

    def begin(L):
        text = torch.from_numpy(rng.integers(0, V, L).astype(np.int32)).to(DEV)
        counts.copy_(m.mamba_token_counts(text[None], V))
        _, _, state, logits = layer.context(text)
        root.copy_(state), first.copy_(logits)
    begin(30)
    layer.round(root, first, rules)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = layer.round(root, first, rules)
    for L in (30, 1, 700, 64):
        begin(L)
        want = layer.round(root, first, rules)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(kept, want):
            for j in (0, 1, 2, 4, 5, 6):
                assert torch.equal(a[j], b[j]), (L, j)
