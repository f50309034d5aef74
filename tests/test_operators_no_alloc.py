"""The gated-delta core and the constrained choice of children with every output and workspace given by the caller: nothing is allocated."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, to_dev
from test_constrained_children import case as rules_case, gpu
from test_gated_delta import case, device, m, state  # noqa: F401  (m: the fixture)

pytestmark = pytest.mark.gpu


def allocations():
    return torch.cuda.memory_stats()["allocation.all.allocated"], torch.cuda.memory_reserved()


def nothing_allocated(call, *outputs):
    """Twice, the workspaces full of something else the second time: the same bits."""
    call()
    torch.cuda.synchronize()
    first = [o.clone() for o in outputs]
    free, before = torch.cuda.mem_get_info()[0], allocations()
    result = call()
    torch.cuda.synchronize()
    assert allocations() == before and torch.cuda.mem_get_info()[0] >= free
    assert all(torch.equal(a, b) for a, b in zip(first, outputs))
    return result


@pytest.mark.parametrize("L", [5, 300, 2500])
def test_contexts(m, L):  # noqa: F811
    print("\n[gpu-case] gated delta without allocations, L=%d" % L, flush=True)
    rng = np.random.default_rng(L)
    g, h0 = device(case(rng, 1, L, 4, 2, 64, 128)), to_dev(state(rng, 1, 4, 128, 64))
    out, hf = torch.empty(1, L, 4, 128, dtype=torch.bfloat16, device=DEV), torch.empty(1, 4, 128, 64, device=DEV)
    ws = torch.empty(max(16, m.mamba_gated_delta_workspace_bytes(1, L, 4, 2, 128, 64)), dtype=torch.uint8, device=DEV)
    o, h = nothing_allocated(lambda: m.mamba_gated_delta_fwd(**g, h0=h0, out=out, h_final=hf, workspace=ws), out, hf)
    assert o is out and h is hf


def test_steps(m):  # noqa: F811
    print("\n[gpu-case] gated delta step without allocations", flush=True)
    rng = np.random.default_rng(3)
    g = device({n: x[:, 0] if n in ("q", "k", "v", "dt", "beta", "z") else x for n, x in case(rng, 6, 1, 4, 2, 64, 64).items()})
    h, parent = to_dev(state(rng, 3, 4, 64, 64)), torch.tensor([0, 0, 1, 1, 2, 2], dtype=torch.int32, device=DEV)
    ho, out = torch.empty(6, 4, 64, 64, device=DEV), torch.empty(6, 4, 64, dtype=torch.bfloat16, device=DEV)
    nothing_allocated(lambda: m.mamba_gated_delta_step(h, **g, parent_idx=parent, h_out=ho, out=out), ho, out)


def test_constrained_logits_and_children(m):  # noqa: F811
    print("\n[gpu-case] constrained children without allocations", flush=True)
    rng = np.random.default_rng(4)
    M, V, T, k = 7, 9000, 2, 3
    c = gpu(rules_case(rng, M, V, 2, T, [0.5, 0.01]))
    logits, tokens = c.pop("logits"), torch.from_numpy(rng.integers(0, V, (2, 100)).astype(np.int32)).to(DEV)
    out, counts = torch.empty_like(logits), torch.zeros(2, V, dtype=torch.int32, device=DEV)
    idx, val = torch.empty(M, k, dtype=torch.int32, device=DEV), torch.empty(M, k, device=DEV)
    path = torch.empty(M * k, T + 1, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(16, m.mamba_topk_constrained_workspace_bytes(M, V, k)), dtype=torch.uint8, device=DEV)
    nothing_allocated(lambda: m.mamba_logits_constrain_fwd(logits, **c, out=out), out)
    nothing_allocated(lambda: m.mamba_topk_constrained_fwd(logits, k, **c, idx=idx, val=val, path_out=path, workspace=ws), idx, val, path)
    nothing_allocated(lambda: m.mamba_token_counts(tokens, V, counts=counts, prompt=True), counts)
