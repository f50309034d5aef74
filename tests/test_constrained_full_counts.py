"""Counts that are full: an entry of 2^31 - 1 occurrences stays there, and the bit of the prompt above it stays what it was."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from test_constrained_children import I32, case, check, m  # noqa: F401  (m: the fixture)

FULL = (1 << 31) - 1


@pytest.mark.gpu
def test_token_counts_end_at_31_bits(m):  # noqa: F811
    print("\n[gpu-case] token counts near 2^31", flush=True)
    V = 40
    tokens = torch.tensor([[0, 1, 1, 2, 2, 2, 3, 5, 5]], dtype=I32, device=DEV)
    before = np.array([[FULL, FULL - 1, FULL - 3, 0, FULL, -1]], np.int32)        # (-1: full, and in the prompt)
    before = np.concatenate([before, np.full((1, V - 6), -(1 << 31) + 5, np.int32)], 1)
    counts = torch.from_numpy(before).to(DEV)
    m.mamba_token_counts(tokens, V, counts=counts)
    want = before.copy()
    want[0, :6] = [FULL, FULL, FULL, 1, FULL, -1]
    assert np.array_equal(counts.cpu().numpy(), want)
    m.mamba_token_counts(tokens, V, counts=counts, prompt=True)
    want[0, [0, 1, 2, 3]] |= np.int32(-(1 << 31))
    assert np.array_equal(counts.cpu().numpy(), want)


@pytest.mark.gpu
def test_a_path_over_full_counts(m):  # noqa: F811
    """float32 has the same value for 2^31 - 1 and for three more."""
    print("\n[gpu-case] constrained logits, full counts", flush=True)
    rng = np.random.default_rng(4)
    c = case(rng, 4, 5000, 1, 3, None, dtype=torch.float32)
    c["path"] = torch.tensor([[1, 2, 3], [1, 1, 1], [4999, 2, 4999], [-1, 3, 5000]], dtype=I32)
    c["counts"][0, [1, 2, 3, 4999]] = torch.tensor([FULL, -1, FULL - 1, -1], dtype=I32)
    check(m, c, 5)
