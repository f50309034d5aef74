"""Constrained logits where zeros of both signs, subnormals and masked logits stand among ordinary ones under penalties: bit for bit, as in
tests/test_constrained_children.py (a wavefront divides by a rounded reciprocal where all of its quotients allow it)."""
import numpy as np
import pytest
import torch

from test_constrained_children import BF16, F32, case, check, m  # noqa: F401  (m: the fixture)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("among", [[0.0], [-0.0], [0.0, -0.0, float("-inf")], [2.0 ** -126, -2.0 ** -126, 2.0 ** -40, 2.0 ** -41], [1e-39, 0.0], [float("nan"), 0.0],
                                   [float("inf"), 0.0], [3e38, -3e38], [2.0 ** 40, 2.0 ** 41]])
def test_zeros_and_masked_logits_under_penalties(m, among, dtype):  # noqa: F811
    print("\n[gpu-case] constrained logits, %s among them, %s" % (among, dtype), flush=True)
    rng = np.random.default_rng(3)
    c = case(rng, 5, 9000, 2, 3, [0.7], dtype=dtype)
    c["counts"][:] = torch.from_numpy(rng.integers(-1, 3, c["counts"].shape).astype(np.int32))
    for every, value in zip((7, 11, 13, 17), among):
        c["logits"][:, ::every] = value
    c["logits"][4] = among[0]
    check(m, c, 8)
