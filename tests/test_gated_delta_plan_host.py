"""Host side of the gated-delta core's workspaces (no GPU): what the entry point refuses needs none."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def m():
    if not os.path.exists(os.path.join(ROOT, "paper_2506_01206_amd", "libmamba_hip.so")):
        from paper_2506_01206_amd import build
        build.build()
    from paper_2506_01206_amd import binding
    return binding


@pytest.mark.parametrize("batch,L,H,Hk,P,N", [
    (70000, 100, 8, 4, 64, 128), (1, 100, 70000, 1, 64, 128), (1025, 100, 512, 4, 64, 128), (1, (1 << 31) + 1, 8, 4, 64, 128), (1 << 43, 512, 1, 1, 64, 64),
    (1 << 30, 64, 1 << 15, 1, 64, 64), (1, 100, 8, 3, 64, 128), (1, 100, 8, 4, 32, 128), (1, 100, 8, 0, 64, 128), (-1, 100, 8, 4, 64, 128)])
def test_no_workspace_for_what_is_refused(m, batch, L, H, Hk, P, N):
    """0 is the documented answer for an unsupported shape; beyond the limits the size itself overflows."""
    at = [(i + 1) << 50 for i in range(13)]
    status = m.lib.mamba_gated_delta_fwd(*at, 1 << 49, batch, L, H, Hk, P, N, 1.0, 1e-6, 1, 1, 1, 1, None)
    assert status in (m.STATUS["UNSUPPORTED"], m.STATUS["BAD_SHAPE"])
    assert m.mamba_gated_delta_workspace_bytes(batch, L, H, Hk, P, N) == 0
