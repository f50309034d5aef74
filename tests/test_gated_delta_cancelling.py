"""Contexts whose tokens overwrite what the state held with much smaller values: what a token reads back is the small difference of two
large sums, Q S^T and (M X) R in the chunked form.  float64 oracle on the same inputs.

Keys and queries are unit vectors, so that every sum over N has one term that is not zero and every sum over a chunk's tokens at most the two or three
tokens of one key.  The state holds values `ratio` times the new ones; a float32 form rounds the decayed state, R, the entries of X and M X and both
products of an output, 16 roundings of the old values at the most, exp2 among them at one unit (two half steps): 16 * 2^-24 * ratio of the new ones.
The old values are normal deviates, up to 5 times their rms (5.7e-7 beyond): 80 * 2^-24 * ratio.  bfloat16 outputs add their own half step, 2^-8."""
import os

import numpy as np
import pytest
import torch

from paper_2506_01206_amd import synth
from gpu_util import DEV, W, assert_close, to_dev, to_host, values
from test_gated_delta import m, storage  # noqa: F401  (the fixture)


def case(rng, B, L, H, N, P, ratio, decay):
    """Every token writes a value under a key of its own for as long as there are keys; queries are the tokens' own keys."""
    eye = np.eye(N)
    at = np.stack([np.concatenate([rng.permutation(N) for _ in range((L + N - 1) // N)])[:L] for _ in range(B * H)]).reshape(B, H, L)
    k = eye[at].transpose(0, 2, 1, 3)
    c = dict(q=storage(k, synth.BF16), k=storage(k, synth.BF16), v=storage(rng.standard_normal((B, L, H, P)), synth.BF16),
             dt=storage(np.full((B, L, H), 1.0), synth.BF16), beta=storage(np.ones((B, L, H)), synth.BF16), A=np.full(H, -decay, np.float32))
    return c, (ratio * rng.standard_normal((B, H, P, N))).astype(np.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("ratio", [1.0, 100.0, 1000.0])
@pytest.mark.parametrize("B,L,H,N,P,decay,gate,norm", [
    (1, 64, 2, 64, 64, 0.0, False, False), (2, 40, 1, 128, 128, 0.01, False, False), (1, 128, 2, 128, 64, 0.003, True, False),
    (1, 64, 3, 64, 128, 0.01, True, True), (1, 100, 2, 128, 128, 0.0, False, True), (1, 3, 2, 128, 64, 0.01, True, True)])
def test_small_values_over_large_ones(m, B, L, H, N, P, decay, gate, norm, ratio):  # noqa: F811
    from oracle import delta
    print("\n[gpu-case] gated delta, values %g times smaller than the state's: B=%d L=%d H=%d N=%d P=%d" % (ratio, B, L, H, N, P), flush=True)
    rng = np.random.default_rng(L + N)
    c, h0 = case(rng, B, L, H, N, P, ratio, decay)
    if gate:
        c["z"] = storage(rng.standard_normal((B, L, H, P)), synth.BF16)
    if norm:
        c["norm_w"] = np.ones(P, np.float32)
    options = dict(dt_softplus=False, beta_sigmoid=False, qk_norm=False, scale=1.0)
    out, hf = m.mamba_gated_delta_fwd(**{n: to_dev(x) for n, x in c.items()}, h0=to_dev(h0), **options)
    ro, rh = delta.delta_scan(**{n: W(x) for n, x in c.items()}, h0=h0, **options)
    tol = 80 * 2.0 ** -24 * ratio
    assert_close(values(to_host(out)), ro, tol + 2.0 ** -8, "out")
    # a written row of the state is as small as the outputs; a row that is left is as large as before: the error is that of the whole
    assert_close(to_host(hf), rh, max(tol, 1e-5) if L >= N else 1e-5, "final state")
