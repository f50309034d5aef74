"""NaN and infinities in the inputs of a token of the gated-delta core: nothing ahead of the token changes by a bit, everything that the
equations take them to is no number any more (NaN, or an infinity still), and nothing else."""
import numpy as np
import pytest
import torch

from paper_2506_01206_amd import synth
from gpu_util import DEV, to_dev
from test_gated_delta import case, device, m, state  # noqa: F401  (m: the fixture)

NAN, INF = float("nan"), float("inf")
# what a token's NaN reaches: its channel from there on, its head(s) from there on, its own outputs
VALUES = [("v", NAN), ("v", INF), ("v", -INF), ("k", NAN), ("k", INF), ("q", NAN), ("q", -INF), ("dt", NAN), ("beta", NAN)]


def reached(name, shape, Hk, b, s, h, i, norm):
    """bool (B,L,H,P) and (B,H,P): outputs and rows of the state that are no numbers"""
    B, L, H, P = shape
    out, rows = torch.zeros(B, L, H, P, dtype=torch.bool), torch.zeros(B, H, P, dtype=torch.bool)
    heads = slice(h * (H // Hk), (h + 1) * (H // Hk)) if name in ("q", "k") else slice(h, h + 1)
    if name == "v":
        out[b, s:, h, slice(None) if norm else i] = True
        rows[b, h, i] = True
    elif name == "q":
        out[b, s, heads] = True
    else:
        out[b, s:, heads] = True
        rows[b, heads] = True
    return out.to(DEV), rows.to(DEV)


def same_but(got, ref, nan):
    bad = ~torch.isfinite(got)
    assert torch.equal(bad, nan), "%d of %d" % (int((bad != nan).sum()), nan.numel())
    assert torch.equal(torch.where(nan, 0, got), torch.where(nan, 0, ref))


@pytest.mark.gpu
@pytest.mark.parametrize("io", [synth.BF16, synth.F32])
@pytest.mark.parametrize("name,value", VALUES)
@pytest.mark.parametrize("L,s", [(6, 3), (40, 0), (40, 21), (200, 150), (200, 199), (192, 127)])
def test_a_token_reaches_nothing_ahead_of_it(m, L, s, name, value, io):  # noqa: F811
    print("\n[gpu-case] gated delta, %s = %g at token %d of %d, io=%s" % (name, value, s, L, io), flush=True)
    rng = np.random.default_rng(L + s)
    for H, Hk, N, P, z, norm in ((4, 2, 64, 64, False, False), (4, 2, 128, 64, True, False), (2, 2, 64, 128, True, True), (3, 1, 128, 128, False, True)):
        g, h0 = device(case(rng, 2, L, H, Hk, N, P, io, z, norm)), to_dev(state(rng, 2, H, P, N))
        ref, rh = m.mamba_gated_delta_fwd(**g, h0=h0)
        h, i = (Hk if name in ("q", "k") else H) - 1, 7
        g[name][(1, s, h, i) if name in ("q", "k", "v") else (1, s, h)] = value
        out, hf = m.mamba_gated_delta_fwd(**g, h0=h0)
        nan, rows = reached(name, ref.shape, Hk, 1, s, h, i, norm)
        if name == "v" and norm and abs(value) == INF:           # (o / sqrt(mean o^2) is 0 in the other channels where one is infinite, NaN where it is NaN)
            out, ref = torch.where(nan, NAN, out), torch.where(nan, NAN, ref)
        same_but(out, ref, nan)
        same_but(hf, rh, rows[..., None].expand_as(rh))


@pytest.mark.gpu
@pytest.mark.parametrize("N,P,z,norm", [(64, 64, True, False), (128, 128, True, True), (128, 64, False, False)])
@pytest.mark.parametrize("L,s", [(100, 1), (100, 70), (2500, 1300), (2500, 2499)])
def test_rows_behind_the_text_hold_anything(m, L, s, N, P, z, norm):  # noqa: F811
    """A buffer of L tokens of which s are a text: what stands behind it is whatever memory held.  A long context of one head goes in parts."""
    print("\n[gpu-case] gated delta, garbage behind %d of %d tokens, N=%d P=%d" % (s, L, N, P), flush=True)
    rng = np.random.default_rng(s)
    g = device(case(rng, 1, L, 1, 1, N, P, synth.BF16, z, norm))
    ref, _ = m.mamba_gated_delta_fwd(**g)
    for n in ("q", "k", "v", "z", "dt", "beta"):
        if g[n] is not None:
            g[n][:, s:] = torch.from_numpy(rng.choice([NAN, INF, -INF, 3e38, -1.0], g[n][:, s:].shape)).to(DEV)
    out, hf = m.mamba_gated_delta_fwd(**g)
    assert torch.equal(out[:, :s], ref[:, :s]) and not bool(torch.isfinite(hf).any())


@pytest.mark.gpu
@pytest.mark.parametrize("io", [synth.BF16, synth.F32])
def test_a_gate_and_a_state_that_are_not_numbers(m, io):  # noqa: F811
    """z reaches its own output only; a row of the state its own channel."""
    rng = np.random.default_rng(5)
    g, h0 = device(case(rng, 1, 150, 2, 2, 64, 64, io, True, False)), to_dev(state(rng, 1, 2, 64, 64))
    ref, rh = m.mamba_gated_delta_fwd(**g, h0=h0)
    g["z"][0, 77, 1, 5] = NAN
    h0[0, 0, 9, 3] = NAN
    out, hf = m.mamba_gated_delta_fwd(**g, h0=h0)
    nan, rows = torch.zeros_like(ref, dtype=torch.bool), torch.zeros_like(rh, dtype=torch.bool)
    nan[0, 77, 1, 5] = nan[0, :, 0, 9] = True
    rows[0, 0, 9] = True
    same_but(out, ref, nan)
    same_but(hf, rh, rows)


@pytest.mark.gpu
@pytest.mark.parametrize("io", [synth.BF16, synth.F32])
def test_keys_that_are_numbers_but_long(m, io):  # noqa: F811
    """Without a norm a key of 1e19 in every state is a key like others: its square overflows, what it writes does not."""
    from gpu_util import W, assert_close, to_host, values
    from oracle import delta
    from test_gated_delta import TOL, TOL_F32, storage
    print("\n[gpu-case] gated delta, long keys, io=%s" % io, flush=True)
    rng = np.random.default_rng(6)
    c = case(rng, 1, 40, 2, 2, 128, 64, io, False, False)
    k, beta, dt = W(c["k"]) * 0.1, np.zeros((1, 40, 2)), np.full((1, 40, 2), -1e-3)
    k[0, 7], beta[0, 7], beta[0, :7] = 1e19, 1e-20, 0.5
    c["k"], c["beta"], c["dt"], c["dt_bias"], c["A"] = storage(k, io), storage(beta, io), storage(dt, io), None, np.full(2, 1.0, np.float32)
    options = dict(qk_norm=False, beta_sigmoid=False, dt_softplus=False)
    out, hf = m.mamba_gated_delta_fwd(**device(c), **options)
    ro, rh = delta.delta_scan(**{n: W(x) for n, x in c.items()}, **options)
    assert_close(values(to_host(out)), ro, TOL[io], "out")
    assert_close(to_host(hf), rh, TOL_F32, "final state")
