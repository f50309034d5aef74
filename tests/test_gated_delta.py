"""The gated-delta layer core (mamba_gated_delta_fwd, mamba_gated_delta_step): the oracle's own pins, refusals (no GPU needed), and the
kernels against the oracle.

Tolerances, per element, of max(|reference|, rms of the reference).  States and float32 outputs: 1e-4.  On the way to the states the
chunked form carries every computed factor of a product as three bfloat16 terms, exact, and leaves out the three smallest of the nine
products of two such, 3 * 2^-24 of the whole at most; sums are float32 over 128 terms, 128 * 2^-24 = 8e-6 if every rounding leans to one
side, and a term passes through four such sums inside a chunk of 64 (the inverse, the state, u, the state again): 3.1e-5, and the state
forgets what lies more than a chunk or two behind.  bfloat16 outputs take two terms, off by 2^-17: their own rounding, half a step = 2^-8,
and that: 4.1e-3.  A norm over the channels divides by the outputs' own size, which leaves relative errors as they are."""
import os

import numpy as np
import pytest
import torch

from paper_2506_01206_amd import synth
from gpu_util import DEV, W, assert_close, to_dev, to_host, values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TOL_F32, TOL_BF16 = 1e-4, 2.0 ** -8 + 2e-4
TOL = {synth.F32: TOL_F32, synth.BF16: TOL_BF16}


@pytest.fixture(scope="module")
def m():
    if not os.path.exists(os.path.join(ROOT, "paper_2506_01206_amd", "libmamba_hip.so")):
        from paper_2506_01206_amd import build
        build.build()
    from paper_2506_01206_amd import binding
    return binding


def storage(x, io):
    """float64 -> the storage array of the I/O type"""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16 if io == synth.BF16 else torch.float32)
    return t.view(torch.int16).numpy().view(np.uint16) if io == synth.BF16 else t.numpy()


def case(rng, B, L, H, Hk, N, P, io=synth.BF16, z=True, norm=True, alike=0.0):
    """Inputs as a layer has them; alike: how far all keys lean to one direction (1: all the same)."""
    n = rng.standard_normal
    silu = lambda x: x / (1.0 + np.exp(-x))
    k = (1.0 - alike) * silu(n((B, L, Hk, N))) + alike * silu(n((1, 1, Hk, N)))
    dt0 = np.exp(rng.uniform(np.log(1e-3), np.log(0.1), H))
    c = dict(q=storage(silu(n((B, L, Hk, N))), io), k=storage(k, io), v=storage(n((B, L, H, P)), io), dt=storage(n((B, L, H)), io),
             beta=storage(n((B, L, H)), io), A=-rng.uniform(1, 16, H).astype(np.float32),
             dt_bias=(dt0 + np.log(-np.expm1(-dt0))).astype(np.float32))
    c["z"] = storage(n((B, L, H, P)), io) if z else None
    c["norm_w"] = (1.0 + 0.1 * n(P)).astype(np.float32) if norm else None
    return c


def oracle_scan(c, h0=None, **options):
    from oracle import delta
    return delta.delta_scan(**{n: W(x) for n, x in c.items()}, h0=h0, **options)


def device(c):
    return {n: to_dev(x) for n, x in c.items()}


def state(rng, *shape):
    return (0.3 * rng.standard_normal(shape)).astype(np.float32)


# ------------------------------------------------------------------------------------------------ the oracle's own pins
def test_oracle_without_writes_is_a_decaying_state():
    """b = 0: S_t = exp(sum of delta A) S_0, and out = scale S q."""
    rng = np.random.default_rng(1)
    c = case(rng, 2, 5, 4, 2, 64, 64, synth.F32, z=False, norm=False)
    c["beta"] = np.zeros_like(c["beta"])
    h0 = rng.standard_normal((2, 4, 64, 64))
    out, S = oracle_scan(c, h0, beta_sigmoid=False, qk_norm=False, scale=1.0)
    u = c["dt"].astype(np.float64) + c["dt_bias"]
    g = (np.log1p(np.exp(u)) * c["A"]).cumsum(1)
    ref = np.exp(g)[..., None, None] * h0[:, None]
    assert np.allclose(S, ref[:, -1], rtol=1e-12)
    q = np.repeat(c["q"].astype(np.float64), 2, 2)
    assert np.allclose(out, np.einsum("blhpn,blhn->blhp", ref, q), rtol=1e-10, atol=1e-12)


def test_oracle_writes_what_it_reads_back():
    """The delta rule's purpose: with b = 1, no decay and keys of unit length the state returns exactly the last value written under a
    key, whatever stood there; orthogonal keys do not disturb each other."""
    rng = np.random.default_rng(2)
    N = P = 64
    basis = np.linalg.qr(rng.standard_normal((N, N)))[0]
    order = [3, 7, 3, 11, 7, 3]
    k = basis[order][None, :, None]
    v = rng.standard_normal((1, 6, 1, P))
    zero, one = np.zeros((1, 6, 1)), np.ones((1, 6, 1))
    from oracle import delta
    out, S = delta.delta_scan(k, k, v, zero, np.zeros(1), one, h0=rng.standard_normal((1, 1, P, N)), scale=1.0, eps=0.0, dt_softplus=False,
                              beta_sigmoid=False)
    assert np.allclose(out, v, atol=1e-12)                       # read back at once
    for slot, t in ((3, 5), (7, 4), (11, 3)):
        assert np.allclose(S[0, 0] @ basis[slot], v[0, t, 0], atol=1e-12)


def test_oracle_pieces_and_steps_are_the_whole():
    from oracle import delta
    rng = np.random.default_rng(3)
    c = case(rng, 1, 7, 4, 2, 64, 64, synth.F32)
    out, S = oracle_scan(c)
    cut = lambda lo, hi: {n: x if x is None or n in ("A", "dt_bias", "norm_w") else x[:, lo:hi] for n, x in c.items()}
    o1, s1 = oracle_scan(cut(0, 3))
    o2, s2 = oracle_scan(cut(3, 7), s1)
    assert np.allclose(np.concatenate([o1, o2], 1), out, rtol=1e-12) and np.allclose(s2, S, rtol=1e-12)
    h = np.zeros((1, 4, 64, 64))
    for t in range(7):
        w = {n: x if x is None or n in ("A", "dt_bias", "norm_w") else x[:, t] for n, x in c.items()}
        h, o = delta.delta_step(h, parent=[0], **w)
        assert np.allclose(o, out[:, t], rtol=1e-12)
    assert np.allclose(h, S, rtol=1e-12)


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
def Pt(i):
    return (i + 1) << 40


def fwd(b, q=Pt(0), k=Pt(1), v=Pt(2), dt=Pt(3), A=Pt(4), beta=Pt(5), z=Pt(6), nw=Pt(7), db=Pt(8), h0=Pt(9), out=Pt(10), hf=Pt(11), ws=Pt(12),
        ws_bytes=1 << 39, batch=1, L=100, H=8, Hk=4, P=64, N=128, io=1):
    return b.lib.mamba_gated_delta_fwd(q, k, v, dt, A, beta, z, nw, db, h0, out, hf, ws, ws_bytes, batch, L, H, Hk, P, N, 1.0, 1e-6, 1, 1, 1, io, None)


def step(b, ho=Pt(0), hi=Pt(1), parent=Pt(2), q=Pt(3), k=Pt(4), v=Pt(5), dt=Pt(6), A=Pt(7), beta=Pt(8), z=Pt(9), nw=Pt(10), db=Pt(11), out=Pt(12),
         n_out=4, n_in=2, H=8, Hk=4, P=64, N=128, io=1):
    return b.lib.mamba_gated_delta_step(ho, hi, parent, q, k, v, dt, A, beta, z, nw, db, out, n_out, n_in, H, Hk, P, N, 1.0, 1e-6, 1, 1, 1, io, None)


def test_fwd_refusals(m):
    S = m.STATUS
    for name in ("q", "k", "v", "dt", "A", "beta", "out"):
        assert fwd(m, **{name: None}) == S["NULL_POINTER"], name
    for name in ("q", "k", "v", "dt", "A", "beta", "z", "nw", "db", "h0", "out", "hf", "ws"):
        assert fwd(m, **{name: Pt(30) + 4}) == S["MISALIGNED"], name
    for name in ("q", "k", "v", "dt", "A", "beta", "z", "nw", "db", "h0", "hf"):
        assert fwd(m, **{name: Pt(10)}) == S["ALIAS"], name                     # over out
    for name in ("q", "k", "v", "dt", "A", "beta", "z", "nw", "db"):
        assert fwd(m, **{name: Pt(11)}) == S["ALIAS"], name                     # over h_final
    assert fwd(m, hf=Pt(9) + 64) == S["ALIAS"] and fwd(m, h0=Pt(11) + 8 * 64 * 128 * 4 - 16) == S["ALIAS"]
    for bad in (dict(batch=-1), dict(L=-1), dict(H=-8), dict(Hk=-4), dict(P=-64), dict(N=-128), dict(L=1 << 40, H=1 << 30)):
        assert fwd(m, **bad) == S["BAD_SHAPE"], bad
    for bad in (dict(io=2), dict(io=-1), dict(P=32), dict(P=256), dict(N=16), dict(N=96), dict(Hk=3), dict(Hk=0), dict(Hk=16), dict(batch=70000),
                dict(H=70000, Hk=1), dict(batch=1025, H=512), dict(L=(1 << 31) + 1)):
        assert fwd(m, **bad) == S["UNSUPPORTED"], bad
    assert fwd(m, batch=0) == 0 and fwd(m, H=0, Hk=0) == 0 and fwd(m, L=0, hf=None) == 0 and fwd(m, L=0, hf=Pt(9)) == 0
    need = m.mamba_gated_delta_workspace_bytes(1, 100, 8, 4, 64, 128)
    if need:
        assert fwd(m, ws=None) == S["WORKSPACE"] and fwd(m, ws_bytes=need - 1) == S["WORKSPACE"]
        for name in ("q", "k", "v", "dt", "A", "beta", "z", "nw", "db", "h0", "hf", "out"):
            assert fwd(m, **{name: Pt(12)}) == S["ALIAS"], name                 # over the workspace
    assert need > 0 and fwd(m, L=0, hf=None, ws=None) == 0
    for bad in ((0, 8, 8, 4, 64, 128), (1, 0, 8, 4, 64, 128), (1, 8, 8, 3, 64, 128), (1, 8, 8, 4, 64, 32), (1, 1 << 50, 1 << 12, 4, 64, 128)):
        assert m.mamba_gated_delta_workspace_bytes(*bad) == 0


def test_step_refusals(m):
    S = m.STATUS
    for name in ("ho", "hi", "q", "k", "v", "dt", "A", "beta", "out"):
        assert step(m, **{name: None}) == S["NULL_POINTER"], name
    for name in ("ho", "hi", "parent", "q", "k", "v", "dt", "A", "beta", "z", "nw", "db", "out"):
        assert step(m, **{name: Pt(30) + 8}) == S["MISALIGNED"], name
    for name in ("parent", "q", "k", "v", "dt", "A", "beta", "z", "nw", "db"):
        assert step(m, **{name: Pt(0)}) == S["ALIAS"] and step(m, **{name: Pt(12)}) == S["ALIAS"], name
    assert step(m, hi=Pt(0)) == S["ALIAS"] and step(m, ho=Pt(12)) == S["ALIAS"]
    assert step(m, parent=None, n_in=4, hi=Pt(0) + 16) == S["ALIAS"]
    assert step(m, parent=None) == S["BAD_SHAPE"] and step(m, n_in=0) == S["BAD_SHAPE"] and step(m, n_out=-1) == S["BAD_SHAPE"]
    for bad in (dict(io=7), dict(P=16), dict(N=32), dict(Hk=5), dict(n_out=70000)):
        assert step(m, **bad) == S["UNSUPPORTED"], bad
    assert step(m, n_out=0) == 0 and step(m, n_out=0, n_in=0) == 0 and step(m, H=0, Hk=0) == 0


def test_the_binding_refuses(m):
    z, bf = torch.zeros, torch.bfloat16
    q, v, d, A, h = z(1, 8, 2, 64, dtype=bf), z(1, 8, 4, 64, dtype=bf), z(1, 8, 4, dtype=bf), z(4), z(2, 4, 64, 64)
    with pytest.raises(ValueError, match="v must live on the GPU"):
        m.mamba_gated_delta_fwd(q, q, v, d, A, d)
    with pytest.raises(ValueError, match="v must live on the GPU"):
        m.mamba_gated_delta_step(h, q[0], q[0], v[0], d[0], A, d[0])
    for bad in (None, 3, "v", [1.0]):
        with pytest.raises(TypeError, match="v must be a tensor"):
            m.mamba_gated_delta_fwd(q, q, bad, d, A, d)
        with pytest.raises(TypeError, match="v must be a tensor"):
            m.mamba_gated_delta_step(h, q[0], q[0], bad, d[0], A, d[0])
    with pytest.raises(ValueError, match="v must have 4 dimensions, got 3"):
        m.mamba_gated_delta_fwd(q, q, v[0], d, A, d)
    with pytest.raises(ValueError, match="q must have 4 dimensions, got 3"):
        m.mamba_gated_delta_fwd(q[0], q, v, d, A, d)
    with pytest.raises(TypeError, match="I/O tensors must be float32 or bfloat16"):
        m.mamba_gated_delta_fwd(q, q, v.half(), d, A, d)
    for name, n in (("gated_delta_fwd", 20), ("gated_delta_step", 19)):
        for args in ((), (None,) * (n - 1), (None,) * (n + 1)):
            with pytest.raises(TypeError, match="%d arguments expected, got %d" % (n, len(args))):
                getattr(m._delta, name)(*args)


# ------------------------------------------------------------------------------------------------ kernels against the oracle
SHAPES = [  # B, L, H, Hk, N, P, z, norm
    (1, 1, 1, 1, 64, 64, True, True), (2, 2, 2, 1, 128, 64, False, True), (1, 63, 3, 1, 64, 128, True, False),
    (3, 64, 2, 2, 128, 128, True, True), (1, 65, 4, 2, 64, 64, False, False), (2, 130, 6, 2, 128, 64, True, True),
    (1, 333, 3, 3, 64, 128, True, True), (1, 700, 2, 1, 128, 128, False, True), (2, 257, 4, 4, 64, 64, True, True),
    (5, 17, 2, 2, 128, 128, True, False)]


@pytest.mark.gpu
@pytest.mark.parametrize("io", [synth.BF16, synth.F32])
@pytest.mark.parametrize("B,L,H,Hk,N,P,z,norm", SHAPES)
def test_fwd_against_the_oracle(m, B, L, H, Hk, N, P, z, norm, io):
    print("\n[gpu-case] gated delta B=%d L=%d H=%d/%d N=%d P=%d io=%s" % (B, L, H, Hk, N, P, io), flush=True)
    rng = np.random.default_rng(B * 10007 + L * 101 + H)
    c, h0 = case(rng, B, L, H, Hk, N, P, io, z, norm), state(rng, B, H, P, N)
    g = device(c)
    for start in (None, h0):
        out, hf = m.mamba_gated_delta_fwd(**g, h0=to_dev(start))
        ro, rh = oracle_scan(c, start)
        assert_close(values(to_host(out)), ro, TOL[io], "out")
        assert_close(to_host(hf), rh, TOL_F32, "final state")
    # two pieces, the state carried in place, are the whole
    cut = L // 2
    if cut:
        piece = lambda lo, hi: {n: x if x is None or n in ("A", "dt_bias", "norm_w") else x[:, lo:hi].clone() for n, x in g.items()}
        h = to_dev(h0)
        o1, _ = m.mamba_gated_delta_fwd(**piece(0, cut), h0=h, h_final=h)
        o2, _ = m.mamba_gated_delta_fwd(**piece(cut, L), h0=h, h_final=h)
        assert_close(values(to_host(torch.cat([o1, o2], 1))), ro, TOL[io], "out of two pieces")
        assert_close(to_host(h), rh, 2 * TOL_F32, "state of two pieces")


@pytest.mark.gpu
@pytest.mark.parametrize("options", [dict(qk_norm=False, scale=0.02), dict(dt_softplus=False), dict(beta_sigmoid=False), dict(eps=1e-2, scale=1.0)])
@pytest.mark.parametrize("L", [5, 100])
def test_fwd_options(m, L, options):
    print("\n[gpu-case] gated delta options %s L=%d" % (options, L), flush=True)
    rng = np.random.default_rng(L)
    c = case(rng, 1, L, 4, 2, 64, 64)
    if "qk_norm" in options:                                     # keys of a length below one, as the rule needs them
        c["k"] = storage(W(c["k"]) * 0.1, synth.BF16)
    if "dt_softplus" in options:
        c["dt"], c["dt_bias"] = storage(np.abs(W(c["dt"])) * 0.05, synth.BF16), None
    if "beta_sigmoid" in options:                                # write strengths up to two
        c["beta"] = storage(rng.uniform(0, 2, (1, L, 4)), synth.BF16)
    out, hf = m.mamba_gated_delta_fwd(**device(c), **options)
    ro, rh = oracle_scan(c, **options)
    assert_close(values(to_host(out)), ro, TOL_BF16, "out")
    assert_close(to_host(hf), rh, TOL_F32, "final state")


@pytest.mark.gpu
@pytest.mark.parametrize("alike,A,beta", [(1.0, -0.01, 8.0), (0.9, 0.0, 8.0), (0.5, -100.0, 0.0), (0.0, -16.0, 8.0), (1.0, 0.0, -8.0)])
def test_fwd_keys_that_lean_to_one_side_and_extreme_decays(m, alike, A, beta):
    """Keys that are all the same, written with strength one and kept for ever, or forgotten at once: where a triangular system of
    the chunk is worst (its powers grow like binomials, its inverse does not)."""
    print("\n[gpu-case] gated delta alike=%g A=%g beta=%g" % (alike, A, beta), flush=True)
    rng = np.random.default_rng(7)
    c = case(rng, 1, 200, 2, 2, 128, 64, z=False, norm=False, alike=alike)
    c["A"] = np.full(2, A, np.float32)
    c["beta"] = storage(W(c["beta"]) + beta, synth.BF16)
    out, hf = m.mamba_gated_delta_fwd(**device(c))
    ro, rh = oracle_scan(c)
    assert_close(values(to_host(out)), ro, TOL_BF16, "out")
    assert_close(to_host(hf), rh, TOL_F32, "final state")


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,L", [(1, 2, 6), (1, 2, 7), (64, 4, 16), (64, 4, 17), (51, 5, 7)])
def test_fwd_of_a_few_tokens(m, B, H, L):
    """On both sides of the lengths up to which a context goes token after token."""
    print("\n[gpu-case] gated delta few tokens B=%d H=%d L=%d" % (B, H, L), flush=True)
    rng = np.random.default_rng(B + L)
    c, h0 = case(rng, B, L, H, 1, 64, 64), state(rng, B, H, 64, 64)
    out, hf = m.mamba_gated_delta_fwd(**device(c), h0=to_dev(h0))
    ro, rh = oracle_scan(c, h0)
    assert_close(values(to_host(out)), ro, TOL_BF16, "out")
    assert_close(to_host(hf), rh, TOL_F32, "final state")


@pytest.mark.gpu
@pytest.mark.parametrize("z,norm", [(True, True), (True, False), (False, False)])
def test_fwd_of_a_context_in_several_slabs(m, z, norm):
    """More chunks than one preparation takes at once: the state goes from slab to slab, in the caller's tensor or in the workspace."""
    print("\n[gpu-case] gated delta slabs z=%s norm=%s" % (z, norm), flush=True)
    rng = np.random.default_rng(12)
    B, L, H, Hk, N, P = 8, 17 * 64 + 3, 32, 8, 64, 64
    assert m.mamba_gated_delta_workspace_bytes(B, 64 * L, H, Hk, P, N) < 2 * m.mamba_gated_delta_workspace_bytes(B, L, H, Hk, P, N)
    c, h0 = case(rng, B, L, H, Hk, N, P, z=z, norm=norm), state(rng, B, H, P, N)
    g, h = device(c), to_dev(h0)
    out, hf = m.mamba_gated_delta_fwd(**g, h0=h)
    for b, i in ((0, 0), (0, 31), (3, 13), (7, 4), (7, 31)):
        part = {n: x if x is None or n == "norm_w" else x[i:i + 1] if n in ("A", "dt_bias") else
                x[b:b + 1, :, i * Hk // H][:, :, None] if n in ("q", "k") else x[b:b + 1, :, i:i + 1] for n, x in c.items()}
        ro, rh = oracle_scan(part, h0[b:b + 1, i:i + 1])
        assert_close(values(to_host(out[b:b + 1, :, i:i + 1].contiguous())), ro, TOL_BF16, "out")
        assert_close(to_host(hf[b:b + 1, i:i + 1].contiguous()), rh, TOL_F32, "final state")
    o2, none = m.mamba_gated_delta_fwd(**g, h0=h, want_state=False)
    assert none is None and torch.equal(o2, out)
    o3, h3 = m.mamba_gated_delta_fwd(**g, h0=h, h_final=h)
    assert h3 is h and torch.equal(o3, out) and torch.equal(h, hf)


@pytest.mark.gpu
@pytest.mark.parametrize("B,L,H,Hk,N,P,A,z,norm", [(1, 2100, 2, 1, 64, 64, None, True, True), (2, 1999, 2, 2, 128, 64, -0.01, True, False),
                                                   (1, 3001, 3, 3, 64, 128, None, False, False), (1, 2305, 1, 1, 128, 128, -0.01, False, True),
                                                   (1, 17001, 8, 4, 64, 64, None, True, False), (1, 961, 1, 1, 64, 64, -300.0, False, False)])
def test_fwd_of_long_contexts_of_few_heads(m, B, L, H, Hk, N, P, A, z, norm):
    """The parts of a long context at once, joined by their maps of the state; with decays that keep a state through all of it, and with
    ones that leave nothing of it."""
    print("\n[gpu-case] gated delta parts B=%d L=%d H=%d/%d N=%d P=%d A=%s" % (B, L, H, Hk, N, P, A), flush=True)
    rng = np.random.default_rng(L)
    c, h0 = case(rng, B, L, H, Hk, N, P, z=z, norm=norm), state(rng, B, H, P, N)
    if A is not None:
        c["A"] = np.full(H, A, np.float32)
    g, h = device(c), to_dev(h0)
    ro, rh = oracle_scan(c, h0)
    out, hf = m.mamba_gated_delta_fwd(**g, h0=h)
    assert_close(values(to_host(out)), ro, TOL_BF16, "out")
    assert_close(to_host(hf), rh, TOL_F32, "final state")
    for _ in range(2):
        o2, h2 = m.mamba_gated_delta_fwd(**g, h0=h)
        assert torch.equal(o2, out) and torch.equal(h2, hf)
    o2, none = m.mamba_gated_delta_fwd(**g, h0=h, want_state=False)
    assert none is None and torch.equal(o2, out)
    o2, h2 = m.mamba_gated_delta_fwd(**g, h0=h, h_final=h)
    assert h2 is h and torch.equal(o2, out) and torch.equal(h, hf)
    g["v"][0, L // 2, 0, 5] = float("nan")                       # a channel's NaN stays in the channel, also on its way through the joins
    _, h2 = m.mamba_gated_delta_fwd(**g, h0=to_dev(h0))
    want = hf.clone()
    want[0, 0, 5] = float("nan")
    assert torch.equal(torch.isnan(h2), torch.isnan(want)) and torch.equal(torch.nan_to_num(h2), torch.nan_to_num(want))


@pytest.mark.gpu
def test_fwd_without_tokens_and_empty(m):
    rng = np.random.default_rng(5)
    h0 = to_dev(state(rng, 2, 4, 64, 128))
    z, bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV), torch.bfloat16
    args = (z(2, 0, 2, 128), z(2, 0, 2, 128), z(2, 0, 4, 64), z(2, 0, 4), torch.zeros(4, device=DEV), z(2, 0, 4))
    out, hf = m.mamba_gated_delta_fwd(*args, h0=h0)
    assert out.shape == (2, 0, 4, 64) and torch.equal(hf, h0)
    _, hf = m.mamba_gated_delta_fwd(*args)
    assert bool((hf == 0).all())


@pytest.mark.gpu
def test_fwd_leaves_what_is_not_its_own(m):
    """Rows of a larger buffer behind the last sequence, and the inputs, stay as they were; want_state=False writes no state."""
    rng = np.random.default_rng(6)
    c = case(rng, 2, 77, 4, 4, 64, 64)
    g = device(c)
    before = {n: None if x is None else x.clone() for n, x in g.items()}
    big = torch.full((3, 77, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    hbig = torch.full((3, 4, 64, 64), 7.0, device=DEV)
    out, hf = m.mamba_gated_delta_fwd(**g, out=big[:2], h_final=hbig[:2])
    ref, rh = m.mamba_gated_delta_fwd(**g)
    assert torch.equal(big[:2], ref) and torch.equal(hbig[:2], rh)
    assert bool((big[2] == 7).all()) and bool((hbig[2] == 7).all())
    assert all(x is None or torch.equal(x, before[n]) for n, x in g.items())
    out, hf = m.mamba_gated_delta_fwd(**g, want_state=False)
    assert hf is None and torch.equal(out, ref)


@pytest.mark.gpu
def test_fwd_nan_stays_in_its_sequence_and_head(m):
    rng = np.random.default_rng(8)
    c = case(rng, 2, 200, 2, 2, 64, 64)
    g = device(c)
    ref, rh = m.mamba_gated_delta_fwd(**g)
    g["v"][1, 150, 1, 3] = float("nan")
    out, hf = m.mamba_gated_delta_fwd(**g)
    assert torch.equal(out[0], ref[0]) and torch.equal(out[1, :, 0], ref[1, :, 0])
    assert torch.equal(out[1, :150 - 63, 1], ref[1, :150 - 63, 1]) and bool(torch.isnan(out[1, 150:, 1]).any(-1).all())
    assert torch.equal(hf[0], rh[0]) and torch.equal(hf[1, 0], rh[1, 0]) and bool(torch.isnan(hf[1, 1, 3]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("norm", [False, True])
def test_fwd_beyond_32_bit_offsets(m, norm):
    """More than 2^31 values: the last head's outputs and state are those of that head by itself, which goes in other slabs and parts."""
    print("\n[gpu-case] gated delta beyond 2^31 elements norm=%s" % norm, flush=True)
    L, H, N, P = 131072 + 70, 128, 64, 128
    gen = torch.Generator(device=DEV).manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(torch.bfloat16)
    q, k, v, dt, beta = n(1, L, 1, N), n(1, L, 1, N), n(1, L, 1, P), n(1, L, 1), n(1, L, 1)
    A, bias, w = -torch.linspace(0.05, 4, H, device=DEV), torch.full((H,), -3.0, device=DEV), torch.ones(P, device=DEV) if norm else None
    heads = lambda x: x.expand(1, L, H, *x.shape[3:]).contiguous()
    out, hf = m.mamba_gated_delta_fwd(q, k, heads(v), heads(dt), A, heads(beta), norm_w=w, dt_bias=bias)
    for h in (0, H - 1):
        ro, rh = m.mamba_gated_delta_fwd(q, k, v, dt, A[h:h + 1].clone(), beta, norm_w=w, dt_bias=bias[:1])
        # both within TOL_BF16 of the same
        assert_close(values(to_host(out[:, -200:, h:h + 1].contiguous())), values(to_host(ro[:, -200:].contiguous())), 2 * TOL_BF16, "out")
        assert_close(to_host(hf[:, h:h + 1].contiguous()), values(to_host(rh)), 2 * TOL_F32, "state")
    del out
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_step_beyond_32_bit_offsets(m):
    print("\n[gpu-case] gated delta step beyond 2^31 elements", flush=True)
    rng = np.random.default_rng(13)
    n_out, H, N, P = 1030, 128, 128, 128
    c = {n: x[:, 0] if n in ("q", "k", "v", "dt", "beta", "z") and x is not None else x for n, x in case(rng, 2, 1, H, 2, N, P).items()}
    g, h = device(c), to_dev(state(rng, 2, H, P, N))
    rh, ro = m.mamba_gated_delta_step(h, **g)
    many = {n: x.repeat(n_out // 2, *[1] * (x.dim() - 1)) if n in ("q", "k", "v", "dt", "beta", "z") else x for n, x in g.items()}
    parent = torch.arange(n_out, device=DEV, dtype=torch.int32) % 2
    ho, out = m.mamba_gated_delta_step(h, **many, parent_idx=parent)
    assert torch.equal(ho[-2:], rh) and torch.equal(out[-2:], ro) and torch.equal(ho[:2], rh)
    h2, o2 = m.mamba_gated_delta_step(ho, **many, parent_idx=torch.arange(n_out, device=DEV, dtype=torch.int32).flip(0))
    assert torch.equal(h2[0], h2[-2]) and torch.equal(h2[1], h2[-1]) and not torch.equal(h2[0], ho[0])
    del ho, h2
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("io", [synth.BF16, synth.F32])
@pytest.mark.parametrize("n_out,n_in,H,Hk,N,P,z,norm", [
    (1, 1, 1, 1, 64, 64, True, True), (6, 3, 4, 2, 128, 64, True, False), (18, 9, 3, 1, 64, 128, False, True), (33, 33, 2, 2, 128, 128, True, True),
    (2, 5, 24, 24, 128, 64, False, False)])
def test_step_against_the_oracle(m, io, n_out, n_in, H, Hk, N, P, z, norm):
    from oracle import delta
    print("\n[gpu-case] gated delta step n_out=%d H=%d/%d N=%d P=%d io=%s" % (n_out, H, Hk, N, P, io), flush=True)
    rng = np.random.default_rng(n_out * 31 + H)
    c = {n: x[:, 0] if n in ("q", "k", "v", "dt", "beta", "z") and x is not None else x for n, x in case(rng, n_out, 1, H, Hk, N, P, io, z, norm).items()}
    h = state(rng, n_in, H, P, N)
    parent = rng.integers(0, n_in, n_out).astype(np.int32)
    g, w = device(c), {n: W(x) for n, x in c.items()}
    ho, out = m.mamba_gated_delta_step(to_dev(h), **g, parent_idx=to_dev(parent))
    rh, ro = delta.delta_step(h, parent=parent, **w)
    assert_close(values(to_host(out)), ro, TOL[io], "step out")
    assert_close(to_host(ho), rh, 1e-5, "step state")
    # the fork as a launch of its own, and then the step in place, gives the same bits
    _, forked = m.mamba_state_fork(None, to_dev(h).view(1, n_in, H * P, N), to_dev(parent))
    forked = forked.view(n_out, H, P, N)
    h2, out2 = m.mamba_gated_delta_step(forked, **g, h_out=forked)
    assert h2 is forked and torch.equal(h2, ho) and torch.equal(out2, out)
    # and so does a sequence of one token
    if n_in == n_out:
        o3, h3 = m.mamba_gated_delta_fwd(**{n: x[:, None].contiguous() if n in ("q", "k", "v", "dt", "beta", "z") and x is not None else x
                                            for n, x in g.items()}, h0=to_dev(h[parent]))
        assert_close(values(to_host(o3))[:, 0], ro, TOL[io], "sequence of one token")
        assert_close(to_host(h3), rh, TOL_F32, "state of a sequence of one token")


@pytest.mark.gpu
def test_step_with_a_parent_that_is_not_there(m):
    rng = np.random.default_rng(9)
    c = {n: x[:, 0] if n in ("q", "k", "v", "dt", "beta", "z") else x for n, x in case(rng, 4, 1, 4, 2, 64, 64).items()}
    g, h = device(c), to_dev(state(rng, 3, 4, 64, 64))
    ho, out = m.mamba_gated_delta_step(h, **g, parent_idx=torch.tensor([0, 3, -1, 2], dtype=torch.int32, device=DEV))
    good, gout = m.mamba_gated_delta_step(h, **g, parent_idx=torch.tensor([0, 1, 1, 2], dtype=torch.int32, device=DEV))
    for j in (0, 3):
        assert torch.equal(ho[j], good[j]) and torch.equal(out[j], gout[j])
    for j in (1, 2):
        assert bool(torch.isnan(ho[j]).all()) and bool(torch.isnan(out[j]).all())


@pytest.mark.gpu
def test_prefill_and_draft_on_another_stream_and_replayed(m):
    """A context on a side stream, then a tree of draft steps captured into a graph and replayed; every replay is the eager result."""
    rng = np.random.default_rng(10)
    tree, H, Hk, N, P = (3, 2), 4, 2, 64, 64
    g = device(case(rng, 1, 150, H, Hk, N, P))
    ref, rh = m.mamba_gated_delta_fwd(**g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, root = m.mamba_gated_delta_fwd(**g, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, ref) and torch.equal(root, rh)
    steps, width = [], 1
    for n in tree:
        width *= n
        c = device({k: x[:, 0] if k in ("q", "k", "v", "dt", "beta", "z") else x for k, x in case(rng, width, 1, H, Hk, N, P).items()})
        parent = torch.arange(width, device=DEV, dtype=torch.int32) // n
        steps.append((c, parent, torch.empty(width, H, P, N, device=DEV), torch.empty(width, H, P, dtype=torch.bfloat16, device=DEV)))

    def draft():
        h = root
        for c, parent, ho, o in steps:
            m.mamba_gated_delta_step(h, **c, parent_idx=parent, h_out=ho, out=o)
            h = ho
    draft()
    want = [(ho.clone(), o.clone()) for _, _, ho, o in steps]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        draft()
    for _ in range(3):
        for _, _, ho, o in steps:
            ho.fill_(5.0), o.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(ho, a) and torch.equal(o, b) for (_, _, ho, o), (a, b) in zip(steps, want))
        draft()


@pytest.mark.gpu
def test_fwd_of_a_context_captured_and_replayed(m):
    rng = np.random.default_rng(11)
    g = device(case(rng, 1, 300, 4, 2, 128, 64))
    ref, rh = m.mamba_gated_delta_fwd(**g)
    out, hf = torch.empty_like(ref), torch.empty_like(rh)
    ws = torch.empty(max(16, m.mamba_gated_delta_workspace_bytes(1, 300, 4, 2, 64, 128)), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.mamba_gated_delta_fwd(**g, out=out, h_final=hf, workspace=ws)
    for fill in (0, 255, 127):
        out.fill_(3.0), hf.fill_(3.0), ws.fill_(fill)            # nothing in the workspace is taken from before
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(hf, rh)
