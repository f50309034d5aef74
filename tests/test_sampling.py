"""Drawn children and next tokens (mamba_sample_fwd): pins of the oracle, refusals (no GPU needed), and the kernels against the oracle."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import sampling as oracle


# ----------------------------------------------------------------------------------------------------------- the oracle
def test_oracle_distributions_by_hand():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    close = lambda q, r: np.allclose(q, r, rtol=1e-14, atol=0)
    assert close(oracle.distribution(x), [0.1, 0.4, 0.2, 0.3])
    assert close(oracle.distribution(x, top_k=2), [0, 4 / 7, 0, 3 / 7])
    assert close(oracle.distribution(x, top_p=0.65), [0, 4 / 7, 0, 3 / 7])
    assert close(oracle.distribution(x, top_p=0.0), [0, 1, 0, 0])
    assert close(oracle.distribution(x, min_p=0.6), [0, 4 / 7, 0, 3 / 7])
    assert close(oracle.distribution(x, top_k=3, top_p=0.7), [0, 4 / 7, 0, 3 / 7])       # 0.4 + 0.3 of 0.9 is 0.78
    assert close(oracle.distribution(x, 0.5), np.array([1, 16, 4, 9]) / 30)
    assert close(oracle.distribution(x, 0.0), [0, 1, 0, 0])
    assert close(oracle.distribution([1.0, 1.0, 1.0], top_k=2), [0.5, 0.5, 0])
    assert close(oracle.distribution([np.nan, -np.inf, 0.0]), [0, 0, 1])
    assert not oracle.distribution([np.nan, -np.inf]).any()
    assert oracle.distribution(x, -1.0) is None and oracle.distribution(x, 1.0, np.nan) is None


def test_oracle_draws_follow_the_distribution():
    q = np.array([0.1, 0.4, 0.2, 0.3])
    assert [oracle.draw(q, u) for u in (0.0, 0.099, 0.1001, 0.49, 0.51, 0.69, 0.71, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    idx, prob, dist = oracle.sample(np.log(q)[None], np.array([[0.3, 0.0, 0.99]]), np.array([[1.0, 1.0, 0.0]]))
    assert idx.tolist() == [[1, 0, 3]] and np.allclose(prob, [[0.4, 0.1, 0.3]]) and np.allclose(dist, q)


# ----------------------------------------------------------------------------------------------------------- refusals, without a GPU
def P(i):
    return (i + 1) << 40


@pytest.fixture(scope="module")
def m():
    from paper_2506_01206_amd import binding
    return binding


def call(m, logits=P(0), params=P(1), top_k=None, seq_idx=None, path=None, n_seq=1, path_len=0, u=P(2), idx=P(3), prob=P(4), dist=None, path_out=None,
         ws=P(5), ws_bytes=1 << 39, M=4, V=5000, k=2, io=1, s=True):
    st = m.Sampling(params, top_k, seq_idx, path, n_seq, path_len)
    return m.lib.mamba_sample_fwd(logits, ctypes.byref(st) if s else None, u, idx, prob, dist, path_out, ws, ws_bytes, M, V, k, io, None)


def test_refusals(m):
    S = m.STATUS
    for name in ("logits", "params", "u", "idx", "prob"):
        assert call(m, **{name: None}) == S["NULL_POINTER"], name
        assert call(m, **{name: P(9) + 4}) == S["MISALIGNED"], name
    for name in ("top_k", "seq_idx", "path", "path_out", "ws"):
        assert call(m, **{name: P(9) + 4}) == S["MISALIGNED"], name
    assert call(m, dist=P(9) + 2) == S["MISALIGNED"]
    assert call(m, s=False) == S["NULL_POINTER"]
    assert call(m, path_len=3, path_out=P(9)) == S["NULL_POINTER"]
    assert call(m, ws=None) == S["WORKSPACE"] and call(m, ws_bytes=m.mamba_sample_workspace_bytes(4, 5000, 2) - 1) == S["WORKSPACE"]
    for bad in (dict(M=-1), dict(V=-1), dict(V=0), dict(n_seq=-1), dict(n_seq=0), dict(n_seq=3), dict(path_len=-1), dict(M=1 << 40, V=1 << 40)):
        assert call(m, **bad) == S["BAD_SHAPE"], bad
    for bad in (dict(k=0), dict(k=9), dict(io=2), dict(io=-1), dict(V=(1 << 21) + 1), dict(M=1 << 24), dict(path_len=4097, path=P(9))):
        assert call(m, **bad) == S["UNSUPPORTED"], bad
    assert call(m, M=0) == S["OK"]
    # outputs that are inputs, or one another
    for a, b in (("idx", 2), ("prob", 0), ("dist", 1), ("path_out", 3), ("ws", 0), ("idx", 5), ("dist", 5), ("path_out", 4)):
        assert call(m, **{a: P(b)}) == S["ALIAS"], (a, b)
    assert m.mamba_sample_workspace_bytes(4, 5000, 2) > 0
    for bad in ((0, 5000, 2), (4, 0, 2), (4, 5000, 0), (4, 5000, 9), (4, (1 << 21) + 1, 1), (1 << 24, 5000, 1), (-1, 5, 1)):
        assert m.mamba_sample_workspace_bytes(*bad) == 0, bad


def test_binding_refuses_what_is_not_there(m):
    x, u, par = torch.zeros(2, 9), torch.zeros(2, 1), torch.ones(1, 3)
    with pytest.raises(ValueError, match="GPU"):
        m.mamba_sample_fwd(x, u, par)
    with pytest.raises(TypeError):
        m.mamba_sample_fwd(x.half(), u, par)
    with pytest.raises(ValueError):
        m.mamba_sample_fwd(x[0], u, par)


# ----------------------------------------------------------------------------------------------------------- the kernels
gpu = pytest.mark.gpu
DEV = "cuda:0"
HALF = 2.0 ** -24                                                # a rounding to float32


def to_dev(a, dtype=None):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def check(m, x, u, params, top_k=None, seq_idx=None, bf16=False, **kw):
    """One call against the oracle on the same stored inputs: tokens equal, probabilities one rounding away."""
    t = to_dev(x.astype(np.float32), torch.bfloat16 if bf16 else torch.float32)
    stored = t.float().cpu().double().numpy()
    u, params = np.asarray(u, np.float32), np.asarray(params, np.float32)
    d = dict(top_k=to_dev(None if top_k is None else np.asarray(top_k, np.int32)), seq_idx=to_dev(None if seq_idx is None else np.asarray(seq_idx, np.int32)))
    idx, prob, dist, _ = m.mamba_sample_fwd(t, to_dev(u), to_dev(params), want_dist=True, **d, **kw)
    ri, rp, rd = oracle.sample(stored, u, params, top_k, seq_idx)
    assert np.array_equal(idx.cpu().numpy(), ri), (idx.cpu().numpy()[:4], ri[:4])
    # one rounding; the sum of the weights is off by less than V 2^-42 of the largest, the weights by a few roundings of float64
    for got, ref in ((prob, rp), (dist, rd)):
        got = got.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        ok = ~np.isnan(ref)
        assert (np.abs(got[ok] - ref[ok]) <= ref[ok] * (HALF + 1e-9) + 2.0 ** -149).all()
    return idx, prob, dist


def rows(rng, M, V, std=2.5):
    return rng.standard_normal((M, V)) * std


SETTINGS = [(1.0, 1.0, 0.0, 0), (0.7, 0.9, 0.0, 0), (1.3, 1.0, 0.05, 0), (0.8, 1.0, 0.0, 40), (0.9, 0.95, 0.02, 50), (0.0, 0.5, 0.3, 7), (1.0, 0.0, 0.0, 0), (3.0, 0.6, 0.0, 700),
            (0.05, 0.99, 0.0, 30), (1.0, 1.0, 2.0, 0), (50.0, 0.7, 0.0, 0), (1.0, 2.0, -1.0, -5)]


@gpu
@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("M,V,k", [(1, 1, 1), (2, 3, 3), (3, 7, 8), (5, 8, 2), (4, 9, 4), (3, 2047, 2), (3, 2048, 1), (2, 2049, 3), (7, 5001, 2), (2, 50280, 3)])
def test_against_oracle(m, M, V, k, bf16):
    rng = np.random.default_rng(V + k)
    for n, (T, p, q, top_k) in enumerate(SETTINGS):
        check(m, rows(rng, M, V), rng.uniform(size=(M, k)), [[T, p, q]], [top_k], bf16=bf16)


@gpu
def test_sequences_of_their_own(m):
    rng = np.random.default_rng(3)
    S = len(SETTINGS)
    par, top_k = [s[:3] for s in SETTINGS], [s[3] for s in SETTINGS]
    seq = rng.integers(0, S, 40)
    check(m, rows(rng, 40, 3001), rng.uniform(size=(40, 2)), par, top_k, seq)
    check(m, rows(rng, S, 3001), rng.uniform(size=(S, 5)), par, top_k)               # row m's own
    check(m, rows(rng, S, 3001), rng.uniform(size=(S, 5)), par)                      # no top-k


@gpu
def test_rows_whose_settings_are_not_known(m):
    rng = np.random.default_rng(4)
    par = [[1.0, 1.0, 0.0], [-1.0, 1.0, 0.0], [np.nan, 1.0, 0.0], [1.0, np.nan, 0.0], [1.0, 1.0, np.nan], [np.inf, 1.0, 0.0], [-0.0, 1.0, 0.0]]
    seq = [0, 1, 2, 3, 4, 5, 6, -1, 7, 2 ** 31 - 1, -2 ** 31]
    x = rows(rng, len(seq), 777)
    check(m, x, rng.uniform(size=(len(seq), 3)), par, None, seq)


@gpu
@pytest.mark.parametrize("T", [1e-45, 1e-30, 1e-4, 1e6, 1e30, np.inf])
def test_temperatures_at_their_ends(m, T):
    """From rows of one token left to rows whose tokens all weigh the same, under every kind of cut."""
    rng = np.random.default_rng(12)
    x = np.concatenate([rows(rng, 3, 3001), rows(rng, 1, 3001) * 1e37, np.round(rows(rng, 2, 3001))])
    for top_p, min_p, top_k in ((1.0, 0.0, 0), (0.625, 0.0, 0), (1e-45, 0.0, 0), (1.0, 1e-45, 0), (1.0, 1.0, 0), (1.0, 0.0, 2 ** 31 - 1), (0.75, 0.5, 700)):
        check(m, x, rng.uniform(size=(6, 4)), [[T, top_p, min_p]], [top_k])


@gpu
def test_infinities_nan_and_empty_rows(m):
    rng = np.random.default_rng(5)
    x = rows(rng, 12, 5003)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, 1:] = -np.inf
    x[3, ::2] = np.nan
    x[4, [7, 4000]] = np.inf
    x[5, :5002] = -np.inf
    x[6] = 3e38 * np.sign(x[6])
    x[7] = np.finfo(np.float32).min
    x[8] = -0.0
    x[8, ::3] = 0.0
    x[9] = 1e-40
    x[10, 5:] = -np.inf
    x[11, 100:] = -1e30
    for T, p, q, top_k in SETTINGS:
        check(m, x, rng.uniform(size=(12, 3)), [[T, p, q]], [top_k])


@gpu
@pytest.mark.parametrize("V", [50280, 4097, 131071])
def test_ties(m, V):
    """Rows of a few values, whole rows of one: cuts inside ties go by the order of the vocabulary."""
    rng = np.random.default_rng(V)
    x = np.stack([np.zeros(V), rng.integers(0, 2, V), rng.integers(0, 4, V) * 0.25, np.where(np.arange(V) < 10, 5.0, 1.0)])
    for T, p, q, top_k in SETTINGS + [(1.0, 1.0, 0.0, V // 3), (1.0, 0.5, 0.0, 0), (1.0, 0.25, 0.0, V - 1), (1.0, 0.125, 0.0, V), (2.0, 1 - 2.0 ** -24, 0.0, V + 1)]:
        check(m, x, rng.uniform(size=(4, 2)), [[T, p, q]], [top_k])


@gpu
def test_random_numbers_at_their_ends(m):
    rng = np.random.default_rng(6)
    u = np.array([[0.0, 0.0], [1 - 2.0 ** -24, 1 - 2.0 ** -24], [1.0, 2.0], [-1.0, -np.inf], [np.nan, np.nan], [np.inf, 0.5], [1e-30, 2.0 ** -149], [0.5, 0.25]])
    check(m, rows(rng, 8, 6000), u, [[1.0, 1.0, 0.0]])
    check(m, np.zeros((8, 6000)), u, [[1.0, 0.5, 0.0]])


@gpu
@pytest.mark.parametrize("gap", [3.0, 12.0, 30.0, 200.0])
def test_what_is_left_beside_nearly_certain_tokens(m, gap):
    """Weights of the later children are next to nothing beside the first: drawn from all the same, by what they are among themselves."""
    rng = np.random.default_rng(int(gap))
    x = rows(rng, 6, 50280, 0.5)
    for i in range(6):
        at = rng.choice(50280, i, replace=False)
        x[i, at] += gap * (1 + np.arange(i))
    u = rng.uniform(size=(6, 8))
    check(m, x, u, [[1.0, 1.0, 0.0]])
    check(m, x, u, [[0.7, 1.0, 0.0]], [300])


@gpu
def test_paths_and_given_outputs(m):
    rng = np.random.default_rng(7)
    M, V, k, T = 9, 4001, 3, 5
    x, u, path = to_dev(rows(rng, M, V).astype(np.float32)), to_dev(rng.uniform(size=(M, k)).astype(np.float32)), to_dev(rng.integers(0, V, (M, T)).astype(np.int32))
    par = torch.tensor([[1.0, 0.9, 0.0]], device=DEV)
    idx, prob, none, path_out = m.mamba_sample_fwd(x, u, par, path=path, want_path=True)
    assert none is None
    ref = torch.cat([path.repeat_interleave(k, 0), idx.view(-1, 1)], 1)
    assert torch.equal(path_out, ref)
    # a tensor that starts anywhere for the distribution, rows behind the outputs' as they were
    flat = torch.full((M * V + 3,), 7.0, device=DEV)
    big = torch.full((M + 2, k), -7, dtype=torch.int32, device=DEV)
    ws = torch.empty(m.mamba_sample_workspace_bytes(M, V, k), dtype=torch.uint8, device=DEV)
    got = m.mamba_sample_fwd(x, u, par, idx=big[:M], prob=torch.empty(M, k, device=DEV), dist=flat[1:1 + M * V].view(M, V), workspace=ws)
    assert got[0].data_ptr() == big.data_ptr() and torch.equal(big[:M], idx) and bool((big[M:] == -7).all())
    assert float(flat[0]) == 7.0 and bool((flat[1 + M * V:] == 7.0).all())
    assert torch.equal(got[2], m.mamba_sample_fwd(x, u, par, want_dist=True)[2])
    # an empty path
    _, _, _, p0 = m.mamba_sample_fwd(x, u, par, want_path=True)
    assert torch.equal(p0, idx.view(-1, 1))
    assert m.mamba_sample_fwd(x[:0], u[:0], par)[0].shape == (0, k)


@gpu
def test_refusals_of_the_binding(m):
    x, u, par = torch.zeros(4, 100, device=DEV), torch.zeros(4, 2, device=DEV), torch.ones(1, 3, device=DEV)
    for bad in (dict(u=u[:3]), dict(u=torch.zeros(4, 9, device=DEV)), dict(u=u.double()), dict(params=par[:, :2]), dict(top_k=torch.zeros(2, dtype=torch.int32, device=DEV)),
                dict(seq_idx=torch.zeros(4, dtype=torch.int64, device=DEV)), dict(logits=x.t()), dict(logits=x.half()), dict(params=par.cpu()),
                dict(idx=torch.zeros(4, 3, dtype=torch.int32, device=DEV)), dict(dist=torch.zeros(4, 99, device=DEV))):
        with pytest.raises((ValueError, TypeError)):
            m.mamba_sample_fwd(**{**dict(logits=x, u=u, params=par), **bad})
    with pytest.raises(m.MambaError):
        m.mamba_sample_fwd(x, u, torch.ones(3, 3, device=DEV))
    with pytest.raises(m.MambaError):
        m.mamba_sample_fwd(x, u, par, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))


@gpu
def test_streams_graphs_and_repeats(m):
    """The same bits from call to call, on another stream, and from a graph that is replayed between other work."""
    rng = np.random.default_rng(8)
    M, V, k = 24, 50280, 3
    x = to_dev(rows(rng, M, V), torch.bfloat16)
    u = to_dev(rng.uniform(size=(M, k)).astype(np.float32))
    par = to_dev(np.array([SETTINGS[i % len(SETTINGS)][:3] for i in range(M)], np.float32))
    ref = m.mamba_sample_fwd(x, u, par, want_dist=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = m.mamba_sample_fwd(x, u, par, want_dist=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    outs = [torch.empty_like(t) for t in ref[:3]]
    ws = torch.empty(m.mamba_sample_workspace_bytes(M, V, k), dtype=torch.uint8, device=DEV)
    one = lambda: m.mamba_sample_fwd(x, u, par, idx=outs[0], prob=outs[1], dist=outs[2], workspace=ws)
    one()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        one()
    for _ in range(3):
        for t in outs:
            t.zero_()
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(ref, got, outs):
            assert torch.equal(a, b) and torch.equal(a, c)
        u.copy_(torch.rand_like(u))
        ref = got = m.mamba_sample_fwd(x, u, par, want_dist=True)


@gpu
def test_long_offsets(m):
    """Rows whose offsets pass 32 bits."""
    M, V = 2200, 1000003
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    x = torch.empty(M, V, dtype=torch.bfloat16, device=DEV).normal_(0, 2.0, generator=gen)
    u = torch.rand(M, 2, device=DEV, generator=gen)
    par = torch.tensor([[0.9, 0.9, 0.0]], device=DEV)
    idx, prob, _, _ = m.mamba_sample_fwd(x, u, par)
    for r in (0, 1, 1073, M - 1):
        i, p, _, _ = m.mamba_sample_fwd(x[r:r + 1].clone(), u[r:r + 1].clone(), par)
        assert torch.equal(i[0], idx[r]) and torch.equal(p[0], prob[r])
    ri, _, _ = oracle.sample(x[M - 1:].double().cpu().numpy(), u[M - 1:].cpu().numpy(), np.array([[0.9, 0.9, 0.0]], np.float32))
    assert np.array_equal(idx[M - 1:].cpu().numpy(), ri)
