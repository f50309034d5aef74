"""Token counts, constrained logits and the constrained choice of children: refusals (no GPU needed), and the kernels against the oracle.

The rules are single float32 operations in a given order, so that results are compared bit for bit: values in float32, tokens as whole
numbers, and bfloat16 logits after the one rounding to nearest at the store."""
import os

import numpy as np
import pytest
import torch

from gpu_util import DEV

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture(scope="module")
def m():
    if not os.path.exists(os.path.join(ROOT, "paper_2506_01206_amd", "libmamba_hip.so")):
        from paper_2506_01206_amd import build
        build.build()
    from paper_2506_01206_amd import binding
    return binding


def pack(allowed):
    """bool (R,V) -> int32 words (R, ceil(V/32))"""
    R, V = allowed.shape
    wide = np.zeros((R, (V + 31) // 32 * 32), np.uint8)
    wide[:, :V] = allowed
    return np.ascontiguousarray(np.packbits(wide, axis=1, bitorder="little")).view(np.int32)


def case(rng, M, V, S=1, T=0, masks=None, bias=True, counts=True, dtype=BF16):
    """One call's tensors on the CPU; masks: shares of allowed tokens, one mask each."""
    c = dict(logits=torch.from_numpy(rng.standard_normal((M, V)).astype(np.float32) * 3).to(dtype))
    c["penalties"] = torch.from_numpy(np.stack([rng.uniform(0.8, 1.5, S), rng.uniform(-0.5, 1, S), rng.uniform(0, 0.7, S)], 1).astype(np.float32))
    c["seq_idx"] = torch.from_numpy(rng.integers(0, S, M).astype(np.int32))
    if counts:
        n = rng.integers(0, 5, (S, V)) * (rng.random((S, V)) < 0.2)
        n = np.where(rng.random((S, V)) < 0.1, n - (1 << 31), n)
        c["counts"] = torch.from_numpy(n.astype(np.int32))
    if T:
        c["path"] = torch.from_numpy(np.concatenate([rng.integers(0, V, (M, T - 1)), rng.choice([-1, V, 0, V - 1], (M, 1))], 1).astype(np.int32))
    if bias:
        c["bias"] = torch.from_numpy((rng.standard_normal(V) * (rng.random(V) < 0.1)).astype(np.float32))
    if masks is not None:
        allowed = rng.random((len(masks), V)) < np.array(masks)[:, None]
        c["mask"] = torch.from_numpy(pack(allowed))
        c["mask_idx"] = torch.from_numpy(rng.integers(-1, len(masks), M).astype(np.int32))
    return c


def gpu(c):
    return {n: None if x is None else x.to(DEV) for n, x in c.items()}


def reference(c, k):
    from oracle import constrain as oc
    w = {n: x.float().numpy() if n == "logits" else x.numpy() for n, x in c.items() if x is not None}
    x, allowed = oc.constrain(**w)
    return x, allowed, oc.children(x, allowed, k, w.get("path"))


def check(m, c, k):
    x, allowed, (ri, rv, rp) = reference(c, k)
    g = gpu(c)
    want = np.where(allowed, x, np.float32(-np.inf))
    from oracle import constrain as oc
    n = lambda *names: max([c[i].shape[0] for i in names if c.get(i) is not None], default=0)
    host = lambda i: None if c.get(i) is None else c[i].numpy()
    want[~oc.known_rows(x.shape[0], n("counts", "penalties"), host("seq_idx"), n("mask"), host("mask_idx"))] = np.nan
    want = torch.from_numpy(want).to(c["logits"].dtype)
    out = m.mamba_logits_constrain_fwd(**g).cpu()
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(out.float(), 0.0), torch.nan_to_num(want.float(), 0.0))
    logits = g.pop("logits")
    idx, val, path = m.mamba_topk_constrained_fwd(logits, k, **g, want_path=True)
    assert np.array_equal(idx.cpu().numpy(), ri)
    assert np.array_equal(val.cpu().numpy(), rv)
    assert np.array_equal(path.cpu().numpy(), rp)
    return idx, val, path


# ------------------------------------------------------------------------------------------------ oracle pins
def test_oracle_on_a_case_by_hand():
    from oracle import constrain as oc
    counts = oc.token_counts(np.array([[2, 2, 5, -1, 9]]), 6, oc.token_counts(np.array([[0, 1, 1]]), 6, prompt=True))
    assert counts.tolist() == [[-(1 << 31), -(1 << 31), 2, 0, 0, 1]]
    x, allowed = oc.constrain(np.array([[4.0, -4.0, 4.0, 4.0, 4.0, -1.0]]), counts, np.array([[2.0, 0.5, 0.25]]), path=np.array([[5, 3]]),
                              bias=np.array([0, 0, 0, 0, 1.0, 0]), mask=pack(np.array([[1, 1, 1, 1, 0, 1]])), dtype=np.float64)
    # prompt only: divided, or multiplied where negative; generated: both penalties behind it
    assert x.tolist() == [[2.0, -8.0, 2 - 0.5 - 0.5, 2 - 0.25 - 0.5, 5.0, -2 - 0.5 - 0.5]] and allowed.tolist() == [[True] * 4 + [False, True]]
    idx, val, path = oc.children(x, allowed, 3, np.array([[5, 3]]))
    assert idx.tolist() == [[0, 3, 2]] and val.tolist() == [[2.0, 1.25, 1.0]] and path.tolist() == [[5, 3, 0], [5, 3, 3], [5, 3, 2]]


# ------------------------------------------------------------------------------------------------ refusals (no GPU)
def P(i):
    return (i + 1) << 40


def rules(b, counts=P(20), penalties=P(21), seq_idx=P(22), path=P(23), bias=P(24), mask=P(25), mask_idx=P(26), n_seq=2, n_masks=3, path_len=4):
    return b.Constraints(counts, penalties, seq_idx, path, bias, mask, mask_idx, n_seq, n_masks, path_len)


RULE_NAMES = ("counts", "penalties", "seq_idx", "path", "bias", "mask", "mask_idx")


def test_constrain_refusals(m):
    S = m.STATUS
    import ctypes

    def call(c=None, logits=P(0), out=P(1), M=12, V=50280, io=1, none=False):
        r = rules(m) if c is None else c
        return m.lib.mamba_logits_constrain_fwd(logits, None if none else ctypes.byref(r), out, M, V, io, None)
    assert call(none=True) == S["NULL_POINTER"] and call(logits=None) == S["NULL_POINTER"] and call(out=None) == S["NULL_POINTER"]
    assert call(io=3) == S["UNSUPPORTED"] and call(V=(1 << 25) + 1) == S["UNSUPPORTED"] and call(M=1 << 30) == S["UNSUPPORTED"]
    assert call(M=1 << 24, V=1) == S["UNSUPPORTED"] and call(M=1 << 20, V=16 * 2048) == S["UNSUPPORTED"]
    assert call(M=-1) == S["BAD_SHAPE"] and call(V=-1) == S["BAD_SHAPE"]
    assert call(logits=P(0) + 8) == S["MISALIGNED"] and call(out=P(1) + 2) == S["MISALIGNED"] and call(out=P(0) + 16) == S["ALIAS"]
    for name in RULE_NAMES:
        assert call(rules(m, **{name: P(30) + 4})) == S["MISALIGNED"], name
        assert call(rules(m, **{name: P(1)})) == S["ALIAS"], name
    for bad in (dict(n_seq=-1), dict(n_masks=-1), dict(path_len=-1), dict(n_seq=0), dict(n_masks=0), dict(seq_idx=None), dict(mask_idx=None),
                dict(n_seq=1 << 60), dict(n_masks=1 << 60)):
        assert call(rules(m, **bad)) == S["BAD_SHAPE"], bad
    assert call(rules(m, path=None)) == S["NULL_POINTER"] and call(rules(m, path_len=4097)) == S["UNSUPPORTED"]
    assert call(M=0) == 0 and call(V=0) == 0


def test_children_refusals(m):
    S = m.STATUS
    import ctypes
    need = m.mamba_topk_constrained_workspace_bytes(12, 50280, 3)
    assert need > 0 and m.mamba_topk_constrained_workspace_bytes(12, 2048, 3) == 0
    for bad in ((0, 50280, 3), (12, 0, 3), (12, 50280, 0), (12, 50280, 9), (12, (1 << 25) + 1, 3), (1 << 31, 50280, 3)):
        assert m.mamba_topk_constrained_workspace_bytes(*bad) == 0

    def call(c=None, logits=P(0), idx=P(1), val=P(2), path_out=P(3), ws=P(4), ws_bytes=need, M=12, V=50280, k=3, io=1):
        return m.lib.mamba_topk_constrained_fwd(logits, ctypes.byref(rules(m) if c is None else c), idx, val, path_out, ws, ws_bytes, M, V, k, io, None)
    for name in ("logits", "idx", "val"):
        assert call(**{name: None}) == S["NULL_POINTER"], name
    for name in ("logits", "idx", "val", "path_out", "ws"):
        assert call(**{name: P(30) + 4}) == S["MISALIGNED"], name
    assert call(ws=None) == S["WORKSPACE"] and call(ws_bytes=need - 1) == S["WORKSPACE"]
    outs = ("idx", "val", "path_out", "ws")
    for i, name in enumerate(outs):
        assert call(**{name: P(0)}) == S["ALIAS"], name
        for rule in RULE_NAMES:
            assert call(rules(m, **{rule: P(1 + i)})) == S["ALIAS"], (name, rule)
        for j in range(i):
            assert call(**{name: P(1 + j)}) == S["ALIAS"], (name, outs[j])
    for bad in (dict(k=0), dict(k=9), dict(io=2), dict(V=(1 << 25) + 1), dict(M=1 << 30)):
        assert call(**bad) == S["UNSUPPORTED"], bad
    assert call(M=-1) == S["BAD_SHAPE"] and call(V=0) == S["BAD_SHAPE"] and call(M=0) == 0


def test_token_counts_refusals(m):
    S = m.STATUS

    def call(tokens=P(0), counts=P(1), n_seq=3, L=100, V=50280, accumulate=0, prompt=0):
        return m.lib.mamba_token_counts(tokens, counts, n_seq, L, V, accumulate, prompt, None)
    assert call(tokens=None) == S["NULL_POINTER"] and call(counts=None) == S["NULL_POINTER"]
    assert call(tokens=P(0) + 4) == S["MISALIGNED"] and call(counts=P(1) + 4) == S["MISALIGNED"] and call(counts=P(0)) == S["ALIAS"]
    assert call(n_seq=-1) == S["BAD_SHAPE"] and call(L=-1) == S["BAD_SHAPE"] and call(V=-1) == S["BAD_SHAPE"]
    assert call(V=(1 << 25) + 1) == S["UNSUPPORTED"] and call(L=1 << 31) == S["UNSUPPORTED"] and call(n_seq=1 << 31) == S["UNSUPPORTED"]
    assert call(n_seq=1 << 22, V=1) == S["UNSUPPORTED"] and call(n_seq=1 << 20, V=4 * 8192) == S["UNSUPPORTED"]
    assert call(n_seq=0) == 0 and call(V=0) == 0 and call(L=0, accumulate=1) == 0


def test_the_binding_refuses(m):
    logits, i32 = torch.zeros(2, 100, dtype=BF16), torch.zeros(2, dtype=I32)
    with pytest.raises(ValueError, match="logits must live on the GPU"):
        m.mamba_logits_constrain_fwd(logits)
    with pytest.raises(ValueError, match="logits must live on the GPU"):
        m.mamba_topk_constrained_fwd(logits, 2)
    with pytest.raises(ValueError, match="tokens must live on the GPU"):
        m.mamba_token_counts(torch.zeros(1, 5, dtype=I32), 100)
    for bad in (None, 3, [1.0]):
        with pytest.raises(TypeError, match="logits must be a tensor"):
            m.mamba_logits_constrain_fwd(bad)
        with pytest.raises(TypeError, match="tokens must be a tensor"):
            m.mamba_token_counts(bad, 100)
    with pytest.raises(ValueError, match="must have 2 dimensions, got 1"):
        m.mamba_topk_constrained_fwd(logits[0], 2)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        m.mamba_logits_constrain_fwd(logits.half())
    for name, n in (("token_counts", 5), ("logits_constrain_fwd", 10), ("topk_constrained_fwd", 15)):
        for args in ((), (None,) * (n - 1), (None,) * (n + 1)):
            with pytest.raises(TypeError, match="%d arguments expected, got %d" % (n, len(args))):
                getattr(m._delta, name)(*args)


# ------------------------------------------------------------------------------------------------ kernels
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,V,S,T,masks,k", [
    (1, 1, 1, 0, None, 1), (3, 5, 1, 2, [0.5], 8), (2, 7, 2, 1, [0.0, 1.0], 3), (4, 8, 1, 0, [0.3], 2), (5, 9, 3, 3, [0.5, 0.1], 4),
    (7, 33, 2, 2, [0.9, 0.02], 8), (3, 1000, 1, 4, None, 5), (2, 2047, 1, 1, [0.7], 3), (2, 2048, 2, 2, [0.7], 8), (2, 2049, 1, 3, [0.7], 8), (2, 4099, 2, 1, [0.5, 0.0, 0.001], 8), (6, 8192, 3, 2, [0.97], 3), (2, 8193, 1, 2, [0.5], 3),
    (3, 16391, 2, 5, [0.0003, 0.6], 8), (1, 50280, 1, 0, None, 3), (13, 50280, 4, 4, [0.97, 0.5, 0.0001, 0.0], 2), (2, 131071, 2, 3, [0.5], 4),
    (1, 600000, 1, 2, [0.5], 8)])
def test_against_the_oracle(m, M, V, S, T, masks, k, dtype):
    print("\n[gpu-case] constrained children M=%d V=%d S=%d T=%d k=%d %s" % (M, V, S, T, k, dtype), flush=True)
    rng = np.random.default_rng(M * 1000003 + V)
    check(m, case(rng, M, V, S, T, masks, dtype=dtype), k)
    # rules left out, one by one
    c = case(rng, M, V, 1, T, masks, dtype=dtype)
    for name in ("bias", "counts", "path", "penalties", "mask"):
        left = {n: x for n, x in c.items() if n != name and not (name == "mask" and n == "mask_idx") and n != "seq_idx"}
        check(m, left, k)


@pytest.mark.gpu
def test_ties_infinities_and_nans(m):
    """Equal logits everywhere; zeros of both signs; NaN, infinities in allowed and in masked places; biases that are infinite."""
    print("\n[gpu-case] constrained children: special values", flush=True)
    rng = np.random.default_rng(3)
    V = 20000
    c = case(rng, 6, V, 1, 2, [0.5], counts=False)
    c["logits"][:] = 1.5
    c["bias"][:] = 0
    check(m, c, 8)
    c["logits"][0] = -0.0
    c["logits"][0, ::3] = 0.0
    c["logits"][1, ::2] = float("nan")
    c["logits"][2] = float("nan")
    c["logits"][3] = float("-inf")
    c["logits"][4, 7::1000] = float("inf")
    c["logits"][5] = torch.finfo(BF16).min
    c["bias"][5::17] = float("-inf")
    c["bias"][12::1001] = float("nan")
    for dtype in (BF16, F32):
        check(m, dict(c, logits=c["logits"].to(dtype)), 8)


@pytest.mark.gpu
@pytest.mark.parametrize("ordinary", [True, False])
def test_penalties_of_all_sizes_divide_as_float32_does(m, ordinary):
    """Quotients bit for bit: logits of all sizes by penalties of all sizes, among them those whose quotient, or its way there, is
    subnormal or too large, and neighbours of powers of two."""
    print("\n[gpu-case] penalties of all sizes, ordinary=%s" % ordinary, flush=True)
    rng = np.random.default_rng(8)
    f = np.float32
    by = [1.0, 1.3, 0.7, 3.0, 1.1, np.nextafter(f(1), f(2)), np.nextafter(f(1), f(0)), np.nextafter(f(2), f(0)), 2.0 ** -40, 2.0 ** 40, 1e6, 1e-6,
          3e-39, 1e-30, 1e38, 2.0 ** -126, 1.7e-45]
    M, V = len(by), 20000
    bits = rng.integers(0, 1 << 32, (M, V), dtype=np.uint64).astype(np.uint32)
    x = bits.view(f)
    if ordinary:                                                 # of all mantissas, exponents -40 .. 39
        x = ((bits & 0x807fffff) | (rng.integers(87, 167, (M, V)).astype(np.uint32) << 23)).view(f)
    c = dict(logits=torch.from_numpy(x.copy()), counts=torch.ones(M, V, dtype=I32), seq_idx=torch.arange(M, dtype=I32),
             penalties=torch.from_numpy(np.array([[b, 0.0, 0.0] for b in by], f)))
    check(m, c, 4)


@pytest.mark.gpu
def test_a_path_that_repeats_a_token_and_a_row_without_choice(m):
    rng = np.random.default_rng(4)
    c = case(rng, 3, 9000, 1, 0, [0.0], bias=False)
    c["path"] = torch.tensor([[5, 5, 5, 8999], [1, 2, 3, 4], [8192, 8192, 8191, 0]], dtype=I32)
    c["logits"][:, [5, 8999, 8192]] = 50.0                       # still ahead of everything behind their penalties
    c["mask_idx"] = torch.tensor([-1, 0, -1], dtype=I32)
    idx, val, path = check(m, c, 3)
    assert idx[1].tolist() == [-1, -1, -1] and bool(torch.isinf(val[1]).all()) and path[3:6, 4].tolist() == [-1, -1, -1]


@pytest.mark.gpu
def test_indices_out_of_range_read_nothing(m):
    rng = np.random.default_rng(5)
    c = case(rng, 6, 3000, 2, 1, [0.5, 0.5])
    c["seq_idx"] = torch.tensor([0, 1, 2, -1, 0, 1], dtype=I32)
    c["mask_idx"] = torch.tensor([0, 1, 0, 0, 2, -2], dtype=I32)
    idx, val, _ = check(m, c, 2)
    assert bool((idx[2:] == -1).all()) and bool((idx[:2] >= 0).all())


@pytest.mark.gpu
def test_rows_beyond_32_bit_offsets(m):
    """65 rows of the widest vocabulary: more than 2^31 logits."""
    print("\n[gpu-case] constrained logits beyond 2^31 elements", flush=True)
    M, wide = 65, 1 << 25
    logits = torch.zeros(M, wide, dtype=BF16, device=DEV)
    logits[M - 1, wide - 1], logits[M - 1, 7], logits[M - 1, 8] = 5.0, 4.0, 6.0
    logits[M - 2, 3] = 3.0
    counts = torch.zeros(1, wide, dtype=I32, device=DEV)
    counts[0, 7], counts[0, wide - 1] = 2, 1
    rules = dict(counts=counts, penalties=torch.tensor([[2.0, 0.25, 0.5]], device=DEV))
    idx, val, _ = m.mamba_topk_constrained_fwd(logits, 3, **rules)
    assert idx[M - 1].tolist() == [8, wide - 1, 7] and val[M - 1].tolist() == [6.0, 2.5 - 0.5 - 0.25, 2.0 - 1.0 - 0.25]
    assert idx[M - 2].tolist() == [3, 0, 1]
    out = m.mamba_logits_constrain_fwd(logits, **rules, out=logits)
    assert out is logits and out[M - 1, [7, 8, wide - 1]].tolist() == [0.75, 6.0, 1.75] and out[M - 2, [3, 7, wide - 1]].tolist() == [3.0, -1.25, -0.75]
    del logits, out
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_rules_without_rows_are_refused_where_there_are_logits(m):
    logits, none = torch.zeros(2, 40, dtype=BF16, device=DEV), lambda *s, dtype=I32: torch.zeros(*s, dtype=dtype, device=DEV)
    for rule in (dict(mask=none(0, 2)), dict(counts=none(0, 40)), dict(penalties=none(0, 3, dtype=F32)),
                 dict(counts=none(0, 40), penalties=none(0, 3, dtype=F32))):
        with pytest.raises(ValueError, match="must have a row"):
            m.mamba_logits_constrain_fwd(logits, **rule)
        with pytest.raises(ValueError, match="must have a row"):
            m.mamba_topk_constrained_fwd(logits, 2, **rule)
        assert m.mamba_logits_constrain_fwd(logits[:0], **rule).shape == (0, 40)
        assert [tuple(x.shape) for x in m.mamba_topk_constrained_fwd(logits[:0], 2, **rule)[:2]] == [(0, 2), (0, 2)]


@pytest.mark.gpu
@pytest.mark.parametrize("S,L,V", [(1, 1, 1), (3, 17, 5), (2, 4097, 8193), (4, 8000, 50280), (1, 100000, 20000), (2, 0, 30)])
def test_token_counts(m, S, L, V):
    from oracle import constrain as oc
    print("\n[gpu-case] token counts S=%d L=%d V=%d" % (S, L, V), flush=True)
    rng = np.random.default_rng(L + V)
    tokens = (V * rng.random((S, L)) ** 3).astype(np.int32)
    tokens[rng.random((S, L)) < 0.1] = -1
    tokens[rng.random((S, L)) < 0.05] = V
    g = torch.from_numpy(tokens).to(DEV)
    want = oc.token_counts(tokens, V)
    counts = m.mamba_token_counts(g, V)
    assert np.array_equal(counts.cpu().numpy(), want)
    prompt = rng.integers(0, V, (S, 3)).astype(np.int32)
    want = oc.token_counts(tokens, V, oc.token_counts(prompt, V, want, prompt=True))
    assert m.mamba_token_counts(torch.from_numpy(prompt).to(DEV), V, counts=counts, prompt=True) is counts
    m.mamba_token_counts(g, V, counts=counts)
    assert np.array_equal(counts.cpu().numpy(), want)


@pytest.mark.gpu
def test_in_place_other_stream_and_replayed(m):
    """The run of a draft position: counts of the prefix, the children, constrained logits in place; on a side stream, and captured."""
    rng = np.random.default_rng(6)
    c = case(rng, 9, 50280, 3, 2, [0.5, 0.001], counts=False)
    tokens = torch.from_numpy(rng.integers(0, 50280, (3, 500)).astype(np.int32)).to(DEV)
    g = gpu(c)
    logits = g.pop("logits")
    counts = m.mamba_token_counts(tokens, 50280)
    ref = m.mamba_topk_constrained_fwd(logits, 3, counts=counts, **g, want_path=True)
    out = m.mamba_logits_constrain_fwd(logits, counts=counts, **g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = m.mamba_topk_constrained_fwd(logits, 3, counts=counts, **g, want_path=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    work, cbuf = logits.clone(), torch.empty_like(counts)
    bufs = [torch.empty_like(x) for x in ref]
    ws = torch.empty(m.mamba_topk_constrained_workspace_bytes(9, 50280, 3), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.mamba_topk_constrained_fwd(work, 3, counts=cbuf, **g, idx=bufs[0], val=bufs[1], path_out=bufs[2], workspace=ws)
        m.mamba_logits_constrain_fwd(work, counts=cbuf, **g, out=work)
    for _ in range(3):
        work.copy_(logits)
        cbuf.copy_(m.mamba_token_counts(tokens, 50280))
        for b in bufs:
            b.fill_(7)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, bufs)) and torch.equal(work, out)


def small_drafter(layers=2, V=1000, seed=0):
    """A drafter of the widths that the library's kernels take, random weights."""
    from paper_2506_01206_amd import binding as b
    from paper_2506_01206_amd.drafter import MambaDrafter
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s, std=0.05, dtype=BF16: (torch.randn(*s, generator=gen) * std).to(dtype).to(DEV)
    dm, d, N, r = 64, 128, 16, 8
    blocks = [b.Block(dict(norm_w=1 + n(dm, dtype=F32), in_proj_w=n(2 * d, dm, std=0.2), conv_w=n(d, 4, std=0.4, dtype=F32), conv_b=n(d, dtype=F32),
                           x_proj_w=n(r + 2 * N, d, std=0.2), dt_proj_w=n(d, r, std=0.2), dt_bias=n(d, dtype=F32) - 3, Dskip=1 + n(d, dtype=F32),
                           A=-torch.arange(1, N + 1, dtype=F32, device=DEV).repeat(d, 1).contiguous(), out_proj_w=n(dm, d, std=0.2))) for _ in range(layers)]
    return MambaDrafter(n(V, dm, std=1.0), blocks, 1 + n(dm, dtype=F32))


@pytest.mark.gpu
@pytest.mark.parametrize("use_graph", [False, True])
def test_drafter_under_rules(m, use_graph):
    """Draft trees whose every position chooses among the constrained logits of that position, eager and replayed, while the rules and the
    text go on; and without rules as before."""
    from oracle import constrain as oc
    print("\n[gpu-case] drafter under rules, graph=%s" % use_graph, flush=True)
    d = small_drafter()
    V, tree = d.V, (3, 2, 1, 2)
    rng = np.random.default_rng(8)
    prefix = torch.from_numpy(rng.integers(0, V, 40).astype(np.int32)).to(DEV)
    d.prefill(prefix)
    free = [t.clone() for t in d.draft(tree, use_graph)[0]]
    with pytest.raises(RuntimeError, match="constrain"):
        d.observe(prefix)
    with pytest.raises(ValueError, match="above zero"):
        d.constrain(repetition=0.0)
    bias = torch.from_numpy((rng.standard_normal(V) * (rng.random(V) < 0.05)).astype(np.float32)).to(DEV)
    allowed = np.stack([rng.random(V) < 0.5, np.arange(V) < 1, rng.random(V) < 0.9])   # one token for two children at the second position
    mask = torch.from_numpy(pack(allowed)).to(DEV)
    seen = []
    for repetition, presence, frequency, b, mk in ((1.3, 0.2, 0.1, bias, mask), (1.0, 0.0, 0.0, None, mask[2]), (1.2, 0.5, 0.3, bias, None)):
        d.constrain(repetition, presence, frequency, b, mk)
        d.prefill(prefix)
        counts = oc.token_counts(prefix.cpu().numpy()[None], V, prompt=True)
        for round_ in range(2):
            tokens, _ = d.draft(tree, use_graph)
            bufs = d._buffers(tree)
            path = None
            for i in range(1, len(tree) + 1):
                logits = (d.root_logits if i == 1 else bufs["pos"][i - 1]["logits"]).float().cpu().numpy()
                rule = None if mk is None else mk.cpu().numpy().reshape(-1, (V + 31) // 32)
                x, ok = oc.constrain(logits, counts, np.array([[repetition, presence, frequency]], np.float32), path=path,
                                     bias=None if b is None else b.cpu().numpy(), mask=None if rule is None else rule[min(i, len(rule)) - 1][None])
                ri, rv, path = oc.children(x, ok, tree[i - 1], path)
                assert np.array_equal(tokens[i - 1].cpu().numpy(), ri.reshape(-1)), i
                assert np.array_equal(bufs["pos"][i]["cand_val"].cpu().numpy(), rv) and np.array_equal(bufs["pos"][i]["path"].cpu().numpy(), path)
            seen.append([t.cpu().tolist() for t in tokens])
            more = torch.from_numpy(rng.integers(0, V, 5).astype(np.int32)).to(DEV)
            d.observe(more)
            counts = oc.token_counts(more.cpu().numpy()[None], V, counts)
    assert seen[0][1][0::2] == [0] * 3 and seen[0][1][1::2] == [-1] * 3       # the position that allows one token
    d.constrain(None)
    d.prefill(prefix)
    assert all(torch.equal(a, b) for a, b in zip(free, d.draft(tree, use_graph)[0]))
