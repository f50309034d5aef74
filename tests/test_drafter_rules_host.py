"""MambaDrafter.constrain and prefill without a GPU: what they refuse changes nothing.  The drafter's buffers are host tensors here, no kernel is called."""
import os
from types import SimpleNamespace

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
V, WORDS = 1000, 32


@pytest.fixture
def drafter():
    if not os.path.exists(os.path.join(ROOT, "paper_2506_01206_amd", "libmamba_hip.so")):
        from paper_2506_01206_amd import build
        build.build()
    from paper_2506_01206_amd.drafter import MambaDrafter
    block = SimpleNamespace(d_inner=128, d_state=16, d_conv=4)
    return MambaDrafter(torch.zeros(V, 64, dtype=torch.bfloat16), [block], torch.ones(64))


def mask(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype)


REFUSED = [dict(bias=torch.zeros(V - 1)), dict(bias=torch.zeros(1, V)), dict(mask=mask(WORDS - 1)), dict(mask=mask(2, WORDS + 1)),
           dict(mask=mask(0, WORDS)), dict(mask=mask(0)), dict(mask=mask(10 ** 3, WORDS)), dict(mask=mask(WORDS, dtype=torch.int64)),
           dict(mask=torch.zeros((), dtype=torch.int32)), dict(repetition=0.0), dict(repetition=-1.0), dict(repetition=float("nan")),
           dict(bias=torch.zeros(V), mask=mask(3))]


@pytest.mark.parametrize("bad", range(len(REFUSED)))
def test_a_refused_first_call_leaves_the_drafter_free(drafter, bad):
    with pytest.raises(ValueError):
        drafter.constrain(**REFUSED[bad])
    assert drafter._rules is None
    with pytest.raises(RuntimeError, match="constrain"):
        drafter.observe(torch.zeros(1, dtype=torch.int32))


@pytest.mark.parametrize("bad", range(len(REFUSED)))
def test_a_refused_later_call_leaves_the_rules_that_are_there(drafter, bad):
    drafter.constrain(1.5, 0.25, 0.125, torch.arange(V, dtype=torch.float32), torch.arange(2 * WORDS, dtype=torch.int32).view(2, WORDS))
    rules = drafter._rules
    kept = {n: [x.clone() for x in v] if isinstance(v, list) else v.clone() for n, v in rules.items()}
    with pytest.raises(ValueError):
        drafter.constrain(**REFUSED[bad])
    assert drafter._rules is rules
    for n, v in rules.items():
        assert all(torch.equal(a, b) for a, b in zip(v, kept[n])) if isinstance(v, list) else torch.equal(v, kept[n]), n


def test_rules_as_they_are_set(drafter):
    drafter.constrain()
    r = drafter._rules
    assert r["penalties"].tolist() == [[1.0, 0.0, 0.0]] and bool((r["bias"] == 0).all()) and all(bool((x == -1).all()) for x in r["masks"])
    drafter.constrain(2.0, 0.5, 0.25, torch.ones(V), torch.arange(2 * WORDS, dtype=torch.int32).view(2, WORDS))
    assert drafter._rules is r and r["penalties"].tolist() == [[2.0, 0.5, 0.25]] and bool((r["bias"] == 1).all())
    assert r["masks"][0][0, 0] == 0 and all(int(x[0, 0]) == WORDS for x in r["masks"][1:])
    drafter.constrain(mask=torch.arange(WORDS, dtype=torch.int32))
    assert all(torch.equal(x[0], torch.arange(WORDS, dtype=torch.int32)) for x in r["masks"]) and bool((r["bias"] == 0).all())
    drafter.constrain(None)
    assert drafter._rules is None


@pytest.mark.parametrize("prompt_len", [-1, 6, 10 ** 9])
def test_a_prompt_longer_than_the_prefix_is_refused(drafter, prompt_len):
    drafter.constrain()
    drafter._rules["counts"].fill_(3)
    with pytest.raises(ValueError, match="prompt_len"):
        drafter.prefill(torch.zeros(5, dtype=torch.int32), prompt_len=prompt_len)
    assert bool((drafter._rules["counts"] == 3).all())


def test_a_refused_prefix_leaves_the_counts(drafter):
    drafter.constrain()
    drafter._rules["counts"].fill_(3)
    with pytest.raises(ValueError, match="GPU"):
        drafter.prefill(torch.zeros(5, dtype=torch.int32))
    assert bool((drafter._rules["counts"] == 3).all())
