"""What a refused or failed call leaves of a drafter that draws its children."""
from types import SimpleNamespace

import pytest
import torch

from test_sampled_drafting import host_drafter, small_drafter  # noqa: F401 (a fixture)

DEV = "cuda:0"


def test_a_round_that_was_refused_or_failed_is_not_verified(host_drafter):  # noqa: F811
    d, tree = host_drafter, (2, 1)
    cache = SimpleNamespace(batch=[1, 2, 2], gamma=2, set_root=lambda conv, ssm: None)
    cand = lambda *s: dict(cand=torch.zeros(s, dtype=torch.int32), path=None)
    d._trees[tree] = dict(cache=cache, tree=tree, graph=None, constrained_graph=None, pos=[None, cand(1, 2), cand(2, 1)])   # (as after a greedy round)
    p = torch.zeros(5, 1000)
    d.sample(0.8)
    for u in (torch.rand(3), torch.rand(5)):
        with pytest.raises(ValueError, match="random numbers"):
            d.draft(tree, False, u=u)
        with pytest.raises(RuntimeError, match="drawn"):
            d.verify(tree, p)
    with pytest.raises(ValueError, match="GPU"):                 # (the round itself, which has none here)
        d.draft(tree, False)
    with pytest.raises(RuntimeError, match="drawn"):
        d.verify(tree, p)


@pytest.mark.gpu
@pytest.mark.parametrize("use_graph", [False, True])
def test_a_greedy_tree_stays_one_where_random_numbers_are_refused(use_graph):
    d, tree = small_drafter(layers=1), (2, 1)
    d.prefill(torch.arange(20, dtype=torch.int32, device=DEV))
    p = torch.full((5, d.V), 1.0 / d.V, device=DEV)
    d.sample(0.8)
    d.draft(tree, use_graph)
    d.verify(tree, p)
    d.sample(None)
    d.draft(tree, use_graph)
    d.sample(0.8)
    with pytest.raises(ValueError, match="random numbers"):
        d.draft(tree, use_graph, u=torch.rand(3, device=DEV))
    with pytest.raises(RuntimeError, match="drawn"):
        d.verify(tree, p)
    d.draft(tree, use_graph, u=torch.rand(4, device=DEV))
    ua, us = torch.rand(4, device=DEV), torch.rand(1, device=DEV)
    ref = d.verify(tree, p, ua, us)
    with pytest.raises(ValueError, match="random numbers"):      # (a drawn one too)
        d.draft(tree, use_graph, u=torch.rand(3, device=DEV))
    assert all(torch.equal(x, y) for x, y in zip(ref, d.verify(tree, p, ua, us)))
