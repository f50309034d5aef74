"""Verification of drafted trees where probabilities are NaN: such a child is rejected, by the oracle's definition and by the kernel."""
import numpy as np
import pytest

from oracle import sampling as oracle
from test_tree_verify import check, some_trees

NAN = float("nan")


@pytest.fixture(scope="module")
def m():
    from paper_2506_01206_amd import binding
    return binding


def one(p, q, tokens, u_accept, u_sample, tree):
    out, count, node = oracle.verify(np.array([p], np.float32), np.array([q], np.float32), np.array([tokens]), np.array([u_accept], np.float32),
                                     np.array([u_sample], np.float32), tree)
    return out[0].tolist(), int(count[0]), node[0].tolist()


def test_oracle_by_hand():
    fine, leaf = [0.5, 0.25, 0.25], [1.0, 0.0, 0.0]
    # nothing is known of the target: no child, and no token
    assert one([[NAN] * 3, leaf], [fine], [0], [0.0], 0.5, (1,)) == ([-1, -1], 1, [-1])
    # of one token: a child that is another one, that one itself; what is drawn is drawn from what the target is ahead of the drafter, or not at all
    assert one([[0.5, NAN, 0.5], leaf], [fine], [0], [0.0], 0.5, (1,)) == ([0, 0], 2, [0])
    assert one([[0.5, NAN, 0.5], leaf], [fine], [1], [0.0], 0.5, (1,)) == ([2, -1], 1, [-1])
    assert one([[0.25, NAN, 0.25], leaf], [fine], [1], [0.0], 0.5, (1,)) == ([-1, -1], 1, [-1])
    # the drafter's: no child, and no part in what is drawn
    assert one([fine, leaf], [[0.25, NAN, 0.25]], [1], [0.0], 0.5, (1,)) == ([0, -1], 1, [-1])
    assert one([fine, leaf], [[NAN] * 3], [1], [0.0], 0.5, (1,)) == ([1, -1], 1, [-1])
    # the random number
    assert one([fine, leaf], [fine], [1], [NAN], 0.5, (1,)) == ([1, -1], 1, [-1])


@pytest.mark.gpu
@pytest.mark.parametrize("tree", [(1,), (3,), (1, 1, 1), (3, 2, 2), (8, 8)], ids=str)
@pytest.mark.parametrize("V", [3, 500, 9000])
def test_against_oracle(m, tree, V):
    rng = np.random.default_rng(V + len(tree))
    S = 8 if V < 9000 else 3
    for noise in (0.5, 2.0):
        c = some_trees(rng, S, V, tree, noise)
        for name in ("p", "q"):
            rows = c[name].copy()
            rows[rng.uniform(size=rows.shape[:2]) < 0.3] = NAN       # all of a node's
            check(m, {**c, name: rows})
            for share in (0.001, 0.2):
                some = c[name].copy()
                some[rng.uniform(size=some.shape) < share] = NAN
                check(m, {**c, name: some})
        u = c["u_accept"].copy()
        u[rng.uniform(size=u.shape) < 0.3] = NAN
        check(m, {**c, "u_accept": u})


@pytest.mark.gpu
def test_children_that_are_nan(m):
    """Every drawn child's own probability: all are rejected, wherever they would have been accepted with certainty."""
    rng = np.random.default_rng(5)
    tree = (2, 2)
    for name in ("p", "q"):
        c = some_trees(rng, 12, 300, tree, 0.3)
        rows, node, child = oracle.tree_rows(tree), 0, 0
        for r, n in zip(rows, tree):
            for _ in range(r):
                for s in range(12):
                    c[name][s, node, c["tokens"][s, child:child + n]] = NAN
                node, child = node + 1, child + n
        _, count, _ = check(m, {**c, "u_accept": np.zeros_like(c["u_accept"])})
        assert (count == 1).all()
