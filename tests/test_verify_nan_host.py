"""sd_verify where probabilities are NaN: such a token is rejected."""
import numpy as np
import pytest

from oracle import tree_search as oracle

NAN = float("nan")
FINE = [0.5, 0.25, 0.25]
# rows of p, q, token, u -> the emitted tokens (None: nothing to draw from)
CASES = [([[0.5, NAN, 0.5], FINE], [FINE], 1, 0.0, [2]), ([[0.5, NAN, 0.5], FINE], [FINE], 0, 0.0, [0, 0]),
         ([FINE, FINE], [[0.25, NAN, 0.25]], 1, 0.0, [0]), ([FINE, FINE], [FINE], 1, NAN, [0]), ([[NAN] * 3, FINE], [FINE], 0, 0.0, None)]


@pytest.mark.parametrize("p,q,token,u,emitted", CASES)
def test_rejected(p, q, token, u, emitted):
    from paper_2506_01206_amd import tree_search
    from paper_2506_01206_amd.binding import MambaError
    args = [np.array(a, np.float32) for a in (p, q)] + [np.array([token], np.int32), np.array([u], np.float32), 0.25]
    if emitted is None:
        with pytest.raises(MambaError):
            tree_search.sd_verify(*args, greedy=False)
        return
    assert list(tree_search.sd_verify(*args, greedy=False)) == emitted
    assert oracle.verify(*args, False) == emitted
