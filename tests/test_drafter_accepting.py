"""A drafter under rules through several rounds of a serving loop: draft, accept, encode the prefix again with what was accepted.  Every
position of every round chooses as the oracle does whose counts know where the prompt ends (bit for bit, as in tests/test_constrained_children.py)."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from test_constrained_children import m, small_drafter  # noqa: F401  (m: the fixture)

PENALTIES = (1.3, 0.6, 0.4)


def check_round(d, tree, use_graph, counts):
    from oracle import constrain as oc
    tokens, _ = d.draft(tree, use_graph)
    bufs, path = d._buffers(tree), None
    for i in range(1, len(tree) + 1):
        logits = (d.root_logits if i == 1 else bufs["pos"][i - 1]["logits"]).float().cpu().numpy()
        x, ok = oc.constrain(logits, counts, np.array([PENALTIES], np.float32), path=path, bias=np.zeros(d.V, np.float32))
        ri, rv, path = oc.children(x, ok, tree[i - 1], path)
        assert np.array_equal(tokens[i - 1].cpu().numpy(), ri.reshape(-1)), i
        assert np.array_equal(bufs["pos"][i]["cand_val"].cpu().numpy(), rv) and np.array_equal(bufs["pos"][i]["path"].cpu().numpy(), path)
    return path


@pytest.mark.gpu
@pytest.mark.parametrize("use_graph", [False, True])
@pytest.mark.parametrize("n_prompt", [0, 1, 13, 40])
def test_accepted_tokens_stay_generated_when_the_prefix_is_encoded_again(m, n_prompt, use_graph):  # noqa: F811
    from oracle import constrain as oc
    print("\n[gpu-case] drafter under rules, accepted tokens behind a prompt of %d, graph=%s" % (n_prompt, use_graph), flush=True)
    d, tree = small_drafter(), (3, 2, 2)
    rng = np.random.default_rng(n_prompt)
    prompt = rng.integers(0, d.V, n_prompt).astype(np.int32)
    text = np.concatenate([prompt, rng.integers(0, d.V, 3).astype(np.int32)])   # three tokens are there already
    d.constrain(*PENALTIES)
    for _ in range(4):
        d.prefill(torch.from_numpy(text).to(DEV), prompt_len=n_prompt)
        counts = oc.token_counts(text[None, n_prompt:], d.V, oc.token_counts(prompt[None], d.V, prompt=True))
        assert np.array_equal(d._rules["counts"].cpu().numpy(), counts)
        path = check_round(d, tree, use_graph, counts)
        # one more is generated behind this prefix and seen before the prefix is encoded again
        more = rng.integers(0, d.V, 1).astype(np.int32)
        d.observe(torch.from_numpy(more).to(DEV))
        check_round(d, tree, use_graph, oc.token_counts(more[None], d.V, counts))
        text = np.concatenate([text, path[rng.integers(0, len(path))], more])
    d.prefill(torch.from_numpy(text).to(DEV))                    # all of it as the prompt
    assert np.array_equal(d._rules["counts"].cpu().numpy(), oc.token_counts(text[None], d.V, prompt=True))


@pytest.mark.gpu
def test_a_row_of_a_rounds_paths_is_observed(m):  # noqa: F811
    """Rows of three tokens start anywhere; a column has strides."""
    from oracle import constrain as oc
    print("\n[gpu-case] drafter observes rows and columns of its paths", flush=True)
    d, tree = small_drafter(), (3, 2, 2)
    d.constrain(*PENALTIES)
    d.prefill(torch.arange(20, dtype=torch.int32, device=DEV))
    d.draft(tree, use_graph=False)
    path = d._buffers(tree)["pos"][3]["path"]
    counts = d._rules["counts"].cpu().numpy()
    for tokens in (path[1], path[2, 1:], path[:, 1], path[5:7], path[0, :0]):
        d.observe(tokens)
        counts = oc.token_counts(tokens.cpu().numpy().reshape(1, -1), d.V, counts)
        assert np.array_equal(d._rules["counts"].cpu().numpy(), counts)
