"""Drawn children where a unit of logits is millions of bins (low temperatures, large logits): cuts between neighbouring numbers."""
import os
import re

import numpy as np
import pytest

from test_sampling import check

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def m():
    from paper_2506_01206_amd import binding
    return binding


def test_differences_of_marks_are_integers():
    """A row's first mark, rounded up to a whole octave of eight, and its last one are as far apart as an int holds, and the bins behind them."""
    with open(os.path.join(ROOT, "paper_2506_01206_amd", "csrc", "sample.hip")) as f:
        (end,) = re.findall(r"constexpr float kEndMark = 0x1p(\d+)f;", f.read())
    assert 2 * 2 ** int(end) + 8 + 8 * 128 <= 2 ** 31 - 1


# top_p, min_p, top_k: each filter alone, and together
FILTERS = ([(1.0, 0.0, k) for k in (1, 2, 3, 5, 7, 8, 9, 20)] + [(p, 0.0, 0) for p in (0.25, 0.5, 0.7, 0.9)] + [(1.0, q, 0) for q in (0.05, 0.3, 0.8)]
           + [(0.5, 0.0, 8), (0.7, 0.05, 0), (1.0, 0.1, 5), (0.9, 0.02, 9), (1.0, 0.0, 0)])


def neighbours(rng, top, V, span):
    """V float32 numbers from the largest down, some last bits apart, in no order: each once (span None), or of `span` values."""
    steps = np.arange(V) if span is None else rng.integers(0, span, V)
    ulp = np.spacing(np.float32(abs(top) / 2)).astype(np.float64)  # (of the smaller power of two: multiples of it are numbers on both sides)
    step = max(ulp, float(np.spacing(np.float32(abs(top)))))
    x = top - step * steps
    assert np.array_equal(x, x.astype(np.float32))
    return rng.permutation(x)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1e-4, 2e-5, 1e-5, 5e-6, 2e-6, 1e-6])
def test_neighbouring_numbers_at_low_temperatures(m, T):
    rng = np.random.default_rng(round(-np.log10(T) * 100))
    tops = (14.625, 15.0, 19.5, 20.0, 29.125, 30.0, -15.0, -20.0)
    x = np.stack([neighbours(rng, top, 64, None) for top in tops])
    ties = np.stack([neighbours(rng, top, 3001, 61) for top in tops])
    for top_p, min_p, top_k in FILTERS:
        check(m, x, rng.uniform(size=(len(x), 4)), [[T, top_p, min_p]], [top_k])
        check(m, ties, rng.uniform(size=(len(x), 2)), [[T, top_p, min_p]], [top_k])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [2e-5, 1e-5, 5e-6, 2e-6])
def test_bfloat16_rows_at_low_temperatures(m, T):
    """Neighbouring bfloat16 numbers are thousands of nats apart there: what is left is the largest, tied or not."""
    rng = np.random.default_rng(round(-np.log10(T) * 100))
    x = np.repeat(np.arange(8.0, 32.0, 0.125), 2)[:, None] - np.array([0.0, 0.25, 1.0, 5.0, 5.0, 0.0])
    x[::2, 5] = 0.0                                                  # the largest once, and twice
    x = np.concatenate([x, -x[:, ::-1]])
    for top_p, min_p, top_k in ((1.0, 0.0, 1), (1.0, 0.0, 2), (0.5, 0.0, 0), (0.9, 0.0, 0), (1.0, 0.5, 0), (0.5, 0.1, 2), (1.0, 0.0, 0)):
        check(m, x, rng.uniform(size=(len(x), 3)), [[T, top_p, min_p]], [top_k], bf16=True)


@pytest.mark.gpu
@pytest.mark.parametrize("top", [1.5e6, 3e6, 1e7, 3e7, 4.6e7, 1e9, -3e6, -1e7, -4.65e7])
def test_large_logits(m, top):
    """Logits of which a unit is the last bit, or several: also for the first of the largest (temperature 0)."""
    rng = np.random.default_rng(int(abs(top)))
    top = float(np.float32(top))
    x = np.stack([neighbours(rng, top, 64, None), neighbours(rng, top, 64, 9)])
    ties = np.stack([neighbours(rng, top, 3001, 61), neighbours(rng, top, 3001, 3)])
    for T in (0.0, 0.25, 1.0, 4.0):
        for top_p, min_p, top_k in FILTERS:
            check(m, x, rng.uniform(size=(2, 4)), [[T, top_p, min_p]], [top_k])
            check(m, ties, rng.uniform(size=(2, 2)), [[T, top_p, min_p]], [top_k])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1.0, 1e-20, 1e-38])
def test_rows_from_one_end_of_the_marks_to_the_other(m, T):
    rng = np.random.default_rng(17)
    x = rng.standard_normal((6, 5003))
    x[0, [3, 5000]] = np.inf
    x[0, 7::50] = -3e38
    x[1, 4] = 3e38
    x[1, 5::3] = -3e38
    x[2] = -np.abs(x[2])                                             # all of them at the lower end, beside what does not count
    x[2, ::2] = -np.inf
    x[3, 1::2] = -np.inf
    x[3, ::2] = -3e38
    x[4] = 3e38
    x[4, 100:] = -np.inf
    x[5, :4000] = np.nan
    x[5, 4000:] = -4.65e7
    x = x.astype(np.float32)
    for top_p, min_p, top_k in FILTERS + [(1.0, 0.0, 4999), (1.0, 0.0, 2501), (1.0, 0.0, 2502), (1.0, 1.0, 3000)]:
        check(m, x, rng.uniform(size=(6, 3)), [[T, top_p, min_p]], [top_k])
