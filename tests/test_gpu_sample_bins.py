"""lvspec_sample with logits on the border between two bins of its histogram: counted in one and looked for in the other, they would
put a top-k boundary off by a token.  Against the fp64 form of test_gpu_sample_filters."""
import numpy as np
import pytest

from test_gpu_sample_filters import check, ctx                                  # noqa: F401

pytestmark = pytest.mark.gpu


def on_a_border(T, wanted):
    """Distances d from the largest logit for which d times the bins per unit of logit, rounded to fp32, is k + 1/2 although
    it is not exactly: rounded to a bin in one step it falls to one side, in two steps to the even one.  (d, k, exact bin) for `wanted`
    values of k from 40 on."""
    per = np.float32(np.float32(64) / np.float32(T))
    got = []
    for k in range(40, 2000):
        d = np.float32((k + 0.5) / float(per))
        for step in range(-3, 4):
            x = d
            for _ in range(abs(step)):
                x = np.nextafter(x, np.float32(np.inf if step > 0 else 0))
            exact = float(x) * float(per)                   # (24 + 24 bits: exact in fp64)
            if np.float32(x * per) == np.float32(k + 0.5) and exact != k + 0.5:
                once, twice = (k + 1 if exact > k + 0.5 else k), (k if k % 2 == 0 else k + 1)
                if once != twice:
                    got.append((float(x), k, once))
                    break
        if len(got) == wanted:
            break
    return got


@pytest.mark.parametrize("T", [0.7, 0.9, 1.1, 1.3])
def test_a_logit_between_two_bins(ctx, T):                                       # noqa: F811
    """0 at the top, some tokens above the border, one on it, some below: top-k ends among those below."""
    T = np.float32(T)
    per = float(np.float32(np.float32(64) / T))
    borders = on_a_border(T, 32)
    assert len(borders) == 32
    vocab = 5000
    logits = np.full((2 * len(borders), vocab), -60.0, np.float32)
    k = []
    rng = np.random.default_rng(31)
    for i, (d, b, _) in enumerate(borders):
        for side, row in enumerate(logits[2 * i:2 * i + 2]):
            at = rng.permutation(vocab)
            row[at[0]], row[at[1]] = 0.0, -d
            row[at[2:12]] = -(b - 3 - np.arange(10)) / per                      # well inside bins above
            row[at[12:32]] = -(b + 1 - 0.3 + 0.03 * np.arange(20)) / per         # in bin b + 1
            row[at[32:52]] = -(b - 0.3 + 0.03 * np.arange(20)) / per             # in bin b
            # ends among the tokens of bin b (side 0), or of bin b + 1
            k.append(11 + 7 if side == 0 else 11 + 20 + 1 + 7)
    check(ctx, rng, logits, np.full(len(k), T), k, np.ones(len(k)))
