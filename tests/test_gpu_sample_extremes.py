"""lvspec_sample at the ends of what the temperature, min-p and the logits may be: a token and its probability are always written, and
are those of the formula in fp64 (a probability to 2^-20, u in the middle of a token's interval: as in test_gpu_sample_filters)."""
import numpy as np
import pytest

from test_gpu_sample_filters import ctx                                         # noqa: F401

pytestmark = pytest.mark.gpu
INF = float("inf")


def expected(rng, logits, T, k, p, m):
    """(u, token, probability) of one of the row's kept tokens."""
    l = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    order = np.lexsort((np.arange(len(l)), -l))
    with np.errstate(invalid="ignore"):
        w = np.where(l == l.max(), 1.0, np.exp((l - l.max()) / float(T)))
    w[l == -np.inf] = 0
    kept = order[:k] if 0 < k < len(l) else order
    kept = kept[w[kept] > 0] if T == INF else kept
    if p < 1:
        sums = np.cumsum(w[kept])
        kept = kept[:int(np.searchsorted(sums, p * sums[-1])) + 1]
    if m > 0:
        least = l.max() if m >= 1 else l.max() + float(T) * np.log(float(m))
        kept = kept[l[kept] >= least]
    kept = np.sort(kept)
    share = w[kept] / w[kept].sum()
    i = int(rng.choice(len(kept), p=share))
    return float(np.float32(share[:i].sum() + share[i] / 2)), int(kept[i]), float(share[i])


@pytest.mark.parametrize("vocab", [5, 700, 9000, 40000])
def test_extremes(ctx, vocab):                                                  # noqa: F811
    import torch
    rng = np.random.default_rng(vocab)
    base = rng.standard_normal(vocab).astype(np.float32)
    twice = base.copy()
    twice[vocab // 2] = twice[1] = base.max() + 1
    holes = base.copy()
    holes[::3] = -np.inf
    wide = (base.astype(np.float64) * 1e38).clip(-3.3e38, 3.3e38)
    ends = np.where(rng.random(vocab) < 0.5, np.float32(3.4e38), np.float32(-3.4e38))
    infinite = base.copy()
    infinite[[0, vocab - 1]] = np.inf
    rows = []
    for T in (1e-45, 1e-42, 1e-40, 4.2e-39, 1e-38, 1e-30, 1e-20):
        rows += [(base, T, 0, 1, 0), (twice, T, 0, 1, 0), (twice, T, 3, 0.9, 0), (twice, T, 0, 0.3, 0.5), (twice, T, 0, 1, 1),
                 (holes, T, 2, 1, 0.1), (infinite, T, 0, 1, 0), (base * 0, T, 0, 1, 0), (ends, T, 0, 0.4999, 0)]
    for T in (INF, 3e38, 1e31):
        rows += [(holes, T, 0, 1, 0), (base, T, 0, 1, 1), (twice, T, 0, 1, 1), (twice, T, 0, 1, 2), (base, T, 4, 1, 0), (holes, T, 3, 1, 1),
                 (base, T, 0, 1, 0.5), (holes, T, 0, 0.5001, 0), (base, T, 4, 0.6, 0.5), (wide, T, 0, 1, 0), (ends, T, 0, 1, 0)]
    for T in (1e29, 1e36, 1e38):
        rows += [(wide, T, 0, 1, 0), (wide, T, 3, 1, 0), (wide, T, 0, 1, 0.3)]
    logits = np.stack([r[0] for r in rows]).astype(np.float32)
    T, k, p, m = (np.asarray([r[i] for r in rows], np.float32 if i != 2 else np.int32) for i in range(1, 5))
    assert T[0] > 0                                                             # (a denormal number, not zero)
    want = [expected(rng, logits[r], T[r], int(k[r]), float(p[r]), float(m[r])) for r in range(len(rows))]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()            # noqa: E731
    u = dev(np.asarray([w[0] for w in want], np.float32))
    tokens, probs = torch.full((len(rows),), -9, dtype=torch.int32, device="cuda"), torch.full((len(rows),), -9.0, device="cuda")
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    ctx.sample(len(rows), vocab, dev(logits), dev(T), dev(k), dev(p), dev(m), u, tokens, probs)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    for r, (_, token, prob) in enumerate(want):
        assert (int(tokens[r]), r) == (token, r) and abs(float(probs[r]) - prob) <= prob * 2.0 ** -20, (rows[r][1:], float(probs[r]), prob)
