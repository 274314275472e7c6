"""lvspec_sample where top-k and top-p meet: boundaries in bins with more tokens than are ranked at once, low and high temperatures,
batches whose other rows leave larger candidates behind.  Against a plain fp64 form of its own.

top_p lies midway between two running sums of the row's order, so that which tokens are kept is beyond question (the sums are
good to 2^-21 of the whole, the tokens at the border have more), and u at least 1e-5 of the whole inside a token's
interval.  A probability is then good to 2^-20: a weight of 1e-5 of the whole or more is off by 2^-22 of itself and, being rounded to 2^-40 of
the largest, by 2^-24; the sum of what is kept likewise.  One token more or less in it shows where it has 1e-6 of the whole."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2604_05650_b200 import binding
    c = binding.Context(0)
    yield c
    c.close()


class Row:
    """A row's tokens in the order of falling logits, their weights and running sums in fp64."""

    def __init__(self, logits, T, top_k):
        l = np.asarray(logits, np.float64)
        self.order = np.lexsort((np.arange(len(l)), -l))
        if 0 < top_k < len(l):
            self.order = self.order[:top_k]
        self.l = l[self.order]
        self.w = np.exp((self.l - self.l[0]) / T)
        self.sums = np.cumsum(self.w)

    def clear_p(self, p):
        """The value between two running sums nearest above p, and how far (as a share) it is from either."""
        shares = self.sums / self.sums[-1]
        i = min(int(np.searchsorted(shares, p)), len(shares) - 1)
        below = shares[i - 1] if i else 0.0
        return float(np.float32((shares[i] + below) / 2)), (shares[i] - below) / 2

    def kept(self, p, least=-np.inf):
        n = len(self.order) if p >= 1 else int(np.searchsorted(self.sums, p * self.sums[-1])) + 1
        n = min(n, int((self.l >= least).sum()))
        by_index = np.argsort(self.order[:n])
        return self.order[:n][by_index], self.w[:n][by_index]


def clear_u(rng, tokens, weights):
    """u in the middle of the interval of one of the likelier tokens; the token and its probability."""
    share = weights / weights.sum()
    likely = np.flatnonzero(share >= min(2.1e-5, share.max()))
    i = int(rng.choice(likely, p=share[likely] / share[likely].sum()))
    u = float(np.float32(share[:i].sum() + share[i] / 2))
    return u, int(tokens[i]), float(share[i])


def run(ctx, logits, T, k, p, u, bf16=False):
    import torch
    rows, vocab = logits.shape
    x = torch.from_numpy(np.ascontiguousarray(logits, dtype=np.float32)).cuda()
    x = x.bfloat16() if bf16 else x
    f = lambda a: torch.tensor(np.asarray(a, np.float32)).cuda()                                           # noqa: E731
    tokens, probs = torch.full((rows,), -9, dtype=torch.int32, device="cuda"), torch.full((rows,), -9.0, device="cuda")
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    ctx.sample(rows, vocab, x, f(T), torch.tensor(np.asarray(k, np.int32)).cuda(), f(p), None, f(u), tokens, probs, bf16=bf16)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    return tokens.cpu().numpy(), probs.cpu().numpy()


def check(ctx, rng, logits, T, k, p_near, bf16=False, reference=None):
    """`reference`: the rows whose results are compared (all)."""
    rows = len(logits)
    reference = range(rows) if reference is None else reference
    seen = logits
    if bf16:
        import torch
        seen = torch.from_numpy(np.asarray(logits, np.float32)).bfloat16().float().numpy()
    p, u, want = np.asarray(p_near, np.float64).copy(), rng.random(rows), {}
    for r in reference:
        row = Row(seen[r], float(np.float32(T[r])), int(k[r]))
        if p[r] < 1:
            p[r], far = row.clear_p(p[r])
            assert far > 2.0 ** -20
        u[r], *want[r] = clear_u(rng, *row.kept(p[r]))
    tokens, probs = run(ctx, logits, T, k, p, u, bf16)
    wrong = [(r, float(T[r]), int(k[r]), float(p[r]), int(tokens[r]), want[r][0], float(probs[r]), want[r][1]) for r in reference
             if tokens[r] != want[r][0] or not abs(probs[r] - want[r][1]) <= want[r][1] * 2.0 ** -20]
    assert not wrong, (len(wrong), wrong[:4])
    return tokens, probs, p, u


def plateau(vocab, rng):
    """One token above 900 equal ones above 1300 a little lower ones, all of the latter two in one bin, the rest far below."""
    row = np.full(vocab, -60.0, np.float32)
    at = rng.permutation(vocab)[:2201]
    row[at[0]], row[at[1:901]], row[at[901:]] = 9.0, 2.005, 2.0
    return row


def steps(vocab, rng):
    """20 tokens 1e-4 apart, then 8172 from 0.01 below on, 1e-6 apart."""
    row = np.full(vocab, -60.0, np.float32)
    at = rng.permutation(vocab)[:8192]
    row[at[:20]] = 5.0 - 1e-4 * np.arange(20)
    row[at[20:]] = 5.0 - 0.01 - 1e-6 * np.arange(8172)
    return row


def test_a_boundary_among_thousands(ctx):
    """The k-th token's bin is cut by bit patterns; top-p's boundary then is somewhere else altogether."""
    rng = np.random.default_rng(21)
    vocab = 152064
    normal = [(rng.standard_normal(vocab) * s).astype(np.float32) for s in (1, 1, 0.3, 0.3)]
    for x in normal:        # (kept apart from their neighbours: borders that are clear)
        top = np.argsort(x)[-400:]
        x[top] += np.arange(400) * 1e-5
    logits = np.stack([plateau(vocab, rng), steps(vocab, rng), *normal, plateau(vocab, rng), steps(vocab, rng)])
    T = np.asarray([1, 1, 50, 1.5, 1, 1, 1, 1], np.float32)
    k = [2100, 4000, 2000, 40000, 10000, 10000, 2100, 8000]
    check(ctx, rng, logits, T, k, [0.3, 0.001, 0.002, 0.0036, 0.0019, 0.3, 0.9, 0.0015])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab,rows,T", [(152064, 128, 0.1), (152064, 128, 0.05), (152064, 24, 0.3), (33000, 160, 0.15), (9000, 400, 0.1),
                                          (4000, 300, 0.2)])
def test_low_temperature(ctx, vocab, rows, T, bf16):
    """Most of a row is in the last bin, and the k-th token often too.  Every third row leaves candidates behind that are larger than any
    of the others'."""
    rng = np.random.default_rng(vocab + rows)
    import torch
    logits = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(rows)).numpy() * np.float32(3)
    logits[np.arange(rows), rng.integers(0, vocab, rows)] += 9
    logits[2::3] += np.float32(40)
    logits[2::3] /= 8
    T = np.full(rows, T, np.float32)
    T[2::3] *= 0.2
    k = rng.choice([50, 100, 1000, min(vocab - 1, 5000), min(vocab - 1, 40000)], rows)
    k[2::3] = 0
    p = np.exp(rng.uniform(np.log(0.002), np.log(0.99), rows))
    p[::4] = rng.uniform(0.3, 0.99, len(p[::4]))
    # rows whose border would not be clear go without top-p
    seen = torch.from_numpy(logits).bfloat16().float().numpy() if bf16 else logits
    for r in range(rows):
        if Row(seen[r], float(T[r]), int(k[r])).clear_p(p[r])[1] <= 2.0 ** -19:
            p[r] = 1.0
    assert (p < 1).sum() > rows // 2
    tokens, probs, p, u = check(ctx, rng, logits, T, k, p, bf16)
    # a row's result is its own
    for r in rng.choice(rows, 6, replace=False):
        t, pr = run(ctx, logits[r:r + 1], T[r:r + 1], k[r:r + 1], p[r:r + 1], u[r:r + 1], bf16)
        assert t[0] == tokens[r] and pr[0] == probs[r]


@pytest.mark.parametrize("sigma,T", [(1.0, 50.0), (0.3, 1.0), (0.02, 1.0), (3.0, 1.5), (1.0, 2000.0)])
def test_many_kept(ctx, sigma, T):
    """Thousands of tokens kept by top-k, a small or large share of them by top-p."""
    rng = np.random.default_rng(int(T * 10 + sigma * 1000))
    rows, vocab = 40, 50000
    logits = (rng.standard_normal((rows, vocab)) * sigma).astype(np.float32)
    k = rng.choice([1100, 2000, 10000, 40000, 0], rows)
    p = np.exp(rng.uniform(np.log(0.002), np.log(0.9), rows))
    T = np.full(rows, T, np.float32)
    for r in range(rows):
        if Row(logits[r], float(T[r]), int(k[r])).clear_p(p[r])[1] <= 2.0 ** -19:
            p[r] = 1.0
    assert (p < 1).sum() > rows // 2
    check(ctx, rng, logits, T, k, p)


@pytest.mark.parametrize("rows,vocab", [(61, 32800), (512, 33000), (600, 33000), (12, 400000), (38, 40001)])
def test_large_batches(ctx, rows, vocab):
    """All filters in batches of more rows than run at once, every organisation of the clusters."""
    import torch
    rng = np.random.default_rng(rows)
    logits = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(rows)).numpy() * np.float32(3)
    T = rng.choice([0.1, 0.3, 0.7, 1.0, 1.3], rows).astype(np.float32)
    k = rng.choice([0, 0, 40, 3000, 20000], rows)
    p = rng.choice([0.05, 0.5, 0.9, 0.97, 1.0], rows)
    compared = sorted(rng.choice(rows, min(rows, 48), replace=False))
    for r in range(rows):
        if r in compared and p[r] < 1 and Row(logits[r], float(T[r]), int(k[r])).clear_p(p[r])[1] <= 2.0 ** -19:
            p[r] = 1.0
    check(ctx, rng, logits, T, k, p, reference=compared)
