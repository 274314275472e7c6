"""lvspec_sample against the fp64 reference: the same token, and its probability to 2^-20 (2^x to 2^-22,
the rest carried, summed over what is kept).

Tokens are compared where u is at least 1e-5 of the whole away from the border between two tokens' intervals: borders are sums
of weights good to 2^-21, so they are off by 5e-7 at most (and by much less: the errors have either sign).  Filters are compared
where their own borders are as clear: top_p values between two running sums."""
import numpy as np
import pytest

from oracle import paged_step as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2604_05650_b200 import binding
    c = binding.Context(0)
    yield c
    c.close()


def run(ctx, logits, T, k, p, m, u, bf16=False, stride=None, offset=0, probs=True):
    import torch
    rows, vocab = logits.shape
    stride = stride or vocab
    t = torch.full((offset + rows * stride,), 99.0)
    for r in range(rows):
        t[offset + r * stride:offset + r * stride + vocab] = torch.from_numpy(np.asarray(logits[r], np.float32))
    t = (t.bfloat16() if bf16 else t).cuda()[offset:]
    dev = lambda a, dt: None if a is None else torch.tensor(np.asarray(a), dtype=dt).cuda()   # noqa: E731
    tokens = torch.full((rows,), -9, dtype=torch.int32, device="cuda")
    pr = torch.full((rows,), -9.0, device="cuda") if probs else None
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    ctx.sample(rows, vocab, t, dev(T, torch.float32), dev(k, torch.int32), dev(p, torch.float32), dev(m, torch.float32),
               dev(u, torch.float32), tokens, pr, bf16=bf16, row_stride=stride)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), pr.cpu().numpy() if probs else None


def f32(a):
    return np.asarray(a, np.float32).astype(np.float64)


def clear_p(rng, row, T, k):
    """A top_p in the middle between two running sums of the row's order."""
    kept, w = ref.kept_tokens(row, T, k, 1.0, 0.0)
    c = np.cumsum(w[kept]) / w[kept].sum()
    c = c[:max(1, np.searchsorted(c, 0.999))]
    i = rng.integers(len(c))
    return float(np.float32((c[i] + (c[i - 1] if i else 0)) / 2))


def check(ctx, rng, logits, T, k, p, m, **kw):
    rows = len(logits)
    exact = logits
    if kw.get("bf16"):
        import torch
        exact = torch.from_numpy(np.asarray(logits, np.float32)).bfloat16().double().numpy()
    # u: in the middle of a token's interval, or anywhere that is clear
    u = []
    for r in range(rows):
        while True:
            x = float(np.float32(rng.random()))
            if ref.sample(exact[r], T[r], k[r], p[r], m[r], x)[2] > 1e-5:
                break
        u.append(x)
    tokens, probs = run(ctx, logits, T, k, p, m, u, **kw)
    for r in range(rows):
        token, prob, _ = ref.sample(exact[r], T[r], k[r], p[r], m[r], u[r])
        assert tokens[r] == token, (r, T[r], k[r], p[r], m[r], u[r])
        assert abs(probs[r] - prob) <= prob * 2.0 ** -20
    return tokens, u


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("vocab,sigma", [(1, 1.0), (2, 1.0), (33, 3.0), (1000, 3.0), (4096, 1.0), (4097, 3.0), (20001, 3.0),
                                         (50257, 0.2), (152064, 3.0)])
def test_filters(ctx, vocab, sigma, bf16):
    rng = np.random.default_rng(vocab)
    rows = 9 if vocab < 30000 else 5
    logits = f32(rng.standard_normal((rows, vocab)) * sigma)
    T = f32(rng.uniform(0.4, 1.5, rows))
    k = np.asarray([0, 1, 7, 50, 0, 0, 200, vocab, 3][:rows])
    import torch
    seen = torch.from_numpy(logits.astype(np.float32)).bfloat16().double().numpy() if bf16 else logits
    p = np.asarray([1.0 if r in (1, 2) else clear_p(rng, seen[r], T[r], int(k[r])) for r in range(rows)])
    m = f32([0, 0, 0.05, 0, 0, 0.1, 0, 0, 0][:rows])
    check(ctx, rng, logits, T, k, p, m, bf16=bf16)
    check(ctx, rng, logits, T, k * 0, p * 0 + 1, m * 0, bf16=bf16)              # plain sampling


@pytest.mark.parametrize("bf16", [False, True])
def test_strides_and_alignment(ctx, bf16):
    rng = np.random.default_rng(8)
    for vocab, stride, offset in ((999, 1003, 1), (4099, 4100, 3), (9000, 9001, 0), (17, 17, 5)):
        logits = f32(rng.standard_normal((6, vocab)) * 2)
        check(ctx, rng, logits, f32([0.7] * 6), [0, 5, 0, 0, 9, 2], [1.0] * 6, f32([0, 0, 0.02, 0, 0, 0]), bf16=bf16, stride=stride,
              offset=offset)


def test_many_equal_logits(ctx):
    """Bins with more tokens than are ranked at once: all logits the same; few values; a plateau at the boundary."""
    rng = np.random.default_rng(9)
    vocab = 30000
    flat = np.zeros(vocab)
    few = f32(rng.integers(0, 4, vocab) * 1.5)
    plateau = f32(np.where(rng.random(vocab) < 0.5, 2.0, rng.standard_normal(vocab)))
    plateau[777], plateau[20000] = 9.0, 8.5
    close = f32(5.0 + rng.standard_normal(vocab) * 1e-6)            # within one bin, thousands of values
    logits = np.stack([flat, flat, few, few, plateau, plateau, close, close, close, flat])
    k = [500, 0, 3000, 0, 4000, 0, 1500, 0, 2000, 25000]
    p = [1.0, 0.123456, 1.0, 0.4000123, 1.0, 0.7000123, 1.0, 0.30001, 0.5000123, 0.5000123]
    check(ctx, rng, logits, f32([1.0] * 10), k, f32(p), f32([0] * 10))


def test_special_rows(ctx):
    from paper_2604_05650_b200 import binding
    rng = np.random.default_rng(10)
    vocab = 9000
    base = f32(rng.standard_normal((12, vocab)))
    base[0, :] = -np.inf
    base[1, :] = np.nan
    base[2, 5], base[2, 8000] = np.nan, 7.0
    base[3, 100], base[3, 4000] = np.inf, np.inf
    base[4, 17], base[4, 18] = 4.0, 4.0
    base[5, 1:] = -np.inf
    base[6, 2::3] = -np.inf
    base[7] *= 1e30
    base[8, 40], base[8, 41] = 0.0, -0.0
    base[8, 42:] = -5.0
    base[8, :40] = -5.0
    T = f32([1, 1, 0.5, 1, 0, 1, 2, 1, 1, np.nan, 1e-30, -1])
    k = [0, 3, 0, 0, 0, 4, 0, 2, 1, 0, 0, 5]
    p = f32([0.5, 1, 0.9, 0.9, 0.5, 0.5, np.nan, 1, 1, 0.4, 1, 0.2])
    m = f32([0, 0.1, 0, 0.1, 0, 2.0, np.nan, 0, 0, 0, 0.5, 0])
    u = f32([0.3, 0.3, 0.5, 0.75, 0.4, 0.4, 0.123, 0.9, 0.6, 0.2, 0.8, 0.7])
    tokens, probs = run(ctx, base, T, k, p, m, u)
    want = [0, 0, None, 4000, 17, 0, None, int(np.argmax(base[7])), 40, int(np.argmax(base[9])), int(np.argmax(base[10])),
            int(np.argmax(base[11]))]
    for r, t in enumerate(want):
        if t is None:
            pp = 1.0 if np.isnan(p[r]) else p[r]
            t, prob, far = ref.sample(base[r], T[r], k[r], pp, 0.0, u[r])
            assert far > 1e-6 and abs(probs[r] - prob) <= prob * 2.0 ** -20
        assert tokens[r] == t, r
    assert probs[0] == probs[1] == probs[4] == probs[9] == probs[11] == 1 and probs[3] == 0.5
    assert ctx.device_status() == binding.DEV_NAN_LOGIT


def test_ends_of_u(ctx):
    logits = f32(np.random.default_rng(11).standard_normal((1, 5000)))
    kept = sorted(ref.kept_tokens(logits[0], 1.0, 40, 1.0, 0.0)[0])
    for u, t in ((0.0, kept[0]), (-3.0, kept[0]), (float("nan"), kept[0]), (1.0, kept[-1]), (7.0, kept[-1]), (0.99999994, kept[-1])):
        tokens, _ = run(ctx, logits, None, [40], None, None, [u], probs=False)
        assert tokens[0] == t


def test_rows_do_not_depend_on_their_neighbours(ctx):
    rng = np.random.default_rng(12)
    logits = f32(rng.standard_normal((300, 20000)) * 3)
    args = [f32(rng.uniform(0.3, 1.3, 300)), rng.integers(0, 100, 300), f32(rng.uniform(0.3, 1.2, 300)), f32(rng.uniform(-0.1, 0.1, 300)),
            f32(rng.random(300))]
    all_tokens, all_probs = run(ctx, logits, *args)
    for r in (0, 1, 150, 299):
        t, pr = run(ctx, logits[r:r + 1], *[a[r:r + 1] for a in args])
        assert t[0] == all_tokens[r] and pr[0] == all_probs[r]


def test_nothing_to_do_and_refusals(ctx):
    import torch
    from paper_2604_05650_b200 import binding
    x = torch.zeros(64, device="cuda")
    before = ctx.launch_count()
    ctx.sample(0, 5, None, None, None, None, None, None, None)
    bad = [dict(rows=-1), dict(vocab=0), dict(vocab=400001, row_stride=400001), dict(row_stride=7), dict(logits=None), dict(u=None),
           dict(tokens=None), dict(logits=x.data_ptr() + 2), dict(T=x.data_ptr() + 1)]
    for change in bad:
        a = {**dict(rows=1, vocab=8, logits=x, T=None, u=x, tokens=x, row_stride=8), **change}
        with pytest.raises(binding.LvspecError) as e:
            ctx.sample(a["rows"], a["vocab"], a["logits"], a["T"], None, None, None, a["u"], a["tokens"], row_stride=a["row_stride"])
        assert e.value.status == (binding.ERR_UNSUPPORTED if a["vocab"] > 400000 else binding.ERR_INVALID_ARG)
    assert ctx.launch_count() == before
