"""lvspec_sample on batches of more rows than run at once: the order in which rows are taken up (by their filters) changes nothing."""
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


@pytest.mark.parametrize("rows,vocab", [(38, 40001), (61, 32800), (512, 33000), (600, 33000), (12, 400000)])
@pytest.mark.parametrize("given", ["all", "no top_k", "only min_p"])
def test_as_in_small_batches(ctx, rows, vocab, given):
    import torch
    rng = np.random.default_rng(rows)
    g = torch.Generator("cuda").manual_seed(rows)
    logits = torch.randn(rows, vocab, generator=g, device="cuda") * 3
    pick = rng.integers(0, 6, rows)
    T = np.where(pick == 5, 0, rng.uniform(0.5, 1.2, rows)).astype(np.float32)
    k = np.where((pick == 1) | (pick == 4), rng.integers(1, 200, rows), 0).astype(np.int32)
    p = np.where((pick == 2) | (pick == 4), rng.uniform(0.6, 0.99, rows), 1).astype(np.float32)
    m = np.where(pick == 3, rng.uniform(0.01, 0.2, rows), 0).astype(np.float32)
    u = rng.random(rows).astype(np.float32)
    dT, dk, dp, dm, du = (torch.from_numpy(a).cuda() for a in (T, k, p, m, u))
    if given != "all":
        dk = None
        k[:] = 0
    if given == "only min_p":
        dT = dp = None
        T[:], p[:] = 1, 1
    part = lambda t, a, b: None if t is None else t[a:b]                                             # noqa: E731
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)

    def run(step):
        tokens, probs = torch.full((rows,), -1, dtype=torch.int32, device="cuda"), torch.full((rows,), -1.0, device="cuda")
        for a in range(0, rows, step):
            b = min(rows, a + step)
            ctx.sample(b - a, vocab, logits[a:b], part(dT, a, b), part(dk, a, b), part(dp, a, b), part(dm, a, b), du[a:b], tokens[a:b],
                       probs[a:b])
        torch.cuda.synchronize()
        return tokens.cpu().numpy(), probs.cpu().numpy()

    tokens, probs = run(rows)
    one_by_one = run(37 if rows > 37 else 5)
    assert ctx.device_status() == 0
    assert (tokens == one_by_one[0]).all() and (probs == one_by_one[1]).all()
    host = logits.cpu().numpy()
    for r in range(0, rows, max(1, rows // 12)):
        want, prob, margin = ref.sample(host[r], float(T[r]), int(k[r]), float(p[r]), float(m[r]), float(u[r]))
        if margin > 1e-5 and p[r] >= 1:
            assert tokens[r] == want and abs(probs[r] - prob) <= prob * 2.0 ** -20
