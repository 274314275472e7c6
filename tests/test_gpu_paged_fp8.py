"""GPU parity of lvspec_verify_attention_paged_fp8 against the fp64 reference on the same codes,
scales and tables.

Tolerances.  A score is off by what splitting q into two E4M3 terms leaves: half a step of the
subnormals, 2^-10 where q's largest magnitude of the head is at least 2^7, so 2^-17 amax a channel,
    ds <= 2^-17 amax max_j sum_c |k_jc| / sqrt(D) + 2^-20 max|s| + 2^-20      (fp32 sums, products and exp2)
and a probability by a factor within exp(+-2 ds).  The probabilities that go into the product are rounded
to fp16 (2^-11), with their V scale, and `out` to bf16 (2^-8):
    |out - ref| <= 2^-8 |ref| + (2^-10 + 2.1 ds) sum p |v|,    |mass - ref| <= 2.1 ds."""
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


def bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16()


def make(seed, B, gamma, Hq, Hkv, D, page, block, kv_len, span, *, spare=3, junk=0x7F, q_gain=1.0, capacity=None):
    """Pages scattered over the pools; what no sequence owns, and what lies behind a length, is NaN codes."""
    rng = np.random.default_rng(seed)
    capacity = capacity or -(-max(max(kv_len), 1) // page) * page
    per_seq = capacity // page
    used = [-(-n // page) for n in kv_len]
    n_pages = sum(used) + spare
    order = rng.permutation(n_pages)
    table = np.full((B, per_seq), -7, np.int64)
    first = 0
    for b, u in enumerate(used):
        table[b, :u] = order[first:first + u]
        first += u
    pools = [np.full((n_pages, Hkv, page, D), junk, np.uint8) for _ in range(2)]
    scales = [np.exp(rng.standard_normal((n_pages, Hkv, page // block)) * 0.4).astype(np.float32) / 80 for _ in range(2)]
    for b, n in enumerate(kv_len):
        for j in range(used[b]):
            live = min(page, n - j * page)
            for pool in pools:
                pool[table[b, j], :, :live] = ref.e4m3_encode(rng.standard_normal((Hkv, live, D)) * 80)
    q = bf16(rng.standard_normal((B, gamma, Hq, D)) * q_gain)
    return dict(q=q, k=pools[0], v=pools[1], ks=scales[0], vs=scales[1], table=table, kv_len=list(kv_len),
                span=np.asarray(span, np.int32).reshape(B, 2), page=page, block=block, branches=1, capacity=capacity)


def call(ctx, c, cache=None, pools=None, max_kv_len=None, out=None, mass=None):
    import torch
    from paper_2604_05650_b200 import binding
    B, gamma, Hq, D = c["q"].shape
    n_pages, Hkv = c["k"].shape[:2]
    dev = [torch.from_numpy(np.ascontiguousarray(c[x])).cuda() for x in ("k", "v", "ks", "vs")]
    if pools:
        dev[:2] = pools
    table = torch.from_numpy(c["table"].astype(np.int32)).cuda()
    lens, span = torch.tensor(c["kv_len"], dtype=torch.int32).cuda(), torch.from_numpy(c["span"]).cuda()
    out = torch.full((B, gamma, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    mass = torch.full((B, gamma, Hq), float("nan"), device="cuda") if mass is None else mass
    shape = binding.attn_shape(B, gamma, Hq, Hkv, D, c["capacity"])
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    ctx.verify_attention_paged_fp8(shape, cache or binding.paged_fp8(c["page"], n_pages, c["block"]), c["q"].cuda(), *dev, table, lens,
                                   span, out, mass, max_kv_len=max_kv_len, n_branches=c["branches"])
    torch.cuda.synchronize()
    return out, mass


def check(c, out, mass, rows=None):
    q = c["q"].float().numpy().astype(np.float64)
    B, gamma, Hq, D = q.shape
    args = (q, c["k"], c["v"], c["ks"], c["vs"], c["table"], c["kv_len"], c["span"], c["block"], gamma // c["branches"])
    want, wmass = ref.attention(*args)
    weight, _ = ref.attention(*args, absolute=True)
    finite = np.where(np.isfinite(ref.DECODE[c["k"]]), np.abs(ref.DECODE[c["k"]]), 0).sum(-1) * \
        c["ks"].repeat(c["block"], -1)
    amax = np.abs(q).max()
    ds = 2.0 ** -17 * amax * finite.max() / D ** 0.5 + 2.0 ** -20 * (1 + amax * finite.max() / D ** 0.5)
    got, gmass = out.float().cpu().numpy().astype(np.float64), mass.cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all() and np.isfinite(gmass).all()
    off = np.abs(got - want) - (2.0 ** -8 * np.abs(want) + (2.0 ** -10 + 2.1 * ds) * weight)
    assert off.max() <= 0, f"out: worst excess {off.max():.3e} at {np.unravel_index(off.argmax(), off.shape)}"
    assert np.abs(gmass - wmass).max() <= 2.1 * ds, f"mass: {np.abs(gmass - wmass).max():.3e} against {2.1 * ds:.3e}"


CASES = [
    # B, gamma, Hq, Hkv, D, page, block, kv_len, span
    (1, 1, 1, 1, 128, 128, 128, [1], [[0, 1]]),                                # one position
    (1, 1, 8, 2, 64, 16, 16, [333], [[40, 200]]),
    (1, 8, 10, 2, 128, 128, 128, [1500], [[100, 1200]]),
    (2, 8, 8, 2, 128, 64, 32, [700, 389], [[10, 500], [0, 381]]),              # lengths apart, half tiles
    (4, 4, 6, 3, 128, 32, 32, [0, 4, 128, 129], [[0, 0], [0, 0], [3, 100], [64, 125]]),     # an empty place; one tile; one more
    (3, 8, 4, 4, 128, 16, 16, [3, 8, 130], [[0, 2], [0, 0], [1, 122]]),        # fewer positions than queries
    (1, 10, 16, 2, 128, 256, 64, [2077], [[512, 1900]]),                       # 80 rows
    (1, 16, 7, 1, 128, 384, 128, [1153], [[128, 256]]),                        # 112 rows, pages of three tiles, span at tile borders
    (1, 16, 8, 1, 128, 128, 16, [777], [[0, 761]]),                            # 128 rows
    (2, 16, 16, 2, 64, 64, 64, [1027, 500], [[1, 1000], [3, 4]]),              # 128 rows, head_dim 64
    (2, 4, 28, 4, 128, 512, 128, [600, 599], [[256, 500], [1, 2]]),            # G = 7
    (1, 1, 5, 1, 128, 128, 128, [5000], [[1000, 4000]]),                       # one head over many CTAs
    (1, 8, 40, 8, 128, 128, 128, [4096], [[256, 3328]]),
    (40, 2, 8, 8, 128, 32, 16, [37 * b % 600 for b in range(40)], [[b, 3 * b] for b in range(40)]),    # straight cuts
    (128, 1, 4, 2, 64, 16, 16, [(b * b) % 300 for b in range(128)], [[0, 40]] * 128),
    (20, 1, 16, 8, 128, 64, 64, [900 + 13 * b for b in range(20)], [[100, 700]] * 20),
]


@pytest.mark.parametrize("case", CASES, ids=[f"B{c[0]}g{c[1]}h{c[2]}-{c[3]}d{c[4]}p{c[5]}s{c[6]}" for c in CASES])
def test_against_the_reference(ctx, case):
    c = make(sum(map(int, case[:7])), *case)
    out, mass = call(ctx, c)
    assert ctx.device_status() == 0
    check(c, out, mass)
    again, mass2 = call(ctx, c)
    assert (again.view(dtype=__import__("torch").int16) == out.view(dtype=__import__("torch").int16)).all() and (mass == mass2).all()
