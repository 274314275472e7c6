"""lvspec_verify_attention_paged_fp8 where it can go wrong: scores and scales that leave their first tile's range, special values,
layouts, bad tables and lengths, trees, long pools, captured launches, two at once, refusals.

Tolerances are those of the call's parity tests, and where probabilities or scales span many binades what fp16 cannot hold beside the
largest: an element of P^T is off by at most half a step of fp16's subnormals, 2^-25, times a code of at most 448, in units of
2^k0 <= 4 max(v_scale), and the sum that it is divided by is at least 2^6:
    L 448 4 max(v_scale) 2^-31."""
import numpy as np
import pytest

from oracle import paged_step as ref
from test_gpu_paged_fp8 import bf16, call, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2604_05650_b200 import binding
    c = binding.Context(0)
    yield c
    c.close()


def check(c, out, mass, which=None, rows=None, wide=False):
    """Sequences `which` (all), queries `rows` (all), against the reference."""
    which = range(len(c["kv_len"])) if which is None else which
    q = c["q"].float().numpy().astype(np.float64)
    gamma, Hq, D = q.shape[1:]
    Hkv = c["k"].shape[1]
    got, gmass = out.float().cpu().numpy().astype(np.float64), mass.cpu().numpy().astype(np.float64)
    rows = list(range(gamma)) if rows is None else rows
    for b in which:
        L = min(max(c["kv_len"][b], 0), c["capacity"])
        args = (np.where(np.isfinite(q[b:b + 1]), q[b:b + 1], 0), c["k"], c["v"], c["ks"], c["vs"], c["table"][b:b + 1], [L],
                c["span"][b:b + 1], c["block"], gamma // c["branches"])
        want, wmass = ref.attention(*args)
        weight, _ = ref.attention(*args, absolute=True)
        pages = c["table"][b][:-(-L // c["page"])]
        pages = pages[(pages >= 0) & (pages < len(c["k"]))]
        codes = np.abs(ref.DECODE[c["k"][pages]])
        size = np.where(np.isfinite(codes), codes, 0).sum(-1) * np.nan_to_num(c["ks"][pages]).repeat(c["block"], -1)
        biggest = size.max() if size.size else 0.0
        amax = np.abs(args[0]).max()
        ds = 2.0 ** -17 * amax * biggest / D ** 0.5 + 2.0 ** -20 * (1 + amax * biggest / D ** 0.5)
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -10 + 2.1 * ds) * weight
        if wide:
            tol += L * 448 * 4 * np.nan_to_num(c["vs"][pages]).max() * 2.0 ** -31
        off = (np.abs(got[b] - want[0]) - tol[0])[rows]
        assert off.max() <= 0, f"sequence {b}: worst excess {off.max():.3e} at {np.unravel_index(off.argmax(), off.shape)}"
        assert np.abs(gmass[b] - wmass[0])[rows].max() <= 2.1 * ds


def same(a, b):
    import torch
    return torch.equal(a[0].view(torch.int16), b[0].view(torch.int16)) and torch.equal(a[1].view(torch.int32), b[1].view(torch.int32))


def at_positions(c, b, kind, values):
    """Writes values [Hkv, L, D] (floats) of sequence b into the cache as codes under its present scales."""
    for j in range(-(-values.shape[1] // c["page"])):
        part = values[:, j * c["page"]:(j + 1) * c["page"]]
        page = c["table"][b, j]
        s = c[kind + "s"][page].repeat(c["block"], -1)[:, :part.shape[1], None].astype(np.float64)
        c[kind][page][:, :part.shape[1]] = ref.e4m3_encode(part / s)


# batches of so many pairs that a CTA has sixteen tiles or more; query rows for each organisation of the softmax
@pytest.mark.parametrize("gamma,Hq", [(4, 8), (8, 20), (10, 32), (16, 32)])
def test_scores_leave_the_first_tiles_range(ctx, gamma, Hq):
    B, Hkv, L = 40, 4, 2048
    c = make(gamma, B, gamma, Hq, Hkv, 128, 128, 64, [L - 5 * b for b in range(B)], [[100 + b, 1500] for b in range(B)])
    c["q"] = bf16(np.ones(c["q"].shape))
    c["ks"][:] = 1 / 16
    rng = np.random.default_rng(5)
    which = []
    for b in range(0, B, 9):
        n = c["kv_len"][b]
        k = rng.standard_normal((Hkv, n, 128)) * 0.25
        step = (np.arange(n) // 300)[None, :, None] * 1.5            # +17 a step in the score
        if len(which) == 0:
            k = k + step
        elif len(which) == 1:
            k = k - step
        elif len(which) == 2:
            k[:, 0] += 3.0                                            # a sink, everything else 2^49 below it
        elif len(which) == 3:
            k[:, 1777] += 4.0                                         # a late spike
        else:
            k[:, ::2] -= 2.0                                          # two levels side by side
            k[:, n // 2:] += 1.0
        at_positions(c, b, "k", k)
        which.append(b)
    out, mass = call(ctx, c)
    assert ctx.device_status() == 0
    check(c, out, mass, which, wide=True)


@pytest.mark.parametrize("gamma,Hq", [(1, 4), (8, 20), (10, 32), (16, 32)])
def test_value_scales_that_jump(ctx, gamma, Hq):
    B, Hkv, L = 40, 4, 2048
    c = make(gamma + 50, B, gamma, Hq, Hkv, 128, 64, 32, [L - b for b in range(B)], [[100 + b, 1500] for b in range(B)])
    for b in range(B):
        for j in range(-(-c["kv_len"][b] // 64)):
            step = 12.0 * (j // 8)
            c["vs"][c["table"][b, j]] *= np.float32(2.0 ** (step if b % 2 else -step))
    c["vs"][c["table"][3, 4]] = 0                # blocks of nothing
    out, mass = call(ctx, c)
    assert ctx.device_status() == 0
    check(c, out, mass, [0, 1, 3, 20], wide=True)


@pytest.mark.parametrize("gain", [2.0 ** -20, 1.0, 300.0, 2.0 ** 100])
def test_large_and_small_q(ctx, gain):
    c = make(3, 2, 8, 8, 2, 128, 32, 32, [900, 131], [[64, 700], [0, 100]])
    q = c["q"].float().numpy() * np.float32(gain)
    q[0, 3] *= 0.01                              # one query far smaller than the others
    c["q"] = bf16(q)
    c["ks"] = (c["ks"] / np.float32(gain)).astype(np.float32)
    check(c, *call(ctx, c))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("gamma,Hq", [(4, 8), (16, 16)])
def test_a_query_of_nan_spoils_no_other(ctx, bad, gamma, Hq):
    import torch
    c = make(8, 3, gamma, Hq, 2, 128, 128, 64, [700, 2000, 130], [[64, 600], [0, 1500], [3, 90]])
    q = c["q"].float().numpy()
    q[1, 2, 3, 77] = bad
    c["q"] = bf16(q)
    out, mass = call(ctx, c)
    assert torch.isnan(out[1, 2, 3]).all() and torch.isnan(mass[1, 2, 3])
    out[1, 2, 3], mass[1, 2, 3] = 0, 0
    assert torch.isfinite(out).all() and torch.isfinite(mass).all()
    check(c, out, mass, rows=[g for g in range(gamma) if g != 2])


@pytest.mark.parametrize("D,page,block", [(128, 16, 16), (128, 64, 32), (64, 128, 128), (64, 32, 16), (128, 256, 64)])
def test_layouts_of_the_pools_are_all_the_same(ctx, D, page, block):
    import torch
    from paper_2604_05650_b200 import binding
    c = make(D + page, 3, 4, 12, 3, D, page, block, [1000, 77, 300], [[10, 500], [0, 70], [100, 200]])
    n_pages, H = c["k"].shape[:2]
    dense = call(ctx, c)
    check(c, *dense)
    k, v = (torch.from_numpy(c[x]).cuda() for x in "kv")
    by_position = [t.transpose(1, 2).contiguous().clone() for t in (k, v)]
    assert same(dense, call(ctx, c, binding.paged_fp8(page, n_pages, block, page * H * D, D, H * D), by_position))
    both = torch.stack([k, v], 1).contiguous()
    assert same(dense, call(ctx, c, binding.paged_fp8(page, n_pages, block, 2 * H * page * D, page * D, D), [both[:, 0], both[:, 1]]))
    # rows of K and V side by side, spaces between heads and pages
    apart = torch.full((n_pages, H * page * 2 + 3, D + 16), 0x7F, dtype=torch.uint8, device="cuda")
    rows = apart[:, :H * page * 2].view(n_pages, H, page, 2, D + 16)
    rows[:, :, :, 0, :D], rows[:, :, :, 1, :D] = k, v
    st = (apart.stride(0), page * 2 * (D + 16), 2 * (D + 16))
    assert same(dense, call(ctx, c, binding.paged_fp8(page, n_pages, block, *st), [rows[:, :, :, 0], rows[:, :, :, 1]]))


def test_what_no_position_needs_may_be_anything(ctx):
    """Scales of blocks behind the lengths, table entries behind them, pages that nobody owns."""
    c = make(21, 4, 4, 8, 2, 128, 64, 16, [600, 129, 64, 0], [[10, 500], [0, 120], [3, 9], [0, 0]])
    clean = call(ctx, c)
    used = np.zeros(c["ks"].shape, bool)
    for b, n in enumerate(c["kv_len"]):
        for j in range(-(-n // 64)):
            used[c["table"][b, j], :, :-(-min(64, n - 64 * j) // 16)] = True
    for x in ("ks", "vs"):
        c[x] = np.where(used, c[x], np.float32(np.nan))
    c["table"][c["table"] < 0] = 2 ** 31 - 1
    assert same(clean, call(ctx, c))
    assert ctx.device_status() == 0
    check(c, *clean)


def test_entries_outside_the_pool_read_as_zeros(ctx):
    c = make(22, 2, 4, 8, 2, 128, 32, 32, [500, 300], [[10, 400], [5, 200]])
    c["table"][0, 3] = len(c["k"])
    c["table"][0, 9] = -1
    c["table"][1, 2:5] = [2 ** 31 - 1, -2 ** 31, 10 ** 6]
    check(c, *call(ctx, c))


def test_lengths_out_of_range_count_as_empty(ctx):
    import torch
    from paper_2604_05650_b200 import binding
    c = make(23, 5, 2, 8, 4, 128, 128, 128, [500, 100, 256, 300, 50], [[10, 400]] * 5, capacity=512)
    good = call(ctx, c, max_kv_len=500)
    assert ctx.device_status() == 0
    bad = {**c, "kv_len": [500, -1, 257 + 512, 2 ** 31 - 1, 50]}
    out, mass = call(ctx, bad, max_kv_len=500)
    assert ctx.device_status() == binding.DEV_BAD_LENGTH
    for b in (1, 2, 3):
        assert (out[b] == 0).all() and (mass[b] == 0).all()
    check(c, out, mass, [0, 4])
    out, mass = call(ctx, c, max_kv_len=256)
    assert ctx.device_status() == binding.DEV_BAD_LENGTH
    assert (out[0] == 0).all() and (out[3] == 0).all()
    check(c, out, mass, [1, 2, 4])
    assert torch.isfinite(good[0]).all()


@pytest.mark.parametrize("gamma,branches,Hq,Hkv,kv_len", [(8, 2, 8, 2, [700, 130]), (8, 8, 4, 4, [129, 8]), (12, 3, 10, 1, [128, 140]),
                                                         (64, 4, 4, 2, [300, 191]), (64, 64, 2, 1, [64, 1000]), (6, 2, 6, 6, [5, 6])])
def test_trees(ctx, gamma, branches, Hq, Hkv, kv_len):
    c = make(gamma + branches, 2, gamma, Hq, Hkv, 128, 16, 16, kv_len, [[0, n // 2] for n in kv_len])
    c["branches"] = branches
    check(c, *call(ctx, c))


@pytest.mark.parametrize("span", [[0, 0], [0, 10 ** 9], [-5, 100], [300, 200], [699, 10 ** 6], [128, 256], [127, 129]])
def test_any_span(ctx, span):
    """Positions of the span that a query sees; a span is not checked, it is read on the device."""
    c = make(31, 2, 4, 8, 2, 128, 128, 64, [700, 131], [span, span])
    check(c, *call(ctx, c))


def test_positions_beyond_4_gb(ctx):
    """Pages at both ends of pools of 5 GB."""
    import torch
    from paper_2604_05650_b200 import binding
    H, page, D, n_pages = 8, 128, 128, 40000
    c = make(41, 2, 2, 16, H, D, page, 64, [1500, 700], [[10, 1200], [0, 600]])
    old = c["table"].copy()
    far = np.arange(old.max() + 1) * 3              # page p moves to the end, 3 p before it, every other one to the start
    far = np.where(np.arange(len(far)) % 2 == 0, n_pages - 1 - far, far)
    pools = [torch.full((n_pages, H, page, D), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)]
    small = call(ctx, c)
    used = [int(p) for p in np.unique(old) if p >= 0]
    scales = [np.full((n_pages, H, page // 64), np.nan, np.float32) for _ in range(2)]
    for p in used:
        for t, x in zip(pools, "kv"):
            t[int(far[p])] = torch.from_numpy(c[x][p]).cuda()
        scales[0][far[p]], scales[1][far[p]] = c["ks"][p], c["vs"][p]
    table = np.where(old >= 0, far[old], -1)
    big = {**c, "ks": scales[0], "vs": scales[1], "table": table}
    assert same(small, call(ctx, big, binding.paged_fp8(page, n_pages, 64), pools))
    check(c, *small)


def test_a_captured_launch_follows_the_lengths():
    import torch
    from paper_2604_05650_b200 import binding
    ctx = binding.Context(0)
    try:
        B, gamma, Hq, Hkv, D, page = 6, 3, 16, 4, 128, 64
        c = make(51, B, gamma, Hq, Hkv, D, page, 32, [4000] * B, [[0, 0]] * B)
        n_pages = len(c["k"])
        shape = binding.attn_shape(B, gamma, Hq, Hkv, D, c["capacity"])
        cache = binding.paged_fp8(page, n_pages, 32)
        dev = {x: torch.from_numpy(c[x]).cuda() for x in ("k", "v", "ks", "vs")}
        table = torch.from_numpy(c["table"].astype(np.int32)).cuda()
        lens, span = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, 2, dtype=torch.int32, device="cuda")
        q = c["q"].cuda()
        out = torch.full((B, gamma, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        mass = torch.full((B, gamma, Hq), float("nan"), device="cuda")
        need = ctx.attention_paged_fp8_workspace_bytes(shape)
        ctx.reserve(need)
        cap = ctx.workspace_capacity()
        assert cap >= need
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        before = ctx.launch_count()
        with torch.cuda.graph(graph, stream=stream):
            ctx.set_stream(torch.cuda.current_stream().cuda_stream)
            ctx.verify_attention_paged_fp8(shape, cache, q, dev["k"], dev["v"], dev["ks"], dev["vs"], table, lens, span, out, mass)
        assert ctx.launch_count() == before + 2 and ctx.workspace_capacity() == cap
        ctx.set_stream(stream.cuda_stream)
        rng = np.random.default_rng(2)
        for step in range(4):
            c["kv_len"] = [int(x) for x in rng.integers(0, 4001, B)] if step else [1, 0, 4000, 128, 129, 2]
            c["span"] = np.asarray([[n // 4, n // 2] for n in c["kv_len"]], np.int32)
            lens.copy_(torch.tensor(c["kv_len"], dtype=torch.int32))
            span.copy_(torch.from_numpy(c["span"]))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert ctx.device_status() == 0
            check(c, out, mass, [step, 5])
            keep = out.clone(), mass.clone()
            assert same(keep, call(ctx, c))
    finally:
        ctx.close()


def test_scratch_that_would_grow_in_a_capture_is_refused():
    import torch
    from paper_2604_05650_b200 import binding
    ctx = binding.Context(0)
    try:
        shape = binding.attn_shape(1, 16, 8, 1, 128, 1024)
        cache = binding.paged_fp8(128, 8, 128)
        assert ctx.attention_paged_fp8_workspace_bytes(shape) > ctx.workspace_capacity()
        q = torch.zeros(1, 16, 8, 128, dtype=torch.bfloat16, device="cuda")
        pool, scale = torch.zeros(8, 1, 128, 128, dtype=torch.uint8, device="cuda"), torch.ones(8, 1, 1, device="cuda")
        ints = torch.arange(8, dtype=torch.int32, device="cuda")
        out, mass, x = torch.zeros_like(q), torch.zeros(1, 16, 8, device="cuda"), torch.zeros(8, device="cuda")
        torch.cuda.synchronize()
        graph, before = torch.cuda.CUDAGraph(), ctx.launch_count()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            ctx.set_stream(torch.cuda.current_stream().cuda_stream)
            x += 1
            with pytest.raises(binding.LvspecError) as e:
                ctx.verify_attention_paged_fp8(shape, cache, q, pool, pool, scale, scale, ints, ints, ints, out, mass)
            assert e.value.status == binding.ERR_WORKSPACE
        assert ctx.launch_count() == before
        graph.replay()
        torch.cuda.synchronize()
        assert float(x[0]) == 1.0
        ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    finally:
        ctx.close()


def test_two_contexts_at_once():
    """Calls of two contexts on two streams, neither waiting for the other: as alone."""
    import torch
    from paper_2604_05650_b200 import binding
    both = [binding.Context(0) for _ in range(2)]
    try:
        cases = [make(61, 3, 8, 10, 2, 128, 128, 64, [5000, 300, 2000], [[10, 2000]] * 3), make(62, 40, 1, 8, 8, 64, 16, 16, [333] * 40, [[3, 200]] * 40)]
        alone = [call(x, c) for x, c in zip(both, cases)]
        jobs = []
        for x, c in zip(both, cases):
            B, gamma, Hq, D = c["q"].shape
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                t = [c["q"].cuda()] + [torch.from_numpy(np.ascontiguousarray(c[n])).cuda() for n in ("k", "v", "ks", "vs")] + \
                    [torch.from_numpy(c["table"].astype(np.int32)).cuda(), torch.tensor(c["kv_len"], dtype=torch.int32).cuda(),
                     torch.from_numpy(c["span"]).cuda(), torch.full((B, gamma, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda"),
                     torch.full((B, gamma, Hq), float("nan"), device="cuda")]
            jobs.append((x, stream, binding.attn_shape(B, gamma, Hq, c["k"].shape[1], D, c["capacity"]),
                         binding.paged_fp8(c["page"], len(c["k"]), c["block"]), t))
        torch.cuda.synchronize()
        for _ in range(50):
            for x, stream, shape, cache, t in jobs:
                x.set_stream(stream.cuda_stream)
                x.verify_attention_paged_fp8(shape, cache, *t)
        torch.cuda.synchronize()
        for (x, _, _, _, t), want in zip(jobs, alone):
            assert x.device_status() == 0 and same(want, t[-2:])
    finally:
        for x in both:
            x.set_stream(None)
            x.close()


def test_refusals_launch_nothing(ctx):
    import torch
    from paper_2604_05650_b200 import binding
    q = torch.zeros(1, 4, 8, 128, dtype=torch.bfloat16, device="cuda")
    pool, scale = torch.zeros(8, 2, 128, 128, dtype=torch.uint8, device="cuda"), torch.ones(8, 2, 2, device="cuda")
    ints = torch.zeros(64, dtype=torch.int32, device="cuda")
    out, mass = torch.full_like(q, 7), torch.full((1, 4, 8), 7.0, device="cuda")
    before = ctx.launch_count()
    I, U = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    bad = [(I, dict(B=0)), (I, dict(B=129)), (I, dict(gamma=0)), (I, dict(gamma=65)), (I, dict(Hq=9)), (U, dict(gamma=64)), (U, dict(D=96)),
           (I, dict(n_split=1)), (U, dict(kernel=binding.KERNEL_SIMT)), (I, dict(kernel=9)), (I, dict(branches=3)), (I, dict(branches=0)),
           (I, dict(page=48)), (I, dict(page=0)), (I, dict(page=8)), (I, dict(page=192)), (I, dict(block=8)), (I, dict(block=256)),
           (I, dict(page=32, block=64)), (I, dict(n_pages=0)), (I, dict(n_pages=2 ** 24)), (I, dict(strides=(1, 1, 1))),
           (I, dict(strides=(32768, 16384, 120))), (I, dict(strides=(32768, 16384, 112))), (I, dict(strides=(32768, 0, 128))),
           (I, dict(strides=(-32768, 16384, 128))), (I, dict(strides=(2 ** 38, 16384, 128))), (I, dict(capacity=1000)),
           (I, dict(capacity=0)), (I, dict(max_len=0)), (I, dict(max_len=1025)), (I, dict(capacity=2 ** 31 - 128, max_len=2 ** 30 + 1)),
           (I, dict(B=128, Hkv=8, capacity=2 ** 30, max_len=2 ** 30 - 1, n_pages=100))]
    bad += [(I, {name: None}) for name in ("q", "k", "v", "ks", "vs", "table", "lens", "span", "out", "mass")]
    bad += [(I, {name: t.data_ptr() + 1}) for name, t in (("q", q), ("k", pool), ("v", pool), ("ks", scale), ("vs", scale), ("table", ints),
                                                          ("lens", ints), ("span", ints), ("out", out), ("mass", mass))]
    for status, change in bad:
        a = {**dict(B=1, gamma=4, Hq=8, Hkv=2, D=128, capacity=1024, n_split=0, kernel=0, branches=1, page=128, block=64, n_pages=8,
                    strides=(0, 0, 0), max_len=None, q=q, k=pool, v=pool, ks=scale, vs=scale, table=ints, lens=ints, span=ints, out=out,
                    mass=mass), **change}
        shape = binding.attn_shape(a["B"], a["gamma"], a["Hq"], a["Hkv"], a["D"], a["capacity"], a["n_split"], a["kernel"])
        with pytest.raises(binding.LvspecError) as e:
            ctx.verify_attention_paged_fp8(shape, binding.paged_fp8(a["page"], a["n_pages"], a["block"], *a["strides"]), a["q"], a["k"], a["v"],
                                           a["ks"], a["vs"], a["table"], a["lens"], a["span"], a["out"], a["mass"], a["max_len"], a["branches"])
        assert e.value.status == status, change
    torch.cuda.synchronize()
    assert ctx.launch_count() == before and (out == 7).all() and (mass == 7).all()
