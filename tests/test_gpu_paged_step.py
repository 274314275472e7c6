"""lvspec_plan_pages and lvspec_append_paged_fp8 against the reference, exactly: page tables and slots are
integers, and codes and scales follow from roundings that are given in full."""
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


def dev(a, dtype=np.int32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def plan(ctx, page, per_seq, n_pages, max_new, lens, new, held, n_free, free, table, in_place=False):
    import torch
    B = len(lens)
    d = [dev(a) for a in (lens, new, held, [n_free])]
    d_free, d_table = dev(free), dev(table)
    res = [d[0], d[2], d[3]] if in_place else [torch.full((n,), -99, dtype=torch.int32, device="cuda") for n in (B, B, 1)]
    starts, slots = (torch.full((n,), -99, dtype=torch.int32, device="cuda") for n in (B + 1, max_new + 5))
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    ctx.plan_pages(B, page, per_seq, n_pages, max_new, *d, d_free, d_table, *res, starts, slots)
    torch.cuda.synchronize()
    assert (slots[max_new:] == -99).all() and (d_free.cpu().numpy() == free).all()
    return [t.cpu().numpy() for t in (d_table, *res, starts, slots[:max_new])]


def check_plan(ctx, *args, in_place=False):
    from paper_2604_05650_b200 import binding
    got = plan(ctx, *args, in_place=in_place)
    want = ref.plan_pages(*args)
    for g, w in zip(got, want[:6]):
        assert (g == np.asarray(w)).all()
    assert ctx.device_status() == (binding.DEV_REFUSED if want[6] else 0)
    return got


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,page,new,held_len,spare", [
    (1, 16, 1, 0, 0), (1, 16, 1, 15, 3), (1, 16, 1, 16, 0), (7, 1, 3, 10, 1), (16, 16, 8, 1000, 0), (16, 128, 300, 500, 77),
    (128, 32, 200, 40, 1000), (1024, 64, 9, 100, 5), (3, 384, 5000, 700, 3), (1000, 16, 0, 33, 9)])
def test_plan(ctx, B, page, new, held_len, spare, in_place):
    rng = np.random.default_rng(B * 1000 + page)
    lens = rng.integers(0, held_len + 1, B)
    add = rng.integers(0, new + 1, B)
    # some requests hold more pages than their length needs, as after a step with rejected tokens
    held = -(-lens // page) + rng.integers(0, 2, B)
    per_seq = int((-(-(lens + add) // page)).max()) + 2
    n_pages = int(held.sum()) + int((-(-(lens + add) // page)).sum()) + 4
    order = rng.permutation(n_pages)
    table = np.full((B, per_seq), -1)
    at = 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    free = np.concatenate([order[at:], np.full(at, -5)])
    check_plan(ctx, page, per_seq, n_pages, int(add.sum()) + spare, lens, add, held, n_pages - at, free, table, in_place=in_place)


@pytest.mark.parametrize("case", [
    # lens, new, held, n_free, max_new (pages of 16, 4 a row, 12 pages)
    ([0, 0, 5, 0], [20, 40, 3, 1], [0, 0, 1, 0], 4, 70),          # the second finds too few pages, the third needs none
    ([0, 60, 0], [10, 5, 10], [0, 4, 0], 12, 30),                 # beyond its row
    ([0, 0], [30, 30], [0, 0], 12, 40),                           # beyond the slot map
    ([-3, 5, 5, 5], [4, -2, 4, 4], [1, 1, -1, 5], 12, 40),        # senseless
    ([0, 0], [2**31 - 1, 2**31 - 1], [0, 0], 12, 40),
    ([0, 5], [0, 0], [0, 1], 0, 0),                               # nothing to do
    ([0, 0], [10, 10], [0, 0], -4, 20), ([0, 0], [10, 10], [0, 0], 99, 20),
    ([3, 0], [4, 2], [1, 0], 3, 10)])                             # an entry that is no page
def test_plan_refuses_requests(ctx, case):
    lens, new, held, n_free, max_new = case
    table = np.full((len(lens), 4), -1)
    for b, h in enumerate(held):
        table[b, :max(0, min(h, 4))] = 100 if case[0] == [3, 0] else b
    check_plan(ctx, 16, 4, 12, max_new, lens, new, held, n_free, np.arange(12)[::-1].copy(), table)


def run_append(ctx, x, slots, pool, scale, page, block, layout="dense", fused=True):
    """Both K and V are given x, V negated; returns K's (pool, scale) and checks V's against it."""
    import torch
    from paper_2604_05650_b200 import binding
    n, H, D = x.shape
    n_pages = pool.shape[0]
    xt = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16()
    if fused:       # rows of a fused projection
        rows = torch.full((n, 5, H, D), 9.0, dtype=torch.bfloat16, device="cuda")
        rows[:, 1], rows[:, 3] = xt.cuda(), -xt.cuda()
        k, v, st = rows[:, 1], rows[:, 3], 5 * H * D
    else:
        k, v, st = xt.cuda(), -xt.cuda(), H * D
    pt = torch.from_numpy(pool).cuda()
    if layout == "dense":
        pk, pv, cache = pt.clone(), pt.clone(), binding.paged_fp8(page, n_pages, block)
        back = lambda t: t                                                    # noqa: E731
    elif layout == "position":
        pk, pv = (pt.transpose(1, 2).contiguous().clone() for _ in range(2))
        cache = binding.paged_fp8(page, n_pages, block, page * H * D, D, H * D)
        back = lambda t: t.transpose(1, 2)                                    # noqa: E731
    else:
        both = torch.stack([pt, pt], 1).contiguous()
        pk, pv = both[:, 0], both[:, 1]
        cache = binding.paged_fp8(page, n_pages, block, 2 * H * page * D, page * D, D)
        back = lambda t: t                                                    # noqa: E731
    sk, sv = torch.from_numpy(scale).cuda(), torch.from_numpy(scale).cuda()
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    ctx.append_paged_fp8(n, H, D, cache, k, v, st, st, dev(slots), pk, pv, sk, sv)
    torch.cuda.synchronize()
    pk, pv = back(pk).cpu().numpy(), back(pv).cpu().numpy()
    touched = [s for s in slots if 0 <= s < n_pages * page]
    for s in touched:       # (the sign of a NaN code is nobody's business)
        a, b = pk[s // page, :, s % page], pv[s // page, :, s % page]
        assert (((a ^ b) == 0x80) | ((a & 0x7F) == 0x7F)).all()
    assert (sk.cpu().numpy() == sv.cpu().numpy()).all()
    return pk, sk.cpu().numpy()


def old_cache(rng, n_pages, H, page, D, block, power=True):
    pool = ref.e4m3_encode(rng.standard_normal((n_pages, H, page, D)) * 100)
    scale = np.exp2(rng.integers(-9, 2, (n_pages, H, page // block))).astype(np.float32)
    return pool, scale if power else (scale * 0.77).astype(np.float32)


def slots_of(rng, page, n_pages, runs):
    """Runs of consecutive positions (first position, count) of one sequence each, pages at random."""
    order, got = list(rng.permutation(n_pages)), []
    for first, count in runs:
        pages = {}
        for pos in range(first, first + count):
            if pos // page not in pages:
                pages[pos // page] = order.pop()
            got.append(int(pages[pos // page]) * page + pos % page)
    return got


@pytest.mark.parametrize("layout,fused", [("dense", True), ("position", False), ("interleaved", True)])
@pytest.mark.parametrize("H,D,page,block,runs", [
    (2, 128, 16, 16, [(0, 1)]),
    (8, 128, 64, 64, [(3, 8), (60, 8), (128, 8), (0, 8), (63, 1)]),            # a decoding step's
    (3, 64, 32, 16, [(0, 100), (7, 30), (15, 2)]),
    (1, 128, 128, 128, [(0, 300), (127, 129)]),
    (2, 128, 256, 32, [(31, 1), (250, 20), (0, 64)]),
    (4, 64, 384, 128, [(100, 500)])])
def test_append(ctx, H, D, page, block, runs, layout, fused):
    rng = np.random.default_rng(H * 7 + page)
    n_pages = sum(-(-(a + n) // page) for a, n in runs) + 2
    pool, scale = old_cache(rng, n_pages, H, page, D, block)
    slots = slots_of(rng, page, n_pages, runs)
    slots = slots[:1] + [-1, n_pages * page] * 3 + slots[1:] if len(slots) == 1 else slots + [-1] * 5
    import torch
    x = torch.from_numpy(rng.standard_normal((len(slots), H, D)) * np.exp2(rng.integers(-6, 6, (len(slots), H, 1)))).bfloat16().double().numpy()
    got = run_append(ctx, x, slots, pool, scale, page, block, layout, fused)
    want = ref.append(x, slots, pool, scale, page, block)
    assert (got[1] == want[1]).all() and (got[0] == want[0]).all()
    assert ctx.device_status() == 0


def test_append_special_values(ctx):
    """Infinities saturate and do not count for the scale; NaN stays NaN; zeros; the ends of the range of bf16; a cache whose
    scales are no powers of two."""
    rng = np.random.default_rng(5)
    H, D, page, block = 2, 128, 64, 16
    pool, scale = old_cache(rng, 6, H, page, D, block, power=False)
    import torch
    x = torch.from_numpy(rng.standard_normal((48, H, D))).bfloat16().double().numpy()
    x[3, 0, 5], x[3, 1, 6], x[4, 0, 0] = np.inf, -np.inf, np.nan
    x[16:24] = 0
    x[24:26] = 2.0 ** -133
    x[26, 0, 0] = 3.3e38
    x[40:] *= 1e-36
    slots = [s for s in range(64 + 5, 64 + 5 + 24)] + [128 + s for s in range(16)] + [200, 201] + [193 + 64 + s for s in range(6)]
    x = torch.from_numpy(x).bfloat16().double().numpy()
    got = run_append(ctx, x, slots, pool, scale, page, block)
    want = ref.append(x, slots, pool, scale, page, block)
    assert (got[1] == want[1]).all()
    same = (got[0] == want[0]) | (((got[0] & 0x7F) == 0x7F) & ((want[0] & 0x7F) == 0x7F))
    assert same.all()


def test_append_of_nothing(ctx):
    import torch
    from paper_2604_05650_b200 import binding
    t = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    before = ctx.launch_count()
    ctx.append_paged_fp8(0, 1, 64, binding.paged_fp8(16, 2, 16), None, None, 64, 64, None, t, t, t, t)
    assert ctx.launch_count() == before


def test_a_slot_map_of_one_block_only_stays_inside_it(ctx):
    """Slots given twice: what the block then holds is undefined, but nothing else is touched."""
    rng = np.random.default_rng(6)
    pool, scale = old_cache(rng, 3, 2, 32, 64, 16)
    import torch
    x = torch.from_numpy(rng.standard_normal((700, 2, 64))).bfloat16().double().numpy()
    got = run_append(ctx, x * 0 + 1.0, [32 + 16 + i % 3 for i in range(700)], pool, scale, 32, 16)
    rest = np.ones(pool.shape, bool)
    rest[1, :, 16:] = False
    assert (got[0][rest] == pool[rest]).all() and (ref.DECODE[got[0][1, :, 16:19]] * got[1][1, :, 1].reshape(2, 1, 1) == 1).all()
