"""lvspec_verify_attention_paged_fp8 at every number of query rows that has its own organisation, several tiles a CTA; batches of
nothing; pages that sequences share; calls of different shapes one behind the other."""
import numpy as np
import pytest

from test_gpu_paged_fp8 import call, make
from test_gpu_paged_fp8_cases import check, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2604_05650_b200 import binding
    c = binding.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gamma,G", [(7, 1), (3, 5), (4, 6), (8, 4), (1, 33), (5, 8), (47, 1), (6, 8), (7, 8), (57, 1), (8, 8), (13, 5), (9, 8),
                                     (11, 7), (11, 8), (12, 8), (1, 97), (13, 8), (16, 7), (63, 2), (2, 64)])
def test_rows(ctx, gamma, G, D):
    """Shares of seven or eight tiles, straight through the sequences: of a head's end, its begin, or all of one."""
    Hkv = 4
    lens = [1500 - 61 * b for b in range(24)]
    c = make(gamma * G + D, 24, gamma, Hkv * G, Hkv, D, 64, 32, lens, [[n // 5, n // 2] for n in lens])
    out, mass = call(ctx, c)
    assert ctx.device_status() == 0
    check(c, out, mass, [0, 11, 23])


@pytest.mark.parametrize("B", [1, 5])
def test_nothing_but_empty_places(ctx, B):
    c = make(7, B, 3, 8, 2, 128, 32, 32, [0] * B, [[0, 10]] * B, capacity=320)
    out, mass = call(ctx, c)
    assert ctx.device_status() == 0
    assert (out == 0).all() and (mass == 0).all()


def test_pages_that_sequences_share(ctx):
    """A common prompt: the first pages of all sequences are the same ones; and one page twice in a sequence."""
    c = make(9, 4, 2, 8, 2, 128, 64, 16, [700, 650, 420, 300], [[10, 500], [0, 300], [3, 90], [64, 128]])
    for b in (1, 2, 3):
        c["table"][b, :4] = c["table"][0, :4]
    c["table"][0, 6] = c["table"][0, 5]
    out, mass = call(ctx, c)
    assert ctx.device_status() == 0
    check(c, out, mass)


def test_calls_one_behind_the_other(ctx):
    """Different shapes on one context without waiting in between: as each alone."""
    import torch
    from paper_2604_05650_b200 import binding
    cases = [make(1, 2, 8, 10, 2, 128, 128, 64, [5000, 2600], [[10, 2000]] * 2), make(2, 40, 1, 8, 8, 64, 16, 16, [333] * 40, [[3, 200]] * 40),
             make(3, 1, 16, 8, 1, 128, 64, 64, [9000], [[100, 8000]]), make(4, 1, 1, 4, 4, 128, 32, 32, [65], [[0, 60]])]
    alone = [call(ctx, c) for c in cases]
    jobs = []
    for c in cases:
        B, gamma, Hq, D = c["q"].shape
        t = [c["q"].cuda()] + [torch.from_numpy(np.ascontiguousarray(c[n])).cuda() for n in ("k", "v", "ks", "vs")] + \
            [torch.from_numpy(c["table"].astype(np.int32)).cuda(), torch.tensor(c["kv_len"], dtype=torch.int32).cuda(),
             torch.from_numpy(c["span"]).cuda()]
        results = [(torch.full((B, gamma, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda"),
                    torch.full((B, gamma, Hq), float("nan"), device="cuda")) for _ in range(12)]
        jobs.append((binding.attn_shape(B, gamma, Hq, c["k"].shape[1], D, c["capacity"]),
                     binding.paged_fp8(c["page"], len(c["k"]), c["block"]), t, results))
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for i in range(12):
        for shape, cache, t, results in jobs:
            ctx.verify_attention_paged_fp8(shape, cache, *t, *results[i])
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    for (_, _, _, results), want in zip(jobs, alone):
        for got in results:
            assert same(want, got)


@pytest.mark.parametrize("gamma,Hq,branches,D,lens", [(4, 8, 1, 128, [700, 131]), (8, 20, 2, 128, [128, 1290]), (16, 16, 1, 64, [300, 16]),
                                                     (10, 16, 1, 128, [2000, 1030]), (64, 4, 4, 128, [64, 200]), (1, 8, 1, 128, [77, 900])])
def test_nan_in_draft_slots(ctx, gamma, Hq, branches, D, lens):
    """A NaN code of K or V in a draft slot: the queries that see the slot give NaN, the others what they give without it."""
    import torch
    c = make(gamma * 3 + D, 2, gamma, Hq, 2, D, 64, 64, lens, [[n // 5, n // 2] for n in lens])
    c["branches"] = branches
    clean = call(ctx, c)
    check(c, *clean)
    for kind in ("v", "k"):
        for b, slot in ((0, gamma - 1), (1, gamma // 2)):
            spoiled = {**c, kind: c[kind].copy()}
            pos = lens[b] - gamma + slot
            spoiled[kind][c["table"][b, pos // 64], 1, pos % 64, 37] = 0xFF
            out, mass = call(ctx, spoiled)
            assert ctx.device_status() == 0
            bl = gamma // branches
            for g in range(gamma):
                sees = slot <= g and slot // bl == g // bl
                mine, theirs = out[b, g, Hq // 2:], out[b, g, :Hq // 2]
                assert torch.equal(theirs, clean[0][b, g, :Hq // 2]) and torch.equal(mass[b, g, :Hq // 2], clean[1][b, g, :Hq // 2])
                if not sees:
                    assert torch.equal(mine, clean[0][b, g, Hq // 2:]) and torch.equal(mass[b, g, Hq // 2:], clean[1][b, g, Hq // 2:])
                elif kind == "v" and gamma == 1:
                    assert torch.isnan(mine[:, 37]).all() and torch.isfinite(mine[:, :37]).all()
                else:
                    assert torch.isnan(mine).all()
                    assert torch.isnan(mass[b, g, Hq // 2:]).all() == (kind == "k")
            assert torch.equal(out[1 - b], clean[0][1 - b]) and torch.equal(mass[1 - b], clean[1][1 - b])


def test_nan_of_v_before_the_drafts_stays_in_its_channel(ctx):
    import torch
    c = make(5, 1, 4, 8, 2, 128, 64, 64, [700], [[10, 600]])
    clean = call(ctx, c)
    c["v"] = c["v"].copy()
    c["v"][c["table"][0, 695 // 64], 0, 695 % 64, 37] = 0x7F
    out, mass = call(ctx, c)
    keep = [ch for ch in range(128) if ch != 37]
    assert torch.isnan(out[0, :, :4, 37]).all() and torch.equal(out[0, :, :4, keep], clean[0][0, :, :4, keep])
    assert torch.equal(out[0, :, 4:], clean[0][0, :, 4:]) and torch.equal(mass, clean[1])
