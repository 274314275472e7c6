"""The fp64 reference of the decoding step on a paged fp8 cache, pinned: hand-worked page
tables, torch's E4M3 conversion, and the contiguous oracle's attention."""
import numpy as np
import pytest
import torch

from oracle import paged_step as ref
from paper_2604_05650_b200 import workloads as W


def test_encoding_is_torchs():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(20000) * 10.0 ** rng.uniform(-4, 2.5, 20000), ref.DECODE[np.isfinite(ref.DECODE)],
                        (ref._VALUES[1:] + ref._VALUES[:-1]) / 2, [449.0, -1e9, np.inf, 0.0, -0.0]]).astype(np.float32)
    want = torch.from_numpy(x).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert (ref.e4m3_encode(x) == want).all()
    assert ref.e4m3_encode(np.nan) == 0x7F


def test_pages_by_hand():
    # pages of 4; request 0 holds 6 positions in pages 9, 3 and takes 3 more: one page; request 1 is new with 5: two
    # pages; request 2 holds 4 in page 7 and asks for nothing; request 3 wants more pages than are left
    table = np.full((4, 4), -1)
    table[0, :2], table[2, 0] = (9, 3), 7
    free = [5, 1, 8, 2, 0, 0, 0, 0, 0, 0]
    got = ref.plan_pages(4, 4, 10, 18, [6, 0, 4, 0], [3, 5, 0, 8], [2, 0, 1, 0], 4, free, table)
    table, lens, held, n_free, starts, slots, refused = got
    assert table[0].tolist() == [9, 3, 2, -1] and table[1].tolist() == [8, 1, -1, -1]
    assert lens == [9, 5, 4, 0] and held == [3, 2, 1, 0] and n_free == 1 and refused
    assert starts == [0, 3, 8, 8, 16]
    assert slots == [14, 15, 8, 32, 33, 34, 35, 4] + [-1] * 10


def test_scale_is_the_smallest_power_of_two_and_never_falls():
    pool, scale = np.zeros((1, 1, 16, 64), np.uint8), np.zeros((1, 1, 1), np.float32)
    one = lambda v: np.full((1, 1, 64), v, np.float64)   # noqa: E731
    pool, scale = ref.append(one(448.0), [0], pool, scale, 16, 16)
    assert scale.item() == 1.0 and (pool[0, 0, 0] == 0x7E).all()
    pool, scale = ref.append(one(450.0), [1], pool, scale, 16, 16)
    assert scale.item() == 2.0 and (ref.DECODE[pool[0, 0, 0]] == 224).all() and (ref.DECODE[pool[0, 0, 1]] == 224).all()
    pool, scale = ref.append(one(1.0), [2], pool, scale, 16, 16)
    assert scale.item() == 2.0 and (ref.DECODE[pool[0, 0, 2]] == 0.5).all()
    pool, scale = ref.append(one(0.0), [0], pool, scale, 16, 16)      # the block begins anew
    assert scale.item() == np.float32(2.0 ** -100)


@pytest.mark.parametrize("block", [16, 64])
def test_attention_is_the_contiguous_oracles(oracle_mod, block):
    rng = np.random.default_rng(3)
    B, gamma, Hq, Hkv, L, page = 2, 3, 4, 2, 192, 64
    q = W.f32_to_bf16_bits(rng.standard_normal((B, gamma, Hq, 64)).astype(np.float32))
    k8, v8 = (ref.e4m3_encode(rng.standard_normal((B, Hkv, L, 64)) * 100) for _ in range(2))
    ks, vs = (rng.uniform(0.005, 0.02, (B, Hkv)).astype(np.float32) for _ in range(2))
    kv_len, span = np.asarray([192, 70], np.int32), np.asarray([[10, 150], [0, 67]], np.int32)
    want = oracle_mod.verify_attention_fp8(q, k8, v8, ks, vs, kv_len, span)
    order = rng.permutation(B * L // page).reshape(B, L // page)
    pools = []
    for c in (k8, v8):
        pool = np.zeros((B * L // page, Hkv, page, 64), np.uint8)
        for b in range(B):
            for j in range(L // page):
                pool[order[b, j]] = c[b, :, j * page:(j + 1) * page]
        pools.append(pool)
    scales = []
    for s in (ks, vs):
        sc = np.zeros((B * L // page, Hkv, page // block), np.float32)
        for b in range(B):
            sc[order[b]] = s[b][None, :, None]
        scales.append(sc)
    qf = (q.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    got = ref.attention(qf, *pools, *scales, order, kv_len, span, block)
    assert np.abs(got[0] - want[0]).max() < 1e-12 and np.abs(got[1] - want[1]).max() < 1e-12


def test_a_query_that_sees_nothing_gives_zeros():
    q = np.ones((2, 4, 1, 64))
    pool, scale = np.full((1, 1, 16, 64), 0x38, np.uint8), np.ones((1, 1, 1), np.float32)
    out, mass = ref.attention(q, pool, pool, scale, scale, [[0], [0]], [2, 0], [[0, 1], [0, 0]], 16)
    assert (out[0, :2] == 0).all() and (out[0, 2:] == 1).all() and (out[1] == 0).all()
    assert mass[0, :, 0].tolist() == [0, 0, 1, 0.5]


def test_sampling_by_hand():
    l = np.log([0.1, 0.4, 0.2, 0.2, 0.1])
    assert ref.kept_tokens(l, 1.0, 3, 1.0, 0.0)[0] == [1, 2, 3]
    assert ref.kept_tokens(l, 1.0, 0, 0.55, 0.0)[0] == [1, 2]
    assert ref.kept_tokens(l, 1.0, 2, 0.67, 0.0)[0] == [1, 2]              # 0.4 of 0.6 is below 0.67
    assert ref.kept_tokens(l, 1.0, 2, 0.66, 0.0)[0] == [1]
    assert ref.kept_tokens(l, 1.0, 0, 1.0, 0.45)[0] == [1, 2, 3]
    assert ref.kept_tokens(l, 0.5, 0, 1.0, 0.3)[0] == [1]                  # the square of a half
    assert ref.kept_tokens(l, 1.0, 0, 0.0, 0.0)[0] == [1]
    assert [ref.sample(l, 1.0, 0, 1.0, 0.0, u)[0] for u in (0.0, 0.05, 0.15, 0.55, 0.75, 0.95)] == [0, 0, 1, 2, 3, 4]
    assert ref.sample(l, 0.0, 0, 1.0, 0.0, 0.9)[:2] == (1, 1.0)
    assert ref.sample([np.nan, -np.inf, np.nan], 1.0, 0, 1.0, 0.0, 0.9)[0] == 0
    token, prob, _ = ref.sample(l, 1.0, 3, 1.0, 0.0, 0.6)
    assert token == 2 and abs(prob - 0.25) < 1e-12
