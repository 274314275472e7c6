"""Decoding steps on a paged fp8 cache as a serving loop runs them: pages for the new tokens, their K and V into the cache, the
attention of every layer, the acceptance rule and the tokens sampled, on one stream with nothing read back between the calls.
Everything is compared with the reference after each step: tables, lengths, codes, scales and decisions exactly."""
import numpy as np
import pytest

from oracle import paged_step as ref
from test_gpu_paged_fp8 import bf16
from test_gpu_paged_fp8_cases import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("B,gamma,Hq,Hkv,D,page,block", [(5, 4, 8, 2, 128, 16, 16), (3, 8, 10, 1, 64, 64, 32), (9, 1, 4, 4, 128, 128, 64)])
def test_steps(oracle_mod, captured, B, gamma, Hq, Hkv, D, page, block):
    import torch
    from paper_2604_05650_b200 import binding
    layers, V, n_steps, longest = 2, 999, 5, 300
    per_seq = -(-(longest + n_steps * gamma) // page) + 1
    n_pages = B * per_seq
    rng = np.random.default_rng(B * 100 + gamma)
    ctx = binding.Context(0)
    try:
        # ---- the loop's state: of the reference, and on the device
        kv_len, held, n_free = [0] * B, [0] * B, n_pages
        free = rng.permutation(n_pages).astype(np.int64)
        table = np.full((B, per_seq), -1, np.int64)
        pools = [[np.full((n_pages, Hkv, page, D), 0x7F, np.uint8) for _ in range(2)] for _ in range(layers)]
        scales = [[np.full((n_pages, Hkv, page // block), np.nan, np.float32) for _ in range(2)] for _ in range(layers)]
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()                     # noqa: E731
        d_len, d_held, d_free_n, d_free, d_table = i32(kv_len), i32(held), i32([n_free]), i32(free), i32(table)
        d_new, d_start, d_slots = i32([0] * B), i32([-5] * (B + 1)), i32([-5] * (longest * B))
        d_pools = [[torch.from_numpy(x).cuda() for x in layer] for layer in pools]
        d_scales = [[torch.from_numpy(x).cuda() for x in layer] for layer in scales]
        span = np.asarray([[3, 40 + b] for b in range(B)], np.int32)
        d_span = i32(span)
        n = B * gamma
        d_kv = [torch.zeros(longest * B, 2, Hkv, D, dtype=torch.bfloat16, device="cuda") for _ in range(layers)]
        d_q = [torch.zeros(B, gamma, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(layers)]
        out = [torch.full((B, gamma, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(layers)]
        mass = [torch.full((B, gamma, Hq), float("nan"), device="cuda") for _ in range(layers)]
        d_logits = torch.zeros(B, gamma, V, device="cuda")
        d_draft, d_next = i32(np.zeros((B, gamma))), i32(np.zeros((B, gamma)))
        d_T, d_p, d_u, d_prob = (torch.zeros(n, device="cuda") for _ in range(4))
        d_k = i32([0] * n)
        d_tau, d_emitted, d_count = i32([0] * B), i32(np.zeros((B, gamma))), i32([0] * B)
        d_grown = i32([0] * B)
        cache = binding.paged_fp8(page, n_pages, block)
        shape = binding.attn_shape(B, gamma, Hq, Hkv, D, per_seq * page)
        ctx.reserve(ctx.attention_paged_fp8_workspace_bytes(shape) + ctx.accept_workspace_bytes(B, gamma, V))

        def pages_and_rows(max_new):
            ctx.plan_pages(B, page, per_seq, n_pages, max_new, d_len, d_new, d_held, d_free_n, d_free, d_table, d_grown, d_held, d_free_n,
                           d_start, d_slots)
            for rows, pool, scale in zip(d_kv, d_pools, d_scales):
                ctx.append_paged_fp8(max_new, Hkv, D, cache, rows[:, 0], rows[:, 1], 2 * Hkv * D, 2 * Hkv * D, d_slots, *pool, *scale)

        def decode():
            pages_and_rows(n)
            for i in range(layers):
                ctx.verify_attention_paged_fp8(shape, cache, d_q[i], *d_pools[i], *d_scales[i], d_table, d_grown, d_span, out[i], mass[i])
            ctx.loose_accept_emit(B, gamma, V, Hq, d_logits, d_draft, mass[-1], d_tau, d_emitted, d_count, 1, lam=0.5, kv_len=d_grown,
                                  new_kv_len=d_len)
            ctx.sample(n, V, d_logits, d_T, d_k, d_p, None, d_u, d_next, d_prob)

        def reference_pages(new, rows):
            """rows [layer][token, K or V, Hkv, D] fp64"""
            nonlocal table, held, n_free
            table, grown, held, n_free, starts, slots, refused = ref.plan_pages(page, per_seq, n_pages, sum(new), kv_len, new, held, n_free,
                                                                                free, table)
            assert not refused
            for i in range(layers):
                for side in range(2):
                    pools[i][side], scales[i][side] = ref.append(rows[i][:, side], slots, pools[i][side], scales[i][side], page, block)
            return grown

        def cache_is_right():
            assert (d_table.cpu().numpy() == table).all() and d_held.tolist() == held and int(d_free_n) == n_free
            for i in range(layers):
                for side in range(2):
                    assert (d_pools[i][side].cpu().numpy() == pools[i][side]).all()
                    np.testing.assert_array_equal(d_scales[i][side].cpu().numpy(), scales[i][side])

        # ---- the prompts
        ctx.set_stream(torch.cuda.current_stream().cuda_stream)
        new = [int(x) for x in rng.integers(gamma + 1, longest, B)]
        new[0] = longest - 1
        rows = [bf16(rng.standard_normal((sum(new), 2, Hkv, D)) * (1 + 30 * i)) for i in range(layers)]
        for t, r in zip(d_kv, rows):
            t[:sum(new)] = r.cuda()
        d_new.copy_(i32(new))
        torch.cuda.synchronize()
        before = ctx.launch_count()
        pages_and_rows(sum(new))
        assert ctx.launch_count() == before + 1 + layers
        torch.cuda.synchronize()
        kv_len = reference_pages(new, [r.float().numpy().astype(np.float64) for r in rows])
        cache_is_right()
        d_len.copy_(d_grown)
        new = [gamma] * B
        d_new.copy_(i32(new))
        if captured:
            stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph, stream=stream):
                ctx.set_stream(torch.cuda.current_stream().cuda_stream)
                decode()
            ctx.set_stream(stream.cuda_stream)

        # ---- the steps
        taken = set()
        for step in range(n_steps):
            rows = [bf16(rng.standard_normal((n, 2, Hkv, D)) * (1 + 30 * i) * 2.0 ** (step - 2)) for i in range(layers)]
            q = [bf16(rng.standard_normal((B, gamma, Hq, D)) / (1 + 30 * i)) for i in range(layers)]
            logits = rng.standard_normal((B, gamma, V)).astype(np.float32) * 3
            draft = rng.integers(0, V, (B, gamma)).astype(np.int32)
            right = rng.random((B, gamma)) < 0.7
            draft[right] = logits.argmax(-1)[right]
            T = rng.choice([0.0, 0.7, 1.3], n).astype(np.float32)
            k, p, u = rng.choice([0, 5, 50], n).astype(np.int32), rng.choice([0.8, 1.0], n).astype(np.float32), rng.random(n).astype(np.float32)
            for dst, src in zip(d_kv + d_q, rows + q):
                dst[:len(src)] = src.cuda()
            for dst, src in ((d_logits, logits), (d_draft, draft), (d_T, T), (d_k, k), (d_p, p), (d_u, u)):
                dst.copy_(torch.from_numpy(src))
            torch.cuda.synchronize()
            if captured:
                graph.replay()
            else:
                decode()
            torch.cuda.synchronize()
            assert ctx.device_status() == 0

            grown = reference_pages(new, [r.float().numpy().astype(np.float64) for r in rows])
            cache_is_right()
            assert d_grown.tolist() == grown
            for i in range(layers):
                check(dict(q=q[i], k=pools[i][0], v=pools[i][1], ks=scales[i][0], vs=scales[i][1], table=table, kv_len=grown, span=span,
                           page=page, block=block, branches=1, capacity=per_seq * page), out[i], mass[i])
            tau, target, _ = oracle_mod.loose_accept(logits, draft, mass[-1].cpu().numpy(), oracle_mod.n_loose(0.5, gamma), 1)
            emitted, count, kept = oracle_mod.emit(draft, target, tau, np.asarray(grown, np.int32))
            assert d_tau.tolist() == tau.tolist() and (d_emitted.cpu().numpy() == emitted).all()
            assert d_count.tolist() == count.tolist() and d_len.tolist() == kept.tolist()
            got = d_next.cpu().numpy().reshape(-1)
            for r in range(n):
                want, prob, margin = ref.sample(logits.reshape(n, V)[r], float(T[r]), int(k[r]), float(p[r]), 0.0, float(u[r]))
                if margin > 1e-5 and (T[r] <= 0 or clear(logits.reshape(n, V)[r], float(T[r]), int(k[r]), float(p[r]))):
                    assert got[r] == want
                    assert abs(float(d_prob[r]) - prob) <= 1e-5 * prob + 1e-7
            kv_len = [int(x) for x in kept]
            taken.update(tau.tolist())
        assert len(taken) > 1 or gamma == 1           # (lengths moved by different amounts)
    finally:
        ctx.set_stream(None)
        ctx.close()


def clear(row, T, k, p):
    """top_p's border falls between two tokens, not within rounding of one."""
    if p >= 1:
        return True
    kept, w = ref.kept_tokens(row, T, k, 1.0, 0.0)
    shares = np.cumsum([w[i] for i in kept]) / sum(w[i] for i in kept)
    return np.abs(shares - p).min() > 1e-6
