"""Scratch memory that grows after a call has been captured: the graph goes on with the buffer that it holds."""
import numpy as np
import pytest

from test_gpu_paged_fp8 import call, check, make

pytestmark = pytest.mark.gpu


def fresh():
    import torch
    from paper_2604_05650_b200 import binding
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return binding.Context(0)


def test_a_captured_step_outlives_the_growth():
    import torch
    from paper_2604_05650_b200 import binding
    ctx = fresh()
    try:
        B, gamma, Hq, Hkv, D, page = 2, 2, 8, 2, 128, 64
        c = make(71, B, gamma, Hq, Hkv, D, page, 32, [3000, 1700], [[10, 2000], [0, 900]])
        shape, cache = binding.attn_shape(B, gamma, Hq, Hkv, D, c["capacity"]), binding.paged_fp8(page, len(c["k"]), 32)
        dev = [c["q"].cuda()] + [torch.from_numpy(np.ascontiguousarray(c[n])).cuda() for n in ("k", "v", "ks", "vs")] + \
            [torch.from_numpy(c["table"].astype(np.int32)).cuda(), torch.tensor(c["kv_len"], dtype=torch.int32).cuda(),
             torch.from_numpy(c["span"]).cuda()]
        out = torch.full((B, gamma, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        mass = torch.full((B, gamma, Hq), float("nan"), device="cuda")
        need = ctx.attention_paged_fp8_workspace_bytes(shape)
        cap = ctx.workspace_capacity()
        assert 0 < need <= cap
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            ctx.set_stream(torch.cuda.current_stream().cuda_stream)
            ctx.verify_attention_paged_fp8(shape, cache, *dev, out, mass)
        ctx.set_stream(stream.cuda_stream)
        graph.replay()
        torch.cuda.synchronize()
        check(c, out, mass)
        first = out.clone(), mass.clone()
        # ---- grown twice, by a call of 128 rows and ahead of one; what would lie in memory given back is written over
        held = [cap]
        for step in range(2):
            if step == 0:
                big = make(72, 1, 16, 8, 1, D, 128, 128, [3000], [[0, 600]])
                check(big, *call(ctx, big))
            else:
                ctx.reserve(held[-1] + 1)
            held.append(ctx.workspace_capacity())
            assert held[-1] >= 2 * held[-2]                     # (what is kept stays below what is in use)
            junk = [torch.full((held[0] // 4,), float("nan"), device="cuda") for _ in range(4)]
            out.fill_(float("nan"))
            mass.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert ctx.device_status() == 0
            assert torch.equal(out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(mass, first[1])
            assert all(bool(torch.isnan(t).all()) for t in junk)
            del junk
    finally:
        ctx.set_stream(None)
        ctx.close()
