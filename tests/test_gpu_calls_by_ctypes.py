"""The calls of a decoding step through ctypes, as where the module that converts their arguments has not been built: the same results
and the same refusals."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_step_and_its_refusals_either_way(monkeypatch):
    import torch
    from paper_2604_05650_b200 import binding
    ctx = binding.Context(0)
    assert binding._fast is not None
    try:
        ctx.set_stream(torch.cuda.current_stream().cuda_stream)
        g = torch.Generator("cuda").manual_seed(1)
        i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")                                   # noqa: E731
        rows = torch.randn(90, 2, 2, 64, generator=g, device="cuda").bfloat16()
        q = torch.randn(1, 2, 4, 64, generator=g, device="cuda").bfloat16()
        logits = torch.randn(3, 500, generator=g, device="cuda")
        cache, shape = binding.paged_fp8(16, 8, 16), binding.attn_shape(1, 2, 4, 2, 64, 128)

        def step():
            table, lens, held, free = i32(*[-1] * 8), i32(0), i32(0), i32(8)
            slots, start = torch.full((96,), -1, dtype=torch.int32, device="cuda"), i32(0, 0)
            ctx.plan_pages(1, 16, 8, 8, 90, lens, i32(90), held, free, i32(*range(8)), table, lens, held, free, start, slots)
            pools = [torch.zeros(8, 2, 16, 64, dtype=torch.uint8, device="cuda") for _ in range(2)]
            scales = [torch.zeros(8, 2, 1, device="cuda") for _ in range(2)]
            ctx.append_paged_fp8(90, 2, 64, cache, rows[:, 0], rows[:, 1], 256, 256, slots, *pools, *scales)
            out, mass = torch.zeros_like(q), torch.zeros(1, 2, 4, device="cuda")
            ctx.verify_attention_paged_fp8(shape, cache, q, *pools, *scales, table, lens, i32(3, 50), out, mass, max_kv_len=100)
            tokens, probs = i32(0, 0, 0), torch.zeros(3, device="cuda")
            ctx.sample(3, 500, logits, None, i32(5, 0, 50), None, None, torch.tensor([0.1, 0.5, 0.9], device="cuda"), tokens, probs)
            torch.cuda.synchronize()
            assert ctx.device_status() == 0
            return [table, lens, held, free, slots, start, *pools, *scales, out, mass, tokens, probs]

        def refusals():
            texts = []
            for call in (lambda: ctx.plan_pages(0, 16, 8, 8, 90, *[None] * 11), lambda: ctx.sample(1, 0, *[None] * 7),
                         lambda: ctx.append_paged_fp8(-1, 2, 64, cache, *[None] * 2, 256, 256, *[None] * 5),
                         lambda: ctx.verify_attention_paged_fp8(shape, cache, *[None] * 10)):
                with pytest.raises(binding.LvspecError) as e:
                    call()
                texts.append(str(e.value))
            return texts

        first, said = step(), refusals()
        monkeypatch.setattr(binding, "_fast", None)
        assert all(torch.equal(a, b) for a, b in zip(first, step())) and said == refusals()
        assert int(first[1]) == 90 and (first[10].float().abs().sum() > 0).item()
    finally:
        ctx.close()
