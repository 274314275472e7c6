"""Two contexts on two host threads, each on a stream of its own, with calls of different sizes of the same kernels: what one call asks of
a kernel is no limit to the other's."""
import threading

import pytest

pytestmark = pytest.mark.gpu


def both(work):
    """work(context, which) on two threads at once; an exception of either is raised."""
    import torch
    from paper_2604_05650_b200 import binding
    failed, start = [], threading.Barrier(2)

    def thread(which):
        try:
            ctx = binding.Context(0)
            try:
                with torch.cuda.stream(torch.cuda.Stream()):
                    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
                    work(ctx, which, start)
                    torch.cuda.current_stream().synchronize()
            finally:
                ctx.close()
        except BaseException as e:                                                       # noqa: BLE001
            failed.append(e)
            start.abort()

    threads = [threading.Thread(target=thread, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if failed:
        raise failed[0]


def test_sampling():
    """A target's and a draft model's vocabulary."""
    import torch

    def work(ctx, which, start):
        vocab = (152064, 4000)[which]
        logits = torch.zeros(2, vocab, device="cuda")
        logits[0, 77], logits[1, vocab - 1] = 5.0, 5.0
        u, T = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
        tokens = torch.full((2,), -1, dtype=torch.int32, device="cuda")
        start.wait(60)
        for i in range(4000):
            ctx.sample(2, vocab, logits, T, None, None, None, u, tokens)
            if i % 500 == 499:
                assert tokens.tolist() == [77, vocab - 1]

    both(work)


def test_attention():
    """Heads of 64 and of 128 channels."""
    import torch
    from paper_2604_05650_b200 import binding

    def work(ctx, which, start):
        D = (64, 128)[which]
        cache, shape = binding.paged_fp8(64, 4, 64), binding.attn_shape(1, 2, 4, 2, D, 256)
        pools = [torch.full((4, 2, 64, D), 0x38, dtype=torch.uint8, device="cuda") for _ in range(2)]       # (ones)
        scales = [torch.full((4, 2, 1), 2.0, device="cuda") for _ in range(2)]
        q = torch.ones(1, 2, 4, D, dtype=torch.bfloat16, device="cuda")
        table, lens, span = (torch.tensor(a, dtype=torch.int32, device="cuda") for a in ([0, 1, 2, 3], [200], [0, 100]))
        out, mass = torch.zeros_like(q), torch.zeros(1, 2, 4, device="cuda")
        start.wait(60)
        for i in range(4000):
            ctx.verify_attention_paged_fp8(shape, cache, q, *pools, *scales, table, lens, span, out, mass)
            if i % 500 == 499:
                assert (out == 2).all().item() and ctx.device_status() == 0

    both(work)
