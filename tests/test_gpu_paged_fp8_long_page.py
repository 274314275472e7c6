"""lvspec_verify_attention_paged_fp8 on one page as long as a pool may be (2^31 - 128 positions, 128 GiB, K and V the same):
as on short pages."""
import pytest

from test_gpu_paged_fp8 import check, ctx, make                           # noqa: F401

pytestmark = pytest.mark.gpu


def test_the_longest_page(ctx):                                  # noqa: F811
    import torch
    from paper_2604_05650_b200 import binding
    page, D, L = (1 << 31) - 128, 64, 700
    if torch.cuda.mem_get_info()[0] < page * D + (8 << 30):
        pytest.skip("needs 136 GiB of free device memory")
    c = make(81, 1, 2, 4, 1, D, 128, 128, [L], [[10, 600]])
    c["v"], c["vs"] = c["k"], c["ks"]
    pool = torch.empty(page * D, dtype=torch.uint8, device="cuda")
    n_tiles = -(-L // 128)
    order = c["table"][0, :n_tiles]
    pool[:n_tiles * 128 * D] = torch.from_numpy(c["k"][order, 0].reshape(-1)).cuda()
    scale = torch.full((page // 128,), float("nan"), device="cuda")
    scale[:n_tiles] = torch.from_numpy(c["ks"][order, 0, 0]).cuda()
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")          # noqa: E731
    out, mass = torch.full((1, 2, 4, D), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((1, 2, 4), float("nan"), device="cuda")
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    ctx.verify_attention_paged_fp8(binding.attn_shape(1, 2, 4, 1, D, page), binding.paged_fp8(page, 1, 128), c["q"].cuda(), pool, pool, scale,
                                   scale, i32(0), i32(L), i32(10, 600), out, mass, max_kv_len=1 << 30)
    torch.cuda.synchronize()
    assert ctx.device_status() == 0
    check(c, out, mass)
    del pool
    torch.cuda.empty_cache()                                                    # (the tests after this one need room)
