"""lvspec_plan_pages and lvspec_append_paged_fp8: what they refuse, before anything is launched or written."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2604_05650_b200 import binding
    c = binding.Context(0)
    yield c
    c.close()


def test_plan(ctx):
    import torch
    from paper_2604_05650_b200 import binding
    names = ("lens", "new", "held", "n_free", "free", "table", "new_lens", "new_held", "new_free", "start", "slots")
    t = {x: torch.full((64,), 3, dtype=torch.int32, device="cuda") for x in names}
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    before = ctx.launch_count()
    bad = [dict(B=0), dict(B=1025), dict(page=0), dict(per_seq=0), dict(n_pages=0), dict(max_new=-1), dict(n_pages=2 ** 27),
           dict(per_seq=2 ** 27)]
    bad += [{x: None} for x in names] + [{x: t[x].data_ptr() + 2} for x in names] + [dict(slots=t["slots"].data_ptr() + 4)]
    for change in bad:
        a = {**dict(B=2, page=16, per_seq=4, n_pages=8, max_new=8), **t, **change}
        with pytest.raises(binding.LvspecError) as e:
            ctx.plan_pages(a["B"], a["page"], a["per_seq"], a["n_pages"], a["max_new"], *(a[x] for x in names))
        assert e.value.status == binding.ERR_INVALID_ARG, change
    torch.cuda.synchronize()
    assert ctx.launch_count() == before and all((x == 3).all() for x in t.values())
    # without new tokens there is no slot map
    ctx.plan_pages(2, 16, 4, 8, 0, *(t[x] for x in names[:-1]), None)
    torch.cuda.synchronize()
    assert ctx.device_status() == binding.DEV_REFUSED         # (each asks for three)


def test_append(ctx):
    import torch
    from paper_2604_05650_b200 import binding
    x = torch.ones(4, 2, 128, dtype=torch.bfloat16, device="cuda")
    pool = torch.full((8, 2, 128, 128), 3, dtype=torch.uint8, device="cuda")
    scale = torch.full((8, 2, 2), 5.0, device="cuda")
    slots = torch.arange(4, dtype=torch.int32, device="cuda")
    ctx.set_stream(torch.cuda.current_stream().cuda_stream)
    before = ctx.launch_count()
    I, U = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    bad = [(I, dict(n=-1)), (I, dict(H=0)), (I, dict(H=65536)), (U, dict(D=32)), (U, dict(D=256)), (I, dict(page=40)), (I, dict(block=0)),
           (I, dict(page=16, block=32)), (I, dict(n_pages=0)), (I, dict(strides=(32768, 16384, 64))), (I, dict(strides=(32768, 16384, 136))),
           (I, dict(k_stride=255)), (I, dict(k_stride=260)), (I, dict(v_stride=248)), (I, dict(v_stride=2 ** 32))]
    bad += [(I, {name: None}) for name in ("k", "v", "slots", "kp", "vp", "ks", "vs")]
    bad += [(I, {name: t.data_ptr() + off}) for name, t, off in (("k", x, 8), ("v", x, 2), ("slots", slots, 1), ("kp", pool, 8), ("vp", pool, 4),
                                                                ("ks", scale, 2), ("vs", scale, 1))]
    for status, change in bad:
        a = {**dict(n=4, H=2, D=128, page=128, block=64, n_pages=8, strides=(0, 0, 0), k_stride=256, v_stride=256, k=x, v=x, slots=slots,
                    kp=pool, vp=pool, ks=scale, vs=scale), **change}
        with pytest.raises(binding.LvspecError) as e:
            ctx.append_paged_fp8(a["n"], a["H"], a["D"], binding.paged_fp8(a["page"], a["n_pages"], a["block"], *a["strides"]), a["k"], a["v"],
                                 a["k_stride"], a["v_stride"], a["slots"], a["kp"], a["vp"], a["ks"], a["vs"])
        assert e.value.status == status, change
    torch.cuda.synchronize()
    assert ctx.launch_count() == before and (pool == 3).all() and (scale == 5).all()
