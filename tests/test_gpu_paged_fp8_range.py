"""lvspec_verify_attention_paged_fp8 with queries at the ends of bf16's range and K scales at the other end, so that scores are ordinary:
against the fp64 reference, with the tolerances of test_gpu_paged_fp8 (they hold for q of any magnitude: a power of two brings it
into the range that its two E4M3 terms have)."""
import numpy as np
import pytest

from test_gpu_paged_fp8 import bf16, call, check, ctx, make                     # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [-118, -113, -104, -90, 90, 104, 113, 120, 124])
def test_ends_of_qs_range(ctx, power):                                          # noqa: F811
    c = make(7, 2, 8, 8, 2, 128, 32, 32, [900, 131], [[64, 700], [0, 100]])
    c["q"] = bf16(c["q"].float().numpy() * np.float32(2.0 ** power))
    c["ks"] = (c["ks"].astype(np.float64) * 2.0 ** -power).astype(np.float32)
    assert np.isfinite(c["ks"]).all() and (c["ks"] > 0).all()
    out, mass = call(ctx, c)
    assert ctx.device_status() == 0
    check(c, out, mass)
