"""lvspec_verify_attention_fp8 with queries at the ends of bf16's range and K scales at the other end, so that scores are ordinary: the
oracle and the tolerances of test_gpu_fp8."""
import numpy as np
import pytest

from paper_2604_05650_b200 import workloads as W
from test_gpu_fp8 import _case, _check, ctx                                     # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [-118, -113, -104, 104, 113, 120, 124])
def test_ends_of_qs_range(ctx, oracle_mod, power):                              # noqa: F811
    q, k8, v8, ks, vs, kv_len, span = _case(9, 2, 8, 8, 2, 700, [700, 389], [[10, 500], [0, 381]])
    values = (np.asarray(q, np.uint16).astype(np.uint32) << 16).view(np.float32)
    q = W.f32_to_bf16_bits(values * np.float32(2.0 ** power))
    ks = (ks.astype(np.float64) * 2.0 ** -power).astype(np.float32)
    assert np.isfinite(ks).all() and (ks > 0).all()
    _check(ctx, oracle_mod, (q, k8, v8, ks, vs, kv_len, span))
