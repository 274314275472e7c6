"""The calls of a decoding step on a paged fp8 cache, as far as they go without a GPU: the library's exports, the
description's layout, the header's numbers, and a null context, which every call answers."""
import ctypes
import os
import re

import pytest

from paper_2604_05650_b200 import binding

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "lvspec.h")


def test_description_of_a_cache():
    assert ctypes.sizeof(binding.PagedFp8) == 40 and binding.PagedFp8.page_stride.offset == 16
    c = binding.paged_fp8(64, 9, 16, 4096, 2048, 128)
    assert (c.page_size, c.n_pages, c.scale_block, c.reserved, c.page_stride, c.head_stride, c.position_stride) == (64, 9, 16, 0, 4096, 2048, 128)
    c = binding.paged_fp8(64, 9, 16)
    assert (c.page_stride, c.head_stride, c.position_stride) == (0, 0, 0)


def test_numbers_of_the_header():
    text = open(HEADER).read()
    value = lambda name: int(re.search(rf"#define {name}\s+(0x[0-9a-f]+|\d+)", text).group(1), 0)      # noqa: E731
    assert value("LVSPEC_DEV_REFUSED") == binding.DEV_REFUSED and value("LVSPEC_DEV_BAD_LENGTH") == binding.DEV_BAD_LENGTH
    assert (value("LVSPEC_DTYPE_F32"), value("LVSPEC_DTYPE_BF16")) == (0, 1)
    assert value("LVSPEC_MAX_REQUESTS") == 1024 and value("LVSPEC_MAX_SAMPLE_VOCAB") == 400000


@pytest.mark.parametrize("name", ["lvspec_plan_pages", "lvspec_append_paged_fp8", "lvspec_verify_attention_paged_fp8", "lvspec_sample"])
def test_a_null_context(name):
    call = getattr(binding.load_library(), name)
    assert call(*[None if a in (ctypes.c_void_p,) or issubclass(a, ctypes._Pointer) else 1 for a in call.argtypes]) == binding.ERR_INVALID_ARG


def test_a_null_context_needs_no_workspace():
    shape = binding.attn_shape(1, 1, 1, 1, 128, 128)
    assert binding.load_library().lvspec_attention_paged_fp8_workspace_bytes(None, ctypes.byref(shape)) == 0


class Tensor:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


def test_arguments_without_ctypes():
    """The module that converts the arguments, on a null context: every kind of argument, and what it refuses."""
    import numpy as np
    from paper_2604_05650_b200 import build
    build.build_marshal()
    binding.load_library()
    fast = binding._fast
    assert fast is not None
    for pointer in (None, 0, 1 << 63, Tensor(4096), np.zeros(3, np.int32)):
        assert fast.plan_pages(None, 1, np.int64(2), True, 4, 5, *[pointer] * 11) == binding.ERR_INVALID_ARG
        assert fast.sample(0, 1, 2, False, pointer, 4, *[pointer] * 7) == binding.ERR_INVALID_ARG
    cache, shape = binding.paged_fp8(16, 1, 16), binding.attn_shape(1, 1, 1, 1, 128, 128)
    assert fast.append_paged_fp8(None, 1, 1, 64, cache, None, None, 1 << 40, 1, *[None] * 5) == binding.ERR_INVALID_ARG
    assert fast.verify_attention_paged_fp8(None, shape, cache, 1, 1, *[None] * 10) == binding.ERR_INVALID_ARG
    for error, call in ((TypeError, lambda: fast.plan_pages(None, 1)), (TypeError, lambda: fast.sample(None, 1, 2, None, *[None] * 9)),
                        (AttributeError, lambda: fast.plan_pages(None, 1, 1, 1, 1, 1, "x", *[None] * 10)),
                        (OverflowError, lambda: fast.plan_pages(None, 1, 1, 1, 1, 1, -1, *[None] * 10)),
                        (TypeError, lambda: fast.append_paged_fp8(None, 1, 1, 64, shape, None, None, 1, 1, *[None] * 5)),
                        (TypeError, lambda: fast.verify_attention_paged_fp8(None, None, cache, 1, 1, *[None] * 10))):
        with pytest.raises(error):
            call()
