"""Context.set_stream reaches the library at every call, as far as that shows without a GPU: a stream set through the C call in between
is not taken for the one set before, and a context that has been closed says so."""
import types

import pytest

from paper_2604_05650_b200 import binding, build


@pytest.fixture(params=["converted here", "by ctypes"])
def way(request, monkeypatch):
    build.build_marshal()
    binding.load_library()
    assert binding._fast is not None
    if request.param == "by ctypes":
        monkeypatch.setattr(binding, "_fast", None)
    return request.param


def context(lib):
    """A context without a device behind it."""
    ctx = binding.Context.__new__(binding.Context)
    ctx._lib, ctx._h, ctx._handle = lib, None, None
    return ctx


@pytest.mark.parametrize("stream", [0, None, 4096, types.SimpleNamespace(cuda_stream=0), types.SimpleNamespace(cuda_stream=4096)])
def test_a_closed_context(way, stream):
    ctx = context(binding.load_library())
    for _ in range(2):
        with pytest.raises(binding.LvspecError) as e:
            ctx.set_stream(stream)
        assert e.value.status == binding.ERR_INVALID_ARG


def test_every_call_is_made(way, monkeypatch):
    made = []
    ctx = context(types.SimpleNamespace(lvspec_set_stream=lambda h, s: made.append(s.value or 0) or 0))
    if binding._fast is not None:
        monkeypatch.setattr(binding, "_fast", types.SimpleNamespace(set_stream=lambda h, s: made.append(s) or 0))
    for stream in (0, 0, 4096, 4096, types.SimpleNamespace(cuda_stream=4096), None, None):
        ctx.set_stream(stream)
    assert made == [0, 0, 4096, 4096, 4096, 0, 0]
