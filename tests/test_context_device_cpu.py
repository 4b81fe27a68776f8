"""A context lies on its stream's GPU whatever GPU is current, and stays there (no GPU: the
library's two entry points and torch's device switch are stand-ins that record)."""
import contextlib
import os
import types

import pytest

import workload as W


@pytest.fixture()
def recorded(monkeypatch):
    from paper_2609_38984_amd import swam
    if not os.path.exists(swam.LIB_PATH):
        from paper_2609_38984_amd.build import build
        build()
    real = swam.load_library()
    state = types.SimpleNamespace(current=0, created=[], moved=[])

    @contextlib.contextmanager
    def device(index):
        before, state.current = state.current, index
        yield
        state.current = before

    class Library:
        def __getattr__(self, name):
            return getattr(real, name)

        def swam_create(self, cfg, stream, out):
            state.created.append((state.current, stream.value))
            return 0

        def swam_set_stream(self, h, stream):
            state.moved.append(stream.value)
            return 0

    monkeypatch.setattr(swam, "load_library", lambda: Library())
    monkeypatch.setattr(swam.torch.cuda, "device", device)
    return state


def stream(index, value):
    return types.SimpleNamespace(device=types.SimpleNamespace(index=index), cuda_stream=value)


def test_the_workspace_is_on_the_streams_gpu(recorded):
    from paper_2609_38984_amd import swam
    for index in (0, 1, 3):
        ctx = swam.Context(W.preset(1), stream(index, 64 + index))
        assert ctx.device == index and recorded.created[-1] == (index, 64 + index)
        assert recorded.current == 0


def test_a_context_does_not_move_to_another_gpu(recorded):
    from paper_2609_38984_amd import swam
    ctx = swam.Context(W.preset(1), stream(1, 64))
    first = ctx.stream
    with pytest.raises(ValueError, match="GPU 0.*on 1"):
        ctx.set_stream(stream(0, 65))
    assert ctx.stream is first and recorded.moved == []
    ctx.set_stream(stream(1, 66))
    assert recorded.moved == [66] and ctx.stream.cuda_stream == 66
