"""Which stream the binding's calls allocate on and run on, without a GPU: CPU tensors, a library that
only records, and torch's current stream replaced by a name."""
import contextlib
import ctypes
import types

import pytest
import torch

from paper_1909_09010_b200 import binding

CALLER, SIDE = 11, 77


class Library:
    """Answers every call with OK and notes the stream it was given; every product wants a workspace."""

    def __init__(self, ran):
        self.ran = ran

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_workspace"):
                args[2]._obj.value = 4096
            elif "destroy" not in name:
                self.ran.append(args[-1])
            return binding.GBMUF_OK
        return call


@pytest.fixture
def world(monkeypatch):
    w = types.SimpleNamespace(current=CALLER, ran=[], made=[], recorded=[])

    @contextlib.contextmanager
    def within(stream):
        before, w.current = w.current, stream.cuda_stream
        yield
        w.current = before

    def watched(make):
        def made(*args, **kwargs):
            t = make(*args, **kwargs)
            w.made.append((t, w.current))
            return t
        return made

    stream_of = lambda handle, device=None: types.SimpleNamespace(                                   # noqa: E731
        cuda_stream=handle, device=types.SimpleNamespace(index=-1))
    monkeypatch.setattr(torch.cuda, "stream", within)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream_of(w.current))
    monkeypatch.setattr(torch.cuda, "ExternalStream", stream_of)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: w.recorded.append((t, s.cuda_stream)))
    monkeypatch.setattr(torch.Tensor, "new_empty", watched(torch.Tensor.new_empty))
    monkeypatch.setattr(torch, "empty", watched(torch.empty))
    w.side = stream_of(SIDE)
    for cls in (binding.LocalOps, binding.GradClip):
        o = cls.__new__(cls)
        o._torch, o._L, o._h, o.device, o.groups = torch, Library(w.ran), ctypes.c_void_p(), -1, 3
        o._raw_stream = lambda d: w.current
        setattr(w, cls.__name__, o)
    return w


def calls(w):
    x, m, dz = torch.ones(20, 12), torch.ones(7, 12), torch.ones(20, 7)
    t = torch.zeros(20, dtype=torch.int64)
    ops = w.LocalOps
    return [lambda s: ops.linear_forward(x, m, keep_z=True, stream=s),
            lambda s: ops.linear_backward_input(dz, m, z_prev=x, want_dx=True, stream=s),
            lambda s: ops.linear_backward_weight(dz, x, stream=s), lambda s: ops.activation_backward(x, x, "relu", stream=s),
            lambda s: ops.cross_entropy(dz, t, stream=s)]


@pytest.mark.parametrize("i", range(5))
@pytest.mark.parametrize("as_handle", [False, True])
def test_results_and_workspace_belong_to_the_stream_of_the_call(world, i, as_handle):
    w = world
    results = calls(w)[i](SIDE if as_handle else w.side)
    results = results if isinstance(results, tuple) else (results,)
    assert w.ran == [SIDE] and w.current == CALLER
    assert w.made and all(s == SIDE for _, s in w.made), "allocated on another stream than the call's"
    assert all(any(t is r for t, _ in w.made) for r in results)
    # the results, and nothing else, may be dropped on the caller's stream
    assert sorted(id(t) for t, s in w.recorded if s == CALLER) == sorted(id(r) for r in results)


@pytest.mark.parametrize("i", range(5))
def test_without_a_stream_everything_is_on_the_current_one(world, i):
    calls(world)[i](None)
    assert world.ran == [CALLER] and all(s == CALLER for _, s in world.made) and not world.recorded


def test_tensors_handed_in_stay_the_callers(world):
    x, m, out = torch.ones(20, 12), torch.ones(7, 12), torch.ones(20, 7)
    assert world.LocalOps.linear_forward(x, m, out=out, stream=world.side) is out
    assert not world.recorded
    with pytest.raises(ValueError):
        world.LocalOps.linear_forward(x, m, stream=types.SimpleNamespace(cuda_stream=5, device=types.SimpleNamespace(index=0)))
