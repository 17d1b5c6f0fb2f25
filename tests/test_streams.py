"""CPU tests of the binding's buffers on a stream that is not the current one: what a
call makes for itself comes from the memory of the stream that it runs on.  (A block
of the current stream's memory may still be in use by work queued there, which the
other stream does not wait for.)  Streams are stand-ins, nothing is launched."""

import contextlib

import pytest

torch = pytest.importorskip("torch")

from paper_2607_14107_amd import polestar as ps  # noqa: E402


class _Stream:
    def __init__(self, handle, device_index=0):
        self.cuda_stream, self.device_index = handle, device_index


@pytest.fixture
def made(monkeypatch):
    """The (stream in effect, elements) of every tensor made, and the streams recorded on them."""
    main, made, recorded, current = _Stream(1), [], [], []
    current.append(main)
    real = torch.empty

    @contextlib.contextmanager
    def on(s):
        current.append(s)
        yield
        current.pop()

    class Tensor(torch.Tensor):
        def record_stream(self, s):
            recorded.append((tuple(self.shape), s))

    def empty(shape, dtype=None, device=None):
        t = real(shape, dtype=dtype).as_subclass(Tensor)
        made.append((current[-1], tuple(t.shape)))
        return t

    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current[-1])
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", empty)
    return main, made, recorded


def test_microscaled_calls_allocate_on_the_stream_they_run_on(made):
    main, made, recorded = made
    side = _Stream(2)
    out = ps._mx_empty((4, 8), torch.uint8, 0, side)
    assert made == [(side, (4, 8))]
    assert recorded == [((4, 8), main)]                  # the caller may read it on its own stream
    for stream in (None, main):
        ps._mx_empty((3,), torch.uint8, 0, stream)
    assert made[1:] == [(main, (3,))] * 2 and len(recorded) == 1
    assert out.shape == (4, 8)


def test_a_scratch_made_by_a_microscaled_call_belongs_to_its_stream(made, monkeypatch):
    main, made, recorded = made
    side, calls = _Stream(2), []

    class Lib:
        @staticmethod
        def call(*args):
            calls.append(args)
            return ps.STATUS_WORKSPACE if args[-2] < 96 else ps.OK

    monkeypatch.setattr(ps, "lib", lambda: Lib)
    for ws in (None, torch.zeros(16, dtype=torch.uint8)):
        ps._mx_call("call", (7,), lambda: 96, ws, 0, side)
    assert made == [(side, (96,))] * 2 and not recorded  # nobody reads it afterwards
    assert [c[0] for c in calls] == [7] * 3 and all(c[-1] == side.cuda_stream for c in calls)
