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


def _z(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def _i(*shape):
    return _z(*shape, dtype=torch.int32)


CACHE, W = (2, 9, 2, 4), (8, 8)                          # [batch][seq][n_kv_heads][head_dim], [n_out][n_in]
CALLS = {  # the call, the tensors it returns that it made itself
    "drift": (lambda s: ps.drift(_z(2, 9, 8), _z(2, 9, 8), stream=s), 1),
    "select": (lambda s: ps.select(_z(2, 9), 3, 0, 2, stream=s), 2),
    "refresh_kv": (lambda s: ps.refresh_kv(_z(2, 9, 8), None, None, 0, 2, _z(*W), _z(*W), _z(*CACHE), _z(*CACHE),
                                           stream=s), 0),
    "project_qkv": (lambda s: ps.project_qkv(_z(2, 9, 8), 0, 3, _z(*W), _z(*W), _z(*W), _z(2, 3, 2, 4), _z(*CACHE),
                                             _z(*CACHE), stream=s), 0),
    "project_q": (lambda s: ps.project_q(_z(2, 9, 8), _z(*W), 0, 3, 2, stream=s), 1),
    "attend": (lambda s: ps.attend(_z(2, 9, 8), _z(*W), _z(*CACHE), _z(*CACHE), 0, 3, 2, stream=s), 2),
    "commit": (lambda s: ps.commit(_z(2, 3, 16), _i(2, 3), None, 0, None, None, stream=s), 3),
    "suffix_commit": (lambda s: ps.suffix_commit(_z(2, 3, 16), _i(2, 3), _i(2, 3), stream=s), 3),
    "linear": (lambda s: ps.linear(_z(2, 9, 8), 0, 3, _z(4, 8), _z(2, 3, 4), stream=s), 0),
    "linear_swiglu": (lambda s: ps.linear_swiglu(_z(2, 9, 8), 0, 3, _z(8, 8), _z(2, 3, 8), _z(2, 3, 4), stream=s), 0),
    "cluster_means": (lambda s: ps.cluster_means(_z(2, 9, 8), _i(2, 4), _i(2, 9), 3, stream=s), 1),
    "cluster": (lambda s: ps.cluster(_z(2, 9, 8), _i(2, 4), 3, stream=s), 4),
    "proxy_drift": (lambda s: ps.proxy_drift(_z(2, 3, 8), _i(2, 3), _z(*W), _z(*CACHE), 2, _z(2, 3, 2, 9), _z(2, 3, 2),
                                             True, stream=s), 1),
    "attention_drift": (lambda s: ps.attention_drift(_z(2, 3, 2, 4), _z(*CACHE), _z(2, 3, 2, 9), _z(2, 3, 2), True,
                                                     stream=s), 1),
    "cluster_select": (lambda s: ps.cluster_select(_i(2, 9), _z(2, 3), 1, 4, stream=s), 2),
}
SCRATCH = {"refresh_kv", "project_qkv", "project_q", "attend", "commit", "suffix_commit", "linear", "linear_swiglu",
           "proxy_drift", "attention_drift"}


@pytest.mark.parametrize("name", CALLS)
def test_calls_allocate_on_the_stream_they_run_on(made, monkeypatch, name):
    main, made, recorded = made
    side, launched = _Stream(2), []

    class Lib:
        def __getattr__(self, f):
            if f.endswith("_size"):
                return lambda *a: 96
            return lambda *a: launched.append((f, a[-1])) or ps.OK

    monkeypatch.setattr(ps, "lib", Lib)
    monkeypatch.setattr(ps, "_ptr", lambda *a: None)
    call, returned = CALLS[name]
    for stream in (side, None):
        made.clear(), recorded.clear(), launched.clear()
        call(stream)
        s = stream or main
        assert [a for _, a in launched] == [s.cuda_stream]
        assert [a for a, _ in made] == [s] * (returned + (name in SCRATCH))
        assert [a for _, a in recorded] == ([main] * returned if stream else [])


def test_microscaled_calls_refuse_a_stream_of_another_device():
    assert ps._mx_stream(0, _Stream(7)) == 7
    with pytest.raises(ValueError, match="stream"):
        ps._mx_stream(0, _Stream(7, device_index=1))
