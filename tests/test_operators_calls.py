"""The Python side of the operators without a GPU: the streams that it works on."""
import contextlib
import types

import pytest

import paper_2310_14423_amd.operators as ops


class _Tensor:
    device = "cuda:1"

    def __init__(self, index=1):
        self.index = index

    def get_device(self):
        return self.index


def _torch(log, device=1, current=77):
    @contextlib.contextmanager
    def entered(what):
        log.append(what)
        yield
    cuda = types.SimpleNamespace(current_device=lambda: device, device=lambda i: entered(("device", i)), stream=entered,
                                 ExternalStream=lambda address, device: ("external", address), default_stream=lambda device: ("default", device))
    return types.SimpleNamespace(cuda=cuda, _C=types.SimpleNamespace(_cuda_getCurrentRawStream=lambda i: current))


@pytest.mark.parametrize("stream,want", [(0, ("default", "cuda:1")), (55, ("external", 55)), (77, None), (None, None)])
@pytest.mark.parametrize("device", [1, 0])
def test_streams(stream, want, device, monkeypatch):
    """Address 0 is the device's default stream: torch makes another stream of an external one at 0, which would then own the results
    that a kernel on the default stream writes."""
    log = []
    monkeypatch.setattr(ops, "_torch", _torch(log, device))
    s, place = ops._place(_Tensor(), stream)
    assert s == (77 if stream is None else stream)
    with place or contextlib.nullcontext():
        pass
    assert [x for x in log if x[0] != "device"] == ([want] if want else []) and [x for x in log if x[0] == "device"] == ([("device", 1)] if device == 0 else [])
    assert (place is None) == (not log)
