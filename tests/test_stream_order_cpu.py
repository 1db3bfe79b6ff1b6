"""The layer drivers order the weight gradients behind the stream that the dX chain ran on, however the
caller names it.  The library's calls and torch's events are replaced: nothing runs."""
from types import SimpleNamespace

import pytest
import torch

L = pytest.importorskip("paper_2404_19429_amd.lancet_moe", reason="library not built")


class FakeStream:
    """In the place of torch.cuda.Stream; ExternalStream wraps a handle."""
    def __init__(self, handle):
        self.handle = self.cuda_stream = handle

    def wait_event(self, ev):
        FakeEvent.waits.append((self.handle, ev.on))


class FakeEvent:
    waits: list = []

    def record(self, stream):
        self.on = stream.handle


CURRENT, DEFAULT = FakeStream(77), FakeStream(0)
STREAMS = {"object": (FakeStream(4096), 4096), "handle": (8192, 8192), "current": (None, 77), "null handle": (0, 0)}


@pytest.fixture
def calls(monkeypatch):
    """(name, stream handle) of every call of the library."""
    made = []
    FakeEvent.waits = []
    for name, value in (("Stream", FakeStream), ("ExternalStream", FakeStream), ("Event", FakeEvent),
                        ("current_stream", lambda *a: CURRENT), ("default_stream", lambda *a: DEFAULT)):
        monkeypatch.setattr(torch.cuda, name, value)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 77, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for name in ("moe_bwd_dx", "moe_bwd_dx_route", "moe_bwd_dw", "moe_sorted_combine_bwd", "moe_route_bwd", "moe_sorted_bwd_dx",
                 "moe_sorted_dispatch_bwd", "moe_sorted_bwd_dw"):
        monkeypatch.setattr(L, name, lambda *a, _name=name: made.append((_name, L._stream(a[-1]))))
    return made


class Anything:
    """Buffers and configurations of no interest."""
    def __getattr__(self, name):
        return 1 if name in ("T", "E", "k", "renorm") else Anything()


@pytest.mark.parametrize("dw", ["object", "handle"])
@pytest.mark.parametrize("how", sorted(STREAMS))
@pytest.mark.parametrize("router", [False, True])
@pytest.mark.parametrize("driver", ["layer_backward", "sorted_layer_backward"])
def test_weight_gradients_wait_for_the_chain_s_stream(calls, driver, router, how, dw):
    stream, handle = STREAMS[how]
    dw_stream = FakeStream(12288) if dw == "object" else 12288
    b, r = Anything(), SimpleNamespace(cfg=Anything()) if router else None
    getattr(L, driver)(b, None, None, None, stream, dw_stream, r)
    chain = {s for n, s in calls if not n.endswith("bwd_dw")}
    assert chain == {handle}
    assert [s for n, s in calls if n.endswith("bwd_dw")] == [12288]
    assert FakeEvent.waits == [(12288, handle)]


@pytest.mark.parametrize("driver", ["layer_backward", "sorted_layer_backward"])
def test_one_stream_needs_no_event(calls, driver):
    getattr(L, driver)(Anything(), None, None, None, 8192)
    assert {s for _, s in calls} == {8192} and FakeEvent.waits == []
