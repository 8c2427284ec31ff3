"""Host-side logic of the verification-step operators' package, without a GPU."""
import contextlib
import types

import pytest
import torch

from paper_2410_03960_b200 import verify


@pytest.mark.parametrize("device,stream_on,want", [(None, None, 3), ("cuda", None, 3), (torch.device("cuda"), None, 3), ("cuda:1", None, 1), (2, None, 2), ("cuda:0", None, 0),
                                                   (None, 5, 5), ("cuda", 5, 5), ("cuda:5", 5, 5)])
def test_op_status_asks_the_device_that_is_meant(monkeypatch, device, stream_on, want):
    """A device without a number is the current one (3 here), not the first."""
    asked = []

    @contextlib.contextmanager
    def made_current(index):
        asked.append(index)
        yield

    streams = {i: types.SimpleNamespace(cuda_stream=100 + i, device_index=i) for i in range(6)}
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "device", made_current)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: streams[asked[-1]])
    monkeypatch.setattr(verify, "load_library", lambda: types.SimpleNamespace(swiftkv_op_status=lambda s: asked.append(s) or 0))
    verify.op_status(device, stream=None if stream_on is None else streams[stream_on])
    assert asked == [want, 100 + want]


def test_op_status_refuses_a_stream_of_another_device():
    with pytest.raises(ValueError):
        verify.op_status("cuda:0", stream=types.SimpleNamespace(cuda_stream=1, device_index=1))
