"""The stream that the binding's calls go to by default."""
import pytest

from paper_2509_26092_amd import binding as B


def test_a_torch_without_the_handle_by_device_has_the_stream_object(monkeypatch):
    """torch's shortcut to the current stream's handle is no public name:
    where it is missing, the public call gives the handle."""
    import torch

    class Stream:
        cuda_stream = 0x1234

    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    monkeypatch.setattr(B, "_current_handle", None, raising=False)
    assert B._stream() == 0x1234
    assert B._stream(Stream()) == 0x1234


@pytest.mark.gpu
def test_default_stream_is_torchs_current_one():
    import torch
    side = torch.cuda.Stream()
    for _ in range(2):
        assert (B._stream() or 0) == torch.cuda.current_stream().cuda_stream
        with torch.cuda.stream(side):
            assert B._stream() == side.cuda_stream
