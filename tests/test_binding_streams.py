"""Which stream's memory pool a call's own tensors come from: always that of the
stream its kernels run on, also for raw handles."""
import pytest
import torch

from paper_2609_34388_amd import binding


def test_handle_zero_is_the_default_stream(monkeypatch):
    made = []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h: made.append(h) or "external")
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: "default")
    monkeypatch.setattr(torch.cuda, "stream", lambda s: s)
    assert binding._pool_of(0) == "default" and made == []
    assert binding._pool_of(0x1230) == "external" and made == [0x1230]


@pytest.mark.gpu
def test_pool_and_kernels_share_a_stream():
    side = torch.cuda.Stream()
    for stream in (0, torch.cuda.current_stream().cuda_stream, torch.cuda.default_stream(), side, side.cuda_stream):
        with binding._pool_of(stream):
            assert torch.cuda.current_stream().cuda_stream == binding._stream(stream)
    with torch.cuda.stream(side), binding._pool_of(0):
        assert torch.cuda.current_stream() == torch.cuda.default_stream()
