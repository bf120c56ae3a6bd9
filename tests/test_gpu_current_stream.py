"""Calls without a stream go to torch's current one, on its device (needs an MI355X)."""
import pytest

pytestmark = pytest.mark.gpu


def test_calls_follow_the_current_stream():
    import torch
    from paper_2511_10054_amd.binding import _stream
    assert _stream() == torch.cuda.current_stream().cuda_stream
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert _stream() == side.cuda_stream != 0
    assert _stream() == torch.cuda.current_stream().cuda_stream
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert _stream() == torch.cuda.current_stream().cuda_stream
        torch.zeros(1, device="cuda")
