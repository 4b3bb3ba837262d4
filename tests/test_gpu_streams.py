"""The stream that a call without one is given."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2509_03047_amd import flashrestore as F  # noqa: E402


def test_no_stream_is_the_current_one():
    """Outside and inside of stream contexts and of a capture, as torch's own object has it."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")

    def same():
        return F._stream(None) == (torch.cuda.current_stream().cuda_stream or None)

    assert same() and F._stream(None) is None
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        assert same() and F._stream(None) == st.cuda_stream == F._stream(st) == F._stream(st.cuda_stream)
        with torch.cuda.stream(torch.cuda.default_stream()):
            assert same() and F._stream(None) is None
    x = torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert same() and F._stream(None) is not None
        x += 1
    assert same()
