"""The binding enqueues on torch's current stream of the current device, also
when that changes between calls."""
import pytest
import torch

from paper_2606_05484_amd import mapl

pytestmark = pytest.mark.gpu


def test_default_stream_follows_torch():
    assert mapl._stream(None) == torch.cuda.current_stream().cuda_stream
    s = torch.cuda.Stream()
    for _ in range(2):
        with torch.cuda.stream(s):
            assert mapl._stream(None) == s.cuda_stream
        assert mapl._stream(None) == torch.cuda.current_stream().cuda_stream
    assert mapl._stream(s) == s.cuda_stream and mapl._stream(7) == 7
