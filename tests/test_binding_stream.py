"""The stream that a call of the binding goes to by default, without a GPU where there is none."""
import pytest
import torch

from paper_2010_07565_gb300 import binding as B


def outcome(f):
    try:
        return f()
    except Exception as e:
        return type(e), str(e)


@pytest.mark.parametrize("missing", [False, True])
def test_default_stream_is_torch_s(monkeypatch, missing):
    """The current stream's handle; where CUDA cannot be brought up what torch itself says, also in
    a torch without CUDA, which lacks the private calls."""
    if missing:
        if torch.cuda.is_available():
            pytest.skip("a torch without CUDA sees no GPU")
        for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
            monkeypatch.delattr(torch._C, name, raising=False)
    want = outcome(lambda: torch.cuda.current_stream().cuda_stream)
    assert outcome(lambda: B._stream(None)) == want
