"""The stream that a call of the binding takes (no GPU needed): torch is asked each time whether CUDA can be used."""
import pytest
import torch

from paper_2607_20357_gb300 import svl


def test_a_forked_child_gets_torchs_error(monkeypatch):
    """In a child forked behind the first call torch refuses CUDA, whatever the parent had found."""
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 77, raising=False)
    assert svl._stream(None) == 77

    def refuse():
        raise RuntimeError("Cannot re-initialize CUDA in forked subprocess")
    # (what torch says there: not initialised for this process, and no stream to be had)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", refuse)
    with pytest.raises(RuntimeError, match="forked"):
        svl._stream(None)
