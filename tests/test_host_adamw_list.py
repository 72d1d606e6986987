"""Which stream the calls on a list of tensors go to."""
import pytest
import torch

from paper_2204_01205_amd import binding as B


@pytest.mark.parametrize("call", [lambda t: B.fno_adamw_step(t, 1e-3, 0.9, 0.999, 1e-8, 1),
                                  lambda t: B.fno_grad_norm(t, None, torch.empty(0, dtype=torch.uint8)),
                                  lambda t: B.fno_adamw_state_read(t, [], [])])
def test_a_list_on_another_device_is_refused(monkeypatch, call):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    monkeypatch.setattr(B, "_address", lambda *args: None)
    here = B.make_adamw_tensors([], [], [], [], exps=[])
    there = B.AdamwTensors(here.array, 0, [], 8, torch.device("cuda", 1), here.keep)
    with pytest.raises(ValueError, match="cuda:1"):
        call(there)


def test_the_stream_without_the_undocumented_call(monkeypatch):
    class Stream:
        cuda_stream = 77

    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: Stream)
    assert B._raw_stream(0) == 77
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert B._raw_stream() == 77


@pytest.mark.gpu
def test_the_current_streams_handle():
    assert B._raw_stream() == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(torch.cuda.Stream()):
        assert B._raw_stream() == torch.cuda.current_stream().cuda_stream != torch.cuda.default_stream().cuda_stream
