"""`stream` of the sequence operators' calls: one of another device than the tensors' is refused.  On
the CPU, with stand-ins for tensors and streams: nothing is launched."""
import pytest
import torch

from paper_2408_00280_amd import sequence


class OnDevice:
    is_cuda = True

    def __init__(self, device):
        self.device = torch.device("cuda", device)


@pytest.mark.parametrize("fn", [sequence.conv_forward, sequence.conv_backward, sequence.scan_forward, sequence.scan_backward,
                                sequence.norm_forward, sequence.norm_backward])
def test_a_stream_of_another_device_is_refused(fn, monkeypatch):
    class Stream(OnDevice):
        pass
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    name = fn.__wrapped__.__code__.co_varnames[0]
    for args, kw in (((OnDevice(0),), {}), ((), {name: OnDevice(0)})):
        with pytest.raises(ValueError, match="cuda:1"):
            fn(*args, stream=Stream(1), **kw)
