"""What the binding of the head's operators looks at before a call, on the CPU: tensors are stood for by objects that say where they are."""
import pytest
import torch

from paper_1910_00932_amd import binding as B


class Tensor:
    """A contiguous tensor of a device, at an address that nothing reads."""

    def __init__(self, n, dtype=torch.float32, device=0, at=1 << 20):
        self.n, self.dtype, self.device_index, self.at = n, dtype, device, at
        self.is_cuda = True

    def numel(self):
        return self.n

    def element_size(self):
        return self.dtype.itemsize

    def get_device(self):
        return self.device_index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at


class Library:
    """Takes every call."""

    def __getattr__(self, name):
        if name.endswith("_bytes"):
            return lambda desc: 64
        return lambda *a: 0


@pytest.fixture
def here(monkeypatch):
    """Device 0 is the current one."""
    monkeypatch.setattr(B, "_device", lambda: 0)
    monkeypatch.setattr(B, "lib", Library)


def _calls(ws, saved):
    x, m, f = Tensor(512, torch.bfloat16), Tensor(64), Tensor(8)
    rc = B.RecurDesc(N=1, T=8, C=64, H=1, W=1, dtype=B.TSM_BF16)
    ln = B.LayerNormDesc(rows=8, C=64, dtype=B.TSM_BF16, eps=1e-5)
    xe = B.XentDesc(rows=8, features=64, classes=8, dtype=B.TSM_BF16)
    lab = Tensor(8, torch.int32)
    return {
        "recur_fwd": lambda: B.tsm_recur_fwd(rc, x, x, None, x, None, saved, ws, stream=0),
        "recur_bwd": lambda: B.tsm_recur_bwd(rc, x, x, None, saved, x, None, x, x, None, ws, stream=0),
        "layernorm_bwd": lambda: B.tsm_layernorm_bwd(ln, x, x, m, f, f, x, m, m, ws, stream=0),
        "xent_fwd": lambda: B.tsm_xent_fwd(xe, x, x, None, lab, f, f, ws, stream=0),
        "xent_bwd": lambda: B.tsm_xent_bwd(xe, x, x, None, lab, f, f, x, x, None, ws, stream=0),
    }


CALLS = ["recur_fwd", "recur_bwd", "layernorm_bwd", "xent_fwd", "xent_bwd"]


@pytest.mark.parametrize("call", CALLS)
def test_a_workspace_on_another_device_is_refused(here, call):
    near, far = Tensor(64, torch.uint8), Tensor(64, torch.uint8, device=1)
    _calls(near, near)[call]()
    with pytest.raises(ValueError, match="the workspace is on cuda:1, the current device is cuda:0"):
        _calls(far, near)[call]()


@pytest.mark.parametrize("call", ["recur_fwd", "recur_bwd"])
def test_a_saved_buffer_on_another_device_is_refused(here, call):
    near, far = Tensor(64, torch.uint8), Tensor(64, torch.uint8, device=1)
    with pytest.raises(ValueError, match="saved is on cuda:1, the current device is cuda:0"):
        _calls(near, far)[call]()
    with pytest.raises(ValueError, match="saved: expected at least 64 bytes, got 63"):
        _calls(near, Tensor(63, torch.uint8))[call]()


@pytest.mark.parametrize("private", [True, False])
def test_current_stream_with_and_without_torchs_private_call(monkeypatch, private):
    """What a torch without the private call offers is asked in its place; without a device given, about the current one."""
    class Stream:
        def __init__(self, dev):
            self.cuda_stream = 1000 + dev

    def handle(dev):
        return 1000 + dev

    def gone(dev):
        raise AssertionError("not in this torch")
    if private:
        monkeypatch.setattr(B, "_raw_stream", handle)
        monkeypatch.setattr(torch.cuda, "current_stream", gone)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
        monkeypatch.setattr(B, "_raw_stream", None, raising=False)
        monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    assert B._stream(None) == 1003 and B._stream(None, 1) == 1001
    assert B._stream(77) == 77 and B._stream(Stream(5)) == 1005
