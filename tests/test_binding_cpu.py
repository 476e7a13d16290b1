"""CPU: what the binding refuses before it calls the library, with stand-ins for CUDA
tensors that no memory lies behind."""
import pytest
import torch

from paper_2606_05613_gb300 import native as bk

B, F, U8 = torch.bfloat16, torch.float32, torch.uint8


class _T:
    """As much of a contiguous tensor as the binding looks at."""

    def __init__(self, *shape, dtype=B, dev=0, contiguous=True):
        self.shape, self.dtype, self.dev, self.contiguous = torch.Size(shape), dtype, dev, contiguous
        self.device = torch.device("cuda", dev) if dev >= 0 else torch.device("cpu")

    def get_device(self):
        return self.dev

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (self.shape[-1], 1)

    def data_ptr(self):
        return 1 << 40

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return self.contiguous


@pytest.fixture
def called(monkeypatch):
    calls = []
    monkeypatch.setattr(bk, "_call", lambda torch_, dev, where, fn, *a: calls.append(where))
    monkeypatch.setattr(bk, "_raw_stream", lambda *a: 0)
    return calls


def _backward(ws):
    t, w, x = _T(4, 16), _T(16, 8), _T(4, 8)
    bk.bkmoo_gate_backward(t, t, t, x, w, w, "silu", [0, 4], dx=_T(4, 8), ws=ws)


def _norm(ws):
    bk.bkmoo_grad_norm(_T(64, dtype=F), _T(1, dtype=F), ws=ws)


@pytest.mark.parametrize("call", [_backward, _norm])
def test_workspaces_are_on_the_device(called, call):
    """A workspace in host memory or on another device would be written through its
    address all the same."""
    for bad in (_T(1 << 20, dtype=U8, dev=-1), _T(1 << 20, dtype=U8, dev=1), _T(1 << 20, dtype=U8, contiguous=False)):
        with pytest.raises(ValueError, match="ws"):
            call(bad)
    assert called == []
    call(_T(1 << 20, dtype=U8))
    assert len(called) == 1
