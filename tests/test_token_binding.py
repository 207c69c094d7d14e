"""CPU-only: the binding of the calls on tokens refuses outputs that a call would leave unwritten."""
import types

import pytest

from paper_1909_09577_amd import binding as nm


class OnDevice:
    """What the binding looks at in a contiguous device tensor; nothing lies behind its pointer."""
    _next = 0x700000000000

    def __init__(self, *shape, dtype=None):
        import torch
        self.shape, self.dtype, self.is_cuda = torch.Size(shape), dtype or torch.float32, True
        OnDevice._next += 1 << 32
        self._at = OnDevice._next

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self._at

    def new_empty(self, shape, dtype=None):
        return OnDevice(*shape, dtype=dtype or self.dtype)


@pytest.fixture
def torch(monkeypatch):
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return torch


NO_STREAM = types.SimpleNamespace(cuda_stream=None)


@pytest.mark.parametrize("name", ["dq_weight", "dk_weight"])
def test_a_weights_gradient_needs_its_weight(torch, name):
    x = OnDevice(2, 6 * 64, 9)
    with pytest.raises(nm.NmError) as e:
        nm.nm_head_norm_bwd(OnDevice(2, 6 * 64, 9), x, heads=4, kv_heads=2, dx=OnDevice(2, 6 * 64, 9), stream=NO_STREAM, **{name: OnDevice(64)})
    assert e.value.status == nm.NM_ERR_BAD_ARG
