"""CPU-only: what the binding of the attention decoder's calls refuses before it calls the library."""
import types

import pytest

from paper_1909_09577_amd import binding as nm


@pytest.mark.parametrize("n", [0, 2])
def test_a_gradient_scale_has_one_element(n):
    """An empty one would be none at all, of a longer one the rest would be ignored."""
    torch = pytest.importorskip("torch")
    host = torch.zeros(256, dtype=torch.uint8)  # (no plan: the library would refuse it)
    on_device = types.SimpleNamespace(is_cuda=True, is_contiguous=lambda: True, dtype=torch.float32, shape=(n,), numel=lambda: n, data_ptr=lambda: 0)
    with pytest.raises(ValueError, match="one element"):
        nm.nm_adamw_step(nm.AdamWPlan(host, host, {}, 32), lr=1e-3, step=1, grad_scale=on_device, stream=types.SimpleNamespace(cuda_stream=None))


def test_norms_gradients_need_a_gradient():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 4, 8)
    with pytest.raises(nm.NmError) as e:
        nm.nm_residual_norm_bwd(None, None, x, x)
    assert e.value.status == nm.NM_ERR_BAD_ARG
