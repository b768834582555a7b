"""Norms and rotations where a quantity of the formula has no finite value, on the GPU against 64 bits on the CPU (rotary_reference.py, which derives the bounds)."""
import pytest
import torch

from test_gpu_rotary import Case

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("eps", [0.0, 1e-42])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d", [16, 64, 80, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 2), (12, 4), (20, 16), (17, 8), (3, 0), (0, 5)])
def test_gradients_without_eps(hq, hkv, d, interleaved, eps):
    """No head is zero, so everything has a value: that lanes of a wave are left over where heads do not fill it must not show."""
    for dtype in (BF16, F16):
        Case(21, hq, hkv, d, dtype, eps=eps, interleaved=interleaved, seed=hq).check()


@pytest.mark.parametrize("d", [64, 128])
def test_a_head_of_zeros_without_eps_is_the_only_one_without_a_value(d):
    """Its results and gradients are NaN, and so are the weights' it belongs to; other heads and the other weights have theirs."""
    c = Case(21, 4, 2, d, BF16, eps=0.0)
    c.Q[5, 3] = 0.0
    z, k = c.layer.forward(c.Q, c.K, c.positions)
    assert bool(z[5, 3].isnan().all()) and z.isnan().any(2).nonzero().tolist() == [[5, 3]] and k.isfinite().all()
    dQ, dK = c.layer.backward(c.dQ, c.dK, c.Q, c.K, c.positions, out=(torch.empty_like(c.dQ), torch.empty_like(c.dK)))
    assert bool(dQ[5, 3].isnan().all()) and dQ.isnan().any(2).nonzero().tolist() == [[5, 3]] and dK.isfinite().all()
    assert bool(c.layer.dwq.isnan().all()) and c.layer.dwk.isfinite().all()
