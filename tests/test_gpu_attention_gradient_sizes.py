"""Gradients of attention whatever the size of what comes back: dS, which lies between results and operands of another size, costs them nothing."""
import pytest
import torch

from attention_reference import packed

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def gradients(lens, hq, hkv, d, dtype, sizes, seed=0):
    """(gradients, those of 64 bits) of rows dO that are normal numbers times `sizes` (a number, or one for each row)"""
    from paper_2404_01847_amd.attention import Attention
    n, cu = sum(lens), [0]
    for x in lens:
        cu.append(cu[-1] + x)
    gen = torch.Generator().manual_seed(seed)
    draw = lambda h: torch.randn((n, h, d), generator=gen)
    Q, K, V, dO = draw(hq), draw(hkv), draw(hkv), draw(hq)
    K = K * torch.exp(0.5 * torch.randn((1, hkv, d), generator=gen))
    dO = dO * (sizes if isinstance(sizes, float) else sizes.view(-1, 1, 1))
    Q, K, V, dO = (x.to(dtype).cuda() for x in (Q, K, V, dO))
    layer, offsets = Attention(hq, hkv, d, n, n, dtype), torch.tensor(cu, dtype=torch.int32, device="cuda")
    layer.forward(Q, K, V, offsets)
    grads = layer.backward(Q, K, V, dO, offsets)
    ref, _ = packed(Q, K, V, cu, cu, d ** -0.5, True, dO)
    return {name: x.cpu().double() for name, x in zip(("dQ", "dK", "dV"), grads)}, ref


def assert_own_rounding(got, want, dtype, what, allowed=1.2):
    """In the 2-norm, against results of 64 bits that are rounded once; a fifth more for the fp32 of the exponentials and sums."""
    assert want.abs().max() < torch.finfo(dtype).max, what   # (of the test itself)
    off, own = (got - want).norm(), (want.to(dtype).double() - want).norm()
    assert off <= allowed * own, (what, (off / own).item())


# a few parts of one launch; parts of long rows; a launch for each gradient; heads between the tiles' sizes
@pytest.mark.parametrize("lens,heads,d", [([1500], (2, 1), 64), ([4096], (1, 1), 128), ([1100, 1100], (64, 8), 64), ([700, 33, 900], (2, 2), 80)])
@pytest.mark.parametrize("size", [1e-2, 1e-3, 1e-4])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_small_gradients_lose_nothing(lens, heads, d, size, dtype):
    """dS is about dO's size over a row's length: in binary16 that lies among the subnormals, dQ and dK do not."""
    got, ref = gradients(lens, *heads, d, dtype, size, seed=d)
    for name in ("dQ", "dK"):
        assert_own_rounding(got[name], ref[name], dtype, name)


@pytest.mark.parametrize("seed", [0, 2, 4])
@pytest.mark.parametrize("d", [64, 128])
def test_large_gradients_stay_finite(seed, d):
    """dS beyond binary16's largest number (about 7e4 here): results within it are what they are without that.  (Some of dQ and dV are beyond it themselves.)"""
    got, ref = gradients([64], 1, 1, d, F16, 12000.0 if d == 128 else 15000.0, seed)
    for name, want in ref.items():
        if name not in got:
            continue
        fits = want.abs() < torch.finfo(F16).max
        assert got[name][fits].isfinite().all() and int((~fits).sum()) < 10, name
        if name != "dV":
            assert_own_rounding(got[name][fits], want[fits], F16, name)


@pytest.mark.parametrize("d,heads", [(64, (4, 2)), (128, (2, 2))])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_rows_of_very_different_sizes(d, heads, dtype):
    """Each row of dQ, and each key that sees rows of one size alone, as if there were no others: rows of 1e-4 to 1e3, in blocks that do not go by the tiles, the
    last ones small after large ones in one tile."""
    n = 700
    sizes = torch.ones(n)
    blocks = [(0, 100, 1.0), (100, 200, 1e-4), (200, 300, 1e3), (300, 400, 1e-2), (400, 500, 10.0), (500, 600, 1e-3), (600, 684, 1e2), (684, 700, 1e-4)]
    for a, b, size in blocks:
        sizes[a:b] = size
    got, ref = gradients([n], *heads, d, dtype, sizes, seed=d)
    for a, b, _ in blocks:
        for name in ("dQ", "dK"):
            assert_own_rounding(got[name][a:b], ref[name][a:b], dtype, f"{name}[{a}:{b}]")
