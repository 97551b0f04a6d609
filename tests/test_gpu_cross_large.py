"""The forward of attention to other states with values so large that a sum of them is infinite,
though their average is not."""
import pytest
import torch

from paper_2606_28560_amd import fibattn as F

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def _normal(seed, *shape, dtype=FP):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _check(o, want, size):
    """One rounding of the storage type; weights in 16 bits and up to 2^-13 of the values' sizes
    from float32 sums of up to 3000 terms."""
    u = 2.0 ** -8 if o.dtype == BF else 2.0 ** -24
    assert bool(torch.isfinite(o).all())
    assert bool(((o.double() - want).abs() <= u * want.abs() + (2.0 ** -13 + 2.0 ** -16) * size).all())


# (B, Bk, H, Hkv, T, S): by keys and by rows, whole and in pieces
SHAPES = [(1, 1, 2, 1, 1, 70), (2, 2, 4, 2, 5, 300), (1, 1, 8, 8, 1030, 90), (2, 1, 2, 1, 3, 3000), (4, 4, 8, 4, 600, 1000)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_large_values(dtype, D, shape):
    B, Bk, H, Hkv, T, S = shape
    print(dtype, D, shape, flush=True)
    q, k = _normal(1, B, H, T, D, dtype=dtype), _normal(2, Bk, Hkv, S, D, dtype=dtype)
    v = (2.0 ** 127 * (1 + 0.9 * torch.rand((Bk, Hkv, S, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)))).to(dtype)
    v[..., 1::2] *= -1  # every other column negative
    v[..., 2] = _normal(4, Bk, Hkv, S, dtype=dtype)  # and one of ordinary values
    o, lse = F.fibattn_cross_forward(q, k, v)
    kk, vv = (x.double().expand(B, Hkv, S, D).repeat_interleave(H // Hkv, 1) for x in (k, v))
    p = torch.softmax(torch.matmul(q.double(), kk.transpose(2, 3).contiguous()) / D ** 0.5, 3)
    _check(o, torch.matmul(p, vv), torch.matmul(p, vv.abs()))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_large_values_of_a_prefix(dtype):
    B, H, Hkv, T, P, S, D = 3, 4, 2, 2, 2500, 60, 64
    q, k, kp = _normal(5, B, H, T, D, dtype=dtype), _normal(6, B, Hkv, S, D, dtype=dtype), _normal(7, 1, Hkv, P, D, dtype=dtype)
    v, vp = torch.full((B, Hkv, S, D), 1.5 * 2.0 ** 127, device="cuda", dtype=dtype), torch.full((1, Hkv, P, D), 1.5 * 2.0 ** 127, device="cuda", dtype=dtype)
    o, lse = F.fibattn_prefix_forward(q, kp, vp, k, v)
    _check(o, torch.full_like(o, 1.5 * 2.0 ** 127, dtype=torch.float64), 1.5 * 2.0 ** 127)
