"""The forward of attention to other states with logits past 2^32."""
import math

import pytest
import torch

from paper_2606_28560_amd import fibattn as F
from tests import cross_reference as R

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def _normal(seed, *shape, dtype=FP):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _bits(x):
    return x.contiguous().view(torch.int16 if x.dtype == BF else torch.int32)


def _scales(seed, n):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randperm(n, generator=g, device="cuda")


# (B, Bk, H, Hkv, T, S): one token, a few, pieces, many rows
HUGE = [(1, 1, 2, 1, 1, 70), (2, 2, 4, 2, 3, 40), (3, 1, 2, 2, 1, 2100), (1, 1, 8, 8, 1030, 90), (2, 2, 2, 1, 40, 1600)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("shape", HUGE, ids=str)
def test_huge_logits(dtype, D, shape):
    """Logits of 2^33 and more, of either sign: one row of the states has all the weight, so o
    is its value and lse its logit, whichever way the products are rounded.

    The rows have a first element only, with 7 bits behind the leading one, exact in both types;
    the largest of k and its smallest are there once, so the next logit is 2^-8 of it lower."""
    B, Bk, H, Hkv, T, S = shape
    print(dtype, D, shape, flush=True)
    q, v = torch.zeros((B, H, T, D), device="cuda"), _normal(201, Bk, Hkv, S, D, dtype=dtype)
    k = torch.zeros((Bk, Hkv, S, D), device="cuda")
    # 1 .. 2 by steps of 2^-7 (bfloat16's), times 2^19 (q) and 2^20 (k); the largest of k, and its smallest, once
    step = 2.0 ** -7
    q[..., 0] = 2.0 ** 19 * (1 + step * (torch.arange(B * H * T, device="cuda") * 37 % 128)).reshape(B, H, T)
    q[..., 0] *= torch.where(torch.arange(T, device="cuda") % 3 == 1, -1.0, 1.0)
    for b in range(Bk):
        for h in range(Hkv):
            x = 1 + step * (1 + _scales(210 + b * 7 + h, S) % 126)
            top, low = (13 * (b + 1) + 5 * h) % S, (29 * (b + 1) + 3 * h + 1) % S
            x[low], x[top] = 1.0, 1 + 127 * step
            k[b, h, :, 0] = 2.0 ** 20 * x
    q, k = q.to(dtype), k.to(dtype)
    o, lse = F.fibattn_cross_forward(q, k, v)
    kk = k.double().expand(B, Hkv, S, D).repeat_interleave(H // Hkv, 1)
    vv = v.expand(B, Hkv, S, D).repeat_interleave(H // Hkv, 1)
    s = q.double()[..., :1] * kk[..., 0][:, :, None, :] / math.sqrt(D)
    top, at = s.max(3)
    assert float(top.abs().min()) > 2.0 ** 33
    want = torch.gather(vv, 2, at[..., None].expand(B, H, T, D))
    assert torch.equal(_bits(o), _bits(want))
    # tau, its product with log2 e and back, the logit's rounding and the maximum's step: 6 of 2^-24
    assert bool(((lse.double() - top).abs() <= 6 * 2.0 ** -24 * top.abs()).all())
    o2, lse2 = F.fibattn_cross_forward(q, k, v)
    assert torch.equal(_bits(o), _bits(o2)) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,S", [(1, 100), (1, 3000), (700, 100), (33, 1000)])
def test_hugely_negative_logits_beside_ordinary_ones(dtype, T, S):
    """Rows with logits below -2^33 in front of, among and behind ordinary ones count nothing."""
    H, Hkv, D = 4, 2, 64
    q, k, v = _normal(220, 1, H, T, D), _normal(221, 1, Hkv, S, D), _normal(222, 1, Hkv, S, D, dtype=dtype)
    far = torch.zeros(S, dtype=torch.bool, device="cuda")
    far[:40], far[50:60], far[S - 9:] = True, True, True
    q[..., 0] = 2.0 ** 15 + 2.0 ** 9 * (torch.arange(T, device="cuda") % 60)
    k[..., 0] = 0.0
    k[:, :, far] = 0.0
    k[:, :, far, 0] = -(2.0 ** 21 + 2.0 ** 15 * (torch.arange(int(far.sum()), device="cuda") % 60))
    q, k = q.to(dtype), k.to(dtype)
    o, lse = F.fibattn_cross_forward(q, k, v)
    keep = ~far[None, None, :].expand(1, T, S)
    # the far rows out of it, and q's first element with them (it meets only zeros in the others)
    q0 = q.clone()
    q0[..., 0] = 0
    R.check({"o": o, "lse": lse}, R.attention(q0, k, v, keep=keep), "far rows")


def test_huge_logits_of_a_prefix():
    B, H, Hkv, T, P, S, D = 3, 4, 2, 3, 200, 50, 64
    for dtype in (BF, FP):
        q, v, vp = torch.zeros((B, H, T, D), device="cuda"), _normal(230, B, Hkv, S, D, dtype=dtype), _normal(231, 1, Hkv, P, D, dtype=dtype)
        k, kp = torch.zeros((B, Hkv, S, D), device="cuda"), torch.zeros((1, Hkv, P, D), device="cuda")
        q[..., 0] = 2.0 ** 19 * (1 + 2.0 ** -7 * (torch.arange(B * H * T, device="cuda") * 37 % 128)).reshape(B, H, T)
        kp[..., 0] = 2.0 ** 20 * (1 + 2.0 ** -7 * (_scales(232, P) % 100))
        k[..., 0] = 2.0 ** 20 * (1 + 2.0 ** -7 * (_scales(233, S) % 100))
        kp[0, :, 77, 0] = 2.0 ** 20 * (1 + 2.0 ** -7 * 120)
        k[1, :, 20, 0] = 2.0 ** 20 * (1 + 2.0 ** -7 * 125)  # only sequence 1 has a larger one of its own
        o, lse = F.fibattn_prefix_forward(q.to(dtype), kp.to(dtype), vp, k.to(dtype), v)
        for b in range(B):
            want = (v[b, :, 20] if b == 1 else vp[0, :, 77]).repeat_interleave(H // Hkv, 0)[:, None].expand(H, T, D)
            assert torch.equal(_bits(o[b]), _bits(want)), (dtype, b)
        top = torch.maximum(kp[0, 0, 77, 0], torch.where(torch.arange(B, device="cuda") == 1, k[1, 0, 20, 0], 0.0))
        top = q.to(dtype).double()[..., 0] * top.double()[:, None, None] / 8
        assert bool(((lse.double() - top).abs() <= 8 * 2.0 ** -24 * top).all())
