"""Gradients of attention to other states beside keys and queries that are not finite."""
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


# (B, Bk, H, Hkv, T, S, lens): dq and dk, dv by 32 and by 128 rows, whole and in pieces
NEVER = [(1, 1, 1, 1, 3, 70, None), (2, 2, 4, 2, 90, 130, [130, 33]), (1, 1, 2, 1, 5, 3001, [2999]),
         (3, 1, 2, 2, 900, 40, None), (4, 4, 8, 4, 1001, 1030, [1030, 64, 40, 777]), (8, 8, 8, 8, 1023, 90, None)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("shape", NEVER, ids=str)
def test_gradients_beside_a_key_that_counts_nothing(dtype, D, shape):
    """Keys with a first element of -inf, which every query weighs with 0: their dk and dv are 0,
    everything else is as without them, but for dq's first element (0 times -inf)."""
    B, Bk, H, Hkv, T, S, lens = shape
    print(dtype, D, shape, flush=True)
    q, dO = _normal(240, B, H, T, D, dtype=dtype), _normal(241, B, H, T, D, dtype=dtype)
    k, v = _normal(242, Bk, Hkv, S, D, dtype=dtype), _normal(243, Bk, Hkv, S, D, dtype=dtype)
    q[..., 0] = 1.0
    out = [9, S - 3 if lens is None else min(lens) - 3]
    for j in out:
        k[:, :, j] = 0.5
        k[:, :, j, 0] = -math.inf
    n = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    keep = torch.ones((B, T, S), dtype=torch.bool, device="cuda") if n is None else \
        R.lens_mask(n.expand(B) if Bk == 1 else n, T, S).clone()
    keep[:, :, out] = False
    ref = R.attention(q, k, v, dO, keep)
    o, lse = F.fibattn_cross_forward(q, k, v, n)
    R.check({"o": o, "lse": lse}, ref, "forward")
    dq, dk, dv = F.fibattn_cross_backward(q, k, v, o, lse, dO, n)
    assert bool(torch.isnan(dq[..., 0]).all())
    got = {"dq": dq[..., 1:], "dk": dk, "dv": dv}
    ref["dq"], ref["e_dq"] = ref["dq"][..., 1:], ref["e_dq"][..., 1:]
    R.check(got, ref, "backward")
    assert bool((dk[:, :, out] == 0).all()) and bool((dv[:, :, out] == 0).all())
    again = F.fibattn_cross_backward(q, k, v, o, lse, dO, n)
    for a, b in zip((dq, dk, dv), again):
        assert torch.equal(_bits(a), _bits(b))


@pytest.mark.parametrize("D", [32, 64, 128])
def test_gradients_beside_a_query_that_is_not_a_number(D):
    """float32: its own dq, and dk and dv of what it reads, are NaN; the other queries' dq is not."""
    B, H, T, S = 2, 2, 70, 150
    q, dO = _normal(250, B, H, T, D), _normal(251, B, H, T, D)
    k, v = _normal(252, B, H, S, D), _normal(253, B, H, S, D)
    q[0, 1, 33, 2] = math.nan
    o, lse = F.fibattn_cross_forward(q, k, v)
    dq, dk, dv = F.fibattn_cross_backward(q, k, v, o, lse, dO)
    assert bool(torch.isnan(dq[0, 1, 33]).all()) and int(torch.isnan(dq).sum()) == D
    assert bool(torch.isnan(dk[0, 1]).all()) and bool(torch.isnan(dv[0, 1]).all())
    assert int(torch.isnan(dk).sum()) == S * D and int(torch.isnan(dv).sum()) == S * D
