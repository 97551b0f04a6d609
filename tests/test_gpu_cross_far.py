"""Attention to other states, forward and backward, with rows and heads that lie past 2^32 bytes."""
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


@pytest.mark.parametrize("dtype", [BF, FP])
def test_rows_past_4_gigabytes(dtype):
    """Every tensor's rows almost 2^22 elements apart, so that a head's later rows lie past 2^32
    bytes: the results of packed tensors, forward and backward."""
    H, T, S, D, apart = 1, 700, 650, 64, (1 << 22) - 64
    es = 2 if dtype == BF else 4
    assert (S - 1) * apart * es > 1 << 32
    buf = torch.empty(max(T, S) * apart, device="cuda", dtype=dtype)
    places = {n: torch.as_strided(buf, (1, H, r, D), (0, 0, apart, 1), 64 * a)
              for a, (n, r) in enumerate((("q", T), ("k", S), ("v", S), ("o", T), ("dO", T), ("dq", T), ("dk", S), ("dv", S)))}
    q, dO = _normal(260, 1, H, T, D, dtype=dtype), _normal(261, 1, H, T, D, dtype=dtype)
    k, v = _normal(262, 1, H, S, D, dtype=dtype), _normal(263, 1, H, S, D, dtype=dtype)
    for n, x in (("q", q), ("k", k), ("v", v), ("dO", dO)):
        places[n].copy_(x)
    lens = torch.tensor([S - 7], dtype=torch.int32, device="cuda")
    o, lse = F.fibattn_cross_forward(q, k, v, lens)
    want = (o, lse, *F.fibattn_cross_backward(q, k, v, o, lse, dO, lens))
    p = places
    o2, lse2 = F.fibattn_cross_forward(p["q"], p["k"], p["v"], lens, o=p["o"])
    got = (o2, lse2, *F.fibattn_cross_backward(p["q"], p["k"], p["v"], o2, lse2, p["dO"], lens, dq=p["dq"], dk=p["dk"], dv=p["dv"]))
    for a, b in zip(got, want):
        assert torch.equal(_bits(a), _bits(b))
    R.check({"o": o, "lse": lse}, R.attention(q, k, v, keep=R.lens_mask(lens, T, S)), "packed")


def test_heads_past_4_gigabytes():
    """A second head 4.3 GB behind the first, in the states and their gradients."""
    T, S, D, apart = 40, 100, 64, (1 << 31) + 4096
    buf = torch.empty(apart + 5 * S * D, device="cuda", dtype=BF)
    places = [torch.as_strided(buf, (1, 2, S, D), (0, apart, D, 1), a * S * D) for a in range(4)]
    q, dO = _normal(270, 1, 4, T, D, dtype=BF), _normal(271, 1, 4, T, D, dtype=BF)
    k, v = _normal(272, 1, 2, S, D, dtype=BF), _normal(273, 1, 2, S, D, dtype=BF)
    places[0].copy_(k), places[1].copy_(v)
    o, lse = F.fibattn_cross_forward(q, k, v)
    want = (o, lse, *F.fibattn_cross_backward(q, k, v, o, lse, dO))
    o2, lse2 = F.fibattn_cross_forward(q, places[0], places[1])
    got = (o2, lse2, *F.fibattn_cross_backward(q, places[0], places[1], o2, lse2, dO, dk=places[2], dv=places[3]))
    for a, b in zip(got, want):
        assert torch.equal(_bits(a), _bits(b))
