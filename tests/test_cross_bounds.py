"""The bounds that the bfloat16 attention to other states is held to (no GPU): weights in two
rounded parts keep to them, weights rounded once do not."""
import math

import pytest
import torch

from tests import cross_reference as R
from tests import cross_tight

BF = torch.bfloat16


def _parts(x, n):
    """x as the sum of its first n rounded parts."""
    y = torch.zeros_like(x)
    for _ in range(n):
        y = y + (x - y).to(BF).float()
    return y


def _emulated(q, k, v, dO, n):
    """The kernels' arithmetic in float32 torch, the weights p and dS in n bfloat16 parts."""
    tau = 1 / math.sqrt(q.shape[3])
    q, k, v, dO = (x.float() for x in (q, k, v, dO))
    s = q @ k.transpose(2, 3) * tau
    lse = torch.logsumexp(s, 3)
    m = s.amax(3, keepdim=True)
    p = torch.exp(s - m)
    o = ((_parts(p, n) @ v) / p.sum(3, keepdim=True)).to(BF)
    p = torch.exp(s - lse[..., None])
    ds = p * (dO @ v.transpose(2, 3) - (dO * o.float()).sum(3, keepdim=True))
    out = {"o": o, "lse": lse, "dq": (tau * (_parts(ds, n) @ k)).to(BF)}
    out["dk"] = (tau * (_parts(ds, n).transpose(2, 3) @ q)).to(BF)
    out["dv"] = (_parts(p, n).transpose(2, 3) @ dO).to(BF)
    return out


def _reference(q, k, v, dO, got):
    ref = cross_tight.attention(q, k, v)
    ref.update(cross_tight.gradients(q, k, v, got["o"], got["lse"], dO))
    return ref


@pytest.mark.parametrize("T,S,D", [(40, 33, 64), (90, 130, 128), (33, 257, 32)])
def test_bounds_tell_one_part_from_two(T, S, D):
    g = torch.Generator().manual_seed(3)
    q, dO = (torch.randn((1, 2, T, D), generator=g).to(BF) for _ in range(2))
    k, v = (torch.randn((1, 2, S, D), generator=g).to(BF) for _ in range(2))
    two, one = (_emulated(q, k, v, dO, n) for n in (2, 1))
    R.check(two, _reference(q, k, v, dO, two), "two parts")
    ref = _reference(q, k, v, dO, one)
    for n in ("o", "dq", "dk", "dv"):
        with pytest.raises(AssertionError):
            R.check({n: one[n]}, ref, "one part")
    # the wider bounds do not see the difference
    R.check(one, R.attention(q, k, v, dO), "one part")


def test_bounds_see_a_value_row_in_another_ones_place():
    g = torch.Generator().manual_seed(5)
    q, dO = (torch.randn((1, 1, 40, 64), generator=g).to(BF) for _ in range(2))
    k, v = (torch.randn((1, 1, 130, 64), generator=g).to(BF) for _ in range(2))
    w = v.clone()
    w[0, 0, 77] = v[0, 0, 78]
    got = _emulated(q, k, w, dO, 2)
    ref = _reference(q, k, v, dO, got)
    for n in ("o", "dq", "dk"):
        with pytest.raises(AssertionError):
            R.check({n: got[n]}, ref, "a row in another one's place")
