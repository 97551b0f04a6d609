"""bfloat16 attention to other states within the bounds of weights in two parts."""
import pytest
import torch

from paper_2606_28560_amd import fibattn as F
from tests import cross_reference as R
from tests import cross_tight
from tests.test_gpu_cross import CASES, PREFIX, _inputs, _lens

pytestmark = pytest.mark.gpu

BF = torch.bfloat16
MANY = [(BF, 4, 4, 8, 4, 1001, 130, D, [130, 0, 1, 77]) for D in (32, 64, 128)] + \
       [(BF, 8, 8, 8, 8, 1023, 90, D, None) for D in (32, 64, 128)] + \
       [(BF, 8, 8, 8, 8, 90, 1024, D, None) for D in (32, 64, 128)] + \
       [(BF, 64, 1, 8, 8, 1, 256, 64, None), (BF, 33, 1, 4, 1, 7, 40, 128, [37])]


def _name(c):
    return "-".join(str(x).replace("torch.", "") for x in c)


@pytest.mark.parametrize("case", [c for c in CASES if c[0] == BF] + MANY, ids=_name)
def test_forward_and_gradients(case):
    dtype, B, Bk, H, Hkv, T, S, D, lens = case
    print(case, flush=True)
    q, k, v, dO = _inputs(*case[:8], seed=300)
    n, keep = _lens(lens), None
    if n is not None:
        m = n.clamp(0, S)
        keep = R.lens_mask(m.expand(B) if Bk == 1 else m, T, S)
    o, lse = F.fibattn_cross_forward(q, k, v, n)
    R.check({"o": o, "lse": lse}, cross_tight.attention(q, k, v, keep=keep), "forward")
    dq, dk, dv = F.fibattn_cross_backward(q, k, v, o, lse, dO, n)
    R.check({"dq": dq, "dk": dk, "dv": dv}, cross_tight.gradients(q, k, v, o, lse, dO, keep), "backward")


@pytest.mark.parametrize("case", [c for c in PREFIX if c[0] == BF], ids=_name)
def test_prefix(case):
    dtype, B, H, Hkv, T, P, S, D, lens = case
    print(case, flush=True)
    q, k, v, _ = _inputs(dtype, B, B, H, Hkv, T, S, D, seed=310)
    _, kp, vp, _ = _inputs(dtype, B, 1, H, Hkv, T, P, D, seed=320)
    n = _lens(lens)
    m = torch.full((B,), S, device="cuda") if n is None else n
    keep = torch.cat([torch.ones((B, T, P), dtype=torch.bool, device="cuda"), R.newest_mask(m, T, S)], dim=2)
    ref = cross_tight.attention(q, torch.cat([kp.expand(B, -1, -1, -1), k], 2),
                                torch.cat([vp.expand(B, -1, -1, -1), v], 2), keep=keep)
    o, lse = F.fibattn_prefix_forward(q, kp, vp, k, v, n)
    R.check({"o": o, "lse": lse}, ref, "prefix")
