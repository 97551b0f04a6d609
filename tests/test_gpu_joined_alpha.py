"""The gradient of alpha (and theta) of a sparse self-attention layer whose rows are a part of
a softmax: its queries also read rows that the batch shares (fibattn_cross_forward,
fibattn_join), against 64 bits."""
import math

import pytest
import torch

from paper_2606_28560_amd import fibattn as F
from paper_2606_28560_amd import schedules

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32


def _inputs(dtype, B, H, Hkv, T, M, D, seed):
    """Queries and keys that alternate along one direction with the position, so that a rung's
    <q, k[r1] - k[r0]> has one sign, and shared values that lie along dO: the sums over the
    queries do not cancel, and the shared rows have a part in Delta."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    q, dO = 0.5 * normal(B, H, T, D), 0.25 * normal(B, H, T, D)
    k, v = 0.5 * normal(B, Hkv, T, D), 0.5 * normal(B, Hkv, T, D)
    km, vm = 0.5 * normal(1, Hkv, M, D), 0.5 * normal(1, Hkv, M, D)
    sign = 1.0 - 2.0 * (torch.arange(T, device="cuda") % 2)
    q[..., 0] = 2.0 * sign
    k[..., 0] += 2.0 * sign
    dO[..., 1] = 2.0
    vm[..., 1] += 6.0
    return [x.to(dtype) for x in (q, k, v, km, vm, dO)]


class Layer:
    """The layer's entries in 64 bits: the window, the rungs (the last n), the shared rows."""

    def __init__(self, q, k, v, km, vm, dO, W, rungs):
        B, H, T, D = q.shape
        G, self.tau, self.n, self.D = H // k.shape[1], 1 / math.sqrt(D), len(rungs), D
        self.dtype = q.dtype
        q, dO = q.double(), dO.double()
        k, v, km, vm = (x.double().repeat_interleave(G, dim=1) for x in (k, v, km, vm))
        self.dO = dO
        i = torch.arange(T, device="cuda")

        def back(x, d):  # row i - d of every query (a zero row before the first)
            d = min(d, T)
            return torch.cat([torch.zeros((B, H, d, D), device="cuda", dtype=x.dtype), x[:, :, :T - d]], 2)

        s, g, a, has, ds, dv, dsz, dvz = ([] for _ in range(8))
        for d, w in [(d, 0.0) for d in range(W + 1)] + [(d0, float(w)) for d0, w, _ in rungs]:
            k0, k1, v0, v1 = back(k, d), back(k, d + 1), back(v, d), back(v, d + 1)
            vb = (1 - w) * v0 + w * v1
            s.append((q * ((1 - w) * k0 + w * k1)).sum(3) * self.tau)
            g.append((dO * vb).sum(3)), a.append((dO.abs() * vb.abs()).sum(3))
            has.append((i >= d) if w == 0.0 else (i > d))
            # along the blend, and what their float32 sums are relative to
            ds.append((q * (k1 - k0)).sum(3)), dv.append((dO * (v1 - v0)).sum(3))
            dsz.append((q.abs() * (k1.abs() + k0.abs())).sum(3)), dvz.append((dO.abs() * (v0.abs() + v1.abs())).sum(3))
        self.s, self.g, self.a = torch.stack(s), torch.stack(g), torch.stack(a)
        self.has = torch.stack(has)[:, None, None, :].expand(self.s.shape)
        n = self.n
        self.ds, self.dv, self.dsz, self.dvz = (torch.stack(x[-n:]) for x in (ds, dv, dsz, dvz))
        self.f = torch.tensor([r[2] for r in rungs], device="cuda", dtype=torch.float64)[:, None, None, None]
        self.sm = torch.matmul(q, km.transpose(2, 3).contiguous()) * self.tau
        self.gm = torch.matmul(dO, vm.transpose(2, 3).contiguous())
        self.am = torch.matmul(dO.abs(), vm.abs().transpose(2, 3).contiguous())
        # a logit's products in magnitude, at most
        keys = torch.cat([k, km.expand(B, -1, -1, -1)], 2).abs().transpose(2, 3).contiguous()
        self.mag = float(torch.matmul(q.abs(), keys).max()) * self.tau

    def weights(self, lse):
        return torch.where(self.has, torch.exp(self.s - lse.double()), torch.zeros_like(self.s))

    def given(self, lse, delta):
        """dalpha of the formula on a given lse and Delta."""
        p = self.weights(lse)[-self.n:]
        return float((self.f * (self.tau * p * (self.g[-self.n:] - delta) * self.ds + p * self.dv)).sum())

    def own_delta(self, lse):
        return (self.weights(lse) * self.g).sum(0)

    def stored_delta(self, o):
        return (self.dO * o.double()).sum(3)

    def arithmetic(self, lse, o):
        """What float32 arithmetic may add to `given`: sums of D products, each relative to the
        sum of their magnitudes (16 more roundings for the products of the terms); the weight's
        exponent takes the errors of a logit (D + 8 roundings) and of lse log2 e (three)."""
        rel = 2.0 ** -24 * ((self.D + 8) * self.mag + 3 * float(lse.abs().max()) + 4 * (self.D + 16))
        p = self.weights(lse)[-self.n:]
        big = (self.dO.abs() * o.double().abs()).sum(3)
        return rel * float((self.f * p * (self.tau * (self.dvz + big) * self.dsz + self.dvz)).sum())

    def rounding(self, lse, joined):
        """What the roundings of the stored o add by Delta: bfloat16 rounds the sparse weights, the
        parts' o and the joined o, each by at most 2^-8 of sum p |dO| |v|; float32 sums of
        n entries (D of a logit beside) 2^-24 each."""
        p = self.weights(lse)
        a = (p * self.a).sum(0)
        if joined:
            a = a + (torch.exp(self.sm - lse.double()[..., None]) * self.am).sum(3)
        u = (3 * 2.0 ** -8 if self.dtype == BF else 0) + 2.0 ** -24 * (self.s.shape[0] + 3 * self.D * (1 + self.mag))
        return u * float((self.f * p[-self.n:] * self.tau * self.ds.abs() * a).sum())

    def differentiated(self, joined):
        """The gradient by differentiation of the layer."""
        n = self.n
        w = torch.zeros((n, 1, 1, 1), device="cuda", dtype=torch.float64, requires_grad=True)
        z = torch.cat([self.s[:-n], self.s[-n:] + self.tau * w * self.ds])
        z = torch.where(self.has, z, torch.full_like(z, -math.inf)).permute(1, 2, 3, 0)
        y = torch.cat([self.g[:-n], self.g[-n:] + w * self.dv]).permute(1, 2, 3, 0)
        if joined:
            z, y = torch.cat([z, self.sm], 3), torch.cat([y, self.gm], 3)
        loss = (torch.softmax(z, 3) * y).sum()
        return float((self.f * torch.autograd.grad(loss, w)[0]).sum())


# (dtype, B, H, Hkv, T, M, D, W, alpha): each family of backward kernels, integer and blended rungs
CASES = [
    (BF, 2, 8, 2, 200, 40, 64, 8, 1.0),
    (BF, 2, 4, 4, 333, 17, 64, 8, 0.9),
    (BF, 1, 4, 2, 260, 64, 64, 24, 0.9),
    (BF, 2, 4, 4, 200, 40, 128, 8, 1.0),
    (BF, 2, 2, 1, 150, 33, 32, 10, 0.7),
    (FP, 2, 4, 4, 200, 40, 32, 8, 1.0),
    (FP, 1, 4, 2, 300, 40, 64, 8, 0.9),
    (FP, 4, 8, 8, 512, 20, 64, 8, 0.9),
    (FP, 1, 2, 2, 130, 9, 128, 3, 0.9),
]


@pytest.mark.parametrize("how", ["host", "strided", "device"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_joined_dalpha(case, how):
    dtype, B, H, Hkv, T, M, D, W, alpha = case
    print(case, how, flush=True)
    base = schedules.FIB15
    q, k, v, km, vm, dO = _inputs(dtype, B, H, Hkv, T, M, D, seed=7)
    theta = torch.tensor([math.log((alpha - 0.5) / (1.5 - alpha))], device="cuda")
    if how == "device":
        al = torch.empty(1, device="cuda")
        table = F.fibattn_device_table_theta(theta, base, W, alpha=al)
        alpha = float(al)
        o1, l1 = F.fibattn_forward_dt(q, k, v, W, table)
    else:
        if how == "strided":
            q, k, v, dO = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v, dO))
        o1, l1 = F.fibattn_forward(q, k, v, W, base, alpha)
    o2, l2 = F.fibattn_cross_forward(q, km, vm)
    o, lse = F.fibattn_join(o1, l1, o2, l2)
    dtheta = torch.full((1,), math.nan, device="cuda")
    if how == "device":
        got = F.fibattn_backward_dt(q, k, v, o, lse, dO, W, table, dtheta=dtheta, joined=True)
        plain = F.fibattn_backward_dt(q, k, v, o, lse, dO, W, table)
    else:
        got = F.fibattn_backward(q, k, v, o, lse, dO, W, base, alpha, joined=True)
        plain = F.fibattn_backward(q, k, v, o, lse, dO, W, base, alpha)
    for a, b in zip(got[:3], plain[:3]):  # dq, dk, dv are the same either way
        assert torch.equal(a, b)
    dalpha = float(got[3])

    x = Layer(q, k, v, km, vm, dO, W, F.fibattn_rung_table(alpha, base, W))
    # the formula on what the call was given, lse and Delta = <dO, o>
    want, near = x.given(lse, x.stored_delta(o)), x.arithmetic(lse, o)
    assert abs(dalpha - want) <= near + 2.0 ** -23 * abs(want), (dalpha, want, near)
    # the gradient itself
    true, tol = x.differentiated(True), 2 * near + x.rounding(lse, True)
    assert abs(dalpha - true) <= tol, (dalpha, true, tol)
    # with the Delta of the sparse rows alone it would be another number
    assert abs(x.given(lse, x.own_delta(lse)) - true) > 2 * tol
    if how == "device":
        sig = 1 / (1 + math.exp(-float(theta)))
        assert abs(float(dtheta) - dalpha * sig * (1 - sig)) <= 2.0 ** -20 * abs(dalpha)


@pytest.mark.parametrize("dtype,W,D", [(BF, 8, 64), (BF, 24, 64), (BF, 8, 128), (FP, 8, 64)])
def test_joined_of_the_whole_softmax(dtype, W, D):
    """Where the sparse rows are all of it, both ways give the gradient."""
    B, H, T, base = 2, 4, 256, schedules.FIB15
    q, k, v, km, vm, dO = _inputs(dtype, B, H, H, T, 4, D, seed=9)
    o, lse = F.fibattn_forward(q, k, v, W, base, 0.9)
    a = F.fibattn_backward(q, k, v, o, lse, dO, W, base, 0.9)
    b = F.fibattn_backward(q, k, v, o, lse, dO, W, base, 0.9, joined=True)
    for x, y in zip(a[:3], b[:3]):
        assert torch.equal(x, y)
    x = Layer(q, k, v, km, vm, dO, W, F.fibattn_rung_table(0.9, base, W))
    tol = 2 * x.arithmetic(lse, o) + x.rounding(lse, False)
    for g in (a[3], b[3]):
        assert abs(float(g) - x.differentiated(False)) <= tol


def test_joined_in_a_graph_and_on_a_stream():
    B, H, T, M, D, W, base = 2, 4, 128, 16, 64, 8, schedules.FIB15
    q, k, v, km, vm, dO = _inputs(BF, B, H, H, T, M, D, seed=11)

    def step():
        o1, l1 = F.fibattn_forward(q, k, v, W, base, 0.9)
        o2, l2 = F.fibattn_cross_forward(q, km, vm)
        o, lse = F.fibattn_join(o1, l1, o2, l2)
        return F.fibattn_backward(q, k, v, o, lse, dO, W, base, 0.9, joined=True)

    want = [x.clone() for x in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for r in range(3):
        q.mul_(0.75)
        want = [x.clone() for x in step()]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), r
