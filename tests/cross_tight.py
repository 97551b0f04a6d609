"""Closer bounds than cross_reference's of the attention to other states (test infrastructure).

A bfloat16 weight goes into its product as a rounded part and that part's rounded rest, each
off by at most half a step (2^-8 of it), so the weight is off by at most 2^-8 2^-8 = 2^-16
(cross_reference allows 2^-8, which one rounded part would keep to).  And the gradients are
compared with the formula's on the o and lse that the call was given, so that the rounding of
o, which their Delta = <dO, o> takes, has no part in their bounds.  Everything else is as in
cross_reference."""
import math

import torch

from tests import cross_reference as R

U = {torch.bfloat16: 2.0 ** -16, torch.float32: 0.0}


def attention(*args, **kw):
    """cross_reference.attention with weights in two parts."""
    loose = R.HALF[torch.bfloat16]
    R.HALF[torch.bfloat16] = U[torch.bfloat16]
    try:
        return R.attention(*args, **kw)
    finally:
        R.HALF[torch.bfloat16] = loose


def gradients(q, k, v, o, lse, dO, keep=None):
    """float64 dq, dk, dv of p = exp(s - lse), dS = p (<dO, v> - <dO, o>) with the given o and
    lse, and their bounds; keep as in cross_reference."""
    dt, (B, H, T, D), (Bk, Hkv, S, _) = q.dtype, q.shape, k.shape
    u, us, tau, G, e = U[dt], R.STORE[dt], 1.0 / math.sqrt(D), H // Hkv, 2.0 ** -24
    if keep is None:
        keep = torch.ones((B, T, S), dtype=torch.bool, device=q.device)
    read = keep.any(dim=1)
    if Bk == 1:
        read = read.any(dim=0, keepdim=True)
    q, k, v, o, dO, lse = (x.double() for x in (q, k, v, o, dO, lse))
    k, v = (torch.where(read[:, None, :, None], x, torch.zeros_like(x)) for x in (k, v))
    kk, vv = (x.expand(B, Hkv, S, D).repeat_interleave(G, dim=1) for x in (k, v))
    keep = keep[:, None].expand(B, H, T, S) & (lse > -math.inf)[..., None]

    def tr(x):
        return x.transpose(2, 3).contiguous()

    ref = torch.where(lse > -math.inf, lse, torch.zeros_like(lse))[..., None]
    p = torch.where(keep, torch.exp(torch.matmul(q, tr(kk)) * tau - ref), torch.zeros_like(ref))
    delta = (dO * o).sum(3, keepdim=True)
    d = p * (torch.matmul(dO, tr(vv)) - delta)
    # of a weight: a logit's products (D + 8 roundings), lse log2 e and its subtraction (4 of |lse|), 8 more
    size = (torch.matmul(q.abs(), tr(kk.abs())) * tau).amax(dim=3, keepdim=True)
    g = 2 * ((D + 8) * e * size + 4 * e * ref.abs()) + 8 * e
    e_u = (D + 4) * e * (torch.matmul(dO.abs(), tr(vv.abs())) + (dO.abs() * o.abs()).sum(3, keepdim=True))
    e_d = (u + g) * d.abs() + p * e_u
    rows = (B // Bk * G * T + 64) * e

    def fold(x):  # query heads of a group, and the batch entries that share the states
        x = x.reshape(B, Hkv, G, S, D).sum(2)
        return x.sum(0, keepdim=True) if Bk == 1 else x

    out = {"dq": tau * torch.matmul(d, kk), "dk": tau * fold(torch.matmul(tr(d), q)), "dv": fold(torch.matmul(tr(p), dO))}
    out["e_dq"] = tau * torch.matmul(e_d + (S + 64) * e * d.abs(), kk.abs()) + us * out["dq"].abs()
    out["e_dk"] = tau * fold(torch.matmul(tr(e_d + rows * d.abs()), q.abs())) + us * out["dk"].abs()
    out["e_dv"] = fold(torch.matmul(tr((u + g + rows) * p), dO.abs())) + us * out["dv"].abs()
    return out
