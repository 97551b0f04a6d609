"""Attention to other states in 64 bits, and bounds of what 32-bit sums and the storage
type's roundings may add to it (test infrastructure).

A value computed as sum_j w_j x_j with weights rounded to the storage type (relative error
u, at most half a step: 2^-8 in bfloat16, none in float32), summed in float32 and stored
(relative error us: 2^-8 or 2^-24) is off by at most (u + g) sum |w_j x_j| + us |value|.
g = n 2^-24 counts the float32 operations one after the other: n terms of the sums, and the
error of a logit, whose products and exponent add (D + 8) 2^-24 tau sum |q_i k_i| to it
(float32 products of three bfloat16 parts, two of the nine left out at 2^-24 each, among them).
The gradient's Delta = <dO, o> takes the stored o, so that o's own bound enters dS.
"""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
STORE = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def attention(q, k, v, dO=None, keep=None, extra=None):
    """float64 o, lse (and dq, dk, dv with dO), and the bounds "e_*" of each.

    q [B,H,T,D]; k, v [B or 1,H_kv,S,D]; keep: bool [B,T,S] (None: all); rows of k and v that
    no query keeps may hold anything.  extra: float64 (o, lse) [B,H,T,..] of further keys in
    the same softmax (their own bounds are not counted)."""
    dt, (B, H, T, D), (Bk, Hkv, S, _) = q.dtype, q.shape, k.shape
    u, us, tau, G = HALF[dt], STORE[dt], 1.0 / math.sqrt(D), H // Hkv
    if keep is None:
        keep = torch.ones((B, T, S), dtype=torch.bool, device=q.device)
    read = keep.any(dim=1)  # [B,S]: rows some query reads; the others never enter
    if Bk == 1:
        read = read.any(dim=0, keepdim=True)
    q, k, v = q.double(), k.double(), v.double()
    k, v = (torch.where(read[:, None, :, None], x, torch.zeros_like(x)) for x in (k, v))
    kk, vv = (x.expand(B, Hkv, S, D).repeat_interleave(G, dim=1) for x in (k, v))
    keep = keep[:, None].expand(B, H, T, S)
    s = torch.matmul(q, kk.transpose(2, 3)) * tau
    s = torch.where(keep, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, dim=3)
    both = lse if extra is None else torch.logaddexp(lse, extra[1])
    ref = torch.where(both == -math.inf, torch.zeros_like(both), both)
    p = torch.where(keep, torch.exp(s - ref[..., None]), torch.zeros_like(s))
    o = torch.matmul(p, vv)
    if extra is not None:
        w = torch.where(both == -math.inf, torch.zeros_like(both), torch.exp(extra[1] - ref))
        o = o + w[..., None] * extra[0]
    size = (torch.matmul(q.abs(), kk.abs().transpose(2, 3)) * tau).amax(dim=3, keepdim=True)
    ds = (D + 8) * 2.0 ** -24 * size  # of a logit
    g = (S + 16) * 2.0 ** -24 + 2 * ds
    out = {"o": o, "lse": both}
    e_o = (u + g) * torch.matmul(p, vv.abs()) + us * o.abs()
    if extra is not None:
        e_o = e_o + (2 * us + g) * (w[..., None] * extra[0].abs())
    out["e_o"] = e_o
    out["e_lse"] = g[..., 0] + 2.0 ** -22 * (ref.abs() + 1)
    if dO is None:
        return out
    dO = dO.double()
    dp = torch.matmul(dO, vv.transpose(2, 3))
    delta = (dO * o).sum(3, keepdim=True)
    d = p * (dp - delta)
    e_delta = (dO.abs() * e_o).sum(3, keepdim=True) + D * 2.0 ** -24 * (dO.abs() * o.abs()).sum(3, keepdim=True)
    e_dp = D * 2.0 ** -24 * torch.matmul(dO.abs(), vv.abs().transpose(2, 3))
    e_d = (u + g) * d.abs() + p * (e_delta + e_dp)
    rows = (B // Bk * G * T + 64) * 2.0 ** -24

    def fold(x):  # query heads of a group, and the batch entries that share the states
        x = x.reshape(B, Hkv, G, S, D).sum(2)
        return x.sum(0, keepdim=True) if Bk == 1 else x

    def tr(x):
        return x.transpose(2, 3).contiguous()

    out["dq"] = tau * torch.matmul(d, kk)
    out["e_dq"] = tau * torch.matmul(e_d + (S + 64) * 2.0 ** -24 * d.abs(), kk.abs()) + us * out["dq"].abs()
    out["dk"] = tau * fold(torch.matmul(tr(d), q))
    out["e_dk"] = tau * fold(torch.matmul(tr(e_d + rows * d.abs()), q.abs())) + us * out["dk"].abs()
    out["dv"] = fold(torch.matmul(tr(p), dO))
    out["e_dv"] = fold(torch.matmul(tr((u + g + rows) * p), dO.abs())) + us * out["dv"].abs()
    return out


def check(got, ref, what):
    """Every value of `got` within its bound; non-finite values must be the same."""
    for n, x in got.items():
        x, r, e = x.double(), ref[n], ref["e_" + n]
        assert x.shape == r.shape, (what, n, x.shape, r.shape)
        fin = torch.isfinite(r)
        assert torch.equal(x[~fin].nan_to_num(), r[~fin].nan_to_num()), f"{what}: {n} where not finite"
        assert torch.isfinite(x[fin]).all(), f"{what}: {n} is not finite"
        err = torch.where(fin, (x - r).abs() - e, torch.zeros_like(r))
        at = int(err.argmax())
        assert float(err.max()) <= 0, (f"{what}: {n} off by {float((x - r).abs().flatten()[at]):.3e}, bound "
                                       f"{float(e.flatten()[at]):.3e}, value {float(r.flatten()[at]):.3e}")


def lens_mask(lens, T, S):
    """keep [B,T,S] of every query reading the first lens[b] rows."""
    j = torch.arange(S, device=lens.device)
    return (j[None, :] < lens[:, None])[:, None, :].expand(lens.shape[0], T, S)


def newest_mask(lens, T, S):
    """keep [B,T,S] of query t reading the rows j <= lens[b] - T + t."""
    j, t = torch.arange(S, device=lens.device), torch.arange(T, device=lens.device)
    return j[None, None, :] <= (lens[:, None] - T + t[None, :])[:, :, None]
