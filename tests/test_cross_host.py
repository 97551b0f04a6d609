"""Refusals of the attention to other states, before any launch (no GPU)."""
import ctypes

import pytest
import torch

from paper_2606_28560_amd import fibattn as F

P = 4096  # an aligned address that is never followed: every call here is refused first
BIG = 1 << 40


def forward(q=P, k=P, v=P, o=P, lse=P, lens=None, ws=P, bytes_=BIG, lay=None, B=2, Bk=2, H=4, Hkv=2, T=8, S=40, D=64,
            dtype=1):
    return F.lib().fibattn_cross_forward(q, k, v, o, lse, lens, ws, bytes_, lay, B, Bk, H, Hkv, T, S, D, dtype, None)


def backward(q=P, k=P, v=P, o=P, lse=P, g=P, dq=P, dk=P, dv=P, lens=None, ws=P, bytes_=BIG, lay=None, B=2, Bk=2, H=4,
             Hkv=2, T=8, S=40, D=64, dtype=1):
    return F.lib().fibattn_cross_backward(q, k, v, o, lse, g, dq, dk, dv, lens, ws, bytes_, lay, B, Bk, H, Hkv, T, S,
                                          D, dtype, None)


def prefix(q=P, kp=P, vp=P, k=P, v=P, o=P, lse=P, lens=None, ws=P, bytes_=BIG, lay=None, B=2, H=4, Hkv=2, T=8, n=100,
           S=40, D=64, dtype=1):
    return F.lib().fibattn_prefix_forward(q, kp, vp, k, v, o, lse, lens, ws, bytes_, lay, B, H, Hkv, T, n, S, D, dtype,
                                          None)


def join(a=P, la=P, b=P, lb=P, o=P, lse=P, lay=None, B=2, H=4, T=8, D=64, dtype=1):
    return F.lib().fibattn_join(a, la, b, lb, o, lse, lay, B, H, T, D, dtype, None)


def layouts(*rows):
    return (ctypes.c_int64 * (3 * len(rows)))(*[x for r in rows for x in r])


@pytest.mark.parametrize("call,names", [(forward, "q k v o lse"), (backward, "q k v o lse g dq dk dv"),
                                        (prefix, "q kp vp k v o lse"), (join, "a la b lb o lse")])
def test_pointers(call, names):
    for n in names.split():
        assert call(**{n: None}) == 1, n
        assert call(**{n: P + 8}) == 1, n
    if call is not join:
        assert call(lens=P + 2) == 1


@pytest.mark.parametrize("call", [forward, backward, prefix, join])
def test_sizes(call):
    for bad in ({"B": 0}, {"H": 0}, {"T": 0}, {"T": -5}, {"dtype": 2}, {"dtype": -1}):
        assert call(**bad) == 1, bad
    for bad in ({"D": 48}, {"D": 256}, {"D": 0}, {"B": 65536, **({} if call in (join, prefix) else {"Bk": 1})},
                {"T": 1 << 30}):
        assert call(**bad) == 2, bad
    if call is join:
        return
    for bad in ({"S": 0}, {"Hkv": 0}, {"Hkv": 3}, {"Hkv": 8}):
        assert call(**bad) == 1, bad
    assert call(S=(1 << 30) + 1) == 2
    if call is prefix:
        assert call(n=0) == 1 and call(n=(1 << 30) + 1) == 2
    else:
        assert call(Bk=3) == 1 and call(Bk=0) == 1


def test_workspaces():
    L = F.lib()
    need = L.fibattn_cross_workspace_bytes(1, 1, 4, 4, 1, 4000, 64)
    assert need > 0 and need % 16 == 0
    kw = dict(B=1, Bk=1, H=4, Hkv=4, T=1, S=4000)
    assert forward(**kw, ws=None) == 3 and forward(**kw, bytes_=need - 1) == 3 and forward(**kw, ws=P + 8) == 3
    # many rows over short states: one piece, no workspace
    assert L.fibattn_cross_workspace_bytes(8, 8, 8, 8, 1024, 64, 64) == 0
    need = L.fibattn_cross_backward_workspace_bytes(2, 2, 4, 2, 8, 40, 64)
    assert need > 0
    assert backward(ws=None) == 3 and backward(bytes_=need - 1) == 3 and backward(ws=P + 8) == 3
    need = L.fibattn_prefix_workspace_bytes(2, 4, 2, 8, 100, 40, 64)
    assert need > 0
    assert prefix(ws=None) == 3 and prefix(bytes_=need - 1) == 3 and prefix(ws=P + 8) == 3
    for f in (L.fibattn_cross_workspace_bytes, L.fibattn_cross_backward_workspace_bytes):
        assert f(0, 0, 4, 4, 1, 10, 64) == 0 and f(2, 3, 4, 4, 1, 10, 64) == 0 and f(2, 2, 4, 4, 1, 10, 48) == 0
    assert L.fibattn_prefix_workspace_bytes(2, 4, 2, 8, 0, 40, 64) == 0


def test_layouts():
    ok = (4096, 1024, 64)
    for call, n in ((forward, 4), (backward, 8), (prefix, 6), (join, 3)):
        for a in range(n):
            for bad in ((-64, 1024, 64), (4096, 1028, 64), (4096, 1024, 36), (4097, 1024, 64)):
                assert call(lay=layouts(*[bad if i == a else ok for i in range(n)])) == 1, (call, a, bad)
            assert call(lay=layouts(*[(0, 0, 1 << 22) if i == a else ok for i in range(n)])) == 2, (call, a)


def test_binding_refuses_host_tensors_and_bad_shapes():
    q, k = torch.zeros(1, 2, 3, 64), torch.zeros(1, 2, 5, 64)
    lse = torch.zeros(1, 2, 3)
    with pytest.raises(ValueError):
        F.fibattn_cross_forward(q, k, k)
    with pytest.raises(ValueError):
        F.fibattn_cross_backward(q, k, k, q, lse, q)
    with pytest.raises(ValueError):
        F.fibattn_prefix_forward(q, k, k, k, k)
    with pytest.raises(ValueError):
        F.fibattn_join(q, lse, q, lse)
