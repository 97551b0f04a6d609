"""Refusals of fibattn_backward_joined, before any launch (no GPU)."""
import ctypes

import pytest

from paper_2606_28560_amd import fibattn as F
from paper_2606_28560_amd import schedules

BASE = (ctypes.c_int32 * 15)(*schedules.FIB15)
P = 4096  # an aligned address that is never followed: every call here is refused first
NAMES = "q k v o lse g dq dk dv dalpha".split()


def call(ptrs=None, dtheta=None, ws=P, bytes_=1 << 40, lay=None, B=2, H=4, Hkv=2, T=8, D=64, W=8, base=BASE, K=15,
         alpha=1.0, table=None, rope=0.0, dtype=1):
    p = [dict.fromkeys(NAMES, P), ptrs or {}]
    return F.lib().fibattn_backward_joined(*({**p[0], **p[1]}[n] for n in NAMES), dtheta, ws, bytes_, lay, B, H, Hkv, T,
                                           D, W, base, K, ctypes.c_float(alpha), table, ctypes.c_float(rope), dtype, None)


def layouts(*rows):
    return (ctypes.c_int64 * (3 * len(rows)))(*[x for r in rows for x in r])


@pytest.mark.parametrize("table", [None, P])
def test_refusals(table):
    for n in NAMES:
        assert call({n: None}, table=table) == 1, n
        if n != "dalpha":
            assert call({n: P + 8}, table=table) == 1, n
    for bad in ({"B": 0}, {"T": 0}, {"Hkv": 0}, {"Hkv": 3}, {"Hkv": 8}, {"W": -1}, {"dtype": 7}, {"rope": 0.5}):
        assert call(table=table, **bad) == 1, bad
    for bad in ({"D": 48}, {"W": 129}, {"B": 65536}):
        assert call(table=table, **bad) == 2, bad
    assert call(table=table, ws=None) == 3 and call(table=table, bytes_=255) == 3 and call(table=table, ws=P + 8) == 3


def test_host_and_device_tables_do_not_mix():
    ok = (4096, 1024, 64)
    assert call(dtheta=P) == 1  # theta belongs to a device table
    assert call(table=P + 8) == 1
    assert call(table=P, lay=layouts(*[ok] * 8)) == 1  # a device table comes with packed tensors
    assert call(base=None) == 1 and call(alpha=-1.0) == 1
    for a in range(8):
        assert call(lay=layouts(*[(4096, 1024, 36) if i == a else ok for i in range(8)])) == 1, a
        assert call(lay=layouts(*[(0, 0, 1 << 30) if i == a else ok for i in range(8)])) == 2, a


def test_workspace_is_that_of_the_other_calls():
    ws = F.fibattn_backward_workspace_bytes
    assert call(bytes_=ws(2, 4, 8, 64, 8, 15) - 1) == 3
    assert call(table=P, bytes_=ws(2, 4, 8, 64, 8, 0) - 1) == 3
