"""Refusals and sizes of the class layer on rows that need no GPU: they come before any launch."""
import ctypes as C

import pytest

from paper_1302_1690_amd import mpcnn

BASE = 1 << 40
GOOD = dict(x=BASE, x_pitch=16, w=2 * BASE, w_pitch=16, bias=3 * BASE, labels=4 * BASE, roww=5 * BASE, rows=20, features=16, classes=30, dtype=0,
            rowloss=6 * BASE, lse=7 * BASE, loss=8 * BASE, dx=9 * BASE, dx_pitch=16, dw=10 * BASE, db=11 * BASE, ws=12 * BASE, ws_bytes=1 << 30)


def _call(backward, **change):
    a = dict(GOOD, **change)
    L = mpcnn.lib()
    head = [a[k] for k in ("x", "x_pitch", "w", "w_pitch", "bias", "labels", "roww", "rows", "features", "classes", "dtype", "rowloss")]
    tail = [a["ws"], a["ws_bytes"], None]
    if backward:
        return L.mpcnn_class_backward(*head, a["loss"], a["dx"], a["dx_pitch"], a["dw"], a["db"], *tail)
    return L.mpcnn_class_loss(*head, a["lse"], a["loss"], *tail)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), 1), (dict(w=None), 1), (dict(labels=None), 1), (dict(ws=None), 1), (dict(rows=-1), 1), (dict(features=0), 1), (dict(classes=0), 1),
    (dict(dtype=2), 1), (dict(dtype=-1), 1), (dict(x_pitch=15), 1), (dict(w_pitch=0), 1), (dict(w_pitch=-16), 1), (dict(x_pitch=1 << 41), 1),
    (dict(x=BASE + 2), 1), (dict(dtype=1, w=2 * BASE + 1), 1), (dict(bias=3 * BASE + 2), 1), (dict(labels=4 * BASE + 1), 1), (dict(roww=5 * BASE + 3), 1),
    (dict(rowloss=6 * BASE + 2), 1), (dict(loss=8 * BASE + 4), 1), (dict(ws=12 * BASE + 128), 1), (dict(ws_bytes=100), 3),
    (dict(rows=(1 << 20) + 1), 4), (dict(features=(1 << 20) + 1, x_pitch=1 << 21, w_pitch=1 << 21, dx_pitch=1 << 21), 4), (dict(classes=1 << 31), 4),
    (dict(rowloss=BASE + 64), 1), (dict(ws=2 * BASE), 1), (dict(rowloss=12 * BASE + 256), 1), (dict(loss=6 * BASE + 72), 1),
], ids=range(29))
@pytest.mark.parametrize("backward", [False, True])
def test_refusals(change, status, backward):
    assert _call(backward, **change) == status, mpcnn.lib().mpcnn_last_error().decode()
    assert mpcnn.lib().mpcnn_last_error()


@pytest.mark.parametrize("change", [dict(dx=BASE + 64), dict(dw=2 * BASE + 1916), dict(db=3 * BASE), dict(dx_pitch=15), dict(dx=9 * BASE + 1), dict(dw=10 * BASE + 2),
                                    dict(dw=9 * BASE + 1276), dict(db=6 * BASE + 76)])
def test_refusals_of_the_backward(change):
    assert _call(True, **change) == 1


def test_workspace():
    size = mpcnn.class_workspace_bytes
    assert size(-1, 16, 30, 0, True) == size(20, 0, 30, 0, True) == size(20, 16, 0, 0, True) == size(20, 16, 30, 2, True) == 0
    assert size((1 << 20) + 1, 16, 30, 0, False) == 0
    assert size(0, 16, 30, 0, True) > 0
    for dtype in (0, 1):
        # no room for the scores of everything: with a vocabulary ten times as large the workspace grows by what the loss's statistics take
        a, b = size(8192, 1024, 50000, dtype, True), size(8192, 1024, 500000, dtype, True)
        assert b - a < 8192 * 8 * (500000 // 128 + 64)
        assert a < 8192 * 50000 * 4 * 2
