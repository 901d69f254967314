"""Refusals of the weights' gradient from rows in 8 bits that need no GPU: they come before any launch."""
import ctypes as C

import pytest
import torch

from paper_1302_1690_amd import mpcnn

BASE = 1 << 40
EINVAL, EWORKSPACE, EUNSUPPORTED = 1, 3, 4
GOOD = dict(dy=BASE, pitch=60, x=(2 * BASE, 3 * BASE, 2), rows=5000, outs=60, features=40, dtype=0, dw=4 * BASE, dw_dtype=0, ws=5 * BASE, ws_bytes=1 << 30)


def _call(**change):
    a = dict(GOOD, **change)
    a["x"] = None if a["x"] is None else C.byref(mpcnn._Packed(*a["x"]))
    return mpcnn.lib().mpcnn_rows_weight_grad(*a.values(), None)


@pytest.mark.parametrize("change,status", [
    (dict(dy=None), EINVAL), (dict(x=None), EINVAL), (dict(x=(None, 3 * BASE, 2)), EINVAL), (dict(x=(2 * BASE, None, 2)), EINVAL), (dict(x=(2 * BASE, 3 * BASE, 1)), EINVAL),
    (dict(x=(2 * BASE + 8, 3 * BASE, 2)), EINVAL), (dict(dw=None), EINVAL), (dict(ws=None), EINVAL), (dict(rows=-1), EINVAL), (dict(outs=0), EINVAL), (dict(features=0), EINVAL),
    (dict(dtype=2), EINVAL), (dict(dw_dtype=3), EINVAL), (dict(pitch=59), EINVAL), (dict(pitch=1 << 41), EINVAL), (dict(dy=BASE + 2), EINVAL), (dict(dw=4 * BASE + 2), EINVAL),
    (dict(ws=5 * BASE + 64), EINVAL), (dict(ws_bytes=100), EWORKSPACE), (dict(rows=(1 << 31) - 1), EUNSUPPORTED), (dict(outs=(1 << 20) + 1, pitch=1 << 21), EUNSUPPORTED),
    (dict(features=(1 << 20) + 1), EUNSUPPORTED), (dict(outs=1 << 20, features=1 << 18, pitch=1 << 20), EUNSUPPORTED), (dict(dw=BASE + 1199996), EINVAL),
    (dict(dw=2 * BASE), EINVAL), (dict(dw=3 * BASE + 9996), EINVAL), (dict(ws=BASE), EINVAL), (dict(dw=5 * BASE), EINVAL),
], ids=range(28))
def test_refusals(change, status):
    assert _call(**change) == status, mpcnn.lib().mpcnn_last_error().decode()


def test_workspace():
    size = mpcnn.weight_grad_workspace_bytes
    assert size(-1, 60, 40, 0) == size(5, 0, 40, 0) == size(5, 60, 0, 0) == size(5, 60, 40, 2) == 0
    for dtype in (0, 1):
        assert size(0, 60, 40, dtype) >= 256 and size(16384, 60, 40, dtype) > 60 * 40 * 4
        assert size(16384, 8192, 8192, dtype) <= 256 << 20


def test_binding_refuses_what_is_no_packed_rows():
    with pytest.raises(mpcnn.MpcnnError):
        mpcnn.rows_weight_grad(torch.zeros(3, 4), torch.zeros(3, 5))
