"""Refusals of the norm of rows and of rows in 8 bits that need no GPU: they come before any launch."""
import ctypes as C

import pytest
import torch

from paper_1302_1690_amd import mpcnn

BASE = 1 << 40
EINVAL, EWORKSPACE, EUNSUPPORTED = 1, 3, 4
NORM = dict(x=BASE, x_pitch=40, residual=2 * BASE, residual_pitch=40, gain=3 * BASE, rows=20, features=40, dtype=0, eps=1e-6, y=4 * BASE, y_pitch=40, y8=None,
            h=5 * BASE, h_pitch=40, h8=None, rstd=6 * BASE)
BACK = dict(dy=BASE, dy_pitch=40, h=2 * BASE, h_pitch=40, h8=None, gain=3 * BASE, rstd=4 * BASE, dh=5 * BASE, dh_pitch=40, rows=20, features=40, dtype=0,
            dx=6 * BASE, dx_pitch=40, dgain=7 * BASE, ws=8 * BASE, ws_bytes=1 << 30)


def _p(values, scales, kind=2):
    return mpcnn._Packed(values, scales, kind)


def _arg(v):
    return C.byref(v) if isinstance(v, mpcnn._Packed) else v


def _norm(**change):
    a = dict(NORM, **change)
    return mpcnn.lib().mpcnn_rows_norm(*[_arg(v) for v in a.values()], None)


def _back(**change):
    a = dict(BACK, **change)
    return mpcnn.lib().mpcnn_rows_norm_backward(*[_arg(v) for v in a.values()], None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), EINVAL), (dict(gain=None), EINVAL), (dict(rows=-1), EINVAL), (dict(features=0), EINVAL), (dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL),
    (dict(x_pitch=39), EINVAL), (dict(residual_pitch=39), EINVAL), (dict(y_pitch=39), EINVAL), (dict(h_pitch=0), EINVAL), (dict(x_pitch=1 << 41), EINVAL),
    (dict(x=BASE + 2), EINVAL), (dict(residual=2 * BASE + 1), EINVAL), (dict(gain=3 * BASE + 2), EINVAL), (dict(rstd=6 * BASE + 1), EINVAL),
    (dict(eps=-1e-9), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(eps=float("inf")), EINVAL), (dict(eps=1e39), EINVAL),
    (dict(rows=1 << 31), EUNSUPPORTED), (dict(features=(1 << 20) + 1, x_pitch=1 << 21, residual_pitch=1 << 21, y_pitch=1 << 21, h_pitch=1 << 21), EUNSUPPORTED),
    (dict(y=BASE + 4), EINVAL), (dict(y=BASE, y_pitch=41), EINVAL), (dict(h=2 * BASE + 3196), EINVAL), (dict(y=3 * BASE), EINVAL), (dict(rstd=BASE), EINVAL),
    (dict(h=4 * BASE), EINVAL), (dict(rstd=4 * BASE + 3196), EINVAL),
    (dict(y8=_p(7 * BASE, None)), EINVAL), (dict(y8=_p(7 * BASE + 8, 8 * BASE)), EINVAL), (dict(y8=_p(7 * BASE, 8 * BASE, 1)), EINVAL),
    (dict(h8=_p(7 * BASE, 7 * BASE + 1279)), EINVAL), (dict(y8=_p(7 * BASE, 8 * BASE), h8=_p(7 * BASE + 1264, 9 * BASE)), EINVAL),
    (dict(h8=_p(2 * BASE, 8 * BASE)), EINVAL),
], ids=range(34))
def test_norm_refusals(change, status):
    assert _norm(**change) == status, mpcnn.lib().mpcnn_last_error().decode()


@pytest.mark.parametrize("change,status", [
    (dict(dy=None), EINVAL), (dict(h=None), EINVAL), (dict(gain=None), EINVAL), (dict(rstd=None), EINVAL), (dict(ws=None), EINVAL), (dict(rows=-1), EINVAL),
    (dict(features=-3), EINVAL), (dict(dtype=3), EINVAL), (dict(dy_pitch=39), EINVAL), (dict(h_pitch=39), EINVAL), (dict(dh_pitch=39), EINVAL), (dict(dx_pitch=39), EINVAL),
    (dict(dy=BASE + 1), EINVAL), (dict(dx=6 * BASE + 2), EINVAL), (dict(dgain=7 * BASE + 2), EINVAL), (dict(ws=8 * BASE + 64), EINVAL), (dict(ws_bytes=100), EWORKSPACE),
    (dict(h8=_p(9 * BASE, 10 * BASE)), EINVAL), (dict(h=None, h8=_p(9 * BASE, 10 * BASE, 0)), EINVAL), (dict(dx=BASE + 4), EINVAL), (dict(dx=BASE, dx_pitch=44), EINVAL),
    (dict(dx=3 * BASE), EINVAL), (dict(dgain=2 * BASE), EINVAL), (dict(dgain=6 * BASE), EINVAL), (dict(ws=BASE), EINVAL), (dict(dgain=8 * BASE), EINVAL),
    (dict(rows=1 << 31), EUNSUPPORTED), (dict(h=None, h8=_p(6 * BASE, 10 * BASE)), EINVAL),
], ids=range(28))
def test_backward_refusals(change, status):
    assert _back(**change) == status, mpcnn.lib().mpcnn_last_error().decode()


@pytest.mark.parametrize("y,y_pitch,h", [(BASE + 156, 100, 5 * BASE), (BASE + 244, 100, 5 * BASE), (BASE + 160, 101, 5 * BASE), (BASE + 160, 100, BASE + 316), (BASE - 244, 100, 5 * BASE)])
def test_beside_each_other_but_not_apart(y, y_pitch, h):
    """Columns of one buffer, rows 400 bytes apart, 160 of them a matrix's: one number too near."""
    assert _norm(x_pitch=100, y=y, y_pitch=y_pitch, h=h, h_pitch=100) == EINVAL
    assert b"overlap" in mpcnn.lib().mpcnn_last_error()


@pytest.mark.parametrize("x,pitch,rows,features,dtype,out,status", [
    (None, 40, 20, 40, 0, _p(BASE, 2 * BASE), EINVAL), (3 * BASE, 39, 20, 40, 0, _p(BASE, 2 * BASE), EINVAL), (3 * BASE + 2, 40, 20, 40, 0, _p(BASE, 2 * BASE), EINVAL),
    (3 * BASE, 40, -1, 40, 0, _p(BASE, 2 * BASE), EINVAL), (3 * BASE, 40, 20, 0, 0, _p(BASE, 2 * BASE), EINVAL), (3 * BASE, 40, 20, 40, 7, _p(BASE, 2 * BASE), EINVAL),
    (3 * BASE, 40, 20, 40, 0, None, EINVAL), (3 * BASE, 40, 20, 40, 0, _p(None, 2 * BASE), EINVAL), (3 * BASE, 40, 20, 40, 0, _p(BASE, None), EINVAL),
    (3 * BASE, 40, 20, 40, 0, _p(BASE + 4, 2 * BASE), EINVAL), (3 * BASE, 40, 20, 40, 0, _p(BASE, 2 * BASE, 1), EINVAL), (3 * BASE, 40, 20, 40, 0, _p(3 * BASE, 2 * BASE), EINVAL),
    (3 * BASE, 40, 20, 40, 0, _p(BASE, 3 * BASE + 3199), EINVAL), (3 * BASE, 40, 1 << 31, 40, 0, _p(BASE, 2 * BASE), EUNSUPPORTED),
], ids=range(14))
def test_pack_refusals(x, pitch, rows, features, dtype, out, status):
    L = mpcnn.lib()
    assert L.mpcnn_rows_pack(x, pitch, rows, features, dtype, _arg(out), None) == status, L.mpcnn_last_error().decode()
    assert L.mpcnn_rows_unpack(_arg(out), rows, features, dtype, x, pitch, None) == status, L.mpcnn_last_error().decode()


def test_workspace():
    size = mpcnn.norm_workspace_bytes
    assert size(-1, 40) == size(20, 0) == size(1 << 31, 40) == size(20, (1 << 20) + 1) == 0
    for features in (1, 40, 700, 5000, 30000):
        got = [size(rows, features) for rows in (0, 1, 2, 5, 17, 300, 5000, 1 << 20)]
        assert got == sorted(got) and got[0] > 0


def test_binding_refuses_what_is_on_the_host():
    x, gain = torch.zeros(3, 40), torch.ones(40)
    for call in (lambda: mpcnn.rows_norm(x, gain), lambda: mpcnn.rows_pack(x), lambda: mpcnn.rows_norm_backward(x, x, gain, torch.ones(3)),
                 lambda: mpcnn.PackedRows(torch.zeros(3, 64, dtype=torch.int8), torch.zeros(3, 2, dtype=torch.uint8), 40),
                 lambda: mpcnn.PackedRows(torch.zeros(3, 64), torch.zeros(3, 2, dtype=torch.uint8), 40), lambda: mpcnn.PackedRows.empty(3, 40, 1, "cpu"),
                 lambda: mpcnn.PackedRows.empty(3, 40, True, "cpu")):
        with pytest.raises(mpcnn.MpcnnError):
            call()


def test_packed_rows_keep_their_tensors():
    p = mpcnn.PackedRows.empty(3, 40, mpcnn.E4M3, "cpu")
    assert (p.rows, p.features, p.kind, p.device.type) == (3, 40, mpcnn.E4M3, "cpu") and p.values.shape == (3, 64) and p.scales.shape == (3, 2)
    for name in ("values", "scales", "features", "kind", "rows", "device"):
        with pytest.raises(AttributeError):
            setattr(p, name, getattr(p, name))
