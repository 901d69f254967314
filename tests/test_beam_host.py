"""Refusals of beam search's selection and of lists of states that need no GPU: they come before any device call."""
import ctypes as C

import pytest
import torch

from paper_1302_1690_amd import mpcnn

BASE = 1 << 40
EINVAL, EWORKSPACE, EUNSUPPORTED = 1, 3, 4
GOOD = dict(scores=BASE, pitch=1000, bias=2 * BASE, totals=3 * BASE, done=4 * BASE, end=5, sequences=3, beams=4, width=4, classes=1000, dtype=0, totals_out=5 * BASE,
            parents=6 * BASE, classes_out=7 * BASE, done_out=8 * BASE, ws=9 * BASE, ws_bytes=1 << 30)


@pytest.mark.parametrize("change,status", [
    (dict(scores=None), EINVAL), (dict(totals=None), EINVAL), (dict(totals_out=None), EINVAL), (dict(parents=None), EINVAL), (dict(classes_out=None), EINVAL),
    (dict(ws=None), EINVAL), (dict(sequences=-1), EINVAL), (dict(beams=0), EINVAL), (dict(width=0), EINVAL), (dict(classes=0), EINVAL), (dict(dtype=2), EINVAL),
    (dict(pitch=999), EINVAL), (dict(pitch=1 << 41), EINVAL), (dict(end=-2), EINVAL), (dict(end=1000), EINVAL), (dict(end=-1), EINVAL),
    (dict(scores=BASE + 2), EINVAL), (dict(dtype=1, scores=BASE + 1), EINVAL), (dict(bias=2 * BASE + 1), EINVAL), (dict(totals=3 * BASE + 2), EINVAL),
    (dict(parents=6 * BASE + 2), EINVAL), (dict(classes_out=7 * BASE + 3), EINVAL), (dict(totals_out=5 * BASE + 1), EINVAL),
    (dict(ws=9 * BASE + 128), EINVAL), (dict(ws_bytes=100), EWORKSPACE), (dict(beams=65, width=4), EUNSUPPORTED), (dict(width=65), EUNSUPPORTED),
    (dict(sequences=(1 << 18) + 1), EUNSUPPORTED), (dict(classes=(1 << 31) - 1024, pitch=1 << 32), EUNSUPPORTED),
    (dict(totals_out=3 * BASE), EINVAL), (dict(parents=BASE + 47996), EINVAL), (dict(done_out=4 * BASE + 11), EINVAL), (dict(classes_out=6 * BASE + 44), EINVAL),
    (dict(ws=2 * BASE), EINVAL), (dict(totals_out=9 * BASE), EINVAL),
], ids=range(35))
def test_select_refusals(change, status):
    a = dict(GOOD, **change)
    assert mpcnn.lib().mpcnn_beam_select(*a.values(), None) == status, mpcnn.lib().mpcnn_last_error().decode()


CLASS = dict(x=BASE, x_pitch=64, w=10 * BASE, w_pitch=64, bias=2 * BASE, totals=3 * BASE, done=4 * BASE, end=5, sequences=3, beams=4, width=4, features=64, classes=1000,
             dtype=0, totals_out=5 * BASE, parents=6 * BASE, classes_out=7 * BASE, done_out=8 * BASE, ws=9 * BASE, ws_bytes=1 << 30)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), EINVAL), (dict(w=None), EINVAL), (dict(totals=None), EINVAL), (dict(ws=None), EINVAL), (dict(features=0), EINVAL), (dict(classes=0), EINVAL), (dict(width=0), EINVAL),
    (dict(dtype=2), EINVAL), (dict(x_pitch=63), EINVAL), (dict(w_pitch=63), EINVAL), (dict(w_pitch=1 << 41), EINVAL), (dict(x=BASE + 2), EINVAL), (dict(w=10 * BASE + 1), EINVAL),
    (dict(ws=9 * BASE + 128), EINVAL), (dict(ws_bytes=10000), EWORKSPACE), (dict(width=65), EUNSUPPORTED), (dict(classes=(1 << 27) + 1), EUNSUPPORTED),
    (dict(features=(1 << 20) + 1, x_pitch=1 << 21, w_pitch=1 << 21), EUNSUPPORTED), (dict(sequences=1 << 15, classes=1 << 20), EUNSUPPORTED),
    (dict(parents=10 * BASE + 255996), EINVAL), (dict(totals_out=BASE), EINVAL), (dict(ws=10 * BASE), EINVAL), (dict(done_out=10 * BASE), EINVAL),
], ids=range(23))
def test_class_beam_refusals(change, status):
    a = dict(CLASS, **change)
    assert mpcnn.lib().mpcnn_class_beam(*a.values(), None) == status, mpcnn.lib().mpcnn_last_error().decode()


def test_class_beam_workspace():
    size = mpcnn.class_beam_workspace_bytes
    assert size(-1, 4, 64, 100, 0) == size(3, 4, 0, 100, 0) == size(3, 4, 64, 0, 1) == size(3, 4, 64, 100, 2) == 0
    for dtype in (0, 1):
        for beams, features, classes in ((1, 7, 1), (4, 1024, 32000), (8, 4096, 50021), (16, 100, 1000)):
            got = [size(n, beams, features, classes, dtype) for n in (0, 1, 2, 3, 5, 9, 17, 40, 100)]
            assert got == sorted(got) and got[0] > 0


def test_workspace():
    size = mpcnn.beam_workspace_bytes
    assert size(-1, 4, 100) == size(3, 0, 100) == size(3, 65, 100) == size(3, 4, 0) == size(1 << 20, 2, 100) == size(3, 4, 1 << 31) == 0
    for beams, classes in ((1, 1), (4, 1000), (8, 50021), (64, 2000000)):
        got = [size(n, beams, classes) for n in (0, 1, 2, 3, 10, 100, 1000, 10000)]
        assert got == sorted(got) and got[0] > 0


def _state(data=BASE, row=4096, segment=1024, unit=64, units=16, segments=4):
    return data, row, segment, unit, units, segments


def _create(states, sequences=3, beams=4, count=None, out=True):
    arr = (mpcnn._BeamState * max(1, len(states)))(*[mpcnn._BeamState(*s) for s in states])
    h = C.c_void_p()
    st = mpcnn.lib().mpcnn_beam_states_create(arr if states else None, len(states) if count is None else count, sequences, beams, C.byref(h) if out else None)
    assert not h.value
    return st


@pytest.mark.parametrize("states,more,status", [
    ([_state(data=0)], {}, EINVAL), ([_state(row=4095)], {}, EINVAL), ([_state(segment=1023)], {}, EINVAL), ([_state(unit=-1)], {}, EINVAL), ([_state(units=-1)], {}, EINVAL),
    ([_state(segments=-1)], {}, EINVAL), ([_state(row=-4096)], {}, EINVAL), ([_state(unit=1 << 41)], {}, EINVAL), ([_state(unit=1 << 30, units=1 << 30)], {}, EINVAL),
    ([_state(), _state(data=BASE + 12 * 4096 - 1)], {}, EINVAL), ([_state(), _state()], {}, EINVAL), ([_state(data=BASE + 64), _state(data=BASE)], {}, EINVAL),
    ([_state(row=8192), _state(data=BASE + 4095, row=8192)], {}, EINVAL), ([_state(row=8192), _state(data=BASE + 4097, row=8192)], {}, EINVAL),
    ([_state(row=8192), _state(data=BASE + 4096, row=8256)], {}, EINVAL), ([_state(row=12288), _state(data=BASE + 4096, row=12288), _state(data=BASE + 12288 + 64, row=12288)], {}, EINVAL),
    ([_state(row=1 << 35, unit=1 << 35, units=1, segments=1)], {}, EUNSUPPORTED), ([_state()], dict(beams=0), EINVAL), ([_state()], dict(sequences=-1), EINVAL),
    ([_state()], dict(beams=65), EUNSUPPORTED), ([_state()], dict(sequences=1 << 19), EUNSUPPORTED), ([], dict(count=2), EINVAL), ([], dict(count=-1), EINVAL),
    ([_state()], dict(out=False), EINVAL),
], ids=range(24))
def test_states_refusals(states, more, status):
    assert _create(states, **more) == status, mpcnn.lib().mpcnn_last_error().decode()


def test_null_lists():
    assert mpcnn.lib().mpcnn_beam_reorder(None, BASE, -1, None) == EINVAL
    mpcnn.lib().mpcnn_beam_states_destroy(None)


def test_binding_refuses_what_is_on_the_host():
    for call in (lambda: mpcnn.beam_select(torch.zeros(4, 10), torch.zeros(1, 4)), lambda: mpcnn.BeamStates([torch.zeros(4, 10)], 1, 4)):
        with pytest.raises(mpcnn.MpcnnError):
            call()
