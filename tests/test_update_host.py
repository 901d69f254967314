"""Refusals of the lists of gradients and of the clipped step that need no GPU: they come before any device call."""
import ctypes as C

import pytest

from paper_1302_1690_amd import mpcnn, workloads as wl

EINVAL = 1


def _create(rows, count=None, out=True):
    arr = (mpcnn._Tensor * max(1, len(rows)))(*[mpcnn._Tensor(*r) for r in rows])
    h = C.c_void_p()
    st = mpcnn.lib().mpcnn_grad_list_create(arr if rows else None, len(rows) if count is None else count, C.byref(h) if out else None)
    assert not h.value
    return st, mpcnn.lib().mpcnn_last_error().decode()


BASE = 1 << 40


@pytest.mark.parametrize("rows,says", [
    ([(0, 0, 5, 0, 0)], "null gradient"),
    ([(BASE, 0, -1, 0, 0)], "numbers"),
    ([(BASE, 0, 5, 2, 0)], "unknown type"),
    ([(BASE, BASE * 2, 5, 0, 7)], "unknown type"),
    ([(BASE + 2, 0, 5, 0, 0)], "multiple"),
    ([(BASE + 1, 0, 5, 1, 0)], "multiple"),
    ([(BASE, 2 * BASE + 2, 5, 1, 0)], "multiple"),
    ([(BASE, 2 * BASE, 5, 0, 0), (BASE + 64, 0, 5, 0, 0)], "all or none"),
    ([(BASE, 2 * BASE, 50, 0, 0), (3 * BASE, BASE + 196, 5, 0, 0)], "overlap"),    # a parameter and another one's gradient, by one number
    ([(BASE, 2 * BASE, 500, 0, 0), (BASE + 400, 3 * BASE, 5, 0, 0), (4 * BASE, BASE + 800, 5, 0, 0)], "overlap"),   # behind one inside another
    ([(3 * BASE, BASE + 8, 5, 1, 1), (BASE, 2 * BASE, 5, 1, 1)], "overlap"),       # in whatever order
    ([(BASE, BASE, 5, 0, 0)], "overlap"),                                         # a gradient that is its own parameter
], ids=range(12))
def test_list_refusals(rows, says):
    st, text = _create(rows)
    assert st == EINVAL and says in text, text


def test_too_many_numbers():
    st, text = _create([(BASE, 0, 1 << 40, 0, 0), (8 * BASE, 0, 1 << 40, 0, 0)])
    assert st == EINVAL and "2^40" in text


def test_null_arguments():
    assert _create([], count=2)[0] == EINVAL
    assert _create([], count=-1)[0] == EINVAL
    assert _create([(BASE, 0, 5, 0, 0)], out=False)[0] == EINVAL
    L = mpcnn.lib()
    assert L.mpcnn_grad_norm(None, 1.0, BASE, None) == EINVAL
    assert L.mpcnn_grad_clip(None, 1.0, None, None) == EINVAL
    assert L.mpcnn_sgd_step_list(None, 0.1, 1.0, 1.0, None, None) == EINVAL
    L.mpcnn_grad_list_destroy(None)
    assert L.mpcnn_sgd_step_clipped(None, 0.1, 1.0, 1.0, None, None) == EINVAL


def test_net_without_parameters_is_refused():
    cfg = wl.CONFIGS[0]
    net = mpcnn.Net(cfg.layers, cfg.in_channels, cfg.patch)
    assert mpcnn.lib().mpcnn_sgd_step_clipped(net._h, 0.1, 1.0, 1.0, None, None) == EINVAL
    assert "never set" in mpcnn.lib().mpcnn_last_error().decode()
    net.close()
