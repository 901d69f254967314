"""The class layer on rows of features (loss and gradients, any number of classes) against its formulas in 64 bits.

Tolerances, with u = 2^-24 (half a step of fp32) and sums bounded by the number of their terms:
  a score is a sum of `features` products and a bias; bf16 products are exact in fp32, fp32 ones are made of two fp16 parts per number
  (each number to 2^-22 of itself or 2^-39 of the tensor's largest, the left-out product 2^-22): e_s = (features + 4) u S + parts,
  S = the largest sum |x w| + |bias| of the row, parts = 3 2^-22 S + features 2^-38 max|x| max|w|  (fp32 only);
  lse and -log p: two scores' errors and a few roundings of numbers up to |lse| (log, differences: 8 u (|lse| + |s| + 1));
  p = exp(s - lse) has a relative error of 2 e_s + 8 u (|s - lse| + 2) =: e_p (in exponents, times 2 where it is small: expm1(x) < 2 x);
  delta is rounded to bf16 (2^-8 of itself) or to two fp16 parts (2^-22 of itself, 2^-38 of 1): e_d = e_p p + r |delta|;
  dx is a sum over the classes of delta w (their errors, classes u), dw one over the rows; both are rounded (u or 2^-8)."""
import gc
import math

import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _nothing_is_left():
    """Tensors that caught exceptions keep in reference cycles go now, not while another test watches the allocator."""
    yield
    gc.collect()


F, B = torch.float32, torch.bfloat16
U = 2.0 ** -24
ROUND = {F: U, B: 2.0 ** -8}


def _inputs(rows, features, classes, dtype, seed, ignored=0.2, weights=True, spread=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, features), generator=gen, device="cuda").to(dtype)
    w = (torch.randn((classes, features), generator=gen, device="cuda") * (spread / math.sqrt(features))).to(dtype)
    bias = torch.randn((classes,), generator=gen, device="cuda")
    labels = torch.randint(0, classes, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    skip = torch.rand((rows,), generator=gen, device="cuda")
    labels[skip < ignored] = -1
    labels[skip > 1 - ignored / 4] = classes
    roww = torch.rand((rows,), generator=gen, device="cuda") + 0.1 if weights else None
    if weights and rows > 2:
        roww[rows // 2] = 0.0
    return x, w, bias, labels, roww


def _want(x, w, bias, labels, roww):
    """Results in 64 bits and how far off they may be."""
    dtype, (rows, features), classes = x.dtype, x.shape, w.shape[0]
    live = (labels >= 0) & (labels < classes)
    if roww is not None:
        live &= roww != 0
    at = torch.nonzero(live).squeeze(1)
    xs, ws, t = x[at].double(), w.double(), labels[at].long()
    c = torch.ones(len(at), dtype=torch.float64, device="cuda") if roww is None else roww[at].double()
    b = torch.zeros(classes, dtype=torch.float64, device="cuda") if bias is None else bias.double()
    s = xs @ ws.t() + b
    fin = torch.where(torch.isinf(s), torch.zeros_like(s), s)
    size = (xs.abs() @ ws.abs().t() + torch.where(torch.isinf(b), torch.zeros_like(b), b.abs())).amax(1, keepdim=True) if len(at) else fin[:, :1]
    e_s = (features + 4) * U * size
    if dtype == F and len(at):
        e_s = e_s + 3 * 2.0 ** -22 * size + features * 2.0 ** -38 * xs.abs().max() * ws.abs().max()
    lse = torch.logsumexp(s, 1, keepdim=True)
    idx = torch.arange(len(at), device="cuda")
    off = torch.isinf(s[idx, t])
    nll = torch.where(off, torch.full_like(lse[:, 0], math.inf), lse[:, 0] - s[idx, t])
    near = lambda v: torch.where(torch.isinf(v), torch.zeros_like(v), v.abs())  # noqa: E731
    e_lse = e_s[:, 0] * 1.01 + 8 * U * (near(lse[:, 0]) + 1) + classes * U
    p = torch.where(torch.isinf(s), torch.zeros_like(s), torch.exp(s - lse))
    hot = torch.zeros_like(p)
    hot[idx, t] = 1.0
    delta = p - hot
    e_p = 2 * (2 * e_s + classes * U + 8 * U * (near(s - lse) + 2))
    e_d = e_p * p + (2.0 ** -8 * delta.abs() if dtype == B else 2.0 ** -22 * delta.abs() + 2.0 ** -38) + 2 * U
    out = {}

    def put(name, value, error, shape, rounding):
        full, err = (torch.zeros(shape, dtype=torch.float64, device="cuda") for _ in range(2))
        if name in ("rowloss", "lse", "dx"):
            full[at], err[at] = value, error + rounding * near(value)
        else:
            full, err = value, error + rounding * near(value)
        out[name] = (full, err)
    put("rowloss", c * nll, c.abs() * (e_lse + e_s[:, 0] + 8 * U * near(s[idx, t])), (rows,), 4 * U)
    put("lse", lse[:, 0], e_lse, (rows,), 4 * U)
    cc = c[:, None]
    extra = 2.0 ** -21 if dtype == F else 2.0 ** -8          # parts of the other operand / dw's delta, weighted and rounded in one
    put("dx", cc * (delta @ ws), cc.abs() * (e_d @ ws.abs() + (classes * U + (extra if dtype == F else 0)) * (delta.abs() @ ws.abs())), (rows, features),
        ROUND[dtype] + 4 * U)
    wd = (cc * delta).abs()
    top = c.abs().max() if len(at) else 0.0
    small = 2.0 ** -38 * top * xs.abs().sum(0) if dtype == F else 0.0
    put("dw", (cc * delta).t() @ xs, (cc.abs() * e_d).t() @ xs.abs() + (len(at) * U + extra) * (wd.t() @ xs.abs()) + small, (classes, features),
        ROUND[dtype] + 4 * U)
    put("db", (cc * delta).sum(0), (cc.abs() * (e_p * p + 4 * U)).sum(0) + (len(at) + 4) * U * wd.sum(0), (classes,), 2 * U)
    return out


def _near(name, got, want):
    full, err = want
    if got.numel() > 1 << 30:             # (indexing by truth values takes 32-bit counts)
        return max(_near(name, got[i:i + 8192], (full[i:i + 8192], err[i:i + 8192])) for i in range(0, len(got), 8192))
    got = got.double()
    inf = torch.isinf(full)
    assert torch.equal(got[inf], full[inf]), name
    bad = ~((got - full)[~inf].abs() <= err[~inf] + 1e-37)
    worst = ((got - full)[~inf].abs() / (err[~inf] + 1e-37)).max().item() if bad.numel() else 0.0
    assert not bad.any(), "%s: %d of %d off, worst %.3g of what is allowed" % (name, int(bad.sum()), bad.numel(), worst)
    return worst


def _check(x, w, bias, labels, roww, what=""):
    want = _want(x, w, bias, labels, roww)
    loss, rowloss, lse = mpcnn.class_loss(x, w, labels, bias=bias, roww=roww)
    loss2, rowloss2, dx, dw, db = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
    # (there the loss alone and the gradients' loss come from kernels of their own, each as far from the formula as it may be)
    work = x.shape[0] * w.numel()
    if not (1.2e9 < work <= 2e9 or (x.dtype == F and 8 < x.shape[0] <= 128 and work > 1.2e9)):
        assert torch.equal(rowloss, rowloss2)
    _near("rowloss", rowloss2, want["rowloss"])
    for l, r in ((loss, rowloss), (loss2, rowloss2)):
        total = r.double().sum().item()
        assert l.item() == total or abs(l.item() - total) <= 1e-12 * rowloss.double().abs().sum().item()
    got = {"rowloss": rowloss, "lse": lse, "dx": dx, "dw": dw}
    if bias is not None:
        got["db"] = db
    else:
        assert db is None
    print(what, {k: "%.2g" % _near(k, v, want[k]) for k, v in got.items()}, flush=True)
    return got


SIZES = [(1, 1, 1), (1, 1, 2), (2, 3, 1), (3, 5, 7), (1, 64, 129), (5, 100, 37), (63, 65, 64), (64, 64, 63), (65, 63, 65), (127, 33, 257), (130, 128, 128),
         (257, 96, 255), (31, 1000, 300), (300, 200, 1000), (513, 31, 77), (129, 257, 4097), (1000, 40, 3), (700, 520, 1500)]


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,features,classes", SIZES)
def test_sizes(rows, features, classes, dtype):
    _check(*_inputs(rows, features, classes, dtype, rows + features + classes), "%dx%dx%d" % (rows, features, classes))


# on both sides of where another kernel takes over: few rows with many classes, scores of few rows, large weights read as they are, much work
PATHS = [(1, 70, 1100), (2, 100, 1023), (2, 64, 24577), (3, 129, 1024), (4, 31, 4097), (5, 33, 4096), (8, 40, 24576), (9, 72, 24600), (15, 1025, 4100),
         (16, 40, 5000), (17, 40, 5000), (16, 2048, 19600), (64, 1024, 39100), (65, 256, 20000), (300, 320, 13000), (257, 70, 70001), (1500, 1000, 801),
         (700, 127, 20011), (700, 128, 20011), (1030, 511, 5003), (1030, 512, 5003),
         (200, 4000, 3001), (129, 4096, 5003),
         (3, 50, 1024), (12, 100, 24576), (13, 100, 24576), (4, 700, 100000), (12, 1501, 100003), (12, 1504, 100003), (11, 1536, 100003), (13, 1501, 100003),
         (8, 1200, 10011), (9, 1200, 10011), (13, 999, 10011), (32, 999, 13011), (33, 1001, 9991), (64, 33, 303031), (65, 1031, 9700), (128, 1031, 9700), (129, 1031, 9700), (100, 4096, 20001)]


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,features,classes", PATHS)
def test_paths(rows, features, classes, dtype):
    _check(*_inputs(rows, features, classes, dtype, rows + features + classes), "%dx%dx%d" % (rows, features, classes))


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
def test_without_bias_weights_or_gaps(dtype):
    x, w, _, labels, _ = _inputs(200, 128, 500, dtype, 3, ignored=0.0, weights=False)
    _check(x, w, None, labels, None)


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,features,classes", [(70, 64, 200), (70, 50, 200), (3, 128, 300)])
def test_strides_and_addresses(rows, features, classes, dtype):
    x, w, bias, labels, roww = _inputs(rows, features, classes, dtype, 9)
    want = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
    for pad, shift in ((0, 1), (7, 0), (8, 8), (24, 3)):
        def wide(m):
            flat = torch.full((m.shape[0] * (m.shape[1] + pad) + shift + 8,), math.nan, device="cuda").to(dtype)
            view = flat[shift:shift + m.shape[0] * (m.shape[1] + pad)].view(m.shape[0], m.shape[1] + pad)[:, :m.shape[1]]
            view.copy_(m)
            return view, flat
        (xv, _), (wv, _) = wide(x), wide(w)
        dxv, flat = wide(torch.zeros_like(x))
        got = mpcnn.class_backward(xv, wv, labels, bias=bias, roww=roww, dx=dxv)
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        assert int(torch.isnan(flat).sum()) == flat.numel() - x.numel()          # nothing between the rows or behind them


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 6, 200])
def test_rows_that_add_nothing_may_hold_anything(rows, dtype):
    x, w, bias, labels, roww = _inputs(rows + 3, 70, 150, dtype, 5, ignored=0.0)
    roww[:] = roww.abs() + 0.5
    x[0], x[1], x[rows] = math.nan, math.inf, 3e38
    labels[0], labels[1] = -1, 150
    roww[rows] = 0.0
    got = _check(x, w, bias, labels, roww)
    for name in ("rowloss", "lse", "dx"):
        assert (got[name][[0, 1, rows]] == 0).all()
    labels[:] = -5                                                              # nothing is left
    loss, rowloss, dx, dw, db = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
    assert loss.item() == 0
    for t in (rowloss, dx, dw, db):
        assert (t == 0).all()


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [2, 90])
def test_classes_that_are_off(rows, dtype):
    x, w, bias, labels, roww = _inputs(rows, 48, 400, dtype, 6, ignored=0.0)
    off = torch.zeros(400, dtype=torch.bool, device="cuda")
    off[100:390:2] = True
    off[128:256] = True                                                         # a whole tile
    labels[:] = 101
    bias[off] = -math.inf
    got = _check(x, w, bias, labels, roww)
    assert (got["dw"][off] == 0).all() and (got["db"][off] == 0).all()
    bias[off] = torch.finfo(F).min
    again = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
    for a, b in zip((got["rowloss"], got["dx"], got["dw"], got["db"]), again[1:]):
        assert torch.equal(a, b)
    labels[0] = 100                                                             # a label that is off
    bias[off] = -math.inf
    assert _check(x, w, bias, labels, roww)["rowloss"][0].item() == math.inf
    bias[:] = -math.inf                                                         # no class is left: p = 0
    loss, rowloss, dx, dw, db = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
    r = torch.ones(rows, device="cuda") if roww is None else roww
    live = r != 0
    assert (rowloss[live] == math.inf).all() and loss.item() == math.inf
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
    want = torch.zeros(400, dtype=torch.float64, device="cuda").index_add_(0, labels.long(), -r.double())
    assert (db.double() - want).abs().max().item() <= rows * U * r.double().sum().item()


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
def test_magnitudes(dtype):
    """Features and weights far from 1, rows far from each other, one class that wins by far."""
    for fx, fw in ((1e-6, 1e6), (1e5, 1e-5), (1e-3, 1e3)):
        x, w, bias, labels, roww = _inputs(150, 80, 333, F, 8)
        _check((x * fx).to(dtype), (w * fw).to(dtype), bias, labels, roww * 1e-4)
    x, w, bias, labels, roww = _inputs(150, 80, 333, dtype, 8)
    x[::3] *= 1.0 / 64
    bias[17] += 60.0
    _check(x, w, bias, labels, roww)
    _check(x, w, bias, labels, -roww)


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
def test_classes_in_pieces(dtype):
    """More scores than a piece holds."""
    rows, features, classes = 8192, 24, 40003
    _check(*_inputs(rows, features, classes, dtype, 4, weights=dtype == F), "pieces")


def test_wide_weights_in_pieces():
    """More class weights than a piece brings into blocks."""
    _check(*_inputs(3, 4096, 33500, F, 4, ignored=0.0, weights=False), "wide")
    _check(*_inputs(140, 4096, 33500, F, 5, weights=False), "wide")


def test_very_many_classes():
    x, w, bias, labels, roww = _inputs(5, 16, 1200000, B, 4, ignored=0.0, weights=False)
    labels[0], labels[1] = 1199999, 0
    _check(x, w, bias, labels, roww, "many")


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
def test_very_many_rows(dtype):
    """So many rows that a workgroup takes several tiles of them, up to the most that there may be."""
    for rows in (300001, 1 << 20):
        _check(*_inputs(rows, 5, 6, dtype, 6), "rows")


def test_no_rows():
    w, bias = torch.randn(50, 8, device="cuda"), torch.randn(50, device="cuda")
    x, labels = torch.empty(0, 8, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    loss, rowloss, lse = mpcnn.class_loss(x, w, labels, bias=bias)
    assert loss.item() == 0 and rowloss.numel() == 0 and lse.numel() == 0
    loss, rowloss, dx, dw, db = mpcnn.class_backward(x, w, labels, bias=bias, dw=torch.ones_like(w), db=torch.ones_like(bias))
    assert loss.item() == 0 and dx.shape == (0, 8) and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
def test_gradients_against_differences(dtype):
    """L moves by the gradient times a step, up to the second-order term: central differences in the inputs, from losses of this package.
    For steps h d the difference of two losses, each off by a few 2^-24 per row, over 2 h; third derivatives of L along d are below
    2 |d . score|^3 per row."""
    rows, features, classes = 40, 24, 60
    x, w, bias, labels, roww = _inputs(rows, features, classes, F, 12)
    x, w = x.to(dtype).float(), w.to(dtype).float()
    _, _, dx, dw, db = mpcnn.class_backward(x.to(dtype), w.to(dtype), labels, bias=bias, roww=roww)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for which, grad in (("x", dx), ("w", dw), ("b", db)):
        base = {"x": x, "w": w, "b": bias}
        d = torch.randn(grad.shape, generator=gen, device="cuda") * 0.25
        h = 2.0 ** -6
        losses = []
        for sign in (1.0, -1.0):
            moved = dict(base)
            moved[which] = base[which] + sign * h * d
            losses.append(mpcnn.class_loss(moved["x"], moved["w"], labels, bias=moved["b"], roww=roww)[0].item())
        got = (losses[0] - losses[1]) / (2 * h)
        want = float((grad.double() * d.double()).sum())
        scores = {"x": lambda: d @ w.t(), "w": lambda: x @ d.t(), "b": lambda: d[None, :].expand(rows, -1)}[which]().abs().amax(1).double()
        c = torch.where((labels >= 0) & (labels < classes), roww, torch.zeros_like(roww)).double()
        third = float((c * 2 * (2 * scores) ** 3).sum()) * h * h / 6
        rounding = float(c.sum()) * 64 * 2.0 ** -22 / h
        stored = (2.0 ** -7 if dtype == B else 2.0 ** -20) * float((grad.double() * d.double()).abs().sum()) + (2.0 ** -7 * float(c.sum()) if dtype == B else 0)
        assert abs(got - want) <= third + rounding + stored, (which, got, want, third, rounding, stored)


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,features,classes", [(2, 72, 30000), (6, 70, 5000), (7, 300, 30000), (40, 500, 30000), (100, 500, 30000), (300, 70, 60000), (300, 128, 33000), (200, 2000, 3000)])
def test_rows_that_add_nothing_may_hold_anything_with_more_classes(rows, features, classes, dtype):
    x, w, bias, labels, roww = _inputs(rows + 3, features, classes, dtype, 5, ignored=0.0)
    roww[:] = roww.abs() + 0.5
    x[0], x[1], x[rows] = math.nan, math.inf, 3e38
    labels[0], labels[1] = -2147483648, 2147483647
    roww[rows] = 0.0
    got = _check(x, w, bias, labels, roww)
    for name in ("rowloss", "lse", "dx"):
        assert (got[name][[0, 1, rows]] == 0).all()
    labels[:] = -5
    for t in mpcnn.class_backward(x, w, labels, bias=bias, roww=roww):
        assert (t == 0).all()


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,features,classes", [(300, 320, 13000), (300, 324, 13000), (14, 320, 9000), (20, 1001, 13000), (100, 1001, 13000), (12, 500, 25000), (250, 2000, 3000)])
def test_strides_and_addresses_with_more_classes(rows, features, classes, dtype):
    """Nothing between the rows or behind the last one is read into a result, or written."""
    x, w, bias, labels, roww = _inputs(rows, features, classes, dtype, 9)
    want = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
    for pad, shift in ((0, 1), (8, 0), (64, 8), (24, 3)):
        def wide(m):
            flat = torch.full((m.shape[0] * (m.shape[1] + pad) + shift + 4096,), math.nan, device="cuda").to(dtype)
            view = flat[shift:shift + m.shape[0] * (m.shape[1] + pad)].view(m.shape[0], m.shape[1] + pad)[:, :m.shape[1]]
            view.copy_(m)
            return view, flat
        (xv, _), (wv, _) = wide(x), wide(w)
        dxv, flat = wide(torch.zeros_like(x))
        got = mpcnn.class_backward(xv, wv, labels, bias=bias, roww=roww, dx=dxv)
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        assert int(torch.isnan(flat).sum()) == flat.numel() - x.numel()


def test_pieces_of_weights_that_are_read_as_they_are():
    x, w, bias, labels, roww = _inputs(8192, 64, 40003, B, 4)
    flat = torch.full((40003, 128), math.nan, dtype=B, device="cuda")
    flat[:, 32:96] = w
    want = _check(x, w, bias, labels, roww)
    loss, rowloss, dx, dw, db = mpcnn.class_backward(x, flat[:, 32:96], labels, bias=bias, roww=roww)
    for a, b in ((rowloss, "rowloss"), (dx, "dx"), (dw, "dw"), (db, "db")):
        assert torch.equal(a, want[b])


@pytest.mark.parametrize("rows", [3, 300])
def test_weights_that_lie_far_apart(rows):
    """Offsets beyond 2^32 numbers in the class weights."""
    x, w, bias, labels, roww = _inputs(rows, 64, 70000, B, 4)
    wide = torch.empty((70000, 65536), dtype=B, device="cuda")
    wide[:, 100:164] = w
    want = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
    for shift in (100, 128):
        wide[:, shift:shift + 64] = w
        for a, b in zip(want, mpcnn.class_backward(x, wide[:, shift:shift + 64], labels, bias=bias, roww=roww)):
            assert torch.equal(a, b)
    del wide
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows", [3, 40])
def test_weights_of_more_than_2_to_the_31_numbers(rows):
    _check(*_inputs(rows, 65536, 33000, B, 4), "wide")
    torch.cuda.empty_cache()


def test_two_calls_at_once():
    """Two streams, a workspace each, much and little work side by side."""
    sizes = ((F, (300, 72, 60000)), (B, (260, 320, 16000)), (B, (4, 128, 30000)), (F, (100, 64, 900)))
    inputs = [_inputs(*size, dtype, 2) for dtype, size in sizes]
    want = [mpcnn.class_backward(x, w, labels, bias=bias, roww=roww) for x, w, bias, labels, roww in inputs]
    streams = [torch.cuda.Stream() for _ in sizes]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [mpcnn.class_backward(x, w, labels, bias=bias, roww=roww, stream=s) for (x, w, bias, labels, roww), s in zip(inputs, streams)]
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            for p, q in zip(a, b):
                assert torch.equal(p, q)


def test_same_results_every_time_and_on_streams():
    for dtype, size in ((F, (300, 72, 900)), (B, (260, 128, 3000)), (B, (3, 128, 3000))):
        x, w, bias, labels, roww = _inputs(*size, dtype, 2)
        want = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        for stream in (None, s, s.cuda_stream, None):
            got = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww, stream=stream)
            torch.cuda.synchronize()
            for a, b in zip(want, got):
                assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [4, 150])
def test_recorded_into_a_graph(rows, dtype):
    x, w, bias, labels, roww = _inputs(rows, 64, 700, dtype, 2)
    x2 = _inputs(rows, 64, 700, dtype, 3)[0]
    outs = dict(rowloss=torch.zeros(rows, device="cuda"), loss=torch.zeros(1, dtype=torch.float64, device="cuda"), dx=torch.zeros_like(x),
                dw=torch.zeros_like(w), db=torch.zeros_like(bias))
    n = mpcnn.class_workspace_bytes(rows, 64, 700, mpcnn.BF16 if dtype == B else mpcnn.F32, True)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        mpcnn.class_backward(x, w, labels, bias=bias, roww=roww, ws=ws, **outs)
    for k in range(4):
        x.copy_(x2 * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        want = mpcnn.class_backward(x.clone(), w, labels, bias=bias, roww=roww)
        torch.cuda.synchronize()
        for a, b in zip(want, (outs["loss"], outs["rowloss"], outs["dx"], outs["dw"], outs["db"])):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F, B], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [300, 14])
def test_two_graphs_with_more_classes(rows, dtype):
    """Two graphs with a workspace each, replayed in turn and on new inputs; one workspace for both would do on one stream, too."""
    size = (rows, 320, 14000)
    x, w, bias, labels, roww = _inputs(*size, dtype, 2)
    n = mpcnn.class_workspace_bytes(*size, mpcnn.BF16 if dtype == B else mpcnn.F32, True)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        outs = dict(rowloss=torch.zeros(rows, device="cuda"), loss=torch.zeros(1, dtype=torch.float64, device="cuda"), dx=torch.zeros_like(x),
                    dw=torch.zeros_like(w), db=torch.zeros_like(bias))
        own = x.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            mpcnn.class_backward(own, w, labels, bias=bias, roww=roww, ws=ws, **outs)
        graphs.append((graph, own, outs))
    for k in range(3):
        for j, (graph, own, outs) in enumerate(graphs):
            own.copy_(x * (0.5 + k + 2 * j))
            graph.replay()
        torch.cuda.synchronize()
        for graph, own, outs in graphs:
            want = mpcnn.class_backward(own.clone(), w, labels, bias=bias, roww=roww)
            torch.cuda.synchronize()
            for a, b in zip(want, (outs["loss"], outs["rowloss"], outs["dx"], outs["dw"], outs["db"])):
                assert torch.equal(a, b)


def test_parts_of_the_results():
    x, w, bias, labels, roww = _inputs(100, 64, 300, B, 2)
    want = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww)
    for leave in range(5):
        names = ["loss", "rowloss", "dx", "dw", "db"]
        got = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww, **{names[leave]: False})
        for k, (a, b) in enumerate(zip(want, got)):
            assert (b is None) if k == leave else torch.equal(a, b)
    assert mpcnn.class_loss(x, w, labels, bias=bias, roww=roww, lse=False, rowloss=False)[0].item() == want[0].item()


def test_refusals():
    x, w, bias, labels, roww = _inputs(20, 16, 30, F, 2)
    wrong = [
        lambda: mpcnn.class_loss(x.cpu(), w, labels), lambda: mpcnn.class_loss(x.half(), w.half(), labels), lambda: mpcnn.class_loss(x, w.to(B), labels),
        lambda: mpcnn.class_loss(x, w[:, :8], labels), lambda: mpcnn.class_loss(x, w, labels.long()), lambda: mpcnn.class_loss(x, w, labels[:10]),
        lambda: mpcnn.class_loss(x, w, labels, bias=bias[:10]), lambda: mpcnn.class_loss(x, w, labels, roww=roww.double()),
        lambda: mpcnn.class_loss(x.t().contiguous().t(), w, labels), lambda: mpcnn.class_loss(x[0].expand(20, 16), w, labels),
        lambda: mpcnn.class_loss(x, w[:0], labels), lambda: mpcnn.class_loss(x[0], w, labels), lambda: mpcnn.class_backward(x, w, labels, dx=x),
        lambda: mpcnn.class_backward(x, w, labels, dw=w), lambda: mpcnn.class_backward(x, w, labels, dx=torch.empty(20, 16, dtype=B, device="cuda")),
        lambda: mpcnn.class_backward(x, w, labels, bias=bias, db=bias), lambda: mpcnn.class_backward(x, w, labels, dw=torch.empty(16, 30, device="cuda").t()),
        lambda: mpcnn.class_loss(x, w, labels, loss=torch.zeros(1, device="cuda")),
    ]
    for k, call in enumerate(wrong):
        with pytest.raises(mpcnn.MpcnnError) as e:
            call()
        assert e.value.status == 1, k
    with pytest.raises(mpcnn.MpcnnError) as e:
        mpcnn.class_backward(x, w, labels, ws=torch.empty(1024, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3
    assert mpcnn.class_loss(x, w, labels, bias=bias)[0].item() > 0


def test_a_training_step_of_a_class_layer():
    """Loss, gradients, their norm bounded, the step: the pieces together, against the same steps in 64 bits."""
    rows, features, classes = 96, 40, 700
    x, w, bias, labels, _ = _inputs(rows, features, classes, F, 21, ignored=0.1, weights=False)
    roww = torch.full((rows,), 1.0 / rows, device="cuda")
    dw, db = torch.empty_like(w), torch.empty_like(bias)
    steps = mpcnn.GradList([dw, db], [w, bias])
    W, b, X = w.double(), bias.double(), x.double()
    live = (labels >= 0) & (labels < classes)
    t = torch.where(live, labels, torch.zeros_like(labels)).long()
    c = live.double() / rows
    for k in range(4):
        loss = mpcnn.class_backward(x, w, labels, bias=bias, roww=roww, dw=dw, db=db, dx=False)[0]
        norm = steps.sgd_step(5.0, max_norm=0.05)
        logp = torch.log_softmax(X @ W.t() + b, 1)
        want = -(c * logp.gather(1, t[:, None])[:, 0]).sum()
        d = logp.exp()
        d[torch.arange(rows, device="cuda"), t] -= 1
        d *= c[:, None]
        gw, gb = d.t() @ X, d.sum(0)
        size = torch.sqrt((gw * gw).sum() + (gb * gb).sum())
        f = 5.0 * min(1.0, 0.05 / size.item())
        W, b = W - f * gw, b - f * gb
        # (losses to 2^-20 or so, gradients to a few 2^-20 of their norm; steps of 0.25 at most, errors add up over four)
        assert abs(loss.item() - want.item()) <= (k + 1) * 2.0 ** -17 * abs(want.item())
        assert abs(norm.item() - size.item()) <= (k + 1) * 2.0 ** -16 * size.item()
        assert (w.double() - W).norm().item() <= (k + 1) * (2.0 ** -16 * 0.25 + 2.0 ** -24 * W.norm().item())
