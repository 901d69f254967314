"""The root-mean-square norm of rows, its gradients, and rows in 8 bits, against their formulas in 64 bits.

u = 2^-24 is fp32's half step.  A sum of n terms added one after the other is off by at most n u of the terms' magnitudes; a lane adds 8 features per
piece one after the other (`_chain`), and at most 6 steps between lanes and 16 between waves follow."""
import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
MOST = {mpcnn.I8: 127.0, mpcnn.E4M3: 448.0}
TYPES = [torch.float32, torch.bfloat16]
KINDS = [mpcnn.I8, mpcnn.E4M3]
SIZES = [(1, 1), (2, 7), (3, 32), (5, 33), (19, 128), (16, 129), (1, 256), (70, 257), (9, 512), (130, 513), (33, 1024), (6, 1025), (1, 2048), (3, 2051),
         (40, 4096), (2, 4104), (5, 8192), (3, 8193), (2, 16384), (3, 16390), (5000, 40), (4100, 768), (1, 100003)]


def _ids(v):
    return str(v).replace("torch.", "").replace(" ", "")


def _chain(features):
    return 16 if features <= 16384 else 8 * (-(-features // 8192))


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rand(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def scales_of(v, kind):
    """Exponents of blocks of 32 features of fp64 values."""
    rows, features = v.shape
    v = torch.cat([v, v.new_zeros((rows, -features % 32))], 1).view(rows, (features + 31) // 32, 32).abs().amax(2)
    fraction, exponent = torch.frexp(v)                  # v = fraction 2^exponent, fraction in [1/2, 1)
    whole, power = (127.0 / 128.0, 7) if kind == mpcnn.I8 else (448.0 / 512.0, 9)
    exponent = torch.where(fraction <= whole, exponent - power, exponent - power + 1)
    return torch.where(v == 0, -100, torch.clamp(exponent, min=-100, max=121 if kind == mpcnn.I8 else 120))      # (nothing has no exponent)


def packed_in_64(v, kind):
    """What fp64 values become in 8 bits: numbers (without their scales' powers) and exponents."""
    e = scales_of(v, kind)
    scaled = v * torch.exp2(-e.double()).repeat_interleave(32, 1)[:, :v.shape[1]]
    step = torch.ones_like(scaled)
    if kind == mpcnn.E4M3:
        step = torch.exp2(torch.clamp(torch.floor(torch.log2(scaled.abs().clamp(min=2.0 ** -20))), min=-6.0) - 3.0)
    wide = e.repeat_interleave(32, 1)[:, :v.shape[1]]
    end = torch.where(wide < 120, 448.0, 240.0) if kind == mpcnn.E4M3 else torch.full_like(scaled, 127.0)      # (beyond would read back as infinity)
    return torch.clamp(torch.round(scaled / step) * step, -end, end), e


def read_in_64(p):
    scale = torch.exp2(p.scales.double() - 127.0).repeat_interleave(32, 1)
    return (p.values.float().double() * scale)[:, :p.features]


# ---- 8 bits

@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,features", [(1, 1), (3, 31), (2, 32), (5, 33), (300, 100), (7, 4096), (2049, 65), (1, 70000), (0, 40)])
def test_pack_and_unpack_are_exact(rows, features, kind, dtype):
    gen = _gen(rows + features)
    x = _rand(gen, rows, features) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=gen, device="cuda").float())
    x = x.to(dtype)
    p = mpcnn.rows_pack(x, kind)
    want, e = packed_in_64(x.double(), kind)
    assert torch.equal(p.values.float().double()[:, :features], want)
    assert torch.equal(p.scales.to(torch.int32), e.to(torch.int32) + 127)
    assert (p.values.view(torch.uint8)[:, features:] == 0).all()
    for out in (None, torch.empty((rows, features), device="cuda"), torch.empty((rows, features + 3), device="cuda", dtype=torch.bfloat16)[:, 1:features + 1]):
        assert torch.equal(mpcnn.rows_unpack(p, out).double(), read_in_64(p))


@pytest.mark.parametrize("kind", KINDS)
def test_pack_at_the_borders(kind):
    most = MOST[kind]
    rows = []
    for top in (most, most * (1 + 2.0 ** -23), most * 2.0 ** 100, 2.0 ** -126, 2.0 ** -149, 0.0, 2.0 ** -100 * most, 2.0 ** -99 * most, 3.4e38):
        row = [top] + [top * f for f in (-1.0, 0.5, 1 / 3, -1e-3, 1e-6)] + [(2 * i + 1) * 0.5 * top / most for i in range(26)]   # half steps: to even
        rows.append(row)
    x = torch.tensor(rows, dtype=torch.float64).float().cuda()
    p = mpcnn.rows_pack(x, kind)
    want, e = packed_in_64(x.double(), kind)
    assert torch.equal(p.values.float().double(), want) and torch.equal(p.scales.to(torch.int32), e.to(torch.int32) + 127)
    assert torch.equal(mpcnn.rows_unpack(p, torch.empty_like(x)).double(), read_in_64(p))
    assert torch.equal(mpcnn.rows_unpack(p).double(), read_in_64(p))          # bf16 holds every one of them


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_blocks_that_are_not_finite(kind, bad):
    x = _rand(_gen(3), 4, 96)
    x[1, 40] = bad
    p = mpcnn.rows_pack(x, kind)
    back = mpcnn.rows_unpack(p, torch.empty_like(x))
    assert p.scales[1].tolist()[1] == 255 and torch.isnan(back[1, 32:64]).all()
    back[1, 32:64] = 0
    good = x.clone()
    good[1, 32:64] = 0
    assert torch.isfinite(back).all() and torch.equal(back, mpcnn.rows_unpack(mpcnn.rows_pack(good, kind), torch.empty_like(x)))


def test_strided_rows_and_given_memory():
    gen = _gen(9)
    for dtype in TYPES:
        for offset in (0, 1, 3):
            x = _rand(gen, 50, 150).to(dtype)[:, offset:offset + 101]
            p = mpcnn.PackedRows.empty(50, 101, mpcnn.E4M3, x.device)
            assert mpcnn.rows_pack(x, p) is p
            want, e = packed_in_64(x.double(), mpcnn.E4M3)
            assert torch.equal(p.values.float().double()[:, :101], want)
            around = torch.full((50, 150), 7.0, device="cuda", dtype=dtype)
            mpcnn.rows_unpack(p, around[:, offset:offset + 101])
            assert torch.equal(around[:, offset:offset + 101].double(), read_in_64(p))
            around[:, offset:offset + 101] = 7.0
            assert (around == 7.0).all()


# ---- the norm

def _norm_in_64(x, residual, gain, eps):
    h = x.double() if residual is None else x.double() + residual.double()
    rstd = 1.0 / torch.sqrt(h.square().mean(1) + eps)
    return h, rstd, h * rstd[:, None] * gain.double()


def _norm_off(features):
    """rstd: half of what the sum of squares is off by (its terms: two roundings of h each, counted twice by the square), the mean, eps, the root and the
    quotient; y: h's rounding and two products more."""
    rstd = (_chain(features) + 22 + 4) / 2 * U + 4 * U
    return rstd, rstd + 3 * U


def _check_norm(x, residual, gain, eps, y, h, rstd):
    h64, r64, y64 = _norm_in_64(x, residual, gain, eps)
    off_r, off_y = _norm_off(x.shape[1])
    assert ((rstd.double() - r64).abs() <= off_r * r64).all()
    half = HALF[y.dtype]
    assert ((y.double() - y64).abs() <= (off_y + half) * (1 + off_y) * y64.abs() + 1e-38).all()
    if h is not None:
        assert torch.equal(h, (x.float() + residual.float()).to(h.dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("rows,features", SIZES)
def test_norm(rows, features, with_residual, dtype):
    gen = _gen(rows * 7 + features)
    x = (_rand(gen, rows, features) * 3).to(dtype)
    residual = _rand(gen, rows, features).to(dtype) if with_residual else None
    gain = 1 + _rand(gen, features)
    y, h, kept, rstd = mpcnn.rows_norm(x, gain, residual=residual, eps=1e-5)
    assert kept is None and (h is None) == (residual is None)
    _check_norm(x, residual, gain, 1e-5, y, h, rstd)


def _check_packed(p, v64, off):
    """8 bits of numbers that are known to `off` of themselves: the scale suits them, and each is rounded to its nearest."""
    rows, features = v64.shape
    top = torch.cat([v64, v64.new_zeros((rows, -features % 32))], 1).view(rows, (features + 31) // 32, 32).abs().amax(2)
    scale = torch.exp2(p.scales.double() - 127.0)
    most = MOST[p.kind]
    assert (top <= most * scale * (1 + off)).all()
    assert ((top >= most * scale / 2 * (1 - off)) | (p.scales == 27)).all()
    got, wide = read_in_64(p), scale.repeat_interleave(32, 1)[:, :features]
    if p.kind == mpcnn.I8:
        half = wide / 2
    else:
        half = torch.maximum(v64.abs() * 2.0 ** -4, wide * 2.0 ** -10)
    assert ((got - v64).abs() <= half * (1 + off) + off * v64.abs()).all()
    assert (p.values.view(torch.uint8)[:, features:] == 0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,features", SIZES)
def test_norm_into_8_bits(rows, features, kind, dtype):
    gen = _gen(rows * 11 + features)
    x, residual = (_rand(gen, rows, features) * 3).to(dtype), _rand(gen, rows, features).to(dtype)
    gain = 1 + _rand(gen, features)
    y, h, kept, rstd = mpcnn.rows_norm(x, gain, residual=residual, y=kind, kept=kind)
    h64, r64, y64 = _norm_in_64(x, residual, gain, 1e-6)
    _check_packed(y, y64, _norm_off(features)[1])
    _check_packed(kept, h64, U)
    assert torch.equal(h, (x.float() + residual.float()).to(dtype))
    assert mpcnn.rows_norm(x, gain, y=False, rstd=False) == (None, None, None, None)


def test_norm_where_it_lies_and_among_others():
    gen = _gen(5)
    for dtype in TYPES:
        x, residual = _rand(gen, 300, 200).to(dtype), _rand(gen, 300, 200).to(dtype)
        gain = 1 + _rand(gen, 200)
        want = mpcnn.rows_norm(x, gain, residual=residual)
        a, b = x.clone(), residual.clone()
        got = mpcnn.rows_norm(a, gain, residual=b, y=a, h=b)
        assert got[0] is a and got[1] is b and torch.equal(a, want[0]) and torch.equal(b, want[1])
        a, b = x.clone(), residual.clone()
        mpcnn.rows_norm(a, gain, residual=b, y=b, h=a)
        assert torch.equal(b, want[0]) and torch.equal(a, want[1])
        wide = torch.full((300, 333), 5.0, device="cuda", dtype=dtype)     # odd addresses, numbers between the rows left alone
        wide[:, 3:203], out = x, torch.full((300, 333), 5.0, device="cuda", dtype=dtype)
        mpcnn.rows_norm(wide[:, 3:203], gain, residual=residual, y=out[:, 1:201])
        assert torch.equal(out[:, 1:201], want[0])
        out[:, 1:201] = 5.0
        assert (out == 5.0).all()


@pytest.mark.parametrize("features", [100, 700, 3000, 9000, 20000])
def test_norm_of_unusual_rows(features):
    gen = _gen(features)
    x = _rand(gen, 6, features)
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 0] = float("inf")
    x[4] *= 1e-30
    gain = torch.ones(features, device="cuda")
    y, _, kept, rstd = mpcnn.rows_norm(x, gain, eps=1e-6, kept=mpcnn.I8)
    fine = [0, 1, 4, 5]
    _check_norm(x[fine], None, gain, 1e-6, y[fine], None, rstd[fine])
    assert (y[1] == 0).all() and abs(rstd[1].item() - 1e3) < 1e-3
    assert torch.isnan(y[2]).all() and torch.isnan(y[3, 0]) and (kept.scales[[2, 3]] == 255).sum() == 2
    y, _, _, _ = mpcnn.rows_norm(x, gain, eps=0.0)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[0]).all()


# ---- its gradients

def _back_in_64(dy, h, gain, rstd, dh):
    dy, gain, rstd = dy.double(), gain.double(), rstd.double()[:, None]
    unit, u = h * rstd, dy * gain
    c = (u * unit).mean(1, keepdim=True)
    dx = rstd * (u - unit * c)
    return (dx if dh is None else dx + dh.double()), (dy * unit).sum(0), (unit, u, c, rstd)


def _check_back(dy, h, gain, rstd, dh, dx, dgain):
    rows, features = dy.shape
    dx64, dg64, (unit, u, c, by) = _back_in_64(dy, h, gain, rstd, dh)
    # c: unit's, u's and the product's roundings, the sum, the quotient; dx: two fused steps on terms that carry the same
    off_c = (_chain(features) + 22 + 5) * U * (u * unit).abs().mean(1, keepdim=True)
    off = by.abs() * (unit.abs() * off_c + 4 * U * (u.abs() + (unit * c).abs())) + 2 * U * dx64.abs()
    assert ((dx.double() - dx64).abs() <= off * (1 + HALF[dx.dtype]) + HALF[dx.dtype] * dx64.abs() + 1e-38).all()
    # rows one after the other in a workgroup (at least 256 of them where there are that many rows), its rows at once, the shares
    steps = -(-rows // 256) + 16 + 32 + 32 + 2
    if dgain is not None:
        assert ((dgain.double() - dg64).abs() <= steps * U * (dy.double() * unit).abs().sum(0) + 1e-38).all()


def _back_inputs(gen, rows, features, dtype, kept):
    h = _rand(gen, rows, features) * 2
    dy, dh = _rand(gen, rows, features).to(dtype), _rand(gen, rows, features).to(dtype)
    gain = 1 + _rand(gen, features)
    rstd = (1 / torch.sqrt(h.double().square().mean(1) + 1e-6)).float()
    if kept is None:
        h = h.to(dtype)
        return dy, h, h.double(), gain, rstd, dh
    p = mpcnn.rows_pack(h, kept)
    return dy, p, read_in_64(p), gain, rstd, dh


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("kept", [None, *KINDS])
@pytest.mark.parametrize("rows,features", SIZES)
def test_norm_backward(rows, features, kept, dtype):
    dy, h, h64, gain, rstd, dh = _back_inputs(_gen(rows * 13 + features), rows, features, dtype, kept)
    for more in (None, dh):
        dx, dgain = mpcnn.rows_norm_backward(dy, h, gain, rstd, dh=more)
        _check_back(dy, h64, gain, rstd, more, dx, dgain)
    assert torch.equal(mpcnn.rows_norm_backward(dy, h, gain, rstd, dgain=False)[0], mpcnn.rows_norm_backward(dy, h, gain, rstd)[0])
    assert torch.equal(mpcnn.rows_norm_backward(dy, h, gain, rstd, dx=False)[1], dgain)


@pytest.mark.parametrize("features", [60, 900, 5000, 9000])
def test_rows_without_a_gradient_add_nothing(features):
    gen = _gen(features)
    dy, h, _, gain, rstd, dh = _back_inputs(gen, 40, features, torch.float32, None)
    dy[5], dy[7], dy[39] = 0.0, -0.0, 0.0
    h[5], h[7, 3], rstd[39] = float("nan"), float("inf"), float("nan")
    clean, fine = h.clone(), rstd.clone()
    clean[5], clean[7, 3], fine[39] = 0.0, 0.0, 1.0
    dx, dgain = mpcnn.rows_norm_backward(dy, h, gain, rstd, dh=dh)
    want = mpcnn.rows_norm_backward(dy, clean, gain, fine, dh=dh)
    assert torch.equal(dx, want[0]) and torch.equal(dgain, want[1]) and torch.equal(dx[[5, 7, 39]], dh[[5, 7, 39]])
    p = mpcnn.rows_pack(h, mpcnn.I8)
    dx, dgain = mpcnn.rows_norm_backward(dy, p, gain, rstd, dh=dh)
    want = mpcnn.rows_norm_backward(dy, mpcnn.rows_pack(clean, mpcnn.I8), gain, fine, dh=dh)
    assert torch.equal(dx, want[0]) and torch.equal(dgain, want[1])


def test_no_rows():
    for features in (5, 3000, 20000):
        none = torch.empty((0, features), device="cuda")
        gain, rstd = torch.ones(features, device="cuda"), torch.empty(0, device="cuda")
        y, h, kept, r = mpcnn.rows_norm(none, gain, residual=none, kept=mpcnn.I8)
        assert y.shape == h.shape == none.shape and r.shape == (0,) and kept.rows == 0
        dx, dgain = mpcnn.rows_norm_backward(none, none, gain, rstd, dgain=torch.full((features,), 3.0, device="cuda"))
        assert dx.shape == none.shape and (dgain == 0).all()


def test_backward_where_it_lies_and_strided():
    gen = _gen(12)
    for dtype in TYPES:
        dy, h, h64, gain, rstd, dh = _back_inputs(gen, 77, 333, dtype, None)
        want = mpcnn.rows_norm_backward(dy, h, gain, rstd, dh=dh)
        for which in range(3):
            t = [dy.clone(), dh.clone(), h.clone()]
            got = mpcnn.rows_norm_backward(t[0], t[2], gain, rstd, dh=t[1], dx=t[which])
            assert got[0] is t[which] and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        wide = torch.zeros((77, 1001), device="cuda", dtype=dtype)
        wide[:, 1:334], wide[:, 335:668] = dy, h
        out = torch.full((77, 400), 9.0, device="cuda", dtype=dtype)
        got = mpcnn.rows_norm_backward(wide[:, 1:334], wide[:, 335:668], gain, rstd, dh=dh, dx=out[:, 5:338])
        assert torch.equal(out[:, 5:338], want[0]) and torch.equal(got[1], want[1]) and (out[:, :5] == 9.0).all() and (out[:, 338:] == 9.0).all()


def test_gradients_against_differences():
    gen = _gen(21)
    x, dy, gain = _rand(gen, 3, 50), _rand(gen, 3, 50), 1 + _rand(gen, 50)
    _, _, _, rstd = mpcnn.rows_norm(x, gain, y=False)
    dx, dgain = mpcnn.rows_norm_backward(dy, x, gain, rstd)
    loss = lambda x, g: (_norm_in_64(x, None, g, 1e-6)[2] * dy.double()).sum()    # noqa: E731
    step = 1e-6
    for i, j in ((0, 0), (1, 17), (2, 49)):
        d = torch.zeros_like(x, dtype=torch.float64)
        d[i, j] = step
        slope = (loss(x.double() + d, gain) - loss(x.double() - d, gain)) / (2 * step)
        assert abs(slope.item() - dx[i, j].item()) < 1e-5 * (1 + abs(slope.item()))
        g = torch.zeros(50, dtype=torch.float64, device="cuda")
        g[j] = step
        slope = (loss(x, gain.double() + g) - loss(x, gain.double() - g)) / (2 * step)
        assert abs(slope.item() - dgain[j].item()) < 1e-5 * (1 + abs(slope.item()))


def test_offsets_beyond_32_bits():
    """Rows 1.5e9 numbers apart: the third one's begin beyond 2^31 numbers, and 2^32 bytes."""
    pitch, features = 1500000000, 700
    gen = _gen(8)
    far = torch.empty(2 * pitch + features, dtype=torch.bfloat16, device="cuda").as_strided((3, features), (pitch, 1))
    near = _rand(gen, 3, features).to(torch.bfloat16)
    far.copy_(near)
    gain, dy = 1 + _rand(gen, features), _rand(gen, 3, features).to(torch.bfloat16)
    y, _, kept, rstd = mpcnn.rows_norm(near, gain, kept=mpcnn.I8)
    y2, _, kept2, rstd2 = mpcnn.rows_norm(far, gain, kept=mpcnn.I8)
    assert torch.equal(y, y2) and torch.equal(kept.values, kept2.values) and torch.equal(rstd, rstd2)
    want = mpcnn.rows_norm_backward(dy, near, gain, rstd)
    got = mpcnn.rows_norm_backward(dy, far, gain, rstd, dx=far)
    assert torch.equal(far, want[0]) and torch.equal(got[1], want[1])
    del far
    rows = 70000                                           # and packed rows beyond 2^31 bytes
    p = mpcnn.PackedRows.empty(rows, 32768, mpcnn.E4M3, "cuda:%d" % torch.cuda.current_device())
    x = _rand(gen, 1, 32768).to(torch.bfloat16)
    mpcnn.rows_pack(x.expand(rows, 32768).contiguous(), p)
    one = mpcnn.rows_pack(x, mpcnn.E4M3)
    assert torch.equal(p.values[-1].view(torch.uint8), one.values[0].view(torch.uint8)) and torch.equal(p.scales[-1], one.scales[0])
    assert torch.equal(mpcnn.rows_unpack(p)[-1], mpcnn.rows_unpack(one)[0])


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("rows,features", [(1, 40), (7, 33), (300, 513), (5, 4104)])
def test_in_one_buffers_columns(rows, features, dtype):
    """Inputs and outputs beside each other in one buffer, with columns of nobody's behind them."""
    gen = _gen(rows + features)
    buffer = torch.full((rows, 6 * features + 3), 7.0, dtype=dtype, device="cuda")
    x, y, residual, h, dy, dx = (buffer[:, i * features:(i + 1) * features] for i in range(6))
    for t in (x, residual, dy):
        t.copy_(_rand(gen, rows, features))
    gain = 1 + _rand(gen, features)
    inputs = [t.clone() for t in (x, residual, dy)]
    want = mpcnn.rows_norm(inputs[0], gain, residual=inputs[1])
    want_dx, want_dgain = mpcnn.rows_norm_backward(inputs[2], want[1], gain, want[3])
    rstd = mpcnn.rows_norm(x, gain, residual=residual, y=y, h=h)[3]
    dgain = mpcnn.rows_norm_backward(dy, h, gain, rstd, dx=dx)[1]
    for got, wanted in ((y, want[0]), (h, want[1]), (rstd, want[3]), (dx, want_dx), (dgain, want_dgain), (x, inputs[0]), (residual, inputs[1]), (dy, inputs[2])):
        assert torch.equal(got, wanted)
    assert (buffer[:, 6 * features:] == 7.0).all()


def test_streams_and_graphs():
    gen = _gen(31)
    dy, _, _, gain, _, dh = _back_inputs(gen, 600, 513, torch.bfloat16, None)
    x = _rand(gen, 600, 513).to(torch.bfloat16)
    side = torch.cuda.Stream()
    y, h, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(600, device="cuda")
    kept = mpcnn.PackedRows.empty(600, 513, mpcnn.I8, x.device)
    dx, dgain = torch.empty_like(x), torch.empty(513, device="cuda")
    ws = torch.empty(mpcnn.norm_workspace_bytes(600, 513), dtype=torch.uint8, device="cuda")
    residual = torch.empty_like(x)

    def step(stream=None):
        mpcnn.rows_norm(x, gain, residual=residual, y=y, h=h, kept=kept, rstd=rstd, stream=stream)
        mpcnn.rows_norm_backward(dy, kept, gain, rstd, dh=dh, dx=dx, dgain=dgain, ws=ws, stream=stream)

    residual.copy_(dh)
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    first = [t.clone() for t in (y, h, rstd, dx, dgain, kept.values, kept.scales)]
    step()
    for a, b in zip(first, (y, h, rstd, dx, dgain, kept.values, kept.scales)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        residual.copy_(_rand(gen, 600, 513))
        x.copy_(_rand(gen, 600, 513))
        [t.zero_() for t in (y, h, rstd, dx, dgain)]
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, h, rstd, dx, dgain, kept.values, kept.scales)]
        step()
        for a, b in zip(got, (y, h, rstd, dx, dgain, kept.values, kept.scales)):
            assert torch.equal(a, b)
