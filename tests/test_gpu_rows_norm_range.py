"""The norm of rows whose squares, or the sum of them, fp32 does not hold, against the formula in 64 bits.

u = 2^-24.  A lane adds 8 squares a piece one after the other, then at most 6 steps between lanes and 16 between waves follow; a power of two that the numbers are multiplied by
changes no bits.  rstd: half of what the sum is off by (and the mean, eps), the root and the quotient; y: h's rounding and two products more, and its own."""
import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
FEATURES = [1, 40, 100, 256, 700, 1500, 3000, 9000, 16384, 20001]        # 16 lanes a row to rows that no workgroup's registers hold


def _ids(v):
    return str(v).replace("torch.", "")


def _rows(gen, features, sizes, dtype):
    """Rows of about the given sizes, the first number of each the size itself."""
    x = torch.randn((len(sizes), features), generator=gen, device="cuda").clamp(-3, 3)
    x[:, 0] = 1.0
    return (x.double() * torch.tensor(sizes, dtype=torch.float64, device="cuda")[:, None]).to(dtype)


def _check(x, gain, eps, y, rstd):
    h = x.double()
    r64 = 1.0 / torch.sqrt(h.square().mean(1) + eps)
    y64 = h * r64[:, None] * gain.double()
    chain = 16 if x.shape[1] <= 16384 else 8 * (-(-x.shape[1] // 8192))
    off_r = (chain + 22 + 4) / 2 * U + 4 * U
    off_y = off_r + 3 * U
    least = 2.0 ** -149                                   # (half a step of fp32's smallest numbers, and of bf16's)
    assert ((rstd.double() - r64).abs() <= off_r * r64 + least).all(), (rstd, r64)
    assert ((y.double() - y64).abs() <= (off_y + HALF[y.dtype]) * (1 + off_y) * y64.abs() + 1e-38).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=_ids)
@pytest.mark.parametrize("features", FEATURES)
def test_sums_of_squares_beyond_fp32(features, dtype):
    gen = torch.Generator(device="cuda").manual_seed(features)
    gain = 1 + 0.3 * torch.randn(features, generator=gen, device="cuda")
    # on both sides of where the sum, a square and the mean of them pass fp32's largest
    x = _rows(gen, features, [1.0, 1e15, 2e17, 1e18, 5e18, 1.5e19, 1.8e19, 3e19, 1e22, 1e30, 1e36], dtype)
    for eps in (1e-6, 0.0):
        y, _, _, rstd = mpcnn.rows_norm(x, gain, eps=eps)
        _check(x, gain, eps, y, rstd)
    lone = torch.zeros((3, features), device="cuda", dtype=dtype)
    lone[0, features // 2], lone[1, 0], lone[2, features - 1] = 1e20, -3e38, 1.9e19      # one number's square is enough
    y, _, _, rstd = mpcnn.rows_norm(lone, gain, eps=1e-6)
    _check(lone, gain, 1e-6, y, rstd)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=_ids)
@pytest.mark.parametrize("features", FEATURES)
def test_squares_below_fp32(features, dtype):
    gen = torch.Generator(device="cuda").manual_seed(features + 1)
    gain = 1 + 0.3 * torch.randn(features, generator=gen, device="cuda")
    x = _rows(gen, features, [1.0, 2.0 ** -48, 2.0 ** -50, 2.0 ** -52, 1e-18, 1e-20, 1e-22, 1e-25, 1e-30, 1e-35], dtype)
    for eps in (0.0, 2.0 ** -90, 2.0 ** -110, 2.0 ** -130):
        y, _, _, rstd = mpcnn.rows_norm(x, gain, eps=eps)
        _check(x, gain, eps, y, rstd)


@pytest.mark.parametrize("features", [100, 700, 3000, 9000, 20001])
def test_among_others_and_where_it_lies(features):
    """A row that takes another way among rows that do not: these are as without it, in the order that a workgroup has them, and what is not finite stays so."""
    gen = torch.Generator(device="cuda").manual_seed(features + 2)
    rows = 3000 if features < 9000 else 1200
    x = torch.randn((rows, features), generator=gen, device="cuda")
    residual, gain = torch.randn((rows, features), generator=gen, device="cuda"), 1 + 0.3 * torch.randn(features, generator=gen, device="cuda")
    want = mpcnn.rows_norm(x, gain, residual=residual, eps=0.0, kept=mpcnn.I8)
    large, small, bad = slice(3, None, 7), slice(5, None, 7), slice(6, None, 49)
    for part, by in ((large, 2.0 ** 62), (small, 2.0 ** -70)):
        x[part] *= by
        residual[part] *= by
    x[bad, 1] = float("inf")
    for _ in range(2):
        a, b = x.clone(), residual.clone()
        y, h, kept, rstd = mpcnn.rows_norm(a, gain, residual=b, eps=0.0, y=a, h=b, kept=mpcnn.I8)
        fine = torch.ones(rows, dtype=torch.bool, device="cuda")
        fine[bad] = False
        # powers of two change no bits: the same norm, rstd and sum by the power
        assert torch.equal(y[fine], want[0][fine])
        scale = torch.ones(rows, device="cuda")
        scale[large], scale[small] = 2.0 ** 62, 2.0 ** -70
        assert torch.equal((rstd * scale)[fine], want[3][fine]) and torch.equal((h / scale[:, None])[fine], want[1][fine])
        assert torch.equal(kept.values[fine], want[2].values[fine])
        assert not torch.isfinite(y[bad]).all(1).any()


def test_gradients_of_far_rows():
    """Rows times a power of two, the gradients of the others: dx by the inverse power, dgain the same."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    for features in (300, 5000):
        x, dy = torch.randn((40, features), generator=gen, device="cuda"), torch.randn((40, features), generator=gen, device="cuda")
        gain = 1 + 0.3 * torch.randn(features, generator=gen, device="cuda")
        want = mpcnn.rows_norm_backward(dy, x, gain, mpcnn.rows_norm(x, gain, eps=0.0)[3])
        for by in (2.0 ** 62, 2.0 ** 80, 2.0 ** -70, 2.0 ** -90):
            far = x * by
            got = mpcnn.rows_norm_backward(dy, far, gain, mpcnn.rows_norm(far, gain, eps=0.0)[3])
            assert torch.equal(got[0] * by, want[0]) and torch.equal(got[1], want[1])
