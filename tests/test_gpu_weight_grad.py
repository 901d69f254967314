"""The gradient of a linear layer's weights from rows in 8 bits, against its formula in 64 bits.

u = 2^-24.  Products are exact (fp32 dy: but for its third part's rounding, u of it); the matrix instruction adds 16 of them to a sum, and each addition inside it is off
by at most one unit, 2 u, of the terms' magnitudes: a sum of n terms by 2 (n + 16) u of the terms' magnitudes.  The result is rounded once."""
import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.bfloat16]
KINDS = [mpcnn.I8, mpcnn.E4M3]


def _ids(v):
    return str(v).replace("torch.", "")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _read(p):
    return mpcnn.rows_unpack(p).double()                  # (exact: test_gpu_rows_norm.py)


def _inputs(gen, rows, outs, features, dtype, kind):
    dy = torch.randn((rows, outs), generator=gen, device="cuda") * torch.exp2(torch.randint(-6, 6, (1, outs), generator=gen, device="cuda").float())
    x = torch.randn((rows, features), generator=gen, device="cuda") * torch.exp2(torch.randint(-6, 6, (1, features), generator=gen, device="cuda").float())
    return dy.to(dtype), mpcnn.rows_pack(x, kind)


def check(dw, dy, p):
    x, dy = _read(p), dy.double()
    want, size = dy.t() @ x, dy.abs().t() @ x.abs()
    off = (2 * (dy.shape[0] + 16) + 1) * U * size + HALF[dw.dtype] * want.abs() + 1e-38
    assert ((dw.double() - want).abs() <= off * (1 + 2.0 ** -7)).all()


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,outs,features", [(1, 1, 1), (1, 128, 128), (2, 7, 33), (31, 129, 31), (32, 37, 32), (33, 256, 257), (64, 300, 100), (65, 513, 129),
                                                (213, 37, 100), (1000, 64, 1000), (4097, 130, 70), (20000, 5, 3), (300, 3500, 3400), (129, 4096, 4096)])
def test_weight_grad(rows, outs, features, kind, dtype):
    dy, p = _inputs(_gen(rows + outs * 3 + features * 7), rows, outs, features, dtype, kind)
    dw = mpcnn.rows_weight_grad(dy, p)
    assert dw.dtype == dtype
    check(dw, dy, p)
    assert torch.equal(dw, mpcnn.rows_weight_grad(dy, p))
    wide = mpcnn.rows_weight_grad(dy, p, dw=torch.empty((outs, features), device="cuda"))
    check(wide, dy, p)
    assert torch.equal(wide.to(dtype), dw)
    check(mpcnn.rows_weight_grad(dy, p, dw=torch.empty((outs, features), device="cuda", dtype=torch.bfloat16)), dy, p)


@pytest.mark.parametrize("kind", KINDS)
def test_largest_numbers(kind):
    """fp32's largest numbers, which are nearer to bf16's infinity than to its largest, with small ones of x: as large as it gets, and finite."""
    gen = _gen(77 + kind)
    dy, p = _inputs(gen, 100, 40, 70, torch.float32, kind)
    most = torch.finfo(torch.float32).max
    dy[::3] = torch.where(dy[::3] > 0, most, -most)
    small = mpcnn.PackedRows(p.values, (p.scales - 40).contiguous(), 70)          # (x times 2^-40)
    dw = mpcnn.rows_weight_grad(dy, small)
    assert torch.isfinite(dw).all()
    check(dw, dy, small)


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
def test_every_place_of_a_tile(dtype):
    """One row at a time has one number: every product lands where it belongs, exactly."""
    outs, features, rows = 300, 290, 97
    gen = _gen(5)
    for n in (0, 1, 2, 3, 4, 7, 8, 15, 16, 31, 32, 63, 64, 96):
        dy = torch.zeros((rows, outs), device="cuda")
        x = torch.zeros((rows, features), device="cuda")
        dy[n] = torch.randint(-100, 100, (outs,), generator=gen, device="cuda").float()
        x[n] = torch.randint(-64, 64, (features,), generator=gen, device="cuda").float()
        x[n, ::32] = 64.0                                 # (blocks' scales are 1: the numbers are kept as they are)
        p = mpcnn.rows_pack(x, mpcnn.I8)
        got = mpcnn.rows_weight_grad(dy.to(dtype), p, dw=torch.empty((outs, features), device="cuda"))
        assert torch.equal(got.double(), dy[n].double()[:, None] * _read(p)[n][None])


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
def test_strides_and_odd_addresses(dtype):
    dy, p = _inputs(_gen(8), 150, 133, 77, dtype, mpcnn.E4M3)
    want = mpcnn.rows_weight_grad(dy, p)
    for offset, pitch in ((0, 136), (1, 135), (3, 400)):
        wide = torch.full((150, pitch), float("nan"), device="cuda", dtype=dtype)
        wide[:, offset:offset + 133] = dy
        assert torch.equal(mpcnn.rows_weight_grad(wide[:, offset:offset + 133], p), want)


def test_no_rows_and_what_is_not_finite():
    none = mpcnn.PackedRows.empty(0, 50, mpcnn.I8, "cuda:%d" % torch.cuda.current_device())
    for dtype in TYPES:
        dw = torch.full((20, 50), 3.0, device="cuda", dtype=dtype)
        assert (mpcnn.rows_weight_grad(torch.empty((0, 20), device="cuda"), none, dw=dw) == 0).all()
        dy, _ = _inputs(_gen(9), 70, 40, 100, dtype, mpcnn.I8)
        x = torch.randn((70, 100), generator=_gen(10), device="cuda")
        x[5, 40] = float("nan")
        for kind in KINDS:
            dw = mpcnn.rows_weight_grad(dy, mpcnn.rows_pack(x, kind))
            assert torch.isnan(dw[:, 32:64]).all() and torch.isfinite(dw[:, :32]).all() and torch.isfinite(dw[:, 64:]).all()
        dy[3, 7] = float("inf")
        dw = mpcnn.rows_weight_grad(dy, mpcnn.rows_pack(torch.nan_to_num(x), mpcnn.I8))
        assert not torch.isfinite(dw[7]).any() and torch.isfinite(dw[:7]).all() and torch.isfinite(dw[8:]).all()


@pytest.mark.parametrize("scale", [2.0 ** -90, 2.0 ** 90])
def test_far_scales(scale):
    """Blocks' powers of two at the ends: fp32 results where the products have them."""
    dy, p = _inputs(_gen(14), 64, 20, 64, torch.float32, mpcnn.I8)
    q = mpcnn.rows_pack(mpcnn.rows_unpack(p).float() * scale, mpcnn.I8)
    assert torch.equal(mpcnn.rows_weight_grad(dy, q).double(), mpcnn.rows_weight_grad(dy, p).double() * scale)


def test_offsets_beyond_32_bits():
    pitch = 1500000000
    dy, p = _inputs(_gen(15), 3, 200, 90, torch.bfloat16, mpcnn.I8)
    far = torch.empty(2 * pitch + 200, dtype=torch.bfloat16, device="cuda").as_strided((3, 200), (pitch, 1))
    far.copy_(dy)
    assert torch.equal(mpcnn.rows_weight_grad(far, p), mpcnn.rows_weight_grad(dy, p))
    del far
    rows, features = 70001, 32768                          # packed rows beyond 2^31 bytes: the last one counts
    p = mpcnn.PackedRows.empty(rows, features, mpcnn.E4M3, dy.device)
    p.values.view(torch.uint8).zero_()
    p.scales.fill_(127)
    one = mpcnn.rows_pack(torch.randn((1, features), generator=_gen(16), device="cuda"), mpcnn.E4M3)
    p.values[-1:].view(torch.uint8).copy_(one.values.view(torch.uint8))
    p.scales[-1:].copy_(one.scales)
    dy = torch.randn((rows, 8), generator=_gen(17), device="cuda").to(torch.bfloat16)
    assert torch.equal(mpcnn.rows_weight_grad(dy, p), mpcnn.rows_weight_grad(dy[-1:], one))


def test_streams_and_graphs():
    gen = _gen(20)
    dy, p = _inputs(gen, 2000, 150, 200, torch.bfloat16, mpcnn.I8)
    dw = torch.empty((150, 200), device="cuda", dtype=torch.bfloat16)
    ws = torch.empty(max(256, mpcnn.weight_grad_workspace_bytes(2000, 150, 200, mpcnn.BF16)), dtype=torch.uint8, device="cuda")
    want = mpcnn.rows_weight_grad(dy, p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    mpcnn.rows_weight_grad(dy, p, dw=dw, ws=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(dw, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mpcnn.rows_weight_grad(dy, p, dw=dw, ws=ws)
    for _ in range(4):
        dy.copy_(torch.randn(dy.shape, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, mpcnn.rows_weight_grad(dy, p))
