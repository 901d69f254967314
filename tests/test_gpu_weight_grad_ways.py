"""The ways of the weights' gradient that large sizes take: rows of bf16 that are no whole 16-byte pieces, copied before the products, and tiles of 256 x 256 with split rows.

u = 2^-24.  Products are exact (fp32 dy: three bf16 parts hold its 24 bits); the matrix instruction adds 16 of them to a sum, and each addition inside it is off by at most one unit, 2 u, of the terms'
magnitudes; the sums of the parts are as many additions more, of at most 64 parts.  The result is rounded once."""
import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def _ids(v):
    return str(v).replace("torch.", "")


def _inputs(seed, rows, outs, features, dtype, kind):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dy = torch.randn((rows, outs), generator=gen, device="cuda") * torch.exp2(torch.randint(-6, 6, (1, outs), generator=gen, device="cuda").float())
    x = torch.randn((rows, features), generator=gen, device="cuda") * torch.exp2(torch.randint(-6, 6, (1, features), generator=gen, device="cuda").float())
    return dy.to(dtype), mpcnn.rows_pack(x, kind)


def check(dw, dy, p):
    x, dy = mpcnn.rows_unpack(p).double(), dy.double()
    want, size = dy.t() @ x, dy.abs().t() @ x.abs()
    off = (2 * (dy.shape[0] + 16) + 64 + 2) * U * size + HALF[dw.dtype] * want.abs() + 1e-38
    assert ((dw.double() - want).abs() <= off * (1 + 2.0 ** -7)).all()


# from 2048 rows and 1024 features on, outputs that are no multiple of 8: small tiles split, large tiles split and whole, the last row of a block and the first of one
COPIED = [(2048, 1, 1024), (2049, 9, 1024), (2500, 37, 1100), (2111, 1001, 1030), (4097, 1001, 1024), (2048, 4095, 4097), (3000, 2047, 2060), (4400, 1537, 1030)]


@pytest.mark.parametrize("kind", [mpcnn.I8, mpcnn.E4M3])
@pytest.mark.parametrize("rows,outs,features", COPIED)
def test_ragged_rows_that_are_copied(rows, outs, features, kind):
    dy, p = _inputs(rows + outs, rows, outs, features, torch.bfloat16, kind)
    dw = mpcnn.rows_weight_grad(dy, p)
    check(dw, dy, p)
    full = mpcnn.rows_weight_grad(dy, p, dw=torch.empty((outs, features), device="cuda"))
    check(full, dy, p)
    assert torch.equal(full.to(torch.bfloat16), dw)
    for offset, pitch in ((1, outs + 3), (3, outs + 8), (0, (outs + 15) // 8 * 8)):       # rows at odd addresses, numbers between them that do not count
        wide = torch.full((rows, pitch + offset), float("nan"), device="cuda", dtype=torch.bfloat16)[:, offset:offset + outs]
        wide.copy_(dy)
        assert torch.equal(mpcnn.rows_weight_grad(wide, p), dw)
    # a workspace that holds what a call on fewer rows left, and whose last bytes are nobody's
    size = mpcnn.weight_grad_workspace_bytes(rows, outs, features, mpcnn.BF16)
    room = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
    mpcnn.rows_weight_grad(dy[:-5], mpcnn.PackedRows(p.values[:-5], p.scales[:-5], features), ws=room[:size])
    assert torch.equal(mpcnn.rows_weight_grad(dy, p, ws=room[:size]), dw) and (room[size:] == 255).all()


# tiles of 256 x 256 in several parts of the rows, the last one shorter
SPLIT = [(2500, 2000, 2000), (5000, 1000, 1000), (6001, 1001, 1000), (3300, 520, 4200), (6001, 2048, 520), (4400, 1536, 1031)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=_ids)
@pytest.mark.parametrize("rows,outs,features", SPLIT)
def test_large_tiles_of_split_rows(rows, outs, features, dtype):
    for kind in (mpcnn.I8, mpcnn.E4M3):
        dy, p = _inputs(rows + features, rows, outs, features, dtype, kind)
        dw = mpcnn.rows_weight_grad(dy, p)
        check(dw, dy, p)
        assert torch.equal(dw, mpcnn.rows_weight_grad(dy, p))
        wide = torch.full((rows, outs + 9), float("nan"), device="cuda", dtype=dtype)[:, 1:outs + 1]      # (bf16: not straight into LDS)
        wide.copy_(dy)
        check(mpcnn.rows_weight_grad(wide, p), dy, p)


@pytest.mark.parametrize("size", [-100, -112, -120, -126, -130])
def test_smallest_numbers(size):
    """fp32 dy down to its smallest numbers, with large ones of x: the three parts have every bit from 2^-133 on, so that a number is off by at most as much."""
    gen = torch.Generator(device="cuda").manual_seed(-size)
    dy = (torch.randn((200, 70), generator=gen, device="cuda").double() * 2.0 ** size).float()
    p = mpcnn.rows_pack(torch.randn((200, 90), generator=gen, device="cuda") * 2.0 ** 80, mpcnn.I8)
    x, dw = mpcnn.rows_unpack(p).double(), mpcnn.rows_weight_grad(dy, p).double()
    want, terms = dy.double().t() @ x, dy.double().abs().t() @ x.abs()
    assert ((dw - want).abs() <= (2 * (200 + 16) + 64 + 2) * U * terms + U * want.abs() + 2.0 ** -133 * x.abs().sum(0) + 1e-38).all()
    halves = dy.to(torch.bfloat16)                        # (bf16 numbers are taken as they are)
    got = mpcnn.rows_weight_grad(halves, p, dw=torch.empty((70, 90), device="cuda")).double()
    want, terms = halves.double().t() @ x, halves.double().abs().t() @ x.abs()
    assert ((got - want).abs() <= (2 * (200 + 16) + 64 + 2) * U * terms + U * want.abs() + 1e-38).all()
