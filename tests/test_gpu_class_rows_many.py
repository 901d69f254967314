"""The class layer on rows at the most classes that launches can be made for, against the formulas in 64 bits.

Tolerances, u = 2^-24.  A score s = x . w + bias with S = sum |x w|: (features + 4) u S + 2 u |s|, in fp32 2^-20 S more (parts: 3 2^-22, and 2^-38 of the largest x
and w times the features).  lse: a number of the sum passes 64 additions in its tile, then those of the joins, of which one of at least 64 threads makes
tiles / 64, and at most 64 behind: (tiles / 64 + 128) u + 8 u (|lse| + 1).  p: 2 (both + 8 u |s - lse|)."""
import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16
U = 2.0 ** -24


def _lse(x, w, bias=None):
    """log sum exp of the scores in 64 bits, over pieces of the classes; and the largest sum of magnitudes"""
    parts, size = [], 0.0
    step = max(1, (1 << 28) // x.shape[0])
    for at in range(0, w.shape[0], step):
        s = x.double() @ w[at:at + step].double().t()
        size = max(size, float((x.double().abs() @ w[at:at + step].double().abs().t()).max()))
        parts.append(torch.logsumexp(s if bias is None else s + bias[at:at + step].double(), 1))
    return torch.logsumexp(torch.stack(parts), 0), size


def _e_lse(lse, size, features, classes, dtype):
    return ((features + 4) * U + (2.0 ** -20 if dtype == F else 0)) * size + (classes / 128 / 64 + 128) * U + 8 * U * (lse.abs() + 1)


@pytest.mark.parametrize("dtype,rows,classes", [(F, 70, (1 << 28) - 64), (B, 14, (1 << 30) - 64)], ids=["f32-70-below", "bf16-14-below"])
def test_loss_over_hundreds_of_millions_of_classes(dtype, rows, classes):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    w = torch.empty((classes, 1), dtype=dtype, device="cuda").normal_(generator=gen)
    w[classes - 1], w[0] = 24.0, -24.0                       # the last class is a good part of a positive row's sum, the first of a negative one's
    x = (torch.rand((rows, 1), generator=gen, device="cuda") * 0.1 + 0.8).to(dtype)
    x[1::2] *= -1
    labels = torch.tensor([0, classes - 1, classes // 2, classes - 2, 77], dtype=torch.int32, device="cuda").repeat(rows)[:rows]
    loss, rowloss, lse = mpcnn.class_loss(x, w, labels)
    want, size = _lse(x, w)
    e = _e_lse(want, size, 1, classes, dtype)
    assert ((lse.double() - want).abs() <= e).all()
    nll = want - (x.double() * w[labels.long()].double()).sum(1)
    assert ((rowloss.double() - nll).abs() <= 2 * e).all()
    assert abs(loss.item() - rowloss.double().sum().item()) <= 1e-12 * rowloss.double().abs().sum().item()
    del w
    torch.cuda.empty_cache()
