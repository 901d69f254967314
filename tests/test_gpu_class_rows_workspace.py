"""One workspace of the class layer on rows for batches of different sizes."""
import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,smaller,features,classes", [(17, (16, 5, 1), 1000, 30011), (6207, (5106, 700, 16), 520, 50257), (65, (64, 33, 12), 256, 20000)])
def test_the_largest_batch_s_workspace_does_for_smaller_ones(rows, smaller, features, classes, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn((rows, features), generator=gen, device="cuda").to(dtype)
    w = (torch.randn((classes, features), generator=gen, device="cuda") * features ** -0.5).to(dtype)
    labels = torch.randint(0, classes, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    bias = torch.randn((classes,), generator=gen, device="cuda")
    kind = mpcnn.BF16 if dtype == torch.bfloat16 else mpcnn.F32
    behind = 4096                                          # (and it is left alone behind what was said)
    n = mpcnn.class_workspace_bytes(rows, features, classes, kind, True)
    ws = torch.full((n + behind,), 255, dtype=torch.uint8, device="cuda")
    for r in (rows, *smaller):
        got = mpcnn.class_backward(x[:r], w, labels[:r], bias=bias, ws=ws[:n])
        want = mpcnn.class_backward(x[:r], w, labels[:r], bias=bias)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert (ws[n:] == 255).all()
    n = mpcnn.class_workspace_bytes(rows, features, classes, kind, False)
    for r in (rows, *smaller):
        for a, b in zip(mpcnn.class_loss(x[:r], w, labels[:r], bias=bias, ws=ws[:n]), mpcnn.class_loss(x[:r], w, labels[:r], bias=bias)):
            assert torch.equal(a, b)
