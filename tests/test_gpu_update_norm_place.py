"""The norm's place may be beside the tensors of a list, not inside one."""
import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu


def test_a_norm_inside_a_tensor_is_refused():
    b = torch.randn(4096, device="cuda")
    places = b.view(torch.float64)
    grads, params = [b[100:200], b[200:300], b[1000:1003]], [b[500:600], b[700:800], b[601:604]]
    lists = mpcnn.GradList(grads), mpcnn.GradList(grads, params)
    kept = b.clone()
    inside = [50, 99, 100, 149, 500, 501]                    # of 8 bytes each: numbers 2 k and 2 k + 1
    for l in lists:
        for k in inside:
            for call in (lambda: l.norm(norm=places[k:k + 1]), lambda: l.clip(1e-3, norm=places[k:k + 1])):
                with pytest.raises(mpcnn.MpcnnError) as e:
                    call()
                assert e.value.status == 1 and "norm" in str(e.value)
    for k in (250, 299, 300, 301, 399, *inside):             # parameters too: 500 .. 599 and 601 .. 603, 700 .. 799
        with pytest.raises(mpcnn.MpcnnError):
            lists[1].sgd_step(0.1, norm=places[k:k + 1])
    assert torch.equal(b, kept)
    want = sum(g.double().square().sum() for g in grads).sqrt().item()
    for k in (0, 49, 150, 499, 502, 2047):
        assert abs(lists[0].norm(norm=places[k:k + 1]).item() - want) <= 1e-10 * want
    for k in (249, 302, 349, 400):
        assert abs(lists[1].norm(norm=places[k:k + 1]).item() - want) <= 1e-10 * want
