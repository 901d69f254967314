"""Beam search's candidates of equal values, of either sign of zero."""
import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu


def _ids(v):
    return str(v).replace("torch.", "")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=_ids)
def test_zeros_of_either_sign_are_equals(dtype):
    """Candidates of minus zero and zero: the lower beam comes first."""
    totals = torch.tensor([[-0.0, 0.0, -0.0, 0.0], [0.0, -0.0, 0.0, -0.0]], device="cuda")
    scores = torch.zeros((8, 1), device="cuda", dtype=dtype)
    scores[::2] = -0.0                                    # one class: the values are 0
    for done in (None, torch.ones((2, 4), dtype=torch.bool, device="cuda"), torch.tensor([[True, False] * 2, [False, True] * 2], device="cuda")):
        got = mpcnn.beam_select(scores, totals, done=done, end=-1 if done is None else 0)
        assert (got[0] == 0).all() and got[1].tolist() == [[0, 1, 2, 3]] * 2 and (got[2] == 0).all()
        x, w = torch.ones((8, 3), device="cuda", dtype=dtype), torch.zeros((1, 3), device="cuda", dtype=dtype)
        got = mpcnn.class_beam(x, w, totals, done=done, end=-1 if done is None else 0)
        assert (got[0] == 0).all() and got[1].tolist() == [[0, 1, 2, 3]] * 2 and (got[2] == 0).all()
    # many finished beams among chunks of others
    totals = torch.where(torch.arange(64, device="cuda") % 3 == 0, -0.0, 0.0).view(1, 64).contiguous()
    done = torch.ones((1, 64), dtype=torch.bool, device="cuda")
    got = mpcnn.beam_select(torch.zeros((64, 3000), device="cuda", dtype=dtype), totals, done=done, end=7)
    assert got[1][0].tolist() == list(range(64)) and (got[2] == 7).all() and got[3].all()
