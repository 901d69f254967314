"""Beam search's selection and its states against plain forms in 64 bits.

A log sum is off by what its exponentials are: their argument x - top (which counts up to 24 before nothing is left), log2 e times it and its own rounding,
3 u of the argument, the exponential's two half steps, and the sums one after the other in a lane: 16 of each chunk of 1024 classes that a wave has."""
import math

import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]
INF = math.inf


def _ids(v):
    return str(v).replace("torch.", "")


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _off(classes, rows):
    chunks = -(-classes // 1024)
    wave = -(-max(4, -(-chunks // max(1, 1024 // max(1, rows)))) // 4)
    return (3 * 24 + 4 + 16 * wave + 8 + 8) * U


def values_in_64(scores, totals, bias, done, end):
    """[sequences, beams, classes] of values, minus infinity where there is no candidate."""
    b, k = totals.shape
    s = scores.float()
    if bias is not None:
        s = torch.where(bias == -INF, -INF, s + bias)
    s = s.double().view(b, k, -1)
    lse = torch.logsumexp(torch.nan_to_num(s, nan=INF, posinf=INF, neginf=-INF), 2, keepdim=True)
    lse = torch.where(torch.isfinite(lse), lse, INF)                     # (such a beam offers nothing)
    value = totals.double()[:, :, None] + (s - lse)
    value = torch.where(torch.isfinite(lse) & (s > -INF), value, -INF)
    if done is not None:
        over = torch.full_like(value, -INF)
        over[:, :, end] = totals.double()
        value = torch.where(done[:, :, None], over, value)
    return torch.where(torch.isfinite(totals)[:, :, None], value, -INF)


def check(got, scores, totals, width, bias=None, done=None, end=-1, more=0.0):
    b, k = totals.shape
    value = values_in_64(scores, totals, bias, done, end)
    v = value.shape[2]
    flat = value.view(b, k * v)
    order = torch.sort(flat, dim=1, descending=True, stable=True)       # (equals by the lowest place)
    want, at = order.values[:, :width + 1], order.indices[:, :width + 1]
    if want.shape[1] < width + 1:
        fill = width + 1 - want.shape[1]
        want, at = torch.nn.functional.pad(want, (0, fill), value=-INF), torch.nn.functional.pad(at, (0, fill))
    off = 2 * (_off(v, b * k) + more)
    gaps = want[:, :-1] - want[:, 1:]
    beams = at // v
    close = (gaps < off) & (beams[:, :-1] != beams[:, 1:]) & (want[:, 1:] > -INF) & (gaps > 0)
    sure = ~close.any(1)
    assert sure.float().mean() > 0.9                                     # (the inputs are no test otherwise)
    want, at = want[:, :width], at[:, :width]
    none = want == -INF
    totals_out, parents, classes, over = got
    assert totals_out.shape == parents.shape == classes.shape == over.shape == (b, width)
    assert torch.equal(totals_out == -INF, none)
    near = (totals_out.double() - want).abs() <= off + U * want.abs()
    assert (near | none).all()
    assert torch.equal(parents[sure].long(), torch.where(none, -1, at // v)[sure])
    assert torch.equal(classes[sure].long(), torch.where(none, -1, at % v)[sure])
    place = parents.long() * v + classes.long()
    picked = torch.where(none, want, flat.gather(1, place.clamp(min=0)))
    assert ((picked - want).abs().nan_to_num(0.0) <= off).all()
    gone = torch.zeros((b, k), dtype=torch.bool, device="cuda") if done is None else done
    assert torch.equal(over, none | gone.gather(1, parents.long().clamp(min=0)) | (classes == end))


def _inputs(gen, b, k, v, dtype, with_bias=False, finished=0.0):
    scores = (torch.randn((b * k, v), generator=gen, device="cuda") * 2.5).to(dtype)
    totals = -torch.rand((b, k), generator=gen, device="cuda") * 5
    bias = None
    if with_bias:
        bias = torch.randn(v, generator=gen, device="cuda")
        bias[torch.rand(v, generator=gen, device="cuda") < 0.1] = -INF
    done = torch.rand((b, k), generator=gen, device="cuda") < finished if finished else None
    return scores, totals, bias, done


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("with_bias,finished", [(False, 0.0), (True, 0.3)])
@pytest.mark.parametrize("b,k,v,width", [(1, 1, 1, 1), (1, 1, 7, 7), (3, 2, 5, 4), (1, 4, 1000, 4), (2, 3, 1023, 5), (2, 3, 1024, 1), (4, 2, 1025, 8),
                                         (1, 4, 32000, 4), (5, 8, 50021, 8), (2, 64, 3000, 64), (1, 16, 160001, 16), (40, 1, 2049, 33), (300, 4, 700, 4),
                                         (1, 1, 1000003, 64), (1100, 1, 300, 2)])
def test_select(b, k, v, width, with_bias, finished, dtype):
    scores, totals, bias, done = _inputs(_gen(b * 1000 + k * 10 + v), b, k, v, dtype, with_bias, finished)
    end = v // 3 if finished else -1
    got = mpcnn.beam_select(scores, totals, width=width, bias=bias, done=done, end=end)
    check(got, scores, totals, width, bias, done, end)
    again = mpcnn.beam_select(scores, totals, width=width, bias=bias, done=done, end=end)
    assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
def test_strides_and_odd_addresses(dtype):
    gen = _gen(4)
    scores, totals, bias, done = _inputs(gen, 3, 4, 5001, dtype, True, 0.2)
    want = mpcnn.beam_select(scores, totals, bias=bias, done=done, end=9)
    for offset, pitch in ((1, 5003), (3, 5008), (0, 6001)):
        wide = torch.full((12, pitch), float("nan"), device="cuda", dtype=dtype)
        wide[:, offset:offset + 5001] = scores
        got = mpcnn.beam_select(wide[:, offset:offset + 5001], totals, bias=bias, done=done, end=9)
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
def test_equals_go_by_beam_and_class(dtype):
    """Beams that hold the same, at addresses of which some are odd, and scores of few values."""
    gen = _gen(6)
    for v in (37, 3001, 20011):
        row = torch.randint(0, 4, (v,), generator=gen, device="cuda").to(dtype)
        scores, totals = row.repeat(6, 1), torch.full((1, 6), -2.5, device="cuda")
        total, parents, classes, _ = mpcnn.beam_select(scores, totals, width=40)
        best = torch.nonzero(row == 3).squeeze(1)
        if len(best) >= 40:                                  # all of the first beam, in the classes' order
            assert (parents == 0).all() and torch.equal(classes[0].long(), best[:40]) and (total == total[0, 0]).all()
        else:
            want = [(k, int(c)) for k in range(6) for c in best][:40]
            assert [(int(p), int(c)) for p, c in zip(parents[0], classes[0])][:len(want)] == want


def test_all_in_one_chunk_or_one_beam():
    scores = torch.zeros((4, 9000), device="cuda")
    scores[2, 3000:3064] = 20 + torch.arange(64, device="cuda") * 0.01
    totals = torch.zeros((1, 4), device="cuda")
    got = mpcnn.beam_select(scores, totals, width=64)
    check(got, scores, totals, 64)
    assert (got[1] == 2).all() and torch.equal(got[2][0].long(), torch.arange(3063, 2999, -1, device="cuda"))
    scores = torch.zeros((4, 9000), device="cuda")            # 64 chunks' worth of the same
    got = mpcnn.beam_select(scores, totals, width=64)
    assert (got[1] == 0).all() and torch.equal(got[2][0].long(), torch.arange(64, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
def test_dead_beams_masked_classes_and_bad_scores(dtype):
    gen = _gen(7)
    scores, totals, bias, _ = _inputs(gen, 7, 3, 2500, dtype, True)
    totals[0, 1] = totals[1, :2] = totals[2] = -INF
    scores[1] = float("nan")                                  # dead: not looked at
    off = torch.nonzero(bias == -INF).squeeze(1)
    scores[:, off[0]], scores[:, off[1]] = float("nan"), INF   # switched off, whatever they hold
    scores[9, 77 if bias[77] > -INF else 78] = float("nan")   # sequence 3, beam 0: offers nothing
    scores[13, 5 if bias[5] > -INF else 6] = INF              # sequence 4, beam 1
    scores[15] = -INF                                         # sequence 5, beam 0: no class on
    scores[18:21] = -INF                                      # sequence 6: nothing
    done = torch.zeros((7, 3), dtype=torch.bool, device="cuda")
    done[5, 1] = done[2, 0] = True
    scores[16] = float("nan")                                 # finished: not looked at
    totals[4, 2], totals[3, 2] = float("nan"), INF
    got = mpcnn.beam_select(scores, totals, width=5, bias=bias, done=done, end=11)
    check(got, scores, totals, 5, bias, done, 11)
    assert (got[1][2] == -1).all() and (got[1][6] == -1).all() and (got[1][1] == 2).all() and not (got[1][3] == 0).any()
    assert ((got[1][5] == 1).sum() == 1) and not (got[1][4] == 1).any() and not (got[1][4] == 2).any() and not (got[1][3] == 2).any() and got[3][2].all()


def test_few_candidates():
    scores = torch.randn((2, 3), generator=_gen(1), device="cuda")
    totals = torch.tensor([[-1.0, -2.0]], device="cuda")
    got = mpcnn.beam_select(scores, totals, width=64)
    check(got, scores, totals, 64)
    assert (got[1][0, :6] >= 0).all() and (got[1][0, 6:] == -1).all() and (got[2][0, 6:] == -1).all() and got[3][0, 6:].all()
    done = torch.ones((1, 2), dtype=torch.bool, device="cuda")
    total, parents, classes, over = mpcnn.beam_select(torch.full_like(scores, float("nan")), totals, width=3, done=done, end=1)
    assert total.tolist() == [[-1.0, -2.0, -INF]] and parents.tolist() == [[0, 1, -1]] and classes.tolist() == [[1, 1, -1]] and over.all()
    none = mpcnn.beam_select(torch.empty((0, 5), device="cuda"), torch.empty((0, 4), device="cuda"))
    assert all(t.shape == (0, 4) for t in none)


def test_binding_refusals():
    scores, totals = torch.zeros((6, 50), device="cuda"), torch.zeros((2, 3), device="cuda")
    done, cache = torch.zeros((2, 3), dtype=torch.bool, device="cuda"), torch.zeros((6, 4), device="cuda")
    states = mpcnn.BeamStates([cache], 2, 3)
    good = mpcnn.beam_select(scores, totals, done=done, end=0)
    x, w = torch.zeros((6, 8), device="cuda"), torch.zeros((50, 8), device="cuda")
    calls = [(lambda width=width: mpcnn.beam_select(scores, totals, width)) for width in (0, -1, 65, 1 << 40)] + [
        lambda: mpcnn.beam_select(scores, totals, done=done), lambda: mpcnn.beam_select(scores, totals, done=done, end=50), lambda: mpcnn.beam_select(scores, totals.double()),
        lambda: mpcnn.beam_select(scores, totals.t()), lambda: mpcnn.beam_select(scores, totals.view(3, 2), done=done, end=0), lambda: mpcnn.beam_select(scores[:5], totals),
        lambda: mpcnn.beam_select(scores.half(), totals), lambda: mpcnn.beam_select(scores.t().contiguous().t(), totals), lambda: mpcnn.beam_select(scores, totals, bias=scores[0, :49]),
        lambda: mpcnn.beam_select(scores, totals, done=done.int(), end=0), lambda: mpcnn.beam_select(scores, totals.cpu()), lambda: mpcnn.beam_select(scores, totals, width=2, out=good),
        lambda: mpcnn.beam_select(scores, totals, out=(totals,) + good[1:]), lambda: mpcnn.beam_select(scores, totals, out=(good[0], good[1], good[1], good[3])),
        lambda: mpcnn.beam_select(scores, totals, ws=torch.empty(64, dtype=torch.uint8, device="cuda")), lambda: mpcnn.class_beam(x, w[:, :7], totals),
        lambda: mpcnn.class_beam(x, w.bfloat16(), totals), lambda: mpcnn.class_beam(x, w, totals, width=0), lambda: mpcnn.class_beam(x[:4], w, totals),
        lambda: mpcnn.BeamStates([cache[:5]], 2, 3), lambda: mpcnn.BeamStates([cache.t().contiguous().t()], 2, 3), lambda: mpcnn.BeamStates([cache], 2, 3, axis=2),
        lambda: mpcnn.BeamStates([cache, cache], 2, 3), lambda: states.reorder(good[1].long()), lambda: states.reorder(good[1][:1]), lambda: states.reorder(good[1], length=-1),
        lambda: states.reorder(cache.view(torch.int32)[:2, :3].contiguous().t())]
    for k, call in enumerate(calls):
        with pytest.raises(mpcnn.MpcnnError):
            call()
            pytest.fail("call %d was not refused" % k)


def test_far_classes_and_far_rows():
    """A class beyond 2^24 and rows beyond 2^32 bytes."""
    v = 40000001
    scores = torch.zeros((2, v), device="cuda", dtype=torch.bfloat16)
    scores[0, v - 1], scores[1, 33554433], scores[1, 33554434] = 30.0, 29.0, 28.0
    totals = torch.tensor([[-1.0, -1.5]], device="cuda")
    got = mpcnn.beam_select(scores, totals, width=3)
    assert got[1].tolist() == [[0, 1, 1]] and got[2].tolist() == [[v - 1, 33554433, 33554434]]
    pitch = 1500000000
    far = torch.empty(2 * pitch + 3000, dtype=torch.bfloat16, device="cuda").as_strided((3, 3000), (pitch, 1))
    near = torch.randn((3, 3000), generator=_gen(2), device="cuda").to(torch.bfloat16)
    far.copy_(near)
    totals = torch.zeros((1, 3), device="cuda")
    assert all(torch.equal(x, y) for x, y in zip(mpcnn.beam_select(far, totals), mpcnn.beam_select(near, totals)))


# ---- from rows of features

# The class layer adds at most 64 exponentials one after the other in a lane where `_off` counts 16 of a wave's chunk (48 u more), and the tiles' sums are joined by one more
# exponential (3 u of its argument, its two half steps and two products: 76 u)
TILES = (48 + 76) * U


def _whole(gen, rows, features, dtype, most):
    return torch.randint(-most, most + 1, (rows, features), generator=gen, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("with_bias,finished", [(False, 0.0), (True, 0.3)])
@pytest.mark.parametrize("b,k,features,v,width", [(1, 1, 5, 3, 2), (1, 4, 1024, 32000, 4), (1, 2, 64, 30011, 8), (2, 3, 100, 2000, 3), (3, 4, 1000, 25000, 6), (5, 8, 333, 5001, 8),
                                                  (1, 64, 96, 1025, 64), (16, 8, 256, 700, 8), (20, 16, 64, 9000, 4), (16, 4, 512, 24001, 4), (25, 4, 600, 20001, 4), (1, 4, 2050, 35001, 4), (8, 4, 2048, 20480, 4), (4, 2, 4096, 33000, 2)])
def test_class_beam(b, k, features, v, width, with_bias, finished, dtype):
    """Features and class weights are whole numbers, biases multiples of 1/64: every order of the products' sum gives the same score, exactly."""
    gen = _gen(b * 7 + k * 11 + features + v)
    x, w = _whole(gen, b * k, features, dtype, 3), _whole(gen, v, features, dtype, 2)
    _, totals, bias, done = _inputs(gen, b, k, 1, dtype, False, finished)
    if with_bias:
        bias = torch.randint(-64, 64, (v,), generator=gen, device="cuda").float() / 64
        bias[torch.rand(v, generator=gen, device="cuda") < 0.1] = -INF
    if b > 1:
        totals[1, 1:] = -INF
        x[k + 1:2 * k] = float("nan")                     # dead beams' rows may hold anything
    scores = torch.nan_to_num(x.double(), nan=0.0) @ w.double().t()
    assert scores.abs().max() < 2.0 ** 18
    end = v // 3 if finished else -1
    got = mpcnn.class_beam(x, w, totals, width=width, bias=bias, done=done, end=end)
    check(got, scores.float(), totals, width, bias, done, end, TILES)
    assert all(torch.equal(p, q) for p, q in zip(got, mpcnn.class_beam(x, w, totals, width=width, bias=bias, done=done, end=end)))


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
def test_class_beam_of_strided_rows_and_real_numbers(dtype):
    gen = _gen(77)
    b, k, features, v = 2, 3, 200, 3001
    x, w = torch.randn((b * k, features), generator=gen, device="cuda").to(dtype), (torch.randn((v, features), generator=gen, device="cuda") * 0.1).to(dtype)
    totals = -torch.rand((b, k), generator=gen, device="cuda")
    want = mpcnn.class_beam(x, w, totals)
    for offset in (1, 2):
        wide_x, wide_w = torch.zeros((b * k, 207), device="cuda", dtype=dtype), torch.zeros((v, 211), device="cuda", dtype=dtype)
        wide_x[:, offset:offset + 200], wide_w[:, offset:offset + 200] = x, w
        got = mpcnn.class_beam(wide_x[:, offset:offset + 200], wide_w[:, offset:offset + 200], totals)
        assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    # a score is off by 2 (n + 16) u of its products' magnitudes, and by 2^-22 of them with fp32 (three parts); a value by that, and its log sum's
    size = (x.double().abs() @ w.double().abs().t()).max()
    off = 2 * ((2 * (features + 16) + 4) * U * size + _off(v, b * k) + TILES)
    value = values_in_64(x.double() @ w.double().t(), totals, None, None, -1).view(b, -1)
    best = torch.sort(value, dim=1, descending=True).values[:, :k]
    assert ((want[0].double() - best).abs() <= off + U * best.abs()).all()
    place = want[1].long() * v + want[2].long()
    assert ((value.gather(1, place) - best).abs() <= off).all()


PATHS = [(2, 4, 1024, 32000), (16, 8, 256, 5000), (1, 3, 64, 300003), (1, 2, 40, 700000), (3, 5, 200, 1000), (2, 8, 512, 24001), (8, 4, 768, 40021), (1, 1, 9, 65)]


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("b,k,features,v", PATHS)
def test_class_beam_of_equal_beams(b, k, features, v, dtype):
    """Beams that hold the same offer the same: the best class by each beam in turn."""
    gen = _gen(b + k + features + v)
    one, w = torch.randn((b, 1, features), generator=gen, device="cuda").to(dtype), torch.randn((v, features), generator=gen, device="cuda").to(dtype)
    x = one.expand(b, k, features).reshape(b * k, features).contiguous()      # (rows that share memory are refused)
    totals = (-torch.rand((b, 1), generator=gen, device="cuda")).expand(b, k).contiguous()
    got = mpcnn.class_beam(x, w, totals)
    assert torch.equal(got[1], torch.arange(k, device="cuda", dtype=torch.int32).expand(b, k)) and (got[2] == got[2][:, :1]).all() and (got[0] == got[0][:, :1]).all()
    best = (one[:, 0].double() @ w.double().t()).argmax(1)             # (no two scores of random numbers are nearer than a score's error here)
    assert torch.equal(got[2][:, 0].long(), best)


@pytest.mark.parametrize("dtype", TYPES, ids=_ids)
@pytest.mark.parametrize("b,k,features,v", PATHS)
def test_class_beam_of_bad_rows_and_masks(b, k, features, v, dtype):
    """A live beam whose scores are NaN offers nothing, nor does any where every class is off; a single class that is on is offered at its total."""
    gen = _gen(b + k + features + v)
    x, w = torch.randn((b * k, features), generator=gen, device="cuda").to(dtype), torch.randn((v, features), generator=gen, device="cuda").to(dtype)
    totals = -torch.rand((b, k), generator=gen, device="cuda")
    x[0, 3] = float("nan")
    got = mpcnn.class_beam(x, w, totals)
    assert not (got[1][0] == 0).any() and (b * k == 1 or (got[1][-1] >= 0).all())
    bias = torch.full((v,), -INF, device="cuda")
    none = mpcnn.class_beam(x, w, totals, bias=bias)
    assert (none[0] == -INF).all() and (none[1] == -1).all() and (none[2] == -1).all() and none[3].all()
    bias[v - 2] = 1.0
    one = mpcnn.class_beam(x, w, totals, bias=bias)
    totals[0, 0] = -INF
    want = torch.sort(totals, dim=1, descending=True)
    assert torch.equal(one[0], want.values) and torch.equal(one[2] == v - 2, want.values > -INF)
    assert torch.equal(one[1].long(), torch.where(want.values > -INF, want.indices, -1))


def test_class_beam_in_a_graph_and_with_one_workspace():
    gen = _gen(78)
    b, k, features, v = 4, 4, 256, 6000
    x, w = _whole(gen, b * k, features, torch.bfloat16, 3), _whole(gen, v, features, torch.bfloat16, 2)
    totals = -torch.rand((b, k), generator=gen, device="cuda")
    n = mpcnn.class_beam_workspace_bytes(b, k, features, v, mpcnn.BF16)
    ws = torch.full((n + 512,), 255, dtype=torch.uint8, device="cuda")
    for less in (b, 2, 1):
        got = mpcnn.class_beam(x[:less * k], w, totals[:less], ws=ws[:n])
        assert all(torch.equal(p, q) for p, q in zip(got, mpcnn.class_beam(x[:less * k], w, totals[:less])))
    assert (ws[n:] == 255).all()
    out = mpcnn.class_beam(x, w, totals, ws=ws[:n])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mpcnn.class_beam(x, w, totals, out=out, ws=ws[:n])
    for _ in range(3):
        x.copy_(_whole(gen, b * k, features, torch.bfloat16, 3))
        graph.replay()
        torch.cuda.synchronize()
        check(out, (x.double() @ w.double().t()).float(), totals, k)


# ---- states

def _plain_reorder(t, parents, length=None, axis=None):
    b, k = parents.shape
    kept = torch.where((parents >= 0) & (parents < k), parents.long(), torch.arange(k, device="cuda"))
    rows = (torch.arange(b, device="cuda")[:, None] * k + kept).view(-1)
    new = t.clone()
    if length is None:
        new.copy_(t[rows])
    else:
        at = (slice(None),) * axis + (slice(0, length),)
        new[at] = t[rows][at]
    return new


@pytest.mark.parametrize("b,k", [(1, 1), (1, 2), (3, 4), (2, 5), (5, 8), (2, 13), (3, 16), (1, 31), (2, 33), (1, 64)])
def test_reorder(b, k):
    gen = _gen(b * 100 + k)
    n = b * k
    tensors = [torch.randn((n, 3, 17, 5), generator=gen, device="cuda"), torch.randn((n, 2, 17, 64), generator=gen, device="cuda").to(torch.bfloat16),
               torch.randint(0, 255, (n, 1, 17, 3), generator=gen, device="cuda", dtype=torch.uint8), torch.randn((n, 1, 40, 33), generator=gen, device="cuda").half(),
               torch.randn((n, 4, 17), generator=gen, device="cuda").double(), torch.randn((n, 7, 900, 8), generator=gen, device="cuda"),
               torch.randn((n, 2, 0, 3), generator=gen, device="cuda")]
    for length in (None, 0, 1, 9, 17, 1000):
        parents = torch.randint(-1, k + 1, (b, k), generator=gen, device="cuda", dtype=torch.int32)
        got = [t.clone() for t in tensors]
        states = mpcnn.BeamStates(got, b, k, axis=2)
        states.reorder(parents, length=length)
        for t, g in zip(tensors, got):
            assert torch.equal(g, _plain_reorder(t, parents, length, 2))
        states.close()
    flat = [torch.randn((n, 501), generator=gen, device="cuda"), torch.arange(n, device="cuda"), torch.randn((n, 3), generator=gen, device="cuda").to(torch.bfloat16)]
    got = [t.clone() for t in flat]
    parents = torch.randint(0, k, (b, k), generator=gen, device="cuda", dtype=torch.int32)
    mpcnn.BeamStates(got, b, k).reorder(parents)
    for t, g in zip(flat, got):
        assert torch.equal(g, _plain_reorder(t, parents))


@pytest.mark.parametrize("parents", [[1, 2, 3, 0], [3, 2, 1, 0], [0, 1, 2, 3], [2, 2, 2, 2], [1, 0, 0, 1], [-1, 0, -1, 2]])
def test_reorder_moves_what_was_there(parents):
    t = torch.arange(4 * 70000, device="cuda", dtype=torch.float32).view(4, 70000)
    p = torch.tensor([parents], dtype=torch.int32, device="cuda")
    want = _plain_reorder(t, p)
    mpcnn.BeamStates([t], 1, 4).reorder(p)
    assert torch.equal(t, want)


def test_reorder_with_pitch_leaves_the_rest_alone():
    wide = torch.randn((6, 100), generator=_gen(3), device="cuda")
    was = wide.clone()
    part = wide[:, 3:70]
    p = torch.tensor([[1, 0], [0, 0], [1, 1]], dtype=torch.int32, device="cuda")
    mpcnn.BeamStates([part], 3, 2).reorder(p)
    assert torch.equal(part, _plain_reorder(was[:, 3:70], p)) and torch.equal(wide[:, :3], was[:, :3]) and torch.equal(wide[:, 70:], was[:, 70:])


def test_reorder_of_tensors_that_lie_in_turn():
    both = torch.randn((12, 2, 5, 33), generator=_gen(13), device="cuda").to(torch.bfloat16)      # keys and values of one buffer
    was = both.clone()
    p = torch.tensor([[1, 0, 3, 3], [0, 0, 0, 0], [3, 2, 1, 0]], dtype=torch.int32, device="cuda")
    mpcnn.BeamStates([both[:, 0], both[:, 1]], 3, 4).reorder(p)
    assert torch.equal(both, _plain_reorder(was, p))


def test_reorder_of_many_tensors_and_sequences():
    """More workgroups than a launch has, were every sequence of every tensor one's."""
    buffer = torch.arange(2 * 65535 * 300, dtype=torch.int32, device="cuda").view(2 * 65535, 300)
    p = torch.tensor([1, 0], dtype=torch.int32, device="cuda").repeat(65535, 1)
    p[::7] = torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    want = _plain_reorder(buffer, p)
    mpcnn.BeamStates([buffer[:, i] for i in range(300)], 65535, 2).reorder(p)
    assert torch.equal(buffer, want)


def test_reorder_far_rows():
    t = torch.empty((4, 1200000007), dtype=torch.uint8, device="cuda")       # rows at odd addresses beyond 2^32 bytes
    for i in range(4):
        t[i, :50], t[i, -50:] = i + 1, i + 11
    p = torch.tensor([[3, 0, 2, 2]], dtype=torch.int32, device="cuda")
    mpcnn.BeamStates([t], 1, 4).reorder(p)
    assert t[:, 0].tolist() == [4, 1, 3, 3] and t[:, -1].tolist() == [14, 11, 13, 13] and t[:, 49].tolist() == [4, 1, 3, 3]


def test_a_step_on_another_stream_and_in_a_graph():
    """Selection and reordering together, as a decoding step has them."""
    gen = _gen(11)
    b, k, v = 3, 4, 4001
    scores, totals, bias, done = _inputs(gen, b, k, v, torch.bfloat16, True, 0.2)
    cache = torch.randn((b * k, 2, 50, 16), generator=gen, device="cuda").to(torch.bfloat16)
    first = cache.clone()
    states = mpcnn.BeamStates([cache], b, k, axis=2)
    out = (torch.empty((b, k), device="cuda"), torch.empty((b, k), device="cuda", dtype=torch.int32), torch.empty((b, k), device="cuda", dtype=torch.int32),
           torch.empty((b, k), device="cuda", dtype=torch.bool))
    ws = torch.empty(mpcnn.beam_workspace_bytes(b, k, v), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        mpcnn.beam_select(scores, totals, bias=bias, done=done, end=5, out=out, ws=ws, stream=stream)
        states.reorder(out[1], length=33, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    torch.cuda.current_stream().wait_stream(side)
    check(out, scores, totals, k, bias, done, 5)
    assert torch.equal(cache, _plain_reorder(first, out[1], 33, 2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        scores.copy_((torch.randn((b * k, v), generator=gen, device="cuda") * 2.5))
        cache.copy_(torch.randn(cache.shape, generator=gen, device="cuda"))
        was = cache.clone()
        graph.replay()
        torch.cuda.synchronize()
        check(out, scores, totals, k, bias, done, 5)
        assert torch.equal(cache, _plain_reorder(was, out[1], 33, 2))
    states.close()
