"""Lists of which few tensors share memory: what they do not concern takes no launches of its own, and the results are those of the list's order.

Tolerance: a step p - f g is one fused operation with f rounded to fp32 (2^-24 of |f g|) and rounded once (2^-24 of the result), twice for a tensor that is named
twice; a clipped gradient is g fl(c), rounded once (2^-23 in all), twice for one that is named twice."""
import ctypes
import gc
import math

import pytest
import torch

from paper_1302_1690_amd import mpcnn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _nothing_is_left():
    yield
    gc.collect()


def _launches(call):
    """What a call launches: the nodes of a graph that it is recorded into, which is then run."""
    graph, side = torch.cuda.CUDAGraph(keep_graph=True), torch.cuda.Stream()
    norm = torch.zeros(1, dtype=torch.float64, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call(norm)
    path = next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line)
    nodes = ctypes.c_size_t()
    assert ctypes.CDLL(path).hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(nodes)) == 0
    graph.instantiate()
    graph.replay()
    torch.cuda.synchronize()
    return nodes.value, norm.item()


def _tensors(count, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(500 + 7 * k, generator=gen, device="cuda") for k in range(count)]


def test_a_tied_weight():
    grads, params = _tensors(200, 1), _tensors(200, 2)
    params[150] = params[3].view(-1)                                      # the same memory again
    grads[150] = torch.randn_like(params[3])
    start = [p.double() for p in params]
    norm64 = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    steps = mpcnn.GradList(grads, params)
    nodes, norm = _launches(lambda norm: steps.sgd_step(0.5, max_norm=norm64 / 4, norm=norm))
    assert abs(norm - norm64) <= 1e-10 * norm64
    assert nodes == 3, nodes                                             # the norm's, and the two runs'
    f = 0.5 / 4
    for k, (g, p) in enumerate(zip(grads, params)):
        moved = f * g.double()
        if k in (3, 150):
            moved = f * (grads[3].double() + grads[150].double())
            size = f * (grads[3].double().abs() + grads[150].double().abs())
        else:
            size = moved.abs()
        off = (p.double() - (start[k] - moved)).abs()
        assert (off <= 2.0 ** -22 * (start[k].abs() + size)).all(), k


def test_what_is_only_read_may_be_shared():
    """A step writes no gradient, clipping no parameter: two launches, however much of them is shared."""
    params = _tensors(80, 3)
    g = torch.randn(4000, device="cuda")
    shared = [g[k:k + p.numel()] for k, p in enumerate(params)]
    start = [p.double() for p in params]
    steps = mpcnn.GradList(shared, params)
    nodes, _ = _launches(lambda norm: steps.sgd_step(0.25, norm=norm))
    assert nodes == 2, nodes
    for p, s, q in zip(params, start, shared):
        assert ((p.double() - (s - 0.25 * q.double())).abs() <= 2.0 ** -22 * (s.abs() + q.double().abs())).all()
    grads = _tensors(80, 4)
    weight = torch.randn(4000, device="cuda")
    kept = [q.double() for q in grads]
    norm64 = math.sqrt(sum(float(q.square().sum()) for q in kept))
    steps = mpcnn.GradList(grads, [weight[:q.numel()] for q in grads])
    nodes, _ = _launches(lambda norm: steps.clip(norm64 / 2, norm=norm))
    assert nodes == 2, nodes
    for q, k in zip(grads, kept):
        assert ((q.double() - k / 2).abs() <= 2.0 ** -23 * k.abs()).all()


def test_runs_end_where_a_tensor_meets_one_of_its_run():
    """Neighbours that touch share nothing; one inside another, one across two others, and one named three times do."""
    b = torch.randn(60000, device="cuda")
    cuts = [(0, 20000), (20000, 20001), (20001, 40000), (5000, 5010), (39990, 40010), (45000, 60000), (45000, 60000), (45000, 60000), (100, 200)]
    kept = b.double()
    want, views = kept.clone(), [b[i:j] for i, j in cuts]
    norm64 = math.sqrt(sum(float(v.double().square().sum()) for v in views))
    for i, j in cuts:
        want[i:j] /= 2
    steps = mpcnn.GradList(views)
    nodes, norm = _launches(lambda norm: steps.clip(norm64 / 2, norm=norm))
    assert abs(norm - norm64) <= 1e-10 * norm64
    assert nodes == 1 + 4, nodes               # 0-2 | 3, 4, 5 | 6 | 7, 8
    assert ((b.double() - want).abs() <= 2.0 ** -22 * want.abs()).all()
