"""Norm, clipping and gradient step over lists of tensors, and the net's clipped step, against the definitions in 64 bits.

Tolerances.  The norm is summed in fp64: n additions of one sign are off by less than n 2^-53 (here n per chain is under 2^18), and the
comparison's own sum as much.  A clipped gradient is g fl(c): c rounded to fp32 (half a step, 2^-24), the product rounded to the tensor's
type (2^-24, or fp32 and then bf16: 2^-24 + 2^-8).  A step p - f g is one fused operation with f rounded to fp32 (2^-24 of |f g|), rounded
once to fp32 (2^-24 of the result) and, for bf16 parameters, once more (2^-8)."""
import gc
import math

import numpy as np
import pytest
import torch

from paper_1302_1690_amd import mpcnn, workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _nothing_is_left():
    """Tensors that caught exceptions keep in reference cycles go now, not while another test watches the allocator."""
    yield
    gc.collect()


F, B = torch.float32, torch.bfloat16
HALF = {F: 2.0 ** -24, B: 2.0 ** -8 + 2.0 ** -24}


def _tensors(sizes, types, seed, spread=1.0, offset=0):
    """Views of one buffer per tensor that start `offset` elements in."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n + offset, generator=gen, device="cuda") * spread).to(t)[offset:] for n, t in zip(sizes, types)]


def _norm64(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


CASES = [
    ([1], [F], 0), ([7], [B], 1), ([0, 5, 0], [F, B, F], 0), ([511, 512, 513], [F, B, F], 0), ([2049, 3, 4096 + 511], [B, F, B], 3),
    ([16384], [F], 0), ([16385], [F], 1),                                  # the last list in one launch, the first in two
    ([1 + 37 * k % 300 for k in range(65)], [B if k % 2 else F for k in range(65)], 1),
    ([3000 + k for k in range(40)], [F] * 40, 1), ([1000003], [B], 5), ([8192 * 5 + 1, 777777, 12], [F, F, B], 2),
    ([5000011, 4999999], [F, B], 1),
]


@pytest.mark.parametrize("sizes,types,offset", CASES, ids=range(len(CASES)))
def test_norm_clip_and_step(sizes, types, offset):
    grads = _tensors(sizes, types, 1, offset=offset)
    others = [B if k % 2 else F for k in range(len(sizes))]
    params = _tensors(sizes, others, 2, offset=(offset * 3) % 5)
    want = _norm64(grads)
    kept_g, kept_p = [g.clone() for g in grads], [p.clone() for p in params]
    with_params = mpcnn.GradList(grads, params)
    for scale in (1.0, -0.25):
        got = with_params.norm(grad_scale=scale)
        assert abs(got.item() - abs(scale) * want) <= 1e-10 * want
    # step, bounded at half the norm and not bounded
    for bound, lr, scale in ((0.25 * want + 1e-30, 0.3, 0.5), (math.inf, 0.01, 1.0)):
        before = [p.clone() for p in params]
        got = with_params.sgd_step(lr, grad_scale=scale, max_norm=bound)
        assert abs(got.item() - scale * want) <= 1e-10 * want
        f = lr * scale * min(1.0, bound / (scale * want))
        for g, k, p, b in zip(grads, kept_g, params, before):
            assert torch.equal(g, k)                                       # gradients are read only
            exact = b.double() - f * g.double()
            # (2^-22: three roundings of at most 2^-24 of |f g| and the fp64 factor's)
            off = (p.double() - exact).abs() - (HALF[p.dtype] * exact.abs() * 1.01 + 2.0 ** -22 * f * g.double().abs())
            assert off.numel() == 0 or off.max().item() <= 1e-40
    # clipping: nothing within the bound, half otherwise
    grads_only = mpcnn.GradList(grads)
    assert abs(grads_only.clip(want * 1.001).item() - want) <= 1e-10 * want
    for g, k in zip(grads, kept_g):
        assert torch.equal(g, k)
    assert abs(grads_only.clip(want / 2).item() - want) <= 1e-10 * want
    for g, k in zip(grads, kept_g):
        exact = 0.5 * k.double()
        off = (g.double() - exact).abs() - (HALF[g.dtype] + 2.0 ** -23) * exact.abs() * 1.01
        assert off.numel() == 0 or off.max().item() <= 1e-40
    with_params.close()
    grads_only.close()


def test_what_lies_beside_a_tensor_is_left_alone():
    for t, n in ((F, 1000), (B, 1001), (B, 40001), (F, 70003)):
        buffer = torch.full((n + 64,), 3.0, device="cuda").to(t)
        at = buffer[31:31 + n]
        at.copy_(torch.randn(n, device="cuda"))
        mpcnn.GradList([at]).clip(0.5)
        pbuf = torch.full((n + 64,), 5.0, device="cuda").to(t)
        mpcnn.GradList([at], [pbuf[33:33 + n]]).sgd_step(0.1)
        assert (buffer[:31] == 3).all() and (buffer[31 + n:] == 3).all()
        assert (pbuf[:33] == 5).all() and (pbuf[33 + n:] == 5).all()


def test_empty_list_and_zero_gradients():
    e = mpcnn.GradList([])
    assert e.norm().item() == 0.0 and e.clip(1.0).item() == 0.0 and e.sgd_step(0.1).item() == 0.0
    z = torch.zeros(100, device="cuda")
    p = torch.ones(100, device="cuda")
    l = mpcnn.GradList([z], [p])
    assert l.sgd_step(0.1, max_norm=1e-3).item() == 0.0
    assert (p == 1).all() and (z == 0).all()


def test_large_and_small_magnitudes():
    """Squares beyond fp32's range on both sides."""
    for size in (1e30, 1e-30):
        g = torch.full((5000,), size, device="cuda")
        l = mpcnn.GradList([g])
        want = float(g[0].double()) * math.sqrt(5000.0)
        assert abs(l.norm().item() / want - 1) < 1e-10
        l.clip(want / 4)
        assert abs(l.norm().item() / want - 0.25) < 1e-6


@pytest.mark.parametrize("n", [100, 50000])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_a_norm_that_is_not_finite_changes_nothing(n, bad):
    g = torch.randn(n, device="cuda")
    g[n // 3] = bad
    p = torch.randn(n, device="cuda")
    kg, kp = g.clone(), p.clone()
    l = mpcnn.GradList([g], [p])
    for got in (l.sgd_step(0.1, max_norm=1.0), l.clip(1.0), l.norm()):
        assert math.isnan(got.item()) if math.isnan(bad) else got.item() == math.inf
    assert torch.equal(p, kp) and torch.equal(g.view(torch.int32), kg.view(torch.int32))


def test_equal_results_every_time():
    sizes = [100001, 33, 250007]
    g = _tensors(sizes, [F, B, B], 4)
    l = mpcnn.GradList(g)
    first = l.norm().item()
    for _ in range(20):
        assert l.norm().item() == first


@pytest.mark.parametrize("which", [0, 1])
def test_net_clipped_step(which):
    """The net's own parameters: small (one launch) and larger (two)."""
    cfg = wl.crop(wl.CONFIGS[which], 1, wl.CONFIGS[which].patch + 9, wl.CONFIGS[which].patch + 12)
    img, lab = wl.make_inputs(cfg)
    net = mpcnn.Net(cfg.layers, cfg.in_channels, cfg.patch)
    p0 = wl.make_params(cfg)
    net.set_params(p0)
    d_img, d_lab = torch.from_numpy(img).cuda(), torch.from_numpy(lab).cuda()
    net.seg_backward(d_img, d_lab)
    g = net.get_grads().astype(np.float64)
    norm = torch.zeros(1, dtype=torch.float64, device="cuda")
    want = np.sqrt((g * g).sum())
    for bound, lr, scale in ((0.1 * want, 0.5, 1.0), (math.inf, 0.01, 0.125), (1e3 * want, 0.02, 1.0)):
        before = net.get_params().astype(np.float64)
        net.sgd_step_clipped(lr, bound, grad_scale=scale, norm=norm)
        assert abs(norm.item() - scale * want) <= 1e-10 * want
        f = lr * scale * min(1.0, bound / (scale * want))
        exact = before - f * g
        off = np.abs(net.get_params() - exact) - (2.0 ** -24 * np.abs(exact) * 1.01 + 2.0 ** -22 * f * np.abs(g))
        assert off.max() <= 1e-40
    # without a bound it is sgd_step's sum, up to that one's rounding of lr * grad_scale
    before = net.get_params()
    net.sgd_step_clipped(0.25, math.inf, grad_scale=0.5)
    a = net.get_params()
    net.set_params(before)                                                 # (the gradient stays in the net)
    net.sgd_step(0.25, 0.5)
    np.testing.assert_array_equal(a, net.get_params())
    # and the next forward sees the new parameters
    probs = net.seg_forward(d_img).cpu().numpy()
    net.set_params(net.get_params())
    np.testing.assert_array_equal(probs, net.seg_forward(d_img).cpu().numpy())
    net.close()


@pytest.mark.parametrize("n", [60, 30000])
def test_tensors_that_share_memory(n):
    """One weight with two gradients, a list that names a gradient twice, one that overlaps the next: tensor by tensor, in order."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    w, g = torch.randn(n, generator=gen, device="cuda"), [torch.randn(n, generator=gen, device="cuda") for _ in range(2)]
    start = w.clone()
    norm = mpcnn.GradList(g, [w, w]).sgd_step(0.5, max_norm=1.0)
    want = _norm64(g)
    assert abs(norm.item() - want) <= 1e-10 * want
    f = torch.tensor(0.5 / want, dtype=torch.float64).float().double()
    one = (start.double() - f * g[0].double()).float().double()
    assert ((one - f * g[1].double()) - w.double()).abs().max().item() <= 2.0 ** -22 * (w.abs().max().item() + 1)
    # the same through lists without anything shared: equal up to the two factors' rounding
    kept = g[0].clone()
    norm = mpcnn.GradList([g[0], g[0]]).clip(_norm64([g[0]]) / 2)
    assert abs(norm.item() - math.sqrt(2) * _norm64([kept])) <= 1e-10 * norm.item()
    c = 1 / (2 * math.sqrt(2))
    assert (g[0].double() - kept.double() * c * c).abs().max().item() <= 2.0 ** -22 * kept.abs().max().item()
    kept = g[1].clone()
    a, b = g[1][:n - 10], g[1][n - 20:]
    total = _norm64([a, b])
    mpcnn.GradList([a, b]).clip(total / 4)
    assert (g[1][:n - 20].double() - kept[:n - 20].double() / 4).abs().max().item() <= 2.0 ** -23 * kept.abs().max().item()
    assert (g[1][n - 20:n - 10].double() - kept[n - 20:n - 10].double() / 16).abs().max().item() <= 2.0 ** -23 * kept.abs().max().item()
    assert (g[1][n - 10:].double() - kept[n - 10:].double() / 4).abs().max().item() <= 2.0 ** -23 * kept.abs().max().item()


def test_recorded_into_a_graph():
    g = _tensors([40000, 77], [F, B], 6)
    p = _tensors([40000, 77], [F, B], 7)
    e_p = [t.clone() for t in p]
    norm, e_norm = (torch.zeros(1, dtype=torch.float64, device="cuda") for _ in range(2))
    l, e = mpcnn.GradList(g, p), mpcnn.GradList([t.clone() for t in g], e_p)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        l.sgd_step(0.1, max_norm=1.0, norm=norm)
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        e.sgd_step(0.1, max_norm=1.0, norm=e_norm)
        torch.cuda.synchronize()
        for a, b in zip(p, e_p):
            assert torch.equal(a, b)
        assert norm.item() == e_norm.item()


def test_a_tensor_of_more_than_2_to_the_32_numbers():
    n = (1 << 32) + 5
    g, p = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g[0], g[n - 1] = 3.0, 4.0
    l = mpcnn.GradList([g], [p])
    assert l.norm().item() == 5.0
    l.sgd_step(1.0, max_norm=2.5)
    assert p[0].item() == -1.5 and p[n - 1].item() == -2.0 and int(torch.count_nonzero(p)) == 2
    l.clip(1.25)
    assert g[0].item() == 0.75 and g[n - 1].item() == 1.0 and int(torch.count_nonzero(g)) == 2
    del l, g, p
    torch.cuda.empty_cache()


def test_on_another_stream():
    s = torch.cuda.Stream()
    g = torch.randn(300000, device="cuda")
    l = mpcnn.GradList([g])
    want = l.norm().item()
    torch.cuda.synchronize()
    for stream in (s, s.cuda_stream):
        got = l.norm(stream=stream)
        s.synchronize()
        assert got.item() == want


def test_refusals():
    a = torch.randn(10, device="cuda")
    for grads, params in (([a.half()], None), ([torch.randn(4, 6, device="cuda").t()], None), ([torch.randn(5)], None), ([a], [a.clone()[:5]]),
                          ([a], []), ([a], [a]), ([a, a.clone()], [a.clone(), a])):
        with pytest.raises(mpcnn.MpcnnError) as e:
            mpcnn.GradList(grads, params)
        assert e.value.status == 1
    l = mpcnn.GradList([a])
    for call in (lambda: l.clip(0.0), lambda: l.clip(-1.0), lambda: l.clip(math.nan), lambda: l.norm(grad_scale=math.inf), lambda: l.sgd_step(0.1),
                 lambda: l.norm(norm=torch.zeros(1, device="cuda")), lambda: l.norm(norm=torch.zeros(2, dtype=torch.float64, device="cuda")),
                 lambda: l.norm(norm=torch.zeros(1, dtype=torch.float64))):
        with pytest.raises(mpcnn.MpcnnError) as e:
            call()
        assert e.value.status == 1
    kept = a.clone()
    step = mpcnn.GradList([a], [kept])
    norm = torch.zeros(2, dtype=torch.float64, device="cuda")
    shifted = norm.view(torch.uint8)[4:12]
    for call in (lambda: step.sgd_step(1e30, grad_scale=1e30), lambda: step.sgd_step(1e300, grad_scale=1e300), lambda: step.sgd_step(1e39),
                 lambda: mpcnn._check(mpcnn.lib().mpcnn_grad_norm(l._h, 1.0, shifted.data_ptr(), None))):
        with pytest.raises(mpcnn.MpcnnError) as e:
            call()
        assert e.value.status == 1
    assert torch.equal(kept, a) and (norm == 0).all()
