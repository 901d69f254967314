"""Operators of large label sets and of the update step, one dict a case: what they compute, in plain torch and by this package.

A class layer over many classes (a vocabulary) with its softmax cross-entropy, on rows of features:

  loss    per-row loss -w log p[label] and the log of the softmax's denominator (scoring rows, line searches)
  train   per-row loss and the gradients of the features, the class weights and the biases

Rows with a label below zero or beyond the last class, or of weight zero, add nothing.

The update behind it, on lists of gradient (and parameter) tensors that are held in one buffer each:

  norm    the 2-norm over all gradients
  clip    gradients of a step come in, and are scaled down where their norm exceeds a bound
  step    parameters move against the gradients, as far as their clipped norm goes

The plain forms compute in 32 bits (norms in 64, long sums) and round once, at the end.
"""
import math

import torch

own = False


def _class(op, rows, features, classes, dtype, weights=False, ignored=0.0):
    return {"op": op, "rows": rows, "features": features, "classes": classes, "dtype": dtype, "weights": weights, "ignored": ignored}


def _list(op, tensors, total, dtype, excess, scale=1.0):
    return {"op": op, "tensors": tensors, "total": total, "dtype": dtype, "excess": excess, "scale": scale}


def listed():
    return [
        # one token scored against a vocabulary: the class weights pass by once
        dict(_class("loss", 1, 1024, 32000, "bf16"), name="loss_1x1024x32000_bf16"),
        # a batch of sequences scored, an odd vocabulary, the padding ignored
        dict(_class("loss", 4096, 1024, 50021, "bf16", ignored=0.1), name="loss_4096x1024x50021_bf16"),
        # a crop's pixels, the steel net's hidden units, a small label set: launches
        dict(_class("train", 213, 100, 37, "f32"), name="train_213x100x37_f32"),
        # a frame's pixels, the deep net's hidden units, balanced by weights
        dict(_class("train", 16384, 200, 1000, "f32", weights=True, ignored=0.1), name="train_16384x200x1000_f32"),
        # a training batch in full precision, ragged everywhere
        dict(_class("train", 4100, 768, 16001, "f32", ignored=0.05), name="train_4100x768x16001_f32"),
        # a few rows: bound by the passes over the class weights and their gradient
        dict(_class("train", 5, 1000, 30011, "bf16", weights=True), name="train_5x1000x30011_bf16"),
        # a training batch of a large model's last layer
        dict(_class("train", 8192, 4096, 128000, "bf16", ignored=0.05), name="train_8192x4096x128000_bf16"),
        # as many tensors and numbers as the deep net has: latency
        dict(_list("norm", 12, 332186, "f32", 0.5), name="norm_12_332k_f32"),
        # a large model's gradients
        dict(_list("norm", 300, 500000000, "mixed", 2.0), name="norm_300_500m_mixed"),
        # a small model's many little tensors (biases, scales), the update in two types
        dict(_list("step", 1000, 3000000, "mixed", 2.0, scale=0.01), name="step_1000_3m_mixed"),
        # a large model's step
        dict(_list("step", 300, 400000000, "f32", 2.0, scale=0.125), name="step_300_400m_f32"),
        # gradients in half the bytes scaled in place, as they come from a backward pass
        dict(_list("clip", 150, 80000000, "bf16", 4.0), name="clip_150_80m_bf16"),
    ]


def _between(rng, least, most):
    return int(round(math.exp(rng.uniform(math.log(least), math.log(most)))))


def draw(rng):
    op = rng.choice(["loss", "loss", "train", "train", "train", "norm", "clip", "step"])
    if op in ("loss", "train"):
        dtype = rng.choice(["f32", "bf16", "bf16"])
        while True:
            rows, features, classes = _between(rng, 1, 16384), _between(rng, 16, 4096), _between(rng, 2, 128000)
            if rng.random() < 0.5:      # widths of real layers are round more often than not
                features = max(16, features // 16 * 16)
            if rows * features * classes <= (1.5e12 if dtype == "bf16" else 3.0e11) and rows * classes <= 8.0e8:
                return _class(op, rows, features, classes, dtype, rng.random() < 0.4, rng.choice([0.0, 0.0, 0.05, 0.5]))
    dtype = rng.choice(["f32", "f32", "bf16", "mixed"])
    tensors = _between(rng, 1, 1000)
    total = max(tensors, _between(rng, 100, 3.0e8))
    return _list(op, tensors, total, dtype, rng.choice([0.5, 1.5, 20.0]), rng.choice([1.0, 0.125, 0.01]))


# ---- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _class_inputs(case, seed):
    gen = _generator(seed)
    n, d, v = case["rows"], case["features"], case["classes"]
    kind = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    w = torch.randn((v, d), generator=gen, device="cuda") * (1.5 / math.sqrt(d))
    labels = torch.randint(0, v, (n,), generator=gen, device="cuda")
    # rows lean towards their label's weights, as in a net that has learned something
    x = torch.randn((n, d), generator=gen, device="cuda") + w[labels] * torch.rand((n, 1), generator=gen, device="cuda") * 2.0
    x, w = x.to(kind), w.to(kind)
    bias = torch.randn((v,), generator=gen, device="cuda") * 0.5
    skip = torch.rand((n,), generator=gen, device="cuda") < case["ignored"]
    labels = torch.where(skip, torch.full_like(labels, -1), labels).to(torch.int32)
    roww = torch.rand((n,), generator=gen, device="cuda") * 2.0 / n if case["weights"] else None
    return x, w, bias, labels, roww


def _sizes(case):
    """Sizes of a list's tensors: spread over two powers of ten, none a round number."""
    n, total = case["tensors"], case["total"]
    gen = torch.Generator().manual_seed(n + total)
    share = torch.exp(torch.rand((n,), generator=gen, dtype=torch.float64) * 4.6)
    sizes = torch.clamp((share / share.sum() * total).to(torch.int64), min=1)
    sizes[sizes.argmax()] += total - int(sizes.sum())
    return sizes.tolist()


def _types(case):
    """Each tensor's type: mixed lists alternate in runs, as layers with scales and biases in 32 bits do."""
    if case["dtype"] != "mixed":
        return [torch.float32 if case["dtype"] == "f32" else torch.bfloat16] * case["tensors"]
    return [torch.float32 if i % 3 == 0 else torch.bfloat16 for i in range(case["tensors"])]


def _flat(case, gen, spread):
    """Per type one buffer, and the tensors as views of them, in the list's order."""
    sizes, types = _sizes(case), _types(case)
    flat = {t: torch.randn((sum(s for s, u in zip(sizes, types) if u == t),), generator=gen, device="cuda").mul_(spread).to(t)
            for t in (torch.float32, torch.bfloat16) if t in types}
    return flat, _views(flat, sizes, types)


def _views(flat, sizes, types):
    at, views = {t: 0 for t in flat}, []
    for s, t in zip(sizes, types):
        views.append(flat[t][at[t]:at[t] + s])
        at[t] += s
    return views


def prepare(case, seed):
    if case["op"] in ("loss", "train"):
        x, w, bias, labels, roww = _class_inputs(case, seed)
        return {"case": case, "x": x, "w": w, "bias": bias, "labels": labels, "roww": roww}
    gen = _generator(seed)
    fresh, grads = _flat(case, gen, 1e-2)
    state = {"case": case, "grads": grads, "params": None, "rate": 0.05}
    # the gradients' norm is about 1e-2 sqrt(total): the bound is that much smaller (or larger) than the scaled norm
    state["bound"] = 1e-2 * math.sqrt(case["total"]) * case["scale"] / case["excess"]
    if case["op"] == "clip":
        buffers = {t: torch.empty_like(f) for t, f in fresh.items()}
        state["fresh"], state["buffers"] = fresh, buffers
        state["grads"] = _views(buffers, _sizes(case), _types(case))
    if case["op"] == "step":
        state["flat"], state["params"] = _flat(case, gen, 0.1)
    if own:
        from paper_1302_1690_amd import mpcnn
        state["list"] = mpcnn.GradList(state["grads"], state["params"])
    return state


# ---- one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return _own(state, op)
    if op in ("loss", "train"):
        return _plain_class(state, op)
    return _plain_list(state, op)


def _own(state, op):
    from paper_1302_1690_amd import mpcnn
    if op == "loss":
        _, rowloss, lse = mpcnn.class_loss(state["x"], state["w"], state["labels"], bias=state["bias"], roww=state["roww"])
        return [rowloss, lse]
    if op == "train":
        _, rowloss, dx, dw, db = mpcnn.class_backward(state["x"], state["w"], state["labels"], bias=state["bias"], roww=state["roww"])
        return [rowloss, dx, dw, db]
    scale = state["case"]["scale"]
    if op == "norm":
        return [state["list"].norm(grad_scale=scale)]
    if op == "clip":
        _refill(state)
        return [state["list"].clip(state["bound"]), *state["buffers"].values()]
    return [state["list"].sgd_step(state["rate"], grad_scale=scale, max_norm=state["bound"]), *state["flat"].values()]


def _refill(state):
    """The next step's gradients arrive in the list's buffers."""
    [b.copy_(f) for b, f in zip(state["buffers"].values(), state["fresh"].values())]


def _plain_class(state, op):
    x, w, labels = state["x"].float(), state["w"].float(), state["labels"].long()
    v = w.shape[0]
    roww = torch.ones_like(labels, dtype=torch.float32) if state["roww"] is None else state["roww"]
    live = (labels >= 0) & (labels < v) & (roww != 0)
    roww = torch.where(live, roww, torch.zeros_like(roww))
    at = torch.where(live, labels, torch.zeros_like(labels)).unsqueeze(1)
    logits = x @ w.t() + state["bias"]
    top = logits.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(logits - top).sum(1, keepdim=True))
    rowloss = roww * (lse - logits.gather(1, at)).squeeze(1)
    if op == "loss":
        return [torch.where(live, rowloss, torch.zeros_like(rowloss)), torch.where(live, lse.squeeze(1), torch.zeros_like(rowloss))]
    g = torch.exp(logits - lse)
    g.scatter_add_(1, at, torch.full_like(lse, -1.0))
    g *= roww.unsqueeze(1)
    return [torch.where(live, rowloss, torch.zeros_like(rowloss)), (g @ w).to(state["x"].dtype), (g.t() @ x).to(state["w"].dtype), g.sum(0)]


def _plain_list(state, op):
    if op == "clip":
        _refill(state)
    scale = 1.0 if op == "clip" else state["case"]["scale"]
    norm = scale * torch.stack([g.double().square().sum() for g in state["grads"]]).sum().sqrt()
    if op == "norm":
        return [norm.reshape(1)]
    factor = torch.clamp(state["bound"] / norm, max=1.0).float()
    if op == "clip":
        [g.copy_(g.float() * factor) for g in state["grads"]]
        return [norm.reshape(1), *state["buffers"].values()]
    factor = factor * (state["rate"] * scale)
    [p.copy_(p.float() - factor * g.float()) for p, g in zip(state["params"], state["grads"])]
    return [norm.reshape(1), *state["flat"].values()]


# ---- what a pass cannot do without

def work(case):
    size = {"f32": 4.0, "bf16": 2.0, "mixed": 8.0 / 3.0}[case["dtype"]]
    if case["op"] in ("loss", "train"):
        n, d, v = case["rows"], case["features"], case["classes"]
        read = size * (n * d + v * d) + 4.0 * v + (8.0 if case["weights"] else 4.0) * n
        if case["op"] == "loss":
            return {"bytes": read + 8.0 * n, "flops": 2.0 * n * d * v}
        return {"bytes": read + size * (n * d + v * d) + 4.0 * (v + n), "flops": 6.0 * n * d * v}
    passes = {"norm": 1.0, "clip": 2.0, "step": 3.0}[case["op"]]
    return {"bytes": passes * size * case["total"], "flops": passes * 2.0 * case["total"]}


# ---- the same in 64 bits, from the definitions

def exact(case, seed):
    if case["op"] in ("loss", "train"):
        return _exact_class(case, seed)
    gen = _generator(seed)
    fresh, grads = _flat(case, gen, 1e-2)
    bound = 1e-2 * math.sqrt(case["total"]) * case["scale"] / case["excess"]
    squares = sum(float(torch.dot(g.double(), g.double())) for g in grads)
    norm = math.sqrt(squares) * (1.0 if case["op"] == "clip" else case["scale"])
    said = torch.tensor([norm], dtype=torch.float64)
    if case["op"] == "norm":
        return [said]
    factor = bound / norm if norm > bound else 1.0
    if case["op"] == "clip":
        return [said] + [f.double() * factor for f in fresh.values()]
    flat, _ = _flat(case, gen, 0.1)
    return [said] + [flat[t].double() - 0.05 * case["scale"] * factor * fresh[t].double() for t in fresh]


def _exact_class(case, seed):
    x, w, bias, labels, roww = _class_inputs(case, seed)
    n, d, v = case["rows"], case["features"], case["classes"]
    w64, b64 = w.double(), bias.double()
    rowloss, lse = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    dx, dw, db = torch.zeros((n, d), dtype=torch.float64, device="cuda"), torch.zeros_like(w64), torch.zeros_like(b64)
    live = torch.nonzero(labels >= 0).squeeze(1)
    if roww is None:
        roww = torch.ones(n, device="cuda")
    for rows in torch.split(live, 2048):
        xs, t, ws = x[rows].double(), labels[rows].long(), roww[rows].double()
        logp = torch.log_softmax(torch.addmm(b64, xs, w64.t()), dim=1)
        own_logp = logp[torch.arange(len(rows), device="cuda"), t]
        rowloss[rows] = -ws * own_logp
        lse[rows] = (xs * w64[t]).sum(1) + b64[t] - own_logp
        if case["op"] == "train":
            delta = logp.exp_()
            delta[torch.arange(len(rows), device="cuda"), t] -= 1.0
            delta *= ws[:, None]
            dx[rows] = torch.mm(delta, w64)
            dw += torch.mm(delta.t(), xs)
            db += delta.sum(0)
    return [rowloss, lse] if case["op"] == "loss" else [rowloss, dx, dw, db]
