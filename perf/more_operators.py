"""The matrix products of a language-model training program of M workers next to the optimizer step, as timed cases.

Four operators on the workers' matrices:

* ``ffn``: the gated feed-forward block down(silu(gate h) * (up h)) of every worker with its own weights;
* ``ffn_grad``: its backward pass, to the block's input and to the three weights' gradients as ``DesLoc.step`` reads them;
* ``orth``: every worker's momentum of a list of matrices, orthogonalised by Newton-Schulz products;
* ``orth_step``: the same as a step of the replicas: momentum in, weights (decayed) moved along its orthogonalised look-ahead.

``own`` = False computes them from elementary torch operations in 32 bits, rounded once at the end; True makes the package's calls.
"""
import math

import torch

own = False

# width, key and value width, feed-forward width of the workloads of the step
MINI = dict(width=72, kv=24, ffn=200)            # 0.2 M parameters, ragged
D576 = dict(width=576, kv=192, ffn=1536)         # 135 M parameters, 30 layers
D960 = dict(width=960, kv=320, ffn=2560)         # 360 M, 32 layers
D2048 = dict(width=2048, kv=2048, ffn=8192)      # 1.7 B, 24 layers

BASE = dict(op="", M=4, tokens=1, width=0, kv=0, ffn=0, layers=1, attention=True, src="f32", dst="bf16", ahead=False, keep=False, accumulate=False)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
STEPS = ((3.4445, -4.7750, 2.0315),) * 5         # the polynomials of the five products
BETA, EPS, LR, DECAY = 0.95, 1e-7, 2e-4, 0.1     # (the rate: late in a schedule)


def _case(name, **kw):
    return dict(BASE, name=name, **kw)


def listed():
    return [
        # one new token per worker (generation from the replicas): all weights read for four rows
        _case("ffn_decode_w2048_m4", op="ffn", **D2048),
        # a tiny model's forward pass, odd numbers of tokens
        _case("ffn_mini_m4", op="ffn", tokens=37, keep=True, **MINI),
        # a training batch of the 1.7 B-parameter model: one sequence of 2048 per worker; keeps what the way back needs
        _case("ffn_2048_w2048_m4", op="ffn", tokens=2048, keep=True, **D2048),
        # a tiny model's way back
        _case("ffn_grad_mini_m4", op="ffn_grad", tokens=37, **MINI),
        # the 135 M-parameter model's, four sequences of 2048 per worker
        _case("ffn_grad_8192_w576_m4", op="ffn_grad", tokens=8192, **D576),
        # the 1.7 B-parameter model's, onto the gradients of an earlier part of the batch
        _case("ffn_grad_2048_w2048_m4", op="ffn_grad", tokens=2048, accumulate=True, **D2048),
        # one projection of a tiny model, two workers: latency of a call
        _case("orth_72_m2", op="orth", M=2, width=72, kv=0, ffn=0),
        # a layer's matrices of the 360 M-parameter model, bf16 updates
        _case("orth_layer_w960_m8", op="orth", M=8, src="bf16", **D960),
        # the feed-forward matrices of a layer of the 1.7 B-parameter model
        _case("orth_ffn_w2048_m4", op="orth", attention=False, **D2048),
        # all matrices of a tiny model as a step
        _case("orth_step_mini_m4", op="orth_step", layers=2, ahead=True, **MINI),
        # all matrices of the 135 M-parameter model as a step, with the look-ahead of their bf16 gradients: 840 matrices
        _case("orth_step_135m_m4", op="orth_step", layers=30, ahead=True, **D576),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    c = dict(BASE, op=rng.choice(["ffn", "ffn_grad", "orth", "orth_step"]), M=rng.choice([1, 2, 3, 4, 5, 8]))
    wide = rng.random() < 0.6                                   # multiples of eight, as most models have, or any width
    size = lambda lo, hi: 8 * _log_uniform(rng, lo / 8, hi / 8) if wide else _log_uniform(rng, lo, hi)
    c.update(width=size(24, 2048))
    c.update(ffn=max(1, int(c["width"] * rng.uniform(1.5, 4.0)) // (8 if wide else 1) * (8 if wide else 1)))
    if c["op"] in ("ffn", "ffn_grad"):
        c.update(tokens=_log_uniform(rng, 1, 8192), keep=rng.random() < 0.5, accumulate=c["op"] == "ffn_grad" and rng.random() < 0.5)
        while c["M"] * c["tokens"] * c["width"] * c["ffn"] > 70_000_000_000:
            c["M"], c["tokens"] = max(1, c["M"] // 2), max(1, c["tokens"] * 2 // 3)
        return c
    c.update(kv=max(1, c["width"] // rng.choice([1, 2, 3, 4])), layers=rng.choice([1, 1, 2, 4]), attention=rng.random() < 0.7, src=rng.choice(["f32", "bf16"]))
    c.update(ahead=rng.random() < 0.5)
    if c["op"] == "orth_step":
        c.update(src="f32")
    while work(c)["flops"] > 4e12:
        c["M"], c["layers"] = max(1, c["M"] // 2), max(1, c["layers"] // 2)
        if c["M"] * c["layers"] == 1:
            c["width"], c["kv"], c["ffn"] = c["width"] // 2, max(1, c["kv"] // 2), c["ffn"] // 2
    return c


# ---- inputs ------------------------------------------------------------------------------------------
def _groups(c):
    """(count, rows, columns) of the matrices of a worker, those of one shape together."""
    d, kv, ffn, n = c["width"], c["kv"], c["ffn"], c["layers"]
    attention = [(2 * n, d, d), (2 * n, kv, d)] if kv else [(n, d, d)]
    return (attention if c["attention"] else []) + ([(2 * n, ffn, d), (n, d, ffn)] if ffn else [])


def _lists(groups):
    """Nested lists, a worker's matrices in the order of the groups."""
    return [[matrix for g in groups for matrix in g[m]] for m in range(len(groups[0]))]


def prepare(case, seed):
    c, M = case, case["M"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    s = dict(case=c)
    if c["op"] in ("ffn", "ffn_grad"):
        T, D, F = c["tokens"], c["width"], c["ffn"]
        s["h"] = normal(M, T, D).bfloat16()                                        # behind a norm
        s["weights"] = [(normal(M, *shape) * shape[1] ** -0.5).bfloat16() for shape in ((F, D), (F, D), (D, F))]
        if c["op"] == "ffn_grad":
            s["kept"] = normal(M, T, F).bfloat16(), normal(M, T, F).bfloat16()     # gate h and up h of the forward pass
            s["dy"] = (normal(M, T, D) * 1e-3).bfloat16()
            s["start"] = [(normal(M, *w.shape[1:]) * 1e-3).bfloat16() if c["accumulate"] else torch.zeros_like(w) for w in s["weights"]]
            s["grads"] = [w.clone() for w in s["start"]]
        if own:
            import paper_2505_22549_b200 as desloc
            x = [torch.zeros(w.shape, device="cuda") for w in s["weights"]]
            s["opt"] = desloc.DesLoc(_rows(x), _rows([torch.zeros_like(w) for w in x]), None, opt="sgdm", grad_dtype="bf16", K=(16, 64, 256))
            s["weight_lists"], s["grad_lists"] = _rows(s["weights"]), _rows(s.get("grads", []))
        return s
    s["u"], s["grads"], s["x"], s["out"] = [], [], [], []
    for count, rows, cols in _groups(c):
        # a few directions that many batches share, and noise
        shared = normal(M, count, rows, 4) @ normal(M, count, 4, cols)
        s["u"].append((1e-4 * (normal(M, count, rows, cols) + 0.5 * shared)).to(TYPES[c["src"]]))
        s["grads"].append((1e-3 * normal(M, count, rows, cols)).bfloat16() if c["ahead"] else None)
        if c["op"] == "orth_step":
            s["x"].append(0.02 * normal(M, count, rows, cols))
        else:
            s["out"].append(torch.zeros(M, count, rows, cols, dtype=TYPES[c["dst"]], device="cuda"))
    if own:
        import paper_2505_22549_b200 as desloc
        x = s["x"] or [torch.zeros(u.shape, device="cuda") for u in s["u"]]
        u = s["u"] if c["op"] == "orth_step" else [torch.zeros(u.shape, device="cuda") for u in s["u"]]
        s["opt"] = desloc.DesLoc(_lists(x), _lists(u), None, opt="sgdm", beta1=BETA, weight_decay=DECAY, grad_dtype="bf16", K=(16, 64, 256))
        s["tensors"] = list(range(sum(count for count, _, _ in _groups(c))))
        s["lists"] = _lists(s["u"]), _lists(s["grads"]) if c["ahead"] else None, _lists(s["out"]) if s["out"] else None
    return s


def _rows(tensors):
    """Nested lists of the block's three weights, a list per worker."""
    return [list(worker) for worker in zip(*tensors)]


# ---- one pass ----------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)(state["case"], state)


def _own(c, s):
    if c["op"] == "ffn":
        return s["opt"].gated_ffn((0, 1, 2), s["h"], s["weight_lists"], keep=c["keep"])
    if c["op"] == "ffn_grad":
        dh = s["opt"].gated_ffn_grad((0, 1, 2), s["h"], s["kept"], s["dy"], s["weight_lists"], s["grad_lists"], accumulate=c["accumulate"])
        return [dh] + s["grads"]
    updates, grads, out = s["lists"]
    if c["op"] == "orth":
        s["opt"].orthogonalize(s["tensors"], updates, grads=grads, out=out)
        return s["out"]
    s["opt"].orthogonal_step(s["tensors"], LR, grads=grads, scale="aspect")
    return s["x"]


def _silu(g):
    return g / (1.0 + torch.exp(-g))


def _orthogonal(u, g):
    x = u.float() if g is None else BETA * u.float() + (1.0 - BETA) * g.float()
    x = x / (x.square().sum((-2, -1), keepdim=True, dtype=torch.float64).sqrt().float() + EPS)
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT if tall else x
    for a, b, c in STEPS:
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT if tall else x


def _aspect(x):
    return math.sqrt(max(1.0, x.shape[-2] / x.shape[-1]))


def _plain(c, s):
    if c["op"] == "ffn":
        gate, up, down = (w.float() for w in s["weights"])
        h = s["h"].float()
        g, u = h @ gate.mT, h @ up.mT
        y = ((_silu(g) * u) @ down.mT).bfloat16()
        return (y, (g.bfloat16(), u.bfloat16())) if c["keep"] else y
    if c["op"] == "ffn_grad":
        gate, up, down = (w.float() for w in s["weights"])
        h, dy, g, u = (t.float() for t in (s["h"], s["dy"], *s["kept"]))
        sigmoid = 1.0 / (1.0 + torch.exp(-g))
        dz = dy @ down
        du = dz * g * sigmoid
        dg = dz * u * sigmoid * (1.0 + g * (1.0 - sigmoid))
        sums = dg.mT @ h, du.mT @ h, dy.mT @ (g * sigmoid * u)
        new = [total + w.float() if c["accumulate"] else total for total, w in zip(sums, s["grads"])]
        [w.copy_(total) for w, total in zip(s["grads"], new)]
        return [(dg @ gate + du @ up).bfloat16()] + s["grads"]
    if c["op"] == "orth":
        [to.copy_(_orthogonal(u, g)) for to, u, g in zip(s["out"], s["u"], s["grads"])]
        return s["out"]
    [x.mul_(1.0 - LR * DECAY).sub_(LR * _aspect(x) * _orthogonal(u, g)) for x, u, g in zip(s["x"], s["u"], s["grads"])]
    return s["x"]


# ---- what a pass cannot do without -------------------------------------------------------------------
def work(case):
    c, M = case, case["M"]
    if c["op"] in ("ffn", "ffn_grad"):
        T, D, F = c["tokens"], c["width"], c["ffn"]
        if c["op"] == "ffn":
            return {"bytes": 2 * M * (2 * T * D + 3 * D * F + 2 * T * F * c["keep"]), "flops": 6.0 * M * T * D * F}
        return {"bytes": 2 * M * (3 * T * D + 2 * T * F + 3 * D * F * (2 + c["accumulate"])), "flops": 12.0 * M * T * D * F}
    elements, flops = 0, 0.0
    for count, rows, cols in _groups(c):
        n, m = min(rows, cols), max(rows, cols)
        elements += M * count * n * m
        # of the two products whose results are symmetric, half
        flops += M * count * len(STEPS) * (1.0 * n * n * m + 1.0 * n ** 3 + 2.0 * n * n * m)
    moved = 8 if c["op"] == "orth_step" else BYTES[c["dst"]]
    return {"bytes": elements * (BYTES[c["src"]] + 2 * c["ahead"] + moved), "flops": flops}


# ---- the definitions in 64 bits ----------------------------------------------------------------------
def _exact_orthogonal(u, g):
    """The same polynomials, of the squared singular values alone, times the matrix."""
    x = u.double() if g is None else torch.lerp(g.double(), u.double(), BETA)
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + EPS)
    wide = x if x.shape[-2] <= x.shape[-1] else x.transpose(-2, -1)
    square = torch.matmul(wide, wide.transpose(-2, -1))
    whole = one = torch.eye(square.shape[-1], dtype=torch.float64, device=x.device)
    for a, b, c in STEPS:
        factor = a * one + square @ (b * one + c * square)
        whole, square = factor @ whole, factor @ square @ factor
    return torch.matmul(whole, wide) if wide is x else torch.matmul(whole, wide).transpose(-2, -1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] in ("orth", "orth_step"):
        found = []
        for k, u in enumerate(s["u"]):
            turned = _exact_orthogonal(u, s["grads"][k])
            if c["op"] == "orth_step":
                rows, cols = u.shape[-2:]
                turned = s["x"][k].double() * (1.0 - LR * DECAY) - LR * max(1.0, rows / cols) ** 0.5 * turned
            found.append(turned)
        return found
    results = []
    for m in range(c["M"]):
        gate, up, down = (w[m].double() for w in s["weights"])
        h = s["h"][m].double()
        if c["op"] == "ffn":
            g, u = torch.nn.functional.linear(h, gate), torch.nn.functional.linear(h, up)
            results.append([torch.nn.functional.linear(torch.nn.functional.silu(g) * u, down), g, u])
            continue
        dy = s["dy"][m].double()
        leaves = [t.detach().requires_grad_() for t in (s["kept"][0][m].double(), s["kept"][1][m].double())]
        z = torch.nn.functional.silu(leaves[0]) * leaves[1]
        dg, du = torch.autograd.grad(z, leaves, torch.matmul(dy, down))
        totals = [torch.einsum("tf,td->fd", dg, h), torch.einsum("tf,td->fd", du, h), torch.einsum("td,tf->df", dy, z.detach())]
        if c["accumulate"]:
            totals = [t + w[m].double() for t, w in zip(totals, s["start"])]
        results.append([torch.matmul(dg, gate) + torch.matmul(du, up)] + totals)
    stacked = [torch.stack(r) for r in zip(*results)]
    if c["op"] == "ffn":
        return (stacked[0], (stacked[1], stacked[2])) if c["keep"] else stacked[0]
    return stacked
