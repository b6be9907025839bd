"""What a language-model training program of M workers does next to the optimizer step, as timed cases.

Five operators, from the tokens to the gradients that ``DesLoc.step`` reads:

* ``embed``: rows of every worker's fp32 embedding replica, looked up by token and scaled, in the type of the activations;
* ``embed_grad``: its gradient by sorted tokens, written as the dense gradient of that tensor in the step's gradient type;
* ``logprobs``: log probabilities of given tokens from the workers' logits, with the distribution's entropy and its top alternatives;
* ``logprobs_grad``: the gradient of weighted sums of these log probabilities and entropies with respect to the logits;
* ``clip``: every worker's gradient norm over its whole tensor list, and the gradients scaled to a largest norm, in the step's type.

``own`` = False computes them from elementary torch operations in 32 bits, rounded once at the end; True makes the package's calls.
Tokens outside the vocabulary (-1 here) are padding: their embedding is zero, they have no part in any gradient and their log
probability is 0.
"""
import math

import numpy as np
import torch

own = False

MODEL_135M = dict(layers=30, width=576, kv=192, ffn=1536, vocab=49152)    # 134.5 M parameters, 272 tensors
MODEL_MINI = dict(layers=2, width=72, kv=24, ffn=200, vocab=1031)         # 0.2 M parameters, 21 tensors, ragged sizes

BASE = dict(op="", M=4, tokens=1, vocab=0, width=0, layers=0, kv=0, ffn=0, n=0, align=4, src="bf16", dst="bf16", index="i64", scale=1.0,
            pad=0.0, top=0, entropy=False)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
INDEX = {"i32": torch.int32, "i64": torch.int64}
BYTES = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
MAX_NORM = 1.0


def _case(name, **kw):
    return dict(BASE, name=name, **kw)


def listed():
    return [
        # one small tensor, two workers, fp32: latency of a call
        _case("clip_4096_m2", op="clip", M=2, n=4096, src="f32", dst="f32"),
        # a tiny model with ragged tensors in packed buffers
        _case("clip_mini_packed_m4", op="clip", **MODEL_MINI, align=1),
        # the 135 M-parameter model: gradients accumulated in fp32, handed to the step as bf16: the largest
        _case("clip_135m_m4", op="clip", **MODEL_135M, src="f32"),
        # one new token per worker (generation from the replicas)
        _case("embed_decode_m4", op="embed", vocab=49152, width=576),
        # a training batch of the 1.7 B-parameter model's width, four sequences of 2048 per worker, scaled by the width's root
        _case("embed_8192_w2048_m4", op="embed", tokens=8192, vocab=49152, width=2048, scale=math.sqrt(2048)),
        # a tiny model, fp32 gradients, a padded batch
        _case("embed_grad_mini_m4", op="embed_grad", tokens=300, vocab=1031, width=72, src="f32", dst="f32", index="i32", pad=0.2),
        # the 135 M-parameter model's embedding, four sequences of 2048 per worker
        _case("embed_grad_8192_w576_m4", op="embed_grad", tokens=8192, vocab=49152, width=576),
        # the 1.7 B-parameter model's, scaled
        _case("embed_grad_8192_w2048_m4", op="embed_grad", tokens=8192, vocab=49152, width=2048, scale=math.sqrt(2048)),
        # one new token per worker with the alternatives shown beside it
        _case("logprobs_decode_m4", op="logprobs", vocab=49152, top=20, entropy=True),
        # evaluation: 1024 tokens per worker, entropy and the five likeliest tokens
        _case("logprobs_1024_m4", op="logprobs", tokens=1024, vocab=49152, top=5, entropy=True),
        # a tiny model's loss with a bonus for entropy, ragged vocabulary, fp32 logits, a padded batch
        _case("logprobs_grad_mini_m4", op="logprobs_grad", tokens=37, vocab=1031, src="f32", entropy=True, pad=0.1),
        # the loss of a training batch
        _case("logprobs_grad_1024_m4", op="logprobs_grad", tokens=1024, vocab=49152),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["clip", "embed", "embed_grad", "logprobs", "logprobs_grad"])
    c = dict(BASE, op=op, M=rng.choice([1, 2, 3, 4, 5, 8, 16]), src=rng.choice(["f32", "bf16"]), dst=rng.choice(["f32", "bf16"]),
             index=rng.choice(["i32", "i64"]), pad=rng.choice([0.0, 0.0, rng.uniform(0.01, 0.5)]))
    if op == "clip":
        c.update(layers=rng.randint(1, 12), width=8 * rng.randint(8, 96) + rng.choice([0, 0, rng.randint(1, 7)]), align=rng.choice([1, 4]))
        c.update(kv=c["width"] // 3, ffn=2 * c["width"] + rng.randint(0, c["width"]), vocab=_log_uniform(rng, 1000, 50000), pad=0.0)
        while c["M"] * sum(_tensors(c)) > 400_000_000:
            c["layers"], c["vocab"], c["M"] = max(1, c["layers"] // 2), c["vocab"] // 2, max(1, c["M"] // 2)
        return c
    c.update(vocab=_log_uniform(rng, 500, 100000), tokens=_log_uniform(rng, 1, 16384))
    if op in ("embed", "embed_grad"):
        c.update(width=rng.choice([8 * rng.randint(8, 256), rng.randint(64, 1024)]), scale=rng.choice([1.0, round(rng.uniform(0.1, 50.0), 3)]))
        while c["M"] * (c["vocab"] + c["tokens"]) * c["width"] > 300_000_000:
            c["M"], c["tokens"], c["vocab"] = max(1, c["M"] // 2), max(1, c["tokens"] * 3 // 4), max(500, c["vocab"] * 3 // 4)
        return c
    while c["M"] * c["tokens"] * c["vocab"] > 150_000_000:
        c["M"], c["tokens"] = max(1, c["M"] // 2), max(1, c["tokens"] * 2 // 3)
    c.update(entropy=rng.random() < 0.5, top=rng.choice([0, 1, 5, rng.randint(2, 32)]) if op == "logprobs" else 0, dst=c["src"])
    return c


# ---- inputs ------------------------------------------------------------------------------------------
def _tensors(c):
    """Element counts of the tensor list: one tensor of n elements, or a Llama-style list, embedding first."""
    if c["n"]:
        return [c["n"]]
    d, kv, ffn = c["width"], c["kv"], c["ffn"]
    return [c["vocab"] * d] + c["layers"] * [d * d, d * kv, d * kv, d * d, ffn * d, ffn * d, d * ffn, d, d] + [d]


def _offsets(c):
    """Where each tensor begins in a flat buffer per worker, and the buffer's length."""
    at, pos = [], 0
    for n in _tensors(c):
        pos = -(-pos // c["align"]) * c["align"]
        at.append(pos)
        pos += n
    return at, -(-pos // 8) * 8


def _views(c, buf):
    at, _ = _offsets(c)
    return [[row[a:a + n] for a, n in zip(at, _tensors(c))] for row in buf]


def _token_weights(c):
    """Falling like 1 / rank, as words do; the ranks are scattered over the vocabulary."""
    w = 1.0 / (np.arange(c["vocab"]) + 2.7)
    return w / w.sum()


def _draw_tokens(c, gen):
    edges = torch.from_numpy(np.cumsum(_token_weights(c))).cuda()
    u = torch.rand(c["M"], c["tokens"], generator=gen, device="cuda", dtype=torch.float64)
    rank = torch.searchsorted(edges, u).clamp_(max=c["vocab"] - 1)
    tokens = torch.randperm(c["vocab"], generator=gen, device="cuda")[rank]
    padded = int(c["pad"] * c["tokens"])          # the end of every worker's batch
    if padded:
        tokens[:, c["tokens"] - padded:] = -1
    return tokens.to(INDEX[c["index"]])


def _context(c, x, shape):
    """The program's optimizer object for these replicas."""
    import paper_2505_22549_b200 as desloc
    u = torch.zeros_like(x)
    lists = lambda buf: [[row.view(shape)] for row in buf] if shape else _views(c, buf)
    return desloc.DesLoc(lists(x), lists(u), None, opt="sgdm", grad_dtype=c["dst"], K=(16, 64, 256))


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape, dtype=torch.float32: torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)
    s = dict(case=c)
    if c["op"] == "clip":
        total = _offsets(c)[1]
        # norms on both sides of the bound, another for every worker
        size = torch.exp(torch.rand(c["M"], 1, generator=gen, device="cuda") * 3.0 - 1.0) / math.sqrt(total)
        s["grads"] = torch.zeros(c["M"], total, dtype=TYPES[c["src"]], device="cuda")
        for k, (a, n) in enumerate(zip(_offsets(c)[0], _tensors(c))):
            s["grads"][:, a:a + n] = normal(c["M"], n) * size
        s["out"] = torch.zeros(c["M"], total, dtype=TYPES[c["dst"]], device="cuda")
        if own:
            s["opt"] = _context(c, torch.zeros(c["M"], total, device="cuda"), None)
            s["lists"] = _views(c, s["grads"]), _views(c, s["out"])
        return s
    s["tokens"] = _draw_tokens(c, gen)
    if c["op"] in ("embed", "embed_grad"):
        M, V, D = c["M"], c["vocab"], c["width"]
        x = normal(M, V * D) * 0.02 if c["op"] == "embed" else torch.zeros(M, V * D, device="cuda")
        if c["op"] == "embed":
            s["table"] = x
        else:
            s["dout"] = (normal(M, c["tokens"], D) * 1e-3).to(TYPES[c["src"]])
            s["grads"] = torch.zeros(M, V, D, dtype=TYPES[c["dst"]], device="cuda")
        if own:
            s["opt"] = _context(c, x, (V, D))
            s["lists"] = [[g] for g in s["grads"]] if c["op"] == "embed_grad" else None
        return s
    shape = (c["M"], c["tokens"], c["vocab"])
    s["logits"] = (normal(*shape) * 2.0).to(TYPES[c["src"]])
    if c["op"] == "logprobs_grad":
        # what the program has from the forward pass, and the gradients that come back for it
        x = s["logits"].double()
        s["lse"] = torch.logsumexp(x, -1).float()
        s["dlogp"] = -torch.rand(*shape[:2], generator=gen, device="cuda") / (c["M"] * c["tokens"])
        if c["entropy"]:
            logp = x - torch.logsumexp(x, -1, keepdim=True)
            s["entropy"] = -(logp.exp() * logp).sum(-1).float()
            s["dentropy"] = torch.rand(*shape[:2], generator=gen, device="cuda") * 0.01 / (c["M"] * c["tokens"])
        s["out"] = torch.empty_like(s["logits"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)(state["case"], state)


def _own(c, s):
    import paper_2505_22549_b200 as desloc
    if c["op"] == "clip":
        norms, factors = s["opt"].clip_grads(s["lists"][0], MAX_NORM, out=s["lists"][1])
        return s["out"], norms, factors
    if c["op"] == "embed":
        return s["opt"].embed(0, s["tokens"], scale=c["scale"], dtype=c["dst"])
    if c["op"] == "embed_grad":
        s["opt"].embed_grad(0, s["tokens"], s["dout"], s["lists"], scale=c["scale"])
        return s["grads"]
    if c["op"] == "logprobs":
        r = desloc.token_logprobs(s["logits"], s["tokens"], entropy=c["entropy"], top=c["top"])
        return [r.logp, r.lse] + [r.entropy] * c["entropy"] + [r.top_ids, r.top_logp] * (c["top"] > 0)
    return desloc.token_logprobs_grad(s["logits"], s["tokens"], s["lse"], s["dlogp"], entropy=s.get("entropy"), dentropy=s.get("dentropy"),
                                      out=s["out"])


def _in_vocabulary(c, s):
    t = s["tokens"].long()
    valid = (t >= 0) & (t < c["vocab"])
    return valid, torch.where(valid, t, 0)


def _plain(c, s):
    if c["op"] == "clip":
        g = s["grads"].float()
        norms = g.square().sum(1, dtype=torch.float64).sqrt()
        factors = torch.where(norms > MAX_NORM, MAX_NORM / norms, 1.0).float()
        s["out"].copy_(g * factors[:, None])
        return s["out"], norms.float(), factors
    valid, t = _in_vocabulary(c, s)
    workers = torch.arange(c["M"], device=t.device)[:, None]
    if c["op"] == "embed":
        rows = s["table"].view(c["M"], c["vocab"], c["width"])[workers, t] * c["scale"]
        return torch.where(valid[..., None], rows, 0.0).to(TYPES[c["dst"]])
    if c["op"] == "embed_grad":
        total = torch.zeros(c["M"] * c["vocab"] + 1, c["width"], device=t.device)
        row = torch.where(valid, workers * c["vocab"] + t, c["M"] * c["vocab"])       # padding goes to a row of its own
        total.index_add_(0, row.view(-1), s["dout"].view(-1, c["width"]).float())
        s["grads"].copy_((total[:-1] * c["scale"]).view_as(s["grads"]))
        return s["grads"]
    x = s["logits"].float()
    if c["op"] == "logprobs":
        d = x - x.amax(-1, keepdim=True)
        e = d.exp()
        total = e.sum(-1)
        lse = total.log() + x.amax(-1)
        out = [torch.where(valid, x.gather(-1, t[..., None])[..., 0] - lse, 0.0), lse]
        if c["entropy"]:
            out.append(total.log() - (e * d).sum(-1) / total)
        if c["top"]:
            bits = (x + 0.0).view(torch.int32)
            order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()             # whole numbers that rise as the logits do
            places = torch.arange(c["vocab"], device=x.device)
            best = ((order << 32) + (c["vocab"] - 1 - places)).topk(c["top"], -1).values
            ids = c["vocab"] - 1 - (best & 0xffffffff)
            out += [ids, x.gather(-1, ids) - lse[..., None]]
        return out
    logp = x - s["lse"][..., None]
    p = logp.exp()
    hit = torch.arange(c["vocab"], device=x.device) == t[..., None]
    g = torch.where(valid, s["dlogp"], 0.0)[..., None] * (hit.float() - p)
    if c["entropy"]:
        g = g - s["dentropy"][..., None] * p * (logp + s["entropy"][..., None])
    s["out"].copy_(g)
    return s["out"]


# ---- what a pass cannot do without -------------------------------------------------------------------
def work(case):
    c, size = case, lambda key: BYTES[case[key]]
    if c["op"] == "clip":
        n = c["M"] * sum(_tensors(c))
        return {"bytes": n * (size("src") + size("dst")) + 8 * c["M"], "flops": 3.0 * n}
    rows = c["M"] * c["tokens"]
    ids = rows * size("index")
    real = c["tokens"] - int(c["pad"] * c["tokens"])
    if c["op"] == "embed":
        distinct = c["M"] * float(np.sum(-np.expm1(real * np.log1p(-_token_weights(c)))))    # expected rows of the tables that are read
        return {"bytes": ids + c["width"] * (4.0 * distinct + rows * size("dst")), "flops": rows * c["width"]}
    if c["op"] == "embed_grad":
        return {"bytes": ids + c["M"] * c["width"] * (real * size("src") + c["vocab"] * size("dst")), "flops": c["M"] * c["width"] * (real + c["vocab"])}
    if c["op"] == "logprobs":
        return {"bytes": ids + rows * (c["vocab"] * size("src") + 8 + 4 * c["entropy"] + 12 * c["top"]), "flops": rows * c["vocab"] * (4.0 + 2 * c["entropy"])}
    read = rows if c["entropy"] else c["M"] * real
    return {"bytes": ids + size("src") * c["vocab"] * (read + rows) + rows * (8 + 8 * c["entropy"]), "flops": rows * c["vocab"] * (4.0 + 3 * c["entropy"])}


# ---- the definitions in 64 bits ----------------------------------------------------------------------
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "clip":
        out, norms, factors = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), [], []
        for m, g in enumerate(s["grads"]):
            g = g.to(torch.float64)
            norm = float(torch.linalg.vector_norm(g))
            norms.append(norm)
            factors.append(min(1.0, MAX_NORM / norm))
            out[m] = g * factors[-1]
        return out, torch.tensor(norms, dtype=torch.float64), torch.tensor(factors, dtype=torch.float64)
    tokens = s["tokens"].long().cpu().numpy()
    if c["op"] == "embed":
        V, D = c["vocab"], c["width"]
        out = torch.zeros(c["M"], c["tokens"], D, dtype=torch.float64, device="cuda")
        for m in range(c["M"]):
            real = np.flatnonzero((tokens[m] >= 0) & (tokens[m] < V))
            picked = torch.from_numpy(tokens[m][real]).cuda()
            out[m, torch.from_numpy(real).cuda()] = s["table"][m].view(V, D).index_select(0, picked).double() * c["scale"]
        return out
    if c["op"] == "embed_grad":
        V, D = c["vocab"], c["width"]
        out = torch.zeros(c["M"], V, D, dtype=torch.float64, device="cuda")
        for m in range(c["M"]):
            real = np.flatnonzero((tokens[m] >= 0) & (tokens[m] < V))
            order = real[np.argsort(tokens[m][real], kind="stable")]
            if not len(order):
                continue
            distinct, first = np.unique(tokens[m][order], return_index=True)
            run_sums = torch.cumsum(s["dout"][m].double().index_select(0, torch.from_numpy(order).cuda()), 0)
            ends = run_sums[torch.from_numpy(np.append(first[1:], len(order)) - 1).cuda()]
            out[m, torch.from_numpy(distinct).cuda()] = torch.diff(ends, dim=0, prepend=torch.zeros(1, D, dtype=torch.float64, device="cuda")) * c["scale"]
        return out
    results = []
    for m in range(c["M"]):
        logp = torch.log_softmax(s["logits"][m].double(), -1)
        real = torch.from_numpy((tokens[m] >= 0) & (tokens[m] < c["vocab"])).cuda()
        picked = torch.from_numpy(np.clip(tokens[m], 0, c["vocab"] - 1)).cuda()
        entropy = torch.special.entr(logp.exp()).sum(-1)
        if c["op"] == "logprobs":
            one = [logp.gather(1, picked[:, None])[:, 0] * real, torch.logsumexp(s["logits"][m].double(), -1)]
            one += [entropy] if c["entropy"] else []
            if c["top"]:
                best = torch.sort(s["logits"][m].double(), dim=-1, descending=True, stable=True).indices[:, :c["top"]]
                one += [best, logp.gather(1, best)]
            results.append(one)
            continue
        weight = s["dlogp"][m].double() * real
        g = -weight[:, None] * logp.exp()
        g.scatter_add_(1, picked[:, None], weight[:, None])
        if c["entropy"]:
            g -= s["dentropy"][m].double()[:, None] * logp.exp() * (logp + entropy[:, None])
        results.append(g)
    return [torch.stack(r) for r in zip(*results)] if c["op"] == "logprobs" else torch.stack(results)
