"""Operators around the step against their definitions in 64 bits: embedding lookup and gradient, log probabilities and gradient, clipping.

Tolerances count roundings (u = 2^-24 for fp32, half a step of the output's type where it is rounded to fewer bits) and, for 2^t, the
2^-22 of the hardware's exponential; n additions in any order are off by at most n u times the sum of magnitudes.
"""
import math

import pytest
import torch

import paper_2505_22549_b200 as d

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
BF, F32 = torch.bfloat16, torch.float32


def gen_of(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def context(M, shapes, grad_dtype="bf16", seed=0, packed=False):
    """(DesLoc, x): M workers' replicas of tensors of these shapes, N(0, 1), another for every worker; packed = the tensors follow one another."""
    g = gen_of(seed)
    total = sum(math.prod(s) for s in shapes)
    x = []
    for m in range(M):
        flat = torch.randn(total + 64, generator=g, device="cuda")
        row, at = [], 0
        for s in shapes:
            n = math.prod(s)
            row.append(flat[at:at + n].view(s) if packed else torch.randn(s, generator=g, device="cuda"))
            at += n
        x.append(row)
    u = [[torch.zeros_like(t) for t in row] for row in x]
    return d.DesLoc(x, u, None, opt="sgdm", grad_dtype=grad_dtype, K=(2, 3, 4)), x


def tokens_of(M, n, V, seed, index=torch.int64, pad=0):
    g = gen_of(seed)
    # falling like 1 / rank: long runs of the first ones
    t = ((V + 1.0) ** torch.rand(M, n, generator=g, device="cuda", dtype=torch.float64) - 1).long().clamp(max=V - 1)
    if pad:
        t[:, n - pad:] = torch.tensor([-1, -100, V, V + 5, -(2 ** 31)], device="cuda").repeat(pad)[:pad]
    return t.to(index)


def check(got, want, tol):
    """|got - want| <= tol elementwise, infinities and NaN in the same places."""
    assert got.shape == want.shape
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.isinf(got), torch.isinf(want)) and torch.equal(got[torch.isinf(got)], want[torch.isinf(want)])
    fine = torch.isfinite(want)
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, f"off by {float(over.max()):.3e} more than allowed"


# ---- embedding ---------------------------------------------------------------------------------------
def embed_ref(x, k, tokens, scale, width):
    M = tokens.shape[0]
    t = tokens.long().reshape(M, -1)
    out = torch.zeros(M, t.shape[1], width, dtype=torch.float64, device="cuda")
    for m in range(M):
        table = x[m][k].double().reshape(-1, width)
        real = (t[m] >= 0) & (t[m] < table.shape[0])
        out[m, real] = table[t[m][real]] * scale
    return out.view(*tokens.shape, width)


@pytest.mark.parametrize("M,V,D,n,dtype,index,pad,packed", [
    (1, 1, 1, 1, "f32", torch.int64, 0, False), (2, 5, 3, 7, "bf16", torch.int32, 2, False), (4, 1031, 72, 1, "bf16", torch.int64, 0, False),
    (4, 1031, 72, 300, "f32", torch.int32, 60, True), (3, 769, 577, 129, "bf16", torch.int64, 5, True), (2, 500, 2048, 1500, "bf16", torch.int64, 3, False),
    (16, 300, 132, 333, "f32", torch.int64, 1, False), (2, 64, 4100, 17, "bf16", torch.int32, 0, True), (8, 97, 8, 0, "bf16", torch.int64, 0, False)])
def test_embed(M, V, D, n, dtype, index, pad, packed):
    opt, x = context(M, [(5,), (V, D), (3, 3)], packed=packed)
    tokens = tokens_of(M, n, V, 1, index, pad)
    for scale in (1.0, -2.5):
        out = opt.embed(1, tokens, scale=scale, dtype=dtype)
        want = embed_ref(x, 1, tokens, scale, D)
        assert out.dtype == {"f32": F32, "bf16": BF}[dtype]
        check(out, want, want.abs() * (HALF[out.dtype] * (1 + U) + U) + 1e-40)


def test_embed_layouts():
    """Token grids, strided tokens and outputs, a flat tensor taken as rows; what lies around the output stays as it was."""
    M, V, D = 3, 211, 24
    opt, x = context(M, [(V * D,)])
    grid = tokens_of(M, 4 * 10, V, 2).view(M, 4, 10)
    assert opt.embed(0, grid, width=D).shape == (M, 4, 10, D)
    for tokens in (grid[:, :, 1:], grid[:, ::2], grid.transpose(1, 2), tokens_of(M, 20, V, 3, torch.int32)[:, ::2]):
        check(opt.embed(0, tokens, width=D, dtype="f32"), embed_ref(x, 0, tokens, 1.0, D), 0.0)
    for dtype, cut in ((F32, slice(4, 4 + D)), (BF, slice(1, 1 + D)), (BF, slice(4, 4 + D))):
        buf = torch.full((M, 12, D + 9), 7.0, dtype=dtype, device="cuda")
        tokens = tokens_of(M, 10, V, 4)
        opt.embed(0, tokens, width=D, out=buf[:, 1:11, cut])
        want = torch.full(buf.shape, 7.0, dtype=torch.float64, device="cuda")
        want[:, 1:11, cut] = embed_ref(x, 0, tokens, 1.0, D)
        check(buf, want, want.abs() * HALF[dtype])
    buf = torch.full((10, M, D), 7.0, device="cuda")        # worker-minor
    opt.embed(0, tokens, width=D, out=buf.transpose(0, 1))
    check(buf.transpose(0, 1), embed_ref(x, 0, tokens, 1.0, D), 0.0)


def embed_grad_ref(tokens, dout, V, scale, out_dtype, old=None):
    """(sum, tolerance)"""
    M, D = tokens.shape[0], dout.shape[-1]
    t, g = tokens.long().reshape(M, -1), dout.double().reshape(M, -1, D)
    total = torch.zeros(M, V, D, dtype=torch.float64, device="cuda")
    size, count = torch.zeros_like(total), torch.zeros(M, V, 1, dtype=torch.float64, device="cuda")
    for m in range(M):
        real = (t[m] >= 0) & (t[m] < V)
        total[m].index_add_(0, t[m][real], g[m][real])
        size[m].index_add_(0, t[m][real], g[m][real].abs())
        count[m].index_add_(0, t[m][real], torch.ones(int(real.sum()), 1, dtype=torch.float64, device="cuda"))
    want = total * scale + (0 if old is None else old.double())
    tol = size * abs(scale) * (count + 2) * U * 1.01 + want.abs() * (HALF[out_dtype] * 1.01 + U) + 1e-40
    return want, torch.where(count > 0, tol, 0.0)


@pytest.mark.parametrize("M,V,D,n,src,dst,index,pad", [
    (1, 1, 1, 1, F32, F32, torch.int64, 0), (2, 5, 3, 7, BF, BF, torch.int32, 2), (4, 1031, 72, 300, F32, F32, torch.int32, 60),
    (4, 768, 64, 63, BF, BF, torch.int64, 0), (3, 769, 577, 129, BF, F32, torch.int64, 5), (2, 500, 256, 5000, F32, BF, torch.int64, 3),
    (16, 300, 132, 333, BF, BF, torch.int64, 1), (2, 64, 4100, 200, BF, BF, torch.int32, 0), (2, 2000, 40, 20000, BF, BF, torch.int64, 100),
    (1, 20011, 16, 4097, F32, F32, torch.int32, 7), (5, 97, 8, 0, BF, BF, torch.int64, 0), (1, 3, 520, 30000, BF, F32, torch.int64, 0),
    (256, 33, 8, 70, BF, BF, torch.int64, 4)])
def test_embed_grad(M, V, D, n, src, dst, index, pad):
    opt, _ = context(M, [(5,), (V, D)], grad_dtype="bf16" if dst == BF else "f32")
    tokens = tokens_of(M, n, V, 1, index, pad)
    dout = torch.randn(M, n, D, generator=gen_of(2), device="cuda").to(src)
    if pad:
        dout[:, n - pad:] = float("nan")        # what stands in padded places has no part in anything
    guard = torch.full((M, V * D + 32), 5.0, dtype=dst, device="cuda")
    grads = [[None, row[16:16 + V * D].view(V, D)] for row in guard]
    for scale in (1.0, 3.25):
        guard.fill_(5.0)
        opt.embed_grad(1, tokens, dout, grads, scale=scale)
        got = guard[:, 16:16 + V * D].view(M, V, D)
        want, tol = embed_grad_ref(tokens, dout, V, scale, dst)
        check(got, want, tol)
        assert bool((guard[:, :16] == 5).all()) and bool((guard[:, 16 + V * D:] == 5).all())
    first = got.clone()
    opt.embed_grad(1, tokens, dout, grads, scale=scale)
    assert torch.equal(first, got)                      # the same bits
    old = torch.randn(M, V, D, generator=gen_of(3), device="cuda").to(dst)
    got.copy_(old)
    opt.embed_grad(1, tokens, dout, grads, scale=scale, accumulate=True)
    want, tol = embed_grad_ref(tokens, dout, V, scale, dst, old)
    check(got, want, tol)                               # (no tolerance where there is no token: as it was)


@pytest.mark.parametrize("D", [8, 33, 512])
@pytest.mark.parametrize("n", [63, 64, 65, 127, 128, 129, 8191, 16385])
def test_embed_grad_of_one_token_and_of_two(n, D):
    """Runs that are cut into pieces: all positions the same token; a long run in front of another."""
    opt, _ = context(2, [(70, D)])
    tokens = torch.full((2, n), 69, dtype=torch.int64, device="cuda")
    tokens[1, : n // 3] = 5
    dout = torch.randn(2, n, D, generator=gen_of(5), device="cuda").to(BF)
    grads = [[torch.empty(70, D, dtype=BF, device="cuda")] for _ in range(2)]
    opt.embed_grad(0, tokens, dout, grads)
    want, tol = embed_grad_ref(tokens, dout, 70, 1.0, BF)
    check(torch.stack([g[0] for g in grads]), want, tol)


def test_embed_grad_layouts():
    M, V, D = 3, 211, 24
    opt, _ = context(M, [(7,), (V * D,)], packed=True)
    grads = [[torch.zeros(7, dtype=BF, device="cuda"), torch.empty(V * D, dtype=BF, device="cuda")] for _ in range(M)]
    grid = tokens_of(M, 40, V, 2).view(M, 4, 10)
    big = torch.randn(M, 4, 10, D + 8, generator=gen_of(3), device="cuda")
    for tokens, dout in ((grid, big[..., :D]), (grid, big[..., 3:3 + D]), (grid[:, :, 1:], big[:, :, 1:, 8:]), (grid[:, ::2], big[:, ::2, :, 4:4 + D].to(BF)),
                         (grid, big.transpose(-1, -2)[..., :D, :].transpose(-1, -2)),
                         (grid, big[:1, :, :, :D].expand(M, 4, 10, D))):
        for given in (grads, opt.bind_grads(grads)):
            opt.embed_grad(1, tokens, dout, given, width=D)
            want, tol = embed_grad_ref(tokens, dout, V, 1.0, BF)
            check(torch.stack([g[1] for g in grads]).view(M, V, D), want, tol)
    one = dout.new_ones(M, 4, 10, 1).expand(M, 4, 10, D)        # a broadcast gradient: columns of stride 0
    opt.embed_grad(1, grid, one, grads, width=D)
    want, tol = embed_grad_ref(grid, one, V, 1.0, BF)
    check(torch.stack([g[1] for g in grads]).view(M, V, D), want, tol)


def test_embed_grad_is_the_difference_quotient():
    """sum(w * embed(x + h v)) - sum(w * embed(x - h v)) over 2 h against <gradient, v>, in numbers that fp32 holds exactly."""
    M, V, D, n = 2, 50, 12, 90
    opt, x = context(M, [(V, D)], grad_dtype="f32")
    g = gen_of(9)
    small = lambda *s: torch.randint(-8, 9, s, generator=g, device="cuda").float()
    for row in x:
        row[0].copy_(small(V, D))
    tokens, w, v = tokens_of(M, n, V, 4, pad=5), small(M, n, D), small(M, V, D)
    value = lambda: float((opt.embed(0, tokens, scale=0.5, dtype="f32").double() * w).sum())
    for m in range(M):
        x[m][0].add_(v[m])
    up = value()
    for m in range(M):
        x[m][0].sub_(2 * v[m])
    down = value()
    grads = [[torch.empty(V, D, device="cuda")] for _ in range(M)]
    opt.embed_grad(0, tokens, w, grads, scale=0.5)
    assert (up - down) / 2 == sum(float((grads[m][0].double() * v[m]).sum()) for m in range(M))


# ---- log probabilities -------------------------------------------------------------------------------
def log_softmax_ref(x):
    """(log p, lse, which rows are nothing but -inf): differences to the largest logit first, which 64 bits hold where the logits are huge."""
    x = x.double()
    m = x.amax(-1, keepdim=True)
    empty = torch.isneginf(m)
    lp = x - torch.where(empty, 0.0, m)
    log_sum = lp.exp().sum(-1, keepdim=True).log()
    lp = torch.where(empty, -math.inf, lp - log_sum)
    return lp, torch.where(empty, -math.inf, m + log_sum)[..., 0], empty[..., 0]


def logprob_ref(x, t):
    lp, lse, empty = log_softmax_ref(x)
    real = (t >= 0) & (t < x.shape[-1])
    logp = lp.gather(-1, torch.where(real, t, 0).long()[..., None])[..., 0]
    H = -torch.where(torch.isneginf(lp), 0.0, lp.exp() * lp).sum(-1)
    return torch.where(real, logp, 0.0), lse, torch.where(empty, 0.0, H)


def top_ref(x, k):
    x = torch.where(torch.isnan(x), -math.inf, x.float())
    kk = min(k, x.shape[-1])
    ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[..., :kk]
    v = x.gather(-1, ids)
    ids = torch.where(torch.isneginf(v), -1, ids)
    return torch.nn.functional.pad(ids, (0, k - kk), value=-1)


def logprob_tol(x):
    """Bound on the error of log S, and of the entropy.  A term 2^t: t has two roundings and the multiplication by log2 e, the exponential
    2^-22, and it is added to at most V / 128 others in a thread and 60 more on the way through lanes, warps and blocks, rescaled as often."""
    xd = x.double()
    m = xd.nan_to_num(nan=0.0, neginf=-1e38).amax(-1, keepdim=True)
    dist = (m - xd).clamp(0, 200).nan_to_num(0.0)                        # (further below, a term is 0 either way)
    p = torch.softmax(xd.nan_to_num(nan=-1e38, neginf=-1e38, posinf=1e38), -1)
    V = x.shape[-1]
    far = (p * dist).sum(-1)
    rel = 2.0 ** -22 + 3 * U * far + 2 * (V / 128 + 70) * U
    return rel, rel * (2 + 3 * far) + 3 * U * (p * dist * dist).sum(-1)


def check_logprobs(x, t, top=0):
    r = d.token_logprobs(x, t, entropy=True, top=top)
    logp, lse, H = logprob_ref(x, t)
    rel, tol_H = logprob_tol(x)
    base = lse.abs().nan_to_num(0.0, posinf=0.0, neginf=0.0)
    biggest = x.double().nan_to_num(0.0, posinf=0.0, neginf=0.0).abs().amax(-1)
    log_sum = math.log(x.shape[-1]) + 1
    check(r.lse, lse, rel + U * (base + biggest + 2 * log_sum))
    # (differences of logits, not the logits, are rounded on the way to logp)
    check(r.logp, logp, rel + 4 * U * (logp.abs().nan_to_num(0.0, neginf=0.0) + log_sum))
    check(r.entropy, H, tol_H + 4 * U * log_sum)
    plain = d.token_logprobs(x, t)
    assert plain.entropy is None and plain.top_ids is None and plain.top_logp is None
    check(plain.lse, lse, rel + U * (base + biggest + 2 * log_sum))
    if top:
        ids = top_ref(x, top)
        assert torch.equal(r.top_ids, ids)
        want = torch.where(ids >= 0, log_softmax_ref(x)[0].gather(-1, ids.clamp(min=0)), -math.inf)
        check(r.top_logp, want, rel[..., None] + 4 * U * (want.abs().nan_to_num(0.0, neginf=0.0) + log_sum))
        again = d.token_logprobs(x, t, entropy=True, top=top)
        for a, b in zip(r, again):
            assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
    return r


LENGTHS = [1, 2, 7, 8, 9, 31, 33, 100, 500, 1031, 4100, 8191, 8192, 16383, 16384, 16389, 49152]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", LENGTHS)
def test_logprobs(V, dtype):
    for rows, top in ((1, 20), (3, 1), (50, 32), (25, 16), (25, 17)):
        g = gen_of(V + rows)
        x = (torch.randn(2, rows, V, generator=g, device="cuda") * 3).to(dtype)
        t = torch.randint(-1, V + 1, (2, rows), generator=g, device="cuda")
        check_logprobs(x, t, top)


def _masked(x, kind):
    x = x.clone()
    lowest = torch.finfo(x.dtype).min
    if kind == "one left":
        x[..., 1:] = -math.inf
    elif kind == "none left":
        x[:, ::2] = -math.inf
    elif kind == "half":
        x[..., ::2] = -math.inf
    elif kind == "lowest":
        x[..., 3:] = lowest
    elif kind == "all lowest":
        x[:] = lowest
    elif kind == "nan":
        x[:, 0, x.shape[-1] // 2] = math.nan
        x[:, 1, -1] = math.inf
    elif kind == "constant":
        x[:] = 1.5
    elif kind == "steps":
        x = (x * 0.3).round()
    elif kind == "large":
        x = x * 1e30
    elif kind == "rising":
        x[:] = torch.arange(x.shape[-1], device="cuda").to(x.dtype) * 0.01
    return x


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [5, 1031, 9001, 49152])
@pytest.mark.parametrize("kind", ["one left", "none left", "half", "lowest", "all lowest", "nan", "constant", "steps", "large", "rising"])
def test_logprobs_of_masked_and_tied_rows(kind, V, dtype):
    for rows in (3, 25):
        g = gen_of(V)
        x = _masked((torch.randn(2, rows, V, generator=g, device="cuda") * 3).to(dtype), kind)
        t = torch.randint(0, V, (2, rows), generator=g, device="cuda", dtype=torch.int32)
        check_logprobs(x, t.long() if rows == 3 else t, 7)


def test_logprobs_when_most_values_of_a_thread_are_among_the_largest():
    """More values at the line than there is room for, not all equal: the largest of all lie together, in threads' own pieces."""
    V = 49152
    x = torch.randn(2, 20, V, generator=gen_of(1), device="cuda")
    for k in range(32):
        x[:, :, torch.arange(k * 4, V, 512 * 4, device="cuda")[:, None] + torch.arange(4, device="cuda")] += 40.0
    check_logprobs(x, torch.zeros(2, 20, dtype=torch.int64, device="cuda"), 32)
    check_logprobs(x[:1, :2].contiguous(), torch.zeros(1, 2, dtype=torch.int64, device="cuda"), 32)


@pytest.mark.parametrize("offset", [-3e6, -1e6, 3e2, 2e4, 1e6, 3e6, 2e9, 1e30])
def test_logprobs_of_rows_far_from_zero(offset):
    """Offsets that fp32 logits can have, differences from them as large as the type's steps there: in front of, across and behind 1e6."""
    for V, rows in ((1031, 5), (20000, 3), (9000, 30)):
        x = torch.randn(2, rows, V, generator=gen_of(V), device="cuda") * 3 + offset
        if abs(offset) == 1e6:
            x[:, 1] += 10.0
        check_logprobs(x, torch.randint(0, V, (2, rows), generator=gen_of(1), device="cuda"), 5)
        check_grad(x, torch.randint(0, V, (2, rows), generator=gen_of(1), device="cuda"), in_place=rows == 3)


def test_logprobs_layouts():
    g = gen_of(7)
    for dtype, V in ((BF, 1000), (F32, 1001), (BF, 8193)):
        x = torch.randn(4, 9, V + 3, generator=g, device="cuda").to(dtype)
        t = torch.randint(0, V, (4, 9), generator=g, device="cuda")
        for a, b in ((x[:, :-1], t[:, 1:]), (x[..., 1:V + 1], t), (x[:, ::2], t[:, ::2]), (x[1::2, :, 3:], t[1::2]), (x.transpose(0, 1), t.t()),
                     (x[0], t[0]), (x[0, 0], t[0, 0]), (x[:, :1].expand(4, 9, V + 3), t), (x[:0], t[:0]), (x.view(2, 2, 9, V + 3)[:, :, ::2], t.view(2, 2, 9)[:, :, ::2])):
            if a.numel():
                check_logprobs(a, b, 3)
            else:
                assert d.token_logprobs(a, b, entropy=True, top=3).top_ids.shape == (0, 9, 3)


def grad_ref(x, t, lse, a, H=None, b=None):
    """(gradient, tolerance): p has the roundings of lse (where lse is large, 256 for fp32 and 16384 for bf16, it is not taken from it but
    from the row: the forward's bound), of x - lse and of the exponential's argument, and 2^-22."""
    V = x.shape[-1]
    real = (t >= 0) & (t < V)
    a = torch.where(real, a.double(), 0.0)[..., None]
    lp = log_softmax_ref(x)[0]
    p = lp.exp()
    hit = torch.arange(V, device="cuda") == t.long()[..., None]
    size = lp.abs().clamp(max=1e4).nan_to_num(0.0)
    far = lse.double().abs().nan_to_num(0.0).clamp(max=256.0 if x.dtype == F32 else 16384.0)[..., None]
    rel = 2.0 ** -22 + 4 * U * (1 + size) + U * far * 1.01 + logprob_tol(x)[0][..., None]
    g = a * (hit.double() - p)
    tol = a.abs() * p * rel + a.abs() * hit * U + 1e-38
    if b is not None:
        b = b.double()[..., None]
        low = torch.where(torch.isneginf(lp), 0.0, lp) + H.double()[..., None]
        g = g - torch.where(torch.isneginf(lp), 0.0, b * p * low)
        # log p + entropy may cancel: the rounding of lse (U |lse|, or the row's own sum) is in log p as it stands, not relative to the sum
        tol = tol + b.abs() * p * (U * far * 1.01 + logprob_tol(x)[0][..., None])
        tol = tol + b.abs() * p * ((size + H.double().abs()[..., None]) * (rel + 3 * U)) + 2 * U * (a.abs() + b.abs() * (size + H.double().abs()[..., None])) * p
        nothing = (a == 0) & (b == 0)
    else:
        nothing = a == 0
    nothing = nothing | torch.isneginf(lse)[..., None]
    g = torch.where(nothing, 0.0, g)
    return g, (tol + g.abs() * HALF[x.dtype] * 1.01).nan_to_num(0.0)


def check_grad(x, t, seed=0, in_place=False):
    gen = gen_of(seed)
    shape = x.shape[:-1]
    _, lse, H = logprob_ref(x, t)
    lse, H = lse.float(), H.float()
    a, b = torch.randn(shape, generator=gen, device="cuda"), torch.randn(shape, generator=gen, device="cuda")
    if a.numel() > 2:
        a.view(-1)[1], b.view(-1)[1] = 0.0, 0.0
        a.view(-1)[2] = 0.0
    for H1, b1 in ((None, None), (H, b)):
        want, tol = grad_ref(x, t, lse, a, H1, b1)
        out = x.clone() if in_place else None
        got = d.token_logprobs_grad(out if in_place else x, t, lse, a, H1, b1, out=out)
        assert got.dtype == x.dtype and (not in_place or got is out)
        check(got, want, tol)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", LENGTHS)
def test_logprobs_grad(V, dtype):
    for rows in (1, 13):
        g = gen_of(V + rows)
        x = (torch.randn(2, rows, V, generator=g, device="cuda") * 3).to(dtype)
        t = torch.randint(-1, V + 1, (2, rows), generator=g, device="cuda")
        check_grad(x, t, V, in_place=rows == 13)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("kind", ["one left", "none left", "half", "lowest", "all lowest", "nan", "constant"])
def test_logprobs_grad_of_masked_rows(kind, dtype):
    x = _masked((torch.randn(2, 5, 1031, generator=gen_of(3), device="cuda") * 3).to(dtype), kind)
    check_grad(x, torch.randint(0, 1031, (2, 5), generator=gen_of(4), device="cuda", dtype=torch.int32))


@pytest.mark.parametrize("weight", [40.0, 1e5, 1e10, -1e29, 1e31, 1e36])
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("lowest", [False, True])
def test_logprobs_grad_of_masked_logits_is_zero_whatever_the_weights(lowest, dtype, weight):
    """A probability of 0 takes any weight to 0: in pieces of 16 bytes, in front of them and behind, near zero and where rows are summed anew."""
    V = 1031
    low = torch.finfo(dtype).min if lowest else -math.inf
    for offset, first in ((0.0, 0), (0.0, 3), (-100.0, 5), (3e4, 1)):
        x = (torch.randn(2, 5, V, generator=gen_of(6), device="cuda") * 3 + offset).to(dtype)
        x[..., ::3] = low
        x[:, 1, 10:] = low
        x = torch.cat([x.new_zeros(2, 5, first), x], -1)[..., first:]
        t = torch.randint(0, V, (2, 5), generator=gen_of(7), device="cuda")
        _, lse, H = logprob_ref(x, t)
        lse, H = lse.float(), H.float()
        a, b = torch.randn(2, 5, generator=gen_of(8), device="cuda"), torch.randn(2, 5, generator=gen_of(9), device="cuda") * 0.1
        b = b + math.copysign(1.0, weight)          # nowhere near 0
        for a1, b1 in ((a, b * abs(weight)), (a * abs(weight), b), (a * abs(weight), b * abs(weight))):
            want, tol = grad_ref(x, t, lse, a1, H, b1)
            got = d.token_logprobs_grad(x, t, lse, a1, H, b1)
            masked = (x <= low) & (torch.arange(V, device="cuda") != t[..., None])
            assert bool((got[masked] == 0).all())
            # (a probability below 2^-126 is 0)
            check(got, want, tol + 2.0 ** -126 * (a1.abs() + 100 * b1.abs()).double()[..., None])


@pytest.mark.parametrize("offset", [0.0, 304.0, 600.0, -1016.0, 1504.0, -1504.0, 1968.0])
def test_logprobs_grad_of_confident_bf16_rows_far_from_zero(offset):
    """1 - p at the token of rows whose next logits are a few steps below: what is left of it does not drown in the rounding of a large lse."""
    V = 1031
    x = torch.full((4, 3, V), offset - 200.0, device="cuda").to(BF)
    t = torch.randint(0, V, (4, 3), generator=gen_of(3), device="cuda")
    for k in range(1, 4):
        x.scatter_(-1, ((t + 7 * k) % V)[..., None], offset - 8.0)
    x.scatter_(-1, t[..., None], offset)
    r = d.token_logprobs(x, t, entropy=True)
    a = torch.full((4, 3), -0.75, device="cuda")
    lp = log_softmax_ref(x)[0].gather(-1, t[..., None])[..., 0]
    want = a.double() * -torch.expm1(lp)
    got = d.token_logprobs_grad(x, t, r.lse, a).gather(-1, t[..., None])[..., 0]
    # near zero: lse, x - lse and 2^t, 2^-22 each at most; far: a sum of a few terms, its logarithm, a product
    check(got, want, want.abs() * HALF[BF] * 1.01 + a.abs().double() * (2.0 ** -22 + 16 * U))


def test_logprobs_grad_layouts():
    g = gen_of(8)
    for dtype, V in ((BF, 1000), (F32, 1001), (BF, 9001)):
        x = torch.randn(4, 9, V + 3, generator=g, device="cuda").to(dtype)
        t = torch.randint(0, V, (4, 9), generator=g, device="cuda")
        for a, b in ((x[:, :-1], t[:, 1:]), (x[..., 1:V + 1], t), (x[..., 3:], t), (x[:, ::2], t[:, ::2]), (x.transpose(0, 1), t.t()), (x[0, 0], t[0, 0])):
            check_grad(a, b)
        _, lse, _ = logprob_ref(x, t)
        buf = torch.full((4, 11, V + 20), 5.0, dtype=dtype, device="cuda")
        w = torch.randn(4, 9, generator=g, device="cuda")
        for at in (1, 8):
            buf.fill_(5.0)
            got = d.token_logprobs_grad(x, t, lse.float(), w, out=buf[:, 1:10, at:at + V + 3])
            want, tol = grad_ref(x, t, lse.float(), w)
            check(got, want, tol)
            got.fill_(5.0)
            assert bool((buf == 5).all())


def test_logprobs_grad_is_the_difference_quotient():
    """(f(x + h v) - f(x - h v)) / 2 h of f = sum(a logp + b H), f from the forward pass in fp32: errors of f over 2 h, and h^2."""
    M, n, V, h = 2, 3, 40, 2.0 ** -5
    g = gen_of(11)
    x, v = torch.randn(M, n, V, generator=g, device="cuda"), torch.randn(M, n, V, generator=g, device="cuda")
    t = torch.randint(0, V, (M, n), generator=g, device="cuda")
    a, b = torch.randn(M, n, generator=g, device="cuda"), torch.randn(M, n, generator=g, device="cuda")

    def f(x):
        r = d.token_logprobs(x, t, entropy=True)
        return (a * r.logp + b * r.entropy).double().sum()

    r = d.token_logprobs(x, t, entropy=True)
    grad = d.token_logprobs_grad(x, t, r.lse, a, r.entropy, b)
    quotient = float((f(x + h * v) - f(x - h * v)) / (2 * h))
    slope = float((grad.double() * v).sum())
    # third derivatives of logp and H along v are at most a few |v|^3; errors of f at most 1e-5 a row
    assert abs(quotient - slope) <= h * h * 6 * float((a.abs() + 4 * b.abs()).sum()) * float(v.abs().max()) ** 3 + M * n * 1e-5 * 2 / h


# ---- clipping ----------------------------------------------------------------------------------------
def lists(M, numel, dtype, seed, packed, size=None):
    g = gen_of(seed)
    out = []
    for m in range(M):
        scale = 1.0 if size is None else size[m]
        flat = torch.empty(sum(numel) + 1, dtype=dtype, device="cuda")
        row, at = [], 1 if packed else 0
        for n in numel:
            v = (torch.randn(n, generator=g, device="cuda") * scale).to(dtype)
            row.append(flat[at:at + n].copy_(v) if packed else v)
            at += n
        out.append(row)
    return out


NUMEL = {"one": [1], "small": [4096], "ragged": [1, 7, 4097, 72, 5000, 33, 8], "many": [(i * 37) % 300 + 1 for i in range(700)], "large": [300000, 3, 1 << 20, 77777],
         "mid": [200000, 5, 4096, 33] + [70] * 40, "chunks": [4000, 90] * 200}


@pytest.mark.parametrize("src,dst", [(F32, F32), (F32, BF), (BF, BF), (BF, F32)])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("M,which", [(1, "one"), (2, "small"), (4, "ragged"), (3, "many"), (4, "large"), (40, "ragged"), (256, "small"), (3, "mid"), (18, "mid"),
                                     (19, "mid"), (2, "chunks")])
def test_clip_grads(M, which, packed, src, dst):
    numel = NUMEL[which]
    opt, _ = context(M, [(n,) for n in numel], grad_dtype="bf16")
    size = [(10.0 ** ((m % 5) - 2)) / math.sqrt(sum(numel)) for m in range(M)]
    grads, out = lists(M, numel, src, 1, packed, size), lists(M, numel, dst, 2, packed)
    before = [[t.clone() for t in row] for row in grads]
    norms, factors = opt.clip_grads(grads, 1.5, out=out)
    for m in range(M):
        flat = torch.cat([t.double() for t in before[m]])
        norm = float(flat.norm())
        # squares and their sums: at most 128 of a thread, the lanes' tree and the warps' in fp32, then fp64; half of it behind the root
        assert abs(float(norms[m]) - norm) <= norm * (75 * U)
        f = min(1.0, 1.5 / norm)
        assert abs(float(factors[m]) - f) <= f * 76 * U and (f < 1 or float(factors[m]) == 1.0)
        for k, t in enumerate(out[m]):
            want = before[m][k].double() * f
            check(t, want, want.abs() * (HALF[dst] * 1.01 + 78 * U) + 1e-40)
            assert torch.equal(grads[m][k], before[m][k])
    if src == dst:
        n2, f2 = opt.clip_grads(grads, 1.5)        # in place
        assert torch.equal(n2, norms) and torch.equal(f2, factors)
        for m in range(M):
            for k in range(len(numel)):
                assert torch.equal(grads[m][k], out[m][k])


def test_clip_grads_of_zeros_infinities_and_nan():
    numel = [4096, 100]
    opt, _ = context(5, [(n,) for n in numel])
    grads = lists(5, numel, F32, 1, False)
    for t in grads[0]:
        t.zero_()
    grads[1][1][7] = math.inf
    grads[2][0][9] = math.nan
    grads[3][0][:] = 1e-30
    grads[3][1][:] = 0.0
    out = lists(5, numel, F32, 2, False)
    norms, factors = opt.clip_grads(grads, 1.0, out=out)
    assert float(norms[0]) == 0.0 and float(factors[0]) == 1.0 and not bool(out[0][0].any())
    assert math.isinf(float(norms[1])) and float(factors[1]) == 0.0
    assert math.isnan(float(out[1][1][7])) and not bool(out[1][0].any())        # 0 * infinity
    assert math.isnan(float(norms[2])) and float(factors[2]) == 1.0 and torch.equal(out[2][1], grads[2][1])
    assert float(factors[3]) == 1.0 and torch.equal(out[3][0], grads[3][0])
    assert 0 < float(factors[4]) < 1


def test_clip_grads_scales_as_a_norm_clipped_step_does():
    for which in ("ragged", "large"):
        numel = NUMEL[which]
        for M in (3, 60):
            opt, _ = context(M, [(n,) for n in numel], grad_dtype="f32")
            grads = lists(M, numel, F32, 1, False, [0.1 * m / math.sqrt(sum(numel)) for m in range(M)])
            norms, factors = opt.clip_grads(grads, 0.15, out=lists(M, numel, F32, 2, False))
            opt.step_normclip(0, 1e-3, grads, 0.15)
            n, f = opt.grad_norms()
            # (the same kernels' sums up to 131072 parameters, else another order of additions: 75 roundings on either side)
            for a, b in zip(norms.tolist() + factors.tolist(), n + f):
                assert a == b if sum(numel) <= 131072 and M <= 37 else abs(a - b) <= 150 * U * b


# ---- together ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("grad_dtype", ["f32", "bf16"])
def test_a_tied_language_model_of_several_workers(grad_dtype):
    """Embedding, a layer, tied logits, loss with an entropy term, its gradients back through all of it, clipping, steps -- against the same in
    64 bits with torch's own differentiation, from the same parameters at every step."""
    M, V, D, n, scale = 3, 257, 40, 70, 2.0
    opt, x = context(M, [(V, D), (D, D)], grad_dtype=grad_dtype)
    for row in x:
        for t in row:
            t.mul_(0.3)
    dt = {"f32": F32, "bf16": BF}[grad_dtype]
    grads = [[torch.empty(V, D, dtype=dt, device="cuda"), torch.empty(D, D, dtype=dt, device="cuda")] for _ in range(M)]
    clipped = [[torch.empty_like(t) for t in row] for row in grads]
    for t in range(4):
        tokens = tokens_of(M, n + 1, V, 20 + t)
        tokens[:, -3:] = -1
        inputs, targets = tokens[:, :-1], tokens[:, 1:]
        want, losses = [], []
        for m in range(M):
            E, W = x[m][0].double().requires_grad_(), x[m][1].double().requires_grad_()
            real_in, real = inputs[m] >= 0, targets[m] >= 0
            h = torch.zeros(n, D, dtype=torch.float64, device="cuda").index_put((real_in.nonzero()[:, 0],), scale * E[inputs[m][real_in]])
            logp = torch.log_softmax(torch.tanh(h @ W) @ E.t(), -1)
            H = -(logp.exp() * logp).sum(-1)
            loss = -(logp.gather(1, targets[m].clamp(min=0)[:, None])[:, 0] * real).sum() / n - 0.01 * H.mean()
            want.append(torch.autograd.grad(loss, [E, W]))
            losses.append(float(loss.detach()))
        E, W = torch.stack([r[0] for r in x]), torch.stack([r[1] for r in x])
        h = opt.embed(0, inputs, scale=scale, dtype="f32")
        pre = torch.tanh(h @ W)
        logits = pre @ E.transpose(1, 2)
        r = d.token_logprobs(logits, targets, entropy=True)
        assert torch.allclose(-r.logp.sum(1) / n - 0.01 * r.entropy.mean(1), torch.tensor(losses, device="cuda"), rtol=1e-5)
        dl = d.token_logprobs_grad(logits, targets, r.lse, torch.full_like(r.logp, -1 / n), r.entropy, torch.full_like(r.logp, -0.01 / n), out=logits)
        dpre = (dl @ E) * (1 - pre * pre)
        head = dl.transpose(1, 2) @ pre
        dW, dh = h.transpose(1, 2) @ dpre, dpre @ W.transpose(1, 2)
        for m in range(M):
            grads[m][0].copy_(head[m])
            grads[m][1].copy_(dW[m])
        opt.embed_grad(0, inputs, dh, grads, scale=scale, accumulate=True)
        # two roundings to the gradients' type for the embedding; products of 40 to 257 terms in fp32
        for m in range(M):
            for k in range(2):
                size = float(want[m][k].abs().max())
                twice = head[m].double().abs() if k == 0 else 0.0
                check(grads[m][k], want[m][k], 2.1 * HALF[dt] * (want[m][k].abs() + twice) + 600 * U * size)
        norms, factors = opt.clip_grads(grads, 0.05, out=clipped)
        for m in range(M):
            norm = float(torch.cat([g.double().flatten() for g in grads[m]]).norm())
            assert abs(float(norms[m]) - norm) <= 75 * U * norm and abs(float(factors[m]) - min(1, 0.05 / norm)) <= 76 * U
        opt.step(t, 0.5, clipped)
    assert opt.counters()[0] == 4


# ---- offsets that do not fit 32 bits -----------------------------------------------------------------
def test_tables_of_more_than_two_to_the_31_elements():
    V, D, n = (1 << 20) + 77, 2056, 50
    x = torch.empty(1, V * D, device="cuda")
    assert x.numel() > 1 << 31
    opt = d.DesLoc([[x[0].view(V, D)]], [[torch.empty_like(x[0])]], None, opt="sgdm", grad_dtype="bf16", K=(1, 1, 1))
    tokens = torch.cat([torch.arange(V - 20, V), torch.tensor([V - 1] * 40), torch.tensor([0, 5, V // 2])]).cuda()[None]
    rows = torch.randn(tokens.shape[1], D, generator=gen_of(1), device="cuda")
    x.view(V, D)[tokens[0]] = rows
    assert torch.equal(opt.embed(0, tokens, dtype="f32")[0], x.view(V, D)[tokens[0]])
    grads = [[torch.full((V, D), 5.0, dtype=BF, device="cuda")]]
    dout = torch.randn(1, tokens.shape[1], D, generator=gen_of(2), device="cuda").to(BF)
    opt.embed_grad(0, tokens, dout, grads)
    seen = tokens.unique()
    want = torch.stack([dout[0][tokens[0] == v].double().sum(0) for v in seen])
    size = torch.stack([dout[0][tokens[0] == v].double().abs().sum(0) for v in seen])
    check(grads[0][0][seen], want, size * 62 * U + want.abs() * HALF[BF] * 1.01)
    empty = torch.ones(V, dtype=torch.bool, device="cuda")
    empty[seen] = False
    assert not bool(grads[0][0][-5000:][empty[-5000:]].any()) and not bool(grads[0][0][:5000][empty[:5000]].any())
    assert int((grads[0][0] != 0).any(1).sum()) == len(seen)


def test_rows_more_than_two_to_the_31_elements_apart():
    V, far = 9000, (1 << 31) + 4096
    buf = torch.empty(2 * far + V, dtype=BF, device="cuda")
    x = buf.as_strided((3, V), (far, 1))
    x.copy_(torch.randn(3, V, generator=gen_of(1), device="cuda") * 3)
    t = torch.tensor([1, 2, V - 1], device="cuda")
    check_logprobs(x, t, 5)
    near = x.clone()
    _, lse, _ = logprob_ref(near, t)
    w = torch.ones(3, device="cuda")
    want = d.token_logprobs_grad(near, t, lse.float(), w)
    assert torch.equal(d.token_logprobs_grad(x, t, lse.float(), w, out=x), want)


# ---- streams, graphs, refusals -----------------------------------------------------------------------
def _all_calls(opt, s):
    out = opt.embed(0, s["tokens"], out=s["emb"])
    r = d.token_logprobs(s["logits"], s["tokens"], entropy=True, top=4)
    dl = d.token_logprobs_grad(s["logits"], s["tokens"], r.lse, s["w"], r.entropy, s["w"])
    opt.embed_grad(0, s["tokens"], s["dout"], s["grads"])
    norms, factors = opt.clip_grads(s["grads"], 0.5, out=s["clipped"])
    return [out, *r, dl, norms, factors] + [g[0] for g in s["grads"]] + [g[0] for g in s["clipped"]]


def _state(M, V, D, n):
    g = gen_of(1)
    r = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    return dict(tokens=tokens_of(M, n, V, 2), logits=r(M, n, V), w=r(M, n), dout=r(M, n, D).to(BF), emb=torch.empty(M, n, D, dtype=BF, device="cuda"),
                grads=[[torch.empty(V, D, dtype=BF, device="cuda")] for _ in range(M)], clipped=[[torch.empty(V, D, dtype=BF, device="cuda")] for _ in range(M)])


def _refill(s, seed):
    g = gen_of(seed)
    s["tokens"].copy_(tokens_of(*s["tokens"].shape, s["logits"].shape[-1], seed))
    for k in ("logits", "w", "dout"):
        s[k].copy_(torch.randn(s[k].shape, generator=g, device="cuda"))


@pytest.mark.parametrize("V,n", [(300, 70), (20000, 9)])
def test_captured_calls_see_what_the_buffers_hold(V, n):
    M, D = 3, 64
    opt, x = context(M, [(V, D)])
    s = _state(M, V, D, n)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for _ in range(2):                               # two graphs of the same context, with working memory of their own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = _all_calls(opt, s)
        graphs.append((graph, got))
    for seed in (5, 6):
        _refill(s, seed)
        x[0][0].mul_(1.5)
        for graph, got in graphs:
            graph.replay()
        torch.cuda.synchronize()
        kept = [[t.clone() for t in got] for _, got in graphs]
        fresh = _all_calls(opt, s)
        for got in kept:
            for a, b in zip(got, fresh):
                assert torch.equal(a, b)


def test_captured_clipping_of_many_tensors():
    """Thousands of addresses travel with the captured launches."""
    numel = NUMEL["many"]
    opt, _ = context(3, [(n,) for n in numel])
    grads, out = lists(3, numel, F32, 1, True, [0.1, 1.0, 10.0]), lists(3, numel, BF, 2, True)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        norms, factors = opt.clip_grads(grads, 2.0, out=out)
    other = lists(3, numel, F32, 3, True)
    opt.clip_grads(other, 2.0, out=lists(3, numel, BF, 4, True))        # other lists in between
    for k in range(2):
        for row in grads:
            for t in row:
                t.mul_(1.5)
        for row in out:
            for t in row:
                t.zero_()
        graph.replay()
        got = [[t.clone() for t in row] for row in out]
        n, f = norms.clone(), factors.clone()
        n2, f2 = opt.clip_grads(grads, 2.0, out=out)
        assert torch.equal(n, n2) and torch.equal(f, f2)
        assert all(torch.equal(a, b) for x, y in zip(got, out) for a, b in zip(x, y))


def test_a_wait_that_runs_out_is_reported_by_the_next_call():
    numel = NUMEL["large"]
    opt, _ = context(4, [(n,) for n in numel], grad_dtype="f32")
    grads, out = lists(4, numel, F32, 1, False), lists(4, numel, F32, 2, False)
    d.desloc_testing_set_wait_limit(opt.ctx, 0)
    opt.clip_grads(grads, 1.0, out=out)
    torch.cuda.synchronize()
    tokens = torch.zeros(4, 3, dtype=torch.int64, device="cuda")
    for call in (lambda: opt.clip_grads(grads, 1.0, out=out), lambda: opt.embed(0, tokens, width=1),
                 lambda: opt.embed_grad(0, tokens, torch.zeros(4, 3, 1, device="cuda"), grads, width=1), lambda: opt.step(0, 1e-3, grads)):
        with pytest.raises(d.DeslocError) as e:
            call()
        assert e.value.status == d.DESLOC_E_DEVICE_WAIT
    d.desloc_testing_set_wait_limit(opt.ctx, -1)
    norms, _ = opt.clip_grads(grads, 1.0, out=out)
    for m in range(4):
        want = float(torch.cat([t.double() for t in grads[m]]).norm())
        assert abs(float(norms[m]) - want) <= 75 * U * want


def test_calls_run_on_the_current_stream():
    M, V, D, n = 2, 500, 32, 40
    opt, _ = context(M, [(V, D)])
    s = _state(M, V, D, n)
    want = [t.clone() for t in _all_calls(opt, s)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        big = torch.ones(1 << 26, device="cuda")
        for _ in range(20):
            big = big * 1.0001                       # the buffers are written behind this
        for k in ("emb",):
            s[k].zero_()
        got = [t.clone() for t in _all_calls(opt, s)]
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_calls_read_and_write_behind_what_is_on_their_stream():
    """Inputs are overwritten and outputs spoiled on a side stream, behind work that takes longer than the host: each call has to see that."""
    M, V, D, n = 2, 500, 32, 40
    opt, _ = context(M, [(V, D)])
    s, coming = _state(M, V, D, n), _state(M, V, D, n)
    _refill(coming, 11)
    want = [t.clone() for t in _all_calls(opt, coming)]
    old = _all_calls(opt, s)
    lse, H = old[2].clone(), old[3].clone()          # (the forward's, of the inputs that come)
    lse.copy_(want[2]), H.copy_(want[3])
    dl = d.token_logprobs_grad(coming["logits"], coming["tokens"], lse, coming["w"], H, coming["w"])
    grads = [[torch.empty_like(g[0])] for g in coming["grads"]]
    for g, c in zip(grads, coming["grads"]):
        g[0].copy_(c[0])
    big = torch.ones(1 << 26, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def late():
        for _ in range(100):
            big.mul_(1.0001)
        for k in ("tokens", "logits", "w", "dout"):
            s[k].copy_(coming[k])
        s["emb"].fill_(3.0)
        for k in ("grads", "clipped"):
            for row in s[k]:
                row[0].fill_(3.0)

    for again in range(2):                           # (the first time memory is allocated)
        _refill(s, 5)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            late()
            emb = opt.embed(0, s["tokens"], out=s["emb"]).clone()
            fresh = opt.embed(0, s["tokens"])
            r = d.token_logprobs(s["logits"], s["tokens"], entropy=True, top=4)
            grad = d.token_logprobs_grad(s["logits"], s["tokens"], lse, s["w"], H, s["w"])
            opt.embed_grad(0, s["tokens"], s["dout"], s["grads"])
            own = [row[0].clone() for row in s["grads"]]
            for row, g in zip(s["grads"], grads):
                row[0].copy_(g[0])
            norms, factors = opt.clip_grads(s["grads"], 0.5, out=s["clipped"])
            clipped = [row[0].clone() for row in s["clipped"]]
            assert again == 0 or not side.query()        # (the work in front was still running when all of this was called)
        side.synchronize()
        for a, b in zip([emb, fresh, *r, grad, norms, factors, *own, *clipped], [want[0], want[0], *want[1:6], dl, *want[7:9], *want[9:9 + M], *want[9 + M:]]):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    """Calls without common working memory do not disturb one another."""
    M, V, D, n = 2, 3000, 256, 2000
    opt, _ = context(M, [(V, D)])
    states = [_state(M, V, D, n), _state(M, V, D, n)]
    _refill(states[1], 9)
    want = [[t.clone() for t in _all_calls(opt, s)] for s in states]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(5):
        for k in (0, 1):
            with torch.cuda.stream(streams[k]):
                got[k] = _all_calls(opt, states[k])
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        for u, v in zip(a, b):
            assert torch.equal(u, v)


def test_refusals():
    M, V, D = 2, 50, 8
    opt, _ = context(M, [(V, D), (13,)])
    tokens, dev = torch.zeros(M, 4, dtype=torch.int64, device="cuda"), "cuda"
    dout = torch.zeros(M, 4, D, device=dev)
    g = [[torch.zeros(V, D, dtype=BF, device=dev), torch.zeros(13, dtype=BF, device=dev)] for _ in range(M)]

    def refused(kind, call, status=None):
        with pytest.raises(kind) as e:
            call()
        if status is not None:
            assert e.value.status == status

    for bad in (tokens.cpu(), tokens[:1], tokens.float(), tokens[0, 0]):
        refused(ValueError, lambda: opt.embed(0, bad))
        refused(ValueError, lambda: opt.embed_grad(0, bad, dout, g))
    refused(ValueError, lambda: opt.embed(5, tokens))
    refused(ValueError, lambda: opt.embed(0, tokens, dtype="f16"))
    refused(ValueError, lambda: opt.embed(0, tokens, dtype=torch.float16))
    assert opt.embed(0, tokens, dtype=torch.float32).dtype == F32
    none = torch.zeros(M, 0, dtype=torch.int64, device="cuda")
    assert opt.embed(0, none, out=torch.zeros(M, 0, D, device="cuda")).shape == (M, 0, D)
    opt.embed_grad(0, none, torch.zeros(M, 0, D, device="cuda"), tuple(g))
    refused(ValueError, lambda: opt.embed(-1, tokens))
    refused(ValueError, lambda: opt.embed(1, tokens))                            # one dimension and no width
    refused(d.DeslocError, lambda: opt.embed(1, tokens, width=5), d.DESLOC_E_RANGE)
    refused(d.DeslocError, lambda: opt.embed(0, tokens, width=0), d.DESLOC_E_RANGE)
    refused(d.DeslocError, lambda: opt.embed(0, tokens, scale=math.inf), d.DESLOC_E_RANGE)
    refused(d.DeslocError, lambda: opt.embed_grad(0, tokens, dout, g, scale=math.nan), d.DESLOC_E_RANGE)
    refused(ValueError, lambda: opt.embed(0, tokens, out=torch.zeros(M, 4, D + 1, device=dev)))
    refused(ValueError, lambda: opt.embed(0, tokens, out=torch.zeros(M, 4, D, device=dev, dtype=torch.float16)))
    refused(ValueError, lambda: opt.embed(0, tokens, out=torch.zeros(M, 4, D)))
    refused(ValueError, lambda: opt.embed(0, tokens, out=torch.zeros(M, 4, 2 * D, device=dev)[..., ::2]))
    refused(ValueError, lambda: opt.embed_grad(0, tokens, dout[:, 1:], g))
    refused(ValueError, lambda: opt.embed_grad(0, tokens, dout.half(), g))
    refused(ValueError, lambda: opt.embed_grad(0, tokens, dout.cpu(), g))
    refused(ValueError, lambda: opt.embed_grad(0, tokens, dout, g[:1]))
    refused(ValueError, lambda: opt.embed_grad(0, tokens, dout, [[t.float() for t in row] for row in g]))
    refused(ValueError, lambda: opt.embed_grad(0, tokens, dout, [[t.cpu() for t in row] for row in g]))
    for bad in (0.0, -1.0, math.inf, math.nan):
        refused(d.DeslocError, lambda: opt.clip_grads(g, bad), d.DESLOC_E_RANGE)
    refused(ValueError, lambda: opt.clip_grads([[t.cpu() for t in row] for row in g], 1.0))
    refused(ValueError, lambda: opt.clip_grads(g, 1.0, out=[[t.cpu() for t in row] for row in g]))
    refused(ValueError, lambda: opt.clip_grads([[t.half() for t in row] for row in g], 1.0))
    refused(ValueError, lambda: opt.clip_grads([[g[0][0], g[0][1].float()], g[1]], 1.0))
    refused(ValueError, lambda: opt.clip_grads(g[:1], 1.0))
    x, t = torch.zeros(2, 3, 8, device=dev), torch.zeros(2, 3, dtype=torch.int64, device=dev)
    w = torch.zeros(2, 3, device=dev)
    refused(ValueError, lambda: d.token_logprobs(x.half(), t))
    refused(ValueError, lambda: d.token_logprobs(x, t[:1]))
    refused(ValueError, lambda: d.token_logprobs(x, t.cpu()))
    refused(ValueError, lambda: d.token_logprobs(x, t.float()))
    refused(d.DeslocError, lambda: d.token_logprobs(x, t, top=d.DESLOC_MAX_TOP + 1), d.DESLOC_E_RANGE)
    refused(ValueError, lambda: d.token_logprobs_grad(x, t, w[:1], w))
    refused(ValueError, lambda: d.token_logprobs_grad(x, t, w, w.double()))
    refused(ValueError, lambda: d.token_logprobs_grad(x, t, w, w, dentropy=w))
    refused(ValueError, lambda: d.token_logprobs_grad(x, t, w, w, out=x.bfloat16()))
    refused(ValueError, lambda: d.token_logprobs_grad(x, t, w, w, out=torch.zeros(2, 3, 16, device=dev)[..., ::2]))
    # the C entry points' own
    B = d.binding if hasattr(d, "binding") else __import__("paper_2505_22549_b200.binding", fromlist=["x"])
    rows = lambda t, k, *s: B.rows(t.data_ptr(), k, *s)
    ok, to = rows(tokens, d.DESLOC_I64, 4, 1), rows(dout, d.DESLOC_F32, 4 * D, D)
    ptrs = [r.data_ptr() for row in g for r in row]
    need = B.desloc_embed_grad_bytes(opt.ctx, 0, D, 4)
    work = torch.zeros(need + 256, dtype=torch.uint8, device=dev)
    at = -(-work.data_ptr() // 256) * 256
    call = lambda **k: (lambda a: B.desloc_embed_grad(opt.ctx, a["tensor"], a["width"], a["tokens"], a["n"], a["dout"], 1.0, False, a["g"], a["work"],
                                                      a["bytes"]))({**dict(tensor=0, width=D, tokens=ok, n=4, dout=to, g=ptrs, work=at, bytes=need), **k})
    call()
    refused(d.DeslocError, lambda: call(bytes=need - 1), d.DESLOC_E_RANGE)
    refused(d.DeslocError, lambda: call(work=at + 64), d.DESLOC_E_INVALID)
    refused(d.DeslocError, lambda: call(work=0), d.DESLOC_E_NULL)
    refused(d.DeslocError, lambda: call(n=-1), d.DESLOC_E_RANGE)
    refused(d.DeslocError, lambda: call(n=(1 << 30) + 1), d.DESLOC_E_RANGE)
    refused(d.DeslocError, lambda: call(tensor=2), d.DESLOC_E_RANGE)
    refused(d.DeslocError, lambda: call(width=1 << 21), d.DESLOC_E_RANGE)
    refused(d.DeslocError, lambda: call(g=[0] * 4), d.DESLOC_E_NULL)
    refused(d.DeslocError, lambda: call(tokens=B.rows(0, d.DESLOC_I64, 4, 1)), d.DESLOC_E_NULL)
    refused(d.DeslocError, lambda: call(dout=rows(dout, 5, 4 * D, D)), d.DESLOC_E_INVALID)
    clip = lambda **k: (lambda a: B.desloc_clip_grads(opt.ctx, 1.0, a["gt"], a["g"], a["ot"], a["o"], 0, 0, a["work"], a["bytes"]))(
        {**dict(gt=1, g=ptrs, ot=1, o=ptrs, work=at2, bytes=need2), **k})
    need2 = B.desloc_clip_grads_bytes(opt.ctx)
    work2 = torch.zeros(need2 + 256, dtype=torch.uint8, device=dev)
    at2 = -(-work2.data_ptr() // 256) * 256
    clip()
    refused(d.DeslocError, lambda: clip(bytes=need2 - 1), d.DESLOC_E_RANGE)
    refused(d.DeslocError, lambda: clip(work=at2 + 8), d.DESLOC_E_INVALID)
    refused(d.DeslocError, lambda: clip(gt=2), d.DESLOC_E_INVALID)
    refused(d.DeslocError, lambda: clip(ot=0), d.DESLOC_E_INVALID)               # in place, another type
    refused(d.DeslocError, lambda: clip(g=[0] * 4), d.DESLOC_E_NULL)
    refused(d.DeslocError, lambda: clip(o=[ptrs[0] + 1] + ptrs[1:]), d.DESLOC_E_INVALID)


@pytest.mark.parametrize("M", [2, 5])
def test_outputs_that_overlap_are_refused(M):
    V, D, dev = 50, 8, "cuda"
    opt, _ = context(M, [(V, D), (13,)])
    tokens, dout = torch.zeros(M, 4, dtype=torch.int64, device=dev), torch.ones(M, 4, D, device=dev)
    g = [[torch.zeros(V, D, dtype=BF, device=dev), torch.zeros(13, dtype=BF, device=dev)] for _ in range(M)]

    def invalid(call):
        with pytest.raises(d.DeslocError) as e:
            call()
        assert e.value.status == d.DESLOC_E_INVALID

    one = torch.zeros(D, device=dev)
    invalid(lambda: opt.embed(0, tokens, out=one.expand(M, 4, D)))
    invalid(lambda: opt.embed(0, tokens, out=torch.zeros(4, D, device=dev).expand(M, 4, D)))
    invalid(lambda: opt.embed(0, tokens, out=torch.zeros(M * 4 * D, device=dev).as_strided((M, 4, D), (4 * D, D - 1, 1))))
    both = torch.zeros(4, M, D, device=dev)
    opt.embed(0, tokens, out=both.transpose(0, 1))                               # rows of the workers in turn do not
    assert torch.equal(both.transpose(0, 1), opt.embed(0, tokens, dtype="f32"))
    whole = torch.zeros(2 * V * D, dtype=BF, device=dev)
    invalid(lambda: opt.embed_grad(0, tokens, dout, g[:M - 1] + g[:1]))
    invalid(lambda: opt.embed_grad(0, tokens, dout, [[whole[V * D:], g[0][1]]] + g[:M - 2] + [[whole[V * D - 1:-1], g[0][1]]]))
    opt.embed_grad(0, tokens, dout, [[whole[V * D:], g[0][1]]] + g[:M - 2] + [[whole[:V * D], g[0][1]]])   # one behind the other do not
    assert whole[::V * D].tolist() == [4, 4]
    invalid(lambda: opt.clip_grads(g[:1] * M, 1.0))
    invalid(lambda: opt.clip_grads(g, 1.0, out=[[a[0].clone(), g[0][1]] for a in g]))
    opt.clip_grads(g[:1] * M, 1.0, out=g[1:] + [[t.clone() for t in g[0]]])      # read by all of them is fine
    x, t = torch.zeros(8, device=dev).expand(2, 3, 8), torch.zeros(2, 3, dtype=torch.int64, device=dev)
    r, w = d.token_logprobs(x, t), torch.ones(2, 3, device=dev)
    invalid(lambda: d.token_logprobs_grad(x, t, r.lse, w, out=x))                # rows that all are one
    assert d.token_logprobs_grad(x, t, r.lse, w).shape == x.shape


def test_bound_gradients_of_other_workers_or_from_the_host_are_refused():
    V, D, dev = 50, 8, "cuda"
    opt, state = context(1, [(V, D)])
    two, _ = context(2, [(V, D)])
    tokens, dout = torch.zeros(2, 4, dtype=torch.int64, device=dev), torch.ones(2, 4, D, device=dev)
    few = opt.bind_grads([[torch.zeros(V, D, dtype=BF, device=dev)]])
    host = two.bind_grads([[torch.zeros(V, D, dtype=BF)] for _ in range(2)])
    for bound in (few, host):
        for call in (lambda: two.embed_grad(0, tokens, dout, bound), lambda: two.clip_grads(bound, 1.0)):
            with pytest.raises(ValueError, match="gradient tensor"):
                call()


def test_clipping_refuses_lists_that_share_memory():
    M, numel = 3, [40, 13]
    opt, _ = context(M, [(n,) for n in numel])
    new = lambda dtype=BF: [[torch.ones(n, dtype=dtype, device="cuda") for n in numel] for _ in range(M)]

    def invalid(call):
        with pytest.raises(d.DeslocError) as e:
            call()
        assert e.value.status == d.DESLOC_E_INVALID

    g, to = new(), new()
    for lists in ([g[0], g[1], g[0]], [g[0], g[1], [g[0][0], g[2][1]]], [[g[0][0], g[0][0][:13]], g[1], g[2]]):
        invalid(lambda: opt.clip_grads(lists, 1.0))
        invalid(lambda: opt.clip_grads(new(F32), 1.0, out=lists))
    invalid(lambda: opt.clip_grads(g, 1.0, out=[g[1], g[0], g[2]]))
    buf = torch.ones(41, dtype=BF, device="cuda")
    invalid(lambda: opt.clip_grads([[buf[:40], g[0][1]], g[1], g[2]], 1.0, out=[[buf[1:], to[0][1]], to[1], to[2]]))
    assert all(bool((t == 1).all()) for row in g + to for t in row)      # nothing ran
    opt.clip_grads([g[0], g[1], g[0]], 1.0, out=to)                       # read by two of them
    assert torch.equal(to[0][0], to[2][0])
    mixed = [to[0], g[1], to[2]]                                          # one worker in place
    opt.clip_grads(g, 1.0, out=mixed)
    for m in range(M):
        for k in range(2):
            check(mixed[m][k], torch.full((numel[k],), 1 / math.sqrt(53), dtype=torch.float64, device="cuda"), HALF[BF] * 1.01 / math.sqrt(53))


def test_what_is_written_counts_as_changed():
    """torch's version counters rise for what a call writes, and for nothing else: a saved tensor that was overwritten is refused in backward()."""
    M, V, D, n = 2, 50, 8, 6
    opt, _ = context(M, [(V, D), (13,)], grad_dtype="f32")
    tokens, dout = tokens_of(M, n, V, 1), torch.ones(M, n, D, device="cuda")
    new = lambda: [[torch.zeros(V, D, device="cuda"), torch.zeros(13, device="cuda")] for _ in range(M)]
    versions = lambda lists: [[t._version for t in row] for row in lists]
    out = torch.zeros(M, n, D, device="cuda")
    before = out._version, tokens._version
    opt.embed(0, tokens, out=out)
    assert out._version > before[0] and tokens._version == before[1]
    for bind in (False, True):
        grads, to = new(), new()
        given, given_to = (opt.bind_grads(grads), opt.bind_grads(to)) if bind else (grads, to)
        v = versions(grads)
        opt.embed_grad(0, tokens, dout, given)
        opt.embed_grad(0, tokens[:, ::2], dout[:, ::2], given, accumulate=True)
        assert all(row[0]._version > w[0] and row[1]._version == w[1] for row, w in zip(grads, v))
        v, w = versions(grads), versions(to)
        opt.clip_grads(given, 1.0, out=given_to)
        assert versions(grads) == v and all(a > b for x, y in zip(versions(to), w) for a, b in zip(x, y))
        opt.clip_grads(given, 1.0)
        assert all(a > b for x, y in zip(versions(grads), v) for a, b in zip(x, y))
    z = torch.randn(M, n, V, generator=gen_of(2), device="cuda", requires_grad=True)
    for view in (lambda x: x, lambda x: x[:, ::2], lambda x: x[:, None, None]):
        logits = torch.tanh(z)
        own, t = view(logits.detach()), view(tokens)
        r = d.token_logprobs(own, t)
        assert logits._version == 0
        d.token_logprobs_grad(own, t, r.lse, torch.ones_like(r.lse), out=own)
        assert logits._version == 1
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            logits.sum().backward()


def test_outputs_made_in_inference_mode_are_taken():
    M, V, D, n = 2, 50, 8, 6
    opt, _ = context(M, [(V, D)], grad_dtype="f32")
    tokens = tokens_of(M, n, V, 1)
    with torch.inference_mode():
        out, grads, x = torch.zeros(M, n, D, device="cuda"), [[torch.zeros(V, D, device="cuda")] for _ in range(M)], torch.zeros(M, n, V, device="cuda")
    for mode in (False, True):
        with torch.inference_mode(mode):
            opt.embed(0, tokens, out=out)
            opt.embed_grad(0, tokens, out, grads)
            opt.clip_grads(grads, 1.0)
            r = d.token_logprobs(x, tokens)
            d.token_logprobs_grad(x, tokens, r.lse, torch.ones_like(r.lse), out=x)
    torch.cuda.synchronize()
