"""Products of the workers' matrices next to one another and to other work: calls in a row, lists that fill launches and rounds, every element of the results."""
import pytest
import torch

import paper_2505_22549_b200 as d
from paper_2505_22549_b200 import binding as B
import test_matrices_gpu as base

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def test_small_matrices_and_the_block_in_turn():
    """Blocks that take some of an SM's TMEM and little shared memory next to those of a kernel that takes all of it, each kernel beginning while the one in front still runs."""
    shapes = [(8, 8), (16, 24), (72, 72)]
    opt = base.context(3, shapes)
    u = base.matrices(3, shapes, 1)
    out = [[torch.empty(s, device="cuda") for s in shapes] for _ in range(3)]
    blocks = [base.Block(2, 300, 64, 512), base.Block(1, 8, 40, 72), base.Block(2, 1024, 512, 1024)]
    opt.orthogonalize(range(3), u, out=out)
    wants = [t.clone() for row in out for t in row], [b.opt.gated_ffn(b.TENSORS, b.h, b.weights).clone() for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.current_stream(), torch.cuda.Stream()]
    for t in (t for row in out for t in row):
        t.zero_()
    torch.cuda.synchronize()
    ys = []
    for _ in range(30):
        for k, b in enumerate(blocks):
            opt.orthogonalize(range(3), u, out=out)
            with torch.cuda.stream(streams[1]):
                other = b.opt.gated_ffn(b.TENSORS, b.h, b.weights)
            ys.append((k, b.opt.gated_ffn(b.TENSORS, b.h, b.weights)))
            ys.append((k, other))
    torch.cuda.synchronize()
    assert all(torch.equal(y, wants[1][k]) for k, y in ys)
    assert all(torch.equal(t, w) for t, w in zip((t for row in out for t in row), wants[0]))


@pytest.mark.parametrize("tokens,width,hidden", [(8, 40, 72), (300, 512, 640)])
def test_polls_are_not_spent_on_earlier_kernels(tokens, width, hidden):
    """A kernel that began while one in front of it has 32 steps of a small matrix to go, 700 us or 400 polls: its own waits are a few microseconds, and only those count."""
    shape = (128, 500)
    long, b = base.context(1, [shape]), base.Block(2, tokens, width, hidden)
    u, out = base.matrices(1, [shape]), [[torch.empty(shape, device="cuda")]]
    steps = [(1.5, -0.5, 0.0)] * 32
    want = b.opt.gated_ffn(b.TENSORS, b.h, b.weights).clone()
    long.orthogonalize([0], u, out=out, coefficients=steps)
    torch.cuda.synchronize()
    B.desloc_testing_set_wait_limit(b.opt.ctx, 128)
    for _ in range(3):
        long.orthogonalize([0], u, out=out, coefficients=steps)
        y = b.opt.gated_ffn(b.TENSORS, b.h, b.weights)
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    b.opt.gated_ffn(b.TENSORS, b.h, b.weights)     # (refused where a wait had run out)
    torch.cuda.synchronize()


# ---- what shares memory ------------------------------------------------------------------------------
def addresses(lists):
    return B.ptr_array([t.data_ptr() for row in lists for t in row])


def test_results_over_the_contexts_momentum_are_refused_at_the_entry():
    """updates NULL, the context's u: a result at the place of another matrix's u, or of another type at its own.  (No working memory: no call gets as far as a launch.)"""
    shapes = [(16, 24), (16, 24), (130, 200)]
    u = base.matrices(2, shapes, 1)
    opt = base.context(2, shapes, u=u)
    how = B.orthogonal([0, 1, 2], [24, 24, 200])
    go = lambda out, dtype=d.DESLOC_F32: B.raw_lib().desloc_orthogonalize(opt.ctx, how, dtype, addresses(out), None, 0, None)
    fresh = base.matrices(2, shapes, 2)
    assert go(fresh) == d.DESLOC_E_NULL and go(u) == d.DESLOC_E_NULL      # apart; each in place
    swapped = [[u[0][1], u[0][0], u[0][2]], u[1]]
    workers = [[u[1][0], *u[0][1:]], [u[0][0], *u[1][1:]]]
    behind = [[fresh[0][0], u[0][2].view(-1)[4:4 + 384], fresh[0][2]], fresh[1]]
    for out in (swapped, workers, behind):
        assert go(out) == d.DESLOC_E_INVALID
    assert go(u, d.DESLOC_BF16) == d.DESLOC_E_INVALID
    assert B.raw_lib().desloc_orthogonalize(opt.ctx, B.orthogonal([0], [24]), d.DESLOC_F32, addresses(behind), None, 0, None) == d.DESLOC_E_NULL   # (what is not read may be written)


def test_a_step_along_what_lies_in_another_matrix_is_refused():
    """At the entry without working memory, so that no call gets as far as a launch; then from Python, what is fine."""
    shapes = [(16, 24), (16, 24), (130, 200)]
    x, fresh = base.matrices(2, shapes, 1), base.matrices(2, shapes, 2)
    opt = base.context(2, shapes, x=x, grad_dtype="f32")
    bf = B.DESLOC_BF16

    def go(updates=None, grads=None, dtype=d.DESLOC_F32):
        how = B.orthogonal([0, 1, 2], [24, 24, 200], updates_dtype=dtype, updates=addresses(updates) if updates else None, grads=addresses(grads) if grads else None)
        return B.raw_lib().desloc_orthogonal_step(opt.ctx, how, 0.1, None, 0, None)

    swapped = [[x[0][1], x[0][0], x[0][2]], x[1]]
    workers = [[x[1][0], *x[0][1:]], [x[0][0], *x[1][1:]]]
    behind = [[fresh[0][0], x[0][2].view(-1)[4:4 + 384], fresh[0][2]], fresh[1]]
    for lists in (swapped, workers, behind):
        assert go(updates=lists) == d.DESLOC_E_INVALID and go(grads=lists) == d.DESLOC_E_INVALID and go(updates=fresh, grads=lists) == d.DESLOC_E_INVALID
    assert go(updates=x, dtype=bf) == d.DESLOC_E_INVALID
    for lists in (x, fresh):
        assert go(updates=lists) == d.DESLOC_E_NULL and go(grads=lists) == d.DESLOC_E_NULL
    assert go() == d.DESLOC_E_NULL


def test_a_step_along_the_weights_themselves():
    shapes = [(16, 24), (130, 200)]
    x = base.matrices(1, shapes, 1)
    opt = base.context(1, shapes, x=x)
    before = [t.double() for t in x[0]]
    opt.orthogonal_step([0, 1], 1e-4, updates=x, scale="none")
    for t, was in zip(x[0], before):
        want, off = base.allowed(was)
        base.close(t, was - float(torch.tensor(1e-4)) * want, 1e-4 * off + 4 * base.U * float(was.norm() + 1e-4 * want.norm()))


# ---- the look-ahead ----------------------------------------------------------------------------------
@pytest.mark.parametrize("grad_dtype", ["bf16", "f32"])
@pytest.mark.parametrize("src", ["bf16", "f32"])
def test_look_ahead_of_clipped_gradients(grad_dtype, src):
    """Of gradients of which a third lie beyond the clip radius, for matrices that a block takes alone and others."""
    shapes, rho = [(24, 60), (23, 61), (300, 200), (200, 301), (576, 192), (131, 130)], 1e-4
    opt = base.context(2, shapes, grad_dtype, beta1=0.9, clip_rho=rho)
    u, g = base.matrices(2, shapes, 1, base.TYPE[src]), base.matrices(2, shapes, 2, base.TYPE[grad_dtype])
    out = [[torch.empty(s, device="cuda") for s in shapes] for _ in range(2)]
    opt.orthogonalize(range(len(shapes)), u, grads=g, out=out)
    beta, bound = float(torch.tensor(0.9)), float(torch.tensor(rho))
    for m in range(2):
        for k in range(len(shapes)):
            ahead = beta * u[m][k].double() + (1 - beta) * g[m][k].double().clamp(-bound, bound)
            want, off = base.allowed(ahead)
            # (the look-ahead is formed in fp32: three roundings of it, which no product enlarges by more than 3.5^5)
            base.close(out[m][k], want, off + 3 * base.U * 3.5 ** 5 * float(want.norm()))
    g[1][2][5, 7] = float("nan")
    g[1][0][3, 2] = float("nan")
    g[0][0][3, 2] = float("inf")       # (clipped as any other)
    opt.orthogonalize(range(len(shapes)), u, grads=g, out=out)
    assert not bool(torch.isfinite(out[1][2]).all()) and not bool(torch.isfinite(out[1][0]).all()) and bool(torch.isfinite(out[0][0]).all())


def test_a_step_with_clipping_in_both_halves():
    """step() at rate 0 and orthogonal_step() of the same gradients, in a context that clips coordinates: momentum and look-ahead of the same clipped gradients."""
    M, shapes, rho, lr = 3, [(40, 96), (300, 130), (7,)], 0.5, 0.01
    g = base.gen_of(3)
    x = [[torch.randn(s, generator=g, device="cuda") * 0.1 for s in shapes] for _ in range(M)]
    opt = base.context(M, shapes, x=x, grad_dtype="f32", beta1=0.9, clip_rho=rho)
    momentum = [[torch.zeros(s, dtype=torch.float64, device="cuda") for s in shapes] for _ in range(M)]
    beta = float(torch.tensor(0.9))
    for t in (1, 5):                     # (K = 2, 3, 4: nothing is averaged)
        grads = [[torch.randn(s, generator=g, device="cuda") for s in shapes] for _ in range(M)]
        before = [[w.double() for w in row] for row in x]
        assert opt.step(t, 0.0, grads) == 0
        opt.orthogonal_step([0, 1], lr, grads=grads, scale="none")
        for m in range(M):
            for k in range(3):
                clipped = grads[m][k].double().clamp(-rho, rho)
                momentum[m][k] = beta * momentum[m][k] + (1 - beta) * clipped
                base.check(opt._keep[1][m][k], momentum[m][k], 8 * base.U * rho)
                if k == 2:
                    assert torch.equal(x[m][k].double(), before[m][k])
                    continue
                want, off = base.allowed(beta * momentum[m][k] + (1 - beta) * clipped)
                rate = float(torch.tensor(lr))
                base.close(x[m][k], before[m][k] - rate * want, rate * (off + 8 * base.U * 3.5 ** 5 * float(want.norm())) + 4 * base.U * float(before[m][k].norm()))


def test_a_step_of_the_momentum_where_averages_come_behind_is_refused():
    shapes = [(16, 24), (5,)]
    def made(M, K):
        zeros = lambda: [[torch.ones(s, device="cuda") for s in shapes] for _ in range(M)]
        return d.DesLoc(zeros(), zeros(), None, opt="sgdm", grad_dtype="f32", K=K, flags=d.DESLOC_FLAG_POST_AVERAGE)
    for K in ((2, 0, 0), (0, 3, 0), (2, 3, 4)):
        opt = made(2, K)
        for call in (lambda: opt.orthogonal_step([0], 0.1), lambda: opt.orthogonal_step([0], 0.1, grads=base.matrices(2, [(16, 24), (5, 1)], 1)),
                     lambda: opt.orthogonal_step([0], 0.1, columns=[48])):
            with pytest.raises(d.DeslocError) as e:
                call()
            assert e.value.status == d.DESLOC_E_INVALID
        assert all(bool((t == 1).all()) for row in opt._keep[0] for t in row)
        opt.orthogonal_step([0], 0.1, updates=base.matrices(2, [(16, 24), (5, 1)], 1))
        assert not any(bool((row[0] == 1).all()) for row in opt._keep[0])
    for M, K in ((1, (2, 3, 4)), (2, (0, 0, 4))):
        opt = made(M, K)
        opt.orthogonal_step([0], 0.1)
        assert not any(bool((row[0] == 1).all()) for row in opt._keep[0])


@pytest.mark.parametrize("shape", [(300, 400), (400, 300), (576, 1536)])
def test_a_matrix_beside_one_of_few_rows_keeps_its_bits(shape):
    """Products of few rows begin with another k in every tile; what stands beside them in a launch does not."""
    shapes = [shape, (5000, 60)]
    opt = base.context(1, shapes)
    u = base.matrices(1, shapes, 1)
    out = [[torch.empty(s, device="cuda") for s in shapes]]
    opt.orthogonalize([0], u, out=out)
    alone = out[0][0].clone()
    opt.orthogonalize([0, 1], u, out=out)
    assert torch.equal(out[0][0], alone)


@pytest.mark.parametrize("shape", [(40, 24), (200, 130)])
def test_ends_of_the_norms_range(shape):
    """Values whose squares are no normal numbers any more, down to those that count as 0, and beyond fp32's."""
    opt = base.context(1, [shape])
    u, out = base.matrices(1, [shape], 5), [[torch.empty(shape, device="cuda")]]
    start = u[0][0] * 1e4
    for far, eps in ((1e-19, 0.0), (1e-24, 1e-7), (1e20, 1e-7)):
        u[0][0].copy_(start.clamp(-4, 4) * far)
        opt.orthogonalize([0], u, out=out, eps=eps)
        if far == 1e-19:
            # (squares between 1e-45 and 2e-37, off by 2^-150 or 2^-24 of them: the norm by far less than the operands)
            base.close(out[0][0], *base.allowed(u[0][0], eps=eps))
        else:
            assert bool((out[0][0] == 0).all())


# ---- every element of orthogonalised updates ---------------------------------------------------------
def definition(u, steps=base.DEFAULT, eps=1e-7, rounded=False):
    """Of matrices [count, rows, columns] in 64 bits; `rounded`: with what the grouped kernels round to fp16 rounded there."""
    x = u.double()
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + eps)
    tall = x.shape[1] > x.shape[2]
    x = x.mT if tall else x
    half = (lambda v, unit=256.0: (v * unit).half().double() / unit) if rounded else lambda v: v
    one = torch.eye(x.shape[1], dtype=torch.float64, device=x.device)
    for k, (a, b, c) in enumerate(steps):
        hi = half(x)
        rest = half((x - hi) * 2048.0) / 2048.0 if rounded and k + 1 < len(steps) else torch.zeros_like(x)
        gram = half(hi @ hi.mT)
        x = half(a * one + b * gram + c * (gram @ gram)) @ hi + a * rest
    return x.mT if tall else x


def elements(got, u, dst, factor=1.0, steps=base.DEFAULT, eps=1e-7):
    """[count, rows, columns] of results, each element for itself.  An element's error is the sum of thousands of independent roundings, near normal, and the emulation's errors are
    another draw of the same: of a million such values none is beyond eight times their root mean square, and the kernels' is at most twice the emulation's (sums in fp32,
    cut off, beside fp16's roundings).  The result's own rounding on top."""
    want = definition(u, steps, eps)
    error = definition(u, steps, eps, True) - want
    rms = error.square().mean((1, 2), keepdim=True).sqrt()
    want = want * factor
    tol = 16 * rms * factor + base.HALF[dst] * want.abs() + 8 * base.U * want.abs()
    assert bool(torch.isfinite(got).all())
    over = (got.double() - want).abs() - tol
    assert float(over.max()) <= 0, f"off by {float(over.max()):.3e} more than allowed, {float(tol.max()):.3e}"
    # (a row or an element of zeros, or of another place, would be far outside)
    assert float((want.abs() > 3 * tol).double().mean()) > 0.8


def placed(t, shift):
    """The same values `shift` elements off a boundary of 16 bytes."""
    buf = torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda")[shift:shift + t.numel()].view(t.shape)
    return buf.copy_(t)


LARGE = [(300, 200), (576, 192), (200, 301), (131, 130), (257, 129), (160, 600)]


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("grad", [None, "bf16", "f32"])
@pytest.mark.parametrize("src,dst", [("f32", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("scale", ["aspect", "rms"])
def test_every_element_of_larger_matrices(src, dst, grad, scale, shift):
    """Both sides above what a block takes alone: with and without the look-ahead, of all types, on and off boundaries, scaled, into another tensor and in place."""
    M = 2
    opt = base.context(M, LARGE, grad or "bf16", beta1=0.9)
    S, D = base.TYPE[src], base.TYPE[dst]
    at = lambda lists: [[placed(t, shift) for t in row] for row in lists]
    u = at(base.matrices(M, LARGE, 1, S))
    g = at(base.matrices(M, LARGE, 2, base.TYPE[grad])) if grad else None
    out = at([[torch.empty(s, dtype=D, device="cuda") for s in LARGE] for _ in range(M)])
    opt.orthogonalize(range(len(LARGE)), u, grads=g, out=out, scale=scale)
    beta = torch.tensor(0.9)
    for k, (r, c) in enumerate(LARGE):
        ahead = torch.stack([row[k] for row in u])
        if grad:     # (formed in fp32, as the kernels do: two roundings next to fp16's are none)
            ahead = float(beta) * ahead.double() + (1 - float(beta)) * torch.stack([row[k] for row in g]).double()
        factor = max(1.0, r / c) ** 0.5 if scale == "aspect" else 0.2 * max(r, c) ** 0.5
        elements(torch.stack([row[k] for row in out]), ahead, D, factor)
    if src == dst:
        opt.orthogonalize(range(len(LARGE)), u, grads=g, scale=scale)
        assert all(torch.equal(p, q) for r, s in zip(u, out) for p, q in zip(r, s))
    if grad == dst:      # in the place of the gradients
        u = at(base.matrices(M, LARGE, 1, S))
        opt.orthogonalize(range(len(LARGE)), u, grads=g, out=g, scale=scale)
        assert all(torch.equal(p, q) for r, s in zip(g, out) for p, q in zip(r, s))


@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("grad", [None, "bf16"])
def test_every_element_of_a_step(grad, shift):
    M, shapes, lr, decay = 2, LARGE + [(40, 96), (96, 40), (23, 61)], 0.05, 0.1
    x = [[placed(torch.randn(s, generator=base.gen_of(9 + m), device="cuda") * 0.02, shift) for s in shapes] for m in range(M)]
    u = base.matrices(M, shapes, 6)
    g = base.matrices(M, shapes, 7, BF) if grad else None
    before = [[t.double() for t in row] for row in x]
    opt = base.context(M, shapes, x=x, u=u, weight_decay=decay, beta1=0.9)
    opt.orthogonal_step(range(len(shapes)), lr, grads=g, scale="aspect")
    lr, decay, beta = float(torch.tensor(lr)), float(torch.tensor(decay)), float(torch.tensor(0.9))
    for k, (r, c) in enumerate(shapes):
        ahead = torch.stack([row[k] for row in u]).double()
        if grad:
            ahead = beta * ahead + (1 - beta) * torch.stack([row[k] for row in g]).double()
        was, now = torch.stack([row[k] for row in before]), torch.stack([row[k] for row in x]).double()
        f = lr * max(1.0, r / c) ** 0.5
        want = definition(ahead)
        rms = (definition(ahead, rounded=True) - want).square().mean((1, 2), keepdim=True).sqrt()
        total = was * (1 - lr * decay) - f * want
        over = (now - total).abs() - (16 * rms * f + 4 * base.U * (was.abs() + f * want.abs()))
        assert float(over.max()) <= 0, f"{(r, c)}: off by {float(over.max()):.3e} more than allowed"


def test_more_matrices_than_a_round_and_more_shapes_than_a_launch():
    """660 matrices, none for a block alone: 21 shapes (a launch takes 16), 600 matrices of one (a round takes 512).  Each of them against the definition; the same bits in another order."""
    M = 3
    shapes = [(129 + 5 * k, 131 + (k * 37) % 120) for k in range(20)] + [(130, 133)] * 200
    opt = base.context(M, shapes)
    u = base.matrices(M, shapes, 7)
    out, again = ([[torch.zeros(s, device="cuda") for s in shapes] for _ in range(M)] for _ in range(2))
    opt.orthogonalize(range(len(shapes)), u, out=out)
    opt.orthogonalize(list(range(len(shapes)))[::-1], u, out=again)
    assert all(torch.equal(p, q) for r, s in zip(out, again) for p, q in zip(r, s))
    for k in range(20):
        elements(torch.stack([row[k] for row in out]), torch.stack([row[k] for row in u]), F32)
    for m in range(M):
        elements(torch.stack(out[m][20:]), torch.stack(u[m][20:]), F32)


def test_more_than_a_rounds_bytes():
    """2.6 GB of working memory, of which a round takes 2: the second round's matrices use the first one's memory again, and one of the shapes is cut in two."""
    shapes = [(4096, 2048)] * 13 + [(2048, 4090)] * 29
    opt = base.context(1, shapes)
    u = base.matrices(1, shapes, 8)
    out = [[torch.zeros(s, dtype=BF, device="cuda") for s in shapes]]
    steps = base.DEFAULT[:2]
    opt.orthogonalize(range(len(shapes)), u, out=out, coefficients=steps)
    for k in range(len(shapes)):
        elements(out[0][k][None], u[0][k][None], BF, steps=steps)


# ---- matrices that a block takes alone ---------------------------------------------------------------
def by_pairs(u, steps=base.DEFAULT, eps=1e-7, terms=(1, 1), lo_of="XGP", cut=0.0):
    """In 64 bits with every operand as two fp16 numbers and three products of them, as those matrices are multiplied.  terms, lo_of: with one of the products, or the smaller numbers
    of X, G or the polynomial, left out.  cut: with sums cut off: an instruction adds sixteen products to an fp32 accumulator, off by four units of 2^-24 of the
    magnitudes at most, all in the same direction at worst."""
    x = u.double()
    x = x / (x.norm() + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.mT if tall else x
    one = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)

    def two(v, name):
        hi = (v * 1024.0).half().double()
        return hi / 1024.0, (v * 1024.0 - hi).half().double() / 1024.0 * (name in lo_of)

    def product(a, b):
        total = a[0] @ b[0] + terms[0] * (a[0] @ b[1]) + terms[1] * (a[1] @ b[0])
        return total - torch.sign(total) * cut * 12 * -(-a[0].shape[1] // 16) * base.U * (a[0].abs() @ b[0].abs())

    for a, b, c in steps:
        X = two(x, "X")
        G = two(product(X, [t.mT for t in X]), "G")
        x = product(two(a * one + b * (G[0] + G[1]) + c * product(G, [t.mT for t in G]), "P"), X)
    return x.mT if tall else x


@pytest.mark.parametrize("shape", [(1, 5), (8, 8), (24, 72), (64, 64), (72, 72), (200, 72), (128, 128), (128, 250)])
def test_small_matrices_are_as_exact_as_pairs_of_numbers(shape):
    """fp32 results; 2^-20 of the norm stands for the roundings to fp32 between the products.  Without any one of the products or of the smaller numbers a result would be outside."""
    opt = base.context(1, [shape])
    u, out = base.matrices(1, [shape], 3), [[torch.empty(shape, device="cuda")]]
    opt.orthogonalize([0], u, out=out)
    u, want = u[0][0], base.newton_schulz(u[0][0])
    pairs = by_pairs(u)
    bound = 2 * float((pairs - want).norm()) + float((by_pairs(u, cut=1.0) - pairs).norm()) + 2.0 ** -20 * float(want.norm())
    base.close(out[0][0], want, bound)
    if shape != (1, 5):
        for less in (dict(terms=(0, 1)), dict(terms=(1, 0)), dict(lo_of="GP"), dict(lo_of="XP"), dict(lo_of="XG")):
            assert float((by_pairs(u, **less) - want).norm()) > bound


# ---- the block in calls of other kinds ---------------------------------------------------------------
def all_of_it(b, M):
    """y, kept, dh and the weights' gradients of a block against the definition."""
    (g, u, y), tols = b.forward(b.h)
    got, kept = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)
    for have, want, tol in zip((*kept, got), (g, u, y), tols):
        base.check(have, want, tol)
    grads = [[torch.zeros(s, dtype=BF, device="cuda") for s in ((b.F, b.D), (b.D, b.F), (5,), (b.F, b.D))] for _ in range(M)]
    dh = b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, grads)
    (want, tol), *weights = b.backward(b.h, *kept, b.dy)
    base.check(dh, want, tol + base.HB * (want.abs() + tol) + 1e-30)
    for k, (want, tol) in zip(b.TENSORS, weights):
        for m in range(M):
            base.check(grads[m][k], want[m], tol[m] + (base.HB + 2 * base.U) * (want[m].abs() + tol[m]) + 1e-30)


@pytest.mark.parametrize("M,T,D,F,shift", [(70, 6, 15, 23, 1), (70, 2, 16, 24, 1), (130, 9, 8, 16, 3), (256, 5, 8, 8, 0), (18, 40, 72, 200, 4)])
def test_more_workers_than_a_launch_with_weights_off_boundaries(M, T, D, F, shift):
    all_of_it(base.Block(M, T, D, F, shift=shift), M)


@pytest.mark.parametrize("off", [(0, 1, 0), (1, 0, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1)])
@pytest.mark.parametrize("M,T", [(2, 50), (18, 7)])
def test_some_weights_on_and_some_off_boundaries(M, T, off):
    b = base.Block(M, T, 40, 72)
    for k, shift in zip(b.TENSORS, off):
        for row in b.weights[1:]:        # (the first worker's lie well)
            row[k] = placed(row[k], shift)
    all_of_it(b, M)


def test_after_the_workers_have_changed():
    b = base.Block(2, 30, 40, 72)
    want = b.opt.gated_ffn(b.TENSORS, b.h, b.weights)
    shapes = ((72, 40), (40, 72), (5,), (72, 40))
    x, u = ([[torch.zeros(s, device="cuda") for s in shapes] for _ in range(3)] for _ in range(2))
    keep = b.opt._keep
    b.opt.set_workers([keep[0][0], keep[0][1], x[2]], [keep[1][0], keep[1][1], u[2]], None, 2)
    h = torch.cat([b.h, b.h[:1]])
    y = b.opt.gated_ffn(b.TENSORS, h, b.weights + [b.weights[0]])
    assert torch.equal(y[:2], want) and torch.equal(y[2], want[0])
    with pytest.raises(ValueError):
        b.opt.gated_ffn(b.TENSORS, b.h, b.weights)
    new = base.matrices(3, [(72, 40), (40, 72), (5, 1), (72, 40)], 4)
    for row, values in zip(b.opt._keep[1], new):
        for t, v in zip(row, values):
            t.copy_(v.view(t.shape))
    before = [[t.double() for t in row] for row in b.opt._keep[0]]
    b.opt.orthogonal_step([0, 1], 0.01, scale="none")
    for m in range(3):
        for k in (0, 1):
            want, off = base.allowed(new[m][k])
            rate = float(torch.tensor(0.01))
            base.close(b.opt._keep[0][m][k], before[m][k] - rate * want, rate * off + 4 * base.U * float(want.norm()))
    # the momentum's addresses are the new ones
    how = B.orthogonal([0, 1], [40, 72])
    rows = b.opt._keep[1]
    go = lambda out: B.raw_lib().desloc_orthogonalize(b.opt.ctx, how, d.DESLOC_F32, addresses(out), None, 0, None)
    assert go(rows) == d.DESLOC_E_NULL and go([rows[0], rows[2], rows[1]]) == d.DESLOC_E_INVALID


def test_one_weight_in_several_places():
    """gate and up the same tensor; one set of weights for all workers."""
    b = base.Block(3, 33, 40, 72)
    row = list(b.weights[0])
    row[b.TENSORS[1]] = row[b.TENSORS[0]]
    b.weights = [row] * 3
    b.gate, b.up, b.down = (torch.stack([r[k] for r in b.weights]).double() for k in b.TENSORS)
    all_of_it(b, 3)


def test_contexts_of_two_threads():
    """Each with its own context and stream, calls at the same time: what launches are made of is a thread's own."""
    import threading
    blocks = [base.Block(2, 200 + 60 * k, 64 + 8 * k, 256, seed=k) for k in range(2)]
    shapes = [[(300, 200), (64, 40)], [(200, 301), (24, 72)]]
    opts, us = [base.context(2, s) for s in shapes], [base.matrices(2, s, 5 + k) for k, s in enumerate(shapes)]
    outs = [[[torch.empty(s, device="cuda") for s in row] for _ in range(2)] for row in shapes]
    wants = []
    for k in range(2):
        opts[k].orthogonalize([0, 1], us[k], out=outs[k])
        wants.append([blocks[k].opt.gated_ffn(blocks[k].TENSORS, blocks[k].h, blocks[k].weights)] + [t.clone() for row in outs[k] for t in row])
    torch.cuda.synchronize()
    failed = []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(60):
                    y = blocks[k].opt.gated_ffn(blocks[k].TENSORS, blocks[k].h, blocks[k].weights)
                    opts[k].orthogonalize([0, 1], us[k], out=outs[k])
                    got = [y] + [t for row in outs[k] for t in row]
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(p, q) for p, q in zip(got, wants[k])):
                        failed.append(k)
                    torch.cuda.current_stream().synchronize()
        except Exception as e:     # noqa: BLE001 (told to the test below)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed


def test_as_many_tokens_as_there_may_be():
    """2^24 of one worker: sums of the weights' gradients over 262144 boxes, gradients of the first and last tokens alone."""
    T, D, F, few = 1 << 24, 8, 16, 8
    b = base.Block(1, T, D, F)
    ends = lambda t: torch.cat([t[:, :few], t[:, -few:]], 1)
    y, kept = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)
    want, tol = b.forward(ends(b.h))
    for got, w, t in zip((*kept, y), want, tol):
        base.check(ends(got), w, t)
    b.dy[:, few:-few] = 0
    grads = [[torch.zeros(s, dtype=BF, device="cuda") for s in ((F, D), (D, F), (5,), (F, D))]]
    dh = b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, grads)
    (want, tol), *weights = b.backward(ends(b.h), *map(ends, kept), ends(b.dy))
    base.check(ends(dh), want, tol + base.HB * (want.abs() + tol) + 1e-30)
    for k, (want, tol) in zip(b.TENSORS, weights):
        base.check(grads[0][k], want[0], tol[0] + (base.HB + 2 * base.U) * (want[0].abs() + tol[0]) + 1e-30)
    b.opt.gated_ffn(b.TENSORS, b.h[:, :4], b.weights)      # (refused where a wait had run out)
    with pytest.raises(d.DeslocError) as e:
        b.opt.gated_ffn(b.TENSORS, b.h.new_empty(1, T + 1, D), b.weights)
    assert e.value.status == d.DESLOC_E_RANGE
