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
