"""The gated feed-forward block, its way back and orthogonalised updates against their definitions in 64 bits.

Tolerances count roundings: half a step of a type (bf16 2^-8, fp16 2^-11, fp32 2^-24) where a value is rounded to it; n products added in fp32 in any order, possibly
cut off instead of rounded, are off by at most 2 n 2^-24 times the sum of magnitudes.
"""
import itertools
import math

import pytest
import torch

import paper_2505_22549_b200 as d
from paper_2505_22549_b200 import binding as B

pytestmark = pytest.mark.gpu

U, HB, HH = 2.0 ** -24, 2.0 ** -8, 2.0 ** -11
BF, F32 = torch.bfloat16, torch.float32
HALF = {F32: U, BF: HB}
TYPE = {"f32": F32, "bf16": BF}


def gen_of(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def check(got, want, tol):
    assert got.shape == want.shape
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine)
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, f"off by {float(over.max()):.3e} more than allowed"


def context(M, shapes, grad_dtype="bf16", u=None, x=None, **kw):
    zeros = lambda: [[torch.zeros(s, device="cuda") for s in shapes] for _ in range(M)]
    x, u = x or zeros(), u or zeros()
    return d.DesLoc(x, u, None, opt="sgdm", grad_dtype=grad_dtype, K=(2, 3, 4), **kw)


# ---- the gated feed-forward block --------------------------------------------------------------------
class Block:
    """M workers' block among other tensors: gate, up and down are tensors 3, 0 and 1 of the list."""
    TENSORS = (3, 0, 1)

    def __init__(self, M, T, D, F, grad_dtype="bf16", seed=0, shift=0, scale=1.0):
        g = gen_of(seed)
        self.M, self.T, self.D, self.F = M, T, D, F
        self.h = torch.randn(M, T, D, generator=g, device="cuda").to(BF)
        self.dy = torch.randn(M, T, D, generator=g, device="cuda").to(BF)
        self.opt = context(M, [(F, D), (D, F), (5,), (F, D)], grad_dtype)

        def weight(rows, cols):     # `shift` elements off a boundary of 16 bytes
            buf = torch.empty(rows * cols + 8, dtype=BF, device="cuda")[shift:shift + rows * cols].view(rows, cols)
            return buf.copy_(torch.randn(rows, cols, generator=g, device="cuda") * (scale * cols ** -0.5))

        self.weights = [[weight(F, D), weight(D, F), None, weight(F, D)] for _ in range(M)]
        self.gate, self.up, self.down = (torch.stack([row[k] for row in self.weights]).double() for k in self.TENSORS)

    def forward(self, h):
        """(g, u, y) and how far each may be off"""
        h = h.double()
        g, u = h @ self.gate.mT, h @ self.up.mT
        z = torch.nn.functional.silu(g) * u
        n = 2 * (self.D + 8) * U
        eg, eu = n * (h.abs() @ self.gate.abs().mT), n * (h.abs() @ self.up.abs().mT)
        ez = u.abs() * 1.1 * eg + torch.nn.functional.silu(g).abs() * eu + eg * eu * 1.1 + z.abs() * (HB + 16 * U)
        y = z @ self.down.mT
        ey = (ez + 2 * (self.F + 8) * U * (z.abs() + ez)) @ self.down.abs().mT
        rounded = lambda v, e: e + HB * (v.abs() + e)
        return (g, u, y), (rounded(g, eg), rounded(u, eu), rounded(y, ey) + 1e-30)

    def backward(self, h, g, u, dy):
        """dh, dgate, dup, ddown and how far each may be off before it is rounded"""
        h, dy = h.double(), dy.double()
        leaves = [t.double().requires_grad_() for t in (g, u)]
        z = torch.nn.functional.silu(leaves[0]) * leaves[1]
        dz = dy @ self.down
        dg, du = torch.autograd.grad(z, leaves, dz)
        g, u, z = leaves[0].detach(), leaves[1].detach(), z.detach()
        s = torch.sigmoid(g)
        edz = 2 * (self.D + 8) * U * (dy.abs() @ self.down.abs())
        few = HB + 32 * U
        slope = s + (g * s).abs() * (1 - s)
        edg = u.abs() * slope * (edz + few * dz.abs())
        edu = (g * s).abs() * (edz + few * dz.abs())
        ez = few * z.abs()
        nh, nw = 4 * (self.F + 8) * U, 2 * (h.shape[1] + 8) * U
        full = lambda v, e, n: e + n * (v.abs() + e)
        dh = dg @ self.gate + du @ self.up
        edh = full(dg, edg, nh) @ self.gate.abs() + full(du, edu, nh) @ self.up.abs()
        return [(dh, edh), (dg.mT @ h, full(dg, edg, nw).mT @ h.abs()), (du.mT @ h, full(du, edu, nw).mT @ h.abs()), (dy.mT @ z, dy.abs().mT @ full(z, ez, nw))]


SIZES = [(1, 1, 1, 1), (2, 1, 8, 16), (1, 3, 5, 7), (4, 37, 72, 200), (2, 129, 71, 203), (3, 300, 576, 1536), (2, 128, 64, 64), (1, 257, 130, 66),
         (17, 5, 24, 40), (3, 2, 201, 77), (2, 3, 2048, 1000), (5, 4, 576, 1536), (2, 60, 136, 264), (2, 1000, 200, 520), (1, 2048, 512, 1024), (4, 1, 512, 2048), (200, 1, 8, 16),
         (40, 6, 16, 24), (2, 257, 1030, 300)]


@pytest.mark.parametrize("M,T,D,F", SIZES)
@pytest.mark.parametrize("keep", [False, True])
def test_gated_ffn(M, T, D, F, keep):
    b = Block(M, T, D, F)
    got = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=keep)
    want, tol = b.forward(b.h)
    if keep:
        y, (g, u) = got
        check(g, want[0], tol[0])
        check(u, want[1], tol[1])
        assert torch.equal(y, b.opt.gated_ffn(b.TENSORS, b.h, b.weights))
    else:
        y = got
    check(y, want[2], tol[2])


@pytest.mark.parametrize("M,T,D,F", SIZES)
@pytest.mark.parametrize("grad_dtype,accumulate", [("bf16", False), ("f32", True), ("bf16", True), ("f32", False)])
def test_gated_ffn_grad(M, T, D, F, grad_dtype, accumulate):
    b = Block(M, T, D, F, grad_dtype)
    kept = [torch.randn(M, T, F, generator=gen_of(k), device="cuda").mul_(3).to(BF) for k in (5, 6)]
    start = lambda shape: torch.randn(shape, generator=gen_of(7), device="cuda").to(TYPE[grad_dtype])
    grads = [[start(s) for s in ((F, D), (D, F), (5,), (F, D))] for _ in range(M)]
    before = [[t.double() for t in row] for row in grads]
    dh = b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, grads, accumulate=accumulate)
    (want, tol), *weights = b.backward(b.h, *kept, b.dy)
    check(dh, want, tol + HB * (want.abs() + tol) + 1e-30)
    half = HALF[TYPE[grad_dtype]]
    for k, (want, tol) in zip(b.TENSORS, weights):
        for m in range(M):
            total = want[m] + (before[m][k] if accumulate else 0)
            check(grads[m][k], total, tol[m] + (half + 2 * U) * (total.abs() + want[m].abs() + tol[m]) + 1e-30)
    for m in range(M):
        assert torch.equal(grads[m][2].double(), before[m][2])


def test_gated_ffn_grad_against_differences():
    """Of the definition in 64 bits: the directional derivative by central differences, and what the kernels return, within what they may be off."""
    b = Block(2, 24, 40, 56)
    c = b.dy.double()
    loss = lambda h: float((b.forward(h)[0][2] * c).sum())
    _, (g, u) = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)
    grads = [[torch.zeros(s, dtype=BF, device="cuda") for s in ((56, 40), (40, 56), (5,), (56, 40))] for _ in range(2)]
    dh = b.opt.gated_ffn_grad(b.TENSORS, b.h, (g, u), b.dy, b.weights, grads).double()
    v = torch.randn(b.h.shape, generator=gen_of(3), device="cuda", dtype=torch.float64)
    step = 1e-5
    difference = (loss(b.h.double() + step * v) - loss(b.h.double() - step * v)) / (2 * step)
    # kept g and u are rounded: |silu''| <= 0.5, |silu'| <= 1.1; then what the way back itself may be off
    (G, UU, _), _ = b.forward(b.h)
    (want, tol), *_ = b.backward(b.h, g, u, b.dy)
    dz = (c @ b.down).abs()
    shift = ((dz * (0.5 * UU.abs() * HB * G.abs() + 1.1 * HB * UU.abs()) * 1.02) @ b.gate.abs() + (dz * 1.1 * HB * G.abs() * 1.02) @ b.up.abs())
    bound = float(((shift + tol + HB * (want.abs() + tol)) * v.abs()).sum())
    assert abs(float((dh * v).sum()) - difference) <= bound + 1e-6


def test_gated_ffn_layouts():
    """Token grids, strided and broadcast inputs, outputs inside larger buffers, weights off every boundary; what lies around an output stays as it was."""
    M, T, D, F = 3, 12, 40, 72
    for shift in (0, 1, 4):
        b = Block(M, T, D, F, shift=shift)
        (_, _, want), (_, _, tol) = b.forward(b.h)
        wide = torch.full((M, T + 2, D + 9), 3.0, dtype=BF, device="cuda")
        wide[:, 1:T + 1, 1:D + 1] = b.h
        for h in (b.h, wide[:, 1:T + 1, 1:D + 1], b.h.view(M, 3, 4, D), b.h.view(M, 3, 4, D).transpose(1, 2).contiguous().transpose(1, 2),
                  b.h.transpose(0, 1).contiguous().transpose(0, 1), b.h.transpose(1, 2).contiguous().transpose(1, 2)):
            check(b.opt.gated_ffn(b.TENSORS, h, b.weights).reshape(M, T, D), want, tol)
        for cut in (slice(0, D), slice(1, D + 1), slice(8, D + 8)):
            buf = torch.full((M, T + 2, D + 9), 7.0, dtype=BF, device="cuda")
            y = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, out=buf[:, 1:T + 1, cut])
            check(y, want, tol)
            buf[:, 1:T + 1, cut] = 7.0
            assert bool((buf == 7.0).all())
        # one row for all tokens, one batch for all workers
        for h in (b.h[:, :1].expand(M, T, D), b.h[:1].expand(M, T, D)):
            (_, _, w), (_, _, t) = b.forward(h)
            check(b.opt.gated_ffn(b.TENSORS, h, b.weights), w, t)
        kept = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)[1]
        grads = lambda: [[torch.zeros(s, dtype=BF, device="cuda") for s in ((F, D), (D, F), (5,), (F, D))] for _ in range(M)]
        first, second = grads(), grads()
        dh = b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, first)
        strided = torch.empty(M, T, D + 3, dtype=BF, device="cuda")[:, :, 2:D + 2].copy_(b.dy)
        buf = torch.full((M, T + 2, D + 9), 7.0, dtype=BF, device="cuda")
        same = b.opt.gated_ffn_grad(b.TENSORS, wide[:, 1:T + 1, 1:D + 1], kept, strided, b.weights, b.opt.bind_grads(second), out=buf[:, 1:T + 1, 1:D + 1])
        assert torch.equal(dh, same) and all(torch.equal(p, q) for r, s in zip(first, second) for p, q in zip(r, s))


@pytest.mark.parametrize("T,D,F", [(3, 40, 72), (50, 40, 72), (50, 41, 72), (400, 512, 640)])
def test_gated_ffn_in_the_place_of_what_it_reads(T, D, F):
    b = Block(2, T, D, F)
    y, kept = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)
    h = b.h.clone()
    assert b.opt.gated_ffn(b.TENSORS, h, b.weights, out=h) is h and torch.equal(h, y)
    grads = lambda: [[torch.zeros(s, dtype=BF, device="cuda") for s in ((F, D), (D, F), (5,), (F, D))] for _ in range(2)]
    want = grads()
    dh = b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, want)
    for place in range(2):
        h, dy, got = b.h.clone(), b.dy.clone(), grads()
        out = (h, dy)[place]
        b.opt.gated_ffn_grad(b.TENSORS, h, kept, dy, b.weights, got, out=out)
        assert torch.equal(out, dh) and all(torch.equal(p, q) for r, s in zip(want, got) for p, q in zip(r, s))


def test_gated_ffn_beyond_32_bits():
    """More than 2^31 elements per worker of what lies between the products; gradients of the first and last tokens alone, all others add zeros."""
    M, T, D, F, few = 2, 525000, 64, 4104, 8
    b = Block(M, T, D, F)
    ends = lambda t: torch.cat([t[:, :few], t[:, -few:]], 1)
    y, kept = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)
    want, tol = b.forward(ends(b.h))
    for got, w, t in zip((*kept, y), want, tol):
        check(ends(got), w, t)
    b.dy[:, few:-few] = 0
    grads = [[torch.zeros(s, dtype=BF, device="cuda") for s in ((F, D), (D, F), (5,), (F, D))] for _ in range(M)]
    dh = b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, grads)
    (want, tol), *weights = b.backward(ends(b.h), *map(ends, kept), ends(b.dy))
    check(ends(dh), want, tol + HB * (want.abs() + tol) + 1e-30)
    assert bool((dh[:, few:-few] == 0).all())
    for k, (want, tol) in zip(b.TENSORS, weights):
        for m in range(M):
            check(grads[m][k], want[m], tol[m] + (HB + 2 * U) * (want[m].abs() + tol[m]) + 1e-30)


def test_gated_ffn_extremes():
    """Far gates, zeros, infinities and NaN: each row for itself."""
    b = Block(1, 6, 16, 24)
    h = b.h.clone()
    h[0, 0] = 0
    h[0, 1] *= 1e4              # gates beyond +-1e3: silu is g or 0
    h[0, 2] *= 1e30             # u g leaves the range of fp32
    h[0, 3, 5] = math.nan
    h[0, 4, 5] = math.inf
    y = b.opt.gated_ffn(b.TENSORS, h, b.weights)
    (_, _, want), (_, _, tol) = b.forward(h)
    for r in (0, 1, 5):
        check(y[:, r], want[:, r], tol[:, r])
    assert bool((y[0, 0] == 0).all()) and bool(torch.isnan(y[0, 3]).all()) and not bool(torch.isfinite(y[0, 4]).any()) and not bool(torch.isfinite(y[0, 2]).any())
    # kept values far from zero: the way back has no NaN in it
    kept = torch.full((1, 6, 24), 300.0, dtype=BF, device="cuda"), torch.ones(1, 6, 24, dtype=BF, device="cuda")
    kept[0][0, 1] = -300.0
    kept[0][0, 2] = -3e38
    kept[0][0, 3] = 3e38
    grads = [[torch.zeros(s, dtype=BF, device="cuda") for s in ((24, 16), (16, 24), (5,), (24, 16))]]
    dh = b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, grads)
    (want, tol), *_ = b.backward(b.h, kept[0].clamp(-1e30, 1e30), kept[1], b.dy)
    rows = [0, 1, 2, 4, 5]
    check(dh[:, rows], want[:, rows], (tol + HB * (want.abs() + tol) + 1e-30)[:, rows])


def test_no_tokens():
    b = Block(2, 0, 8, 16)
    assert b.opt.gated_ffn(b.TENSORS, b.h, b.weights).shape == (2, 0, 8)
    y, kept = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)
    assert kept[0].shape == (2, 0, 16)
    for accumulate in (True, False):
        grads = [[torch.ones(s, dtype=BF, device="cuda") for s in ((16, 8), (8, 16), (5,), (16, 8))] for _ in range(2)]
        assert b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, grads, accumulate=accumulate).shape == (2, 0, 8)
        assert all(bool((row[k] == (1 if accumulate or k == 2 else 0)).all()) for row in grads for k in range(4))


def test_gated_ffn_refusals():
    b = Block(2, 4, 8, 16)
    bad = lambda error, f: pytest.raises(error, f)
    run = lambda **kw: b.opt.gated_ffn(kw.get("tensors", b.TENSORS), kw.get("h", b.h), kw.get("weights", b.weights), out=kw.get("out"))
    bad(ValueError, lambda: run(tensors=(3, 3, 1)))
    bad(ValueError, lambda: run(tensors=(3, 0, 4)))
    bad(ValueError, lambda: run(tensors=(3, 0, 2)))
    bad(ValueError, lambda: run(h=b.h.float()))
    bad(ValueError, lambda: run(h=b.h[:1]))
    bad(ValueError, lambda: run(h=b.h.cpu()))
    bad(ValueError, lambda: run(h=b.h[..., :7]))
    bad(ValueError, lambda: run(weights=[[t if t is None else t.float() for t in row] for row in b.weights]))
    bad(ValueError, lambda: run(weights=b.weights[:1]))
    bad(ValueError, lambda: run(weights=[row[:3] for row in b.weights]))
    bad(ValueError, lambda: run(out=torch.empty(2, 4, 9, dtype=BF, device="cuda")))
    bad(d.DeslocError, lambda: run(out=torch.empty(2, 1, 8, dtype=BF, device="cuda").expand(2, 4, 8)))
    kept = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)[1]
    grads = [[torch.zeros(s, dtype=BF, device="cuda") for s in ((16, 8), (8, 16), (5,), (16, 8))] for _ in range(2)]
    back = lambda **kw: b.opt.gated_ffn_grad(b.TENSORS, b.h, kw.get("kept", kept), kw.get("dy", b.dy), b.weights, kw.get("grads", grads))
    bad(ValueError, lambda: back(kept=(kept[0], kept[1][:1])))
    bad(ValueError, lambda: back(kept=(kept[0], kept[1].float())))
    bad(ValueError, lambda: back(dy=b.dy[..., :4]))
    bad(ValueError, lambda: back(grads=grads[:1]))
    bad(ValueError, lambda: back(grads=[[t.float() for t in row] for row in grads]))
    shared = [list(row) for row in grads]
    shared[1][0] = shared[0][0]
    with pytest.raises(d.DeslocError) as e:
        back(grads=shared)
    assert e.value.status == d.DESLOC_E_INVALID
    # at the entry itself
    status = lambda f: B.raw_lib() and f()
    L, rows = B.raw_lib(), B.rows(b.h.data_ptr(), d.DESLOC_BF16, 32, 8)
    table = B.ptr_array([t.data_ptr() if t is not None else 0 for row in b.weights for t in row])
    f = lambda **kw: B.ffn(*kw.get("tensors", b.TENSORS), kw.get("width", 8), kw.get("hidden", 16), kw.get("tokens", 4), kw.get("weights", table), kw.get("h", rows))
    assert L.desloc_gated_ffn_bytes(b.opt.ctx, f()) > 0
    for kw, want in ((dict(tensors=(0, 0, 1)), d.DESLOC_E_INVALID), (dict(tensors=(0, 3, 9)), d.DESLOC_E_RANGE), (dict(tensors=(0, 3, -1)), d.DESLOC_E_RANGE),
                     (dict(width=0), d.DESLOC_E_RANGE), (dict(width=16), d.DESLOC_E_RANGE), (dict(hidden=8), d.DESLOC_E_RANGE), (dict(tokens=-1), d.DESLOC_E_RANGE),
                     (dict(tokens=(1 << 24) + 1), d.DESLOC_E_RANGE), (dict(weights=None), d.DESLOC_E_NULL), (dict(h=B.rows(0, d.DESLOC_BF16, 32, 8)), d.DESLOC_E_NULL),
                     (dict(h=B.rows(64, d.DESLOC_F32, 32, 8)), d.DESLOC_E_INVALID), (dict(h=B.rows(65, d.DESLOC_BF16, 32, 8)), d.DESLOC_E_INVALID)):
        assert L.desloc_gated_ffn_bytes(b.opt.ctx, f(**kw)) == want, kw
    work = torch.empty(B.desloc_gated_ffn_bytes(b.opt.ctx, f()), dtype=torch.uint8, device="cuda")
    out = B.rows(torch.empty_like(b.h).data_ptr(), d.DESLOC_BF16, 32, 8)
    go = lambda w, n, kg=None, ku=None, to=out: L.desloc_gated_ffn(b.opt.ctx, f(), kg, ku, to, w, n, None)
    assert go(None, 0) == d.DESLOC_E_NULL and go(work.data_ptr() + 16, work.numel()) == d.DESLOC_E_INVALID
    assert go(work.data_ptr(), work.numel() - 1) == d.DESLOC_E_RANGE and go(work.data_ptr(), work.numel(), kg=64) == d.DESLOC_E_NULL
    assert go(work.data_ptr(), work.numel(), to=B.rows(out.data, d.DESLOC_BF16, 32, 4)) == d.DESLOC_E_INVALID


# ---- orthogonalised updates --------------------------------------------------------------------------
DEFAULT = [(3.4445, -4.7750, 2.0315)] * 5


def normal_form(u, eps):
    x = u.double()
    n = torch.linalg.matrix_norm(x)
    return x / (n + eps)


def newton_schulz(u, steps=DEFAULT, eps=1e-7, rounded=False):
    """The definition in 64 bits; `rounded`: with what the kernels round to fp16 rounded there, all else in 64 bits."""
    x = normal_form(u, eps)
    tall = x.shape[0] > x.shape[1]
    x = x.mT if tall else x
    unit, lo = 256.0, 2048.0
    half = lambda v: (v * unit).half().double() / unit if rounded else v
    one = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for k, (a, b, c) in enumerate(steps):
        hi = half(x)
        rest = half((x - hi) * lo) / lo if not rounded or k + 1 < len(steps) else 0.0
        g = half(hi @ hi.mT)
        x = half(a * one + b * g + c * (g @ g)) @ hi + a * rest
    return x.mT if tall else x


def allowed(u, steps=DEFAULT, eps=1e-7):
    """How far a result may be off, over its norm.  The kernels round at the places where `rounded` does, but sums in fp32 come out a little differently, so that single
    values are rounded the other way: that is another draw of the same errors, of twice their size at most; 2^-10 stands for matrices of few values."""
    want = newton_schulz(u, steps, eps)
    norm = float(torch.linalg.matrix_norm(want))
    return want, 2 * float(torch.linalg.matrix_norm(newton_schulz(u, steps, eps, True) - want)) + 2.0 ** -10 * norm


def close(got, want, off):
    assert got.shape == want.shape and bool(torch.isfinite(got).all())
    far = float(torch.linalg.matrix_norm(got.double() - want))
    assert far <= off, f"off by {far:.3e}, {off:.3e} allowed"


def matrices(M, shapes, seed=0, dtype=F32, kind="normal"):
    g = gen_of(seed)
    def one(s):
        if kind == "few":     # three directions and a little noise
            v = torch.randn(s[0], 3, generator=g, device="cuda") @ torch.randn(3, s[1], generator=g, device="cuda") + 1e-3 * torch.randn(s, generator=g, device="cuda")
        else:
            v = torch.randn(s, generator=g, device="cuda")
        return (v * 1e-4).to(dtype)
    return [[one(s) for s in shapes] for _ in range(M)]


SHAPES = [[(1, 1)], [(1, 5), (5, 1)], [(8, 8), (7, 9), (9, 7)], [(72, 72), (24, 72), (200, 72), (72, 200)], [(64, 64), (128, 128), (129, 127)], [(71, 33), (300, 301)],
          [(576, 576), (192, 576), (1536, 576), (576, 1536)], [(1000, 1000), (260, 1030)], [(3, 4000), (4000, 3)],
          [(128, 250), (128, 330), (340, 128), (129, 129), (120, 500), (16, 1600), (1750, 16), (17, 900), (64, 790)]]   # on both sides of what a block takes alone


@pytest.mark.parametrize("shapes", SHAPES)
@pytest.mark.parametrize("src,dst", [("f32", "bf16"), ("bf16", "f32")])
def test_orthogonalize(shapes, src, dst):
    M = 2
    opt = context(M, shapes)
    u = matrices(M, shapes, dtype=TYPE[src])
    out = [[torch.full(s, 7.0, dtype=TYPE[dst], device="cuda") for s in shapes] for _ in range(M)]
    opt.orthogonalize(range(len(shapes)), u, out=out)
    for m, k in itertools.product(range(M), range(len(shapes))):
        want, off = allowed(u[m][k])
        close(out[m][k], want, off + HALF[TYPE[dst]] * float(torch.linalg.matrix_norm(want)))


@pytest.mark.parametrize("shape", [(40, 90), (576, 1536), (300, 100)])
def test_few_directions(shape):
    """Where few directions dominate, the others grow by 3.4 a step, and what was rounded away next to them must not."""
    opt = context(1, [shape])
    u = matrices(1, [shape], kind="few")
    out = [[torch.empty(shape, device="cuda")]]
    opt.orthogonalize([0], u, out=out)
    close(out[0][0], *allowed(u[0][0]))


@pytest.mark.parametrize("grad_dtype", ["bf16", "f32"])
def test_look_ahead_scales_and_coefficients(grad_dtype):
    M, shapes = 3, [(24, 60), (5,), (96, 40), (40, 40)]
    opt = context(M, shapes, grad_dtype, beta1=0.9)
    u = matrices(M, [(24, 60), (5, 1), (96, 40), (40, 40)], 1)
    u = [[t.view(s) for t, s in zip(row, shapes)] for row in u]
    g = [[t.view(s) for t, s in zip(row, shapes)] for row in matrices(M, [(24, 60), (5, 1), (96, 40), (40, 40)], 2, TYPE[grad_dtype])]
    steps = [(1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (3.4445, -4.7750, 2.0315)]
    for scale, factor in (("none", lambda r, c: 1.0), ("aspect", lambda r, c: math.sqrt(max(1.0, r / c))), ("rms", lambda r, c: 0.2 * math.sqrt(max(r, c)))):
        out = [[torch.zeros(s, device="cuda") for s in shapes] for _ in range(M)]
        opt.orthogonalize([3, 0, 2], u, grads=opt.bind_grads(g), out=out, coefficients=steps, scale=scale)
        beta = float(torch.tensor(0.9))
        for m, k in itertools.product(range(M), (0, 2, 3)):
            ahead = beta * u[m][k].double() + (1 - beta) * g[m][k].double()
            want, off = allowed(ahead, steps)
            f = factor(*shapes[k])
            close(out[m][k], want * f, (off + 1e-5 * float(torch.linalg.matrix_norm(want))) * f)
        assert all(bool((row[1] == 0).all()) for row in out)


@pytest.mark.parametrize("shape", [(72, 72), (200, 72), (130, 260), (576, 1536)])
def test_triples_that_change_from_step_to_step(shape):
    """Of large coefficients at first, which take singular values up to two on the way."""
    steps = [(8.3, -23.6, 17.3), (4.1, -2.95, 0.55), (3.95, -2.9, 0.55), (3.3, -2.5, 0.51), (2.3, -1.7, 0.42)]
    opt = context(1, [shape])
    u = matrices(1, [shape], 13)
    out = [[torch.empty(shape, device="cuda")]]
    opt.orthogonalize([0], u, out=out, coefficients=steps)
    close(out[0][0], *allowed(u[0][0], steps))


@pytest.mark.parametrize("shapes", [[(130, 260)] * 5, [(260, 130)] * 5, [(300, 200), (200, 300), (300, 200), (129, 129), (576, 192)], [(40, 24)] * 5])
def test_a_matrix_that_is_not_finite_leaves_the_others_alone(shapes):
    opt = context(1, shapes)
    u = matrices(1, shapes, 14)
    out = [[torch.empty(s, device="cuda") for s in shapes]]
    opt.orthogonalize(range(5), u, out=out)
    was = [t.clone() for t in out[0]]
    u[0][1][3, 5] = math.nan
    u[0][3][-1, -1] = -math.inf
    opt.orthogonalize(range(5), u, out=out)
    assert all(torch.equal(out[0][k], was[k]) for k in (0, 2, 4))
    assert not any(bool(torch.isfinite(out[0][k]).all()) for k in (1, 3))
    u[0][1].zero_()
    opt.orthogonalize(range(5), u, out=out)
    assert all(torch.equal(out[0][k], was[k]) for k in (0, 2, 4)) and bool((out[0][1] == 0).all())


@pytest.mark.parametrize("tall", [True, False])
def test_orthogonalize_beyond_32_bits(tall):
    """2.2e9 elements: rows at both ends against the definition, of which the square matrices are small."""
    long, short = (1 << 20) - 3, 2056
    shape = (long, short) if tall else (short, long)
    opt = context(1, [shape])
    g = gen_of(15)
    u = [[torch.randn(shape, generator=g, device="cuda", dtype=BF)]]
    out = [[torch.empty(shape, device="cuda", dtype=BF)]]
    opt.orthogonalize([0], u, out=out, steps=2)
    x = u[0][0] if tall else u[0][0].mT
    gram = sum(p.double().mT @ p.double() for p in x.split(1 << 16))
    norm = gram.diagonal().sum().sqrt() + 1e-7
    gram, product, (a, b, c) = gram / norm ** 2, torch.eye(short, dtype=torch.float64, device="cuda"), DEFAULT[0]
    for _ in range(2):
        p = a * torch.eye(short, dtype=torch.float64, device="cuda") + b * gram + c * gram @ gram
        product, gram = product @ p, p @ gram @ p
    got = out[0][0] if tall else out[0][0].mT
    for rows in (slice(0, 100), slice(-100, None)):
        # fp16 operands are off by 2^-11, of X, of the polynomial twice a step (its square, itself), and bf16's half step: 2^-7 of the norm is above all of them together
        close(got[rows], x[rows].double() / norm @ product, 2.0 ** -7 * float(torch.linalg.matrix_norm(x[rows].double() / norm @ product)))


def test_in_place_and_flat_tensors():
    M, shape = 2, (48, 100)
    flat = [[t.view(-1) for t in row] for row in matrices(M, [shape], 3)]
    opt = context(M, [(4800,)], u=flat)
    wants = [allowed(row[0].view(shape)) for row in flat]
    opt.orthogonalize([0], flat, columns=[100])
    first = [row[0].clone() for row in flat]
    for t, (want, off) in zip(first, wants):
        close(t.view(shape), want, off)
    for row, new in zip(flat, matrices(M, [shape], 3)):
        row[0].copy_(new[0].view(-1))
    opt.orthogonalize([0], None, columns=[100])       # the context's momentum, in place
    assert all(torch.equal(row[0], t) for row, t in zip(flat, first))


def test_zeros_and_values_that_are_not_finite_stay_where_they_are():
    shapes = [(16, 40)] * 6
    opt = context(1, shapes)
    u = matrices(1, shapes, 4)
    u[0][1].zero_()
    u[0][2][3, 5] = math.nan
    u[0][3][0, 0] = math.inf
    u[0][4][1:] = 0            # rank one
    u[0][5] *= 1e-8            # beside eps
    out = [[torch.full(s, 7.0, dtype=BF, device="cuda") for s in shapes]]
    opt.orthogonalize(range(6), u, out=out)
    assert bool((out[0][1] == 0).all())
    assert not bool(torch.isfinite(out[0][2]).all()) and not bool(torch.isfinite(out[0][3]).all())
    for k in (0, 4, 5):
        want, off = allowed(u[0][k])
        close(out[0][k], want, off + HB * float(torch.linalg.matrix_norm(want)))


@pytest.mark.parametrize("far", [1e-18, 1.0, 1e15])
def test_range_of_the_norm(far):
    opt = context(1, [(40, 24)])
    u = matrices(1, [(40, 24)], 5)
    u[0][0] *= far * 1e4
    out = [[torch.empty(40, 24, device="cuda")]]
    opt.orthogonalize([0], u, out=out, eps=0.0)
    close(out[0][0], *allowed(u[0][0], eps=0.0))


@pytest.mark.parametrize("scale,decay", [("aspect", 0.1), ("none", 0.0)])
def test_orthogonal_step(scale, decay):
    M, shapes = 2, [(64, 24), (7,), (24, 64), (201, 203), (576, 1536)]
    x = [[torch.randn(s, generator=gen_of(9 + m), device="cuda") for s in shapes] for m in range(M)]
    u = [[t.view(s) for t, s in zip(row, shapes)] for row in matrices(M, [s if len(s) == 2 else (s[0], 1) for s in shapes], 6)]
    before = [[t.double() for t in row] for row in x]
    opt = context(M, shapes, x=x, u=u, weight_decay=decay)
    opt.orthogonal_step([0, 2, 3, 4], 0.05, scale=scale)
    lr, wd = float(torch.tensor(0.05)), float(torch.tensor(decay))
    for m, k in itertools.product(range(M), (0, 2, 3, 4)):
        f = math.sqrt(max(1.0, shapes[k][0] / shapes[k][1])) if scale == "aspect" else 1.0
        want, off = allowed(u[m][k])
        total = before[m][k] * (1 - lr * wd) - lr * f * want
        close(x[m][k], total, lr * f * off + 4 * U * float(torch.linalg.matrix_norm(total)))
    assert all(torch.equal(row[1].double(), old[1]) for row, old in zip(x, before))


def test_many_matrices_and_shapes():
    """More matrices than a round takes, more shapes than a launch; the same bits again."""
    shapes = [(8 + k, 16 + (k % 5)) for k in range(40)] + [(16, 16)] * 60
    M = 3
    opt = context(M, shapes)
    u = matrices(M, shapes, 7)
    out, again = ([[torch.zeros(s, dtype=BF, device="cuda") for s in shapes] for _ in range(M)] for _ in range(2))
    opt.orthogonalize(range(len(shapes)), u, out=out)
    opt.orthogonalize(list(range(len(shapes)))[::-1], u, out=again)
    assert all(torch.equal(p, q) for r, s in zip(out, again) for p, q in zip(r, s))
    for m, k in ((0, 0), (1, 17), (2, 39), (2, 99)):
        want, off = allowed(u[m][k])
        close(out[m][k], want, off + HB * float(torch.linalg.matrix_norm(want)))


def test_orthogonal_refusals():
    shapes = [(16, 24), (16, 24), (10,)]
    opt = context(2, shapes)
    u, out = (matrices(2, [(16, 24), (16, 24), (10, 1)], s) for s in (1, 2))
    u, out = ([[t.view(s) for t, s in zip(row, shapes)] for row in v] for v in (u, out))
    for error, call in ((ValueError, lambda: opt.orthogonalize([0, 0], u, out=out)), (ValueError, lambda: opt.orthogonalize([3], u, out=out)),
                        (ValueError, lambda: opt.orthogonalize([2], u, out=out)), (ValueError, lambda: opt.orthogonalize([0], u, out=out, scale="size")),
                        (ValueError, lambda: opt.orthogonalize([0], [[t.double() for t in row] for row in u], out=out)),
                        (ValueError, lambda: opt.orthogonalize([0], u, out=out, grads=u)),
                        (ValueError, lambda: opt.orthogonalize([0], u, out=out, columns=[24, 24])),
                        (ValueError, lambda: opt.orthogonalize([0], u, out=[[t.mT for t in row[:2]] + row[2:] for row in out])),
                        (d.DeslocError, lambda: opt.orthogonalize([0], u, out=out, columns=[7])), (d.DeslocError, lambda: opt.orthogonalize([0], u, out=out, steps=0)),
                        (d.DeslocError, lambda: opt.orthogonalize([0], u, out=out, steps=33)), (d.DeslocError, lambda: opt.orthogonalize([0], u, out=out, eps=-1.0)),
                        (d.DeslocError, lambda: opt.orthogonalize([0], u, out=out, coefficients=[(30.0, -30.0, 0.1)])),
                        (d.DeslocError, lambda: opt.orthogonalize([0], u, out=out, coefficients=[(math.nan, 0.0, 0.0)])),
                        (d.DeslocError, lambda: opt.orthogonal_step([0], math.inf)),
                        (d.DeslocError, lambda: opt.orthogonalize([0, 1], u, out=[[row[0], row[0], row[2]] for row in out])),
                        (d.DeslocError, lambda: opt.orthogonalize([0, 1], u, out=[[row[1], row[0], row[2]] for row in u]))):
        with pytest.raises(error):
            call()
    opt.orthogonalize([], u, out=out)
    opt.orthogonal_step([], 0.1)


# ---- all of them -------------------------------------------------------------------------------------
def test_a_training_step_of_all_of_them():
    """Tokens to embeddings to the block and back, momentum and averages by the step at rate 0, the replicas moved along the orthogonalised look-ahead."""
    M, V, D, F, n, lr = 3, 50, 40, 96, 60, 0.02
    shapes = [(V, D), (F, D), (F, D), (D, F)]
    g = gen_of(11)
    x = [[torch.randn(s, generator=g, device="cuda") * 0.1 for s in shapes] for _ in range(M)]
    opt = context(M, shapes, x=x, beta1=0.9)           # K = (2, 3, 4): at t = 1 nothing is averaged, at t = 2 x is
    momentum = [[torch.zeros(s, dtype=torch.float64, device="cuda") for s in shapes] for _ in range(M)]
    beta = float(torch.tensor(0.9))
    for t in (1, 2):
        tokens = torch.randint(0, V, (M, n), generator=g, device="cuda")
        c = torch.randn(M, n, D, generator=g, device="cuda").to(BF)
        before = [[w.double() for w in row] for row in x]
        weights = [[w.to(BF) for w in row] for row in x]
        h = opt.embed(0, tokens, scale=4.0)
        y, kept = opt.gated_ffn((1, 2, 3), h, weights, keep=True)
        grads = [[torch.zeros(s, dtype=BF, device="cuda") for s in shapes] for _ in range(M)]
        dh = opt.gated_ffn_grad((1, 2, 3), h, kept, c, weights, grads)
        opt.embed_grad(0, tokens, dh, grads, scale=4.0)
        # 64 bits, from the same rounded weights
        for m in range(M):
            leaves = [w.double().requires_grad_() for w in weights[m]]
            table = leaves[0]
            hh = (4.0 * before[m][0][tokens[m]]).requires_grad_()
            z = torch.nn.functional.silu(hh @ leaves[1].mT) * (hh @ leaves[2].mT)
            ((z @ leaves[3].mT) * c[m].double()).sum().backward()
            dtable = torch.zeros_like(table).index_add_(0, tokens[m], 4.0 * hh.grad)
            for got, want in zip(grads[m], [dtable] + [w.grad for w in leaves[1:]]):
                # h, g, u, z, dg, du and the result are rounded to bf16: in norm, no more than the sum of all of those, with silu's and its slope's steepest, 1.1, between
                assert float((got.double() - want).norm()) <= 12 * HB * float(want.norm())
        mask = opt.step(t, 0.0, grads)
        for k in range(4):
            mean, size = sum(row[k] for row in before) / M, sum(row[k].abs() for row in before) / M
            for m in range(M):
                momentum[m][k] = beta * momentum[m][k] + (1 - beta) * grads[m][k].double()
                if mask & d.DESLOC_SYNC_X:
                    before[m][k] = mean
                # (a sum of M values is off by at most M U of the sum of their magnitudes, however small it is itself; the mean by another rounding of 1 / M and of the product)
                check(x[m][k], before[m][k], (M + 3) * U * size + 1e-30)
        opt.orthogonal_step([1, 2, 3], lr, grads=grads, scale="none")
        for m, k in itertools.product(range(M), (1, 2, 3)):
            ahead = beta * momentum[m][k] + (1 - beta) * grads[m][k].double()
            want, off = allowed(ahead)
            # (the momentum itself is fp32: 4 U of it, as the look-ahead's roundings, which no product enlarges by more than 3.5^5)
            close(x[m][k], before[m][k] - lr * want, lr * (off + 8 * U * 3.5 ** 5 * float(want.norm())) + 4 * U * float(before[m][k].norm()))


def test_captured_and_on_another_stream():
    """Captured, replayed on inputs that changed; launched on a side stream behind long work there."""
    b = Block(2, 70, 48, 80)
    kept = [torch.empty(2, 70, 80, dtype=BF, device="cuda") for _ in range(2)]
    grads = [[torch.zeros(s, dtype=BF, device="cuda") for s in ((80, 48), (48, 80), (5,), (80, 48))] for _ in range(2)]
    u = matrices(2, [(80, 48), (48, 80), (5, 1), (80, 48)], 8)
    u = [[t.view(s) for t, s in zip(row, ((80, 48), (48, 80), (5,), (80, 48)))] for row in u]
    out = [[torch.zeros_like(t) for t in row] for row in u]

    def run():
        y, k = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)
        for to, t in zip(kept, k):
            to.copy_(t)
        dh = b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, grads)
        b.opt.orthogonalize([0, 1, 3], u, out=out)
        return [y, dh] + [row[k] for row in grads for k in (0, 1, 3)] + [row[k] for row in out for k in (0, 1, 3)]

    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for seed in (20, 21):
        b.h.copy_(torch.randn(b.h.shape, generator=gen_of(seed), device="cuda"))
        for row in u:
            row[0].copy_(torch.randn(row[0].shape, generator=gen_of(seed), device="cuda"))
        graph.replay()
        replayed = [t.clone() for t in captured]
        assert all(torch.equal(p, q) for p, q in zip(replayed, run()))
    want = [t.clone() for t in run()]
    new = torch.randn(b.h.shape, generator=gen_of(30), device="cuda").to(BF)
    old = b.h.clone()
    side, long = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    b.h.copy_(new)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            long = long @ long * 1e-3
        b.h.copy_(old)
        got = run()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))


@pytest.mark.parametrize("tokens,width,hidden,shape", [(300, 64, 512, (300, 500)), (1024, 512, 1024, (1024, 2048)), (8, 2048, 64, (60, 90))])
@pytest.mark.parametrize("polls", [0, 2, 30])
def test_a_wait_that_runs_out_is_reported(tokens, width, hidden, shape, polls):
    """No poll at all, or so few that some blocks give up in the middle: the calls end, the context says so, and the next ones are right."""
    b = Block(2, tokens, width, hidden)
    opt = context(1, [shape])
    u = matrices(1, [shape])
    out = [[torch.empty(shape, device="cuda")]]
    for o, call in ((b.opt, lambda: b.opt.gated_ffn(b.TENSORS, b.h, b.weights)), (opt, lambda: opt.orthogonalize([0], u, out=out))):
        call()
        torch.cuda.synchronize()
        B.desloc_testing_set_wait_limit(o.ctx, polls)
        call()
        torch.cuda.synchronize()
        try:
            call()
            assert polls > 0
        except d.DeslocError as e:
            assert e.status == d.DESLOC_E_DEVICE_WAIT
        torch.cuda.synchronize()
        B.desloc_testing_set_wait_limit(o.ctx, -1)
    want, tol = b.forward(b.h)
    check(b.opt.gated_ffn(b.TENSORS, b.h, b.weights), want[2], tol[2])
    opt.orthogonalize([0], u, out=out)
    close(out[0][0], *allowed(u[0][0]))


def test_what_is_written_counts_as_changed():
    b = Block(1, 8, 16, 24)
    kept = b.opt.gated_ffn(b.TENSORS, b.h, b.weights, keep=True)[1]
    grads = [[torch.zeros(s, dtype=BF, device="cuda") for s in ((24, 16), (16, 24), (5,), (24, 16))]]
    out = torch.empty_like(b.h)
    versions = lambda: [t._version for t in (out, *grads[0])]
    was = versions()
    b.opt.gated_ffn(b.TENSORS, b.h, b.weights, out=out)
    b.opt.gated_ffn_grad(b.TENSORS, b.h, kept, b.dy, b.weights, grads)
    now = versions()
    assert now[0] > was[0] and all(now[1 + k] > was[1 + k] for k in b.TENSORS) and now[3] == was[3]
    u = matrices(1, [(24, 16), (16, 24)], 1)
    opt = context(1, [(24, 16), (16, 24)], x=matrices(1, [(24, 16), (16, 24)], 2))
    was = [t._version for t in (*u[0], *opt._keep[0][0])]
    opt.orthogonalize([1], u)
    opt.orthogonal_step([0], 0.1, updates=u)
    now = [t._version for t in (*u[0], *opt._keep[0][0])]
    assert [n > w for n, w in zip(now, was)] == [False, True, True, False]
