"""Layer norm, forward and backward, against the formulas in 64 bits.

Tolerances, element by element: half a step of the stored type relative to the
value, and float32's arithmetic.  A sum over a row is at most CH additions deep
for any one element (the elements of a lane, then the exchanges between
lanes), so it is off by at most CH 2^-24 of the sum of its terms' sizes."""
import pytest
import torch

import paper_2212_14052_amd as h3

pytestmark = pytest.mark.gpu
E32 = 2.0 ** -24
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# one element, widths that divide nothing, each way that a row is laid over threads, rows wider than the registers
SHAPES = [(1, 1), (3, 2), (7, 63), (5, 64), (1, 257), (130, 768), (64, 1031), (33, 2056), (9, 2560), (4, 5120),
          (2, 9000), (3, 40000), (2, 33001)]


def chain(d):
    return min(d, 64 + d // 1024)


def half_step(ref, dt):
    return ref.abs() * torch.finfo(dt).eps / 2 + (2.0 ** -25 if dt is torch.float16 else 0.0)


def inputs(rows, d, dtype, seed=0, offset=0.5):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, d, generator=gen) + offset) * torch.empty(rows, 1).uniform_(0.2, 3.0, generator=gen)
    dy = torch.randn(rows, d, generator=gen)
    w, b = 1 + 0.2 * torch.randn(d, generator=gen), 0.1 * torch.randn(d, generator=gen)
    return [t.to(DTYPES[dtype]).cuda() for t in (x, dy)] + [w.cuda(), b.cuda()]


def stats64(x, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    r = ((x - mean) ** 2).mean(-1, keepdim=True).add(eps).rsqrt()
    return mean, r, (x - mean) * r


def check_fwd(x, w, b, eps, got):
    y, mean, rstd = got
    m, r, xh = stats64(x, eps)
    one = torch.ones((), dtype=torch.float64, device=x.device)
    wd, bd = (one if w is None else w.double()), (0 * one if b is None else b.double())
    ch, A = chain(x.shape[-1]), x.double().abs().amax(-1, keepdim=True) * r
    ref = xh * wd + bd
    tol = half_step(ref, y.dtype) + E32 * (ch * wd.abs() * (2 * A + xh.abs()) + 4 * (ref.abs() + bd.abs()))
    assert ((y.double() - ref).abs() <= tol).all()
    assert ((mean.double() - m[..., 0]).abs() <= E32 * ch * (A / r)[..., 0]).all()
    assert ((rstd.double() - r[..., 0]).abs() <= E32 * (ch + 8) * r[..., 0] * (1 + A[..., 0] * E32 * ch * A[..., 0])).all()


def check_bwd(dy, x, w, eps, got):
    dx, dw, db = got
    m, r, h = stats64(x, eps)
    g = dy.double()
    t = g * (1.0 if w is None else w.double())
    ch, A = chain(x.shape[-1]), x.double().abs().amax(-1, keepdim=True) * r
    dh = E32 * ch * (2 * A + h.abs())   # how far a normalised value may be off
    m0, m1 = t.mean(-1, keepdim=True), (t * h).mean(-1, keepdim=True)
    if dx is not None:
        ref = r * (t - m0 - h * m1)
        a0, a1 = t.abs().mean(-1, keepdim=True), (t * h).abs().mean(-1, keepdim=True)
        off1 = E32 * (ch + 4) * a1 + (t.abs() * dh).mean(-1, keepdim=True)
        tol = half_step(ref, dx.dtype) + r * (E32 * (ch + 4) * (a0 + t.abs() + h.abs() * m1.abs()) + h.abs() * off1 + dh * (m1.abs() + off1))
        assert ((dx.double() - ref).abs() <= tol).all()
    rows = x.shape[0]
    if dw is not None:
        tol = E32 * (min(rows, 64 + rows // 256) + 4) * (g * h).abs().sum(0) + (g.abs() * dh).sum(0)
        assert ((dw.double() - (g * h).sum(0)).abs() <= tol).all()
    if db is not None:
        assert ((db.double() - g.sum(0)).abs() <= E32 * min(rows, 64 + rows // 256) * g.abs().sum(0)).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,d", SHAPES)
def test_forward_and_backward(rows, d, dtype):
    x, dy, w, b = inputs(rows, d, dtype)
    y, mean, rstd = h3.layernorm(x, w, b, 1e-5)
    check_fwd(x, w, b, 1e-5, (y, mean, rstd))
    check_bwd(dy, x, w, 1e-5, h3.layernorm_bwd(dy, x, w, mean, rstd))


@pytest.mark.parametrize("rows,d", [(5000, 96), (3001, 520), (1100, 2560)])
def test_many_rows(rows, d):
    """More rows than a launch's workgroups hold at once."""
    x, dy, w, b = inputs(rows, d, "bf16", 1)
    y, mean, rstd = h3.layernorm(x, w, b)
    check_fwd(x, w, b, 1e-5, (y, mean, rstd))
    check_bwd(dy, x, w, 1e-5, h3.layernorm_bwd(dy, x, w, mean, rstd))


def test_far_from_zero():
    """A mean a thousand times the spread: squares would cancel."""
    x, dy, w, b = inputs(50, 512, "f32", 2, offset=1000.0)
    got = h3.layernorm(x, w, b)
    check_fwd(x, w, b, 1e-5, got)
    check_bwd(dy, x, w, 1e-5, h3.layernorm_bwd(dy, x, w, *got[1:]))


def test_without_weight_and_bias_and_single_gradients():
    x, dy, w, b = inputs(37, 200, "f16", 3)
    got = h3.layernorm(x)
    check_fwd(x, None, None, 1e-5, got)
    for want in ((True, False, False), (False, True, False), (False, False, True), (False, True, True)):
        r = h3.layernorm_bwd(dy, x, None, *got[1:], *want)
        assert [t is not None for t in r] == list(want)
        check_bwd(dy, x, None, 1e-5, r)


def test_leading_shape_strides_and_alignment():
    """(B, L, d) rows, a transposed view, and rows that start 2 bytes off a 16-byte boundary."""
    x, dy, w, b = inputs(60, 256, "bf16", 4)
    flat = h3.layernorm(x, w, b)
    y, mean, rstd = h3.layernorm(x.view(3, 20, 256), w, b)
    assert y.shape == (3, 20, 256) and mean.shape == (3, 20) and torch.equal(y.view(60, 256), flat[0])
    turned = x.view(3, 20, 256).transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(h3.layernorm(turned, w, b)[0], y)
    off = torch.empty(60 * 256 + 1, dtype=x.dtype, device="cuda")[1:].view(60, 256)
    off.copy_(x)
    got = h3.layernorm(off, w, b)
    check_fwd(x, w, b, 1e-5, got)
    check_bwd(dy, x, w, 1e-5, h3.layernorm_bwd(dy, off, w, *got[1:]))


def test_in_place_and_out():
    x, dy, w, b = inputs(40, 768, "bf16", 5)
    y, mean, rstd = h3.layernorm(x, w, b)
    x2 = x.clone()
    assert h3.layernorm(x2, w, b, out=x2)[0] is x2 and torch.equal(x2, y)


def test_not_finite_and_constant_rows():
    """A row with an Inf or a NaN does not reach others; a constant row gives the bias."""
    x, dy, w, b = inputs(20, 300, "f32", 6)
    ref = h3.layernorm(x, w, b)[0].clone()
    x[3, 7], x[5, 9], x[8] = float("inf"), float("nan"), 2.5
    y, mean, rstd = h3.layernorm(x, w, b)
    assert not torch.isfinite(y[3]).all() and torch.isnan(y[5]).all()
    assert torch.equal(y[8], b)   # its deviations are exact zeros: 2.5 is summed exactly
    keep = [i for i in range(20) if i not in (3, 5, 8)]
    assert torch.equal(y[keep], ref[keep])


def test_repeats_bit_for_bit_and_in_a_graph():
    x, dy, w, b = inputs(700, 768, "f16", 7)

    def call():
        y, mean, rstd = h3.layernorm(x, w, b)
        return (y, mean, rstd) + h3.layernorm_bwd(dy, x, w, mean, rstd)

    want = [t.clone() for t in call()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        assert all(torch.equal(p, q) for p, q in zip(call(), want))


def test_gradient_against_differences():
    gen = torch.Generator().manual_seed(8)
    x, dy = torch.randn(4, 24, generator=gen).cuda(), torch.randn(4, 24, generator=gen).cuda()
    w, b = torch.randn(24, generator=gen).cuda(), torch.randn(24, generator=gen).cuda()
    y, mean, rstd = h3.layernorm(x, w, b)
    dx, dw, db = h3.layernorm_bwd(dy, x, w, mean, rstd)
    # central differences at 2^-6: y's float32 error (a few 2^-24 of values of a few) over 2^-5 is under 1e-4 a term of
    # the sum, the third derivative's term h^2 / 6 y''' is of the order 1e-4 r^3: 5e-3 of the gradient's size covers both
    h = 2.0 ** -6
    for t, grad in ((x, dx), (w, dw), (b, db)):
        flat, num = t.view(-1), torch.empty_like(t).view(-1)
        for i in range(0, flat.numel(), 5):
            at = flat[i].item()
            flat[i] = at + h
            up = (h3.layernorm(x, w, b)[0].double() * dy.double()).sum().item()
            flat[i] = at - h
            down = (h3.layernorm(x, w, b)[0].double() * dy.double()).sum().item()
            flat[i] = at
            num[i] = (up - down) / (2 * h)
            assert abs(num[i].item() - grad.view(-1)[i].item()) <= 5e-3 * max(1.0, grad.abs().max().item())
