"""The residual's addition with the RMS norm behind it, and its gradient, against the formula in 64 bits.

Bounds: a fp32 sum over a row of d values is off by at most d 2^-24 of the sum
of absolute values, so the norm's factor by (d + 8) 2^-24 of itself (a root and
a quotient of 2 ulp each); each output is rounded once to its type. The
weight's gradient sums T rows in fp32.
"""
import pytest
import torch

from paper_2607_20652_gb300 import build, dpb

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build()
    dpb.load()


def ulp(t):
    return 2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -24


def draw(T, d, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return (n(T, d) * 2).to(dtype), n(T, d).to(dtype), (1 + 0.3 * n(d)).to(dtype), n(T, d).to(dtype), n(T, d).to(dtype)


def formula(s, w, eps=EPS):
    return s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps) * (1.0 if w is None else w)


def check(got, want, size):
    tol = size + ulp(got) * want.abs() + 1e-30
    off = ((got.double() - want).abs() / tol).nan_to_num(1e9).max() if got.numel() else torch.zeros(())
    assert float(off) <= 1, float(off)


def check_forward(y, total, w, eps=EPS):
    want = formula(total.double(), None if w is None else w.double(), eps)
    check(y, want, (total.shape[1] + 8) * 2.0 ** -24 * want.abs())


def check_gradient(dx, dw, total, w, dy, dtotal, eps=EPS):
    T, d = total.shape
    s = total.double().requires_grad_()
    wd = (torch.ones(d, device="cuda") if w is None else w).double().requires_grad_()
    gx, gw = torch.autograd.grad(formula(s, wd, eps), (s, wd), dy.double())
    s, r = s.detach().abs(), torch.rsqrt((s * s).mean(-1, keepdim=True) + eps).detach()
    u = (dy.double() * wd).detach().abs()
    size = r * u + r ** 3 * s * (u * s).mean(-1, keepdim=True)
    rest = 0 if dtotal is None else dtotal.double()
    check(dx, gx + rest, 4 * (d + 12) * 2.0 ** -24 * size + 2.0 ** -23 * (rest if dtotal is None else rest.abs()))
    if dw is not None:
        check(dw, gw, (T + d + 12) * 2.0 ** -24 * (dy.double().abs() * s * r).sum(0))


SIZES = [(1, 1), (1, 8), (5, 7), (128, 64), (33, 100), (300, 768), (65, 1000), (7, 1032), (40, 1025), (9, 2048), (12, 2050),
         (3, 4100), (5, 4096), (4, 8200), (3, 8192), (2, 16384), (2, 16383), (5000, 24), (20000, 520), (70003, 64), (1001, 40),
         (2777, 16), (99991, 8), (333, 4), (4099, 3), (1234, 128), (3001, 256)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d", SIZES)
def test_norm_and_gradient(T, d, dtype):
    x, delta, w, dy, dt = draw(T, d, dtype, seed=T + d)
    y, total = dpb.add_norm(x, delta, w, EPS)
    assert torch.equal(total, x + delta)
    check_forward(y, total, w)
    check_gradient(*dpb.add_norm_backward(total, dy, dt, w, EPS), total, w, dy, dt)
    # without the residual, without a weight
    y, same = dpb.add_norm(x, eps=EPS)
    assert same is x
    check_forward(y, x, None)
    dx, dw = dpb.add_norm_backward(x, dy, eps=EPS)
    check_gradient(dx, dw, x, None, dy, None)
    again, none = dpb.add_norm_backward(x, dy, eps=EPS, weight_grad=False)
    assert none is None and torch.equal(again, dx)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_rows(dtype):
    x, delta, w, dy, dt = draw(0, 24, dtype)
    y, total = dpb.add_norm(x, delta, w)
    assert y.shape == total.shape == (0, 24)
    dx, dw = dpb.add_norm_backward(total, dy, dt, w)
    assert dx.shape == (0, 24) and not dw.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,stride,first", [(24, 40, 8), (24, 33, 0), (768, 770, 2), (7, 9, 1), (64, 128, 64), (1000, 1001, 3)])
def test_strides_and_addresses(d, stride, first, dtype):
    T = 70
    x, delta, w, dy, dt = draw(T, d, dtype)

    def wide(t=None):
        flat = torch.full((T * stride + first,), 3.0, device="cuda", dtype=dtype)
        v = flat.as_strided((T, d), (stride, 1), first)
        if t is not None:
            v.copy_(t)
        return flat, v

    out, total = wide(), wide()
    dpb.add_norm(wide(x)[1], wide(delta)[1], w, EPS, out=out[1], total=total[1])
    assert torch.equal(total[1], x + delta)
    check_forward(out[1], total[1], w)
    grad = wide()
    _, dw = dpb.add_norm_backward(total[1], wide(dy)[1], wide(dt)[1], w, EPS, grad_x=grad[1])
    check_gradient(grad[1], dw, total[1], w, dy, dt)
    inside = torch.zeros(T * stride + first, dtype=torch.bool, device="cuda")
    inside.as_strided((T, d), (stride, 1), first)[:] = True
    for flat, _ in (out, total, grad):
        assert (flat[~inside] == 3).all()
    # a weight at an odd address
    odd = torch.empty(d + 1, device="cuda", dtype=dtype)[1:].copy_(w)
    check_forward(dpb.add_norm(x, delta, odd, EPS)[0], x + delta, w)


def test_in_place():
    x, delta, w, dy, dt = draw(300, 264, torch.bfloat16)
    y, total = dpb.add_norm(x, delta, w)
    a, b = x.clone(), delta.clone()
    dpb.add_norm(a, b, w, out=b, total=a)
    assert torch.equal(a, total) and torch.equal(b, y)
    want, dw = dpb.add_norm_backward(total, dy, dt, w)
    for i in range(3):
        rows = [t.clone() for t in (total, dy, dt)]
        got, dw2 = dpb.add_norm_backward(*rows, w, grad_x=rows[i])
        assert torch.equal(got, want) and torch.equal(dw, dw2)


def test_rows_of_zeros_and_what_is_not_finite():
    x, _, w, dy, _ = draw(64, 100, torch.float32)
    x[3] = 0
    y, _ = dpb.add_norm(x, weight=w)
    assert not y[3].any()
    check_gradient(*dpb.add_norm_backward(x, dy, weight=w), x, w, dy, None)
    want = dpb.add_norm_backward(x, dy, weight=w)[0]
    x[5], dy[9] = float("nan"), float("inf")
    y2, _ = dpb.add_norm(x, weight=w)
    keep = (torch.arange(64, device="cuda") != 5)
    assert torch.equal(y2[keep], y[keep]) and y2[5].isnan().all()
    dx, dw = dpb.add_norm_backward(x, dy, weight=w)
    keep[9] = False
    assert torch.equal(dx[keep], want[keep]) and not dw.isfinite().any()


def test_eps_of_zero():
    x, _, w, dy, _ = draw(64, 100, torch.float32)
    check_forward(dpb.add_norm(x, weight=w, eps=0.0)[0], x, w, 0.0)
    check_gradient(*dpb.add_norm_backward(x, dy, weight=w, eps=0.0), x, w, dy, None, 0.0)


def test_gradient_against_differences():
    """f(x + s) - f(x - s) over 2, s of 2^-10: f is smooth where the row's rms is near 2, third derivatives below 10 r^3."""
    x, _, w, dy, dt = draw(20, 50, torch.float32)
    dx, dw = dpb.add_norm_backward(x, dy, dt, w)
    g = torch.Generator(device="cuda").manual_seed(9)
    s = torch.randn(20, 50, generator=g, device="cuda") * 2.0 ** -10

    def f(x, w):
        y, total = dpb.add_norm(x, torch.zeros_like(x), w)
        return (y.double() * dy.double()).sum() + (total.double() * dt.double()).sum()

    got, want = float(f(x + s, w) - f(x - s, w)) / 2, float((dx.double() * s.double()).sum())
    size = float((dy.double() * formula(x.double(), w.double())).abs().sum() + (dt.double() * x.double()).abs().sum())
    assert abs(got - want) <= 60 * 2.0 ** -24 * size + 10 * 2.0 ** -30 * float(dy.double().abs().sum())
    v = torch.randn(50, generator=g, device="cuda") * 2.0 ** -6
    got, want = float(f(x, w + v) - f(x, w - v)) / 2, float((dw.double() * v.double()).sum())
    assert abs(got - want) <= 60 * 2.0 ** -24 * size  # linear in w


def test_equal_bits_another_stream_and_a_graph():
    x, delta, w, dy, dt = draw(9000, 264, torch.bfloat16)
    y, total = dpb.add_norm(x, delta, w)
    dx, dw = dpb.add_norm_backward(total, dy, dt, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = (*dpb.add_norm(x, delta, w, stream=s), *dpb.add_norm_backward(total, dy, dt, w, stream=s))
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, total, dx, dw), got))
    graph = torch.cuda.CUDAGraph()
    xx = torch.zeros_like(x)
    with torch.cuda.graph(graph):
        y2, t2 = dpb.add_norm(xx, delta, w)
        dx2, dw2 = dpb.add_norm_backward(t2, dy, dt, w)
    xx.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((y, total, dx, dw), (y2, t2, dx2, dw2)))


def test_refusals():
    x, delta, w, dy, dt = draw(30, 24, torch.float32)
    for bad in (dict(x=x.half()), dict(delta=delta.bfloat16()), dict(delta=delta[:20]), dict(weight=w[:20]), dict(weight=w.bfloat16()),
                dict(x=x[0]), dict(x=x[:, ::2]), dict(out=delta[:20]), dict(total=delta.bfloat16()), dict(eps=-1.0),
                dict(eps=float("nan")), dict(delta=delta.cpu())):
        with pytest.raises((ValueError, dpb.DPBError)):
            dpb.add_norm(**(dict(x=x, delta=delta, weight=w) | bad))
    for bad in (dict(total=x.half()), dict(grad_out=dy[:20]), dict(grad_total=dt.bfloat16()), dict(weight=w[:20]),
                dict(grad_x=dy[:, :20]), dict(eps=-1.0), dict(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, dpb.DPBError)):
            dpb.add_norm_backward(**(dict(total=x, grad_out=dy, grad_total=dt, weight=w) | bad))
    big = torch.zeros(2, 16385, device="cuda")
    with pytest.raises(dpb.DPBError):
        dpb.add_norm(big)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 50, 768, 4101])
@pytest.mark.parametrize("rms,eps", [(1e14, EPS), (1e15, EPS), (1e17, EPS), (1e-13, 0.0), (1e-14, 0.0), (1e-17, 0.0)])
def test_gradient_of_large_and_of_small_rows(rms, eps, d, dtype):
    """r^3 leaves fp32 here, the gradient does not: sums of squares stay between 1e-33 and 5e37. The gradient that comes
    leans along the row, so that its mean product with the row counts."""
    x, _, w, dy, dt = draw(20, d, dtype, seed=d)
    dy = (dy.double() + x.double()).to(dtype)
    x = (x.double() * (rms / 2)).to(dtype)
    check_gradient(*dpb.add_norm_backward(x, dy, None, w, eps), x, w, dy, None, eps)
    dt = (dt.double() / rms).to(dtype)
    check_gradient(*dpb.add_norm_backward(x, dy, dt, w, eps), x, w, dy, dt, eps)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_of_zeros_with_a_small_eps(dtype):
    """r = 1e15 and more, r^3 beyond fp32: without a row only r u is left."""
    x, _, w, dy, dt = draw(12, 64, dtype)
    x[::3] = 0
    for eps in (1e-26, 1e-30, 1e-36):
        check_gradient(*dpb.add_norm_backward(x, dy, dt, w, eps), x, w, dy, dt, eps)


def test_offsets_past_32_bits():
    """2^31 values and more: 512 times the same rows, each time the same bits."""
    T, d, n = 4099, 1024, 512
    x, delta, w, dy, dt = draw(T, d, torch.bfloat16)
    y0, total0 = dpb.add_norm(x, delta, w)
    dx0, dw0 = dpb.add_norm_backward(total0, dy, dt, w)
    many = lambda t: t.repeat(n, 1)  # noqa: E731
    y, total = dpb.add_norm(many(x), many(delta), w)
    assert y.numel() > 2 ** 31
    assert (y.view(n, T, d) == y0).all() and (total.view(n, T, d) == total0).all()
    del y
    dx, dw = dpb.add_norm_backward(total, many(dy), many(dt), w)
    assert (dx.view(n, T, d) == dx0).all()
    # fp32 sums of some 4000 rows a block and warp, of at most 608 blocks in 32 chains and 5 joins of these
    r = torch.rsqrt(total0.double().square().mean(-1, keepdim=True) + EPS)
    size = (dy.double() * total0.double() * r).abs().sum(0) * n
    assert ((dw.double() - dw0.double() * n).abs() <= (4000 + 19 + 5 + d + 12) * 2.0 ** -23 * size).all()
