"""Norm and rotation of query and key heads against the formula in 64 bits.

Bounds: fp32 arithmetic over a head of D values is off by at most (D + 12)
2^-24 of the sums of absolute values; bf16 outputs (8 bits) are rounded once
more, by at most 2^-8 of themselves.
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


def formula(x, w, cos, sin, pos, rot, interleaved, normalise=True):
    """The rotation as complex numbers, differentiable."""
    n = x
    if normalise:
        n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * (1.0 if w is None else w)
    if not rot:
        return n
    turn = torch.complex(cos.double(), sin.double())[pos.long()][:, None]
    head = n[..., :rot].unflatten(-1, (rot // 2, 2)) if interleaved else \
        n[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2)
    y = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
    y = y if interleaved else y.transpose(-1, -2)
    return torch.cat([y.flatten(-2), n[..., rot:]], -1)


def draw(T, H, Hk, D, rot, dtype, seed=0, P=300):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = torch.randn(T, H + 2 * Hk, D, generator=g, device="cuda").mul_(2).to(dtype)
    w = [(1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dtype) for _ in range(2)]
    cos, sin = dpb.rope_tables(P, rot) if rot else (None, None)
    pos = torch.randint(0, P, (T,), generator=g, device="cuda", dtype=torch.int32)
    gy = [torch.randn(T, h, D, generator=g, device="cuda").to(dtype) for h in (H, Hk)]
    return qkv[:, :H], qkv[:, H:H + Hk], w, cos, sin, pos, gy


def close(got, want, size, D, extra=1.0):
    """size: the sum of absolute values that the result is a sum of."""
    u = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    tol = extra * (D + 12) * 2.0 ** -24 * size + u * want.abs() + 1e-30
    off = ((got.double() - want).abs() / tol).max() if got.numel() else torch.zeros(())
    assert float(off) <= 1, float(off)


SHAPES = [  # tokens, q heads, k heads, dim, rotated, interleaved
    (1, 1, 1, 64, 64, False), (37, 12, 12, 64, 64, False), (300, 16, 4, 128, 96, True), (65, 4, 4, 16, 16, True),
    (20, 5, 3, 24, 8, False), (33, 3, 1, 128, 20, False), (50, 2, 2, 30, 30, True), (17, 7, 2, 96, 2, False),
    (9, 3, 0, 64, 64, True), (12, 40, 9, 256, 256, False), (1000, 2, 1, 8, 8, False), (64, 4, 4, 64, 0, False),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H,Hk,D,rot,inter", SHAPES)
def test_forward_and_gradient(T, H, Hk, D, rot, inter, dtype):
    q, k, w, cos, sin, pos, gy = draw(T, H, Hk, D, rot, dtype, seed=D + rot)
    at = dict(weight_q=w[0], weight_k=w[1], cos=cos, sin=sin, positions=pos if rot else None, eps=EPS, interleaved=inter)
    y = dpb.qk_norm_rope(q, k, **at)
    dx = dpb.qk_norm_rope_backward(q, k, *gy, **at)
    for i, x in enumerate((q, k)):
        xd, wd = x.double().requires_grad_(), w[i].double().requires_grad_()
        want = formula(xd, wd, cos, sin, pos, rot, inter)
        size = (xd / torch.sqrt((xd * xd).mean(-1, keepdim=True) + EPS) * wd).detach().abs().amax(-1, keepdim=True) * 2
        close(y[i], want.detach(), size, D)
        gx, gw = torch.autograd.grad(want, (xd, wd), gy[i].double())
        r = torch.rsqrt((xd * xd).mean(-1, keepdim=True) + EPS).detach()
        n = xd.detach().abs() * r
        u = 2 * gy[i].double().abs().amax(-1, keepdim=True) * wd.detach().abs().amax()
        close(dx[i], gx, r * (u + n * (u * n).mean(-1, keepdim=True)), D, extra=2)
        close(dx[2 + i], gw, (2 * gy[i].double().abs().amax(-1, keepdim=True) * n).sum((0, 1)), D, extra=T * H / D + 2)
    assert dpb.status() == 0


@pytest.mark.parametrize("rot,inter", [(64, False), (64, True), (48, False)])
def test_unaligned_rows_and_in_place(rot, inter):
    """Rows at odd addresses take the scalar accesses and give the same bits as aligned ones."""
    T, H, D = 45, 3, 64
    q, k, w, cos, sin, pos, _ = draw(T, H, H, D, rot, torch.bfloat16, seed=2)
    at = dict(weight_q=w[0], weight_k=w[1], cos=cos, sin=sin, positions=pos, interleaved=inter)
    y = dpb.qk_norm_rope(q, k, **at)
    odd = torch.empty(T * H * (D + 1) + 1, dtype=torch.bfloat16, device="cuda")[1:].view(T, H, D + 1)[:, :, :D]
    odd.copy_(q)
    z = dpb.qk_norm_rope(odd, k, **at)
    for a, b in zip(y, z):
        assert float((a.double() - b.double()).abs().max()) <= 2.0 ** -8 * float(a.abs().max())
    q2, k2 = q.clone(), k.clone()
    dpb.qk_norm_rope(q2, k2, **at, q_out=q2, k_out=k2)
    assert torch.equal(q2, y[0]) and torch.equal(k2, y[1])


def test_rotation_alone_and_back():
    """Without a norm the gradient is the rotation the other way: the two undo each other."""
    q, k, _, cos, sin, pos, _ = draw(70, 4, 2, 64, 64, torch.float32, seed=3)
    at = dict(cos=cos, sin=sin, positions=pos, normalise=False)
    y = dpb.qk_norm_rope(q, k, **at)
    close(y[0], formula(q.double(), None, cos, sin, pos, 64, False, False), q.double().abs().amax() * 2, 64)
    back = dpb.qk_norm_rope_backward(q, k, *y, **at)
    assert back[2] is None and back[3] is None
    for a, b in zip(back, (q, k)):
        # cos^2 + sin^2 is 1 within 2^-23, four products and two sums each way
        assert float((a - b).abs().max()) <= 16 * 2.0 ** -23 * float(b.abs().max())


def test_gradient_against_differences():
    T, H, D = 20, 2, 64
    q, k, w, cos, sin, pos, gy = draw(T, H, H, D, 64, torch.float32, seed=4)
    at = dict(weight_q=w[0], weight_k=w[1], cos=cos, sin=sin, positions=pos, eps=EPS)
    dq, _, dwq, _ = dpb.qk_norm_rope_backward(q, k, *gy, **at)
    g = torch.Generator(device="cuda").manual_seed(5)

    def loss(x, wx):
        return float((formula(x, wx, cos, sin, pos, 64, False) * gy[0].double()).sum())

    for x, grad, f in ((q, dq, lambda z: loss(z, w[0].double())), (w[0], dwq, lambda z: loss(q.double(), z))):
        d = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        diff = (f(x.double() + h * d) - f(x.double() - h * d)) / (2 * h)
        size = float((grad.double() * d).abs().sum())
        assert abs(float((grad.double() * d).sum()) - diff) <= 1e-5 * size


def test_zero_rows_and_weight_sums_of_nothing():
    q = torch.zeros((5, 2, 64), device="cuda")
    cos, sin = dpb.rope_tables(8, 64)
    y, _ = dpb.qk_norm_rope(q, q, cos=cos, sin=sin)
    assert not y.any()
    dq, dk, dwq, dwk = dpb.qk_norm_rope_backward(q, q, q + 1, q + 1, cos=cos, sin=sin)
    assert torch.isfinite(dq).all() and not dwq.any() and not dwk.any()
    e = q[:0]
    out = dpb.qk_norm_rope_backward(e, e, e, e, cos=cos, sin=sin)
    assert out[0].shape == e.shape and not out[2].any() and not out[3].any()


def test_equal_inputs_give_equal_bits():
    q, k, w, cos, sin, pos, gy = draw(5000, 12, 4, 64, 64, torch.bfloat16, seed=6)
    at = dict(weight_q=w[0], weight_k=w[1], cos=cos, sin=sin, positions=pos)
    one, two = (dpb.qk_norm_rope_backward(q, k, *gy, **at) for _ in range(2))
    assert all(torch.equal(a, b) for a, b in zip(one, two))


def test_bad_position_is_flagged():
    q, k, _, cos, sin, pos, _ = draw(40, 2, 2, 64, 64, torch.float32, seed=7)
    pos[3], pos[9] = -1, 300
    dpb.status()
    y, _ = dpb.qk_norm_rope(q, k, cos=cos, sin=sin, positions=pos)
    assert dpb.status() == dpb.DEV_BAD_LENGTH
    n = formula(q.double(), None, None, None, None, 0, False)
    for t in (3, 9):  # normalised, not rotated
        assert torch.allclose(y[t].double(), n[t], rtol=1e-5, atol=1e-6)


def test_offsets_that_pass_32_bits():
    T, ts = 150, 1 << 24
    buf = torch.empty(T * ts, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((T, 1, 64), (ts, 64, 1))
    q, k, w, cos, sin, pos, gy = draw(T, 1, 1, 64, 64, torch.bfloat16, seed=8)
    far.copy_(q)
    at = dict(weight_q=w[0], weight_k=w[1], cos=cos, sin=sin, positions=pos)
    one, two = dpb.qk_norm_rope(q, k, **at), dpb.qk_norm_rope(far, k, **at)
    assert torch.equal(one[0], two[0])


def test_tables():
    cos, sin = dpb.rope_tables(50, 16, base=500.0)
    i, p = torch.arange(8, dtype=torch.float64), torch.arange(50, dtype=torch.float64)
    ang = p[:, None] * 500.0 ** (-2 * i / 16)
    assert torch.allclose(cos.cpu().double(), ang.cos(), atol=1e-7) and torch.allclose(sin.cpu().double(), ang.sin(), atol=1e-7)
    lin, _ = dpb.rope_tables(100, 16, base=500.0, scaling="linear", factor=2.0)
    assert torch.allclose(lin[2 * 7], cos[7], atol=1e-6)
    ntk, _ = dpb.rope_tables(50, 16, base=500.0, scaling="ntk", factor=4.0)
    # the fastest pair keeps its frequency, the slowest is divided by the factor
    assert torch.allclose(ntk[:, 0], cos[:, 0], atol=1e-6)
    slow, _ = dpb.rope_tables(200, 16, base=500.0)
    assert torch.allclose(ntk[40, 7], slow[10, 7], atol=1e-5)
    yarn, _ = dpb.rope_tables(50, 16, base=500.0, scaling="yarn", factor=4.0, original=64)
    gain = 0.1 * torch.log(torch.tensor(4.0)) + 1
    assert abs(float(yarn[0, 0]) - float(gain)) < 1e-6
    for kw in (dict(rot_dim=15), dict(scaling="none"), dict(scaling="yarn", factor=2.0), dict(scaling="linear", factor=0.5)):
        with pytest.raises(ValueError):
            dpb.rope_tables(**{"positions": 8, "rot_dim": 16, **kw})


def test_refusals():
    q = torch.zeros((6, 2, 64), device="cuda")
    cos, sin = dpb.rope_tables(8, 64)
    bad = [
        (dict(k=q[:5]), ValueError), (dict(k=q.bfloat16()), ValueError), (dict(q=q.half(), k=q.half()), ValueError),
        (dict(sin=None), ValueError), (dict(cos=cos[:, :16]), ValueError),
        (dict(positions=torch.zeros(6, dtype=torch.int64, device="cuda")), ValueError),
        (dict(weight_q=torch.ones(32, device="cuda")), ValueError),
        (dict(weight_q=torch.ones(64, device="cuda"), normalise=False), dpb.DPBError),
        (dict(eps=-1.0), dpb.DPBError), (dict(q=q.cpu()), ValueError),
    ]
    for kw, err in bad:
        at = dict(q=q, k=q, cos=cos, sin=sin)
        at.update(kw)
        with pytest.raises(err):
            dpb.qk_norm_rope(**at)
    for D in (7, 258):
        x = torch.zeros((6, 2, D), device="cuda")
        with pytest.raises(dpb.DPBError):
            dpb.qk_norm_rope(x, x)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,Hk,D", [(5, 2, 64), (3, 1, 128), (4, 4, 16), (1, 7, 24), (33, 2, 8)])
def test_without_eps(H, Hk, D, dtype):
    """eps = 0 with head counts that leave lane groups of a warp without a head: the formula's gradients, all finite."""
    T = 40
    q, k, w, cos, sin, pos, gy = draw(T, H, Hk, D, D, dtype, seed=31)
    at = dict(weight_q=w[0], weight_k=w[1], cos=cos, sin=sin, positions=pos, eps=0.0)
    y, dx = dpb.qk_norm_rope(q, k, **at), dpb.qk_norm_rope_backward(q, k, *gy, **at)
    for i, x in enumerate((q, k)):
        xd, wd = x.double().requires_grad_(), w[i].double().requires_grad_()
        r = torch.rsqrt((xd * xd).mean(-1, keepdim=True))
        want = formula(xd * r * wd, None, cos, sin, pos, D, False, normalise=False)
        close(y[i], want.detach(), (xd * r * wd).detach().abs().amax(-1, keepdim=True) * 2, D)
        gx, gw = torch.autograd.grad(want, (xd, wd), gy[i].double())
        n, r = (xd * r).detach().abs(), r.detach()
        u = 2 * gy[i].double().abs().amax(-1, keepdim=True) * wd.detach().abs().amax()
        close(dx[i], gx, r * (u + n * (u * n).mean(-1, keepdim=True)), D, extra=2)
        close(dx[2 + i], gw, (2 * gy[i].double().abs().amax(-1, keepdim=True) * n).sum((0, 1)), D, extra=T * (H, Hk)[i] / D + 2)
        assert torch.isfinite(dx[2 + i]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rot,inter", [(64, False), (64, True), (48, False), (20, True), (30, False)])
def test_unaligned_rows_element_by_element(rot, inter, dtype):
    """Rows at odd addresses, and gradients into them: each value within its own rounding of the formula's."""
    T, H, D = 45, 3, 64
    q, k, w, cos, sin, pos, gy = draw(T, H, H, D, rot, dtype, seed=32)

    def odd(x):
        y = torch.empty(T * H * (D + 1) + 1, dtype=dtype, device="cuda")[1:].view(T, H, D + 1)[:, :, :D]
        return y.copy_(x)

    at = dict(weight_q=w[0], weight_k=w[1], cos=cos, sin=sin, positions=pos, eps=EPS, interleaved=inter)
    rows = [odd(x) for x in (q, k, *gy)]
    outs = [odd(torch.zeros_like(q)) for _ in range(4)]
    dpb.qk_norm_rope(*rows[:2], **at, q_out=outs[0], k_out=outs[1])
    *_, dwq, dwk = dpb.qk_norm_rope_backward(*rows, **at, grad_q=outs[2], grad_k=outs[3])
    for i, x in enumerate((q, k)):
        xd, wd = x.double().requires_grad_(), w[i].double().requires_grad_()
        want = formula(xd, wd, cos, sin, pos, rot, inter)
        r = torch.rsqrt((xd * xd).mean(-1, keepdim=True) + EPS).detach()
        n = xd.detach().abs() * r
        close(outs[i], want.detach(), (n * wd.detach().abs()).amax(-1, keepdim=True) * 2, D)
        gx, gw = torch.autograd.grad(want, (xd, wd), gy[i].double())
        u = 2 * gy[i].double().abs().amax(-1, keepdim=True) * wd.detach().abs().amax()
        close(outs[2 + i], gx, r * (u + n * (u * n).mean(-1, keepdim=True)), D, extra=2)
        close((dwq, dwk)[i], gw, (2 * gy[i].double().abs().amax(-1, keepdim=True) * n).sum((0, 1)), D, extra=T * H / D + 2)
