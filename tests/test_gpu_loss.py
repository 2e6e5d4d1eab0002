"""Cross entropy over the vocabulary from the hidden rows, and its gradient,
against the formula in 64 bits.

Bounds. A score is a sum of d exact products in fp32; an addition is off by at
most 2^-23 of the sums of absolute values (the tensor cores may truncate), so
a score by e_z = d 2^-23 sum |h w|. A sum of exponentials has relative errors
of 2^-21 (exponentials of 2 ulp, factors of log2 e to 2^-24, sums of at most 64
terms in a chain, joined in a tree), its exponents 2^-22 of the largest
score's size; lse and the loss are each rounded once (2^-24). dz enters the
gradients' products in bf16 (2^-8) with the errors of its exponential; each
gradient is a fp32 sum and rounded to bf16 (2^-8) once.
"""
import pytest
import torch

from paper_2607_20652_gb300 import build, dpb

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build()
    dpb.load()


def draw(T, V, d, seed=0, left_out="none", even=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn(T, d, generator=g, device="cuda").to(BF)
    w = (torch.randn(V, d, generator=g, device="cuda") * 1.5 / d ** 0.5).to(BF)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    if left_out == "some":
        y[torch.rand(T, generator=g, device="cuda") < 0.4] = -100
    elif left_out == "runs":
        y[torch.arange(T, device="cuda") % 300 < 200] = -100
    elif left_out == "all":
        y[:] = -100
    gl = torch.full((1,), 1 / max(T, 1), device="cuda").expand(T) if even else \
        torch.randn(T, generator=g, device="cuda") / max(T, 1)
    return h, w, y, gl


def formula(h, w, y, gl):
    """loss, lse, dh, dw, and the sums of absolute values behind them."""
    h, w, gl = h.double(), w.double(), gl.double()
    ok = y >= 0
    at = y.clamp(min=0)[:, None]
    z = h @ w.t()
    lse = torch.where(ok, torch.logsumexp(z, 1), 0)
    loss = torch.where(ok, lse - z.gather(1, at)[:, 0], 0)
    dz = torch.exp(z - lse[:, None]).scatter_add(1, at, -torch.ones_like(at, dtype=torch.float64))
    dz = torch.where(ok[:, None], dz * gl[:, None], 0)
    e_z = h.shape[1] * 2.0 ** -23 * (h.abs() @ w.abs().t()).amax(1) if len(w) else None
    return loss, lse, dz @ w, dz.t() @ h, z.abs().amax(1), e_z, dz.abs() @ w.abs(), dz.abs().t() @ h.abs()


def check(got, want, tol):
    off = ((got.double() - want).abs() / tol).nan_to_num(1e9).max() if got.numel() else torch.zeros(())
    assert float(off) <= 1, float(off)


def near(got, want):
    """Roundings of dz and of the result, each 2^-8 at most and spread evenly: rms 2^-8 / sqrt 3 each."""
    n = want.norm()
    assert float((got.double() - want).norm()) <= 2.0 ** -8 * (2 / 3) ** 0.5 * 1.2 * float(n) + 1e-30


def compare(h, w, y, gl, loss, lse, dh=None, dw=None):
    T, V, d = h.shape[0], w.shape[0], h.shape[1]
    ls, le, gh, gw, top, e_z, sh, sw = formula(h, w, y, gl)
    e = e_z + 2.0 ** -21 + 2.0 ** -22 * top
    check(lse, le, e + 2.0 ** -24 * le.abs())
    check(loss, ls, 2 * e + 2.0 ** -24 * ls.abs())
    e = 2.0 ** -8 + 2 * float(e.max())
    if dh is not None:
        check(dh, gh, (e + V * 2.0 ** -23) * sh + 2.0 ** -8 * gh.abs() + 1e-30)
        near(dh, gh)
    if dw is not None:
        check(dw, gw, (e + T * 2.0 ** -23) * sw + 2.0 ** -8 * gw.abs() + 1e-30)
        near(dw, gw)


SIZES = [  # tokens, vocabulary, columns
    (1, 50, 8), (33, 777, 72), (128, 97, 64), (255, 256, 64), (257, 257, 264), (300, 1000, 128), (513, 5003, 520),
    (64, 9001, 2048), (1, 20000, 1000),
    (8449, 9001, 72), (2000, 30011, 264), (12289, 4355, 128),  # pieces of the vocabulary, their sums apart
    (24001, 5003, 136), (20001, 9001, 72), (7001, 17001, 72),  # and one after the other: two, three, four pieces
    (20001, 300, 264), (65537, 700, 72), (4097, 97, 520), (9000, 5000, 64),  # the weight's sums of parts of the tokens apart
]


@pytest.mark.parametrize("left_out,even", [("none", True), ("some", False), ("runs", True)])
@pytest.mark.parametrize("T,V,d", SIZES)
def test_loss_and_gradient(T, V, d, left_out, even):
    if T == 1 and left_out != "none":
        left_out = "none"
    h, w, y, gl = draw(T, V, d, seed=T + V, left_out=left_out, even=even)
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    assert dpb.status() == 0
    compare(h, w, y, gl, loss, lse, dh, dw)
    assert not loss[y < 0].any() and not lse[y < 0].any() and not dh[y < 0].any()


def test_a_single_word():
    h, w, y, gl = draw(70, 1, 16)
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    # the loss is 0; p - 1 is the rounding of lse in p = exp(z - lse): of the score's errors
    e = float((16 * 2.0 ** -22 * (h.double().abs() @ w.double().abs().t())).max()) + 2.0 ** -20
    assert float(loss.abs().max()) <= e and float(dh.abs().max()) <= e * float(w.abs().max()) / 70
    assert float(dw.abs().max()) <= e * float(h.abs().max())


def test_small_losses_keep_their_digits():
    """Tokens that the model is sure of: the loss is log1p of a small sum, not the difference of large scores."""
    V, d = 500, 64
    w = torch.zeros(V, d, device="cuda", dtype=BF)
    w[:, 0] = 1.0
    w[7, 1] = 1.0
    h = torch.zeros(40, d, device="cuda", dtype=BF)
    h[:, 0] = 64.0
    h[:, 1] = torch.arange(40, device="cuda") * 0.5
    y = torch.full((40,), 7, device="cuda")
    loss, _ = dpb.linear_cross_entropy_forward(h, w, y)
    want = torch.log1p(499 * torch.exp(-0.5 * torch.arange(40, device="cuda", dtype=torch.float64)))
    # The scores are exact and the largest gives 1 exactly; what is added to it goes through at most 4 additions of a
    # chain, 3 of the chains, 1 of each piece of 32 (4 of them), 1 of the halves and 5 of the joining warp: 17 roundings of
    # 2^-24 of a sum near 1, below 2^-19.9 in its logarithm. The other exponentials are off by 2^-21 of themselves.
    check(loss, want, 2.0 ** -21 * want + 2.0 ** -19.9)


@pytest.mark.parametrize("T,V", [(300, 700), (9000, 700), (24001, 5003)])
def test_all_ignored(T, V):
    h, w, y, gl = draw(T, V, 64, left_out="all")
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    for t in (loss, lse, dh, dw):
        assert not t.any()


def test_no_tokens():
    h, w = torch.empty(0, 64, device="cuda", dtype=BF), torch.randn(700, 64, device="cuda").to(BF)
    y = torch.empty(0, dtype=torch.long, device="cuda")
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, loss)
    assert loss.shape == (0,) and dh.shape == (0, 64) and dw.shape == w.shape and not dw.any()


def test_ignored_rows_are_not_read():
    h, w, y, gl = draw(600, 1000, 72, left_out="runs", even=False)
    outs = []
    for fill in (0.0, float("nan"), float("inf")):
        h[y < 0] = fill
        gl = gl.clone()
        gl[y < 0] = fill
        loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
        outs.append((loss, lse, *dpb.linear_cross_entropy_backward(h, w, y, lse, gl)))
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            assert torch.equal(a, b)


def test_another_ignored_target_and_32_bit_targets():
    h, w, y, gl = draw(300, 700, 64, left_out="some")
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    want = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    for k, ignore in ((torch.where(y < 0, -1, y).int(), -1), (torch.where(y < 0, 1 << 40, y), 1 << 40)):
        got = dpb.linear_cross_entropy_forward(h, w, k, ignore_index=ignore)
        assert torch.equal(loss, got[0]) and torch.equal(lse, got[1])
        for a, b in zip(want, dpb.linear_cross_entropy_backward(h, w, k, lse, gl, ignore_index=ignore)):
            assert torch.equal(a, b)
    assert dpb.status() == 0


def test_a_word_that_is_ignored():
    """ignore_index may be a word: its tokens take no part, its row of the gradient is of the other tokens."""
    h, w, y, gl = draw(300, 50, 64)
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y, ignore_index=3)
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl, ignore_index=3)
    compare(h, w, torch.where(y == 3, -100, y), gl, loss, lse, dh, dw)


def test_targets_out_of_range_are_flagged():
    h, w, y, gl = draw(300, 700, 64)
    y[5], y[250] = 700, -1
    dpb.status()
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    assert dpb.status() == dpb.DEV_BAD_INDEX
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    assert dpb.status() == dpb.DEV_BAD_INDEX
    y[5] = y[250] = -100
    compare(h, w, y, gl, loss, lse, dh, dw)


def test_strides_and_what_lies_between_is_left_alone():
    h, w, y, gl = draw(300, 700, 72, left_out="some")
    hs, ws = torch.full((300, 104), float("nan"), device="cuda", dtype=BF), torch.full((700, 80), float("nan"), device="cuda",
                                                                                      dtype=BF)
    hs[:, 16:88], ws[:, :72] = h, w
    gh, gw = torch.full((300, 96), 3.0, device="cuda", dtype=BF), torch.full((700, 200), 3.0, device="cuda", dtype=BF)
    loss, lse = dpb.linear_cross_entropy_forward(hs[:, 16:88], ws[:, :72], y)
    dpb.linear_cross_entropy_backward(hs[:, 16:88], ws[:, :72], y, lse, gl, grad_hidden=gh[:, 8:80], grad_weight=gw[:, 64:136])
    compare(h, w, y, gl, loss, lse, gh[:, 8:80], gw[:, 64:136])
    for t, a, b in ((gh, 8, 80), (gw, 64, 136)):
        assert (t[:, :a] == 3).all() and (t[:, b:] == 3).all()


@pytest.mark.parametrize("T,V", [(300, 700), (9000, 4500), (24001, 5003), (12000, 700)])
def test_one_gradient_alone(T, V):
    h, w, y, gl = draw(T, V, 64)
    _, lse = dpb.linear_cross_entropy_forward(h, w, y)
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    a, none = dpb.linear_cross_entropy_backward(h, w, y, lse, gl, want_weight=False)
    assert none is None and torch.equal(a, dh)
    none, b = dpb.linear_cross_entropy_backward(h, w, y, lse, gl, want_hidden=False)
    assert none is None and torch.equal(b, dw)
    assert dpb.linear_cross_entropy_backward(h, w, y, lse, gl, want_hidden=False, want_weight=False) == (None, None)


def test_gradients_that_are_zero_large_small_or_not_finite():
    h, w, y, _ = draw(300, 700, 64)
    _, lse = dpb.linear_cross_entropy_forward(h, w, y)
    for gl in (torch.zeros(300, device="cuda"), torch.full((1,), -0.0, device="cuda").expand(300)):
        assert not any(t.any() for t in dpb.linear_cross_entropy_backward(h, w, y, lse, gl))
    for size in (1e30, 1e-30):
        gl = torch.randn(300, device="cuda") * size
        _, _, gh, gw, *_ = formula(h, w, y, gl)
        dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
        near(dh, gh)
        near(dw, gw)
    gl = torch.randn(300, device="cuda")
    want, _ = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    gl[3] = float("nan")
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    assert dh[3].isnan().all() and dw.isnan().all()
    keep = torch.arange(300, device="cuda") != 3
    check(dh[keep], want[keep].double(), 2.0 ** -6 * want[keep].double().abs() + 2.0 ** -7 * want.double().abs().max())


def test_few_tokens_lose_nothing_to_the_products_type():
    """Up to 512 tokens dz is held in two bf16, so that only the results are rounded: 2^-8 each, evenly, rms 2^-8 / sqrt 3."""
    for T in (1, 2, 5, 31, 200, 512):
        h, w, y, gl = draw(T, 3001, 128, seed=T, even=False)
        _, lse = dpb.linear_cross_entropy_forward(h, w, y)
        _, _, gh, gw, *_ = formula(h, w, y, gl)
        for got, want in zip(dpb.linear_cross_entropy_backward(h, w, y, lse, gl), (gh, gw)):
            assert float((got.double() - want).norm()) <= 2.0 ** -8 / 3 ** 0.5 * 1.05 * float(want.norm())


def test_gradient_against_differences():
    """Rows on a grid of 2^-4, moved by 2^-4 along random directions: f(x + s) - f(x - s) over 2 s, whose third-order
    term is at most |s|^3 / 6 times the largest third central moment of the scores' changes, 2 max|s w|^3."""
    T, V, d = 40, 300, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    h = (torch.randint(-16, 17, (T, d), generator=g, device="cuda") / 16.0).to(BF)
    w = (torch.randint(-16, 17, (V, d), generator=g, device="cuda") / 32.0).to(BF)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    gl = torch.rand(T, generator=g, device="cuda")
    _, lse = dpb.linear_cross_entropy_forward(h, w, y)
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    for x, grad, other in ((h, dh, w), (w, dw, h)):
        s = (torch.randint(0, 2, x.shape, generator=g, device="cuda") * 2 - 1) * (torch.rand(x.shape, generator=g, device="cuda")
                                                                               < 0.1) / 16.0
        s = s.to(BF)
        up, down = ((x + s), (x - s))
        f = [(dpb.linear_cross_entropy_forward(*((a, w) if x is h else (h, a)), y)[0].double() * gl.double()).sum() for a in
             (up, down)]
        got = float((f[0] - f[1]) / 2)
        change = (s.double() @ other.double().t()).abs().max() if x is h else (other.double() @ s.double().t()).abs().max()
        tol = float(gl.double().sum()) * (float(change) ** 3 / 3 + 2 * (2.0 ** -20 + 2.0 ** -21 * float(lse.max())))
        tol += 2.0 ** -7 * float((grad.double() * s.double()).abs().sum()) + 2.0 ** -8 * float(gl.sum()) * float(change)
        want = float((grad.double() * s.double()).sum())
        assert abs(got - want) <= tol, (got, want, tol)


@pytest.mark.parametrize("T,V,d", [(300, 5000, 520), (9000, 5000, 264), (24001, 5003, 72), (30000, 600, 136)])
def test_equal_inputs_give_equal_bits(T, V, d):
    h, w, y, gl = draw(T, V, d, left_out="some", even=False)
    first = None
    for _ in range(3):
        loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
        out = (loss, lse, *dpb.linear_cross_entropy_backward(h, w, y, lse, gl))
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(first, out))


def test_scratch_may_hold_anything():
    """Workspaces full of NaN, and one shared by calls of different sizes."""
    n = 1 << 30
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    ws[:4] = 0
    for T, V, d, left in ((24001, 5003, 72, "runs"), (8449, 5001, 72, "some"), (300, 1000, 64, "none"), (30000, 600, 136, "some"), (64, 257, 200, "runs")):
        h, w, y, gl = draw(T, V, d, left_out=left, even=False)
        loss, lse = dpb.linear_cross_entropy_forward(h, w, y, workspace=ws)
        dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl, workspace=ws)
        assert dpb.workspace_status(ws) == 0
        compare(h, w, y, gl, loss, lse, dh, dw)


def test_another_stream_and_a_graph():
    h, w, y, gl = draw(700, 1000, 64, left_out="some", even=False)
    want = dpb.linear_cross_entropy_forward(h, w, y)
    grads = dpb.linear_cross_entropy_backward(h, w, y, want[1], gl)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = dpb.linear_cross_entropy_forward(h, w, y, stream=s)
    got_grads = dpb.linear_cross_entropy_backward(h, w, y, got[1], gl, stream=s)
    s.synchronize()
    for a, b in zip((*want, *grads), (*got, *got_grads)):
        assert torch.equal(a, b)
    h2, w2, y2, gl2 = draw(700, 1000, 64, seed=5, left_out="runs", even=False)
    graph = torch.cuda.CUDAGraph()
    hh, ww, yy, gg = h.clone(), w.clone(), y.clone(), gl.clone()
    with torch.cuda.graph(graph):
        loss, lse = dpb.linear_cross_entropy_forward(hh, ww, yy)
        dh, dw = dpb.linear_cross_entropy_backward(hh, ww, yy, lse, gg)
    for a, b, c, k in ((h2, w2, y2, gl2), (h, w, y, gl)):
        for t, v in ((hh, a), (ww, b), (yy, c), (gg, k)):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        compare(a, b, c, k, loss, lse, dh, dw)
    assert dpb.status() == 0


def test_scores_far_below_zero():
    """Maxima near the lowest fp32 values: 300 words in seven ranks, the highest of 43 equal scores."""
    V, d, big = 300, 8, 1.5 * 2.0 ** 60
    rank = torch.arange(V, device="cuda") % 7
    h = torch.full((7, d), big, device="cuda", dtype=torch.bfloat16)
    w = (-big * (1 + rank.double() / 4))[:, None].expand(V, d).to(torch.bfloat16).contiguous()
    y = torch.arange(7, device="cuda")
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    z = h.double() @ w.double().T  # about -2e37: exact in fp32, as the factors have few bits
    top = z.max(1).values
    rest = torch.logsumexp(z - top[:, None], 1)  # the logarithm of 43
    # lse: a rounding and the logarithm's; the loss another
    assert ((lse.double() - (top + rest)).abs() <= 2.0 ** -22 * top.abs()).all()
    want = top - z[torch.arange(7), y] + rest
    assert ((loss.double() - want).abs() <= 2.0 ** -22 * want).all()


def test_two_streams_at_once():
    """Losses and gradients of different sizes under way at the same time, their blocks side by side on the device."""
    work = []
    for T, V, d, left in ((3000, 9000, 264, "some"), (24001, 4500, 72, "runs"), (300, 20000, 128, "none")):
        h, w, y, gl = draw(T, V, d, seed=T, left_out=left, even=False)
        loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
        work.append(((h, w, y, gl), (loss, lse, *dpb.linear_cross_entropy_backward(h, w, y, lse, gl)), torch.cuda.Stream()))
    torch.cuda.synchronize()
    got = []
    for _ in range(8):
        for (h, w, y, gl), want, s in work:
            with torch.cuda.stream(s):
                loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
                got.append((want, (loss, lse, *dpb.linear_cross_entropy_backward(h, w, y, lse, gl))))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for want, out in got for a, b in zip(want, out))
    assert all(dpb.status(stream=s) == 0 for _, _, s in work)


def test_refusals():
    h, w, y, gl = draw(30, 70, 64)
    for bad in (dict(hidden=h.float()), dict(weight=w.float()), dict(hidden=h[:, :60]), dict(targets=y.float()),
                dict(targets=y[:20]), dict(weight=w.t()[:64].t()[:, ::2]), dict(hidden=h[0])):
        at = dict(hidden=h, weight=w, targets=y, **{}) | bad
        with pytest.raises((ValueError, dpb.DPBError)):
            dpb.linear_cross_entropy_forward(**at)
    with pytest.raises(dpb.DPBError):  # 60 columns of rows of 64
        dpb.linear_cross_entropy_forward(h[:, :60], w[:, :60], y)
    with pytest.raises(dpb.DPBError):  # rows at an odd address
        dpb.linear_cross_entropy_forward(h[:, 1:57], w[:, :56], y)
    _, lse = dpb.linear_cross_entropy_forward(h, w, y)
    for bad in (gl.double(), gl[:20], torch.rand(60, device="cuda")[::2], torch.rand((), device="cuda")):
        with pytest.raises(ValueError):
            dpb.linear_cross_entropy_backward(h, w, y, lse, bad)
    with pytest.raises(ValueError):
        dpb.linear_cross_entropy_backward(h, w, y, lse[:20], gl)
    with pytest.raises(dpb.DPBError):
        dpb.linear_cross_entropy_forward(h, w, y, workspace=torch.zeros(1024, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("T", [70, 700, 9000])
@pytest.mark.parametrize("size", [1.0, 8.0, 64.0])
def test_a_single_word_has_no_gradient(T, size):
    """lse is the word's own score, the same sum in both directions, so exp(z - lse) - 1 is 0 exactly, however large z is."""
    h, w, y, gl = draw(T, 1, 64, seed=T)
    h = (h * size).to(BF)
    _, lse = dpb.linear_cross_entropy_forward(h, w, y)
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    assert lse.any() and not dh.any() and not dw.any()


@pytest.mark.parametrize("T,V", [(300, 700), (3000, 5003), (9000, 13001)])
def test_tokens_that_the_model_is_sure_of_have_no_gradient(T, V):
    """Scores of up to 1000 whose target lies 110 above all others: exp(-110) is 0 in fp32, so lse is the target's score."""
    d = 64
    g = torch.Generator(device="cuda").manual_seed(T)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[::3] = 5  # the word of the sure rows below
    h = torch.zeros(T, d, device="cuda")
    h[:, 0] = torch.randint(1, 100, (T,), generator=g, device="cuda") * 9.0
    h[::3, 1] = 110.0
    w = torch.zeros(V, d, device="cuda")
    w[:, 0] = 1.0
    w[5, 1] = 1.0
    h, w = h.to(BF), w.to(BF)
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    gl = torch.rand(T, generator=g, device="cuda") * 10
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    assert not loss[::3].any() and not dh[::3].any()
    assert loss[1::3].all()
    sure = torch.full_like(y, -100)
    sure[::3] = 5
    dh, dw = dpb.linear_cross_entropy_backward(h, w, sure, lse, gl)
    assert not dh.any() and not dw.any()


def test_the_widest_rows():
    """2^20 columns. Values of 0, 1 and -1, and of 2^-9 of these: every partial sum of a score is exact in fp32."""
    T, V, d = 40, 300, 1 << 20
    g = torch.Generator(device="cuda").manual_seed(6)
    h = torch.randint(-1, 2, (T, d), generator=g, device="cuda").to(BF)
    w = (torch.randint(-1, 2, (V, d), generator=g, device="cuda") / 512.0).to(BF)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    gl = torch.rand(T, generator=g, device="cuda")
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    z = h.double() @ w.double().t()
    want = torch.logsumexp(z, 1)
    assert ((lse.double() - want).abs() <= 2.0 ** -21 + 2.0 ** -22 * z.abs().amax(1) + 2.0 ** -24 * want.abs()).all()
    dh, dw = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    dz = torch.softmax(z, 1)
    dz[torch.arange(T, device="cuda"), y] -= 1
    dz *= gl.double()[:, None]
    near(dh, dz @ w.double())
    near(dw, dz.t() @ h.double())
    assert dpb.status() == 0


@pytest.mark.parametrize("T,V,d", [(300, 700, 64), (2000, 9001, 264), (24001, 5003, 72), (20001, 300, 264)])
def test_waits_that_give_up_are_flagged_and_leave_the_context_usable(T, V, d):
    """With waits of 0 polls for other blocks, every pair of blocks ends at the first unit that waits: pieces all held, in
    two bf16 and in one, one after the other, and parts of the tokens. A call right after is right again; the forward has
    no such wait."""
    h, w, y, gl = draw(T, V, d, seed=T, left_out="some", even=False)
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    want = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    assert dpb.status() == 0
    try:
        dpb.set_wait_limit(0)
        again = dpb.linear_cross_entropy_forward(h, w, y)
        assert dpb.status() == 0 and torch.equal(again[0], loss) and torch.equal(again[1], lse)
        dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
        assert dpb.status() == dpb.DEV_TIMEOUT
    finally:
        dpb.set_wait_limit(-1)
    got = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    assert dpb.status() == 0 and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("left_out", ["none", "some"])
def test_offsets_past_32_bits(left_out):
    """Hidden rows of 2^31 values and more: 512 times the same rows, each time the same bits (as given, and closed up)."""
    T, V, d, n = 4099, 97, 1024, 512
    h, w, y, _ = draw(T, V, d, seed=8, left_out=left_out)
    gl = torch.rand(T, device="cuda")
    loss0, lse0 = dpb.linear_cross_entropy_forward(h, w, y)
    dh0, _ = dpb.linear_cross_entropy_backward(h, w, y, lse0, gl)
    hh, yy, gg = h.repeat(n, 1), y.repeat(n), gl.repeat(n)
    assert hh.numel() > 2 ** 31
    loss, lse = dpb.linear_cross_entropy_forward(hh, w, yy)
    assert (loss.view(n, T) == loss0).all() and (lse.view(n, T) == lse0).all()
    dh, dw = dpb.linear_cross_entropy_backward(hh, w, yy, lse, gg)
    assert (dh.view(n, T, d) == dh0).all()
    near(dw, formula(h, w, y, gl)[3] * n)
    assert dpb.status() == 0


@pytest.mark.parametrize("V,d", [(500, 64), (500, 1000), (20000, 1024)])
def test_the_smallest_losses_keep_their_digits(V, d):
    """As above, with losses down to 1e-19: the logarithm of 1 and a sum that is far smaller, 2^-21 of itself off by the
    exponentials, as much by the sum's roundings and by an exponential of 2 ulp and a log1p of 2. With the target's score
    as it is multiplied, summed in the join and summed beside the products."""
    n = 100
    w = torch.zeros(V, d, device="cuda", dtype=BF)
    w[:, 0] = 1.0
    w[7, d - 1] = 1.0
    h = torch.zeros(n, d, device="cuda", dtype=BF)
    h[:, 0] = 64.0
    h[:, d - 1] = torch.arange(n, device="cuda") * 0.5
    y = torch.full((n,), 7, device="cuda")
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    gap = 0.5 * torch.arange(n, device="cuda", dtype=torch.float64)
    want = torch.log1p((V - 1) * torch.exp(-gap))
    check(loss, want, 2.0 ** -19 * want)
    check(lse, 64 + gap + want, 2.0 ** -23 * (64 + gap + want))


@pytest.mark.parametrize("T,V,d", [(33, 50257, 768), (300, 700, 1024), (2000, 1000, 2048)])
def test_the_targets_scores_are_rounded_not_cut(T, V, d):
    """Every score but the target's is 0 exactly, the target's a sum of d random products: the loss is off by that sum's
    roundings, of lanes' chains of d / 64 products each and 6 joins, and by a few ulp of exponential and logarithm."""
    g = torch.Generator(device="cuda").manual_seed(d)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    w = torch.zeros(V, d, device="cuda", dtype=BF)
    w[y[0]] = (torch.randn(d, generator=g, device="cuda") * 0.1).to(BF)
    y[:] = y[0]
    h = torch.randn(T, d, generator=g, device="cuda").to(BF)
    h = (h.float() + w[y].float() * 8 / (w[y].float() ** 2).sum(1, keepdim=True)).to(BF)
    loss, _ = dpb.linear_cross_entropy_forward(h, w, y)
    z, size = (h.double() * w[y].double()).sum(1), (h.double() * w[y].double()).abs().sum(1)
    want = torch.log1p((V - 1) * torch.exp(-z))
    check(loss, want, ((d / 64 + 8) * 2.0 ** -24 * size + 2.0 ** -20) * want.clamp(min=0) + 2.0 ** -23 * want +
          (d / 64 + 8) * 2.0 ** -24 * size * (want > 1))


def test_an_infinite_score_has_no_loss():
    h, w, y, _ = draw(40, 300, 64, seed=9)
    h[3], w[y[3]] = 1e30, 1e30
    y[4:] = (y[3] + 1) % 300
    h[:, :] = torch.where(torch.arange(40, device="cuda")[:, None] == 3, h, 0)
    loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
    want = torch.log(torch.full((36,), 300.0, device="cuda"))
    assert loss[3].isnan() and (loss[4:] - want).abs().max() < 2.0 ** -20


@pytest.mark.parametrize("even", [True, False])
@pytest.mark.parametrize("T,V,d", [(513, 3001, 128), (3000, 3001, 264), (9000, 13001, 72), (20001, 300, 264), (40, 200000, 64)])
def test_hidden_gradients_are_rounded_once(T, V, d, even):
    """dz of the targets loses nothing to the products' type: what is left is the result's rounding, 2^-7 / sqrt 12 of each
    value's binade, 0.2123 2^-7 of the norm over evenly spread digits, and that of the other words' dz, which is as much of
    sqrt(e^2.25 / V) of the norm at scores of a deviation of 1.5. Sums of pieces apart, one after the other, and one piece."""
    h, w, y, gl = draw(T, V, d, seed=T, even=even)
    _, lse = dpb.linear_cross_entropy_forward(h, w, y)
    dh, _ = dpb.linear_cross_entropy_backward(h, w, y, lse, gl)
    want = formula(h, w, y, gl)[2]
    assert float((dh.double() - want).norm()) <= 2.0 ** -7 * 0.2123 * 1.08 * (1 + 9.5 / V) ** 0.5 * float(want.norm())
