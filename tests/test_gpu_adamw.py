"""AdamW over many tensors against the formula in 64 bits: fp32 states, 8-bit
states, odd sizes and alignments, skipped steps."""
import math

import pytest
import torch

from paper_2607_20652_gb300 import build, dpb

pytestmark = pytest.mark.gpu
H = dict(lr=1e-2, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
BLOCK = dpb.STATE_BLOCK


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build()
    dpb.load()


def tensors(sizes, dtype, bits, seed=0, shift=0):
    """Parameters, gradients and states, each `shift` values off an aligned address."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def off(n, dt):
        return torch.empty(n + shift, device="cuda", dtype=dt)[shift:]

    out = dict(p=[], g=[], m=[], v=[], ms=[], vs=[])
    for n in sizes:
        size = 10 ** float(torch.randint(-4, 1, (1,), generator=g, device="cuda"))
        p, gr = off(n, dtype), off(n, dtype)
        p.copy_(torch.randn(n, generator=g, device="cuda"))
        gr.copy_(torch.randn(n, generator=g, device="cuda") * size)
        m, v = torch.randn(n, generator=g, device="cuda") * size * 0.3, torch.rand(n, generator=g, device="cuda") * size ** 2
        if bits == 32:
            ms = [off(n, torch.float32).copy_(m), off(n, torch.float32).copy_(v)]
        else:
            ms = []
            for x, k in ((m, "ms"), (v.sqrt(), "vs")):
                nb = -(-n // BLOCK)
                pad = torch.zeros(nb * BLOCK, device="cuda")
                pad[:n] = x
                top = pad.view(nb, BLOCK).abs().amax(1)
                code = (pad.view(nb, BLOCK) * (448 / top.clamp(min=1e-30))[:, None]).to(torch.float8_e4m3fn).view(-1)[:n]
                ms.append(off(n, torch.uint8).view(torch.float8_e4m3fn).copy_(code) if shift == 0 else
                          torch.cat([code.view(torch.uint8)[:1].repeat(shift), code.view(torch.uint8)])[shift:].view(
                              torch.float8_e4m3fn))
                out[k].append(top / 448)
        out["p"].append(p), out["g"].append(gr), out["m"].append(ms[0]), out["v"].append(ms[1])
    return out


def held(t, i, bits):
    """(m, v) of tensor i as the values they stand for, 64 bits."""
    if bits == 32:
        return t["m"][i].double(), t["v"][i].double()
    n = t["p"][i].numel()
    rep = [t[k][i].double().repeat_interleave(BLOCK)[:n] for k in ("ms", "vs")]
    return t["m"][i].float().double() * rep[0], (t["v"][i].float().double() * rep[1]) ** 2


def formula(p, g, m, v, step, lr, betas, eps, weight_decay):
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    p = p - lr * weight_decay * p - lr * (m / (1 - betas[0] ** step)) / ((v / (1 - betas[1] ** step)).sqrt() + eps)
    return p, m, v


def group(t, bits):
    return dpb.AdamWGroup(t["p"], t["m"], t["v"], *((t["ms"], t["vs"]) if bits == 8 else ()))


SIZES = [1, 7, 8, 255, 256, 257, 2048, 2049, 5000, 100003]


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_step(dtype, bits, shift):
    t = tensors(SIZES, dtype, bits, seed=1, shift=shift)
    want = [formula(p.double(), g.double(), *held(t, i, bits), 3, **H) for i, (p, g) in enumerate(zip(t["p"], t["g"]))]
    group(t, bits).step(t["g"], step=3, seed=5, **H)
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for i, (p, m, v) in enumerate(want):
        # the step itself is off by some fp32 roundings (16 of them at most), the parameter is rounded once
        step = (H["lr"] / math.sqrt(1 - H["betas"][1] ** 3)) * (m.abs() / (v.sqrt() + 1e-12)).clamp(max=1e6)
        assert bool(((t["p"][i].double() - p).abs() <= u * p.abs() + 16 * 2.0 ** -23 * (p.abs() + 10 * step)).all()), i
        gm, gv = held(t, i, bits)
        if bits == 32:
            for got, x in ((gm, m), (gv, v)):
                assert bool(((got - x).abs() <= 4 * 2.0 ** -23 * x.abs().amax()).all())
            continue
        n, nb = p.numel(), -(-p.numel() // BLOCK)
        for got, x, k in ((gm, m, "ms"), (gv.sqrt(), v.sqrt(), "vs")):
            pad = torch.zeros(nb * BLOCK, device="cuda", dtype=torch.float64)
            pad[:n] = x
            top = pad.view(nb, BLOCK).abs().amax(1)
            assert bool(((t[k][i].double() * 448 - top).abs() <= 8 * 2.0 ** -23 * top).all())
            # one of the two neighbouring codes: less than one step of the code away
            y = x.abs() / (top / 448).repeat_interleave(BLOCK)[:n].clamp(min=1e-300)
            gap = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3) * (top / 448).repeat_interleave(BLOCK)[:n]
            assert bool(((got - x).abs() <= gap * (1 + 1e-4)).all()), (i, k)
        assert bool((gv > 0)[v > 0].all())  # a root above zero never becomes zero


def test_rounding_keeps_small_changes_on_average():
    """Values halfway (and at other places) between two codes: the mean over many roundings is the value, within five
    standard deviations of the mean (a rounding's deviation is at most half a step)."""
    n = 1 << 18
    for share in (0.1, 0.5, 0.75):
        # beta1 = 0: m becomes the gradient. One value of each block fixes the scale at 1.
        g = torch.full((n,), 16.0 + 2 * share, device="cuda")
        g[::BLOCK] = 448.0
        m, v = (torch.zeros(n, device="cuda").to(torch.float8_e4m3fn) for _ in range(2))
        ms, vs = (torch.zeros(n // BLOCK, device="cuda") for _ in range(2))
        p = torch.zeros(n, device="cuda")
        dpb.AdamWGroup([p], [m], [v], [ms], [vs]).step([g], lr=0.0, betas=(0.0, 0.5), step=1, seed=7)
        x = (m.float().view(-1, BLOCK) * ms[:, None])[:, 1:].double()
        assert set(x.unique().tolist()) <= {16.0, 18.0}
        assert abs(float(x.mean()) - (16 + 2 * share)) <= 5 * 1.0 / math.sqrt(x.numel())


def test_small_steps_are_not_lost_over_time():
    """A second moment that decays by a thousandth a step: after 700 steps without gradients its root has halved almost as
    in 64 bits, where rounding to the nearest code would leave all but the block's largest... the same share of it."""
    n = 64 * BLOCK
    g = torch.Generator(device="cuda").manual_seed(2)
    u0 = torch.rand(n, generator=g, device="cuda") * 0.5 + 0.5
    u0[::BLOCK] = 1.0
    t = dict(m=torch.zeros(n, device="cuda").to(torch.float8_e4m3fn), ms=torch.zeros(n // BLOCK, device="cuda"),
             v=(u0 * 448).to(torch.float8_e4m3fn), vs=torch.full((n // BLOCK,), 1 / 448, device="cuda"))
    p, grad = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    grad[::BLOCK] = 1.0  # the largest of each block stays, so the scale does: the others have to decay by themselves
    grp = dpb.AdamWGroup([p], [t["m"]], [t["v"]], [t["ms"]], [t["vs"]])
    start = (t["v"].float().view(-1, BLOCK) * t["vs"][:, None])[:, 1:].double().mean()
    for s in range(700):
        grp.step([grad], lr=0.0, betas=(0.9, 0.998), step=s + 1, seed=3)
    now = (t["v"].float().view(-1, BLOCK) * t["vs"][:, None])[:, 1:].double().mean()
    want = start * 0.998 ** 350
    # 64 x 255 values, each a random walk of 700 roundings with a deviation of at most half a step of 32/448
    assert abs(float(now - want)) <= 5 * 0.5 * 32 / 448 * math.sqrt(700) / math.sqrt(n - 64)


def test_equal_seeds_give_equal_bits():
    runs = []
    for seed, step in ((1, 4), (1, 4), (2, 4), (1, 5)):
        t = tensors([3000, 700], torch.float32, 8, seed=9)
        group(t, 8).step(t["g"], step=step, seed=seed, **H)
        runs.append(torch.cat([x.view(torch.uint8) for x in t["m"] + t["v"]]))
    assert torch.equal(runs[0], runs[1])
    assert not torch.equal(runs[0], runs[2]) and not torch.equal(runs[0], runs[3])


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors_and_missing_gradients(bits):
    """More tensors than one launch takes; those without a gradient, and empty ones, stay as they are."""
    sizes = [(i * 37) % 700 for i in range(1000)]
    t = tensors(sizes, torch.float32, bits, seed=3)
    before = [p.clone() for p in t["p"]]
    want = [formula(p.double(), g.double(), *held(t, i, bits), 1, **H)[0] for i, (p, g) in enumerate(zip(t["p"], t["g"]))]
    grads = [g if i % 3 else None for i, g in enumerate(t["g"])]
    grp = group(t, bits)
    grp.step(grads, step=1, **H)
    for i, p in enumerate(t["p"]):
        if i % 3 == 0:
            assert torch.equal(p, before[i])
        elif p.numel():
            assert torch.allclose(p.double(), want[i], rtol=1e-5, atol=1e-6)
    grp.step(t["g"], step=2, **H)  # and now all of them
    assert all(p.numel() == 0 or not torch.equal(p, b) for p, b in zip(t["p"], before))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [0.25, math.inf, math.nan])
def test_gradient_scale(bits, scale):
    a, b = (tensors([4000], torch.float32, bits, seed=4) for _ in range(2))
    keep = [x.clone() for x in (a["p"][0], a["m"][0].view(torch.uint8) if bits == 8 else a["m"][0])]
    group(a, bits).step(a["g"], step=2, grad_scale=torch.full((1,), scale, device="cuda"), **H)
    if math.isfinite(scale):
        b["g"][0].mul_(scale)
        group(b, bits).step(b["g"], step=2, **H)
        assert torch.equal(a["p"][0], b["p"][0])
    else:
        assert torch.equal(a["p"][0], keep[0])
        assert torch.equal(a["m"][0].view(torch.uint8) if bits == 8 else a["m"][0], keep[1])


def test_a_nan_stays_where_it_is():
    t = tensors([600], torch.float32, 8, seed=5)
    t["g"][0][300] = math.nan
    group(t, 8).step(t["g"], step=1, **H)
    assert torch.isnan(t["p"][0]).nonzero().flatten().tolist() == [300]
    assert torch.isnan(t["m"][0].float()).nonzero().flatten().tolist() == [300]
    assert torch.isfinite(t["ms"][0]).all()


def test_more_than_32_bits_of_values():
    n = (1 << 31) + 777
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = (torch.zeros(-(-n // BLOCK), device="cuda") for _ in range(2))
    dpb.AdamWGroup([p], [m], [v], [ms], [vs]).step([g], lr=0.5, step=1)
    torch.cuda.synchronize()
    for s in (slice(0, 1000), slice((1 << 31) - 500, None)):
        assert bool((p[s] == -0.5).all())  # a first step of size lr
        assert bool((m[s].float() == 448).all())


def test_rebound_parameters_and_streams():
    t = tensors([500, 600], torch.float32, 32, seed=6)
    ps = [torch.nn.Parameter(p.clone()) for p in t["p"]]
    grp = dpb.AdamWGroup(ps, t["m"], t["v"])
    grp.step(t["g"], step=1, **H)
    one = ps[0].detach().clone()
    ps[0].data = ps[0].data.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    grp.step(t["g"], step=2, stream=side, **H)
    side.synchronize()
    assert not torch.equal(ps[0].detach(), one)
    ps[1].data = torch.zeros(5, device="cuda")
    with pytest.raises(ValueError):
        grp.step(t["g"], step=3, **H)


def test_refusals():
    p, m = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    f8, sc = m.to(torch.float8_e4m3fn), torch.zeros(2, device="cuda")
    for args in (([], [], []), ([p.half()], [m], [m]), ([p], [m[:200]], [m]), ([p], [m, m], [m]), ([p], [f8], [f8]),
                 ([p], [f8], [f8], [sc], None), ([p], [f8], [f8], [sc], [sc[:1]]), ([p.view(10, 30).t()], [m], [m])):
        with pytest.raises(ValueError):
            dpb.AdamWGroup(*args)
    grp = dpb.AdamWGroup([p], [m], [m.clone()])
    for kw in (dict(lr=-1.0), dict(lr=math.nan), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1e-8), dict(step=0),
               dict(weight_decay=-1.0)):
        with pytest.raises(dpb.DPBError):
            grp.step([m], **{**H, "step": 1, **kw})
    for g in ([], [p[:5]], [p.bfloat16()], [p.cpu()]):
        with pytest.raises(ValueError):
            grp.step(g, step=1, **H)
    with pytest.raises(ValueError):
        grp.step([m], step=1, grad_scale=torch.ones(2, device="cuda"), **H)


def test_8bit_states_follow_the_formula_rounding_by_rounding():
    """The states' fp32 arithmetic is the formula's with every product and sum rounded by itself, so the scales are those
    of the formula computed one operation at a time, bit for bit (a multiply-add in its place moves one in five)."""
    n = 1 << 20
    t = tensors([n], torch.float32, 8, seed=4)
    (m8, v8, ms, vs, g), (b1, b2) = (t[k][0] for k in ("m", "v", "ms", "vs", "g")), H["betas"]
    m = b1 * (m8.float().view(-1, BLOCK) * ms[:, None]) + (1 - b1) * g.view(-1, BLOCK)
    v = (v8.float().view(-1, BLOCK) * vs[:, None]).square()
    v = b2 * v + (1 - b2) * g.view(-1, BLOCK) * g.view(-1, BLOCK)
    want = [x.abs().amax(1) * (1 / 448) for x in (m, v.sqrt())]
    group(t, 8).step(t["g"], step=3, seed=5, **H)
    assert torch.equal(t["ms"][0], want[0]) and torch.equal(t["vs"][0], want[1])


@pytest.mark.parametrize("bits", [32, 8])
def test_a_copied_group_steps_its_own_tensors(bits):
    """A deep copy, and one saved and loaded, hold copies of the tensors: the original's stay as they are."""
    import copy
    import io
    t = tensors([5000, 257], torch.float32, bits, seed=8)
    grp = group(t, bits)
    file = io.BytesIO()
    torch.save(grp, file)
    file.seek(0)
    for other in (copy.deepcopy(grp), torch.load(file, weights_only=False)):
        kinds = lambda x: [y.view(torch.uint8).clone() for ts in (x.params, x.exp_avg, x.exp_avg_sq) for y in ts]
        before = kinds(grp)
        other.step(t["g"], step=2, seed=5, **H)
        assert all(torch.equal(a, b) for a, b in zip(kinds(grp), before))
        assert not any(torch.equal(a, b) for a, b in zip(kinds(other), before))
    grp.step(t["g"], step=2, seed=5, **H)
    assert all(torch.equal(a, b) for a, b in zip(kinds(grp), kinds(other)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, 1e30])
def test_an_infinity_stays_where_it_is(bad, dtype):
    """An infinite gradient: its own states become NaN, every other value and scale is what it is with a gradient of 0 in its
    place, in this step and in the next. The same of the second moments where only the gradient's square is infinite (the
    first moment is finite then, and the largest of its block)."""
    runs = []
    for g in (bad, 0.0):
        t = tensors([600, 300], dtype, 8, seed=5)
        grp = group(t, 8)
        t["m"][0].view(torch.uint8)[300] = t["v"][0].view(torch.uint8)[300] = 0
        t["g"][0][300] = g
        grp.step(t["g"], step=3, seed=2, **H)
        t["g"][0][300] = 0.0
        grp.step(t["g"], step=4, seed=2, **H)
        runs.append({k: torch.cat([x.float() for x in t[k]]) for k in ("p", "m", "v", "ms", "vs")})
    other = torch.arange(900, device="cuda") != 300
    for k in ("p", "m", "v", "ms", "vs") if math.isinf(bad) else ("v", "vs"):
        a, b = (r[k] if k in ("ms", "vs") else r[k][other] for r in runs)
        assert torch.isfinite(b).all() and torch.equal(a, b), k
    assert runs[0]["v"][300].isnan()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-38, 1e-40, 1e-300])
def test_the_smallest_eps(eps, bits):
    """Values that never had a gradient: 0 / (0 + eps) is 0 for any eps above 0; others do not notice it."""
    t = tensors([600], torch.float32, bits, seed=6)
    for x in (t["g"][0], t["m"][0].view(torch.uint8) if bits == 8 else t["m"][0],
              t["v"][0].view(torch.uint8) if bits == 8 else t["v"][0]):
        x[100:400] = 0
    p, g = t["p"][0].double(), t["g"][0].double()
    want = formula(p, g, *held(t, 0, bits), 2, **{**H, "eps": eps})[0]
    group(t, bits).step(t["g"], step=2, **{**H, "eps": eps})
    assert torch.isfinite(t["p"][0]).all()
    assert torch.allclose(t["p"][0].double(), want, rtol=1e-5, atol=1e-6)
