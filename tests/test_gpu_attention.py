"""Attention over packed sequences and its gradient against the formulas in
64 bits, element by element.

The bounds follow from where the kernels round to bf16 (8 bits, u = 2^-8 relative):
the probabilities before their product with v and with grad_o, dS before its
products with k and q, o inside delta, and every output; scores are fp32 sums
of D exact products, off by at most D 2^-23 sum |q k| scale. Each bound is
carried through the sums with absolute values.
"""
import math

import pytest
import torch

from paper_2607_20652_gb300 import build, dpb

pytestmark = pytest.mark.gpu
U = 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build()
    dpb.load()


def offsets(n):
    return torch.tensor([0] + list(n), device="cuda").cumsum(0).to(torch.int32)


def formula(q, k, v, do, nq, nk, causal, scale):
    """(o, lse, dq, dk, dv) and a bound on the error of each, in 64 bits."""
    q, k, v, do = (x.double() for x in (q, k, v, do))
    g = q.shape[1] // k.shape[1]
    D = q.shape[2]
    out = {n: torch.zeros_like(x) for n, x in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    tol = {n: torch.zeros_like(x) for n, x in out.items()}
    out["lse"] = torch.full((q.shape[1], q.shape[0]), -math.inf, dtype=torch.float64, device=q.device)
    tol["lse"] = torch.zeros_like(out["lse"])
    a = b = 0
    for n, m in zip(nq, nk):
        for h in range(q.shape[1]):
            sa, sb, hk = slice(a, a + n), slice(b, b + m), h // g
            if n == 0 or m == 0:
                continue
            qh, kh, vh, dh = q[sa, h], k[sb, hk], v[sb, hk], do[sa, h]
            see = torch.ones(n, m, dtype=torch.bool, device=q.device)
            if causal:
                see = torch.arange(m, device=q.device)[None] <= torch.arange(n, device=q.device)[:, None] + m - n
            s = (qh @ kh.T * scale).masked_fill(~see, -math.inf)
            es = D * 2.0 ** -23 * scale * (qh.abs() @ kh.abs().T).max() + 1e-6  # error of a score
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None])
            o = p @ vh
            eo = (U + 2 * es) * (p @ vh.abs()) + U * o.abs()
            out["o"][sa, h], tol["o"][sa, h] = o, eo
            out["lse"][h, sa], tol["lse"][h, sa] = lse, 2 * es + 1e-6 * lse.abs()
            out["dv"][sb, hk] += p.T @ dh
            tol["dv"][sb, hk] += (U + 4 * es) * (p.T @ dh.abs())
            dp, delta = dh @ vh.T, (dh * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            ed = (dh.abs() * eo).sum(1, keepdim=True) + D * 2.0 ** -22 * (dh.abs() @ vh.abs().T)
            eds = p * ed + (U + 4 * es) * (ds.abs() + p * ed)
            out["dq"][sa, h] = scale * (ds @ kh)
            tol["dq"][sa, h] = scale * (eds @ kh.abs())
            out["dk"][sb, hk] += scale * (ds.T @ qh)
            tol["dk"][sb, hk] += scale * (eds.T @ qh.abs())
        a, b = a + n, b + m
    for n in ("dq", "dk", "dv"):
        tol[n] += U * out[n].abs()
    return out, {n: t * 1.01 + 1e-30 for n, t in tol.items()}


def run(q, k, v, do, nq, nk, causal=True, scale=None, **kw):
    at = dict(cu_q=offsets(nq), cu_k=offsets(nk), max_q=max(nq), max_k=max(nk), causal=causal, scale=scale)
    o, lse = dpb.attention_forward(q, k, v, **at)
    dq, dk, dv = dpb.attention_backward(q, k, v, o, lse, do, **at, **kw)
    torch.cuda.synchronize()
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def draw(nq, nk, H, Hk, D, seed=0, packed=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if packed and nq == nk:
        qkv = torch.randn(sum(nq), H + 2 * Hk, D, generator=g, device="cuda").bfloat16()
        q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    else:
        q = torch.randn(sum(nq), H, D, generator=g, device="cuda").bfloat16()
        k, v = (torch.randn(sum(nk), Hk, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    return q, k, v, torch.randn(sum(nq), H, D, generator=g, device="cuda").bfloat16()


def check(got, want, tol):
    for n, w in want.items():
        x = got[n].double()
        inf = torch.isinf(w)
        assert torch.equal(torch.isinf(x) & (x < 0), inf), n
        off = torch.where(inf, 0.0, (x - w).abs() / tol[n])
        assert bool((off <= 1).all()), (n, float(off.max()))


CASES = [  # queries and keys of each sequence, heads, key heads, dim, causal
    ([1], [1], 1, 1, 64, True),
    ([1], [777], 4, 2, 64, True),                       # one new token against a cache
    ([128], [128], 2, 2, 64, True),
    ([129], [129], 2, 2, 128, True),
    ([255, 256, 257], [255, 256, 257], 2, 1, 64, True),
    ([383, 1, 640], [383, 1, 640], 3, 3, 128, True),
    ([70, 0, 5, 300], [70, 0, 5, 300], 4, 4, 16, True),  # an empty sequence between
    ([200, 300], [57, 1], 2, 2, 64, True),              # fewer keys than queries: rows that see nothing
    ([200, 33, 1], [0, 400, 2], 6, 2, 96, True),        # a sequence without keys
    ([3, 130], [500, 131], 8, 1, 128, True),            # appended to earlier keys
    ([190, 300], [300, 190], 4, 4, 40, False),
    ([517], [517], 5, 1, 8, False),
    ([130, 7], [1100, 900], 16, 4, 128, False),
    ([1300], [1300], 1, 1, 72, True),
]


@pytest.mark.parametrize("nq,nk,H,Hk,D,causal", CASES)
def test_against_the_formula(nq, nk, H, Hk, D, causal):
    q, k, v, do = draw(nq, nk, H, Hk, D, seed=D + sum(nq))
    want, tol = formula(q, k, v, do, nq, nk, causal, D ** -0.5)
    check(run(q, k, v, do, nq, nk, causal), want, tol)
    assert dpb.status() == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("size,scale", [(6.0, None), (0.01, None), (1.0, 3.0)])
def test_sharp_and_flat_softmax(D, size, scale):
    """Scores far apart (one key takes all, running maxima that grow along the
    keys) and all alike."""
    nq = [300]
    q, k, v, do = draw(nq, nq, 2, 2, D, seed=5)
    ramp = torch.linspace(0.1, 1, 300, device="cuda")[:, None, None]
    q, k = (q * size).bfloat16(), (k * ramp * size).bfloat16()
    want, tol = formula(q, k, v, do, nq, nq, True, scale or D ** -0.5)
    check(run(q, k, v, do, nq, nq, True, scale), want, tol)


@pytest.mark.parametrize("D", [64, 128])
def test_sequences_see_nothing_of_their_neighbours(D):
    nq = [150, 37, 210]
    q, k, v, do = draw(nq, nq, 2, 2, D, seed=9, packed=False)
    one = run(q, k, v, do, nq, nq)
    for bad in (math.nan, math.inf):
        b = [x.clone() for x in (q, k, v, do)]
        for x in b:
            x[:150] = bad
            x[187:] = bad
        two = run(*b, nq, nq)
        for n in one:
            s = (slice(None), slice(150, 187)) if n == "lse" else slice(150, 187)
            assert torch.equal(one[n][s], two[n][s]), n


def test_equal_inputs_give_equal_bits_on_any_stream():
    nq = [900, 33, 500]
    q, k, v, do = draw(nq, nq, 8, 2, 64, seed=3)
    one = run(q, k, v, do, nq, nq)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    at = dict(cu_q=offsets(nq), max_q=900, stream=side)
    o, lse = dpb.attention_forward(q, k, v, **at)
    dq, dk, dv = dpb.attention_backward(q, k, v, o, lse, do, **at)
    side.synchronize()
    for n, x in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        assert torch.equal(x, one[n]), n


def test_without_offsets_and_into_given_outputs():
    q, k, v, do = draw([333], [333], 4, 2, 64, seed=4)
    one = run(q, k, v, do, [333], [333])
    o, lse = dpb.attention_forward(q, k, v)
    assert torch.equal(o, one["o"]) and torch.equal(lse, one["lse"])
    # the gradients side by side in one buffer, rows that other data surrounds
    buf = torch.full((333, 9, 64), 7.0, device="cuda", dtype=torch.bfloat16)
    dpb.attention_backward(q, k, v, o, lse, do, grad_q=buf[:, :4], grad_k=buf[:, 4:6], grad_v=buf[:, 6:8])
    assert torch.equal(buf[:, :8], torch.cat([one["dq"], one["dk"], one["dv"]], 1)) and bool((buf[:, 8] == 7).all())


def test_offsets_that_pass_32_bits():
    """Rows 2^24 values apart: the last token lies beyond 2^31 values."""
    T, D, ts = 150, 64, 1 << 24
    buf = torch.empty(T * ts, dtype=torch.bfloat16, device="cuda")
    far = buf.as_strided((T, 1, 4 * D), (ts, 4 * D, 1))
    q, k, v, do = draw([T], [T], 1, 1, D, seed=6, packed=False)
    views = [far[:, :, i * D:(i + 1) * D] for i in range(4)]
    for x, y in zip(views, (q, k, v, do)):
        x.copy_(y)
    one, two = run(q, k, v, do, [T], [T]), run(*views, [T], [T])
    for n in one:
        assert torch.equal(one[n], two[n]), n


@pytest.mark.parametrize("cu", [[0, 50, 40, 120], [0, 50, 130, 120], [-3, 50, 90, 120], [0, 50, 120, 121]])
def test_bad_offsets_are_flagged_and_skipped(cu):
    q, k, v, do = draw([120], [120], 2, 2, 64, seed=7)
    cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    dpb.status()
    o = torch.full_like(q, 3.0)
    dpb.attention_forward(q, k, v, cu_q=cu, cu_k=cu, max_q=120, max_k=120, out=o)
    with pytest.raises(dpb.DPBError):
        dpb._check(6 if dpb.status() & dpb.DEV_BAD_LENGTH else 0)
    ok, _ = dpb.attention_forward(q, k, v, cu_q=torch.tensor([0, 50], dtype=torch.int32, device="cuda"), max_q=50)
    if int(cu[0]) == 0:  # the first sequence is sound, where no later one (sound by itself) claims its rows too
        rows = min(50, int(cu[2]))
        assert torch.equal(o[:rows], ok[:rows])
    assert dpb.status() == 0


def test_longer_than_announced_is_flagged():
    q, k, v, _ = draw([300], [300], 1, 1, 64)
    dpb.status()
    dpb.attention_forward(q, k, v, cu_q=offsets([300]), max_q=100, max_k=100)
    assert dpb.status() == dpb.DEV_BAD_LENGTH


def test_no_tokens():
    q = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    o, lse = dpb.attention_forward(q, q, q)
    assert o.shape == q.shape and lse.shape == (2, 0)
    k = torch.randn(5, 2, 64, device="cuda").bfloat16()
    dq, dk, dv = dpb.attention_backward(q, k, k, o, lse, q)
    assert dq.shape == q.shape and not dk.any() and not dv.any()


def test_gradients_against_differences():
    """The kernel's gradient along a direction against the 64-bit loss's central
    difference along it. Off by at most the sum over the direction of the
    element bounds, plus the difference's own error of order h^2."""
    nq, D = [90], 64
    q, k, v, do = draw(nq, nq, 2, 1, D, seed=8, packed=False)
    got = run(q, k, v, do, nq, nq)
    _, tol = formula(q, k, v, do, nq, nq, True, D ** -0.5)
    g = torch.Generator(device="cuda").manual_seed(1)

    def loss(*x):
        return float((formula(*x, do, nq, nq, True, D ** -0.5)[0]["o"] * do.double()).sum())

    for i, n in enumerate(("dq", "dk", "dv")):
        x = [t.double() for t in (q, k, v)]
        d = torch.randn(x[i].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-4
        up, down = [y.clone() for y in x], [y.clone() for y in x]
        up[i] += h * d
        down[i] -= h * d
        diff = (loss(*up) - loss(*down)) / (2 * h)
        assert abs(float((got[n].double() * d).sum()) - diff) <= float((tol[n] * d.abs()).sum()) + 1e-4 * abs(diff), n


def test_refusals():
    q = torch.zeros((8, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((8, 2, 64), dtype=torch.bfloat16, device="cuda")
    bad = [
        (dict(q=q.float()), ValueError), (dict(q=q[0]), ValueError), (dict(k=k[:, :, :32]), ValueError),
        (dict(v=k[:7]), ValueError), (dict(k=torch.zeros((8, 3, 64), dtype=torch.bfloat16, device="cuda")), ValueError),
        (dict(cu_q=torch.zeros(2, dtype=torch.int64, device="cuda")), ValueError),
        (dict(scale=0.0), dpb.DPBError), (dict(scale=-1.0), dpb.DPBError), (dict(scale=math.nan), dpb.DPBError),
        (dict(lse=torch.zeros(3, device="cuda")), ValueError),
        (dict(q=torch.zeros((8, 4, 128), dtype=torch.bfloat16, device="cuda")[:, :, ::2]), ValueError),
        (dict(q=torch.zeros((8, 4, 65), dtype=torch.bfloat16, device="cuda")[:, :, :64]), dpb.DPBError),
        (dict(q=torch.zeros(8 * 256 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(8, 4, 64)), dpb.DPBError),
        (dict(q=q.cpu()), ValueError),
    ]
    for kw, err in bad:
        at = dict(q=q, k=k, v=k)
        at.update(kw)
        with pytest.raises(err):
            dpb.attention_forward(**at)
    for D in (4, 12, 136):
        x = torch.zeros((8, 2, D), dtype=torch.bfloat16, device="cuda")
        with pytest.raises(dpb.DPBError):
            dpb.attention_forward(x, x, x)
    with pytest.raises(dpb.DPBError):
        dpb.attention_forward(q, k, k, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda"))


PARTS = [  # long tiles for few heads: their blocks are shared out over several thread blocks
    ([2500], [2500], 2, 1, 64, True),
    ([1400, 60], [1400, 2100], 4, 1, 128, False),
    ([1], [5000], 2, 2, 128, True),
    ([3000, 10], [100, 4000], 1, 1, 72, True),
]


@pytest.mark.parametrize("nq,nk,H,Hk,D,causal", PARTS)
def test_long_tiles_in_parts(nq, nk, H, Hk, D, causal):
    q, k, v, do = draw(nq, nk, H, Hk, D, seed=D + sum(nq))
    want, tol = formula(q, k, v, do, nq, nk, causal, D ** -0.5)
    got = run(q, k, v, do, nq, nk, causal)
    check(got, want, tol)
    again = run(q, k, v, do, nq, nk, causal)
    assert all(torch.equal(got[n], again[n]) for n in got)
    assert dpb.status() == 0


@pytest.mark.parametrize("cu", [[0, 50, 40, 120], [0, 50, 130, 120], [-3, 50, 90, 120], [0, 50, 120, 121]])
def test_bad_offsets_are_flagged_by_the_gradient(cu):
    q, k, v, do = draw([120], [120], 2, 2, 64, seed=7)
    cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    o, lse = dpb.attention_forward(q, k, v)
    assert dpb.status() == 0
    dpb.attention_backward(q, k, v, o, lse, do, cu_q=cu, cu_k=cu, max_q=120, max_k=120)
    assert dpb.status() == dpb.DEV_BAD_LENGTH


@pytest.mark.parametrize("D", [64, 128])
def test_sequences_of_very_unequal_lengths(D):
    nq, nk = [5, 2100, 0, 300, 1, 64, 129], [5, 2100, 0, 500, 3000, 64, 100]
    q, k, v, do = draw(nq, nk, 4, 2, D, seed=D)
    want, tol = formula(q, k, v, do, nq, nk, True, D ** -0.5)
    got = run(q, k, v, do, nq, nk)
    check(got, want, tol)
    again = run(q, k, v, do, nq, nk)
    assert all(torch.equal(got[n], again[n]) for n in got)
    assert dpb.status() == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rising", [True, False])
def test_sharp_softmax_in_parts(D, rising):
    """Parts whose maxima lie far apart, the largest in the last or in the first."""
    nq = [2600]
    q, k, v, do = draw(nq, nq, 1, 1, D, seed=11)
    ramp = torch.linspace(0.1, 4, 2600, device="cuda")[:, None, None]
    k = (k * (ramp if rising else ramp.flip(0))).bfloat16()
    want, tol = formula(q, k, v, do, nq, nq, True, D ** -0.5)
    check(run(q, k, v, do, nq, nq), want, tol)


@pytest.mark.parametrize("D", [64, 128])
def test_long_sequences_see_nothing_of_their_neighbours(D):
    nq, mine = [150, 2200, 2100], slice(150, 2350)
    q, k, v, do = draw(nq, nq, 2, 2, D, seed=9, packed=False)
    one = run(q, k, v, do, nq, nq)
    b = [x.clone() for x in (q, k, v, do)]
    for x in b:
        x[:150] = math.nan
        x[2350:] = math.nan
    two = run(*b, nq, nq)
    for n in one:
        s = (slice(None), mine) if n == "lse" else mine
        assert torch.equal(one[n][s], two[n][s]), n


def test_a_workspace_that_is_too_small_is_refused():
    q = torch.zeros((4096, 1, 64), dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    dpb.attention_forward(q, q, q, workspace=ws)  # needs the status word alone
    with pytest.raises(dpb.DPBError):
        dpb.attention_backward(q, q, q, q, torch.zeros((1, 4096), device="cuda"), q, workspace=ws)


@pytest.mark.parametrize("D", [64, 128])
def test_many_tiles_without_a_block(D):
    """Sequences whose rows see no key, between some that do: their tiles have no products to wait for."""
    nq, nk = [300] + [130] * 9 + [200], [300] + [0] * 9 + [64]
    q, k, v, do = draw(nq, nk, 4, 1, D, seed=12)
    want, tol = formula(q, k, v, do, nq, nk, True, D ** -0.5)
    check(run(q, k, v, do, nq, nk), want, tol)
    assert dpb.status() == 0


def test_heads_further_apart_than_tokens():
    """[heads][tokens][dim] memory: the head stride is the larger one."""
    q, k, v, do = draw([333], [333], 4, 2, 64, seed=4, packed=False)
    one = run(q, k, v, do, [333], [333])
    two = run(*(x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v, do)), [333], [333])
    assert all(torch.equal(one[n], two[n]) for n in one)


def test_longest_unannounced_and_many_short_sequences():
    """Without max_q the grid is for the sum of all lengths: equal bits with and without it."""
    nq = [(37 * i) % 100 for i in range(300)] + [1500] + [1, 700, 3]
    q, k, v, do = draw(nq, nq, 4, 2, 64, seed=13)
    want, tol = formula(q, k, v, do, nq, nq, True, 0.125)
    got = run(q, k, v, do, nq, nq)
    check(got, want, tol)
    o, lse = dpb.attention_forward(q, k, v, cu_q=offsets(nq))
    assert torch.equal(o, got["o"]) and torch.equal(lse, got["lse"])
    assert dpb.status() == 0


@pytest.mark.parametrize("D,nq", [(64, [900, 33, 500]), (128, [2500, 7])])
def test_in_a_cuda_graph(D, nq):
    """Forward and gradient captured once and replayed on other values."""
    one, two = draw(nq, nq, 4, 2, D, seed=14, packed=False), draw(nq, nq, 4, 2, D, seed=15, packed=False)
    want = [run(*x, nq, nq) for x in (one, two)]
    q, k, v, do = (x.clone() for x in one)
    at = dict(cu_q=offsets(nq), max_q=max(nq), workspace=torch.zeros(64 << 20, dtype=torch.uint8, device="cuda"))
    got = {}

    def step():
        got["o"], got["lse"] = dpb.attention_forward(q, k, v, **at)
        got["dq"], got["dk"], got["dv"] = dpb.attention_backward(q, k, v, got["o"], got["lse"], do, **at)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for values, w in ((two, want[1]), (one, want[0])):
        for x, y in zip((q, k, v, do), values):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], w[n]) for n in got)


def into_nan(q, k, v, do, cu_q, cu_k, **kw):
    """Forward and gradient into memory full of NaN."""
    at = dict(cu_q=torch.tensor(cu_q, dtype=torch.int32, device="cuda"), cu_k=torch.tensor(cu_k, dtype=torch.int32, device="cuda"),
              **kw)

    def nan(*like):
        return [torch.full(x.shape, math.nan, dtype=x.dtype, device="cuda") for x in like]

    o, = nan(q)
    lse = torch.full((q.shape[1], q.shape[0]), math.nan, device="cuda")
    dpb.attention_forward(q, k, v, **at, out=o, lse=lse)
    dq, dk, dv = nan(q, k, v)
    dpb.attention_backward(q, k, v, o, lse, do, **at, grad_q=dq, grad_k=dk, grad_v=dv)
    torch.cuda.synchronize()
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def gaps(x, cu, fill, dim=0):
    """x with `fill` outside of [cu[0], cu[-1])."""
    x = x.clone()
    x.narrow(dim, 0, cu[0]).fill_(fill)
    x.narrow(dim, cu[-1], x.shape[dim] - cu[-1]).fill_(fill)
    return x


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("before,nq,after", [(0, [130, 60], 70), (40, [130, 0, 257], 0), (300, [5], 5000), (1, [900, 1, 300], 1),
                                             (129, [], 300)])
def test_rows_outside_of_every_sequence(before, nq, after, D):
    """Padding before and after the sequences, of other sizes for the keys: zeros, lse -inf, no gradient, no flag, and the
    sequences' own results bit for bit those without padding, whatever the padding holds."""
    kb, ka = (7 * before) % 400, (3 * after) % 700
    q, k, v, do = draw([before, sum(nq), after], [kb, sum(nq), ka], 4, 2, D, seed=21, packed=False)
    for x, b, a in ((q, before, after), (k, kb, ka), (v, kb, ka), (do, before, after)):
        x[:b], x[x.shape[0] - a:] = math.nan, math.inf
    cq = [before + sum(nq[:i]) for i in range(len(nq) + 1)]
    ck = [kb + sum(nq[:i]) for i in range(len(nq) + 1)]
    got = into_nan(q, k, v, do, cq, ck, max_q=max(nq, default=0), max_k=max(nq, default=0))
    assert dpb.status() == 0
    for n, x in got.items():
        cu, fill, dim = ck if n in ("dk", "dv") else cq, -math.inf if n == "lse" else 0.0, 1 if n == "lse" else 0
        assert torch.equal(x, gaps(x, cu, fill, dim)), n
    if nq:
        sq, sk = slice(cq[0], cq[-1]), slice(ck[0], ck[-1])
        alone = run(q[sq], k[sk], v[sk], do[sq], nq, nq)
        for n, x in alone.items():
            assert torch.equal(x, got[n][:, sq] if n == "lse" else got[n][sk if n in ("dk", "dv") else sq]), n


@pytest.mark.parametrize("cu,longest,sound", [
    ([0, 50, 130, 120], 120, [(0, 50)]),            # an end beyond the last row, then a step back
    ([-3, 50, 90, 120], 120, [(50, 90), (90, 120)]),
    ([0, 50, 120, 121], 120, [(0, 50), (50, 120)]),
    ([0, 30, 110, 120], 40, [(0, 30), (110, 120)]),  # longer than announced
    ([30, 10, 20], 120, [(10, 20)]),
    ([90, 100, 20, 45, 5, 10], 120, [(90, 100), (20, 45), (5, 10)]),
    ([500, 700], 120, []), ([-9, -5], 120, []), ([200], 120, []),
])
def test_rows_of_skipped_sequences(cu, longest, sound):
    q, k, v, do = draw([120], [120], 2, 2, 64, seed=22)
    dpb.status()
    got = into_nan(q, k, v, do, cu, cu, max_q=longest, max_k=longest)
    assert dpb.status() == (dpb.DEV_BAD_LENGTH if len(sound) < len(cu) - 1 else 0)
    want = {n: torch.full_like(x, -math.inf if n == "lse" else 0.0) for n, x in got.items()}
    for a, b in sound:
        one = run(q[a:b], k[a:b], v[a:b], do[a:b], [b - a], [b - a])
        for n, x in one.items():
            (want[n][:, a:b] if n == "lse" else want[n][a:b]).copy_(x)
    # rows of a sound sequence that the way to another offset passes as well may hold zeros
    both = torch.zeros(120, dtype=torch.bool, device="cuda")
    for a, b in zip([0] + cu, cu + [120]):
        if (a, b) not in sound and max(a, 0) < min(b, 120):
            both[max(a, 0):min(b, 120)] = True
    for n in got:
        x, w = (t.transpose(0, 1) if n == "lse" else t for t in (got[n], want[n]))
        zero = torch.full_like(x, -math.inf if n == "lse" else 0.0)
        same, none = ((x == t).flatten(1).all(1) for t in (w, zero))
        assert bool((same | (none & both)).all()), n


def test_overlapping_sequences_leave_no_row_out():
    """The same rows given over and over: more pairs of tiles than sound offsets can have."""
    T = 4096
    q, k, v, do = draw([T], [T], 2, 1, 64, seed=23)
    dpb.status()
    got = into_nan(q, k, v, do, [0, T] * 8, [0, T] * 8, max_q=T, max_k=T)
    assert dpb.status() == dpb.DEV_BAD_LENGTH
    one = run(q, k, v, do, [T], [T])
    assert torch.equal(got["o"], one["o"]) and torch.equal(got["lse"], one["lse"])
    assert all(torch.isfinite(x).all() for n, x in got.items())


@pytest.mark.parametrize("D", [24, 32, 48, 56, 80, 88, 104, 112, 120])
@pytest.mark.parametrize("causal", [True, False])
def test_other_head_widths(D, causal):
    """Widths between those that the products have columns for."""
    nq, nk = [300, 1, 130], [300, 200, 257]
    q, k, v, do = draw(nq, nk, 4, 2, D, seed=D)
    want, tol = formula(q, k, v, do, nq, nk, causal, D ** -0.5)
    check(run(q, k, v, do, nq, nk, causal), want, tol)
    assert dpb.status() == 0


@pytest.mark.parametrize("lens", [[3, 130], [40] * 90, []])
def test_long_padding(lens):
    """Padding that is most of the rows, written by all blocks: by as many as there are sequences' tiles, or by more."""
    n, T = sum(lens), 30011
    q, k, v, do = draw([T], [T], 3, 1, 64, seed=24)
    cu = [2000 + sum(lens[:i]) for i in range(len(lens) + 1)]
    got = into_nan(q, k, v, do, cu, cu, max_q=max(lens, default=0), max_k=max(lens, default=0))
    assert dpb.status() == 0
    for name, x in got.items():
        assert torch.equal(x, gaps(x, cu, -math.inf if name == "lse" else 0.0, 1 if name == "lse" else 0)), name
    if n:
        rows = slice(2000, 2000 + n)
        alone = run(q[rows], k[rows], v[rows], do[rows], lens, lens)
        for name, x in alone.items():
            assert torch.equal(x, got[name][:, rows] if name == "lse" else got[name][rows]), name


def test_no_keys():
    q = torch.randn(300, 2, 64, device="cuda").bfloat16()
    got = into_nan(q, q[:0], q[:0], q, [0, 300], [0, 0])
    assert not got["o"].any() and not got["dq"].any() and bool((got["lse"] == -math.inf).all())
    assert got["dk"].shape == (0, 2, 64) and dpb.status() == 0
