"""Embedding lookup and its gradient by sorted tokens against the definitions in 64 bits.

Bounds: a looked-up value is one product (2^-24), rounded to its type; a row of
the gradient is a fp32 sum of its n tokens' rows, off by at most n 2^-24 of
their absolute values' sum, times the scale (2^-24) and rounded to its type.
"""
import math

import pytest
import torch

from paper_2607_20652_gb300 import build, dpb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build()
    dpb.load()


def ulp(t):
    return 2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -24


def draw_ids(kind, T, V, g):
    if kind == "same":
        return torch.full((T,), V - 1, device="cuda")
    if kind == "few":
        return torch.randint(0, min(V, 3), (T,), generator=g, device="cuda") * max(1, (V - 1) // 3)
    if kind == "frequent":
        return ((V + 1.0) ** torch.rand(T, generator=g, device="cuda", dtype=torch.float64) - 1).long().clamp(0, V - 1)
    return torch.randint(0, V, (T,), generator=g, device="cuda")


SIZES = [  # tokens, words, columns
    (1, 1, 1), (1, 50257, 64), (5, 3, 7), (128, 97, 64), (255, 255, 16), (256, 256, 33), (1000, 65536, 24), (2049, 5003, 500),
    (40000, 700, 8), (70001, 300, 5), (16385, 2000, 130), (300, 1000, 1100), (3000, 16777217, 1),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,d", SIZES)
def test_lookup(T, V, d, dtype):
    g = torch.Generator(device="cuda").manual_seed(T)
    w = torch.randn(V, d, generator=g, device="cuda").to(dtype)
    for kind, scale in (("any", 1.0), ("frequent", math.sqrt(d))):
        ids = draw_ids(kind, T, V, g)
        y = dpb.embedding(w, ids, scale=scale)
        want = w.double()[ids] * scale
        assert ((y.double() - want).abs() <= (ulp(y) + 2.0 ** -23) * want.abs()).all() if scale != 1 else torch.equal(y, w[ids])
        assert torch.equal(y, dpb.embedding(w, ids.int(), scale=scale))
    assert dpb.status() == 0


def check_gradient(got, dy, ids, V, scale):
    n = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, ids, torch.ones_like(ids, dtype=torch.float64))
    at = torch.zeros(V, dy.shape[1], dtype=torch.float64, device="cuda")
    want = at.clone().index_add_(0, ids, dy.double()) * scale
    size = at.index_add_(0, ids, dy.double().abs()) * scale
    tol = (n[:, None] + 2) * 2.0 ** -24 * size + ulp(got) * want.abs()
    assert ((got.double() - want).abs() <= tol).all()
    assert not got[n == 0].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["any", "same", "few", "frequent"])
@pytest.mark.parametrize("T,V,d", SIZES)
def test_gradient(T, V, d, kind, dtype):
    g = torch.Generator(device="cuda").manual_seed(T + 1)
    dy = torch.randn(T, d, generator=g, device="cuda").to(dtype)
    ids = draw_ids(kind, T, V, g)
    scale = 1.0 if kind != "few" else 1.7
    dw = dpb.embedding_backward(dy, ids, V, scale=scale)
    check_gradient(dw, dy, ids, V, float(torch.tensor(scale, dtype=torch.float32)))
    assert torch.equal(dw, dpb.embedding_backward(dy, ids.int(), V, scale=scale))  # the same bits again
    assert dpb.status() == 0


@pytest.mark.parametrize("T", [0, 1, 7, 8, 9, 31, 32, 33, 64, 16384, 16385, 16416])
def test_lengths_at_the_stretches_ends(T):
    dy = torch.randn(T, 8, device="cuda")
    for ids in (torch.arange(T, device="cuda") // 8, torch.arange(T, device="cuda") // 32, torch.arange(T, device="cuda") // 40,
                torch.zeros(T, dtype=torch.long, device="cuda")):
        check_gradient(dpb.embedding_backward(dy, ids, 2200), dy, ids, 2200, 1.0)


@pytest.mark.parametrize("T", [65535, 65536, 65537, 131072, 131073, 196609])
def test_many_tokens(T):
    """Either side of where the sort holds 4 and 8 tokens a lane; two passes of it, and three."""
    dy = torch.randn(T, 8, device="cuda").bfloat16()
    g = torch.Generator(device="cuda").manual_seed(T)
    for V in (50257, 70000):
        for kind in ("any", "frequent"):
            ids = draw_ids(kind, T, V, g)
            check_gradient(dpb.embedding_backward(dy, ids, V), dy, ids, V, 1.0)


def test_the_order_of_a_rows_sum_is_the_tokens():
    """2^24 + 1 - 2^24: what a fp32 sum in the tokens' order gives, within one stretch."""
    dy = torch.tensor([2.0 ** 24, 1.0, -2.0 ** 24], device="cuda")[:, None].contiguous()
    ids = torch.tensor([4, 4, 4], device="cuda")
    assert float(dpb.embedding_backward(dy, ids, 9)[4, 0]) == 0.0
    assert float(dpb.embedding_backward(dy[[0, 2, 1]], ids, 9)[4, 0]) == 1.0


def test_no_tokens():
    w = torch.randn(50, 24, device="cuda")
    none = torch.empty(0, dtype=torch.long, device="cuda")
    assert dpb.embedding(w, none).shape == (0, 24)
    dw = dpb.embedding_backward(torch.empty(0, 24, device="cuda"), none, 50)
    assert dw.shape == (50, 24) and not dw.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ids_out_of_range_are_flagged(dtype):
    w = torch.randn(50, 24, device="cuda").to(dtype)
    ids = torch.randint(0, 50, (300,), device="cuda")
    ids[[0, 100, 299]] = torch.tensor([50, -1, 1 << 40], device="cuda")
    dpb.status()
    y = dpb.embedding(w, ids)
    assert dpb.status() == dpb.DEV_BAD_INDEX
    ok = (ids >= 0) & (ids < 50)
    assert torch.equal(y[ok], w[ids[ok]]) and not y[~ok].any()
    dy = torch.randn(300, 24, device="cuda").to(dtype)
    dw = dpb.embedding_backward(dy, ids, 50)
    assert dpb.status() == dpb.DEV_BAD_INDEX
    check_gradient(dw, dy[ok], ids[ok], 50, 1.0)
    dw = dpb.embedding_backward(dy, torch.full((300,), -7, device="cuda"), 50)
    assert dpb.status() == dpb.DEV_BAD_INDEX and not dw.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d,stride,first", [(24, 40, 8), (24, 33, 0), (24, 40, 3), (7, 9, 1), (64, 64, 0)])
def test_strides_and_addresses(d, stride, first, dtype):
    V, T = 300, 500
    wide = torch.randn(V * stride + first, device="cuda").to(dtype)
    w = wide[first:].as_strided((V, d), (stride, 1), first)
    ids = torch.randint(0, V, (T,), device="cuda")
    out = torch.full((T * stride + first,), 3.0, device="cuda", dtype=dtype)
    y = out.as_strided((T, d), (stride, 1), first)
    dpb.embedding(w, ids, out=y)
    assert torch.equal(y, w[ids])
    grad = torch.full((V * stride + first,), 3.0, device="cuda", dtype=dtype)
    dw = grad.as_strided((V, d), (stride, 1), first)
    dpb.embedding_backward(y, ids, V, grad_weight=dw)
    check_gradient(dw, y, ids, V, 1.0)
    for t, rows in ((out, T), (grad, V)):
        inside = torch.zeros_like(t, dtype=torch.bool)
        inside.as_strided((rows, d), (stride, 1), first)[:] = True
        assert (t[~inside] == 3).all()


def test_values_that_are_not_finite_stay_in_their_rows():
    dy = torch.randn(3000, 24, device="cuda").bfloat16()
    ids = torch.randint(0, 50, (3000,), device="cuda")
    dy[ids == 9] = float("nan")
    dy[ids == 11] = float("inf")
    dw = dpb.embedding_backward(dy, ids, 50)
    assert dw[9].isnan().all() and (dw[11] == float("inf")).all()
    rest = (ids != 9) & (ids != 11)
    check_gradient(torch.cat([dw[:9], dw[10:11], dw[12:]]), dy[rest],
                   (ids - (ids > 9).long() - (ids > 11).long())[rest], 48, 1.0)


def test_offsets_past_32_bits():
    """A weight of 2^31 + values: rows at both ends are found."""
    V, d = (1 << 31) // 1024 + 5, 1024
    w = torch.zeros(V, d, device="cuda", dtype=torch.bfloat16)
    w[-1], w[0] = 2.0, 1.0
    ids = torch.tensor([V - 1, 0, V - 1, V - 2], device="cuda")
    y = dpb.embedding(w, ids)
    assert (y[0] == 2).all() and (y[1] == 1).all() and (y[2] == 2).all() and not y[3].any()
    dw = dpb.embedding_backward(y, ids, V, grad_weight=w)
    assert (dw[-1] == 4).all() and (dw[0] == 1).all() and not dw[1:-1].any()


def test_scratch_another_stream_and_a_graph():
    V, T, d = 300, 5000, 40
    ids, dy = torch.randint(0, V, (T,), device="cuda"), torch.randn(T, d, device="cuda")
    want = dpb.embedding_backward(dy, ids, V)
    ws = torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda")
    ws[:4] = 0
    assert torch.equal(want, dpb.embedding_backward(dy, ids, V, workspace=ws)) and dpb.workspace_status(ws) == 0
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = dpb.embedding_backward(dy, ids, V, stream=s)
    y = dpb.embedding(want, ids, stream=s)
    s.synchronize()
    assert torch.equal(got, want) and torch.equal(y, want[ids])
    graph = torch.cuda.CUDAGraph()
    i2, w2 = torch.randint(0, V, (T,), device="cuda"), torch.randn(V, d, device="cuda")
    ids_in = ids.clone()
    with torch.cuda.graph(graph):
        y = dpb.embedding(w2, ids_in)
        dw = dpb.embedding_backward(y, ids_in, V)
    for i in (i2, ids):
        ids_in.copy_(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, w2[i])
        check_gradient(dw, w2[i], i, V, 1.0)


def test_refusals():
    w, ids = torch.randn(50, 24, device="cuda"), torch.randint(0, 50, (30,), device="cuda")
    for bad in (dict(weight=w.half()), dict(ids=ids.float()), dict(ids=ids[::2]), dict(ids=ids.cpu()), dict(weight=w[0]),
                dict(ids=ids[:, None]), dict(weight=w[:, ::2]), dict(out=w), dict(scale=float("inf"))):
        with pytest.raises((ValueError, dpb.DPBError)):
            dpb.embedding(**(dict(weight=w, ids=ids) | bad))
    dy = torch.randn(30, 24, device="cuda")
    for bad in (dict(grad_out=dy.half()), dict(grad_out=dy[:20]), dict(vocab=0), dict(grad_weight=w[:20]), dict(ids=ids.int()[::2]),
                dict(scale=float("nan")), dict(workspace=torch.zeros(512, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, dpb.DPBError)):
            dpb.embedding_backward(**(dict(grad_out=dy, ids=ids, vocab=50) | bad))


def test_gradient_offsets_past_32_bits():
    """Rows of 2^31 values and more, of ones: each word's count, exact in fp32."""
    T, V, d = (1 << 21) + 77, 5003, 1024
    ids = torch.randint(0, V, (T,), device="cuda")
    dw = dpb.embedding_backward(torch.ones(T, d, device="cuda"), ids, V)
    assert (dw == torch.bincount(ids, minlength=V).float()[:, None]).all()
    w = torch.arange(V, device="cuda", dtype=torch.float32)[:, None].expand(V, d).contiguous()
    assert (dpb.embedding(w, ids) == ids.float()[:, None]).all()
