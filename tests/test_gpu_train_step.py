"""The training step's operators together: the autograd functions, the
attention module, the optimiser and the ParityTransformer built from them."""
import copy

import numpy as np
import pytest
import torch
import torch.nn.functional as F

from paper_2607_20652_gb300 import build, dpb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build()
    dpb.load()


def plain(m, x, cu):
    """The module in 64 bits on packed rows."""
    w = {n: p.detach().double() for n, p in m.named_parameters()}
    qkv = (x @ w["qkv.weight"].T).view(-1, m.heads + 2 * m.kv_heads, m.dim)
    out = []
    for a, b in zip(cu[:-1], cu[1:]):
        q, k, v = qkv[a:b].split([m.heads, m.kv_heads, m.kv_heads], 1)
        if m.q_norm is not None:
            q, k = (t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6) * w[n] for t, n in ((q, "q_norm"), (k, "k_norm")))
        if m.cos is not None:
            c, s = (t[:b - a].double()[:, None] for t in (m.cos, m.sin))
            h = m.dim // 2
            q, k = (torch.cat([t[..., :h] * c - t[..., h:] * s, t[..., h:] * c + t[..., :h] * s], -1) for t in (q, k))
        k, v = (t.repeat_interleave(m.heads // m.kv_heads, 1) for t in (k, v))
        s = torch.einsum("ihd,jhd->hij", q, k) * m.dim ** -0.5
        s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device=s.device).triu(1), -torch.inf)
        out.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v))
    return torch.cat(out).flatten(1) @ w["out.weight"].T


@pytest.mark.parametrize("kv,qk_norm,rotary", [(4, True, True), (2, True, False), (1, False, True), (4, False, False)])
def test_module_and_its_gradients(kv, qk_norm, rotary):
    from paper_2607_20652_gb300.attention import Attention
    torch.manual_seed(0)
    m = Attention(256, 4, kv, qk_norm, rotary, context=128, device="cuda", dtype=torch.bfloat16)
    assert m.cos is None or m.cos.dtype == torch.float32
    x = torch.randn(3, 100, 256, device="cuda").bfloat16().requires_grad_()
    gy = torch.randn(3, 100, 256, device="cuda").bfloat16()
    y = m(x)
    y.backward(gy)
    xd = x.detach().double().view(-1, 256).requires_grad_()
    want = plain(m, xd, [0, 100, 200, 300])
    want.backward(gy.double().view(-1, 256))
    # bf16 throughout: the projections' outputs, q and k after their norm, P, dS and every gradient are each rounded by
    # at most 2^-8; independent, about ten of them in a row stay within ten times that
    assert float((y.double().view(-1, 256) - want).norm() / want.norm()) < 10 * 2.0 ** -8
    assert float((x.grad.double().view(-1, 256) - xd.grad).norm() / xd.grad.norm()) < 10 * 2.0 ** -8
    assert all(torch.isfinite(p.grad).all() and p.grad.any() for p in m.parameters())
    assert dpb.status() == 0


def test_packed_rows_equal_the_batch():
    from paper_2607_20652_gb300.attention import Attention
    torch.manual_seed(1)
    m = Attention(128, 2, device="cuda", dtype=torch.bfloat16, context=64)
    x = torch.randn(2, 50, 128, device="cuda").bfloat16()
    cu = torch.tensor([0, 50, 100], dtype=torch.int32, device="cuda")
    assert torch.equal(m(x).view(100, 128), m(x.view(100, 128), cu, 50))
    with pytest.raises(ValueError):
        m(torch.randn(1, 65, 128, device="cuda").bfloat16())


def test_functions_match_the_calls():
    from paper_2607_20652_gb300 import attention as A
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn(90, h, 64, device="cuda", generator=g).bfloat16().requires_grad_() for h in (4, 2, 2))
    w = torch.rand(64, device="cuda", generator=g).bfloat16().requires_grad_()
    cos, sin = dpb.rope_tables(90, 64)
    qr, kr = A.qk_norm_rope(q, k, w, w, cos, sin)
    o = A.attention(qr, kr, v)
    go = torch.randn(90, 4, 64, device="cuda", generator=g).bfloat16()
    o.backward(go)
    q1, k1 = dpb.qk_norm_rope(q.detach(), k.detach(), w.detach(), w.detach(), cos, sin)
    o1, lse = dpb.attention_forward(q1, k1, v.detach())
    dq, dk, dv = dpb.attention_backward(q1, k1, v.detach(), o1, lse, go)
    dq, dk, dwq, dwk = dpb.qk_norm_rope_backward(q.detach(), k.detach(), dq, dk, w.detach(), w.detach(), cos, sin)
    assert torch.equal(o, o1) and torch.equal(v.grad, dv) and torch.equal(q.grad, dq) and torch.equal(k.grad, dk)
    assert torch.equal(w.grad, dwq.bfloat16() + dwk.bfloat16())


@pytest.mark.parametrize("bits", [32, 8])
def test_optimiser_follows_torch(bits):
    """Ten steps beside torch's AdamW on the same gradients; one parameter joins late. 32-bit states: fp32 rounding only.
    8-bit states: a moment is off by at most a sixteenth each step, so a step by less than a fifth."""
    from paper_2607_20652_gb300.optim import AdamW
    torch.manual_seed(3)
    a = [torch.nn.Parameter(torch.randn(s, device="cuda")) for s in ((300, 7), (513,), (64, 64))]
    b = [torch.nn.Parameter(p.detach().clone()) for p in a]
    kw = dict(lr=1e-2, betas=(0.9, 0.95), weight_decay=0.1)
    mine, ref = AdamW(a, state_bits=bits, **kw), torch.optim.AdamW(b, **kw)
    for s in range(10):
        for p, r in zip(a, b):
            g = torch.randn_like(p) + 1
            p.grad, r.grad = (g, g.clone()) if s >= 2 or p is not a[1] else (None, None)
        mine.step()
        ref.step()
    for p, r in zip(a, b):
        tol = 1e-5 if bits == 32 else 0.2 * 10 * 1e-2
        assert float((p - r).abs().max()) < tol
    # states as torch's keep them, and a run that goes on from a saved state goes on the same
    keep = copy.deepcopy(mine.state_dict())
    c = [torch.nn.Parameter(p.detach().clone()) for p in a]
    other = AdamW(c, state_bits=bits, **kw)
    other.load_state_dict(keep)
    for p, q in zip(a, c):
        p.grad = torch.ones_like(p)
        q.grad = torch.ones_like(q)
    mine.step()
    other.step()
    assert all(torch.equal(p, q) for p, q in zip(a, c))


@pytest.mark.parametrize("bits,kv", [(32, 4), (8, 2)])
def test_small_parity_transformer_trains(bits, kv):
    from paper_2607_20652_gb300.optim import AdamW
    from paper_2607_20652_gb300.transformer import ParityTransformer
    dev = torch.device("cuda")
    torch.manual_seed(0)
    model = ParityTransformer(layers=2, d=64, heads=4, d_mlp=128, vocab=97, context=32, attention="dpb", kv_heads=kv,
                              dpb=dict(levels=3, m_bits=12, children=16, beam=8, k=8), device=dev)
    opt = AdamW(model.parameters(), lr=3e-3, state_bits=bits)
    g = torch.Generator().manual_seed(1)
    ids = torch.randint(0, 97, (4, 32), generator=g).to(dev)
    tgt = torch.randint(0, 97, (4, 32), generator=g).to(dev)
    losses = []
    for _ in range(30):
        opt.zero_grad(set_to_none=True)
        loss = model(ids, tgt)
        loss.backward()
        assert all(p.grad is None or torch.isfinite(p.grad).all() for p in model.parameters())
        opt.step()
        losses.append(float(loss.detach()))
    assert np.isfinite(losses).all() and losses[-1] < losses[0] - 0.5, losses
    assert dpb.status() == 0


def test_default_model_is_as_before():
    from paper_2607_20652_gb300.transformer import ParityTransformer
    torch.manual_seed(0)
    m = ParityTransformer(layers=1, d=64, heads=4, d_mlp=128, vocab=97, context=32, device="cuda")
    assert m.pos is not None and [n for n, _ in m.blocks[0].attn.named_parameters()] == ["qkv.weight", "out.weight"]
    for kw in (dict(attention="other"), dict(kv_heads=2)):
        with pytest.raises(ValueError):
            ParityTransformer(layers=1, d=64, heads=4, d_mlp=128, vocab=97, context=32, **kw)


def test_padding_takes_no_part_in_the_gradients():
    """A packed batch that ends in padding, in memory that held NaN before: outputs and every parameter's gradient are those
    of the batch without it (its sums in another order: fp32 sums of bf16 products, then one rounding to bf16)."""
    from paper_2607_20652_gb300.attention import Attention
    torch.manual_seed(5)
    m = Attention(256, 4, 2, context=256, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(700, 256, device="cuda").bfloat16()
    gy = torch.randn(700, 256, device="cuda").bfloat16()
    cu = torch.tensor([0, 100, 300, 410], dtype=torch.int32, device="cuda")

    def grads(rows):
        torch.cuda.empty_cache()
        poison = [torch.full((700, 1024), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(20)]
        del poison
        m.zero_grad(set_to_none=True)
        xr = x[:rows].clone().requires_grad_()
        y = m(xr, cu, 200)
        y.backward(gy[:rows])
        return y.detach(), xr.grad, {n: p.grad for n, p in m.named_parameters()}

    y, gx, gw = grads(700)
    y0, gx0, gw0 = grads(410)
    assert not y[410:].any() and not gx[410:].any()
    assert torch.equal(gx[:410], gx0) and torch.equal(y[:410], y0)
    for n, g in gw.items():
        assert float((g.double() - gw0[n].double()).abs().max()) <= 2.0 ** -7 * float(gw0[n].abs().max()), n
    assert dpb.status() == 0


def test_threads_on_one_stream():
    """Two threads enqueue gradients of different shapes on one stream: each gets what it gets alone."""
    import threading
    g = torch.Generator(device="cuda").manual_seed(7)
    work = []
    for lens, h, hk, d in (([900, 33, 500], 4, 2, 64), ([64, 2500, 7, 300], 8, 1, 128)):
        t = sum(lens)
        q, k, v, do = (torch.randn(t, n, d, device="cuda", generator=g).bfloat16() for n in (h, hk, hk, h))
        cu = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
        cos, sin = dpb.rope_tables(t, d)
        o, lse = dpb.attention_forward(q, k, v, cu_q=cu, max_q=max(lens))

        def step(q=q, k=k, v=v, do=do, o=o, lse=lse, cu=cu, longest=max(lens), cos=cos, sin=sin):
            return (*dpb.attention_backward(q, k, v, o, lse, do, cu_q=cu, max_q=longest),
                    *dpb.qk_norm_rope_backward(q, k, do, k, cos=cos, sin=sin))

        work.append(step)
    want = [f() for f in work]
    torch.cuda.synchronize()
    wrong = []

    def loop(f, w):
        for _ in range(150):
            got = f()
            if not all(torch.equal(a, b) for a, b in zip(got, w)):
                wrong.append(1)

    threads = [threading.Thread(target=loop, args=(f, w)) for f, w in zip(work, want) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and dpb.status() == 0


def test_module_in_a_cuda_graph():
    """A module's step captured without a workspace of its own; then larger calls on the capture's stream, memory given back
    and filled with other data, and the replay: the graph's scratch is still its own. Its status bits are found, too."""
    from paper_2607_20652_gb300.attention import Attention
    torch.manual_seed(6)
    m = Attention(256, 4, 2, context=4096, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(600, 256, device="cuda").bfloat16().requires_grad_()
    gy = torch.randn(600, 256, device="cuda").bfloat16()
    cu = torch.tensor([0, 450, 600], dtype=torch.int32, device="cuda")

    def step():
        y = m(x, cu, 450)
        return [y, *torch.autograd.grad(y, [x, *m.parameters()], gy)]

    want = [t.detach().clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    with torch.cuda.stream(side):
        big = torch.randn(4000, 256, device="cuda").bfloat16().requires_grad_()
        z = m(big, torch.tensor([0, 4000], dtype=torch.int32, device="cuda"), 4000)
        torch.autograd.grad(z, [big, *m.parameters()], torch.ones_like(z))
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    other = [torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    for t in got:
        t.detach().zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(bool((t == 7).all()) for t in other)
    assert dpb.status() == 0
    cu.copy_(torch.tensor([0, 700, 600]))
    graph.replay()
    assert dpb.status() == dpb.DEV_BAD_LENGTH and dpb.status() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_a_copied_or_resumed_optimiser_goes_on_the_same(bits):
    """A deep copy of model and optimiser, and a run resumed from saved states by an optimiser built with another seed: the
    next steps are the original's bit for bit, and the original is not touched by the others' steps."""
    from paper_2607_20652_gb300.optim import AdamW
    torch.manual_seed(9)
    ps = torch.nn.ParameterList([torch.nn.Parameter(torch.randn(n, device="cuda")) for n in (300, 5000)])
    opt = AdamW(ps.parameters(), lr=1e-2, state_bits=bits, seed=123)

    def steps(params, o, n, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for _ in range(n):
            for p in params:
                p.grad = torch.randn(p.shape, generator=g, device="cuda")
            o.step()

    def held(params, o):
        return [t.view(torch.uint8).clone() for p in params for t in (p.detach(), o.state[p]["exp_avg"], o.state[p]["exp_avg_sq"])]

    steps(ps, opt, 3, 1)
    ps2, opt2 = copy.deepcopy((ps, opt))
    ps3 = torch.nn.ParameterList([torch.nn.Parameter(p.detach().clone()) for p in ps])
    opt3 = AdamW(ps3.parameters(), lr=1e-2, state_bits=bits, seed=77)
    opt3.load_state_dict(opt.state_dict())
    before = held(ps, opt)
    steps(ps2, opt2, 2, 2)
    steps(ps3, opt3, 2, 2)
    assert all(torch.equal(a, b) for a, b in zip(held(ps, opt), before))
    steps(ps, opt, 2, 2)
    for params, o in ((ps2, opt2), (ps3, opt3)):
        assert all(torch.equal(a, b) for a, b in zip(held(ps, opt), held(params, o)))


def test_a_captured_optimiser_step_is_refused():
    """A replay would repeat one step's bias corrections: refused before anything is counted or launched."""
    from paper_2607_20652_gb300.optim import AdamW
    p = torch.nn.Parameter(torch.ones(300, device="cuda"))
    opt = AdamW([p], lr=1e-2)
    p.grad = torch.ones_like(p)
    opt.step()
    keep = p.detach().clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other = p.detach() + 1
        with pytest.raises(RuntimeError, match="captured"):
            opt.step()
    graph.replay()
    torch.cuda.synchronize()
    assert opt.state[p]["step"] == 1 and torch.equal(p.detach(), keep) and torch.equal(other, keep + 1)
    opt.step()
    assert opt.state[p]["step"] == 2 and not torch.equal(p.detach(), keep)


def test_second_derivatives_are_refused():
    """A gradient penalty must not lose its term silently."""
    from paper_2607_20652_gb300 import attention as A
    m = A.Attention(128, 2, device="cuda", dtype=torch.bfloat16, context=32)
    q = torch.randn(20, 2, 64, device="cuda").bfloat16().requires_grad_()
    x = torch.randn(1, 20, 128, device="cuda").bfloat16().requires_grad_()
    for y, of in ((A.attention(q, q, q), q), (A.qk_norm_rope(q, q)[0], q), (m(x), x)):
        loss = (y.float() ** 2).sum()
        g, = torch.autograd.grad(loss, of, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            (loss + (g.float() ** 2).sum()).backward()


def test_offsets_changed_before_the_backward_are_noticed():
    """Offsets are kept for the backward as the inputs are: changed in place, they raise as an input does."""
    from paper_2607_20652_gb300 import attention as A
    torch.manual_seed(3)
    m = A.Attention(128, 2, device="cuda", dtype=torch.bfloat16, context=128)
    q = torch.randn(100, 2, 64, device="cuda").bfloat16().requires_grad_()
    for call in (lambda cu: A.attention(q, q, q, cu, max_q=100), lambda cu: A.attention(q, q, q, cu, cu.clone(), 100, 100),
                 lambda cu: m(q.flatten(1), cu, 100)):
        cu = torch.tensor([0, 50, 100], dtype=torch.int32, device="cuda")
        want, = torch.autograd.grad(call(cu).float().sum(), q)
        y = call(cu)
        cu[1] = 30
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.float().sum().backward()
        cu[1] = 50
        assert torch.equal(torch.autograd.grad(call(cu).float().sum(), q)[0], want)


def test_a_gradient_at_any_address():
    """An output that is one part of a longer vector gets its gradient as a part of that vector's, at an address that no vector
    load takes."""
    from paper_2607_20652_gb300 import attention as A
    torch.manual_seed(4)
    q = torch.randn(20, 2, 64, device="cuda").bfloat16().requires_grad_()
    gy = torch.randn(3 + 20 * 128, device="cuda").bfloat16()
    odd, = torch.autograd.grad(torch.cat([gy[:3], A.attention(q, q, q).flatten()]), q, gy)
    want, = torch.autograd.grad(A.attention(q, q, q), q, gy[3:].clone().view(20, 2, 64))
    assert torch.equal(odd, want)


def test_fp32_parameters_under_autocast():
    """The module with fp32 parameters under bf16 autocast computes what it does in bf16, keeps its gradients in fp32, and
    follows steps far below bf16's spacing."""
    from paper_2607_20652_gb300 import attention as A
    from paper_2607_20652_gb300.optim import AdamW
    torch.manual_seed(8)
    m = A.Attention(128, 2, 1, device="cuda", context=64)
    with torch.no_grad():
        for p in (m.q_norm, m.k_norm):
            p.copy_(1 + 0.3 * torch.randn_like(p))
    low = copy.deepcopy(m).bfloat16()
    x, gy = torch.randn(2, 50, 128, device="cuda"), torch.randn(2, 50, 128, device="cuda").bfloat16()
    with torch.autocast("cuda", torch.bfloat16):
        y = m(x)
    y.backward(gy)
    z = low(x.bfloat16())
    z.backward(gy)
    assert y.dtype == torch.bfloat16 and torch.equal(y, z)
    for (n, p), r in zip(m.named_parameters(), low.parameters()):
        assert p.grad.dtype == torch.float32 and torch.equal(p.grad.bfloat16(), r.grad), n
    q = torch.randn(30, 2, 64, device="cuda").bfloat16().requires_grad_()
    wq = torch.rand(64, device="cuda").requires_grad_()
    A.qk_norm_rope(q, q, wq, None)[0].float().sum().backward()
    wr = wq.detach().bfloat16().requires_grad_()
    A.qk_norm_rope(q, q, wr, None)[0].float().sum().backward()
    assert torch.equal(wq.grad.bfloat16(), wr.grad)
    before = m.q_norm.detach().clone()
    AdamW(m.parameters(), lr=1e-5, weight_decay=0.0).step()
    moved = (m.q_norm.detach() - before).abs()
    assert bool((moved > 0.9e-5).all()) and bool((moved < 1.1e-5).all())


def test_sequences_beyond_the_tables_are_refused():
    """Whether their length is given or not; without a length, and more rows than the tables have, it is read from the offsets."""
    from paper_2607_20652_gb300.attention import Attention
    torch.manual_seed(2)
    m = Attention(128, 2, device="cuda", dtype=torch.bfloat16, context=64)
    x = torch.randn(200, 128, device="cuda").bfloat16()
    offsets = lambda *n: torch.tensor(n, dtype=torch.int32, device="cuda")
    for longest in (100, None):
        with pytest.raises(ValueError, match="rotary tables"):
            m(x, offsets(0, 50, 150, 200), longest)
    cu = offsets(0, 50, 114, 178)
    assert torch.equal(m(x, cu), m(x, cu, 64))
    assert not m(x, offsets(7)).any()
    plain = Attention(128, 2, rotary=False, device="cuda", dtype=torch.bfloat16)
    assert plain(x, offsets(0, 200)).shape == x.shape
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError, match="longest is needed"):
            m(x, cu)
    assert dpb.status() == 0


@pytest.mark.parametrize("kv,qk_norm,rotary", [(4, True, True), (2, True, False), (1, False, True), (1, True, True)])
def test_gradients_of_the_parameters(kv, qk_norm, rotary):
    """Each parameter's gradient against the module in 64 bits with differentiable weights; the norms' weights differ, so
    that neither gradient can stand for the other. Bound as for the module's gradients above."""
    from paper_2607_20652_gb300.attention import Attention
    torch.manual_seed(10)
    m = Attention(256, 4, kv, qk_norm, rotary, context=128, device="cuda", dtype=torch.bfloat16)
    if qk_norm:
        with torch.no_grad():
            m.q_norm.copy_(1 + 0.5 * torch.randn(64, device="cuda"))
            m.k_norm.copy_(1 - 0.5 * torch.randn(64, device="cuda"))
    cu = [0, 100, 101, 220, 300]
    x = torch.randn(300, 256, device="cuda").bfloat16()
    gy = torch.randn(300, 256, device="cuda").bfloat16()
    m(x, torch.tensor(cu, dtype=torch.int32, device="cuda"), 119).backward(gy)
    w = {n: p.detach().double().requires_grad_() for n, p in m.named_parameters()}

    class Double:  # what plain() reads of a module
        heads, kv_heads, dim, cos, sin, q_norm = m.heads, m.kv_heads, m.dim, m.cos, m.sin, m.q_norm

        @staticmethod
        def named_parameters():
            return [(n, Kept(p)) for n, p in w.items()]

    class Kept:
        def __init__(self, p):
            self.p = p

        def detach(self):
            return self

        def double(self):
            return self.p

    want = dict(zip(w, torch.autograd.grad(plain(Double, x.double(), cu), list(w.values()), gy.double())))
    for n, p in m.named_parameters():
        assert float((p.grad.double() - want[n]).norm() / want[n].norm()) < 10 * 2.0 ** -8, n


def test_functions_keep_the_norms_apart():
    """Different weights for queries and keys: each gets its own gradient, bit for bit the call's."""
    from paper_2607_20652_gb300 import attention as A
    g = torch.Generator(device="cuda").manual_seed(12)
    q, k = (torch.randn(90, h, 64, device="cuda", generator=g).bfloat16().requires_grad_() for h in (4, 2))
    wq, wk = (torch.rand(64, device="cuda", generator=g).bfloat16().requires_grad_() for _ in range(2))
    cos, sin = dpb.rope_tables(90, 64)
    gq, gk = (torch.randn(x.shape, device="cuda", generator=g).bfloat16() for x in (q, k))
    torch.autograd.backward(A.qk_norm_rope(q, k, wq, wk, cos, sin), (gq, gk))
    want = dpb.qk_norm_rope_backward(q.detach(), k.detach(), gq, gk, wq.detach(), wk.detach(), cos, sin)
    for x, y in zip((q, k, wq, wk), want):
        assert torch.equal(x.grad, y.to(x.dtype))
    assert not torch.equal(wq.grad, wk.grad)


def test_groups_that_change():
    """A group or a parameter taken out of the optimiser stays as it is, and the others go on with their own numbers."""
    from paper_2607_20652_gb300.optim import AdamW
    ps = [torch.nn.Parameter(torch.zeros(300, device="cuda")) for _ in range(4)]
    opt = AdamW([{"params": ps[:1], "lr": 1.0}, {"params": ps[1:3], "lr": 1e-3}, {"params": ps[3:], "lr": 1e-2}],
                weight_decay=0.0)

    def moved():
        before = [float(p[0]) for p in ps]
        for p in ps:
            p.grad = torch.ones_like(p)
        opt.step()
        return [round(b - float(p[0]), 6) for p, b in zip(ps, before)]

    assert moved() == [1.0, 0.001, 0.001, 0.01]
    del opt.param_groups[0]
    assert moved() == [0.0, 0.001, 0.001, 0.01]
    opt.param_groups[0]["params"] = ps[2:3]
    assert moved() == [0.0, 0.0, 0.001, 0.01]
    opt.param_groups[1]["params"][0] = ps[0]
    assert moved() == [0.01, 0.0, 0.001, 0.0]
