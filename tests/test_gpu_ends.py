"""The operators at both ends of the model and of the residual, together: the
autograd functions, the modules, and the ParityTransformer that uses them."""
import copy
import threading

import pytest
import torch
import torch.nn.functional as F

from paper_2607_20652_gb300 import build, dpb

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _library():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build()
    dpb.load()


def rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


def test_functions_match_the_calls():
    from paper_2607_20652_gb300 import ends
    torch.manual_seed(0)
    w = torch.randn(97, 64, device="cuda").to(BF).requires_grad_()
    ids, y = torch.randint(0, 97, (3, 20), device="cuda"), torch.randint(0, 97, (3, 20), device="cuda")
    y[0, :7] = -100
    e = ends.embedding(w, ids, 2.0)
    assert torch.equal(e, dpb.embedding(w.detach(), ids.view(-1), 2.0).view(3, 20, 64))
    g = torch.randn_like(e)
    dw, = torch.autograd.grad(e, w, g)
    assert torch.equal(dw, dpb.embedding_backward(g.view(-1, 64), ids.view(-1), 97, 2.0))

    x, d, k = (torch.randn(3, 20, 64, device="cuda").to(BF).requires_grad_() for _ in range(3))
    nw = torch.randn(64, device="cuda").to(BF).requires_grad_()
    n, total = ends.add_norm(x, d, nw, 1e-5)
    gn, gt = torch.randn_like(n), torch.randn_like(n)
    grads = torch.autograd.grad((n, total), (x, d, nw), (gn, gt))
    want, gw = dpb.add_norm_backward(total.detach().view(-1, 64), gn.view(-1, 64), gt.view(-1, 64), nw.detach(), 1e-5)
    assert torch.equal(grads[0].view(-1, 64), want) and torch.equal(grads[1], grads[0]) and torch.equal(grads[2], gw.to(BF))
    # one output's gradient alone
    n, total = ends.add_norm(x, d, nw)
    assert all(torch.equal(a, gt) for a in torch.autograd.grad(total, (x, d), gt))
    n, same = ends.add_norm(k, None, nw)
    assert same is k
    dk, = torch.autograd.grad(n, k, gn)
    assert torch.equal(dk.view(-1, 64), dpb.add_norm_backward(k.detach().view(-1, 64), gn.view(-1, 64), weight=nw.detach())[0])

    h = torch.randn(3, 20, 64, device="cuda").to(BF).requires_grad_()
    loss, lse = dpb.linear_cross_entropy_forward(h.detach().view(-1, 64), w.detach(), y.view(-1))
    none = ends.linear_cross_entropy(h, w, y, reduction="none")
    assert torch.equal(none.view(-1), loss)
    for red, total, weight in (("none", None, torch.randn(3, 20, device="cuda")), ("sum", loss.sum(), None),
                               ("mean", loss.sum() / 53, None)):
        got = ends.linear_cross_entropy(h, w, y, reduction=red)
        assert total is None or torch.equal(got, total)
        dh, dw = torch.autograd.grad(got, (h, w), weight)
        gl = weight.view(-1) if red == "none" else torch.full((1,), 1.0, device="cuda").div(53 if red == "mean" else 1).expand(60)
        want = dpb.linear_cross_entropy_backward(h.detach().view(-1, 64), w.detach(), y.view(-1), lse, gl)
        assert torch.equal(dh.view(-1, 64), want[0]) and torch.equal(dw, want[1])
    hd, wd = h.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    ref = F.cross_entropy((hd @ wd.t()).view(-1, 97), y.view(-1))
    ref.backward()
    # dz and the result rounded to bf16, 2^-8 each; the loss a mean of fp32 sums
    assert abs(float(got.detach()) - float(ref.detach())) < 2.0 ** -18 * float(ref.detach())
    assert rel(dh, hd.grad) < 2.0 ** -7 and rel(dw, wd.grad) < 2.0 ** -7


def test_gradients_of_any_layout():
    """Gradients that come expanded, transposed or at an odd address, and a weight that is a view."""
    from paper_2607_20652_gb300 import ends
    torch.manual_seed(1)
    w = torch.randn(64, 97, device="cuda").to(BF).requires_grad_()
    ids = torch.randint(0, 97, (50,), device="cuda")
    want = torch.zeros(97, 64, device="cuda").index_add_(0, ids, torch.ones(50, 64, device="cuda"))
    got, = torch.autograd.grad(ends.embedding(w.t(), ids).float().sum(), w)
    assert torch.equal(got.t().float(), want)
    x, d = (torch.randn(50, 64, device="cuda").to(BF).requires_grad_() for _ in range(2))
    odd = torch.randn(50 * 64 + 1, device="cuda").to(BF)[1:].view(50, 64)
    for gy, gt in ((torch.ones((), device="cuda", dtype=BF).expand(50, 64), None), (odd, odd),
                   (torch.randn(64, 50, device="cuda").to(BF).t(), None)):
        n, total = ends.add_norm(x, d)
        outs = (n,) if gt is None else (n, total)
        dx, = torch.autograd.grad(outs, x, (gy,) if gt is None else (gy, gt))
        assert torch.equal(dx, dpb.add_norm_backward(total.detach(), gy.contiguous().clone(),
                                                     None if gt is None else gt.clone(), weight_grad=False)[0])
    # hidden rows and a weight at odd addresses
    h = torch.randn(50 * 64 + 1, device="cuda").to(BF)[1:].view(50, 64)
    v = torch.randn(97, 70, device="cuda").to(BF)[:, 3:67]
    y = torch.randint(0, 97, (50,), device="cuda")
    hh, vv = h.clone().requires_grad_(), v.clone().requires_grad_()
    a, b = ends.linear_cross_entropy(hh, vv, y), ends.linear_cross_entropy(h.requires_grad_(), v.requires_grad_(), y)
    assert torch.equal(a, b)
    for p, q in zip(torch.autograd.grad(a, (hh, vv)), torch.autograd.grad(b, (h, v))):
        assert torch.equal(p, q)


def test_shifted_targets_and_strided_indices():
    """The next token's loss: parts of the batch's rows and ids, and indices that are not dense."""
    from paper_2607_20652_gb300 import ends
    torch.manual_seed(3)
    h, w = torch.randn(4, 33, 64, device="cuda").to(BF), torch.randn(97, 64, device="cuda").to(BF)
    ids = torch.randint(0, 97, (4, 33), device="cuda")
    hh = h.clone().requires_grad_()
    loss = ends.linear_cross_entropy(hh[:, :-1], w, ids[:, 1:])
    want = ends.linear_cross_entropy(h[:, :-1].contiguous().requires_grad_(), w, ids[:, 1:].contiguous())
    assert torch.equal(loss, want)
    loss.backward()
    assert hh.grad[:, :-1].any() and not hh.grad[:, -1].any()
    wide = torch.randint(0, 97, (40,), device="cuda")
    assert torch.equal(ends.embedding(w, wide[::2]), w[wide[::2]])
    x = h[0, :20].clone().requires_grad_()
    torch.autograd.grad(ends.linear_cross_entropy(x, w, wide[::2]), x)
    g, = torch.autograd.grad(ends.embedding(w.requires_grad_(), wide[::2]), w, torch.ones(20, 64, device="cuda", dtype=BF))
    assert torch.equal(g.float(), torch.zeros(97, 64, device="cuda").index_add_(0, wide[::2], torch.ones(20, 64, device="cuda")))


def test_means_without_tokens():
    from paper_2607_20652_gb300 import ends
    h, w = torch.randn(20, 64, device="cuda").to(BF).requires_grad_(), torch.randn(97, 64, device="cuda").to(BF).requires_grad_()
    y = torch.full((20,), -100, device="cuda")
    loss = ends.linear_cross_entropy(h, w, y)
    assert loss.isnan()
    assert not any(g.any() for g in torch.autograd.grad(loss, (h, w)))
    loss = ends.linear_cross_entropy(h, w, y, reduction="sum")
    assert float(loss.detach()) == 0 and not any(g.any() for g in torch.autograd.grad(loss, (h, w)))
    none = ends.linear_cross_entropy(h[:0], w, y[:0], reduction="sum")
    assert float(none.detach()) == 0 and not any(g.any() for g in torch.autograd.grad(none, (h, w)))


def test_frozen_parts_and_fp32_parameters():
    from paper_2607_20652_gb300 import ends
    torch.manual_seed(2)
    h, y = torch.randn(40, 64, device="cuda").to(BF), torch.randint(0, 97, (40,), device="cuda")
    w = torch.randn(97, 64, device="cuda")
    for a, b in ((True, False), (False, True)):
        hh, ww = h.clone().requires_grad_(a), w.clone().requires_grad_(b)
        ends.linear_cross_entropy(hh, ww, y).backward()
        assert (hh.grad is not None) == a and (ww.grad is not None) == b
        if b:
            assert ww.grad.dtype == torch.float32
            full = w.to(BF).requires_grad_()
            ends.linear_cross_entropy(h, full, y).backward()
            assert torch.equal(ww.grad, full.grad.float())
    m = ends.AddRMSNorm(64, device="cuda")
    n, _ = m(h, h)
    n.float().sum().backward()
    assert n.dtype == BF and m.weight.grad.dtype == torch.float32 and m.weight.grad.any()
    e = ends.Embedding(97, 64, 0.5, device="cuda")
    z = e(y)
    z.sum().backward()
    assert z.dtype == torch.float32 and torch.equal(z, e.weight[y] * 0.5) and e.weight.grad.any()


def small(**kw):
    from paper_2607_20652_gb300.transformer import ParityTransformer
    torch.manual_seed(0)
    return ParityTransformer(layers=2, d=64, heads=4, d_mlp=128, vocab=97, context=32, device="cuda", **kw)


@pytest.mark.parametrize("attention", ["torch", "dpb"])
def test_model_is_the_same_model(attention):
    """Its loss and gradients against the same weights in fp32, beside those of the model on torch's operators."""
    own, other = small(ends="dpb", attention=attention), small(attention=attention)
    wide = None if attention == "dpb" else copy.deepcopy(other).float()
    assert own.state_dict().keys() == other.state_dict().keys()
    ids, tgt = (torch.randint(0, 97, (4, 32), device="cuda") for _ in range(2))
    tgt[:, :5] = -100
    losses = []
    for m in (own, other, wide):
        if m is not None:
            loss = m(ids, tgt)
            loss.backward()
            losses.append(float(loss.detach()))
    # the other model's scores are bf16: each off by 2^-8 of its size (below 1 here) in about log 97
    assert abs(losses[0] - losses[1]) < 2.0 ** -8
    assert torch.equal(own(ids).argmax(-1), own(ids).argmax(-1)) and rel(own(ids), other(ids)) < 12 * 2.0 ** -8
    for (n, p), q in zip(own.named_parameters(), other.parameters()):
        # about a dozen roundings of 2^-8 a block on the way, of either model, and two blocks
        assert p.grad.dtype == q.grad.dtype and rel(p.grad, q.grad) < 24 * 2.0 ** -8, n
    if wide is not None:
        assert abs(losses[0] - losses[2]) < 2.0 ** -8
        for (n, p), q in zip(own.named_parameters(), wide.parameters()):
            assert rel(p.grad, q.grad) < 24 * 2.0 ** -8, n
    assert dpb.status() == 0


def test_training_step_runs():
    """Lookup, residual norms, attention, bottleneck, loss and optimiser as they are used together."""
    from paper_2607_20652_gb300.optim import AdamW
    m = small(ends="dpb", attention="dpb", dpb=dict(levels=3, m_bits=12, children=16, beam=8, k=8))
    opt = AdamW(m.parameters(), lr=3e-3, state_bits=8)
    for _ in range(3):
        opt.zero_grad(set_to_none=True)
        loss = m(torch.randint(0, 97, (4, 32), device="cuda"), torch.randint(0, 97, (4, 32), device="cuda"))
        loss.backward()
        assert torch.isfinite(loss) and all(torch.isfinite(p.grad).all() and p.grad.any() for p in m.parameters())
        opt.step()
    assert dpb.status() == 0


def test_model_refuses():
    from paper_2607_20652_gb300.transformer import ParityTransformer
    at = dict(layers=1, d=64, heads=4, d_mlp=128, vocab=97, context=32)
    for kw in (dict(ends="other"), dict(ends="dpb", dtype=torch.float32), dict(ends="dpb", d=60)):
        with pytest.raises(ValueError):
            ParityTransformer(**(at | kw))


def test_second_derivatives_and_changed_inputs_raise():
    from paper_2607_20652_gb300 import ends
    w = torch.randn(97, 64, device="cuda").to(BF).requires_grad_()
    x = torch.randn(20, 64, device="cuda").to(BF).requires_grad_()
    y = torch.randint(0, 97, (20,), device="cuda")
    for f, of in ((lambda: ends.embedding(w, y), w), (lambda: ends.add_norm(x, x)[0], x),
                  (lambda: ends.linear_cross_entropy(x, w, y, reduction="none"), x)):
        loss = (f().float() ** 2).sum()
        g, = torch.autograd.grad(loss, of, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            (loss + (g.float() ** 2).sum()).backward()
    for f in (lambda: ends.embedding(w, y).float().sum(), lambda: ends.linear_cross_entropy(x, w, y)):
        loss = f()
        y[0] = 3
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()


def test_refusals():
    from paper_2607_20652_gb300 import ends
    w, x = torch.randn(97, 64, device="cuda").to(BF), torch.randn(20, 64, device="cuda").to(BF)
    y = torch.randint(0, 97, (20,), device="cuda")
    for bad in (lambda: ends.linear_cross_entropy(x, w, y, reduction="other"), lambda: ends.linear_cross_entropy(x, w, y[:5]),
                lambda: ends.linear_cross_entropy(x.float(), w, y), lambda: ends.linear_cross_entropy(x, w[:, :32], y),
                lambda: ends.add_norm(x, x[:5]), lambda: ends.add_norm(x, None, w[0, :5]), lambda: ends.embedding(w.half(), y)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(dpb.DPBError):
        ends.linear_cross_entropy(x[:, :60], w[:, :60], y)


def test_threads_on_one_stream():
    """Two kinds of threads enqueue calls of different sizes on one stream: each gets what it gets alone."""
    work = []
    for T, V, d in ((900, 1000, 64), (300, 5000, 128)):
        h, w = torch.randn(T, d, device="cuda").to(BF), torch.randn(V, d, device="cuda").to(BF)
        y, g = torch.randint(0, V, (T,), device="cuda"), torch.rand(T, device="cuda")
        y[::3] = -100
        ids = y.clamp(min=0)

        def step(h=h, w=w, y=y, g=g, ids=ids, V=V):
            loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
            return (loss, *dpb.linear_cross_entropy_backward(h, w, y, lse, g), dpb.embedding_backward(h, ids, V),
                    *dpb.add_norm_backward(h, h))

        work.append(step)
    want = [f() for f in work]
    torch.cuda.synchronize()
    wrong = []

    def loop(f, v):
        for _ in range(60):
            if not all(torch.equal(a, b) for a, b in zip(f(), v)):
                wrong.append(1)

    threads = [threading.Thread(target=loop, args=(f, v)) for f, v in zip(work, want) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and dpb.status() == 0


def test_model_in_a_cuda_graph():
    """A step captured without workspaces of its own; then other calls on the capture's stream, memory given back and filled
    with other data, and the replay with other tokens: the graph's scratch is still its own."""
    m = small(ends="dpb", attention="dpb")
    ids, tgt = (torch.randint(0, 97, (4, 32), device="cuda") for _ in range(2))
    tgt[0, :9] = -100
    ps = list(m.parameters())

    def step():
        loss = m(ids, tgt)
        return [loss, *torch.autograd.grad(loss, ps)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    other = [torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    for seed in (1, 2):
        g = torch.Generator(device="cuda").manual_seed(seed)
        ids.copy_(torch.randint(0, 97, (4, 32), generator=g, device="cuda"))
        tgt.copy_(torch.randint(0, 97, (4, 32), generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        first = [t.detach().clone() for t in got]
        assert all(torch.equal(a, b) for a, b in zip(first, step()))
    assert all(bool((t == 7).all()) for t in other) and dpb.status() == 0
    tgt[0, 0] = 97
    graph.replay()
    assert dpb.status() == dpb.DEV_BAD_INDEX and dpb.status() == 0


def test_every_call_refuses_a_workspace_of_another_place():
    """Also the step's other operators: a workspace on the host, one that repeats itself, one with gaps."""
    w, x = torch.randn(97, 64, device="cuda").to(BF), torch.randn(20, 64, device="cuda").to(BF)
    y, g = torch.randint(0, 97, (20,), device="cuda"), torch.ones(20, device="cuda")
    q = torch.randn(20, 2, 64, device="cuda").to(BF)
    _, lse = dpb.linear_cross_entropy_forward(x, w, y)
    o, l2 = dpb.attention_forward(q, q, q)
    host = torch.zeros(1 << 24, dtype=torch.uint8)
    there = host[:1 << 10].cuda()
    for ws in (host, there[:1].expand(1 << 24), there[::2]):
        for f in (lambda **k: dpb.linear_cross_entropy_forward(x, w, y, **k), lambda **k: dpb.embedding(w, y, **k),
                  lambda **k: dpb.linear_cross_entropy_backward(x, w, y, lse, g, **k),
                  lambda **k: dpb.embedding_backward(x, y, 97, **k), lambda **k: dpb.add_norm_backward(x, x, **k),
                  lambda **k: dpb.qk_norm_rope(q, q, **k), lambda **k: dpb.qk_norm_rope_backward(q, q, q, q, **k),
                  lambda **k: dpb.attention_forward(q, q, q, **k), lambda **k: dpb.attention_backward(q, q, q, o, l2, q, **k)):
            with pytest.raises(ValueError, match="workspace"):
                f(workspace=ws)


def test_hooks_of_the_model_run():
    """Every module of the model is called as one: hooks on blocks, norms and the embedding see what they see elsewhere."""
    ids, tgt = (torch.randint(0, 97, (4, 32), device="cuda") for _ in range(2))
    dpb_kw = dict(levels=3, m_bits=12, children=16, beam=8, k=8)
    called = {}
    for kind in ("torch", "dpb"):
        m, seen = small(ends=kind, dpb=dpb_kw), []
        for name, sub in m.named_modules():
            if name:
                sub.register_forward_hook(lambda s, a, out, name=name: seen.append(name))
        m(ids, tgt).backward()
        called[kind] = seen
    assert called["dpb"] == called["torch"] and {"tok", "norm", "blocks.1", "blocks.0.n1", "blocks.1.n2"} <= set(called["dpb"])


def test_blocks_behind_a_checkpoint():
    """Blocks in a wrapper that computes them again in the backward pass: equal bits."""
    from torch.utils.checkpoint import checkpoint

    class Again(torch.nn.Module):
        def __init__(self, block):
            super().__init__()
            self.block = block

        def forward(self, *args):
            return checkpoint(self.block, *args, use_reentrant=False)

    m = small(ends="dpb", attention="dpb")
    ids, tgt = (torch.randint(0, 97, (4, 32), device="cuda") for _ in range(2))
    ps = list(m.parameters())
    loss = m(ids, tgt)
    want = (loss.detach(), *torch.autograd.grad(loss, ps))
    for i, b in enumerate(m.blocks):
        m.blocks[i] = Again(b)
    loss = m(ids, tgt)
    assert all(torch.equal(a, b) for a, b in zip(want, (loss.detach(), *torch.autograd.grad(loss, ps))))


def test_fp32_parameters_under_autocast():
    """Modules with fp32 parameters under bf16 autocast, as attention's: the residual stream is fp32, the loss takes its rows
    in bf16 as a linear layer would, every gradient is fp32. Without autocast fp32 rows are refused, as under fp16's."""
    from paper_2607_20652_gb300 import ends
    torch.manual_seed(4)
    emb, norm, lin = ends.Embedding(97, 64, device="cuda"), ends.AddRMSNorm(64, device="cuda"), \
        torch.nn.Linear(64, 64, bias=False, device="cuda")
    ids, y = (torch.randint(0, 97, (3, 20), device="cuda") for _ in range(2))
    ps = [emb.weight, norm.weight, lin.weight]
    with torch.autocast("cuda", torch.bfloat16):
        x = emb(ids)
        delta = lin(x)
        h, total = norm(x, delta)
        assert x.dtype == h.dtype == total.dtype == torch.float32 and delta.dtype == BF
        loss = ends.linear_cross_entropy(h, emb.weight, y)
    got = torch.autograd.grad(loss, (*ps, h), retain_graph=True)
    assert loss.dtype == torch.float32 and all(g.dtype == torch.float32 and g.any() for g in got)
    hb, wb = h.detach().to(BF).requires_grad_(), emb.weight.detach().to(BF).requires_grad_()
    want = ends.linear_cross_entropy(hb, wb, y)
    dh, _ = torch.autograd.grad(want, (hb, wb))
    assert torch.equal(loss, want) and torch.equal(got[3], dh.float())
    for f in (lambda: ends.linear_cross_entropy(h, emb.weight, y),):
        with pytest.raises(ValueError):
            f()
        with torch.autocast("cuda", torch.float16), pytest.raises(ValueError):
            f()


def test_threads_on_one_stream_all_finish():
    """As above, with whatever a thread raises told, and each of its calls counted."""
    work = []
    for T, V, d in ((900, 1000, 64), (300, 5000, 128)):
        h, w = torch.randn(T, d, device="cuda").to(BF), torch.randn(V, d, device="cuda").to(BF)
        y, g = torch.randint(0, V, (T,), device="cuda"), torch.rand(T, device="cuda")
        y[::3] = -100
        ids = y.clamp(min=0)

        def step(h=h, w=w, y=y, g=g, ids=ids, V=V):
            loss, lse = dpb.linear_cross_entropy_forward(h, w, y)
            return (loss, *dpb.linear_cross_entropy_backward(h, w, y, lse, g), dpb.embedding(w, ids),
                    dpb.embedding_backward(h, ids, V), *dpb.add_norm(h, h), *dpb.add_norm_backward(h, h))

        work.append(step)
    want = [f() for f in work]
    torch.cuda.synchronize()
    raised, same = [], []

    def loop(f, v):
        try:
            for _ in range(60):
                same.append(all(torch.equal(a, b) for a, b in zip(f(), v)))
        except BaseException as e:
            raised.append(e)

    threads = [threading.Thread(target=loop, args=(f, v)) for f, v in zip(work, want) for _ in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not raised and len(same) == 4 * 60 and all(same) and dpb.status() == 0


def test_models_choose_the_same_words():
    """The highest score of each token, where it leads by more than both models' roundings (a dozen of 2^-8 each) may move."""
    own, other = small(ends="dpb"), small()
    with torch.no_grad():
        for m in (own, other):
            m.tok.weight.mul_(20)  # scores some 3 apart in place of 0.2
        ids = torch.randint(0, 97, (4, 32), device="cuda")
        a, b = own(ids).double(), other(ids).double()
    top = b.topk(2, -1).values
    clear = top[..., 0] - top[..., 1] > 24 * 2.0 ** -8 * b.abs().amax(-1)
    assert clear.sum() > 10 and torch.equal(a.argmax(-1)[clear], b.argmax(-1)[clear])
    assert len(b.argmax(-1)[clear].unique()) > 3
