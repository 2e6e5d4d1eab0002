"""Measured cases of the training step's operators at both ends of the model and along its residual stream: cross
entropy over the vocabulary from the last hidden rows, embedding lookup with its gradient, and the residual's addition
with the RMS norm behind it.

`run` takes a state through one pass: in plain 32-bit torch operations, or, with `own` set, through the framework's
entry points (`paper_2607_20652_gb300.dpb`). `exact` gives the same outputs from the definitions in 64 bits.

Definitions.
Loss: z = hidden weight^T, lse_t = log sum_v exp z_tv, loss_t = lse_t - z_t,target; a token whose target is -100 has
loss 0, lse 0 and no gradient. Its gradient for given dL/dloss_t: dz_tv = dL/dloss_t (exp(z_tv - lse_t) - [v = target]),
d hidden = dz weight, d weight = dz^T hidden. A step is both.
Embedding: y_t = scale weight[id_t]; its gradient, in dense form: d weight[v] = scale sum of dy_t over id_t = v.
Norm: total = x + delta, rounded to the rows' type; y = weight total (mean total^2 + eps)^(-1/2). Its gradient: with
r = (mean total^2 + eps)^(-1/2) and u = weight dy, dx = d total + r u - total r^3 mean(u total),
d weight = sum_t dy total r.
"""
import math

import torch

own = False

EPS = 1e-6
IGNORE = -100
MOST_FLOPS = 8 * 8192 * 50257 * 768   # of a drawn loss: the largest listed one's
MOST_VALUES = 65536 * 768             # of a drawn embedding's or norm's rows, in bf16: the largest listed one's
BF16, F32 = "bf16", "f32"


# ---- cases ------------------------------------------------------------------

def listed():
    return [
        # a training step of the small ParityTransformer of the tests: latency alone
        loss("loss step: small model", "step", tokens=128, vocab=97, d=64),
        # the score of one short answer of 33 tokens by the GPT-2-small shape: the weights are read for few rows
        loss("loss: 33 tokens", "forward", tokens=33, vocab=50257, d=768),
        # an evaluation batch of the bench's training step, 8 sequences of 1024 tokens
        loss("loss: evaluation batch", "forward", tokens=8192, vocab=50257, d=768),
        # the bench's training step, forward and gradients, mean over the batch
        loss("loss step: 8 x 1024", "step", tokens=8192, vocab=50257, d=768),
        # answers behind prompts that take no part, the paper's small width, odd sizes, a weight of its own for each token
        loss("loss step: prompts left out", "step", tokens=9001, vocab=32003, d=1024, ignored=0.6, runs=True, even=False),
        # the small model's lookup in 32 bits: latency alone
        embedding("embedding: small model", "forward", tokens=128, vocab=97, d=64, dtype=F32, ids="zipf"),
        # the wide workload's 65536 tokens at the GPT-2-small shape
        embedding("embedding: 65536 tokens", "forward", tokens=65536, vocab=50257, d=768, dtype=BF16, ids="zipf"),
        # their gradient, frequent tokens thousands of times among them
        embedding("embedding gradient: 65536", "backward", tokens=65536, vocab=50257, d=768, dtype=BF16, ids="zipf"),
        # odd sizes in 32 bits, scaled, every token about as frequent
        embedding("embedding gradient: odd", "backward", tokens=9999, vocab=5003, d=500, dtype=F32, ids="uniform",
                  scaled=True),
        # one block of the small model: latency alone
        norm("norm: small model", "forward", tokens=128, d=64, dtype=F32),
        # the residual's addition and the norm of one block of the wide workload
        norm("norm: 65536 tokens", "forward", tokens=65536, d=768, dtype=BF16),
        # a block's gradient at a width that is no power of two, odd token count
        norm("norm gradient", "backward", tokens=49999, d=1000, dtype=BF16),
    ]


def loss(name, direction, tokens, vocab, d, ignored=0.0, runs=False, even=True):
    return dict(name=name, op="loss", direction=direction, tokens=tokens, vocab=vocab, d=d, ignored=ignored, runs=runs,
                even=even)


def embedding(name, direction, tokens, vocab, d, dtype, ids, scaled=False, wide=True):
    return dict(name=name, op="embedding", direction=direction, tokens=tokens, vocab=vocab, d=d, dtype=dtype, ids=ids,
                scaled=scaled, wide=wide)


def norm(name, direction, tokens, d, dtype, residual=True):
    return dict(name=name, op="norm", direction=direction, tokens=tokens, d=d, dtype=dtype, residual=residual)


def log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["loss", "loss", "embedding", "norm"])
    if op == "loss":
        case = loss("", rng.choice(["forward", "step", "step"]), log_int(rng, 1, 16384), log_int(rng, 50, 65536),
                    8 * log_int(rng, 1, 256), rng.choice([0.0, 0.0, 0.3, 0.9]), rng.random() < 0.5, rng.random() < 0.5)
        while 8 * case["tokens"] * case["vocab"] * case["d"] > MOST_FLOPS:
            case["tokens"] = int(case["tokens"] * 0.8)
    else:
        dtype = rng.choice([BF16, BF16, F32])
        d = log_int(rng, 1 if op == "embedding" else 8, 4096)
        most = MOST_VALUES // (2 if dtype == F32 else 1)
        tokens = log_int(rng, 1, min(65536, most // d))
        if op == "embedding":
            case = embedding("", rng.choice(["forward", "backward", "backward"]), tokens,
                             log_int(rng, 1, min(65536, most // d)), d, dtype, rng.choice(["zipf", "uniform", "few"]),
                             rng.random() < 0.5, rng.random() < 0.5)
        else:
            case = norm("", rng.choice(["forward", "backward"]), tokens, d, dtype, rng.random() < 0.75)
    del case["name"]
    return case


def work(case):
    T, d = case["tokens"], case["d"]
    if case["op"] == "loss":
        n, V = counted(case), case["vocab"]
        fwd = 2 * d * (n + V) + 16 * T                   # hidden rows that count and the weight; targets; loss, lse
        # a step reads dL/dloss and writes d hidden, d weight; its products: the scores twice (they are not kept), two gradients
        if case["direction"] == "forward":
            return {"bytes": fwd, "flops": 2 * n * V * d}
        return {"bytes": fwd + 4 * T + 2 * d * (T + V), "flops": 8 * n * V * d}
    b = 4 if case["dtype"] == F32 else 2
    if case["op"] == "embedding":
        ids = T * (8 if case["wide"] else 4)
        if case["direction"] == "forward":
            return {"bytes": b * d * (T + min(T, case["vocab"])) + ids, "flops": T * d}
        return {"bytes": b * d * (T + case["vocab"]) + ids, "flops": T * d}
    rows = (4 if case["residual"] else 2) if case["direction"] == "forward" else (4 if case["residual"] else 3)
    return {"bytes": b * d * T * rows, "flops": T * d * (5 if case["direction"] == "forward" else 12)}


def left_out(case):
    """Places whose target is ignored, when they come in runs at the start of each of up to five sequences."""
    period = -(-case["tokens"] // 5)
    return [t % period < int(case["ignored"] * period) for t in range(case["tokens"])]


def counted(case):
    if case["runs"]:
        return case["tokens"] - sum(left_out(case))
    return case["tokens"] - int(case["ignored"] * case["tokens"])


# ---- inputs -----------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"loss": prepare_loss, "embedding": prepare_embedding, "norm": prepare_norm}[case["op"]](case, gen)


def normal(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def zipf(gen, n, most):
    """Token numbers whose frequency falls as 1 / number."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    return ((most + 1.0) ** u - 1).long().clamp_(0, most - 1)


def prepare_loss(case, gen):
    T, V, d = case["tokens"], case["vocab"], case["d"]
    # scores of a deviation of 1.5, whose lse is about log V + 1.1
    weight = normal(gen, V, d, std=1.5 / math.sqrt(d), dtype=torch.bfloat16)
    target = zipf(gen, T, V)
    # rows behind a norm that lean towards their target, some hardly and some so far that the model nearly knows it
    lean = torch.nn.functional.normalize(weight[target].float(), dim=1) * \
        (0.8 * (math.log(V) + 1.1) / 1.5 * torch.rand(T, 1, generator=gen, device="cuda"))
    hidden = (normal(gen, T, d) + lean).to(torch.bfloat16)
    if case["runs"]:
        target[torch.tensor(left_out(case), device="cuda")] = IGNORE
    elif case["ignored"]:
        target[torch.randperm(T, generator=gen, device="cuda")[:int(case["ignored"] * T)]] = IGNORE
    n = max(1, counted(case))
    # the gradient of a mean is one number for all; advantages differ from token to token
    grad = torch.full((1,), 1 / n, device="cuda").expand(T) if case["even"] else normal(gen, T, std=1 / n)
    return dict(case=case, hidden=hidden, weight=weight, target=target, grad=grad)


def prepare_embedding(case, gen):
    T, V, d = case["tokens"], case["vocab"], case["d"]
    dt = torch.float32 if case["dtype"] == F32 else torch.bfloat16
    ids = zipf(gen, T, V) if case["ids"] == "zipf" else \
        torch.randint(0, V if case["ids"] == "uniform" else min(V, 3), (T,), generator=gen, device="cuda")
    st = dict(case=case, ids=ids if case["wide"] else ids.int(), scale=math.sqrt(d) if case["scaled"] else 1.0)
    if case["direction"] == "forward":
        st["weight"] = normal(gen, V, d, std=0.02, dtype=dt)
    else:
        st["dy"] = normal(gen, T, d, std=1e-3, dtype=dt)
    return st


def prepare_norm(case, gen):
    T, d = case["tokens"], case["d"]
    dt = torch.float32 if case["dtype"] == F32 else torch.bfloat16
    st = dict(case=case, x=normal(gen, T, d, std=2.0, dtype=dt), weight=1 + normal(gen, d, std=0.2))
    st["weight"] = st["weight"].to(dt)
    if case["direction"] == "forward":
        st["delta"] = normal(gen, T, d, std=0.5, dtype=dt) if case["residual"] else None
    else:
        st["dy"] = normal(gen, T, d, dtype=dt)
        st["dtotal"] = normal(gen, T, d, dtype=dt) if case["residual"] else None
    return st


# ---- one pass ---------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return {"loss": own_loss, "embedding": own_embedding, "norm": own_norm}[c["op"]](state, c)
    return {"loss": plain_loss, "embedding": plain_embedding, "norm": plain_norm}[c["op"]](state, c)


def own_loss(s, c):
    from paper_2607_20652_gb300 import dpb
    loss, lse = dpb.linear_cross_entropy_forward(s["hidden"], s["weight"], s["target"], ignore_index=IGNORE)
    if c["direction"] == "forward":
        return {"loss": loss, "lse": lse}
    dh, dw = dpb.linear_cross_entropy_backward(s["hidden"], s["weight"], s["target"], lse, s["grad"],
                                               ignore_index=IGNORE)
    return {"loss": loss, "dh": dh, "dw": dw}


def plain_loss(s, c):
    h, w, target = s["hidden"].float(), s["weight"].float(), s["target"]
    counts = target != IGNORE
    at = torch.where(counts, target, torch.zeros_like(target))[:, None]
    z = h @ w.t()
    top = z.amax(1, keepdim=True)
    # a small loss is the difference of large scores: the last sums in 64 bits
    log_sum = torch.log(torch.exp(z - top).sum(1, keepdim=True, dtype=torch.float64))
    lse = (top + log_sum).float()
    loss = torch.where(counts, (top.double() - z.gather(1, at) + log_sum).float()[:, 0], torch.zeros_like(lse[:, 0]))
    if c["direction"] == "forward":
        return {"loss": loss, "lse": torch.where(counts, lse[:, 0], torch.zeros_like(loss))}
    dz = torch.exp(z - lse)
    del z
    dz.scatter_add_(1, at, torch.full_like(lse, -1.0))
    dz *= torch.where(counts, s["grad"], torch.zeros_like(loss))[:, None]
    return {"loss": loss, "dh": (dz @ w).to(s["hidden"].dtype), "dw": (dz.t() @ h).to(s["weight"].dtype)}


def own_embedding(s, c):
    from paper_2607_20652_gb300 import dpb
    if c["direction"] == "forward":
        return dpb.embedding(s["weight"], s["ids"], scale=s["scale"])
    return dpb.embedding_backward(s["dy"], s["ids"], c["vocab"], scale=s["scale"])


def plain_embedding(s, c):
    if c["direction"] == "forward":
        return (s["weight"][s["ids"].long()].float() * s["scale"]).to(s["weight"].dtype)
    dy = s["dy"]
    dw = torch.zeros(c["vocab"], c["d"], device="cuda").index_add_(0, s["ids"].long(), dy.float())
    return (dw * s["scale"]).to(dy.dtype)


def own_norm(s, c):
    from paper_2607_20652_gb300 import dpb
    if c["direction"] == "forward":
        y, total = dpb.add_norm(s["x"], s["delta"], s["weight"], eps=EPS)
        return {"y": y, "total": total} if c["residual"] else {"y": y}
    dx, dw = dpb.add_norm_backward(s["x"], s["dy"], s["dtotal"], s["weight"], eps=EPS)
    return {"dx": dx, "dw": dw}


def plain_norm(s, c):
    dt, w = s["x"].dtype, s["weight"].float()
    if c["direction"] == "forward":
        total = (s["x"].float() + s["delta"].float()).to(dt) if c["residual"] else s["x"]
        t = total.float()
        y = (t * torch.rsqrt(t.square().mean(1, keepdim=True) + EPS) * w).to(dt)
        return {"y": y, "total": total} if c["residual"] else {"y": y}
    t, g = s["x"].float(), s["dy"].float()
    r = torch.rsqrt(t.square().mean(1, keepdim=True) + EPS)
    u = g * w
    dx = r * u - t * r ** 3 * (u * t).mean(1, keepdim=True)
    if c["residual"]:
        dx = dx + s["dtotal"].float()
    return {"dx": dx.to(dt), "dw": (g * t * r).sum(0)}


# ---- from the definitions, in 64 bits ---------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"loss": exact_loss, "embedding": exact_embedding, "norm": exact_norm}[case["op"]](s, case)


def exact_loss(s, c):
    """1024 tokens at a time, ignored ones left out."""
    f8 = dict(dtype=torch.float64, device="cuda")
    T, V, d = c["tokens"], c["vocab"], c["d"]
    w = s["weight"].double()
    loss, lse, dh, dw = (torch.zeros(n, **f8) for n in ((T,), (T,), (T, d), (V, d)))
    for rows in (s["target"] != IGNORE).nonzero()[:, 0].split(1024):
        h, y, k = s["hidden"][rows].double(), s["target"][rows], torch.arange(len(rows), device="cuda")
        z = h @ w.t()
        lse[rows] = torch.logsumexp(z, 1)
        loss[rows] = lse[rows] - z[k, y]
        if c["direction"] == "step":
            p = torch.softmax(z, 1)
            p[k, y] -= 1
            p *= s["grad"][rows].double()[:, None]
            dh[rows] = p @ w
            dw += p.t() @ h
    return {"loss": loss, "lse": lse} if c["direction"] == "forward" else {"loss": loss, "dh": dh, "dw": dw}


def exact_embedding(s, c):
    """The gradient by sorted tokens: differences of the running sums would lose digits, so each row is summed alone."""
    if c["direction"] == "forward":
        return torch.nn.functional.embedding(s["ids"].long(), s["weight"].double()) * s["scale"]
    ids, order = s["ids"].long().sort(stable=True)
    dw = torch.zeros(c["vocab"], c["d"], dtype=torch.float64, device="cuda")
    rows, counts = ids.unique_consecutive(return_counts=True)
    dy = s["dy"].double()[order]
    dw[rows] = torch.segment_reduce(dy, "sum", lengths=counts, axis=0)
    return dw * s["scale"]


def exact_norm(s, c):
    """The gradient by automatic differentiation."""
    x, w = s["x"].double(), s["weight"].double()
    if c["direction"] == "forward":
        total = (x + s["delta"].double()).to(s["x"].dtype) if c["residual"] else s["x"]
        x = total.double()
        y = x / torch.sqrt((x * x).sum(1, keepdim=True) / c["d"] + EPS) * w
        return {"y": y, "total": total.double()} if c["residual"] else {"y": y}
    x.requires_grad_()
    w.requires_grad_()
    y = x / torch.sqrt((x * x).sum(1, keepdim=True) / c["d"] + EPS) * w
    dx, dw = torch.autograd.grad(y, (x, w), s["dy"].double())
    return {"dx": dx + s["dtotal"].double() if c["residual"] else dx, "dw": dw}
