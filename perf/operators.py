"""Measured cases of the training-step operators beside the bottleneck: norm and rotation of queries and keys,
attention with its gradient, and AdamW over many tensors.

`run` takes a state through one pass: in plain 32-bit torch operations, or, with `own` set, through the framework's
entry points (`paper_2607_20652_gb300.dpb`). `exact` gives the same outputs from the definitions in 64 bits.

Layouts. Queries, keys and values are the three parts of one packed projection [tokens, q heads + 2 kv heads, dim],
as a qkv linear layer leaves them; sequences are packed end to end, offsets in int32. A causal query i of a sequence
with n queries and m keys sees keys j <= i + m - n. Parameters are views of one flat buffer, each starting at a
multiple of 256 values, as a trainer with gradient buckets keeps them.
"""
import math
import random

import torch

own = False

EPS = 1e-6
ADAM = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=1000, seed=12345)
BLOCK = 256      # values that share a scale where the states are held in 8 bits
E4M3_MAX = 448.0
MOST_FLOPS = 8.1e11  # of a drawn attention: the longest listed case's


# ---- cases ------------------------------------------------------------------

def listed():
    return [
        # four prompts of 32 tokens through the small ParityTransformer of the tests: latency alone
        attention("attention: short prompts", "forward", seqs=4, shortest=32, longest=32, heads=4, kv=4, dim=16),
        # an evaluation batch at the GPT-2-small shape of the bench: 8 sequences of 1024 tokens
        attention("attention: evaluation batch", "forward", seqs=8, shortest=1024, longest=1024, heads=12, kv=12, dim=64),
        # the attention of one layer of the bench's training step, forward and backward
        attention("attention step: 8 x 1024", "step", seqs=8, shortest=1024, longest=1024, heads=12, kv=12, dim=64),
        # documents of odd lengths packed into one batch, grouped heads of 128
        attention("attention step: documents", "step", seqs=12, shortest=1, longest=3001, heads=16, kv=4, dim=128),
        # one long document of odd length
        attention("attention step: one long", "step", seqs=1, shortest=12289, longest=12289, heads=12, kv=12,
                  dim=64),
        # the small model's queries and keys in 32 bits: latency alone
        rotary("rotation: small model", "forward", tokens=128, heads=4, kv=4, dim=16, rot=16, interleaved=False,
               dtype="f32"),
        # the wide workload's 65536 tokens at the GPT-2-small head layout
        rotary("rotation: 65536 tokens", "forward", tokens=65536, heads=12, kv=12, dim=64, rot=64, interleaved=False,
               dtype="bf16"),
        # gradient at grouped heads of 128, three quarters of the head rotated, interleaved pairs, odd token count
        rotary("rotation gradient", "backward", tokens=49999, heads=16, kv=4, dim=128, rot=96,
               interleaved=True, dtype="bf16"),
        # the small ParityTransformer of the tests, everything in 32 bits: latency alone
        adamw("AdamW: small model", layers=2, d=64, mlp=128, vocab=97, context=32, dtype="f32", state="f32"),
        # the paper's small width (d = 1024, 12 layers), bf16 parameters, 32-bit states
        adamw("AdamW: d = 1024 model", layers=12, d=1024, mlp=4096, vocab=50257, context=1024, dtype="bf16", state="f32"),
        # odd widths and tails shorter than a block, 8-bit states
        adamw("AdamW 8-bit: odd widths", layers=5, d=500, mlp=1303, vocab=5003, context=257, dtype="f32", state="f8"),
        # the paper's small width with 8-bit states
        adamw("AdamW 8-bit: d = 1024 model", layers=12, d=1024, mlp=4096, vocab=50257, context=1024, dtype="bf16",
              state="f8"),
    ]


def attention(name, direction, seqs, shortest, longest, heads, kv, dim, causal=True, past=0, short_keys=False):
    return dict(name=name, op="attention", direction=direction, seqs=seqs, shortest=shortest, longest=longest,
                heads=heads, kv=kv, dim=dim, causal=causal, past=past, short_keys=short_keys)


def rotary(name, direction, tokens, heads, kv, dim, rot, interleaved, dtype):
    return dict(name=name, op="rotary", direction=direction, tokens=tokens, heads=heads, kv=kv, dim=dim, rot=rot,
                interleaved=interleaved, dtype=dtype)


def adamw(name, layers, d, mlp, vocab, context, dtype, state):
    return dict(name=name, op="adamw", layers=layers, d=d, mlp=mlp, vocab=vocab, context=context, dtype=dtype, state=state)


def log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "rotary", "adamw"])
    if op == "attention":
        heads, kv = rng.choice([(4, 4), (12, 12), (16, 16), (16, 4), (8, 1), (6, 2)])
        direction = rng.choice(["forward", "step"])
        # a query that sees one key has no gradient but rounding: a step has at least four
        longest = log_int(rng, 4 if direction == "step" else 1, 12289)
        most = max(1, min(48, int(12 * 12289 ** 2 / (heads * longest ** 2)), 65536 // longest))
        seqs = log_int(rng, 1, most)
        case = attention("", direction, seqs, log_int(rng, 1, longest), longest, heads, kv,
                         rng.choice([16, 40, 64, 64, 96, 128]), causal=rng.random() < 0.75,
                         past=rng.choice([0, 0, log_int(rng, 1, 500)]), short_keys=rng.random() < 0.25)
        while work(case)["flops"] > MOST_FLOPS:  # fewer sequences, then shorter ones
            if case["seqs"] > 1:
                case["seqs"] -= 1
            else:
                case["longest"] = int(case["longest"] * 0.9)
                case["shortest"] = min(case["shortest"], case["longest"])
    elif op == "rotary":
        heads, kv = rng.choice([(4, 4), (12, 12), (16, 4), (8, 1), (5, 3)])
        dim = rng.choice([16, 24, 64, 64, 96, 128])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        tokens = log_int(rng, 1, int(49999 * 20 * 128 / ((heads + kv) * dim)) // (2 if dtype == "f32" else 1))
        case = rotary("", rng.choice(["forward", "backward"]), min(tokens, 131072), heads, kv, dim,
                      rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)]), rng.random() < 0.5, dtype)
    else:
        d = log_int(rng, 16, 1000)
        case = adamw("", rng.randint(1, 12), d, d * rng.choice([2, 4]) + rng.choice([0, 0, 1, 7]), log_int(rng, 50, 50257),
                     log_int(rng, 8, 1024), rng.choice(["bf16", "f32"]), rng.choice(["f32", "f8"]))
    del case["name"]
    return case


def lengths(case):
    """Queries and keys of each sequence: the longest, the shortest, the others spread over their logarithm."""
    rng = random.Random(case["seqs"] * 1000003 + case["longest"])
    nq = [case["longest"], case["shortest"]][: case["seqs"]]
    nq += [log_int(rng, case["shortest"], case["longest"]) for _ in range(case["seqs"] - len(nq))]
    rng.shuffle(nq)
    nk = [n + (rng.randint(0, case["past"]) if case["past"] else 0) for n in nq]
    if case["short_keys"]:  # a sequence with fewer keys than queries, or none: causal rows that see nothing
        nk[0] = nq[0] // 2 if case["seqs"] > 1 else max(1, nq[0] // 2)
    return nq, nk


def shapes(case):
    """Parameter shapes of a ParityTransformer (two norm weights, qkv, out, up, down a layer; tied embedding)."""
    d, mlp = case["d"], case["mlp"]
    one = [(d,), (3 * d, d), (d, d), (d,), (mlp, d), (d, mlp)]
    return [(case["vocab"], d), (case["context"], d)] + one * case["layers"] + [(d,)]


def work(case):
    if case["op"] == "attention":
        nq, nk = lengths(case)
        pairs = sum(visible(n, m, case["causal"]) for n, m in zip(nq, nk))
        q, kv, d = sum(nq) * case["heads"], sum(nk) * case["kv"], case["dim"]
        fwd = 2 * d * (2 * q + 2 * kv) + 4 * q                     # q, k, v read; o, lse written
        step = 2 * d * (4 * q + 4 * kv) + 4 * q                    # and do read; dq, dk, dv written (o stays whole)
        return {"bytes": fwd if case["direction"] == "forward" else step,
                "flops": (4 if case["direction"] == "forward" else 14) * d * pairs * case["heads"]}
    if case["op"] == "rotary":
        n = case["tokens"] * (case["heads"] + case["kv"]) * case["dim"]
        b = 4 if case["dtype"] == "f32" else 2
        fwd = case["direction"] == "forward"
        return {"bytes": n * b * (2 if fwd else 3) + case["tokens"] * 4, "flops": n * (10 if fwd else 20)}
    n = sum(math.prod(s) for s in shapes(case))
    b = 4 if case["dtype"] == "f32" else 2
    return {"bytes": n * (3 * b + 16) if case["state"] == "f32" else n * (3 * b + 4) + 16 * (n // BLOCK),
            "flops": 14 * n}


def visible(n, m, causal):
    if not causal:
        return n * m
    first = max(0, n - m)  # queries before it see no key
    seen = n - first
    return seen * (first + m - n + 1) + seen * (seen - 1) // 2


# ---- inputs -----------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"attention": prepare_attention, "rotary": prepare_rotary, "adamw": prepare_adamw}[case["op"]](case, gen)


def normal(gen, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)


def offsets(n):
    return torch.tensor([0] + n, device="cuda").cumsum(0).to(torch.int32)


def prepare_attention(case, gen):
    nq, nk = lengths(case)
    h, hk, d = case["heads"], case["kv"], case["dim"]
    bf = torch.bfloat16
    if nq == nk:
        qkv = normal(gen, sum(nq), h + 2 * hk, d, dtype=bf)
        q, k, v = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
    else:
        q, kv = normal(gen, sum(nq), h, d, dtype=bf), normal(gen, sum(nk), 2 * hk, d, dtype=bf)
        k, v = kv[:, :hk], kv[:, hk:]
    return dict(case=case, q=q, k=k, v=v, do=normal(gen, sum(nq), h, d, dtype=bf), cu_q=offsets(nq), cu_k=offsets(nk),
                max_q=max(nq), max_k=max(nk), scale=1 / math.sqrt(d))


def prepare_rotary(case, gen):
    T, h, hk, d = case["tokens"], case["heads"], case["kv"], case["dim"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    qkv = normal(gen, T, h + 2 * hk, d, std=2.0, dtype=dt)
    # positions of packed documents: each restarts at 0
    start = torch.randint(0, 2048, (1,), generator=gen, device="cuda")
    pos = ((torch.arange(T, device="cuda") + start) % 2048).to(torch.int32)
    freq = 10000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / max(1, case["rot"]))
    ang = torch.arange(2048, device="cuda", dtype=torch.float64)[:, None] * freq
    return dict(case=case, q=qkv[:, :h], k=qkv[:, h:h + hk], wq=1 + normal(gen, d, std=0.2).to(dt),
                wk=1 + normal(gen, d, std=0.2).to(dt), cos=ang.cos().float(), sin=ang.sin().float(), pos=pos,
                dq=normal(gen, T, h, d, dtype=dt), dk=normal(gen, T, hk, d, dtype=dt))


def prepare_adamw(case, gen):
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    sh = shapes(case)
    starts, total = [], 0
    for s in sh:
        starts.append(total)
        total += -(-math.prod(s) // BLOCK) * BLOCK
    live = torch.zeros(total, dtype=torch.bool, device="cuda")
    for s, at in zip(sh, starts):
        live[at:at + math.prod(s)] = True
    # gradients differ in size from one block of values to the next
    size = torch.exp(torch.randn(total // BLOCK, generator=gen, device="cuda") - 7).repeat_interleave(BLOCK)
    p = (normal(gen, total, std=0.02) * live).to(dt)
    g = (normal(gen, total) * size * live).to(dt)
    m, v = normal(gen, total, std=0.3) * size * live, (normal(gen, total) * size * live).square() * 0.7
    st = dict(case=case, p=p, g=g, live=v)
    if case["state"] == "f8":
        st["m"], st["ms"] = nearest8(m)
        st["v"], st["vs"] = nearest8(v.sqrt())
    else:
        st["m"], st["v"] = m, v

    def cut(t):
        return [t[at:at + math.prod(s)].view(s) for s, at in zip(sh, starts)]

    def flat(t):
        return [t[at:at + math.prod(s)] for s, at in zip(sh, starts)]

    def blocks(t):
        return [t[at // BLOCK:at // BLOCK - (-math.prod(s) // BLOCK)] for s, at in zip(sh, starts)]

    st["params"], st["grads"] = cut(st["p"]), cut(st["g"])
    st["exp_avg"], st["exp_avg_sq"] = flat(st["m"]), flat(st["v"])
    if case["state"] == "f8":
        st["m_scale"], st["v_scale"] = blocks(st["ms"]), blocks(st["vs"])
    return st


def nearest8(x):
    """Starting states in 8 bits: nearest e4m3 with a scale for each block."""
    b = x.view(-1, BLOCK)
    top = b.abs().amax(1)
    inv = torch.where(top > 0, E4M3_MAX / top, torch.zeros_like(top))
    return (b * inv[:, None]).to(torch.float8_e4m3fn).view(-1), top / E4M3_MAX


# ---- one pass ---------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return {"attention": own_attention, "rotary": own_rotary, "adamw": own_adamw}[c["op"]](state, c)
    return {"attention": plain_attention, "rotary": plain_rotary, "adamw": plain_adamw}[c["op"]](state, c)


def own_attention(s, c):
    from paper_2607_20652_gb300 import dpb
    at = dict(cu_q=s["cu_q"], cu_k=s["cu_k"], max_q=s["max_q"], max_k=s["max_k"], causal=c["causal"], scale=s["scale"])
    o, lse = dpb.attention_forward(s["q"], s["k"], s["v"], **at)
    if c["direction"] == "forward":
        return {"o": o, "lse": lse}
    dq, dk, dv = dpb.attention_backward(s["q"], s["k"], s["v"], o, lse, s["do"], **at)
    return {"o": o, "dq": dq, "dk": dk, "dv": dv}


def plain_attention(s, c):
    q, k, v, g = s["q"], s["k"], s["v"], c["heads"] // c["kv"]
    iq, okq, bq, tq = padded(s["cu_q"], s["max_q"], q.shape[0])
    ik, okk, bk, tk = padded(s["cu_k"], s["max_k"], k.shape[0])
    n, m = okq.sum(1), okk.sum(1)
    see = okq[:, :, None] & okk[:, None, :]
    if c["causal"]:
        i, j = torch.arange(s["max_q"], device="cuda"), torch.arange(s["max_k"], device="cuda")
        see = see & (j[None, None, :] <= i[None, :, None] + (m - n)[:, None, None])
    see = see[:, None]
    # [sequence, head, token, dim] in 32 bits
    qf = q[iq].float().transpose(1, 2)
    kf = k[ik].float().transpose(1, 2).repeat_interleave(g, 1)
    vf = v[ik].float().transpose(1, 2).repeat_interleave(g, 1)
    sc = (qf @ kf.transpose(2, 3)) * s["scale"]
    sc = sc.masked_fill(~see, -math.inf)
    top = sc.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(sc - top)
    del sc
    z = p.sum(3, keepdim=True)
    p = p / torch.where(z == 0, torch.ones_like(z), z)
    o = p @ vf
    out = {"o": o[bq, :, tq].to(q.dtype)}
    if c["direction"] == "forward":
        out["lse"] = (top + torch.log(z))[bq, :, tq, 0].t().contiguous()
        return out
    do = s["do"][iq].float().transpose(1, 2) * okq[:, None, :, None]
    dv = p.transpose(2, 3) @ do
    ds = p * (do @ vf.transpose(2, 3) - (do * o).sum(3, keepdim=True)) * s["scale"]
    del p
    dq, dk = ds @ kf, ds.transpose(2, 3) @ qf
    dk, dv = (x.view(x.shape[0], c["kv"], g, *x.shape[2:]).sum(2)[bk, :, tk].to(q.dtype) for x in (dk, dv))
    return {**out, "dq": dq[bq, :, tq].to(q.dtype), "dk": dk, "dv": dv}


def padded(cu, longest, total):
    """Rows of a packed tensor for each (sequence, place), whether the place exists, and where each row stands."""
    at = torch.arange(longest, device="cuda")
    first, end = cu[:-1, None].long(), cu[1:, None].long()
    rows = torch.arange(total, device="cuda")
    b = torch.searchsorted(cu[1:].long(), rows, right=True)
    return (first + at).clamp(max=max(0, total - 1)), first + at < end, b, rows - cu[b].long()


def own_rotary(s, c):
    from paper_2607_20652_gb300 import dpb
    at = dict(weight_q=s["wq"], weight_k=s["wk"], cos=s["cos"], sin=s["sin"], positions=s["pos"], eps=EPS,
              interleaved=c["interleaved"])
    if c["direction"] == "forward":
        q, k = dpb.qk_norm_rope(s["q"], s["k"], **at)
        return {"q": q, "k": k}
    dq, dk, dwq, dwk = dpb.qk_norm_rope_backward(s["q"], s["k"], s["dq"], s["dk"], **at)
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def plain_rotary(s, c):
    cos, sin = s["cos"][s["pos"].long()][:, None], s["sin"][s["pos"].long()][:, None]
    if c["direction"] == "forward":
        return {"q": plain_norm_rope(s["q"], s["wq"], cos, sin, c), "k": plain_norm_rope(s["k"], s["wk"], cos, sin, c)}
    dq, dwq = plain_norm_rope_grad(s["q"], s["wq"], s["dq"], cos, sin, c)
    dk, dwk = plain_norm_rope_grad(s["k"], s["wk"], s["dk"], cos, sin, c)
    return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}


def turned(x, cos, sin, c):
    """The rotation of the first `rot` coordinates."""
    r = c["rot"]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def plain_norm_rope(x, w, cos, sin, c):
    xf = x.float()
    n = xf * torch.rsqrt(xf.square().mean(-1, keepdim=True) + EPS) * w.float()
    return turned(n, cos, sin, c).to(x.dtype)


def plain_norm_rope_grad(x, w, dy, cos, sin, c):
    xf = x.float()
    r = torch.rsqrt(xf.square().mean(-1, keepdim=True) + EPS)
    g = turned(dy.float(), cos, -sin, c)
    u = g * w.float()
    dx = r * u - xf * r ** 3 * (u * xf).mean(-1, keepdim=True)
    return dx.to(x.dtype), (g * xf * r).sum((0, 1))


def own_adamw(s, c):
    from paper_2607_20652_gb300 import dpb
    if "group" not in s:  # what an optimiser keeps of its parameters and states
        s["group"] = dpb.AdamWGroup(s["params"], s["exp_avg"], s["exp_avg_sq"], s.get("m_scale"), s.get("v_scale"))
    s["group"].step(s["grads"], lr=ADAM["lr"], betas=(ADAM["beta1"], ADAM["beta2"]), eps=ADAM["eps"],
                    weight_decay=ADAM["weight_decay"], step=ADAM["step"], seed=ADAM["seed"])
    return adamw_outputs(s)


def adamw_outputs(s):
    return {k: s[k] for k in ("p", "m", "v", "ms", "vs") if k in s}


def plain_adamw(s, c):
    a = ADAM
    g = s["g"].float()
    if c["state"] == "f8":
        m = s["m"].float().view(-1, BLOCK) * s["ms"][:, None]
        v = (s["v"].float().view(-1, BLOCK) * s["vs"][:, None]).square()
        m, v = m.view(-1), v.view(-1)
    else:
        m, v = s["m"], s["v"]
    m = a["beta1"] * m + (1 - a["beta1"]) * g
    v = a["beta2"] * v + (1 - a["beta2"]) * g * g
    c1, c2 = 1 / (1 - a["beta1"] ** a["step"]), 1 / math.sqrt(1 - a["beta2"] ** a["step"])
    p = s["p"].float() * (1 - a["lr"] * a["weight_decay"])
    root = v.sqrt()
    s["p"].copy_(p - a["lr"] * (m * c1) / (root * c2 + a["eps"]))
    if c["state"] == "f8":
        low, high = bits(torch.arange(g.numel(), device="cuda"), a["seed"], a["step"])
        stochastic8(m, low, s["m"], s["ms"], False)
        stochastic8(root, high, s["v"], s["vs"], True)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return adamw_outputs(s)


def mix(x):
    """A published 32-bit integer hash (two rounds of xor-shift and multiply, constants of hash-prospector's lowbias32)."""
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def bits(index, seed, step):
    """Two 16-bit random numbers of a value: from its index in the padded list of tensors, the seed and the step."""
    key = mix((seed & 0xFFFFFFFF) ^ mix((step + 0x9E3779B9 * (1 + (seed >> 32))) & 0xFFFFFFFF))
    r = mix((index & 0xFFFFFFFF) ^ ((key + 0x9E3779B9 * (index >> 32)) & 0xFFFFFFFF))
    return r & 0xFFFF, r >> 16


def stochastic8(x, r, codes, scales, keep):
    """Rounds each value to one of its two e4m3 neighbours, up with the probability of its share of the gap; with
    `keep` nothing that is not zero becomes zero. The block's largest is held exactly, by its scale."""
    b = x.view(-1, BLOCK)
    top = b.abs().amax(1)
    live = top >= 1e-30
    inv = torch.where(live, E4M3_MAX / torch.where(live, top, torch.ones_like(top)), torch.zeros_like(top))
    y = (b * inv[:, None]).view(-1)
    a = y.abs()
    up = ((a.view(torch.int32) + (r << 4).to(torch.int32)) & ~0xFFFFF).view(torch.float32)
    sub = torch.floor(a * 512 + r.float() * (1 / 65536)) * (1 / 512)
    q = torch.where(a >= 2.0 ** -6, up, sub).clamp(max=E4M3_MAX)
    if keep:
        q = torch.where((a > 0) & (q == 0), torch.full_like(q, 2.0 ** -9), q)
    codes.copy_(torch.copysign(q, y).to(torch.float8_e4m3fn))
    scales.copy_(torch.where(live, top * (1 / E4M3_MAX), torch.zeros_like(top)))


# ---- from the definitions, in 64 bits ---------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": exact_attention, "rotary": exact_rotary, "adamw": exact_adamw}[case["op"]](s, case)


def exact_attention(s, c):
    """One head of one sequence at a time."""
    nq, nk = lengths(c)
    group = c["heads"] // c["kv"]
    f8 = dict(dtype=torch.float64, device="cuda")
    o, lse = torch.zeros(s["q"].shape, **f8), torch.full((c["heads"], s["q"].shape[0]), -math.inf, **f8)
    dq, dk, dv = (torch.zeros(t.shape, **f8) for t in (s["q"], s["k"], s["v"]))
    a0 = b0 = 0
    for n, m in zip(nq, nk):
        for h in range(c["heads"] if n and m else 0):
            q = s["q"][a0:a0 + n, h].double()
            k, v = s["k"][b0:b0 + m, h // group].double(), s["v"][b0:b0 + m, h // group].double()
            x = q @ k.t() / math.sqrt(c["dim"])
            if c["causal"]:
                x.masked_fill_(torch.ones(n, m, dtype=torch.bool, device="cuda").triu_(m - n + 1), -math.inf)
            lse[h, a0:a0 + n] = torch.logsumexp(x, 1)
            x = torch.softmax(x, 1).nan_to_num_(0.0)
            o[a0:a0 + n, h] = x @ v
            if c["direction"] == "step":
                do = s["do"][a0:a0 + n, h].double()
                dv[b0:b0 + m, h // group] += x.t() @ do
                x *= do @ v.t() - (do * o[a0:a0 + n, h]).sum(1, keepdim=True)
                x /= math.sqrt(c["dim"])
                dq[a0:a0 + n, h] = x @ k
                dk[b0:b0 + m, h // group] += x.t() @ q
            del x
        a0, b0 = a0 + n, b0 + m
    return {"o": o, "lse": lse} if c["direction"] == "forward" else {"o": o, "dq": dq, "dk": dk, "dv": dv}


def exact_rotary(s, c):
    """The rotation as complex numbers, the gradient by automatic differentiation."""
    turn = torch.complex(s["cos"].double(), s["sin"].double())[s["pos"].long()][:, None]
    r = c["rot"]

    def forward(x, w):
        n = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["dim"] + EPS) * w
        head = n[..., :r].unflatten(-1, (r // 2, 2)) if c["interleaved"] else \
            n[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
        y = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
        y = y if c["interleaved"] else y.transpose(-1, -2)
        return torch.cat([y.flatten(-2), n[..., r:]], -1)

    out = {}
    for name in ("q", "k"):
        x, w = s[name].double().requires_grad_(), s["w" + name].double().requires_grad_()
        y = forward(x, w)
        if c["direction"] == "forward":
            out[name] = y.detach()
        else:
            out["d" + name], out["dw" + name] = torch.autograd.grad(y, (x, w), s["d" + name].double())
    return out


def exact_adamw(s, c):
    a = {k: (v if k in ("step", "seed") else float(v)) for k, v in ADAM.items()}
    g, p = s["g"].double(), s["p"].double()
    if c["state"] == "f8":
        m = s["m"].double() * s["ms"].double().repeat_interleave(BLOCK)
        v = (s["v"].double() * s["vs"].double().repeat_interleave(BLOCK)) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m = m.mul_(a["beta1"]).add_(g, alpha=1 - a["beta1"])
    v = v.mul_(a["beta2"]).addcmul_(g, g, value=1 - a["beta2"])
    del g
    hat = (v / (1 - a["beta2"] ** a["step"])).sqrt_().add_(a["eps"])
    p = p - a["lr"] * a["weight_decay"] * p - a["lr"] * (m / (1 - a["beta1"] ** a["step"])) / hat
    del hat
    if c["state"] == "f32":
        return {"p": p, "m": m, "v": v}
    low, high = bits(torch.arange(m.numel(), device="cuda"), a["seed"], a["step"])
    m, ms = exact_round8(m, low.double() / 65536)
    v, vs = exact_round8(v.sqrt(), high.double() / 65536)
    return {"p": p, "m": m, "v": torch.where((v == 0) & (vs.repeat_interleave(BLOCK) > 0) & (s["live"] > 0), 2.0 ** -9, v),
            "ms": ms, "vs": vs}


def exact_round8(x, share):
    """Each value's place on the e4m3 grid of its block: steps of 2^-9 up to 2^-6, then 8 to each power of two."""
    top = x.view(-1, BLOCK).abs().amax(1)
    y = x / torch.where(top > 0, top / E4M3_MAX, torch.ones_like(top)).repeat_interleave(BLOCK)
    gap = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.sign(y) * (torch.floor(y.abs() / gap + share) * gap).clamp(max=E4M3_MAX), top / E4M3_MAX
