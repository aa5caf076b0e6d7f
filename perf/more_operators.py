"""Measured cases of the operators of a language model's training step: embedding, policy loss, Muon step.

  embed        rows of a table, looked up by token and scaled
  embed_grad   the gradient of the table: scaled sums of the rows of every token
  policy       clipped policy loss with a KL term out of logits, and its gradient in the logits
  muon         one Muon step: momentum, an update orthogonalised by Newton-Schulz products, decay

Where `own` is false, `run` computes the operators out of elementary torch operations; where it is true
it makes the calls of the package's entry points.  `exact` restates the definitions in 64 bits.

Tokens are negative where there is none (padding): such a row of a look-up is zero and has no gradient,
and such a row of a loss has none.
"""

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
NS = (3.4445, -4.7750, 2.0315)            # coefficients of a Newton-Schulz step
STEPS, NS_EPS = 5, 1e-7
LR, MU, DECAY = 0.02, 0.95, 0.01


def listed():
    return [
        # a few sequences' worth of tokens: the call's latency counts
        {"name": "embed 512 of 32000x1024 bf16", "op": "embed", "n": 512, "vocab": 32000, "width": 1024, "table": "bf16", "out": "bf16", "bits": 64},
        # a large batch of a large model: fp32 master table, bf16 activations
        {"name": "embed 65536 of 131072x2048 f32 to bf16", "op": "embed", "n": 65536, "vocab": 131072, "width": 2048, "table": "f32", "out": "bf16", "bits": 64},
        # small batch, small table, odd width
        {"name": "embed_grad 1000 of 10007x321 f16", "op": "embed_grad", "n": 1000, "vocab": 10007, "width": 321, "table": "f32", "out": "f16", "bits": 32},
        # one step of a middle-sized model, gradient in fp32
        {"name": "embed_grad 16384 of 50257x768 bf16", "op": "embed_grad", "n": 16384, "vocab": 50257, "width": 768, "table": "f32", "out": "bf16", "bits": 64},
        # one step of a large model, all 16-bit
        {"name": "embed_grad 65536 of 131072x2048 bf16", "op": "embed_grad", "n": 65536, "vocab": 131072, "width": 2048, "table": "bf16", "out": "bf16", "bits": 64},
        # a short answer, fp32 logits
        {"name": "policy 48x32000 f32", "op": "policy", "n": 48, "vocab": 32000, "type": "f32", "pad": 0, "warm": 1.0},
        # answers of a small model; rows of an odd length, so no row is aligned like the one before it
        {"name": "policy 2047x50257 f16", "op": "policy", "n": 2047, "vocab": 50257, "type": "f16", "pad": 0, "warm": 1.0},
        # answers of a large model, sampled at another temperature, logits padded to a multiple of 128
        {"name": "policy 4096x128256 bf16", "op": "policy", "n": 4096, "vocab": 128256, "type": "bf16", "pad": 64, "warm": 0.8},
        # one odd matrix: latency
        {"name": "muon 1 of 257x129 f32", "op": "muon", "count": 1, "rows": 257, "cols": 129, "heads": 0, "type": "f32", "grad": "f32"},
        # hidden and output weights of 64 workers' MLPs 784-512-10
        {"name": "muon 64 of 512x784 and 10x512 f32", "op": "muon", "count": 64, "rows": 512, "cols": 784, "heads": 10, "type": "f32", "grad": "f32"},
        # the projections of a few layers, higher than wide
        {"name": "muon 6 of 4096x1024 bf16", "op": "muon", "count": 6, "rows": 4096, "cols": 1024, "heads": 0, "type": "bf16", "grad": "bf16"},
        # two large square matrices, fp32 masters of bf16 gradients
        {"name": "muon 2 of 4096x4096 bf16", "op": "muon", "count": 2, "rows": 4096, "cols": 4096, "heads": 0, "type": "bf16", "grad": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "policy", "muon"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op in ("embed", "embed_grad"):
        width = rng.choice([_log(rng, 1, 4096), 8 * _log(rng, 1, 512)])
        vocab = min(_log(rng, 2, 200_000), 250_000_000 // width)
        return {"op": op, "n": min(_log(rng, 1, 100_000), 130_000_000 // width), "vocab": vocab, "width": width,
                "table": rng.choice(["f32", kind]), "out": kind, "bits": rng.choice([32, 64])}
    if op == "policy":
        vocab = _log(rng, 2, 200_000)
        return {"op": op, "n": min(_log(rng, 1, 8192), max(1, 500_000_000 // vocab)), "vocab": vocab, "type": kind,
                "pad": rng.choice([0, 0, 8, 64]), "warm": rng.choice([1.0, 0.7])}
    rows, cols = _log(rng, 1, 4096), _log(rng, 1, 4096)
    low, high = min(rows, cols), max(rows, cols)
    count = max(1, min(_log(rng, 1, 64), int(1e12 / (30.0 * low * low * high))))
    return {"op": op, "count": count, "rows": rows, "cols": cols, "heads": rng.choice([0, 0, 10]),
            "type": rng.choice(["f32", kind]), "grad": kind}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _tokens(n, vocab, gen, dev):
    """Tokens as text has them: few words often, most words rarely; one in fifty is padding."""
    u = torch.rand(n, generator=gen, device=dev, dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab + 1.0)) - 1.0).long().clamp_(0, vocab - 1)
    step = 7919 if vocab % 7919 else 7907                    # frequent words are spread over the table
    t = (rank * step) % vocab
    return torch.where(torch.rand(n, generator=gen, device=dev) < 0.02, torch.full_like(t, -1), t)


def _shapes(case):
    return [(case["rows"], case["cols"])] + ([(case["heads"], case["rows"])] if case["heads"] else [])


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    st = {"op": case["op"], "case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    if case["op"] in ("embed", "embed_grad"):
        st["t"] = _tokens(case["n"], case["vocab"], gen, dev).to(torch.int32 if case["bits"] == 32 else torch.int64)
        st["scale"] = math.sqrt(case["width"])
        if case["op"] == "embed":
            st["table"] = (normal(case["vocab"], case["width"]) * 0.02).to(DTYPES[case["table"]])
        else:
            st["dout"] = (normal(case["n"], case["width"]) * 1e-2).to(DTYPES[case["out"]])
        return st
    if case["op"] == "policy":
        n, v = case["n"], case["vocab"]
        z = normal(n, v + case["pad"]).mul_(2.0).to(DTYPES[case["type"]])
        st["z"] = z[:, :v]
        st["t"] = _tokens(n, v, gen, dev)
        at = st["t"].clamp_min(0)
        logp = torch.cat([torch.log_softmax(part.float() / case["warm"], 1).gather(1, k[:, None])[:, 0]
                          for part, k in zip(st["z"].split(512), at.split(512))])
        st["old"] = logp + 0.2 * normal(n)                   # the policy that sampled the tokens, some updates ago
        st["ref"] = logp + 0.3 * normal(n)
        st["adv"] = normal(n)
        keep = (torch.rand(n, generator=gen, device=dev) < 0.9).float()
        st["w"] = keep / keep.sum().clamp_min(1.0)
        # 16-bit gradients of a mean over tokens need a factor to stay in their range
        st["up"] = torch.full((1,), 65536.0 if case["type"] == "f16" else 1.0, device=dev)
        return st
    st["p"], st["g"], st["m"] = [], [], []
    for rows, cols in _shapes(case):
        k, r = case["count"], min(8, rows, cols)

        def slope():
            """A gradient: a few directions over noise, each matrix with a size of its own."""
            size = torch.exp(normal(k, 1, 1) - 6.0)
            return size * (torch.bmm(normal(k, rows, r), normal(k, r, cols)) + normal(k, rows, cols))

        st["p"].append((0.04 * normal(k, rows, cols)).to(DTYPES[case["type"]]))
        st["g"].append(slope().to(DTYPES[case["grad"]]))
        st["m"].append(0.5 * slope())
    return st


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def _plain_embed(st):
    t, table = st["t"].long(), st["table"]
    rows = table[t.clamp_min(0)].float() * st["scale"]
    return torch.where(t[:, None] >= 0, rows, torch.zeros_like(rows)).to(DTYPES[st["case"]["out"]])


def _plain_embed_grad(st):
    case, t = st["case"], st["t"].long()
    d = st["dout"].float() * (t >= 0).float()[:, None]
    grad = torch.zeros(case["vocab"], case["width"], device=d.device).index_add_(0, t.clamp_min(0), d)
    return (grad * st["scale"]).to(DTYPES[case["table"]])


def _plain_policy(st):
    case, t = st["case"], st["t"]
    some = (t >= 0) & (st["w"] != 0)
    at = t.clamp_min(0)[:, None]
    z = st["z"].float()
    d = z - z.amax(1, keepdim=True)
    e = (d * (1.0 / case["warm"])).exp()
    # what belongs to a row is held in 64 bits: a ratio next to a border of the clip has to fall on its own side
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    logp = (d.gather(1, at).double() / case["warm"] - total.log())[:, 0]
    ratio = (logp - st["old"]).exp()
    a, w = st["adv"], torch.where(some, st["w"], torch.zeros_like(st["w"]))
    one, two = ratio * a, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * a
    d = st["ref"] - logp
    kl = d.exp() - d - 1.0
    each = w * (KL * kl - torch.minimum(one, two))
    each = torch.where(some, each, torch.zeros_like(each))
    slope = w * (KL * (1.0 - d.exp()) - torch.where(one <= two, one, torch.zeros_like(one)))
    slope = torch.where(some, slope, torch.zeros_like(slope)) * (st["up"] / case["warm"])
    dz = e * (-slope[:, None] / total).float()
    dz.scatter_add_(1, at, slope[:, None].float())
    logp = torch.where(some, logp, torch.zeros_like(logp))
    return each.sum().float(), each.float(), logp.float(), dz.to(st["z"].dtype)


def _plain_muon_one(p, g, m):
    rows, cols = p.shape[1:]
    g = g.float()
    m.copy_(m * MU + g * (1.0 - MU))
    u = m * MU + g * (1.0 - MU)
    if rows > cols:
        u = u.transpose(1, 2)
    norm = u.square().sum((1, 2), keepdim=True, dtype=torch.float64).sqrt().clamp_min(NS_EPS)
    x = (u / norm).float()
    a, b, c = NS
    for _ in range(STEPS):
        s = x @ x.transpose(1, 2)
        x = a * x + (b * s + c * (s @ s)) @ x
    if rows > cols:
        x = x.transpose(1, 2)
    size = math.sqrt(max(1.0, rows / cols))
    p.copy_(p.float() * (1.0 - LR * DECAY) - (LR * size) * x)
    return p, m


def _plain_muon(st):
    return [x for group in zip(st["p"], st["g"], st["m"]) for x in _plain_muon_one(*group)]


def _own_embed(st, pkg, stream):
    case = st["case"]
    out = torch.empty(case["n"], case["width"], dtype=DTYPES[case["out"]], device="cuda")
    pkg.rfast_embedding(st["t"].data_ptr(), st["table"].data_ptr(), out.data_ptr(), tokens=case["n"], vocab=case["vocab"], width=case["width"],
                        scale=st["scale"], token_bits=case["bits"], table_type=case["table"], out_type=case["out"], cuda_stream=stream)
    return out


def _own_embed_grad(st, pkg, stream):
    case = st["case"]
    grad = torch.empty(case["vocab"], case["width"], dtype=DTYPES[case["table"]], device="cuda")
    need = pkg.rfast_embedding_workspace(tokens=case["n"], vocab=case["vocab"], width=case["width"])
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    pkg.rfast_embedding_backward(st["t"].data_ptr(), st["dout"].data_ptr(), grad.data_ptr(), tokens=case["n"], vocab=case["vocab"],
                                 width=case["width"], scale=st["scale"], token_bits=case["bits"], out_type=case["out"], table_type=case["table"],
                                 workspace=work.data_ptr(), workspace_bytes=need, cuda_stream=stream)
    return grad


def _own_policy(st, pkg, stream):
    case, z = st["case"], st["z"]
    n, v = case["n"], case["vocab"]
    dz = torch.empty(n, v, dtype=z.dtype, device="cuda")
    small = torch.empty(2 * n + 1, device="cuda")
    loss, each, logp = small[2 * n], small[:n], small[n:2 * n]
    pkg.rfast_policy_loss(z.data_ptr(), st["t"].data_ptr(), st["old"].data_ptr(), st["adv"].data_ptr(), tokens=n, vocab=v, d_loss=loss.data_ptr(),
                          d_token_loss=each.data_ptr(), d_logp=logp.data_ptr(), d_dlogits=dz.data_ptr(), d_ref_logp=st["ref"].data_ptr(),
                          d_weight=st["w"].data_ptr(), d_loss_scale=st["up"].data_ptr(), temperature=case["warm"], clip_low=CLIP_LOW,
                          clip_high=CLIP_HIGH, kl_coef=KL, type=case["type"], logits_stride=z.stride(0), cuda_stream=stream)
    return loss, each, logp, dz


def _own_muon(st, pkg, stream):
    case = st["case"]
    rows, cols, p, g, m = [], [], [], [], []
    for (r, c), pp, gg, mm in zip(_shapes(case), st["p"], st["g"], st["m"]):
        rows += [r] * case["count"]
        cols += [c] * case["count"]
        for to, t in ((p, pp), (g, gg), (m, mm)):
            to += [t.data_ptr() + k * r * c * t.element_size() for k in range(case["count"])]
    need = pkg.rfast_muon_workspace(rows, cols, param_type=case["type"])
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    pkg.rfast_muon_step(p, g, m, rows, cols, lr=LR, momentum=MU, weight_decay=DECAY, nesterov=True, eps=NS_EPS, iterations=STEPS,
                        size_rule="spectral", param_type=case["type"], grad_type=case["grad"], workspace=work.data_ptr(), workspace_bytes=need,
                        cuda_stream=stream)
    return [x for group in zip(st["p"], st["m"]) for x in group]


def run(state):
    op = state["op"]
    if own:
        import paper_2307_11617_b200 as pkg
        stream = torch.cuda.current_stream().cuda_stream
        return {"embed": _own_embed, "embed_grad": _own_embed_grad, "policy": _own_policy, "muon": _own_muon}[op](state, pkg, stream)
    return {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "policy": _plain_policy, "muon": _plain_muon}[op](state)


def work(case):
    if case["op"] in ("embed", "embed_grad"):
        n, v, w = case["n"], case["vocab"], case["width"]
        # distinct tokens of n draws that are even in the logarithm of their rank, 98 % of n
        ranks = (1 << k for k in range(v.bit_length()))
        distinct = sum((min(v + 1, 2 * r) - r) * -math.expm1(-0.98 * n * math.log1p(1.0 / (1.5 * r)) / math.log(v + 1.0)) for r in ranks)
        if case["op"] == "embed":
            return {"bytes": int(distinct) * w * BYTES[case["table"]] + n * w * BYTES[case["out"]] + n * case["bits"] // 8, "flops": n * w}
        return {"bytes": v * w * BYTES[case["table"]] + int(0.98 * n) * w * BYTES[case["out"]] + n * case["bits"] // 8, "flops": 2 * n * w}
    if case["op"] == "policy":
        n, v = case["n"], case["vocab"]
        # a tenth of the rows has no weight and needs no logits, but a gradient of zero
        return {"bytes": int(1.88 * n * v) * BYTES[case["type"]] + 32 * n, "flops": 8 * n * v}
    size = flops = 0
    for rows, cols in _shapes(case):
        low, high = min(rows, cols), max(rows, cols)
        # two of the three products of an iteration are symmetric: half of each is enough
        flops += case["count"] * STEPS * (3 * low * low * high + low ** 3)
        size += case["count"] * rows * cols * (2 * BYTES[case["type"]] + BYTES[case["grad"]] + 8)
    return {"bytes": size, "flops": flops}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_policy(st):
    case = st["case"]
    parts = []
    for rows in torch.arange(case["n"], device="cuda").split(256):
        z = st["z"][rows].double() / case["warm"]
        t, w = st["t"][rows], st["w"][rows].double()
        live = torch.logical_and(t >= 0, w != 0).double()
        pick = torch.where(t >= 0, t, 0)
        lse = torch.logsumexp(z, 1)
        logp = z[torch.arange(len(t), device="cuda"), pick] - lse
        rho = torch.exp(logp - st["old"][rows].double())
        a = st["adv"][rows].double()
        held = torch.minimum(torch.maximum(rho, torch.full_like(rho, 1 - CLIP_LOW)), torch.full_like(rho, 1 + CLIP_HIGH))
        gap = st["ref"][rows].double() - logp
        loss = w * live * (-torch.minimum(rho * a, held * a) + KL * (torch.expm1(gap) - gap))
        # the clip holds where the ratio has left the range on the side that the advantage favours
        stuck = ((a > 0) & (rho > 1 + CLIP_HIGH)) | ((a < 0) & (rho < 1 - CLIP_LOW))
        dlogp = w * live * (-a * rho * (~stuck).double() - KL * torch.expm1(gap)) * st["up"].double()
        dz = -torch.exp(z - lse[:, None])
        dz[torch.arange(len(t), device="cuda"), pick] += 1.0
        parts.append((loss, logp * live, dz * (dlogp / case["warm"])[:, None]))
    loss, logp, dz = (torch.cat(x) for x in zip(*parts))
    return loss.sum(), loss, logp, dz


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "embed":
        t = st["t"].long()
        out = torch.index_select(st["table"], 0, torch.where(t < 0, 0, t)).double().mul_(st["scale"])
        out[t < 0] = 0.0
        return out
    if case["op"] == "embed_grad":
        t = st["t"].long()
        order = torch.argsort(t, stable=True)
        order = order[int((t < 0).sum()):]
        grad = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
        for part in order.split(1 << 14):
            grad.index_put_((t[part],), st["dout"][part].double(), accumulate=True)
        return grad.mul_(st["scale"])
    if case["op"] == "policy":
        return _exact_policy(st)
    out = []
    for p, g, m in zip(st["p"], st["g"], st["m"]):
        rows, cols = p.shape[1:]
        g, m = g.double(), m.double()
        m = MU * m + (1 - MU) * g
        x = (1 - MU) * g + MU * m
        x = x / torch.linalg.matrix_norm(x, keepdim=True).clamp_min(NS_EPS)
        # the other side's products give the same matrix: a x + x (b x'x + c (x'x)^2)
        for _ in range(STEPS):
            if rows <= cols:
                s = torch.matmul(x, x.mT)
                x = NS[0] * x + torch.matmul(NS[1] * s + NS[2] * torch.matmul(s, s), x)
            else:
                s = torch.matmul(x.mT, x)
                x = NS[0] * x + torch.matmul(x, NS[1] * s + NS[2] * torch.matmul(s, s))
        out += [p.double() * (1 - LR * DECAY) - LR * math.sqrt(max(1.0, rows / cols)) * x, m]
    return out
