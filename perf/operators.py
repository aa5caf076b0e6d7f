"""Measured cases of the training-step operators: gradient norm, AdamW step, group norm.

  grad_norm   2-norm over many gradient tensors and the factor that clips it
  adamw       one AdamW step over many tensors, moments in 32 bits
  adamw8      the same step, moments in 8 bits with one scale for each block of 256 values
  gn          group norm with an activation, channels last
  gn_grad     its backward pass: gradients of the input, the scale and the shift

Where `own` is false, `run` computes the operators out of elementary torch operations; where it is true
it makes the calls of the package's entry points.  `exact` restates the definitions in 64 bits.

Tensors of one list lie in one flat buffer, each from a multiple of 256 elements on, as a
program lays out parameters, gradients and moments of a network (and as the engine lays out the
rows of its workers); what lies between them is zero and stays zero.
"""

import math

import numpy as np
import torch

own = False

BLOCK = 256                      # values that share a scale in the 8-bit moments
TOP = 448.0                      # largest e4m3 value
FLOOR = 2.0 ** -100              # least scale of a block
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 1e-2
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
GN_EPS = 1e-5


def listed():
    return [
        # the clip of a small model: 16 workers' softmax regressions (10 x 784 weights and 10 biases each)
        {"name": "grad_norm softmax rows f32", "op": "grad_norm", "sizes": "softmax", "count": 16, "grad": "f32"},
        # the clip of a large model whose gradients are bf16
        {"name": "grad_norm large bf16", "op": "grad_norm", "sizes": "even", "count": 9, "each": 11_200_000, "grad": "bf16"},
        # a step of those 16 regressions: little data, the call's latency counts
        {"name": "adamw softmax rows f32", "op": "adamw", "sizes": "softmax", "count": 16, "param": "f32", "grad": "f32", "clip": False},
        # 64 workers' MLPs 784-512-10: 256 tensors from 10 to 401408 values, clipped
        {"name": "adamw mlp f32 clipped", "op": "adamw", "sizes": "mlp", "count": 64, "param": "f32", "grad": "f32", "clip": True},
        # the same MLPs with moments in 8 bits
        {"name": "adamw8 mlp f32", "op": "adamw8", "sizes": "mlp", "count": 64, "param": "f32", "grad": "f32", "clip": False},
        # a large model held in bf16, odd tensor sizes, clipped
        {"name": "adamw8 large bf16 clipped", "op": "adamw8", "sizes": "even", "count": 7, "each": 11_199_983, "param": "bf16", "grad": "bf16", "clip": True},
        # hidden layer of 64 workers' MLPs, 64 rows each, every worker with a scale and shift of its own
        {"name": "gn mlp hidden f32", "op": "gn", "n": 4096, "s": 1, "c": 512, "groups": 16, "sets": 64, "type": "f32", "act": "relu", "pad": 0},
        # an image network's early stage
        {"name": "gn 32x56x56x256 bf16", "op": "gn", "n": 32, "s": 56 * 56, "c": 256, "groups": 32, "sets": 1, "type": "bf16", "act": "silu", "pad": 0},
        # few large images, ten channels a group, read out of a wider tensor
        {"name": "gn 2x128x128x320 f16", "op": "gn", "n": 2, "s": 128 * 128, "c": 320, "groups": 32, "sets": 1, "type": "f16", "act": "silu", "pad": 64},
        # the backward pass of the hidden layer
        {"name": "gn_grad mlp hidden f32", "op": "gn_grad", "n": 4096, "s": 1, "c": 512, "groups": 16, "sets": 64, "type": "f32", "act": "silu", "pad": 0},
        # the backward pass of the early stage
        {"name": "gn_grad 32x56x56x256 bf16", "op": "gn_grad", "n": 32, "s": 56 * 56, "c": 256, "groups": 32, "sets": 1, "type": "bf16", "act": "silu", "pad": 0},
        # a ragged one: three channels a group, odd picture
        {"name": "gn_grad 5x57x33x96 f16", "op": "gn_grad", "n": 5, "s": 57 * 33, "c": 96, "groups": 32, "sets": 1, "type": "f16", "act": "none", "pad": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["grad_norm", "adamw", "adamw8", "gn", "gn_grad"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op in ("grad_norm", "adamw", "adamw8"):
        count = _log(rng, 1, 300)
        each = min(_log(rng, 10, 20_000_000), 70_000_000 // count)
        case = {"op": op, "sizes": "spread", "count": count, "each": each, "grad": kind}
        if op != "grad_norm":
            case["param"] = rng.choice(["f32", kind])
            case["clip"] = rng.random() < 0.5
        return case
    cg = rng.choice([1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 32, 64])
    groups = rng.choice([1, 2, 4, 8, 16, 32])
    c = cg * groups
    s = rng.choice([1, _log(rng, 1, 20_000)])
    n = min(_log(rng, 1, 8192), max(1, 12_000_000 // (s * c)))
    sets = rng.choice([1, 1, n]) if n <= 64 else 1
    return {"op": op, "n": n, "s": s, "c": c, "groups": groups, "sets": sets, "type": kind,
            "act": rng.choice(["none", "relu", "silu"] if op == "gn" else ["none", "silu"]), "pad": rng.choice([0, 0, 8, 24])}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _sizes(case):
    """Element counts of the case's tensors."""
    n = case["count"]
    if case["sizes"] == "softmax":
        return [10 * 784, 10] * n
    if case["sizes"] == "mlp":
        return [512 * 784, 512, 10 * 512, 10] * n
    if case["sizes"] == "even":
        return [case["each"]] * n
    # spread: from a tenth of `each` up to it, odd sizes among them
    return [max(1, case["each"] * (1 + (7 * k) % 10) // 10 - k % 3) for k in range(n)]


def _layout(case):
    numel = np.asarray(_sizes(case), dtype=np.int64)
    room = (numel + BLOCK - 1) // BLOCK * BLOCK
    start = np.concatenate([[0], np.cumsum(room)[:-1]]).astype(np.int64)
    return numel, start, int(room.sum())


def _quantised(v):
    """Codes and scales of [blocks, 256] values in 8 bits."""
    scale = (v.abs().amax(1, keepdim=True) * (1.0 / TOP)).clamp_min(FLOOR)
    code = (v * (1.0 / scale)).clamp(-TOP, TOP).to(torch.float8_e4m3fn)
    return code, scale


def _second_codes(r, scale):
    """Codes of the roots of the second moments: a positive root keeps a positive code."""
    u = (r * (1.0 / scale)).clamp(max=TOP)
    return torch.where((r > 0) & (u < 2.0 ** -9), torch.full_like(u, 2.0 ** -9), u).to(torch.float8_e4m3fn)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    st = {"op": case["op"], "case": case}
    if case["op"] in ("grad_norm", "adamw", "adamw8"):
        numel, start, total = _layout(case)
        st["numel"], st["start"] = numel, start
        # elements that belong to a tensor; what lies between is zero
        edge = torch.zeros(total + 1, dtype=torch.int8, device=dev)
        edge[torch.as_tensor(start, device=dev)] += 1
        ends = torch.as_tensor(start + numel, device=dev)
        edge[ends] -= 1
        live = torch.cumsum(edge[:-1], 0, dtype=torch.int8).bool()

        def normal(scale):
            return torch.randn(total, generator=gen, device=dev) * scale * live

        # blocks of very different gradients, some that saw none (rows of a table that were not used)
        blocks = total // BLOCK
        size = torch.exp(2.0 * torch.randn(blocks, generator=gen, device=dev) - 7.0)
        size = torch.where(torch.rand(blocks, generator=gen, device=dev) < 0.05, torch.zeros_like(size), size)
        size = size.repeat_interleave(BLOCK)
        st["g"] = normal(size).to(DTYPES[case["grad"]])
        st["max_norm"] = 1.0
        if case["op"] == "grad_norm":
            return st
        st["p"] = normal(0.05).to(DTYPES[case["param"]])
        st["t"] = 500                                            # steps taken before
        m = normal(0.3 * size)
        r = (size * live) * torch.exp(0.5 * torch.randn(total, generator=gen, device=dev))   # root of the second moment
        if case["op"] == "adamw":
            st["m"], st["v"] = m, r * r
        else:
            code, scale = _quantised(m.view(-1, BLOCK))
            st["m"], st["ms"] = code.view(torch.uint8).view(-1), scale.view(-1)
            _, scale = _quantised(r.view(-1, BLOCK))
            st["v"], st["vs"] = _second_codes(r.view(-1, BLOCK), scale).view(torch.uint8).view(-1), scale.view(-1)
        return st
    n, s, c, g = case["n"], case["s"], case["c"], case["groups"]
    kind = DTYPES[case["type"]]
    wide = torch.randn(n, s, c + case["pad"], generator=gen, device=dev)
    # every channel with a level and a spread of its own
    wide = wide * (0.5 + torch.rand(c + case["pad"], generator=gen, device=dev)) + torch.randn(c + case["pad"], generator=gen, device=dev)
    st["x"] = wide.to(kind)[:, :, :c]
    st["gamma"] = 1.0 + 0.2 * torch.randn(case["sets"], c, generator=gen, device=dev)
    st["beta"] = 0.2 * torch.randn(case["sets"], c, generator=gen, device=dev)
    if case["op"] == "gn_grad":
        st["dy"] = torch.randn(n, s, c, generator=gen, device=dev).to(kind)
        x = st["x"].double().reshape(n, s, g, c // g)            # what the forward pass left
        mean = x.mean((1, 3))
        var = (x - mean[:, None, :, None]).square().mean((1, 3))
        st["mean"], st["rstd"] = mean.float(), (var + GN_EPS).rsqrt().float()
    return st


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def _plain_norm(st):
    norm = st["g"].double().square().sum().sqrt()
    return norm.float(), (st["max_norm"] / norm.clamp_min(st["max_norm"])).float()


def _plain_adamw(st):
    t = st["t"] = st["t"] + 1
    g = st["g"].float()
    out = []
    if st["case"]["clip"]:
        norm, scale = _plain_norm(st)
        out = [norm, scale]
        g = g * scale
    if st["op"] == "adamw":
        m0, v0 = st["m"], st["v"]
    else:
        m0 = (st["m"].view(torch.float8_e4m3fn).float().view(-1, BLOCK) * st["ms"][:, None]).view(-1)
        r0 = (st["v"].view(torch.float8_e4m3fn).float().view(-1, BLOCK) * st["vs"][:, None]).view(-1)
        v0 = r0 * r0
    m = m0 * BETA1 + g * (1.0 - BETA1)
    v = v0 * BETA2 + g * g * (1.0 - BETA2)
    r = v.sqrt()
    step = m / (r * (1.0 / math.sqrt(1.0 - BETA2 ** t)) + EPS)
    p = st["p"].float()
    st["p"].copy_(p * (1.0 - LR * DECAY) - step * (LR / (1.0 - BETA1 ** t)))
    if st["op"] == "adamw":
        st["m"].copy_(m)
        st["v"].copy_(v)
        return out + [st["p"], st["m"], st["v"]]
    code, scale = _quantised(m.view(-1, BLOCK))
    st["m"].copy_(code.view(torch.uint8).view(-1))
    st["ms"].copy_(scale.view(-1))
    _, scale = _quantised(r.view(-1, BLOCK))
    st["v"].copy_(_second_codes(r.view(-1, BLOCK), scale).view(torch.uint8).view(-1))
    st["vs"].copy_(scale.view(-1))
    return out + [st["p"]] + _values(st)


def _values(st):
    """The 8-bit moments as the numbers they hold, the first moment and the root of the second, in units
    of the scales that follow."""
    return [st["m"].view(torch.float8_e4m3fn), st["v"].view(torch.float8_e4m3fn), st["ms"], st["vs"]]


def _own_norm(st, pkg, stream):
    out = torch.empty(2, device="cuda")
    work = torch.empty(pkg.GRAD_NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    g = st["g"]
    pkg.rfast_grad_norm(g.data_ptr() + st["start"] * g.element_size(), st["numel"], st["max_norm"], out.data_ptr(), out.data_ptr() + 4,
                        work.data_ptr(), work.numel(), grad_type=st["case"]["grad"], cuda_stream=stream)
    return out


def _own_adamw(st, pkg, stream):
    t = st["t"] = st["t"] + 1
    out, clip = [], None
    if st["case"]["clip"]:
        clip = _own_norm(st, pkg, stream)
        out = [clip[0], clip[1]]
    at, p, g, m, v = st["start"], st["p"], st["g"], st["m"], st["v"]
    more = {}
    if st["op"] == "adamw8":
        more = {"m_scale": st["ms"].data_ptr() + at // BLOCK * 4, "v_scale": st["vs"].data_ptr() + at // BLOCK * 4}
    pkg.rfast_adamw_step(p.data_ptr() + at * p.element_size(), g.data_ptr() + at * g.element_size(), m.data_ptr() + at * m.element_size(),
                         v.data_ptr() + at * v.element_size(), st["numel"], step=t, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY,
                         param_type=st["case"]["param"], grad_type=st["case"]["grad"],
                         d_grad_scale=0 if clip is None else clip.data_ptr() + 4, cuda_stream=stream, **more)
    return out + [p] + (_values(st) if st["op"] == "adamw8" else [m, v])


def _plain_gn(st):
    case, x = st["case"], st["x"].float()
    n, s, c, g = case["n"], case["s"], case["c"], case["groups"]
    q = x.reshape(n, s, g, c // g)
    # 64 bits for the long sums
    mean = q.mean((1, 3), dtype=torch.float64).float()
    d = q - mean[:, None, :, None]
    rstd = (d.square().mean((1, 3), dtype=torch.float64) + GN_EPS).rsqrt().float()
    u = (d * rstd[:, None, :, None]).reshape(case["sets"], -1, s, c) * st["gamma"][:, None, None, :] + st["beta"][:, None, None, :]
    u = u.reshape(n, s, c)
    y = u.clamp_min(0) if case["act"] == "relu" else u / (1 + (-u).exp()) if case["act"] == "silu" else u
    return y.to(st["x"].dtype), mean, rstd


def _plain_gn_grad(st):
    case, x, dy = st["case"], st["x"].float(), st["dy"].float()
    n, s, c, g, k = case["n"], case["s"], case["c"], case["groups"], case["sets"]
    h = ((x.reshape(n, s, g, c // g) - st["mean"][:, None, :, None]) * st["rstd"][:, None, :, None]).reshape(k, -1, s, c)
    gamma, beta = st["gamma"][:, None, None, :], st["beta"][:, None, None, :]
    du = dy.reshape(k, -1, s, c)
    if case["act"] == "silu":
        u = h * gamma + beta
        sig = 1 / (1 + (-u).exp())
        du = du * sig * (1 + u * (1 - sig))
    elif case["act"] == "relu":
        du = du * (h * gamma + beta > 0)
    dgamma = (du * h).sum((1, 2), dtype=torch.float64).float()
    dbeta = du.sum((1, 2), dtype=torch.float64).float()
    dh = (du * gamma).reshape(n, s, g, c // g)
    h = h.reshape(n, s, g, c // g)
    one = dh.mean((1, 3), keepdim=True, dtype=torch.float64).float()
    two = (dh * h).mean((1, 3), keepdim=True, dtype=torch.float64).float()
    dx = (dh - one - h * two) * st["rstd"][:, None, :, None]
    return dx.reshape(n, s, c).to(st["x"].dtype), dgamma, dbeta


def _own_gn(st, pkg, stream):
    case, x = st["case"], st["x"]
    n, s, c, g = case["n"], case["s"], case["c"], case["groups"]
    y = torch.empty(n, s, c, dtype=x.dtype, device="cuda")
    stats = torch.empty(2, n, g, device="cuda")
    shape = {"samples": n, "positions": s, "channels": c, "groups": g, "samples_per_set": n // case["sets"], "type": case["type"], "act": case["act"]}
    need = pkg.rfast_group_norm_workspace(**shape)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    pkg.rfast_group_norm(x.data_ptr(), st["gamma"].data_ptr(), st["beta"].data_ptr(), y.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(),
                         eps=GN_EPS, x_strides=x.stride()[:2], workspace=work.data_ptr(), workspace_bytes=need, cuda_stream=stream, **shape)
    return y, stats[0], stats[1]


def _own_gn_grad(st, pkg, stream):
    case, x, dy = st["case"], st["x"], st["dy"]
    n, s, c, g = case["n"], case["s"], case["c"], case["groups"]
    dx = torch.empty(n, s, c, dtype=x.dtype, device="cuda")
    dgamma = torch.empty(case["sets"], c, device="cuda")
    dbeta = torch.empty(case["sets"], c, device="cuda")
    shape = {"samples": n, "positions": s, "channels": c, "groups": g, "samples_per_set": n // case["sets"], "type": case["type"], "act": case["act"]}
    need = pkg.rfast_group_norm_workspace(backward=True, **shape)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    pkg.rfast_group_norm_backward(dy.data_ptr(), x.data_ptr(), st["gamma"].data_ptr(), st["beta"].data_ptr(), st["mean"].data_ptr(),
                                  st["rstd"].data_ptr(), dx.data_ptr(), dgamma.data_ptr(), dbeta.data_ptr(), x_strides=x.stride()[:2],
                                  workspace=work.data_ptr(), workspace_bytes=need, cuda_stream=stream, **shape)
    return dx, dgamma, dbeta


def run(state):
    op = state["op"]
    if own:
        import paper_2307_11617_b200 as pkg
        stream = torch.cuda.current_stream().cuda_stream
        if op == "grad_norm":
            out = _own_norm(state, pkg, stream)
            return out[0], out[1]
        if op in ("adamw", "adamw8"):
            return _own_adamw(state, pkg, stream)
        return _own_gn(state, pkg, stream) if op == "gn" else _own_gn_grad(state, pkg, stream)
    if op == "grad_norm":
        return _plain_norm(state)
    if op in ("adamw", "adamw8"):
        return _plain_adamw(state)
    return _plain_gn(state) if op == "gn" else _plain_gn_grad(state)


def work(case):
    if case["op"] in ("grad_norm", "adamw", "adamw8"):
        n = sum(_sizes(case))
        blocks = sum(-(-k // BLOCK) for k in _sizes(case))
        if case["op"] == "grad_norm":
            return {"bytes": n * BYTES[case["grad"]] + 8, "flops": 2 * n}
        moments = 16 * n if case["op"] == "adamw" else 4 * n + 16 * blocks
        return {"bytes": n * (2 * BYTES[case["param"]] + BYTES[case["grad"]]) + moments, "flops": (18 if case["clip"] else 15) * n}
    n, b = case["n"] * case["s"] * case["c"], BYTES[case["type"]]
    small = 8 * case["n"] * case["groups"] + 8 * case["sets"] * case["c"]
    if case["op"] == "gn":
        return {"bytes": 2 * n * b + small, "flops": 10 * n}
    return {"bytes": 3 * n * b + small + 8 * case["sets"] * case["c"], "flops": 24 * n}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def _e4m3_values():
    """The non-negative values of the 8-bit type: 3 bits of fraction, exponent bias 7."""
    return [(f / 8.0) * 2.0 ** -6 if e == 0 else (1 + f / 8.0) * 2.0 ** (e - 7) for e in range(16) for f in range(8) if not (e == 15 and f == 7)]


def _nearest(v):
    """Nearest representable value, a tie to the even code."""
    table = torch.tensor(_e4m3_values(), dtype=torch.float64, device=v.device)
    half = (table[1:] + table[:-1]) / 2
    a = v.abs()
    low = torch.searchsorted(half, a)                      # number of borders below a
    tie = (low < half.numel()) & (a == half[low.clamp_max(half.numel() - 1)])
    low = torch.where(tie & (low % 2 == 1), low + 1, low)
    return torch.sign(v) * table[low]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("grad_norm", "adamw", "adamw8"):
        g = st["g"].double()
        norm = torch.linalg.vector_norm(g)
        clip = 1.0 if norm <= 1.0 else 1.0 / norm
        if case["op"] == "grad_norm":
            return norm, torch.as_tensor(clip, dtype=torch.float64)
        out = [norm, torch.as_tensor(clip, dtype=torch.float64)] if case["clip"] else []
        if case["clip"]:
            g = clip * g
        t = 501
        if case["op"] == "adamw":
            m, v = st["m"].double(), st["v"].double()
        else:
            value = torch.tensor(_e4m3_values() + [math.nan], dtype=torch.float64, device=g.device)
            sign = 1.0 - 2.0 * (st["m"] >= 128).double()
            m = sign * value[(st["m"] & 127).long()] * st["ms"].double().repeat_interleave(BLOCK)
            v = (value[st["v"].long()] * st["vs"].double().repeat_interleave(BLOCK)) ** 2
        m.mul_(BETA1).add_(g, alpha=1 - BETA1)
        v.mul_(BETA2).addcmul_(g, g, value=1 - BETA2)
        p = st["p"].double()
        p = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
        if case["op"] == "adamw":
            return out + [p, m, v]
        held, scales = [], []
        for q, least in ((m, 0.0), (v.sqrt(), 2.0 ** -9)):
            q = q.view(-1, BLOCK)
            scale = (q.abs().amax(1, keepdim=True) / TOP).clamp_min(FLOOR)
            if least:                                        # a positive root keeps a positive code
                q = torch.where((q > 0) & (q < least * scale), least * scale, q)
            code = torch.cat([_nearest(part / size) for part, size in zip(q.split(1 << 16), scale.split(1 << 16))])
            held.append(code.view(-1))
            scales.append(scale.view(-1))
        return out + [p] + held + scales
    n, s, c, g, k = case["n"], case["s"], case["c"], case["groups"], case["sets"]
    x = st["x"].double().unflatten(2, (g, c // g))
    gamma = st["gamma"].double().repeat_interleave(n // k, 0).view(n, 1, g, c // g)
    beta = st["beta"].double().repeat_interleave(n // k, 0).view(n, 1, g, c // g)
    var, mean = torch.var_mean(x, (1, 3), correction=0, keepdim=True)
    if case["op"] == "gn":
        rstd = 1 / torch.sqrt(var + GN_EPS)
        u = (x - mean) * rstd * gamma + beta
        y = torch.relu(u) if case["act"] == "relu" else u * torch.sigmoid(u) if case["act"] == "silu" else u
        return y.flatten(2), mean.view(n, g), rstd.view(n, g)
    mean, rstd = st["mean"].double().view(n, 1, g, 1), st["rstd"].double().view(n, 1, g, 1)
    h = (x - mean) * rstd
    u = h * gamma + beta
    slope = torch.ones_like(u)
    if case["act"] == "silu":
        sig = torch.sigmoid(u)
        slope = sig + u * sig * (1 - sig)
    elif case["act"] == "relu":
        slope = (u > 0).double()
    du = st["dy"].double().unflatten(2, (g, c // g)) * slope
    size = s * (c // g)
    dh = du * gamma
    dx = rstd * (dh - dh.sum((1, 3), keepdim=True) / size - h * ((dh * h).sum((1, 3), keepdim=True) / size))
    per = lambda a: a.sum(1).view(k, n // k, c).sum(1)  # noqa: E731
    return dx.flatten(2), per(du * h), per(du)
