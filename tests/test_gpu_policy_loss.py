"""Policy loss and its gradient against a plain restatement in 64 bits.

u = 2^-24.  With R = log2(e) / T times the spread of a row's finite logits: a term 2^(z k - c) of the running sum is off by 2^-22 (the
power) + ln 2 (u R' + ...) where the exponent's rounding is u of at most R + 1; the sum adds u per addition of a chain of at most
n / team + 16 (team = 32 up to 1024 logits, 128 up to 8192, 512 beyond), and a rescale (2^-22 + u) each time the merged maximum grows, and
at three merges.
Rounding k to fp32 is a change of T by u / 2, which moves logp by u / 2 of |logp| + R.  In all
    E = 2^-18 + u (2 R + chain)
covers the relative error of a row's sum and the absolute one of logp (a power counted 2^-22, 11 of them below 2^-18).
  logp        E + u |logp|
  token_loss  its slope's magnitude times E, u of itself:  w (|A| r + kl |e^d - 1|) E (1 + E)
  dlogits     s = scale dl/dlogp / T:  ds = scale w (|A| r + kl e^d) E / T;  ds (1[t] + p) + |s| p (2 E + 2^-22 + u R) + 3 u |s| 1[t], half a step
A power below 2^-126 of its row's largest, the least normal number, counts as 0: p is then off by at most 2^-126 (the largest has a p of at
least 1 / n, and p = power / sum with sum >= 1), so dlogits by |s| 2^-126 more.
Ratios are set away from the borders of the clip, as both sides of a border are right next to it."""

from __future__ import annotations

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
LO, HI = 0.2, 0.3


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _case(n, v, kind, warm, seed, stride=None, lead=0, forbid=0.0, spread=3.0, bits=64):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    stride = stride or v
    flat = torch.full((lead + n * stride + 16,), 55.0, dtype=_dt(kind), device="cuda")
    z = flat[lead:lead + n * stride].view(n, stride)[:, :v]
    x = torch.randn(n, v, generator=gen, device="cuda") * spread
    t = torch.randint(0, v, (n,), generator=gen, device="cuda")
    if forbid:
        x = x.masked_fill(torch.rand(n, v, generator=gen, device="cuda") < forbid, -math.inf)
        x[torch.arange(n, device="cuda"), t] = 0.5
    z.copy_(x)
    logp = torch.log_softmax(z.double() / warm, 1).gather(1, t[:, None])[:, 0]
    far = torch.tensor([-0.9, -0.5, -0.1, 0.0, 0.1, 0.15, 0.5, 1.0], device="cuda", dtype=torch.float64)
    pick = far[torch.randint(0, 8, (n,), generator=gen, device="cuda")]
    c = {"n": n, "v": v, "kind": kind, "warm": warm, "z": z, "flat": flat, "stride": stride, "lead": lead, "bits": bits}
    c["t"] = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.1, torch.randint(0, 2, (n,), generator=gen, device="cuda") * (v + 1) - 1, t)   # -1 or v
    c["t"] = c["t"].to(torch.int32 if bits == 32 else torch.int64)
    c["old"] = (logp - pick).float()
    c["ref"] = (logp + 0.5 * torch.randn(n, generator=gen, device="cuda")).float()
    c["adv"] = torch.randn(n, generator=gen, device="cuda")
    c["w"] = torch.rand(n, generator=gen, device="cuda") * (torch.rand(n, generator=gen, device="cuda") < 0.9)
    c["up"] = torch.tensor([3.0], device="cuda")
    return c


def _formula(c, kl, use_ref=True, use_w=True, use_up=True):
    import torch
    n, v, warm = c["n"], c["v"], c["warm"]
    z = c["z"].double() / warm
    t = c["t"].long()
    w = c["w"].double() if use_w else torch.ones(n, dtype=torch.float64, device="cuda")
    live = (t >= 0) & (t < v) & (w != 0)
    at = t.clamp(0, v - 1)
    logp = z.gather(1, at[:, None])[:, 0] - torch.logsumexp(z, 1)
    r = torch.exp(logp - c["old"].double())
    a = c["adv"].double()
    one, two = r * a, r.clamp(1 - LO, 1 + HI) * a
    loss, dl, size = -torch.minimum(one, two), torch.where(one <= two, -one, torch.zeros_like(one)), one.abs()
    if use_ref:
        d = c["ref"].double() - logp
        loss = loss + kl * (torch.expm1(d) - d)
        dl = dl - kl * torch.expm1(d)
        size = size + kl * (torch.exp(d) + 1)
    zero = torch.zeros_like(loss)
    loss, dl, size, logp = (torch.where(live, x, zero) for x in (w * loss, w * dl, w * size, logp))
    up = float(c["up"]) if use_up else 1.0
    p = torch.softmax(z, 1)
    s = up * dl / warm
    hot = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    dz = torch.where(live[:, None], s[:, None] * (hot - p), torch.zeros_like(p))
    fin = torch.isfinite(z)
    spread = torch.where(fin, z, -math.inf).amax(1) - torch.where(fin, z, math.inf).amin(1)
    R = spread * 1.4427
    E = 2.0 ** -18 + U * (2 * R + v / (32 if v <= 1024 else 128 if v <= 8192 else 512) + 16)
    tol_logp = E + U * logp.abs()
    tol_loss = size * E * (1 + E) + 2 * U * loss.abs()
    ds = up * size * E / warm
    tol_dz = ds[:, None] * (hot + p) + s.abs()[:, None] * (p * (2 * E + 2.0 ** -22 + U * R)[:, None] + 3 * U * hot + 2.0 ** -126)
    tol_dz = tol_dz + HALF[c["kind"]] * (dz.abs() + tol_dz) + TINY[c["kind"]]
    return live, (loss, logp, dz), (tol_loss, torch.where(live, tol_logp, zero), torch.where(live[:, None], tol_dz, torch.zeros_like(dz)))


def _run(c, kl, use_ref=True, use_w=True, use_up=True, grad=True, in_place=False, out_stride=None, out_lead=None, stream=None):
    import torch
    import paper_2307_11617_b200 as pkg
    n, v = c["n"], c["v"]
    small = torch.full((2 * n + 1,), 9.0, device="cuda")
    out_stride = c["stride"] if in_place else out_stride or c["stride"]
    out_lead = c["lead"] if out_lead is None else out_lead
    flat = c["flat"] if in_place else torch.full((out_lead + n * out_stride + 16,), 55.0, dtype=_dt(c["kind"]), device="cuda")
    dz = flat[out_lead:out_lead + n * out_stride].view(n, out_stride)[:, :v]
    pkg.rfast_policy_loss(c["z"].data_ptr(), c["t"].data_ptr(), c["old"].data_ptr(), c["adv"].data_ptr(), n, v, d_loss=small[2 * n:].data_ptr(), d_token_loss=small.data_ptr(),
                          d_logp=small[n:].data_ptr(), d_dlogits=dz.data_ptr() if grad else 0, d_ref_logp=c["ref"].data_ptr() if use_ref else 0,
                          d_weight=c["w"].data_ptr() if use_w else 0, d_loss_scale=c["up"].data_ptr() if use_up else 0, temperature=c["warm"], clip_low=LO,
                          clip_high=HI, kl_coef=kl, type=c["kind"], token_bits=c["bits"], logits_stride=c["stride"], dlogits_stride=out_stride,
                          cuda_stream=torch.cuda.current_stream().cuda_stream if stream is None else stream)
    return small[2 * n], small[:n], small[n:2 * n], dz, flat


def _check(c, got, kl, grad=True, **kw):
    import torch
    live, want, tol = _formula(c, kl, **kw)
    total, loss, logp, dz, flat = got
    for name, g, x, e in (("loss", loss, want[0], tol[0]), ("logp", logp, want[1], tol[1])) + ((("dz", dz, want[2], tol[2]),) if grad else ()):
        bad = ~((g.double() - x).abs() <= e)
        assert not bad.any(), (name, int(bad.sum()), bad.nonzero()[:3].tolist(), (g.double() - x).abs().max().item())
    assert abs(float(total) - float(loss.double().sum())) <= U * abs(float(loss.double().sum())) + 1e-12
    if grad:
        assert bool((dz[~live] == 0).all())


SHAPES = [(1, 1), (1, 2), (5, 3), (9, 31), (17, 32), (8, 257), (64, 1000), (3, 1024), (3, 1025), (7, 2049), (11, 8191), (6, 8192), (5, 8193), (5, 32000), (3, 50257),
          (2, 131071), (4, 100_000), (700, 9001), (320, 50001), (2, 350_003), (1, 800_001)]


@pytest.mark.parametrize("n,v", SHAPES)
@pytest.mark.parametrize("kind,warm,pad,lead,bits", [("f32", 1.0, 0, 0, 64), ("bf16", 0.7, 8, 0, 32), ("f16", 1.0, 0, 3, 64), ("bf16", 2.0, 5, 1, 64), ("f32", 0.5, 1, 1, 32)])
def test_against_the_formula(n, v, kind, warm, pad, lead, bits):
    import torch
    c = _case(n, v, kind, warm, n * 31 + v, stride=v + pad, lead=lead, bits=bits)
    before = c["flat"].clone()
    got = _run(c, 0.1)
    _check(c, got, 0.1)
    assert torch.equal(before, c["flat"])
    keep = torch.ones_like(got[4], dtype=torch.bool)
    keep[lead:lead + n * (v + pad)].view(n, v + pad)[:, :v] = False
    assert bool((got[4][keep].double() == 55.0).all())
    # gradients that lie otherwise within eight values
    _check(c, _run(c, 0.1, out_stride=v + pad + 3, out_lead=lead + 1), 0.1)
    # without a gradient
    for a, b in zip(got[:3], _run(c, 0.1, grad=False)[:3]):
        assert torch.equal(a, b)
    # in the place of the logits
    for a, b in zip(got[:4], _run(c, 0.1, in_place=True)[:4]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("use_ref", [False, True])
@pytest.mark.parametrize("use_w", [False, True])
@pytest.mark.parametrize("use_up", [False, True])
def test_operands_left_out(use_ref, use_w, use_up):
    kw = dict(use_ref=use_ref, use_w=use_w, use_up=use_up)
    c = _case(40, 5003, "f32", 1.0, 5)
    _check(c, _run(c, 0.2, **kw), 0.2, **kw)


@pytest.mark.parametrize("v", [700, 9001])
def test_forbidden_words_and_rows_of_no_weight(v):
    import torch
    c = _case(30, v, "bf16", 1.0, 8, forbid=0.7)
    c["w"][3] = 0.0
    c["z"][3] = math.nan                                     # rows that do not count are not read
    c["t"][4] = -1
    c["z"][4] = math.inf
    c["old"][4] = c["adv"][4] = c["ref"][3] = math.nan
    got = _run(c, 0.1)
    c["z"][3:5] = 0.0
    c["old"][4] = c["adv"][4] = c["ref"][3] = 0.0
    _check(c, got, 0.1)
    assert bool((got[3][c["z"] == -math.inf] == 0).all())


@pytest.mark.parametrize("v", [50, 4099])
def test_what_is_not_finite_stays_in_its_row(v):
    import torch
    c = _case(12, v, "f32", 1.0, 4)
    c["w"].fill_(1.0)
    c["t"].copy_(torch.arange(12) % v)
    c["old"].fill_(-3.0)
    c["ref"].fill_(-3.0)
    c["z"][2] = -math.inf
    c["z"][5, 7] = math.nan
    c["z"][7, 9] = math.inf
    total, loss, logp, dz, _ = _run(c, 0.1)
    for r in range(12):
        bad = r in (2, 5, 7)
        assert math.isnan(float(loss[r])) == bad and math.isnan(float(logp[r])) == bad and bool(torch.isnan(dz[r]).all()) == bad, r
        assert bad or bool(torch.isfinite(dz[r]).all())
    assert math.isnan(float(total))


@pytest.mark.parametrize("v", [1500, 30_011])
def test_logits_far_from_zero(v):
    """Large offsets, a peaked row, a wide one: sums are relative to the largest logit."""
    import torch
    c = _case(6, v, "f32", 1.0, 6)
    c["z"][0] += 1e4
    c["z"][1] -= 1e4
    c["z"][2, 5] = 80.0
    c["z"][3] *= 30.0
    c["z"][4] = 2.0
    c["w"].fill_(1.0)
    c["t"].copy_(torch.tensor([1, 2, 5, 6, 7, 8]))
    logp = torch.log_softmax(c["z"].double(), 1).gather(1, c["t"].long()[:, None])[:, 0]
    c["old"], c["ref"] = (logp - 0.1).float(), (logp + 0.2).float()
    # old and ref are rounded to fp32; that is part of the inputs, not of the error
    _check(c, _run(c, 0.1), 0.1)


def test_gradient_against_differences():
    import torch
    c = _case(8, 301, "f32", 0.9, 12)
    c["w"].fill_(0.5)
    c["t"].copy_(torch.arange(8))
    logp = torch.log_softmax(c["z"].double() / 0.9, 1).gather(1, c["t"][:, None])[:, 0]
    c["old"] = (logp - torch.tensor([-0.9, -0.1, 0.0, 0.1, 0.15, 0.6, 1.0, 0.05], device="cuda")).float()
    c["ref"] = (logp + 0.3).float()
    dz = _run(c, 0.3, use_up=False)[3].double()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    e = torch.randn(8, 301, generator=gen, device="cuda", dtype=torch.float64)
    h = 1e-5
    z = c["z"].double()
    side = []
    for s in (h, -h):
        d = dict(c, z=z + s * e)
        side.append(_formula(d, 0.3, use_up=False)[1][0])
    slope = (side[0] - side[1]) / (2 * h)
    # the difference is off by h^2 / 6 of the third derivative (below 10 |e|^3 here) and 1e-16 / h of the loss
    assert ((dz * e).sum(1) - slope).abs().max() <= 1e-6 + 1e-5 * slope.abs().max()


def test_recorded_into_a_graph_with_two_streams():
    import torch
    cs = [_case(20, 6001, "bf16", 1.0, 21), _case(300, 800, "f32", 1.0, 22)]
    for c in cs:
        _run(c, 0.1)
    torch.cuda.synchronize()
    held = []
    for c in cs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = _run(c, 0.1)
        held.append((g, out, torch.cuda.Stream()))
    for rep in range(2):
        for c in cs:
            c["z"].copy_(_case(c["n"], c["v"], c["kind"], 1.0, 30 + rep)["z"])
            logp = torch.log_softmax(c["z"].double(), 1).gather(1, c["t"].long().clamp(0, c["v"] - 1)[:, None])[:, 0]
            c["old"].copy_(logp - 0.1)
        torch.cuda.synchronize()
        for g, _, s in held:
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for c, (_, out, _) in zip(cs, held):
            _check(c, out, 0.1)


def test_no_rows():
    import torch
    import paper_2307_11617_b200 as pkg
    loss = torch.full((1,), 4.0, device="cuda")
    pkg.rfast_policy_loss(0, 0, 0, 0, 0, 50, d_loss=loss.data_ptr(), d_token_loss=loss.data_ptr(), cuda_stream=torch.cuda.current_stream().cuda_stream)
    assert float(loss) == 0.0


def test_offsets_beyond_32_bits():
    """Logits of 2.3e9 values: the last rows lie beyond 2^31 values and 2^32 bytes."""
    import torch
    import paper_2307_11617_b200 as pkg
    n, v, k = 18_000, 128_256, 4
    z = torch.zeros(n, v, dtype=torch.bfloat16, device="cuda")
    c = _case(k, v, "bf16", 1.0, 40)
    z[-k:] = c["z"]
    t = torch.full((n,), -1, dtype=torch.int64, device="cuda")
    t[-k:] = c["t"]
    dz = torch.full((n, v), 3.0, dtype=torch.bfloat16, device="cuda")
    full = {}
    for name in ("old", "ref", "adv", "w"):
        full[name] = torch.full((n,), math.nan, device="cuda")
        full[name][-k:] = c[name]
    small = torch.empty(2 * n + 1, device="cuda")
    pkg.rfast_policy_loss(z.data_ptr(), t.data_ptr(), full["old"].data_ptr(), full["adv"].data_ptr(), n, v, d_loss=small[2 * n:].data_ptr(), d_token_loss=small.data_ptr(),
                          d_logp=small[n:].data_ptr(), d_dlogits=dz.data_ptr(), d_ref_logp=full["ref"].data_ptr(), d_weight=full["w"].data_ptr(), d_loss_scale=c["up"].data_ptr(),
                          clip_low=LO, clip_high=HI, kl_coef=0.1, type="bf16", cuda_stream=torch.cuda.current_stream().cuda_stream)
    _check(c, (small[2 * n], small[n - k:n], small[2 * n - k:2 * n], dz[-k:], None), 0.1)
    assert bool((dz[:-k] == 0).all()) and bool((small[:n - k] == 0).all())


@pytest.mark.parametrize("v", [300, 3001, 20_001, 90_000])
def test_single_results(v):
    """Each result alone is what it is among the others."""
    import torch
    import paper_2307_11617_b200 as pkg
    c = _case(9, v, "f16", 1.0, v)
    got = _run(c, 0.1)
    for which in ("d_token_loss", "d_logp", "d_dlogits"):
        out = torch.full_like(got[3], 7.0) if which == "d_dlogits" else torch.full((9,), 7.0, device="cuda")
        pkg.rfast_policy_loss(c["z"].data_ptr(), c["t"].data_ptr(), c["old"].data_ptr(), c["adv"].data_ptr(), 9, v, d_ref_logp=c["ref"].data_ptr(), d_weight=c["w"].data_ptr(),
                              d_loss_scale=c["up"].data_ptr(), clip_low=LO, clip_high=HI, kl_coef=0.1, type="f16", cuda_stream=torch.cuda.current_stream().cuda_stream,
                              **{which: out.data_ptr()})
        assert torch.equal(out, got[{"d_token_loss": 1, "d_logp": 2, "d_dlogits": 3}[which]]), which


def test_logits_of_one_row_for_all():
    """A stride of 0: many tokens scored by the same logits."""
    import torch
    for v in (700, 40_001):
        c = _case(1, v, "f32", 1.0, 50)
        n = 30
        one = dict(c, n=n, stride=v, z=c["z"].expand(n, v), t=torch.arange(n, device="cuda"), adv=torch.ones(n, device="cuda"), w=torch.ones(n, device="cuda"))
        logp = torch.log_softmax(c["z"].double(), 1)[0, :n]
        one["old"], one["ref"] = (logp - 0.1).float(), (logp + 0.2).float()
        import paper_2307_11617_b200 as pkg
        small = torch.empty(2 * n + 1, device="cuda")
        dz = torch.empty(n, v, device="cuda")
        pkg.rfast_policy_loss(c["z"].data_ptr(), one["t"].data_ptr(), one["old"].data_ptr(), one["adv"].data_ptr(), n, v, d_loss=small[2 * n:].data_ptr(),
                              d_token_loss=small.data_ptr(), d_logp=small[n:].data_ptr(), d_dlogits=dz.data_ptr(), d_ref_logp=one["ref"].data_ptr(), d_weight=one["w"].data_ptr(),
                              d_loss_scale=c["up"].data_ptr(), clip_low=LO, clip_high=HI, kl_coef=0.1, logits_stride=0,
                              cuda_stream=torch.cuda.current_stream().cuda_stream)
        _check(one, (small[2 * n], small[:n], small[n:2 * n], dz, None), 0.1)


def test_more_rows_than_a_grid_has_groups_of_blocks():
    """2^29 + 1 rows of one long row of zeros: eight blocks to a row would be more than a launch takes.  Three rows count."""
    import torch
    import paper_2307_11617_b200 as pkg
    n, v = (1 << 29) + 1, 600_000
    z = torch.zeros(v, device="cuda")
    t = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    old, adv = torch.full((n,), -math.log(v), device="cuda"), torch.ones(n, device="cuda")
    loss = torch.full((n,), 3.0, device="cuda")
    rows = [0, n // 2, n - 1]
    for k in rows:
        t[k] = k % v
    pkg.rfast_policy_loss(z.data_ptr(), t.data_ptr(), old.data_ptr(), adv.data_ptr(), n, v, d_token_loss=loss.data_ptr(), logits_stride=0, token_bits=32,
                          cuda_stream=torch.cuda.current_stream().cuda_stream)
    # the sum of v powers of zero is exact; old_logp, 13.3, is rounded by at most 2^-21, the ratio next to 1 moves by as much; then the result's 2^-24
    for k in rows:
        assert abs(float(loss[k]) + 1.0) < 2.0 ** -21 + 2.0 ** -23, k
        loss[k] = 0.0
    assert not bool(loss.any())


@pytest.mark.parametrize("v", [64, 5000, 70_000])
def test_a_token_that_may_not_be_used(v):
    """Its own logit is -infinity: logp = -infinity, a ratio of 0, no gradient; NaN where a KL term asks for more."""
    import torch
    c = _case(6, v, "f32", 1.0, 61)
    c["w"].fill_(1.0)
    c["t"].copy_(torch.arange(6))
    c["z"][2, 2] = -math.inf
    c["old"].fill_(-4.0)
    c["ref"].fill_(-4.0)
    c["adv"].fill_(1.0)
    total, loss, logp, dz, _ = _run(c, 0.0, use_ref=False)
    assert float(logp[2]) == -math.inf and float(loss[2]) == 0.0 and bool((dz[2] == 0).all()) and bool(torch.isfinite(total))
    total, loss, logp, dz, _ = _run(c, 0.1)
    assert math.isnan(float(loss[2])) and bool(torch.isfinite(loss[[0, 1, 3, 4, 5]]).all()) and bool(torch.isfinite(dz[[0, 1, 3, 4, 5]]).all())
