"""Policy loss: words that are masked by a large negative logit in the place of -infinity, down to the lowest value of the type, in front, behind and
all over a row; rows that nothing but such logits fill; rows far from zero.  What is masked is e^-100000 of the rest or less, so the formula is the one with -infinity;
where all logits of a row are one value the distribution is even.  Tolerances are those of test_gpu_policy_loss_rows, the spread taken of what is not masked."""

from __future__ import annotations

import math

import pytest

from test_gpu_policy_loss import _case, _dt, _formula, _run
from test_gpu_policy_loss_rows import _within

pytestmark = pytest.mark.gpu


def _masked(n, v, kind, warm, how, mask, seed):
    import torch
    c = _case(n, v, kind, warm, seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    t = c["t"].long().clamp(0, v - 1)[:, None]
    at = torch.arange(v, device="cuda")[None, :].expand(n, v)
    if how == "front":                                       # what a thread reads first, of every thread
        off = at < (v * 3) // 4
    elif how == "behind":
        off = at >= v // 4
    else:
        off = torch.rand(n, v, generator=gen, device="cuda") < 0.97
    off = off & (at != t)
    z = torch.where(off, torch.full((), mask, dtype=torch.float32, device="cuda"), c["z"].float())
    c["z"].copy_(z)
    logp = torch.log_softmax(c["z"].double().masked_fill(off, -math.inf) / warm, 1).gather(1, t)[:, 0]
    c["old"] = (logp + 0.1 * torch.randn(n, generator=gen, device="cuda").clamp(-0.5, 0.5)).float()
    c["ref"] = (logp + 0.2).float()
    return c, off


def _lowest(kind):
    import torch
    return torch.finfo(_dt(kind)).min


@pytest.mark.parametrize("kind,mask", [("f32", -1e6), ("f32", -1e10), ("f32", -3.3e12), ("f32", -1.7e30), ("f32", "lowest"), ("bf16", -1e10), ("bf16", -1e30), ("bf16", "lowest"),
                                       ("f16", "lowest")])
@pytest.mark.parametrize("warm", [0.7, 1.0, 2.5])
@pytest.mark.parametrize("v", [40, 1000, 6001, 33_000, 90_003])
def test_masked_by_a_large_number(kind, mask, warm, v):
    import torch
    mask = _lowest(kind) if mask == "lowest" else mask
    for how in ("front", "behind", "most"):
        c, off = _masked(12, v, kind, warm, how, mask, v)
        plain = dict(c, z=c["z"].float().masked_fill(off, -math.inf))
        got = _run(c, 0.1)
        _within(plain, got, 0.1)
        assert not bool(got[3][off].any()), how
        live = _formula(plain, 0.1)[0]
        assert bool(torch.isfinite(got[1]).all()) and bool(torch.isfinite(got[0])) and bool((got[2][live] > -100).all())
        # a gradient that lies otherwise
        other = _run(c, 0.1, out_stride=v + 3, out_lead=1)
        _within(plain, other, 0.1, align=False)
        assert not bool(other[3][off].any()), how
        # in the place of the logits
        for x, y in zip(got[:4], _run(c, 0.1, in_place=True)[:4]):
            assert torch.equal(x, y)


@pytest.mark.parametrize("kind,value", [("f32", -1e10), ("f32", -1.7e30), ("f32", "lowest"), ("f32", 2.9e33), ("f32", 1e9), ("bf16", -1e30), ("bf16", "lowest"), ("f16", "lowest")])
@pytest.mark.parametrize("warm", [0.7, 1.0, 2.5])
@pytest.mark.parametrize("v", [40, 1000, 6001, 90_003])
def test_rows_of_one_value(kind, value, warm, v):
    """The distribution is even, whatever the value is: that of a row of zeros."""
    import torch
    value = _lowest(kind) if value == "lowest" else value
    c = _case(4, v, kind, warm, v)
    c["z"].fill_(value)
    c["t"].copy_(torch.tensor([0, v // 2, v - 1, 3]))
    c["w"].fill_(1.0)
    c["old"].fill_(-math.log(v) + 0.05)
    c["ref"].fill_(-math.log(v) - 0.1)
    plain = dict(c, z=torch.zeros_like(c["z"]))
    got = _run(c, 0.1)
    _within(plain, got, 0.1)
    _within(plain, _run(c, 0.1, out_stride=v + 3, out_lead=1), 0.1, align=False)
    for x, y in zip(got[:3], _run(c, 0.1, grad=False)[:3]):
        assert torch.equal(x, y)
    for x, y in zip(got[:4], _run(c, 0.1, in_place=True)[:4]):
        assert torch.equal(x, y)


@pytest.mark.parametrize("base", [1e10, -1e10, 1e37, -1e37])
@pytest.mark.parametrize("v", [600, 5000, 60_000])
def test_two_values_far_from_zero(base, v):
    """Eight logits of one value, the others next to it, hundreds and more below: their distribution is even, and the others' is nothing."""
    import torch
    c = _case(3, v, "f32", 1.0, 9)
    c["z"].fill_(torch.nextafter(torch.tensor(base), torch.tensor(-3e38)).item())
    c["z"][:, 100:108] = base
    c["t"].copy_(torch.tensor([100, 105, 107]))
    c["w"].fill_(1.0)
    c["old"].fill_(-2.0)
    c["ref"].fill_(-2.2)
    plain = dict(c, z=torch.where(c["z"] == base, 0.0, -math.inf))
    got = _run(c, 0.1)
    _within(plain, got, 0.1)
    assert not bool(got[3][:, :100].any()) and not bool(got[3][:, 108:].any())


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("warm", [0.7, 1.0, 1.3])
@pytest.mark.parametrize("v", [64, 3000, 50_001])
def test_no_log_probability_is_above_zero(kind, warm, v):
    """Words that have all, or nearly all, of a row: their powers are off either way, their log probabilities are not above that of certainty."""
    import torch
    n = 200
    c = _case(n, v, kind, warm, v)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(v)
    c["t"].copy_(torch.randint(0, v, (n,), generator=gen, device="cuda"))
    c["w"].fill_(1.0)
    top = 40.0 + 20.0 * torch.rand(n, 1, generator=gen, device="cuda")
    c["z"].scatter_(1, c["t"].long()[:, None], top.to(c["z"].dtype))
    logp = torch.log_softmax(c["z"].double() / warm, 1).gather(1, c["t"].long()[:, None])[:, 0]
    c["old"], c["ref"] = (logp - 0.1).float(), (logp + 0.1).float()
    got = _run(c, 0.1)
    assert bool((got[2] <= 0).all())
    _within(c, got, 0.1)
