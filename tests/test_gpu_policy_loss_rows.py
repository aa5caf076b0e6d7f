"""Policy loss: rows at the borders between the ways that rows are done, single rows, log probabilities by themselves.

What the sums of a row are off by, u = 2^-24, R = log2(e) / T times the spread of the row's logits:
  * a power of two is off by 2^-22 of itself (what the instruction promises), its exponent, of at most R + 40 either way (the reference may lie
    2^40 below the maximum), by u of that and u of little more (it is formed in two steps), which is ln 2 u (2 (R + 40) + 1) of the power;
  * a sum is taken to another reference at most R / 40 + 1 times while a thread reads and once at each of three merges (2^-22 for the factor, u for
    the product);
  * a thread adds up its logits one after the other, and at most 15 additions merge the threads' sums (a warp's, a block's, a cluster's): u each.
    A row of up to 1024 logits is a warp's, one of up to 40 KB 128 threads', one of up to 128 KB 256 threads' where its gradient lies as it does,
    512 threads' elsewhere; a thread takes groups of eight and one value beside them.
    E = 2^-22 (5 + R / 40) + u (ln 2 (2 (R + 40) + 1) + chain + 15 + 4 + R / 40)
is the relative error of a sum and the absolute one of logp.  The results' tolerances follow:
  logp        E, and u |logp| for its rounding
  token_loss  w (|A| r + kl (e^d + 1)) E (1 + E) and 2 u of itself
  dlogits     s = scale dl/dlogp / T, p = softmax:  scale w (|A| r + kl (e^d + 1)) E / T (1[t] + p) + |s| p (2 E + 2^-21 + u ln 2 (2 R + 40) + 3 u) + 3 u |s| 1[t]
              (log2(e) / T is rounded to fp32 here, u ln 2 R; two powers),
              2^-126 |s| (a power below counts as 0), half a step of the type."""

from __future__ import annotations

import math

import pytest

from test_gpu_policy_loss import HALF, HI, LO, TINY, U, _case, _formula, _run

pytestmark = pytest.mark.gpu

LN2 = math.log(2.0)
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _chain(v, kind, align):
    size = v * BYTES[kind]
    team = 32 if v <= 1024 else 128 if size <= 40 * 1024 else 256 if align and size <= 128 * 1024 else 512
    return 8 * -(-(v // 8) // team) + 1


def _sums(c, align):
    """Of every row: R, E and the exact logp."""
    import torch
    z = c["z"].double() / c["warm"]
    t = c["t"].long().clamp(0, c["v"] - 1)[:, None]
    R = (z.amax(1) - torch.where(torch.isfinite(z), z, math.inf).amin(1)) / LN2
    E = 2.0 ** -22 * (5 + R / 40) + U * (LN2 * (2 * (R + 40) + 1) + _chain(c["v"], c["kind"], align) + 19 + R / 40)
    return R, E, z.gather(1, t)[:, 0] - torch.logsumexp(z, 1)


def _within(c, got, kl, align=True):
    import torch
    live, (loss0, logp0, dz0), _ = _formula(c, kl)
    _, loss, logp, dz, _ = got
    R, E, lp = _sums(c, align)
    size = c["w"].double() * (c["adv"].double().abs() * torch.exp(lp - c["old"].double()) + kl * (torch.exp(c["ref"].double() - lp) + 1))
    p = torch.softmax(c["z"].double() / c["warm"], 1)
    hot = torch.zeros_like(p).scatter_(1, c["t"].long().clamp(0, c["v"] - 1)[:, None], 1.0)
    # |s|, out of the formula's gradient: dz = s (1[t] - p)
    s = dz0.abs().sum(1) / (hot - p).abs().sum(1).clamp_min(1e-300)
    tol = (float(c["up"]) * size * E / c["warm"])[:, None] * (hot + p) + s[:, None] * (p * (2 * E + 2.0 ** -21 + U * (LN2 * (2 * R + 40) + 3))[:, None] + 3 * U * hot + 2.0 ** -126)
    tol = tol + HALF[c["kind"]] * (dz0.abs() + tol) + TINY[c["kind"]]
    for name, g, x, e in (("logp", logp, logp0, E + U * logp0.abs()), ("loss", loss, loss0, size * E * (1 + E) + 2 * U * loss0.abs()), ("dz", dz, dz0, tol)):
        off = (g.double() - x).abs()[live] / e[live]
        assert bool((off <= 1).all()), (name, int((off > 1).sum()), float(off.max()))
        assert not bool(g[~live].any()), name


BORDERS = [("f32", v) for v in (1023, 1024, 1025, 10_240, 10_241, 32_768, 32_769)] + [(k, v) for k in ("bf16", "f16") for v in (1024, 1025, 20_480, 20_481, 65_536, 65_537)]


@pytest.mark.parametrize("kind,v", BORDERS)
@pytest.mark.parametrize("n", [5, 400])
def test_rows_at_the_borders_of_their_teams(kind, v, n):
    """Few rows (shared out over clusters where they are long) and many, gradients that lie as the logits do and otherwise."""
    c = _case(n, v, kind, 0.8, v + n)
    _within(c, _run(c, 0.1), 0.1)
    _within(c, _run(c, 0.1, out_stride=v + 3, out_lead=1), 0.1, align=False)


@pytest.mark.parametrize("kind,v,stride", [("f32", 10_300, 10_301), ("f32", 50_257, 50_304), ("bf16", 50_257, 50_304), ("bf16", 128_256, 128_259), ("f16", 30_001, 30_007), ("f32", 700, 701)])
def test_one_row_has_no_stride(kind, v, stride):
    """What a row would be away from the next one does not matter where there is one: the same results, bit for bit, whatever the strides say."""
    import torch
    c = _case(1, v, kind, 1.0, v, stride=stride)
    c["w"].fill_(0.7)
    c["t"].fill_(v // 3)
    want = _run(c, 0.1, out_stride=stride)
    for out_stride in (v, v + 5, 0):
        got = _run(c, 0.1, out_stride=max(out_stride, v)) if out_stride else _run(dict(c, stride=0), 0.1, out_stride=v)
        for a, b in zip(got[:4], want[:4]):
            assert torch.equal(a.reshape(-1), b.reshape(-1)), out_stride
    _within(c, want, 0.1)


@pytest.mark.parametrize("n,v,kind,bits", [(1, 1, "f32", 64), (7, 1000, "bf16", 32), (30, 5003, "f32", 64), (9, 50_257, "f16", 64), (3, 400_000, "f32", 32)])
def test_log_probabilities_by_themselves(n, v, kind, bits):
    """They need no policy to compare with and no advantage; the bits are those of a call that has them."""
    import torch
    import paper_2307_11617_b200 as pkg
    c = _case(n, v, kind, 0.7, n + v, bits=bits)
    want = _run(c, 0.1)[2]
    for w in (c["w"].data_ptr(), 0):
        out = torch.full((n,), 7.0, device="cuda")
        pkg.rfast_policy_loss(c["z"].data_ptr(), c["t"].data_ptr(), 0, 0, n, v, d_logp=out.data_ptr(), d_weight=w, temperature=0.7, type=kind, token_bits=bits,
                              cuda_stream=torch.cuda.current_stream().cuda_stream)
        if w:
            assert torch.equal(out, want)
            continue
        on = (c["t"].long() >= 0) & (c["t"].long() < v)      # rows without a weight count as well
        _, bound, logp = _sums(c, True)
        assert torch.equal(out[c["w"] != 0], want[c["w"] != 0]) and not bool(out[~on].any())
        assert bool(((out.double() - logp).abs() <= bound + U * logp.abs())[on].all())


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("k", [1 + 2.0 ** -24, 1.0, 2 - 2.0 ** -24, 1.25 + 3 * 2.0 ** -25, math.log2(math.e), math.log2(math.e) / 0.7])
@pytest.mark.parametrize("v", [50, 5000, 70_001])
def test_the_temperature_is_the_one_that_was_given(kind, k, v):
    """Rows of zeros but for the token, far below: the powers of zero are 1 and their sum is exact, so that the ratio, in 64 bits, shows T alone
    (log2(e) / T in fp32 would be up to 2^-24 of 60 / T off).  Tolerance: the rounding of the loss; of the gradients, two more roundings."""
    import torch
    warm = math.log2(math.e) / k
    n = 4
    c = _case(n, v, kind, warm, v)
    c["z"].zero_()
    c["t"].copy_(torch.tensor([0, 7, v // 2, v - 1]))
    c["z"][torch.arange(n), c["t"].long()] = torch.tensor([-60.0, -50.0, -61.5, -48.0], device="cuda").to(c["z"].dtype)
    c["w"].fill_(1.0)
    c["adv"].fill_(1.0)
    zt = c["z"].double().gather(1, c["t"].long()[:, None])[:, 0] / warm
    logp = zt - math.log(v - 1)                              # and e^-48 or less of a word
    c["old"] = logp.float()
    total, loss, got, dz, _ = _run(c, 0.0, use_ref=False, use_up=False)
    ratio = torch.exp(logp - c["old"].double())
    assert bool(((loss.double() + ratio).abs() <= (U + 2.0 ** -33) * ratio).all()), (loss.double() + ratio).abs().max().item()
    assert bool(((got.double() - logp).abs() <= (U + 2.0 ** -40) * logp.abs()).all())
    want = (ratio / (v - 1) / warm)[:, None].expand(n, v).clone()
    want.scatter_(1, c["t"].long()[:, None], -(ratio / warm)[:, None])
    assert bool(((dz.double() - want).abs() <= (HALF[kind] + 4 * U) * want.abs() + TINY[kind]).all())
