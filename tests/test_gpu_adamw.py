"""Gradient norm and AdamW step over many tensors against a plain 64-bit restatement.

u = 2^-24 is half a step of fp32.  The tolerances count the roundings of the kernel's expression, in which the factors that
do not change from value to value are multiplied together first:
  m   g1 = scale (1 - beta1): 2 u; g1 g + beta1 m: the constant, its product and the sum: at most 5 u of
      |beta1 m| + |(1 - beta1) g'|
  v   (a sum of positive terms) h = (scale sqrt(1 - beta2)) g: constant, product, product, 3 u; its square 7 u; the sum 8 u
  p   quotient q = step m / (r root + eps): r is off by half of v's 8 u and the root's 1 ulp = 2 u, 6 u; root, eps, their
      sum 9 u; the reciprocal's 1 ulp = 2 u and its product 12 u; step and the sum 14 u, in all at most 16 u of q plus m's
      error carried along; the decay's constant, its product and the sum: 3 u of p; then half a step of p's type
  8-bit moments: half a step of the code (2^-4 of the value, 2^-10 of the scale below 2^-6 scales),
      plus the error of the value before it and 3 u of the scale's and the quotient's roundings"""

from __future__ import annotations

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}     # half a step relative to the value, at worst
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
LR, B1, B2, EPS, WD = 1e-2, 0.9, 0.99, 1e-8, 0.05


def _torch():
    import torch
    return torch, {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _values8(code, scale, numel):
    """What 8-bit codes stand for, in 64 bits, straight from the format's definition."""
    c = code.astype(np.int64)
    e, f = (c >> 3) & 15, c & 7
    mag = np.where(e == 0, f / 8.0 * 2.0 ** -6, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    mag = np.where((e == 15) & (f == 7), np.nan, mag)
    return np.where(c & 128, -mag, mag) * np.repeat(scale.astype(np.float64), 256)[:numel]


class _Buf:
    """Tensors at chosen element offsets of one allocation, canaries in between."""

    def __init__(self, values, dtype, lead):
        torch, _ = _torch()
        self.numel = [len(v) for v in values]
        self.lead = lead
        at, self.at = lead, []
        for n in self.numel:
            self.at.append(at)
            at += (n + 15) // 16 * 16 + 16
        fill = 77 if dtype == torch.uint8 else 77.0
        self.t = torch.full((at + 16,), fill, dtype=dtype, device="cuda")
        for v, a in zip(values, self.at):
            if len(v):
                self.t[a:a + len(v)] = torch.as_tensor(np.ascontiguousarray(v)).to(dtype).cuda()

    def addresses(self):
        return [self.t.data_ptr() + a * self.t.element_size() for a in self.at]

    def get(self, k):
        import torch
        x = self.t[self.at[k]:self.at[k] + self.numel[k]]
        return (x if x.dtype == torch.uint8 else x.double()).cpu().numpy()

    def canaries_stand(self):
        import torch
        keep = torch.ones_like(self.t, dtype=torch.bool)
        for a, n in zip(self.at, self.numel):
            keep[a:a + n] = False
        return bool((self.t[keep].double() == 77.0).all())


SIZES = {
    "one": [1],
    "edges": [0, 1, 3, 4, 5, 127, 128, 129, 255, 256, 257, 511, 513, 4095, 4097],
    "long": [100_003, 8192, 70_001],
    "many": [(k * 37) % 300 for k in range(1000)],           # three launches
}
TYPES = [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "bf16")]


def _case(sizes, param, grad, bits, lead, seed):
    torch, dt = _torch()
    rng = np.random.default_rng(seed)
    scale = [10.0 ** rng.uniform(-5, 1) for _ in sizes]
    p = [rng.standard_normal(n) for n in sizes]
    g = [s * rng.standard_normal(n) * (rng.random(n) < 0.9) for n, s in zip(sizes, scale)]
    c = {"p": _Buf(p, dt[param], lead), "g": _Buf(g, dt[grad], lead)}
    m = [0.5 * s * rng.standard_normal(n) for n, s in zip(sizes, scale)]
    v = [(s * np.exp(rng.standard_normal(n))) ** 2 for n, s in zip(sizes, scale)]
    if bits == 32:
        c["m"], c["v"] = _Buf(m, torch.float32, lead), _Buf(v, torch.float32, lead)
    else:
        blocks = [-(-n // 256) for n in sizes]
        c["m"] = _Buf([rng.choice(np.r_[0:127, 128:255], n).astype(np.uint8) for n in sizes], torch.uint8, lead)
        c["v"] = _Buf([rng.integers(0, 127, n).astype(np.uint8) for n in sizes], torch.uint8, lead)
        c["ms"] = _Buf([s * 10.0 ** rng.uniform(-4, -2, b) for b, s in zip(blocks, scale)], torch.float32, lead)
        c["vs"] = _Buf([s * 10.0 ** rng.uniform(-4, -2, b) for b, s in zip(blocks, scale)], torch.float32, lead)
    return c


def _moments(c, k, bits, n):
    if bits == 32:
        return c["m"].get(k), c["v"].get(k)
    return _values8(c["m"].get(k), c["ms"].get(k), n), _values8(c["v"].get(k), c["vs"].get(k), n) ** 2


def _step(c, param, grad, bits, step=1, d_step=0, d_scale=0, stream=0, **kw):
    import paper_2307_11617_b200 as pkg
    more = {} if bits == 32 else {"m_scale": c["ms"].addresses(), "v_scale": c["vs"].addresses()}
    pkg.rfast_adamw_step(c["p"].addresses(), c["g"].addresses(), c["m"].addresses(), c["v"].addresses(), c["p"].numel, step=step, lr=LR, beta1=B1,
                         beta2=B2, eps=EPS, weight_decay=WD, param_type=param, grad_type=grad, d_step=d_step, d_grad_scale=d_scale, cuda_stream=stream, **more, **kw)


def _near8(got, want, err, scale):
    """|got - want| within half a code step plus `err`, the doubt about want."""
    top = np.maximum(np.abs(want), np.abs(got))
    assert np.all(np.abs(got - want) <= np.maximum(2.0 ** -4 * top, 2.0 ** -10 * scale) + err + 8 * U * top)


def _check(before, c, k, param, bits, step, gscale):
    p, g, (m, v) = before
    gp = gscale * g
    s = np.abs(B1 * m) + np.abs((1 - B1) * gp)
    m1, v1 = B1 * m + (1 - B1) * gp, B2 * v + (1 - B2) * gp * gp
    r1 = np.sqrt(v1)
    den = r1 / math.sqrt(1 - B2 ** step) + EPS
    lr = LR / (1 - B1 ** step)
    q = lr * m1 / den
    want = p * (1 - LR * WD) - q
    dm = 5 * U * s + 2.0 ** -149
    tol = 16 * U * np.abs(q) + lr * dm / den + 3 * U * np.abs(p)
    tol += HALF[param] * (np.abs(want) + tol) + TINY[param]
    got = c["p"].get(k)
    # beyond its type's range a parameter is infinite (f16 rounds from 65520 on; a first moment whose second
    # moment is zero is divided by eps alone), and what was infinite does not come back
    over = {"f16": 65520.0}.get(param, 3.4e38)
    gone = ~np.isfinite(got)
    assert np.all((np.abs(want) + tol)[gone & np.isfinite(p)] >= over) and not np.isfinite(got[~np.isfinite(p)]).any()
    with np.errstate(invalid="ignore"):
        assert np.all((np.abs(got - want) <= tol) | gone), np.nanmax(np.abs(got - want) / tol)
    n = len(p)
    if bits == 32:
        assert np.all(np.abs(c["m"].get(k) - m1) <= dm)
        assert np.all(np.abs(c["v"].get(k) - v1) <= 8 * U * v1 + 2.0 ** -148)
        return
    ms, vs = c["ms"].get(k), c["vs"].get(k)
    blocks = -(-n // 256)
    pad = lambda a: np.concatenate([a, np.zeros(blocks * 256 - n)]).reshape(blocks, 256)  # noqa: E731
    dr = 6 * U * r1                                          # as in the quotient
    for scale, val, err in ((ms, np.abs(m1), dm), (vs, r1, dr)):
        top, doubt = pad(val).max(1), pad(err).max(1)
        assert np.all(np.abs(scale - np.maximum(top / 448, 2.0 ** -100)) <= doubt / 448 + 3 * U * top / 448)
    per = lambda a: np.repeat(a, 256)[:n]  # noqa: E731
    _near8(_values8(c["m"].get(k), ms, n), m1, dm, per(ms))
    rv = _values8(c["v"].get(k), vs, n)
    least = np.where(r1 > 0, 2.0 ** -9 * per(vs), 0)
    assert np.all((rv > 0) == (r1 > 0))
    _near8(rv, np.maximum(r1, least), dr, per(vs))


@pytest.mark.parametrize("lead", [0, 16, 1], ids=["aligned", "offset16", "odd"])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", TYPES, ids=["-".join(t) for t in TYPES])
@pytest.mark.parametrize("sizes", list(SIZES))
def test_adamw_step_against_64_bits(rfast_lib, sizes, param, grad, bits, lead):
    torch, _ = _torch()
    c = _case(SIZES[sizes], param, grad, bits, lead, seed=len(sizes) + bits + lead)
    for step in (1, 2, 100):
        before = [(c["p"].get(k), c["g"].get(k), _moments(c, k, bits, n)) for k, n in enumerate(SIZES[sizes])]
        _step(c, param, grad, bits, step)
        torch.cuda.synchronize()
        for k in range(len(before)):
            if SIZES[sizes][k]:
                _check(before[k], c, k, param, bits, step, 1.0)
    assert all(b.canaries_stand() for b in c.values())


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_runs_repeat_bit_for_bit_and_on_any_stream(rfast_lib, bits):
    torch, _ = _torch()
    got = []
    for stream in (None, torch.cuda.Stream(), None):
        c = _case(SIZES["long"], "bf16", "bf16", bits, 0, seed=3)
        torch.cuda.synchronize()
        for step in (1, 2, 3):
            _step(c, "bf16", "bf16", bits, step, stream=0 if stream is None else stream.cuda_stream)
        torch.cuda.synchronize()
        got.append({k: b.t.clone() for k, b in c.items()})
    for other in got[1:]:
        assert all(torch.equal(got[0][k], other[k]) for k in got[0])


@pytest.mark.parametrize("bits", [32, 8])
def test_clipped_step_recorded_and_replayed(rfast_lib, bits):
    """Norm, clip factor and step with the step count on the device, captured once and replayed, equal
    the same calls made one by one."""
    import paper_2307_11617_b200 as pkg
    torch, _ = _torch()
    runs = []
    for recorded in (False, True):
        c = _case(SIZES["edges"] + SIZES["long"], "f32", "f32", bits, 0, seed=8)
        norm = torch.zeros(2, device="cuda")
        work = torch.empty(pkg.GRAD_NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
        count = torch.zeros(1, dtype=torch.int64, device="cuda")
        stream = torch.cuda.Stream()

        def once():
            count.add_(1)
            pkg.rfast_grad_norm(c["g"].addresses(), c["g"].numel, 0.5, norm.data_ptr(), norm.data_ptr() + 4, work.data_ptr(), work.numel(),
                                cuda_stream=stream.cuda_stream)
            _step(c, "f32", "f32", bits, d_step=count.data_ptr(), d_scale=norm.data_ptr() + 4, stream=stream.cuda_stream)

        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            if recorded:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    once()
                for _ in range(4):
                    graph.replay()
            else:
                for _ in range(4):
                    once()
        torch.cuda.synchronize()
        assert int(count) == 4
        runs.append({k: b.t.clone() for k, b in c.items()} | {"norm": norm.clone()})
    assert all(torch.equal(runs[0][k], runs[1][k]) for k in runs[0])
    # and the host's step count gives the same bits as the device's
    c = _case(SIZES["edges"] + SIZES["long"], "f32", "f32", bits, 0, seed=8)
    scale = runs[0]["norm"][1:].clone()
    for step in range(1, 5):
        _step(c, "f32", "f32", bits, step, d_scale=scale.data_ptr())
    torch.cuda.synchronize()
    for k in ("m", "v"):
        assert torch.equal(c[k].t, runs[0][k])


@pytest.mark.parametrize("bits", [32, 8])
def test_clip_factor_enters_the_gradients(rfast_lib, bits):
    torch, _ = _torch()
    c = _case(SIZES["long"], "f32", "bf16", bits, 0, seed=5)
    before = [(c["p"].get(k), c["g"].get(k), _moments(c, k, bits, n)) for k, n in enumerate(SIZES["long"])]
    scale = torch.tensor([0.375], device="cuda")
    _step(c, "f32", "bf16", bits, 7, d_scale=scale.data_ptr())
    torch.cuda.synchronize()
    for k in range(len(before)):
        _check(before[k], c, k, "f32", bits, 7, 0.375)


def test_zero_gradients_leave_zero_moments(rfast_lib):
    """All bytes zero are moments of zero; with no gradient only the decay acts."""
    torch, _ = _torch()
    n = [300, 5]
    c = {"p": _Buf([np.ones(k) for k in n], torch.float32, 0), "g": _Buf([np.zeros(k) for k in n], torch.float32, 0),
         "m": _Buf([np.zeros(k, np.uint8) for k in n], torch.uint8, 0), "v": _Buf([np.zeros(k, np.uint8) for k in n], torch.uint8, 0),
         "ms": _Buf([np.zeros(2), np.zeros(1)], torch.float32, 0), "vs": _Buf([np.zeros(2), np.zeros(1)], torch.float32, 0)}
    _step(c, "f32", "f32", 8, 1)
    torch.cuda.synchronize()
    for k in range(2):
        assert not c["m"].get(k).any() and not c["v"].get(k).any()
        assert np.all(c["p"].get(k) == np.float32(1.0) * np.float32(1 - LR * WD))
        assert np.all(c["ms"].get(k) == 2.0 ** -100)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_bad_gradients_stay_in_their_block(rfast_lib, bits, bad):
    """A NaN or an infinity spoils its own value (32 bits) or its own block of moments (8 bits), nothing else."""
    torch, _ = _torch()
    n = 256 * 5 + 9
    plain, hurt = (_case([n], "f32", "f32", bits, 0, seed=4) for _ in range(2))
    at = 256 * 2 + 100
    hurt["g"].t[hurt["g"].at[0] + at] = bad
    for c in (plain, hurt):
        _step(c, "f32", "f32", bits, 3)
    torch.cuda.synchronize()
    a, b = plain["p"].get(0), hurt["p"].get(0)
    keep = np.arange(n) != at
    assert np.array_equal(a[keep], b[keep]) and not math.isfinite(b[at])
    for k in ("m", "v"):
        x, y = plain[k].get(0), hurt[k].get(0)
        if bits == 32:
            assert np.array_equal(x[keep], y[keep]) and not math.isfinite(y[at])
        else:
            out = np.arange(n) // 256 != 2
            assert np.array_equal(x[out], y[out])
            s = hurt[k + "s"].get(0)
            assert not math.isfinite(s[2]) and np.isfinite(np.delete(s, 2)).all()
            assert not np.isfinite(_values8(y, s, n)[~out]).any() or bad == math.inf
            assert not math.isfinite(_values8(y, s, n)[at])


def test_small_blocks_keep_their_range(rfast_lib):
    """Gradients far below and far above the usual: scales hold them, nothing overflows or vanishes."""
    torch, _ = _torch()
    for size in (1e-25, 1e-12, 1e12):
        g = size * np.linspace(0.5, 1, 512)
        c = {"p": _Buf([np.ones(512)], torch.float32, 0), "g": _Buf([g], torch.float32, 0),
             "m": _Buf([np.zeros(512, np.uint8)], torch.uint8, 0), "v": _Buf([np.zeros(512, np.uint8)], torch.uint8, 0),
             "ms": _Buf([np.zeros(2)], torch.float32, 0), "vs": _Buf([np.zeros(2)], torch.float32, 0)}
        before = [(c["p"].get(0), c["g"].get(0), _moments(c, 0, 8, 512))]
        _step(c, "f32", "f32", 8, 1)
        torch.cuda.synchronize()
        m, v = _moments(c, 0, 8, 512)
        # 2^-4 half a code step, and what fp32 leaves of a square below its normal range
        assert np.all(np.abs(m / ((1 - B1) * g) - 1) <= 2.0 ** -4 + 1e-6)
        if size > 1e-18:
            _check(before[0], c, 0, "f32", 8, 1, 1.0)
            assert np.all(np.abs(np.sqrt(v) / (math.sqrt(1 - B2) * g) - 1) <= 2.0 ** -4 + 1e-6)


def test_more_than_2_31_values(rfast_lib):
    """The end of a tensor of more than 2^31 values steps like a tensor of its own; only it has a gradient, and the norm finds it."""
    import paper_2307_11617_b200 as pkg
    torch, _ = _torch()
    tail, n = 256 * 40 + 77, 2 ** 31 + 256 * 40 + 77
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros(-(-n // 256), device="cuda") for _ in range(2))
    torch.manual_seed(3)
    p[-tail:], g[-tail:] = torch.randn(tail, device="cuda"), torch.randn(tail, device="cuda")
    small = [t[-tail:].clone() for t in (p, g, m, v)] + [t[-(-(-tail // 256)):].clone() for t in (ms, vs)]
    norm, work = torch.zeros(1, device="cuda"), torch.empty(pkg.GRAD_NORM_WORKSPACE, dtype=torch.uint8, device="cuda")
    pkg.rfast_grad_norm([g.data_ptr()], [n], 1.0, norm.data_ptr(), 0, work.data_ptr(), work.numel(), grad_type="bf16",
                        cuda_stream=torch.cuda.current_stream().cuda_stream)
    for t, k in (((p, g, m, v, ms, vs), n), (small, tail)):
        a = [[x.data_ptr()] for x in t]
        pkg.rfast_adamw_step(a[0], a[1], a[2], a[3], [k], step=1, lr=LR, m_scale=a[4], v_scale=a[5], param_type="bf16", grad_type="bf16",
                             cuda_stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(x[-y.numel():], y) for x, y in zip((p, m, v, ms, vs), (small[0], *small[2:])))
    assert not m[:256].any() and not p[:256].any() and bool((ms[:8] == 2.0 ** -100).all())
    want = float(np.sqrt((g[-tail:].double().cpu().numpy() ** 2).sum()))
    assert abs(float(norm) - want) <= 5 * U * want           # eight squares summed in fp32, 8 u; half of it in the root; the result


def test_host_and_foreign_addresses_are_refused(rfast_lib):
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200.binding import EINVAL, RFastError
    torch, _ = _torch()
    d = torch.zeros(1024, device="cuda")
    h = np.zeros(1024, np.float32)
    a = d.data_ptr()
    with pytest.raises(RFastError) as ei:
        pkg.rfast_adamw_step([a], [h.ctypes.data], [a + 512], [a + 1024], [4], step=1)
    assert ei.value.code == EINVAL and "grad: not device memory" in str(ei.value)
    with pytest.raises(RFastError) as ei:
        pkg.rfast_grad_norm([a], [4], 1.0, h.ctypes.data, 0, a, 1 << 20)
    assert ei.value.code == EINVAL and "d_norm: not device memory" in str(ei.value)


# ---- gradient norm -----------------------------------------------------------------------------------
def _norm(bufs, kind, max_norm, stream=0):
    import paper_2307_11617_b200 as pkg
    torch, _ = _torch()
    out = torch.full((2,), 55.0, device="cuda")
    work = torch.full((pkg.GRAD_NORM_WORKSPACE,), 255, dtype=torch.uint8, device="cuda")      # NaNs: read only what was written
    torch.cuda.synchronize()
    pkg.rfast_grad_norm(bufs.addresses(), bufs.numel, max_norm, out.data_ptr(), out.data_ptr() + 4, work.data_ptr(), work.numel(), grad_type=kind,
                        cuda_stream=stream)
    torch.cuda.synchronize()
    return [float(x) for x in out]


@pytest.mark.parametrize("lead", [0, 1], ids=["aligned", "odd"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("sizes", list(SIZES) + ["thousands"])
def test_grad_norm_against_64_bits(rfast_lib, sizes, kind, lead):
    """Groups of eight squares are summed in fp32 (8 u of the sum at most), everything above in 64 bits, so
    the norm is off by 4 u and its own rounding; the factor by its rounding on top."""
    _, dt = _torch()
    n = SIZES.get(sizes) or [1 + k % 5 for k in range(4000)]
    rng = np.random.default_rng(len(n) + lead)
    b = _Buf([10.0 ** rng.uniform(-3, 3) * rng.standard_normal(k) for k in n], dt[kind], lead)
    want = math.sqrt(math.fsum(float((b.get(k) ** 2).sum()) for k in range(len(n))))
    norm, scale = _norm(b, kind, 0.25)
    assert abs(norm - want) <= 6 * U * want
    ratio = 1.0 if want <= 0.25 else 0.25 / want
    assert abs(scale - ratio) <= 7 * U * ratio
    assert _norm(b, kind, 0.25) == [norm, scale]
    assert _norm(b, kind, 1e30) == [norm, 1.0]
    assert b.canaries_stand()


@pytest.mark.parametrize("values,norm", [
    ([0.0, 0.0], 0.0), ([3e30, 4e30], 5e30), ([3e-30, 4e-30], 5e-30), ([3e25, 4e-30], 3e25), ([1e-40], 1e-40),
    ([math.inf, 1.0], math.inf), ([math.nan, math.inf], math.nan), ([1e38] * 20, math.sqrt(20) * 1e38), ([], 0.0)])
def test_grad_norm_at_the_ends_of_the_range(rfast_lib, values, norm):
    torch, _ = _torch()
    b = _Buf([np.asarray(values, np.float64), np.zeros(0)], torch.float32, 0)
    got, scale = _norm(b, "f32", 1.0)
    if math.isnan(norm):
        assert math.isnan(got) and math.isnan(scale)
    elif norm > 3.4028235e38:
        assert got == math.inf and (scale == 0 or norm < math.inf)
    else:
        assert abs(got - norm) <= 6 * U * norm + 2.0 ** -149
        assert scale == (1.0 if norm <= 1 else pytest.approx(1 / norm, rel=1e-6))


@pytest.mark.parametrize("clip", [1.0, 0.30078125, 0.3])
@pytest.mark.parametrize("lead", [0, 1], ids=["aligned", "odd"])
def test_first_moments_codes_are_those_of_the_formula_in_32_bits(rfast_lib, lead, clip):
    """Codes and scales of the first moment equal, bit for bit, those of the formula evaluated one operation after the other in fp32.
    A moment near a border between two codes falls on one side or the other by its last bits; over 2^24 values some twenty are that near."""
    import paper_2307_11617_b200 as pkg
    torch, _ = _torch()
    n = 2 ** 24 + 77
    torch.manual_seed(11 + lead)
    size = torch.exp(2 * torch.randn(-(-n // 256), device="cuda") - 7).repeat_interleave(256)[:n]
    at = lambda values: torch.cat([torch.zeros(lead, dtype=values.dtype, device="cuda"), values])  # noqa: E731
    p, g = at(torch.randn(n, device="cuda")), at(size * torch.randn(n, device="cuda"))
    m = at(torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda") & 0xFE)           # no code is a NaN
    v = at(torch.randint(1, 127, (n,), dtype=torch.uint8, device="cuda"))
    ms, vs = size[::256] * 1e-3, size[::256] * 1e-2
    b1 = torch.tensor(B1, dtype=torch.float32, device="cuda")
    g1 = torch.tensor(1.0 - B1, dtype=torch.float32, device="cuda")
    scale = torch.tensor([clip], device="cuda")
    old = m[lead:].view(torch.float8_e4m3fn).float() * ms.repeat_interleave(256)[:n]
    want = old * b1 + (g[lead:] * scale) * g1
    full = torch.cat([want, torch.zeros(-n % 256, device="cuda")]).view(-1, 256)
    top = (full.abs().amax(1) * torch.tensor(1 / 448, device="cuda")).clamp_min(2.0 ** -100)
    code = (full * (1.0 / top)[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).view(-1)[:n]
    a = lambda t: [t.data_ptr() + lead * t.element_size()]  # noqa: E731
    pkg.rfast_adamw_step(a(p), a(g), a(m), a(v), [n], step=3, lr=LR, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD, m_scale=[ms.data_ptr()],
                         v_scale=[vs.data_ptr()], d_grad_scale=scale.data_ptr(), cuda_stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(ms, top)
    assert int((m[lead:] != code).sum()) == 0


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("lead", [0, 1], ids=["aligned", "odd"])
@pytest.mark.parametrize("low,high", [(-36, -36), (-30, -30), (-25, -25), (-21, -21), (-18, -18), (17, 17), (22, 22), (30, 30), (37.9, 37.9), (-36, 37)])
def test_roots_of_8_bit_moments_reach_as_far_as_fp32(rfast_lib, monkeypatch, low, high, lead, grad):
    """Gradients of any finite size, alike or mixed in one block: their squares leave fp32, their roots do not.  With the least eps
    a first moment meets its root or nothing.  The tolerances are those of the other sizes: scaling by powers of two rounds nothing,
    and no root here is below 2^-126."""
    torch, _ = _torch()
    monkeypatch.setitem(globals(), "EPS", 2.0 ** -126)
    n = 256 * 5 + 100
    rng = np.random.default_rng(int(10 * low) + 1000)
    g = [10.0 ** rng.uniform(low, high, n) * rng.uniform(0.5, 1, n) * rng.choice([-1, 1], n) for _ in range(3)]
    for k in range(3):
        g[k][rng.random(n) < 0.1] = 0
        g[k][512:768] = 0                                    # a block that sees nothing
    c = {"p": _Buf([rng.standard_normal(n)], torch.float32, lead), "g": _Buf([g[0]], _torch()[1][grad], lead),
         "m": _Buf([np.zeros(n, np.uint8)], torch.uint8, lead), "v": _Buf([np.zeros(n, np.uint8)], torch.uint8, lead),
         "ms": _Buf([np.zeros(6)], torch.float32, lead), "vs": _Buf([np.zeros(6)], torch.float32, lead)}
    for step in (1, 2, 3):
        c["g"].t[c["g"].at[0]:c["g"].at[0] + n] = torch.as_tensor(g[step - 1]).to(c["g"].t.dtype).cuda()
        before = (c["p"].get(0), c["g"].get(0), _moments(c, 0, 8, n))
        assert np.isfinite(before[1]).all()
        _step(c, "f32", grad, 8, step)
        torch.cuda.synchronize()
        assert all(np.isfinite(c[k].get(0)).all() for k in ("p", "ms", "vs"))
        _check(before, c, 0, "f32", 8, step, 1.0)
    assert all(b.canaries_stand() for b in c.values())


def test_an_infinite_gradient_takes_its_whole_block(rfast_lib):
    """Every moment of the block is infinite or NaN afterwards, those of the other blocks are as without it."""
    torch, _ = _torch()
    n = 256 * 3
    plain, hurt = (_case([n], "f32", "f32", 8, 0, seed=14) for _ in range(2))
    hurt["g"].t[hurt["g"].at[0] + 300] = math.inf
    for c in (plain, hurt):
        _step(c, "f32", "f32", 8, 3)
    torch.cuda.synchronize()
    inside = np.arange(n) // 256 == 1
    for k in ("m", "v"):
        assert np.array_equal(plain[k].get(0)[~inside], hurt[k].get(0)[~inside])
        with np.errstate(invalid="ignore"):
            assert not np.isfinite(_values8(hurt[k].get(0), hurt[k + "s"].get(0), n)[inside]).any()


@pytest.mark.parametrize("lead", [0, 1], ids=["aligned", "odd"])
@pytest.mark.parametrize("size", [1e-17, 1e-18, 1e-19, 1e-20])
def test_small_second_moments_of_32_bits_count(rfast_lib, size, lead):
    """Second moments below 2^-126, with an eps far below their roots: the quotient is that of the roots, not m / eps.
    A square down there is held to half of 2^-149, its product with 1 - beta2 and the sum each: 2^-149 in all, which the root halves
    relative to itself; the rest of the quotient is off by 16 u as elsewhere."""
    torch, _ = _torch()
    import paper_2307_11617_b200 as pkg
    n, eps = 256 * 3 + 10, 2.0 ** -126
    rng = np.random.default_rng(9)
    g = size * rng.uniform(0.5, 1, n) * rng.choice([-1, 1], n)
    c = {"p": _Buf([rng.standard_normal(n)], torch.float32, lead), "g": _Buf([g], torch.float32, lead),
         "m": _Buf([np.zeros(n)], torch.float32, lead), "v": _Buf([np.zeros(n)], torch.float32, lead)}
    for step in (1, 2, 3):
        p, m, v, gg = (c[k].get(0) for k in ("p", "m", "v", "g"))
        pkg.rfast_adamw_step(*[c[k].addresses() for k in ("p", "g", "m", "v")], [n], step=step, lr=LR, beta1=B1, beta2=B2, eps=eps, weight_decay=WD)
        torch.cuda.synchronize()
        m1, v1 = B1 * m + (1 - B1) * gg, B2 * v + (1 - B2) * gg * gg
        q = LR / (1 - B1 ** step) * m1 / (np.sqrt(v1) / math.sqrt(1 - B2 ** step) + eps)
        tol = np.abs(q) * (2.0 ** -149 / (2 * v1) * 1.01 + 16 * U) + LR / (1 - B1 ** step) * (5 * U * (np.abs(B1 * m) + np.abs((1 - B1) * gg))) / np.sqrt(v1)
        tol += 3 * U * np.abs(p) + U * np.abs(p)
        assert v1.max() < 2.0 ** -100 and np.all(np.abs(c["v"].get(0) - v1) <= 8 * U * v1 + 2.0 ** -149)
        assert np.all(np.abs(c["p"].get(0) - (p * (1 - LR * WD) - q)) <= tol)


@pytest.mark.parametrize("step", [1, 2, 3, 100, 10 ** 6])
@pytest.mark.parametrize("bits", [32, 8])
def test_step_count_on_the_device_enters_the_parameters(rfast_lib, bits, step):
    """The count that d_step points to forms both bias corrections: parameters and moments against 64 bits, beside a host count that
    must not be read."""
    torch, _ = _torch()
    c = _case(SIZES["edges"], "f32", "f32", bits, 0, seed=21)
    before = [(c["p"].get(k), c["g"].get(k), _moments(c, k, bits, n)) for k, n in enumerate(SIZES["edges"])]
    count = torch.tensor([step], dtype=torch.int64, device="cuda")
    _step(c, "f32", "f32", bits, step=7, d_step=count.data_ptr())
    torch.cuda.synchronize()
    for k, n in enumerate(SIZES["edges"]):
        if n:
            _check(before[k], c, k, "f32", bits, step, 1.0)


@pytest.mark.parametrize("bits", [32, 8])
def test_recorded_count_moves_the_parameters_as_the_hosts(rfast_lib, bits):
    """A recorded step with its count on the device, replayed, against 64 bits at every step."""
    torch, _ = _torch()
    c = _case(SIZES["long"], "f32", "f32", bits, 0, seed=22)
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        count.add_(1)
        _step(c, "f32", "f32", bits, d_step=count.data_ptr(), stream=stream.cuda_stream)
    for step in (1, 2, 3, 4):
        before = [(c["p"].get(k), c["g"].get(k), _moments(c, k, bits, n)) for k, n in enumerate(SIZES["long"])]
        graph.replay()
        torch.cuda.synchronize()
        assert int(count) == step
        for k in range(len(before)):
            _check(before[k], c, k, "f32", bits, step, 1.0)


@pytest.mark.parametrize("change", [1.0, 0.1, 10.0])
@pytest.mark.parametrize("beta2", [0.9, 0.95, 0.99, 0.999])
def test_8_bit_moments_beside_32_bit_ones_over_many_steps(rfast_lib, beta2, change):
    """How far nearest codes follow the average, as the header states it: 2000 steps on four blocks, from step 500 on with half of every
    block's gradients `change` times as large."""
    import paper_2307_11617_b200 as pkg
    torch, _ = _torch()
    n, steps = 1024, 2000
    torch.manual_seed(17)
    factor = torch.ones(n, device="cuda")
    factor[(torch.arange(n, device="cuda") % 256) < 128] = change
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    q, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
    cm, cv = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    sm, sv = (torch.zeros(4, device="cuda") for _ in range(2))
    a = lambda t: [t.data_ptr()]  # noqa: E731
    stream = torch.cuda.current_stream().cuda_stream
    steady, changed = [], []
    for step in range(1, steps + 1):
        g.copy_(torch.randn(n, device="cuda") * (factor if step > 500 else 1.0))
        pkg.rfast_adamw_step(a(p), a(g), a(m), a(v), [n], step=step, beta2=beta2, cuda_stream=stream)
        pkg.rfast_adamw_step(a(q), a(g), a(cm), a(cv), [n], step=step, beta2=beta2, m_scale=a(sm), v_scale=a(sv), cuda_stream=stream)
        if step % 100 == 0:
            torch.cuda.synchronize()
            ratio = _values8(cv.cpu().numpy(), sv.cpu().numpy(), n) / np.sqrt(v.double().cpu().numpy())
            (steady if step <= 500 or change == 1.0 else changed).append(ratio)
            first = _values8(cm.cpu().numpy(), sm.cpu().numpy(), n)
            assert np.abs(first - m.double().cpu().numpy()).mean() <= 0.1 * np.abs(m.double().cpu().numpy()).mean()
    steady = np.array(steady)
    assert np.median(steady) <= (1.2 if beta2 <= 0.95 else 1.6) and 0.5 <= steady.min() and steady.max() <= (1.6 if beta2 <= 0.95 else 2.2)
    if changed:
        late = np.array(changed[5:])                         # 500 steps and more after the change
        if beta2 <= 0.95:
            assert 0.6 <= late.min() and late.max() <= 1.7
        else:
            assert 0.1 <= late.min() and late.max() <= 22.0  # by the change's factor, times the two of steady gradients
