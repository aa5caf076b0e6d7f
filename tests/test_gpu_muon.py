"""Muon step against a plain restatement in 64 bits.

The iteration multiplies errors along directions in which the update is small (by up to 3.4445 an iteration), so tolerances come from the
64-bit iteration itself: it is run again with every factor off by a random relative error of up to d (half a step of what holds a factor: 2^-11
for one fp16 number, 2^-21 for the sum of two, the missing low-by-low product included, plus 2^-24 for the fp32 value that is rounded) and every
product smaller by a random share of up to (instructions) 2^-23 of itself (the tensor cores' sums round towards zero, once in 16 terms; terms = 2
has three products), and may be off by three times the largest response of four such runs, in Frobenius norm and in one value.  (The largest
value, not a multiple of the root mean square: the error of x_ij varies as |x_ij|, and with a few large directions x is a product of normal
numbers, whose spread over 2 million values is beyond 10.  Given the x_ij the errors are sums of many small ones, so the largest of four
runs' 8 million is at least 5 standard deviations of the widest elements out, and three times that is 15.)  On top:
  M   mu M + (1 - mu) g': constants, products, sum: 4 u of |mu M| + |(1 - mu) g'|  (u = 2^-24)
  p   the decay's constant, product and sum 3 u of |p|, the step's constant and product 3 u of the update, half a step of p's type."""

from __future__ import annotations

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
A, B, C = 3.4445, -4.7750, 2.0315


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


class _List:
    """Matrices at odd places of one allocation, marks in between."""

    def __init__(self, values, kind, lead=0):
        import torch
        self.shapes = [tuple(v.shape) for v in values]
        at, self.at = lead, []
        for v in values:
            self.at.append(at)
            at += (v.numel() + 15) // 16 * 16 + 16
        self.t = torch.full((at + 16,), 77.0, dtype=_dt(kind), device="cuda")
        for v, a in zip(values, self.at):
            self.t[a:a + v.numel()] = v.reshape(-1).to(_dt(kind))

    def __getitem__(self, k):
        a, s = self.at[k], self.shapes[k]
        return self.t[a:a + s[0] * s[1]].view(s)

    def addresses(self):
        return [self.t.data_ptr() + a * self.t.element_size() for a in self.at]

    def marks_stand(self):
        import torch
        keep = torch.ones_like(self.t, dtype=torch.bool)
        for a, s in zip(self.at, self.shapes):
            keep[a:a + s[0] * s[1]] = False
        return bool((self.t[keep].double() == 77.0).all())


def _iterate(u, eps, iterations, terms=0, seed=None):
    """The update orthogonalised, in 64 bits; with a seed: with random errors of the size that the kernel's have."""
    import torch
    x = u.double()
    turned = x.shape[0] > x.shape[1]
    if turned:
        x = x.T
    x = x / max(float(torch.linalg.vector_norm(x)), eps)
    gen = None
    if seed is not None:
        gen = torch.Generator(device=x.device)
        gen.manual_seed(seed)
    d = 2.0 ** -24 + (2.0 ** -11 if terms == 1 else 2.0 ** -21)

    def held(t):
        return t if gen is None else t * (1 + d * (2 * torch.rand(t.shape, generator=gen, device=t.device, dtype=t.dtype) - 1))

    def times(a, b):
        p = a @ b
        if gen is None:
            return p
        steps = -(-a.shape[1] // 16) * (1 if terms == 1 else 3)
        return p * (1 - steps * 2.0 ** -23 * torch.rand((), generator=gen, device=a.device, dtype=a.dtype))

    for _ in range(iterations):
        x = held(x)
        s = held(times(x, x.T))
        poly = held(B * s + C * times(s, s))
        x = A * x + times(poly, x)
    return x.T if turned else x


def _slope(gen, rows, cols, low, size=1.0):
    import torch
    g = torch.randn(rows, cols, generator=gen, device="cuda")
    if low:
        r = min(4, rows, cols)
        g = 0.3 * g + torch.randn(rows, r, generator=gen, device="cuda") @ torch.randn(r, cols, generator=gen, device="cuda")
    return g * size


def _step(shapes, param="f32", grad="f32", terms=0, lead=0, low=False, seed=0, sizes=None, scale=None, zero_m=False, **kw):
    import torch
    import paper_2307_11617_b200 as pkg
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 17)
    sizes = sizes or [10.0 ** ((3 * k) % 5 - 4) for k in range(len(shapes))]
    c = {"p": _List([0.05 * torch.randn(r, q, generator=gen, device="cuda") for r, q in shapes], param, lead),
         "g": _List([_slope(gen, r, q, low, s) for (r, q), s in zip(shapes, sizes)], grad, lead),
         "m": _List([_slope(gen, r, q, low, 0.0 if zero_m else 0.5 * s) for (r, q), s in zip(shapes, sizes)], "f32", lead)}
    c["scale"] = None if scale is None else torch.tensor([scale], device="cuda")
    c["before"] = {k: [c[k][i].double().clone() for i in range(len(shapes))] for k in "pgm"}
    rows, cols = [s[0] for s in shapes], [s[1] for s in shapes]
    need = pkg.rfast_muon_workspace(rows, cols, param_type=param, terms=terms)
    c["work"] = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    c["call"] = lambda stream: pkg.rfast_muon_step(  # noqa: E731
        c["p"].addresses(), c["g"].addresses(), c["m"].addresses(), rows, cols, terms=terms, param_type=param, grad_type=grad,
        d_grad_scale=0 if scale is None else c["scale"].data_ptr(), workspace=c["work"].data_ptr(), workspace_bytes=need, cuda_stream=stream, **kw)
    c["call"](torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert int(c["work"][:4].view(torch.int32)) == 0
    assert bool((c["work"][need:] == 255).all())
    c["terms"] = terms or (1 if param == "bf16" else 2)
    return c


def _check(c, shapes, param, lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True, eps=1e-7, iterations=5, size_rule="spectral", only=None):
    import torch
    scale = 1.0 if c["scale"] is None else float(c["scale"])
    assert c["p"].marks_stand() and c["g"].marks_stand() and c["m"].marks_stand()
    for k, (rows, cols) in enumerate(shapes):
        if rows == 0 or cols == 0 or (only is not None and k not in only):
            continue
        g, m0 = c["before"]["g"][k] * scale, c["before"]["m"][k]
        m = momentum * m0 + (1 - momentum) * g
        tol = 4 * U * (abs(momentum) * m0.abs() + (1 - momentum) * g.abs()) + 2.0 ** -149
        assert bool(((c["m"][k].double() - m).abs() <= tol).all()), ("momentum", k)
        u = (1 - momentum) * g + momentum * m if nesterov else m
        x = _iterate(u, eps, iterations)
        off = [_iterate(u, eps, iterations, c["terms"], seed) - x for seed in range(4)]
        norm = 3 * max(float(d.norm()) for d in off)
        size = math.sqrt(max(1.0, rows / cols)) if size_rule == "spectral" else 0.2 * math.sqrt(max(rows, cols))
        p0 = c["before"]["p"][k]
        p = p0 * (1 - lr * weight_decay) - lr * size * x
        rounding = 3 * U * (p0.abs() + abs(lr) * size * x.abs()) + HALF[param] * p.abs() + TINY[param]
        d = (c["p"][k].double() - p).abs()
        most = abs(lr) * size * 3 * max(float(d.abs().max()) for d in off)
        bad = d > rounding * (1 + HALF[param]) + most
        assert not bool(bad.any()), ("p", k, (rows, cols), int(bad.sum()), float((d - rounding).max()), most)
        assert float((d - rounding).clamp_min(0).norm()) <= abs(lr) * size * norm, ("p norm", k, (rows, cols))


SHAPES = [(1, 1), (1, 7), (9, 1), (64, 64), (63, 65), (128, 129), (257, 129), (10, 512), (512, 10), (130, 784), (300, 700), (700, 301), (1, 4096), (2100, 33)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("terms", [1, 2])
def test_orthogonalised_update(rows, cols, terms):
    """The update by itself: parameters of zero, a rate of one; one iteration and five."""
    import torch
    for iterations in (1, 5):
        for low in (False, True):
            c = _step([(rows, cols)], terms=terms, low=low, lr=1.0, iterations=iterations, weight_decay=1.0, sizes=[1.0])
            _check(c, [(rows, cols)], "f32", lr=1.0, iterations=iterations, weight_decay=1.0)


@pytest.mark.parametrize("param,grad,lead", [("f32", "f32", 0), ("f32", "bf16", 1), ("bf16", "bf16", 0), ("bf16", "f32", 3), ("f16", "f16", 5), ("f16", "bf16", 8)])
def test_lists_of_many_shapes(param, grad, lead):
    """More shapes than one run of launches takes, with matrices of nothing among them."""
    shapes = [(96, 40), (40, 96), (0, 5), (96, 40), (33, 33), (200, 130), (17, 300), (300, 17), (64, 128), (5, 0), (129, 65), (250, 260), (1, 1), (12, 700), (96, 40), (80, 81), (81, 82)]
    kw = dict(lr=0.1, weight_decay=0.3, size_rule="rms")
    c = _step(shapes, param, grad, lead=lead, low=True, **kw)
    _check(c, shapes, param, **kw)


def test_more_matrices_than_one_run_takes():
    shapes = [(24, 40)] * 150 + [(40, 24)] * 20 + [(8, 8)] * 100
    c = _step(shapes, "f32", "f32", sizes=[1.0] * 270)
    _check(c, shapes, "f32", only=[0, 1, 77, 127, 128, 149, 150, 169, 170, 200, 255, 256, 269])


@pytest.mark.parametrize("shapes,param,terms", [([(512, 784)] * 40 + [(10, 512)] * 40, "f32", 2), ([(512, 784)] * 40, "bf16", 1), ([(2048, 1030)] * 3, "bf16", 1),
                                                ([(1100, 2048)] * 3, "f32", 2), ([(2500, 2400)], "f32", 1), ([(769, 515)] * 30, "f16", 2)])
def test_pairs_of_blocks(shapes, param, terms):
    """Enough tiles for pairs of thread blocks; last tiles that are cut in rows, in columns, in the sum."""
    c = _step(shapes, param, "f32", terms=terms, low=True, lr=0.5, sizes=[1.0] * len(shapes))
    _check(c, shapes, param, lr=0.5, only=[0, len(shapes) // 2, len(shapes) - 1])


@pytest.mark.parametrize("kw", [dict(nesterov=False), dict(momentum=0.0), dict(scale=0.25), dict(iterations=2), dict(iterations=9, lr=0.3), dict(lr=-0.1), dict(eps=10.0),
                                dict(weight_decay=2.0, lr=0.4), dict(size_rule="rms")])
def test_options(kw):
    shapes = [(70, 50), (50, 90)]
    scale = kw.pop("scale", None)
    c = _step(shapes, scale=scale, sizes=[1.0, 1.0], **kw)
    _check(c, shapes, "f32", **kw)


@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-12, 1e12, 1e30, 1e36])
def test_gradients_of_any_size(size):
    c = _step([(60, 100)], sizes=[size], eps=1e-60)
    _check(c, [(60, 100)], "f32", eps=1e-60)


def test_no_gradient_leaves_the_decay():
    import torch
    c = _step([(60, 100), (33, 20)], sizes=[0.0, 1.0], weight_decay=0.5, lr=0.1)
    _check(c, [(60, 100), (33, 20)], "f32", weight_decay=0.5, lr=0.1)
    assert torch.equal(c["p"][0], (c["before"]["p"][0] * (1 - 0.1 * 0.5)).float()) or float((c["p"][0].double() - c["before"]["p"][0] * 0.95).abs().max()) < 1e-7


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_not_finite_stays_in_its_matrix(bad):
    import torch
    shapes = [(40, 60), (40, 60), (60, 40), (300, 300)]
    c = _step(shapes, sizes=[1.0] * 4)
    c["g"][1][3, 4] = bad
    c["m"][2][0, 0] = bad
    for k in range(4):
        c["before"]["p"][k] = c["p"][k].double().clone()
        c["before"]["m"][k] = c["m"][k].double().clone()
    c["call"](torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert bool(torch.isnan(c["p"][1]).all()) and bool(torch.isnan(c["p"][2]).all())
    _check(c, shapes, "f32", only=[0, 3])


def test_the_same_bits_again_and_recorded():
    """Two lists recorded into graphs and replayed side by side, a workspace each, against calls one after another."""
    import torch
    lists = [[(300, 200), (64, 64)], [(512, 784)] * 12]
    cs = [_step(s, "f32", "f32", sizes=[1.0] * len(s), seed=k) for k, s in enumerate(lists)]
    start = [{k: c[k].t.clone() for k in "pm"} for c in cs]
    want = []
    for c in cs:
        for _ in range(3):
            c["call"](torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        want.append({k: c[k].t.clone() for k in "pm"})
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in cs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c["call"](torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for _ in range(2):
        for c, s in zip(cs, start):
            for k in "pm":
                c[k].t.copy_(s[k])
            c["work"].fill_(255)
        torch.cuda.synchronize()
        for _ in range(3):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        for c, w in zip(cs, want):
            assert torch.equal(c["p"].t, w["p"]) and torch.equal(c["m"].t, w["m"])


def test_update_is_nearly_orthogonal():
    """What the iteration is for: singular values between 0.6 and 1.3 wherever they began above 1 % of the norm."""
    import torch
    c = _step([(256, 400)], zero_m=True, weight_decay=1.0, lr=1.0, sizes=[1.0])
    x = c["p"][0].double()
    u = c["before"]["g"][0]
    a, s, b = torch.linalg.svd(u, full_matrices=False)
    inner = (a.T @ x @ b.T)
    keep = s > 0.01 * s.norm()
    d = -torch.diagonal(inner)[keep]
    assert bool(((d > 0.6) & (d < 1.3)).all())
    assert float((inner - torch.diag(torch.diagonal(inner))).abs().max()) < 1e-3


@pytest.mark.parametrize("rows,cols", [(65536, 1), (3, 65536), (40_001, 70)])
def test_the_longest_sides(rows, cols):
    c = _step([(rows, cols)], sizes=[1.0], low=True, lr=0.5)
    _check(c, [(rows, cols)], "f32", lr=0.5)


def test_calls_from_several_threads():
    """Two host threads, a stream, matrices and a workspace each."""
    import threading
    import torch
    lists = [[(200, 300)] * 5, [(64, 500), (500, 64), (33, 7)]]
    cs = [_step(s, sizes=[1.0] * len(s), seed=10 + k) for k, s in enumerate(lists)]
    start = [{k: c[k].t.clone() for k in "pm"} for c in cs]
    want = []
    for c in cs:
        for _ in range(5):
            c["call"](torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        want.append(c["p"].t.clone())
    for c, s in zip(cs, start):
        for k in "pm":
            c[k].t.copy_(s[k])
    torch.cuda.synchronize()
    streams, failed = [torch.cuda.Stream() for _ in cs], []

    def work(c, s):
        try:
            for _ in range(5):
                c["call"](s.cuda_stream)
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=work, args=a) for a in zip(cs, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for c, w in zip(cs, want):
        assert torch.equal(c["p"].t, w)
