"""What rfast.h promises of the Muon update, asserted as it stands there: how far X is from 64 bits, relative, in Frobenius norm, and that the
same call gives the same bits.

Parameters of zero, a rate of one, a decay that leaves nothing of them, no momentum: U is the gradient itself, and the parameters are -size X, where
size and the step's constant are two fp32 roundings of one number (2^-23 of it) and every value is rounded once (2^-24)."""

from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

A, B, C = 3.4445, -4.7750, 2.0315


def _exact(u, iterations=5):
    x = u.double()
    turned = x.shape[0] > x.shape[1]
    x = x.T if turned else x
    x = x / x.norm()
    for _ in range(iterations):
        s = x @ x.T
        x = A * x + (B * s + C * (s @ s)) @ x
    return x.T if turned else x


def _off(u, terms):
    """Of the update from _exact, relative."""
    import torch
    import paper_2307_11617_b200 as pkg
    rows, cols = u.shape
    p, m = torch.zeros_like(u), torch.zeros_like(u)
    need = pkg.rfast_muon_workspace([rows], [cols], terms=terms)
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    pkg.rfast_muon_step([p.data_ptr()], [u.data_ptr()], [m.data_ptr()], [rows], [cols], lr=1.0, momentum=0.0, weight_decay=1.0, size_rule="rms", terms=terms,
                        workspace=work.data_ptr(), workspace_bytes=need, cuda_stream=torch.cuda.current_stream().cuda_stream)
    x = _exact(u)
    d = p.double() / -(0.2 * math.sqrt(max(rows, cols))) - x
    assert int(work[:4].view(torch.int32)) == 0
    return float(d.norm() / x.norm())


def _gradients(rows, cols):
    """Noise; directions of twice its size over it, eight and (0.3 of it) four; noise of a seventieth of four directions."""
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows * 5 + cols)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def low(k):
        k = min(k, rows, cols)
        return normal(rows, k) @ normal(k, cols)

    yield "noise", normal(rows, cols)
    yield "directions", normal(rows, cols) + low(8)
    yield "directions", 0.3 * normal(rows, cols) + low(4)
    yield "steep", 0.03 * normal(rows, cols) + low(4)


# every side up to 300, then up to 4096, odd ones among them, single rows and columns, squares; tiles of single blocks and of pairs
SHAPES = [(1, 1), (1, 300), (17, 5), (64, 64), (128, 128), (129, 257), (257, 129), (300, 10), (300, 300), (1, 4096), (4096, 1), (10, 512), (512, 784), (700, 301), (1100, 2048),
          (2048, 2048), (4001, 2999), (700, 4096), (4096, 1024), (4096, 4096)]


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_two_terms(rows, cols):
    short = max(rows, cols) <= 300
    for kind, u in _gradients(rows, cols):
        bound = (3e-5 if short else 3e-4) if kind == "steep" else 1e-5 if short else 3e-5
        if min(rows, cols) == 1:
            bound = 5e-6                                     # one long sum of squares, which does not come out small
        off = _off(u, 2)
        assert off <= bound, (kind, off)


@pytest.mark.parametrize("rows,cols", SHAPES + [(64, 65_536), (65_536, 300), (8192, 2000)])
def test_one_term(rows, cols):
    for kind, u in _gradients(rows, cols):
        off = _off(u, 1)
        assert off <= (2e-3 if kind == "noise" else 2e-2), (kind, off)


@pytest.mark.parametrize("count,rows,cols,param,grad", [(6, 4096, 1024, "bf16", "bf16"), (2, 4096, 4096, "bf16", "bf16"), (20, 512, 784, "f32", "f32"), (3, 257, 129, "f16", "bf16"),
                                                        (2, 1100, 2048, "f32", "bf16")])
def test_the_same_call_gives_the_same_bits(count, rows, cols, param, grad):
    """Ten times over, whatever the workspace held, with another stream's work beside it every other time."""
    import torch
    import paper_2307_11617_b200 as pkg
    types = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
    gen = torch.Generator(device="cuda")
    gen.manual_seed(rows + cols)
    p0 = (0.04 * torch.randn(count, rows, cols, generator=gen, device="cuda")).to(types[param])
    g = (0.01 * torch.randn(count, rows, cols, generator=gen, device="cuda")).to(types[grad])
    m0 = 0.01 * torch.randn(count, rows, cols, generator=gen, device="cuda")
    need = pkg.rfast_muon_workspace([rows] * count, [cols] * count, param_type=param)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    other, side = torch.randn(3000, 3000, device="cuda"), torch.cuda.Stream()
    want = None
    for k in range(10):
        p, m = p0.clone(), m0.clone()
        work.fill_(k * 25)
        torch.cuda.synchronize()
        if k % 2:
            with torch.cuda.stream(side):
                other = torch.sin(other @ other)
        at = [[t.data_ptr() + i * rows * cols * t.element_size() for i in range(count)] for t in (p, g, m)]
        pkg.rfast_muon_step(*at, [rows] * count, [cols] * count, param_type=param, grad_type=grad, weight_decay=0.01, workspace=work.data_ptr(), workspace_bytes=need,
                            cuda_stream=torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert int(work[:4].view(torch.int32)) == 0
        want = want or (p, m)
        assert torch.equal(p, want[0]) and torch.equal(m, want[1]), k
