"""That every value enters the sums of the group norm, once, and bounds that count the additions a value really goes through.

Worst-case bounds of a sum over S positions hide a position that is left out where S is large.  Here
  * the backward sums are of whole numbers (mean 0, rstd 1, no activation), exact in fp32: dgamma and dbeta have to be equal;
  * one value of a group stands out and is moved through all positions: without it the statistics would be another group's;
  * mean, rstd and y are held to the length of the chains that the routes build."""

from __future__ import annotations

import numpy as np
import pytest

from group_norm_reference import forward
from test_gpu_group_norm import EPS, HALF, LONG, SHAPES, TINY, U, _Case, _check_backward, _check_forward, _np, _torch

pytestmark = pytest.mark.gpu

ROWS = {                                                     # 16-bit rows with four accesses per lane, f32 with four
    "264 a group": (33, 1, 1056, 4, 3),
    "520 a group": (20, 1, 1040, 2, 1),
    "1016 a group": (9, 1, 1016, 1, 1),
    "1024 a group": (70, 1, 2048, 2, 2),
    "many rows of 512": (3000, 1, 512, 1, 1),
    "many rows of 272": (1500, 1, 816, 3, 1500),
}
MORE = {
    "samples at the border of one slab, below": (31, 65, 96, 32, 1),
    "samples at the border of one slab": (32, 65, 96, 32, 1),
    "kept whole, many": (300, 30, 48, 4, 3),
    "kept whole, wide": (40, 4, 512, 16, 2),
    "read twice": (7, 20, 6000, 1, 7),
    "two samples, many chunks": (2, 3001, 24, 3, 1),
}
ALL = {**SHAPES, **ROWS, **MORE}


def _positions_of_a_thread(c, backward):
    """(positions that a thread adds up one after the other, channels of an access) for contiguous operands: the rules of the launch."""
    es = 4 if c.kind == "f32" else 2
    cg, v = c.c // c.g, 16 // es
    broad = cg * es >= 128
    while (cg if broad else c.c) % v:
        v //= 2
    if v * es == 8:
        v //= 2
    gs = 1
    if not broad:
        unit = next(k for k in range(1, c.g + 1) if k * cg % v == 0)
        gs = next((k for k in range(unit, c.g, unit) if k * cg * es >= 128), c.g)
        if c.n >= 32 and c.s > 1 and c.g % gs and c.c * es < 256:
            gs = c.g
    w, slabs = gs * cg, -(-c.g // gs)
    ty = 256 // min(w // v, 256)
    item, items = c.s * w * es, c.n * slabs
    chunks = 1
    if not (c.s < 64 or (item <= (32 if backward else 64) * 1024 and (items >= 148 or item <= 16 * 1024))):
        at_a_time = (2 if backward else 4 if cg % v == 0 else 2) * 148
        chunks = max(1, min(at_a_time // items, item // 8192, c.s // 32))
    return -(-(-(-c.s // chunks)) // min(c.s, ty)), v


def _whole_numbers(c, seed):
    """x and dy without a zero among them, scales that are powers of two."""
    torch, dt = _torch()
    rng = np.random.default_rng(seed)
    pick = lambda values, shape: rng.choice(np.array(values, np.float64), shape)  # noqa: E731
    c.x, c.dy = c.put(pick([-2, -1, 1, 2], (c.n, c.s, c.c))), c.put(pick([-3, -2, -1, 1, 2, 3], (c.n, c.s, c.c)))
    c.gamma = torch.as_tensor(pick([-1, 0.5, 1, 2], (c.sets, c.c)), dtype=torch.float32).cuda()
    c.beta = torch.zeros(c.sets, c.c, device="cuda")


@pytest.mark.parametrize("pad", [0, 3], ids=["tight", "odd stride"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", list(ALL))
def test_backward_sums_hold_every_value_once(rfast_lib, shape, kind, pad):
    """dx: the two group sums are exact, 1 / M, its products and the sums are 4 u of the terms."""
    torch, _ = _torch()
    c = _Case(ALL[shape], kind, seed=1, pad=pad)
    _whole_numbers(c, len(shape))
    mean, rstd = torch.zeros(c.n, c.g, device="cuda"), torch.ones(c.n, c.g, device="cuda")
    dx, dgamma, dbeta = c.backward("none", mean, rstd)
    x, dy = c.x.double(), c.dy.double()
    per = lambda t: t.reshape(c.sets, -1, c.c).sum(1)  # noqa: E731
    assert torch.equal(dbeta.double(), per(dy)) and torch.equal(dgamma.double(), per(dy * x))
    dh = dy * c.gamma.double().repeat_interleave(c.n // c.sets, 0)[:, None, :]
    group = lambda t: t.reshape(c.n, c.s, c.g, -1).mean((1, 3)).repeat_interleave(c.c // c.g, 1)[:, None, :]  # noqa: E731
    one, two = group(dh), group(dh * x)
    want = dh - one - x * two
    tol = 6 * U * (one.abs() + (x * two).abs()) + 2 * U * dh.abs()
    tol += HALF[kind] * (want.abs() + tol) + TINY[kind]
    assert bool(((dx.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape", list(ALL))
def test_statistics_hold_every_position(rfast_lib, shape, kind):
    """One value of 1024 among zeros, in another place in every group: mean 1024 / M, and a variance to match.  Both come from sums of whole
    numbers and a few roundings, far from the 1e-4 that they are held to, and left out or counted twice it would be seen."""
    import paper_2307_11617_b200 as pkg
    torch, dt = _torch()
    n, s, ch, g, sets = ALL[shape]
    cg, m = ch // g, s * (ch // g)
    shape_of = dict(samples=n, positions=s, channels=ch, groups=g, type=kind, act="none")
    x, y = torch.zeros(n, s, ch, dtype=dt[kind], device="cuda"), torch.empty(n, s, ch, dtype=dt[kind], device="cuda")
    gamma, beta, stats = torch.ones(ch, device="cuda"), torch.zeros(ch, device="cuda"), torch.empty(2, n, g, device="cuda")
    need = pkg.rfast_group_norm_workspace(**shape_of)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    mean = 1024.0 / m
    rstd = (1024.0 * mean - mean * mean + EPS) ** -0.5
    groups = torch.arange(n * g, device="cuda")
    worst = torch.zeros(2, device="cuda")
    calls = max(-(-s // (n * g)), min(cg, 40))
    for k in range(calls):
        at = (k * n * g + groups) % s, (groups * 5 + k * max(1, cg // 40)) % cg
        where = ((groups // g) * s + at[0]) * ch + (groups % g) * cg + at[1]
        x.view(-1)[where] = 1024.0
        pkg.rfast_group_norm(x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), y.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(), eps=EPS,
                             workspace=work.data_ptr(), workspace_bytes=need, cuda_stream=torch.cuda.current_stream().cuda_stream, **shape_of)
        worst = torch.maximum(worst, torch.stack([(stats[0] / mean - 1).abs().max(), (stats[1] / rstd - 1).abs().max()]))
        x.view(-1)[where] = 0.0
    if m == 1:
        assert bool((stats[0] == 1024).all())               # a group of one: no spread
    else:
        assert bool((worst <= 1e-4).all()), worst


CASES = [(s, k) for s in ALL for k in ("f32", "bf16", "f16") if s not in LONG or k != "f16"]


@pytest.mark.parametrize("shape,kind", CASES, ids=["-".join(c) for c in CASES])
def test_statistics_within_the_chains_of_the_routes(rfast_lib, shape, kind):
    """As the bounds of the other file, with the additions that a value really goes through: those of its thread, then at most 64 of a
    lane over the block's entries, 5 between lanes, and as many again over the chunks."""
    c = _Case(ALL[shape], kind, seed=len(shape) + 1)
    got = c.forward("none")
    rows, v = _positions_of_a_thread(c, False)
    k = min(c.s + 64, rows * max(1, v // 2) + 100)
    x = _np(c.x)
    y, mean, rstd, _ = forward(x, _np(c.gamma), _np(c.beta), c.g, EPS, "none")
    dev = np.abs(x.reshape(c.n, c.s, c.g, -1) - mean[:, None, :, None]).max((1, 3))
    e_mean = 2 * dev * k * U + 4 * U * np.abs(mean)
    e_rstd = rstd * (4 * k * U * dev ** 2 * rstd ** 2 + 2 * U)
    assert np.all(np.abs(_np(got[1]) - mean) <= e_mean + 2.0 ** -149)
    assert np.all(np.abs(_np(got[2]) - rstd) <= e_rstd + rstd * (e_mean * rstd) ** 2 + U * rstd)
    wide = lambda q: np.repeat(q, c.c // c.g, axis=1)[:, None, :]  # noqa: E731
    ga, be = (np.abs(np.repeat(_np(t), c.n // c.sets, axis=0))[:, None, :] for t in (c.gamma, c.beta))
    h = np.abs((x - wide(mean)) * wide(rstd))
    tol = ga * (wide(e_mean * rstd) + h * wide(e_rstd / rstd) + 4 * U * h) + 2 * U * (ga * h + be) + 8 * U * np.abs(y)
    tol += HALF[kind] * (np.abs(y) + tol) + TINY[kind]
    assert np.all(np.abs(_np(got[0]) - y) <= tol)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", list(ROWS) + list(MORE))
def test_more_shapes_and_their_gradients(rfast_lib, shape, kind, act):
    import torch
    c = _Case(ALL[shape], kind, seed=2 * len(shape))
    if act == "relu":                                        # no slope at 0: no gradient comes in near it
        u = forward(_np(c.x), _np(c.gamma), _np(c.beta), c.g, EPS, act)[3]
        c.dy[torch.as_tensor(np.abs(u) < 1e-3).cuda()] = 0
    got = c.forward(act)
    _check_forward(c, act, got)
    _check_backward(c, act, got[1], got[2], c.backward(act, got[1], got[2]))


def test_an_outlier_in_front_costs_few_digits(rfast_lib):
    """800 positions of 32 channels a group, the first position at 1000 among values near 0.  12 chunks, 32 rows of threads: a thread
    adds up 3 positions of 4 channels, and where the outlier is its first value 8 deviations of 1000 in 12, squares and sums of which
    are off by 30 u of 8e6.  8 threads of a group have it, and the sum of all squares is 3.2e7: 8 * 30 u * 8e6 / 3.2e7 = 3.6e-6 of the
    variance, half of it in rstd.  The mean is off by 12 u of 1000 in those threads, 8 of 2134."""
    c = _Case((1, 800, 64, 2, 1), "f32", seed=8)
    c.x[:, 0] = 1000.0
    assert _positions_of_a_thread(c, False) == (3, 4)
    y, mean, rstd = (_np(t) for t in c.forward("none"))
    want = forward(_np(c.x), _np(c.gamma), _np(c.beta), c.g, EPS, "none")
    assert np.all(np.abs(rstd / want[2] - 1) <= 1e-5)
    assert np.all(np.abs(mean - want[1]) <= 1e-4 * 12 / 100 + 100 * U * np.abs(want[1]))
    # half of the variance's error, the mean's share of a spread of 35, and 8 u
    assert np.all(np.abs(y - want[0]) <= 2e-5 * np.abs(want[3]) + 1e-6 + 8 * U * np.abs(_np(c.beta)))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ["long", "long, wide groups", "ten a group", "long, sets", "two samples, many chunks", "ragged slab, many long samples"])
def test_chunks_of_positions_outermost_in_memory(rfast_lib, shape, kind):
    """Samples interleaved with positions, cut into chunks: the same bits as contiguous samples."""
    torch, _ = _torch()
    c = _Case(ALL[shape], kind, seed=23)
    near = c.forward("silu")
    back = c.backward("silu", near[1], near[2])
    swap = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    x, dy = swap(c.x), swap(c.dy)
    assert c.n == 1 or x.stride(1) > x.stride(0)
    far = c.forward("silu", out=torch.full_like(x, 7.0), x=x)
    assert all(torch.equal(a, b) for a, b in zip(near, far))
    far = c.backward("silu", near[1], near[2], out=torch.full_like(x, 7.0), dy=dy, x=x)
    assert all(torch.equal(a, b) for a, b in zip(back, far))
    far = c.backward("silu", near[1], near[2], out=dy, dy=dy, x=x)
    assert all(torch.equal(a, b) for a, b in zip(back, far))


EXTREME = {
    "most runs of groups, one position": (1, 1, 32 * 65534, 65534, 1),
    "most runs of groups": (2, 3, 32 * 65534, 65534, 2),
    "most sets, one position": (65535, 1, 16, 2, 65535),
    "most sets": (65535, 3, 16, 2, 65535),
    "most channels": (1, 2, 1 << 24, 2048, 1),
    "many rows": (300_001, 1, 24, 3, 1),
}


@pytest.mark.parametrize("shape", list(EXTREME))
def test_the_largest_counts(rfast_lib, monkeypatch, shape):
    """As many runs of groups, sets and channels as the header allows: sums and statistics as elsewhere."""
    monkeypatch.setitem(ALL, shape, EXTREME[shape])
    test_backward_sums_hold_every_value_once(rfast_lib, shape, "f32", 0)
    test_statistics_hold_every_position(rfast_lib, shape, "f32")


def test_one_more_is_refused(rfast_lib):
    import paper_2307_11617_b200 as pkg
    torch, _ = _torch()
    d = torch.zeros(64, device="cuda").data_ptr()             # nothing is read: the call is refused
    for shape, text in ((dict(samples=65536, positions=1, channels=16, groups=2, samples_per_set=1), "too many groups or sets"),
                        (dict(samples=1, positions=2, channels=32 * 65535, groups=65535, samples_per_set=1), "too many groups or sets")):
        need = pkg.rfast_group_norm_workspace(backward=True, **shape)
        work = torch.empty(need, dtype=torch.uint8, device="cuda")
        with pytest.raises(pkg.RFastError) as ei:
            pkg.rfast_group_norm_backward(d, d, d, d, d, d, d, d, d, workspace=work.data_ptr(), workspace_bytes=need, **shape)
        assert text in str(ei.value)
