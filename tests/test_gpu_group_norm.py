"""Group norm with an activation, forward and backward, against 64 bits.

u = 2^-24.  A thread adds up at most S positions one after the other, the rest of a sum is a tree of
fewer than 64 additions: k = S + 64 bounds the additions a term goes through.  With D the largest
deviation from a group's mean (a thread's first value is 2 D from another at most):
  mean   off by 2 D k u, and 4 u of itself
  rstd   half the variance's relative error, which the cancellation against the first value makes 8 k u (D / std)^2 at
         most, and 2 u
  the value before the activation: gamma (dmean rstd + |h| drstd / rstd + 4 u |h|) + 2 u (|gamma h| + |beta|)
  the activation: slopes of 1.1 at most, 8 u of its value; then half a step of the type.
Backward, mean and rstd given: h is off by 2 u of itself, the value before the activation by 4 u (|gamma h| + |beta|),
its slope by half of that (second derivatives are 0.5 at most) and 8 u; sums by k' = S + samples + 64 additions."""

from __future__ import annotations

import numpy as np
import pytest

from group_norm_reference import backward, forward

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
EPS = 1e-5

#        samples, positions, channels, groups, sets
SHAPES = {
    "single": (1, 1, 1, 1, 1),
    "one position": (5, 1, 32, 4, 1),
    "one channel a group": (3, 4, 16, 16, 1),
    "odd": (3, 7, 15, 5, 3),
    "hidden layer": (96, 1, 512, 16, 12),
    "hidden layer, one set": (200, 1, 384, 8, 1),
    "hidden layer, many rows": (3001, 1, 256, 8, 1),
    "hidden layer, twenty a group": (70, 1, 120, 6, 2),
    "hidden layer, wide groups": (33, 1, 1000, 2, 3),
    "hidden layer, one row a set": (6, 1, 64, 2, 6),
    "hidden layer, narrow groups": (130, 1, 72, 9, 2),
    "three a group": (2, 50, 96, 32, 1),
    "ten a group": (2, 330, 320, 32, 2),
    "ragged slab": (2, 19, 200, 25, 1),
    "ragged slab, few positions": (7, 3, 200, 25, 1),
    "prime groups": (2, 5, 309, 103, 1),
    "ragged slab, many samples": (40, 19, 200, 25, 2),
    "three a group, many samples": (40, 70, 96, 32, 1),
    "prime groups, many samples": (33, 5, 309, 103, 1),
    "ragged slab, many long samples": (36, 1100, 200, 25, 1),
    "twenty a group": (2, 301, 40, 2, 1),
    "long": (1, 5001, 128, 32, 1),
    "long, wide groups": (2, 4000, 256, 2, 1),
    "long, sets": (4, 1300, 64, 4, 2),
    "many of middle length": (200, 81, 64, 8, 4),
    "wide group": (2, 3, 8192, 1, 1),
    "wide odd group": (2, 9, 4097, 1, 2),
    "wide group, too large to keep": (2, 20, 8192, 1, 2),
    "very long": (1, 40_003, 64, 8, 1),
    "very long, wide odd group": (1, 700, 4097, 1, 1),
    "seventeen positions": (9, 17, 64, 4, 3),
}
LONG = ("very long", "very long, wide odd group", "ragged slab, many long samples")


def _torch():
    import torch
    return torch, {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class _Case:
    def __init__(self, shape, kind, seed, pad=0, lead=0):
        torch, dt = _torch()
        self.n, self.s, self.c, self.g, self.sets = shape
        self.kind, self.pad, self.lead = kind, pad, lead
        rng = np.random.default_rng(seed)
        level, spread = 3 * rng.standard_normal(self.c), 0.2 + rng.random(self.c)
        self.x = self.put(level + spread * rng.standard_normal((self.n, self.s, self.c)))
        self.dy = self.put(rng.standard_normal((self.n, self.s, self.c)))
        self.gamma = torch.as_tensor(1 + 0.3 * rng.standard_normal((self.sets, self.c)), dtype=torch.float32).cuda()
        self.beta = torch.as_tensor(0.3 * rng.standard_normal((self.sets, self.c)), dtype=torch.float32).cuda()

    def room(self):
        torch, dt = _torch()
        flat = torch.full((self.lead + self.n * self.s * (self.c + self.pad) + 8,), 7.0, dtype=dt[self.kind], device="cuda")
        return flat[self.lead:self.lead + self.n * self.s * (self.c + self.pad)].view(self.n, self.s, self.c + self.pad)[:, :, :self.c]

    def put(self, v):
        torch, _ = _torch()
        t = self.room()
        t.copy_(torch.as_tensor(v).cuda())
        return t

    def shape(self, act):
        return dict(samples=self.n, positions=self.s, channels=self.c, groups=self.g, samples_per_set=self.n // self.sets, type=self.kind, act=act)

    def forward(self, act, out=None, stream=0, x=None):
        import paper_2307_11617_b200 as pkg
        torch, _ = _torch()
        x = self.x if x is None else x
        y = self.room() if out is None else out
        stats = torch.full((2, self.n, self.g), 7.0, device="cuda")
        need = pkg.rfast_group_norm_workspace(**self.shape(act))
        work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")         # NaNs: only what was written may be read
        torch.cuda.synchronize()
        pkg.rfast_group_norm(x.data_ptr(), self.gamma.data_ptr(), self.beta.data_ptr(), y.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(), eps=EPS,
                             x_strides=x.stride()[:2], y_strides=y.stride()[:2], workspace=work.data_ptr(), workspace_bytes=need, cuda_stream=stream,
                             **self.shape(act))
        torch.cuda.synchronize()
        return y, stats[0], stats[1]

    def backward(self, act, mean, rstd, out=None, stream=0, dy=None, x=None):
        import paper_2307_11617_b200 as pkg
        torch, _ = _torch()
        dy, x = self.dy if dy is None else dy, self.x if x is None else x
        dx = self.room() if out is None else out
        da = torch.full((2, self.sets, self.c), 7.0, device="cuda")
        need = pkg.rfast_group_norm_workspace(backward=True, **self.shape(act))
        work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")         # NaNs: only what was written may be read
        torch.cuda.synchronize()
        pkg.rfast_group_norm_backward(dy.data_ptr(), x.data_ptr(), self.gamma.data_ptr(), self.beta.data_ptr(), mean.data_ptr(), rstd.data_ptr(),
                                      dx.data_ptr(), da[0].data_ptr(), da[1].data_ptr(), dy_strides=dy.stride()[:2], x_strides=x.stride()[:2],
                                      dx_strides=dx.stride()[:2], workspace=work.data_ptr(), workspace_bytes=need, cuda_stream=stream, **self.shape(act))
        torch.cuda.synchronize()
        return dx, da[0], da[1]


def _np(t):
    return t.double().cpu().numpy()


def _outside_stands(t):
    """Nothing but the view itself was written."""
    import torch
    base = t._base if t._base is not None else t
    keep = torch.ones(base.numel(), dtype=torch.bool, device="cuda")
    keep[torch.as_strided(torch.arange(base.numel(), device="cuda"), t.size(), t.stride(), t.storage_offset()).reshape(-1)] = False
    return bool((base.reshape(-1)[keep].double() == 7.0).all())


def _check_forward(c, act, got, x=None):
    x = _np(c.x) if x is None else x
    gamma, beta = _np(c.gamma), _np(c.beta)
    y, mean, rstd, u = forward(x, gamma, beta, c.g, EPS, act)
    k = c.s + 64
    q = x.reshape(c.n, c.s, c.g, -1)
    dev = np.abs(q - mean[:, None, :, None]).max((1, 3))
    var = 1 / rstd ** 2 - EPS
    e_mean = 2 * dev * k * U + 4 * U * np.abs(mean)
    e_rstd = rstd * (4 * k * U * dev ** 2 / np.maximum(var + EPS, 1e-300) + 2 * U)
    assert np.all(np.abs(_np(got[1]) - mean) <= e_mean + 2.0 ** -149)
    # a wrong mean adds its square to the variance
    assert np.all(np.abs(_np(got[2]) - rstd) <= e_rstd + rstd * (e_mean * rstd) ** 2 + U * rstd)
    wide = lambda v: np.repeat(v, c.c // c.g, axis=1)[:, None, :]  # noqa: E731
    ga = np.abs(np.repeat(gamma, c.n // c.sets, axis=0))[:, None, :]
    be = np.abs(np.repeat(beta, c.n // c.sets, axis=0))[:, None, :]
    h = np.abs((x - wide(mean)) * wide(rstd))
    e_u = ga * (wide(e_mean * rstd) + h * wide(e_rstd / rstd) + 4 * U * h) + 2 * U * (ga * h + be)
    tol = 1.1 * e_u + 8 * U * np.abs(y)
    tol += HALF[c.kind] * (np.abs(y) + tol) + TINY[c.kind]
    off = np.abs(_np(got[0]) - y)
    assert np.all(off <= tol), (off / tol).max()


def _check_backward(c, act, mean, rstd, got, dy=None, x=None):
    x, dy = _np(c.x) if x is None else x, _np(c.dy) if dy is None else dy
    gamma, beta, mean, rstd = _np(c.gamma), _np(c.beta), _np(mean), _np(rstd)
    dx, dgamma, dbeta, h, u, du = backward(dy, x, gamma, beta, mean, rstd, c.g, act)
    ga = np.abs(np.repeat(gamma, c.n // c.sets, axis=0))[:, None, :]
    be = np.abs(np.repeat(beta, c.n // c.sets, axis=0))[:, None, :]
    e_du = 0 if act != "silu" else np.abs(dy) * (0.5 * 4 * U * (ga * np.abs(h) + be) + 8 * U)
    k = c.s + c.n + 64
    per = lambda v: np.broadcast_to(v, x.shape).reshape(c.sets, -1, c.c).sum(1)  # noqa: E731
    assert np.all(np.abs(_np(got[2]) - dbeta) <= per(e_du + k * U * np.abs(du)) + U * np.abs(dbeta) + 2.0 ** -149)
    assert np.all(np.abs(_np(got[1]) - dgamma) <= per(e_du * np.abs(h) + (k + 3) * U * np.abs(du * h)) + U * np.abs(dgamma) + 2.0 ** -149)
    grp = lambda v: np.repeat(np.broadcast_to(v, x.shape).reshape(c.n, c.s, c.g, -1).mean((1, 3)), c.c // c.g, axis=1)[:, None, :]  # noqa: E731
    rs = np.repeat(rstd, c.c // c.g, axis=1)[:, None, :]
    ah, adu = np.abs(h), np.abs(du)
    one, two = grp(ga * adu), grp(ga * adu * ah)
    e_one = grp(ga * e_du) + (k + 4) * U * one
    e_two = grp(ga * e_du * ah) + (k + 6) * U * two
    tol = rs * (ga * e_du + 6 * U * ga * adu + e_one + ah * e_two + 6 * U * (one + ah * two))
    tol += HALF[c.kind] * (np.abs(dx) + tol) + TINY[c.kind]
    off = np.abs(_np(got[0]) - dx)
    assert np.all(off <= tol), (off / tol).max()


def _away_from_zero(c, act):
    """max(u, 0) has no slope at 0, and either side of it may be taken there: no gradient comes in there."""
    import torch
    if act == "relu":
        u = forward(_np(c.x), _np(c.gamma), _np(c.beta), c.g, EPS, act)[3]
        c.dy[torch.as_tensor(np.abs(u) < 1e-3).cuda()] = 0


CASES = [(s, k, a) for i, s in enumerate(SHAPES) for j, k in enumerate(("f32", "bf16", "f16")) for a in ("none", "relu", "silu")
         if s not in LONG or (j, a) in ((0, "silu"), (1, "relu"), (2, "none"))]


@pytest.mark.parametrize("shape,kind,act", CASES, ids=["-".join(c) for c in CASES])
def test_group_norm_and_its_gradients(rfast_lib, shape, kind, act):
    c = _Case(SHAPES[shape], kind, seed=len(shape))
    _away_from_zero(c, act)
    got = c.forward(act)
    _check_forward(c, act, got)
    assert _outside_stands(got[0])
    back = c.backward(act, got[1], got[2])
    _check_backward(c, act, got[1], got[2], back)
    assert _outside_stands(back[0])


@pytest.mark.parametrize("pad,lead", [(8, 0), (8, 8), (2, 0), (3, 0), (0, 1), (5, 3)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ["odd", "ten a group", "hidden layer", "long", "seventeen positions"])
def test_strides_and_alignment(rfast_lib, shape, kind, pad, lead):
    """Operands inside wider tensors, from any address: what lies around the results stays."""
    c = _Case(SHAPES[shape], kind, seed=2, pad=pad, lead=lead)
    got = c.forward("silu")
    _check_forward(c, "silu", got)
    assert _outside_stands(got[0])
    back = c.backward("silu", got[1], got[2])
    _check_backward(c, "silu", got[1], got[2], back)
    assert _outside_stands(back[0])


@pytest.mark.parametrize("shape", ["hidden layer", "ten a group", "long", "very long", "wide odd group"])
def test_in_place_and_repeated_runs_give_the_same_bits(rfast_lib, shape):
    torch, _ = _torch()
    c = _Case(SHAPES[shape], "bf16", seed=3)
    stream = torch.cuda.Stream()
    a, b = c.forward("silu"), c.forward("silu", stream=stream.cuda_stream)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    x = c.put(_np(c.x))
    inside = c.forward("silu", out=x, x=x)
    assert all(torch.equal(p, q) for p, q in zip(a, inside))
    ga, gb = c.backward("silu", a[1], a[2]), c.backward("silu", a[1], a[2], stream=stream.cuda_stream)
    assert all(torch.equal(p, q) for p, q in zip(ga, gb))
    dy = c.put(_np(c.dy))
    assert all(torch.equal(p, q) for p, q in zip(ga, c.backward("silu", a[1], a[2], out=dy, dy=dy)))
    x = c.put(_np(c.x))
    assert all(torch.equal(p, q) for p, q in zip(ga, c.backward("silu", a[1], a[2], out=x, x=x)))


def test_positions_of_another_order_and_repeated_ones(rfast_lib):
    """Samples interleaved with positions; one position read for all (stride 0)."""
    import paper_2307_11617_b200 as pkg
    torch, _ = _torch()
    c = _Case((4, 30, 24, 3, 1), "f32", seed=5)
    swapped = c.x.transpose(0, 1).contiguous().transpose(0, 1)              # positions outermost in memory
    y = torch.full((30, 4, 24), 7.0, device="cuda").transpose(0, 1)
    got = c.forward("silu", out=y, x=swapped)
    _check_forward(c, "silu", got)
    one = c.x[:, :1].expand(4, 30, 24)
    got = c.forward("none", x=one)
    _check_forward(c, "none", got, x=_np(one))
    back = c.backward("none", got[1], got[2], x=one)
    _check_backward(c, "none", got[1], got[2], back, x=_np(one))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("shape,kind", [("ten a group", "f32"), ("hidden layer", "f32"), ("long", "f32"), ("one channel a group", "bf16"),
                                        ("three a group", "bf16"), ("prime groups", "f16")])
def test_bad_values_stay_in_their_group(rfast_lib, shape, kind, bad):
    c = _Case(SHAPES[shape], kind, seed=6)
    good = [_np(t) for t in c.forward("silu")]
    n, s, ch = c.n - 1, c.s // 2, c.c // 2
    c.x[n, s, ch] = bad
    hurt = [_np(t) for t in c.forward("silu")]
    w = c.c // c.g
    g = ch // w
    hit = np.zeros(good[0].shape, bool)
    hit[n, :, g * w:(g + 1) * w] = True
    assert np.array_equal(good[0][~hit], hurt[0][~hit]) and np.isnan(hurt[0][hit]).all()
    rows = np.zeros(good[1].shape, bool)
    rows[n, g] = True
    for a, b in ((good[1], hurt[1]), (good[2], hurt[2])):
        assert np.array_equal(a[~rows], b[~rows]) and not np.isfinite(b[rows]).any()


@pytest.mark.parametrize("shape", ["one channel a group", "ten a group", "hidden layer", "long", "seventeen positions"])
def test_a_bad_shift_stays_in_its_channel(rfast_lib, shape):
    """A NaN in one channel's beta reaches that channel's values alone, forward and backward."""
    c = _Case(SHAPES[shape], "bf16", seed=16)
    good = [_np(t) for t in c.forward("silu")]
    ch = c.c // 2
    c.beta[0, ch] = np.nan
    hurt = [_np(t) for t in c.forward("silu")]
    hit = np.zeros(good[0].shape, bool)
    hit[:c.n // c.sets, :, ch] = True
    assert np.array_equal(good[0][~hit], hurt[0][~hit]) and np.isnan(hurt[0][hit]).all()
    assert np.array_equal(good[1], hurt[1]) and np.array_equal(good[2], hurt[2])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ["ten a group", "hidden layer", "long", "seventeen positions", "wide odd group"])
def test_slopes_far_from_zero(rfast_lib, shape, kind):
    """Values of hundreds before the activation: its slope there is 1 or 0, however large they are."""
    c = _Case(SHAPES[shape], kind, seed=17)
    c.gamma *= 100.0
    got = c.forward("silu")
    _check_forward(c, "silu", got)
    _check_backward(c, "silu", got[1], got[2], c.backward("silu", got[1], got[2]))


def test_far_levels_and_flat_groups(rfast_lib):
    """A level far above the spread costs no digits of the spread; a constant group gives beta."""
    torch, _ = _torch()
    for level in (1e4, -3e5):
        c = _Case((2, 500, 32, 2, 1), "f32", seed=7)
        c.x += level
        _check_forward(c, "none", c.forward("none"))
    c = _Case((2, 500, 32, 2, 1), "f32", seed=7)
    c.x.fill_(123.456)
    y, mean, rstd = c.forward("none")
    assert torch.equal(y, c.beta[:, None, :].expand_as(y)) and bool((mean == np.float32(123.456)).all())
    assert np.allclose(_np(rstd), EPS ** -0.5, rtol=4 * U)


def test_an_outlier_in_front(rfast_lib):
    """The first value a thread sees is its reference: far out, it must not cost the others their digits."""
    c = _Case((1, 800, 64, 2, 1), "f32", seed=8)
    c.x[:, 0] = 1000.0
    _check_forward(c, "none", c.forward("none"))


def test_recorded_passes_and_side_by_side(rfast_lib):
    """Both passes captured and replayed; two graphs with a workspace each replayed on two streams."""
    import paper_2307_11617_b200 as pkg
    torch, _ = _torch()
    cases = [_Case(SHAPES[name], "f16", seed=k) for k, name in ((11, "ten a group"), (12, "ten a group"), (13, "long"), (14, "long"))]
    want, graphs, outs, streams = [], [], [], []
    for c in cases:
        f = c.forward("silu")
        want.append([*f, *c.backward("silu", f[1], f[2])])
        stream = torch.cuda.Stream()
        y, dx = c.room(), c.room()
        stats, da = torch.zeros(2, c.n, c.g, device="cuda"), torch.zeros(2, c.sets, c.c, device="cuda")
        first, need = (pkg.rfast_group_norm_workspace(backward=b, **c.shape("silu")) for b in (False, True))
        work = torch.empty(first + need, dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            pkg.rfast_group_norm(c.x.data_ptr(), c.gamma.data_ptr(), c.beta.data_ptr(), y.data_ptr(), stats[0].data_ptr(), stats[1].data_ptr(), eps=EPS,
                                 workspace=work.data_ptr(), workspace_bytes=first, cuda_stream=stream.cuda_stream, **c.shape("silu"))
            pkg.rfast_group_norm_backward(c.dy.data_ptr(), c.x.data_ptr(), c.gamma.data_ptr(), c.beta.data_ptr(), stats[0].data_ptr(),
                                          stats[1].data_ptr(), dx.data_ptr(), da[0].data_ptr(), da[1].data_ptr(), workspace=work.data_ptr() + first,
                                          workspace_bytes=need, cuda_stream=stream.cuda_stream, **c.shape("silu"))
        graphs.append(graph)
        outs.append([y, stats[0], stats[1], dx, da[0], da[1], work])
        streams.append(stream)
    for _ in range(5):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(a, b) for a, b in zip(w, o))


@pytest.mark.parametrize("shape", ["hidden layer, one row a set", "seventeen positions", "long, wide groups"])
def test_offsets_beyond_32_bits(rfast_lib, shape):
    """Samples more than 2^31 values apart give what neighbouring ones give."""
    torch, _ = _torch()
    n, s, ch, g, sets = SHAPES[shape]
    c = _Case((2, s, ch, g, 1), "bf16", seed=40)
    apart = 2 ** 31 + 4096
    x, y = (torch.empty(apart + s * ch, dtype=torch.bfloat16, device="cuda").as_strided((2, s, ch), (apart, ch, 1)) for _ in range(2))
    x.copy_(c.x)
    near, far = c.forward("silu"), c.forward("silu", out=y, x=x)
    assert all(torch.equal(p, q) for p, q in zip(near, far))
    near, far = c.backward("silu", near[1], near[2]), c.backward("silu", near[1], near[2], out=y, x=x)
    assert all(torch.equal(p, q) for p, q in zip(near, far))


def test_more_samples_than_a_grid_holds(rfast_lib):
    """Pieces of more than 65535 samples go out in several launches; samples on both sides of the border and the sums over all."""
    torch, _ = _torch()
    n, s, ch, g = 65538, 520, 64, 4
    c = _Case((4, s, ch, g, 1), "bf16", seed=41)
    c.n = n
    torch.manual_seed(5)
    c.x, c.dy = (torch.randn(n, s, ch, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    y = torch.empty_like(c.x)
    got = c.forward("relu", out=y)
    few = [0, 65534, 65535, 65537]
    small = _Case((4, s, ch, g, 1), "bf16", seed=41)
    small.gamma, small.beta, small.x, small.dy = c.gamma, c.beta, c.x[few], c.dy[few]
    _check_forward(small, "relu", [t[few] for t in got])
    back = c.backward("none", got[1], got[2], out=y)
    ref = small.backward("none", got[1][few].contiguous(), got[2][few].contiguous())
    _check_backward(small, "none", got[1][few], got[2][few], (back[0][few], ref[1], ref[2]))
    total, size = (sum(f(c.dy[k:k + 4096].double()).sum((0, 1)) for k in range(0, n, 4096)) for f in (lambda t: t, torch.abs))
    # a thread block adds up a sample's positions in fp32, all else in 64 bits
    assert bool(((back[2][0].double() - total).abs() <= (s + 64) * U * size + U * total.abs()).all())


def test_calls_of_two_threads(rfast_lib):
    """Threads that launch one kernel with buffers of different sizes do not disturb each other."""
    import threading
    torch, _ = _torch()
    cases = [_Case((160, s, 64, 1, 1), "f32", seed=30 + s) for s in (200, 255)]
    want = [[t.clone() for t in c.forward("silu")] for c in cases]
    torch.cuda.synchronize()
    failed = []

    def many(c, w):
        try:
            for _ in range(200):
                got = c.forward("silu")
                if not all(torch.equal(a, b) for a, b in zip(got, w)):
                    raise AssertionError("values differ")
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=many, args=a) for a in zip(cases, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed[0]


def test_no_positions_and_foreign_addresses(rfast_lib):
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200.binding import EINVAL, RFastError
    torch, _ = _torch()
    da = torch.full((2, 2, 12), 7.0, device="cuda")
    pkg.rfast_group_norm_backward(0, 0, 0, 0, 0, 0, 0, da[0].data_ptr(), da[1].data_ptr(), samples=4, positions=0, channels=12, groups=3, samples_per_set=2)
    torch.cuda.synchronize()
    assert not da.any()
    host = np.zeros(1000, np.float32)
    d = torch.zeros(1000, device="cuda").data_ptr()
    with pytest.raises(RFastError) as ei:
        pkg.rfast_group_norm(d, host.ctypes.data, d, d, d, d, samples=2, positions=3, channels=12, groups=3)
    assert ei.value.code == EINVAL and "gamma: not device memory" in str(ei.value)


@pytest.mark.parametrize("shift", [-1e3, -1e12, -1e20, -3e38])
@pytest.mark.parametrize("shape,kind", [("one channel a group", "f32"), ("ten a group", "f16"), ("hidden layer", "f32"), ("hidden layer", "bf16"),
                                        ("hidden layer, wide groups", "f32"), ("long", "bf16"), ("seventeen positions", "f32"), ("wide odd group", "f16")])
def test_values_far_below_zero_vanish(rfast_lib, shape, kind, shift):
    """u / (1 + exp(-u)) and its slope go to 0 on the left, however far u is: a channel whose shift says "off" adds nothing."""
    torch, _ = _torch()
    c = _Case(SHAPES[shape], kind, seed=18)
    ch = c.c // 2
    c.beta[:, ch] = -100.0
    near = c.forward("silu")
    near_back = c.backward("silu", near[1], near[2])
    c.beta[:, ch] = shift
    far = c.forward("silu")
    far_back = c.backward("silu", near[1], near[2])
    # exp(41) = 6e17: the values are of 41.6 / (1 + exp(41.6)) = 3.6e-17 at most, their slopes likewise
    y = _np(far[0])[:, :, ch]
    assert np.all((y <= 0) & (y >= -4e-17))
    for got, by in ((far_back[1], _np(c.dy) * 10), (far_back[2], _np(c.dy))):
        assert np.all(np.abs(_np(got)[:, ch]) <= 4e-17 * np.abs(by[:, :, ch]).sum())
    assert all(torch.equal(a, b) for a, b in zip((*near, *near_back), (*far, *far_back)))


@pytest.mark.parametrize("shape,kind", [("ten a group", "f32"), ("hidden layer", "bf16"), ("long", "f32"), ("seventeen positions", "f16")])
def test_huge_scales_keep_the_sign(rfast_lib, shape, kind):
    """With a scale of 1e30 a value before the activation is far to the right or far to the left: y is itself, or nothing."""
    c = _Case(SHAPES[shape], kind, seed=19)
    c.gamma[:] = 1e30
    c.beta[:] = 0
    y, mean, rstd = (_np(t) for t in c.forward("silu"))
    h = ((_np(c.x).reshape(c.n, c.s, c.g, -1) - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(c.n, c.s, c.c)
    off = h < -1e-3
    assert off.any() and np.all(np.abs(y[off]) <= 4e-17)
    on = h > 1e-3
    with np.errstate(over="ignore"):
        want = h[on] * 1e30
    assert np.all(y[on] == np.inf) if kind == "f16" else np.allclose(y[on], want, rtol=1e-2)
