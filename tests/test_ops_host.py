"""Refusals of the training-step operators.  Every one of them is decided on the host before any
device is looked at, so these run without a GPU; the addresses are never followed."""

from __future__ import annotations

import numpy as np
import pytest

A = 1 << 20          # an address nobody reads


def _refused(text, call, *a, **kw):
    from paper_2307_11617_b200.binding import EINVAL, RFastError
    with pytest.raises(RFastError) as ei:
        call(*a, **kw)
    assert ei.value.code == EINVAL and text in str(ei.value), ei.value


def _adamw(**kw):
    import paper_2307_11617_b200 as pkg
    n = kw.pop("numel", [5, 7])
    base = dict(param=[A, A], grad=[A, A], m=[A, A], v=[A, A], numel=n, step=1)
    base.update(kw)
    pkg.rfast_adamw_step(**base)


@pytest.mark.parametrize("text,kw", [
    ("step counts from 1", dict(step=0)),
    ("beta1 and beta2", dict(beta1=1.0)),
    ("beta1 and beta2", dict(beta2=float("nan"))),
    ("beta1 and beta2", dict(beta2=-0.1)),
    ("eps must be", dict(eps=0.0)),
    ("eps must be", dict(eps=1e-60)),
    ("eps must be", dict(eps=float("nan"))),
    ("lr and weight_decay", dict(lr=float("inf"))),
    ("lr and weight_decay", dict(weight_decay=float("nan"))),
    ("numel of tensor 1", dict(numel=[5, -1])),
    ("numel of tensor 0", dict(numel=[1 << 41, 3])),
    ("tensor 1 has a null address", dict(grad=[A, 0])),
    ("tensor 0 has a null address", dict(m=[0, A])),
    ("tensor 0 has a null address", dict(m_scale=[0, A], v_scale=[A, A])),
    ("not aligned", dict(param=[A + 2, A])),
    ("not aligned", dict(param=[A + 1, A], param_type="bf16")),
    ("not aligned", dict(v=[A, A + 1])),
    ("not aligned", dict(m_scale=[A, A + 2], v_scale=[A, A])),
])
def test_adamw_refuses(rfast_lib, text, kw):
    _refused(text, _adamw, **kw)


def test_adamw_c_entry_refuses(rfast_lib):
    """What the binding cannot be made to pass."""
    import ctypes as C
    from paper_2307_11617_b200 import binding as B
    err = C.create_string_buffer(256)
    assert B.lib().rfast_adamw_step(None, None, err, 256) == B.EINVAL and b"null arguments" in err.value
    assert B.lib().rfast_adamw_step(None, None, None, 0) == B.EINVAL
    one = np.ones(1, np.int64)
    a = B._AdamW(1, 0, 0, 32, one.ctypes.data, one.ctypes.data, one.ctypes.data, one.ctypes.data, None, None, None, 1e-3, 0.9, 0.99, 1e-8, 0, 1, None, None)
    assert B.lib().rfast_adamw_step(C.byref(a), None, err, 256) == B.EINVAL and b"null array" in err.value
    for field, value, text in (("state_bits", 16, b"state_bits"), ("param_type", 7, b"unknown type"), ("grad_type", -1, b"unknown type"),
                               ("n_tensors", -1, b"n_tensors")):
        a = B._AdamW(1, 0, 0, 32, *[one.ctypes.data] * 5, None, None, 1e-3, 0.9, 0.99, 1e-8, 0, 1, None, None)
        setattr(a, field, value)
        assert B.lib().rfast_adamw_step(C.byref(a), None, err, 256) == B.EINVAL and text in err.value, err.value


def test_adamw_nothing_to_do_needs_no_device(rfast_lib):
    import paper_2307_11617_b200 as pkg
    pkg.rfast_adamw_step([], [], [], [], [], step=1)
    pkg.rfast_adamw_step([0], [0], [0], [0], [0], step=1)          # an empty tensor has no address


def test_lists_of_unlike_length_are_refused(rfast_lib):
    import paper_2307_11617_b200 as pkg
    with pytest.raises(ValueError):
        pkg.rfast_adamw_step([A], [A, A], [A], [A], [3], step=1)
    with pytest.raises(ValueError):
        pkg.rfast_adamw_step([A], [A], [A], [A], [3], step=1, m_scale=[A])
    with pytest.raises(ValueError):
        pkg.rfast_adamw_step([A], [A], [A], [A], [3], step=1, param_type="f64")
    with pytest.raises(ValueError):
        pkg.rfast_grad_norm([A], [3, 4], 1.0, A, A, A, 16384)


@pytest.mark.parametrize("text,kw", [
    ("neither", dict(d_norm=0, d_scale=0)),
    ("max_norm", dict(max_norm=0.0)),
    ("max_norm", dict(max_norm=float("nan"))),
    ("workspace must be given", dict(workspace=0)),
    ("aligned to 8", dict(workspace=A + 4)),
    ("workspace needs", dict(workspace_bytes=8)),
    ("output is not aligned", dict(d_norm=A + 2)),
    ("numel of tensor 0", dict(numel=[-2, 1])),
    ("tensor 1 has a null address", dict(grad=[A, 0])),
    ("address of tensor 1", dict(grad=[A, A + 1], grad_type="f16")),
])
def test_grad_norm_refuses(rfast_lib, text, kw):
    import paper_2307_11617_b200 as pkg
    base = dict(grad=[A, A], numel=[5, 7], max_norm=1.0, d_norm=A, d_scale=A, workspace=A, workspace_bytes=pkg.GRAD_NORM_WORKSPACE)
    base.update(kw)
    _refused(text, pkg.rfast_grad_norm, **base)


def test_constants_of_the_binding_are_the_headers(rfast_lib, repo_root):
    import os
    import re
    from paper_2307_11617_b200 import binding as B
    text = open(os.path.join(repo_root, "include", "rfast.h")).read()
    assert int(re.search(r"#define RFAST_GRAD_NORM_WORKSPACE (\d+)", text).group(1)) == B.GRAD_NORM_WORKSPACE
    assert int(re.search(r"#define RFAST_ADAMW_BLOCK (\d+)", text).group(1)) == B.ADAMW_BLOCK


# ---- group norm --------------------------------------------------------------------------------------
SHAPE = dict(samples=4, positions=6, channels=12, groups=3)


@pytest.mark.parametrize("text,kw", [
    ("samples and positions", dict(samples=-1)),
    ("samples and positions", dict(positions=1 << 31)),
    ("multiple of groups", dict(groups=5)),
    ("multiple of groups", dict(groups=0)),
    ("multiple of groups", dict(channels=0)),
    ("8192 channels", dict(channels=8193, groups=1)),
    ("2^24 channels", dict(channels=1 << 25, groups=1 << 25)),
    ("multiple of samples_per_set", dict(samples_per_set=3)),
    ("multiple of samples_per_set", dict(samples_per_set=0)),
])
def test_group_norm_refuses_shapes(rfast_lib, text, kw):
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200.binding import EINVAL, RFastError
    shape = {**SHAPE, **kw}
    _refused(text, pkg.rfast_group_norm, A, A, A, A, A, A, **shape)
    _refused(text, pkg.rfast_group_norm_backward, A, A, A, A, A, A, A, A, A, workspace=A, workspace_bytes=1 << 30, **shape)
    with pytest.raises(RFastError) as ei:
        pkg.rfast_group_norm_workspace(backward=True, **shape)
    assert ei.value.code == EINVAL


@pytest.mark.parametrize("text,kw", [
    ("eps must be", dict(eps=0.0)), ("eps must be", dict(eps=float("nan"))), ("eps must be", dict(eps=-1.0)),
    ("x is null", dict(x=0)), ("beta is null", dict(beta=0)), ("rstd is null", dict(rstd=0)),
    ("x is not aligned", dict(x=A + 2)), ("y is not aligned", dict(y=A + 1, type="bf16")), ("gamma is not aligned", dict(gamma=A + 2, type="bf16")),
    ("stride of x is negative", dict(x_strides=(72, -12))), ("strides of y", dict(y_strides=(72, 11))),
    ("strides of y", dict(y_strides=(71, 12))), ("strides of y", dict(y_strides=(12, 47))), ("strides of y", dict(y_strides=(0, 12))),
])
def test_group_norm_refuses_operands(rfast_lib, text, kw):
    import paper_2307_11617_b200 as pkg
    _refused(text, pkg.rfast_group_norm, **{**dict(x=A, gamma=A, beta=A, y=A, mean=A, rstd=A), **SHAPE, **kw})


@pytest.mark.parametrize("text,kw", [
    ("dy is null", dict(dy=0)), ("dgamma is null", dict(dgamma=0)), ("mean is null", dict(mean=0)), ("dx is not aligned", dict(dx=A + 2)),
    ("workspace needs", dict(workspace_bytes=0)), ("workspace needs", dict(workspace=0)), ("workspace needs", dict(workspace=A + 4)),
    ("strides of dx", dict(dx_strides=(60, 12))), ("stride of dy is negative", dict(dy_strides=(-72, 12))),
])
def test_group_norm_backward_refuses_operands(rfast_lib, text, kw):
    import paper_2307_11617_b200 as pkg
    base = dict(dy=A, x=A, gamma=A, beta=A, mean=A, rstd=A, dx=A, dgamma=A, dbeta=A, workspace=A, workspace_bytes=1 << 30)
    _refused(text, pkg.rfast_group_norm_backward, **{**base, **SHAPE, **kw})


def test_group_norm_of_nothing_needs_no_device(rfast_lib):
    import paper_2307_11617_b200 as pkg
    pkg.rfast_group_norm(0, 0, 0, 0, 0, 0, **{**SHAPE, "samples": 0})
    pkg.rfast_group_norm(0, 0, 0, 0, 0, 0, **{**SHAPE, "positions": 0})
    pkg.rfast_group_norm_backward(0, 0, 0, 0, 0, 0, 0, 0, 0, **{**SHAPE, "samples": 0})
    assert pkg.rfast_group_norm_workspace(**SHAPE) == 0
    assert pkg.rfast_group_norm_workspace(backward=True, **SHAPE) > 0


def test_unknown_names_are_refused(rfast_lib):
    import paper_2307_11617_b200 as pkg
    with pytest.raises(ValueError):
        pkg.rfast_group_norm(A, A, A, A, A, A, act="gelu", **SHAPE)
    with pytest.raises(ValueError):
        pkg.rfast_group_norm(A, A, A, A, A, A, type="f64", **SHAPE)


def test_group_norm_gradient_formula_against_differences():
    """The backward formula that the GPU tests compare with, against central differences of the forward one."""
    from group_norm_reference import backward, forward
    rng = np.random.default_rng(0)
    n, s, c, g, sets = 4, 5, 6, 3, 2
    for act in ("none", "relu", "silu"):
        x, dy = rng.standard_normal((n, s, c)), rng.standard_normal((n, s, c))
        gamma, beta = 1 + 0.3 * rng.standard_normal((sets, c)), 0.3 * rng.standard_normal((sets, c))
        y, mean, rstd, _ = forward(x, gamma, beta, g, 1e-3, act)
        dx, dgamma, dbeta = backward(dy, x, gamma, beta, mean, rstd, g, act)[:3]
        f = lambda *a: (dy * forward(*a, g, 1e-3, act)[0]).sum()  # noqa: E731
        for got, k in ((dx, 0), (dgamma, 1), (dbeta, 2)):
            args = [x, gamma, beta]
            for at in np.ndindex(*args[k].shape):
                h = np.zeros_like(args[k])
                h[at] = 1e-6
                up, down = [a.copy() for a in args], [a.copy() for a in args]
                up[k] += h
                down[k] -= h
                # differences of step 1e-6 carry 1e-6^2 of curvature and 1e-16 / 1e-6 of rounding
                assert abs((f(*up) - f(*down)) / 2e-6 - got[at]) < 1e-7 * (1 + abs(got[at])) * 10, (act, k, at)


# ---- the engine's options -----------------------------------------------------------------------------
@pytest.mark.parametrize("name,ov,text", [
    ("quad_tree64", dict(p=16, K=2, descent={"kind": "adamw"}), "plain descent only"),
    ("softmax_exp16", dict(n=4, F=8, C=3, rows=8, K=2, batch=2, descent={"kind": "adamw", "beta1": 1.0}), "beta1 and beta2"),
    ("softmax_exp16", dict(n=4, F=8, C=3, rows=8, K=2, batch=2, descent={"kind": "adamw8", "eps": 0.0}), "adam_eps"),
    ("softmax_exp16", dict(n=4, F=8, C=3, rows=8, K=2, batch=2, descent={"kind": "adamw8", "weight_decay": float("inf")}), "weight_decay"),
    ("mlp_tree64", dict(n=3, F=16, H=128, C=3, rows=64, K=2, batch=64, norm_groups=3), "divide n_hidden"),
])
def test_engine_refuses_options(rfast_lib, name, ov, text):
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200.binding import EINVAL
    from workloads import build_config
    wl = build_config(name, seed=0, **ov)
    with pytest.raises(pkg.RFastError) as ei:
        pkg.Engine(wl)
    assert ei.value.code == EINVAL and text in str(ei.value)


def test_only_the_mlp_has_a_norm(rfast_lib):
    import paper_2307_11617_b200 as pkg
    from workloads import build_config
    wl = build_config("softmax_exp16", seed=0, n=4, F=8, C=3, rows=8, K=2, batch=2)
    wl.dims["norm_groups"] = 1
    with pytest.raises(pkg.RFastError) as ei:
        pkg.Engine(wl)
    assert "hidden layer" in str(ei.value)


@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("groups", [1, 3, 6])
def test_oracle_normalised_mlp_gradient_against_differences(groups, act):
    from oracle.models import MLP
    rng = np.random.default_rng(groups)
    F, H, C = 4, 6, 3
    feat, lab = rng.standard_normal((1, 5, F)), rng.integers(0, C, (1, 5))
    m = MLP(feat, lab, H, C, l2=0.1, round_inputs=False, norm_groups=groups, norm_act=act, norm_eps=1e-3)
    x = rng.standard_normal(H * F + H + C * H + C + 2 * H)
    idx = np.arange(5)
    g = m.grad(0, x, idx)
    for k in range(len(x)):
        e = np.zeros_like(x)
        e[k] = 1e-6
        diff = (m.loss(0, x + e, idx) - m.loss(0, x - e, idx)) / 2e-6
        # curvature 1e-12 and rounding 1e-16 / 1e-6, the loss's third derivative up to 1e3
        assert abs(diff - g[k]) <= 1e-7 * (1 + abs(g[k])), k


def test_oracle_adamw_step_is_the_definition():
    """Two steps of one worker without neighbours, moments in 64 and in 8 bits, written out."""
    from oracle.rfast_oracle import RFastOracle, _held8
    from workloads import graph_from_edges
    rng = np.random.default_rng(1)
    p, lr = 700, 0.01
    for kind in ("adamw", "adamw8"):
        d = {"kind": kind, "beta1": 0.8, "beta2": 0.95, "eps": 1e-6, "weight_decay": 0.1}
        orc = RFastOracle(1, p, lr, graph_from_edges(1, [], "row"), graph_from_edges(1, [], "col"), lambda i, x, idx: 3.0 * x, np.ones((1, p)), descent=d)
        orc.init_gradients()
        z = rng.standard_normal(p)
        orc.z[0] = z.copy()
        m, s, x = np.zeros(p), np.zeros(p), np.ones(p)
        for t in (1, 2):
            zt = orc.z[0].copy()
            m, s = 0.8 * m + 0.2 * zt, 0.95 * s + 0.05 * zt * zt
            x = x - lr * 0.1 * x - lr * (m / (1 - 0.8 ** t)) / (np.sqrt(s / (1 - 0.95 ** t)) + 1e-6)
            orc.activate(0, t - 1, [], [], None)
            assert np.allclose(orc.x[0], x, rtol=1e-12)
            if kind == "adamw8":
                mq, sq = _held8(m, 0.0), _held8(np.sqrt(s), 2.0 ** -9) ** 2
                assert np.all(np.abs(mq - m) <= 2.0 ** -4 * np.maximum(np.abs(m), np.abs(mq)) + np.abs(m).max() * 2.0 ** -10 / 448)
                m, s = mq, sq
            assert np.allclose(orc.m[0], m, rtol=1e-12) and np.allclose(orc.s[0], s, rtol=1e-12)      # roundings of 64 bits
            m, s = orc.m[0], orc.s[0]


@pytest.mark.parametrize("kw", [dict(x_strides=(72, 16)), dict(y_strides=(80, 12)), dict(x_strides=(0, 12)), dict(x_strides=(12, 48)), dict(positions=1, y_strides=(16, 12)),
                                dict(samples=1, x_strides=(72, 0))])
def test_results_in_place_want_the_operands_strides(rfast_lib, kw):
    """y may be x, dx may be x or dy, in the same strides; in others a value would be overwritten before it is read."""
    import paper_2307_11617_b200 as pkg
    _refused("y is x", pkg.rfast_group_norm, **{**dict(x=A, gamma=A, beta=A, y=A, mean=A, rstd=A), **SHAPE, **kw})
    back = {{"y_strides": "dx_strides"}.get(k, k): v for k, v in kw.items()}
    base = dict(dy=A + 4096, x=A, gamma=A, beta=A, mean=A, rstd=A, dx=A, dgamma=A, dbeta=A, workspace=A, workspace_bytes=1 << 30)
    _refused("dx is x or dy", pkg.rfast_group_norm_backward, **{**base, **SHAPE, **back})
    back = {{"x_strides": "dy_strides"}.get(k, k): v for k, v in back.items()}
    _refused("dx is x or dy", pkg.rfast_group_norm_backward, **{**base, "dy": A, "x": A + 4096, **SHAPE, **back})


@pytest.mark.parametrize("kw", [dict(), dict(x_strides=(72, 12)), dict(samples=1, x_strides=(5, 12)), dict(positions=1, x_strides=(12, 7))])
def test_results_in_place_with_the_operands_strides_pass(rfast_lib, kw):
    """Equal strides, and unlike ones along a dimension of one, go on to the next check."""
    import paper_2307_11617_b200 as pkg
    _refused("rstd is null", pkg.rfast_group_norm, **{**dict(x=A, gamma=A, beta=A, y=A, mean=A, rstd=0), **SHAPE, **kw})
    base = dict(dy=A, x=A, gamma=A, beta=A, mean=A, rstd=0, dx=A, dgamma=A, dbeta=A, workspace=A, workspace_bytes=1 << 30)
    _refused("rstd is null", pkg.rfast_group_norm_backward, **{**base, **SHAPE, **kw})


@pytest.mark.parametrize("strides", [(1 << 62, 1 << 62), (0, 1 << 61), (1 << 61, 12), (12, (1 << 63) - 1)])
def test_strides_beyond_any_memory_are_refused(rfast_lib, strides):
    """Offsets that leave 64 bits wrap round to small ones: the host must not take them for rows that lie apart."""
    import paper_2307_11617_b200 as pkg
    for which in ("x", "y"):
        _refused(f"strides of {which} reach beyond", pkg.rfast_group_norm,
                 **{**dict(x=A, gamma=A, beta=A, y=2 * A, mean=A, rstd=0), **SHAPE, f"{which}_strides": strides})
    base = dict(dy=A, x=2 * A, gamma=A, beta=A, mean=A, rstd=0, dx=3 * A, dgamma=A, dbeta=A, workspace=A, workspace_bytes=1 << 30)
    for which in ("x", "dy", "dx"):
        _refused(f"strides of {which} reach beyond", pkg.rfast_group_norm_backward, **{**base, **SHAPE, f"{which}_strides": strides})


@pytest.mark.parametrize("kw", [dict(d_step=A + 4), dict(d_step=A + 1), dict(d_grad_scale=A + 2), dict(d_step=A, d_grad_scale=A + 1)])
def test_adamw_refuses_misaligned_scalars(rfast_lib, kw):
    """The kernel reads 8 and 4 bytes there: off their alignment that is a fault on the device, and the host's to refuse."""
    _refused("d_step or d_grad_scale is not aligned", _adamw, **kw)


def test_strides_of_nothing_are_not_compared(rfast_lib):
    """Without positions nothing is read or written but dgamma and dbeta: null operands in any strides are no results in place."""
    import paper_2307_11617_b200 as pkg
    _refused("dgamma is null", pkg.rfast_group_norm_backward, 0, 0, 0, 0, 0, 0, 0, 0, 0, x_strides=(5, 7), dx_strides=(9, 9), **{**SHAPE, "positions": 0})
