"""The engine with an AdamW step in the place of S1, and with a group norm in the MLP's hidden layer, against the oracle.

With eps = 1e-3, near the size of the trackers' entries, the adaptive step is smooth where a tracker's entry passes
through zero (its slope is lr / eps at most, not a jump of 2 lr), so that the trajectories are held to the
bars of the plain ones.  8-bit moments: where fp32 and 64 bits leave a moment on different sides of a border between
codes, that entry's next steps differ by up to 2^-4 of themselves; entries whose moments are within 1e-6
of a border are about one in 1e5 per step, so x, which moves by lr of an entry's size per step, is held to 1e-4."""

from __future__ import annotations

import numpy as np
import pytest

from oracle import from_workload, make_model, rel_l2, run_schedule
from workloads import build_config

pytestmark = pytest.mark.gpu

ADAM = {"beta1": 0.9, "beta2": 0.99, "eps": 1e-3, "weight_decay": 0.05}
CASES = {
    "ls": ("ls_ring4", dict(K=60, p=300)),
    "softmax": ("softmax_exp16", dict(n=8, F=48, C=5, rows=64, K=30, batch=8)),
    "logistic": ("logistic_tree1024", dict(n=24, p=3000, rows=8, K=16, batch=4, nnz=60)),
    "mlp": ("mlp_tree64", dict(n=5, F=48, H=256, C=3, rows=96, K=12, batch=64)),
    "mlp norm": ("mlp_tree64", dict(n=5, F=48, H=256, C=3, rows=96, K=12, batch=64, norm_groups=8, norm_act="silu")),
}


def _build(case, kind, seed=3, **more):
    name, ov = CASES[case]
    return build_config(name, seed=seed, **{**ov, "alpha": 0.003, "descent": {"kind": kind, **ADAM}, **more})


def _oracle(wl):
    orc = from_workload(wl, make_model(wl).grad)
    Bs = wl.batch
    orc.init_gradients([wl.schedule.batch_idx[i * Bs:(i + 1) * Bs] for i in range(wl.n)] if Bs else None)
    return orc


@pytest.mark.parametrize("kind", ["adamw", "adamw8"])
@pytest.mark.parametrize("case", list(CASES))
def test_trajectory_against_the_oracle(rfast_lib, case, kind):
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    wl = _build(case, kind)
    orc = _oracle(wl)
    x0, z0 = np.linalg.norm(orc.X()), np.linalg.norm(orc.Z())
    run_schedule(orc, wl.schedule)
    with pkg.Engine(wl) as eng:
        eng.load_schedule(wl.schedule)
        eng.run()
        x, y, m, v = (eng.read(w) for w in (B.STATE_X, B.STATE_Y, B.STATE_ADAM_M, B.STATE_ADAM_V))
        assert eng.read(B.STATE_USED_TAU_V).tolist() == orc.used_tau_v
        d = eng.diagnostics()
    bar = 1e-5 if kind == "adamw" else 1e-4
    assert rel_l2(x, orc.X(), x0) <= bar
    assert rel_l2(y, orc.Z(), z0) <= max(bar, 1e-4 if case.startswith("mlp") else bar)
    # moments: 32 bits as the trackers; 8 bits up to the codes that differ
    assert rel_l2(m, np.stack(orc.m)) <= (1e-4 if kind == "adamw" else 2.0 ** -8)
    assert rel_l2(v, np.stack(orc.s)) <= (1e-4 if kind == "adamw" else 2.0 ** -8)
    # the tracker's mass is conserved whatever the local step does (Lemma 3)
    assert d["conservation_residual"] <= 1e-4 * max(d["gradient_sum_max"], 1e-3 * z0)


@pytest.mark.parametrize("kind", ["adamw", "adamw8"])
@pytest.mark.parametrize("case", ["softmax", "logistic", "mlp norm"])
def test_graphs_streams_and_checkpoints_give_the_same_bits(rfast_lib, case, kind):
    import torch
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    wl = _build(case, kind)
    views = (B.STATE_X, B.STATE_Y, B.STATE_G_LAST, B.STATE_ADAM_M, B.STATE_ADAM_V)
    K = wl.schedule.K
    with pkg.Engine(wl) as eng:
        eng.load_schedule(wl.schedule)
        eng.run()
        want = [eng.read(w) for w in views]
        eng.reset()
        assert not eng.read(B.STATE_ADAM_M).any() and not eng.read(B.STATE_ADAM_V).any()
        eng.run(K // 2)
        blob = eng.checkpoint()
    stream = torch.cuda.Stream()
    with pkg.Engine(wl, stream.cuda_stream) as eng:                  # recorded into graphs, replayed after a reset
        eng.load_schedule(wl.schedule)
        for _ in range(2):
            eng.run()
            assert all(np.array_equal(a, eng.read(w)) for a, w in zip(want, views))
            eng.reset()
        eng.restore(blob)
        eng.run()
        assert all(np.array_equal(a, eng.read(w)) for a, w in zip(want, views))
    other = _build(case, "adamw" if kind == "adamw8" else "adamw8")
    with pkg.Engine(other) as eng:
        eng.load_schedule(other.schedule)
        with pytest.raises(pkg.RFastError):
            eng.restore(blob)


def test_appended_rounds_equal_the_whole(rfast_lib):
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    from workloads import split_schedule
    wl = _build("softmax", "adamw8")
    parts = split_schedule(wl.schedule, wl.G_R, wl.G_C, [wl.schedule.K // 3])
    with pkg.Engine(wl) as eng:
        eng.load_schedule(wl.schedule)
        eng.run()
        want = eng.read(B.STATE_X)
    with pkg.Engine(wl) as eng:
        eng.set_option(B.OPT_OPEN_END, 1)
        eng.load_schedule(parts[0])
        eng.run()
        eng.append_schedule(parts[1])
        eng.run()
        assert np.array_equal(want, eng.read(B.STATE_X))


def test_step_size_of_the_round_and_written_moments(rfast_lib):
    """gamma^t is the step's lr; moments written with rfast_write_state are the ones the next step takes."""
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    wl = _build("softmax", "adamw")
    wl.schedule.alpha_round = np.linspace(0.004, 0.001, wl.schedule.K).astype(np.float32)
    orc = _oracle(wl)
    x0 = np.linalg.norm(orc.X())
    run_schedule(orc, wl.schedule, K=10)
    with pkg.Engine(wl) as eng:
        eng.load_schedule(wl.schedule)
        eng.run(10)
        assert rel_l2(eng.read(B.STATE_X), orc.X(), x0) <= 1e-5
        m, v = eng.read(B.STATE_ADAM_M), eng.read(B.STATE_ADAM_V)
        eng.write(B.STATE_ADAM_M, 2 * m)
        eng.write(B.STATE_ADAM_V, 4 * v)
        assert np.array_equal(eng.read(B.STATE_ADAM_M), 2 * m)
        orc.m, orc.s = [2 * a for a in orc.m], [4 * a for a in orc.s]
        run_schedule(orc, wl.schedule)
        eng.run()
        assert rel_l2(eng.read(B.STATE_X), orc.X(), x0) <= 1e-5


def test_moments_of_other_descents_are_refused(rfast_lib):
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    plain = build_config("softmax_exp16", seed=1, n=4, F=16, C=3, rows=16, K=4, batch=4)
    with pkg.Engine(plain) as eng:
        eng.load_schedule(plain.schedule)
        for call in (lambda: eng.read(B.STATE_ADAM_M), lambda: eng.write(B.STATE_ADAM_V, np.zeros((plain.n, plain.p)))):
            with pytest.raises(pkg.RFastError) as ei:
                call()
            assert ei.value.code == B.ESTATE
    wl = _build("softmax", "adamw8")
    with pkg.Engine(wl) as eng:
        eng.load_schedule(wl.schedule)
        with pytest.raises(pkg.RFastError) as ei:
            eng.write(B.STATE_ADAM_M, np.zeros((wl.n, wl.p)))
        assert ei.value.code == B.ESTATE and "checkpoints" in str(ei.value)


# ---- group norm in the hidden layer -----------------------------------------------------------------
NORMS = [
    dict(n=6, F=64, H=128, C=10, rows=128, K=8, batch=64, norm_groups=4, norm_act="relu"),
    dict(n=5, F=48, H=256, C=3, rows=96, K=8, batch=64, norm_groups=1, norm_act="silu"),
    dict(n=3, F=784, H=512, C=10, rows=128, K=6, batch=64, norm_groups=16, norm_act="silu", l2=1e-2),
    dict(n=4, F=32, H=1152, C=4, rows=64, K=5, batch=64, norm_groups=6, norm_act="none"),
    dict(n=4, F=32, H=128, C=16, rows=64, K=5, batch=64, norm_groups=64, norm_act="relu", l2=1e-3),
    dict(n=70, F=16, H=128, C=7, rows=64, K=4, batch=64, norm_groups=8, norm_act="silu"),
]
IDS = ["H128 G4 relu", "H256 G1 silu", "H512 G16 l2", "H1152 G6 none", "G64 two a group", "n70"]


def _blocks(wl):
    H, F, C = wl.dims["n_hidden"], wl.dims["n_features"], wl.dims["n_classes"]
    at = np.cumsum([0, H * F, H, C * H, C, H, H])
    return {nm: (at[k], at[k + 1]) for k, nm in enumerate(("W1", "b1", "W2", "b2", "gamma", "beta"))}


@pytest.mark.parametrize("ov", NORMS, ids=IDS)
def test_normalised_mlp_gradient_from_identical_state(rfast_lib, ov):
    """As for the plain MLP: all blocks to fp32 accuracy but W1, whose rounding of the computed dpre to bf16 may flip by an
    ulp.  The bias in front of a norm moves a whole group's level in part only: its gradient is what is left of cancelling
    terms (exactly 0 for one group without activation), so b1 is held to 1e-5 of the terms, the size of dgamma."""
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    wl = build_config("mlp_tree64", seed=1, **ov)
    rng = np.random.default_rng(0)
    H = wl.dims["n_hidden"]
    wl.x0 = wl.x0.copy()
    wl.x0[:, -2 * H:] += 0.2 * rng.standard_normal((wl.n, 2 * H)).astype(np.float32)      # each node a scale and shift of its own
    m, Bs = make_model(wl), wl.batch
    with pkg.Engine(wl) as eng:
        eng.load_schedule(wl.schedule)
        g = eng.read(B.STATE_G_LAST)
    ref = np.stack([m.grad(i, wl.x0[i].astype(np.float64), wl.schedule.batch_idx[i * Bs:(i + 1) * Bs]) for i in range(wl.n)])
    blocks = _blocks(wl)
    a, b = blocks["gamma"]
    terms = np.linalg.norm(ref[:, a:b])
    for nm, (a, b) in blocks.items():
        if nm == "b1":
            assert np.linalg.norm(g[:, a:b] - ref[:, a:b]) <= 1e-5 * max(terms, np.linalg.norm(ref[:, a:b])), nm
        else:
            assert rel_l2(g[:, a:b], ref[:, a:b]) <= (1e-4 if nm == "W1" else 1e-5), nm


@pytest.mark.parametrize("ov", NORMS[:3], ids=IDS[:3])
def test_normalised_mlp_trajectory_and_objective(rfast_lib, ov):
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    wl = build_config("mlp_tree64", seed=2, **ov)
    orc = _oracle(wl)
    x0, z0 = np.linalg.norm(orc.X()), np.linalg.norm(orc.Z())
    run_schedule(orc, wl.schedule)
    with pkg.Engine(wl) as eng:
        eng.load_schedule(wl.schedule)
        eng.run()
        x, y = eng.read(B.STATE_X), eng.read(B.STATE_Y)
        d = eng.diagnostics()
    assert rel_l2(x, orc.X(), x0) <= 1e-5 and rel_l2(y, orc.Z(), z0) <= 1e-4
    m = make_model(wl)
    xbar = x.astype(np.float64).mean(axis=0)
    want = sum(m.loss(i, xbar.astype(np.float32).astype(np.float64), np.arange(wl.rows)) for i in range(wl.n))
    assert abs(d["objective"] - want) <= 1e-4 * abs(want)


def test_checkpoints_of_other_moments_or_layers_are_refused(rfast_lib):
    """Moments formed with other betas, or gradients of another hidden layer, are not taken for one's own; a rate, an eps or a decay may change."""
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    wl = _build("mlp norm", "adamw")
    with pkg.Engine(wl) as eng:
        eng.load_schedule(wl.schedule)
        eng.run(4)
        blob = eng.checkpoint()

    def restored(**more):
        descent = {"kind": "adamw", **ADAM, **more.pop("descent", {})}
        other = _build("mlp norm", "adamw", descent=descent, **{k: v for k, v in more.items() if k != "norm_eps"})
        if "norm_eps" in more:
            other.dims["norm_eps"] = more["norm_eps"]
        with pkg.Engine(other) as eng:
            eng.load_schedule(other.schedule)
            x = eng.read(B.STATE_X)
            try:
                eng.restore(blob)
            except pkg.RFastError as e:
                assert e.code == B.EINVAL and np.array_equal(x, eng.read(B.STATE_X))
                return False
            return True

    assert restored()
    assert restored(alpha=0.001) and restored(descent={"eps": 1e-4}) and restored(descent={"weight_decay": 0.0})
    for other in ({"norm_act": "relu"}, {"norm_eps": 1e-3}, {"norm_groups": 4}, {"descent": {"beta1": 0.8}}, {"descent": {"beta2": 0.999}},
                  {"descent": {"kind": "adamw8"}}, {"descent": {"kind": "plain"}}):
        assert not restored(**other), other


WIDE = [dict(n=3, F=32, H=768, C=4, rows=64, K=4, batch=64), dict(n=3, F=32, H=1152, C=4, rows=72, K=4, batch=64),
        dict(n=2, F=16, H=4096, C=3, rows=64, K=3, batch=64), dict(n=3, F=32, H=1152, C=4, rows=64, K=4, batch=64, norm_groups=6, norm_act="silu")]


@pytest.mark.parametrize("ov", WIDE, ids=["H768", "H1152", "H4096", "H1152 G6"])
def test_objective_of_wide_hidden_layers(rfast_lib, ov):
    """More hidden units than eight rows of them fit 48 KB."""
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    wl = build_config("mlp_tree64", seed=4, **ov)
    m = make_model(wl)
    with pkg.Engine(wl) as eng:
        eng.load_schedule(wl.schedule)
        eng.run()
        x, d = eng.read(B.STATE_X), eng.diagnostics()
    xbar = x.astype(np.float64).mean(axis=0).astype(np.float32).astype(np.float64)
    want = sum(m.loss(i, xbar, np.arange(wl.rows)) for i in range(wl.n))
    assert abs(d["objective"] - want) <= 1e-4 * abs(want)


DIAG = [("mlp_tree64", dict(n=5, F=64, H=128, C=4, rows=128, K=12, batch=64, norm_groups=8, norm_act="silu")),
        ("mlp_tree64", dict(n=4, F=32, H=256, C=3, rows=192, K=10, batch=64, norm_groups=1, norm_act="relu", l2=1e-2)),
        ("mlp_tree64", dict(n=5, F=48, H=256, C=3, rows=128, K=12, batch=64, norm_groups=8, norm_act="none", alpha=0.003, descent={"kind": "adamw", **ADAM})),
        ("softmax_exp16", dict(n=8, F=48, C=5, rows=64, K=30, batch=8, alpha=0.003, descent={"kind": "adamw", **ADAM}))]


@pytest.mark.parametrize("name,ov", DIAG, ids=["silu", "relu l2", "none adamw", "softmax adamw"])
def test_full_gradient_and_merit_of_the_options(rfast_lib, name, ov):
    """Diagnostics in mid-run and at the end, full gradient and merit function among them, with a normalised layer and an adaptive
    step: the checks of the plain problems."""
    import test_gpu_aux
    test_gpu_aux.test_diagnostics_match_the_oracle_state(rfast_lib, name, ov)
