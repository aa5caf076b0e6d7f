"""One training step out of the operators, as a caller with tensors of its own puts it together: look-up, group norm, logits, policy loss, the
gradients back to the table, the norm over all of them, AdamW for table, scale and shift, Muon for the matrix.

Everything is fp32.  Each stage is off by at most (its longest chain of additions) u of its result's norm, u = 2^-24: look-up 1, group norm of 32
values 40, logits 64, loss and its gradient 2^-18 / u + 64 (the docstring of its own tests), products back 600 and 96, sums of the table 70; the
norms' projections do not enlarge an error, the division by the standard deviation does what it does to the result.  In all below 1200 u = 7.2e-5
of a gradient's norm; 1e-4 is asserted.  The loss itself is a sum of 96 such terms: 1e-4 of their magnitudes."""

from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

N, V, D, G = 96, 601, 64, 2
LOW, HIGH, KL, SCALE = 0.2, 0.3, 0.05, 8.0


def _state(seed):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    st = {"table": 0.1 * r(V, D), "W": 0.2 * r(V, D), "gamma": 1 + 0.1 * r(1, D), "beta": 0.1 * r(1, D)}
    st["t"] = torch.randint(-1, V, (N,), generator=gen, device="cuda")
    st["next"] = torch.randint(0, V, (N,), generator=gen, device="cuda")
    st["adv"], st["w"] = r(N), (torch.rand(N, generator=gen, device="cuda") < 0.9).float() / N
    z = _logits({k: v.double() for k, v in st.items() if k in ("table", "W", "gamma", "beta")}, st["t"])
    logp = torch.log_softmax(z, 1).gather(1, st["next"][:, None])[:, 0]
    far = torch.tensor([-0.5, -0.1, 0.0, 0.1, 0.6], device="cuda")
    st["old"] = (logp - far[torch.arange(N, device="cuda") % 5]).float()
    st["ref"] = (logp + 0.3 * r(N)).float()
    return st


def _logits(p, t):
    """In 64 bits."""
    import torch
    e = torch.where((t >= 0)[:, None], SCALE * p["table"][t.clamp_min(0)], torch.zeros((), dtype=torch.float64, device="cuda"))
    q = e.view(N, G, D // G)
    h = (q - q.mean(2, keepdim=True)) / (q.var(2, correction=0, keepdim=True) + 1e-5).sqrt()
    y = torch.relu(h.reshape(N, D) * p["gamma"] + p["beta"])
    return y @ p["W"].T


def _loss(st, p):
    import torch
    logp = torch.log_softmax(_logits(p, st["t"]), 1).gather(1, st["next"][:, None])[:, 0]
    r, a = torch.exp(logp - st["old"].double()), st["adv"].double()
    d = st["ref"].double() - logp
    return (st["w"].double() * (-torch.minimum(r * a, r.clamp(1 - LOW, 1 + HIGH) * a) + KL * (torch.expm1(d) - d))).sum()


class _Step:
    def __init__(self, st):
        import torch
        import paper_2307_11617_b200 as pkg
        e = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
        self.st = st
        self.buf = {"e": e(N, D), "y": e(N, D), "mean": e(N, G), "rstd": e(N, G), "z": e(N, V), "loss": e(1), "each": e(N), "logp": e(N),
                    "dy": e(N, D), "dx": e(N, D), "table": e(V, D), "W": e(V, D), "gamma": e(1, D), "beta": e(1, D), "norm": e(2)}
        self.m = {k: torch.zeros_like(st[k]) for k in ("table", "gamma", "beta", "W")}
        self.v = {k: torch.zeros_like(st[k]) for k in ("table", "gamma", "beta")}
        byte = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")  # noqa: E731
        self.shape = dict(samples=N, positions=1, channels=D, groups=G, act="relu")
        self.need = {"gn": pkg.rfast_group_norm_workspace(**self.shape), "gnb": pkg.rfast_group_norm_workspace(backward=True, **self.shape),
                     "emb": pkg.rfast_embedding_workspace(N, V, D), "muon": pkg.rfast_muon_workspace([V], [D]), "norm": pkg.GRAD_NORM_WORKSPACE}
        self.work = {k: byte(n) for k, n in self.need.items()}
        self.t = torch.ones(1, dtype=torch.int64, device="cuda")

    def _w(self, k):
        return dict(workspace=self.work[k].data_ptr(), workspace_bytes=self.need[k])

    def __call__(self):
        import torch
        import paper_2307_11617_b200 as pkg
        st, b = self.st, self.buf
        at = lambda x: x.data_ptr()  # noqa: E731
        s = dict(cuda_stream=torch.cuda.current_stream().cuda_stream)
        pkg.rfast_embedding(at(st["t"]), at(st["table"]), at(b["e"]), N, V, D, scale=SCALE, **s)
        pkg.rfast_group_norm(at(b["e"]), at(st["gamma"]), at(st["beta"]), at(b["y"]), at(b["mean"]), at(b["rstd"]), **self.shape, **self._w("gn"), **s)
        torch.matmul(b["y"], st["W"].T, out=b["z"])
        pkg.rfast_policy_loss(at(b["z"]), at(st["next"]), at(st["old"]), at(st["adv"]), N, V, d_loss=at(b["loss"]), d_token_loss=at(b["each"]), d_logp=at(b["logp"]),
                              d_dlogits=at(b["z"]), d_ref_logp=at(st["ref"]), d_weight=at(st["w"]), clip_low=LOW, clip_high=HIGH, kl_coef=KL, **s)
        torch.matmul(b["z"].T, b["y"], out=b["W"])
        torch.matmul(b["z"], st["W"], out=b["dy"])
        pkg.rfast_group_norm_backward(at(b["dy"]), at(b["e"]), at(st["gamma"]), at(st["beta"]), at(b["mean"]), at(b["rstd"]), at(b["dx"]), at(b["gamma"]), at(b["beta"]),
                                      **self.shape, **self._w("gnb"), **s)
        pkg.rfast_embedding_backward(at(st["t"]), at(b["dx"]), at(b["table"]), N, V, D, scale=SCALE, **self._w("emb"), **s)
        names = ("table", "gamma", "beta")
        pkg.rfast_grad_norm([at(b[k]) for k in names + ("W",)], [b[k].numel() for k in names + ("W",)], 0.05, at(b["norm"]), at(b["norm"]) + 4, at(self.work["norm"]),
                            self.need["norm"], **s)
        pkg.rfast_adamw_step([at(st[k]) for k in names], [at(b[k]) for k in names], [at(self.m[k]) for k in names], [at(self.v[k]) for k in names],
                             [st[k].numel() for k in names], d_step=at(self.t), lr=1e-2, d_grad_scale=at(b["norm"]) + 4, **s)
        pkg.rfast_muon_step([at(st["W"])], [at(b["W"])], [at(self.m["W"])], [V], [D], lr=0.05, weight_decay=0.1, d_grad_scale=at(b["norm"]) + 4, **self._w("muon"), **s)
        self.t += 1


def test_gradients_and_step():
    import torch
    st = _state(3)
    p = {k: st[k].double().requires_grad_() for k in ("table", "W", "gamma", "beta")}
    loss = _loss(st, p)
    want = dict(zip(p, torch.autograd.grad(loss, list(p.values()))))
    before = {k: st[k].clone() for k in p}
    step = _Step(st)
    step()
    torch.cuda.synchronize()
    b = step.buf
    assert abs(float(b["loss"]) - float(loss.detach())) <= 1e-4 * float(b["each"].abs().sum())
    for k in p:
        assert float((b[k].double() - want[k]).norm()) <= 1e-4 * float(want[k].norm()), k
    norm = float(sum(g.square().sum() for g in want.values()).sqrt())
    assert abs(float(b["norm"][0]) - norm) <= 1e-4 * norm and abs(float(b["norm"][1]) - min(1.0, 0.05 / norm)) <= 1e-4
    # rows of the table that no token names move by their decay alone
    idle = torch.ones(V, dtype=torch.bool, device="cuda")
    idle[st["t"][st["t"] >= 0]] = False
    assert torch.allclose(st["table"][idle], before["table"][idle] * (1 - 1e-2 * 1e-2), rtol=3e-7, atol=0)
    # the matrix moves by lr size along a nearly orthogonal matrix
    move = (st["W"].double() - before["W"].double() * (1 - 0.05 * 0.1)) / (0.05 * (V / D) ** 0.5)
    s = torch.linalg.svdvals(move)
    assert float(s.max()) < 1.3 and float((s > 0.3).sum()) >= D // 2


def test_recorded_steps_equal_called_ones():
    import torch
    called, recorded = _Step(_state(5)), _Step(_state(5))
    for _ in range(4):
        called()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        recorded()
    for _ in range(4):
        g.replay()
    torch.cuda.synchronize()
    for k in ("table", "W", "gamma", "beta"):
        assert torch.equal(called.st[k], recorded.st[k]), k
        assert torch.equal(called.m[k], recorded.m[k]), k
    assert torch.equal(called.buf["loss"], recorded.buf["loss"])
