"""Embedding look-up and its gradient against plain restatements in 64 bits.

u = 2^-24 is half a step of fp32.  A look-up is one fp32 product rounded once to its type, and so is the restatement: equal bits.
A gradient is a sum in fp32: chunks of up to 16 terms, sixteen of those to a span of 256, and of a run at most two pieces, 15 chunks before and
15 behind its n / 256 spans.  Each addition is off by at most u of the sum of magnitudes: (chain) u sum|x| with chain = min(count, 16 + 16 +
32 + n / 256), 2 u for the scale's product (and the sum with what was there, u of that), then half a step of the gradient's type."""

from __future__ import annotations

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _strided(rows, width, stride, kind, lead, fill=77.0):
    """A tensor of rows * stride values (rows of `width`), `lead` elements off its allocation; the rest holds a mark."""
    import torch
    flat = torch.full((lead + max(rows, 1) * stride + 16,), fill, dtype=_dt(kind), device="cuda")
    return flat, flat[lead:lead + max(rows, 1) * stride].view(max(rows, 1), stride)[:rows, :width]


def _marks_stand(flat, view, lead, rows, width, stride, fill=77.0):
    import torch
    keep = torch.ones_like(flat, dtype=torch.bool)
    keep[lead:lead + max(rows, 1) * stride].view(max(rows, 1), stride)[:rows, :width] = False
    return bool((flat[keep].double() == fill).all())


def _tokens(n, vocab, how, rng):
    if how == "even":
        t = rng.integers(0, vocab, n)
    elif how == "text":
        t = (np.exp(rng.random(n) * math.log(vocab + 1.0)) - 1.0).astype(np.int64).clip(0, vocab - 1) * 7919 % vocab
    elif how == "one":
        t = np.full(n, vocab // 2)
    elif how == "runs":                     # runs that begin and end at, before and behind multiples of 16 and 256
        t = np.zeros(n, np.int64)
        at, k = 0, 0
        for size in [64, 1, 63, 65, 1024, 1, 1023, 128, 2, 62, 2048, 1000, 1048, 3000, 16, 15, 1, 17, 255, 256, 257, 32, 240] * (n // 10000 + 1):
            t[at:at + size] = k % vocab
            at, k = at + size, k + 1
        t = t[rng.permutation(n)]
    elif how == "none":
        t = np.full(n, -1)
    elif how == "falling":
        t = np.arange(n)[::-1] % vocab
    t = t.astype(np.int64)
    if how in ("even", "text", "falling") and n > 4:
        t[rng.integers(0, n, max(1, n // 20))] = -1
        t[rng.integers(0, n, 2)] = [vocab, vocab + 1000]    # beyond the table: none either
    return t


FORWARD = [(1, 1, 1), (3, 2, 5), (37, 11, 8), (100, 1000, 256), (33, 97, 321), (257, 500, 1024), (70, 40, 1032), (5000, 300, 33), (0, 5, 8)]


@pytest.mark.parametrize("n,vocab,width", FORWARD)
@pytest.mark.parametrize("table,out,bits,lead,pad", [("f32", "f32", 64, 0, 0), ("f32", "bf16", 32, 0, 8), ("bf16", "bf16", 64, 8, 16), ("f16", "f16", 32, 1, 3),
                                                     ("bf16", "f32", 64, 4, 4), ("f16", "bf16", 64, 0, 0)])
def test_look_up(n, vocab, width, table, out, bits, lead, pad):
    import torch
    import paper_2307_11617_b200 as pkg
    rng = np.random.default_rng(n * 7 + width)
    t = torch.as_tensor(_tokens(n, vocab, "even", rng)).cuda()
    ft, tab = _strided(vocab, width, width + pad, table, lead)
    tab.copy_(torch.as_tensor(rng.standard_normal((vocab, width)).astype(np.float32)))
    fo, got = _strided(n, width, width + 2 * pad, out, lead)
    scale = 0.3 + width
    tt = t.to(torch.int32 if bits == 32 else torch.int64)
    pkg.rfast_embedding(tt.data_ptr(), tab.data_ptr(), got.data_ptr() if n else 0, tokens=n, vocab=vocab, width=width, scale=scale, token_bits=bits, table_type=table,
                        out_type=out, table_stride=width + pad, out_stride=width + 2 * pad, cuda_stream=torch.cuda.current_stream().cuda_stream)
    some = (t >= 0) & (t < vocab)
    want = torch.where(some[:, None], tab[t.clamp(0, vocab - 1)].float() * torch.tensor(scale, dtype=torch.float32).cuda(), torch.zeros((), device="cuda")).to(_dt(out))
    assert torch.equal(got, want)
    assert _marks_stand(fo, got, lead, n, width, width + 2 * pad)


def _gradient(t, dout, vocab, scale, before=None):
    """Sums in 64 bits, sums of magnitudes, counts."""
    import torch
    t = torch.as_tensor(t, device=dout.device)
    some = (t >= 0) & (t < vocab)
    d = dout.double()[some]
    total = torch.zeros(vocab, dout.shape[1], dtype=torch.float64, device=dout.device).index_add_(0, t[some], d)
    size = torch.zeros_like(total).index_add_(0, t[some], d.abs())
    count = torch.bincount(t[some], minlength=vocab).double()
    return total * scale, size * abs(scale), count


def _check_gradient(got, t, dout, vocab, scale, kind, before=None):
    import torch
    total, size, count = _gradient(t, dout, vocab, scale)
    n = dout.shape[0]
    chain = torch.clamp(count, max=64 + n / 256)[:, None]
    tol = (chain + 2) * U * size
    if before is not None:
        tol = tol + U * (before.abs() + total.abs())
        total = total + before
    tol = tol + HALF[kind] * (total.abs() + tol) + TINY[kind]
    bad = (got.double() - total).abs() > tol
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:3].tolist())


BACKWARD = [(0, 5, 8, "even"), (1, 1, 1, "even"), (1, 300, 16, "even"), (2, 2, 7, "even"), (64, 10, 24, "one"), (65, 10, 257, "one"), (1000, 1023, 256, "even"),
            (2047, 1024, 40, "text"), (2048, 1025, 264, "text"), (2049, 100_003, 33, "text"), (5000, 7, 520, "text"), (20_000, 200, 72, "runs"), (20_001, 31, 5, "runs"),
            (131_072, 3, 16, "one"), (140_001, 250_000, 8, "even"), (3000, 50, 64, "none"), (4096, 70_000, 128, "falling"), (300_000, 1 << 21, 2, "text")]


@pytest.mark.parametrize("n,vocab,width,how", BACKWARD)
@pytest.mark.parametrize("out,table,bits,lead,pad", [("f32", "f32", 64, 0, 0), ("bf16", "f32", 32, 8, 8), ("bf16", "bf16", 64, 0, 16), ("f16", "f16", 32, 3, 5)])
def test_gradient(n, vocab, width, how, out, table, bits, lead, pad):
    import torch
    import paper_2307_11617_b200 as pkg
    rng = np.random.default_rng(n + 13 * width)
    t = _tokens(n, vocab, how, rng)
    _, dout = _strided(n, width, width + pad, out, lead)
    if n:
        dout.copy_(torch.as_tensor(rng.standard_normal((n, width)).astype(np.float32)))
        dout[torch.as_tensor((t < 0) | (t >= vocab)).cuda()] = math.nan         # rows of no token are not read
    fg, got = _strided(vocab, width, width + pad, table, lead)
    need = pkg.rfast_embedding_workspace(tokens=n, vocab=vocab, width=width)
    work = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    tt = torch.as_tensor(t).to(torch.int32 if bits == 32 else torch.int64).cuda()
    call = dict(tokens=n, vocab=vocab, width=width, scale=1.7, token_bits=bits, out_type=out, table_type=table, dout_stride=width + pad, dtable_stride=width + pad,
                workspace=work.data_ptr(), workspace_bytes=need, cuda_stream=torch.cuda.current_stream().cuda_stream)
    pkg.rfast_embedding_backward(tt.data_ptr(), dout.data_ptr(), got.data_ptr(), **call)
    clean = torch.nan_to_num(dout.float(), nan=0.0)
    scale = float(np.float32(1.7))
    _check_gradient(got, t, clean, vocab, scale, table)
    assert _marks_stand(fg, got, lead, vocab, width, width + pad)
    assert bool((work[need:] == 255).all())
    # the same once more: equal bits, whatever the workspace held
    first = got.clone()
    got.fill_(5.0)
    work.fill_(0)
    pkg.rfast_embedding_backward(tt.data_ptr(), dout.data_ptr(), got.data_ptr(), **call)
    assert torch.equal(first, got)
    # on top of what is there
    got.copy_(torch.as_tensor(rng.standard_normal((vocab, width)).astype(np.float32)))
    before = got.double()
    pkg.rfast_embedding_backward(tt.data_ptr(), dout.data_ptr(), got.data_ptr(), accumulate=True, **call)
    _check_gradient(got, t, clean, vocab, scale, table, before)
    unused = np.ones(vocab, bool)
    unused[t[(t >= 0) & (t < vocab)]] = False
    unused = torch.as_tensor(unused).cuda()
    assert torch.equal(got.double()[unused], before[unused])


def test_a_nan_reaches_its_token_only():
    import torch
    import paper_2307_11617_b200 as pkg
    n, vocab, width = 5000, 40, 24
    t = torch.arange(n, device="cuda") % vocab
    dout = torch.ones(n, width, device="cuda")
    dout[1234, 5] = math.nan
    dout[1235, 6] = math.inf
    got = torch.empty(vocab, width, device="cuda")
    need = pkg.rfast_embedding_workspace(n, vocab, width)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    pkg.rfast_embedding_backward(t.data_ptr(), dout.data_ptr(), got.data_ptr(), n, vocab, width, workspace=work.data_ptr(), workspace_bytes=need,
                                 cuda_stream=torch.cuda.current_stream().cuda_stream)
    want = torch.full((vocab, width), n / vocab, device="cuda")
    want[1234 % vocab, 5] = math.nan
    want[1235 % vocab, 6] = math.inf
    assert torch.equal(torch.nan_to_num(got, nan=-1.0, posinf=-2.0), torch.nan_to_num(want, nan=-1.0, posinf=-2.0))


def test_a_broadcast_gradient():
    """dout with a stride of 0, as the gradient of a sum over positions has it."""
    import torch
    import paper_2307_11617_b200 as pkg
    n, vocab, width = 3000, 17, 40
    t = (torch.arange(n, device="cuda") * 7) % vocab
    one = torch.randn(width, device="cuda")
    got = torch.empty(vocab, width, device="cuda")
    need = pkg.rfast_embedding_workspace(n, vocab, width)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    pkg.rfast_embedding_backward(t.data_ptr(), one.data_ptr(), got.data_ptr(), n, vocab, width, dout_stride=0, workspace=work.data_ptr(), workspace_bytes=need,
                                 cuda_stream=torch.cuda.current_stream().cuda_stream)
    _check_gradient(got, t.cpu().numpy(), one.expand(n, width), vocab, 1.0, "f32")


def test_recorded_into_a_graph_and_on_two_streams():
    import torch
    import paper_2307_11617_b200 as pkg
    n, vocab, width = 9000, 5000, 96
    rng = np.random.default_rng(3)
    need = pkg.rfast_embedding_workspace(n, vocab, width)
    jobs = []
    for k in range(2):
        t = torch.as_tensor(_tokens(n, vocab, "text", rng)).cuda()
        tab = torch.randn(vocab, width, device="cuda")
        jobs.append(dict(t=t, tab=tab, out=torch.empty(n, width, device="cuda"), grad=torch.empty(vocab, width, device="cuda"),
                         work=torch.empty(need, dtype=torch.uint8, device="cuda"), stream=torch.cuda.Stream()))

    def both(j, stream):
        pkg.rfast_embedding(j["t"].data_ptr(), j["tab"].data_ptr(), j["out"].data_ptr(), n, vocab, width, scale=2.0, cuda_stream=stream)
        pkg.rfast_embedding_backward(j["t"].data_ptr(), j["out"].data_ptr(), j["grad"].data_ptr(), n, vocab, width, workspace=j["work"].data_ptr(), workspace_bytes=need,
                                     cuda_stream=stream)

    torch.cuda.synchronize()
    graphs = []
    for j in jobs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            both(j, torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    for rep in range(3):
        for j in jobs:
            j["tab"].normal_()
            j["t"].copy_(torch.as_tensor(_tokens(n, vocab, "text", rng)))
        torch.cuda.synchronize()
        for j, g in zip(jobs, graphs):                      # side by side, a workspace each
            with torch.cuda.stream(j["stream"]):
                g.replay()
        torch.cuda.synchronize()
        for j in jobs:
            got = j["grad"].clone()
            _check_gradient(got, j["t"].cpu().numpy(), j["out"], vocab, 1.0, "f32")
            both(j, torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            assert torch.equal(got, j["grad"])


def test_gradient_against_differences():
    """<dout, out(table + h e) - out(table)> = h <dtable, e>: the look-up is linear, so differences are exact up to roundings."""
    import torch
    import paper_2307_11617_b200 as pkg
    n, vocab, width, scale = 4000, 301, 64, 3.0
    rng = np.random.default_rng(9)
    t = torch.as_tensor(_tokens(n, vocab, "text", rng)).cuda()
    dout, e = torch.randn(n, width, device="cuda"), torch.randn(vocab, width, device="cuda")
    out, grad = torch.empty(n, width, device="cuda"), torch.empty(vocab, width, device="cuda")
    need = pkg.rfast_embedding_workspace(n, vocab, width)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    pkg.rfast_embedding(t.data_ptr(), e.data_ptr(), out.data_ptr(), n, vocab, width, scale=scale, cuda_stream=st)
    pkg.rfast_embedding_backward(t.data_ptr(), dout.data_ptr(), grad.data_ptr(), n, vocab, width, scale=scale, workspace=work.data_ptr(), workspace_bytes=need, cuda_stream=st)
    a, b = (dout.double() * out.double()).sum(), (grad.double() * e.double()).sum()
    size = (grad.double() * e.double()).abs().sum() + (dout.double() * out.double()).abs().sum()
    assert abs(a - b) <= 260 * U * size


def test_offsets_beyond_32_bits():
    """A table of 2.3e9 values: its last rows lie beyond 2^31 values and 2^32 bytes."""
    import torch
    import paper_2307_11617_b200 as pkg
    vocab, width, n = 70_000, 32_768, 300
    table = torch.zeros(vocab, width, dtype=torch.bfloat16, device="cuda")
    t = torch.arange(vocab - n, vocab, device="cuda")[torch.randperm(n, device="cuda")]
    t[::7] = torch.arange(0, (n + 6) // 7, device="cuda")
    table[t] = torch.randn(n, width, device="cuda").bfloat16()
    out = torch.empty(n, width, dtype=torch.bfloat16, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    pkg.rfast_embedding(t.data_ptr(), table.data_ptr(), out.data_ptr(), n, vocab, width, scale=0.5, table_type="bf16", out_type="bf16", cuda_stream=st)
    assert torch.equal(out, table[t] * 0.5)
    need = pkg.rfast_embedding_workspace(n, vocab, width)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    grad = torch.full((vocab, width), 3.0, dtype=torch.bfloat16, device="cuda")
    pkg.rfast_embedding_backward(t.data_ptr(), out.data_ptr(), grad.data_ptr(), n, vocab, width, scale=2.0, out_type="bf16", table_type="bf16", workspace=work.data_ptr(),
                                 workspace_bytes=need, cuda_stream=st)
    assert torch.equal(grad[t], table[t])                      # every token once: exact
    assert int((grad != 0).any(1).sum()) == len(t.unique())


def test_rows_read_over_one_another():
    """A table whose rows overlap (a stride below its width), as sliding windows of one sequence."""
    import torch
    import paper_2307_11617_b200 as pkg
    flat = torch.randn(4096, device="cuda")
    for stride, width in ((8, 64), (3, 17), (0, 40)):
        vocab, n = 200, 333
        t = torch.randint(0, vocab, (n,), device="cuda")
        out = torch.empty(n, width, device="cuda")
        pkg.rfast_embedding(t.data_ptr(), flat.data_ptr(), out.data_ptr(), n, vocab, width, table_stride=stride, cuda_stream=torch.cuda.current_stream().cuda_stream)
        assert torch.equal(out, flat.as_strided((vocab, width), (stride, 1))[t])


@pytest.mark.parametrize("width", [1, 2, 8, 16, 63, 64, 65, 128, 248, 256, 264])
@pytest.mark.parametrize("lead,pad", [(0, 0), (8, 8), (1, 2)])
def test_short_rows(width, lead, pad):
    """Rows of fewer columns than a warp takes, many of them."""
    import torch
    import paper_2307_11617_b200 as pkg
    n, vocab = 5003, 700
    rng = np.random.default_rng(width)
    t = torch.as_tensor(_tokens(n, vocab, "even", rng)).cuda()
    ft, tab = _strided(vocab, width, width + pad, "bf16", lead)
    tab.copy_(torch.as_tensor(rng.standard_normal((vocab, width)).astype(np.float32)))
    fo, got = _strided(n, width, width + 2 * pad, "f32", lead)
    pkg.rfast_embedding(t.data_ptr(), tab.data_ptr(), got.data_ptr(), n, vocab, width, scale=1.5, table_type="bf16", out_type="f32", table_stride=width + pad,
                        out_stride=width + 2 * pad, cuda_stream=torch.cuda.current_stream().cuda_stream)
    some = (t >= 0) & (t < vocab)
    want = torch.where(some[:, None], tab[t.clamp(0, vocab - 1)].float() * 1.5, torch.zeros((), device="cuda"))
    assert torch.equal(got, want)
    assert _marks_stand(fo, got, lead, n, width, width + 2 * pad)


def test_more_short_rows_than_32_bits_count():
    import torch
    import paper_2307_11617_b200 as pkg
    n, vocab, width = 65_100_000, 10, 33                       # 2.15e9 values
    t = torch.randint(0, vocab, (n,), dtype=torch.int32, device="cuda")
    table = torch.randn(vocab, width, device="cuda").bfloat16()
    out = torch.empty(n, width, dtype=torch.bfloat16, device="cuda")
    pkg.rfast_embedding(t.data_ptr(), table.data_ptr(), out.data_ptr(), n, vocab, width, token_bits=32, table_type="bf16", out_type="bf16",
                        cuda_stream=torch.cuda.current_stream().cuda_stream)
    for part in (slice(0, 1000), slice(n // 2, n // 2 + 1000), slice(n - 2_000_000, n)):
        assert torch.equal(out[part], table[t[part].long()])
