"""The table's gradient where one token has half of the places of a large vocabulary (a word of padding that is not masked, the first word of
every sequence), as a list that is long and as one that is not sorted already.  Tolerance: a run's sum is a chain of at most 16 places, 16 chunks (as
8 pairs) and, of the run, a piece at each end, 15 chunks at each end and its spans of 256: 16 + 9 + 2 + 30 + count / 256 additions, u = 2^-24 of the sum of
magnitudes each, 2 u for the scale's product (and the sum with what was there, u of it), then half a step of the gradient's type."""

from __future__ import annotations

import numpy as np
import pytest

from test_gpu_embedding import HALF, TINY, U, _dt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,vocab,width", [(200_000, 131_072, 40), (131_071, 50_257, 264), (70_000, 200_003, 33), (1 << 20, 131_072, 8), (40_000, 100_000, 513)])
@pytest.mark.parametrize("out,table,bits", [("f32", "f32", 64), ("bf16", "f32", 32), ("f16", "bf16", 64)])
def test_one_token_in_half_of_the_places(n, vocab, width, out, table, bits):
    import torch
    import paper_2307_11617_b200 as pkg
    rng = np.random.default_rng(n + width)
    t = rng.integers(0, vocab, n)
    t[rng.random(n) < 0.5] = vocab - 1                       # the largest key
    t[rng.random(n) < 0.02] = -1
    t[rng.random(n) < 0.1] = 7                               # and one that is only frequent
    tt = torch.as_tensor(t).to(torch.int32 if bits == 32 else torch.int64).cuda()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    dout = (torch.randn(n, width, generator=gen, device="cuda").abs() if width % 2 == 0 else torch.randn(n, width, generator=gen, device="cuda")).to(_dt(out))
    got = torch.full((vocab, width), 5.0, dtype=_dt(table), device="cuda")
    need = pkg.rfast_embedding_workspace(n, vocab, width)
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    call = dict(tokens=n, vocab=vocab, width=width, scale=0.5, token_bits=bits, out_type=out, table_type=table, workspace=work.data_ptr(), workspace_bytes=need,
                cuda_stream=torch.cuda.current_stream().cuda_stream)
    some = tt >= 0
    at, d = tt[some].long(), dout[some].double()
    total = 0.5 * torch.zeros(vocab, width, dtype=torch.float64, device="cuda").index_add_(0, at, d)
    size = 0.5 * torch.zeros(vocab, width, dtype=torch.float64, device="cuda").index_add_(0, at, d.abs())
    count = torch.bincount(at, minlength=vocab).double()[:, None]
    tol = (torch.minimum(count, 57 + count / 256) + 2) * U * size
    for accumulate in (False, True):
        before = got.double() if accumulate else torch.zeros_like(total)
        pkg.rfast_embedding_backward(tt.data_ptr(), dout.data_ptr(), got.data_ptr(), accumulate=accumulate, **call)
        want = total + before
        e = tol + (U * (before.abs() + total.abs()) if accumulate else 0.0)
        e = e + HALF[table] * (want.abs() + e) + TINY[table]
        bad = (got.double() - want).abs() > e
        assert not bool(bad.any()), (accumulate, int(bad.sum()), bad.nonzero()[:3].tolist())
        if not accumulate:
            first = got.clone()
    got.fill_(1.0)
    pkg.rfast_embedding_backward(tt.data_ptr(), dout.data_ptr(), got.data_ptr(), **call)
    assert torch.equal(got, first)
