"""Refusals of the embedding, policy loss and Muon operators.  Every one of them is decided on the host before any device is looked at,
so these run without a GPU; the addresses are never followed."""

from __future__ import annotations

import pytest

A = 1 << 20          # an address nobody reads
INF, NAN = float("inf"), float("nan")


def _refused(text, call, *a, **kw):
    from paper_2307_11617_b200.binding import EINVAL, RFastError
    with pytest.raises(RFastError) as ei:
        call(*a, **kw)
    assert ei.value.code == EINVAL and text in str(ei.value), ei.value


SHAPE = dict(tokens=4, vocab=6, width=8)
BAD_SHAPES = [("tokens must be", dict(tokens=-1)), ("tokens must be", dict(tokens=(1 << 30) + 1)), ("vocab must be", dict(vocab=0)),
              ("vocab must be", dict(vocab=(1 << 30) + 1)), ("width must be", dict(width=0)), ("width must be", dict(width=(1 << 24) + 1))]


@pytest.mark.parametrize("text,kw", BAD_SHAPES)
def test_embedding_refuses_shapes(rfast_lib, text, kw):
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200.binding import RFastError
    shape = {**SHAPE, **kw}
    _refused(text, pkg.rfast_embedding, A, A, A, **shape)
    _refused(text, pkg.rfast_embedding_backward, A, A, A, workspace=A, workspace_bytes=1 << 40, **shape)
    with pytest.raises(RFastError):
        pkg.rfast_embedding_workspace(**shape)


@pytest.mark.parametrize("text,kw", [
    ("token_bits", dict(token_bits=16)), ("tokens are null", dict(d_tokens=0)), ("tokens are null or not aligned", dict(d_tokens=A + 4)),
    ("tokens are null or not aligned", dict(d_tokens=A + 2, token_bits=32)), ("table is null", dict(d_table=0)), ("table is not aligned", dict(d_table=A + 2)),
    ("table has rows that overlap", dict(table_stride=-1)), ("table spans", dict(table_stride=1 << 55)), ("out is null", dict(d_out=0)),
    ("out is not aligned", dict(d_out=A + 1, out_type="bf16")), ("out has rows that overlap", dict(out_stride=7)), ("out has rows that overlap", dict(out_stride=0)),
    ("out spans", dict(out_stride=1 << 55)), ("scale must be finite", dict(scale=NAN)), ("scale must be finite", dict(scale=INF))])
def test_embedding_refuses_operands(rfast_lib, text, kw):
    import paper_2307_11617_b200 as pkg
    _refused(text, pkg.rfast_embedding, **{**dict(d_tokens=A, d_table=A, d_out=A), **SHAPE, **kw})


@pytest.mark.parametrize("text,kw", [
    ("token_bits", dict(token_bits=8)), ("tokens are null", dict(d_tokens=0)), ("dout is null", dict(d_dout=0)), ("dout is not aligned", dict(d_dout=A + 2)),
    ("dout has rows that overlap", dict(dout_stride=-8)), ("dtable is null", dict(d_dtable=0)), ("dtable is not aligned", dict(d_dtable=A + 1, table_type="f16")),
    ("dtable has rows that overlap", dict(dtable_stride=7)), ("dtable spans", dict(dtable_stride=1 << 55)), ("workspace must be given", dict(workspace=0)),
    ("workspace must be given", dict(workspace=A + 8)), ("workspace needs", dict(workspace_bytes=100)), ("scale must be finite", dict(scale=-INF))])
def test_embedding_backward_refuses(rfast_lib, text, kw):
    import paper_2307_11617_b200 as pkg
    _refused(text, pkg.rfast_embedding_backward, **{**dict(d_tokens=A, d_dout=A, d_dtable=A, workspace=A, workspace_bytes=1 << 30), **SHAPE, **kw})


def test_embedding_of_nothing_needs_no_device(rfast_lib):
    import paper_2307_11617_b200 as pkg
    pkg.rfast_embedding(0, 0, 0, tokens=0, vocab=3, width=2)
    pkg.rfast_embedding_backward(0, 0, A, tokens=0, vocab=3, width=2, accumulate=True, workspace=A, workspace_bytes=1 << 30)


@pytest.mark.parametrize("text,kw", [
    ("tokens must be", dict(tokens=-1)), ("tokens must be", dict(tokens=1 << 31)), ("vocab must be", dict(vocab=0)), ("vocab must be", dict(vocab=1 << 31)),
    ("token_bits", dict(token_bits=0)), ("temperature", dict(temperature=0.0)), ("temperature", dict(temperature=NAN)), ("temperature", dict(temperature=INF)),
    ("clip_low", dict(clip_low=-0.1)), ("clip_low", dict(clip_low=1.1)), ("clip_low", dict(clip_high=NAN)), ("clip_low", dict(clip_high=-1.0)),
    ("kl_coef", dict(kl_coef=NAN)), ("d_loss is summed", dict(d_token_loss=0)), ("no result", dict(d_loss=0, d_token_loss=0, d_logp=0, d_dlogits=0)),
    ("logits are null", dict(d_logits=0)), ("logits are null or not aligned", dict(d_logits=A + 2)), ("dlogits are not aligned", dict(d_dlogits=A + 1, type="f16")),
    ("tokens are null", dict(d_tokens=0)), ("tokens are null or not aligned", dict(d_tokens=A + 4)), ("old_logp or advantage", dict(d_old_logp=0)),
    ("old_logp or advantage", dict(d_advantage=0)), ("stride of logits", dict(logits_stride=-1)), ("stride of logits", dict(logits_stride=1 << 55)),
    ("stride of dlogits", dict(dlogits_stride=8)), ("stride of dlogits", dict(dlogits_stride=1 << 55)),
    ("in the place of the logits", dict(d_dlogits=A, dlogits_stride=10)), ("fp32 operand", dict(d_logp=A + 2)), ("fp32 operand", dict(d_weight=A + 1))])
def test_policy_loss_refuses(rfast_lib, text, kw):
    import paper_2307_11617_b200 as pkg
    _refused(text, pkg.rfast_policy_loss, **{**dict(d_logits=A, d_tokens=A, d_old_logp=A, d_advantage=A, tokens=4, vocab=9, d_loss=A, d_token_loss=A, d_logp=A,
                                                    d_dlogits=2 * A, d_ref_logp=A), **kw})


def test_policy_loss_of_nothing_needs_no_device(rfast_lib):
    import paper_2307_11617_b200 as pkg
    pkg.rfast_policy_loss(0, 0, 0, 0, tokens=0, vocab=9, d_token_loss=A)


def test_unknown_types_are_refused(rfast_lib):
    import ctypes as C
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    with pytest.raises(ValueError):
        pkg.rfast_embedding(A, A, A, table_type="f64", **SHAPE)
    err = C.create_string_buffer(256)
    assert B.lib().rfast_embedding(None, None, None, 1, 1.0, None, 1, None, err, 256) == B.EINVAL and b"null shape" in err.value
    shape = B._EmbShape(1, 1, 1, 64, 5, 0)
    assert B.lib().rfast_embedding(C.byref(shape), A, A, 1, 1.0, A, 1, None, err, 256) == B.EINVAL and b"unknown type" in err.value
    assert B.lib().rfast_policy_loss(None, None, None, 0) == B.EINVAL
    p = B._Policy(1, 1, 9, 64)
    assert B.lib().rfast_policy_loss(C.byref(p), None, err, 256) == B.EINVAL and b"unknown type" in err.value


def _muon(**kw):
    import paper_2307_11617_b200 as pkg
    base = dict(param=[A, A], grad=[A, A], momentum_buffer=[A, A], rows=[5, 7], cols=[3, 9], workspace=A, workspace_bytes=1 << 40)
    base.update(kw)
    pkg.rfast_muon_step(**base)


@pytest.mark.parametrize("text,kw", [
    ("rows and cols must be", dict(rows=[5, -1])), ("rows and cols must be", dict(cols=[3, 65537])), ("terms must be", dict(terms=3)), ("terms must be", dict(terms=-1)),
    ("momentum must be", dict(momentum=1.0)), ("momentum must be", dict(momentum=NAN)), ("momentum must be", dict(momentum=-0.1)), ("eps must be", dict(eps=0.0)),
    ("eps must be", dict(eps=NAN)), ("eps must be", dict(eps=INF)), ("lr and weight_decay", dict(lr=INF)), ("lr and weight_decay", dict(weight_decay=NAN)),
    ("iterations must be", dict(iterations=0)), ("iterations must be", dict(iterations=33)), ("d_grad_scale is not aligned", dict(d_grad_scale=A + 2)),
    ("tensor 1 has a null address", dict(param=[A, 0])), ("tensor 0 has a null address", dict(grad=[0, A])), ("tensor 1 has a null address", dict(momentum_buffer=[A, 0])),
    ("address of tensor 1 is not aligned", dict(param=[A, A + 2])), ("address of tensor 0 is not aligned", dict(grad=[A + 1, A], grad_type="bf16")),
    ("address of tensor 0 is not aligned", dict(momentum_buffer=[A + 2, A])), ("workspace must be given", dict(workspace=0)), ("workspace must be given", dict(workspace=A + 128)),
    ("workspace needs", dict(workspace_bytes=1000))])
def test_muon_refuses(rfast_lib, text, kw):
    _refused(text, _muon, **kw)


def test_muon_c_entry_refuses(rfast_lib):
    import ctypes as C
    import numpy as np
    import paper_2307_11617_b200 as pkg
    from paper_2307_11617_b200 import binding as B
    err = C.create_string_buffer(256)
    assert B.lib().rfast_muon_step(None, None, 0, None, err, 256) == B.EINVAL and b"null arguments" in err.value
    assert B.lib().rfast_muon_step(None, None, 0, None, None, 0) == B.EINVAL
    assert B.lib().rfast_muon_workspace(1, None, None, 1) == B.EINVAL
    one = np.ones(2, np.int32)
    at = one.ctypes.data
    for field, value, text in (("param_type", 4, b"unknown type"), ("grad_type", -1, b"unknown type"), ("size_rule", 2, b"unknown size_rule"), ("n_tensors", -1, b"n_tensors"),
                               ("rows", None, b"null array"), ("grad", None, b"null array")):
        a = B._Muon(1, 0, 0, 0, at, at, at, at, at, 0.1, 0.9, 0.0, 1e-7, 1, 5, 0, None)
        setattr(a, field, value)
        assert B.lib().rfast_muon_step(C.byref(a), A, 1 << 40, None, err, 256) == B.EINVAL and text in err.value, err.value
    with pytest.raises(ValueError):
        _muon(rows=[5])
    with pytest.raises(ValueError):
        _muon(grad=[A])
    with pytest.raises(ValueError):
        _muon(size_rule="none")
    with pytest.raises(B.RFastError):
        pkg.rfast_muon_workspace([1], [1], terms=3)


def test_muon_of_nothing_needs_no_device(rfast_lib):
    import paper_2307_11617_b200 as pkg
    pkg.rfast_muon_step([], [], [], [], [])
    pkg.rfast_muon_step([0], [0], [0], [0], [7])


def test_muon_workspace_holds_its_largest_run(rfast_lib):
    """Runs use it one after another: a second run of the same size asks for no more."""
    import paper_2307_11617_b200 as pkg
    one = pkg.rfast_muon_workspace([64] * 128, [96] * 128)
    assert pkg.rfast_muon_workspace([64] * 256, [96] * 256) == one
    assert pkg.rfast_muon_workspace([64], [96], param_type="bf16") < pkg.rfast_muon_workspace([64], [96]) < one
    # halves of X (two buffers), A and B in 16 bits, twice for two terms
    assert one >= 128 * (2 * 64 * 96 + 2 * 64 * 64) * 2 * 2
