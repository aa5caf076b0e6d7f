"""Which operands the policy loss wants for which results: decided on the host, so these run without a GPU; the addresses are never followed."""

from __future__ import annotations

import pytest

A = 1 << 20          # an address nobody reads


@pytest.mark.parametrize("d_old_logp,d_advantage", [(0, 0), (A, 0), (0, A)])
def test_log_probabilities_alone_want_neither_an_old_policy_nor_an_advantage(rfast_lib, d_old_logp, d_advantage):
    import paper_2307_11617_b200 as pkg
    call = dict(tokens=4, vocab=9)
    with pytest.raises(pkg.RFastError) as ei:                # the address, or that there is no device: what is looked at last
        pkg.rfast_policy_loss(A, A, d_old_logp, d_advantage, d_logp=A, **call)
    assert "old_logp or advantage" not in str(ei.value)
    for wanted in (dict(d_token_loss=A), dict(d_dlogits=2 * A), dict(d_token_loss=A, d_loss=A), dict(d_logp=A, d_dlogits=2 * A)):
        with pytest.raises(pkg.RFastError) as ei:
            pkg.rfast_policy_loss(A, A, d_old_logp, d_advantage, **wanted, **call)
        assert "old_logp or advantage" in str(ei.value), wanted
