"""The cases that tell 64 bits from 32 do tell them apart: the oracle with 32 bits planted gives other answers."""
import numpy as np
import pytest

import decoding_oracle
import decoding_rounding as cases


@pytest.mark.parametrize("kind", list(cases.KINDS))
def test_products_in_32_bits_are_found(kind):
    target, draft, drafts, u = cases.product_case(kind, 50)
    t, d = target.double().numpy(), draft.double().numpy()
    assert len(drafts) >= 8
    _, accepted = decoding_oracle.verify(t, d, drafts, None, u)
    assert accepted.tolist() == [1, 0] * (len(drafts) // 2)
    _, planted = cases.verify_in_32_bits(t, d, drafts, u)
    assert not planted.any()                                  # in 32 bits u * q is p


@pytest.mark.parametrize("kind", list(cases.KINDS))
@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("v", [2001, 45001])
def test_sums_in_32_bits_are_found(kind, with_draft, v):
    target, draft, drafts, u = cases.draw_case(kind, v, with_draft)
    t, d = target.double().numpy(), None if draft is None else draft.double().numpy()
    tokens, accepted = decoding_oracle.verify(t, d, drafts, None, u)
    planted, _ = cases.verify_in_32_bits(t, d, drafts, u)
    assert not accepted.any() and (tokens[:, 0] > 1).all()    # among the small entries
    assert (planted[:, 0] != tokens[:, 0]).sum() > len(tokens) // 2
