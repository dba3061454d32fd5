"""Verification multiplies, subtracts and adds in 64 bits: cases whose answers 32 bits would change (tests/test_decoding_rounding_host.py plants that), on
the route of one launch and of two.  All of it is exact in 64 bits, so the answers have to be equal."""
import numpy as np
import pytest
import torch

import decoding_oracle
import decoding_rounding as cases

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nms():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_00535_amd.binding as binding

    return binding


def verify(nms, target, draft, drafts, uniforms):
    s, k1, v = target.shape
    tokens, accepted = torch.full((s, k1), -9, dtype=torch.int32, device="cuda"), torch.full((s,), -9, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(256, nms.nms_verify_workspace_bytes(v, s)), dtype=torch.uint8, device="cuda")
    nms.nms_verify_batched(target.cuda(), None if draft is None else draft.cuda(), torch.from_numpy(drafts).cuda(), None, k1 - 1, v, s,
                           torch.from_numpy(uniforms).cuda(), tokens, accepted, ws)
    return tokens.cpu().numpy(), accepted.cpu().numpy()


@pytest.mark.parametrize("kind", list(cases.KINDS))
@pytest.mark.parametrize("v", [50, 45001])
def test_products(nms, kind, v):
    target, draft, drafts, u = cases.product_case(kind, v)
    tokens, accepted = verify(nms, target, draft, drafts, u)
    assert accepted.tolist() == [1, 0] * (len(drafts) // 2)
    assert np.array_equal(tokens, decoding_oracle.verify(target.double().numpy(), draft.double().numpy(), drafts, None, u)[0])


@pytest.mark.parametrize("kind", list(cases.KINDS))
@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("v", [2001, 45001])
def test_sums(nms, kind, with_draft, v):
    target, draft, drafts, u = cases.draw_case(kind, v, with_draft)
    assert (nms.nms_verify_workspace_bytes(v, len(u)) > 0) == (v == 45001)
    tokens, accepted = verify(nms, target, draft, drafts, u)
    want = decoding_oracle.verify(target.double().numpy(), None if draft is None else draft.double().numpy(), drafts, None, u)
    assert np.array_equal(accepted, want[1]) and np.array_equal(tokens, want[0]), (tokens[:, 0] - want[0][:, 0])
