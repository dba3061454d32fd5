"""Arguments of the decoding step's calls that a caller can get wrong, as far as the kernels see them."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nms():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_00535_amd.binding as binding

    return binding


@pytest.mark.parametrize("count,moved", [(-2147483648, 0), (-1, 0), (33, 33), (2147483647, 100)])
def test_a_list_may_say_any_number_of_moves(nms, count, moved):
    n, budget = 200, 100
    rows = torch.arange(n, dtype=torch.int32, device="cuda").view(1, 1, n, 1).clone()
    moves = torch.zeros((1, 1, budget + 1, 2), dtype=torch.int32, device="cuda")
    moves[0, 0, 0, 0] = count
    moves[0, 0, 1:, 0] = torch.arange(budget)
    moves[0, 0, 1:, 1] = torch.arange(budget, n)
    nms.nms_cache_move_batched(moves, n, 1, 1, budget, [rows])
    want = np.arange(n)
    want[:moved] = np.arange(budget, budget + moved)
    assert np.array_equal(rows.flatten().cpu().numpy(), want)
