"""Verification of drafted tokens against its definition in 64 bits: whole numbers, so the two have to be equal.

Inputs are such that rounding cannot decide: a sum of V probabilities in 64 bits is off by at most V * 2^-53 of its value in any order
(2^-35 at the largest V here), and a random number falls that close to one of V borders with a chance of V * V * 2^-52 at most
(2^-16 there; the seeds are fixed)."""
import numpy as np
import pytest
import torch

import decoding_oracle

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def nms():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_00535_amd.binding as binding

    return binding


def wide(x, pad):
    """The same values in rows that lie `pad` elements apart, with numbers between them that would be drawn if they were read."""
    if x is None:
        return None
    held = torch.full((*x.shape[:-1], x.shape[-1] + pad), 1e4, dtype=x.dtype, device="cuda")
    held[..., :x.shape[-1]] = x
    return held[..., :x.shape[-1]]


def call(nms, target, draft, drafts, counts, uniforms, pad=0, stream=None):
    s, k1, v = target.shape
    dev = lambda x, t=None: None if x is None else torch.as_tensor(x).to("cuda", t)
    tokens = torch.full((s, k1), -9, dtype=torch.int32, device="cuda")
    accepted = torch.full((s,), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((max(256, nms.nms_verify_workspace_bytes(v, s)),), 0xff, dtype=torch.uint8, device="cuda")
    nms.nms_verify_batched(wide(dev(target), pad), wide(dev(draft), pad), dev(drafts, torch.int32), dev(counts, torch.int32), k1 - 1, v, s,
                           dev(uniforms, torch.float32), tokens, accepted, ws, stream=stream)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), accepted.cpu().numpy()


def agree(nms, target, draft, drafts, counts, uniforms, pad=0):
    want = decoding_oracle.verify(target.double().numpy(), None if draft is None else draft.double().numpy(), np.asarray(drafts),
                                  None if counts is None else np.asarray(counts), np.asarray(uniforms, np.float32))
    got = call(nms, target, draft, drafts, counts, uniforms, pad)
    assert np.array_equal(got[1], want[1]), (got[1], want[1])
    assert np.array_equal(got[0], want[0]), (got[0], want[0])
    return got


def inputs(s, k, v, kind, with_draft, seed):
    g = torch.Generator().manual_seed(seed)
    logits = 2.5 * torch.randn((s, k + 1, v), generator=g)
    target = torch.softmax(logits, -1).to(TYPES[kind])
    near = torch.softmax(logits[:, :k] + 0.5 * torch.randn((s, k, v), generator=g), -1).to(TYPES[kind])
    drafts = torch.zeros((s, k), dtype=torch.int32)
    if k:
        drafts = (near.float() / torch.empty((s, k, v)).exponential_(generator=g)).argmax(-1).int()
    return target, near if with_draft else None, drafts, torch.rand((s, k + 1), generator=g)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("s,k,v,pad", [(1, 0, 1, 0), (3, 1, 2, 1), (5, 4, 63, 0), (2, 3, 64, 3), (4, 2, 65, 0), (3, 4, 1000, 24), (2, 2, 2047, 0),
                                       (2, 1, 2048, 8), (3, 2, 2049, 1), (1, 70, 300, 0), (2, 1, 50001, 0), (1, 4, 32000, 0), (300, 2, 777, 5),
                                       (1, 1, 300001, 0)])
def test_against_the_definition(nms, kind, with_draft, s, k, v, pad):
    agree(nms, *inputs(s, k, v, kind, with_draft, 7 * v + s)[:3], None, inputs(s, k, v, kind, with_draft, 7 * v + s)[3], pad)


@pytest.mark.parametrize("with_draft", [True, False])
def test_counts_of_a_padded_batch(nms, with_draft):
    target, draft, drafts, u = inputs(9, 5, 700, "f32", with_draft, 3)
    tokens, accepted = agree(nms, target, draft, drafts, [5, 0, -1, 3, 99, 1, -2147483648, 2, 4], u)
    assert accepted[2] == 0 and (tokens[2] == -1).all() and (tokens[6] == -1).all() and tokens[1, 0] >= 0


@pytest.mark.parametrize("v", [700, 60001])
def test_counts_where_there_is_no_room_for_drafts(nms, v):
    """A plain draw: counts above 0 are 0, below 0 there is no sequence."""
    target, _, drafts, u = inputs(4, 0, v, "f32", False, 9)
    tokens, accepted = agree(nms, target, None, drafts, [5, 0, -1, 2147483647], u)
    assert not accepted.any() and tokens[2, 0] == -1 and (tokens[[0, 1, 3], 0] >= 0).all()


def test_a_token_does_not_depend_on_the_batch(nms):
    target, draft, drafts, u = inputs(260, 2, 9001, "bf16", True, 5)
    tokens, accepted = call(nms, target, draft, drafts, None, u)
    for i in (0, 1, 100, 259):
        t, a = call(nms, target[i:i + 1], draft[i:i + 1], drafts[i:i + 1], None, u[i:i + 1])
        assert np.array_equal(t[0], tokens[i]) and a[0] == accepted[i]
    t, a = call(nms, target[:40], draft[:40], drafts[:40], None, u[:40])
    assert np.array_equal(t, tokens[:40]) and np.array_equal(a, accepted[:40])


@pytest.mark.parametrize("with_draft", [True, False])
def test_a_long_row_in_large_and_small_batches(nms, with_draft):
    """One launch for the large batch, two for the small one: the same tokens, and those of the definition."""
    target, draft, drafts, u = inputs(4, 1, 60001, "f16", with_draft, 31)
    few = agree(nms, target, draft, drafts, None, u)
    many = [None if x is None else x.repeat(33, *[1] * (x.dim() - 1)) for x in (target, draft, drafts, u)]
    tokens, accepted = call(nms, many[0], many[1], many[2], None, many[3])
    assert np.array_equal(tokens, np.tile(few[0], (33, 1))) and np.array_equal(accepted, np.tile(few[1], 33))


def test_nothing_left_of_the_difference_in_a_long_row(nms):
    """The target's row in the difference's place, on the route of two launches."""
    target = torch.zeros((2, 2, 100000))
    target[:, :, [40000, 99999]] = 0.5
    draft = torch.full((2, 1, 100000), 1.0)
    tokens, accepted = agree(nms, target, draft, np.array([[7], [8]]), None, np.array([[0.0, 0.4], [0.9, 0.6]]))
    assert accepted.tolist() == [0, 0] and tokens[:, 0].tolist() == [40000, 99999]
    target[:, 0] = float("nan")
    tokens, accepted = agree(nms, target, draft, np.array([[7], [8]]), [1, 0], np.array([[0.0, 0.4], [0.9, 0.6]]))
    assert tokens.tolist() == [[-1, -1], [-1, -1]]


@pytest.mark.parametrize("v", [64, 1024, 4096, 65536])
def test_borders_between_equal_entries(nms, v):
    """Entries 1 / V, V a power of two: every sum is exact, and u = j / V lies on the border, where entry j begins."""
    s = 64
    j = np.unique(np.linspace(0, v - 1, s).astype(int))
    target = torch.full((len(j), 1, v), 1.0 / v)
    tokens, _ = agree(nms, target, None, np.zeros((len(j), 0), np.int32), None, (j / v).reshape(-1, 1).astype(np.float32))
    assert np.array_equal(tokens[:, 0], j)


def test_ends_of_the_random_numbers(nms):
    """u = 0 is the first entry that has any weight, the largest u below 1 (and what lies beyond it) the last."""
    below_one = float(np.nextafter(np.float32(1), np.float32(0)))
    target = torch.zeros((6, 1, 5000))
    target[:, 0, 17] = 0.3
    target[:, 0, 2500] = 0.3
    target[:, 0, 4990] = 1e-30
    tokens, _ = call(nms, target, None, np.zeros((6, 0)), None, np.array([[0.0], [0.5], [below_one], [1.0], [2.0], [-1.0]]))
    assert tokens[:, 0].tolist() == [17, 2500, 2500, 4990, 4990, 17]


def test_entries_that_are_no_probabilities(nms):
    nan, inf = float("nan"), float("inf")
    target, draft, drafts, u = inputs(8, 2, 300, "f32", True, 11)
    target[0, 0, :100] = nan
    target[1, :, 50] = inf
    target[2, 0, ::2] = -1.0
    target[3] = nan                                     # nothing to draw from
    draft[4] = nan                                      # the draft says nothing of its own tokens: q = 0
    draft[5, 0] = inf
    target[6, :] = 0.0
    drafts[7, 0] = 300                                  # outside the vocabulary
    drafts[6, 0] = -5
    tokens, accepted = agree(nms, target, draft, drafts, None, u)
    assert tokens[3, 0] == -1 and accepted[3] == 0 and accepted[4] == 2 and accepted[7] == 0
    agree(nms, target, None, drafts, None, u)
    u[0], u[1, 0] = nan, nan                            # memory-safe, whatever comes out
    call(nms, target, draft, drafts, None, u)


def test_nothing_left_of_the_difference(nms):
    """A draft that lies above the target everywhere (rounded up): the token comes from the target's row."""
    target = torch.zeros((2, 2, 4000))
    target[:, :, 100] = target[:, :, 3900] = 0.5
    draft = torch.full((2, 1, 4000), 1.0)
    drafts = np.array([[7], [100]], np.int32)           # p = 0: refused; 0.9 * 1 < 0.5: refused
    tokens, accepted = agree(nms, target, draft, drafts, None, np.array([[0.0, 0.4], [0.9, 0.6]]))
    assert accepted.tolist() == [0, 0] and tokens[:, 0].tolist() == [100, 3900]
    target[:, 0] = 0.0
    target[:, 0, 7] = 1.0                                # all weight on the one refused token
    tokens, accepted = agree(nms, target, None, np.array([[7], [7]]), None, np.array([[1.0, 0.4], [0.5, 0.6]]))
    assert accepted.tolist() == [0, 1] and tokens[0, 0] == 7


def test_the_product_is_exact(nms):
    """u * q and p one part in 2^40 apart: equal in 32 bits, not in 64."""
    u = np.float32(1 - 2.0 ** -24)
    q = np.float32(1 - 2.0 ** -20)
    p = np.float32(np.float64(u) * np.float64(q))
    target, draft = torch.zeros((2, 2, 10)), torch.zeros((2, 1, 10))
    for i, x in enumerate((p, np.nextafter(p, np.float32(0)))):
        target[i, :, 3], draft[i, 0, 3] = float(x), float(q)
        target[i, :, 4] = 1e-3
    _, accepted = agree(nms, target, draft, np.full((2, 1), 3), None, np.full((2, 2), u))
    assert accepted[0] == int(np.float64(u) * np.float64(q) < np.float64(p)) and accepted[1] == 0


def test_rows_behind_2_to_the_32(nms):
    """The last sequence's rows begin beyond 2^32 elements (and 2^33 bytes)."""
    v, s = 4194304, 1030
    target = torch.empty((s, 1, v), dtype=torch.float16, device="cuda")
    target[-1] = 0.0
    target[-1, 0, [5, 4000000]] = 0.25
    counts = torch.full((s,), -1, dtype=torch.int32, device="cuda")
    counts[-1] = 0
    u = torch.full((s, 1), 0.75, device="cuda")
    tokens, accepted = (torch.empty(n, dtype=torch.int32, device="cuda") for n in ((s, 1), (s,)))
    ws = torch.empty(max(256, nms.nms_verify_workspace_bytes(v, s)), dtype=torch.uint8, device="cuda")
    nms.nms_verify_batched(target, None, None, counts, 0, v, s, u, tokens, accepted, ws)
    assert int(tokens[-1, 0]) == 4000000 and int(tokens[:-1].max()) == -1


@pytest.mark.parametrize("v,places", [(50, (None, 0, 63, 64, 1023)), (45001, (None, 1023))])
def test_the_most_drafts(nms, v, places):
    """NMS_MAX_DRAFTS tokens: with draft and target the same all stand, and refusals at either end of a run of 64 tests."""
    s, k = len(places), 1024
    target = torch.softmax(torch.randn((1, 1, v), generator=torch.Generator().manual_seed(v)), -1).expand(s, k + 1, v).clone()
    drafts = torch.arange(s * k, dtype=torch.int32).view(s, k) % v
    for i, place in enumerate(places):
        if place is not None:
            drafts[i, place] = -1
    _, accepted = agree(nms, target, target[:, :k], drafts, None, torch.rand((s, k + 1), generator=torch.Generator().manual_seed(1)))
    assert accepted.tolist() == [k if place is None else place for place in places]


def test_the_most_sequences(nms):
    agree(nms, *inputs(65535, 1, 3, "f32", True, 3)[:3], None, inputs(65535, 1, 3, "f32", True, 3)[3])


def test_on_another_stream_in_a_graph_and_by_a_plan(nms):
    target, draft, drafts, u = inputs(6, 3, 20011, "bf16", True, 23)
    want = call(nms, target, draft, drafts, None, u)
    d = [x.cuda() for x in (target, draft, drafts, u)]
    tokens, accepted = torch.zeros((6, 4), dtype=torch.int32, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(256, nms.nms_verify_workspace_bytes(20011, 6)), dtype=torch.uint8, device="cuda")
    plan = nms.VerifyPlan(d[0], d[1], d[2], None, 3, 20011, 6, d[3], tokens, accepted, ws)

    def check():
        torch.cuda.synchronize()
        assert np.array_equal(tokens.cpu().numpy(), want[0]) and np.array_equal(accepted.cpu().numpy(), want[1])
        tokens.zero_(), accepted.zero_()
        torch.cuda.synchronize()
    side = torch.cuda.Stream()
    nms.nms_verify_batched(d[0], d[1], d[2], None, 3, 20011, 6, d[3], tokens, accepted, ws, stream=side)
    check()
    plan()
    check()
    with torch.cuda.stream(side):
        plan()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan()
    for i in range(4):
        graph.replay()
        check()
        d[3].copy_(torch.rand((6, 4), generator=torch.Generator().manual_seed(i)))
        want = call(nms, target, draft, drafts, None, d[3].cpu())
