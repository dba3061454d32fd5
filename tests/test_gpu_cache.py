"""Eviction from a cache against its definition in 64 bits.  Keep vectors, kept counts, moves, positions and moved rows have to be equal.
Sums are one rounding of a sum in 64 bits: with weights of 8 or 11 bits and few query rows that sum is exact in any order, and with weights in
32 bits another order changes it by 2^-52 of its value, which moves the rounding of one sum in 2^27 (none at these seeds): equal as well."""
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


class Cache:
    """A cache on the GPU, its copy on the host, and what a call on it should give."""

    def __init__(self, nms, s, h, n, budget, first=0, recent=0, sums=None, positions="mixed", counts=None, lengths=None, weights=None,
                 valid=None, tensors=(), page=0, seed=0):
        g = np.random.default_rng(seed)
        self.nms, self.sizes, self.window, self.page = nms, (n, h, s, budget), (first, recent), page
        self.sums = (g.standard_exponential((s, h, n)) if sums is None else np.broadcast_to(sums, (s, h, n))).astype(np.float32)
        self.positions = g.permuted(np.broadcast_to(np.arange(n), (s, h, n)), axis=-1).astype(np.int32) if isinstance(positions, str) else positions
        self.counts, self.lengths, self.valid = (None if x is None else np.asarray(x, np.int32) for x in (counts, lengths, valid))
        self.weights, self.tensors = weights, [t(g, (s, h, n)) for t in tensors]
        self.g = g

    def upload(self):
        dev = lambda x: None if x is None else torch.as_tensor(np.ascontiguousarray(x)).cuda()
        n, h, s, budget = self.sizes
        self.d_sums, self.d_positions, self.d_counts, self.d_lengths, self.d_valid = (
            dev(x) for x in (self.sums, self.positions, self.counts, self.lengths, self.valid))
        self.d_weights = None if self.weights is None else self.weights.cuda()
        self.table, self.d_tensors = None, []
        if self.page:
            each = -(-n // self.page)
            self.table = self.g.permutation(s * each + 3)[:s * each].reshape(s, each).astype(np.int32)
            self.d_table = dev(self.table)
        for t in self.tensors:
            if self.page:
                pool = np.full((s * each + 3, h, self.page, *t.shape[3:]), 99, t.dtype)
                for i in range(s):
                    for b in range(each):
                        rows = t[i, :, b * self.page:(b + 1) * self.page]
                        pool[self.table[i, b], :, :rows.shape[1]] = rows
                self.d_tensors.append(dev(pool))
            else:
                self.d_tensors.append(dev(t))
        self.d_keep = torch.full((s, h, n), 77, dtype=torch.uint8, device="cuda")
        self.d_kept = torch.full((s,), -7, dtype=torch.int32, device="cuda")
        self.workspace = torch.full((max(256, self.nms.nms_cache_workspace_bytes(n, h, s, budget)),), 0xff, dtype=torch.uint8, device="cuda")

    def arguments(self):
        n, h, s, budget = self.sizes
        return ((self.d_sums, self.d_positions, self.d_counts, self.d_lengths, n, h, s, budget, *self.window, self.d_tensors, self.d_keep,
                 self.d_kept, self.workspace),
                dict(weights=self.d_weights, valid_tokens=self.d_valid, page_table=self.d_table if self.page else None))

    def host_tensors(self):
        n, h, s, _ = self.sizes
        if not self.page:
            return [t.cpu().numpy() for t in self.d_tensors]
        out = []
        for t in self.d_tensors:
            pool = t.cpu().numpy()
            rows = np.concatenate([pool[self.table[:, b]] for b in range(self.table.shape[1])], axis=2)
            out.append(rows[:, :, :n])
        return out

    def wanted(self):
        w = None if self.weights is None else self.weights.double().numpy()
        return decoding_oracle.evict(self.sums, self.positions, self.counts, self.lengths, w, self.valid, self.sizes[3], *self.window, self.tensors)

    def compare(self, want):
        torch.cuda.synchronize()
        keep, kept, sums, positions, tensors = want
        assert np.array_equal(self.d_kept.cpu().numpy(), kept)
        got = self.d_keep.cpu().numpy()
        assert np.array_equal(got, keep), f"{(got != keep).sum()} differing keep bytes"
        assert np.array_equal(self.d_sums.cpu().numpy(), sums, equal_nan=True)
        if positions is not None:
            assert np.array_equal(self.d_positions.cpu().numpy(), positions)
        for got, t in zip(self.host_tensors(), tensors):
            assert np.array_equal(got, t)

    def evict(self):
        self.upload()
        args, options = self.arguments()
        self.nms.nms_cache_evict_batched(*args, **options)
        self.compare(self.wanted())

    def steps(self):
        """The step calls: keep vector and list of moves, sums added but not moved; then the rows by that list."""
        self.upload()
        n, h, s, budget = self.sizes
        moves = torch.full((s, h, self.nms.nms_cache_moves_max(n, budget) + 1, 2), -5, dtype=torch.int32, device="cuda")
        (sums, positions, counts, lengths, *_), options = self.arguments()
        table = options.pop("page_table")
        self.nms.nms_cache_keep_batched(sums, positions, counts, lengths, n, h, s, budget, *self.window, self.d_keep, self.d_kept, moves,
                                        self.workspace, **options)
        w = None if self.weights is None else self.weights.double().numpy()
        added = decoding_oracle.add_weights(self.sums, w, self.counts, self.valid)
        keep, kept, wanted = decoding_oracle.keep(added, self.positions, self.counts, self.lengths, budget, *self.window)
        self.compare((keep, kept, added, self.positions, self.tensors))
        got = moves.cpu().numpy()
        for i in range(s):
            for j in range(h):
                m = len(wanted[i][j])
                assert got[i, j, 0].tolist() == [m, 0]
                assert got[i, j, 1:m + 1].tolist() == [list(x) for x in wanted[i][j]]
                assert (got[i, j, m + 1:] == -5).all()
        self.nms.nms_cache_move_batched(moves, n, h, s, budget, self.d_tensors, page_table=table)
        self.compare((keep, kept, added, self.positions, self.wanted()[4]))


def rows_of(dtype, *row):
    if np.dtype(dtype).kind == "f":
        return lambda g, shape: g.standard_normal((*shape, *row)).astype(dtype)
    return lambda g, shape: g.integers(0, np.iinfo(dtype).max, (*shape, *row), dtype=dtype)


def attention(s, h, group, tokens, columns, kind, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.softmax(2.0 * torch.randn((s, h, group, tokens, columns), generator=g), -1).to(TYPES[kind])


SIZES = [(1, 1, 1, 1), (1, 1, 1, 0), (2, 1, 2, 1), (1, 3, 63, 20), (2, 2, 64, 64), (1, 2, 65, 64), (1, 1, 65, 200), (3, 2, 127, 1), (2, 3, 1000, 999), (1, 8, 1025, 1024),
         (2, 2, 1024, 0), (1, 2, 2047, 512), (2, 1, 4097, 4000), (2, 2, 5003, 1501), (1, 2, 9001, 100), (1, 1, 20011, 19000), (1, 2, 33333, 4096), (1, 1, 65536, 32768), (1, 1, 66001, 8192), (1, 2, 1025, 961), (2, 2, 8192, 8128), (2, 1, 16385, 16000), (300, 1, 200, 150)]


@pytest.mark.parametrize("s,h,n,budget", SIZES)
def test_sizes(nms, s, h, n, budget):
    Cache(nms, s, h, n, budget, first=min(2, budget), recent=min(16, budget // 4), tensors=(rows_of("float16", 8),), seed=n).evict()
    Cache(nms, s, h, n, budget, first=1, recent=5, positions=None, tensors=(rows_of("int32", 1),), seed=n + 1).steps()


@pytest.mark.parametrize("s,h,n,budget", [x for x in SIZES if x[2] > 60])
@pytest.mark.parametrize("sums", [0.0, float("nan"), float("inf"), float("-inf"), -1.5])
def test_ties_everywhere(nms, s, h, n, budget, sums):
    """Equal sums: the lowest slots stay, so nothing but protected rows moves."""
    Cache(nms, s, h, n, budget, sums=sums, seed=1).steps()
    Cache(nms, s, h, n, budget, sums=sums, first=3, recent=7, tensors=(rows_of("uint8", 4),), seed=2).evict()


@pytest.mark.parametrize("s,h,n,budget", [(4, 8, 17001, 3000), (3, 11, 17001, 16990), (40, 8, 1100, 600), (256, 8, 1500, 1400), (64, 16, 1700, 900), (130, 8, 300, 299), (1, 33, 33000, 32990), (5, 8, 20000, 3000), (1, 33, 32768, 16384)])
def test_routes_of_large_batches(nms, s, h, n, budget):
    """Batches on either side of the rules: several workgroups to a frame or one, one vector of slots to a lane or two, weights with the cut or before it."""
    for tokens in (1, 4):
        Cache(nms, s, h, n, budget, first=3, recent=20, counts=np.random.default_rng(n).integers(0, n + 1, s), weights=attention(s, h, 4, tokens, n, "bf16", n),
              tensors=(rows_of("uint8", 4),), seed=n).evict()


@pytest.mark.parametrize("n,budget", [(900, 500), (5000, 4900), (30000, 8000), (50000, 3)])
@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1.0, 300.0, 1e6, 1e35])
def test_sums_of_every_size(nms, n, budget, scale):
    """Sums far from those that the counting expects, alone and next to such, below zero and beside protected rows and infinite ones."""
    c = Cache(nms, 2, 2, n, budget, 1, budget // 3, tensors=(rows_of("uint8", 4),), seed=n)
    c.sums[0] *= np.float32(scale)
    c.sums[1, :, ::2] *= np.float32(-scale)
    c.sums[1, :, ::7] = np.inf
    c.evict()
    c.window = (0, 0)
    c.steps()


@pytest.mark.parametrize("n", [900, 3000, 20000, 50000])
@pytest.mark.parametrize("ties", [1, 2, 60])
def test_one_row_goes(nms, n, ties):
    """A step of one token: the least sum goes, of several such the highest slot."""
    c = Cache(nms, 2, 2, n, n - 1, recent=5, tensors=(rows_of("float16", 32),), seed=n)
    c.sums += 1.0
    c.sums[:, :, np.random.default_rng(1).choice(n, ties, replace=False)] = 0.25
    c.evict()
    c.positions[:] = 0                                   # all protected: the last slot's row goes
    c.window = (1, 0)
    c.evict()


@pytest.mark.parametrize("n,budget", [(700, 300), (4097, 1000), (9001, 8000), (40000, 5000)])
def test_few_values_and_every_kind_of_sum(nms, n, budget):
    g = np.random.default_rng(n)
    few = g.integers(0, 4, (2, 3, n)).astype(np.float32)
    Cache(nms, 2, 3, n, budget, recent=9, sums=few, tensors=(rows_of("float32", 2),)).evict()
    kinds = np.array([np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-45, -1e-45, 1.0, -1.0, 3e38, -3e38], np.float32)
    sums = kinds[g.integers(0, len(kinds), (2, 3, n))]
    sums[0, 0] = np.frombuffer(g.bytes(4 * n), np.float32)   # any bits
    Cache(nms, 2, 3, n, budget, first=3, sums=sums, tensors=(rows_of("float32", 2),)).evict()
    Cache(nms, 2, 3, n, budget, sums=np.where(sums == 0, sums, -0.0), seed=4).steps()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("group,tokens", [(1, 1), (4, 1), (3, 5), (2, 33)])
@pytest.mark.parametrize("n,columns", [(257, 257), (1030, 1030), (1030, 500), (1030, 2001), (10007, 10007)])
def test_weights(nms, kind, group, tokens, n, columns):
    w = attention(2, 2, group, tokens, columns, kind, n + tokens)
    Cache(nms, 2, 2, n, n // 3, recent=8, weights=w, tensors=(rows_of("float16", 16),)).evict()
    Cache(nms, 2, 2, n, n // 2, first=1, weights=w, valid=[tokens // 2, 99], counts=[n - 3, n // 2], lengths=[4 * n, 4 * n]).steps()
    Cache(nms, 2, 2, n, n // 2, weights=w, valid=[0, -4], counts=[0, -1], tensors=(rows_of("float16", 16),)).evict()


def test_weights_that_are_no_numbers(nms):
    """A query row that was masked as a whole comes out of a softmax as NaN, and slots behind the count hold anything."""
    n = 1500
    w = attention(2, 2, 2, 4, n, "bf16", 1)
    w[0, 0, 1, 2] = float("nan")
    w[1, 1, :, :, 5] = float("inf")
    w[:, :, :, :, 1200:] = float("nan")
    w[1, 0, 0, 0, 0] = torch.finfo(torch.bfloat16).min
    Cache(nms, 2, 2, n, 700, weights=w, counts=[1200, 1100], tensors=(rows_of("float16", 16),)).evict()


@pytest.mark.parametrize("kind", list(TYPES))
def test_rows_of_weights_that_lie_apart(nms, kind):
    n, room = 600, attention(2, 3, 2, 2, 777, kind, 5)
    c = Cache(nms, 2, 3, n, 200, weights=room[..., 3:603], tensors=(rows_of("float16", 4),))
    c.upload()
    c.d_weights = room.cuda()[..., 3:603]
    args, options = c.arguments()
    nms.nms_cache_evict_batched(*args, **options)
    c.compare(c.wanted())


@pytest.mark.parametrize("first,recent", [(0, 0), (4, 64), (500, 700), (0, 5000), (1 << 30, 0), (0, 2147483647)])
def test_windows(nms, first, recent):
    """Protected rows outrank all sums, lower slots first; there may be more of them than the budget holds."""
    c = Cache(nms, 2, 2, 1300, 900, first, recent, lengths=[1300, 9000], tensors=(rows_of("uint8", 20),))
    c.sums[0, 0, :100] = np.inf
    c.evict()
    Cache(nms, 2, 2, 1300, 900, first, recent, positions=None, lengths=[1300, -2147483648]).steps()


def test_positions_at_the_ends_of_their_range(nms):
    g = np.random.default_rng(0)
    p = np.frombuffer(g.bytes(4 * 2 * 800), np.int32).reshape(1, 2, 800).copy()
    p[0, 0, :4] = [2147483647, -2147483648, 0, -1]
    for length in (2147483647, -2147483648, 0):
        Cache(nms, 1, 2, 800, 300, 2147483647 if length == 0 else 5, 2147483647, positions=p, lengths=[length]).evict()


@pytest.mark.parametrize("page", [0, 1, 16, 24])
def test_tensors_of_every_row_size(nms, page):
    rows = [rows_of("uint8", 1), rows_of("uint8", 2), rows_of("uint8", 7), rows_of("float16", 10), rows_of("float16", 64), rows_of("float32", 3, 5),
            rows_of("float64", 3), rows_of("uint8", 4096)]
    Cache(nms, 2, 3, 301, 150, 2, 9, counts=[301, 280], lengths=[301, 280], tensors=rows, page=page).evict()
    Cache(nms, 2, 3, 301, 150, 2, 9, counts=[301, 150], lengths=[301, 280], tensors=rows[:1], page=page).steps()
    Cache(nms, 2, 3, 301, 300, 2, 9, tensors=(), page=page).evict()


def test_other_orders_of_strides(nms):
    """[sequence, slot, head, row] seen as [sequence, head, slot, row], a cache with more heads and slots than the call names, and rows
    that begin at odd addresses."""
    s, h, n = 2, 3, 500
    c = Cache(nms, s, h, n, 200, recent=4, tensors=(rows_of("float16", 40), rows_of("uint8", 48), rows_of("uint8", 33)))
    c.upload()
    want = c.wanted()
    a = torch.zeros((s, n, h, 40), dtype=torch.float16, device="cuda")
    a.copy_(c.d_tensors[0].transpose(1, 2))
    b = torch.full((s + 1, h + 2, n + 7, 64), 3, dtype=torch.uint8, device="cuda")
    b[:s, :h, :n, 8:56] = c.d_tensors[1]
    d = torch.full((s * h * n * 33 + 1,), 5, dtype=torch.uint8, device="cuda")[1:].view(s, h, n, 33)
    d.copy_(c.d_tensors[2])
    c.d_tensors = [a.transpose(1, 2), b[:, :, :, 8:56], d]
    args, options = c.arguments()
    nms.nms_cache_evict_batched(*args, **options)
    torch.cuda.synchronize()
    assert np.array_equal(b[s:].cpu().numpy(), np.full((1, h + 2, n + 7, 64), 3)) and int(b[:s, h:].max()) == 3 and int(b[:s, :h, n:].max()) == 3
    assert int(b[:, :, :, :8].max()) == 3 and int(b[:, :, :, 56:].max()) == 3
    c.d_tensors[1] = b[:s, :h, :n, 8:56]
    c.compare(want)


def test_rows_behind_2_to_the_32(nms):
    """A tensor of more than 2^32 bytes: the kept rows of the last slots move to the first."""
    n, row = 70001, 65536
    t = torch.zeros((1, 1, n, row), dtype=torch.uint8, device="cuda")
    t[0, 0, -3:] = torch.arange(1, 4, device="cuda", dtype=torch.uint8)[:, None]
    sums = torch.zeros((1, 1, n), device="cuda")
    sums[0, 0, -3:] = 5.0
    positions = torch.arange(n, dtype=torch.int32, device="cuda").view(1, 1, n)
    ws = torch.empty(nms.nms_cache_workspace_bytes(n, 1, 1, 3), dtype=torch.uint8, device="cuda")
    nms.nms_cache_evict_batched(sums, positions, None, None, n, 1, 1, 3, 0, 0, [t], None, None, ws)
    assert [int(t[0, 0, i].min()) for i in range(3)] == [1, 2, 3] and [int(t[0, 0, i].max()) for i in range(3)] == [1, 2, 3]
    assert positions[0, 0, :3].tolist() == [n - 3, n - 2, n - 1] and sums[0, 0, :4].tolist() == [5.0, 5.0, 5.0, 0.0]


def test_what_is_not_wanted_may_be_left_out(nms):
    c = Cache(nms, 2, 2, 900, 300, recent=10, tensors=(rows_of("float16", 8),))
    c.upload()
    n, h, s, budget = c.sizes
    ws = torch.empty(nms.nms_cache_workspace_bytes(n, h, s, budget), dtype=torch.uint8, device="cuda")
    nms.nms_cache_evict_batched(c.d_sums, c.d_positions, None, None, n, h, s, budget, 0, 10, c.d_tensors, None, None, ws)
    want = c.wanted()
    c.d_keep.copy_(torch.from_numpy(want[0])), c.d_kept.copy_(torch.from_numpy(want[1]))
    c.compare(want)
    before = c.d_sums.clone()
    nms.nms_cache_keep_batched(c.d_sums, c.d_positions, None, None, n, h, s, budget, 0, 10, None, None, None, ws)
    assert torch.equal(before, c.d_sums)
    # without positions: the slots are the places, and rows may still move
    c = Cache(nms, 2, 2, 900, 300, first=6, positions=None, tensors=(rows_of("float16", 8),))
    c.evict()


def test_moves_that_name_no_slot_of_the_list_are_left_out(nms):
    """A list from elsewhere: pairs outside the slots that the sizes allow, and page numbers outside the pool, move nothing."""
    n, budget, page = 64, 32, 16
    t = torch.arange(6 * 16, dtype=torch.int32, device="cuda").view(6, 1, 16, 1).clone()
    before = t.clone()
    moves = torch.zeros((1, 1, 33, 2), dtype=torch.int32, device="cuda")
    bad = [(-1, 40), (32, 40), (5, 64), (5, 31), (40, 50), (-2147483648, 2147483647), (7, -3)]
    moves[0, 0, 0, 0] = 1000
    moves[0, 0, 1:] = torch.tensor((bad * 5)[:32], dtype=torch.int32)
    nms.nms_cache_move_batched(moves, n, 1, 1, budget, [t], page_table=torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device="cuda"))
    assert torch.equal(t, before)
    moves[0, 0, 0, 0] = -3
    nms.nms_cache_move_batched(moves, n, 1, 1, budget, [t], page_table=torch.tensor([[0, 1, 2, 3]], dtype=torch.int32, device="cuda"))
    assert torch.equal(t, before)
    moves[0, 0, :4] = torch.tensor([[3, 0], [0, 32], [16, 33], [17, 48]], dtype=torch.int32)
    nms.nms_cache_move_batched(moves, n, 1, 1, budget, [t], page_table=torch.tensor([[-1, 5, 6, 2147483647]], dtype=torch.int32, device="cuda"))
    assert torch.equal(t, before)
    nms.nms_cache_move_batched(moves, n, 1, 1, budget, [t], page_table=torch.tensor([[-1, 5, 2, 6]], dtype=torch.int32, device="cuda"))
    before[5, 0, 0] = before[2, 0, 1]
    assert torch.equal(t, before)


def test_a_decoding_loop(nms):
    """Verification and eviction as they are used: a step writes its rows behind the cached ones, verification says how many of
    them stand, eviction goes by that and leaves the cache ready for the next step."""
    s, h, group, k, v, budget, d = 4, 2, 2, 3, 500, 96, 16
    n_max = budget + k + 1
    g = torch.Generator().manual_seed(0)
    c = Cache(nms, s, h, n_max, budget, 2, 24, counts=[budget] * s, lengths=[budget] * s, valid=[0] * s,
              weights=torch.zeros((s, h, group, k + 1, n_max)), tensors=(rows_of("float32", d), rows_of("float32", d)))
    c.sums[:, :, budget:] = 0
    c.positions = np.broadcast_to(np.arange(n_max, dtype=np.int32), (s, h, n_max)).copy()
    c.upload()
    filled, length = np.full(s, budget), np.full(s, budget)
    for step in range(60):
        target = torch.softmax(torch.randn((s, k + 1, v), generator=g), -1)
        draft = torch.softmax(target[:, :k].log() + 0.5 * torch.randn((s, k, v), generator=g), -1)
        drafts = torch.multinomial(draft.view(-1, v), 1, generator=g).view(s, k).int()
        u = torch.rand((s, k + 1), generator=g)
        tokens = torch.empty((s, k + 1), dtype=torch.int32, device="cuda")
        accepted = torch.empty((s,), dtype=torch.int32, device="cuda")
        ws = torch.empty(max(256, nms.nms_verify_workspace_bytes(v, s)), dtype=torch.uint8, device="cuda")
        nms.nms_verify_batched(target.cuda(), draft.cuda(), drafts.cuda(), None, k, v, s, u.cuda(), tokens, accepted, ws)
        want_tokens, want_accepted = decoding_oracle.verify(target.double().numpy(), draft.double().numpy(), drafts.numpy(), None, u.numpy())
        assert np.array_equal(tokens.cpu().numpy(), want_tokens) and np.array_equal(accepted.cpu().numpy(), want_accepted)
        # the step's k + 1 rows, of which the accepted ones and the one before them stand
        stands = accepted + 1
        weights = attention(s, h, group, k + 1, n_max, "f16", step)
        for i in range(s):
            for t in c.tensors:
                t[i, :, filled[i]:filled[i] + k + 1] = torch.randn((h, k + 1, d), generator=g).numpy()
            c.positions[i, :, filled[i]:filled[i] + k + 1] = length[i] + np.arange(k + 1)
        for mine, theirs in zip([*c.tensors, c.positions], [*c.d_tensors, c.d_positions]):
            theirs.copy_(torch.from_numpy(mine))
        c.weights, c.d_weights, c.d_valid = weights, weights.cuda(), stands
        c.d_counts, c.d_lengths = torch.from_numpy(filled).cuda().int() + stands, torch.from_numpy(length).cuda().int() + stands
        c.counts, c.lengths, c.valid = c.d_counts.cpu().numpy(), c.d_lengths.cpu().numpy(), stands.cpu().numpy()
        args, options = c.arguments()
        nms.nms_cache_evict_batched(*args, **options)
        want = c.wanted()
        c.compare(want)
        _, kept, c.sums, c.positions, c.tensors = want
        filled, length = kept.copy(), c.lengths
        # what stays are 96 different tokens of the text, the newest 24 and the first two among them
        for i in range(s):
            for j in range(h):
                p = np.sort(c.positions[i, j, :budget])
                assert len(np.unique(p)) == budget and (p[-24:] == length[i] - 24 + np.arange(24)).all() and p[:2].tolist() == [0, 1]
        assert not c.sums[:, :, budget:].any()


def test_on_another_stream_in_graphs_and_by_a_plan(nms):
    """A graph captured once and replayed on other contents, two graphs with one workspace, and eager calls between their replays."""
    n, h, s, budget = 1100, 2, 3, 700
    w = attention(s, h, 2, 1, n, "bf16", 9)

    def fresh(seed):
        return Cache(nms, s, h, n, budget, 2, 30, counts=[1100, 900, 300], lengths=[1100, 900, 300], weights=w,
                     tensors=(rows_of("float16", 32), rows_of("uint8", 12)), seed=seed)
    a, b = fresh(1), fresh(2)
    a.upload(), b.upload()
    b.workspace = a.workspace
    plans = [nms.CachePlan(*x.arguments()[0], **x.arguments()[1]) for x in (a, b)]
    side = torch.cuda.Stream()
    graphs = []
    for plan in plans:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan()
        graphs.append(graph)

    def load(cache, seed):
        other = fresh(seed)
        cache.sums, cache.positions, cache.tensors = other.sums, other.positions, other.tensors
        for mine, theirs in zip([cache.sums, cache.positions, *cache.tensors], [cache.d_sums, cache.d_positions, *cache.d_tensors]):
            theirs.copy_(torch.from_numpy(mine))
    for i in range(4):
        load(a, 10 + i), load(b, 20 + i)
        graphs[0].replay(), graphs[1].replay()
        a.compare(a.wanted()), b.compare(b.wanted())
        load(a, 30 + i)
        plans[0]()
        a.compare(a.wanted())
        load(b, 40 + i)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            plans[1]()
        b.compare(b.wanted())
        load(a, 50 + i)
        torch.cuda.synchronize()
        args, options = a.arguments()
        nms.nms_cache_evict_batched(*args, **options, stream=side)
        a.compare(a.wanted())


@pytest.mark.parametrize("budget,sums", [(100003, None), (60, None), (1048575, None), (524288, 0.0), (3, float("nan"))])
def test_the_most_slots(nms, budget, sums):
    """A frame of NMS_MAX_SLOTS: few moves and as many as there can be, equal sums that no bin parts."""
    options = {} if sums is None else dict(sums=sums)
    Cache(nms, 1, 1, 1048576, budget, first=2, recent=min(50, budget), tensors=(rows_of("uint8", 4),), seed=budget, **options).evict()


@pytest.mark.parametrize("tokens", [1, 7])
def test_the_most_frames(nms, tokens):
    """NMS_MAX_FRAMES frames, with the weights in the launch of the cut (three query rows) and in one of their own (21)."""
    Cache(nms, 65535, 1, 9, 4, first=1, recent=1, weights=attention(65535, 1, 3, tokens, 9, "bf16", tokens), tensors=(rows_of("uint8", 4),), seed=tokens).evict()


def test_two_calls_at_once(nms):
    """Two streams, each with its own buffers and workspace."""
    caches = [Cache(nms, 2, 8, 6000, 1000, 4, 64, weights=attention(2, 8, 2, 4, 6000, "f16", i), tensors=(rows_of("float16", 64),), seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in caches]
    for c in caches:
        c.upload()
    torch.cuda.synchronize()
    for c, stream in zip(caches, streams):
        args, options = c.arguments()
        nms.nms_cache_evict_batched(*args, **options, stream=stream)
    for c in caches:
        c.compare(c.wanted())


def test_sizes_of_nothing(nms):
    z = torch.zeros(256, dtype=torch.uint8, device="cuda")
    f = torch.zeros(4, device="cuda")
    for n, h, s in ((0, 2, 2), (5, 0, 2), (5, 2, 0)):
        nms.nms_cache_evict_batched(f, None, None, None, n, h, s, 3, 0, 0, [], None, None, z)
        nms.nms_cache_keep_batched(f, None, None, None, n, h, s, 3, 0, 0, None, None, None, z)
    nms.nms_cache_move_batched(torch.zeros(64, dtype=torch.int32, device="cuda"), 0, 2, 2, 3, [])
    torch.cuda.synchronize()
