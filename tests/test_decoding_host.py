"""The decoding step's choices without a GPU: keys, sizes and addresses compiled by a plain host compiler with the sanitizers on, and every
refusal of the C ABI and of the binding, all before anything is launched."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    exe = tmp_path_factory.mktemp("host") / "decoding_driver"
    subprocess.run(["g++", "-std=c++17", "-O2", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "host", "decoding_driver.cpp"), "-o", str(exe)], check=True)

    def run(what, lines):
        proc = subprocess.run([str(exe), what], input="\n".join(lines) + "\n", capture_output=True, text=True)
        assert proc.returncode == 0, proc.stderr[-2000:]
        return proc.stdout.split("\n")[:-1]
    return run


@pytest.fixture(scope="module")
def nms():
    from paper_2502_00535_amd import build as nms_build

    if nms_build.is_stale():
        nms_build.build_library()
    import paper_2502_00535_amd.binding as binding

    return binding


def test_keys_order_every_kind_of_sum(driver):
    g = np.random.default_rng(0)
    values = np.concatenate([np.frombuffer(g.bytes(4 * 3000), np.float32), g.standard_normal(500).astype(np.float32),
                             np.array([0.0, -0.0, np.inf, -np.inf, np.nan, 1e-45, -1e-45, 3.4e38, -3.4e38], np.float32)])
    bits = values.view(np.uint32)
    keys = np.array([int(x) for x in driver("keys", [f"{b:x}" for b in bits])], np.int64)
    nan = np.isnan(values)
    assert (keys[nan] == 0).all() and (keys[~nan] > 0).all() and keys.max() < 0xffffffff
    order = np.argsort(keys[~nan], kind="stable")
    with np.errstate(invalid="ignore"):
        v = values[~nan].astype(np.float64)
    assert (np.diff(v[order]) >= 0).all()
    assert np.array_equal(np.diff(v[order]) == 0, np.diff(keys[~nan][order]) == 0)   # equal sums, both zeros, equal keys


def test_moves_and_scratch(driver, nms):
    sizes = [(0, 0), (1, 1), (10, 3), (10, 7), (10, 10), (10, 50), (10, 0), (1048576, 500000), (5, 2147483647)]
    for (n, b), line in zip(sizes, driver("moves", [f"{n} {b}" for n, b in sizes])):
        moves, scratch = (int(x) for x in line.split())
        assert moves == max(0, min(b, n - b)) == nms.nms_cache_moves_max(n, b)
        assert scratch >= 3 * 8 * (moves + 1) and scratch % 256 == 0
        assert n == 0 or nms.nms_cache_workspace_bytes(n, 3, 1, b) >= scratch
    assert nms.nms_cache_moves_max(-1, 3) == -1 and nms.nms_cache_moves_max(1048577, 3) == -1 and nms.nms_cache_moves_max(3, -1) == -1
    assert nms.nms_cache_workspace_bytes(1048577, 1, 1, 5) == 0 and nms.nms_cache_workspace_bytes(10, 256, 256, 5) == 0
    assert nms.nms_verify_workspace_bytes(0, 1) == 0 and nms.nms_verify_workspace_bytes(4194305, 1) == 0 and nms.nms_verify_workspace_bytes(5, 65536) == 0


def test_routes_of_eviction_fit_their_kernels(driver):
    """One workgroup: at most sixteen wavefronts whose lanes hold every slot, 16-bit slot numbers, the lists within 160 KiB of LDS.  Several: parts that
    cover the frame with one to spare, 16-bit counts, a list of parts within the cut's LDS, and scratch without overlaps."""
    sizes = sorted({1, 2, 255, 256, 1023, 1024, 1025, 2048, 3583, 3584, 3585, 4096, 4097, 8192, 8193, 16384, 16385, 32768, 32769, 65536, 100003, 524288, 1048575, 1048576})
    cases = [(n, f, r, m) for n in sizes for f in (1, 8, 32, 33, 300, 512, 1024, 65535) for r in (1, 8, 9, 16, 17) for m in (0, 1)]
    for (n, f, rows, many), line in zip(cases, driver("route", [" ".join(map(str, c)) for c in cases])):
        split, vecs, together, part, parts, keys, bins, cuts, stays, total = (int(x) for x in line.split())
        if not split:
            waves = -(-n // (256 * vecs))
            assert vecs in (1, 2, 4, 8) and 1 <= waves <= 16 and n <= 65536
            most_moves = n // 2
            assert 8192 + 1024 + most_moves * (8 if together else 4) <= 160 * 1024
            assert not together or vecs <= 4
        else:
            assert not together
        assert part in (1024, 2048, 4096) and (parts - 1) * part >= n and parts <= 2048
        assert bins - keys >= 4 * n * f and cuts - bins >= f * parts * 4096 and stays - cuts >= 8 * f and total - stays >= 4 * f * parts
        assert all(x % 256 == 0 for x in (keys, bins, cuts, stays, total))


def test_routes_of_verification(driver, nms):
    cases = [(v, s) for v in (1, 2048, 2049, 40960, 40961, 131072, 4194304) for s in (1, 127, 128, 65535)]
    for (v, s), line in zip(cases, driver("verify", [f"{v} {s}" for v, s in cases])):
        segments, one, sums, scratch = (int(x) for x in line.split())
        assert segments == -(-v // 2048) <= 2048 and one == (segments <= 20 or s >= 128)
        assert scratch == nms.nms_verify_workspace_bytes(v, s) and (scratch == 0) == one
        assert one or (sums >= 8 * segments * s and scratch - sums >= 8 * s and sums % 256 == 0)


def test_pieces_divide_every_address(driver):
    cases = [(4096, 256, 1 << 20, 4096, 256, 16), (4096, 80, 8000, 800, 80, 16), (4096, 84, 8400, 840, 84, 4), (4104, 256, 4096, 512, 256, 8),
             (4097, 256, 4096, 512, 256, 1), (4096, 7, 70, 7, 7, 1), (4096, 20, 4000, 200, 20, 4), (4096, 10, 100, 20, 10, 2), (4096, 64, 0, 0, 64, 16)]
    for (*case, want), line in zip(cases, driver("piece", [" ".join(map(str, c[:5])) for c in cases])):
        assert int(line) == want, case


def test_addresses_and_bad_pages(driver):
    table = "3 -1 5 6 0 2147483647 1 -2147483648"
    plain = (1 << 40, 1 << 20, 1 << 33)
    cases = [(*plain, 1, 2, 70000, 0, 0, (1 << 40) + 2 * (1 << 20) + 70000 * (1 << 33)),
             (1000, 100, 10, 0, 1, 3, 16, 6, 3 * 1000 + 100 + 30),        # page 3
             (1000, 100, 10, 0, 1, 17, 16, 6, -1),                        # page -1
             (1000, 100, 10, 0, 0, 33, 16, 6, 5 * 1000 + 10),
             (1000, 100, 10, 0, 0, 50, 16, 6, -1),                        # page 6 of 6
             (1000, 100, 10, 1, 0, 15, 16, 6, 150),
             (1000, 100, 10, 1, 0, 16, 16, 6, -1), (1000, 100, 10, 1, 0, 63, 16, 6, -1),
             (1 << 32, 100, 10, 1, 3, 40, 16, 6, (1 << 32) + 300 + 80)]
    for (*case, want), line in zip(cases, driver("offset", [" ".join(map(str, c[:8])) + " " + table for c in cases])):
        assert int(line) == want, case


def test_refusals_of_verification(nms):
    L, p, bad, large = nms.lib, ctypes.c_void_p(0x1000), nms.NMS_ERR_INVALID_ARG, nms.NMS_ERR_TOO_LARGE

    def call(target=p, t_row=100, draft=p, d_row=100, kind=0, drafts=p, counts=None, k=2, v=100, s=3, u=p, tokens=p, accepted=p, ws=p, size=1 << 40):
        return L.nms_verify_batched(target, t_row, draft, d_row, kind, drafts, counts, k, v, s, u, tokens, accepted, ws, size, None)
    for wrong in (dict(kind=3), dict(kind=-1), dict(k=-1), dict(v=0), dict(v=-5), dict(s=-1), dict(t_row=99), dict(d_row=99), dict(target=None),
                  dict(drafts=None), dict(u=None), dict(tokens=None), dict(accepted=None)):
        assert call(**wrong) == bad, wrong
    assert call(k=1025) == large and call(v=4194305, t_row=1 << 40, d_row=1 << 40) == large and call(s=65536) == large
    assert call(s=0, target=None, u=None, tokens=None, accepted=None, ws=None, size=0) == nms.NMS_OK
    need = nms.nms_verify_workspace_bytes(100, 3)
    if need:
        assert call(ws=None) == nms.NMS_ERR_WORKSPACE and call(size=need - 1) == nms.NMS_ERR_WORKSPACE
        assert call(ws=ctypes.c_void_p(0x1010)) == nms.NMS_ERR_WORKSPACE


def test_refusals_of_eviction(nms):
    L, p, bad, large = nms.lib, ctypes.c_void_p(0x1000), nms.NMS_ERR_INVALID_ARG, nms.NMS_ERR_TOO_LARGE
    tensor, pages = nms.NmsCacheTensor(0x1000, 16, 4096, 1024, 16), nms.NmsCachePages(0x1000, 4, 16, 9, 0)

    def weights(at=0x1000, row=50, kind=0, group=1, tokens=1, columns=50):
        return nms.NmsCacheWeights(at, row, kind, group, tokens, columns, None)

    def evict(sums=p, positions=p, n=50, h=2, s=3, w=None, budget=10, first=0, recent=4, t=tensor, many=1, pg=None, ws=p, size=1 << 40):
        return L.nms_cache_evict_batched(sums, positions, None, None, n, h, s, w, budget, first, recent, t, many, pg, None, None, ws, size, None)

    def keep(sums=p, n=50, h=2, s=3, w=None, budget=10, first=0, recent=4, ws=p, size=1 << 40, **_):
        return L.nms_cache_keep_batched(sums, None, None, None, n, h, s, w, budget, first, recent, None, None, None, ws, size, None)

    def move(moves=p, n=50, h=2, s=3, budget=10, t=tensor, many=1, pg=None):
        return L.nms_cache_move_batched(moves, n, h, s, budget, t, many, pg, None)
    for wrong in (dict(n=-1), dict(h=-1), dict(s=-1), dict(budget=-1)):
        assert evict(**wrong) == bad and keep(**wrong) == bad and move(**wrong) == bad, wrong
    for wrong in (dict(first=-1), dict(recent=-1), dict(sums=None), dict(w=weights(kind=3)), dict(w=weights(group=-1)), dict(w=weights(tokens=-1)),
                  dict(w=weights(columns=-1)), dict(w=weights(row=49)), dict(w=weights(at=None))):
        assert evict(**wrong) == bad and keep(**wrong) == bad, wrong
    for wrong in (dict(n=1048577), dict(h=65536, s=1), dict(h=300, s=300), dict(h=2147483647, s=2147483647)):
        assert evict(**wrong) == large and keep(**wrong) == large and move(**wrong) == large, wrong
    for counts, lengths, w in ((p, None, None), (None, p, None), (None, None, nms.NmsCacheWeights(0x2000, 50, 0, 1, 1, 50, 0x1000))):  # kept_out is one of them
        assert L.nms_cache_evict_batched(p, p, counts, lengths, 50, 2, 3, w, 10, 0, 4, tensor, 1, None, None, p, p, 1 << 40, None) == bad
        assert L.nms_cache_keep_batched(p, p, counts, lengths, 50, 2, 3, w, 10, 0, 4, None, p, None, p, 1 << 40, None) == bad
    assert evict(positions=None) == bad                               # a window by places that nobody keeps
    for t in (nms.NmsCacheTensor(None, 16, 0, 0, 0), nms.NmsCacheTensor(0x1000, 0, 0, 0, 0), nms.NmsCacheTensor(0x1000, -5, 0, 0, 0),
              nms.NmsCacheTensor(0x1000, (1 << 20) + 1, 0, 0, 0)):
        assert evict(t=t) == bad and move(t=t) == bad
    assert evict(many=-1) == bad and move(many=-1) == bad and evict(t=None) == bad and evict(many=9) == large and move(many=9) == large
    for pg in (nms.NmsCachePages(None, 4, 16, 9, 0), nms.NmsCachePages(0x1000, 3, 16, 9, 0), nms.NmsCachePages(0x1000, 4, 0, 9, 0),
               nms.NmsCachePages(0x1000, 4, 16, -1, 0), nms.NmsCachePages(0x1000, 4, 16, 9, 1), nms.NmsCachePages(0x1000, -4, -16, 9, 0)):
        assert evict(pg=pg) == bad and move(pg=pg) == bad
    assert move(moves=None) == bad
    assert evict(w=weights(group=1025, tokens=1024)) == large and keep(w=weights(group=2147483647, tokens=2147483647)) == large
    need = nms.nms_cache_workspace_bytes(50, 2, 3, 10)
    for wrong in (dict(ws=None), dict(size=need - 1), dict(ws=ctypes.c_void_p(0x1010))):
        assert evict(**wrong) == nms.NMS_ERR_WORKSPACE and keep(**wrong) == nms.NMS_ERR_WORKSPACE, wrong
    for none in (dict(n=0), dict(h=0), dict(s=0)):
        assert evict(sums=None, ws=None, size=0, **none) == nms.NMS_OK and keep(sums=None, ws=None, size=0, **none) == nms.NMS_OK
        assert move(moves=None, **none) == nms.NMS_OK
    assert move(moves=None, many=0, t=None) == nms.NMS_OK


class OnGpu(torch.Tensor):
    """A CPU tensor that says it lies on the current GPU: the binding's checks of shapes and strides without one."""
    is_cuda = True

    @property
    def device(self):
        return torch.device("cuda", 0)

    def get_device(self):
        return 0


def gpu(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture
def recorded(nms, monkeypatch):
    """The library replaced by one that writes the calls down."""
    calls = []

    class Library:
        def __getattr__(self, name):
            real = getattr(nms_lib, name)
            if name in ("nms_verify_batched", "nms_cache_keep_batched", "nms_cache_move_batched", "nms_cache_evict_batched"):
                return lambda *a: calls.append((name, a)) or 0
            return real
    nms_lib = nms.lib
    monkeypatch.setattr(nms, "lib", Library())
    monkeypatch.setattr(nms, "_stream", lambda s: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return calls


def test_binding_of_verification(nms, recorded):
    k, v, s = 2, 50, 3
    i32 = torch.int32

    def good():
        return dict(target=gpu(s, k + 1, v), draft=gpu(s, k, v), drafts=gpu(s, k, dtype=i32), counts=None, drafts_max=k, vocabulary=v, sequences=s,
                    uniforms=gpu(s, k + 1), tokens_out=gpu(s, k + 1, dtype=i32), accepted_out=gpu(s, dtype=i32), workspace=gpu(4096, dtype=torch.uint8))
    nms.nms_verify_batched(**good())
    nms.nms_verify_batched(**{**good(), "target": gpu(s, k + 1, v + 6)[..., 3:], "draft": None})
    plan = nms.VerifyPlan(**good())
    plan()
    (_, a), (_, b), (_, c) = recorded
    assert a[1] == 50 and a[3] == 50 and a[4] == 0 and a[7:10] == (2, 50, 3) and b[1] == 56 and b[2] is None and c[7:10] == (2, 50, 3)
    wrong = dict(target=[gpu(s, k, v), gpu(s, k + 1, v - 1), gpu(s, k + 1, v, 1), gpu(s, k + 1, 2 * v)[..., ::2], gpu(s + 1, k + 1, v),
                         gpu(1, 1, v).expand(s, k + 1, v), gpu(2 * s, k + 1, v)[::2], gpu(s, v, k + 1).transpose(1, 2), torch.zeros(s, k + 1, v)],
                 draft=[gpu(s, k + 1, v), gpu(s, k, v - 1), torch.zeros(s, k, v)],
                 drafts=[gpu(s, k - 1, dtype=i32), torch.zeros(s, k, dtype=i32)], counts=[gpu(s - 1, dtype=i32)],
                 uniforms=[gpu(s, k)], tokens_out=[gpu(s, k, dtype=i32)], accepted_out=[gpu(s - 1, dtype=i32)])
    for name, values in wrong.items():
        for value in values:
            with pytest.raises(ValueError, match=name):
                nms.nms_verify_batched(**{**good(), name: value})
    for name, value in (("target", gpu(s, k + 1, v, dtype=torch.float64)), ("target", gpu(s, k + 1, v, dtype=torch.int32)), ("target", None),
                        ("draft", gpu(s, k, v, dtype=torch.float16)), ("drafts", gpu(s, k, dtype=torch.int64)), ("uniforms", gpu(s, k + 1, dtype=torch.float64))):
        with pytest.raises(TypeError):
            nms.nms_verify_batched(**{**good(), name: value})
    assert len(recorded) == 3


def test_binding_of_eviction(nms, recorded):
    n, h, s, budget = 40, 2, 3, 16
    i32 = torch.int32

    def good():
        return dict(sums=gpu(s, h, n), positions=gpu(s, h, n, dtype=i32), counts=gpu(s, dtype=i32), lengths=None, n_max=n, heads=h, sequences=s,
                    budget=budget, first=1, recent=4, tensors=[gpu(s, h, n, 8), gpu(s, n, h, 4).transpose(1, 2)], keep_out=None, kept_out=None,
                    workspace=gpu(1 << 16, dtype=torch.uint8))
    nms.nms_cache_evict_batched(**good())
    nms.nms_cache_evict_batched(**good(), weights=gpu(s, h, 2, 3, 44, dtype=torch.float16)[..., 2:42], valid_tokens=gpu(s, dtype=i32))
    table = gpu(s, 3, dtype=i32)
    paged = {**good(), "tensors": [gpu(9, h, 16, 8), gpu(9, h, 16, 2, 3)], "page_table": table}
    nms.CachePlan(**paged)()
    (_, a), (_, b), (_, c) = recorded
    assert (a[11][0].row_bytes, a[11][0].sequence_stride, a[11][0].head_stride, a[11][0].slot_stride) == (32, h * n * 32, n * 32, 32)
    assert (a[11][1].row_bytes, a[11][1].sequence_stride, a[11][1].head_stride, a[11][1].slot_stride) == (16, h * n * 16, 16, h * 16)
    w = b[7]
    assert a[7] is None and (w.row_stride, w.type, w.group, w.tokens, w.columns) == (44, 1, 2, 3, 40) and w.valid_tokens
    assert (c[13].table_stride, c[13].page_slots, c[13].pages) == (3, 16, 9) and c[11][1].row_bytes == 24
    cpu = torch.zeros(s, h, n)
    wrong = dict(sums=[gpu(s, h, n - 1), cpu], positions=[gpu(s, h, n - 1, dtype=i32)], counts=[gpu(s - 1, dtype=i32)], lengths=[gpu(s - 1, dtype=i32)],
                 keep_out=[gpu(s, h, n - 1, dtype=torch.uint8)], kept_out=[gpu(s - 1, dtype=i32)],
                 weights=[gpu(s, h, 2, 3), gpu(s, h + 1, 2, 3, n), gpu(s - 1, h, 2, 3, n), gpu(s, h, 2, 3, 2 * n)[..., ::2], gpu(s, h, 1, 1, n).expand(s, h, 2, 3, n),
                          torch.zeros(s, h, 2, 3, n)],
                 tensors=[[gpu(s, h, n - 1, 8)], [gpu(s, h - 1, n, 8)], [gpu(s - 1, h, n, 8)], [gpu(s, h)], [gpu(s, h, n, 16)[..., ::2]],
                          [gpu(s, h, 1, 8).expand(s, h, n, 8)], [gpu(1, h, n, 8).expand(s, h, n, 8)], [gpu(s, h, n + 7).as_strided((s, h, n, 8), (h * n, n, 1, 1))],
                          [torch.zeros(s, h, n, 8)]])
    for name, values in wrong.items():
        for value in values:
            with pytest.raises(ValueError, match=name):
                nms.nms_cache_evict_batched(**{**good(), name: value})
    with pytest.raises(ValueError, match="valid_tokens"):
        nms.nms_cache_evict_batched(**good(), weights=gpu(s, h, 1, 1, n), valid_tokens=gpu(s - 1, dtype=i32))
    for name, value, match in (("page_table", gpu(s, 2, dtype=i32), "page_table"), ("page_table", gpu(s - 1, 3, dtype=i32), "page_table"),
                               ("page_table", gpu(s * 3, dtype=i32), "page_table"), ("page_table", torch.zeros(s, 3, dtype=i32), "page_table"),
                               ("tensors", [gpu(9, h, 16, 8), gpu(9, h, 8, 8)], "tensors"), ("tensors", [gpu(9, h, 16, 8), gpu(8, h, 16, 8)], "tensors")):
        with pytest.raises(ValueError, match=match):
            nms.nms_cache_evict_batched(**{**paged, name: value})
    with pytest.raises(TypeError):
        nms.nms_cache_evict_batched(**{**good(), "weights": gpu(s, h, 1, 1, n, dtype=torch.float64)})
    with pytest.raises(TypeError):
        nms.nms_cache_evict_batched(**{**good(), "tensors": ["keys"]})
    m = nms.nms_cache_moves_max(n, budget)
    step = dict(sums=gpu(s, h, n), positions=None, counts=None, lengths=None, n_max=n, heads=h, sequences=s, budget=budget, first=0, recent=0,
                keep_out=None, kept_out=None, moves_out=gpu(s * h * (m + 1) * 2, dtype=i32), workspace=gpu(1 << 16, dtype=torch.uint8))
    nms.nms_cache_keep_batched(**step)
    with pytest.raises(ValueError, match="moves_out"):
        nms.nms_cache_keep_batched(**{**step, "moves_out": gpu(s * h * (m + 1) * 2 - 1, dtype=i32)})
    with pytest.raises(ValueError, match="moves"):
        nms.nms_cache_move_batched(gpu(s * h * (m + 1) * 2 - 1, dtype=i32), n, h, s, budget, [gpu(s, h, n, 8)])
    assert len(recorded) == 4


def test_tensors_may_come_from_an_iterator(nms, recorded, monkeypatch):
    n, h, s, budget = 40, 2, 3, 16
    rows = [gpu(s, h, n, 8), gpu(s, h, n, 4)]
    moves = gpu(s * h * (nms.nms_cache_moves_max(n, budget) + 1) * 2, dtype=torch.int32)
    rest = (gpu(s, h, n), None, None, None, n, h, s, budget, 0, 0)
    after = (None, None, gpu(1 << 16, dtype=torch.uint8))
    nms.nms_cache_evict_batched(*rest, iter(rows), *after)
    nms.nms_cache_move_batched(moves, n, h, s, budget, (t for t in rows))
    nms.CachePlan(*rest, iter(rows), *after)()
    nms.nms_cache_evict_batched(*rest, None, *after)
    evict, move, plan, none = (a for _, a in recorded)
    assert evict[12] == move[6] == plan[12] == 2 and none[12] == 0
    assert [t.row_bytes for t in evict[11]] == [t.row_bytes for t in move[5]] == [t.row_bytes for t in plan[11]] == [32, 16]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="tensors.*current device"):
        nms.nms_cache_move_batched(None, n, h, s, budget, iter(rows))


def test_binding_refuses_tensors_of_another_device(nms, recorded, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        nms.nms_verify_batched(gpu(1, 1, 9), None, None, None, 0, 9, 1, gpu(1, 1), gpu(1, 1, dtype=torch.int32), gpu(1, dtype=torch.int32), None)
    with pytest.raises(ValueError, match="current device"):
        nms.nms_cache_evict_batched(gpu(1, 1, 9), None, None, None, 9, 1, 1, 4, 0, 0, [], None, None, gpu(4096, dtype=torch.uint8))
    with pytest.raises(ValueError, match="current device"):
        nms.nms_cache_move_batched(gpu(64, dtype=torch.int32), 9, 1, 1, 4, [gpu(1, 1, 9, 4)])


def test_the_oracle_of_verification_by_hand():
    import decoding_oracle

    target, draft = np.zeros((1, 3, 4)), np.zeros((1, 2, 4))
    target[0] = [[0.1, 0.2, 0.3, 0.4], [0.25, 0.25, 0.5, 0.0], [0.0, 0.0, 0.0, 1.0]]
    draft[0] = [[0.4, 0.2, 0.2, 0.2], [0.0, 0.0, 0.0, 1.0]]
    # 3: 0.9 * 0.2 < 0.4 stands; 3: 0.0 * 1.0 < 0.0 does not; what is left of row 1 is (0.25, 0.25, 0.5, 0)
    for u, token in ((0.0, 0), (0.2, 0), (0.25, 1), (0.5, 2), (0.99, 2)):
        tokens, accepted = decoding_oracle.verify(target, draft, np.array([[3, 3]]), None, np.array([[0.9, 0.0, u]], np.float32))
        assert accepted[0] == 1 and tokens[0].tolist() == [3, token, -1]
    tokens, accepted = decoding_oracle.verify(target, draft, np.array([[0, 3]]), None, np.array([[0.25, 0.0, 0.6]], np.float32))
    # 0: 0.25 * 0.4 < 0.1 does not hold (0.1 in 64 bits); left: (0, 0, 0.1, 0.2)
    assert accepted[0] == 0 and tokens[0].tolist() == [3, -1, -1]


def test_the_oracle_of_eviction_by_hand():
    import decoding_oracle

    sums = np.array([[[5, 1, 4, 1, 3, 2, 9, 7]]], np.float32)
    keep, kept, moves = decoding_oracle.keep(sums, None, [7], None, 4, 1, 1)    # slots 0 (first) and 6 (newest), then 2 and 4
    assert keep[0, 0].tolist() == [1, 0, 1, 0, 1, 0, 1, 0] and kept[0] == 4 and moves[0][0] == [(1, 4), (3, 6)]
    keep, kept, moves = decoding_oracle.keep(np.zeros((1, 1, 5), np.float32), None, None, None, 2, 0, 1)
    assert keep[0, 0].tolist() == [1, 0, 0, 0, 1] and moves[0][0] == [(1, 4)]
