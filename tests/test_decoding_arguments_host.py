"""Arguments of the decoding step's calls that a caller can get wrong, without a GPU: each is refused before anything is launched, or does no harm."""
import ctypes
import os
import subprocess

import pytest
import torch

from test_decoding_host import gpu, nms, recorded  # noqa: F401  (fixtures, and CPU tensors that say they lie on the GPU)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000          # an address that nothing looks at


def test_a_list_may_say_any_number_of_moves(tmp_path):
    """A workgroup takes 32 moves of a list that has room for moves_max: whatever the list says, it reads none behind them."""
    exe = tmp_path / "moves_driver"
    subprocess.run(["g++", "-std=c++17", "-O2", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "host", "moves_driver.cpp"), "-o", str(exe)], check=True)
    counts = (-2147483648, -2147483647, -33, -1, 0, 1, 31, 32, 33, 64, 99, 100, 101, 2147483647)
    cases = [(count, moves_max, begin) for moves_max in (1, 32, 100, 524288) for count in counts for begin in range(0, min(moves_max, 200), 32)]
    proc = subprocess.run([str(exe)], input="\n".join(f"{c} {m} {b} 32" for c, m, b in cases), capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr[-2000:]
    got = [int(x) for x in proc.stdout.split()]
    assert got == [len(range(b, min(max(c, 0), m, b + 32))) for c, m, b in cases]


def test_strides_below_0_are_refused(nms):
    """An offset below 0 would be taken for a page that is none of the pool's, and the row left where it is without an error."""
    p, pages = ctypes.c_void_p(P), nms.NmsCachePages(P, 4, 16, 9, 0)
    for strides in ((-4096, 1024, 16), (4096, -1024, 16), (4096, 1024, -16), (-(1 << 62), 0, 0)):
        bad = nms.NmsCacheTensor(P, 16, *strides)
        both = (nms.NmsCacheTensor * 2)(nms.NmsCacheTensor(P, 16, 4096, 1024, 16), bad)
        for pg in (None, pages):
            for tensors, many in ((bad, 1), (both, 2)):
                assert nms.lib.nms_cache_evict_batched(p, p, None, None, 50, 2, 3, None, 10, 0, 4, tensors, many, pg, None, None, None, 0,
                                                       None) == nms.NMS_ERR_INVALID_ARG, strides
                assert nms.lib.nms_cache_move_batched(p, 0, 2, 3, 10, tensors, many, pg, None) == nms.NMS_ERR_INVALID_ARG, strides


def test_outputs_of_verification_overlap_nothing(nms):
    """A workgroup writes its sequence's outputs while others still read their inputs.  (The workspace is too small in these calls, and that is looked at
    after the buffers.)"""
    k, v, s = 3, 50000, 6
    assert nms.nms_verify_workspace_bytes(v, s) > 0
    places = dict(drafts=0x10000, counts=0x20000, uniforms=0x30000, tokens=0x40000, accepted=0x50000)
    sizes = dict(drafts=4 * s * k, counts=4 * s, uniforms=4 * s * (k + 1), tokens=4 * s * (k + 1), accepted=4 * s)

    def call(**at):
        a = {name: ctypes.c_void_p(place) for name, place in {**places, **at}.items()}
        return nms.lib.nms_verify_batched(P, v, None, v, 0, a["drafts"], a["counts"], k, v, s, a["uniforms"], a["tokens"], a["accepted"], None, 0, None)
    assert call() == call(counts=None) == nms.NMS_ERR_WORKSPACE
    for out in ("tokens", "accepted"):
        for other in places:
            if other == out:
                continue
            begin, end = places[other] - sizes[out], places[other] + sizes[other]
            for at in (begin + 4, places[other], end - 4):
                assert call(**{out: at}) == nms.NMS_ERR_INVALID_ARG, (out, other, at)
            for at in (begin, end):
                assert call(**{out: at}) == nms.NMS_ERR_WORKSPACE, (out, other, at)


def test_outputs_of_eviction_overlap_no_number_of_a_sequence(nms):
    """counts, lengths and valid_tokens are read by every head's workgroup, and some of them have written their outputs by then."""
    n, h, s, budget = 50, 2, 6, 10
    places = dict(sums=0x100000, positions=0x200000, keep=0x300000, kept=0x400000, moves=0x500000)
    sizes = dict(sums=4 * s * h * n, positions=4 * s * h * n, keep=s * h * n, kept=4 * s, moves=8 * s * h * (nms.nms_cache_moves_max(n, budget) + 1))

    def call(whole, counts=None, lengths=None, valid=None):
        w = nms.NmsCacheWeights(P, n, 0, 1, 1, n, valid)
        a = {name: ctypes.c_void_p(place) for name, place in places.items()}
        if whole:
            return nms.lib.nms_cache_evict_batched(a["sums"], a["positions"], counts, lengths, n, h, s, w, budget, 0, 4, None, 0, None, a["keep"],
                                                   a["kept"], None, 0, None)
        return nms.lib.nms_cache_keep_batched(a["sums"], a["positions"], counts, lengths, n, h, s, w, budget, 0, 4, a["keep"], a["kept"],
                                              a["moves"], None, 0, None)
    for whole in (True, False):
        assert call(whole) == nms.NMS_ERR_WORKSPACE
        for name in ("counts", "lengths", "valid"):
            for out in places:
                if out == ("moves" if whole else "positions"):   # the whole path has no list, the other call only reads positions
                    continue
                begin, end = places[out] - 4 * s, places[out] + sizes[out]
                for at in (begin + 4, places[out], end - 4):
                    assert call(whole, **{name: at}) == nms.NMS_ERR_INVALID_ARG, (name, out, at)
                for at in (begin, end):
                    assert call(whole, **{name: at}) == nms.NMS_ERR_WORKSPACE, (name, out, at)


BEYOND = (2 ** 32, -2 ** 32, 2 ** 31, -2 ** 31 - 2 ** 20, 2 ** 64)  # and stay beyond when a size is added


@pytest.mark.parametrize("beyond", BEYOND)
def test_numbers_beyond_32_bits_are_refused(nms, recorded, beyond):
    """Not taken by their low 32 bits: a budget of 2^32 + 16 is not 16, and 2^32 + 40 slots are not 40 of buffers that nobody has looked at."""
    n, h, s, budget = 40, 2, 3, 16
    i32 = torch.int32
    cache = dict(sums=gpu(s, h, n), positions=None, counts=None, lengths=None, n_max=n, heads=h, sequences=s, budget=budget, first=0, recent=0,
                 keep_out=None, kept_out=None, workspace=gpu(1 << 16, dtype=torch.uint8))
    move = dict(moves=gpu(s * h * (budget + 1) * 2, dtype=i32), n_max=n, heads=h, sequences=s, budget=budget, tensors=[gpu(s, h, n, 4)])
    verify = dict(target=gpu(s, 3, 50), draft=None, drafts=gpu(s, 2, dtype=i32), counts=None, drafts_max=2, vocabulary=50, sequences=s,
                  uniforms=gpu(s, 3), tokens_out=gpu(s, 3, dtype=i32), accepted_out=gpu(s, dtype=i32), workspace=gpu(4096, dtype=torch.uint8))
    calls = [(nms.nms_cache_evict_batched, {**cache, "tensors": []}, ("n_max", "heads", "sequences", "budget", "first", "recent")),
             (nms.CachePlan, {**cache, "tensors": []}, ("n_max", "heads", "sequences", "budget", "first", "recent")),
             (nms.nms_cache_keep_batched, {**cache, "moves_out": None}, ("n_max", "heads", "sequences", "budget", "first", "recent")),
             (nms.nms_cache_move_batched, move, ("n_max", "heads", "sequences", "budget")),
             (nms.nms_verify_batched, verify, ("drafts_max", "vocabulary", "sequences")), (nms.VerifyPlan, verify, ("drafts_max", "vocabulary", "sequences"))]
    for call, good, names in calls:
        call(**good)
        before = len(recorded)
        for name in names:
            with pytest.raises(ValueError, match=name):
                call(**{**good, name: beyond + good[name]})
        assert len(recorded) == before
    for size, good in ((nms.nms_cache_moves_max, (n, budget)), (nms.nms_cache_workspace_bytes, (n, h, s, budget)), (nms.nms_verify_workspace_bytes, (50, s))):
        for i in range(len(good)):
            with pytest.raises(ValueError):
                size(*good[:i], good[i] + beyond, *good[i + 1:])


def test_dimensions_beyond_32_bits_are_refused(nms, recorded):
    """Tensors of nothing can have any shape."""
    n, h, s = 40, 1, 1
    rest = (gpu(s, h, n), None, None, None, n, h, s, 16, 0, 0)
    after = (None, None, gpu(1 << 16, dtype=torch.uint8))
    for group, tokens, columns in ((2 ** 32 + 1, 1, 0), (1, 2 ** 32 + 1, 0), (1, 0, 2 ** 32 + n)):
        with pytest.raises(ValueError, match="weights"):
            nms.nms_cache_evict_batched(*rest, [], *after, weights=gpu(s, h, group, tokens, columns))
    with pytest.raises(ValueError, match="page_table|tensors"):
        nms.nms_cache_evict_batched(*rest, [gpu(2 ** 32 + 9, h, 16, 0)], *after, page_table=gpu(s, 3, dtype=torch.int32))
    assert not recorded


def test_a_plan_is_called_on_its_own_device(nms, recorded, monkeypatch):
    """Its kernels would run on the current device otherwise, with addresses of another one."""
    n, h, s, budget = 40, 2, 3, 16
    cache = nms.CachePlan(gpu(s, h, n), None, None, None, n, h, s, budget, 0, 0, [], None, None, gpu(1 << 16, dtype=torch.uint8))
    verify = nms.VerifyPlan(gpu(1, 1, 9), None, None, None, 0, 9, 1, gpu(1, 1), gpu(1, 1, dtype=torch.int32), gpu(1, dtype=torch.int32), None)
    cache(), verify()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for plan in (cache, verify):
        with pytest.raises(ValueError, match="cuda:0.*cuda:1"):
            plan()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    cache(), verify()
    assert len(recorded) == 4
