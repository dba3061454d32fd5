"""Arguments of the decoding step's calls that a caller can get wrong, without a GPU: each is refused before anything is launched, or does no harm."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000          # an address that nothing looks at


@pytest.fixture(scope="module")
def nms():
    from paper_2502_00535_amd import build as nms_build

    if nms_build.is_stale():
        nms_build.build_library()
    import paper_2502_00535_amd.binding as binding

    return binding


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
