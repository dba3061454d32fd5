"""Arguments of the decoding step's calls that a caller can get wrong, without a GPU: each is refused before anything is launched, or does no harm."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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
