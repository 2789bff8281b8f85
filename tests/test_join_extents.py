"""Extents of a join beyond what its tensors have: groups of more rows than there are, counts near the ends of 64 bits (runs without a
GPU; in a process of its own, since a division by zero in the library would end the test run)."""
import subprocess
import sys
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def B():
    from paper_1805_11046_b200 import build
    build.build_library()
    from paper_1805_11046_b200 import binding
    return binding


def workspaces(*descs):
    """qbp_resnorm_bwd_workspace_bytes of (rows, cols, gate_rows) each, asked in another process."""
    code = ("from paper_1805_11046_b200 import binding as B\n"
            f"for rows, cols, gate_rows in {descs!r}:\n"
            "    print(B.qbp_resnorm_bwd_workspace_bytes(B.ResnormDesc(rows, cols, 0, 1, 1, 1, 1e-6, 1.0, gate_rows, 0.0, 0, 0, 0)))\n")
    got = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert got.returncode == 0, got
    return [int(line) for line in got.stdout.split()]


@pytest.mark.parametrize("rows,cols", [(4, 64), (1, 1), (1000, 4096), (4096, 520)])
def test_a_group_of_more_rows_than_there_are_is_all_of_them(B, rows, cols):
    want, *got = workspaces((rows, cols, rows), (rows, cols, rows + 1), (rows, cols, 1 << 20), (rows, cols, 1 << 40), (rows, cols, (1 << 63) - 1))
    assert want >= 256 and got == [want] * 4


def test_extents_that_no_tensor_has(B):
    """Refused, and a workspace is asked for that any program can have."""
    most = (1 << 63) - 1
    bad = [(4, 64, -1), (4, 64, -8), (4, 64, -most), (-1, 64, 0), (4, -8, 0), (most, 64, 0), (most, 64, 1), (most // 64, 64, 7), (1 << 60, 16, most), (4, most, 0)]
    assert workspaces(*bad) == [256] * len(bad)
    from tests.test_f8_refusals import bwd, desc, fwd
    for rows, cols, gate_rows in bad:
        d = desc(B, rows=rows, cols=cols, gate_rows=gate_rows)
        assert fwd(B, d) in (-1, -2) and bwd(B, d) in (-1, -2)
