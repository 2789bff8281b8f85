"""Which of a join's kernels a width runs on, and the shared memory that its ring is given: that of the layout the kernel uses, rows on
16-byte boundaries without the padding of others (the host's rules, compiled by themselves; runs without a GPU)."""
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_1805_11046_b200" / "csrc"
PROGRAM = r"""
#include "qbp_resnorm.cuh"
#include <cstdio>
namespace qbp { int fail(int status, const char *, ...) { return status; } int sm_count() { return 148; } }
int main()
{
    qbp_resnorm_desc d{};
    long long cols;
    int x, b, tensors, vec;
    while (scanf("%lld %d %d %d %d", &cols, &x, &b, &tensors, &vec) == 5) {
        d.rows = 1000; d.cols = cols; d.x_dtype = x; d.b_dtype = b;
        const qbp::JoinShape s = qbp::join_shape(&d, tensors, vec != 0);
        printf("%d %d %d %lld %d %lld\n", s.ch, s.threads, s.warp ? 8 : 1, (long long)qbp::join_ring(&d, s, tensors), qbp::join_slots(&d, s, tensors), (long long)qbp::join_blocks(&d, s, tensors));
    }
    return 0;
}
"""
SIZE = {0: 4, 1: 2, 2: 2}


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    at = tmp_path_factory.mktemp("ring")
    (at / "ring.cu").write_text(PROGRAM)
    subprocess.run(["/usr/local/cuda/bin/nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", str(CSRC), str(at / "ring.cu"), "-o", str(at / "ring")], check=True)

    def ask(cases):
        got = subprocess.run([str(at / "ring")], input="\n".join(" ".join(str(v) for v in c) for c in cases), capture_output=True, text=True)
        assert got.returncode == 0, got
        return [tuple(int(v) for v in line.split()) for line in got.stdout.splitlines()]
    return ask


def test_rings_are_as_large_as_the_kernels_lay_them_out(shape):
    cases = [(cols, x, b, tensors, vec) for cols in [*range(8, 16385, 88), 512, 520, 4096, 4104, 6392, 6400, 6408, 8192, 8200, 16384] for x, b in ((0, 0), (0, 1), (1, 1), (1, 0), (2, 2))
             for tensors in (1, 2) for vec in (0, 1)]
    cases += [(cols, x, b, tensors, 0) for cols in range(1, 16385, 91) for x, b in ((0, 0), (0, 1), (2, 2)) for tensors in (1, 2)]
    for (cols, x, b, tensors, vec), (ch, threads, rows, ring, slots, blocks) in zip(cases, shape(cases)):
        section = lambda size: cols * size if vec else (cols * size + 15) // 16 * 16 + 16
        slot = tensors * (section(SIZE[x]) + section(SIZE[b]))
        if ch <= 2:
            assert ring == slots * rows * slot <= 200 * 1024, (cols, x, b, tensors, vec)
            assert threads * 8 * ch >= cols * rows and threads <= 512 and slots in (2, 3)
        else:
            assert 32 * threads >= cols and threads <= 512
        assert blocks % 148 == 0 and blocks >= 148


def test_the_widest_rows_with_a_ring(shape):
    """Every width up to 8192 columns, but backwards in fp32 alone as far as two slots of four rows have room."""
    ring = lambda *c: shape([c])[0][0] <= 2
    for x, b in ((0, 1), (1, 0), (1, 1), (2, 2), (0, 2)):
        for vec in (0, 1):
            assert all(ring(8192, x, b, tensors, vec) and not ring(8200, x, b, tensors, vec) for tensors in (1, 2))
    assert ring(8192, 0, 0, 1, 0) and ring(8192, 0, 0, 1, 1)
    assert ring(6400, 0, 0, 2, 1) and not ring(6408, 0, 0, 2, 1)
    assert ring(6396, 0, 0, 2, 0) and not ring(6397, 0, 0, 2, 0)


WORKSPACES = r"""
#include "qbp_resnorm.cuh"
#include <cstdio>
namespace qbp { int fail(int status, const char *, ...) { return status; } int sm_count() { return 148; } }
int main()
{
    qbp_resnorm_desc d{};
    long long rows, cols, gate_rows;
    int x, b;
    while (scanf("%lld %lld %lld %d %d", &rows, &cols, &gate_rows, &x, &b) == 5) {
        d.rows = rows; d.cols = cols; d.gate_rows = gate_rows; d.x_dtype = x; d.b_dtype = b;
        size_t most = 0;
        for (bool vec : {false, true})
            for (bool per_gate : {false, true}) {
                const qbp::JoinShape s = qbp::join_shape(&d, 2, vec);
                const qbp::JoinCut c = qbp::join_cut(&d, s, per_gate, qbp::join_blocks(&d, s, 2), s.warp ? 2 : 4, true);
                const size_t row = (size_t)d.cols * 4, blocks = (size_t)c.blocks * row, parts = c.it.splits > 1 ? (size_t)(c.it.gates * c.it.splits) * row : 0;
                most = std::max(most, 2 * ((blocks + 255) / 256 * 256) + (parts + 255) / 256 * 256);
            }
        printf("%zu\n", 256 + most);
    }
    return 0;
}
"""


def test_a_backward_pass_asks_for_the_workspace_of_every_way_it_may_be_cut(tmp_path):
    """With and without a gate, on the 16-byte boundaries and off them: the call does not know which when it is asked for the size."""
    import ctypes as C
    import random

    from paper_1805_11046_b200 import binding as B
    (tmp_path / "ws.cu").write_text(WORKSPACES)
    subprocess.run(["/usr/local/cuda/bin/nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", str(CSRC), str(tmp_path / "ws.cu"), "-o", str(tmp_path / "ws")], check=True)
    r = random.Random(3)
    cases = [(r.randint(1, 40000), r.choice([r.randint(1, 16384), 8 * r.randint(1, 2048), 8 * r.randint(800, 801)]), r.choice([0, 1, 7, 100, 5000, r.randint(1, 40000), 1 << 50]),
              r.randint(0, 2), r.randint(0, 2)) for _ in range(4000)]
    got = subprocess.run([str(tmp_path / "ws")], input="\n".join(" ".join(str(v) for v in c) for c in cases), capture_output=True, text=True)
    assert got.returncode == 0, got
    for (rows, cols, gate_rows, x, b), need in zip(cases, got.stdout.split()):
        d = B.ResnormDesc(rows, cols, x, b, 1, 1, 1e-6, 1.0, gate_rows, 0.0, 0, 0, 0)
        assert B.lib.qbp_resnorm_bwd_workspace_bytes(C.addressof(d)) == int(need), (rows, cols, gate_rows, x, b)
