"""How a join's rows are cut into items for the blocks of a grid: every row once, no block with much more than its share (the host's rule,
compiled by itself; runs without a GPU)."""
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_1805_11046_b200" / "csrc"
PROGRAM = r"""
#include "qbp_resnorm.cuh"
#include <cstdio>
#include <vector>
namespace qbp { int fail(int status, const char *, ...) { return status; } int sm_count() { return 148; } }
int main()
{
    long long rows, cols, gate_rows, most, few;
    int warp, sums;
    while (scanf("%lld %lld %lld %d %lld %lld %d", &rows, &cols, &gate_rows, &warp, &most, &few, &sums) == 7) {
        qbp_resnorm_desc d{};
        d.rows = rows; d.cols = cols; d.gate_rows = gate_rows;
        const qbp::JoinShape s{1, 256, warp != 0, true};
        const qbp::JoinCut c = qbp::join_cut(&d, s, true, most, few, sums != 0);
        std::vector<long long> load(c.blocks, 0);
        long long next = 0;
        const long long share = gate_rows ? std::min(gate_rows, rows) : rows;
        for (long long item = 0; item < c.it.gates * c.it.splits; ++item) {
            const long long gate = item / c.it.splits, first = gate * c.it.gate_rows + item % c.it.splits * c.it.split_rows;
            const long long end = std::min({first + c.it.split_rows, (gate + 1) * c.it.gate_rows, (long long)rows});
            if (first < end) {
                if (first != next || first / share != (end - 1) / share) return 1;      // every row once, in order, an item of one gate
                next = end;
                load[item % c.blocks] += end - first;
            }
        }
        if (next != rows || c.blocks > most || c.blocks < 1) return 2;
        printf("%lld %lld\n", *std::max_element(load.begin(), load.end()), (long long)c.blocks);
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    at = tmp_path_factory.mktemp("cut")
    (at / "cut.cu").write_text(PROGRAM)
    subprocess.run(["/usr/local/cuda/bin/nvcc", "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-I", str(CSRC), str(at / "cut.cu"), "-o", str(at / "cut")], check=True)

    def ask(cases):
        text = "\n".join(" ".join(str(int(v)) for v in c) for c in cases)
        got = subprocess.run([str(at / "cut")], input=text, capture_output=True, text=True)
        assert got.returncode == 0, got
        return [tuple(int(v) for v in line.split()) for line in got.stdout.splitlines()]
    return ask


@pytest.mark.parametrize("most", [148, 296, 592])
def test_no_block_has_much_more_than_its_share(cut, most):
    """16384 rows in 1 to 2048 gates, whole and ragged: the busiest block has at most a quarter more than an even share (and a few rows, as
    another item would cost), but where gates stay whole because there are at least a third as many as blocks and cutting them costs more."""
    rows = 16384
    cases = [(rows, 4096, -(-rows // gates), 0, most, few, sums) for gates in (1, 2, 3, 6, 8, 12, 16, 24, 32, 50, 64, 100, 128, 140, 148, 200, 296, 300, 512, 1000, 2048) for few, sums in ((1, 0), (4, 1))]
    for case, (busiest, blocks) in zip(cases, cut(cases)):
        gate_rows, few, sums = case[2], case[5], case[6]
        gates = -(-rows // gate_rows)
        even = max(rows / most, min(gate_rows, few))              # (no items of fewer rows than `few`)
        whole = 3 * gates >= most and (sums or gates > 3 * most)
        assert busiest <= 1.25 * even + 2 * few + 1 or whole and busiest <= -(-gates // most) * gate_rows, (case, busiest, even)


def test_one_gate_is_cut_evenly(cut):
    cases = [(rows, 1000, 0, warp, most, few, sums) for rows in (1, 7, 148, 149, 1998, 30000, 123457) for warp in (0, 1) for most in (148, 296) for few in (1, 2, 4) for sums in (0, 1)]
    for (rows, _, _, warp, most, few, _), (busiest, blocks) in zip(cases, cut(cases)):
        at_least = few * (8 if warp else 1)
        assert busiest <= max(-(-rows // most), min(rows, at_least)), (rows, warp, most, few, busiest)


def test_every_row_once_whatever_the_groups(cut):
    cases = [(rows, 64, g, warp, most, few, sums) for rows in (1, 2, 9, 100, 777, 4097) for g in (1, 2, 3, 7, 8, 64, 99, 100, 101, 5000, 1 << 40, (1 << 63) - 1)
             for warp in (0, 1) for most in (1, 5, 148) for few in (1, 4) for sums in (0, 1)]
    assert len(cut(cases)) == len(cases)
