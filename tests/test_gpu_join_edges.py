"""Joins and dropout at the edges of what their definitions allow, against the definitions in 64 bits or against an equal call whose
result other tests have checked."""
import numpy as np
import pytest

from tests.test_gpu_resnorm import EPS, check, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_1805_11046_b200.binding as binding
    return binding


def both_passes(B, i, **kw):
    d = B.resnorm_desc(i["x"], i["b"], eps=EPS, **kw)
    r, h, q1, q2 = B.qbp_resnorm_fwd(d, i["x"], i["b"], i["w1"], i["gate"], i["w2"])
    return (r, h, q1, q2) + B.qbp_resnorm_bwd(d, i["dr"], i["dh"], i["b"], r, q1, q2, i["w1"], i["gate"], i["w2"])


@pytest.mark.parametrize("rows,cols", [(100, 4096), (700, 1000), (333, 64), (5, 9000)])
def test_a_group_of_more_rows_than_there_are(B, rows, cols):
    """A sequence shorter than the rows its gate is for: the bits of a group of just its rows."""
    import torch
    check(B, rows, cols, "float32", "bfloat16", gate_rows=rows + 7, p=0.1, alpha=0.5)
    i = {k: v[0] for k, v in inputs(rows, cols, "float32", "bfloat16", 1, 5).items()}
    want = both_passes(B, i, gate_rows=rows)
    for gate_rows in (rows + 1, 8192, 1 << 40, (1 << 63) - 1):
        assert all(torch.equal(a, b) for a, b in zip(both_passes(B, i, gate_rows=gate_rows), want)), gate_rows
