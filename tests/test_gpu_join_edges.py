"""Joins and dropout at the edges of what their definitions allow, against the definitions in 64 bits or against an equal call whose
result other tests have checked."""
import numpy as np
import pytest

from oracle import f8_oracle as F
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


SHAPES = [(6, 64), (40, 512), (30, 520), (12, 4096), (7, 8192), (5, 9000), (41, 77), (30, 1001), (6, 4095), (5, 9001)]       # a row a warp's and a block's, on and off the 16-byte boundaries, wide


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("stream", ["float32", "bfloat16"])
def test_what_is_dropped_of_a_row_without_a_norm(B, rows, cols, stream):
    """A block output whose row has no finite norm (a NaN, an infinity, zeros without eps): n is not a number there, but d is zero where the
    draw drops it, and the stream goes on untouched.  Backwards: nothing of it reaches the gradients of these columns' parameters."""
    import torch
    i = {k: v[0] for k, v in inputs(rows, cols, stream, "float32", 1, 17).items()}
    i["b"][0] = torch.randn(cols, device="cuda")
    i["b"][1] = 0.0                                              # without eps: 0 / 0
    i["b"][2, cols // 2] = float("nan")
    i["b"][3, cols - 1] = float("inf")
    k = torch.from_numpy(F.keep((rows, cols), 0.5, 12, 3) != 0).cuda()
    d = B.resnorm_desc(i["x"], i["b"], eps=0.0, p=0.5, seed=12, tensor_id=3, pre=False)
    r, _, q1, _ = B.qbp_resnorm_fwd(d, i["x"], i["b"], i["w1"], i["gate"])
    assert torch.equal(r[~k], i["x"][~k])
    bad = torch.zeros_like(k)
    bad[1] = k[1]; bad[2] = k[2]; bad[3, -1] = k[3, -1]           # (finite / infinity is zero)
    assert torch.equal(torch.isfinite(r), ~bad)
    dx, db, dw1, dg, _ = B.qbp_resnorm_bwd(d, i["dr"], None, i["b"], r, q1, None, i["w1"], i["gate"])
    assert torch.equal(dx, i["dr"])
    good = [j for j in range(rows) if j not in (1, 2, 3)]
    assert bool(torch.isfinite(db[good]).all())
    for got in (dw1, dg[0]):
        assert torch.equal(torch.isfinite(got), ~bad.any(0))
    # columns of which the bad rows have nothing: the sums of a call in which these rows have no gradient and an ordinary output
    b2, dr2 = i["b"].clone(), i["dr"].clone()
    b2[1:4] = 1.0; dr2[1:4] = 0.0
    _, _, e1, eg, _ = B.qbp_resnorm_bwd(d, dr2, None, b2, r, q1.clone().index_fill_(0, torch.tensor([1, 2, 3], device="cuda"), 1.0), None, i["w1"], i["gate"])
    gone = ~k[1:4].any(0)
    assert torch.equal(dw1[gone], e1[gone]) and torch.equal(dg[0][gone], eg[0][gone])


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("types", [("float32", "float32"), ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_gradient_that_is_not_finite(B, rows, cols, types, bad):
    """One element of dr: its own dx, its row's db and its column's dgate and dw_post, none of these but dx where the element was dropped."""
    import torch
    i = {k: v[0] for k, v in inputs(rows, cols, *types, 1, 23).items()}
    k = F.keep((rows, cols), 0.5, 12, 3) != 0
    kw = dict(p=0.5, seed=12, tensor_id=3)
    want = both_passes(B, i, **kw)
    at = {on: next((a, c) for a in range(rows - 1, -1, -1) for c in range(cols - 1, -1, -1) if k[a, c] == on) for on in (True, False)}
    for on, (a, c) in at.items():
        dr = i["dr"].clone()
        dr[a, c] = bad
        got = both_passes(B, {**i, "dr": dr}, **kw)
        spoilt = [torch.zeros_like(t, dtype=torch.bool) for t in want]
        spoilt[4][a, c] = True                                   # dx
        if on:
            spoilt[5][a] = True                                  # db
            spoilt[6][c] = True; spoilt[7][0, c] = True          # dw_post, dgate
        for n, (g, w, s) in enumerate(zip(got, want, spoilt)):
            assert torch.equal(~torch.isfinite(g), s), (n, on)
            assert torch.equal(g[~s], w[~s]), (n, on)
