"""Joins and dropout at the edges of what their definitions allow, against the definitions in 64 bits or against an equal call whose
result other tests have checked."""
import numpy as np
import pytest

from oracle import f8_oracle as F
from tests.test_gpu_resnorm import EPS, U, check, close, host, inputs

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


@pytest.mark.parametrize("rows,cols", SHAPES)
def test_a_block_output_or_gradient_of_h_that_is_not_finite(B, rows, cols):
    """An infinity in dh or a NaN in b: the rows that hold them and, of the parameters' gradients, every column that such a row enters; no other row."""
    import torch
    i = {k: v[0] for k, v in inputs(rows, cols, "float32", "bfloat16", 1, 29).items()}
    want = both_passes(B, i)
    dh, b = i["dh"].clone(), i["b"].clone()
    dh[3, 2] = float("inf"); b[4, cols - 1] = float("nan")
    r, h, q1, q2, dx, db, dw1, dg, dw2 = both_passes(B, {**i, "dh": dh, "b": b})
    rest = [j for j in range(rows) if j not in (3, 4)]
    for got, w in zip((r, h, q1, q2, dx, db), want):
        assert torch.equal(got[rest], w[rest])
    assert torch.equal(r[3], want[0][3]) and not torch.isfinite(r[4]).any() and not torch.isfinite(h[4]).any()
    assert not torch.isfinite(dx[3:5]).any() and not torch.isfinite(db[3:5]).any()
    assert not torch.isfinite(dw1).any() and not torch.isfinite(dg).any() and not torch.isfinite(dw2).any()      # (row 4's norms are of no number)


# ------------------------------------------------------------------------ whole 16-byte pieces from another boundary
@pytest.mark.parametrize("rows,cols", [(21, 512), (40, 1000), (14, 4096), (9, 8192), (5, 16384)])
@pytest.mark.parametrize("off", ["x", "b", "w1", "w2", "gate", "dr", "dh"])
def test_a_tensor_off_the_16_byte_boundary_against_the_definition(B, rows, cols, off, monkeypatch):
    """One input an element behind a boundary: every output within the bounds of an aligned call."""
    import torch
    import tests.test_gpu_resnorm as R

    def moved(*args):
        i = inputs(*args)
        t, v = i[off]
        return {**i, off: (torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape).copy_(t), v)}

    monkeypatch.setattr(R, "inputs", moved)
    check(B, rows, cols, "float32", "bfloat16", gate_rows=0, p=0.3, alpha=0.5)


@pytest.mark.parametrize("cols", [512, 4096, 16384])
def test_outputs_off_the_16_byte_boundary(B, cols):
    """Any one of them: the bits of the call with an input there."""
    import torch
    i = {k: v[0] for k, v in inputs(19, cols, "float32", "bfloat16", 1, 31).items()}
    off = lambda t: torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape)
    d = B.resnorm_desc(i["x"], i["b"], p=0.3, seed=4)
    params = i["w1"], i["gate"], i["w2"]
    want = B.qbp_resnorm_fwd(d, off(i["x"]).copy_(i["x"]), i["b"], *params)
    for kw in (dict(r=off(i["x"])), dict(h=off(i["b"]))):
        assert all(torch.equal(a, c) for a, c in zip(B.qbp_resnorm_fwd(d, i["x"], i["b"], *params, **kw), want))
    r, _, q1, q2 = want
    grads = B.qbp_resnorm_bwd(d, off(i["dr"]).copy_(i["dr"]), i["dh"], i["b"], r, q1, q2, *params)
    for kw in (dict(dx=off(i["x"])), dict(db=off(i["b"]))):
        assert all(torch.equal(a, c) for a, c in zip(B.qbp_resnorm_bwd(d, i["dr"], i["dh"], i["b"], r, q1, q2, *params, **kw), grads))


# ------------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype,n", [("float32", 10_000_003), ("bfloat16", 20_000_003), ("float16", 20_000_005)])
@pytest.mark.parametrize("off", [0, 16, 0.5])
def test_long_dropout_is_that_of_its_pieces(B, dtype, n, off):
    """More elements than the device's threads take one block of eight each of: every element is that of a call on a short piece; from a 32-byte
    boundary, from a 16-byte one (off: bytes; 0.5: one element) and from neither, with a ragged end."""
    import torch
    t = getattr(torch, dtype)
    first = int(off / t.itemsize) if off > 1 else int(off > 0)
    x = torch.randn(n + 16, device="cuda", generator=torch.Generator("cuda").manual_seed(n)).to(t)[first:first + n]
    assert x.data_ptr() % 32 == int(off if off != 0.5 else t.itemsize)
    y = torch.empty(n + 16, dtype=t, device="cuda")[first:first + n]
    base = (1 << 33) + 40
    B.qbp_dropout(x, 0.3, 99, tensor_id=2, index_base=base, y=y)
    step = 1 << 20
    for at in range(0, n, step):
        assert torch.equal(y[at:at + step], B.qbp_dropout(x[at:at + step], 0.3, 99, tensor_id=2, index_base=base + at)), at
    for at in (0, n // 2 // 8 * 8, n - n % 8 - 4096):
        piece = slice(at, min(at + 5000, n))
        k = F.keep((piece.stop - at,), 0.3, 99, 2, base + at)
        close(y[piece], host(x[piece]) * k, 2 * U * np.abs(host(x[piece]) * k), dtype)


@pytest.mark.parametrize("cols", [6392, 6396, 6397, 6400, 6408])
@pytest.mark.parametrize("off", [False, True])
def test_the_widest_fp32_rows_with_a_ring_backwards(B, cols, off, monkeypatch):
    """The last widths whose ring has room and the first ones beyond, on the 16-byte boundaries and off them."""
    import torch
    import tests.test_gpu_resnorm as R

    def moved(*args):
        i = inputs(*args)
        t, v = i["dr"]
        return {**i, "dr": (torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape).copy_(t), v)} if off else i

    monkeypatch.setattr(R, "inputs", moved)
    check(B, 330, cols, "float32", "float32", gate_rows=0, p=0.1, alpha=0.5)
