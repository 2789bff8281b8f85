"""The join of two blocks, its gradients and dropout against their definitions in 64 bits.

Tolerances, with u = 2^-24 and every sum taken from the inputs alone:
  1 / RMS          a thread adds at most 32 squares, a warp 5 sums, a block 16: 60 u of a sum of positive terms, half of it after the root,
                   then the mean, eps, the root and the quotient: 40 u.
  r                products of the block's part 5 u, its 1 / RMS 40 u, the sum 2 u: 48 u (|alpha x| + |gate d|); then half a step of r's type.
  h                from the stored r: 40 u + 3 u; half a step of its type.
  R (dx)           1 / RMS enters up to three times (120 u), the mean's sum 60 u, the elementwise steps 10 u: 200 u of the sum of the
                   terms' magnitudes.
  db               the same of the other norm on top: 400 u of the terms' magnitudes.
  sums over rows   one addition a row on top of what their terms are off: (rows + 300) u of the sum of magnitudes.
Dropout is one product, rounded to fp32 and then to the type: bit for bit for fp32; for the halves the value in 64 bits is off by
half a step of the type and u."""
import numpy as np
import pytest

from oracle import f8_oracle as F

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-6


@pytest.fixture(scope="module")
def B():
    import paper_1805_11046_b200.binding as binding
    return binding


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def real(a, dtype):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(getattr(torch, dtype)).cuda()
    return t, t.double().cpu().numpy()


def host(t):
    return t.double().cpu().numpy()


def half_step(dtype):
    import torch
    return torch.finfo(getattr(torch, dtype)).eps / 2


def close(got, want, tol, dtype="float32"):
    tol = tol + half_step(dtype) * (np.abs(want) + tol) + (2.0 ** -25 if dtype == "float16" else 2.0 ** -149)
    off = np.abs(host(got).reshape(want.shape) - want)
    assert (off <= tol).all(), f"{(off / tol).max()} of the tolerance"


def inputs(rows, cols, stream, dtype, gates, seed):
    g = rng(seed)
    x = g.standard_normal((rows, cols)) * np.exp2(g.integers(-3, 4, (rows, 1)))
    b = g.standard_normal((rows, cols)) * np.exp2(g.integers(-3, 4, (rows, 1)))
    if rows > 2: b[1] = 0.0                                         # a block that puts out nothing
    out = dict(x=real(x, stream), b=real(b, dtype), w1=real(1 + 0.2 * g.standard_normal(cols), "float32"),
               w2=real(1 + 0.2 * g.standard_normal(cols), "float32"), gate=real(0.5 + 0.3 * g.standard_normal((gates, cols)), "float32"),
               dr=real(g.standard_normal((rows, cols)), stream), dh=real(g.standard_normal((rows, cols)), dtype))
    return out


def check(B, rows, cols, stream, dtype, gate_rows, p, alpha, post=True, pre=True, w1=True, w2=True, gate=True, dr=True, seed=0, index_base=0):
    i = inputs(rows, cols, stream, dtype, -(-rows // gate_rows) if gate_rows else 1, seed + rows + cols)
    x, b = i["x"], i["b"]
    none = (None, None)
    w1, w2, gt = i["w1"] if w1 else none, i["w2"] if w2 else none, i["gate"] if gate else none
    d = B.resnorm_desc(x[0], b[0], alpha=alpha, eps=EPS, gate_rows=gate_rows, p=p, seed=77, tensor_id=5, index_base=index_base, post=post, pre=pre)
    r, h, q1, q2 = B.qbp_resnorm_fwd(d, x[0], b[0], w1[0], gt[0], w2[0])
    mask = F.keep((rows, cols), p, 77, 5, index_base) if p else np.ones((rows, cols))
    rd = host(r)
    exact, _, hw, e1, e2 = F.join(x[1], b[1], w1[1], gt[1], w2[1], alpha, EPS, gate_rows, mask, lambda v: rd, post, pre)
    close(r, exact, 48 * U * (np.abs(alpha * x[1]) + np.abs(exact - alpha * x[1])), stream)
    if post: close(q1, e1, 40 * U * e1)
    if pre:
        close(q2, e2, 40 * U * e2)
        close(h, hw, 43 * U * np.abs(hw), dtype)
    dr_, dh = i["dr"] if dr else none, i["dh"] if pre else none
    dx, db, dw1, dg, dw2 = B.qbp_resnorm_bwd(d, dr_[0], dh[0], b[0], r, q1, q2, w1[0], gt[0], w2[0])
    ones = np.ones(cols)
    W1, W2 = (ones if w1[1] is None or not post else w1[1]), (ones if w2[1] is None else w2[1])
    ex, eb, ew1, eg, ew2 = F.join_gradients(dr_[1], dh[1], b[1], rd, e1, e2, w1[1], gt[1], w2[1], alpha, gate_rows, mask, post, pre)
    SR = np.zeros((rows, cols)) if not dr else np.abs(dr_[1])
    if pre:
        a, rh = np.abs(dh[1] * W2), np.abs(rd * e2[:, None])
        SR = SR + e2[:, None] * (a + rh * (a * rh).mean(1, keepdims=True))
        close(dw2, ew2, (rows + 300) * U * (np.abs(dh[1]) * rh).sum(0))
    close(dx, ex, 200 * U * abs(alpha) * SR, stream)
    at = np.arange(rows) // gate_rows if gate_rows else np.zeros(rows, int)
    g = np.ones((rows, cols)) if gt[1] is None else gt[1][at]
    bh = np.abs(b[1] * e1[:, None]) if post else np.abs(b[1])
    Sz = SR * np.abs(g * mask * W1)
    Sdb = e1[:, None] * (Sz + bh * (Sz * bh).mean(1, keepdims=True)) if post else Sz
    close(db, eb, 400 * U * Sdb, dtype)
    if post: close(dw1, ew1, (rows + 300) * U * (SR * np.abs(g * mask) * bh).sum(0))
    if gate:
        Sg = np.zeros_like(eg)
        np.add.at(Sg, at, SR * np.abs(mask * W1) * bh)
        close(dg, eg, (rows + 300) * U * Sg)
    else:
        assert dg is None


# rows of one element, of part of a chunk of eight, of whole chunks; one group of threads of every kind just filled and just passed
SHAPES = [(1, 1), (1, 8), (3, 7), (5, 64), (17, 256), (33, 257), (9, 264), (12, 512), (64, 1000), (7, 1024), (9, 1032), (4, 2048), (5, 2049), (6, 4096), (3, 4100),
          (2, 8192), (3, 8200), (2, 16384), (1, 16383), (777, 96), (2100, 520), (400, 1500)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("stream,dtype", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("float32", "float32"), ("float16", "float16"), ("bfloat16", "float32")])
def test_join_and_gradients(B, rows, cols, stream, dtype):
    check(B, rows, cols, stream, dtype, gate_rows=0, p=0.2, alpha=0.75)


# rows off the 16-byte boundaries in every kind of group, enough of them for a block to take several; rows shorter than 32 bytes; the last
# lanes' columns missing
@pytest.mark.parametrize("rows,cols", [(4000, 3), (5000, 13), (3000, 201), (3000, 333), (1300, 513), (1300, 1001), (1000, 2047), (700, 3331), (700, 4095), (500, 5003), (400, 8191)])
@pytest.mark.parametrize("stream,dtype", [("float32", "bfloat16"), ("bfloat16", "bfloat16"), ("float32", "float32"), ("float16", "float32")])
def test_rows_off_the_16_byte_boundaries(B, rows, cols, stream, dtype):
    check(B, rows, cols, stream, dtype, gate_rows=[0, rows // 3, 1][rows // 100 % 3] if cols < 3000 else 0, p=0.1 if cols % 4 == 1 else 0.0, alpha=0.5)


@pytest.mark.parametrize("cols", [7, 333, 1001, 4095])
def test_outputs_over_inputs_off_the_16_byte_boundaries(B, cols):
    """A row's copy takes bytes of the rows beside it, which another block may be writing: they count for nothing."""
    import torch
    i = inputs(2500, cols, "float32", "bfloat16", 1, 4)
    x, b, dr, dh = (i[k][0] for k in ("x", "b", "dr", "dh"))
    d = B.resnorm_desc(x, b, alpha=0.5, eps=EPS, p=0.2, seed=3)
    r, h, q1, q2 = B.qbp_resnorm_fwd(d, x, b, i["w1"][0], i["gate"][0], i["w2"][0])
    want = B.qbp_resnorm_bwd(d, dr, dh, b, r, q1, q2, i["w1"][0], i["gate"][0], i["w2"][0])
    x2, b2, dr2, dh2 = x.clone(), b.clone(), dr.clone(), dh.clone()
    got = B.qbp_resnorm_fwd(d, x2, b2, i["w1"][0], i["gate"][0], i["w2"][0], r=x2, h=b2)
    assert all(torch.equal(u, v) for u, v in zip(got, (r, h, q1, q2)))
    got = B.qbp_resnorm_bwd(d, dr2, dh2, b, r, q1, q2, i["w1"][0], i["gate"][0], i["w2"][0], dx=dr2, db=dh2)
    assert all(torch.equal(u, v) for u, v in zip(got, want))


@pytest.mark.parametrize("rows,cols,gate_rows", [(1, 64, 1), (10, 64, 1), (10, 200, 3), (333 * 3, 1000, 333), (1000, 48, 7), (50, 2056, 20), (600, 1536, 600), (601, 1536, 600), (4, 16384, 2)])
def test_gates_of_groups_of_rows(B, rows, cols, gate_rows):
    check(B, rows, cols, "float32", "bfloat16", gate_rows=gate_rows, p=0.0, alpha=1.0)


@pytest.mark.parametrize("cols", [72, 2504])
@pytest.mark.parametrize("post,pre", [(True, False), (False, True), (False, False), (True, True)])
@pytest.mark.parametrize("w,gate,dr", [(True, True, True), (False, False, True), (True, False, False), (False, True, True)])
def test_parts_left_out(B, cols, post, pre, w, gate, dr):
    if not pre and not dr: dr = True                                # (a join of which nothing has a gradient)
    check(B, 41, cols, "float32", "float32", gate_rows=0, p=0.1, alpha=1.0, post=post, pre=pre, w1=w, w2=w, gate=gate, dr=dr)


def test_everything_dropped_and_nothing(B):
    check(B, 5, 80, "float32", "float32", gate_rows=0, p=1.0, alpha=1.0)
    check(B, 5, 80, "float32", "float32", gate_rows=0, p=2.0 ** -18, alpha=1.0)     # rounds to none
    check(B, 5, 77, "bfloat16", "float32", gate_rows=2, p=0.5, alpha=1.0, index_base=(1 << 35) + 8)


@pytest.mark.parametrize("cols", [64, 1000, 4096])
def test_the_norm_before_a_first_block(B, cols):
    import torch
    i = inputs(30, cols, "bfloat16", "float32", 1, 3)
    (x, xv), (w, wv), (dh, dhv), (dr, drv) = i["x"], i["w2"], real(rng(4).standard_normal((30, cols)), "bfloat16"), i["dr"]
    d = B.resnorm_desc(x, eps=EPS)
    r, h, q1, q2 = B.qbp_resnorm_fwd(d, x, w_pre=w)
    assert r is None and q1 is None
    e2 = 1 / np.sqrt((xv * xv).mean(1) + EPS)
    close(h, xv * e2[:, None] * wv, 43 * U * np.abs(xv * e2[:, None] * wv), "bfloat16")
    dx, db, dw1, dg, dw2 = B.qbp_resnorm_bwd(d, dr, dh, None, x, None, q2, w_pre=w)
    assert db is None and dw1 is None and dg is None
    rh = xv * e2[:, None]; u = dhv * wv
    want = drv + e2[:, None] * (u - rh * (u * rh).mean(1, keepdims=True))
    S = np.abs(drv) + e2[:, None] * (np.abs(u) + np.abs(rh) * (np.abs(u * rh)).mean(1, keepdims=True))
    close(dx, want, 200 * U * S, "bfloat16")
    close(dw2, (dhv * rh).sum(0), 330 * U * np.abs(dhv * rh).sum(0))


@pytest.mark.parametrize("off", ["x", "b", "w1", "gate", "dr", "dh"])
def test_tensors_off_the_16_byte_boundary(B, off):
    """Any one of them: the values of the aligned call, up to the other form's order of sums."""
    import torch
    i = {k: v[0] for k, v in inputs(21, 512, "float32", "bfloat16", 1, 31).items()}
    moved = torch.empty(i[off].numel() + 1, dtype=i[off].dtype, device="cuda")[1:].view(i[off].shape).copy_(i[off])
    outs = []
    for t in (i, {**i, off: moved}):
        d = B.resnorm_desc(t["x"], t["b"], p=0.3, seed=4)
        r, h, q1, q2 = B.qbp_resnorm_fwd(d, t["x"], t["b"], t["w1"], t["gate"], t["w2"])
        outs.append((r, h, q1, q2) + B.qbp_resnorm_bwd(d, t["dr"], t["dh"], t["b"], r, q1, q2, t["w1"], t["gate"], t["w2"]))
    # both are within the bounds above of the same values: twice the largest of them, relative to each tensor's largest value
    for a, b in zip(*outs):
        assert torch.equal(a == 0, b == 0) or a.dtype == torch.bfloat16
        assert float((a.double() - b.double()).abs().max()) <= 2 * (800 * U + half_step(str(a.dtype).split(".")[1])) * 16 * float(a.double().abs().max())


def test_more_than_2_to_the_32_elements(B):
    """The last rows of a long join and the last elements of a long dropout are those of calls on them alone."""
    import torch
    rows, cols, last = 270000, 16384, 3
    x = torch.randn(1024, cols, device="cuda", dtype=torch.bfloat16).repeat(264, 1)[:rows]
    b = x.flip(0)
    g = torch.rand(cols, device="cuda")
    d = B.resnorm_desc(x, b, p=0.25, seed=6)
    r, h, q1, q2 = B.qbp_resnorm_fwd(d, x, b, g, g, g)
    at = (rows - last) * cols
    e = B.resnorm_desc(x[-last:], b[-last:], p=0.25, seed=6, index_base=at)
    r2, h2, p1, p2 = B.qbp_resnorm_fwd(e, x[-last:], b[-last:], g, g, g)
    assert torch.equal(r[-last:], r2) and torch.equal(h[-last:], h2) and torch.equal(q1[-last:], p1)
    dr3, dh3 = x[-last:].clone(), h2.clone()
    dx, db, _, _, _ = B.qbp_resnorm_bwd(d, x, h, b, r, q1, q2, g, g, g, want_params=False, dx=x, db=h)
    dx3, db3, _, _, _ = B.qbp_resnorm_bwd(e, dr3, dh3, b[-last:], r2, p1, p2, g, g, g, want_params=False)
    assert torch.equal(dx[-last:], dx3) and torch.equal(db[-last:], db3)
    del d, dx, db
    y = B.qbp_dropout(r, 0.5, 9)
    assert torch.equal(y.view(-1)[at:], B.qbp_dropout(r[-last:], 0.5, 9, index_base=at).view(-1))


def test_outputs_over_inputs(B):
    """r over x, h over b; dx over dr, db over dh: the same bits."""
    import torch
    for cols in (200, 4096):
        i = inputs(19, cols, "bfloat16", "bfloat16", 1, 9)
        x, b, w1, w2, gate, dr, dh = (i[k][0] for k in ("x", "b", "w1", "w2", "gate", "dr", "dh"))
        d = B.resnorm_desc(x, b, p=0.3, seed=1)
        r, h, q1, q2 = B.qbp_resnorm_fwd(d, x, b, w1, gate, w2)
        x2, b2 = x.clone(), b.clone()
        r2, h2, p1, p2 = B.qbp_resnorm_fwd(d, x2, b2, w1, gate, w2, r=x2, h=b2)
        assert torch.equal(r, r2) and torch.equal(h, h2) and torch.equal(q1, p1) and torch.equal(q2, p2)
        first = B.qbp_resnorm_bwd(d, dr, dh, b, r, q1, q2, w1, gate, w2)
        dr2, dh2 = dr.clone(), dh.clone()
        second = B.qbp_resnorm_bwd(d, dr2, dh2, b, r, q1, q2, w1, gate, w2, dx=dr2, db=dh2)
        assert all(torch.equal(a, c) for a, c in zip(first, second))


def test_the_gradient_against_differences(B):
    """sum(r a) + sum(h c) along a direction in every input at once, by central differences of the forward in fp32: steps of 2^-7,
    whose third-order term is below 1e-3 of the slope here and whose rounding is 2 sqrt(n) u / 2^-7 of the sum's terms."""
    import torch
    rows, cols = 24, 200
    i = inputs(rows, cols, "float32", "float32", 3, 21)
    t = {k: i[k][0] for k in ("x", "b", "w1", "w2", "gate")}
    t["b"][1] += 1.0                                                # (a row of zeros has no derivative in RMS at this step)
    d = B.resnorm_desc(t["x"], t["b"], alpha=0.8, eps=EPS, gate_rows=8, p=0.2, seed=9, tensor_id=1)
    a, c = i["dr"][0], i["dh"][0]
    g = rng(22)
    step = {k: torch.from_numpy(g.standard_normal(v.shape).astype(np.float32)).cuda() * v.abs().mean() for k, v in t.items()}

    def value(s):
        m = {k: t[k] + s * step[k] for k in t}
        r, h, _, _ = B.qbp_resnorm_fwd(d, m["x"], m["b"], m["w1"], m["gate"], m["w2"])
        return float((r.double() * a.double()).sum() + (h.double() * c.double()).sum())

    r, h, q1, q2 = B.qbp_resnorm_fwd(d, t["x"], t["b"], t["w1"], t["gate"], t["w2"])
    dx, db, dw1, dg, dw2 = B.qbp_resnorm_bwd(d, a, c, t["b"], r, q1, q2, t["w1"], t["gate"], t["w2"])
    slope = sum(float((x.double() * step[k].double()).sum()) for x, k in ((dx, "x"), (db, "b"), (dw1, "w1"), (dg, "gate"), (dw2, "w2")))
    s = 2.0 ** -7
    size = sum(float((x.double() * step[k].double()).abs().sum()) for x, k in ((dx, "x"), (db, "b"), (dw1, "w1"), (dg, "gate"), (dw2, "w2")))
    assert abs((value(s) - value(-s)) / (2 * s) - slope) <= 1e-3 * size


# ------------------------------------------------------------------------ dropout
@pytest.mark.parametrize("n", [1, 7, 8, 9, 2048, 12345, 100003])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_dropout(B, n, dtype):
    x, v = real(rng(n).standard_normal(n), dtype)
    for p, base in ((0.0, 0), (0.1, 0), (0.25, 8), (0.5, (1 << 36) + 16), (0.9999, 0), (1.0, 0)):
        y = B.qbp_dropout(x, p, 1234567890123, tensor_id=7, index_base=base)
        k = F.keep((n,), p, 1234567890123, 7, base)
        assert np.array_equal(host(y) != 0, (k != 0) & (v != 0))
        if dtype == "float32":
            assert np.array_equal(y.cpu().numpy(), (v * np.float32(k)).astype(np.float32))
        close(y, v * k, 2 * U * np.abs(v * k), dtype)


def test_dropout_of_a_shard_continues_the_whole(B):
    import torch
    x = torch.randn(4096 + 24, device="cuda")
    whole = B.qbp_dropout(x, 0.3, 5, 2, index_base=64)
    assert torch.equal(B.qbp_dropout(x[1000:], 0.3, 5, 2, index_base=64 + 1000), whole[1000:])
    assert torch.equal(B.qbp_dropout(x[8:].clone()[:777], 0.3, 5, 2, index_base=72), whole[8:785])
    assert torch.equal(B.qbp_dropout(x, 0.3, 5, 2, index_base=64, y=x), whole) and torch.equal(x, whole)     # in place
    off = torch.randn(1001, device="cuda").to(torch.bfloat16)[1:]                                            # off the 16-byte boundary
    assert torch.equal(B.qbp_dropout(off, 0.3, 5), B.qbp_dropout(off.clone(), 0.3, 5))


def test_what_is_dropped_is_zero_whatever_it_was(B):
    import torch
    x = torch.full((4096,), float("nan"), device="cuda")
    x[::3] = float("inf")
    y = host(B.qbp_dropout(x, 0.5, 3))
    k = F.keep((4096,), 0.5, 3, 0)
    assert (y[k == 0] == 0).all() and not np.isfinite(y[k != 0]).any()
    # the same in a join: the dropped places of the block's output count for nothing
    b = torch.ones(2, 512, device="cuda"); b[0] = x[:512]
    xs = torch.randn(2, 512, device="cuda")
    d = B.resnorm_desc(xs, b, p=0.5, seed=3, post=False)
    r, h, _, q2 = B.qbp_resnorm_fwd(d, xs, b)
    k = k[:1024].reshape(2, 512)
    assert np.array_equal(host(r)[0][k[0] == 0], host(xs)[0][k[0] == 0]) and not np.isfinite(host(r)[0][k[0] != 0]).any()
    assert np.isfinite(host(h)[1]).all()


def test_draws_are_spread_evenly(B):
    """Of 2^22 draws a share p goes, to 5 standard deviations; neighbours' masks are independent to the same."""
    import torch
    n = 1 << 22
    for p in (0.1, 0.5):
        kept = (B.qbp_dropout(torch.ones(n, device="cuda"), p, 17, 4) != 0).double()
        t = np.floor(float(np.float32(p)) * 65536 + 0.5) / 65536
        sd = np.sqrt(t * (1 - t) / n)
        assert abs(float(kept.mean()) - (1 - t)) < 5 * sd
        z = kept - (1 - t)
        assert abs(float((z[1:] * z[:-1]).mean())) < 5 * t * (1 - t) / np.sqrt(n)
