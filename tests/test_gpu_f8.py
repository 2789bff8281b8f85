"""8-bit floating point with a scale for each block of 128 against its definition in 64 bits: codes and scales bit for bit, products
within what fp32 accumulation can lose.

Tolerance of a product.  The tensor core adds 32 products at a time to an fp32 accumulator, and adding up a split reduction's
parts takes at most 8 more additions.  An addition drops what lies below 2^-23 of the larger operand (truncation; a rounding
would drop half of that), and no operand exceeds S = the sum of the products' magnitudes.  So an output is off by at most
(ceil(K / 32) * 2 + 8) * 2^-23 * S: two roundings for each instruction (its 32 products against one another, and with the
accumulator).  Then half a step of the output's type."""
import numpy as np
import pytest

from oracle import f8_oracle as F

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")


@pytest.fixture(scope="module")
def B():
    import paper_1805_11046_b200.binding as binding
    return binding


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def real(a, dtype):
    """A device tensor of the type, and its values in 64 bits."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(getattr(torch, dtype)).cuda()
    return t, t.double().cpu().numpy()


def half_step(dtype):
    import torch
    return torch.finfo(getattr(torch, dtype)).eps / 2


def host(t):
    return t.cpu().numpy()


def wide_values(rows, cols, seed, span=8):
    """Values over a range of magnitudes, zeros and whole blocks of zeros among them."""
    g = rng(seed)
    x = g.standard_normal((rows, cols)) * np.exp2(g.integers(-span, span + 1, (rows, 1)))
    x[g.random((rows, cols)) < 0.05] = 0.0
    x[: min(rows, 1), : min(cols, 128)] = 0.0
    return x


SHAPES = [(1, 16), (1, 4096), (2, 128), (3, 144), (127, 128), (128, 256), (129, 272), (300, 1008), (513, 640), (1000, 80)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fmt", [0, 1])
def test_codes_and_scales(B, rows, cols, dtype, fmt):
    x, v = real(wide_values(rows, cols, 11 * rows + cols), dtype)
    qr, sr, qc, sc = B.qbp_quantize_f8(x, format=fmt, cols=True)
    wq, we = F.quantize(v, fmt, 1, 128)
    assert np.array_equal(host(qr), wq) and np.array_equal(host(sr), F.pack(we, rows))
    cq, ce = F.quantize(v, fmt, 128, 1)
    assert np.array_equal(host(qc), cq) and np.array_equal(host(sc), F.pack(ce.T, cols))
    # each copy on its own
    assert all(np.array_equal(host(a), host(b)) for a, b in zip(B.qbp_quantize_f8(x, format=fmt), (qr, sr)))
    assert all(np.array_equal(host(a), host(b)) for a, b in zip(B.qbp_quantize_f8(x, format=fmt, rows=False, cols=True), (qc, sc)))
    q, s1, s2 = B.qbp_quantize_f8_square(x, format=fmt)
    sq, se = F.quantize(v, fmt, 128, 128)
    assert np.array_equal(host(q), sq)
    assert np.array_equal(host(s1), F.pack(F.spread(se, rows, 0), rows)) and np.array_equal(host(s2), F.pack(F.spread(se.T, cols, 0), cols))
    assert np.array_equal(host(B.qbp_f8_exponents(sr, rows, cols)), we)


@pytest.mark.parametrize("fmt", [0, 1])
def test_every_value_of_a_format_and_what_lies_between(B, fmt):
    """Blocks that hold every code's value, the middles between neighbours (ties) and their fp32 neighbours: at a scale of one, and
    of two where the neighbour above the largest value is among them."""
    t = F.table(fmt)
    t = np.sort(np.abs(t[np.isfinite(t)]))
    mid = ((t[1:] + t[:-1]) / 2).astype(np.float32)
    v = np.concatenate([t.astype(np.float32), mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(np.inf))])
    v = np.concatenate([v, -v, np.zeros(-len(v) * 2 % 120, np.float32)]).reshape(-1, 120)
    x = np.full((len(v), 128), F.MAX[fmt], np.float32)          # the largest value in every row's block: 2^0
    x[:, :120] = v
    xt, d = real(x, "float32")
    q, s = B.qbp_quantize_f8(xt, format=fmt)
    wq, we = F.quantize(d, fmt)
    assert set(we.ravel()) == {0, 1} and np.array_equal(host(q), wq) and np.array_equal(host(s), F.pack(we, len(x)))


def test_scales_at_the_ends_of_fp32(B):
    """Largest magnitudes just at, below and above 448 * 2^e, the smallest and the largest fp32 values."""
    amax = []
    for e in (-127, -126, -120, -1, 0, 1, 100, 119):
        m = np.float32(448.0 * 2.0 ** e)
        amax += [m, np.nextafter(m, np.float32(0)), np.nextafter(m, np.float32(np.inf))]
    amax += [np.float32(1e-45), np.float32(1.2e-38), np.finfo(np.float32).max, np.finfo(np.float32).tiny]
    x = np.zeros((len(amax), 128), np.float32)
    x[:, 5] = amax
    x[:, 77] = -np.array(amax, np.float32) / 3
    for fmt in (0, 1):
        xt, d = real(x, "float32")
        q, s = B.qbp_quantize_f8(xt, format=fmt)
        wq, we = F.quantize(d, fmt)
        assert np.array_equal(host(q), wq) and np.array_equal(host(s), F.pack(we, len(x)))


def test_rows_with_padding_and_off_the_16_byte_boundary(B):
    import torch
    for dtype in (torch.float32, torch.bfloat16):
        base = torch.from_numpy(wide_values(140, 300, 5).astype(np.float32)).to(dtype).cuda()
        for first, cols in ((0, 144), (16, 272), (3, 160), (1, 16)):
            x = base[:, first:first + cols]                      # rows 300 elements apart, first element anywhere
            for got, want in zip(B.qbp_quantize_f8(x, cols=True), B.qbp_quantize_f8(x.contiguous(), cols=True)):
                assert torch.equal(got, want)
            for got, want in zip(B.qbp_quantize_f8_square(x), B.qbp_quantize_f8_square(x.contiguous())):
                assert torch.equal(got, want)


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_block_that_is_not_finite_is_nan_and_no_other(B, bad):
    import torch
    M, N, K = 200, 144, 400
    x = rng(3).standard_normal((M, K)).astype(np.float32)
    x[17, 300] = bad
    w = rng(4).standard_normal((N, K)).astype(np.float32)
    xt, wt = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    q, s, qc, sc = B.qbp_quantize_f8(xt, cols=True)
    ex = host(B.qbp_f8_exponents(s, M, K)); assert (ex == 128).sum() == 1 and ex[17, 2] == 128
    assert (host(q)[17, 256:384] == 0x7F).all()
    exc = host(B.qbp_f8_exponents(sc, K, M)); assert (exc == 128).sum() == 1 and exc[300, 0] == 128
    wq, ws, wsc = B.qbp_quantize_f8_square(wt)
    y = host(B.qbp_gemm_f8(q, s, wq, ws, transB=True))
    assert np.isnan(y[17]).all() and np.isfinite(np.delete(y, 17, 0)).all()
    assert np.array_equal(host(B.qbp_linear_f8(xt, wq, ws)), y, equal_nan=True)
    for rows in (slice(15, 18), slice(17, 18), slice(10, 26)):                   # few rows: quantised on the way
        assert np.array_equal(host(B.qbp_linear_f8(xt[rows], wq, ws)), y[rows], equal_nan=True)
    # a product over the rows: only the outputs of column 300
    gq, gs = B.qbp_quantize_f8(torch.from_numpy(rng(5).standard_normal((M, 32)).astype(np.float32)).cuda(), rows=False, cols=True)
    dw = host(B.qbp_gemm_f8(gq, gs, qc, sc, transA=True))
    assert np.isnan(dw[:, 300]).all() and np.isfinite(np.delete(dw, 300, 1)).all()


def operand(B, outer, K, trans, fmt, seed, span=4):
    """Codes [outer, K] (trans: stored [K, outer]) with scales of many sizes, and the values they stand for [outer, K]."""
    import torch
    x = wide_values(outer, K, seed, span)
    xt = torch.from_numpy(np.ascontiguousarray(x.T if trans else x, np.float32)).cuda()
    q, s = B.qbp_quantize_f8(xt, format=fmt, rows=not trans, cols=trans)
    ex = host(B.qbp_f8_exponents(s, outer, K))
    codes = host(q).T if trans else host(q)
    return q, s, F.values(codes, fmt, F.spread(ex, K))


def check_product(got, a, b, K, dtype):
    want = a @ b.T
    size = np.abs(a) @ np.abs(b).T
    off = np.abs(got.double().cpu().numpy() - want)
    tol = (2 * -(-K // 32) + 8) * 2.0 ** -23 * size
    tol = tol + half_step(dtype) * (np.abs(want) + tol)
    if dtype == "float16": tol = tol + 2.0 ** -25                # half a step of the smallest fp16 values
    assert (off <= tol).all(), f"{(off / np.maximum(tol, 1e-300)).max()} of the tolerance"


# rows, columns, reduction: one token to many; a reduction in one block, in part of one, over several pieces of scales; odd outer extents
PRODUCTS = [(1, 16, 16), (1, 128, 128), (1, 4096, 4096), (2, 144, 512), (15, 1000, 640), (16, 128, 144), (17, 272, 2048), (33, 256, 1024),
            (64, 512, 528), (77, 1008, 2048), (100, 130, 256), (128, 128, 384), (129, 257, 512), (256, 256, 128), (300, 400, 1040),
            (513, 1024, 1024), (1111, 1520, 1024), (700, 640, 4112)]


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("transA,transB", [(False, True), (False, False), (True, False), (True, True)])
def test_products(B, M, N, K, transA, transB):
    if transA: M = -(-M // 16) * 16
    if not transB: N = -(-N // 16) * 16
    if transA and not transB: K = K + 5                          # a reduction that is nobody's innermost extent
    fa, fb = (M + N) % 2, (N // 16) % 2
    qa, sa, a = operand(B, M, K, transA, fa, M + 1)
    qb, sb, b = operand(B, N, K, not transB, fb, N + 2)
    import torch
    for dtype in TYPES[: 1 if M * N > 200000 else 3]:
        got = B.qbp_gemm_f8(qa, sa, qb, sb, transA=transA, transB=transB, formatA=fa, formatB=fb, out_dtype=getattr(torch, dtype))
        if dtype == "float16" and np.abs(a @ b.T).max() > 60000: continue
        check_product(got, a, b, K, dtype)
    assert B.status_word(B.workspace(256)) == 0


def check_on_device(got, a, b, K, dtype):
    """check_product with the 64-bit products taken on the device."""
    import torch
    a, b = torch.from_numpy(a).cuda(), torch.from_numpy(np.ascontiguousarray(b)).cuda()
    want = a @ b.T
    size = a.abs() @ b.abs().T
    tol = (2 * -(-K // 32) + 8) * 2.0 ** -23 * size
    tol = tol + half_step(dtype) * (want.abs() + tol)
    assert bool(((got.double() - want).abs() <= tol).all())


# more output tiles than the device has pairs of SMs, several rounds of them, ragged in every direction; an odd number of columns
# (rows that start off a 16-byte boundary); a reduction of one block and of many
@pytest.mark.parametrize("M,N,K,transA,transB", [(2600, 2100, 640, False, True), (5000, 4208, 272, False, False), (4112, 4000, 1003, True, False),
                                                 (2704, 2563, 400, True, True), (9000, 1001, 128, False, True), (2048, 2560, 2048, False, True),
                                                 (70000, 144, 256, False, False), (260, 40000, 144, False, True)])
def test_products_of_many_tiles(B, M, N, K, transA, transB):
    import torch
    qa, sa, a = operand(B, M, K, transA, 0, M + 1)
    qb, sb, b = operand(B, N, K, not transB, 1, N + 2)
    for dtype in ("float32", "bfloat16"):
        got = B.qbp_gemm_f8(qa, sa, qb, sb, transA=transA, transB=transB, formatB=1, out_dtype=getattr(torch, dtype))
        check_on_device(got, a, b, K, dtype)
    again = B.qbp_gemm_f8(qa, sa, qb, sb, transA=transA, transB=transB, formatB=1, out_dtype=torch.bfloat16)
    assert torch.equal(again, got)                                # the same bits every time
    assert B.status_word(B.workspace(256)) == 0


# few rows are quantised on the way to the tensor cores, more by the quantiser: one row, part of sixteen, more than sixteen, a part of a
# block of columns, several blocks and pieces; the rows padded
@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (1, 4096, 4096), (3, 256, 144), (15, 1008, 2048), (16, 8192, 1040), (17, 256, 8192), (33, 144, 528), (64, 2048, 2048),
                                   (77, 1008, 2048), (100, 4096, 4096), (128, 128, 4096), (129, 512, 1024), (300, 4096, 4096), (2000, 640, 256)])
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_is_the_quantiser_and_the_product(B, M, N, K, dtype):
    import torch
    x = torch.from_numpy(wide_values(M, K + 24, M + K).astype(np.float32)).to(getattr(torch, dtype)).cuda()[:, 8:8 + K]
    w = torch.from_numpy(rng(N).standard_normal((N, K)).astype(np.float32) * 2.0 ** -6).cuda()
    for fmt in (0, 1):
        wq, sw, _ = B.qbp_quantize_f8_square(w, format=fmt)
        q, s = B.qbp_quantize_f8(x)
        want = B.qbp_gemm_f8(q, s, wq, sw, transB=True, formatB=fmt, out_dtype=x.dtype)
        assert torch.equal(B.qbp_linear_f8(x, wq, sw, w_format=fmt), want)
        assert torch.equal(B.qbp_linear_f8(x.contiguous(), wq, sw, w_format=fmt), want)
    assert B.status_word(B.workspace(256)) == 0


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_of_rows_off_the_16_byte_boundary(B, dtype):
    import torch
    w = torch.from_numpy(rng(1).standard_normal((200, 400)).astype(np.float32)).cuda()
    wq, sw, _ = B.qbp_quantize_f8_square(w)
    for M in (1, 2, 9, 16, 17, 50):
        x = torch.from_numpy(wide_values(M, 407, M).astype(np.float32)).to(getattr(torch, dtype)).cuda()[:, 3:403]
        assert torch.equal(B.qbp_linear_f8(x, wq, sw), B.qbp_linear_f8(x.contiguous(), wq, sw))


@pytest.mark.parametrize("M,N,K,transA,transB", [(5, 256, 640, False, True), (100, 272, 1024, False, False), (144, 300, 512, True, True), (2600, 2112, 640, False, True),
                                                 (2608, 2112, 640, True, False)])
def test_a_nan_enters_its_own_outputs_alone(B, M, N, K, transA, transB):
    import torch
    x = torch.from_numpy(wide_values(M, K, 1).astype(np.float32)).cuda()
    y = torch.from_numpy(wide_values(N, K, 2).astype(np.float32)).cuda()
    ops = lambda x, y: B.qbp_quantize_f8(x.t().contiguous() if transA else x, rows=not transA, cols=transA) + B.qbp_quantize_f8(y if transB else y.t().contiguous(), rows=transB, cols=not transB)
    good = B.qbp_gemm_f8(*ops(x, y), transA=transA, transB=transB)
    assert bool(torch.isfinite(good).all())
    x[M // 2, K - 1] = float("nan"); y[3, 0] = float("inf")
    got = B.qbp_gemm_f8(*ops(x, y), transA=transA, transB=transB)
    bad = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    bad[M // 2] = True; bad[:, 3] = True
    assert torch.equal(torch.isnan(got), bad) and torch.equal(got[~bad], good[~bad])


@pytest.mark.parametrize("M,N,K", [(1, 32768, 4096), (2, 32768, 4096), (16, 19200, 2560), (3, 24016, 1040), (9, 20000, 528), (1, 19072, 16384), (16, 8192, 16384), (4, 8192, 8192), (8, 4096, 4096),
                                   (5, 512, 1024), (8, 20000, 256), (7, 144, 400)])
def test_linear_of_few_rows_and_many_features(B, M, N, K):
    """More tiles than SMs: two CTAs share one, each with a short ring that its quantising warps go round many times."""
    import torch
    x = torch.from_numpy(wide_values(M, K, M).astype(np.float32)).to(torch.bfloat16).cuda()
    w = torch.randint(0, 120, (N, K), dtype=torch.uint8, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    sw = torch.full((B._scale_bytes(N, K),), 120, dtype=torch.uint8, device="cuda")
    q, s = B.qbp_quantize_f8(x)
    want = B.qbp_gemm_f8(q, s, w, sw, transB=True, out_dtype=x.dtype)
    for _ in range(5): assert torch.equal(B.qbp_linear_f8(x, w, sw), want)
    assert B.status_word(B.workspace(256)) == 0


def test_small_products_of_many_streams(B):
    """Products in clusters that come to the SMs together: each has the tensor memory it needs, and the results are those of one at a time."""
    import torch
    shapes = [(1, 1024, 2048), (16, 512, 4096), (3, 2048, 1536), (40, 768, 2048), (100, 512, 2048), (128, 1024, 1024)]
    cases = []
    for i, (M, N, K) in enumerate(shapes):
        x = torch.from_numpy(wide_values(M, K, i).astype(np.float32)).cuda()
        wq, sw, _ = B.qbp_quantize_f8_square(torch.from_numpy(rng(i).standard_normal((N, K)).astype(np.float32)).cuda())
        cases.append((x, wq, sw, B.qbp_linear_f8(x, wq, sw), torch.cuda.Stream(), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    outs = [[torch.empty_like(c[3]) for _ in range(20)] for c in cases]
    for k in range(20):
        for (x, wq, sw, _, stream, ws), o in zip(cases, outs):
            with torch.cuda.stream(stream): B.qbp_linear_f8(x, wq, sw, y=o[k], ws=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(y, c[3]) for c, o in zip(cases, outs) for y in o) and all(B.status_word(c[5]) == 0 for c in cases)


def test_offsets_beyond_32_bits(B):
    """Codes, products and quantisation of more than 2^32 elements: the last rows are those of a call on the last rows alone."""
    import torch
    g = torch.Generator(device="cuda"); g.manual_seed(3)
    M, N, K, last = 70016, 65536, 256, 128
    x = torch.randn((M, K), generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.randn((N, K), generator=g, device="cuda", dtype=torch.bfloat16)
    q, s = B.qbp_quantize_f8(x)
    wq, sw = B.qbp_quantize_f8(w)
    y = B.qbp_gemm_f8(q, s, wq, sw, transB=True, out_dtype=torch.bfloat16)       # 4.6 G elements
    tail = B.qbp_quantize_f8(x[-last:].contiguous())
    assert torch.equal(q[-last:], tail[0])
    assert torch.equal(y[-last:], B.qbp_gemm_f8(*tail, wq, sw, transB=True, out_dtype=torch.bfloat16))
    del q, s, wq, sw, x, w
    yq, ys, yc, ysc = B.qbp_quantize_f8(y, cols=True)
    want = B.qbp_quantize_f8(y[-last:].contiguous(), cols=True)
    assert torch.equal(yq[-last:], want[0]) and torch.equal(yc[-last:], want[2])
    # a product that reads operands of that size: the last rows' outputs against 64 bits (a call on them alone adds up in another order)
    v = torch.randn((16, N), generator=g, device="cuda", dtype=torch.bfloat16)
    vq, vs = B.qbp_quantize_f8(v)
    z = B.qbp_gemm_f8(vq, vs, yq, ys, transB=True)
    a = F.values(host(vq), 0, F.spread(host(B.qbp_f8_exponents(vs, 16, N)), N))
    b = F.values(host(want[0]), 0, F.spread(host(B.qbp_f8_exponents(want[1], last, N)), N))
    check_on_device(z[:, -last:], a, b, N, "float32")
