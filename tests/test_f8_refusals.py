"""What the 8-bit floating-point products, the joins and dropout refuse, found on the host before anything is launched (runs
without a GPU), and the sizes they ask for."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_1805_11046_b200 import build
    build.build_library()
    from paper_1805_11046_b200 import binding
    return binding


P = 4096                                   # an address that is never followed: the call fails first
BIG = 1 << 40


def refused(B, status, call, *args, text=None):
    assert call(*args) == status, B.lib.qbp_last_error()
    if text: assert text in B.lib.qbp_last_error().decode()


def test_scale_bytes(B):
    for outer, k, want in ((0, 128, 0), (128, 0, 0), (1, 1, 512), (128, 512, 512), (129, 512, 1024), (128, 513, 1024), (300, 4096, 3 * 8 * 512)):
        assert B.lib.qbp_f8_scale_bytes(outer, k) == want == (B._scale_bytes(outer, k) if outer and k else 0)
    assert B.lib.qbp_gemm_f8_workspace_bytes(1, 1, 1) >= 4
    assert B.lib.qbp_linear_f8_workspace_bytes(100, 64, 256) >= 100 * 256 + 512 and B.lib.qbp_linear_f8_workspace_bytes(0, 64, 256) > 0


def test_quantiser(B):
    q = B.lib.qbp_quantize_f8
    ok = dict(x=P, dtype=0, rows=4, cols=32, ld=32, format=0, qr=P, sr=P, qc=P, sc=P)
    for change, status, text in ((dict(dtype=3), -1, "dtype"), (dict(dtype=-1), -1, "dtype"), (dict(format=2), -1, "format"), (dict(rows=-1), -1, "rows"),
                                 (dict(ld=31), -1, "ld"), (dict(cols=40, ld=40), -2, "multiple of 16"), (dict(x=None), -1, "x is NULL"), (dict(x=P + 2), -1, "misaligned"),
                                 (dict(sr=None), -1, "both"), (dict(qc=None), -1, "both"), (dict(qr=None, sr=None, qc=None, sc=None), -1, "both"),
                                 (dict(qr=P + 8), -1, "16-byte"), (dict(sc=P + 1), -1, "16-byte"), (dict(rows=1 << 24), -2, None)):
        a = {**ok, **change}
        refused(B, status, q, *a.values(), None, text=text)
    s = B.lib.qbp_quantize_f8_square
    for args, status in (((P, 1, 4, 32, 32, 0, None, P, P), -1), ((P, 1, 4, 32, 32, 0, P, None, None), -1), ((P, 1, 4, 33, 33, 0, P, P, P), -2), ((P + 1, 1, 4, 32, 32, 0, P, P, P), -1)):
        refused(B, status, s, *args, None)
    assert q(None, 0, 0, 32, 32, 0, P, P, None, None, None) == 0        # nothing to do, nothing launched
    assert q(None, 0, 0, 32, 32, 0, None, None, None, None, None) == 0  # (an empty tensor has no address)


def test_products(B):
    g = B.lib.qbp_gemm_f8
    ok = dict(ta=0, tb=1, M=5, N=7, K=32, fa=0, A=P, sA=P, fb=0, B=P, sB=P, dtype=0, out=P, ws=P, n=BIG)
    for change, status, text in ((dict(M=-1), -1, None), (dict(fa=2), -1, "format"), (dict(fb=-1), -1, "format"), (dict(dtype=7), -1, "dtype"), (dict(K=24), -2, "multiples of 16"),
                                 (dict(ta=1), -2, "multiples of 16"), (dict(tb=0), -2, "multiples of 16"), (dict(ta=1, M=16, tb=0, N=17, K=3), -2, None), (dict(A=None), -1, "16-byte"),
                                 (dict(B=P + 8), -1, "16-byte"), (dict(sA=P + 4), -1, "16-byte"), (dict(sB=None), -1, "16-byte"), (dict(out=None), -1, "out"), (dict(out=P + 2), -1, "out"),
                                 (dict(ws=None), -4, "workspace"), (dict(ws=P + 4), -4, "workspace"), (dict(n=8), -4, "workspace"), (dict(K=(1 << 30) + 16), -2, None)):
        a = {**ok, **change}
        refused(B, status, g, *a.values(), None, text=text)
    lin = B.lib.qbp_linear_f8
    ok = dict(x=P, dtype=1, ld=32, M=5, N=7, K=32, f=0, w=P, sw=P, y=P, ws=P, n=BIG)
    for change, status in ((dict(x=None), -1), (dict(ld=16), -1), (dict(K=40, ld=40), -2), (dict(w=None), -1), (dict(sw=P + 2), -1), (dict(y=None), -1), (dict(y=P + 1), -1),
                           (dict(f=9), -1), (dict(dtype=5), -1), (dict(n=300), -4), (dict(ws=None), -4)):
        a = {**ok, **change}
        refused(B, status, lin, *a.values(), None)


def desc(B, **change):
    d = dict(rows=4, cols=64, x_dtype=0, b_dtype=1, post=1, pre=1, eps=1e-6, alpha=1.0, gate_rows=0, p=0.0, tensor_id=0, seed=0, index_base=0)
    return B.ResnormDesc(**{**d, **change})


def fwd(B, d, x=P, b=P, w1=P, gate=P, w2=P, r=P, h=P, q1=P, q2=P, ws=P, n=BIG):
    return B.lib.qbp_resnorm_fwd(C.addressof(d) if d else None, x, b, w1, gate, w2, r, h, q1, q2, ws, n, None)


def bwd(B, d, dr=P, dh=P, b=P, r=P, q1=P, q2=P, w1=P, gate=P, w2=P, dx=P, db=P, dw1=P, dg=P, dw2=P, ws=P, n=BIG):
    return B.lib.qbp_resnorm_bwd(C.addressof(d) if d else None, dr, dh, b, r, q1, q2, w1, gate, w2, dx, db, dw1, dg, dw2, ws, n, None)


@pytest.mark.parametrize("change", [dict(x_dtype=3), dict(b_dtype=-1), dict(rows=-1), dict(cols=-8), dict(gate_rows=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                    dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(index_base=4)])
def test_join_descriptors(B, change):
    assert fwd(B, desc(B, **change)) == -1 and bwd(B, desc(B, **change)) == -1
    assert fwd(B, None) == -1 and bwd(B, None) == -1


def test_joins(B):
    assert fwd(B, desc(B, cols=B.QBP_RESNORM_MAX_COLS + 1)) == -2
    for kw in (dict(x=None), dict(x=P + 2), dict(b=P + 1), dict(h=None), dict(h=P + 1), dict(r=None), dict(w1=P + 2), dict(gate=P + 1), dict(q1=P + 2), dict(q2=P + 1)):
        assert fwd(B, desc(B), **kw) == -1, kw
    assert fwd(B, desc(B), ws=None) == -4 and fwd(B, desc(B), n=128) == -4 and fwd(B, desc(B), ws=P + 4) == -4
    # without a block output: no norm after it, gate or dropout; r may be left out where it is x
    assert fwd(B, desc(B), b=None) == -1 and fwd(B, desc(B, post=0), b=None) == -1 and fwd(B, desc(B, post=0, p=0.5), b=None, gate=None) == -1
    assert fwd(B, desc(B, post=0, alpha=0.5), b=None, gate=None, r=None) == -1 and fwd(B, desc(B, post=0, pre=0), b=None, gate=None, r=None) == -1
    for kw in (dict(dh=None), dict(r=None), dict(q1=None), dict(q2=None), dict(b=P + 1), dict(dx=P + 2), dict(db=P + 1), dict(dw1=P + 2), dict(dx=None, db=None, dw1=None, dg=None, dw2=None)):
        assert bwd(B, desc(B), **kw) == -1, kw
    assert bwd(B, desc(B), b=None) == -1                                # db of no block output
    assert bwd(B, desc(B, post=0)) == -1 and bwd(B, desc(B, pre=0)) == -1          # gradients of norms that are not there
    assert bwd(B, desc(B, pre=0), dr=None, dw2=None) == -1              # neither r nor h has a gradient
    assert bwd(B, desc(B), ws=None) == -4 and bwd(B, desc(B), n=700) == -4 and bwd(B, desc(B), ws=P + 16) == -4
    assert all(f(B, desc(B, **kw), ws=None) == 0 for f, kw in ((fwd, dict(rows=0)), (fwd, dict(cols=0)), (bwd, dict(cols=0))))


def test_join_workspace_covers_every_cut(B):
    need = lambda **kw: B.qbp_resnorm_bwd_workspace_bytes(desc(B, **kw))
    for kw in (dict(rows=1), dict(rows=10 ** 6), dict(cols=1), dict(cols=16384, rows=9), dict(rows=1000, gate_rows=1), dict(rows=1000, gate_rows=999), dict(rows=0)):
        assert need(**kw) >= 256
    # a partial row of each gate's gradient for each of its items, but none where a gate's rows are one item
    few, many = need(rows=10 ** 6, gate_rows=1), need(rows=10 ** 6, gate_rows=10 ** 6)
    assert few <= many and few < 10 ** 6 * 64 * 4 and many >= 3 * 100 * 64 * 4


def test_a_layers_words_and_scratch():
    """Each call has a status word of its own; outgrown workspaces stay where they are."""
    import torch
    from paper_1805_11046_b200 import layer
    s = layer._F8Space(3, "cpu")
    assert s.status() == 0
    a = s.at(1)
    a[:4].view(torch.int32)[0] = -6
    assert s.status() == -6 and s.get().numel() == 768 and s.at(2).data_ptr() == a.data_ptr() + 256
    b = s.at(2, 5000)
    assert b.numel() >= 5256 and b.data_ptr() % 256 == s.get().data_ptr() % 256 and s.at(1).data_ptr() != a.data_ptr()
    assert s.status() == -6 and int(a[:4].view(torch.int32)[0]) == -6
    a[:4] = 0
    assert s.status() == 0
    for n in range(5000, 9000, 7): s.get(n)
    assert len(s.kept) <= 4 and sum(t.numel() for t in s.kept) <= 2 * s.get().numel()


def test_dropout(B):
    d = B.lib.qbp_dropout
    for args in ((None, 0, 8, 0.5, 0, 0, 0, P), (P, 0, 8, 0.5, 0, 0, 0, None), (P + 2, 0, 8, 0.5, 0, 0, 0, P), (P, 1, 8, 0.5, 0, 0, 0, P + 1), (P, 3, 8, 0.5, 0, 0, 0, P), (P, 0, -1, 0.5, 0, 0, 0, P),
                 (P, 0, 8, -0.01, 0, 0, 0, P), (P, 0, 8, 1.01, 0, 0, 0, P), (P, 0, 8, float("nan"), 0, 0, 0, P), (P, 0, 8, 0.5, 0, 0, 4, P)):
        refused(B, -1, d, *args, None)
    assert d(None, 0, 0, 0.5, 0, 0, 0, None, None) == 0


class Elsewhere:
    """As much of a tensor as the check of devices looks at."""
    device = "cuda:1"

    def get_device(self):
        return 1


def test_tensors_of_another_device_and_type(B, monkeypatch):
    import torch
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:1"):
        B._here(None, Elsewhere())
    with pytest.raises(TypeError, match="float64"):
        B._dtype(torch.float64)
    with pytest.raises(TypeError, match="bytes"):
        B._codes(torch.zeros(4))
    with pytest.raises(ValueError, match="dense"):
        B._rows_of(torch.zeros(4, 6).t())
    with pytest.raises(ValueError, match="contiguous"):
        B._rows_of(torch.zeros(4, 6, 8).transpose(0, 1))
    assert B._rows_of(torch.zeros(4, 6)[:, 1:3]) == (4, 2, 6) and B._rows_of(torch.zeros(2, 3, 8)) == (6, 8, 8) and B._rows_of(torch.zeros(1, 6)[:, :4]) == (1, 4, 4)
    with pytest.raises(ValueError, match="scales of"):
        B._scales_fit(torch.zeros(511, dtype=torch.uint8), 128, 512, "sA")
    with pytest.raises(ValueError, match="elements"):
        B._real(torch.zeros(5), 4, torch.float32, "x")
    with pytest.raises(TypeError, match="bfloat16 is wanted"):
        B._real(torch.zeros(4), 4, torch.bfloat16, "x")
    with pytest.raises(ValueError, match="dense"):
        B._real(torch.zeros(2, 4).t(), 8, torch.float32, "x")


def test_structs_match_the_header(B):
    assert C.sizeof(B.ResnormDesc) == 72
