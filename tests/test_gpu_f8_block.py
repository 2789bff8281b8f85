"""Residual blocks of 8-bit floating-point linear layers, joined by norms, gate and dropout: forward, backward and update as a
training program runs them, each stage against its definition in 64 bits on the tensors that the device produced; the same in a
captured graph, on other streams and from several threads."""
import threading

import numpy as np
import pytest

from oracle import f8_oracle as F
from tests.test_gpu_f8 import check_product, half_step, host
from tests.test_gpu_resnorm import U, close, real, rng
from tests.test_gpu_resnorm import host as values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_1805_11046_b200.binding as binding
    return binding


def make(rows, C, blocks, p, stream="float32", seed=0, **kw):
    import torch
    from paper_1805_11046_b200 import layer
    g = rng(seed)
    w = [torch.from_numpy((g.uniform(-1, 1, (C, C)) * np.sqrt(6.0 / C)).astype(np.float32)).cuda() for _ in range(blocks)]
    x = real(g.standard_normal((rows, C)), stream)[0]
    dh = real(g.standard_normal((rows, C)) * 0.01, "bfloat16")[0]
    return layer.F8ResidualStack(w, alpha=0.9, p=p, seed=5, **kw), x, dh


def codes_are(B, q, s, x, fmt, along, square=False):
    """Codes and scales of a tensor, bit for bit, and the values they stand for."""
    v = values(x)
    wq, e = F.quantize(v, fmt, 128 if square or not along else 1, 128 if square or along else 1)
    assert np.array_equal(host(q), wq)
    outer, k = v.shape if along else v.shape[::-1]
    e = e if along else e.T
    if square: e = F.spread(e, outer, 0)
    assert np.array_equal(host(s), F.pack(e, outer))
    full = F.spread(e, k)
    return F.values(wq, fmt, full if along else full.T)


@pytest.mark.parametrize("rows,C,p", [(96, 128, 0.0), (200, 400, 0.25), (33, 1024, 0.1)])
def test_a_training_step_stage_by_stage(B, rows, C, p):
    import torch
    st, x, dh = make(rows, C, 2, p)
    lin, calls = st.linears[0], []
    # what passes between the stages, as the device has it
    fwd_, bwd_ = [l.forward for l in st.linears], [l.backward for l in st.linears]
    for i, l in enumerate(st.linears):
        l.forward = lambda h, i=i: calls.append(("f", i, h, fwd_[i](h))) or calls[-1][3]
        l.backward = lambda g, i=i: calls.append(("b", i, g, bwd_[i](g))) or calls[-1][3]
    h = st.forward(x)
    dx = st.backward(dh)
    torch.cuda.synchronize()
    assert st.status() == 0
    first, _, q, joins = st.saved
    xv = values(x)
    e = 1 / np.sqrt((xv * xv).mean(1) + 1e-6)
    close(calls[0][2], xv * e[:, None], 43 * U * np.abs(xv * e[:, None]), "bfloat16")
    stream = xv
    for (_, i, hin, b), (d, _, r, q1, q2) in zip(calls[:2], joins):
        l = st.linears[i]
        a = codes_are(B, *B.qbp_quantize_f8(hin), hin, 0, True)
        w = codes_are(B, l.codes[0], l.codes[1], l.w, 0, True, square=True)
        check_product(b, a, w, C, "bfloat16")
        mask = F.keep((rows, C), p, 5, i) if p else np.ones((rows, C))
        bv, rv = values(b), values(r)
        exact, _, hw, e1, e2 = F.join(stream, bv, np.ones(C), np.ones((1, C)), np.ones(C), float(np.float32(0.9)), 1e-6, 0, mask, lambda v: rv)
        close(r, exact, 48 * U * (np.abs(0.9 * stream) + np.abs(exact - 0.9 * stream)))
        close(q1, e1, 40 * U * e1); close(q2, e2, 40 * U * e2)
        close(calls[i + 1][2] if i == 0 else h, hw, 43 * U * np.abs(hw), "bfloat16")
        stream = rv
    # backwards: the gradient at the last h, then block by block
    dr, grad = None, dh
    for _, i, db, dhin in calls[2:]:
        d, b, r, q1, q2 = joins[i]
        mask = F.keep((rows, C), p, 5, i) if p else np.ones((rows, C))
        rv, bv = values(r), values(b)
        e1, e2 = 1 / np.sqrt((bv * bv).mean(1) + 1e-6), 1 / np.sqrt((rv * rv).mean(1) + 1e-6)
        ex, eb, ew1, eg, ew2 = F.join_gradients(None if dr is None else values(dr), values(grad), bv, rv, e1, e2, None, np.ones((1, C)), None, float(np.float32(0.9)), 0, mask)
        a, rh = np.abs(values(grad)), np.abs(rv * e2[:, None])
        SR = (0 if dr is None else np.abs(values(dr))) + e2[:, None] * (a + rh * (a * rh).mean(1, keepdims=True))
        Sz, bh = SR * mask, np.abs(bv * e1[:, None])
        close(db, eb, 400 * U * e1[:, None] * (Sz + bh * (Sz * bh).mean(1, keepdims=True)), "bfloat16")
        close(st.grads[0][i][1], ew1, (rows + 300) * U * (Sz * bh).sum(0))
        close(st.grads[0][i][2], eg[0], (rows + 300) * U * (Sz * bh).sum(0))
        close(st.grads[0][i][3], ew2, (rows + 300) * U * (a * rh).sum(0))
        l, hin = st.linears[i], calls[i][2]
        g8 = codes_are(B, *B.qbp_quantize_f8(db, format=1), db, 1, True)
        w = codes_are(B, l.codes[0], l.codes[2], l.w, 0, False, square=True)
        check_product(dhin, g8, w.T, C, "bfloat16")
        gt = codes_are(B, *B.qbp_quantize_f8(db, format=1, rows=False, cols=True), db, 1, False)
        ht = codes_are(B, *l.saved, hin, 0, False)
        check_product(l.dw, gt.T, ht.T, rows, "float32")
        # the gradient at the stream before this join (a call of its own: the stack hands it on at once)
        dr, _, _, _, _ = B.qbp_resnorm_bwd(d, dr, grad, b, r, q1, q2, st.w_post[i], st.gate[i], st.w_pre[i])
        close(dr, ex, 200 * U * 0.9 * SR)
        grad = dhin
    assert dx.shape == x.shape and bool(torch.isfinite(dx).all())
    # the update: weights, norms and gates move against their gradients (momentum starts at zero)
    before = [t.clone() for t in (lin.w, st.w_post[0], st.gate[0], st.w_pre[1], st.w_first)]
    st.update()
    after = [lin.w, st.w_post[0], st.gate[0], st.w_pre[1], st.w_first]
    for w0, w1, g in zip(before, after, (st.grads[0][0][0], st.grads[0][0][1], st.grads[0][0][2], st.grads[0][1][3], st.grads[1])):
        assert torch.equal(w1, w0 - st.lr * g)


def test_steps_repeat_bit_for_bit_and_draws_move_on(B):
    import torch
    outs = []
    for _ in range(2):
        st, x, dh = make(130, 256, 3, 0.2, lr=0.01)
        got = []
        for _ in range(3):
            got += [st.forward(x), st.backward(dh)]
            st.update()
        outs.append(got + [l.w for l in st.linears])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    st, x, dh = make(130, 256, 1, 0.5)
    a = st.forward(x); st.step += 1; b = st.forward(x)
    assert not torch.equal(a, b)


@pytest.mark.parametrize("rows", [5, 300])
def test_a_captured_step_replays_on_new_inputs(B, rows):
    """Forward and backward captured once (their workspaces of their own), replayed on other inputs: the eager step's results."""
    import torch
    st, x, dh = make(rows, 384, 2, 0.1)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    sx, sdh = x.clone(), dh.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        st.forward(sx); st.backward(sdh)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        h = st.forward(sx)
        dx = st.backward(sdh)
    params = [t for g in st.grads[0] for t in g] + [st.grads[1]]
    for seed in (1, 2):
        x2, dh2 = real(rng(seed).standard_normal((rows, 384)), "float32")[0], real(rng(seed + 9).standard_normal((rows, 384)), "bfloat16")[0]
        sx.copy_(x2); sdh.copy_(dh2)
        graph.replay()
        got = [t.clone() for t in [h, dx] + params]
        eager, _, _ = make(rows, 384, 2, 0.1)
        want = [eager.forward(x2), eager.backward(dh2)]
        want += [t for g in eager.grads[0] for t in g] + [eager.grads[1]]
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_streams_and_threads_do_not_disturb_one_another(B):
    import torch
    cases = [make(64 + 70 * k, 256, 2, 0.3, seed=k) for k in range(3)]
    want = []
    for st, x, dh in cases:
        want.append([st.forward(x).clone(), st.backward(dh).clone()] + [l.dw.clone() for l in st.linears])
    torch.cuda.synchronize()
    failures = []

    def work(k):
        st, x, dh = cases[k]
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(10):
                got = [st.forward(x), st.backward(dh)] + [l.dw for l in st.linears]
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want[k])): failures.append(k)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(3)]
    [t.start() for t in threads]; [t.join() for t in threads]
    assert not failures


def test_serving_from_kept_codes(B):
    """One token and a ragged batch through a layer whose codes were made once: the training forward's rows, where a row's blocks
    decide about its codes alone."""
    import torch
    from paper_1805_11046_b200 import layer
    w = torch.from_numpy(rng(8).standard_normal((400, 528)).astype(np.float32) * 0.05).cuda()
    x = real(rng(9).standard_normal((300, 528)), "bfloat16")[0]
    L = layer.F8Linear(w)
    y = L.forward(x)
    L.quantise()
    a = codes_are(B, *B.qbp_quantize_f8(x), x, 0, True)
    wv = codes_are(B, L.codes[0], L.codes[1], w, 0, True, square=True)
    for rows in (x[:1], x[7:8], x[:77], x):
        got = L.serve(rows)
        at = x.shape[0] if rows.shape[0] == x.shape[0] else None
        first = 7 if rows.data_ptr() != x.data_ptr() else 0
        check_product(got, a[first:first + rows.shape[0]], wv, 528, "bfloat16")
    assert torch.equal(L.serve(x), y)
    assert L.serve(x.view(3, 100, 528)).shape == (3, 100, 400)
    assert L.serve(x[:0]).shape == (0, 400)


def test_a_captured_serve_outlives_larger_calls_and_new_weights(B):
    """A graph of serve() keeps its workspace when a later call needs a larger one, and answers with the weights as quantised last."""
    import torch
    from paper_1805_11046_b200 import layer
    w = torch.from_numpy(rng(18).standard_normal((256, 384)).astype(np.float32) * 0.05).cuda()
    x = real(rng(19).standard_normal((40, 384)), "bfloat16")[0]
    L = layer.F8Linear(w)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side): L.serve(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = L.serve(x)
    L.serve(real(rng(20).standard_normal((5000, 384)), "bfloat16")[0])
    junk = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (1024, 16384, 17408, 32768, 1 << 16)]     # (whatever was freed)
    for _ in range(2):
        graph.replay()
        assert torch.equal(y, L.serve(x)) and bool(torch.isfinite(y).all())
        w.mul_(-1.5)
        L.quantise()
    assert all(bool((t == 255).all()) for t in junk) and L.status() == 0


def test_a_failed_call_of_a_step_is_not_forgotten(B):
    """Every call of a step has a status word of its own, which a later call does not clear."""
    import torch
    st, x, dh = make(40, 128, 2, 0.1)
    st.forward(x); st.backward(dh)
    assert st.status() == 0
    space = st.space.get()
    for k in range(st.space.words):
        word = space[256 * k:256 * k + 4].view(torch.int32)
        word[0] = -6
        assert st.status() == -6
        if k <= 2: st.backward(dh)                                # (the forward's words)
        assert st.status() == -6
        st.forward(x); st.backward(dh)
        assert st.status() == 0
    lin = st.linears[0]
    for k in range(3):
        lin.space.at(k)[:4].view(torch.int32)[0] = -6
        assert st.status() == -6
        st.forward(x); st.backward(dh)
        assert st.status() == 0


def test_empty_and_tiny_extents(B):
    import torch
    q, s = B.qbp_quantize_f8(torch.randn(32, 64, device="cuda"))
    none, ns = B.qbp_quantize_f8(torch.randn(0, 64, device="cuda"))
    assert none.shape == (0, 64) and ns.numel() == 0
    assert B.qbp_gemm_f8(none, ns, q, s, transB=True).shape == (0, 32)
    # a weight gradient over no rows is zero, over one row an outer product
    _, _, gt, gs = B.qbp_quantize_f8(torch.randn(0, 64, device="cuda"), cols=True)
    dw = B.qbp_gemm_f8(gt, gs, gt, gs, transA=True)
    assert dw.shape == (64, 64) and not dw.any()
    x = torch.randn(1, 64, device="cuda")
    _, _, xt, xs = B.qbp_quantize_f8(x, cols=True)
    v = F.values(host(xt), 0, F.spread(host(B.qbp_f8_exponents(xs, 64, 1)), 1).T)
    assert np.array_equal(host(B.qbp_gemm_f8(xt, xs, xt, xs, transA=True)), (v.T @ v).astype(np.float32))
    e = torch.empty(0, 96, device="cuda")
    d = B.resnorm_desc(e, e)
    g = torch.ones(96, device="cuda")
    ws = torch.full((512,), 255, dtype=torch.uint8, device="cuda")
    r, h, q1, q2 = B.qbp_resnorm_fwd(d, e, e, g, g, g, ws=ws)
    assert B.status_word(ws) == 0                                 # (cleared where there is nothing to do, too)
    dx, db, dw1, dg, dw2 = B.qbp_resnorm_bwd(d, e, e, e, r, q1, q2, g, g, g)
    assert h.shape == (0, 96) and not dw1.any() and not dg.any() and not dw2.any()
    assert B.qbp_dropout(e, 0.5, 1).shape == (0, 96)
