"""8-bit floating-point codes, products and layers at the edges of what their definitions allow."""
import numpy as np
import pytest

from oracle import f8_oracle as F
from tests.test_gpu_f8 import host, rng

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import paper_1805_11046_b200.binding as binding
    return binding


@pytest.mark.parametrize("shape", [(3, 0), (2, 3, 0), (2, 1, 5, 0), (0,)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_a_layer_of_no_inputs_puts_out_zeros(B, shape, dtype):
    """A sum of nothing, for activations of any number of dimensions."""
    import torch
    x = torch.empty(shape, dtype=getattr(torch, dtype), device="cuda")
    w, sw = torch.empty((48, 0), dtype=torch.uint8, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda")
    y = torch.full((*shape[:-1], 48), 7.0, dtype=x.dtype, device="cuda")
    assert B.qbp_linear_f8(x, w, sw, y=y) is y and not y.any()


@pytest.mark.parametrize("rows", [(5, 3), (64, 100), (1000, 777)])
def test_one_layer_serves_on_several_streams_and_threads(B, rows):
    """Calls of one layer in turn on two streams and from two threads on each, with activations of their own: the results of one at a time."""
    import threading

    import torch
    from paper_1805_11046_b200 import layer
    N, K = 1024, 4096
    L = layer.F8Linear(torch.from_numpy(rng(1).standard_normal((N, K)).astype(np.float32)).cuda())
    L.quantise()
    cases = [[torch.from_numpy(rng(10 * k + j).standard_normal((m, K)).astype(np.float32)).cuda() for j, m in enumerate(rows)] for k in range(4)]
    want = [[B.qbp_linear_f8(x, L.codes[0], L.codes[1]) for x in c] for c in cases]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[] for _ in cases]

    def work(k):
        with torch.cuda.stream(streams[k % 2]):
            for _ in range(15): got[k].append([L.serve(x) for x in cases[k]])

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    [t.start() for t in threads]; [t.join() for t in threads]
    for _ in range(15):                                           # one thread, two streams in turn
        for k in range(2):
            with torch.cuda.stream(streams[k]): got[k].append([L.serve(x) for x in cases[k]])
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for g, ws in zip(got, want) for ys in g for y, w in zip(ys, ws))
    assert L.status() == 0


def test_graphs_of_one_layer_replay_at_the_same_time(B):
    """Captured serve() calls with a workspace each, replayed on two streams; one captured without any call before it."""
    import torch
    from paper_1805_11046_b200 import layer
    N, K, M = 512, 2048, 90
    L = layer.F8Linear(torch.from_numpy(rng(2).standard_normal((N, K)).astype(np.float32)).cuda())
    L.quantise()
    xs = [torch.from_numpy(rng(5 + k).standard_normal((M, K)).astype(np.float32)).cuda().to(torch.bfloat16) for k in range(2)]
    want = [B.qbp_linear_f8(x, L.codes[0], L.codes[1]) for x in xs]
    torch.cuda.synchronize()
    graphs, ys, wss, streams = [], [], [], [torch.cuda.Stream() for _ in range(2)]
    for x in xs:
        g = torch.cuda.CUDAGraph()
        wss.append(torch.zeros(B.qbp_linear_f8_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda"))
        with torch.cuda.graph(g): ys.append(L.serve(x, ws=wss[-1]))
        graphs.append(g)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g): y = L.serve(xs[0])                  # (its workspace is first asked for here)
    assert L.status() == 0
    for _ in range(20):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s): graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ys, want))
        [t.zero_() for t in ys]
        torch.cuda.synchronize()
    assert all(B.status_word(ws) == 0 for ws in wss)
    g.replay()
    assert torch.equal(y, want[0]) and L.status() == 0


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("bad", [np.nan, -np.nan, np.inf, -np.inf])
def test_blocks_that_are_not_finite_in_every_type_and_direction(B, dtype, bad):
    """One such element in a first, a middle and a ragged last block: NaN codes and scales there, all other codes and scales as ever; products
    and layers of few and of many rows answer NaN where these blocks enter and nowhere else."""
    import torch
    rows, cols, N = 300, 400, 48
    v = rng(6).standard_normal((rows, cols)).astype(np.float32)
    at = [(0, 0), (130, 200), (299, 399)]
    x = torch.from_numpy(v).to(getattr(torch, dtype)).cuda()
    for i, j in at: x[i, j] = bad
    d = x.double().cpu().numpy()
    qr, sr, qc, sc = B.qbp_quantize_f8(x, cols=True)
    for q, s, got in ((*F.quantize(d, 0, 1, 128), (qr, sr)), (*[t for t in F.quantize(d, 0, 128, 1)], (qc, sc))):
        across = got[0] is qc
        assert np.array_equal(host(got[0]), q) and np.array_equal(host(got[1]), F.pack(s.T if across else s, cols if across else rows))
        assert (s == 128).sum() == 3
    q, s1, s2 = B.qbp_quantize_f8_square(x)
    wq, we = F.quantize(d, 0, 128, 128)
    assert (we == 128).sum() == 3 and np.array_equal(host(q), wq)
    assert np.array_equal(host(s1), F.pack(F.spread(we, rows, 0), rows)) and np.array_equal(host(s2), F.pack(F.spread(we.T, cols, 0), cols))
    w, sw, _ = B.qbp_quantize_f8_square(torch.from_numpy(rng(7).standard_normal((N, cols)).astype(np.float32)).cuda())
    want = np.zeros((rows, N), bool)
    want[[i for i, _ in at]] = True
    for some in (slice(0, 300), slice(128, 133), slice(299, 300), slice(290, 300)):
        y = B.qbp_linear_f8(x[some], w, sw)
        assert np.array_equal(np.isnan(host(y.float())), want[some]) and bool(torch.isfinite(y[~torch.isnan(y)]).all())
    # as weights, one scale for 128 x 128: the columns of the outputs whose blocks hold one of them
    z = B.qbp_gemm_f8(w, sw, q, s1, transB=True)
    assert np.array_equal(np.isnan(host(z)).all(0), F.spread((we == 128).any(1)[None], rows)[0]) and np.array_equal(np.isnan(host(z)).any(0), np.isnan(host(z)).all(0))


@pytest.mark.parametrize("fmt", [0, 1])
def test_weights_quantised_into_storage_made_before(B, fmt):
    """Codes and scales written over storage that qbp_f8_scales sized, whatever it held."""
    import torch
    rows, cols = 210, 144
    x = torch.from_numpy(rng(8).standard_normal((rows, cols)).astype(np.float32)).cuda()
    out = torch.full((rows, cols), 255, dtype=torch.uint8, device="cuda"), B.qbp_f8_scales(rows, cols).fill_(3), B.qbp_f8_scales(cols, rows).fill_(3)
    got = B.qbp_quantize_f8_square(x, format=fmt, out=out)
    assert all(a is b for a, b in zip(got, out)) and all(torch.equal(a, b) for a, b in zip(got, B.qbp_quantize_f8_square(x, format=fmt)))
