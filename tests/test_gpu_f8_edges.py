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
