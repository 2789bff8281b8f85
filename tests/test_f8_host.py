"""What the host does around the 8-bit floating-point layers: shapes, workspaces, imports (runs without a GPU)."""
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_1805_11046_b200 import build
    build.build_library()
    from paper_1805_11046_b200 import binding
    return binding


def test_rows_without_columns_are_rows(B):
    import torch
    for shape, rows in (((3, 0), 3), ((2, 3, 0), 6), ((2, 0, 0), 0), ((0,), 1), ((4, 0, 16), 0), ((2, 3, 16), 6)):
        assert B._rows_of(torch.empty(shape)) == (rows, shape[-1], shape[-1])


def test_serving_from_several_streams_and_threads_shares_no_scratch(B, monkeypatch):
    """Calls that may run at the same time quantise their activations into workspaces of their own; those of one stream and thread keep theirs."""
    import threading

    import torch
    from paper_1805_11046_b200 import layer
    now, used = {"stream": 7}, []
    monkeypatch.setattr(B, "_stream_handle", lambda device: now["stream"])
    monkeypatch.setattr(B, "qbp_linear_f8", lambda x, q, s, ws: used.append((ws.data_ptr(), ws.numel(), ws)))
    L = layer.F8Linear(torch.zeros(32, 64))
    L.codes = torch.zeros(32, 64, dtype=torch.uint8), None, None
    x, more = torch.zeros(100, 64), torch.zeros(4000, 64)
    L.serve(x)
    now["stream"] = 9
    L.serve(x)
    t = threading.Thread(target=lambda: L.serve(x))
    t.start(); t.join()
    spans = sorted((a, a + n) for a, n, _ in used)
    assert all(end <= start for (_, end), (start, _) in zip(spans, spans[1:]))
    assert all(n >= B.qbp_linear_f8_workspace_bytes(100, 32, 64) for _, n, _ in used)
    L.serve(x)
    assert used[-1][0] == used[1][0]                        # this stream's again
    L.serve(more)
    assert used[-1][1] >= B.qbp_linear_f8_workspace_bytes(4000, 32, 64)
    own = torch.zeros(1 << 20, dtype=torch.uint8)
    L.serve(x, ws=own)
    assert used[-1][2] is own
    # a failed call of any of them is not forgotten, nor one of a training step's
    for ws in (used[0][2], used[2][2], L.space.at(1)):
        assert L.status() == 0
        ws[:4].view(torch.int32)[0] = -6
        assert L.status() == -6
        ws[:4] = 0


def test_the_binding_imports_on_a_torch_without_cuda(B):
    """Such a torch has no raw lookups of the current device and stream; the module's own are looked up with something to fall back on."""
    import subprocess
    import sys
    from pathlib import Path
    code = ("import torch\n"
            "for name in ('_cuda_getDevice', '_cuda_getCurrentRawStream'):\n"
            "    if hasattr(torch._C, name): delattr(torch._C, name)\n"
            "from paper_1805_11046_b200 import binding, layer\n"
            "assert binding._current_device is torch.cuda.current_device and binding._raw_stream is None\n")
    got = subprocess.run([sys.executable, "-c", code], cwd=Path(__file__).resolve().parent.parent, capture_output=True, text=True)
    assert got.returncode == 0, got.stderr


def test_blocks_that_share_weights_are_refused(B):
    """Their update would be two writers of the same memory."""
    import torch
    from paper_1805_11046_b200 import layer
    w = [torch.zeros(16, 16) for _ in range(3)]
    assert len(layer.F8ResidualStack(w).linears) == 3
    both = torch.zeros(31, 16)
    for weights in ([w[0], w[1], w[0]], [both[:16], both[15:]]):
        with pytest.raises(ValueError, match="share memory"):
            layer.F8ResidualStack(weights)
    assert len(layer.F8ResidualStack([both[:15], both[15:30]]).linears) == 2


def test_extents_that_the_grids_cannot_have(B):
    """Refused on the host, up to the ends of 64 bits; the largest ones pass these checks and fail a later one here."""
    P, most = 4096, (1 << 63) - 1
    rows, wide = 128 * 65535, 1 << 30
    for r, c in ((rows + 1, 16), (most, 16), (most - 126, 32), (1 << 40, 16), (1, wide + 16), (16, most - 15)):
        assert B.lib.qbp_quantize_f8(P, 0, r, c, c, 0, P, P, P, P, None) == -2, (r, c)
        assert B.lib.qbp_quantize_f8_square(P, 0, r, c, c, 0, P, P, P, None) == -2, (r, c)
        assert B.lib.qbp_linear_f8(P, 0, c, r, 16, c, 0, P, P, P, P, most, None) == -2, (r, c)
    assert B.lib.qbp_quantize_f8(P, 0, rows, wide, wide, 0, None, None, None, None, None) == -1      # (no output)
    for M, N, K in ((rows + 1, 16, 16), (most, 16, 16), (16, wide + 1, 16), (16, most, 16), (16, 16, wide + 16), (16, 16, most - 15)):
        assert B.lib.qbp_gemm_f8(0, 1, M, N, K, 0, P, P, 0, P, P, 0, P, P, most, None) == -2, (M, N, K)
    assert B.lib.qbp_gemm_f8(0, 1, rows, wide, wide, 0, P, P, 0, P, P, 0, None, P, most, None) == -1
