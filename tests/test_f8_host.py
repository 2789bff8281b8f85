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
