"""CPU: sizes that the grouped calls work out for the largest arguments that they take."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2306_08367_amd", "liblq.so")), reason="liblq.so not built")


@pytest.fixture(scope="module")
def b():
    from paper_2306_08367_amd import binding
    return binding


@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
def test_a_gradient_with_more_tiles_than_workgroups_needs_no_partial_sums(b, dtype):
    """Where one tile of a matrix keeps every compute unit busy over all rows, groups are whole: the number of rows of a chunk stays one of 32
    bits, and the product of rows and tiles one of 64."""
    most = 1 << 30
    for n, k, l in [(most, most, most), (1 << 25, 1 << 20, 1024), (most, 1 << 20, 1 << 20), (1, most, most), (0, most, most)]:
        assert b.lq_grouped_gradient_workspace_bytes(n, b.LQ_MAX_MODELS, k, l, dtype) == 0, (n, k, l)
    # (shared out as before: 32,768 rows over 32 tiles of 256 x 256, 8 chunks and less than one more a group)
    assert b.lq_grouped_gradient_workspace_bytes(32_768, 16, 2048, 1024, 1) == 16 * 2049 * 1024 * 4


@pytest.mark.parametrize("n,rank", [(1 << 30, 256), (1 << 28, 256), (1 << 30, 33)])
def test_an_adapter_product_of_too_many_ranks_is_refused(b, n, rank):
    """A thread scales eight ranks of a row, and a launch has fewer than 2^32 threads.  Refused before anything is enqueued."""
    import ctypes
    at = 0x10000
    mat = lambda rows, cols: ctypes.byref(b.lq_mat(at, rows, cols, cols, 0))
    groups, A, B = b.lq_groups(n, 2, at, None), b.lq_stack(at, 2, 1, rank, 0, rank, rank), b.lq_stack(at, 2, rank, 1, 0, 1, rank)
    rc = b._lib.lq_adapter_product(ctypes.byref(groups), mat(n, 1), mat(1, 1), None, ctypes.byref(A), ctypes.byref(B), None, mat(n, 1), at, 1 << 50, 0, None)
    assert rc == 6 and f"{n} rows of rank {rank}" in b.lq_last_error(), (rc, b.lq_last_error())


@pytest.mark.parametrize("keys,offsets,order", [(0, 0x1000, 0), (0, 0x1000, 36), (36, 0x1000, 0), (0, 36, 0x1000), (16, 0, 0x1000), (0x1000, 0, 16), (0x1000, 36, 0)])
def test_rows_of_groups_in_place_are_refused(b, keys, offsets, order):
    """10 keys, 4 groups: order or offsets over the keys, which are read while these are written, or over each other (bytes from one base)."""
    at = 0x100000
    rc = b._lib.lq_group_rows(at + keys, 10, 4, at + offsets, at + order, None, 0, 0, None)
    assert rc == 2 and "overlap" in b.lq_last_error(), (rc, b.lq_last_error())
