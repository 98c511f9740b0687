"""Columns that are not one run of memory are refused, however many dimensions their view has: an [n x 1] piece of a wider tensor would else
be read as if it were contiguous, its neighbours' values for its own."""
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lq():
    if not os.path.exists(os.path.join(ROOT, "paper_2306_08367_amd", "liblq.so")):
        pytest.skip("liblq.so not built")
    import paper_2306_08367_amd as lq
    return lq


def _views(column):
    """The column as every other element, as [n x 1] of a wider tensor, and as [n x 2] (whose first entries are not the column)."""
    wide = torch.stack([column, torch.full_like(column, 1 << 30)], 1)
    return wide[:, 0], wide[:, :1], wide


def test_host_refusals(lq):
    """Said before a GPU is asked for."""
    for keys in _views(torch.arange(6, dtype=torch.int32))[:2]:
        with pytest.raises(ValueError, match="keys must be contiguous"):
            lq.lq_group_rows(keys, 3)
        with pytest.raises(ValueError, match="key column must be contiguous"):
            lq.lq_keymap_build(keys)


@pytest.mark.gpu
def test_groups(lq):
    X, W = torch.ones((4, 8), device="cuda"), torch.ones((2, 8, 8), device="cuda")
    A, B, W0 = torch.ones((2, 8, 2), device="cuda"), torch.ones((2, 2, 8), device="cuda"), torch.ones((8, 8), device="cuda")
    off, order = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda"), torch.tensor([3, 1, 0, 2], dtype=torch.int32, device="cuda")
    calls = [lambda o, r: lq.lq_grouped_product(X, W, o, r), lambda o, r: lq.lq_grouped_gradient(X, X, o, r)[0],
             lambda o, r: lq.lq_adapter_product(X, W0, A, B, o, r)]
    for call in calls:
        want = call(off, order)
        for o in _views(off):
            with pytest.raises(ValueError, match="offsets must"):
                call(o, order)
        for r in _views(order):
            with pytest.raises(ValueError, match="order must"):
                call(off, r)
        assert torch.equal(call(off[:, None].contiguous(), order[:, None].contiguous()), want)     # (one run of memory)
        scale = torch.ones((2, 2), device="cuda")[:, 0]
        with pytest.raises(ValueError, match="scale must be contiguous"):
            lq.lq_adapter_product(X, W0, A, B, off, order, scale=scale)
