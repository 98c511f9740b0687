"""Gradients of groups whose row numbers do not fit in LDS at once (more than 2,048 rows of a chunk), for every tile and way of reading rows, and
calls on two streams at once on the largest tiles.  Integers whose sums stay below 2^24: float64 gives the results bit for bit."""
import ctypes

import numpy as np
import pytest
import torch

from tests.test_gpu_grouped import BF16, F32, _grouping, _keys, _values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lq():
    import paper_2306_08367_amd as lq
    return lq


def _want(X, dY, off, order, slots=1):
    """(dW, db) in float64 on the GPU."""
    X, dY, r = X.cuda().double(), dY.cuda().double(), torch.from_numpy(order.astype(np.int64)).cuda()
    G = len(off) - 1
    dW, db = torch.zeros((G, X.shape[1], dY.shape[1]), dtype=torch.float64, device="cuda"), torch.zeros((G, dY.shape[1]), dtype=torch.float64, device="cuda")
    for g in range(G):
        at = r[off[g]:off[g + 1]]
        dW[g], db[g] = X[torch.div(at, slots, rounding_mode="floor")].T.contiguous() @ dY[at], dY[at].sum(0)
    return dW, db


# sizes of groups: around one, two and three times the rows whose numbers LDS holds, none and one
ROWS = [2047, 0, 2048, 2049, 1, 4096, 4097, 6200]


@pytest.mark.parametrize("dtype,k,l", [(F32, 48, 40), (F32, 132, 136), (F32, 49, 35), (F32, 131, 133), (BF16, 64, 56), (BF16, 128, 136), (BF16, 62, 50),
                                       (BF16, 130, 134), (BF16, 33, 45), (BF16, 129, 131), (BF16, 7, 70), (BF16, 264, 256)])
@pytest.mark.parametrize("slots", [1, 2])
def test_whole_groups_without_a_workspace(lq, dtype, k, l, slots):
    """The C entry point without a workspace: each group is one chunk."""
    from paper_2306_08367_amd import binding as B
    rng = np.random.default_rng(k + l)
    n = (sum(ROWS) + 37) // 2 * 2
    keys = rng.permutation(np.concatenate([np.full(c, g) for g, c in enumerate(ROWS)] + [np.full(n - sum(ROWS), -1)]))
    off, order = _grouping(keys, len(ROWS))
    X, dY = _values(rng, (n // slots, k), dtype, True), _values(rng, (n, l), dtype, True)
    want, want_b = _want(X, dY, off, order, slots)
    X, dY, o, r = X.cuda(), dY.cuda(), torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda()
    dW, db = torch.full(want.shape, float("nan"), device="cuda"), torch.full(want_b.shape, float("nan"), device="cuda")
    groups, stack = B.lq_groups(n, len(ROWS), o.data_ptr(), r.data_ptr()), B.lq_stack(dW.data_ptr(), len(ROWS), k, l, 0, l, k * l)
    rc = B._lib.lq_grouped_gradient(ctypes.byref(groups), ctypes.byref(B._mat(X)), slots, ctypes.byref(B._mat(dY)), ctypes.byref(stack),
                                    ctypes.byref(B._mat(db)), None, 0, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(dW.double(), want) and torch.equal(db.double(), want_b)
    # chunks and their partial sums give the same (integers)
    dW, db = lq.lq_grouped_gradient(X, dY, o, r, dw_dtype=F32, want_bias=True, x_slots=slots)
    assert torch.equal(dW.double(), want) and torch.equal(db.double(), want_b)


@pytest.mark.parametrize("dtype,k,l", [(F32, 1024, 1024), (F32, 1022, 1021), (BF16, 1024, 1024), (BF16, 1022, 1026), (BF16, 1023, 1025)])
def test_chunks_of_several_thousand_rows(lq, dtype, k, l):
    """Wide matrices and many rows: a workgroup's share is 4,096 rows and more."""
    rng = np.random.default_rng(k)
    n = 32_768 + 100
    off, order = _grouping(np.where(np.arange(n) % 331 == 5, -1, 0), 1)
    X, dY = _values(rng, (n, k), dtype, True), _values(rng, (n, l), dtype, True)
    want, want_b = _want(X, dY, off, order)
    dW, db = lq.lq_grouped_gradient(X.cuda(), dY.cuda(), torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda(), dw_dtype=F32, want_bias=True)
    assert torch.equal(dW.double(), want) and torch.equal(db.double(), want_b)


def test_two_gradients_at_once_on_the_largest_tiles(lq):
    """Tiles of 256 x 256, with partial sums and the launch that adds them up."""
    rng = np.random.default_rng(5)
    n, G, k, l = 12_289, 4, 264, 512
    off, order = (torch.from_numpy(t).cuda() for t in _grouping(_keys(rng, n, G, "ragged"), G))
    X, dY = _values(rng, (n, k), BF16, False).cuda(), _values(rng, (n, l), BF16, False).cuda()
    assert lq.lq_grouped_gradient_workspace_bytes(n, G, k, l, 1) > 0
    call = lambda s: lq.lq_grouped_gradient(X, dY, off, order, dw_dtype=F32, want_bias=True, stream=s)
    want = call(None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [call(s) for s in streams]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
