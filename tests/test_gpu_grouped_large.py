"""The grouped operators where their largest tiles (256 x 256, eight wavefronts) run: many rows, wide results.  Integers, so that
results are exact (see test_gpu_grouped.py)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_grouped import BF16, F32, _check, _grouping, _keys, _product, _run_adapter, _run_gradient, _strided, _values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lq():
    import paper_2306_08367_amd as lq
    return lq


N, WIDE = 12_289, 2048      # 49 x 8 tiles of 256 x 256 and a part of one more for every group: they fill the compute units


@pytest.mark.parametrize("transposed", [False, True], ids=["forward", "transposed"])
@pytest.mark.parametrize("inner,how,out,extra", [(96, "ragged", BF16, 0), (32, "even", F32, 8), (8, "one", BF16, 1), (200, "ragged", F32, 3), (40, "none", BF16, 0)])
def test_product(lq, transposed, inner, how, out, extra):
    rng = np.random.default_rng(inner)
    G, wide = 5, WIDE - 8 * (inner % 3)
    off, order = _grouping(_keys(rng, N, G, how), G)
    X, W = _values(rng, (N, inner), BF16, True), _values(rng, (G, wide, inner) if transposed else (G, inner, wide), BF16, True)
    b = None if transposed else _values(rng, (G, wide), BF16, True)
    h = _values(rng, (N, wide), BF16, True) if transposed else None
    want, _ = _product(X, W, off, order, b, h, transposed, not transposed, False, True, 1)
    buf, Y = _strided(torch.zeros((N, wide), dtype=out), 0, extra, fill=7.0)
    lq.lq_grouped_product(X.cuda(), W.cuda(), torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda(), bias=None if b is None else b.cuda(),
                          gate=None if h is None else h.cuda(), Y=Y, transposed=transposed, relu=not transposed, y_grouped=True)
    assert torch.equal(Y.cpu(), want.float().to(out))
    Y.fill_(7.0)
    assert bool((buf == 7.0).all()), "written outside the result"


def test_rows_of_several_groups(lq):
    rng = np.random.default_rng(2)
    G, n, slots, k = 6, 6_200, 2, 64
    off, order = _grouping(_keys(rng, n * slots, G, "ragged"), G)
    X, W = _values(rng, (n, k), BF16, True), _values(rng, (G, k, WIDE), BF16, True)
    want, _ = _product(X, W, off, order, None, None, False, False, False, False, slots)
    got = lq.lq_grouped_product(X.cuda(), W.cuda(), torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda(), x_slots=slots)
    assert torch.equal(got.cpu(), want.float().to(BF16))


@pytest.mark.parametrize("n,G,k,l,slots", [(5000, 4, 256, 512, 1), (3000, 3, 264, 1016, 2), (100, 9, 512, 256, 1), (9001, 70, 208, 200, 1)])
@pytest.mark.parametrize("how", ["ragged", "even", "one"])
def test_gradient(lq, n, G, k, l, slots, how):
    _run_gradient(lq, n, G, k, l, BF16, how=how, out=F32, integers=True, slots=slots)
    _run_gradient(lq, n, G, k, l, BF16, how=how, integers=True, slots=1, extra=8, y_grouped=True, seed=1)


def test_gradient_without_a_workspace_adds_up_whole_groups(lq):
    """The C entry point takes no workspace as well: the same sums (of integers), from one workgroup a tile."""
    from paper_2306_08367_amd import binding as B
    import ctypes
    rng = np.random.default_rng(3)
    n, G, k, l = 7000, 3, 256, 320
    off, order = _grouping(_keys(rng, n, G, "ragged"), G)
    X, dY = (_values(rng, s, BF16, True).cuda() for s in ((n, k), (n, l)))
    o, r = torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda()
    want, want_b = lq.lq_grouped_gradient(X, dY, o, r, dw_dtype=F32, want_bias=True)
    dW, db = torch.empty_like(want), torch.empty_like(want_b)
    groups, stack = B.lq_groups(n, G, o.data_ptr(), r.data_ptr()), B.lq_stack(dW.data_ptr(), G, k, l, 0, l, k * l)
    rc = B._lib.lq_grouped_gradient(ctypes.byref(groups), ctypes.byref(B._mat(X)), 1, ctypes.byref(B._mat(dY)), ctypes.byref(stack), ctypes.byref(B._mat(db)),
                                    None, 0, 0, torch.cuda.current_stream().cuda_stream)
    assert rc == 0 and torch.equal(dW, want) and torch.equal(db, want_b)


@pytest.mark.parametrize("G,runs,how,rank", [(3, 900, "even", 32), (40, 50, "ragged", 8), (400, 2, "ragged", 5), (5, 1, "none", 16)])
def test_adapter(lq, G, runs, how, rank):
    _run_adapter(lq, N, G, 64, WIDE, rank, BF16, how=how, integers=True, runs=runs)
    _run_adapter(lq, N, G, 72, WIDE, rank, BF16, how=how, integers=True, runs=runs, out=F32, extra=8, bias=False, seed=1)


def test_an_adapter_of_other_rows_does_not_reach_a_row(lq):
    rng = np.random.default_rng(1)
    G, k, rank = 4, 32, 8
    keys = np.arange(N) // 100 % (G + 1) - 1
    off, order = (torch.from_numpy(t).cuda() for t in _grouping(keys, G))
    X, W, A, B = (_values(rng, s, BF16, True).cuda() for s in ((N, k), (k, WIDE), (G, k, rank), (G, rank, WIDE)))
    before = lq.lq_adapter_product(X, W, A, B, off, order)
    A[1] = float("nan")
    B[2] = float("inf")
    after = lq.lq_adapter_product(X, W, A, B, off, order)
    other = torch.from_numpy((keys != 1) & (keys != 2)).cuda()
    assert torch.equal(before[other], after[other]) and bool(torch.isnan(after[torch.from_numpy(keys == 1).cuda()]).all())


def test_values_within_the_bounds(lq):
    """Normal values over a long inner dimension: the tolerances of test_gpu_grouped.py."""
    rng = np.random.default_rng(4)
    G, k, n = 3, 1000, 12_400
    off, order = _grouping(_keys(rng, n, G, "ragged"), G)
    X, W = _values(rng, (n, k), BF16, False), _values(rng, (G, k, WIDE), BF16, False)
    got = lq.lq_grouped_product(X.cuda(), W.cuda(), torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda(), y_dtype=F32)
    some = rng.integers(0, n, 300)
    keys = np.zeros(n, dtype=np.int64) - 1
    for g in range(G):
        keys[order[off[g]:off[g + 1]]] = g
    want = torch.stack([X[i].double() @ W[keys[i]].double() if keys[i] >= 0 else torch.zeros(WIDE, dtype=torch.float64) for i in some])
    size = torch.stack([X[i].double().abs() @ W[keys[i]].double().abs() if keys[i] >= 0 else torch.zeros(WIDE, dtype=torch.float64) for i in some])
    _check(got.cpu()[some], want, k, size, F32, False, "long rows")


def test_two_calls_at_once_on_the_largest_tiles(lq):
    rng = np.random.default_rng(5)
    G, k = 4, 128
    off, order = (torch.from_numpy(t).cuda() for t in _grouping(_keys(rng, N, G, "ragged"), G))
    X, W = _values(rng, (N, k), BF16, False).cuda(), _values(rng, (G, k, WIDE), BF16, False).cuda()
    call = lambda s: (lq.lq_grouped_product(X, W, off, order, stream=s), lq.lq_grouped_gradient(X, X, off, order, stream=s)[0])
    want = call(None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [call(s) for s in streams]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))
