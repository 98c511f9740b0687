"""Infinities and NaNs of lq_adapter_product: the same as those of the formula, Y = X W + b + scale_g U B_g with U = X A_g as ONE number, whatever
the tile, the copies and the number of rows.  All finite values are integers whose sums stay below 2^24, and U stays below 2^16 (beside
bf16 matrices it is held in two bf16 numbers: 16 bits), so that float64 gives the results bit for bit."""
import numpy as np
import pytest
import torch

from tests.test_gpu_grouped import BF16, F32, _grouping, _strided, _values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lq():
    import paper_2306_08367_amd as lq
    return lq


INF, NAN = float("inf"), float("nan")

# rows, columns: few rows (a kernel of their own), then tiles of 64 with steps ahead, 64, 128 and 256 (the last one: bf16, 16-byte rows)
SIZES = [(100, 48), (2000, 1024), (3000, 1024), (6000, 1024), (12_289, 2048)]


def _inputs(rng, n, k, l, rank, dtype, G):
    X, W, A, B, b = (_values(rng, s, dtype, True) for s in ((n, k), (k, l), (G, k, rank), (G, rank, l), (l,)))
    A = torch.where(torch.from_numpy(rng.random(A.shape) < 6.0 / k), A, 0)
    scale = torch.from_numpy(rng.choice([1.0, 171.0, 511.0], G).astype(np.float32))     # (most U are no bf16 numbers)
    return X, W, A, B, b, scale


def _want(X, W, A, B, b, scale, off, order):
    Y = X.double() @ W.double() + b.double()
    for g in range(A.shape[0]):
        r = torch.from_numpy(order[off[g]:off[g + 1]].astype(np.int64))
        # (term by term: a product of matrices may leave out zeros)
        u = scale[g].double() * (X[r].double()[:, :, None] * A[g].double()[None]).sum(1)
        for j in range(u.shape[1]):
            Y[r] += u[:, j, None] * B[g, j].double()
    return Y


def _same(got, want, dtype):
    got, want = got.cpu(), want.to(torch.float32).to(dtype)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), f"{int((torch.isnan(got) != nan).sum())} of {nan.numel()} are NaN and should not be, or the reverse"
    assert torch.equal(got[~nan], want[~nan])


@pytest.mark.parametrize("dtype,k", [(F32, 32), (F32, 33), (BF16, 32), (BF16, 34), (BF16, 33)], ids=["f32-16", "f32-4", "bf16-16", "bf16-4", "bf16-2"])
@pytest.mark.parametrize("n,l", SIZES)
@pytest.mark.parametrize("out", [F32, BF16], ids=["to-f32", "to-bf16"])
def test_special_values_are_those_of_the_formula(lq, n, l, dtype, k, out):
    if dtype == F32 and out == BF16:
        out, l = F32, l - 3                          # (fp32: results of an odd width instead)
    rng = np.random.default_rng(n + k)
    G, rank = 7, 11
    keys = np.arange(n) // 3 % (G + 1) - 1           # three rows an adapter, and three without one, side by side in the call's order
    keys = keys if n % 2 else np.sort(keys)          # or in long runs
    off, order = _grouping(keys, G)
    X, W, A, B, b, scale = _inputs(rng, n, k, l, rank, dtype, G)
    B[1, 2, ::5] = INF
    B[1, 9, 3::10] = -INF
    B[2, 0, 1] = -INF
    B[2, 10, l - 1] = INF
    B[3, 1, 7] = NAN
    A[4, 5, 3] = INF
    X[n // 2, 1] = NAN
    X[n // 3, 2] = -INF
    W[6, 9] = INF
    want = _want(X, W, A, B, b, scale, off, order)
    assert bool(torch.isinf(want[keys == 1][:, ::5]).any()) and bool(torch.isnan(want).any()) and bool(torch.isfinite(want[keys == 5][:, 10:]).any())
    got = lq.lq_adapter_product(*(t.cuda() for t in (X, W, A, B)), torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda(), scale=scale.cuda(),
                                bias=b.cuda(), y_dtype=out)
    _same(got, want, out)


@pytest.mark.parametrize("n,l", SIZES)
def test_special_values_into_rows_with_gaps(lq, n, l):
    """Y whose rows lie apart and are not aligned: what lies between stays."""
    rng = np.random.default_rng(n)
    G, rank, k = 5, 8, 32
    keys = np.arange(n) // 40 % (G + 1) - 1
    off, order = _grouping(keys, G)
    X, W, A, B, b, scale = _inputs(rng, n, k, l, rank, BF16, G)
    B[1, 2, ::3] = INF
    B[3, :, l // 2] = -INF
    buf, Y = _strided(torch.zeros((n, l), dtype=F32), 0, 3, fill=7.0, offset=1)
    lq.lq_adapter_product(*(t.cuda() for t in (X, W, A, B)), torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda(), scale=scale.cuda(), bias=b.cuda(), Y=Y)
    _same(Y, _want(X, W, A, B, b, scale, off, order), F32)
    Y.fill_(7.0)
    assert bool((buf == 7.0).all()), "written outside the result"


@pytest.mark.parametrize("n,l", SIZES)
def test_rows_beside_a_special_value_keep_their_bits(lq, n, l):
    """Normal values: rows of other adapters, and finite results of the adapter's own rows, are as they are without the infinity."""
    rng = np.random.default_rng(n + 1)
    G, k, rank = 6, 48, 8
    keys = np.arange(n) % (G + 1) - 1
    off, order = (torch.from_numpy(t).cuda() for t in _grouping(keys, G))
    X, W, A, B = (_values(rng, s, BF16, False).cuda() for s in ((n, k), (k, l), (G, k, rank), (G, rank, l)))
    before = lq.lq_adapter_product(X, W, A, B, off, order, y_dtype=F32)
    B[2, 3, 5] = INF
    B[4, 1, l - 1] = NAN
    after = lq.lq_adapter_product(X, W, A, B, off, order, y_dtype=F32)
    keys, touched = torch.from_numpy(keys).cuda(), torch.zeros((n, l), dtype=torch.bool, device="cuda")
    touched[keys == 2, 5] = True
    touched[keys == 4, l - 1] = True
    assert torch.equal(before[~touched], after[~touched])
    assert bool(torch.isinf(after[keys == 2, 5]).all()) and bool(torch.isnan(after[keys == 4, l - 1]).all())


@pytest.mark.parametrize("n,l", SIZES)
def test_a_factor_above_the_largest_bf16_number_stays_finite(lq, n, l):
    """U = +-3.4e38 in fp32.  Tolerance: 2^-16 of U beside bf16 matrices, and a rounding for each of the k + 5 terms at most."""
    rng = np.random.default_rng(n)
    G, k, rank = 3, 16, 2
    keys = np.arange(n) % (G + 1) - 1
    off, order = _grouping(keys, G)
    X, W = _values(rng, (n, k), BF16, True), _values(rng, (k, l), BF16, True)
    X[:, 0] = torch.from_numpy(rng.choice([-1.0, 1.0], n)).to(BF16)
    A = torch.zeros((G, k, rank), dtype=BF16)
    A[:, 0, 0] = 1.0
    B = torch.from_numpy(rng.choice([0.0, 2.0 ** -100, 2.0 ** -120, -2.0 ** -2], (G, rank, l)).astype(np.float32)).to(BF16)
    scale = torch.tensor([3.4e38, -3.4e38, 1.0])
    want = _want(X, W, A, B, torch.zeros(l), scale, off, order)
    low = torch.zeros((n, l), dtype=torch.float64)
    for g in range(G):
        low[keys == g] = (scale[g].double() * X[keys == g, :1].double() * B[g, 0].double()).abs()
    size = X.double().abs() @ W.double().abs() + low
    got = lq.lq_adapter_product(*(t.cuda() for t in (X, W, A, B)), torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda(), scale=scale.cuda(), y_dtype=F32)
    err = (got.cpu().double() - want).abs()
    assert bool((err <= 2.0 ** -16 * low + (k + 6) * 2.0 ** -24 * size).all()), float(torch.nan_to_num(err, nan=1e40).max())
    assert bool((got.cpu()[low == 0].double() == want[low == 0]).all())
