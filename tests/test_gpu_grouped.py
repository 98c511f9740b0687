"""The grouped operators (a key chooses the matrix of a row) against the same sums in float64.

Tolerances, per result.  A result is a sum of products of the inputs' own values, summed in fp32 in some order: with m terms and
S = the sum of their absolute values it is off by at most (m + 1) 2^-24 S (one rounding a term), and rounding the
result adds half a step of its type: 2^-24 |y| for fp32, 2^-8 |y| for bf16.  The adapters' inner product U has such an error of
its own, and beside bf16 matrices U is held as two bf16 numbers, 2^-16 of it away.  Inputs that are small integers give
exact sums (all partial sums are integers below 2^24), so there the result is the rounded sum, bit for bit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U24 = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def lq():
    import paper_2306_08367_amd as lq
    return lq


def _grouping(keys, G):
    """(offsets, order) as lists, from the definition."""
    keys = np.asarray(keys)
    of = [np.flatnonzero(keys == g) for g in range(G)]
    off = np.concatenate([[0], np.cumsum([len(o) for o in of])])
    order = np.concatenate(of + [np.flatnonzero((keys < 0) | (keys >= G))])
    return off.astype(np.int32), order.astype(np.int32)


def _keys(rng, n, G, how):
    if how == "even":
        return rng.integers(0, G, n)
    if how == "ragged":       # few large groups, many small and empty ones, some rows without a group
        k = np.minimum((rng.random(n) ** 4 * G).astype(np.int64), G - 1)
        return np.where(rng.random(n) < 0.1, -1, k)
    if how == "one":          # all rows in the last group
        return np.full(n, G - 1)
    if how == "none":
        return np.full(n, -1)
    raise ValueError(how)


def _values(rng, shape, dtype, integers):
    v = rng.integers(-3, 4, shape) if integers else rng.standard_normal(shape)
    return torch.from_numpy(np.asarray(v, dtype=np.float32)).to(dtype)


def _dev(t):
    return None if t is None else t.cuda()


def _check(got, want, terms, size, dtype, exact, what):
    """got within the bounds above of want (float64); `size`: the sums of absolute values."""
    got = got.detach().cpu()
    assert got.dtype == dtype and tuple(got.shape) == tuple(want.shape), what
    if exact:
        assert torch.equal(got, want.to(torch.float32).to(dtype)), f"{what}: not the rounded sum"
        return
    err = (got.double() - want).abs()
    bound = (terms + 1) * U24 * size + STEP[dtype] * (want.abs() + (terms + 1) * U24 * size)
    worst = int((err - bound).argmax())
    assert bool((err <= bound).all()), f"{what}: element {worst} is {err.flatten()[worst]:.3e} off, {bound.flatten()[worst]:.3e} allowed"


# ------------------------------------------------------------------ rows of the groups

@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 1023, 1025, 16_384, 16_385, 70_001, 1_000_003])
@pytest.mark.parametrize("G,how", [(1, "even"), (2, "ragged"), (7, "one"), (64, "ragged"), (65, "even"), (1000, "none"), (4096, "ragged")])
def test_rows_of_groups(lq, n, G, how):
    rng = np.random.default_rng(n + G)
    keys = _keys(rng, n, G, how)
    keys[rng.random(n) < 0.01] = G + 5               # outside on the other side
    off, order = lq.lq_group_rows(torch.from_numpy(keys.astype(np.int32)).cuda(), G)
    place = np.where((keys < 0) | (keys >= G), G, keys)
    np.testing.assert_array_equal(order.cpu().numpy(), np.argsort(place, kind="stable"))
    np.testing.assert_array_equal(off.cpu().numpy(), np.searchsorted(np.sort(place), np.arange(G + 1)))


@pytest.mark.parametrize("n", [10_240, 10_241, 11_265, 262_144, 262_145, 2_097_152, 2_097_153])
@pytest.mark.parametrize("G,how", [(3, "ragged"), (300, "even"), (4096, "even")])
def test_rows_of_groups_where_the_shares_of_workgroups_change(lq, n, G, how):
    keys = _keys(np.random.default_rng(n - G), n, G, how)
    off, order = lq.lq_group_rows(torch.from_numpy(keys.astype(np.int32)).cuda(), G)
    place = np.where(keys < 0, G, keys)
    np.testing.assert_array_equal(order.cpu().numpy(), np.argsort(place, kind="stable"))
    np.testing.assert_array_equal(off.cpu().numpy(), np.searchsorted(np.sort(place), np.arange(G + 1)))


def test_rows_of_groups_at_the_ends_of_the_key_type(lq):
    keys = torch.tensor([2 ** 31 - 1, -2 ** 31, 0, -1, 1, 2, 0], dtype=torch.int32, device="cuda")
    off, order = lq.lq_group_rows(keys, 2)
    assert off.tolist() == [0, 2, 3] and order.tolist() == [2, 6, 4, 0, 1, 3, 5]
    with pytest.raises(lq.LQError, match="FK_RANGE"):
        lq.lq_group_rows(keys, 2, flags=lq.LQ_CHECK_FKS)
    off, order = lq.lq_group_rows(keys.clamp(-1, 2) - 1, 2, flags=lq.LQ_CHECK_FKS)
    assert off.tolist() == [0, 1, 3] and order.tolist() == [4, 0, 5, 1, 2, 3, 6]


# ------------------------------------------------------------------ products

def _product(X, W, off, order, bias, gate, transposed, relu, x_grouped, y_grouped, slots):
    """(result, sum of absolute values) in float64."""
    n, G = len(order), W.shape[0]
    N = W.shape[1] if transposed else W.shape[2]
    Y, S = torch.zeros((n, N), dtype=torch.float64), torch.zeros((n, N), dtype=torch.float64)
    for g in range(G):
        p = np.arange(off[g], off[g + 1])
        if len(p) == 0:
            continue
        r = order[p]
        x, w = X[p if x_grouped else r // slots].double(), W[g].double()
        w = w.T if transposed else w
        y, s = x @ w, x.abs() @ w.abs()
        if bias is not None:
            y, s = y + bias[g].double(), s + bias[g].double().abs()
        at = p if y_grouped else r
        Y[at], S[at] = torch.relu(y) if relu else y, s
    if gate is not None:
        Y = torch.where(gate.double() > 0, Y, 0.0)
    return Y, S


def _run_product(lq, n, G, k, l, dtype, how="ragged", out=None, bias=False, gate=False, transposed=False, relu=False, x_grouped=False,
                 y_grouped=False, slots=1, ordered=True, integers=False, seed=0):
    rng = np.random.default_rng(seed + n + 3 * k + 5 * l)
    keys = _keys(rng, n * slots, G, how)
    if not ordered:
        keys = np.concatenate([np.sort(keys[keys >= 0]), keys[keys < 0]])
    off, order = _grouping(keys, G)
    K, N = (l, k) if transposed else (k, l)
    X, W = _values(rng, (n, K), dtype, integers), _values(rng, (G, k, l), dtype, integers)
    b = _values(rng, (G, N), dtype, integers) if bias else None
    h = _values(rng, (n * slots, N), dtype, integers) if gate else None
    want, size = _product(X, W, off, order, b, h, transposed, relu, x_grouped, y_grouped, slots)
    got = lq.lq_grouped_product(X.cuda(), W.cuda(), _dev(torch.from_numpy(off)), _dev(torch.from_numpy(order)) if ordered else None, bias=_dev(b),
                                gate=_dev(h), y_dtype=out, transposed=transposed, relu=relu, x_grouped=x_grouped, y_grouped=y_grouped,
                                x_slots=slots)
    _check(got, want, K + 1, size, out or dtype, integers, f"product {n} {G} {k} {l} {dtype}")


SHAPES = [(1, 1, 1, 1), (1, 4, 16, 8), (3, 2, 7, 5), (5, 300, 64, 128), (16, 64, 256, 64), (64, 8, 100, 36), (130, 3, 33, 129), (257, 5, 128, 256),
          (700, 40, 72, 24), (1000, 7, 683, 250), (2500, 6, 264, 520)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,G,k,l", SHAPES)
@pytest.mark.parametrize("transposed", [False, True], ids=["forward", "transposed"])
def test_product_of_integers_is_exact(lq, n, G, k, l, dtype, transposed):
    _run_product(lq, n, G, k, l, dtype, transposed=transposed, integers=True)
    _run_product(lq, n, G, k, l, dtype, transposed=transposed, integers=True, bias=True, relu=True, gate=True, y_grouped=True, out=F32, seed=1)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,G,k,l", SHAPES)
@pytest.mark.parametrize("transposed", [False, True], ids=["forward", "transposed"])
def test_product(lq, n, G, k, l, dtype, transposed):
    _run_product(lq, n, G, k, l, dtype, transposed=transposed, bias=not transposed, relu=not transposed, gate=transposed)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("how", ["even", "one", "none"])
@pytest.mark.parametrize("more", [dict(x_grouped=True), dict(y_grouped=True), dict(x_grouped=True, y_grouped=True, transposed=True, gate=True),
                                  dict(slots=3, relu=True), dict(slots=2, y_grouped=True, bias=True), dict(ordered=False, bias=True), dict(out=F32)],
                         ids=["x", "y", "xy", "slots", "slots-y", "identity", "f32-out"])
def test_product_row_orders(lq, dtype, how, more):
    _run_product(lq, 333, 9, 96, 80, dtype, how=how, integers=True, **more)
    _run_product(lq, 40, 9, 96, 81, dtype, how=how, integers=True, **more)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,G,k,l", [(1, 1, 4100, 8), (5, 3, 2053, 70), (320, 10, 3509, 53), (60, 64, 4096, 64), (33, 2, 2500, 300)])
def test_products_of_few_rows_over_a_long_inner_dimension(lq, n, G, k, l, dtype):
    """These run in splits of the inner dimension, whose partial sums a second launch adds up."""
    for how in ("ragged", "even", "none"):
        _run_product(lq, n, G, k, l, dtype, how=how, integers=True, bias=True, relu=True, gate=True)
        _run_product(lq, n, G, l, k, dtype, how=how, integers=True, transposed=True, gate=True, y_grouped=True, out=F32)
        _run_product(lq, n, G, k, l, dtype, how=how, slots=2, bias=True)


@pytest.mark.parametrize("n", [3, 900, 6000])
def test_the_most_groups(lq, n):
    for dtype in (F32, BF16):
        _run_product(lq, n, 4096, 16, 24, dtype, integers=True, bias=True)
        _run_product(lq, n, 4096, 24, 16, dtype, how="one", integers=True, transposed=True)
        _run_gradient(lq, n, 4096, 16, 24, dtype, integers=True)
        _run_adapter(lq, n, 4096, 32, 24, 3, dtype, integers=True)
        _run_adapter(lq, n, 4096, 32, 24, 3, dtype, how="one", integers=True)


def test_products_of_many_rows(lq):
    for dtype, n in ((BF16, 40_000), (F32, 20_000)):
        for transposed in (False, True):
            _run_product(lq, n, 5, 192, 320, dtype, integers=True, transposed=transposed, y_grouped=True, relu=True)


def _strided(t, rows, extra, fill=float("nan"), offset=0):
    """t [.. x r x c] inside a larger buffer full of `fill`: rows `extra` elements further apart, a start `offset` elements in."""
    lead = t.shape[:-2]
    r, c = t.shape[-2:]
    count = int(np.prod(lead)) if lead else 1
    buf = torch.full((offset + count * (r + rows) * (c + extra) + 8,), fill, dtype=t.dtype, device="cuda")
    strides = ((r + rows) * (c + extra),) * len(lead) + (c + extra, 1)
    v = buf.as_strided(tuple(t.shape), strides, offset)
    v.copy_(t)
    return buf, v


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("extra,offset", [(8, 0), (8, 8), (4, 4), (3, 1), (1, 0)])
@pytest.mark.parametrize("transposed", [False, True], ids=["forward", "transposed"])
@pytest.mark.parametrize("n", [20, 300])
def test_product_of_strided_matrices(lq, n, dtype, extra, offset, transposed):
    """Rows and matrices apart, NaN between them: nothing of it is read into a result and none of it is written."""
    rng = np.random.default_rng(5)
    G, k, l = 4, 48, 72
    off, order = _grouping(_keys(rng, n, G, "ragged"), G)
    K, N = (l, k) if transposed else (k, l)
    X, W, b, h = (_values(rng, s, dtype, True) for s in ((n, K), (G, k, l), (G, N), (n, N)))
    want, _ = _product(X, W, off, order, b, h, transposed, False, False, False, 1)
    (_, Xs), (_, Ws), (_, bs), (_, hs) = (_strided(t, 2, extra, offset=offset) for t in (X, W, b, h))
    buf, Y = _strided(torch.zeros((n, N), dtype=dtype), 0, extra, fill=7.0, offset=offset)
    got = lq.lq_grouped_product(Xs, Ws, torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda(), bias=bs, gate=hs, Y=Y, transposed=transposed)
    assert got is Y and torch.equal(Y.cpu(), want.to(dtype))
    Y.fill_(7.0)
    assert bool((buf == 7.0).all()), "written outside the result"


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n", [6, 90, 400])
def test_special_values_stay_in_their_row_group_and_column(lq, dtype, n):
    rng = np.random.default_rng(n)
    G, k, l = 3, 40, 24
    keys = np.arange(n) % G
    off, order = _grouping(keys, G)
    X, W = _values(rng, (n, k), dtype, True), _values(rng, (G, k, l), dtype, True)
    W[1, :, :] = float("nan")
    W[2, 3, 5] = float("inf")
    X[:, 3] = 1.0
    X[0, 7] = float("nan")
    X[5, :] = float("inf")
    want, _ = _product(X, W, off, order, None, None, False, False, False, False, 1)
    got = lq.lq_grouped_product(X.cuda(), W.cuda(), torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda()).double().cpu()
    ok = torch.ones(n, dtype=torch.bool)
    ok[5] = False                      # inf * 0 and inf - inf: NaN in both, compared below
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got[ok], nan=0.0), torch.nan_to_num(want[ok].to(dtype).double(), nan=0.0))
    # a gate that is NaN or zero is not positive
    gate = torch.tensor([float("nan"), 0.0, -0.0, 1.0, -1.0, float("inf")] * 4, dtype=dtype, device="cuda").repeat(n, 1)
    got = lq.lq_grouped_product(X.cuda(), torch.ones((G, k, l), dtype=dtype, device="cuda"), torch.from_numpy(off).cuda(),
                                torch.from_numpy(order).cuda(), gate=gate)
    assert bool((got[1:5].float().view(-1, 4, 6)[:, :, [0, 1, 2, 4]] == 0).all())


# ------------------------------------------------------------------ gradients

def _run_gradient(lq, n, G, k, l, dtype, how="ragged", out=None, bias=True, x_grouped=False, y_grouped=False, slots=1, ordered=True,
                  integers=False, seed=0, extra=0):
    rng = np.random.default_rng(seed + n + 3 * k + 5 * l)
    keys = _keys(rng, n * slots, G, how)
    if not ordered:
        keys = np.concatenate([np.sort(keys[keys >= 0]), keys[keys < 0]])
    off, order = _grouping(keys, G)
    X, dY = _values(rng, (n, k), dtype, integers), _values(rng, (n * slots, l), dtype, integers)
    dW, S = torch.zeros((G, k, l), dtype=torch.float64), torch.zeros((G, k, l), dtype=torch.float64)
    db, s = torch.zeros((G, l), dtype=torch.float64), torch.zeros((G, l), dtype=torch.float64)
    for g in range(G):
        p = np.arange(off[g], off[g + 1])
        r = order[p]
        x, d = X[p if x_grouped else r // slots].double(), dY[p if y_grouped else r].double()
        dW[g], S[g], db[g], s[g] = x.T @ d, x.abs().T @ d.abs(), d.sum(0), d.abs().sum(0)
    Xs, Ds = (_strided(t, 0, extra)[1] if extra else t.cuda() for t in (X, dY))
    gotW, gotb = lq.lq_grouped_gradient(Xs, Ds, torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda() if ordered else None, dw_dtype=out,
                                        want_bias=bias, x_grouped=x_grouped, y_grouped=y_grouped, x_slots=slots)
    most = int(max(off[1:] - off[:-1]))
    _check(gotW, dW, most, S, out or dtype, integers, f"dW {n} {G} {k} {l} {dtype}")
    if bias:
        _check(gotb, db, most, s, out or dtype, integers, f"db {n} {G} {k} {l} {dtype}")
    else:
        assert gotb is None


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,G,k,l", SHAPES)
def test_gradient(lq, n, G, k, l, dtype):
    _run_gradient(lq, n, G, k, l, dtype, integers=True)
    _run_gradient(lq, n, G, k, l, dtype, out=F32, y_grouped=True, seed=1)
    _run_gradient(lq, n, G, k, l, dtype, integers=True, extra=3, bias=False, seed=2)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("how", ["even", "one", "none"])
@pytest.mark.parametrize("more", [dict(x_grouped=True), dict(x_grouped=True, y_grouped=True), dict(slots=3), dict(slots=2, y_grouped=True),
                                  dict(ordered=False)], ids=["x", "xy", "slots", "slots-y", "identity"])
def test_gradient_row_orders(lq, dtype, how, more):
    _run_gradient(lq, 333, 9, 96, 80, dtype, how=how, integers=True, **more)


def test_gradients_of_many_rows(lq):
    for dtype, n in ((BF16, 60_000), (F32, 60_000)):
        _run_gradient(lq, n, 3, 64, 96, dtype, integers=True, out=F32)
        _run_gradient(lq, n, 3, 100, 64, dtype, integers=True, out=F32, seed=3)
    _run_gradient(lq, 3000, 4, 640, 512, BF16, integers=True, out=F32)


def test_gradient_of_no_rows_is_zero(lq):
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    dW, db = lq.lq_grouped_gradient(torch.empty((0, 20), device="cuda"), torch.empty((0, 12), device="cuda"), off, want_bias=True)
    assert dW.shape == (3, 20, 12) and bool((dW == 0).all()) and bool((db == 0).all())


def test_gradients_are_those_of_the_product_by_differences(lq):
    """fp32: (f(W + h D) - f(W - h D)) / 2 h of f = sum(C * product) is the sum of D * dW, likewise for x and the bias.  f is linear in each
    of them, so the differences carry rounding only: with integers and h = 1 none."""
    rng = np.random.default_rng(3)
    n, G, k, l = 77, 5, 24, 16
    off, order = (torch.from_numpy(t).cuda() for t in _grouping(_keys(rng, n, G, "ragged"), G))
    X, W, b, C, dX, dW_, db_ = (_values(rng, s, F32, True).cuda() for s in ((n, k), (G, k, l), (G, l), (n, l), (n, k), (G, k, l), (G, l)))
    f = lambda x, w, c: float((C.double() * lq.lq_grouped_product(x, w, off, order, bias=c).double()).sum())
    gW, gb = lq.lq_grouped_gradient(X, C, off, order, want_bias=True)
    gX = lq.lq_grouped_product(C, W, off, order, transposed=True)
    dot = lambda a, c: float((a.double() * c.double()).sum())
    assert f(X, W + dW_, b) - f(X, W - dW_, b) == 2 * dot(gW, dW_)
    assert f(X, W, b + db_) - f(X, W, b - db_) == 2 * dot(gb, db_)
    assert f(X + dX, W, b) - f(X - dX, W, b) == 2 * dot(gX, dX)


# ------------------------------------------------------------------ adapters

def _run_adapter(lq, n, G, k, l, rank, dtype, how="ragged", out=None, bias=True, scale=True, ordered=True, integers=False, seed=0, extra=0, runs=1):
    rng = np.random.default_rng(seed + n + 3 * k + 5 * l + rank)
    keys = np.repeat(_keys(rng, -(-n // runs), G, how), runs)[:n]
    if not ordered:
        keys = np.concatenate([np.sort(keys[keys >= 0]), keys[keys < 0]])
    off, order = _grouping(keys, G)
    X, W, A, B, b = (_values(rng, s, dtype, integers) for s in ((n, k), (k, l), (G, k, rank), (G, rank, l), (l,)))
    sc = torch.from_numpy(rng.choice([0.5, 1.0, 2.0], G).astype(np.float32)) if scale else None
    if integers:                    # (sparse factors keep U and the sums among the exact ones)
        A = torch.where(torch.from_numpy(rng.random(A.shape) < 4.0 / k), A, 0)
    want, S = X.double() @ W.double(), X.double().abs() @ W.double().abs()
    if bias:
        want, S = want + b.double(), S + b.double().abs()
    loss = torch.zeros_like(want)
    for g in range(G):
        r = order[off[g]:off[g + 1]]
        u, su = X[r].double() @ A[g].double(), X[r].double().abs() @ A[g].double().abs()
        f = float(sc[g]) if scale else 1.0
        want[r] += f * u @ B[g].double()
        S[r] += f * u.abs() @ B[g].double().abs()
        loss[r] += f * ((k + 2) * U24 * su + (2.0 ** -16 if dtype == BF16 else 0.0) * u.abs()) @ B[g].double().abs()
    Xs, Ws, As, Bs = ((_strided(t, 0, extra)[1] if extra else t.cuda()) for t in (X, W, A, B))
    got = lq.lq_adapter_product(Xs, Ws, As, Bs, torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda() if ordered else None,
                                scale=_dev(sc), bias=_dev(b) if bias else None, y_dtype=out)
    if integers:
        _check(got, want, 0, S, out or dtype, True, f"adapter {n} {G} {k} {l} {rank} {dtype}")
    else:
        # (the steps of the extended sum are k + 2 ranks of every adapter of the tile at most; zeros add no rounding)
        terms = k + 2 * rank + 2
        _check(got, want, terms, S + loss / ((terms + 1) * U24), out or dtype, False, f"adapter {n} {G} {k} {l} {rank} {dtype}")


ADAPTER_SHAPES = [(1, 1, 16, 8, 1), (1, 300, 64, 64, 16), (3, 2, 7, 5, 3), (64, 48, 256, 128, 16), (65, 64, 100, 36, 7), (200, 3, 683, 130, 33),
                  (300, 200, 128, 256, 8), (513, 11, 96, 72, 64), (1000, 30, 264, 520, 20)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n,G,k,l,rank", ADAPTER_SHAPES)
def test_adapter(lq, n, G, k, l, rank, dtype):
    _run_adapter(lq, n, G, k, l, rank, dtype)
    _run_adapter(lq, n, G, k, l, rank, dtype, integers=True, how="even", bias=False, seed=1)
    _run_adapter(lq, n, G, k, l, rank, dtype, integers=True, out=F32, scale=False, extra=3, runs=5, seed=2)
    _run_adapter(lq, n, G, k, l, rank, dtype, out=F32, ordered=False, extra=8, seed=3)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("how", ["even", "one", "none"])
def test_adapter_row_orders(lq, dtype, how):
    for n in (17, 333):
        _run_adapter(lq, n, 9, 96, 80, 12, dtype, how=how, integers=True)
        _run_adapter(lq, n, 9, 96, 80, 12, dtype, how=how, integers=True, ordered=False)


def test_adapters_of_many_rows(lq):
    _run_adapter(lq, 30_000, 6, 192, 320, 16, BF16, integers=True, runs=700)
    _run_adapter(lq, 30_000, 400, 192, 320, 16, BF16, integers=True, runs=3)
    _run_adapter(lq, 12_000, 60, 100, 300, 5, F32, integers=True, runs=9)
    _run_adapter(lq, 40, 5, 64, 64, 256, BF16, integers=True)


def test_an_adapter_of_other_rows_does_not_reach_a_row(lq):
    """NaN and infinity in one adapter: the other rows, those without an adapter among them, are as without it."""
    rng = np.random.default_rng(1)
    for dtype in (F32, BF16):
        for n in (12, 200):
            G, k, l, rank = 4, 64, 48, 8
            keys = np.arange(n) % (G + 1) - 1
            off, order = (torch.from_numpy(t).cuda() for t in _grouping(keys, G))
            X, W, A, B = (_values(rng, s, dtype, True).cuda() for s in ((n, k), (k, l), (G, k, rank), (G, rank, l)))
            before = lq.lq_adapter_product(X, W, A, B, off, order)
            A[1] = float("nan")
            B[2] = float("inf")
            after = lq.lq_adapter_product(X, W, A, B, off, order)
            other = torch.from_numpy((keys != 1) & (keys != 2)).cuda()
            assert torch.equal(before[other], after[other])
            assert bool(torch.isnan(after[torch.from_numpy(keys == 1).cuda()]).all())


# ------------------------------------------------------------------ together, as a program uses them

def test_two_layer_experts_forward_and_backward(lq):
    """Keys -> grouping -> two layers, the hidden rows in the order of the groups -> gradients of everything, against float64 autograd."""
    rng = np.random.default_rng(8)
    n, slots, G, k, h, l = 150, 2, 6, 40, 56, 24
    keys = _keys(rng, n * slots, G, "ragged").astype(np.int32)
    X, W1, b1, W2, b2, C = (_values(rng, s, F32, False) for s in ((n, k), (G, k, h), (G, h), (G, h, l), (G, l), (n * slots, l)))
    off, order = lq.lq_group_rows(torch.from_numpy(keys).cuda(), G)
    d = [t.cuda() for t in (X, W1, b1, W2, b2, C)]
    H = lq.lq_grouped_product(d[0], d[1], off, order, bias=d[2], relu=True, x_slots=slots, y_grouped=True)
    Y = lq.lq_grouped_product(H, d[3], off, order, bias=d[4], x_grouped=True)
    dW2, db2 = lq.lq_grouped_gradient(H, d[5], off, order, want_bias=True, x_grouped=True)
    dH = lq.lq_grouped_product(d[5], d[3], off, order, transposed=True, gate=H, y_grouped=True)
    dW1, db1 = lq.lq_grouped_gradient(d[0], dH, off, order, want_bias=True, x_slots=slots, y_grouped=True)
    dX = lq.lq_grouped_product(dH, d[1], off, order, transposed=True, x_grouped=True).view(n, slots, k).sum(1)
    leaves = [t.double().requires_grad_() for t in (X, W1, b1, W2, b2)]
    x, w1, c1, w2, c2 = leaves
    rows = torch.arange(n * slots) // slots
    y = torch.zeros((n * slots, l), dtype=torch.float64)
    for g in range(G):
        at = torch.from_numpy(np.flatnonzero(keys == g))
        y = y.index_add(0, at, torch.relu(x[rows[at]] @ w1[g] + c1[g]) @ w2[g] + c2[g])
    (y * C.double()).sum().backward()
    # sums of up to max(k, h, rows of a group) terms of values around 1..10 one after the other: 2^-24 of a few hundred a term
    for name, got, want in [("Y", Y, y.detach()), ("dX", dX, x.grad), ("dW1", dW1, w1.grad), ("db1", db1, c1.grad), ("dW2", dW2, w2.grad), ("db2", db2, c2.grad)]:
        err = float((got.double().cpu() - want).norm() / want.norm())
        assert err < 300 * U24, f"{name}: {err:.2e}"


def test_serving_from_raw_keys(lq):
    """Key values -> rows of the key map -> groups -> adapters and a model per group, twice with the same bits."""
    rng = np.random.default_rng(9)
    G, n, k, l, rank = 20, 96, 128, 64, 8
    names = torch.from_numpy(rng.permutation(1000)[:G].astype(np.int32) * 7).cuda()
    who = torch.from_numpy(rng.integers(-2, G, n)).cuda()
    raw = torch.where(who >= 0, names[who.clamp_min(0)], -5).to(torch.int32)
    keys = lq.lq_keymap_lookup(lq.lq_keymap_build(names), raw)
    off, order = lq.lq_group_rows(keys, G)
    X, W, A, B, W2 = (_values(rng, s, BF16, False).cuda() for s in ((n, k), (k, l), (G, k, rank), (G, rank, l), (G, l, 16)))
    Z = lq.lq_adapter_product(X, W, A, B, off, order)
    Y = lq.lq_grouped_product(Z, W2, off, order)
    again = lq.lq_grouped_product(lq.lq_adapter_product(X, W, A, B, off, order), W2, off, order)
    assert torch.equal(Y, again) and bool((Y[who < 0] == 0).all()) and bool((Y[who >= 0] != 0).any())


def test_captured_calls_replay_with_the_same_bits(lq):
    """Two graphs that share a workspace, replayed in turn with eager work between, on new inputs."""
    rng = np.random.default_rng(10)
    n, G, k, l, rank = 300, 7, 128, 96, 16
    keys = torch.from_numpy(_keys(rng, n, G, "ragged").astype(np.int32)).cuda()
    off, order = torch.empty(G + 1, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    X, W0, W, A, B = (_values(rng, s, BF16, False).cuda() for s in ((n, k), (k, l), (G, k, l), (G, k, rank), (G, rank, l)))
    need = max(lq.lq_grouped_workspace_bytes(n, G, k, l, 1), lq.lq_adapter_workspace_bytes(n, G, k, l, rank, 1),
               lq.lq_grouped_gradient_workspace_bytes(n, G, k, l, 1), 256)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    Y, Z = torch.empty((n, l), dtype=BF16, device="cuda"), torch.empty((n, l), dtype=BF16, device="cuda")
    dW = torch.empty((G, k, l), device="cuda")

    def first():
        lq.lq_group_rows(keys, G, offsets=off, order=order, ws=ws)
        lq.lq_grouped_product(X, W, off, order, Y=Y, ws=ws)
        lq.lq_grouped_gradient(X, Y, off, order, dW=dW, ws=ws)

    def second():
        lq.lq_adapter_product(X, W0, A, B, off, order, Y=Z, ws=ws)

    def capture(fn):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            fn()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            fn()
        return graph
    one, two = capture(first), capture(second)
    for seed in range(4):
        keys.copy_(torch.from_numpy(_keys(np.random.default_rng(seed), n, G, "ragged").astype(np.int32)))
        X.copy_(_values(np.random.default_rng(seed), (n, k), BF16, False))
        first(), second()
        want = [t.clone() for t in (Y, Z, dW, off, order)]
        for t in (Y, Z, dW):
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        one.replay(), two.replay(), one.replay()
        torch.cuda.synchronize()
        for got, w in zip((Y, Z, dW, off, order), want):
            assert torch.equal(got, w)


def test_calls_on_another_stream(lq):
    rng = np.random.default_rng(11)
    n, G, k, l, rank = 500, 5, 256, 192, 8
    keys = torch.from_numpy(_keys(rng, n, G, "ragged").astype(np.int32)).cuda()
    X, W0, W, A, B = (_values(rng, s, BF16, False).cuda() for s in ((n, k), (k, l), (G, k, l), (G, k, rank), (G, rank, l)))
    calls = lambda s: [lq.lq_grouped_product(X, W, *g, stream=s) for g in [lq.lq_group_rows(keys, G, stream=s)]] + [
        lq.lq_adapter_product(X, W0, A, B, *lq.lq_group_rows(keys, G, stream=s), stream=s),
        lq.lq_grouped_gradient(X, X, *lq.lq_group_rows(keys, G, stream=s), stream=s)[0]]
    want = calls(None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [calls(s) for s in streams]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g in got for a, b in zip(g, want))


def test_offsets_beyond_32_bits(lq):
    """Rows of X and Y, and matrices, more than 2^31 elements apart."""
    n, G, k, l = 3, 2, 64, 64
    far = (1 << 30) + 64
    buf = torch.zeros(2 * far + 4096, dtype=BF16, device="cuda")
    X = buf.as_strided((n, k), (far, 1))
    rng = np.random.default_rng(12)
    values = _values(rng, (n, k), BF16, True)
    X.copy_(values)
    W = _values(rng, (G, k, l), BF16, True)
    off, order = _grouping([1, 0, 1], G)
    o, r = torch.from_numpy(off).cuda(), torch.from_numpy(order).cuda()
    want, _ = _product(values, W, off, order, None, None, False, False, False, False, 1)
    got = lq.lq_grouped_product(X, W.cuda(), o, r)
    assert torch.equal(got.cpu(), want.to(BF16))
    dW, _ = lq.lq_grouped_gradient(X, got, o, r, dw_dtype=F32)
    near, _ = lq.lq_grouped_gradient(values.cuda(), got, o, r, dw_dtype=F32)
    assert torch.equal(dW, near)
    Y = buf.as_strided((n, l), (far, 1), 2048)
    lq.lq_grouped_product(X, W.cuda(), o, r, Y=Y)
    assert torch.equal(Y.cpu(), want.to(BF16))
    Wfar = buf.as_strided((G, k, l), (2 * far - 64 * 64, l, 1), 4096 - 64)[:, :, :]
    Wfar.copy_(W)
    assert torch.equal(lq.lq_grouped_product(values.cuda(), Wfar, o, r).cpu(), want.to(BF16))


def test_groups_are_verified_on_request(lq):
    X, W = torch.ones((4, 8), device="cuda"), torch.ones((2, 8, 8), device="cuda")
    A, B, W0 = torch.ones((2, 8, 2), device="cuda"), torch.ones((2, 2, 8), device="cuda"), torch.ones((8, 8), device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    calls = [lambda o, r: lq.lq_grouped_product(X, W, o, r, flags=lq.LQ_CHECK_FKS), lambda o, r: lq.lq_grouped_gradient(X, X, o, r, flags=lq.LQ_CHECK_FKS),
             lambda o, r: lq.lq_adapter_product(X, W0, A, B, o, r, flags=lq.LQ_CHECK_FKS)]
    for call in calls:
        call(i32(0, 2, 4), i32(3, 1, 0, 2))
        for o, r in [(i32(0, 3, 2), i32(3, 1, 0, 2)), (i32(0, 2, 5), i32(3, 1, 0, 2)), (i32(1, 2, 4), i32(3, 1, 0, 2)), (i32(0, 2, 4), i32(3, 4, 0, 2)),
                     (i32(0, 2, 4), i32(3, -1, 0, 2))]:
            with pytest.raises(lq.LQError, match="FK_RANGE"):
                call(o, r)
