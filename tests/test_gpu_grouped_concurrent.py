"""The grouped operators in their forms of several launches: captured into graphs that share a workspace and replayed on new inputs, and called
from two host threads at once.  Every result is compared with the eager call's bits."""
import threading

import numpy as np
import pytest
import torch

from tests.test_gpu_grouped import BF16, F32, _keys, _values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lq():
    import paper_2306_08367_amd as lq
    return lq


def _column(seed, n, G):
    return torch.from_numpy(_keys(np.random.default_rng(seed), n, G, "ragged").astype(np.int32)).cuda()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_captured_calls_of_several_launches_replay_with_the_same_bits(lq, dtype):
    """Grouping over many workgroups, partial sums of gradients and of products in splits, adapters with U in a launch of its own."""
    rng = np.random.default_rng(1)
    n, G, k, l, rank, few, long = 30_000, 12, 96, 264, 16, 40, 4096
    code = 1 if dtype == BF16 else 0
    keys, keys_few = _column(0, n, G), _column(1, few, G)
    X, dY, W0, A, B, Xl, Wl = (_values(rng, s, dtype, False).cuda() for s in ((n, k), (n, l), (k, l), (G, k, rank), (G, rank, l), (few, long), (G, long, 64)))
    assert lq.lq_grouped_workspace_bytes(few, G, long, 64, code) > 0 and lq.lq_grouped_gradient_workspace_bytes(n, G, k, l, code) > 0
    need = max(lq.lq_group_rows_workspace_bytes(n, G), lq.lq_grouped_workspace_bytes(few, G, long, 64, code), lq.lq_adapter_workspace_bytes(n, G, k, l, rank, code),
               lq.lq_grouped_gradient_workspace_bytes(n, G, k, l, code))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    off, order = torch.empty(G + 1, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    off_few, order_few = torch.empty(G + 1, dtype=torch.int32, device="cuda"), torch.empty(few, dtype=torch.int32, device="cuda")
    Z, Y = torch.empty((n, l), dtype=dtype, device="cuda"), torch.empty((few, 64), dtype=dtype, device="cuda")
    dW, db = torch.empty((G, k, l), device="cuda"), torch.empty((G, l), device="cuda")
    outputs = (off, order, off_few, order_few, Z, Y, dW, db)

    def first():
        lq.lq_group_rows(keys, G, offsets=off, order=order, ws=ws)
        lq.lq_grouped_gradient(X, dY, off, order, dW=dW, db=db, ws=ws)

    def second():
        lq.lq_group_rows(keys_few, G, offsets=off_few, order=order_few)
        lq.lq_grouped_product(Xl, Wl, off_few, order_few, Y=Y, ws=ws)
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

    graphs = capture(first), capture(second)
    for seed in range(4):
        keys.copy_(_column(10 + seed, n, G))
        keys_few.copy_(_column(20 + seed, few, G))
        for t, shape in ((X, (n, k)), (Xl, (few, long))):
            t.copy_(_values(np.random.default_rng(seed), shape, dtype, False))
        first(), second()
        want = [t.clone() for t in outputs]
        for t in outputs:
            t.fill_(0 if t.dtype == torch.int32 else float("nan"))
        torch.cuda.synchronize()
        graphs[0].replay(), graphs[1].replay(), graphs[0].replay()
        torch.cuda.synchronize()
        for got, w in zip(outputs, want):
            assert torch.equal(got, w)


def test_calls_from_two_host_threads(lq):
    """Different sizes of one operator at once, each thread on a stream of its own."""
    rng = np.random.default_rng(2)
    G, n, k, l, rank = (5, 3000), (20_000, 70_001), 64, 96, 8
    inputs = []
    for g, m in zip(G, n):
        inputs.append((_column(m, m, g), g, *(_values(rng, s, BF16, False).cuda() for s in ((m, k), (k, l), (g, k, l), (g, k, rank), (g, rank, l)))))

    def calls(keys, g, X, W0, W, A, B):
        groups = lq.lq_group_rows(keys, g)
        Y = lq.lq_grouped_product(X, W, *groups)
        return *groups, Y, lq.lq_adapter_product(X, W0, A, B, *groups), lq.lq_grouped_gradient(X, Y, *groups, dw_dtype=F32)[0]

    want = [calls(*i) for i in inputs]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def work(at):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(20):
                    got[at] = calls(*inputs[at])
            stream.synchronize()
        except Exception as e:      # (said by the main thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(at,)) for at in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    torch.cuda.synchronize()
    assert not errors and not any(t.is_alive() for t in threads), errors
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
