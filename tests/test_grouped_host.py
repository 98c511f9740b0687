"""CPU-only checks of the grouped operators: what the host refuses, before anything is enqueued (no device pointer is
dereferenced), and workspace sizes."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "paper_2306_08367_amd", "liblq.so")), reason="liblq.so not built")

FAKE = 0x10000   # non-NULL, aligned
NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4, 6


@pytest.fixture(scope="module")
def b():
    from paper_2306_08367_amd import binding
    return binding


def test_struct_layouts_match_the_header(b):
    assert ctypes.sizeof(b.lq_stack) == 40 and b.lq_stack.ld.offset == 24 and b.lq_stack.stride.offset == 32
    assert ctypes.sizeof(b.lq_groups) == 32 and b.lq_groups.offsets.offset == 16 and b.lq_groups.order.offset == 24


def _message(b, rc, code, text):
    assert rc == code and text in b.lq_last_error(), (rc, b.lq_last_error())


@pytest.mark.parametrize("change,code,text", [
    (dict(n=-1), SHAPE, "n -1"), (dict(n=(1 << 30) + 1), SHAPE, "outside 0..2^30"), (dict(G=0), SHAPE, "n_groups 0"),
    (dict(G=4097), SHAPE, "n_groups 4097"), (dict(keys=None), NULL, "keys"), (dict(off=None), NULL, "offsets"), (dict(order=None), NULL, "order"),
    (dict(off=FAKE + 2), SHAPE, "4-byte"), (dict(flags=2), UNSUPPORTED, "flags 0x2"), (dict(n=100_000), WORKSPACE, "workspace"),
    (dict(flags=1), WORKSPACE, "256"), (dict(n=100_000, ws=FAKE, ws_bytes=100), WORKSPACE, "workspace"),
    (dict(n=100_000, ws=FAKE + 16, ws_bytes=1 << 30), WORKSPACE, "aligned"),
])
def test_group_rows_refuses(b, change, code, text):
    a = dict(keys=FAKE, n=10, G=4, off=FAKE, order=FAKE, ws=None, ws_bytes=0, flags=0)
    a.update(change)
    _message(b, b._lib.lq_group_rows(a["keys"], a["n"], a["G"], a["off"], a["order"], a["ws"], a["ws_bytes"], a["flags"], None), code, text)


def _parts(b):
    n, G, k, l = 12, 3, 8, 5
    return dict(groups=b.lq_groups(n, G, FAKE, FAKE), X=b.lq_mat(FAKE, n, k, k, 0), slots=1, W=b.lq_stack(FAKE, G, k, l, 0, l, k * l),
                bias=b.lq_mat(FAKE, G, l, l, 0), gate=b.lq_mat(FAKE, n, l, l, 0), Y=b.lq_mat(FAKE, n, l, l, 0), ws=None, ws_bytes=0, flags=0)


def _ref(v):
    return None if v is None else ctypes.byref(v)


PRODUCT_REFUSALS = [
    ("groups", None, NULL, "groups"), ("groups.n", -1, SHAPE, "n -1"), ("groups.n_groups", 0, SHAPE, "n_groups"), ("groups.n_groups", 4097, SHAPE, "4097"),
    ("groups.offsets", None, NULL, "offsets"), ("groups.order", FAKE + 1, SHAPE, "4-byte"), ("X", None, NULL, "X"), ("X.data", None, NULL, "X: data"),
    ("X.rows", 11, SHAPE, "X is 11 x 8"), ("X.cols", 7, SHAPE, "X is 12 x 7"), ("X.ld", 7, SHAPE, "ld 7"), ("X.dtype", 1, DTYPE, "X and W"),
    ("X.dtype", 3, DTYPE, "dtype 3"), ("X.data", FAKE + 2, SHAPE, "aligned"), ("slots", 0, SHAPE, "x_slots 0"), ("slots", 5, SHAPE, "multiple of x_slots"),
    ("slots", 2, SHAPE, "expected 6 x 8"), ("W.count", 4, SHAPE, "W is 4"), ("W.data", None, NULL, "W: data"), ("W.ld", 4, SHAPE, "W: ld"),
    ("W.stride", -1, SHAPE, "stride"), ("W.rows", 0, SHAPE, "no rows"), ("W.dtype", 9, DTYPE, "W: unknown"), ("bias.rows", 2, SHAPE, "bias is 2 x 5"),
    ("bias.dtype", 1, DTYPE, "bias"), ("gate.cols", 4, SHAPE, "gate is"), ("gate.dtype", 1, DTYPE, "gate"), ("Y.rows", 13, SHAPE, "Y is 13"),
    ("Y.dtype", 1, DTYPE, "bf16 output"), ("Y.data", None, NULL, "Y: data"), ("Y.ld", 3, SHAPE, "Y: ld"), ("flags", 0x100, UNSUPPORTED, "flags"),
    ("flags", 1, WORKSPACE, "256"), ("flags", 0x20, SHAPE, "X is 12 x 8, expected 12 x 5"), ("W.rows", (1 << 30) + 1, SHAPE, "2^30"),
    ("ws", FAKE + 8, WORKSPACE, "aligned"),
]


def _set(parts, name, value):
    if "." in name:
        at, field = name.split(".")
        setattr(parts[at], field, value)
    else:
        parts[name] = value


@pytest.mark.parametrize("name,value,code,text", PRODUCT_REFUSALS)
def test_product_refuses(b, name, value, code, text):
    p = _parts(b)
    _set(p, name, value)
    rc = b._lib.lq_grouped_product(_ref(p["groups"]), _ref(p["X"]), p["slots"], _ref(p["W"]), _ref(p["bias"]), _ref(p["gate"]), _ref(p["Y"]),
                                   p["ws"], p["ws_bytes"], p["flags"], None)
    _message(b, rc, code, text)


def test_slots_need_rows_by_number(b):
    p = _parts(b)
    p["X"].rows = 6
    for flags in (0x20, 0x40):
        rc = b._lib.lq_grouped_product(_ref(p["groups"]), _ref(p["X"]), 2, _ref(p["W"]), None, None, _ref(p["Y"]), None, 0, flags, None)
        _message(b, rc, SHAPE, "x_slots 2")
    rc = b._lib.lq_grouped_gradient(_ref(p["groups"]), _ref(p["X"]), 2, _ref(p["Y"]), _ref(p["W"]), None, None, 0, 0x40, None)
    _message(b, rc, SHAPE, "x_slots 2")


@pytest.mark.parametrize("name,value,code,text", [
    ("groups", None, NULL, "groups"), ("X", None, NULL, "X"), ("Y", None, NULL, "dY"), ("W", None, NULL, "dW"), ("X.rows", 3, SHAPE, "X is 3"),
    ("Y.rows", 3, SHAPE, "dY is 3"), ("Y.dtype", 1, DTYPE, "X and dY"), ("W.rows", 7, SHAPE, "dW is"), ("W.stride", 39, SHAPE, "overlap"),
    ("W.dtype", 1, DTYPE, "bf16 output"), ("bias.cols", 4, SHAPE, "db is"), ("bias.dtype", 1, DTYPE, "db and dW"), ("flags", 0x10, UNSUPPORTED, "flags"),
    ("flags", 1, WORKSPACE, "256"), ("X.cols", 0, SHAPE, "no columns"), ("ws", FAKE + 8, WORKSPACE, "aligned"),
])
def test_gradient_refuses(b, name, value, code, text):
    p = _parts(b)
    _set(p, name, value)
    rc = b._lib.lq_grouped_gradient(_ref(p["groups"]), _ref(p["X"]), p["slots"], _ref(p["Y"]), _ref(p["W"]), _ref(p["bias"]), p["ws"], p["ws_bytes"],
                                    p["flags"], None)
    _message(b, rc, code, text)


@pytest.mark.parametrize("name,value,code,text", [
    ("groups", None, NULL, "groups"), ("X", None, NULL, "X"), ("A", None, NULL, "A"), ("W.rows", 0, SHAPE, "no rows"), ("A.cols", 0, SHAPE, "rank 0"),
    ("A.cols", 257, SHAPE, "rank 257"), ("A.rows", 7, SHAPE, "A is"), ("B.rows", 3, SHAPE, "B is"), ("B.count", 2, SHAPE, "B is 2"), ("X.cols", 7, SHAPE, "X is"),
    ("Y.cols", 4, SHAPE, "Y is"), ("B.dtype", 1, DTYPE, "differ"), ("Y.dtype", 1, DTYPE, "bf16 output"), ("bias.rows", 2, SHAPE, "bias is 2 x 5"),
    ("bias.dtype", 1, DTYPE, "bias"), ("scale", FAKE + 1, SHAPE, "scale"), ("ws", None, WORKSPACE, "workspace"), ("ws_bytes", 100, WORKSPACE, "workspace"),
    ("ws", FAKE + 8, WORKSPACE, "aligned"), ("flags", 0x10, UNSUPPORTED, "flags"),
])
def test_adapter_refuses(b, name, value, code, text):
    n, G, k, l, r = 12, 3, 8, 5, 2
    p = dict(groups=b.lq_groups(n, G, FAKE, FAKE), X=b.lq_mat(FAKE, n, k, k, 0), W=b.lq_mat(FAKE, k, l, l, 0), bias=b.lq_mat(FAKE, 1, l, l, 0),
             A=b.lq_stack(FAKE, G, k, r, 0, r, k * r), B=b.lq_stack(FAKE, G, r, l, 0, l, r * l), scale=FAKE, Y=b.lq_mat(FAKE, n, l, l, 0), ws=FAKE,
             ws_bytes=1 << 20, flags=0)
    _set(p, name, value)
    rc = b._lib.lq_adapter_product(_ref(p["groups"]), _ref(p["X"]), _ref(p["W"]), _ref(p["bias"]), _ref(p["A"]), _ref(p["B"]), p["scale"], _ref(p["Y"]),
                                   p["ws"], p["ws_bytes"], p["flags"], None)
    _message(b, rc, code, text)


def test_workspace_sizes(b):
    assert b.lq_group_rows_workspace_bytes(100, 8) == 0 and b.lq_group_rows_workspace_bytes(-1, 8) == 0 and b.lq_group_rows_workspace_bytes(100, 4097) == 0
    small, large = b.lq_group_rows_workspace_bytes(100_000, 8), b.lq_group_rows_workspace_bytes(1 << 30, 4096)
    assert 0 < small < large and small % 256 == 0
    assert b.lq_adapter_workspace_bytes(0, 4, 8, 8, 300, 0) == 0 and b.lq_adapter_workspace_bytes(8, 4, 8, 8, 4, 5) == 0
    # a few rows over a long inner dimension: partial sums; many rows or a short one: nothing
    assert b.lq_grouped_workspace_bytes(16, 4, 4096, 64, 1) >= 2 * 16 * 64 * 4 and b.lq_grouped_workspace_bytes(16, 4, 128, 64, 1) == 0
    assert b.lq_grouped_workspace_bytes(100_000, 4, 4096, 4096, 1) == 0 and b.lq_grouped_workspace_bytes(16, 0, 4096, 64, 1) == 0
    assert b.lq_grouped_gradient_workspace_bytes(100_000, 4, 64, 32, 0) >= 65 * 32 * 4 and b.lq_grouped_gradient_workspace_bytes(100, 4, 64, 32, 0) == 0
    assert b.lq_adapter_workspace_bytes(8, 4, 64, 64, 4, 1) >= 8 * 8 * 4 + 8 * 4 + 256


def test_the_binding_refuses_before_it_touches_a_gpu(b):
    X, W, off = torch.zeros(4, 8), torch.zeros(2, 8, 3), torch.zeros(3, dtype=torch.int32)
    calls = [lambda: b.lq_group_rows(off, 2), lambda: b.lq_grouped_product(X, W, off), lambda: b.lq_grouped_gradient(X, X, off),
             lambda: b.lq_adapter_product(X, W[0], W, W, off)]
    for call in calls:
        with pytest.raises(ValueError, match="must live on the GPU"):
            call()
    with pytest.raises(TypeError, match="torch.int32"):
        b.lq_group_rows(off.long(), 2)
    with pytest.raises(TypeError, match="expected a tensor"):
        b.lq_grouped_product(None, W, off)
