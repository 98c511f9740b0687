"""Performance cases of the grouped operators: products whose matrix is chosen row by row through a key.

The key of a row says which of G models it belongs to (a store, a segment, an expert, a request's adapter), the way a
foreign key says which dimension row it joins.  Four operators:

  rows      the row numbers of every group, in order, from a column of keys (lq_group_rows)
  product   Y_i = x_i W_g(i) + b_g(i), with ReLU, or the gradient of x: the same with W_g transposed and the ReLU of the
            layer below (lq_grouped_product)
  gradient  dW_g = sum over the rows of group g of x_i^T dy_i, and db_g (lq_grouped_gradient)
  adapter   Y_i = x_i W + b + scale_g (x_i A_g) B_g: one shared matrix and a low-rank one per key (lq_adapter_product)

Sizes: widths from 16 to 4,096 around those of this repository's models (100 -> 64, 683, 1024 -> 256), one row to tens of
thousands (millions of keys), 1 to 256 groups of ragged sizes, empty ones and rows without a group among them.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _rows(n, groups, **more):
    return {"op": "rows", "n": n, "groups": groups, "dropped": 0.0, **more}


def _product(n, groups, k, l, dtype, **more):
    return {"op": "product", "n": n, "slots": 1, "groups": groups, "k": k, "l": l, "dtype": dtype, "bias": False, "relu": False,
            "transposed": False, "gate": False, "x_grouped": False, "y_grouped": False, "dropped": 0.0, **more}


def _gradient(n, groups, k, l, dtype, **more):
    return {"op": "gradient", "n": n, "slots": 1, "groups": groups, "k": k, "l": l, "dtype": dtype, "out": dtype, "bias": False,
            "x_grouped": False, "y_grouped": False, "dropped": 0.0, **more}


def _adapter(n, requests, groups, k, l, r, dtype, **more):
    return {"op": "adapter", "n": n, "requests": requests, "groups": groups, "k": k, "l": l, "r": r, "dtype": dtype, "bias": False,
            "dropped": 0.0, **more}


def listed():
    return [
        # A serving batch: each of 64 requests names one of 8 models, a few none.
        _rows(64, 8, dropped=0.1, name="rows_batch"),
        # The fact table of the aggregate configuration grouped by its 2,000-row dimension.
        _rows(6_000_000, 2000, name="rows_fact_table"),
        # One row, two models for it: the first layer of the wide bf16 model.
        _product(1, 8, 1024, 256, "bf16", slots=2, bias=True, relu=True, name="product_one_row"),
        # A step of a few requests, eight of 64 experts each: nearly every expert is read for two rows.
        _product(16, 64, 2048, 1024, "bf16", slots=8, name="product_few_rows"),
        # A long batch, two of 32 experts a row, results in the order of the groups for the next layer.
        _product(16_384, 32, 2048, 4096, "bf16", slots=2, relu=True, y_grouped=True, name="product_batch"),
        # fp32 models of seven segments over the joined width of a star schema, some rows in no segment.
        _product(10_007, 7, 683, 250, "f32", bias=True, relu=True, dropped=0.03, name="product_segments_f32"),
        # The gradient of a hidden layer, through the ReLU that made it.
        _product(16_384, 16, 1024, 2048, "bf16", transposed=True, gate=True, x_grouped=False, y_grouped=True, name="product_gradient_of_x"),
        # The weights' gradient of a long batch, in fp32 as an optimiser adds it up.
        _gradient(16_384, 16, 2048, 1024, "bf16", out="f32", bias=True, slots=2, name="gradient_batch"),
        # The first layer of the headline model, one for each of twelve segments.
        _gradient(20_001, 12, 100, 64, "f32", bias=True, dropped=0.03, name="gradient_segments_f32"),
        # One new row for each of 64 requests with 48 adapters between them, some without one.
        _adapter(64, 64, 48, 4096, 4096, 16, "bf16", dropped=0.1, name="adapter_few_rows"),
        # Prompts of 24 requests at once.
        _adapter(8_192, 24, 16, 4096, 4096, 32, "bf16", bias=True, dropped=0.1, name="adapter_prompts"),
        # fp32, adapters of odd rank over an odd width.
        _adapter(1_001, 90, 40, 683, 512, 7, "f32", bias=True, name="adapter_f32"),
    ]


def _spread(rng, lo, hi):
    """A size of lo .. hi, spread over its logarithm; half of the larger ones are multiples of 8."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = v - v % 8 if v >= 64 and rng.random() < 0.5 else v
    return min(max(v, lo), hi)


def _too_much(c):
    if c["op"] == "rows":
        return False
    w, most = work(c), max(c["k"], c["l"])
    rows = c["n"] * c.get("slots", 1)
    matrices = c["groups"] * (c["k"] * c["l"] if c["op"] != "adapter" else (c["k"] + c["l"]) * c["r"])
    return w["flops"] > (5e11 if c["dtype"] == "bf16" else 5e10) or matrices > 2 ** 27 or rows * most > 2 ** 27


def draw(rng):
    while True:
        op = rng.choice(["rows", "product", "product", "gradient", "adapter"])
        dtype = rng.choice(["f32", "bf16", "bf16"])
        dropped = rng.choice([0.0, 0.0, 0.05])
        groups = _spread(rng, 1, 256)
        k, l = _spread(rng, 16, 4096), _spread(rng, 16, 4096)
        n = _spread(rng, 1, 32_768)
        slots = min(rng.choice([1, 1, 2, 4]), groups)
        if op == "rows":
            c = _rows(_spread(rng, 1, 6_000_000), _spread(rng, 1, 4096), dropped=dropped)
        elif op == "product":
            transposed = rng.random() < 0.35
            c = _product(n, groups, k, l, dtype, slots=1 if transposed else slots, dropped=dropped, transposed=transposed,
                         gate=transposed and rng.random() < 0.5, bias=not transposed and rng.random() < 0.5,
                         relu=not transposed and rng.random() < 0.5, x_grouped=transposed and rng.random() < 0.5,
                         y_grouped=rng.random() < 0.5)
        elif op == "gradient":
            c = _gradient(n, groups, k, l, dtype, slots=slots, dropped=dropped, bias=rng.random() < 0.5,
                          out="f32" if rng.random() < 0.5 else dtype, y_grouped=rng.random() < 0.5)
        else:
            c = _adapter(n, min(n, _spread(rng, 1, 256)), groups, k, l, _spread(rng, 1, 64), dtype, dropped=dropped, bias=rng.random() < 0.5)
        if not _too_much(c):
            return c


def _normal(gen, dtype, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * scale).to(TYPES[dtype])


def _group(keys, groups):
    """(offsets, order) of a column of keys: the rows of group 0, 1, ..., then those without a group."""
    keys = keys.long()
    place = torch.where((keys >= 0) & (keys < groups), keys, groups)
    order = torch.sort(place, stable=True)
    offsets = torch.searchsorted(order.values, torch.arange(groups + 1, device=DEV))
    return offsets.to(torch.int32), order.indices.to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, groups, n = case["op"], case["groups"], case["n"]
    state = {"case": dict(case)}
    # ragged groups: their shares are exponential random numbers, and the last of several groups is empty
    share = -torch.log(torch.rand(groups, generator=gen, device=DEV).clamp_min(1e-6))
    if groups > 2:
        share[groups - 1] = 0
    if op == "adapter":
        cuts = torch.sort(torch.randint(1, max(n, 2), (case["requests"] - 1,), generator=gen, device=DEV)).values
        if case["requests"] == n:
            cuts = torch.arange(1, n, device=DEV)
        request = torch.searchsorted(cuts, torch.arange(n, device=DEV), right=True)
        keys = torch.multinomial(share.clamp_min(1e-6), case["requests"], replacement=True, generator=gen)[request]
        off = (torch.rand(case["requests"], generator=gen, device=DEV) < case["dropped"])[request]
    elif op == "product" or op == "gradient":
        slots = case["slots"]
        if slots > 1:
            keys = torch.topk(torch.log(share.clamp_min(1e-9)) - torch.log(-torch.log(torch.rand((n, groups), generator=gen, device=DEV).clamp(1e-6, 1 - 1e-6))), slots).indices.reshape(-1)
        else:
            keys = torch.multinomial(share.clamp_min(1e-9), n, replacement=True, generator=gen)
        off = torch.rand(n * slots, generator=gen, device=DEV) < case["dropped"]
    else:
        keys = torch.bucketize(torch.rand(n, generator=gen, device=DEV), torch.cumsum(share.clamp_min(1e-9) / share.clamp_min(1e-9).sum(), 0)).clamp_max(groups - 1)
        off = torch.rand(n, generator=gen, device=DEV) < case["dropped"]
    state["keys"] = torch.where(off, -1, keys).to(torch.int32)
    if op == "rows":
        return state
    # a program keeps the grouping of its batch for all layers, forward and backward
    state["offsets"], state["order"] = _group(state["keys"], groups)
    state["most"] = int((state["offsets"][1:] - state["offsets"][:-1]).max())
    k, l, dt = case["k"], case["l"], case["dtype"]
    rows = n * case.get("slots", 1)
    if op == "product":
        state["W"] = _normal(gen, dt, groups, k, l, scale=k ** -0.5)
        state["bias"] = _normal(gen, dt, groups, l) if case["bias"] else None
        state["X"] = _normal(gen, dt, n, l if case["transposed"] else k)
        state["gate"] = _normal(gen, dt, rows, k).clamp_min_(0) if case["gate"] else None
    elif op == "gradient":
        state["X"] = _normal(gen, dt, n, k).clamp_min_(0)
        state["dY"] = _normal(gen, dt, rows, l, scale=0.1)
    else:
        state["X"] = _normal(gen, dt, n, k)
        state["W"] = _normal(gen, dt, k, l, scale=k ** -0.5)
        state["A"] = _normal(gen, dt, groups, k, case["r"], scale=k ** -0.5)
        state["B"] = _normal(gen, dt, groups, case["r"], l, scale=case["r"] ** -0.5)
        state["scale"] = torch.rand(groups, generator=gen, device=DEV) + 0.5
        state["bias"] = _normal(gen, dt, l) if case["bias"] else None
    return state


# ---------------------------------------------------------------- plain forms

def _places(s):
    """Group and place within it of every position of the order, one group more for the rows without one."""
    groups, n = s["case"]["groups"], s["order"].numel()
    p = torch.arange(n, device=DEV)
    off = s["offsets"].long()
    g = torch.searchsorted(off[1:].contiguous(), p, right=True)
    return g, p - off[g], p < off[groups]


def _padded(s, rows):
    """fp32 rows in the order of the groups as a [groups x longest group x width] stack, zeros behind the short ones."""
    g, at, inside = _places(s)
    out = torch.zeros((s["case"]["groups"] + 1, max(s["most"], 1), rows.shape[1]), device=DEV)
    out[torch.where(inside, g, s["case"]["groups"]), torch.where(inside, at, 0)] = rows
    return out[:-1]


def _unpadded(s, stack):
    """The reverse: rows in the order of the groups, zeros for those without a group."""
    g, at, inside = _places(s)
    return torch.where(inside[:, None], stack[g.clamp_max(s["case"]["groups"] - 1), torch.where(inside, at, 0)], 0)


def _plain_rows(s):
    return _group(s["keys"], s["case"]["groups"])


def _plain_product(s):
    c, order = s["case"], s["order"].long()
    X, W = s["X"].float(), s["W"].float()
    rows = X if c["x_grouped"] else X[order // c["slots"]]
    Y = torch.bmm(_padded(s, rows), W.transpose(1, 2).contiguous() if c["transposed"] else W)
    if s["bias"] is not None:
        Y = Y + s["bias"].float()[:, None, :]
    if c["relu"]:
        Y = Y.clamp_min(0)
    Y = _unpadded(s, Y)
    if not c["y_grouped"]:
        Y = torch.empty_like(Y).index_copy_(0, order, Y)
    if s["gate"] is not None:
        Y = torch.where(s["gate"] > 0, Y, 0)
    return Y.to(s["X"].dtype)


def _plain_gradient(s):
    c, order = s["case"], s["order"].long()
    X = s["X"].float()
    dY = s["dY"].float()
    X = _padded(s, X if c["x_grouped"] else X[order // c["slots"]])
    dY = _padded(s, dY if c["y_grouped"] else dY[order])
    dW = torch.bmm(X.transpose(1, 2).contiguous(), dY).to(TYPES[c["out"]])
    return [dW, dY.sum(1).to(TYPES[c["out"]])] if c["bias"] else [dW]


def _plain_adapter(s):
    order, X = s["order"].long(), s["X"].float()
    U = torch.bmm(_padded(s, X[order]), s["A"].float()) * s["scale"][:, None, None]
    low = _unpadded(s, torch.bmm(U, s["B"].float()))
    Y = X @ s["W"].float() + torch.empty_like(low).index_copy_(0, order, low)
    if s["bias"] is not None:
        Y = Y + s["bias"].float()
    return Y.to(s["X"].dtype)


# ---------------------------------------------------------------- the framework's calls

def _own(s):
    import paper_2306_08367_amd as lq
    c = s["case"]
    if c["op"] == "rows":
        return lq.lq_group_rows(s["keys"], c["groups"])
    if c["op"] == "product":
        return lq.lq_grouped_product(s["X"], s["W"], s["offsets"], s["order"], bias=s["bias"], gate=s["gate"], transposed=c["transposed"],
                                     relu=c["relu"], x_grouped=c["x_grouped"], y_grouped=c["y_grouped"], x_slots=c["slots"])
    if c["op"] == "gradient":
        dW, db = lq.lq_grouped_gradient(s["X"], s["dY"], s["offsets"], s["order"], dw_dtype=TYPES[c["out"]], want_bias=c["bias"],
                                        x_grouped=c["x_grouped"], y_grouped=c["y_grouped"], x_slots=c["slots"])
        return [dW, db] if c["bias"] else [dW]
    return lq.lq_adapter_product(s["X"], s["W"], s["A"], s["B"], s["offsets"], s["order"], scale=s["scale"], bias=s["bias"])


def run(state):
    if own:
        return _own(state)
    return {"rows": _plain_rows, "product": _plain_product, "gradient": _plain_gradient, "adapter": _plain_adapter}[state["case"]["op"]](state)


def work(case):
    if case["op"] == "rows":
        return {"bytes": 8 * case["n"] + 4 * (case["groups"] + 1), "flops": 0}
    size = 2 if case["dtype"] == "bf16" else 4
    n, groups, k, l = case["n"], case["groups"], case["k"], case["l"]
    rows = n * case.get("slots", 1)
    # (of a few rows, only the groups that have some are read)
    busy = min(groups, rows)
    index = 4 * (rows + groups + 1)
    if case["op"] == "product":
        wide, out = (l, k) if case["transposed"] else (k, l)
        elements = n * wide + busy * k * l + rows * out * (2 if case["gate"] else 1) + (busy * l if case["bias"] else 0)
        return {"bytes": size * elements + index, "flops": 2 * rows * k * l}
    if case["op"] == "gradient":
        out = 4 if case["out"] == "f32" else 2
        return {"bytes": size * (n * k + rows * l) + out * groups * (k + (1 if case["bias"] else 0)) * l + index,
                "flops": 2 * rows * k * l + (rows * l if case["bias"] else 0)}
    r, busy = case["r"], min(groups, case["requests"])
    return {"bytes": size * (n * (k + l) + k * l + busy * r * (k + l) + (l if case["bias"] else 0)) + index + 4 * groups,
            "flops": 2 * n * (k * l + r * (k + l))}


def exact(case, seed):
    s = prepare(case, seed)
    groups = case["groups"]
    if case["op"] == "rows":
        keys = s["keys"].cpu().numpy()
        of = [np.flatnonzero(keys == g) for g in range(groups)] if groups * keys.size < 5e8 else None
        if of is None:
            # (many groups over many keys: the pairs key * n + row sorted as single numbers)
            pairs = np.sort(np.where(keys < 0, groups, keys).astype(np.int64) * keys.size + np.arange(keys.size))
            order, group = pairs % keys.size, pairs // keys.size
            offsets = np.concatenate([[0], np.cumsum(np.bincount(group, minlength=groups + 1)[:groups])])
        else:
            order = np.concatenate(of + [np.flatnonzero(keys < 0)])
            offsets = np.concatenate([[0], np.cumsum([len(o) for o in of])])
        return torch.from_numpy(offsets.astype(np.int32)), torch.from_numpy(order.astype(np.int32))
    off, order = s["offsets"].tolist(), s["order"].long()
    of = [order[off[g]:off[g + 1]] for g in range(groups)]            # the rows of each group
    at = [torch.arange(off[g], off[g + 1], device=DEV) for g in range(groups)]   # and their positions
    if case["op"] == "product":
        Y = torch.zeros((order.numel(), case["k"] if case["transposed"] else case["l"]), dtype=torch.float64, device=DEV)
        for g in range(groups):
            X = s["X"][at[g] if case["x_grouped"] else torch.div(of[g], case["slots"], rounding_mode="floor")].double()
            W = s["W"][g].double()
            y = X @ (W.T.contiguous() if case["transposed"] else W)
            if case["bias"]:
                y += s["bias"][g].double()
            Y[at[g] if case["y_grouped"] else of[g]] = torch.relu(y) if case["relu"] else y
        return Y * (s["gate"] > 0) if case["gate"] else Y
    if case["op"] == "gradient":
        dW, db = [], []
        for g in range(groups):
            X = s["X"][at[g] if case["x_grouped"] else torch.div(of[g], case["slots"], rounding_mode="floor")].double()
            dY = s["dY"][at[g] if case["y_grouped"] else of[g]].double()
            dW.append(X.T.contiguous() @ dY)
            db.append(dY.sum(0))
        return [torch.stack(dW), torch.stack(db)] if case["bias"] else [torch.stack(dW)]
    Y = s["X"].double() @ s["W"].double()
    if case["bias"]:
        Y += s["bias"].double()
    for g in range(groups):
        Y[of[g]] += s["scale"][g].double() * ((s["X"][of[g]].double() @ s["A"][g].double()) @ s["B"][g].double())
    return Y
