"""Products routed by a sparse factor, as measurable cases: R is a CSR matrix (rows x columns, e.g. tokens x experts) whose
entries pick blocks of a dense factor, where an entry of A in C = A * B picks a row of B.

Kinds
  product        the entries sorted by column, then a row P[p] = X[row] W[column]^T for each entry: what a layer does first
  train          the same with both gradients: dX (summed over a row's entries) and dW (summed over a column's)
  sum            the entries sorted by column, then Y[i] = sum of r * P over the entries of row i: what a layer does last
  sum_grads      its gradients: dP, and those of R's values
  product_8bit   rows of X quantised to e4m3 with a scale for each 1 x 128, times e4m3 blocks with a scale for each 128 x 128 (or 1 x 128)
  quantize       blocks of weights, or rows, to e4m3 with a scale for each 128 x 128 or 1 x 128

`skew` is the exponent of the columns' popularity (0: all alike), `keep` the share of a row's `k` entries that are there (rows
without any occur), `drop` the share of entries that are routed nowhere (column -1).
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
LARGEST = {"bytes": 2.0e9, "flops": 9.0e11}  # of a drawn case


def listed():
    return [
        # one row: a single token is generated, nothing but latency and the weights of eight columns
        {"name": "product 1 row", "kind": "product", "n": 1, "k": 8, "E": 64, "K": 2048, "N": 1024, "dtype": "bf16", "skew": 0.0, "keep": 1.0, "drop": 0.0},
        # a step of a server with a batch of rows: all columns are in use, few rows each, their weights bound it
        {"name": "product 129 rows", "kind": "product", "n": 129, "k": 8, "E": 128, "K": 4096, "N": 1536, "dtype": "bf16", "skew": 0.5, "keep": 1.0, "drop": 0.0},
        # a prompt, or a training step's forward pass: matrix products of ragged sizes
        {"name": "product 4096 rows", "kind": "product", "n": 4096, "k": 8, "E": 64, "K": 2048, "N": 2048, "dtype": "bf16", "skew": 0.7, "keep": 1.0, "drop": 0.0},
        # ragged in every direction: rows with some or none of their entries, some routed nowhere, an odd width
        {"name": "product ragged f16", "kind": "product", "n": 777, "k": 4, "E": 19, "K": 1000, "N": 1237, "dtype": "f16", "skew": 1.0, "keep": 0.7, "drop": 0.1},
        # a training step: the product and both gradients, few large columns
        {"name": "train 8192 rows", "kind": "train", "n": 8192, "k": 2, "E": 8, "K": 2048, "N": 4096, "dtype": "bf16", "skew": 0.3, "keep": 1.0, "drop": 0.0},
        # a smaller one in the other type, many columns, popularity skewed
        {"name": "train 2047 rows f16", "kind": "train", "n": 2047, "k": 4, "E": 32, "K": 1024, "N": 1408, "dtype": "f16", "skew": 1.0, "keep": 1.0, "drop": 0.0},
        # the end of a layer, a step of a server
        {"name": "sum 128 rows", "kind": "sum", "n": 128, "k": 8, "E": 128, "N": 4096, "dtype": "bf16", "skew": 0.5, "keep": 1.0, "drop": 0.0},
        # the end of a layer for a long prompt, and its gradients
        {"name": "sum 16384 rows", "kind": "sum", "n": 16384, "k": 8, "E": 64, "N": 2048, "dtype": "bf16", "skew": 0.7, "keep": 1.0, "drop": 0.0},
        {"name": "sum grads 8191 rows", "kind": "sum_grads", "n": 8191, "k": 6, "E": 64, "N": 2880, "dtype": "bf16", "skew": 0.7, "keep": 0.9, "drop": 0.05},
        # the same layers served in 8 bits: a step of a server, and a prompt
        {"name": "8-bit product 64 rows", "kind": "product_8bit", "n": 64, "k": 8, "E": 128, "K": 4096, "N": 1536, "wrows": 128, "dtype": "bf16", "skew": 0.5, "keep": 1.0, "drop": 0.0},
        {"name": "8-bit product 4096 rows", "kind": "product_8bit", "n": 4096, "k": 8, "E": 64, "K": 4096, "N": 2048, "wrows": 128, "dtype": "bf16", "skew": 0.7, "keep": 1.0, "drop": 0.0},
        # weights that a step has changed, made ready for 8-bit products
        {"name": "quantize 16 blocks", "kind": "quantize", "E": 16, "N": 2048, "K": 4096, "wrows": 128, "dtype": "bf16"},
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["product", "product", "train", "sum", "sum_grads", "product_8bit", "product_8bit", "quantize"])
    case = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f16"])}
    if kind == "quantize":
        # activations (1 x 128) or weights (128 x 128)
        case |= {"E": log_int(1, 32), "N": log_int(1, 8192), "K": 8 * log_int(4, 768), "wrows": rng.choice([1, 128])}
    else:
        E = log_int(1, 160)
        case |= {"n": log_int(1, 16384), "k": rng.randint(1, min(E, 8)), "E": E, "N": log_int(64, 4096)}
        case |= {"skew": round(rng.uniform(0.0, 1.2), 3), "keep": rng.choice([1.0, 1.0, round(rng.uniform(0.5, 1.0), 3)]), "drop": rng.choice([0.0, 0.0, round(rng.uniform(0.0, 0.2), 3)])}
        if kind in ("product", "train"):
            case["K"] = 8 * log_int(8, 512) if rng.random() < 0.9 else log_int(64, 4096)  # most widths are multiples of eight
        if kind == "train" and rng.random() < 0.9:
            case["N"] = 8 * -(-case["N"] // 8)
        if kind == "product_8bit":
            case |= {"K": 16 * log_int(4, 256), "wrows": rng.choice([128, 128, 1])}
    size = "N" if kind == "quantize" else "n"
    while any(v > LARGEST[m] for m, v in work(case).items()) and case[size] > 1:
        case[size] = max(1, case[size] * 2 // 3)
    while any(v > LARGEST[m] for m, v in work(case).items()):
        case["E"] = max(case.get("k", 1), case["E"] * 2 // 3)
    return case


def work(case):
    if case["kind"] == "quantize":
        values = case["E"] * case["N"] * case["K"]
        scales = case["E"] * -(-case["N"] // case["wrows"]) * -(-case["K"] // 128)
        return {"bytes": 3.0 * values + 4.0 * scales, "flops": 2.0 * values}
    n, E, N = case["n"], case["E"], case["N"]
    entries = _entries(case)
    if case["kind"] == "sum":
        return {"bytes": 2 * entries * N + 2 * n * N + 16 * entries, "flops": 2 * entries * N}
    if case["kind"] == "sum_grads":
        return {"bytes": 4 * entries * N + 2 * n * N + 20 * entries, "flops": 3 * entries * N}
    K, used = case["K"], min(E, entries)
    if case["kind"] == "product":
        return {"bytes": 2 * (n * K + used * N * K + entries * N) + 12 * entries, "flops": 2 * entries * N * K}
    if case["kind"] == "train":
        return {"bytes": 2 * (2 * n * K + used * N * K + E * N * K + 2 * entries * N) + 12 * entries, "flops": 6 * entries * N * K}
    return {"bytes": 2 * n * K + used * N * K + 2 * entries * N + 12 * entries, "flops": 2 * entries * N * K}


# ---------------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------------
def _entries(case):
    return max(1, round(case["n"] * case["k"] * case["keep"]))


def _routing(case, g):
    """R as a router makes it: the k best columns of each row by noise on the columns' popularity, ascending, and the weights of a softmax."""
    n, k, E = case["n"], case["k"], case["E"]
    popularity = -case["skew"] * torch.log1p(torch.randperm(E, generator=g, device="cuda").float())
    noise = -torch.log(-torch.log(torch.rand(n, E, generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    score, col = torch.topk(popularity + noise, k, dim=1)
    col, at = torch.sort(col, dim=1)
    val = torch.softmax(score, dim=1).gather(1, at)
    there = torch.zeros(n * k, dtype=torch.bool, device="cuda")
    there[torch.randperm(n * k, generator=g, device="cuda")[: _entries(case)]] = True
    there = there.view(n, k)
    if case["drop"] > 0:
        col = torch.where(torch.rand(n, k, generator=g, device="cuda") < case["drop"], -1, col)
    row_ptr = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    row_ptr[1:] = torch.cumsum(there.sum(1), 0)
    col = col[there].to(torch.int32)
    most = int(torch.bincount(col[col >= 0].long(), minlength=1).max()) if col.numel() else 0
    return {"n": n, "E": E, "row_ptr": row_ptr, "col": col, "val": val[there].contiguous(), "most": max(1, most)}


def _normal(shape, g, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _spread(x, g):
    """Channels of different size, a few of them large: what quantisers meet."""
    size = torch.exp(0.7 * torch.randn(x.shape[-1], generator=g, device="cuda"))
    size *= torch.where(torch.rand(x.shape[-1], generator=g, device="cuda") < 0.01, 20.0, 1.0)
    return (x.float() * size).to(x.dtype)


def _ready_weights(w, rows):
    """Blocks in 8 bits as a server has loaded them."""
    E, N, K = w.shape
    q = torch.empty(E, N, K, dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.empty(E, -(-N // rows), -(-K // 128), device="cuda")
    for e in range(E):
        v = torch.nn.functional.pad(w[e].float(), (0, -K % 128, 0, -N % rows)).view(s.shape[1], rows, s.shape[2], 128)
        amax = v.abs().amax((1, 3)).clamp(min=2.0 ** -100)
        s[e] = amax / 448
        q[e] = (v / s[e][:, None, :, None]).clamp(-448, 448).view(s.shape[1] * rows, -1)[:N, :K].to(q.dtype)
    return q, s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype, state = TYPES[case["dtype"]], dict(case)
    if case["kind"] == "quantize":
        return state | {"x": _spread(_normal((case["E"], case["N"], case["K"]), g, dtype), g)}
    state["R"] = _routing(case, g)
    entries, N = state["R"]["col"].numel(), case["N"]
    if case["kind"] in ("sum", "sum_grads"):
        state["P"] = _normal((entries, N), g, dtype)
        if case["kind"] == "sum_grads":
            state["dY"] = _normal((case["n"], N), g, dtype)
        return state
    K = case["K"]
    state["X"] = _normal((case["n"], K), g, dtype)
    W = _normal((case["E"], N, K), g, dtype, K ** -0.5)
    if case["kind"] == "product_8bit":
        state["X"] = _spread(state["X"], g)
        state["Wq"], state["Ws"] = _ready_weights(W, case["wrows"])
    else:
        state["W"] = W
    if case["kind"] == "train":
        state["dP"] = _normal((entries, N), g, dtype)
    return state


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _route(R):
    """The entries in the order of their columns (stable), those that are routed nowhere last."""
    entries = R["col"].numel()
    row = torch.repeat_interleave(torch.arange(R["n"], device="cuda"), R["row_ptr"].diff(), output_size=entries)
    column = torch.where((R["col"] >= 0) & (R["col"] < R["E"]), R["col"], R["E"]).long()
    order = torch.argsort(column, stable=True)
    by_column = column[order]
    offsets = torch.searchsorted(by_column, torch.arange(R["E"] + 1, device="cuda"))
    pos = torch.empty_like(order)
    pos[order] = torch.arange(entries, device="cuda")
    # where a place lies in a batch of equally long columns; those routed nowhere share one behind it
    slot = by_column * R["most"] + torch.arange(entries, device="cuda") - offsets[by_column]
    slot = torch.where(by_column < R["E"], slot, R["E"] * R["most"])
    return {"row": row, "column": column, "order": order, "rows": row[order], "offsets": offsets, "pos": pos, "slot": slot, "E": R["E"], "most": R["most"], "n": R["n"]}


def _batched(t, rows):
    """Rows by place -> (E, most, width), zero where a column has fewer."""
    out = torch.zeros(t["E"] * t["most"] + 1, rows.shape[1], device="cuda")
    out[t["slot"]] = rows
    return out[:-1].view(t["E"], t["most"], -1)


def _placed(t, batch):
    flat = torch.cat([batch.reshape(t["E"] * t["most"], -1), torch.zeros(1, batch.shape[2], device="cuda")])
    return flat[t["slot"]]


def _blocks_of(x, rows):
    E, N, K = x.shape
    return torch.nn.functional.pad(x, (0, -K % 128, 0, -N % rows)).view(E, -(-N // rows), rows, -(-K // 128), 128)


def _quantized(x, rows):
    """(e4m3 values, scales) of (E, N, K): in 64 bits, so that values next to a border fall on their side of it."""
    v = _blocks_of(x.double(), rows)
    s = v.abs().amax((2, 4)).clamp(min=2.0 ** -100) / 448
    q = (v / s[:, :, None, :, None]).float().to(torch.float8_e4m3fn)
    q = q.view(v.shape[0], v.shape[1] * rows, -1)[:, : x.shape[1], : x.shape[2]].contiguous()
    return q, s.float()


def _values(q, s, rows):
    v = _blocks_of(q.float(), rows) * s[:, :, None, :, None]
    return v.view(v.shape[0], v.shape[1] * rows, -1)[:, : q.shape[1], : q.shape[2]]


def _run_plain(s):
    if s["kind"] == "quantize":
        return _quantized(s["x"], s["wrows"])
    t, dtype = _route(s["R"]), TYPES[s["dtype"]]
    if s["kind"] in ("sum", "sum_grads"):
        fits = t["column"] < t["E"]
        weight = torch.where(fits, s["R"]["val"], 0.0)[:, None]
        P = torch.where(fits[:, None], s["P"].float()[t["pos"]], 0.0)  # by entry
        if s["kind"] == "sum":
            return {"Y": torch.zeros(t["n"], s["N"], device="cuda").index_add_(0, t["row"], weight * P).to(dtype)}
        dY = s["dY"].float()[t["row"]]
        return {"dP": (weight * dY)[t["order"]].to(dtype), "dval": (dY * P).sum(1)}
    ints = {"offsets": t["offsets"], "rows": t["rows"].to(torch.int32)}
    if s["kind"] == "product_8bit":
        xq, xs = _quantized(s["X"][None], 1)
        X, W = _values(xq, xs, 1)[0], _values(s["Wq"], s["Ws"], s["wrows"])
    else:
        X, W = s["X"].float(), s["W"].float()
    X = _batched(t, X[t["rows"]])
    P = _placed(t, torch.bmm(X, W.transpose(1, 2))).to(dtype)
    if s["kind"] != "train":
        return ints | {"P": P}
    dP = _batched(t, s["dP"].float())
    dX = torch.zeros(t["n"], s["K"], device="cuda").index_add_(0, t["rows"], _placed(t, torch.bmm(dP, W)))
    return ints | {"P": P, "dX": dX.to(dtype), "dW": torch.bmm(dP.transpose(1, 2), X).to(dtype)}


def _run_own(s):
    import paper_2607_22866_b200 as gm

    if s["kind"] == "quantize":
        return gm.block_quantize(s["x"], s["wrows"])
    R = s["R"]
    route = gm.route_plan(gm.DeviceCSR(R["n"], R["E"], R["row_ptr"], R["col"], R["val"]))
    if s["kind"] == "sum":
        return {"Y": gm.route_sum(route, s["P"])}
    if s["kind"] == "sum_grads":
        dP, dval = gm.route_sum_grads(route, s["dY"], s["P"])
        return {"dP": dP, "dval": dval}
    ints = {"offsets": route.offsets, "rows": route.rows}
    if s["kind"] == "product_8bit":
        xq, xs = gm.block_quantize(s["X"], 1)
        return ints | {"P": gm.route_product_scaled(route, xq, xs, s["Wq"], s["Ws"], dtype=s["X"].dtype)}
    P = gm.route_product(route, s["X"], s["W"])
    if s["kind"] == "product":
        return ints | {"P": P}
    return ints | {"P": P, "dX": gm.route_product_dx(route, s["dP"], s["W"]), "dW": gm.route_product_dw(route, s["dP"], s["X"])}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _e4m3(y):
    """The nearest value of e4m3 (ties to the even one), |y| <= 448."""
    exponent = torch.frexp(y).exponent - 1
    step = torch.ldexp(torch.ones_like(y), exponent.clamp(min=-6) - 3)
    return torch.round(y / step) * step


def _exact_blocks(x, rows):
    E, N, K = x.shape
    q, s = torch.empty(E, N, K, dtype=torch.float64, device="cuda"), torch.empty(E, -(-N // rows), -(-K // 128), dtype=torch.float64, device="cuda")
    for b in range(s.shape[2]):
        part = x[:, :, 128 * b: 128 * b + 128].double()
        most = part.abs().amax(2)
        if rows > 1:
            most = torch.stack([c.amax(1) for c in most.split(rows, 1)], 1)
        most = most.clamp(min=2.0 ** -100)
        s[:, :, b] = most / 448
        q[:, :, 128 * b: 128 * b + 128] = _e4m3(part * 448 / most.repeat_interleave(rows, 1)[:, :N, None])
    return q, s


def _wide(s, K, rows, N):
    return s.repeat_interleave(128, -1)[..., :K] if rows == 1 else s.repeat_interleave(128, -1)[..., :K].repeat_interleave(rows, -2)[..., :N, :]


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quantize":
        return _exact_blocks(s["x"], case["wrows"])
    R, E, N = s["R"], case["E"], case["N"]
    entries = R["col"].numel()
    row = torch.searchsorted(R["row_ptr"], torch.arange(entries, device="cuda"), right=True) - 1
    places = [torch.nonzero(R["col"] == e).flatten() for e in range(E)]
    nowhere = torch.nonzero((R["col"] < 0) | (R["col"] >= E)).flatten()
    order = torch.cat(places + [nowhere])
    starts = [0]
    for p in places:
        starts.append(starts[-1] + p.numel())
    val = R["val"].double()
    if case["kind"] == "sum":
        Y = torch.zeros(case["n"], N, dtype=torch.float64, device="cuda")
        for e in range(E):  # (the rows of one column are distinct)
            Y[row[places[e]]] += val[places[e], None] * s["P"][starts[e]: starts[e + 1]].double()
        return {"Y": Y}
    if case["kind"] == "sum_grads":
        dP, dval = torch.zeros(entries, N, dtype=torch.float64, device="cuda"), torch.zeros(entries, dtype=torch.float64, device="cuda")
        for e in range(E):
            dY = s["dY"][row[places[e]]].double()
            dP[starts[e]: starts[e + 1]] = val[places[e], None] * dY
            dval[places[e]] = (dY * s["P"][starts[e]: starts[e + 1]].double()).sum(1)
        return {"dP": dP, "dval": dval}
    K = case["K"]
    if case["kind"] == "product_8bit":
        q, scale = _exact_blocks(s["X"][None], 1)
        X = (q * _wide(scale, K, 1, case["n"]))[0]
    else:
        X = s["X"].double()
    out = {"offsets": None, "rows": row[order].to(torch.int32), "P": torch.zeros(entries, N, dtype=torch.float64, device="cuda")}
    if case["kind"] == "train":
        out |= {"dX": torch.zeros(case["n"], K, dtype=torch.float64, device="cuda"), "dW": torch.zeros(E, N, K, dtype=torch.float64, device="cuda")}
    for e in range(E):
        x, a, b = X[row[places[e]]], starts[e], starts[e + 1]
        W = s["W"][e].double() if "W" in s else s["Wq"][e].double() * _wide(s["Ws"][e].double(), K, case["wrows"], N)
        out["P"][a:b] = x @ W.T
        if case["kind"] == "train":
            dP = s["dP"][a:b].double()
            out["dX"][row[places[e]]] += dP @ W
            out["dW"][e] = dP.T @ x
    return out
