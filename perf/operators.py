"""Rows by index: lookups, expert order and weighted sums with their gradients, as programs use them, with the work they cannot do without.

Each case is one pass through the public calls of ``paper_2511_10442_amd.binding`` or, where ``own`` is false, the same
result in elementary torch operations.

``op``
    lookup           rows of a table by token, scaled
    lookup_grad      the table's gradient: tokens sorted, rows of one token summed
    dispatch         choices of experts sorted, every token's row copied to its places in that order
    combine          the experts' rows back to their tokens, weighted and summed
    combine_grad     the gradients of those rows and weights
    neighbours       every point's weighted sum over the features of its neighbours in a graph
    neighbours_grad  the gradients of features (which many points share) and weights
``drop``: share of the indices that name nothing (padding, tokens over an expert's capacity, neighbours that a small split lacks).
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_MOST_BYTES = 2_000_000_000     # work of the largest drawn case, below that of the largest listed one
_MOST_PRODUCT = 600_000_000     # values of the plain form's largest intermediate


def listed():
    return [
        # one step of serving: the tokens of 64 sequences, a large vocabulary; latency is all there is
        _rows("lookup_64_bf16", "lookup", 64, 131072, 4096, "bf16"),
        # a training batch's embedding: frequent tokens come again and again, a few places are padding
        _rows("lookup_64k_bf16", "lookup", 65536, 131072, 2048, "bf16", drop=0.03),
        # that batch's gradient, kept in 32 bits for the optimiser; the commonest token comes some four thousand times
        _rows("lookup_grad_64k_bf16", "lookup_grad", 65536, 131072, 2048, "bf16", drop=0.03),
        # a small model's embedding with a width that is no multiple of anything
        _rows("lookup_grad_1k_f32", "lookup_grad", 1000, 5003, 257, "f32"),
        # one step of serving a mixture of experts
        _experts("dispatch_32_bf16", "dispatch", 32, 8, 128, 4096, "bf16"),
        # a training batch of it
        _experts("dispatch_32k_bf16", "dispatch", 32768, 8, 64, 2048, "bf16"),
        # the way back, when serving and in training
        _experts("combine_32_bf16", "combine", 32, 8, 128, 4096, "bf16"),
        _experts("combine_32k_bf16", "combine", 32768, 8, 64, 2048, "bf16"),
        # messages along a graph of 200,000 points, 40 neighbours each
        _graph("neighbours_200k_k40_f32", "neighbours", 200000, 40, 64, "f32", drop=0.01),
        # gradients of the way back, in training; and of a small ragged one whose experts turn some tokens away
        _experts("combine_grad_32k_bf16", "combine_grad", 32768, 8, 64, 2048, "bf16"),
        _experts("combine_grad_4k_f16", "combine_grad", 4099, 3, 10, 1000, "f16", drop=0.1),
        # gradients of messages along a graph of two clouds of 50,000 points
        _graph("neighbours_grad_100k_k40_f32", "neighbours_grad", 100000, 40, 64, "f32"),
    ]


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "lookup_grad", "dispatch", "combine", "combine_grad", "neighbours", "neighbours_grad"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    drop = rng.choice([0.0, 0.0, 0.03, 0.2])
    while True:
        if op.startswith("lookup"):
            c = _width(rng, 32, 8192)
            case = _rows(None, op, _log_int(rng, 1, 131072), _log_int(rng, 2, 200000), c, kind, drop)
        elif op.startswith("neighbours"):
            case = _graph(None, op, _log_int(rng, 500, 400000), _log_int(rng, 4, 64), _width(rng, 8, 128), kind, drop)
        else:
            k = rng.choice([1, 2, 2, 3, 4, 6, 8, 8])
            case = _experts(None, op, _log_int(rng, 1, 65536), k, max(k, _log_int(rng, 4, 512)), _width(rng, 64, 8192), kind, drop)
        if work(case)["bytes"] <= _MOST_BYTES and case["m"] * case["c"] <= _MOST_PRODUCT:
            return case


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    c = _log_int(rng, lo, hi)
    return c if rng.random() < 0.3 else max(8, c // 8 * 8)


def _case(name, **case):
    return dict(case, name=name) if name else case


def _rows(name, op, m, rows, c, kind, drop=0.0):
    return _case(name, op=op, m=m, rows=rows, c=c, kind=kind, drop=drop)


def _experts(name, op, tokens, k, experts, c, kind, drop=0.0):
    return _case(name, op=op, tokens=tokens, k=k, experts=experts, c=c, kind=kind, drop=drop, m=tokens * k)


def _graph(name, op, points, k, c, kind, drop=0.0):
    return _case(name, op=op, tokens=points, k=k, c=c, kind=kind, drop=drop, m=points * k)


def work(case):
    op, m, c = case["op"], case["m"], case["c"]
    size = 4 if case["kind"] == "f32" else 2
    row = float(c * size)
    kept = m * (1 - case["drop"])
    if op == "lookup":
        # a row that is named twice is read once
        v = np.arange(1, case["rows"] + 1)
        p = np.log1p(1.0 / v) / math.log(case["rows"] + 1)
        named = float(-np.expm1(kept * np.log1p(-p)).sum())
        return {"bytes": 4.0 * m + named * row + m * row, "flops": float(m) * c}
    if op == "lookup_grad":
        return {"bytes": 4.0 * m + kept * row + 4.0 * case["rows"] * c, "flops": kept * c}
    t = case["tokens"]
    if op == "dispatch":
        return {"bytes": 4.0 * m + t * row + kept * row + 8.0 * m + 4.0 * case["experts"], "flops": 0.0}
    if op == "combine":
        return {"bytes": 8.0 * m + kept * row + t * row, "flops": 2.0 * kept * c}
    if op == "combine_grad":
        return {"bytes": 8.0 * m + t * row + 2 * kept * row + 4.0 * m, "flops": 3.0 * kept * c}
    if op == "neighbours":
        return {"bytes": 8.0 * m + 2 * t * row, "flops": 2.0 * kept * c}
    return {"bytes": 8.0 * m + 3 * t * row + 4.0 * m, "flops": 4.0 * kept * c}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    op, m, c, kind = case["op"], case["m"], case["c"], _TYPES[case["kind"]]
    s = {"case": case}

    def normal(*shape):
        x = torch.empty(shape, dtype=kind, device="cuda")
        return x.normal_(generator=g)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    if op in ("lookup", "lookup_grad"):
        rows = case["rows"]
        # the n-th commonest token comes 1/n times as often as the commonest; which token that is, is left to chance
        rank = torch.floor((rows + 1.0) ** uniform(m).double()).long().sub(1).clamp(0, rows - 1)
        names = torch.randperm(rows, generator=g, device="cuda")
        index = names[rank]
        s["index"] = torch.where(uniform(m) < case["drop"], -1, index).int()
        s["scale"] = math.sqrt(c)
        if op == "lookup":
            s["table"] = normal(rows, c) * 0.02
        else:
            s["grad"] = normal(m, c) * 0.01
            s["rows"] = rows
        return s
    t, k = case["tokens"], case["k"]
    if op.startswith("neighbours"):
        # points come in no order; in one that follows their places a point's neighbours are near it
        names = torch.randperm(t, generator=g, device="cuda")
        at = torch.arange(t, device="cuda")
        reach = max(1, min(2 * k, t // 2))
        near = (at[:, None] + (uniform(t, k) * (2 * reach + 1)).long() - reach) % t
        near[:, 0] = at
        index = torch.empty((t, k), dtype=torch.long, device="cuda")
        index[names] = names[near]
        s["index"] = torch.where(uniform(t, k) < case["drop"], -1, index).int()
        s["weights"] = torch.exp(-4.0 * uniform(t, k))
        s["rows"] = normal(t, c)
        s["grad"] = normal(t, c) if op == "neighbours_grad" else None
        return s
    e = case["experts"]
    # a router's scores: some experts are liked better
    scores = torch.randn((t, e), generator=g, device="cuda") + torch.randn((e,), generator=g, device="cuda") * 0.7
    top, experts = torch.topk(scores, k, dim=1)
    s["index"] = torch.where(uniform(t, k) < case["drop"], -1, experts).int()
    s["experts"] = e
    if op == "dispatch":
        s["x"] = normal(t, c)
        s["out"] = torch.zeros((m, c), dtype=kind, device="cuda")
        return s
    s["weights"] = torch.softmax(top, dim=1)
    flat = torch.where(s["index"].reshape(-1) < 0, e, s["index"].reshape(-1))
    place = torch.empty(m, dtype=torch.int32, device="cuda")
    place[torch.sort(flat, stable=True)[1]] = torch.arange(m, dtype=torch.int32, device="cuda")
    s["place"] = torch.where(flat.reshape(t, k) == e, -1, place.reshape(t, k)).contiguous()
    s["rows"] = normal(m, c)
    if op == "combine_grad":
        s["grad"] = normal(t, c)
        s["grad_rows"] = torch.zeros((m, c), dtype=kind, device="cuda")      # rows that no token names stay as they are
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    from paper_2511_10442_amd import binding as fg
    op = s["case"]["op"]
    if op == "lookup":
        return fg.fg_lookup(s["table"], s["index"], s["scale"])
    if op == "lookup_grad":
        by = fg.fg_index_sort(s["index"], s["rows"], place=False)
        return fg.fg_lookup_backward(s["grad"], by, s["scale"], dtype=torch.float32)
    if op == "dispatch":
        by = fg.fg_index_sort(s["index"], s["experts"])
        return by.order, by.bounds, by.place, fg.fg_dispatch(s["x"], by.place, s["out"])
    if op == "combine":
        return fg.fg_combine(s["rows"], s["place"], s["weights"])
    if op == "combine_grad":
        return fg.fg_combine_backward(s["grad"], s["rows"], s["place"], s["weights"], grad_rows=s["grad_rows"])
    if op == "neighbours":
        return fg.fg_combine(s["rows"], s["index"], s["weights"])
    by = fg.fg_index_sort(s["index"], s["rows"].shape[0], place=False)
    return fg.fg_combine_backward(s["grad"], s["rows"], s["index"], s["weights"], sort=by)


def _plain(s):
    op, kind = s["case"]["op"], _TYPES[s["case"]["kind"]]
    index = s["index"]
    if op == "lookup":
        out = s["table"][index.clamp(min=0)].float() * s["scale"]
        return torch.where((index >= 0)[:, None], out, 0.0).to(kind)
    if op == "lookup_grad":
        # (padding goes to a row of its own behind the table)
        to = torch.where(index < 0, s["rows"], index)
        out = torch.zeros((s["rows"] + 1, s["case"]["c"]), device="cuda").index_add_(0, to, s["grad"].float())
        return out[:-1] * s["scale"]
    if op == "dispatch":
        t, k = index.shape
        flat = index.reshape(-1)
        _, order = torch.sort(torch.where(flat < 0, s["experts"], flat), stable=True)
        bounds = torch.cat([flat.new_zeros(1), (flat[:, None] == torch.arange(s["experts"], device="cuda")).sum(0).cumsum(0).int()])
        place = torch.empty_like(flat)
        place[order] = torch.arange(t * k, dtype=torch.int32, device="cuda")
        place = torch.where(flat < 0, -1, place)
        # places of choices that name no expert are at the end: their rows are written there once more as they are
        token = torch.where((torch.arange(t * k, device="cuda") < bounds[-1])[:, None], s["x"][order // k], s["out"])
        s["out"].copy_(token)
        return order.int(), bounds, place.reshape(t, k), s["out"]
    by = s["place"] if op.startswith("combine") else index
    named = by >= 0
    weights = torch.where(named, s["weights"], 0.0)
    at = by.clamp(min=0)
    if op in ("combine", "neighbours"):
        return (s["rows"][at].float() * weights[:, :, None]).sum(1).to(kind)
    grad = s["grad"].float()
    grad_weights = torch.where(named, (s["rows"][at].float() * grad[:, None, :]).sum(2), 0.0)
    parts = (grad[:, None, :] * weights[:, :, None]).reshape(-1, grad.shape[1])
    n = s["rows"].shape[0]
    to = torch.where(named, by, n).reshape(-1)
    grad_rows = torch.zeros((n + 1, grad.shape[1]), device="cuda").index_add_(0, to, parts)[:n].to(kind)
    if op == "combine_grad":
        s["grad_rows"].copy_(grad_rows)
        grad_rows = s["grad_rows"]
    return grad_rows, grad_weights


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    index = s["index"].long()
    if op == "lookup":
        out = torch.zeros((case["m"], case["c"]), dtype=torch.float64, device="cuda")
        for at in torch.nonzero(index >= 0)[:, 0].split(16384):
            out[at] = s["table"][index[at]].double().mul_(s["scale"])
        return out
    if op == "lookup_grad":
        return _summed(index, s["grad"], None, s["rows"]) * s["scale"]
    if op == "dispatch":
        flat = index.reshape(-1).cpu().numpy()
        k = case["k"]
        order = np.concatenate([np.flatnonzero(flat == e) for e in range(s["experts"])] + [np.flatnonzero(flat < 0)])
        kept = int((flat >= 0).sum())
        place = np.full(flat.size, -1)
        place[order[:kept]] = np.arange(kept)
        bounds = [int(((flat >= 0) & (flat < e)).sum()) for e in range(s["experts"] + 1)]
        out = torch.zeros((case["m"], case["c"]), dtype=torch.float64, device="cuda")
        out[:kept] = s["x"].double()[torch.from_numpy(order[:kept] // k).cuda()]
        return torch.from_numpy(order), torch.tensor(bounds), torch.from_numpy(place.reshape(-1, k)), out
    by = (s["place"] if op.startswith("combine") else s["index"]).long()
    weights, rows = s["weights"].double(), s["rows"].double()
    if op in ("combine", "neighbours"):
        out = torch.zeros((case["tokens"], case["c"]), dtype=torch.float64, device="cuda")
        for j in range(case["k"]):
            t = torch.nonzero(by[:, j] >= 0)[:, 0]
            out[t] += weights[t, j, None] * rows[by[t, j]]
        return out
    grad = s["grad"].double()
    grad_weights = torch.zeros_like(weights)
    for j in range(case["k"]):
        t = torch.nonzero(by[:, j] >= 0)[:, 0]
        grad_weights[t, j] = torch.linalg.vecdot(grad[t], rows[by[t, j]])
    return _summed(by.reshape(-1), grad, weights.reshape(-1), rows.shape[0]), grad_weights


def _summed(index, grad, weights, rows):
    """Rows of `grad` (one for every len(index) / len(grad) indices) summed by index: the first of every row, then the second, and so on."""
    order = torch.sort(index, stable=True)[1]
    order = order[index[order] >= 0]
    name = index[order]
    first = torch.searchsorted(name, name, right=False)
    nth = torch.arange(name.numel(), device="cuda") - first
    out = torch.zeros((rows, grad.shape[1]), dtype=torch.float64, device="cuda")
    fan = index.numel() // grad.shape[0]
    by_turn = torch.sort(nth, stable=True)[1]
    for turn in by_turn.split(torch.bincount(nth).tolist()):
        part = grad[order[turn] // fan].double()
        out[name[turn]] += part if weights is None else part * weights[order[turn], None]
    return out
