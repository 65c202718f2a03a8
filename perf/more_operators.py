"""Performance cases of what brings tokens to weights of their own: routing, the exchange
between tokens and rows sorted by expert, and low-rank adapters.

The operators: the choice of experts from a router's logits with their weights, the number of
tokens that each got, the balance loss and its gradient; the order of (token, choice) slots by
expert, rows copied into that order and joined back by weight, with their gradients; low-rank
adapters, one for each request, beside a shared projection, with their gradients.

The ranges that the cases stand for: 1 to 16384 tokens, 4 to 512 experts of which a token takes
1 to 8, padded batches, rows of 128 to 8192 values, 1 to 128 adapters of rank 4 to 128 some of
which no request uses, requests without an adapter; fp16 and bf16, logits and outputs in 32 bits too.

Keys of a case: "op" ("route", "route_train", "dispatch", "combine", "exchange_back", "adapters",
"adapters_train"), "dtype", "m" tokens, "experts", "k" choices of a token, "renormalize", "padding"
(share of the tokens that are padding), "width" (values in a row), "n" and "k_in" (a projection's
outputs and inputs), "adapters", "idle" (adapters without a request), "requests", "bare" (requests
without an adapter), "rank", "out" (type of the projection's output, or of the gradients).
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
SIZES = {"fp16": 2, "bf16": 2, "fp32": 4}


def _route(name, op, dtype, m, experts, k, renormalize, padding):
    return {"name": name, "op": op, "dtype": dtype, "m": m, "experts": experts, "k": k,
            "renormalize": renormalize, "padding": padding}


def _exchange(name, op, dtype, m, experts, k, width, padding):
    return {"name": name, "op": op, "dtype": dtype, "m": m, "experts": experts, "k": k, "width": width,
            "padding": padding}


def _adapters(name, op, dtype, out, m, n, k_in, rank, adapters, idle, requests, bare):
    return {"name": name, "op": op, "dtype": dtype, "out": out, "m": m, "n": n, "k_in": k_in, "rank": rank,
            "adapters": adapters, "idle": idle, "requests": requests, "bare": bare}


def listed():
    return [
        # decode: the tokens of 17 requests choose two of 32 experts
        _route("route_17x32", "route", "fp32", 17, 32, 2, True, 0.0),
        # prefill: a padded batch in 16 bits, an odd number of experts
        _route("route_8191x61", "route", "bf16", 8191, 61, 4, False, 0.2),
        # a training step's routing: many small experts, choices, loss and gradient
        _route("route_train_16384x256", "route_train", "fp32", 16384, 256, 8, True, 0.0),
        # decode: 64 requests' hidden states, two rows each, to 32 experts
        _exchange("dispatch_64x4096", "dispatch", "bf16", 64, 32, 2, 4096, 0.0),
        # prefill: 8192 tokens, of a padded batch, in rows by expert
        _exchange("dispatch_8192x4096", "dispatch", "bf16", 8192, 16, 2, 4096, 0.1),
        # prefill: the experts' outputs back to their tokens, eight of 64 experts each
        _exchange("combine_8191x2048", "combine", "fp16", 8191, 64, 8, 2048, 0.0),
        # a training step's way back: gradients of the rows, of their weights and of the tokens
        _exchange("exchange_back_8192x4096", "exchange_back", "bf16", 8192, 8, 2, 4096, 0.0),
        # decode: one request with its adapter
        _adapters("adapters_1x4096x4096", "adapters", "bf16", "bf16", 1, 4096, 4096, 16, 1, 0, 1, 0),
        # decode: 64 requests with 29 of 32 adapters, five of them without one
        _adapters("adapters_64x4096x4096", "adapters", "bf16", "bf16", 64, 4096, 4096, 16, 32, 3, 64, 5),
        # prefill of six requests of any length, no size a multiple of anything, 32-bit outputs
        _adapters("adapters_1733x5003x4100", "adapters", "fp16", "fp32", 1733, 5003, 4100, 11, 4, 0, 6, 1),
        # prefill: long requests through a wide layer, larger adapters
        _adapters("adapters_16384x8192x4096", "adapters", "bf16", "bf16", 16384, 8192, 4096, 64, 7, 1, 12, 1),
        # a training step of four adapters at once, gradients in 32 bits for the optimizer
        _adapters("adapters_train_8191x4096x4096", "adapters_train", "bf16", "fp32", 8191, 4096, 4096, 16, 4, 0, 8, 0),
    ]


def _size(rng, low, high):
    """A size between `low` and `high`, even over its logarithm; half of them odd."""
    n = round(2.0 ** rng.uniform(math.log2(low), math.log2(high)))
    return n | 1 if rng.random() < 0.5 else n


def draw(rng):
    op = rng.choice(["route", "route_train", "dispatch", "combine", "exchange_back", "adapters", "adapters",
                     "adapters_train"])
    dtype = rng.choice(["fp16", "bf16"])
    padding = rng.choice([0.0, 0.0, 0.1, 0.4])
    if op.startswith("route"):
        experts = _size(rng, 4, 256)
        return {"op": op, "dtype": rng.choice([dtype, "fp32"]), "m": _size(rng, 1, 16383), "experts": experts,
                "k": rng.randint(1, min(8, experts)), "renormalize": rng.random() < 0.5, "padding": padding}
    if op in ("dispatch", "combine", "exchange_back"):
        experts = _size(rng, 4, 256)
        k, width = rng.randint(1, min(8, experts)), _size(rng, 128, 8191)
        return {"op": op, "dtype": dtype, "m": _size(rng, 1, min(16383, (1 << 26) // (k * width))),
                "experts": experts, "k": k, "width": width, "padding": padding}
    adapters = _size(rng, 1, 127 if op == "adapters" else 8)
    idle = rng.randint(0, adapters // 4)
    n, k_in = _size(rng, 128, 8191), _size(rng, 128, 8191)
    rank = _size(rng, 4, 127)
    m = _size(rng, 1 if op == "adapters" else 64,
              min(8191, (1 << 28) // (n + k_in) // adapters,
                  (1 << 32) // (rank * (n + k_in)) * (2 if op == "adapters" else 1) * 7 // 8))
    requests = rng.randint(1, min(m, 2 * adapters))
    return {"op": op, "dtype": dtype, "out": rng.choice([dtype, "fp32"]), "m": m, "n": n, "k_in": k_in,
            "rank": rank, "adapters": adapters, "idle": idle, "requests": requests,
            "bare": rng.randint(0, requests // 4)}


# ---- inputs -------------------------------------------------------------------


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _hidden(gen, m, width, dtype):
    """N(0, 1) rows with 16 columns x50, as hidden states have them."""
    v = _normal(gen, m, width)
    v[:, torch.randperm(width, generator=gen, device="cuda")[:16]] *= 50
    return v.to(DTYPES[dtype])


def _valid(case, gen):
    """Which tokens of a padded batch are none of its padding."""
    valid = torch.rand(case["m"], generator=gen, device="cuda") >= case["padding"]
    valid[0] = True
    return valid


def _logits(case, gen):
    """Logits of a router that likes some experts more."""
    return (_normal(gen, case["m"], case["experts"]) + 0.5 * _normal(gen, case["experts"])).to(DTYPES[case["dtype"]])


def _choices(case, gen):
    """Different experts for each token, in no order; padding takes none (-1)."""
    likes = _normal(gen, case["m"], case["experts"]) + 0.5 * _normal(gen, case["experts"])
    ids = likes.argsort(dim=1)[:, : case["k"]].to(torch.int32)
    if case["padding"]:
        ids = torch.where(_valid(case, gen)[:, None], ids, -1)
    return ids.contiguous()


def _requests(case, gen):
    """The adapter of each token (-1: none): tokens of a request lie together, every adapter that is
    not idle has a request where there are enough."""
    m, requests = case["m"], case["requests"]
    cuts = torch.randperm(m - 1, generator=gen, device="cuda")[: requests - 1] + 1 if m > 1 else []
    request = torch.zeros(m, dtype=torch.int64, device="cuda")
    if len(cuts):
        request[cuts] = 1
    request = request.cumsum(0)
    live = torch.randperm(case["adapters"], generator=gen, device="cuda")[: case["adapters"] - case["idle"]]
    adapter = live[torch.arange(requests, device="cuda") % len(live)]
    order = torch.randperm(requests, generator=gen, device="cuda")
    adapter[requests - case["bare"]:] = -1
    return adapter[order][request].to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, m = case["op"], case["m"]
    state = {"op": op, "case": case}
    if op.startswith("route"):
        state["logits"] = _logits(case, gen)
        state["valid"] = _valid(case, gen) if case["padding"] else None
        if op == "route_train":
            state["dweights"] = _normal(gen, m, case["k"])
            state["dloss"] = torch.full((), 0.01, device="cuda")
    elif op in ("dispatch", "combine", "exchange_back"):
        state["ids"] = _choices(case, gen)
        rows, width = m * case["k"], case["width"]
        if op == "dispatch":
            state["x"] = _hidden(gen, m, width, case["dtype"])
        else:
            # what the grouping gave on the way out
            state["ends"], state["rows"], _ = _group(state["ids"], case["experts"])
            state["weights"] = torch.rand((m, case["k"]), generator=gen, device="cuda") / case["k"]
            state["y"] = _normal(gen, rows, width).to(DTYPES[case["dtype"]])
        if op == "exchange_back":
            state["dout"] = _normal(gen, m, width).to(DTYPES[case["dtype"]])
            state["dxs"] = _normal(gen, rows, width).to(DTYPES[case["dtype"]])
    else:
        k_in, n, rank, adapters = case["k_in"], case["n"], case["rank"], case["adapters"]
        dtype = DTYPES[case["dtype"]]
        state["x"] = _hidden(gen, m, k_in, case["dtype"])
        state["down"] = (_normal(gen, adapters, rank, k_in) / math.sqrt(k_in)).to(dtype)
        state["up"] = (0.1 * _normal(gen, adapters, rank, n)).to(dtype)
        state["scales"] = 0.5 + 1.5 * torch.rand(adapters, generator=gen, device="cuda")
        # the order of a step's tokens by adapter, which all its layers share
        ids = _requests(case, gen)
        state["ends"], _, state["slots"] = _group(ids[:, None], adapters)
        state["y"] = _normal(gen, m, n).to(DTYPES[case["out"]] if op == "adapters" else dtype)
        if op == "adapters_train":
            state["dout"] = _normal(gen, m, n).to(dtype)
        # what the plain form needs to know of the groups without asking the GPU
        state["most"] = int(torch.bincount(ids[ids >= 0], minlength=1).max())
    return state


# ---- plain forms --------------------------------------------------------------


def _group(ids, groups):
    """Ends of the groups, the place of each (token, choice) slot and the slot of each place;
    slots without a group come last and have no place (-1)."""
    flat = ids.reshape(-1).long()
    flat = torch.where((flat >= 0) & (flat < groups), flat, groups)
    slots = torch.sort(flat, stable=True).indices
    counts = (flat[:, None] == torch.arange(groups, device=ids.device)).sum(0)
    place = torch.empty_like(slots)
    place[slots] = torch.arange(len(slots), device=ids.device)
    rows = torch.where(flat < groups, place, -1).view(ids.shape)
    return counts.cumsum(0).to(torch.int32), rows.to(torch.int32), slots.to(torch.int32)


def _softmax(logits, valid):
    e = torch.exp(logits - logits.amax(dim=1, keepdim=True))
    p = e / e.sum(dim=1, keepdim=True)
    return p if valid is None else p * valid[:, None]


def _route_plain(state):
    case, valid = state["case"], state["valid"]
    m, experts, k = case["m"], case["experts"], case["k"]
    logits = state["logits"].float()
    p = _softmax(logits, valid)
    chosen = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    weights = p.gather(1, chosen)
    if case["renormalize"]:
        total = weights.sum(dim=1, keepdim=True)
        weights = weights / torch.where(total > 0, total, 1.0)
    if valid is not None:
        chosen = torch.where(valid[:, None], chosen, -1)
    flat = chosen.reshape(-1)
    counts = (flat[:, None] == torch.arange(experts, device="cuda")).sum(0)
    tokens = m if valid is None else valid.sum()
    slopes = counts * (experts / (k * tokens * tokens)) if valid is None else \
        counts * (experts / (k * tokens.double() * tokens)).float()
    loss = (p.sum(0) * slopes).sum()
    out = chosen.to(torch.int32), weights, counts.to(torch.int32), loss
    if state["op"] == "route":
        return out
    u = state["dloss"] * slopes[None, :]
    dw = state["dweights"]
    one = torch.zeros_like(p)
    if case["renormalize"]:
        dlogits = p * (u - (p * u).sum(dim=1, keepdim=True))
        one = weights * (dw - (weights * dw).sum(dim=1, keepdim=True))
        dlogits = dlogits.scatter_add(1, chosen.clamp(min=0), one)
    else:
        u = u + one.scatter_add(1, chosen.clamp(min=0), dw)
        dlogits = p * (u - (p * u).sum(dim=1, keepdim=True))
    return *out, dlogits.to(DTYPES[case["dtype"]])


def _combine_plain(y, rows, weights):
    """The rows of each token, by their weights; a slot without a place adds nothing."""
    keep = rows >= 0
    picked = y.float()[torch.where(keep, rows, 0).long()]
    if weights is not None:
        keep = keep * weights
    return (picked * keep[..., None]).sum(dim=1)


def _exchange_plain(state):
    case, op = state["case"], state["op"]
    dtype = DTYPES[case["dtype"]]
    if op == "dispatch":
        ends, rows, slots = _group(state["ids"], case["experts"])
        xs = state["x"][slots.long() // case["k"]]
        there = torch.arange(len(slots), device="cuda") < ends[-1]
        return ends, rows, slots, torch.where(there[:, None], xs, torch.zeros((), dtype=dtype, device="cuda"))
    rows, weights = state["rows"], state["weights"]
    if op == "combine":
        return _combine_plain(state["y"], rows, weights).to(dtype)
    keep = rows >= 0
    place = torch.where(keep, rows, 0).long()
    dout = state["dout"].float()
    dweights = (state["y"].float()[place] * dout[:, None]).sum(dim=2) * keep
    # one row more takes what has no place
    dy = torch.zeros((len(state["y"]) + 1, case["width"]), device="cuda")
    dy[torch.where(keep, rows, len(state["y"])).long()] = weights[..., None] * dout[:, None]
    return dy[:-1].to(dtype), dweights, _combine_plain(state["dxs"], rows, None).to(dtype)


def _adapters_plain(state):
    case = state["case"]
    m, adapters, most = case["m"], case["adapters"], state["most"]
    ends = state["ends"].long()
    low = torch.cat([ends.new_zeros(1), ends[:-1]])
    # every adapter's tokens padded to the most that one has; m is no token
    place = low[:, None] + torch.arange(most, device="cuda")
    token = torch.where(place < ends[:, None], state["slots"].long()[place.clamp(max=m - 1)], m)
    scales = state["scales"][:, None, None]
    down, up = state["down"].float(), state["up"].float()

    def take(v):
        return torch.nn.functional.pad(v.float(), (0, 0, 0, 1))[token]

    x = take(state["x"])
    h = torch.bmm(x, down.transpose(1, 2).contiguous())
    out = torch.nn.functional.pad(state["y"].float(), (0, 0, 0, 1))
    out[token] = out[token] + scales * torch.bmm(h, up)
    out = out[:m].to(state["y"].dtype)
    if state["op"] == "adapters":
        return out
    d = take(state["dout"])
    dh = scales * torch.bmm(d, up.transpose(1, 2).contiguous())
    dx = torch.zeros((m + 1, case["k_in"]), device="cuda")
    dx[token] = torch.bmm(dh, down)
    d_down = torch.bmm(dh.transpose(1, 2).contiguous(), x)
    d_up = torch.bmm((scales * h).transpose(1, 2).contiguous(), d)
    grad = DTYPES[case["out"]]
    return out, dx[:m].to(state["x"].dtype), d_down.to(grad), d_up.to(grad)


def run(state):
    case, op = state["case"], state["op"]
    if not own:
        if op.startswith("route"):
            return _route_plain(state)
        return _adapters_plain(state) if op.startswith("adapters") else _exchange_plain(state)
    from paper_2412_08832_amd import hadacore

    if op.startswith("route"):
        routes = hadacore.route_tokens(state["logits"], case["k"], renormalize=case["renormalize"],
                                       valid=state["valid"])
        if op == "route":
            return routes[:4]
        return *routes[:4], hadacore.route_tokens_gradient(
            state["logits"], routes, dweights=state["dweights"], dloss=state["dloss"])
    if op == "dispatch":
        groups = hadacore.group_tokens(state["ids"], case["experts"])
        return *groups, hadacore.dispatch_rows(state["x"], groups.rows, groups.ends)
    if op == "combine":
        return hadacore.combine_rows(state["y"], state["rows"], state["weights"])
    if op == "exchange_back":
        dy, dweights = hadacore.combine_rows_gradient(state["dout"], state["y"], state["rows"],
                                                      state["ends"], state["weights"])
        return dy, dweights, hadacore.combine_rows(state["dxs"], state["rows"])
    x, y, down, up = state["x"], state["y"], state["down"], state["up"]
    plan = {"ends": state["ends"], "slots": state["slots"], "scales": state["scales"]}
    if op == "adapters":
        return hadacore.adapt_rows(x, down, up, y=y, **plan)
    dout, grad = state["dout"], DTYPES[case["out"]]
    out, h = hadacore.adapt_rows(x, down, up, y=y, hidden=True, **plan)
    dx, dh = hadacore.adapt_rows(dout, up, down, hidden=True, **plan)
    return (out, dx, hadacore.adapter_gradient(dh, x, dtype=grad, **plan),
            hadacore.adapter_gradient(h, dout, dtype=grad, **plan))


def work(case):
    op, m = case["op"], case["m"]
    b = SIZES[case["dtype"]]
    if op.startswith("route"):
        e, k = case["experts"], case["k"]
        once = m * e * b + 8 * m * k + 4 * e + 4
        flops = 5 * m * e
        if op == "route_train":
            once, flops = once + m * e * b + 4 * m * k, 10 * m * e
        return {"bytes": once, "flops": flops}
    if op in ("dispatch", "combine", "exchange_back"):
        k, width = case["k"], case["width"]
        row = m * width * b
        if op == "dispatch":
            return {"bytes": row * (1 + k) + 12 * m * k, "flops": 0}
        if op == "combine":
            return {"bytes": row * (1 + k) + 8 * m * k, "flops": 2 * m * k * width}
        return {"bytes": row * (2 + 3 * k) + 12 * m * k, "flops": 4 * m * k * width}
    n, k_in, rank, wide = case["n"], case["k_in"], case["rank"], SIZES[case["out"]]
    used = min(case["requests"] - case["bare"], case["adapters"] - case["idle"])
    weights = used * rank * (n + k_in) * b
    flops = 2 * m * rank * (n + k_in)
    if op == "adapters":
        return {"bytes": m * k_in * b + 2 * m * n * wide + weights, "flops": flops}
    return {"bytes": 2 * m * k_in * b + 3 * m * n * b + weights
            + case["adapters"] * rank * (n + k_in) * wide, "flops": 3 * flops}


# ---- 64 bits --------------------------------------------------------------------


def _route64(state):
    case = state["case"]
    m, experts, k = case["m"], case["experts"], case["k"]
    logits = state["logits"].double()
    there = torch.ones(m, dtype=torch.bool, device="cuda") if state["valid"] is None else state["valid"]
    p = torch.zeros_like(logits)
    p[there] = torch.exp(logits[there] - torch.logsumexp(logits[there], dim=1, keepdim=True))
    # an expert's place among a token's: how many are larger, or as large and before it
    chosen = torch.full((m, k), -1, dtype=torch.int32, device="cuda")
    step = max(1, (1 << 26) // experts ** 2)
    index = torch.arange(experts, device="cuda")
    for t in range(0, m, step):
        l = logits[t : t + step]
        ahead = (l[:, None, :] > l[:, :, None]) | \
            ((l[:, None, :] == l[:, :, None]) & (index[None, :] < index[:, None]))
        place = ahead.sum(dim=2)
        token, expert = torch.nonzero(place < k, as_tuple=True)
        chosen[t + token, place[token, expert]] = expert.to(torch.int32)
    chosen[~there] = -1
    picked = torch.zeros((m, k), dtype=torch.float64, device="cuda")
    for j in range(k):
        picked[there, j] = p[there, chosen[there, j].long()]
    total = picked.sum(dim=1)
    weights = picked.clone()
    if case["renormalize"]:
        weights[there] /= total[there, None]
    counts = torch.bincount(chosen[there].reshape(-1).long(), minlength=experts)
    tokens = int(there.sum())
    share = counts.double() / (tokens * k)
    loss = experts * (share * p.sum(dim=0) / tokens).sum()
    out = [chosen, weights, counts.to(torch.int32), loss]
    if state["op"] == "route":
        return tuple(out)
    # derivatives with respect to the probabilities, then through the softmax
    dp = (state["dloss"].double() * experts / tokens * share)[None, :].repeat(m, 1)
    dw = state["dweights"].double()
    for j in range(k):
        if case["renormalize"]:
            d = (dw[:, j] - (dw * weights).sum(dim=1)) / total.clamp(min=1e-300)
        else:
            d = dw[:, j]
        dp[there, chosen[there, j].long()] += d[there]
    out.append(p * (dp - (p * dp).sum(dim=1, keepdim=True)))
    return tuple(out)


def _exchange64(state):
    case, op = state["case"], state["op"]
    m, k, width = case["m"], case["k"], case["width"]
    ids = state["ids"].cpu()
    # the slots of expert after expert
    order = [torch.nonzero(ids.reshape(-1) == e).reshape(-1) for e in range(case["experts"])]
    ends = torch.tensor([len(o) for o in order]).cumsum(0)
    taken = torch.cat(order)
    rows = torch.full((m * k,), -1)
    rows[taken] = torch.arange(len(taken))
    slots = torch.cat([taken, torch.nonzero(rows < 0).reshape(-1)])
    token = (taken // k).cuda()
    if op == "dispatch":
        xs = torch.zeros((m * k, width), dtype=torch.float64, device="cuda")
        xs[: len(taken)] = state["x"][token].double()
        return tuple(v.to(torch.int32).cuda() for v in (ends, rows.view(m, k), slots)) + (xs,)
    w = state["weights"].double().reshape(-1)[taken.cuda()]
    if op == "combine":
        out = torch.zeros((m, width), dtype=torch.float64, device="cuda")
        return out.index_add_(0, token, state["y"][: len(taken)].double() * w[:, None])
    there = state["dout"].double()[token]
    dy = torch.zeros((m * k, width), dtype=torch.float64, device="cuda")
    dy[: len(taken)] = there * w[:, None]
    dweights = torch.zeros(m * k, dtype=torch.float64, device="cuda")
    dweights[taken.cuda()] = (there * state["y"][: len(taken)].double()).sum(dim=1)
    dx = torch.zeros((m, width), dtype=torch.float64, device="cuda")
    dx.index_add_(0, token, state["dxs"][: len(taken)].double())
    return dy, dweights.view(m, k), dx


def _adapters64(state):
    case = state["case"]
    out = state["y"].double()
    train = state["op"] == "adapters_train"
    dx = torch.zeros((case["m"], case["k_in"]), dtype=torch.float64, device="cuda")
    d_down = torch.zeros(state["down"].shape, dtype=torch.float64, device="cuda")
    d_up = torch.zeros(state["up"].shape, dtype=torch.float64, device="cuda")
    low = 0
    for a, high in enumerate(state["ends"].tolist()):
        t = state["slots"][low:high].long()
        low = high
        s = float(state["scales"][a])
        down, up = state["down"][a].double(), state["up"][a].double()
        x = state["x"][t].double()
        h = x @ down.t()
        out[t] += s * (h @ up)
        if train:
            d = state["dout"][t].double()
            dh = s * (d @ up.t())
            dx[t] = dh @ down
            d_down[a] = dh.t() @ x
            d_up[a] = s * (h.t() @ d)
    return (out, dx, d_down, d_up) if train else out


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"].startswith("route"):
        return _route64(state)
    return _adapters64(state) if case["op"].startswith("adapters") else _exchange64(state)
