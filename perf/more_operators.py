"""Cases for timing what a token's index chooses in a partitioned language model: its row of the vocabulary matrix, and its experts.

Embedding: y[t] = scale * w[id[t]] over a vocabulary matrix w, [V, M] or [M, V], split y ways (tokens split x ways); its gradient is
dw[v] = scale * (sum of dy[t] over the tokens t with id v), the tokens of one entry added up in float32.  An id outside the vocabulary is a token without one.

Routing: a token takes the k experts of its largest logits (ties: the lowest; -infinity: none) with weights from a softmax over all experts, or over its own.  All
choices, ordered by expert and then by token, are the slots: a slot is a row of the arrays that the experts work on, expert e's slots follow those of expert e - 1.
Exchange: rows[slot] = x[token of the slot], y[t] = sum over t's slots of weight * rows[slot], and the gradients of both.
Experts: out[slot] = rows[slot] w[expert of the slot], the same with w transposed (the gradient of the rows), and dw[e] = sum over e's slots of rows[slot]^T d[slot]:
matrix products grouped by expert, of as many rows as the routing gave each, which only the device knows.

`listed()` names twelve cases, `draw(rng)` makes more of the same kinds with other sizes.
"""
import math

import torch

own = False


def listed():
    return [
        # the next token of one sequence
        {"name": "embed_one", "kind": "embed", "dtype": "bf16", "t": 1, "m": 2048, "v": 32000, "x": 1, "y": 1, "order": "vm", "pad": True, "scaled": False},
        # 8 sequences of 2048 tokens of a wide model on a 2 x 4 mesh, rows scaled by sqrt(M)
        {"name": "embed_prefill", "kind": "embed", "dtype": "bf16", "t": 16384, "m": 8192, "v": 32000, "x": 2, "y": 4, "order": "vm", "pad": True, "scaled": True},
        # a training step of one sequence; most rows of dw are zeros
        {"name": "embed_grad_step", "kind": "embed_grad", "dtype": "bf16", "t": 2048, "m": 2048, "v": 32000, "x": 1, "y": 1, "order": "vm", "pad": True, "scaled": False},
        # packed sequences of any length on a 2 x 4 mesh, sizes that divide by nothing, the matrix in the other order
        {"name": "embed_grad_uneven", "kind": "embed_grad", "dtype": "bf16", "t": 9999, "m": 1001, "v": 32003, "x": 2, "y": 4, "order": "mv", "pad": False, "scaled": True},
        # 32 sequences' next tokens
        {"name": "route_decode", "kind": "route", "dtype": "f32", "t": 32, "e": 64, "k": 8, "x": 1, "norm": True, "grad": False},
        # a training step of 8 sequences of 2048 tokens, with the gradient of the logits
        {"name": "route_train", "kind": "route", "dtype": "f32", "t": 16384, "e": 128, "k": 8, "x": 2, "norm": False, "grad": True},
        # forward: tokens to their experts' rows and back
        {"name": "exchange_step", "kind": "exchange", "dtype": "bf16", "t": 2048, "m": 2048, "e": 32, "k": 2, "x": 1, "y": 4, "pad": True, "grad": False},
        # backward of the same for 4 sequences of 2048 tokens, four experts a token
        {"name": "exchange_grad", "kind": "exchange", "dtype": "bf16", "t": 8192, "m": 4096, "e": 64, "k": 4, "x": 2, "y": 4, "pad": True, "grad": True},
        # decoding: 32 sequences' next tokens, 8 of 64 experts each; every expert's matrix is read for a few rows
        {"name": "experts_decode", "kind": "experts", "way": "forward", "dtype": "bf16", "t": 32, "k": 8, "e": 64, "m": 2048, "h": 4096, "y": 1, "pad": True, "relu": True},
        # prefill and training forward: 8 sequences of 2048 tokens, the largest of the list
        {"name": "experts_forward", "kind": "experts", "way": "forward", "dtype": "bf16", "t": 16384, "k": 2, "e": 16, "m": 2048, "h": 8192, "y": 4, "pad": True, "relu": True},
        # gradients of a step of 2 sequences: of the rows, and of the experts' matrices
        {"name": "experts_backward", "kind": "experts", "way": "backward", "dtype": "bf16", "t": 4096, "k": 2, "e": 8, "m": 4096, "h": 8192, "y": 1, "pad": True, "relu": False},
        # a small layer kept in float32, odd sizes, dense rows
        {"name": "experts_uneven", "kind": "experts", "way": "backward", "dtype": "f32", "t": 777, "k": 3, "e": 12, "m": 515, "h": 1023, "y": 2, "pad": False, "relu": False},
    ]


def draw(rng):
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["embed", "embed_grad", "embed_grad", "route", "exchange", "experts", "experts", "experts"])
    whole = rng.random() < 0.6            # sizes of models, or any
    wide = lambda lo, hi, to: min(hi, _up(between(lo, hi), to)) if whole else between(lo, hi)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if kind in ("embed", "embed_grad"):
        while True:
            t, m, v = between(1, 32768), wide(64, 8192, 64), wide(90, 128000, 128)
            if t * m <= 16384 * 4096 and v * m <= 32000 * 8192:
                break
        case = {"kind": kind, "dtype": dtype, "t": t, "m": m, "v": v, "x": rng.choice([1, 1, 2, 3]), "y": rng.choice([1, 1, 2, 4, 8]), "order": rng.choice(["vm", "vm", "vm", "mv"]),
                "pad": whole or rng.random() < 0.5, "scaled": rng.random() < 0.5}
        return case
    if kind == "route":
        e = between(4, 256)
        return {"kind": kind, "dtype": rng.choice(["f32", "f32", "bf16"]), "t": between(1, 32768), "e": e, "k": rng.randint(1, min(8, e)), "x": rng.choice([1, 1, 2, 3]), "norm": rng.random() < 0.5,
                "grad": rng.random() < 0.5}
    e = between(4, 128)
    k = rng.randint(1, min(8, e))
    if kind == "exchange":
        while True:
            t, m = between(1, 16384), wide(64, 8192, 64)
            if t * k * m <= 16384 * 8192:
                break
        return {"kind": kind, "dtype": dtype, "t": t, "m": m, "e": e, "k": k, "x": rng.choice([1, 1, 2, 3]), "y": rng.choice([1, 1, 2, 4]), "pad": whole or rng.random() < 0.5, "grad": rng.random() < 0.5}
    way = rng.choice(["forward", "forward", "input", "backward"])
    most = (16384 * 2 * 2048 * 8192) // (32 if dtype == "f32" else 2)
    while True:
        t, m, h = between(1, 16384), wide(256, 4096, 64), wide(256, 8192, 64)
        if t * k * m * h <= most and e * m * h <= 64 * 2048 * 4096:
            break
    return {"kind": kind, "way": way, "dtype": dtype, "t": t, "k": k, "e": e, "m": m, "h": h, "y": rng.choice([1, 1, 2, 4]), "pad": whole or rng.random() < 0.6, "relu": way == "forward" and rng.random() < 0.5}


def _up(n, to):
    return -(-n // to) * to


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _scale(case):
    return math.sqrt(case["m"]) if case.get("scaled") else 1.0


# ------------------------------------------------------------------------------------------------- what a program has in hand
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    state = {"case": case}
    if case["kind"] in ("embed", "embed_grad"):
        _prepare_embed(case, gen, state)
    elif case["kind"] == "route":
        _prepare_route(case, gen, state)
    elif case["kind"] == "exchange":
        _prepare_exchange(case, gen, state)
    else:
        _prepare_experts(case, gen, state)
    if own:
        state["call"] = _call(state)
    return state


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _tokens(case, gen, cols):
    """Rows of all tokens in static shards one after the other, [x, ts, ld]; what lies beyond their valid part may hold anything."""
    ts, ld = -(-case["t"] // case["x"]), _up(cols, 8) if case["pad"] else cols
    a = torch.full((case["x"] * ts, ld), float("nan"), dtype=_dtype(case), device="cuda")
    if gen is not None:
        a[:case["t"], :cols] = _randn(gen, case["t"], cols)
    return a.view(case["x"], ts, ld)


def _prepare_embed(case, gen, state):
    t, m, v, nb, grad = case["t"], case["m"], case["v"], case["y"], case["kind"] == "embed_grad"
    ts, vs = -(-t // case["x"]), -(-v // nb)
    ids = torch.full((case["x"] * ts,), -1, dtype=torch.int32, device="cuda")
    # texts: an entry's frequency falls with its rank; here and there a token without an entry
    ranks = torch.exp(torch.rand(t, generator=gen, device="cuda", dtype=torch.float64) * math.log(v + 1)).long() - 1
    ranks = (ranks.clamp_(0, v - 1) * 7919) % v
    ids[:t] = torch.where(torch.rand(t, generator=gen, device="cuda") < 0.02, torch.full_like(ranks, -1), ranks).int() if t > 1 else ranks.int()
    cols = m if case["order"] == "vm" else vs
    ldw = _up(cols, 8) if case["pad"] else cols
    w = torch.full((nb, vs if case["order"] == "vm" else m, ldw), float("nan"), dtype=_dtype(case), device="cuda")
    if not grad:
        full = _randn(gen, v, m) * 0.05
        if case["order"] == "vm":
            w.view(nb * vs, ldw)[:v, :m] = full
        else:
            for j in range(nb):
                part = full[j * vs:(j + 1) * vs].t()
                w[j, :, :part.shape[1]] = part
    state.update(ids=ids, w=w, rows=_tokens(case, gen if grad else None, m))


def _prepare_route(case, gen, state):
    t, e, k = case["t"], case["e"], case["k"]
    ts = -(-t // case["x"])
    logits = torch.full((case["x"] * ts, e), float("nan"), dtype=_dtype(case), device="cuda")
    logits[:t] = _logits(case, gen)
    state["logits"] = logits.view(case["x"], ts, e)
    state.update(experts=_ints(t, k), slots=_ints(t, k), order=_ints(t * k), sizes=_ints(e), weights=torch.zeros((t, k), device="cuda"))
    if case["grad"]:
        state["dweights"] = _randn(gen, t, k)
        state["dlogits"] = torch.zeros_like(state["logits"])


def _ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device="cuda")


def _logits(case, gen):
    """Experts are not liked alike; one token in fifty (a padded place) goes to none."""
    z = _randn(gen, case["t"], case["e"]) + 0.7 * _randn(gen, 1, case["e"])
    empty = torch.rand((case["t"], 1), generator=gen, device="cuda") < 0.02
    return torch.where(empty, torch.full_like(z, -math.inf), z) if case["t"] > 1 else z


def _routing(case, gen):
    """A routing as `route` makes it: experts, weights, slots [t, k], order [t k], sizes [e]."""
    return _plain_route(_logits(case, gen), case["k"], False)


def _prepare_exchange(case, gen, state):
    t, k, m, nb = case["t"], case["k"], case["m"], case["y"]
    state.update(zip(("experts", "weights", "slots", "order", "sizes"), _routing(case, gen)))
    state["x"], state["y"] = _tokens(case, gen, m), _tokens(case, None, m)
    ld = state["x"].shape[2]
    state["rows"] = torch.zeros((t * k, ld), dtype=_dtype(case), device="cuda")
    if case["grad"]:
        state["rows"][:, :m] = _randn(gen, t * k, m)
        state["drows"] = torch.zeros_like(state["rows"])
        state["dweights"] = torch.zeros((t, k), device="cuda")


def _prepare_experts(case, gen, state):
    t, k, e, m, h, nb = case["t"], case["k"], case["e"], case["m"], case["h"], case["y"]
    sizes = _routing(case, gen)[4]
    state.update(sizes=sizes, most=max(1, int(sizes.max())))
    s, es, ldm, ldh = t * k, -(-e // nb), *(_up(n, 8) if case["pad"] else n for n in (m, h))
    def rows(cols, ld, filled):
        a = torch.zeros((s, ld), dtype=_dtype(case), device="cuda")
        if filled:
            a[:, :cols] = _randn(gen, s, cols)
        return a
    w = torch.full((nb * es, m, ldh), float("nan"), dtype=_dtype(case), device="cuda")
    for i in range(e):
        w[i, :, :h] = _randn(gen, m, h) * 0.02
    forward = case["way"] == "forward"
    state.update(w=w.view(nb, es, m, ldh), wide=rows(h, ldh, not forward), narrow=rows(m, ldm, forward or case["way"] == "backward"))
    if case["way"] == "backward":
        state["dnarrow"], state["dw"] = torch.zeros_like(state["narrow"]), torch.zeros_like(state["w"])


# ------------------------------------------------------------------------------------------------- the framework's calls
def _call(state):
    """The framework's calls on these shards, their arguments made once as a program's loop would."""
    import paper_2105_04663_amd as g

    case = state["case"]
    na, nb = case.get("x", 1), case.get("y", 1)
    mesh = g.Mesh((na, nb), tuple(range(na * nb)))
    places = [(i, j) for i in range(na) for j in range(nb)]
    bufs = lambda a, which: [g.ShardBuf.of(a[p[which]], a.shape[-1]) for p in places]      # [shards, .., row stride]
    one = lambda a: [g.ShardBuf.of(a, a.shape[-1])] * len(places)                          # all partitions hold it
    stream = lambda: torch.cuda.current_stream().cuda_stream
    t, k = case["t"], case.get("k")

    def space(size):
        state["space"] = torch.empty(size + 256, dtype=torch.uint8, device="cuda")
        return {"workspace": _up(state["space"].data_ptr(), 256), "workspace_bytes": size}

    if case["kind"] in ("embed", "embed_grad"):
        v, m, vocab_dim = case["v"], case["m"], 0 if case["order"] == "vm" else 1
        rows_sh = g.Sharding((t, m), (0, -1))
        w_sh = g.Sharding((v, m), (1, -1)) if vocab_dim == 0 else g.Sharding((m, v), (-1, 1))
        ts = state["rows"].shape[1]
        ids = [state["ids"].data_ptr() + 4 * i * ts for i, _ in places]
        ws, rows = bufs(state["w"], 1), bufs(state["rows"], 0)
        if case["kind"] == "embed":
            return lambda: g.embed(mesh, ids, ws, w_sh, rows, rows_sh, vocab_dim=vocab_dim, scale=_scale(case), stream=stream())
        more = space(g.embed_grad_workspace_bytes(mesh, rows_sh, w_sh, vocab_dim, g.BF16 if case["dtype"] == "bf16" else g.F32))
        return lambda: g.embed_grad(mesh, ids, rows, rows_sh, ws, w_sh, vocab_dim=vocab_dim, scale=_scale(case), stream=stream(), **more)
    address = lambda name: state[name].data_ptr() if name in state else 0
    route = g.RouteBuf(experts=address("experts"), weights=address("weights"), slots=address("slots"), order=address("order"), sizes=address("sizes"))
    if case["kind"] == "route":
        sh = g.Sharding((t, case["e"]), (0, -1))
        logits, more = bufs(state["logits"], 0), space(g.route_workspace_bytes(mesh, sh, k))
        def call():
            g.route(mesh, logits, sh, k, route, normalise=case["norm"], stream=stream(), **more)
            if case["grad"]:
                g.route_grad(mesh, logits, sh, k, route, state["dweights"].data_ptr(), dlogits, normalise=case["norm"], stream=stream())
        dlogits = bufs(state["dlogits"], 0) if case["grad"] else None
        return call
    e, m = case["e"], case["m"]
    narrow_sh = g.Sharding((e, t * k, m), (1, -1, -1))
    if case["kind"] == "exchange":
        x_sh, x, y, rows = g.Sharding((t, m), (0, -1)), bufs(state["x"], 0), bufs(state["y"], 0), one(state["rows"])
        if not case["grad"]:
            def call():
                g.dispatch(mesh, x, x_sh, k, route, rows, narrow_sh, stream=stream())
                g.combine(mesh, rows, narrow_sh, k, route, y, x_sh, stream=stream())
            return call
        drows = one(state["drows"])
        def call():
            g.combine_grad(mesh, x, x_sh, rows, narrow_sh, k, route, drows, state["dweights"].data_ptr(), stream=stream())
            g.combine(mesh, drows, narrow_sh, k, route, y, x_sh, weighted=False, stream=stream())
        return call
    h = case["h"]
    wide_sh, w_sh = g.Sharding((e, t * k, h), (1, -1, -1)), g.Sharding((e, m, h), (1, -1, -1))
    forward, back, weight = g.DotDims((0,), (0,), (2,), (1,)), g.DotDims((0,), (0,), (2,), (2,)), g.DotDims((0,), (0,), (1,), (1,))
    w, narrow, wide, sizes = bufs(state["w"], 1), one(state["narrow"]), one(state["wide"]), state["sizes"].data_ptr()
    if case["way"] == "forward":
        epilogue = g.EPILOGUE_RELU if case["relu"] else g.EPILOGUE_NONE
        return lambda: g.ragged_dot(mesh, forward, narrow, narrow_sh, w, w_sh, wide, wide_sh, sizes, stream=stream(), epilogue=epilogue)
    if case["way"] == "input":
        return lambda: g.ragged_dot(mesh, back, wide, wide_sh, w, w_sh, narrow, narrow_sh, sizes, stream=stream())
    dnarrow, dw = one(state["dnarrow"]), bufs(state["dw"], 1)
    def call():
        g.ragged_dot(mesh, back, wide, wide_sh, w, w_sh, dnarrow, narrow_sh, sizes, stream=stream())
        g.ragged_dot(mesh, weight, narrow, narrow_sh, wide, wide_sh, dw, w_sh, sizes, stream=stream())
    return call


# ------------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if own:
        state["call"]()
    else:
        _plain(state)
    if case["kind"] == "embed":
        return {"y": state["rows"][:, :, :case["m"]]}
    if case["kind"] == "embed_grad":
        return {"dw": state["w"][:, :, :case["m"] if case["order"] == "vm" else -(-case["v"] // case["y"])]}
    if case["kind"] == "route":
        out = {name: state[name] for name in ("experts", "weights", "slots", "order", "sizes")}
        return out | ({"dlogits": state["dlogits"]} if case["grad"] else {})
    if case["kind"] == "exchange":
        out = {"y": state["y"][:, :, :case["m"]]}
        return out | ({"drows": state["drows"][:, :case["m"]], "dweights": state["dweights"]} if case["grad"] else {"rows": state["rows"][:, :case["m"]]})
    if case["way"] == "forward":
        return {"out": state["wide"][:, :case["h"]]}
    if case["way"] == "input":
        return {"out": state["narrow"][:, :case["m"]]}
    return {"drows": state["dnarrow"][:, :case["m"]], "dw": state["dw"][..., :case["h"]]}


def _plain(state):
    """The definitions in elementary float32 operations, every result written to the state's buffers."""
    case = state["case"]
    if case["kind"] == "embed":
        _plain_embed(state, case)
    elif case["kind"] == "embed_grad":
        _plain_embed_grad(state, case)
    elif case["kind"] == "route":
        logits = state["logits"].flatten(0, 1)[:case["t"]].float()
        for name, value in zip(("experts", "weights", "slots", "order", "sizes"), _plain_route(logits, case["k"], case["norm"])):
            state[name].copy_(value)
        if case["grad"]:
            _plain_route_grad(state, case, logits)
    elif case["kind"] == "exchange":
        _plain_exchange(state, case)
    else:
        _plain_experts(state, case)


def _plain_embed(state, case):
    t, m, v = case["t"], case["m"], case["v"]
    ids = state["ids"][:t].long()
    there = (ids >= 0) & (ids < v)
    at = torch.where(there, ids, torch.zeros_like(ids))
    if case["order"] == "vm":
        rows = state["w"].flatten(0, 1)[at, :m].float()
    else:
        vs = -(-v // case["y"])
        rows = state["w"][at // vs, :, at % vs].float()
    y = state["rows"].flatten(0, 1)
    y[:, :m] = 0
    y[:t, :m] = torch.where(there[:, None], rows * _scale(case), torch.zeros_like(rows))


def _plain_embed_grad(state, case):
    t, m, v, nb = case["t"], case["m"], case["v"], case["y"]
    vs = -(-v // nb)
    ids = state["ids"][:t].long()
    at = torch.where((ids >= 0) & (ids < v), ids, torch.full_like(ids, v))
    sums = torch.zeros((nb * vs + 1, m), device="cuda")
    sums.index_add_(0, torch.where(at < v, at, torch.full_like(at, nb * vs)), state["rows"].flatten(0, 1)[:t, :m].float())
    dw = (sums[:nb * vs] * _scale(case)).view(nb, vs, m)
    if case["order"] == "vm":
        state["w"][:, :, :m] = dw
    else:
        state["w"][:, :, :vs] = dw.transpose(1, 2)


def _plain_route(z, k, normalise):
    t, e = z.shape
    top, experts = torch.sort(z, dim=1, descending=True, stable=True)
    top, experts = top[:, :k], experts[:, :k]
    there = top > -math.inf
    most = torch.where(there[:, :1], top[:, :1], torch.zeros_like(top[:, :1]))
    shares = torch.exp(top - most)
    total = shares.sum(dim=1, keepdim=True) if normalise else torch.exp(z - most).sum(dim=1, keepdim=True)
    weights = torch.where(there, shares / total, torch.zeros_like(top))
    flat = torch.where(there, experts, torch.full_like(experts, e)).view(-1)
    ordered, order = torch.sort(flat, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(t * k, device=z.device)
    sizes = torch.zeros(e + 1, dtype=torch.int64, device=z.device).scatter_add_(0, flat, torch.ones_like(flat))[:e]
    none = torch.full_like(place, -1)
    return (torch.where(there, experts, none.view(t, k)).int(), weights, torch.where(flat < e, place, none).view(t, k).int(), torch.where(ordered < e, order, none).int(), sizes.int())


def _plain_route_grad(state, case, z):
    there = state["experts"] >= 0
    at = torch.where(there, state["experts"], torch.zeros_like(state["experts"])).long()
    w = state["weights"]
    g = torch.where(there, state["dweights"], torch.zeros_like(w))
    mean = (g * w).sum(dim=1, keepdim=True)
    if case["norm"]:
        d = torch.zeros_like(z)
    else:
        most = z.amax(dim=1, keepdim=True)
        shares = torch.exp(z - torch.where(most > -math.inf, most, torch.zeros_like(most)))
        total = shares.sum(dim=1, keepdim=True)
        d = -mean * shares / torch.where(total > 0, total, torch.ones_like(total))
    d.scatter_add_(1, at, w * (g - mean) if case["norm"] else w * g)
    out = state["dlogits"].flatten(0, 1)
    out.zero_()
    out[:case["t"]] = d


def _plain_exchange(state, case):
    t, k, m = case["t"], case["k"], case["m"]
    order, slots = state["order"].long(), state["slots"].long()
    taken, there = order >= 0, slots >= 0
    token = torch.where(taken, order, torch.zeros_like(order)) // k
    at = torch.where(there, slots, torch.zeros_like(slots))
    weights = torch.where(there, state["weights"], torch.zeros_like(state["weights"]))
    x, y = state["x"].flatten(0, 1)[:, :m], state["y"].flatten(0, 1)
    y[:, :m] = 0
    if not case["grad"]:
        state["rows"][:, :m] = torch.where(taken[:, None], x[token], state["rows"][:, :m])
        y[:t, :m] = (state["rows"][:, :m][at].float() * weights[:, :, None]).sum(dim=1)
        return
    dy = x[:t].float()
    picked = state["rows"][:, :m][at].float()
    state["dweights"].copy_(torch.where(there, (picked * dy[:, None, :]).sum(dim=2), torch.zeros_like(weights)))
    share = weights.view(-1)[torch.where(taken, order, torch.zeros_like(order))]
    state["drows"][:, :m] = torch.where(taken[:, None], dy[token] * share[:, None], state["drows"][:, :m].float())
    back = state["drows"][:, :m][at].float()
    y[:t, :m] = torch.where(there[:, :, None], back, torch.zeros_like(back)).sum(dim=1)


def _plain_experts(state, case):
    e, m, h, s, most = case["e"], case["m"], case["h"], case["t"] * case["k"], state["most"]
    ends = torch.cumsum(state["sizes"].long(), 0)
    starts = ends - state["sizes"]
    at = torch.arange(most, device="cuda")
    inside = (at < state["sizes"][:, None])[:, :, None]
    places = (starts[:, None] + at).clamp_(max=s - 1)
    slot = torch.arange(s, device="cuda")
    owner = torch.searchsorted(ends, slot, right=True).clamp_(max=e - 1)
    taken = (slot < ends[-1])[:, None]
    w = state["w"].flatten(0, 1)[:e, :, :h].float()
    def grouped(rows, cols):
        rows = rows[:, :cols][places].float()
        return torch.where(inside, rows, torch.zeros_like(rows))
    def put(to, cols, blocks):
        to[:, :cols] = torch.where(taken, blocks[owner, (slot - starts[owner]).clamp_(0, most - 1)].to(to.dtype), to[:, :cols])
    if case["way"] == "forward":
        out = torch.bmm(grouped(state["narrow"], m), w)
        put(state["wide"], h, torch.relu(out) if case["relu"] else out)
        return
    wide = grouped(state["wide"], h)
    put(state["narrow"] if case["way"] == "input" else state["dnarrow"], m, torch.bmm(wide, w.transpose(1, 2)))
    if case["way"] == "backward":
        dw = state["dw"].flatten(0, 1)
        dw[e:] = 0
        dw[:e, :, :h] = torch.bmm(grouped(state["narrow"], m).transpose(1, 2), wide)


# ------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """What run() returns, in float64, from the definitions."""
    state = prepare(case, seed)
    state.pop("call", None)
    t, nb = case["t"], case.get("y", 1)
    double = dict(dtype=torch.float64, device="cuda")
    if case["kind"] in ("embed", "embed_grad"):
        v, m, vs = case["v"], case["m"], -(-case["v"] // nb)
        ids = state["ids"][:t].cpu().numpy()
        tokens = [i for i in range(t) if 0 <= ids[i] < v]
        rows = torch.tensor(tokens, dtype=torch.int64, device="cuda")
        entries = state["ids"][:t].long()[rows]
        if case["kind"] == "embed":
            y = torch.zeros(state["rows"].flatten(0, 1).shape[0], m, **double)
            by_entry = state["w"][:, :, :m].reshape(nb * vs, m) if case["order"] == "vm" else state["w"][:, :, :vs].transpose(1, 2).reshape(nb * vs, m)
            y[rows] = by_entry.double()[entries] * _scale(case)
            return {"y": y.view(state["rows"].shape[0], -1, m)}
        dw = torch.zeros(nb * vs, m, **double)
        dw.index_put_((entries,), state["rows"].flatten(0, 1)[rows, :m].double() * _scale(case), accumulate=True)
        return {"dw": dw.view(nb, vs, m) if case["order"] == "vm" else dw.view(nb, vs, m).transpose(1, 2)}
    if case["kind"] == "route":
        z = state["logits"].flatten(0, 1)[:t].double()
        k = case["k"]
        experts = torch.argsort(z, dim=1, descending=True, stable=True)[:, :k]
        chosen = torch.zeros_like(z, dtype=torch.bool).scatter_(1, experts, True) & (z > -math.inf)
        among = torch.where(chosen, z, torch.full_like(z, -math.inf)) if case["norm"] else z
        p = torch.nan_to_num(torch.softmax(among, dim=1))
        out = {"experts": None, "weights": (p * chosen).gather(1, experts), "slots": None, "order": None, "sizes": None}
        if case["grad"]:
            g = torch.zeros_like(z).scatter_(1, experts, state["dweights"].double()) * chosen
            d = torch.zeros_like(state["logits"].flatten(0, 1), dtype=torch.float64)
            d[:t] = p * (g - (p * g).sum(dim=1, keepdim=True))
            out["dlogits"] = d.view(state["logits"].shape)
        return out
    k = case["k"]
    if case["kind"] == "exchange":
        m = case["m"]
        x = state["x"].flatten(0, 1)[:t, :m].double()
        rows = state["rows"][:, :m].double()
        y = torch.zeros(state["x"].flatten(0, 1).shape[0], m, **double)
        out = {}
        if case["grad"]:
            drows, dweights = torch.zeros_like(rows), torch.zeros(t, k, **double)
        for i in range(k):
            here = (state["slots"][:, i] >= 0).nonzero()[:, 0]
            slot = state["slots"][here, i].long()
            w = state["weights"][here, i].double()[:, None]
            if case["grad"]:
                drows[slot] = w * x[here]
                dweights[here, i] = (rows[slot] * x[here]).sum(dim=1)
                y[here] += w * x[here]
            else:
                rows[slot] = x[here]
                y[here] += w * x[here]
        out["y"] = y.view(state["x"].shape[0], -1, m)
        return out | ({"drows": drows, "dweights": dweights} if case["grad"] else {"rows": rows})
    e, m, h = case["e"], case["m"], case["h"]
    sizes = state["sizes"].tolist()
    narrow, wide, w = state["narrow"][:, :m].double(), state["wide"][:, :h].double(), state["w"].flatten(0, 1)
    dw = torch.zeros(w.shape[0], m, h, **double) if case["way"] == "backward" else None
    at = 0
    for i, n in enumerate(sizes):
        mine, matrix = slice(at, at + n), w[i, :, :h].double()
        if case["way"] == "forward":
            wide[mine] = narrow[mine] @ matrix
            if case["relu"]:
                wide[mine] = wide[mine].clamp(min=0)
        else:
            if case["way"] == "backward":
                dw[i] = narrow[mine].t() @ wide[mine]
            narrow[mine] = wide[mine] @ matrix.t()
        at += n
    if case["way"] == "forward":
        return {"out": wide}
    if case["way"] == "input":
        return {"out": narrow}
    narrow[at:] = 0
    return {"drows": narrow, "dw": dw.view(state["dw"].shape[:-1] + (h,))}


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    t, k = case["t"], case.get("k", 1)
    if case["kind"] == "embed":
        rows = min(t, case["v"])
        return {"bytes": (rows + t) * case["m"] * size + t * 4, "flops": t * case["m"] if case["scaled"] else 0}
    if case["kind"] == "embed_grad":
        return {"bytes": (t + case["v"]) * case["m"] * size + t * 4, "flops": t * case["m"]}
    if case["kind"] == "route":
        logits = t * case["e"] * size
        return {"bytes": logits + t * k * 16 + case["e"] * 4 + (logits + t * k * 4 if case["grad"] else 0), "flops": 4 * t * case["e"]}
    if case["kind"] == "exchange":
        row = case["m"] * size
        if case["grad"]:
            return {"bytes": t * row + 2 * t * k * row + t * row + t * k * 12, "flops": 4 * t * k * case["m"]}
        return {"bytes": t * row + t * k * row + t * row + t * k * 12, "flops": 2 * t * k * case["m"]}
    s, e, m, h = t * k, case["e"], case["m"], case["h"]
    matrices = min(e, s) * m * h
    if case["way"] == "backward":
        return {"bytes": (s * (2 * m + h) + matrices + e * m * h) * size, "flops": 4 * s * m * h}
    return {"bytes": (s * (m + h) + matrices) * size, "flops": 2 * s * m * h}
