"""Cases for timing the losses over a vocabulary that is split on a mesh: softmax cross entropy and distillation from a
teacher's top logits, each with and without its gradients.

Activations x [T, M] (tokens split x ways) meet the vocabulary matrix w, [V, M] or [M, V] (vocabulary split y ways):
logits z = x w^T.  A token's loss is lse(z) - z[label], or, with teacher's entries (id, logit) of temperature tau, the
divergence of softmax(z / tau) from the softmax of the teacher's logits / tau over its entries.  With gradients a pass also
returns d(sum of weight * loss) with respect to x and w.

`listed()` names twelve cases, `draw(rng)` makes more of the same kinds with other sizes.
"""
import math

import torch

own = False


def listed():
    return [
        # the smallest call: float32, the vocabulary split unevenly over 4 partitions (23, 23, 23, 21 columns), with gradients
        {"name": "tiny_f32", "kind": "xent", "grad": True, "dtype": "f32", "t": 8, "m": 64, "v": 90, "x": 1, "y": 4, "order": "mv", "pad": False},
        # the log-probability of one token
        {"name": "score_one", "kind": "xent", "grad": False, "dtype": "bf16", "t": 1, "m": 2048, "v": 32000, "x": 1, "y": 1, "order": "vm", "pad": True},
        # 32 sequences' next tokens scored by a wide model
        {"name": "score_decode", "kind": "xent", "grad": False, "dtype": "bf16", "t": 32, "m": 8192, "v": 32000, "x": 1, "y": 1, "order": "mv", "pad": True},
        # evaluation of 8 sequences of 2048 tokens, on a 2 x 4 mesh
        {"name": "score_long", "kind": "xent", "grad": False, "dtype": "bf16", "t": 16384, "m": 2048, "v": 32000, "x": 2, "y": 4, "order": "vm", "pad": True},
        # a training step of one sequence
        {"name": "train_step", "kind": "xent", "grad": True, "dtype": "bf16", "t": 2048, "m": 2048, "v": 32000, "x": 1, "y": 1, "order": "vm", "pad": True},
        # a training step of 8 sequences of a wide model; the largest of the list
        {"name": "train_large", "kind": "xent", "grad": True, "dtype": "bf16", "t": 16384, "m": 8192, "v": 32000, "x": 1, "y": 1, "order": "mv", "pad": True},
        # packed sequences of any length, sizes that divide by nothing, dense rows, on a 2 x 4 mesh
        {"name": "train_uneven", "kind": "xent", "grad": True, "dtype": "bf16", "t": 1999, "m": 1001, "v": 32003, "x": 2, "y": 4, "order": "mv", "pad": False},
        # a model kept in float32
        {"name": "train_f32", "kind": "xent", "grad": True, "dtype": "f32", "t": 512, "m": 512, "v": 3000, "x": 1, "y": 2, "order": "vm", "pad": True},
        # a few tokens of a student, 64 entries of the teacher's each
        {"name": "distill_few", "kind": "distill", "grad": True, "dtype": "bf16", "t": 16, "m": 4096, "v": 32000, "k": 64, "tau": 1.0, "x": 1, "y": 1, "order": "vm", "pad": True},
        # a distillation step of two sequences, the vocabulary split over 4 partitions
        {"name": "distill_step", "kind": "distill", "grad": True, "dtype": "bf16", "t": 4096, "m": 2048, "v": 32000, "k": 32, "tau": 2.0, "x": 1, "y": 4, "order": "vm", "pad": True},
        # sizes that divide by nothing
        {"name": "distill_uneven", "kind": "distill", "grad": True, "dtype": "bf16", "t": 777, "m": 515, "v": 10007, "k": 21, "tau": 1.5, "x": 2, "y": 2, "order": "mv", "pad": False},
        # a student's distance from its teacher over a held-out text, a vocabulary of many languages
        {"name": "distill_score", "kind": "distill", "grad": False, "dtype": "bf16", "t": 1024, "m": 1024, "v": 128000, "k": 100, "tau": 1.0, "x": 1, "y": 1, "order": "vm", "pad": True},
    ]


def draw(rng):
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["xent", "xent", "distill"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    most = 16384 * 8192 * 32000 // (16 if dtype == "f32" else 1)
    while True:
        t, m, v = between(1, 16384), between(64, 8192), between(90, 128000)
        if t * m * v <= most and t * v <= 16384 * 32000:
            break
    whole = rng.random() < 0.5            # sizes of models, or any
    if whole:
        m, v = -(-m // 64) * 64, -(-v // 128) * 128
    case = {"kind": kind, "grad": rng.random() < 0.7, "dtype": dtype, "t": t, "m": min(m, 8192), "v": min(v, 128000), "x": rng.choice([1, 1, 2, 3]), "y": rng.choice([1, 1, 2, 4, 8]),
            "order": rng.choice(["vm", "mv"]), "pad": whole or rng.random() < 0.5}
    if kind == "distill":
        case["k"] = min(between(1, 128), v)
        case["tau"] = rng.choice([1.0, 2.0, 3.5])
    return case


def _up(n, to):
    return -(-n // to) * to


def _sizes(case):
    """Shard extents and row strides: tokens and vocabulary entries of a shard, row stride of x and of w."""
    ts, vs = -(-case["t"] // case["x"]), -(-case["v"] // case["y"])
    last = case["m"] if case["order"] == "vm" else vs
    return ts, vs, _up(case["m"], 8) if case["pad"] else case["m"], _up(last, 8) if case["pad"] else last


def _tokens(case, gen):
    """ids, teacher's logits (or none) and weights of the tokens; one in ten has no label or no entries."""
    t, v, k = case["t"], case["v"], case.get("k", 1)
    def rand(*shape):
        return torch.rand(shape, generator=gen, device="cuda")
    start = (rand(t, 1) * v).long().clamp_(max=v - 1)
    step = 1 + (rand(t, 1) * (v // k)).long().clamp_(max=v // k - 1)
    at = torch.arange(k, device="cuda")
    ids = (start + at * step) % v                                         # distinct: k * step is at most v
    kept = 1 + (rand(t, 1) * k).long().clamp_(max=k - 1)                  # entries that the teacher gives
    kept = torch.where(rand(t, 1) < 0.1, torch.zeros_like(kept), kept) if t > 1 else kept
    ids = torch.where(at < kept, ids, torch.full_like(ids, -1)).to(torch.int32)
    logits = None
    if case["kind"] == "distill":
        logits = torch.randn((t, k), generator=gen, device="cuda").mul_(2.0).sort(dim=1, descending=True).values
    weights = torch.full((t,), 1.0 / t, device="cuda") * (0.5 + rand(t))
    return ids, logits, weights


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    ts, vs, ldx, ldw = _sizes(case)
    t, m, v, na, nb = case["t"], case["m"], case["v"], case["x"], case["y"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    # shards one after the other in static shape; what lies beyond their valid part may hold anything
    x = torch.full((na * ts, ldx), float("nan"), dtype=dtype, device="cuda")
    x[:t, :m] = torch.randn((t, m), generator=gen, device="cuda").to(dtype)
    full = (torch.randn((v, m), generator=gen, device="cuda") * 0.05).to(dtype)
    if case["order"] == "vm":
        w = torch.full((nb, vs, ldw), float("nan"), dtype=dtype, device="cuda")
        w.view(nb * vs, ldw)[:v, :m] = full
    else:
        w = torch.full((nb, m, ldw), float("nan"), dtype=dtype, device="cuda")
        for j in range(nb):
            part = full[j * vs:(j + 1) * vs].t()
            w[j, :, :part.shape[1]] = part
    ids, logits, weights = _tokens(case, gen)
    k = ids.shape[1]
    state = {"case": case, "x": x.view(na, ts, ldx), "w": w}
    state["ids"] = torch.full((na * ts, k), -1, dtype=torch.int32, device="cuda")
    state["ids"][:t] = ids
    state["weights"] = torch.zeros(na * ts, device="cuda")
    state["weights"][:t] = weights
    state["logits"] = None
    if logits is not None:
        state["logits"] = torch.full((na * ts, k), float("nan"), device="cuda")
        state["logits"][:t] = logits
    # what a user's program keeps: output buffers, and with the framework its descriptions of the shards and a workspace
    state["loss"], state["lse"] = torch.empty(na * ts, device="cuda"), torch.empty(na * ts, device="cuda")
    if case["grad"]:
        state["dx"], state["dw"] = torch.empty_like(state["x"]), torch.empty_like(w)
    if own:
        state["call"] = _call(state)
    return state


def _call(state):
    """The framework's call on these shards, its arguments made once as a training loop would."""
    import paper_2105_04663_amd as g

    case, x, w = state["case"], state["x"], state["w"]
    ts, vs, ldx, ldw = _sizes(case)
    na, nb, k = case["x"], case["y"], state["ids"].shape[1]
    mesh = g.Mesh((na, nb), tuple(range(na * nb)))
    vocab_dim = 0 if case["order"] == "vm" else 1
    x_sh = g.Sharding((case["t"], case["m"]), (0, -1))
    w_sh = g.Sharding((case["v"], case["m"]), (1, -1)) if vocab_dim == 0 else g.Sharding((case["m"], case["v"]), (-1, 1))
    places = [(i, j) for i in range(na) for j in range(nb)]
    bufs = lambda a, ld, which: [g.ShardBuf.of(a[p[which]], ld) for p in places]
    def tokens(i):
        at = lambda a, per: 0 if a is None else a.data_ptr() + i * ts * per * 4
        return g.TokenBuf(ids=at(state["ids"], k), loss=at(state["loss"], 1), lse=at(state["lse"], 1), weights=at(state["weights"], 1), logits=at(state["logits"], k))
    args = dict(vocab_dim=vocab_dim, dx_shards=None, dw_shards=None)
    if case["grad"]:
        args.update(dx_shards=bufs(state["dx"], ldx, 0), dw_shards=bufs(state["dw"], ldw, 1))
    size = g.softmax_workspace_bytes(mesh, x_sh, w_sh, vocab_dim, g.BF16 if case["dtype"] == "bf16" else g.F32, case["grad"])
    state["space"] = torch.empty(size + 256, dtype=torch.uint8, device="cuda")
    base = _up(state["space"].data_ptr(), 256)
    first = (mesh, bufs(x, ldx, 0), x_sh, bufs(w, ldw, 1), w_sh, [tokens(i) for i, _ in places])
    args.update(workspace=base, workspace_bytes=size)
    if case["kind"] == "xent":
        return lambda: g.softmax_xent(*first, stream=torch.cuda.current_stream().cuda_stream, **args)
    return lambda: g.softmax_distill(*first, k, case["tau"], stream=torch.cuda.current_stream().cuda_stream, **args)


def run(state):
    case = state["case"]
    if own:
        state["call"]()
    else:
        _plain(state)
    out = {"loss": state["loss"], "lse": state["lse"]}
    if case["grad"]:
        ts, vs, _, _ = _sizes(case)
        out["dx"] = state["dx"][:, :, :case["m"]]
        out["dw"] = state["dw"][:, :, :case["m"] if case["order"] == "vm" else vs]
    return out


def _plain(state):
    """The definition in elementary float32 operations, every result written to the state's buffers."""
    case = state["case"]
    ts, vs, ldx, ldw = _sizes(case)
    t, m, v, na, nb = case["t"], case["m"], case["v"], case["x"], case["y"]
    x = state["x"].view(na * ts, ldx)[:t, :m].float()
    vm = case["order"] == "vm"
    w = state["w"].view(nb * vs, ldw)[:v, :m].float() if vm else state["w"][:, :, :vs].permute(1, 0, 2).reshape(m, nb * vs)[:, :v].float()
    tau = case.get("tau", 1.0)
    z = x @ (w.t() if vm else w)
    if tau != 1.0:
        z = z / tau
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    ids = state["ids"][:t].long()
    there = (ids >= 0) & (ids < v)
    at = torch.where(there, ids, torch.zeros_like(ids))
    if case["kind"] == "xent":
        p = there.float()
        loss = torch.where(there, lse - z.gather(1, at), torch.zeros_like(lse)).sum(dim=1)
    else:
        q = torch.where(there, state["logits"][:t] / tau, torch.full_like(state["logits"][:t], -math.inf))
        most = q.amax(dim=1, keepdim=True)
        most = torch.where(most > -math.inf, most, torch.zeros_like(most))
        shares = torch.exp(q - most)
        sums = shares.sum(dim=1, keepdim=True)
        sums = torch.where(sums > 0, sums, torch.ones_like(sums))
        p = shares / sums
        terms = p * (q - most - torch.log(sums) - z.gather(1, at) + lse)
        loss = torch.where(p > 0, terms, torch.zeros_like(p)).sum(dim=1)
    state["loss"].zero_()
    state["lse"].zero_()
    state["loss"][:t] = loss
    state["lse"][:t] = lse[:, 0]
    if not case["grad"]:
        return
    scale = torch.where(p.amax(dim=1, keepdim=True) > 0, state["weights"][:t, None] / tau, torch.zeros_like(lse))
    d = e * (scale / total)
    d.scatter_add_(1, at, -p * scale)
    state["dx"].view(na * ts, ldx)[:, :m] = 0
    state["dx"].view(na * ts, ldx)[:t, :m] = d @ (w if vm else w.t())
    state["dw"][:, :, :m if vm else vs] = 0
    if vm:
        state["dw"].view(nb * vs, ldw)[:v, :m] = d.t() @ x
    else:
        dw = torch.zeros((m, nb * vs), device="cuda")
        dw[:, :v] = x.t() @ d
        state["dw"][:, :, :vs] = dw.view(m, nb, vs).permute(1, 0, 2)


def exact(case, seed):
    """What run() returns, in float64, a block of tokens at a time."""
    state = prepare(case, seed)
    state.pop("call", None)
    ts, vs, ldx, ldw = _sizes(case)
    t, m, v, na, nb = case["t"], case["m"], case["v"], case["x"], case["y"]
    x = torch.cat([state["x"][i, :, :m] for i in range(na)])[:t].double()
    if case["order"] == "vm":
        w = torch.cat([state["w"][j, :, :m] for j in range(nb)])[:v].double()
    else:
        w = torch.cat([state["w"][j, :, :vs].t() for j in range(nb)])[:v].double().contiguous()
    loss, lse = torch.zeros(na * ts, dtype=torch.float64, device="cuda"), torch.zeros(na * ts, dtype=torch.float64, device="cuda")
    dx, dw = torch.zeros((na * ts, m), dtype=torch.float64, device="cuda"), torch.zeros((nb * vs, m), dtype=torch.float64, device="cuda")
    tau = case.get("tau", 1.0)
    block = max(1, min(2048, (1 << 27) // v))
    for a in range(0, t, block):
        b = min(t, a + block)
        u = (x[a:b] @ w.t()) / tau
        lse[a:b] = torch.logsumexp(u, dim=1)
        ids = state["ids"][a:b].long()
        target = torch.zeros_like(u)
        rows = torch.arange(b - a, device="cuda")
        for n in range(ids.shape[1]):
            here = (ids[:, n] >= 0) & (ids[:, n] < v)
            share = torch.ones(b - a, dtype=torch.float64, device="cuda")
            if case["kind"] == "distill":
                masked = torch.where((ids >= 0) & (ids < v), state["logits"][a:b].double() / tau, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
                share = torch.exp(masked[:, n] - torch.logsumexp(masked, dim=1))
            r = rows[here]
            target[r, ids[here, n]] += share[here]
            loss[a:b][here] += share[here] * (torch.log(share[here]) - u[r, ids[here, n]] + lse[a:b][here])
        if case["grad"]:
            d = torch.softmax(u, dim=1) - target
            d *= (torch.where((target > 0).any(dim=1), state["weights"][a:b].double(), torch.zeros(b - a, dtype=torch.float64, device="cuda")) / tau)[:, None]
            dx[a:b] = d @ w
            dw[:v] += d.t() @ x[a:b]
    out = {"loss": loss, "lse": lse}
    if case["grad"]:
        out["dx"] = dx.view(na, ts, m)
        out["dw"] = dw.view(nb, vs, m) if case["order"] == "vm" else dw.view(nb, vs, m).permute(0, 2, 1)
    return out


def work(case):
    t, m, v, k = case["t"], case["m"], case["v"], case.get("k", 1)
    size = 2 if case["dtype"] == "bf16" else 4
    operands = (t * m + v * m) * size
    entries = t * k * (8 if case["kind"] == "distill" else 4)
    return {"bytes": operands * (2 if case["grad"] else 1) + entries + t * (12 if case["grad"] else 8), "flops": (6 if case["grad"] else 2) * t * m * v}
