"""Operators that choose by a token's index on tensors of more than 2^31 elements: rows, columns and slots that lie beyond, compared on the GPU with torch's own indexing."""
import pytest
import torch

import paper_2105_04663_amd as g
from tests.tokens import KEPT, stream

pytestmark = pytest.mark.gpu
ONE = g.Mesh((1,), (0,))


def space(n):
    t = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    return t, (t.data_ptr() + 255) // 256 * 256


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("order", ["vm", "mv"])
def test_embedding(order):
    """Matrices of 2.4 and 2.8 billion elements: entries in the first, the middle and the last rows or columns."""
    V, M = (300000, 8192) if order == "vm" else (40000, 70000)
    shape = (V, M) if order == "vm" else (M, V)
    w = torch.randint(-2 ** 14, 2 ** 14, shape, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    ids = torch.tensor([0, V - 1, V - 2, V // 2, -1, 262143 % V, 262144 % V, V - 1], dtype=torch.int32, device="cuda")
    T, there = len(ids), ids >= 0
    rows_sh, w_sh, dim = g.Sharding((T, M), (-1, -1)), g.Sharding(shape, (-1, -1)), 0 if order == "vm" else 1
    y = torch.full((T, M), KEPT, dtype=torch.bfloat16, device="cuda")
    g.embed(ONE, [ids.data_ptr()], [g.ShardBuf.of(w, shape[1])], w_sh, [g.ShardBuf.of(y, M)], rows_sh, vocab_dim=dim, stream=stream())
    want = (w if order == "vm" else w.t())[ids.long().clamp(min=0)].contiguous()
    assert torch.equal(y[there].view(torch.int16), want[there].view(torch.int16)) and (y[~there] == 0).all()
    del want
    w.fill_(KEPT)
    dy = torch.randint(-8, 9, (T, M), device="cuda").bfloat16()
    n = g.embed_grad_workspace_bytes(ONE, rows_sh, w_sh, dim, g.BF16)
    keep, at = space(n)
    g.embed_grad(ONE, [ids.data_ptr()], [g.ShardBuf.of(dy, M)], rows_sh, [g.ShardBuf.of(w, shape[1])], w_sh, vocab_dim=dim, workspace=at, workspace_bytes=n, stream=stream())
    dw = w if order == "vm" else w.t()
    used = ids[there].unique().long()
    for v in used.tolist():
        assert torch.equal(dw[v].float(), dy[ids == v].float().sum(dim=0)), v
    nonzero = sum(int((part != 0).sum()) for part in w.split(8192))
    assert nonzero == sum(int((dw[v] != 0).sum()) for v in used.tolist())


def test_exchange_and_products():
    """600000 slots of 4096: rows behind the 2^31st element go where they belong and back."""
    T, k, E, M, H = 300000, 2, 8, 4096, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(T, E, generator=gen, device="cuda")
    ints = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")
    experts, slots, order, sizes, weights = ints(T, k), ints(T, k), ints(T * k), ints(E), torch.zeros(T, k, device="cuda")
    buf = g.RouteBuf(experts.data_ptr(), weights.data_ptr(), slots.data_ptr(), order.data_ptr(), sizes.data_ptr())
    sh = g.Sharding((T, E), (-1, -1))
    n = g.route_workspace_bytes(ONE, sh, k)
    keep, at = space(n)
    g.route(ONE, [g.ShardBuf.of(logits, E)], sh, k, buf, normalise=True, workspace=at, workspace_bytes=n, stream=stream())
    assert torch.equal(experts.long(), logits.topk(k, dim=1).indices) and int(sizes.sum()) == T * k
    x = torch.randint(-64, 65, (T, M), device="cuda", dtype=torch.int8).bfloat16()
    rows = torch.full((T * k, M), KEPT, dtype=torch.bfloat16, device="cuda")
    x_sh, r_sh, one = g.Sharding((T, M), (-1, -1)), g.Sharding((E, T * k, M), (-1, -1, -1)), lambda t: [g.ShardBuf.of(t, t.shape[-1])]
    g.dispatch(ONE, one(x), x_sh, k, buf, one(rows), r_sh, stream=stream())
    for t in range(0, T, 50000):
        for i in range(k):
            assert torch.equal(rows[slots[t:t + 50000, i].long()], x[t:t + 50000])
    y = torch.full((T, M), KEPT, dtype=torch.bfloat16, device="cuda")
    g.combine(ONE, one(rows), r_sh, k, buf, one(y), x_sh, weighted=False, stream=stream())
    assert torch.equal(y, x + x)
    drows, dweights = torch.full((T * k, M), KEPT, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, k, device="cuda")
    g.combine_grad(ONE, one(x), x_sh, one(rows), r_sh, k, buf, one(drows), dweights.data_ptr(), stream=stream())
    last = slice(T - 1000, T)
    for i in range(k):
        assert torch.equal(drows[slots[last, i].long()], (x[last].float() * weights[last, i:i + 1]).bfloat16())
    assert not (drows == KEPT).all(dim=1).any()
    assert torch.equal(dweights, x.float().square().sum(dim=1, keepdim=True).expand(T, k))          # whole numbers below 2^24
    del drows, y
    w = torch.randint(-2, 3, (E, M, H), device="cuda").bfloat16()
    out = torch.full((T * k, H), KEPT, device="cuda")
    dims = g.DotDims((0,), (0,), (2,), (1,))
    w_sh, o_sh = g.Sharding((E, M, H), (-1, -1, -1)), g.Sharding((E, T * k, H), (-1, -1, -1))
    g.ragged_dot(ONE, dims, one(rows), r_sh, one(w), w_sh, one(out), o_sh, sizes.data_ptr(), stream=stream())
    ends = torch.cumsum(sizes.long(), 0).tolist()
    for e in range(E):
        for a, b in (((ends[e - 1] if e else 0), (ends[e - 1] if e else 0) + 300), (ends[e] - 300, ends[e])):
            assert torch.equal(out[a:b], rows[a:b].float() @ w[e].float())                          # whole numbers below 2^24


def test_as_many_choices_as_there_may_be():
    """2^24 tokens with a choice each: the routing's order, and the gradient of an embedding of as many."""
    T, E = 1 << 24, 6
    gen = torch.Generator(device="cuda").manual_seed(2)
    logits = torch.randint(-4, 5, (T, E), generator=gen, device="cuda").float()
    logits[5::1001] = -float("inf")
    ints = lambda *s: torch.full(s, -7, dtype=torch.int32, device="cuda")
    experts, slots, order, sizes, weights = ints(T, 1), ints(T, 1), ints(T), ints(E), torch.zeros(T, 1, device="cuda")
    buf = g.RouteBuf(experts.data_ptr(), weights.data_ptr(), slots.data_ptr(), order.data_ptr(), sizes.data_ptr())
    sh = g.Sharding((T, E), (-1, -1))
    n = g.route_workspace_bytes(ONE, sh, 1)
    keep, at = space(n)
    g.route(ONE, [g.ShardBuf.of(logits, E)], sh, 1, buf, normalise=True, workspace=at, workspace_bytes=n, stream=stream())
    most, there = logits.amax(dim=1), logits[:, 0] != -float("inf")
    want = torch.where(there, (logits == most[:, None]).int().argmax(dim=1), torch.full((T,), E, device="cuda"))
    assert torch.equal(experts[:, 0].long(), torch.where(there, want, torch.full_like(want, -1)))
    by_expert = torch.argsort(want, stable=True)
    total = int(there.sum())
    assert torch.equal(order[:total].long(), by_expert[:total]) and (order[total:] == -1).all()
    assert torch.equal(sizes.long(), torch.bincount(want, minlength=E + 1)[:E])
    assert torch.equal(slots[by_expert[:total], 0].long(), torch.arange(total, device="cuda")) and (slots[~there] == -1).all()
    assert (weights[there] == 1).all() and (weights[~there] == 0).all()
    del by_expert, want, logits
    V, M = 50, 2
    ids = torch.randint(-1, V + 1, (T,), generator=gen, device="cuda", dtype=torch.int32)
    dy = torch.ones(T, M, device="cuda")
    dy[:, 1] = -0.5
    dw = torch.full((V, M), KEPT, device="cuda")
    rows_sh, w_sh = g.Sharding((T, M), (-1, -1)), g.Sharding((V, M), (-1, -1))
    n = g.embed_grad_workspace_bytes(ONE, rows_sh, w_sh, 0, g.F32)
    keep, at = space(n)
    g.embed_grad(ONE, [ids.data_ptr()], [g.ShardBuf.of(dy, M)], rows_sh, [g.ShardBuf.of(dw, M)], w_sh, workspace=at, workspace_bytes=n, stream=stream())
    count = torch.bincount(ids[(ids >= 0) & (ids < V)].long(), minlength=V).float()
    assert torch.equal(dw[:, 0], count) and torch.equal(dw[:, 1], -0.5 * count)                      # whole numbers below 2^24
