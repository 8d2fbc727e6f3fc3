"""gspmd_embed and gspmd_embed_grad on the GPU against their definitions in float64."""
import pytest
import torch

import paper_2105_04663_amd as g
from tests.tokens import Embed

pytestmark = pytest.mark.gpu
ORDERS = ["vm", "mv"]


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T, M, V", [(1, 8, 5), (1, 2048, 300), (5, 64, 90), (7, 1, 3), (33, 515, 1000), (64, 72, 1), (130, 130, 4097), (200, 4100, 50), (3, 9, 70000)])
def test_lookup(order, dtype, T, M, V):
    for kw in (dict(scale=1.0, pad=True), dict(scale=11.3137, pad=False, shift=1), dict(scale=-0.5, pad=False), dict(scale=0.0, pad=True, x=2, y=3, copies=2)):
        e = Embed(T, M, V, order=order, dtype=dtype, **kw).stage_lookup()
        e.lookup()
        e.check_lookup()


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("x, y, copies", [(1, 4, 1), (3, 1, 1), (2, 4, 2), (5, 3, 3), (4, 16, 1), (64, 1, 1), (1, 64, 1)])
def test_lookup_over_a_mesh(order, x, y, copies):
    """Uneven splits, shards that lie behind the last token or entry, a buffer for every replica."""
    e = Embed(21, 48, 37, x=x, y=y, order=order, copies=copies, seed=1).stage_lookup()
    e.lookup()
    e.check_lookup()


def test_lookup_copies_bits():
    """NaN, infinities, zeros and numbers below normal of the row that is read, and nothing of others."""
    e = Embed(4, 16, 8, ids=torch.tensor([2, -1, 5, 2 ** 31 - 1]))
    e.w[2, :6] = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0, 1e-40, 3.0]).bfloat16()
    e.stage_lookup().lookup()
    got = e.yc.whole()
    assert torch.equal(got[0].view(torch.int16), e.w[2].view(torch.int16)) and torch.equal(got[2], e.w[5])
    assert (got[[1, 3]] == 0).all()


IDS = {"uniform": None, "one entry": lambda T, V: torch.full((T,), V - 1), "none": lambda T, V: torch.full((T,), -1), "two": lambda T, V: torch.arange(T) % 2 * (V - 1),
       "half one": lambda T, V: torch.where(torch.arange(T) % 2 == 0, torch.zeros(T, dtype=torch.int64), torch.arange(T) * 31 % V)}


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ids", sorted(IDS))
@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 129, 300, 1025])
def test_gradient(order, dtype, ids, T):
    for M, V, kw in ((40, 50, dict()), (515, 333, dict(pad=False, scale=3.25)), (8, 1, dict(accumulate=True)), (72, 130, dict(accumulate=True, pad=False, shift=1, scale=0.125))):
        e = Embed(T, M, V, order=order, dtype=dtype, ids=IDS[ids](T, V) if IDS[ids] else None, **kw).stage_gradient()
        e.gradient()
        e.check_gradient()


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("x, y, copies", [(1, 4, 1), (3, 1, 1), (2, 4, 2), (5, 3, 3), (4, 16, 1), (64, 1, 1), (1, 64, 1)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_over_a_mesh(order, x, y, copies, accumulate):
    e = Embed(150, 56, 37, x=x, y=y, order=order, copies=copies, accumulate=accumulate, seed=2).stage_gradient()
    e.gradient()
    e.check_gradient()


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("T, V", [(4096, 1023), (4097, 1024), (12288, 32000), (12289, 500), (12289, 70000), (30000, 1025), (70000, 128000)])
def test_gradient_of_long_texts(order, T, V):
    """Sorted by one workgroup and by many, with keys of one digit and of two; an entry that is a quarter of the text."""
    ids = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(T))
    ids[::4] = min(17, V - 1)
    ids[5] = -3
    e = Embed(T, 24, V, x=3, y=2, order=order, ids=ids, seed=3).stage_gradient()
    e.gradient()
    e.check_gradient()


@pytest.mark.parametrize("order", ORDERS)
def test_gradient_of_wide_rows(order):
    for dtype, M in (("bf16", 4360), ("f32", 2100)):
        e = Embed(200, M, 70, order=order, dtype=dtype, ids=torch.arange(200) * 7 % 3 * 20, seed=4).stage_gradient()
        e.gradient()
        e.check_gradient()


def test_nothing():
    e = Embed(0, 16, 20, y=2).stage_lookup().stage_gradient()
    e.lookup()
    e.gradient()
    e.check_gradient()
    e = Embed(6, 0, 20).stage_lookup().stage_gradient()
    e.lookup()
    e.gradient()


def test_gradient_is_the_lookups():
    """sum of c * y in whole numbers: its difference along a direction of w is the product with dw."""
    e = Embed(60, 24, 17, dtype="f32", scale=2.0, seed=5)
    c = torch.randint(-4, 5, (60, 24)).float()
    e.w, d = torch.randint(-4, 5, (17, 24)).float(), torch.randint(-4, 5, (17, 24)).float()
    def loss(w):
        e.w = w
        e.stage_lookup().lookup()
        return (e.yc.whole().double() * c).sum()
    base = e.w
    e.dy = c
    e.stage_gradient().gradient()
    assert (loss(base + d) - loss(base - d)) / 2 == (e.dwc.whole().double() * d).sum()


@pytest.mark.parametrize("order", ORDERS)
def test_graph(order):
    """Replays with other ids and rows, eager work between."""
    e = Embed(700, 72, 300, order=order, y=2, x=2, seed=6).stage_lookup().stage_gradient()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        e.lookup()
        e.gradient()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        e.lookup()
        e.gradient()
    for turn in range(4):
        e.ids = torch.randint(-1, 301, (700,), generator=torch.Generator().manual_seed(turn)) if turn < 3 else torch.full((700,), 9)
        e.ids_t[:700].copy_(e.ids.int())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        e.check_lookup()
        e.check_gradient()
        first = [t.clone() for t in e.dwc.t[0]]
        e.gradient()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, e.dwc.t[0]))


def test_after_the_loss():
    """One matrix at both ends: the loss's gradient with respect to it, and the embedding's added."""
    e = Embed(48, 64, 90, y=2, dtype="f32", seed=7, accumulate=True).stage_gradient()
    x = Embed(48, 64, 90, y=2, dtype="f32", seed=8)
    x.scale = 1.0
    loss, label = torch.empty(48, device="cuda"), torch.randint(0, 90, (48,), dtype=torch.int32, device="cuda")
    wc, xc, dxc = x.vocab(x.w), x.cut(x.dy, 1), x.cut(torch.zeros(48, 64), 1)
    n = g.softmax_workspace_bytes(e.mesh, e.rows_sh, e.w_sh, 0, g.F32, True)
    space = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    def of_loss():
        g.softmax_xent(e.mesh, [xc.buf(0)] * 2, e.rows_sh, [wc.buf(j) for _, j in x.places], e.w_sh, [g.TokenBuf(label.data_ptr(), loss.data_ptr())] * 2, dx_shards=[dxc.buf(0)] * 2,
                       dw_shards=e.dw_bufs, workspace=(space.data_ptr() + 255) // 256 * 256, workspace_bytes=n, stream=torch.cuda.current_stream().cuda_stream)
    of_loss()
    torch.cuda.synchronize()
    e.w = e.dwc.whole()[:90].clone()
    e.gradient()
    e.check_gradient()


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("ids", sorted(IDS))
@pytest.mark.parametrize("T", [8192, 8193, 16399])
def test_gradient_of_many_tokens(order, ids, T):
    """Chunks of either size; runs that begin and end in them, at their ends and beyond them; rows shorter than 16 bytes, that divide by them or not, written or added to."""
    for M, kw in ((5, dict()), (40, dict(accumulate=True)), (515, dict(pad=False, scale=0.5)), (515, dict(accumulate=True, pad=False, shift=1))):
        e = Embed(T, M, 333, order=order, ids=IDS[ids](T, 333) if IDS[ids] else None, seed=9, **kw).stage_gradient()
        e.gradient()
        e.check_gradient()


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("V", [131072, 131073, 600000])
def test_gradient_of_large_vocabularies(order, V):
    """Ranges of up to 1024 entries for a workgroup, and more workgroups than there are compute units."""
    for T in (100, 9000):
        ids = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(V))
        ids[::7], ids[3], ids[5] = V - 1, V, -1
        for accumulate in (False, True):
            e = Embed(T, 8, V, y=3, order=order, ids=ids, accumulate=accumulate, seed=10).stage_gradient()
            e.gradient()
            e.check_gradient()


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [2, 3, 4, 6, 7, 9, 127, 128, 129, 255, 256, 257, 264, 511, 512, 520, 1023, 2047, 2049])
def test_ends_of_rows(order, dtype, M):
    for kw in (dict(pad=False), dict(pad=True, accumulate=True), dict(pad=False, shift=1, accumulate=True, x=2, y=2)):
        e = Embed(37, M, 23, order=order, dtype=dtype, seed=11, scale=1.5, **kw).stage_lookup().stage_gradient()
        e.lookup()
        e.check_lookup()
        e.gradient()
        e.check_gradient()


@pytest.mark.parametrize("order", ORDERS)
def test_two_streams_at_once(order):
    """Two gradients with workspaces of their own, side by side, many times over: the bits of one alone."""
    both = [Embed(3000, 264, 900, order=order, seed=s, y=2).stage_gradient() for s in (12, 13)]
    alone = []
    for e in both:
        e.gradient()
        torch.cuda.synchronize()
        e.check_gradient()
        alone.append([t.clone() for t in e.dwc.t[0]])
        for t in e.dwc.t[0]:
            t[:, :e.dwc.cols] = 55.0
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(8):
        for e, s in zip(both, streams):
            with torch.cuda.stream(s):
                e.gradient()
    torch.cuda.synchronize()
    for e, want in zip(both, alone):
        assert all(torch.equal(a, b) for a, b in zip(e.dwc.t[0], want))


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_scale_of_one_copies_any_bits(order, dtype):
    """Every pattern of 16 bits, and float32 ones of each kind: signalling NaN with their payloads among them."""
    if dtype == "bf16":
        w = torch.arange(-2 ** 15, 2 ** 15, dtype=torch.int32).to(torch.int16).view(64, 1024)
    else:
        w = (torch.arange(2 ** 16, dtype=torch.int64) * 65537 + 2 ** 23 * 255 - 7).to(torch.int32).view(64, 1024)
    e = Embed(64, 1024, 64, order=order, dtype=dtype, ids=torch.arange(64) * 37 % 64)
    e.w = w.view(torch.bfloat16 if dtype == "bf16" else torch.float32)
    e.stage_lookup().lookup()
    got = e.yc.whole()[:64]
    assert torch.equal(got.view(w.dtype), w[e.ids])


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("ids", sorted(IDS))
@pytest.mark.parametrize("T", [7, 8, 9, 15, 16, 17, 24, 33, 100, 127, 128, 136])
def test_gradient_of_few_tokens(order, ids, T):
    """Runs that are added up by the chunk they begin in, over several others, in rows of each kind."""
    for M, kw in ((5, dict()), (40, dict(accumulate=True)), (515, dict(pad=False, scale=0.5)), (515, dict(accumulate=True, pad=False, shift=1)), (1024, dict(x=3, y=2))):
        e = Embed(T, M, 29, order=order, ids=IDS[ids](T, 29) if IDS[ids] else None, seed=14, **kw).stage_gradient()
        e.gradient()
        e.check_gradient()
