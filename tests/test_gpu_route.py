"""gspmd_route, gspmd_dispatch, gspmd_combine and their gradients on the GPU, each against its definition in float64, and the layer that they make with gspmd_ragged_dot."""
import pytest
import torch

import paper_2105_04663_amd as g
from tests.ragged import DIMS, BACK, FORWARD, WEIGHT
from tests.tokens import HALF, KEPT, NAN, TYPES, Cut, Embed, Routed, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("normalise", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T, E, k", [(1, 1, 1), (1, 64, 8), (2, 5, 5), (3, 16, 16), (17, 17, 2), (40, 33, 4), (65, 64, 1), (64, 128, 8), (9, 129, 3), (100, 257, 16), (50, 512, 7), (700, 6, 2), (2000, 60, 4)])
def test_route(normalise, dtype, T, E, k):
    for kw in (dict(), dict(ties=True, x=2), dict(masked=0.7, pad=False, x=3)):
        r = Routed(T, E, k, dtype=dtype, normalise=normalise, **kw).stage()
        r.call()
        r.check()


@pytest.mark.parametrize("T, E, k", [(256, 4, 1), (257, 4, 1), (512, 300, 2), (513, 300, 2), (1536, 40, 8), (1537, 40, 8), (20000, 512, 2), (6000, 3, 3), (40000, 31, 16)])
def test_route_orders_any_number_of_choices(T, E, k):
    """Sorted by workgroups of each size, and by many."""
    r = Routed(T, E, k, ties=True, masked=0.2, seed=1).stage()
    r.call()
    r.check()


def test_route_strange_logits():
    """NaN is never chosen and makes weights over all experts NaN; +infinity is chosen first."""
    for normalise in (False, True):
        r = Routed(4, 20, 3, masked=0.0, normalise=normalise, seed=2)
        r.z[0, 4], r.z[1, 7], r.z[2] = NAN, float("inf"), NAN
        r.stage().call()
        experts, weights = r.experts.cpu(), r.weights.cpu()
        clean = r.z[0].clone()
        clean[4] = -float("inf")
        assert experts[0].tolist() == clean.argsort(descending=True)[:3].tolist()
        assert torch.isnan(weights[0]).all() != normalise and (normalise or torch.isnan(weights[0]).all())
        assert experts[1, 0] == 7 and torch.isnan(weights[1, 0])
        assert (experts[2] == -1).all() and (weights[2] == 0).all() and (r.slots.cpu()[2] == -1).all()
        assert torch.isfinite(weights[3]).all() and r.sizes.sum() == 9


def test_no_tokens():
    r = Routed(0, 12, 3).stage()
    r.call()
    torch.cuda.synchronize()
    assert (r.sizes == 0).all()


@pytest.mark.parametrize("normalise", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T, E, k, x, copies", [(1, 1, 1, 1, 1), (5, 8, 3, 2, 2), (33, 40, 8, 1, 1), (70, 100, 2, 3, 1), (20, 300, 16, 1, 3), (130, 512, 4, 4, 1)])
def test_route_gradient(normalise, dtype, T, E, k, x, copies):
    r = Routed(T, E, k, x=x, dtype=dtype, normalise=normalise, copies=copies, seed=3).stage()
    r.call()
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(T))
    d = Cut(torch.full((T, E), KEPT, dtype=r.dtype), x, fill=KEPT, copies=copies)
    given = torch.where(r.experts[:T].cpu() >= 0, dw, torch.full_like(dw, NAN)).cuda()          # what is given for no expert is not read
    g.route_grad(r.mesh, r.z_bufs, r.sh, k, r.buf, given.data_ptr(), [d.buf(i, c) for i, c in r.places], normalise=normalise, stream=stream())
    for c in range(copies):
        r.check_gradient(dw, d, c)


def test_route_gradient_against_differences():
    """sum of g * weights along a direction of the logits, by central differences of the definition in float64 at the library's choices."""
    for normalise in (False, True):
        r = Routed(12, 24, 4, masked=0.0, normalise=normalise, seed=4).stage()
        r.call()
        gen = torch.Generator().manual_seed(5)
        dw, along = torch.randn(12, 4, generator=gen), torch.randn(12, 24, generator=gen).double()
        d = Cut(torch.zeros(12, 24), 1)
        given = dw.cuda()
        g.route_grad(r.mesh, r.z_bufs, r.sh, 4, r.buf, given.data_ptr(), [d.buf(0)], normalise=normalise, stream=stream())
        z, experts = r.z.double(), r.experts.cpu().long()
        live = experts[:, 0] >= 0
        def value(z):
            s = torch.exp(z).gather(1, experts.clamp(min=0))
            return (s / (s.sum(dim=1, keepdim=True) if normalise else torch.exp(z).sum(dim=1, keepdim=True)) * dw)[live].sum()
        h = 1e-5
        slope = (value(torch.where(live[:, None], z, torch.zeros_like(z)) + h * along) - value(torch.where(live[:, None], z, torch.zeros_like(z)) - h * along)) / (2 * h)
        got = (d.whole().double() * along)[live].sum()
        assert abs(got - slope) <= 1e-8 * 1e5 * h + (24 + 80) * 2.0 ** -23 * along.abs().sum() * dw.abs().max()


class Exchange:
    """A routing, tokens' rows x and experts' rows, the latter in one buffer or one for each shard of the experts in which all but its own slots are NaN."""

    def __init__(self, T, E, k, M, x=1, y=1, dtype="bf16", share=True, pad=True, shift=0, copies=1, seed=0):
        self.r = Routed(T, E, k, masked=0.15, seed=seed).stage()
        self.r.call()
        self.r.check()
        self.experts, self.weights, self.slots, self.order, self.sizes = self.r.expected()
        self.weights = self.r.weights[:T].cpu()                                 # the operators' input
        self.T, self.E, self.k, self.M, self.x, self.y, self.share, self.copies = T, E, k, M, x, y, share, copies
        self.dtype = TYPES[dtype]
        self.pad, self.shift = pad, shift
        self.mesh = g.Mesh((x, y), tuple(range(x * y)))
        self.places = [(i, j) for i in range(x) for j in range(y)]
        gen = torch.Generator().manual_seed(seed + 99)
        self.tok, self.rows = torch.randn(T, M, generator=gen).to(self.dtype), torch.randn(T * k, M, generator=gen).to(self.dtype)
        self.x_sh, self.rows_sh = g.Sharding((T, M), (0, -1)), g.Sharding((E, T * k, M), (1, -1, -1))
        self.es = -(-E // y)
        ends = torch.cumsum(self.sizes, 0)
        self.total = int(ends[-1])
        self.owner = torch.searchsorted(ends, torch.arange(T * k), right=True) // self.es      # of a slot: its expert's shard
        self.owner[self.total:] = -1

    def tokens(self, full, fill=NAN, copies=1):
        return Cut(full, self.x, pad=self.pad, shift=self.shift, fill=fill, copies=copies)

    def packed(self, full, fill=NAN, copies=1):
        """Buffers of the packed rows: one for all, or one for each shard of the experts."""
        if self.share:
            return [Cut(torch.where((self.owner >= 0)[:, None], full, torch.full_like(full, fill)), 1, pad=self.pad, shift=self.shift, fill=fill, copies=1)]
        return [Cut(torch.where((self.owner == j)[:, None], full, torch.full_like(full, fill)), 1, pad=self.pad, shift=self.shift, fill=fill, copies=copies) for j in range(self.y)]

    def bufs(self, packed, copies=1):
        return [packed[0].buf(0) if self.share else packed[j].buf(0, i % copies) for i, j in self.places]

    def check_packed(self, packed, want, most, copies=1):
        for j, cut in enumerate(packed):
            for c in range(1 if self.share else copies):
                got = cut.whole(c).double()
                mine = self.owner >= 0 if self.share else self.owner == j
                assert ((got - want).abs() <= most)[mine].all()
                assert (got[~mine] == KEPT).all() and (cut.gaps(c) == KEPT).all()


CASES = [dict(T=1, E=4, k=2, M=64), dict(T=7, E=3, k=3, M=1), dict(T=33, E=10, k=4, M=515, pad=False), dict(T=64, E=8, k=1, M=8, dtype="f32"), dict(T=130, E=40, k=8, M=72, x=3, y=4),
         dict(T=50, E=5, k=2, M=260, x=2, y=4, share=False, copies=2), dict(T=20, E=12, k=5, M=2100, y=3, share=False, shift=1, pad=False), dict(T=11, E=70, k=16, M=4100, dtype="f32", x=2)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join("%s%s" % i for i in c.items()))
def test_dispatch_and_combine(case):
    e = Exchange(**case)
    copies = case.get("copies", 1)
    xc, rows = e.tokens(e.tok), e.packed(torch.full_like(e.rows, KEPT), KEPT, copies)
    g.dispatch(e.mesh, [xc.buf(i) for i, _ in e.places], e.x_sh, e.k, e.r.buf, e.bufs(rows, copies), e.rows_sh, stream=stream())
    want = torch.zeros(e.T * e.k, e.M, dtype=torch.float64)
    want[:e.total] = e.tok.double()[e.order[:e.total] // e.k]
    e.check_packed(rows, want, torch.zeros_like(want), copies)
    for weighted in (True, False):
        given, y = e.packed(e.rows), e.tokens(torch.full_like(e.tok, KEPT), KEPT, copies)
        g.combine(e.mesh, e.bufs(given), e.rows_sh, e.k, e.r.buf, [y.buf(i, j % copies) for i, j in e.places], e.x_sh, weighted=weighted, stream=stream())
        there = e.slots >= 0
        picked = e.rows.double()[e.slots.clamp(min=0)] * (there * (e.weights.double() if weighted else 1.0))[:, :, None]
        want = torch.zeros(y.per * e.x, e.M, dtype=torch.float64)
        want[:e.T] = picked.sum(dim=1)
        most = torch.zeros_like(want)
        most[:e.T] = (1 + 2.0 ** -8) * (e.k + 1) * 2.0 ** -24 * picked.abs().sum(dim=1) + 2.0 ** -126      # k multiplications and additions in one rounding each
        for c in range(copies):
            assert ((y.whole(c).double() - want).abs() <= most + HALF[e.dtype] * want.abs()).all()
            assert (y.gaps(c) == KEPT).all()


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join("%s%s" % i for i in c.items()))
def test_combine_gradient(case):
    e = Exchange(**case)
    copies = case.get("copies", 1)
    dy, rows, drows = e.tokens(e.tok), e.packed(e.rows), e.packed(torch.full_like(e.rows, KEPT), KEPT, copies)
    dw = torch.full((e.T, e.k), NAN, device="cuda")
    g.combine_grad(e.mesh, [dy.buf(i) for i, _ in e.places], e.x_sh, e.bufs(rows), e.rows_sh, e.k, e.r.buf, e.bufs(drows, copies), dw.data_ptr(), stream=stream())
    want = torch.zeros(e.T * e.k, e.M, dtype=torch.float64)
    o = e.order[:e.total]
    want[:e.total] = e.tok.double()[o // e.k] * e.weights.double().flatten()[o][:, None]
    e.check_packed(drows, want, (HALF[e.dtype] * (1 + 2.0 ** -8) + 2.0 ** -24) * want.abs() + 2.0 ** -126, copies)
    picked = e.rows.double()[e.slots.clamp(min=0)] * (e.slots >= 0)[:, :, None] * e.tok.double()[:, None, :]
    assert ((dw.cpu().double() - picked.sum(dim=2)).abs() <= (e.M + 2) * 2.0 ** -24 * picked.abs().sum(dim=2) + 2.0 ** -126).all()


def test_arrays_that_make_no_sense_lead_nowhere():
    """Experts, slots and an order beyond what there is count as none."""
    e = Exchange(T=9, E=4, k=2, M=16, y=2, share=False)
    bad = torch.tensor([-5, 2 ** 31 - 1, 18, 100, -2 ** 31, 19, 64, 1000, -1], dtype=torch.int32, device="cuda").repeat(2)
    for name in ("order", "slots", "experts"):
        getattr(e.r, name).view(-1)[:18].copy_(bad)
    xc, rows, y = e.tokens(e.tok), e.packed(torch.full_like(e.rows, KEPT), KEPT), e.tokens(torch.full_like(e.tok, KEPT), KEPT)
    g.dispatch(e.mesh, [xc.buf(i) for i, _ in e.places], e.x_sh, e.k, e.r.buf, e.bufs(rows), e.rows_sh, stream=stream())
    g.combine(e.mesh, e.bufs(rows), e.rows_sh, e.k, e.r.buf, [y.buf(i) for i, _ in e.places], e.x_sh, stream=stream())
    dw = torch.full((9, 2), NAN, device="cuda")
    g.combine_grad(e.mesh, [xc.buf(i) for i, _ in e.places], e.x_sh, e.bufs(rows), e.rows_sh, e.k, e.r.buf, e.bufs(rows), dw.data_ptr(), stream=stream())
    d = Cut(torch.zeros(9, 4), 1)
    g.route_grad(e.r.mesh, e.r.z_bufs, e.r.sh, 2, e.r.buf, dw.data_ptr(), [d.buf(0)], stream=stream())
    torch.cuda.synchronize()
    assert all((c.whole() == KEPT).all() for c in rows) and (y.whole() == 0).all() and (dw == 0).all() and (d.whole() == 0).all()


@pytest.mark.parametrize("y, dtype", [(1, "bf16"), (3, "bf16"), (2, "f32")])
def test_a_layer_and_its_gradients(y, dtype):
    """Route, dispatch, two products with a Relu between, combine; then backwards: against autograd of the definition in float64 with the library's choices.  Each stage rounds to the type, so the
    result is held to a few of those roundings of its size."""
    T, E, k, M, H = 150, 7, 2, 64, 96
    r = Routed(T, E, k, masked=0.1, seed=11).stage()
    r.call()
    torch.cuda.synchronize()
    t = TYPES[dtype]
    gen = torch.Generator().manual_seed(12)
    x, w1, w2, dy = (torch.randn(*s, generator=gen).mul(a).to(t) for s, a in (((T, M), 1.0), ((E, M, H), M ** -0.5), ((E, H, M), H ** -0.5), ((T, M), 1.0)))
    mesh = g.Mesh((1, y), tuple(range(y)))
    es, S = -(-E // y), T * k
    def matrices(full):
        a = torch.zeros((y * es,) + tuple(full.shape[1:]), dtype=t, device="cuda")
        a[:E] = full.cuda()
        a = a.view((y, es) + tuple(full.shape[1:]))
        return a, [g.ShardBuf.of(a[j], a.shape[-1]) for j in range(y)]
    (w1t, w1b), (w2t, w2b) = matrices(w1), matrices(w2)
    (dw1t, dw1b), (dw2t, dw2b) = matrices(torch.zeros_like(w1)), matrices(torch.zeros_like(w2))
    def buffer(rows, cols):
        a = torch.zeros(rows, cols, dtype=t, device="cuda")
        return a, [g.ShardBuf.of(a, cols)] * y
    (xt, xb), (rows, rows_b), (mid, mid_b), (out, out_b), (yt, yb) = buffer(T, M), buffer(S, M), buffer(S, H), buffer(S, M), buffer(T, M)
    xt.copy_(x)
    x_sh, narrow, wide = g.Sharding((T, M), (0, -1)), g.Sharding((E, S, M), (1, -1, -1)), g.Sharding((E, S, H), (1, -1, -1))
    w1_sh, w2_sh, sizes, st = g.Sharding((E, M, H), (1, -1, -1)), g.Sharding((E, H, M), (1, -1, -1)), r.sizes.data_ptr(), stream()
    g.dispatch(mesh, xb, x_sh, k, r.buf, rows_b, narrow, stream=st)
    g.ragged_dot(mesh, DIMS[FORWARD], rows_b, narrow, w1b, w1_sh, mid_b, wide, sizes, stream=st, epilogue=g.EPILOGUE_RELU)
    g.ragged_dot(mesh, DIMS[FORWARD], mid_b, wide, w2b, w2_sh, out_b, narrow, sizes, stream=st)
    g.combine(mesh, out_b, narrow, k, r.buf, yb, x_sh, stream=st)
    (dyt, dyb), (dout, dout_b), (dmid, dmid_b), (drows, drows_b), (dx, dxb) = buffer(T, M), buffer(S, M), buffer(S, H), buffer(S, M), buffer(T, M)
    dyt.copy_(dy)
    dweights = torch.zeros(T, k, device="cuda")
    g.combine_grad(mesh, dyb, x_sh, out_b, narrow, k, r.buf, dout_b, dweights.data_ptr(), stream=st)
    g.ragged_dot(mesh, DIMS[WEIGHT], mid_b, wide, dout_b, narrow, dw2b, w2_sh, sizes, stream=st)
    g.ragged_dot(mesh, DIMS[BACK], dout_b, narrow, w2b, w2_sh, dmid_b, wide, sizes, stream=st)
    dmid.masked_fill_(mid <= 0, 0)
    g.ragged_dot(mesh, DIMS[WEIGHT], rows_b, narrow, dmid_b, wide, dw1b, w1_sh, sizes, stream=st)
    g.ragged_dot(mesh, DIMS[BACK], dmid_b, wide, w1b, w1_sh, drows_b, narrow, sizes, stream=st)
    g.combine(mesh, drows_b, narrow, k, r.buf, dxb, x_sh, weighted=False, stream=st)
    dz = Cut(torch.zeros(T, E), 1)
    g.route_grad(r.mesh, r.z_bufs, r.sh, k, r.buf, dweights.data_ptr(), [dz.buf(0)], stream=st)
    torch.cuda.synchronize()
    # the definition
    X, W1, W2 = x.double().requires_grad_(), w1.double().requires_grad_(), w2.double().requires_grad_()
    Z = torch.where(torch.isfinite(r.z), r.z, torch.full_like(r.z, -1e4)).double().requires_grad_()
    experts = r.experts.cpu().long()
    there = experts >= 0
    p = torch.softmax(Z, dim=1).gather(1, experts.clamp(min=0)) * there
    hidden = torch.relu(torch.einsum("tm,tkmh->tkh", X, W1[experts.clamp(min=0)]))
    Y = (torch.einsum("tkh,tkhm->tkm", hidden, W2[experts.clamp(min=0)]) * p[:, :, None]).sum(dim=1)
    (Y * dy.double()).sum().backward()
    live = there.any(dim=1)
    roundings = 6 * HALF[t] + 300 * 2.0 ** -24
    for got, want in ((yt, Y.detach()), (dx, X.grad), (dw1t.flatten(0, 1)[:E], W1.grad), (dw2t.flatten(0, 1)[:E], W2.grad), (dz.whole(), Z.grad * live[:, None])):
        got, want = got.cpu().double(), want
        assert (got - want).norm() <= roundings * want.norm(), float((got - want).norm() / want.norm())


def test_a_layer_in_a_graph():
    """Router and exchange recorded once, replayed with other logits: bits of the eager calls."""
    r = Routed(300, 20, 4, seed=13, pad=False).stage()
    M = 48
    mesh, S = r.mesh, 1200
    x, rows, y = torch.randn(300, M, device="cuda"), torch.zeros(S, M, device="cuda"), torch.zeros(300, M, device="cuda")
    bx, br, by = ([g.ShardBuf.of(a, M)] for a in (x, rows, y))
    sh, rs = g.Sharding((300, M), (0, -1)), g.Sharding((20, S, M), (-1, -1, -1))
    def run():
        r.call()
        g.dispatch(mesh, bx, sh, 4, r.buf, br, rs, stream=stream())
        g.combine(mesh, br, rs, 4, r.buf, by, sh, stream=stream())
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for turn in range(4):
        r.z = torch.randn(300, 20, generator=torch.Generator().manual_seed(turn))
        r.zc.t[0][0].copy_(r.z)
        rows.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        r.check()
        got = rows.clone(), y.clone()
        rows.zero_()
        run()
        torch.cuda.synchronize()
        assert torch.equal(got[0], rows) and torch.equal(got[1], y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [2, 3, 7, 9, 127, 129, 256, 257, 264, 511, 1023, 2049, 4103])
def test_ends_of_rows(M, dtype):
    for case in (dict(T=21, E=6, k=3, M=M, dtype=dtype, pad=False), dict(T=10, E=5, k=5, M=M, dtype=dtype, x=2, y=2, share=False, shift=1, pad=False)):
        test_dispatch_and_combine(case)
        test_combine_gradient(case)


@pytest.mark.parametrize("E, k", [(3, 3), (16, 4), (100, 8), (512, 16)])
def test_equal_logits_go_to_the_lowest(E, k):
    """Zeros of both signs are equal, as are infinities; numbers below normal are not."""
    r = Routed(70, E, k, masked=0.0, seed=21)
    gen = torch.Generator().manual_seed(22)
    values = torch.tensor([0.0, -0.0, 1e-40, -1e-40, 2e-40, -float("inf"), -3.0e38, 3.0e38])
    r.z = values[torch.randint(0, 8, (70, E), generator=gen)]
    r.stage().call()
    torch.cuda.synchronize()
    experts, _, slots, order, sizes = r.expected()
    assert torch.equal(r.experts.cpu().long(), experts) and torch.equal(r.slots.cpu().long(), slots)
    assert torch.equal(r.order.cpu().long(), order) and torch.equal(r.sizes.cpu().long(), sizes)


@pytest.mark.parametrize("normalise", [False, True])
def test_gradient_of_an_expert_twice(normalise):
    """A routing that a program made by itself may name an expert more than once: its choices' gradients add up, in their order."""
    r = Routed(40, 24, 4, masked=0.0, normalise=normalise, seed=23).stage()
    r.z[20] = 0.0
    r.stage().call()
    experts = r.experts.cpu().long()
    experts[::3, 2] = experts[::3, 0]
    experts[5, :] = experts[5, 1]
    r.experts.copy_(experts.int())
    dw = torch.randn(40, 4, generator=torch.Generator().manual_seed(24))
    d, given = Cut(torch.zeros(40, 24), 1), dw.cuda()
    outs = []
    for _ in range(2):
        g.route_grad(r.mesh, r.z_bufs, r.sh, 4, r.buf, given.data_ptr(), [d.buf(0)], normalise=normalise, stream=stream())
        outs.append(d.whole())
    assert torch.equal(outs[0], outs[1])
    # p (all experts') or nothing minus the mean of w g over the choices, and what each choice adds, from the weights that the call was given
    w = r.weights.cpu().double() * dw.double()
    mean = w.sum(dim=1, keepdim=True)
    p = torch.softmax(r.z.double(), dim=1)
    want = torch.zeros(40, 24, dtype=torch.float64) if normalise else -p * mean
    want.scatter_add_(1, experts, w - r.weights.cpu().double() * mean if normalise else w)
    mag = (p + 1) * (w.abs().sum(dim=1, keepdim=True) + (r.weights.cpu().double().sum(dim=1, keepdim=True) + 1) * mean.abs())
    assert ((d.whole().double() - want).abs() <= (24 + 80) * 2.0 ** -23 * mag).all()


def test_the_same_through_ctypes(monkeypatch):
    from paper_2105_04663_amd import binding
    monkeypatch.setattr(binding, "_CALL", None)
    test_a_layer_and_its_gradients(3, "bf16")
    test_route_gradient(True, "f32", 70, 100, 2, 3, 1)
    e = Embed(150, 56, 37, x=2, y=3, copies=2, accumulate=True).stage_lookup().stage_gradient()
    e.lookup()
    e.check_lookup()
    e.gradient()
    e.check_gradient()


@pytest.mark.parametrize("T, x", [(70, 8), (70, 9), (300, 64), (10, 64)])
def test_route_over_many_shards(T, x):
    """Tables of few shards and of many; shards that lie behind the last token."""
    r = Routed(T, 40, 3, x=x, seed=25).stage()
    r.call()
    r.check()
    dw = torch.randn(T, 3, generator=torch.Generator().manual_seed(26))
    d, given = Cut(torch.full((T, 40), KEPT), x, fill=KEPT), dw.cuda()
    g.route_grad(r.mesh, r.z_bufs, r.sh, 3, r.buf, given.data_ptr(), [d.buf(i) for i, _ in r.places], stream=stream())
    r.check_gradient(dw, d)
