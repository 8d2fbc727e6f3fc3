"""The exchange between tokens and experts where its indexes make no sense, each kind by itself, and on the mesh dimension that splits both."""
import pytest
import torch

import paper_2105_04663_amd as g
from tests.test_gpu_route import Exchange
from tests.tokens import HALF, KEPT, NAN, Cut, Routed, stream

pytestmark = pytest.mark.gpu
STRANGE = [-5, 2 ** 31 - 1, -2 ** 31, -1, 100000, 2 ** 24, 2 ** 30]


def run(e):
    """dispatch, combine (both ways) and combine_grad, by e's arrays on the GPU, against the definition by them: what is no slot, or no expert, is none."""
    places, r, T, k, M = e.places, e.r, e.T, e.k, e.M
    experts, slots, weights = r.experts[:T].cpu().long(), r.slots[:T].cpu().long(), r.weights[:T].cpu().double()
    there = (slots >= 0) & (slots < T * k)
    if not e.share:
        there &= (experts >= 0) & (experts < e.E)
    at, owner = torch.where(there, slots, torch.zeros_like(slots)), torch.where(there, experts, torch.zeros_like(experts)) // e.es
    def expected(per_choice, j):
        """The packed rows of expert shard j: a choice's row in its slot, all else as it was."""
        want = torch.full((T * k, M), KEPT, dtype=torch.float64)
        mine = there if e.share else there & (owner == j)
        want[at[mine]] = per_choice[mine]
        return want
    x = e.tok.double()
    xc, packed = e.tokens(e.tok), e.packed(torch.full_like(e.rows, KEPT), KEPT)
    bufs = [xc.buf(i) for i, _ in places]
    g.dispatch(e.mesh, bufs, e.x_sh, k, r.buf, e.bufs(packed), e.rows_sh, stream=stream())
    for j, cut in enumerate(packed):
        assert torch.equal(cut.whole().double(), expected(x[:, None, :].expand(T, k, M), j)) and (cut.gaps() == KEPT).all()
    given = [Cut(e.rows, 1, pad=e.pad, shift=e.shift) for _ in packed]                # each shard's buffer whole: what is read shows
    picked = e.rows.double()[at] * there[:, :, None]
    for weighted in (True, False):
        y = e.tokens(torch.full_like(e.tok, KEPT), KEPT)
        g.combine(e.mesh, e.bufs(given), e.rows_sh, k, r.buf, [y.buf(i) for i, _ in places], e.x_sh, weighted=weighted, stream=stream())
        parts = picked * torch.where(there, weights, torch.zeros_like(weights))[:, :, None] if weighted else picked
        want = torch.zeros(y.per * e.x, M, dtype=torch.float64)
        most = torch.zeros_like(want)
        want[:T], most[:T] = parts.sum(dim=1), (1 + 2.0 ** -8) * (k + 1) * 2.0 ** -24 * parts.abs().sum(dim=1) + 2.0 ** -126
        assert ((y.whole().double() - want).abs() <= most + HALF[e.dtype] * want.abs()).all() and (y.gaps() == KEPT).all()
    drows, dw = e.packed(torch.full_like(e.rows, KEPT), KEPT), torch.full((T, k), NAN, device="cuda")
    g.combine_grad(e.mesh, bufs, e.x_sh, e.bufs(given), e.rows_sh, k, r.buf, e.bufs(drows), dw.data_ptr(), stream=stream())
    shares = x[:, None, :] * torch.where(there, weights, torch.zeros_like(weights))[:, :, None]
    for j, cut in enumerate(drows):
        want = expected(shares, j)
        assert ((cut.whole().double() - want).abs() <= (HALF[e.dtype] * (1 + 2.0 ** -8) + 2.0 ** -24) * want.abs() + 2.0 ** -126).all() and (cut.gaps() == KEPT).all()
    products = picked * x[:, None, :]
    assert ((dw.cpu().double() - products.sum(dim=2)).abs() <= (M + 2) * 2.0 ** -24 * products.abs().sum(dim=2) + 2.0 ** -126).all()


SHAPES = [dict(T=9, E=4, k=2, M=16, y=2, share=False), dict(T=31, E=7, k=3, M=515, x=2, y=3, share=False, pad=False), dict(T=20, E=12, k=5, M=2100, y=4, share=False, shift=1, pad=False),
          dict(T=14, E=70, k=16, M=600, dtype="f32", y=2, share=False), dict(T=25, E=6, k=2, M=300, y=3), dict(T=40, E=5, k=4, M=3, x=3, y=2, share=False)]


@pytest.mark.parametrize("what", ["experts", "slots", "both, here and there"])
@pytest.mark.parametrize("case", SHAPES, ids=lambda c: "-".join("%s%s" % i for i in c.items()))
def test_strange_experts_and_slots(case, what):
    """All experts strange and the slots as they were; the other way round; some of each among choices that go where they belong."""
    e = Exchange(**case)
    n, gen = e.T * e.k, torch.Generator().manual_seed(e.M)
    strange = torch.tensor(STRANGE + [e.E, n])[torch.arange(n) % (len(STRANGE) + 2)]
    strange[strange < e.E] = -7                                             # (E and T k are strange for one of the two each)
    bad = {"experts": strange, "slots": torch.where(strange < n, torch.full_like(strange, -1), strange)}
    for name in ("experts", "slots"):
        if what in (name, "both, here and there"):
            array = getattr(e.r, name)
            take = torch.rand(n, generator=gen) < (0.3 if what != name else 2.0)
            array.view(-1)[:n].copy_(torch.where(take, bad[name], array.view(-1)[:n].cpu().long()).int())
    run(e)


class OneDimension(Exchange):
    """Tokens and experts split along the same mesh dimension: partition i has the i-th shard of both."""

    def __init__(self, n, copies=1, **kw):
        super().__init__(x=1, y=n, share=False, **kw)
        self.x, self.mesh = n, g.Mesh((copies, n), tuple(range(copies * n)))
        self.places = [(i, i) for _ in range(copies) for i in range(n)]
        self.x_sh, self.rows_sh = g.Sharding((self.T, self.M), (1, -1)), g.Sharding((self.E, self.T * self.k, self.M), (1, -1, -1))

    def bufs(self, packed, copies=1):
        return [packed[j].buf(0) for _, j in self.places]


@pytest.mark.parametrize("n, copies, case", [(2, 1, dict(T=10, E=4, k=2, M=64)), (4, 2, dict(T=33, E=10, k=4, M=515, pad=False)), (3, 1, dict(T=130, E=40, k=8, M=72)), (5, 1, dict(T=3, E=2, k=1, M=2049, shift=1, pad=False)),
                                             (64, 1, dict(T=100, E=64, k=6, M=24, dtype="f32"))], ids=lambda v: str(v) if isinstance(v, int) else "-".join("%s%s" % i for i in v.items()))
def test_tokens_and_experts_on_one_mesh_dimension(n, copies, case):
    run(OneDimension(n, copies, **case))


@pytest.mark.parametrize("T", [32768, 32769, 65536, 65537])
@pytest.mark.parametrize("E, k", [(5, 2), (130, 1)])
def test_routes_of_many_tiles(T, E, k):
    """Tiles of 64 tokens: 512 of them, whose counts every workgroup adds up itself, and 513; 1024, which a workgroup of route_sums_kernel takes in one round, and 1025."""
    r = Routed(T, E, k, ties=True, masked=0.2, seed=41).stage()
    r.call()
    r.check()
