"""gspmd_route_grad where logits, weights or their gradients are not finite: what has no part in a token's softmax has a gradient of zero."""
import pytest
import torch

import paper_2105_04663_amd as g
from tests.tokens import HALF, KEPT, NAN, Cut, Routed, stream

pytestmark = pytest.mark.gpu
INF = float("inf")


def gradient(r, dweights):
    d, given = Cut(torch.full((r.T, r.E), KEPT, dtype=r.dtype), r.x, fill=KEPT), dweights.cuda()
    g.route_grad(r.mesh, r.z_bufs, r.sh, r.k, r.buf, given.data_ptr(), [d.buf(i) for i, _ in r.places], normalise=r.normalise, stream=stream())
    out = d.whole()
    assert (out[r.T:] == 0).all() and (d.gaps() == KEPT).all()
    return out[:r.T].double()


def check_ordinary(r, rows, got, dw):
    """The definition in float64 of tokens `rows`, whose logits are finite or -infinity, as Routed.check_gradient bounds it."""
    z, experts = r.z.double()[rows], r.experts.cpu().long()[rows]
    there, at = experts >= 0, experts.clamp(min=0)
    p = torch.exp(z - z.amax(dim=1, keepdim=True))
    if r.normalise:
        p = p * torch.zeros_like(p).scatter_add_(1, at, there.double())
    p = p / p.sum(dim=1, keepdim=True)
    gr = torch.zeros_like(p).scatter_add_(1, at, dw.double()[rows] * there)
    mean, mag = (p * gr).sum(dim=1, keepdim=True), (p * gr.abs()).sum(dim=1, keepdim=True)
    want = p * (gr - mean)
    assert ((got[rows] - want).abs() <= (r.E + 80) * 2.0 ** -23 * p * (gr.abs() + mag) + HALF[r.dtype] * want.abs() + 2.0 ** -126).all()


@pytest.mark.parametrize("normalise", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E, k, x", [(1, 1, 1), (7, 3, 2), (16, 4, 1), (64, 8, 3), (200, 5, 1), (512, 16, 1)])
def test_a_token_without_experts_has_no_gradient(normalise, dtype, E, k, x):
    """Logits all NaN; NaN and -infinity; all -infinity; NaN, of a token whose experts the program took away; beside tokens with a NaN that have experts, and ordinary ones."""
    T = 23
    r = Routed(T, E, k, x=x, dtype=dtype, normalise=normalise, masked=0.0, seed=31)
    r.z[T // 2] = 1.0
    r.z[1] = NAN
    r.z[4], r.z[4, ::2] = -INF, NAN
    r.z[9] = -INF
    r.z[12, 0] = r.z[13, E // 2] = NAN
    r.stage().call()
    r.experts[12] = -1
    r.weights[12], r.weights[15] = 0, 0
    r.experts[15] = -1
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(E))
    got = gradient(r, torch.where(r.experts.cpu() >= 0, dw, torch.full_like(dw, NAN)))
    assert (got[[1, 4, 9, 12, 15]] == 0).all()
    if E == 1:
        assert (got[13] == 0).all()                                     # its one logit is NaN
    elif normalise:
        r.z[13, E // 2] = -INF                                          # the same as if it were masked
        check_ordinary(r, torch.tensor([13]), got, dw)
    else:
        assert got[13].isnan().all()
    check_ordinary(r, torch.tensor([i for i in range(T) if i not in (1, 4, 9, 12, 13, 15)]), got, dw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E, k, x", [(7, 3, 2), (16, 4, 1), (40, 2, 1), (64, 8, 3), (200, 5, 1), (512, 15, 1)])
def test_experts_outside_the_softmax_have_no_gradient(dtype, E, k, x):
    """Weights over the chosen experts: a NaN or an infinity among a token's weights or their gradients stays with those experts."""
    T = 19
    r = Routed(T, E, k, x=x, dtype=dtype, normalise=True, masked=0.0, seed=32)
    r.z[T // 2] = 1.0
    r.z[2, E // 2], r.z[5, 0], r.z[5, E - 1] = INF, INF, INF
    r.stage().call()
    experts = r.experts.cpu().long()
    assert r.weights.cpu()[[2, 5]].isnan().any(dim=1).all()
    dw = torch.randn(T, k, generator=torch.Generator().manual_seed(E))
    dw[7, 0], dw[8, k - 1], dw[11, k // 2] = INF, NAN, -INF
    got = gradient(r, dw)
    strange = [2, 5, 7, 8, 11]
    chosen = torch.zeros(T, E, dtype=torch.bool).scatter_(1, experts, True)
    assert (got[~chosen] == 0).all()
    for t in strange:
        assert not got[t][chosen[t]].isfinite().all()
    check_ordinary(r, torch.tensor([i for i in range(T) if i not in strange]), got, dw)
