"""Equal calls give equal bits on every path of the losses."""
import pytest
import torch

from tests.losses import Problem

pytestmark = pytest.mark.gpu


def calls(p, n):
    outputs = [b[1] for b in (p.dxs or []) + (p.dws or [])] + [t[1][name] for t in p.ts for name in ("loss", "lse")]
    first = None
    for turn in range(n):
        for o in outputs:
            o.fill_(float(turn))
        p.space.fill_(turn) if getattr(p, "space", None) is not None else None
        p.call()
        torch.cuda.synchronize()
        here = [o.nan_to_num(7.0) for o in outputs]
        gaps = [o != float(turn) for o in here]                # (row gaps are not written)
        if first is None:
            first, there = [o.clone() for o in here], [g.clone() for g in gaps]
            continue
        for a, b, g, h in zip(first, here, gaps, there):
            assert torch.equal(a[g & h], b[g & h])


# [M, V] of one launch: shards that end one to three columns into a group of 64, with sums that the groups' waves begin at other places
@pytest.mark.parametrize("T,M,V,mesh", [(5, 900, 65, (1, 1)), (40, 900, 65, (1, 1)), (16, 300, 195, (1, 3)), (33, 500, 129, (1, 1)), (16, 96, 322, (1, 1)), (9, 500, 131, (1, 1)), (200, 300, 195, (2, 3))])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_small_vocabulary_matrix(T, M, V, mesh, dtype):
    M = M if dtype == "bf16" else M // 2                       # of up to 128 KiB
    for vocab_dim in (1, 0):
        for grad in ((True, True), (False, False)):
            p = Problem(T, M, V, dtype, vocab_dim=vocab_dim, mesh=mesh).stage(grad)
            p.call().check()
            calls(p, 12)


@pytest.mark.parametrize("T,M,V,kw,grad", [(3, 64, 2000, {}, True), (5, 300, 1003, dict(dtype="f32", vocab_dim=1, mesh=(1, 3)), True), (100, 130, 2003, dict(mesh=(2, 2), vocab_dim=1, pad=False, K=5), True),
                                           (700, 512, 30001, dict(mesh=(2, 1)), False), (2100, 300, 400, dict(mesh=(2, 3)), True), (66, 40, 2000, dict(mesh=(66, 1)), True)])
def test_other_paths(T, M, V, kw, grad):
    calls(Problem(T, M, V, **kw).stage((grad, grad)), 6)
