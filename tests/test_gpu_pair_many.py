"""dot_pair_kernel (pinned) on several problems of short K, in rows of whole lines and not: outputs past the caches and through them.  Small integers, compared exactly."""
import numpy as np
import pytest
import torch

import paper_2105_04663_amd as g
from tests.pin import PAIR, last, pinned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E", [1, 2, 3, 8])
@pytest.mark.parametrize("K", [40, 96, 97, 192, 193])
@pytest.mark.parametrize("N,ld", [(520, 520), (521, 523), (512, 576)])
def test_products(E, K, N, ld):
    M, up = 300, lambda n: -(-n // 8) * 8
    gen = torch.Generator().manual_seed(E * 1000 + K)
    a, b = (torch.randint(-2, 3, (E, K, n), generator=gen).double() for n in (M, N))
    lhs, rhs = (torch.zeros((E, K, up(t.shape[2])), dtype=torch.bfloat16, device="cuda") for t in (a, b))
    lhs[:, :, :M], rhs[:, :, :N] = a.cuda(), b.cuda()
    out = torch.full((E, M, ld), float("nan"), dtype=torch.bfloat16, device="cuda")
    mesh, dims, whole = g.Mesh((1,), (0,)), g.DotDims((0,), (0,), (1,), (1,)), (-1, -1, -1)
    shs = [g.Sharding(s, whole) for s in ((E, K, M), (E, K, N), (E, M, N))]
    n = g.dot_workspace_bytes(mesh, dims, *shs, -1)
    space = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    with pinned(PAIR):
        g.local_dot(mesh, dims, g.ShardBuf.of(lhs, up(M)), shs[0], g.ShardBuf.of(rhs, up(N)), shs[1], g.ShardBuf.of(out, ld), shs[2], 0, None, -(-space.data_ptr() // 256) * 256, n,
                    torch.cuda.current_stream().cuda_stream)
        assert last() == (PAIR, 0, 0)
    torch.cuda.synchronize()
    want = torch.matmul(a.transpose(1, 2).contiguous(), b).to(torch.bfloat16)
    assert torch.equal(out[:, :, :N].cpu(), want)
    assert np.isnan(out[:, :, N:].float().cpu().numpy()).all()
