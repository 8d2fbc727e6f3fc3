"""Rows of 2^24 tokens from a vocabulary matrix [M, V]: 2^32 threads and more, compared on the GPU with torch's own indexing."""
import pytest
import torch

import paper_2105_04663_amd as g
from tests.tokens import KEPT, stream

pytestmark = pytest.mark.gpu
ONE = g.Mesh((1,), (0,))


@pytest.fixture(autouse=True)
def give_back():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M", [2048 - 256, 2048, 2048 + 32])
def test_rows_of_as_many_tokens_as_there_may_be(M):
    """Seven, eight and nine times eight blocks of columns: 7/8 of 2^32 threads, as many, more."""
    T, V = 1 << 24, 29
    gen = torch.Generator(device="cuda").manual_seed(M)
    w = torch.randint(-2 ** 14, 2 ** 14, (M, V), dtype=torch.int16, generator=gen, device="cuda").view(torch.bfloat16)
    ids = torch.randint(-1, V + 1, (T,), dtype=torch.int32, generator=gen, device="cuda")
    y = torch.full((T, M), KEPT, dtype=torch.bfloat16, device="cuda")
    g.embed(ONE, [ids.data_ptr()], [g.ShardBuf.of(w, V)], g.Sharding((M, V), (-1, -1)), [g.ShardBuf.of(y, M)], g.Sharding((T, M), (-1, -1)), vocab_dim=1, stream=stream())
    rows = torch.cat([w.t().contiguous(), torch.zeros(1, M, dtype=torch.bfloat16, device="cuda")])        # the last: no entry
    at = torch.where((ids >= 0) & (ids < V), ids, torch.full_like(ids, V)).long()
    for a in range(0, T, 1 << 20):
        assert torch.equal(y[a:a + (1 << 20)].view(torch.int16), rows[at[a:a + (1 << 20)]].view(torch.int16)), a
