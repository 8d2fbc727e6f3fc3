"""Losses whose tokens lie in more shards than a launch has room for (64): several launches for one piece, with and without x's second copy."""
import pytest

from tests.losses import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("T,mesh", [(64, (64, 1)), (66, (66, 1)), (100, (100, 1)), (128, (128, 2)), (150, (75, 1)), (300, (100, 1))])
def test_tokens_in_more_shards_than_a_table_has(T, mesh, vocab_dim):
    for dtype, K, M in (("bf16", None, 24), ("bf16", 3, 130), ("f32", None, 24)):
        p = Problem(T, M, 90, dtype, K=K, vocab_dim=vocab_dim, mesh=mesh, pad=M != 130).stage()
        print(T, mesh, dtype, flush=True)
        p.call().check()
        p.call(p.least + (p.bytes - p.least) // 2).check()             # in pieces
        Problem(T, M, 90, dtype, K=K, vocab_dim=vocab_dim, mesh=mesh).stage((False, True)).call().check()
        Problem(T, M, 90, dtype, K=K, vocab_dim=vocab_dim, mesh=mesh).stage((False, False)).call().check()
