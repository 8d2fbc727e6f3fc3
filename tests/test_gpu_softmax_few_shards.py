"""At most 16 tokens of a small vocabulary matrix, whose shards with their padding are more than the 16 rows of a workgroup."""
import pytest

from tests.losses import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,M,V,mesh", [(16, 24, 40, (3, 1)), (16, 130, 90, (3, 4)), (10, 64, 90, (9, 1)), (13, 9, 300, (6, 2)), (16, 24, 77, (15, 2))])
def test_dw_of_tokens_with_padding_beyond_a_workgroup(T, M, V, mesh, dtype, vocab_dim):
    for grad in ((True, True), (False, True)):
        Problem(T, M, V, dtype, vocab_dim=vocab_dim, mesh=mesh, K=3 if T == 13 else None).stage(grad).call().check()
