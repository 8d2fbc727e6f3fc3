"""Padding of dw is zeros, also where a token's activations are not finite (and its dw is NaN)."""
import numpy as np
import pytest

from tests.losses import Problem

pytestmark = pytest.mark.gpu


# T: a handful and more; shards with fewer entries than their places and without any, in one launch (small) and not; M of whole vectors and not
@pytest.mark.parametrize("T", [1, 3, 4, 8, 20, 200])
@pytest.mark.parametrize("M,V,mesh", [(64, 3001, (1, 4)), (515, 301, (1, 8)), (24, 9, (1, 4)), (130, 1003, (2, 3)), (40, 20001, (1, 2))])
@pytest.mark.parametrize("dtype,vocab_dim", [("bf16", 0), ("bf16", 1), ("f32", 0), ("f32", 1)])
def test_padding_of_dw_beside_a_token_that_is_not_finite(T, M, V, mesh, dtype, vocab_dim):
    p = Problem(T, M, V, dtype, vocab_dim=vocab_dim, mesh=mesh, missing=0.0)
    p.xt[T // 2, 1] = float("nan")
    for grad in ((False, True), (True, True)):
        got = p.stage(grad).call().results()              # (reads the padding)
        assert np.isnan(got["loss"][T // 2]) and np.isnan(got["dw"]).all()
