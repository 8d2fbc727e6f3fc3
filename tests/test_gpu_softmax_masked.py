"""Entries that the vocabulary matrix itself masks: -infinity where x is positive.  Their logits are -infinity, wherever in a row of w it stands, and nobody else's."""
import numpy as np
import pytest

from tests.losses import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("T,M,V", [(1, 13, 3000), (4, 515, 600), (8, 77, 3001), (20, 77, 100), (40, 77, 3000), (300, 515, 600)])
def test_an_entry_of_minus_infinity(T, M, V, vocab_dim, dtype):
    for at in sorted({0, 1, M // 2} | set(range(M - 9, M))):
        p = Problem(T, M, V, dtype, vocab_dim=vocab_dim, pad=False, missing=0.0)
        p.ids[:] = 1                                      # (a label on another entry)
        p.xt = p.xt.abs() + 1
        p.x = p.xt.double().numpy()
        p.wt[5, at] = -np.inf
        got = p.stage((False, False)).call().results()
        # the same without the entry, held to the bounds of such a problem
        z = p.x @ np.delete(p.w, 5, axis=0).T
        top = z.max(axis=1)
        lse = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
        off = 2 * (M + 2) * 2.0 ** -24 * (np.abs(p.x) @ np.abs(p.w).T).max(axis=1) + 24 * 2.0 ** -24 * (np.abs(z).max(axis=1) + 1) + 2.0 ** -18
        assert (np.abs(got["lse"] - lse) <= off).all(), (at, np.abs(got["lse"] - lse).max())
        assert (np.abs(got["loss"] - (lse - p.x @ p.w[1])) <= 2 * off).all(), at
